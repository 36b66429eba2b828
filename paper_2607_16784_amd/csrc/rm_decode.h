// rm_decode.h -- definitions shared by the kernels of a served model's layer
// (norm.hip, linear.hip, cache.hip, attend.hip; headnorm.hip, prompt.hip, f8.hip).  Not part of the C ABI.
#pragma once

#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "roomie.h"

namespace rm {

// Keeps a HIP error's name for rm_status_string (api.hip); RM_ELAUNCH.
int launch_failed(hipError_t e);

typedef __bf16 bf16;
typedef _Float16 f16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Vec;
template <> struct Vec<bf16> { typedef bf16x8 x8; typedef bf16x2 x2; };
template <> struct Vec<f16> { typedef f16x8 x8; typedef f16x2 x2; };

// Eight elements by one 16-byte access at any alignment of an element: global
// accesses of gfx950 need no more, so rows of odd length keep wide accesses.
template <typename T>
__device__ inline typename Vec<T>::x8 load8(const T* p)
{
    typedef typename Vec<T>::x8 V __attribute__((aligned(2)));
    return *reinterpret_cast<const V*>(p);
}

template <typename T>
__device__ inline void store8(T* p, typename Vec<T>::x8 v)
{
    typedef typename Vec<T>::x8 V __attribute__((aligned(2)));
    *reinterpret_cast<V*>(p) = v;
}

// The first n (may be <= 0) of eight elements, zeros behind them.
template <typename T>
__device__ inline typename Vec<T>::x8 load_some(const T* p, int64_t n)
{
    if (n >= 8) return load8(p);
    typename Vec<T>::x8 v = {};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) v[i] = p[i];
    return v;
}

template <typename T>
__device__ inline void store_some(T* p, typename Vec<T>::x8 v, int64_t n)
{
    if (n >= 8) {
        store8(p, v);
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) p[i] = v[i];
}

template <int CTRL>
__device__ inline float dpp_float(float v)
{
    const int b = __builtin_bit_cast(int, v);
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(b, b, CTRL, 0xF, 0xF, false));
}

struct Add { __device__ static float of(float a, float b) { return a + b; } };
struct Max { __device__ static float of(float a, float b) { return fmaxf(a, b); } };
// the larger, or NaN where either is one
struct MaxNan {
    __device__ static float of(float a, float b) { return a > b || a != a ? a : b; }
};

// Reduction over the four 16-lane rows of a wave, lane by lane: every lane
// gets the result of its column.  Two swaps of rows between registers.
template <class Op>
__device__ inline float rows_reduce(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    // named first: __builtin_bit_cast of a vector's element reads element 0
    const uint32_t h0 = h[0], h1 = h[1];
    const float w = Op::of(__builtin_bit_cast(float, h0), __builtin_bit_cast(float, h1));
    const uint32_t c = __builtin_bit_cast(uint32_t, w);
    const auto r = __builtin_amdgcn_permlane16_swap(c, c, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return Op::of(__builtin_bit_cast(float, r0), __builtin_bit_cast(float, r1));
}

// Reduction over the wave; every lane gets the result (a fixed tree).
template <class Op>
__device__ inline float wave_reduce(float v)
{
    v = Op::of(v, dpp_float<0xB1>(v));     // lanes 1 apart
    v = Op::of(v, dpp_float<0x4E>(v));     // 2 apart
    v = Op::of(v, dpp_float<0x141>(v));    // half rows mirrored
    v = Op::of(v, dpp_float<0x140>(v));    // rows mirrored
    return rows_reduce<Op>(v);
}

constexpr int kComputeUnits = 256;   // of an MI355X

// Records a launch for rm_trace_begin / rm_trace_end (decode_api.hip); nothing
// outside a recording.
void note_launch(const void* kernel, int64_t blocks, unsigned threads, size_t dynamic_lds);

// Events that take the start and end of the next launch on s in a recording
// with times; null outside one.
hipError_t launch_events(hipStream_t s, hipEvent_t& begin, hipEvent_t& end);

// A dispatch holds fewer than 2^32 work-items.
constexpr int64_t most_blocks(unsigned threads) { return 0xffffffffll / threads; }

// Launches `kernel` and records its shape.
template <typename... P, typename... A>
inline hipError_t launch(void (*kernel)(P...), dim3 grid, unsigned threads, size_t lds,
                         hipStream_t s, A... args)
{
    if (grid.x > most_blocks(threads)) return hipErrorInvalidConfiguration;
    hipEvent_t begin, end;
    hipError_t e = launch_events(s, begin, end);
    if (e != hipSuccess) return e;
    if (begin) hipExtLaunchKernelGGL(kernel, grid, dim3(threads), lds, s, begin, end, 0, args...);
    else hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, s, args...);
    e = hipGetLastError();
    if (e == hipSuccess)
        note_launch(reinterpret_cast<const void*>(kernel),
                    (int64_t)grid.x * grid.y * grid.z, threads, lds);
    return e;
}

// Sequence b of a call: its new tokens' first row and number, its length;
// n = 0 where the sequence is out of range.
struct Sequence {
    int32_t first, n, length;
    bool bad;
};

__device__ inline Sequence sequence_of(const rm_sequences& s, int32_t page_tokens, int32_t b)
{
    Sequence q;
    q.first = s.token_offsets ? s.token_offsets[b] : b;
    const int64_t n = s.token_offsets ? (int64_t)s.token_offsets[b + 1] - q.first : 1;
    q.length = s.lengths[b];
    // One token a sequence without token_offsets: an empty sequence has none.
    q.bad = q.first < 0 || n < 0 || n > s.max_tokens || q.first + n > s.n_tokens ||
            q.length < 0 || (int64_t)q.length > (int64_t)s.table_stride * page_tokens ||
            (s.token_offsets && n > q.length);
    q.n = q.bad ? 0 : (int32_t)(n < q.length ? n : q.length);
    if (q.bad) q.length = 0;
    return q;
}

// The most workgroups that an attention or an append is laid out in; beyond
// most_blocks they come in several launches.
constexpr int64_t kMostBlocks = 0x7fffffff;

// New tokens that a sequence is laid out for; 1 at least, so that every sequence
// has a workgroup that reports one out of range.  Not bounded by n_tokens: a
// workspace stays right for calls of fewer tokens.
inline int64_t most_tokens(const rm_sequences& s) { return s.max_tokens > 1 ? s.max_tokens : 1; }

struct NormArgs {
    int32_t rows, width, gate_width;
    const void *x, *y, *gate, *post_weight, *pre_weight, *pre_bias;
    int64_t x_stride, y_stride, gate_stride;
    float alpha, eps;
    void *x_out, *n_out;
};
hipError_t launch_norm(int type, int kind, const NormArgs& a, hipStream_t s);

struct LinearArgs {
    int32_t rows, n, k, group;
    const void* x;
    const uint8_t* codes;
    const void* scales;
    const uint8_t* zeros;
    const void* bias;
    void *y, *workspace;
    uint32_t inverse;             // 2^32 / (group / 32), rounded up; 0 for 32
    int64_t x_stride, code_stride, y_stride;
};
// Workspace bytes of launch_linear; 0 where it needs none.
size_t linear_workspace(int32_t rows, int32_t n, int32_t k, int act);
hipError_t launch_linear(int type, int act, const LinearArgs& a, hipStream_t s);

struct AppendArgs {
    rm_cache cache;
    rm_sequences seqs;
    int32_t heads, rot, layout;
    const void *q, *k, *v;
    int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head;
    const int32_t* positions;
    const float* inv_freq;
    float rot_scale;
    void* q_out;
    int32_t* status;
};
bool append_fits(const rm_cache& c, const rm_sequences& s, int32_t heads);
hipError_t launch_append(int type, const AppendArgs& a, hipStream_t s);
hipError_t launch_cache_read(int type, const rm_cache& c, int32_t n, const int32_t* pages,
                             void* k, void* v, int32_t* status, hipStream_t s);

struct AttendArgs {
    rm_cache cache;
    rm_sequences seqs;
    int32_t heads, window;
    const void* q;
    int64_t q_stride, q_head;
    float scale;
    void *out, *workspace;
    int32_t* status;
};
bool attend_fits(const rm_cache& c, const rm_sequences& s, int32_t heads);
size_t attend_workspace(const rm_cache& c, const rm_sequences& s, int32_t heads);
hipError_t launch_attend(int type, const AttendArgs& a, hipStream_t s);

struct HeadNormArgs {
    int32_t n_tokens, heads, kv_heads, head_dim, rot, layout;
    const void *q, *k;
    int64_t q_stride, q_head, k_stride, k_head;
    const void *q_weight, *k_weight;
    const int32_t* positions;
    const float* inv_freq;
    float rot_scale, eps;
    void *q_out, *k_out;
    int64_t q_out_stride, q_out_head, k_out_stride, k_out_head;
};
hipError_t launch_head_norm(int type, const HeadNormArgs& a, hipStream_t s);

struct PromptArgs {
    int32_t n_tokens, heads, kv_heads, n_seqs, max_tokens, window;
    const void *q, *k, *v;
    int64_t q_stride, q_head, k_stride, k_head, v_stride, v_head;
    const int32_t* offsets;
    float scale;
    void* out;
    int32_t* status;
};
constexpr float kLog2e = 1.44269504088896340736f;
// Whether the workgroups of a call can be counted in 31 bits.
bool prompt_fits(const PromptArgs& a);
hipError_t launch_prompt(int type, int head_dim, const PromptArgs& a, hipStream_t s);

struct QuantizeArgs {
    int32_t rows, k;
    const void* x;
    int64_t x_stride;
    uint8_t* codes;
    int64_t code_stride;
    float* scales;
};
hipError_t launch_quantize(int type, int block_rows, const QuantizeArgs& a, hipStream_t s);

struct F8Args {
    int32_t rows, n, k, act;
    const void* x;
    int64_t x_stride;
    const float* x_scales;
    const uint8_t* codes;
    int64_t code_stride;
    const float* scales;
    const void *bias;
    void *y;
    int64_t y_stride;
    void* workspace;
};
// Workspace bytes of launch_f8; 0 where it needs none.
size_t f8_workspace(int32_t rows, int32_t n, int32_t k, int32_t act);
hipError_t launch_f8(int type, const F8Args& a, hipStream_t s);

}  // namespace rm
