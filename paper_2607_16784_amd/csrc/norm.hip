// norm.hip -- the gated, scaled residual between two blocks with the norms
// around it (rm_norm_residual).
//
// One pass: a row stays in registers between its reads and its writes, so each
// input is read once and each output written once; the kernel is bound by that
// traffic.  A thread holds 8 neighbouring elements a chunk (16-byte accesses).
// Rows of up to 1024 elements take a wave each and need no barrier, wider ones a
// workgroup, the widest striding over the rows with the gains in registers.
//
// Statistics are fp32 sums over a fixed tree; the variance is the mean square
// of the differences from the mean (a second sum over registers), which
// cancels nothing.
#include "rm_decode.h"

namespace rm {
namespace {

// Sum over the row's threads: the wave's, then the waves' through LDS.  Two
// buffers in turn, so one barrier a sum is enough.
template <bool WAVE>
__device__ inline float row_sum(float v, float (*part)[16], int& turn)
{
    v = wave_reduce<Add>(v);
    if (WAVE) return v;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    if ((threadIdx.x & 63) == 0) part[turn][wave] = v;
    __syncthreads();
    float s = part[turn][0];
    for (int w = 1; w < waves; ++w) s += part[turn][w];
    turn ^= 1;
    return s;
}

// v[] (zeros outside the row) normalised in place.
template <int KIND, int C, bool WAVE>
__device__ inline void normalise(float (&v)[C][8], int32_t width, int first, int step, float eps,
                                 float (*part)[16], int& turn)
{
    if (KIND == RM_NORM_LAYER) {
        float s = 0;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[c][i];
        const float mean = row_sum<WAVE>(s, part, turn) / (float)width;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                v[c][i] = first + c * step + i < width ? v[c][i] - mean : 0.0f;
    }
    float s = 0;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) s = __builtin_fmaf(v[c][i], v[c][i], s);
    const float r = 1.0f / sqrtf(row_sum<WAVE>(s, part, turn) / (float)width + eps);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[c][i] *= r;
}

// The 8 elements from `at` on of a row.  TAIL: the row may end inside them, what
// is behind is 0.  Else the row is of whole eights, and a thread behind its end
// reads the last ones again: a load under no condition can stay in flight.
template <bool TAIL, typename T>
__device__ inline typename Vec<T>::x8 row_load(const T* row, int at, int width)
{
    return TAIL ? load_some(row + at, width - at) : load8(row + min(at, width - 8));
}

template <bool TAIL, typename T>
__device__ inline void row_store(T* row, int at, int width, typename Vec<T>::x8 v)
{
    if (TAIL) store_some(row + at, v, width - at);
    else if (at < width) store8(row + at, v);
}

// C chunks a thread; THREADS a row, 64 (a wave, four rows a workgroup) or the
// whole workgroup.
template <typename T, int KIND, int C, int THREADS, bool TAIL>
__global__ __launch_bounds__(THREADS < 256 ? 256 : THREADS) void norm_kernel(NormArgs a)
{
    constexpr bool WAVE = THREADS == 64, KEEP = C <= 2;      // gains in registers
    typedef typename Vec<T>::x8 V;
    __shared__ float part[2][16];
    int turn = 0;
    const int64_t rows_here = WAVE ? 4 : 1;
    const int first = (threadIdx.x % THREADS) * 8;
    constexpr int step = THREADS * 8;
    const T* post = static_cast<const T*>(a.post_weight);
    const T* pre = static_cast<const T*>(a.pre_weight);
    const T* bias = static_cast<const T*>(a.pre_bias);
    V w_post[C], w_pre[C], w_bias[C];
    auto gains = [&](V (&w)[C], const T* from) {
        if (!from) return;
#pragma unroll
        for (int c = 0; c < C; ++c) w[c] = row_load<TAIL>(from, first + c * step, a.width);
    };
    if (KEEP) gains(w_post, post), gains(w_pre, pre), gains(w_bias, bias);
    const int64_t by = gridDim.x * rows_here;
    for (int64_t row = blockIdx.x * rows_here + (WAVE ? threadIdx.x >> 6 : 0); row < a.rows;
         row += by) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* y = static_cast<const T*>(a.y) + row * a.y_stride;
        const T* g = static_cast<const T*>(a.gate) + row * a.gate_stride;
        const bool wide_gate = a.gate && a.gate_width > 1;
        V vx[C], vy[C], vg[C];
        float g1 = 1.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = first + c * step;
            vx[c] = row_load<TAIL>(x, at, a.width);
            if (a.y) vy[c] = row_load<TAIL>(y, at, a.width);
            if (wide_gate) vg[c] = row_load<TAIL>(g, at, a.width);
        }
        if (a.gate && !wide_gate) g1 = (float)g[0];
        if (!KEEP) gains(w_post, post);
        float v[C][8];
        if (a.y) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = TAIL || first + c * step < a.width ? (float)vy[c][i] : 0.0f;
            if (post) {
                normalise<KIND, C, WAVE>(v, a.width, first, step, a.eps, part, turn);
#pragma unroll
                for (int c = 0; c < C; ++c)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] *= (float)w_post[c][i];
            }
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[c][i] = __builtin_fmaf(a.alpha,
                                             v[c][i] * (wide_gate ? (float)vg[c][i] : g1),
                                             (float)vx[c][i]);
        } else {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (float)vx[c][i];
        }
        if (a.x_out) {
            T* out = static_cast<T*>(a.x_out) + row * a.width;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                V o;
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = (T)v[c][i];
                const int at = first + c * step;
                row_store<TAIL>(out, at, a.width, o);
            }
        }
        if (!a.n_out) continue;
        // what is behind the row's end must not reach the sums
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (first + c * step + (TAIL ? i : 0) >= a.width) v[c][i] = 0.0f;
        if (!KEEP) gains(w_pre, pre), gains(w_bias, bias);
        normalise<KIND, C, WAVE>(v, a.width, first, step, a.eps, part, turn);
        T* out = static_cast<T*>(a.n_out) + row * a.width;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            V o;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float r = v[c][i];
                if (pre) r *= (float)w_pre[c][i];
                if (bias) r += (float)w_bias[c][i];
                o[i] = (T)r;
            }
            const int at = first + c * step;
            row_store<TAIL>(out, at, a.width, o);
        }
    }
}

template <typename T, int KIND, int C, int THREADS, bool TAIL>
hipError_t launch_form(const NormArgs& a, hipStream_t s)
{
    constexpr int rows_here = THREADS == 64 ? 4 : 1, threads = THREADS < 256 ? 256 : THREADS;
    const int64_t want = ((int64_t)a.rows + rows_here - 1) / rows_here;
    // A workgroup a row (four of a wave each): the hardware evens them out better
    // than a stride over the rows, 8190 x 5120 with layer norms 95 us, striding 104,
    // 8000 x 2048 24 and 25.  Workgroups of 1024 threads gain more from their gains
    // in registers: 4000 x 16384 114 us striding, 126 so.
    const int64_t most = threads == 1024 ? 2 * kComputeUnits : most_blocks(threads);
    return launch(norm_kernel<T, KIND, C, THREADS, TAIL>,
                  dim3((unsigned)(want < most ? want : most)), threads, 0, s, a);
}

// Two or three chunks a thread in as few waves as that takes: 8190 rows of 4096
// (layer norms, a gate for every element) 64 us = 5.2 TB/s with two chunks in 256
// threads, 74 with one in 512.
template <typename T, int KIND, bool TAIL>
hipError_t launch_tail(const NormArgs& a, hipStream_t s)
{
    const int vectors = (a.width + 7) / 8;
    if (vectors <= 64) return launch_form<T, KIND, 1, 64, TAIL>(a, s);
    if (vectors <= 128) return launch_form<T, KIND, 2, 64, TAIL>(a, s);
    if (vectors <= 256) return launch_form<T, KIND, 1, 256, TAIL>(a, s);
    if (vectors <= 512) return launch_form<T, KIND, 2, 256, TAIL>(a, s);
    if (vectors <= 768) return launch_form<T, KIND, 3, 256, TAIL>(a, s);
    if (vectors <= 1024) return launch_form<T, KIND, 2, 512, TAIL>(a, s);
    if (vectors <= 1536) return launch_form<T, KIND, 3, 512, TAIL>(a, s);
    if (vectors <= 2048) return launch_form<T, KIND, 2, 1024, TAIL>(a, s);
    if (vectors <= 3072) return launch_form<T, KIND, 3, 1024, TAIL>(a, s);
    return launch_form<T, KIND, 4, 1024, TAIL>(a, s);
}

template <typename T, int KIND>
hipError_t launch_kind(const NormArgs& a, hipStream_t s)
{
    return a.width % 8 ? launch_tail<T, KIND, true>(a, s) : launch_tail<T, KIND, false>(a, s);
}

}  // namespace

hipError_t launch_norm(int type, int kind, const NormArgs& a, hipStream_t s)
{
    if (type == RM_TYPE_BF16)
        return kind == RM_NORM_RMS ? launch_kind<bf16, RM_NORM_RMS>(a, s)
                                   : launch_kind<bf16, RM_NORM_LAYER>(a, s);
    return kind == RM_NORM_RMS ? launch_kind<f16, RM_NORM_RMS>(a, s)
                               : launch_kind<f16, RM_NORM_LAYER>(a, s);
}

}  // namespace rm
