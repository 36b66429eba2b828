// prompt.hip -- causal attention of packed whole prompts (rm_prompt_attention).
//
// The rows of a tile are 128 (token, query head) pairs that share a kv head,
// tokens first, 32 a wave.  A workgroup takes 64 keys and values at a time through
// LDS, with the running maximum and sum of the softmax:
//   S^T = K Q^T    v_mfma_f32_32x32x16, keys as the 32 rows
//   O^T += V^T P   the same, value channels as the 32 rows
// A lane ends up with 32 of the 64 logits of one row, which are, in their order,
// the operand that the second product wants from it; what it wants of the values,
// four keys of one channel, is a transposing read of LDS.  Rows never leave their
// lane, so nothing but maxima and sums passes between lanes, and those between two.
//
// A step of a wave is 1024 cycles of matrix instructions for heads of 128 and about 900
// of exponentials, sums and maxima.  32 rows a wave leave two waves a SIMD (213
// registers), but little of one's products falls beside the other's softmax: by the
// counters both are 110% of the kernel's cycles.  16 384 tokens of 32 heads 2.03 to 2.16
// ms from card to card (1080 to 1020 TFLOP/s, the matrix cores busy for 51 to 56% of the
// cycles); with keys and values staged in registers and one wave a SIMD 3.57 ms.  Heads
// of 64 have half of the products for the same softmax (8192 tokens of 32 heads 310 us,
// 890 TFLOP/s); heads of 256 one wave a SIMD (8192 tokens of 16 heads 760 us, 720).
#include "rm_common.h"
#include "rm_decode.h"
#include "rm_lds.h"
#include "rm_slots.h"

namespace rm {
namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kKeys = kStepKeys;
constexpr int kRows = kTileRows;
static_assert(kRows == kWaves * 32, "32 rows a wave");
// Weights are 2^(logit - m + lift) with m at most kSlack below the row's largest logit
// so far (powers of two): m moves, and the sums with it, only where a logit passes it
// by more, which after the first keys is seldom.  In f16 the lift is 2^9: a weight of
// 2^kSlack times it is within the type, and one of 2^-23 keeps all its bits.  In bf16
// it takes the sum over all keys to 1/2 at most, so that no sum of weighted values
// leaves fp32 where the values are near the largest number; what goes is the bits of
// results below 2^-118 times the number of keys.
constexpr float kSlack = 6.0f;

__device__ inline float lift_of(bf16, int keys) { return -(kSlack + 1 + (32 - __builtin_clz(keys))); }
__device__ inline float lift_of(f16, int) { return 9.0f; }
template <typename T> struct Largest;
template <> struct Largest<bf16> { static constexpr float value = 0x1.fep127f; };
template <> struct Largest<f16> { static constexpr float value = 65504.0f; };
// the bits of the exponent, all of them set where a number is not finite
template <typename T> struct Exponent;
template <> struct Exponent<bf16> { static constexpr uint32_t bits = 0x7f80; };
template <> struct Exponent<f16> { static constexpr uint32_t bits = 0x7c00; };

__device__ inline f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x16 mfma(f16x8 a, f16x8 b, f32x16 c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// The two lanes of a row, 32 apart.
template <class Op>
__device__ inline float halves(float v)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    const auto h = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const uint32_t h0 = h[0], h1 = h[1];
    return Op::of(__builtin_bit_cast(float, h0), __builtin_bit_cast(float, h1));
}

__device__ inline SlotShape shape_of(const PromptArgs& a)
{
    return SlotShape{a.n_tokens, a.max_tokens, a.window, a.heads / a.kv_heads, a.kv_heads};
}

// The last sequence whose first slot is at most `slot`, found by 64 lanes that ask at
// once, with its borders; -1 for none.  Where offsets decrease the lanes that say yes
// are not the first ones, and it may be any sequence: tile_of takes what fits it.
struct Found {
    int sequence;
    int32_t begin, end;
};
__device__ inline Found sequence_at(const PromptArgs& a, const SlotShape& shape, int64_t slot)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = a.n_seqs;
    while (true) {
        const int step = (n + 63) / 64, b = lo + lane * step;
        const int32_t offset = a.offsets[min(b, a.n_seqs)];
        const bool before = lane * step < n && first_slot(shape, offset, b) <= slot;
        const int hit = __popcll(__ballot(before)) - 1;
        if (hit < 0) return Found{-1, 0, 0};
        lo += hit * step;
        n = min(step, n - hit * step);
        if (step > 1) continue;
        lo = __builtin_amdgcn_readfirstlane(lo);
        // the next lane has the end, mostly: a load less to wait for
        const int at = __builtin_amdgcn_readfirstlane(hit);
        return Found{lo, __builtin_amdgcn_readlane(offset, at),
                     at < 63 ? __builtin_amdgcn_readlane(offset, at + 1) : a.offsets[lo + 1]};
    }
}

// Zeros for rows [lo, hi) of out.
template <typename T, int D>
__device__ inline void clear(const PromptArgs& a, int64_t lo, int64_t hi)
{
    const int64_t row = (int64_t)a.heads * D;
    T* out = static_cast<T*>(a.out);
    for (int64_t i = lo * row + threadIdx.x * 8; i < hi * row; i += kWaves * 64 * 8)
        store8(out + i, typename Vec<T>::x8{});
}

// Rows that are in front of the first sequence or behind the last, and the check of
// the offsets.
constexpr int kClear = 128;      // rows a workgroup

template <typename T, int D>
__device__ inline void clear_rows(const PromptArgs& a, int64_t group)
{
    const int64_t lo = group * kClear, hi = min(lo + kClear, (int64_t)a.n_tokens);
    const int64_t begin = a.n_seqs ? a.offsets[0] : a.n_tokens;
    const int64_t end = a.n_seqs ? a.offsets[a.n_seqs] : a.n_tokens;
    if (begin > lo) clear<T, D>(a, lo, min(hi, begin));
    if (end < hi) clear<T, D>(a, max(lo, max(begin, end)), hi);
    if (group || !a.status) return;
    bool bad = false;
    for (int b = threadIdx.x; b < a.n_seqs; b += kWaves * 64) {
        const int64_t from = a.offsets[b], n = a.offsets[b + 1] - from;
        bad = bad || from < 0 || n < 0 || n > a.max_tokens || from + n > a.n_tokens;
    }
    if (bad) atomicOr(a.status, RM_ST_BAD_LENGTH);
}

// A step's keys and values in LDS: rows of D channels, chunks of 16 bytes swapped
// within a row so that what an access takes at once is spread over the 64 banks: a
// chunk of eight keys, or two pairs of chunks of four keys' values.
template <int D>
__device__ inline int key_at(int row, int chunk)
{
    return row * D + (chunk ^ (row & 7)) * 8;
}
template <int D>
__device__ inline int value_swap(int row)
{
    return (D == 64 ? row >> 1 & 1 : row & 3) * 4;
}
template <int D>
__device__ inline int value_at(int row, int chunk)
{
    return row * D + (chunk ^ value_swap<D>(row)) * 8;
}

// The operand of channels 32 d .. and the keys 16 t + 4 h + {0 .. 3, 8 .. 11} of the
// lane's half h, in the order of the weights.
template <typename T, int D>
__device__ inline typename Vec<T>::x8 values_of(const T* values, int d, int t)
{
    typedef short s16x8 __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63;
    const int row = t * 16 + (lane >> 5) * 4 + (lane & 15) / 4;
    const int chunk = d * 4 + (lane >> 4 & 1) * 2 + (lane & 3) / 2;
    auto four = [&](int r) {
        const T* from = values + value_at<D>(r, chunk) + (lane & 1) * 4;
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4*)from);
    };
    const s16x4 x = four(row), y = four(row + 8);
    return __builtin_bit_cast(typename Vec<T>::x8,
                              (s16x8){x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]});
}

// Whether any of the step's values is not finite; each lane of a wave has a part.  By
// the largest magnitude: with a branch for each value 97 tokens took 1.7 us longer, of 8.
template <typename T, int D>
__device__ inline bool any_odd(const T* values)
{
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 top = {0, 0};                  // of the magnitudes' bits, which are in their order
#pragma unroll
    for (int i = 0; i < kKeys * D / 512; ++i) {
        const u32x4 v = reinterpret_cast<const u32x4*>(values)[i * 64 + (threadIdx.x & 63)];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t magnitude = v[j] & 0x7fff7fffu;
            top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, magnitude));
        }
    }
    return max(top[0], top[1]) >= Exponent<T>::bits;
}

struct PromptPlan {
    uint32_t slots, first;       // of the tiles; the launch's first workgroup
};

// ALIGNED: keys and values by 16 bytes at addresses that are multiples of it, which go
// to LDS directly; others go through registers.
template <typename T, int D, bool ALIGNED>
__global__ __launch_bounds__(kWaves * 64) __attribute__((amdgpu_waves_per_eu(D <= 128 ? 2 : 1)))
void prompt_kernel(PromptArgs a, PromptPlan plan)
{
    typedef typename Vec<T>::x8 V;
    typedef typename Vec<T>::x2 V2;
    constexpr int CHUNKS = D / 8, LOADS = kKeys * CHUNKS / (kWaves * 64), ROWS = 64 / CHUNKS;
    __shared__ __align__(1024) T keys[2][kKeys * D], values[2][kKeys * D];

    const int KV = a.kv_heads, G = a.heads / KV;
    const uint32_t at = plan.first + blockIdx.x;         // 31 bits (prompt_fits)
    const uint32_t tiles = plan.slots * KV;
    if (at >= tiles) {
        clear_rows<T, D>(a, at - tiles);
        return;
    }
    const uint32_t slot = at / (uint32_t)KV;
    const int head = (int)(at - slot * KV);
    const SlotShape shape = shape_of(a);
    const Found found = sequence_at(a, shape, slot);
    if (found.sequence < 0) return;
    const int32_t begin = found.begin, end = found.end;
    const SlotTile tile = tile_of(shape, head, slot, found.sequence, begin, end);
    if (tile.what == SlotTile::CLEAR) clear<T, D>(a, tile.clear_from, tile.clear_upto);
    if (tile.what != SlotTile::ATTEND) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 31, h = lane >> 5;
    const int n = end - begin, r0 = tile.first_row, last_row = tile.last_row;
    const int first_pos = r0 / G, last_pos = last_row / G;
    const int lo = tile.first_step, hi = tile.end_step;
    // of this wave's rows
    const int wave_r0 = r0 + wave * 32;
    const int wave_first = min(wave_r0, last_row) / G;
    const int wave_last = min(wave_r0 + 31, last_row) / G;
    const int mine = min(wave_r0 + li, last_row), pos = mine / G;
    const int64_t q_token = begin + pos;
    const int q_head = head * G + mine % G;

    const T* k_base = static_cast<const T*>(a.k) + begin * a.k_stride + head * a.k_head;
    const T* v_base = static_cast<const T*>(a.v) + begin * a.v_stride + head * a.v_head;
    // Chunk c of a row lies at c with the row's bits in it (key_at, value_at), and a wave
    // loads ROWS rows at a time.
    const int row0 = wave * ROWS + lane / CHUNKS, chunk = lane % CHUNKS;
    const uint32_t key_chunk = (chunk ^ (row0 & 7)) * 16, value_chunk = (chunk ^ value_swap<D>(row0)) * 16;
    static_assert(ROWS * kWaves % 8 == 0, "the swapped chunks are those of every load");
    const uint32_t k_row = (uint32_t)(a.k_stride * 2), v_row = (uint32_t)(a.v_stride * 2);
    const uint32_t k_lds = __builtin_amdgcn_readfirstlane(lds_address(&keys[0][0]));
    const uint32_t v_lds = __builtin_amdgcn_readfirstlane(lds_address(&values[0][0]));
    V kr[ALIGNED ? 1 : LOADS], vr[ALIGNED ? 1 : LOADS];
    auto load = [&](int step, int buffer) {
        // behind the sequence's end its last row again, which the mask takes away
        const int t0 = step * kKeys;
        const uint32_t most = (uint32_t)(n - 1 - t0);
        const T* kp = k_base + t0 * a.k_stride;
        const T* vp = v_base + t0 * a.v_stride;
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t row = min((uint32_t)(row0 + i * ROWS * kWaves), most);
            if (ALIGNED) {
                const uint32_t to = buffer * (kKeys * D * 2) + (i * kWaves + wave) * 1024;
                to_lds16(k_lds + to, row * k_row + key_chunk, scalar((const uint8_t*)kp));
                to_lds16(v_lds + to, row * v_row + value_chunk, scalar((const uint8_t*)vp));
            } else {
                kr[ALIGNED ? 0 : i] = load8(kp + row * a.k_stride + key_chunk / 2);
                vr[ALIGNED ? 0 : i] = load8(vp + row * a.v_stride + value_chunk / 2);
            }
        }
    };
    auto store = [&](int buffer) {
#pragma unroll
        for (int i = 0; i < (ALIGNED ? 0 : LOADS); ++i) {
            const int to = (i * kWaves + wave) * 512 + lane * 8;
            *reinterpret_cast<V*>(&keys[buffer][to]) = kr[ALIGNED ? 0 : i];
            *reinterpret_cast<V*>(&values[buffer][to]) = vr[ALIGNED ? 0 : i];
        }
    };

    load(lo, lo & 1);
    V q[D / 16];
    {
        const T* row = static_cast<const T*>(a.q) + q_token * a.q_stride + q_head * a.q_head;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) {
            q[i] = load8(row + i * 16 + h * 8);
            if (a.scale <= 0) q[i] = q[i] * (T)(a.scale < 0 ? -1.0f : 0.0f);
        }
    }
    // positive, so that the largest logit is that of the largest product, and so that
    // what is masked stays -infinity
    const float to_log2 = a.scale == 0 ? 1.0f : fabsf(a.scale) * kLog2e;
    f32x16 o[D / 32];
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.0f;
    const float lift = lift_of(T(), last_pos + 1);
    float ref = -INFINITY, l = 0.0f;         // the row's m - lift, and its sum
    // whether the mask cuts the keys from t0 on, for some row of the tile
    auto cut = [&](int t0) {
        return t0 + kKeys - 1 > first_pos || (a.window > 0 && t0 <= last_pos - a.window);
    };
    bool odd = false;

    for (int step = lo; step < hi; ++step) {
        const int buffer = step & 1, t0 = step * kKeys;
        store(buffer);
        // the step's keys are there, and what the step before read is free
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (step + 1 < hi) load(step + 1, buffer ^ 1);
        // 0 times a value that is not finite would reach rows that do not see it.  Where
        // the mask cuts a step's keys and some value is not finite, the product is without
        // it, and the rows that see it get it behind the last step.  Every wave finds the
        // same.
        if (cut(t0) && __builtin_expect(__any(any_odd<T, D>(values[buffer])), 0)) {
            odd = true;
            __syncthreads();
            for (int i = threadIdx.x; i < kKeys * D; i += kWaves * 64)
                if (!(fabsf((float)values[buffer][i]) < INFINITY)) values[buffer][i] = (T)0.0f;
            __syncthreads();
        }
        if (t0 > wave_last || (a.window > 0 && t0 + kKeys <= wave_first - a.window + 1)) continue;

        // one wave's matrix instructions go before the other's softmax: without that 16 384
        // tokens of 32 heads take 2% longer
        __builtin_amdgcn_s_setprio(1);
        f32x16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const V e = *reinterpret_cast<const V*>(
                    &keys[buffer][key_at<D>(u * 32 + li, i * 2 + h)]);
                s[u] = mfma(e, q[i], s[u]);
            }
        }
        __builtin_amdgcn_s_setprio(0);
        // of register i of part u: key t0 + 32 u + 8 (i / 4) + 4 h + i % 4
        const bool masked = t0 + kKeys - 1 > wave_first ||
                            (a.window > 0 && t0 <= wave_last - a.window);
        if (masked) {
            const int upto = pos - t0 - 4 * h, from = a.window > 0 ? upto - a.window : -kKeys - 8;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int j = u * 32 + i / 4 * 8 + i % 4;
                    if (j > upto || j <= from) s[u][i] = -INFINITY;
                }
        }
        float top = s[0][0];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[u][i]);
        top = halves<Max>(top) * to_log2 - lift;
        if (__any(top > ref + kSlack)) {
            // rows that have seen nothing yet have sums of 0
            const float to = fmaxf(ref, top);
            const float f = to == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(ref - to);
            ref = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float off = ref == -INFINITY ? 0.0f : ref;
        V p[4];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], to_log2, -off));
                l += e;
                p[u * 2 + i / 8][i % 8] = (T)e;
            }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int t = 0; t < 4; ++t) o[d] = mfma(values_of<T, D>(values[buffer], d, t), p[t], o[d]);
        __builtin_amdgcn_s_setprio(0);
    }
    l = halves<Add>(l);
    const float inv = 1.0f / l;
    if (__builtin_expect(odd, 0)) {
        // Of the steps that are cut: what is not finite as it is, or NaN where its weight is
        // 0 in the products' type.  Key by key, from memory: beside the last step's weights
        // it would take registers from every step.
        typedef T V4 __attribute__((ext_vector_type(4)));
        typedef V4 V4u __attribute__((aligned(2)));
        for (int key = lo * kKeys; key <= last_pos; ++key) {
            if (key % kKeys == 0 && !cut(key)) {
                key += kKeys - 1;
                continue;
            }
            const T* v = v_base + key * a.v_stride + h * 4;
            bool any = false;
#pragma unroll
            for (int c = 0; c < D; c += 8)
#pragma unroll
                for (int i = 0; i < 4; ++i) any = any || !(fabsf((float)v[c + i]) < INFINITY);
            if (!__any(any)) continue;
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
                const V e = load8(k_base + key * a.k_stride + i * 16 + h * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = __builtin_fmaf((float)e[j], (float)q[i][j], s);
            }
            s = halves<Add>(s);
            const float off = ref == -INFINITY ? 0.0f : ref;
            const T weight = (T)__builtin_amdgcn_exp2f(__builtin_fmaf(s, to_log2, -off));
            if (key > pos || (a.window > 0 && key <= pos - a.window)) continue;
#pragma unroll
            for (int d = 0; d < D / 32; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const V4 four = *reinterpret_cast<const V4u*>(v + d * 32 + g * 8);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (!(fabsf((float)four[i]) < INFINITY))
                            o[d][g * 4 + i] += (float)weight > 0.0f ? (float)four[i] : __builtin_nanf("");
                }
        }
    }
    // The sum has the weights before their rounding, so a mean of the largest numbers may
    // come out beyond them.
    float largest = 0.0f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) largest = fmaxf(largest, fabsf(o[d][i]));
    if (__builtin_expect(__any(largest * inv > Largest<T>::value), 0)) {
        const float most = Largest<T>::value * l;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (fabsf(o[d][i]) < INFINITY) o[d][i] = fminf(fmaxf(o[d][i], -most), most);
    }
    T* out = static_cast<T*>(a.out) + (q_token * a.heads + q_head) * D;
    const bool mine_too = wave_r0 + li <= last_row;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            // channels 4 h .. and 8 + 4 h ..: the halves of a row swap to get eight
            uint32_t w[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int r = (j * 2 + i) * 4 + e * 2;
                    const V2 two = {(T)(o[d][r] * inv), (T)(o[d][r + 1] * inv)};
                    w[i][e] = __builtin_bit_cast(uint32_t, two);
                }
            const auto x = __builtin_amdgcn_permlane32_swap(w[0][0], w[1][0], false, false);
            const auto y = __builtin_amdgcn_permlane32_swap(w[0][1], w[1][1], false, false);
            const uint32_t x0 = x[0], x1 = x[1], y0 = y[0], y1 = y[1];
            if (mine_too)
                store8(out + d * 32 + j * 16 + h * 8,
                       __builtin_bit_cast(V, (u32x4){x0, y0, x1, y1}));
        }
}

int64_t slots_of(const PromptArgs& a)
{
    return a.n_seqs ? (int64_t)a.n_tokens * (a.heads / a.kv_heads) / kRows + a.n_seqs : 0;
}
int64_t clears_of(const PromptArgs& a) { return ((int64_t)a.n_tokens + kClear - 1) / kClear; }

template <typename T, int D, bool ALIGNED>
hipError_t launch_form(const PromptArgs& a, hipStream_t s)
{
    const int64_t slots = slots_of(a), all = slots * a.kv_heads + clears_of(a);
    const int64_t most = most_blocks(kWaves * 64) / 8 * 8;
    for (int64_t first = 0; first < all; first += most) {
        const int64_t n = all - first < most ? all - first : most;
        const PromptPlan p = {(uint32_t)slots, (uint32_t)first};
        const hipError_t e = launch(prompt_kernel<T, D, ALIGNED>, dim3((unsigned)n), kWaves * 64, 0, s, a, p);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, int D>
hipError_t launch_width(const PromptArgs& a, hipStream_t s)
{
    const uint64_t bits = (uint64_t)(uintptr_t)a.k | (uint64_t)(uintptr_t)a.v |
                          (uint64_t)(a.k_stride | a.k_head | a.v_stride | a.v_head) * 2;
    // a step's rows are counted in 32 bits
    const bool near = a.k_stride >= 0 && a.v_stride >= 0 && a.k_stride < 1 << 24 &&
                      a.v_stride < 1 << 24;
    return bits % 16 == 0 && near ? launch_form<T, D, true>(a, s) : launch_form<T, D, false>(a, s);
}

template <typename T>
hipError_t launch_type(int head_dim, const PromptArgs& a, hipStream_t s)
{
    if (head_dim == 64) return launch_width<T, 64>(a, s);
    if (head_dim == 128) return launch_width<T, 128>(a, s);
    return launch_width<T, 256>(a, s);
}

}  // namespace

bool prompt_fits(const PromptArgs& a)
{
    return slots_of(a) * a.kv_heads + clears_of(a) <= 0x7fffffff;
}

hipError_t launch_prompt(int type, int head_dim, const PromptArgs& a, hipStream_t s)
{
    return type == RM_TYPE_BF16 ? launch_type<bf16>(head_dim, a, s)
                                : launch_type<f16>(head_dim, a, s);
}

}  // namespace rm
