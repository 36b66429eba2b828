// attend.hip -- attention over the paged 8-bit cache (rm_cache_attention).
//
// The rows of a tile are the (token, query head) pairs that share a kv head,
// tokens first: 16 for a decode step, 32 for a chunk of a prompt.  A wave
// takes 64 cached tokens at a time, all in registers, with the running maximum
// and sum of the softmax:
//   S^T = K Q^T   v_mfma_f32_16x16x32 in q's type, keys as the 16 rows
//   O^T += V^T P  the same in f16, value channels as the 16 rows
// Which token a row of the first product stands for is free, so row i of
// instruction t is token (i / 4) * 16 + 4 t + i % 4: a lane then ends up with the
// weights of 16 neighbouring tokens, exactly the operand that the second
// product wants from it, and with values stored channel by channel its other
// operand is one 16-byte load.  Nothing passes through LDS until the waves join.
//
// Codes are exact in bf16 and f16.  Scales are constant over a page, so they
// multiply the logits and the weights: what enters the second product is weight
// times scale, relative to the row's own largest such product so far, which is
// kept beside the maximum of its logits.
//
// That operand is f16, 2^-11 of each weight: in a mean over the tokens less than the
// rounding of a bf16 output and about that of an f16 one (chunks of prompts in f16
// are 3.0e-4 from 64 bits, a plain form in fp32 2.1e-4).  Matrix instructions in
// fp32 have a sixteenth of the rate.
//
// A step of decoding is bound by reading the codes once.  The token axis is
// split over the workgroup's waves and, when there are few tiles, over
// workgroups whose partial results a second kernel joins.
#include "rm_common.h"
#include "rm_decode.h"

namespace rm {
namespace {

constexpr int kBlock = 64;    // cached tokens a wave takes at a time
constexpr int kWaves = 4;
constexpr int kMostSplits = 256;
// Weights and their sums carry 2^kLift, which the quotient takes off again: f16
// holds a weight times its page's scale in full down to 2^-28 of the row's largest,
// below that to 2^-39.
constexpr float kLift = 15.0f;

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Eight codes as elements of the product's type; exact.
template <int FMT>
__device__ inline void decode8(uint32_t lo, uint32_t hi, bf16x8& out)
{
    if (FMT == RM_CODES_E4M3) {
        const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false);
        const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
        const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false);
        const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
        out = bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        // Else the compiler carries the next block's codes as bytes, a register
        // each: 83 registers spilt, chunks of prompts in bf16 took 212 us, 105 so; two
        // sequences of 125 000 tokens 106 and 99.
        asm("" : "+v"(lo), "+v"(hi));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            out[i] = (bf16)(float)(int8_t)(lo >> (8 * i));
            out[4 + i] = (bf16)(float)(int8_t)(hi >> (8 * i));
        }
    }
}
template <int FMT>
__device__ inline void decode8(uint32_t lo, uint32_t hi, f16x8& out)
{
    if (FMT == RM_CODES_E4M3) {
        const f16x2 a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, false);
        const f16x2 b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.0f, true);
        const f16x2 c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, false);
        const f16x2 d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.0f, true);
        out = f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    } else {
        // code + 128 in the low bits of 1024 is 1152 + code; the difference is exact
        const uint32_t w[2] = {lo ^ 0x80808080u, hi ^ 0x80808080u};
        u32x4 r;
        const f16x2 c = {(f16)1152.0f, (f16)1152.0f};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = __builtin_amdgcn_perm(0x64646464u, w[i >> 1],
                                                     i & 1 ? 0x04030402u : 0x04010400u);
            r[i] = __builtin_bit_cast(uint32_t, (f16x2)(__builtin_bit_cast(f16x2, p) - c));
        }
        out = __builtin_bit_cast(f16x8, r);
    }
}

// 2^x; results below the normal range are 0.
__device__ inline float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

struct Plan {
    int32_t tiles, splits;      // tiles of rows a sequence and kv head; splits of a tile
    int32_t rows;               // of a tile that a sequence can have
    int32_t columns;            // a tile has 16 times as many rows
    int32_t clear;              // workgroups behind the tiles', for clear_rows
    int64_t parts;              // splits of all tiles
};

// Rows and token range of a tile.
struct Tile {
    int32_t rows, first_pos, lo, hi, all_lo, all_hi;
};

__device__ inline Tile tile_of(const Sequence& s, int32_t group, int32_t window, int32_t tile,
                               int32_t height)
{
    Tile t;
    const int32_t r0 = tile * height;
    t.rows = min(height, s.n * group - r0);
    t.first_pos = s.length - s.n;
    const int32_t p0 = t.first_pos + r0 / group, p1 = t.first_pos + (r0 + t.rows - 1) / group;
    t.lo = window > 0 ? max(0, p0 - window + 1) : 0;        // seen by some row
    t.hi = p1 + 1;
    t.all_lo = window > 0 ? max(0, p1 - window + 1) : 0;    // seen by every row
    t.all_hi = p0 + 1;
    return t;
}

// Zeros for those of the rows from kClear * group on that no sequence holds, or one
// that is out of range.  The sequences need not be in order, so all of them are
// asked; the rows that they hold are marked in LDS.
constexpr int kClear = 512;

template <typename T, int D>
__device__ inline void clear_rows(const AttendArgs& a, int group)
{
    __shared__ uint32_t held[kClear / 32];
    const int64_t r0 = (int64_t)group * kClear;
    const int count = (int)min((int64_t)kClear, a.seqs.n_tokens - r0);
    if (threadIdx.x < kClear / 32) held[threadIdx.x] = 0;
    __syncthreads();
    for (int b = threadIdx.x; b < a.seqs.n_seqs; b += kWaves * 64) {
        const Sequence s = sequence_of(a.seqs, a.cache.page_tokens, b);
        const int64_t lo = max((int64_t)s.first, r0) - r0;
        const int64_t hi = min((int64_t)s.first + s.n, r0 + count) - r0;
        for (int64_t r = lo; r < hi; r = (r / 32 + 1) * 32) {
            const int n = (int)min((int64_t)32, hi - r / 32 * 32);
            atomicOr(&held[r / 32], (n == 32 ? ~0u : (1u << n) - 1) & ~0u << (r % 32));
        }
    }
    __syncthreads();
    const int64_t row = (int64_t)a.heads * D;
    for (int w = 0; w < (count + 31) / 32; ++w) {
        uint32_t none = ~(uint32_t)__builtin_amdgcn_readfirstlane(held[w]);
        for (; none; none &= none - 1) {
            const int r = w * 32 + __ffs(none) - 1;
            if (r >= count) break;
            for (int64_t i = threadIdx.x * 8; i < row; i += kWaves * 64 * 8)
                store8(static_cast<T*>(a.out) + (r0 + r) * row + i, typename Vec<T>::x8{});
        }
    }
}

// Two waves a SIMD where the registers allow it: left to itself the compiler
// takes all registers for one (32 rows, chunks of prompts: 209 us, with two 134).
template <typename T, int FMT, int D, int C>
__global__ __launch_bounds__(kWaves * 64)
__attribute__((amdgpu_waves_per_eu(D <= 128 ? 2 : 1))) void
attend_kernel(AttendArgs a, Plan plan, uint32_t first)
{
    typedef typename Vec<T>::x8 V;
    constexpr int H = 16 * C, W = kWaves;      // rows of a tile
    extern __shared__ __align__(16) float join[];
    __shared__ float join_m[W][H], join_l[W][H];

    const int KV = a.cache.kv_heads, TK = a.cache.page_tokens, G = a.heads / KV;
    // 31 bits at most (kMostBlocks): with 64-bit divisions one sequence of 501 tokens
    // takes 10.7 us, so 10.3
    const uint32_t part_at = first + blockIdx.x;
    if (part_at >= (uint32_t)plan.parts) {
        clear_rows<T, D>(a, (int)(part_at - (uint32_t)plan.parts));
        return;
    }
    uint32_t at = part_at;
    const int split = (int)(at % (uint32_t)plan.splits);
    at /= (uint32_t)plan.splits;
    const int tile = (int)(at % (uint32_t)plan.tiles);
    at /= (uint32_t)plan.tiles;
    const int head = (int)(at % (uint32_t)KV), b = (int)(at / (uint32_t)KV);
    const Sequence s = sequence_of(a.seqs, TK, b);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, quad = lane >> 4;

    if (s.n == 0) {
        if (s.bad && a.status && threadIdx.x == 0) atomicOr(a.status, RM_ST_BAD_LENGTH);
        // with token_offsets the rows are cleared by clear_rows
        if (a.seqs.token_offsets || tile || split) return;
        for (int i = threadIdx.x; i < G * D; i += W * 64)
            static_cast<T*>(a.out)[((int64_t)b * a.heads + head * G) * D + i] = (T)0.0f;
        return;
    }
    if (tile * H >= s.n * G) return;
    const Tile t = tile_of(s, G, a.window, tile, H);
    const int b0 = t.lo / kBlock, b1 = (t.hi + kBlock - 1) / kBlock;
    const int per = (b1 - b0 + plan.splits - 1) / plan.splits;
    const int from = b0 + split * per, upto = min(b1, from + per);

    const int32_t* table = a.seqs.table + (int64_t)b * a.seqs.table_stride;
    const int shift = __ffs(TK) - 1, last_page = (s.length - 1) >> shift;
    // the pages of the 16 tokens of a block whose keys and whose values the lane
    // loads; an id out of range becomes page 0 and the tokens are not seen
    struct Pages {
        int32_t k, v;
        bool bad;
    };
    auto ids = [&](int block) {
        const int t0 = block * kBlock;
        Pages p;
        p.k = table[min((t0 + (li >> 2) * 16) >> shift, last_page)];
        p.v = table[min((t0 + quad * 16) >> shift, last_page)];
        return p;
    };
    auto checked = [&](Pages p) {
        p.bad = (uint32_t)p.v >= (uint32_t)a.cache.n_pages;
        if (p.bad) p.v = 0;
        if ((uint32_t)p.k >= (uint32_t)a.cache.n_pages) p.k = 0;
        return p;
    };
    u32x4 kc[4][D / 64], vc[D / 16];
    float ks, vs;
    auto load_k = [&](int block, const Pages& p) {
        const int tk = block * kBlock + (li >> 2) * 16;
        const uint8_t* kp = static_cast<const uint8_t*>(a.cache.k) +
                            (((int64_t)p.k * KV + head) * TK + (tk & (TK - 1)) + (li & 3)) * D +
                            quad * 16;
        ks = a.cache.k_scale[(int64_t)p.v * KV + head];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < D / 64; ++j)
                kc[i][j] = *reinterpret_cast<const u32x4*>(kp + i * 4 * D + j * 64);
    };
    auto load_v = [&](int block, const Pages& p) {
        const int tv = block * kBlock + quad * 16;
        const int64_t bv = (int64_t)p.v * KV + head;
        const uint8_t* vp = static_cast<const uint8_t*>(a.cache.v) + (bv * D + li) * TK +
                            (tv & (TK - 1));
        vs = a.cache.v_scale[bv];
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
            vc[d] = *reinterpret_cast<const u32x4*>(vp + d * 16 * TK);
    };

    // queries: row 16 c + li of the tile, channels 64 j + 16 quad + 8 k of the
    // operand for the k-th half of the j-th 16-byte load of keys
    V q[C][D / 32];
    int32_t pos[C];
    f32x4 o[D / 16][C];
    // m and r: the largest logit so far, alone and times the scale of its values,
    // both as powers of two
    float m[C], l[C], r[C];
    Pages now, next;
    int block = from + wave;
    if (block < upto) {
        now = ids(block);
        next = ids(min(block + W, upto - 1));
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int r = tile * H + min(c * 16 + li, t.rows - 1);
        pos[c] = t.first_pos + r / G;
        const T* row = static_cast<const T*>(a.q) + (s.first + r / G) * a.q_stride +
                       (head * G + r % G) * a.q_head;
#pragma unroll
        for (int k = 0; k < D / 32; ++k)
            q[c][k] = load8(row + (k >> 1) * 64 + quad * 16 + (k & 1) * 8);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
        m[c] = -INFINITY;
        r[c] = -INFINITY;
        l[c] = 0.0f;
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d][c] = f32x4{0, 0, 0, 0};
    }
    const float to_log2 = a.scale * 1.44269504088896340736f;
    int32_t st = 0;
    if (block < upto) {
        now = checked(now);
        load_k(block, now);
        load_v(block, now);
    }
    for (; block < upto; block += W) {
        const int t0 = block * kBlock, tv = t0 + quad * 16;
        const int following = min(block + W, upto - 1);      // the last block again at the end
        f32x4 sc[4][C];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
            for (int c = 0; c < C; ++c) sc[i][c] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < D / 32; ++k) {
                V e;
                decode8<FMT>(kc[i][k >> 1][(k & 1) * 2], kc[i][k >> 1][(k & 1) * 2 + 1], e);
#pragma unroll
                for (int c = 0; c < C; ++c) sc[i][c] = mfma(e, q[c][k], sc[i][c]);
            }
        }
        // the next block's keys fly while this one's weights are taken, its values
        // while its keys are multiplied, and the page after it is looked up
        __builtin_amdgcn_sched_barrier(0);         // the codes stay codes until their turn
        const float k_log2 = ks * to_log2;
        // the lane's 16 tokens share a page; one that no row sees has no say
        const bool near = tv < t.hi && tv + 16 > t.lo, bad = now.bad;
        if (bad && near) st = RM_ST_BAD_PAGE;
        next = checked(next);
        load_k(following, next);
        const Pages after = ids(min(following + W, upto - 1));
        __builtin_amdgcn_sched_barrier(0);
        const bool whole = t0 >= t.all_lo && t0 + kBlock <= t.all_hi && !__any(bad);
        // scale = part * 2^power; one that is not finite goes into the weights as it
        // is and reaches the rows that see the page, not what their others are
        // relative to
        const float v_scale = near && !bad ? vs : 0.0f;
        const bool finite = fabsf(v_scale) < INFINITY;
        const float power = finite && v_scale != 0.0f
                                ? (float)__builtin_amdgcn_frexp_expf(v_scale) : -INFINITY;
        float x[C], share[C];
        bool moved = false;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            x[c] = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float v = sc[i][c][k] * k_log2;
                    if (!whole) {
                        const int token = tv + 4 * i + k;
                        const bool seen = token <= pos[c] && !bad &&
                                          (a.window <= 0 || token > pos[c] - a.window);
                        v = seen ? v : -INFINITY;
                    }
                    sc[i][c][k] = v;
                    x[c] = fmaxf(x[c], v);
                }
            moved |= x[c] > m[c] || x[c] + power > r[c];
        }
        // no lane has more than its row's maxima after the first blocks, mostly
        if (__any(moved)) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const float top = fmaxf(m[c], rows_reduce<Max>(x[c]));
                const float high = fmaxf(r[c], rows_reduce<Max>(x[c] + power));
                l[c] *= top == -INFINITY ? 1.0f : exp2_of(m[c] - top);
                const float shrink = high == -INFINITY ? 1.0f : exp2_of(r[c] - high);
                m[c] = top;
                r[c] = high;
#pragma unroll
                for (int d = 0; d < D / 16; ++d) o[d][c] *= shrink;
            }
        }
        // the exponent is bounded where the weights beside it are 0
#pragma unroll
        for (int c = 0; c < C; ++c)
            share[c] = finite ? __builtin_amdgcn_frexp_mantf(v_scale) *
                                    exp2_of(fminf(m[c] - r[c] + power, 126.0f))
                              : v_scale;
        f16x8 p[2][C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const float base = m[c] == -INFINITY ? 0.0f : m[c] - kLift;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float e = exp2_of(sc[i][c][k] - base);
                    l[c] += e;
                    float w = e * share[c];
                    if (!whole) w = e == 0.0f ? 0.0f : w;
                    p[i >> 1][c][(i & 1) * 4 + k] = (f16)w;
                }
        }
        if (!whole) {
            // bytes of tokens that no row sees, which may hold anything
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const bool keep = tv + i >= t.lo && tv + i < t.hi && !bad;
                const uint32_t mask = keep ? ~0u : ~(255u << (8 * (i & 3)));
#pragma unroll
                for (int d = 0; d < D / 16; ++d) vc[d][i >> 2] &= mask;
            }
        }
#pragma unroll
        for (int d = 0; d < D / 16; ++d)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                f16x8 e;
                decode8<FMT>(vc[d][2 * k], vc[d][2 * k + 1], e);
#pragma unroll
                for (int c = 0; c < C; ++c) o[d][c] = mfma(e, p[k][c], o[d][c]);
            }
        __builtin_amdgcn_sched_barrier(0);
        load_v(following, next);
        __builtin_amdgcn_sched_barrier(0);
        now = next;
        next = after;
    }
    report_status(a.status, st);

    // join the waves: common maximum, then the upper half's sums onto the lower
    // half's, and so on
#pragma unroll
    for (int c = 0; c < C; ++c) {
        l[c] = rows_reduce<Add>(l[c]);
        if (quad == 0) join_m[wave][c * 16 + li] = m[c], join_l[wave][c * 16 + li] = l[c];
    }
    __syncthreads();
    // a row's maximum and sum over the waves
    auto statistics = [&](int row, float& top, float& sum) {
        top = join_m[0][row];
        for (int w = 1; w < W; ++w) top = fmaxf(top, join_m[w][row]);
        const float base = top == -INFINITY ? 0.0f : top;
        sum = 0.0f;
        for (int w = 0; w < W; ++w) sum += join_l[w][row] * exp2_of(join_m[w][row] - base);
    };
    // [wave][d / 4][row][4]: neighbouring lanes write neighbouring rows
#pragma unroll
    for (int c = 0; c < C; ++c) {
        float top, sum;
        statistics(c * 16 + li, top, sum);
        // the wave's share of the mean, so that no sum passes the largest value
        const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
        const float f = exp2_of(r[c] - (top == -INFINITY ? 0.0f : top) - kLift) *
                        (inv * (float)(1 << (int)kLift));
#pragma unroll
        for (int d = 0; d < D / 16; ++d) o[d][c] *= f;
    }
    f32x4* sums = reinterpret_cast<f32x4*>(join);
    auto place = [&](int w, int d, int c) { return ((w * (D / 4) + d * 4 + quad) * H) + c * 16 + li; };
#pragma unroll
    for (int half = W / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int d = 0; d < D / 16; ++d) sums[place(wave - half, d, c)] = o[d][c];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int d = 0; d < D / 16; ++d) o[d][c] += sums[place(wave, d, c)];
        }
        __syncthreads();
    }
    if (wave == 0) {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int d = 0; d < D / 16; ++d) sums[place(0, d, c)] = o[d][c];
    }
    __syncthreads();
    float* part = static_cast<float*>(a.workspace);
    for (int u = threadIdx.x; u < t.rows * (D / 8); u += W * 64) {
        const int row = u / (D / 8), d = u % (D / 8) * 8;
        const f32x4 v0 = sums[(d / 4) * H + row], v1 = sums[(d / 4 + 1) * H + row];
        if (plan.splits == 1) {
            V r;
#pragma unroll
            for (int i = 0; i < 4; ++i) r[i] = (T)v0[i], r[4 + i] = (T)v1[i];
            const int rr = tile * H + row;
            store8(static_cast<T*>(a.out) +
                       ((int64_t)(s.first + rr / G) * a.heads + head * G + rr % G) * D + d, r);
        } else {
            float* to = part + ((int64_t)part_at * H + row) * D + d;
            reinterpret_cast<f32x4*>(to)[0] = v0;
            reinterpret_cast<f32x4*>(to)[1] = v1;
            if (d == 0) {
                float* ml = part + plan.parts * H * D + ((int64_t)part_at * H + row) * 2;
                statistics(row, ml[0], ml[1]);
            }
        }
    }
}

// A workgroup a row of a tile: the splits' means, weighted.  A wave takes every
// fourth split, a lane the splits' maxima and sums first.
template <typename T, int D, int C>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a, Plan plan)
{
    constexpr int H = 16 * C, N = D / 64;
    __shared__ float factor[kMostSplits];
    __shared__ float sums[4][D];
    const int KV = a.cache.kv_heads, G = a.heads / KV;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t at = blockIdx.x;
    const int row = (int)(at % plan.rows);
    at /= plan.rows;
    const int64_t block = at * plan.splits;
    const int tile = (int)(at % plan.tiles);
    at /= plan.tiles;
    const int head = (int)(at % KV);
    const Sequence s = sequence_of(a.seqs, a.cache.page_tokens, (int)(at / KV));
    const int rr = tile * H + row;
    if (rr >= s.n * G) return;
    const float* part = static_cast<const float*>(a.workspace);
    const float* ml = part + plan.parts * H * D + (block * H + row) * 2;
    // every wave the same: one split a lane, then the next 64
    float top = -INFINITY;
    for (int i = lane; i < plan.splits; i += 64) top = fmaxf(top, ml[(int64_t)i * H * 2]);
    top = wave_reduce<Max>(top);
    const float base = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f;
    for (int i = lane; i < plan.splits; i += 64) {
        const float f = exp2_of(ml[(int64_t)i * H * 2] - base), l = ml[(int64_t)i * H * 2 + 1];
        sum = __builtin_fmaf(l, f, sum);
        // a split that saw nothing may not have written its mean
        if (wave == 0) factor[i] = l == 0.0f ? -1.0f : f * l;
    }
    sum = wave_reduce<Add>(sum);
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    __syncthreads();
    float v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = 0.0f;
    const float* from = part + (block * H + row) * D + lane * N;
    typedef float Vn __attribute__((ext_vector_type(N)));
#pragma unroll 4
    for (int i = wave; i < plan.splits; i += 4) {
        const float weight = factor[i], f = weight * inv;
        const Vn x = *reinterpret_cast<const Vn*>(from + (int64_t)i * H * D);
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] = weight < 0.0f ? v[k] : __builtin_fmaf(x[k], f, v[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < N; ++k) sums[wave][lane * N + k] = v[k];
    __syncthreads();
    T* out = static_cast<T*>(a.out) +
             ((int64_t)(s.first + rr / G) * a.heads + head * G + rr % G) * D;
    for (int d = threadIdx.x; d < D; d += 256)
        out[d] = (T)(sums[0][d] + sums[1][d] + sums[2][d] + sums[3][d]);
}

// 64 rows a tile need all registers of a SIMD for one wave: chunks of prompts
// took 238 us with 64, 134 with 32, 182 with 16.
int columns_of(int64_t rows)
{
    return rows <= 16 ? 1 : 2;
}

Plan plan_of(const rm_cache& c, const rm_sequences& s, int32_t heads)
{
    const int64_t rows = most_tokens(s) * (heads / c.kv_heads);
    Plan p;
    p.columns = columns_of(rows);
    const int height = 16 * p.columns;
    p.clear = s.token_offsets ? (int32_t)(((int64_t)s.n_tokens + kClear - 1) / kClear) : 0;
    p.tiles = (int32_t)((rows + height - 1) / height);
    p.rows = (int32_t)(rows < height ? rows : height);
    const int64_t units = (int64_t)s.n_seqs * c.kv_heads * p.tiles;
    // Two workgroups a CU, as far as every wave has a block of the longest possible
    // sequence and there are three each without: the join is a launch.  One sequence
    // of 501 tokens: 9.7 us in one part, 11.0 in two; one of 2000: 11.4 in eight, 13.0
    // in four; 26 ragged ones of up to 1457: 13.5 in five, 15.6 in two; two of 125 000:
    // 108 in 32, 115 in 64; 64 ragged ones of up to 4096, 512 workgroups already: 65, in
    // two parts 69; 40 of up to 16 000, 320 workgroups: 269 in one part, 183 in two.
    const int64_t blocks = ((int64_t)s.table_stride * c.page_tokens + kBlock - 1) / kBlock;
    const int64_t want = units > 0 ? (2 * kComputeUnits + units - 1) / units : 1;
    const int64_t most = blocks < 3 * kWaves ? 1 : blocks / kWaves;
    p.splits = (int32_t)(want < most ? want : most);
    if (p.splits > kMostSplits) p.splits = kMostSplits;
    if (p.splits < 1) p.splits = 1;
    p.parts = units * p.splits;
    return p;
}

template <typename T, int FMT, int D, int C>
hipError_t launch_columns(const AttendArgs& a, const Plan& p, hipStream_t s)
{
    const int64_t blocks = p.parts + p.clear, rows = p.parts / p.splits * p.rows;
    constexpr int64_t most = most_blocks(kWaves * 64);
    const size_t lds = (size_t)(kWaves / 2) * 16 * C * D * sizeof(float);    // 64 KB at most
    const auto kernel = attend_kernel<T, FMT, D, C>;
    if (lds > 60 * 1024) {      // with the static arrays over 64 KB
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    hipError_t e = hipSuccess;
    for (int64_t first = 0; first < blocks && e == hipSuccess; first += most)
        e = launch(kernel, dim3((unsigned)(blocks - first < most ? blocks - first : most)),
                   kWaves * 64, lds, s, a, p, (uint32_t)first);
    if (e != hipSuccess || p.splits == 1 || rows == 0) return e;
    return launch(attend_join_kernel<T, D, C>, dim3((unsigned)rows), 256, 0, s, a, p);
}

template <typename T, int FMT, int D>
hipError_t launch_dim(const AttendArgs& a, hipStream_t s)
{
    const Plan p = plan_of(a.cache, a.seqs, a.heads);
    if (p.columns == 1)
        return launch_columns<T, FMT, D, 1>(a, p, s);
    return launch_columns<T, FMT, D, 2>(a, p, s);
}

template <typename T, int FMT>
hipError_t launch_codes(const AttendArgs& a, hipStream_t s)
{
    if (a.cache.head_dim == 64) return launch_dim<T, FMT, 64>(a, s);
    if (a.cache.head_dim == 128) return launch_dim<T, FMT, 128>(a, s);
    return launch_dim<T, FMT, 256>(a, s);
}

}  // namespace

bool attend_fits(const rm_cache& c, const rm_sequences& s, int32_t heads)
{
    const Plan p = plan_of(c, s, heads);
    return p.parts + p.clear <= kMostBlocks;
}

size_t attend_workspace(const rm_cache& c, const rm_sequences& s, int32_t heads)
{
    const Plan p = plan_of(c, s, heads);
    if (p.splits == 1) return 256;
    return ((size_t)p.parts * 16 * p.columns * (c.head_dim + 2) * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_attend(int type, const AttendArgs& a, hipStream_t s)
{
    if (type == RM_TYPE_BF16)
        return a.cache.codes == RM_CODES_INT8 ? launch_codes<bf16, RM_CODES_INT8>(a, s)
                                              : launch_codes<bf16, RM_CODES_E4M3>(a, s);
    return a.cache.codes == RM_CODES_INT8 ? launch_codes<f16, RM_CODES_INT8>(a, s)
                                          : launch_codes<f16, RM_CODES_E4M3>(a, s);
}

}  // namespace rm
