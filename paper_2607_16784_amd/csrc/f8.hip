// f8.hip -- 8-bit floating codes with a scale for each block of 128 columns
// (rm_f8_quantize) and the projection of such rows (rm_f8_linear).
//
// v_mfma_f32_16x16x128_f8f6f4 multiplies one block of 128 columns of 16 weight
// rows and 16 rows of x: a lane gets four neighbouring outputs of one row of x, so
// a block's sums take one factor a lane, x_scale times scale, and four fused
// multiply-adds into the fp32 totals.  The order of the 128 columns is free as
// long as both operands keep it: lane l has the bytes 16 (l / 16) .. and
// 64 + 16 (l / 16) .. of its row.
//
// Up to 16 rows of x (few_kernel): one row is bound by reading the codes, more also by
// what every workgroup does again, reading and quantising x.  The blocks go round the
// waves of a workgroup, x is quantised in the registers of the wave that multiplies it,
// and the waves' totals are joined through LDS.  In a graph, with weights that come
// from memory: 28672 x 4096 with 1 row 28.1 us (4.2 TB/s), 16 rows 32.1; 4096 x 4096
// 7.2 and 8.6.  With the same weights again and again, which a cache of 256 MB then
// holds: 20.9 and 26.3, 5.5 and 8.2; so are the figures beside the choices below.
//
// More (tile_kernel): x is quantised once into the workspace (4.7 to 5.4 TB/s for many
// rows), then tiles of both go through LDS, a step of 128 columns or more ahead.  A
// matrix instruction takes 32 cycles and the four multiply-adds behind it 16 or more of
// a SIMD's issue, so two waves a SIMD are bound by issue, and by the wait at a step's
// barrier: the cube of 8192 columns 520 us beside the 37 of the quantising, 2.1 PFLOP/s,
// the matrix cores busy for half of the cycles (which are 1.7 GHz then).
#include "rm_common.h"
#include "rm_decode.h"
#include "rm_lds.h"

namespace rm {
namespace {

constexpr int kBlock = 128;

typedef int i32x8 __attribute__((ext_vector_type(8)));

// One block's products of 16 x 16 rows.
__device__ inline f32x4 products(i32x8 w, i32x8 x)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0,
                                                            0);
}

// Two chunks of 16 bytes as one operand.
__device__ inline i32x8 operand(u32x4 lo, u32x4 hi)
{
    return i32x8{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3],
                 (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
}

// The biased exponent of the smallest power of two p, 2^-126 at least, with
// top <= 448 p = 1.75 * 2^8 p; 0 where top is not finite.
__device__ inline int scale_exponent(float top)
{
    if (!(top < INFINITY)) return 0;
    const uint32_t b = __builtin_bit_cast(uint32_t, top);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, 1);
}
__device__ inline float power_of(int biased) { return __builtin_bit_cast(float, biased << 23); }
__device__ inline float scale_from(int e) { return e ? power_of(e) : __builtin_nanf(""); }
// the divisor of the codes; where the scale is NaN they do not count
__device__ inline float divisor_from(int e) { return power_of(e ? e : 127); }

// Largest magnitudes as bits, which are in the numbers' order with infinities and
// NaN above them.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t larger(uint32_t a, uint32_t b)       // of two pairs
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a),
                                                                  __builtin_bit_cast(u16x2, b)));
}
template <typename T>
__device__ inline uint32_t largest8(uint32_t top, typename Vec<T>::x8 v)
{
    const u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) top = larger(top, w[i] & 0x7fff7fffu);
    return top;
}
template <typename T>
__device__ inline float largest_of(uint32_t pair)
{
    const uint16_t top = (uint16_t)max(pair & 0xffffu, pair >> 16);
    return (float)__builtin_bit_cast(T, top);
}
template <int CTRL>
__device__ inline uint32_t dpp_bits(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xF, 0xF, false);
}
// Largest pairs of 16 neighbouring lanes.
__device__ inline uint32_t row16_larger(uint32_t v)
{
    v = larger(v, dpp_bits<0xB1>(v));
    v = larger(v, dpp_bits<0x4E>(v));
    v = larger(v, dpp_bits<0x141>(v));
    return larger(v, dpp_bits<0x140>(v));
}
// Of the four lanes 16 apart, for every lane.
__device__ inline uint32_t rows_larger(uint32_t v)
{
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t h0 = h[0], h1 = h[1], w = larger(h0, h1);
    const auto r = __builtin_amdgcn_permlane16_swap(w, w, false, false);
    const uint32_t r0 = r[0], r1 = r[1];
    return larger(r0, r1);
}

// Codes of eight values by the hardware's conversion, which divides by the power of
// two `scale` and rounds once.
typedef short s16x2 __attribute__((ext_vector_type(2)));
__device__ inline uint32_t codes4(bf16x2 a, bf16x2 b, float scale)
{
    const s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, a, scale, false);
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, b, scale, true));
}
__device__ inline uint32_t codes4(f16x2 a, f16x2 b, float scale)
{
    const s16x2 lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(s16x2{0, 0}, a, scale, false);
    return __builtin_bit_cast(uint32_t,
                              __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(lo, b, scale, true));
}
template <typename T>
__device__ inline u32x2 codes8(typename Vec<T>::x8 v, float scale)
{
    typedef typename Vec<T>::x2 V2;
    return u32x2{codes4(V2{v[0], v[1]}, V2{v[2], v[3]}, scale),
                 codes4(V2{v[4], v[5]}, V2{v[6], v[7]}, scale)};
}

// 16 bytes of codes at any alignment.
__device__ inline u32x4 load16(const uint8_t* p)
{
    typedef u32x4 V __attribute__((aligned(1)));
    return *reinterpret_cast<const V*>(p);
}
// The 16 bytes from byte c on of a row of `size` bytes, zeros behind its end: what the
// end cuts off is the row's last 16 bytes moved down.
__device__ inline u32x4 load16_of(const uint8_t* row, int64_t c, int64_t size)
{
    if (c + 16 <= size) return load16(row + c);
    if (c >= size) return u32x4{0, 0, 0, 0};
    uint64_t lo = 0, hi = 0;
    if (size >= 16) {
        const u32x4 v = load16(row + size - 16);
        const int bits = (int)(c + 16 - size) * 8;        // 8 .. 120
        lo = (uint64_t)v[1] << 32 | v[0];
        hi = (uint64_t)v[3] << 32 | v[2];
        lo = bits < 64 ? lo >> bits | hi << (64 - bits) : hi >> (bits - 64);
        hi = bits < 64 ? hi >> bits : 0;
    } else {
        for (int i = 0; c + i < size; ++i)
            (i < 8 ? lo : hi) |= (uint64_t)row[c + i] << (8 * (i & 7));
    }
    return u32x4{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32)};
}

// ---- codes and scales ------------------------------------------------------

// Blocks of one row: 16 lanes a block, 16 blocks a workgroup.  PACK: codes (zeros
// behind k) and scales block by block, as tile_kernel reads them.
template <typename T, bool PACK>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a, int32_t blocks)
{
    const int t = threadIdx.x & 15;
    const int64_t all = (int64_t)a.rows * blocks, by = (int64_t)gridDim.x * 16;
    for (int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); at < all; at += by) {
        const bool small = all <= 0x7fffffff;       // wave-uniform
        const int64_t row = small ? (uint32_t)at / (uint32_t)blocks : at / blocks;
        const int block = (int)(at - row * blocks), c = block * kBlock + t * 8;
        const typename Vec<T>::x8 v = __builtin_bit_cast(
            typename Vec<T>::x8,
            load16_of(static_cast<const uint8_t*>(a.x) + 2 * row * a.x_stride, 2 * (int64_t)c,
                      2 * (int64_t)a.k));
        const int e = scale_exponent(largest_of<T>(row16_larger(largest8<T>(0, v))));
        const u32x2 code = codes8<T>(v, divisor_from(e));
        uint8_t* out = PACK ? a.codes + ((int64_t)block * a.rows + row) * kBlock + t * 8
                            : a.codes + row * a.code_stride + c;
        typedef u32x2 V __attribute__((aligned(1)));
        if (PACK || c + 8 <= a.k) {
            *reinterpret_cast<V*>(out) = code;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c + i < a.k) out[i] = (uint8_t)(code[i >> 2] >> (8 * (i & 3)));
        }
        if (t == 0) a.scales[PACK ? (int64_t)block * a.rows + row : at] = scale_from(e);
    }
}

// Blocks of 128 rows: a workgroup each, in registers between the read and the write.
template <typename T>
__global__ __launch_bounds__(256) void quantize_square_kernel(QuantizeArgs a, int32_t blocks)
{
    __shared__ uint32_t part[2][4];
    const int t = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int64_t all = ((int64_t)a.rows + kBlock - 1) / kBlock * blocks;
    int turn = 0;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x, turn ^= 1) {
        const int64_t row = at / blocks * kBlock + r0;
        const int c = (int)(at % blocks) * kBlock + t * 8;
        typename Vec<T>::x8 v[8];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row + i * 16;
            v[i] = load_some(static_cast<const T*>(a.x) + r * a.x_stride + c,
                             r < a.rows ? a.k - c : 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = largest8<T>(top, v[i]);
        top = rows_larger(row16_larger(top));
        if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = top;
        __syncthreads();
        top = larger(larger(part[turn][0], part[turn][1]), larger(part[turn][2], part[turn][3]));
        const int e = scale_exponent(largest_of<T>(top));
        const float divisor = divisor_from(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row + i * 16;
            if (r >= a.rows) continue;
            const u32x2 code = codes8<T>(v[i], divisor);
            uint8_t* out = a.codes + r * a.code_stride + c;
            typedef u32x2 V __attribute__((aligned(1)));
            if (c + 8 <= a.k) {
                *reinterpret_cast<V*>(out) = code;
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (c + j < a.k) out[j] = (uint8_t)(code[j >> 2] >> (8 * (j & 3)));
            }
        }
        if (threadIdx.x == 0) a.scales[at] = scale_from(e);
    }
}

// Codes that a caller has, as quantize_kernel packs them: 8 lanes a block.
__global__ __launch_bounds__(256) void pack_kernel(F8Args a, int32_t blocks, uint8_t* codes,
                                                   float* scales)
{
    const int t = threadIdx.x & 7;
    const int64_t all = (int64_t)a.rows * blocks, by = (int64_t)gridDim.x * 32;
    for (int64_t at = (int64_t)blockIdx.x * 32 + (threadIdx.x >> 3); at < all; at += by) {
        const int64_t row = at / blocks;
        const int block = (int)(at - row * blocks), c = block * kBlock + t * 16;
        const u32x4 v = load16_of(static_cast<const uint8_t*>(a.x) + row * a.x_stride, c, a.k);
        const int64_t to = (int64_t)block * a.rows + row;
        *reinterpret_cast<u32x4*>(codes + to * kBlock + t * 16) = v;
        if (t == 0) scales[to] = a.x_scales[at];
    }
}

// ---- rows of the weights ---------------------------------------------------

// Rows of a tile of `height` rows come in two runs of half of it: neighbours, or
// with GATED rows of the gates and of what they gate.
template <bool GATED>
struct Runs {
    int64_t row[2];          // first row of each run
    int64_t last[2];         // the last row that may be read
    int32_t scale[2];        // row of the scales
    __device__ Runs(int64_t tile, int height, int32_t n)
    {
        const int half = height / 2;
        if (GATED) {
            const int64_t j = tile * half, outs = n / 2;
            row[0] = j, row[1] = outs + j;
            last[0] = outs - 1, last[1] = n - 1;
            scale[0] = (int32_t)(min(j, outs - 1) / kBlock);
            scale[1] = (int32_t)((outs + kBlock - 1) / kBlock) + scale[0];
        } else {
            row[0] = tile * height, row[1] = row[0] + half;
            last[0] = last[1] = n - 1;
            scale[0] = (int32_t)(min(row[0], last[0]) / kBlock);
            scale[1] = (int32_t)(min(row[1], last[1]) / kBlock);
        }
    }
};

__device__ inline float silu(float g) { return g / (1.0f + __expf(-g)); }

// ---- few rows --------------------------------------------------------------

// of a workgroup: with 16 28672 x 4096 takes 23.0 us for 20.9, 1 x 4096 x 4096 the same
constexpr int kMostWaves = 8;

// NT x 16 rows of the weights, 16 of x a workgroup.  AHEAD: blocks of weights and of x
// that a wave has in flight.
template <typename T, int NT, int AHEAD, bool GIVEN, bool GATED>
__global__ __launch_bounds__(kMostWaves * 64) void few_kernel(F8Args a, int32_t blocks)
{
    typedef typename Vec<T>::x8 V;
    constexpr int PITCH = NT * 16 + 4;
    __shared__ __align__(16) float part[kMostWaves][16 * PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, li = lane & 15, quad = lane >> 4;
    const Runs<GATED> runs(blockIdx.x, NT * 16, a.n);

    const uint8_t* w[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 16 + li;
        const bool second = r >= NT * 8;          // no index: runs stays in registers
        w[t] = a.codes +
               min((second ? runs.row[1] : runs.row[0]) + r % (NT * 8),
                   second ? runs.last[1] : runs.last[0]) * a.code_stride;
    }
    const int64_t row = min(li, a.rows - 1);
    const uint8_t* x = static_cast<const uint8_t*>(a.x) +
                       row * a.x_stride * (GIVEN ? 1 : 2);
    const float* scale0 = a.scales + (int64_t)runs.scale[0] * blocks;
    const float* scale1 = a.scales + (int64_t)runs.scale[1] * blocks;
    f32x4 acc[NT] = {};

    // a block's weights, x and scales
    constexpr int X = GIVEN ? 2 : 4;
    auto column = [](int64_t c, int h) {          // byte of the h-th load of x
        return GIVEN ? c + h * 64 : 2 * c + h / 2 * 128 + h % 2 * 16;
    };
    struct Block {
        u32x4 w[NT][2], x[X];
        float sx, s0, s1;
    };
    const int whole = a.k / kBlock;
    auto load = [&](int block, Block& b) {
        const int64_t c = block * kBlock + quad * 16;
        if (block < whole) {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) b.w[t][h] = load16(w[t] + c + h * 64);
#pragma unroll
            for (int h = 0; h < X; ++h) b.x[h] = load16(x + column(c, h));
        } else {
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) b.w[t][h] = load16_of(w[t], c + h * 64, a.k);
#pragma unroll
            for (int h = 0; h < X; ++h)
                b.x[h] = load16_of(x, column(c, h), (int64_t)a.k * (GIVEN ? 1 : 2));
        }
        b.sx = GIVEN ? a.x_scales[row * blocks + block] : 0.0f;
        b.s0 = scale0[block];
        b.s1 = GATED || NT > 1 ? scale1[block] : b.s0;
    };
    auto multiply = [&](const Block& b) {
        i32x8 xq;
        float sx = b.sx;
        if (GIVEN) {
            xq = operand(b.x[0], b.x[1]);
        } else {
            uint32_t top = 0;
#pragma unroll
            for (int h = 0; h < 4; ++h)
                top = largest8<T>(top, __builtin_bit_cast(V, b.x[h % X]));
            const int e = scale_exponent(largest_of<T>(rows_larger(top)));
            sx = scale_from(e);
            u32x2 q[4];
#pragma unroll
            for (int h = 0; h < 4; ++h)
                q[h] = codes8<T>(__builtin_bit_cast(V, b.x[h % X]), divisor_from(e));
            xq = operand(u32x4{q[0][0], q[0][1], q[1][0], q[1][1]},
                         u32x4{q[2][0], q[2][1], q[3][0], q[3][1]});
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x4 p = products(operand(b.w[t][0], b.w[t][1]), xq);
            // NT 1: a lane's four outputs are of one run, lanes differ
            const bool second = NT == 1 ? quad >= 2 : t >= NT / 2;
            const float s = sx * (second ? b.s1 : b.s0);
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[t][i] = __builtin_fmaf(p[i], s, acc[t][i]);
        }
    };
    Block b[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
        if (wave + i * waves < blocks) load(wave + i * waves, b[i]);
    for (int block = wave; block < blocks; block += AHEAD * waves) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (block + i * waves >= blocks) break;
            multiply(b[i]);
            const int next = block + (i + AHEAD) * waves;
            if (next < blocks) load(next, b[i]);
        }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
        *reinterpret_cast<f32x4*>(&part[wave][li * PITCH + t * 16 + quad * 4]) = acc[t];
    __syncthreads();
    constexpr int OUT = GATED ? NT * 8 : NT * 16;
    const int64_t outs = GATED ? a.n / 2 : a.n;
    const T* bias = static_cast<const T*>(a.bias);
    for (int i = threadIdx.x; i < a.rows * OUT; i += blockDim.x) {
        const int j = i % OUT, m = i / OUT;
        const int64_t to = runs.row[0] + j;
        if (to >= outs) continue;
        float g = 0.0f, u = 0.0f;
        for (int v = 0; v < waves; ++v) {
            const float* p = &part[v][m * PITCH + j];
            g += p[0];
            if (GATED) u += p[NT * 8];
        }
        if (bias) {
            g += (float)bias[to];
            if (GATED) u += (float)bias[outs + to];
        }
        static_cast<T*>(a.y)[m * a.y_stride + to] = (T)(GATED ? silu(g) * u : g);
    }
}

// ---- many rows -------------------------------------------------------------

// x as quantize_kernel packs it.
struct Packed {
    const uint8_t* codes;       // [blocks][rows][128]
    const float* scales;        // [blocks][rows]
    int32_t blocks;
    uint32_t tiles, tiles_m, first;      // 31 bits: y has a tile's outputs for each
    // The columns of a tile are split over `parts` workgroups, whose totals join_kernel
    // adds.
    uint32_t parts;
    f32x4* join;                // [parts][tiles][TN * TM][threads]
};

// Bytes of a step in LDS: codes of the weights and of x, scales of x and 64 of the
// weights (two a wave, and what the other lanes of their load bring).
constexpr int tile_stage(int weights, int rows) { return (weights + rows) * kBlock + rows * 4 + 256; }

// Bias, activation and the result of a wave's totals: outputs of tile `tile` of TN x 16
// weight rows, rows of x from row0.
template <typename T, int TN, int TM, bool GATED>
__device__ inline void finish(const F8Args& a, int64_t tile, int row0, const f32x4 (&acc)[TN][TM])
{
    const int lane = threadIdx.x & 63, li = lane & 15, quad = lane >> 4;
    const Runs<GATED> runs(tile, TN * 16, a.n);
    const T* bias = static_cast<const T*>(a.bias);
    const int64_t outs = GATED ? a.n / 2 : a.n;
    constexpr int OUT = GATED ? TN / 2 : TN;
#pragma unroll
    for (int t = 0; t < OUT; ++t) {
        const int64_t to = runs.row[0] + t * 16 + quad * 4;
        float b0[4], b1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool there = bias && to + i < outs;
            b0[i] = there ? (float)bias[to + i] : 0.0f;
            b1[i] = there && GATED ? (float)bias[outs + to + i] : 0.0f;
        }
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const int64_t row = (int64_t)row0 + m * 16 + li;
            if (row >= a.rows) continue;
            typedef T V4 __attribute__((ext_vector_type(4)));
            typedef V4 V4u __attribute__((aligned(2)));
            V4 o;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float g = acc[t][m][i] + b0[i];
                o[i] = (T)(GATED ? silu(g) * (acc[(t + TN / 2) % TN][m][i] + b1[i]) : g);
            }
            T* y = static_cast<T*>(a.y) + row * a.y_stride + to;
            if (to + 4 <= outs) {
                *reinterpret_cast<V4u*>(y) = o;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (to + i < outs) y[i] = o[i];
            }
        }
    }
}

// Output tile and row tile of a tile's number: four of x beside each other, so that an
// L2 that is given tiles behind each other holds what they share.
__device__ inline uint2 place_of(uint32_t tile, uint32_t tiles_n, uint32_t tiles_m)
{
    const uint32_t group = tile / (4 * tiles_n), in = tile - group * 4 * tiles_n;
    const uint32_t wide = min(4u, tiles_m - group * 4);
    return make_uint2(in / wide, group * 4 + in % wide);
}

// TN x 16 weight rows and TM x 16 rows of x a wave, WN x WM waves a workgroup.
//
// Both operands pass through LDS, STAGES steps of 128 columns in a ring.  A step has
// one barrier, in front of its last 16 rows of x: what it has read is free then, the
// next step is there, and that one's weights and first rows are read beside the last
// matrix instructions.  A product goes into its total kLag matrix instructions
// behind its own, so that no vector instruction waits for one.
// ALIGNED: weights by 16 bytes at addresses that are multiples of it; they go to LDS
// directly, others through registers.
template <typename T, int WN, int WM, int TN, int TM, int STAGES, bool GATED, bool ALIGNED>
__global__ __launch_bounds__(WN * WM * 64) __attribute__((amdgpu_waves_per_eu(2))) void
tile_kernel(F8Args a, Packed x)
{
    constexpr int WAVES = WN * WM, NB = WN * TN * 16, MB = WM * TM * 16;
    constexpr int W_GROUPS = NB / 8 / WAVES, X_GROUPS = MB / 8 / WAVES;    // of 8 rows
    constexpr int X_AT = NB * kBlock, S_AT = X_AT + MB * kBlock;
    constexpr int STAGE = tile_stage(NB, MB);
    constexpr int LOADS = (ALIGNED ? W_GROUPS : 0) + X_GROUPS + 2;
    static_assert(NB % (8 * WAVES) == 0 && MB % (8 * WAVES) == 0, "groups");
    static_assert((STAGES - 2) * LOADS < 64, "s_waitcnt counts 63 loads");
    extern __shared__ __align__(1024) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, quad = lane >> 4, wn = wave % WN, wm = wave / WN;

    // The XCDs take the workgroups in turn; each gets tiles behind each other.
    const uint32_t all = x.tiles * x.parts, per = (all + 7) / 8, block_at = x.first + blockIdx.x;
    const uint32_t number = block_at % 8 * per + block_at / 8;
    if (block_at / 8 >= per || number >= all) return;
    const uint32_t part = number / x.tiles;
    const uint2 place = place_of(number - part * x.tiles, x.tiles / x.tiles_m, x.tiles_m);
    const int tile_n = __builtin_amdgcn_readfirstlane((int)place.x);
    const int m0 = __builtin_amdgcn_readfirstlane((int)(place.y * MB));
    // its blocks of columns
    const int chunk = (x.blocks + x.parts - 1) / x.parts;
    const int from_step = __builtin_amdgcn_readfirstlane((int)(part * chunk));
    const int end = min(x.blocks, from_step + chunk);

    // Sources of the loads.  A chunk of 16 columns lies at (chunk ^ row) % 8 of its
    // row in LDS, so that the 16 rows of an operand are spread over the banks.
    const int row8 = lane >> 3, column = ((lane & 7) ^ row8) * 16;
    const uint8_t* w_base[W_GROUPS];
    uint32_t w_from[W_GROUPS], x_from[X_GROUPS];
#pragma unroll
    for (int i = 0; i < W_GROUPS; ++i) {
        const int r = (i * WAVES + wave) * 8;             // all 8 in one run
        const Runs<GATED> runs((int64_t)tile_n * WN + r / (TN * 16), TN * 16, a.n);
        const int run = r % (TN * 16) / (TN * 8);
        const int64_t row = min(runs.row[run] + r % (TN * 8), runs.last[run]);
        w_base[i] = scalar(a.codes + row * a.code_stride);
        w_from[i] = (uint32_t)(min((int64_t)row8, runs.last[run] - row) * a.code_stride);
    }
    const uint8_t* x_base = scalar(x.codes + (int64_t)m0 * kBlock);
#pragma unroll
    for (int i = 0; i < X_GROUPS; ++i) {
        const int r = (i * WAVES + wave) * 8 + row8;
        x_from[i] = (uint32_t)(min(r, a.rows - 1 - m0) * kBlock + column);
    }
    // scales: of x's rows, 64 a wave and round again, and two of each wave's weights
    const int s_row = (wave * 64 + lane) % MB;
    const float* xs_base = x.scales + m0 + min(s_row, a.rows - 1 - m0);
    const Runs<GATED> mine((int64_t)tile_n * WN + lane / 2 % WN, TN * 16, a.n);
    const float* ws_base = a.scales + (int64_t)mine.scale[lane & 1] * x.blocks;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_address(lds));

    u32x4 kept[ALIGNED ? 1 : W_GROUPS];
    auto fetch = [&](int step, int stage) {
        const uint32_t to = lds0 + stage * STAGE;
        const int64_t c = (int64_t)step * kBlock, rows_at = (int64_t)step * a.rows;
#pragma unroll
        for (int i = 0; i < X_GROUPS; ++i)
            to_lds16(to + X_AT + (i * WAVES + wave) * 1024, x_from[i], x_base + rows_at * kBlock);
        to_lds4(to + S_AT + wave * 64 % MB * 4, xs_base + rows_at);
        to_lds4(to + S_AT + MB * 4, ws_base + step);
        // behind k the row's last codes again: x is 0 there, and a code that is NaN makes
        // its row's results NaN anyhow
        const uint32_t inside = (uint32_t)min(column, a.k - 16 - (int)c);
#pragma unroll
        for (int i = 0; i < W_GROUPS; ++i) {
            if (ALIGNED) to_lds16(to + (i * WAVES + wave) * 1024, w_from[i] + inside, w_base[i] + c);
            else kept[ALIGNED ? 0 : i] = load16_of(w_base[i] + w_from[i], c + column, a.k);
        }
    };
    auto put = [&](int stage) {
#pragma unroll
        for (int i = 0; i < (ALIGNED ? 0 : W_GROUPS); ++i)
            *reinterpret_cast<u32x4*>(lds + stage * STAGE + (i * WAVES + wave) * 1024 + lane * 16) =
                kept[i];
    };
    const int swizzle0 = li * kBlock + (quad ^ (li & 7)) * 16;
    const int swizzle1 = li * kBlock + ((quad + 4) ^ (li & 7)) * 16;
    auto sixteen = [&](const uint8_t* from) {
        return operand(*reinterpret_cast<const u32x4*>(from + swizzle0),
                       *reinterpret_cast<const u32x4*>(from + swizzle1));
    };
    auto rows_of = [&](int stage, int m, i32x8& v, float& s) {
        const uint8_t* from = lds + stage * STAGE;
        v = sixteen(from + X_AT + (wm * TM + m) * 2048);
        s = *reinterpret_cast<const float*>(from + S_AT + ((wm * TM + m) * 16 + li) * 4);
    };
    i32x8 wq[TN];
    float sw0, sw1;
    auto weights_of = [&](int stage, int t) {
        wq[t] = sixteen(lds + stage * STAGE + (wn * TN + t) * 2048);
    };
    auto weight_scales_of = [&](int stage) {
        const float* s = reinterpret_cast<const float*>(lds + stage * STAGE + S_AT + MB * 4);
        sw0 = s[wn * 2];
        sw1 = GATED ? s[wn * 2 + 1] : sw0;
    };

    constexpr int kLag = TN < 3 ? TN : 3, kRing = 4;
    static_assert(TN * TM % kRing == 0 && kLag < kRing && TM % 2 == 0, "rings");
    f32x4 acc[TN][TM] = {}, p[kRing] = {};
    i32x8 xm[2];
    float sx[2], s0 = 0.0f, s1 = 0.0f;
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        fetch(min(from_step + i, end - 1), i);
        put(i);
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    fetch(min(from_step + STAGES - 1, end - 1), STAGES - 1);
#pragma unroll
    for (int t = 0; t < TN; ++t) weights_of(0, t);
    weight_scales_of(0);
    rows_of(0, 0, xm[0], sx[0]);
    int stage = 0;
    for (int step = from_step; step < end; ++step) {
        const int following = stage == STAGES - 1 ? 0 : stage + 1;
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            if (m == TM - 1) {
                put(stage == 0 ? STAGES - 1 : stage - 1);
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier"
                             :: "n"((STAGES - 2) * LOADS) : "memory");
                // behind the last step the last one again: a branch would part the
                // matrix instructions from what stands between them
                fetch(min(step + STAGES, end - 1), stage);
            }
            rows_of(m + 1 < TM ? stage : following, (m + 1) % TM, xm[(m + 1) & 1], sx[(m + 1) & 1]);
            const float before0 = s0, before1 = s1;
            s0 = sx[m & 1] * sw0, s1 = GATED ? sx[m & 1] * sw1 : s0;
            if (m == TM - 1) weight_scales_of(following);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const int j = m * TN + t, done = (j - kLag + TN * TM) % (TN * TM);
                p[j % kRing] = products(wq[t], xm[m & 1]);
                if (m == TM - 1) weights_of(following, t);
                const float s = done / TN == m ? (done % TN < TN / 2 ? s0 : s1)
                                               : (done % TN < TN / 2 ? before0 : before1);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[done % TN][done / TN][i] = __builtin_fmaf(p[done % kRing][i], s,
                                                                  acc[done % TN][done / TN][i]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        stage = following;
    }
#pragma unroll
    for (int j = TN * TM - kLag; j < TN * TM; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            acc[j % TN][j / TN][i] = __builtin_fmaf(p[j % kRing][i], j % TN < TN / 2 ? s0 : s1,
                                                    acc[j % TN][j / TN][i]);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // LDS is this workgroup's until here

    if (x.parts > 1) {
        f32x4* to = x.join + ((int64_t)number * TN * TM * (WAVES * 64) + threadIdx.x);
#pragma unroll
        for (int j = 0; j < TN * TM; ++j) to[j * (WAVES * 64)] = acc[j % TN][j / TN];
        return;
    }
    finish<T, TN, TM, GATED>(a, (int64_t)tile_n * WN + wn, m0 + wm * TM * 16, acc);
}

// The totals of the parts of a tile, in the parts' order.
template <typename T, int WN, int WM, int TN, int TM, bool GATED>
__global__ __launch_bounds__(WN * WM * 64) void join_kernel(F8Args a, Packed x)
{
    constexpr int THREADS = WN * WM * 64;
    const uint32_t tile = blockIdx.x, tiles_n = x.tiles / x.tiles_m;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m = blockIdx.y;            // of the wave's 16 rows of x
    f32x4 acc[TN][1];
#pragma unroll
    for (int t = 0; t < TN; ++t) acc[t][0] = f32x4{0, 0, 0, 0};
    // four parts in flight; behind the last one the last again, for nothing
    for (uint32_t part = 0; part < x.parts; part += 4) {
        f32x4 v[4][TN];
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i) {
            const int64_t at = (int64_t)min(part + i, x.parts - 1) * x.tiles + tile;
#pragma unroll
            for (int t = 0; t < TN; ++t)
                v[i][t] = x.join[(at * TN * TM + m * TN + t) * THREADS + threadIdx.x];
        }
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < TN; ++t)
                if (part + i < x.parts) acc[t][0] += v[i][t];
    }
    const uint2 place = place_of(tile, tiles_n, x.tiles_m);
    finish<T, TN, 1, GATED>(a, (int64_t)place.x * WN + wave % WN,
                            (int)place.y * (WM * TM * 16) + (wave / WN * TM + m) * 16, acc);
}

// ---- launches --------------------------------------------------------------

// The most rows that few_kernel takes.  Weights from memory, 16 rows and 17 (tile_kernel):
// 4096 x 4096 8.6 and 15.2 us, 28672 x 4096 32.1 and 36.2, 1022 x 5150 12.4 and 17.4,
// 40960 x 4096 45.8 and 65.1.
constexpr int kFewRows = 16;

// tile_kernel counts the bytes of 8 rows of weights in 32 bits
bool few(int32_t rows, int64_t code_stride) { return rows <= kFewRows || code_stride >= 1 << 28; }

int blocks_of(int32_t k) { return (k + kBlock - 1) / kBlock; }

size_t packed_bytes(int32_t rows, int32_t k)
{
    return ((size_t)rows * blocks_of(k) * (kBlock + 4) + 255) / 256 * 256;
}

int64_t tiles_of(int32_t rows, int32_t n, int weights, int height)
{
    return (((int64_t)rows + height - 1) / height) * (((int64_t)n + weights - 1) / weights);
}

// Smaller tiles where larger ones leave a quarter of the card without any, and at last
// their columns in parts of 6 blocks or more.  300 x 1024 x 4096: tiles of 128 weight
// rows 18.0 us, of 64 16.3; 200 x 6144 x 4096 23.2 and 25.6.  40 x 2048 x 11008 took
// 43 us without parts, 25 with them (tiles of 128).
bool fills(int32_t rows, int32_t n, int weights, int height)
{
    return tiles_of(rows, n, weights, height) >= kComputeUnits * 3 / 4;
}
bool middle(int32_t rows, int32_t n) { return rows > 64 && fills(rows, n, 128, 128); }
uint32_t parts_of(int32_t rows, int32_t n, int32_t k)
{
    if (middle(rows, n) || fills(rows, n, 128, 64)) return 1;
    const int64_t fill = kComputeUnits / tiles_of(rows, n, 64, 64), most = blocks_of(k) / 6;
    const int64_t parts = fill < most ? fill : most;
    return parts < 2 ? 1 : (uint32_t)parts;
}

template <typename T, int NT, int AHEAD, bool GIVEN, bool GATED>
hipError_t launch_few_form(const F8Args& a, hipStream_t s)
{
    const int blocks = blocks_of(a.k), waves = blocks < kMostWaves ? blocks : kMostWaves;
    const int64_t tiles = ((int64_t)a.n + NT * 16 - 1) / (NT * 16);
    return launch(few_kernel<T, NT, AHEAD, GIVEN, GATED>, dim3((unsigned)tiles),
                  (unsigned)(waves * 64), 0, s, a, blocks);
}

template <typename T, bool GIVEN, bool GATED>
hipError_t launch_few(const F8Args& a, hipStream_t s)
{
    // 64 weight rows a workgroup where that is one for every CU (1 x 28672 x 4096 21 us,
    // 16 or 32 rows 25 to 27), else 16 (1 x 4096 x 4096 5.5 us, 32 rows 7.1)
    if (a.n >= 64 * kComputeUnits) return launch_few_form<T, 4, 1, GIVEN, GATED>(a, s);
    return launch_few_form<T, 1, 2, GIVEN, GATED>(a, s);
}

template <typename T, int WN, int WM, int TN, int TM, int STAGES, bool SPLIT, bool GATED,
          bool ALIGNED>
hipError_t launch_tiles(const F8Args& a, Packed x, hipStream_t s)
{
    constexpr int MB = WM * TM * 16, NB = WN * TN * 16, THREADS = WN * WM * 64;
    const int64_t tiles = tiles_of(a.rows, a.n, NB, MB);
    x.tiles_m = (uint32_t)(((int64_t)a.rows + MB - 1) / MB);
    x.tiles = (uint32_t)tiles;
    const int64_t all = tiles * x.parts, upto = (all + 7) / 8 * 8;
    if (upto > 0x7fffffff) return hipErrorInvalidConfiguration;
    constexpr size_t lds = (size_t)STAGES * tile_stage(NB, MB);
    auto kernel = tile_kernel<T, WN, WM, TN, TM, STAGES, GATED, ALIGNED>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    const int64_t most = most_blocks(THREADS) / 8 * 8;
    for (int64_t first = 0; first < upto; first += most) {
        x.first = (uint32_t)first;
        const int64_t n = upto - first < most ? upto - first : most;
        const hipError_t e = launch(kernel, dim3((unsigned)n), THREADS, lds, s, a, x);
        if (e != hipSuccess) return e;
    }
    if constexpr (SPLIT)
        if (x.parts > 1)
            return launch(join_kernel<T, WN, WM, TN, TM, GATED>, dim3(x.tiles, TM), THREADS, 0, s, a, x);
    return hipSuccess;
}

template <typename T, bool GATED, bool ALIGNED>
hipError_t launch_sizes(const F8Args& a, const Packed& x, hipStream_t s)
{
    // The largest tiles, a CU each, from nine sixteenths of the card on: 128 of them
    // (2048 x 4096 x 4096) 72 us, in tiles of 128 x 128 65; 160 (2048 x 5120 x 8192) 125
    // and 157.  Registers hold no copy of unaligned weights beside their totals.
    if (ALIGNED && tiles_of(a.rows, a.n, 256, 256) >= kComputeUnits * 9 / 16)
        return launch_tiles<T, 4, 2, 4, 8, 2, false, GATED, true>(a, x, s);
    if (middle(a.rows, a.n)) return launch_tiles<T, 2, 2, 4, 4, 3, false, GATED, ALIGNED>(a, x, s);
    if (fills(a.rows, a.n, 128, 64))
        return launch_tiles<T, 4, 1, 2, 4, 3, false, GATED, ALIGNED>(a, x, s);
    return launch_tiles<T, 2, 1, 2, 4, 3, true, GATED, ALIGNED>(a, x, s);
}

template <typename T, bool GATED>
hipError_t launch_many(const F8Args& a, hipStream_t s)
{
    const int blocks = blocks_of(a.k);
    uint8_t* codes = static_cast<uint8_t*>(a.workspace);
    float* scales = reinterpret_cast<float*>(codes + (size_t)a.rows * blocks * kBlock);
    const int64_t all = (int64_t)a.rows * blocks, most = most_blocks(256);
    hipError_t e;
    if (a.x_scales) {
        const int64_t n = (all + 31) / 32;
        e = launch(pack_kernel, dim3((unsigned)(n < most ? n : most)), 256, 0, s, a, blocks, codes,
                   scales);
    } else {
        const QuantizeArgs q = {a.rows, a.k, a.x, a.x_stride, codes, 0, scales};
        const int64_t n = (all + 15) / 16;
        e = launch(quantize_kernel<T, true>, dim3((unsigned)(n < most ? n : most)), 256, 0, s, q,
                   blocks);
    }
    if (e != hipSuccess) return e;
    Packed x = {};
    x.codes = codes;
    x.scales = scales;
    x.blocks = blocks;
    x.parts = parts_of(a.rows, a.n, a.k);
    x.join = reinterpret_cast<f32x4*>(codes + packed_bytes(a.rows, a.k));
    const bool aligned = ((uintptr_t)a.codes | (uintptr_t)a.code_stride | (uintptr_t)a.k) % 16 == 0;
    return aligned ? launch_sizes<T, GATED, true>(a, x, s) : launch_sizes<T, GATED, false>(a, x, s);
}

// Rows whose strides pass 2^28 go a few at a time.
template <typename T>
hipError_t launch_type(const F8Args& a, hipStream_t s)
{
    const bool gated = a.act == RM_ACT_SWIGLU;
    if (a.rows > kFewRows && few(a.rows, a.code_stride)) {
        for (int32_t r = 0; r < a.rows; r += kFewRows) {
            F8Args b = a;
            b.rows = a.rows - r < kFewRows ? a.rows - r : kFewRows;
            b.x = static_cast<const uint8_t*>(a.x) + r * a.x_stride * (a.x_scales ? 1 : 2);
            if (a.x_scales) b.x_scales = a.x_scales + (int64_t)r * blocks_of(a.k);
            b.y = static_cast<T*>(a.y) + r * a.y_stride;
            const hipError_t e = launch_type<T>(b, s);
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    if (!few(a.rows, a.code_stride)) return gated ? launch_many<T, true>(a, s) : launch_many<T, false>(a, s);
    if (a.x_scales) return gated ? launch_few<T, true, true>(a, s) : launch_few<T, true, false>(a, s);
    return gated ? launch_few<T, false, true>(a, s) : launch_few<T, false, false>(a, s);
}

template <typename T>
hipError_t launch_quantize_type(int block_rows, const QuantizeArgs& a, hipStream_t s)
{
    const int blocks = blocks_of(a.k);
    const int64_t most = most_blocks(256);
    const int64_t n = block_rows == 1 ? ((int64_t)a.rows * blocks + 15) / 16
                                      : ((int64_t)a.rows + kBlock - 1) / kBlock * blocks;
    return launch(block_rows == 1 ? quantize_kernel<T, false> : quantize_square_kernel<T>,
                  dim3((unsigned)(n < most ? n : most)), 256, 0, s, a, blocks);
}

}  // namespace

size_t f8_workspace(int32_t rows, int32_t n, int32_t k, int32_t act)
{
    (void)act;
    if (few(rows, 0)) return 0;
    const uint32_t parts = parts_of(rows, n, k);
    const size_t join = parts > 1 ? (size_t)parts * tiles_of(rows, n, 64, 64) * 64 * 64 * 4 : 0;
    return packed_bytes(rows, k) + join;
}

hipError_t launch_f8(int type, const F8Args& a, hipStream_t s)
{
    return type == RM_TYPE_BF16 ? launch_type<bf16>(a, s) : launch_type<f16>(a, s);
}

hipError_t launch_quantize(int type, int block_rows, const QuantizeArgs& a, hipStream_t s)
{
    return type == RM_TYPE_BF16 ? launch_quantize_type<bf16>(block_rows, a, s)
                                : launch_quantize_type<f16>(block_rows, a, s);
}

}  // namespace rm
