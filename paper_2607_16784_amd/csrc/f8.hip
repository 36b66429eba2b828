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
// Few rows of x (few_kernel): bound by reading the codes once.  The blocks go
// round the waves of a workgroup, x is quantised in the registers of the wave that
// multiplies it, and the waves' totals are joined through LDS.
//
// Many rows (tile_kernel): x is quantised once into the workspace and passes
// through LDS, 64 weight rows a wave straight into registers, both a step of 128
// columns or more ahead.
#include "rm_common.h"
#include "rm_decode.h"

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
// 1 / scale; what is not finite stays so
__device__ inline float inverse_from(int e) { return power_of(254 - (e ? e : 127)); }

__device__ inline uint32_t codes4(float a, float b, float c, float d)
{
    const int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

template <typename T>
__device__ inline u32x2 codes8(typename Vec<T>::x8 v, float inv)
{
    return u32x2{codes4((float)v[0] * inv, (float)v[1] * inv, (float)v[2] * inv, (float)v[3] * inv),
                 codes4((float)v[4] * inv, (float)v[5] * inv, (float)v[6] * inv, (float)v[7] * inv)};
}

template <typename T>
__device__ inline float largest8(float top, typename Vec<T>::x8 v)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) top = MaxNan::of(top, fabsf((float)v[i]));
    return top;
}

// 16 bytes of codes at any alignment.
__device__ inline u32x4 load16(const uint8_t* p)
{
    typedef u32x4 V __attribute__((aligned(1)));
    return *reinterpret_cast<const V*>(p);
}
// The first n (may be <= 0) of 16 codes, zeros behind them.
__device__ inline u32x4 load16_some(const uint8_t* p, int64_t n)
{
    if (n >= 16) return load16(p);
    u32x4 v = {};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) v[i >> 2] |= (uint32_t)p[i] << (8 * (i & 3));
    return v;
}

// ---- codes and scales ------------------------------------------------------

// Largest of 16 neighbouring lanes.
__device__ inline float row16_max(float v)
{
    v = MaxNan::of(v, dpp_float<0xB1>(v));
    v = MaxNan::of(v, dpp_float<0x4E>(v));
    v = MaxNan::of(v, dpp_float<0x141>(v));
    return MaxNan::of(v, dpp_float<0x140>(v));
}

// Blocks of one row: 16 lanes a block, 16 blocks a workgroup.  PACK: rows of whole
// blocks (zeros behind k) and scales block by block, as tile_kernel reads them.
template <typename T, bool PACK>
__global__ __launch_bounds__(256) void quantize_kernel(QuantizeArgs a, int32_t blocks)
{
    const int t = threadIdx.x & 15;
    const int64_t all = (int64_t)a.rows * blocks, by = (int64_t)gridDim.x * 16;
    for (int64_t at = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4); at < all; at += by) {
        const bool small = all <= 0x7fffffff;       // wave-uniform
        const int64_t row = small ? (uint32_t)at / (uint32_t)blocks : at / blocks;
        const int block = (int)(at - row * blocks), c = block * kBlock + t * 8;
        const typename Vec<T>::x8 v =
            load_some(static_cast<const T*>(a.x) + row * a.x_stride + c, a.k - c);
        const int e = scale_exponent(row16_max(largest8<T>(0.0f, v)));
        const u32x2 code = codes8<T>(v, inverse_from(e));
        uint8_t* out = a.codes + row * a.code_stride + c;
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
    __shared__ float part[2][4];
    const int t = threadIdx.x & 15, r0 = threadIdx.x >> 4;
    const int64_t all = ((int64_t)a.rows + kBlock - 1) / kBlock * blocks;
    int turn = 0;
    for (int64_t at = blockIdx.x; at < all; at += gridDim.x, turn ^= 1) {
        const int64_t row = at / blocks * kBlock + r0;
        const int c = (int)(at % blocks) * kBlock + t * 8;
        typename Vec<T>::x8 v[8];
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row + i * 16;
            v[i] = load_some(static_cast<const T*>(a.x) + r * a.x_stride + c,
                             r < a.rows ? a.k - c : 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = largest8<T>(top, v[i]);
        top = wave_reduce<MaxNan>(top);
        if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = top;
        __syncthreads();
        top = MaxNan::of(MaxNan::of(part[turn][0], part[turn][1]),
                         MaxNan::of(part[turn][2], part[turn][3]));
        const int e = scale_exponent(top);
        const float inv = inverse_from(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int64_t r = row + i * 16;
            if (r >= a.rows) continue;
            const u32x2 code = codes8<T>(v[i], inv);
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
        const u32x4 v = load16_some(static_cast<const uint8_t*>(a.x) + row * a.x_stride + c,
                                    a.k - c);
        *reinterpret_cast<u32x4*>(codes + row * (int64_t)blocks * kBlock + c) = v;
        if (t == 0) scales[(int64_t)block * a.rows + row] = a.x_scales[at];
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

// The most waves of a workgroup: totals of a wave are NT x MT x 1 KB of LDS.
constexpr int few_waves(int nt, int mt) { return nt * mt >= 8 ? 4 : nt * mt >= 4 ? 8 : 16; }

// NT x 16 rows of the weights and MT x 16 of x a workgroup.
template <typename T, int NT, int MT, bool GIVEN, bool GATED>
__global__ __launch_bounds__(few_waves(NT, MT) * 64) void few_kernel(F8Args a, int32_t blocks)
{
    typedef typename Vec<T>::x8 V;
    extern __shared__ __align__(16) float part[];      // [waves][MT * 16][NT * 16 + 4]
    constexpr int PITCH = NT * 16 + 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int waves = blockDim.x >> 6, li = lane & 15, quad = lane >> 4;
    const int64_t tile = blockIdx.x;
    const int m0 = blockIdx.y * (MT * 16);
    const Runs<GATED> runs(tile, NT * 16, a.n);

    const uint8_t* w[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int r = t * 16 + li, run = r / (NT * 8);
        w[t] = a.codes + min(runs.row[run] + r % (NT * 8), runs.last[run]) * a.code_stride;
    }
    int64_t row[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) row[t] = min(m0 + t * 16 + li, a.rows - 1);
    f32x4 acc[NT][MT] = {};

    auto load_w = [&](int block, u32x4 (&v)[NT][2]) {
        const int c = block * kBlock + quad * 16;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int at = c + h * 64;
                v[t][h] = (block + 1) * kBlock <= a.k ? load16(w[t] + at)
                                                      : load16_some(w[t] + at, a.k - at);
            }
    };
    u32x4 now[NT][2], next[NT][2];
    if (wave < blocks) load_w(wave, now);
    for (int block = wave; block < blocks; block += waves) {
        if (block + waves < blocks) load_w(block + waves, next);
        const float s0 = a.scales[(int64_t)runs.scale[0] * blocks + block];
        const float s1 = a.scales[(int64_t)runs.scale[1] * blocks + block];
        const int c = block * kBlock + quad * 16;
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            i32x8 x;
            float sx;
            if (GIVEN) {
                const uint8_t* p = static_cast<const uint8_t*>(a.x) + row[m] * a.x_stride + c;
                sx = a.x_scales[row[m] * blocks + block];
                x = operand(load16_some(p, a.k - c), load16_some(p + 64, a.k - c - 64));
            } else {
                const T* p = static_cast<const T*>(a.x) + row[m] * a.x_stride + c;
                V v[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    const int off = (h >> 1) * 64 + (h & 1) * 8;
                    v[h] = load_some(p + off, a.k - c - off);
                }
                float top = 0.0f;
#pragma unroll
                for (int h = 0; h < 4; ++h) top = largest8<T>(top, v[h]);
                const int e = scale_exponent(rows_reduce<MaxNan>(top));
                const float inv = inverse_from(e);
                sx = scale_from(e);
                u32x2 q[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) q[h] = codes8<T>(v[h], inv);
                x = operand(u32x4{q[0][0], q[0][1], q[1][0], q[1][1]},
                            u32x4{q[2][0], q[2][1], q[3][0], q[3][1]});
            }
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const f32x4 p = products(operand(now[t][0], now[t][1]), x);
                // NT 1: a lane's four outputs are of one run, lanes differ
                const bool second = NT == 1 ? quad >= 2 : t >= NT / 2;
                const float s = sx * (second ? s1 : s0);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][m][i] = __builtin_fmaf(p[i], s, acc[t][m][i]);
            }
        }
#pragma unroll
        for (int t = 0; t < NT; ++t) now[t][0] = next[t][0], now[t][1] = next[t][1];
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            *reinterpret_cast<f32x4*>(part + ((size_t)wave * MT * 16 + m * 16 + li) * PITCH +
                                      t * 16 + quad * 4) = acc[t][m];
    __syncthreads();
    constexpr int OUT = GATED ? NT * 8 : NT * 16;
    const int64_t outs = GATED ? a.n / 2 : a.n;
    const T* bias = static_cast<const T*>(a.bias);
    for (int i = threadIdx.x; i < MT * 16 * OUT; i += blockDim.x) {
        const int j = i % OUT, m = i / OUT;
        const int64_t to = runs.row[0] + j;
        if (m0 + m >= a.rows || to >= outs) continue;
        float g = 0.0f, u = 0.0f;
        for (int v = 0; v < waves; ++v) {
            const float* p = part + ((size_t)v * MT * 16 + m) * PITCH + j;
            g += p[0];
            if (GATED) u += p[NT * 8];
        }
        if (bias) {
            g += (float)bias[to];
            if (GATED) u += (float)bias[outs + to];
        }
        static_cast<T*>(a.y)[(int64_t)(m0 + m) * a.y_stride + to] = (T)(GATED ? silu(g) * u : g);
    }
}

// ---- many rows -------------------------------------------------------------

constexpr int kWaves = 4;       // of a tile, side by side along the outputs

// x as quantize_kernel packs it.
struct Packed {
    const uint8_t* codes;       // [rows][blocks * 128]
    const float* scales;        // [blocks][rows]
    int32_t blocks;
    int64_t tiles, tiles_m, first;
};

// 16 bytes a lane from base + offset to LDS, lane by lane behind each other.  Not
// the builtin: the compiler would wait for all of it before the next read of LDS.
// m0 is a register that the compiler sets only beside its use.
__device__ inline void to_lds16(uint32_t lds, uint32_t offset, const uint8_t* base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ inline void to_lds4(uint32_t lds, uint32_t offset, const void* base)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2"
                 :: "s"(lds), "v"(offset), "s"(base) : "memory");
}
__device__ inline uint32_t lds_address(const void* p)
{
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// TN x 16 weight rows a wave, TM x 16 rows of x a workgroup, SETS steps in flight.
template <typename T, int TN, int TM, int SETS, bool GATED>
__global__ __launch_bounds__(kWaves * 64) void tile_kernel(F8Args a, Packed x)
{
    constexpr int MB = TM * 16, STAGE = MB * kBlock, GROUPS = MB / 8 / kWaves;
    extern __shared__ __align__(1024) uint8_t lds[];          // [SETS][STAGE], [SETS][MB] scales
    float* lds_scales = reinterpret_cast<float*>(lds + SETS * STAGE);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int li = lane & 15, quad = lane >> 4;

    // The XCDs take the workgroups in turn; each gets tiles behind each other, four
    // of x beside each other, so that its L2 holds what they share.
    const int64_t per = (x.tiles + 7) / 8, block_at = x.first + blockIdx.x;
    const int64_t at = block_at % 8 * per + block_at / 8;
    if (block_at / 8 >= per || at >= x.tiles) return;
    const int64_t tiles_n = x.tiles / x.tiles_m, group = at / (4 * tiles_n);
    const int64_t wide = min((int64_t)4, x.tiles_m - group * 4), in = at - group * 4 * tiles_n;
    const int64_t m0 = (group * 4 + in % wide) * MB;
    const Runs<GATED> runs(in / wide * kWaves + wave, TN * 16, a.n);

    const uint8_t* w[TN];
#pragma unroll
    for (int t = 0; t < TN; ++t) {
        const int r = t * 16 + li, run = t >= TN / 2;
        w[t] = a.codes + min(runs.row[run] + r % (TN * 8), runs.last[run]) * a.code_stride +
               quad * 16;
    }
    const float* scale0 = a.scales + (int64_t)runs.scale[0] * x.blocks;
    const float* scale1 = a.scales + (int64_t)runs.scale[1] * x.blocks;
    // a chunk of 16 columns lies at (chunk ^ row) % 8 of its row in LDS, so that the
    // 16 rows of an operand are spread over the banks
    const int64_t pitch = (int64_t)x.blocks * kBlock;
    const uint8_t* x_base = x.codes + m0 * pitch;
    const float* s_base = x.scales + m0;
    uint32_t from[GROUPS];
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
        const int r = (i * kWaves + wave) * 8 + (lane >> 3);
        from[i] = (uint32_t)(min((int64_t)r, a.rows - 1 - m0) * pitch) +
                  (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
    }
    const int s_row = wave * 64 % MB + lane;
    const uint32_t s_from = (uint32_t)min((int64_t)(s_row % MB), a.rows - 1 - m0) * 4;
    const uint32_t x_lds = __builtin_amdgcn_readfirstlane(lds_address(lds));
    const uint32_t s_lds = __builtin_amdgcn_readfirstlane(lds_address(lds_scales));

    u32x4 wq[SETS][TN][2];
    float sw0[SETS], sw1[SETS];
    auto fetch = [&](int step, int set) {
        const uint8_t* base = x_base + (int64_t)step * kBlock;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i)
            to_lds16(x_lds + set * STAGE + (i * kWaves + wave) * 1024, from[i], base);
        to_lds4(s_lds + set * (MB * 4) + wave * 64 % MB * 4, s_from,
                s_base + (int64_t)step * a.rows);
        const int c = step * kBlock;
        if (c + kBlock <= a.k) {
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) wq[set][t][h] = load16(w[t] + c + h * 64);
        } else {
#pragma unroll
            for (int t = 0; t < TN; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    wq[set][t][h] = load16_some(w[t] + c + h * 64, a.k - c - quad * 16 - h * 64);
        }
        sw0[set] = scale0[step];
        sw1[set] = scale1[step];
    };
    f32x4 acc[TN][TM] = {};
    const int swizzle0 = (quad ^ (li & 7)) * 16, swizzle1 = ((quad + 4) ^ (li & 7)) * 16;
    auto multiply = [&](int set) {
        const uint8_t* stage = lds + set * STAGE + li * kBlock;
        const float* scales = lds_scales + set * MB + li;
#pragma unroll
        for (int m = 0; m < TM; ++m) {
            const u32x4 lo = *reinterpret_cast<const u32x4*>(stage + m * 16 * kBlock + swizzle0);
            const u32x4 hi = *reinterpret_cast<const u32x4*>(stage + m * 16 * kBlock + swizzle1);
            const float sx = scales[m * 16], s0 = sx * sw0[set], s1 = sx * sw1[set];
            const i32x8 xm = operand(lo, hi);
#pragma unroll
            for (int t = 0; t < TN; ++t) {
                const f32x4 p = products(operand(wq[set][t][0], wq[set][t][1]), xm);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    acc[t][m][i] = __builtin_fmaf(p[i], t < TN / 2 ? s0 : s1, acc[t][m][i]);
            }
        }
    };
    // In flight before a step: SETS - 1 steps of GROUPS + 1 + 2 TN loads; the oldest
    // has to be there, and what the step before has read may be overwritten behind
    // the barrier.
    constexpr int LOADS = GROUPS + 1 + 2 * TN, AHEAD = (SETS - 2) * LOADS;
    static_assert(AHEAD < 64, "s_waitcnt counts 63 loads");
#pragma unroll
    for (int i = 0; i < SETS - 1; ++i)
        if (i < x.blocks) fetch(i, i);
    for (int step = 0; step < x.blocks; step += SETS) {
#pragma unroll
        for (int set = 0; set < SETS; ++set) {
            if (step + set >= x.blocks) break;
            // behind the last fetch fewer are in flight
            if (AHEAD > 0 && step + set + SETS - 1 <= x.blocks)
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" :: "n"(AHEAD) : "memory");
            else
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (step + set + SETS - 1 < x.blocks)
                fetch(step + set + SETS - 1, (set + SETS - 1) % SETS);
            multiply(set);
        }
    }

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
            const int64_t row = m0 + m * 16 + li;
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

// ---- launches --------------------------------------------------------------

constexpr int kFewRows = 64;       // the most rows that few_kernel takes

int blocks_of(int32_t k) { return (k + kBlock - 1) / kBlock; }

template <typename T, int NT, int MT, bool GIVEN, bool GATED>
hipError_t launch_few_form(const F8Args& a, hipStream_t s)
{
    const int blocks = blocks_of(a.k), most = few_waves(NT, MT), waves = blocks < most ? blocks : most;
    const int64_t tiles = (a.n + NT * 16 - 1) / (NT * 16);
    const size_t lds = (size_t)waves * MT * 16 * (NT * 16 + 4) * 4;
    auto kernel = few_kernel<T, NT, MT, GIVEN, GATED>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    const int32_t rows = (a.rows + MT * 16 - 1) / (MT * 16);
    return launch(kernel, dim3((unsigned)tiles, (unsigned)rows), (unsigned)(waves * 64), lds, s, a,
                  blocks);
}

template <typename T, int MT, bool GIVEN, bool GATED>
hipError_t launch_few_rows(const F8Args& a, hipStream_t s)
{
    if (a.n >= 64 * 2 * kComputeUnits) return launch_few_form<T, 4, MT, GIVEN, GATED>(a, s);
    if (a.n >= 32 * 2 * kComputeUnits) return launch_few_form<T, 2, MT, GIVEN, GATED>(a, s);
    return launch_few_form<T, 1, MT, GIVEN, GATED>(a, s);
}

template <typename T, bool GIVEN, bool GATED>
hipError_t launch_few(const F8Args& a, hipStream_t s)
{
    if (a.rows <= 16) return launch_few_rows<T, 1, GIVEN, GATED>(a, s);
    if (a.rows <= 32) return launch_few_rows<T, 2, GIVEN, GATED>(a, s);
    return launch_few_rows<T, 4, GIVEN, GATED>(a, s);
}

template <typename T, int TN, int TM, int SETS, bool GATED>
hipError_t launch_tiles(const F8Args& a, Packed x, hipStream_t s)
{
    constexpr int MB = TM * 16, NB = kWaves * TN * 16;
    x.tiles_m = ((int64_t)a.rows + MB - 1) / MB;
    x.tiles = x.tiles_m * (((int64_t)a.n + NB - 1) / NB);
    const size_t lds = (size_t)SETS * MB * (kBlock + 4);
    auto kernel = tile_kernel<T, TN, TM, SETS, GATED>;
    if (lds > 65536) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    const int64_t all = (x.tiles + 7) / 8 * 8, most = most_blocks(kWaves * 64) / 8 * 8;
    for (x.first = 0; x.first < all; x.first += most) {
        const int64_t n = all - x.first < most ? all - x.first : most;
        const hipError_t e = launch(kernel, dim3((unsigned)n), kWaves * 64, lds, s, a, x);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename T, bool GATED>
hipError_t launch_many(const F8Args& a, hipStream_t s)
{
    const int blocks = blocks_of(a.k);
    uint8_t* codes = static_cast<uint8_t*>(a.workspace);
    const size_t size = ((size_t)a.rows * blocks * kBlock + 255) / 256 * 256;
    float* scales = reinterpret_cast<float*>(codes + size);
    const int64_t all = (int64_t)a.rows * blocks, most = most_blocks(256);
    hipError_t e;
    if (a.x_scales) {
        const int64_t n = (all + 31) / 32;
        e = launch(pack_kernel, dim3((unsigned)(n < most ? n : most)), 256, 0, s, a, blocks, codes,
                   scales);
    } else {
        const QuantizeArgs q = {a.rows, a.k, a.x, a.x_stride, codes, (int64_t)blocks * kBlock,
                                scales};
        const int64_t n = (all + 15) / 16;
        e = launch(quantize_kernel<T, true>, dim3((unsigned)(n < most ? n : most)), 256, 0, s, q,
                   blocks);
    }
    if (e != hipSuccess) return e;
    const Packed x = {codes, scales, blocks, 0, 0, 0};
    const int64_t middle = (((int64_t)a.rows + 127) / 128) * (((int64_t)a.n + 255) / 256);
    if (middle >= kComputeUnits) return launch_tiles<T, 4, 8, 2, GATED>(a, x, s);
    return launch_tiles<T, 2, 4, 4, GATED>(a, x, s);
}

template <typename T>
hipError_t launch_type(const F8Args& a, hipStream_t s)
{
    const bool gated = a.act == RM_ACT_SWIGLU;
    if (a.rows > kFewRows) return gated ? launch_many<T, true>(a, s) : launch_many<T, false>(a, s);
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
    (void)n, (void)act;
    if (rows <= kFewRows) return 0;
    const size_t blocks = (size_t)blocks_of(k);
    return ((size_t)rows * blocks * kBlock + 255) / 256 * 256 + (size_t)rows * blocks * 4;
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
