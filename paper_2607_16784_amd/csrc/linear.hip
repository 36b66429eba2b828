// linear.hip -- projection with 4-bit weights and group scales (rm_w4_linear).
//
// y = x W^T on the matrix cores, 16 rows of x by 16 rows of W a tile
// (v_mfma_f32_16x16x32).  With one to some tens of rows of x the kernel is
// bound by reading the codes once, so everything serves that: the codes are
// read as they are, row by row, 16 bytes a lane, and expanded in registers.
//
// Expansion, by the usual exact conversion of small integers through a fixed
// exponent (Kim et al. 2022): two codes sit 4 nibbles apart in a word, so (w >> 4s) & 0x000f000f
// is the pair (s, s+4) in the low bits of two 16-bit numbers, and OR-ing an
// exponent makes it (128 + code) * 2^-15 (bf16) or 1024 + code (f16), exactly.  x is
// put into the same order 0 4 1 5 2 6 3 7.  f16 then subtracts 1024 + zero (exact).
// bf16 has no packed addition: the product is taken with 128 + code and
// (128 + zero) * (sum of x) is subtracted from each group's fp32 sum, so partial
// sums are up to 143 times the terms: in fp32 still 2^8 finer than the output's
// rounding.  The 2^-15 keeps the sum over a group of the largest bf16 numbers
// finite; 2^5 of it come off with the group's scale, 2^10 with the bias, so that
// neither end of fp32 costs a result that bf16 holds.  Both keep the code exact;
// the group's scale multiplies the fp32 sum.
//
// What costs next to the codes is the number of vector memory accesses, not
// their bytes: an operand's 16 rows are 64 accesses of 16 bytes an instruction,
// about one a clock, and a scale read by every lane costs as much as 16 codes.
// So x and the scales pass through LDS, read once a workgroup with neighbouring
// lanes on neighbouring addresses (16 x 28672 x 4096 gated: 39 us with both read
// by each lane, 20 so; 1 x 28672 x 8192: 40 and 26 us = 4.7 TB/s).
#include "rm_decode.h"

namespace rm {
namespace {

__device__ inline f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline f32x4 mfma(f16x8 a, f16x8 b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

constexpr size_t kMostLds = 144 * 1024;

// The codes of columns at .. at+31 of one row, no byte read behind its end.
__device__ inline u32x4 load_codes(const uint8_t* row, int32_t at, int32_t row_bytes)
{
    typedef u32x4 V __attribute__((aligned(1)));
    const int32_t byte = at >> 1;
    if (byte + 16 <= row_bytes) return *reinterpret_cast<const V*>(row + byte);
    u32x4 r = {0, 0, 0, 0};
    for (int i = 0; i < 16; ++i)
        if (byte + i < row_bytes) r[i >> 2] |= (uint32_t)row[byte + i] << (8 * (i & 3));
    return r;
}

// 4x4 transpose of words between the four 16-lane rows of a wave: afterwards
// lane row q's word j is what lane row j held as word q.
__device__ inline u32x4 transpose_rows(u32x4 w)
{
    const auto a = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
    const auto c = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto d = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return u32x4{c[0], c[1], d[0], d[1]};
}

// x in the order of the expanded codes.
template <typename V>
__device__ inline V order(V x)
{
    const u32x4 w = __builtin_bit_cast(u32x4, x);
    return __builtin_bit_cast(V, u32x4{__builtin_amdgcn_perm(w[2], w[0], 0x05040100),
                                       __builtin_amdgcn_perm(w[2], w[0], 0x07060302),
                                       __builtin_amdgcn_perm(w[3], w[1], 0x05040100),
                                       __builtin_amdgcn_perm(w[3], w[1], 0x07060302)});
}

// The mask and the exponent in registers: v_and_or_b32 takes no literal.
struct Expander {
    uint32_t mask, exponent;
    __device__ Expander(uint32_t e) : mask(0x000f000fu), exponent(e)
    {
        asm("" : "+s"(mask));
        asm("" : "+v"(exponent));
    }
    __device__ uint32_t pair(uint32_t w) const { return (w & mask) | exponent; }
};

__device__ inline bf16x8 expand(const Expander& x, uint32_t w, bf16x2)
{
    return __builtin_bit_cast(bf16x8, u32x4{x.pair(w), x.pair(w >> 4), x.pair(w >> 8),
                                            x.pair(w >> 12)});
}
__device__ inline f16x8 expand(const Expander& x, uint32_t w, f16x2 zero)
{
    u32x4 r;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const f16x2 p = __builtin_bit_cast(f16x2, x.pair(w >> (4 * s)));
        r[s] = __builtin_bit_cast(uint32_t, (f16x2)(p - zero));
    }
    return __builtin_bit_cast(f16x8, r);
}

template <int ACT>
__device__ inline float finish(float t, float other)
{
    return ACT == RM_ACT_SWIGLU ? t / (1.0f + expf(-t)) * other : t;
}

// Unit of the accumulators.
template <typename T> constexpr float kUnit = __is_same(T, f16) ? 1.0f : 0x1p10f;

constexpr int kStep = 128;    // columns of a step: 16 bytes of codes a lane

// Shape of a workgroup.  RG waves side by side, each with 16 R rows of W, and
// KP such groups that share the columns; 16 M rows of x.  PER matrix
// instructions of 32 columns share a group of W.
template <typename T, int R_, int M_, int PER_, int ACT_, int U_, int RG_, int KP_>
struct Shape {
    typedef T type;
    static constexpr int R = R_, M = M_, PER = PER_, ACT = ACT_, U = U_, RG = RG_, KP = KP_;
    static constexpr bool HALF = __is_same(T, f16);
    static constexpr bool NATURAL = PER < 4;        // an instruction's columns are neighbours
    static constexpr int NP = 4 / PER;              // groups a step
    static constexpr int HALVES = ACT == RM_ACT_SWIGLU ? 2 : 1, HR = R / HALVES;
    static constexpr int WAVES = RG * KP, THREADS = WAVES * 64;
    static constexpr int ROWS = RG * R * 16;        // of W
    static constexpr int BATCH = U * kStep;         // columns a wave takes at a time
    static constexpr int SUMS = HALF ? 0 : 16 * M;  // sums of x a group (bf16 only)
};

// A tile's accumulators and the arithmetic of one step.
template <class S>
struct Tile {
    typedef typename S::type T;
    typedef typename Vec<T>::x8 V;
    f32x4 acc[S::R][S::M];
    Expander expander;

    __device__ Tile() : expander(S::HALF ? 0x64006400u : 0x3b803b80u)
    {
#pragma unroll
        for (int r = 0; r < S::R; ++r)
#pragma unroll
            for (int m = 0; m < S::M; ++m) acc[r][m] = f32x4{0, 0, 0, 0};
    }

    // x_of(m, j) in the expanded order, sum_of(p, m) in units of 2^7; group_of(p, r): the
    // scale's bits below, the zero above
    template <class X, class Sum, class Group>
    __device__ inline void step(X x_of, Sum sum_of, u32x4 (&w)[S::R], Group group_of)
    {
        if (S::NATURAL) {
#pragma unroll
            for (int r = 0; r < S::R; ++r) w[r] = transpose_rows(w[r]);
        }
#pragma unroll
        for (int p = 0; p < S::NP; ++p) {
            f32x4 part[S::R][S::M];
            float scale[S::R], z[S::R];
#pragma unroll
            for (int r = 0; r < S::R; ++r) {
                const uint32_t g = group_of(p, r);
                scale[r] = (float)__builtin_bit_cast(T, (uint16_t)g);
                z[r] = (float)(g >> 16);
#pragma unroll
                for (int m = 0; m < S::M; ++m) part[r][m] = f32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int j = p * S::PER; j < (p + 1) * S::PER; ++j) {
                V x[S::M];
#pragma unroll
                for (int m = 0; m < S::M; ++m) x[m] = x_of(m, j);
#pragma unroll
                for (int r = 0; r < S::R; ++r) {
                    typename Vec<T>::x2 zero;
                    zero[0] = zero[1] = (T)(1024.0f + z[r]);
                    const V e = expand(expander, w[r][j], zero);
#pragma unroll
                    for (int m = 0; m < S::M; ++m) part[r][m] = mfma(x[m], e, part[r][m]);
                }
            }
#pragma unroll
            for (int m = 0; m < S::M; ++m) {
                f32x4 sum = {0, 0, 0, 0};
                if (!S::HALF) sum = sum_of(p, m);
#pragma unroll
                for (int r = 0; r < S::R; ++r) {
                    const float bias = __builtin_fmaf(z[r], -0x1p-8f, -0.5f);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float q = S::HALF ? part[r][m][i]
                                                : __builtin_fmaf(bias, sum[i], part[r][m][i]);
                        acc[r][m][i] = __builtin_fmaf(scale[r], q, acc[r][m][i]);
                    }
                }
            }
        }
    }
};

// What a workgroup stages in LDS of a stretch of `cols` columns: x [rows][cols +
// 8] in the expanded order, its sums [cols / (32 PER)][16 M] and the groups'
// scales and zeros [groups][ROWS].  A pitch is 16 bytes off a row of banks.
template <class S>
struct Stage {
    char* x;
    float* sums;
    uint32_t* table;
    int pitch;

    __host__ __device__ static size_t x_bytes(int rows, int cols)
    {
        return (size_t)rows * (cols + 8) * 2;
    }
    __host__ __device__ static size_t bytes(int rows, int cols, int groups)
    {
        return x_bytes(rows, cols) + (size_t)(cols / (32 * S::PER)) * S::SUMS * 4 +
               (size_t)groups * S::ROWS * 4;
    }
    __device__ Stage(char* at, int rows, int cols)
        : x(at), sums(reinterpret_cast<float*>(at + x_bytes(rows, cols))),
          table(reinterpret_cast<uint32_t*>(sums + cols / (32 * S::PER) * S::SUMS)), pitch(cols + 8)
    {
    }
    // 8 columns of x from `at` on; the 4 PER threads of a group are neighbours
    __device__ inline void put(int row, int at, typename Vec<typename S::type>::x8 v) const
    {
        *reinterpret_cast<typename Vec<typename S::type>::x8*>(x + ((size_t)row * pitch + at) * 2) =
            order(v);
        if (!S::HALF) {
            float s = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) s = __builtin_fmaf((float)v[k], 0x1p-7f, s);
            s += dpp_float<0xB1>(s);
            s += dpp_float<0x4E>(s);
            if (S::PER >= 2) s += dpp_float<0x141>(s);
            if (S::PER >= 4) s += dpp_float<0x140>(s);
            if (at % (32 * S::PER) == 0) sums[at / (32 * S::PER) * S::SUMS + row] = s;
        }
    }
    // the step from column `col` of the stretch on, whose group p has number g0 + p
    // in the table (group_at(p))
    template <class Group>
    __device__ inline void take(Tile<S>& tile, u32x4 (&w)[S::R], int rows, int col, int rg,
                                Group group_at) const
    {
        const int li = threadIdx.x & 15, quad = (threadIdx.x & 63) >> 4;
        tile.step(
            [&](int m, int j) {
                return *reinterpret_cast<const typename Tile<S>::V*>(
                    x + ((size_t)min(m * 16 + li, rows - 1) * pitch + col +
                         (S::NATURAL ? j * 32 + quad * 8 : quad * 32 + j * 8)) * 2);
            },
            [&](int p, int m) {
                return reinterpret_cast<const f32x4*>(
                    sums)[(col / (32 * S::PER) + p) * (4 * S::M) + m * 4 + quad];
            },
            w,
            [&](int p, int r) { return table[group_at(p) * S::ROWS + (rg * S::R + r) * 16 + li]; });
    }
};

// Row of W that row `local` of the workgroup stands for: under SWIGLU a wave's
// first tiles are gates, its others the rows they multiply.
template <class S>
__device__ inline int64_t row_of(const LinearArgs& a, int local)
{
    const int out_n = a.n / S::HALVES;
    const int rg = local / (16 * S::R), r = local / 16 % S::R;
    const int j = (blockIdx.x * S::RG + rg) * (16 * S::HR) + (r % S::HR) * 16 + local % 16;
    return min(j, out_n - 1) + (r / S::HR) * out_n;
}

// Group of column k: k / a.group by the reciprocal of the group's 32s.
__device__ inline int group_of(const LinearArgs& a, int k)
{
    return a.inverse ? (int)__umulhi((uint32_t)k >> 5, a.inverse) : k >> 5;
}

template <class S>
__device__ inline uint32_t group_word(const LinearArgs& a, int64_t row, int g)
{
    const int groups = (a.k + a.group - 1) / a.group;
    typedef typename S::type T;
    T s = static_cast<const T*>(a.scales)[row * groups + g];
    if (!S::HALF) s = (T)((float)s * 32.0f);       // exact
    const uint32_t scale = __builtin_bit_cast(uint16_t, s);
    return scale | (a.zeros ? (uint32_t)a.zeros[row * groups + g] : 8u) << 16;
}

// The steps from `first` on, every `by`-th up to the row's end, x straight from
// memory: what no whole batch covers.
template <class S>
__device__ inline void rest(const LinearArgs& a, Tile<S>& tile, int rg, int m0, int rows, int first,
                            int by)
{
    typedef typename S::type T;
    typedef typename Vec<T>::x8 V;
    const int li = threadIdx.x & 15, quad = (threadIdx.x & 63) >> 4;
    const int steps = (a.k + kStep - 1) / kStep, row_bytes = (a.k + 1) / 2;
    const int groups = (a.k + a.group - 1) / a.group;
    for (int step = first; step < steps; step += by) {
        const int k0 = step * kStep;
        u32x4 w[S::R];
        V x[S::M][4], units;
#pragma unroll
        for (int r = 0; r < S::R; ++r)
            w[r] = load_codes(a.codes + row_of<S>(a, (rg * S::R + r) * 16 + li) * a.code_stride,
                              k0 + quad * 32, row_bytes);
#pragma unroll
        for (int i = 0; i < 8; ++i) units[i] = (T)0x1p-7f;
#pragma unroll
        for (int m = 0; m < S::M; ++m) {
            const T* row = static_cast<const T*>(a.x) +
                           (m0 + min(m * 16 + li, rows - 1)) * a.x_stride;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = k0 + (S::NATURAL ? j * 32 + quad * 8 : quad * 32 + j * 8);
                x[m][j] = order(load_some(row + at, a.k - at));
            }
        }
        tile.step([&](int m, int j) { return x[m][j]; },
                  [&](int p, int m) {
                      f32x4 sum = {0, 0, 0, 0};
#pragma unroll
                      for (int j = p * S::PER; j < (p + 1) * S::PER; ++j)
                          sum = mfma(x[m][j], units, sum);
                      return sum;
                  },
                  w,
                  [&](int p, int r) {
                      return group_word<S>(a, row_of<S>(a, (rg * S::R + r) * 16 + li),
                                           min(group_of(a, k0 + p * S::PER * 32), groups - 1));
                  });
    }
}

// The groups' sums, the upper half of them onto the lower half, and the outputs.
template <class S>
__device__ inline void finish_tile(const LinearArgs& a, Tile<S>& tile, char* lds, int rg, int kp,
                                   int m0, int parts_z)
{
    typedef typename S::type T;
    constexpr int R = S::R, M = S::M, HR = S::HR;
    const int lane = threadIdx.x & 63, li = lane & 15, quad = lane >> 4;
    f32x4(*parts)[R * M][64] = reinterpret_cast<f32x4(*)[R * M][64]>(lds);
#pragma unroll
    for (int half = S::KP / 2; half > 0; half >>= 1) {
        __syncthreads();
        if (kp >= half && kp < 2 * half) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m)
                    parts[(kp - half) * S::RG + rg][r * M + m][lane] = tile.acc[r][m];
        }
        __syncthreads();
        if (kp < half) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m)
                    tile.acc[r][m] += parts[kp * S::RG + rg][r * M + m][lane];
        }
    }
    if (kp != 0) return;
    const int out_n = a.n / S::HALVES, n0 = (blockIdx.x * S::RG + rg) * (16 * HR);
    const T* bias = static_cast<const T*>(a.bias);
    const int64_t pitch = (a.rows + 3) / 4 * 4;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = n0 + (r % HR) * 16 + li;
        if (j >= out_n || (parts_z == 1 && r >= HR)) continue;
        const float b0 = bias ? (float)bias[j] : 0.0f;
        const float b1 = S::HALVES == 2 && bias ? (float)bias[j + out_n] : 0.0f;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int row = m0 + m * 16 + quad * 4;
            if (row >= a.rows) continue;
            if (parts_z > 1) {
                // [part][output][row of x]: a lane's four rows are neighbours
                *reinterpret_cast<f32x4*>(
                    static_cast<float*>(a.workspace) +
                    ((int64_t)blockIdx.z * a.n + j + (r / HR) * out_n) * pitch + row) =
                    tile.acc[r][m];
                continue;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (row + i < a.rows)
                    static_cast<T*>(a.y)[(row + i) * a.y_stride + j] = (T)finish<S::ACT>(
                        __builtin_fmaf(tile.acc[r][m][i], kUnit<T>, b0),
                        __builtin_fmaf(tile.acc[(r + R - HR) % R][m][i], kUnit<T>, b1));
        }
    }
}

typedef u32x4 Codes __attribute__((aligned(1)));

// One tile of rows of x (M = 1): LDS holds x and the groups of as many columns as
// fit, mostly all of them, and between two barriers a wave's loop has loads of
// codes alone, the next batch in flight during one.
template <class S>
__global__ __launch_bounds__(S::THREADS) void linear_kernel(LinearArgs a, int32_t cols)
{
    typedef typename S::type T;
    typedef typename Vec<T>::x8 V;
    extern __shared__ __align__(16) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave % S::RG, kp = wave / S::RG, li = lane & 15, quad = lane >> 4;
    const int m0 = blockIdx.y * (16 * S::M), rows = min(a.rows - m0, 16 * S::M);
    const uint8_t* codes[S::R];
#pragma unroll
    for (int r = 0; r < S::R; ++r)
        codes[r] = a.codes + row_of<S>(a, (rg * S::R + r) * 16 + li) * a.code_stride + quad * 16;
    auto load_w = [&](u32x4 (&w)[S::U][S::R], int batch) {
#pragma unroll
        for (int u = 0; u < S::U; ++u)
#pragma unroll
            for (int r = 0; r < S::R; ++r)
                w[u][r] = *reinterpret_cast<const Codes*>(codes[r] +
                                                          (batch * S::U + u) * (kStep / 2));
    };
    Tile<S> tile;
    const T* x0 = static_cast<const T*>(a.x) + m0 * a.x_stride;
    const int batches = a.k / S::BATCH;
    const int per = cols / S::BATCH;
    const Stage<S> stage(lds, rows, cols);
    for (int b0 = 0; b0 < batches; b0 += per) {
        const int count = min(per, batches - b0), c0 = b0 * S::BATCH, here = count * S::BATCH;
        const int from = b0 + kp * count / S::KP, upto = b0 + (kp + 1) * count / S::KP;
        const int g0 = group_of(a, c0), groups = group_of(a, c0 + here - 1) + 1 - g0;
        if (b0 > 0) __syncthreads();
        // x in stretches of 512 columns of a row, a wave each and 8 in flight; the
        // groups of a row of W, a wave each: neighbours in memory.  The first
        // turn of both and the first codes are on their way together.
        const int stretches = (here + 511) / 512, items = rows * stretches;
        V v[8];
        uint32_t g[8];
        u32x4 w[2][S::U][S::R];
        auto fetch_x = [&](int i0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int item = min(i0 + i, items - 1), row = item / stretches;
                const int at = (item - row * stretches) * 512 + lane * 8;
                v[i] = load8(x0 + row * a.x_stride + c0 + min(at, here - 8));
            }
        };
        auto store_x = [&](int i0) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int item = min(i0 + i, items - 1), row = item / stretches;
                const int at = (item - row * stretches) * 512 + lane * 8;
                if (at < here) stage.put(row, at, v[i]);
            }
        };
        auto fetch_g = [&](int l0, int k) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                g[i] = group_word<S>(a, row_of<S>(a, min(l0 + i * S::WAVES, S::ROWS - 1)),
                                     g0 + min(k + lane, groups - 1));
        };
        auto store_g = [&](int l0, int k) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (l0 + i * S::WAVES < S::ROWS && k + lane < groups)
                    stage.table[(k + lane) * S::ROWS + l0 + i * S::WAVES] = g[i];
        };
        fetch_x(wave * 8);
        fetch_g(wave, 0);
        load_w(w[0], min(from, b0 + count - 1));
        if (wave * 8 < items) store_x(wave * 8);
        if (wave < S::ROWS) store_g(wave, 0);
        for (int i0 = (S::WAVES + wave) * 8; i0 < items; i0 += S::WAVES * 8) {
            fetch_x(i0);
            store_x(i0);
        }
        for (int k = 0; k < groups; k += 64)
            for (int l0 = wave; l0 < S::ROWS; l0 += S::WAVES * 8) {
                if (k == 0 && l0 == wave) continue;
                fetch_g(l0, k);
                store_g(l0, k);
            }
        __syncthreads();
        for (int i0 = from; i0 < upto; i0 += 2) {
            // two register sets in turn: a copy would wait for the loads
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int i = i0 + d;
                if (i >= upto) break;
                load_w(w[1 - d], min(i + 1, upto - 1));
#pragma unroll
                for (int u = 0; u < S::U; ++u) {
                    const int col = (i - b0) * S::BATCH + u * kStep;
                    stage.take(tile, w[d][u], rows, col, rg, [&](int p) {
                        return group_of(a, c0 + col + p * S::PER * 32) - g0;
                    });
                }
            }
        }
    }
    rest<S>(a, tile, rg, m0, rows, batches * S::U + kp, S::KP);
    finish_tile<S>(a, tile, lds, rg, kp, m0, 1);
}

// Several tiles of rows of x: the columns go by in chunks of a batch for every
// group, x, its sums and the groups through two buffers in LDS.  DEPTH register
// sets in turn keep DEPTH - 1 chunks of everything in flight.
template <class S, int DEPTH>
__global__ __launch_bounds__(S::THREADS) void linear_stream_kernel(LinearArgs a, int32_t parts_z)
{
    typedef typename S::type T;
    typedef typename Vec<T>::x8 V;
    extern __shared__ __align__(16) char lds[];
    constexpr int COLS = S::KP * S::BATCH, UNITS = COLS / 8;
    constexpr int TURNS = (16 * S::M * UNITS + S::THREADS - 1) / S::THREADS;
    constexpr int GROUPS = COLS / (32 * S::PER) + 1;       // a chunk may start inside one
    constexpr int G_TURNS = (S::ROWS * GROUPS + S::THREADS - 1) / S::THREADS;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int rg = wave % S::RG, kp = wave / S::RG, li = lane & 15, quad = lane >> 4;
    const int m0 = blockIdx.y * (16 * S::M), rows = min(a.rows - m0, 16 * S::M);
    const int last_group = (a.k + a.group - 1) / a.group - 1;
    const uint8_t* codes[S::R];
#pragma unroll
    for (int r = 0; r < S::R; ++r)
        codes[r] = a.codes + row_of<S>(a, (rg * S::R + r) * 16 + li) * a.code_stride + quad * 16;
    Tile<S> tile;
    const T* x0 = static_cast<const T*>(a.x) + m0 * a.x_stride;
    const int batches = a.k / S::BATCH;
    const int begin = (int)((int64_t)blockIdx.z * batches / parts_z);
    const int end = (int)((int64_t)(blockIdx.z + 1) * batches / parts_z);
    const int chunks = (end - begin + S::KP - 1) / S::KP, c_end = end * S::BATCH;
    const Stage<S> stage[2] = {Stage<S>(lds, rows, COLS),
                               Stage<S>(lds + Stage<S>::bytes(rows, COLS, GROUPS), rows, COLS)};
    struct Set {
        u32x4 w[S::U][S::R];
        V x[TURNS];
        uint32_t group[G_TURNS];
    };
    Set set[DEPTH];
    // addresses behind the part's end are clamped into it: no branch, so the
    // compiler counts the loads in flight exactly
    auto fetch = [&](Set& s, int chunk) {
        const int c0 = begin * S::BATCH + min(chunk, chunks - 1) * COLS, g0 = group_of(a, c0);
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int u = threadIdx.x + t * S::THREADS;
            s.x[t] = load8(x0 + min(u / UNITS, rows - 1) * a.x_stride +
                           min(c0 + u % UNITS * 8, c_end - 8));
        }
#pragma unroll
        for (int t = 0; t < G_TURNS; ++t) {
            const int u = threadIdx.x + t * S::THREADS;
            s.group[t] = group_word<S>(a, row_of<S>(a, min(u / GROUPS, S::ROWS - 1)),
                                       min(g0 + u % GROUPS, last_group));
        }
        const int batch = min(begin + min(chunk, chunks - 1) * S::KP + kp, end - 1);
#pragma unroll
        for (int u = 0; u < S::U; ++u)
#pragma unroll
            for (int r = 0; r < S::R; ++r)
                s.w[u][r] = *reinterpret_cast<const Codes*>(codes[r] +
                                                            (batch * S::U + u) * (kStep / 2));
    };
    auto store = [&](const Set& s, int which) {
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int u = threadIdx.x + t * S::THREADS;
            if (u / UNITS < rows) stage[which].put(u / UNITS, u % UNITS * 8, s.x[t]);
        }
#pragma unroll
        for (int t = 0; t < G_TURNS; ++t) {
            const int u = threadIdx.x + t * S::THREADS;
            if (u / GROUPS < S::ROWS) stage[which].table[u % GROUPS * S::ROWS + u / GROUPS] = s.group[t];
        }
    };
    if (chunks > 0) {
#pragma unroll
        for (int d = 0; d < DEPTH - 1; ++d) fetch(set[d], d);
        store(set[0], 0);
    }
    __syncthreads();
    static_assert(DEPTH % 2 == 0, "a set and a buffer go together");
    for (int i0 = 0; i0 < chunks; i0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int i = i0 + d;
            if (i >= chunks) break;
            fetch(set[(d + DEPTH - 1) % DEPTH], i + DEPTH - 1);
            const int c0 = (begin + i * S::KP) * S::BATCH, g0 = group_of(a, c0);
            if (begin + i * S::KP + kp < end) {
#pragma unroll
                for (int u = 0; u < S::U; ++u) {
                    const int col = kp * S::BATCH + u * kStep;
                    stage[d & 1].take(tile, set[d].w[u], rows, col, rg, [&](int p) {
                        return group_of(a, c0 + col + p * S::PER * 32) - g0;
                    });
                }
            }
            store(set[(d + 1) % DEPTH], (d + 1) & 1);
            __syncthreads();
        }
    }
    rest<S>(a, tile, rg, m0, rows, batches * S::U + blockIdx.z * S::KP + kp, parts_z * S::KP);
    finish_tile<S>(a, tile, lds, rg, kp, m0, parts_z);
}

// The parts of the columns, in order; a thread an output and four rows of x.
template <typename T, int ACT>
__global__ __launch_bounds__(256) void linear_join_kernel(LinearArgs a, int32_t parts_z)
{
    const int out_n = ACT == RM_ACT_SWIGLU ? a.n / 2 : a.n;
    const int quads = (a.rows + 3) / 4;
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int j = (int)(t % out_n), quad = (int)(t / out_n);
    if (quad >= quads) return;
    const float* part = static_cast<const float*>(a.workspace) + quad * 4;
    f32x4 sum[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll 4
    for (int z = 0; z < parts_z; ++z)
#pragma unroll
        for (int h = 0; h < (ACT == RM_ACT_SWIGLU ? 2 : 1); ++h)
            sum[h] += *reinterpret_cast<const f32x4*>(
                part + ((int64_t)z * a.n + j + h * out_n) * (quads * 4));
    const T* bias = static_cast<const T*>(a.bias);
    const float b0 = bias ? (float)bias[j] : 0.0f;
    const float b1 = ACT == RM_ACT_SWIGLU && bias ? (float)bias[j + out_n] : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (quad * 4 + i < a.rows)
            static_cast<T*>(a.y)[(quad * 4 + i) * a.y_stride + j] =
                (T)finish<ACT>(__builtin_fmaf(sum[0][i], kUnit<T>, b0),
                               __builtin_fmaf(sum[1][i], kUnit<T>, b1));
}

template <class S, typename K, typename... A>
hipError_t launch_shape(K kernel, size_t lds, const LinearArgs& a, int parts_z, hipStream_t s,
                        A... more)
{
    const int out_n = a.n / S::HALVES, width = 16 * S::HR * S::RG;
    const dim3 grid((unsigned)((out_n + width - 1) / width),
                    (unsigned)((a.rows + 16 * S::M - 1) / (16 * S::M)), (unsigned)parts_z);
    const size_t parts = (size_t)(S::KP / 2) * S::RG * S::R * S::M * 64 * sizeof(f32x4);
    if (lds < parts) lds = parts;
    if (lds > 64 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)lds);
        if (e != hipSuccess) return e;
    }
    const hipError_t e = launch(kernel, grid, S::THREADS, lds, s, a, more...);
    if (e != hipSuccess || parts_z == 1) return e;
    const int64_t threads = (int64_t)out_n * ((a.rows + 3) / 4);
    return launch(linear_join_kernel<typename S::type, S::ACT>,
                  dim3((unsigned)((threads + 255) / 256)), 256, 0, s, a, (int32_t)parts_z);
}

template <typename T, int R, int PER, int ACT, int U, int RG, int KP>
hipError_t launch_few(const LinearArgs& a, size_t most_lds, hipStream_t s)
{
    typedef Shape<T, R, 1, PER, ACT, U, RG, KP> S;
    const int rows = a.rows < 16 ? a.rows : 16;
    int cols = a.k / S::BATCH * S::BATCH;
    auto bytes = [&](int c) { return Stage<S>::bytes(rows, c, c / a.group + 2); };
    if (bytes(cols) > most_lds) {
        cols = S::BATCH * KP;
        while (bytes(cols + S::BATCH * KP) <= most_lds) cols += S::BATCH * KP;
    }
    return launch_shape<S>(linear_kernel<S>, bytes(cols), a, 1, s, (int32_t)cols);
}

template <typename T, int R, int M, int PER, int ACT, int U, int RG, int KP, int DEPTH>
hipError_t launch_many(const LinearArgs& a, int parts_z, hipStream_t s)
{
    typedef Shape<T, R, M, PER, ACT, U, RG, KP> S;
    constexpr int COLS = KP * S::BATCH;
    const int rows = a.rows < 16 * M ? a.rows : 16 * M;
    return launch_shape<S>(linear_stream_kernel<S, DEPTH>,
                           2 * Stage<S>::bytes(rows, COLS, COLS / (32 * PER) + 1), a, parts_z, s,
                           (int32_t)parts_z);
}

// What is taken for which sizes; us at the sizes named, measured one after the
// other on buffers that rotate through 3 copies.
enum Kind { kRows, kRowsWide, kTile, kTile2, kTile2Tall, kTile4 };
struct Plan {
    Kind kind;
    int parts_z;
};

Plan plan_of(int32_t rows, int32_t n, int32_t k, int act)
{
    const int out_n = act == RM_ACT_SWIGLU ? n / 2 : n;
    const int64_t tiles = (out_n + 15) / 16;
    Plan p = {kTile4, 1};
    int64_t blocks;
    if (rows <= 4 || (rows <= 16 && tiles < 512)) {
        // few rows: x fits in LDS whole.  Four waves side by side where that
        // fills the CUs (1 x 28672 x 8192: 26.0 us, one 32.2), else all waves of a
        // workgroup on the same rows (1 x 4096 x 4096: 5.0 us, two side by side 6.9;
        // 16 x 4096 x 4096: 8.2 against 10.9 in a stream)
        p.kind = tiles >= 1024 ? kRowsWide : kRows;
        return p;
    }
    if (rows <= 16) {
        // x in a stream, two tiles of W a wave: 16 x 28672 x 4096 gated 20.6 us, from
        // LDS whole 23.5
        p.kind = kTile;
        blocks = (tiles + (act == RM_ACT_SWIGLU ? 3 : 7)) / (act == RM_ACT_SWIGLU ? 4 : 8);
    } else if (rows <= 32) {
        // 32 x 8192 x 8192: 38.4 us in one part of the columns, 18.3 in four
        p.kind = kTile2;
        blocks = (tiles + (act == RM_ACT_SWIGLU ? 3 : 7)) / (act == RM_ACT_SWIGLU ? 4 : 8);
    } else {
        // 64 x 8192 x 28672: 78 us in eight parts, 90 in sixteen (here and below in a
        // graph whose calls alternate between two sets of weights)
        blocks = (tiles + (act == RM_ACT_SWIGLU ? 7 : 15)) / (act == RM_ACT_SWIGLU ? 8 : 16) *
                 ((rows + 63) / 64);
    }
    // Parts of the columns until the CUs have about a workgroup each, of 512 columns
    // at least (64 x 512 x 8192: 17.6 us, of 1024 at least 19.5).  224 workgroups in
    // one part and in two: 16 x 28672 x 4096 gated 22.1 and 24.1 us, 32 rows 30.0 and
    // 37.4, 64 rows 45.7 and 59.2.
    const int64_t want = (kComputeUnits + blocks / 2) / blocks, most = k / 512;
    p.parts_z = (int)(want < most ? want : most);
    // 64 x 2048 x 28672: 34.6 us in sixteen parts, 51.2 in eight
    if (p.parts_z > 16) p.parts_z = 16;
    if (p.parts_z < 1) p.parts_z = 1;
    // 64 rows of x a workgroup where that fills the CUs (64 x 8192 x 28672: 78 us,
    // 32 rows 99), else 32 (64 x 4096 x 14336 in groups of 32: 44 us, 64
    // rows 80; 48 x 6000 x 5000: 29 and 35; 128 x 4096 x 4096: 21 and 27)
    if (p.kind == kTile4 && blocks * p.parts_z < kComputeUnits) p.kind = kTile2Tall;
    return p;
}

template <typename T, int PER, int ACT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t s)
{
    constexpr int ONE = ACT == RM_ACT_SWIGLU ? 2 : 1;       // the least tiles a wave
    const Plan p = plan_of(a.rows, a.n, a.k, ACT);
    switch (p.kind) {
    case kRows: return launch_few<T, ONE, PER, ACT, 2, 1, 8>(a, kMostLds, s);
    case kRowsWide: return launch_few<T, ONE, PER, ACT, 2, 4, 2>(a, 64 * 1024, s);
    case kTile: return launch_many<T, 2, 1, PER, ACT, 2, 4, 2, 2>(a, p.parts_z, s);
    case kTile2: return launch_many<T, 2, 2, PER, ACT, 1, 4, 2, 2>(a, p.parts_z, s);
    case kTile2Tall: return launch_many<T, 2, 2, PER, ACT, 1, 8, 1, 2>(a, p.parts_z, s);
    default: return launch_many<T, 2, 4, PER, ACT, 1, 8, 1, 2>(a, p.parts_z, s);
    }
}

template <typename T, int ACT>
hipError_t launch_group(const LinearArgs& a, hipStream_t s)
{
    if (a.group % 128 == 0 || a.group >= a.k) return launch_rows<T, 4, ACT>(a, s);
    if (a.group % 64 == 0) return launch_rows<T, 2, ACT>(a, s);
    return launch_rows<T, 1, ACT>(a, s);
}

}  // namespace

size_t linear_workspace(int32_t rows, int32_t n, int32_t k, int act)
{
    const Plan p = plan_of(rows, n, k, act);
    return p.parts_z > 1 ? (size_t)p.parts_z * n * ((rows + 3) / 4 * 4) * sizeof(float) : 0;
}

hipError_t launch_linear(int type, int act, const LinearArgs& a, hipStream_t s)
{
    if (type == RM_TYPE_BF16)
        return act == RM_ACT_NONE ? launch_group<bf16, RM_ACT_NONE>(a, s)
                                  : launch_group<bf16, RM_ACT_SWIGLU>(a, s);
    return act == RM_ACT_NONE ? launch_group<f16, RM_ACT_NONE>(a, s)
                              : launch_group<f16, RM_ACT_SWIGLU>(a, s);
}

}  // namespace rm
