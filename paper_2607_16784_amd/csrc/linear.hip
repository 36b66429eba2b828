// linear.hip -- projection with 4-bit weights and group scales (rm_w4_linear).
//
// y = x W^T on the matrix cores, 16 rows of x by 16 rows of W a tile
// (v_mfma_f32_16x16x32).  With one to some tens of rows of x the kernel is
// bound by reading the codes once, so everything serves that: the codes are
// read as they are, row by row, 16 bytes a lane, and expanded in registers.
//
// Expansion: two codes sit 4 nibbles apart in a word, so (w >> 4s) & 0x000f000f
// is the pair (s, s+4) in the low bits of two 16-bit numbers, and OR-ing an
// exponent makes it 128 + code (bf16) or 1024 + code (f16), exactly.  x is put
// into the same order 0 4 1 5 2 6 3 7.  f16 then subtracts 1024 + zero (exact).
// bf16 has no packed addition: the product is taken with 128 + code and
// (128 + zero) * (sum of x) is subtracted from each group's fp32 sum, where the
// sum of x comes from one more matrix instruction against ones.  Both keep the
// code exact; the group's scale multiplies the fp32 sum.
//
// A workgroup owns 16 R rows of W and 16 M rows of x; its waves take the steps
// of 128 columns in turn and add up through LDS in a fixed order.
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

constexpr int kStep = 128;    // columns of a step: 16 bytes of codes a lane

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

__device__ inline bf16x8 expand(uint32_t w, bf16x2)
{
    return __builtin_bit_cast(bf16x8, u32x4{(w & 0x000f000fu) | 0x43004300u,
                                            ((w >> 4) & 0x000f000fu) | 0x43004300u,
                                            ((w >> 8) & 0x000f000fu) | 0x43004300u,
                                            ((w >> 12) & 0x000f000fu) | 0x43004300u});
}
__device__ inline f16x8 expand(uint32_t w, f16x2 zero)
{
    u32x4 r;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        const f16x2 p = __builtin_bit_cast(f16x2, ((w >> (4 * s)) & 0x000f000fu) | 0x64006400u);
        r[s] = __builtin_bit_cast(uint32_t, (f16x2)(p - zero));
    }
    return __builtin_bit_cast(f16x8, r);
}

// PER: matrix instructions (32 columns each) that share a group: 4, 2 or 1.
template <typename T, int R, int M, int PER, int ACT, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void linear_kernel(LinearArgs a)
{
    typedef typename Vec<T>::x8 V;
    typedef typename Vec<T>::x2 P;
    constexpr bool HALF = __is_same(T, f16);
    constexpr bool NATURAL = PER < 4;     // columns of an instruction are neighbours
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int li = lane & 15, quad = lane >> 4;
    const int row_bytes = (a.k + 1) / 2;
    const int groups = (a.k + a.group - 1) / a.group;
    const int halves = ACT == RM_ACT_SWIGLU ? 2 : 1;
    const int out_n = a.n / halves;
    constexpr int HR = ACT == RM_ACT_SWIGLU ? R / 2 : R;     // tiles of outputs
    const int n0 = blockIdx.x * (16 * HR), m0 = blockIdx.y * (16 * M);

    const uint8_t* codes[R];
    const T* scales[R];
    const uint8_t* zeros[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int j = min(n0 + (r % HR) * 16 + li, out_n - 1) + (r / HR) * out_n;
        codes[r] = a.codes + j * a.code_stride;
        scales[r] = static_cast<const T*>(a.scales) + (int64_t)j * groups;
        zeros[r] = a.zeros ? a.zeros + (int64_t)j * groups : nullptr;
    }
    const T* x[M];
#pragma unroll
    for (int m = 0; m < M; ++m)
        x[m] = static_cast<const T*>(a.x) + min(m0 + m * 16 + li, a.rows - 1) * a.x_stride;

    f32x4 acc[R][M];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int m = 0; m < M; ++m) acc[r][m] = f32x4{0, 0, 0, 0};
    V ones;
#pragma unroll
    for (int i = 0; i < 8; ++i) ones[i] = (T)1.0f;

    const int steps = (a.k + kStep - 1) / kStep;
    u32x4 w[R], next[R];
    const int off = quad * 32;
#pragma unroll
    for (int r = 0; r < R; ++r)
        next[r] = wave < steps ? load_codes(codes[r], wave * kStep + off, row_bytes)
                               : u32x4{0, 0, 0, 0};
    for (int step = wave; step < steps; step += WAVES) {
        const int k0 = step * kStep;
        V xv[M][4];
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int at = k0 + (NATURAL ? j * 32 + quad * 8 : quad * 32 + j * 8);
                xv[m][j] = load_some(x[m] + at, a.k - at);
            }
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = next[r];
        if (step + WAVES < steps) {
#pragma unroll
            for (int r = 0; r < R; ++r)
                next[r] = load_codes(codes[r], k0 + WAVES * kStep + off, row_bytes);
        }
        if (NATURAL) {
#pragma unroll
            for (int r = 0; r < R; ++r) w[r] = transpose_rows(w[r]);
        }
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int j = 0; j < 4; ++j) xv[m][j] = order(xv[m][j]);
#pragma unroll
        for (int j0 = 0; j0 < 4; j0 += PER) {
            const int g = min((k0 + j0 * 32) / a.group, groups - 1);
            f32x4 sum[M];
            if (!HALF) {
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    sum[m] = f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int j = j0; j < j0 + PER; ++j) sum[m] = mfma(xv[m][j], ones, sum[m]);
                }
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float scale = (float)scales[r][g];
                const int z = zeros[r] ? zeros[r][g] : 8;
                P zero;
                zero[0] = zero[1] = (T)(float)(1024 + z);
                f32x4 part[M];
#pragma unroll
                for (int m = 0; m < M; ++m) part[m] = f32x4{0, 0, 0, 0};
#pragma unroll
                for (int j = j0; j < j0 + PER; ++j) {
                    const V e = expand(w[r][j], zero);
#pragma unroll
                    for (int m = 0; m < M; ++m) part[m] = mfma(xv[m][j], e, part[m]);
                }
                const float bias = -(float)(128 + z);
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float p = HALF ? part[m][i]
                                             : __builtin_fmaf(bias, sum[m][i], part[m][i]);
                        acc[r][m][i] = __builtin_fmaf(scale, p, acc[r][m][i]);
                    }
            }
        }
    }

    // the waves' sums, upper half onto lower half
    __shared__ f32x4 parts[WAVES / 2 > 0 ? WAVES / 2 : 1][R * M][64];
#pragma unroll
    for (int half = WAVES / 2; half > 0; half >>= 1) {
        if (wave >= half && wave < 2 * half) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m) parts[wave - half][r * M + m][lane] = acc[r][m];
        }
        __syncthreads();
        if (wave < half) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int m = 0; m < M; ++m) acc[r][m] += parts[wave][r * M + m][lane];
        }
        __syncthreads();
    }
    if (wave != 0) return;
    const T* bias = static_cast<const T*>(a.bias);
#pragma unroll
    for (int r = 0; r < HR; ++r) {
        const int j = n0 + r * 16 + li;
        if (j >= out_n) continue;
        const float b0 = bias ? (float)bias[j] : 0.0f;
        const float b1 = ACT == RM_ACT_SWIGLU && bias ? (float)bias[j + out_n] : 0.0f;
#pragma unroll
        for (int m = 0; m < M; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int row = m0 + m * 16 + quad * 4 + i;
                if (row >= a.rows) continue;
                float t = acc[r][m][i] + b0;
                if (ACT == RM_ACT_SWIGLU)
                    t = t / (1.0f + expf(-t)) * (acc[r + R - HR][m][i] + b1);
                static_cast<T*>(a.y)[row * a.y_stride + j] = (T)t;
            }
    }
}

template <typename T, int R, int M, int PER, int ACT>
hipError_t launch_tile(const LinearArgs& a, hipStream_t s)
{
    constexpr int WAVES = 8;
    const int out_n = ACT == RM_ACT_SWIGLU ? a.n / 2 : a.n;
    constexpr int HR = ACT == RM_ACT_SWIGLU ? R / 2 : R;
    const dim3 grid((unsigned)((out_n + 16 * HR - 1) / (16 * HR)),
                    (unsigned)((a.rows + 16 * M - 1) / (16 * M)));
    return launch(linear_kernel<T, R, M, PER, ACT, WAVES>, grid, WAVES * 64, 0, s, a);
}

template <typename T, int PER, int ACT>
hipError_t launch_rows(const LinearArgs& a, hipStream_t s)
{
    if (a.rows <= 16) return launch_tile<T, 2, 1, PER, ACT>(a, s);
    if (a.rows <= 32) return launch_tile<T, 2, 2, PER, ACT>(a, s);
    return launch_tile<T, 2, 4, PER, ACT>(a, s);
}

template <typename T, int ACT>
hipError_t launch_group(const LinearArgs& a, hipStream_t s)
{
    if (a.group % 128 == 0 || a.group >= a.k) return launch_rows<T, 4, ACT>(a, s);
    if (a.group % 64 == 0) return launch_rows<T, 2, ACT>(a, s);
    return launch_rows<T, 1, ACT>(a, s);
}

}  // namespace

hipError_t launch_linear(int type, int act, const LinearArgs& a, hipStream_t s)
{
    if (type == RM_TYPE_BF16)
        return act == RM_ACT_NONE ? launch_group<bf16, RM_ACT_NONE>(a, s)
                                  : launch_group<bf16, RM_ACT_SWIGLU>(a, s);
    return act == RM_ACT_NONE ? launch_group<f16, RM_ACT_NONE>(a, s)
                              : launch_group<f16, RM_ACT_SWIGLU>(a, s);
}

}  // namespace rm
