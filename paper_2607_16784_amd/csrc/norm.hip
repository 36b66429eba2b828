// norm.hip -- the gated, scaled residual between two blocks with the norms
// around it (rm_norm_residual).
//
// One pass: a row stays in registers between its reads and its writes, so each
// input is read once and each output written once; the kernel is bound by that
// traffic.  A thread holds 8 neighbouring elements a chunk (16-byte accesses).
// Rows of up to 1024 elements take a wave each and need no barrier; wider ones
// a workgroup with one chunk a thread where that fits.  Workgroups stride over
// the rows with the gains in registers.
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

template <typename T, int KIND, int C, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void norm_kernel(NormArgs a)
{
    typedef typename Vec<T>::x8 V;
    __shared__ float part[2][16];
    int turn = 0;
    const int per_row = WAVE ? 64 : blockDim.x;
    const int lane = WAVE ? threadIdx.x & 63 : threadIdx.x;
    const int64_t rows_here = WAVE ? blockDim.x >> 6 : 1;
    const int first = lane * 8, step = per_row * 8;
    const T* post = static_cast<const T*>(a.post_weight);
    const T* pre = static_cast<const T*>(a.pre_weight);
    const T* bias = static_cast<const T*>(a.pre_bias);
    V w_post[C], w_pre[C], w_bias[C];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = first + c * step;
        if (post) w_post[c] = load_some(post + at, a.width - at);
        if (pre) w_pre[c] = load_some(pre + at, a.width - at);
        if (bias) w_bias[c] = load_some(bias + at, a.width - at);
    }
    for (int64_t row = blockIdx.x * rows_here + (WAVE ? threadIdx.x >> 6 : 0); row < a.rows;
         row += gridDim.x * rows_here) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* y = static_cast<const T*>(a.y) + row * a.y_stride;
        const T* g = static_cast<const T*>(a.gate) + row * a.gate_stride;
        V vx[C], vy[C], vg[C];
        float g1 = 1.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = first + c * step;
            vx[c] = load_some(x + at, a.width - at);
            if (a.y) vy[c] = load_some(y + at, a.width - at);
            if (a.gate && a.gate_width > 1) vg[c] = load_some(g + at, a.width - at);
        }
        if (a.gate && a.gate_width == 1) g1 = (float)g[0];
        float v[C][8];
        if (a.y) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (float)vy[c][i];
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
                for (int i = 0; i < 8; ++i) {
                    const float gi = a.gate && a.gate_width > 1 ? (float)vg[c][i] : g1;
                    v[c][i] = __builtin_fmaf(a.alpha, v[c][i] * gi, (float)vx[c][i]);
                }
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
                store_some(out + at, o, a.width - at);
            }
        }
        if (!a.n_out) continue;
        // behind the row's end v is alpha * 0 * 0 + 0 = 0 unless alpha or a
        // gate is not finite; those lanes must not reach the sums
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (first + c * step + i >= a.width) v[c][i] = 0.0f;
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
            store_some(out + at, o, a.width - at);
        }
    }
}

template <typename T, int KIND>
hipError_t launch_kind(const NormArgs& a, hipStream_t s)
{
    const int vectors = (a.width + 7) / 8;
    if (vectors <= 128) {
        const int64_t want = ((int64_t)a.rows + 3) / 4;
        const unsigned grid = (unsigned)(want < 8 * kComputeUnits ? want : 8 * kComputeUnits);
        return vectors <= 64 ? launch(norm_kernel<T, KIND, 1, true>, grid, 256, 0, s, a)
                             : launch(norm_kernel<T, KIND, 2, true>, grid, 256, 0, s, a);
    }
    const int chunks = vectors <= 1024 ? 1 : vectors <= 2048 ? 2 : 4;
    const unsigned threads = (unsigned)((vectors + chunks - 1) / chunks + 63) / 64 * 64;
    const int64_t most = (int64_t)kComputeUnits * (2048 / threads);
    const unsigned grid = (unsigned)(a.rows < most ? a.rows : most);
    if (chunks == 1) return launch(norm_kernel<T, KIND, 1, false>, grid, threads, 0, s, a);
    if (chunks == 2) return launch(norm_kernel<T, KIND, 2, false>, grid, threads, 0, s, a);
    return launch(norm_kernel<T, KIND, 4, false>, grid, threads, 0, s, a);
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
