// headnorm.hip -- norms of each head's queries and keys with the rotation behind
// them (rm_head_norm_rotary).
//
// A row is one head of one token.  LANES neighbouring lanes hold it, 8 channels
// each, between its read and its write, so the kernel is bound by that traffic.
// With u = r x w, r the row's 1 / root mean square, a turned channel is
//   r (x (w cos) +- x' (w' sin)),  x' the channel that x turns with,
// so gain, angle and rot_scale are one factor a channel, taken once a token and
// side for all of a wave's heads.  Sines and cosines are taken once a token, a pair a
// lane, and pass through LDS: each lane taking its own eight channels' took 8190 tokens
// of 40 heads of 128 from 33 (5.1 TB/s) to 50 us.  Halves of a `rot` that is no multiple
// of 16 begin within another lane's chunk, and partners are read one by one: the same
// tokens 66 (rot 72 and 120) to 76 us (36).
#include "rm_decode.h"
#include "rm_rotary.h"

namespace rm {
namespace {

constexpr int kWaves = 4;
constexpr int kAhead = 4;      // rows that a lane has in flight
constexpr int kMostPairs = RM_MAX_HEAD_WIDTH / 2;

// Where the channel that a channel turns with is found.
enum { NEIGHBOUR = 0, LANE = 1, ANYWHERE = 2 };

// Sum over LANES (4 or more) neighbouring lanes.
template <int LANES>
__device__ inline float group_sum(float v)
{
    v += dpp_float<0xB1>(v);
    v += dpp_float<0x4E>(v);
    if (LANES >= 8) v += dpp_float<0x141>(v);
    if (LANES >= 16) v += dpp_float<0x140>(v);
    if (LANES >= 32) v += __shfl_xor(v, 16);
    if (LANES >= 64) v += __shfl_xor(v, 32);
    return v;
}

// Rows of one side (queries or keys) of one token.
struct Side {
    const void *x, *weight;
    void* out;
    int64_t head, out_head;
    int32_t heads;
};

// turn: sine and cosine of the token's pairs, once `angles` has put them there.
template <typename T, int LANES, int WHERE, typename F>
__device__ inline void turn_side(const HeadNormArgs& a, const Side& side, int part, int parts,
                                 const float2* turn, F angles)
{
    typedef typename Vec<T>::x8 V;
    constexpr int ROWS = 64 / LANES;             // a wave takes at a time
    const int lane = threadIdx.x & 63, c0 = lane % LANES * 8, row0 = lane / LANES;
    const int D = a.head_dim, half = a.rot >> 1;
    const bool in = c0 < D;
    const T* x = static_cast<const T*>(side.x);
    const T* weight = static_cast<const T*>(side.weight);
    const int passes = (side.heads + ROWS - 1) / ROWS;
    if (part >= passes) {
        angles();
        return;
    }

    V v[kAhead];
    T w[kAhead][WHERE == ANYWHERE ? 8 : 1];
    int partner[WHERE == ANYWHERE ? 8 : 1];
    if (WHERE == ANYWHERE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = c0 + i;
            partner[i] = c >= a.rot || !in ? min(c, D - 1) : c < half ? c + half : c - half;
        }
    }
    auto load = [&](int slot, int pass) {
        const int row = min(pass * ROWS + row0, side.heads - 1);
        const T* at = x + row * side.head;
        v[slot] = load8(at + (in ? c0 : 0));
        if (WHERE == ANYWHERE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[slot][i] = at[partner[i]];
        }
    };
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(i, min(part + i * parts, passes - 1));

    // own: factor of the channel itself, other: of the one that it turns with
    float own[8], other[8];
    const int step = a.rot >> 4;                 // LANE: chunks of half the turned channels
    const int c1 = WHERE == LANE ? (c0 < half ? c0 + half : c0 - half) : c0;
    const bool turned = in && c0 < a.rot;
    V w0, w1;
    if (weight) {
        w0 = load8(weight + (in ? c0 : 0));
        if (WHERE == LANE) w1 = load8(weight + (turned ? c1 : 0));
    }
    angles();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int c = c0 + i;
        own[i] = weight ? (float)w0[i] : 1.0f;
        other[i] = 0.0f;
        if (c >= a.rot || !in) continue;
        const bool first = WHERE == NEIGHBOUR ? (i & 1) == 0 : WHERE == LANE ? c0 < half : c < half;
        const float2 t = turn[WHERE == NEIGHBOUR ? c >> 1 : first ? c : c - half];
        float with = 1.0f;
        if (weight)
            with = WHERE == NEIGHBOUR ? (float)w0[i ^ 1]
                   : WHERE == LANE    ? (float)w1[i]
                                      : (float)weight[first ? c + half : c - half];
        other[i] = (first ? -t.y : t.y) * with;
        own[i] *= t.x;
    }
    // the lane that holds the partners of this lane's channels
    const int chunk = lane % LANES;
    const int with_lane = chunk < step ? lane + step : chunk < 2 * step ? lane - step : lane;

    for (int pass = part; pass < passes; pass += parts * kAhead) {
        if (pass != part) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load(i, min(pass + i * parts, passes - 1));
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int row = (pass + i * parts) * ROWS + row0;
            if (pass + i * parts >= passes) break;
            float f[8], g[8], s = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                f[j] = in ? (float)v[i][j] : 0.0f;
                s = __builtin_fmaf(f[j], f[j], s);
            }
            const float r = 1.0f / sqrtf(group_sum<LANES>(s) / (float)D + a.eps);
            if (WHERE == LANE) {
                const u32x4 mine = __builtin_bit_cast(u32x4, v[i]);
                u32x4 theirs;
#pragma unroll
                for (int j = 0; j < 4; ++j) theirs[j] = (uint32_t)__shfl((int)mine[j], with_lane);
                const V o = __builtin_bit_cast(V, theirs);
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = (float)o[j];
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    g[j] = WHERE == NEIGHBOUR ? f[j ^ 1] : (float)w[i][WHERE == NEIGHBOUR ? 0 : j];
            }
            V o;
#pragma unroll
            for (int j = 0; j < 8; ++j)
                o[j] = (T)(r * __builtin_fmaf(f[j], own[j], g[j] * other[j]));
            if (in && row < side.heads)
                store8(static_cast<T*>(side.out) + row * side.out_head + c0, o);
        }
    }
}

// `parts` waves a token.
template <typename T, int LANES, int WHERE>
__global__ __launch_bounds__(kWaves * 64) void headnorm_kernel(HeadNormArgs a, int32_t parts)
{
    __shared__ float2 turns[kWaves][kMostPairs];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float2* turn = turns[wave];
    const int64_t all = (int64_t)a.n_tokens * parts, by = (int64_t)gridDim.x * kWaves;
    for (int64_t at = (int64_t)blockIdx.x * kWaves + wave; at < all; at += by) {
        const int64_t token = at / parts;
        const int part = (int)(at % parts);
        const int32_t position = a.rot ? a.positions[token] : 0;
        auto angles = [&]() {
            for (int p = threadIdx.x & 63; p < a.rot >> 1; p += 64) {
                float cs, sn;
                turn_of(turns_of(a.inv_freq, p), position, a.rot_scale, cs, sn);
                turn[p] = make_float2(cs, sn);
            }
            // the wave's own
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        };
        const Side q = {static_cast<const T*>(a.q) + token * a.q_stride, a.q_weight,
                        static_cast<T*>(a.q_out) + token * a.q_out_stride, a.q_head,
                        a.q_out_head, a.heads};
        turn_side<T, LANES, WHERE>(a, q, part, parts, turn, angles);
        const Side k = {static_cast<const T*>(a.k) + token * a.k_stride, a.k_weight,
                        static_cast<T*>(a.k_out) + token * a.k_out_stride, a.k_head,
                        a.k_out_head, a.kv_heads};
        // the keys' first rows go to the wave behind the one with the queries' last
        turn_side<T, LANES, WHERE>(a, k, parts - 1 - part, parts, turn, [] {});
    }
}

template <typename T, int LANES, int WHERE>
hipError_t launch_form(const HeadNormArgs& a, hipStream_t s)
{
    constexpr int ROWS = 64 / LANES;
    const int32_t most = a.heads > a.kv_heads ? a.heads : a.kv_heads;
    const int32_t passes = (most + ROWS - 1) / ROWS;
    // waves for every SIMD of the card before a wave takes several rows after each other
    const int64_t want = (kComputeUnits * 8 + (int64_t)a.n_tokens - 1) / a.n_tokens;
    const int32_t parts = (int32_t)(want < passes ? want : passes);
    const int64_t blocks = ((int64_t)a.n_tokens * parts + kWaves - 1) / kWaves;
    const int64_t limit = most_blocks(kWaves * 64);
    return launch(headnorm_kernel<T, LANES, WHERE>, dim3((unsigned)(blocks < limit ? blocks : limit)),
                  kWaves * 64, 0, s, a, parts);
}

template <typename T, int LANES>
hipError_t launch_lanes(const HeadNormArgs& a, hipStream_t s)
{
    if (a.layout == RM_ROTARY_INTERLEAVED || a.rot == 0) return launch_form<T, LANES, NEIGHBOUR>(a, s);
    if (a.rot % 16 == 0) return launch_form<T, LANES, LANE>(a, s);
    return launch_form<T, LANES, ANYWHERE>(a, s);
}

template <typename T>
hipError_t launch_type(const HeadNormArgs& a, hipStream_t s)
{
    const int chunks = a.head_dim / 8;
    if (chunks <= 4) return launch_lanes<T, 4>(a, s);
    if (chunks <= 8) return launch_lanes<T, 8>(a, s);
    if (chunks <= 16) return launch_lanes<T, 16>(a, s);
    if (chunks <= 32) return launch_lanes<T, 32>(a, s);
    return launch_lanes<T, 64>(a, s);
}

}  // namespace

hipError_t launch_head_norm(int type, const HeadNormArgs& a, hipStream_t s)
{
    return type == RM_TYPE_BF16 ? launch_type<bf16>(a, s) : launch_type<f16>(a, s);
}

}  // namespace rm
