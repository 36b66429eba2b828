// cache.hip -- rotary positions with the append to the paged 8-bit cache
// (rm_rotary_append) and the read-back of pages (rm_cache_read).
//
// Append, one launch: the first workgroups turn the queries, a wave or more a
// token, the others own each one (page, kv head, keys or values) that gets new
// tokens, so no two write the same codes and no atomic is needed.  A thread holds 4 tokens x 8
// channels in registers: the tile that makes both sides of the page wide, 8
// consecutive key codes a token and 4 consecutive tokens a value channel.  A
// page's old codes are read only where a new token raises the scale; the rest
// of the time a decode step writes its own token's codes, and zeros to the slots
// behind it: what a table or a length that went back had left there is gone.  The
// zeros are most of what such a step writes (pages of 128: 63 slots on average).
// Bound by the traffic of the tokens and of the pages' codes.
//
// Angles: position * inv_freq in fp64, the whole turns taken off, then sine and
// cosine in fp32; at position 1e6 an fp32 product would be off by up to 0.03.
#include "rm_decode.h"

#include "rm_common.h"

namespace rm {
namespace {

constexpr int kMostPairs = 128;   // rotary pairs of a head: head_dim / 2

// Turns a position of pair `pair`, fp64.
__device__ inline double turns_of(const float* inv_freq, int pair)
{
    return (double)inv_freq[pair] * 0.15915494309189533577;
}

// Sine and cosine of position * turns whole turns, times scale.  What is left
// of the last turn goes through v_sin_f32 and v_cos_f32, which take turns: off
// by up to 1.3e-7 over [-1/2, 1/2] (measured), against 5e-8 of sincospif, whose
// instructions bound the prompts' append (7600 tokens, the same again and again:
// 47.5 us, 40.3 so, 35.2 without any angle; 51 with inputs that change).  The
// angle's own rounding to fp32 is 9e-8; of a million results in f16 each is the
// exact value's neighbour but for 1.2e-7 around the middle between two.
__device__ inline void turn_of(double turns, int32_t position, float scale, float& cs, float& sn)
{
    const double a = (double)position * turns;
    const float r = (float)(a - rint(a));
    cs = __builtin_amdgcn_cosf(r) * scale;
    sn = __builtin_amdgcn_sinf(r) * scale;
}

// Channels of pair p: the pairs of the layout first, then the pairs of
// neighbours that are copied.
__device__ inline void channels_of(int p, int rot, int layout, int& a, int& b)
{
    const int half = rot >> 1;
    if (p >= half) {
        a = 2 * p;
        b = a + 1;
    } else if (layout == RM_ROTARY_HALF) {
        a = p;
        b = p + half;
    } else {
        a = 2 * p;
        b = a + 1;
    }
}

// Pairs p0 .. p0+3 of a token's head as 8 values (first and second channels in
// turn).  wide: rot is a multiple of 8, so four pairs are two runs of four
// neighbours or one of eight.
template <typename T>
__device__ inline void load_pairs(const T* x, int p0, int rot, int layout, bool wide, float (&v)[8])
{
    typedef T V4 __attribute__((ext_vector_type(4), aligned(2)));
    if (wide && layout == RM_ROTARY_HALF && 2 * p0 < rot) {
        const V4 a = *reinterpret_cast<const V4*>(x + p0);
        const V4 b = *reinterpret_cast<const V4*>(x + p0 + (rot >> 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) v[2 * i] = (float)a[i], v[2 * i + 1] = (float)b[i];
    } else if (wide || layout == RM_ROTARY_INTERLEAVED) {
        const typename Vec<T>::x8 a = load8(x + 2 * p0);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (float)a[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            int a, b;
            channels_of(p0 + i, rot, layout, a, b);
            v[2 * i] = (float)x[a];
            v[2 * i + 1] = (float)x[b];
        }
    }
}

__device__ inline void turn_pair(float& a, float& b, float cs, float sn)
{
    const float x = a, y = b;
    a = __builtin_fmaf(x, cs, -(y * sn));
    b = __builtin_fmaf(x, sn, y * cs);
}

// a / b from b's rounded reciprocal, corrected by the remainder.
__device__ inline float quotient(float a, float b, float inv)
{
    const float q = a * inv;
    return __builtin_fmaf(__builtin_fmaf(-q, b, a), inv, q);
}

// Eight codes of `FMT` from values in units of the scale.
template <int FMT>
__device__ inline u32x2 encode8(const float (&v)[8])
{
    u32x2 r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if (FMT == RM_CODES_INT8) {
            uint32_t w = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float c = fminf(fmaxf(rintf(v[4 * h + i]), -127.0f), 127.0f);
                w |= ((uint32_t)(int)c & 255u) << (8 * i);
            }
            r[h] = w;
        } else {
            float c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = fminf(fmaxf(v[4 * h + i], -448.0f), 448.0f);
            int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[0], c[1], 0, false);
            r[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c[2], c[3], w, true);
        }
    }
    return r;
}

template <int FMT>
__device__ inline float decode_byte(uint32_t byte)
{
    if (FMT == RM_CODES_INT8) return (float)(int8_t)byte;
    return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0);
}

constexpr int kAhead = 4;         // units of 4 pairs that a lane has in flight

// The queries of one token, by `parts` waves of which this is number `part`: 4
// pairs a lane and head, the token's sines and cosines in the wave's LDS.
template <typename T>
__device__ inline void turn_queries(const AppendArgs& a, int32_t token, int part, int parts,
                                    float2* turn)
{
    typedef typename Vec<T>::x8 V;
    const int lane = threadIdx.x & 63, half = a.rot >> 1, D = a.cache.head_dim;
    const int units = D >> 3, all = a.heads * units;   // of 4 pairs
    const bool wide = (a.rot & 7) == 0;
    const T* q = static_cast<const T*>(a.q) + token * a.q_stride;
    auto load = [&](int u, float (&v)[8]) {
        load_pairs(q + u / units * a.q_head, u % units * 4, a.rot, a.layout, wide, v);
    };
    // the first turns' queries are on their way while the token is placed
    const int begin = part * (kAhead * 64) + lane;
    float ahead[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load(min(begin + i * 64, all - 1), ahead[i]);
    int32_t position = 0;
    if (a.positions) {
        position = a.positions[token];
    } else {
        // the token's sequence: each lane asks some of them
        int32_t found = 0;
        for (int b = lane; b < a.seqs.n_seqs; b += 64) {
            const Sequence s = sequence_of(a.seqs, a.cache.page_tokens, b);
            if (token >= s.first && token < s.first + s.n) found = s.length - s.n + token - s.first;
        }
        position = wave_or(found);       // sequences in order: one lane at most has it
    }
    for (int p = lane; p < half; p += 64) {
        float cs, sn;
        turn_of(turns_of(a.inv_freq, p), position, a.rot_scale, cs, sn);
        turn[p] = make_float2(cs, sn);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    auto finish = [&](int u, float (&v)[8]) {
        const int p0 = u % units * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (p0 + i < half) turn_pair(v[2 * i], v[2 * i + 1], turn[p0 + i].x, turn[p0 + i].y);
        T* out = static_cast<T*>(a.q_out) + ((int64_t)token * a.heads + u / units) * D;
        typedef T V4 __attribute__((ext_vector_type(4)));
        if (wide && a.layout == RM_ROTARY_HALF && p0 < half) {
            V4 x, y;
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = (T)v[2 * i], y[i] = (T)v[2 * i + 1];
            *reinterpret_cast<V4*>(out + p0) = x;
            *reinterpret_cast<V4*>(out + p0 + half) = y;
        } else if (wide || a.layout == RM_ROTARY_INTERLEAVED) {
            V x;
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (T)v[i];
            store8(out + 2 * p0, x);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int c0, c1;
                channels_of(p0 + i, a.rot, a.layout, c0, c1);
                out[c0] = (T)v[2 * i];
                out[c1] = (T)v[2 * i + 1];
            }
        }
    };
    for (int u0 = begin; u0 - lane < all; u0 += parts * (kAhead * 64)) {
        if (u0 != begin) {
#pragma unroll
            for (int i = 0; i < kAhead; ++i) load(min(u0 + i * 64, all - 1), ahead[i]);
        }
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
            if (u0 + i * 64 < all) finish(u0 + i * 64, ahead[i]);
    }
}

template <typename T, int FMT>
__global__ __launch_bounds__(1024) void append_kernel(AppendArgs a, int32_t q_blocks,
                                                      int32_t q_parts, int32_t pages_a_seq,
                                                      int32_t group, uint32_t first)
{
    __shared__ float2 turn[16][kMostPairs];
    __shared__ float part[16];
    const uint32_t index = first + blockIdx.x;      // 31 bits at most (kMostBlocks)
    if (index < (uint32_t)q_blocks) {
        const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
        const int64_t at = (int64_t)index * waves + wave, token = at / q_parts;
        if (token < a.seqs.n_tokens)
            turn_queries<T>(a, (int32_t)token, (int)(at % q_parts), q_parts, turn[wave]);
        return;
    }
    // `group` threads a (page, head, side); the groups of a workgroup share
    // the sequence and page and take neighbouring (head, side)
    const int TK = a.cache.page_tokens, D = a.cache.head_dim, KV = a.cache.kv_heads;
    const int groups = blockDim.x / group, sides = 2 * KV;
    const int per_page = (sides + groups - 1) / groups;
    uint32_t at = index - (uint32_t)q_blocks;
    const int part_of = (int)(at % (uint32_t)per_page);
    at /= (uint32_t)per_page;
    const int page_no = (int)(at % (uint32_t)pages_a_seq), b = (int)(at / (uint32_t)pages_a_seq);
    const Sequence s = sequence_of(a.seqs, TK, b);
    if (s.bad && a.status && threadIdx.x == 0) atomicOr(a.status, RM_ST_BAD_LENGTH);
    const int start = s.length - s.n;                       // first new token
    const int page_at = start / TK + page_no;
    if (s.n == 0 || (int64_t)page_at * TK >= s.length) return;
    const int32_t page = a.seqs.table[(int64_t)b * a.seqs.table_stride + page_at];
    if (page < 0 || page >= a.cache.n_pages) {
        if (a.status && threadIdx.x == 0) atomicOr(a.status, RM_ST_BAD_PAGE);
        return;
    }
    const int older = max(0, start - page_at * TK), upto = min(TK, s.length - page_at * TK);
    const int g = threadIdx.x / group, t = threadIdx.x % group;
    const int side = part_of * groups + g;
    const bool mine = side < sides;
    const int head = side >> 1, value = side & 1;
    const int units = D >> 3;                               // of 8 channels
    // neighbouring lanes: neighbouring units for keys, whose tokens are rows,
    // and neighbouring tokens for values, whose channels are
    const int quads = TK >> 2;
    const int unit = value ? t / quads : t % units;
    const int slot0 = 4 * (value ? t % quads : t / units);
    const bool in = mine && unit < units && slot0 < TK;
    const bool wide = (a.rot & 7) == 0;
    float v[4][8];
    float top = 0.0f;
    const bool turned = !value && in && 8 * unit < a.rot;
    double turns[4] = {};
    if (turned) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * unit + i < (a.rot >> 1)) turns[i] = turns_of(a.inv_freq, 4 * unit + i);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int slot = slot0 + j;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
        if (!in || slot < older || slot >= upto) continue;
        const int64_t token = s.first + (int64_t)page_at * TK + slot - start;
        if (value) {
            const typename Vec<T>::x8 x = load8(static_cast<const T*>(a.v) + token * a.v_stride +
                                                head * a.v_head + 8 * unit);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = (float)x[i];
        } else {
            load_pairs(static_cast<const T*>(a.k) + token * a.k_stride + head * a.k_head,
                       4 * unit, a.rot, a.layout, wide, v[j]);
            if (turned) {
                const int32_t position = a.positions ? a.positions[token]
                                                     : page_at * TK + slot;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (4 * unit + i >= (a.rot >> 1)) continue;
                    float cs, sn;
                    turn_of(turns[i], position, a.rot_scale, cs, sn);
                    turn_pair(v[j][2 * i], v[j][2 * i + 1], cs, sn);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) top = MaxNan::of(top, fabsf(v[j][i]));
    }
    const float Q = FMT == RM_CODES_INT8 ? 127.0f : 448.0f;
    float* scales = value ? a.cache.v_scale : a.cache.k_scale;
    const int64_t block = (int64_t)page * KV + head;
    const float was = mine && older ? scales[block] : 0.0f;
    // largest magnitude of the group: whole waves
    top = wave_reduce<MaxNan>(top);
    if (group > 64) {
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
        __syncthreads();
        top = part[g * (group >> 6)];
        for (int w = 1; w < group >> 6; ++w) top = MaxNan::of(top, part[g * (group >> 6) + w]);
    }
    if (!mine) return;
    const float now = MaxNan::of(was, top / Q);
    const bool raised = !(now == was);
    // value / scale = value * num / den.  With den the largest magnitude itself a
    // quotient halfway between two codes comes out halfway; a scale in fp32's
    // subnormal range is not that magnitude / Q to the last place, so there the
    // codes count in the scale as it is stored
    const bool by_top = raised && now >= 0x1p-126f;
    float num = by_top ? Q : 1.0f, den = by_top ? top : now;
    // both times the power of two that brings den to [1/2, 1), or near it where den
    // is subnormal: a value times Q itself passes fp32 from 3.4e38 / Q on, and the
    // reciprocal of a small den would be no number
    const int power = max(__builtin_amdgcn_frexp_expf(den), -120);
    num = ldexpf(num, -power);
    den = ldexpf(den, -power);
    const float inv = den > 0.0f ? 1.0f / den : 0.0f;
    if (t == 0) scales[block] = now;                // all have read the old one
    if (!in) return;
    uint8_t* codes = static_cast<uint8_t*>(value ? a.cache.v : a.cache.k) + block * TK * D;
    const bool rescale = older > 0 && raised;
    const float ratio = rescale ? was / now : 0.0f;
    // what is written: the new tokens and zeros behind them, and with a raised
    // scale the older ones too
    const int lo = rescale ? 0 : older;
    if (slot0 + 3 < lo) return;
    if (value) {
        // channel by channel the four tokens of the thread: one word
        const bool whole = slot0 >= lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint8_t* at_c = codes + (8 * unit + i) * TK + slot0;
            float c[8] = {};
            if (rescale && slot0 < older) {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(at_c);
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (slot0 + j < older) c[j] = decode_byte<FMT>(w >> (8 * j) & 255u) * ratio;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (slot0 + j >= older) c[j] = quotient(v[j][i] * num, den, inv);
            const uint32_t w = encode8<FMT>(c)[0];
            if (whole) {
                *reinterpret_cast<uint32_t*>(at_c) = w;
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (slot0 + j >= lo) at_c[j] = (uint8_t)(w >> (8 * j));
            }
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int slot = slot0 + j;
        if (slot < lo) continue;
        uint8_t* row = codes + slot * D;
        float c[8];
        const int half = a.rot >> 1;
        const bool split = a.layout == RM_ROTARY_HALF && 8 * unit < a.rot;
        if (slot < older) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int c0, c1;
                channels_of(4 * unit + i, a.rot, a.layout, c0, c1);
                c[2 * i] = decode_byte<FMT>(row[c0]) * ratio;
                c[2 * i + 1] = decode_byte<FMT>(row[c1]) * ratio;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = quotient(v[j][i] * num, den, inv);
        }
        if (wide && split) {
            const float d[8] = {c[0], c[2], c[4], c[6], c[1], c[3], c[5], c[7]};
            const u32x2 w = encode8<FMT>(d);
            *reinterpret_cast<uint32_t*>(row + 4 * unit) = w[0];
            *reinterpret_cast<uint32_t*>(row + half + 4 * unit) = w[1];
        } else if (wide || !split) {
            const u32x2 w = encode8<FMT>(c);
            *reinterpret_cast<u32x2*>(row + 8 * unit) = w;
        } else {
            const u32x2 w = encode8<FMT>(c);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                int c0, c1;
                channels_of(4 * unit + i, a.rot, a.layout, c0, c1);
                row[c0] = (uint8_t)(w[i >> 1] >> (16 * (i & 1)));
                row[c1] = (uint8_t)(w[i >> 1] >> (16 * (i & 1) + 8));
            }
        }
    }
}

// A thread: 4 tokens x 8 channels of one (page, head), keys or values.
template <typename T, int FMT>
__global__ __launch_bounds__(256) void cache_read_kernel(rm_cache c, int32_t n,
                                                         const int32_t* pages, T* k, T* v,
                                                         int32_t* status)
{
    const int TK = c.page_tokens, D = c.head_dim, units = D >> 3, quads = TK >> 2;
    const int tile = quads * units;                     // threads a (page, head, side)
    const int64_t all = (int64_t)n * c.kv_heads * 2 * tile;
    int32_t st = 0;
    for (int64_t u = (int64_t)blockIdx.x * 256 + threadIdx.x; u < all;
         u += (int64_t)gridDim.x * 256) {
        const int t = (int)(u % tile);
        const int64_t side = u / tile;
        const int value = (int)(side & 1), head = (int)(side / 2 % c.kv_heads);
        const int64_t at = side / 2 / c.kv_heads;
        const int32_t page = pages[at];
        const bool known = page >= 0 && page < c.n_pages;
        if (!known) st = RM_ST_BAD_PAGE;
        // neighbouring lanes take neighbouring channels of a token, which are
        // consecutive in the output
        const int unit = t % units, slot0 = t / units * 4;
        const int64_t block = known ? (int64_t)page * c.kv_heads + head : 0;
        const float scale = known ? (value ? c.v_scale : c.k_scale)[block] : 0.0f;
        typename Vec<T>::x8 o[4];
        uint32_t w[8] = {};
        if (known) {
            const uint8_t* codes = static_cast<const uint8_t*>(value ? c.v : c.k) +
                                   block * TK * D;
            if (value) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    w[i] = *reinterpret_cast<const uint32_t*>(codes + (8 * unit + i) * TK + slot0);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const u32x2 r = *reinterpret_cast<const u32x2*>(codes + (slot0 + j) * D +
                                                                    8 * unit);
                    w[2 * j] = r[0];
                    w[2 * j + 1] = r[1];
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t byte = value ? w[i] >> (8 * j) & 255u
                                            : w[2 * j + (i >> 2)] >> (8 * (i & 3)) & 255u;
                o[j][i] = (T)(known ? decode_byte<FMT>(byte) * scale : 0.0f);
            }
            T* out = (value ? v : k) + ((at * TK + slot0 + j) * c.kv_heads + head) * D + 8 * unit;
            store8(out, o[j]);
        }
    }
    report_status(status, st);
}

}  // namespace

namespace {

// How an append is laid out.
struct AppendPlan {
    int group, threads;       // threads a (page, head, side), and a workgroup
    int32_t pages, q_parts;   // pages a sequence, waves a token for its queries
    int64_t q_blocks, blocks;
};

AppendPlan append_plan(const rm_cache& c, const rm_sequences& s, int32_t heads)
{
    const int TK = c.page_tokens, tile = TK * c.head_dim / 32;
    AppendPlan p;
    p.pages = (int32_t)((most_tokens(s) + 2 * TK - 2) / TK);
    p.group = tile < 64 ? 64 : tile;
    p.threads = p.group < 256 ? 256 : p.group;
    const int groups = p.threads / p.group, waves = p.threads / 64;
    // Waves a token: as many as its queries fill once, while all are 16 a CU at
    // most (17 tokens of 64 heads of 256, with the read back: 10.6 us, a wave a
    // token 31.6; 64 tokens of 32 heads of 128: 10.1 and 12.0).
    const int64_t fill = ((int64_t)heads * (c.head_dim / 8) + kAhead * 64 - 1) / (kAhead * 64);
    const int64_t room = 16 * kComputeUnits / s.n_tokens;
    p.q_parts = (int32_t)(room < 1 ? 1 : room < fill ? room : fill < 1 ? 1 : fill);
    p.q_blocks = heads > 0 ? ((int64_t)s.n_tokens * p.q_parts + waves - 1) / waves : 0;
    const int64_t per_page = (2 * (int64_t)c.kv_heads + groups - 1) / groups;
    p.blocks = p.q_blocks + (int64_t)s.n_seqs * p.pages * per_page;
    return p;
}

}  // namespace

bool append_fits(const rm_cache& c, const rm_sequences& s, int32_t heads)
{
    return append_plan(c, s, heads).blocks <= kMostBlocks;
}

hipError_t launch_append(int type, const AppendArgs& a, hipStream_t s)
{
    const AppendPlan p = append_plan(a.cache, a.seqs, a.heads);
    const int64_t most = most_blocks((unsigned)p.threads);
    auto run = [&](auto kernel) {
        hipError_t e = hipSuccess;
        for (int64_t first = 0; first < p.blocks && e == hipSuccess; first += most)
            e = launch(kernel, dim3((unsigned)(p.blocks - first < most ? p.blocks - first : most)),
                       (unsigned)p.threads, 0, s, a, (int32_t)p.q_blocks, p.q_parts, p.pages,
                       (int32_t)p.group, (uint32_t)first);
        return e;
    };
    if (type == RM_TYPE_BF16)
        return a.cache.codes == RM_CODES_INT8 ? run(append_kernel<bf16, RM_CODES_INT8>)
                                              : run(append_kernel<bf16, RM_CODES_E4M3>);
    return a.cache.codes == RM_CODES_INT8 ? run(append_kernel<f16, RM_CODES_INT8>)
                                          : run(append_kernel<f16, RM_CODES_E4M3>);
}

hipError_t launch_cache_read(int type, const rm_cache& c, int32_t n, const int32_t* pages,
                             void* k, void* v, int32_t* status, hipStream_t s)
{
    const int64_t all = (int64_t)n * c.kv_heads * 2 * (c.page_tokens * c.head_dim / 32);
    const int64_t want = (all + 255) / 256, most = 16 * kComputeUnits;
    const dim3 grid((unsigned)(want < most ? want : most));
    if (want == 0) return hipSuccess;
#define RM_READ(T, FMT) \
    return launch(cache_read_kernel<T, FMT>, grid, 256u, 0, s, c, n, pages, \
                  static_cast<T*>(k), static_cast<T*>(v), status)
    if (type == RM_TYPE_BF16) {
        if (c.codes == RM_CODES_INT8) RM_READ(bf16, RM_CODES_INT8);
        RM_READ(bf16, RM_CODES_E4M3);
    }
    if (c.codes == RM_CODES_INT8) RM_READ(f16, RM_CODES_INT8);
    RM_READ(f16, RM_CODES_E4M3);
#undef RM_READ
}

}  // namespace rm
