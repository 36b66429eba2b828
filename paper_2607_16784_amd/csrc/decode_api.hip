// decode_api.hip -- the extern "C" entry points of the decode-layer kernels:
// host-side argument checks, launches and the record of launch shapes.
#include <cmath>
#include <new>

#include "rm_common.h"
#include "rm_decode.h"

namespace rm {

namespace {

struct Recording {
    rm_launch* records = nullptr;
    float* microseconds = nullptr;       // nullptr: without times
    hipEvent_t* events = nullptr;        // start and end of each launch
    int32_t capacity = 0, count = 0;
    bool on = false;
};
thread_local Recording g_recording;

int begin(rm_launch* records, float* microseconds, hipEvent_t* events, int32_t capacity)
{
    Recording& r = g_recording;
    r.records = records;
    r.microseconds = microseconds;
    r.events = events;
    r.capacity = capacity;
    r.count = 0;
    r.on = true;
    return RM_OK;
}

int done(hipError_t e)
{
    return e == hipSuccess ? RM_OK : launch_failed(e);
}

bool type_ok(int32_t type)
{
    return type == RM_TYPE_BF16 || type == RM_TYPE_F16;
}

// RM_OK, or what is wrong with a cache.
int check_cache(const rm_cache* c)
{
    if (!c || c->n_pages < 0 || c->kv_heads < 1) return RM_EINVAL;
    if (c->codes != RM_CODES_INT8 && c->codes != RM_CODES_E4M3) return RM_EINVAL;
    if (c->n_pages > 0 && (!c->k || !c->v || !c->k_scale || !c->v_scale)) return RM_EINVAL;
    // the kernels read and write codes 16 bytes at a time
    if (((uintptr_t)c->k | (uintptr_t)c->v) & 15) return RM_EINVAL;
    const int32_t t = c->page_tokens, d = c->head_dim;
    if (t != 16 && t != 32 && t != 64 && t != 128) return RM_EUNSUPPORTED;
    if (d != 64 && d != 128 && d != 256) return RM_EUNSUPPORTED;
    if (c->kv_heads > 65535) return RM_EUNSUPPORTED;
    return RM_OK;
}

int check_seqs(const rm_sequences* s, const rm_cache* c)
{
    if (!s || s->n_seqs < 0 || s->table_stride < 0 || s->n_tokens < 0 || s->max_tokens < 0)
        return RM_EINVAL;
    if (s->n_seqs > 0 && (!s->lengths || (s->table_stride > 0 && !s->table))) return RM_EINVAL;
    if (!s->token_offsets && (s->n_tokens != s->n_seqs || (s->n_seqs > 0 && s->max_tokens < 1)))
        return RM_EINVAL;
    if (s->n_seqs > RM_MAX_SEQUENCES) return RM_EUNSUPPORTED;
    // token indexes are 32 bits
    if ((int64_t)s->table_stride * c->page_tokens > 0x7fffff00) return RM_EUNSUPPORTED;
    return RM_OK;
}

// (token, head) pairs of a sequence and kv head are counted in 32 bits, and so
// are the workgroups.
bool rows_fit(const rm_sequences* s, const rm_cache* c, int32_t heads)
{
    return (int64_t)s->max_tokens * (heads / c->kv_heads) <= 0x7fffff00 &&
           attend_fits(*c, *s, heads);
}

// floor(k / group) = umulhi(k / 32, inverse) for every column below k: the
// product's error, k / 32 / 2^32, stays below 32 / group for k <= 2^21.
uint32_t inverse_of(int32_t group)
{
    const uint32_t d = (uint32_t)group / 32;
    return d <= 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + d - 1) / d);
}

}  // namespace

void note_launch(const void* kernel, int64_t blocks, unsigned threads, size_t dynamic_lds)
{
    Recording& r = g_recording;
    if (!r.on) return;
    if (r.count < r.capacity) {
        rm_launch& l = r.records[r.count];
        l.grid = (int32_t)(blocks < 0x7fffffff ? blocks : 0x7fffffff);
        l.threads = (int32_t)threads;
        hipFuncAttributes f;
        const bool known = hipFuncGetAttributes(&f, kernel) == hipSuccess;
        l.regs = known ? f.numRegs : 0;
        l.smem = (int32_t)(dynamic_lds + (known ? f.sharedSizeBytes : 0));
    }
    if (r.count < 0x7fffffff) ++r.count;
}

hipError_t launch_events(hipStream_t s, hipEvent_t& begin, hipEvent_t& end)
{
    begin = end = nullptr;
    const Recording& r = g_recording;
    if (!r.events || r.count >= r.capacity) return hipSuccess;
    hipStreamCaptureStatus capture;
    hipError_t e = hipStreamIsCapturing(s, &capture);
    if (e != hipSuccess) return e;
    if (capture != hipStreamCaptureStatusNone) return hipErrorStreamCaptureUnsupported;
    hipEvent_t* at = r.events + 2 * (int64_t)r.count;
    for (int i = 0; i < 2; ++i)
        if (!at[i] && (e = hipEventCreate(&at[i])) != hipSuccess) return e;
    begin = at[0];
    end = at[1];
    return hipSuccess;
}

}  // namespace rm

extern "C" {

size_t rm_w4_linear_workspace_bytes(int32_t rows, int32_t n, int32_t k, int32_t act)
{
    if (rows < 1 || n < 1 || k < 1 || k > RM_MAX_W4_COLUMNS || n > RM_MAX_W4_OUTPUTS ||
        rows > RM_MAX_W4_ROWS)
        return 0;
    return rm::linear_workspace(rows, n, k, act);
}

int rm_w4_linear(int32_t type, int32_t rows, int32_t n, int32_t k, const void* x,
                 int64_t x_stride, const uint8_t* codes, int64_t code_stride, int32_t group,
                 const void* scales, const uint8_t* zeros, const void* bias, int32_t act,
                 void* y, int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!rm::type_ok(type) || rows < 0 || n < 1 || k < 1 || group < 1 || group % 32)
        return RM_EINVAL;
    if (act != RM_ACT_NONE && act != RM_ACT_SWIGLU) return RM_EINVAL;
    if (act == RM_ACT_SWIGLU && n % 2) return RM_EINVAL;
    const int32_t out = act == RM_ACT_SWIGLU ? n / 2 : n;
    if (x_stride < k || code_stride < (k + 1) / 2 || y_stride < out) return RM_EINVAL;
    if (k > RM_MAX_W4_COLUMNS || n > RM_MAX_W4_OUTPUTS || rows > RM_MAX_W4_ROWS)
        return RM_EUNSUPPORTED;
    // a group beyond k is the one group of k: sums of sizes stay within 32 bits
    if (group > k) group = (k + 31) / 32 * 32;
    if (rows == 0) return RM_OK;
    if (!x || !codes || !scales || !y) return RM_EINVAL;
    const size_t need = rm::linear_workspace(rows, n, k, act);
    if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255)))
        return RM_EWORKSPACE;
    rm::LinearArgs a = {rows, n, k, group, x, codes, scales, zeros, bias, y, workspace,
                        rm::inverse_of(group), x_stride, code_stride, y_stride};
    return rm::done(rm::launch_linear(type, act, a, (hipStream_t)stream));
}

int rm_rotary_append(int32_t type, const rm_cache* cache, const rm_sequences* seqs,
                     int32_t heads, const void* q, int64_t q_stride, int64_t q_head_stride,
                     const void* k, int64_t k_stride, int64_t k_head_stride, const void* v,
                     int64_t v_stride, int64_t v_head_stride, const int32_t* positions,
                     const float* inv_freq, int32_t rot, int32_t layout, float rot_scale,
                     void* q_out, int32_t* status, void* stream)
{
    int e = rm::check_cache(cache);
    if (e == RM_OK) e = rm::check_seqs(seqs, cache);
    if (e != RM_OK) return e;
    if (!rm::type_ok(type) || heads < 0 || rot < 0 || rot % 2 || rot > cache->head_dim)
        return RM_EINVAL;
    if (layout != RM_ROTARY_HALF && layout != RM_ROTARY_INTERLEAVED) return RM_EINVAL;
    if (heads > 65535) return RM_EUNSUPPORTED;
    if (seqs->n_tokens == 0) return RM_OK;
    if (cache->n_pages < 1) return RM_EINVAL;
    if (!k || !v || (heads > 0 && (!q || !q_out)) || (rot > 0 && !inv_freq)) return RM_EINVAL;
    if (!rm::append_fits(*cache, *seqs, heads)) return RM_EUNSUPPORTED;
    rm::AppendArgs a = {*cache, *seqs, heads, rot, layout, q, k, v, q_stride, q_head_stride,
                        k_stride, k_head_stride, v_stride, v_head_stride, positions, inv_freq,
                        rot_scale, q_out, status};
    return rm::done(rm::launch_append(type, a, (hipStream_t)stream));
}

int rm_cache_read(int32_t type, const rm_cache* cache, int32_t n, const int32_t* pages, void* k,
                  void* v, int32_t* status, void* stream)
{
    const int e = rm::check_cache(cache);
    if (e != RM_OK) return e;
    if (!rm::type_ok(type) || n < 0) return RM_EINVAL;
    if (n == 0) return RM_OK;
    if (!pages || !k || !v || cache->n_pages < 1) return RM_EINVAL;
    return rm::done(rm::launch_cache_read(type, *cache, n, pages, k, v, status,
                                          (hipStream_t)stream));
}

size_t rm_cache_attention_workspace_bytes(const rm_cache* cache, const rm_sequences* seqs,
                                          int32_t heads)
{
    if (rm::check_cache(cache) != RM_OK || rm::check_seqs(seqs, cache) != RM_OK) return 0;
    if (heads < 1 || heads % cache->kv_heads || !rm::rows_fit(seqs, cache, heads)) return 0;
    return rm::attend_workspace(*cache, *seqs, heads);
}

int rm_cache_attention(int32_t type, const rm_cache* cache, const rm_sequences* seqs,
                       int32_t heads, const void* q, int64_t q_stride, int64_t q_head_stride,
                       float scale, int32_t window, void* out, void* workspace,
                       size_t workspace_bytes, int32_t* status, void* stream)
{
    int e = rm::check_cache(cache);
    if (e == RM_OK) e = rm::check_seqs(seqs, cache);
    if (e != RM_OK) return e;
    if (!rm::type_ok(type) || heads < 1 || heads % cache->kv_heads || window < 0 ||
        !std::isfinite(scale))
        return RM_EINVAL;
    if (!rm::rows_fit(seqs, cache, heads)) return RM_EUNSUPPORTED;
    if (seqs->n_tokens == 0) return RM_OK;
    if (!q || !out || cache->n_pages < 1) return RM_EINVAL;
    const size_t need = rm::attend_workspace(*cache, *seqs, heads);
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255))
        return RM_EWORKSPACE;
    rm::AttendArgs a = {*cache, *seqs, heads, window, q, q_stride, q_head_stride, scale, out,
                        workspace, status};
    return rm::done(rm::launch_attend(type, a, (hipStream_t)stream));
}

int rm_norm_residual(int32_t type, int32_t kind, int32_t rows, int32_t width, const void* x,
                     int64_t x_stride, const void* y, int64_t y_stride, const void* gate,
                     int64_t gate_stride, int32_t gate_width, const void* post_weight,
                     const void* pre_weight, const void* pre_bias, float alpha, float eps,
                     void* x_out, void* n_out, void* stream)
{
    if (!rm::type_ok(type) || (kind != RM_NORM_RMS && kind != RM_NORM_LAYER)) return RM_EINVAL;
    if (rows < 0 || width < 1 || !std::isfinite(alpha) || !std::isfinite(eps)) return RM_EINVAL;
    if (width > RM_MAX_NORM_WIDTH) return RM_EUNSUPPORTED;
    if (rows == 0) return RM_OK;
    if (!x || (!x_out && !n_out) || (!y && (gate || post_weight))) return RM_EINVAL;
    if (x_stride < width || (y && y_stride < width)) return RM_EINVAL;
    if (gate && gate_width != width && gate_width != 1) return RM_EINVAL;
    if (gate && gate_stride != 0 && gate_stride < gate_width) return RM_EINVAL;
    rm::NormArgs a = {rows, width, gate ? gate_width : 0, x, y, gate, post_weight, pre_weight,
                      pre_bias, x_stride, y_stride, gate_stride, alpha, eps, x_out, n_out};
    return rm::done(rm::launch_norm(type, kind, a, (hipStream_t)stream));
}

int rm_head_norm_rotary(int32_t type, int32_t n_tokens, int32_t heads, int32_t kv_heads,
                        int32_t head_dim, const void* q, int64_t q_stride, int64_t q_head_stride,
                        const void* k, int64_t k_stride, int64_t k_head_stride,
                        const void* q_weight, const void* k_weight, const int32_t* positions,
                        const float* inv_freq, int32_t rot, int32_t layout, float rot_scale,
                        float eps, void* q_out, int64_t q_out_stride, int64_t q_out_head_stride,
                        void* k_out, int64_t k_out_stride, int64_t k_out_head_stride,
                        void* stream)
{
    if (!rm::type_ok(type) || n_tokens < 0 || heads < 0 || kv_heads < 0 || head_dim < 1 ||
        rot < 0 || rot % 2 || rot > head_dim)
        return RM_EINVAL;
    if (layout != RM_ROTARY_HALF && layout != RM_ROTARY_INTERLEAVED) return RM_EINVAL;
    if (!std::isfinite(rot_scale) || !std::isfinite(eps)) return RM_EINVAL;
    if (head_dim % 8 || head_dim > RM_MAX_HEAD_WIDTH || heads > 65535 || kv_heads > 65535)
        return RM_EUNSUPPORTED;
    if (n_tokens == 0 || (heads == 0 && kv_heads == 0)) return RM_OK;
    if ((heads > 0 && (!q || !q_out)) || (kv_heads > 0 && (!k || !k_out))) return RM_EINVAL;
    if (rot > 0 && (!positions || !inv_freq)) return RM_EINVAL;
    rm::HeadNormArgs a = {n_tokens, heads, kv_heads, head_dim, rot, layout, q, k, q_stride,
                          q_head_stride, k_stride, k_head_stride, q_weight, k_weight, positions,
                          inv_freq, rot_scale, eps, q_out, k_out, q_out_stride, q_out_head_stride,
                          k_out_stride, k_out_head_stride};
    return rm::done(rm::launch_head_norm(type, a, (hipStream_t)stream));
}

int rm_prompt_attention(int32_t type, int32_t n_tokens, int32_t heads, int32_t kv_heads,
                        int32_t head_dim, const void* q, int64_t q_stride, int64_t q_head_stride,
                        const void* k, int64_t k_stride, int64_t k_head_stride, const void* v,
                        int64_t v_stride, int64_t v_head_stride, const int32_t* token_offsets,
                        int32_t n_seqs, int32_t max_tokens, float scale, int32_t window,
                        void* out, int32_t* status, void* stream)
{
    if (!rm::type_ok(type) || n_tokens < 0 || n_seqs < 0 || max_tokens < 0 || kv_heads < 1 ||
        heads < 1 || heads % kv_heads || window < 0 || !std::isfinite(scale * rm::kLog2e))
        return RM_EINVAL;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return RM_EUNSUPPORTED;
    if (n_seqs > RM_MAX_SEQUENCES || heads > 65535) return RM_EUNSUPPORTED;
    if ((int64_t)max_tokens * (heads / kv_heads) > 0x7fffff00) return RM_EUNSUPPORTED;
    rm::PromptArgs a = {n_tokens, heads, kv_heads, n_seqs, max_tokens, window, q, k, v, q_stride,
                        q_head_stride, k_stride, k_head_stride, v_stride, v_head_stride,
                        token_offsets, scale, out, status};
    if (!rm::prompt_fits(a)) return RM_EUNSUPPORTED;
    if (n_tokens == 0) return RM_OK;
    if (!q || !k || !v || !out || !token_offsets) return RM_EINVAL;
    return rm::done(rm::launch_prompt(type, head_dim, a, (hipStream_t)stream));
}

int rm_f8_quantize(int32_t type, int32_t rows, int32_t k, const void* x, int64_t x_stride,
                   int32_t block_rows, uint8_t* codes, int64_t code_stride, float* scales,
                   void* stream)
{
    if (!rm::type_ok(type) || rows < 0 || k < 1 || x_stride < k || code_stride < k ||
        (block_rows != 1 && block_rows != 128))
        return RM_EINVAL;
    if (k > RM_MAX_F8_COLUMNS) return RM_EUNSUPPORTED;
    if (rows == 0) return RM_OK;
    if (!x || !codes || !scales) return RM_EINVAL;
    rm::QuantizeArgs a = {rows, k, x, x_stride, codes, code_stride, scales};
    return rm::done(rm::launch_quantize(type, block_rows, a, (hipStream_t)stream));
}

size_t rm_f8_linear_workspace_bytes(int32_t rows, int32_t n, int32_t k, int32_t act)
{
    if (rows < 1 || n < 1 || k < 1 || k > RM_MAX_F8_COLUMNS || n > RM_MAX_F8_OUTPUTS ||
        rows > RM_MAX_F8_ROWS)
        return 0;
    return rm::f8_workspace(rows, n, k, act);
}

int rm_f8_linear(int32_t type, int32_t rows, int32_t n, int32_t k, const void* x,
                 int64_t x_stride, const float* x_scales, const uint8_t* codes,
                 int64_t code_stride, const float* scales, const void* bias, int32_t act, void* y,
                 int64_t y_stride, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!rm::type_ok(type) || rows < 0 || n < 1 || k < 1) return RM_EINVAL;
    if (act != RM_ACT_NONE && act != RM_ACT_SWIGLU) return RM_EINVAL;
    if (act == RM_ACT_SWIGLU && n % 2) return RM_EINVAL;
    if (x_stride < k || code_stride < k || y_stride < (act == RM_ACT_SWIGLU ? n / 2 : n))
        return RM_EINVAL;
    if (k > RM_MAX_F8_COLUMNS || n > RM_MAX_F8_OUTPUTS || rows > RM_MAX_F8_ROWS)
        return RM_EUNSUPPORTED;
    if (rows == 0) return RM_OK;
    if (!x || !codes || !scales || !y) return RM_EINVAL;
    const size_t need = rm::f8_workspace(rows, n, k, act);
    if (need > 0 && (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255)))
        return RM_EWORKSPACE;
    rm::F8Args a = {rows, n, k, act, x, x_stride, x_scales, codes, code_stride, scales, bias, y,
                    y_stride, workspace};
    return rm::done(rm::launch_f8(type, a, (hipStream_t)stream));
}

int rm_trace_begin(rm_launch* records, int32_t capacity)
{
    if (rm::g_recording.on || capacity < 0 || (capacity > 0 && !records)) return RM_EINVAL;
    return rm::begin(records, nullptr, nullptr, capacity);
}

int rm_trace_begin_timed(rm_launch* records, float* microseconds, int32_t capacity)
{
    if (rm::g_recording.on || capacity < 0 || (capacity > 0 && (!records || !microseconds)))
        return RM_EINVAL;
    hipEvent_t* events = new (std::nothrow) hipEvent_t[2 * (size_t)capacity + 1]();
    if (!events) return rm::launch_failed(hipErrorOutOfMemory);
    return rm::begin(records, microseconds, events, capacity);
}

int rm_trace_end(int32_t* n_launches)
{
    rm::Recording& r = rm::g_recording;
    if (!r.on || !n_launches) return RM_EINVAL;
    *n_launches = r.count;
    hipError_t failed = hipSuccess;
    for (int64_t i = 0; r.events && i < r.capacity; ++i) {
        hipEvent_t* at = r.events + 2 * i;
        if (i < r.count) {
            float ms = 0.0f;
            hipError_t e = hipEventSynchronize(at[1]);
            if (e == hipSuccess) e = hipEventElapsedTime(&ms, at[0], at[1]);
            if (failed == hipSuccess) failed = e;
            r.microseconds[i] = ms * 1e3f;
        }
        for (int k = 0; k < 2; ++k)
            if (at[k]) (void)hipEventDestroy(at[k]);
    }
    delete[] r.events;
    r = rm::Recording();
    return rm::done(failed);
}

}  // extern "C"
