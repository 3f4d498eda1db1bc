// C entries of the operators on device tensors (include/ppipe.h): argument
// checks, then one launcher each.  Every check comes before any device work.
#include "operators.h"
#include "ppipe.h"

#include <cmath>
#include <string>

using namespace ppipe;

namespace {

int bad(const std::string& msg) { return set_error(PPIPE_E_INVALID, msg); }
int unsupported(const std::string& msg) { return set_error(PPIPE_E_UNSUPPORTED, msg); }

int launched(const char* what, hipError_t e)
{
    if (e == hipSuccess) return PPIPE_OK;
    return set_error(PPIPE_E_HIP, std::string(what) + ": " + hipGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}  // namespace

int ppipe::device_cus()
{
    int dev = 0, n = 0;
    if (hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && n > 0)
        return n;
    return 256;
}

int ppipe::check_group_norm(int dt, int64_t batch, int64_t pixels, int C, int G, float eps, int act,
                            const std::string& who)
{
    if (dt < PPIPE_F32 || dt > PPIPE_BF16) return bad(who + "unknown dtype " + std::to_string(dt));
    if (batch < 0 || pixels < 0 || C < 1 || G < 1)
        return bad(who + "need batch, pixels >= 0 and channels, groups >= 1");
    if (C % G) return bad(who + "channels must be a multiple of the groups");
    if (act < PPIPE_ACT_NONE || act > PPIPE_ACT_GELU) return bad(who + "unknown activation");
    if (!(eps >= 0.0f) || std::isinf(eps)) return bad(who + "eps must be finite and >= 0");
    const int epv = 16 / dtype_size(dt);
    if (C % epv || C > GROUP_NORM_MAX_C)
        return unsupported(who + "group norm needs channels % " + std::to_string(epv) +
                           " == 0, at most " + std::to_string(GROUP_NORM_MAX_C));
    if (batch * pixels > 0x7fffffff ||
        (batch && pixels && !group_norm_fits(dt, (int)batch, (int)pixels, C, G, device_cus())))
        return unsupported(who + "group norm of this many images or pixels is not supported");
    return PPIPE_OK;
}

namespace {

// Strides between (batch items, tokens, heads) of a tensor with these sizes:
// whole 16-byte vectors, none negative.
int check_strides(const char* what, const int64_t* st, const int64_t* n, int esz)
{
    const int64_t epv = 16 / esz;
    for (int i = 0; i < 3; ++i) {
        if (n[i] <= 1) continue;
        if (st[i] < 0) return bad(std::string(what) + ": negative stride");
        if (st[i] % epv)
            return unsupported(std::string(what) + ": strides must be multiples of 16 bytes");
        if (i > 0 && st[i] >= ROW_STRIDE_LIMIT)
            return unsupported(std::string(what) + ": token and head strides must be below 2^22");
        if (i == 0 && st[i] > ((int64_t)1 << 56) / n[i])
            return unsupported(std::string(what) + ": batch stride too large");
    }
    return PPIPE_OK;
}

// Strides between batch items of positions and spans.
int check_batch_stride(int64_t st, int64_t batch, const std::string& who)
{
    if (st < 0) return bad(who + "negative stride");
    if (batch > 1 && st > ((int64_t)1 << 56) / batch)
        return unsupported(who + "batch stride too large");
    return PPIPE_OK;
}

// Whether two elements of a tensor written by these strides share memory.
bool overlaps_itself(const int64_t* st, const int64_t* n, int d)
{
    int64_t s[3], m[3];
    int k = 0;
    if (!n[0] || !n[1] || !n[2]) return false;
    for (int i = 0; i < 3; ++i)
        if (n[i] > 1) {
            s[k] = st[i];
            m[k++] = n[i];
        }
    for (int i = 0; i < k; ++i)
        for (int j = i + 1; j < k; ++j)
            if (s[j] < s[i]) {
                std::swap(s[i], s[j]);
                std::swap(m[i], m[j]);
            }
    int64_t reach = d;
    for (int i = 0; i < k; ++i) {
        if (s[i] < reach) return true;
        reach += s[i] * (m[i] - 1);
    }
    return false;
}

}  // namespace

int ppipe::check_rotary(const ppipe_rotary_desc& r, const std::string& who)
{
    if (r.dtype < PPIPE_F32 || r.dtype > PPIPE_BF16)
        return bad(who + "unknown dtype " + std::to_string(r.dtype));
    if (r.batch < 0 || r.tokens < 0 || r.heads < 0)
        return bad(who + "negative batch, tokens or heads");
    if (r.head_dim < 8 || r.head_dim > HEAD_DIM_MAX || r.head_dim % 8)
        return unsupported(who + "head_dim must be a multiple of 8, at most " +
                           std::to_string(HEAD_DIM_MAX));
    if (r.axes < 1 || r.axes > 3) return bad(who + "rotary takes one to three axes");
    int64_t total = 0;
    for (int a = 0; a < r.axes; ++a) {
        if (r.pairs[a] < 0) return bad(who + "negative number of rotary pairs");
        total += r.pairs[a];
    }
    if (total < 1 || 2 * total > r.head_dim)
        return bad(who + "rotary pairs must be one to head_dim / 2 in all");
    if ((r.shared | r.adjacent) & ~1) return bad(who + "shared and adjacent are 0 or 1");
    if (!(r.base > 0.0) || std::isinf(r.base)) return bad(who + "rotary base must be positive");
    if ((int64_t)r.batch * r.tokens >= 1 << 24)       // a block each at most, 256 threads
        return unsupported(who + "2^24 tokens and more");
    if (r.heads > MAX_HEADS) return unsupported(who + "more than 65536 heads");
    const int64_t n[3] = {r.batch, r.tokens, r.heads};
    int rc = check_batch_stride(r.positions_stride, r.batch, who);
    if (rc == PPIPE_OK) rc = check_strides("x", r.x_strides, n, dtype_size(r.dtype));
    if (rc == PPIPE_OK) rc = check_strides("y", r.y_strides, n, dtype_size(r.dtype));
    if (rc != PPIPE_OK) return rc;
    if (overlaps_itself(r.y_strides, n, r.head_dim)) return bad(who + "y overlaps itself");
    return PPIPE_OK;
}

RotaryArgs ppipe::rotary_args(const ppipe_rotary_desc& r, const void* x, const int* pos, void* y)
{
    RotaryArgs a;
    a.x = x;
    a.y = y;
    a.pos = pos;
    a.N = r.batch; a.L = r.tokens; a.H = r.heads; a.d = r.head_dim; a.A = r.axes;
    for (int i = 0; i < 3; ++i) {
        a.pairs[i] = i < r.axes ? r.pairs[i] : 0;
        a.xs[i] = r.x_strides[i];
        a.ys[i] = r.y_strides[i];
    }
    a.shared = r.shared;
    a.adjacent = r.adjacent;
    a.base = r.base;
    a.ps = r.positions_stride;
    return a;
}

int ppipe::check_attention(const ppipe_attention_desc& t, const std::string& who)
{
    if (t.dtype < PPIPE_F32 || t.dtype > PPIPE_BF16)
        return bad(who + "unknown dtype " + std::to_string(t.dtype));
    if (t.batch < 0 || t.q_len < 0 || t.kv_len < 0) return bad(who + "negative size");
    if (t.heads < 1 || t.kv_heads < 1 || t.heads % t.kv_heads)
        return bad(who + "heads must be a multiple of kv_heads, both at least 1");
    if (t.head_dim < 8 || t.head_dim > HEAD_DIM_MAX || t.head_dim % 8)
        return unsupported(who + "head_dim must be a multiple of 8, at most " +
                           std::to_string(HEAD_DIM_MAX));
    // (an infinity or a NaN fails these)
    if (!(std::fabs(t.scale) <= 0x1p100f) || !(t.softcap >= 0.0f && t.softcap <= 0x1p100f))
        return bad(who + "scale and softcap must be at most 2^100, softcap >= 0");
    if (t.axes < 0 || t.axes > 3) return bad(who + "positions have one to three axes");
    if (t.spans_stride % 2) return bad(who + "spans stride must be even");
    if (t.heads > MAX_HEADS || t.kv_len > ATTENTION_MAX_LEN || t.q_len > ATTENTION_MAX_LEN ||
        (t.q_len && t.heads && t.batch > 0x7fffffff / ((int64_t)t.q_len * t.heads)))
        return unsupported(who + "attention of this size is not supported");
    const int esz = dtype_size(t.dtype);
    const int64_t nq[3] = {t.batch, t.q_len, t.heads}, nk[3] = {t.batch, t.kv_len, t.kv_heads};
    int rc = check_batch_stride(t.q_positions_stride, t.batch, who);
    if (rc == PPIPE_OK) rc = check_batch_stride(t.k_positions_stride, t.batch, who);
    if (rc == PPIPE_OK) rc = check_batch_stride(t.spans_stride, t.batch, who);
    if (rc == PPIPE_OK) rc = check_strides("q", t.q_strides, nq, esz);
    if (rc == PPIPE_OK) rc = check_strides("k", t.k_strides, nk, esz);
    if (rc == PPIPE_OK) rc = check_strides("v", t.v_strides, nk, esz);
    if (rc == PPIPE_OK) rc = check_strides("out", t.out_strides, nq, esz);
    if (rc != PPIPE_OK) return rc;
    if (overlaps_itself(t.out_strides, nq, t.head_dim)) return bad(who + "out overlaps itself");
    if (t.batch && t.q_len &&
        !attention_fits(t.dtype, attention_args(t, nullptr, nullptr, nullptr, nullptr, nullptr,
                                                nullptr, nullptr, nullptr), device_cus()))
        return unsupported(who + "attention of this size is not supported");
    return PPIPE_OK;
}

AttentionArgs ppipe::attention_args(const ppipe_attention_desc& t, const void* q, const void* k,
                                    const void* v, void* out, const float* slopes, const int* qpos,
                                    const int* kpos, const int* spans)
{
    AttentionArgs a;
    a.q = q; a.k = k; a.v = v; a.out = out;
    a.slopes = slopes; a.qpos = qpos; a.kpos = kpos; a.spans = spans;
    a.N = t.batch; a.Lq = t.q_len; a.Lk = t.kv_len;
    a.H = t.heads; a.Hk = t.kv_heads; a.d = t.head_dim; a.A = t.axes;
    a.scale = t.scale; a.cap = t.softcap;
    for (int i = 0; i < 3; ++i) {
        a.qs[i] = t.q_strides[i]; a.ks[i] = t.k_strides[i];
        a.vs[i] = t.v_strides[i]; a.os[i] = t.out_strides[i];
    }
    a.qps = t.q_positions_stride; a.kps = t.k_positions_stride; a.sps = t.spans_stride;
    return a;
}

extern "C" {

int64_t ppipe_group_norm_workspace(int32_t dtype, int32_t batch, int32_t pixels, int32_t channels,
                                   int32_t groups)
{
    const int rc = check_group_norm(dtype, batch, pixels, channels, groups, 0.0f, 0, "");
    if (rc != PPIPE_OK) return rc;
    if (!batch || !pixels) return 0;
    return (int64_t)group_norm_workspace(dtype, batch, pixels, channels, groups, device_cus());
}

int ppipe_group_norm(const void* x, void* y, int32_t dtype, int32_t batch, int32_t pixels,
                     int32_t channels, int32_t groups, const float* gamma, const float* beta,
                     float eps, int32_t act, void* workspace, int64_t workspace_bytes, void* stream)
{
    const int rc = check_group_norm(dtype, batch, pixels, channels, groups, eps, act, "");
    if (rc != PPIPE_OK) return rc;
    if (!batch || !pixels) return PPIPE_OK;
    if (!x || !y) return bad("null buffer");
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(gamma, 4) || !aligned(beta, 4))
        return bad("buffers must be 16-byte aligned, gamma and beta 4-byte");
    const int cus = device_cus();
    const size_t need = group_norm_workspace(dtype, batch, pixels, channels, groups, cus);
    if (need && (!workspace || workspace_bytes < (int64_t)need || !aligned(workspace, 16)))
        return bad("workspace of " + std::to_string(need) + " bytes needed, 16-byte aligned");
    const GroupNormArgs a{x, y, gamma, beta, batch, pixels, channels, groups, eps, act};
    const int n = group_norm_launches(dtype, batch, pixels, channels, groups, cus);
    hipError_t e = hipSuccess;
    for (int i = 0; i < n && e == hipSuccess; ++i)
        e = launch_group_norm(dtype, a, workspace, cus, i, (hipStream_t)stream);
    return launched("group norm launch", e);
}

int ppipe_rotary(const ppipe_rotary_desc* desc, const void* x, const int32_t* positions, void* y,
                 void* stream)
{
    if (!desc) return bad("null description");
    const int rc = check_rotary(*desc, "");
    if (rc != PPIPE_OK) return rc;
    if (!desc->batch || !desc->tokens || !desc->heads) return PPIPE_OK;
    if (!x || !y || !positions) return bad("null buffer");
    if (!aligned(x, 16) || !aligned(y, 16) || !aligned(positions, 4))
        return bad("buffers must be 16-byte aligned, positions 4-byte");
    if (x == y) {
        const int64_t n[3] = {desc->batch, desc->tokens, desc->heads};
        for (int i = 0; i < 3; ++i)
            if (n[i] > 1 && desc->x_strides[i] != desc->y_strides[i])
                return bad("in place, x and y must have the same strides");
    }
    return launched("rotary launch",
                    launch_rotary(desc->dtype, rotary_args(*desc, x, positions, y),
                                  device_cus(), (hipStream_t)stream));
}

int ppipe_attention_spans(int32_t* spans, int32_t batch, int32_t q_len, int32_t kv_len,
                          const int32_t* doc_offsets, int32_t n_docs, const int32_t* prefix,
                          int32_t causal, const int32_t* q_start, void* stream)
{
    if (batch < 0 || q_len < 0 || kv_len < 0 || n_docs < 1)
        return bad("need batch, q_len, kv_len >= 0 and n_docs >= 1");
    if (!doc_offsets && n_docs != 1) return bad("documents need doc_offsets");
    if ((int64_t)batch * q_len > 0x7fffffff || q_len > ATTENTION_MAX_LEN ||
        kv_len > ATTENTION_MAX_LEN || n_docs > ATTENTION_MAX_LEN)
        return unsupported("attention of this size is not supported");
    if (!batch || !q_len) return PPIPE_OK;
    if (!spans) return bad("null buffer");
    if (!aligned(spans, 8) || !aligned(doc_offsets, 4) || !aligned(prefix, 4) ||
        !aligned(q_start, 4))
        return bad("buffers must be 4-byte aligned, spans 8-byte");
    const SpansArgs a{spans, doc_offsets, prefix, q_start, batch, q_len, kv_len, n_docs,
                      causal ? 1 : 0};
    return launched("attention spans launch", launch_attention_spans(a, (hipStream_t)stream));
}

int64_t ppipe_attention_workspace(const ppipe_attention_desc* desc)
{
    if (!desc) return bad("null description");
    const int rc = check_attention(*desc, "");
    if (rc != PPIPE_OK) return rc;
    if (!desc->batch || !desc->q_len) return 0;
    const AttentionArgs a = attention_args(*desc, nullptr, nullptr, nullptr, nullptr, nullptr,
                                           nullptr, nullptr, nullptr);
    return (int64_t)attention_workspace(desc->dtype, a, device_cus());
}

int ppipe_attention(const ppipe_attention_desc* desc, const void* q, const void* k, const void* v,
                    void* out, const float* slopes, const int32_t* q_positions,
                    const int32_t* k_positions, const int32_t* spans, void* workspace,
                    int64_t workspace_bytes, void* stream)
{
    if (!desc) return bad("null description");
    const int rc = check_attention(*desc, "");
    if (rc != PPIPE_OK) return rc;
    if (slopes ? (!q_positions || !k_positions || desc->axes < 1) : (q_positions || k_positions))
        return bad("a distance bias takes slopes, both positions and their axes");
    if (!desc->batch || !desc->q_len) return PPIPE_OK;
    if (!q || !out || (desc->kv_len && (!k || !v))) return bad("null buffer");
    if (out == q || out == k || out == v) return bad("out must not overlap the inputs");
    if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) ||
        !aligned(slopes, 4) || !aligned(q_positions, 4) || !aligned(k_positions, 4) ||
        !aligned(spans, 8))
        return bad("tensors must be 16-byte aligned, spans 8-byte, slopes and positions 4-byte");
    const AttentionArgs a = attention_args(*desc, q, k, v, out, slopes, q_positions, k_positions,
                                           spans);
    const int cus = device_cus();
    const size_t need = attention_workspace(desc->dtype, a, cus);
    if (need && (!workspace || workspace_bytes < (int64_t)need || !aligned(workspace, 16)))
        return bad("workspace of " + std::to_string(need) + " bytes needed, 16-byte aligned");
    const int n = attention_launches(desc->dtype, a, cus);
    hipError_t e = hipSuccess;
    for (int i = 0; i < n && e == hipSuccess; ++i)
        e = launch_attention(desc->dtype, a, workspace, cus, i, (hipStream_t)stream);
    return launched("attention launch", e);
}

}  // extern "C"
