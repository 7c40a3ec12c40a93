// seq_api.cu -- entry points of attention over sequences and of the floating-point
// embedding: argument checks, then the launchers.
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>

#include "train.h"

using namespace mnmt;

namespace {

constexpr int32_t MAX_DIM = 1 << 30;
constexpr int64_t MAX_LD = (int64_t)1 << 36;  // bytes of a stride stay below 2^40

int fail(int code, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return set_error(code, buf);
}

int done(cudaError_t e, const char *call) {
    return e == cudaSuccess ? MNMT_OK : fail(MNMT_ECUDA, "%s: %s", call, cudaGetErrorString(e));
}

int type_size(int32_t dtype) { return dtype == MNMT_F32 ? 4 : dtype == MNMT_BF16 || dtype == MNMT_F16 ? 2 : 0; }
bool aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
bool matrix_ok(const void *p, int32_t dtype, int64_t ld, int32_t cols) {
    const int e = type_size(dtype);
    return e && p && aligned(p, e) && ld >= cols && ld <= MAX_LD;
}

// one-time set-up of the attention kernels on the current device
int seq_ready() {
    if (int rc = ensure_device()) return rc;
    static std::mutex mu;
    static bool ready[64] = {false};
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return fail(MNMT_ECUDA, "attention: no usable current device");
    std::lock_guard<std::mutex> lk(mu);
    if (!ready[dev]) {
        cudaError_t e = seq_attn_init();
        if (e == cudaSuccess) e = seq_attn_backward_init();
        if (e == cudaSuccess) e = seq_attn_token_init();
        if (e != cudaSuccess) return fail(MNMT_ECUDA, "attention kernel set-up failed: %s", cudaGetErrorString(e));
        ready[dev] = true;
    }
    return MNMT_OK;
}

// 0 if the shape is valid; with a shape alone (sizes of workspaces) nothing of its arrays is looked at
int check_shape(const char *call, const mnmt_attention_shape *s, SeqAttn &a, bool arrays, bool token) {
    if (!s) return fail(MNMT_EINVAL, "%s: null shape", call);
    if (s->n_seqs < 0 || s->q_rows < 0 || s->k_rows < 0 || s->n_seqs > MAX_DIM || s->q_rows > MAX_DIM || s->k_rows > MAX_DIM)
        return fail(MNMT_EINVAL, "%s: bad size: %d sequences, %d and %d rows", call, s->n_seqs, s->q_rows, s->k_rows);
    if (s->q_heads < 1 || s->kv_heads < 1 || s->q_heads > 4096 || s->q_heads % s->kv_heads)
        return fail(MNMT_EINVAL, "%s: %d query heads cannot share %d key heads", call, s->q_heads, s->kv_heads);
    if (s->d_head < 8 || s->d_head > 128 || s->d_head % 8) return fail(MNMT_EINVAL, "%s: head size %d is no multiple of 8 up to 128", call, s->d_head);
    if (s->dtype != MNMT_BF16 && s->dtype != MNMT_F16) return fail(MNMT_EINVAL, "%s: type %d is neither bf16 nor fp16", call, s->dtype);
    if (!(s->scale > 0.0f && s->scale <= 0x1p60f)) return fail(MNMT_EINVAL, "%s: scale %g outside (0, 2^60]", call, s->scale);
    // blocks of a launch: tiles of 128 rows x heads x the CTAs that may share a walk (one query per sequence: units and rows)
    const int64_t most = 0x7FFFFFFF, tiles = token ? s->n_seqs : ((int64_t)(s->q_rows > s->k_rows ? s->q_rows : s->k_rows) + 127) / 128 * 8;
    if (tiles * s->q_heads > most) return fail(MNMT_EINVAL, "%s: %d rows of %d heads are more than a launch takes", call, s->q_rows, s->q_heads);
    if (token && s->q_rows != s->n_seqs) return fail(MNMT_EINVAL, "%s: %d query rows for %d sequences", call, s->q_rows, s->n_seqs);
    if (arrays && s->n_seqs > 0 && ((!token && !s->q_start) || !s->k_start)) return fail(MNMT_EINVAL, "%s: null starts of the sequences", call);
    if (!aligned(s->q_start, 4) || !aligned(s->q_len, 4) || !aligned(s->k_start, 4) || !aligned(s->k_len, 4))
        return fail(MNMT_EINVAL, "%s: starts and lengths must be 4-byte aligned", call);
    a = SeqAttn{};
    a.n_seqs = s->n_seqs, a.q_rows = s->q_rows, a.k_rows = s->k_rows;
    a.hq = s->q_heads, a.hkv = s->kv_heads, a.dh = s->d_head;
    a.dtype = s->dtype, a.causal = s->causal != 0, a.scale = s->scale;
    a.q_start = s->q_start, a.q_len = s->q_len, a.k_start = s->k_start, a.k_len = s->k_len;
    return MNMT_OK;
}

// 0 if an operand of rows x heads x d can be read (and, as an output, rows do not share elements)
int check_heads(const char *call, const char *name, const mnmt_heads *m, int32_t rows, int32_t heads, int32_t d, HeadRows &out) {
    out = HeadRows{nullptr, 0, 0};
    if (!m) return fail(MNMT_EINVAL, "%s: null %s", call, name);
    if (rows == 0) return MNMT_OK;
    if (!m->data || !aligned(m->data, 16)) return fail(MNMT_EINVAL, "%s: %s must be given, 16-byte aligned", call, name);
    const bool row = rows > 1, head = heads > 1;
    if ((row && (m->row < d || m->row > MAX_LD || m->row % 8)) || (head && (m->head < d || m->head > MAX_LD || m->head % 8)))
        return fail(MNMT_EINVAL, "%s: strides of %s must be multiples of 8 elements, %d at least", call, name, d);
    // heads inside a row, or rows inside a head
    if (row && head && m->row < (int64_t)(heads - 1) * m->head + d && m->head < (int64_t)(rows - 1) * m->row + d)
        return fail(MNMT_EINVAL, "%s: rows and heads of %s overlap", call, name);
    out.p = m->data;
    out.ld = row ? m->row : (int64_t)heads * (head ? m->head : d);
    out.hd = head ? m->head : d;
    return MNMT_OK;
}

int check_scratch(const char *call, const void *workspace, const int32_t *status) {
    if (!workspace || !aligned(workspace, 16)) return fail(MNMT_EINVAL, "%s: workspace must be given, 16-byte aligned", call);
    if (!aligned(status, 4)) return fail(MNMT_EINVAL, "%s: status must be 4-byte aligned", call);
    return MNMT_OK;
}

bool same(const HeadRows &x, const HeadRows &y) { return x.p && x.p == y.p; }

int check_forward(const char *call, const mnmt_attention_shape *s, const mnmt_heads *q, const mnmt_heads *k, const mnmt_heads *v, const mnmt_heads *o,
                  float *lse, void *workspace, int32_t *status, bool token, SeqAttn &a) {
    int rc = check_shape(call, s, a, true, token);
    if (rc) return rc;
    if ((rc = check_heads(call, "q", q, a.q_rows, a.hq, a.dh, a.q)) || (rc = check_heads(call, "k", k, a.k_rows, a.hkv, a.dh, a.k)) ||
        (rc = check_heads(call, "v", v, a.k_rows, a.hkv, a.dh, a.v)) || (rc = check_heads(call, "o", o, a.q_rows, a.hq, a.dh, a.o)))
        return rc;
    if (same(a.o, a.q) || same(a.o, a.k) || same(a.o, a.v)) return fail(MNMT_EINVAL, "%s: o is an input", call);
    if (!aligned(lse, 4)) return fail(MNMT_EINVAL, "%s: lse must be 4-byte aligned", call);
    if ((rc = check_scratch(call, workspace, status))) return rc;
    a.lse = lse;
    a.workspace = workspace;
    a.status = status;
    return MNMT_OK;
}

int check_embed(const char *call, const void *ids, int32_t T, int32_t V, int32_t d, int32_t dtype, int32_t otype, float scale, const int32_t *status) {
    if (T < 0 || V < 1 || d < 1 || T > MAX_DIM || V > MAX_DIM || d > MAX_DIM) return fail(MNMT_EINVAL, "%s: bad size: %d tokens of %d, width %d", call, T, V, d);
    if (!type_size(dtype) || !type_size(otype)) return fail(MNMT_EINVAL, "%s: unknown type", call);
    if (!std::isfinite(scale)) return fail(MNMT_EINVAL, "%s: scale %g", call, scale);
    if ((T > 0 && !ids) || !aligned(ids, 4) || !aligned(status, 4)) return fail(MNMT_EINVAL, "%s: ids must be given; ids and status 4-byte aligned", call);
    return MNMT_OK;
}

}  // namespace

extern "C" size_t mnmt_attention_forward_workspace(const mnmt_attention_shape *shape) {
    SeqAttn a;
    return check_shape("attention_forward_workspace", shape, a, false, false) ? 0 : seq_attn_forward_workspace(a);
}
extern "C" size_t mnmt_attention_backward_workspace(const mnmt_attention_shape *shape) {
    SeqAttn a;
    return check_shape("attention_backward_workspace", shape, a, false, false) ? 0 : seq_attn_backward_workspace(a);
}
extern "C" size_t mnmt_attention_token_workspace(const mnmt_attention_shape *shape) {
    SeqAttn a;
    return check_shape("attention_token_workspace", shape, a, false, true) ? 0 : seq_attn_token_workspace(a);
}

extern "C" int mnmt_attention_forward(const mnmt_attention_shape *shape, const mnmt_heads *q, const mnmt_heads *k, const mnmt_heads *v, const mnmt_heads *o,
                                      float *lse, void *workspace, int32_t *status, void *cuda_stream) {
    SeqAttn a;
    int rc = check_forward("attention_forward", shape, q, k, v, o, lse, workspace, status, false, a);
    if (rc || (rc = seq_ready())) return rc;
    if (a.n_seqs == 0 || a.q_rows == 0) return MNMT_OK;
    return done(launch_seq_attn_forward(a, static_cast<cudaStream_t>(cuda_stream)), "attention_forward");
}

extern "C" int mnmt_attention_token(const mnmt_attention_shape *shape, const mnmt_heads *q, const mnmt_heads *k, const mnmt_heads *v, const mnmt_heads *o,
                                    float *lse, void *workspace, int32_t *status, void *cuda_stream) {
    SeqAttn a;
    int rc = check_forward("attention_token", shape, q, k, v, o, lse, workspace, status, true, a);
    if (rc || (rc = seq_ready())) return rc;
    if (a.n_seqs == 0) return MNMT_OK;
    return done(launch_seq_attn_token(a, static_cast<cudaStream_t>(cuda_stream)), "attention_token");
}

extern "C" int mnmt_attention_backward(const mnmt_attention_shape *shape, const mnmt_heads *q, const mnmt_heads *k, const mnmt_heads *v,
                                       const mnmt_heads *o, const float *lse, const mnmt_heads *g, const mnmt_heads *dq, const mnmt_heads *dk,
                                       const mnmt_heads *dv, void *workspace, int32_t *status, void *cuda_stream) {
    const char *call = "attention_backward";
    SeqAttn a;
    int rc = check_forward(call, shape, q, k, v, o, const_cast<float *>(lse), workspace, status, false, a);
    if (rc) return rc;
    if ((rc = check_heads(call, "g", g, a.q_rows, a.hq, a.dh, a.g)) || (rc = check_heads(call, "dq", dq, a.q_rows, a.hq, a.dh, a.dq)) ||
        (rc = check_heads(call, "dk", dk, a.k_rows, a.hkv, a.dh, a.dk)) || (rc = check_heads(call, "dv", dv, a.k_rows, a.hkv, a.dh, a.dv)))
        return rc;
    if (!lse && a.q_rows > 0) return fail(MNMT_EINVAL, "%s: null lse", call);
    const HeadRows *in[] = {&a.q, &a.k, &a.v, &a.o, &a.g}, *out[] = {&a.dq, &a.dk, &a.dv};
    for (int i = 0; i < 3; i++) {
        for (const HeadRows *x : in)
            if (same(*out[i], *x)) return fail(MNMT_EINVAL, "%s: a gradient's buffer is an input", call);
        for (int j = 0; j < i; j++)
            if (same(*out[i], *out[j])) return fail(MNMT_EINVAL, "%s: two gradients in one buffer", call);
    }
    if ((rc = seq_ready())) return rc;
    if (a.n_seqs == 0 || (a.q_rows == 0 && a.k_rows == 0)) return MNMT_OK;
    return done(launch_seq_attn_backward(a, static_cast<cudaStream_t>(cuda_stream)), call);
}

extern "C" int mnmt_embed(const int32_t *ids, int32_t T, const void *table, int32_t dtype, int64_t ldt, int32_t V, int32_t d, float scale,
                          const int32_t *pos, const float *pe, int64_t ldpe, int32_t P, void *out, int32_t otype, int64_t ldo, int32_t *status,
                          void *cuda_stream) {
    const char *call = "embed";
    int rc = check_embed(call, ids, T, V, d, dtype, otype, scale, status);
    if (rc) return rc;
    if (!matrix_ok(table, dtype, ldt, d) || (T > 0 && !matrix_ok(out, otype, ldo, d))) return fail(MNMT_EINVAL, "%s: bad pointer or row stride", call);
    if (pe && (P < 1 || P > MAX_DIM || !matrix_ok(pe, MNMT_F32, ldpe, d) || !aligned(pos, 4))) return fail(MNMT_EINVAL, "%s: bad positional table", call);
    if (out == table || out == pe) return fail(MNMT_EINVAL, "%s: the output is a table", call);
    if ((rc = ensure_device())) return rc;
    if (T == 0) return MNMT_OK;
    EmbedRowsArgs a{};
    a.ids = ids, a.pos = pe ? pos : nullptr, a.T = T, a.V = V, a.d = d, a.P = P;
    a.table = table, a.dtype = dtype, a.ld = ldt, a.scale = scale, a.pe = pe, a.ldpe = ldpe;
    a.out = out, a.otype = otype, a.ldo = ldo, a.status = status;
    return done(launch_embed_rows(a, static_cast<cudaStream_t>(cuda_stream)), call);
}

extern "C" size_t mnmt_embed_backward_workspace(int32_t T, int32_t V, int32_t d) {
    return T < 0 || V < 1 || d < 1 || T > MAX_DIM || V > MAX_DIM || d > MAX_DIM ? 0 : embed_rows_backward_workspace(T, V, d);
}

extern "C" int mnmt_embed_backward(const int32_t *ids, int32_t T, const void *g, int32_t gtype, int64_t ldg, float scale, int32_t pad_id, int32_t V,
                                   int32_t d, void *gtable, int32_t otype, int64_t ldt, int32_t accumulate, void *workspace, int32_t *status,
                                   void *cuda_stream) {
    const char *call = "embed_backward";
    int rc = check_embed(call, ids, T, V, d, gtype, otype, scale, status);
    if (rc) return rc;
    if ((T > 0 && !matrix_ok(g, gtype, ldg, d)) || !matrix_ok(gtable, otype, ldt, d)) return fail(MNMT_EINVAL, "%s: bad pointer or row stride", call);
    if (g == gtable) return fail(MNMT_EINVAL, "%s: the gradient's buffer is an input", call);
    if ((rc = check_scratch(call, workspace, status)) || (rc = ensure_device())) return rc;
    if (T == 0 && accumulate) return MNMT_OK;
    EmbedRowsArgs a{};
    a.ids = ids, a.T = T, a.V = V, a.d = d;
    a.table = g, a.dtype = gtype, a.ld = ldg, a.scale = scale;
    a.out = gtable, a.otype = otype, a.ldo = ldt, a.pad_id = pad_id, a.accumulate = accumulate != 0;
    a.workspace = workspace, a.status = status;
    return done(launch_embed_rows_backward(a, static_cast<cudaStream_t>(cuda_stream)), call);
}
