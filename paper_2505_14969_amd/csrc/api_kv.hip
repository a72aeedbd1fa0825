// C-ABI entry points of the attention layers: argument validation and dispatch.  The one thing computed here is the table of
// rotary frequencies, which is host data.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/stree.h"
#include "launch_kv.hpp"

namespace {

int check_kv(const stree_kv *kv, bool one_layer) {
    if (!kv) return STREE_ERR_NULL_ARG;
    if (kv->io_dtype != STREE_F32 && kv->io_dtype != STREE_BF16) return STREE_ERR_BAD_DTYPE;
    if (kv->nlayers < 1 || kv->nlayers > 65535 || (one_layer && kv->nlayers != 1)) return STREE_ERR_BAD_SHAPE;
    if (kv->npages < 1 || kv->max_pages < 1) return STREE_ERR_BAD_SHAPE;
    if (kv->page < 16 || kv->page > 256 || (kv->page & (kv->page - 1))) return STREE_ERR_BAD_SHAPE;
    if ((int64_t)kv->max_pages * kv->page > (1LL << 30)) return STREE_ERR_BAD_SHAPE;
    if (kv->nheads_kv < 1 || kv->nheads_kv > 65535 || kv->headdim < 1 || kv->headdim > 256) return STREE_ERR_BAD_SHAPE;
    if ((int64_t)kv->nlayers * kv->nheads_kv > (1 << 23)) return STREE_ERR_BAD_SHAPE;      // (a grid dimension)
    // (a page of all heads is moved with 32-bit offsets)
    if ((int64_t)kv->nheads_kv * kv->headdim * kv->page > (1LL << 28)) return STREE_ERR_BAD_SHAPE;
    return STREE_OK;
}

int check_nodes(const stree_attn *a, bool chain) {
    if (a->batch < 0 || a->batch > 65535) return STREE_ERR_BAD_SHAPE;
    if (a->nnodes < 1 || a->nnodes > (chain ? 1 << 24 : STREE_MAX_NODES)) return STREE_ERR_BAD_SHAPE;
    return STREE_OK;
}

int check_heads(const stree_attn *a, const stree_kv *kv) {
    if (a->nheads < 1 || a->nheads > 65535 || a->nheads % kv->nheads_kv != 0) return STREE_ERR_BAD_SHAPE;
    const int64_t heads = (int64_t)a->nheads + 2 * (int64_t)kv->nheads_kv;
    if ((int64_t)a->batch * a->nnodes * heads > 0x7fffffffLL) return STREE_ERR_BAD_SHAPE;
    return STREE_OK;
}

int hip_status(hipError_t e) { return e == hipSuccess ? STREE_OK : STREE_ERR_HIP; }

bool overlap(const void *a, size_t na, const void *b, size_t nb) {
    const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
    return a0 < b0 + nb && b0 < a0 + na;
}
// bytes from the first to the last element of all sequences' rows
size_t span(const stree_attn &a, int64_t stride, int64_t row, size_t e) {
    return a.batch > 0 ? (size_t)(((int64_t)a.batch * a.nnodes - 1) * stride + row) * e : 0;
}
// 0 = dense; a row has to fit, and the rows of all sequences have to lie within 2^60 bytes
bool resolve(int64_t &stride, int64_t row, const stree_attn &a) {
    if (stride == 0) stride = row;
    int64_t all;
    return stride >= row && !__builtin_mul_overflow(stride, (int64_t)a.batch * a.nnodes, &all) && all <= 1LL << 58;
}

int check_pool(const stree_kv *kv, const stree_pool *pool, int32_t batch, bool idle) {
    if (!pool) return STREE_ERR_NULL_ARG;
    if (idle) return batch < 0 || batch > 4096 ? STREE_ERR_BAD_SHAPE : STREE_OK;      // (empty arrays may be null)
    if (!pool->held || !pool->refs || !pool->free || !pool->nfree || !kv->table) return STREE_ERR_NULL_ARG;
    if (batch < 0 || batch > 4096 || (int64_t)batch * kv->max_pages > (1LL << 29)) return STREE_ERR_BAD_SHAPE;
    return STREE_OK;
}

}  // namespace

extern "C" {

int stree_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double low, double high,
                           double original, double *turns) {
    if (rotary_dim < 0 || rotary_dim > 256 || rotary_dim % 2 != 0) return STREE_ERR_BAD_SHAPE;
    if (!turns && rotary_dim > 0) return STREE_ERR_NULL_ARG;
    if (scaling < STREE_ROPE_NONE || scaling > STREE_ROPE_RAMP) return STREE_ERR_BAD_SHAPE;
    if (!(base > 0) || !std::isfinite(base)) return STREE_ERR_BAD_SHAPE;
    if (scaling != STREE_ROPE_NONE && (!(factor >= 1) || !std::isfinite(factor))) return STREE_ERR_BAD_SHAPE;
    if (scaling == STREE_ROPE_RAMP &&
        (!(low >= 0) || !(high > low) || !std::isfinite(high) || !(original > 0) || !std::isfinite(original)))
        return STREE_ERR_BAD_SHAPE;
    const double r = rotary_dim, two_pi = 6.283185307179586476925286766559;
    if (scaling == STREE_ROPE_BASE && rotary_dim > 2) base *= std::pow(factor, r / (r - 2));
    for (int j = 0; j < rotary_dim / 2; ++j) {
        double f = std::pow(base, -2.0 * j / r) / two_pi;
        if (scaling == STREE_ROPE_LINEAR) f /= factor;
        if (scaling == STREE_ROPE_RAMP) {
            const double w = std::fmin(std::fmax((original * f - low) / (high - low), 0.0), 1.0);
            f *= w + (1 - w) / factor;
        }
        turns[j] = f;
    }
    return STREE_OK;
}

int stree_tree_rope(const stree_attn *attn, const stree_kv *kv, const int32_t *parent, const int32_t *lengths, const void *q,
                    const void *k, const void *v, const void *q_norm, const void *k_norm, const double *turns, void *q_out,
                    int32_t *seq_status, void *hip_stream) {
    if (!attn) return STREE_ERR_NULL_ARG;
    int rc = check_kv(kv, true);
    if (!rc) rc = check_nodes(attn, !parent);
    if (!rc) rc = check_heads(attn, kv);
    if (rc) return rc;
    stree_attn a = *attn;
    if (a.rotary_dim < 0 || a.rotary_dim > kv->headdim || a.rotary_dim % 2 != 0) return STREE_ERR_BAD_SHAPE;
    if (!(a.eps >= 0.f)) return STREE_ERR_BAD_SHAPE;
    if (a.batch == 0) return STREE_OK;                 // (empty arrays may be null)
    if (!lengths || !q || !k || !v || !q_out || !kv->k || !kv->v || !kv->table || (a.rotary_dim && !turns)) return STREE_ERR_NULL_ARG;
    const int64_t qr = (int64_t)a.nheads * kv->headdim, kr = (int64_t)kv->nheads_kv * kv->headdim;
    if (!resolve(a.q_stride_n, qr, a) || !resolve(a.k_stride_n, kr, a) || !resolve(a.v_stride_n, kr, a)) return STREE_ERR_BAD_STRIDE;
    const size_t e = kv->io_dtype == STREE_BF16 ? 2 : 4, out = span(a, qr, qr, e);
    if ((overlap(q_out, out, q, span(a, a.q_stride_n, qr, e)) && !(q_out == q && a.q_stride_n == qr)) ||
        overlap(q_out, out, k, span(a, a.k_stride_n, kr, e)) || overlap(q_out, out, v, span(a, a.v_stride_n, kr, e)))
        return STREE_ERR_BAD_ALIAS;
    return hip_status(stree::launch_tree_rope(a, *kv, parent, lengths, q, k, v, q_norm, k_norm, turns, q_out, seq_status,
                                              (hipStream_t)hip_stream));
}

size_t stree_attn_workspace_bytes(const stree_attn *attn, const stree_kv *kv) {
    if (!attn || check_kv(kv, true) || check_nodes(attn, true) || check_heads(attn, kv)) return (size_t)-1;
    return attn->batch == 0 ? 0 : stree::tree_attn_workspace(*attn, *kv);
}

int stree_tree_attn(const stree_attn *attn, const stree_kv *kv, const int32_t *parent, const int32_t *lengths, const void *q,
                    void *out, int32_t *seq_status, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!attn) return STREE_ERR_NULL_ARG;
    int rc = check_kv(kv, true);
    if (!rc) rc = check_nodes(attn, !parent);
    if (!rc) rc = check_heads(attn, kv);
    if (rc) return rc;
    stree_attn a = *attn;
    if (!std::isfinite(a.softmax_scale)) return STREE_ERR_BAD_SHAPE;
    if (a.batch == 0) return STREE_OK;
    if (!lengths || !q || !out || !kv->k || !kv->v || !kv->table) return STREE_ERR_NULL_ARG;
    const int64_t row = (int64_t)a.nheads * kv->headdim;
    if (!resolve(a.q_stride_n, row, a)) return STREE_ERR_BAD_STRIDE;
    if (a.softmax_scale == 0.f) a.softmax_scale = (float)(1.0 / std::sqrt((double)kv->headdim));
    const size_t need = stree::tree_attn_workspace(a, *kv);
    if (need && !workspace) return STREE_ERR_NULL_ARG;
    if (need > workspace_bytes || (need && (uintptr_t)workspace % 16)) return STREE_ERR_BAD_SHAPE;
    const size_t e = kv->io_dtype == STREE_BF16 ? 2 : 4;
    if (overlap(out, span(a, row, row, e), q, span(a, a.q_stride_n, row, e))) return STREE_ERR_BAD_ALIAS;
    return hip_status(stree::launch_tree_attn(a, *kv, parent, lengths, q, out, seq_status, workspace, (hipStream_t)hip_stream));
}

int stree_commit_kv(const stree_attn *attn, const stree_kv *kv, const int32_t *parent, const int32_t *accepted,
                    const int32_t *lengths, int32_t *lengths_out, int32_t *seq_status, void *hip_stream) {
    if (!attn) return STREE_ERR_NULL_ARG;
    int rc = check_kv(kv, false);
    if (!rc) rc = check_nodes(attn, !parent);
    if (rc) return rc;
    if (attn->batch == 0) return STREE_OK;
    if (!accepted || !lengths || !lengths_out || !kv->k || !kv->v || !kv->table) return STREE_ERR_NULL_ARG;
    const size_t n = (size_t)attn->batch * sizeof(int32_t);
    for (const int32_t *in : {lengths, accepted})
        if (lengths_out != in && overlap(in, n, lengths_out, n)) return STREE_ERR_BAD_ALIAS;
    return hip_status(stree::launch_commit_kv(*attn, *kv, parent, accepted, lengths, lengths_out, seq_status,
                                              (hipStream_t)hip_stream));
}

int stree_resize_kv(const stree_kv *kv, const stree_pool *pool, int32_t batch, const int32_t *tokens, int32_t *seq_status,
                    void *hip_stream) {
    int rc = check_kv(kv, false);
    if (!rc) rc = check_pool(kv, pool, batch, batch == 0);
    if (rc) return rc;
    if (batch == 0) return STREE_OK;
    if (!tokens) return STREE_ERR_NULL_ARG;
    return hip_status(stree::launch_resize_kv(*kv, *pool, batch, tokens, seq_status, (hipStream_t)hip_stream));
}

int stree_fork_kv(const stree_kv *kv, const stree_pool *pool, int32_t batch, int32_t nforks, const int32_t *src, const int32_t *dst,
                  int32_t *lengths, int32_t *fork_status, void *hip_stream) {
    int rc = check_kv(kv, false);
    if (!rc) rc = check_pool(kv, pool, batch, nforks == 0);
    if (rc) return rc;
    if (nforks < 0 || nforks > 4096) return STREE_ERR_BAD_SHAPE;
    if (nforks == 0) return STREE_OK;
    if (!src || !dst || !lengths || !fork_status || !kv->k || !kv->v) return STREE_ERR_NULL_ARG;
    return hip_status(stree::launch_fork_kv(*kv, *pool, batch, nforks, src, dst, lengths, fork_status, (hipStream_t)hip_stream));
}

}  // extern "C"
