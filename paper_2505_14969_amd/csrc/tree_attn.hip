// stree_tree_attn: attention of a tree's nodes over a paged cache and the nodes of their paths,
//   out(b,i,h) = sum_t softmax_t(scale <q, K_t>) V_t,   t < length or t = length + j with j on the path of i,
// one pass over the keys with the running maximum and sum of the softmax.  Here the plain kernel, for rows that are no whole
// 16-byte pieces, and the choice; tree_attn_stream.hip has the tuned one.
#include "attn.hpp"

namespace stree {

namespace {

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// A wave per query row, 64 keys at a time, in fp32 FMA: any head size, any alignment.  Lane = key in the first product and
// = column in the second, where keys that the row does not see are skipped.
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_plain_kernel(AttnArgs a, KvView<T> kv) {
    __shared__ TreeLds tree;
    __shared__ uint32_t bits[kMaxNodes * kMaxWords];
    __shared__ float qrow[kThreads / 64][256], prob[kThreads / 64][64];
    __shared__ int pages[kThreads / 64][64];
    const int b = blockIdx.y, P = kv.dim, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, R = a.heads / kv.heads;
    const int len = a.lengths[b], words = (a.n + 31) / 32;
    int bad = 0;
    if (len >= 0) {
        if (!kv.fits((int64_t)len + a.n)) bad = STREE_SEQ_LENGTH;
        else if (int node = index_nodes(tree, bits, a.parent, b, a.n, words)) bad = node;
        else if (pages_missing(kv, b, 0, (int64_t)len + a.n)) bad = STREE_SEQ_PAGE;
    }
    if (a.status && blockIdx.x == 0 && threadIdx.x == 0) a.status[b] = bad;
    const bool dead = len < 0 || bad;
    const T *const q = static_cast<const T *>(a.q);
    T *const out = static_cast<T *>(a.out);
    const int rows = a.n * a.heads;
    for (long r0 = blockIdx.x * (kThreads / 64); r0 < rows; r0 += gridDim.x * (kThreads / 64)) {
        const int r = (int)min(r0 + wave, (long)INT32_MAX);
        if (r >= rows) continue;
        const int i = r / a.heads, h = r % a.heads, g = h / R;
        const size_t token = (size_t)b * a.n + i;
        T *const dst = out + (token * a.heads + h) * P;
        if (dead) {
            for (int e = lane; e < P; e += 64) from_f32(0.f, dst[e]);
            continue;
        }
        wave_sync();
        for (int e = lane; e < P; e += 64) qrow[wave][e] = to_f32(q[token * a.q_sn + (size_t)h * P + e]);
        wave_sync();
        float acc[4] = {0.f, 0.f, 0.f, 0.f}, top = -INFINITY, sum = 0.f;
        const int keys = len + i + 1;                  // (a node's ancestors have smaller numbers)
        for (int t0 = 0; t0 < keys; t0 += 64) {
            const int t = t0 + lane, j = t - len;
            const bool seen = t < keys && (j < 0 || !a.parent || mask_bit(bits, words, i, j));
            float s = -INFINITY;
            int pg = 0;
            if (seen) {
                pg = kv.page_of(b, t);
                const T *krow = kv.key(pg, g, t);
                float d = 0.f;
                for (int e = 0; e < P; ++e) d = fmaf(qrow[wave][e], to_f32(krow[e]), d);
                s = d * a.scale;
            }
            unsigned long long live = __ballot(seen);
            if (!live) continue;
            // (NaN is in no maximum, and reaches the sum through exp2)
            const float above = fmaxf(top, wave_max(s)), base = above == -INFINITY ? 0.f : above;
            const float p = seen ? exp2f(s - base) : 0.f, keep = rescale(top, above);
            top = above;
            sum = sum * keep + wave_sum(p);
            prob[wave][lane] = p;
            pages[wave][lane] = pg;
            wave_sync();
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[c] *= keep;
            while (live) {
                const int l = __ffsll((long long)live) - 1;
                live &= live - 1;
                const float w = prob[wave][l];
                const T *col = kv.value(pages[wave][l], g, t0 + l);
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (lane + 64 * c < P) acc[c] = fmaf(w, to_f32(col[(size_t)(lane + 64 * c) << kv.shift]), acc[c]);
            }
            wave_sync();
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 64 * c < P) from_f32(acc[c] / sum, dst[lane + 64 * c]);
    }
}

template <typename T>
hipError_t launch(const AttnArgs &a, const stree_kv &kv, int batch, hipStream_t st) {
    const long groups = ((long)a.n * a.heads + kThreads / 64 - 1) / (kThreads / 64);
    hipLaunchKernelGGL((attn_plain_kernel<T>), dim3((unsigned)(groups < (1 << 20) ? groups : 1 << 20), (unsigned)batch), dim3(kThreads),
                       0, st, a, KvView<T>(kv));
    return hipGetLastError();
}

}  // namespace

size_t tree_attn_workspace(const stree_attn &a, const stree_kv &kv) { return attn_stream_workspace(a, kv); }

hipError_t launch_tree_attn(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *lengths, const void *q,
                            void *out, int32_t *status, void *workspace, hipStream_t st) {
    const AttnArgs r = {parent, lengths, q, out, status, (long)a.q_stride_n, a.nnodes, a.nheads, a.softmax_scale * 1.44269504088896340736f};
    if (!(a.flags & STREE_ATTN_PLAIN) && attn_stream_supported(a, kv, q, out)) return launch_attn_stream(a, kv, r, workspace, st);
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(r, kv, a.batch, st) : launch<float>(r, kv, a.batch, st);
}

}  // namespace stree
