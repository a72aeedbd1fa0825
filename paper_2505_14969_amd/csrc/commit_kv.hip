// stree_commit_kv: the rows of the accepted path, root first, moved together behind the text, in every layer, and the new lengths.
//   [len + t] <- [len + p_t], t = 0 .. d
// p_t >= t and p grows with t, so a row that is still to be read never lies where an earlier one was put: each thread moves its
// own columns in the order of t, in place.
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

namespace {

struct CommitArgs {
    const int32_t *parent, *accepted, *lengths;
    int32_t *lengths_out, *status;      // null: not written by this launch
    int n;
};

// Workgroup (layer x head, sequence); MOVE false: lengths and status only, one workgroup per sequence.
template <typename T, bool MOVE>
__global__ __launch_bounds__(kThreads) void commit_kv_kernel(CommitArgs a, KvView<T> kv, size_t layer_elems) {
    __shared__ TreeLds tree;
    __shared__ uint32_t bits[kMaxNodes * kMaxWords];
    __shared__ int path[kMaxNodes];
    const int b = blockIdx.y, tid = threadIdx.x;
    const int len = a.lengths[b], k = a.accepted[b], words = (a.n + 31) / 32;
    int bad = 0, count = 0;
    if (len >= 0) {
        if (!kv.fits((int64_t)len + a.n)) {
            bad = STREE_SEQ_LENGTH;
        } else if (int node = index_nodes(tree, bits, a.parent, b, a.n, words)) {
            bad = node;
        } else if (k < -1 || k >= a.n) {
            bad = STREE_SEQ_ACCEPTED;
        } else if (k >= 0) {
            count = a.parent ? tree.cnt[k] : k + 1;
            if (pages_missing(kv, b, len, (int64_t)len + k + 1)) bad = STREE_SEQ_PAGE, count = 0;
        }
    }
    if (blockIdx.x == 0 && tid == 0) {
        if (a.lengths_out) a.lengths_out[b] = len + count;
        if (a.status) a.status[b] = bad;
    }
    if (!MOVE || count == 0 || !a.parent) return;
    if (tid <= k && mask_bit(bits, words, k, tid)) {
        int t = 0;
        for (int w = 0; w < words; ++w)
            t += __popc(bits[k * words + w] & (w < (tid >> 5) ? ~0u : w == (tid >> 5) ? (1u << (tid & 31)) - 1u : 0u));
        path[t] = tid;
    }
    __syncthreads();
    const int layer = blockIdx.x / kv.heads, g = blockIdx.x % kv.heads;
    kv.k += layer * layer_elems;
    kv.v += layer * layer_elems;
    for (int e = tid; e < kv.dim; e += kThreads)
        for (int t = 0; t < count; ++t) {
            const int from = len + path[t], to = len + t;
            if (from == to) continue;
            const int pf = kv.page_of(b, from), pt = kv.page_of(b, to);
            kv.key(pt, g, to)[e] = kv.key(pf, g, from)[e];
            kv.value(pt, g, to)[(size_t)e << kv.shift] = kv.value(pf, g, from)[(size_t)e << kv.shift];
        }
}

template <typename T>
hipError_t launch(CommitArgs a, const stree_kv &kv, int batch, hipStream_t st) {
    const KvView<T> view(kv);
    const size_t layer = (size_t)kv.npages * kv.nheads_kv * kv.page * kv.headdim;
    // A chain's rows stand where they should.  Lengths that are overwritten are so when every workgroup has read them.
    const CommitArgs after = a;
    const bool apart = !a.parent || a.lengths == a.lengths_out;
    if (a.parent) {
        if (apart) a.lengths_out = a.status = nullptr;
        hipLaunchKernelGGL((commit_kv_kernel<T, true>), dim3((unsigned)kv.nlayers * kv.nheads_kv, (unsigned)batch), dim3(kThreads), 0, st, a,
                           view, layer);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (apart)
        hipLaunchKernelGGL((commit_kv_kernel<T, false>), dim3(1, (unsigned)batch), dim3(kThreads), 0, st, after, view, layer);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_commit_kv(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *accepted,
                            const int32_t *lengths, int32_t *lengths_out, int32_t *status, hipStream_t st) {
    const CommitArgs c = {parent, accepted, lengths, lengths_out, status, a.nnodes};
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(c, kv, a.batch, st) : launch<float>(c, kv, a.batch, st);
}

}  // namespace stree
