// stree_commit_kv: the rows of the accepted path, root first, moved together behind the text, in every layer, and the new lengths.
//   [len + t] <- [len + p_t], t = 0 .. d
// p_t >= t and p grows with t, so a row that is still to be read never lies where an earlier one was put: each thread moves its
// own columns in the order of t, a few rows at once, in place.
//
// A few rows of a few hundred bytes in each of many places: bound by the chain length -> tree -> page numbers -> rows (one sequence
// 5 us), and by how many places are worked on at once: 48 of 64 sequences, 9 of 49 nodes, 8 layers of 8 heads of 128: 24.4 us for 28 MB
// of rows, which are 43 MB read and 25 written as memory moves them, a token's column of V being 2 bytes in each of 128 pieces of 32.
// So a workgroup takes several heads of a layer behind one look at the tree, where there are enough workgroups, and page numbers are
// looked up for all rows at once.
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

namespace {

struct CommitArgs {
    const int32_t *parent, *accepted, *lengths;
    int32_t *lengths_out, *status;      // null: not written by this launch
    int n;
};

constexpr int kBatch = 8;              // rows that a thread has on their way

// The accepted path of sequence b: its nodes, root first, in `path`, and how many (0: nothing to move), or what is wrong.  Up
// to 64 nodes every wave follows the parents in its own lanes.
template <typename T>
__device__ __forceinline__ int find_path(const CommitArgs &a, const KvView<T> &kv, TreeLds &tree, uint32_t *bits, int *path, int b, int len,
                                         int k, int &count) {
    count = 0;
    if (len < 0) return 0;
    if (!kv.fits((int64_t)len + a.n)) return STREE_SEQ_LENGTH;
    const int tid = threadIdx.x, lane = tid & 63;
    if (a.parent && a.n <= 64) {
        const int p = lane < a.n ? a.parent[(size_t)b * a.n + lane] : -1;
        const unsigned long long wrong = __ballot(lane < a.n && (lane == 0 ? p != -1 : (p < 0 || p >= lane)));
        if (wrong) return __ffsll((long long)wrong);
        if (k < -1 || k >= a.n) return STREE_SEQ_ACCEPTED;
        unsigned long long on = 0;
        for (int j = __builtin_amdgcn_readfirstlane(k); j >= 0; j = __builtin_amdgcn_readlane(p, j)) on |= 1ull << j;      // (p < j)
        count = __popcll(on);
        if ((on >> lane) & 1ull) path[__popcll(on & ((1ull << lane) - 1ull))] = lane;
    } else {
        const int words = (a.n + 31) / 32;
        if (const int node = index_nodes(tree, bits, a.parent, b, a.n, words)) return node;
        if (k < -1 || k >= a.n) return STREE_SEQ_ACCEPTED;
        if (k >= 0) count = a.parent ? tree.cnt[k] : k + 1;
        if (a.parent && k >= 0 && tid <= k && tid < kMaxNodes && mask_bit(bits, words, k, tid)) {
            int t = 0;
            for (int w = 0; w < words; ++w)
                t += __popc(bits[k * words + w] & (w < (tid >> 5) ? ~0u : w == (tid >> 5) ? (1u << (tid & 31)) - 1u : 0u));
            path[t] = tid;
        }
    }
    if (k >= 0 && pages_missing(kv, b, len, (int64_t)len + k + 1)) {          // (a barrier: `path` is there)
        count = 0;
        return STREE_SEQ_PAGE;
    }
    return 0;
}

// Workgroup (heads of a layer, sequence); MOVE false: lengths and status only, one workgroup per sequence.  E: elements of K
// moved at once.
template <typename T, bool MOVE, int E>
__global__ __launch_bounds__(kThreads) void commit_kv_kernel(CommitArgs a, KvView<T> kv, size_t layer_elems, int chunks, int per) {
    typedef T Run __attribute__((ext_vector_type(E)));
    __shared__ TreeLds tree;
    __shared__ uint32_t bits[kMaxNodes * kMaxWords];
    __shared__ int path[kMaxNodes];
    __shared__ int2 from[kMaxNodes], to[kMaxNodes];              // (page, token within it)
    const int b = blockIdx.y, tid = threadIdx.x, len = a.lengths[b], k = a.accepted[b];
    int count;
    const int bad = find_path(a, kv, tree, bits, path, b, len, k, count);
    if (!MOVE) __syncthreads();                                  // (every wave has its length and node, where these may be written)
    if (blockIdx.x == 0 && tid == 0) {
        if (a.lengths_out) a.lengths_out[b] = len + count;
        if (a.status) a.status[b] = bad;
    }
    if (!MOVE || count == 0 || !a.parent) return;
    if (tid < count) {
        const int s = len + path[tid], d = len + tid;
        from[tid] = make_int2(kv.page_of(b, s), s & kv.mask());
        to[tid] = make_int2(kv.page_of(b, d), d & kv.mask());
    }
    int first = 0;                                               // (the first rows mostly stand where they should)
    while (first < count && path[first] == first) ++first;
    __syncthreads();
    const int layer = blockIdx.x / chunks, g0 = blockIdx.x % chunks * per, heads = min(per, kv.heads - g0);
    T *const kl = kv.k + layer * layer_elems, *const vl = kv.v + layer * layer_elems;
    const int runs = kv.dim / E, keys = heads * runs, values = heads * kv.dim;
    const size_t block = (size_t)kv.dim << kv.shift;
    // a thread's pieces of K and of V are on their way together (one after the other: 28.9 us in place of 24.4)
    for (int y = tid; y < max(keys, values); y += kThreads) {
        const bool key = y < keys, value = y < values;
        const int gk = g0 + y / runs, gv = g0 + y / kv.dim, c = y % runs * E;
        const size_t p = (size_t)(y % kv.dim) << kv.shift;
        auto in_k = [&](const int2 &w) { return reinterpret_cast<Run *>(kl + ((size_t)w.x * kv.heads + gk) * block + (size_t)w.y * kv.dim + c); };
        auto in_v = [&](const int2 &w) { return vl + ((size_t)w.x * kv.heads + gv) * block + p + w.y; };
        for (int t = first; t < count; t += kBatch) {
            Run rk[kBatch];
            T rv[kBatch];
            if (key) {
#pragma unroll
                for (int x = 0; x < kBatch; ++x) rk[x] = *in_k(from[min(t + x, count - 1)]);
            }
            if (value) {
#pragma unroll
                for (int x = 0; x < kBatch; ++x) rv[x] = *in_v(from[min(t + x, count - 1)]);
            }
#pragma unroll
            for (int x = 0; x < kBatch; ++x) {
                if (t + x >= count) break;
                if (key) *in_k(to[t + x]) = rk[x];
                if (value) *in_v(to[t + x]) = rv[x];
            }
        }
    }
}

template <typename T, int E>
hipError_t launch_runs(CommitArgs a, const stree_kv &kv, int batch, hipStream_t st) {
    const KvView<T> view(kv);
    const size_t layer = (size_t)kv.npages * kv.nheads_kv * kv.page * kv.headdim;
    // Heads of a workgroup: one until there are as many workgroups as the chip holds at once, then more (64 sequences, 8 layers of 8
    // heads: two 24.4 us, one 25.2, three 28.4).
    const int64_t places = (int64_t)batch * kv.nlayers * kv.nheads_kv;
    int per = (int)((places + 2047) / 2048);
    per = per < kv.nheads_kv ? per : kv.nheads_kv;
    const int chunks = (kv.nheads_kv + per - 1) / per;
    // A chain's rows stand where they should.  Lengths, and accepted nodes, that are overwritten are so when every workgroup has read them.
    const CommitArgs after = a;
    const bool apart = !a.parent || a.lengths == a.lengths_out || a.accepted == a.lengths_out;
    if (a.parent) {
        if (apart) a.lengths_out = a.status = nullptr;
        hipLaunchKernelGGL((commit_kv_kernel<T, true, E>), dim3((unsigned)kv.nlayers * chunks, (unsigned)batch), dim3(kThreads), 0, st, a, view,
                           layer, chunks, per);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (apart)
        hipLaunchKernelGGL((commit_kv_kernel<T, false, E>), dim3(1, (unsigned)batch), dim3(kThreads), 0, st, after, view, layer, chunks, per);
    return hipGetLastError();
}

template <typename T>
hipError_t launch(const CommitArgs &a, const stree_kv &kv, int batch, hipStream_t st) {
    constexpr int E = 16 / sizeof(T);
    if (kv.headdim % E == 0 && (uintptr_t)kv.k % 16 == 0) return launch_runs<T, E>(a, kv, batch, st);
    return launch_runs<T, 1>(a, kv, batch, st);
}

}  // namespace

hipError_t launch_commit_kv(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *accepted,
                            const int32_t *lengths, int32_t *lengths_out, int32_t *status, hipStream_t st) {
    const CommitArgs c = {parent, accepted, lengths, lengths_out, status, a.nnodes};
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(c, kv, a.batch, st) : launch<float>(c, kv, a.batch, st);
}

}  // namespace stree
