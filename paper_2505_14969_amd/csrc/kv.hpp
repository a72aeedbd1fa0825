// The paged cache of the attention layers as the kernels see it.
#pragma once
#include "common.hpp"

namespace stree {

// One layer's keys [npages, heads, page, dim] and values [npages, heads, dim, page], and the table of page numbers.
// Offsets into the cache are 64-bit: a pool may be larger than 4 GB.
template <typename T>
struct KvView {
    T *k, *v;
    const int32_t *table;
    int npages, shift, max_pages, heads, dim;       // a page holds 1 << shift tokens
    KvView(const stree_kv &kv, int layer = 0)
        : table(kv.table), npages(kv.npages), shift(__builtin_ctz((unsigned)kv.page)), max_pages(kv.max_pages),
          heads(kv.nheads_kv), dim(kv.headdim) {
        const size_t all = (size_t)kv.npages * kv.nheads_kv * kv.page * kv.headdim * layer;
        k = static_cast<T *>(kv.k) + all;
        v = static_cast<T *>(kv.v) + all;
    }
    __device__ __forceinline__ bool fits(int64_t tokens) const { return tokens <= (int64_t)max_pages << shift; }
    __device__ __forceinline__ int mask() const { return (1 << shift) - 1; }
    // number of the page that token t of sequence b stands in, whatever the table holds there
    __device__ __forceinline__ int page_of(int b, int t) const { return table[(size_t)b * max_pages + (t >> shift)]; }
    __device__ __forceinline__ bool exists(int pg) const { return (unsigned)pg < (unsigned)npages; }
    // first element of head h of a page
    __device__ __forceinline__ size_t block(int pg, int h) const { return ((size_t)pg * heads + h) * ((size_t)dim << shift); }
    __device__ __forceinline__ T *key(int pg, int h, int t) const { return k + block(pg, h) + (size_t)(t & mask()) * dim; }
    // column 0 of token t; columns are 1 << shift elements apart
    __device__ __forceinline__ T *value(int pg, int h, int t) const { return v + block(pg, h) + (t & mask()); }
};

// What this wave's lanes wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Whether any page that tokens [t0, t1) of sequence b stand in is missing; the whole workgroup calls it (one barrier).
template <typename T>
__device__ __forceinline__ bool pages_missing(const KvView<T> &kv, int b, int64_t t0, int64_t t1) {
    int bad = 0;
    if (t1 > t0)
        for (int j = (int)(t0 >> kv.shift) + (int)threadIdx.x; j <= (int)((t1 - 1) >> kv.shift); j += (int)blockDim.x)
            bad |= !kv.exists(kv.table[(size_t)b * kv.max_pages + j]);
    return __syncthreads_or(bad);
}

// The tree of sequence b, or the chain where parent is null: depths in tree.cnt (counting the node itself) and, with words > 0,
// the ancestor bit rows in `bits`.  0, or first bad node + 1.  256 threads; nothing is done for a chain.
__device__ __forceinline__ int index_nodes(TreeLds &tree, uint32_t *bits, const int32_t *parent, int b, int n, int words) {
    return parent ? build_tree_index(tree, bits, parent + (size_t)b * n, n, n, words, 0.f, 0.f) : 0;
}

}  // namespace stree
