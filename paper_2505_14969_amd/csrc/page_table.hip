// stree_resize_kv and stree_fork_kv: who holds which page of the cache.  Whole numbers, kept by one workgroup, so that what a
// call does depends on the order of rows and entries alone: a page given back by several rows at once is put on the stack by
// the first of its entries, found by an atomic minimum over the entries' numbers in refs[] itself.
//
// A few thousand numbers at most: bound by the chain of dependent phases (reads, atomics in L2, barriers).
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

namespace {

constexpr int kPool = 1024;                        // threads of the one workgroup
constexpr int kRows = 4096;                        // most rows, and forks, of a call
constexpr int kClaim = INT32_MIN;                  // kClaim + number of the entry: far below any count

__device__ __forceinline__ int load_count(const int32_t *p) {       // (counts change by atomics, which L1 does not see)
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void store_count(int32_t *p, int v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive prefix sums of v over the workgroup; the sum of all in `total`.  Two barriers.
__device__ __forceinline__ int block_scan(int v, int *part, int &total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int s = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(s, o);
        if (lane >= o) s += u;
    }
    __syncthreads();                               // (the last call's parts are read)
    if (lane == 63) part[wave] = s;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kPool / 64; ++w) {
        const int p = part[w];
        if (w < wave) before += p;
        total += p;
    }
    return before + s - v;
}

// Exclusive prefix sums, in place, of n <= kRows numbers in LDS (v[n] = the sum); every thread gets the sum.
__device__ __forceinline__ int scan_rows(int *v, int n, int *part) {
    int run = 0;
    for (int r0 = 0; r0 < n; r0 += kPool) {
        const int r = r0 + threadIdx.x;
        int all;
        const int at = run + block_scan(r < n ? v[r] : 0, part, all);
        if (r < n) v[r] = at;
        run += all;
    }
    if (threadIdx.x == 0) v[n] = run;
    __syncthreads();
    return run;
}

// the row that entry x of all rows' entries belongs to: the last r with first[r] <= x
__device__ __forceinline__ int row_of(const int *first, int n, int x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= x) lo = mid;
        else hi = mid;
    }
    return lo;
}

struct PoolView {
    int32_t *table, *held, *refs, *free, *nfree;
    int npages, shift, max_pages;
    PoolView(const stree_kv &kv, const stree_pool &p)
        : table(kv.table), held(p.held), refs(p.refs), free(p.free), nfree(p.nfree), npages(kv.npages),
          shift(__builtin_ctz((unsigned)kv.page)), max_pages(kv.max_pages) {}
    __device__ __forceinline__ bool exists(int pg) const { return (unsigned)pg < (unsigned)npages; }
    __device__ __forceinline__ int pages(int tokens) const { return (int)(((int64_t)tokens + (1 << shift) - 1) >> shift); }
    __device__ __forceinline__ int32_t *row(int b) const { return table + (size_t)b * max_pages; }
};

__global__ __launch_bounds__(kPool) void resize_kernel(PoolView p, int batch, const int32_t *__restrict__ tokens, int32_t *status) {
    __shared__ int first[kRows + 1], need[kRows], state[kRows], part[kPool / 64];
    const int tid = threadIdx.x;
    int nf = *p.nfree;
    if (nf < 0 || nf > p.npages) {
        if (status)
            for (int b = tid; b < batch; b += kPool) status[b] = STREE_SEQ_POOL;
        return;
    }
    // what each row drops
    for (int b = tid; b < batch; b += kPool) {
        const int h = p.held[b], t = tokens[b];
        const bool ok = h >= 0 && h <= p.max_pages && (int64_t)t <= (int64_t)p.max_pages << p.shift;
        const int n = !ok || t < 0 ? h : p.pages(t);
        need[b] = n;
        state[b] = ok ? 0 : STREE_SEQ_LENGTH;
        first[b] = h > n ? h - n : 0;
    }
    __syncthreads();
    const int drops = scan_rows(first, batch, part);
    if (drops) {                                       // (alike in all threads)
        // An entry's row and page: a thread's first entry is looked up once.
        struct Entry { int b, j, pg; };
        auto entry = [&](int x) {
            Entry e;
            e.b = row_of(first, batch, x), e.j = need[e.b] + x - first[e.b], e.pg = p.row(e.b)[e.j];
            return e;
        };
        Entry mine = {0, 0, -1};
        if (tid < drops) mine = entry(tid);
        auto at = [&](int x) { return x == tid ? mine : entry(x); };
        for (int x = tid; x < drops; x += kPool) {
            const int pg = at(x).pg;
            if (p.exists(pg)) atomicSub(&p.refs[pg], 1);
        }
        __syncthreads();
        // the first entry of a page that nobody holds any more claims it
        for (int x = tid; x < drops; x += kPool) {
            const Entry e = at(x);
            if (!p.exists(e.pg)) {
                state[e.b] = STREE_SEQ_PAGE;
                continue;
            }
            const int r = load_count(&p.refs[e.pg]);
            if (r == 0 || r < kClaim / 2) atomicMin(&p.refs[e.pg], kClaim + x);
            else if (r < 0) state[e.b] = STREE_SEQ_PAGE;              // (dropped more often than held)
        }
        __syncthreads();
        int held_on = 1;                               // what refs says of a thread's first page: other than negative, nothing is to be done
        for (int x0 = 0; x0 < drops; x0 += kPool) {
            const int x = x0 + tid;
            int pg = -1;
            if (x < drops) {
                const Entry e = at(x);
                const int r = p.exists(e.pg) ? load_count(&p.refs[e.pg]) : 1;
                if (x0 == 0) held_on = r;
                if (r == kClaim + x) pg = e.pg;
            }
            int all;
            const int to = nf + block_scan(pg >= 0, part, all);
            if (pg >= 0 && to < p.npages) p.free[to] = pg;
            nf = min(nf + all, p.npages);
        }
        __syncthreads();
        for (int x = tid; x < drops; x += kPool) {
            const Entry e = at(x);
            if (p.exists(e.pg) && (x == tid ? held_on : load_count(&p.refs[e.pg])) < 0) store_count(&p.refs[e.pg], 0);
            p.row(e.b)[e.j] = -1;
        }
        __syncthreads();
    }
    // growth: a prefix of the growing rows, as far as the free pages go
    for (int b = tid; b < batch; b += kPool) {
        const int h = p.held[b];
        first[b] = need[b] > h ? need[b] - h : 0;
    }
    __syncthreads();
    int taken = 0;
    if (scan_rows(first, batch, part)) {
        for (int b0 = 0; b0 < batch; b0 += kPool) {
            const int b = b0 + tid;
            int grow = 0;
            if (b < batch) {
                grow = first[b + 1] - first[b];
                if (grow && first[b + 1] > nf) {
                    state[b] = STREE_SEQ_POOL;
                    grow = 0;
                }
            }
            int all;
            block_scan(grow, part, all);
            taken += all;
        }
        for (int x = tid; x < taken; x += kPool) {
            const int b = row_of(first, batch, x), pg = p.free[nf - 1 - x];
            p.row(b)[need[b] - first[b + 1] + x] = pg;                // (the row's own entries end at need - growth)
            if (p.exists(pg)) store_count(&p.refs[pg], 1);
            else state[b] = STREE_SEQ_PAGE;                           // (the stack of free pages is damaged)
        }
        __syncthreads();
    }
    for (int b = tid; b < batch; b += kPool) {
        if (state[b] != STREE_SEQ_POOL) p.held[b] = need[b];
        if (status) status[b] = state[b];
    }
    if (tid == 0) *p.nfree = nf - taken;
}

__global__ __launch_bounds__(kPool) void fork_kernel(PoolView p, int batch, int nforks, const int32_t *__restrict__ src,
                                                     const int32_t *__restrict__ dst, int32_t *lengths, int32_t *status) {
    __shared__ int length[kRows], state[kRows], before[kRows + 1], part[kPool / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int nf = *p.nfree;
    if (nf < 0 || nf > p.npages) {
        for (int f = tid; f < nforks; f += kPool) status[f] = STREE_SEQ_POOL;
        return;
    }
    for (int f = tid; f < nforks; f += kPool) {
        const int s = src[f], d = dst[f];
        int st = STREE_SEQ_LENGTH, len = 0;
        if (s >= 0 && s < batch && d >= 0 && d < batch) {
            len = lengths[s];
            const int h = p.held[s];
            if (len >= 0 && h >= 0 && h <= p.max_pages && p.pages(len) <= h) st = p.held[d] != 0 ? STREE_SEQ_HELD : 0;
        }
        length[f] = len;
        state[f] = st;
    }
    __syncthreads();
    // src's pages, a wave per fork
    for (int f = wave; f < nforks; f += kPool / 64) {
        if (state[f] == STREE_SEQ_LENGTH) continue;
        const int32_t *row = p.row(src[f]);
        bool bad = false;
        for (int j = lane; j < p.pages(length[f]); j += 64) bad |= !p.exists(row[j]) || load_count(&p.refs[row[j]]) <= 0;
        const bool any = __any(bad);               // (all lanes have read state[f])
        if (lane == 0 && any) state[f] = STREE_SEQ_PAGE;
    }
    __syncthreads();
    for (int f = tid; f < nforks; f += kPool)
        if (state[f] == 0) atomicMin(&p.held[dst[f]], kClaim + f);
    __syncthreads();
    for (int f = tid; f < nforks; f += kPool) {
        if (state[f] == 0 && load_count(&p.held[dst[f]]) != kClaim + f) state[f] = STREE_SEQ_HELD;
        before[f] = state[f] == 0 && (length[f] & ((1 << p.shift) - 1));
    }
    __syncthreads();
    scan_rows(before, nforks, part);
    const int taken = min(before[nforks], nf);
    for (int f = tid; f < nforks; f += kPool) {
        if (state[f]) continue;
        const int d = dst[f], full = length[f] >> p.shift;
        const bool partial = before[f + 1] > before[f];
        int fresh = -1;
        if (partial) {
            if (before[f] >= nf) state[f] = STREE_SEQ_POOL;
            else if (fresh = p.free[nf - 1 - before[f]]; !p.exists(fresh)) state[f] = STREE_SEQ_PAGE;
        }
        if (state[f]) {
            store_count(&p.held[d], 0);
            continue;
        }
        if (partial) {
            p.row(d)[full] = fresh;
            store_count(&p.refs[fresh], 1);
        }
        store_count(&p.held[d], full + partial);
        lengths[d] = length[f];
    }
    __syncthreads();
    for (int f = wave; f < nforks; f += kPool / 64) {
        if (state[f]) continue;
        const int32_t *from = p.row(src[f]);
        int32_t *to = p.row(dst[f]);
        for (int j = lane; j < length[f] >> p.shift; j += 64) {
            const int pg = from[j];
            to[j] = pg;
            atomicAdd(&p.refs[pg], 1);
        }
    }
    for (int f = tid; f < nforks; f += kPool) status[f] = state[f];
    if (tid == 0) *p.nfree = nf - taken;
}

// The partial pages: workgroups (piece, layer, fork), whole pages of all heads, in pieces of V.
template <typename V>
__global__ __launch_bounds__(kThreads) void fork_copy_kernel(const int32_t *__restrict__ src, const int32_t *__restrict__ dst,
                                                             const int32_t *__restrict__ lengths, const int32_t *__restrict__ status,
                                                             const int32_t *__restrict__ table, int max_pages, int shift, V *k, V *v,
                                                             size_t layer, int page_pieces) {
    const int f = blockIdx.z;
    if (status[f]) return;
    const int d = dst[f], len = lengths[d], full = len >> shift;
    if (!(len & ((1 << shift) - 1))) return;
    const int from = table[(size_t)src[f] * max_pages + full], to = table[(size_t)d * max_pages + full];
    k += blockIdx.y * layer;
    v += blockIdx.y * layer;
    for (int x = blockIdx.x * kThreads + threadIdx.x; x < page_pieces; x += gridDim.x * kThreads) {
        const V a = k[(size_t)from * page_pieces + x], c = v[(size_t)from * page_pieces + x];
        k[(size_t)to * page_pieces + x] = a;
        v[(size_t)to * page_pieces + x] = c;
    }
}

}  // namespace

hipError_t launch_resize_kv(const stree_kv &kv, const stree_pool &pool, int batch, const int32_t *tokens, int32_t *status,
                            hipStream_t st) {
    hipLaunchKernelGGL(resize_kernel, dim3(1), dim3(kPool), 0, st, PoolView(kv, pool), batch, tokens, status);
    return hipGetLastError();
}

hipError_t launch_fork_kv(const stree_kv &kv, const stree_pool &pool, int batch, int nforks, const int32_t *src, const int32_t *dst,
                          int32_t *lengths, int32_t *status, hipStream_t st) {
    const PoolView p(kv, pool);
    hipLaunchKernelGGL(fork_kernel, dim3(1), dim3(kPool), 0, st, p, batch, nforks, src, dst, lengths, status);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const size_t bytes = (size_t)kv.nheads_kv * kv.page * kv.headdim * (kv.io_dtype == STREE_BF16 ? 2 : 4);
    const bool wide = (((uintptr_t)kv.k | (uintptr_t)kv.v) % 16) == 0;       // (a page is a whole number of 16 bytes)
    const size_t pieces = wide ? bytes / 16 : bytes / 2;
    const unsigned groups = (unsigned)((pieces + 4 * kThreads - 1) / (4 * kThreads));
    const dim3 grid(groups, (unsigned)kv.nlayers, (unsigned)nforks);
    if (wide)
        hipLaunchKernelGGL((fork_copy_kernel<uint4>), grid, dim3(kThreads), 0, st, src, dst, lengths, status, kv.table, kv.max_pages, p.shift,
                           (uint4 *)kv.k, (uint4 *)kv.v, pieces * kv.npages, (int)pieces);
    else
        hipLaunchKernelGGL((fork_copy_kernel<uint16_t>), grid, dim3(kThreads), 0, st, src, dst, lengths, status, kv.table, kv.max_pages,
                           p.shift, (uint16_t *)kv.k, (uint16_t *)kv.v, pieces * kv.npages, (int)pieces);
    return hipGetLastError();
}

}  // namespace stree
