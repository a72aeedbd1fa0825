// stree_resize_kv and stree_fork_kv: who holds which page of the cache.  Whole numbers, kept by one workgroup, so that what a
// call does depends on the order of rows and entries alone: a page given back by several rows at once is put on the stack by
// the first of its entries, found by an atomic minimum over the entries' numbers in refs[] itself.
//
// A few thousand numbers at most: bound by the chain of dependent phases (reads, atomics in L2, barriers).  48 rows that drop up to
// 33 pages each 11 us, 64 that take one or two 5; 48 forks in 8 layers of 8 heads of 128, pages of 32 tokens: 9 us for the numbers
// and 14.5 for the pages (some 100 MB read and written, 6.9 TB/s).  Each phase of a drop looks up four entries of a thread at once:
// one at a time the same drop took 17 us.
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

namespace {

constexpr int kPool = 1024;                        // threads of the one workgroup
constexpr int kRows = 4096;                        // most rows, and forks, of a call
constexpr int kOwn = 4;                            // entries that a thread looks at together
static_assert(kOwn * (kPool / 64) == 64, "a round's counts are a wave's lanes");
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
    __shared__ int first[kRows + 1], need[kRows], state[kRows], part[64];
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
        // Entries are looked at in rounds of kOwn a thread, all of them at the same time; those of the first round stay in registers.
        struct Entry { int b, j, pg; };
        auto look_up = [&](int x, Entry (&e)[kOwn]) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int at = x + kPool * i;
                e[i] = {0, 0, -1};
                if (at < drops) e[i].b = row_of(first, batch, at), e[i].j = need[e[i].b] + at - first[e[i].b], e[i].pg = p.row(e[i].b)[e[i].j];
            }
        };
        Entry own[kOwn];
        int left[kOwn];                                // what refs says of the first round's pages in the end
        look_up(tid, own);
        // f(number of the round's first entry, its entries): by the whole workgroup
        auto rounds = [&](auto &&f) {
            f(tid, own);
            for (int x = tid + kOwn * kPool; x - tid < drops; x += kOwn * kPool) {
                Entry e[kOwn];
                look_up(x, e);
                f(x, e);
            }
        };
        auto counts = [&](const Entry (&e)[kOwn], int (&r)[kOwn]) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i) r[i] = p.exists(e[i].pg) ? load_count(&p.refs[e[i].pg]) : 1;
        };
        rounds([&](int, const Entry (&e)[kOwn]) {
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                if (p.exists(e[i].pg)) atomicSub(&p.refs[e[i].pg], 1);
        });
        __syncthreads();
        // the first entry of a page that nobody holds any more claims it
        rounds([&](int x, const Entry (&e)[kOwn]) {
            int r[kOwn];
            counts(e, r);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (x + kPool * i >= drops) break;
                if (!p.exists(e[i].pg)) state[e[i].b] = STREE_SEQ_PAGE;
                else if (r[i] == 0 || r[i] < kClaim / 2) atomicMin(&p.refs[e[i].pg], kClaim + x + kPool * i);
                else if (r[i] < 0) state[e[i].b] = STREE_SEQ_PAGE;    // (dropped more often than held)
            }
        });
        __syncthreads();
        // those that did put their pages on the stack, in the order of the entries: counted by waves, a round's counts in a wave's lanes
        const int lane = tid & 63, wave = tid >> 6;
        rounds([&](int x, const Entry (&e)[kOwn]) {
            int r[kOwn];
            counts(e, r);
            unsigned long long who[kOwn];
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                who[i] = __ballot(r[i] == kClaim + x + kPool * i);
                if (lane == 0) part[i * (kPool / 64) + wave] = __popcll(who[i]);
                if (x == tid) left[i] = r[i];
            }
            __syncthreads();
            const int mine = part[lane];
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int u = __shfl_up(sum, o);
                if (lane >= o) sum += u;
            }
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int to = nf + __shfl(sum - mine, i * (kPool / 64) + wave) + __popcll(who[i] & ((1ull << lane) - 1ull));
                if (((who[i] >> lane) & 1ull) && to < p.npages) p.free[to] = e[i].pg;
            }
            nf = min(nf + __shfl(sum, 63), p.npages);
            __syncthreads();
        });
        rounds([&](int x, const Entry (&e)[kOwn]) {
            int r[kOwn];
            if (x != tid) counts(e, r);
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (x + kPool * i >= drops) break;
                if ((x == tid ? left[i] : r[i]) < 0) store_count(&p.refs[e[i].pg], 0);
                p.row(e[i].b)[e[i].j] = -1;
            }
        });
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
