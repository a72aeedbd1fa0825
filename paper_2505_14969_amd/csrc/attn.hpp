// What the kernels of stree_tree_attn share: arguments, and how a sequence's keys are split over workgroups.
#pragma once
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

struct AttnArgs {
    const int32_t *parent, *lengths;
    const void *q;
    void *out;
    int32_t *status;
    long q_sn;
    int n, heads;
    float scale;                       // of <q, k>, in units of log2(e): probabilities are powers of two
};

// Queries as a matrix operand: the sign of the scale is theirs, so that the largest product is the largest score.
template <typename Frag>
__device__ __forceinline__ Frag signed_query(Frag q, float scale) { return scale < 0.f ? -q : q; }

// Factor of sums that were relative to the maximum m when the maximum is `top` >= m.  Never zero: an infinity among the sums,
// an infinite value that a row sees, stays one; what FLT_MIN leaves of anything else is nothing.
__device__ __forceinline__ float rescale(float m, float top) {
    return m == top ? 1.f : fmaxf(__builtin_amdgcn_exp2f(m - top), 1.17549435e-38f);
}

// sum + the values of a bf16 operand
__device__ __forceinline__ float sum_of(bf16x8 v, float sum) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const uint4 u = __builtin_bit_cast(uint4, v);
    const bf16x2_t one = {(__bf16)1.f, (__bf16)1.f};
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, u.x), one, sum, false);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, u.y), one, sum, false);
    sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, u.z), one, sum, false);
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, u.w), one, sum, false);
}
__device__ __forceinline__ float sum_of(floatx4 v, float sum) { return sum + ((v[0] + v[1]) + (v[2] + v[3])); }

constexpr int kTileKeys = 128;         // keys that the work is counted in: a step of bf16 keys for each of four waves

// The work of a call is B sequences x heads x tiles of their keys, which the device alone knows how many there are of: every
// worker (a workgroup, or one for each tile of rows) takes an equal share of the tiles in that order, so that lengths may
// differ as they like, and a sequence's head is cut where a share ends.  Parts of a head that was cut go to scratch, which has
// two slots a worker: only the first head of a share can have begun in an earlier one (slot 2 w), and only the last can go on
// (slot 2 w + 1).
struct AttnSplit {
    int workers, tiles, rows, batch;   // tiles of rows; rows: kept of each (fewer than the tile's where there is only one)
    bool spread;                       // a worker's tiles of rows are spread over the XCDs, not on one of them
    Divisor group;                     // query heads of a key/value head
    int2 *plan;                        // [units]: first worker of the unit and how many, written by the first
    float2 *sums;                      // [2 workers, tiles, rows]: (top, sum of 2^(s - top)); a negative sum: -attn_code()
    float *parts;                      // [2 workers, tiles, rows, dim]: sums of 2^(s - top) V
    explicit AttnSplit(int r) : group(r) {}
    // What a workgroup is: worker, and which of its workgroups.  On one XCD the tiles of rows share the keys and values through its
    // L2; spread out they fill the chip whatever their number.  (Workgroups go to the eight XCDs in turn.)
    unsigned grid() const { return (unsigned)(spread ? workers : (workers + 7) / 8 * 8) * (unsigned)tiles; }
    __device__ __forceinline__ int2 place(unsigned x) const {
        return spread ? make_int2((int)x / tiles, (int)x % tiles) : make_int2(((int)(x >> 3) / tiles) * 8 + (int)(x & 7), (int)(x >> 3) % tiles);
    }
    // row 0 of a worker's part of a tile of rows: of a head that begins there, or of one that began before
    __device__ __forceinline__ size_t part(int worker, bool begins, int tile) const {
        return ((size_t)(2 * worker + begins) * tiles + tile) * rows;
    }
};

// A value that all lanes of a wave have alike, for the compiler to keep it once.
__device__ __forceinline__ int uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) {
    return (int64_t)((uint64_t)(uint32_t)uniform((int)(v >> 32)) << 32 | (uint32_t)uniform((int)v));
}

// The same value, which the compiler takes for another: what is worked out from it inside a loop is not moved in front of the
// loop, to lie in registers all the while.
__device__ __forceinline__ int again(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

__device__ __forceinline__ int64_t quotient64(int64_t a, int64_t d) {       // a >= 0, d > 0; most are small
    return (a | d) >> 31 ? a / d : (int64_t)((uint32_t)a / (uint32_t)d);
}

// Equal shares of `total` tiles: the first `more` workers take one more than `each`.
struct Shares {
    int64_t each, bound;
    int workers, more;
    __device__ __forceinline__ Shares(int64_t total, int most) {
        workers = total < most ? (int)total : most;
        each = uniform(quotient64(total, workers));
        more = uniform((int)(total - each * workers));
        bound = (each + 1) * more;
    }
    __device__ __forceinline__ int64_t begin(int w) const { return w * each + min(w, more); }
    __device__ __forceinline__ int worker(int64_t x) const {
        return (int)(x < bound ? quotient64(x, each + 1) : more + quotient64(x - bound, each));
    }
};

// Tiles of a sequence; one for a sequence that gets zeros.
template <typename T>
__device__ __forceinline__ int tiles_of(const KvView<T> &kv, int len, int n) {
    return len < 0 || !kv.fits((int64_t)len + n) ? 1 : (len + n + kTileKeys - 1) / kTileKeys;
}

// Where a worker stands: head g of sequence b, of whose `tiles` tiles it takes [t0, t1); `left` tiles of its share from t0 on.
struct Share {
    int b, g, t0, t1, tiles, len;
    int64_t left;
    int workers;                       // of this call: none without a tile
    int64_t x;
    Shares shares;

    // Finds the worker's first tile; the whole workgroup calls it (`first`: a number of LDS for every thread, free again behind the next
    // barrier).  Up to 64 sequences each wave finds it by itself.
    template <int THREADS = kThreads, typename T>
    __device__ __forceinline__ static Share start(const AttnArgs &a, const KvView<T> &kv, const AttnSplit &sp, int worker, int64_t *first) {
        const int lane = threadIdx.x & 63;
        if (sp.batch <= 64) {
            const int l = lane < sp.batch ? a.lengths[lane] : 0, mine = lane < sp.batch ? tiles_of(kv, l, a.n) : 0;
            int sum = mine;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int u = __shfl_up(sum, o);
                if (lane >= o) sum += u;
            }
            Share s(Shares((int64_t)__builtin_amdgcn_readlane(sum, 63) * kv.heads, sp.workers));
            if (worker >= s.workers) return s;
            s.x = s.shares.begin(worker);
            s.b = uniform(__ffsll((long long)__ballot((int64_t)sum * kv.heads > s.x)) - 1);
            s.tiles = __builtin_amdgcn_readlane(mine, s.b), s.len = __builtin_amdgcn_readlane(l, s.b);
            s.place(s.x - (int64_t)(__builtin_amdgcn_readlane(sum, s.b) - s.tiles) * kv.heads, worker);
            return s;
        }
        // tiles in front of every run of sequences, one run a thread
        const int run = (sp.batch + THREADS - 1) / THREADS, wave = threadIdx.x >> 6;
        int64_t sum = 0;
        for (int y = threadIdx.x * run; y < min((int)(threadIdx.x + 1) * run, sp.batch); ++y) sum += tiles_of(kv, a.lengths[y], a.n);
        const int64_t mine = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t u = __shfl_up(sum, o);
            if (lane >= o) sum += u;
        }
        if (lane == 63) first[wave] = sum;
        __syncthreads();
        int64_t total = 0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            const int64_t u = first[w];
            if (w < wave) sum += u;
            total += u;
        }
        __syncthreads();
        first[threadIdx.x] = sum - mine;
        __syncthreads();
        Share s(Shares(uniform(total) * kv.heads, sp.workers));
        if (worker >= s.workers) return s;
        s.x = s.shares.begin(worker);
        int lo = 0, hi = THREADS;
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (first[mid] * kv.heads <= s.x) lo = mid;
            else hi = mid;
        }
        lo = uniform(lo);
        int64_t at = uniform(first[lo]) * kv.heads;
        for (s.b = min(lo * run, sp.batch - 1);; ++s.b) {
            s.len = a.lengths[s.b], s.tiles = tiles_of(kv, s.len, a.n);
            if (s.x < at + (int64_t)s.tiles * kv.heads || s.b == sp.batch - 1) break;
            at += (int64_t)s.tiles * kv.heads;
        }
        s.place(s.x - at, worker);
        return s;
    }
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == tiles; }
    // Which of `n` tiles of rows the workgroup `of` a worker's takes here: of every other head the last ones first, since of a long
    // chain the last rows see twice as many keys as the average (a prompt of 8192 tokens: 630 us, without 1095).
    __device__ __forceinline__ int row_tile(int heads, int of, int n) const { return (b * heads + g) & 1 ? n - 1 - of : of; }
    // on to the next head or sequence; false at the end of the share
    template <typename T>
    __device__ __forceinline__ bool next(const AttnArgs &a, const KvView<T> &kv) {
        const int done = t1 - t0;
        x += done, left -= done;
        if (left <= 0) return false;
        t0 = 0;
        if (++g == kv.heads) {
            g = 0, ++b;
            len = a.lengths[b], tiles = tiles_of(kv, len, a.n);
        }
        t1 = (int)min((int64_t)tiles, left);
        return true;
    }

  private:
    __device__ __forceinline__ explicit Share(const Shares &s) : left(0), workers(s.workers), shares(s) {}
    __device__ __forceinline__ void place(int64_t within, int worker) {
        g = uniform((int)quotient64(within, tiles)), t0 = uniform((int)(within - (int64_t)g * tiles));
        left = shares.begin(worker + 1) - x;
        t1 = (int)min((int64_t)tiles, t0 + left);
    }
};

// Numbers of the pages that a wave walks over, 64 at a time in its lanes and the next 64 on their way.
template <typename T>
struct PageWalk {
    int cur, next, first, seq = -1, stop;              // the windows of sequence `seq` from page `first` on, up to `stop`
    bool bad = false;
    __device__ __forceinline__ int window(const KvView<T> &kv, int b, int j0, int end, int lane) {
        const int j = j0 + lane;
        int pg = 0;
        if (j < end) {
            pg = kv.table[(size_t)b * kv.max_pages + j];
            if (!kv.exists(pg)) bad = true, pg = 0;
        }
        return pg;
    }
    __device__ __forceinline__ void none() { bad = false, seq = -1; }
    // The next head of a short sequence finds its pages where the last one left them (2048 sequences of 100 tokens: 292 us, with
    // the table read for every head 300).
    __device__ __forceinline__ void start(const KvView<T> &kv, int b, int j0, int end, int lane) {
        if (seq == b && first == j0 && stop == end) return;
        bad = false;
        first = j0, seq = b, stop = end;
        cur = window(kv, b, j0, end, lane);
        next = window(kv, b, j0 + 64, end, lane);
    }
    // pages from j on (j grows from call to call by less than 64)
    __device__ __forceinline__ void reach(const KvView<T> &kv, int b, int j, int end, int lane) {
        if (j - first >= 64) {
            first += 64;
            cur = next;
            next = window(kv, b, first + 64, end, lane);
        }
    }
    __device__ __forceinline__ int at(int j) const {
        const int r = j - first;
        return r < 64 ? __builtin_amdgcn_readlane(cur, r) : __builtin_amdgcn_readlane(next, r - 64);
    }
};

// The ancestor bit rows of the tree of sequence b, or first bad node + 1; the whole workgroup calls it.  Up to 64 nodes every wave
// finds all of them in its lanes, in as many steps as its depth has bits, and writes them where the others write the
// same: no barrier (16 trees of 64 nodes: 1 us in place of 5).
__device__ __forceinline__ int index_paths(TreeLds &tree, uint32_t *bits, const int32_t *__restrict__ parent, int b, int n) {
    const int words = (n + 31) / 32, lane = threadIdx.x & 63;
    if (n > 64) return index_nodes(tree, bits, parent, b, n, words);
    int p = lane < n ? parent[(size_t)b * n + lane] : -1;
    const unsigned long long wrong = __ballot(lane < n && (lane == 0 ? p != -1 : (p < 0 || p >= lane)));
    if (wrong) return __ffsll((long long)wrong);
    unsigned long long path = 1ull << lane;
    while (__any(p >= 0)) {                            // (at most six times: the way left is halved)
        const int at = p >= 0 ? p : lane, next = wave_read(p, at);
        const unsigned long long up = wave_read(path, at);
        if (p >= 0) path |= up, p = next;
    }
    if (lane < n)
        for (int w = 0; w < words; ++w) bits[lane * words + w] = (uint32_t)(path >> (32 * w));
    wave_sync();
    return 0;
}

// Which of E consecutive nodes from j0 on (negative: text) node i sees, bit by bit.
template <int E>
__device__ __forceinline__ uint32_t seen_nodes(const uint32_t *bits, int words, bool tree, int i, int j0) {
    constexpr uint32_t kAll = (1u << E) - 1u;
    if (!tree) {
        const int c = min(max(i - j0 + 1, 0), E);
        return (1u << c) - 1u;
    }
    if (j0 <= -E) return kAll;
    const int w = j0 >> 5;
    const uint32_t lo = w >= 0 && w < words ? bits[i * words + w] : 0u, hi = w + 1 < words ? bits[i * words + w + 1] : 0u;
    uint32_t v = (uint32_t)((((unsigned long long)hi << 32) | lo) >> (j0 & 31));
    if (j0 < 0) v |= (1u << -j0) - 1u;
    return v & kAll;
}

// What is wrong with a sequence as a small positive number, the first bad node before a page (two pieces may find both).
__device__ __forceinline__ int attn_code(int status) { return status > 0 ? status : 1000; }
__device__ __forceinline__ int attn_status(int code) { return code < 1000 ? code : STREE_SEQ_PAGE; }

// the streaming kernel (tree_attn_stream.hip)
bool attn_stream_supported(const stree_attn &a, const stree_kv &kv, const void *q, const void *out);
size_t attn_stream_workspace(const stree_attn &a, const stree_kv &kv);
hipError_t launch_attn_tile(const AttnArgs &a, const stree_kv &kv, const AttnSplit &sp, int rows, hipStream_t st);   // (tree_attn_tile.hip)
hipError_t launch_attn_stream(const stree_attn &at, const stree_kv &kv, const AttnArgs &a, void *workspace, hipStream_t st);

}  // namespace stree
