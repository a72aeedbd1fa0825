// The tuned kernel of stree_tree_attn: the cache streamed once from memory straight into operand registers.
//
// A workgroup takes 16 or 32 query rows (node, head) of one key/value head and one piece of the sequence's keys; its
// four waves take the piece's keys in turn, STEP at a time.  Products are formed transposed, so that in
// every accumulator a lane owns one query row (column lane % 16):
//   S^T = K Q^T,   P = 2^(S - m),   O^T += V^T P^T
// Which key stands in which row of S^T is free, so keys are read in the order that makes a lane's probabilities the very
// operand of the second product; V lies transposed in the cache, so its operand too is 16 consecutive bytes.  No LDS, no
// barrier and no shuffle in the loop: the maximum is moved only when a score passes it by kSlack (2^kSlack is harmless in
// fp32), which a vote finds out.  Waves are joined through LDS at the end, pieces by a second kernel.
//
// Bound by memory: 16 rows take 384 cycles of the matrix unit per 32 keys (bf16, heads of 128) where the chip's memory needs 5000 to
// bring them.  4 rows of 8 key/value heads: 64 sequences of up to 4096 tokens 116 us (676 MB, 5.8 TB/s), one of 131071 100 us
// (537 MB, 5.4 TB/s); a read of nothing but such pages reaches 6.8 TB/s here.  fp32, 64 sequences of up to 2048 124 us (677 MB,
// 5.5 TB/s); 60 rows behind 500 tokens 16.5 us, of which 3.9 join parts, the rest is the chain launch -> lengths -> pages -> keys
// -> products.
#include "attn.hpp"

namespace stree {

namespace {

constexpr float kSlack = 8.f;
constexpr int kWaves = kThreads / 64;
constexpr int kChip = 256;                            // CUs

// 16 bytes of a row as a matrix operand, and the two products, per type.
template <typename T>
struct Mma;
template <>
struct Mma<bf16_t> {
    typedef bf16x8 Frag;
    static constexpr int E = 8, KB = 2;               // values of 16 bytes; blocks of 16 keys a step
    static __device__ __forceinline__ floatx4 qk(Frag k, Frag q, floatx4 s) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q, s, 0, 0, 0); }
    static __device__ __forceinline__ floatx4 pv(Frag v, Frag p, floatx4 o) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0); }
    static __device__ __forceinline__ Frag round(const float (&p)[8]) {
        Frag f;
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (bf16_t)p[e];
        return f;
    }
};
template <>
struct Mma<float> {
    typedef floatx4 Frag;
    static constexpr int E = 4, KB = 1;
    static __device__ __forceinline__ floatx4 qk(Frag k, Frag q, floatx4 s) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_16x16x4f32(k[e], q[e], s, 0, 0, 0);
        return s;
    }
    static __device__ __forceinline__ floatx4 pv(Frag v, Frag p, floatx4 o) { return qk(v, p, o); }
    static __device__ __forceinline__ Frag round(const float (&p)[4]) { return Frag{p[0], p[1], p[2], p[3]}; }
};

template <typename T, int PP, int MB>
struct StreamShape {
    static constexpr int kRows = 16 * MB;
    static constexpr int kSlice = PP * kRows <= 2048 ? PP : 2048 / kRows;        // columns joined at a time: 32 KB of LDS
    static constexpr int kLd = kSlice + 4;
    // Waves on a SIMD: one where a head's operands need more than half of the registers (64 sequences of 2000 tokens, heads of
    // 256: 175 us, with two 295), else two (32 rows of 128, 16 sequences of 2000 tokens: 40 us, with one 49).
    static constexpr int kMinWaves = PP <= 128 ? 2 : 1;
};

template <typename T, int PP, int MB, bool WHOLE>
__global__ __launch_bounds__(kThreads, (StreamShape<T, PP, MB>::kMinWaves)) void attn_stream_kernel(AttnArgs a, KvView<T> kv, AttnSplit sp) {
    typedef Mma<T> M;
    typedef typename M::Frag Frag;
    typedef StreamShape<T, PP, MB> Shape;
    constexpr int E = M::E, KB = M::KB, STEP = 16 * KB, NK = PP / (4 * E), NP = PP / 16, ROWS = Shape::kRows, STRIDE = kWaves * STEP, SL = Shape::kSlice, LD = Shape::kLd;
    // What a rounding to bf16 leaves of a probability goes through a second product, and 15 bits of it count (half a step, 2^-8, of a
    // rest of at most 2^-7).  That costs the matrix unit time that memory leaves over: 64 sequences, one token, 116 us with and
    // without.  With 32 rows one rounding is all: the second product would take up to 5 % there (heads of 80, two prompts of 512: 97
    // and 102 us), and 18 to 35 % in the kernel of many rows.  The first part is kept below the whole, so that the rest is above
    // zero like it: an infinite value then gives the same infinity twice.
    constexpr bool REST = sizeof(T) == 2 && MB == 1;
    struct Index { TreeLds tree; uint32_t bits[kMaxNodes * kMaxWords]; };
    __shared__ union { Index index; float o[kWaves][ROWS][LD]; int64_t first[kThreads + 1]; } lds;
    __shared__ float ml[kWaves][ROWS][2];
    const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), P = kv.dim;
    const int2 here = sp.place(blockIdx.x);
    const int worker = here.x, group = here.y;
    if (worker >= sp.workers) return;
    const int R = sp.group.d, rows = a.n * R;
    T *const out = static_cast<T *>(a.out);
    const float scale = fabsf(a.scale);
    Share at = Share::start(a, kv, sp, worker, lds.first);
    if (worker >= at.workers) return;
    if (sp.batch > 64) __syncthreads();                // (its numbers lay where the tree goes)

    // What the waves are at: the piece's keys up to k1 (these rows see no more of it) and `whole` (where it ends), the page
    // numbers, the queries, and the keys and values of the next step, always on their way.  The waves take the piece's steps
    // in turn: a line of a page of many tokens holds the values of several steps, which are then asked for at nearly the same
    // time.
    const int shift = kv.shift, mask = kv.mask();
    const size_t block = (size_t)P << shift;
    const bool lines = (sizeof(T) << shift) <= 64;
    int k0 = 0, k1 = 0, whole = 0, end = 0;
    PageWalk<T> walk;
    Frag q[MB][NK], kf[KB][NK], vf[NP];
    const T *kp, *vp;                                  // this lane's key row and first value of the step
    // Keys in the order that gives lane group `grp` the tokens E grp .. E grp + E - 1 of the step.
    auto place = [&](int t, int col, int grp) {
        const int ktok = E * (col >> 2) + (col & 3), vtok = E * grp, vrow = WHOLE || col < P ? col : 0;
        walk.reach(kv, at.b, t >> shift, end, lane);
        const int pa = walk.at(t >> shift);
        int pk = pa, pv = pa;
        if (STEP > 16 && shift == 4) {                 // a step of two pages
            const int pb = (t >> 4) + 1 < end ? walk.at((t >> 4) + 1) : pa;
            pk = ktok < 16 ? pa : pb, pv = vtok < 16 ? pa : pb;
        }
        kp = kv.k + ((size_t)pk * kv.heads + at.g) * block + (size_t)((t + ktok) & mask) * P + grp * E;
        vp = kv.v + ((size_t)pv * kv.heads + at.g) * block + ((size_t)vrow << shift) + ((t + vtok) & mask);
    };
    // Pages of up to 64 bytes a row of V come in whole lines, once: with the streaming hint.  Larger pages have the values of
    // several steps in a line, and without the hint the next wave finds it in L2.
    auto load_k = [&](int grp) {
        auto from = [&](int x, int c) { return reinterpret_cast<const uint4 *>(kp + 4 * x * P + (WHOLE || (4 * c + grp) * E < P ? 4 * c * E : -grp * E)); };
        if (lines) {
            asm volatile("; whole lines");             // (the two kinds of loads are not to be made one)
#pragma unroll
            for (int x = 0; x < KB; ++x)
#pragma unroll
                for (int c = 0; c < NK; ++c) kf[x][c] = __builtin_bit_cast(Frag, load_stream16(from(x, c)));
            asm volatile("; whole lines");
        } else {
#pragma unroll
            for (int x = 0; x < KB; ++x)
#pragma unroll
                for (int c = 0; c < NK; ++c) kf[x][c] = __builtin_bit_cast(Frag, *from(x, c));
        }
    };
    auto load_v = [&](int col) {
        auto from = [&](int p) { return reinterpret_cast<const uint4 *>(vp + (WHOLE || 16 * p + col < P ? (size_t)(16 * p) << shift : (size_t)0)); };
        if (lines) {
            asm volatile("; whole lines");
#pragma unroll
            for (int p = 0; p < NP; ++p) vf[p] = __builtin_bit_cast(Frag, load_stream16(from(p)));
            asm volatile("; whole lines");
        } else {
#pragma unroll
            for (int p = 0; p < NP; ++p) vf[p] = __builtin_bit_cast(Frag, *from(p));
        }
    };
    // A new piece: everything that does not wait for its first keys.
    auto enter = [&]() {
        const int col = again(lane) & 15, grp = again(lane) >> 4;
        const int row0 = at.row_tile(kv.heads, group, sp.tiles) * ROWS;
        k0 = k1 = whole = 0;
        if (at.len >= 0 && kv.fits((int64_t)at.len + a.n)) {
            const int last = sp.group.quotient(min(row0 + ROWS, rows) - 1);
            k0 = at.t0 * kTileKeys, whole = min(at.t1 * kTileKeys, at.len + a.n);
            k1 = min(whole, at.len + last + 1);
        }
        const int t = k0 + wave * STEP;
        end = ((k1 - 1) >> shift) + 1;                 // (alike in all waves, those that have no keys of their own too: they share the pages behind)
        if (t >= k1) return walk.none();
        walk.start(kv, at.b, t >> shift, end, lane);
        // queries: row `col` of each block, 16 bytes at column (4 c + grp) E; zeros behind the head and the last row
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int r = row0 + mb * 16 + col, rr = min(r, rows - 1), i = sp.group.quotient(rr), h = at.g * R + rr - i * R;
            const T *src = static_cast<const T *>(a.q) + ((size_t)at.b * a.n + i) * a.q_sn + (size_t)h * P;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const int x = (4 * c + grp) * E;
                const bool there = r < rows && x < P;
                const uint4 v = *reinterpret_cast<const uint4 *>(src + (there ? x : 0));
                q[mb][c] = signed_query(__builtin_bit_cast(Frag, there ? v : make_uint4(0u, 0u, 0u, 0u)), a.scale);
            }
        }
        place(t, col, grp);
        load_k(grp);
        load_v(col);
    };
    enter();
    for (;;) {
        // tiles [t0, t1) of head g of sequence b
        const int b = at.b, g = at.g, len = at.len, w1 = k1, col = again(lane) & 15, grp = again(lane) >> 4, vtok = E * grp;
        const int tile = at.row_tile(kv.heads, group, sp.tiles), row0 = tile * ROWS, mine = min(ROWS, rows - row0);
        const int unit = b * kv.heads + g;
        const bool direct = at.whole(), begins = at.t0 == 0;
        if (begins && sp.plan && tile == 0 && threadIdx.x == 0)
            sp.plan[unit] = make_int2(worker, direct ? 1 : at.shares.worker(at.x + at.tiles - 1) - worker + 1);
        int bad = len >= 0 && !kv.fits((int64_t)len + a.n) ? STREE_SEQ_LENGTH : 0;
        if (whole > len && len >= 0 && whole > 0 && a.parent) bad = index_paths(lds.index.tree, lds.index.bits, a.parent, b, a.n);

        float m[MB], base[MB], l[MB];
        floatx4 o[MB][NP];
        int node[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            node[mb] = sp.group.quotient(min(row0 + mb * 16 + col, rows - 1));
            m[mb] = -INFINITY, base[mb] = 0.f, l[mb] = 0.f;
#pragma unroll
            for (int p = 0; p < NP; ++p) o[mb][p] = floatx4{0.f, 0.f, 0.f, 0.f};
        }
        const int clear = min(w1, len + (a.parent ? 0 : sp.group.quotient(row0) + 1));     // all of these rows see the keys up to here
        for (int t = k0 + wave * STEP; t < w1; t += STRIDE) {
            if (!WHOLE) {
                // Behind the head stand other columns of the row, which may be infinite: zeros, as the query has there.
#pragma unroll
                for (int c = 0; c < NK; ++c)
#pragma unroll
                    for (int x = 0; x < KB; ++x) {
                        const uint4 v = __builtin_bit_cast(uint4, kf[x][c]);
                        kf[x][c] = __builtin_bit_cast(Frag, (4 * c + grp) * E < P ? v : make_uint4(0u, 0u, 0u, 0u));
                    }
            }
            floatx4 s[MB][KB];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int x = 0; x < KB; ++x) {
                    s[mb][x] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < NK; ++c) s[mb][x] = M::qk(kf[x][c], q[mb][c], s[mb][x]);
                }
            __builtin_amdgcn_sched_barrier(0);         // (the next keys take these keys' registers, not others)
            const bool more = t + STRIDE < w1;
            if (more) {
                place(t + STRIDE, col, grp);
                load_k(grp);
            }
            const bool tail = t + STEP > clear;
            uint32_t seen[MB];
            float p[MB][E], top[MB];
            bool above = false;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                top[mb] = -INFINITY;
                if (tail) {
                    seen[mb] = seen_nodes<E>(lds.index.bits, (a.n + 31) / 32, a.parent != nullptr, node[mb], t + vtok - len);
                    const int left = w1 - t - vtok;            // (keys behind the last)
                    seen[mb] &= left >= E ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float v = s[mb][e >> 2][e & 3];
                    if (tail && !((seen[mb] >> e) & 1u)) v = -INFINITY;
                    p[mb][e] = v;
                    top[mb] = fmaxf(top[mb], v);
                }
                top[mb] *= scale;
                above |= top[mb] > m[mb] + kSlack;
            }
            if (__builtin_expect(__any(above), 0)) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    float v = fmaxf(top[mb], __shfl_xor(top[mb], 16));
                    v = fmaxf(m[mb], fmaxf(v, __shfl_xor(v, 32)));
                    const float b2 = v == -INFINITY ? 0.f : v, keep = rescale(m[mb], v);
                    m[mb] = v, base[mb] = b2;
                    l[mb] *= keep;
#pragma unroll
                    for (int x = 0; x < NP; ++x) o[mb][x] *= keep;
                }
            }
            if (__builtin_expect(tail, 0)) {
                // Values behind the last key are no numbers anybody wrote.  Those of nodes may be infinite or NaN, which zero
                // probabilities would not keep from the rows that do not see the node: they are counted per row instead.
                const int left = w1 - t - vtok;
                bool odd = false;
#pragma unroll
                for (int x = 0; x < NP; ++x)
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        if (e >= left) vf[x][e] = (T)0.f;
                        odd |= !(fabsf((float)vf[x][e]) < INFINITY);
                    }
                if (__builtin_expect(__any(odd), 0)) {
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) {
                        Frag see;
#pragma unroll
                        for (int e = 0; e < E; ++e) see[e] = (T)((seen[mb] >> e) & 1u ? 1.f : 0.f);
#pragma unroll
                        for (int x = 0; x < NP; ++x) {
                            Frag up, down;
#pragma unroll
                            for (int e = 0; e < E; ++e) {
                                const float v = (float)vf[x][e];
                                up[e] = (T)(v < INFINITY ? 0.f : 1.f);             // +inf, NaN
                                down[e] = (T)(v > -INFINITY ? 0.f : 1.f);          // -inf, NaN
                            }
                            const floatx4 zero = {0.f, 0.f, 0.f, 0.f};
                            const floatx4 cu = M::pv(up, see, zero), cd = M::pv(down, see, zero);
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                if (cu[e] > 0.f) o[mb][x][e] += INFINITY;
                                if (cd[e] > 0.f) o[mb][x][e] -= INFINITY;          // (both: NaN)
                            }
                        }
                    }
#pragma unroll
                    for (int x = 0; x < NP; ++x)
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (!(fabsf((float)vf[x][e]) < INFINITY)) vf[x][e] = (T)0.f;
                }
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
#pragma unroll
                for (int e = 0; e < E; ++e) p[mb][e] = __builtin_amdgcn_exp2f(fmaf(p[mb][e], scale, -base[mb]));
                if constexpr (REST) {
                    float most[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) most[e] = p[mb][e] * (1.f - 0x1p-8f);
                    const Frag pf = M::round(most);
#pragma unroll
                    for (int e = 0; e < E; ++e) p[mb][e] -= (float)pf[e];
                    const Frag rest = M::round(p[mb]);
                    l[mb] = sum_of(rest, sum_of(pf, l[mb]));
#pragma unroll
                    for (int x = 0; x < NP; ++x) o[mb][x] = M::pv(vf[x], pf, o[mb][x]);
#pragma unroll
                    for (int x = 0; x < NP; ++x) o[mb][x] = M::pv(vf[x], rest, o[mb][x]);
                } else {
                    const Frag pf = M::round(p[mb]);   // bf16: one rounding of each probability, and their sum is the rounded ones'
                    l[mb] = sum_of(pf, l[mb]);
#pragma unroll
                    for (int x = 0; x < NP; ++x) o[mb][x] = M::pv(vf[x], pf, o[mb][x]);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_v(col);
        }
        // (pages of the piece that only later rows see)
        int missing = walk.bad;
        for (int j = (k0 < k1 ? end : k0 >> shift) + (int)threadIdx.x; j < (whole + mask) >> shift; j += kThreads) missing |= !kv.exists(kv.table[(size_t)b * kv.max_pages + j]);
        if (__syncthreads_or(missing) && bad == 0) bad = STREE_SEQ_PAGE;
        // the next piece's first keys are on their way while this one's waves are joined
        const bool more = at.next(a, kv);
        if (more) enter();

        // join the waves
        {
        const int tid = again((int)threadIdx.x), col = tid & 15, grp = (tid >> 4) & 3;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            l[mb] += __shfl_xor(l[mb], 16);
            l[mb] += __shfl_xor(l[mb], 32);
            if (grp == 0) ml[wave][mb * 16 + col][0] = m[mb], ml[wave][mb * 16 + col][1] = l[mb];
        }
        __syncthreads();
        float keep[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int r = mb * 16 + col;
            float top = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][r][0]);
            keep[mb] = rescale(m[mb], top);
        }
        const bool dead = len < 0 || bad != 0;
        const size_t slot = sp.part(worker, begins, tile);
        for (int c0 = 0; c0 < PP; c0 += SL) {
            if (c0) __syncthreads();
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int x = 0; x < NP; ++x)
                    if (16 * x >= c0 && 16 * x < c0 + SL)
                        *reinterpret_cast<floatx4 *>(&lds.o[wave][mb * 16 + col][16 * x - c0 + 4 * grp]) = o[mb][x] * keep[mb];
            __syncthreads();
            for (int y = tid; y < mine * (SL / 4); y += kThreads) {
                const int r = y / (SL / 4), c = c0 + y % (SL / 4) * 4;
                if (c >= P) continue;
                floatx4 v = {0.f, 0.f, 0.f, 0.f};
                float top = -INFINITY, all = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][r][0]);
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    all += ml[w][r][1] * rescale(ml[w][r][0], top);
                    v += *reinterpret_cast<const floatx4 *>(&lds.o[w][r][c - c0]);
                }
                if (direct) {
                    const int i = sp.group.quotient(row0 + r), h = g * R + row0 + r - i * R;
                    T *dst = out + (((size_t)b * a.n + i) * a.heads + h) * P + c;
#pragma unroll
                    for (int e = 0; e < 4; ++e) from_f32(dead ? 0.f : v[e] / all, dst[e]);
                } else {
                    if (!dead) *reinterpret_cast<floatx4 *>(sp.parts + (slot + r) * P + c) = v;
                    if (c == 0) sp.sums[slot + r] = make_float2(top, bad ? -(float)attn_code(bad) : all);
                }
            }
        }
        }
        if (direct && a.status && g == 0 && tile == 0 && threadIdx.x == 0) a.status[b] = bad;
        if (!more) break;
        __syncthreads();                                   // (LDS is read)
    }
}

// Joins the parts of the rows of a unit that was cut: workgroup (some rows, unit).  A few parts: a row's columns over lanes,
// as many rows at once as there are lanes for.  Many: one row at a time, lanes over columns and parts.
constexpr int kFewParts = 8;
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs a, KvView<T> kv, AttnSplit sp, int tile_rows) {
    __shared__ float4 acc[kThreads];
    __shared__ float factor[kThreads], red[kWaves][2];
    const int unit = blockIdx.y, P = kv.dim, R = sp.group.d, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int2 plan = sp.plan[unit];
    if (plan.y == 1) return;
    const int g = unit % kv.heads, b = unit / kv.heads, rows = a.n * R;
    const int quads = P / 4, over = kThreads / quads, c = tid % quads, s0 = tid / quads;
    auto slot_of = [&](int tile, int r, int s) { return sp.part(plan.x + s, s == 0, tile) + r; };
    if (plan.y <= kFewParts) {
        if (s0 >= over) return;
        for (int row = blockIdx.x * over + s0; row < rows; row += gridDim.x * over) {
            const int tile = row / tile_rows, r = row - tile * tile_rows;
            float2 w[kFewParts];
            float4 p[kFewParts];
            float top = -INFINITY, code = -INFINITY;
#pragma unroll
            for (int s = 0; s < kFewParts; ++s) {
                w[s] = make_float2(-INFINITY, 0.f);
                if (s < plan.y) {
                    const size_t slot = slot_of(tile, r, s);
                    w[s] = sp.sums[slot];
                    p[s] = *reinterpret_cast<const float4 *>(sp.parts + slot * P + 4 * c);
                }
            }
#pragma unroll
            for (int s = 0; s < kFewParts; ++s) {
                top = fmaxf(top, w[s].x);
                if (w[s].y < 0.f) code = fmaxf(code, w[s].y);
            }
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
#pragma unroll
            for (int s = 0; s < kFewParts; ++s)
                if (s < plan.y) {
                    const float f = rescale(w[s].x, top);
                    sum += w[s].y * f;
                    v.x = fmaf(p[s].x, f, v.x), v.y = fmaf(p[s].y, f, v.y), v.z = fmaf(p[s].z, f, v.z), v.w = fmaf(p[s].w, f, v.w);
                }
            if (code > -INFINITY) v = make_float4(0.f, 0.f, 0.f, 0.f), sum = 1.f;
            const int i = sp.group.quotient(row), h = g * R + row - i * R;
            T *const dst = static_cast<T *>(a.out) + (((size_t)b * a.n + i) * a.heads + h) * P + 4 * c;
            from_f32(v.x / sum, dst[0]), from_f32(v.y / sum, dst[1]), from_f32(v.z / sum, dst[2]), from_f32(v.w / sum, dst[3]);
            if (a.status && g == 0 && row == 0 && c == 0) a.status[b] = code > -INFINITY ? attn_status((int)-code) : 0;
        }
        return;
    }
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const int tile = row / tile_rows, r = row - tile * tile_rows;
        // maximum of all parts, or what one of them found wrong (a negative sum)
        float top = -INFINITY, code = -INFINITY;
        for (int s = tid; s < plan.y; s += kThreads) {
            const float2 v = sp.sums[slot_of(tile, r, s)];
            top = fmaxf(top, v.x);
            if (v.y < 0.f) code = fmaxf(code, v.y);
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o)), code = fmaxf(code, __shfl_xor(code, o));
        if (lane == 0) red[wave][0] = top, red[wave][1] = code;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, red[w][0]), code = fmaxf(code, red[w][1]);
        const int i = sp.group.quotient(row), h = g * R + row - i * R;
        T *const dst = static_cast<T *>(a.out) + (((size_t)b * a.n + i) * a.heads + h) * P;
        if (a.status && g == 0 && row == 0 && tid == 0) a.status[b] = code > -INFINITY ? attn_status((int)-code) : 0;
        if (code > -INFINITY) {
            for (int e = tid; e < P; e += kThreads) from_f32(0.f, dst[e]);
        } else {
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
            float sum = 0.f;
            if (s0 < over) {
#pragma unroll 4
                for (int s = s0; s < plan.y; s += over) {
                    const size_t slot = slot_of(tile, r, s);
                    const float2 w = sp.sums[slot];
                    const float4 p = *reinterpret_cast<const float4 *>(sp.parts + slot * P + 4 * c);
                    const float f = rescale(w.x, top);
                    sum += w.y * f;
                    v.x = fmaf(p.x, f, v.x), v.y = fmaf(p.y, f, v.y), v.z = fmaf(p.z, f, v.z), v.w = fmaf(p.w, f, v.w);
                }
            }
            acc[tid] = v;
            factor[tid] = sum;
            __syncthreads();
            if (tid < quads) {
                for (int s = 1; s < over; ++s) {
                    const float4 u = acc[s * quads + c];
                    v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
                    sum += factor[s * quads + c];
                }
                from_f32(v.x / sum, dst[4 * c]), from_f32(v.y / sum, dst[4 * c + 1]);
                from_f32(v.z / sum, dst[4 * c + 2]), from_f32(v.w / sum, dst[4 * c + 3]);
            }
        }
        __syncthreads();
    }
}

// Rows of a workgroup, in blocks of 16, and workers: as many rows as there are, up to what the registers hold, unless the
// keys that the table has room for would then leave CUs idle; as many workers as the chip holds workgroups at once.
//
// Which kernel, bf16 heads of 128: from 33 rows on the one that shares tiles (64 sequences of 4000 tokens, 64 rows: 209 us, here in
// two tiles 300; 16 of 2000, 36 rows: 46 and 50; 32 rows: 46, here 40).  Only one short sequence is better off here (60 rows behind
// 500 tokens: 19 and 15 us).  Tiles of 64 rows up to 128, of 256 beyond (16 sequences of 2000 tokens, 128 rows in two tiles 62 us, in
// half of one 70; 192 rows in three 119, in one 69).  Here one tile of 32 rows rather than two of 16: 64 sequences of 4000 tokens
// 170 us, not 276.  That holds although the kernels of 32 rows and heads of more than 64 spill registers (heads of 128 56 of them in
// bf16, 72 in fp32, heads of 80 and 96 214 and 114, of 256 166 and 197; with 16 rows at most 8): 16 sequences of 2000 tokens, 64 rows,
// fp32 heads of 128 117 us, with 16 147; bf16 heads of 80 49 and 68, of 256 116 and 142.  Two shapes go the other way and are not
// told apart: fp32 heads of 256 (64 rows 320 us, with 16 273; 32 rows 182 and 150) and bf16 heads of 192 (32 rows 83 and 78).
struct Shape {
    int blocks, tiles, workers;
    bool shared;                                     // the kernel that shares tiles of keys through LDS
    bool spread;                                     // (AttnSplit)
    Shape(const stree_attn &a, const stree_kv &kv) {
        const int rows = a.nnodes * (a.nheads / kv.nheads_kv);
        const int64_t units = (int64_t)a.batch * kv.nheads_kv, most = units * (((int64_t)kv.max_pages * kv.page + kTileKeys - 1) / kTileKeys);
        shared = kv.io_dtype == STREE_BF16 && (kv.headdim == 64 || kv.headdim == 128) && rows > 32;
        if (shared) {
            blocks = rows <= 128 ? 4 : 16;
            tiles = (rows + 16 * blocks - 1) / (16 * blocks);
            crowd(blocks == 4 ? 2 * kChip : kChip, most);
            return;
        }
        blocks = rows <= 16 ? 1 : 2;
        while (blocks > 1 && most * ((rows + 16 * blocks - 1) / (16 * blocks)) < kChip) blocks /= 2;
        tiles = (rows + 16 * blocks - 1) / (16 * blocks);
        crowd(kChip * (kv.headdim <= 128 ? 2 : 1), most);                            // (kMinWaves)
    }
    // As many workers as `chip` workgroups make; on one XCD each where that leaves out an eighth of them at most (a prompt of 8192
    // tokens, 128 tiles of rows: two workers on two of the eight XCDs took 2436 us, spread out 630).  Workers are whole numbers, so
    // tiles just beyond a half, or the whole, of the chip leave nearly half of it idle: 8256 tokens, 129 tiles, 1140 us; 16448, 257
    // tiles, 4700.
    void crowd(int chip, int64_t most) {
        int w = chip / tiles < 1 ? 1 : chip / tiles;
        spread = w / 8 * 64 < w * 7;
        if (!spread) w &= ~7;
        workers = (int)(w < most ? w : most);
    }
};

AttnSplit split_of(const stree_attn &a, const stree_kv &kv) {
    const int R = a.nheads / kv.nheads_kv, rows = a.nnodes * R;
    const Shape shape(a, kv);
    AttnSplit s(R);
    s.workers = shape.workers;
    s.tiles = shape.tiles;
    s.spread = shape.spread;
    s.rows = rows < 16 * shape.blocks ? rows : 16 * shape.blocks;
    s.batch = a.batch;
    s.plan = nullptr, s.sums = nullptr, s.parts = nullptr;
    return s;
}

// scratch: plan, sums, parts, each on 16 bytes; none where nothing can be cut, with one worker or one tile a unit
size_t lay_out(AttnSplit &s, const stree_attn &a, const stree_kv &kv, void *workspace) {
    if (s.workers == 1 || (int64_t)kv.max_pages * kv.page <= kTileKeys) return 0;
    const size_t units = (size_t)a.batch * kv.nheads_kv, slots = (size_t)2 * s.workers * s.tiles * s.rows;
    const size_t plan = (units * sizeof(int2) + 15) / 16 * 16, sums = (slots * sizeof(float2) + 15) / 16 * 16;
    char *at = static_cast<char *>(workspace);
    s.plan = reinterpret_cast<int2 *>(at);
    s.sums = reinterpret_cast<float2 *>(at + plan);
    s.parts = reinterpret_cast<float *>(at + plan + sums);
    return plan + sums + slots * kv.headdim * sizeof(float);
}

template <typename T, int PP, int MB>
void launch_stream(const AttnArgs &a, const KvView<T> &kv, const AttnSplit &sp, hipStream_t st) {
    const unsigned grid = sp.grid();
    if (kv.dim == PP) hipLaunchKernelGGL((attn_stream_kernel<T, PP, MB, true>), dim3(grid), dim3(kThreads), 0, st, a, kv, sp);
    else hipLaunchKernelGGL((attn_stream_kernel<T, PP, MB, false>), dim3(grid), dim3(kThreads), 0, st, a, kv, sp);
}

template <typename T, int PP>
void launch_rows(const AttnArgs &a, const KvView<T> &kv, const AttnSplit &sp, int blocks, hipStream_t st) {
    if (blocks == 1) launch_stream<T, PP, 1>(a, kv, sp, st);
    else launch_stream<T, PP, 2>(a, kv, sp, st);
}

template <typename T>
hipError_t launch(const AttnArgs &a, const stree_attn &at, const stree_kv &kv, void *workspace, hipStream_t st) {
    AttnSplit sp = split_of(at, kv);
    const bool cut = lay_out(sp, at, kv, workspace) > 0;
    const Shape shape(at, kv);
    const int blocks = shape.blocks, rows = at.nnodes * sp.group.d, units = at.batch * kv.nheads_kv;
    const KvView<T> view(kv);
    hipError_t e;
    if (shape.shared) {
        e = launch_attn_tile(a, kv, sp, 16 * blocks, st);
        if (e != hipSuccess) return e;
    }
    else if (kv.headdim <= 64) launch_rows<T, 64>(a, view, sp, blocks, st);
    else if (kv.headdim <= 128) launch_rows<T, 128>(a, view, sp, blocks, st);
    else launch_rows<T, 256>(a, view, sp, blocks, st);
    e = hipGetLastError();
    if (e != hipSuccess || !cut) return e;
    // a workgroup per row where that is what fills the chip, several rows each where there are many
    const int groups = rows * (int64_t)units <= 4 * kChip ? rows : (4 * kChip + units - 1) / units;
    hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)(groups < rows ? groups : rows), (unsigned)units), dim3(kThreads), 0, st, a, view,
                       sp, 16 * blocks);
    return hipGetLastError();
}

}  // namespace

bool attn_stream_supported(const stree_attn &a, const stree_kv &kv, const void *q, const void *out) {
    const int e = kv.io_dtype == STREE_BF16 ? 8 : 4;
    if (kv.headdim % e || a.q_stride_n % e || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)kv.k | (uintptr_t)kv.v) % 16)) return false;
    // grid dimensions: workgroups (of up to 512 threads), and units in the joining kernel
    const Shape s(a, kv);
    return ((int64_t)s.workers + 8) * s.tiles < (1 << 23) && (int64_t)a.batch * kv.nheads_kv < 65536;
}

size_t attn_stream_workspace(const stree_attn &a, const stree_kv &kv) {
    AttnSplit s = split_of(a, kv);
    return lay_out(s, a, kv, nullptr);
}

hipError_t launch_attn_stream(const stree_attn &at, const stree_kv &kv, const AttnArgs &a, void *workspace, hipStream_t st) {
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(a, at, kv, workspace, st) : launch<float>(a, at, kv, workspace, st);
}

}  // namespace stree
