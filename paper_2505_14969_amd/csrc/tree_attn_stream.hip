// The tuned kernel of stree_tree_attn: the cache streamed once from memory straight into operand registers.
//
// A workgroup takes 16, 32 or 64 query rows (node, head) of one key/value head and one piece of the sequence's keys; each of
// its four waves walks a quarter of the piece by itself, STEP keys at a time.  Products are formed transposed, so that in
// every accumulator a lane owns one query row (column lane % 16):
//   S^T = K Q^T,   P = 2^(S - m),   O^T += V^T P^T
// Which key stands in which row of S^T is free, so keys are read in the order that makes a lane's probabilities the very
// operand of the second product; V lies transposed in the cache, so its operand too is 16 consecutive bytes.  No LDS, no
// barrier and no shuffle in the loop: the maximum is moved only when a score passes it by kSlack (2^kSlack is harmless in
// fp32), which a vote finds out.  Waves are joined through LDS at the end, pieces by a second kernel.
//
// Bound by memory: 16 rows take 256 cycles of the matrix unit per 32 keys where the chip's memory needs 5000 to bring them.
#include "attn.hpp"

namespace stree {

namespace {

constexpr float kSlack = 8.f;
constexpr int kWaves = kThreads / 64;

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

// Numbers of the pages that a wave walks over, 64 at a time in its lanes and the next 64 on their way.
template <typename T>
struct PageWalk {
    int cur, next, first;
    bool bad;
    __device__ __forceinline__ int window(const KvView<T> &kv, int b, int j0, int end, int lane) {
        const int j = j0 + lane;
        int pg = 0;
        if (j < end) {
            pg = kv.table[(size_t)b * kv.max_pages + j];
            if (!kv.exists(pg)) bad = true, pg = 0;
        }
        return pg;
    }
    __device__ __forceinline__ void start(const KvView<T> &kv, int b, int j0, int end, int lane) {
        bad = false;
        first = j0;
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

template <typename T, int PP, int MB>
struct StreamShape {
    static constexpr int kRows = 16 * MB;
    static constexpr int kSlice = PP * kRows <= 2048 ? PP : 2048 / kRows;        // columns joined at a time: 32 KB of LDS
    static constexpr int kLd = kSlice + 4;
    static constexpr int kMinWaves = PP * MB <= 128 ? 3 : PP * MB <= 256 ? 2 : 1;
};

template <typename T, int PP, int MB, bool WHOLE>
__global__ __launch_bounds__(kThreads, (StreamShape<T, PP, MB>::kMinWaves)) void attn_stream_kernel(AttnArgs a, KvView<T> kv, AttnSplit sp) {
    typedef Mma<T> M;
    typedef typename M::Frag Frag;
    typedef StreamShape<T, PP, MB> Shape;
    constexpr int E = M::E, KB = M::KB, STEP = 16 * KB, NK = PP / (4 * E), NP = PP / 16, ROWS = Shape::kRows, SL = Shape::kSlice, LD = Shape::kLd;
    struct Index { TreeLds tree; uint32_t bits[kMaxNodes * kMaxWords]; };
    __shared__ union { Index index; float o[kWaves][ROWS][LD]; } lds;
    __shared__ float ml[kWaves][ROWS][2];
    // The workgroups of one piece's row tiles follow one another on one XCD, whose L2 they share the piece through.
    const int tile = (int)(blockIdx.x >> 3) % sp.tiles, unit = ((int)(blockIdx.x >> 3) / sp.tiles) * 8 + (int)(blockIdx.x & 7);
    if (unit >= sp.units) return;
    const int piece = unit % sp.pieces, g = unit / sp.pieces % kv.heads, b = unit / sp.pieces / kv.heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4, P = kv.dim;
    const int R = sp.group.d, rows = a.n * R, row0 = tile * ROWS;
    const int len = a.lengths[b];
    T *const out = static_cast<T *>(a.out);
    // pieces of this sequence; what this workgroup's rows see of its piece
    int bad = 0, count = 1;
    int k0 = 0, k1 = 0, whole = 0;
    if (len >= 0) {
        if (!kv.fits((int64_t)len + a.n)) {
            bad = STREE_SEQ_LENGTH;
        } else {
            const int keys = len + a.n, each = sp.piece_keys(keys);
            count = (keys + each - 1) / each;
            if (piece < count) {
                const int last = sp.group.quotient(min(row0 + ROWS, rows) - 1);
                k0 = piece * each, whole = min(k0 + each, keys);
                k1 = min(whole, len + last + 1);
                if (whole > len && a.parent) bad = index_nodes(lds.index.tree, lds.index.bits, a.parent, b, a.n, (a.n + 31) / 32);
            }
        }
    }
    if (piece >= count) return;

    float m[MB], base[MB], l[MB];
    floatx4 o[MB][NP];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
        m[mb] = -INFINITY, base[mb] = 0.f, l[mb] = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) o[mb][p] = floatx4{0.f, 0.f, 0.f, 0.f};
    }
    const int part = ((k1 - k0 + kWaves - 1) / kWaves + STEP - 1) / STEP * STEP;
    const int w0 = k0 + wave * part, w1 = min(w0 + part, k1);
    bool missing = false;
    if (bad == 0 && w0 < w1) {
        const int shift = kv.shift, mask = kv.mask(), end = ((w1 - 1) >> shift) + 1;
        PageWalk<T> walk;
        walk.start(kv, b, w0 >> shift, end, lane);
        // queries: row `col` of each block, 16 bytes at column (4 c + grp) E; zeros behind the head and the last row
        Frag q[MB][NK];
        int node[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int r = row0 + mb * 16 + col, rr = min(r, rows - 1);
            const int i = sp.group.quotient(rr), h = g * R + rr - i * R;
            node[mb] = i;
            const T *src = static_cast<const T *>(a.q) + ((size_t)b * a.n + i) * a.q_sn + (size_t)h * P;
#pragma unroll
            for (int c = 0; c < NK; ++c) {
                const int x = (4 * c + grp) * E;
                const bool there = r < rows && x < P;
                const uint4 v = *reinterpret_cast<const uint4 *>(src + (there ? x : 0));
                q[mb][c] = __builtin_bit_cast(Frag, there ? v : make_uint4(0u, 0u, 0u, 0u));
            }
        }
        // Places within a page: keys in the order that gives lane group `grp` the tokens E grp .. E grp + E - 1 of the step.
        const int ktok = E * (col >> 2) + (col & 3), vtok = E * grp, vrow = WHOLE || col < P ? col : 0;
        const size_t block = (size_t)P << shift;
        const T *kp, *vp;                              // this lane's key row and first value of the step
        auto place = [&](int t) {
            walk.reach(kv, b, t >> shift, end, lane);
            const int pa = walk.at(t >> shift);
            int pk = pa, pv = pa;
            if (STEP > 16 && shift == 4) {             // a step of two pages
                const int pb = (t >> 4) + 1 < end ? walk.at((t >> 4) + 1) : pa;
                pk = ktok < 16 ? pa : pb, pv = vtok < 16 ? pa : pb;
            }
            kp = kv.k + ((size_t)pk * kv.heads + g) * block + (size_t)((t + ktok) & mask) * P + grp * E;
            vp = kv.v + ((size_t)pv * kv.heads + g) * block + ((size_t)vrow << shift) + ((t + vtok) & mask);
        };
        Frag kf[KB][NK], vf[NP];
        auto load_k = [&]() {
#pragma unroll
            for (int x = 0; x < KB; ++x)
#pragma unroll
                for (int c = 0; c < NK; ++c) kf[x][c] = __builtin_bit_cast(Frag, load_stream16(kp + 4 * x * P + (WHOLE || (4 * c + grp) * E < P ? 4 * c * E : -grp * E)));
        };
        auto load_v = [&]() {
#pragma unroll
            for (int p = 0; p < NP; ++p) vf[p] = __builtin_bit_cast(Frag, load_stream16(vp + (WHOLE || 16 * p + col < P ? (size_t)(16 * p) << shift : (size_t)0)));
        };
        place(w0);
        load_k();
        load_v();
        for (int t = w0; t < w1; t += STEP) {
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
            const bool more = t + STEP < w1;
            if (more) {
                place(t + STEP);
                load_k();
            }
            const bool tail = t + STEP > len || t + STEP > w1;
            uint32_t seen[MB];
            float p[MB][E], top[MB];
            bool above = false;
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                top[mb] = -INFINITY;
                if (tail) {
                    seen[mb] = seen_nodes<E>(lds.index.bits, (a.n + 31) / 32, a.parent != nullptr, node[mb], t + vtok - len);
                    const int left = w1 - t - vtok;            // (keys behind the wave's last)
                    seen[mb] &= left >= E ? ~0u : left > 0 ? (1u << left) - 1u : 0u;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float v = s[mb][e >> 2][e & 3] * a.scale;
                    if (tail && !((seen[mb] >> e) & 1u)) v = -INFINITY;
                    p[mb][e] = v;
                    top[mb] = fmaxf(top[mb], v);
                }
                above |= top[mb] > m[mb] + kSlack;
            }
            if (__builtin_expect(__any(above), 0)) {
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) {
                    float v = fmaxf(top[mb], __shfl_xor(top[mb], 16));
                    v = fmaxf(m[mb], fmaxf(v, __shfl_xor(v, 32)));
                    const float b2 = v == -INFINITY ? 0.f : v, keep = m[mb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[mb] - b2);
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
                for (int e = 0; e < E; ++e) p[mb][e] = __builtin_amdgcn_exp2f(p[mb][e] - base[mb]);
                const Frag pf = M::round(p[mb]);       // bf16: one rounding of each probability, and their sum is the rounded ones'
#pragma unroll
                for (int e = 0; e < E; ++e) l[mb] += (float)pf[e];
#pragma unroll
                for (int x = 0; x < NP; ++x) o[mb][x] = M::pv(vf[x], pf, o[mb][x]);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (more) load_v();
        }
        missing = walk.bad;
    }
    // (pages of the piece that only later rows see)
    if (bad == 0)
        for (int j = (k1 >> kv.shift) + (int)threadIdx.x; j < (whole + kv.mask()) >> kv.shift; j += kThreads)
            missing |= !kv.exists(kv.table[(size_t)b * kv.max_pages + j]);
    if (__syncthreads_or(missing) && bad == 0) bad = STREE_SEQ_PAGE;

    // join the waves
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
        // (rows without a finite score: their sums stay what they are)
        keep[mb] = m[mb] == top ? 1.f : m[mb] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[mb] - top);
    }
    const int mine = min(ROWS, rows - row0);
    const bool dead = len < 0 || bad != 0, direct = count == 1;
    const size_t slot = ((size_t)unit * sp.tiles + tile) * sp.rows;
    for (int c0 = 0; c0 < PP; c0 += SL) {
        if (c0) __syncthreads();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int x = 0; x < NP; ++x)
                if (16 * x >= c0 && 16 * x < c0 + SL)
                    *reinterpret_cast<floatx4 *>(&lds.o[wave][mb * 16 + col][16 * x - c0 + 4 * grp]) = o[mb][x] * keep[mb];
        __syncthreads();
        for (int x = threadIdx.x; x < mine * (SL / 4); x += kThreads) {
            const int r = x / (SL / 4), c = c0 + x % (SL / 4) * 4;
            if (c >= P) continue;
            floatx4 v = {0.f, 0.f, 0.f, 0.f};
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[w][r][0]);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float mw = ml[w][r][0], f = mw == top ? 1.f : mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - top);
                sum += ml[w][r][1] * f;
                v += *reinterpret_cast<const floatx4 *>(&lds.o[w][r][c - c0]);
            }
            if (direct) {
                const int i = sp.group.quotient(row0 + r), h = g * R + row0 + r - i * R;
                T *dst = out + (((size_t)b * a.n + i) * a.heads + h) * P + c;
#pragma unroll
                for (int e = 0; e < 4; ++e) from_f32(dead ? 0.f : v[e] / sum, dst[e]);
            } else {
                if (!dead) *reinterpret_cast<floatx4 *>(sp.parts + (slot + r) * P + c) = v;
                if (c == 0) sp.sums[slot + r] = make_float2(top, bad ? -(float)attn_code(bad) : sum);
            }
        }
    }
    if (direct && a.status && g == 0 && tile == 0 && threadIdx.x == 0) a.status[b] = bad;
}

// Joins the pieces of a row: a workgroup per row, lanes over columns and pieces.
template <typename T>
__global__ __launch_bounds__(kThreads) void attn_join_kernel(AttnArgs a, KvView<T> kv, AttnSplit sp, int tile_rows) {
    __shared__ float4 acc[kThreads];
    __shared__ float2 ms[kThreads];
    const int g = blockIdx.y % kv.heads, b = blockIdx.y / kv.heads, P = kv.dim, R = sp.group.d, tid = threadIdx.x;
    const int len = a.lengths[b];
    if (len < 0 || !kv.fits((int64_t)len + a.n)) return;
    const int keys = len + a.n, each = sp.piece_keys(keys), count = (keys + each - 1) / each;
    if (count == 1) return;
    const int row = blockIdx.x, tile = row / tile_rows, r = row - tile * tile_rows;
    const size_t unit0 = ((size_t)b * kv.heads + g) * sp.pieces;
    auto slot = [&](int s) { return ((unit0 + s) * sp.tiles + tile) * sp.rows + r; };
    // maximum and sum of all pieces, or what one of them found wrong (a negative sum)
    float top = -INFINITY;
    int code = INT32_MAX;
    for (int s = tid; s < count; s += kThreads) {
        const float2 v = sp.sums[slot(s)];
        top = fmaxf(top, v.x);
        if (v.y < 0.f) code = min(code, (int)-v.y);
    }
    ms[tid] = make_float2(top, __int_as_float(code));
    __syncthreads();
    for (int o = kThreads / 2; o > 0; o >>= 1) {
        if (tid < o) {
            const float2 u = ms[tid], v = ms[tid + o];
            ms[tid] = make_float2(fmaxf(u.x, v.x), __int_as_float(min(__float_as_int(u.y), __float_as_int(v.y))));
        }
        __syncthreads();
    }
    top = ms[0].x, code = __float_as_int(ms[0].y);
    const int i = sp.group.quotient(row), h = g * R + row - i * R;
    T *const dst = static_cast<T *>(a.out) + (((size_t)b * a.n + i) * a.heads + h) * P;
    if (a.status && g == 0 && row == 0 && tid == 0) a.status[b] = code == INT32_MAX ? 0 : attn_status(code);
    if (code != INT32_MAX) {
        for (int c = tid; c < P; c += kThreads) from_f32(0.f, dst[c]);
        return;
    }
    // lanes: `quads` of four columns, the rest over pieces
    const int quads = P / 4, over = kThreads / quads, c = tid % quads, s0 = tid / quads;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
    float sum = 0.f;
    if (s0 < over)
        for (int s = s0; s < count; s += over) {
            const float2 w = sp.sums[slot(s)];
            if (w.x == -INFINITY && w.y == 0.f) continue;          // (nothing seen: its rows were not written)
            const float f = w.x == top ? 1.f : w.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(w.x - top);
            const float4 p = *reinterpret_cast<const float4 *>(sp.parts + slot(s) * P + 4 * c);
            sum += w.y * f;
            v.x = fmaf(p.x, f, v.x), v.y = fmaf(p.y, f, v.y), v.z = fmaf(p.z, f, v.z), v.w = fmaf(p.w, f, v.w);
        }
    __syncthreads();
    acc[tid] = v;
    ms[tid].x = sum;
    __syncthreads();
    if (tid < quads) {
        for (int s = 1; s < over; ++s) {
            const float4 u = acc[s * quads + c];
            v.x += u.x, v.y += u.y, v.z += u.z, v.w += u.w;
            sum += ms[s * quads + c].x;
        }
        from_f32(v.x / sum, dst[4 * c]), from_f32(v.y / sum, dst[4 * c + 1]);
        from_f32(v.z / sum, dst[4 * c + 2]), from_f32(v.w / sum, dst[4 * c + 3]);
    }
}

// row blocks of a workgroup: as many of 16 rows as there are, up to what the registers hold
int blocks_of(int rows, int headdim) {
    return rows <= 16 ? 1 : rows <= 32 || headdim > 128 ? 2 : 4;
}

AttnSplit split_of(const stree_attn &a, const stree_kv &kv) {
    const int R = a.nheads / kv.nheads_kv, rows = a.nnodes * R, tile = 16 * blocks_of(rows, kv.headdim);
    AttnSplit s(R);
    s.tiles = (rows + tile - 1) / tile;
    s.rows = rows < tile ? rows : tile;
    const int64_t heads = (int64_t)a.batch * kv.nheads_kv, most = ((int64_t)kv.max_pages * kv.page + kPieceKeys - 1) / kPieceKeys;
    int64_t want = (kWorkgroups + heads * s.tiles - 1) / (heads * s.tiles);
    if (want > most) want = most;
    s.pieces = (int)want;
    s.units = 0;
    return s;
}

template <typename T, int PP, int MB>
void launch_stream(const AttnArgs &a, const KvView<T> &kv, const AttnSplit &sp, hipStream_t st) {
    const unsigned grid = (unsigned)((sp.units + 7) / 8 * 8) * (unsigned)sp.tiles;
    if (kv.dim == PP) hipLaunchKernelGGL((attn_stream_kernel<T, PP, MB, true>), dim3(grid), dim3(kThreads), 0, st, a, kv, sp);
    else hipLaunchKernelGGL((attn_stream_kernel<T, PP, MB, false>), dim3(grid), dim3(kThreads), 0, st, a, kv, sp);
}

template <typename T, int PP>
void launch_rows(const AttnArgs &a, const KvView<T> &kv, const AttnSplit &sp, int blocks, hipStream_t st) {
    if (blocks == 1) launch_stream<T, PP, 1>(a, kv, sp, st);
    else if (blocks == 2 || PP > 128) launch_stream<T, PP, 2>(a, kv, sp, st);
    else launch_stream<T, PP, (PP > 128 ? 2 : 4)>(a, kv, sp, st);
}

template <typename T>
hipError_t launch(const AttnArgs &a, const stree_attn &at, const stree_kv &kv, void *workspace, hipStream_t st) {
    AttnSplit sp = split_of(at, kv);
    const int R = at.nheads / kv.nheads_kv, blocks = blocks_of(at.nnodes * R, kv.headdim);
    sp.units = at.batch * kv.nheads_kv * sp.pieces;
    const size_t slots = (size_t)sp.units * sp.tiles * sp.rows;
    sp.parts = static_cast<float *>(workspace);
    sp.sums = reinterpret_cast<float2 *>(sp.parts + slots * kv.headdim);
    const KvView<T> view(kv);
    if (kv.headdim <= 64) launch_rows<T, 64>(a, view, sp, blocks, st);
    else if (kv.headdim <= 128) launch_rows<T, 128>(a, view, sp, blocks, st);
    else launch_rows<T, 256>(a, view, sp, blocks, st);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || sp.pieces == 1) return e;
    hipLaunchKernelGGL((attn_join_kernel<T>), dim3((unsigned)(at.nnodes * R), (unsigned)(at.batch * kv.nheads_kv)), dim3(kThreads), 0, st, a,
                       view, sp, 16 * blocks);
    return hipGetLastError();
}

}  // namespace

bool attn_stream_supported(const stree_attn &a, const stree_kv &kv, const void *q, const void *out) {
    const int e = kv.io_dtype == STREE_BF16 ? 8 : 4;
    if (kv.headdim % e || a.q_stride_n % e || (((uintptr_t)q | (uintptr_t)out | (uintptr_t)kv.k | (uintptr_t)kv.v) % 16)) return false;
    // grid dimensions: workgroups and, in the joining kernel, rows and heads
    const AttnSplit s = split_of(a, kv);
    const int64_t heads = (int64_t)a.batch * kv.nheads_kv, rows = (int64_t)a.nnodes * (a.nheads / kv.nheads_kv);
    return (heads * s.pieces + 8) * s.tiles < (1 << 24) && (s.pieces == 1 || (heads < 65536 && rows < (1 << 24)));
}

size_t attn_stream_workspace(const stree_attn &a, const stree_kv &kv) {
    const AttnSplit s = split_of(a, kv);
    if (s.pieces == 1) return 0;
    const size_t slots = (size_t)a.batch * kv.nheads_kv * s.pieces * s.tiles * s.rows;
    return slots * (kv.headdim * sizeof(float) + sizeof(float2));
}

hipError_t launch_attn_stream(const stree_attn &at, const stree_kv &kv, const AttnArgs &a, void *workspace, hipStream_t st) {
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(a, at, kv, workspace, st) : launch<float>(a, at, kv, workspace, st);
}

}  // namespace stree
