// stree_tree_rope: per head of q and k an RMS norm and the rotation to the node's position, k and v appended to the paged cache.
//   x^ = x / sqrt(mean x^2 + eps) * w;  pairs (u, w) turn by 2 pi frac(position * turns[j]), frac in 64 bits
// Rows are read once and written once: bound by memory where there are many in fp32, two prompts of 2047 tokens with 32 + 8 + 8 heads
// of 128 40 us (201 MB, 5.0 TB/s); in bf16, with twice the values a byte, by the workgroups of q and k and not by memory: four of 2048
// 54 us (201 MB, 3.7 TB/s; without the workgroups of v, which read their rows twice, 51), one of 65536 370 us (4.4 TB/s).  Few nodes are
// bound by the chain length -> tree, pages -> angles -> rows: one token 5.4 us, 16 trees of 64 nodes 12.7 to 14.6 us (25 MB, 6 us at
// the fp32 rate); the angles, which every group of heads works out for itself, are 0.6 of them.
#include "kv.hpp"
#include "launch_kv.hpp"

namespace stree {

namespace {

struct RopeArgs {
    const int32_t *parent, *lengths;
    const void *q, *k, *v, *q_norm, *k_norm;
    const double *turns;
    void *q_out;
    int32_t *status;
    long q_sn, k_sn, v_sn;
    int n, heads, rotary, interleaved;
    float eps, scale;
};

// cosine and sine of 2 pi position * turns, times `scale`: far positions lose nothing, the product is reduced in 64 bits.  What the
// fraction loses in 32 bits, up to 2^-25 half turns, is made up for by the first order: without it the small ones of the two
// would be off by up to 1e-7, however small they are.
__device__ __forceinline__ float2 rotation(double turns, int position, float scale) {
    double t = turns * (double)position;
    t = 2. * (t - rint(t));                            // half turns
    const float x = (float)t, rest = 3.14159265358979324f * (float)(t - (double)x);
    float s, c;
    sincospif(x, &s, &c);
    return make_float2(fmaf(-s, rest, c) * scale, fmaf(c, rest, s) * scale);
}

// One workgroup per node, a wave per head: any head size, any alignment, any pairs.
template <typename T>
__global__ __launch_bounds__(kThreads) void rope_plain_kernel(RopeArgs a, KvView<T> kv) {
    __shared__ TreeLds tree;
    __shared__ float2 turn[128];
    __shared__ float row[kThreads / 64][256];
    const int b = blockIdx.y, P = kv.dim, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int len = a.lengths[b];
    const T *const q = static_cast<const T *>(a.q), *const k = static_cast<const T *>(a.k), *const v = static_cast<const T *>(a.v);
    T *const out = static_cast<T *>(a.q_out);
    int bad = 0;
    if (len >= 0) {
        if (!kv.fits((int64_t)len + a.n)) bad = STREE_SEQ_LENGTH;
        else if (int node = index_nodes(tree, nullptr, a.parent, b, a.n, 0)) bad = node;
        else if (pages_missing(kv, b, len, (int64_t)len + a.n)) bad = STREE_SEQ_PAGE;
    }
    if (a.status && blockIdx.x == 0 && threadIdx.x == 0) a.status[b] = bad;
    const bool dead = len < 0 || bad;
    for (int i = blockIdx.x; i < a.n; i += gridDim.x) {
        const size_t token = (size_t)b * a.n + i;
        if (dead) {
            T zero;
            from_f32(0.f, zero);
            for (int e = threadIdx.x; e < a.heads * P; e += kThreads) out[token * a.heads * P + e] = zero;
            continue;
        }
        const int slot = len + i, position = len + (a.parent ? tree.cnt[i] - 1 : i);
        __syncthreads();
        for (int j = threadIdx.x; j < a.rotary / 2; j += kThreads) turn[j] = rotation(a.turns[j], position, a.scale);
        __syncthreads();
        const int pg = kv.page_of(b, slot);
        for (int h = wave; h < a.heads + 2 * kv.heads; h += kThreads / 64) {
            if (h >= a.heads + kv.heads) {
                const int g = h - a.heads - kv.heads;
                for (int e = lane; e < P; e += 64) kv.value(pg, g, slot)[(size_t)e << kv.shift] = v[token * a.v_sn + (size_t)g * P + e];
                continue;
            }
            const bool key = h >= a.heads;
            const T *src = key ? k + token * a.k_sn + (size_t)(h - a.heads) * P : q + token * a.q_sn + (size_t)h * P;
            T *dst = key ? kv.key(pg, h - a.heads, slot) : out + (token * a.heads + h) * P;
            const T *w = static_cast<const T *>(key ? a.k_norm : a.q_norm);
            float ss = 0.f;
            for (int e = lane; e < P; e += 64) {
                const float x = to_f32(src[e]);
                row[wave][e] = x;
                ss = fmaf(x, x, ss);
            }
            if (w) {
                for (int o = 32; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
                const float r = 1.f / sqrtf(ss / (float)P + a.eps);
                for (int e = lane; e < P; e += 64) row[wave][e] *= r * to_f32(w[e]);
            }
            wave_sync();
            const int half = a.rotary / 2;
            for (int e = lane; e < P; e += 64) {
                float x = row[wave][e];
                if (e < a.rotary) {
                    const bool first = a.interleaved ? !(e & 1) : e < half;
                    const int j = a.interleaved ? e >> 1 : first ? e : e - half;
                    const float y = row[wave][a.interleaved ? e ^ 1 : first ? e + half : e - half];
                    x = first ? x * turn[j].x - y * turn[j].y : y * turn[j].y + x * turn[j].x;
                }
                from_f32(x, dst[e]);
            }
            wave_sync();
        }
    }
}

// Depth of every node of a tree of at most 64 by one wave (lane = node), or first bad node + 1 (alike in all lanes).
__device__ __forceinline__ int wave_depths(const int32_t *__restrict__ parent, int n, int lane, int &depth) {
    int p = lane < n ? parent[lane] : -1;
    const unsigned long long wrong = __ballot(lane < n && (lane == 0 ? p != -1 : (p < 0 || p >= lane)));
    if (wrong) return __ffsll((long long)wrong);
    depth = p >= 0 ? 1 : 0;
    while (__any(p >= 0)) {                            // (at most six times: the way left is halved)
        const int q = p >= 0 ? p : lane, up = wave_read(depth, q), next = wave_read(p, q);
        if (p >= 0) depth += up, p = next;
    }
    return 0;
}

constexpr int kSlots = 16;             // slots of a tile: what a page holds at least, and whole 32 bytes of a row of V

template <typename T>
struct Piece;                          // 16 bytes of a row
template <>
struct Piece<bf16_t> {
    static constexpr int E = 8;
    static __device__ __forceinline__ void widen(const uint4 &v, float (&o)[8]) {
        o[0] = bf16_lo(v.x), o[1] = bf16_hi(v.x), o[2] = bf16_lo(v.y), o[3] = bf16_hi(v.y);
        o[4] = bf16_lo(v.z), o[5] = bf16_hi(v.z), o[6] = bf16_lo(v.w), o[7] = bf16_hi(v.w);
    }
    static __device__ __forceinline__ uint4 round(const float (&o)[8]) {
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (bf16_t)o[e];
        return __builtin_bit_cast(uint4, v);
    }
};
template <>
struct Piece<float> {
    static constexpr int E = 4;
    static __device__ __forceinline__ void widen(const uint4 &v, float (&o)[4]) {
        o[0] = __uint_as_float(v.x), o[1] = __uint_as_float(v.y), o[2] = __uint_as_float(v.z), o[3] = __uint_as_float(v.w);
    }
    static __device__ __forceinline__ uint4 round(const float (&o)[4]) {
        return make_uint4(__float_as_uint(o[0]), __float_as_uint(o[1]), __float_as_uint(o[2]), __float_as_uint(o[3]));
    }
};

// Tiles of 16 slots as they lie in the cache, so that a row of V of 16 tokens is written whole: workgroup (tile, sequence, up
// to HC heads of q, of k or of v).  q and k: TL lanes hold a row, 16 bytes each; a team stays with its node, whose cosines and
// sines it keeps, and all of its rows are requested at once.  Pairs half the rotated columns apart are another lane's 16 bytes.
// v: turned round in LDS, so that 16 bytes of a column of the tile go out at once.
// Every workgroup looks at the page numbers of all nodes' slots before it writes; of a long prompt (LONG) it then takes a tile after
// the other, every gridDim.x-th (node_groups()).  Others leave behind their one tile, which takes fewer registers: 80 and not 97 for
// four bf16 heads of 128, six waves a SIMD and not four (63 trees of 4 nodes 12.0 us and not 14.1).
template <typename T, int TL, int HC, bool HALF, bool LONG>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a, KvView<T> kv, int zq, int zk) {
    constexpr int E = Piece<T>::E, TEAMS = kThreads / TL;
    __shared__ TreeLds tree;
    __shared__ union { float2 turn[kSlots][128]; T v[kSlots][256 + 2]; } lds;
    const int b = blockIdx.y, P = kv.dim, tid = threadIdx.x, lane = tid & 63, z = blockIdx.z;
    const int len = a.lengths[b];
    const bool fits = len >= 0 && kv.fits((int64_t)len + a.n), query = z < zq, value = z >= zq + zk;
    int slot0 = (fits ? len & ~(kSlots - 1) : 0) + (int)blockIdx.x * kSlots, node0 = slot0 - (fits ? len : 0);     // node of slot 0
    if (node0 >= a.n) return;                          // (no first tile does)
    const int stride = (int)gridDim.x * kSlots;        // to this workgroup's next tile
    const int h0 = (query ? z : value ? z - zq - zk : z - zq) * HC, heads = min(HC, (query ? a.heads : kv.heads) - h0);
    const size_t row0 = (size_t)b * a.n;
    const long sn = query ? a.q_sn : value ? a.v_sn : a.k_sn;
    const T *const src = static_cast<const T *>(query ? a.q : value ? a.v : a.k);
    const int c = tid & (TL - 1), pieces = P / E, cc = min(c, pieces - 1), col = cc * E;
    // the first rows are on their way while the tree and the pages are looked at
    uint4 raw[HC];
    auto request = [&](int s) {
        const T *const row = src + (row0 + min(max(node0 + s, 0), a.n - 1)) * sn + col;
#pragma unroll
        for (int h = 0; h < HC; ++h) raw[h] = *reinterpret_cast<const uint4 *>(row + (size_t)(h0 + min(h, heads - 1)) * P);
    };
    request(tid / TL);
    int pg = fits ? kv.page_of(b, slot0) : 0;
    int bad = 0;
    if (len >= 0) {
        if (!fits) {
            bad = STREE_SEQ_LENGTH;
        } else if (a.parent && a.n <= 64) {            // (all waves find the same)
            int depth = 0;
            bad = wave_depths(a.parent + (size_t)b * a.n, a.n, lane, depth);
            tree.cnt[lane] = depth + 1;
        } else {
            bad = index_nodes(tree, nullptr, a.parent, b, a.n, 0);
        }
        if (bad == 0 && pages_missing(kv, b, len, (int64_t)len + a.n)) bad = STREE_SEQ_PAGE;      // (a barrier)
    }
    if (a.status && blockIdx.x == 0 && z == 0 && tid == 0) a.status[b] = bad;
    const bool dead = len < 0 || bad;
    if (dead && !query) return;
    if (value) {
        for (;;) {
            for (int h = 0; h < heads; ++h) {
                for (int s = tid / TL; s < kSlots; s += TEAMS) {
                    const int i = node0 + s;
                    if (i >= 0 && i < a.n && c < pieces) {
                        const uint4 v = *reinterpret_cast<const uint4 *>(src + (row0 + i) * sn + (size_t)(h0 + h) * P + col);
                        const T *const w = reinterpret_cast<const T *>(&v);
#pragma unroll
                        for (int e = 0; e < E; ++e) lds.v[s][col + e] = w[e];
                    }
                }
                __syncthreads();
                T *const dst = kv.value(pg, h0 + h, slot0);
                for (int y = tid; y < P * (kSlots / E); y += kThreads) {
                    const int p = y / (kSlots / E), s = y % (kSlots / E) * E, i = node0 + s;
                    T *const to = dst + ((size_t)p << kv.shift) + s;
                    T w[E];
#pragma unroll
                    for (int e = 0; e < E; ++e) w[e] = lds.v[s + e][p];
                    if (i >= 0 && i + E <= a.n) {
                        uint4 v;
                        __builtin_memcpy(&v, w, sizeof(v));
                        *reinterpret_cast<uint4 *>(to) = v;
                    } else {
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (i + e >= 0 && i + e < a.n) to[e] = w[e];
                    }
                }
                __syncthreads();
            }
            if (!LONG || a.n - node0 <= stride) return;
            slot0 += stride, node0 += stride;
            pg = kv.page_of(b, slot0);
        }
    }
    T *const out = static_cast<T *>(a.q_out);
    if (dead) {
        for (;; node0 += stride) {
            for (int s = tid / TL; s < kSlots; s += TEAMS)
                if (node0 + s >= 0 && node0 + s < a.n && c < pieces)
                    for (int h = 0; h < heads; ++h)
                        *reinterpret_cast<uint4 *>(out + ((row0 + node0 + s) * a.heads + h0 + h) * P + c * E) = make_uint4(0u, 0u, 0u, 0u);
            if (!LONG || a.n - node0 <= stride) return;
        }
    }
    const int half = a.rotary / 2;
    auto turn_nodes = [&]() {
        for (int y = tid; y < kSlots * half; y += kThreads) {
            const int s = y / half, j = y - s * half, i = node0 + s;
            if (i >= 0 && i < a.n) {
                const int d = a.parent ? tree.cnt[i] - 1 : i;
                lds.turn[s][j] = rotation(a.turns[j], len + d, a.scale);
            }
        }
        __syncthreads();
    };
    turn_nodes();
    // of this lane's columns: the weights, and where its pairs' other halves are
    const bool norm = query ? a.q_norm != nullptr : a.k_norm != nullptr;
    const T *const w = static_cast<const T *>(query ? a.q_norm : a.k_norm);
    const int team = lane & ~(TL - 1);
    const bool second = HALF && col >= half && col < a.rotary, turns = col < a.rotary;
    const int other = !HALF || !turns ? cc : second ? cc - half / E : cc + half / E;
    float wo[E], wp[E];
#pragma unroll
    for (int e = 0; e < E; ++e) wo[e] = wp[e] = 1.f;
    if (norm) {
        Piece<T>::widen(*reinterpret_cast<const uint4 *>(w + col), wo);
        Piece<T>::widen(*reinterpret_cast<const uint4 *>(w + other * E), wp);
    }
    for (;;) {
        for (int s0 = 0; s0 < kSlots; s0 += TEAMS) {
            const int s = s0 + tid / TL, i = node0 + s;
            const bool there = s < kSlots && i >= 0 && i < a.n;
            // y = r (A x + B x'), x' the pair's other half: weights, cosine and sine (its sign that of the place) of each column
            float A[E], B[E];
#pragma unroll
            for (int e = 0; e < E; ++e) {
                A[e] = wo[e], B[e] = 0.f;
                const int x = col + e;
                if (x < a.rotary) {
                    const float2 t = lds.turn[min(s, kSlots - 1)][HALF ? (second ? x - half : x) : x >> 1];
                    A[e] = wo[e] * t.x;
                    B[e] = (HALF ? wp[e] : wo[e ^ 1]) * ((HALF ? second : (e & 1)) ? t.y : -t.y);
                }
            }
#pragma unroll
            for (int h = 0; h < HC; ++h) {
                if (h >= heads) break;
                float x[E], y[E], r = 1.f;
                Piece<T>::widen(raw[h], x);
                if (norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int e = 0; e < E; ++e) ss = fmaf(x[e], x[e], ss);
                    if (c >= pieces) ss = 0.f;
#pragma unroll
                    for (int o = TL / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
                    r = 1.f / sqrtf(ss / (float)P + a.eps);
                }
                if (HALF) {
                    uint4 q;
                    q.x = wave_read(raw[h].x, team + other), q.y = wave_read(raw[h].y, team + other);
                    q.z = wave_read(raw[h].z, team + other), q.w = wave_read(raw[h].w, team + other);
                    Piece<T>::widen(q, y);
                }
                float out8[E];
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float turned = fmaf(HALF ? y[e] : x[e ^ 1], B[e], x[e] * A[e]);
                    out8[e] = r * (col + e < a.rotary ? turned : x[e] * A[e]);
                }
                if (there && c < pieces)
                    *reinterpret_cast<uint4 *>((query ? out + ((row0 + i) * a.heads + h0 + h) * P : kv.key(pg, h0 + h, slot0 + s)) + col) = Piece<T>::round(out8);
            }
            if (s0 + TEAMS < kSlots) request(s + TEAMS);
        }
        if (!LONG || a.n - node0 <= stride) return;
        slot0 += stride, node0 += stride;
        pg = kv.page_of(b, slot0);
        request(tid / TL);
        __syncthreads();                               // (the angles are read)
        turn_nodes();
    }
}

// Workgroups over the nodes of a sequence, which take `steps` steps, next to `others` for other heads and sequences: one a step, unless
// there are more page numbers, all of which every workgroup looks at, than a workgroup has threads.  Then as many in all as the chip
// holds at once, so that the time grows with a prompt and not with its square (131072 tokens of 8 + 2 + 2 heads of 128 205 us,
// with a workgroup a tile 297; a million of one head of 16 0.41 ms and 4.6).
constexpr int kLong = 16 * kThreads;   // nodes, in pages of 16
inline unsigned node_groups(int n, int64_t steps, int64_t others) {
    if (n <= kLong) return (unsigned)steps;
    const int64_t most = others < 2048 ? 2048 / others : 1;
    return (unsigned)(steps < most ? steps : most);
}

template <typename T, int TL, int HC>
void launch_tuned(const RopeArgs &a, const stree_kv &kv, int batch, hipStream_t st) {
    const int zq = (a.heads + HC - 1) / HC, zk = (kv.nheads_kv + HC - 1) / HC;
    const int tiles = (a.n + 2 * kSlots - 2) / kSlots;
    dim3 grid((unsigned)tiles, (unsigned)batch, (unsigned)(zq + 2 * zk));
    const KvView<T> view(kv);
    if constexpr (HC > 2) {                            // (two heads a workgroup are for few nodes)
        if (a.n > kLong) {
            grid.x = node_groups(a.n, tiles, (int64_t)batch * grid.z);
            if (a.interleaved) hipLaunchKernelGGL((rope_kernel<T, TL, HC, false, true>), grid, dim3(kThreads), 0, st, a, view, zq, zk);
            else hipLaunchKernelGGL((rope_kernel<T, TL, HC, true, true>), grid, dim3(kThreads), 0, st, a, view, zq, zk);
            return;
        }
    }
    if (a.interleaved) hipLaunchKernelGGL((rope_kernel<T, TL, HC, false, false>), grid, dim3(kThreads), 0, st, a, view, zq, zk);
    else hipLaunchKernelGGL((rope_kernel<T, TL, HC, true, false>), grid, dim3(kThreads), 0, st, a, view, zq, zk);
}

template <typename T>
hipError_t launch(const RopeArgs &a, const stree_kv &kv, int batch, hipStream_t st) {
    constexpr int E = Piece<T>::E;
    const int pieces = kv.headdim / E;
    const bool whole = kv.headdim % E == 0 && a.q_sn % E == 0 && a.k_sn % E == 0 && a.v_sn % E == 0 && (a.interleaved || a.rotary / 2 % E == 0) &&
                       (((uintptr_t)a.q | (uintptr_t)a.k | (uintptr_t)a.v | (uintptr_t)a.q_out | (uintptr_t)a.q_norm | (uintptr_t)a.k_norm |
                         (uintptr_t)kv.k | (uintptr_t)kv.v) % 16) == 0 && a.heads <= 65535 / 2 && kv.nheads_kv <= 65535 / 4;
    if (!whole) {
        hipLaunchKernelGGL((rope_plain_kernel<T>), dim3(node_groups(a.n, a.n, batch), (unsigned)batch), dim3(kThreads), 0, st, a, KvView<T>(kv));
        return hipGetLastError();
    }
    // Heads of a workgroup: two where there are few workgroups, so that a step of a few nodes is over sooner; eight bf16 heads,
    // which share their node's angles, where there are many (four prompts of 2048 tokens 55 us, with four heads 58); else four
    // (16 trees of 64 nodes 13.8 us, with eight 14.4; two fp32 prompts of 2047 tokens 39 and 43 us).
    const int64_t groups = (int64_t)batch * ((a.n + kSlots - 1) / kSlots) * ((a.heads + 2 * kv.nheads_kv + 7) / 8);
    constexpr int kMany = E == 8 ? 8 : 4;
#define STREE_ROPE(TL)                                                        \
    (groups < 128 ? launch_tuned<T, TL, 2>(a, kv, batch, st)                  \
                  : groups < 2048 ? launch_tuned<T, TL, 4>(a, kv, batch, st) : launch_tuned<T, TL, kMany>(a, kv, batch, st))
    if (pieces <= 8) STREE_ROPE(8);
    else if (pieces <= 16) STREE_ROPE(16);
    else if (pieces <= 32) STREE_ROPE(32);
    else STREE_ROPE(64);
#undef STREE_ROPE
    return hipGetLastError();
}

}  // namespace

hipError_t launch_tree_rope(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *lengths, const void *q,
                            const void *k, const void *v, const void *q_norm, const void *k_norm, const double *turns,
                            void *q_out, int32_t *status, hipStream_t st) {
    const RopeArgs r = {parent, lengths, q, k, v, q_norm, k_norm, turns, q_out, status, (long)a.q_stride_n, (long)a.k_stride_n,
                        (long)a.v_stride_n, a.nnodes, a.nheads, a.rotary_dim, a.flags & STREE_ROPE_INTERLEAVED, a.eps, a.rope_scale};
    return kv.io_dtype == STREE_BF16 ? launch<bf16_t>(r, kv, a.batch, st) : launch<float>(r, kv, a.batch, st);
}

}  // namespace stree
