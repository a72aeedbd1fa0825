// stree_tree_rope: per head of q and k an RMS norm and the rotation to the node's position, k and v appended to the paged cache.
//   x^ = x / sqrt(mean x^2 + eps) * w;  pairs (u, w) turn by 2 pi frac(position * turns[j]), frac in 64 bits
// Rows are read once and written once: bound by memory, and for a few nodes by the chain length -> tree -> angles -> rows.
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

// cosine and sine of 2 pi position * turns, times `scale`: far positions lose nothing, the product is reduced in 64 bits
__device__ __forceinline__ float2 rotation(double turns, int position, float scale) {
    double t = turns * (double)position;
    t -= rint(t);
    float s, c;
    sincospif(2.f * (float)t, &s, &c);
    return make_float2(c * scale, s * scale);
}

// One workgroup per node, a wave per head: any head size, any alignment.
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

template <typename T>
hipError_t launch(const RopeArgs &a, const stree_kv &kv, int batch, hipStream_t st) {
    hipLaunchKernelGGL((rope_plain_kernel<T>), dim3((unsigned)(a.n < (1 << 20) ? a.n : 1 << 20), (unsigned)batch), dim3(kThreads), 0, st, a,
                       KvView<T>(kv));
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
