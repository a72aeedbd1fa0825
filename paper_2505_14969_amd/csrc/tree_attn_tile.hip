// The kernel of stree_tree_attn for many query rows: 64 or 256 rows (node, head) of one key/value head share every tile of
// 64 keys through LDS, products on the bf16 matrix units.
//
// As in the streaming kernel a lane owns a query row in every accumulator (S^T = K Q^T, O^T += V^T P^T), keys stand in S^T in the
// order that makes the probabilities the operand of the second product, and the maximum moves only when a score passes it by
// kSlack.  A wave has 32 rows, and two waves are on a SIMD: 256 rows are eight waves side by side; 64 rows are two, and two more
// take the other half of a tile's keys, with two such workgroups on a CU.  Tiles go from memory straight into LDS, up to three on
// their way; one barrier a tile.  The first product of the next 32 keys is issued with the exponentials of these, which it does
// not wait for.
//
// With 256 rows a tile takes 2048 cycles of a SIMD's matrix unit, about as many of LDS reads and as many of exponentials and sums,
// and two waves a SIMD overlap the three in part only: that bounds it, at some 3800 cycles a tile (2 us a CU at the 1.9 GHz that
// the clock then has).  Around the tiles stand 10 us of the chain to the first one and two ends of a share, so that of the whole
// kernel's cycles the matrix units are busy in 22 %.  The clock falls further where there is more to move, to 1.6 GHz at 64 rows of
// 131000 tokens (537 MB): 2.25 us a tile; where the keys come from L2 1.6.  16 trees of 64 nodes behind 2900 tokens on average
// 89 to 96 us (44.6 Gflop, 190 MB), of which 12.6 join parts; two prompts of 512 behind 1537 69 to 74 us, of which 12; one of 8192
// 615 to 630 us (550 Gflop, 0.88 Pflop/s), with 64 tokens more 1140 (Shape::crowd).  Tried beside this: 64 rows a
// wave, half the LDS reads, one wave a SIMD (138 us where this took 99: accumulators move between two register files), 128 rows and
// two workgroups a CU (108 and 97), the streaming hint (the prompts: 88 and 80, tiles of rows share keys in L2).
#include "attn.hpp"

namespace stree {

namespace {

constexpr float kSlack = 8.f;
constexpr int kKeys = 64;                            // keys of a tile

// Sixteen lanes that follow one another read 16 bytes each of different rows in one cycle if they are different 16 bytes of 256
// (64 banks).  So the 16-byte pieces of a row of K are permuted by the key's place in S^T, and the two halves of a row of 16
// tokens of V change places every eight rows.  (Every four rows, and keys by three bits: 8.4 million cycles of conflicts for 16
// trees of 64 nodes behind 4000 tokens, now none.)
template <int PP>
__device__ __forceinline__ int key_swizzle(int key) {
    const int row = (key & 3) | ((key >> 1) & 4) | ((key << 1) & 8);         // its row of S^T, within 16
    return PP == 128 ? row : row >> 1;                                        // (rows of 128 bytes: two to a line of banks)
}
template <int PP, int NB>
struct TileLds {
    static constexpr int kTile = kKeys * PP;         // elements
    bf16_t t[NB][2][kTile];                          // keys, values
    uint32_t bits[kMaxNodes * kMaxWords];
};

// 64 lanes' 16 bytes from memory to LDS, one lane's after the other's from `to` on (alike in all lanes).
__device__ __forceinline__ void load_to_lds(const bf16_t *from, bf16_t *to) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from, (__attribute__((address_space(3))) void *)to, 16, 0, 0);
}

// RW waves side by side over the rows, TH / 64 / RW over a tile's keys; NB tiles in LDS, NB - 1 of them on their way.
template <int PP, int RW, int TH, int NB>
__global__ __launch_bounds__(TH, 2) void attn_tile_kernel(AttnArgs a, KvView<bf16_t> kv, AttnSplit sp) {
    constexpr int WAVES = TH / 64, ROWS = 32 * RW, KW = WAVES / RW, KB = 2 / KW, NC = PP / 16, NPB = PP / 32;    // key waves; blocks of 32 keys a wave
    constexpr int LOADS = kKeys * PP / 512 / WAVES;                                   // a wave's loads of 1 KB for a tile's keys, and for its values
    static_assert(KW * KB == 2, "64 keys a tile");
    static_assert(sizeof(TreeLds) <= 2 * kKeys * PP * sizeof(bf16_t), "the tree is looked at in a tile's place");
    typedef TileLds<PP, NB> Lds;
    __shared__ Lds lds;
    __shared__ float ml[KW > 1 ? ROWS : 1][2];
    const int tid = threadIdx.x, lane = tid & 63, wave = uniform(tid >> 6), wr = wave % RW, wk = wave / RW;
    const int col = lane & 31, half = lane >> 5;
    const int2 here = sp.place(blockIdx.x);
    const int worker = here.x, group = here.y;
    if (worker >= sp.workers) return;
    const int R = sp.group.d, rows = a.n * R, words = (a.n + 31) / 32;
    bf16_t *const out = static_cast<bf16_t *>(a.out);
    const float scale = fabsf(a.scale);
    Share at = Share::start<TH>(a, kv, sp, worker, reinterpret_cast<int64_t *>(lds.t[0]));
    if (worker >= at.workers) return;
    __syncthreads();                                   // (its numbers lay where the first tile goes)

    const int shift = kv.shift, mask = kv.mask();
    const size_t block = (size_t)PP << shift;
    bf16_t *const scratch = lds.t[NB - 1][0];          // (no tile of a new piece is on its way to the last buffer)
    // where a lane's operands lie
    const int ktok = (col & 3) | ((col >> 1) & 4) | ((col << 1) & 8) | (col & 16);      // S^T row -> key
    // (row r = 4 h + e of a block of 16 holds key 8 h + e, row 8 + 4 h + e key 8 h + 4 + e)
    const int kx = half ^ key_swizzle<PP>(ktok);
    const int kget = ktok * PP + kx * 8;               // (chunk c of 16 columns: ^ 16 c)
    const int vget = col * 16 + (half ^ ((col >> 3) & 1)) * 8;

    int k0 = 0, k1 = 0, whole = 0, end = 0;
    PageWalk<bf16_t> walk;
    bf16x8 q[NC];
    // A tile on its way to a buffer: K by rows of 16-byte pieces, V by runs of 16 tokens, 32 rows of it a load.  What lies where is
    // a matter of which lane fetches what.
    auto fetch = [&](int t, int buf) {
        walk.reach(kv, at.b, t >> shift, end, lane);
        constexpr int KR = PP / 8, VR = PP / 32;       // pieces of a row of K; loads of a run of V
        const int lane = again(tid) & 63;
#pragma unroll
        for (int x = 0; x < LOADS; ++x) {
            const int y = x * WAVES + wave;
            const int r = y * (64 / KR) + lane / KR, piece = (lane % KR) ^ key_swizzle<PP>(r);
            const int tk = t + ((y * (64 / KR)) & ~15), pk = walk.at(min(tk >> shift, end - 1));
            load_to_lds(kv.k + ((size_t)pk * kv.heads + at.g) * block + (size_t)((t + r) & mask) * PP + piece * 8, &lds.t[buf][0][y * 512]);
            const int run = y / VR, p = (y % VR) * 32 + (lane >> 1), vhalf = (lane & 1) ^ ((p >> 3) & 1);
            const int tv = t + 16 * run, pv = walk.at(min(tv >> shift, end - 1));
            load_to_lds(kv.v + ((size_t)pv * kv.heads + at.g) * block + ((size_t)p << shift) + (tv & mask) + vhalf * 8, &lds.t[buf][1][y * 512]);
        }
    };
    auto enter = [&]() {
        const int lane2 = again(lane), col = lane2 & 31, half = lane2 >> 5;
        const int row0 = at.row_tile(kv.heads, group, sp.tiles) * ROWS;
        k0 = k1 = whole = 0;
        if (at.len >= 0 && kv.fits((int64_t)at.len + a.n)) {
            const int last = sp.group.quotient(min(row0 + ROWS, rows) - 1);
            k0 = at.t0 * kTileKeys, whole = min(at.t1 * kTileKeys, at.len + a.n);
            k1 = min(whole, at.len + last + 1);
        }
        if (k0 >= k1) return walk.none();
        end = ((k1 - 1) >> shift) + 1;
        walk.start(kv, at.b, k0 >> shift, end, lane);
        const int r = min(row0 + wr * 32 + col, rows - 1), i = sp.group.quotient(r), h = at.g * R + r - i * R;
        const bf16_t *src = static_cast<const bf16_t *>(a.q) + ((size_t)at.b * a.n + i) * a.q_sn + (size_t)h * PP + half * 8;
#pragma unroll
        for (int c = 0; c < NC; ++c) q[c] = signed_query(*reinterpret_cast<const bf16x8 *>(src + c * 16), a.scale);
#pragma unroll 1
        for (int x = 0; x < NB - 1; ++x)
            if (k0 + x * kKeys < k1) fetch(k0 + x * kKeys, x);
    };
    enter();
    for (;;) {
        const int b = at.b, g = at.g, len = at.len, w1 = k1, unit = b * kv.heads + g, tile = at.row_tile(kv.heads, group, sp.tiles), row0 = tile * ROWS;
        const bool direct = at.whole(), begins = at.t0 == 0;
        if (begins && sp.plan && tile == 0 && tid == 0)
            sp.plan[unit] = make_int2(worker, direct ? 1 : at.shares.worker(at.x + at.tiles - 1) - worker + 1);
        int bad = len >= 0 && !kv.fits((int64_t)len + a.n) ? STREE_SEQ_LENGTH : 0;
        if (whole > len && len >= 0 && whole > 0 && a.parent) bad = index_paths(*reinterpret_cast<TreeLds *>(scratch), lds.bits, a.parent, b, a.n);
        const int col = again(lane) & 31, half = again(lane) >> 5;
        const int node = sp.group.quotient(min(row0 + wr * 32 + col, rows - 1));
        float m = -INFINITY, base = 0.f, l = 0.f;
        floatx16 o[NPB];
#pragma unroll
        for (int p = 0; p < NPB; ++p)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[p][e] = 0.f;
        const int clear = min(w1, len + (a.parent ? 0 : sp.group.quotient(row0) + 1));     // all of these rows see the keys up to here
        int buf = 0;
        floatx16 s;                                    // of the wave's next 32 keys, always a step ahead
        float top = -INFINITY;
        bf16x8 kf[NC];
        const int mine = wk * KB * 32 * PP;            // (this wave's keys of a tile)
        auto load_k = [&](int from, int kb) {
            const int at8 = again(kget) + mine + from * 2 * Lds::kTile + kb * 32 * PP;
#pragma unroll
            for (int c = 0; c < NC; ++c) kf[c] = *reinterpret_cast<const bf16x8 *>(lds.t[0][0] + (at8 ^ (16 * c)));
        };
        auto product = [&]() {
            floatx16 r;
#pragma unroll
            for (int e = 0; e < 16; ++e) r[e] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) r = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], q[c], r, 0, 0, 0);
            return r;
        };
        auto largest = [&](const floatx16 &v) {
            float r = v[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) r = fmaxf(r, v[e]);
            return r;
        };
        // This wave's part of tile t is there; up to `behind` tiles that follow it may be on their way.
        auto arrived = [&](int t, int behind) {
            if (behind >= 2 && t + 2 * kKeys < w1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(4 * LOADS) : "memory");
            else if (behind >= 1 && t + kKeys < w1) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(2 * LOADS) : "memory");
            else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        };
        if (k0 < w1) {
            arrived(k0, NB - 2);
            if (k0 + (NB - 1) * kKeys < w1) fetch(k0 + (NB - 1) * kKeys, NB - 1);
            load_k(0, 0);
            s = product();
            top = largest(s);
        }
        for (int t = k0; t < w1; t += kKeys) {
            const bool tail = t + kKeys > clear;
            const bf16_t *const vt = lds.t[buf][1] + mine;
            uint32_t seen[KB];                         // 16 keys a block and lane: bits 0 - 7 of its first 16, 8 - 15 of its last
            int odd = 0;
            if (__builtin_expect(tail, 0)) {
                // Values behind the last node are no numbers anybody wrote.
                for (int y = tid; y < kKeys * PP / 8; y += TH) {
                    bf16x8 *const at8 = reinterpret_cast<bf16x8 *>(lds.t[buf][1]) + y;
                    const int run = y / (2 * PP), p = y % (2 * PP) >> 1, left = len + a.n - (t + 16 * run + ((y ^ (p >> 3)) & 1) * 8);
                    bf16x8 f = *at8;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        if (e >= left) f[e] = (bf16_t)0.f;
                        odd |= !(fabsf((float)f[e]) < INFINITY);
                    }
                    *at8 = f;
                }
                odd = __syncthreads_or(odd);
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    seen[kb] = 0;
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int t8 = t + (wk * KB + kb) * 32 + y * 16 + half * 8, left = w1 - t8;
                        uint32_t v = seen_nodes<8>(lds.bits, words, a.parent != nullptr, node, t8 - len);
                        v &= left >= 8 ? 0xffu : left > 0 ? (1u << left) - 1u : 0u;
                        seen[kb] |= v << (8 * y);
                    }
                }
                if (__builtin_expect(odd, 0)) {
                    // Infinities and NaN among the values of nodes: zero probabilities would not keep them from the rows that do
                    // not see the node.  They are counted per row, and are zeros for the products below.
#pragma unroll 1
                    for (int y = 0; y < 2 * KB; ++y) {
                        const int kb = y >> 1;
#pragma unroll
                        for (int p = 0; p < NPB; ++p) {
                            const bf16x8 v = *reinterpret_cast<const bf16x8 *>(vt + y * 16 * PP + vget + p * 32 * 16);
                            bf16x8 up, down;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                up[e] = (bf16_t)((float)v[e] < INFINITY ? 0.f : 1.f);              // +inf, NaN
                                down[e] = (bf16_t)((float)v[e] > -INFINITY ? 0.f : 1.f);           // -inf, NaN
                            }
                            const uint32_t bits = (KB > 1 && kb ? seen[KB - 1] : seen[0]) >> (8 * (y & 1));
                            bf16x8 see;
#pragma unroll
                            for (int e = 0; e < 8; ++e) see[e] = (bf16_t)((bits >> e) & 1u ? 1.f : 0.f);
                            floatx16 cu, cd;
#pragma unroll
                            for (int e = 0; e < 16; ++e) cu[e] = cd[e] = 0.f;
                            cu = __builtin_amdgcn_mfma_f32_32x32x16_bf16(up, see, cu, 0, 0, 0);
                            cd = __builtin_amdgcn_mfma_f32_32x32x16_bf16(down, see, cd, 0, 0, 0);
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                if (cu[e] > 0.f) o[p][e] += INFINITY;
                                if (cd[e] > 0.f) o[p][e] -= INFINITY;
                            }
                        }
                    }
                    __syncthreads();
                    for (int x = tid; x < kKeys * PP; x += TH)
                        if (!(fabsf((float)lds.t[buf][1][x]) < INFINITY)) lds.t[buf][1][x] = (bf16_t)0.f;
                    __syncthreads();
                }
            }
            const int after = buf == NB - 1 ? 0 : buf + 1;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) {          // 32 keys
                bf16x8 vf[2][NPB];
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int p = 0; p < NPB; ++p) vf[y][p] = *reinterpret_cast<const bf16x8 *>(vt + (2 * kb + y) * 16 * PP + vget + p * 32 * 16);
                if (kb < KB - 1) {
                    load_k(buf, kb + 1);
                } else if (t + kKeys < w1) {
                    // This wave has this tile's last operands, and its part of the next tile is there (younger loads, those of the
                    // tiles behind it, may be on their way); with the barrier that holds for everybody, and the tile's place is free.
                    arrived(t + kKeys, NB - 2);
                    if (t + NB * kKeys < w1) fetch(t + NB * kKeys, buf);
                    load_k(after, 0);
                }
                if (__builtin_expect(tail, 0)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (!((seen[kb] >> e) & 1u)) s[e] = -INFINITY;
                    top = largest(s);
                }
                top *= scale;
                if (__builtin_expect(__any(top > m + kSlack), 0)) {
                    const float v = fmaxf(m, fmaxf(top, __shfl_xor(top, 32)));
                    const float b2 = v == -INFINITY ? 0.f : v, keep = rescale(m, v);
                    m = v, base = b2;
                    l *= keep;
#pragma unroll
                    for (int p = 0; p < NPB; ++p) o[p] *= keep;
                }
                // the products of the next 32 keys (of none behind the last, of old ones) go along with these keys' exponentials
                const floatx16 next = product();
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    // one rounding of each probability; their sum is the rounded ones'
                    bf16x8 pf;
#pragma unroll
                    for (int e = 0; e < 8; ++e) pf[e] = (bf16_t)__builtin_amdgcn_exp2f(fmaf(s[8 * y + e], scale, -base));
                    l = sum_of(pf, l);
#pragma unroll
                    for (int p = 0; p < NPB; ++p) o[p] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[y][p], pf, o[p], 0, 0, 0);
                }
                s = next;
                top = largest(s);
            }
            buf = after;
        }
        // (pages of the piece that only later rows see)
        int missing = walk.bad;
        for (int j = (k0 < k1 ? end : k0 >> shift) + tid; j < (whole + mask) >> shift; j += TH) missing |= !kv.exists(kv.table[(size_t)b * kv.max_pages + j]);
        if (__syncthreads_or(missing) && bad == 0) bad = STREE_SEQ_PAGE;
        const bool more = at.next(a, kv);
        if (more) enter();                             // the next piece's first tile is on its way

        {
        const int lane2 = again(lane), col = lane2 & 31, half = lane2 >> 5;
        const bool dead = len < 0 || bad != 0;
        const size_t slot = sp.part(worker, begins, tile);
        l += __shfl_xor(l, 32);
        if constexpr (KW > 1) {
            // the second half of the keys is handed to the first's waves, 32 rows at a time: [wave][p][row]
            float *const give = reinterpret_cast<float *>(scratch) + wr * (PP * 32);
            static_assert(RW * PP * 32 * sizeof(float) <= sizeof(lds.t[0]), "room for it");
            const int r = wr * 32 + col;
            if (wk == 1) {
                if (half == 0) ml[r][0] = m, ml[r][1] = l;
#pragma unroll
                for (int p = 0; p < NPB; ++p)
#pragma unroll
                    for (int e = 0; e < 16; ++e) give[(p * 32 + 8 * (e >> 2) + 4 * half + (e & 3)) * 32 + col] = o[p][e];
            }
            __syncthreads();
            if (wk == 0) {
                const float m2 = ml[r][0], hi = fmaxf(m, m2);
                const float f1 = rescale(m, hi);
                const float f2 = rescale(m2, hi);
                m = hi;
                l = l * f1 + ml[r][1] * f2;
#pragma unroll
                for (int p = 0; p < NPB; ++p)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[p][e] = o[p][e] * f1 + give[(p * 32 + 8 * (e >> 2) + 4 * half + (e & 3)) * 32 + col] * f2;
            }
            __syncthreads();
        }
        // The results turned round in LDS, a quarter of the columns at a time: a lane's row becomes runs of 16-byte pieces of rows.
        constexpr int QS = PP / 16;                    // pieces of four columns of a quarter of a row
        float *const turn = reinterpret_cast<float *>(scratch) + wr * (32 * PP / 4);
        static_assert(RW * 8 * PP * sizeof(float) <= sizeof(lds.t[0]), "room for it");
        if (wk == 0) {
            const int r0 = row0 + wr * 32;
            const float by = !direct ? 1.f : dead ? 0.f : 1.f / l;
            if (!direct && half == 0 && r0 + col < rows) sp.sums[slot + wr * 32 + col] = make_float2(m, bad ? -(float)attn_code(bad) : l);
#pragma unroll
            for (int hp = 0; hp < 4; ++hp) {
                constexpr int ES = PP / 8;             // accumulators of a quarter: 16 of a block of 32 columns, or 8
                const floatx16 &v = o[hp * ES / 16];
#pragma unroll
                for (int e = 0; e < ES; e += 4) {
                    const int f = hp * ES % 16 + e, piece = e / 2 + half;
                    *reinterpret_cast<float4 *>(turn + (col * QS + (piece ^ (col & (QS - 1)))) * 4) = make_float4(v[f] * by, v[f + 1] * by, v[f + 2] * by, v[f + 3] * by);
                }
                wave_sync();
#pragma unroll
                for (int x = 0; x < 32 * QS / 64; ++x) {
                    const int y = x * 64 + lane2, r = y / QS, piece = y % QS, row = r0 + r;
                    const float4 v = *reinterpret_cast<const float4 *>(turn + (r * QS + (piece ^ (r & (QS - 1)))) * 4);
                    const int c = hp * (PP / 4) + piece * 4;
                    if (row >= rows) continue;
                    if (direct) {
                        const int i = sp.group.quotient(row), h = g * R + row - i * R;
                        *reinterpret_cast<uint2 *>(out + (((size_t)b * a.n + i) * a.heads + h) * PP + c) = dead ? make_uint2(0u, 0u) : pack_bf16x4(v.x, v.y, v.z, v.w);
                    } else if (!dead) {
                        *reinterpret_cast<float4 *>(sp.parts + (slot + wr * 32 + r) * PP + c) = v;
                    }
                }
                wave_sync();
            }
        }
        }
        if (direct && a.status && g == 0 && tile == 0 && tid == 0) a.status[b] = bad;
        if (!more) break;
        __syncthreads();                               // (LDS is read)
    }
}

template <int PP, int RW, int TH, int NB>
void launch_tile(const AttnArgs &a, const stree_kv &kv, const AttnSplit &sp, hipStream_t st) {
    hipLaunchKernelGGL((attn_tile_kernel<PP, RW, TH, NB>), dim3(sp.grid()), dim3(TH), 0, st, a, KvView<bf16_t>(kv), sp);
}

}  // namespace

hipError_t launch_attn_tile(const AttnArgs &a, const stree_kv &kv, const AttnSplit &sp, int rows, hipStream_t st) {
    if (kv.headdim == 64) rows == 64 ? launch_tile<64, 2, 256, 2>(a, kv, sp, st) : launch_tile<64, 8, 512, 4>(a, kv, sp, st);
    else rows == 64 ? launch_tile<128, 2, 256, 2>(a, kv, sp, st) : launch_tile<128, 8, 512, 4>(a, kv, sp, st);
    return hipGetLastError();
}

}  // namespace stree
