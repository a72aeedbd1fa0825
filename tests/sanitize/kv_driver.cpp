// Host-side validation of the attention layers' entry points under the address / undefined-behaviour sanitizers.  Built by
// tests/test_kv_sanitizers.py from paper_2505_14969_amd/csrc/api_kv.hip (host pass only) and this file, whose stand-ins for
// the launchers count their calls: calls that the validation turns down must not reach one, whole ones must.
#include <cmath>
#include <cstdio>

#include "../../paper_2505_14969_amd/csrc/launch_kv.hpp"

static int launches = 0;
namespace stree {
hipError_t launch_tree_rope(const stree_attn &a, const stree_kv &, const int32_t *, const int32_t *, const void *, const void *, const void *, const void *, const void *, const double *, void *, int32_t *, hipStream_t) { launches += a.q_stride_n > 0 && a.k_stride_n > 0 && a.v_stride_n > 0; return hipSuccess; }
size_t tree_attn_workspace(const stree_attn &, const stree_kv &) { return 64; }
hipError_t launch_tree_attn(const stree_attn &a, const stree_kv &, const int32_t *, const int32_t *, const void *, void *, int32_t *, void *, hipStream_t) { launches += a.softmax_scale == 0.125f; return hipSuccess; }
hipError_t launch_commit_kv(const stree_attn &, const stree_kv &, const int32_t *, const int32_t *, const int32_t *, int32_t *, int32_t *, hipStream_t) { ++launches; return hipSuccess; }
hipError_t launch_resize_kv(const stree_kv &, const stree_pool &, int, const int32_t *, int32_t *, hipStream_t) { ++launches; return hipErrorInvalidValue; }
hipError_t launch_fork_kv(const stree_kv &, const stree_pool &, int, int, const int32_t *, const int32_t *, int32_t *, int32_t *, hipStream_t) { ++launches; return hipSuccess; }
}  // namespace stree

static int fails = 0;
#define EXPECT(call, want)                                                                                              \
    do {                                                                                                                \
        const long got_ = (long)(call);                                                                                 \
        if (got_ != (long)(want)) { printf("line %d: got %ld, want %ld\n", __LINE__, got_, (long)(want)); ++fails; }    \
    } while (0)

int main() {
    alignas(16) static char all[1 << 17];
    char *const buf = all, *const far = all + (1 << 15);               // rows that start at buf end before far + 32768
    int32_t *ip = reinterpret_cast<int32_t *>(buf), *io = reinterpret_cast<int32_t *>(far);
    double *dp = reinterpret_cast<double *>(buf);
    stree_kv kv = {1, 9, 16, 4, 2, 64, STREE_BF16, 0, buf, buf, ip};
    stree_attn a = {2, 6, 8, 0, 64, 1e-6f, 1.f, 0.f, 0, 0, 0};
    stree_pool pool = {ip, ip, ip, ip};
    const size_t none = (size_t)-1;
    EXPECT(stree_tree_rope(nullptr, &kv, ip, ip, buf, buf, buf, nullptr, nullptr, dp, far, nullptr, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_tree_rope(&a, nullptr, ip, ip, buf, buf, buf, nullptr, nullptr, dp, far, nullptr, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_tree_attn(&a, nullptr, ip, ip, buf, far, nullptr, buf, 64, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_tree_attn(&a, &kv, ip, ip, buf, far, nullptr, nullptr, 64, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_tree_attn(&a, &kv, ip, ip, buf, far, nullptr, buf, 63, nullptr), STREE_ERR_BAD_SHAPE);
    EXPECT(stree_tree_attn(&a, &kv, ip, ip, buf, far, nullptr, buf + 8, 64, nullptr), STREE_ERR_BAD_SHAPE);
    EXPECT(stree_attn_workspace_bytes(&a, nullptr), none);
    stree_attn d = a;
    d.batch = 65535, d.nnodes = 256, d.nheads = 65534;                    // products beyond 64 bits' comfort
    EXPECT(stree_attn_workspace_bytes(&d, &kv), none);
    stree_kv big = kv;
    big.nheads_kv = 65535, big.headdim = 256, big.page = 256;
    EXPECT(stree_commit_kv(&a, &big, ip, ip, ip, io, nullptr, nullptr), STREE_ERR_BAD_SHAPE);
    big = kv, big.max_pages = INT32_MAX;
    EXPECT(stree_resize_kv(&big, &pool, 1, ip, nullptr, nullptr), STREE_ERR_BAD_SHAPE);
    d = a, d.q_stride_n = INT64_MAX;
    EXPECT(stree_tree_attn(&d, &kv, ip, ip, buf, far, nullptr, buf, 64, nullptr), STREE_ERR_BAD_STRIDE);
    d = a, d.v_stride_n = INT64_MIN;
    EXPECT(stree_tree_rope(&d, &kv, ip, ip, buf, buf, buf, nullptr, nullptr, dp, far, nullptr, nullptr), STREE_ERR_BAD_STRIDE);
    EXPECT(stree_fork_kv(&kv, nullptr, 2, 1, ip, ip, ip, ip, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_rope_frequencies(8, 1e4, STREE_ROPE_NONE, 0, 0, 0, 0, nullptr), STREE_ERR_NULL_ARG);
    EXPECT(stree_rope_frequencies(8, NAN, STREE_ROPE_NONE, 0, 0, 0, 0, dp), STREE_ERR_BAD_SHAPE);
    EXPECT(stree_rope_frequencies(8, 1e4, 4, 1, 0, 1, 1, dp), STREE_ERR_BAD_SHAPE);
    EXPECT(stree_rope_frequencies(16, 1e4, STREE_ROPE_RAMP, 8, 1, 4, 8192, dp), STREE_OK);      // 8 numbers in 64 bytes
    EXPECT(launches, 0);
    EXPECT(stree_tree_rope(&a, &kv, ip, ip, buf, buf, buf, nullptr, nullptr, dp, far + 32768, nullptr, nullptr), STREE_OK);
    EXPECT(stree_tree_attn(&a, &kv, nullptr, ip, buf, far + 32768, nullptr, buf, 64, nullptr), STREE_OK);
    EXPECT(stree_commit_kv(&a, &kv, ip, ip, ip, ip, nullptr, nullptr), STREE_OK);
    EXPECT(stree_resize_kv(&kv, &pool, 2, ip, nullptr, nullptr), STREE_ERR_HIP);
    EXPECT(stree_fork_kv(&kv, &pool, 2, 1, ip, ip, ip, ip, nullptr), STREE_OK);
    EXPECT(launches, 5);
    printf("%d mismatches\n", fails);
    return fails != 0;
}
