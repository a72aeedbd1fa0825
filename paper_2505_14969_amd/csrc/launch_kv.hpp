// Host-side launchers of the attention layers' kernels.  Arguments are already validated by the C-ABI layer (api_kv.hip);
// strides are resolved (never 0).
#pragma once
#include <hip/hip_runtime.h>

#include "../../include/stree.h"

namespace stree {

hipError_t launch_tree_rope(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *lengths, const void *q,
                            const void *k, const void *v, const void *q_norm, const void *k_norm, const double *turns,
                            void *q_out, int32_t *status, hipStream_t st);

size_t tree_attn_workspace(const stree_attn &a, const stree_kv &kv);
hipError_t launch_tree_attn(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *lengths, const void *q,
                            void *out, int32_t *status, void *workspace, hipStream_t st);

hipError_t launch_commit_kv(const stree_attn &a, const stree_kv &kv, const int32_t *parent, const int32_t *accepted,
                            const int32_t *lengths, int32_t *lengths_out, int32_t *status, hipStream_t st);

hipError_t launch_resize_kv(const stree_kv &kv, const stree_pool &pool, int batch, const int32_t *tokens, int32_t *status,
                            hipStream_t st);
hipError_t launch_fork_kv(const stree_kv &kv, const stree_pool &pool, int batch, int nforks, const int32_t *src, const int32_t *dst,
                          int32_t *lengths, int32_t *status, hipStream_t st);

}  // namespace stree
