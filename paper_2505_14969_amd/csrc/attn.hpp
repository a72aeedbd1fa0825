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

constexpr int kPieceKeys = 256;        // keys of a piece, at least: 64 for each wave
constexpr int kWorkgroups = 768;       // workgroups that a call is split into, if its keys allow: three to a CU

// The host knows how far the table reaches, the device how long the sequences are: the grid has `pieces` workgroups for each
// (sequence, head, tile of rows), and a sequence uses as many of them as its keys fill.
struct AttnSplit {
    int pieces, tiles, rows, units;    // rows: kept of each tile (fewer than the tile's where there is only one)
    Divisor group;                     // query heads of a key/value head
    float *parts;                      // [units, tiles, rows, dim]: sums of 2^(s - top) V
    float2 *sums;                      // [units, tiles, rows]: (top, sum of 2^(s - top)); a negative sum: -attn_code()
    explicit AttnSplit(int r) : group(r) {}
    __device__ __forceinline__ int piece_keys(int keys) const {
        const int each = (keys + pieces - 1) / pieces;
        return max((each + 127) & ~127, kPieceKeys);
    }
};

// What is wrong with a sequence as a small positive number, the first bad node before a page (two pieces may find both).
__device__ __forceinline__ int attn_code(int status) { return status > 0 ? status : 1000; }
__device__ __forceinline__ int attn_status(int code) { return code < 1000 ? code : STREE_SEQ_PAGE; }

// the streaming kernel (tree_attn_stream.hip)
bool attn_stream_supported(const stree_attn &a, const stree_kv &kv, const void *q, const void *out);
size_t attn_stream_workspace(const stree_attn &a, const stree_kv &kv);
hipError_t launch_attn_stream(const stree_attn &at, const stree_kv &kv, const AttnArgs &a, void *workspace, hipStream_t st);

}  // namespace stree
