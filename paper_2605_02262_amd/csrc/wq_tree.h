// What the two kernels of wq_tree_attention share: their arguments, and who sees whom in a tree.
#pragma once
#include "wq_attend.h"

struct TreeArgs {
    const char *q, *k, *v;
    int64_t q_stride, k_stride, v_stride;      // bytes from row to row
    const int32_t *row_off, *parent;
    int64_t total;
    int B, Hq, rep;
    int units, splits;                         // (tile of rows, KV head) pairs, and the parts that each one's keys are cut into
    float scale;                               // log2(e) * sm_scale
    uint32_t* status;
    wq_packed_kv kv;
    void* out;                                 // as in Out
    float *lse, *part, *part_ml;
    int longest;                               // wavefronts that bring their own keys: blocks of 32 keys of the longest sequence, or 0
};

typedef void (*TreeKernel)(TreeArgs);
// The kernel in which every wavefront brings its own keys, for tiles of 16 * columns query rows: see wq_tree_stream.hip
constexpr int WQ_STREAM_WAVES = 4;
constexpr int WQ_STREAM_SLOTS = 512;           // workgroups that the card holds at a time
void wq_launch_tree_stream(wq_ctx* ctx, const TreeArgs& a, int dtype, int columns);

namespace {

constexpr int WORDS = WQ_MAX_TREE / 64;        // of a row's ancestors

// Which new rows each of the rows node0 .. node0 + n - 1 sees, a bit each: itself, its parent, its parent's parent ..  (a parent lies in front of its
// child, so every walk ends).  For all threads of a workgroup.
__device__ __forceinline__ void find_ancestors(const int32_t* parent, int node0, int n, uint64_t* seen, int32_t* s_parent, int threads)
{
    const int last = node0 + n < WQ_MAX_TREE ? node0 + n : WQ_MAX_TREE;
    for (int i = threadIdx.x; i < last; i += threads) s_parent[i] = parent[i];
    for (int i = threadIdx.x; i < n * WORDS; i += threads) seen[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += threads) {
        int j = node0 + i;
        if (j >= WQ_MAX_TREE) continue;
        uint64_t word = 0;
        int at = j >> 6;
        while (true) {
            if (j >> 6 != at) seen[i * WORDS + at] = word, word = 0, at = j >> 6;
            word |= uint64_t(1) << (j & 63);
            const int up = s_parent[j];
            if (up < 0 || up >= j) break;
            j = up;
        }
        seen[i * WORDS + at] = word;
    }
    __syncthreads();
}

}  // namespace
