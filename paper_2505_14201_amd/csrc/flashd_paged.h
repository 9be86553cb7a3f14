// A cache of keys and values kept in pages, as the kernels that read and write it see it.
//
// K and V are pools of pages [P][Hkv][page][d], pages page_stride apart; row b of the table names the
// pages of sequence b in the order of its keys, -1 where it has none, -2 - p where page p is held back.  New tokens of sequence b are rows
// q_start[b] .. q_start[b + 1] - 1 of packed [T][heads][d] tensors and stand at keys lens[b] + i.
// All of that is device memory which the host never reads, so every number taken from it is checked
// here before it becomes an address: a page outside the pool is no page, a sequence ends at the
// end of its table and its tokens at T.
#pragma once

#include "flashd_common.h"

namespace flashd {

constexpr int kCacheMaxSeqs = 4096;

struct Paged {
    char* k;                // of the call's layer
    char* v;
    int* table;
    const int* lens;
    const int* q_start;
    int64_t page_bytes;     // from one page to the next
    int64_t layer_bytes;    // from one layer to the next (calls that work on all layers)
    int64_t head_bytes;     // page * d elements
    int layers, P, page_log2, max_pages, B, Hkv, d;
    int esz;                // bytes of an element
    int T;                  // rows of the packed tensors
    float kscale, vscale;
};

// Sequence b's place in the packed tensors and in its table.
struct Seq {
    int row0;       // first row of its new tokens
    int n;          // new tokens
    int len;        // keys in the cache before them
};

// New tokens of a sequence whose rows begin at `start` (>= 0) and end before `next`.  Whatever `next` is, it is brought between 0 and T before the
// difference is formed, which then has no overflow.
__host__ __device__ __forceinline__ int tokens_of(int start, int next, int T) {
    return max(min(max(next, 0), T) - start, 0);
}

// `most`: keys that a row of the table has room for
__host__ __device__ __forceinline__ Seq seq_of(int start, int next, int len, int T, int most) {
    Seq s;
    s.row0 = max(start, 0);
    s.len = min(max(len, 0), most);
    s.n = min(tokens_of(s.row0, next, T), most - s.len);
    return s;
}

// Columns that `tokens` new tokens need behind the end of the table, where the first n have a key.
__host__ __device__ __forceinline__ int columns_beyond(int tokens, int n, int page_log2) {
    return (int)(((uint32_t)(tokens - n) + (1u << page_log2) - 1u) >> page_log2);
}

__device__ __forceinline__ Seq seq_at(const Paged& c, int b) {
    return seq_of(c.q_start[b], c.q_start[b + 1], c.lens[b], c.T, c.max_pages << c.page_log2);
}

// The page that an entry of the table names, -1 if none.  An entry of -2 - p names page p like one of p (it counts in refs), but holds it
// back: to all who read or write keys it is no page.
__host__ __device__ __forceinline__ int named_page(int entry) { return entry < -1 ? -2 - entry : entry; }

// The page of column `col` (>= 0) of sequence b, -1 if there is none.
__device__ __forceinline__ int page_at(const Paged& c, int b, int col) {
    if (col >= c.max_pages) return -1;
    const int p = c.table[(size_t)b * c.max_pages + col];
    return (unsigned)p < (unsigned)c.P ? p : -1;
}

// Sum over the lanes up to this one: within rows of 16 lanes, then the last of row 0 and of row 2 to the next row, then that of row 1 to
// rows 2 and 3.  (Moves between lanes in the vector units; by LDS, as a shuffle goes, six of them one after the other take 0.3 us.)
__device__ __forceinline__ int lanes_up_to(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);       // from 1, 2, 4 and 8 lanes before
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);       // lane 15 of a row to rows 1 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);       // lane 31 to rows 2 and 3
    return x;
}

// What cache_append works on beside the cache: strides in elements.
struct AppendArgs {
    const void *q, *k, *v;
    void* q_out;
    const int* positions;       // or NULL: the token's key
    const float* inv_freq;      // NULL: no rotation
    const void *q_weight, *k_weight;    // NULL: not normed
    int64_t q_stride, k_stride, v_stride, qo_stride;
    int Hq, rot, interleaved, dtype, fp8;
    float eps;
};

hipError_t launch_cache_append(const Paged& c, const AppendArgs& a, hipStream_t st);

// New tokens that attend to the cache and to each other.
struct TreeArgs {
    const void* q;
    void* o;
    const uint32_t* tree;       // [T][words] bits, or NULL: a chain
    int64_t q_stride, o_stride; // elements
    int words;                  // 32-bit words of a row's bits
    int Hq, max_q, dtype, fp8;
    float scale;
    float* ws;
    float* lse;                 // [T][Hq], or NULL
};

hipError_t launch_attn_tree(const Paged& c, const TreeArgs& a, hipStream_t st);
size_t attn_tree_workspace(int Hq, int Hkv, int max_q, int d, int dtype);

// Drafted tokens that are asked whether they stay: strides in elements.
struct VerifyArgs {
    const void *logits, *draft;         // draft NULL: drafts were not sampled
    const int *tokens, *parent;         // parent NULL: chains
    const float *uniform, *temperature; // temperature NULL: 1
    const int* q_start;
    int *keep, *n_keep, *next;
    int64_t logits_stride, draft_stride;
    int B, T, V, dtype, draft_dtype, max_keep;
};

hipError_t launch_verify(const VerifyArgs& a, void* ws, hipStream_t st);
size_t verify_workspace(int T, int V);

// New tokens whose attention weights are added to the keys' scores.
struct ScoreArgs {
    const void* q;
    const uint32_t* tree;       // [T][words] bits, or NULL: a chain
    const float *lse, *weight;  // [T][Hq], [T] or NULL
    float* score;               // [B][Hkv][score_stride]
    int64_t q_stride, score_stride;
    int words;                  // 32-bit words of a row's bits
    int Hq, dtype, fp8;
    float scale, decay;
};

hipError_t launch_cache_score(const Paged& c, const ScoreArgs& a, hipStream_t st);

constexpr int kEvictMostUnits = 1 << 20;       // sequences times kv heads (times layers) of a launch

// Keys that go, of all layers.
struct EvictArgs {
    const int *refs, *budgets;  // budgets NULL: `budget` of every sequence
    float* score;               // [layers][B][Hkv][score_stride]
    int64_t score_stride, score_layer_stride;
    int budget, first, recent;
    int* lens_out;
};

hipError_t launch_cache_evict(const Paged& c, const EvictArgs& a, void* ws, hipStream_t st);
size_t evict_workspace(const Paged& c, int budget);

hipError_t launch_cache_fork(const Paged& c, int* refs, const int* parent, int B_out, int* table_out,
                             int* lens_out, hipStream_t st);
hipError_t launch_cache_reserve(const Paged& c, int* refs, int* report, hipStream_t st);
hipError_t launch_cache_commit(const Paged& c, const int* keep, int max_keep, const int* n_keep,
                               int* lens_out, hipStream_t st);

}  // namespace flashd
