// Host-side declarations of the paged cache's launchers (paged.hip) and the argument structs they take.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ss {

// One layer of a paged cache (or, for eviction, the first of several, `layer_*` apart).  Strides in elements.
struct PagedArgs {
    void *k, *v;
    int64_t page_stride, head_stride, slot_stride;
    float *weight;     // [n_pages][Hk][page]
    int32_t *position; // [n_pages][Hk][page]
    const int32_t *table; // [B][max_pages]
    const int32_t *len;   // [B]; below zero: an idle place
    int32_t *status;      // may be NULL
    int B, Hk, hd, page_bits, n_pages, max_pages;
};
enum : int { PAGED_BAD_PAGE = 8, PAGED_BAD_LENGTH = 16 };

struct PagedAppendArgs {
    PagedArgs kv;
    const void *k_new, *v_new; // row r = b*M + m; element e of head h at r*ld + h*head + (e * elem for values of a ring, else e)
    int64_t ld_k, head_k, ld_v, head_v;
    const int32_t *next_pos; // [B], or NULL: positions are the slots
    int M;
    int ring; // > 0: k_new, v_new are a contiguous cache of `ring` slots a head (ss_kv_cache's layout) that holds position p at p mod ring
};
void launch_paged_append(int dtype, const PagedAppendArgs &a, hipStream_t st);
// pos[b] = next_pos[b] (NULL: len[b]), brought into [0, last]; idle places: 0
void launch_paged_positions(const int32_t *len, const int32_t *next_pos, int B, int last, int32_t *pos, int32_t *status, hipStream_t st);
void launch_paged_advance(int32_t *len, int32_t *next_pos, int B, int M, hipStream_t st);

struct PagedAttnArgs {
    PagedArgs kv;
    const void *q, *q_lo; // row r = b*M + m at r*ldq, head h at h*q_head; q_lo: second plane of fp32 activations, or NULL
    void *out, *out_lo;
    int64_t ldq, q_head, ldo, o_head;
    float *weight_out; // NULL: no weights
    int H, G, M, GM;   // GM = G * M query rows to a key head: row x is head x / M of the group, new row x % M
    int pending;       // rows appended behind len
    int max_n;         // host's bound on a sequence's positions
    float scale_log2e; // > 0
    int turn;          // the queries' signs are turned (a negative scale)
    int stream;        // ask for keys and values with the non-temporal bit
    // set by the launcher
    int rowblocks, row_tiles, workgroups; // workgroups: parts of the positions, each of a workgroup to a block of rows
    float2 *part_ml; // [rowblocks][2 * workgroups][16 * row_tiles] largest score and sum of weights of a piece
    float *part_o;   // [rowblocks][2 * workgroups][16 * row_tiles][hd] unnormalised
    float2 *row_stats; // [B*Hk*GM] largest score and reciprocal sum of weights of the rows of units that one workgroup had (with weights and several row blocks)
    float *scores;   // [B*Hk*GM][ld_scores] products of queries and keys
    int64_t ld_scores;
};
// units of a call (sequences, key heads, blocks of query rows), and the blocks of positions that all of them walk over at most
long long paged_attention_blocks(int dtype, int B, int Hk, int GM, int max_n, long long &units);
size_t paged_attention_workspace(int dtype, int B, int Hk, int hd, int G, int M, int max_n, bool weights);
void launch_paged_attention(int dtype, PagedAttnArgs a, void *ws, hipStream_t st);

struct PagedEvictArgs {
    PagedArgs kv;
    int64_t layer_stride; // of k and v
    int n_layers;
    float *weight_out;
    int32_t *position_out, *len_out;
    int budget, keep_first, keep_recent, max_n;
    // set by the launcher
    uint32_t *moves; // [n_layers*B*Hk][2][list] places (page * page size + place in it) that are filled and places that fill them
    int32_t *n_moves;
    int list;
    int elem, row_units; // bytes of an element; 16-byte units of a row (logarithm)
};
size_t paged_evict_workspace(int n_layers, int B, int Hk, int max_n, int budget);
void launch_paged_evict(int dtype, PagedEvictArgs a, void *ws, hipStream_t st);

} // namespace ss
