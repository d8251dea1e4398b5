// Contexts in 8-bit pages and attention over whole prompts: launch interface (see pages.hip, paged_attn.hip, prompt.hip).
#pragma once
#include "common.hpp"

constexpr int PAGE_TOK = 64;       // tokens per page
constexpr int PAGED_MAX_REQ = 32;  // requests of one attention or store launch (FS_MAX_BATCH)
constexpr int SEQ_LIST = 256;      // sequences, or pairs of pages, one launch takes as kernel arguments

// A pool of pages on the device.  Tile (page, layer, K|V, head) is 64 * hd bytes at ((page * n_layers + layer) * 2 + kv) * Hkv + head:
// K as [hd / 64][64 tokens][64 columns], V as [hd][64 tokens] with token 16 a + 4 b + c at place 16 b + 4 a + c.  Both are the operand order of the attention kernel, which fetches 16 bytes per lane, 1 KiB per wave.
struct PoolDev {
    unsigned char* codes;
    float* scales;
    int32_t *ref, *table, *length, *work;
    int n_pages, n_layers, Hkv, hd, n_seqs, max_pages;
};

struct SeqLists {
    int n;
    int32_t a[SEQ_LIST], b[SEQ_LIST];
};

struct StoreItem {
    const void* base;  // token slot0 of (layer 0, K, head 0)
    long long stride_layer, stride_kv, stride_head, stride_tok;  // elements
    int seq, first_page, n_tokens, page0;                        // page0: pages of the items before this one
};
struct StoreArgs {
    PoolDev p;
    int32_t* written;  // [pages of all items] or null
    int n;
    StoreItem it[PAGED_MAX_REQ];
};

hipError_t launch_paged_store(int dtype, const StoreArgs& a, int pages, hipStream_t s);
hipError_t launch_page_grow(const PoolDev& p, const SeqLists& l, int32_t* status, hipStream_t s);
hipError_t launch_page_fork(const PoolDev& p, const SeqLists& l, int32_t* status, hipStream_t s);
hipError_t launch_page_free(const PoolDev& p, const SeqLists& l, hipStream_t s);
hipError_t launch_page_compact(const PoolDev& p, int32_t* status, hipStream_t s);
hipError_t launch_page_copy(const PoolDev& dst, const PoolDev& src, const SeqLists& l, hipStream_t s);

// One request of a paged attention launch: rows [row0, row0 + M) of the stacked arrays, its settled slots [0, n_paged) in the pages of
// table row `seq`, slot s >= n_paged at tail slot s - n_paged.
struct PagedReq {
    const void* tail;  // K of (layer 0, head 0), tail slot 0; null if no slot lies there
    int seq, n_paged, row0, M, l_glo, seg_off;
};
struct PagedArgs {
    const void* q;
    void* o;
    long long ldq, ldo;     // elements between rows; ldo == 0: `o` in the fragment-major layout of the output projection
    const unsigned char* codes;
    const float* scales;
    const int32_t* table;
    const uint64_t* anc;    // [rows][FS_ANC_WORDS], or null: rows are a chain
    long long page_tiles;   // tiles per page
    int n_pages, max_pages, tile0;  // tile0: index of (page 0, layer, K, head 0)
    int Hq, Hkv, hd, G;
    long long layer_off, stride_kv, stride_head, stride_tok;  // tail strides, elements
    float scale_log2;
    int n_req, rows, n_splits, units_per_split, tail_w, Rpad, row_blocks;
    float* part_o;   // [n_splits][Hkv][Rpad][hd]
    float* part_ml;  // [n_splits][Hkv][Rpad][2]
    PagedReq req[PAGED_MAX_REQ];
};
// Fills the split plan of `a` (req, n_req, Hkv, G, rows set) and returns the row tiles of a workgroup.
int paged_plan(int dtype, PagedArgs& a);
// Splits of a plan are at most this many for so many stacked rows of one KV head.
int paged_max_splits(int Hkv, long long R);
hipError_t launch_paged_attention(int dtype, const PagedArgs& a, int row_tiles, hipStream_t s);

constexpr int PROMPT_MAX_SEQ = 320;  // sequences, and levels of blocks, of one launch
struct PromptArgs {
    const void *q, *k, *v;
    void* o;
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head, o_tok, o_head;  // elements
    float scale_log2;
    int Hq, Hkv, G, hd;
    int rows, units, cus;             // rows of a block; workgroups; compute units
    int levels, width;                // see unit_of
    int32_t start[PROMPT_MAX_SEQ];    // first token of a sequence, the longest sequence first
    int32_t len[PROMPT_MAX_SEQ];      // its tokens, at least one
    int32_t first[PROMPT_MAX_SEQ];    // units of one head before a level, the highest level first
};
static_assert(sizeof(PromptArgs) <= 4096, "the kernel-argument segment");
// cu: host offsets [n_seq + 1]
hipError_t launch_prompt_attention(int dtype, PromptArgs& a, const int32_t* cu, int n_seq, hipStream_t s);
