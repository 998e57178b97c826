// What the two halves of the calls on a paged cache share: cache_api.hip checks, sizes and launches; cache.hip and paged_attn.hip hold the kernels.
#pragma once
#include "kernels.h"
#include "paged.h"

namespace dcp {

// What a workgroup copies at a time: kPieceChunks chunks (16 KiB) of a page, so that pages that are filled unevenly, or few, still fill the chip
// (64 sequences forked, 4 layers, pages of 512 KiB: 93 us with a workgroup a page, 47 so).
static constexpr int kPieceChunks = 1024;
// Workgroups that share such pieces, each taking every kCopyWorkers-th: 2 430 pages of 512 KiB moved, 5.1 GB read and written, in 995 us with
// 4 096, 980 with 16 384 and 64 KiB at a time, 842 to 960 (by where the pages lie) so: 5.3 to 6.0 TB/s.
static constexpr int kCopyWorkers = 32768;
inline int pieces_of(const KCache& c) { return (int)(((int64_t)c.page.d * c.hkv * c.head_chunks() + kPieceChunks - 1) / kPieceChunks); }

// What the two launches of dcp_cache_compact share: the pages that move, and where every page goes.
struct Moves {
  int32_t *count, *from, *to, *where;   // [1], [n_pages / 2 + 1], [n_pages / 2 + 1], [n_pages]: of the pages behind those in use, -1: free
};

struct NewTokens {
  const char *k, *v;
  int64_t k_st, k_sh, v_st, v_sh;   // bytes
  int64_t n;
};

struct PagedArgs {
  const char* q;
  char* out;
  float* lse;
  const int32_t *seqs, *status;
  int64_t q_st, q_sh, o_st, o_sh;   // bytes
  int32_t n, group, window, sink;   // group: query heads of a KV head
  // Query heads that share a KV head are taken in sets of up to 16 (or 8, see Tile::weigh); a workgroup's waves take `abreast` (1, 2 or 4) sets
  // that lie side by side, and where there are fewer than four, the waves of a set take its tiles in turn.
  int32_t per_kv, set_heads, abreast, log_abreast, groups;   // sets of a KV head, heads of a set at most, ..., sets / abreast
  int32_t whole;   // items are not cut: nothing to join
  float scale_log2e;
};

// Partial results of items (place, group of sets) that several workers share, unnormalised, in units of log2.  A worker's share of the tiles
// begins in the middle of at most one item and ends in the middle of at most one: slot 2 w holds the first, 2 w + 1 the second.
struct PagedParts {
  int4* joins;     // [kWorkers] (place, group, first worker, last worker), place -1: nothing to join.  By item where there are no more
                   // items than workers (not written for padding), else by the worker that has the item's first tile
  float2* ml;      // [2 kWorkers][abreast][set_heads] running maximum, sum
  float* o;        // [2 kWorkers][abreast][set_heads][D]
  int32_t by_item;
};

// Two workgroups on a CU, all resident.  The four waves read neighbouring heads of the same keys: where each workgroup walks one head, a
// quarter of what the memory reads lies in pages that others open again (8 KV heads of 256 bytes, a plain read of all keys
// and values 5.8 TB/s against 6.9; linear 7.0).
static constexpr int kLogWorkers = 9, kWorkers = 1 << kLogWorkers;
static constexpr int kPagedWaves = 4, kPagedThreads = 64 * kPagedWaves;
static constexpr int kSetHeads = 16;     // query heads of a matrix tile
static constexpr int kPagedKeys = 32, kPagedKeysF32 = 16;   // keys of a tile, in fp32 caches

struct ReadTokens {
  char *k, *v;
  int64_t k_st, k_sh, v_st, v_sh;   // bytes
  int64_t n;
};

// The checks that the calls share (cache_api.hip).
dcp_status_t pack_cache(const dcp_cache_t* cache, KCache* out);
dcp_status_t check_places(const KCache& c, const int32_t* seqs, int32_t n);
dcp_status_t check_attn_args(const KCache& c, const dcp_paged_attn_t& t);
dcp_status_t check_rows(const char* name, const void* p, int64_t stride_t, int64_t stride_h, const dcp_cache_t* cache);
inline bool is_aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

// dcp_paged_attn_chunk_fwd: the rows of a place and KV head (token after token, of each the query heads that share it) are taken in tiles, the items; kWorkers
// workgroups share all items' key tiles, KV head after KV head, evenly.  Tiles have 128 rows and 64 keys in LDS, or, where places have kFewRows between
// them on average at most or all heads of all tokens are kFewAll at most, 16 rows and 32 keys in registers, as for one token.  Whole calls in a graph, us, with keys in LDS / in registers, 32/8 heads of
// 128, 16 sequences of 300, 2 048 and 8 192 tokens: 6 rows 20.7 / 16.0, 38.4 / 27.8, 92 / 61; 12 rows 22.0 / 17.9, 40.0 / 30.3, 93 / 68; 24 rows 25.2 / 17.9, 42.8 / 34.6, 100 / 87; 39 rows
// 28.9 / 23.3, 45.0 / 43.8, 103 / 143; 80 rows 36.7 / 29.6, 50.6 / 63.7, 116 / 240; 16/4 heads of 64, 39 rows 17.4 / 14.6, 29.8 / 23.4, 48 / 67.  By all heads of all tokens, sequences of 300, 4 096 and
// 32 768 tokens: 32/8 of 128, one, 1 088 21.4 / 17.7, 40.0 / 30.0, 91 / 93; two, 800 18.1 / 14.3, 37.2 / 28.8, 83 / 91; four, 1 056 18.1 / 14.3, 36.7 / 30.2, 106 / 129; 2 528 21.9 / 19.7, 42.9 / 39.3,
// 134 / 220; 16/1 of 128, one, 848 20.1 / 16.1, 55.6 / 28.0, 78 / 71 (few items of many parts, which are long to join); 128 18.3 / 11.8, 49.7 / 25.7, 242 / 46; 64/2 of 64, two, 768 16.6 / 12.0, 50.1 / 19.6,
// 73 / 64; 1 216 17.0 / 12.2, 47.0 / 21.1, 62 / 75.  Items of 32 rows in registers were between the two.
// These are batches of places that are alike.  The rule knows no others: places that are padding count, and all go the same way.  32/8 heads of 128 behind 8 192 tokens, a piece of 300 new
// tokens alone 84, padded to 64 places, where it goes by registers, 152; of 512 120, padded to 128 245; 63 single tokens alone 237, with a piece of 300 beside them 358 (registers, 37 more
// than the two alone), of 512 413 (LDS, 56 more), of 2 048 691 (64 more).
static constexpr int kChunkRows = 128, kChunkKeys = 64, kFewRows = 24, kFewItem = 16, kFewAll = 1024, kOwnItems = 256;
struct ChunkArgs {
  const char* q;
  char* out;
  float* lse;
  const int32_t *seqs, *status, *cu;
  int64_t q_st, q_sh, o_st, o_sh;   // bytes
  int64_t n_tokens;
  int32_t n, window, sink, max_items;
  int32_t rows, tile;               // of an item at most; keys of a tile
  FastDiv group;                    // query heads of a KV head
  float scale_log2e;
};
struct ChunkItem {
  int32_t seq, first, pos, rows;      // first token of the place (of the packed ones) and its position; rows of the place
  int32_t row0, tiles, before, pad;   // first row of the item; its key tiles, and those of the items before
};
struct ChunkJoin {
  int32_t hk, first_worker, last_worker, pad;   // last_worker -1: nothing to join
  int32_t first, rows, row0, pad2;              // of the item
};
struct ChunkPlan {
  int4* head;        // [1] items, their key tiles (of one KV head)
  ChunkItem* items;  // [max_items]
  int4* starts;      // [kWorkers] KV head, item, key tile of it
  ChunkJoin* joins;  // [kWorkers] by the worker that begins an item and does not end it
  float2* ml;        // [2 kWorkers][rows] running maximum, sum: of an item that a worker does not begin slot 2 w, of one that it does 2 w + 1
  float* o;          // [2 kWorkers][rows][D], unnormalised
};

// One launch each, of `grid` workgroups where it goes by the call.
void launch_take(bool fork, const KCache& c, const int32_t* a, const int32_t* b, int32_t n, int32_t* status, hipStream_t s);
void launch_fork(uint32_t grid, const KCache& c, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* status, int32_t pieces, hipStream_t s);
void launch_free(uint32_t grid, const KCache& c, const int32_t* seqs, hipStream_t s);
void launch_list_moves(const KCache& c, const Moves& m, int32_t* counts, hipStream_t s);
void launch_move(uint32_t grid, const KCache& c, const Moves& m, const int32_t* counts, int32_t pieces, hipStream_t s);
void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t s);   // each: tokens of a workgroup, 1 or 4
void launch_append8(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                    const NewTokens& x, hipStream_t s);   // of launch_append, for a cache in 8 bits: each 1, 16 or 64, with blocks of one token 1 or 4
void launch_read(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                 const ReadTokens& x, hipStream_t s);     // each: 1 or 4
// The plan, the walk and the join.
void launch_chunk_few(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s);   // the walk with keys in registers
void launch_chunk(int32_t d, const KCache& c, const ChunkArgs& a, const ChunkPlan& plan, hipStream_t s);
// and the join where items are cut
void launch_paged_attn8(int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s);
void launch_paged_attn(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s);

}  // namespace dcp
