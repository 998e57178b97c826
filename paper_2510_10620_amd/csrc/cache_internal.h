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

// One launch each, of `grid` workgroups where it goes by the call.
void launch_take(bool fork, const KCache& c, const int32_t* a, const int32_t* b, int32_t n, int32_t* status, hipStream_t s);
void launch_fork(uint32_t grid, const KCache& c, const int32_t* src, const int32_t* dst, int32_t n, const int32_t* status, int32_t pieces, hipStream_t s);
void launch_free(uint32_t grid, const KCache& c, const int32_t* seqs, hipStream_t s);
void launch_list_moves(const KCache& c, const Moves& m, int32_t* counts, hipStream_t s);
void launch_move(uint32_t grid, const KCache& c, const Moves& m, const int32_t* counts, int32_t pieces, hipStream_t s);
void launch_append(int32_t each, uint32_t grid, const KCache& c, int32_t layer, const int32_t* seqs, const int32_t* cu, int32_t n, const int32_t* status,
                   const NewTokens& x, hipStream_t s);   // each: tokens of a workgroup, 1 or 4
// and the join where items are cut
void launch_paged_attn(int32_t dtype, int32_t d, uint32_t grid, const KCache& c, const PagedArgs& a, const PagedParts& parts, hipStream_t s);

}  // namespace dcp
