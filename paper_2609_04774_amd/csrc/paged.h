// Internal declarations of the operators over a paged cache: attention of a
// batch's newest rows or of a rank's rows through a window, and the cache's pages.
#pragma once

#include "internal.h"

namespace cpattn {

constexpr int kMaxTokens = 1 << 30;  // positions of one sequence

// Blocks of rows (of one KV head) and their order.
struct Blocks {
  int32_t rows;         // of a block
  int32_t n;            // blocks of a segment, at most
  int32_t stride, run;  // place i of the order is block (i % run) * stride + i / run
};

// One launch of attention over a paged cache, of a batch's sequences (tables,
// lengths and row starts in device memory) or of a rank's two chunks.
struct PagedParams {
  const uint16_t* q;
  uint16_t* o;             // bf16 [rows][Hq][128]
  float* lse;              // fp32 [rows][Hq], or null
  int64_t q_stride;        // elements between rows of q
  int64_t n_rows;          // rows of q (a batch's; at most 2^30)
  int32_t Hq, Hkv, G;      // G = Hq / Hkv
  int32_t window, n_sink;  // window 0: none
  float scale_log2;

  const unsigned char* k_cache;
  const unsigned char* v_cache;
  int64_t kv_stride;       // bytes between keys of one head
  int32_t n_blocks;
  int32_t table_len;       // entries of a table
  const int32_t* tables;
  int64_t table_stride;
  int32_t streamed;        // more pages than the Infinity Cache holds
  int32_t paged_end;       // positions below it are read through the table
  int32_t key_end;         // and from this one on there are no keys

  // A batch: sequence s has rows q_start[s] .. q_start[s + 1] (or uniform_q each),
  // the last of its kv_len[s] positions.
  int32_t n_segments;
  const int32_t* q_start;
  const int32_t* kv_len;
  int32_t uniform_q, max_q;

  // A rank (n_chunks 2): its chunks' first row in q and o, length and position;
  // positions from paged_end on are rows of k_new and v_new.
  int32_t n_chunks;
  int32_t chunk_len[2], chunk_pos[2];
  int64_t chunk_row[2], chunk_out[2];
  const unsigned char* k_new;
  const unsigned char* v_new;

  // Workspace: where each workgroup's share of the walks begins, then two slots of
  // partial results per workgroup.
  int32_t n_shares;
  Blocks blocks[3];        // ways to cut the rows into blocks: of 16 or 32 rows, or
  int32_t n_ways;          // (kChunkRows) two or three
  int32_t* choice;         // of these, by the lengths; null: the first
  struct ShareStart* starts;
  float* slots;
};

// Where a workgroup's share of the launch begins: a step (of tiles) of the walk of
// one block of rows (its place in the launch's order) and KV head.
struct ShareStart {
  int32_t place, kvh, step, reserved;
};

constexpr int kRowsThreads = 256;
constexpr int kChunkThreads = 512;
// Rows of a block of the kernels of many rows; the last only for long launches.
constexpr int kChunkRows[3] = {128, 256, 384};
constexpr int kRowsShares = 512;   // workgroups: two per compute unit
constexpr int kChunkShares = 256;  // one

__host__ __device__ constexpr size_t slot_floats(int rows) { return (size_t)rows * (kHeadDim + 1); }

int launch_attn_rows(const PagedParams& p, void* stream, const char* who);
int launch_attn_chunk(const PagedParams& p, void* stream, const char* who);
int launch_attn_merge(const PagedParams& p, void* stream, const char* who);

// ---------------------------------------------------------------------------
// The pages of a cache.

struct AppendParams {
  const unsigned char* k_rows;
  const unsigned char* v_rows;
  int64_t k_stride, v_stride;  // bytes between rows
  int64_t first_row, n_rows;  // of this launch, and of all
  int64_t row_bytes;
  unsigned char* k_cache;
  unsigned char* v_cache;
  int64_t n_blocks;
  const int32_t* tables;
  int64_t table_stride;
  const int32_t* kv_len;
  const int32_t* q_start;
  int32_t n_seqs, uniform_q;
};

int launch_append(AppendParams p, void* stream);

struct CacheSet {
  unsigned char* cache[CP_KV_MAX_CACHES];
  int32_t n;
  int64_t n_blocks, page_bytes;
};

int launch_copy_pages(const CacheSet& c, const int32_t* src, const int32_t* dst, int64_t n, void* stream);
int launch_reserve(const cp_kv_pool& pool, const int32_t* seqs, const int32_t* add, int32_t n, int32_t* missing,
                   void* stream);
int launch_fork(const cp_kv_pool& pool, const CacheSet& c, const int32_t* parents, const int32_t* children, int32_t n,
                int32_t* missing, void* stream);
int launch_free(const cp_kv_pool& pool, const int32_t* seqs, const int32_t* begin, const int32_t* end, int32_t n,
                void* stream);
// Workspace of a compaction, in int32: the number of moves, their sources and
// destinations, and each page's new place.
__host__ __device__ constexpr size_t compact_ints(int64_t n_blocks) { return 64 + 2 * (size_t)n_blocks + 64; }
int launch_compact(const cp_kv_pool& pool, const CacheSet& c, int32_t* work, void* stream);

}  // namespace cpattn
