// Host side of attention over a paged cache: argument checks and kernel
// parameters for cp_attn_paged and cp_attn_window (include/cp_attn.h).  Nothing is
// planned here: the kernels cut the work by the lengths that they read.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <string>

#include "paged.h"

using namespace cpattn;

namespace {

constexpr int64_t kInfinityCacheBytes = 256 << 20;

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_heads(int32_t Hq, int32_t Hkv, const std::string& who) {
  if (Hq < 1 || Hkv < 1 || Hq % Hkv)
    return fail(CP_ERR_INVALID, who + "head counts must be >= 1, n_heads_q a multiple of n_heads_kv");
  if (Hq > 4096) return fail(CP_ERR_UNSUPPORTED, who + "more than 4096 query heads");
  return CP_OK;
}

// What both calls check of the heads and the mask, and set.
int set_common(PagedParams* p, const std::string& who, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale,
               int64_t window, int64_t n_sink) {
  const int st = check_heads(Hq, Hkv, who);
  if (st != CP_OK) return st;
  if (head_dim != CP_HEAD_DIM) return fail(CP_ERR_UNSUPPORTED, who + "head_dim must be 128");
  if (!(scale == scale) || std::isinf(scale)) return fail(CP_ERR_INVALID, who + "softmax_scale is not finite");
  if (window < 0 || n_sink < 0) return fail(CP_ERR_INVALID, who + "window and n_sink must be >= 0");
  p->Hq = Hq;
  p->Hkv = Hkv;
  p->G = Hq / Hkv;
  p->scale_log2 = (scale > 0.f ? scale : 1.f / std::sqrt((float)head_dim)) * 1.4426950408889634f;
  if (std::isinf(p->scale_log2)) return fail(CP_ERR_INVALID, who + "softmax_scale is too large");
  // No position is beyond 2^30: a longer window shows every key.
  p->window = window >= kMaxTokens ? 0 : (int32_t)window;
  p->n_sink = (int32_t)(n_sink < kMaxTokens ? n_sink : kMaxTokens);
  p->kv_stride = (int64_t)Hkv * kHeadDim * 2;
  return CP_OK;
}

// Rows of a block: the fewest that hold the most rows of a sequence and KV head, up to
// 32 with the kernel of few rows; else those of the other.
int block_rows(int64_t max_q, int32_t G) {
  const int64_t rows = max_q * G;
  return rows <= 16 ? 16 : rows <= 32 ? 32 : kChunkRows[0];
}
int shares_of(int block_rows) { return block_rows == kChunkRows[0] ? kChunkShares : kRowsShares; }

// Ways to cut the rows into blocks, of which the lengths choose.  The widest blocks
// are worth a second kernel's launch (4 us where it has nothing to do) to calls of many
// rows only.  One prompt's 4096 rows of 32 and 8 heads with and without the choice:
// alone 177 and 175 us, after 8K tokens 614 and 639, after 32K 1923 and 2032.  Of 2048 rows
// blocks of 384 alone take 99 us, the others as chosen 81; after 8K 306 and 305, after 32K
// 973 and 1006.
int ways_of(int block_rows, int64_t n_rows, int32_t Hq) {
  return block_rows != kChunkRows[0] ? 1 : n_rows * Hq >= 131072 ? 3 : 2;
}

// The shares' starts and, behind them, the choice of blocks.
size_t starts_bytes(int shares) { return ((size_t)shares * sizeof(ShareStart) + 255) / 256 * 256 + 256; }

size_t workspace_bytes_of(int64_t n_rows, int64_t max_q, int32_t Hq, int32_t G) {
  const int rows = block_rows(max_q, G), ways = ways_of(rows, n_rows, Hq);
  return starts_bytes(shares_of(rows)) + 2 * (size_t)shares_of(rows) * slot_floats(ways > 1 ? kChunkRows[ways - 1] : rows) * 4;
}

// How a launch is cut into blocks of so many rows.
Blocks cut(const PagedParams& p, int rows) {
  Blocks b;
  b.rows = rows;
  b.n = (int32_t)(((int64_t)p.max_q * p.G + rows - 1) / rows);
  const int64_t places = (int64_t)p.n_segments * b.n;
  // Blocks of a share, where each has several; not where most places have no rows
  // (few long chunks among many sequences: those places are passed over in order).
  // Against the order of the blocks themselves (before the sums of rounded weights): rank
  // 0 of a 32K prompt at degree 4 1977 us, 2132; through a window of 4096 433, 459.
  const int64_t full = p.n_rows * p.G / rows;
  const int64_t run = places * p.Hkv / p.n_shares;
  b.run = rows >= kChunkRows[0] && run > 1 && 2 * full >= places ? (int32_t)run : 1;
  b.stride = (int32_t)((places + b.run - 1) / b.run);
  return b;
}

int launch(PagedParams* p, const std::string& who, int64_t max_q, void* workspace, size_t workspace_bytes, void* stream) {
  const size_t need = workspace_bytes_of(p->n_rows, max_q, p->Hq, p->G);
  if (!workspace) return fail(CP_ERR_INVALID, who + "workspace is NULL");
  if (!aligned(workspace, 256)) return fail(CP_ERR_INVALID, who + "workspace must be 256-byte aligned");
  if (workspace_bytes < need)
    return fail(CP_ERR_CAPACITY, who + "workspace needs " + std::to_string(need) + " bytes");
  const int rows = block_rows(max_q, p->G);
  if (p->n_segments * ((max_q * p->G + rows - 1) / rows) > INT32_MAX / 2)
    return fail(CP_ERR_UNSUPPORTED, who + "too many sequences of so many rows");
  p->max_q = (int32_t)max_q;
  p->n_shares = shares_of(rows);
  unsigned char* const slots = static_cast<unsigned char*>(workspace) + starts_bytes(p->n_shares);
  p->n_ways = ways_of(rows, p->n_rows, p->Hq);
  for (int y = 0; y < p->n_ways; ++y) p->blocks[y] = cut(*p, p->n_ways > 1 ? kChunkRows[y] : rows);
  if (p->n_ways > 1) p->choice = reinterpret_cast<int32_t*>(slots - 256);
  p->starts = static_cast<ShareStart*>(workspace);
  p->slots = reinterpret_cast<float*>(slots);
  const std::string name = who.substr(0, who.size() - 2);
  return p->n_ways > 1 ? launch_attn_chunk(*p, stream, name.c_str()) : launch_attn_rows(*p, stream, name.c_str());
}

// The most rows of a sequence, from a batch's arguments.
int check_rows(const std::string& who, int32_t n_seqs, int64_t n_rows, bool uniform, int64_t* max_q, int32_t G) {
  if (n_seqs < 0 || n_rows < 0) return fail(CP_ERR_INVALID, who + "n_seqs and n_rows must be >= 0");
  if (n_rows > kMaxTokens || n_rows * G > INT32_MAX) return fail(CP_ERR_UNSUPPORTED, who + "too many rows");
  if (n_rows == 0 || n_seqs == 0) return CP_OK;
  if (uniform) {
    if (n_rows % n_seqs) return fail(CP_ERR_INVALID, who + "without q_start n_rows must be a multiple of n_seqs");
    *max_q = n_rows / n_seqs;
  } else {
    if (*max_q < 1) return fail(CP_ERR_INVALID, who + "max_q must be >= 1");
    if (*max_q > n_rows) *max_q = n_rows;
  }
  return CP_OK;
}

}  // namespace

extern "C" size_t cp_attn_paged_workspace_size(int32_t n_seqs, int64_t n_rows, int64_t max_q, int32_t n_heads_q,
                                               int32_t n_heads_kv) {
  size_t total = 0;
  const int st = guarded([&]() -> int {
    const std::string who = "cp_attn_paged_workspace_size: ";
    int s = check_heads(n_heads_q, n_heads_kv, who);
    if (s != CP_OK) return s;
    s = check_rows(who, n_seqs, n_rows, false, &max_q, n_heads_q / n_heads_kv);
    if (s != CP_OK) return s;
    if (n_rows > 0 && n_seqs > 0) total = workspace_bytes_of(n_rows, max_q, n_heads_q, n_heads_q / n_heads_kv);
    return CP_OK;
  });
  if (st != CP_OK) return 0;
  clear_error();
  return total;
}

extern "C" int cp_attn_paged(const cp_paged_kv* kv, const void* q, int64_t q_stride, int64_t n_rows,
                             const int32_t* q_start, int64_t max_q, int32_t n_heads_q, int32_t head_dim,
                             float softmax_scale, int64_t window, int64_t n_sink, void* o, float* lse, void* workspace,
                             size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    const std::string who = "cp_attn_paged: ";
    if (!kv) return fail(CP_ERR_INVALID, who + "kv is NULL");
    PagedParams p;
    std::memset(&p, 0, sizeof(p));
    int st = set_common(&p, who, n_heads_q, kv->n_heads_kv, head_dim, softmax_scale, window, n_sink);
    if (st != CP_OK) return st;
    st = check_rows(who, kv->n_seqs, n_rows, q_start == nullptr, &max_q, p.G);
    if (st != CP_OK) return st;
    if (q_stride != 0 && (q_stride < (int64_t)n_heads_q * kHeadDim || q_stride % 8))
      return fail(CP_ERR_INVALID, who + "q_stride must be 0 or a multiple of 8 that holds a row");
    if (kv->n_blocks < 0 || kv->table_stride < 0) return fail(CP_ERR_INVALID, who + "n_blocks or table_stride < 0");
    if (n_rows == 0 || kv->n_seqs == 0) {
      clear_error();
      return CP_OK;
    }
    if (!q || !o || !kv->k_cache || !kv->v_cache || !kv->tables || !kv->kv_len)
      return fail(CP_ERR_INVALID, who + "q, o, caches, tables and kv_len are required");
    if (!aligned(q, 16) || !aligned(o, 16) || !aligned(kv->k_cache, 16) || !aligned(kv->v_cache, 16) ||
        !aligned(kv->tables, 4) || !aligned(kv->kv_len, 4) || !aligned(q_start, 4) || !aligned(lse, 4))
      return fail(CP_ERR_INVALID, who + "q, o and the caches must be 16-byte, the other arrays 4-byte aligned");
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.q_stride = q_stride ? q_stride : (int64_t)n_heads_q * kHeadDim;
    p.n_rows = n_rows;
    p.k_cache = static_cast<const unsigned char*>(kv->k_cache);
    p.v_cache = static_cast<const unsigned char*>(kv->v_cache);
    p.n_blocks = (int32_t)std::min<int64_t>(INT32_MAX, kv->n_blocks);
    p.tables = kv->tables;
    p.table_stride = kv->table_stride;
    p.table_len = (int32_t)std::min<int64_t>(INT32_MAX, kv->table_stride);
    p.streamed = kv->n_blocks > kInfinityCacheBytes / (2 * kBlockTokens * p.kv_stride);
    p.paged_end = INT32_MAX;
    p.key_end = (int32_t)(std::min<int64_t>(kMaxTokens / kBlockTokens, kv->table_stride) * kBlockTokens);
    p.n_segments = kv->n_seqs;
    p.q_start = q_start;
    p.kv_len = kv->kv_len;
    p.uniform_q = q_start ? 0 : (int32_t)max_q;
    st = launch(&p, who, max_q, workspace, workspace_bytes, stream);
    if (st == CP_OK) clear_error();
    return st;
  });
}

extern "C" size_t cp_attn_window_workspace_size(const cp_rank_plan* plan, int32_t n_heads_q, int32_t n_heads_kv) {
  size_t total = 0;
  const int st = guarded([&]() -> int {
    const std::string who = "cp_attn_window_workspace_size: ";
    if (!plan) return fail(CP_ERR_INVALID, who + "plan is NULL");
    const int s = check_heads(n_heads_q, n_heads_kv, who);
    if (s != CP_OK) return s;
    if (plan->n_rows > 0) total = workspace_bytes_of(plan->n_rows, plan->chunk_len, n_heads_q, n_heads_q / n_heads_kv);
    return CP_OK;
  });
  if (st != CP_OK) return 0;
  clear_error();
  return total;
}

extern "C" int cp_attn_window(const cp_rank_plan* plan, const void* q, const void* k_new, const void* v_new,
                              const void* k_cache, const void* v_cache, int64_t n_blocks, const int32_t* block_table,
                              int64_t table_len, int32_t n_heads_q, int32_t n_heads_kv, int32_t head_dim,
                              float softmax_scale, int64_t window, int64_t n_sink, void* o, float* lse,
                              int32_t out_order, void* workspace, size_t workspace_bytes, void* stream) {
  return guarded([&]() -> int {
    const std::string who = "cp_attn_window: ";
    if (!plan) return fail(CP_ERR_INVALID, who + "plan is NULL");
    cp_rank_plan ref;
    if (make_plan(plan->prefix_len, plan->new_len, plan->C, plan->rank, &ref) != CP_OK || !plan_equal(ref, *plan))
      return fail(CP_ERR_INVALID, who + "plan does not match cp_shard_plan");
    PagedParams p;
    std::memset(&p, 0, sizeof(p));
    int st = set_common(&p, who, n_heads_q, n_heads_kv, head_dim, softmax_scale, window, n_sink);
    if (st != CP_OK) return st;
    const int64_t P = plan->prefix_len, R = plan->new_len;
    if (P + R > kMaxTokens) return fail(CP_ERR_UNSUPPORTED, who + "sequence beyond 2^30 tokens");
    if (plan->n_rows * p.G > INT32_MAX) return fail(CP_ERR_UNSUPPORTED, who + "too many rows");
    if (out_order != CP_OUT_LOCAL && out_order != CP_OUT_SEQUENCE)
      return fail(CP_ERR_INVALID, who + "out_order must be CP_OUT_LOCAL or CP_OUT_SEQUENCE");
    if (n_blocks < 0 || table_len < 0) return fail(CP_ERR_INVALID, who + "n_blocks or table_len < 0");
    if (P % CP_KV_BLOCK_TOKENS) return fail(CP_ERR_INVALID, who + "prefix_len must be a multiple of 16");
    if (plan->n_rows == 0) {
      clear_error();
      return CP_OK;
    }
    if (!q || !k_new || !v_new || !o) return fail(CP_ERR_INVALID, who + "q, k_new, v_new and o are required");
    if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(o, 16) || !aligned(lse, 4))
      return fail(CP_ERR_INVALID, who + "q, k_new, v_new and o must be 16-byte and lse 4-byte aligned");
    if (P > 0) {
      if (!k_cache || !v_cache || !block_table)
        return fail(CP_ERR_INVALID, who + "k_cache, v_cache and block_table are required");
      if (!aligned(k_cache, 16) || !aligned(v_cache, 16) || !aligned(block_table, 4))
        return fail(CP_ERR_INVALID, who + "k_cache/v_cache must be 16-byte and block_table 4-byte aligned");
      if (table_len < P / CP_KV_BLOCK_TOKENS) return fail(CP_ERR_INVALID, who + "block table shorter than P / 16");
    }
    p.q = static_cast<const uint16_t*>(q);
    p.o = static_cast<uint16_t*>(o);
    p.lse = lse;
    p.q_stride = (int64_t)n_heads_q * kHeadDim;
    p.n_rows = plan->n_rows;
    p.k_cache = static_cast<const unsigned char*>(k_cache);
    p.v_cache = static_cast<const unsigned char*>(v_cache);
    p.n_blocks = (int32_t)std::min<int64_t>(INT32_MAX, n_blocks);
    p.tables = block_table;
    p.table_len = (int32_t)(P / CP_KV_BLOCK_TOKENS);
    p.paged_end = (int32_t)P;
    p.key_end = kMaxTokens;
    p.k_new = static_cast<const unsigned char*>(k_new);
    p.v_new = static_cast<const unsigned char*>(v_new);
    p.n_chunks = p.n_segments = 2;
    for (int c = 0; c < 2; ++c) {
      const cp_chunk& x = plan->chunk[c];
      p.chunk_len[c] = (int32_t)x.q_len;
      p.chunk_pos[c] = (int32_t)x.q_begin;
      p.chunk_row[c] = x.local_offset;
      p.chunk_out[c] = out_order == CP_OUT_SEQUENCE ? x.q_begin - P : x.local_offset;
    }
    st = launch(&p, who, plan->chunk_len, workspace, workspace_bytes, stream);
    if (st == CP_OK) clear_error();
    return st;
  });
}
