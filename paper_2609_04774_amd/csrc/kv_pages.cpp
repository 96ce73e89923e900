// Host side of the calls on the pages of a cache: argument checks and kernel
// parameters for cp_kv_append, cp_kv_copy_pages, cp_kv_reserve, cp_kv_fork,
// cp_kv_free and cp_kv_compact (include/cp_attn.h).
#include <cstring>
#include <string>

#include "paged.h"

using namespace cpattn;

namespace {

bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

int check_pool(const cp_kv_pool* pool, const std::string& who) {
  if (!pool) return fail(CP_ERR_INVALID, who + "pool is NULL");
  if (pool->n_seqs < 0 || pool->table_stride < 0 || pool->n_blocks < 0)
    return fail(CP_ERR_INVALID, who + "n_seqs, table_stride or n_blocks < 0");
  if (pool->n_blocks > INT32_MAX) return fail(CP_ERR_UNSUPPORTED, who + "more than 2^31 - 1 pages");
  if (pool->reserved != 0) return fail(CP_ERR_INVALID, who + "reserved must be 0");
  if ((pool->n_seqs > 0 && (!pool->kv_len || (pool->table_stride > 0 && !pool->tables))) ||
      (pool->n_blocks > 0 && !pool->refs))
    return fail(CP_ERR_INVALID, who + "tables, kv_len and refs are required");
  if (!aligned(pool->tables, 4) || !aligned(pool->kv_len, 4) || !aligned(pool->refs, 4))
    return fail(CP_ERR_INVALID, who + "tables, kv_len and refs must be 4-byte aligned");
  return CP_OK;
}

int check_list(int64_t n, const std::string& who) {
  if (n < 0) return fail(CP_ERR_INVALID, who + "n < 0");
  if (n > CP_KV_MAX_LIST) return fail(CP_ERR_UNSUPPORTED, who + "more than 4096 entries");
  return CP_OK;
}

int set_caches(CacheSet* c, void* const* caches, int32_t n, int64_t n_blocks, int64_t page_bytes, int least,
               const std::string& who) {
  std::memset(c, 0, sizeof(*c));
  if (n < least || n > CP_KV_MAX_CACHES)
    return fail(CP_ERR_INVALID, who + "n_caches must be " + std::to_string(least) + "..256");
  if (n_blocks < 0) return fail(CP_ERR_INVALID, who + "n_blocks < 0");
  if (n > 0 && !caches) return fail(CP_ERR_INVALID, who + "caches is NULL");
  if (n > 0 && (page_bytes <= 0 || page_bytes % 16))
    return fail(CP_ERR_INVALID, who + "page_bytes must be a positive multiple of 16");
  for (int i = 0; i < n; ++i) {
    if (n_blocks > 0 && (!caches[i] || !aligned(caches[i], 16)))
      return fail(CP_ERR_INVALID, who + "cache " + std::to_string(i) + " is NULL or not 16-byte aligned");
    c->cache[i] = static_cast<unsigned char*>(caches[i]);
  }
  c->n = n;
  c->n_blocks = n_blocks;
  c->page_bytes = page_bytes;
  return CP_OK;
}

int arrays(std::initializer_list<const void*> ptrs, const std::string& who, const char* what) {
  for (const void* x : ptrs)
    if (!x || !aligned(x, 4)) return fail(CP_ERR_INVALID, who + what + " are required, 4-byte aligned");
  return CP_OK;
}

template <class F>
int run(F&& body) {
  return guarded([&]() -> int {
    const int st = body();
    if (st == CP_OK) clear_error();
    return st;
  });
}

}  // namespace

extern "C" int cp_kv_append(const cp_paged_kv* kv, const void* k_rows, const void* v_rows, int64_t k_stride,
                            int64_t v_stride, int64_t n_rows, const int32_t* q_start, int32_t head_dim, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_append: ";
    if (!kv) return fail(CP_ERR_INVALID, who + "kv is NULL");
    if (kv->n_heads_kv < 1 || head_dim < 8 || head_dim % 8)
      return fail(CP_ERR_INVALID, who + "n_heads_kv must be >= 1 and head_dim a positive multiple of 8");
    if (kv->n_seqs < 0 || n_rows < 0 || kv->n_blocks < 0 || kv->table_stride < 0)
      return fail(CP_ERR_INVALID, who + "n_seqs, n_rows, n_blocks or table_stride < 0");
    if (n_rows > kMaxTokens) return fail(CP_ERR_UNSUPPORTED, who + "more than 2^30 rows");
    const int64_t row = (int64_t)kv->n_heads_kv * head_dim;
    for (int64_t x : {k_stride, v_stride})
      if (x != 0 && (x < row || x % 8))
        return fail(CP_ERR_INVALID, who + "strides must be 0 or multiples of 8 that hold a row");
    if (n_rows == 0 || kv->n_seqs == 0) return CP_OK;
    if (!q_start && n_rows % kv->n_seqs)
      return fail(CP_ERR_INVALID, who + "without q_start n_rows must be a multiple of n_seqs");
    if (!k_rows || !v_rows || !kv->k_cache || !kv->v_cache || !kv->tables || !kv->kv_len)
      return fail(CP_ERR_INVALID, who + "rows, caches, tables and kv_len are required");
    if (!aligned(k_rows, 16) || !aligned(v_rows, 16) || !aligned(kv->k_cache, 16) || !aligned(kv->v_cache, 16) ||
        !aligned(kv->tables, 4) || !aligned(kv->kv_len, 4) || !aligned(q_start, 4))
      return fail(CP_ERR_INVALID, who + "rows and caches must be 16-byte, the other arrays 4-byte aligned");
    AppendParams p;
    std::memset(&p, 0, sizeof(p));
    p.k_rows = static_cast<const unsigned char*>(k_rows);
    p.v_rows = static_cast<const unsigned char*>(v_rows);
    p.k_stride = 2 * (k_stride ? k_stride : row);
    p.v_stride = 2 * (v_stride ? v_stride : row);
    p.n_rows = n_rows;
    p.row_bytes = 2 * row;
    p.k_cache = static_cast<unsigned char*>(kv->k_cache);
    p.v_cache = static_cast<unsigned char*>(kv->v_cache);
    p.n_blocks = kv->n_blocks;
    p.tables = kv->tables;
    p.table_stride = kv->table_stride;
    p.kv_len = kv->kv_len;
    p.q_start = q_start;
    p.n_seqs = kv->n_seqs;
    p.uniform_q = q_start ? 1 : (int32_t)(n_rows / kv->n_seqs);
    return launch_append(p, stream);
  });
}

extern "C" int cp_kv_copy_pages(void* const* caches, int32_t n_caches, int64_t n_blocks, int64_t page_bytes,
                                const int32_t* src, const int32_t* dst, int64_t n, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_copy_pages: ";
    CacheSet c;
    int st = set_caches(&c, caches, n_caches, n_blocks, page_bytes, 1, who);
    if (st != CP_OK) return st;
    if (n < 0) return fail(CP_ERR_INVALID, who + "n < 0");
    if (n == 0 || n_blocks == 0) return CP_OK;
    st = arrays({src, dst}, who, "src and dst");
    if (st != CP_OK) return st;
    return launch_copy_pages(c, src, dst, n, stream);
  });
}

extern "C" int cp_kv_reserve(const cp_kv_pool* pool, const int32_t* seqs, const int32_t* add, int64_t n,
                             int32_t* missing, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_reserve: ";
    int st = check_pool(pool, who);
    if (st == CP_OK) st = check_list(n, who);
    if (st == CP_OK) st = arrays({missing}, who, "missing");
    if (st == CP_OK && n > 0) st = arrays({seqs, add}, who, "seqs and add");
    if (st != CP_OK) return st;
    return launch_reserve(*pool, seqs, add, (int32_t)n, missing, stream);
  });
}

extern "C" int cp_kv_fork(const cp_kv_pool* pool, void* const* caches, int32_t n_caches, int64_t page_bytes,
                          const int32_t* parents, const int32_t* children, int64_t n, int32_t* missing, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_fork: ";
    int st = check_pool(pool, who);
    CacheSet c;
    if (st == CP_OK) st = set_caches(&c, caches, n_caches, pool->n_blocks, page_bytes, 0, who);
    if (st == CP_OK) st = check_list(n, who);
    if (st == CP_OK) st = arrays({missing}, who, "missing");
    if (st == CP_OK && n > 0) st = arrays({parents, children}, who, "parents and children");
    if (st != CP_OK) return st;
    return launch_fork(*pool, c, parents, children, (int32_t)n, missing, stream);
  });
}

extern "C" int cp_kv_free(const cp_kv_pool* pool, const int32_t* seqs, const int32_t* begin, const int32_t* end,
                          int64_t n, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_free: ";
    int st = check_pool(pool, who);
    if (st == CP_OK) st = check_list(n, who);
    if (st != CP_OK || n == 0) return st;
    st = arrays({seqs, begin, end}, who, "seqs, begin and end");
    if (st != CP_OK) return st;
    return launch_free(*pool, seqs, begin, end, (int32_t)n, stream);
  });
}

extern "C" size_t cp_kv_compact_workspace_size(int64_t n_blocks) {
  if (n_blocks < 0 || n_blocks > INT32_MAX) {
    (void)fail_static(CP_ERR_INVALID, "cp_kv_compact_workspace_size: n_blocks out of range");
    return 0;
  }
  clear_error();
  return compact_ints(n_blocks) * 4;
}

extern "C" int cp_kv_compact(const cp_kv_pool* pool, void* const* caches, int32_t n_caches, int64_t page_bytes,
                             void* workspace, size_t workspace_bytes, void* stream) {
  return run([&]() -> int {
    const std::string who = "cp_kv_compact: ";
    int st = check_pool(pool, who);
    CacheSet c;
    if (st == CP_OK) st = set_caches(&c, caches, n_caches, pool->n_blocks, page_bytes, 0, who);
    if (st != CP_OK || pool->n_blocks == 0) return st;
    if (!workspace || !aligned(workspace, 256))
      return fail(CP_ERR_INVALID, who + "workspace is NULL or not 256-byte aligned");
    const size_t need = compact_ints(pool->n_blocks) * 4;
    if (workspace_bytes < need) return fail(CP_ERR_CAPACITY, who + "workspace needs " + std::to_string(need) + " bytes");
    return launch_compact(*pool, c, static_cast<int32_t*>(workspace), stream);
  });
}
