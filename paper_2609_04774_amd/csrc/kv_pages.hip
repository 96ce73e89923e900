// The pages of a cache: a ragged batch's new rows stored at any position, pages
// copied, reserved, shared with new sequences, given back and moved to the front
// of the pool (Sec. 2.2, 7.1, 8).  Rows and pages are copied, never computed: all
// of it is exact.
//
// The copies are bound by HBM (each byte read once and written once); the calls
// that only change tables are bound by latency, and are one launch each.  Free
// pages are given lowest first, found by one workgroup that scans the reference
// counts 8192 at a time, so that which page a sequence gets never depends on
// timing.
//
// Measured: 20.7K rows of 8 heads appended 28 us, 6.1 TB/s, 64 rows 3.1; 64 sequences
// forked off 8, with 56 pages copied in 8 caches, 13 us to find the pages and 8 for the
// tables and copies; 128 sequences' pages freed 4.8; 1000 pages of 8 caches moved, 526 MB,
// 8 us for the list and 96 for the moves, 5.5 TB/s.  A token of 64 sequences reserved 6 to
// 8 us where no page is needed; where all need one and all but the last 2048 pages are in
// use, 14 of a pool of 4096 pages, 28 of 32768 and 85 of 131072: the search passes over the
// pages in use, 8192 in about 5 us.
#include <hip/hip_runtime.h>

#include "paged.h"

namespace cpattn {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kScanThreads = 1024;
constexpr int kScanWaves = kScanThreads / 64;

// ---------------------------------------------------------------------------
// Append.  kLanes lanes move a row of K and V, 16 bytes each at a time.  The row's
// sequence is found in q_start by bisection (its entries are in a cache after the
// first rows).
template <int kLanes>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p) {
  const int64_t t = p.first_row + (int64_t)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes;
  if (t >= p.n_rows) return;
  int s;
  int64_t end;
  if (p.q_start) {
    if (t < p.q_start[0] || t >= p.q_start[p.n_seqs]) return;
    int lo = 0, hi = p.n_seqs;  // q_start[lo] <= t < q_start[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.q_start[mid] <= t)
        lo = mid;
      else
        hi = mid;
    }
    s = lo;
    end = p.q_start[hi];
  } else {
    s = (int)(t / p.uniform_q);
    end = (int64_t)(s + 1) * p.uniform_q;
  }
  int len = p.kv_len[s];
  len = len < 0 ? 0 : (len > kMaxTokens ? kMaxTokens : len);
  const int64_t pos = len - (end - t);
  if (pos < 0 || pos / kBlockTokens >= p.table_stride) return;
  const int64_t page = p.tables[s * p.table_stride + pos / kBlockTokens];
  if (page < 0 || page >= p.n_blocks) return;
  const int64_t dst = (page * kBlockTokens + pos % kBlockTokens) * p.row_bytes;
  const u32x4* k = reinterpret_cast<const u32x4*>(p.k_rows + t * p.k_stride);
  const u32x4* v = reinterpret_cast<const u32x4*>(p.v_rows + t * p.v_stride);
  const int64_t n = p.row_bytes >> 4;
  constexpr int kPieces = 2;
  for (int64_t i0 = threadIdx.x % kLanes; i0 < n; i0 += kPieces * kLanes) {
    u32x4 x[kPieces], y[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (i0 + j * kLanes < n) {
        x[j] = k[i0 + j * kLanes];
        y[j] = v[i0 + j * kLanes];
      }
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (i0 + j * kLanes < n) {
        __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4*>(p.k_cache + dst) + i0 + j * kLanes);
        __builtin_nontemporal_store(y[j], reinterpret_cast<u32x4*>(p.v_cache + dst) + i0 + j * kLanes);
      }
  }
}

// ---------------------------------------------------------------------------
// A page copied by a workgroup, eight loads of 16 bytes in flight per thread.
__device__ __forceinline__ void copy_page(const unsigned char* src, unsigned char* dst, int64_t bytes) {
  constexpr int kPieces = 8;
  const int64_t n = bytes >> 4;
  for (int64_t i0 = threadIdx.x; i0 < n; i0 += kPieces * kThreads) {
    u32x4 x[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (i0 + j * kThreads < n)
        x[j] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(src) + i0 + j * kThreads);
#pragma unroll
    for (int j = 0; j < kPieces; ++j)
      if (i0 + j * kThreads < n)
        __builtin_nontemporal_store(x[j], reinterpret_cast<u32x4*>(dst) + i0 + j * kThreads);
  }
}

__device__ __forceinline__ bool in_pool(int64_t page, int64_t n_blocks) { return page >= 0 && page < n_blocks; }

__global__ __launch_bounds__(kThreads) void copy_pages_kernel(CacheSet c, const int32_t* src, const int32_t* dst,
                                                              int64_t n) {
  unsigned char* cache = c.cache[blockIdx.y];
  for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
    const int64_t a = src[i], b = dst[i];
    if (in_pool(a, c.n_blocks) && in_pool(b, c.n_blocks) && a != b)
      copy_page(cache + a * c.page_bytes, cache + b * c.page_bytes, c.page_bytes);
  }
}

// ---------------------------------------------------------------------------
// Sums over a workgroup of kScanThreads.
struct Scan {
  int64_t before, total;  // of the threads before this one, and of all
};

__device__ Scan scan(int64_t mine, int64_t* wave_sum) {
  int64_t x = mine;
#pragma unroll
  for (int k = 1; k < 64; k *= 2) {
    const int64_t y = __shfl_up(x, k);
    if ((int)(threadIdx.x & 63) >= k) x += y;
  }
  __syncthreads();  // wave_sum may still be read from the last scan
  if ((threadIdx.x & 63) == 63) wave_sum[threadIdx.x >> 6] = x;
  __syncthreads();
  int64_t total = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) {
    if (w < (int)(threadIdx.x >> 6)) x += wave_sum[w];
    total += wave_sum[w];
  }
  return Scan{x - mine, total};
}

__device__ __forceinline__ int clamp_len(int len) { return len < 0 ? 0 : (len > kMaxTokens ? kMaxTokens : len); }
__device__ __forceinline__ int64_t pages_of(int64_t len) { return (len + kBlockTokens - 1) / kBlockTokens; }

// What entry i of a list asks for: n pages, for the table entries of sequence seq
// from `first` on, and the length that it then has.
struct Want {
  int32_t seq, n;  // n < 0: nothing can be done for it; seq < 0: passed over
  int32_t len;
  int64_t first;
};

// Whether one of the first n entries of a list in LDS (16-byte aligned, readable up to
// the next multiple of 8) is x.
__device__ __forceinline__ bool named(const int32_t* list, int n, int x) {
  bool hit = false;
  for (int i = 0; i < n; i += 8) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(list + i), b = *reinterpret_cast<const i32x4*>(list + i + 4);
#pragma unroll
    for (int k = 0; k < 4; ++k) hit |= ((a[k] == x) & (i + k < n)) | ((b[k] == x) & (i + 4 + k < n));
  }
  return hit;
}

struct ReserveList {
  const int32_t* seqs;
  const int32_t* add;
  __device__ Want operator()(const cp_kv_pool& p, const int32_t* list, const int32_t*, int i) const {
    Want w{-1, 0, 0, 0};
    const int s = list[i];
    if (s < 0 || s >= p.n_seqs || named(list, i, s)) return w;
    w.seq = s;
    const int64_t len = clamp_len(p.kv_len[s]), to = len + add[i];
    w.first = pages_of(len);
    w.n = add[i] < 0 || to > kMaxTokens || pages_of(to) > p.table_stride ? -1 : (int32_t)(pages_of(to) - w.first);
    // The first new tokens belong into the last page.  If it was given back, they have no
    // place: a fresh page would show another request's tokens before them.
    if (w.n >= 0 && add[i] > 0 && len % kBlockTokens && !in_pool(p.tables[s * p.table_stride + w.first - 1], p.n_blocks))
      w.n = -1;
    w.len = (int32_t)to;
    return w;
  }
};

struct ForkList {
  const int32_t* seqs;  // the children
  const int32_t* parents;
  __device__ Want operator()(const cp_kv_pool& p, const int32_t* list, const int32_t* second, int i) const {
    Want w{-1, 0, 0, 0};
    const int c = list[i], a = second[i];
    if (c < 0 || c >= p.n_seqs || a < 0 || a >= p.n_seqs || named(list, i, c)) return w;
    w.seq = c;
    const int len = clamp_len(p.kv_len[a]);
    w.first = len / kBlockTokens;
    const bool part = len % kBlockTokens != 0;  // of a page, to be copied
    w.n = pages_of(len) > p.table_stride || (part && !in_pool(p.tables[a * p.table_stride + w.first], p.n_blocks)) ? -1 : part;
    w.len = len;
    return w;
  }
};

// One workgroup gives the lowest free pages to the wants of a list, in its order.
// kFork: a child that is also a parent is left alone (the sharing of its pages
// would depend on timing).
template <class List, bool kFork>
__global__ __launch_bounds__(kScanThreads) void take_pages_kernel(cp_kv_pool p, List list, int n, int32_t* missing) {
  __shared__ __attribute__((aligned(16))) int32_t seqs[CP_KV_MAX_LIST], second[kFork ? CP_KV_MAX_LIST : 4];
  __shared__ int64_t need_end[CP_KV_MAX_LIST];  // pages that the entries up to this one want
  __shared__ int32_t first_of[CP_KV_MAX_LIST];  // table entry of an entry's first page
  __shared__ int64_t wave_sum[kScanWaves];
  __shared__ int32_t n_missing;
  const int tid = threadIdx.x;
  // Which of kEach pages from `at` on are free.  The first are looked up at once, while
  // the lists are read.
  constexpr int kEach = 8;
  auto free_from = [&](int64_t at) {
    int32_t refs[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) refs[j] = at + j < p.n_blocks ? p.refs[at + j] : 1;
    uint32_t free = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) free |= (uint32_t)(refs[j] == 0) << j;
    return free;
  };
  uint32_t free = free_from((int64_t)tid * kEach);
  for (int i = tid; i < n; i += kScanThreads) {
    seqs[i] = list.seqs[i];
    if constexpr (kFork) second[i] = list.parents[i];
  }
  if (tid == 0) n_missing = 0;
  __syncthreads();
  const int per = (n + kScanThreads - 1) / kScanThreads;  // at most CP_KV_MAX_LIST / kScanThreads
  constexpr int kPer = CP_KV_MAX_LIST / kScanThreads;
  Want w[kPer];
  bool refused[kPer];
  int64_t mine = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = tid * per + k;
    w[k].seq = -1;
    w[k].n = 0;
    refused[k] = false;
    if (k >= per || i >= n) continue;
    w[k] = list(p, seqs, second, i);
    refused[k] = w[k].seq >= 0 && w[k].n < 0;
    if (kFork && w[k].seq >= 0 && named(second, n, w[k].seq)) {
      refused[k] = true;
      w[k].seq = -2;  // a parent: unchanged
    }
    if (refused[k]) w[k].n = 0;
    mine += w[k].n;
  }
  const Scan s = scan(mine, wave_sum);
  int64_t end = s.before;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = tid * per + k;
    if (k >= per || i >= n) continue;
    end += w[k].n;
    need_end[i] = end;
    first_of[i] = (int32_t)w[k].first;
  }
  __syncthreads();
  // Pages of rank 0 .. total - 1 among the free ones, each into its entry.
  const int64_t total = s.total;
  int64_t found = 0;
  for (int64_t base = 0; base < p.n_blocks && found < total; base += (int64_t)kScanThreads * kEach) {
    const int64_t at = base + (int64_t)tid * kEach;
    if (base > 0) free = free_from(at);
    const Scan f = scan(__builtin_popcount(free), wave_sum);
    int64_t rank = found + f.before;
    while (free && rank < total) {
      const int64_t page = at + __builtin_ctz(free);
      free &= free - 1;
      int lo = 0, hi = n - 1;  // the first entry whose pages end behind this rank
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (need_end[mid] > rank)
          hi = mid;
        else
          lo = mid + 1;
      }
      // Its first page's rank is the end of the entry before.
      const int64_t k = rank - (lo ? need_end[lo - 1] : 0);
      p.tables[seqs[lo] * p.table_stride + first_of[lo] + k] = (int32_t)page;
      p.refs[page] = 1;
      ++rank;
    }
    found += f.total;
  }
  __syncthreads();  // every length has been read
  // An entry that was not served whole gives its pages back.
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int i = tid * per + k;
    if (k >= per || i >= n || w[k].seq == -1) continue;
    bool served = !refused[k];
    if (served && w[k].n > 0 && need_end[i] > found) {
      served = false;
      const int64_t rank0 = need_end[i] - w[k].n;
      for (int64_t j = 0; j < w[k].n && rank0 + j < found; ++j) {
        int32_t* entry = p.tables + w[k].seq * p.table_stride + w[k].first + j;
        p.refs[*entry] = 0;
        *entry = -1;
      }
    }
    if (!served) atomicAdd(&n_missing, 1);
    if (w[k].seq >= 0) {
      if (served)
        p.kv_len[w[k].seq] = w[k].len;
      else if (kFork)
        p.kv_len[w[k].seq] = 0;
    }
  }
  __syncthreads();
  if (tid == 0) *missing = n_missing;
}

// The child's table, the counts of the pages that it shares (block y == 0), and the
// copy of a page filled in part in cache y - 1 (as many blocks as caches).
__global__ __launch_bounds__(kThreads) void fork_kernel(cp_kv_pool p, CacheSet c, const int32_t* parents,
                                                        const int32_t* children, int n) {
  const int i = blockIdx.x;
  const int a = parents[i], b = children[i];
  if (a < 0 || a >= p.n_seqs || b < 0 || b >= p.n_seqs) return;
  // As take_pages_kernel decides: a child named before, or a parent.
  bool skip = false;
  for (int j = threadIdx.x; j < n; j += kThreads) skip |= (j < i && children[j] == b) || parents[j] == b;
  if (__syncthreads_or(skip)) return;
  const int len = p.kv_len[b];  // the parent's, or 0 where it got nothing
  const int64_t whole = len / kBlockTokens;
  const int32_t* from = p.tables + a * p.table_stride;
  int32_t* to = p.tables + b * p.table_stride;
  if (blockIdx.y == 0) {
    for (int64_t j = threadIdx.x; j < p.table_stride; j += kThreads) {
      if (j < whole) {
        const int32_t page = from[j];
        to[j] = page;
        if (in_pool(page, p.n_blocks)) atomicAdd(p.refs + page, 1);
      } else if (j > whole || len % kBlockTokens == 0) {
        to[j] = -1;
      }
    }
  } else if (len % kBlockTokens) {
    const int64_t src = from[whole], dst = to[whole];
    unsigned char* cache = c.cache[blockIdx.y - 1];
    if (in_pool(src, p.n_blocks) && in_pool(dst, p.n_blocks))
      copy_page(cache + src * c.page_bytes, cache + dst * c.page_bytes, c.page_bytes);
  }
}

__global__ __launch_bounds__(kThreads) void free_kernel(cp_kv_pool p, const int32_t* seqs, const int32_t* begin,
                                                        const int32_t* end) {
  const int i = blockIdx.x;
  const int s = seqs[i];
  if (s < 0 || s >= p.n_seqs) return;
  bool again = false;
  for (int j = threadIdx.x; j < i; j += kThreads) again |= seqs[j] == s;
  if (__syncthreads_or(again)) return;
  const int64_t len = clamp_len(p.kv_len[s]), lo = begin[i], hi = end[i];
  int64_t stop = pages_of(len);
  stop = stop < p.table_stride ? stop : p.table_stride;
  int64_t j0 = lo <= 0 ? 0 : pages_of(lo);
  for (int64_t j = j0 + threadIdx.x; j < stop; j += kThreads) {
    const int64_t last = (j + 1) * kBlockTokens < len ? (j + 1) * kBlockTokens : len;
    if (last > hi) break;
    int32_t* entry = p.tables + s * p.table_stride + j;
    const int32_t page = *entry;
    if (page == -1) continue;
    *entry = -1;
    if (in_pool(page, p.n_blocks)) atomicSub(p.refs + page, 1);
  }
  if (lo <= 0 && hi >= len) {
    __syncthreads();
    if (threadIdx.x == 0) p.kv_len[s] = 0;
  }
}

// ---------------------------------------------------------------------------
// Compaction: one workgroup lists the moves, then every block moves pages or
// rewrites table entries.
struct CompactWork {
  int32_t* count;
  int32_t* src;  // and dst: at most n_blocks / 2 moves
  int32_t* dst;
  int32_t* to;   // a page's new place
  __host__ __device__ CompactWork(int32_t* w, int64_t n) : count(w), src(w + 64), dst(w + 64 + n / 2), to(w + 64 + 2 * (n / 2)) {}
};

__global__ __launch_bounds__(kScanThreads) void compact_list_kernel(cp_kv_pool p, int32_t* work) {
  __shared__ int64_t wave_sum[kScanWaves];
  const CompactWork w(work, p.n_blocks);
  int64_t live = 0;
  for (int64_t i = threadIdx.x; i < p.n_blocks; i += kScanThreads) live += p.refs[i] > 0;
  const int64_t n_live = scan(live, wave_sum).total;
  // The k-th page in use behind the first n_live goes to the k-th free one of them:
  // there are as many of either.
  constexpr int kEach = 8;
  int64_t n_src = 0, n_dst = 0;
  for (int64_t base = 0; base < p.n_blocks; base += (int64_t)kScanThreads * kEach) {
    const int64_t at = base + (int64_t)threadIdx.x * kEach;
    uint32_t leave = 0, hole = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
      if (at + j >= p.n_blocks) continue;
      const bool used = p.refs[at + j] > 0;
      if (used && at + j >= n_live) leave |= 1u << j;
      if (!used && at + j < n_live) hole |= 1u << j;
      w.to[at + j] = (int32_t)(at + j);
    }
    const Scan s = scan((int64_t)__builtin_popcount(leave) << 32 | __builtin_popcount(hole), wave_sum);
    int64_t a = n_src + (s.before >> 32), b = n_dst + (s.before & 0xffffffff);
    for (; leave; leave &= leave - 1) w.src[a++] = (int32_t)(at + __builtin_ctz(leave));
    for (; hole; hole &= hole - 1) w.dst[b++] = (int32_t)(at + __builtin_ctz(hole));
    n_src += s.total >> 32;
    n_dst += s.total & 0xffffffff;
  }
  __syncthreads();
  for (int64_t k = threadIdx.x; k < n_src; k += kScanThreads) w.to[w.src[k]] = w.dst[k];
  if (threadIdx.x == 0) *w.count = (int32_t)n_src;
}

// Blocks of row 0 rewrite tables and counts, those of row y the pages of cache y - 1.
__global__ __launch_bounds__(kThreads) void compact_kernel(cp_kv_pool p, CacheSet c, int32_t* work) {
  const CompactWork w(work, p.n_blocks);
  const int64_t n = *w.count;
  if (blockIdx.y == 0) {
    const int64_t first = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
    for (int64_t i = first; i < (int64_t)p.n_seqs * p.table_stride; i += step) {
      const int32_t page = p.tables[i];
      if (in_pool(page, p.n_blocks)) p.tables[i] = w.to[page];
    }
    for (int64_t k = first; k < n; k += step) {
      p.refs[w.dst[k]] = p.refs[w.src[k]];
      p.refs[w.src[k]] = 0;
    }
    return;
  }
  unsigned char* cache = c.cache[blockIdx.y - 1];
  for (int64_t k = blockIdx.x; k < n; k += gridDim.x)
    copy_page(cache + w.src[k] * c.page_bytes, cache + w.dst[k] * c.page_bytes, c.page_bytes);
}

int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CP_OK : fail(CP_ERR_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
}

// Blocks of one row of a grid that copies up to `pages` pages in each of n caches:
// about 4096 in all, eight resident on a compute unit and as many waiting.
unsigned page_blocks(int64_t pages, int n) {
  const int64_t most = 4096 / (n > 0 ? n : 1) + 1;
  return (unsigned)(pages < most ? (pages > 0 ? pages : 1) : most);
}

}  // namespace

// A launch holds fewer than 2^32 threads: more rows take several.
int launch_append(AppendParams p, void* stream) {
  const int64_t pieces = p.row_bytes >> 4;
  const int lanes = pieces <= 16 ? 16 : pieces <= 32 ? 32 : 64;
  const int64_t per_block = kThreads / lanes, most = (int64_t)1 << 20;
  for (; p.first_row < p.n_rows; p.first_row += most * per_block) {
    const int64_t blocks = (p.n_rows - p.first_row + per_block - 1) / per_block;
    hipLaunchKernelGGL(lanes == 16 ? append_kernel<16> : lanes == 32 ? append_kernel<32> : append_kernel<64>,
                       dim3((unsigned)(blocks < most ? blocks : most)), dim3(kThreads), 0, (hipStream_t)stream, p);
    const int st = launched("cp_kv_append");
    if (st != CP_OK) return st;
  }
  return CP_OK;
}

int launch_copy_pages(const CacheSet& c, const int32_t* src, const int32_t* dst, int64_t n, void* stream) {
  hipLaunchKernelGGL(copy_pages_kernel, dim3(page_blocks(n, c.n), (unsigned)c.n), dim3(kThreads), 0,
                     (hipStream_t)stream, c, src, dst, n);
  return launched("cp_kv_copy_pages");
}

int launch_reserve(const cp_kv_pool& pool, const int32_t* seqs, const int32_t* add, int32_t n, int32_t* missing,
                   void* stream) {
  hipLaunchKernelGGL((take_pages_kernel<ReserveList, false>), dim3(1), dim3(kScanThreads), 0, (hipStream_t)stream, pool,
                     ReserveList{seqs, add}, n, missing);
  return launched("cp_kv_reserve");
}

int launch_fork(const cp_kv_pool& pool, const CacheSet& c, const int32_t* parents, const int32_t* children, int32_t n,
                int32_t* missing, void* stream) {
  hipLaunchKernelGGL((take_pages_kernel<ForkList, true>), dim3(1), dim3(kScanThreads), 0, (hipStream_t)stream, pool,
                     ForkList{children, parents}, n, missing);
  const int st = launched("cp_kv_fork");
  if (st != CP_OK || n == 0) return st;
  hipLaunchKernelGGL(fork_kernel, dim3((unsigned)n, (unsigned)c.n + 1), dim3(kThreads), 0, (hipStream_t)stream, pool, c,
                     parents, children, n);
  return launched("cp_kv_fork");
}

int launch_free(const cp_kv_pool& pool, const int32_t* seqs, const int32_t* begin, const int32_t* end, int32_t n,
                void* stream) {
  hipLaunchKernelGGL(free_kernel, dim3((unsigned)n), dim3(kThreads), 0, (hipStream_t)stream, pool, seqs, begin, end);
  return launched("cp_kv_free");
}

int launch_compact(const cp_kv_pool& pool, const CacheSet& c, int32_t* work, void* stream) {
  hipLaunchKernelGGL(compact_list_kernel, dim3(1), dim3(kScanThreads), 0, (hipStream_t)stream, pool, work);
  const int st = launched("cp_kv_compact");
  if (st != CP_OK) return st;
  hipLaunchKernelGGL(compact_kernel, dim3(page_blocks(pool.n_blocks / 2, c.n + 1), (unsigned)c.n + 1), dim3(kThreads), 0,
                     (hipStream_t)stream, pool, c, work);
  return launched("cp_kv_compact");
}

}  // namespace cpattn
