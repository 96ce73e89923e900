// Building blocks of the attention kernels over a paged cache (attn_rows.hip,
// attn_chunk.hip): where a segment's keys lie, which of them a block of rows
// walks, and 32-key tiles of K and V in LDS as operands of the matrix cores.
#pragma once

#include <hip/hip_runtime.h>

#include <cmath>

#include "paged.h"

namespace cpattn {
namespace tile {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kTileKeys = 32;
constexpr int kRowBytes = kHeadDim * 2;
constexpr int kHalfBytes = kBlockTokens * kRowBytes;  // one page's keys of one head
constexpr int kTileBytes = kTileKeys * kRowBytes;

// Exponents are kept in units of log2.  A running maximum starts at a finite
// value far below any score's: a masked score (-inf) then weighs
// exp2(-inf - kNoMax) = 0 without a special case.
constexpr float kNoMax = -1e30f;
constexpr float kLn2 = 0.69314718055994531f;

// ---------------------------------------------------------------------------
// Segments: consecutive query positions that share their keys -- one sequence
// of a batch, or one chunk of a rank.

struct Segment {
  int64_t q_row;         // its first row in q
  int64_t o_row;         // and in o and lse
  int n;                 // query positions
  int pos0;              // position of the first (negative: it sees no key)
  const int32_t* table;  // pages of its positions
};

// Positions are below 2^30: lengths beyond (or below 0) are contents that the
// host cannot check, and are cut to it.
__device__ __forceinline__ Segment segment_at(const PagedParams& p, int s) {
  Segment x;
  if (p.n_chunks) {
    x.q_row = s ? p.chunk_row[1] : p.chunk_row[0];
    x.o_row = s ? p.chunk_out[1] : p.chunk_out[0];
    x.n = s ? p.chunk_len[1] : p.chunk_len[0];
    x.pos0 = s ? p.chunk_pos[1] : p.chunk_pos[0];
    x.table = p.tables;
    return x;
  }
  const int n_rows = (int)p.n_rows;
  int a = s * p.uniform_q, b = a + p.uniform_q;
  if (p.q_start) {
    a = p.q_start[s];
    b = p.q_start[s + 1];
  }
  a = a < 0 ? 0 : (a > n_rows ? n_rows : a);
  b = b < a ? a : (b > n_rows ? n_rows : b);
  int len = p.kv_len[s];
  len = len < 0 ? 0 : (len > kMaxTokens ? kMaxTokens : len);
  x.q_row = x.o_row = a;
  x.n = b - a < p.max_q ? b - a : p.max_q;
  x.pos0 = len - (b - a);
  x.table = p.tables + (int64_t)s * p.table_stride;
  return x;
}

// Row r of a segment's KV head is query head r % G of position r / G.
// The keys that rows [r0, r1) walk, in tiles of 32: the first tokens that stay
// visible, then the window of the first row up to the last row's position (from
// a page's first key).  Without a window, or where the two meet, all from 0.
struct Walk {
  int end;         // one past the last key that a row sees
  int lo;          // first key of the window of the first row (0: none)
  int sink;        // keys below it are visible to every row behind them
  int p_lo, p_hi;  // positions of the first and the last row
  int n_sink_tiles;
  int base;        // first key of the tiles after the sink tiles
  int n;           // tiles
};

__device__ __forceinline__ Walk walk_of(const PagedParams& p, const Segment& s, int r0, int r1) {
  Walk w;
  w.p_lo = s.pos0 + (int)((unsigned)r0 / (unsigned)p.G);
  w.p_hi = s.pos0 + (int)((unsigned)(r1 - 1) / (unsigned)p.G);
  w.end = w.p_hi + 1 > 0 ? w.p_hi + 1 : 0;
  w.end = w.end < p.key_end ? w.end : p.key_end;
  w.lo = 0;
  w.sink = 0;
  w.n_sink_tiles = 0;
  w.base = 0;
  if (p.window && w.p_lo - p.window + 1 > 0) {
    w.lo = w.p_lo - p.window + 1;
    w.sink = p.n_sink < w.end ? p.n_sink : w.end;
    w.n_sink_tiles = (w.sink + kTileKeys - 1) / kTileKeys;
    w.base = w.lo & ~(kBlockTokens - 1);
    if (w.n_sink_tiles && w.base <= w.n_sink_tiles * kTileKeys) w.n_sink_tiles = w.base = 0;
  }
  w.n = w.n_sink_tiles + (w.end > w.base ? (w.end - w.base + kTileKeys - 1) / kTileKeys : 0);
  return w;
}

__device__ __forceinline__ int tile_begin(const Walk& w, int t) {
  return t < w.n_sink_tiles ? t * kTileKeys : w.base + (t - w.n_sink_tiles) * kTileKeys;
}

// Some row of the block sees key j (no row sees the others: they read as zeros,
// whatever the cache holds there).
__device__ __forceinline__ bool walked(const Walk& w, int j) { return j < w.end && (j >= w.lo || j < w.sink); }

// Every key of the tile at t0 is walked; and every row sees all of them.
__device__ __forceinline__ bool whole_tile(const Walk& w, int t0) {
  return t0 + kTileKeys <= w.end && (t0 >= w.lo || t0 + kTileKeys <= w.sink);
}
__device__ __forceinline__ bool open_tile(const PagedParams& p, const Walk& w, int t0) {
  return t0 + kTileKeys <= w.p_lo + 1 && t0 + kTileKeys <= w.end &&
         (!p.window || t0 > w.p_hi - p.window || t0 + kTileKeys <= p.n_sink);
}

// The run [*first, *end) of tiles that every row sees whole (sink tiles aside).
__device__ __forceinline__ void open_tiles(const PagedParams& p, const Walk& w, int* first, int* end) {
  const int below = p.window ? w.p_hi - p.window + 1 - w.base : 0;  // keys from base on that some row does not see
  const int a = w.n_sink_tiles + (below > 0 ? (below + kTileKeys - 1) / kTileKeys : 0);
  const int keys = (w.p_lo + 1 < w.end ? w.p_lo + 1 : w.end) - w.base;
  const int b = w.n_sink_tiles + (keys > 0 ? keys / kTileKeys : 0);
  *first = a < w.n ? a : w.n;
  *end = b > *first ? b : *first;
}

// ---------------------------------------------------------------------------
// Shares.  The walks of all blocks of rows are counted in steps of kTiles tiles and
// cut into equal shares, one per workgroup.  Blocks are numbered as if every segment
// had as many as the longest may have (the others have no rows and no steps), and
// come in an order (Blocks::run) that gives a workgroup, of a launch of several
// blocks each, blocks far apart: those of neighbouring workgroups then pass over the
// same keys at the same time.  The walks of a block's KV heads follow one another
// (neighbouring workgroups read the same pages: what HBM serves best) or, with
// kHeadsOuter, all blocks of a KV head do (the workgroups of an XCD share their keys in
// its L2).

__device__ __forceinline__ Walk block_walk(const PagedParams& p, const Blocks& b, const Segment& s, int block) {
  const int r0 = block * b.rows;
  const int rows = s.n * p.G;
  return walk_of(p, s, r0, r0 + b.rows < rows ? r0 + b.rows : rows);
}

// Steps of a walk; one at least, which stores the rows of a block without keys.
template <int kTiles>
__device__ __forceinline__ int steps_of(const Walk& w) {
  const int n = (w.n + kTiles - 1) / kTiles;
  return n > 0 ? n : 1;
}

__device__ __forceinline__ bool same_walk(const ShareStart& a, const ShareStart& b) {
  return a.place == b.place && a.kvh == b.kvh;
}
__device__ __forceinline__ bool same(const ShareStart& a, const ShareStart& b) { return same_walk(a, b) && a.step == b.step; }
__device__ __forceinline__ ShareStart uniform(const ShareStart& x) {
  return ShareStart{__builtin_amdgcn_readfirstlane(x.place), __builtin_amdgcn_readfirstlane(x.kvh),
                    __builtin_amdgcn_readfirstlane(x.step), 0};
}

// Places of the launch's order: run * stride, at least a place for each block.
__device__ __forceinline__ int places(const Blocks& b) { return b.run * b.stride; }

struct Block {
  Segment s;
  int seg, block;
  bool rows;  // it has any
  int next;   // the first place after this one whose block may have rows
};

__device__ __forceinline__ Block block_at(const PagedParams& p, const Blocks& b, int place) {
  Block x;
  const int i = b.run == 1 ? place : place % b.run * b.stride + place / b.run;
  const int seg = b.n == 1 ? i : (int)((unsigned)i / (unsigned)b.n);
  x.seg = seg;
  x.block = i - seg * b.n;
  x.rows = false;
  x.next = place + 1;
  if (seg < p.n_segments) {
    x.s = segment_at(p, seg);
    const int64_t left = (int64_t)x.s.n * p.G - (int64_t)x.block * b.rows;
    x.rows = left > 0;
    if (b.run == 1 && left <= b.rows) x.next = (seg + 1) * b.n;  // the segment's last one
  }
  return x;
}

// The walk after this one, at its block; false behind the last.
template <bool kHeadsOuter>
__device__ __forceinline__ bool next_walk(const PagedParams& p, const Blocks& b, Block* x, int* place, int* kvh) {
  if (!kHeadsOuter) {
    if (++*kvh < p.Hkv) return true;
    *kvh = 0;
  }
  do {
    *place = x->next;
    if (*place >= places(b)) {
      if (!kHeadsOuter || ++*kvh >= p.Hkv) return false;
      *place = 0;
    }
    *x = block_at(p, b, *place);
  } while (!x->rows);
  return true;
}

// 64-bit division costs hundreds of instructions; nearly always 32 bits hold it.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  if (((uint64_t)a | (uint64_t)b) >> 32 == 0) return (int64_t)((uint32_t)a / (uint32_t)b);
  return a / b;
}

// A share is [at, end); behind the last walk is place places(b).  A walk counts as its
// steps and kSetup more (its rows fetched, the first tiles waited for, the rows
// stored).  A cut within those, or less than kSnap steps from the walk's start or end,
// moves there: a shorter part costs more than it evens out.
struct Share {
  ShareStart at, end;
};

// Every thread counts the steps of its run of places [i0, i1), `per` each, of one KV
// head; `before` are those of the threads before it.
struct Counted {
  int64_t mine, before, total;
  int i0, i1, per;
};

template <int kTiles, int kSetup>
__device__ __forceinline__ int cost_of(const PagedParams& p, const Blocks& b, const Block& x) {
  return x.rows ? kSetup + steps_of<kTiles>(block_walk(p, b, x.s, x.block)) : 0;
}

// For each of the launch's ways to cut the rows, at most kWays.
template <int kThreads, int kTiles, int kSetup, int kWays>
__device__ void count_steps(const PagedParams& p, int ways, Counted (&counted)[kWays]) {
  __shared__ int64_t wave_sum[kWays][kThreads / 64];
  const int tid = threadIdx.x;
#pragma unroll
  for (int y = 0; y < kWays; ++y) {
    const Blocks& b = p.blocks[y];
    const int n_places = y < ways ? places(b) : 0;
    Counted& c = counted[y];
    c.per = (n_places + kThreads - 1) / kThreads;
    c.i0 = tid * c.per < n_places ? tid * c.per : n_places;
    c.i1 = c.i0 + c.per < n_places ? c.i0 + c.per : n_places;
    c.mine = 0;
    for (int i = c.i0; i < c.i1;) {
      const Block x = block_at(p, b, i);
      c.mine += cost_of<kTiles, kSetup>(p, b, x);
      i = x.next;
    }
    c.before = c.mine;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
      const int64_t x = __shfl_up(c.before, k);
      if ((tid & 63) >= k) c.before += x;
    }
    if ((tid & 63) == 63) wave_sum[y][tid >> 6] = c.before;
  }
  __syncthreads();
#pragma unroll
  for (int y = 0; y < kWays; ++y) {
    Counted& c = counted[y];
    c.total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
      if (w < (tid >> 6)) c.before += wave_sum[y][w];
      c.total += wave_sum[y][w];
    }
    c.before -= c.mine;
  }
}

// The thread whose places hold a share's end finds the walk there.
template <int kTiles, int kSetup, int kSnap, bool kHeadsOuter>
__device__ Share find_share(const PagedParams& p, const Blocks& b, const Counted& c, int share) {
  __shared__ ShareStart found[2];
  const int64_t per_head = c.total > 0 ? c.total : 1;
  const int64_t total = c.total * p.Hkv;
  const int heads = kHeadsOuter ? 1 : p.Hkv;  // that share a step's place in the order
  // With fewer steps than shares the last shares are empty; of the others each end but
  // the last is found by one thread.
  const int64_t n = total < p.n_shares ? total : p.n_shares;
  for (int e = 0; e < 2; ++e) {
    if (share + e >= n) continue;
    int64_t u = quotient(total * (share + e), n);
    const int head = kHeadsOuter ? (int)quotient(u, per_head) : 0;
    u -= head * per_head + c.before * heads;
    if (u < 0 || u >= c.mine * heads) continue;
    for (int i = c.i0, next; i < c.i1; i = next) {
      int cost = (int)c.mine;
      next = i + 1;
      if (c.per > 1) {
        const Block x = block_at(p, b, i);
        cost = cost_of<kTiles, kSetup>(p, b, x);
        next = x.next;
      }
      if (u >= (int64_t)cost * heads) {
        u -= (int64_t)cost * heads;
        continue;
      }
      const int k = (int)quotient(u, cost);
      int place = i, kvh = head + k, step = (int)(u - (int64_t)k * cost) - kSetup;
      if (step < kSnap) step = 0;
      if (step && cost - kSetup - step < kSnap) {
        Block x = block_at(p, b, i);
        step = 0;
        if (!next_walk<kHeadsOuter>(p, b, &x, &place, &kvh)) place = places(b), kvh = 0;
      }
      found[e] = ShareStart{place, kvh, step, 0};
      break;
    }
  }
  __syncthreads();
  const ShareStart behind = {places(b), 0, 0, 0};
  return Share{share < n ? found[0] : behind, share + 1 < n ? found[1] : behind};
}

// ---------------------------------------------------------------------------
// K and V tiles in LDS.  A half is one page's 16 keys of one KV head, 256 bytes
// each; 16-byte chunk c of key k (of the half) lies at slot c ^ swizzle(k) of the
// key's 256 bytes.  The K reads (16 keys, one chunk) then touch every bank once,
// and so do the transposed V reads (8 keys, two chunks).
__device__ __forceinline__ int swizzle(int k) { return ((k & 7) << 1) | ((k >> 3) & 1); }

__device__ __forceinline__ uint32_t lds_addr(const unsigned char* p) {
  return (uint32_t)(uintptr_t)((const __attribute__((address_space(3))) unsigned char*)p);
}

// 256 zero bytes: what a key without a page, or that no row sees, reads.
static __device__ __attribute__((aligned(256))) unsigned char g_zeros[kRowBytes];

// One direct-to-LDS load: lane l's 16 bytes at its address land at LDS byte lds_base
// + 16 l.  Inline assembly, so that the compiler does not make every later LDS
// read wait for it: the kernels count these loads themselves.  The LDS address is
// an input bound to m0; one wait state between its write and the load.
__device__ __forceinline__ void load_lds_from(const void* addr, uint32_t lds_base) {
  asm volatile(
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off\n\t" ::"v"(addr),
      "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_base))
      : "memory");
}
// The same with the non-temporal hint.
__device__ __forceinline__ void stream_lds_from(const void* addr, uint32_t lds_base) {
  asm volatile(
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, off nt\n\t" ::"v"(addr),
      "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_base))
      : "memory");
}

// A loaded value is waited for here, and not where it is used: in a loop that would
// be a wait for every load in flight, the direct ones among them, each time around
// (the compiler cannot tell whether the value was loaded in this iteration).
template <class T>
__device__ __forceinline__ void landed(T& x) {
  asm volatile("" : "+v"(x));
}

// s_waitcnt immediate: at most n of this wave's vector-memory operations
// outstanding (vmcnt[3:0] at [3:0], vmcnt[5:4] at [15:14]).
constexpr int wait_vm(int n) { return 0x0F70 | (n & 15) | ((n >> 4) << 14); }

// Where a half's keys lie: their page, or rows of k_new (same offsets for V).
struct HalfSource {
  int64_t offset;  // bytes from the cache's (or k_new's) start to key 0, this KV head
  bool paged, none;
};

__device__ __forceinline__ HalfSource half_source(const PagedParams& p, int page, int hp, int kvh) {
  HalfSource h;
  h.paged = hp < p.paged_end;
  h.none = h.paged && (uint32_t)page >= (uint32_t)p.n_blocks;
  const int64_t key = h.paged ? (int64_t)page * kBlockTokens : (int64_t)(hp - p.paged_end);
  h.offset = key * p.kv_stride + (int64_t)kvh * kRowBytes;
  return h;
}

// The page of the half at position hp (any value where there is none to read).
__device__ __forceinline__ int page_of(const PagedParams& p, const Segment& s, int hp) {
  const int b = hp / kBlockTokens;
  return hp < p.paged_end && b < p.table_len ? s.table[b] : -1;
}

// ---------------------------------------------------------------------------
// Fragments (v_mfma_f32_16x16x32_bf16; lane 16 g + i).

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Sums of a tile's rounded weights P^T, each row's in its four lanes: the product of
// ones with them.
__device__ __forceinline__ f32x4 weight_sums(const bf16x8& pf) {
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.f;
  return mfma16(ones, pf, f32x4{});
}
__device__ __forceinline__ float weight_sum(const bf16x8& pf) { return weight_sums(pf)[0]; }

// A of S^T = K Q^T: key i of the half, head dims 32 step + 8 g ..
__device__ __forceinline__ bf16x8 k_frag(const unsigned char* k, int lane, int half, int step) {
  const int g = lane >> 4, i = lane & 15;
  return *reinterpret_cast<const bf16x8*>(k + half * kHalfBytes + i * kRowBytes + (((4 * step + g) ^ swizzle(i)) << 4));
}

// A of O^T += V^T P^T: head dim 16 db + i, keys 4 g .. 4 g + 3 of each half, by
// the transposing read.
__device__ __forceinline__ bf16x8 v_frag(const unsigned char* v, int lane, int db) {
  const int g = lane >> 4, i = lane & 15;
  const int k = 4 * g + (i >> 2);
  const unsigned char* at = v + k * kRowBytes + (((2 * db + ((i & 3) >> 1)) ^ swizzle(k)) << 4) + 8 * (i & 1);
  typedef __attribute__((address_space(3))) s16x4* Lds;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + kHalfBytes));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Maximum (NaN if any is) and sum over the four lanes that hold one query.
__device__ __forceinline__ float quad_max(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  x = __builtin_elementwise_maximum(__builtin_bit_cast(float, (unsigned)a[0]), __builtin_bit_cast(float, (unsigned)a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_elementwise_maximum(__builtin_bit_cast(float, (unsigned)b[0]), __builtin_bit_cast(float, (unsigned)b[1]));
}
__device__ __forceinline__ float quad_sum(float x) {
  auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  x = __builtin_bit_cast(float, (unsigned)a[0]) + __builtin_bit_cast(float, (unsigned)a[1]);
  auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_bit_cast(float, (unsigned)b[0]) + __builtin_bit_cast(float, (unsigned)b[1]);
}

// Scores of keys that the row at position pos does not see become -inf.
// s[half][r] is key t0 + 16 half + 4 g + r.  A key at distance pos - j is seen if that
// is in [0, window): one comparison of unsigned numbers.
__device__ __forceinline__ void mask_scores(const PagedParams& p, f32x4 (&s)[2], int t0, int g, int pos) {
  const unsigned window = p.window ? (unsigned)p.window : 1u << 31;
  const int away = pos - (t0 + 4 * g);
  if (__builtin_expect(t0 + kTileKeys > p.key_end, 0)) {  // no keys from there on
    const int end = p.key_end - (t0 + 4 * g);
#pragma unroll
    for (int c = 0; c < 8; ++c) s[c >> 2][c & 3] = 16 * (c >> 2) + (c & 3) < end ? s[c >> 2][c & 3] : -INFINITY;
  }
  if (__builtin_expect(p.window && t0 < p.n_sink, 0)) {
    const int sinks = p.n_sink - (t0 + 4 * g);
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const int key = 16 * (c >> 2) + (c & 3);
      const bool seen = ((unsigned)(away - key) < window) | ((key < sinks) & (key <= away));
      s[c >> 2][c & 3] = seen ? s[c >> 2][c & 3] : -INFINITY;
    }
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c)
      s[c >> 2][c & 3] = (unsigned)(away - (16 * (c >> 2) + (c & 3))) < window ? s[c >> 2][c & 3] : -INFINITY;
  }
}

// Whether a V tile (its fragments v(db)) holds an infinity or a NaN: its product with
// zeros is not 0.
template <class Frag>
__device__ __forceinline__ bool not_finite(Frag&& v) {
  f32x4 z = {};
  bf16x8 zeros = {};
#pragma unroll
  for (int db = 0; db < 8; ++db) z = mfma16(v(db), zeros, z);
  const bool bad = !(z[0] == 0.f && z[1] == 0.f && z[2] == 0.f && z[3] == 0.f);
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}

// The keys of this lane's scores that the row at position pos sees: bit 4 half + r of
// each.  (A loop: this rare path has to leave registers to the common one.)
__device__ __forceinline__ unsigned keys_seen(const PagedParams& p, int t0, int g, int pos) {
  unsigned seen = 0;
#pragma unroll 1
  for (int e = 0; e < 8; ++e) {
    const int key = t0 + 16 * (e >> 2) + 4 * g + (e & 3);
    const bool sees = key <= pos && key < p.key_end && (!p.window || key > pos - p.window || key < p.n_sink);
    seen |= (sees ? 1u : 0u) << e;
  }
  return seen;
}

// O^T += V^T P^T of such a tile, where some of its keys are hidden from some rows
// of the block: a weight of 0 times an infinity would be a NaN.  The finite values
// are added as ever; a row takes the others from the keys that it sees (as keys_seen
// gives them), also from those whose weight is 0: so they show in O wherever a tile or a
// part begins.
template <int NB, class Frag>
__device__ __forceinline__ void pv_not_finite(Frag&& v, const bf16x8 (&pf)[NB], const unsigned (&keys)[NB],
                                              f32x4 (&o)[8][NB]) {
  // (One fragment at a time, for the same reason.)
  auto products = [&](auto&& of_value, auto&& use) {
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      bf16x8 f = v(db);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (__bf16)of_value((float)f[e]);
#pragma unroll
      for (int b = 0; b < NB; ++b) use(db, b, f);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto count_seen = [&](int b, const bf16x8& f) {
    bf16x8 seen;
#pragma unroll
    for (int e = 0; e < 8; ++e) seen[e] = (__bf16)(float)(keys[b] >> e & 1);
    return mfma16(f, seen, f32x4{});
  };
  products([](float x) { return __builtin_isfinite(x) ? x : 0.f; },
           [&](int db, int b, const bf16x8& f) { o[db][b] = mfma16(f, pf[b], o[db][b]); });
  auto add = [&](auto&& is, float what) {
    products([&](float x) { return is(x) ? 1.f : 0.f; },
             [&](int db, int b, const bf16x8& f) {
               const f32x4 n = count_seen(b, f);
#pragma unroll
               for (int r = 0; r < 4; ++r) o[db][b][r] += n[r] > 0.f ? what : 0.f;
             });
  };
  add([](float x) { return x == INFINITY; }, INFINITY);
  add([](float x) { return x == -INFINITY; }, -INFINITY);
  add([](float x) { return x != x; }, NAN);
}

}  // namespace tile
}  // namespace cpattn
