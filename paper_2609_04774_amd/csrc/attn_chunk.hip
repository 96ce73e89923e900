// Attention over a paged cache, or of a rank's rows through a window, of blocks of
// many rows: chunks of prompts.  The mathematics, the rounding and the shares are
// those of attn_rows.hip; what differs is what bounds it, the matrix cores.
//
// A workgroup of 8 waves (two per SIMD: one's vector work issues while the other's
// products run) owns a block of 128, 256 or 384 rows of one KV head, 16 NB per wave, and
// walks their keys in tiles of 32 that all waves read from LDS: every fragment of K or V that
// is read feeds NB products, one for each 16 rows.  One iteration runs O += V_{j-1}^T P_{j-1}, the
// softmax of tile j and S_{j+1} = K_{j+1} Q^T as one sequence of 16 slots, each
// with one fragment, its products and a share of the vector work; the loads of tile
// j + kAhead go straight to LDS.  Weights are taken against the running maximum of
// the tiles before, which needs no look at the tile's own scores: they stay exact
// relative to each other at any size, so only a tile whose weights could
// overflow is done again with its own maximum (as in attn_partial.hip).
// The sum of the rounded weights, which divides O, is one more product per 16 rows and
// tile (2 to 3 % of a long launch; added up by vector instructions 6 to 14 %, by
// 4 x 4 x 4 products 3 to 5 %).
//
// Measured (calls, 32 query and 8 KV heads): 4096 rows after 32768 tokens (2.34 TFLOP) 1923
// us, 1215 TFLOP/s, where a product of two 8192 x 8192 matrices runs at 1210; 256 rows to
// a block 2012.  A tile takes 0.63 us of 128 rows, 0.92 of 256 and 1.30 of 384, and larger
// blocks pad more and have fewer walks to share out: alone, 4096 rows take 200 us in
// blocks of 384 and 175 in those of 256; 200 rows 27.6 of 256 and 20.8 of 128; 63 single
// tokens after 256 to 32768 keys and a chunk of 2048 605 and 520.  So the lengths choose,
// within 1 % of a kernel of the better size alone (200 rows 21.7, as both ways are counted;
// 2048 rows after 32768 1006 and 973, as they are not offered 384).  One kernel holds the
// bodies of 128 and 256; with that of 384 its registers were spilled, which is a second
// kernel that the first may leave the work to.  A rank's 8192 rows through a window of
// 4096 436 us (0.41 TFLOP), 22 of them the merge.  One barrier for two tiles against one
// each: 5 % faster.  KV heads one after another, blocks inside, against the reverse: 4 to
// 7 %.
#include <hip/hip_runtime.h>

#include "attn_tile.h"

namespace cpattn {

namespace {

using namespace tile;

constexpr int kWaves = kChunkThreads / 64;
constexpr int kBufs = 8;   // LDS buffers of K and of V; tile t uses buffer t % kBufs
constexpr int kAhead = 5;  // iteration j loads tile j + kAhead
constexpr int kSetup = 10;  // of a walk, in tiles
constexpr int kSnap = 4;   // tiles: a part costs its set-up, and its rows a merge
// A tile of 128, 256 and 384 rows takes about 21/32, 1 and 11/8 of 0.92 us.  A share of larger
// blocks costs more besides, in tiles: its set-ups and its parts' merge are larger, and
// so are, at both edges of a window, the tiles that some row sees in part.
constexpr int kNarrowSteps = 5;
constexpr int kWideSteps = 40, kWideWindowSteps = 80;

// LDS tiles by 16-byte columns: column c of a half holds chunk c of its 16 keys, key
// k at slot k ^ 8 (c % 2).  The K reads (16 keys of a column) and the transposed V
// reads (8 keys of two columns) touch every bank once, and the addresses of a
// lane's fragments differ by constants.
constexpr int kColBytes = kBlockTokens * 16;
__device__ __forceinline__ int column_slot(int key, int c) { return c * kColBytes + ((key ^ (8 * (c & 1))) << 4); }

struct Fragments {
  uint32_t k, v;  // this lane's byte offsets in a K and in a V buffer
};

__device__ __forceinline__ bf16x8 load_k(const unsigned char* buf, const Fragments& f, int q) {  // q = 2 step + half
  return *reinterpret_cast<const bf16x8*>(buf + f.k + (q & 1) * kHalfBytes + (q >> 1) * 4 * kColBytes);
}
__device__ __forceinline__ bf16x8 load_v(const unsigned char* buf, const Fragments& f, int db) {
  typedef __attribute__((address_space(3))) s16x4* Lds;
  const unsigned char* at = buf + f.v + db * 2 * kColBytes;
  const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
  const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + kHalfBytes));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A direct-to-LDS load from a wave-uniform base plus this lane's offset.
__device__ __forceinline__ void load_lds(const void* base, uint32_t off, uint32_t lds_base) {
  const uint64_t b = (uint64_t)(uintptr_t)base;
  const uint64_t bs = ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(b >> 32)) << 32) |
                      (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)b);
  asm volatile(
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %0, %1\n\t" ::"v"(off), "s"((const void*)(uintptr_t)bs),
      "{m0}"(__builtin_amdgcn_readfirstlane((int)lds_base))
      : "memory");
}

template <typename T>
__device__ __forceinline__ void pin(const T& x) {  // computed before this point of the schedule
  asm volatile("" ::"v"(x));
}

template <int NB>
using Scores = f32x4[NB][2];  // [block][half]

template <int NB>
struct Weights {
  float sum[NB];     // fp32 sums of this lane's weights
  bf16x2 pair[NB][4];
};

constexpr float kMaxSum = 65536.f;  // of a lane's 8 weights of a tile; beyond it is done again

// One unit of a tile's softmax (of 12 NB, about equal): two exponentials of a pair
// of scores, or the pair's rounding and sum.
template <int NB>
__device__ __forceinline__ void softmax_unit(int u, Scores<NB>& s, Weights<NB>& w, const float (&m)[NB], float sl2) {
  const int b = u / 12, t = u % 12 / 3, kind = u % 3;  // block, pair
  const int half = t >> 1, r = 2 * (t & 1);
  if (kind < 2) {
    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][half][r + kind], sl2, -m[b]));
    pin(x);
    s[b][half][r + kind] = x;
  } else {
    w.pair[b][t] = bf16x2{(__bf16)s[b][half][r], (__bf16)s[b][half][r + 1]};
    w.sum[b] = t == 0 ? s[b][half][r] + s[b][half][r + 1] : w.sum[b] + (s[b][half][r] + s[b][half][r + 1]);
    pin(w.sum[b]);
    pin(w.pair[b][t]);
  }
}

template <int NB>
__device__ __forceinline__ void qk_step(Scores<NB>& s, const bf16x8& k, const bf16x8 (&qf)[NB][4], int q) {
#pragma unroll
  for (int b = 0; b < NB; ++b)
    s[b][q & 1] = mfma16(k, qf[b][q >> 1], (q >> 1) == 0 ? f32x4{} : s[b][q & 1]);
}

template <int NB>
__device__ __forceinline__ void qk_tile(const unsigned char* buf, const Fragments& f, const bf16x8 (&qf)[NB][4],
                                        Scores<NB>& s) {
#pragma unroll
  for (int q = 0; q < 8; ++q) qk_step(s, load_k(buf, f, q), qf, q);
}

// Raises the running maxima to a tile's own where that is higher; O and the sums
// follow.
template <int NB>
__device__ __forceinline__ void raise_max(const Scores<NB>& s, float (&m)[NB], float (&l)[NB], float (&mass)[NB],
                                          f32x4 (&o)[8][NB], float sl2) {
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    float top = s[b][0][0];
#pragma unroll
    for (int r = 1; r < 8; ++r) top = __builtin_elementwise_maximum(top, s[b][r >> 2][r & 3]);
    const float m_new = __builtin_elementwise_maximum(m[b], quad_max(top) * sl2);
    const float alpha = __builtin_amdgcn_exp2f(m[b] - m_new);
    l[b] *= alpha;
    mass[b] *= alpha;
#pragma unroll
    for (int db = 0; db < 8; ++db) o[db][b] *= alpha;
    m[b] = m_new;
  }
}

// The weights become the operand of the second product.
template <int NB>
__device__ __forceinline__ void finish(const Weights<NB>& w, float (&l)[NB], bf16x8 (&pf)[NB]) {
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    l[b] += w.sum[b];
    pf[b] = __builtin_shufflevector(__builtin_shufflevector(w.pair[b][0], w.pair[b][1], 0, 1, 2, 3),
                                    __builtin_shufflevector(w.pair[b][2], w.pair[b][3], 0, 1, 2, 3), 0, 1, 2, 3, 4, 5,
                                    6, 7);
  }
}

template <int NB>
__device__ __forceinline__ void pv_tile(const unsigned char* buf, const Fragments& f, const bf16x8 (&pf)[NB],
                                        float (&mass)[NB], f32x4 (&o)[8][NB]) {
#pragma unroll
  for (int b = 0; b < NB; ++b) mass[b] += weight_sum(pf[b]);
#pragma unroll
  for (int db = 0; db < 8; ++db) {
    const bf16x8 v = load_v(buf, f, db);
#pragma unroll
    for (int b = 0; b < NB; ++b) o[db][b] = mfma16(v, pf[b], o[db][b]);
  }
}

// The order of the units over an iteration: the exponentials of all blocks but the
// last first, and the roundings from slot 8 on, when the products with the tile
// before have freed their operand's registers.
template <int NB>
struct Order {
  int unit[12 * NB];
  constexpr Order() : unit{} {
    int n = 0;
    for (int b = 0; b + 1 < NB; ++b)
      for (int t = 0; t < 4; ++t)
        for (int k = 0; k < 2; ++k) unit[n++] = 12 * b + 3 * t + k;
    const int last = 12 * (NB - 1);
    int te = 0;
    for (; n < 6 * NB; ++te)
      for (int k = 0; k < 2; ++k) unit[n++] = last + 3 * te + k;
    for (int b = 0; b + 1 < NB; ++b)
      for (int t = 0; t < 4; ++t) unit[n++] = 12 * b + 3 * t + 2;
    for (int t = 0; t < 4; ++t)
      for (int k = t < te ? 2 : 0; k < 3; ++k) unit[n++] = last + 3 * t + k;
  }
};
template <int NB>
constexpr Order<NB> kOrder{};

// The fields are the same for all lanes: scalar registers hold them.
__device__ __forceinline__ Walk uniform_walk(const Walk& w) {
  auto u = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  return Walk{u(w.end), u(w.lo), u(w.sink), u(w.p_lo), u(w.p_hi), u(w.n_sink_tiles), u(w.base), u(w.n)};
}

// One workgroup's share, of blocks of 16 NB rows per wave.
template <int NB>
__device__ __forceinline__ void attend(const PagedParams& p, const Blocks& blocks, const Share& share, int number,
                                       unsigned char* smem) {
  constexpr int kRows = 16 * NB * kWaves;
  constexpr int kLookahead = NB == 1 ? 6 : NB == 2 ? 3 : 2;  // slots a fragment is read ahead of its products
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, i16 = lane & 15;

  unsigned char* const kbuf = smem;
  unsigned char* const vbuf = smem + kBufs * kTileBytes;
  unsigned char* const vzero = smem + 2 * kBufs * kTileBytes;
  static_assert(kTileBytes == 16 * kChunkThreads, "one 16-byte store per thread");
  *reinterpret_cast<f32x4*>(vzero + 16 * tid) = f32x4{};
  const Fragments fr = {(uint32_t)column_slot(i16, g),
                        (uint32_t)(column_slot(4 * g + (i16 >> 2), (i16 & 3) >> 1) + 8 * (i16 & 1))};
  // This wave's part of a tile's load: 1 KB of K and of V, four columns of one half.
  const int load_half = wave >> 2;
  const int load_key = i16 ^ (8 * (g & 1));
  const int load_chunk = 4 * (wave & 3) + g;
  const uint32_t load_off = (uint32_t)(load_key * p.kv_stride) + load_chunk * 16;
  const uint32_t load_dst = lds_addr(smem) + load_half * kHalfBytes + (wave & 3) * 4 * kColBytes;
  const float sl2 = p.scale_log2;

  // The start of the share's last walk comes first, then the end of its first walk,
  // then the walks between: the workgroups of an XCD, whose shares are cut at any
  // place of walks over the same keys, so pass over the keys together.
  const ShareStart at = uniform(share.at), end = uniform(share.end);
  bool ahead = end.step > 0 && !same_walk(at, end);
  int place = ahead ? end.place : at.place, kvh = ahead ? end.kvh : at.kvh;
  Block x = block_at(p, blocks, place);
  const Segment& s = x.s;

  // One part of a walk after another.  While the rows of one are stored, the queries
  // and the first tiles of the next are on their way.
  struct Rows {
    int64_t o_row;
    int rows, r0, kvh;  // of the segment and KV head; the wave's first
    float* slot;        // of a part of a walk, or null
  };
  Rows out = {0, 0, 0, 0, nullptr};
  Walk w;
  int step = 0, n = 0;  // the part's first tile, and its tiles
  int open0 = 0, open1 = 0;  // tiles of the walk that every row of the block sees whole
  int ids = -1, ids_of = 0;  // pages of this wave's half of 64 tiles, one per lane
  int pos[NB];
  bf16x8 qf[NB][4];
  f32x4 o[8][NB];
  float m[NB], l[NB];
  float mass[NB];  // sums of the rounded weights, of all four lanes of a row
  bf16x8 pf[NB];

  auto fetch_ids = [&](int j) {
    ids_of = j;
    ids = -1;
    if (j + lane < n) ids = page_of(p, s, tile_begin(w, step + j + lane) + load_half * kBlockTokens);
    landed(ids);
  };
  // Tile j of the part into buffer j % kBufs; past the last it is loaded again, into
  // a buffer nobody reads, so that the waits can count.
  auto load = [&](int j) {
    const uint32_t dst = load_dst + (j & (kBufs - 1)) * kTileBytes;
    const int jj = j < n ? j : n - 1;
    const int t0 = tile_begin(w, step + jj);
    const int hp = t0 + load_half * kBlockTokens;
    if (__builtin_expect((jj & ~63) != ids_of, 0)) fetch_ids(jj & ~63);
    const HalfSource h = half_source(p, __builtin_amdgcn_readlane(ids, jj & 63), hp, kvh);
    const unsigned char* kb = (h.paged ? p.k_cache : p.k_new) + h.offset;
    const unsigned char* vb = (h.paged ? p.v_cache : p.v_new) + h.offset;
    if (__builtin_expect(whole_tile(w, t0) && !h.none, 1)) {
      load_lds(kb, load_off, dst);
      load_lds(vb, load_off, dst + kBufs * kTileBytes);
    } else {
      const bool read = !h.none && walked(w, hp + load_key);
      const unsigned char* zeros = g_zeros + load_chunk * 16;
      load_lds_from(read ? kb + load_off : zeros, dst);
      load_lds_from(read ? vb + load_off : zeros, dst + kBufs * kTileBytes);
    }
  };
  auto closed = [&](int j) { return (step + j < open0) | (step + j >= open1); };
  auto mask = [&](int j, Scores<NB>& sc) {
    if (__builtin_expect(!closed(j), 1)) return;
    const int t0 = tile_begin(w, step + j);
#pragma unroll
    for (int b = 0; b < NB; ++b) mask_scores(p, sc[b], t0, g, pos[b]);
  };
  // A tile with keys that some row does not see, and an infinity or a NaN in V (a
  // weight of 0 times it would be a NaN): taken by itself.  Every wave looks at the
  // same values.
  auto apart = [&](int j) {
    if (__builtin_expect(!closed(j), 1)) return false;
    const unsigned char* v = vbuf + (j & (kBufs - 1)) * kTileBytes;
    return not_finite([&](int db) { return load_v(v, fr, db); });
  };
  auto store = [&]() {
    if (out.r0 >= out.rows) return;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = out.r0 + 16 * b + i16;
      const float sum = quad_sum(l[b]);
      const bool live = m[b] > 0.5f * kNoMax && sum > 0.f;
      const float inv = live ? 1.f / mass[b] : (sum != sum ? sum : 0.f);
      const float lse = live ? m[b] * kLn2 + logf(sum) : -INFINITY;
      if (out.slot) {
        const int rb = 16 * (NB * wave + b) + i16;
#pragma unroll
        for (int db = 0; db < 8; ++db)
          *reinterpret_cast<f32x4*>(out.slot + rb * kHeadDim + 16 * db + 4 * g) = o[db][b] * inv;
        // A NaN among the scores is an LSE of NaN here: the merge tells it from a part without keys.
        if (g == 0) out.slot[kRows * kHeadDim + rb] = sum != sum ? sum : lse;
      } else if (r < out.rows) {
        const int q = (int)((unsigned)r / (unsigned)p.G);
        const int64_t row = (out.o_row + q) * p.Hq + out.kvh * p.G + (r - q * p.G);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (__bf16)(o[db][b][e] * inv);
          *reinterpret_cast<bf16x4*>(p.o + row * kHeadDim + 16 * db + 4 * g) = v;
        }
        if (g == 0 && p.lse) p.lse[row] = lse;
      }
    }
  };

  for (bool first = true, more = true;; first = false) {
    const ShareStart here = {place, kvh, 0, 0};
    Rows now = out;
    if (more) {
      w = uniform_walk(block_walk(p, blocks, s, x.block));
      const int n_steps = steps_of<1>(w);
      step = same_walk(here, at) ? at.step : 0;
      const int stop = same_walk(here, end) ? end.step : n_steps;
      n = w.n ? stop - step : 0;
      now.o_row = s.o_row;
      now.rows = s.n * p.G;
      now.r0 = x.block * kRows + 16 * NB * wave;
      now.kvh = kvh;
      now.slot = step > 0 || stop < n_steps
                     ? p.slots + (2 * (size_t)number + (step > 0 ? 0 : 1)) * slot_floats(kRows)
                     : nullptr;
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        int r = now.r0 + 16 * b + i16;
        r = r < now.rows ? r : now.rows - 1;
        const int q = (int)((unsigned)r / (unsigned)p.G), h = r - q * p.G;
        pos[b] = s.pos0 + q;
        const uint16_t* from = p.q + (s.q_row + q) * p.q_stride + (int64_t)(kvh * p.G + h) * kHeadDim + 8 * g;
#pragma unroll
        for (int d = 0; d < 4; ++d) qf[b][d] = *reinterpret_cast<const bf16x8*>(from + 32 * d);
      }
      open_tiles(p, w, &open0, &open1);
      fetch_ids(0);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int d = 0; d < 4; ++d) landed(qf[b][d]);
      if (n > 0)
        for (int j = 0; j < kAhead; ++j) load(j);
    }
    if (!first) store();
    if (!more) return;
    out = now;
    const bool active = out.r0 < out.rows;  // a wave without rows only loads
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int db = 0; db < 8; ++db) o[db][b] = f32x4{};
      pf[b] = bf16x8{};
      m[b] = kNoMax;
      l[b] = mass[b] = 0.f;
    }

    if (n > 0) {
      int j = 0;
#pragma unroll 1
      while (j < n) {
        // Tile j has landed for every wave, and the tiles before it have been read.
        __builtin_amdgcn_s_waitcnt(wait_vm(2 * (kAhead - 1)));
        __syncthreads();
        const unsigned char* k_now = kbuf + (j & (kBufs - 1)) * kTileBytes;
        const unsigned char* v_now = vbuf + (j & (kBufs - 1)) * kTileBytes;
        Scores<NB> sa, sb;
        Weights<NB> wt;
        if (active) {
          qk_tile(k_now, fr, qf, sa);
          mask(j, sa);
          raise_max(sa, m, l, mass, o, sl2);
        }
        if (__builtin_expect(apart(j), 0)) {
          load(j + kAhead);
          if (active) {
            unsigned keys[NB] = {};  // by the masked scores (by the positions: 384 rows 1 % slower)
#pragma unroll
            for (int x = 0; x < 8 * NB; ++x)
              keys[x / 8] |= (sa[x / 8][x % 8 / 4][x % 4] != -INFINITY ? 1u : 0u) << (x % 8);
#pragma unroll
            for (int u = 0; u < 12 * NB; ++u) softmax_unit(u, sa, wt, m, sl2);
            finish(wt, l, pf);
#pragma unroll
            for (int b = 0; b < NB; ++b) mass[b] += weight_sum(pf[b]);
            pv_not_finite<NB>([&](int db) { return load_v(v_now, fr, db); }, pf, keys, o);
          }
          ++j;
          continue;
        }
        // The tiles up to the next such one, pipelined.  No tile before the first: its V
        // is zeros.
        bf16x8 pre[kLookahead];
        const unsigned char* v_before = vzero;
        Fragments at_lane = fr;  // (spilled around the loop at most)
        landed(at_lane.k);
        landed(at_lane.v);
        auto iteration = [&](int j, Scores<NB>& s_in, Scores<NB>& s_out) {
          const unsigned char* k_next = kbuf + ((j + 1) & (kBufs - 1)) * kTileBytes;
          const unsigned char* v_this = vbuf + (j & (kBufs - 1)) * kTileBytes;
          load(j + kAhead);
          bf16x8 f[16];
          f32x4 sums;  // of a block's rounded weights; added two slots later
#pragma unroll
          for (int x = 0; x < kLookahead; ++x) f[x] = pre[x];
#pragma unroll
          for (int slot = 0; slot < 16; ++slot) {
            const int x = slot + kLookahead;
            if (x < 8)
              f[x] = load_v(v_before, at_lane, x);
            else if (x < 16)
              f[x] = load_k(k_next, at_lane, x - 8);
            else
              pre[x - 16] = load_v(v_this, at_lane, x - 16);
            if (slot < 8) {
#pragma unroll
              for (int b = 0; b < NB; ++b) o[slot][b] = mfma16(f[slot], pf[b], o[slot][b]);
              if (slot % 2 == 0) {
                if (slot > 0 && slot / 2 <= NB) mass[slot / 2 - 1] += sums[0];
                if (slot / 2 < NB) sums = weight_sums(pf[slot / 2]);
              }
            } else {
              qk_step(s_out, f[slot], qf, slot - 8);
            }
#pragma unroll
            for (int u = slot * 12 * NB / 16; u < (slot + 1) * 12 * NB / 16; ++u)
              softmax_unit(kOrder<NB>.unit[u], s_in, wt, m, sl2);
            __builtin_amdgcn_sched_barrier(0);
          }
          bool fine = true;
#pragma unroll
          for (int b = 0; b < NB; ++b) fine = fine && wt.sum[b] <= kMaxSum;
          if (__builtin_expect(__builtin_amdgcn_ballot_w64(!fine) != 0, 0)) {
            qk_tile(kbuf + (j & (kBufs - 1)) * kTileBytes, fr, qf, s_in);
            mask(j, s_in);
            raise_max(s_in, m, l, mass, o, sl2);
#pragma unroll
            for (int u = 0; u < 12 * NB; ++u) softmax_unit(u, s_in, wt, m, sl2);
          }
          finish(wt, l, pf);
          v_before = v_this;
        };
        // In pairs behind one barrier (the first pair's is above): at a pair's start
        // every tile up to j + 2 has landed, and the buffers that its loads fill were
        // last read before it.
        if (active) {
#pragma unroll
          for (int b = 0; b < NB; ++b) pf[b] = bf16x8{};
#pragma unroll
          for (int x = 0; x < kLookahead; ++x) pre[x] = load_v(vzero, at_lane, x);
          for (;;) {
            __builtin_amdgcn_s_waitcnt(wait_vm(2 * (kAhead - 3)));
            __syncthreads();
            iteration(j, sa, sb);
            if (++j >= n || apart(j)) break;
            mask(j, sb);
            iteration(j, sb, sa);
            if (++j >= n || apart(j)) break;
            mask(j, sa);
          }
          pv_tile(v_before, fr, pf, mass, o);
        } else {
          for (;;) {
            __builtin_amdgcn_s_waitcnt(wait_vm(2 * (kAhead - 3)));
            __syncthreads();
            load(j + kAhead);
            if (++j >= n || apart(j)) break;
            load(j + kAhead);
            if (++j >= n || apart(j)) break;
          }
        }
      }
      __builtin_amdgcn_s_waitcnt(wait_vm(0));  // no load may still be writing LDS
    }

    if (ahead) {
      ahead = false;
      place = at.place;
      kvh = at.kvh;
      x = block_at(p, blocks, place);
    } else {
      more = !same_walk(here, end) && next_walk<true>(p, blocks, &x, &place, &kvh) &&
             !same_walk(end, ShareStart{place, kvh, 0, 0});
    }
    __syncthreads();  // every wave is done with the buffers
  }
}

// The buffers of K, of V, and a V tile of zeros.
struct Tiles {
  unsigned char bytes[(2 * kBufs + 1) * kTileBytes];
};

// Shares are numbered so that an XCD's workgroups (every eighth) have neighbouring
// ones, whose walks meet in its L2.
__device__ __forceinline__ int share_number(const PagedParams& p) {
  return p.n_shares % 8 == 0 ? (int)(blockIdx.x % 8) * (p.n_shares / 8) + (int)(blockIdx.x / 8) : (int)blockIdx.x;
}

// Looks at the lengths for the way to cut the rows, and does the work unless that is the
// last of three.
__global__ __launch_bounds__(kChunkThreads, 1) void attn_chunk_kernel(PagedParams p) {
  __shared__ __attribute__((aligned(1024))) Tiles tiles;
  const int number = share_number(p);
  Counted counted[3];
  count_steps<kChunkThreads, 1, kSetup>(p, p.n_ways, counted);
  const int64_t narrow = counted[0].total * p.Hkv, middle = counted[1].total * p.Hkv, wide = counted[2].total * p.Hkv;
  int way = narrow * 21 / 32 < middle + kNarrowSteps * p.n_shares ? 0 : 1;
  if (p.n_ways == 3 && wide * 11 / 8 + (p.window ? kWideWindowSteps : kWideSteps) * p.n_shares < middle) way = 2;
  way = __builtin_amdgcn_readfirstlane(way);
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.choice = way;
  if (way == 2) return;
  const Blocks blocks = p.blocks[way];
  const Share share = find_share<1, kSetup, kSnap, true>(p, blocks, way ? counted[1] : counted[0], number);
  if (threadIdx.x == 0) p.starts[number] = share.at;
  if (same(share.at, share.end)) return;
  if (way == 0)
    attend<1>(p, blocks, share, number, tiles.bytes);
  else
    attend<2>(p, blocks, share, number, tiles.bytes);
}

__global__ __launch_bounds__(kChunkThreads, 1) void attn_wide_kernel(PagedParams p) {
  __shared__ __attribute__((aligned(1024))) Tiles tiles;
  if (*p.choice != 2) return;
  const int number = share_number(p);
  Counted counted[3];
  count_steps<kChunkThreads, 1, kSetup>(p, 3, counted);
  const Blocks blocks = p.blocks[2];
  const Share share = find_share<1, kSetup, kSnap, true>(p, blocks, counted[2], number);
  if (threadIdx.x == 0) p.starts[number] = share.at;
  if (same(share.at, share.end)) return;
  attend<3>(p, blocks, share, number, tiles.bytes);
}

}  // namespace

int launch_attn_chunk(const PagedParams& p, void* stream, const char* who) {
  const dim3 grid((unsigned)p.n_shares), block(kChunkThreads);
  hipStream_t st = (hipStream_t)stream;
  hipLaunchKernelGGL(attn_chunk_kernel, grid, block, 0, st, p);
  if (p.n_ways == 3) hipLaunchKernelGGL(attn_wide_kernel, grid, block, 0, st, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(CP_ERR_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
  return launch_attn_merge(p, stream, who);
}

}  // namespace cpattn
