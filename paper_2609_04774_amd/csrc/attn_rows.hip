// Attention over a paged cache of blocks of few rows: the step that decodes one
// token (or a few) of every sequence.  A row is a (position, query head) pair of
// one KV head, so that grouped query heads share every key that is read.
//
// For the row at position p, over the visible keys j (j <= p, within the window
// or among the first tokens):  x_j = scale q.k_j,  LSE = ln sum_j e^{x_j},
// O = sum_j e^{x_j - LSE} v_j, in one pass with a running maximum and sum (Milakov
// & Gimelshein 2018; Dao 2023).  Scores, statistics and O are fp32; the weights
// are rounded to bf16 for the second product (half a step at most, 2^-8 of each), and O
// is divided by the sum of the rounded ones, so that it is a mean of the values whatever
// the roundings; LSE takes the sum before them.  O is rounded once more as it is stored.
//
// Bound by HBM: 512 bytes per key and KV head, each read once, for 16 or 32 rows.
// The walks of all blocks, in steps of 128 keys, are cut into equal parts,
// one per workgroup (two on each compute unit), wherever the cut falls (the lengths are
// read from the device, so that a captured launch follows them): no unit waits
// for another's longer sequence.  A part that ends inside a walk leaves a partial
// result, and share_merge_kernel combines a walk's.  Each of a workgroup's four
// waves takes every fourth tile of 32 keys into its own LDS (K and V, loaded
// directly, the next tile's K as soon as this one's is in registers), so the waves
// meet only at the end of a walk; the eight waves of a compute unit keep about 128
// KB in flight.
//
// Long walks over a pool that the Infinity Cache (256 MB) cannot hold stream (loads with
// the non-temporal hint), but for pages that another sequence of the batch names too
// (a shared prefix).  64 sequences of 8192 keys 338 us against 370 with plain loads; of
// one prefix of 8192 keys 117 to 126, of 32768 keys for 32 sequences 225 (streamed, 346).  Walks of
// fewer keys than 1280 do not: at 300 they take 246 us plain and 278 streamed, at 1024
// 229 and 233, at 1536 226 and 222, at 4096 230 and 215 (1.2 GB each).  Sequences past the
// 512th, or whose first page is gone, find no other: their long walks stream.
//
// Measured (32 query and 8 KV heads): 64 sequences of 8192 keys 338 us, 6.35 TB/s, where
// a plain read of as much runs at 6.0 to 6.5.  One sequence of 4101 keys 19 us, of which
// the merge is 6: latency (the lengths, the pages, the keys, one after another).
// Four or eight waves with a head each, as many shares again, or shares numbered by XCD
// were no faster.
#include <hip/hip_runtime.h>

#include "attn_tile.h"

namespace cpattn {

namespace {

using namespace tile;

constexpr int kWaves = kRowsThreads / 64;
constexpr int kWaveBytes = 2 * kTileBytes;  // a tile of K and one of V
constexpr int kSetup = 1;                   // of a walk, in steps
constexpr int kStreamTiles = 40;            // of a walk whose loads stream
constexpr int kLoads = kTileBytes / 1024;   // direct-to-LDS loads of a tile and tensor, 1 KB each

// One tile's loads of K (tensor 0) or V: 1 KB each, four keys of 256 bytes.  `off`
// are this lane's offsets within a half (four loads of it).  Bit `half` of kept: with
// plain loads, else with streaming ones.
__device__ __forceinline__ void load_tile(const PagedParams& p, const Walk& w, int t0, int kvh, int pages, int first,
                                          uint64_t kept, const uint32_t (&off)[4], int lane, uint32_t dst, int tensor) {
  const unsigned char* cache = tensor ? p.v_cache : p.k_cache;
  const unsigned char* fresh = tensor ? p.v_new : p.k_new;
  const bool whole = whole_tile(w, t0);
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int hp = t0 + half * kBlockTokens;
    const HalfSource h = half_source(p, __builtin_amdgcn_readlane(pages, first + half), hp, kvh);
    const unsigned char* base = (h.paged ? cache : fresh) + h.offset;
    const bool plain = whole && !h.none;
    const unsigned char* from[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      from[q] = base + off[q];
      if (!plain && (h.none || !walked(w, hp + 4 * q + (lane >> 4)))) from[q] = g_zeros + ((lane & 15) << 4);
    }
    const uint32_t at = dst + half * kHalfBytes;
    if (kept >> (first + half) & 1) {
#pragma unroll
      for (int q = 0; q < 4; ++q) load_lds_from(from[q], at + q * 1024);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q) stream_lds_from(from[q], at + q * 1024);
    }
  }
}

// Sequences that share a prefix name the same first page.  For each of the first
// kPartners sequences: another one with its first page, or -1.  (Found through a table of
// the largest and the smallest such sequence of each page, by its low bits: one page's
// sequences may hide another's, which then counts as not shared.)
constexpr int kPartners = 512;
constexpr int kPartnerPer = kPartners / kRowsThreads;

struct Partners {
  unsigned long long lo[kPartners], hi[kPartners];
};

__device__ __forceinline__ void first_pages(const PagedParams& p, int (&page)[kPartnerPer]) {
#pragma unroll
  for (int k = 0; k < kPartnerPer; ++k) {
    const int s = threadIdx.x + k * kRowsThreads;
    page[k] = s < p.n_segments && p.table_len > 0 ? p.tables[s * p.table_stride] : -1;
  }
}

__device__ __forceinline__ void enter_partners(const int (&page)[kPartnerPer], Partners& t) {
#pragma unroll
  for (int k = 0; k < kPartnerPer; ++k) {
    if (page[k] < 0) continue;
    const unsigned long long key = (unsigned long long)page[k] << 32 | (threadIdx.x + k * kRowsThreads);
    atomicMin(&t.lo[page[k] % kPartners], key);
    atomicMax(&t.hi[page[k] % kPartners], key);
  }
}

__device__ __forceinline__ void find_partners(const int (&page)[kPartnerPer], const Partners& t, int16_t* partner_of) {
#pragma unroll
  for (int k = 0; k < kPartnerPer; ++k) {
    const int s = threadIdx.x + k * kRowsThreads;
    int found = -1;
    if (page[k] >= 0) {
      const unsigned long long lo = t.lo[page[k] % kPartners], hi = t.hi[page[k] % kPartners];
      if ((int)(lo >> 32) == page[k] && (int)lo != s) found = (int)lo;
      if ((int)(hi >> 32) == page[k] && (int)hi != s) found = (int)hi;
    }
    partner_of[s] = (int16_t)found;
  }
}

template <int NB>
__global__ __launch_bounds__(kRowsThreads, 2) void attn_rows_kernel(PagedParams p) {
  __shared__ __attribute__((aligned(1024))) unsigned char smem[kWaves * kWaveBytes];
  __shared__ float stat[3][kWaves][16 * NB];  // per wave and row: maximum, sum, sum of the rounded weights
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = lane >> 4, i16 = lane & 15;
  __shared__ int16_t partner_of[kPartners];
  static_assert(sizeof(Partners) <= sizeof(smem), "in the tiles' memory, before them");
  const Blocks blocks = p.blocks[0];
  Partners& partners = *reinterpret_cast<Partners*>(smem);
  int page0[kPartnerPer];
  if (p.streamed) {
    first_pages(p, page0);
    for (int i = tid; i < kPartners; i += kRowsThreads) {
      partners.lo[i] = ~0ull;
      partners.hi[i] = 0;
    }
  }
  Counted counted[1];
  count_steps<kRowsThreads, kWaves, kSetup>(p, 1, counted);
  if (p.streamed) enter_partners(page0, partners);
  const Share share = find_share<kWaves, kSetup, 1, false>(p, blocks, counted[0], blockIdx.x);
  if (tid == 0) p.starts[blockIdx.x] = share.at;
  if (same(share.at, share.end)) return;
  if (p.streamed) {
    find_partners(page0, partners, partner_of);
    __syncthreads();
  }

  unsigned char* const mine = smem + wave * kWaveBytes;
  const uint32_t lds = lds_addr(mine);
  uint32_t off[4];  // this lane's key and chunk in each load of a half
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int key = 4 * q + g;
    off[q] = (uint32_t)(key * p.kv_stride) + ((i16 ^ swizzle(key)) << 4);
  }

  const ShareStart end = uniform(share.end);
  int place = __builtin_amdgcn_readfirstlane(share.at.place), kvh = __builtin_amdgcn_readfirstlane(share.at.kvh);
  int step = __builtin_amdgcn_readfirstlane(share.at.step);
  Block x = block_at(p, blocks, place);
  const Segment& s = x.s;

  // One part of a walk after another.  While the rows of one are combined and stored,
  // the queries and the pages of the next are on their way.
  struct Rows {
    int64_t o_row;
    int rows, r0, kvh;  // of the segment and KV head; the block's first
    float* slot;        // of a part of a walk, or null
  };
  Rows out = {0, 0, 0, 0, nullptr};
  Walk w;
  int n_mine = 0;  // this wave's tiles: kWaves (step + j) + wave for j below n_mine
  int ids = -1;    // pages of the halves of tiles 32 (j / 32) .. of this wave, one per lane
  int other = -1;  // and another sequence's there, if it shares the first page
  int partner = -1;
  uint64_t kept = ~0ull;  // halves that another sequence reads too
  int pos[NB];
  bf16x8 qf[NB][4];  // B of S^T = K Q^T: row i16 of block b, head dims 32 step + 8 g ..
  f32x4 o[8][NB];
  float m[NB], l[NB];
  float mass[NB];  // sums of the rounded weights, of all four lanes of a row
  auto tile_at = [&](int j) { return tile_begin(w, kWaves * (step + j) + wave); };
  auto fetch_ids = [&](int j) {
    ids = other = -1;
    const int jj = j + (lane >> 1);
    if (jj < n_mine) {
      const int hp = tile_at(jj) + (lane & 1) * kBlockTokens;
      ids = page_of(p, s, hp);
      if (partner >= 0) other = page_of(p, Segment{0, 0, 0, 0, p.tables + partner * p.table_stride}, hp);
    }
  };
  auto have_ids = [&]() {
    landed(ids);
    landed(other);
    kept = p.streamed && w.n >= kStreamTiles ? __builtin_amdgcn_ballot_w64(ids == other) : ~0ull;
  };
  auto load = [&](int j, int tensor) {
    load_tile(p, w, tile_at(j), kvh, ids, 2 * (j & 31), kept, off, lane, lds + tensor * kTileBytes, tensor);
  };
  // The four waves' results, unnormalised, row by row through LDS: float4 c of row r at
  // slot c ^ (r % 16) of its row.
  auto store = [&]() {
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int r = 16 * b + i16;
      const float sum = quad_sum(l[b]);
      if (g == 0) {
        stat[0][wave][r] = m[b];
        stat[1][wave][r] = sum;
        stat[2][wave][r] = mass[b];
      }
#pragma unroll
      for (int db = 0; db < 8; ++db)
        *reinterpret_cast<f32x4*>(mine + r * (kHeadDim * 4) + (((4 * db + g) ^ i16) << 4)) = o[db][b];
    }
    __syncthreads();
    for (int y = tid; y < 16 * NB * 16; y += kRowsThreads) {  // 8 values of a row each
      const int r = y >> 4, c = (y & 15) * 2;
      float top = kNoMax;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) top = __builtin_elementwise_maximum(top, stat[0][k][r]);
      float sum = 0.f, rounded = 0.f;
      f32x4 a0 = {}, a1 = {};
#pragma unroll
      for (int k = 0; k < kWaves; ++k) {
        const float wk = __builtin_amdgcn_exp2f(stat[0][k][r] - top);
        sum += wk * stat[1][k][r];
        rounded += wk * stat[2][k][r];
        const unsigned char* row = smem + k * kWaveBytes + r * (kHeadDim * 4);
        a0 += wk * *reinterpret_cast<const f32x4*>(row + ((c ^ (r & 15)) << 4));
        a1 += wk * *reinterpret_cast<const f32x4*>(row + (((c + 1) ^ (r & 15)) << 4));
      }
      const bool live = top > 0.5f * kNoMax && sum > 0.f;  // false for a NaN too
      const float inv = live ? 1.f / rounded : (sum != sum ? sum : 0.f);
      const float lse = live ? top * kLn2 + logf(sum) : -INFINITY;
      a0 *= inv;
      a1 *= inv;
      if (out.slot) {
        // A NaN among the scores is an LSE of NaN here: the merge tells it from a part without keys.
        *reinterpret_cast<f32x4*>(out.slot + r * kHeadDim + 4 * c) = a0;
        *reinterpret_cast<f32x4*>(out.slot + r * kHeadDim + 4 * c + 4) = a1;
        if (c == 0) out.slot[16 * NB * kHeadDim + r] = sum != sum ? sum : lse;
      } else if (out.r0 + r < out.rows) {
        const int at = (int)((unsigned)(out.r0 + r) / (unsigned)p.G);
        const int64_t row = (out.o_row + at) * p.Hq + out.kvh * p.G + (out.r0 + r - at * p.G);
        bf16x8 v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[e] = (__bf16)a0[e];
          v[4 + e] = (__bf16)a1[e];
        }
        *reinterpret_cast<bf16x8*>(p.o + row * kHeadDim + 4 * c) = v;
        if (c == 0 && p.lse) p.lse[row] = lse;
      }
    }
    __syncthreads();  // the LDS is free for the next part's tiles
  };

  for (bool first = true, more = true;; first = false) {
    Rows now = out;
    if (more) {
      w = block_walk(p, blocks, s, x.block);
      const int n_steps = steps_of<kWaves>(w);
      const int stop = same_walk(end, ShareStart{place, kvh, 0, 0}) ? end.step : n_steps;
      now.o_row = s.o_row;
      now.rows = s.n * p.G;
      now.r0 = x.block * (16 * NB);
      now.kvh = kvh;
      now.slot = step > 0 || stop < n_steps
                     ? p.slots + (2 * (size_t)blockIdx.x + (step > 0 ? 0 : 1)) * slot_floats(16 * NB)
                     : nullptr;
      // Rows past the block's end repeat its last one and are not stored.
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        int r = now.r0 + 16 * b + i16;
        r = r < now.rows ? r : now.rows - 1;
        const int at = (int)((unsigned)r / (unsigned)p.G), h = r - at * p.G;
        pos[b] = s.pos0 + at;
        const uint16_t* q = p.q + (s.q_row + at) * p.q_stride + (int64_t)(kvh * p.G + h) * kHeadDim + 8 * g;
#pragma unroll
        for (int d = 0; d < 4; ++d) qf[b][d] = *reinterpret_cast<const bf16x8*>(q + 32 * d);
      }
      const int t_end = w.n < kWaves * stop ? w.n : kWaves * stop;
      n_mine = (t_end - kWaves * step - wave + kWaves - 1) / kWaves;
      if (p.streamed) partner = __builtin_amdgcn_readfirstlane(x.seg < kPartners ? partner_of[x.seg] : -1);
      fetch_ids(0);
    }
    if (!first) store();
    if (!more) return;
    out = now;
    have_ids();
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int d = 0; d < 4; ++d) landed(qf[b][d]);
    int ids_of = 0;
    if (n_mine > 0) {
      load(0, 0);
      load(0, 1);
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int db = 0; db < 8; ++db) o[db][b] = f32x4{};
      m[b] = kNoMax;
      l[b] = mass[b] = 0.f;
    }
    const unsigned char* kt = mine;
    const unsigned char* vt = mine + kTileBytes;
    for (int j = 0; j < n_mine; ++j) {
      const int t0 = tile_at(j);
      // Past the last tile it is loaded again, so that the waits can count; nobody reads it.
      const int jn = j + 1 < n_mine ? j + 1 : j;
      if ((jn & ~31) != ids_of) {
        ids_of = jn & ~31;
        fetch_ids(ids_of);
        have_ids();
      }
      __builtin_amdgcn_s_waitcnt(wait_vm(kLoads));  // K of tile j is in LDS
      asm volatile("" ::: "memory");
      f32x4 sc[NB][2];
      {
        bf16x8 kf[2][4];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int d = 0; d < 4; ++d) kf[half][d] = k_frag(kt, lane, half, d);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            sc[b][half] = f32x4{};
#pragma unroll
            for (int d = 0; d < 4; ++d) sc[b][half] = mfma16(kf[half][d], qf[b][d], sc[b][half]);
          }
      }
      // The K fragments are in registers (the products used them): the buffer is free.
      __builtin_amdgcn_s_waitcnt(0xC07F);
      asm volatile("" ::: "memory");
      load(jn, 0);

      const bool open = open_tile(p, w, t0);
      bf16x8 pf[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (!open) mask_scores(p, sc[b], t0, g, pos[b]);
        float top = sc[b][0][0];
#pragma unroll
        for (int r = 1; r < 8; ++r) top = __builtin_elementwise_maximum(top, sc[b][r >> 2][r & 3]);
        const float m_new = __builtin_elementwise_maximum(m[b], quad_max(top) * p.scale_log2);
        const float alpha = __builtin_amdgcn_exp2f(m[b] - m_new);
        m[b] = m_new;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 8; ++r) {
          const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][r >> 2][r & 3], p.scale_log2, -m_new));
          sum += x;
          pf[b][r] = (__bf16)x;
        }
        l[b] = l[b] * alpha + sum;
        mass[b] = mass[b] * alpha + weight_sum(pf[b]);
#pragma unroll
        for (int db = 0; db < 8; ++db) o[db][b] *= alpha;
      }
      __builtin_amdgcn_s_waitcnt(wait_vm(kLoads));  // V of tile j
      asm volatile("" ::: "memory");
      // Keys hidden from every row are zeros; hidden from some, they may be anything.
      auto frag = [&](int db) { return v_frag(vt, lane, db); };
      if (__builtin_expect(!open && w.p_lo != w.p_hi && not_finite(frag), 0)) {
        unsigned keys[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) keys[b] = keys_seen(p, t0, g, pos[b]);
        pv_not_finite<NB>(frag, pf, keys, o);
      } else {
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const bf16x8 vf = v_frag(vt, lane, db);
#pragma unroll
          for (int b = 0; b < NB; ++b) o[db][b] = mfma16(vf, pf[b], o[db][b]);
        }
      }
      __builtin_amdgcn_s_waitcnt(0xC07F);
      asm volatile("" ::: "memory");
      load(jn, 1);
    }
    __builtin_amdgcn_s_waitcnt(wait_vm(0));  // no load may still be writing LDS
    asm volatile("" ::: "memory");

    const bool last = same_walk(end, ShareStart{place, kvh, 0, 0});
    more = !last && next_walk<false>(p, blocks, &x, &place, &kvh) && !same(end, ShareStart{place, kvh, 0, 0});
    step = 0;
  }
}

int launched(const char* who) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CP_OK : fail(CP_ERR_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
}

}  // namespace

int launch_attn_rows(const PagedParams& p, void* stream, const char* who) {
  const dim3 grid((unsigned)p.n_shares), block(kRowsThreads);
  hipStream_t st = (hipStream_t)stream;
  if (p.blocks[0].rows == 16)
    hipLaunchKernelGGL(attn_rows_kernel<1>, grid, block, 0, st, p);
  else
    hipLaunchKernelGGL(attn_rows_kernel<2>, grid, block, 0, st, p);
  const int rc = launched(who);
  return rc == CP_OK ? launch_attn_merge(p, stream, who) : rc;
}

}  // namespace cpattn
