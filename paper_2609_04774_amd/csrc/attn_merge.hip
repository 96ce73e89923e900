// The combination of the parts of key walks that were cut between workgroups
// (attn_rows.hip, attn_chunk.hip).
#include <hip/hip_runtime.h>

#include "attn_tile.h"

namespace cpattn {

namespace {

using namespace tile;

// The parts of a walk (they cover disjoint keys): LSE = M + ln sum_k e^{LSE_k - M}, O
// = sum_k e^{LSE_k - LSE} O_k.  A walk's first part is the second slot of the share
// that it begins in, the others are the first slots of the shares that begin within
// it.  Block (x, y): the walk that share x + 1 begins within, if it is the first to do
// so; a wave takes kRows rows.
//
// Bound by latency for blocks of few rows: what tells the walk and its parts is read at
// once, and eight parts' rows are in flight (6 us, 64 parts or two; with the parts
// dealt to four waves, and the rows fetched along with their LSEs, 6 to 9).  Blocks of
// 384 rows: the 496 parts of 248 walks, 98 MB read and 25 written, take 32 us, 3.9 TB/s
// where a copy runs at 4.9; a wave's reads (starts, LSEs, rows) follow one another.
template <int kRows>
__global__ __launch_bounds__(256) void share_merge_kernel(PagedParams p) {
  constexpr int kParts = 8 / kRows;
  const int lane = threadIdx.x & 63;
  const int share = blockIdx.x + 1;
  const ShareStart none = {-1, 0, 0, 0};
  const ShareStart before = share > 1 ? p.starts[share - 1] : none;
  const ShareStart at = p.starts[share];
  ShareStart next = share + 1 + lane < p.n_shares ? p.starts[share + 1 + lane] : none;
  if (at.step == 0 || (same_walk(before, at) && before.step > 0)) return;
  const Blocks& b = p.blocks[p.choice ? *p.choice : 0];
  const Block x = block_at(p, b, at.place);
  const Segment& s = x.s;
  const int r0 = kRows * (4 * blockIdx.y + (threadIdx.x >> 6));  // of the block
  const int rows = s.n * p.G - x.block * b.rows;
  if (r0 >= rows || r0 >= b.rows) return;
  int n = 2;  // parts
  for (;;) {
    const uint64_t in = __builtin_amdgcn_ballot_w64(same_walk(next, at) && next.step > 0);
    if (in != ~0ull) {
      n += __builtin_ctzll(~in);
      break;
    }
    n += 64;
    next = share + n - 1 + lane < p.n_shares ? p.starts[share + n - 1 + lane] : none;
  }
  const size_t size = slot_floats(b.rows);
  auto slot_of = [&](int k) { return p.slots + (2 * (size_t)(share - 1 + k) + (k == 0 ? 1 : 0)) * size; };
  auto lse_of = [&](int k, int r) { return slot_of(k)[(size_t)b.rows * kHeadDim + r]; };
  float top[kRows], sum[kRows];
  float2 acc[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    top[i] = -INFINITY;
    sum[i] = 0.f;
    acc[i] = make_float2(0.f, 0.f);
  }
  for (int k = lane; k < n; k += 64)
#pragma unroll
    for (int i = 0; i < kRows; ++i) top[i] = __builtin_elementwise_maximum(top[i], lse_of(k, r0 + i));  // NaN if one is
#pragma unroll
  for (int i = 0; i < kRows; ++i)
#pragma unroll
    for (int k = 1; k < 64; k *= 2) top[i] = __builtin_elementwise_maximum(top[i], __shfl_xor(top[i], k));
  for (int k0 = 0; k0 < n; k0 += 64) {
    const int end = n - k0 < 64 ? n - k0 : 64;
    float w[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const float l = lane < end ? lse_of(k0 + lane, r0 + i) : -INFINITY;
      w[i] = l == -INFINITY ? 0.f : expf(l - top[i]);
      sum[i] += w[i];
    }
    for (int k = 0; k < end; k += kParts) {
      float2 v[kParts][kRows];
#pragma unroll
      for (int j = 0; j < kParts; ++j) {
        const float* slot = slot_of(k0 + (k + j < end ? k + j : end - 1));
#pragma unroll
        for (int i = 0; i < kRows; ++i)
          v[j][i] = reinterpret_cast<const float2*>(slot + (size_t)(r0 + i) * kHeadDim)[lane];
      }
      float wk[kParts][kRows];
#pragma unroll
      for (int j = 0; j < kParts; ++j)
#pragma unroll
        for (int i = 0; i < kRows; ++i)
          wk[j][i] = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w[i]), (k + j) & 63));
      // (A part without keys adds 0 times 0; an infinity or NaN shows whatever its weight.)
#pragma unroll
      for (int j = 0; j < kParts; ++j)
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float2 a = make_float2(acc[i].x + wk[j][i] * v[j][i].x, acc[i].y + wk[j][i] * v[j][i].y);
          acc[i] = k + j < end ? a : acc[i];
        }
    }
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum[i] += __shfl_xor(sum[i], k);
    if (r0 + i >= rows) continue;
    const float inv = top[i] == -INFINITY ? 0.f : 1.f / sum[i];
    const int row = x.block * b.rows + r0 + i;
    const int q = (int)((unsigned)row / (unsigned)p.G);
    const int64_t out = (s.o_row + q) * p.Hq + at.kvh * p.G + (row - q * p.G);
    reinterpret_cast<bf16x2*>(p.o + out * kHeadDim)[lane] = bf16x2{(__bf16)(acc[i].x * inv), (__bf16)(acc[i].y * inv)};
    if (lane == 0 && p.lse) p.lse[out] = top[i] == top[i] && top[i] != -INFINITY ? top[i] + logf(sum[i]) : -INFINITY;
  }
}

}  // namespace

int launch_attn_merge(const PagedParams& p, void* stream, const char* who) {
  if (p.n_shares == 1) return CP_OK;
  const unsigned shares = (unsigned)p.n_shares - 1;
  if (p.choice)  // few parts of many rows
    hipLaunchKernelGGL(share_merge_kernel<4>, dim3(shares, (unsigned)(p.blocks[p.n_ways - 1].rows / 16)), dim3(256), 0,
                       (hipStream_t)stream, p);
  else
    hipLaunchKernelGGL(share_merge_kernel<1>, dim3(shares, (unsigned)(p.blocks[0].rows / 4)), dim3(256), 0,
                       (hipStream_t)stream, p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CP_OK : fail(CP_ERR_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
}

}  // namespace cpattn
