// The combination of the parts of key walks that were cut between workgroups
// (attn_rows.hip, attn_chunk.hip).
#include <hip/hip_runtime.h>

#include "attn_tile.h"

namespace cpattn {

namespace {

using namespace tile;

// The parts of a walk that was cut, combined (they cover disjoint keys): LSE = M +
// ln sum_k e^{LSE_k - M}, O = sum_k e^{LSE_k - LSE} O_k.  A walk's first part is
// the second slot of the share that it begins in, the others are the first slots of
// the shares that begin within it.  Block (x, y): the walk that share x begins
// within, if it is the first to do so, rows 4 y .. 4 y + 3, one wave each.
__global__ __launch_bounds__(256) void share_merge_kernel(PagedParams p) {
  const int share = blockIdx.x + 1;
  const ShareStart at = p.starts[share];
  if (at.step == 0) return;
  if (share > 1) {
    const ShareStart before = p.starts[share - 1];
    if (same_walk(before, at) && before.step > 0) return;
  }
  const Segment s = segment_at(p, at.segment);
  const int lane = threadIdx.x & 63;
  const int r = 4 * blockIdx.y + (threadIdx.x >> 6);
  const int row = at.block * p.block_rows + r;
  if (r >= p.block_rows || row >= s.n * p.G) return;
  const size_t size = slot_floats(p.block_rows);
  // The walk's shares: this one and those after it that begin within the walk.
  int n = 1;
  for (;; n += 64) {
    const int k = share + n + lane;
    bool in = k < p.n_shares;
    if (in) {
      const ShareStart x = p.starts[k];
      in = same_walk(x, at) && x.step > 0;
    }
    const uint64_t mask = __builtin_amdgcn_ballot_w64(in);
    if (mask != ~0ull) {
      n += __builtin_ctzll(~mask);
      break;
    }
  }
  // Part 0 lies in the share before; part k in share + k - 1.
  auto slot_of = [&](int k) { return p.slots + (2 * (size_t)(share - 1 + k) + (k == 0 ? 1 : 0)) * size; };
  auto lse_of = [&](int k) { return slot_of(k)[(size_t)p.block_rows * kHeadDim + r]; };
  float top = -INFINITY;
  for (int k = lane; k <= n; k += 64) top = __builtin_elementwise_maximum(top, lse_of(k));
#pragma unroll
  for (int k = 1; k < 64; k *= 2) top = __builtin_elementwise_maximum(top, __shfl_xor(top, k));
  float2 acc = make_float2(0.f, 0.f);
  float sum = 0.f;
  if (top != -INFINITY) {
    for (int k0 = 0; k0 <= n; k0 += 64) {
      const float l = k0 + lane <= n ? lse_of(k0 + lane) : -INFINITY;
      const float w = l == -INFINITY ? 0.f : expf(l - top);
      sum += w;
      const int end = n + 1 - k0 < 64 ? n + 1 - k0 : 64;
      for (int k = 0; k < end; ++k) {
        const float wk = __shfl(w, k);
        const float2 v = reinterpret_cast<const float2*>(slot_of(k0 + k) + (size_t)r * kHeadDim)[lane];
        acc.x += wk * v.x;
        acc.y += wk * v.y;
      }
    }
#pragma unroll
    for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
    acc.x /= sum;
    acc.y /= sum;
  }
  const int i = (int)((unsigned)row / (unsigned)p.G);
  const int64_t out = (s.o_row + i) * p.Hq + at.kvh * p.G + (row - i * p.G);
  const bf16x2 v = {(__bf16)acc.x, (__bf16)acc.y};
  reinterpret_cast<bf16x2*>(p.o + out * kHeadDim)[lane] = v;
  if (lane == 0 && p.lse) p.lse[out] = top == top && top != -INFINITY ? top + logf(sum) : -INFINITY;
}

}  // namespace

int launch_attn_merge(const PagedParams& p, void* stream, const char* who) {
  if (p.n_shares == 1) return CP_OK;
  hipLaunchKernelGGL(share_merge_kernel, dim3((unsigned)p.n_shares - 1, (unsigned)(p.block_rows / 4)), dim3(256), 0,
                     (hipStream_t)stream, p);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CP_OK : fail(CP_ERR_HIP, std::string(who) + " launch: " + hipGetErrorString(e));
}

}  // namespace cpattn
