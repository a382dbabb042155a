// the eviction decision by accumulated attention weight.
// Part of one translation unit: included by corm_blocks.hip, after blocks.hpp.
#ifndef CORM_EVICT_WEIGHT_HPP
#define CORM_EVICT_WEIGHT_HPP

namespace {

constexpr int EVW_WG = 1024;

// Grid (units): keep of a unit.  The r newest slots stay, and the budget - r heaviest of the others (equal ones: the lowest slots).
__global__ __launch_bounds__(EVW_WG) void corm_evict_weight_kernel(const float* weight, const int32_t* lens, uint8_t* keep, int Lcap,
                                                                   int r, int budget) {
  __shared__ uint32_t sh_hist[256], sh_pick[2];
  __shared__ int sh_cnt[EVW_WG / 64];
  const int unit = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int L = min(max(lens[unit], 0), Lcap);
  const float* w = weight + (size_t)unit * Lcap;
  uint8_t* to = keep + (size_t)unit * Lcap;
  if (L <= budget) {
    for (int i = tid; i < L; i += EVW_WG) to[i] = 1;
    return;
  }
  const int open = L - r, k = budget - r;   // (budget >= r, so 0 <= k < open)
  uint2 cut = make_uint2(0xffffffffu, 0u);
  if (k > 0) cut = kth_largest<EVW_WG>(open, k, [&](int i) { return order_key(w[i]); }, sh_hist, sh_pick);
  int equal = 0;
  for (int i0 = 0; i0 < L; i0 += EVW_WG) {
    const int i = i0 + tid;
    const uint32_t x = i < open ? order_key(w[i]) : 0u;
    const bool eq = k > 0 && i < open && x == cut.x;
    const unsigned long long me = __ballot(eq);
    __syncthreads();
    if (lane == 0) sh_cnt[wv] = __popcll(me);
    __syncthreads();
    int ne = equal;
    for (int v = 0; v < EVW_WG / 64; ++v) {
      if (v < wv) ne += sh_cnt[v];
      equal += sh_cnt[v];
    }
    ne += __popcll(me & ((1ull << lane) - 1ull));
    if (i < L) to[i] = i >= open || (k > 0 && x > cut.x) || (eq && ne < (int)cut.y);
  }
}

}  // namespace

#endif  // CORM_EVICT_WEIGHT_HPP
