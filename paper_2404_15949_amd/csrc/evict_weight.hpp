// the eviction decision by accumulated attention weight.
// Part of one translation unit: included by corm_blocks.hip, after select.hpp.
#ifndef CORM_EVICT_WEIGHT_HPP
#define CORM_EVICT_WEIGHT_HPP

namespace {

// The r newest slots stay, and the budget - r heaviest of the others, equal ones by the lower slot: the keys above a cut (select.hpp).

constexpr int EVW_WG = 1024, EVW_BITS = 11;
constexpr int EVW_KEYS = 16384;       // keys a workgroup holds in LDS (64 KB)

// Grid (units).
__global__ __launch_bounds__(EVW_WG) void corm_evict_weight_kernel(const float* weight, const int32_t* lens, uint8_t* keep, int Lcap,
                                                                   int r, int budget, int held) {
  extern __shared__ uint32_t sh_key[];   // held: the unit's keys
  __shared__ CutLds<EVW_WG, EVW_BITS> sh;
  const int unit = blockIdx.x, tid = threadIdx.x;
  const int L = min(max(lens[unit], 0), Lcap);
  const float* w = weight + (size_t)unit * Lcap;
  uint8_t* to = keep + (size_t)unit * Lcap;
  if (L <= budget) {
    for (int i = tid; i < L; i += EVW_WG) to[i] = 1;
    return;
  }
  const int open = L - r, k = budget - r;   // (0 <= k < open)
  Cut cut = {0xffffffffu, 0u};
  auto item = [&](int i, uint32_t& x, uint32_t& slot) {
    x = held ? sh_key[i] : order_key(w[i]);
    slot = (uint32_t)i;
    return true;
  };
  if (k > 0) {
    if (held)
      for (int i = tid; i < open; i += EVW_WG) sh_key[i] = order_key(w[i]);   // (a thread asks for its own)
    cut = find_cut<EVW_WG, EVW_BITS, 32>(open, (uint32_t)k, item, sh);
  }
  for (int i = tid; i < L; i += EVW_WG) {
    uint32_t x = 0u, slot;
    if (k > 0 && i < open) item(i, x, slot);
    to[i] = i >= open || (k > 0 && (x > cut.key || (x == cut.key && (uint32_t)i <= cut.last)));
  }
}

// Few long units: three launches, of which the first two share a unit among workgroups ("splits" of split_slots slots).
//   count    the top 11 bits of a split's keys
//   part     which of these digits the cut lies in; slots with a larger or a smaller one are decided, the others (as a rule a few percent)
//            are listed
//   settle   a workgroup a unit: the cut among the listed ones
// What they hand on lies in the workspace, written whole before it is read.
struct EvictLongArgs {
  const float* weight;
  const int32_t* lens;
  uint8_t* keep;
  uint32_t* hist;      // [units, splits, 2048]
  uint32_t* listed;    // [units, Lcap]: slots, a split's from its first slot on
  uint32_t* counts;    // [units, splits]
  uint2* digit;        // [units]: the digit of the cut, keys needed of it
  int32_t Lcap, r, budget, splits, split_slots;
};
constexpr int SETTLE_KEYS = 8192;
constexpr int EVW_SPLIT = 8192, EVW_MOST_SPLITS = 2048;   // slots of a split, at least (64 splits at most); splits of all units

__global__ __launch_bounds__(EVW_WG) void corm_evict_count_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_hist[1 << EVW_BITS];
  const int unit = blockIdx.y, split = blockIdx.x, tid = threadIdx.x;
  const int L = min(max(a.lens[unit], 0), a.Lcap);
  if (L <= a.budget) return;
  const float* w = a.weight + (size_t)unit * a.Lcap;
  const int first = split * a.split_slots, end = min(first + a.split_slots, L - a.r);
  for (int i = tid; i < (1 << EVW_BITS); i += EVW_WG) sh_hist[i] = 0u;
  __syncthreads();
  for (int i = first + tid; i < end; i += EVW_WG) atomicAdd(&sh_hist[order_key(w[i]) >> (32 - EVW_BITS)], 1u);
  __syncthreads();
  uint32_t* to = a.hist + ((size_t)unit * a.splits + split) * (1 << EVW_BITS);
  for (int i = tid; i < (1 << EVW_BITS); i += EVW_WG) to[i] = sh_hist[i];
}

__global__ __launch_bounds__(EVW_WG) void corm_evict_part_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_hist[1 << EVW_BITS], sh_pick[3], sh_n;
  const int unit = blockIdx.y, split = blockIdx.x, tid = threadIdx.x;
  const int L = min(max(a.lens[unit], 0), a.Lcap);
  const int first = split * a.split_slots, end = min(first + a.split_slots, L), open = L - a.r, k = a.budget - a.r;
  uint8_t* to = a.keep + (size_t)unit * a.Lcap;
  const bool all = L <= a.budget;
  if (all || k == 0) {
    for (int i = first + tid; i < end; i += EVW_WG) to[i] = all || i >= open;
    return;
  }
  const float* w = a.weight + (size_t)unit * a.Lcap;
  const uint32_t* hist = a.hist + (size_t)unit * a.splits * (1 << EVW_BITS);
  for (int i = tid; i < (1 << EVW_BITS); i += EVW_WG) {
    uint32_t sum = 0u;
#pragma unroll 16
    for (int s = 0; s < a.splits; ++s) sum += hist[(size_t)s * (1 << EVW_BITS) + i];
    sh_hist[i] = sum;
  }
  if (tid == 0) sh_n = 0u;
  __syncthreads();
  find_digit<EVW_WG, EVW_BITS>(sh_hist, sh_pick, (uint32_t)k);
  const uint32_t digit = sh_pick[0];
  uint32_t* list = a.listed + (size_t)unit * a.Lcap + first;
  for (int i = first + tid; i < end; i += EVW_WG) {
    const uint32_t x = i < open ? order_key(w[i]) >> (32 - EVW_BITS) : digit + 1u;
    if (x == digit) list[atomicAdd(&sh_n, 1u)] = (uint32_t)i;
    else to[i] = x > digit;
  }
  __syncthreads();
  if (tid == 0) {
    a.counts[(size_t)unit * a.splits + split] = sh_n;
    if (split == 0) a.digit[unit] = make_uint2(digit, sh_pick[1]);
  }
}

__global__ __launch_bounds__(EVW_WG) void corm_evict_settle_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_slot[SETTLE_KEYS], sh_key[SETTLE_KEYS];
  __shared__ CutLds<EVW_WG, EVW_BITS> sh;
  constexpr uint32_t LOW = (1u << (32 - EVW_BITS)) - 1u;
  const int unit = blockIdx.x, tid = threadIdx.x;
  const int L = min(max(a.lens[unit], 0), a.Lcap);
  if (L <= a.budget || a.budget == a.r) return;
  const float* w = a.weight + (size_t)unit * a.Lcap;
  uint8_t* to = a.keep + (size_t)unit * a.Lcap;
  const uint32_t* counts = a.counts + (size_t)unit * a.splits;
  const uint32_t* listed = a.listed + (size_t)unit * a.Lcap;
  const uint2 digit = a.digit[unit];
  const int lane = tid & 63, wv = tid >> 6;
  // (at most 64 splits: a lane each; what the lists in front of a split hold is where its own go)
  const uint32_t mine = lane < a.splits ? counts[lane] : 0u, upto = wave_prefix_sum(mine);
  const int total = __builtin_amdgcn_readlane((int)upto, 63);
  const bool held = total <= SETTLE_KEYS;
  if (held) {
    for (int s = wv; s < a.splits; s += EVW_WG / 64) {
      const int c = __builtin_amdgcn_readlane((int)mine, s), at = __builtin_amdgcn_readlane((int)upto, s) - c;
      for (int j = lane; j < c; j += 64) {
        const uint32_t slot = listed[(size_t)s * a.split_slots + j];
        sh_slot[at + j] = slot;
        sh_key[at + j] = order_key(w[slot]) & LOW;
      }
    }
    __syncthreads();
  }
  // (very many with one digit, as where all weights are equal: every slot is looked at in every round)
  const int n = held ? total : L - a.r;
  auto item = [&](int i, uint32_t& x, uint32_t& slot) {
    if (held) {
      x = sh_key[i];
      slot = sh_slot[i];
      return true;
    }
    const uint32_t full = order_key(w[i]);
    x = full & LOW;
    slot = (uint32_t)i;
    return full >> (32 - EVW_BITS) == digit.x;
  };
  const Cut cut = find_cut<EVW_WG, EVW_BITS, 32 - EVW_BITS>(n, digit.y, item, sh);
  for (int i = tid; i < n; i += EVW_WG) {
    uint32_t x, slot;
    if (item(i, x, slot)) to[slot] = x > cut.key || (x == cut.key && slot <= cut.last);
  }
}

}  // namespace

#endif  // CORM_EVICT_WEIGHT_HPP
