// the k-th largest of many numbers, by a workgroup.
// Part of one translation unit: included by corm_blocks.hip, after common.hpp.
#ifndef CORM_SELECT_HPP
#define CORM_SELECT_HPP

namespace {

// An fp32 number as an unsigned one of the same order (-0 as 0, what is not a number below all others).
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The border between what is chosen and what is not: chosen are the keys above `key` and, of those equal to it, the ones in slots up to `last`.
struct Cut {
  uint32_t key, last;
};
constexpr uint32_t SLOT_TOP = (1u << 22) - 1u;   // not below any slot (Lcap < 2^22)

// Sum over this lane and the lanes below it, by row shifts and row broadcasts of the vector ALU.
__device__ __forceinline__ uint32_t wave_prefix_sum(uint32_t x) {
#define CORM_ADD_DPP(CTRL, ROWS) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, true)
  CORM_ADD_DPP(0x111, 0xf);   // row_shr:1, 2, 4, 8: sums inside the rows of 16
  CORM_ADD_DPP(0x112, 0xf);
  CORM_ADD_DPP(0x114, 0xf);
  CORM_ADD_DPP(0x118, 0xf);
  CORM_ADD_DPP(0x142, 0xa);   // row_bcast:15 into rows 1 and 3
  CORM_ADD_DPP(0x143, 0xc);   // row_bcast:31 into rows 2 and 3
#undef CORM_ADD_DPP
  return x;
}

// From counts of the 2^BITS digits in sh_hist: the digit in which the need-th largest lies -> sh_pick = (digit, how many of its keys are
// needed, how many it has).  By NT threads; sh_pick is ready behind the barrier at the end.
template <int NT, int BITS>
__device__ __forceinline__ void find_digit(const uint32_t* sh_hist, uint32_t* sh_pick, uint32_t need) {
  constexpr int BINS = 1 << BITS, W = BINS <= 256 ? 64 : BINS / 4 < NT ? BINS / 4 : NT, PER = BINS / W;   // threads with digits, digits of a thread
  __shared__ uint32_t sh_sum[W / 64];
  const int t = threadIdx.x;
  uint32_t c[PER], sum = 0u, before = 0u;
  if (t < W) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {   // from the largest digit down
      c[j] = sh_hist[BINS - 1 - PER * t - j];
      sum += c[j];
    }
    before = wave_prefix_sum(sum);
    if (W > 64 && (t & 63) == 63) sh_sum[t >> 6] = before;
    before -= sum;
  }
  if (W > 64) {
    __syncthreads();
    for (int w = 0; w < W / 64; ++w) before += w < (t >> 6) ? sh_sum[w] : 0u;
  }
  if (t < W) {
#pragma unroll
    for (int j = 0; j < PER; ++j) {
      if (before < need && before + c[j] >= need) {
        sh_pick[0] = (uint32_t)(BINS - 1 - PER * t - j);
        sh_pick[1] = need - before;
        sh_pick[2] = c[j];
      }
      before += c[j];
    }
  }
  __syncthreads();
}

// Keys that are counted against each other (512 units x 4352 weights, us: 64 8.9, 128 8.9, 256 9.0; 512 x 1500 10.5, 7.7, 7.1).
constexpr int CUT_LISTED = 128;

// Memory of find_cut.
template <int NT, int BITS>
struct CutLds {
  unsigned long long listed[CUT_LISTED];
  uint32_t hist[1 << BITS], pick[3], n, front[CUT_LISTED];
  static_assert(NT % CUT_LISTED == 0, "whole groups of threads");
};

// One digit: of the keys that item(i, x, slot) gives for i < n (where it says so) and that agree with `prefix` above their low `open` bits, BITS bits
// from there down are counted in LDS -> sh.pick, as find_digit leaves it.
template <int NT, int BITS, typename Item>
__device__ __forceinline__ void cut_round(int n, uint32_t need, uint32_t prefix, int open, const Item& item, CutLds<NT, BITS>& sh) {
  const int shift = max(open - BITS, 0);   // (the last digit may overlap the one before)
  for (int i = threadIdx.x; i < (1 << BITS); i += NT) sh.hist[i] = 0u;
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += NT) {
    uint32_t x, slot;
    if (item(i, x, slot) && (open >= 32 || (x >> (open & 31)) == (prefix >> (open & 31)))) atomicAdd(&sh.hist[(x >> shift) & ((1u << BITS) - 1u)], 1u);
  }
  __syncthreads();
  find_digit<NT, BITS>(sh.hist, sh.pick, need);
}

// The cut that leaves k (1 <= k <= the number of keys) above it, by the whole workgroup.  item(i, x, slot): key below 2^TOP and slot number i of
// n, or false; asked several times, for the same i by the same thread.  Digits from the top until few keys are left in the digit of
// the cut (with weights and scores after one or two); these are listed, and each is counted against all others.  With
// many keys 11 bits a digit rather than 8: an exponent alone has few values, so that the lanes of a wave would count in the same words (512 units of
// 4352 weights 48 us with 8 bits, 9.3 with 11; 512 scores a unit 1.5 us less with 8).
template <int NT, int BITS, int TOP, typename Item>
__device__ __forceinline__ Cut find_cut(int n, uint32_t k, const Item& item, CutLds<NT, BITS>& sh) {
  uint32_t prefix = 0u, need = k, have = (uint32_t)n;
  int open = TOP;
  while (have > (uint32_t)CUT_LISTED && open > 0) {   // (uniform)
    cut_round<NT, BITS>(n, need, prefix, open, item, sh);
    prefix |= sh.pick[0] << max(open - BITS, 0);
    need = sh.pick[1];
    have = sh.pick[2];
    open = max(open - BITS, 0);
    __syncthreads();
  }
  if (have <= (uint32_t)CUT_LISTED) {
    if (threadIdx.x == 0) sh.n = 0u;
    if (threadIdx.x < CUT_LISTED) sh.front[threadIdx.x] = 0u;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
      uint32_t x, slot;
      if (item(i, x, slot) && (open >= 32 || (x >> (open & 31)) == (prefix >> (open & 31))))
        sh.listed[atomicAdd(&sh.n, 1u)] = (unsigned long long)x << 32 | (SLOT_TOP - slot);
    }
    __syncthreads();
    // each listed key against all others, NT / CUT_LISTED threads a key
    const uint32_t m = sh.n, mine_at = threadIdx.x % CUT_LISTED;
    if (mine_at < m) {
      const unsigned long long mine = sh.listed[mine_at];
      uint32_t front = 0u;
#pragma unroll 4
      for (uint32_t j = threadIdx.x / CUT_LISTED; j < m; j += NT / CUT_LISTED) front += sh.listed[j] > mine;
      if (front) atomicAdd(&sh.front[mine_at], front);
    }
    __syncthreads();
    if (threadIdx.x < m && sh.front[threadIdx.x] == need - 1u) {
      const unsigned long long mine = sh.listed[threadIdx.x];
      sh.pick[0] = (uint32_t)(mine >> 32);
      sh.pick[1] = SLOT_TOP - (uint32_t)mine;
    }
    __syncthreads();
    const Cut cut = {sh.pick[0], sh.pick[1]};
    __syncthreads();
    return cut;
  }
  // more equal keys than the list holds: the need-th lowest of their slots, by digits of the slots
  Cut cut = {prefix, SLOT_TOP};
  if (need == have) return cut;
  auto slots = [&](int i, uint32_t& x, uint32_t& slot) {
    uint32_t key;
    const bool ok = item(i, key, slot) && key == prefix;
    x = SLOT_TOP - slot;
    return ok;
  };
  uint32_t high = 0u;
  for (int left = 22; left > 0; left = max(left - BITS, 0)) {
    cut_round<NT, BITS>(n, need, high, left, slots, sh);
    high |= sh.pick[0] << max(left - BITS, 0);
    need = sh.pick[1];
    __syncthreads();
  }
  cut.last = SLOT_TOP - high;
  return cut;
}

}  // namespace

#endif  // CORM_SELECT_HPP
