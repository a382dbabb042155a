// the eviction decision by accumulated attention weight.
// Part of one translation unit: included by corm_blocks.hip, after select.hpp.
#ifndef CORM_EVICT_WEIGHT_HPP
#define CORM_EVICT_WEIGHT_HPP

namespace {

// The r newest slots stay, and the budget - r heaviest of the others, equal ones by the lower slot: the keys above a cut (select.hpp).

constexpr int EVW_WG = 1024, EVW_BITS = 11;
constexpr int EVW_KEYS = 16384;       // keys a workgroup holds in LDS (64 KB)

// f(i, key of w[i]) for the thread's i in [first, end); several loads in flight, as nothing in f has to be done first.
template <typename F>
__device__ __forceinline__ void for_keys(const float* w, int first, int end, const F& f) {
  constexpr int N = 4;
  for (int i0 = first + threadIdx.x; i0 < end; i0 += N * EVW_WG) {
    float x[N];
#pragma unroll
    for (int j = 0; j < N; ++j) x[j] = w[min(i0 + j * EVW_WG, end - 1)];
#pragma unroll
    for (int j = 0; j < N; ++j)
      if (i0 + j * EVW_WG < end) f(i0 + j * EVW_WG, order_key(x[j]));
  }
}

// Grid (units).  Bound by the chain of latencies: keys, two rounds of digits (about 2.5 us each: clear, count, find), the listed ones, the decision; 512 units
// x 4352 slots 9 us (10 MB).
__global__ __launch_bounds__(EVW_WG) void corm_evict_weight_kernel(const float* weight, const int32_t* lens, uint8_t* keep, int Lcap,
                                                                   int r, int budget) {
  extern __shared__ uint32_t sh_key[];   // the unit's keys
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
    x = sh_key[i];
    slot = (uint32_t)i;
    return true;
  };
  if (k > 0) {
    for_keys(w, 0, open, [&](int i, uint32_t x) { sh_key[i] = x; });   // (a thread asks for its own)
    cut = find_cut<EVW_WG, EVW_BITS, 32>(open, (uint32_t)k, item, sh);
  }
  for (int i = tid; i < L; i += EVW_WG) {
    uint32_t x = 0u, slot;
    if (k > 0 && i < open) item(i, x, slot);
    to[i] = i >= open || (k > 0 && (x > cut.key || (x == cut.key && (uint32_t)i <= cut.last)));
  }
}

// Long units: three launches, of which the first two share a unit among workgroups ("splits" of split_slots slots).
//   count    the top 11 bits of a split's keys, and the top 6 of those (so that the next launch reads a few kilobytes of a unit's counts and not
//            8 for every split: the dies' caches do not see each other's, and 16 units of 131072 slots took 12 us there)
//   part     which of these digits the cut lies in; slots with a larger or a smaller one are decided, the others (as a rule a few percent)
//            are listed
//   settle   a workgroup a unit: the cut among the listed ones
// What they hand on lies in the workspace, written whole before it is read.
struct EvictLongArgs {
  const float* weight;
  const int32_t* lens;
  uint8_t* keep;
  uint32_t* hist;      // [units, splits, 64 + 2048]: coarse counts, then fine ones
  uint32_t* listed;    // [units, Lcap]: slots, a split's from its first slot on
  uint32_t* counts;    // [units, splits]
  uint2* digit;        // [units]: the digit of the cut, keys needed of it
  int32_t Lcap, r, budget, splits, split_slots;
};
constexpr int SETTLE_KEYS = 8192;
constexpr int EVW_COARSE = 64, EVW_FINE = (1 << EVW_BITS) / EVW_COARSE, EVW_COUNTS = EVW_COARSE + (1 << EVW_BITS);   // counts of a split
constexpr int EVW_SPLIT = 8192;   // slots of a split, at least (64 splits at most)

__global__ __launch_bounds__(EVW_WG) void corm_evict_count_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_hist[1 << EVW_BITS];
  const int unit = blockIdx.y, split = blockIdx.x, tid = threadIdx.x;
  const int L = min(max(a.lens[unit], 0), a.Lcap);
  if (L <= a.budget) return;
  const float* w = a.weight + (size_t)unit * a.Lcap;
  const int first = split * a.split_slots, end = min(first + a.split_slots, L - a.r);
  for (int i = tid; i < (1 << EVW_BITS); i += EVW_WG) sh_hist[i] = 0u;
  __syncthreads();
  for_keys(w, first, end, [&](int, uint32_t x) { atomicAdd(&sh_hist[x >> (32 - EVW_BITS)], 1u); });
  __syncthreads();
  uint32_t* to = a.hist + ((size_t)unit * a.splits + split) * EVW_COUNTS;
  for (int i = tid; i < (1 << EVW_BITS); i += EVW_WG) {   // EVW_FINE neighbouring lanes have a coarse digit
    const uint32_t c = sh_hist[i];
    to[EVW_COARSE + i] = c;
    uint32_t sum = c;
#pragma unroll
    for (int o = 1; o < EVW_FINE; o <<= 1) sum += __shfl_xor(sum, o);
    if (i % EVW_FINE == 0) to[i / EVW_FINE] = sum;
  }
}

__global__ __launch_bounds__(EVW_WG) void corm_evict_part_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_hist[EVW_COARSE], sh_pick[3], sh_n;
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
  const uint32_t* hist = a.hist + (size_t)unit * a.splits * EVW_COUNTS;
  // the coarse digit of the cut, then the fine one in it; 64 counts of every split at a time (fine ones: half of them none)
  uint32_t need = (uint32_t)k, digit = 0u;
  if (tid == 0) sh_n = 0u;
#pragma unroll
  for (int round = 0; round < 2; ++round) {
    if (tid < EVW_COARSE) sh_hist[tid] = 0u;
    __syncthreads();
    const int c = tid % EVW_COARSE;
    uint32_t sum = 0u;
    if (round == 0 || c < EVW_FINE) {
      const int at = round == 0 ? c : EVW_COARSE + (int)digit * EVW_FINE + c;
#pragma unroll
      for (int s = tid / EVW_COARSE; s < 64; s += EVW_WG / EVW_COARSE)
        if (s < a.splits) sum += hist[(size_t)s * EVW_COUNTS + at];
    }
    if (sum) atomicAdd(&sh_hist[c], sum);
    __syncthreads();
    find_digit<EVW_WG, 6>(sh_hist, sh_pick, need);
    digit = digit * EVW_FINE + sh_pick[0];
    need = sh_pick[1];
    __syncthreads();
  }
  uint32_t* list = a.listed + (size_t)unit * a.Lcap + first;
  for_keys(w, first, end, [&](int i, uint32_t x) {
    x = i < open ? x >> (32 - EVW_BITS) : digit + 1u;
    if (x == digit) list[atomicAdd(&sh_n, 1u)] = (uint32_t)i;
    else to[i] = x > digit;
  });
  __syncthreads();
  if (tid == 0) {
    a.counts[(size_t)unit * a.splits + split] = sh_n;
    if (split == 0) a.digit[unit] = make_uint2(digit, need);
  }
}

__global__ __launch_bounds__(EVW_WG) void corm_evict_settle_kernel(const EvictLongArgs a) {
  __shared__ uint32_t sh_slot[SETTLE_KEYS], sh_key[SETTLE_KEYS], sh_count[64];
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
  if (wv == 0) sh_count[lane] = mine;
  if (held) {
    for (int s = wv; s < a.splits; s += EVW_WG / 64) {
      const int c = __builtin_amdgcn_readlane((int)mine, s), at = __builtin_amdgcn_readlane((int)upto, s) - c;
      for (int j = lane; j < c; j += 64) {
        const uint32_t slot = listed[(size_t)s * a.split_slots + j];
        sh_slot[at + j] = slot;
        sh_key[at + j] = order_key(w[slot]) & LOW;
      }
    }
  }
  __syncthreads();
  // More than that have the digit (accounts within a factor of two or three, or very many slots): they are walked from memory in every round, by their
  // lists, side by side in rows of 2^shift places; but where over a quarter of the slots is listed, slot by slot, which is one load less in a chain.
  // Whole calls, us, slots | lists: lognormal accounts of sigma 2, a sixteenth kept, 8 units x 1048576 1026 | 60; of 0.5, half kept (a seventh listed),
  // 16 x 131072 102 | 58, 8 x 1048576 1065 | 460, 256 x 100000 203 | 147; of 0.18 (two fifths) 94 | 101, 1170 | 1333, 213 | 203; all equal 404 | 477,
  // 3248 | 4388, 478 | 585.
  uint32_t most = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, o));
  const int shift = 32 - __clz((int)max(most, 2u) - 1);
  auto settle = [&](int n, const auto& item) {
    const Cut cut = find_cut<EVW_WG, EVW_BITS, 32 - EVW_BITS>(n, digit.y, item, sh);
    for (int i = tid; i < n; i += EVW_WG) {
      uint32_t x, slot;
      if (item(i, x, slot)) to[slot] = x > cut.key || (x == cut.key && slot <= cut.last);
    }
  };
  if (held) {
    settle(total, [&](int i, uint32_t& x, uint32_t& slot) {
      x = sh_key[i];
      slot = sh_slot[i];
      return true;
    });
  } else if (total <= (L - a.r) / 4) {
    settle(a.splits << shift, [&](int i, uint32_t& x, uint32_t& slot) {
      const uint32_t s = (uint32_t)i >> shift, j = (uint32_t)i & ((1u << shift) - 1u);
      if (j >= sh_count[s]) return false;
      slot = listed[(size_t)s * a.split_slots + j];
      x = order_key(w[slot]) & LOW;
      return true;
    });
  } else {
    settle(L - a.r, [&](int i, uint32_t& x, uint32_t& slot) {
      const uint32_t full = order_key(w[i]);
      x = full & LOW;
      slot = (uint32_t)i;
      return full >> (32 - EVW_BITS) == digit.x;
    });
  }
}

}  // namespace

#endif  // CORM_EVICT_WEIGHT_HPP
