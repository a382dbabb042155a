// attention over chosen blocks: bounds of the blocks' keys, the choice, and decode attention over what was chosen.
// Part of one translation unit: included by corm_blocks.hip, after common.hpp, attend.hpp and q8.hpp.
#ifndef CORM_BLOCKS_HPP
#define CORM_BLOCKS_HPP

namespace {

// ---------------------------------------------------------------- bounds

// Grid (blocks, units), or (1 or a few, units) for the newest: block `from + blockIdx.x` of a unit, counted from its first (newest <= 0) or from the
// block that holds slot lens - newest.  A wave reads whole rows, 16 bytes a lane, and keeps the smallest and largest of its channels;
// lanes of the same slice and the waves meet at the end.  Bound by HBM: 512 units of up to 4096 rows of 256 bytes 73 us, 6.2 TB/s.
template <typename DT, int D>
__global__ __launch_bounds__(WG) void corm_block_bounds_kernel(const char* K, const int32_t* lens, char* bounds, int Lcap, int nblk,
                                                               int newest) {
  constexpr int EPL = DT::EPL, ROWB = D * DT::ESZ, LPR = ROWB / 16, RPL = 64 / LPR, LOADS = QBLK / (RPL * WAVES);
  __shared__ float sh[2][WAVES][D];
  const int unit = blockIdx.y, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int L = min(max(lens[unit], 0), Lcap);
  const int blk = (newest > 0 ? max(L - newest, 0) / QBLK : 0) + blockIdx.x;
  if (blk * QBLK >= L) return;
  const int rows = min(L - blk * QBLK, QBLK);
  const int sub = lane / LPR, cl = lane % LPR;
  const char* at = K + ((size_t)unit * Lcap + (size_t)blk * QBLK) * ROWB + (size_t)cl * 16;
  float lo[EPL], hi[EPL];
#pragma unroll
  for (int e = 0; e < EPL; ++e) {
    lo[e] = __builtin_inff();
    hi[e] = neg_inf();
  }
  uint4 x[LOADS];
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {   // (rows past the last: the last again, which changes nothing)
    const int row = min((j * WAVES + wv) * RPL + sub, rows - 1);
    x[j] = load_once(at + (size_t)row * ROWB);
  }
#pragma unroll
  for (int j = 0; j < LOADS; ++j)
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      lo[e] = fminf(lo[e], element<DT>(x[j], e));
      hi[e] = fmaxf(hi[e], element<DT>(x[j], e));
    }
#pragma unroll
  for (int o = LPR; o < 64; o <<= 1)
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      lo[e] = fminf(lo[e], __shfl_xor(lo[e], o));
      hi[e] = fmaxf(hi[e], __shfl_xor(hi[e], o));
    }
  if (sub == 0) {
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      sh[0][wv][cl * EPL + e] = lo[e];
      sh[1][wv][cl * EPL + e] = hi[e];
    }
  }
  __syncthreads();
  char* to = bounds + ((size_t)unit * nblk + blk) * 2 * ROWB;
  for (int i = threadIdx.x; i < 2 * D; i += WG) {
    const int s = i / D, c = i % D;
    float v = sh[s][0][c];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = s ? fmaxf(v, sh[s][w][c]) : fminf(v, sh[s][w][c]);
    put_element<DT>(to + (size_t)i * DT::ESZ, v);
  }
}

// ---------------------------------------------------------------- the choice

// Upper bound of a block's logits: sum over channels of the larger of q*lo and q*hi, which is q+ * hi + q- * lo; the largest over the
// heads of the group.  In 64 bits, rounded once to fp32, so that the choice does not hang on the order of a sum (two blocks
// next to each other at the border of the choice differ by 1e-5 of their scores now and then, never by 1e-15).
// q- (taken with the smaller elements) and q+ (with the larger) of the group's heads; what is not a number is so in both.  Ends without a barrier.
template <typename DT, int D, int G, int NT>
__device__ __forceinline__ void stage_signed_q(const char* qu, double2 (&sh_q)[G][D]) {
  for (int i = threadIdx.x; i < G * D; i += NT) {
    const float x = DT::ESZ == 2 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(qu)[i] << 16)
                                 : reinterpret_cast<const float*>(qu)[i];
    sh_q[i / D][i % D] = make_double2((double)(x > 0.f ? 0.f : x), (double)(x < 0.f ? 0.f : x));
  }
}

// A share of the channels of the lane's block (bounds at `at`): its sums for every head.  The definition takes the larger product whichever of the two bounds it
// is of, and so does this.  (From the bounds' sum and distance one number of a query per channel would do, a little faster, but one bound of 1e30 would take
// all digits of the other.)
template <typename DT, int D, int G, int SHARES>
__device__ __forceinline__ void share_score(const char* at, int share, const double2 (&sh_q)[G][D], double (&sum)[G]) {
  // pieces of 16 bytes, STEP of them in flight from both rows
  constexpr int EPL = DT::EPL, ROWB = D * DT::ESZ, PIECES = ROWB / 16 / SHARES, CH = D / SHARES, STEP = PIECES < 2 ? PIECES : 2;
  at += (size_t)share * (PIECES * 16);
#pragma unroll
  for (int g = 0; g < G; ++g) sum[g] = 0.;
#pragma unroll
  for (int j0 = 0; j0 < PIECES; j0 += STEP) {
    uint4 x[STEP], y[STEP];
#pragma unroll
    for (int j = 0; j < STEP; ++j) {
      x[j] = *reinterpret_cast<const uint4*>(at + (size_t)(j0 + j) * 16);
      y[j] = *reinterpret_cast<const uint4*>(at + (size_t)ROWB + (size_t)(j0 + j) * 16);
    }
#pragma unroll
    for (int j = 0; j < STEP; ++j)
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const float a = element<DT>(x[j], e), b = element<DT>(y[j], e);   // (whichever is the smaller)
        const double lo = (double)fminf(a, b), hi = (double)fmaxf(a, b);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const double2 h = sh_q[g][share * CH + (j0 + j) * EPL + e];
          sum[g] = fma(hi, h.y, fma(lo, h.x, sum[g]));
        }
      }
  }
}

// The shares' sums of the lane's block -> its score, from the heads for which it is a number.
template <int G, int SHARES>
__device__ __forceinline__ float joined_score(const double (&part)[SHARES][G][64]) {
  const int lane = threadIdx.x & 63;
  double best = 0.;
#pragma unroll
  for (int g = 0; g < G; ++g) {
    double t = part[0][g][lane];
#pragma unroll
    for (int s = 1; s < SHARES; ++s) t += part[s][g][lane];
    best = g == 0 ? t : fmax(best, t);
  }
  return (float)best;
}

// Grid (groups of 64 blocks, units).  Lane = block, wave = an eighth of the channels: what bounds it are the chains of 64-bit products behind the queries'
// LDS reads, and more waves have shorter ones (whole steps of 128 units x 440 blocks by 2 | 4 | 8 | 16 waves, us: 73.7 | 71.4 | 68.9 | 70.7).
constexpr int SCORE_SHARES = 8;
template <typename DT, int D, int G>
__global__ __launch_bounds__(64 * SCORE_SHARES) void corm_block_score_kernel(const char* q, const char* bounds, const int32_t* lens, float* scores,
                                                              int Lcap, int nblk) {
  constexpr int ROWB = D * DT::ESZ;
  __shared__ double2 sh_q[G][D];
  __shared__ double sh_part[SCORE_SHARES][G][64];
  const int unit = blockIdx.y, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int L = min(max(lens[unit], 0), Lcap), used = (L + QBLK - 1) / QBLK;
  const int blk = blockIdx.x * 64 + lane;
  if ((int)blockIdx.x * 64 >= used) return;
  stage_signed_q<DT, D, G, 64 * SCORE_SHARES>(q + (size_t)unit * G * ROWB, sh_q);
  __syncthreads();
  double sum[G];
  share_score<DT, D, G, SCORE_SHARES>(bounds + ((size_t)unit * nblk + min(blk, used - 1)) * 2 * ROWB, wv, sh_q, sum);
#pragma unroll
  for (int g = 0; g < G; ++g) sh_part[wv][g][lane] = sum[g];
  __syncthreads();
  if (wv == 0 && blk < used) scores[(size_t)unit * nblk + blk] = joined_score<G, SCORE_SHARES>(sh_part);
}

// The choice of a unit from the order_keys of its blocks below `open` (key(i)), by a workgroup of NT threads.
template <int NT, typename Key>
__device__ __forceinline__ void pick_blocks(int used, int nsel, int nlast, int32_t* to, const Key& key, CutLds<NT, 8>& sh, int* sh_cnt) {
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int chosen = min(used, nsel), open = used - min(nlast, used), k = chosen - (used - open);   // blocks to choose from, how many
  for (int i = chosen + tid; i < nsel; i += NT) to[i] = -1;
  if (k == open) {   // all of them
    for (int i = tid; i < chosen; i += NT) to[i] = i;
    return;
  }
  for (int i = tid; i < used - open; i += NT) to[k + i] = open + i;
  if (k == 0) return;
  auto item = [&](int i, uint32_t& x, uint32_t& slot) {
    x = key(i);
    slot = (uint32_t)i;
    return true;
  };
  const Cut cut = find_cut<NT, 8, 32>(open, (uint32_t)k, item, sh);
  int before = 0;   // chosen in front of this tile
  for (int i0 = 0; i0 < open; i0 += NT) {
    const int i = i0 + tid;
    const uint32_t x = i < open ? key(i) : 0u;
    const bool in = i < open && (x > cut.key || (x == cut.key && (uint32_t)i <= cut.last));
    const unsigned long long mask = __ballot(in);
    __syncthreads();
    if (lane == 0) sh_cnt[wv] = __popcll(mask);
    __syncthreads();
    int at = before + __popcll(mask & ((1ull << lane) - 1ull));
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
      at += w < wv ? sh_cnt[w] : 0;
      before += sh_cnt[w];
    }
    if (in) to[at] = i;
  }
}

// Grid (units): the nlast newest blocks and the best of the others, ascending, -1 behind them.
// The keys are read once where they fit in LDS (scores of 262144 slots), else in every round from memory.
constexpr int PICK_WG = 256, PICK_KEYS = 4096;
__global__ __launch_bounds__(PICK_WG) void corm_block_pick_kernel(const float* scores, const int32_t* lens, int32_t* blocks, int Lcap,
                                                                  int nblk, int nsel, int nlast) {
  __shared__ CutLds<PICK_WG, 8> sh;
  __shared__ uint32_t sh_key[PICK_KEYS];
  __shared__ int sh_cnt[PICK_WG / 64];
  const int unit = blockIdx.x;
  const int L = min(max(lens[unit], 0), Lcap), used = (L + QBLK - 1) / QBLK, open = max(used - nlast, 0);
  const float* sc = scores + (size_t)unit * nblk;
  const bool held = open <= PICK_KEYS;
  if (held)
    for (int i = threadIdx.x; i < open; i += PICK_WG) sh_key[i] = order_key(sc[i]);   // (a thread reads back its own)
  pick_blocks<PICK_WG>(used, nsel, nlast, blocks + (size_t)unit * nsel, [&](int i) { return held ? sh_key[i] : order_key(sc[i]); }, sh,
                       sh_cnt);
}

// Scores and choice in one launch, a workgroup a unit, where a unit has few blocks: a launch less, but the scores of a unit are then one compute unit's
// work.  Whole steps, us, one launch | two: 288 units x 5 blocks 23.5 | 28.0, 34 x 10 19.6 | 23.1, 32 x 44 23.2 | 27.2, 256 x 65 39.8 | 42.4, 8 x 127
// 17.5 | 18.3, 8 x 251 19.3 | 18.0, 64 x 257 50.2 | 48.2, 8 x 513 25.7 | 20.1.
constexpr int CHOOSE_BLOCKS = 128, CHOOSE_WG = CHOOSE_BLOCKS * WAVES;
template <typename DT, int D, int G>
__global__ __launch_bounds__(CHOOSE_WG) void corm_block_choose_kernel(const char* q, const char* bounds, const int32_t* lens,
                                                                      int32_t* blocks, int Lcap, int nblk, int nsel, int nlast) {
  constexpr int ROWB = D * DT::ESZ;
  __shared__ double2 sh_q[G][D];
  __shared__ double sh_part[CHOOSE_BLOCKS / 64][WAVES][G][64];
  __shared__ uint32_t sh_key[CHOOSE_BLOCKS];
  __shared__ CutLds<CHOOSE_WG, 8> sh;
  __shared__ int sh_cnt[CHOOSE_WG / 64];
  const int unit = blockIdx.x, lane = threadIdx.x & 63, wv = threadIdx.x >> 6, grp = wv / WAVES, quarter = wv % WAVES;
  const int L = min(max(lens[unit], 0), Lcap), used = (L + QBLK - 1) / QBLK, open = max(used - nlast, 0);
  if (nsel < used && open > 0) {   // (else all of them are chosen, or the newest; these need no score)
    const int blk = grp * 64 + lane;
    stage_signed_q<DT, D, G, CHOOSE_WG>(q + (size_t)unit * G * ROWB, sh_q);
    __syncthreads();
    if (grp * 64 < open) {   // (uniform over the wave)
      double sum[G];
      share_score<DT, D, G, WAVES>(bounds + ((size_t)unit * nblk + min(blk, open - 1)) * 2 * ROWB, quarter, sh_q, sum);
#pragma unroll
      for (int g = 0; g < G; ++g) sh_part[grp][quarter][g][lane] = sum[g];
    }
    __syncthreads();
    if (quarter == 0 && blk < open) sh_key[blk] = order_key(joined_score<G, WAVES>(sh_part[grp]));
    __syncthreads();
  }
  pick_blocks<CHOOSE_WG>(used, nsel, nlast, blocks + (size_t)unit * nsel, [&](int i) { return sh_key[i]; }, sh, sh_cnt);
}

// ---------------------------------------------------------------- attention over the listed blocks

struct BlockAttendArgs {
  const char* q;
  const char* K;
  const char* V;
  const int32_t* lens;
  const int32_t* blocks;
  float* partials;
  float* out;
  int32_t* status;
  int32_t Lcap, nsel, part_blocks;
  int32_t npart;   // partials per head; with one the workgroup writes out itself
  float scale_log2;
};

constexpr int LIST_PART = 8;   // listed blocks per workgroup, at most

// The workgroup's part of the list: sh_first = first slot of each block, L where there is none.  Returns the unit's length L, and how many places
// of the part are to be looked at (up to its last block).  Ends with a barrier.
__device__ __forceinline__ int2 listed_blocks(const BlockAttendArgs& a, int unit, int* sh_first) {
  const int lane = threadIdx.x & 63, at = blockIdx.x * a.part_blocks + lane;
  int L = a.lens[unit], flags = 0;
  if (L < 0 || L > a.Lcap) {
    flags = CORM_DEV_BAD_LENS;
    L = L < 0 ? 0 : a.Lcap;
  }
  const int id = lane < a.part_blocks && at < a.nsel ? a.blocks[(size_t)unit * a.nsel + at] : -1;   // (every wave asks, for the count)
  const bool ok = id >= 0 && id < (L + QBLK - 1) / QBLK;
  if (!ok && id != -1) flags |= CORM_DEV_BAD_BLOCK;
  const unsigned long long mask = __ballot(ok);
  if (threadIdx.x < LIST_PART) {
    sh_first[lane] = ok ? id * QBLK : L;
    if (flags && a.status) atomicOr(a.status, flags);
  }
  __syncthreads();
  return make_int2(L, mask ? 64 - __clzll((long long)mask) : 0);
}

// A part without blocks: nothing to add.
template <int D, int G>
__device__ __forceinline__ void empty_partial(const BlockAttendArgs& a, int unit) {
  if (a.npart == 1) {
    for (int i = threadIdx.x; i < G * D; i += WG) a.out[(size_t)unit * G * D + i] = 0.f;
  } else if (threadIdx.x < G) {   // (the merge takes no sums of a partial with this maximum)
    float* part = partial_of(a.partials, unit * G + threadIdx.x, a.npart, blockIdx.x, D);
    part[0] = neg_inf();
    part[1] = 0.f;
  }
}

// The waves' sums, folded into the workgroup's partial.
template <int D, int G>
__device__ __forceinline__ void block_partial(const BlockAttendArgs& a, int unit, const float (&sh_m)[G][WAVES], const float (&sh_z)[G][WAVES],
                                              const float (&sh_acc)[G][WAVES][D]) {
  for (int idx = threadIdx.x; idx < G * D; idx += WG) {
    const int g = idx / D, c = idx - g * D;
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mx = fmaxf(mx, sh_m[g][i]);
    const float ms = mx == neg_inf() ? 0.f : mx;
    float zt = 0.f, at = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float f = fast_exp2(sh_m[g][i] - ms);
      zt = fmaf(sh_z[g][i], f, zt);
      at = fmaf(sh_acc[g][i][c], f, at);
    }
    if (a.npart == 1) {
      a.out[(size_t)(unit * G + g) * D + c] = zt == 0.f ? 0.f : at / zt;
      continue;
    }
    float* part = partial_of(a.partials, unit * G + g, a.npart, blockIdx.x, D);
    part[2 + c] = at;
    if (c == 0) {
      part[0] = mx;
      part[1] = zt;
    }
  }
}

// Grid (parts of the list, units).  The rows of the listed blocks, one behind the other, are streamed as corm_attend_kernel streams a chunk;
// a lane looks the block of its row up in LDS, and rows that are not in use get an offset past the descriptor's end.  Bound by HBM with one and
// two heads (5.5 TB/s), by the vector ALU with eight.
template <typename DT, int D, int G>
__global__ __launch_bounds__(WG) void corm_block_attend_kernel(const BlockAttendArgs a) {
  using A = Attend<DT, D, G, WAVES>;
  constexpr int EPL = A::EPL, ROWB = A::ROWB, LPR = A::LPR, RPL = A::RPL;
  constexpr int ROWS = LIST_PART * QBLK;
  __shared__ float sh_m[G][WAVES], sh_z[G][WAVES];
  __shared__ float sh_acc[G][WAVES][D];
  __shared__ float sh_logit[G][ROWS];
  __shared__ int sh_first[LIST_PART];
  const int unit = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int sub = lane / LPR, cl = lane % LPR;
  const int2 listed = listed_blocks(a, unit, sh_first);
  const int L = listed.x, count = listed.y;
  if (count == 0) return empty_partial<D, G>(a, unit);

  uint4 qreg[G];
#pragma unroll
  for (int g = 0; g < G; ++g) qreg[g] = *reinterpret_cast<const uint4*>(a.q + ((size_t)unit * G + g) * ROWB + (size_t)cl * 16);
  float m_run[G], z_run[G], acc[G][EPL];
#pragma unroll
  for (int g = 0; g < G; ++g) {
    m_run[g] = neg_inf();
    z_run[g] = 0.f;
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[g][e] = 0.f;
  }
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.K + (size_t)unit * a.Lcap * ROWB, (uint32_t)L * ROWB);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(a.V + (size_t)unit * a.Lcap * ROWB, (uint32_t)L * ROWB);
  const int lane_row = wv * RPL + sub;
  auto load = [&](typename A::Stage& st, int stage) {
    uint32_t off[A::U];
    st.live = 0u;
#pragma unroll
    for (int j = 0; j < A::U; ++j) {
      const int row = stage * A::STAGE_ROWS + j * A::LOAD_ROWS + lane_row;
      const int slot = row < ROWS ? sh_first[row / QBLK] + row % QBLK : L;
      if (slot < L) st.live |= 1u << j;
      off[j] = slot < L ? (uint32_t)slot * ROWB + (uint32_t)cl * 16 : DEAD_OFFSET;
    }
#pragma unroll
    for (int j = 0; j < A::U; ++j) st.k[j] = buffer_load16_stream(rk, off[j]);
#pragma unroll
    for (int j = 0; j < A::U; ++j) st.v[j] = buffer_load16_stream(rv, off[j]);
  };
  auto compute = [&](const typename A::Stage& st, int stage) {
    const int row = stage * A::STAGE_ROWS + lane_row;
    A::compute(st, row, row, ROWS, cl, qreg, a.scale_log2, &sh_logit[0][0], ROWS, m_run, z_run, acc);
  };
  constexpr int PAIRS = ROWS / (2 * A::STAGE_ROWS);
  static_assert(PAIRS >= 1 && ROWS % (2 * A::STAGE_ROWS) == 0, "whole stage pairs");
  typename A::Stage s0, s1;
  load(s0, 0);
#pragma unroll
  for (int i = 0; i < PAIRS; ++i) {
    if (i * 2 * A::STAGE_ROWS >= count * QBLK) break;
    load(s1, 2 * i + 1);
    compute(s0, 2 * i);
    if (i + 1 < PAIRS) load(s0, 2 * i + 2);
    if ((2 * i + 1) * A::STAGE_ROWS < count * QBLK) compute(s1, 2 * i + 1);
  }

#pragma unroll
  for (int g = 0; g < G; ++g) {
    A::merge_rows(m_run[g], z_run[g], acc[g]);
    if (sub == 0) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) sh_acc[g][wv][cl * EPL + e] = acc[g][e];
      if (cl == 0) {
        sh_m[g][wv] = m_run[g];
        sh_z[g][wv] = z_run[g];
      }
    }
  }
  __syncthreads();
  block_partial<D, G>(a, unit, sh_m, sh_z, sh_acc);
}

// Grouped bf16 queries of d 128: q.K^T on the matrix cores, as corm_attend_gqa_kernel does it (a wave takes 16 rows of each listed block).
// Bound by HBM: 128 units x 64 blocks, four heads, 47 us for 268 MB (5.7 TB/s).
template <int G>
__global__ __launch_bounds__(WG) __attribute__((amdgpu_waves_per_eu(G <= 4 ? 3 : 2)))
void corm_block_attend_gqa_kernel(const BlockAttendArgs a) {
  using A = AttendGqa<G>;
  constexpr int D = A::D, ROWB = A::ROWB, EPL = A::EPL;
  static_assert(A::STAGE_ROWS == QBLK, "a stage is a block");
  __shared__ float sh_m[G][WAVES], sh_z[G][WAVES];
  __shared__ float sh_acc[G][WAVES][D];
  __shared__ __attribute__((aligned(16))) float sh_logit[G][A::TILE];   // (written by compute, not read)
  __shared__ uint4 sh_kt[WAVES][A::TILE * 16];
  __shared__ __attribute__((aligned(16))) float sh_p[WAVES][A::TILE * G];
  __shared__ __attribute__((aligned(16))) float sh_alpha[WAVES][G];
  __shared__ int sh_first[LIST_PART];
  const int unit = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int n = lane & 15, lg = lane >> 4;
  uint4 qb[4];
#pragma unroll
  for (int kb = 0; kb < 4; ++kb) {
    qb[kb] = make_uint4(0u, 0u, 0u, 0u);
    if (n < G) qb[kb] = *reinterpret_cast<const uint4*>(a.q + ((size_t)unit * G + n) * ROWB + (size_t)(64 * kb + 16 * lg));
  }
  const int2 listed = listed_blocks(a, unit, sh_first);
  const int L = listed.x, count = listed.y;
  if (count == 0) return empty_partial<D, G>(a, unit);
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.K + (size_t)unit * a.Lcap * ROWB, (uint32_t)L * ROWB);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(a.V + (size_t)unit * a.Lcap * ROWB, (uint32_t)L * ROWB);
  float m_run = neg_inf(), z_run = 0.f, acc[G][EPL];
#pragma unroll
  for (int g = 0; g < G; ++g)
#pragma unroll
    for (int e = 0; e < EPL; ++e) acc[g][e] = 0.f;
  auto load = [&](typename A::Stage& st, int i) {   // (rows at or above L lie behind the descriptor: zeros, and no memory traffic)
    const int row = __builtin_amdgcn_readfirstlane(sh_first[i]) + wv * A::TILE;
    A::template load<false>(st, rk, rv, (uint32_t)(row + lg) * ROWB + (uint32_t)(16 * n), nullptr, 0, lg);
  };
  auto compute = [&](const typename A::Stage& st, int i) {
    A::compute(st, __builtin_amdgcn_readfirstlane(sh_first[i]) + wv * A::TILE, 0, L, n, lg, qb, a.scale_log2, &sh_logit[0][0], A::TILE, sh_kt[wv],
               sh_p[wv], sh_alpha[wv], m_run, z_run, acc);
  };
  typename A::Stage s0, s1;
  load(s0, 0);
#pragma unroll
  for (int i = 0; i < LIST_PART; i += 2) {
    if (i >= count) break;
    load(s1, i + 1);
    compute(s0, i);
    if (i + 2 < LIST_PART) load(s0, i + 2);
    if (i + 1 < count) compute(s1, i + 1);
  }
  z_run += __shfl_xor(z_run, 16);
  z_run += __shfl_xor(z_run, 32);
#pragma unroll
  for (int g = 0; g < G; ++g) {
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      acc[g][e] += __shfl_xor(acc[g][e], 16);
      acc[g][e] += __shfl_xor(acc[g][e], 32);
    }
    if (lg == 0) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) sh_acc[g][wv][n * EPL + e] = acc[g][e];
    }
  }
  if (lg == 0 && n < G) {
    sh_m[n][wv] = m_run;
    sh_z[n][wv] = z_run;
  }
  __syncthreads();
  block_partial<D, G>(a, unit, sh_m, sh_z, sh_acc);
}

}  // namespace

#endif  // CORM_BLOCKS_HPP
