// attention over chosen blocks: bounds of the blocks' keys, the choice, and decode attention over what was chosen.
// Part of one translation unit: included by corm_blocks.hip, after common.hpp, attend.hpp and q8.hpp.
#ifndef CORM_BLOCKS_HPP
#define CORM_BLOCKS_HPP

namespace {

// ---------------------------------------------------------------- bounds

// Grid (blocks, units), or (1 or a few, units) for the newest: block `from + blockIdx.x` of a unit, counted from its first (newest <= 0) or from the
// block that holds slot lens - newest.  A wave reads whole rows, 16 bytes a lane, and keeps the smallest and largest of its channels;
// lanes of the same slice and the waves meet at the end.
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
    x[j] = *reinterpret_cast<const uint4*>(at + (size_t)row * ROWB);
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
// Grid (groups of 64 blocks, units); lane = block, wave = a quarter of the channels, whose products meet in LDS.
template <typename DT, int D, int G>
__global__ __launch_bounds__(WG) void corm_block_score_kernel(const char* q, const char* bounds, const int32_t* lens, float* scores,
                                                              int Lcap, int nblk) {
  constexpr int EPL = DT::EPL, ROWB = D * DT::ESZ, PIECES = ROWB / 16 / WAVES, CH = D / WAVES;
  __shared__ double sh_q[G][2][D];          // q- (with the smallest elements), q+ (with the largest)
  __shared__ double sh_part[WAVES][G][64];
  const int unit = blockIdx.y, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int L = min(max(lens[unit], 0), Lcap), used = (L + QBLK - 1) / QBLK;
  const int blk = blockIdx.x * 64 + lane;
  if ((int)blockIdx.x * 64 >= used) return;
  const char* qu = q + (size_t)unit * G * ROWB;
  for (int i = threadIdx.x; i < G * D; i += WG) {
    const float x = DT::ESZ == 2 ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(qu)[i] << 16)
                                 : reinterpret_cast<const float*>(qu)[i];
    sh_q[i / D][0][i % D] = (double)fminf(x, 0.f);
    sh_q[i / D][1][i % D] = (double)fmaxf(x, 0.f);
  }
  __syncthreads();
  const char* at = bounds + ((size_t)unit * nblk + min(blk, used - 1)) * 2 * ROWB + (size_t)wv * (PIECES * 16);
  double sum[G];
#pragma unroll
  for (int g = 0; g < G; ++g) sum[g] = 0.;
#pragma unroll
  for (int s = 0; s < 2; ++s) {
    uint4 x[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) x[j] = *reinterpret_cast<const uint4*>(at + (size_t)s * ROWB + (size_t)j * 16);
#pragma unroll
    for (int j = 0; j < PIECES; ++j)
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const double v = (double)element<DT>(x[j], e);
#pragma unroll
        for (int g = 0; g < G; ++g) sum[g] = fma(v, sh_q[g][s][wv * CH + j * EPL + e], sum[g]);
      }
  }
#pragma unroll
  for (int g = 0; g < G; ++g) sh_part[wv][g][lane] = sum[g];
  __syncthreads();
  if (wv == 0 && blk < used) {
    double best = 0.;
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const double t = (sh_part[0][g][lane] + sh_part[1][g][lane]) + (sh_part[2][g][lane] + sh_part[3][g][lane]);
      best = g == 0 ? t : fmax(best, t);
    }
    scores[(size_t)unit * nblk + blk] = (float)best;
  }
}

// An fp32 number as an unsigned one of the same order (-0 as 0, what is not a number below all others).
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return (u >> 31) ? ~u : u | 0x80000000u;
}

// The k-th largest of n keys (1 <= k <= n), by the whole workgroup: digits of 8 bits from the top, counted in LDS.  key(i) is asked
// for anew in each of the four rounds.  -> (key, how many of the keys equal to it belong to the k largest)
template <int NT, typename Key>
__device__ __forceinline__ uint2 kth_largest(int n, int k, const Key& key, uint32_t* sh_hist, uint32_t* sh_pick) {
  uint32_t prefix = 0u, need = (uint32_t)k;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += NT) sh_hist[i] = 0u;
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += NT) {
      const uint32_t x = key(i);
      if (shift == 24 || (x >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&sh_hist[(x >> shift) & 255u], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 64) {   // lane l: digits 255-4l .. 252-4l
      const int l = threadIdx.x;
      uint32_t c[4], sum = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        c[j] = sh_hist[255 - 4 * l - j];
        sum += c[j];
      }
      uint32_t before = sum;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(before, o);
        if (l >= o) before += x;
      }
      before -= sum;   // keys with a larger digit than this lane's
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (before < need && before + c[j] >= need) {
          sh_pick[0] = (uint32_t)(255 - 4 * l - j);
          sh_pick[1] = need - before;
        }
        before += c[j];
      }
    }
    __syncthreads();
    prefix |= sh_pick[0] << shift;
    need = sh_pick[1];
    __syncthreads();
  }
  return make_uint2(prefix, need);
}

// Grid (units): the nlast newest blocks and the best of the others, ascending, -1 behind them.
constexpr int PICK_WG = 256;
__global__ __launch_bounds__(PICK_WG) void corm_block_pick_kernel(const float* scores, const int32_t* lens, int32_t* blocks, int Lcap,
                                                                  int nblk, int nsel, int nlast) {
  __shared__ uint32_t sh_hist[256], sh_pick[2];
  __shared__ int sh_cnt[PICK_WG / 64][2];
  const int unit = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int L = min(max(lens[unit], 0), Lcap), used = (L + QBLK - 1) / QBLK;
  const float* sc = scores + (size_t)unit * nblk;
  int32_t* to = blocks + (size_t)unit * nsel;
  const int chosen = min(used, nsel);
  for (int i = chosen + tid; i < nsel; i += PICK_WG) to[i] = -1;
  const int open = used - min(nlast, used), k = chosen - (used - open);   // blocks to choose from, how many
  if (k == open) {   // all of them
    for (int i = tid; i < chosen; i += PICK_WG) to[i] = i;
    return;
  }
  for (int i = tid; i < used - open; i += PICK_WG) to[k + i] = open + i;
  if (k == 0) return;
  const uint2 cut = kth_largest<PICK_WG>(open, k, [&](int i) { return order_key(sc[i]); }, sh_hist, sh_pick);
  int above = 0, equal = 0;   // in front of this tile
  for (int i0 = 0; i0 < open; i0 += PICK_WG) {
    const int i = i0 + tid;
    const uint32_t x = i < open ? order_key(sc[i]) : 0u;
    const bool gt = i < open && x > cut.x, eq = i < open && x == cut.x;
    const unsigned long long mg = __ballot(gt), me = __ballot(eq);
    __syncthreads();
    if (lane == 0) {
      sh_cnt[wv][0] = __popcll(mg);
      sh_cnt[wv][1] = __popcll(me);
    }
    __syncthreads();
    int ng = above, ne = equal;
    for (int w = 0; w < PICK_WG / 64; ++w) {
      if (w < wv) {
        ng += sh_cnt[w][0];
        ne += sh_cnt[w][1];
      }
      above += sh_cnt[w][0];
      equal += sh_cnt[w][1];
    }
    const unsigned long long below = (1ull << lane) - 1ull;
    ng += __popcll(mg & below);
    ne += __popcll(me & below);
    // equal ones: the first cut.y of them
    if (gt || (eq && ne < (int)cut.y)) to[ng + min(ne, (int)cut.y)] = i;
  }
}

// ---------------------------------------------------------------- attention over the listed blocks

struct BlockAttendArgs {
  const char* q;
  const char* K;
  const char* V;
  const int32_t* lens;
  const int32_t* blocks;
  float* partials;
  int32_t* status;
  int32_t Lcap, nsel, part_blocks, npart;
  float scale_log2;
};

constexpr int LIST_PART = 8;   // listed blocks per workgroup, at most

// Grid (parts of the list, units).  The rows of the listed blocks, one behind the other, are streamed as corm_attend_kernel streams a chunk;
// a lane looks the block of its row up in LDS, and rows that are not in use get an offset past the descriptor's end.
template <typename DT, int D, int G>
__global__ __launch_bounds__(WG) void corm_block_attend_kernel(const BlockAttendArgs a) {
  using A = Attend<DT, D, G, WAVES>;
  constexpr int EPL = A::EPL, ROWB = A::ROWB, LPR = A::LPR, RPL = A::RPL;
  constexpr int ROWS = LIST_PART * QBLK;
  __shared__ float sh_m[G][WAVES], sh_z[G][WAVES];
  __shared__ float sh_acc[G][WAVES][D];
  __shared__ float sh_logit[G][ROWS];
  __shared__ int sh_first[LIST_PART + 1];   // first slot of a listed block, or Lcap
  const int unit = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int sub = lane / LPR, cl = lane % LPR;
  int L = a.lens[unit];
  int flags = 0;
  if (L < 0 || L > a.Lcap) {
    flags = CORM_DEV_BAD_LENS;
    L = L < 0 ? 0 : a.Lcap;
  }
  const int first = blockIdx.x * a.part_blocks, count = min(a.part_blocks, a.nsel - first);
  if (tid < LIST_PART) {
    const int id = tid < count ? a.blocks[(size_t)unit * a.nsel + first + tid] : -1;
    const bool ok = id >= 0 && id < (L + QBLK - 1) / QBLK;
    if (!ok && id != -1) flags |= CORM_DEV_BAD_BLOCK;
    sh_first[tid] = ok ? id * QBLK : L;
  }
  if (flags && a.status) atomicOr(a.status, flags);
  __syncthreads();

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
    compute(s1, 2 * i + 1);
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
  for (int idx = tid; idx < G * D; idx += WG) {
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
    float* part = partial_of(a.partials, unit * G + g, a.npart, blockIdx.x, D);
    part[2 + c] = at;
    if (c == 0) {
      part[0] = mx;
      part[1] = zt;
    }
  }
}

}  // namespace

#endif  // CORM_BLOCKS_HPP
