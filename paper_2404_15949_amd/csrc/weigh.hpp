// decode attention that accounts for every key's attention weight: the launch behind the split attend (many units: unit.hpp alone).
// Part of one translation unit: included by corm_kernels.hip, after record.hpp.
#ifndef CORM_WEIGH_HPP
#define CORM_WEIGH_HPP

namespace {

// weight_out = weight_in + sum over the heads of the group of the normalized scores (Eq. 2), from the logits and partials that the attend
// launch left; out by the last n_out rows of the grid, as in the record launch.  A thread has ROUNDS times four consecutive keys (16-byte
// loads where rows of the arrays begin at multiples of 16 bytes); many keys a workgroup, since its time is its chain of latencies
// (512 units x 4352 keys: 512 keys a workgroup 15 us, 2048 9.8).
constexpr int WEIGH_KEYS = 4 * WG;   // keys of a round
template <int G, int ROUNDS>
__global__ __launch_bounds__(WG) void corm_weigh_kernel(const Params p, const int D, const int n_out) {
  const int PSTRIDE = D + 2;
  const int unit = blockIdx.x;
  const UnitLen ul = unit_len(p, unit);
  const int L = ul.L, nparts = (L + p.part_keys - 1) / p.part_keys;
  const int groups = gridDim.y - n_out, group = blockIdx.y;
  if (group >= groups) {
    record_out<G, WG>(p, unit, L, nparts, D, group - groups, n_out,
                      [&](int, const float* part0, int nparts) { return head_stats(part0, PSTRIDE, nparts); });
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (group == 0 && tid == 0 && ul.flags && p.status) atomicOr(p.status, ul.flags);
  const int first = group * (ROUNDS * WEIGH_KEYS);
  if (first >= L) return;
  __shared__ float sh_M[G], sh_Z[G];
  const int head0 = unit * G;
  const float* in = accounts_in(p) + (size_t)unit * p.Lcap;
  float* out = accounts_out(p) + (size_t)unit * p.Lcap;
  const float* logits = p.logits + (size_t)head0 * p.Lcap;
  const bool wide = ((p.Lcap & 3) | ((reinterpret_cast<uintptr_t>(p.pos) | reinterpret_cast<uintptr_t>(p.last_hit)) & 15)) == 0;
  auto get = [&](const float* a, int i, float (&x)[4]) {
    if (wide && i + 4 <= L) {
      const float4 v = *reinterpret_cast<const float4*>(a + i);
      x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = i + j < L ? a[i + j] : 0.f;
    }
  };
  float acct[ROUNDS][4], lg[ROUNDS][G][4];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * WEIGH_KEYS + 4 * tid;
    get(in, i, acct[r]);
#pragma unroll
    for (int g = 0; g < G; ++g) get(logits + (size_t)g * p.Lcap, i, lg[r][g]);
  }
  for (int g = wv; g < G; g += WAVES) {
    const float2 st = head_stats(p.partials + (size_t)(head0 + g) * p.npart * PSTRIDE, PSTRIDE, nparts);
    if (lane == 0) {
      sh_M[g] = st.x;
      sh_Z[g] = 1.f / st.y;
    }
  }
  __syncthreads();
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int i = first + r * WEIGH_KEYS + 4 * tid;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] = fmaf(fast_exp2(lg[r][g][j] - sh_M[g]), sh_Z[g], sum[j]);
    if (wide && i + 4 <= L) {
      *reinterpret_cast<float4*>(out + i) = make_float4(acct[r][0] + sum[0], acct[r][1] + sum[1], acct[r][2] + sum[2], acct[r][3] + sum[3]);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < L) out[i + j] = acct[r][j] + sum[j];
    }
  }
}

}  // namespace

#endif  // CORM_WEIGH_HPP
