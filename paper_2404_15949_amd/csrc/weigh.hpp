// decode attention that accounts for every key's attention weight: the launch behind the split attend.
// Part of one translation unit: included by corm_kernels.hip, after record.hpp.
#ifndef CORM_WEIGH_HPP
#define CORM_WEIGH_HPP

namespace {

// weight_out = weight_in + sum over the heads of the group of the normalized scores (Eq. 2), from the logits and partials that the attend
// launch left; out by the last n_out rows of the grid, as in the record launch.
template <int G, int NT>
__global__ __launch_bounds__(NT) void corm_weigh_kernel(const Params p, const float* weight_in, float* weight, const int D,
                                                        const int n_out) {
  constexpr int KPT = CHUNK / NT, NW = NT / 64;
  const int PSTRIDE = D + 2;
  const int unit = blockIdx.x;
  const UnitLen ul = unit_len(p, unit);
  const int L = ul.L, nparts = (L + p.part_keys - 1) / p.part_keys;
  const int chunk = blockIdx.y;
  if (chunk >= p.nsplit) {
    record_out<G, NT>(p, unit, L, nparts, D, chunk - p.nsplit, n_out,
                      [&](int, const float* part0, int nparts) { return head_stats(part0, PSTRIDE, nparts); });
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  if (chunk == 0 && tid == 0 && ul.flags && p.status) atomicOr(p.status, ul.flags);
  if (chunk * CHUNK >= L) return;
  __shared__ float sh_M[G], sh_Z[G];
  const int head0 = unit * G;
  float lg[KPT][G], acct[KPT];
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    const int i = min(chunk * CHUNK + k * NT + tid, L - 1);
    acct[k] = weight_in[(size_t)unit * p.Lcap + i];
#pragma unroll
    for (int g = 0; g < G; ++g) lg[k][g] = p.logits[(size_t)(head0 + g) * p.Lcap + i];
  }
  for (int g = wv; g < G; g += NW) {
    const float2 st = head_stats(p.partials + (size_t)(head0 + g) * p.npart * PSTRIDE, PSTRIDE, nparts);
    if (lane == 0) {
      sh_M[g] = st.x;
      sh_Z[g] = st.y;
    }
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < KPT; ++k) {
    const int i = chunk * CHUNK + k * NT + tid;
    float sum = 0.f;
#pragma unroll
    for (int g = 0; g < G; ++g) sum += exp2f(lg[k][g] - sh_M[g]) / sh_Z[g];
    if (i < L) weight[(size_t)unit * p.Lcap + i] = acct[k] + sum;
  }
}

}  // namespace

#endif  // CORM_WEIGH_HPP
