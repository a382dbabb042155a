// attention of one new token over a cache of pages.
// Part of one translation unit: included by corm_paged.hip, after common.hpp, attend.hpp, codes.hpp and rows.hpp.
#ifndef CORM_PAGED_HPP
#define CORM_PAGED_HPP

namespace {

struct PagedArgs {
  PageView pages;
  const void* q;
  const int32_t* lens;     // [B,TH]
  float* out;
  float* partials;         // [B*Hq, npart, d+2]
  int32_t* status;
  int32_t units, Hkv, G, Lcap;
  int32_t part_tiles;      // tiles per workgroup
  int32_t npart;           // partials per head; with one the workgroup writes out itself
  float scale_log2;
};

// 16, 8 or 4 bytes of a row, which are read once.
template <int N>
struct Slice;
template <>
struct Slice<4> {
  u32x4_t w;
  __device__ __forceinline__ void load(const char* at) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(at)); }
  __device__ __forceinline__ void clear() { w = u32x4_t{0u, 0u, 0u, 0u}; }
  __device__ __forceinline__ uint32_t word(int i) const { return w[i]; }
};
template <>
struct Slice<2> {
  u32x2_t w;
  __device__ __forceinline__ void load(const char* at) { w = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(at)); }
  __device__ __forceinline__ void clear() { w = u32x2_t{0u, 0u}; }
  __device__ __forceinline__ uint32_t word(int i) const { return w[i]; }
};
template <>
struct Slice<1> {
  uint32_t w;
  __device__ __forceinline__ void load(const char* at) { w = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(at)); }
  __device__ __forceinline__ void clear() { w = 0u; }
  __device__ __forceinline__ uint32_t word(int) const { return w; }
};

__device__ __forceinline__ bf16x8_t bf16x8_of(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __builtin_bit_cast(bf16x8_t, u32x4_t{a, b, c, d});
}
// the upper halves of two numbers, side by side
__device__ __forceinline__ uint32_t uppers(uint32_t lo, uint32_t hi) { return __builtin_amdgcn_perm(hi, lo, 0x07060302u); }

// Eight numbers as three bf16 each, towards zero: 24 bits together, so nothing is lost.
__device__ __forceinline__ void split3(const float* x, bf16x8_t (&part)[3]) {
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u[3][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float f = x[2 * i + k];
      u[0][k] = __float_as_uint(f);
      const float r = f - __uint_as_float(u[0][k] & 0xffff0000u);
      u[1][k] = __float_as_uint(r);
      u[2][k] = __float_as_uint(r - __uint_as_float(u[1][k] & 0xffff0000u));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][i] = uppers(u[p][0], u[p][1]);
  }
#pragma unroll
  for (int p = 0; p < 3; ++p) part[p] = bf16x8_of(w[p][0], w[p][1], w[p][2], w[p][3]);
}

// What a pool holds, and how many slots a wave takes at a time.  Every int8 and every e4m3 value is a bf16, so all products of the matrix cores are exact.
struct PoolF32 {
  static constexpr int ESZ = 4, TILE = 16;
  static constexpr bool CODES = false;
};
struct PoolBF16 {
  static constexpr int ESZ = 2, TILE = 32;
  static constexpr bool CODES = false;
};
struct PoolI8 {
  static constexpr int ESZ = 1, TILE = 64;
  static constexpr bool CODES = true;
  // four codes -> two words of two bf16 (an integer of eight bits lies in the upper half of its fp32)
  __device__ static __forceinline__ void unpack(uint32_t x, uint32_t& lo, uint32_t& hi) {
    auto f = [&](int i) { return __float_as_uint((float)(int8_t)(x >> (8 * i))); };
    lo = uppers(f(0), f(1));
    hi = uppers(f(2), f(3));
  }
};
struct PoolE4M3 {
  static constexpr int ESZ = 1, TILE = 64;
  static constexpr bool CODES = true;
  __device__ static __forceinline__ void unpack(uint32_t x, uint32_t& lo, uint32_t& hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true));
  }
};

// The query heads of a unit in columns 0 .. G-1 of the B operand: lane (n = l % 16, lg = l / 16) holds head n's channels of its group lg, in the
// order in which the pool's rows are loaded.  fp32 queries over codes: three bf16 each.
template <typename P, typename DT, int D>
struct PagedQuery {
  static constexpr int PARTS = P::CODES && DT::ESZ == 4 ? 3 : 1, STEPS = D / 32;
  bf16x8_t part[PARTS][STEPS];
  float f[P::ESZ == 4 ? D / 4 : 1];

  __device__ __forceinline__ void load(const char* q, int n, int lg, int G) {
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    const char* row = q + (size_t)n * D * DT::ESZ;
    if constexpr (P::ESZ == 4) {
#pragma unroll
      for (int kb = 0; kb < D / 16; ++kb) {
        const uint4 x = n < G ? *reinterpret_cast<const uint4*>(row + (16 * kb + 4 * lg) * 4) : none;
#pragma unroll
        for (int e = 0; e < 4; ++e) f[4 * kb + e] = element<F32>(x, e);
      }
    } else {
#pragma unroll
      for (int kb = 0; kb < STEPS; ++kb) {
        const int c = P::CODES ? 64 * (kb / 2) + 16 * lg + 8 * (kb % 2) : 32 * kb + 8 * lg;
        uint4 x[DT::ESZ / 2];
#pragma unroll
        for (int i = 0; i < DT::ESZ / 2; ++i) x[i] = n < G ? *reinterpret_cast<const uint4*>(row + c * DT::ESZ + 16 * i) : none;
        if constexpr (PARTS == 1) {
          part[0][kb] = bf16x8_of(x[0].x, x[0].y, x[0].z, x[0].w);
        } else {
          float y[8];
          bf16x8_t s[3];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = element<DT>(x[e / DT::EPL], e % DT::EPL);
          split3(y, s);
#pragma unroll
          for (int p = 0; p < 3; ++p) part[p][kb] = s[p];
        }
      }
    }
  }
};

// A workgroup is a part of a unit, a wave takes every fourth tile of it.  Workgroups go to the 8 dies in turn: each die gets whole units.
//
// A tile is TILE slots; the lanes of group lg = l / 16 work for its slots GROUP*lg .. +GROUP (GROUP = TILE / 4 slots, which lie in one page).
// S^T = K q^T: A = 16 keys x 32 channels (fp32: x 4) of rows as they lie, B = the heads in columns 0 .. G-1.  Row m of product t is key
// GROUP*(m/4) + 4*t + m%4, so that lane (n, lg) gets the scores of head n for its own slots -- whose probabilities are the B operand of O^T = V^T P^T
// as they lie.  Its A operand are slots of a channel where memory has channels of a slot; a lane loads the same CPL = d/16 channels of all of its
// slots, and has the operand of each channel after exchanging halves (bytes) between its own registers: one instruction for two elements (four).
// Softmax in the log2 domain with the running maximum.  Probabilities (with codes: times the row's scale) go into the bf16 products as three bf16
// each, without loss, so everything is exact but for the sums, which are fp32.
template <typename P, typename DT, int D, int OCC>
__global__ __launch_bounds__(WG, OCC) void corm_paged_attend_kernel(const PagedArgs a) {
  constexpr int TILE = P::TILE, GROUP = TILE / 4, T = GROUP / 4;
  constexpr int RB = D * P::ESZ;                       // bytes of a row
  constexpr int KL = RB / 64;                          // 16-byte loads of a key by the four lanes that share it
  constexpr int VL = P::ESZ == 4 ? D / 64 : 1;         // loads of a value row by its sixteen lanes,
  constexpr int VW = P::ESZ == 4 ? 4 : RB / 64;        // of so many words
  constexpr int CT = D / 16;
  __shared__ float sh_acc[WAVES][8][D];
  __shared__ float sh_m[WAVES][8], sh_z[WAVES][8];
  const int item = (int)(blockIdx.x % Q8_XCDS) * (int)(gridDim.x / Q8_XCDS) + (int)(blockIdx.x / Q8_XCDS);
  const int unit = item / a.npart, part = item - unit * a.npart;
  if (unit >= a.units) return;
  const int G = a.G, head0 = unit * G;
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, lg = lane >> 4;
  int L = a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
  if (L < 0 || L > a.Lcap) {
    if (part == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_LENS);
    L = L < 0 ? 0 : a.Lcap;
  }
  const int tiles = (L + TILE - 1) / TILE;
  const int first = part * a.part_tiles, end = min(first + a.part_tiles, tiles);
  if (first >= end && a.npart > 1) return;   // (a partial that the merge does not ask for)

  const int32_t* table = table_of(a.pages, b, h);
  const int last_page = a.pages.max_pages - 1;
  auto page_at = [&](int slot) { return table[min(slot >> a.pages.shift, last_page)]; };
  // bytes from a pool's base to the row of a slot (with a number that is none: of some row)
  auto row_at = [&](int id, int slot) { return pool_row(a.pages, is_page(a.pages, id) ? id : 0, h, slot); };

  PagedQuery<P, DT, D> q;
  float m_run = neg_inf(), z_run = 0.f;   // of head n; the sum is of this lane's slots
  f32x4_t acc[CT] = {};                   // CPL channels of this lane's columns (f32: four of each 64)
  int tile = first + wv;
  if (tile < end) {
    const int kgroup = GROUP * (n >> 2), vgroup = GROUP * lg;
    int idk = page_at(tile * TILE + kgroup), idv = page_at(tile * TILE + vgroup);
    Slice<4> K[T][KL];
    Slice<VW> V[GROUP][VL];
    f32x4_t kscale[T], vscale[T];
    auto load_k = [&](int id, int slot) {
      const size_t row = row_at(id, slot);
      const char* at = a.pages.K + (row + (n & 3)) * RB + 16 * lg;
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < KL; ++c) K[t][c].load(at + 4 * t * RB + 64 * c);
    };
    auto load_v = [&](int id, int slot) {
      const size_t row = row_at(id, slot);
      const char* at = a.pages.V + row * RB + (P::ESZ == 4 ? 16 : RB / 16) * n;
#pragma unroll
      for (int j = 0; j < GROUP; ++j)
#pragma unroll
        for (int c = 0; c < VL; ++c) V[j][c].load(at + j * RB + 256 * c);
    };
    auto load_scales = [&](int id, int slot) {
      if constexpr (P::CODES) {
        const size_t row = row_at(id, slot);
#pragma unroll
        for (int t = 0; t < T; ++t) {
          kscale[t] = *reinterpret_cast<const f32x4_t*>(a.pages.ks + row + 4 * t);
          vscale[t] = *reinterpret_cast<const f32x4_t*>(a.pages.vs + row + 4 * t);
        }
      }
    };
    q.load(reinterpret_cast<const char*>(a.q) + (size_t)head0 * D * DT::ESZ, n, lg, G);
    load_k(idk, tile * TILE + kgroup);
    load_scales(idv, tile * TILE + vgroup);
    load_v(idv, tile * TILE + vgroup);
    int next = min(tile + WAVES, end - 1);
    idk = page_at(next * TILE + kgroup);
    int idv_next = page_at(next * TILE + vgroup);
    for (; tile < end; tile += WAVES) {
      const int slot0 = tile * TILE + vgroup;
      const bool page_ok = is_page(a.pages, idv);
      const bool all_in = tile * TILE + TILE <= L && __all(page_ok);
      next = min(tile + WAVES, end - 1);
      // scores
      f32x4_t s[T];
#pragma unroll
      for (int t = 0; t < T; ++t) {
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KL; ++c) {
          const u32x4_t k = K[t][c].w;
          if constexpr (P::ESZ == 4) {
#pragma unroll
            for (int e = 0; e < 4; ++e) d = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[e]), q.f[4 * c + e], d, 0, 0, 0);
          } else if constexpr (P::ESZ == 2) {
            d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k), q.part[0][c], d, 0, 0, 0);
          } else {
#pragma unroll
            for (int u = 0; u < 2; ++u) {
              uint32_t w[4];
              P::unpack(k[2 * u], w[0], w[1]);
              P::unpack(k[2 * u + 1], w[2], w[3]);
              const bf16x8_t x = bf16x8_of(w[0], w[1], w[2], w[3]);
#pragma unroll
              for (int p = 0; p < q.PARTS; ++p) d = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q.part[p][2 * c + u], d, 0, 0, 0);
            }
          }
        }
        s[t] = d;
      }
      if (tile + WAVES < end) load_k(idk, next * TILE + kgroup);
      const int after = min(next + WAVES, end - 1);
      idk = page_at(after * TILE + kgroup);
      float top = neg_inf();
#pragma unroll
      for (int t = 0; t < T; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float x = s[t][j] * a.scale_log2;
          if constexpr (P::CODES) x *= kscale[t][j];
          if (!all_in && !(page_ok && slot0 + 4 * t + j < L)) x = neg_inf();
          s[t][j] = x;
          top = fmaxf(top, x);
        }
      top = rows_allreduce_max(top);
      const float m = fmaxf(m_run, top);
      const float less = m == neg_inf() ? 0.f : m;
      const float fade = fast_exp2(m_run - less);
      m_run = m;
      if (!all_in) {   // what lies in slots that are not to be seen need not be a number
#pragma unroll
        for (int j = 0; j < GROUP; ++j)
          if (!(page_ok && slot0 + j < L)) {
#pragma unroll
            for (int c = 0; c < VL; ++c) V[j][c].clear();
            if constexpr (P::CODES) vscale[j / 4][j % 4] = 0.f;
          }
        if (!page_ok && slot0 < L && n == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_PAGE);
      }
      float p[GROUP], zs = 0.f;
#pragma unroll
      for (int j = 0; j < GROUP; ++j) {
        p[j] = fast_exp2(s[j / 4][j % 4] - less);
        zs += p[j];
        if constexpr (P::CODES) p[j] *= vscale[j / 4][j % 4];
      }
      z_run = fmaf(z_run, fade, zs);
      if (tile + WAVES < end) load_scales(idv_next, next * TILE + vgroup);
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[c][j] *= fade;
      // values
      if constexpr (P::ESZ == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int c = 0; c < VL; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              acc[4 * c + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(V[j][c].word(e)), p[j], acc[4 * c + e], 0, 0, 0);
      } else {
#pragma unroll
        for (int u = 0; u < GROUP / 8; ++u) {
          bf16x8_t pp[3];
          split3(p + 8 * u, pp);
          auto product = [&](int i, const uint32_t (&w)[4]) {
            const bf16x8_t x = bf16x8_of(w[0], w[1], w[2], w[3]);
#pragma unroll
            for (int k = 0; k < 3; ++k) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, pp[k], acc[i], 0, 0, 0);
          };
          if constexpr (P::ESZ == 2) {
#pragma unroll
            for (int i = 0; i < CT; ++i) {
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t x = V[8 * u + 2 * j][0].word(i / 2), y = V[8 * u + 2 * j + 1][0].word(i / 2);
                w[j] = __builtin_amdgcn_perm(y, x, i % 2 ? 0x07060302u : 0x05040100u);
              }
              product(i, w);
            }
          } else {
#pragma unroll
            for (int i = 0; i < CT; i += 2) {   // two channels at a time: their bytes of two slots make a word
              uint32_t w[2][4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t x = V[8 * u + 2 * j][0].word(i / 4), y = V[8 * u + 2 * j + 1][0].word(i / 4);
                P::unpack(__builtin_amdgcn_perm(y, x, i % 4 ? 0x07030602u : 0x05010400u), w[0][j], w[1][j]);
              }
              product(i, w[0]);
              product(i + 1, w[1]);
            }
          }
        }
      }
      if (tile + WAVES < end) load_v(idv_next, next * TILE + vgroup);
      idv = idv_next;
      idv_next = page_at(after * TILE + vgroup);
    }
  }

  // the waves meet
  z_run = rows_allreduce_sum(z_run);
  if (n < G) {
#pragma unroll
    for (int i = 0; i < CT; ++i)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int row = 4 * lg + r;   // of the product
        sh_acc[wv][n][P::ESZ == 4 ? 64 * (i / 4) + 4 * row + i % 4 : CT * row + i] = acc[i][r];
      }
    if (lg == 0) {
      sh_m[wv][n] = m_run;
      sh_z[wv][n] = z_run;
    }
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < G * D; idx += WG) {
    const int g = idx / D, c = idx - g * D;
    float mx = neg_inf();
#pragma unroll
    for (int i = 0; i < WAVES; ++i) mx = fmaxf(mx, sh_m[i][g]);
    const float ms = mx == neg_inf() ? 0.f : mx;
    float zt = 0.f, at = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
      const float f = fast_exp2(sh_m[i][g] - ms);
      zt = fmaf(sh_z[i][g], f, zt);
      at = fmaf(sh_acc[i][g][c], f, at);
    }
    if (a.npart == 1) {
      a.out[(size_t)(head0 + g) * D + c] = zt == 0.f ? 0.f : at / zt;
    } else {
      float* to = partial_of(a.partials, head0 + g, a.npart, part, D);
      to[2 + c] = at;
      if (c == 0) {
        to[0] = mx;
        to[1] = zt;
      }
    }
  }
}

// out of a head from the partials of its unit's tiles: every wave finds the head's maximum and sum with a lane a partial; then a thread has a channel,
// and the groups of D threads share the partials, eight in flight each.
constexpr int PAGED_MERGE_WG = 256, PAGED_MERGE_BATCH = 8;
template <int D>
__global__ __launch_bounds__(PAGED_MERGE_WG) void corm_paged_merge_kernel(const PagedArgs a, int tile) {
  constexpr int GROUPS = PAGED_MERGE_WG / D;
  __shared__ float sh[GROUPS][D];
  const int head = blockIdx.x, unit = head / a.G, lane = threadIdx.x & 63;
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int L = min(max(a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)], 0), a.Lcap);
  const int parts = ((L + tile - 1) / tile + a.part_tiles - 1) / a.part_tiles;
  const float* p0 = a.partials + (size_t)head * a.npart * (D + 2);
  float mx = neg_inf(), z = 0.f;
  for (int s = lane; s < parts; s += 64) {
    const float2 x = *reinterpret_cast<const float2*>(p0 + (size_t)s * (D + 2));
    const float m = fmaxf(mx, x.x), ms = m == neg_inf() ? 0.f : m;
    z = fmaf(z, fast_exp2(mx - ms), x.y * fast_exp2(x.x - ms));
    mx = m;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const float mo = __shfl_xor(mx, o), zo = __shfl_xor(z, o);
    const float m = fmaxf(mx, mo), ms = m == neg_inf() ? 0.f : m;
    z = fmaf(z, fast_exp2(mx - ms), zo * fast_exp2(mo - ms));
    mx = m;
  }
  const float ms = mx == neg_inf() ? 0.f : mx;
  const int grp = threadIdx.x / D, c = threadIdx.x % D;
  float sum = 0.f;
  for (int s0 = grp; s0 < parts; s0 += GROUPS * PAGED_MERGE_BATCH) {
    float m[PAGED_MERGE_BATCH], v[PAGED_MERGE_BATCH];
#pragma unroll
    for (int u = 0; u < PAGED_MERGE_BATCH; ++u) {
      const float* p = p0 + (size_t)min(s0 + u * GROUPS, parts - 1) * (D + 2);
      m[u] = p[0];
      v[u] = p[2 + c];
    }
#pragma unroll
    for (int u = 0; u < PAGED_MERGE_BATCH; ++u)
      if (s0 + u * GROUPS < parts) sum = fmaf(v[u], fast_exp2(m[u] - ms), sum);
  }
  sh[grp][c] = sum;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) sum += sh[i][c];
    a.out[(size_t)head * D + c] = z == 0.f ? 0.f : sum / z;
  }
}

}  // namespace

#endif  // CORM_PAGED_HPP
