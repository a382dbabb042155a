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
  float* partials;         // not shared: [B*Hq, npart, d+2]; shared: [workgroups, 2, G, d+2]
  int2* parts;             // shared: [units], where a unit's first partial lies (its number in workgroups x 2) and how many there are
  int32_t* status;
  int32_t units, tables, Hkv, G, Lcap;
  int32_t npart;           // not shared: workgroups of a unit; with one it writes out itself
  int32_t workgroups;      // shared: all of them
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

// Eight numbers as three bf16 each, cut off: 24 bits together, so nothing is lost.
// WEIGHTS: the numbers are not negative, and no part of one above 0 is 0, so that an infinite value times its parts is infinite and not 0 x infinity: what
// is cut is a last place of fp32 less.  Nothing is lost so either: with R the first rest in last places of x, 1 <= R <= 2^16, the second part is below R by
// at most 2^8 of them, a whole number, which the third has (where it is in range: x at and above 2^-95; 0 stays 0).
template <bool WEIGHTS>
__device__ __forceinline__ void split3(const float* x, bf16x8_t (&part)[3]) {
  auto cut = [](float f) { return WEIGHTS ? __builtin_elementwise_sub_sat(__float_as_uint(f), 1u) : __float_as_uint(f); };
  uint32_t w[3][4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t u[3][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float f = x[2 * i + k];
      u[0][k] = cut(f);
      const float r = f - __uint_as_float(u[0][k] & 0xffff0000u);
      u[1][k] = cut(r);
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
  static constexpr int ESZ = 1, TILE = 32;
  static constexpr bool CODES = true;
  // four codes -> two words of two bf16 (an integer of eight bits lies in the upper half of its fp32)
  __device__ static __forceinline__ void unpack(uint32_t x, uint32_t& lo, uint32_t& hi) {
    auto f = [&](int i) { return __float_as_uint((float)(int8_t)(x >> (8 * i))); };
    lo = uppers(f(0), f(1));
    hi = uppers(f(2), f(3));
  }
};
struct PoolE4M3 {
  static constexpr int ESZ = 1, TILE = 32;
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
          split3<false>(y, s);
#pragma unroll
          for (int p = 0; p < 3; ++p) part[p][kb] = s[p];
        }
      }
    }
  }
};

__device__ __forceinline__ int slots_of(const PagedArgs& a, int unit) {
  const int b = unit / a.Hkv, h = unit - b * a.Hkv;
  return a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
}

__device__ __forceinline__ int clamped(const PagedArgs& a, int L) { return min(max(L, 0), a.Lcap); }

// Tiles of a unit, shared: an empty one has a tile of which nothing is seen, so that somebody writes its out.
__device__ __forceinline__ int shared_tiles(const PagedArgs& a, int L, int tile) { return max(1, (clamped(a, L) + tile - 1) / tile); }

// A workgroup's share of the tiles of all units, one unit behind the other: as many as every other's (in whole rounds over its waves), however the
// lengths, which the host does not know, differ.  Every workgroup adds them up itself, a thread two tables.
constexpr int SHARE_TABLES = 2 * WG;   // at most
struct Share {
  int each;              // tiles of a workgroup
  int unit, tile, slots; // where this one's begin, and the slots of that unit (as lens has them); unit < 0: it has none
};
__device__ __forceinline__ Share share_of(const PagedArgs& a, int wg, int tile_slots, int* sh) {
  const int heads = a.pages.HP, lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  int L[2], t[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = 2 * threadIdx.x + i;
    L[i] = r < a.tables ? a.lens[r] : 0;
    t[i] = r < a.tables ? shared_tiles(a, L[i], tile_slots) * heads : 0;
  }
  int scan = t[0] + t[1];
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(scan, o);
    if (lane >= o) scan += x;
  }
  if (lane == 63) sh[wv] = scan;
  __syncthreads();
  int total = 0, before = scan - t[0] - t[1];
#pragma unroll
  for (int i = 0; i < WAVES; ++i) {
    if (i < wv) before += sh[i];
    total += sh[i];
  }
  Share s;
  s.each = ((total + a.workgroups - 1) / a.workgroups + WAVES - 1) / WAVES * WAVES;
  s.unit = -1;
  const long long want = (long long)wg * s.each;
  if (want >= total) return s;
  int at = (int)want - before;
  if (at >= 0 && at < t[0] + t[1]) {
    const int i = at >= t[0];
    if (i) at -= t[0];
    const int each = (i ? t[1] : t[0]) / heads, k = at / each;
    sh[WAVES] = (2 * threadIdx.x + i) * heads + k;   // (with a table for each head that is the table's number)
    sh[WAVES + 1] = at - k * each;
    sh[WAVES + 2] = i ? L[1] : L[0];
  }
  __syncthreads();
  s.unit = __builtin_amdgcn_readfirstlane(sh[WAVES]);
  s.tile = __builtin_amdgcn_readfirstlane(sh[WAVES + 1]);
  s.slots = __builtin_amdgcn_readfirstlane(sh[WAVES + 2]);
  s.each = __builtin_amdgcn_readfirstlane(s.each);
  return s;
}

// SHARED: a workgroup has a run of tiles, which may begin and end inside units (its segments); else a unit has one workgroup, or one for each round over its
// waves (npart), so that a wave's first tile does not depend on the length and its page is looked up while that is on its way.
//
// A tile is TILE slots; the lanes of group lg = l / 16 work for its slots GROUP*lg .. +GROUP (GROUP = TILE / 4 slots, which lie in one page).
// S^T = K q^T: A = 16 keys x 32 channels (fp32: x 4) of rows as they lie, B = the heads in columns 0 .. G-1.  Row m of product t is key
// GROUP*(m/4) + 4*t + m%4, so that lane (n, lg) gets the scores of head n for its own slots -- whose probabilities are the B operand of O^T = V^T P^T
// as they lie.  Its A operand are slots of a channel where memory has channels of a slot; a lane loads the same CPL = d/16 channels of all of its
// slots, and has the operand of each channel after exchanging halves (bytes) between its own registers: one instruction for two elements (four).
// Softmax in the log2 domain.  Probabilities (with codes: times the row's scale) go into the bf16 products as three bf16
// each, without loss, so everything is exact but for the sums, which are fp32.
//
// Bound by HBM: 16 x 32 units of 3352 .. 4352 bf16 slots, d 128, 162 us (6.2 TB/s), vector ALU 14 % and matrix cores 8 % busy (8 int8 units of 131072: 44 and
// 12 %).  What was compared, each pair one build beside the other on one card (the launch as it is takes 54 us of 8 int8 units of 131072 and 72 of 128 bf16
// units of 4192 .. 8192 without a pause between the calls, single ones up to 67 and 90):
//   tiles of 32 slots for codes | 64, which take the registers of a third wave: 512 int8 units x 8192 180 us | 198
//   sums that fade in tiles that raise the maximum | that fade where it is 2^8 short, hardly ever: 8 int8 units of 131072 65.7 us | 66.6, others the same, and
//   2^8 less range of the sums | that fade in every tile, where all lanes have to agree on the maximum first: 63.4, the second 62.4 beside it
//   two workgroups per compute unit, one, three: shares of 128 units of 4192 .. 8192 bf16 slots 74, 72, 78; of 8 int8 units of 131072 56, 78, 60
template <typename P, typename DT, int D, bool SHARED>
__global__ __launch_bounds__(WG, 2) void corm_paged_attend_kernel(const PagedArgs a) {
  constexpr int TILE = P::TILE, GROUP = TILE / 4, T = GROUP / 4;
  constexpr int RB = D * P::ESZ;                       // bytes of a row
  constexpr int KL = RB / 64;                          // 16-byte loads of a key by the four lanes that share it
  constexpr int VL = P::ESZ == 4 ? D / 64 : 1;         // loads of a value row by its sixteen lanes,
  constexpr int VW = P::ESZ == 4 ? 4 : RB / 64;        // of so many words
  constexpr int CT = D / 16;
  __shared__ float sh_acc[WAVES][8][D];
  __shared__ float sh_m[WAVES][8], sh_z[WAVES][8];
  __shared__ int sh_share[SHARED ? WAVES + 3 : 1];
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, lg = lane >> 4;
  const int kgroup = GROUP * (n >> 2), vgroup = GROUP * lg;
  const int G = a.G, stride = SHARED ? WAVES : WAVES * a.npart;
  int unit, first, L, left = 0, each = 0, part = 0;    // first: the workgroup's first tile of the unit; left: tiles it still has to take
  if constexpr (SHARED) {
    const Share s = share_of(a, blockIdx.x, TILE, sh_share);
    if (s.unit < 0) return;
    unit = s.unit; first = s.tile; L = s.slots; left = each = s.each;
  } else {
    const int item = (int)(blockIdx.x % Q8_XCDS) * (int)(gridDim.x / Q8_XCDS) + (int)(blockIdx.x / Q8_XCDS);   // (each die gets whole units)
    unit = item / a.npart;
    part = item - unit * a.npart;
    if (unit >= a.units) return;
    first = part * WAVES;
  }
  const int last_page = a.pages.max_pages - 1;
  auto page_at = [&](const int32_t* table, int slot) { return table[min(slot >> a.pages.shift, last_page)]; };
  const int32_t* table = table_of(a.pages, unit / a.Hkv, unit % a.Hkv);
  int idk = page_at(table, (first + wv) * TILE + kgroup), idv = page_at(table, (first + wv) * TILE + vgroup);
  if constexpr (!SHARED) L = slots_of(a, unit);
  for (int segment = 0;; ++segment) {
    const int h = unit % a.Hkv, head0 = unit * G;
    const int tiles = SHARED ? shared_tiles(a, L, TILE) : (clamped(a, L) + TILE - 1) / TILE, end = SHARED ? min(tiles, first + left) : tiles;
    if ((L < 0 || L > a.Lcap) && first == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_LENS);
    L = clamped(a, L);
    if (!SHARED && first >= end && a.npart > 1) return;   // (a partial that the merge does not ask for)
    // (row of a slot in the pool; with a number that is none: some row)
    auto row_at = [&](int id, int slot) { return pool_row(a.pages, is_page(a.pages, id) ? id : 0, h, slot); };
    PagedQuery<P, DT, D> q;
    float m_run = neg_inf(), z_run = 0.f;   // head n's maximum (the same in all its lanes), the exponentials' sum over this lane's slots
    f32x4_t acc[CT] = {};                   // CPL channels of this lane's columns (f32: four of each 64)
    int tile = first + wv;
    // the unit behind this one, if the run goes on there
    int L_next = 0, idk_ahead = 0, idv_ahead = 0;
    const bool goes_on = SHARED && left > end - first && unit + 1 < a.units;
    if (goes_on) {
      const int32_t* ahead = table_of(a.pages, (unit + 1) / a.Hkv, (unit + 1) % a.Hkv);
      L_next = slots_of(a, unit + 1);
      idk_ahead = page_at(ahead, wv * TILE + kgroup);
      idv_ahead = page_at(ahead, wv * TILE + vgroup);
    }
    if (tile < end) {
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
      int next = min(tile + stride, end - 1);
      idk = page_at(table, next * TILE + kgroup);
      int idv_next = page_at(table, next * TILE + vgroup);
      for (; tile < end; tile += stride) {
        const int slot0 = tile * TILE + vgroup;
        const bool page_ok = is_page(a.pages, idv);
        const bool all_in = tile * TILE + TILE <= L && __all(page_ok);
        next = min(tile + stride, end - 1);
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
        if (tile + stride < end) load_k(idk, next * TILE + kgroup);
        const int after = min(next + stride, end - 1);
        idk = page_at(table, after * TILE + kgroup);
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
        if (__any(top > m_run)) {   // (no weight is above 1, so sums overflow only where the values' own sum does)
          const float m = fmaxf(m_run, rows_allreduce_max(top));
          const float fade = m == neg_inf() ? 0.f : fast_exp2(m_run - m);
          m_run = m;
          z_run *= fade;
#pragma unroll
          for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[c][j] *= fade;
        }
        const float less = m_run == neg_inf() ? 0.f : m_run;
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
        z_run += zs;
        if (tile + stride < end) load_scales(idv_next, next * TILE + vgroup);
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
            split3<!P::CODES>(p + 8 * u, pp);   // (codes are finite)
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
        if (tile + stride < end) load_v(idv_next, next * TILE + vgroup);
        idv = idv_next;
        idv_next = page_at(table, after * TILE + vgroup);
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
    const bool whole = SHARED ? first == 0 && end == tiles : a.npart == 1;
    const int place = 2 * (int)blockIdx.x + (segment > 0);
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
      if (whole) {
        a.out[(size_t)(head0 + g) * D + c] = zt == 0.f ? 0.f : at / zt;
      } else {
        float* to = SHARED ? a.partials + ((size_t)place * G + g) * (D + 2) : partial_of(a.partials, head0 + g, a.npart, part, D);
        to[2 + c] = at;
        if (c == 0) {
          to[0] = mx;
          to[1] = zt;
        }
      }
    }
    if constexpr (!SHARED) return;
    if (first == 0 && threadIdx.x == 0)   // the workgroup with a unit's first tile says where its partials are: the others' begin their runs
      a.parts[unit] = whole ? make_int2(0, 1) : make_int2(place, 1 + (tiles - left + each - 1) / each);
    if (!goes_on) return;
    left -= end - first;
    first = 0;
    ++unit;
    table = table_of(a.pages, unit / a.Hkv, unit % a.Hkv);
    L = L_next;
    idk = idk_ahead;
    idv = idv_ahead;
    __syncthreads();   // (sh_acc is read no more)
  }
}

// out of a head from the partials of its unit.  A few kilobytes a head, so its time is that of its latencies: a thread has a channel and every GROUPS'th
// partial, a batch of them under way at once (not shared: before it is known how many the unit has; the others are memory of the workspace, not used).
// By 256 threads for up to 32 partials, else by 1024: 24 partials of 24 heads, the whole call 8.4 us | 9.6.
constexpr int PAGED_MERGE_BATCH = 8;
template <int D, bool SHARED, int MERGE_WG>
__global__ __launch_bounds__(MERGE_WG) void corm_paged_merge_kernel(const PagedArgs a, int tile) {
  constexpr int GROUPS = MERGE_WG / D;
  __shared__ float sh_m[GROUPS], sh_z[GROUPS], sh_v[GROUPS][D];
  const int head = blockIdx.x, unit = head / a.G, grp = threadIdx.x / D, c = threadIdx.x % D;
  int2 where = make_int2(0, 0);
  if constexpr (SHARED) {
    where = a.parts[unit];
    if (where.y == 1) return;
  }
  const int parts = SHARED ? where.y : min(a.npart, ((clamped(a, slots_of(a, unit)) + tile - 1) / tile + WAVES - 1) / WAVES);
  const int most = SHARED ? parts : a.npart;
  auto at = [&](int s) {
    if constexpr (SHARED) return a.partials + ((size_t)(s == 0 ? where.x : (where.x & ~1) + 2 * s) * a.G + (head - unit * a.G)) * (D + 2);
    else return partial_of(a.partials, head, a.npart, s, D);
  };
  float mx = neg_inf(), z = 0.f, v = 0.f;
  for (int s0 = grp; s0 < most; s0 += GROUPS * PAGED_MERGE_BATCH) {
    float2 mz[PAGED_MERGE_BATCH];
    float x[PAGED_MERGE_BATCH];
#pragma unroll
    for (int u = 0; u < PAGED_MERGE_BATCH; ++u) {
      const float* p = at(min(s0 + u * GROUPS, most - 1));
      mz[u] = *reinterpret_cast<const float2*>(p);
      x[u] = p[2 + c];
    }
    float top = mx;
#pragma unroll
    for (int u = 0; u < PAGED_MERGE_BATCH; ++u)
      if (s0 + u * GROUPS < parts) top = fmaxf(top, mz[u].x);
    const float ms = top == neg_inf() ? 0.f : top, fade = fast_exp2(mx - ms);
    z *= fade;
    v *= fade;
    mx = top;
#pragma unroll
    for (int u = 0; u < PAGED_MERGE_BATCH; ++u)
      if (s0 + u * GROUPS < parts) {
        const float f = fast_exp2(mz[u].x - ms);
        z = fmaf(mz[u].y, f, z);
        v = fmaf(x[u], f, v);
      }
  }
  sh_v[grp][c] = v;
  if (c == 0) {
    sh_m[grp] = mx;
    sh_z[grp] = z;
  }
  __syncthreads();
  if (grp == 0) {
    float top = neg_inf();
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) top = fmaxf(top, sh_m[i]);
    const float ms = top == neg_inf() ? 0.f : top;
    z = v = 0.f;
#pragma unroll
    for (int i = 0; i < GROUPS; ++i) {
      const float f = fast_exp2(sh_m[i] - ms);
      z = fmaf(sh_z[i], f, z);
      v = fmaf(sh_v[i][c], f, v);
    }
    a.out[(size_t)head * D + c] = z == 0.f ? 0.f : v / z;
  }
}

}  // namespace

#endif  // CORM_PAGED_HPP
