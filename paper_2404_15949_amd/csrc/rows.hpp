// rows on their way into a cache and out of it: norms of queries and keys per head, the position rotation, pages of slots.
// Part of one translation unit: included by corm_paged.hip, after common.hpp, attend.hpp and codes.hpp.
#ifndef CORM_ROWS_HPP
#define CORM_ROWS_HPP

namespace {

// Where the rows of a cache of pages lie.
struct PageView {
  char* K;
  char* V;
  float* ks;             // codes: a scale per row, laid out as the rows
  float* vs;
  const int32_t* table;  // [B, TH, max_pages]
  int32_t npages, max_pages, TH, HP, shift;   // tables per sequence, KV heads per page (TH * HP = Hkv), log2 of the slots per page
};

__device__ __forceinline__ const int32_t* table_of(const PageView& p, int b, int h) {
  return p.table + ((size_t)b * p.TH + (p.TH == 1 ? 0 : h)) * p.max_pages;
}
// Row of slot `slot` of KV head h in the pool, its page's number being id (one that is a page).
__device__ __forceinline__ size_t pool_row(const PageView& p, int id, int h, int slot) {
  return (((size_t)(uint32_t)id * p.HP + (p.TH == 1 ? h : 0)) << p.shift) + (slot & ((1 << p.shift) - 1));
}
__device__ __forceinline__ bool is_page(const PageView& p, int id) { return (uint32_t)id < (uint32_t)p.npages; }

struct RowStrides {
  int64_t seq, token, head;   // bytes
};

struct RowsArgs {
  const char* q;
  const char* k;
  const char* v;
  RowStrides qs, ks, vs;
  char* q_out;               // [B,Hq,n,d]
  char* k_out;               // [B,Hkv,n,d], or null: into the pages
  char* v_out;
  PageView pages;
  const float* inv_freq;     // [rot/2]
  const char* q_norm;        // [d] or null
  const char* k_norm;
  const int32_t* positions;  // [axes,B,n]
  const int32_t* n_new;      // [B] or null: n for all
  const int32_t* lens;       // [B,TH]
  int32_t* lens_out;
  int32_t* status;
  int32_t B, n, Hq, Hkv, Lcap;   // Hq = 0: no queries
  int32_t rot, neighbours, axes, in_turn, section[4];
  float eps, gain;
  int32_t tok_shift;         // log2 of the tokens of a workgroup
  int32_t lens_here;         // this launch writes the new lengths (not where they replace the old ones and a sequence has several workgroups)
};

constexpr int ROWS_TOKENS = 8;   // of a workgroup, at most
constexpr double HALF_TURNS = 0.318309886183790671537767526745;   // 1 / pi

// The axis that turns pair i of channels.
__device__ __forceinline__ int axis_of(const RowsArgs& a, int i) {
  if (a.axes == 1) return 0;
  if (a.in_turn) {
    const int x = i % a.axes;
    return x > 0 && i < a.axes * (x == 1 ? a.section[1] : x == 2 ? a.section[2] : a.section[3]) ? x : 0;
  }
  int x = 0, end = a.section[0];
  if (i >= end) { x = 1; end += a.section[1]; }
  if (x == 1 && i >= end) { x = 2; end += a.section[2]; }
  if (x == 2 && i >= end) x = 3;
  return x;
}

// Rows as they are in a pool or an array, rounded once.
struct AsIs {
  static constexpr int ID = -1;
};

template <typename DT>
__device__ __forceinline__ uint4 round_row(const float* y) {
  uint4 o;
  uint32_t* w = &o.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (DT::ESZ == 2) w[i] = (uint32_t)f32_to_bf16_rne(y[2 * i]) | (uint32_t)f32_to_bf16_rne(y[2 * i + 1]) << 16;
    else w[i] = __float_as_uint(y[i]);
  }
  return o;
}

template <int LPR>
__device__ __forceinline__ uint32_t row_allreduce_max(uint32_t v) {
  auto other = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
  v = max(v, other(v, std::integral_constant<int, 0xB1>()));     // quad_perm [1,0,3,2]
  v = max(v, other(v, std::integral_constant<int, 0x4E>()));     // quad_perm [2,3,0,1]
  v = max(v, other(v, std::integral_constant<int, 0x141>()));    // row_half_mirror
  if (LPR >= 16) v = max(v, other(v, std::integral_constant<int, 0x140>()));   // row_mirror
  if (LPR >= 32) v = max(v, (uint32_t)__shfl_xor((int)v, 16));
  return v;
}

// The lanes of a row put it into a slot of a pool: in the KV type, or in codes with the row's scale.
template <typename C, typename DT, int D>
__device__ __forceinline__ void put_row(char* pool, float* scales, size_t row, int cl, const float* y) {
  constexpr int EPL = DT::EPL, LPR = D / EPL;
  if constexpr (C::ID < 0) {
    *reinterpret_cast<uint4*>(pool + row * (D * DT::ESZ) + (size_t)cl * 16) = round_row<DT>(y);
  } else {
    uint32_t top = 0;   // as bits: what is not a number is above infinity, and that above all others
#pragma unroll
    for (int e = 0; e < EPL; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
    const float amax = __uint_as_float(row_allreduce_max<LPR>(top));
    const bool some = amax >= 0x1p-100f, none = __float_as_uint(amax) >= 0x7f800000u;
    const float up = some && !none ? __fdiv_rn(C::QMAX, amax) : 0.f;
    uint32_t w[EPL / 4];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i)
      w[i] = none ? 0u : C::pack(y[4 * i] * up, y[4 * i + 1] * up, y[4 * i + 2] * up, y[4 * i + 3] * up);
    char* to = pool + row * D + (size_t)cl * EPL;
    if constexpr (EPL == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
    else *reinterpret_cast<uint32_t*>(to) = w[0];
    if (cl == 0) scales[row] = none ? __uint_as_float(0x7fc00000u) : some ? __fdiv_rn(amax, C::QMAX) : 0.f;
  }
}

// Does a unit take the rows of a call?  All of them or none.
__device__ __forceinline__ bool has_room(int L0, int take, int Lcap) { return L0 >= 0 && L0 <= Lcap && take <= Lcap - L0; }

__device__ __forceinline__ int rows_taken(const RowsArgs& a, int b) { return a.n_new ? min(max(a.n_new[b], 0), a.n) : a.n; }

// The new lengths of a sequence, by one workgroup, and what is to be reported about the old ones.
__device__ __forceinline__ void write_lens(const RowsArgs& a, int b, int take) {
  for (int i = threadIdx.x; i < a.pages.TH; i += blockDim.x) {
    const size_t at = (size_t)b * a.pages.TH + i;
    const int L0 = a.lens[at];
    const bool room = has_room(L0, take, a.Lcap);
    if (!room && a.status) atomicOr(a.status, L0 < 0 || L0 > a.Lcap ? CORM_DEV_BAD_LENS : CORM_DEV_UNIT_FULL);
    a.lens_out[at] = room ? L0 + take : L0;
  }
}

// y = norm(x): x * weight / sqrt(mean x^2 + eps), then every pair of channels i turned by positions[axis of i] * inv_freq[i], for queries and keys;
// values go as they are.  The angle is formed in 64 bits (an int32 times an fp32 is exact but for two bits) and brought to a turn there: at position
// 10^6 32 bits would leave an error of 0.06.  Everything else is fp32, rounded once at the end.
//
// Few operations a byte: a token's 64 angles are shared by its heads, so the workgroup of a few tokens forms them first (LDS); then a row
// is the work of D * ESZ / 16 lanes.  A lane reads its own 16 bytes and those of the pairs' other halves (the second time from the L1).
template <typename C, typename DT, int D, int U>
__global__ __launch_bounds__(1024) void corm_rows_kernel(const RowsArgs a) {
  constexpr int EPL = DT::EPL, LPR = D / EPL;
  __shared__ float2 turn[ROWS_TOKENS][D / 2];
  const int b = blockIdx.y, t0 = (int)blockIdx.x << a.tok_shift;
  const int take = rows_taken(a, b), half = a.rot / 2;
  const int ntok = min(1 << a.tok_shift, take - t0);
  if (ntok > 0) {
    for (int i = threadIdx.x; i < ntok * half; i += blockDim.x) {
      const int tok = i / half, pair = i - tok * half;
      const int pos = a.positions[((size_t)axis_of(a, pair) * a.B + b) * a.n + t0 + tok];
      const double x = (double)pos * (double)a.inv_freq[pair] * HALF_TURNS;
      float s, c;
      sincospif((float)(x - 2.0 * rint(0.5 * x)), &s, &c);
      turn[tok][pair] = make_float2(c * a.gain, s * a.gain);
    }
    __syncthreads();
    const int sub = threadIdx.x / LPR, cl = threadIdx.x % LPR, c0 = cl * EPL;
    const int rows = blockDim.x / LPR, items = (a.Hq + 2 * a.Hkv) << a.tok_shift;
    const int mask = (1 << a.tok_shift) - 1;
    // (of the channels that are turned: does this lane hold the first or the second ones of its pairs, and where are the others)
    const bool turned = c0 < a.rot, second = !a.neighbours && c0 >= half;
    const int o0 = a.neighbours || !turned ? c0 : second ? c0 - half : c0 + half;
    for (int i0 = sub; i0 < items; i0 += rows * U) {
      uint4 own[U], other[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * rows, tok = i & mask, head = i >> a.tok_shift;
        if (i >= items || tok >= ntok) continue;
        const bool isq = head < a.Hq, isk = !isq && head < a.Hq + a.Hkv;
        const RowStrides& st = isq ? a.qs : isk ? a.ks : a.vs;
        const int h = isq ? head : isk ? head - a.Hq : head - a.Hq - a.Hkv;
        const char* row = (isq ? a.q : isk ? a.k : a.v) + b * st.seq + (t0 + tok) * st.token + h * st.head;
        own[u] = *reinterpret_cast<const uint4*>(row + (size_t)c0 * DT::ESZ);
        if ((isq || isk) && o0 != c0) other[u] = *reinterpret_cast<const uint4*>(row + (size_t)o0 * DT::ESZ);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * rows, tok = i & mask, head = i >> a.tok_shift;
        if (i >= items || tok >= ntok) continue;
        const bool isq = head < a.Hq, isk = !isq && head < a.Hq + a.Hkv;
        const int h = isq ? head : isk ? head - a.Hq : head - a.Hq - a.Hkv;
        float y[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) y[e] = element<DT>(own[u], e);
        if (isq || isk) {
          float z[EPL];
#pragma unroll
          for (int e = 0; e < EPL; ++e) z[e] = o0 != c0 ? element<DT>(other[u], e) : y[e];
          const char* w = isq ? a.q_norm : a.k_norm;
          if (w) {
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < EPL; ++e) ss = fmaf(y[e], y[e], ss);
            const float r = 1.0f / sqrtf(row_allreduce_sum<LPR>(ss) * (1.0f / D) + a.eps);
            const uint4 wy = *reinterpret_cast<const uint4*>(w + (size_t)c0 * DT::ESZ);
            const uint4 wz = *reinterpret_cast<const uint4*>(w + (size_t)o0 * DT::ESZ);
#pragma unroll
            for (int e = 0; e < EPL; ++e) {
              y[e] *= r * element<DT>(wy, e);
              z[e] *= r * element<DT>(wz, e);
            }
          }
          if (turned) {
            if (a.neighbours) {
#pragma unroll
              for (int e = 0; e < EPL; e += 2) {
                const float2 t = turn[tok][(c0 + e) / 2];
                y[e] = z[e] * t.x - z[e + 1] * t.y;
                y[e + 1] = z[e + 1] * t.x + z[e] * t.y;
              }
            } else {
#pragma unroll
              for (int e = 0; e < EPL; ++e) {
                const float2 t = turn[tok][(second ? o0 : c0) + e];
                y[e] = second ? y[e] * t.x + z[e] * t.y : y[e] * t.x - z[e] * t.y;
              }
            }
          }
        }
        char* dense = isq ? a.q_out : isk ? a.k_out : a.v_out;
        if (dense) {
          const size_t row = ((size_t)b * (isq ? a.Hq : a.Hkv) + h) * a.n + t0 + tok;
          *reinterpret_cast<uint4*>(dense + row * (D * DT::ESZ) + (size_t)cl * 16) = round_row<DT>(y);
        } else if (!isq) {
          const int L0 = a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
          if (has_room(L0, take, a.Lcap)) {   // (the same for all lanes of the row)
            const int slot = L0 + t0 + tok, id = table_of(a.pages, b, h)[slot >> a.pages.shift];
            if (is_page(a.pages, id)) {
              put_row<C, DT, D>(isk ? a.pages.K : a.pages.V, isk ? a.pages.ks : a.pages.vs, pool_row(a.pages, id, h, slot), cl, y);
            } else if (cl == 0 && a.status) {
              atomicOr(a.status, CORM_DEV_BAD_PAGE);
            }
          }
        }
      }
    }
  }
  if (a.lens_here && blockIdx.x == 0) {
    __syncthreads();   // (behind the last read of the old lengths; lens_out may be lens)
    write_lens(a, b, take);
  }
}

__global__ __launch_bounds__(WG) void corm_rows_lens_kernel(const RowsArgs a) { write_lens(a, blockIdx.x, rows_taken(a, blockIdx.x)); }

// ---------------------------------------------------------------- rows out of the pages

struct ReadArgs {
  PageView pages;
  const int32_t* lens;
  char* K_out;   // [B,Hkv,n,d]
  char* V_out;
  int32_t* status;
  int32_t Hkv, Lcap, n;
};

constexpr int READ_ROWS = 4;   // of K and of V in flight per lane

template <typename C, typename DT, int D>
__device__ __forceinline__ uint4 widen_row(const char* pool, const float* scales, size_t row, int cl) {
  constexpr int EPL = DT::EPL;
  if constexpr (C::ID < 0) {
    return load_once(pool + row * (D * DT::ESZ) + (size_t)cl * 16);
  } else {
    const char* at = pool + row * D + (size_t)cl * EPL;
    uint32_t w[2];
    if constexpr (EPL == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(at);
      w[0] = x.x;
      w[1] = x.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(at);
    }
    const float scale = scales[row];
    float y[EPL];
#pragma unroll
    for (int i = 0; i < EPL / 4; ++i) {
      half2_t lo, hi;
      C::unpack(w[i], lo, hi);
      y[4 * i] = (float)lo[0] * scale;
      y[4 * i + 1] = (float)lo[1] * scale;
      y[4 * i + 2] = (float)hi[0] * scale;
      y[4 * i + 3] = (float)hi[1] * scale;
    }
    return round_row<DT>(y);
  }
}

// Rows at and above the unit's length stay as they were, and those of slots without a page.
template <typename C, typename DT, int D>
__global__ __launch_bounds__(WG) void corm_paged_read_kernel(const ReadArgs a) {
  constexpr int LPR = D / DT::EPL, ROWS = WG / LPR;
  const int unit = blockIdx.y, b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int sub = threadIdx.x / LPR, cl = threadIdx.x % LPR;
  int L = a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
  if (L < 0 || L > a.Lcap) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_LENS);
    L = L < 0 ? 0 : a.Lcap;
  }
  L = min(L, a.n);
  const int32_t* table = table_of(a.pages, b, h);
  const int s0 = (int)blockIdx.x * (ROWS * READ_ROWS) + sub;
  int id[READ_ROWS];
#pragma unroll
  for (int u = 0; u < READ_ROWS; ++u) id[u] = s0 + u * ROWS < L ? table[(s0 + u * ROWS) >> a.pages.shift] : -1;
  uint4 k[READ_ROWS], v[READ_ROWS];
#pragma unroll
  for (int u = 0; u < READ_ROWS; ++u) {
    if (!is_page(a.pages, id[u])) continue;
    const size_t row = pool_row(a.pages, id[u], h, s0 + u * ROWS);
    k[u] = widen_row<C, DT, D>(a.pages.K, a.pages.ks, row, cl);
    v[u] = widen_row<C, DT, D>(a.pages.V, a.pages.vs, row, cl);
  }
#pragma unroll
  for (int u = 0; u < READ_ROWS; ++u) {
    const int slot = s0 + u * ROWS;
    if (is_page(a.pages, id[u])) {
      const size_t to = (((size_t)unit * a.n + slot) * D) * DT::ESZ + (size_t)cl * 16;
      *reinterpret_cast<uint4*>(a.K_out + to) = k[u];
      *reinterpret_cast<uint4*>(a.V_out + to) = v[u];
    } else if (slot < L && cl == 0 && a.status) {
      atomicOr(a.status, CORM_DEV_BAD_PAGE);
    }
  }
}

}  // namespace

#endif  // CORM_ROWS_HPP
