// rows on their way into a cache and out of it: norms of queries and keys per head, the position rotation, pages of slots.
// Part of one translation unit: included by corm_paged.hip, after common.hpp, attend.hpp and codes.hpp.
#ifndef CORM_ROWS_HPP
#define CORM_ROWS_HPP

namespace {

typedef unsigned int u32x2_t __attribute__((ext_vector_type(2)));

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
  int32_t rot, axes, in_turn, section[4];
  int32_t joined;            // pairs of channels are neighbours, or nothing is turned
  float eps, gain;
  int32_t lens_here;         // this launch writes the new lengths (not where they replace the old ones and a sequence has several workgroups)
};

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

// Two fp32 as two bf16, rounded to nearest even (what is not a number stays none).
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
  const bf16x2_t x = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(uint32_t, x);
}

// Four channels of a row in the KV type: 16 or 8 bytes.
template <typename DT>
struct Four {
  uint32_t w[DT::ESZ];
  __device__ __forceinline__ void load(const char* at) {
    if constexpr (DT::ESZ == 4) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t*>(at);
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t*>(at);
      w[0] = x.x; w[1] = x.y;
    }
  }
  __device__ __forceinline__ void store(char* at) const {
    if constexpr (DT::ESZ == 4) __builtin_nontemporal_store(u32x4_t{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4_t*>(at));
    else __builtin_nontemporal_store(u32x2_t{w[0], w[1]}, reinterpret_cast<u32x2_t*>(at));
  }
  __device__ __forceinline__ void widen(float* y) const {
    if constexpr (DT::ESZ == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = __uint_as_float(w[i]);
    } else {
      y[0] = bf16_lo(w[0]); y[1] = bf16_hi(w[0]); y[2] = bf16_lo(w[1]); y[3] = bf16_hi(w[1]);
    }
  }
  __device__ __forceinline__ void round(const float* y) {
    if constexpr (DT::ESZ == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = __float_as_uint(y[i]);
    } else {
      w[0] = two_bf16(y[0], y[1]);
      w[1] = two_bf16(y[2], y[3]);
    }
  }
};

// A lane's eight channels, four and four that lie `apart` bytes behind.  JOINED: side by side, one access where the type is small enough.
template <typename DT, bool JOINED>
__device__ __forceinline__ void load_eight(Four<DT> (&f)[2], const char* at, int apart) {
  if constexpr (JOINED && DT::ESZ == 2) {
    const u32x4_t x = *reinterpret_cast<const u32x4_t*>(at);
    f[0].w[0] = x.x; f[0].w[1] = x.y; f[1].w[0] = x.z; f[1].w[1] = x.w;
  } else {
    f[0].load(at);
    f[1].load(at + apart);
  }
}
template <typename DT, bool JOINED>
__device__ __forceinline__ void store_eight(char* at, int apart, const float* y) {
  Four<DT> f[2];
  f[0].round(y);
  f[1].round(y + 4);
  if constexpr (JOINED && DT::ESZ == 2) {
    __builtin_nontemporal_store(u32x4_t{f[0].w[0], f[0].w[1], f[1].w[0], f[1].w[1]}, reinterpret_cast<u32x4_t*>(at));
  } else {
    f[0].store(at);
    f[1].store(at + apart);
  }
}

// Four numbers, in steps of the scale and not beyond the largest code, as codes.  int8: 1.5 * 2^23 has a last place of 1, so that the low byte of the
// sum is the nearest (even) integer.
template <typename C>
__device__ __forceinline__ uint32_t four_codes(const float* y, float up) {
#pragma clang fp contract(off)   // (the product is rounded before the sum is)
  if constexpr (C::ID == CORM_I8) {
    uint32_t u[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) u[e] = __float_as_uint(y[e] * up + 12582912.f);
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(u[3], u[2], 0x0c0c0400u), __builtin_amdgcn_perm(u[1], u[0], 0x0c0c0400u), 0x05040100u);
  } else {
    return C::pack(y[0] * up, y[1] * up, y[2] * up, y[3] * up);
  }
}

template <int LPR>
__device__ __forceinline__ uint32_t row_allreduce_max(uint32_t v) {
  auto other = [](uint32_t x, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(ctrl)::value, 0xf, 0xf, true); };
  v = max(v, other(v, std::integral_constant<int, 0xB1>()));     // quad_perm [1,0,3,2]
  v = max(v, other(v, std::integral_constant<int, 0x4E>()));     // quad_perm [2,3,0,1]
  v = max(v, other(v, std::integral_constant<int, 0x141>()));    // row_half_mirror
  if (LPR >= 16) v = max(v, other(v, std::integral_constant<int, 0x140>()));   // row_mirror
  return v;
}

// The lanes of a row put it into row `row` of a pool, each its eight channels: in the KV type, or in codes with the row's scale.
template <typename C, typename DT, int D, bool JOINED>
__device__ __forceinline__ void put_row(char* pool, float* scales, size_t row, int cl, int c0, int c1, const float* y) {
  if constexpr (C::ID < 0) {
    store_eight<DT, JOINED>(pool + row * (D * DT::ESZ) + c0 * DT::ESZ, (c1 - c0) * DT::ESZ, y);
  } else {
    uint32_t top = 0;   // as bits: what is not a number is above infinity, and that above all others
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(y[e]) & 0x7fffffffu);
    const float amax = __uint_as_float(row_allreduce_max<D / 8>(top));
    const bool some = amax >= 0x1p-100f, none = __float_as_uint(amax) >= 0x7f800000u;
    const float up = some && !none ? __fdiv_rn(C::QMAX, amax) : 0.f;
    const uint32_t w0 = none ? 0u : four_codes<C>(y, up), w1 = none ? 0u : four_codes<C>(y + 4, up);
    char* to = pool + row * D;
    if constexpr (JOINED) {
      *reinterpret_cast<uint2*>(to + c0) = make_uint2(w0, w1);
    } else {
      *reinterpret_cast<uint32_t*>(to + c0) = w0;
      *reinterpret_cast<uint32_t*>(to + c1) = w1;
    }
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
// A row is the work of D / 8 lanes; a lane has four channels and the four that are paired with them, so nothing but the sum of squares goes from lane to
// lane.  A workgroup has a group of tokens (TOKENS: as many as a wave has rows, so that what depends on the head is uniform; else one token, a head a
// row), its waves share their heads.  The angles are formed once, a pair a thread, and handed out through LDS.
//
// Bound by HBM, where a 1 GiB copy moves 5.1 TB/s read and written: 4 x 4096 tokens of 48 heads, d 128, bf16, 80 us (5.05 TB/s; 75 without the arithmetic, vector
// ALU half busy).  What that took, us, there and for 8 prompts of up to 4096 tokens into pages: a lane with 16 bytes in a row and its pairs' other halves
// read again 162 and 264; pairs within a lane, next rows under way 87 and 159; four waves to a group of tokens (one 88 and 162, eight 97 and 159, with
// pairs of heads in flight 86 and 135, four 84 and 139); a token's pointers formed once 82 and 132; angles once a workgroup, not once a wave 80 and 128.
// Stores past the caches: 8 us less than others.  One token of a sequence: 4.2 us, its chain of positions, angles, norm.
template <typename C, typename DT, int D, bool TOKENS, bool JOINED>
__global__ __launch_bounds__(TOKENS ? 256 : 1024) void corm_rows_kernel(const RowsArgs a) {
  constexpr int LPR = D / 8, RPW = 64 / LPR, TW = TOKENS ? RPW : 1, U = TOKENS ? 4 : 1;   // lanes of a row, rows and tokens of a wave, heads in flight
  __shared__ float2 turns[TW][D / 2 + 2];   // (a token's angles start on other banks than its neighbours')
  const int b = blockIdx.y, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int shares = blockDim.x >> 6, t0 = (int)blockIdx.x * TW;
  const int take = rows_taken(a, b);
  if (t0 < take) {
    const int lane = threadIdx.x & 63, sub = lane / LPR, cl = lane % LPR;
    const int half = a.rot / 2, tok = t0 + (TOKENS ? sub : 0);
    const bool in = tok < take;
    // this lane's channels: JOINED eight that lie together (pairs of neighbours, or nothing is turned); else four of the first halves and their partners
    const bool turned = JOINED ? 8 * cl < a.rot : 4 * cl < half;
    const int c0 = JOINED ? 8 * cl : turned ? 4 * cl : a.rot + 8 * (cl - half / 4), c1 = !JOINED && turned ? c0 + half : c0 + 4;
    const int heads = a.Hq + 2 * a.Hkv, step = TOKENS ? 1 : RPW;
    const int each = ((heads + step - 1) / step + shares - 1) / shares * step;   // heads of a wave
    const int end = min(heads, (wv + 1) * each);
    // a batch of U heads: their rows, and the lengths of the units that they go to
    struct Batch {
      Four<DT> x[U][2];
      int L0[U];
    };
    const int nq = a.Hq, nqk = a.Hq + a.Hkv;
    const bool paged = !a.k_out;
    // Where this lane's channels of its token lie.  TOKENS: what does not depend on the head is formed once (else a wave has hardly more than one).
    const char *q0 = nullptr, *k0 = nullptr, *v0 = nullptr;
    if constexpr (TOKENS) {
      q0 = a.q + b * a.qs.seq + tok * a.qs.token + c0 * DT::ESZ;
      k0 = a.k + b * a.ks.seq + tok * a.ks.token + c0 * DT::ESZ;
      v0 = a.v + b * a.vs.seq + tok * a.vs.token + c0 * DT::ESZ;
    }
    const int64_t qh = a.qs.head, kh = a.ks.head, vh = a.vs.head, oh = (int64_t)a.n * (D * DT::ESZ);   // bytes from head to head
    char* const qo = a.q_out + ((int64_t)b * a.Hq * a.n + tok) * (D * DT::ESZ) + c0 * DT::ESZ;
    const int64_t kv_row = ((int64_t)b * a.Hkv * a.n + tok) * (D * DT::ESZ) + c0 * DT::ESZ;
    const int apart = (c1 - c0) * DT::ESZ;   // bytes between the lane's two fours
    auto load = [&](Batch& t, int h0) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int head = h0 + u * step + (TOKENS ? 0 : sub);
        if (head >= end || !in) continue;
        const bool isq = head < nq, isk = !isq && head < nqk;
        const int h = head - (isq ? 0 : isk ? nq : nqk);
        if constexpr (TOKENS) {
          load_eight<DT, JOINED>(t.x[u], isq ? q0 + h * qh : isk ? k0 + h * kh : v0 + h * vh, apart);
        } else {
          const char* base = isq ? a.q : isk ? a.k : a.v;
          const int64_t sq = isq ? a.qs.seq : isk ? a.ks.seq : a.vs.seq, st = isq ? a.qs.token : isk ? a.ks.token : a.vs.token,
                        sh = isq ? a.qs.head : isk ? a.ks.head : a.vs.head;
          load_eight<DT, JOINED>(t.x[u], base + b * sq + h * sh + tok * st + c0 * DT::ESZ, apart);
        }
        if (paged && head >= nq) t.L0[u] = a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
      }
    };
    Batch now;
    load(now, wv * each);
    // the angles, behind the loads of the first rows
    for (int i = threadIdx.x; i < TW * half; i += blockDim.x) {
      const int t = TOKENS ? i / half : 0, pair = i - t * half;
      const int pos = a.positions[((size_t)axis_of(a, pair) * a.B + b) * a.n + min(t0 + t, a.n - 1)];
      const double x = (double)pos * (double)a.inv_freq[pair] * HALF_TURNS;
      float s, c;
      sincospif((float)(x - 2.0 * rint(0.5 * x)), &s, &c);
      turns[t][pair] = make_float2(c * a.gain, s * a.gain);
    }
    __syncthreads();
    float2 turn[4];
    if (turned) {
#pragma unroll
      for (int e = 0; e < 4; ++e) turn[e] = turns[TOKENS ? sub : 0][4 * cl + e];
    }
    Four<DT> wq[2], wk[2];
    if (a.q_norm) load_eight<DT, JOINED>(wq, a.q_norm + c0 * DT::ESZ, apart);
    if (a.k_norm) load_eight<DT, JOINED>(wk, a.k_norm + c0 * DT::ESZ, apart);
    for (int h0 = wv * each; h0 < end; h0 += step * U) {
      Batch next;
      load(next, h0 + step * U);
      int id[U];
      if (paged) {   // the pages, behind the loads of the next rows
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int head = h0 + u * step + (TOKENS ? 0 : sub);
          if (head >= end || !in || head < nq || !has_room(now.L0[u], take, a.Lcap)) continue;
          id[u] = table_of(a.pages, b, head < nqk ? head - nq : head - nqk)[(now.L0[u] + tok) >> a.pages.shift];
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int head = h0 + u * step + (TOKENS ? 0 : sub);
        if (head >= end || !in) continue;
        float y[8];
        now.x[u][0].widen(y);
        now.x[u][1].widen(y + 4);
        if (head < nqk) {
          if (head < nq ? a.q_norm : a.k_norm) {
            float ss = 0.f, w[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) ss = fmaf(y[e], y[e], ss);
            const float r = rsqrtf(row_allreduce_sum<LPR>(ss) * (1.0f / D) + a.eps);
            const Four<DT> f[2] = {head < nq ? wq[0] : wk[0], head < nq ? wq[1] : wk[1]};
            f[0].widen(w);
            f[1].widen(w + 4);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= r * w[e];
          }
          if (turned) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float &first = y[JOINED ? 2 * e : e], &second = y[JOINED ? 2 * e + 1 : e + 4];
              const float p = first, q = second;
              first = p * turn[e].x - q * turn[e].y;
              second = q * turn[e].x + p * turn[e].y;
            }
          }
        }
        if (head < nq) {
          store_eight<DT, JOINED>(qo + head * oh, apart, y);
        } else if (!paged) {
          store_eight<DT, JOINED>((head < nqk ? a.k_out + kv_row + (head - nq) * oh : a.v_out + kv_row + (head - nqk) * oh), apart, y);
        } else if (has_room(now.L0[u], take, a.Lcap)) {   // (the same for all lanes of the row)
          const bool isk = head < nqk;
          const int h = head - (isk ? nq : nqk);
          if (is_page(a.pages, id[u])) {
            put_row<C, DT, D, JOINED>(isk ? a.pages.K : a.pages.V, isk ? a.pages.ks : a.pages.vs, pool_row(a.pages, id[u], h, now.L0[u] + tok), cl, c0, c1,
                                      y);
          } else if (cl == 0 && a.status) {
            atomicOr(a.status, CORM_DEV_BAD_PAGE);
          }
        }
      }
      now = next;
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

// One lane's 16 bytes of a row of a pool, in the KV type.
template <typename C, typename DT, int D>
__device__ __forceinline__ u32x4_t widen_row(const char* pool, const float* scales, size_t row, int cl) {
  constexpr int EPL = DT::EPL;
  if constexpr (C::ID < 0) {
    return __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(pool + row * (D * DT::ESZ) + (size_t)cl * 16));
  } else {
    const char* at = pool + row * D + (size_t)cl * EPL;
    uint32_t w[2];
    if constexpr (EPL == 8) {
      const u32x2_t x = __builtin_nontemporal_load(reinterpret_cast<const u32x2_t*>(at));
      w[0] = x.x;
      w[1] = x.y;
    } else {
      w[0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(at));
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
    if constexpr (DT::ESZ == 4) return u32x4_t{__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3])};
    else return u32x4_t{two_bf16(y[0], y[1]), two_bf16(y[2], y[3]), two_bf16(y[4], y[5]), two_bf16(y[6], y[7])};
  }
}

// Rows at and above the unit's length stay as they were, and those of slots without a page.  A lane has 16 bytes of a key and of a value: bound by HBM, and
// many short workgroups, which nothing holds up but one another, keep it busiest (rows of each per lane, 16 x 32 units of up to 4352 int8 slots, d 128: one
// 230 us (5.8 TB/s), two 238, four 264; with loads and stores that caches are to keep 264).
template <typename C, typename DT, int D>
__global__ __launch_bounds__(WG) void corm_paged_read_kernel(const ReadArgs a) {
  constexpr int LPR = D / DT::EPL, ROWS = WG / LPR;
  const int unit = blockIdx.y, b = unit / a.Hkv, h = unit - b * a.Hkv;
  const int cl = threadIdx.x % LPR, slot = (int)blockIdx.x * ROWS + (int)threadIdx.x / LPR;
  int L = a.lens[(size_t)b * a.pages.TH + (a.pages.TH == 1 ? 0 : h)];
  if (L < 0 || L > a.Lcap) {
    if (blockIdx.x == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_LENS);
    L = L < 0 ? 0 : a.Lcap;
  }
  if (slot >= min(L, a.n)) return;
  const int id = table_of(a.pages, b, h)[slot >> a.pages.shift];
  if (!is_page(a.pages, id)) {
    if (cl == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_PAGE);
    return;
  }
  const size_t row = pool_row(a.pages, id, h, slot), to = (((size_t)unit * a.n + slot) * D) * DT::ESZ + (size_t)cl * 16;
  const u32x4_t k = widen_row<C, DT, D>(a.pages.K, a.pages.ks, row, cl), v = widen_row<C, DT, D>(a.pages.V, a.pages.vs, row, cl);
  __builtin_nontemporal_store(k, reinterpret_cast<u32x4_t*>(a.K_out + to));
  __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(a.V_out + to));
}

}  // namespace

#endif  // CORM_ROWS_HPP
