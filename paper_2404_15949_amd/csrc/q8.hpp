// the 8-bit cache: rows quantised into it, and decode attention over it.
// Part of one translation unit: included by corm_blocks.hip, after common.hpp and attend.hpp.
//
// A unit's slots are cut into blocks of 64.  A full block is held in 8-bit codes with one fp32 scale for its keys and one
// for its values; the rows of the last, unfinished block stay in the KV type (the tail), so that a block is quantised once, from exact rows.
//   K codes  [B,Hkv,nblk, d/64, 64 keys, 64 channels]
//   V codes  [B,Hkv,nblk, d, 64 keys]
// In these orders the 16 bytes that a lane loads are operands of the matrix instructions as they stand: eight channels of
// a key, eight keys of a channel.  Nothing is transposed on the way.
#ifndef CORM_Q8_HPP
#define CORM_Q8_HPP

namespace {

constexpr int QBLK = 64;   // slots per block
constexpr int Q8_XCDS = 8;
constexpr int Q8_MOST = 256;   // blocks of a part, at most

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));

// Element i of a 16-byte slice of a row.
template <typename DT>
__device__ __forceinline__ float element(const uint4& x, int i) {
  const uint32_t w = (&x.x)[DT::ESZ == 2 ? i >> 1 : i];
  return DT::ESZ == 2 ? ((i & 1) ? bf16_hi(w) : bf16_lo(w)) : __uint_as_float(w);
}

// 16 bytes that are not needed again soon: rows on their way into codes or bounds are gigabytes of which nobody finds anything in a cache (with the
// codes stored so too, 16 prompts of up to 4096 rows, 32 heads: 245 -> 218 us; loads alone 249; bounds of as many keys 80 -> 73).
__device__ __forceinline__ uint4 load_once(const char* at) {
  const u32x4_t v = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(at));
  return make_uint4(v.x, v.y, v.z, v.w);
}

struct Q8Args {
  const void* q;
  const unsigned char* Kc;
  const unsigned char* Vc;
  const float* ks;
  const float* vs;
  const void* Kt;
  const void* Vt;
  const int32_t* lens;
  const int32_t* blocks;   // [units, nsel] or null: every block
  float* out;
  float* partials;         // [B*Hq, npart, d+2]
  int32_t* status;
  int32_t units, Hq, Hkv, Lcap, nblk, nsel;
  int32_t part_blocks;     // blocks per workgroup
  int32_t npart;           // partials per head, the last one the tail's; with one the workgroup has the tail too and writes out itself
  float scale_log2;
};

// Codes to halves.  Every int8 and every e4m3 value is a half, so the products of the matrix cores are exact.
struct CodeI8 {
  static constexpr int ID = CORM_I8;
  static constexpr float QMAX = 127.f;
  // 0x6400 | u is 1024 + u; with u = code + 128 a subtraction of 1152 gives the code
  __device__ static __forceinline__ void unpack(uint32_t x, half2_t& lo, half2_t& hi) {
    x ^= 0x80808080u;
    const half2_t off = {(_Float16)1152.f, (_Float16)1152.f};
    lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, x, 0x04010400u)) - off;
    hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_perm(0x64646464u, x, 0x04030402u)) - off;
  }
  // four values, already in steps of the scale
  __device__ static __forceinline__ uint32_t pack(float a, float b, float c, float d) {
    auto one = [](float v) { return (uint32_t)(int)fminf(fmaxf(rintf(v), -127.f), 127.f) & 0xffu; };
    return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
  }
};

struct CodeE4M3 {
  static constexpr int ID = CORM_E4M3;
  static constexpr float QMAX = 448.f;
  __device__ static __forceinline__ void unpack(uint32_t x, half2_t& lo, half2_t& hi) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.f, true);
  }
  __device__ static __forceinline__ uint32_t pack(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    w = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
    return (uint32_t)w;
  }
};

template <typename C>
__device__ __forceinline__ half8_t unpack8(uint32_t x, uint32_t y) {
  half2_t h[4];
  C::unpack(x, h[0], h[1]);
  C::unpack(y, h[2], h[3]);
  return __builtin_shufflevector(__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3), __builtin_shufflevector(h[2], h[3], 0, 1, 2, 3), 0,
                                 1, 2, 3, 4, 5, 6, 7);
}

// x = hi + lo in halves: hi towards zero, so that the difference is exact; together 22 bits.  NEAREST: lo to the nearest (queries, whose error grows with
// the score; for probabilities, of which there is one for every key, the packed conversion will do)
template <bool NEAREST>
__device__ __forceinline__ void split_half(float x, float y, half2_t& hi, half2_t& lo) {
  hi = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(x, y));
  const float a = x - (float)hi[0], b = y - (float)hi[1];
  if (NEAREST) lo = half2_t{(_Float16)a, (_Float16)b};
  else lo = __builtin_bit_cast(half2_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}

// ---------------------------------------------------------------- attention

// Partial of a workgroup: (max, sum, sums of p*v) of a head.
__device__ __forceinline__ float* partial_of(float* partials, int head, int npart, int part, int D) {
  return partials + ((size_t)head * npart + part) * (D + 2);
}

// The rows of the unfinished block, which are in the KV type (vector ALU: at most 63 rows).  With one or two heads the waves share the rows, else
// the heads: folding the lanes of a head's rows costs more than reading them again.  What a wave finds goes to sh_*[set], `times` over;
// returns the sets that are filled.
template <typename DT, int D, typename Acc, typename Row>
__device__ __forceinline__ int tail_attend(const void* q, const char* Kt, const char* Vt, int rows, int head0, int G, float times,
                                           float scale_log2, float* sh_junk, Row* sh_m, Row* sh_z, Acc* sh_acc) {
  using A = Attend<DT, D, 1, 1>;
  constexpr int EPL = A::EPL, ROWB = A::ROWB, LPR = A::LPR;
  constexpr int STAGES = QBLK / A::STAGE_ROWS, BATCH = STAGES < 4 ? STAGES : 4;   // of the block; in flight together
  const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
  const int sub = lane / LPR, cl = lane % LPR;
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(Kt, (uint32_t)rows * ROWB), rv = make_rsrc(Vt, (uint32_t)rows * ROWB);
  auto load = [&](typename A::Stage& st, int s) {   // (rows past the last lie behind the descriptor: zeros, and no memory traffic)
    A::template load<false>(st, rk, rv, (uint32_t)(s * A::STAGE_ROWS + sub) * ROWB + (uint32_t)cl * 16, nullptr, 0);
  };
  const bool by_rows = G <= 2;
  for (int g = by_rows ? 0 : wv; g < G; g += by_rows ? 1 : WAVES) {
    const uint4 qreg[1] = {*reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(q) + (size_t)(head0 + g) * ROWB + (size_t)cl * 16)};
    float m[1] = {neg_inf()}, z[1] = {0.f}, acc[1][EPL] = {};
    auto compute = [&](const typename A::Stage& st, int s) {
      A::compute(st, s * A::STAGE_ROWS + sub, sub, rows, cl, qreg, scale_log2, sh_junk, 0, m, z, acc);
    };
    if (by_rows) {
      for (int s = wv; s < STAGES; s += WAVES) {
        typename A::Stage st;
        load(st, s);
        compute(st, s);
      }
    } else {
#pragma unroll
      for (int s0 = 0; s0 < STAGES; s0 += BATCH) {
        typename A::Stage st[BATCH];
#pragma unroll
        for (int s = 0; s < BATCH; ++s) load(st[s], s0 + s);
#pragma unroll
        for (int s = 0; s < BATCH; ++s) compute(st[s], s0 + s);
      }
    }
    A::merge_rows(m[0], z[0], acc[0]);
    const int set = by_rows ? wv : 0;
    if (sub == 0) {
#pragma unroll
      for (int e = 0; e < EPL; ++e) sh_acc[set][g][cl * EPL + e] = acc[0][e] * times;
      if (cl == 0) {
        sh_m[set][g] = m[0];
        sh_z[set][g] = z[0] * times;
      }
    }
  }
  return by_rows ? WAVES : 1;
}

// A query head in the B operand of the products: lane (n = l%16, lg = l/16) holds channels 64*(kb/2) + 16*lg + 8*(kb%2) .. +8 of head n in step
// kb, as halves of q times a power of two that brings the head's largest element to 2^13..2^14 (bf16: exact down to 2^-27 of it; fp32 in two parts).
template <typename DT, int D>
struct QueryOperand {
  static constexpr int STEPS = D / 32;
  static constexpr int PARTS = DT::ESZ == 4 ? 2 : 1;
  half8_t part[PARTS][STEPS];
  float undo;   // 1 / the power of two
  uint4 raw[STEPS][DT::ESZ / 2];

  __device__ __forceinline__ void load(const char* q, int n, int lg, int G) {
#pragma unroll
    for (int kb = 0; kb < STEPS; ++kb) {
      const int c = 64 * (kb / 2) + 16 * lg + 8 * (kb % 2);
#pragma unroll
      for (int i = 0; i < DT::ESZ / 2; ++i) {
        raw[kb][i] = make_uint4(0u, 0u, 0u, 0u);
        if (n < G) raw[kb][i] = reinterpret_cast<const uint4*>(q + ((size_t)n * D + c) * DT::ESZ)[i];
      }
    }
  }

  __device__ __forceinline__ void convert() {
    float x[STEPS][8];
    float top = 0.f;
#pragma unroll
    for (int kb = 0; kb < STEPS; ++kb)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        x[kb][i] = element<DT>(raw[kb][i / DT::EPL], i % DT::EPL);
        top = fmaxf(top, fabsf(x[kb][i]));
      }
    top = rows_allreduce_max(top);
    const uint32_t e = min(max(__float_as_uint(top) >> 23, 14u), 254u);
    const float up = __uint_as_float((267u - e) << 23);
    undo = __uint_as_float((e - 13u) << 23);
#pragma unroll
    for (int kb = 0; kb < STEPS; ++kb) {
      half2_t hi[4], lo[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) split_half<true>(x[kb][2 * i] * up, x[kb][2 * i + 1] * up, hi[i], lo[i]);
      auto join = [](const half2_t(&h)[4]) {
        return __builtin_shufflevector(__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3), __builtin_shufflevector(h[2], h[3], 0, 1, 2, 3),
                                       0, 1, 2, 3, 4, 5, 6, 7);
      };
      part[0][kb] = join(hi);
      if (PARTS == 2) part[PARTS - 1][kb] = join(lo);
    }
  }
};

// A workgroup is a part of a unit, a wave takes every fourth block of it; the tail is the last part, or a workgroup has the whole unit.  Workgroups go to
// the 8 dies in turn: each die gets whole units, one after the other, so that no die has all first or all last parts, nor all units of a head.
//
// S^T = K q^T: four tiles of 16 keys, A = 16 keys x 32 channels of codes, B = the heads of the unit in columns 0 .. G-1.  Row m of
// tile t is key 16*(m/4) + 4*t + m%4, so that lane (n, lg) gets the scores of head n for keys 16*lg .. +16 in the order of its 16 registers --
// the keys whose values the lane's 16-byte loads of V hold.  So the probabilities are the B operand of O^T = V^T P^T as
// they lie, and no lane hands anything to another but the maximum.
// Softmax in the log2 domain with the running maximum m; p = 2^(s - m + 15) is rounded to hi + lo in halves (22 bits; the 15 keeps
// what is 2^-40 of the largest), so the products with the codes are exact and everything is summed in fp32.  The scales are
// taken in where they cost least: a block's key scale with the softmax scale (one product a score), its value scale (and 2^-15) with the sum of
// the block.
//
// Bound by HBM: 512 units x 4352 slots, d 128, 88 us (6.5 TB/s), vector ALU 38 % and matrix cores 12 % busy.  Three workgroups a compute unit (168
// registers; fp32 with d 128 spills a few of its set-up into scratch, 51 us against 53 with two; 1536 short units 17 against 20).
template <typename C, typename DT, int D>
__global__ __launch_bounds__(WG, 3) void corm_q8_attend_kernel(const Q8Args a) {
  constexpr int PANELS = D / 64, CT = D / 16, STEPS = D / 32;
  constexpr float RAISE = 15.f, LOWER = 0x1p-15f;
  __shared__ float sh_acc[2 * WAVES][8][D];   // of the waves' blocks; of their rows of the tail
  __shared__ float sh_m[2 * WAVES][8], sh_z[2 * WAVES][8];
  __shared__ float sh_junk[QBLK];
  __shared__ int sh_ids[Q8_MOST];
  __shared__ int sh_n, sh_times;
  const int G = a.Hq / a.Hkv;
  const int item = (int)(blockIdx.x % Q8_XCDS) * (int)(gridDim.x / Q8_XCDS) + (int)(blockIdx.x / Q8_XCDS);
  const int unit = item / a.npart, part = item - unit * a.npart;
  if (unit >= a.units) return;
  const int head0 = unit * G;   // b * Hq + hkv * G
  const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = lane & 15, lg = lane >> 4;
  const bool has_tail = part == a.npart - 1, has_blocks = !has_tail || a.npart == 1;
  QueryOperand<DT, D> qo;
  if (has_blocks) qo.load(reinterpret_cast<const char*>(a.q) + (size_t)head0 * D * DT::ESZ, n, lg, G);
  int L = a.lens[unit];
  if (L < 0 || L > a.Lcap) {
    if (part == 0 && threadIdx.x == 0 && a.status) atomicOr(a.status, CORM_DEV_BAD_LENS);
    L = L < 0 ? 0 : a.Lcap;
  }
  const int full = L / QBLK, rest = L % QBLK;
  const int32_t* list = a.blocks ? a.blocks + (size_t)unit * a.nsel : nullptr;
  int times = has_tail && rest > 0 ? 1 : 0;   // the tail counts as often as it is listed
  if (list && has_tail) {
    if (threadIdx.x == 0) sh_times = 0;
    __syncthreads();
    int mine = 0;
    bool bad = false;
    for (int i = threadIdx.x; i < a.nsel; i += WG) {
      const int id = list[i];
      mine += rest > 0 && id == full;
      bad |= id < -1 || id >= full + (rest > 0);
    }
    if (mine) atomicAdd(&sh_times, mine);
    if (bad && a.status) atomicOr(a.status, CORM_DEV_BAD_BLOCK);
    __syncthreads();
    times = sh_times;
  }

  // this workgroup's blocks
  const int first = part * a.part_blocks;
  int count = 0;
  if (!has_blocks) {
  } else if (list) {
    if (wv == 0) {
      int n = 0;
      for (int i0 = 0; i0 < a.part_blocks; i0 += 64) {
        const int i = first + i0 + lane;
        const int id = i0 + lane < a.part_blocks && i < a.nsel ? list[i] : -1;
        const bool ok = id >= 0 && id < full;
        const unsigned long long mask = __ballot(ok);
        if (ok) sh_ids[n + __popcll(mask & ((1ull << lane) - 1ull))] = id;
        n += __popcll(mask);
      }
      if (lane == 0) sh_n = n;
    }
    __syncthreads();
    count = sh_n;
  } else {
    count = min(a.part_blocks, full - first);
    if (count <= 0 && a.npart > 1) return;   // (a partial that the merge does not ask for)
  }
  if (count <= 0 && !times && a.npart > 1) {   // nothing to add (the merge takes no sums of a partial with this maximum)
    if (threadIdx.x < G) {
      float* to = partial_of(a.partials, head0 + threadIdx.x, a.npart, part, D);
      to[0] = neg_inf();
      to[1] = 0.f;
    }
    return;
  }

  constexpr uint32_t BLKB = QBLK * D;   // bytes of a block's codes
  const __amdgpu_buffer_rsrc_t rk = make_rsrc(a.Kc + (size_t)unit * a.nblk * BLKB, (uint32_t)full * BLKB);
  const __amdgpu_buffer_rsrc_t rv = make_rsrc(a.Vc + (size_t)unit * a.nblk * BLKB, (uint32_t)full * BLKB);
  const float* ks = a.ks + (size_t)unit * a.nblk;
  const float* vs = a.vs + (size_t)unit * a.nblk;
  const uint32_t koff = (uint32_t)((16 * (n >> 2) + (n & 3)) * 64 + 16 * lg);   // key of tile 0, this lane's channels
  const uint32_t voff = (uint32_t)lane / 16 * 16 + (uint32_t)n * 64;            // channel n, keys 16*lg ..

  auto id_of = [&](int i) { return i < count ? (list ? __builtin_amdgcn_readfirstlane(sh_ids[i]) : first + i) : full; };
  u32x4_t K[4][PANELS], V[CT];
  auto load_k = [&](int id) {   // (block `full` lies behind the descriptor: zeros, and no memory traffic)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int c = 0; c < PANELS; ++c)
        K[t][c] = __builtin_amdgcn_raw_buffer_load_b128(rk, (int)(koff + (uint32_t)(t * 256 + c * 4096)), (int)((uint32_t)id * BLKB), 2);
  };
  auto load_v = [&](int id) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
      V[c] = __builtin_amdgcn_raw_buffer_load_b128(rv, (int)(voff + (uint32_t)c * 1024), (int)((uint32_t)id * BLKB), 2);
  };

  float m_run = neg_inf(), z_run = 0.f;   // of head n; the sum is of this lane's keys
  f32x4_t acc[CT] = {};                   // channels 16*ct + 4*lg .. +4 of head n
  if (count > 0) {   // (not the part that is the tail alone)
    int id = id_of(wv);
    load_k(id);
    load_v(id);
    qo.convert();   // (behind the loads of the first block: its time is hidden in theirs)
    const float qscale = qo.undo * a.scale_log2;
    float knext = ks[min(id, a.nblk - 1)], vnext = vs[min(id, a.nblk - 1)];
    for (int i = wv; i < count; i += WAVES) {
      const float kscale = knext * qscale, vscale = vnext * LOWER;
      id = id_of(i + WAVES);
      knext = ks[min(id, a.nblk - 1)];
      vnext = vs[min(id, a.nblk - 1)];
      f32x4_t s[4];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kb = 0; kb < STEPS; ++kb) {
          const u32x4_t k = K[t][kb / 2];
          const half8_t x = kb % 2 ? unpack8<C>(k.z, k.w) : unpack8<C>(k.x, k.y);
#pragma unroll
          for (int w = 0; w < qo.PARTS; ++w) d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, qo.part[w][kb], d, 0, 0, 0);
        }
        s[t] = d;
      }
      load_k(id);
      float top = neg_inf();
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[t][j] *= kscale;
          top = fmaxf(top, s[t][j]);
        }
      top = rows_allreduce_max(top);
      const float m = fmaxf(m_run, top);
      const float less = (m == neg_inf() ? 0.f : m) - RAISE;
      const float fade = fast_exp2(m_run - RAISE - less);
      m_run = m;
      half2_t hi[8], lo[8];
      float zs = 0.f;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
          const float x = fast_exp2(s[t][j] - less), y = fast_exp2(s[t][j + 1] - less);
          zs += x + y;
          split_half<false>(x, y, hi[2 * t + j / 2], lo[2 * t + j / 2]);
        }
      z_run = fmaf(z_run, fade, zs);
      auto join = [](const half2_t* h) {
        return __builtin_shufflevector(__builtin_shufflevector(h[0], h[1], 0, 1, 2, 3), __builtin_shufflevector(h[2], h[3], 0, 1, 2, 3), 0,
                                       1, 2, 3, 4, 5, 6, 7);
      };
      const half8_t ph[2] = {join(hi), join(hi + 4)}, pl[2] = {join(lo), join(lo + 4)};
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        f32x4_t d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const half8_t x = u ? unpack8<C>(V[c].z, V[c].w) : unpack8<C>(V[c].x, V[c].y);
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, ph[u], d, 0, 0, 0);
          d = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, pl[u], d, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[c][j] = fmaf(d[j], vscale, acc[c][j] * fade);
      }
      load_v(id);
    }
  }

  // the waves meet, and the tail
  const int from = count > 0 ? 0 : WAVES;
  z_run = rows_allreduce_sum(z_run);
  if (n < G && count > 0) {
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4_t*>(&sh_acc[wv][n][16 * c + 4 * lg]) = acc[c];
    if (lg == 0) {
      sh_m[wv][n] = m_run;
      sh_z[wv][n] = z_run * LOWER;
    }
  }
  int sets = WAVES;
  if (times) {
    const char* Kt = reinterpret_cast<const char*>(a.Kt) + (size_t)unit * QBLK * D * DT::ESZ;
    const char* Vt = reinterpret_cast<const char*>(a.Vt) + (size_t)unit * QBLK * D * DT::ESZ;
    sets += tail_attend<DT, D>(a.q, Kt, Vt, rest, head0, G, (float)times, a.scale_log2, sh_junk, sh_m + WAVES, sh_z + WAVES, sh_acc + WAVES);
  }
  __syncthreads();
  for (int idx = threadIdx.x; idx < G * D; idx += WG) {
    const int g = idx / D, c = idx - g * D;
    float m[2 * WAVES], z[2 * WAVES], x[2 * WAVES], mx = neg_inf();
#pragma unroll
    for (int i = 0; i < 2 * WAVES; ++i) {   // (all at once: one latency)
      const bool in = i >= from && i < sets;
      m[i] = in ? sh_m[i][g] : neg_inf();
      z[i] = in ? sh_z[i][g] : 0.f;
      x[i] = in ? sh_acc[i][g][c] : 0.f;
      mx = fmaxf(mx, m[i]);
    }
    const float ms = mx == neg_inf() ? 0.f : mx;
    float zt = 0.f, at = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * WAVES; ++i) {
      const float f = fast_exp2(m[i] - ms);
      zt = fmaf(z[i], f, zt);
      at = fmaf(x[i], f, at);
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

// out of a head from its partials: npart of them, or (part_blocks > 0) one for every so many full blocks of the unit and the last.  A few
// kilobytes a head, so its time is its chain of latencies: every wave finds the head's maximum and sum with a lane a partial; then a thread has a
// channel, the groups of D threads share the partials and take eight at a time.  (One after the other by D threads alone: 32 partials 16 us, so 4.)
constexpr int MERGE_WG = 256, MERGE_BATCH = 8;
template <int D>
__global__ __launch_bounds__(MERGE_WG) void corm_parts_merge_kernel(const float* partials, const int32_t* lens, float* out, int G,
                                                                    int npart, int part_blocks, int Lcap) {
  constexpr int GROUPS = MERGE_WG / D;
  __shared__ float sh[GROUPS][D];
  const int head = blockIdx.x, lane = threadIdx.x & 63;
  const float* p0 = partials + (size_t)head * npart * (D + 2);
  int n = npart;
  if (part_blocks > 0) n = (min(max(lens[head / G], 0), Lcap) / QBLK + part_blocks - 1) / part_blocks + 1;
  auto at = [&](int s) { return p0 + (size_t)(s < n - 1 ? s : npart - 1) * (D + 2); };
  float mx = neg_inf(), z = 0.f;
  for (int s = lane; s < n; s += 64) {
    const float2 x = *reinterpret_cast<const float2*>(at(s));
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
  for (int s0 = grp; s0 < n; s0 += GROUPS * MERGE_BATCH) {
    float m[MERGE_BATCH], v[MERGE_BATCH];
#pragma unroll
    for (int u = 0; u < MERGE_BATCH; ++u) {
      const float* p = at(min(s0 + u * GROUPS, n - 1));
      m[u] = p[0];
      v[u] = p[2 + c];
    }
#pragma unroll
    for (int u = 0; u < MERGE_BATCH; ++u) sum = fmaf(s0 + u * GROUPS < n && m[u] > neg_inf() ? v[u] : 0.f, fast_exp2(m[u] - ms), sum);
  }
  sh[grp][c] = sum;
  __syncthreads();
  if (grp == 0) {
#pragma unroll
    for (int i = 1; i < GROUPS; ++i) sum += sh[i][c];
    out[(size_t)head * D + c] = z == 0.f ? 0.f : sum / z;
  }
}

// ---------------------------------------------------------------- rows into the cache

struct Q8AppendArgs {
  const char* k_new;
  const char* v_new;
  const int32_t* n_new;    // [B] or null: n for all
  unsigned char* Kc;
  unsigned char* Vc;
  float* ks;
  float* vs;
  char* Kt;
  char* Vt;
  const int32_t* lens;
  int32_t* lens_out;
  char* bounds;            // optional [units, nblk, 2, d]
  int32_t* status;
  int32_t Hkv, Lcap, nblk, n;
  int32_t lens_here;       // this launch writes the new lengths (not where they replace the old ones and a unit has several workgroups)
};

// What a unit gets from this call: its length before, and the rows that come (0 where they do not fit, or lens is none).
struct Arrival {
  int L0, n, flags;
};
__device__ __forceinline__ Arrival arrival(const Q8AppendArgs& a, int unit) {
  Arrival r;
  r.flags = 0;
  r.L0 = a.lens[unit];
  r.n = a.n_new ? min(max(a.n_new[unit / a.Hkv], 0), a.n) : a.n;
  if (r.L0 < 0 || r.L0 > a.Lcap) {
    r.flags = CORM_DEV_BAD_LENS;
    r.n = 0;
  } else if (r.n > a.Lcap - r.L0) {
    r.flags = CORM_DEV_UNIT_FULL;
    r.n = 0;
  }
  return r;
}

__global__ __launch_bounds__(WG) void corm_q8_lens_kernel(const Q8AppendArgs a, int units) {
  const int unit = blockIdx.x * WG + threadIdx.x;
  if (unit >= units) return;
  const Arrival r = arrival(a, unit);
  if (r.flags && a.status) atomicOr(a.status, r.flags);
  a.lens_out[unit] = r.L0 + r.n;
}

template <typename DT>
__device__ __forceinline__ void put_element(char* at, float v) {   // (v is an element: nothing is rounded)
  if (DT::ESZ == 2) *reinterpret_cast<uint16_t*>(at) = (uint16_t)(__float_as_uint(v) >> 16);
  else *reinterpret_cast<float*>(at) = v;
}

// Grid (blocks a call can touch, units).  A workgroup takes a block that gets full: a thread has four consecutive rows of a
// 16-byte column slice, so that it packs four channels of a key and four keys of a channel into words; the value words take a turn
// through LDS to lie by channel.  Bound by HBM (16 prompts of up to 4096 rows, 32 heads: 6.1 TB/s read and written; fp32, 16 heads 5.9; with bounds kept up 2
// to 4 % more time).  The first workgroup of a unit also writes the rows that stay unfinished (behind its own loads: the block it has may be made of the
// old tail) and, unless others still have to read the old one, the new length.
template <typename C, typename DT, int D>
__global__ __launch_bounds__(WG) void corm_q8_append_kernel(const Q8AppendArgs a) {
  constexpr int ESZ = DT::ESZ, EPL = DT::EPL, ROWB = D * ESZ, SL = ROWB / 16;   // 16-byte slices of a row
  constexpr int QUADS = 16 * SL, QPT = (QUADS + WG - 1) / WG;
  __shared__ uint32_t sh_v[D][17];     // four keys a word
  __shared__ uint32_t sh_top[2][WAVES];
  __shared__ float sh_lo[16][D], sh_hi[16][D];
  const int unit = blockIdx.y, blk = blockIdx.x, tid = threadIdx.x;
  const Arrival r = arrival(a, unit);
  const int have = r.L0 >= 0 ? r.L0 % QBLK : 0, total = have + r.n;
  const bool whole = r.n > 0 && (blk + 1) * QBLK <= total;
  if (!whole && blk > 0) return;
  const char* knew = a.k_new + (size_t)unit * a.n * ROWB;
  const char* vnew = a.v_new + (size_t)unit * a.n * ROWB;
  char* kt = a.Kt + (size_t)unit * QBLK * ROWB;
  char* vt = a.Vt + (size_t)unit * QBLK * ROWB;
  const size_t dst = (size_t)unit * a.nblk + (r.L0 >= 0 ? r.L0 / QBLK : 0) + blk;

  if (whole) {
    uint4 k[QPT][4], v[QPT][4];
    uint32_t kbits = 0u, vbits = 0u;   // largest magnitudes, as bits: what is not a number lies above all numbers (fmaxf would drop it)
#pragma unroll
    for (int p = 0; p < QPT; ++p) {
      const int quad = tid + p * WG, rg = quad / SL, sl = quad % SL;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        k[p][j] = v[p][j] = make_uint4(0u, 0u, 0u, 0u);
        if (QUADS % WG == 0 || quad < QUADS) {
          const int at = blk * QBLK + 4 * rg + j;
          const size_t off = (size_t)(at < have ? at : at - have) * ROWB + (size_t)sl * 16;
          k[p][j] = load_once((at < have ? kt : knew) + off);
          v[p][j] = load_once((at < have ? vt : vnew) + off);
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          kbits = max(kbits, __float_as_uint(fabsf(element<DT>(k[p][j], e))));
          vbits = max(vbits, __float_as_uint(fabsf(element<DT>(v[p][j], e))));
        }
      }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      kbits = max(kbits, (uint32_t)__shfl_xor((int)kbits, o));
      vbits = max(vbits, (uint32_t)__shfl_xor((int)vbits, o));
    }
    if ((tid & 63) == 0) {
      sh_top[0][tid >> 6] = kbits;
      sh_top[1][tid >> 6] = vbits;
    }
    if (a.bounds) {
#pragma unroll
      for (int p = 0; p < QPT; ++p) {
        const int quad = tid + p * WG, rg = quad / SL, sl = quad % SL;
        if (QUADS % WG == 0 || quad < QUADS) {
#pragma unroll
          for (int e = 0; e < EPL; ++e) {
            float lo = element<DT>(k[p][0], e), hi = lo;
#pragma unroll
            for (int j = 1; j < 4; ++j) {
              lo = fminf(lo, element<DT>(k[p][j], e));
              hi = fmaxf(hi, element<DT>(k[p][j], e));
            }
            sh_lo[rg][sl * EPL + e] = lo;
            sh_hi[rg][sl * EPL + e] = hi;
          }
        }
      }
    }
    __syncthreads();
    // (a block whose largest magnitude is below 2^-100 is held as zeros: 1 / it is near the end of fp32's range.  The scale of a block with an element that is
    // infinite or not a number is not a number: int8 has no code for these)
    auto top = [](const uint32_t(&w)[WAVES]) {
      const uint32_t bits = max(max(w[0], w[1]), max(w[2], w[3]));
      return bits < 0x7f800000u ? __uint_as_float(bits) : __builtin_nanf("");
    };
    const float ktop = top(sh_top[0]), vtop = top(sh_top[1]);
    const bool knone = ktop < 0x1p-100f, vnone = vtop < 0x1p-100f;
    const float kinv = knone ? 0.f : __fdiv_rn(C::QMAX, ktop), vinv = vnone ? 0.f : __fdiv_rn(C::QMAX, vtop);
    if (tid == 0) {
      a.ks[dst] = knone ? 0.f : __fdiv_rn(ktop, C::QMAX);
      a.vs[dst] = vnone ? 0.f : __fdiv_rn(vtop, C::QMAX);
    }
    unsigned char* kc = a.Kc + dst * (QBLK * D);
    unsigned char* vc = a.Vc + dst * (QBLK * D);
#pragma unroll
    for (int p = 0; p < QPT; ++p) {
      const int quad = tid + p * WG, rg = quad / SL, sl = quad % SL;
      if (QUADS % WG == 0 || quad < QUADS) {
        const int c0 = sl * EPL;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t w[EPL / 4];
#pragma unroll
          for (int e = 0; e < EPL; e += 4)
            w[e / 4] = C::pack(element<DT>(k[p][j], e) * kinv, element<DT>(k[p][j], e + 1) * kinv, element<DT>(k[p][j], e + 2) * kinv,
                               element<DT>(k[p][j], e + 3) * kinv);
          unsigned char* at = kc + (c0 / 64) * (QBLK * 64) + (4 * rg + j) * 64 + c0 % 64;
          if (EPL == 8) __builtin_nontemporal_store((unsigned long long)w[EPL / 4 - 1] << 32 | w[0], reinterpret_cast<unsigned long long*>(at));
          else __builtin_nontemporal_store(w[0], reinterpret_cast<uint32_t*>(at));
        }
#pragma unroll
        for (int e = 0; e < EPL; ++e)
          sh_v[c0 + e][rg] = C::pack(element<DT>(v[p][0], e) * vinv, element<DT>(v[p][1], e) * vinv, element<DT>(v[p][2], e) * vinv,
                                     element<DT>(v[p][3], e) * vinv);
      }
    }
    if (a.bounds) {
      char* bd = a.bounds + dst * 2 * ROWB;
      for (int c = tid; c < 2 * D; c += WG) {
        float x = c < D ? sh_lo[0][c % D] : sh_hi[0][c % D];
#pragma unroll
        for (int i = 1; i < 16; ++i) x = c < D ? fminf(x, sh_lo[i][c % D]) : fmaxf(x, sh_hi[i][c % D]);
        put_element<DT>(bd + (size_t)c * ESZ, x);
      }
    }
    __syncthreads();
    for (int i = tid; i < D * 4; i += WG) {
      const uint32_t* w = &sh_v[i / 4][4 * (i % 4)];
      __builtin_nontemporal_store(u32x4_t{w[0], w[1], w[2], w[3]}, reinterpret_cast<u32x4_t*>(vc) + i);
    }
  }
  if (blk > 0) return;

  // the rows that stay: new ones only (the old ones are where they belong, or in the block above)
  const int done = total / QBLK * QBLK;            // rows of the touched blocks that are full
  const int from = max(done, have), keep = total - from;
  if (r.n > 0 && keep > 0) {
    for (int i = tid; i < keep * SL; i += WG) {
      const int row = i / SL, sl = i % SL;
      const size_t src = (size_t)(from - have + row) * ROWB + (size_t)sl * 16, to = (size_t)(from - done + row) * ROWB + (size_t)sl * 16;
      *reinterpret_cast<uint4*>(kt + to) = *reinterpret_cast<const uint4*>(knew + src);
      *reinterpret_cast<uint4*>(vt + to) = *reinterpret_cast<const uint4*>(vnew + src);
    }
    if (a.bounds) {
      char* bd = a.bounds + ((size_t)unit * a.nblk + (r.L0 + r.n) / QBLK) * 2 * ROWB;
      for (int c = tid; c < D; c += WG) {
        const char* at = knew + (size_t)(from - have) * ROWB + (size_t)c * ESZ;
        auto get = [](const char* p) {
          return ESZ == 2 ? __uint_as_float((uint32_t)*reinterpret_cast<const uint16_t*>(p) << 16) : *reinterpret_cast<const float*>(p);
        };
        float lo = get(at), hi = lo;
        for (int i = 1; i < keep; ++i) {
          const float x = get(at + (size_t)i * ROWB);
          lo = fminf(lo, x);
          hi = fmaxf(hi, x);
        }
        if (from > done) {   // the block had rows before this call
          lo = fminf(lo, get(bd + (size_t)c * ESZ));
          hi = fmaxf(hi, get(bd + (size_t)(D + c) * ESZ));
        }
        put_element<DT>(bd + (size_t)c * ESZ, lo);
        put_element<DT>(bd + (size_t)(D + c) * ESZ, hi);
      }
    }
  }
  __syncthreads();   // (lens_out may be lens: every wave has read it)
  if (a.lens_here && tid == 0) {
    if (r.flags && a.status) atomicOr(a.status, r.flags);
    a.lens_out[unit] = r.L0 + r.n;
  }
}

}  // namespace

#endif  // CORM_Q8_HPP
