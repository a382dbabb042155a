// what the calls over 8-bit codes and partials share.
// Included by corm_blocks.hip and corm_paged.hip, after common.hpp and attend.hpp.
#ifndef CORM_CODES_HPP
#define CORM_CODES_HPP

namespace {

constexpr int Q8_XCDS = 8;

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

// Partial of a workgroup: (max, sum, sums of p*v) of a head.
__device__ __forceinline__ float* partial_of(float* partials, int head, int npart, int part, int D) {
  return partials + ((size_t)head * npart + part) * (D + 2);
}

}  // namespace

#endif  // CORM_CODES_HPP
