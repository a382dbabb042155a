// HIP kernels (gfx950 / CDNA4, wave64) and C ABI of what bounds a decode step's reads beside CORM's own rule: a cache held in 8
// bits, attention over chosen blocks of it or of the plain cache, and the eviction decision by accumulated attention weight.
// One translation unit:
//   q8.hpp             rows quantised into blocks of 64, and attention over them (q.K^T and p.V on the matrix cores)
//   select.hpp         the k-th largest of many numbers
//   blocks.hpp         bounds of the blocks' keys, the choice, attention over the chosen ones
//   evict_weight.hpp   the decision by weight (the weights themselves are summed behind corm_kernels.hip's attend launch)
// Kernel boundaries are the only synchronization between workgroups, and nothing is kept from one call for the next.
#include <hip/hip_runtime.h>
#include <stdint.h>
#include <math.h>
#include <algorithm>
#include <cmath>
#include <mutex>

#include "corm.h"

#include "common.hpp"
#include "attend.hpp"
#include "q8.hpp"
#include "select.hpp"
#include "blocks.hpp"
#include "evict_weight.hpp"
#include "checks.hpp"

namespace {

int blocks_of(const corm_desc* d) { return (d->Lcap + QBLK - 1) / QBLK; }

// Partials a head can have: parts of at least four blocks, or of a list of up to 512, and the tail.
int max_parts(const corm_desc* d) { return std::max((blocks_of(d) + 3) / 4, 128) + 1; }
int max_listed(const corm_desc* d) { return std::max(blocks_of(d), 512); }

// Splits of a unit in the eviction decision of long units, 0 where a workgroup takes a unit alone: where it can hold the unit's keys.  Us, one
// workgroup | splits: 8, 128 and 512 units x 9000 slots 9.7 | 14.1, 10.1 | 16.4 and 15.9 | 31.5, x 16000 14.4 | 13.8, 15.8 | 17.3 and 23.1 | 33.0;
// keys from memory in every round | splits: 8, 512 and 2000 x 20000 22 | 14, 40 | 42 and 169 | 157, 256 x 40000 69 | 42, 256 x 100000 185 | 101,
// 8 x 500000 530 | 29.
struct EvictSplits {
  int splits, slots;
  size_t listed_off, counts_off, digit_off, total;
};
EvictSplits evict_splits(const corm_desc* d) {
  EvictSplits e = {};
  const size_t units = (size_t)d->B * d->Hkv;
  if (d->Lcap <= EVW_KEYS) return e;
  e.slots = std::max(EVW_SPLIT, ((d->Lcap + 63) / 64 + EVW_WG - 1) / EVW_WG * EVW_WG);
  e.splits = (d->Lcap + e.slots - 1) / e.slots;
  e.listed_off = align_up(units * e.splits * EVW_COUNTS * sizeof(uint32_t), 256);
  e.counts_off = e.listed_off + align_up(units * d->Lcap * sizeof(uint32_t), 256);
  e.digit_off = e.counts_off + align_up(units * e.splits * sizeof(uint32_t), 256);
  e.total = e.digit_off + align_up(units * sizeof(uint2), 256);
  return e;
}

// Each of the calls below has the whole workspace to itself: partials, scores, or what the eviction of long units hands on.
size_t blocks_workspace(const corm_desc* d) {
  const size_t partials = (size_t)d->B * d->Hq * max_parts(d) * (d->d + 2) * sizeof(float);
  const size_t scores = (size_t)d->B * d->Hkv * blocks_of(d) * sizeof(float);
  return align_up(std::max({partials, scores, evict_splits(d).total}), 256);
}

int check_blocks_workspace(const corm_desc* d, const void* workspace, size_t bytes) {
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return CORM_EINVAL;
  return bytes < blocks_workspace(d) ? CORM_ECAPACITY : CORM_OK;
}

float scale_log2(const corm_desc* d) { return (d->sm_scale > 0.f ? d->sm_scale : 1.0f / sqrtf((float)d->d)) * LOG2E; }

int merge_parts(const corm_desc* d, const float* partials, const int32_t* lens, float* out, int npart, int part_blocks, hipStream_t s) {
  const int G = d->Hq / d->Hkv;
  const dim3 grid(d->B * d->Hq);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(MERGE_WG), 0, s, partials, lens, out, G, npart, part_blocks, d->Lcap); };
  if (d->d == 64) launch(corm_parts_merge_kernel<64>);
  else launch(corm_parts_merge_kernel<128>);
  return launch_status();
}

// kernel<code, element type, d> by the call's types
template <typename F>
int by_types(const corm_desc* d, int32_t code, const F& f) {
  auto inner = [&](auto c) {
    if (d->kv_dtype == CORM_F32) return d->d == 64 ? f(c, F32(), std::integral_constant<int, 64>()) : f(c, F32(), std::integral_constant<int, 128>());
    return d->d == 64 ? f(c, BF16(), std::integral_constant<int, 64>()) : f(c, BF16(), std::integral_constant<int, 128>());
  };
  return code == CORM_I8 ? inner(CodeI8()) : inner(CodeE4M3());
}
template <typename F>
int by_group(const corm_desc* d, const F& f) {
  switch (d->Hq / d->Hkv) {
    case 1: return f(std::integral_constant<int, 1>());
    case 2: return f(std::integral_constant<int, 2>());
    case 4: return f(std::integral_constant<int, 4>());
    case 8: return f(std::integral_constant<int, 8>());
    default: return CORM_EUNSUPPORTED;
  }
}
template <typename F>
int by_row(const corm_desc* d, const F& f) {
  if (d->kv_dtype == CORM_F32) return d->d == 64 ? f(F32(), std::integral_constant<int, 64>()) : f(F32(), std::integral_constant<int, 128>());
  return d->d == 64 ? f(BF16(), std::integral_constant<int, 64>()) : f(BF16(), std::integral_constant<int, 128>());
}

int check_code(int32_t code) { return code == CORM_I8 || code == CORM_E4M3 ? CORM_OK : CORM_EUNSUPPORTED; }

}  // namespace

extern "C" {

int corm_blocks_workspace_bytes(const corm_desc* desc, size_t* bytes) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!bytes) return CORM_EINVAL;
  *bytes = blocks_workspace(desc);
  return CORM_OK;
}

int corm_q8_append(const corm_desc* desc, int32_t code_dtype, const void* k_new, const void* v_new, int32_t n, const int32_t* n_new,
                   void* K_codes, void* V_codes, float* k_scale, float* v_scale, void* K_tail, void* V_tail, const int32_t* lens,
                   int32_t* lens_out, void* bounds, int32_t* status, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  rc = check_code(code_dtype);
  if (rc) return rc;
  if (!k_new || !v_new || !K_codes || !V_codes || !k_scale || !v_scale || !K_tail || !V_tail || !lens || !lens_out) return CORM_EINVAL;
  if (misaligned16(k_new) || misaligned16(v_new) || misaligned16(K_codes) || misaligned16(V_codes) || misaligned16(K_tail) ||
      misaligned16(V_tail) || misaligned16(bounds))
    return CORM_EINVAL;
  if (misaligned4(n_new) || misaligned4(k_scale) || misaligned4(v_scale) || misaligned4(lens) || misaligned4(lens_out) || misaligned4(status))
    return CORM_EINVAL;
  if (n < 1 || n > desc->Lcap) return CORM_EINVAL;
  Q8AppendArgs a;
  a.k_new = reinterpret_cast<const char*>(k_new); a.v_new = reinterpret_cast<const char*>(v_new); a.n_new = n_new;
  a.Kc = reinterpret_cast<unsigned char*>(K_codes); a.Vc = reinterpret_cast<unsigned char*>(V_codes);
  a.ks = k_scale; a.vs = v_scale;
  a.Kt = reinterpret_cast<char*>(K_tail); a.Vt = reinterpret_cast<char*>(V_tail);
  a.lens = lens; a.lens_out = lens_out; a.bounds = reinterpret_cast<char*>(bounds); a.status = status;
  a.Hkv = desc->Hkv; a.Lcap = desc->Lcap; a.nblk = blocks_of(desc); a.n = n;
  const int units = desc->B * desc->Hkv;
  const dim3 grid((n + 2 * QBLK - 2) / QBLK, units);   // blocks that n rows behind up to 63 others can touch
  a.lens_here = grid.x == 1 || lens_out != lens;
  hipStream_t s = (hipStream_t)stream;
  rc = by_types(desc, code_dtype, [&](auto c, auto dt, auto dd) {
    hipLaunchKernelGGL((corm_q8_append_kernel<decltype(c), decltype(dt), decltype(dd)::value>), grid, dim3(WG), 0, s, a);
    return launch_status();
  });
  if (rc || a.lens_here) return rc;
  hipLaunchKernelGGL(corm_q8_lens_kernel, dim3((units + WG - 1) / WG), dim3(WG), 0, s, a, units);
  return launch_status();
}

int corm_q8_attend(const corm_desc* desc, int32_t code_dtype, const void* q, const void* K_codes, const void* V_codes,
                   const float* k_scale, const float* v_scale, const void* K_tail, const void* V_tail, const int32_t* lens,
                   const int32_t* blocks, int32_t nsel, float* out, void* workspace, size_t workspace_bytes, int32_t* status,
                   void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  rc = check_code(code_dtype);
  if (rc) return rc;
  if (!q || !K_codes || !V_codes || !k_scale || !v_scale || !K_tail || !V_tail || !lens || !out) return CORM_EINVAL;
  if (misaligned16(q) || misaligned16(K_codes) || misaligned16(V_codes) || misaligned16(K_tail) || misaligned16(V_tail)) return CORM_EINVAL;
  if (misaligned4(k_scale) || misaligned4(v_scale) || misaligned4(lens) || misaligned4(blocks) || misaligned4(out) || misaligned4(status))
    return CORM_EINVAL;
  if (blocks ? nsel < 1 || nsel > max_listed(desc) : nsel != 0) return CORM_EINVAL;
  rc = check_blocks_workspace(desc, workspace, workspace_bytes);
  if (rc) return rc;
  Q8Args a;
  a.q = q; a.Kc = reinterpret_cast<const unsigned char*>(K_codes); a.Vc = reinterpret_cast<const unsigned char*>(V_codes);
  a.ks = k_scale; a.vs = v_scale; a.Kt = K_tail; a.Vt = V_tail; a.lens = lens; a.blocks = blocks;
  a.out = out; a.partials = reinterpret_cast<float*>(workspace); a.status = status;
  a.Hq = desc->Hq; a.Hkv = desc->Hkv; a.Lcap = desc->Lcap; a.nblk = blocks_of(desc); a.nsel = blocks ? nsel : 0;
  a.scale_log2 = scale_log2(desc);
  const long units = (long)desc->B * desc->Hkv;
  const int listed = blocks ? nsel : a.nblk, real = std::min(listed, a.nblk);   // (a list holds at most the unit's blocks in earnest)
  const long cus = device_cus();
  // A workgroup takes a whole unit where there are two units per compute unit, or where a unit has few blocks; else parts of whole rounds of blocks
  // over the waves, at least two rounds unless the launch would then be small, up to 16 workgroups per compute unit, and a merge.
  // Whole calls, us, parts | whole: 512 units x 540 .. 2048 slots 47 | 36, 1000 x 1500 113 | 62, 1536 x 200 27 | 17; 256 x 190 .. 8192 56 | 76, 300 x 3000
  // 42 | 49; 8 to 128 units, 2 blocks 7.4 | 5.5 and 9.1 | 7.1, 5 blocks 8.5 | 7.6 and 10.7 | 8.4, 9 blocks 9.1 | 9.9 and 12.4 | 11.2, 17 blocks
  // 8.8 | 12.6 and 14.8 | 15.9.  Parts of 4 | 8 blocks: 32 x 4096 12.4 | 13.8, 8 x 32768 24.0 | 20.0.
  if (listed <= Q8_MOST && (units >= 2 * cus || real <= 2 * WAVES || (2 * units >= cus && real <= 4 * WAVES))) {
    a.part_blocks = (listed + WAVES - 1) / WAVES * WAVES;
    a.npart = 1;
  } else {
    const int least = units * ((listed + 2 * WAVES - 1) / (2 * WAVES)) < 2 * cus ? WAVES : 2 * WAVES;
    const int want = (int)std::min<long>((16 * cus + units - 1) / units, (listed + least - 1) / least);
    a.part_blocks = std::min(Q8_MOST, ((listed + want - 1) / want + WAVES - 1) / WAVES * WAVES);
    a.npart = (listed + a.part_blocks - 1) / a.part_blocks + 1;
  }
  a.units = (int)units;
  const long groups = (units * a.npart + Q8_XCDS - 1) / Q8_XCDS * Q8_XCDS;
  if (groups * WG > 4294967295L) return CORM_EUNSUPPORTED;   // (threads of a launch)
  hipStream_t s = (hipStream_t)stream;
  rc = by_types(desc, code_dtype, [&](auto c, auto dt, auto dd) {
    hipLaunchKernelGGL((corm_q8_attend_kernel<decltype(c), decltype(dt), decltype(dd)::value>), dim3((unsigned)groups), dim3(WG), 0, s, a);
    return launch_status();
  });
  if (rc) return rc;
  if (a.npart == 1) return CORM_OK;
  return merge_parts(desc, a.partials, lens, out, a.npart, blocks ? 0 : a.part_blocks, s);
}

int corm_block_bounds(const corm_desc* desc, const void* K, const int32_t* lens, int32_t newest, void* bounds, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!K || !lens || !bounds || misaligned16(K) || misaligned16(bounds) || misaligned4(lens) || newest < 0) return CORM_EINVAL;
  const int nblk = blocks_of(desc);
  const int n = newest > 0 ? (int)std::min<long long>(nblk, ((long long)newest + 2 * QBLK - 2) / QBLK) : nblk;
  return by_row(desc, [&](auto dt, auto dd) {
    hipLaunchKernelGGL((corm_block_bounds_kernel<decltype(dt), decltype(dd)::value>), dim3(n, desc->B * desc->Hkv), dim3(WG), 0,
                       (hipStream_t)stream, reinterpret_cast<const char*>(K), lens, reinterpret_cast<char*>(bounds), desc->Lcap, nblk,
                       newest);
    return launch_status();
  });
}

int corm_block_select(const corm_desc* desc, const void* q, const void* bounds, const int32_t* lens, int32_t nsel, int32_t nlast,
                      int32_t* blocks, void* workspace, size_t workspace_bytes, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!q || !bounds || !lens || !blocks || misaligned16(q) || misaligned16(bounds) || misaligned4(lens) || misaligned4(blocks))
    return CORM_EINVAL;
  if (nsel < 1 || nsel > max_listed(desc) || nlast < 1 || nlast > nsel) return CORM_EINVAL;
  rc = check_blocks_workspace(desc, workspace, workspace_bytes);
  if (rc) return rc;
  const int nblk = blocks_of(desc), units = desc->B * desc->Hkv;
  float* scores = reinterpret_cast<float*>(workspace);
  hipStream_t s = (hipStream_t)stream;
  const bool one = nblk <= CHOOSE_BLOCKS;
  rc = by_row(desc, [&](auto dt, auto dd) {
    return by_group(desc, [&](auto g) {
      using T = decltype(dt);
      constexpr int D = decltype(dd)::value, G = decltype(g)::value;
      const char* qc = reinterpret_cast<const char*>(q);
      const char* bc = reinterpret_cast<const char*>(bounds);
      if (one)
        hipLaunchKernelGGL((corm_block_choose_kernel<T, D, G>), dim3(units), dim3(CHOOSE_WG), 0, s, qc, bc, lens, blocks, desc->Lcap, nblk,
                           nsel, nlast);
      else
        hipLaunchKernelGGL((corm_block_score_kernel<T, D, G>), dim3((nblk + 63) / 64, units), dim3(64 * SCORE_SHARES), 0, s, qc, bc, lens, scores,
                           desc->Lcap, nblk);
      return launch_status();
    });
  });
  if (rc || one) return rc;
  hipLaunchKernelGGL(corm_block_pick_kernel, dim3(units), dim3(PICK_WG), 0, s, scores, lens, blocks, desc->Lcap, nblk, nsel, nlast);
  return launch_status();
}

int corm_block_attend(const corm_desc* desc, const void* q, const void* K, const void* V, const int32_t* lens, const int32_t* blocks,
                      int32_t nsel, float* out, void* workspace, size_t workspace_bytes, int32_t* status, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!q || !K || !V || !lens || !blocks || !out || misaligned16(q) || misaligned16(K) || misaligned16(V)) return CORM_EINVAL;
  if (misaligned4(lens) || misaligned4(blocks) || misaligned4(out) || misaligned4(status)) return CORM_EINVAL;
  if (nsel < 1 || nsel > max_listed(desc)) return CORM_EINVAL;
  rc = check_blocks_workspace(desc, workspace, workspace_bytes);
  if (rc) return rc;
  BlockAttendArgs a;
  a.q = reinterpret_cast<const char*>(q); a.K = reinterpret_cast<const char*>(K); a.V = reinterpret_cast<const char*>(V);
  a.lens = lens; a.blocks = blocks; a.partials = reinterpret_cast<float*>(workspace); a.out = out; a.status = status;
  a.Lcap = desc->Lcap; a.nsel = nsel; a.scale_log2 = scale_log2(desc);
  const long units = (long)desc->B * desc->Hkv;
  // The shortest parts (1, 2, 4 or 8 blocks) with which the launch has at most two workgroups for each compute unit, four where rows are 512 bytes; parts
  // of 8 where it has more all the same (a list holds at most the unit's blocks in earnest).  Whole steps, us, at most two | four | eight:
  // bf16 64 units x 64 blocks of eight heads 47.6 | 50.8 | 57.2, 288 units of up to 4 blocks in a list of 65 27.7 | 37.6 | 53.5; fp32 64 x 32
  // 42.7 | 39.1 | 39.2; bf16 128 x 64 parts of 8 (1024 workgroups, with two and with four) 69.7, of 4 (with eight) 71.7.
  const int room = max_parts(desc), real = std::min(nsel, blocks_of(desc));
  const long wgs = (row_bytes(desc) > 256 ? 4L : 2L) * device_cus();
  auto parts_of = [&](int n) { return (n + a.part_blocks - 1) / a.part_blocks; };
  a.part_blocks = 1;
  // (few blocks: one part, which writes out itself.  Whole steps, us, parts and merge | one part: bf16, 8 to 128 units, 2 blocks 15.6 | 13.5 and
  // 17.3 | 14.5, 4 blocks 15.5 | 14.9 and 20.4 | 16.4, 8 blocks 15.5 | 17.6 and 23.0 | 20.1; fp32 2 blocks 15.0 | 13.8 and 17.6 | 16.0, of eight heads
  // 21.3 | 22.2 and 25.3 | 24.5, 4 blocks 15.3 | 18.3)
  const bool few = nsel <= (desc->kv_dtype == CORM_F32 ? 2 : 4);
  while (a.part_blocks < LIST_PART && (few || units * parts_of(real) > wgs || parts_of(nsel) > room)) a.part_blocks *= 2;
  const int parts = parts_of(nsel);
  a.npart = parts;
  hipStream_t s = (hipStream_t)stream;
  const dim3 grid(parts, (unsigned)units);
  rc = by_group(desc, [&](auto g) {
    constexpr int G = decltype(g)::value;
    // (whole steps, vector ALU | matrix cores: 64 units of eight heads 61.5 | 49.9 us, 128 of four 71.9 | 69.8, 256 of two 108.9 | 109.3)
    if constexpr (G >= 4) {
      if (desc->kv_dtype == CORM_BF16 && desc->d == 128) {
        hipLaunchKernelGGL((corm_block_attend_gqa_kernel<G>), grid, dim3(WG), 0, s, a);
        return launch_status();
      }
    }
    return by_row(desc, [&](auto dt, auto dd) {
      hipLaunchKernelGGL((corm_block_attend_kernel<decltype(dt), decltype(dd)::value, G>), grid, dim3(WG), 0, s, a);
      return launch_status();
    });
  });
  if (rc || parts == 1) return rc;
  return merge_parts(desc, a.partials, lens, out, parts, 0, s);
}

int corm_evict_mask_weight(const corm_desc* desc, const float* weight, const int32_t* lens, int32_t budget, uint8_t* keep, void* workspace,
                           size_t workspace_bytes, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!weight || !lens || !keep || misaligned4(weight) || misaligned4(lens) || budget < desc->r) return CORM_EINVAL;
  rc = check_blocks_workspace(desc, workspace, workspace_bytes);
  if (rc) return rc;
  const int units = desc->B * desc->Hkv;
  hipStream_t s = (hipStream_t)stream;
  const EvictSplits e = evict_splits(desc);
  if (e.splits == 0) {
    hipLaunchKernelGGL(corm_evict_weight_kernel, dim3(units), dim3(EVW_WG), (size_t)desc->Lcap * sizeof(uint32_t), s, weight, lens, keep,
                       desc->Lcap, desc->r, budget);
    return launch_status();
  }
  char* ws = reinterpret_cast<char*>(workspace);
  EvictLongArgs a;
  a.weight = weight; a.lens = lens; a.keep = keep;
  a.hist = reinterpret_cast<uint32_t*>(ws);
  a.listed = reinterpret_cast<uint32_t*>(ws + e.listed_off);
  a.counts = reinterpret_cast<uint32_t*>(ws + e.counts_off);
  a.digit = reinterpret_cast<uint2*>(ws + e.digit_off);
  a.Lcap = desc->Lcap; a.r = desc->r; a.budget = budget; a.splits = e.splits; a.split_slots = e.slots;
  hipLaunchKernelGGL(corm_evict_count_kernel, dim3(e.splits, units), dim3(EVW_WG), 0, s, a);
  hipLaunchKernelGGL(corm_evict_part_kernel, dim3(e.splits, units), dim3(EVW_WG), 0, s, a);
  hipLaunchKernelGGL(corm_evict_settle_kernel, dim3(units), dim3(EVW_WG), 0, s, a);
  return launch_status();
}

}  // extern "C"
