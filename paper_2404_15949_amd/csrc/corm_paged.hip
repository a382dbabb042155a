// HIP kernels (gfx950 / CDNA4, wave64) and C ABI of a cache of pages and of the rows on their way into it.
// One translation unit:
//   codes.hpp   8-bit codes
//   rows.hpp    norms of queries and keys, the position rotation, rows into pages and out of them
//   paged.hpp   attention of one new token over pages
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
#include "codes.hpp"
#include "rows.hpp"
#include "paged.hpp"
#include "checks.hpp"

namespace {

int elem_bytes(const corm_desc* d) { return d->kv_dtype == CORM_F32 ? 4 : 2; }
bool in_codes(const corm_pages* p) { return p->dtype == CORM_I8 || p->dtype == CORM_E4M3; }

int check_pages(const corm_desc* d, const corm_pages* p) {
  if (!p || !p->K || !p->V || !p->table || p->reserved != 0) return CORM_EINVAL;
  if (!in_codes(p) && p->dtype != d->kv_dtype) return CORM_EUNSUPPORTED;
  if (misaligned16(p->K) || misaligned16(p->V) || misaligned4(p->table)) return CORM_EINVAL;
  if (in_codes(p) && (!p->k_scale || !p->v_scale || misaligned16(p->k_scale) || misaligned16(p->v_scale))) return CORM_EINVAL;
  if (p->page != 16 && p->page != 32 && p->page != 64 && p->page != 128 && p->page != 256) return CORM_EUNSUPPORTED;
  if (p->npages < 1 || p->max_pages < 1) return CORM_EINVAL;
  if (p->table_heads != 1 && p->table_heads != d->Hkv) return CORM_EINVAL;
  if ((long long)p->max_pages * p->page < d->Lcap) return CORM_EINVAL;
  return CORM_OK;
}

PageView view_of(const corm_desc* d, const corm_pages* p) {
  PageView v;
  v.K = reinterpret_cast<char*>(p->K); v.V = reinterpret_cast<char*>(p->V); v.ks = p->k_scale; v.vs = p->v_scale;
  v.table = p->table; v.npages = p->npages; v.max_pages = p->max_pages; v.TH = p->table_heads; v.HP = d->Hkv / p->table_heads;
  v.shift = 4;
  while ((1 << v.shift) < p->page) ++v.shift;
  return v;
}

int check_rotation(const corm_desc* d, const corm_rotation* r, const int32_t* positions) {
  if (!r) return CORM_OK;
  if (r->rot < 0 || r->rot > d->d || r->rot % 16 != 0 || r->axes < 1 || r->axes > 4) return CORM_EINVAL;
  if (r->pairing != CORM_HALVES && r->pairing != CORM_NEIGHBOURS) return CORM_EINVAL;
  if (!(r->eps >= 0.f) || !std::isfinite(r->eps) || !std::isfinite(r->gain)) return CORM_EINVAL;
  if (misaligned16(r->q_norm) || misaligned16(r->k_norm)) return CORM_EINVAL;
  if (r->rot == 0) return CORM_OK;
  if (!r->inv_freq || misaligned4(r->inv_freq) || !positions || misaligned4(positions)) return CORM_EINVAL;
  long long sum = 0;
  for (int x = 0; x < r->axes; ++x) {
    if (r->section[x] < 0) return CORM_EINVAL;
    sum += r->section[x];
    // dealt in turn, the axis has pairs x, x + axes, ..: there have to be as many
    if (r->in_turn && x > 0 && r->section[x] > 0 && x + ((long long)r->section[x] - 1) * r->axes >= r->rot / 2) return CORM_EINVAL;
  }
  return sum == r->rot / 2 ? CORM_OK : CORM_EINVAL;
}

int check_rows(const corm_desc* d, const corm_rows* r, int n, bool with_q) {
  if (!r || !r->k || !r->v || misaligned16(r->k) || misaligned16(r->v)) return CORM_EINVAL;
  if (with_q && (!r->q || misaligned16(r->q))) return CORM_EINVAL;
  // strides: none is beyond any memory, and the last row's offset is well within 64 bits
  auto bad = [&](const int64_t* s, int heads) {
    const int rows[3] = {d->B, n, heads};
    __int128 span = 0;
    for (int i = 0; i < 3; ++i) {
      if (s[i] < 0 || s[i] > (1LL << 40) || s[i] % (16 / elem_bytes(d)) != 0) return true;
      span += (__int128)s[i] * (rows[i] - 1) * elem_bytes(d);
    }
    return span > ((__int128)1 << 62);
  };
  return bad(r->k_stride, d->Hkv) || bad(r->v_stride, d->Hkv) || (with_q && bad(r->q_stride, d->Hq)) ? CORM_EINVAL : CORM_OK;
}

RowStrides bytes_of(const int64_t* s, int esz) { return RowStrides{s[0] * esz, s[1] * esz, s[2] * esz}; }

void bind_rows(const corm_desc* d, const corm_rows* r, const corm_rotation* rot, const int32_t* positions, int n, const int32_t* n_new,
               RowsArgs& a) {
  const int esz = elem_bytes(d);
  a = RowsArgs();
  a.q = reinterpret_cast<const char*>(r->q); a.k = reinterpret_cast<const char*>(r->k); a.v = reinterpret_cast<const char*>(r->v);
  a.qs = bytes_of(r->q_stride, esz); a.ks = bytes_of(r->k_stride, esz); a.vs = bytes_of(r->v_stride, esz);
  a.n_new = n_new; a.B = d->B; a.n = n; a.Hkv = d->Hkv; a.Lcap = d->Lcap;
  a.axes = 1;
  if (rot) {
    a.inv_freq = rot->inv_freq; a.positions = positions;
    a.q_norm = reinterpret_cast<const char*>(rot->q_norm); a.k_norm = reinterpret_cast<const char*>(rot->k_norm);
    a.rot = rot->rot; a.axes = rot->axes; a.in_turn = rot->in_turn != 0;
    for (int i = 0; i < 4; ++i) a.section[i] = i < rot->axes ? rot->section[i] : 0;
    a.eps = rot->eps; a.gain = rot->gain;
  }
  a.joined = a.rot == 0 || rot->pairing == CORM_NEIGHBOURS;
}

template <typename C, typename DT, int D>
int launch_rows_d(RowsArgs& a, hipStream_t s) {
  constexpr int RPW = 512 / D;   // rows of a wave
  const int heads = a.Hq + 2 * a.Hkv;
  // Groups of tokens once they make two workgroups per compute unit, else a workgroup a token.  Us, a token | a group: bf16, d 128, 48 heads, 512, 1024,
  // 2048, 4096 and 8192 tokens 6.5 | 12.2, 10.0 | 13.1, 16.9 | 15.9, 31.2 | 22.2 and 67 | 47; fp32, d 64, 10 heads, 2048 and 8192 4.9 | 5.8 and 10.4 | 9.7.
  const bool tokens = a.n >= RPW && (long)a.n * a.B >= 2L * RPW * device_cus();
  const dim3 grid((unsigned)(tokens ? ((long)a.n + RPW - 1) / RPW : a.n), a.B), wg(64 * (tokens ? 4 : std::min(16, (heads + RPW - 1) / RPW)));
  if ((long long)grid.x * wg.x > 4294967295LL) return CORM_EUNSUPPORTED;   // (threads of a launch)
  a.lens_here = a.lens_out && (grid.x == 1 || a.lens_out != a.lens);
  auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, wg, 0, s, a); };
  if (tokens) a.joined ? launch(corm_rows_kernel<C, DT, D, true, true>) : launch(corm_rows_kernel<C, DT, D, true, false>);
  else a.joined ? launch(corm_rows_kernel<C, DT, D, false, true>) : launch(corm_rows_kernel<C, DT, D, false, false>);
  const int rc = launch_status();
  if (rc || !a.lens_out || a.lens_here) return rc;
  hipLaunchKernelGGL(corm_rows_lens_kernel, dim3(a.B), dim3(WG), 0, s, a);
  return launch_status();
}

template <typename C>
int launch_rows(const corm_desc* d, RowsArgs& a, hipStream_t s) {
  if (d->kv_dtype == CORM_F32) return d->d == 64 ? launch_rows_d<C, F32, 64>(a, s) : launch_rows_d<C, F32, 128>(a, s);
  return d->d == 64 ? launch_rows_d<C, BF16, 64>(a, s) : launch_rows_d<C, BF16, 128>(a, s);
}

// Workgroups that the workspace has room for, two partials each (of those that share all units' tiles; a round's workgroup of a short unit has one).
constexpr int PAGED_MOST = 1024;
struct PagedWorkspace {
  size_t parts_off, total;
};
PagedWorkspace paged_workspace(const corm_desc* d) {
  PagedWorkspace w;
  w.parts_off = align_up((size_t)PAGED_MOST * 2 * (d->Hq / d->Hkv) * (d->d + 2) * sizeof(float), 256);
  w.total = align_up(w.parts_off + (size_t)d->B * d->Hkv * sizeof(int2), 256);
  return w;
}

// How the tiles of a call are dealt out to workgroups.
// A workgroup takes a whole unit where there are two units per compute unit, or one and they are short, or where they are very short; units whose rounds
// all fit the chip at once get a workgroup for each; else all units' tiles are shared out.  The host knows the bound of the lengths, not the lengths: of two units
// per compute unit and more, one that is far longer than the others holds the call up (64 sequences of 8 heads, one of 131072 slots and 63 of 500: 1750 us, where 63
// such sequences, whose tiles are shared out, take 120).  Us, bf16, d 128, four heads a unit, rounds of 128 slots:
//   whole | shared           256 units x 760, 1500 and 4096 slots 20.0 | 25.3, 34.8 | 42.4 and 84.7 | 90.9; 384 x 760 and 4096 32.2 | 37.1 and 149 | 132;
//                            320 x 0 .. 1500 and 1000 .. 6000 44.8 | 50.3 and 157 | 100; 512 x 548 .. 2048 67 | 71
//   whole | one each, merged 8 x 250, 380 and 510 6.9 | 8.4, 7.9 | 8.2 and 9.4 | 8.4; 128 x 380 10.9 | 13.3
//   shared | units in equal parts, whatever their lengths   128 x 4192 .. 8192 73 | 77, x 0 .. 16384 102 | 120, x 4096 51 | 50; 8 x 131072 int8 55 | 53 (each pair on one card)
constexpr int PAGED_CUS = 256;   // compute units that the rule goes by, at most
struct Deal {
  bool shared;
  int npart;        // not shared: workgroups of a unit, one or one for each round over its waves
  int workgroups;   // shared: of all units
};
constexpr Deal deal_out(long units, long rounds, long cus) {   // rounds: of a unit as long as the lengths' bound allows
  const bool alone = units >= 2 * cus || (units >= cus && rounds <= 16) || rounds <= 3;
  const bool shared = !alone && units * rounds > 2 * cus;
  return Deal{shared, alone || shared ? 1 : (int)rounds, (int)(2 * cus)};
}
// Units that are not dealt out whole are fewer than 2 PAGED_CUS, and those with parts have no more than so many of them: a workgroup can add the tables up, the
// workspace holds the partials, and 32 bits count the tiles (of units of less than 2^31 / 512 slots).
static_assert(2 * PAGED_CUS <= SHARE_TABLES && 2 * PAGED_CUS <= PAGED_MOST, "");
static_assert(2L * PAGED_CUS * ((1L << 31) / 512 / PoolF32::TILE + 2 * WAVES) + 2 * PAGED_CUS < 2147483647L, "");

// kernel<pool, query type, d> by the call's types
template <typename F>
int by_pool(const corm_desc* d, const corm_pages* p, const F& f) {
  auto inner = [&](auto pool, auto dt) {
    return d->d == 64 ? f(pool, dt, std::integral_constant<int, 64>()) : f(pool, dt, std::integral_constant<int, 128>());
  };
  const bool f32 = d->kv_dtype == CORM_F32;
  if (p->dtype == CORM_I8) return f32 ? inner(PoolI8(), F32()) : inner(PoolI8(), BF16());
  if (p->dtype == CORM_E4M3) return f32 ? inner(PoolE4M3(), F32()) : inner(PoolE4M3(), BF16());
  return f32 ? inner(PoolF32(), F32()) : inner(PoolBF16(), BF16());
}

}  // namespace

extern "C" {

int corm_rotate(const corm_desc* desc, const corm_rows* rows, const corm_rotation* rotation, const int32_t* positions, int32_t n,
                const int32_t* n_new, void* q_out, void* k_out, void* v_out, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!rotation || !k_out || !v_out || misaligned16(q_out) || misaligned16(k_out) || misaligned16(v_out)) return CORM_EINVAL;
  if (n < 1 || misaligned4(n_new)) return CORM_EINVAL;
  rc = check_rows(desc, rows, n, q_out != nullptr);
  if (rc) return rc;
  rc = check_rotation(desc, rotation, positions);
  if (rc) return rc;
  RowsArgs a;
  bind_rows(desc, rows, rotation, positions, n, n_new, a);
  a.Hq = q_out ? desc->Hq : 0;
  a.q_out = reinterpret_cast<char*>(q_out); a.k_out = reinterpret_cast<char*>(k_out); a.v_out = reinterpret_cast<char*>(v_out);
  return launch_rows<AsIs>(desc, a, (hipStream_t)stream);
}

int corm_paged_append(const corm_desc* desc, const corm_pages* pages, const corm_rows* rows, const corm_rotation* rotation,
                      const int32_t* positions, int32_t n, const int32_t* n_new, void* q_out, const int32_t* lens, int32_t* lens_out,
                      int32_t* status, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  rc = check_pages(desc, pages);
  if (rc) return rc;
  if (!lens || !lens_out || misaligned4(lens) || misaligned4(lens_out) || misaligned4(status) || misaligned4(n_new) || misaligned16(q_out))
    return CORM_EINVAL;
  if (n < 1 || n > desc->Lcap) return CORM_EINVAL;
  rc = check_rows(desc, rows, n, q_out != nullptr);
  if (rc) return rc;
  rc = check_rotation(desc, rotation, positions);
  if (rc) return rc;
  RowsArgs a;
  bind_rows(desc, rows, rotation, positions, n, n_new, a);
  a.Hq = q_out ? desc->Hq : 0;
  a.q_out = reinterpret_cast<char*>(q_out);
  a.pages = view_of(desc, pages);
  a.lens = lens; a.lens_out = lens_out; a.status = status;
  hipStream_t s = (hipStream_t)stream;
  if (pages->dtype == CORM_I8) return launch_rows<CodeI8>(desc, a, s);
  if (pages->dtype == CORM_E4M3) return launch_rows<CodeE4M3>(desc, a, s);
  return launch_rows<AsIs>(desc, a, s);
}

int corm_paged_read(const corm_desc* desc, const corm_pages* pages, const int32_t* lens, int32_t n, void* K_out, void* V_out,
                    int32_t* status, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  rc = check_pages(desc, pages);
  if (rc) return rc;
  if (!lens || !K_out || !V_out || misaligned4(lens) || misaligned16(K_out) || misaligned16(V_out) || misaligned4(status) || n < 1)
    return CORM_EINVAL;
  ReadArgs a;
  a.pages = view_of(desc, pages);
  a.lens = lens; a.K_out = reinterpret_cast<char*>(K_out); a.V_out = reinterpret_cast<char*>(V_out); a.status = status;
  a.Hkv = desc->Hkv; a.Lcap = desc->Lcap; a.n = n;
  const int rows = WG / (row_bytes(desc) / 16);   // of a workgroup
  const dim3 grid((std::min(n, desc->Lcap) + rows - 1) / rows, desc->B * desc->Hkv);
  return by_pool(desc, pages, [&](auto pool, auto dt, auto dd) {
    using P = decltype(pool);
    using C = std::conditional_t<std::is_same_v<P, PoolI8>, CodeI8, std::conditional_t<std::is_same_v<P, PoolE4M3>, CodeE4M3, AsIs>>;
    hipLaunchKernelGGL((corm_paged_read_kernel<C, decltype(dt), decltype(dd)::value>), grid, dim3(WG), 0, (hipStream_t)stream, a);
    return launch_status();
  });
}

int corm_paged_workspace_bytes(const corm_desc* desc, size_t* bytes) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  if (!bytes) return CORM_EINVAL;
  *bytes = paged_workspace(desc).total;
  return CORM_OK;
}

int corm_paged_attend(const corm_desc* desc, const corm_pages* pages, const void* q, const int32_t* lens, float* out, void* workspace,
                      size_t workspace_bytes, int32_t* status, void* stream) {
  int rc = validate_desc(desc);
  if (rc) return rc;
  rc = check_pages(desc, pages);
  if (rc) return rc;
  if (!q || !lens || !out || misaligned16(q) || misaligned4(lens) || misaligned4(out) || misaligned4(status)) return CORM_EINVAL;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u)) return CORM_EINVAL;
  const PagedWorkspace w = paged_workspace(desc);
  if (workspace_bytes < w.total) return CORM_ECAPACITY;
  PagedArgs a;
  a.pages = view_of(desc, pages);
  a.q = q; a.lens = lens; a.out = out; a.partials = reinterpret_cast<float*>(workspace);
  a.parts = reinterpret_cast<int2*>(reinterpret_cast<char*>(workspace) + w.parts_off); a.status = status;
  a.Hkv = desc->Hkv; a.G = desc->Hq / desc->Hkv; a.Lcap = desc->Lcap;
  a.scale_log2 = (desc->sm_scale > 0.f ? desc->sm_scale : 1.0f / sqrtf((float)desc->d)) * LOG2E;
  a.units = desc->B * desc->Hkv;
  const int tile = in_codes(pages) ? PoolI8::TILE : desc->kv_dtype == CORM_F32 ? PoolF32::TILE : PoolBF16::TILE;
  const Deal deal = deal_out(a.units, ((desc->Lcap + tile - 1) / tile + WAVES - 1) / WAVES, std::min(device_cus(), PAGED_CUS));
  a.tables = desc->B * pages->table_heads;
  a.workgroups = deal.workgroups;
  a.npart = deal.npart;
  hipStream_t s = (hipStream_t)stream;
  auto merge = [&](auto shared_, int parts) {
    constexpr bool SHARED = decltype(shared_)::value;
    const bool many = parts > 32;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3((unsigned)(desc->B * desc->Hq)), dim3(many ? 1024 : 256), 0, s, a, tile); };
    if (desc->d == 64) many ? launch(corm_paged_merge_kernel<64, SHARED, 1024>) : launch(corm_paged_merge_kernel<64, SHARED, 256>);
    else many ? launch(corm_paged_merge_kernel<128, SHARED, 1024>) : launch(corm_paged_merge_kernel<128, SHARED, 256>);
    return launch_status();
  };
  if (deal.shared) {
    rc = by_pool(desc, pages, [&](auto pool, auto dt, auto dd) {
      hipLaunchKernelGGL((corm_paged_attend_kernel<decltype(pool), decltype(dt), decltype(dd)::value, true>), dim3(a.workgroups), dim3(WG), 0, s, a);
      return launch_status();
    });
    return rc ? rc : merge(std::true_type(), a.workgroups / a.units + 2);
  }
  const long groups = ((long)a.units * a.npart + Q8_XCDS - 1) / Q8_XCDS * Q8_XCDS;
  rc = by_pool(desc, pages, [&](auto pool, auto dt, auto dd) {
    hipLaunchKernelGGL((corm_paged_attend_kernel<decltype(pool), decltype(dt), decltype(dd)::value, false>), dim3((unsigned)groups), dim3(WG), 0, s, a);
    return launch_status();
  });
  return rc || a.npart == 1 ? rc : merge(std::false_type(), a.npart);
}

}  // extern "C"
