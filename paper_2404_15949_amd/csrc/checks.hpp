// host side: what every translation unit's entry points share -- descriptor and pointer checks, sizes, the device's compute units.
// Included after <hip/hip_runtime.h>, <cmath>, <mutex> and corm.h.
#ifndef CORM_CHECKS_HPP
#define CORM_CHECKS_HPP

namespace {

size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

int row_bytes(const corm_desc* d) { return d->d * (d->kv_dtype == CORM_F32 ? 4 : 2); }

int validate_desc(const corm_desc* d) {
  if (!d) return CORM_EINVAL;
  if (d->B < 1 || d->Hq < 1 || d->Hkv < 1 || d->Lcap < 1 || d->Tcap < 1 || d->w < 1 || d->r < 1) return CORM_EINVAL;
  if (d->Hq % d->Hkv != 0) return CORM_EINVAL;
  if (!(d->thr_scale >= 0.f) || !std::isfinite(d->thr_scale)) return CORM_EINVAL;
  if (!(d->sm_scale >= 0.f) || !std::isfinite(d->sm_scale)) return CORM_EINVAL;
  if ((long long)d->B * d->Hkv > 2147483647LL / 2 || (long long)d->B * d->Hq > 2147483647LL / 2) return CORM_EINVAL;
  if (d->B * d->Hkv > 65535) return CORM_EUNSUPPORTED;  // grid.y limit
  if ((long long)d->Lcap * 512 >= (1LL << 31)) return CORM_EUNSUPPORTED;  // byte offsets inside a unit are 32-bit
  if (d->kv_dtype != CORM_F32 && d->kv_dtype != CORM_BF16) return CORM_EUNSUPPORTED;
  if (d->score_dtype != CORM_F32 && d->score_dtype != CORM_BF16 && d->score_dtype != CORM_BIT) return CORM_EUNSUPPORTED;
  if (d->d != 64 && d->d != 128) return CORM_EUNSUPPORTED;
  const int G = d->Hq / d->Hkv;
  if (G != 1 && G != 2 && G != 4 && G != 8) return CORM_EUNSUPPORTED;
  return CORM_OK;
}

bool misaligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) != 0; }
bool misaligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) != 0; }

int launch_status() { return hipGetLastError() == hipSuccess ? CORM_OK : CORM_EHIP; }

// Compute units of the current device, asked once per device (thread safe); 256 where no device answers.
constexpr int MAX_DEVICES = 64;
std::mutex g_device_mutex;
int g_device_cus[MAX_DEVICES] = {};

int device_cus() {
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= MAX_DEVICES) return 256;
  std::lock_guard<std::mutex> lock(g_device_mutex);
  if (g_device_cus[dev] == 0) {
    int n = 0;
    if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || n <= 0) n = 256;
    g_device_cus[dev] = n;
  }
  return g_device_cus[dev];
}

}  // namespace

#endif  // CORM_CHECKS_HPP
