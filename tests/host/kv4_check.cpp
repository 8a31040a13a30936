// Argument checks and size arithmetic of the 4-bit cache's entry points under AddressSanitizer / UndefinedBehaviorSanitizer: every integer
// argument at its extremes.  No call gets past its checks, so nothing touches a device.
#include <climits>
#include <cstdint>
#include <cstdio>
#include <cstring>

#include "../../include/s2d2_kv4.h"

static int g_bad = 0;
#define EXPECT(cond) do { if (!(cond)) { std::printf("FAILED line %d: %s (last error: %s)\n", __LINE__, #cond, s2d2_last_error()); ++g_bad; } } while (0)

int main() {
  void* fake = (void*)(uintptr_t)0x7f0000000000ull;
  s2d2_kv4_view good;
  std::memset(&good, 0, sizeof good);
  good.k_codes = good.v_codes = good.k_scales = good.v_scales = fake;
  good.mass = (float*)fake;
  good.position = good.entries = good.seq_len = good.status = (int32_t*)fake;
  good.page_table = (const int32_t*)fake;
  good.n_layers = 36; good.n_pages = 10000; good.page_size = 16; good.max_pages_per_seq = 1024; good.n_kv_heads = 8; good.head_dim = 128;
  s2d2_kv4_rows rows;
  std::memset(&rows, 0, sizeof rows);
  rows.N = 16; rows.T = 32; rows.rows = 512; rows.n_q_heads = 32; rows.dtype = S2D2_BF16; rows.scale = 0.1f;
  rows.q = rows.k = rows.v = fake; rows.q_stride = rows.out_stride = 32 * 128; rows.kv_stride = 8 * 128;
  rows.row0 = rows.n_rows = (const int32_t*)fake; rows.out = fake; rows.lse = (float*)fake;
  const int32_t* ints = (const int32_t*)fake;

  EXPECT(s2d2_kv4_attention_bytes(&good, 16, 32, 32) > 0);
  const int32_t extremes[] = {INT32_MIN, -1, 0, 1, 31, 32, 33, 1023, 1024, 1025, 65536, 1 << 30, INT32_MAX - 1, INT32_MAX};
  for (size_t f = 0; f < 6; ++f)
    for (int32_t v : extremes) {
      s2d2_kv4_view w = good;
      (&w.n_layers)[f] = v;
      const int64_t b = s2d2_kv4_attention_bytes(&w, 1024, 8192, 1024);
      EXPECT(b >= 0 || b == S2D2_EINVAL);
      // (a scratch that is always too small, a layer that is never there, a budget that is never allowed: nothing is launched)
      EXPECT(s2d2_kv4_attention(nullptr, &w, -1, &rows, fake, 0) == S2D2_EINVAL);
      EXPECT(s2d2_kv4_evict(nullptr, &w, 16, 0, 0, 0, 0, fake, SIZE_MAX) == S2D2_EINVAL && s2d2_kv4_evict_bytes(&w, 1024) != 0);
      EXPECT(s2d2_kv4_append(nullptr, &w, 16, 32, 512, 9, fake, fake, 0, 0, ints, ints) == S2D2_EINVAL);
      EXPECT(s2d2_kv4_read(nullptr, &w, 16, 32, 9, ints, fake, fake) == S2D2_EINVAL);
    }
  for (int32_t n : extremes)
    for (int32_t t : extremes)
      for (int32_t h : extremes) {
        const int64_t b = s2d2_kv4_attention_bytes(&good, n, t, h);
        const bool ok = n >= 1 && n <= 1024 && t >= 1 && t <= 8192 && h >= 1 && h <= 1024 && h % 8 == 0 && (int64_t)n * t * h <= 1 << 25;
        EXPECT(ok ? b > 0 : b == S2D2_EINVAL);
      }
  for (int32_t v : extremes)
    for (size_t f = 0; f < 4; ++f) {
      s2d2_kv4_rows r = rows;
      (&r.N)[f] = v;
      const int32_t rc = s2d2_kv4_attention(nullptr, &good, 0, &r, fake, 16);
      EXPECT(rc == S2D2_EINVAL || rc == S2D2_ENOSPC);
      r.lse = nullptr;
      EXPECT(s2d2_kv4_weigh(nullptr, &good, 0, &r) == S2D2_EINVAL);
    }
  const int64_t strides[] = {INT64_MIN, -8, 0, 8 * 128 - 8, 8 * 128 + 1, 1ll << 31, INT64_MAX};
  for (int64_t s : strides) {
    s2d2_kv4_rows r = rows;
    r.kv_stride = s;
    EXPECT(s2d2_kv4_attention(nullptr, &good, 0, &r, fake, 16) == S2D2_EINVAL);
    EXPECT(s2d2_kv4_append(nullptr, &good, 16, 32, 512, S2D2_BF16, fake, fake, 1 << 20, s, ints, ints) == S2D2_EINVAL);
    if (s != 1ll << 31) EXPECT(s2d2_kv4_append(nullptr, &good, 16, 32, 512, S2D2_BF16, fake, fake, s, 8 * 128, ints, ints) == S2D2_EINVAL);
  }
  for (int32_t a : extremes)
    for (int32_t b : extremes)
      if (a < 0 || b < 0 || (int64_t)a + b > 8) EXPECT(s2d2_kv4_evict(nullptr, &good, 16, 8, 0, a, b, fake, SIZE_MAX) == S2D2_EINVAL);
      else EXPECT(s2d2_kv4_evict(nullptr, &good, 16, 8, 0, a, b, fake, 8) == S2D2_ENOSPC);
  EXPECT(s2d2_kv4_attention_bytes(nullptr, 1, 1, 8) == S2D2_EINVAL);
  EXPECT(s2d2_set_kv4(nullptr, &good, fake, 0, nullptr) == S2D2_EINVAL && s2d2_set_kv4(nullptr, nullptr, nullptr, 0, nullptr) == S2D2_EINVAL);

  std::printf("kv4_check: %d failed expectation(s)\n", g_bad);
  return g_bad ? 1 : 0;
}
