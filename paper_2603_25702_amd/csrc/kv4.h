// The 4-bit cache on the device, as its kernels see it.  Format and semantics: include/s2d2_kv4.h.
#pragma once
#include "s2d2_internal.h"
#include "../../include/s2d2_kv4.h"

namespace s2d2 {

// x / d for 0 <= x < 2^31: the high half of 2 x * m, m = ceil(2^(31 + s) / d), s = ceil(log2 d).  m d - 2^(31 + s) < d <= 2^s, so
// the error of the product stays below 2^(31 + s) / d and the quotient is exact.
struct Divisor {
  uint32_t mul, shift;
  int32_t d;
  __device__ __forceinline__ int div(int x) const { return (int)(__umulhi((uint32_t)x << 1, mul) >> shift); }
};
inline Divisor divisor_of(int d) {
  Divisor v{0, 0, d};
  while ((1ll << v.shift) < d) ++v.shift;
  v.mul = (uint32_t)(((1ull << (31 + v.shift)) + d - 1) / (uint64_t)d);
  return v;
}

struct Kv4 {
  uint8_t *kc, *vc, *ks, *vs;   // of layer 0
  float* mass;
  int32_t* position;
  const int32_t* page_table;
  int32_t *entries, *seq_len, *status;
  int32_t n_layers, n_pages, max_pages, H, D, cap;
  Divisor ps;
  size_t layer_entries;         // entries of a layer: n_pages * H * page size
  __device__ __forceinline__ int held(int n) const { return max(0, min(entries[n], cap)); }
  // Entry index (of K / V head 0) of a page's slot; the page as it is
  __device__ __forceinline__ size_t at(int page, int head, int slot) const { return ((size_t)page * H + head) * ps.d + slot; }
};
Kv4 kv4_of(const s2d2_kv4_view* view);
int32_t check_kv4(const s2d2_kv4_view* view);
int32_t kv4_ready();            // once a device: 0, or what s2d2_last_error says

// Smallest e with 6 * 2^e >= a, cut to what the format has: a = f * 2^p with 1 <= f < 2, and 6 = 1.5 * 2^2.
__device__ __forceinline__ int kv4_exponent(float a) {
  const uint32_t u = __float_as_uint(a);
  const int e = (int)(u >> 23) - 127 - 2 + ((u & 0x7fffffu) > 0x400000u ? 1 : 0);
  return max(-23, min(13, e));
}

// Windows and their operands as the attention kernels take them.  q_lo: offset of a second plane of the queries (0: none); o_lo: storage of
// the output rows of a bf16 model (act_put4); f32 models take and leave fp32 rows.
struct Kv4Attn {
  Kv4 kv;
  int32_t N, T, rows, Hq, grp;
  const void *q, *k, *v;
  int64_t q_ld, kv_ld, o_ld;
  int32_t q_lo, o_lo;
  const int32_t *row0, *n_rows, *lo, *hi;
  void* out;
  float* lse;
  float* row_mass;     // weighing: [rows, KV heads], what the window's rows give each other (k, lo and hi needed), or NULL
  const void* window_k;   // weighing: the window's keys
  float scale_log2e;   // scores to base 2
  float *part_o, *part_ml;
  int2* part_of;     // [N] of a sequence with several splits: its first item, its splits
  int32_t expect;    // rows that a sequence is expected to have (at most T): what the splits are chosen for
  int32_t groups;    // groups of query tiles of T rows
  int32_t q_tiles, per_wg;   // query tiles of T rows, and of a workgroup
  int32_t items;     // (sequence, split) pairs the grid holds
  int32_t per_item;  // workgroups of one with the expected rows: KV heads * groups of query tiles
  int32_t room;      // splits beyond one a sequence that the scratch holds
  int32_t target;    // workgroups to aim for
  int32_t min_run;   // tiles of a split, at least
  int32_t cached_wgs;  // weighing: workgroups of the cached entries; those of the window's tiles follow
  Divisor group;     // by query heads per KV head
};

// Queries and window rows: bf16; bf16 queries in two planes; queries and window keys as half values; fp32
enum Kv4Query { Q_BF16 = 0, Q_BF16X2 = 1, Q_F16 = 2, Q_F32 = 3 };
bool launch_kv4_attention(hipStream_t st, int mode, Kv4Attn& a, int layer, void* scratch);   // whether a sequence may have several splits, for launch_kv4_merge to join
void launch_kv4_merge(hipStream_t st, int mode, const Kv4Attn& a);
size_t kv4_attention_bytes(const Kv4& kv, int N, int T, int Hq);
void launch_kv4_weigh(hipStream_t st, int mode, Kv4Attn& a, int layer);
int kv4_evict_init();
int kv4_attention_init();

// Rows to append of sequence n: n_rows[n], or a verification's: lead[n] + min(accepted[n], span[n] - hold_back).
struct Kv4Rows {
  const int32_t *row0, *n_rows, *accepted, *span;
  int32_t hold_back, most, rows;   // most: of one sequence; rows: that there are
  __device__ __forceinline__ int count(int n) const {
    const int c = min(n_rows[n], most) + (accepted ? max(0, min(accepted[n], span[n] - hold_back)) : 0);
    return row0[n] < 0 || c < 0 ? 0 : min(c, most);
  }
};
// row_mass: [layers, mass_stride / KV heads rows, KV heads], the mass that the rows bring along; NULL: 0
void launch_kv4_append(hipStream_t st, int dtype, const Kv4& kv, int N, const Kv4Rows& r, const void* k, const void* v, int64_t layer_stride, int64_t row_stride,
                       const float* row_mass, int64_t mass_stride);
void launch_kv4_read(hipStream_t st, int dtype, const Kv4& kv, int N, int T, const int32_t* first, void* k, void* v);
void launch_kv4_evict(hipStream_t st, const Kv4& kv, int N, int budget, int slack, int sink, int recent, void* scratch);
size_t kv4_evict_bytes(const Kv4& kv, int N);

}  // namespace s2d2
