// C entry points of the 4-bit cache: argument checks and launches.  The contract: include/s2d2_kv4.h.
#include "kv4.h"

#include <atomic>

using namespace s2d2;

namespace s2d2 {

int32_t check_kv4(const s2d2_kv4_view* kv) {
  if (!kv || !kv->k_codes || !kv->v_codes || !kv->k_scales || !kv->v_scales || !kv->page_table || !kv->entries || !kv->seq_len) return fail(S2D2_EINVAL, "4-bit cache or one of its pointers is NULL");
  if (((uintptr_t)kv->k_codes | (uintptr_t)kv->v_codes) & 15) return fail(S2D2_EINVAL, "4-bit cache: codes must be 16-byte aligned");
  if (((uintptr_t)kv->k_scales | (uintptr_t)kv->v_scales) & 7) return fail(S2D2_EINVAL, "4-bit cache: scales must be 8-byte aligned");
  if (((uintptr_t)kv->mass | (uintptr_t)kv->position | (uintptr_t)kv->page_table | (uintptr_t)kv->entries | (uintptr_t)kv->seq_len | (uintptr_t)kv->status) & 3) return fail(S2D2_EINVAL, "4-bit cache: mass, position, page_table, entries, seq_len and status must be 4-byte aligned");
  if (kv->n_layers < 1 || kv->n_layers > 4096 || kv->n_pages < 1 || kv->page_size < 1 || kv->max_pages_per_seq < 1) return fail(S2D2_EINVAL, "4-bit cache: n_layers (1-4096), n_pages, page_size and max_pages_per_seq must be positive");
  if ((int64_t)kv->max_pages_per_seq * kv->page_size >= (1 << 30)) return fail(S2D2_EINVAL, "4-bit cache: max_pages_per_seq * page_size must be below 2^30");
  if (kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return fail(S2D2_EINVAL, "4-bit cache: n_kv_heads must be in [1, 1024]");
  if (kv->head_dim != 32 && kv->head_dim != 64 && kv->head_dim != 128 && kv->head_dim != 256) return fail(S2D2_EINVAL, "4-bit cache: head_dim must be 32, 64, 128 or 256");
  return S2D2_OK;
}

int32_t kv4_ready() {
  static std::atomic<uint64_t> done{0};   // devices whose kernels have their LDS limit (a second call to the runtime does no harm)
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) { (void)hipGetLastError(); return fail(S2D2_EARCH, "no usable HIP device"); }
  if (dev < 64 && (done.load(std::memory_order_acquire) >> dev) & 1) return S2D2_OK;
  if (kv4_attention_init() || kv4_evict_init()) { (void)hipGetLastError(); return fail(S2D2_ELAUNCH, "could not raise the LDS limit of the 4-bit cache's kernels (device not gfx950?)"); }
  if (dev < 64) done.fetch_or(1ull << dev, std::memory_order_release);
  return S2D2_OK;
}

}  // namespace s2d2

namespace {

int32_t check_launch(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(S2D2_ELAUNCH, "%s: %s", what, hipGetErrorString(e));
  return S2D2_OK;
}

int32_t check_dtype(int32_t dtype) {
  if (dtype != S2D2_F32 && dtype != S2D2_BF16) return fail(S2D2_EINVAL, "dtype must be S2D2_F32 or S2D2_BF16");
  return S2D2_OK;
}
int32_t check_batch(int32_t N, int32_t T, int32_t most) {
  if (N < 1 || N > 1024) return fail(S2D2_EINVAL, "N=%d outside [1, 1024]", N);
  if (T < 1 || T > most) return fail(S2D2_EINVAL, "T=%d outside [1, %d]", T, most);
  return S2D2_OK;
}
int32_t check_rows(int32_t N, int32_t T) {
  if (((int64_t)T + 3) / 4 * N >= 1 << 24) return fail(S2D2_EINVAL, "N=%d sequences of up to T=%d rows are too many for one call", N, T);
  return S2D2_OK;
}
int32_t check_lists(const s2d2_kv4_view* kv, int32_t N) {
  if ((int64_t)N * kv->n_layers * kv->n_kv_heads >= 1 << 22) return fail(S2D2_EINVAL, "N * n_layers * n_kv_heads must be below 2^22");
  return S2D2_OK;
}
int32_t check_q_heads(const s2d2_kv4_view* kv, int32_t n_q_heads) {
  if (n_q_heads < 1 || n_q_heads > 1024 || n_q_heads % kv->n_kv_heads) return fail(S2D2_EINVAL, "n_q_heads=%d must be a positive multiple of n_kv_heads=%d, at most 1024", n_q_heads, kv->n_kv_heads);
  return S2D2_OK;
}
// Key tiles of a batch are counted in 31 bits; a launch has less than 2^32 threads a dimension.
int32_t check_keys(const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t n_q_heads) {
  if ((int64_t)N * T * n_q_heads > 1 << 25) return fail(S2D2_EINVAL, "N * T * n_q_heads = %lld above 2^25", (long long)N * T * n_q_heads);
  if (((int64_t)kv->max_pages_per_seq * kv->page_size + T + 64) * N >= (1ll << 36)) return fail(S2D2_EINVAL, "N=%d sequences of up to %lld keys are too many for one call", N, (long long)kv->max_pages_per_seq * kv->page_size + T);
  return S2D2_OK;
}
// A row stride in elements: whole 16 bytes, at least a row, and offsets of all rows in 63 bits
bool stride_ok(int64_t stride, int64_t width, int32_t dtype) { return stride >= width && stride < (1ll << 31) && stride % (dtype == S2D2_F32 ? 4 : 8) == 0; }

int32_t attn_args(const s2d2_kv4_view* kv, int32_t layer, const s2d2_kv4_rows* r, bool weigh, Kv4Attn& a) {
  int32_t rc;
  if ((rc = check_kv4(kv))) return rc;
  if (layer < 0 || layer >= kv->n_layers) return fail(S2D2_EINVAL, "layer=%d outside [0, n_layers=%d)", layer, kv->n_layers);
  if (!r) return fail(S2D2_EINVAL, "rows are NULL");
  if ((rc = check_batch(r->N, r->T, 8192)) || (rc = check_dtype(r->dtype)) || (rc = check_q_heads(kv, r->n_q_heads)) || (rc = check_keys(kv, r->N, r->T, r->n_q_heads))) return rc;
  if (r->rows < 1) return fail(S2D2_EINVAL, "rows=%d must be positive", r->rows);
  if (!(r->scale > 0.f) || r->scale > 2.35e38f) return fail(S2D2_EINVAL, "scale must be positive and at most 2.35e38 (scores are taken to base 2: scale * 1.4427 must be finite)");
  if (!r->q || !r->row0 || !r->n_rows) return fail(S2D2_EINVAL, "q, row0 or n_rows is NULL");
  const int64_t width = (int64_t)r->n_q_heads * kv->head_dim;
  if (((uintptr_t)r->q & 15) || !stride_ok(r->q_stride, width, r->dtype)) return fail(S2D2_EINVAL, "q must be 16-byte aligned, its row stride whole 16 bytes and at least %lld elements", (long long)width);
  if (((uintptr_t)r->row0 | (uintptr_t)r->n_rows | (uintptr_t)r->lo | (uintptr_t)r->hi | (uintptr_t)r->lse) & 3) return fail(S2D2_EINVAL, "row0, n_rows, lo, hi and lse must be 4-byte aligned");
  if (weigh) {
    if (!r->lse || !kv->mass) return fail(S2D2_EINVAL, "weighing needs lse and the cache's mass");
  } else {
    if (!r->out || ((uintptr_t)r->out & 15) || !stride_ok(r->out_stride, width, r->dtype)) return fail(S2D2_EINVAL, "out must be given and 16-byte aligned, its row stride whole 16 bytes and at least %lld elements", (long long)width);
    if (!r->k != !r->v || !r->lo != !r->hi) return fail(S2D2_EINVAL, "k and v, and lo and hi, are given together or not at all");
    if (r->k && ((((uintptr_t)r->k | (uintptr_t)r->v) & 15) || !stride_ok(r->kv_stride, (int64_t)kv->n_kv_heads * kv->head_dim, r->dtype))) return fail(S2D2_EINVAL, "k and v must be 16-byte aligned, their row stride whole 16 bytes and at least a row");
  }
  a = Kv4Attn{};
  a.kv = kv4_of(kv);
  a.N = r->N; a.T = a.expect = r->T; a.rows = r->rows; a.Hq = r->n_q_heads; a.grp = r->n_q_heads / kv->n_kv_heads;
  a.q = r->q; a.q_ld = r->q_stride; a.row0 = r->row0; a.n_rows = r->n_rows; a.lse = r->lse;
  a.group = divisor_of(a.grp);
  a.scale_log2e = r->scale * 1.44269504088896340736f;
  if (!weigh) { a.k = r->k; a.v = r->v; a.kv_ld = r->kv_stride; a.lo = r->k ? r->lo : nullptr; a.hi = r->k ? r->hi : nullptr; a.out = r->out; a.o_ld = r->out_stride; }
  return S2D2_OK;
}

}  // namespace

extern "C" {

int32_t s2d2_kv4_append(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t rows, int32_t dtype, const void* k, const void* v,
                        int64_t layer_stride, int64_t row_stride, const int32_t* row0, const int32_t* n_rows) {
  int32_t rc;
  if ((rc = check_kv4(kv)) || (rc = check_batch(N, T, 1 << 20)) || (rc = check_rows(N, T)) || (rc = check_dtype(dtype))) return rc;
  if (rows < 1) return fail(S2D2_EINVAL, "rows=%d must be positive", rows);
  if (!k || !v || !row0 || !n_rows) return fail(S2D2_EINVAL, "k, v, row0 or n_rows is NULL");
  if ((((uintptr_t)k | (uintptr_t)v) & 15) || (((uintptr_t)row0 | (uintptr_t)n_rows) & 3)) return fail(S2D2_EINVAL, "k and v must be 16-byte aligned, row0 and n_rows 4-byte");
  const int64_t width = (int64_t)kv->n_kv_heads * kv->head_dim, e = dtype == S2D2_F32 ? 4 : 8;
  if (!stride_ok(row_stride, width, dtype)) return fail(S2D2_EINVAL, "row_stride must be whole 16 bytes and at least %lld elements", (long long)width);
  if (layer_stride < 0 || layer_stride % e || layer_stride >= (1ll << 50) || (kv->n_layers > 1 && layer_stride < width)) return fail(S2D2_EINVAL, "layer_stride must be whole 16 bytes and at least a row");
  if ((rc = kv4_ready())) return rc;
  launch_kv4_append((hipStream_t)stream, dtype, kv4_of(kv), N, Kv4Rows{row0, n_rows, nullptr, nullptr, 0, T, rows}, k, v, layer_stride, row_stride, nullptr, 0);
  return check_launch("s2d2_kv4_append");
}

int32_t s2d2_kv4_read(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t dtype, const int32_t* first, void* k, void* v) {
  int32_t rc;
  if ((rc = check_kv4(kv)) || (rc = check_batch(N, T, 1 << 20)) || (rc = check_rows(N, T)) || (rc = check_dtype(dtype))) return rc;
  if (!first || !k || !v || (((uintptr_t)k | (uintptr_t)v) & 15) || ((uintptr_t)first & 3)) return fail(S2D2_EINVAL, "first, k or v is NULL or not aligned (k, v: 16 bytes)");
  if ((rc = kv4_ready())) return rc;
  launch_kv4_read((hipStream_t)stream, dtype, kv4_of(kv), N, T, first, k, v);
  return check_launch("s2d2_kv4_read");
}

int64_t s2d2_kv4_attention_bytes(const s2d2_kv4_view* kv, int32_t N, int32_t T, int32_t n_q_heads) {
  int32_t rc;
  if ((rc = check_kv4(kv)) || (rc = check_batch(N, T, 8192)) || (rc = check_q_heads(kv, n_q_heads)) || (rc = check_keys(kv, N, T, n_q_heads))) return rc;
  return (int64_t)kv4_attention_bytes(kv4_of(kv), N, T, n_q_heads);
}

int32_t s2d2_kv4_attention(void* stream, const s2d2_kv4_view* kv, int32_t layer, const s2d2_kv4_rows* rows, void* scratch, size_t scratch_bytes) {
  Kv4Attn a;
  int32_t rc;
  if ((rc = attn_args(kv, layer, rows, false, a))) return rc;
  const size_t need = kv4_attention_bytes(a.kv, a.N, a.T, a.Hq);
  if (scratch_bytes < need) return fail(S2D2_ENOSPC, "scratch has %zu bytes, %zu needed", scratch_bytes, need);
  if (need && (!scratch || ((uintptr_t)scratch & 15))) return fail(S2D2_EINVAL, "scratch is NULL or not 16-byte aligned");
  if ((rc = kv4_ready())) return rc;
  const int mode = rows->dtype == S2D2_F32 ? Q_F32 : Q_BF16;
  if (launch_kv4_attention((hipStream_t)stream, mode, a, layer, scratch)) launch_kv4_merge((hipStream_t)stream, mode, a);
  return check_launch("s2d2_kv4_attention");
}

int32_t s2d2_kv4_weigh(void* stream, const s2d2_kv4_view* kv, int32_t layer, const s2d2_kv4_rows* rows) {
  Kv4Attn a;
  int32_t rc;
  if ((rc = attn_args(kv, layer, rows, true, a)) || (rc = kv4_ready())) return rc;
  launch_kv4_weigh((hipStream_t)stream, rows->dtype == S2D2_F32 ? Q_F32 : Q_BF16, a, layer);
  return check_launch("s2d2_kv4_weigh");
}

int64_t s2d2_kv4_evict_bytes(const s2d2_kv4_view* kv, int32_t N) {
  int32_t rc;
  if ((rc = check_kv4(kv)) || (rc = check_batch(N, 1, 1)) || (rc = check_lists(kv, N))) return rc;
  return (int64_t)kv4_evict_bytes(kv4_of(kv), N);
}

int32_t s2d2_kv4_evict(void* stream, const s2d2_kv4_view* kv, int32_t N, int32_t budget, int32_t slack, int32_t sink, int32_t recent, void* scratch,
                       size_t scratch_bytes) {
  int32_t rc;
  if ((rc = check_kv4(kv)) || (rc = check_batch(N, 1, 1)) || (rc = check_lists(kv, N))) return rc;
  if (!kv->mass || !kv->position) return fail(S2D2_EINVAL, "eviction needs the cache's mass and position");
  if (budget < 1 || slack < 0 || sink < 0 || recent < 0 || (int64_t)sink + recent > budget) return fail(S2D2_EINVAL, "budget=%d must be positive, slack=%d, sink=%d and recent=%d non-negative, sink + recent at most budget", budget, slack, sink, recent);
  const size_t need = kv4_evict_bytes(kv4_of(kv), N);
  if (scratch_bytes < need) return fail(S2D2_ENOSPC, "scratch has %zu bytes, %zu needed", scratch_bytes, need);
  if (!scratch || ((uintptr_t)scratch & 3)) return fail(S2D2_EINVAL, "scratch is NULL or not 4-byte aligned");
  if ((rc = kv4_ready())) return rc;
  launch_kv4_evict((hipStream_t)stream, kv4_of(kv), N, budget, slack, sink, recent, scratch);
  return check_launch("s2d2_kv4_evict");
}

}  // extern "C"
