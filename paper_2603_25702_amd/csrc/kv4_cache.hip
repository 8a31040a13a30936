// The 4-bit cache: quantising append, entries read back, eviction by gathered attention weight.
// Format and semantics: include/s2d2_kv4.h.  Append, read and move take few operations a byte; 24 MB, 5 us at a copy's rate, take 10 to 12 (each workgroup makes one pass
// behind a chain of counts, entries and page table).  Picking makes several passes over a list.
#include "kv4.h"

#include <algorithm>

namespace s2d2 {

Kv4 kv4_of(const s2d2_kv4_view* view) {
  const s2d2_kv4_view& w = *view;
  Kv4 k;
  k.kc = (uint8_t*)w.k_codes; k.vc = (uint8_t*)w.v_codes; k.ks = (uint8_t*)w.k_scales; k.vs = (uint8_t*)w.v_scales;
  k.mass = w.mass; k.position = w.position; k.page_table = w.page_table; k.entries = w.entries; k.seq_len = w.seq_len; k.status = w.status;
  k.n_layers = w.n_layers; k.n_pages = w.n_pages; k.max_pages = w.max_pages_per_seq; k.H = w.n_kv_heads; k.D = w.head_dim;
  k.cap = w.max_pages_per_seq * w.page_size;
  k.ps = divisor_of(w.page_size);
  k.layer_entries = (size_t)w.n_pages * w.n_kv_heads * w.page_size;
  return k;
}

// ---------------------------------------------------------------------------------------------
// Append.  A thread takes 8 values of a row (a 16-byte load of bf16), four neighbours make a group: the group's largest |x| goes round
// by two DPP moves as an integer (the bits of |x| order as |x| does, with NaN above infinity above all else), v_cvt_scalef32_pk_fp4_f32
// rounds x / 2^e to nearest-even codes.
// 36 layers x 16 sequences of up to 16 rows, 8 heads of 128, bf16: 12 us; 8 layers x 4 of up to 192 rows, fp32: 9.5.  The counts follow in a launch of
// their own (2 to 4 us): a row's place depends on the count that every workgroup of the first one reads.
// ---------------------------------------------------------------------------------------------
static constexpr int APPEND_ROWS = 4;   // rows of a sequence per workgroup, all in flight at once

template <typename T>
__device__ __forceinline__ void load8(const T* p, float (&x)[8]) {
  if (sizeof(T) == 2) {
    const uint4 r = *(const uint4*)p;
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
  } else {
    const float4 a = ((const float4*)p)[0], b = ((const float4*)p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
}

// Codes of the 8 values of this lane and the scale byte of its group (lanes 4 g .. 4 g + 3 hold a group).
__device__ __forceinline__ uint32_t kv4_quantise(const float (&x)[8], uint32_t& scale) {
  int a = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) a = max(a, (int)(__float_as_uint(x[i]) & 0x7fffffffu));
  a = max(a, __builtin_amdgcn_mov_dpp(a, 0xb1, 0xf, 0xf, true));
  a = max(a, __builtin_amdgcn_mov_dpp(a, 0x4e, 0xf, 0xf, true));
  const int e = kv4_exponent(__int_as_float(a));
  const float s = __int_as_float((e + 127) << 23);
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  const bool bad = a >= 0x7f800000;
  scale = bad ? 255u : (uint32_t)(e + 127);
  return bad ? 0u : c;
}

template <typename T>
__global__ __launch_bounds__(256) void kv4_append_kernel(Kv4 kv, Kv4Rows r, int per_seq, const T* __restrict__ k, const T* __restrict__ v,
                                                         int64_t layer_stride, int64_t row_stride, const float* __restrict__ row_mass, int64_t mass_stride) {
  const int n = blockIdx.x / per_seq, l = blockIdx.y;
  const int rows = r.count(n), S = kv.held(n), t0 = (blockIdx.x % per_seq) * APPEND_ROWS;
  if (t0 >= rows || r.row0[n] > r.rows - rows || S + rows > kv.cap) return;   // (the commit flags a sequence without room)
  const int pos0 = kv.seq_len[n], units = kv.H * kv.D / 8, per_head = kv.D / 8;
  const int here = min(APPEND_ROWS, rows - t0);
  const int64_t row = l * layer_stride + (int64_t)(r.row0[n] + t0) * row_stride;
  int page[APPEND_ROWS], slot[APPEND_ROWS];
#pragma unroll
  for (int t = 0; t < APPEND_ROWS; ++t) {
    const int place = S + t0 + min(t, here - 1), p = kv.ps.div(place);
    page[t] = kv.page_table[(size_t)n * kv.max_pages + p];
    slot[t] = place - p * kv.ps.d;
  }
  for (int i = threadIdx.x; i < 2 * units; i += 256) {   // (a multiple of four: the lanes of a group stay together)
    const int value = i >= units, w = i - value * units, head = w / per_head, part = w % per_head;
    const T* src = (value ? v : k) + row + (size_t)w * 8;
    float x[APPEND_ROWS][8];
#pragma unroll
    for (int t = 0; t < APPEND_ROWS; ++t) load8(src + min(t, here - 1) * row_stride, x[t]);
#pragma unroll
    for (int t = 0; t < APPEND_ROWS; ++t) {
      uint32_t scale;
      const uint32_t codes = kv4_quantise(x[t], scale);
      if (t >= here || page[t] < 0 || page[t] >= kv.n_pages) continue;
      const size_t at = l * kv.layer_entries + kv.at(page[t], head, slot[t]);
      ((uint32_t*)((value ? kv.vc : kv.kc) + at * (kv.D / 2)))[part] = codes;
      if ((part & 3) == 0) (value ? kv.vs : kv.ks)[at * (kv.D / 32) + part / 4] = (uint8_t)scale;
      if (part == 0 && !value) {
        if (kv.mass) kv.mass[at] = row_mass ? row_mass[l * mass_stride + (int64_t)(r.row0[n] + t0 + t) * kv.H + head] : 0.f;
        if (kv.position) kv.position[at] = pos0 + t0 + t;
      }
    }
  }
}

__global__ void kv4_append_commit_kernel(Kv4 kv, Kv4Rows r, int N) {
  const int n = blockIdx.x * blockDim.x + threadIdx.x;
  if (n >= N) return;
  const int rows = r.count(n), S = kv.held(n);
  if (rows == 0 || r.row0[n] > r.rows - rows) return;
  if (S + rows > kv.cap) {
    if (kv.status) kv.status[n] = S2D2_ENOSPC;
    return;
  }
  kv.entries[n] = S + rows;
  kv.seq_len[n] += rows;
}

void launch_kv4_append(hipStream_t st, int dtype, const Kv4& kv, int N, const Kv4Rows& r, const void* k, const void* v, int64_t layer_stride, int64_t row_stride,
                       const float* row_mass, int64_t mass_stride) {
  const int per_seq = (r.most + APPEND_ROWS - 1) / APPEND_ROWS;
  const dim3 grid(N * per_seq, kv.n_layers);
  if (dtype == S2D2_BF16)
    S2D2_LAUNCH(kv4_append_kernel<bf16_t>, grid, dim3(256), 0, st, kv, r, per_seq, (const bf16_t*)k, (const bf16_t*)v, layer_stride, row_stride, row_mass, mass_stride);
  else
    S2D2_LAUNCH(kv4_append_kernel<float>, grid, dim3(256), 0, st, kv, r, per_seq, (const float*)k, (const float*)v, layer_stride, row_stride, row_mass, mass_stride);
  S2D2_LAUNCH(kv4_append_commit_kernel, dim3((N + 255) / 256), dim3(256), 0, st, kv, r, N);
}

// ---------------------------------------------------------------------------------------------
// Entries read back: 8 values a thread of each of READ_ROWS entries.  10.5 us for the rows of either append above.
// ---------------------------------------------------------------------------------------------
typedef __attribute__((ext_vector_type(2))) float f32x2_t;
static constexpr int READ_ROWS = 4;
template <typename T>
__global__ __launch_bounds__(256) void kv4_read_kernel(Kv4 kv, int N, int T_, int per_seq, const int32_t* __restrict__ first, T* __restrict__ k, T* __restrict__ v) {
  const int n = blockIdx.x / per_seq, t0 = (blockIdx.x % per_seq) * READ_ROWS, l = blockIdx.y;
  const int held = kv.held(n);
  const int64_t place0 = (int64_t)first[n] + t0;
  if (place0 >= held || place0 <= -READ_ROWS) return;
  const int units = kv.H * kv.D / 8, per_head = kv.D / 8;
  size_t entry[READ_ROWS];
  bool there[READ_ROWS];
#pragma unroll
  for (int t = 0; t < READ_ROWS; ++t) {
    const int64_t place = place0 + t;
    there[t] = t0 + t < T_ && place >= 0 && place < held;
    const int i = (int)max((int64_t)0, min(place, (int64_t)held - 1)), p = kv.ps.div(i);
    entry[t] = l * kv.layer_entries + kv.at(max(0, min(kv.page_table[(size_t)n * kv.max_pages + p], kv.n_pages - 1)), 0, i - p * kv.ps.d);
  }
  for (int i = threadIdx.x; i < 2 * units; i += 256) {
    const int value = i >= units, w = i - value * units, head = w / per_head, part = w % per_head;
    const uint8_t *codes = value ? kv.vc : kv.kc, *scales = value ? kv.vs : kv.ks;
    uint32_t c[READ_ROWS], e[READ_ROWS];
#pragma unroll
    for (int t = 0; t < READ_ROWS; ++t) {
      const size_t at = entry[t] + (size_t)head * kv.ps.d;
      c[t] = ((const uint32_t*)(codes + at * (kv.D / 2)))[part];
      e[t] = scales[at * (kv.D / 32) + part / 4];
    }
#pragma unroll
    for (int t = 0; t < READ_ROWS; ++t) {
      if (!there[t]) continue;
      const float s = __uint_as_float(e[t] << 23);   // (255: the conversion gives NaN)
      const f32x2_t x[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[t], s, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[t], s, 1),
                            __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[t], s, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[t], s, 3)};
      T* to = (value ? v : k) + (((size_t)l * N + n) * T_ + t0 + t) * kv.H * kv.D + (size_t)w * 8;
      if (sizeof(T) == 2) {
        // (exact: a code times a power of two has two significant bits)
        auto two = [](f32x2_t y) { return (__float_as_uint(y[0]) >> 16) | (__float_as_uint(y[1]) & 0xffff0000u); };
        *(uint4*)to = make_uint4(two(x[0]), two(x[1]), two(x[2]), two(x[3]));
      } else {
        ((float4*)to)[0] = make_float4(x[0][0], x[0][1], x[1][0], x[1][1]);
        ((float4*)to)[1] = make_float4(x[2][0], x[2][1], x[3][0], x[3][1]);
      }
    }
  }
}

void launch_kv4_read(hipStream_t st, int dtype, const Kv4& kv, int N, int T, const int32_t* first, void* k, void* v) {
  const int per_seq = (T + READ_ROWS - 1) / READ_ROWS;
  const dim3 grid(N * per_seq, kv.n_layers);
  if (dtype == S2D2_BF16) S2D2_LAUNCH(kv4_read_kernel<bf16_t>, grid, dim3(256), 0, st, kv, N, T, per_seq, first, (bf16_t*)k, (bf16_t*)v);
  else S2D2_LAUNCH(kv4_read_kernel<float>, grid, dim3(256), 0, st, kv, N, T, per_seq, first, (float*)k, (float*)v);
}

// ---------------------------------------------------------------------------------------------
// Eviction, in two launches.
//
// kv4_pick_kernel: a workgroup per list (sequence, layer, KV head).  The list's masses become integers that order as they do (keys), kept in LDS;
// three histograms of 11, 11 and 10 bits find the key of the budget-th largest; of the entries that hold exactly that key the first ones
// stay.  Entries below the budget that go are filled from those behind it that stay, in order: the list's moves go to the scratch.
// A wavefront owns a run of consecutive entries where ranks are needed: its counts go through LDS once, ranks inside it come from ballots.
// kv4_move_kernel: the moves of all lists by as many workgroups as there are compute units for.  Places that are written lie below the budget,
// places that are read behind it, so the moves need no order among themselves; and a list that is a little too long moves a few entries only.
// 512 lists of 4160 entries to 4096: 33 us to pick, 7 to move; 32 lists of 32768 to 4096: 69 and 15.  The 512 lists are one round of workgroups, two a compute
// unit: vector instructions issue in 52 % of the time, a wavefront waits (barriers, LDS, memory) for 61 % of its life.  The 32 long lists keep 32 of 256 compute units busy.
// ---------------------------------------------------------------------------------------------
static constexpr int EVICT_KEYS = 36864;   // keys kept in LDS (144 KB); those of longer lists are formed again from memory
// Lists up to here by eight wavefronts, two workgroups a compute unit.  Both launches, us, by eight / sixteen: 4608 lists of 4160 entries (36 layers) 179 / 246, 512 of them 30 / 35, 1024 of
// 600 25 / 39, 32 of 1000 16 / 18; few long ones the other way, 256 of 8192 34 / 28; by four, 512 of 4160 take a fifth longer than by eight.
static constexpr int PICK_SHORT = 8192;
static constexpr int EVICT_AHEAD = 4;      // entries or moves that a thread has in flight

__device__ __forceinline__ uint32_t evict_key(float mass, int position, int sink, int tail) {
  if (position < sink || position >= tail) return 0xffffffffu;
  if (mass != mass) return 0u;
  const uint32_t u = __float_as_uint(mass + 0.f);   // (-0 as 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Sum over the workgroup's wavefronts before this one, and over all: `mine` of each wavefront (uniform in it).
template <int W>
__device__ __forceinline__ int waves_before(int mine, int32_t* s /* [W] */, int& all) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[wave] = mine;
  __syncthreads();
  int before = 0;
  all = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    const int x = s[w];
    before += w < wave ? x : 0;
    all += x;
  }
  return before;
}

// The moves of a list: count[list] of them (-1: the list is not cut), to[list][m] <- from[list][m], entries of the list.
struct EvictMoves {
  int32_t *count, *to, *from;
  size_t most;   // of a list
};

template <int W>
__global__ __launch_bounds__(64 * W, W == 16 ? 8 : 4) void kv4_pick_kernel(Kv4 kv, int budget, int slack, int sink, int recent, int keys, EvictMoves mv) {
  extern __shared__ uint32_t s_mem[];
  uint32_t* s_key = s_mem;                             // [keys]
  uint32_t* s_hist = s_key + keys;                     // [2048]
  int32_t* s_sum = (int32_t*)(s_hist + 2048);          // [W]
  uint32_t* s_pick = (uint32_t*)(s_sum + W); // [3]: bin, entries of it that stay, entries of it
  const int head = blockIdx.x % kv.H, n = blockIdx.x / kv.H, l = blockIdx.y;
  const size_t list = ((size_t)n * kv.n_layers + l) * kv.H + head;
  const int E = kv.held(n), tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (E <= budget || E - budget <= slack) {
    if (tid == 0) mv.count[list] = -1;
    return;
  }
  const int32_t* pt = kv.page_table + (size_t)n * kv.max_pages;
  const int tail = kv.seq_len[n] - recent;
  auto form = [&](int i) __attribute__((always_inline)) {
    const int p = kv.ps.div(i), page = max(0, min(pt[p], kv.n_pages - 1));   // (a page outside the cache is read as the nearest one)
    const size_t at = l * kv.layer_entries + kv.at(page, head, i - p * kv.ps.d);
    return evict_key(kv.mass[at], kv.position[at], sink, tail);
  };
  auto key = [&](int i) __attribute__((always_inline)) { return i < keys ? s_key[i] : form(i); };
  auto key_of = [&](int i) __attribute__((always_inline)) { return i < E ? key(i) : 0u; };
  constexpr int STEP = 64 * W;

  // ---- the budget-th largest key ----
  uint32_t prefix = 0;
  int need = budget;   // among the keys with this prefix
  int shift = 32;
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10;
    for (int i = tid; i < 2048; i += STEP) s_hist[i] = 0;
    __syncthreads();
    for (int i0 = tid; i0 - tid < E; i0 += EVICT_AHEAD * STEP) {
      uint32_t k[EVICT_AHEAD];
      if (pass == 0) {
#pragma unroll
        for (int u = 0; u < EVICT_AHEAD; ++u) k[u] = form(min(i0 + u * STEP, E - 1));
#pragma unroll
        for (int u = 0; u < EVICT_AHEAD; ++u)
          if (i0 + u * STEP < min(E, keys)) s_key[i0 + u * STEP] = k[u];
      } else
#pragma unroll
        for (int u = 0; u < EVICT_AHEAD; ++u) k[u] = key_of(i0 + u * STEP);
#pragma unroll
      for (int u = 0; u < EVICT_AHEAD; ++u) {
        const bool counts = i0 + u * STEP < E && (pass == 0 || (k[u] >> shift) == prefix);
        const int bin = (int)((k[u] >> (shift - bits)) & ((1u << bits) - 1));
        // entries without weight share a bin: the lanes that agree with the first one add once
        const unsigned long long who = __ballot(counts);
        if (who) {
          const int lead = __ffsll((long long)who) - 1, first = __builtin_amdgcn_readlane(bin, lead);
          const unsigned long long same = __ballot(counts && bin == first);
          if (lane == lead) atomicAdd(&s_hist[first], (uint32_t)__popcll(same));
          else if (counts && bin != first) atomicAdd(&s_hist[bin], 1u);
        }
      }
    }
    __syncthreads();
    // counts from the top: thread t holds bins 2047 - BINS t and on downwards
    constexpr int BINS = 2048 / STEP;
    int x[BINS], mine = 0;
#pragma unroll
    for (int u = 0; u < BINS; ++u) { x[u] = (int)s_hist[2047 - BINS * tid - u]; mine += x[u]; }
    int incl = mine;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int y = __shfl_up(incl, off, 64);
      if (lane >= off) incl += y;
    }
    int all, above = waves_before<W>(__builtin_amdgcn_readlane(incl, 63), s_sum, all) + incl - mine;
#pragma unroll
    for (int u = 0; u < BINS; ++u) {
      if (above < need && above + x[u] >= need) { s_pick[0] = 2047 - BINS * tid - u; s_pick[1] = need - above; s_pick[2] = x[u]; }
      above += x[u];
    }
    __syncthreads();
    shift -= bits;
    prefix = (prefix << bits) | s_pick[0];
    need = (int)s_pick[1];
  }
  const uint32_t last = prefix;   // of the entries with this key the first `need` stay

  // ---- who stays: wavefront w walks entries [w0, w1) ----
  const int run = ((E + STEP - 1) / STEP) * 64, w0 = min(E, wave * run), w1 = min(E, w0 + run);
  auto lanes_below = [&](unsigned long long m) __attribute__((always_inline)) { return __popcll(m & ((1ull << lane) - 1)); };
  int all, equal0 = 0;
  const bool tied = (int)s_pick[2] != need;   // some entries with the last key go
  if (tied) {
    int equal = 0;
    for (int i = w0 + lane; i - lane < w1; i += 64) equal += __popcll(__ballot(i < w1 && key(i) == last));
    equal0 = waves_before<W>(equal, s_sum, all);
  }
  // calls put(entry, whether it goes and is written, whether it stays and is read) for the wavefront's entries in order, all lanes together
  auto walk = [&](auto put) __attribute__((always_inline)) {
    int seen = equal0;
    for (int i0 = w0 + lane; i0 - lane < w1; i0 += 64 * EVICT_AHEAD) {
      uint32_t k[EVICT_AHEAD];
#pragma unroll
      for (int u = 0; u < EVICT_AHEAD; ++u) k[u] = key_of(i0 + 64 * u);
#pragma unroll
      for (int u = 0; u < EVICT_AHEAD; ++u) {
        const int i = i0 + 64 * u;
        const bool in = i < w1;
        bool stays = in && k[u] >= last;
        if (tied) {
          const unsigned long long eq = __ballot(in && k[u] == last);
          if (k[u] == last && seen + lanes_below(eq) >= need) stays = false;
          seen += __popcll(eq);
        }
        put(i, in && i < budget && !stays, stays && i >= budget);
      }
    }
  };
  int holes = 0, kept = 0;
  walk([&](int, bool hole, bool source) __attribute__((always_inline)) {
    holes += __popcll(__ballot(hole));
    kept += __popcll(__ballot(source));
  });
  int moves;
  int hole0 = waves_before<W>(holes, s_sum, moves), kept0 = waves_before<W>(kept, s_sum, all);   // (as many of one as of the other)
  int32_t *to = mv.to + list * mv.most, *from = mv.from + list * mv.most;
  walk([&](int i, bool hole, bool source) __attribute__((always_inline)) {
    const unsigned long long goes = __ballot(hole), comes = __ballot(source);
    if (hole) to[hole0 + lanes_below(goes)] = i;
    if (source) from[kept0 + lanes_below(comes)] = i;
    hole0 += __popcll(goes);
    kept0 += __popcll(comes);
  });
  if (tid == 0) mv.count[list] = moves;
}

// width: threads of a move, enough for the 16-byte pieces of K and V and for scales, mass and position (a power of two); per_list: workgroups
__global__ __launch_bounds__(256) void kv4_move_kernel(Kv4 kv, int budget, int width, int per_list, EvictMoves mv) {
  const size_t list = blockIdx.x / per_list;
  const int slice = blockIdx.x % per_list, head = (int)(list % kv.H), l = (int)(list / kv.H % kv.n_layers), n = (int)(list / kv.H / kv.n_layers);
  const int moves = mv.count[list];
  if (moves < 0) return;
  if (l == 0 && head == 0 && slice == 0 && threadIdx.x == 0) kv.entries[n] = budget;
  const int codes = kv.D / 32, j = threadIdx.x % width, step = 256 / width * per_list;
  if (j >= 2 * codes + 4) return;
  const int32_t *pt = kv.page_table + (size_t)n * kv.max_pages, *to_of = mv.to + list * mv.most, *from_of = mv.from + list * mv.most;
  for (int m0 = slice * (256 / width) + threadIdx.x / width; m0 < moves; m0 += EVICT_AHEAD * step) {
    size_t to[EVICT_AHEAD], from[EVICT_AHEAD];
    bool there[EVICT_AHEAD];
#pragma unroll
    for (int u = 0; u < EVICT_AHEAD; ++u) {
      const int m = min(m0 + u * step, moves - 1), a = to_of[m], b = from_of[m], pa = kv.ps.div(a), pb = kv.ps.div(b), page = pt[pa];
      there[u] = m0 + u * step < moves && page >= 0 && page < kv.n_pages;   // (a page outside the cache is never written)
      to[u] = l * kv.layer_entries + kv.at(max(0, min(page, kv.n_pages - 1)), head, a - pa * kv.ps.d);
      from[u] = l * kv.layer_entries + kv.at(max(0, min(pt[pb], kv.n_pages - 1)), head, b - pb * kv.ps.d);
    }
    auto move = [&](auto word, void* base, int per_entry, int piece) __attribute__((always_inline)) {
      using W = decltype(word);
      W x[EVICT_AHEAD];
#pragma unroll
      for (int u = 0; u < EVICT_AHEAD; ++u) x[u] = ((const W*)base)[from[u] * per_entry + piece];
#pragma unroll
      for (int u = 0; u < EVICT_AHEAD; ++u)
        if (there[u]) ((W*)base)[to[u] * per_entry + piece] = x[u];
    };
    if (j < 2 * codes) move(u32x4_t{}, j < codes ? kv.kc : kv.vc, codes, j < codes ? j : j - codes);
    else if (j >= 2 * codes + 2) move(uint32_t{}, j == 2 * codes + 2 ? (void*)kv.mass : (void*)kv.position, 1, 0);
    else {   // the scales of an entry: one word of 1, 2, 4 or 8 bytes
      void* base = j == 2 * codes ? kv.ks : kv.vs;
      if (codes == 1) move(uint8_t{}, base, 1, 0);
      else if (codes == 2) move(uint16_t{}, base, 1, 0);
      else if (codes == 4) move(uint32_t{}, base, 1, 0);
      else move(uint64_t{}, base, 1, 0);
    }
  }
}

static size_t pick_lds(int keys) { return ((size_t)keys + 2048 + 16 + 3) * sizeof(uint32_t); }

// A list has at most as many moves as entries below the budget, and as behind it: half its places.
size_t kv4_evict_bytes(const Kv4& kv, int N) {
  const size_t lists = (size_t)N * kv.n_layers * kv.H;
  return (lists * (1 + 2 * (size_t)(kv.cap / 2)) * sizeof(int32_t) + 255) & ~(size_t)255;
}

void launch_kv4_evict(hipStream_t st, const Kv4& kv, int N, int budget, int slack, int sink, int recent, void* scratch) {
  const int keys = kv.cap < EVICT_KEYS ? kv.cap : EVICT_KEYS, most = std::min(budget, kv.cap - budget);
  if (most <= 0) return;   // (no list is longer)
  const size_t lists = (size_t)N * kv.n_layers * kv.H;
  EvictMoves mv{(int32_t*)scratch, (int32_t*)scratch + lists, nullptr, (size_t)most};
  mv.from = mv.to + lists * mv.most;
  const dim3 grid(N * kv.H, kv.n_layers);
  if (kv.cap <= PICK_SHORT) S2D2_LAUNCH(kv4_pick_kernel<8>, grid, dim3(512), pick_lds(keys), st, kv, budget, slack, sink, recent, keys, mv);
  else S2D2_LAUNCH(kv4_pick_kernel<16>, grid, dim3(1024), pick_lds(keys), st, kv, budget, slack, sink, recent, keys, mv);
  const int codes = kv.D / 32, width = 2 * codes + 4 <= 8 ? 8 : 2 * codes + 4 <= 16 ? 16 : 32, at_once = 256 / width * EVICT_AHEAD;
  const int per_list = std::max(1, std::min((int)((2048 + lists - 1) / lists), (most + at_once - 1) / at_once));
  S2D2_LAUNCH(kv4_move_kernel, dim3((unsigned)(lists * per_list)), dim3(256), 0, st, kv, budget, width, per_list, mv);
}

// LDS above 64 KB has to be asked for, once a device.
int kv4_evict_init() {
  return hipFuncSetAttribute((const void*)kv4_pick_kernel<16>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)pick_lds(EVICT_KEYS)) != hipSuccess;
}

}  // namespace s2d2
