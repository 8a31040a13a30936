// Attention over the 4-bit cache and the windows' own rows, and the weights its entries gather.
// Format and semantics: include/s2d2_kv4.h.
#include "kv4.h"

#include <algorithm>
#include <type_traits>

namespace s2d2 {

// ---------------------------------------------------------------------------------------------
// kv4_attention_kernel: split-key attention on 32x32x16 MFMA.
//
// A query row is a (window row, query head of the group) pair, so a KV head's entries are read once for its group.  A
// workgroup has one sequence, one KV head, QT tiles of 32 query rows and a run of tiles of 32 keys; its wavefronts take every NW-th of
// them, each with a running maximum and sum of its own, and are merged at the end.
//   S^T = K Q^T   the codes of a key become bf16 in the registers that the matrix instruction reads (v_cvt_scalef32_pk_bf16_fp4 applies the
//                 group's power of two; every value is exact), so a lane holds one key's half row; the order of the dimensions in the
//                 contraction is free and is the one that makes that half row contiguous in memory
//   O^T = V^T P^T the contraction runs over keys while a lane holds one key: V goes through LDS as half values (exact as well) and
//                 comes back transposed (ds_read_b64_tr_b16).  The rows of S^T are fed in an order that leaves the accumulators of a lane,
//                 packed to half, as the operand P^T
// A lane owns one query row (its column of S^T), so maximum, sum and scale need an exchange between two lanes only.  Scores are exponentiated
// against a reference that lies 2^7 below the maximum it was taken from and follows the maximum when the weights of a tile sum up to more than
// 2^15: most tiles need no maximum and rescale nothing, and half keeps 11 bits of a weight down to 2^-21 of the largest and 2^-32 of it below (with the maximum itself as the
// reference a million entries of 2^-24 each would lose a tenth of their weights).  Sums are in 32 bits.
// Operands of more than 16 bits (fp32 models; queries in two planes) are split into planes of bf16, whose products are exact in 32 bits: 3
// planes hold the 24 bits of a float.  Softmax weights are half (11 bits; off by at most 2^-12 of the weight); of fp32 models three planes of bf16, V then goes
// through LDS as bf16.
// The window's own rows, a few tiles, take the same way with K in the caller's type and V, weights in planes of bf16.
// Measured (us, head dimension 128): 16 sequences x 32 rows x 32 heads on 8 over 8192 entries, 98 (69 GFLOP at 700 TFLOP/s).  By its counters the vector
// instructions issue in 51 % of that time and the matrix cores are busy in 36 %, while a wavefront waits for 39 % of its life: the chain of a tile (V
// into LDS, scores, softmax, V back) with two wavefronts a SIMD to cover it.  4 x 1 row over 60000 to 65536 entries, 55 (283 MB at 5.1 TB/s, read from three caches in
// turn, more than the memory-side cache holds; a copy of 4 GiB reads and writes 4.7); 1 x 1 row over 512 entries, 12 (launch, dependent loads, the join of the
// wavefronts).  fp32 rows: the 16 x 32 rows 228; with their weights in two half planes, which lose the small ones, 200.
// ---------------------------------------------------------------------------------------------
static constexpr float LN2 = 0.69314718055994530942f;
static constexpr float LOWEST = -3.402823466e38f;   // reference of a row that has seen nothing
static constexpr float BELOW = 7.f;                 // a reference is taken this far below a maximum (base 2)
static constexpr float MOST = 32768.f;              // and moves when the weights of a tile of keys sum up to more
// Wavefronts of a workgroup, one workgroup a compute unit: two a SIMD cover each other's waits.  A pass by four / eight of them: 16 x 32 rows over 8192 entries
// 139 / 104 us, 4 x 1 row over 60000 to 65536 86 / 62, 1 x 1 row over 512 20 / 12.  Heads of 256 take 128 registers for the output alone: four wavefronts of up to 512 registers, else eight of up to 256.
constexpr int waves_of(int D) { return D == 256 ? 4 : 8; }
constexpr int min_run_of(int D) { return 4 * waves_of(D); }   // tiles of a split, at least: four a wavefront (a join costs a launch of 4 to 5 us)

template <int QM> struct Mode;
// QP: planes of the queries; PP: of the softmax weights on cached values (half; of fp32 models bf16); WP: of the window's keys and values; WPP: of the weights on them (bf16)
template <> struct Mode<Q_BF16> { typedef bf16_t T; static constexpr int QP = 1, PP = 1, WP = 1, WPP = 2; };
template <> struct Mode<Q_BF16X2> { typedef bf16_t T; static constexpr int QP = 2, PP = 1, WP = 1, WPP = 2; };
template <> struct Mode<Q_F16> { typedef bf16_t T; static constexpr int QP = 1, PP = 1, WP = 1, WPP = 2; };
template <> struct Mode<Q_F32> { typedef float T; static constexpr int QP = 3, PP = 3, WP = 3, WPP = 3; };

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
typedef __attribute__((ext_vector_type(4))) short s16x4_t;
typedef __attribute__((address_space(3))) s16x4_t* lds_s16x4_t;

__device__ __forceinline__ int tile_key(int rr) {  // row of the score tile -> key of the tile of 32
  const int a = rr >> 3, hh = (rr >> 2) & 1, b = rr & 3;
  return (a >> 1) * 16 + hh * 8 + (a & 1) * 4 + b;
}

__device__ __forceinline__ f32x16_t mfma_bf16(const u32x4_t& a, const u32x4_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ __forceinline__ f32x16_t mfma_f16(const u32x4_t& a, const u32x4_t& b, const f32x16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}

// 8 codes at a group's power of two, as bf16 / half
__device__ __forceinline__ u32x4_t codes_bf16(uint32_t w, float s) {
  u32x4_t r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3));
  return r;
}
__device__ __forceinline__ u32x4_t codes_f16(uint32_t w, float s) {
  u32x4_t r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 0));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 1));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 2));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, 3));
  return r;
}

// 8 codes and the product with queries in a mode's operand type
template <int QM>
__device__ __forceinline__ u32x4_t codes_for(uint32_t w, float s) { return QM == Q_F16 ? codes_f16(w, s) : codes_bf16(w, s); }
template <int QM>
__device__ __forceinline__ f32x16_t score_mfma(const u32x4_t& a, const u32x4_t& b, const f32x16_t& c) { return QM == Q_F16 ? mfma_f16(a, b, c) : mfma_bf16(a, b, c); }

// 8 values as P planes of bf16 whose sum is the value (P = 3: exactly, above the subnormals).  WIDE: finite values above bf16's largest, 3.39e38, too, which
// would round to infinity: the first plane is cut to it and the others take the rest (an infinity or a NaN is a NaN in the last plane then).
static constexpr float BF16_MAX = 3.38953139e38f;
template <int P, bool WIDE = false>
__device__ __forceinline__ void split8(const float (&x)[8], u32x4_t (&p)[P]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
    for (int k = 0; k < P; ++k) {
      const bool cut = WIDE && k == 0;
      bf16x2_t h;
      h[0] = (__bf16)(cut ? __builtin_amdgcn_fmed3f(a, -BF16_MAX, BF16_MAX) : a);
      h[1] = (__bf16)(cut ? __builtin_amdgcn_fmed3f(b, -BF16_MAX, BF16_MAX) : b);
      p[k][i] = __builtin_bit_cast(uint32_t, h);
      if (k + 1 < P) { a -= (float)h[0]; b -= (float)h[1]; }
    }
  }
}

// 8 values of a row of the caller's type as P planes; lo: offset of a second plane, for P = 2
template <int P>
__device__ __forceinline__ void load_planes(const bf16_t* p, int lo, u32x4_t (&r)[P]) {
  r[0] = *(const u32x4_t*)p;
  if (P > 1) r[P - 1] = *(const u32x4_t*)(p + lo);
}
template <int P>
__device__ __forceinline__ void load_planes(const float* p, int, u32x4_t (&r)[P]) {
  const f32x4_t a = ((const f32x4_t*)p)[0], b = ((const f32x4_t*)p)[1];
  const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
  split8<P, true>(x, r);
}

// ---- the batch as runs of key tiles ----
struct SeqTiles { int rows, row0, S, cached, tiles; };   // tiles: cached and the window's own
__device__ __forceinline__ SeqTiles seq_tiles(const Kv4Attn& a, int n) {
  SeqTiles s{0, 0, 0, 0, 0};
  if (n >= a.N) return s;
  const int rows = max(0, min(a.n_rows[n], a.T)), row0 = a.row0[n], S = a.kv.held(n);
  if (rows == 0 || row0 < 0 || row0 > a.rows - rows) return s;
  s.rows = rows; s.row0 = row0; s.S = S;
  s.cached = (S + 31) >> 5;
  s.tiles = s.cached + (a.k ? (rows + 31) >> 5 : 0);
  return s;
}
// Inclusive sums over the lanes by DPP moves (vector-ALU operands, no trips through LDS): inside the rows of 16 lanes, then lane 15 of
// rows 0 and 2 to the next row, then lane 31 to the upper half.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // row_bcast:15
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // row_bcast:31
  return v;
}
__device__ __forceinline__ int wave_sum(int v) { return __builtin_amdgcn_readlane(wave_scan(v), 63); }
__device__ __forceinline__ int splits_of_seq(const SeqTiles& s, int run) { return s.rows == 0 ? 0 : max(1, (s.tiles + run - 1) / run); }

// Tiles of a split.  The batch's tiles over the workgroups that are resident at once (target), less half a split a sequence, since the last split of each
// is a partial one and a workgroup over the target would start when the others are done; at most half as much again as an equal share,
// so that a long sequence among many short ones is still split.
__device__ __forceinline__ int run_of(const Kv4Attn& a, int total) {
  const long long wanted = 2ll * total * a.per_item, over = max(2ll * a.target - (long long)a.N * a.per_item, 4ll * a.target / 3);
  const int fits = a.room > 0 ? (total + a.room - 1) / a.room : 1 << 30;   // (the scratch holds them)
  return max(max(a.min_run, fits), (int)((wanted + over - 1) / over));
}

// The sequence and split of item w; false: there is none.  All lanes of the wavefront, the same answer in each.
struct Item { int n, z, splits, run; SeqTiles s; };
__device__ __forceinline__ bool find_item(const Kv4Attn& a, int w, int lane, Item& it) {
  SeqTiles s = seq_tiles(a, lane);
  int total = s.tiles;
  for (int n0 = 64; n0 < a.N; n0 += 64) total += seq_tiles(a, n0 + lane).tiles;
  it.run = run_of(a, wave_sum(total));
  int before = 0;
  for (int n0 = 0;;) {
    const int mine = splits_of_seq(s, it.run);
    const int incl = wave_scan(mine);
    const unsigned long long hit = __ballot(w - before < incl && w - before >= incl - mine);
    if (hit) {
      const int src = __ffsll((long long)hit) - 1;
      it.n = n0 + src;
      it.splits = __builtin_amdgcn_readlane(mine, src);
      it.z = w - before - (__builtin_amdgcn_readlane(incl, src) - it.splits);
      it.s.rows = __builtin_amdgcn_readlane(s.rows, src);
      it.s.row0 = __builtin_amdgcn_readlane(s.row0, src);
      it.s.S = __builtin_amdgcn_readlane(s.S, src);
      it.s.cached = __builtin_amdgcn_readlane(s.cached, src);
      it.s.tiles = __builtin_amdgcn_readlane(s.tiles, src);
      return true;
    }
    before += __builtin_amdgcn_readlane(incl, 63);
    n0 += 64;
    if (n0 >= a.N) return false;
    s = seq_tiles(a, n0 + lane);
  }
}

// Half a key's codes (dimensions half * D / 2 and on) and the scale bytes of its groups
template <int D>
struct HalfRow {
  static constexpr int W = D / 16;                    // words of 8 codes
  static constexpr int G = D >= 64 ? D / 64 : 1;      // groups
  uint32_t w[W];
  uint32_t scales;
  __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* sc, size_t at, int half) {
    const uint8_t* p = codes + at * (D / 2) + half * (D / 4);
    if (W == 2) { const uint2 x = *(const uint2*)p; w[0] = x.x; w[1] = x.y; }
    else
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const uint4 x = ((const uint4*)p)[i];
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
      }
    const uint8_t* q = sc + at * (D / 32) + (D >= 64 ? half * G : 0);
    scales = G == 4 ? *(const uint32_t*)q : G == 2 ? *(const uint16_t*)q : *q;
  }
  __device__ __forceinline__ float scale(int word) const { return __uint_as_float(((scales >> (8 * (word / 4))) & 0xffu) << 23); }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
    scales = 0x7f7f7f7fu;
  }
};

// Scores of one tile (accumulators of a lane: query row c; keys 16 (i / 8) + 8 h + i % 8) into softmax weights against the row's
// reference, which first follows the maximum if it has to.
template <int D>
struct RowState {
  float m, l;            // l: of this lane's keys only
  f32x16_t o[D / 32];
  __device__ __forceinline__ void init() {
    m = LOWEST;
    l = 0.f;
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  }
  // The sum of a tile's weights says whether one of them may exceed the bound (an overflow sums to infinity; a row with a NaN stays one).
  __device__ __forceinline__ void weights(const f32x16_t& s, float scale, float (&p)[16]) {
    float sum = 0.f;
    auto form = [&]() __attribute__((always_inline)) {
      sum = 0.f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -m));
        sum += p[i];
      }
    };
    form();
    if (__ballot(sum > MOST)) {
      float mx = fmaxf(fmaxf(s[0], s[1]), s[2]);
#pragma unroll
      for (int i = 3; i < 15; i += 2) mx = fmaxf(fmaxf(s[i], s[i + 1]), mx);
      mx = fmaxf(mx, s[15]) * scale;
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float to = fmaxf(m, mx - BELOW), f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= f;
#pragma unroll
      for (int t = 0; t < D / 32; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= f;
      form();
    }
    l += sum;
  }
};

// V in LDS: a row of D half values a key, rows 2 D + 64 bytes apart, bit 5 of a byte's place in its row flipped in keys with bit 3 set.  Then neither the
// 16-byte writes (8 lanes: keys k .. k + 3 and k + 8 .. k + 11) nor the transposing reads (32 lanes: 64 bytes of keys k .. k + 3) meet in a bank.
template <int D>
static constexpr int V_LD = 2 * D + 64;

// QT == 1: queries in registers, the next tile's codes requested a tile ahead.  QT == 2: the conversion of K and V serves two query tiles;
// their outputs take 128 registers, so the queries stay in LDS (one copy for the workgroup, in operand order) and the next codes are requested
// into the registers of the converted ones.
template <int D, int QM, int QT>
__global__ __launch_bounds__(64 * waves_of(D)) void kv4_attention_kernel(const Kv4Attn a, int layer) {
  typedef typename Mode<QM>::T T;
  constexpr int QP = Mode<QM>::QP, PP = Mode<QM>::PP, WP = Mode<QM>::WP, WPP = Mode<QM>::WPP, NW = waves_of(D), DT = D / 32, DS = D / 16;
  constexpr bool Q_LDS = QT > 1;
  extern __shared__ __attribute__((aligned(16))) uint8_t s_mem[];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
  const Kv4& kv = a.kv;
  // The workgroups of one run of keys lie a multiple of 8 apart: on one XCD, whose cache they share.  Groups of rows that fewer sequences have come last.
  const int groups = a.groups, per_group = gridDim.x / groups, qg = blockIdx.x / per_group, w = blockIdx.x % per_group, kvh = w % kv.H;
  Item it;
  if (!find_item(a, w / kv.H, lane, it)) return;
  const SeqTiles& sq = it.s;
  const int nq = sq.rows * a.grp, q0 = qg * QT * 32;
  if (q0 >= nq) return;
  const int t0 = it.z * it.run, t1 = min(sq.tiles, t0 + it.run), c1 = min(t1, sq.cached);
  const int tiles_q = min(QT, (nq - q0 + 31) / 32);

  // Cached keys: lane (c, h) takes half h of key tile_key(c) of a tile.
  const int kperm = tile_key(c);
  const int32_t* pt = kv.page_table + (size_t)it.n * kv.max_pages;
  const uint8_t *kc = kv.kc + layer * kv.layer_entries * (D / 2), *vc = kv.vc + layer * kv.layer_entries * (D / 2);
  const uint8_t *ks = kv.ks + layer * kv.layer_entries * (D / 32), *vs = kv.vs + layer * kv.layer_entries * (D / 32);
  auto place_of = [&](int tile) __attribute__((always_inline)) { return min(tile * 32 + kperm, sq.S - 1); };
  HalfRow<D> kn, vn;
  int page_next = 0;
  auto request_page = [&](int tile) __attribute__((always_inline)) { page_next = pt[kv.ps.div(place_of(tile))]; };
  auto entry_of = [&](int tile) __attribute__((always_inline)) {
    const int key = place_of(tile), p = kv.ps.div(key), page = max(0, min(page_next, kv.n_pages - 1));
    return kv.at(page, kvh, key - p * kv.ps.d);
  };
  auto request = [&](int tile) __attribute__((always_inline)) {
    const size_t at = entry_of(tile);
    kn.load(kc, ks, at, h);
    vn.load(vc, vs, at, h);
  };
  int tile = t0 + wave;
  if (tile < c1) request_page(tile);

  // ---- queries: lane (c, h) has row c's dimensions h D / 2 + 8 ds .. + 7 for step ds ----
  u32x4_t q[Q_LDS ? 1 : QT][Q_LDS ? 1 : DS][QP];
  u32x4_t* s_q = (u32x4_t*)(s_mem + NW * 32 * V_LD<D>);   // [QT][DS][QP][64]
  int row[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int qi = min(q0 + t * 32 + c, nq - 1), r = a.group.div(qi);
    row[t] = sq.row0 + r;
    const T* p = (const T*)a.q + row[t] * a.q_ld + (size_t)(kvh * a.grp + qi - r * a.grp) * D + h * (D / 2);
    if (Q_LDS) {
      for (int ds = wave; ds < DS; ds += NW) {
        u32x4_t x[QP];
        load_planes<QP>(p + 8 * ds, a.q_lo, x);
#pragma unroll
        for (int e = 0; e < QP; ++e) s_q[((t * DS + ds) * QP + e) * 64 + lane] = x[e];
      }
    } else
#pragma unroll
      for (int ds = 0; ds < DS; ++ds) load_planes<QP>(p + 8 * ds, a.q_lo, q[Q_LDS ? 0 : t][Q_LDS ? 0 : ds]);
  }
  auto query = [&](int t, int ds, int e) __attribute__((always_inline)) { return Q_LDS ? s_q[((t * DS + ds) * QP + e) * 64 + lane] : q[Q_LDS ? 0 : t][Q_LDS ? 0 : ds][e]; };
  RowState<D> st[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) st[t].init();

  uint8_t* s_v = s_mem + (size_t)wave * 32 * V_LD<D>;   // this wavefront's tile of V
  const int g16 = lane >> 4, i16 = lane & 15;
  // transposing read: 16 lanes take 16 dimensions of 4 keys; lanes 0-31 keys 0-7, lanes 32-63 keys 8-15 of a step
  const uint8_t* s_tr = s_v + (8 * h + (i16 >> 2)) * V_LD<D> + ((g16 & 1) ^ h) * 32 + (i16 & 3) * 8;
  auto v_operand = [&](int dt, int j) __attribute__((always_inline)) {
    const uint8_t* p = s_tr + 16 * j * V_LD<D> + dt * 64;
    const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)p), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t)(p + 4 * V_LD<D>));
    const uint2 u = __builtin_bit_cast(uint2, x), v = __builtin_bit_cast(uint2, y);
    return u32x4_t{u.x, u.y, v.x, v.y};
  };
  // this lane's half row of V: the 16 bytes of word i
  const int flip = (kperm >> 3) & 1;
  uint8_t* s_vrow = s_v + kperm * V_LD<D> + (D == 32 ? (h ^ flip) * 32 : h * D);
  auto v_word = [&](int i) __attribute__((always_inline)) -> u32x4_t& { return *(u32x4_t*)(s_vrow + 16 * i + (D == 32 ? 0 : i & 2 ? -32 * flip : 32 * flip)); };
  auto lds_written = []() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };
  auto lds_read = []() __attribute__((always_inline)) {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  };

  // One tile of cached keys from k, v.  after_v(), after_k() run once V and K are converted.  The matrix instructions go ahead of the other
  // wavefront's vector work (s_setprio; 2 % of the verification windows).  Queries in LDS: the first half of a tile's operands is
  // requested before V is converted, every further one when its predecessor's registers are free.
  auto cached_tile = [&](int tile, const HalfRow<D>& k, HalfRow<D>& v, auto after_v, auto after_k) __attribute__((always_inline)) {
    constexpr int AHEAD = Q_LDS ? (DS < 4 ? DS : 4) : 1;
    u32x4_t qa[AHEAD][QT][QP];
    if (Q_LDS) {
#pragma unroll
      for (int ds = 0; ds < AHEAD; ++ds)
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int p = 0; p < QP; ++p) qa[ds][t][p] = query(t, ds, p);
      __builtin_amdgcn_sched_barrier(0);
    }
    const bool part = tile * 32 + 32 > sq.S;
    if (part && tile * 32 + kperm >= sq.S) v.clear();   // (what lies behind the entries may be anything)
#pragma unroll
    for (int i = 0; i < DS; ++i) v_word(i) = QM == Q_F32 ? codes_bf16(v.w[i], v.scale(i)) : codes_f16(v.w[i], v.scale(i));
    lds_written();
    after_v();
    __builtin_amdgcn_s_setprio(1);
    f32x16_t s[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      const u32x4_t kf = codes_for<QM>(k.w[ds], k.scale(ds));
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int p = 0; p < QP; ++p) {
          s[t] = score_mfma<QM>(kf, Q_LDS ? qa[ds % AHEAD][t][p] : query(t, ds, p), s[t]);
          if (Q_LDS && ds + AHEAD < DS) qa[ds % AHEAD][t][p] = query(t, ds + AHEAD, p);
        }
      if (Q_LDS) __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_setprio(0);
    after_k();
    u32x4_t pw[QT][2][PP];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      if (part) {
        const int left = sq.S - tile * 32 - 8 * h;
#pragma unroll
        for (int i = 0; i < 16; ++i) s[t][i] = 16 * (i >> 3) + (i & 7) < left ? s[t][i] : -INFINITY;
      }
      float p[16];
      st[t].weights(s[t], a.scale_log2e, p);
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if constexpr (QM == Q_F32) {   // (half planes would end at 2^-24: 2^-31 of the largest weight, and their low bits before that)
          const float x[8] = {p[8 * j], p[8 * j + 1], p[8 * j + 2], p[8 * j + 3], p[8 * j + 4], p[8 * j + 5], p[8 * j + 6], p[8 * j + 7]};
          split8<PP>(x, pw[t][j]);
        } else
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f16x2_t hv;
            hv[0] = (_Float16)p[8 * j + 2 * i];
            hv[1] = (_Float16)p[8 * j + 2 * i + 1];
            pw[t][j][0][i] = __builtin_bit_cast(uint32_t, hv);
          }
    }
    __builtin_amdgcn_s_setprio(1);
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const u32x4_t vf = v_operand(dt, j);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int e = 0; e < PP; ++e) st[t].o[dt] = QM == Q_F32 ? mfma_bf16(vf, pw[t][j][e], st[t].o[dt]) : mfma_f16(vf, pw[t][j][e], st[t].o[dt]);
      }
    __builtin_amdgcn_s_setprio(0);
    lds_read();
  };
  auto first = [&]() __attribute__((always_inline)) {
    if (tile < c1) {
      request(tile);
      if (tile + NW < c1) request_page(tile + NW);
    }
  };
  constexpr bool EARLY = QT == 1 && QM != Q_F32;   // codes on their way while the window is computed: 18 registers that the others have not
  if (EARLY) first();
  if (Q_LDS) __syncthreads();

  // ---- the window's own keys: V plane by plane through LDS.  The last wavefronts first: they have the fewer cached tiles ----
  for (int tile = max(t0, sq.cached) + NW - 1 - wave; tile < t1; tile += NW) {
    const int base = (tile - sq.cached) * 32, key = base + kperm;
    const bool there = key < sq.rows;
    const int64_t at = (int64_t)(sq.row0 + min(key, sq.rows - 1)) * a.kv_ld + kvh * D + h * (D / 2);
    bool bad = false;   // a value of this key that is not finite: the rows that see it become NaN, the others must not
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      u32x4_t v[WP];
      load_planes<WP>((const T*)a.v + at + 8 * ds, 0, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) bad |= (v[WP - 1][i] & 0x7f80u) == 0x7f80u || (v[WP - 1][i] & 0x7f800000u) == 0x7f800000u;
      v_word(ds) = there ? v[0] : u32x4_t{0, 0, 0, 0};
    }
    bad |= (bool)__shfl_xor((int)bad, 32, 64);
    const unsigned long long bad_at = __ballot(there && bad);   // bit c: key tile_key(c)
    if (bad_at) {
#pragma unroll
      for (int ds = 0; ds < DS; ++ds)
        if (bad) v_word(ds) = u32x4_t{0, 0, 0, 0};
    }
    lds_written();
    f32x16_t s[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[t][i] = 0.f;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      u32x4_t kf[WP];
      load_planes<WP>((const T*)a.k + at + 8 * ds, 0, kf);
#pragma unroll
      for (int t = 0; t < QT; ++t)
#pragma unroll
        for (int e = 0; e < WP; ++e)
#pragma unroll
          for (int p = 0; p < QP; ++p)
            if (e + p < (QP > WP ? QP : WP)) s[t] = score_mfma<QM>(kf[e], query(t, ds, p), s[t]);
    }
    u32x4_t pw[QT][2][WPP];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      const int lo = a.lo ? a.lo[row[t]] : sq.row0, hi = a.hi ? a.hi[row[t]] : row[t] + 1;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int rr = 8 * (i >> 2) + 4 * h + (i & 3), k = base + tile_key(rr), r = sq.row0 + k;
        const bool seen = k < sq.rows && ((r >= lo && r < hi) || r == row[t]);
        s[t][i] = !seen ? -INFINITY : (bad_at >> rr) & 1 ? NAN : s[t][i];
      }
      float p[16];
      st[t].weights(s[t], a.scale_log2e, p);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float x[8] = {p[8 * j], p[8 * j + 1], p[8 * j + 2], p[8 * j + 3], p[8 * j + 4], p[8 * j + 5], p[8 * j + 6], p[8 * j + 7]};
        split8<WPP>(x, pw[t][j]);
      }
    }
#pragma unroll
    for (int e = 0; e < WP; ++e) {
      if (e > 0) {
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) {
          u32x4_t v[WP];
          load_planes<WP>((const T*)a.v + at + 8 * ds, 0, v);
          v_word(ds) = there && !bad ? v[e] : u32x4_t{0, 0, 0, 0};
        }
        lds_written();
      }
#pragma unroll
      for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4_t vo = v_operand(dt, j);
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int p = 0; p < WPP; ++p)
              if (e + p < WPP) st[t].o[dt] = mfma_bf16(vo, pw[t][j][p], st[t].o[dt]);
        }
      lds_read();
    }
  }

  // ---- cached keys ----
  if (!EARLY) first();
  if (Q_LDS) {
    size_t at = 0;
    for (; tile < c1; tile += NW)
      cached_tile(tile, kn, vn, [&]() __attribute__((always_inline)) {
        if (tile + NW < c1) {
          at = entry_of(tile + NW);
          vn.load(vc, vs, at, h);
          if (tile + 2 * NW < c1) request_page(tile + 2 * NW);
        }
      }, [&]() __attribute__((always_inline)) {
        if (tile + NW < c1) kn.load(kc, ks, at, h);
      });
  } else {
    for (; tile < c1; tile += NW) {
      const HalfRow<D> k = kn;
      HalfRow<D> v = vn;
      if (tile + NW < c1) {
        request(tile + NW);
        if (tile + 2 * NW < c1) request_page(tile + 2 * NW);
      }
      cached_tile(tile, k, v, []() {}, []() {});
    }
  }

  // ---- the wavefronts' states into one: each deposits its own, every thread adds up four outputs of a row, in the order of the wavefronts ----
  constexpr int SLOT = 32 * D + 64;   // floats: output in the accumulators' order, maxima, sums
  float* s_st = (float*)s_mem;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (t >= tiles_q) break;
    st[t].l += __shfl_xor(st[t].l, 32, 64);
    __syncthreads();
    float* p = s_st + (size_t)wave * SLOT;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        ((float4*)p)[(dt * 4 + i) * 64 + lane] = make_float4(st[t].o[dt][4 * i], st[t].o[dt][4 * i + 1], st[t].o[dt][4 * i + 2], st[t].o[dt][4 * i + 3]);
    if (h == 0) { p[32 * D + c] = st[t].m; p[32 * D + 32 + c] = st[t].l; }
    __syncthreads();
    const int qi = q0 + t * 32 + c, head = kvh * a.grp + qi - a.group.div(min(qi, nq - 1)) * a.grp;
    float m = s_st[32 * D + c], f[NW], l = 0.f;
#pragma unroll
    for (int k = 1; k < NW; ++k) m = fmaxf(m, s_st[k * SLOT + 32 * D + c]);
#pragma unroll
    for (int k = 0; k < NW; ++k) {
      f[k] = __builtin_amdgcn_exp2f(s_st[k * SLOT + 32 * D + c] - m);
      l += f[k] * s_st[k * SLOT + 32 * D + 32 + c];
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    const size_t at = ((size_t)w * groups + qg) * QT + t;
#pragma unroll
    for (int g = wave; g < 4 * DT; g += NW) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < NW; ++k) {
        const float4 v = ((const float4*)(s_st + k * SLOT))[g * 64 + lane];
        o.x += f[k] * v.x; o.y += f[k] * v.y; o.z += f[k] * v.z; o.w += f[k] * v.w;
      }
      if (qi >= nq) continue;
      if (it.splits > 1) {
        ((float4*)(a.part_o + at * 32 * D))[g * 64 + lane] = o;
      } else {
        const int d = head * D + (g >> 2) * 32 + 8 * (g & 3) + 4 * h;
        if (QM == Q_F32) *(float4*)((float*)a.out + row[t] * a.o_ld + d) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
        else act_put4((bf16_t*)a.out, a.o_lo, row[t], d, (int)a.o_ld, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
      }
    }
    if (wave == 0 && h == 0 && qi < nq) {
      if (it.splits > 1) {
        a.part_ml[at * 64 + c] = m;
        a.part_ml[at * 64 + 32 + c] = l;
        // the first split says where the sequence's are
        if (t == 0 && qg == 0 && kvh == 0 && it.z == 0 && c == 0) a.part_of[it.n] = make_int2(w / kv.H, it.splits);
      } else if (a.lse) a.lse[(size_t)row[t] * a.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
    }
  }
}

// The splits of a (sequence, KV head, query tile) into its rows, in the order of the splits; a workgroup has 32 dimensions, a thread four of a
// row: 4 to 5 us, a launch and two dependent loads.  Sequences of one split are done; Z: splits of a sequence, at most `most`.
template <int D, int QM>
__global__ __launch_bounds__(256) void kv4_merge_kernel(const Kv4Attn a, int tiles, int per_wg) {
  const Kv4& kv = a.kv;
  const int tid = threadIdx.x, c = tid & 31, h = (tid >> 5) & 1, g = tid >> 6;
  const int dt = blockIdx.x % (D / 32), b = blockIdx.x / (D / 32), qt = b % tiles, kvh = (b / tiles) % kv.H, n = b / tiles / kv.H;
  const int2 of = a.part_of[n];     // (of a sequence with one split, or none: what the scratch held)
  const SeqTiles sq = seq_tiles(a, n);
  const int nq = sq.rows * a.grp, qi = qt * 32 + c;
  if (qt * 32 >= nq || sq.tiles <= a.min_run) return;
  int total = 0;
  for (int n0 = tid & 63; n0 < a.N; n0 += 64) total += seq_tiles(a, n0).tiles;
  if (sq.tiles <= run_of(a, wave_sum(total))) return;
  if (qi >= nq) return;
  const int Z = of.y, groups = a.groups;
  const size_t step = (size_t)kv.H * groups * per_wg, at0 = (((size_t)of.x * kv.H + kvh) * groups + qt / per_wg) * per_wg + qt % per_wg;
  const float* ml = a.part_ml + at0 * 64 + c;
  const float4* po = (const float4*)(a.part_o + at0 * 32 * D) + (dt * 4 + g) * 64 + 32 * h + c;
  float m = LOWEST, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  constexpr int AHEAD = 8;   // splits in flight
  for (int z0 = 0; z0 < Z; z0 += AHEAD) {
    float mz[AHEAD], lz[AHEAD];
    float4 v[AHEAD];
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const int z = min(z0 + k, Z - 1);
      mz[k] = ml[z * step * 64];
      lz[k] = ml[z * step * 64 + 32];
      v[k] = po[z * step * 8 * D];
    }
    float to = m;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) to = fmaxf(to, mz[k]);
    const float f0 = __builtin_amdgcn_exp2f(m - to);
    l *= f0; o.x *= f0; o.y *= f0; o.z *= f0; o.w *= f0;
    m = to;
#pragma unroll
    for (int k = 0; k < AHEAD; ++k) {
      const float f = z0 + k < Z ? __builtin_amdgcn_exp2f(mz[k] - m) : 0.f;
      if (z0 + k < Z) { l += f * lz[k]; o.x += f * v[k].x; o.y += f * v[k].y; o.z += f * v[k].z; o.w += f * v[k].w; }
    }
  }
  const int r = a.group.div(qi), row = sq.row0 + r, head = kvh * a.grp + qi - r * a.grp, d = head * D + dt * 32 + 8 * g + 4 * h;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  if (QM == Q_F32) *(float4*)((float*)a.out + row * a.o_ld + d) = make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  else act_put4((bf16_t*)a.out, a.o_lo, row, d, (int)a.o_ld, o.x * inv, o.y * inv, o.z * inv, o.w * inv);
  if (a.lse && dt == 0 && g == 0 && h == 0) a.lse[(size_t)row * a.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * LN2;
}

// ---------------------------------------------------------------------------------------------
// kv4_weigh_kernel: the weights that a sequence's rows give its entries.  A workgroup has one sequence, one KV head and a run of key tiles, a
// wavefront every fourth pair of them.  Scores are computed as S = Q K^T, so that a lane owns a key and the sum over rows stays in it; the queries
// lie in LDS in operand order, up to QC tiles of 32 rows at a time, each read for two tiles of keys.  The sums of a pair over these rows are
// added to the mass by one lane a key, tile of rows after tile of rows: a fixed order.
// 16 x 32 rows x 32 heads on 8 over 8192 entries of 128: 50 us (34 GFLOP, 690 TFLOP/s).  By its counters the vector instructions issue in 69 % of that
// time (an exponential takes 16 cycles, with a multiply-add and an add 24 for 64 scores) and the matrix cores are busy in 39 %: partly beside each other, on three
// wavefronts a SIMD, each of which waits for 47 % of its life.  A pass with two workgroups a compute unit instead of three: 57 us for 51.
// ---------------------------------------------------------------------------------------------
static constexpr int WEIGH_WAVES = 4;
template <int D, int QM>
static constexpr int QC = D * Mode<QM>::QP <= 384 ? 4 : 2;
template <int D, int QM>
static constexpr size_t weigh_lds() { return (size_t)QC<D, QM> * (32 * D * 2 * Mode<QM>::QP + 33 * sizeof(float)); }

// The weights that a window's rows give each other, into row_mass: a workgroup has one sequence, one KV head and 32 keys, a wavefront every fourth tile of
// 32 query rows that sees one of them (of a causal window half the tiles).  S = Q K^T as below, keys and queries from memory; the wavefronts' sums are added up
// in their order.  In one launch with the cached entries: a layer of 16 x 32 rows behind 8192 takes 54 us, 53 without the window's 128 workgroups.
template <int D, int QM>
__device__ __forceinline__ void weigh_window(const Kv4Attn& a, int block, uint8_t* s_mem) {
  typedef typename Mode<QM>::T T;
  constexpr int QP = Mode<QM>::QP, WP = Mode<QM>::WP, NW = WEIGH_WAVES, DS = D / 16;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
  const int kvh = block % a.kv.H, tiles = (a.T + 31) >> 5, key0 = block / a.kv.H % tiles * 32;
  const SeqTiles sq = seq_tiles(a, block / a.kv.H / tiles);
  if (key0 >= sq.rows) return;
  float* s_ref = (float*)s_mem + wave * 32;                              // [NW][32] minus a row's lse to base 2; -inf: the row adds nothing
  int4* s_row = (int4*)(s_mem + NW * 32 * sizeof(float)) + wave * 32;    // [NW][32] the row and the rows that it sees
  float* s_sum = (float*)(s_mem + NW * 32 * (sizeof(float) + sizeof(int4)));   // [NW][32]
  const int key = sq.row0 + min(key0 + c, sq.rows - 1), k0 = sq.row0 + key0, k1 = sq.row0 + min(key0 + 32, sq.rows), nq = sq.rows * a.grp;
  float sum = 0.f;
  for (int q0 = wave * 32; q0 < nq; q0 += NW * 32) {
    const int qi = min(q0 + c, nq - 1), r = a.group.div(qi), row = sq.row0 + r, head = kvh * a.grp + qi - r * a.grp;
    const int lo = a.lo[row], hi = a.hi[row];
    if (!__ballot((lo < k1 && hi > k0) || (row >= k0 && row < k1))) continue;
    const float lse = a.lse[(size_t)row * a.Hq + head];
    if (h == 0) {
      s_ref[c] = q0 + c >= nq || lse == -INFINITY ? -INFINITY : -lse * (1.f / LN2);
      s_row[c] = make_int4(row, lo, hi, 0);
    }
    f32x16_t s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int ds = 0; ds < DS; ++ds) {
      u32x4_t q[QP], k[WP];
      load_planes<QP>((const T*)a.q + row * a.q_ld + (size_t)head * D + h * (D / 2) + 8 * ds, a.q_lo, q);
      load_planes<WP>((const T*)a.window_k + key * a.kv_ld + (size_t)kvh * D + h * (D / 2) + 8 * ds, 0, k);
#pragma unroll
      for (int e = 0; e < WP; ++e)
#pragma unroll
        for (int p = 0; p < QP; ++p)
          if (e + p < (QP > WP ? QP : WP)) s = score_mfma<QM>(q[p], k[e], s);
    }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int rr = 8 * (i >> 2) + 4 * h + (i & 3);
      const float ref = s_ref[rr];
      const int4 see = s_row[rr];
      const bool seen = (key >= see.y && key < see.z) || key == see.x;
      sum += seen && ref != -INFINITY ? __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], a.scale_log2e, ref)) : 0.f;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
  sum += __shfl_xor(sum, 32, 64);
  if (h == 0) s_sum[wave * 32 + c] = sum;
  __syncthreads();
  if (wave == 0 && h == 0 && key0 + c < sq.rows) {
#pragma unroll
    for (int w = 1; w < NW; ++w) sum += s_sum[w * 32 + c];
    a.row_mass[(size_t)key * a.kv.H + kvh] = sum;
  }
}

// WINDOW: the window's own rows too, by the workgroups from cached_wgs on
template <int D, int QM, bool WINDOW>
__global__ __launch_bounds__(64 * WEIGH_WAVES, D <= 128 ? 3 : 2) void kv4_weigh_kernel(const Kv4Attn a, int layer) {
  typedef typename Mode<QM>::T T;
  constexpr int QP = Mode<QM>::QP, NW = WEIGH_WAVES, DS = D / 16, C = QC<D, QM>;
  extern __shared__ __attribute__((aligned(16))) uint8_t s_mem[];
  if (WINDOW && (int)blockIdx.x >= a.cached_wgs) {
    weigh_window<D, QM>(a, blockIdx.x - a.cached_wgs, s_mem);
    return;
  }
  u32x4_t* s_q = (u32x4_t*)s_mem;                       // [C][DS][QP][64]
  float* s_ref = (float*)(s_q + C * DS * QP * 64);      // [C][32] minus a row's lse to base 2; -inf: the row adds nothing
  int* s_some = (int*)(s_ref + C * 32);                 // [C] whether there is such a row
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
  const Kv4& kv = a.kv;
  const int kvh = blockIdx.x % kv.H;
  Item it;
  if (!find_item(a, blockIdx.x / kv.H, lane, it)) return;
  const SeqTiles& sq = it.s;
  const int nq = sq.rows * a.grp, t0 = it.z * it.run, t1 = min(sq.cached, t0 + it.run);
  const int32_t* pt = kv.page_table + (size_t)it.n * kv.max_pages;
  const uint8_t *kc = kv.kc + layer * kv.layer_entries * (D / 2), *ks = kv.ks + layer * kv.layer_entries * (D / 32);
  HalfRow<D> next[2];
  auto entry = [&](int key, int& page) __attribute__((always_inline)) {
    const int k = min(key, sq.S - 1), p = kv.ps.div(k);
    page = pt[p];
    return kv.at(max(0, min(page, kv.n_pages - 1)), kvh, k - p * kv.ps.d);
  };
  auto request = [&](int tile) __attribute__((always_inline)) {
    int page;
#pragma unroll
    for (int x = 0; x < 2; ++x) next[x].load(kc, ks, entry((tile + x) * 32 + c, page), h);   // (a tile behind the last: entries that are there)
  };
  for (int q0 = 0; q0 < nq; q0 += 32 * C) {
    const int tiles = min(C, (nq - q0 + 31) / 32);
    if (q0) __syncthreads();
    for (int i = wave; i < tiles * DS; i += NW) {
      const int t = i / DS, ds = i % DS, qi = min(q0 + t * 32 + c, nq - 1), r = a.group.div(qi), head = kvh * a.grp + qi - r * a.grp;
      u32x4_t x[QP];
      load_planes<QP>((const T*)a.q + (sq.row0 + r) * a.q_ld + (size_t)head * D + h * (D / 2) + 8 * ds, a.q_lo, x);
#pragma unroll
      for (int e = 0; e < QP; ++e) s_q[(i * QP + e) * 64 + lane] = x[e];
      if (ds == 0) {
        const float lse = a.lse[(size_t)(sq.row0 + r) * a.Hq + head];
        const float ref = q0 + t * 32 + c >= nq || lse == -INFINITY ? -INFINITY : -lse * (1.f / LN2);
        if (h == 0) s_ref[t * 32 + c] = ref;
        const bool some = __ballot(ref == -INFINITY) != 0;
        if (lane == 0) s_some[t] = some;
      }
    }
    int tile = t0 + 2 * wave;
    if (tile < t1) request(tile);
    __syncthreads();
    for (; tile < t1; tile += 2 * NW) {
      u32x4_t kf[2][DS];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int ds = 0; ds < DS; ++ds) kf[x][ds] = codes_for<QM>(next[x].w[ds], next[x].scale(ds));
      if (tile + 2 * NW < t1) request(tile + 2 * NW);
      float sum[2] = {0.f, 0.f};
      for (int t = 0; t < tiles; ++t) {
        f32x16_t s[2];
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[x][i] = 0.f;
#pragma unroll
        for (int ds = 0; ds < DS; ++ds)
#pragma unroll
          for (int e = 0; e < QP; ++e) {
            const u32x4_t qf = s_q[((t * DS + ds) * QP + e) * 64 + lane];
#pragma unroll
            for (int x = 0; x < 2; ++x) s[x] = score_mfma<QM>(qf, kf[x][ds], s[x]);
          }
        float ref[16];   // of rows 8 (i / 4) + 4 h + i % 4
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float4 v = *(const float4*)(s_ref + t * 32 + 8 * i + 4 * h);
          ref[4 * i] = v.x; ref[4 * i + 1] = v.y; ref[4 * i + 2] = v.z; ref[4 * i + 3] = v.w;
        }
        const bool some = __builtin_amdgcn_readfirstlane(s_some[t]);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          float p[16];
#pragma unroll
          for (int i = 0; i < 16; ++i) p[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][i], a.scale_log2e, ref[i]));
          if (some)   // (a key that reads as NaN has no weight from rows that add nothing)
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = ref[i] == -INFINITY ? 0.f : p[i];
#pragma unroll
          for (int i = 0; i < 16; ++i) sum[x] += p[i];
        }
      }
#pragma unroll
      for (int x = 0; x < 2; ++x) sum[x] += __shfl_xor(sum[x], 32, 64);
      // lane (c, h): key c of the pair's tile h
      const int key = (tile + h) * 32 + c;
      int page;
      const size_t at = layer * kv.layer_entries + entry(key, page);
      if (tile + h < t1 && key < sq.S && page >= 0 && page < kv.n_pages) kv.mass[at] += h ? sum[1] : sum[0];
    }
  }
}

// ---------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------
static constexpr int WEIGH_TARGET = 768, WEIGH_MIN_RUN = 16;   // three workgroups a compute unit (four wavefronts of up to 168 registers); two pairs of tiles a wavefront
static constexpr int TARGET = 256;   // workgroups that are resident at once: one a compute unit (eight wavefronts of up to 256 registers)

// Query tiles per workgroup: two share the conversion of K and V; one where there is no second, and where two would not leave registers (outputs of
// heads of 256, planes of queries).  A pass of 16 x 32 rows x 4 heads over 8192 entries: 130 us by one, 104 by two.
static int tiles_per_wg(int D, int mode, int q_tiles) { return D <= 128 && (mode == Q_BF16 || mode == Q_F16) && q_tiles >= 2 ? 2 : 1; }

struct AttnShape { int q_tiles, per_wg, groups, per_item, items, most, room; };
// Slots of partial results that the scratch holds: those of four times the resident workgroups (a launch for fewer rows than T allows has more
// splits than one for T rows), and of one run a sequence, KV head and query tile, with what rounding up adds.  Grows with N and T.
static size_t slots_of(const Kv4& kv, int N, int q_tiles) { return 4 * TARGET + ((size_t)(N + 1) * kv.H + 8) * (q_tiles + 1); }
static AttnShape shape_of(const Kv4& kv, int mode, int N, int T, int expect, int Hq, bool window) {
  AttnShape s;
  s.q_tiles = (T * (Hq / kv.H) + 31) / 32;
  s.per_wg = tiles_per_wg(kv.D, mode, s.q_tiles);
  s.groups = (s.q_tiles + s.per_wg - 1) / s.per_wg;
  const int expected = (std::min(expect, T) * (Hq / kv.H) + 31) / 32;
  s.per_item = kv.H * ((expected + s.per_wg - 1) / s.per_wg);
  // runs of the batch: at most the target, and one more a sequence, what the scratch holds; a sequence has no more than its pages hold
  s.room = (int)((slots_of(kv, N, s.q_tiles) / (s.groups * s.per_wg) - 8) / kv.H) - N;
  s.most = std::max(1, ((kv.cap + 31) / 32 + (window ? (T + 31) / 32 : 0) + min_run_of(kv.D) - 1) / min_run_of(kv.D));
  s.items = (int)std::min<long long>((long long)N * s.most, std::max(0, std::min((TARGET + s.per_item - 1) / s.per_item, s.room)) + (long long)N);
  return s;
}

size_t kv4_attention_bytes(const Kv4& kv, int N, int T, int Hq) {
  const AttnShape s = shape_of(kv, Q_BF16, N, T, T, Hq, true);
  if (s.most < 2) return 0;
  return ((slots_of(kv, N, s.q_tiles) * (32 * kv.D + 64) + 2 * N) * sizeof(float) + 255) & ~(size_t)255;
}

// Tiles of V and the queries, and after them the wavefronts' states.
template <int D, int QT>
static constexpr size_t attn_lds() {
  return std::max((size_t)waves_of(D) * 32 * V_LD<D> + (QT > 1 ? (size_t)QT * 32 * D * 2 : 0), (size_t)waves_of(D) * (32 * D + 64) * sizeof(float));
}

template <int D, int QM, int QT>
static void launch_attn(hipStream_t st, const Kv4Attn& a, int layer, const AttnShape& s) {
  const int wgs = (a.items * a.kv.H + 7) / 8 * 8 * s.groups;
  S2D2_LAUNCH((kv4_attention_kernel<D, QM, QT>), dim3(wgs), dim3(64 * waves_of(D)), (attn_lds<D, QT>()), st, a, layer);
}

template <typename F>
static void by_head_dim(int D, const F& f) {
  if (D == 32) f(std::integral_constant<int, 32>{});
  else if (D == 64) f(std::integral_constant<int, 64>{});
  else if (D == 128) f(std::integral_constant<int, 128>{});
  else f(std::integral_constant<int, 256>{});
}

bool launch_kv4_attention(hipStream_t st, int mode, Kv4Attn& a, int layer, void* scratch) {
  const AttnShape s = shape_of(a.kv, mode, a.N, a.T, a.expect, a.Hq, a.k != nullptr);
  a.items = s.items;
  a.per_item = s.per_item;
  a.groups = s.groups;
  a.room = s.room;
  a.target = TARGET;
  a.min_run = min_run_of(a.kv.D);
  a.q_tiles = s.q_tiles;
  a.per_wg = s.per_wg;
  const size_t slots = (size_t)((s.items * a.kv.H + 7) / 8 * 8) * s.groups * s.per_wg;
  a.part_o = (float*)scratch;
  a.part_ml = a.part_o + slots * 32 * a.kv.D;
  a.part_of = (int2*)(a.part_ml + slots * 64);
  by_head_dim(a.kv.D, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    constexpr int D2 = D <= 128 ? D : 128;
    if (mode == Q_F32) launch_attn<D, Q_F32, 1>(st, a, layer, s);
    else if (mode == Q_BF16X2) launch_attn<D, Q_BF16X2, 1>(st, a, layer, s);
    else if (mode == Q_F16 && s.per_wg == 2) launch_attn<D2, Q_F16, 2>(st, a, layer, s);
    else if (mode == Q_F16) launch_attn<D, Q_F16, 1>(st, a, layer, s);
    else if (s.per_wg == 2) launch_attn<D2, Q_BF16, 2>(st, a, layer, s);
    else launch_attn<D, Q_BF16, 1>(st, a, layer, s);
  });
  return s.most > 1;
}

void launch_kv4_merge(hipStream_t st, int mode, const Kv4Attn& a) {
  by_head_dim(a.kv.D, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const dim3 grid(a.N * a.kv.H * a.q_tiles * (D / 32)), wg(256);
    if (mode == Q_F32) S2D2_LAUNCH((kv4_merge_kernel<D, Q_F32>), grid, wg, 0, st, a, a.q_tiles, a.per_wg);
    else S2D2_LAUNCH((kv4_merge_kernel<D, Q_BF16>), grid, wg, 0, st, a, a.q_tiles, a.per_wg);
  });
}

void launch_kv4_weigh(hipStream_t st, int mode, Kv4Attn& a, int layer) {
  a.window_k = a.row_mass ? a.k : nullptr;
  a.k = a.v = nullptr;   // (the runs are those of the cached entries)
  a.per_item = a.kv.H;
  a.room = 1 << 30;
  a.target = WEIGH_TARGET;
  a.min_run = WEIGH_MIN_RUN;
  const int most = std::max(1, ((a.kv.cap + 31) / 32 + WEIGH_MIN_RUN - 1) / WEIGH_MIN_RUN);
  a.items = (int)std::min<long long>((long long)a.N * most, (WEIGH_TARGET + a.kv.H - 1) / a.kv.H + (long long)a.N);
  a.cached_wgs = a.items * a.kv.H;
  by_head_dim(a.kv.D, [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    const dim3 wg(64 * WEIGH_WAVES);
    if (a.row_mass) {   // (forwards)
      const dim3 grid(a.cached_wgs + a.N * a.kv.H * ((a.T + 31) / 32));
      if (mode == Q_F32) S2D2_LAUNCH((kv4_weigh_kernel<D, Q_F32, true>), grid, wg, (weigh_lds<D, Q_F32>()), st, a, layer);
      else if (mode == Q_BF16X2) S2D2_LAUNCH((kv4_weigh_kernel<D, Q_BF16X2, true>), grid, wg, (weigh_lds<D, Q_BF16X2>()), st, a, layer);
      else if (mode == Q_F16) S2D2_LAUNCH((kv4_weigh_kernel<D, Q_F16, true>), grid, wg, (weigh_lds<D, Q_F16>()), st, a, layer);
      else S2D2_LAUNCH((kv4_weigh_kernel<D, Q_BF16, true>), grid, wg, (weigh_lds<D, Q_BF16>()), st, a, layer);
    } else {
      const dim3 grid(a.cached_wgs);
      if (mode == Q_F32) S2D2_LAUNCH((kv4_weigh_kernel<D, Q_F32, false>), grid, wg, (weigh_lds<D, Q_F32>()), st, a, layer);
      else S2D2_LAUNCH((kv4_weigh_kernel<D, Q_BF16, false>), grid, wg, (weigh_lds<D, Q_BF16>()), st, a, layer);
    }
  });
}

// LDS above 64 KB has to be asked for, once a device.
int kv4_attention_init() {
  hipError_t e = hipSuccess;
  auto limit = [&](const void* f, size_t bytes) { if (e == hipSuccess) e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes); };
  for (int D : {32, 64, 128, 256})
    by_head_dim(D, [&](auto dim) {
      constexpr int D = decltype(dim)::value;
      limit((const void*)kv4_attention_kernel<D, Q_BF16, 1>, attn_lds<D, 1>());
      limit((const void*)kv4_attention_kernel<D, Q_BF16X2, 1>, attn_lds<D, 1>());
      limit((const void*)kv4_attention_kernel<D, Q_F32, 1>, attn_lds<D, 1>());
      limit((const void*)kv4_attention_kernel<D, Q_F16, 1>, attn_lds<D, 1>());
      limit((const void*)kv4_weigh_kernel<D, Q_BF16, false>, weigh_lds<D, Q_BF16>());
      limit((const void*)kv4_weigh_kernel<D, Q_F32, false>, weigh_lds<D, Q_F32>());
      limit((const void*)kv4_weigh_kernel<D, Q_BF16, true>, weigh_lds<D, Q_BF16>());
      limit((const void*)kv4_weigh_kernel<D, Q_BF16X2, true>, weigh_lds<D, Q_BF16X2>());
      limit((const void*)kv4_weigh_kernel<D, Q_F16, true>, weigh_lds<D, Q_F16>());
      limit((const void*)kv4_weigh_kernel<D, Q_F32, true>, weigh_lds<D, Q_F32>());
      constexpr int D2 = D <= 128 ? D : 128;
      limit((const void*)kv4_attention_kernel<D2, Q_BF16, 2>, attn_lds<D2, 2>());
      limit((const void*)kv4_attention_kernel<D2, Q_F16, 2>, attn_lds<D2, 2>());
    });
  return e == hipSuccess ? 0 : -1;
}

}  // namespace s2d2
