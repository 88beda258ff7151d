// Causal attention of new tokens over a paged cache, and the attention weight
// each cached key received.
//
//   z_n = alpha <q, K_n>, n <= lens + i;  out = sum w_n V_n / sum w_n,
//   w_n = exp(z_n - max z);  mass_n (+)= sum over rows of w_n / sum w.
//
// The g query heads of a KV head and a sequence's new tokens are rows of one
// product with that head's keys (row i * g + h), so a key is read once for all
// of them.  Two kernels share the work by the number of rows:
//
//   few rows (new * g <= 16, single and drafted tokens): bound by HBM.  Every
//   byte goes from memory straight into a matrix operand: a wave owns units of
//   32 keys, S^T = K q^T in 16x16x32 products with the keys as rows; the
//   accumulators are then the B operand of O^T = V^T P^T, whose A operand is
//   eight rows of V transposed in registers (one byte permute per pair).
//   many rows (chunks): bound by the matrix cores.  Workgroups of 128 or 256
//   rows stage tiles of 64 keys in LDS; V is read from there transposed.
//
// Keys are split over workgroups where there are too few rows to fill the
// chip; partial sums (acc, max, sum) then go through a workspace and a second
// launch joins them, which also turns the logits into masses.
#include "paged_dev.h"

#include <float.h>

#include <algorithm>
#include <type_traits>

namespace hyq {
namespace {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef unsigned v4u __attribute__((ext_vector_type(4)));
typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int kBf16 = -1;            // page format beside HYQ_FMT_INT / HYQ_FMT_FP8 (8-bit codes)
constexpr int kFewRows = 16;         // rows per KV head of the few-row kernel
constexpr int kFewThreads = 256, kFewWaves = 4, kUnit = 32;
constexpr int kFewSplits = 256;      // most splits of a sequence's keys there
constexpr int kKeyTile = 64;         // keys of a tile of the many-row kernel
constexpr float kLazy = 8.0f;        // rescale only when the maximum grows by more than 2^8
constexpr float kNever = 3.0e38f;    // the "maximum" of a row that sees nothing: exp2(z - it) is 0
constexpr float kFloor = -FLT_MAX;   // start of a running maximum (finite: exp2 of -inf - it is 0)

struct AttnArgs {
  PagedGeom g;
  const uint8_t *k, *v;
  const float *ks, *vs;
  float* mass;
  const uint16_t* q;
  void* out;
  int out_bf16;
  int mass_mode;
  float c_log2;        // softmax_scale * log2(e)
  int few_max;         // sequences of at most so many rows go to the few-row kernel
  int S_few, S_many;   // splits of the keys in the two kernels
  int join_few;        // whether the few-row kernel leaves partials
  // Partial sums over a split's keys and their (max, sum): of chunks
  // [S_many][T][Hq][kHeadDim] and [T][Hq][S_many], of few rows
  // [S_few][B][Hkv][few_rows][kHeadDim] and [B][Hkv][few_rows][S_few] (by token they
  // would grow with the chunks of a mixed batch).
  float *many_part, *few_part;
  float2 *many_ml, *few_ml;
  int few_rows;
  float* logit;        // few rows with mass: [B][Hkv][few_rows][logit_stride]
  int logit_stride;
  uint32_t inv_g;      // ceil(2^32 / g) (g > 1): r / g for the rows of a step
  float2* stat;        // many rows with mass: (max, 1 / sum) of every query row [T][Hq]
};

// How far score z (times c) is above the reference m of its row, which is such a
// product rounded alike: the largest scores get weight 1 at any size.  One fused
// operation would leave up to half a step of m, and weights of 0 or infinity from
// scores of 2^31 on.
__device__ __forceinline__ float above(float z, float c, float m) {
#pragma clang fp contract(off)
  const float zc = z * c;
  return zc - m;
}

// Token of row r of a KV head's rows: r / g.  Exact for r < 2^29 (the quotient
// is too large by less than r / 2^32 < 1 / g, g <= 8).
__device__ __forceinline__ int token_of(const AttnArgs& a, int r) {
  return a.g.g == 1 ? r : (int)__umulhi((uint32_t)r, a.inv_g);
}

// Four codes (one dword) -> two pairs of bf16, exact (both formats have at
// most 8 significant bits).
template <int FMT>
__device__ __forceinline__ void codes4_to_bf16(uint32_t w, uint32_t& lo, uint32_t& hi) {
  if constexpr (FMT == HYQ_FMT_FP8) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true));
  } else {
    const uint32_t u = w ^ 0x80808080u;   // biased by 128: the unsigned byte conversions
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = (float)((u >> (8 * i)) & 0xffu) - 128.0f;
    lo = __builtin_amdgcn_perm(__float_as_uint(f[1]), __float_as_uint(f[0]), 0x07060302u);
    hi = __builtin_amdgcn_perm(__float_as_uint(f[3]), __float_as_uint(f[2]), 0x07060302u);
  }
}

// Eight consecutive elements of a page row as bf16, from 16 bytes of bf16 or
// 8 bytes of codes.
template <int FMT>
struct Eight {
  using type = v2u;
};
template <>
struct Eight<kBf16> {
  using type = v4u;
};
template <int FMT>
__device__ __forceinline__ v4u to_bf16(const typename Eight<FMT>::type& w) {
  if constexpr (FMT == kBf16) {
    return w;
  } else {
    v4u r;
    uint32_t a, b;
    codes4_to_bf16<FMT>(w[0], a, b);
    r[0] = a;
    r[1] = b;
    codes4_to_bf16<FMT>(w[1], a, b);
    r[2] = a;
    r[3] = b;
    return r;
  }
}
template <int FMT>
constexpr int row_bytes() {
  return FMT == kBf16 ? 2 * kHeadDim : kHeadDim;
}

// Channel j of eight rows (each row's 8 channels as 4 pairs) in key order.
__device__ __forceinline__ v4u column(const v4u (&r)[8], int j) {
  v4u o;
  const uint32_t sel = j & 1 ? 0x07060302u : 0x05040100u;
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = __builtin_amdgcn_perm(r[2 * e + 1][j >> 1], r[2 * e][j >> 1], sel);
  return o;
}

// ---------------------------------------------------------------------------
// Few rows.
// ---------------------------------------------------------------------------

// Registers of one unit of 32 keys: K rows of two 16-key tiles (four steps of
// 32 channels each), eight V rows, and the scales of this lane's 8 keys.
template <int FMT>
struct Unit {
  v4u k[2][FMT == kBf16 ? 4 : 2];
  typename Eight<FMT>::type v[8];
  v4f ks[2], vs[2];
  bool gone;   // the page of this lane's 8 keys is missing
};

// Key of tile t, A-operand row m, within a unit: lane group G's accumulators
// are then keys 8G .. 8G+7.
__device__ __forceinline__ int unit_key(int t, int m) { return ((m >> 2) << 3) + (t << 2) + (m & 3); }

// Channels of step s held by lane group G: any set as long as both operands
// use the same; bf16 rows 32s + 8G, code rows 16 consecutive bytes per load.
template <int FMT>
__device__ __forceinline__ int step_channel(int s, int G) {
  return FMT == kBf16 ? s * 32 + G * 8 : (s >> 1) * 64 + G * 16 + (s & 1) * 8;
}

// Pages of a unit's two halves of 16 keys (a page is at least 16 slots).
struct UnitPages {
  int p0, p1;
};
__device__ __forceinline__ UnitPages unit_pages(const PagedGeom& a, const int* __restrict__ row, int u) {
  const int i0 = (u * kUnit) >> a.page_log2, i1 = (u * kUnit + 16) >> a.page_log2;
  return UnitPages{i0 < a.max_pages ? row[i0] : -1, i1 < a.max_pages ? row[i1] : -1};
}

template <int FMT>
__device__ __forceinline__ void load_unit(Unit<FMT>& r, const AttnArgs& a, UnitPages pg, int j, int u,
                                          int hl, int G) {
  const int mask = (1 << a.g.page_log2) - 1, base = u * kUnit;
  const int np = a.g.n_pages;
  const bool ok0 = (unsigned)pg.p0 < (unsigned)np, ok1 = (unsigned)pg.p1 < (unsigned)np;
  const size_t r0 = ((size_t)(ok0 ? pg.p0 : 0) * a.g.Hkv + j) << a.g.page_log2;
  const size_t r1 = ((size_t)(ok1 ? pg.p1 : 0) * a.g.Hkv + j) << a.g.page_log2;
  const bool kh = hl >= 8, vh = G >= 2;   // K rows: keys 8 (hl / 4) ..; V rows: keys 8G ..
  r.gone = !(vh ? ok1 : ok0);
  const size_t krow = kh ? r1 : r0;
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    const uint8_t* p = a.k + (krow + ((base + unit_key(t, hl)) & mask)) * row_bytes<FMT>();
#pragma unroll
    for (int s = 0; s < (FMT == kBf16 ? 4 : 2); ++s)
      r.k[t][s] = __builtin_nontemporal_load(
          reinterpret_cast<const v4u*>(p + s * 64 + G * 16));
  }
  const size_t vrow = (vh ? r1 : r0) + ((base + 8 * G) & mask);
  const uint8_t* p = a.v + vrow * row_bytes<FMT>() + hl * (row_bytes<FMT>() / 16);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    r.v[e] = __builtin_nontemporal_load(
        reinterpret_cast<const typename Eight<FMT>::type*>(p + e * row_bytes<FMT>()));
  if constexpr (FMT != kBf16) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      r.ks[e] = *reinterpret_cast<const v4f*>(a.ks + vrow + 4 * e);
      r.vs[e] = *reinterpret_cast<const v4f*>(a.vs + vrow + 4 * e);
    }
  }
}

// Online softmax of one wave: lane (n = lane % 16, G): row n, O^T tiles j:
// channels 8 (4G + r) + j of row n in register r.
struct FewState {
  v4f acc[8];
  float m, l;   // running maximum (log2 units, the same on a row's 4 lanes); this lane's sum
};

__device__ __forceinline__ float rows_max(float x) {
  x = fmaxf(x, __shfl_xor(x, 16, 64));
  return fmaxf(x, __shfl_xor(x, 32, 64));
}

// last: the last key the lane's row sees.  lg: where this lane's 8 logits go,
// or NULL.
template <int FMT>
__device__ __forceinline__ void few_unit(FewState& st, const Unit<FMT>& r, const v8bf (&q)[4],
                                         float c, int base, int last, int n_kv, float* lg, int G) {
  v4f s[2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    s[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v4u ka;
      if constexpr (FMT == kBf16) ka = r.k[t][i];
      else ka = to_bf16<FMT>(v2u{r.k[t][i >> 1][(i & 1) * 2], r.k[t][i >> 1][(i & 1) * 2 + 1]});
      s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, ka), q[i], s[t], 0, 0, 0);
    }
  }
  const int key0 = base + 8 * G;
  // keys of a missing page, behind the sequence or the row's own token take no part
  const int lim = r.gone ? -1 : last;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float x = s[e >> 2][e & 3];
    if constexpr (FMT != kBf16) x *= r.ks[e >> 2][e & 3];
    y[e] = key0 + e <= lim ? x : -INFINITY;
  }
  if (lg) {
    *reinterpret_cast<v4f*>(lg) = v4f{y[0], y[1], y[2], y[3]};
    *reinterpret_cast<v4f*>(lg + 4) = v4f{y[4], y[5], y[6], y[7]};
  }
  float top = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
  top = rows_max(top) * c;
  const float mnew = top > st.m + kLazy ? top : st.m;
  if (__ballot(mnew != st.m)) {
    const float f = __builtin_amdgcn_exp2f(st.m - mnew);
#pragma unroll
    for (int t = 0; t < 8; ++t) st.acc[t] *= f;
    st.l *= f;
    st.m = mnew;
  }
  const int there = r.gone ? 0 : n_kv - key0;   // of the lane's 8 keys, those somebody owns
  // weights as a high (truncated, 8 bits) + low (rounded) bf16 pair, 2^-16
  // relative: the kernel waits for memory, the second product is free
  uint32_t hi[8], lo[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float p = __builtin_amdgcn_exp2f(above(y[e], c, st.m));
    st.l += p;
    if constexpr (FMT != kBf16) p *= e < there ? r.vs[e >> 2][e & 3] : 0.0f;
    hi[e] = __float_as_uint(p) & 0xffff0000u;
    lo[e] = __float_as_uint(p - __uint_as_float(hi[e]));
  }
  v4u ph, pl;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    ph[e] = __builtin_amdgcn_perm(hi[2 * e + 1], hi[2 * e], 0x07060302u);
    const v2bf b = {(__bf16)__uint_as_float(lo[2 * e]), (__bf16)__uint_as_float(lo[2 * e + 1])};
    pl[e] = __builtin_bit_cast(uint32_t, b);
  }
  // rows of V nobody owns are zero (they may hold NaN)
  v4u rows[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    rows[e] = to_bf16<FMT>(r.v[e]);
    if (e >= there) rows[e] = v4u{0u, 0u, 0u, 0u};
  }
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const v8bf va = __builtin_bit_cast(v8bf, column(rows, t));
    st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(v8bf, ph), st.acc[t], 0, 0, 0);
    st.acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(va, __builtin_bit_cast(v8bf, pl), st.acc[t], 0, 0, 0);
  }
}

__device__ __forceinline__ void store4(const AttnArgs& a, size_t row, int ch, v4f x) {
  if (a.out_bf16) {
    const v2bf p = {(__bf16)x[0], (__bf16)x[1]}, q = {(__bf16)x[2], (__bf16)x[3]};
    *reinterpret_cast<v2u*>(static_cast<uint16_t*>(a.out) + row * kHeadDim + ch) =
        v2u{__builtin_bit_cast(uint32_t, p), __builtin_bit_cast(uint32_t, q)};
  } else {
    *reinterpret_cast<v4f*>(static_cast<float*>(a.out) + row * kHeadDim + ch) = x;
  }
}

// Workgroup (b, s, j) (j fastest: the heads of a sequence go to different
// XCDs, the splits of one head to one): its 4 waves take even shares of the
// units, the next unit's loads in flight beside the one being computed; their
// states are joined in LDS.  16 sequences of 32k slots, 32 heads over 8: 348 to
// 352 us with the logits written (4.9 TB/s; a large copy moves 4.8 to 5.2, the
// norms 5.6), 32 of 8k in E4M3 pages with 40 heads 82 to 85 us (4.9 to 5.1 TB/s).
template <int FMT>
__global__ void __launch_bounds__(kFewThreads, 2)
paged_few_kernel(AttnArgs a) {
  __shared__ float w_acc[kFewWaves][kFewRows][kHeadDim];
  __shared__ float w_m[kFewWaves][kFewRows], w_l[kFewWaves][kFewRows];
  const int j = blockIdx.x % a.g.Hkv, bs = blockIdx.x / a.g.Hkv;
  const int sp = bs % a.S_few, b = bs / a.S_few;
  const Seq sq = seq_of(a.g, b);
  const int rows = sq.n_new * a.g.g;
  if (rows == 0 || rows > a.few_max) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, hl = lane & 15, G = lane >> 4;
  const int n = min(hl, rows - 1);   // lanes past the last row repeat it
  const int i = n / a.g.g, h = n - i * a.g.g;
  const size_t qrow = (size_t)(sq.t0 + i) * a.g.Hq + (size_t)j * a.g.g + h;
  v8bf q[4];
#pragma unroll
  for (int s = 0; s < 4; ++s)
    q[s] = *reinterpret_cast<const v8bf*>(a.q + qrow * kHeadDim + step_channel<FMT>(s, G));
  const int last = min(sq.len + i, sq.n_kv - 1);

  FewState st;
#pragma unroll
  for (int t = 0; t < 8; ++t) st.acc[t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
  st.m = kFloor;
  st.l = 0.0f;

  const int nu = (sq.n_kv + kUnit - 1) / kUnit, nw = a.S_few * kFewWaves, gw = sp * kFewWaves + w;
  const int first = (int)((int64_t)gw * nu / nw), end = (int)((int64_t)(gw + 1) * nu / nw);
  const int* trow = a.g.table + (size_t)b * a.g.max_pages;
  float* lg = a.logit ? a.logit + ((size_t)((size_t)b * a.g.Hkv + j) * a.few_rows + hl) * a.logit_stride + 8 * G
                      : nullptr;
  if (lg && hl >= rows) lg = nullptr;
  Unit<FMT> r0, r1;
  auto proc = [&](const Unit<FMT>& r, int u) {
    // keep the next unit's waits out of this one
    __builtin_amdgcn_sched_barrier(0);
    few_unit<FMT>(st, r, q, a.c_log2, u * kUnit, last, sq.n_kv, lg ? lg + (size_t)u * kUnit : nullptr, G);
    __builtin_amdgcn_sched_barrier(0);
  };
  int u = first;
  if (u < end) {
    load_unit<FMT>(r0, a, unit_pages(a.g, trow, u), j, u, hl, G);
    UnitPages pg = unit_pages(a.g, trow, min(u + 1, end - 1));
    for (; u + 2 < end; u += 2) {
      load_unit<FMT>(r1, a, pg, j, u + 1, hl, G);
      pg = unit_pages(a.g, trow, u + 2);
      proc(r0, u);
      load_unit<FMT>(r0, a, pg, j, u + 2, hl, G);
      pg = unit_pages(a.g, trow, min(u + 3, end - 1));
      proc(r1, u + 1);
    }
    if (u + 1 < end) {
      load_unit<FMT>(r1, a, pg, j, u + 1, hl, G);
      proc(r0, u);
      proc(r1, u + 1);
    } else {
      proc(r0, u);
    }
  }

  float l = st.l;
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (G == 0) {
    w_m[w][hl] = st.m;
    w_l[w][hl] = l;
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
#pragma unroll
    for (int t = 0; t < 8; ++t) w_acc[w][hl][8 * (4 * G + r) + t] = st.acc[t][r];
  __syncthreads();
  for (int e = threadIdx.x; e < rows * (kHeadDim / 4); e += kFewThreads) {
    const int rw = e >> 5, ch = (e & 31) * 4;
    float M = w_m[0][rw];
#pragma unroll
    for (int x = 1; x < kFewWaves; ++x) M = fmaxf(M, w_m[x][rw]);
    v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    float sum = 0.0f;
#pragma unroll
    for (int x = 0; x < kFewWaves; ++x) {
      const float f = __builtin_amdgcn_exp2f(w_m[x][rw] - M);
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] += w_acc[x][rw][ch + c] * f;
      sum += w_l[x][rw] * f;
    }
    const int ii = rw / a.g.g;
    const size_t row = (size_t)(sq.t0 + ii) * a.g.Hq + (size_t)j * a.g.g + (rw - ii * a.g.g);
    if (a.join_few) {
      const size_t heads = (size_t)a.g.B * a.g.Hkv, at = ((size_t)b * a.g.Hkv + j) * a.few_rows + rw;
      *reinterpret_cast<v4f*>(a.few_part + (sp * heads * a.few_rows + at) * kHeadDim + ch) = acc;
      if (ch == 0) a.few_ml[at * a.S_few + sp] = make_float2(M, sum);
    } else {
      store4(a, row, ch, acc * (sum > 0.0f ? 1.0f / sum : 0.0f));
    }
  }
}

// ---------------------------------------------------------------------------
// Many rows.
// ---------------------------------------------------------------------------

// Tiles of 64 keys in LDS, rows of 16 chunks of 16 bytes: chunk c of K row r at
// c ^ (r & 15), of V row r at c ^ 4 (r & 3).  The first makes the 16 lanes of a
// read phase (16 rows, one chunk) meet different banks, the second the 32 of a
// transposing read (4 rows, 4 chunks).
struct ManyLds {
  v4u k[2][kKeyTile * 16];
  v4u v[2][kKeyTile * 16];
  // of K's tiles
  float ks[2][kKeyTile], vs[2][kKeyTile];
  uint8_t gone[2][kKeyTile / 4];   // 4-key groups whose page is missing
};

// What one thread holds of a tile's K or V: U rows (keys U kg ..) of eight
// channels (chunk).
template <int FMT, int U>
struct Stage {
  typename Eight<FMT>::type x[U];
  float ks, vs;   // codes: scales of key U kg + chunk % U, loaded with K
  int page;       // -1: missing
};

template <int FMT, bool IS_K, int U>
__device__ __forceinline__ void stage_load(Stage<FMT, U>& g, const AttnArgs& a, int page, int j, int tile,
                                           int kg, int chunk) {
  g.page = page;
  const size_t row = pool_row(a.g, max(page, 0), j, tile * kKeyTile + kg * U);
  const uint8_t* p = (IS_K ? a.k : a.v) + row * row_bytes<FMT>() + chunk * (row_bytes<FMT>() / 16);
#pragma unroll
  for (int e = 0; e < U; ++e)
    g.x[e] = *reinterpret_cast<const typename Eight<FMT>::type*>(p + e * row_bytes<FMT>());
  if constexpr (FMT != kBf16 && IS_K) {
    g.ks = a.ks[row + (chunk & (U - 1))];
    g.vs = a.vs[row + (chunk & (U - 1))];
  }
}

template <int FMT, int U>
__device__ __forceinline__ void store_k(const Stage<FMT, U>& g, ManyLds& m, int buf, int tile, int n_kv,
                                        int kg, int chunk, float c_log2) {
#pragma unroll
  for (int e = 0; e < U; ++e) {
    const int r = kg * U + e;
    m.k[buf][r * 16 + (chunk ^ (r & 15))] = to_bf16<FMT>(g.x[e]);
  }
  if (chunk == 0 && (kg * U) % 4 == 0) m.gone[buf][kg * U / 4] = g.page < 0;
  if constexpr (FMT != kBf16) {   // finite and positive, so that hidden scores stay -inf
    const int there = g.page < 0 ? 0 : n_kv - (tile * kKeyTile + kg * U);
    if (chunk < U) {
      m.ks[buf][kg * U + chunk] = chunk < there ? fmaxf(g.ks * c_log2, 1e-37f) : c_log2;
      m.vs[buf][kg * U + chunk] = chunk < there ? g.vs : 0.0f;
    }
  }
}

template <int FMT, int U>
__device__ __forceinline__ void store_v(const Stage<FMT, U>& g, ManyLds& m, int buf, int tile, int n_kv,
                                        int kg, int chunk) {
  const int there = g.page < 0 ? 0 : n_kv - (tile * kKeyTile + kg * U);   // rows nobody owns are zero
#pragma unroll
  for (int e = 0; e < U; ++e) {
    const int r = kg * U + e;
    v4u x = to_bf16<FMT>(g.x[e]);
    if (e >= there) x = v4u{0u, 0u, 0u, 0u};
    m.v[buf][r * 16 + (chunk ^ ((r & 3) << 2))] = x;
  }
}

// Key (within 32) of A-operand row m: bits 2 and 3 swapped, so that a lane's
// accumulators 8a .. 8a+7 are the eight keys 16a + 8h .. of the next product's
// B operand.
__device__ __forceinline__ int many_key(int m) { return (m & 0x13) | ((m & 4) << 1) | ((m & 8) >> 1); }

// S^T = K q^T of one tile: s[x][e] is key 32x + 16 (e / 8) + 8 hf + e % 8, row n.
__device__ __forceinline__ void many_scores(v16f (&s)[2], const v4u* kt, const v8bf (&q)[8], int n, int hf) {
  const int r = many_key(n);
  v4u ka[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) ka[c] = kt[r * 16 + ((2 * c + hf) ^ (r & 15))];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int e = 0; e < 16; ++e) s[x][e] = 0.0f;
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    s[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, ka[c]), q[c], s[0], 0, 0, 0);
    ka[c] = kt[(r + 32) * 16 + ((2 * c + hf) ^ (r & 15))];
  }
#pragma unroll
  for (int c = 0; c < 8; ++c)
    s[1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf, ka[c]), q[c], s[1], 0, 0, 0);
  // eight reads in flight, then one behind each product of the first half
  __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
}

// A operand of step (o, d) of O^T = V^T P^T: lane (channel 32 d + lane % 32,
// half hf) holds keys 16 o + 8 hf .. + 7 of its channel: two transposing reads,
// each of which gives the 16 lanes of a group one column of the 4 x 16 block
// whose rows 4 lanes each point at.  `lane_v` is the lane's part of the address
// (bytes), without the chunk bits of d.
__device__ __forceinline__ int lane_v(int lane) {
  const int i = lane & 15, row = ((lane >> 5) << 3) + (i >> 2);
  const int chunk = (((lane >> 4) & 1) << 1) + ((i >> 1) & 1);
  return row * 256 + ((chunk ^ ((i >> 2) << 2)) << 4) + ((i & 1) << 3);
}
__device__ __forceinline__ v8bf read_v(const v4u* vt, int lane_part, int o, int d) {
  typedef short v4s __attribute__((ext_vector_type(4)));
  typedef short v8s __attribute__((ext_vector_type(8)));
  const char* base = reinterpret_cast<const char*>(vt);
  v4s x[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {   // keys + 4 u
    const char* p = base + ((lane_part ^ (d << 6)) + (o * 16 + u * 4) * 256);
    x[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) v4s*)reinterpret_cast<const v4s*>(p));
  }
  const v8s r = {x[0][0], x[0][1], x[0][2], x[0][3], x[1][0], x[1][1], x[1][2], x[1][3]};
  return __builtin_bit_cast(v8bf, r);
}

// Workgroup (b, t, sp, j) of NW waves: rows [32 NW t, 32 NW (t + 1)) of a
// sequence's rows for KV head j, share sp of the keys they see.  One barrier a tile: iteration c
// takes the scores of tile c, then the weights of tile c step by step between
// the products of V with the weights of tile c - 1, so that exponentials and
// matrix cores run side by side.  K is staged a tile ahead, V in time, the
// loads of both a tile earlier still.
//
// The reference of a row's weights is the maximum of the first tile it sees;
// later tiles need no maximum of their own: bf16 weights keep their precision
// at any size, so the reference moves only when a lane's weights of a tile sum
// to more than 2^16 (which leaves the accumulators their range).
//
// Weights (times a value row's scale with codes) are rounded to bf16, the type of
// the products; the row sum keeps them as they are.  Outputs in bf16 are then
// 0.0024 off (relative, of normal values; up to 0.003 where few keys of 8-bit pages
// hold the weight), 0.0017 by their own rounding alone.  A high + low pair as
// above would make 48 products of 32 a tile where products are the bound.
//
// 512 tokens over 32256 slots, 32 heads over 8, bf16: 272 us and 11 to join (1.0
// PFLOP/s, a large matrix product reaches 1.18 to 1.22); 3 x 2k over 6011 int8
// slots, 40 heads over 8: 844 us (0.82 PFLOP/s).  Power sets the clock there:
// running two groups of waves half a tile apart cut cycles but not time.
//
// Weights come from one fused operation each; where a row of the wave has its
// reference beyond 2^16 (up to there the exponent differs from `above` by 2^-8 at
// most), they are taken once more by `above`, in every tile.
constexpr float kFarSum = 0x1p16f;
constexpr float kFarScore = 0x1p16f;

template <int FMT, int NW>
__global__ void __launch_bounds__(NW * 64, 2)
paged_many_kernel(AttnArgs a, const int32_t* __restrict__ table, int tiles) {
  constexpr int kRowTile = NW * 32, U = 16 / NW;
  __shared__ ManyLds lds;
  const int j = blockIdx.x % a.g.Hkv;
  int id = blockIdx.x / a.g.Hkv;
  const int sp = id % a.S_many;
  id /= a.S_many;
  const int t = tiles - 1 - id % tiles, b = id / tiles;   // the longest scans first
  const Seq sq = seq_of(a.g, b);
  const int rows = sq.n_new * a.g.g;
  if (rows <= a.few_max || t * kRowTile >= rows) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
  const int r_mine = t * kRowTile + w * 32 + n;
  const int rr = min(r_mine, rows - 1);
  const int i = rr / a.g.g, h = rr - i * a.g.g;
  const size_t qrow = (size_t)(sq.t0 + i) * a.g.Hq + (size_t)j * a.g.g + h;
  v8bf q[8];
#pragma unroll
  for (int s = 0; s < 8; ++s)
    q[s] = *reinterpret_cast<const v8bf*>(a.q + qrow * kHeadDim + 16 * s + 8 * hf);
  const int last = min(sq.len + i, sq.n_kv - 1);
  // keys any row of the workgroup sees, keys every row of it sees
  const int i_first = (t * kRowTile) / a.g.g, i_last = (min((t + 1) * kRowTile, rows) - 1) / a.g.g;
  const int n_keys = min(sq.len + i_last + 1, sq.n_kv), n_all = min(sq.len + i_first + 1, sq.n_kv);
  const int nt = (n_keys + kKeyTile - 1) / kKeyTile;
  const int first = (int)((int64_t)sp * nt / a.S_many), end = (int)((int64_t)(sp + 1) * nt / a.S_many);

  v16f acc[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[d][e] = 0.0f;
  float m = kFloor, l = 0.0f;
  bool far = false;   // some row of the wave has its reference beyond kFarScore

  if (first < end) {
    const int kg = threadIdx.x >> 4, chunk = threadIdx.x & 15;
    // the wave's rows of a tile (4 U, aligned) lie in one page: a scalar lookup
    // an iteration ahead of its use, looked at when it is used
    auto entry_of = [&](int tile) {
      return __builtin_amdgcn_readfirstlane((min(tile, end - 1) * kKeyTile + w * (4 * U)) >> a.g.page_log2);
    };
    auto entry_at = [&](int tile) { return table[(size_t)b * a.g.max_pages + min(entry_of(tile), a.g.max_pages - 1)]; };
    auto page_at = [&](int tile, int entry) {
      return entry_of(tile) < a.g.max_pages && (unsigned)entry < (unsigned)a.g.n_pages ? entry : -1;
    };
    auto tile_at = [&](int tile) { return min(tile, end - 1); };
    // of the keys of accumulators 4 f .. 4 f + 3 of half x: what takes a score to
    // log2 units, and the scale of the value row
    auto four = [&](const float* p, int x, int f) {
      return *reinterpret_cast<const v4f*>(p + x * 32 + (f >> 1) * 16 + hf * 8 + (f & 1) * 4);
    };
    auto factor = [&](int buf, int x, int f) {
      if constexpr (FMT == kBf16) return v4f{a.c_log2, a.c_log2, a.c_log2, a.c_log2};
      else return four(lds.ks[buf], x, f);
    };
    auto value_scale = [&](int buf, int x, int f) {
      if constexpr (FMT == kBf16) return v4f{1.0f, 1.0f, 1.0f, 1.0f};
      else return four(lds.vs[buf], x, f);
    };
    Stage<FMT, U> gk, gv;
    int pk = page_at(first, entry_at(first));
    stage_load<FMT, true, U>(gk, a, pk, j, first, kg, chunk);
    stage_load<FMT, false, U>(gv, a, pk, j, first, kg, chunk);
    store_k<FMT, U>(gk, lds, first & 1, first, sq.n_kv, kg, chunk, a.c_log2);
    pk = page_at(first + 1, entry_at(first + 1));
    stage_load<FMT, true, U>(gk, a, pk, j, tile_at(first + 1), kg, chunk);
    int next = entry_at(first + 2);   // table entry of the tile after the next
    v8bf pprev[4];
#pragma unroll
    for (int o = 0; o < 4; ++o) pprev[o] = v8bf{};
    // zeros where the first iteration multiplies V of "tile first - 1"
#pragma unroll
    for (int x = 0; x < U; ++x) lds.v[(first + 1) & 1][threadIdx.x + x * NW * 64] = v4u{0u, 0u, 0u, 0u};
    const int lv = lane_v(lane);
    for (int tile = first; tile < end; ++tile) {
      const int kb = tile & 1, vb = kb ^ 1;
      __syncthreads();
      v16f s[2];
      many_scores(s, lds.k[kb], q, n, hf);
      // K of the next tile (past the end the last one again: no branch); its
      // buffer was last read before the barrier
      store_k<FMT, U>(gk, lds, kb ^ 1, tile_at(tile + 1), sq.n_kv, kg, chunk, a.c_log2);
      const int pn = page_at(tile + 2, next);
      next = entry_at(tile + 3);
      stage_load<FMT, true, U>(gk, a, pn, j, tile_at(tile + 2), kg, chunk);
      const uint64_t* gp = reinterpret_cast<const uint64_t*>(lds.gone[kb]);
      const uint64_t g0 = gp[0], g1 = gp[1];
      if ((g0 | g1) != 0 || (tile + 1) * kKeyTile > n_all) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int grp = (e >> 3) * 4 + hf * 2 + ((e >> 2) & 1), key = tile * kKeyTile + x * 32 + grp * 4 + (e & 3);
            const bool hid = key > last || (((x ? g1 : g0) >> (8 * grp)) & 1);
            s[x][e] = hid ? -INFINITY : s[x][e];
          }
      }
      v8bf pcur[4];
      float ps = 0.0f, ps1 = 0.0f;
      __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int u = 0; u < 16; ++u) {
        const int d = u & 3, o = u >> 2;
        acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(lds.v[vb], lv, o, d), pprev[o], acc[d], 0, 0, 0);
        const int x = u >> 3, e = (u & 7) * 2;
        const v4f f = factor(kb, x, e >> 2);
        const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], f[e & 3], -m));
        const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e + 1], f[(e & 3) + 1], -m));
        ps += p0;
        ps1 += p1;
        const v4f vs = value_scale(kb, x, e >> 2);
        pcur[x * 2 + (e >> 3)][e & 7] = (__bf16)(p0 * vs[e & 3]);
        pcur[x * 2 + (e >> 3)][(e & 7) + 1] = (__bf16)(p1 * vs[(e & 3) + 1]);
      }
      // the weights stay here, beside the products
      asm volatile("" : "+v"(pcur[0]), "+v"(pcur[1]), "+v"(pcur[2]), "+v"(pcur[3]), "+v"(ps), "+v"(ps1));
      ps += ps1;
      __builtin_amdgcn_s_setprio(0);
      if (tile == first || far || __ballot(!(ps <= kFarSum))) {
        float top = -INFINITY;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
          for (int e = 0; e < 16; ++e) top = fmaxf(top, s[x][e] * factor(kb, x, e >> 2)[e & 3]);
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float mnew = fmaxf(m, top);
        const float f = __builtin_amdgcn_exp2f(m - mnew);
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) acc[d][e] *= f;
        l *= f;
        m = mnew;
        far = __ballot(m > kFloor && fabsf(m) > kFarScore) != 0;
        ps = 0.0f;
        auto weights = [&](auto fused) {
#pragma unroll
          for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float c = factor(kb, x, e >> 2)[e & 3];
              const float d = decltype(fused)::value ? __builtin_fmaf(s[x][e], c, -m) : above(s[x][e], c, m);
              const float pw = __builtin_amdgcn_exp2f(d);
              ps += pw;
              pcur[x * 2 + (e >> 3)][e & 7] = (__bf16)(pw * value_scale(kb, x, e >> 2)[e & 3]);
            }
        };
        if (far) weights(std::false_type{});
        else weights(std::true_type{});
      }
      l += ps;
      // V of this tile: its buffer was last read before the barrier too
      store_v<FMT, U>(gv, lds, kb, tile, sq.n_kv, kg, chunk);
      stage_load<FMT, false, U>(gv, a, pk, j, tile_at(tile + 1), kg, chunk);
      pk = pn;
#pragma unroll
      for (int o = 0; o < 4; ++o) pprev[o] = pcur[o];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 16; ++u) {
      const int d = u & 3, o = u >> 2;
      acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(read_v(lds.v[(end + 1) & 1], lv, o, d), pprev[o], acc[d],
                                                       0, 0, 0);
    }
  }
  l += __shfl_xor(l, 32, 64);
  if (r_mine >= rows) return;
  if (a.S_many > 1) {
    float* dst = a.many_part + ((size_t)sp * a.g.T * a.g.Hq + qrow) * kHeadDim;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<v4f*>(dst + d * 32 + e * 8 + hf * 4) =
            v4f{acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]};
    if (hf == 0) a.many_ml[(size_t)qrow * a.S_many + sp] = make_float2(m, l);
  } else {
    const float inv = l > 0.0f ? 1.0f / l : 0.0f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        store4(a, qrow, d * 32 + e * 8 + hf * 4,
               v4f{acc[d][4 * e], acc[d][4 * e + 1], acc[d][4 * e + 2], acc[d][4 * e + 3]} * inv);
    if (a.stat && hf == 0) a.stat[qrow] = make_float2(l > 0.0f ? m : kNever, inv);
  }
}

// ---------------------------------------------------------------------------
// Joining the splits, and masses.
// ---------------------------------------------------------------------------

constexpr int kJoinThreads = 128;     // chunks: at most 64 splits, in practice a handful
constexpr int kFinishThreads = 256;   // few rows: up to kFewSplits
constexpr int kStatThreads = kFinishThreads / kFewRows;   // threads that join a row's maximum and sum
constexpr int kMassKeys = kFinishThreads * 4;   // keys of a mass workgroup of the few-row path

// Row `row` (token * Hq + head) of the output from its S partials, `stride` floats
// apart, and their (max, sum): shares of them, 32 lanes of 4 channels each, joined
// through LDS.
template <int THREADS>
__device__ __forceinline__ void join_row(const AttnArgs& a, size_t row, const float* part, size_t stride,
                                         const float2* mls, int S) {
  constexpr int kShares = THREADS / 32;
  __shared__ v4f x_acc[kShares][32];
  __shared__ float x_m[kShares], x_l[kShares];
  const int c4 = threadIdx.x & 31, ph = threadIdx.x >> 5;
  const float* base = part + c4 * 4;
  float M = kFloor, L = 0.0f;
  v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int s = ph; s < S; s += kShares) {
    const v4f x = *reinterpret_cast<const v4f*>(base + s * stride);
    const float2 ml = mls[s];
    const float mn = fmaxf(M, ml.x);
    const float f = __builtin_amdgcn_exp2f(M - mn), e = __builtin_amdgcn_exp2f(ml.x - mn);
    acc = acc * f + x * e;
    L = L * f + ml.y * e;
    M = mn;
  }
  x_acc[ph][c4] = acc;
  if (c4 == 0) {
    x_m[ph] = M;
    x_l[ph] = L;
  }
  __syncthreads();
  if (ph != 0) return;
#pragma unroll
  for (int s = 1; s < kShares; ++s) {
    const float mn = fmaxf(M, x_m[s]);
    const float f = __builtin_amdgcn_exp2f(M - mn), e = __builtin_amdgcn_exp2f(x_m[s] - mn);
    acc = acc * f + x_acc[s][c4] * e;
    L = L * f + x_l[s] * e;
    M = mn;
  }
  const float inv = L > 0.0f ? 1.0f / L : 0.0f;
  store4(a, row, c4 * 4, acc * inv);
  if (a.stat && c4 == 0) a.stat[row] = make_float2(L > 0.0f ? M : kNever, inv);
}

// Chunks whose keys were split: one workgroup per query row of the step.
__global__ void __launch_bounds__(kJoinThreads)
paged_join_kernel(AttnArgs a) {
  const int t = blockIdx.x / a.g.Hq;
  const int b = seq_of_token(a.g, t);
  if (b < 0) return;
  const Seq sq = seq_of(a.g, b);
  if (t - sq.t0 >= sq.n_new || sq.n_new * a.g.g <= a.few_max) return;
  const size_t row = blockIdx.x;
  join_row<kJoinThreads>(a, row, a.many_part + row * kHeadDim, (size_t)a.g.T * a.g.Hq * kHeadDim,
                         a.many_ml + row * a.S_many, a.S_many);
}

// After the few-row kernel (one launch for both, 15 us at 16 x 32k slots; 33 as
// two): workgroups (b, j, y) with y < kFewRows join query row y; the others
// (with masses) take 1024 keys each: the maximum and the sum of every row from
// the partials, then the weights from the stored logits (4 keys a thread, rows in
// order).  Maxima and sums of a row lie together (32768 slots, 32 heads over 8:
// 26.8 us, 27.6 inside the partials); 16 threads join them for the masses (65536
// E4M3 slots, 8 heads over 2, 128 splits: 27 us with 4 threads, 19 with 8).
__global__ void __launch_bounds__(kFinishThreads)
paged_few_finish_kernel(AttnArgs a) {
  const int j = blockIdx.x % a.g.Hkv, b = blockIdx.x / a.g.Hkv;
  const Seq sq = seq_of(a.g, b);
  const int rows = sq.n_new * a.g.g;
  if (rows == 0 || rows > a.few_max) return;
  const size_t first = ((size_t)b * a.g.Hkv + j) * a.few_rows;   // of the head's partials
  if (blockIdx.y < kFewRows) {
    if ((int)blockIdx.y < rows) {
      const size_t at = first + blockIdx.y;
      const int i = (int)blockIdx.y / a.g.g;
      join_row<kFinishThreads>(a, (size_t)(sq.t0 + i) * a.g.Hq + (size_t)j * a.g.g + (blockIdx.y - i * a.g.g),
                               a.few_part + at * kHeadDim, (size_t)a.g.B * a.g.Hkv * a.few_rows * kHeadDim,
                               a.few_ml + at * a.S_few, a.S_few);
    }
    return;
  }
  const int key = (blockIdx.y - kFewRows) * kMassKeys + (int)threadIdx.x * 4;
  if (key - (int)threadIdx.x * 4 >= sq.n_kv) return;
  __shared__ float2 st[kFewRows];
  if ((int)threadIdx.x < rows * kStatThreads) {
    const int r = threadIdx.x / kStatThreads;
    const float2* mls = a.few_ml + (first + r) * a.S_few;
    float M = kFloor, L = 0.0f;
#pragma unroll 8
    for (int s = threadIdx.x % kStatThreads; s < a.S_few; s += kStatThreads) {
      const float2 ml = mls[s];
      const float mn = fmaxf(M, ml.x);
      L = L * __builtin_amdgcn_exp2f(M - mn) + ml.y * __builtin_amdgcn_exp2f(ml.x - mn);
      M = mn;
    }
#pragma unroll
    for (int o = 1; o < kStatThreads; o <<= 1) {
      const float m2 = __shfl_xor(M, o, 64), l2 = __shfl_xor(L, o, 64);
      const float mn = fmaxf(M, m2);
      L = L * __builtin_amdgcn_exp2f(M - mn) + l2 * __builtin_amdgcn_exp2f(m2 - mn);
      M = mn;
    }
    if (threadIdx.x % kStatThreads == 0) st[r] = make_float2(L > 0.0f ? M : kNever, L > 0.0f ? 1.0f / L : 0.0f);
  }
  __syncthreads();
  if (key >= sq.n_kv) return;
  const float* lg = a.logit + first * a.logit_stride + key;
  v4f sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
  for (int r = 0; r < rows; ++r) {
    const v4f z = *reinterpret_cast<const v4f*>(lg + (size_t)r * a.logit_stride);
    const float2 ml = st[r];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      sum[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(above(z[e], a.c_log2, ml.x)), ml.y, sum[e]);
  }
  const int p = page_of(a.g, b, key);
  if (p < 0) return;
  float* m = a.mass + pool_row(a.g, p, j, key);
  const int n = min(4, sq.n_kv - key);
  if (n == 4) {
    v4f* m4 = reinterpret_cast<v4f*>(m);
    *m4 = a.mass_mode == HYQ_MASS_ADD ? *m4 + sum : sum;
  } else {
    for (int e = 0; e < n; ++e) m[e] = a.mass_mode == HYQ_MASS_ADD ? m[e] + sum[e] : sum[e];
  }
}

// Many rows: the products again, now that every row's maximum and sum are
// known.  A wave owns 32 keys (their K rows stay in registers); the workgroup
// walks the rows that see any of its 128 keys in tiles of 64, staged in LDS for
// its four waves (chunk c of row r at c ^ (r & 15)), the next tile's loads in
// flight.  512 tokens over 32256 slots, 32 heads over 8: 180 us, matrix cores busy
// 35%, VALU 61%; with every row read from L2 by every wave it was 539.  Fused
// exponents would save 5 us; taken only where no row of a half tile needs `above`,
// the branch between the halves costs 6.
constexpr int kMassThreads = 256, kMassTile = 64;

template <int FMT>
__global__ void __launch_bounds__(kMassThreads, FMT == kBf16 ? 3 : 2)
paged_many_mass_kernel(AttnArgs a) {
  __shared__ v4u qs[2][kMassTile * 16];
  __shared__ float2 ss[2][kMassTile];
  const int j = blockIdx.x % a.g.Hkv, b = blockIdx.x / a.g.Hkv;
  const Seq sq = seq_of(a.g, b);
  const int rows = sq.n_new * a.g.g;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lane = threadIdx.x & 63, n = lane & 31, hf = lane >> 5;
  const int wg_key = blockIdx.y * 128, key0 = wg_key + w * 32;
  if (rows <= a.few_max || wg_key >= sq.n_kv) return;
  v8bf kf[8];
  float kse[16], sum[16];   // of key 8 (e / 4) + 4 hf + e % 4: what takes its scores to log2 units; its mass
  {
    const int key = key0 + n, p = page_of(a.g, b, key);
    const size_t row = pool_row(a.g, max(p, 0), j, key);
    const uint8_t* src = a.k + row * row_bytes<FMT>();
#pragma unroll
    for (int c = 0; c < 8; ++c)
      kf[c] = __builtin_bit_cast(v8bf, to_bf16<FMT>(*reinterpret_cast<const typename Eight<FMT>::type*>(
                                           src + (2 * c + hf) * (row_bytes<FMT>() / 16))));
    float ks = 1.0f;
    if constexpr (FMT != kBf16) ks = a.ks[row];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      // positive, so that hidden scores stay -inf
      kse[e] = FMT == kBf16 ? a.c_log2 : fmaxf(__shfl(ks, 8 * (e >> 2) + 4 * hf + (e & 3), 64) * a.c_log2, 1e-37f);
      sum[e] = 0.0f;
    }
  }
  // rows that see the first of the workgroup's keys: from token wg_key - len on
  const int first = max(0, wg_key - sq.len) * a.g.g / kMassTile, end = (rows + kMassTile - 1) / kMassTile;
  const int sr = threadIdx.x >> 2, sc = (threadIdx.x & 3) * 4;   // the row and chunks this thread stages
  const uint16_t* const qh = a.q + ((size_t)sq.t0 * a.g.Hq + (size_t)j * a.g.g) * kHeadDim + sc * 8;
  const float2* const sh = a.stat + (size_t)sq.t0 * a.g.Hq + (size_t)j * a.g.g;
  v4u g[4];
  float2 gs;
  auto load = [&](int tile) {
    const int r = tile * kMassTile + sr, rr = min(r, rows - 1), i = token_of(a, rr);
    const size_t at = (size_t)i * a.g.Hq + (rr - i * a.g.g);
#pragma unroll
    for (int x = 0; x < 4; ++x) g[x] = reinterpret_cast<const v4u*>(qh + at * kHeadDim)[x];
    gs = sh[at];
    if (r >= rows) gs.y = 0.0f;
  };
  auto store = [&](int buf) {
#pragma unroll
    for (int x = 0; x < 4; ++x) qs[buf][sr * 16 + ((sc + x) ^ (sr & 15))] = g[x];
    if (sc == 0) ss[buf][sr] = gs;
  };
  load(first);
  store(first & 1);
  for (int tile = first; tile < end; ++tile) {
    load(min(tile + 1, end - 1));
    __syncthreads();
    const int buf = tile & 1;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      v16f s;
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e] = 0.0f;
      v4u q[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) q[c] = qs[buf][(u * 32 + n) * 16 + ((2 * c + hf) ^ (n & 15))];
      const float2 ml = ss[buf][u * 32 + n];
#pragma unroll
      for (int c = 0; c < 8; ++c)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[c], __builtin_bit_cast(v8bf, q[c]), s, 0, 0, 0);
      // all reads in flight before the first product
      __builtin_amdgcn_sched_group_barrier(0x100, 9, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 8, 0);
      // some row of these 32 does not see some key of the wave
      const int r0 = tile * kMassTile + u * 32;
      if (key0 + 32 > min(sq.len + token_of(a, min(r0, rows - 1)) + 1, sq.n_kv)) {
        const int last = min(sq.len + token_of(a, min(r0 + n, rows - 1)), sq.n_kv - 1);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = key0 + 8 * (e >> 2) + 4 * hf + (e & 3) <= last ? s[e] : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e)
        sum[e] = __builtin_fmaf(__builtin_amdgcn_exp2f(above(s[e], kse[e], ml.x)), ml.y, sum[e]);
    }
    store((tile + 1) & 1);
  }
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    float v = sum[e];
#pragma unroll
    for (int o = 16; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
    const int key = key0 + 8 * (e >> 2) + 4 * hf + (e & 3);
    if (n != 0 || key >= sq.n_kv) continue;
    const int p = page_of(a.g, b, key);
    if (p < 0) continue;
    float* m = a.mass + pool_row(a.g, p, j, key);
    *m = a.mass_mode == HYQ_MASS_ADD ? *m + v : v;
  }
}

// ---------------------------------------------------------------------------
// Plan.
// ---------------------------------------------------------------------------

struct Plan {
  bool few, many;      // which kernels the batch can need
  int few_max;
  int S_few, S_many;
  bool join_few, join_many;
  int waves;           // of a workgroup of the many-row kernel (32 rows each)
  int row_tiles;       // row tiles of a sequence there
  int64_t n_kv;        // bound on a sequence's slots
  int few_rows, logit_stride;
  size_t many_part, many_ml, few_part, few_ml, logit, stat;   // workspace bytes
  size_t total() const { return many_part + many_ml + few_part + few_ml + logit + stat; }
};

size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

Plan plan_of(const hyq_pcache& c, const hyq_pbatch& b, int mass) {
  Plan p = {};
  const int g = c.Hq / c.Hkv;
  const int rows = std::max(b.max_new, 1) * g;   // not of T: the workspace then only grows with T
  p.many = rows > kFewRows;
  p.few = !p.many || b.B > 1;   // a mixed batch may hold single tokens
  p.few_max = p.few ? kFewRows : 0;
  p.n_kv = std::min((int64_t)b.max_len + b.max_new, (int64_t)b.max_pages * c.page);
  const int64_t heads = (int64_t)b.B * c.Hkv;
  const int64_t units = std::max<int64_t>(1, (p.n_kv + kUnit - 1) / kUnit);
  const int64_t ktiles = std::max<int64_t>(1, (p.n_kv + kKeyTile - 1) / kKeyTile);
  // Two workgroups to a CU, at least 8 units each; one KV head fills the chip by
  // itself from 2048 units on (131072 slots, 8 heads over 1: 19.9 us with 256
  // splits at most, 25.7 with 128, 41 with 64; 65536 E4M3 slots, 8 over 2, with
  // masses: 20.0, 18.3 and 28).
  p.S_few = (int)std::max<int64_t>(1, std::min({(512 + heads - 1) / heads, (units + 7) / 8, (int64_t)kFewSplits}));
  // Up to 128 rows, and below 4096 slots, workgroups of 128 rows (two to a CU)
  // balance better: 2048 tokens from nothing 61 us against 66 with 256 rows, 8 x
  // 200 over 1000 slots 44 and 47, 4 x 8 over 9001 33 and 40.  Longer scans gain
  // more from eight waves sharing a tile's staging: 3 x 2k over 6011 int8 slots
  // 839 and 966, 512 over 32k 276 and 295, 100 over 16k 50 and 52.  Near the limit
  // the two differ little (512 over 2500, 3400, 4000, 4600: four waves 50, 56, 59,
  // 64, eight 50, 55, 58, 62; 8 x 200 over 4000 and 5000: 122, 149 and 123, 148),
  // except where a step is large: 3 x 2k over 2500 slots 318 with eight and 328 with
  // four, int8 372 and 418.
  p.waves = rows <= 128 || p.n_kv < 4096 ? 4 : 8;
  const int64_t wg = heads * ((rows + p.waves * 32 - 1) / (p.waves * 32));
  const int launched = std::min(b.max_new, b.T) * g;   // the grid (the splits go by max_new alone)
  p.row_tiles = (launched + p.waves * 32 - 1) / (p.waves * 32);
  p.S_many = (int)std::max<int64_t>(1, std::min({(p.waves == 4 ? 512 : 256) / wg, (ktiles + 7) / 8, (int64_t)64}));
  p.join_few = p.few && (p.S_few > 1 || mass);
  p.join_many = p.many && p.S_many > 1;
  const size_t qrows = (size_t)b.T * c.Hq;
  p.few_rows = p.many ? kFewRows : rows;
  const size_t frows = (size_t)heads * p.few_rows;
  if (p.join_many) {
    p.many_part = up256(p.S_many * qrows * kHeadDim * 4);
    p.many_ml = up256(p.S_many * qrows * sizeof(float2));
  }
  if (p.join_few) {
    p.few_part = up256(p.S_few * frows * kHeadDim * 4);
    p.few_ml = up256(p.S_few * frows * sizeof(float2));
  }
  if (mass && p.many) p.stat = up256(qrows * sizeof(float2));
  if (mass && p.few) {
    p.logit_stride = (int)(units * kUnit);
    p.logit = up256(frows * p.logit_stride * 4);
  }
  return p;
}

template <int FMT>
hipError_t launch(const Plan& p, const AttnArgs& a, hipStream_t st) {
  const unsigned heads = (unsigned)(a.g.B * a.g.Hkv);
  if (p.few) paged_few_kernel<FMT><<<heads * p.S_few, kFewThreads, 0, st>>>(a);
  if (p.many) {
    const unsigned wg = heads * p.row_tiles * p.S_many;
    if (p.waves == 4) paged_many_kernel<FMT, 4><<<wg, 256, 0, st>>>(a, a.g.table, p.row_tiles);
    else paged_many_kernel<FMT, 8><<<wg, 512, 0, st>>>(a, a.g.table, p.row_tiles);
  }
  const bool mass = a.mass_mode != HYQ_MASS_NONE;
  if (p.join_few) {
    const unsigned keys = mass ? (unsigned)((p.n_kv + kMassKeys - 1) / kMassKeys) : 0u;
    paged_few_finish_kernel<<<dim3(heads, kFewRows + keys), kFinishThreads, 0, st>>>(a);
  }
  if (p.join_many) paged_join_kernel<<<(unsigned)(a.g.T * a.g.Hq), kJoinThreads, 0, st>>>(a);
  if (p.many && mass)
    paged_many_mass_kernel<FMT><<<dim3(heads, (unsigned)((p.n_kv + 127) / 128)), kMassThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

bool paged_grid_fits(const hyq_pcache& c, const hyq_pbatch& b) {
  const Plan p = plan_of(c, b, HYQ_MASS_NONE);
  return (int64_t)b.B * c.Hkv * p.row_tiles * p.S_many <= (int64_t)1 << 22;
}

size_t paged_ws_bytes(const hyq_pcache& c, const hyq_pbatch& b, int mass) {
  return plan_of(c, b, mass).total();
}

hipError_t launch_paged_attn(const hyq_pcache& c, const hyq_pbatch& b, const uint16_t* q,
                             float softmax_scale, int mass, void* out, int out_dtype, void* ws,
                             hipStream_t st) {
  const Plan p = plan_of(c, b, mass);
  AttnArgs a = {};
  a.g = paged_geom(c, b);
  a.k = static_cast<const uint8_t*>(c.k);
  a.v = static_cast<const uint8_t*>(c.v);
  a.ks = c.k_scale;
  a.vs = c.v_scale;
  a.mass = c.mass;
  a.q = q;
  a.out = out;
  a.out_bf16 = out_dtype;
  a.mass_mode = mass;
  a.inv_g = (uint32_t)((((uint64_t)1 << 32) + a.g.g - 1) / a.g.g);
  a.c_log2 = softmax_scale * 1.44269504088896340736f;
  a.few_max = p.few_max;
  a.S_few = p.S_few;
  a.S_many = p.S_many;
  a.join_few = p.join_few;
  char* w = static_cast<char*>(ws);
  auto take = [&w](size_t n) {
    char* at = n ? w : nullptr;
    w += n;
    return at;
  };
  a.many_part = reinterpret_cast<float*>(take(p.many_part));
  a.many_ml = reinterpret_cast<float2*>(take(p.many_ml));
  a.few_part = reinterpret_cast<float*>(take(p.few_part));
  a.few_ml = reinterpret_cast<float2*>(take(p.few_ml));
  a.logit = reinterpret_cast<float*>(take(p.logit));
  a.stat = reinterpret_cast<float2*>(take(p.stat));
  a.few_rows = p.few_rows;
  a.logit_stride = p.logit_stride;
  if (c.bits_kv == 16) return launch<kBf16>(p, a, st);
  if (c.kv_format == HYQ_FMT_FP8) return launch<HYQ_FMT_FP8>(p, a, st);
  return launch<HYQ_FMT_INT>(p, a, st);
}

}  // namespace hyq
