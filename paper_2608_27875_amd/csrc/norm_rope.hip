// Per-head RMS norms of queries and keys and the position rotation in one
// pass over a projection's rows, into the dense tensors of the prefill and
// decode calls or into the pages of a cache.
//
//   y = x w / sqrt(mean(x^2) + eps);  (a, c) -> (a cos - c sin, c cos + a sin)
//
// Every row (256 bytes) is read once and written once, about ten operations
// an element: bound by HBM, and by latency where there are few tokens.
//   - 16 lanes hold a row, 8 channels (16 bytes) each, so the mean is a
//     reduction over 16 lanes, the partner of a half-split pair sits
//     rot_dim/16 lanes away, and that of an interleaved pair in the same lane;
//   - the angles of a token are shared by all its heads: rot_dim/2 threads of
//     the workgroup take one sine and cosine each into LDS.  The product
//     pos * inv_freq is taken in float64 and reduced to a turn there (a float32
//     angle is off by radians from positions of a few million on), the sine
//     and cosine in float32;
//   - one rounding: everything between the loads and the stores is float32
//     (float64 for rows whose squares leave its range).
// 65516 tokens of 56 rows (1.9 GB) take 338 us (5.6 TB/s); 8192 of 48 rows (201
// MB) 44 us where inputs change from pass to pass (4.6 TB/s) and 34 where they
// stay in the last-level cache; 16 tokens 3.6 us; 2106 tokens of a ragged batch
// into bf16 pages 13.1 us, int8 15.1, E4M3 14.3 to 14.8 (3.3 TB/s; latency).
// Loading a lane's rows of all passes up front was slower (40.8 us at 8192
// tokens): the arithmetic, about 150 instructions per 4 rows of a wave, is as
// tight as HBM.
#include "paged_dev.h"
#include "quant_dev.h"

namespace hyq {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRowsPerPass = kRopeThreads / 16;   // head rows a workgroup takes at once

struct RopeArgs {
  RopeRows x;
  const uint16_t *qw, *kw;
  const float* inv_freq;
  int rot, interleaved;
  float eps;
  int T, Hq, Hkv;
  // dense outputs: [B][H][L][D], token t = b * L + i
  uint16_t *Q, *K, *V;
  int L;
  // paged outputs (Q then holds q_out [T][Hq][D])
  PagedGeom g;
  uint8_t *pk, *pv;
  float *pks, *pvs, *mass;
};

// x of the lane `N` places on in the same 16 (cyclic).
template <int N>
__device__ __forceinline__ float rotate16(float x) {
  return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xf, 0xf, false));
}
// Sum and maximum over a row's 16 lanes, the same bits in each.
__device__ __forceinline__ float sum16(float v) {
  v += rotate16<8>(v);
  v += rotate16<4>(v);
  v += rotate16<2>(v);
  return v + rotate16<1>(v);
}
__device__ __forceinline__ float max16(float v) {
  v = fmaxf(v, rotate16<8>(v));
  v = fmaxf(v, rotate16<4>(v));
  v = fmaxf(v, rotate16<2>(v));
  return fmaxf(v, rotate16<1>(v));
}

__device__ __forceinline__ void widen8(const uint4& w, float (&x)[8]) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = bf16_lo(u[e]);
    x[2 * e + 1] = bf16_hi(u[e]);
  }
}

// Whether a row's mean square (with eps) is below 2^-100 or infinite: squares of
// its entries may then have left float32's range.
__device__ __forceinline__ bool squares_lost(float ms) {
  constexpr uint32_t kLeast = 0x0d800000u, kInf = 0x7f800000u;   // bits of 2^-100 and infinity
  return __float_as_uint(ms) - kLeast >= kInf - kLeast;
}

// The norm of such a row in float64, which holds the square of every float.  A
// row of zeros stays zero without eps too: a dead head or padding must not put
// NaN into a page.  The row's 16 lanes call it together.  Never taken in earnest;
// to ask costs an append of 2106 tokens 0.4 us of 14.
__device__ __forceinline__ void norm_wide(float (&x)[8], const uint4& raw, const float (&w)[8], float eps) {
  widen8(raw, x);
  double ss = 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) ss += (double)x[e] * (double)x[e];
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) ss += __shfl_xor(ss, o, 16);
  const double ms = ss * (1.0 / kHeadDim) + (double)eps;
  const double inv = ms > 0.0 ? 1.0 / sqrt(ms) : 0.0;
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = (float)((double)x[e] * inv * (double)w[e]);
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  const v2bf r = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, r);
}

// Eight codes of x / s (s > 0), one per byte; the correctly rounded quotient.
template <int FMT>
__device__ __forceinline__ void codes8f(const float (&x)[8], float s, float c, uint32_t (&o)[2]) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = x[4 * h + e] / s;
    if constexpr (FMT == HYQ_FMT_FP8) {   // two conversions fill the word
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = fminf(fmaxf(y[e], -448.0f), 448.0f);
      int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
      v = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true);
      o[h] = (uint32_t)v;
    } else {
      uint32_t v = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) v |= (uint32_t)(code_int(y[e], c) & 0xff) << (8 * e);
      o[h] = v;
    }
  }
}

// PAGES: 0 dense outputs, 16 bf16 pages, 8 pages of codes FMT.  Workgroup
// (t, c): token t, head rows [16c * passes, 16(c + 1) * passes).
template <int PAGES, int FMT>
__global__ void __launch_bounds__(kRopeThreads)
norm_rope_kernel(RopeArgs a, int passes) {
  __shared__ float2 cs[kHeadDim / 2];
  const int t = blockIdx.x;
  const int sub = threadIdx.x & 15;
  int slot = 0, page = -1;
  if (PAGES) {
    const int b = seq_of_token(a.g, t);
    const int i = b < 0 ? 0 : t - max(a.g.cu[b], 0);
    if (b < 0 || i >= a.g.max_new) return;   // nobody's row
    const int64_t n = (int64_t)min(max(a.g.lens[b], 0), a.g.max_len) + i;
    if (n < ((int64_t)a.g.max_pages << a.g.page_log2)) {
      slot = (int)n;
      page = page_of(a.g, b, slot);
    }
  }
  if ((int)threadIdx.x < a.rot / 2) {
    const double turns = (double)a.x.pos[t] * (double)a.inv_freq[threadIdx.x] *
                         0.15915494309189533576888;   // 1 / (2 pi)
    float s, c;
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    cs[threadIdx.x] = make_float2(c, s);
  }
  __syncthreads();
  const int rows = a.Hq + 2 * a.Hkv;
  // dense outputs: rows of sequence b = t / L
  size_t q_at = (size_t)t * a.Hq, kv_at = 0;
  int L = 1;
  if (PAGES == 0) {
    const int b = t / a.L, i = t - b * a.L;
    L = a.L;
    q_at = (size_t)b * a.Hq * L + i;
    kv_at = (size_t)b * a.Hkv * L + i;
  }
  for (int p = 0; p < passes; ++p) {
    const int r = (blockIdx.y * passes + p) * kRowsPerPass + (int)(threadIdx.x >> 4);
    const bool is_q = r < a.Hq, is_v = r >= a.Hq + a.Hkv;
    const int h = is_q ? r : is_v ? r - a.Hq - a.Hkv : r - a.Hq;
    const uint16_t* src = is_q ? a.x.q : is_v ? a.x.v : a.x.k;
    const bool live = r < rows && src != nullptr && (PAGES == 0 || is_q || page >= 0);
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (live) {
      const int64_t stride = is_q ? a.x.q_stride : is_v ? a.x.v_stride : a.x.k_stride;
      raw = reinterpret_cast<const uint4*>(src + (size_t)t * stride + h * kHeadDim)[sub];
    }
    float x[8];
    widen8(raw, x);
    uint4 o = raw;   // values are copied as they are
    if (__ballot(!is_v)) {   // a wave of value rows has nothing to work out
      const uint16_t* w = is_q ? a.qw : a.kw;
      if (w && !is_v) {
        uint4 wr = reinterpret_cast<const uint4*>(w)[sub];
        float ss = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) ss = __builtin_fmaf(x[e], x[e], ss);
        ss = sum16(ss);
        const float ms = ss * (1.0f / kHeadDim) + a.eps;
        const float inv = 1.0f / sqrtf(ms);
        float wf[8];
        widen8(wr, wf);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] *= inv * wf[e];
        if (__builtin_expect(__ballot(squares_lost(ms)) != 0, 0)) {
          if (squares_lost(ms)) norm_wide(x, raw, wf, a.eps);
        }
      }
      if (a.interleaved) {
        if (!is_v && sub * 8 < a.rot) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = cs[sub * 4 + e];
            const float u = x[2 * e], v = x[2 * e + 1];
            x[2 * e] = u * f.x - v * f.y;
            x[2 * e + 1] = v * f.x + u * f.y;
          }
        }
      } else {
        const int half = a.rot >> 4;   // lanes of the first half of the pairs
        const bool second = sub >= half;
        const bool turned = !is_v && sub < 2 * half;
        float y[8];   // the other entries of this lane's pairs
        if (half == 8) {
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = rotate16<8>(x[e]);
        } else {
          const int lane = threadIdx.x & 63;
          const int mate = turned ? (second ? lane - half : lane + half) : lane;
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = __shfl(x[e], mate, 64);
        }
        if (turned) {
          const float sign = second ? 1.0f : -1.0f;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 f = cs[(second ? sub - half : sub) * 8 + e];
            x[e] = x[e] * f.x + y[e] * (sign * f.y);
          }
        }
      }
      if (!is_v)
        o = make_uint4(pack2(x[0], x[1]), pack2(x[2], x[3]), pack2(x[4], x[5]), pack2(x[6], x[7]));
    }
    if (PAGES == 0 || is_q) {
      uint16_t* dst = is_q ? a.Q : is_v ? a.V : a.K;
      const size_t row = (is_q ? q_at : kv_at) + (size_t)h * L;
      if (live) reinterpret_cast<uint4*>(dst + row * kHeadDim)[sub] = o;
    } else {
      const size_t row = pool_row(a.g, max(page, 0), min(h, a.Hkv - 1), slot);
      if (PAGES == 16) {
        if (live) reinterpret_cast<uint4*>((is_v ? a.pv : a.pk) + row * kHeadDim * 2)[sub] = o;
      } else {
        constexpr float C = code_bound<8, FMT>();
        float m = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[e]));
        const float s = max16(m) / C;
        uint32_t cw[2] = {0u, 0u};
        if (s > 0.0f) codes8f<FMT>(x, s, C, cw);
        if (live) {
          reinterpret_cast<uint2*>((is_v ? a.pv : a.pk) + row * kHeadDim)[sub] =
              make_uint2(cw[0], cw[1]);
          if (sub == 0) (is_v ? a.pvs : a.pks)[row] = s;
        }
      }
      if (live && !is_v && sub == 0 && a.mass) a.mass[row] = 0.0f;
    }
  }
}

template <int PAGES, int FMT>
hipError_t launch(const RopeArgs& a, hipStream_t st) {
  const int groups = (a.Hq + 2 * a.Hkv + kRowsPerPass - 1) / kRowsPerPass;
  // A token's rows go to several workgroups where there are few tokens (16
  // tokens of 48 rows: 3.7 us in 48 workgroups, 5.5 in 16); otherwise one takes
  // them all and works out the angles once.
  const int passes = (int64_t)a.T * groups <= 1024 ? 1 : groups;
  norm_rope_kernel<PAGES, FMT>
      <<<dim3((unsigned)a.T, (unsigned)((groups + passes - 1) / passes)), kRopeThreads, 0, st>>>(a, passes);
  return hipGetLastError();
}

RopeArgs rope_args(const hyq_rope& r, const RopeRows& x, int T, int Hq, int Hkv) {
  RopeArgs a = {};
  a.x = x;
  a.qw = static_cast<const uint16_t*>(r.q_weight);
  a.kw = static_cast<const uint16_t*>(r.k_weight);
  a.inv_freq = r.inv_freq;
  a.rot = r.rot_dim;
  a.interleaved = r.interleaved;
  a.eps = r.eps;
  a.T = T;
  a.Hq = Hq;
  a.Hkv = Hkv;
  return a;
}

}  // namespace

hipError_t launch_norm_rope(const hyq_shape& s, const hyq_rope& r, const RopeRows& x, uint16_t* Q,
                            uint16_t* K, uint16_t* V, hipStream_t st) {
  RopeArgs a = rope_args(r, x, s.B * s.L, s.Hq, s.Hkv);
  a.Q = Q;
  a.K = K;
  a.V = V;
  a.L = s.L;
  return launch<0, HYQ_FMT_INT>(a, st);
}

hipError_t launch_paged_append(const hyq_pcache& c, const hyq_pbatch& b, const hyq_rope& r,
                               const RopeRows& x, uint16_t* q_out, hipStream_t st) {
  RopeArgs a = rope_args(r, x, b.T, c.Hq, c.Hkv);
  a.Q = q_out;
  a.g = paged_geom(c, b);
  a.pk = static_cast<uint8_t*>(c.k);
  a.pv = static_cast<uint8_t*>(c.v);
  a.pks = c.k_scale;
  a.pvs = c.v_scale;
  a.mass = c.mass;
  if (c.bits_kv == 16) return launch<16, HYQ_FMT_INT>(a, st);
  if (c.kv_format == HYQ_FMT_FP8) return launch<8, HYQ_FMT_FP8>(a, st);
  return launch<8, HYQ_FMT_INT>(a, st);
}

}  // namespace hyq
