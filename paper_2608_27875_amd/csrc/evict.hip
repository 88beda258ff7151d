// Eviction from a paged cache by accumulated attention weight: each KV head of
// each sequence keeps its last `recent` slots and, of the others, those with
// the largest mass, in ascending order, in new pages.
//
// Two launches.  The selection (one workgroup per KV head) reads 4 bytes a
// slot: the budget-th largest order key by three radix passes over a
// histogram in LDS, the keys held in registers, then the kept slots in order
// by ballots.  It is bound by latency (the passes follow each other).  The
// move copies the kept rows, 16 lanes to a row: HBM.
#include "paged_dev.h"

namespace hyq {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kChunk = kSelThreads * 4;   // slots of one float4 per thread
constexpr int kBins = 2048;
constexpr int kMoveThreads = 256, kMoveRows = kMoveThreads / 16;

struct EvictArgs {
  PagedGeom g;   // lens, table of the old pages; max_new unused
  const int32_t* new_table;
  int new_pages;
  int budget, recent, row_bytes;
  uint8_t *k, *v;
  float *ks, *vs, *mass;
  int32_t *keep, *new_lens;
};

__device__ __forceinline__ int slots_of(const EvictArgs& a, int b) {
  const int64_t cap = (int64_t)a.g.max_pages << a.g.page_log2;
  return (int)min((int64_t)min(max(a.g.lens[b], 0), a.g.max_len), cap);
}

// Order keys of the four slots from n0 on (n0 a multiple of 4, so in one
// page): recent slots above every mass, NaN and missing pages below.
__device__ __forceinline__ void keys4(const EvictArgs& a, int b, int j, int n0, int n, uint32_t (&k)[4]) {
  float4 m = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const int p = n0 < n ? page_of(a.g, b, n0) : -1;
  if (p >= 0) m = *reinterpret_cast<const float4*>(a.mass + pool_row(a.g, p, j, n0));
  const float f[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t u = p < 0 || f[e] != f[e] ? 0u : order_key(f[e]);
    k[e] = n0 + e >= n - a.recent ? 0xffffffffu : u;
  }
}

// C > 0: up to C chunks of slots, their keys in registers; C = 0: any number,
// read again for every pass.
template <int C>
__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(EvictArgs a) {
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t wsum[2][kSelWaves];
  __shared__ uint32_t found[2];   // bin, count above it
  const int bj = blockIdx.x, b = bj / a.g.Hkv, j = bj - b * a.g.Hkv;
  const int n = slots_of(a, b), m = min(n, a.budget);
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  int32_t* keep = a.keep + (size_t)bj * a.budget;
  for (int i = m + tid; i < a.budget; i += kSelThreads) keep[i] = HYQ_KQ_POS_PAD;
  if (j == 0 && tid == 0) a.new_lens[b] = m;
  if (n <= a.budget) {
    for (int i = tid; i < n; i += kSelThreads) keep[i] = i;
    return;
  }
  const int nc = (n + kChunk - 1) / kChunk;
  uint32_t key[C > 0 ? C : 1][4];
  if constexpr (C > 0) {
#pragma unroll
    for (int c = 0; c < C; ++c) keys4(a, b, j, c * kChunk + tid * 4, n, key[c]);
  }
  // body(c, keys of this thread's 4 slots, first of them)
  auto each = [&](auto body) {
    if constexpr (C > 0) {
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (c < nc) body(key[c], c * kChunk + tid * 4);
    } else {
      for (int c = 0; c < nc; ++c) {
        keys4(a, b, j, c * kChunk + tid * 4, n, key[0]);
        body(key[0], c * kChunk + tid * 4);
      }
    }
  };
  // the m-th largest key, bits from the top; `left` of the keys that share the
  // bits found so far are still wanted
  uint32_t prefix = 0, left = (uint32_t)m;
  int shift = 32;
  for (int pass = 0; pass < 3; ++pass) {
    const int bits = pass < 2 ? 11 : 10, below = shift - bits;
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = 0u;
    __syncthreads();
    each([&](const uint32_t (&k)[4], int n0) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (n0 + e < n && (pass == 0 || (k[e] >> shift) == prefix))
          atomicAdd(&hist[(k[e] >> below) & ((1u << bits) - 1)], 1u);
    });
    __syncthreads();
    // thread t takes the bins 2047 - 2t and 2046 - 2t: counts from the top
    const uint32_t c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
    uint32_t sum = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t up = __shfl_up(sum, o, 64);
      if (lane >= o) sum += up;
    }
    if (lane == 63) wsum[0][w] = sum;
    __syncthreads();
    for (int x = 0; x < w; ++x) sum += wsum[0][x];
    const uint32_t before = sum - c0 - c1;   // keys in higher bins
    if (before < left && sum >= left) {
      const bool second = before + c0 < left;
      found[0] = (uint32_t)(kBins - 1 - 2 * tid) - (second ? 1u : 0u);
      found[1] = before + (second ? c0 : 0u);
    }
    __syncthreads();
    prefix = (prefix << bits) | found[0];
    left -= found[1];
    shift = below;
    __syncthreads();
  }
  // slots in order: a kept one's place is the number of larger keys before it
  // plus the equal ones before it, of which the first `left` are kept
  uint32_t gt0 = 0, eq0 = 0;   // of all chunks before
  each([&](const uint32_t (&k)[4], int n0) {
    const uint64_t lower = (1ull << lane) - 1;
    uint32_t gt = 0, eq = 0, wgt = 0, weq = 0;
    bool is_gt[4], is_eq[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      is_gt[e] = n0 + e < n && k[e] > prefix;
      is_eq[e] = n0 + e < n && k[e] == prefix;
      const uint64_t bg = __ballot(is_gt[e]), be = __ballot(is_eq[e]);
      gt += __popcll(bg & lower);
      eq += __popcll(be & lower);
      wgt += __popcll(bg);
      weq += __popcll(be);
    }
    if (lane == 0) {
      wsum[0][w] = wgt;
      wsum[1][w] = weq;
    }
    __syncthreads();
    uint32_t all_gt = 0, all_eq = 0;
#pragma unroll
    for (int x = 0; x < kSelWaves; ++x) {
      const uint32_t g1 = wsum[0][x], e1 = wsum[1][x];
      if (x < w) {
        gt += g1;
        eq += e1;
      }
      all_gt += g1;
      all_eq += e1;
    }
    gt += gt0;
    eq += eq0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (is_gt[e] || (is_eq[e] && eq < left)) keep[gt + min(eq, left)] = n0 + e;
      gt += is_gt[e];
      eq += is_eq[e];
    }
    gt0 += all_gt;
    eq0 += all_eq;
    __syncthreads();
  });
}

// Workgroup (rows, bj): 16 kept rows at a time, 16 lanes to a row.  A row of a
// missing page becomes zero.
template <typename W>   // a lane's part of a row: uint4 (bf16) or uint2 (codes)
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(EvictArgs a) {
  const int bj = blockIdx.y, b = bj / a.g.Hkv, j = bj - b * a.g.Hkv;
  const int m = min(slots_of(a, b), a.budget);
  const int i = blockIdx.x * kMoveRows + (int)(threadIdx.x >> 4), sub = threadIdx.x & 15;
  if (i >= m) return;
  const int ni = i >> a.g.page_log2;
  const int np = a.new_table[(size_t)b * a.new_pages + ni];
  if ((unsigned)np >= (unsigned)a.g.n_pages) return;
  const int from = a.keep[(size_t)bj * a.budget + i];
  const int p = page_of(a.g, b, from);
  const size_t src = pool_row(a.g, max(p, 0), j, from), dst = pool_row(a.g, np, j, i);
  W kw = {}, vw = {};
  if (p >= 0) {
    kw = reinterpret_cast<const W*>(a.k + src * a.row_bytes)[sub];
    vw = reinterpret_cast<const W*>(a.v + src * a.row_bytes)[sub];
  }
  reinterpret_cast<W*>(a.k + dst * a.row_bytes)[sub] = kw;
  reinterpret_cast<W*>(a.v + dst * a.row_bytes)[sub] = vw;
  if (sub == 0) a.mass[dst] = p >= 0 ? a.mass[src] : 0.0f;
  if (a.ks && sub == 1) a.ks[dst] = p >= 0 ? a.ks[src] : 0.0f;
  if (a.vs && sub == 2) a.vs[dst] = p >= 0 ? a.vs[src] : 0.0f;
}

}  // namespace

hipError_t launch_evict(const hyq_pcache& c, int B, const int32_t* lens, const int32_t* table,
                        int max_pages, int max_len, int budget, int recent,
                        const int32_t* new_table, int new_pages, int32_t* keep, int32_t* new_lens,
                        hipStream_t st) {
  EvictArgs a = {};
  hyq_pbatch pb = {};
  pb.B = B;
  pb.max_len = max_len;
  pb.max_pages = max_pages;
  pb.lens = lens;
  pb.table = table;
  a.g = paged_geom(c, pb);
  a.new_table = new_table;
  a.new_pages = new_pages;
  a.budget = budget;
  a.recent = recent;
  a.row_bytes = c.bits_kv == 16 ? 2 * kHeadDim : kHeadDim;
  a.k = static_cast<uint8_t*>(c.k);
  a.v = static_cast<uint8_t*>(c.v);
  a.ks = c.bits_kv == 16 ? nullptr : c.k_scale;
  a.vs = c.bits_kv == 16 ? nullptr : c.v_scale;
  a.mass = c.mass;
  a.keep = keep;
  a.new_lens = new_lens;
  const unsigned heads = (unsigned)(B * c.Hkv);
  const int chunks = (max_len + kChunk - 1) / kChunk;
  if (chunks <= 1) evict_select_kernel<1><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= 2) evict_select_kernel<2><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= 4) evict_select_kernel<4><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= 8) evict_select_kernel<8><<<heads, kSelThreads, 0, st>>>(a);
  else evict_select_kernel<0><<<heads, kSelThreads, 0, st>>>(a);
  const int rows = budget < max_len ? budget : max_len;
  if (rows > 0) {
    const dim3 grid((unsigned)((rows + kMoveRows - 1) / kMoveRows), heads);
    if (c.bits_kv == 16) evict_move_kernel<uint4><<<grid, kMoveThreads, 0, st>>>(a);
    else evict_move_kernel<uint2><<<grid, kMoveThreads, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace hyq
