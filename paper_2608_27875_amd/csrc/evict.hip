// Eviction from a paged cache by accumulated attention weight: each KV head of
// each sequence keeps its last `recent` slots and, of the others, those with
// the largest mass, in ascending order, in new pages.
//
// Two launches.  The selection (one workgroup per KV head) reads 4 bytes a
// slot: the budget-th largest order key by radix passes over a histogram in LDS,
// three at most (usually two: the budget then ends with a bin), the keys held in
// registers, then the kept slots in order by lane scans.  It is bound by latency:
// 17 us for 32k slots, of which 8 until the keys are there, 2 and 1.5 in the two
// passes, 3 to place; 10 us for 8k.  Above 32768 slots every pass and the placement
// read the keys again: 131072 slots to 2048 take 62 to 64 us with the move.  The
// move copies the kept rows, 16 lanes to a row: HBM, 16 x 8 x 1000 E4M3 rows in
// 15 us (4.6 TB/s).
#include "paged_dev.h"

namespace hyq {
namespace {

constexpr int kSelThreads = 1024, kSelWaves = kSelThreads / 64;
constexpr int kChunk = kSelThreads * 4;   // slots of one float4 per thread
constexpr int kBins = 2048, kCopies = 4;
constexpr int kMaxHeld = 8;   // chunks whose keys fit the registers
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

// Inclusive sum over the lanes of a wave (row shifts, then the last lanes of
// rows 0 and 2 into rows 1 and 3, then of the lower half into the upper).
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, false);
  x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, false);
  return x;
}

// Wave w holds 256 C consecutive slots of each group of C chunks, lane l the
// four from 256 c + 4 l on for every c (one group unless there are more slots
// than kMaxHeld chunks; their keys are then read again for every pass).  Order
// keys: recent slots above every mass; NaN, missing pages and slots past the
// last below (those are the last equals, and m <= n of them are taken).
template <int C, bool MORE>
__global__ void __launch_bounds__(kSelThreads)
evict_select_kernel(EvictArgs a) {
  // kCopies counts of each bin, by lane: masses crowd into few exponents, and
  // equal bins of a wave are added one after the other
  __shared__ uint4 hist[kBins];
  __shared__ uint32_t wsum[kSelWaves];
  __shared__ uint32_t found[3];   // bin, keys above it, keys in it
  uint32_t* const h32 = reinterpret_cast<uint32_t*>(hist);
  const int bj = blockIdx.x, b = bj / a.g.Hkv, j = bj - b * a.g.Hkv;
  const int n = slots_of(a, b), m = min(n, a.budget);
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  int32_t* keep = a.keep + (size_t)bj * a.budget;
  // unsigned: i may pass 2^31 where a budget is near it
  for (uint32_t i = (uint32_t)(m + tid); i < (uint32_t)a.budget; i += kSelThreads) keep[i] = HYQ_KQ_POS_PAD;
  if (j == 0 && tid == 0) a.new_lens[b] = m;
  if (n <= a.budget) {
    for (int i = tid; i < n; i += kSelThreads) keep[i] = i;
    return;
  }
  const int groups = MORE ? (n + C * kChunk - 1) / (C * kChunk) : 1;
  uint32_t key[C * 4];
  float4 f[C];
  int p[C];
  auto fetch = [&](int grp) {
    const int n0 = (grp * kSelWaves + w) * C * 256 + lane * 4;
#pragma unroll
    for (int c = 0; c < C; ++c) {   // 4 slots from a multiple of 4 on: one page
      p[c] = page_of(a.g, b, n0 + 256 * c);
      f[c] = *reinterpret_cast<const float4*>(a.mass + pool_row(a.g, max(p[c], 0), j, n0 + 256 * c));
    }
  };
  auto convert = [&](int grp) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int first = ((grp * kSelWaves + w) * C + c) * 256;   // of the wave's slots
      const float x[4] = {f[c].x, f[c].y, f[c].z, f[c].w};
#pragma unroll
      for (int e = 0; e < 4; ++e) key[4 * c + e] = p[c] < 0 || x[e] != x[e] ? 0u : order_key(x[e]);
      if (first + 256 > n - a.recent) {   // the same for the whole wave, rarely
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int slot = first + lane * 4 + e;
          if (slot >= n - a.recent) key[4 * c + e] = slot < n ? 0xffffffffu : 0u;
        }
      }
    }
  };
  if (!MORE) fetch(0);
  // the m-th largest key, bits from the top; `left` of the keys that share the
  // bits found so far are still wanted
  uint32_t prefix = 0, left = (uint32_t)m;
  int shift = 32;
  bool whole = false;   // all keys that share them are
  for (int pass = 0; pass < 3 && !whole; ++pass) {
    const int bits = pass < 2 ? 11 : 10, below = shift - bits;
    for (int i = tid; i < kBins; i += kSelThreads) hist[i] = make_uint4(0u, 0u, 0u, 0u);
    __syncthreads();
    if (!MORE && pass == 0) convert(0);
    for (int grp = 0; grp < groups; ++grp) {
      if (MORE) {
        fetch(grp);
        convert(grp);
      }
#pragma unroll
      for (int e = 0; e < 4 * C; ++e)
        if (pass == 0 || (key[e] >> shift) == prefix)
          atomicAdd(&h32[((key[e] >> below) & ((1u << bits) - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
    }
    __syncthreads();
    // thread t takes the bins 2047 - 2t and 2046 - 2t: counts from the top
    const uint4 u0 = hist[kBins - 1 - 2 * tid], u1 = hist[kBins - 2 - 2 * tid];
    const uint32_t c0 = u0.x + u0.y + u0.z + u0.w, c1 = u1.x + u1.y + u1.z + u1.w;
    uint32_t sum = wave_scan(c0 + c1);
    if (lane == 63) wsum[w] = sum;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kSelWaves; ++x) sum += x < w ? wsum[x] : 0u;
    const uint32_t before = sum - c0 - c1;   // keys in higher bins
    if (before < left && sum >= left) {
      const bool second = before + c0 < left;
      found[0] = (uint32_t)(kBins - 1 - 2 * tid) - (second ? 1u : 0u);
      found[1] = before + (second ? c0 : 0u);
      found[2] = second ? c1 : c0;
    }
    __syncthreads();
    prefix = (prefix << bits) | (uint32_t)__builtin_amdgcn_readfirstlane((int)found[0]);
    left -= (uint32_t)__builtin_amdgcn_readfirstlane((int)found[1]);
    whole = (uint32_t)__builtin_amdgcn_readfirstlane((int)found[2]) == left;
    shift = below;
  }
  // Counts of the lane's four slots per chunk, three chunks to a word (a wave's
  // are at most 256), are scanned over the lanes.
  constexpr int kWords = (C + 2) / 3;
  auto field = [](uint32_t x, int c) { return (x >> (10 * (c % 3))) & 1023u; };
  // Usually all keys that share the threshold's bits are kept: places are then
  // counts of keys that are not below it.
  if (whole) {
    uint32_t least = prefix << shift;
    uint32_t kept0 = 0;   // of all groups before
    for (int grp = 0; grp < groups; ++grp) {
      if (MORE) {
        fetch(grp);
        convert(grp);
      }
      uint32_t cnt[kWords] = {}, scan[kWords], kept = 0, before[C];
#pragma unroll
      for (int c = 0; c < C; ++c) {
        uint32_t own = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) own += key[4 * c + e] >= least;
        cnt[c / 3] += own << (10 * (c % 3));
      }
#pragma unroll
      for (int x = 0; x < kWords; ++x) scan[x] = wave_scan(cnt[x]);
#pragma unroll
      for (int c = 0; c < C; ++c) {
        before[c] = kept + field(scan[c / 3] - cnt[c / 3], c);
        kept += field(__builtin_amdgcn_readlane((int)scan[c / 3], 63), c);
      }
      if (lane == 0) wsum[w] = kept;
      __syncthreads();
      uint32_t lower = kept0;
#pragma unroll
      for (int x = 0; x < kSelWaves; ++x) {
        const uint32_t v = wsum[x];
        lower += x < w ? v : 0u;
        kept0 += v;
      }
      const int n0 = (grp * kSelWaves + w) * C * 256 + lane * 4;
      asm volatile("" : "+s"(least));   // compare again: the masks of all keys do not fit
#pragma unroll
      for (int c = 0; c < C; ++c) {
        uint32_t at = lower + before[c];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (key[4 * c + e] >= least) keep[at++] = n0 + 256 * c + e;
      }
      __syncthreads();
    }
    return;
  }
  // Otherwise (all 32 bits are found) a kept slot's place is the number of larger
  // keys before it plus the equal ones before it, of which the first `left` are kept.
  uint32_t gt0 = 0, eq0 = 0;   // of all groups before
  for (int grp = 0; grp < groups; ++grp) {
    if (MORE) {
      fetch(grp);
      convert(grp);
    }
    uint32_t gw[kWords] = {}, ew[kWords] = {}, gs[kWords], es[kWords];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        gw[c / 3] += key[4 * c + e] > prefix ? 1u << (10 * (c % 3)) : 0u;
        ew[c / 3] += key[4 * c + e] == prefix ? 1u << (10 * (c % 3)) : 0u;
      }
    uint32_t all_g = 0, all_e = 0, before_g[C], before_e[C];
#pragma unroll
    for (int x = 0; x < kWords; ++x) {
      gs[x] = wave_scan(gw[x]);
      es[x] = wave_scan(ew[x]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) {
      before_g[c] = all_g + field(gs[c / 3] - gw[c / 3], c);
      before_e[c] = all_e + field(es[c / 3] - ew[c / 3], c);
      all_g += field(__builtin_amdgcn_readlane((int)gs[c / 3], 63), c);
      all_e += field(__builtin_amdgcn_readlane((int)es[c / 3], 63), c);
    }
    if (lane == 0) wsum[w] = all_g | all_e << 16;   // a group holds at most 2^15 slots
    __syncthreads();
    uint32_t lower = 0, all = 0;
#pragma unroll
    for (int x = 0; x < kSelWaves; ++x) {
      const uint32_t v = wsum[x];
      lower += x < w ? v : 0u;
      all += v;
    }
    const int n0 = (grp * kSelWaves + w) * C * 256 + lane * 4;
    asm volatile("" : "+s"(prefix));
#pragma unroll
    for (int c = 0; c < C; ++c) {
      uint32_t gt = gt0 + (lower & 0xffffu) + before_g[c], eq = eq0 + (lower >> 16) + before_e[c];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool is_gt = key[4 * c + e] > prefix, is_eq = key[4 * c + e] == prefix;
        if (is_gt || (is_eq && eq < left)) keep[gt + min(eq, left)] = n0 + 256 * c + e;
        gt += is_gt;
        eq += is_eq;
      }
    }
    gt0 += all & 0xffffu;
    eq0 += all >> 16;
    __syncthreads();
  }
}

// Workgroup (rows, bj): 16 lanes to a row, kMoveEach rows in flight per lane.
// A row of a missing page becomes zero.
constexpr int kMoveEach = 4;
template <typename W>   // a lane's part of a row: uint4 (bf16) or uint2 (codes)
__global__ void __launch_bounds__(kMoveThreads)
evict_move_kernel(EvictArgs a) {
  const int bj = blockIdx.y, b = bj / a.g.Hkv, j = bj - b * a.g.Hkv;
  const int m = min(slots_of(a, b), a.budget);
  const int i0 = blockIdx.x * (kMoveRows * kMoveEach) + (int)(threadIdx.x >> 4), sub = threadIdx.x & 15;
  if (i0 >= m) return;
  size_t src[kMoveEach], dst[kMoveEach];
  bool there[kMoveEach], take[kMoveEach];
#pragma unroll
  for (int e = 0; e < kMoveEach; ++e) {
    const int i = i0 + e * kMoveRows, at = min(i, m - 1);
    const int np = a.new_table[(size_t)b * a.new_pages + (at >> a.g.page_log2)];
    const int from = a.keep[(size_t)bj * a.budget + at];
    const int p = page_of(a.g, b, from);
    there[e] = p >= 0;
    take[e] = i < m && (unsigned)np < (unsigned)a.g.n_pages;
    src[e] = pool_row(a.g, max(p, 0), j, from);
    dst[e] = pool_row(a.g, take[e] ? np : 0, j, at);
  }
  W kw[kMoveEach], vw[kMoveEach];
  // lanes 0, 1, 2 also carry the row's mass and scales
  float* side = sub == 0 ? a.mass : sub == 1 ? a.ks : sub == 2 ? a.vs : nullptr;
  float f[kMoveEach];
#pragma unroll
  for (int e = 0; e < kMoveEach; ++e) {
    kw[e] = reinterpret_cast<const W*>(a.k + src[e] * a.row_bytes)[sub];
    vw[e] = reinterpret_cast<const W*>(a.v + src[e] * a.row_bytes)[sub];
    f[e] = side ? side[src[e]] : 0.0f;
  }
#pragma unroll
  for (int e = 0; e < kMoveEach; ++e) {
    if (!take[e]) continue;
    reinterpret_cast<W*>(a.k + dst[e] * a.row_bytes)[sub] = there[e] ? kw[e] : W{};
    reinterpret_cast<W*>(a.v + dst[e] * a.row_bytes)[sub] = there[e] ? vw[e] : W{};
    if (side) side[dst[e]] = there[e] ? f[e] : 0.0f;
  }
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
  if (chunks <= 1) evict_select_kernel<1, false><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= 2) evict_select_kernel<2, false><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= 4) evict_select_kernel<4, false><<<heads, kSelThreads, 0, st>>>(a);
  else if (chunks <= kMaxHeld) evict_select_kernel<kMaxHeld, false><<<heads, kSelThreads, 0, st>>>(a);
  else evict_select_kernel<kMaxHeld, true><<<heads, kSelThreads, 0, st>>>(a);
  const int rows = budget < max_len ? budget : max_len;
  if (rows > 0) {
    const dim3 grid((unsigned)((rows + kMoveRows * kMoveEach - 1) / (kMoveRows * kMoveEach)), heads);
    if (c.bits_kv == 16) evict_move_kernel<uint4><<<grid, kMoveThreads, 0, st>>>(a);
    else evict_move_kernel<uint2><<<grid, kMoveThreads, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace hyq
