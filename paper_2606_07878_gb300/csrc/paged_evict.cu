// Eviction from a paged cache: of every sequence and KV-head the first `sinks` slots, the last
// `recent` and the heaviest of the others, `keep` in all, move to pages of their own, in their
// order.
//
// Two launches. The first one chooses: weights become 32-bit keys in their order (slots that stay
// in any case above all others, NaN below), and three steps of 11, 11 and 10 bits find the smallest
// key that is kept and how many of its equals are (those of the lowest slots). A cluster of CTAs
// takes a sequence's KV-head, each a part of its slots whose keys stay in shared memory where they
// fit; a step's histograms are added up through distributed shared memory, by every CTA for itself.
// The second one moves: 16 bytes a thread, rows of K and V.
//
// 131,072 slots of 8 KV-heads of 128 channels to 16,384 take 49 us, 24 to choose and 22 to move
// (134 MB, 6.2 TB/s); 32 sequences of 700 to 1,500 slots of 2 heads to 164 take 13 to 15. What is left of
// the choice is latency: the reads of pages and weights (4.8 us; 16 slots a thread, four reads on
// their way; one slot at a time took 40 us for the choice) and three rounds of histograms (count,
// wait for the cluster, read eight histograms, 3 to 4 us each). Sums over warps and CTAs by a lane
// each instead of one after another: 33 -> 24 us.
//
// A head may keep other tokens than its neighbour: a slot's rows of two heads are of two tokens
// then. Attention does not mind, keys are rotated to their positions already.
#include <algorithm>

#include "launch.cuh"
#include "paged_dev.cuh"

namespace still {

namespace {

constexpr int kChooseThreads = 1024;
constexpr int kChooseWarps = kChooseThreads / 32;
static_assert(kChooseWarps == 32, "a lane a warp");
constexpr int kDigits = 2048;
constexpr int kChooseCluster = 8;
constexpr int kChooseKeys = 48 * 1024;  // of a CTA in shared memory
constexpr int kChooseBytes = kChooseKeys * 4;

STILL_DEV uint32_t key_of(float w) {
  if (w != w) return 0;                                        // NaN
  const uint32_t x = __float_as_uint(w + 0.f);                 // -0 is 0
  return x & 0x80000000u ? ~x : x | 0x80000000u;
}

STILL_DEV uint2 ld_cluster_u32x2(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared::cluster.v2.u32 {%0, %1}, [%2];"
               : "=r"(v.x), "=r"(v.y)
               : "r"(addr)
               : "memory");
  return v;
}
// What the warps before this one have, of kChooseWarps = 32.
STILL_DEV uint32_t sum_before(const uint32_t* of_warp, int warp) {
  const int lane = threadIdx.x & 31;
  return __reduce_add_sync(0xffffffffu, lane < warp ? of_warp[lane] : 0u);
}

template <int kCluster>
__global__ void __launch_bounds__(kChooseThreads, 1)
    paged_choose_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedEvict f,
                        int in_smem) {
  extern __shared__ __align__(16) uint32_t keys[];
  __shared__ __align__(8) uint32_t hist[2][kDigits];
  __shared__ uint32_t warp_sum[kChooseWarps], warp_equal[kChooseWarps];
  __shared__ uint32_t found[2];   // digit, kept among those above it
  __shared__ __align__(8) uint32_t counts[2];  // of this CTA: above the smallest key, equal to it
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = kCluster > 1 ? cluster_ctarank() : 0;
  const int set = blockIdx.x / kCluster, b = set / a.H, h = set % a.H;
  const Seq s = paged_seq(a, b);
  const int count = min(s.len, f.keep);
  int32_t* kept = f.kept + ((int64_t)b * a.H + h) * f.keep;
  for (int64_t r = (int64_t)count + rank * kChooseThreads + threadIdx.x; r < f.keep;
       r += kCluster * kChooseThreads)
    kept[r] = -1;
  if (h == 0 && rank == 0 && threadIdx.x == 0) {
    f.to_len[b] = count;
    if (f.to_offset != nullptr)
      f.to_offset[b] = (a.pos_offset != nullptr ? a.pos_offset[b] : 0) + s.len - count;
  }
  if (s.len <= f.keep) {  // (of the whole cluster)
    for (int64_t r = rank * kChooseThreads + threadIdx.x; r < count;
         r += kCluster * kChooseThreads)
      kept[r] = (int)r;
    return;
  }
  const int32_t* table = a.table + (int64_t)b * a.s_table;
  // slots [j0, j1) of this CTA (unsigned, as loops step past an end that may be 2^31 - 256)
  using Slot = uint32_t;
  const Slot len = s.len;
  const Slot per = ((len + kCluster - 1) / kCluster + 31) & ~31u;
  const Slot j0 = min(len, rank * per), j1 = min(len, j0 + per);
  // Keys of four slots from j (a multiple of 4) on: they lie in one page.
  auto read = [&](Slot j) {
    uint32_t k[4] = {0, 0, 0, 0};
    const int pg = paged_page(a, table, j);
    const float* at = f.weight + ((((int64_t)max(pg, 0) * a.H + h) << a.page_shift) +
                                  (j & ((1 << a.page_shift) - 1)));
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e >= j1) continue;
      const bool stays = j + e < (Slot)f.sinks || j + e >= len - f.recent;
      k[e] = stays ? 0xffffffffu : pg < 0 ? 0 : key_of(at[e]);
    }
    return make_uint4(k[0], k[1], k[2], k[3]);
  };
  const bool held = j1 - j0 <= (Slot)in_smem;
  uint4* const keys4 = reinterpret_cast<uint4*>(keys);
  auto four = [&](Slot j) { return held ? keys4[(j - j0) / 4] : read(j); };
  for (int i = threadIdx.x; i < kDigits; i += kChooseThreads) hist[0][i] = 0;
  __syncthreads();
  uint32_t prefix = 0;       // the digits found so far, in place
  uint32_t need = f.keep;    // to be kept among the keys that have them
#pragma unroll 1
  for (int step = 0; step < 3; ++step) {
    const int shift = step == 0 ? 21 : step == 1 ? 10 : 0;
    const uint32_t digits = step == 2 ? 1024 : 2048;
    const uint32_t above = step == 0 ? 0u : ~0u << (step == 1 ? 21 : 10);
    uint32_t* const mine = hist[step & 1];
    auto count = [&](Slot j, const uint4& k) {
      const uint32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (j + e < j1 && (x[e] & above) == prefix)
          atomicAdd(&mine[(x[e] >> shift) & (digits - 1)], 1u);
    };
    if (step == 0) {  // several reads on their way at a time: page, weight
      constexpr int kAtOnce = 4;
      for (Slot j = j0 + 4 * threadIdx.x; j < j1; j += 4 * kAtOnce * kChooseThreads) {
        uint4 k[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const Slot x = j + 4 * i * kChooseThreads;
          if (x < j1) k[i] = read(x);
        }
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) {
          const Slot x = j + 4 * i * kChooseThreads;
          if (x >= j1) break;
          if (held) keys4[(x - j0) / 4] = k[i];
          count(x, k[i]);
        }
      }
    } else {
      for (Slot j = j0 + 4 * threadIdx.x; j < j1; j += 4 * kChooseThreads) count(j, four(j));
    }
    if constexpr (kCluster > 1)
      cluster_sync();
    else
      __syncthreads();
    // all CTAs' counts of two digits, this thread's; digits above them come first
    uint32_t c[2] = {0, 0};
    const int top = (int)digits - 1 - 2 * (int)threadIdx.x;  // c[0]: top, c[1]: top - 1
    if (top > 0) {
      uint2 x[kCluster];
#pragma unroll
      for (int r = 0; r < kCluster; ++r)
        x[r] = kCluster > 1 ? ld_cluster_u32x2(cluster_map(smem_u32(mine + top - 1), r))
                            : *reinterpret_cast<const uint2*>(mine + top - 1);
#pragma unroll
      for (int r = 0; r < kCluster; ++r) {
        c[0] += x[r].y;
        c[1] += x[r].x;
      }
    }
    uint32_t upto = c[0] + c[1];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    if (lane == 31) warp_sum[warp] = upto;
    for (int i = threadIdx.x; i < kDigits; i += kChooseThreads) hist[(step + 1) & 1][i] = 0;
    __syncthreads();
    upto += sum_before(warp_sum, warp);
    const uint32_t before = upto - c[0] - c[1];
    if (before < need && upto >= need) {
      const bool first = before + c[0] >= need;
      found[0] = first ? top : top - 1;
      found[1] = first ? before : before + c[0];
    }
    __syncthreads();
    prefix |= found[0] << shift;
    need -= found[1];
    // (the other histogram is written next; nobody reads this one again before the next sync of
    // all)
  }
  // ---- the kept slots, in order: keys above `prefix`, and the first `need` that equal it
  // (counts of both in one word, 16 bits each: a warp has 128 slots at a time)
  const Slot each = ((j1 - j0 + kChooseWarps - 1) / kChooseWarps + 127) & ~127u;
  const Slot w0 = min(j1, j0 + warp * each), w1 = min(j1, w0 + each);
  auto tally = [&](Slot j, const uint4& k) {
    uint32_t n = 0;
    const uint32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (j + e < w1) n += x[e] > prefix ? 1u : x[e] == prefix ? 0x10000u : 0u;
    return n;
  };
  uint32_t more = 0, equal = 0;
  for (Slot j = w0 + 4 * lane; j < w1; j += 128) {
    const uint32_t n = tally(j, four(j));
    more += n & 0xffffu;
    equal += n >> 16;
  }
  more = __reduce_add_sync(0xffffffffu, more);
  equal = __reduce_add_sync(0xffffffffu, equal);
  if (lane == 0) {
    warp_sum[warp] = more;
    warp_equal[warp] = equal;
  }
  __syncthreads();
  if (warp == 0) {
    const uint32_t x = __reduce_add_sync(0xffffffffu, warp_sum[lane]);
    const uint32_t y = __reduce_add_sync(0xffffffffu, warp_equal[lane]);
    if (lane == 0) {
      counts[0] = x;
      counts[1] = y;
    }
  }
  if constexpr (kCluster > 1)
    cluster_sync();
  else
    __syncthreads();
  // before this warp's slots: in the CTAs and in the warps before it
  uint2 ctas = make_uint2(0, 0);
  if (kCluster > 1 && lane < (int)rank)
    ctas = ld_cluster_u32x2(cluster_map(smem_u32(counts), lane));
  more = __reduce_add_sync(0xffffffffu, ctas.x) + sum_before(warp_sum, warp);
  equal = __reduce_add_sync(0xffffffffu, ctas.y) + sum_before(warp_equal, warp);
  for (Slot j0w = w0; j0w < w1; j0w += 128) {
    const Slot j = j0w + 4 * lane;
    const uint4 k = j < w1 ? four(j) : make_uint4(0, 0, 0, 0);
    const uint32_t n = tally(j, k);
    uint32_t upto = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += x;
    }
    const uint32_t all = __shfl_sync(0xffffffffu, upto, 31);
    uint32_t m = more + ((upto - n) & 0xffffu), q = equal + ((upto - n) >> 16);
    const uint32_t x[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (j + e >= w1) break;
      if (x[e] > prefix)
        kept[m++ + min(q, need)] = j + e;
      else if (x[e] == prefix && q++ < need)
        kept[m + q - 1] = j + e;
    }
    more += all & 0xffffu;
    equal += all >> 16;
  }
  if constexpr (kCluster > 1) cluster_sync();  // others may read this CTA's counts
}

// ----------------------------------------------------------------- moving
constexpr int kMoveThreads = 256;

template <int D>
__global__ void __launch_bounds__(kMoveThreads)
    paged_move_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedEvict f) {
  griddep_wait();
  constexpr int kPieces = D / 8;                       // of 16 bytes
  constexpr int kRows = kMoveThreads / kPieces;        // of K and V at a time
  const int c = threadIdx.x % kPieces * 8;
  const PagedArgs& t = f.to;
  const int mask = (1 << a.page_shift) - 1, to_mask = (1 << t.page_shift) - 1;
  const int64_t rows = (int64_t)a.B * f.keep * a.H;
  for (int64_t x = (int64_t)blockIdx.x * kRows + threadIdx.x / kPieces; x < rows;
       x += (int64_t)gridDim.x * kRows) {
    const int r = (int)(x / a.H % f.keep), h = (int)(x % a.H), b = (int)(x / a.H / f.keep);
    const int j = f.kept[((int64_t)b * a.H + h) * f.keep + r];
    if (j < 0) continue;
    const int pg = paged_page(a, a.table + (int64_t)b * a.s_table, j);
    const int to = paged_page(t, t.table + (int64_t)b * t.s_table, r);
    if (pg < 0 || to < 0) continue;
    const int64_t src = (int64_t)pg * a.s_page + (int64_t)(j & mask) * a.s_slot +
                        (int64_t)h * a.s_head + c;
    const int64_t dst = (int64_t)to * t.s_page + (int64_t)(r & to_mask) * t.s_slot +
                        (int64_t)h * t.s_head + c;
    const uint4 k = __ldcs(reinterpret_cast<const uint4*>(a.K + src));
    const uint4 v = __ldcs(reinterpret_cast<const uint4*>(a.V + src));
    *reinterpret_cast<uint4*>(t.K + dst) = k;
    *reinterpret_cast<uint4*>(t.V + dst) = v;
    if (c != 0) continue;
    const int64_t from = (((int64_t)pg * a.H + h) << a.page_shift) + (j & mask);
    const int64_t at = (((int64_t)to * a.H + h) << t.page_shift) + (r & to_mask);
    if (f.to_weight != nullptr) f.to_weight[at] = f.weight[from];
    if (t.beta != nullptr) t.beta[at] = a.beta != nullptr ? a.beta[from] : 0.f;
  }
}

template <int kCluster>
cudaError_t launch_choose(const PagedArgs& a, const PagedEvict& f, const KernelTable& dev,
                          cudaStream_t s) {
  using Id = KernelId<paged_choose_kernel<kCluster>, kChooseThreads, kChooseBytes, kCluster>;
  if (dev.of<Id>().status != cudaSuccess) return dev.of<Id>().status;
  const int64_t slots = ((int64_t)a.table_pages << a.page_shift) / kCluster + 64;
  const int keys = (int)std::min<int64_t>(kChooseKeys, slots);
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.B * a.H * kCluster));
  cfg.blockDim = dim3(kChooseThreads);
  cfg.dynamicSmemBytes = (size_t)keys * 4;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = kCluster > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, paged_choose_kernel<kCluster>, a, f, keys);
}

}  // namespace

cudaError_t launch_paged_evict(const PagedArgs& a, const PagedEvict& f, const KernelTable& dev,
                               cudaStream_t s) {
  // A CTA or a cluster for a sequence's KV-head, by the slots that the table has room for. Measured,
  // us for the call (64 slots kept, 8 KV-heads): one CTA 15 up to 4,000 slots, 19 at 8,000 and 23 at
  // 16,000, about 0.55 for 1,000 more; a cluster 21 at any of them, but a CTA fills an SM: 72 for 8
  // sequences (four waves of clusters, one CTA each 15 to 24) and 440 for 64 (38 to 52).
  const int64_t slots = (int64_t)a.table_pages << a.page_shift;
  const int64_t waves = ((int64_t)a.B * a.H * kChooseCluster + dev.num_sms - 1) / dev.num_sms;
  const cudaError_t e = slots > 38000 * waves - 25000 ? launch_choose<kChooseCluster>(a, f, dev, s)
                                                      : launch_choose<1>(a, f, dev, s);
  if (e != cudaSuccess) return e;
  auto kernel = a.d == 64    ? paged_move_kernel<64>
                : a.d == 128 ? paged_move_kernel<128>
                             : paged_move_kernel<256>;
  const int64_t rows = (int64_t)a.B * f.keep * a.H;
  const int64_t blocks = (rows * (a.d / 8) + kMoveThreads - 1) / kMoveThreads;
  return launch_chained(kernel, dim3((unsigned)std::min<int64_t>(blocks, 8 * dev.num_sms)),
                        dim3(kMoveThreads), 0, s, 1, a, f);
}

}  // namespace still
