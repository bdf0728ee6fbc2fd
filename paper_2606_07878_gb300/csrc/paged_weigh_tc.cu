// Attention weights added up over a paged cache for calls of many rows, on the tensor cores
// (tcgen05): both passes of
//
//   weight_j = decay weight_j + sum over rows r that see j of e^(s_rj - m_r) / l_r
//
// are one kernel. It holds two tiles of 128 of one side and streams tiles of the other past them:
//
//   pass 1   holds rows (tokens x heads of a KV-head), streams slots: a thread has a row, adds up
//            e^(s - m) over the slots and leaves (m, 1 / l)
//   pass 2   holds slots, streams rows: a thread has a slot and adds up e^(s - m) / l over the rows
//
// so that sums stay in a thread's registers in either, in a fixed order, and S (fp32, in TMEM) is
// read once. In pass 1 m is the row's maximum over its first tile, and moves only when a tile's sum
// passes 2^10: any m near the maximum serves, since the second pass divides by the same. Both
// passes compute e^(s - m) by the same instructions from the same S. Sums of a tile are added to
// the total with their rounding carried along (two floats).
//
// Without biases S itself is kept: e^(scale s - m) = 2^(fma(s, scale log2 e, -m log2 e)). With
// biases logits are natural up to the subtraction, as a bias of the lowest float would be -inf in
// units of log 2.
//
// A thread of the sums has a lane of both held tiles and a quarter of the columns: what belongs to
// a column (biases; m and l) is read from shared memory once for two values. With a thread to a
// lane of one held tile and m and 1 / l apart the second pass over 6,001 tokens of 28 heads took
// 212 us. So m and log l are one number there, where it is small enough that its rounding stays
// below 2^-20 of a weight: 149.
//
// Measured: 6,001 tokens of 28 query and 4 KV-heads of 128 channels, 117 us the first pass, 149 the
// second (129 GFLOP each: 1.1 and 0.87 PFLOP/s, the tensor pipe busy 51% and 44%); 64 tokens behind
// each of four sequences of 9,000 to 32,700 slots with biases, 55 and 76 (170 MB of keys, twice).
// What bounds both is the warps that add up: 0.9 us a streamed tile against 0.53 of products, 4.4
// instructions an exponential where the formula has 2, half the rest what a warp does once a tile
// (waits, masks, sums of two floats), and in short items 1 to 2 us from one item to the next.
// Tried without gain: four S tiles apart (a held tile each), a warp of its own for the held tiles'
// copies or for the items' ends, two warps for the columns, a deeper ring with one held item.
//
// Roles: warp 0 TMA (a box per page and 64 channels), 1 MMA issuer and TMEM, 2 what belongs to the
// streamed tile's columns and to held slots, 4 .. 19 sums. Ranges of equal cost as in the prefill
// (paged_tc.cuh); what several CTAs share of an item goes to the
// workspace and a second launch joins it. Every wait is bounded.
#include <type_traits>

#include "launch.cuh"
#include "paged_tc.cuh"

namespace still {

namespace {

constexpr int kWtThreads = 640;
constexpr int kWtSums = 16;          // warps that add up: four to a quarter of the columns
constexpr int kWtHeld = 256;        // rows or slots of an item
constexpr int kWtMost = 1024;       // a tile's sum in units of e^m that moves m
// Streamed tiles whose column values are held, [kWtCols][kWtColFloats]: three of every column, a
// flag, and of the tile that is an item's first the held slots' biases and pages.
constexpr int kWtCols = 4;
constexpr int kWtFlagAt = 384, kWtBiasAt = 388, kWtPageAt = kWtBiasAt + kWtHeld;
constexpr int kWtColFloats = kWtPageAt + kWtHeld / 8;  // (8 slots lie in one page)
constexpr float kWtFold = 32.f;     // |m + log2 l| below which they are one number

// An item of either pass: `x` counts blocks of 2 tile_tokens tokens or of 256 slots.
struct WtItem {
  int b, h, x;
  int first, count, len;  // of its sequence
  int k0, k1;             // streamed tiles [k0, k1) of those that it meets
  int part, last;         // as PfItem
};
struct WtRows {  // pass 1
  using Item = WtItem;
  int tokens;  // of an item
  STILL_DEV int items(const Seq& s) const { return pf_tiles(s, tokens); }
  STILL_DEV int tiles(const Seq& s, int x) const { return pf_slots(s, tokens, x); }
  STILL_DEV void fill(WtItem& it, const Seq& s, int x) const {
    it.x = x;
    it.first = s.first;
    it.count = s.count;
    it.len = s.len;
  }
};
// The first tile of tokens in which slot j is seen.
STILL_DEV int wt_first_tile(int count, int len, int j, int tokens) {
  return max(0, j - (len - count)) / tokens;
}
struct WtSlots {  // pass 2
  using Item = WtItem;
  int tokens;  // of a tile
  STILL_DEV int items(const Seq& s) const {
    return s.count > 0 ? (s.len + kWtHeld - 1) / kWtHeld : 0;
  }
  STILL_DEV int tiles(const Seq& s, int x) const {
    return pf_tiles(s, tokens) - wt_first_tile(s.count, s.len, x * kWtHeld, tokens);
  }
  STILL_DEV void fill(WtItem& it, const Seq& s, int x) const {
    WtRows{tokens}.fill(it, s, x);
  }
};

struct WtParams {
  PagedArgs a;
  PagedQuery q;
  int32_t tile_tokens = 0;     // floor(128 / g)
  float* weight = nullptr;
  float decay = 0.f;
  float2* part = nullptr;      // [2 x CTAs][256] (m, l), or (sum, 0)
  PfSplit* split = nullptr;    // [CTAs]; pass 2: token0 the sequence, tokens the block of slots
};

struct WtPlan {  // in shared memory
  PfStart start;
  WtItem shown[2];  // items n & 1
  int64_t warp_cost[kWtThreads / 32];
};

template <int D>
struct WtShape {
  static constexpr int kChunks = D / 64;               // of 64 channels
  static constexpr int kChunkBytes = 128 * 128;        // of a tile
  static constexpr int kHeldBufs = D <= 128 ? 2 : 1;   // items held at a time
  static constexpr int kHeldBytes = 2 * kChunks * kChunkBytes;
  static constexpr int kStages = D == 64 ? 8 : 5;      // a chunk of a streamed tile each
  static constexpr int kRing = kHeldBufs * kHeldBytes;
  static constexpr int kColAt = kRing + kStages * kChunkBytes;
  static constexpr int kXchAt = kColAt + kWtCols * kWtColFloats * 4;  // [3][256] float2
  static constexpr int kBarAt = kXchAt + 3 * kWtHeld * 8;
  static constexpr int kPlanAt = kBarAt + (2 * kStages + 2 * kWtCols + 13) * 8 + 16;
  static constexpr int kBytes = kPlanAt + sizeof(WtPlan);
  static_assert(kBytes <= 232448, "shared memory budget");
};

// A sum with the rounding of its additions beside it.
struct Sum2 {
  float s = 0.f, c = 0.f;
  STILL_DEV void add(float x) {
    const float y = x - c, t = s + y;
    c = t - s - y;
    s = t;
  }
};

template <int D, bool kBias, bool kSecond>
__global__ void __launch_bounds__(kWtThreads, 1)
    paged_weigh_tc_kernel(const __grid_constant__ CUtensorMap tm_q,
                          const __grid_constant__ CUtensorMap tm_k,
                          const __grid_constant__ WtParams f) {
  using S = WtShape<D>;
  using G = std::conditional_t<kSecond, WtSlots, WtRows>;
  constexpr int kStages = S::kStages, kChunks = S::kChunks;
  constexpr bool kCols = kBias || kSecond;
  extern __shared__ __align__(1024) uint8_t smem[];
  const int cta = blockIdx.x;
  griddep_wait();
  if (threadIdx.x == 0) f.split[cta].last = f.split[cta].first = cta;
  if ((smem_u32(smem) & 1023) != 0) {
    dev_set_error(f.a.err, DEV_BAD_ARG, 640);
    return;
  }
  WtPlan& plan = *reinterpret_cast<WtPlan*>(smem + S::kPlanAt);
  PfStart& start = plan.start;
  WtItem* shown = plan.shown;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBarAt);  // ring slot loaded
  uint64_t* empty = full + kStages;      // ring slot consumed
  uint64_t* colfull = empty + kStages;   // [kWtCols] column values written
  uint64_t* colfree = colfull + kWtCols; // [kWtCols] and read
  uint64_t* qfull = colfree + kWtCols;   // [2] item n & 1 shown and its held tiles loaded
  uint64_t* qfree = qfull + 2;           // [2] its last product complete
  uint64_t* seen = qfree + 2;            // [2] its record read by all
  uint64_t* sfull = seen + 2;            // [2] S of both held tiles, buffer i, complete
  uint64_t* sfree = sfull + 2;           // [2] and read
  uint64_t* xfull = sfree + 2;           // the other quarters' sums of an item
  uint64_t* xfree = xfull + 1;           // and read
  uint64_t* drain = xfree + 1;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kStages + 2 * kWtCols + 13) * 8 + 16 == S::kPlanAt - S::kBarAt, "barriers");

  const PagedArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = f.q.Hq / a.H;
  const int tile_rows = f.tile_tokens * g;
  const int mask = (1 << a.page_shift) - 1;
  const G items{kSecond ? f.tile_tokens : 2 * f.tile_tokens};

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < kWtCols; ++i) {
      mbar_init(&colfull[i], 1);
      mbar_init(&colfree[i], kWtSums);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&qfull[i], 1);
      mbar_init(&qfree[i], 1);
      mbar_init(&seen[i], kWtSums + 2);
      mbar_init(&sfull[i], 1);
      mbar_init(&sfree[i], kWtSums);
    }
    mbar_init(xfull, kWtSums - 4);
    mbar_init(xfree, 4);
    mbar_init(drain, 1);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
  }
  if (warp == 1) {
    tmem_alloc(tmem_slot, 512);
    tmem_relinquish();
  }
  // Rows of a ring slot that no box of tokens covers stay zeros.
  if constexpr (kSecond) {
    for (int s = 0; s < kStages; ++s)
      for (int x = tile_rows * 8 + (int)threadIdx.x; x < 1024; x += kWtThreads)
        reinterpret_cast<uint4*>(smem + S::kRing + s * S::kChunkBytes)[x] = make_uint4(0, 0, 0, 0);
    fence_proxy_async_smem();
  }
  pf_plan<kWtThreads>(a, items, cta, gridDim.x, start, plan.warp_cost, &f.split[cta]);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // Streamed tile k of an item, among all of its sequence.
  auto tile_of = [&](const WtItem& it, int k) {
    return kSecond
               ? wt_first_tile(it.count, it.len, it.x * kWtHeld, f.tile_tokens) + k
               : k;
  };
  // Whether the second held tile has anything.
  auto is_two = [&](const WtItem& it) {
    return kSecond ? it.len > it.x * kWtHeld + 128
                   : it.count > (2 * it.x + 1) * f.tile_tokens;
  };

  if (warp == 0) {
    // ------------------------------------------------------------ TMA producer
    int stage = 0, n_items = 0;
    uint32_t phase = 0;
    uint32_t armed = 0, armed_par = 0;  // stages whose copies were asked for, and their phases
    bool q_armed = false, bad = false;
    auto wait = [&](uint64_t* bar, uint32_t parity, int where) {
      if (!pf_wait(bar, parity, a.err, abort_flag, where)) bad = true;
      return !bad;
    };
    // The page of this lane's box of a tile of slots (8 at most); one outside the pool is zeros.
    const int box_bits = min(a.page_shift, 7), boxes = 128 >> box_bits;
    auto page_of = [&](const WtItem& it, int kt) {
      const int j = kt * 128 + (lane << box_bits);
      const int pg = lane < boxes && j < it.len
                         ? paged_page(a, a.table + (int64_t)it.b * a.s_table, j)
                         : -1;
      return pg < 0 ? a.n_pages : pg;
    };
    auto copy_slots = [&](uint8_t* dst, uint64_t* bar, const WtItem& it, int kt, int pg, int c) {
      if (lane < boxes)
        tma_load_4d(dst + (lane << box_bits) * 128, &tm_k, bar, c * 64,
                    (kt * 128 + (lane << box_bits)) & mask, it.h, pg);
    };
    auto copy_rows = [&](uint8_t* dst, uint64_t* bar, const WtItem& it, int tile, int c) {
      if (lane == 0)
        tma_load_3d(dst, &tm_q, bar, c * 64, it.h * g, it.first + tile * f.tile_tokens);
    };
    PfWalk walk(a, items, start);
    WtItem it;
    while (!bad && !warp_flag(abort_flag) && walk.next(it)) {
      if (it.k0 == it.k1) continue;  // its rows see nothing
      const int n = n_items & 1;
      if (n_items > 1 && !wait(&seen[n], ((n_items >> 1) - 1) & 1, 641)) break;
      const int held = S::kHeldBufs == 2 ? n : 0;
      if (S::kHeldBufs == 2) {
        if (n_items > 1 && !wait(&qfree[n], ((n_items >> 1) - 1) & 1, 642)) break;
      } else {
        if (n_items > 0 && !wait(&qfree[n ^ 1], ((n_items - 1) >> 1) & 1, 643)) break;
      }
      if (lane == 0) {
        shown[n] = it;
        if (it.part == 2) {
          PfSplit& sp = f.split[cta];
          sp.last = it.last;
          sp.token0 = kSecond ? it.b : it.first + it.x * 2 * f.tile_tokens;
          sp.tokens = kSecond ? it.x : min(2 * f.tile_tokens, it.count - it.x * 2 * f.tile_tokens);
          sp.h = it.h;
        }
        mbar_arrive_expect_tx(&qfull[n],
                              2 * kChunks * (kSecond ? S::kChunkBytes : tile_rows * 128));
      }
      __syncwarp();
      for (int t = 0; t < 2; ++t) {
        const int pg = kSecond ? page_of(it, 2 * it.x + t) : 0;
        for (int c = 0; c < kChunks; ++c) {
          uint8_t* const dst = smem + held * S::kHeldBytes + (t * kChunks + c) * S::kChunkBytes;
          if constexpr (kSecond)
            copy_slots(dst, &qfull[n], it, 2 * it.x + t, pg, c);
          else
            copy_rows(dst, &qfull[n], it, 2 * it.x + t, c);
        }
      }
      q_armed = true;
      ++n_items;
      int pg = kSecond ? 0 : page_of(it, it.k0);
#pragma unroll 1
      for (int k = it.k0; k < it.k1 && !bad; ++k) {
        const int tile = tile_of(it, k);
        const int next_pg = !kSecond && k + 1 < it.k1 ? page_of(it, k + 1) : 0;
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
          if (!wait(&empty[stage], phase ^ 1, 644)) break;
          if (lane == 0)
            mbar_arrive_expect_tx(&full[stage], kSecond ? tile_rows * 128 : S::kChunkBytes);
          armed |= 1u << stage;
          armed_par = (armed_par & ~(1u << stage)) | (phase << stage);
          __syncwarp();
          uint8_t* const dst = smem + S::kRing + stage * S::kChunkBytes;
          if constexpr (kSecond)
            copy_rows(dst, &full[stage], it, tile, c);
          else
            copy_slots(dst, &full[stage], it, tile, pg, c);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        pg = next_pg;
      }
    }
    // The CTA may leave only when nothing is on its way into its shared memory: the last arrivals
    // of the issuer's commits, or copies that nobody waited for.
    if (lane == 0 && !bad) {
      for (int i = 0; i < kStages && !bad && !*abort_flag; ++i) {
        if (!mbar_wait(&empty[stage], phase ^ 1)) {
          dev_set_error(a.err, DEV_WAIT_TIMEOUT, 645);
          *abort_flag = 1;
          bad = true;
        }
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1;
        }
      }
      for (int n = max(0, n_items - 2); n < n_items && !bad && !*abort_flag; ++n)
        if (!mbar_wait(&qfree[n & 1], (n >> 1) & 1)) {
          dev_set_error(a.err, DEV_WAIT_TIMEOUT, 646);
          *abort_flag = 1;
          bad = true;
        }
      if (n_items > 1 && !bad && !*abort_flag &&
          !mbar_wait(&seen[n_items & 1], ((n_items >> 1) - 1) & 1)) {
        dev_set_error(a.err, DEV_WAIT_TIMEOUT, 647);
        *abort_flag = 1;
      }
      if (!*abort_flag) {  // no more items
        shown[n_items & 1].k0 = shown[n_items & 1].k1 = 0;
        mbar_arrive(&qfull[n_items & 1]);
      }
    }
    if (lane == 0) {
      if (bad || *abort_flag) {
        for (int s = 0; s < kStages; ++s)
          if (armed & (1u << s)) (void)mbar_wait(&full[s], (armed_par >> s) & 1);
        if (q_armed) (void)mbar_wait(&qfull[(n_items - 1) & 1], ((n_items - 1) >> 1) & 1);
      }
    }
  } else if (warp == 1 && elect_one()) {
    // ------------------------------------------------------------ MMA issuer
    constexpr uint32_t idesc = idesc_f16(128, 128, 1);
    int stage = 0;
    uint32_t phase = 0;
    uint32_t uses = 0;  // of the buffers of S
    bool bad = false, issued = false;
    auto wait = [&](uint64_t* bar, uint32_t parity, int where) {
      if (mbar_wait(bar, parity)) return true;
      dev_set_error(a.err, DEV_WAIT_TIMEOUT, where);
      *abort_flag = 1;
      bad = true;
      return false;
    };
    const uint64_t held_desc = sdesc_k_sw128(smem_u32(smem));
    const uint64_t ring_desc = sdesc_k_sw128(smem_u32(smem + S::kRing));
    constexpr uint64_t kStep = S::kChunkBytes >> 4;
    for (uint32_t n = 0; !bad && !*abort_flag; ++n) {
      if (!wait(&qfull[n & 1], (n >> 1) & 1, 651)) break;
      const WtItem& it = shown[n & 1];
      const int n_k = it.k1 - it.k0;
      const bool two = is_two(it);
      mbar_arrive(&seen[n & 1]);
      if (n_k < 1) break;
      const uint64_t held =
          held_desc + (S::kHeldBufs == 2 ? n & 1 : 0) * (uint64_t)(S::kHeldBytes >> 4);
#pragma unroll 1
      for (int k = 0; k < n_k && !bad; ++k) {
        if (!wait(&sfree[uses & 1], ((uses >> 1) & 1) ^ 1, 652)) break;
#pragma unroll 1
        for (int c = 0; c < kChunks; ++c) {
          if (!wait(&full[stage], phase, 654)) break;
          tc_fence_after();
          const uint64_t b = ring_desc + stage * kStep;
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (t == 1 && !two) break;
            const uint64_t x = held + (t * kChunks + c) * kStep;
#pragma unroll
            for (int e = 0; e < 4; ++e)
              tc_mma_f16(tmem_base + (2 * t + (uses & 1)) * 128, x + 2 * e, b + 2 * e, idesc,
                         c + e > 0);
          }
          issued = true;
          tc_commit(&empty[stage]);
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        if (bad) break;
        tc_commit(&sfull[uses & 1]);
        ++uses;
      }
      if (!bad) tc_commit(&qfree[n & 1]);
    }
    if ((bad || *abort_flag) && issued) {
      tc_commit(drain);
      (void)mbar_wait(drain, 0);
    }
  } else if (warp == 2) {
    // ------------------------------------------------------------ what belongs to columns
    // Lane i: columns 4 i .. 4 i + 3.
    uint32_t uses = 0;
    bool bad = false;
    for (uint32_t n = 0; !bad && !warp_flag(abort_flag); ++n) {
      if (!pf_wait(&qfull[n & 1], (n >> 1) & 1, a.err, abort_flag, 661)) break;
      const WtItem it = shown[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&seen[n & 1]);
      if (it.k1 <= it.k0) break;
      if constexpr (kCols) {
        // held slots, of which lane i has those from 8 i on: one page
        int page = -1;
        float beta[8];
        if constexpr (kSecond) {
          const int j = it.x * kWtHeld + 8 * lane;
          if (j < it.len) page = paged_page(a, a.table + (int64_t)it.b * a.s_table, j);
          const float* at =
              a.beta + ((((int64_t)max(page, 0) * a.H + it.h) << a.page_shift) + (j & mask));
#pragma unroll
          for (int e = 0; e < 8; ++e) beta[e] = kBias && page >= 0 && j + e < it.len ? at[e] : 0.f;
        }
        float v[4], w[4];
        auto load = [&](int k) {
          const int tile = tile_of(it, k);
          if constexpr (kSecond) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int c = 4 * lane + e, token = tile * f.tile_tokens + c / g;
              float2 x = make_float2(0.f, 0.f);
              if (c < tile_rows && token < it.count && token >= it.count - it.len)
                x = f.q.ml[(int64_t)(it.first + token) * f.q.Hq + it.h * g + c % g];
              v[e] = x.x;
              w[e] = x.y;
            }
          } else {
            const int j = tile * 128 + 4 * lane;
            const int pg = j < it.len ? paged_page(a, a.table + (int64_t)it.b * a.s_table, j) : -1;
            const float* at =
                a.beta + ((((int64_t)max(pg, 0) * a.H + it.h) << a.page_shift) + (j & mask));
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = pg >= 0 && j + e < it.len ? at[e] : -INFINITY;
          }
        };
        load(it.k0);
#pragma unroll 1
        for (int k = it.k0; k < it.k1; ++k, ++uses) {
          const int i = uses % kWtCols;
          if (!pf_wait(&colfree[i], ((uses / kWtCols) & 1) ^ 1, a.err, abort_flag, 662)) {
            bad = true;
            break;
          }
          float* const at = reinterpret_cast<float*>(smem + S::kColAt) + kWtColFloats * i;
          float4* const at4 = reinterpret_cast<float4*>(at) + lane;
          bool odd = false;  // the tile's general form is needed
          if constexpr (kSecond) {
            float by[4], sum[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              // a row that sees nothing, or none at all: e^-inf
              const bool none = w[e] == 0.f;
              const float log_l = kBias ? -logf(w[e]) : -log2f(w[e]);
              by[e] = none ? -INFINITY : -v[e];
              sum[e] = none ? -INFINITY : -(v[e] + log_l);
              odd |= !none && !(fabsf(sum[e]) < (kBias ? kWtFold / kLog2e : kWtFold));
            }
            at4[0] = make_float4(by[0], by[1], by[2], by[3]);
            at4[32] = make_float4(w[0], w[1], w[2], w[3]);
            at4[64] = make_float4(sum[0], sum[1], sum[2], sum[3]);
            if (k == it.k0) {
              float4* const b4 = reinterpret_cast<float4*>(at + kWtBiasAt + 8 * lane);
              b4[0] = make_float4(beta[0], beta[1], beta[2], beta[3]);
              b4[1] = make_float4(beta[4], beta[5], beta[6], beta[7]);
              at[kWtPageAt + lane] = __int_as_float(page);
            }
          } else {
            at4[0] = make_float4(v[0], v[1], v[2], v[3]);
#pragma unroll
            for (int e = 0; e < 4; ++e) odd |= v[e] == -INFINITY;
          }
          odd = __any_sync(0xffffffffu, odd);
          if (lane == 0) at[kWtFlagAt] = odd ? 1.f : 0.f;
          if (k + 1 < it.k1) load(k + 1);
          __syncwarp();
          if (lane == 0) mbar_arrive(&colfull[i]);
        }
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ sums
    const int c0 = 32 * ((warp - 4) >> 2);     // columns [c0, c0 + 32)
    const int row = (warp & 3) * 32 + lane;    // of both held tiles
    const uint32_t lanes = tmem_base + ((uint32_t)((warp & 3) * 32) << 16) + c0;
    float2* const xch = reinterpret_cast<float2*>(smem + S::kXchAt) + row;  // [3][2][128]
    const float k_log2 = f.q.scale * kLog2e;
    const float unit = kBias ? kLog2e : 1.f;  // of m, in log 2
    const uint64_t sc = pack2(f.q.scale, f.q.scale);
    const uint64_t k2 = kBias ? pack2(kLog2e, kLog2e) : pack2(k_log2, k_log2);
    uint32_t uses = 0;  // of S, and of the columns' values
    bool bad = false;
    auto wait_all = [&](uint64_t* bar, uint32_t parity, int where) -> bool {
      if (!pf_wait(bar, parity, a.err, abort_flag, where)) bad = true;
      return !bad;
    };
    for (uint32_t n = 0; !bad && !warp_flag(abort_flag); ++n) {
      if (!wait_all(&qfull[n & 1], (n >> 1) & 1, 671)) break;
      const WtItem it = shown[n & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&seen[n & 1]);
      if (it.k1 <= it.k0) break;
      const int past = it.len - it.count;
      // pass 1: rows, the slots that they see; pass 2: slots
      bool valid[2];
      int see[2], page[2] = {-1, -1};
      float beta[2] = {0.f, 0.f}, before[2] = {0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int token = (2 * it.x + t) * f.tile_tokens + row / g;
        valid[t] = !kSecond && row < tile_rows && token < it.count;
        see[t] = valid[t] ? max(0, past + token + 1) : INT32_MAX;
      }
      const int least = kSecond ? 0 : __reduce_min_sync(0xffffffffu, min(see[0], see[1]));
      const int slot0 = it.x * kWtHeld + row;  // the other one 128 behind
      Sum2 sum[2];
      float m[2] = {-INFINITY, -INFINITY};
#pragma unroll 1
      for (int k = it.k0; k < it.k1; ++k, ++uses) {
        const int tile = tile_of(it, k);
        const int i = uses % kWtCols;
        const float* const cols =
            reinterpret_cast<const float*>(smem + S::kColAt) + kWtColFloats * i + c0;
        bool odd = false;
        if constexpr (kCols) {
          if (!wait_all(&colfull[i], (uses / kWtCols) & 1, 672)) break;
          odd = cols[kWtFlagAt - c0] != 0.f;
          if (kSecond && k == it.k0) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              beta[t] = cols[kWtBiasAt - c0 + 128 * t + row];
              page[t] = __float_as_int(cols[kWtPageAt - c0 + 16 * t + row / 8]);
              const int slot = slot0 + 128 * t;
              if (slot >= it.len) page[t] = -1;
              if (c0 == 0 && it.part == 0 && f.decay != 0.f && page[t] >= 0 && slot < past)
                before[t] = f.weight[(((int64_t)page[t] * a.H + it.h) << a.page_shift) +
                                     (slot & mask)];
            }
          }
        }
        if (!wait_all(&sfull[uses & 1], (uses >> 1) & 1, 673)) break;
        tc_fence_after();
        const uint32_t s_at = lanes + (uses & 1) * 128;
        // 16 columns of both tiles
        auto issue = [&](int c, uint32_t* v) {
          tmem_ld16_issue(s_at + c, v);
          tmem_ld16_issue(s_at + 256 + c, v + 16);
        };
        // Four columns of tile t: S, with biases logits; -inf where a row does not see the slot.
        auto logits = [&](auto masked, const uint32_t* v, int t, int c, const float4& b4,
                          uint64_t (&x)[2]) {
          x[0] = pack2(__uint_as_float(v[0]), __uint_as_float(v[1]));
          x[1] = pack2(__uint_as_float(v[2]), __uint_as_float(v[3]));
          if constexpr (kBias) {
            x[0] = fma2(x[0], sc, kSecond ? pack2(beta[t], beta[t]) : pack2(b4.x, b4.y));
            x[1] = fma2(x[1], sc, kSecond ? pack2(beta[t], beta[t]) : pack2(b4.z, b4.w));
          }
          if constexpr (!kSecond && decltype(masked)::value) {
            float u[4];
            unpack2(x[0], u[0], u[1]);
            unpack2(x[1], u[2], u[3]);
            const int upto = see[t] - tile * 128 - c0 - c;
            const float b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
              u[e] = e < upto && !(kBias && b[e] == -INFINITY) ? u[e] : -INFINITY;
            x[0] = pack2(u[0], u[1]);
            x[1] = pack2(u[2], u[3]);
          }
        };
        // e^(s + by), two at a time
        auto weights = [&](uint64_t x, uint64_t by2) {
          float u0, u1;
          unpack2(kBias ? mul2(add2(x, by2), k2) : fma2(x, k2, by2), u0, u1);
          return pack2(ex2_ftz(u0), ex2_ftz(u1));
        };
        auto pass = [&](auto f4) {  // all 32 columns
#pragma unroll
          for (int c = 0; c < 32; c += 16) {
            uint32_t v[32];
            issue(c, v);
            tmem_wait_ld();
            tmem_landed(v);
#pragma unroll
            for (int e = 0; e < 16; e += 4) f4(c + e, v + e);
          }
        };
        auto column4 = [&](int at) { return *reinterpret_cast<const float4*>(cols + at); };
        float x[2];
        if constexpr (!kSecond) {
          auto top = [&]() {  // of both rows, in units of m
            x[0] = x[1] = -INFINITY;
            pass([&](int c, const uint32_t* v) {
              const float4 b4 = kBias ? column4(c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                uint64_t y[2];
                float u[4];
                logits(std::true_type(), v + 16 * t, t, c, b4, y);
                unpack2(y[0], u[0], u[1]);
                unpack2(y[1], u[2], u[3]);
                x[t] = max3(max3(x[t], u[0], u[1]), u[2], u[3]);
              }
            });
#pragma unroll
            for (int t = 0; t < 2; ++t)
              if (!kBias && x[t] != -INFINITY) x[t] *= k_log2;
          };
          auto add_up = [&](auto masked) {
            uint64_t by2[2], s0[2] = {0ull, 0ull}, s1[2] = {0ull, 0ull};
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const float by = m[t] == -INFINITY ? 0.f : -m[t];  // nothing seen yet: 2^-inf
              by2[t] = pack2(by, by);
            }
            pass([&](int c, const uint32_t* v) {
              const float4 b4 = kBias ? column4(c) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                uint64_t y[2];
                logits(masked, v + 16 * t, t, c, b4, y);
                s0[t] = add2(s0[t], weights(y[0], by2[t]));
                s1[t] = add2(s1[t], weights(y[1], by2[t]));
              }
            });
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              float x0, x1;
              unpack2(add2(s0[t], s1[t]), x0, x1);
              x[t] = x0 + x1;
            }
          };
          const bool masked = odd || least < tile * 128 + c0 + 32;
          bool moves = (valid[0] && m[0] == -INFINITY) || (valid[1] && m[1] == -INFINITY);
#pragma unroll 1
          for (int i = 0; i < 2; ++i) {
            if (__any_sync(0xffffffffu, moves)) {
              top();
#pragma unroll
              for (int t = 0; t < 2; ++t)
                if (x[t] > m[t]) {
                  const float down = ex2_ftz((m[t] - x[t]) * unit);
                  sum[t].s *= down;
                  sum[t].c *= down;
                  m[t] = x[t];
                }
            }
            if (masked)
              add_up(std::true_type());
            else
              add_up(std::false_type());
            moves = (valid[0] && !(x[0] <= kWtMost)) || (valid[1] && !(x[1] <= kWtMost));
            if (!__any_sync(0xffffffffu, moves)) break;
          }
        } else {
          // columns [lo, hi) are rows that see the first slot (of old slots, which all rows see, lo is
          // held back: times g it may pass 32 bits)
          const int token0 = tile * f.tile_tokens;
          const int lo = max(slot0 - past - token0, -kWtHeld) * g - c0;
          const int hi = min(f.tile_tokens, it.count - token0) * g - c0;
          uint64_t s0[2] = {0ull, 0ull}, s1[2] = {0ull, 0ull};
          if (!odd && hi + c0 == tile_rows &&
              !__any_sync(0xffffffffu, lo + 128 * g > 0)) {
            pass([&](int c, const uint32_t* v) {
              const float4 b4 = column4(256 + c);
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                uint64_t y[2];
                logits(std::false_type(), v + 16 * t, t, c, b4, y);
                s0[t] = add2(s0[t], weights(y[0], pack2(b4.x, b4.y)));
                s1[t] = add2(s1[t], weights(y[1], pack2(b4.z, b4.w)));
              }
            });
          } else {
            pass([&](int c, const uint32_t* v) {
              const float4 b4 = column4(c), w4 = column4(128 + c);
#pragma unroll
              for (int t = 0; t < 2; ++t) {
                uint64_t y[2];
                float u[4];
                logits(std::false_type(), v + 16 * t, t, c, b4, y);
                // (a row of NaN counts where it is seen alone)
                unpack2(mul2(weights(y[0], pack2(b4.x, b4.y)), pack2(w4.x, w4.y)), u[0], u[1]);
                unpack2(mul2(weights(y[1], pack2(b4.z, b4.w)), pack2(w4.z, w4.w)), u[2], u[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  u[e] = c + e >= lo + 128 * t * g && c + e < hi ? u[e] : 0.f;
                s0[t] = add2(s0[t], pack2(u[0], u[1]));
                s1[t] = add2(s1[t], pack2(u[2], u[3]));
              }
            });
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            float x0, x1;
            unpack2(add2(s0[t], s1[t]), x0, x1);
            x[t] = x0 + x1;
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(&sfree[uses & 1]);
          if (kCols) mbar_arrive(&colfree[i]);
        }
        sum[0].add(x[0]);
        sum[1].add(x[1]);
      }
      if (bad) break;
      // ---- the quarters together, in their order
      if (c0 > 0) {
        if (n > 0 && !wait_all(xfree, (n - 1) & 1, 674)) break;
        xch[8 * c0 - 256] = make_float2(m[0], sum[0].s);
        xch[8 * c0 - 128] = make_float2(m[1], sum[1].s);
        __syncwarp();
        if (lane == 0) mbar_arrive(xfull);
        continue;
      }
      if (!wait_all(xfull, n & 1, 675)) break;
      float2 other[3][2];
#pragma unroll
      for (int i = 0; i < 3; ++i)
#pragma unroll
        for (int t = 0; t < 2; ++t) other[i][t] = xch[256 * i + 128 * t];
      __syncwarp();
      if (lane == 0) mbar_arrive(xfree);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int64_t part = (int64_t)(2 * cta + it.part - 1) * kWtHeld + 128 * t + row;
        if constexpr (kSecond) {
          const int slot = slot0 + 128 * t;
          const float sums = (sum[t].s + other[0][t].y) + (other[1][t].y + other[2][t].y);
          const float all = beta[t] == -INFINITY ? 0.f : sums;  // masked
          if (it.part != 0)
            f.part[part] = make_float2(all, 0.f);
          else if (page[t] >= 0)
            f.weight[(((int64_t)page[t] * a.H + it.h) << a.page_shift) + (slot & mask)] =
                f.decay * before[t] + all;
        } else {
          const float top =
              max3(fmaxf(m[t], other[0][t].x), other[1][t].x, other[2][t].x);
          auto brought = [&](float from, float x) {
            return from == top ? x : x * exp2f((from - top) * unit);
          };
          const float l = (brought(m[t], sum[t].s) + brought(other[0][t].x, other[0][t].y)) +
                          (brought(other[1][t].x, other[1][t].y) +
                           brought(other[2][t].x, other[2][t].y));
          const int token = (2 * it.x + t) * f.tile_tokens + row / g;
          if (it.part != 0)
            f.part[part] = make_float2(top, l);
          else if (valid[t])
            f.q.ml[(int64_t)(it.first + token) * f.q.Hq + it.h * g + row % g] =
                make_float2(top, l == 0.f ? 0.f : 1.f / l);
        }
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, 512);
  }
}

// The items that lie in several CTAs' ranges: block c joins the one that CTA c begins, its parts in
// the order of their ranges, a thread a row or slot.
template <bool kSecond>
__global__ void __launch_bounds__(kWtHeld)
    paged_weigh_join_kernel(const __grid_constant__ WtParams f, float unit) {
  griddep_wait();
  const int c = blockIdx.x;
  const PfSplit sp = f.split[c];
  if (sp.last <= c) return;
  const PagedArgs& a = f.a;
  const int g = f.q.Hq / a.H, r = threadIdx.x;
  auto part = [&](int i) { return f.part[(int64_t)(i == c ? 2 * c + 1 : 2 * i) * kWtHeld + r]; };
  if constexpr (kSecond) {
    const int b = sp.token0, slot = sp.tokens * kWtHeld + r;
    const Seq s = paged_seq<false>(a, b);
    if (slot >= s.len) return;
    const int pg = paged_page<false>(a, a.table + (int64_t)b * a.s_table, slot);
    if (pg < 0) return;
    Sum2 sum;
#pragma unroll 4
    for (int i = c; i <= sp.last; ++i) sum.add(part(i).x);
    float* const w = f.weight + (((int64_t)pg * a.H + sp.h) << a.page_shift) +
                     (slot & ((1 << a.page_shift) - 1));
    *w = (slot < s.len - s.count && f.decay != 0.f ? f.decay * *w : 0.f) + sum.s;
  } else {
    const int in = r & 127, token = (r >> 7) * f.tile_tokens + in / g;
    if (in >= f.tile_tokens * g || token >= sp.tokens) return;
    float m = -INFINITY;
#pragma unroll 4
    for (int i = c; i <= sp.last; ++i) m = fmaxf(m, part(i).x);
    Sum2 l;
#pragma unroll 4
    for (int i = c; i <= sp.last; ++i) {
      const float2 x = part(i);
      l.add(x.x == m ? x.y : x.y * exp2f((x.x - m) * unit));
    }
    f.q.ml[(int64_t)(sp.token0 + token) * f.q.Hq + sp.h * g + in % g] =
        make_float2(m, l.s == 0.f ? 0.f : 1.f / l.s);
  }
}

template <int D, bool kBias>
cudaError_t launch_passes(const PagedArgs& a, const PagedQuery& q, float* weight, float decay,
                          void* ws, const KernelTable& dev, cudaStream_t s) {
  using S = WtShape<D>;
  constexpr auto first = paged_weigh_tc_kernel<D, kBias, false>;
  constexpr auto second = paged_weigh_tc_kernel<D, kBias, true>;
  using First = KernelId<first, kWtThreads, S::kBytes>;
  using Second = KernelId<second, kWtThreads, S::kBytes>;
  if (dev.of<First>().status != cudaSuccess) return dev.of<First>().status;
  if (dev.of<Second>().status != cudaSuccess) return dev.of<Second>().status;
  const int ctas = dev.num_sms;
  WtParams f;
  f.a = a;
  f.q = q;
  f.tile_tokens = 128 / (q.Hq / a.H);
  f.weight = weight;
  f.decay = decay;
  f.part = static_cast<float2*>(ws);
  f.split = reinterpret_cast<PfSplit*>(f.part + (int64_t)2 * ctas * kWtHeld);
  CUtensorMap tq, tk;
  if (!query_tmap(&tq, a, q, f.tile_tokens) || !pool_tmap(&tk, a, a.K, 128))
    return cudaErrorInvalidValue;
  first<<<ctas, kWtThreads, S::kBytes, s>>>(tq, tk, f);
  cudaError_t e = cudaGetLastError();
  if (e == cudaSuccess)
    e = launch_chained(paged_weigh_join_kernel<false>, dim3(ctas), dim3(kWtHeld), 0, s, 1, f,
                       kBias ? kLog2e : 1.f);
  if (e == cudaSuccess)
    e = launch_chained(second, dim3(ctas), dim3(kWtThreads), S::kBytes, s, 1, tq, tk, f);
  if (e == cudaSuccess)
    e = launch_chained(paged_weigh_join_kernel<true>, dim3(ctas), dim3(kWtHeld), 0, s, 1, f, 1.f);
  return e;
}

}  // namespace

bool paged_weigh_tc_serves(const PagedArgs& a, int Hq) {
  // Measured, us, few rows' kernels / this one, 16 sequences of 5,000 slots and 4 KV-heads (256
  // channels: 2): 8 rows 55 / 65, 66 / 73, 59 / 67 for 64, 128, 256 channels; 16 rows 67 / 65,
  // 82 / 73, 82 / 67; 64 rows 169 / 65, 209 / 73, 207 / 67. Two of 60,000 slots (128 channels): 8 rows
  // 86 / 91, 16 rows 107 / 91. The mean is all the host has, as in paged_prefill_serves.
  return Hq / a.H <= 128 && paged_mean_rows(a, Hq) > 8;
}

size_t paged_weigh_tc_workspace(int num_sms) {
  return (size_t)num_sms * (2 * kWtHeld * sizeof(float2) + sizeof(PfSplit));
}

cudaError_t launch_paged_weigh_tc(const PagedArgs& a, const PagedQuery& q, float* weight,
                                  float decay, void* ws, const KernelTable& dev, cudaStream_t s) {
  auto run = [&](auto bias) {
    constexpr bool kBias = decltype(bias)::value;
    return a.d == 64    ? launch_passes<64, kBias>(a, q, weight, decay, ws, dev, s)
           : a.d == 128 ? launch_passes<128, kBias>(a, q, weight, decay, ws, dev, s)
                        : launch_passes<256, kBias>(a, q, weight, decay, ws, dev, s);
  };
  return a.beta != nullptr ? run(std::true_type()) : run(std::false_type());
}

}  // namespace still
