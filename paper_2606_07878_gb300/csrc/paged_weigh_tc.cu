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
// passes 2^10: any m near the maximum serves, since the second pass divides by the same. Both passes
// compute e^(s - m) by the same instructions from the same S. Sums of a tile are added to the total
// with their rounding carried along (two floats).
//
// Without biases S itself is kept: e^(scale s - m) = 2^(fma(s, scale log2 e, -m log2 e)). With biases
// logits are natural up to the subtraction, as a bias of the lowest float would be -inf in units of
// log 2.
//
// Roles: warp 0 TMA (a box per page and 64 channels), 1 MMA issuer and TMEM, 2 what belongs to the
// streamed tile's columns (biases; m and 1 / l), 4 .. 11 sums, four warps per held tile. Ranges of
// equal cost as in the prefill (paged_tc.cuh); what several CTAs share of an item goes to the
// workspace and a second launch joins it. Every wait is bounded.
#include <type_traits>

#include "launch.cuh"
#include "paged_tc.cuh"

namespace still {

namespace {

constexpr int kWtThreads = 384;
constexpr int kWtHeld = 256;        // rows or slots of an item
constexpr int kWtMost = 1024;       // a tile's sum in units of e^m that moves m
constexpr int kWtCols = 4;          // streamed tiles whose column values are held

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
  static constexpr int kColAt = kRing + kStages * kChunkBytes;  // [kWtCols][2][128] floats
  static constexpr int kBarAt = kColAt + kWtCols * 1024;
  static constexpr int kPlanAt = kBarAt + (2 * kStages + 2 * kWtCols + 15) * 8 + 16;
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
  uint64_t* sfull = seen + 2;            // [2][2] S of held tile t, buffer i, complete
  uint64_t* sfree = sfull + 4;           // [2][2] and read
  uint64_t* drain = sfree + 4;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * kStages + 2 * kWtCols + 15) * 8 + 16 == S::kPlanAt - S::kBarAt, "barriers");

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
      mbar_init(&colfree[i], 8);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&qfull[i], 1);
      mbar_init(&qfree[i], 1);
      mbar_init(&seen[i], 10);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&sfree[i], 4);
    }
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
    uint32_t uses[2] = {0, 0};  // of the held tiles
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
        if (!wait(&sfree[uses[0] & 1], ((uses[0] >> 1) & 1) ^ 1, 652)) break;
        if (two && !wait(&sfree[2 + (uses[1] & 1)], ((uses[1] >> 1) & 1) ^ 1, 653)) break;
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
              tc_mma_f16(tmem_base + (2 * t + (uses[t] & 1)) * 128, x + 2 * e, b + 2 * e, idesc,
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
        tc_commit(&sfull[uses[0] & 1]);
        ++uses[0];
        if (two) {
          tc_commit(&sfull[2 + (uses[1] & 1)]);
          ++uses[1];
        }
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
              // a row that sees nothing, or none at all: e^-inf
              v[e] = x.y == 0.f ? -INFINITY : -x.x;
              w[e] = x.y;
            }
          } else {
            const int j = tile * 128 + 4 * lane;
            const int pg = j < it.len ? paged_page(a, a.table + (int64_t)it.b * a.s_table, j) : -1;
            const float* at =
                a.beta + ((((int64_t)max(pg, 0) * a.H + it.h) << a.page_shift) + (j & mask));
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              v[e] = pg >= 0 && j + e < it.len ? at[e] : -INFINITY;
              w[e] = 0.f;
            }
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
          float* const at = reinterpret_cast<float*>(smem + S::kColAt) + 256 * i;
          *reinterpret_cast<float4*>(at + 4 * lane) = make_float4(v[0], v[1], v[2], v[3]);
          if constexpr (kSecond)
            *reinterpret_cast<float4*>(at + 128 + 4 * lane) = make_float4(w[0], w[1], w[2], w[3]);
          if (k + 1 < it.k1) load(k + 1);
          __syncwarp();
          if (lane == 0) mbar_arrive(&colfull[i]);
        }
      }
    }
  } else if (warp >= 4) {
    // ------------------------------------------------------------ sums
    const int t = (warp - 4) >> 2, quarter = warp & 3;
    const int row = quarter * 32 + lane;  // of the held tile
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16) + 256 * t;
    const float k_log2 = f.q.scale * kLog2e;
    const float unit = kBias ? kLog2e : 1.f;  // of m, in log 2
    uint32_t uses = 0, col_uses = 0;
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
      const bool works = t == 0 || is_two(it);
      // pass 1: this row's token among the sequence's; pass 2: this slot
      const int token = (2 * it.x + t) * f.tile_tokens + row / g;
      const int slot = it.x * kWtHeld + 128 * t + row;
      const int past = it.len - it.count;
      const bool valid = kSecond ? slot < it.len : row < tile_rows && token < it.count;
      const int see = valid ? max(0, past + token + 1) : INT32_MAX;         // pass 1: slots
      const int least = kSecond ? 0 : __reduce_min_sync(0xffffffffu, see);  // that every row sees
      float beta = 0.f;
      int page = -1;
      if constexpr (kSecond) {
        if (works && valid) page = paged_page(a, a.table + (int64_t)it.b * a.s_table, slot);
        if constexpr (kBias)
          if (page >= 0)
            beta = a.beta[(((int64_t)page * a.H + it.h) << a.page_shift) + (slot & mask)];
      }
      Sum2 sum;
      float m = -INFINITY;
#pragma unroll 1
      for (int k = it.k0; k < it.k1; ++k) {
        const int tile = tile_of(it, k);
        const int i = col_uses % kWtCols;
        const float* const cols = reinterpret_cast<const float*>(smem + S::kColAt) + 256 * i;
        if constexpr (kCols)
          if (!wait_all(&colfull[i], (col_uses / kWtCols) & 1, 672)) break;
        if (works) {
          if (!wait_all(&sfull[2 * t + (uses & 1)], (uses >> 1) & 1, 673)) break;
          tc_fence_after();
          const uint32_t s_at = lanes + (uses & 1) * 128;
          uint32_t v[64];
          // Columns [c, c + 64): S, with biases logits; -inf where a row does not see the slot.
          auto read = [&](int c) {
            tmem_ld32_issue(s_at + c, v);
            tmem_ld32_issue(s_at + c + 32, v + 32);
            tmem_wait_ld();
            tmem_landed(v);
            tmem_landed(v + 32);
            if constexpr (kBias) {
              const uint64_t sc = pack2(f.q.scale, f.q.scale);
#pragma unroll
              for (int e = 0; e < 64; e += 4) {
                float4 b4 = make_float4(beta, beta, beta, beta);
                if constexpr (!kSecond) b4 = *reinterpret_cast<const float4*>(cols + c + e);
                float u[4];
                unpack2(fma2(pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), sc,
                             pack2(b4.x, b4.y)), u[0], u[1]);
                unpack2(fma2(pack2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), sc,
                             pack2(b4.z, b4.w)), u[2], u[3]);
                if constexpr (!kSecond) {  // whatever a masked slot's K holds
                  u[0] = b4.x == -INFINITY ? -INFINITY : u[0];
                  u[1] = b4.y == -INFINITY ? -INFINITY : u[1];
                  u[2] = b4.z == -INFINITY ? -INFINITY : u[2];
                  u[3] = b4.w == -INFINITY ? -INFINITY : u[3];
                }
#pragma unroll
                for (int x = 0; x < 4; ++x) v[e + x] = __float_as_uint(u[x]);
              }
            }
            if (!kSecond && least < tile * 128 + c + 64) {
              const int upto = see - tile * 128 - c;  // columns that this row sees
#pragma unroll
              for (int e = 0; e < 64; ++e) v[e] = e < upto ? v[e] : 0xff800000u;
            }
          };
          // e^(s - by) of the 64 columns that v holds, two at a time
          auto weights = [&](int e, uint64_t by2, uint64_t k2) {
            const uint64_t x = pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1]));
            float u0, u1;
            unpack2(kBias ? mul2(add2(x, by2), k2) : fma2(x, k2, by2), u0, u1);
            return pack2(ex2_ftz(u0), ex2_ftz(u1));
          };
          const float to_log2 = kBias ? kLog2e : k_log2;
          const uint64_t k2 = pack2(to_log2, to_log2);
          if constexpr (!kSecond) {
            auto top = [&]() {  // of the tile, in units of m
              float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll 1
              for (int c = 0; c < 128; c += 64) {
                read(c);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                  m0 = max3(m0, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
                  m1 = max3(m1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
                }
              }
              const float x = fmaxf(m0, m1);
              return kBias || x == -INFINITY ? x : x * k_log2;
            };
            auto add_up = [&]() {
              const float by = m == -INFINITY ? 0.f : m;  // nothing seen yet: 2^-inf
              const uint64_t by2 = pack2(-by, -by);
              uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll 1
              for (int c = 0; c < 128; c += 64) {
                read(c);
#pragma unroll
                for (int e = 0; e < 64; e += 4) {
                  s0 = add2(s0, weights(e, by2, k2));
                  s1 = add2(s1, weights(e + 2, by2, k2));
                }
              }
              float x0, x1;
              unpack2(add2(s0, s1), x0, x1);
              return x0 + x1;
            };
            if (__any_sync(0xffffffffu, valid && m == -INFINITY)) {
              const float x = top();
              if (m == -INFINITY) m = x;
            }
            float x = add_up();
            if (__any_sync(0xffffffffu, valid && !(x <= (float)kWtMost))) {
              const float higher = fmaxf(m, top());
              if (higher > m) {
                const float down = ex2_ftz((m - higher) * unit);
                sum.s *= down;
                sum.c *= down;
                m = higher;
              }
              x = add_up();
            }
            sum.add(x);
          } else {
            // columns [lo, hi) are rows that see this slot
            const int token0 = tile * f.tile_tokens;
            const int lo = (slot - past - token0) * g;
            const int hi = min(f.tile_tokens, it.count - token0) * g;
            const bool all = !__any_sync(0xffffffffu, lo > 0) && hi == tile_rows;
            uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll 1
            for (int c = 0; c < 128; c += 64) {
              read(c);
#pragma unroll
              for (int e = 0; e < 64; e += 4) {
                const float4 b4 = *reinterpret_cast<const float4*>(cols + c + e);
                const float4 w4 = *reinterpret_cast<const float4*>(cols + 128 + c + e);
                const uint64_t p0 = weights(e, pack2(b4.x, b4.y), k2);
                const uint64_t p1 = weights(e + 2, pack2(b4.z, b4.w), k2);
                if (all) {
                  s0 = fma2(p0, pack2(w4.x, w4.y), s0);
                  s1 = fma2(p1, pack2(w4.z, w4.w), s1);
                } else {  // (a row of NaN counts where it is seen alone)
                  float u[4];
                  unpack2(mul2(p0, pack2(w4.x, w4.y)), u[0], u[1]);
                  unpack2(mul2(p1, pack2(w4.z, w4.w)), u[2], u[3]);
#pragma unroll
                  for (int x = 0; x < 4; ++x)
                    u[x] = c + e + x >= lo && c + e + x < hi ? u[x] : 0.f;
                  s0 = add2(s0, pack2(u[0], u[1]));
                  s1 = add2(s1, pack2(u[2], u[3]));
                }
              }
            }
            float x0, x1;
            unpack2(add2(s0, s1), x0, x1);
            sum.add(x0 + x1);
          }
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&sfree[2 * t + (uses & 1)]);
          ++uses;
        }
        if constexpr (kCols) {
          __syncwarp();
          if (lane == 0) mbar_arrive(&colfree[i]);
          ++col_uses;
        }
      }
      if (bad) break;
      if (!works) continue;
      const int64_t part = (int64_t)(2 * cta + it.part - 1) * kWtHeld + 128 * t + row;
      if constexpr (kSecond) {
        if (beta == -INFINITY) sum.s = 0.f;  // masked
        if (it.part != 0) {
          f.part[part] = make_float2(sum.s, 0.f);
        } else if (page >= 0) {
          float* const w = f.weight + (((int64_t)page * a.H + it.h) << a.page_shift) + (slot & mask);
          *w = (slot < past && f.decay != 0.f ? f.decay * *w : 0.f) + sum.s;
        }
      } else {
        if (it.part != 0)
          f.part[part] = make_float2(m, sum.s);
        else if (valid)
          f.q.ml[(int64_t)(it.first + token) * f.q.Hq + it.h * g + row % g] =
              make_float2(m, sum.s == 0.f ? 0.f : 1.f / sum.s);
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
  return Hq / a.H <= 128 && paged_mean_rows(a, Hq) > 16;
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
