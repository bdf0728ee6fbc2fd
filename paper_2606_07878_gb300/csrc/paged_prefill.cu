// Attention of many new tokens over a paged cache, on the tensor cores (tcgen05).
//
// For a KV-head the rows (token i, query head h g + r) see slots j <= past + i:
//   S = q K^T            128 x 128 tiles, operands from shared memory (TMA, one box per page and 64
//                        channels), fp32 in TMEM
//   P = e^(scale S + beta - m)   one row per thread, running m and sum; bf16, written over S
//   O += P V             P from TMEM, V as the loaded rows (channels are its contiguous dimension)
// An item is a sequence, KV-head and two tiles of floor(128 / g) tokens x g heads (one, for 256
// channels and few rows), so that the heads of a group share every K and V tile. For d <= 128 the
// two tiles take turns on one SM: the softmax of one lies under the products of the other. 256
// channels leave TMEM for one tile (S twice, O once): its two softmax warpgroups take tiles of
// slots in turn, handing the running maximum on, and a pair of CTAs (a cluster) takes the two
// tiles in 2-SM products (cta_group::2, M = 256): each CTA loads half of K (64 slots) and half of V
// (128 channels), where one of its own would take in 128 KB for 2,048 clocks of products.
//
// Order of the tensor pipe, i counting S tiles (kTiles = 2: both tiles of the same slots in turn):
// S_0, S_1, PV_0, S_2, PV_1, S_3, ... PV_i waits for P_i alone; S_(i+2) overwrites P_i behind it.
// P_i comes in halves, the last 64 slots first: they are the ones whose S the maximum left in
// registers, and their product starts under the others' exponentials. The running maximum moves
// (and O is rescaled) only when a tile raises it by more than 2^8.
//
// P is bf16: its rounding, 2^-8 of a weight at most, averages out over the slots, and outputs lie
// 0.0023 of their root mean square from 64-bit ones where the rounding of the outputs alone leaves
// 0.0017. A second product for the rest, as few rows have it, would double PV.
//
// Slots that do not count are zeroed in shared memory before their products (a weight of 0 times
// a stale NaN would be NaN): those past the sequence's end, and those with a bias of -inf.
//
// A pool in 8 bits (pf_fetch, pf_convert) goes through a ring of codes first; two warpgroups turn
// them into bf16 in the ring that the products read. Codes in the products themselves
// (kind::f8f6f4) would want q and P in 8 bits, twice for their rests. The prompt below takes 447 us
// from codes, 1.08 PFLOP/s, where bf16 takes 339 (the tensor pipe busy 48%): 409 with a quarter of
// the conversion, so most of the difference is the codes' second way through shared memory (16 KB
// read and 32 written for a tile's 32 of operands), which the products share. With codes loaded by
// the converters themselves, one ring slot ahead in registers: 843 us with four warps (a warp
// issues an instruction every 4 to 5 clocks, and a tile took 3,600); by TMA with eight 491, and 449
// since they are told what a slot holds instead of walking the items. Four ring slots of bf16 and
// two of codes: 467; three and four: 445, within what two runs differ by.
//
// CTA = 12 warps: 0, 10 and 11 TMA producers (a copy takes about 40 clocks to issue, and pages of
// 16 slots are 64 copies for K and V of 128 slots and 256 channels: 352 us with one producer, 235
// with three), 1 MMA issuer and TMEM allocation, 2..9 softmax and output. Every wait is bounded.
//
// Work: a CTA an SM, equal ranges of the cost of all items; what several CTAs share of an item goes
// to the workspace and a second launch joins it.
//
// 8,192 tokens over themselves, 28 query and 4 KV-heads of 128 channels (481 GFLOP): 339 us, 1.42
// PFLOP/s, 0.75 of the library's matrix product. The tensor pipe is busy 71% of the kernel, tensor
// memory 75%, issue slots 48%: what is left is the chain S, maximum, exponentials, P of two tiles
// that take turns, with S read from TMEM twice. (Held in registers in between: 375 us at a stage of
// this kernel that took 352 otherwise, for the spills.) Biases cost a read of shared memory and two
// packed operations per two logits: 1.2 PFLOP/s. 8,192 tokens of 8 KV- and 16 query heads of 256
// channels (half the softmax for the same products): 331 us, 1.66 PFLOP/s; 381 in pages of 16, for
// the copies; 350 and 412 with pages looked up behind the wait for a ring slot. With a tile and all
// of K and V on each SM: 444 and 577; loaded once for a pair by multicast: 432 and 490. 64 channels
// have as many exponentials for half the products: 8,192 tokens of 8 KV- and 32 query heads 336 us
// where 128 channels take 352, 0.82 against 1.56 PFLOP/s (with biases 416 and 465).
#include <type_traits>

#include "paged_tc.cuh"

namespace still {

namespace {

constexpr int kPfProducers = 3;     // warps
constexpr int kPfConverters = 8;    // warps, of a pool in 8 bits
constexpr float kPfMoveLog2 = 8.f;  // P <= 2^8 needs no more of bf16's range

// The same on a CTA pair, issued by the even CTA: A's rows [0, 128) from its TMEM, [128, 256) from
// the odd CTA's, and half of B's columns from each one's shared memory.
STILL_DEV void mma_ts_2sm(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                          uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The same, its completion on an mbarrier of either CTA of the pair (a shared::cluster address).
STILL_DEV void tma_load_4d_2sm(void* dst, const CUtensorMap* m, uint32_t bar_cluster, int x, int y,
                               int z, int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(bar_cluster), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
// Zeroes rows of a ring slot whose chunks have `rows` rows, slots [first, first + rows) of a tile:
// those that lane i marks in its bits for slots [4 i, 4 i + 4).
STILL_DEV void zero_rows(uint8_t* slot, int chunks, int rows, int first, uint32_t marks) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int r = 0; r < rows; r += 4) {
    const uint32_t n4 = __shfl_sync(0xffffffffu, marks, (first + r) / 4);
    if ((n4 >> (lane >> 3)) & 1)
#pragma unroll 1
      for (int c = 0; c < chunks; ++c)
        *reinterpret_cast<uint4*>(slot + (c * rows + r + (lane >> 3)) * 128 + (lane & 7) * 16) =
            make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  __syncwarp();
}

struct PfPlan {  // in shared memory
  PfStart start;
  PfItem shown[2];  // items n & 1 as the producer shows them to the others
  int64_t warp_cost[20];
};

// The warps of a CTA. Of a pool in 8 bits two warpgroups convert codes, and the softmax warps begin
// at a warpgroup of their own, so that registers can be dealt out: 5 x 128 threads of 96 each
// become 144 for the softmax and 64 for all others, 152 and 56 with biases.
template <bool kBias, bool kQuant>
struct PfRoles {
  static constexpr int kThreads = kQuant ? 640 : 384;
  static constexpr int kSoftmax = kQuant ? 4 : 2;       // the first of eight
  static constexpr int kFirst = kSoftmax + 8;           // producer or converter behind them
  static constexpr int kSoftmaxRegs = kBias ? 152 : 144, kOtherRegs = kBias ? 56 : 64;
  static_assert(256 * kSoftmaxRegs + 384 * kOtherRegs <= 640 * 96, "registers of a CTA");
};
// A ring slot of codes, and what the converters have to know of it.
struct PfRaw {
  float scale[kPfKeys / kScaleBlock];  // of its 16 slots each
  uint32_t counts[4];                  // bit i of word e: slot 4 i + e counts
  int32_t kind[4];                     // [0]: of keys (0), of values (1), none any more (2)
};

template <int D, bool kBias, bool kPair, bool kQuant>
struct PfShape {
  static constexpr int kTiles = D <= 128 ? 2 : 1;  // of an item on an SM
  // A ring slot holds 128 slots of kChan channels; a pair's CTA has one with its half of a tile: of
  // K all channels of 64 slots (kKRows), of V kChan channels of all.
  static constexpr int kChan = D < 128 ? D : 128;
  static constexpr int kHalves = kPair ? 1 : D / kChan;  // ring slots of a K or V tile
  static constexpr int kKRows = kPair ? kPfKeys / 2 : kPfKeys;
  static constexpr int kStageBits = kChan == 64 ? 14 : 15;
  static constexpr int kStageBytes = 1 << kStageBits;
  static_assert(kStageBytes == kPfKeys * kChan * 2, "a ring slot");
  static constexpr int kChunkBytes = kPfKeys * 128;  // 64 channels of 128 rows
  static constexpr int kQBytes = kTiles * (D / 64) * kChunkBytes;
  static constexpr int kStages = kQuant ? (D == 64 ? 5 : 3) : D == 64 ? 8 : kBias ? 4 : 5;
  // ring slots of codes, of 8 bits where those above have 16
  static constexpr int kRaws = kQuant ? (D == 64 ? 4 : 3) : 0, kRawBytes = kStageBytes / 2;
  static constexpr int kOCols = kTiles == 2 ? D : D / 2;  // O columns per softmax thread
  static constexpr int kRing = kQBytes;
  static constexpr int kRawAt = kRing + kStages * kStageBytes;
  static constexpr int kBiasAt = kRawAt + kRaws * kRawBytes;  // [8 warps][128]
  // one tile only: running maxima and sums, [2][128] each
  static constexpr int kXchAt = kBiasAt + (kBias ? 8 * kPfKeys * 4 : 0);
  static constexpr int kBarAt = kXchAt + (kTiles == 1 ? 2048 : 0);
  static constexpr int kPlanAt = kBarAt + (3 * kStages + 30) * 8;
  static constexpr int kRawBarAt = (kPlanAt + sizeof(PfPlan) + 15) / 16 * 16;
  static constexpr int kRawInfoAt = kRawBarAt + 2 * 4 * 8;
  static constexpr int kBytes =
      kQuant ? kRawInfoAt + kRaws * (int)sizeof(PfRaw) : kPlanAt + (int)sizeof(PfPlan);
  static_assert(kBytes <= 232448, "shared memory budget");
};

// A ring slot of codes: half a tile of K or V, all of its channels or of its slots in a pair.
struct PfUnit {
  int b, h, len, kt;
  int half;
  bool v;
};
// The ring slots of a CTA's items in the order in which the issuer takes them.
template <int kHalves, int kAhead>
struct PfUnits {
  PfWalk<PfRowItems> walk;
  PfItem it;
  bool have = false;
  int kt = 0, sub = 0;
  // false at the end; `nothing` gets the items whose rows see nothing
  template <class Zero>
  STILL_DEV bool next(PfUnit& u, volatile int* abort_flag, Zero nothing) {
    for (;;) {
      if (!have) {
        if (warp_flag(abort_flag) || !walk.next(it)) return false;
        if (it.k0 == it.k1) {
          nothing(it);
          continue;
        }
        have = true;
        kt = it.k0 - kAhead;
        sub = 0;
      }
      while (kt < it.k1) {
        const bool v = sub < kHalves;
        const int t = v ? kt : kt + kAhead;
        if (sub < 2 * kHalves && t >= it.k0 && t < it.k1) {
          u = PfUnit{it.b, it.h, it.len, t, v ? sub : sub - kHalves, v};
          ++sub;
          return true;
        }
        if (v) {
          sub = kHalves;
        } else {
          sub = 0;
          ++kt;
        }
      }
      have = false;
    }
  }
};

// A pool in 8 bits: a warp fetches codes into a ring of their own (TMA, a box per page), with their
// scales and which slots count, one slot ahead of the copies; two warpgroups multiply codes by
// their block's scale and store bf16 as TMA would have (rows of 128 bytes, 128-byte swizzle).
// Everything behind works as for a pool in bf16. With scales that are powers of two nothing is
// rounded.
template <int D, bool kBias, bool kPair, class Zero>
STILL_DEV void pf_fetch(const PrefillParams& f, int tokens, const PfStart& start, uint8_t* smem,
                        const CUtensorMap& tm_k, const CUtensorMap& tm_v, volatile int* abort_flag,
                        int rank, Zero zero_item) {
  using S = PfShape<D, kBias, kPair, true>;
  const PagedArgs& a = f.a;
  const int lane = threadIdx.x & 31;
  const int mask = (1 << a.page_shift) - 1;
  uint64_t* const raw_full = reinterpret_cast<uint64_t*>(smem + S::kRawBarAt);
  uint64_t* const raw_empty = raw_full + S::kRaws;
  PfRaw* const info = reinterpret_cast<PfRaw*>(smem + S::kRawInfoAt);
  PfUnits<S::kHalves, S::kTiles == 2 ? 1 : 2> units{PfWalk(a, PfRowItems{tokens}, start)};
  auto rows_of = [&](const PfUnit& u) { return kPair && !u.v ? S::kKRows : kPfKeys; };
  auto first_of = [&](const PfUnit& u) {  // slot of its first row
    return u.kt * kPfKeys + (kPair && !u.v ? rank * S::kKRows : 0);
  };
  // Lane i: the page of its i-th 16 slots (-1: none), the scale there; which of slots 4 i + e
  // count.
  auto page_of = [&](const PfUnit& u) {
    const int j = first_of(u) + kScaleBlock * lane;
    if (kScaleBlock * lane >= rows_of(u) || j >= u.len) return -1;
    return paged_page(a, a.table + (int64_t)u.b * a.s_table, j);
  };
  auto scale_of = [&](const PfUnit& u, int pg) {
    if (pg < 0) return 0.f;
    const int in = (first_of(u) + kScaleBlock * lane) & mask;
    return (u.v ? a.v_scale : a.k_scale)[((((int64_t)pg * a.H + u.h) << a.page_shift) + in) >> 4];
  };
  auto counts_of = [&](const PfUnit& u, int pg) {
    uint32_t m = 0;
    const int j = first_of(u) + 4 * lane;
    const int at = __shfl_sync(0xffffffffu, pg, lane >> 2);
    const float* beta = a.beta + ((((int64_t)max(at, 0) * a.H + u.h) << a.page_shift) + (j & mask));
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (at >= 0 && j + e < u.len && (!kBias || beta[e] != -INFINITY)) m |= 1u << e;
    return m;
  };
  int raw = 0;
  uint32_t phase = 0, armed = 0, armed_par = 0;
  bool bad = false;
  PfUnit u{}, then{};
  bool ok = units.next(u, abort_flag, zero_item);
  int pg = ok ? page_of(u) : -1;
#pragma unroll 1
  while (ok) {
    const float scale = scale_of(u, pg);
    const uint32_t counts = counts_of(u, pg);
    const bool more = units.next(then, abort_flag, zero_item);
    const int then_pg = more ? page_of(then) : -1;
    if (!pf_wait(&raw_empty[raw], phase ^ 1, a.err, abort_flag, 617)) {
      bad = true;
      break;
    }
    if (lane < kPfKeys / kScaleBlock) info[raw].scale[lane] = scale;
    if (lane == 0) info[raw].kind[0] = u.v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t w = __ballot_sync(0xffffffffu, (counts >> e) & 1);
      if (lane == e) info[raw].counts[e] = w;
    }
    __syncwarp();
    if (lane == 0) mbar_arrive_expect_tx(&raw_full[raw], S::kRawBytes);
    armed |= 1u << raw;
    armed_par = (armed_par & ~(1u << raw)) | (phase << raw);
    __syncwarp();
    const int box_bits = min(a.page_shift, kPair && !u.v ? 6 : 7);
    const int r = lane << box_bits, at = __shfl_sync(0xffffffffu, pg, (r >> 4) & 31);
    if (r < rows_of(u)) {
      const int chan = kPair ? (u.v ? rank * S::kChan : 0) : u.half * S::kChan;
      const int pitch = kPair && !u.v ? D : S::kChan;
      tma_load_4d(smem + S::kRawAt + raw * S::kRawBytes + r * pitch, u.v ? &tm_v : &tm_k,
                  &raw_full[raw], chan, (first_of(u) + r) & mask, u.h, at < 0 ? a.n_pages : at);
    }
    if (++raw == S::kRaws) {
      raw = 0;
      phase ^= 1;
    }
    u = then;
    pg = then_pg;
    ok = more;
  }
  // The end; copies have landed when the converters have come so far, or by the waits below.
  if (!bad && !pf_wait(&raw_empty[raw], phase ^ 1, a.err, abort_flag, 618)) bad = true;
  if (lane == 0) {
    if (!bad) {
      info[raw].kind[0] = 2;
      mbar_arrive(&raw_full[raw]);
    }
    if (bad || *abort_flag)
      for (int i = 0; i < S::kRaws; ++i)
        if (armed & (1u << i)) (void)mbar_wait(&raw_full[i], (armed_par >> i) & 1);
  }
}

template <int D, bool kBias, bool kPair>
STILL_DEV void pf_convert(const PagedArgs& a, uint8_t* smem, uint64_t* full, uint64_t* empty,
                          volatile int* abort_flag) {
  using S = PfShape<D, kBias, kPair, true>;
  constexpr int kStages = S::kStages;
  constexpr int kPieces = S::kRawBytes / 16 / (32 * kPfConverters);  // of 16 codes, of a thread
  const int lane = threadIdx.x & 31;
  const int me = threadIdx.x - 32 * PfRoles<kBias, true>::kFirst;
  uint64_t* const raw_full = reinterpret_cast<uint64_t*>(smem + S::kRawBarAt);
  uint64_t* const raw_empty = raw_full + S::kRaws;
  const PfRaw* const info = reinterpret_cast<const PfRaw*>(smem + S::kRawInfoAt);
  int stage = 0, raw = 0;
  uint32_t phase = 0, raw_phase = 0;
  bool bad = false;
#pragma unroll 1
  while (!warp_flag(abort_flag)) {
    if (!pf_wait(&raw_full[raw], raw_phase, a.err, abort_flag, 619)) {
      bad = true;
      break;
    }
    const int kind = info[raw].kind[0];
    if (kind == 2) break;
    const bool k_half = kPair && kind == 0;  // 64 rows of 256 channels
    const int bits = k_half ? 4 : S::kChan == 64 ? 2 : 3, row_bits = k_half ? 6 : 7;
    const uint8_t* const from = smem + S::kRawAt + raw * S::kRawBytes;
    uint4 x[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      x[i] = *reinterpret_cast<const uint4*>(from + 16 * (me + i * 32 * kPfConverters));
    if (!pf_wait(&empty[stage], phase ^ 1, a.err, abort_flag, 610)) {
      bad = true;
      break;
    }
    uint8_t* const slot = smem + S::kRing + stage * S::kStageBytes;
    const int piece = me & ((1 << bits) - 1);
    const int unit = 2 * (piece & 3), flip = (piece >> 2) & 1;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const int row = (me >> bits) + i * (32 * kPfConverters >> bits);
      float s = info[raw].scale[row >> 4];
      if (!((info[raw].counts[row & 3] >> (row >> 2)) & 1)) {
        s = 0.f;  // (a block that is masked whole may have any scale)
        x[i] = make_uint4(0, 0, 0, 0);
      }
      const uint64_t s2 = pack2(s, s);
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = e < 2 ? x[i].x : e < 4 ? x[i].y : e < 6 ? x[i].z : x[i].w;
        const uint32_t y = e & 1 ? f16_of_upper(c) : f16_of_lower(c);
        const float2 z = __half22float2(*reinterpret_cast<const __half2*>(&y));
        float z0, z1;
        unpack2(mul2(pack2(z.x, z.y), s2), z0, z1);
        w[e] = bf16x2_bits(__floats2bfloat162_rn(z0, z1));
      }
      // (the second four of eight lanes begin with their second half: no bank twice)
      uint8_t* const at = slot + (((piece >> 2) << row_bits) + row) * 128;
      const uint4 lo = make_uint4(w[0], w[1], w[2], w[3]), hi = make_uint4(w[4], w[5], w[6], w[7]);
      *reinterpret_cast<uint4*>(at + (((unit + flip) ^ (row & 7)) << 4)) = flip ? hi : lo;
      *reinterpret_cast<uint4*>(at + (((unit + 1 - flip) ^ (row & 7)) << 4)) = flip ? lo : hi;
    }
    fence_proxy_async_smem();
    __syncwarp();
    if (lane == 0) {
      mbar_arrive(&raw_empty[raw]);
      if constexpr (kPair)
        mbar_arrive_cluster(cluster_map(smem_u32(&full[stage]), 0));
      else
        mbar_arrive(&full[stage]);
    }
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1;
    }
    if (++raw == S::kRaws) {
      raw = 0;
      raw_phase ^= 1;
    }
  }
  // The last arrivals of the issuer's commits, before the CTA leaves.
  for (int i = 0; me == 0 && !bad && i < kStages && !*abort_flag; ++i) {
    if (!mbar_wait(&empty[stage], phase ^ 1)) {
      dev_set_error(a.err, DEV_WAIT_TIMEOUT, 612);
      *abort_flag = 1;
    }
    if (++stage == kStages) {
      stage = 0;
      phase ^= 1;
    }
  }
}

template <int D, bool kBias, bool kPair, bool kQuant>
__global__ void __launch_bounds__(PfRoles<kBias, kQuant>::kThreads, 1)
    paged_prefill_kernel(const __grid_constant__ CUtensorMap tm_q,
                         const __grid_constant__ CUtensorMap tm_k,
                         const __grid_constant__ CUtensorMap tm_v,
                         const __grid_constant__ PrefillParams f) {
  using S = PfShape<D, kBias, kPair, kQuant>;
  using R = PfRoles<kBias, kQuant>;
  constexpr int kTiles = S::kTiles, kStages = S::kStages, kHalves = S::kHalves;
  // All of it: no byte is left beside five stages of 256 channels, so the base has to be aligned as
  // it is.
  extern __shared__ __align__(1024) uint8_t smem[];
  const int cta = kPair ? blockIdx.x >> 1 : blockIdx.x;  // or pair of CTAs
  // No split item so far. The join reads this record whatever becomes of this CTA.
  if (threadIdx.x == 0 && (!kPair || (blockIdx.x & 1) == 0))
    f.split[cta].last = f.split[cta].first = cta;
  if ((smem_u32(smem) & 1023) != 0) {
    dev_set_error(f.a.err, DEV_BAD_ARG, 602);
    return;
  }
  PfPlan& plan = *reinterpret_cast<PfPlan*>(smem + S::kPlanAt);
  PfStart& start = plan.start;
  PfItem* shown = plan.shown;
  int64_t* warp_cost = plan.warp_cost;
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kBarAt);  // ring slot loaded
  uint64_t* empty = full + kStages;   // ring slot consumed
  // [2] q of item n loaded and the item shown, n & 1. An item of one tile of slots may pass the
  // issuer without the other softmax warpgroup of 256 channels, and the next one's S behind it: the
  // record is written again only when all warps have said (seen) that they read it.
  uint64_t* qfull = empty + kStages;
  uint64_t* qfree = qfull + 2;       // an item's last S complete
  uint64_t* sfull = qfree + 1;       // [2] S_i complete
  uint64_t* pfull = sfull + 2;       // [2] P_i written (and O rescaled where needed)
  uint64_t* pvdone = pfull + 2;      // [2] O holds P_i V
  uint64_t* ofree = pvdone + 2;      // O drained at the end of an item
  // one tile only, per lane quarter: the running maximum behind S_i (of buffer 0, of buffer 1), and
  // both warps' sums at the end of an item
  uint64_t* mb = ofree + 1;          // [2][4]
  uint64_t* lb = mb + 8;             // [4]
  uint64_t* landed = lb + 4;         // the copies into a ring slot that has rows to be zeroed
  uint64_t* phalf = landed + kStages;  // [2] the last 64 slots of P_i written
  uint64_t* qpeer = phalf + 2;  // the other CTA's q loaded
  uint64_t* drain = qpeer + 1;
  uint64_t* seen = drain + 1;  // [2] the softmax warps have read shown[n & 1]
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(seen + 2);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((3 * kStages + 28) * 8 + 16 == S::kPlanAt - S::kBarAt, "barriers");

  const PagedArgs& a = f.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = f.q.Hq / a.H;
  static_assert(kTiles == 1 || !kPair, "a pair's CTAs have a tile each");
  // A pair's products are 2-SM ones: its even CTA (0) issues them for both, and the barriers that
  // its issuer waits for are the even CTA's.
  constexpr int kSides = kPair ? 2 : 1;
  constexpr int kRows = 128 * kSides * kTiles;  // of an item
  const int tokens = f.tile_tokens * (kRows / 128);  // of an item
  const int rank = kPair ? (int)cluster_ctarank() : 0;  // this CTA's tile of a pair's item
  // TMEM: S at 128 i, P over those of its columns that are read first, O behind both
  constexpr int kSCols = 128, kOAt = 2 * kSCols;
  constexpr int kPAt = 64;

  if (threadIdx.x == 0) {
    for (int s = 0; s < kStages; ++s) {
      mbar_init(&full[s], kQuant ? kPfConverters * kSides : kSides);
      mbar_init(&empty[s], 1);
      mbar_init(&landed[s], 1);
    }
    mbar_init(&qfull[0], 1);
    mbar_init(&qfull[1], 1);
    mbar_init(qfree, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sfull[i], 1);
      mbar_init(&pfull[i], 4 * kSides);
      mbar_init(&phalf[i], 4 * kSides);
      mbar_init(&pvdone[i], 1);
    }
    mbar_init(ofree, 8 * kSides);
    mbar_init(qpeer, 1);
    for (int i = 0; i < 8; ++i) mbar_init(&mb[i], 1);
    for (int i = 0; i < 4; ++i) mbar_init(&lb[i], 2);
    mbar_init(drain, 1);
    if constexpr (kQuant) {
      uint64_t* const raw_full = reinterpret_cast<uint64_t*>(smem + S::kRawBarAt);
      for (int i = 0; i < S::kRaws; ++i) {
        mbar_init(&raw_full[i], 1);
        mbar_init(&raw_full[S::kRaws + i], kPfConverters);
      }
    }
    mbar_init(&seen[0], 8);
    mbar_init(&seen[1], 8);
    *abort_flag = 0;
    fence_mbar_init();
    tma_prefetch_desc(&tm_q);
    tma_prefetch_desc(&tm_k);
    tma_prefetch_desc(&tm_v);
  }
  if (warp == 1) {
    if constexpr (kPair) {
      tmem_alloc_2sm(tmem_slot, 512);
      tmem_relinquish_2sm();
    } else {
      tmem_alloc(tmem_slot, 512);
      tmem_relinquish();
    }
  }
  // no range is shorter than an item's beginning and a tile
  pf_plan<R::kThreads>(a, PfRowItems{tokens}, cta, kPair ? gridDim.x / 2 : gridDim.x, start,
                       warp_cost, rank == 0 ? &f.split[cta] : nullptr);
  tc_fence_before();
  __syncthreads();
  if constexpr (kPair) {  // the other's barriers
    __syncwarp();
    cluster_sync();
  }
  tc_fence_after();
  const uint32_t tmem_base = *tmem_slot;
  // Arrives on a barrier that the issuer waits for, of TMEM (nothing in memory is published).
  auto tell_issuer = [&](uint64_t* bar) {
    if constexpr (kPair)
      mbar_arrive_cluster_relaxed(cluster_map(smem_u32(bar), 0));
    else
      mbar_arrive(bar);
  };

  // Item n_items as the others read it, and its q, by a whole warp. The item of that record has been
  // read: of a pool in 8 bits this waits for it (false at a time-out), else the caller did (waits in
  // here cost short prompts of 256 channels 2%, 174 us against 171).
  auto show = [&](int n_items, const PfItem& it) {
    if constexpr (kQuant) {
      if (n_items > 0 && !pf_wait(qfree, (n_items - 1) & 1, a.err, abort_flag, 611)) return false;
      if (n_items > 1 &&
          !pf_wait(&seen[n_items & 1], ((n_items >> 1) - 1) & 1, a.err, abort_flag, 615))
        return false;
    }
    if (lane == 0) {
      shown[n_items & 1] = it;
      if (it.part == 2 && rank == 0) {
        PfSplit& sp = f.split[cta];
        sp.last = it.last;
        sp.token0 = it.token0;
        sp.tokens = it.tokens;
        sp.h = it.h;
      }
      const uint32_t box = (uint32_t)f.tile_tokens * g * 128;
      mbar_arrive_expect_tx(&qfull[n_items & 1], box * kTiles * (D / 64));
      for (int t = 0; t < kTiles; ++t)
        for (int c = 0; c < D / 64; ++c)
          tma_load_3d(smem + (t * (D / 64) + c) * S::kChunkBytes, &tm_q, &qfull[n_items & 1],
                      c * 64, it.h * g, it.token0 + (t + rank) * f.tile_tokens);
    }
    return true;
  };
  // No more items behind n_items of them: when the last one's q and records have been read.
  auto end_items = [&](int n_items) {
    if (n_items > 0 && !*abort_flag && !mbar_wait(qfree, (n_items - 1) & 1)) {
      dev_set_error(a.err, DEV_WAIT_TIMEOUT, 613);
      *abort_flag = 1;
    }
    if (n_items > 1 && !*abort_flag &&
        !mbar_wait(&seen[n_items & 1], ((n_items >> 1) - 1) & 1)) {
      dev_set_error(a.err, DEV_WAIT_TIMEOUT, 616);
      *abort_flag = 1;
    }
    if (!*abort_flag) {
      shown[n_items & 1].k0 = shown[n_items & 1].k1 = 0;
      mbar_arrive(&qfull[n_items & 1]);
    }
  };
  // Rows that see nothing, by a warp.
  auto zero_item = [&](const PfItem& it) {
    for (int x = lane; x < it.tokens * g * (D / 8); x += 32) {
      const int t = x / (g * (D / 8));
      reinterpret_cast<uint4*>(f.q.out + ((int64_t)(it.token0 + t) * f.q.Hq + it.h * g) *
                                             D)[x % (g * (D / 8))] = make_uint4(0, 0, 0, 0);
    }
  };
  // K tiles that are loaded before the first one of V, in the order in which the issuer takes them
  constexpr int kAhead = kTiles == 2 ? 1 : 2;
  if (warp < R::kSoftmax || warp >= R::kFirst) {
    if constexpr (kQuant)
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(R::kOtherRegs));
    if (kQuant && warp == 0) {
      // ------------------------------------------------------------ items and their q
      int n_items = 0;
      bool bad = false, q_armed = false;
      PfWalk walk(a, PfRowItems{tokens}, start);
      PfItem it;
      while (!bad && !warp_flag(abort_flag) && walk.next(it)) {
        if (it.k0 == it.k1) continue;
        if (!show(n_items, it)) {
          bad = true;
          break;
        }
        q_armed = true;
        ++n_items;
      }
      if (lane == 0) {
        if (!bad) end_items(n_items);
        if ((bad || *abort_flag) && q_armed)
          (void)mbar_wait(&qfull[(n_items - 1) & 1], ((n_items - 1) >> 1) & 1);
      }
    } else if (kQuant && (warp == 2 || warp >= R::kFirst)) {
      // ------------------------------------------------------------ codes, and codes to bf16
      if constexpr (kQuant) {
        if (warp == 2)
          pf_fetch<D, kBias, kPair>(f, tokens, start, smem, tm_k, tm_v, abort_flag, rank,
                                    [&](const PfItem& it) {
                                      if (rank == 0) zero_item(it);
                                    });
        else
          pf_convert<D, kBias, kPair>(a, smem, full, empty, abort_flag);
      }
    } else if (!kQuant && (warp == 0 || warp >= R::kFirst)) {
      // ------------------------------------------------------------ TMA producers
      // 0 also loads q, arms the barriers and zeroes rows
      const int me = warp == 0 ? 0 : warp - R::kFirst + 1;
      int stage = 0, n_items = 0;
      uint32_t phase = 0;
      uint32_t armed = 0, armed_par = 0;  // stages whose copies were asked for, and their phases
      uint32_t marked = 0, land_par = 0;  // the same of `landed`, the phase after
      bool q_armed = false, bad = false;
      auto wait = [&](uint64_t* bar, uint32_t parity, int where) {
        if (!pf_wait(bar, parity, a.err, abort_flag, where)) bad = true;
        return !bad;
      };
      // One half (kChan channels) of tile kt of K or V into the next ring slot; of a pair, this
      // CTA's half of the tile.
      auto load = [&](bool is_v, const PfItem& it, int kt, int half, uint32_t mark) {
        const int row_bits = kPair && !is_v ? 6 : 7;  // of a chunk
        const int chunk_bits = S::kStageBits - 7 - row_bits;
        const int first = kPair && !is_v ? rank << row_bits : 0;
        const int chan = kPair ? (is_v ? rank * S::kChan : 0) : half * S::kChan;
        // this lane's box, if any (16 at most, of 16 slots); its page is looked up ahead of the
        // wait
        const int box_bits = min(a.page_shift, row_bits);
        const int x = me + kPfProducers * lane;
        const bool copies = x < 1 << (row_bits - box_bits + chunk_bits);
        static_assert(S::kStageBytes / (16 * 128) <= 32, "a box a lane");
        const int c = x & ((1 << chunk_bits) - 1), r = x >> chunk_bits << box_bits;
        const int j = kt * kPfKeys + first + r;
        // a box outside the pool (past the last page, or of an entry that names none) is zeros
        int pg = copies && j < it.len ? paged_page(a, a.table + (int64_t)it.b * a.s_table, j) : -1;
        if (pg < 0) pg = a.n_pages;
        if (!wait(&empty[stage], phase ^ 1, 610)) return;
        // A slot with rows to be zeroed is full when that is done, a moment after its copies.
        const bool any = __any_sync(0xffffffffu, mark != 0);
        uint64_t* const bar = any ? &landed[stage] : &full[stage];
        if (me == 0 && lane == 0) {
          if (!kPair || any || rank == 0)
            mbar_arrive_expect_tx(bar, (kPair && !any ? 2 : 1) << S::kStageBits);
          else
            tell_issuer(bar);
        }
        if (!any) {
          armed |= 1u << stage;
          armed_par = (armed_par & ~(1u << stage)) | (phase << stage);
        } else {
          marked |= 1u << stage;
          land_par ^= 1u << stage;
        }
        __syncwarp();
        uint8_t* const slot = smem + S::kRing + stage * S::kStageBytes;
        if (copies) {
          const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
          uint8_t* const dst = slot + ((c << row_bits) + r) * 128;
          const int in = j & ((1 << a.page_shift) - 1);
          if (kPair && !any)
            tma_load_4d_2sm(dst, tm, cluster_map(smem_u32(bar), 0), chan + c * 64, in, it.h, pg);
          else
            tma_load_4d(dst, tm, bar, chan + c * 64, in, it.h, pg);
        }
        if (any && me == 0) {
          if (!wait(&landed[stage], ((land_par >> stage) & 1) ^ 1, 614)) return;
          zero_rows(slot, 1 << chunk_bits, 1 << row_bits, first, mark);
          if (lane == 0) {
            if constexpr (kPair)
              mbar_arrive_cluster(cluster_map(smem_u32(&full[stage]), 0));
            else
              mbar_arrive(&full[stage]);
          }
        }
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1;
        }
      };
      PfBias beta;  // of the next tile of K
      uint32_t mark[2] = {0, 0};  // of the tile of K loaded last and of the one before
      // K of tile kt, tiles in order: which of its slots count is found out here
      auto load_k = [&](const PfItem& it, int kt) {
        uint32_t m = 0;
        const int j = kt * kPfKeys + 4 * lane;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (j + e >= it.len || (kBias && beta.v[e] == -INFINITY)) m |= 1u << e;
        if (kBias && kt + 1 < it.k1) beta.load(a, it, (kt + 1) * kPfKeys, lane);
        mark[1] = mark[0];
        mark[0] = m;
        // without biases the row limits mask what K holds past the end
#pragma unroll 1
        for (int half = 0; half < kHalves && !bad; ++half)
          load(false, it, kt, half, kBias ? m : 0u);
      };
      PfWalk walk(a, PfRowItems{tokens}, start);
      PfItem it;
      while (!bad && !warp_flag(abort_flag) && walk.next(it)) {
        if (it.k0 == it.k1) {  // its rows see nothing
          if (me == 1 && rank == 0) zero_item(it);
          continue;
        }
        if (me == 0 && n_items > 0 && !wait(qfree, (n_items - 1) & 1, 611)) break;
        if (me == 0 && n_items > 1 && !wait(&seen[n_items & 1], ((n_items >> 1) - 1) & 1, 615))
          break;
        if (me == 0) (void)show(n_items, it);
        q_armed = true;
        ++n_items;
        if constexpr (kBias) beta.load(a, it, it.k0 * kPfKeys, lane);
#pragma unroll 1
        for (int kt = it.k0 - kAhead; kt < it.k1 && !bad; ++kt) {
          if (kt >= it.k0) {
            const uint32_t m = kAhead == 2 && kt + 1 < it.k1 ? mark[1] : mark[0];
#pragma unroll 1
            for (int half = 0; half < kHalves && !bad; ++half) load(true, it, kt, half, m);
          }
          if (kt + kAhead < it.k1 && !bad) load_k(it, kt + kAhead);
        }
      }
      // The CTA may leave only when nothing is on its way into its shared memory: the last arrivals
      // of the issuer's commits, or copies that nobody waited for.
      if (me == 0 && lane == 0 && !bad) {
        for (int i = 0; i < kStages && !bad && !*abort_flag; ++i) {
          if (!mbar_wait(&empty[stage], phase ^ 1)) {
            dev_set_error(a.err, DEV_WAIT_TIMEOUT, 612);
            *abort_flag = 1;
            bad = true;
          }
          if (++stage == kStages) {
            stage = 0;
            phase ^= 1;
          }
        }
        end_items(n_items);
      }
      // (The odd CTA's copies count on the even CTA's barriers: its own run out of time here, in
      // which the copies land, as do the even CTA's where one of the two had asked for no more.)
      if (lane == 0) {
        if (bad || *abort_flag) {
          for (int s = 0; s < kStages; ++s) {
            if (armed & (1u << s)) (void)mbar_wait(&full[s], (armed_par >> s) & 1);
            if (marked & (1u << s)) (void)mbar_wait(&landed[s], ((land_par >> s) & 1) ^ 1);
          }
          if (q_armed) (void)mbar_wait(&qfull[(n_items - 1) & 1], ((n_items - 1) >> 1) & 1);
        }
      }
    } else if (warp == 1 && rank == 0 && elect_one()) {
      // ------------------------------------------------------------ MMA issuer
      constexpr uint32_t idesc_s = idesc_f16(128 * kSides, kPfKeys, 1);
      constexpr uint32_t idesc_o = idesc_f16(128 * kSides, S::kChan * kSides, 1) | kIdescBMn;
      int stage = 0;
      uint32_t phase = 0;
      uint32_t n_i = 0, n_odd = 0;  // uses of buffer 0 (two tiles: of both), of buffer 1
      uint32_t n_items = 0;
      bool bad = false, issued = false;
      auto wait = [&](uint64_t* bar, uint32_t parity, int where) {
        if (kPair ? mbar_wait_cluster(bar, parity) : mbar_wait(bar, parity)) return true;
        dev_set_error(a.err, DEV_WAIT_TIMEOUT, where);
        *abort_flag = 1;
        bad = true;
        return false;
      };
      // The next ring slot, loaded; -1 at a time-out.
      auto take = [&]() -> int {
        if (!wait(&full[stage], phase, 620)) return -1;
        const int s = stage;
        if (++stage == kStages) {
          stage = 0;
          phase ^= 1;
        }
        return s;
      };
      const uint64_t q_desc = sdesc_k_sw128(smem_u32(smem));
      const uint64_t k_desc = sdesc_k_sw128(smem_u32(smem + S::kRing));
      const uint64_t v_desc = sdesc_mn_sw128(smem_u32(smem + S::kRing), S::kChunkBytes);
      constexpr uint64_t kChunkStep = S::kChunkBytes >> 4, kStageStep = S::kStageBytes >> 4;
      constexpr uint64_t kKStep = S::kKRows * 128 >> 4;  // from 64 channels of K to the next
      constexpr int kSChunks = D / 64 / kHalves;         // of a ring slot of K
      auto commit = [&](uint64_t* bar) {  // on the barrier of either CTA
        if constexpr (kPair)
          tc_commit_2sm_mc(bar, 3);
        else
          tc_commit(bar);
      };
      // S of tile t into buffer buf, over the channels of one ring slot
      auto mma_s = [&](int buf, int t, int half, int s) {
        tc_fence_after();
        const uint64_t q = q_desc + (t * (D / 64) + half * kSChunks) * kChunkStep;
        const uint64_t k = k_desc + s * kStageStep;
#pragma unroll
        for (int c = 0; c < kSChunks; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            (kPair ? tc_mma_f16_2sm : tc_mma_f16)(
                tmem_base + buf * kSCols, q + c * kChunkStep + 2 * e, k + c * kKStep + 2 * e,
                idesc_s, half + c + e > 0);
        issued = true;
      };
      // O of tile t, the channels of one ring slot, += P in buffer buf times V
      // (slots [16 e0, 16 e1) of the tile)
      auto mma_o = [&](int buf, int t, int half, int s, bool first, int e0 = 0,
                       int e1 = kPfKeys / 16) {
        tc_fence_after();
        const uint64_t v = v_desc + s * kStageStep;
#pragma unroll
        for (int e = e0; e < e1; ++e)
          (kPair ? mma_ts_2sm : mma_ts)(tmem_base + kOAt + t * D + half * S::kChan,
                                        tmem_base + buf * kSCols + kPAt + 8 * e,
                                        v + e * (2048 >> 4), idesc_o, !first || e > e0);
      };
      while (!bad && !*abort_flag) {
        if (!wait(&qfull[n_items & 1], (n_items >> 1) & 1, 621)) break;
        const int n_k = shown[n_items & 1].k1 - shown[n_items & 1].k0;
        if (n_k < 1) break;
        if (kPair && !wait(qpeer, n_items & 1, 636)) break;
        if constexpr (kTiles == 2) {
          int ks = take();
          if (ks < 0) break;
          mma_s(0, 0, 0, ks);
          commit(&sfull[0]);
          mma_s(1, 1, 0, ks);
          commit(&sfull[1]);
          commit(&empty[ks]);
          if (n_k == 1) commit(qfree);
#pragma unroll 1
          for (int j = 0; j < n_k; ++j, ++n_i) {
            const bool more = j + 1 < n_k;
            const int vs = take();
            if (vs < 0 || !wait(&phalf[0], n_i & 1, 622)) break;
            if (j == 0 && n_items > 0 && !wait(ofree, (n_items - 1) & 1, 623)) break;
            mma_o(0, 0, 0, vs, j == 0, 4, 8);
            if (!wait(&pfull[0], n_i & 1, 627)) break;
            mma_o(0, 0, 0, vs, false, 0, 4);
            commit(&pvdone[0]);
            if (more) {
              if ((ks = take()) < 0) break;
              mma_s(0, 0, 0, ks);
              commit(&sfull[0]);
            }
            if (!wait(&phalf[1], n_i & 1, 624)) break;
            mma_o(1, 1, 0, vs, j == 0, 4, 8);
            if (!wait(&pfull[1], n_i & 1, 628)) break;
            mma_o(1, 1, 0, vs, false, 0, 4);
            commit(&pvdone[1]);
            commit(&empty[vs]);
            if (more) {
              mma_s(1, 1, 0, ks);
              commit(&sfull[1]);
              commit(&empty[ks]);
              if (j + 2 == n_k) commit(qfree);
            }
          }
        } else {
          // S and P take buffers 0 and 1 in turn, from 0 on in every item (constants: with a buffer
          // and a half that the loop counts, issuing takes longer than the products)
          auto make_s = [&](auto buf, int i) {
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
              const int s = take();
              if (s < 0) return;
              mma_s(buf, 0, half, s);
              commit(&empty[s]);
            }
            commit(&sfull[buf]);
            if (i + 1 == n_k) commit(qfree);
          };
          auto add_pv = [&](auto buf, uint32_t& uses, int i) {
            if (!wait(&phalf[buf], uses & 1, 625)) return;
            if (i == 0 && n_items > 0 && !wait(ofree, (n_items - 1) & 1, 626)) return;
            int vs[kHalves];
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
              if ((vs[half] = take()) < 0) return;
              mma_o(buf, 0, half, vs[half], i == 0, 4, 8);
            }
            if (!wait(&pfull[buf], uses & 1, 635)) return;
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
              mma_o(buf, 0, half, vs[half], false, 0, 4);
              commit(&empty[vs[half]]);
            }
            commit(&pvdone[buf]);
            ++uses;
          };
          constexpr std::integral_constant<int, 0> b0;
          constexpr std::integral_constant<int, 1> b1;
          make_s(b0, 0);
          if (n_k > 1 && !bad) make_s(b1, 1);
#pragma unroll 1
          for (int i = 0; i < n_k && !bad; i += 2) {
            add_pv(b0, n_i, i);
            if (i + 2 < n_k && !bad) make_s(b0, i + 2);
            if (i + 1 == n_k || bad) break;
            add_pv(b1, n_odd, i + 1);
            if (i + 3 < n_k && !bad) make_s(b1, i + 3);
          }
        }
        ++n_items;
      }
      if ((bad || *abort_flag) && issued) {
        commit(drain);
        (void)mbar_wait(drain, 0);
      }
    } else if (kPair && warp == 1 && rank == 1 && elect_one()) {
      // ------------------------------------------------------------ q of the odd CTA
      for (uint32_t n = 0; !*abort_flag; ++n) {
        if (!mbar_wait(&qfull[n & 1], (n >> 1) & 1)) {
          dev_set_error(a.err, DEV_WAIT_TIMEOUT, 637);
          *abort_flag = 1;
          break;
        }
        if (shown[n & 1].k1 <= shown[n & 1].k0) break;
        mbar_arrive_cluster(cluster_map(smem_u32(qpeer), 0));
      }
    }
  } else {
    if constexpr (kQuant)
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(R::kSoftmaxRegs));
    // ------------------------------------------------------------ softmax and output
    constexpr int kOCols = S::kOCols;
    const int sw = warp - R::kSoftmax;
    const int quarter = warp & 3;  // TMEM lanes [32 quarter, + 32)
    const int wg = sw >> 2;        // its buffer of S: its tile, or every other tile of slots
    const int row = quarter * 32 + lane;
    const uint32_t lanes = tmem_base + ((uint32_t)(quarter * 32) << 16);
    const uint32_t o_at = lanes + kOAt + (kTiles == 2 ? wg * D : 0);
    const uint32_t s_at = lanes + wg * kSCols;
    float* kw = reinterpret_cast<float*>(smem + S::kBiasAt) + sw * kPfKeys;
    float* xm = reinterpret_cast<float*>(smem + S::kXchAt) + row;  // [2][128]
    float* xl = xm + 256;                                          // [2][128]
    // exponents: with biases logits are natural (a bias of the lowest float must stay finite),
    // without them S itself is kept and the scale joins the factor
    const float to_log2 = kBias ? kLog2e : f.q.scale * kLog2e;
    uint32_t mine = 0, other = 0;  // uses of this warp's buffer of S before this item, of the other
    bool bad = false;
    auto wait_all = [&](uint64_t* bar, uint32_t parity, int where) -> bool {
      if (!pf_wait(bar, parity, a.err, abort_flag, where)) bad = true;
      return !bad;
    };
    // The running maximum that the other warp of this lane quarter left behind its use n of its
    // buffer (from 1 on); this warp's sum is brought to it.
    auto follow = [&](uint32_t n, float& m, float& l) {
      if (!wait_all(&mb[4 * (wg ^ 1) + quarter], (n - 1) & 1, 631)) return;
      const float theirs = xm[128 * (wg ^ 1)];
      if (theirs != m) l *= ex2_ftz((m - theirs) * to_log2);
      m = theirs;
    };
    const int tile = kTiles == 2 ? wg : rank;                  // of an item
    const int token = tile * f.tile_tokens + row / g;  // of an item
    for (uint32_t n_items = 0; !bad && !warp_flag(abort_flag); ++n_items) {
      if (!wait_all(&qfull[n_items & 1], (n_items >> 1) & 1, 629)) break;
      const PfItem it = shown[n_items & 1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&seen[n_items & 1]);
      if (it.k1 <= it.k0) break;
      const bool valid = row < f.tile_tokens * g && token < it.tokens;
      // (rows of no token are not stored: they need no masks)
      const int see = valid ? max(0, it.see + token) : INT32_MAX;
      float m_run = -INFINITY, l_run = 0.f;
      PfBias beta;
      const int first = it.k0 + (kTiles == 2 ? 0 : wg);
      constexpr int kStep = 3 - kTiles;  // tiles of slots from one of this warp's to the next
      if (kBias && first < it.k1) beta.load(a, it, first * kPfKeys, lane);
      uint32_t n = mine;  // uses of the buffer
      const int least = __reduce_min_sync(0xffffffffu, see);  // slots that every row sees
#pragma unroll 1
      for (int kt = first; kt < it.k1; kt += kStep, ++n) {
        const int slot0 = kt * kPfKeys;
        if constexpr (kBias) {
#pragma unroll
          for (int e = 0; e < beta.kPer; ++e) kw[beta.kPer * lane + e] = beta.v[e];
          if (kt + kStep < it.k1) beta.load(a, it, slot0 + kStep * kPfKeys, lane);
          __syncwarp();
        }
        if (!wait_all(&sfull[wg], n & 1, 630)) break;
        tc_fence_after();
        uint32_t v[64];
        // Columns [c, c + 64) as logits, -inf where the row does not see the slot.
        auto logits = [&](int c) {
          tmem_ld32_issue(s_at + c, v);
          tmem_ld32_issue(s_at + c + 32, v + 32);
          tmem_wait_ld();
          tmem_landed(v);
          tmem_landed(v + 32);
          if constexpr (kBias) {
            const uint64_t sc = pack2(f.q.scale, f.q.scale);
#pragma unroll
            for (int e = 0; e < 64; e += 4) {
              const float4 b4 = *reinterpret_cast<const float4*>(kw + c + e);
              float u0, u1;
              unpack2(fma2(pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1])), sc,
                           pack2(b4.x, b4.y)), u0, u1);
              v[e] = __float_as_uint(u0);
              v[e + 1] = __float_as_uint(u1);
              unpack2(fma2(pack2(__uint_as_float(v[e + 2]), __uint_as_float(v[e + 3])), sc,
                           pack2(b4.z, b4.w)), u0, u1);
              v[e + 2] = __float_as_uint(u0);
              v[e + 3] = __float_as_uint(u1);
            }
          }
          if (least < slot0 + c + 64) {
            const int seen = see - slot0 - c;  // columns that this row sees
#pragma unroll
            for (int e = 0; e < 64; ++e) v[e] = e < seen ? v[e] : 0xff800000u;
          }
        };
        float m0 = -INFINITY, m1 = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < kPfKeys; c += 64) {
          logits(c);
#pragma unroll
          for (int e = 0; e < 64; e += 4) {
            m0 = max3(m0, __uint_as_float(v[e]), __uint_as_float(v[e + 1]));
            m1 = max3(m1, __uint_as_float(v[e + 2]), __uint_as_float(v[e + 3]));
          }
        }
        const float mx = fmaxf(m0, m1);
        // uses of the buffer that the tile before was in
        const uint32_t before = kTiles == 2 ? n : other + (kt - it.k0 + 1) / 2;
        if (kTiles == 1 && kt > it.k0) {
          follow(before, m_run, l_run);
          if (bad) break;
        }
        bool move = false;
        float fac = 1.f;
        if (m_run == -INFINITY) {
          m_run = mx;  // O and l are 0 so far
        } else if ((mx - m_run) * to_log2 > kPfMoveLog2) {
          fac = ex2_ftz((m_run - mx) * to_log2);
          m_run = mx;
          l_run *= fac;
          move = valid;
        }
        if constexpr (kTiles == 1) {
          xm[128 * wg] = m_run;
          __syncwarp();
          if (lane == 0) mbar_arrive(&mb[4 * wg + quarter]);
        }
        // warp-collective: a warp rescales O when any of its rows needs it
        if (__any_sync(0xffffffffu, move) && kt > it.k0) {
          if (!wait_all(&pvdone[kTiles == 2 ? wg : wg ^ 1], (before - 1) & 1, 632)) break;
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 32) {
            float o[32];
            tmem_ld32(o_at + c, o);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= fac;
            tmem_st32(o_at + c, o);
          }
        }
        // nothing seen yet: every weight is 2^-inf
        const float by = m_run == -INFINITY ? 0.f : m_run;
        const float shift = kBias ? -by : -by * to_log2;
        const uint64_t by2 = pack2(shift, shift), k2 = pack2(to_log2, to_log2);
        uint64_t s0 = 0ull, s1 = 0ull;
        // the last columns first: v still holds them
#pragma unroll 1
        for (int c = kPfKeys - 64; c >= 0; c -= 64) {
          if (c < kPfKeys - 64) logits(c);
#pragma unroll
          for (int e = 0; e < 64; e += 2) {
            float u0, u1;
            const uint64_t x = pack2(__uint_as_float(v[e]), __uint_as_float(v[e + 1]));
            unpack2(kBias ? mul2(add2(x, by2), k2) : fma2(x, k2, by2), u0, u1);
            const float p0 = ex2_ftz(u0), p1 = ex2_ftz(u1);
            if (e & 2)
              s1 = add2(s1, pack2(p0, p1));
            else
              s0 = add2(s0, pack2(p0, p1));
            v[e / 2] = bf16x2_bits(__floats2bfloat162_rn(p0, p1));
          }
          tmem_st32_issue(s_at + kPAt + c / 2, v);
          if (c > 0) {
            tmem_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) tell_issuer(&phalf[wg]);
          }
        }
        float l0, l1;
        unpack2(add2(s0, s1), l0, l1);
        l_run += l0 + l1;
        tmem_wait_st();
        tc_fence_before();
        __syncwarp();  // and kw is written again
        if (lane == 0) tell_issuer(&pfull[wg]);
      }
      if (bad) break;
      // ---- the item's rows
      float l = l_run;
      const int oc = kTiles == 2 ? 0 : wg * kOCols;  // the columns that this warp writes
      if constexpr (kTiles == 2) {
        mine = n;
        if (!wait_all(&pvdone[wg], (n - 1) & 1, 634)) break;
      } else {
        const int tiles = it.k1 - it.k0;
        const bool last_mine = ((tiles - 1) & 1) == wg;
        mine += (tiles + 1 - wg) / 2;
        other += (tiles + wg) / 2;
        if (!last_mine) follow(other, m_run, l);
        if (bad || !wait_all(&pvdone[(tiles - 1) & 1], ((last_mine ? mine : other) - 1) & 1, 634))
          break;
        // (behind that wait nobody reads the sums of the item before any more)
        xl[128 * wg] = l;
        __syncwarp();
        if (lane == 0) mbar_arrive(&lb[quarter]);
        if (!wait_all(&lb[quarter], n_items & 1, 633)) break;
        l += xl[128 * (wg ^ 1)];
      }
      tc_fence_after();
      if (it.part != 0) {  // columns apart, so that a warp's rows lie side by side
        const int64_t part = 2 * cta + it.part - 1;
        const int prow = 128 * tile + row;
        float4* dst = f.part_o + (part * (D / 4) + oc / 4) * kRows + prow;
#pragma unroll 1
        for (int c = 0; c < kOCols; c += 32) {
          float o[32];
          tmem_ld32(o_at + oc + c, o);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            dst[(c / 4 + e) * kRows] =
                make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
        if (kTiles == 2 || wg == 0) f.part_ml[part * kRows + prow] = make_float2(m_run, l);
      } else {
        // Four lanes exchange pieces of 16 bytes, so that they store 64 bytes of one row at a time:
        // a row per lane takes four times as many passes of the store unit.
        const float inv = l == 0.f ? 0.f : 1.f / l;
        const int64_t orow =
            valid ? (int64_t)(it.token0 + token) * f.q.Hq + it.h * g + row % g : -1;
        int64_t at[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = __shfl_sync(0xffffffffu, orow, (lane & ~3) + i);
        const bool odd = lane & 1, high = lane & 2;
#pragma unroll 1
        for (int c = 0; c < kOCols; c += 32) {
          float o[32];
          tmem_ld32(o_at + oc + c, o);
          uint32_t w[4][4];
#pragma unroll
          for (int e = 0; e < 16; ++e)
            w[e / 4][e % 4] =
                bf16x2_bits(__floats2bfloat162_rn(o[2 * e] * inv, o[2 * e + 1] * inv));
#pragma unroll
          for (int m = 0; m < 4; m += 2)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t x = __shfl_xor_sync(0xffffffffu, odd ? w[m][i] : w[m + 1][i], 1);
              (odd ? w[m][i] : w[m + 1][i]) = x;
            }
#pragma unroll
          for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t x = __shfl_xor_sync(0xffffffffu, high ? w[m][i] : w[m + 2][i], 2);
              (high ? w[m][i] : w[m + 2][i]) = x;
            }
          // piece lane & 3 of four rows
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (at[i] >= 0)
              *reinterpret_cast<uint4*>(f.q.out + at[i] * D + oc + c + 8 * (lane & 3)) =
                  make_uint4(w[i][0], w[i][1], w[i][2], w[i][3]);
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) tell_issuer(ofree);
    }
  }
  tc_fence_before();
  __syncthreads();
  if constexpr (kPair) {  // the other may still arrive on this CTA's barriers
    __syncwarp();
    cluster_sync();
  }
  if (warp == 1) {
    tc_fence_after();
    if constexpr (kPair)
      tmem_dealloc_2sm(tmem_base, 512);
    else
      tmem_dealloc(tmem_base, 512);
  }
}

// Rows of the items that lie in several CTAs' ranges: block (c, x) joins rows [32 x, + 32) of the
// item that CTA c begins, its parts in the order of their slots; a lane takes a row, a warp d / 8
// channels. Of an item in kPfMany ranges or more the first eight CTAs' blocks take d / 8 channels
// each (none of the others begins an item), their warps every eighth part: what bounds it is one
// dependent read of memory after another. 32 rows over one sequence of 60,000 slots: 43 us against
// 55 without (4 KV-heads of 128 channels), 42 against 102 (2 of 256).
constexpr int kPfMany = 16;

template <int D>
__global__ void __launch_bounds__(256)
    paged_join_kernel(const __grid_constant__ PrefillParams f, int item_rows, float to_log2) {
  griddep_wait();
  constexpr int kCh = D / 8;  // channels of a warp
  __shared__ float red[8][kCh][32];
  __shared__ float2 red_ml[8][32];
  int c = blockIdx.x;
  PfSplit sp = f.split[c];
  if (sp.last <= c) {
    if (sp.first >= c || c - sp.first >= 8) return;
    c = sp.first;
    sp = f.split[c];
    if (sp.last - c + 1 < kPfMany) return;
  }
  const int parts = sp.last - c + 1;
  const bool many = parts >= kPfMany;
  const int g = f.q.Hq / f.a.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int r = 32 * blockIdx.y + lane, x0 = (many ? (int)blockIdx.x - c : warp) * kCh;
  const int in = r & 127, token = (r >> 7) * f.tile_tokens + in / g;
  const bool valid = in < f.tile_tokens * g && token < sp.tokens;
  const int first = many ? warp : 0, step = many ? 8 : 1;
  auto part = [&](int i) { return (int64_t)(i == 0 ? 2 * c + 1 : 2 * (c + i)); };
  float M = -INFINITY, L = 0.f, O[kCh];
#pragma unroll
  for (int e = 0; e < kCh; ++e) O[e] = 0.f;
  if (valid) {
#pragma unroll 8
    for (int i = first; i < parts; i += step) M = fmaxf(M, f.part_ml[part(i) * item_rows + r].x);
#pragma unroll 4
    for (int i = first; i < parts; i += step) {
      const float2 ml = f.part_ml[part(i) * item_rows + r];
      const float w = ml.x == M ? 1.f : exp2f((ml.x - M) * to_log2);
      const float4* src = f.part_o + (part(i) * (D / 4) + x0 / 4) * item_rows + r;
      L += w * ml.y;
#pragma unroll
      for (int e = 0; e < kCh / 4; ++e) {
        const float4 o = src[e * item_rows];
        O[4 * e] += w * o.x;
        O[4 * e + 1] += w * o.y;
        O[4 * e + 2] += w * o.z;
        O[4 * e + 3] += w * o.w;
      }
    }
  }
  if (many) {  // the warps' sums, in their order
#pragma unroll
    for (int e = 0; e < kCh; ++e) red[warp][e][lane] = O[e];
    red_ml[warp][lane] = make_float2(M, L);
    __syncthreads();
    if (warp != 0) return;
#pragma unroll 1
    for (int w = 1; w < 8; ++w) M = fmaxf(M, red_ml[w][lane].x);
    L = 0.f;
#pragma unroll
    for (int e = 0; e < kCh; ++e) O[e] = 0.f;
#pragma unroll 1
    for (int w = 0; w < 8; ++w) {
      const float2 ml = red_ml[w][lane];
      const float v = ml.x == M ? 1.f : exp2f((ml.x - M) * to_log2);
      L += v * ml.y;
#pragma unroll
      for (int e = 0; e < kCh; ++e) O[e] += v * red[w][e][lane];
    }
  }
  if (!valid) return;
  const float inv = L == 0.f ? 0.f : 1.f / L;
  uint4* dst = reinterpret_cast<uint4*>(
      f.q.out + ((int64_t)(sp.token0 + token) * f.q.Hq + sp.h * g + in % g) * D + x0);
#pragma unroll
  for (int e = 0; e < D / 64; ++e) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = bf16x2_bits(
          __floats2bfloat162_rn(O[8 * e + 2 * i] * inv, O[8 * e + 2 * i + 1] * inv));
    dst[e] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <int D, bool kBias, bool kPair, bool kQuant>
cudaError_t launch_prefill(const PagedArgs& a, const PagedQuery& q, void* ws,
                           const KernelTable& dev, cudaStream_t s) {
  using S = PfShape<D, kBias, kPair, kQuant>;
  constexpr int kCluster = kPair ? 2 : 1;
  constexpr int threads = PfRoles<kBias, kQuant>::kThreads;
  constexpr auto kernel = paged_prefill_kernel<D, kBias, kPair, kQuant>;
  using Id = KernelId<kernel, threads, S::kBytes, kCluster>;
  if (dev.of<Id>().status != cudaSuccess) return dev.of<Id>().status;
  constexpr int rows = 128 * S::kTiles * kCluster;
  const int ranges = kPair ? dev.persistent_clusters<Id>(2) : dev.num_sms;
  PrefillParams f;
  f.a = a;
  f.q = q;
  f.tile_tokens = 128 / (q.Hq / a.H);
  f.part_o = static_cast<float4*>(ws);
  f.part_ml = reinterpret_cast<float2*>(f.part_o + (int64_t)2 * ranges * rows * (D / 4));
  f.split = reinterpret_cast<PfSplit*>(f.part_ml + (int64_t)2 * ranges * rows);
  CUtensorMap tq, tk, tv;
  if (!query_tmap(&tq, a, q, f.tile_tokens)) return cudaErrorInvalidValue;
  if (kQuant ? !codes_tmap(&tk, a, a.K8, kPair ? D : S::kChan, S::kKRows) ||
                   !codes_tmap(&tv, a, a.V8, S::kChan, kPfKeys)
             : !pool_tmap(&tk, a, a.K, S::kKRows) || !pool_tmap(&tv, a, a.V, kPfKeys))
    return cudaErrorInvalidValue;
  cudaLaunchAttribute attr;
  attr.id = cudaLaunchAttributeClusterDimension;
  attr.val.clusterDim.x = kCluster;
  attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCluster * ranges);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = S::kBytes;
  cfg.stream = s;
  cfg.attrs = &attr;
  cfg.numAttrs = kPair ? 1 : 0;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, tq, tk, tv, f);
  if (e != cudaSuccess) return e;
  return launch_chained(paged_join_kernel<D>, dim3(ranges, rows / 32), dim3(256), 0, s, 1, f, rows,
                        (kBias ? 1.f : q.scale) * kLog2e);
}

}  // namespace

bool paged_prefill_serves(const PagedArgs& a, int Hq) {
  // Measured, us, few rows' kernel / this one, 16 sequences of 5,000 slots and 4 KV-heads (256
  // channels: 2): 8 rows 28 / 39, 39 / 48, 42 / 49 for 64, 128, 256 channels; 16 rows 33 / 39,
  // 49 / 48, 64 / 49; 32 rows 49 / 39, 80 / 49, 96 / 49. Groups of more than 128 query heads do not
  // fit a tile.
  //
  // The counts of new tokens are on the device, so the rule has their mean, and a long prompt among
  // many single tokens or idle places may go to the few rows' kernel, which reads its past once for
  // every 8 or 16 of its rows. 256 sequences, 8 KV-heads of 128 channels with 4 query heads each:
  // one of 769 new tokens with 8,192 slots beside 255 single tokens with 400 is at 16 rows on
  // average and takes 1,385 us, with 770 it is above and takes 197; beside 255 idle places 1,184
  // us, and 111 for 1,100 new tokens, which are above. A caller who knows the counts does better
  // with two calls: the prompts in one (86 us alone), the single tokens in the other.
  const int few = a.d == 256 ? 8 : 16;
  // Over a pool in 8 bits, in the same order: 8 rows 36 / 54, 40 / 63, 41 / 58; 16 rows 45 / 54,
  // 56 / 63, 57 / 57; 32 rows 64 / 54, 86 / 62, 85 / 58; two sequences of 60,000 slots (128 channels)
  // 16 rows 75 / 74, 32 rows 117 / 74. Single tokens over it stay with the few rows' kernel, whose
  // weights are exact to 2^-21, while it reads the pool no more than twice.
  if (a.K8 != nullptr && a.cu_new == nullptr && Hq / a.H <= 2 * few) return false;
  return Hq / a.H <= 128 && paged_mean_rows(a, Hq) > few;
}

int64_t paged_prefill_cost(int count, int len, int tokens, int q0, int q1) {
  return pf_cost(PfRowItems{tokens}, Seq{0, count, len}, q0, q1);
}

size_t paged_prefill_workspace(int num_sms) {
  size_t most = 0;
  for (size_t d : {64, 128, 256}) {
    const size_t rows = d <= 128 ? 256 : 128;
    most = std::max(most, (size_t)num_sms * (2 * rows * (d * 4 + 8) + sizeof(PfSplit)));
  }
  return most;
}

cudaError_t launch_paged_prefill(const PagedArgs& a, const PagedQuery& q, void* ws,
                                 const KernelTable& dev, cudaStream_t s) {
  // 256 channels in pairs of CTAs where sequences have rows for two tiles. Three prompts of 900 to
  // 2,300 tokens, 8 KV-heads with 2 query heads each, pages of 16: 172 us against 243. Where the
  // second tile is almost empty (65 tokens of 2 heads over 2,000 slots, 4 KV-heads, 16 sequences):
  // 51 us against 62; 4 sequences of 100 tokens 31 against 33, of 150 without a past 21 and 21.
  // Over 8 bits a pair's CTA also converts half: 8,192 tokens of 8 KV-heads with 2 query heads each
  // 659 us against 779 (with biases 677 against 967), the three prompts 132 against 176; the second
  // tile almost empty 83 against 78.
  const bool pair = paged_mean_rows(a, q.Hq) > 128;
  auto run = [&](auto bias, auto quant) {
    constexpr bool kBias = decltype(bias)::value, kQuant = decltype(quant)::value;
    return a.d == 64    ? launch_prefill<64, kBias, false, kQuant>(a, q, ws, dev, s)
           : a.d == 128 ? launch_prefill<128, kBias, false, kQuant>(a, q, ws, dev, s)
           : pair       ? launch_prefill<256, kBias, true, kQuant>(a, q, ws, dev, s)
                        : launch_prefill<256, kBias, false, kQuant>(a, q, ws, dev, s);
  };
  const std::true_type yes;
  const std::false_type no;
  if (a.K8 != nullptr) return a.beta != nullptr ? run(yes, yes) : run(no, yes);
  return a.beta != nullptr ? run(yes, no) : run(no, no);
}

}  // namespace still
