// What the attention kernels on the tensor cores share: the items of a call, in equal ranges of their
// cost, the join of the items that lie in several ranges, and thin PTX wrappers.
#pragma once
#include <algorithm>

#include "gemm_host.cuh"
#include "paged_dev.cuh"

namespace still {

namespace {

constexpr int kPfKeys = 128;        // slots of a tile
// of an item's beginning and end, in tiles of slots (1: 379 and 249 us for 8,192 tokens and for
// three short prompts of 256 channels; 2: 345 and 240; 4: 350 and 247)
constexpr int kPfItemCost = 2;

struct PrefillParams {
  PagedArgs a;
  PagedQuery q;
  int32_t tile_tokens = 0;  // floor(128 / g)
  // parts of items that lie in several CTAs' ranges: what CTA c continues (2 c), begins (2 c + 1)
  float4* part_o = nullptr;   // [2 x CTAs][d / 4][rows of an item]
  float2* part_ml = nullptr;  // [2 x CTAs][rows of an item] (m, l), m in the kernel's units
  struct PfSplit* split = nullptr;  // [CTAs]
};

// The item that CTA c begins and does not end, and the one in which its range begins.
struct PfSplit {
  int32_t last;    // the CTA that ends it; c: there is none
  int32_t token0, tokens, h;
  int32_t first;   // the CTA that begins that one
};

// D[tmem] (+)= A[tmem, 128 lanes x 16] * B[smem, MN-major], kind::f16.
STILL_DEV void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                      uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n" ::"r"(d_tmem),
      "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// One lane of a converged warp, as the compiler knows: behind it operands stay uniform.
STILL_DEV bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "selp.b32 %0, 1, 0, q;\n}\n"
      : "=r"(r));
  return r != 0;
}
// Shared-memory descriptor of an MN-major operand, 128-byte swizzle: rows (k) of 64 contiguous
// elements, 8 rows an atom of 1024 bytes, atoms along k 1024 bytes apart, the next 64 elements
// `chunk` bytes further.
STILL_DEV uint64_t sdesc_mn_sw128(uint32_t saddr, int chunk) {
  uint64_t d = 0;
  d |= (uint64_t)((saddr & 0x3FFFFu) >> 4);
  d |= (uint64_t)(chunk >> 4) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kIdescBMn = 1u << 16;  // B is MN-major

STILL_DEV void tma_load_3d(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z)
      : "memory");
}
STILL_DEV void tma_load_4d(void* dst, const CUtensorMap* m, uint64_t* bar, int x, int y, int z,
                           int w) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%3, %4, %5, %6}], [%2];" ::"r"(smem_u32(dst)),
      "l"(reinterpret_cast<uint64_t>(m)), "r"(smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
      : "memory");
}
// 32 lanes x 16 columns of 32 bits into registers; complete after tmem_wait_ld.
STILL_DEV void tmem_ld16_issue(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
// 32 lanes x 32 columns of 32 bits from registers; complete after tmem_wait_st.
STILL_DEV void tmem_st32_issue(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(
          taddr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]),
      "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
      "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]),
      "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
STILL_DEV void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// What a CTA does of an item.
struct PfItem {
  int b, h, len;
  int token0, tokens;  // its tokens, packed rows
  int see;             // slots that the first of them sees (below 1: none)
  int k0, k1;          // tiles of slots [k0, k1)
  int part;            // 0: all of the item, else where the part goes: 1 + (it is the first)
  int last;            // the CTA that ends an item which this one begins
};

// Where a CTA's range begins, in shared memory.
struct PfStart {
  int64_t base;  // cost of all items before this one
  int64_t total, left;  // of all items, of this CTA's range
  int b, qt, h, off;    // off: cost of this item that lies before the range
  int nct;              // CTAs that have a range
};

// A whole warp waits for a phase; false (and a record, and the flag for the others) at the limit.
STILL_DEV bool pf_wait(uint64_t* bar, uint32_t parity, int* err, volatile int* abort_flag,
                       int where) {
  const bool ok = __all_sync(0xffffffffu, mbar_wait(bar, parity));
  if (!ok && (threadIdx.x & 31) == 0) {
    dev_set_error(err, DEV_WAIT_TIMEOUT, where);
    *abort_flag = 1;
  }
  return ok;
}

__host__ __device__ __forceinline__ int pf_tiles(const Seq& s, int tokens) {
  return (s.count + tokens - 1) / tokens;
}
// Tiles of slots that item qt of a sequence sees.
__host__ __device__ __forceinline__ int pf_slots(const Seq& s, int tokens, int qt) {
  const int upto = (qt + 1) * tokens, most = s.len - s.count + (upto < s.count ? upto : s.count);
  return most > 0 ? (most + kPfKeys - 1) / kPfKeys : 0;
}
// Items of `tokens` tokens each and the tiles of slots that they see: how many of a sequence, the
// tiles of one, what is shown of it.
struct PfRowItems {
  using Item = PfItem;
  int tokens;
  __host__ __device__ int items(const Seq& s) const { return pf_tiles(s, tokens); }
  __host__ __device__ int tiles(const Seq& s, int x) const { return pf_slots(s, tokens, x); }
  STILL_DEV void fill(PfItem& it, const Seq& s, int x) const {
    it.len = s.len;
    it.token0 = s.first + x * tokens;
    it.tokens = min(tokens, s.count - x * tokens);
    it.see = s.len - s.count + x * tokens + 1;
  }
};

// Cost of items [x0, x1) of a sequence and KV-head: a million tokens pass 32 bits.
template <class G>
__host__ __device__ __forceinline__ int64_t pf_cost(const G& items, const Seq& s, int x0, int x1) {
  int64_t sum = 0;
  for (int x = x0; x < x1; ++x) sum += items.tiles(s, x) + kPfItemCost;
  return sum;
}

// The items of a CTA's range, in order: sequences, their items, KV-heads. An item's cost is its
// tiles, then kPfItemCost for its beginning and end.
template <class G>
struct PfWalk {
  const PagedArgs& a;
  G items;
  int64_t base, left, total;
  int b, qt, h, off, nq, nct;
  Seq s;
  STILL_DEV PfWalk(const PagedArgs& args, const G& g, const PfStart& p)
      : a(args), items(g), base(p.base), left(p.left), total(p.total), b(p.b), qt(p.qt),
        h(p.h), off(p.off), nct(p.nct) {
    if (left > 0) {
      s = paged_seq<false>(a, b);
      nq = items.items(s);
    }
  }
  STILL_DEV bool next(typename G::Item& it) {
    while (left > 0) {
      const int kt = items.tiles(s, qt), cost = kt + kPfItemCost;
      const int end = (int)min((int64_t)cost, off + left);
      const bool begins = off == 0;
      it.b = b;
      it.h = h;
      items.fill(it, s, qt);
      it.k0 = min(off, kt);
      it.k1 = min(end, kt);
      it.part = begins && end >= kt ? 0 : begins ? 2 : 1;
      if (it.part == 2) it.last = (int)(((base + kt) * nct - 1) / total);
      left -= end - off;
      off = 0;
      if (end == cost) {
        base += cost;
        if (++h == a.H) {
          h = 0;
          if (++qt == nq) {
            qt = nq = 0;
            while (left > 0 && nq == 0) {
              s = paged_seq<false>(a, ++b);
              nq = items.items(s);
            }
          }
        }
      }
      if (it.k0 < it.k1 || (begins && kt == 0)) return true;
    }
    return false;
  }
};

// Equal ranges of the cost of all items for `most` CTAs (or pairs) at most, by all threads of a block:
// where the range of CTA `cta` begins, and in split (if any) the CTA that begins its first item. No
// range is shorter than an item's beginning and a tile.
template <int kThreads, class G>
STILL_DEV void pf_plan(const PagedArgs& a, const G& items, int cta, int64_t most, PfStart& start,
                       int64_t* warp_cost, PfSplit* split) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // a thread adds up some sequences, or a share of one's
  const int per = (a.B + kThreads - 1) / kThreads, shares = max(1, kThreads / a.B);
  const int share = threadIdx.x % shares;
  const int sb0 = min(a.B, (int)threadIdx.x / shares * per), sb1 = min(a.B, sb0 + per);
  auto first_item = [&](int nq, int x) { return (int)((int64_t)nq * x / shares); };
  int64_t mine = 0;
  for (int b = sb0; b < sb1; ++b) {
    const Seq s = paged_seq(a, b);
    const int nq = items.items(s);
    mine += pf_cost(items, s, first_item(nq, share), first_item(nq, share + 1)) * a.H;
  }
  int64_t before = mine, total = 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += x;
  }
  if (lane == 31) warp_cost[warp] = before;
  if (threadIdx.x == 0) start.left = 0;
  __syncthreads();
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += warp_cost[w];
    total += warp_cost[w];
  }
  before -= mine;
  const int nct = (int)max((int64_t)1, min(most, total / (kPfItemCost + 1)));
  const int64_t u0 = cta < nct ? total * cta / nct : total;
  if (u0 >= before && u0 < before + mine) {
    PfStart p;
    p.total = total;
    p.left = total * (cta + 1) / nct - u0;
    p.nct = nct;
    for (p.b = sb0;; ++p.b) {
      const Seq s = paged_seq(a, p.b);
      const int nq = first_item(items.items(s), share + 1);
      for (p.qt = first_item(items.items(s), share); p.qt < nq; ++p.qt) {
        const int cost = items.tiles(s, p.qt) + kPfItemCost;
        if (u0 < before + (int64_t)cost * a.H) {
          p.h = (int)((u0 - before) / cost);
          p.base = before + (int64_t)cost * p.h;
          p.off = (int)(u0 - p.base);
          break;
        }
        before += (int64_t)cost * a.H;
      }
      if (p.qt < nq) break;
    }
    start = p;
    if (p.off > 0 && split != nullptr) split->first = (int)(((p.base + 1) * nct - 1) / total);
  }
}

// Biases of a tile of slots, loaded ahead by a warp: lane i holds those of slots [4 i, 4 i + 4).
struct PfBias {
  static constexpr int kPer = kPfKeys / 32;
  float v[kPer];
  STILL_DEV void load(const PagedArgs& a, const PfItem& it, int slot0, int lane) {
    const int j = slot0 + kPer * lane;
#pragma unroll
    for (int e = 0; e < kPer; ++e) v[e] = 0.f;
    if (j >= it.len) return;
    const int pg = paged_page<false>(a, a.table + (int64_t)it.b * a.s_table, j);
    const int in = j & ((1 << a.page_shift) - 1);
    const float* at = a.beta + ((((int64_t)max(pg, 0) * a.H + it.h) << a.page_shift) + in);
#pragma unroll
    for (int e = 0; e < kPer; ++e)
      v[e] = pg < 0 ? -INFINITY : j + e < it.len ? at[e] : 0.f;
  }
};

// dims {channels, slots, KV-heads, pages}; boxes of 64 channels of the slots of a page, at most
// `rows` of them
bool pool_tmap(CUtensorMap* m, const PagedArgs& a, const void* ptr, int rows) {
  auto enc = tensor_map_encoder();
  if (enc == nullptr) return false;
  const cuuint64_t page = (cuuint64_t)1 << a.page_shift;
  cuuint64_t dims[4] = {(cuuint64_t)a.d, page, (cuuint64_t)a.H, (cuuint64_t)a.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)a.s_slot * 2, (cuuint64_t)a.s_head * 2,
                           (cuuint64_t)a.s_page * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)std::min<cuuint64_t>(page, rows), 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(ptr), dims, strides, box,
             estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The same of a pool in 8 bits: boxes of `chan` channels, rows of `chan` bytes.
bool codes_tmap(CUtensorMap* m, const PagedArgs& a, const void* ptr, int chan, int rows) {
  auto enc = tensor_map_encoder();
  if (enc == nullptr) return false;
  const cuuint64_t page = (cuuint64_t)1 << a.page_shift;
  cuuint64_t dims[4] = {(cuuint64_t)a.d, page, (cuuint64_t)a.H, (cuuint64_t)a.n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)a.s_slot, (cuuint64_t)a.s_head, (cuuint64_t)a.s_page};
  cuuint32_t box[4] = {(cuuint32_t)chan, (cuuint32_t)std::min<cuuint64_t>(page, rows), 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(ptr), dims, strides, box, estr,
             CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool query_tmap(CUtensorMap* m, const PagedArgs& a, const PagedQuery& q, int tokens) {
  auto enc = tensor_map_encoder();
  if (enc == nullptr) return false;
  cuuint64_t dims[3] = {(cuuint64_t)a.d, (cuuint64_t)q.Hq, (cuuint64_t)a.n};
  cuuint64_t strides[2] = {(cuuint64_t)a.d * 2, (cuuint64_t)q.s_q * 2};
  cuuint32_t box[3] = {64, (cuuint32_t)(q.Hq / a.H), (cuuint32_t)tokens};
  cuuint32_t estr[3] = {1, 1, 1};
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<__nv_bfloat16*>(q.q), dims,
             strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
             CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

}  // namespace still
