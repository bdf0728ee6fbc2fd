// Attention of few rows over a paged cache, and the join of what several warps share: for pools in
// bf16 (paged.cu), in e4m3 with scales of blocks (paged_quant.cu), and with the logits and the
// rows' maxima and sums kept for a second pass (paged_weigh.cu).
#pragma once
#include <algorithm>
#include <cuda_fp16.h>

#include "launch.cuh"
#include "paged_dev.cuh"

namespace still {

namespace {

// ----------------------------------------------------------------- attention of few rows
//
// Rows of a KV-head (new token i, query head h g + r of the group) over the slots that token i
// sees: s_j = scale q . k_j + beta_j, out = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m) with a
// running m. A warp takes 16 slots at a time:
//   S^T = K q^T   mma.m16n8k16 (16 slots x 8 rows, fp32 sums). The order of the channels inside
//                 the contraction is free as long as K and q agree, so the 16 bytes of a K row
//                 that a lane loads are fragments of two steps
//   P             in registers; movmatrix turns a slots x rows fragment into the rows x slots one
//                 that the next product reads
//   O^T += V^T P^T  the words of a lane's four V rows, two by two, are fragments of channels x
//                 slots; fp32 sums. P goes in as bf16 hi + lo, two products, which leaves 2^-17 of
//                 a weight (hi alone: outputs 1.4 times as far from 64 bits as plain fp32 ones)
// K, V and O never touch shared memory. Logits stay in natural units up to the subtraction of the
// maximum: in units of log 2 a bias of the lowest float would become -inf, which masks.
//
// Work: a set is a sequence's KV-head and block of 8 or 16 rows; its slots are cut into batches of
// 16, and all batches of all sets, one after another, into equal ranges, one per warp, from lengths
// that the kernel itself adds up. A warp streams through its range without meeting another: K and V
// of the next batch are on their way while it computes one, across the ends of sets too. A set that
// lies in one range is written by its warp; the parts of another meet in the workspace, and a
// second launch joins them in their order. Ranges of CTAs instead, whose warps join after every
// set, with the last CTA of a set joining its parts: 36 / 109 / 170 / 193 us where this takes 32 /
// 90 / 169 / 180 (8 sequences of 1,312 to 5,408 slots; 256 of 165 to 701; 24 of 8,192 to 32,768;
// one of 131,072 with 256 channels); the last warp joining in this kernel: 40 / 93 / 181 / 186.
//
// In 8 bits 16 slots are half the bytes for the same instructions and more: codes become fp16 (two
// an instruction), weights fp16 hi + lo of weight x scale / rho, a number that follows the row's
// largest. The 24 sequences take 130 us (0.5 GB, 3.9 TB/s; one of 131,072 slots with 256 channels
// 130, 4.1): memory is busy 50% and issue slots 44%, and what bounds it is latency, as a warp has one
// batch on its way, 4 KB in 8 bits, so that an SM has half of what it has in bf16. They took 145
// where a warp issued 545 instructions a batch, 250 of them in the integer and conversion pipe, with
// an address product for every row, a division and two exponentials more; 153 with two batches on
// their way at a time, 132 with a fourth CTA on an SM (both spill).
//
// Memory bounds the large calls: the 24 sequences are 1.0 GB, 5.95 TB/s and 0.88 of a copy, with
// the mma.sync pipe at 12%, so the tensor cores of tcgen05 would have nothing to gain. Small calls
// are the latency of a chain of reads (lengths, table, K and V) and of the second launch: 32 us
// for 8 sequences, of which 16 are memory.
constexpr int kRowWarps = 4;  // of a CTA
constexpr int kRowThreads = 32 * kRowWarps;
constexpr int kBatch = 16;      // slots
constexpr int kLeastBatches = 2;  // of a range, on average, where a call has few batches

// What the kernel reads and leaves.
enum RowsKind {
  kRowsBf16,
  kRowsE4m3,    // pools of e4m3 codes, a scale for the 16 slots of a batch
  kRowsWeigh,   // bf16, logits and rows' (m, 1 / l) kept
  kRowsStats    // bf16 keys alone: rows' (m, 1 / l)
};

// c (16 x 8) += a (16 x 16 bf16) b (16 x 8 bf16)
STILL_DEV void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit values: lane i holds row i / 4, columns 2 (i % 4) and
// 2 (i % 4) + 1.
STILL_DEV uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}
// Read-once data: past L1, first to leave L2.
STILL_DEV uint4 ld_once(const void* p) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
STILL_DEV uint32_t word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// c (16 x 8) += a (16 x 16 fp16) b (16 x 8 fp16)
STILL_DEV void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                       uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
STILL_DEV uint32_t f16x2_bits(__half2 x) { return *reinterpret_cast<uint32_t*>(&x); }

// NB: blocks of 8 rows of a set.
template <int D, int NB, int kKind>
struct Rows {
  static constexpr int kRows = 8 * NB;
  static constexpr int kMinCtas = D == 64 ? (NB == 1 ? 4 : 3) : D == 128 ? (NB == 1 ? 3 : 2) : 2;
  static constexpr bool kQShared = D == 256;  // no registers left for q beside K, V and O
};

// The set that warp w begins and does not end.
struct RowsSplit {
  int32_t last;  // the warp that ends it; w: there is none
  int32_t token0, row0, rows;  // the sequence's first new token, the set's rows
  int32_t h;
  int32_t cta0, cta1;  // CTAs [cta0, cta1) whose warps have nothing but this set: one part each
  int32_t unused;
};
struct RowsJoin {
  // parts of the sets that several warps share: what warp w continues (2 w), begins (2 w + 1); a
  // CTA's common part is its first warp's
  float* part_o = nullptr;     // [2 x warps][kRows][d]
  float2* part_ml = nullptr;   // [2 x warps][kRows] (m, l)
  RowsSplit* split = nullptr;  // [warps]
};

STILL_DEV int seq_batches(const Seq& s) { return s.count > 0 ? (s.len + kBatch - 1) / kBatch : 0; }
template <int kRows>
STILL_DEV int seq_blocks(const Seq& s, int g) {
  return (int)(((int64_t)s.count * g + kRows - 1) / kRows);
}

template <int D, int NB, int kKind>
__global__ void __launch_bounds__(kRowThreads, Rows<D, NB, kKind>::kMinCtas)
    paged_rows_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedQuery p,
                      const RowsJoin join) {
  constexpr int kRows = Rows<D, NB, kKind>::kRows;
  constexpr bool kE4m3 = kKind == kRowsE4m3, kStats = kKind == kRowsStats;
  __shared__ int64_t warp_sum[kRowWarps];
  __shared__ int64_t at_batch[kRowWarps];  // batches before sequence at_seq
  __shared__ int at_seq[kRowWarps];
  // four rows of each warp, m and l behind
  __shared__ __align__(16) float red[kRowWarps][4][D + 4];
  constexpr bool kQShared = Rows<D, NB, kKind>::kQShared;
  __shared__ uint4 q_shared[kQShared ? kRowWarps : 1][kQShared ? NB * (D / 32) : 1][32];
  const int g = p.Hq / a.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lg = lane >> 2, lj = lane & 3;
  // ---- this warp's range [u0, u1) of all batches, and the sequence in which it begins
  const int per = (a.B + kRowThreads - 1) / kRowThreads;  // consecutive sequences of a thread
  const int sb0 = min(a.B, (int)threadIdx.x * per), sb1 = min(a.B, sb0 + per);
  int64_t mine = 0;
  bool none = false;  // a sequence without slots
  for (int b = sb0; b < sb1; ++b) {
    const Seq s = paged_seq(a, b);
    none |= seq_batches(s) == 0;
    mine += (int64_t)seq_batches(s) * seq_blocks<kRows>(s, g) * a.H;
  }
  int64_t before = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += x;
  }
  if (lane == 31) warp_sum[warp] = before;
  none = __syncthreads_or(none);
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  before -= mine;
  // CTAs and warps that have a range: every warp of these CTAs, if there are batches for it
  const int ctas =
      (int)max((int64_t)1, min((int64_t)gridDim.x, total / (kRowWarps * kLeastBatches)));
  const int nw = (int)max((int64_t)1, min((int64_t)ctas * kRowWarps, total));
  // the first `wider` ranges have one batch more than `width`
  const int64_t width = total / nw;
  const int wider = (int)(total - width * nw);
  auto range_at = [&](int w) { return width * w + min(w, wider); };
  auto warp_at = [&](int64_t u) {  // whose range holds batch u; nw at the end
    const int64_t x = (width + 1) * wider;
    return (int)(u < x ? u / (width + 1) : width > 0 ? wider + (u - x) / width : wider);
  };
  for (int w = 0; w < kRowWarps; ++w) {
    const int64_t u = range_at(min((int)blockIdx.x * kRowWarps + w, nw));
    if (u < before || u >= before + mine) continue;
    int64_t at = before;
    int b = sb0;
    for (;; ++b) {
      const Seq s = paged_seq(a, b);
      const int64_t n = (int64_t)seq_batches(s) * seq_blocks<kRows>(s, g) * a.H;
      if (u < at + n) break;
      at += n;
    }
    at_seq[w] = b;
    at_batch[w] = at;
  }
  for (int b = blockIdx.x; !kStats && none && b < a.B; b += gridDim.x) {  // their rows are zeros
    const Seq s = paged_seq(a, b);
    if (seq_batches(s) > 0) continue;
    uint4* o = reinterpret_cast<uint4*>(p.out + (int64_t)s.first * p.Hq * D);
    for (int64_t i = threadIdx.x; i < (int64_t)s.count * p.Hq * D / 8; i += kRowThreads)
      o[i] = make_uint4(0, 0, 0, 0);
  }
  __syncthreads();
  const int me = blockIdx.x * kRowWarps + warp;
  if (lane == 0) join.split[me].last = me;
  if (me >= nw || total == 0) return;
  const int64_t u0 = range_at(me), u1 = range_at(me + 1);
  const int mask = (1 << a.page_shift) - 1;
  const int64_t beta_page = (int64_t)a.H << a.page_shift;

  // ---- where the loads are: a set, its slots from e0 up to `end`
  struct {
    Seq s;
    int b, h, r0;       // the set
    int nrows, most;    // its rows, the slots that any of them sees
    int batch, nb;      // batch of the set, batches of the set
    int64_t set0;       // batches before the set
  } at{};
  int64_t left = u1 - u0;  // batches of the range that are not loaded yet
  auto enter = [&]() {     // the set's sizes
    at.nrows = min(kRows, at.s.count * g - at.r0);
    at.most = max(0, at.s.len - at.s.count + (at.r0 + at.nrows - 1) / g + 1);
  };
  at.b = at_seq[warp];
  at.s = paged_seq(a, at.b);
  at.nb = seq_batches(at.s);
  {
    const int64_t in = u0 - at_batch[warp];
    const int nblk = seq_blocks<kRows>(at.s, g);
    const int64_t set = in < (int64_t)INT32_MAX ? (int)in / at.nb : in / at.nb;
    at.h = (int)(set / nblk);
    at.r0 = (int)(set % nblk) * kRows;
    at.batch = (int)(in - set * at.nb);
    at.set0 = u0 - at.batch;
    enter();
  }
  // On to the next batch; true if it is another set's.
  auto advance = [&]() -> bool {
    if (--left == 0 || ++at.batch < at.nb) return false;
    at.set0 += at.nb;
    at.batch = 0;
    at.r0 += kRows;
    if (at.r0 >= at.s.count * g) {
      at.r0 = 0;
      if (++at.h == a.H) {
        at.h = 0;
        do {
          at.s = paged_seq(a, ++at.b);
          at.nb = seq_batches(at.s);
        } while (at.nb == 0);
      }
    }
    enter();
    return true;
  };

  // a lane's part of K (its order of channels is 32 c + 8 lj, of e4m3 64 c + 16 lj) and of V
  constexpr int kKx = kE4m3 ? D / 64 : D / 32;
  constexpr int kVw = kE4m3 ? D / 32 : 1;
  uint4 kx[2][kKx], vx[4][kE4m3 || kStats ? 1 : D / 64];
  uint32_t vq[4][kVw];
  float bias[2];
  float ks = 0.f, vs = 0.f;  // the batch's scales
  // K, V and biases of slots [e0, min(e0 + 16, end)) of a KV-head; slots past the end repeat the
  // last one (their weight is 0, their V zeroed). A batch past what its set's rows see is not
  // loaded.
  auto scale_at = [&](int64_t page, int h, int in) {
    return ((page * a.H + h) << (a.page_shift - 4)) + (in >> 4);
  };
  auto load_k = [&](int h, int pg, int e0, int end) {
    const int in = e0 & mask, most = end - e0 - 1;
    const int64_t page = max(pg, 0);
    const __nv_bfloat16* base = a.K + page * a.s_page + (int64_t)h * a.s_head + 8 * lj;
    if constexpr (kE4m3) {
      const int64_t at = scale_at(page, h, in);
      ks = a.k_scale[at];
      vs = a.v_scale[at];
      // (a batch that is whole takes two additions where `min` takes two products)
      const uint8_t* codes =
          a.K8 + page * a.s_page + in * a.s_slot + (int64_t)h * a.s_head + 16 * lj;
      const uint8_t* row = codes + min(lg, most) * a.s_slot;
#pragma unroll
      for (int c = 0; c < kKx; ++c) kx[0][c] = ld_once(row + 64 * c);
      row = most >= 15 ? row + 8 * a.s_slot : codes + min(lg + 8, most) * a.s_slot;
#pragma unroll
      for (int c = 0; c < kKx; ++c) kx[1][c] = ld_once(row + 64 * c);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = in + min(lg + 8 * i, most);
#pragma unroll
      for (int c = 0; !kE4m3 && c < kKx; ++c) kx[i][c] = ld_once(base + r * a.s_slot + 32 * c);
      bias[i] = pg < 0               ? -INFINITY
                : a.beta != nullptr ? a.beta[page * beta_page + ((int64_t)h << a.page_shift) + r]
                                    : 0.f;
    }
  };
  auto load_v = [&](int h, int pg, int e0, int end) {
    const int in = e0 & mask, most = end - e0 - 1;
    if constexpr (kE4m3) {
      const int64_t page = max(pg, 0);
      constexpr int kLane = D < 256 ? D / 8 : 16;  // contiguous channels of a lane
      const uint8_t* codes =
          a.V8 + page * a.s_page + in * a.s_slot + (int64_t)h * a.s_head + kLane * lg;
      const uint8_t* first = codes + 2 * lj * a.s_slot;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const uint8_t* row = most >= 15 ? first + ((v & 1) + 8 * (v >> 1)) * a.s_slot
                                        : codes + min(2 * lj + (v & 1) + 8 * (v >> 1), most) *
                                                      a.s_slot;
        if constexpr (D == 64) {
          const uint2 x = __ldcs(reinterpret_cast<const uint2*>(row));
          vq[v][0] = x.x;
          vq[v][1] = x.y;
        } else {
#pragma unroll
          for (int x = 0; x < D / 128; ++x) {
            const uint4 y = ld_once(row + 128 * x);
#pragma unroll
            for (int w = 0; w < 4; ++w) vq[v][4 * x + w] = word(y, w);
          }
        }
      }
    } else if constexpr (!kStats) {
      const __nv_bfloat16* base =
          a.V + (int64_t)max(pg, 0) * a.s_page + (int64_t)h * a.s_head + 8 * lg;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = in + min(2 * lj + (v & 1) + 8 * (v >> 1), most);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) vx[v][x] = ld_once(base + r * a.s_slot + 64 * x);
      }
    }
  };
  auto page_at = [&](int b, int e0) { return paged_page(a, a.table + (int64_t)b * a.s_table, e0); };

  float m[NB][2], l[NB][2];   // rows 2 lj, 2 lj + 1 of a block; l: this lane's share
  // O^T: rows 2 lj (+1); channels 64 x + 8 lg + 2 w (+1), of e4m3 those of four_at
  float o[NB][kStats ? 1 : D / 64][4][4];
  // e4m3: what O and the products with q are multiples of, the first one's inverse
  float rho[NB][2], by_rho[NB][2], fq[NB][2];
  // the first of the four channels that groups 2 t and 2 t + 1 (group 4 x + w) hold
  auto four_at = [&](int t) {
    if constexpr (kE4m3 && D == 256) return 128 * (t >> 2) + 16 * lg + 4 * (t & 3);
    return kE4m3 ? D / 8 * lg + 4 * t : 64 * (t >> 1) + 8 * lg + 4 * (t & 1);
  };
  uint4 qf[NB][kQShared ? 1 : D / 32];
  int see[NB][2];  // slots that a row sees
  auto begin_set = [&](const Seq& s, int h, int r0, int nrows) {
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int r = 8 * k + lg;
      const bool ok = r < nrows;
      const int tok = s.first + (r0 + r) / g, qh = h * g + (r0 + r) % g;
      const __nv_bfloat16* qp =
          p.q + (ok ? (int64_t)tok * p.s_q + (int64_t)qh * D : 0) + (kE4m3 ? 16 : 8) * lj;
      if constexpr (kE4m3) {
        // q as fp16, exact but for what lies 2^24 below its row's largest: brought to [2^14, 2^15)
        float top = 0.f;
        uint4 x[D / 32];
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          x[c] = ok ? *reinterpret_cast<const uint4*>(qp + 64 * (c >> 1) + 8 * (c & 1))
                    : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t y = word(x[c], w);
            top = max3(top, fabsf(__uint_as_float(y << 16)),
                       fabsf(__uint_as_float(y & 0xffff0000u)));
          }
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // the exponent's bits; a row with infinities stays as it is
        const int e = (int)(__float_as_uint(top) >> 23);
        const int up = e == 255 ? 0 : min(126, 141 - e);  // by 2^up
        const float by = __uint_as_float((uint32_t)(127 + up) << 23);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          uint32_t y[4];
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t z = word(x[c], w);
            y[w] = f16x2_bits(__floats2half2_rn(__uint_as_float(z << 16) * by,
                                                __uint_as_float(z & 0xffff0000u) * by));
          }
          (kQShared ? q_shared[warp][k * (D / 32) + c][lane] : qf[k][kQShared ? 0 : c]) =
              make_uint4(y[0], y[1], y[2], y[3]);
        }
        const float down = p.scale * __uint_as_float((uint32_t)(127 - up) << 23);
#pragma unroll
        for (int e2 = 0; e2 < 2; ++e2)
          fq[k][e2] = __shfl_sync(0xffffffffu, down, 4 * (2 * lj + e2));
      } else {
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          (kQShared ? q_shared[warp][k * (D / 32) + c][lane] : qf[k][kQShared ? 0 : c]) =
              ok ? *reinterpret_cast<const uint4*>(qp + 32 * c) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * k + 2 * lj + e;
        see[k][e] = rr < nrows ? s.len - s.count + (r0 + rr) / g + 1 : 0;
      }
    }
  };
  auto clear = [&]() {
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      m[k][0] = m[k][1] = -INFINITY;
      l[k][0] = l[k][1] = 0.f;
      rho[k][0] = rho[k][1] = by_rho[k][0] = by_rho[k][1] = 0.f;
#pragma unroll
      for (int x = 0; x < (kStats ? 1 : D / 64); ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[k][x][w][e] = 0.f;
    }
  };
  int64_t page_now = 0;  // kRowsWeigh: page of the batch that is computed, and its set
  int head_now = 0, row_now = 0, rows_now = 0;
  // The batch of slots [e0, end) that kx, vx and bias hold. `then_k` and `then_v` may overwrite
  // them where they are done with; rests: with P's rounding rests.
  auto compute = [&](int e0, int end, bool rests, auto then_k, auto then_v) {
    float c[NB][4];
    const float b0 = bias[0], b1 = bias[1];
    [[maybe_unused]] const float kscale = ks;
    [[maybe_unused]] float vscale = vs;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      float c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) c[k][e] = 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint4 q = kQShared ? q_shared[warp][k * (D / 32) + x][lane] : qf[k][kQShared ? 0 : x];
        if constexpr (kE4m3) {  // half a piece of K
          const uint32_t u0 = word(kx[0][x / 2], x % 2 * 2), u1 = word(kx[1][x / 2], x % 2 * 2);
          const uint32_t w0 = word(kx[0][x / 2], x % 2 * 2 + 1);
          const uint32_t w1 = word(kx[1][x / 2], x % 2 * 2 + 1);
          mma_f16(c[k], f16_of_lower(u0), f16_of_lower(u1), f16_of_upper(u0), f16_of_upper(u1),
                  q.x, q.y);
          mma_f16(c2, f16_of_lower(w0), f16_of_lower(w1), f16_of_upper(w0), f16_of_upper(w1), q.z,
                  q.w);
        } else {
          mma_bf16(c[k], kx[0][x].x, kx[1][x].x, kx[0][x].y, kx[1][x].y, q.x, q.y);
          mma_bf16(c2, kx[0][x].z, kx[1][x].z, kx[0][x].w, kx[1][x].w, q.z, q.w);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) c[k][e] += c2[e];
    }
    then_k();
    // slots whose value does not count: 0 * inf would be NaN
    const int n = end - e0;
    const unsigned dead0 = __ballot_sync(0xffffffffu, b0 == -INFINITY || lg >= n);
    const unsigned dead1 = __ballot_sync(0xffffffffu, b1 == -INFINITY || lg + 8 >= n);
    if (dead0 | dead1) {
#pragma unroll
      for (int v = 0; v < 4; ++v)
        if (((v >> 1 ? dead1 : dead0) >> (4 * (2 * lj + (v & 1)))) & 1)
#pragma unroll
          for (int x = 0; x < (kE4m3 ? kVw : kStats ? 0 : D / 64); ++x)
            if constexpr (kE4m3)
              vq[v][x] = 0;
            else
              vx[v][x] = make_uint4(0, 0, 0, 0);
      if ((dead0 & dead1) == 0xffffffffu) vscale = 0.f;  // (it may be anything)
    }
    [[maybe_unused]] uint32_t hi[NB][2], lo[NB][2];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      float top[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // slot lg + 8 (e / 2), row 2 lj + e % 2
        // (e4m3: factors first, as the product, up to 2^32, times a large scale may pass the largest
        // float where the logit does not)
        const float be = e >> 1 ? b1 : b0;
        const bool ok = e0 + lg + 8 * (e >> 1) < see[k][e & 1] && be != -INFINITY;
        if constexpr (kE4m3)
          c[k][e] = ok ? c[k][e] * (kscale * fq[k][e & 1]) + be : -INFINITY;
        else
          c[k][e] = ok ? c[k][e] * p.scale + be : -INFINITY;
      }
      bool moved = false;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top[e] = fmaxf(c[k][e], c[k][e + 2]);
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1)
          top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], x));
        moved |= top[e] > m[k][e];
      }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float n = fmaxf(m[k][e], top[e]);
          const float f = n == m[k][e] ? 1.f : exp2f((m[k][e] - n) * kLog2e);
          m[k][e] = n;
          l[k][e] *= f;
          // e4m3: rho brings O along, down to the smallest normal float, and O takes the rest. (A rho
          // that stayed above it would be the unit of the weights that follow.)
          bool in_rho = kE4m3;
          float rest = f;
          if (kE4m3 && rho[k][e] > 0.f) {
            const float next = rho[k][e] * f;
            in_rho = next >= 0x1p-126f;
            rest = f * 0x1p126f * rho[k][e];
            rho[k][e] = in_rho ? next : 0x1p-126f;
            by_rho[k][e] = 1.f / rho[k][e];
          }
          if (!kStats && !in_rho) {
#pragma unroll
            for (int x = 0; x < (kStats ? 0 : D / 64); ++x)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                o[k][x][w][e] *= rest;
                o[k][x][w][e + 2] *= rest;
              }
          }
        }
      }
      // e4m3: O is a multiple of rho (at least 2^-126, 0 before anything is seen), and a weight times
      // the batch's scale of V enters as a multiple of it too. rho is raised when one of them would
      // pass 2^8 (and how large they are is looked at where the scale alone does), or when the scale
      // over rho would pass the largest float (no weight but 0 is below 2^-126, so the largest of the
      // row times the scale is 4 rho at least then).
      [[maybe_unused]] float by_v[2] = {1.f, 1.f};
      if constexpr (kE4m3) {
        bool none[2] = {false, false};
        if (__any_sync(0xffffffffu, vscale > 256.f * rho[k][0] || vscale > 256.f * rho[k][1])) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float up =
                top[e] == -INFINITY ? 0.f : vscale * ex2_ftz((top[e] - m[k][e]) * kLog2e);
            none[e] = up == 0.f;  // (the scale over rho may be infinite)
            const bool wide = up > 0.f && vscale * by_rho[k][e] > 3.4e38f;  // for small weights
            if (!(up > 256.f * rho[k][e]) && !wide) continue;
            const float next = fmaxf(up, 0x1p-126f);  // it has an inverse
            const float f = rho[k][e] / next;
            rho[k][e] = next;
            by_rho[k][e] = 1.f / next;
#pragma unroll
            for (int x = 0; x < D / 64; ++x)
#pragma unroll
              for (int w = 0; w < 4; ++w) {
                o[k][x][w][e] *= f;
                o[k][x][w][e + 2] *= f;
              }
          }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) by_v[e] = none[e] ? 0.f : vscale * by_rho[k][e];
      }
      if constexpr (kKind == kRowsWeigh) {  // (a batch lies in one page)
        const int64_t row = (page_now * a.H + head_now) * g + row_now + 8 * k + 2 * lj;
        float* at = p.logits + (row << a.page_shift) + (e0 & mask) + lg;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (page_now >= 0 && 8 * k + 2 * lj + (e & 1) < rows_now && lg + 8 * (e >> 1) < n)
            at[((int64_t)(e & 1) << a.page_shift) + 8 * (e >> 1)] = c[k][e];
      }
      // nothing seen yet: every weight is 2^-inf
      const float by0 = m[k][0] == -INFINITY ? 0.f : m[k][0];
      const float by1 = m[k][1] == -INFINITY ? 0.f : m[k][1];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float x0 = (c[k][2 * i] - by0) * kLog2e, x1 = (c[k][2 * i + 1] - by1) * kLog2e;
        const float w0 = kE4m3 ? ex2_ftz(x0) : exp2f(x0), w1 = kE4m3 ? ex2_ftz(x1) : exp2f(x1);
        l[k][0] += w0;
        l[k][1] += w1;
        if constexpr (kE4m3) {
          const float u0 = w0 * by_v[0], u1 = w1 * by_v[1];
          const __half2 ph = __floats2half2_rn(u0, u1);
          const float2 r = __half22float2(ph);
          hi[k][i] = transpose8(f16x2_bits(ph));
          lo[k][i] = transpose8(f16x2_bits(__floats2half2_rn(u0 - r.x, u1 - r.y)));
        } else if constexpr (!kStats) {
          const __nv_bfloat162 ph = __floats2bfloat162_rn(w0, w1);
          const float2 r = __bfloat1622float2(ph);
          hi[k][i] = transpose8(bf16x2_bits(ph));
          lo[k][i] = transpose8(bf16x2_bits(__floats2bfloat162_rn(w0 - r.x, w1 - r.y)));
        }
      }
    }
    if constexpr (kE4m3) {
#pragma unroll
      for (int w = 0; w < kVw; ++w)
#pragma unroll
        for (int e = 0; e < 2; ++e) {  // four slots' codes of two channels
          const uint32_t first = __byte_perm(vq[0][w], vq[1][w], e ? 0x7362 : 0x5140);
          const uint32_t other = __byte_perm(vq[2][w], vq[3][w], e ? 0x7362 : 0x5140);
          const uint32_t a0 = f16_of_lower(first), a1 = f16_of_upper(first);
          const uint32_t a2 = f16_of_lower(other), a3 = f16_of_upper(other);
#pragma unroll
          for (int k = 0; k < NB; ++k) {
            float (&acc)[4] = o[k][(2 * w + e) / 4][(2 * w + e) % 4];
            mma_f16(acc, a0, a1, a2, a3, hi[k][0], hi[k][1]);
            mma_f16(acc, a0, a1, a2, a3, lo[k][0], lo[k][1]);
          }
        }
    }
    if constexpr (!kE4m3 && !kStats) {
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t v0 = word(vx[0][x], w), v1 = word(vx[1][x], w);
          const uint32_t v2 = word(vx[2][x], w), v3 = word(vx[3][x], w);
          const uint32_t a0 = __byte_perm(v0, v1, 0x5410), a1 = __byte_perm(v0, v1, 0x7632);
          const uint32_t a2 = __byte_perm(v2, v3, 0x5410), a3 = __byte_perm(v2, v3, 0x7632);
#pragma unroll
          for (int k = 0; k < NB; ++k) {
            mma_bf16(o[k][x][w], a0, a1, a2, a3, hi[k][0], hi[k][1]);
            if (rests) mma_bf16(o[k][x][w], a0, a1, a2, a3, lo[k][0], lo[k][1]);
          }
        }
    }
    then_v();
  };

  int pg = page_at(at.b, kBatch * at.batch);
  if (kBatch * at.batch < at.most) {
    load_k(at.h, pg, kBatch * at.batch, at.most);
    load_v(at.h, pg, kBatch * at.batch, at.most);
  }
  while (left > 0) {
    // ---- a set, or this warp's part of it
    const Seq s = at.s;
    const int b = at.b, h = at.h, r0 = at.r0, nrows = at.nrows, most = at.most;
    const int first = at.batch, nb = at.nb;
    const int64_t set0 = at.set0;
    begin_set(s, h, r0, nrows);
    clear();
    head_now = h;
    row_now = r0;
    rows_now = nrows;
    int batch = first;
    for (bool other = false; !other && left > 0; ++batch) {
      page_now = pg;
      other = advance();
      const bool more = left > 0 && kBatch * at.batch < at.most;
      if (left > 0) pg = page_at(at.b, kBatch * at.batch);
      auto then_k = [&]() {
        if (more) load_k(at.h, pg, kBatch * at.batch, at.most);
      };
      auto then_v = [&]() {
        if (more) load_v(at.h, pg, kBatch * at.batch, at.most);
      };
      if (kBatch * batch < most) {
        compute(kBatch * batch, most, true, then_k, then_v);
      } else {
        then_k();
        then_v();
      }
    }
    // An infinite value times a rest of 0 (or below 0) is no infinity any more: once more without
    // the rests, where a sum came out as NaN.
    bool nan = false;
    if constexpr (!kE4m3 && !kStats) {  // (e4m3 has no infinities)
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) nan |= o[k][x][w][e] != o[k][x][w][e];
    }
    if (__any_sync(0xffffffffu, nan)) {
      clear();
#pragma unroll 1
      for (int x = first; x < batch && kBatch * x < most; ++x) {
        const int page = page_at(b, kBatch * x);
        page_now = page;
        load_k(h, page, kBatch * x, most);
        load_v(h, page, kBatch * x, most);
        compute(kBatch * x, most, false, [] {}, [] {});
      }
      if (left > 0 && kBatch * at.batch < at.most) {
        load_k(at.h, pg, kBatch * at.batch, at.most);
        load_v(at.h, pg, kBatch * at.batch, at.most);
      }
    }
    // ---- its rows
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) l[k][e] += __shfl_xor_sync(0xffffffffu, l[k][e], x);
    if constexpr (kE4m3) {
#pragma unroll
      for (int k = 0; k < NB; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int x = 0; x < D / 16; ++x) o[k][x / 4][x % 4][e] *= rho[k][e & 1];
    }
    constexpr bool kKeeps = kKind == kRowsWeigh || kStats;  // rows' (m, 1 / l)
    auto ml_at = [&](int r) -> float2& {
      return p.ml[(int64_t)(s.first + (r0 + r) / g) * p.Hq + h * g + (r0 + r) % g];
    };
    auto out_row = [&](int r) {
      return p.out + ((int64_t)(s.first + (r0 + r) / g) * p.Hq + h * g + (r0 + r) % g) * D;
    };
    // CTAs [cta0, cta1) lie in this set whole
    int cta0 = 0, cta1 = 0;
    if (ctas * kRowWarps == nw) {
      const int w0 = warp_at(set0);
      cta0 = (w0 + (range_at(w0) < set0) + kRowWarps - 1) / kRowWarps;
      cta1 = warp_at(set0 + nb) / kRowWarps;
    }
    if ((int)blockIdx.x >= cta0 && (int)blockIdx.x < cta1) {
      // ---- one part of this CTA: its warps' states, four rows at a time
      const bool begins = range_at(kRowWarps * blockIdx.x) == set0;
      const bool ends = range_at(kRowWarps * (blockIdx.x + 1)) == set0 + nb;
      const int64_t part = 2 * (int64_t)kRowWarps * blockIdx.x + (begins ? 1 : 0);
#pragma unroll
      for (int q = 0; q < 2 * NB; ++q) {
        if (4 * q >= nrows) break;
        if (q > 0) __syncthreads();
        if (lj >> 1 == (q & 1)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float* row = red[warp][2 * (lj & 1) + e];
#pragma unroll
            for (int x = 0; x < (kStats ? 0 : D / 64); ++x) {
              *reinterpret_cast<float4*>(row + four_at(2 * x)) =
                  make_float4(o[q / 2][x][0][e], o[q / 2][x][0][e + 2], o[q / 2][x][1][e],
                              o[q / 2][x][1][e + 2]);
              *reinterpret_cast<float4*>(row + four_at(2 * x + 1)) =
                  make_float4(o[q / 2][x][2][e], o[q / 2][x][2][e + 2], o[q / 2][x][3][e],
                              o[q / 2][x][3][e + 2]);
            }
            if (lg == 0) {
              row[D] = m[q / 2][e];
              row[D + 1] = l[q / 2][e];
            }
          }
        }
        __syncthreads();
        const int nr = min(4, nrows - 4 * q);
        constexpr int kCols = kStats ? 1 : D;
        for (int it = threadIdx.x; it < nr * kCols; it += kRowThreads) {
          const int r = it / kCols, col = it % kCols;
          float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) M = fmaxf(M, red[w][r][D]);
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) {
            // a warp that saw nothing has sums of 0, or of NaN
            const float f = red[w][r][D] == M ? 1.f : exp2f((red[w][r][D] - M) * kLog2e);
            L += f * red[w][r][D + 1];
            if constexpr (!kStats) O += f * red[w][r][col];
          }
          if (begins && ends) {
            if constexpr (!kStats)
              out_row(4 * q + r)[col] = __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
            if constexpr (kKeeps)
              if (col == 0) ml_at(4 * q + r) = make_float2(M, L == 0.f ? 0.f : 1.f / L);
          } else {
            if constexpr (!kStats) join.part_o[(part * kRows + 4 * q + r) * D + col] = O;
            if (col == 0) join.part_ml[part * kRows + 4 * q + r] = make_float2(M, L);
          }
        }
      }
      if (begins && !ends && threadIdx.x == 0)
        join.split[me] =
            RowsSplit{warp_at(set0 + nb - 1), s.first, r0, nrows, h, cta0, cta1, 0};
      return;  // it was all of this CTA's range
    }
    const bool begins = first == 0, ends = batch == nb;
    const int64_t part = 2 * (int64_t)me + (begins ? 1 : 0);
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * k + 2 * lj + e;
        if (r >= nrows) continue;
        if (begins && ends) {
          const float inv = l[k][e] == 0.f ? 0.f : 1.f / l[k][e];
          if constexpr (kKeeps)
            if (lg == 0) ml_at(r) = make_float2(m[k][e], inv);
          __nv_bfloat16* dst = out_row(r);
#pragma unroll
          for (int x = 0; x < (kStats ? 0 : D / 64); ++x) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[i] = bf16x2_bits(
                  __floats2bfloat162_rn(o[k][x][i][e] * inv, o[k][x][i][e + 2] * inv));
            *reinterpret_cast<uint4*>(dst + four_at(2 * x)) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
          float* dst = join.part_o + (part * kRows + r) * D;
#pragma unroll
          for (int x = 0; x < (kStats ? 0 : D / 64); ++x) {
            *reinterpret_cast<float4*>(dst + four_at(2 * x)) = make_float4(
                o[k][x][0][e], o[k][x][0][e + 2], o[k][x][1][e], o[k][x][1][e + 2]);
            *reinterpret_cast<float4*>(dst + four_at(2 * x + 1)) = make_float4(
                o[k][x][2][e], o[k][x][2][e + 2], o[k][x][3][e], o[k][x][3][e + 2]);
          }
          if (lg == 0) join.part_ml[part * kRows + r] = make_float2(m[k][e], l[k][e]);
        }
      }
    if (begins && !ends && lane == 0)
      join.split[me] =
          RowsSplit{warp_at(set0 + nb - 1), s.first, r0, nrows, h, cta0, cta1, 0};
  }
}

// The sets that several warps share. A block looks at kJoinSets warps' sets: those of few parts are
// joined row by row, a warp a row; one of many (there is at most one: it begins once in as many
// warps) by all warps, which share its rows and parts out. What bounds it is one dependent read of
// memory after another, of a microsecond each: the set, m and l of its parts, O.
constexpr int kJoinWarps = 16;
constexpr int kJoinSets = 4;
constexpr int kJoinFew = 8;

template <int D, int kKind>
__global__ void __launch_bounds__(32 * kJoinWarps)
    paged_rows_join_kernel(const RowsJoin join, int warps, int kRows, int g, int Hq,
                           __nv_bfloat16* __restrict__ out, float2* __restrict__ ml) {
  griddep_wait();
  constexpr bool kStats = kKind == kRowsStats;
  constexpr int kPer = D / 32;  // channels of a lane
  __shared__ float red[kJoinWarps][D + 2];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float M, L, O[kPer];
  // Parts of a set: its first warps', then those of its whole CTAs, then its last warps'.
  auto parts_of = [](const RowsSplit& q, int from) {
    return q.last - from + 1 - (kRowWarps - 1) * max(0, q.cta1 - q.cta0);
  };
  auto slot_of = [](const RowsSplit& q, int from, int i) -> int64_t {
    int w = from + i;
    if (q.cta1 > q.cta0 && w > kRowWarps * q.cta0) {
      const int c = w - kRowWarps * q.cta0;  // CTAs, then single warps
      w = kRowWarps * q.cta0 + kRowWarps * min(c, q.cta1 - q.cta0) + max(0, c - (q.cta1 - q.cta0));
    }
    return i == 0 ? 2 * w + 1 : 2 * w;
  };
  // parts i, i + step, ... of n of row r of the set that warp `from` begins, in order
  auto add_up = [&](const RowsSplit& q, int from, int n, int r, int i, int step) {
    M = -INFINITY;
    L = 0.f;
#pragma unroll
    for (int e = 0; e < kPer; ++e) O[e] = 0.f;
    for (int i0 = i; i0 < n; i0 += 32 * step) {
      const int here = min(32, (n - i0 - 1) / step + 1);
      // a lane a part
      const int64_t mine = slot_of(q, from, min(i0 + lane * step, n - 1)) * kRows + r;
      const float2 ml = lane < here ? join.part_ml[mine] : make_float2(-INFINITY, 0.f);
      float m = fmaxf(M, ml.x);
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      const float f = M == m ? 1.f : exp2f((M - m) * kLog2e);
      const float weight = ml.x == m ? 1.f : exp2f((ml.x - m) * kLog2e);
      float sum = lane < here ? weight * ml.y : 0.f;
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      M = m;
      L = L * f + sum;
#pragma unroll
      for (int e = 0; e < kPer; ++e) O[e] *= f;
#pragma unroll 4
      for (int j = 0; !kStats && j < here; ++j) {
        const float v = __shfl_sync(0xffffffffu, weight, j);
        const float* src = join.part_o + __shfl_sync(0xffffffffu, mine, j) * D + kPer * lane;
#pragma unroll
        for (int e = 0; e < kPer; e += kPer < 4 ? 2 : 4) {
          float x[4];
          if constexpr (kPer < 4)
            *reinterpret_cast<float2*>(x) = *reinterpret_cast<const float2*>(src + e);
          else
            *reinterpret_cast<float4*>(x) = *reinterpret_cast<const float4*>(src + e);
#pragma unroll
          for (int y = 0; y < (kPer < 4 ? 2 : 4); ++y) O[e + y] += v * x[y];
        }
      }
    }
  };
  auto write = [&](const RowsSplit& q, int r) {
    const float inv = L == 0.f ? 0.f : 1.f / L;
    const int row = q.row0 + r;
    const int64_t to = (int64_t)(q.token0 + row / g) * Hq + q.h * g + row % g;
    if constexpr (kKind == kRowsWeigh || kStats)
      if (lane == 0) ml[to] = make_float2(M, inv);
    if constexpr (kStats) return;
    __nv_bfloat162* dst = reinterpret_cast<__nv_bfloat162*>(out + to * D + kPer * lane);
#pragma unroll
    for (int e = 0; e < kPer; e += 2)
      dst[e / 2] = __floats2bfloat162_rn(O[e] * inv, O[e + 1] * inv);
  };
  // lanes 0 .. 3 hold the sets of the block's warps
  const int first = blockIdx.x * kJoinSets;
  RowsSplit mine{-1, 0, 0, 0, 0, 0, 0, 0};
  if (lane < kJoinSets && first + lane < warps) mine = join.split[first + lane];
  unsigned todo = __ballot_sync(0xffffffffu, mine.last > first + lane);
  int task = warp, large = -1;
  RowsSplit q;
#pragma unroll 1
  while (todo != 0) {  // (one loop for all of it: the code is fetched anew at every launch)
    const int k = __ffs(todo) - 1, from = first + k;
    todo &= todo - 1;
    q.last = __shfl_sync(0xffffffffu, mine.last, k);
    q.token0 = __shfl_sync(0xffffffffu, mine.token0, k);
    q.row0 = __shfl_sync(0xffffffffu, mine.row0, k);
    q.rows = __shfl_sync(0xffffffffu, mine.rows, k);
    q.h = __shfl_sync(0xffffffffu, mine.h, k);
    q.cta0 = __shfl_sync(0xffffffffu, mine.cta0, k);
    q.cta1 = __shfl_sync(0xffffffffu, mine.cta1, k);
    const int parts = parts_of(q, from);
    const int shares = parts > kJoinFew ? max(1, kJoinWarps / q.rows) : 1;  // of a row's parts
    for (; task < q.rows * shares; task += kJoinWarps) {
      add_up(q, from, parts, task / shares, task % shares, shares);
      if (shares == 1) {
        write(q, task);
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e) red[task][kPer * lane + e] = O[e];
        if (lane == 0) {
          red[task][D] = M;
          red[task][D + 1] = L;
        }
      }
    }
    task -= q.rows * shares;
    if (shares > 1) large = k;
  }
  if (large < 0) return;
  __syncthreads();
  q.rows = __shfl_sync(0xffffffffu, mine.rows, large);
  if (warp >= q.rows) return;
  q.token0 = __shfl_sync(0xffffffffu, mine.token0, large);
  q.row0 = __shfl_sync(0xffffffffu, mine.row0, large);
  q.h = __shfl_sync(0xffffffffu, mine.h, large);
  const int shares = kJoinWarps / q.rows;
  const float* sums = red[warp * shares];
  M = -INFINITY;
#pragma unroll 1
  for (int i = 0; i < shares; ++i) M = fmaxf(M, sums[i * (D + 2) + D]);
  L = 0.f;
#pragma unroll
  for (int e = 0; e < kPer; ++e) O[e] = 0.f;
#pragma unroll 2
  for (int i = 0; i < shares; ++i) {
    const float* x = sums + i * (D + 2);
    const float v = x[D] == M ? 1.f : exp2f((x[D] - M) * kLog2e);
    L += v * x[D + 1];
#pragma unroll
    for (int e = 0; e < kPer; ++e) O[e] += v * x[kPer * lane + e];
  }
  write(q, warp);
}

template <int D, int NB, int kKind>
struct RowsLaunch {
  using Form = Rows<D, NB, kKind>;
  static int ctas(int num_sms) { return num_sms * Form::kMinCtas; }
  static size_t bytes(int num_sms) {
    const size_t parts = (size_t)2 * ctas(num_sms) * kRowWarps * Form::kRows;
    return parts * (D * sizeof(float) + sizeof(float2)) +
           (size_t)ctas(num_sms) * kRowWarps * sizeof(RowsSplit);
  }
  static cudaError_t run(const PagedArgs& a, const PagedQuery& p, void* ws, int num_sms,
                         cudaStream_t s) {
    const int warps = ctas(num_sms) * kRowWarps, rows = Form::kRows;
    RowsJoin join;
    join.part_o = static_cast<float*>(ws);
    join.part_ml = reinterpret_cast<float2*>(join.part_o + (int64_t)2 * warps * rows * D);
    join.split = reinterpret_cast<RowsSplit*>(join.part_ml + (int64_t)2 * warps * rows);
    paged_rows_kernel<D, NB, kKind><<<ctas(num_sms), kRowThreads, 0, s>>>(a, p, join);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_chained(paged_rows_join_kernel<D, kKind>,
                          dim3((warps + kJoinSets - 1) / kJoinSets), dim3(32 * kJoinWarps), 0, s, 1,
                          join, warps, rows, p.Hq / a.H, p.Hq, p.out, p.ml);
  }
};

// Calls f with the form that serves d channels and so many rows per sequence and KV-head (on
// average: any form serves any call): a block of 16 that is half empty costs 15% (4 x 60,000 slots
// of 128 channels: 51 us against 41 to 45), two blocks of 8 read everything twice. 16 rows of 256
// channels do not fit a thread's registers beside their K and V.
template <int kKind, class F>
auto rows_form(int d, int rows, F f) {
  const bool two = rows > 8;
  if (d == 64) return two ? f(RowsLaunch<64, 2, kKind>()) : f(RowsLaunch<64, 1, kKind>());
  if (d == 128) return two ? f(RowsLaunch<128, 2, kKind>()) : f(RowsLaunch<128, 1, kKind>());
  return f(RowsLaunch<256, 1, kKind>());
}


}  // namespace

}  // namespace still
