// The paged key-value cache: append (with the base model's RoPE) and attention of few rows.
#include <algorithm>

#include "launch.cuh"
#include "paged_dev.cuh"

namespace still {

namespace {

// ----------------------------------------------------------------- append
//
// Row x of token i (slot j, position p = j + offset) goes to its page, keys and queries rotated in
// pairs (m, m + d/2) by the angle p w_m (the base model's RoPE). Angles are integers: p * turns[m]
// modulo 2^64 is the fraction of a turn, and whole turns cost nothing. turns[m] has the 53 bits of
// a double, 2^-22 rad at positions of 2^31 and less in proportion below; the fraction in fp32,
// 2^-25 turns, adds as much. The sines and cosines of a token are formed once, in shared memory,
// and serve all its heads.
//
// Memory bounds it: rows are read and written once. Two tokens a CTA: 8,192 tokens of 32 + 8 + 8
// heads of 128 channels in 37 us (201 MB: 5.5 TB/s, 0.81 of a copy), against 39 with four or one
// and 41 with eight, whose chain of look-ups and angles fewer other CTAs cover. Asking for the
// rows before the look-ups: 39 to 41.
constexpr int kAppendThreads = 256;  // at most
constexpr int kAppendTokens = 2;  // most tokens of a CTA

__global__ void __launch_bounds__(kAppendThreads)
    paged_append_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedAppend p,
                        const __grid_constant__ RopeTurns w, int tokens) {
  extern __shared__ float2 cs[];  // [tokens][d / 2] (cos, sin)
  __shared__ int page[kAppendTokens], in_page[kAppendTokens];
  __shared__ long long pos[kAppendTokens];
  const int i0 = blockIdx.x * tokens, nt = min(tokens, a.n - i0);
  const int half = a.d / 2;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (warp < nt) {  // a warp looks up where a token goes
    const int i = i0 + warp;
    int b = i;  // the last sequence that begins at or before token i
    if (a.cu_new != nullptr) {
      b = 0;
      for (int n = a.B; n > 1;) {  // among n from b on, 32 at a time
        const int apart = (n + 31) / 32;
        const bool before = lane * apart < n && a.cu_new[b + lane * apart] <= i;
        const int k = max(0, 31 - __clz(__ballot_sync(0xffffffffu, before)));
        b += k * apart;
        n = min(apart, n - k * apart);
      }
    }
    if (lane == 0) {
      const long long offset = a.pos_offset != nullptr ? a.pos_offset[b] : 0;
      const Seq s = paged_seq(a, b);
      const int at = i - s.first;
      const int j = s.len - s.count + at;
      int pg = -1;
      if (at >= 0 && at < s.count && j >= 0)
        pg = paged_page(a, a.table + (int64_t)b * a.s_table, j);
      page[warp] = pg;
      in_page[warp] = j & ((1 << a.page_shift) - 1);
      pos[warp] = j + offset;
    }
  }
  __syncthreads();
  if (p.rotate) {
    for (int x = threadIdx.x; x < nt * half; x += blockDim.x) {
      const unsigned long long t = (unsigned long long)pos[x / half] * w.turns[x % half];
      float sn, cn;  // of pi * y, y = twice the signed fraction of a turn
      sincospif((float)(int)(t >> 32) * 0x1p-31f, &sn, &cn);
      cs[x] = make_float2(cn, sn);
    }
    __syncthreads();
  }
  const int lanes = a.d / 16;  // threads of a row: 8 channels of each half
  const int rows = p.Hq + 2 * a.H;
  for (int x = threadIdx.x; x < nt * rows * lanes; x += blockDim.x) {
    const int c = x % lanes * 8, r = x / lanes % rows, t = x / lanes / rows;
    const int64_t i = i0 + t;
    const int pg = page[t];
    const bool query = r < p.Hq, key = !query && r < p.Hq + a.H;
    const int h = query ? r : key ? r - p.Hq : r - p.Hq - a.H;
    const __nv_bfloat16* src = (query ? p.q + i * p.s_q : key ? p.k + i * p.s_k : p.v + i * p.s_v) +
                               (int64_t)h * a.d + c;
    __nv_bfloat16* dst;
    if (query) {
      dst = p.q_out + (i * p.Hq + h) * a.d + c;
    } else {
      if (pg < 0) continue;
      dst = (key ? a.K : a.V) + (int64_t)pg * a.s_page + (int64_t)in_page[t] * a.s_slot +
            (int64_t)h * a.s_head + c;
      if (key && c == 0 && a.beta != nullptr)
        a.beta[(((int64_t)pg * a.H + h) << a.page_shift) + in_page[t]] =
            p.beta != nullptr ? p.beta[i * a.H + h] : 0.f;
    }
    uint4 lo = *reinterpret_cast<const uint4*>(src);
    uint4 hi = *reinterpret_cast<const uint4*>(src + half);
    if (p.rotate && (query || key)) {
      __nv_bfloat162* l = reinterpret_cast<__nv_bfloat162*>(&lo);
      __nv_bfloat162* u = reinterpret_cast<__nv_bfloat162*>(&hi);
      const float2* ang = cs + t * half + c;
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const float2 x0 = __bfloat1622float2(l[m]), x1 = __bfloat1622float2(u[m]);
        const float2 e = ang[2 * m], o = ang[2 * m + 1];
        l[m] = __floats2bfloat162_rn(x0.x * e.x - x1.x * e.y, x0.y * o.x - x1.y * o.y);
        u[m] = __floats2bfloat162_rn(x1.x * e.x + x0.x * e.y, x1.y * o.x + x0.y * o.y);
      }
    }
    *reinterpret_cast<uint4*>(dst) = lo;
    *reinterpret_cast<uint4*>(dst + half) = hi;
  }
}

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
// Memory bounds the large calls: the 24 sequences are 1.0 GB, 5.95 TB/s and 0.88 of a copy, with
// the mma.sync pipe at 12%, so the tensor cores of tcgen05 would have nothing to gain. Small calls
// are the latency of a chain of reads (lengths, table, K and V) and of the second launch: 32 us
// for 8 sequences, of which 16 are memory.
constexpr int kRowWarps = 4;  // of a CTA
constexpr int kRowThreads = 32 * kRowWarps;
constexpr int kBatch = 16;      // slots
constexpr int kLeastBatches = 2;  // of a range, on average, where a call has few batches

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
STILL_DEV uint4 ld_once(const __nv_bfloat16* p) {
  return __ldcs(reinterpret_cast<const uint4*>(p));
}
STILL_DEV uint32_t word(const uint4& v, int i) {
  return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
}

// NB: blocks of 8 rows of a set.
template <int D, int NB>
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

template <int D, int NB>
__global__ void __launch_bounds__(kRowThreads, Rows<D, NB>::kMinCtas)
    paged_rows_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedQuery p,
                      const RowsJoin join) {
  constexpr int kRows = Rows<D, NB>::kRows;
  __shared__ int64_t warp_sum[kRowWarps];
  __shared__ int64_t at_batch[kRowWarps];  // batches before sequence at_seq
  __shared__ int at_seq[kRowWarps];
  // four rows of each warp, m and l behind
  __shared__ __align__(16) float red[kRowWarps][4][D + 4];
  constexpr bool kQShared = Rows<D, NB>::kQShared;
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
  for (int b = blockIdx.x; none && b < a.B; b += gridDim.x) {  // their rows are zeros
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

  uint4 kx[2][D / 32], vx[4][D / 64];
  float bias[2];
  // K, V and biases of slots [e0, min(e0 + 16, end)) of a KV-head; slots past the end repeat the
  // last one (their weight is 0, their V zeroed). A batch past what its set's rows see is not
  // loaded.
  auto load_k = [&](int h, int pg, int e0, int end) {
    const int in = e0 & mask, most = end - e0 - 1;
    const int64_t page = max(pg, 0);
    const __nv_bfloat16* base = a.K + page * a.s_page + (int64_t)h * a.s_head + 8 * lj;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = in + min(lg + 8 * i, most);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) kx[i][c] = ld_once(base + r * a.s_slot + 32 * c);
      bias[i] = pg < 0               ? -INFINITY
                : a.beta != nullptr ? a.beta[page * beta_page + ((int64_t)h << a.page_shift) + r]
                                    : 0.f;
    }
  };
  auto load_v = [&](int h, int pg, int e0, int end) {
    const int in = e0 & mask, most = end - e0 - 1;
    const __nv_bfloat16* base =
        a.V + (int64_t)max(pg, 0) * a.s_page + (int64_t)h * a.s_head + 8 * lg;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int r = in + min(2 * lj + (v & 1) + 8 * (v >> 1), most);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) vx[v][x] = ld_once(base + r * a.s_slot + 64 * x);
    }
  };
  auto page_at = [&](int b, int e0) { return paged_page(a, a.table + (int64_t)b * a.s_table, e0); };

  float m[NB][2], l[NB][2];   // rows 2 lj, 2 lj + 1 of a block; l: this lane's share
  float o[NB][D / 64][4][4];  // O^T: channels 64 x + 8 lg + 2 w (+1), rows 2 lj (+1)
  uint4 qf[NB][kQShared ? 1 : D / 32];
  int see[NB][2];  // slots that a row sees
  auto begin_set = [&](const Seq& s, int h, int r0, int nrows) {
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      const int r = 8 * k + lg;
      const bool ok = r < nrows;
      const int tok = s.first + (r0 + r) / g, qh = h * g + (r0 + r) % g;
      const __nv_bfloat16* qp = p.q + (ok ? (int64_t)tok * p.s_q + (int64_t)qh * D : 0) + 8 * lj;
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
        (kQShared ? q_shared[warp][k * (D / 32) + c][lane] : qf[k][kQShared ? 0 : c]) =
            ok ? *reinterpret_cast<const uint4*>(qp + 32 * c) : make_uint4(0, 0, 0, 0);
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
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[k][x][w][e] = 0.f;
    }
  };
  // The batch of slots [e0, end) that kx, vx and bias hold. `then_k` and `then_v` may overwrite
  // them where they are done with; rests: with P's rounding rests.
  auto compute = [&](int e0, int end, bool rests, auto then_k, auto then_v) {
    float c[NB][4];
    const float b0 = bias[0], b1 = bias[1];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      float c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < 4; ++e) c[k][e] = 0.f;
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint4 q = kQShared ? q_shared[warp][k * (D / 32) + x][lane] : qf[k][kQShared ? 0 : x];
        mma_bf16(c[k], kx[0][x].x, kx[1][x].x, kx[0][x].y, kx[1][x].y, q.x, q.y);
        mma_bf16(c2, kx[0][x].z, kx[1][x].z, kx[0][x].w, kx[1][x].w, q.z, q.w);
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
          for (int x = 0; x < D / 64; ++x) vx[v][x] = make_uint4(0, 0, 0, 0);
    }
    uint32_t hi[NB][2], lo[NB][2];
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      float top[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // slot lg + 8 (e / 2), row 2 lj + e % 2
        const float be = e >> 1 ? b1 : b0;
        const bool ok = e0 + lg + 8 * (e >> 1) < see[k][e & 1] && be != -INFINITY;
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
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              o[k][x][w][e] *= f;
              o[k][x][w][e + 2] *= f;
            }
        }
      }
      // nothing seen yet: every weight is 2^-inf
      const float by0 = m[k][0] == -INFINITY ? 0.f : m[k][0];
      const float by1 = m[k][1] == -INFINITY ? 0.f : m[k][1];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float w0 = exp2f((c[k][2 * i] - by0) * kLog2e);
        const float w1 = exp2f((c[k][2 * i + 1] - by1) * kLog2e);
        l[k][0] += w0;
        l[k][1] += w1;
        const __nv_bfloat162 ph = __floats2bfloat162_rn(w0, w1);
        const float2 r = __bfloat1622float2(ph);
        hi[k][i] = transpose8(bf16x2_bits(ph));
        lo[k][i] = transpose8(bf16x2_bits(__floats2bfloat162_rn(w0 - r.x, w1 - r.y)));
      }
    }
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
    int batch = first;
    for (bool other = false; !other && left > 0; ++batch) {
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
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int e = 0; e < 4; ++e) nan |= o[k][x][w][e] != o[k][x][w][e];
    if (__any_sync(0xffffffffu, nan)) {
      clear();
#pragma unroll 1
      for (int x = first; x < batch && kBatch * x < most; ++x) {
        const int page = page_at(b, kBatch * x);
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
            for (int x = 0; x < D / 64; ++x) {
              float* dst = row + 64 * x + 8 * lg;
              *reinterpret_cast<float4*>(dst) =
                  make_float4(o[q / 2][x][0][e], o[q / 2][x][0][e + 2], o[q / 2][x][1][e],
                              o[q / 2][x][1][e + 2]);
              *reinterpret_cast<float4*>(dst + 4) =
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
        for (int it = threadIdx.x; it < nr * D; it += kRowThreads) {
          const int r = it / D, col = it % D;
          float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) M = fmaxf(M, red[w][r][D]);
#pragma unroll
          for (int w = 0; w < kRowWarps; ++w) {
            // a warp that saw nothing has sums of 0, or of NaN
            const float f = red[w][r][D] == M ? 1.f : exp2f((red[w][r][D] - M) * kLog2e);
            L += f * red[w][r][D + 1];
            O += f * red[w][r][col];
          }
          if (begins && ends) {
            out_row(4 * q + r)[col] = __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
          } else {
            join.part_o[(part * kRows + 4 * q + r) * D + col] = O;
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
          __nv_bfloat16* dst = out_row(r) + 8 * lg;
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
              w[i] = bf16x2_bits(
                  __floats2bfloat162_rn(o[k][x][i][e] * inv, o[k][x][i][e + 2] * inv));
            *reinterpret_cast<uint4*>(dst + 64 * x) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
          float* dst = join.part_o + (part * kRows + r) * D + 8 * lg;
#pragma unroll
          for (int x = 0; x < D / 64; ++x) {
            *reinterpret_cast<float4*>(dst + 64 * x) = make_float4(
                o[k][x][0][e], o[k][x][0][e + 2], o[k][x][1][e], o[k][x][1][e + 2]);
            *reinterpret_cast<float4*>(dst + 64 * x + 4) = make_float4(
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

template <int D>
__global__ void __launch_bounds__(32 * kJoinWarps)
    paged_rows_join_kernel(const RowsJoin join, int warps, int kRows, int g, int Hq,
                           __nv_bfloat16* __restrict__ out) {
  griddep_wait();
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
      for (int j = 0; j < here; ++j) {
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
    __nv_bfloat162* dst = reinterpret_cast<__nv_bfloat162*>(
        out + ((int64_t)(q.token0 + row / g) * Hq + q.h * g + row % g) * D + kPer * lane);
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

template <int D, int NB>
struct RowsLaunch {
  static int ctas(int num_sms) { return num_sms * Rows<D, NB>::kMinCtas; }
  static size_t bytes(int num_sms) {
    const size_t parts = (size_t)2 * ctas(num_sms) * kRowWarps * Rows<D, NB>::kRows;
    return parts * (D * sizeof(float) + sizeof(float2)) +
           (size_t)ctas(num_sms) * kRowWarps * sizeof(RowsSplit);
  }
  static cudaError_t run(const PagedArgs& a, const PagedQuery& p, void* ws, int num_sms,
                         cudaStream_t s) {
    const int warps = ctas(num_sms) * kRowWarps, rows = Rows<D, NB>::kRows;
    RowsJoin join;
    join.part_o = static_cast<float*>(ws);
    join.part_ml = reinterpret_cast<float2*>(join.part_o + (int64_t)2 * warps * rows * D);
    join.split = reinterpret_cast<RowsSplit*>(join.part_ml + (int64_t)2 * warps * rows);
    paged_rows_kernel<D, NB><<<ctas(num_sms), kRowThreads, 0, s>>>(a, p, join);
    const cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return e;
    return launch_chained(paged_rows_join_kernel<D>, dim3((warps + kJoinSets - 1) / kJoinSets),
                          dim3(32 * kJoinWarps), 0, s, 1, join, warps, rows, p.Hq / a.H, p.Hq,
                          p.out);
  }
};

// Calls f with the form that serves d channels and so many rows per sequence and KV-head (on
// average: any form serves any call): a block of 16 that is half empty costs 15% (4 x 60,000 slots
// of 128 channels: 51 us against 41 to 45), two blocks of 8 read everything twice. 16 rows of 256
// channels do not fit a thread's registers beside their K and V.
template <class F>
auto rows_form(int d, int rows, F f) {
  const bool two = rows > 8;
  if (d == 64) return two ? f(RowsLaunch<64, 2>()) : f(RowsLaunch<64, 1>());
  if (d == 128) return two ? f(RowsLaunch<128, 2>()) : f(RowsLaunch<128, 1>());
  return f(RowsLaunch<256, 1>());
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs& a, const PagedAppend& p, const RopeTurns& turns,
                                int num_sms, cudaStream_t s) {
  const int tokens = std::max(1, std::min(kAppendTokens, a.n / (4 * num_sms)));
  const size_t smem = p.rotate ? (size_t)tokens * (a.d / 2) * sizeof(float2) : 0;
  // Half the threads where two tokens have no more than 256 pieces (16 channels each): the compact
  // slots of 8 KV-heads of 128 channels, 8 x 1,311 of them, take 19.1 us against 20.5 with twice
  // the threads; 32 query heads beside them, 8,192 tokens, 37.2 against 36.8.
  const int pieces = kAppendTokens * (p.Hq + 2 * a.H) * (a.d / 16);
  const int threads = pieces <= kAppendThreads ? 128 : kAppendThreads;
  paged_append_kernel<<<(a.n + tokens - 1) / tokens, threads, smem, s>>>(a, p, turns, tokens);
  return cudaGetLastError();
}

int paged_mean_rows(const PagedArgs& a, int Hq) {
  return (int)(((int64_t)a.n * (Hq / a.H) + a.B - 1) / a.B);
}

size_t paged_rows_workspace(int num_sms) {
  size_t most = 0;
  for (int d : {64, 128, 256})
    for (int rows : {8, 16})
      most = std::max(most, rows_form(d, rows, [&](auto form) { return form.bytes(num_sms); }));
  return most;
}

cudaError_t launch_paged_rows(const PagedArgs& a, const PagedQuery& p, void* ws, int num_sms,
                              cudaStream_t s) {
  return rows_form(a.d, paged_mean_rows(a, p.Hq),
                   [&](auto form) { return form.run(a, p, ws, num_sms, s); });
}

}  // namespace still
