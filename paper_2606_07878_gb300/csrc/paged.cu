// The paged key-value cache: append (with the base model's RoPE) and attention of few rows.
#include <algorithm>

#include "launch.cuh"
#include "paged_dev.cuh"

namespace still {

namespace {

// ----------------------------------------------------------------- append
//
// Row x of token i (slot j, position p = j + offset) goes to its page, keys and queries rotated in
// pairs (m, m + d/2) by the angle p w_m (the base model's RoPE). Angles are exact in integers:
// p * turns[m] modulo 2^64 is the fraction of a turn, whatever p, and its upper half loses 2^-32
// turns. The sines and cosines of a token are formed once, in shared memory, and serve all its
// heads.
constexpr int kAppendThreads = 256;
constexpr int kAppendTokens = 8;  // most tokens of a CTA

__global__ void __launch_bounds__(kAppendThreads)
    paged_append_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedAppend p,
                        const __grid_constant__ RopeTurns w, int tokens) {
  extern __shared__ float2 cs[];  // [tokens][d / 2] (cos, sin)
  __shared__ int page[kAppendTokens], in_page[kAppendTokens];
  __shared__ long long pos[kAppendTokens];
  const int i0 = blockIdx.x * tokens, nt = min(tokens, a.n - i0);
  const int half = a.d / 2;
  if (threadIdx.x < nt) {
    const int i = i0 + threadIdx.x;
    int b = i;  // the last sequence that begins at or before token i
    if (a.cu_new != nullptr) {
      int lo = 0, hi = a.B;
      while (lo + 1 < hi) {
        const int mid = (lo + hi) / 2;
        if (a.cu_new[mid] <= i)
          lo = mid;
        else
          hi = mid;
      }
      b = lo;
    }
    const Seq s = paged_seq(a, b);
    const int at = i - s.first;
    const int j = s.len - s.count + at;
    int pg = -1;
    if (at >= 0 && at < s.count && j >= 0) pg = paged_page(a, a.table + (int64_t)b * a.s_table, j);
    page[threadIdx.x] = pg;
    in_page[threadIdx.x] = j & ((1 << a.page_shift) - 1);
    pos[threadIdx.x] = j + (a.pos_offset != nullptr ? a.pos_offset[b] : 0);
  }
  __syncthreads();
  if (p.rotate) {
    for (int x = threadIdx.x; x < nt * half; x += kAppendThreads) {
      const unsigned long long t = (unsigned long long)pos[x / half] * w.turns[x % half];
      float sn, cn;  // of pi * y, y = twice the signed fraction of a turn
      sincospif((float)(int)(t >> 32) * 0x1p-31f, &sn, &cn);
      cs[x] = make_float2(cn, sn);
    }
    __syncthreads();
  }
  const int lanes = a.d / 16;  // threads of a row: 8 channels of each half
  const int rows = p.Hq + 2 * a.H;
  for (int x = threadIdx.x; x < nt * rows * lanes; x += kAppendThreads) {
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
// Work: a set is a sequence's KV-head and block of 8 or 16 rows; its slots are cut into units of
// 64, and all units of all sets, one after another, into equal ranges, one per CTA, from lengths
// that the kernel itself adds up. A set that lies in one range is written by its CTA; the parts of
// another meet in the workspace, and the CTA that brings the last one joins them in their order, so
// that the result does not depend on who that is. No CTA waits for another.
constexpr int kRowWarps = 4;
constexpr int kRowThreads = 32 * kRowWarps;
constexpr int kUnit = 16 * kRowWarps;  // slots

// c (16 x 8) += a (16 x 16 bf16) b (16 x 8 bf16)
STILL_DEV void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                        uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, "
      "{%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// The transpose of an 8 x 8 matrix of 16-bit values: lane i holds row i / 4, columns 2 (i % 4), + 1.
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
  static constexpr int kPart = kRows * (D + 2);  // floats of a part: O rows, then m, l
  static constexpr int kMinCtas = D == 64 ? (NB == 1 ? 5 : 4) : D == 128 ? (NB == 1 ? 3 : 2) : 2;
};

struct RowsJoin {
  float* parts = nullptr;  // [2 x CTAs][Rows::kPart]: what CTA c continues (2 c), begins (2 c + 1)
  int* arrived = nullptr;  // [CTAs], zero between calls
};

// Units of a sequence's sets, and their number per KV-head.
STILL_DEV int seq_units(const Seq& s) { return s.count > 0 ? (s.len + kUnit - 1) / kUnit : 0; }
template <int kRows>
STILL_DEV int seq_blocks(const Seq& s, int g) {
  return (int)(((int64_t)s.count * g + kRows - 1) / kRows);
}

template <int D, int NB>
__global__ void __launch_bounds__(kRowThreads, Rows<D, NB>::kMinCtas)
    paged_rows_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedQuery p,
                      const RowsJoin join) {
  using R = Rows<D, NB>;
  constexpr int kRows = R::kRows;
  __shared__ __align__(16) float red[kRowWarps][8][D + 4];  // O rows of a block, m and l behind
  __shared__ int64_t warp_sum[kRowWarps];
  __shared__ int64_t at_unit;  // units before sequence at_seq
  __shared__ int at_seq, is_last;
  const int g = p.Hq / a.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lg = lane >> 2, lj = lane & 3;
  // ---- this CTA's range [u0, u1) of all units, and the sequence in which it begins
  const int per = (a.B + kRowThreads - 1) / kRowThreads;  // consecutive sequences of a thread
  const int sb0 = min(a.B, (int)threadIdx.x * per), sb1 = min(a.B, sb0 + per);
  int64_t mine = 0;
  for (int b = sb0; b < sb1; ++b) {
    const Seq s = paged_seq(a, b);
    mine += (int64_t)seq_units(s) * seq_blocks<kRows>(s, g) * a.H;
  }
  int64_t before = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += x;
  }
  if (lane == 31) warp_sum[warp] = before;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kRowWarps; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  before -= mine;
  const int nct = (int)min((int64_t)gridDim.x, total);
  // sequences without slots: zeros
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const Seq s = paged_seq(a, b);
    if (seq_units(s) > 0) continue;
    uint4* o = reinterpret_cast<uint4*>(p.out + (int64_t)s.first * p.Hq * D);
    for (int64_t i = threadIdx.x; i < (int64_t)s.count * p.Hq * D / 8; i += kRowThreads)
      o[i] = make_uint4(0, 0, 0, 0);
  }
  if ((int)blockIdx.x >= nct) return;
  const int64_t u0 = total * blockIdx.x / nct, u1 = total * (blockIdx.x + 1) / nct;
  if (u0 >= before && u0 < before + mine) {
    int b = sb0;
    for (;; ++b) {
      const Seq s = paged_seq(a, b);
      const int64_t n = (int64_t)seq_units(s) * seq_blocks<kRows>(s, g) * a.H;
      if (u0 < before + n) break;
      before += n;
    }
    at_seq = b;
    at_unit = before;
  }
  __syncthreads();
  int b = at_seq;
  int64_t seq_u = at_unit;  // first unit of sequence b
  const int mask = (1 << a.page_shift) - 1;
  const int64_t beta_page = (int64_t)a.H << a.page_shift;

  for (int64_t u = u0; u < u1;) {
    // ---- the set of unit u: sequence b, KV-head h, block rb; its units [su, su + nu)
    Seq s = paged_seq(a, b);
    int nu = seq_units(s), nblk = seq_blocks<kRows>(s, g);
    while (u >= seq_u + (int64_t)nu * nblk * a.H) {
      seq_u += (int64_t)nu * nblk * a.H;
      s = paged_seq(a, ++b);
      nu = seq_units(s);
      nblk = seq_blocks<kRows>(s, g);
    }
    const int64_t set = (u - seq_u) / nu;
    const int h = (int)(set / nblk), r0 = (int)(set % nblk) * kRows;
    const int64_t su = seq_u + set * nu;
    const int ua = (int)(u - su), ub = (int)(min(u1, su + nu) - su);
    const int nrows = min(kRows, s.count * g - r0);
    const int past = s.len - s.count;  // token i sees slots up to past + i
    const int most = max(0, past + (r0 + nrows - 1) / g + 1);
    const int end = min(ub * kUnit, most);
    const int32_t* table = a.table + (int64_t)b * a.s_table;
    const __nv_bfloat16* Kh = a.K + (int64_t)h * a.s_head + 8 * lj;
    const __nv_bfloat16* Vh = a.V + (int64_t)h * a.s_head + 8 * lg;
    const float* Bh = a.beta != nullptr ? a.beta + ((int64_t)h << a.page_shift) : nullptr;
    int see[NB][2];
#pragma unroll
    for (int k = 0; k < NB; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * k + 2 * lj + e;
        see[k][e] = r < nrows ? past + (r0 + r) / g + 1 : 0;
      }
    uint4 kx[2][D / 32], vx[4][D / 64];
    float bias[2];
    int kpage = 0;  // page of the slots in kx
    auto page_of = [&](int e0) { return e0 < end ? paged_page(a, table, e0) : -1; };
    // Slots past the end repeat the last one (their weight is 0, their V zeroed).
    auto load_k = [&](int e0, int pg) {
      const int64_t at = (int64_t)max(pg, 0);
      const int in = e0 & mask, left = end - e0;
      const __nv_bfloat16* base = Kh + at * a.s_page;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int r = in + min(lg + 8 * i, left - 1);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) kx[i][c] = ld_once(base + r * a.s_slot + 32 * c);
        bias[i] = pg < 0 ? -INFINITY : Bh != nullptr ? Bh[at * beta_page + r] : 0.f;
      }
    };
    auto load_v = [&](int e0, int pg) {
      const int in = e0 & mask, left = end - e0;
      const __nv_bfloat16* base = Vh + (int64_t)max(pg, 0) * a.s_page;
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const int r = in + min(2 * lj + (v & 1) + 8 * (v >> 1), left - 1);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) vx[v][x] = ld_once(base + r * a.s_slot + 64 * x);
      }
    };
    float m[NB][2], l[NB][2];       // rows 2 lj, 2 lj + 1 of a block; l: this lane's share
    float o[NB][D / 64][4][4];      // O^T: channels 64 x + 8 lg + 2 u (+1), rows 2 lj (+1)
    uint4 qf[NB][D / 32];
    bool rests = true;  // the product with P's rounding rests
    for (;;) {
      const int e_first = ua * kUnit + 16 * warp;
      kpage = page_of(e_first);
      int next = page_of(e_first + kUnit);  // page of the following slots, one step ahead
      if (e_first < end) {
        load_k(e_first, kpage);
        load_v(e_first, kpage);
      }
#pragma unroll
      for (int k = 0; k < NB; ++k) {
        const int r = 8 * k + lg;
        const bool ok = r < nrows;
        const int tok = s.first + (r0 + r) / g, qh = h * g + (r0 + r) % g;
        const __nv_bfloat16* qp = p.q + (ok ? (int64_t)tok * p.s_q + (int64_t)qh * D : 0) + 8 * lj;
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
          qf[k][c] = ok ? *reinterpret_cast<const uint4*>(qp + 32 * c) : make_uint4(0, 0, 0, 0);
        m[k][0] = m[k][1] = -INFINITY;
        l[k][0] = l[k][1] = 0.f;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int w = 0; w < 4; ++w)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][x][w][e] = 0.f;
      }
#pragma unroll 1
      for (int e0 = e_first; e0 < end; e0 += kUnit) {
        const int left = end - e0;
        float c[NB][4];
        const float b0 = bias[0], b1 = bias[1];
#pragma unroll
        for (int k = 0; k < NB; ++k) {
          float c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) c[k][e] = 0.f;
#pragma unroll
          for (int x = 0; x < D / 32; ++x) {
            mma_bf16(c[k], kx[0][x].x, kx[1][x].x, kx[0][x].y, kx[1][x].y, qf[k][x].x, qf[k][x].y);
            mma_bf16(c2, kx[0][x].z, kx[1][x].z, kx[0][x].w, kx[1][x].w, qf[k][x].z, qf[k][x].w);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) c[k][e] += c2[e];
        }
        // the next slots' K
        if (e0 + kUnit < end) load_k(e0 + kUnit, next);
        kpage = next;
        next = page_of(e0 + 2 * kUnit);
        // slots whose value does not count: 0 * inf would be NaN
        const unsigned dead0 = __ballot_sync(0xffffffffu, b0 == -INFINITY || lg >= left);
        const unsigned dead1 = __ballot_sync(0xffffffffu, b1 == -INFINITY || lg + 8 >= left);
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
        if (e0 + kUnit < end) load_v(e0 + kUnit, kpage);
      }
      // An infinite value times a rest of 0 (or below 0) is no infinity any more: once more
      // without the rests, where a sum came out as NaN.
      bool nan = false;
      if (rests) {
#pragma unroll
        for (int k = 0; k < NB; ++k)
#pragma unroll
          for (int x = 0; x < D / 64; ++x)
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
              for (int e = 0; e < 4; ++e) nan |= o[k][x][w][e] != o[k][x][w][e];
      }
      if (!__any_sync(0xffffffffu, nan)) break;
      rests = false;
    }
    // ---- the warps' states, a block of 8 rows at a time
    const bool begins = ua == 0, ends = ub == nu;
    float* part = join.parts + (int64_t)(2 * blockIdx.x + (begins ? 1 : 0)) * R::kPart;
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      if (8 * k >= nrows) break;
      if (k > 0) __syncthreads();
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float* row = red[warp][2 * lj + e];
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) l[k][e] += __shfl_xor_sync(0xffffffffu, l[k][e], x);
#pragma unroll
        for (int x = 0; x < D / 64; ++x) {
          float* at = row + 64 * x + 8 * lg;
          *reinterpret_cast<float4*>(at) =
              make_float4(o[k][x][0][e], o[k][x][0][e + 2], o[k][x][1][e], o[k][x][1][e + 2]);
          *reinterpret_cast<float4*>(at + 4) =
              make_float4(o[k][x][2][e], o[k][x][2][e + 2], o[k][x][3][e], o[k][x][3][e + 2]);
        }
        if (lg == 0) {
          row[D] = m[k][e];
          row[D + 1] = l[k][e];
        }
      }
      __syncthreads();
      const int nr = min(8, nrows - 8 * k);
      for (int it = threadIdx.x; it < nr * D; it += kRowThreads) {
        const int r = it / D, col = it % D;
        float M = -INFINITY;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) M = fmaxf(M, red[w][r][D]);
        float L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < kRowWarps; ++w) {
          // a warp that saw nothing has sums of 0, or of NaN
          const float f = red[w][r][D] == M ? 1.f : exp2f((red[w][r][D] - M) * kLog2e);
          L += f * red[w][r][D + 1];
          O += f * red[w][r][col];
        }
        const int row = r0 + 8 * k + r;
        if (begins && ends) {
          p.out[((int64_t)(s.first + row / g) * p.Hq + h * g + row % g) * D + col] =
              __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
        } else {
          part[(8 * k + r) * D + col] = O;
          if (col == 0)
            *reinterpret_cast<float2*>(part + kRows * D + 2 * (8 * k + r)) = make_float2(M, L);
        }
      }
    }
    if (!(begins && ends)) {
      // the CTAs that hold the set's first and last unit
      const int c0 = (int)(((su + 1) * nct - 1) / total);
      const int c1 = (int)(((su + nu) * nct - 1) / total);
      __threadfence();
      __syncthreads();
      if (threadIdx.x == 0) is_last = atomicAdd(&join.arrived[c0], 1) == c1 - c0;
      __syncthreads();
      if (is_last) {
        __threadfence();
        for (int it = threadIdx.x; it < nrows * D; it += kRowThreads) {
          const int r = it / D, col = it % D;
          const float* first = join.parts + (int64_t)(2 * c0 + 1) * R::kPart;
          float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll 4
          for (int c = c0; c <= c1; ++c) {
            const float* x = c == c0 ? first : join.parts + (int64_t)(2 * c) * R::kPart;
            const float2 ml = __ldcg(reinterpret_cast<const float2*>(x + kRows * D + 2 * r));
            const float xo = __ldcg(x + r * D + col);
            const float n = fmaxf(M, ml.x);
            const float f = M == n ? 1.f : exp2f((M - n) * kLog2e);
            const float w = ml.x == n ? 1.f : exp2f((ml.x - n) * kLog2e);
            L = L * f + ml.y * w;
            O = O * f + xo * w;
            M = n;
          }
          const int row = r0 + r;
          p.out[((int64_t)(s.first + row / g) * p.Hq + h * g + row % g) * D + col] =
              __float2bfloat16_rn(L == 0.f ? 0.f : O / L);
        }
        if (threadIdx.x == 0) join.arrived[c0] = 0;
      }
    }
    u = su + ub;
    if (u < u1) __syncthreads();  // red and is_last are written again
  }
}

template <int D, int NB>
struct RowsLaunch {
  static int ctas(int num_sms) { return num_sms * Rows<D, NB>::kMinCtas; }
  static cudaError_t run(const PagedArgs& a, const PagedQuery& p, void* ws, int* arrived,
                         int num_sms, cudaStream_t s) {
    RowsJoin join;
    join.parts = static_cast<float*>(ws);
    join.arrived = arrived;
    paged_rows_kernel<D, NB><<<ctas(num_sms), kRowThreads, 0, s>>>(a, p, join);
    return cudaGetLastError();
  }
  static size_t bytes(int num_sms) {
    return (size_t)2 * ctas(num_sms) * Rows<D, NB>::kPart * sizeof(float);
  }
};

// Calls f with the form that serves d channels and groups of g heads. 16 rows of 256 channels do
// not fit a thread's registers beside their K and V: larger groups take several blocks of 8.
template <class F>
auto rows_form(int d, int g, F f) {
  const bool two = g > 8;
  if (d == 64) return two ? f(RowsLaunch<64, 2>()) : f(RowsLaunch<64, 1>());
  if (d == 128) return two ? f(RowsLaunch<128, 2>()) : f(RowsLaunch<128, 1>());
  return f(RowsLaunch<256, 1>());
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs& a, const PagedAppend& p, const RopeTurns& turns,
                                int num_sms, cudaStream_t s) {
  const int tokens = std::max(1, std::min(kAppendTokens, a.n / (4 * num_sms)));
  const size_t smem = p.rotate ? (size_t)tokens * (a.d / 2) * sizeof(float2) : 0;
  paged_append_kernel<<<(a.n + tokens - 1) / tokens, kAppendThreads, smem, s>>>(a, p, turns, tokens);
  return cudaGetLastError();
}

size_t paged_rows_workspace(const PagedArgs& a, int Hq, int num_sms) {
  return rows_form(a.d, Hq / a.H, [&](auto form) { return form.bytes(num_sms); });
}

cudaError_t launch_paged_rows(const PagedArgs& a, const PagedQuery& p, void* ws, int* arrived,
                              int num_sms, cudaStream_t s) {
  return rows_form(a.d, p.Hq / a.H,
                   [&](auto form) { return form.run(a, p, ws, arrived, num_sms, s); });
}

}  // namespace still
