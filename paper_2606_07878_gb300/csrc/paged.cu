// The paged key-value cache: append (with the base model's RoPE) and attention of few rows.
#include "paged.cuh"

#include <algorithm>

#include "launch.cuh"
#include "ptx.cuh"

namespace still {

namespace {

// First new token, number of them and slots of sequence b, whatever the arrays hold: an offset
// outside [0, n] or a length beyond the table is cut and recorded.
struct Seq {
  int first, count, len;
};
STILL_DEV Seq paged_seq(const PagedArgs& a, int b) {
  Seq s;
  int c0 = b, c1 = b + 1;
  if (a.cu_new != nullptr) {
    c0 = a.cu_new[b];
    c1 = a.cu_new[b + 1];
  }
  const int cap = (int)min((int64_t)a.table_pages << a.page_shift, (int64_t)0x7fffff00);
  s.len = a.len[b];
  if (c0 < 0 || c1 < c0 || c1 > a.n || s.len < 0 || s.len > cap) {
    dev_set_error(a.err, DEV_BAD_ARG, 600);
    c0 = min(max(c0, 0), a.n);
    c1 = min(max(c1, c0), a.n);
    s.len = min(max(s.len, 0), cap);
  }
  s.first = c0;
  s.count = c1 - c0;
  return s;
}

// The page that holds slot j of sequence b; -1 (and a record) when the table names none.
STILL_DEV int paged_page(const PagedArgs& a, int b, int j) {
  const int p = a.table[(int64_t)b * a.s_table + (j >> a.page_shift)];
  if ((unsigned)p < (unsigned)a.n_pages) return p;
  dev_set_error(a.err, DEV_BAD_ARG, 601);
  return -1;
}

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
    if (at >= 0 && at < s.count && j >= 0) pg = paged_page(a, b, j);
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
//   P             bf16 in registers; movmatrix turns a slots x rows fragment into the rows x slots
//                 one that the next product reads. The sum of the weights takes them as rounded,
//                 so that a row's weights still add up to 1; a second product with the rounding
//                 rests would turn infinite values into NaN (inf * 0)
//   O^T += V^T P^T  the words of a lane's four V rows, two by two, are fragments of channels x
//                 slots; fp32 sums
// Logits stay in natural units up to the subtraction of the maximum: in units of log 2 a bias of
// the lowest float would become -inf, which masks.
// K, V and O never touch shared memory; the warps of a CTA are combined at the end.
constexpr float kLog2e = 1.44269504f;
constexpr int kRowWarps = 4;
constexpr int kRowThreads = 32 * kRowWarps;

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
STILL_DEV uint32_t bf16x2_bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }

// NB: blocks of 8 rows.
template <int D, int NB>
struct RowState {
  float m[NB][2], l[NB][2];    // rows 2 lj, 2 lj + 1 of a block; l: this lane's share
  float o[NB][D / 64][4][4];   // O^T fragments: channels 64 s + 8 lg + 2 u (+1), rows 2 lj (+1)
};

template <int D, int NB>
__global__ void __launch_bounds__(kRowThreads)
    paged_rows_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedQuery p) {
  constexpr int kRows = 8 * NB;
  constexpr int kPitch = D + 4;
  __shared__ __align__(16) float red[kRowWarps][8][kPitch];  // O rows of a block, m and l behind
  __shared__ int tile_seq, tile_at;
  const int h = blockIdx.y;
  const int g = p.Hq / a.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lg = lane >> 2, lj = lane & 3;
  // the sequence and block of rows of this CTA: every sequence has ceil(count g / kRows)
  if (threadIdx.x == 0) {
    int t = blockIdx.x, b = 0;
    for (; b < a.B; ++b) {
      const Seq s = paged_seq(a, b);
      const int blocks = (int)(((int64_t)s.count * g + kRows - 1) / kRows);
      if (t < blocks) break;
      t -= blocks;
    }
    tile_seq = b;
    tile_at = t;
  }
  __syncthreads();
  const int b = tile_seq;
  if (b >= a.B) return;
  const Seq s = paged_seq(a, b);
  const int r0 = tile_at * kRows;
  const int nrows = min(kRows, s.count * g - r0);
  // slots that a row sees
  int see[NB][2];
  int most = 0;
#pragma unroll
  for (int k = 0; k < NB; ++k)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = r0 + 8 * k + 2 * lj + e;
      see[k][e] = max(0, s.len - s.count + r / g + 1);
      if (8 * k + 2 * lj + e >= nrows) see[k][e] = 0;
    }
  most = max(0, s.len - s.count + (r0 + nrows - 1) / g + 1);
  uint4 qf[NB][D / 32];
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    const int r = 8 * k + lg;
    const bool ok = r < nrows;
    const int tok = s.first + (r0 + r) / g, qh = h * g + (r0 + r) % g;
    const __nv_bfloat16* qp = p.q + (ok ? (int64_t)tok * p.s_q + (int64_t)qh * D : 0) + 8 * lj;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
      qf[k][c] = ok ? *reinterpret_cast<const uint4*>(qp + 32 * c) : make_uint4(0, 0, 0, 0);
  }
  RowState<D, NB> st;
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    st.m[k][0] = st.m[k][1] = -INFINITY;
    st.l[k][0] = st.l[k][1] = 0.f;
#pragma unroll
    for (int x = 0; x < D / 64; ++x)
#pragma unroll
      for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) st.o[k][x][u][e] = 0.f;
  }
  const int mask = (1 << a.page_shift) - 1;
#pragma unroll 1
  for (int e0 = 16 * warp; e0 < most; e0 += 16 * kRowWarps) {
    const int left = min(16, most - e0);
    int pg = paged_page(a, b, e0);
    const bool none = pg < 0;
    if (none) pg = 0;
    const int64_t base = (int64_t)pg * a.s_page + (int64_t)(e0 & mask) * a.s_slot +
                         (int64_t)h * a.s_head;
    uint4 kx[2][D / 32], vx[4][D / 64];
    float bias[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = min(lg + 8 * i, left - 1);  // rows past the end repeat the last one
      const __nv_bfloat16* kp = a.K + base + r * a.s_slot + 8 * lj;
#pragma unroll
      for (int c = 0; c < D / 32; ++c) kx[i][c] = *reinterpret_cast<const uint4*>(kp + 32 * c);
      bias[i] = a.beta != nullptr
                    ? a.beta[(((int64_t)pg * a.H + h) << a.page_shift) + (e0 & mask) + r]
                    : 0.f;
      if (none) bias[i] = -INFINITY;
    }
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const int r = min(2 * lj + (v & 1) + 8 * (v >> 1), left - 1);
      const __nv_bfloat16* vp = a.V + base + r * a.s_slot + 8 * lg;
#pragma unroll
      for (int x = 0; x < D / 64; ++x) vx[v][x] = *reinterpret_cast<const uint4*>(vp + 64 * x);
    }
    // slots whose value does not count: 0 * inf would be NaN
    const unsigned dead0 = __ballot_sync(0xffffffffu, bias[0] == -INFINITY || lg >= left);
    const unsigned dead1 = __ballot_sync(0xffffffffu, bias[1] == -INFINITY || lg + 8 >= left);
    if (dead0 | dead1) {
#pragma unroll
      for (int v = 0; v < 4; ++v) {
        const unsigned m = v >> 1 ? dead1 : dead0;
        if ((m >> (4 * (2 * lj + (v & 1)))) & 1)
#pragma unroll
          for (int x = 0; x < D / 64; ++x) vx[v][x] = make_uint4(0, 0, 0, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < NB; ++k) {
      float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        mma_bf16(c, kx[0][x].x, kx[1][x].x, kx[0][x].y, kx[1][x].y, qf[k][x].x, qf[k][x].y);
        mma_bf16(c2, kx[0][x].z, kx[1][x].z, kx[0][x].w, kx[1][x].w, qf[k][x].z, qf[k][x].w);
      }
      float top[2];
#pragma unroll
      for (int e = 0; e < 4; ++e) {  // slot lg + 8 (e / 2), row 2 lj + e % 2
        const bool ok = e0 + lg + 8 * (e >> 1) < see[k][e & 1] && bias[e >> 1] != -INFINITY;
        c[e] = ok ? (c[e] + c2[e]) * p.scale + bias[e >> 1] : -INFINITY;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        top[e] = fmaxf(c[e], c[e + 2]);
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1)
          top[e] = fmaxf(top[e], __shfl_xor_sync(0xffffffffu, top[e], x));
        const float m = fmaxf(st.m[k][e], top[e]);
        const float by = m == -INFINITY ? 0.f : m;  // nothing seen yet: every p is 2^-inf
        const float f = exp2f((st.m[k][e] - by) * kLog2e);
        st.m[k][e] = m;
        c[e] = exp2f((c[e] - by) * kLog2e);
        c[e + 2] = exp2f((c[e + 2] - by) * kLog2e);
        st.l[k][e] *= f;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            st.o[k][x][u][e] *= f;
            st.o[k][x][u][e + 2] *= f;
          }
      }
      uint32_t pt[2];  // rows x slots
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const __nv_bfloat162 ph = __floats2bfloat162_rn(c[2 * i], c[2 * i + 1]);
        const float2 r = __bfloat1622float2(ph);
        st.l[k][0] += r.x;
        st.l[k][1] += r.y;
        pt[i] = transpose8(bf16x2_bits(ph));
      }
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t v0 = reinterpret_cast<const uint32_t*>(&vx[0][x])[u];
          const uint32_t v1 = reinterpret_cast<const uint32_t*>(&vx[1][x])[u];
          const uint32_t v2 = reinterpret_cast<const uint32_t*>(&vx[2][x])[u];
          const uint32_t v3 = reinterpret_cast<const uint32_t*>(&vx[3][x])[u];
          const uint32_t a0 = __byte_perm(v0, v1, 0x5410), a1 = __byte_perm(v0, v1, 0x7632);
          const uint32_t a2 = __byte_perm(v2, v3, 0x5410), a3 = __byte_perm(v2, v3, 0x7632);
          mma_bf16(st.o[k][x][u], a0, a1, a2, a3, pt[0], pt[1]);
        }
    }
  }
  // ---- the warps' states, a block of 8 rows at a time
#pragma unroll
  for (int k = 0; k < NB; ++k) {
    if (k > 0) __syncthreads();
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float* row = red[warp][2 * lj + e];
#pragma unroll
      for (int x = 4; x <= 16; x <<= 1) st.l[k][e] += __shfl_xor_sync(0xffffffffu, st.l[k][e], x);
#pragma unroll
      for (int x = 0; x < D / 64; ++x) {
        float* at = row + 64 * x + 8 * lg;
        *reinterpret_cast<float4*>(at) =
            make_float4(st.o[k][x][0][e], st.o[k][x][0][e + 2], st.o[k][x][1][e], st.o[k][x][1][e + 2]);
        *reinterpret_cast<float4*>(at + 4) =
            make_float4(st.o[k][x][2][e], st.o[k][x][2][e + 2], st.o[k][x][3][e], st.o[k][x][3][e + 2]);
      }
      if (lg == 0) {
        row[D] = st.m[k][e];
        row[D + 1] = st.l[k][e];
      }
    }
    __syncthreads();
    const int nr = min(8, nrows - 8 * k);
    for (int it = threadIdx.x; it < nr * D; it += kRowThreads) {
      const int r = it / D, col = it % D;
      float m = -INFINITY;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) m = fmaxf(m, red[w][r][D]);
      float l = 0.f, o = 0.f;
#pragma unroll
      for (int w = 0; w < kRowWarps; ++w) {
        const float f = red[w][r][D] == -INFINITY ? 0.f : exp2f((red[w][r][D] - m) * kLog2e);
        l += f * red[w][r][D + 1];
        o += f * red[w][r][col];
      }
      const int row = r0 + 8 * k + r;
      p.out[((int64_t)(s.first + row / g) * p.Hq + h * g + row % g) * D + col] =
          __float2bfloat16_rn(l == 0.f ? 0.f : o / l);
    }
  }
}

template <int D, int NB>
cudaError_t launch_rows(const PagedArgs& a, const PagedQuery& p, cudaStream_t s) {
  const int g = p.Hq / a.H;
  // upper bound of the blocks of rows: one more per sequence than its rows fill
  const int64_t tiles = a.cu_new == nullptr ? (int64_t)a.B * ((g + 8 * NB - 1) / (8 * NB))
                                            : (int64_t)a.n * g / (8 * NB) + a.B;
  paged_rows_kernel<D, NB><<<dim3((unsigned)tiles, a.H), kRowThreads, 0, s>>>(a, p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_append(const PagedArgs& a, const PagedAppend& p, const RopeTurns& turns,
                                int num_sms, cudaStream_t s) {
  const int tokens = std::max(1, std::min(kAppendTokens, a.n / (4 * num_sms)));
  const size_t smem = p.rotate ? (size_t)tokens * (a.d / 2) * sizeof(float2) : 0;
  paged_append_kernel<<<(a.n + tokens - 1) / tokens, kAppendThreads, smem, s>>>(a, p, turns, tokens);
  return cudaGetLastError();
}

cudaError_t launch_paged_rows(const PagedArgs& a, const PagedQuery& p, cudaStream_t s) {
  const bool two = p.Hq / a.H > 8;
  switch (a.d) {
    case 64: return two ? launch_rows<64, 2>(a, p, s) : launch_rows<64, 1>(a, p, s);
    case 128: return two ? launch_rows<128, 2>(a, p, s) : launch_rows<128, 1>(a, p, s);
    case 256: return two ? launch_rows<256, 2>(a, p, s) : launch_rows<256, 1>(a, p, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace still
