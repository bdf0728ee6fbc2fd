// The paged key-value cache: append (with the base model's RoPE) and attention of few rows.
#include "paged_rows.cuh"

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
    const int b = paged_owner(a, i);
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
      most = std::max(most, rows_form<kRowsBf16>(
                                d, rows, [&](auto form) { return form.bytes(num_sms); }));
  return most;
}

cudaError_t launch_paged_rows(const PagedArgs& a, const PagedQuery& p, void* ws, int num_sms,
                              cudaStream_t s) {
  return rows_form<kRowsBf16>(a.d, paged_mean_rows(a, p.Hq),
                              [&](auto form) { return form.run(a, p, ws, num_sms, s); });
}

}  // namespace still
