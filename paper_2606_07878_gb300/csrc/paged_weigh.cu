// Attention weights added up over a paged cache, slot by slot: what a slot got from this call's rows
// (new tokens x the query heads of its KV-head), for evictions (paged_evict.cu).
//
//   weight_j = decay weight_j + sum over rows r that see j of e^(s_rj - m_r) / l_r
//
// with the row's maximum m_r and sum l_r over all slots that it sees. A slot's sum needs them first,
// so there are two passes; sums are in a fixed order, without atomics.
#include "paged_rows.cuh"

namespace still {

namespace {

constexpr int kWeighThreads = 256;

// What a slot had before, 0 for those of this call's own tokens.
STILL_DEV float weighed_before(const float* at, bool old, float decay) {
  return old && decay != 0.f ? decay * *at : 0.f;
}

// ----------------------------------------------------------------- decode
//
// The second pass of a decode: the first one (paged_rows.cuh) leaves the logits, 4 bytes a row and
// slot beside 4 d of K and V, so that K is not read again. A thread takes four slots of a page:
// what it costs is one dependent read after another (lengths, page, logits). 9 us for 8 sequences of
// 5,000 to 9,001 slots with 4 x 8 heads, 13 with a slot a thread (the call 54 to 56, and 58).
constexpr int kWeighSlots = 4;
__global__ void __launch_bounds__(kWeighThreads)
    paged_weigh_logits_kernel(const __grid_constant__ PagedArgs a, const float* logits,
                              const float2* ml, int g, float* weight, float decay) {
  griddep_wait();
  auto units = [&](const Seq& s) {
    constexpr int kUnit = kWeighSlots * kWeighThreads;
    return s.count > 0 ? (int64_t)((s.len - 1) / kUnit + (s.len > 0)) * a.H : 0;
  };
  UnitRange r = unit_range<kWeighThreads>(a, blockIdx.x, gridDim.x, units);
  Seq s{};
  if (r.left > 0) s = paged_seq<false>(a, r.b);
  const int mask = (1 << a.page_shift) - 1;
  for (int64_t n = units(s); r.left > 0; --r.left, ++r.in) {
    while (r.in == n) {
      r.in = 0;
      s = paged_seq<false>(a, ++r.b);
      n = units(s);
    }
    const int h = (int)(r.in % a.H);
    const int64_t j0 = (r.in / a.H * kWeighThreads + threadIdx.x) * kWeighSlots;
    if (j0 >= s.len) continue;
    const int j = (int)j0;
    const int pg = paged_page<false>(a, a.table + (int64_t)r.b * a.s_table, j);
    if (pg < 0) continue;
    const int64_t head = (int64_t)pg * a.H + h;
    const float* x = logits + ((head * g) << a.page_shift) + (j & mask);
    const float2* row = ml + ((int64_t)s.first * a.H + h) * g;
    float* const w = weight + (head << a.page_shift) + (j & mask);
    float sum[kWeighSlots], before[kWeighSlots];
#pragma unroll
    for (int i = 0; i < kWeighSlots; ++i) {
      sum[i] = 0.f;
      before[i] = j + i < s.len ? weighed_before(w + i, j + i < s.len - s.count, decay) : 0.f;
    }
#pragma unroll 4
    for (int i = 0; i < g; ++i) {  // (what lies past the sequence's end is not used)
      const float4 y = *reinterpret_cast<const float4*>(x + ((int64_t)i << a.page_shift));
      const float2 e = row[i];
      if (e.y != 0.f) {  // (NaN: so is what the row gives)
        sum[0] += exp2f((y.x - e.x) * kLog2e) * e.y;
        sum[1] += exp2f((y.y - e.x) * kLog2e) * e.y;
        sum[2] += exp2f((y.z - e.x) * kLog2e) * e.y;
        sum[3] += exp2f((y.w - e.x) * kLog2e) * e.y;
      }
    }
#pragma unroll
    for (int i = 0; i < kWeighSlots; ++i) {
      if (j + i >= s.len) continue;
      // of a masked slot a row of NaN makes e^-inf NaN
      if (sum[i] != sum[i] && a.beta != nullptr &&
          a.beta[(head << a.page_shift) + (j & mask) + i] == -INFINITY)
        sum[i] = 0.f;
      w[i] = before[i] + sum[i];
    }
  }
}

// ----------------------------------------------------------------- any number of tokens
//
// The second pass of a call of many tokens: a warp takes 16 slots, their keys in registers, and goes
// through the rows that see them, 8 at a time.
template <int D>
__global__ void __launch_bounds__(kWeighThreads)
    paged_weigh_rows_kernel(const __grid_constant__ PagedArgs a, const __grid_constant__ PagedQuery p,
                            float* weight, float decay) {
  griddep_wait();
  const int g = p.Hq / a.H;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int lg = lane >> 2, lj = lane & 3;
  constexpr int kSlots = kWeighThreads / 32 * kBatch;  // of a unit
  auto units = [&](const Seq& s) {
    return s.count > 0 ? (int64_t)((s.len + kSlots - 1) / kSlots) * a.H : 0;
  };
  UnitRange r = unit_range<kWeighThreads>(a, blockIdx.x, gridDim.x, units);
  Seq s{};
  if (r.left > 0) s = paged_seq<false>(a, r.b);
  const int mask = (1 << a.page_shift) - 1;
  for (int64_t n = units(s); r.left > 0; --r.left, ++r.in) {
    while (r.in == n) {
      r.in = 0;
      s = paged_seq<false>(a, ++r.b);
      n = units(s);
    }
    const int h = (int)(r.in % a.H);
    const int e0 = (int)(r.in / a.H) * kSlots + warp * kBatch;
    if (e0 >= s.len) continue;
    const int pg = paged_page<false>(a, a.table + (int64_t)r.b * a.s_table, e0);
    if (pg < 0) continue;
    const int in = e0 & mask, most = s.len - e0 - 1;
    const int64_t head = (int64_t)pg * a.H + h;
    uint4 kx[2][D / 32];
    float be[2], sum[2] = {0.f, 0.f};
    const __nv_bfloat16* base = a.K + (int64_t)pg * a.s_page + (int64_t)h * a.s_head + 8 * lj;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int x = in + min(lg + 8 * i, most);
#pragma unroll
      for (int c = 0; c < D / 32; ++c)
        kx[i][c] = *reinterpret_cast<const uint4*>(base + x * a.s_slot + 32 * c);
      be[i] = a.beta != nullptr ? a.beta[(head << a.page_shift) + x] : 0.f;
    }
    const int past = s.len - s.count;
    const int rows = s.count * g;
    for (int r0 = max(0, e0 - past) * g & ~7; r0 < rows; r0 += 8) {
      const int mine = min(r0 + lg, rows - 1);
      const __nv_bfloat16* q = p.q + (int64_t)(s.first + mine / g) * p.s_q +
                               (int64_t)(h * g + mine % g) * D + 8 * lj;
      float c[4] = {0.f, 0.f, 0.f, 0.f}, c2[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < D / 32; ++x) {
        const uint4 y = *reinterpret_cast<const uint4*>(q + 32 * x);
        mma_bf16(c, kx[0][x].x, kx[1][x].x, kx[0][x].y, kx[1][x].y, y.x, y.y);
        mma_bf16(c2, kx[0][x].z, kx[1][x].z, kx[0][x].w, kx[1][x].w, y.z, y.w);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = r0 + 2 * lj + (e & 1);
        if (row >= rows || e0 + lg + 8 * (e >> 1) > past + row / g || be[e >> 1] == -INFINITY)
          continue;
        const float2 m = p.ml[(int64_t)(s.first + row / g) * p.Hq + h * g + row % g];
        const float logit = (c[e] + c2[e]) * p.scale + be[e >> 1];
        if (m.y != 0.f) sum[e >> 1] += exp2f((logit - m.x) * kLog2e) * m.y;
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
      sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
      const int j = e0 + lg + 8 * i;
      if (lj == 0 && j < s.len) {
        float* w = weight + (head << a.page_shift) + (j & mask);
        *w = weighed_before(w, j < past, decay) + sum[i];
      }
    }
  }
}

}  // namespace

size_t paged_rows_weigh_workspace(int num_sms) {
  size_t most = 0;
  for (int d : {64, 128, 256})
    for (int rows : {8, 16}) {
      auto bytes = [&](auto form) { return form.bytes(num_sms); };
      most = std::max({most, rows_form<kRowsWeigh>(d, rows, bytes),
                       rows_form<kRowsStats>(d, rows, bytes)});
    }
  return most;
}

cudaError_t launch_paged_decode_weigh(const PagedArgs& a, const PagedQuery& p, float* weight,
                                      float decay, void* ws, int num_sms, cudaStream_t s) {
  const int g = p.Hq / a.H;
  const cudaError_t e = rows_form<kRowsWeigh>(
      a.d, g, [&](auto form) { return form.run(a, p, ws, num_sms, s); });
  if (e != cudaSuccess) return e;
  return launch_chained(paged_weigh_logits_kernel, dim3(8 * num_sms), dim3(kWeighThreads), 0, s, 1,
                        a, p.logits, p.ml, g, weight, decay);
}

cudaError_t launch_paged_weigh(const PagedArgs& a, const PagedQuery& p, float* weight, float decay,
                               void* ws, int num_sms, cudaStream_t s) {
  const cudaError_t e = rows_form<kRowsStats>(
      a.d, paged_mean_rows(a, p.Hq), [&](auto form) { return form.run(a, p, ws, num_sms, s); });
  if (e != cudaSuccess) return e;
  auto kernel = a.d == 64    ? paged_weigh_rows_kernel<64>
                : a.d == 128 ? paged_weigh_rows_kernel<128>
                             : paged_weigh_rows_kernel<256>;
  return launch_chained(kernel, dim3(4 * num_sms), dim3(kWeighThreads), 0, s, 1, a, p, weight,
                        decay);
}

}  // namespace still
