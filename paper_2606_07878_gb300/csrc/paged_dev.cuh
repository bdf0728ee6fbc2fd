// Device side of what the kernels over a paged cache share.
#pragma once
#include "paged.cuh"
#include "ptx.cuh"

namespace still {

constexpr float kLog2e = 1.44269504f;

STILL_DEV uint32_t bf16x2_bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }
// The lower and the upper two e4m3 codes of a word as fp16 pairs (exact).
STILL_DEV uint32_t f16_of_lower(uint32_t x) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n}\n"
      : "=r"(r) : "r"(x));
  return r;
}
STILL_DEV uint32_t f16_of_upper(uint32_t x) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, h;\n}\n"
      : "=r"(r) : "r"(x));
  return r;
}

// First new token, number of them and slots of sequence b, whatever the arrays hold: an offset
// outside [0, n] or a length beyond the table is cut, and recorded (by one of those who look), as
// are tokens before the first sequence's and behind the last one's, which belong to none.
struct Seq {
  int first, count, len;
};
template <bool kRecord = true>
STILL_DEV Seq paged_seq(const PagedArgs& a, int b) {
  Seq s;
  int c0 = b, c1 = b + 1;
  if (a.cu_new != nullptr) {
    c0 = a.cu_new[b];
    c1 = a.cu_new[b + 1];
  }
  const int cap = (int)min((int64_t)a.table_pages << a.page_shift, (int64_t)0x7fffff00);
  s.len = a.len[b];
  const bool owned = (b > 0 || c0 == 0) && (b + 1 < a.B || c1 == a.n);
  if (!owned || c0 < 0 || c1 < c0 || c1 > a.n || s.len < 0 || s.len > cap) {
    if (kRecord) dev_set_error(a.err, DEV_BAD_ARG, 600);
    c0 = min(max(c0, 0), a.n);
    c1 = min(max(c1, c0), a.n);
    s.len = min(max(s.len, 0), cap);
  }
  s.first = c0;
  s.count = c1 - c0;
  return s;
}

// The page that holds slot j of the sequence whose pages `table` lists; -1 (and a record) when it
// names none.
template <bool kRecord = true>
STILL_DEV int paged_page(const PagedArgs& a, const int32_t* table, int j) {
  const int p = table[j >> a.page_shift];
  if ((unsigned)p < (unsigned)a.n_pages) return p;
  if (kRecord) dev_set_error(a.err, DEV_BAD_ARG, 601);
  return -1;
}

// The sequence that owns token i (the last one that begins at or before it), by a whole warp that
// looks at 32 of them at a time.
STILL_DEV int paged_owner(const PagedArgs& a, int i) {
  if (a.cu_new == nullptr) return i;
  const int lane = threadIdx.x & 31;
  int b = 0;
  for (int n = a.B; n > 1;) {  // among n from b on
    const int apart = (n + 31) / 32;
    const bool before = lane * apart < n && a.cu_new[b + lane * apart] <= i;
    const int k = max(0, 31 - __clz(__ballot_sync(0xffffffffu, before)));
    b += k * apart;
    n = min(apart, n - k * apart);
  }
  return b;
}

// Units of work that sequences have, `units(s)` each, one sequence after another: the share of part
// `part` of `parts`, and where it begins.
struct UnitRange {
  int64_t left;  // units of the share
  int64_t in;    // the first of them, among those of sequence b
  int b;
};
// By all kThreads threads of a block.
template <int kThreads, class F>
STILL_DEV UnitRange unit_range(const PagedArgs& a, int part, int parts, F units) {
  __shared__ int64_t warp_sum[kThreads / 32];
  __shared__ UnitRange range;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (a.B + kThreads - 1) / kThreads;  // consecutive sequences of a thread
  const int b0 = min(a.B, (int)threadIdx.x * per), b1 = min(a.B, b0 + per);
  int64_t mine = 0;
  for (int b = b0; b < b1; ++b) mine += units(paged_seq(a, b));
  int64_t before = mine, total = 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, before, o);
    if (lane >= o) before += x;
  }
  if (lane == 31) warp_sum[warp] = before;
  if (threadIdx.x == 0) range.left = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before += warp_sum[w];
    total += warp_sum[w];
  }
  before -= mine;
  const int64_t each = total / parts, wider = total - each * parts;
  const int64_t u0 = each * part + min((int64_t)part, wider);
  const int64_t u1 = u0 + each + (part < wider);
  if (u1 > u0 && u0 >= before && u0 < before + mine) {
    int b = b0;
    for (;; ++b) {
      const int64_t n = units(paged_seq<false>(a, b));
      if (u0 < before + n) break;
      before += n;
    }
    range = UnitRange{u1 - u0, u0 - before, b};
  }
  __syncthreads();
  return range;
}

}  // namespace still
