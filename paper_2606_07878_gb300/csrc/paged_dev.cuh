// Device side of what the kernels over a paged cache share.
#pragma once
#include "paged.cuh"
#include "ptx.cuh"

namespace still {

constexpr float kLog2e = 1.44269504f;

STILL_DEV uint32_t bf16x2_bits(__nv_bfloat162 x) { return *reinterpret_cast<uint32_t*>(&x); }

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

}  // namespace still
