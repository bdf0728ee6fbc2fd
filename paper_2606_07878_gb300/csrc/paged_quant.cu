// The paged cache in 8 bits: append with quantisation, and attention of few rows.
//
// A pool holds e4m3 codes; slots [16 i, 16 i + 16) of a page and KV-head share a scale of K and one
// of V, and a value is code times scale.
#include "paged_rows.cuh"

namespace still {

namespace {

// ----------------------------------------------------------------- append
//
// Rows are rotated as paged.cu does and keys rounded to bf16, what a 16-bit cache would hold. A
// block of 16 slots then takes the smallest power of two s with max |x| <= 448 s over its new rows,
// or the scale that it has already where that is larger and the block is partly filled; its codes
// are x / s, rounded to nearest even. Powers of two cost no precision (e4m3 has the same 4 bits at
// any size; the block's largest value is above 224 s, so only what lies 2^13.8 below it meets the
// subnormal codes, off by 2^-10 s at most) and let a block change its scale without rounding its
// older codes again, but for those that become subnormal.
//
// A warp takes the K or the V rows of a block and KV-head, at most 16 of them: it holds them in
// registers between their maximum and their codes. The first token of a block (or of a sequence's
// new tokens) leads it; a CTA looks at a window of tokens for leaders. Other CTAs rotate queries.
//
// Memory and the latency of its reads bound it: 8,192 tokens of 32 query and 8 KV-heads of 128
// channels are 185 MB, 43 us (4.3 TB/s); 16 query and 8 KV-heads of 256 channels 235 MB, 64 us (3.7).
// Three CTAs an SM (256 channels: two) cost 44 (108) bytes of spills a thread. One grid for both, a window's queries before its keys and
// values, took 57; keys and values behind the queries 49 (a CTA of theirs takes longer: the grid's
// end waits for it).
constexpr int kQuantThreads = 256;
constexpr int kWindow = 16;       // tokens; 1 where sequences have few of them
constexpr int kQueryWindow = 8;   // of a CTA that rotates queries; or 1

// The smallest power of two, 2^-126 at least, by which `top` is at most 448.
STILL_DEV float least_scale(float top) {
  const uint32_t bits = __float_as_uint(top);  // top = 1.m 2^(e - 127); 448 = 1.75 2^8
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
  return __uint_as_float((uint32_t)(127 + max(e, -126)) << 23);
}

// Four codes of x / s; by = 1 / s. Values beyond 448 s, infinities too, become +-448, NaN stays
// NaN.
STILL_DEV uint32_t codes4(float x0, float x1, float x2, float x3, float by) {
  uint32_t r;
  asm("{\n\t.reg .b16 l, h;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\t"
      "cvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\t"
      "mov.b32 %0, {l, h};\n}\n"
      : "=r"(r)
      : "f"(x0 * by), "f"(x1 * by), "f"(x2 * by), "f"(x3 * by));
  return r;
}
// Codes times `by`, rounded to codes again.
STILL_DEV uint32_t recoded(uint32_t x, float by) {
  const uint32_t lo = f16_of_lower(x), hi = f16_of_upper(x);
  const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&lo));
  const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&hi));
  return codes4(a.x, a.y, b.x, b.y, by);
}

struct Lead {
  int token, slot, count, page, head_room;  // head_room: slots of the block before `slot`
};

template <int D>
__global__ void __launch_bounds__(kQuantThreads, D == 256 ? 2 : 3)
    paged_append_quant_kernel(const __grid_constant__ PagedArgs a,
                              const __grid_constant__ PagedAppend p,
                              const __grid_constant__ RopeTurns w, int kv_blocks, int kv_window,
                              int q_window, int reach) {
  // [window + reach][4][kLanes] two cosines and two sines of tokens from the window's first on: of
  // channels 8 l + 2 m (+1) at [m][l], so that the lanes of a row read 16 bytes side by side (in
  // the channels' order they meet in the same banks: 55 us where this took 50)
  extern __shared__ __align__(16) float2 cs[];
  __shared__ Lead lead[kWindow];
  __shared__ long long pos[kWindow];
  constexpr int kHalf = D / 2;
  constexpr int kLanes = D / 16;  // threads of a row: 8 channels of each half
  const bool queries = (int)blockIdx.x >= kv_blocks;  // (the longer ones first)
  const int window = queries ? q_window : kv_window;
  const int i0 = ((int)blockIdx.x - (queries ? kv_blocks : 0)) * window;
  const int nt = min(window, a.n - i0);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int t = warp; t < nt; t += kQuantThreads / 32) {
    const int i = i0 + t, b = paged_owner(a, i);
    if (lane == 0) {
      const long long offset = a.pos_offset != nullptr ? a.pos_offset[b] : 0;
      const Seq s = paged_seq(a, b);
      const int at = i - s.first, j = s.len - s.count + at;
      Lead x{i, j, 0, -1, j & (kScaleBlock - 1)};
      if (at >= 0 && at < s.count && j >= 0 &&
          (x.head_room == 0 || j == max(0, s.len - s.count))) {
        x.count = min(kScaleBlock - x.head_room, s.len - j);
        x.page = paged_page(a, a.table + (int64_t)b * a.s_table, j);
      }
      lead[t] = x;
      pos[t] = j + offset;
    }
  }
  __syncthreads();
  if (p.rotate) {
    const int table = queries ? nt : window + reach;
    for (int x = threadIdx.x; x < table * kHalf; x += kQuantThreads) {
      // (tokens behind the window matter where they are of the last one's block)
      const int t = x / kHalf, known = min(t, nt - 1);
      const unsigned long long turn =
          (unsigned long long)(pos[known] + t - known) * w.turns[x % kHalf];
      float sn, cn;
      sincospif((float)(int)(turn >> 32) * 0x1p-31f, &sn, &cn);
      const int ch = x % kHalf;
      float* at = reinterpret_cast<float*>(cs + t * kHalf + (ch / 2 % 4 * kLanes + ch / 8) * 2);
      at[ch % 2] = cn;
      at[2 + ch % 2] = sn;
    }
    __syncthreads();
  }
  auto rotate = [&](uint4& lo, uint4& hi, const float2* ang) {
    uint32_t* l = reinterpret_cast<uint32_t*>(&lo);
    uint32_t* u = reinterpret_cast<uint32_t*>(&hi);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const uint64_t x0 = bf16_pair(l[m]), x1 = bf16_pair(u[m]);
      const float4 y = *reinterpret_cast<const float4*>(ang + 2 * m * kLanes);  // of two channels
      const uint64_t c = pack2(y.x, y.y), s = pack2(y.z, y.w);
      float z0, z1;
      unpack2(fma2(x0, c, neg2(mul2(x1, s))), z0, z1);
      l[m] = bf16x2_bits(__floats2bfloat162_rn(z0, z1));
      unpack2(fma2(x0, s, mul2(x1, c)), z0, z1);
      u[m] = bf16x2_bits(__floats2bfloat162_rn(z0, z1));
    }
  };
  // ---- queries: 8 channels of each half of a head, several on their way at a time
  if (queries) {
    constexpr int kAtOnce = 4, kStep = kQuantThreads / kLanes;  // rows
    const int rows = nt * p.Hq, l = threadIdx.x % kLanes;
    const int dt = kStep / p.Hq, dh = kStep % p.Hq;
    const __nv_bfloat16* const from = p.q + i0 * p.s_q + l * 8;
    __nv_bfloat16* const to = p.q_out + (int64_t)i0 * p.Hq * D + l * 8;
    int r = threadIdx.x / kLanes, t = r / p.Hq, h = r % p.Hq;
    while (r < rows) {
      uint4 lo[kAtOnce], hi[kAtOnce];
      int at[kAtOnce];  // the rows' tokens
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        at[i] = t;
        if (r + i * kStep < rows) {
          const __nv_bfloat16* src = from + t * p.s_q + h * D;
          lo[i] = __ldcs(reinterpret_cast<const uint4*>(src));
          hi[i] = __ldcs(reinterpret_cast<const uint4*>(src + kHalf));
        }
        t += dt;
        h += dh;
        if (h >= p.Hq) {
          h -= p.Hq;
          ++t;
        }
      }
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i) {
        if (r + i * kStep >= rows) break;
        rotate(lo[i], hi[i], cs + at[i] * kHalf + l * 2);
        __nv_bfloat16* dst = to + (int64_t)(r + i * kStep) * D;
        *reinterpret_cast<uint4*>(dst) = lo[i];
        *reinterpret_cast<uint4*>(dst + kHalf) = hi[i];
      }
      r += kAtOnce * kStep;
    }
    return;
  }
  // ---- blocks of keys and values
  constexpr int kAtOnce = 32 / kLanes;                 // rows
  constexpr int kSteps = kScaleBlock / kAtOnce;
  const int c = lane % kLanes * 8, r0 = lane / kLanes;
  for (int u = warp; u < nt * 2 * a.H; u += kQuantThreads / 32) {
    const Lead x = lead[u / (2 * a.H)];
    if (x.count == 0 || x.page < 0) continue;
    const int h = u % (2 * a.H) >> 1;
    const bool key = (u & 1) == 0;
    const __nv_bfloat16* src =
        (key ? p.k + x.token * p.s_k : p.v + x.token * p.s_v) + (int64_t)h * D + c;
    const int64_t pitch = key ? p.s_k : p.s_v;
    uint4 lo[kSteps], hi[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = r0 + i * kAtOnce;
      lo[i] = hi[i] = make_uint4(0, 0, 0, 0);
      if (r < x.count) {
        lo[i] = *reinterpret_cast<const uint4*>(src + r * pitch);
        hi[i] = *reinterpret_cast<const uint4*>(src + r * pitch + kHalf);
      }
    }
    const int in = x.slot & ((1 << a.page_shift) - 1);  // in its page
    const int64_t head = (int64_t)x.page * a.H + h;
    float* const scale =
        (key ? a.k_scale : a.v_scale) + (head << (a.page_shift - 4)) + (in >> 4);
    float old = x.head_room > 0 ? *scale : 0.f;
    if (!(old > 0.f && old <= 3.4e38f)) old = 0.f;
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = r0 + i * kAtOnce;
      if (key && p.rotate && r < x.count)
        rotate(lo[i], hi[i], cs + (x.token - i0 + r) * kHalf + c / 4);
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        const uint32_t y = m < 4 ? word(lo[i], m) : word(hi[i], m - 4);
        const float x0 = fabsf(__uint_as_float(y << 16));
        const float x1 = fabsf(__uint_as_float(y & 0xffff0000u));
        top = max3(top, x0 <= 3.4e38f ? x0 : 0.f, x1 <= 3.4e38f ? x1 : 0.f);
      }
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float s = fmaxf(old, least_scale(top)), by = 1.f / s;
    uint8_t* const dst = (key ? a.K8 : a.V8) + (int64_t)x.page * a.s_page +
                         (int64_t)(in - x.head_room) * a.s_slot + (int64_t)h * a.s_head + c;
    if (old > 0.f && s > old) {  // the block's older codes
#pragma unroll 1
      for (int r = r0; r < x.head_room; r += kAtOnce) {
        uint2* l = reinterpret_cast<uint2*>(dst + r * a.s_slot);
        uint2* u2 = reinterpret_cast<uint2*>(dst + r * a.s_slot + kHalf);
        const uint2 y = *l, z = *u2;
        *l = make_uint2(recoded(y.x, old * by), recoded(y.y, old * by));
        *u2 = make_uint2(recoded(z.x, old * by), recoded(z.y, old * by));
      }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int r = r0 + i * kAtOnce;
      if (r >= x.count) continue;
      uint32_t y[4];
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const uint32_t y0 = m < 2 ? word(lo[i], 2 * m) : word(hi[i], 2 * m - 4);
        const uint32_t y1 = m < 2 ? word(lo[i], 2 * m + 1) : word(hi[i], 2 * m - 3);
        y[m] = codes4(__uint_as_float(y0 << 16), __uint_as_float(y0 & 0xffff0000u),
                      __uint_as_float(y1 << 16), __uint_as_float(y1 & 0xffff0000u), by);
      }
      uint8_t* to = dst + (int64_t)(x.head_room + r) * a.s_slot;
      *reinterpret_cast<uint2*>(to) = make_uint2(y[0], y[1]);
      *reinterpret_cast<uint2*>(to + kHalf) = make_uint2(y[2], y[3]);
    }
    if (lane == 0) *scale = s;
    if (key && a.beta != nullptr && lane < x.count)
      a.beta[(head << a.page_shift) + in + lane] =
          p.beta != nullptr ? p.beta[(int64_t)(x.token + lane) * a.H + h] : 0.f;
  }
}

}  // namespace

cudaError_t launch_paged_append_quant(const PagedArgs& a, const PagedAppend& p,
                                      const RopeTurns& turns, cudaStream_t s) {
  const bool many = a.n / a.B >= kWindow / 2;
  const int window = many ? kWindow : 1, q_window = many ? kQueryWindow : 1;
  const int q_blocks = p.Hq > 0 ? (a.n + q_window - 1) / q_window : 0;
  // a block reaches 15 tokens behind the window's last
  const int reach = a.cu_new == nullptr ? 0 : kScaleBlock - 1;
  const size_t smem = p.rotate ? (size_t)(window + reach) * (a.d / 2) * sizeof(float2) : 0;
  auto kernel = a.d == 64    ? paged_append_quant_kernel<64>
                : a.d == 128 ? paged_append_quant_kernel<128>
                             : paged_append_quant_kernel<256>;
  const int kv_blocks = (a.n + window - 1) / window;
  kernel<<<kv_blocks + q_blocks, kQuantThreads, smem, s>>>(a, p, turns, kv_blocks, window, q_window,
                                                           reach);
  return cudaGetLastError();
}

size_t paged_rows_quant_workspace(int num_sms) {
  size_t most = 0;
  for (int d : {64, 128, 256})
    for (int rows : {8, 16})
      most = std::max(most, rows_form<kRowsE4m3>(
                                d, rows, [&](auto form) { return form.bytes(num_sms); }));
  return most;
}

cudaError_t launch_paged_rows_quant(const PagedArgs& a, const PagedQuery& p, void* ws, int num_sms,
                                    cudaStream_t s) {
  return rows_form<kRowsE4m3>(a.d, paged_mean_rows(a, p.Hq),
                              [&](auto form) { return form.run(a, p, ws, num_sms, s); });
}

}  // namespace still
