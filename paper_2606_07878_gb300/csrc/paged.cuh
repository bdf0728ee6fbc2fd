// A paged key-value cache: appending to it and attending over it (launchers in paged.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "kernel_table.cuh"

namespace still {

constexpr int kMinPage = 16;  // slots: the keys of one MMA never leave a page

// A pool of pages and the sequences that own them. Slot j of sequence b is slot j mod page of page
// table[b * s_table + j / page]; its row of KV-head h begins at
// K + page_index * s_page + (j mod page) * s_slot + h * s_head (elements), the same in V, and its
// bias is beta[(page_index * H + h) * page + j mod page].
struct PagedArgs {
  __nv_bfloat16 *K = nullptr, *V = nullptr;
  // a pool in 8 bits instead: e4m3 codes, and the scale of slots [16 i, 16 i + 16) of a page at
  // scale[(page_index * H + h) * (page / 16) + i]
  uint8_t *K8 = nullptr, *V8 = nullptr;
  float *k_scale = nullptr, *v_scale = nullptr;
  float* beta = nullptr;          // or null: no bias
  int64_t s_page = 0, s_slot = 0, s_head = 0;
  int32_t n_pages = 0, page_shift = 0, H = 0, d = 0;
  const int32_t* table = nullptr;
  int64_t s_table = 0;
  int32_t table_pages = 0, B = 0;
  const int32_t* len = nullptr;     // [B] slots in use, this call's tokens included
  const int32_t* cu_new = nullptr;  // [B + 1] offsets of the new tokens, or null: one each
  const int64_t* pos_offset = nullptr;  // [B] position - slot, or null: 0
  int32_t n = 0;                    // new tokens of all sequences
  int* err = nullptr;               // device error record
};

// cos and sin of position * w_m: turns[m] = w_m / 2 pi in units of 2^-64, so that the integer
// product position * turns[m] is the angle's fraction of a turn.
struct RopeTurns {
  unsigned long long turns[128];
};

struct PagedAppend {
  const __nv_bfloat16 *q = nullptr, *k = nullptr, *v = nullptr;  // token i's rows at i * s_*
  int64_t s_q = 0, s_k = 0, s_v = 0;
  const float* beta = nullptr;     // [n][H], or null: 0
  __nv_bfloat16* q_out = nullptr;  // [n][Hq][d]
  int32_t Hq = 0;                  // 0: no queries
  int32_t rotate = 0;
};
cudaError_t launch_paged_append(const PagedArgs& a, const PagedAppend& p, const RopeTurns& turns,
                                int num_sms, cudaStream_t s);

struct PagedQuery {
  const __nv_bfloat16* q = nullptr;  // token i's Hq rows at i * s_q
  int64_t s_q = 0;
  __nv_bfloat16* out = nullptr;      // [n][Hq][d]
  int32_t Hq = 0;
  float scale = 0.f;
  // of a decode whose weights are added up: logits [n_pages][H][Hq / H][page], -inf where a row does
  // not see the slot, and (m, 1 / l) of every row (0: it sees nothing), [n][Hq]
  float* logits = nullptr;
  float2* ml = nullptr;
};
// Few rows (paged.cu), and the join of what several warps share: two launches. ws:
// paged_rows_workspace bytes, enough for every call.
int paged_mean_rows(const PagedArgs& a, int Hq);  // of a sequence and KV-head, rounded up
size_t paged_rows_workspace(int num_sms);
cudaError_t launch_paged_rows(const PagedArgs& a, const PagedQuery& q, void* ws, int num_sms,
                              cudaStream_t s);

// Many rows, on the tensor cores (paged_prefill.cu), and the join of what several CTAs share: two
// launches. paged_prefill_serves: whether a call takes this kernel. ws: paged_prefill_workspace
// bytes, enough for every call.
bool paged_prefill_serves(const PagedArgs& a, int Hq);
size_t paged_prefill_workspace(int num_sms);
cudaError_t launch_paged_prefill(const PagedArgs& a, const PagedQuery& q, void* ws,
                                 const KernelTable& dev, cudaStream_t s);
// What its plan adds up for items [q0, q1), of `tokens` new tokens each, of a sequence with `count`
// of them and `len` slots: tiles of 128 slots, and an item's beginning and end as two more.
int64_t paged_prefill_cost(int count, int len, int tokens, int q0, int q1);

// The same over a pool in 8 bits (paged_quant.cu).
constexpr int kScaleBlock = 16;  // slots that share a scale
cudaError_t launch_paged_append_quant(const PagedArgs& a, const PagedAppend& p,
                                      const RopeTurns& turns, cudaStream_t s);
size_t paged_rows_quant_workspace(int num_sms);
cudaError_t launch_paged_rows_quant(const PagedArgs& a, const PagedQuery& q, void* ws, int num_sms,
                                    cudaStream_t s);

// Attention weights added up slot by slot (paged_weigh.cu), weight as PagedArgs::beta: decay times
// what was there (0 for this call's own slots) plus what this call's rows give. Three launches, with
// the attention (decode) or from keys alone.
size_t paged_rows_weigh_workspace(int num_sms);
cudaError_t launch_paged_decode_weigh(const PagedArgs& a, const PagedQuery& q, float* weight,
                                      float decay, void* ws, int num_sms, cudaStream_t s);
cudaError_t launch_paged_weigh(const PagedArgs& a, const PagedQuery& q, float* weight, float decay,
                               void* ws, int num_sms, cudaStream_t s);
// The same of many rows, on the tensor cores (paged_weigh_tc.cu): four launches.
bool paged_weigh_tc_serves(const PagedArgs& a, int Hq);
size_t paged_weigh_tc_workspace(int num_sms);
cudaError_t launch_paged_weigh_tc(const PagedArgs& a, const PagedQuery& q, float* weight,
                                  float decay, void* ws, const KernelTable& dev, cudaStream_t s);

// Of every sequence and KV-head the `keep` slots that count, into pages of `to` (paged_evict.cu).
struct PagedEvict {
  const float* weight = nullptr;
  int32_t keep = 0, sinks = 0, recent = 0;
  PagedArgs to;                     // pools, table and error record alone
  float* to_weight = nullptr;       // or null
  int32_t* kept = nullptr;          // [B][H][keep]
  int32_t* to_len = nullptr;        // [B]
  int64_t* to_offset = nullptr;     // [B] or null
};
cudaError_t launch_paged_evict(const PagedArgs& a, const PagedEvict& e, const KernelTable& dev,
                               cudaStream_t s);

}  // namespace still
