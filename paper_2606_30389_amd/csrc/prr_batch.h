// A batch of sequences on the device: where a sequence's rows and pages lie, whatever the caller's
// arrays hold.  Needs only int32_t, size_t, min and max, so that it can be compiled for the CPU too.
#pragma once

namespace prr {

struct BatchArgs {
  const int32_t* cu_q;
  const int32_t* kv_len;
  const int32_t* page_table;
  int n_seqs, total_q, max_q, max_kv, table_stride;
};

// New tokens [q0, q1) and cached tokens of sequence s, cut to the batch's bounds.
struct Seq {
  int q0, q1, kv;
};
__device__ __forceinline__ Seq seq_at(const BatchArgs& b, int s) {
  Seq r;
  if (b.cu_q) {
    r.q0 = min(max(b.cu_q[s], 0), b.total_q);
    r.q1 = min(max(b.cu_q[s + 1], r.q0), min(b.total_q - r.q0, b.max_q) + r.q0);
  } else {
    r.q0 = s;
    r.q1 = s + 1;
  }
  r.kv = min(max(b.kv_len[s], 0), b.max_kv);
  return r;
}

// The physical page of logical page lp of sequence s, or -1: no such page.
__device__ __forceinline__ int phys_page(const int32_t* table, int table_stride, int max_pages, int s, int lp) {
  if (!table) return lp >= 0 && lp < max_pages ? lp : -1;
  if (lp < 0 || lp >= table_stride) return -1;
  const int p = table[(size_t)s * table_stride + lp];
  return p >= 0 && p < max_pages ? p : -1;
}

}  // namespace prr
