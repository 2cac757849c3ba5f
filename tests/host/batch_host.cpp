// prr_batch.h on the CPU, behind C entries.
#include <stddef.h>
#include <stdint.h>

#include <algorithm>

#define __device__
#define __forceinline__ inline
using std::max;
using std::min;

#include "prr_batch.h"

extern "C" {

void seq_host(const int32_t* cu, const int32_t* kv, int n, int total_q, int max_q, int max_kv, int s, int32_t* out) {
  prr::BatchArgs b{cu, kv, nullptr, n, total_q, max_q, max_kv, 0};
  const prr::Seq r = prr::seq_at(b, s);
  out[0] = r.q0;
  out[1] = r.q1;
  out[2] = r.kv;
}

int page_host(const int32_t* table, int stride, int max_pages, int s, int lp) {
  return prr::phys_page(table, stride, max_pages, s, lp);
}
}
