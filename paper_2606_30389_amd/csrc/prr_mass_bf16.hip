// The weight that cached tokens receive, bfloat16 queries; how a call is split, and its launches.
#include "prr_mass_impl.h"

namespace prr {

template <>
const void* mass_kernel_of<true>(const MassLaunch& a) {
  return mass_fn_of<true>(a);
}

namespace {

// The parts of the rows, added in order; one thread per key (without lists: parts are made for calls without them).
__global__ __launch_bounds__(256) void mass_join_kernel(const MassLaunch a) {
  const int h = blockIdx.y, s = blockIdx.z;
  const int kv = min(max(a.b.kv_len[s], 0), a.b.max_kv);
  for (int64_t key = (int64_t)blockIdx.x * 256 + threadIdx.x; key < kv; key += (int64_t)gridDim.x * 256) {
    const int phys = phys_page(a.b.page_table, a.b.table_stride, a.c.max_pages, s, (int)(key >> a.c.page_shift));
    if (phys < 0) continue;
    float v = 0.0f;
#pragma unroll 16
    for (int p = 0; p < a.nsplit; ++p)
      v += a.part[(((int64_t)p * a.b.n_seqs + s) * a.c.num_kv_heads + h) * a.part_keys + key];
    const int64_t at = (((int64_t)h * a.c.max_pages + phys) << a.c.page_shift) + (key & (a.c.page_size - 1));
    a.mass[at] = a.before ? fmaf(a.decay, a.before[at], v) : v;
  }
}

}  // namespace

void plan_mass(MassLaunch& a) {
  const int64_t keys = a.cap > 0 ? (int64_t)a.cap * a.c.page_size : a.b.max_kv;
  const int64_t rows = (int64_t)(a.last ? min(a.last, a.b.max_q) : a.b.max_q) * a.group;
  const int64_t units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  const int64_t blocks = max((keys + 15) / 16, (int64_t)1);
  // Four blocks of keys a wave feed the products best (8191 tokens: 680 us with one, 505 with four); where there is too
  // little work to fill the chip with them, one (2000 tokens, 32 / 2 heads, 60 us; 71 with four; 500 tokens 22, 31).
  a.blocks = blocks * units >= 16 * 256 || rows * blocks * units >= (int64_t)1 << 24 ? 4 : 1;
  const int64_t per = 64 * a.blocks;
  int64_t groups = max((keys + per - 1) / per, (int64_t)1);
  a.part_keys = groups * per;
  // The rows in as many parts, of four (one block) or eight tiles at least, as make 2048 workgroups: the first keys have the
  // most rows, and a workgroup of all of them would outlast the others (8191 tokens: 970 us in 512, 505 in 2048, 520 in 4096).
  // A part costs as many floats as there are keys, and the join reads all of them: 64 at most.
  a.nsplit = 1;
  if (a.cap == 0)
    a.nsplit = (int)max((int64_t)1, min(min((int64_t)2048 / (groups * units), rows / (a.blocks == 1 ? 256 : 512)), (int64_t)64));
  // (a workgroup walks over several groups of keys where there are very many)
  groups = min(groups, max((int64_t)1, ((int64_t)1 << 20) / units));
  a.key_groups = (int)groups;
  a.magic = a.group == 1 ? 0u : (uint32_t)(((1ull << 32) + a.group - 1) / a.group);
}

hipError_t launch_mass(const MassLaunch& a, hipStream_t stream) {
  const void* f = a.bf16 ? mass_kernel_of<true>(a) : mass_kernel_of<false>(a);
  const hipError_t e = launch_one(f, dim3(a.key_groups * a.nsplit * a.c.num_kv_heads, 1, a.b.n_seqs), 256, stream, a);
  if (e != hipSuccess || a.nsplit == 1) return e;
  return launch_one((const void*)mass_join_kernel, dim3((unsigned)((a.b.max_kv + 255) / 256), a.c.num_kv_heads, a.b.n_seqs), 256,
                    stream, a);
}

}  // namespace prr
