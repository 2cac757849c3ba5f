// Attention of single tokens: how a call is split, and its launches (prr_decode_impl.h: the kernels).
#include "prr_decode_impl.h"

namespace prr {

void plan_decode(DecodeLaunch& a) {
  int64_t most = a.cap > 0 ? (int64_t)a.cap * a.c.page_size : a.b.max_kv;
  if (a.shape && a.sh.window && a.cap == 0) most = min(most, (int64_t)a.sh.window + kTile - 1);
  const int64_t tiles = max((most + kTile - 1) / kTile, (int64_t)1);
  const int64_t units = (int64_t)a.b.n_seqs * a.c.num_kv_heads;
  // Parts of 64 tiles (eight a wave: less, and starting and merging parts outweighs them; 512 parts of
  // 32 tiles for 2 x 8192: 26.6 us, 256 of 64: 20.0) or of the share of 512 workgroups, two a CU; where that
  // leaves CUs idle, as many parts as CUs, of a tile a wave at least (2 x 256 tiles: 9.7 us, 18.0 in parts of
  // 64).  Lengths are bounds here: parts
  // of at most 256 tiles keep one long sequence among short ones from being one workgroup's (64 sequences x 8
  // KV heads, one of 131072 tokens and 63 of 500: 190 us instead of 1383), unless that takes more than 65536 workgroups,
  // most of which would find nothing to do.
  const int64_t all = tiles * units;
  int64_t per = max((int64_t)64, min((all + 511) / 512, max((int64_t)256, all / 65536)));
  if (all < 64 * 256) per = (all + 255) / 256;
  per = (min(per, tiles) + NW - 1) / NW * NW;
  a.tiles_per_split = (int)per;
  a.nsplit = (int)((tiles + per - 1) / per);
}

hipError_t launch_decode(const DecodeLaunch& a, hipStream_t stream) {
  const void* f = a.shape ? (a.bf16 ? shaped_decode_fn<true>(a, false) : shaped_decode_fn<false>(a, false))
                          : (a.bf16 ? decode_fn<true, 0>(a.e4m3) : decode_fn<false, 0>(a.e4m3));
  const hipError_t e = launch_one(f, dim3(a.nsplit, a.c.num_kv_heads, a.b.n_seqs), NW * kWave, stream, a);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const void* join = a.shape ? (a.bf16 ? shaped_decode_fn<true>(a, true) : shaped_decode_fn<false>(a, true))
                             : (a.bf16 ? (const void*)merge_parts_kernel<true> : (const void*)merge_parts_kernel<false>);
  return launch_one(join, dim3(4 * a.group, a.c.num_kv_heads, a.b.n_seqs), 256, stream, a);
}

}  // namespace prr
