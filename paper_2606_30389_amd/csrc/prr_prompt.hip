// Attention of packed prompts: how a call is split, and its launches (prr_prompt_impl.h: the kernels).
#include "prr_prompt_impl.h"

namespace prr {

void plan_prompt(PromptLaunch& a) {
  int64_t key_tiles = max(((int64_t)a.b.max_kv + kTokens - 1) / kTokens, (int64_t)1);
  if (a.shape && a.sh.window && !a.sh.prefix) {  // the tokens of 256 rows, the window behind the first, whole tiles
    const int64_t tokens = (255 + a.group) / a.group + 1 + (int64_t)a.sh.window;
    key_tiles = min(key_tiles, (tokens + 2 * kTokens - 2) / kTokens);
  }
  // Parts of a row tile's keys.  Fewer workgroups than CUs: as many parts, of at least eight tiles, as fill
  // the chip once (509 new of 65536 tokens, 28 / 4 heads: 460 us in four parts, 1403 in one; twice as many small
  // ones fill it better, but joining them and power take that back: 472 in nine).  With a shape, two workgroups of four waves
  // on a CU (four sequences of 500 new and up to 20000 tokens, window 2000, cap: 71 us, 79 with one, 75 of eight waves).
  // Enough workgroups, but so few that one sequence with many more keys than the others could outlast them
  // all: parts of 512 tiles, eight at most, for 2% where the lengths are alike (16 new tokens of 64 sequences, one of 131072 tokens
  // and 63 of 500, 32 / 8 heads: 2812 us in one part, 766 in four).
  const auto parts_of = [&](int64_t units) -> int64_t {
    const int64_t fill = a.shape && a.waves == 4 ? 512 : 256;
    if (units <= fill) return max((int64_t)1, min(fill / max(units, (int64_t)1), key_tiles / 8));
    return units < 4096 ? min((key_tiles + 511) / 512, (int64_t)8) : 1;
  };
  // Waves of a workgroup.  Four, and two workgroups a CU, start and end under each other's work; eight in turns keep the matrix
  // cores busier over many tiles.  With a cap the softmax outlasts the products, and turns gain less: nine packed prompts
  // with a window of 1024 tokens and a cap 214 us with four, 230 with eight, 2047 tokens with a cap 78, 95; 8192 tokens 705, 701.
  // Without, 2047 tokens 62, 65; two of 12000 with a window of 2000 642, 622.  Where eight waves make fewer workgroups
  // than CUs, four do up to 48 tiles (2500 tokens, 16 / 4 heads, 76, 90; 4000 79, 79; 8 x 160 over 4000 138, 132) and with
  // documents, most of whose parts are empty (5163 tokens, 5 / 1 heads, eight documents, 62, 72); rows that eight waves
  // would not fill by half always do (16 new of 65536 tokens, 32 / 8 heads, 70, 103).
  a.waves = key_tiles <= 16 ? 4 : 8;
  if (a.shape) {
    const int64_t rows = (int64_t)a.b.max_q * a.group;
    const bool few = rows * a.b.n_seqs * a.num_kv_heads <= 256 * 256;
    if (key_tiles <= (a.shape & kShapeCap ? 64 : few ? 48 : 32) || rows <= 128 || (few && a.sh.first)) a.waves = 4;
  }
  a.magic = a.group == 1 ? 0u : (uint32_t)(((1ull << 32) + a.group - 1) / a.group);
  const int rows = 32 * a.waves;
  const int64_t per = ((int64_t)a.b.max_q * a.group + rows - 1) / rows, each = a.b.n_seqs * per;
  const int64_t packed = (int64_t)a.b.total_q * a.group / rows + a.b.n_seqs;
  const bool alike = each <= packed || !a.b.cu_q;
  a.seq_tiles = alike ? (int)per : 0;
  a.tiles = (int)(alike ? each : packed);
  const int64_t parts = parts_of((int64_t)a.tiles * a.num_kv_heads);
  a.part_tiles = (int)((key_tiles + parts - 1) / parts);
  a.nsplit = (int)((key_tiles + a.part_tiles - 1) / a.part_tiles);
}

hipError_t launch_prompt(const PromptLaunch& a, hipStream_t stream) {
  const bool paged = a.b.page_table != nullptr;
  const void* f = a.shape ? (a.bf16 ? shaped_prompt_fn<true>(a) : shaped_prompt_fn<false>(a))
                          : (a.bf16 ? prompt_fn<true, 0>(paged, a.waves) : prompt_fn<false, 0>(paged, a.waves));
  const hipError_t e = launch_one(f, dim3(a.tiles * a.num_kv_heads, a.nsplit), a.waves * kWave, stream, a);
  if (e != hipSuccess || a.nsplit == 1) return e;
  const int64_t rows = (int64_t)a.b.total_q * a.num_kv_heads * a.group;
  if (a.nsplit > 8)  // (few rows; 16 new tokens over 131072, 128 parts: 61 us, 101 with one group a row)
    return launch_one(a.bf16 ? (const void*)merge_prompt_kernel<true, 8> : (const void*)merge_prompt_kernel<false, 8>,
                      dim3((unsigned)rows), 256, stream, a);
  return launch_one(a.bf16 ? (const void*)merge_prompt_kernel<true, 1> : (const void*)merge_prompt_kernel<false, 1>,
                    dim3((unsigned)((rows + 7) / 8)), 256, stream, a);
}

}  // namespace prr
