// Internal declarations of the handle-free calls: exact attention (exact.hip),
// rotary positions and block tables (tokens.hip), their host side (exact.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>
#include <string>

#include "protokv.h"

namespace pkv {

// Message of the last failure without a handle on this thread (protokv.cpp).
std::string& call_error();

constexpr int EX_ROWS = 256;      // query rows per workgroup of the bf16 kernel (8 waves of 32), or half as many
constexpr int EX_ROWS_F32 = 32;   // query rows per workgroup of the float32 kernel
constexpr int EX_MAX_SPLITS = 32, EX_MAX_SPLITS_F32 = 64;
constexpr int EX_MIN_TILES = 4;  // a context of fewer than twice as many tiles (64 keys bf16, 32 float32) is not split
constexpr int EX_FEW = 32;        // rows per kv head of a request that the few-rows kernel takes
constexpr int EX_FEW_WAVES = 2048;  // waves of the few-rows kernel, at most (two to a SIMD)
constexpr int MAX_REQUESTS = 8192;
constexpr int MAX_AXES = 8;

// Context splits of a block with `tiles` key tiles, at most `most`, and tiles of each:
// the last split has what is left, one tile or more.
constexpr int ex_splits(int most, int tiles, int& per) {
  const int room = tiles / EX_MIN_TILES > 1 ? tiles / EX_MIN_TILES : 1, want = most < room ? most : room;
  per = (tiles + want - 1) / want > 1 ? (tiles + want - 1) / want : 1;
  return (tiles + per - 1) / per > 1 ? (tiles + per - 1) / per : 1;
}

// bf16 row blocks over pages: a split's tiles t0 .. t1 - 1 find their rows by page ids
// staged in LDS, runs of ex_run_tiles tiles (16 at least), two runs at a time.  Tiles up
// to ex_ids_last are located before the first period or in it, from the runs of t0 and
// of that tile; tile t + 4 in period t + 1 at the earliest, so that its run, where it
// begins one (ex_ids_due), is staged behind the barrier before period t.
constexpr int EX_KEYS = 64;   // keys per tile
constexpr int EX_IDS = 1024;  // page ids in a run
constexpr int ex_run_tiles(int shift) { return (EX_IDS << shift) / EX_KEYS; }
constexpr int ex_ids_last(int t0, int t1) { return t0 + 3 < t1 ? t0 + 3 : t1 - 1; }
constexpr bool ex_ids_due(int t, int t1, int run_tiles) { return t + 4 < t1 && (t + 4) % run_tiles == 0; }

// One launch of exact attention.  Query rows of a kv head: row r of sequence i
// is token r / grp, query head kvh * grp + r % grp.
struct ExactArgs {
  const void *q, *k, *v;  // k, v: rows (prompt) or pages
  void* o;
  float* lse;
  const void* po;         // prior, or null
  const float* pl;
  const int32_t *cu, *kv_len, *table;
  float *part_o, *part_ml;  // [kv head][row block][split][row][D] and [..][2]: m, l
  long long qs, ks, vs;     // bytes between rows
  int n, total, max_add;
  int Hq, Hkv, grp;
  int stride, shift, num_pages;  // block table row, log2 page size
  // few-rows kernel: two partials per wave [wave][2][few_rows][D], [..][2], and the
  // split item that begins in a wave (see k_exact_few)
  float *few_o, *few_ml;
  int32_t* few_meta;
  int few, few_rows;  // its waves (0: not launched, the row blocks take every request), its rows at most
  int rows;    // query rows of a row block
  int blocks;  // row-block indices per kv head (0: no row blocks)
  int splits;  // most context splits of a row block
  int waves;   // waves of a float32 row block
};

struct RotateArgs {
  const uint8_t *q, *k, *v;
  uint8_t *qo, *ko, *kp, *vp;
  const int32_t *pos, *slots;
  long long qs, ks, vs, qos, kos;  // bytes between rows
  long long ps;                    // entries between axes
  int N, Hq, Hkv, shift;
  int nslots;                      // slots of the pages (0: nothing is stored)
  int parts;                       // waves per token
  uint8_t axis[64];
  double inv[64];                  // theta^(-2i/D)
};

hipError_t launch_exact(const ExactArgs& a, bool fp32, bool paged, hipStream_t st);
hipError_t launch_rotate(const RotateArgs& a, bool fp32, hipStream_t st);
hipError_t launch_page_plan(const protokv_page_plan_args& a, hipStream_t st);

}  // namespace pkv
