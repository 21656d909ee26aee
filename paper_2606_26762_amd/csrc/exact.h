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
constexpr int EX_MIN_TILES = 4;  // 64-key (bf16) or 32-key (float32) tiles that a context split has at least
constexpr int EX_FEW = 32;        // rows per kv head of a request that the few-rows kernel takes
constexpr int EX_FEW_WAVES = 2048;  // waves of the few-rows kernel, at most (two to a SIMD)
constexpr int MAX_REQUESTS = 8192;
constexpr int MAX_AXES = 8;

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
  int min_tiles;  // key tiles that a split has at least
  int waves;      // waves of a float32 row block
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
