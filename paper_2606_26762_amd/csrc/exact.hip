// Exact attention of libprotokv for gfx950: packed prompts over themselves and
// new tokens over a paged cache, causal, grouped heads, joined with a prior.
//
//   o_r = sum_{key <= p_r} e^(s_rk) v_k / sum e^(s_rk),  s_rk = q_r . k_k / sqrt(D)
//
// in one pass over the keys with a running reference m and sum l per row:
// O <- O 2^(m - m') + sum 2^(s log2 e - m') v.  Query rows of a kv head are
// packed: row r of a sequence is token r / grp, query head kvh * grp + r % grp,
// so every key tile serves all heads of the group.
#include <algorithm>
#include <type_traits>

#include "exact.h"
#include "pkv_internal.h"

namespace pkv {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
typedef short v4i16 __attribute__((ext_vector_type(4)));
typedef short v8i16 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4i16 lds_v4i16;
typedef __attribute__((address_space(3))) const u16x8 lds_u16x8;
typedef __attribute__((address_space(1))) const f32x4 gbl_f32x4;

namespace {

constexpr float EX_LOG2E = 1.4426950408889634f;
constexpr float EX_LN2 = 0.6931471805599453f;
constexpr float EX_SCALE = EX_LOG2E * 0.08838834764831845f;  // log2 e / sqrt(D)
// Reference of a row that has seen no key: below every finite score, and
// 2^(-inf - EX_NONE) is 0, not NaN.
constexpr float EX_NONE = -3.402823466e38f;

// A row block: `rows` rows of sequence `seq`, this block's first one `row0`.
struct Item {
  int seq, s0;   // first token row of the sequence in q
  int add, rows; // its tokens; its query rows of one kv head
  int row0;
  int off;       // position of its first token
  int kend;      // keys that the block's last row sees
};

// Row block blk of sequence i, whose rows are c0 .. c1 - 1; false if there is none.
template <int R>
__device__ __forceinline__ bool set_item(const ExactArgs& a, int i, int c0, int c1, int blk, Item& it) {
  it.seq = i;
  it.s0 = c0;
  it.add = c1 - c0;
  if (it.add <= 0 || blk < 0) return false;
  it.rows = min(it.add, a.max_add) * a.grp;
  if (blk >= (it.rows + R - 1) / R || (a.few && it.rows <= EX_FEW)) return false;
  it.row0 = blk * R;
  int kv = it.add;
  it.off = 0;
  if (a.kv_len) {
    kv = min(max(__builtin_amdgcn_readfirstlane(a.kv_len[i]), 0), a.stride << a.shift);
    it.off = kv - it.add;
  }
  const int last = (min(it.rows, it.row0 + R) - 1) / a.grp;
  it.kend = min(max(it.off + last + 1, 0), kv);
  return true;
}

// Row-block index b of R rows: sequence i has the indices from
// f(i) = floor(cu[i] grp / R) + i, non-decreasing, so it is found by comparing 64
// entries at a time; indices behind a sequence's rows are left empty.  Every
// lane of the wave takes part; false (uniform) if the block is empty.
template <int R>
__device__ __forceinline__ bool find_item(const ExactArgs& a, int b, Item& it) {
  const int lane = threadIdx.x & 63;
  auto entry = [&](int i) { return min(max(a.cu[i], 0), a.total); };
  auto first = [&](int c, int i) { return (int)((unsigned)(c * a.grp) / R) + i; };
  int lo = 0, hi = a.n, c0, c1;
  for (;;) {
    const int step = (hi - lo + 63) / 64, i = lo + lane * step;
    const int c = entry(min(i, a.n));
    const bool in = i < hi && first(c, i) <= b;
    const int l = max(__popcll(__ballot(in)), 1) - 1;
    if (step == 1) {  // lane l has the entry, the next lane the one behind it
      c0 = __builtin_amdgcn_readlane(c, l);
      lo = __builtin_amdgcn_readfirstlane(lo + l);
      c1 = l < 63 ? __builtin_amdgcn_readlane(c, l + 1) : __builtin_amdgcn_readfirstlane(entry(lo + 1));
      break;
    }
    lo += l * step;
    hi = min(hi, lo + step);
  }
  return set_item<R>(a, lo, c0, c1, b - first(c0, lo), it);
}

// The sum of x over the wave.
__device__ __forceinline__ int wave_total(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8: rows of 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return __builtin_amdgcn_readlane(x, 63);
}

// Block d of a prompt batch of at most 64 sequences, blocks in the order of falling
// position in their sequences, the dearest first (by sequences, a long one at the
// front of the batch came last: 2000 tokens before 60 times 100, 87 us against 73).  Lane i holds sequence i;
// sum_i max(blocks_i - k, 0) blocks are at position k or behind.
template <int R>
__device__ __forceinline__ bool find_dearest(const ExactArgs& a, int d, Item& it) {
  const int lane = threadIdx.x & 63;
  auto entry = [&](int i) { return min(max(a.cu[min(i, a.n)], 0), a.total); };
  const int c0 = entry(lane), c1 = entry(lane + 1);
  const int nb = lane < a.n ? (min(max(c1 - c0, 0), a.max_add) * a.grp + R - 1) / R : 0;
  int k = 0, hi = a.total * a.grp / R + 1, behind = 0;  // blocks at k or behind: more than d; at hi: `behind`
  if (d >= wave_total(nb)) return false;
  while (hi - k > 1) {  // uniform
    const int mid = (k + hi) >> 1, c = wave_total(max(nb - mid, 0));
    if (c > d) {
      k = mid;
    } else {
      hi = mid;
      behind = c;
    }
  }
  const unsigned long long at = __ballot(nb > k);
  const int rank = __builtin_amdgcn_mbcnt_hi((unsigned)(at >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)at, 0));
  const int i = __ffsll(__ballot(nb > k && rank == d - behind)) - 1;
  return set_item<R>(a, i, __builtin_amdgcn_readlane(c0, i), __builtin_amdgcn_readlane(c1, i), k, it);
}

// Weights of a row's own result (log2 of its sum: own2) and of the prior's (its
// log-sum-exp p), and the log-sum-exp of both.
struct Join {
  float own, prior, lse;
};
__device__ __forceinline__ Join join_of(float own2, float p) {
  const float own = own2 * EX_LN2;
  if (p == -INFINITY) return {1.f, 0.f, own};
  if (own == -INFINITY) return {0.f, 1.f, p};
  const float m = fmaxf(own, p);
  const float e1 = expf(own - m), e2 = expf(p - m), s = e1 + e2;
  return {e1 / s, e2 / s, m + logf(s)};
}

// Output row `row` from N pieces of four dims of this lane, piece i at dim(i) with
// the own value x(i) (normalised): joined with the prior, whose loads go out
// together (one after the other, each beside its store, they were a third of a
// short prompt's time).  -> the row's log-sum-exp.
template <int FP32, int N, typename X, typename DIM>
__device__ __forceinline__ float write_row(const ExactArgs& a, size_t row, float own2, X x, DIM dim) {
  typedef __bf16 half4 __attribute__((ext_vector_type(4)));
  auto store = [&](int i, f32x4 v) {
    const size_t e = row * D + dim(i);
    if constexpr (FP32) {
      *reinterpret_cast<f32x4*>((float*)a.o + e) = v;
    } else {
      half4 b;
#pragma unroll
      for (int c = 0; c < 4; ++c) b[c] = (__bf16)v[c];
      *reinterpret_cast<half4*>((__bf16*)a.o + e) = b;
    }
  };
  if (!a.pl) {  // uniform
#pragma unroll
    for (int i = 0; i < N; ++i) store(i, x(i));
    return own2 * EX_LN2;
  }
  std::conditional_t<FP32 != 0, f32x4, half4> p[N];
  const float pl = a.pl[row];
#pragma unroll
  for (int i = 0; i < N; ++i) p[i] = *(reinterpret_cast<decltype(&p[0])>(const_cast<void*>(a.po)) + (row * D + dim(i)) / 4);
  const Join j = join_of(own2, pl);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    f32x4 v = x(i);
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const float q = (float)p[i][c] * j.prior;
      v[c] = j.prior == 0.f ? v[c] : j.own == 0.f ? q : fmaf(v[c], j.own, q);  // what has no weight may be anything
    }
    store(i, v);
  }
  return j.lse;
}

// A hidden key has weight 0, but 0 x inf and 0 x NaN are not 0.  Where a tile with
// hidden keys holds such values they are taken out of the product (0 in their
// place), and two more products with a 1 where a value was +inf or NaN, or -inf or
// NaN, tell which outputs they belong to: those with a positive weight on one.
// Two bfloat16 at a time, flags in each half's bit 15 (no compares: their masks
// would not fit the scalar registers).
__device__ __forceinline__ uint32_t odd_flags(uint32_t w) { return (w & 0x7F807F80u) + 0x00800080u; }
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint32_t odd_flags(v8i16 v) {
  const u32x4 w = __builtin_bit_cast(u32x4, v);
  return odd_flags(w[0]) | odd_flags(w[1]) | odd_flags(w[2]) | odd_flags(w[3]);
}
constexpr uint32_t ODD = 0x80008000u;
// WHAT 0: the values without the odd ones; 1, -1: a 1 for each of that sign
template <int WHAT>
__device__ __forceinline__ bf16x8 odd_operand(v8i16 v) {
  u32x4 w = __builtin_bit_cast(u32x4, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t odd = odd_flags(w[i]) & ODD;
    if (WHAT == 0) {
      w[i] &= ~((odd >> 15) * 0xFFFFu);
    } else {
      const uint32_t nan = ((w[i] & 0x007F007Fu) + 0x007F007Fu) << 8;
      w[i] = ((odd & (nan | (WHAT > 0 ? ~w[i] : w[i]))) >> 15) * 0x3F80u;
    }
  }
  return __builtin_bit_cast(bf16x8, w);
}
// 0, of which the compiler does not know it: what is read at an address with it
// added is read anew, so that the passes below do not keep each other's operands
__device__ __forceinline__ int anew() {
  int z = 0;
  asm volatile("" : "+v"(z));
  return z;
}
template <int SIGN>
__device__ __forceinline__ void add_odd(f32x16& o, const f32x16& hits) {
#pragma unroll
  for (int i = 0; i < 16; ++i) o[i] += hits[i] > 0.f ? (SIGN > 0 ? INFINITY : -INFINITY) : 0.f;
}

// Barrier for LDS traffic only: outstanding global loads are not waited for.
__device__ __forceinline__ void ex_barrier() {
  __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
  asm volatile("s_barrier" ::: "memory");
}

constexpr int EX_TILE = EX_KEYS * D * 2;  // one K or V tile, 16 KB
constexpr int EX_NBUF = 4;              // tiles t - 1 and t in use, t + 1 and t + 2 loading

// Workgroup = eight waves of 32 query rows each.  Tiles of 64 keys go straight from
// global memory into LDS (global_load_lds_dwordx4), two tiles ahead, four whole rows
// to an instruction (16 bytes of 64 rows each, or 64 of 16, kept the address unit
// busy for most of a tile's time).  Row r lies at r * 256 with its 16-byte chunks
// permuted, chunk c of K at place c ^ (r % 16), of V at c ^ 4 (r % 4), so that the
// operand reads (16 rows of one chunk; 4 rows of 4 chunks) fall on distinct banks.
// S^T = K Q^T and O^T = V^T P on v_mfma_f32_32x32x16_bf16,
// V^T through ds_read_b64_tr_b16: each lane holds one query column, so the
// softmax is lane-local plus one exchange with the partner lane.
// Bound by the matrix cores at the clock that their power leaves: 8192 tokens of
// 32 / 8 heads 503 - 516 us, 1.08 PFLOP/s of what is seen (a plain product of 8192^3
// reaches 1.12), 4 x 512 tokens over 16 384 of 28 / 4 heads 477 - 502 us, 1.0, in one
// round of 224 workgroups: an eighth of the compute units has none.  KH = 2:
// two waves take a row's keys, half of every tile each; 128 rows to a workgroup, for
// launches that 256 would leave in few rounds (the rule and its figures stand
// with the host's block counts).
template <int PAGED, int KH>
__global__ __launch_bounds__(512, 1) void k_exact_bf16(ExactArgs a) {
  __shared__ __attribute__((aligned(256))) uint8_t s_kv[EX_NBUF][2][EX_TILE];
  __shared__ int32_t s_ids[2][PAGED ? EX_IDS : 1];  // two runs of page ids, in turn
  __shared__ unsigned long long s_bad[8];  // keys of a tile on pages that are none
  __shared__ __attribute__((aligned(256))) uint8_t s_zero[EX_TILE];  // V of a tile whose products are done already
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // kv heads innermost: workgroups are dealt round robin to the 8 XCDs, so a
  // head's keys meet in few L2s; the last row blocks, which see the most keys, first
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv;
  const int split = rest % a.splits, blk = a.blocks - 1 - rest / a.splits;
  Item it;
  constexpr int ROWS = EX_ROWS / KH;
  if (!PAGED && a.n <= 64 ? !find_dearest<ROWS>(a, a.blocks - 1 - blk, it) : !find_item<ROWS>(a, blk, it))
    return;  // uniform in the workgroup
  int per;
  const int tiles = (it.kend + EX_KEYS - 1) / EX_KEYS;
  const int nsp = ex_splits(a.splits, tiles, per);
  if (split >= nsp) return;
  const int t0 = split * per, t1 = min(tiles, t0 + per);

  const int m = lane & 31, half = lane >> 5;
  const int kh = KH == 2 ? wave >> 2 : 0;  // key half of every tile that this wave takes
  const int rw = it.row0 + (wave % (8 / KH)) * 32, r = rw + m;
  const bool wvalid = rw < it.rows, rvalid = r < it.rows;  // wvalid is uniform
  const int tok = rvalid ? r / a.grp : 0;
  const int head = kvh * a.grp + (rvalid ? r - tok * a.grp : 0);
  const size_t orow = (size_t)(it.s0 + tok) * a.Hq + head;
  const int klim = rvalid ? it.off + tok : -1;  // last key that this lane's row sees
  const int wtok0 = wvalid ? rw / a.grp : 0, wtok1 = wvalid ? (min(it.rows, rw + 32) - 1) / a.grp : 0;
  const int wfull = it.off + wtok0 + 1;  // keys that every row of the wave sees
  const int wend = it.off + wtok1 + 1;   // keys that some row of it sees

  bf16x8 bq[8];
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 oacc[4] = {zero, zero, zero, zero};
  // (a row's first reference is its first tile's maximum, so a row with one key
  // has weight 1 on it and returns its value exactly)
  float mref = EX_NONE, lrun = 0.f;

  const uint8_t* kb = (const uint8_t*)a.k + (PAGED ? 0 : (size_t)it.s0 * a.ks + kvh * (D * 2));
  const uint8_t* vb = (const uint8_t*)a.v + (PAGED ? 0 : (size_t)it.s0 * a.vs + kvh * (D * 2));
  const int tpc = PAGED ? ex_run_tiles(a.shift) : 1;  // tiles per staged run of page ids
  auto load_ids = [&](int t) {  // the run that tile t is in
    const int e0 = (t / tpc) * EX_IDS, n = min(EX_IDS, ((it.kend - 1) >> a.shift) + 1 - e0);
    const int32_t* row = a.table + (size_t)it.seq * a.stride + e0;
    for (int i = tid; i < n; i += 512) s_ids[(t / tpc) & 1][i] = row[i];
  };
  // byte offset of key's row; bad: its page is none (page 0 is read instead)
  auto paged_row = [&](int key, bool& bad) {
    const int e = key >> a.shift, id = s_ids[(e / EX_IDS) & 1][e & (EX_IDS - 1)];
    bad = (unsigned)id >= (unsigned)a.num_pages;
    const size_t page = bad ? 0 : id;
    return ((((page * a.Hkv + kvh) << a.shift) + (key & ((1 << a.shift) - 1)))) * (size_t)(D * 2);
  };
  // this lane's part of the rows 4 wave + lane / 16 and + 32 of a tile
  const int ckey = ((lane & 15) ^ ((4 * wave + (lane >> 4)) & 15)) * 16;
  const int cval = ((lane & 15) ^ ((lane >> 4) << 2)) * 16;
  const uint8_t *next_k[2], *next_v[2];  // where the parts of the tile to be loaded next lie
  auto locate = [&](int t) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      // keys past the last one repeat it (they are masked)
      const int key = min(t * EX_KEYS + 32 * q + 4 * wave + (lane >> 4), it.kend - 1);
      const uint8_t *rk, *rv;
      if constexpr (PAGED) {
        bool bad;
        const size_t at = paged_row(key, bad);
        rk = kb + at;
        rv = vb + at;
      } else {
        rk = kb + (size_t)key * a.ks;
        rv = vb + (size_t)key * a.vs;
      }
      next_k[q] = rk + ckey;
      next_v[q] = rv + cval;
    }
    if constexpr (PAGED) {
      if (wave == 0) {
        bool bad;
        paged_row(min(t * EX_KEYS + lane, it.kend - 1), bad);
        const unsigned long long bm = __ballot(bad);
        if (lane == 0) s_bad[t & 7] = bm;
      }
    }
  };
  auto load = [&](int t, int part) {  // one of the four instructions that load tile t
    const int q = part >> 1;
    if (part & 1) lds_dma16(next_v[q], s_kv[t % EX_NBUF][1] + (wave + 8 * q) * 1024);
    else lds_dma16(next_k[q], s_kv[t % EX_NBUF][0] + (wave + 8 * q) * 1024);
  };
  auto issue = [&](int t) {
    locate(t);
#pragma unroll
    for (int part = 0; part < 4; ++part) load(t, part);
  };
  const int grp16 = lane >> 4, s16 = lane & 15;
  // One tile's work in two halves: products are the matrix ones (the last tile's
  // P V, then this tile's K Q), weights() the softmax between them.
  constexpr int NH = 2 / KH, NST = 4 / KH;  // a wave's 32-key halves and 16-key steps of a tile, and steps of K
  f32x16 s[2];     // scores, then weights (KH = 2: of even and odd 16-dim steps, then all in the first)
  bf16x8 p_next;   // the first step's weights
  bf16x8 v_next[4];  // and its V operands
  // P operand of 16-key step st: the weights in bfloat16, the type in which the matrix
  // core takes the values at 16 times float32's rate; each is within 2^-8 of itself.  Sums,
  // references and O stay float32, and the sum is of the unrounded weights: outputs are
  // within 2.3e-3 of float64's (relative, in the mean square), 1.7e-3 with the output's own
  // rounding alone.
  auto weight_operand = [&](int st) {
    bf16x8 p;
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (__bf16)s[st >> 1][(st & 1) * 8 + i];
    return p;
  };
  auto key_base = [&](int t) {
    return (uint32_t)(uintptr_t)(lds_u16x8*)s_kv[t % EX_NBUF][0] + kh * 8192 + (m * 256 + ((m & 15) ^ half) * 16);
  };
  // K operand of key half h, 16-dim step kk: chunk 2 kk + half of key 32 h + m
  auto read_k = [&](uint32_t kl, int h, int kk) {
    return __builtin_bit_cast(bf16x8, *((lds_u16x8*)(uintptr_t)(kl ^ (kk * 32)) + h * 512));
  };
  // V^T operand of 32-dim block b, 16-key step st: positions half * 8 + i are
  // keys 16 st + 4 half + {0..3} (i < 4) and + 8 (i >= 4), as P's registers are.
  // Source lane i of 16 reads key i / 4 of its four, dims 4 (i % 4) .. + 3.
  auto value_base = [&](const uint8_t* tile) {
    return (uint32_t)(uintptr_t)(lds_v4i16*)tile + kh * 8192 + (4 * half + (s16 >> 2)) * 256 +
           (((grp16 & 1) * 2 + ((s16 & 3) >> 1)) ^ ((s16 >> 2) << 2)) * 16 + (s16 & 1) * 8;
  };
  auto read_v = [&](uint32_t vl, int b, int st) {
    lds_v4i16* p = (lds_v4i16*)(uintptr_t)(vl ^ (b * 64)) + st * 512;
    const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p);
    const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(p + 256);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  };
  // Eight steps of four products, V's (O of tile tv) and K's (S of tile tk); behind
  // each product the same one's operand of the next step is read (a step's eight
  // transposed reads in a row left the matrix core waiting a fifth of its time).
  // Tile tk + 2's four loads go out between the steps.
  bool done = false;  // the last tile's P V is
  auto products = [&](int tv, int tk, auto with_v, auto with_k) {
    const bool more = tk + 2 < t1;  // uniform
    constexpr int F = decltype(with_v)::value ? 0 : NST, L = decltype(with_k)::value ? 2 * NST : NST;
    const uint32_t vl = value_base(done ? s_zero : s_kv[tv % EX_NBUF][1]), kl = key_base(tk);
    __builtin_amdgcn_s_setprio(1);
    bf16x8 op[2][4], p[2];
    float part[4] = {0.f, 0.f, 0.f, 0.f};
    auto read = [&](int step, int j) {
      const int ks = step - NST;
      op[step & 1][j] = ks < 0 ? __builtin_bit_cast(bf16x8, read_v(vl, j, step))
                               : KH == 1 ? read_k(kl, j & 1, 2 * ks + (j >> 1)) : read_k(kl, 0, 4 * ks + j);
    };
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (F == 0) op[0][j] = v_next[j];
      else read(F, j);
    }
    p[0] = p_next;
#pragma unroll
    for (int step = F; step < L; ++step) {
      if (more) {
        constexpr int N = L - F;  // 8, 4 or 2 steps for the four loads
        if (N == 2) load(tk + 2, 2 * (step - F));
        if (N < 8 || ((step - F) & 1)) load(tk + 2, N == 8 ? (step - F) >> 1 : N == 4 ? step - F : 2 * (step - F) + 1);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        __builtin_amdgcn_sched_barrier(0);
        if (step < NST) {
          oacc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[step & 1][j], p[step & 1], oacc[j], 0, 0, 0);
        } else {
          const int ks = step - NST, kk = KH == 1 ? 2 * ks + (j >> 1) : 4 * ks + j;
          s[j & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(op[step & 1][j], bq[kk], kk < KH ? zero : s[j & 1], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (step + 1 < L) read(step + 1, j);
        if (step < NST) {  // the next step's weights, and the sum of this one's
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            if (step < NST - 1) p[(step + 1) & 1][2 * j + e] = (__bf16)s[(step + 1) >> 1][((step + 1) & 1) * 8 + 2 * j + e];
            part[2 * (j & 1) + e] += s[step >> 1][(step & 1) * 8 + 2 * j + e];
            asm volatile("" : "+v"(part[2 * (j & 1) + e]));  // here, beside the products
          }
        }
      }
    }
    if (tk + 3 < t1) locate(tk + 3);
    if (F == 0) lrun += (part[0] + part[1]) + (part[2] + part[3]);  // this half's keys; the halves meet at the end
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_setprio(0);
  };
  // Softmax weights of tile t; true if its P V is done as well: hidden keys with
  // infinite or NaN values.
  auto weights = [&](int t) {
    if (KH == 2) s[0] += s[1];
    bool hidden = (t + 1) * EX_KEYS > wfull;
    unsigned long long bad = 0;
    if constexpr (PAGED) {
      bad = s_bad[t & 7];
      hidden |= __builtin_amdgcn_readfirstlane((int)(bad != 0)) != 0;
      bad >>= 32 * kh + 4 * half;
    }
    if (hidden) {  // uniform
      const int rel = klim - t * EX_KEYS - 32 * kh - 4 * half;
#pragma unroll
      for (int h = 0; h < NH; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i)  // key 32 h + 8 (i / 4) + i % 4 + 4 half of the tile
          s[h][i] = 32 * h + 8 * (i >> 2) + (i & 3) > rel ? -INFINITY : s[h][i];
      if constexpr (PAGED) {
        if (__ballot(bad != 0)) {
#pragma unroll
          for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int i = 0; i < 16; ++i)
              s[h][i] = (bad >> (32 * h + 8 * (i >> 2) + (i & 3))) & 1 ? -INFINITY : s[h][i];
        }
      }
    }
    float tmax = -INFINITY;
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, s[h][i]);
    tmax = fmaxf(tmax, xor32(tmax)) * EX_SCALE;
    // the reference moves up only when a row's maximum exceeds it by more than 8
    // (weights up to 2^8 keep bf16's relative precision)
    const bool grow = tmax > mref + 8.0f;
    if (__ballot(grow)) {  // uniform
      const float mnew = grow ? tmax : mref;
      const float alpha = __builtin_amdgcn_exp2f(mref - mnew);
      lrun *= alpha;
#pragma unroll
      for (int b = 0; b < 4; ++b) oacc[b] *= alpha;
      mref = mnew;
    }
#pragma unroll
    for (int h = 0; h < NH; ++h)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[h][i] = __builtin_amdgcn_exp2f(fmaf(s[h][i], EX_SCALE, -mref));
    p_next = weight_operand(0);
    if (!hidden) return false;  // uniform
    const uint32_t vl = value_base(s_kv[t % EX_NBUF][1]);
    uint32_t odd = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b) {
#pragma unroll
      for (int st = 0; st < NST; ++st) odd |= odd_flags(read_v(vl, b, st));
      __builtin_amdgcn_sched_barrier(0);
    }
    if (!__ballot((odd & ODD) != 0)) return false;  // uniform
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      f32x16 hits = zero;
      uint32_t vz = vl + anew();
#pragma unroll
      for (int st = 0; st < NST; ++st)
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<0>(read_v(vz, b, st)), weight_operand(st), hits, 0, 0, 0);
      oacc[b] += hits;
      __builtin_amdgcn_sched_barrier(0);
      hits = zero;
      vz = vl + anew();
#pragma unroll
      for (int st = 0; st < NST; ++st)
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<1>(read_v(vz, b, st)), weight_operand(st), hits, 0, 0, 0);
      add_odd<1>(oacc[b], hits);
      __builtin_amdgcn_sched_barrier(0);
      hits = zero;
      vz = vl + anew();
#pragma unroll
      for (int st = 0; st < NST; ++st)
        hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<-1>(read_v(vz, b, st)), weight_operand(st), hits, 0, 0, 0);
      add_odd<-1>(oacc[b], hits);
      __builtin_amdgcn_sched_barrier(0);
    }
    return true;
  };

#pragma unroll
  for (int i = 0; i < EX_TILE / 8192; ++i) reinterpret_cast<uint4*>(s_zero)[tid + i * 512] = make_uint4(0, 0, 0, 0);
  if constexpr (PAGED) {
    if (t0 < t1) {
      const int last = ex_ids_last(t0, t1);
      load_ids(t0);
      if (last / tpc != t0 / tpc) load_ids(last);
    }
  }
  ex_barrier();
  // the first tile and the query together, the second tile once they are there: what
  // the compiler waits for knows of no tile
  if (t0 < t1) issue(t0);
  {
    const u16x8* qr = reinterpret_cast<const u16x8*>((const uint8_t*)a.q + (size_t)(it.s0 + tok) * a.qs + head * (D * 2));
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) bq[kk] = __builtin_bit_cast(bf16x8, qr[2 * kk + half]);
  }
  // the prior is brought near: its lse, and the line 128 half .. of its row
  float pl = -INFINITY, near_o = 0.f;
  if (a.pl && rvalid) {
    pl = a.pl[orow];
    near_o = *reinterpret_cast<const float*>((const uint8_t*)a.po + orow * (D * 2) + half * 128);
  }
  wait_vm<0>();
  asm volatile("" ::"v"(near_o));
  if (t0 + 1 < t1) issue(t0 + 1);
  if (t0 + 2 < t1) locate(t0 + 2);
  // Waves w and w + 4 share a SIMD.  In period t waves 0 - 3 form the products of tile
  // t, then its weights, and waves 4 - 7 the weights of tile t - 1, then the products
  // of tile t, so that one wave of a SIMD has the matrix core while the other has the
  // VALU (in step, both wait for the one and then for the other).  A barrier begins
  // each period.  Tile t + 2 is loaded beside the products of tile t: V of tile t - 2,
  // last read in period t - 1, has left its buffer, and the tile is read from period
  // t + 2 on; the rows of tile t + 3 are located behind them.
  auto even = [&](int t) {  // the barrier before period t
    __builtin_amdgcn_sched_barrier(0);
    if (t + 1 < t1) wait_vm<4>();  // this wave's loads of tile t have landed, those of t + 1 may be in flight
    else wait_vm<0>();
    ex_barrier();
    if constexpr (PAGED) {
      // in the place of the ids of tiles up to t + 3 - tpc
      if (ex_ids_due(t, t1, tpc)) load_ids(t + 4);  // uniform
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  // the tiles of which this wave's rows see something are t0 .. tw - 1
  const int tw = wvalid ? max(t0, min(t1, (wend + EX_KEYS - 1) / EX_KEYS)) : t0;
  constexpr std::true_type yes{};
  constexpr std::false_type no{};
  const bool late = wave >= 4;  // uniform
  auto first_barrier = [&](int t) {
    if (!late) even(t);
  };
  auto second_barrier = [&](int t) {
    if (late && t < t1) even(t + 1);
  };
  auto read_next = [&](int t) {  // the first V operands of tile t, whose weights are done
    const uint32_t vl = value_base(done ? s_zero : s_kv[t % EX_NBUF][1]);
#pragma unroll
    for (int j = 0; j < 4; ++j) v_next[j] = __builtin_bit_cast(bf16x8, read_v(vl, j, 0));
  };
  if (late) even(t0);
  int t = t0;
  if (t < tw) {
    first_barrier(t);
    products(t, t, no, yes);
    second_barrier(t);
    done = weights(t);
    read_next(t);
    for (++t; t < tw; ++t) {
      first_barrier(t);
      products(t - 1, t, yes, yes);
      second_barrier(t);
      done = weights(t);
      read_next(t);
    }
    first_barrier(t);
    products(t - 1, t, yes, no);
    second_barrier(t);
    ++t;
  }
  for (; t <= t1; ++t) {
    first_barrier(t);
    if (t + 2 < t1)
#pragma unroll
      for (int part = 0; part < 4; ++part) load(t + 2, part);
    if (t + 3 < t1) locate(t + 3);
    second_barrier(t);
  }
  lrun += xor32(lrun);
  if constexpr (KH == 2) {
    // the waves of key half 1 hand (reference, sum, O) to those of half 0, each
    // relative to its own reference
    float* part = reinterpret_cast<float*>(&s_kv[0][0][0]) + (wave & 3) * 66 * 64;
    __syncthreads();  // every wave is done with the tiles
    if (kh == 1) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) part[(b * 16 + i) * 64 + lane] = oacc[b][i];
      part[64 * 64 + lane] = mref;
      part[65 * 64 + lane] = lrun;
    }
    __syncthreads();
    if (kh == 1) return;
    const float m2 = part[64 * 64 + lane], M = fmaxf(mref, m2);
    const float w1 = __builtin_amdgcn_exp2f(mref - M), w2 = __builtin_amdgcn_exp2f(m2 - M);
    lrun = lrun * w1 + part[65 * 64 + lane] * w2;
    mref = M;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) oacc[b][i] = oacc[b][i] * w1 + part[(b * 16 + i) * 64 + lane] * w2;
  }
  if constexpr (KH == 1) ex_barrier();  // every wave is done with the tiles
  if (!wvalid) return;
  if (nsp > 1) {
    const size_t pr = (((size_t)kvh * a.blocks + blk) * a.splits + split) * ROWS + (r - it.row0);
    if (rvalid) {
#pragma unroll
      for (int b = 0; b < 4; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4*>(a.part_o + pr * D + b * 32 + i * 8 + half * 4) =
              (f32x4){oacc[b][4 * i], oacc[b][4 * i + 1], oacc[b][4 * i + 2], oacc[b][4 * i + 3]};
      if (half == 0) {
        a.part_ml[pr * 2] = mref;
        a.part_ml[pr * 2 + 1] = lrun;
      }
    }
    return;
  }
  // Whole rows to an instruction in the output, and in the prior's loads, which go
  // out first: O goes through the wave's own LDS, row m at m * 512 with its 16-byte
  // pieces permuted, piece c at place c ^ m.  (Eight bytes of 64 places at a time:
  // half of a short prompt's time with a prior.)
  const int row = rvalid ? (int)orow : -1;
  int rows[8];  // output row of this lane's piece of instruction k: row 4 k + lane / 16 of the wave
#pragma unroll
  for (int k = 0; k < 8; ++k) rows[k] = __builtin_amdgcn_ds_bpermute(4 * (4 * k + (lane >> 4)), row);
  u16x8 prior[8];
  if (a.pl) {  // uniform
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (rows[k] >= 0) prior[k] = reinterpret_cast<const u16x8*>(a.po)[(size_t)rows[k] * (D / 8) + (lane & 15)];
  }
  const float own2 = lrun == 0.f ? -INFINITY : mref + log2f(lrun);
  const Join j = join_of(own2, pl);
  // no key: 0; a NaN stays one
  const float w = j.own == 0.f ? 0.f : (lrun > 0.f || lrun != lrun ? 1.0f / lrun : 0.f) * j.own;
  uint8_t* mine = &s_kv[0][0][0] + (KH == 2 ? (wave & 3) * (66 * 64 * 4) : wave * 16384);
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x4 o = {oacc[b][4 * i], oacc[b][4 * i + 1], oacc[b][4 * i + 2], oacc[b][4 * i + 3]};
      const int c = b * 8 + i * 2 + half;
      *reinterpret_cast<f32x4*>(mine + m * 512 + ((c ^ m) * 16)) = w == 0.f ? (f32x4){0.f, 0.f, 0.f, 0.f} : o * w;
    }
  if (half == 0 && rvalid && a.lse) a.lse[orow] = j.lse;
  asm volatile("" ::: "memory");  // the wave's LDS operations run in order
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int lr = 4 * k + (lane >> 4), c = 2 * (lane & 15);
    const float pw = a.pl ? __int_as_float(__builtin_amdgcn_ds_bpermute(4 * lr, __float_as_int(j.prior))) : 0.f;
    const f32x4 lo = *reinterpret_cast<const f32x4*>(mine + lr * 512 + ((c ^ lr) * 16));
    const f32x4 hi = *reinterpret_cast<const f32x4*>(mine + lr * 512 + (((c + 1) ^ lr) * 16));
    bf16x8 o;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      float x = e < 4 ? lo[e & 3] : hi[e & 3];
      if (a.pl) x = pw == 0.f ? x : fmaf((float)__builtin_bit_cast(bf16x8, prior[k])[e], pw, x);  // without weight it may be anything
      o[e] = (__bf16)x;
    }
    if (rows[k] >= 0) reinterpret_cast<bf16x8*>(a.o)[(size_t)rows[k] * (D / 8) + (lane & 15)] = o;
  }
}

// float32: S^T = K Q^T and O^T = V^T P on v_mfma_f32_32x32x2_f32.  One workgroup =
// one work item (kv head, 32 query rows, context split); its W waves take the
// 32-key tiles in turn, each by itself, and merge at the end (one wave per item left
// long rows to few SIMDs: prompts of up to 1001 tokens 268 us, four waves 153, two 145).  A float32
// product carries 1/16 of a bfloat16 one's rate, so that the matrix cores bound it: they
// are busy 82% of a workgroup's tiles, and half of a launch of three such prompts,
// whose starts, merges and last workgroups they wait for.  K and V go from global
// memory into the operand registers; the query sits in LDS.
//   K: lane (m = lane % 32, h = lane / 32) loads dims 8 j + 4 h .. + 3 of key m.
//   P: register i of S^T holds key 8 (i / 4) + 4 h + i % 4 of query lane % 32.
//   V: lane (m, h) loads dims 4 m .. 4 m + 3 of register i's key of its half; row
//      m of accumulator b is dim 4 m + b.
// A dot product is the sum of eight 16-dim chains: its rounding error is that of
// a pairwise sum.
constexpr int EX_KEYS32 = 32;

template <int PAGED, int W>
__global__ __launch_bounds__(W * 64, 2) void k_exact_f32(ExactArgs a) {
  __shared__ __attribute__((aligned(16))) float s_part[W][66][64];  // the merge; before it the query
  f32x4 (*s_q)[64] = reinterpret_cast<f32x4 (*)[64]>(&s_part[0][0][0]);
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int kvh = blockIdx.x % a.Hkv, rest = blockIdx.x / a.Hkv;
  const int split = rest % a.splits, blk = a.blocks - 1 - rest / a.splits;
  Item it;
  if (!PAGED && a.n <= 64 ? !find_dearest<EX_ROWS_F32>(a, a.blocks - 1 - blk, it) : !find_item<EX_ROWS_F32>(a, blk, it))
    return;  // uniform in the workgroup
  int per;
  const int tiles = (it.kend + EX_KEYS32 - 1) / EX_KEYS32;
  const int nsp = ex_splits(a.splits, tiles, per);
  if (split >= nsp) return;
  const int t0 = split * per + wave, t1 = min(tiles, split * per + per);
  const int m = lane & 31, half = lane >> 5;
  const int r = it.row0 + m;
  const bool rvalid = r < it.rows;
  const int tok = rvalid ? r / a.grp : 0;
  const int head = kvh * a.grp + (rvalid ? r - tok * a.grp : 0);
  const size_t orow = (size_t)(it.s0 + tok) * a.Hq + head;
  const int klim = rvalid ? it.off + tok : -1;
  const int wfull = it.off + it.row0 / a.grp + 1;
  {
    const f32x4* qr = reinterpret_cast<const f32x4*>((const uint8_t*)a.q + (size_t)(it.s0 + tok) * a.qs) + head * (D / 4);
#pragma unroll
    for (int j = 0; j < 16 / W; ++j) s_q[16 / W * wave + j][lane] = qr[2 * (16 / W * wave + j) + half];
  }
  __syncthreads();
  const uint8_t* kb = (const uint8_t*)a.k + (PAGED ? 0 : (size_t)it.s0 * a.ks + kvh * (D * 4));
  const uint8_t* vb = (const uint8_t*)a.v + (PAGED ? 0 : (size_t)it.s0 * a.vs + kvh * (D * 4));
  auto key_of = [&](int t) { return min(t * EX_KEYS32 + m, it.kend - 1); };  // keys past the last repeat it
  auto id_of = [&](int t) { return PAGED ? a.table[(size_t)it.seq * a.stride + (key_of(t) >> a.shift)] : 0; };
  // K and V rows of this lane's key of tile t, which is on page id
  auto resolve = [&](int t, int id, const float*& kp, const float*& vp, bool& bad) {
    const int key = key_of(t);
    bad = false;
    if constexpr (PAGED) {
      bad = (unsigned)id >= (unsigned)a.num_pages;
      const size_t page = bad ? 0 : id;
      const size_t e = ((((page * a.Hkv + kvh) << a.shift) + (key & ((1 << a.shift) - 1)))) * (size_t)D;
      kp = (const float*)kb + e;
      vp = (const float*)vb + e;
    } else {
      kp = reinterpret_cast<const float*>(kb + (size_t)key * a.ks);
      vp = reinterpret_cast<const float*>(vb + (size_t)key * a.vs);
    }
  };
  // half h of a tile: dims 64 h .. 64 h + 63 of K; registers 8 h .. 8 h + 7 of V
  auto load_k = [&](const float* kp, int h, f32x4 (&kr)[8]) {
    gbl_f32x4* p = (gbl_f32x4*)(uintptr_t)kp + half + 16 * h;
#pragma unroll
    for (int j = 0; j < 8; ++j) kr[j] = p[2 * j];
  };
  auto of_key = [&](int x, int i) {  // register i's key's value of x
    return __builtin_amdgcn_ds_bpermute(16 * half + 4 * (8 * (i >> 2) + (i & 3)), x);
  };
  auto load_v = [&](const float* vp, int h, f32x4 (&vr)[8]) {
    const uint64_t p = reinterpret_cast<uint64_t>(vp);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t lo = of_key((int)(uint32_t)p, 8 * h + i), hi = of_key((int)(uint32_t)(p >> 32), 8 * h + i);
      vr[i] = ((gbl_f32x4*)(uintptr_t)((uint64_t)hi << 32 | lo))[m];
    }
  };
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  f32x16 oacc[4] = {zero, zero, zero, zero};
  float mrun = EX_NONE, lrun = 0.f;
  // four chains over the dims of half h
  auto dots = [&](const f32x4 (&kr)[8], int h) {
    f32x16 s = zero;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      f32x16 c = zero;
#pragma unroll
      for (int j = 2 * g; j < 2 * g + 2; ++j) {
        const f32x4 qv = s_q[8 * h + j][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(kr[j][e], qv[e], c, 0, 0, 0);
      }
      s = g ? s + c : c;
      asm("" : "+v"(s));  // summed here, not after every chain is done
    }
    return s;
  };
  auto weigh = [&](const f32x4 (&vr)[8], const f32x16& p, int h, f32x16 (&o)[4]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int b = 0; b < 4; ++b) o[b] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[i][b], p[8 * h + i], o[b], 0, 0, 0);
  };
  f32x4 k0[8], k1[8], v0[8], v1[8];
  const float *kp = nullptr, *vp = nullptr;
  bool bad = false;
  int id = 0;
  if (t0 < t1) {
    resolve(t0, id_of(t0), kp, vp, bad);
    id = id_of(t0 + W);
    load_k(kp, 0, k0);
    load_k(kp, 1, k1);
  }
  for (int t = t0; t < t1; t += W) {
    load_v(vp, 0, v0);
    __builtin_amdgcn_sched_barrier(0);
    f32x16 s = dots(k0, 0);
    __builtin_amdgcn_sched_barrier(0);
    load_v(vp, 1, v1);
    __builtin_amdgcn_sched_barrier(0);
    s = s + dots(k1, 1);
    const unsigned badm = PAGED ? (unsigned)__ballot(bad) >> (4 * half) : 0u;  // lanes 0 .. 31: the tile's keys
    const bool masked = (t + 1) * EX_KEYS32 > wfull || (PAGED && __ballot(bad) != 0);  // uniform
    const int rel = klim - t * EX_KEYS32 - 4 * half;
    if (masked) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = 8 * (i >> 2) + (i & 3);
        s[i] = c > rel || ((badm >> c) & 1) ? -INFINITY : s[i];
      }
    }
    // the next tile's keys load while this tile's values are used (past the
    // last key the loads repeat it)
    resolve(t + W, id, kp, vp, bad);
    id = id_of(t + 2 * W);
    load_k(kp, 0, k0);
    float tmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) tmax = fmaxf(tmax, s[i]);
    tmax = fmaxf(tmax, xor32(tmax)) * EX_SCALE;
    const float mnew = fmaxf(mrun, tmax);
    if (__ballot(!(mnew <= mrun))) {  // uniform
      const float alpha = __builtin_amdgcn_exp2f(mrun - mnew);
      lrun *= alpha;
#pragma unroll
      for (int b = 0; b < 4; ++b) oacc[b] *= alpha;
      mrun = mnew;
    }
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = __builtin_amdgcn_exp2f(fmaf(s[i], EX_SCALE, -mrun));
      part[i & 3] += s[i];
    }
    lrun += (part[0] + part[1]) + (part[2] + part[3]);
    if (masked) {
      uint32_t odd = 0;  // bit 31
#pragma unroll
      for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          odd |= ((__float_as_uint(v0[i][b]) & 0x7F800000u) + 0x00800000u) | ((__float_as_uint(v1[i][b]) & 0x7F800000u) + 0x00800000u);
      if (__ballot((int)odd < 0)) {  // uniform: what is odd goes into the sums at once and out of the values
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          f32x16 hits = zero;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = (i < 8 ? v0 : v1)[i & 7][b];
            hits = __builtin_amdgcn_mfma_f32_32x32x2f32(x == INFINITY || x != x ? 1.f : 0.f, s[i], hits, 0, 0, 0);
          }
          add_odd<1>(oacc[b], hits);
          __builtin_amdgcn_sched_barrier(0);
          hits = zero;
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const float x = (i < 8 ? v0 : v1)[i & 7][b];
            hits = __builtin_amdgcn_mfma_f32_32x32x2f32(x == -INFINITY || x != x ? 1.f : 0.f, s[i], hits, 0, 0, 0);
          }
          add_odd<-1>(oacc[b], hits);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            v0[i][b] = fabsf(v0[i][b]) < INFINITY ? v0[i][b] : 0.f;
            v1[i][b] = fabsf(v1[i][b]) < INFINITY ? v1[i][b] : 0.f;
          }
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    weigh(v0, s, 0, oacc);
    __builtin_amdgcn_sched_barrier(0);
    load_k(kp, 1, k1);
    __builtin_amdgcn_sched_barrier(0);
    weigh(v1, s, 1, oacc);
  }
  lrun += xor32(lrun);
  // merge of the waves, each relative to its own reference; wave w then holds
  // registers NR w .. NR w + NR - 1.  Register i of oacc[0..3]: dims 4 mm .. 4 mm + 3 with
  // mm = 8 (i / 4) + 4 half + i % 4
  __syncthreads();  // every wave is done with the query
#pragma unroll
  for (int b = 0; b < 4; ++b)
#pragma unroll
    for (int i = 0; i < 16; ++i) s_part[wave][b * 16 + i][lane] = oacc[b][i];
  s_part[wave][64][lane] = mrun;
  s_part[wave][65][lane] = lrun;
  __syncthreads();
  float M = EX_NONE, L = 0.f, wgt[W];
#pragma unroll
  for (int w = 0; w < W; ++w) M = fmaxf(M, s_part[w][64][lane]);
#pragma unroll
  for (int w = 0; w < W; ++w) {
    wgt[w] = __builtin_amdgcn_exp2f(s_part[w][64][lane] - M);
    L += wgt[w] * s_part[w][65][lane];
  }
  const float inv = nsp > 1 ? 1.0f : L > 0.f || L != L ? 1.0f / L : 0.f;
  const size_t pr = (((size_t)kvh * a.blocks + blk) * a.splits + split) * EX_ROWS_F32 + m;
  constexpr int NR = 16 / W;  // registers of O that a wave merges
  auto dim = [&](int e) { const int i = NR * wave + e; return 4 * (8 * (i >> 2) + 4 * half + (i & 3)); };
  auto merged = [&](int e) {
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
      for (int b = 0; b < 4; ++b) o[b] += wgt[w] * s_part[w][b * 16 + NR * wave + e][lane];
    return o * inv;
  };
  float lse = 0.f;
  if (rvalid) {
    if (nsp > 1) {
#pragma unroll
      for (int e = 0; e < NR; ++e) *reinterpret_cast<f32x4*>(a.part_o + pr * D + dim(e)) = merged(e);
    } else {
      lse = write_row<1, NR>(a, orow, L == 0.f ? -INFINITY : M + log2f(L), merged, dim);
    }
  }
  __syncthreads();  // every wave has read the prior's lse, which may be lse itself
  if (wave != 0 || half != 0 || !rvalid) return;
  if (nsp > 1) {
    a.part_ml[pr * 2] = M;
    a.part_ml[pr * 2 + 1] = L;
  } else if (a.lse) {
    a.lse[orow] = lse;
  }
}

// A row's partial results joined: O = sum_s w_s O_s, l likewise, with
// w_s = 2^(m_s - max m); four dims to a thread.
struct Sum {
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  float M = EX_NONE, l = 0.f;
  __device__ __forceinline__ void add(float m, float x, f32x4 v) {
    const float top = fmaxf(M, m), p = __builtin_amdgcn_exp2f(M - top), q = __builtin_amdgcn_exp2f(m - top);
    l = l * p + x * q;
    o = o * p + v * q;
    M = top;
  }
  // partials k0, k0 + step, .. below count, eight at a time in flight; row(k): partial k's
  template <typename F>
  __device__ __forceinline__ void gather(const float* po, const float* ml, int k0, int step, int count, int d4, F row) {
    for (; k0 < count; k0 += 8 * step) {
      float m[8], x[8];
      f32x4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const size_t pr = row(min(k0 + u * step, count - 1));
        m[u] = ml[pr * 2];
        x[u] = ml[pr * 2 + 1];
        v[u] = reinterpret_cast<const f32x4*>(po + pr * D)[d4];
      }
      float top = M;
#pragma unroll
      for (int u = 0; u < 8; ++u) top = fmaxf(top, m[u]);
      const float back = __builtin_amdgcn_exp2f(M - top);
      o *= back;
      l *= back;
      M = top;
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        if (k0 + u * step < count) {
          const float wgt = __builtin_amdgcn_exp2f(m[u] - M);
          l += wgt * x[u];
          o += wgt * v[u];
        }
      }
    }
  }
  template <int FP32>
  __device__ __forceinline__ void store(const ExactArgs& a, size_t orow, int d4) const {
    const f32x4 x = o * (l > 0.f || l != l ? 1.0f / l : 0.f);
    const float lse = write_row<FP32, 1>(a, orow, l == 0.f ? -INFINITY : M + log2f(l), [&](int) { return x; },
                                         [&](int) { return 4 * d4; });
    if (d4 == 0 && a.lse) a.lse[orow] = lse;
  }
};

// Joins the splits of a row block.  Workgroup = EJ_ROWS rows of one (kv head, row
// block), 32 threads per row.  A latency chain: block, references, partials (3 x 20
// rows over 2500 tokens in float32 5.3 us).
constexpr int EJ_ROWS = 16;
template <int FP32, int R>
__global__ __launch_bounds__(EJ_ROWS * 32) void k_exact_join(ExactArgs a) {
  const int part = blockIdx.x % (R / EJ_ROWS), rest = blockIdx.x / (R / EJ_ROWS);
  const int kvh = rest % a.Hkv, blk = rest / a.Hkv;
  Item it;
  if (!find_item<R>(a, blk, it)) return;
  int per;
  const int tiles = (it.kend + (FP32 ? EX_KEYS32 : EX_KEYS) - 1) / (FP32 ? EX_KEYS32 : EX_KEYS);
  const int nsp = ex_splits(a.splits, tiles, per);
  if (nsp == 1) return;  // written by the attention itself
  const size_t base = ((size_t)kvh * a.blocks + blk) * a.splits;
  const int lr = part * EJ_ROWS + (threadIdx.x >> 5), r = it.row0 + lr, d4 = threadIdx.x & 31;
  if (r >= it.rows) return;
  Sum s;
  s.gather(a.part_o, a.part_ml, 0, 1, nsp, d4, [&](int k) { return (base + k) * R + lr; });
  const int tok = r / a.grp;
  s.store<FP32>(a, (size_t)(it.s0 + tok) * a.Hq + kvh * a.grp + (r - tok * a.grp), d4);
}

// bf16, requests of at most 32 rows per kv head (single tokens of an answer).
// What they cost is reading the cache once, so the keys are shared out evenly:
// the 32-key tiles of all (request, kv head) items, laid end to end, are cut into
// equal runs, one per wave, whatever the requests' lengths.  A wave goes through
// its run item by item and needs no other wave: K rows straight into the A
// operand, V rows straight into the wave's LDS for the transposed reads, the next
// tile's loads in flight.  An item within one run is written out; of one
// that runs on, each wave leaves a partial (at most two per wave: the item it ends
// in, slot 1, and the one it continues, slot 0), and the wave that the item begins
// in notes it for k_exact_few_join.  Every wave sums the tiles of all requests, n / 64
// steps, which is made for thousands of them.  64 requests over 1.07 GB of pages: 198 us, 5.4
// TB/s; one over 1500 tokens 9.6 us, the chain of its two or three tiles.
constexpr int FW_W = 4;              // waves per workgroup
constexpr int FW_VB = 32 * 64 + 64;  // bytes of one 32-dim block of a V tile (64 of padding: bank spread)

// What k_exact_few takes of request i.
struct Few {
  int s0, add, rows, kv, tiles;  // tiles: one even if its rows see nothing, 0 if it is not that kernel's
};
__device__ __forceinline__ Few few_of(const ExactArgs& a, int i) {
  Few r;
  const int c0 = min(max(a.cu[i], 0), a.total), c1 = min(max(a.cu[i + 1], 0), a.total);
  r.s0 = c0;
  r.add = max(c1 - c0, 0);
  r.rows = (int)min((long long)min(r.add, a.max_add) * a.grp, (long long)EX_FEW + 1);
  r.kv = min(max(a.kv_len[i], 0), a.stride << a.shift);
  r.tiles = r.rows < 1 || r.rows > EX_FEW ? 0 : max(1, (r.kv + 31) / 32);
  return r;
}
__device__ __forceinline__ long long lane_ll(long long x, int l) {
  const unsigned lo = __builtin_amdgcn_readlane((int)(unsigned)x, l), hi = __builtin_amdgcn_readlane((int)(x >> 32), l);
  return (long long)((unsigned long long)hi << 32 | lo);
}
// inclusive running sum over the wave
__device__ __forceinline__ long long wave_sum(long long x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long long y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  return x;
}
__global__ __launch_bounds__(FW_W * 64, 2) void k_exact_few(ExactArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t s_mem[FW_W][2][4 * FW_VB];  // the V tile in use and the next
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int w = blockIdx.x * FW_W + wave;
  const int m = lane & 31, half = lane >> 5;
  int32_t* meta = a.few_meta + w * 4;
  // total tiles and this wave's run: lane l sums the requests of the l-th of 64 blocks
  const int per64 = (a.n + 63) / 64;
  long long mine = 0;
  Few q{};
  for (int j = 0; j < per64; ++j) {
    const int i = lane * per64 + j;
    if (i < a.n) q = few_of(a, i);
    mine += i < a.n ? q.tiles : 0;
  }
  long long upto = wave_sum(mine);
  const long long N = lane_ll(upto, 63) * a.Hkv;
  const long long waves = (long long)gridDim.x * FW_W;
  // tiles of a run: at least 2, and as long as 16 are not reached as many as leave
  // two waves to a compute unit, since more partials cost more than more loads in
  // flight give (30 000 tokens, 4 kv heads, 2048 waves 32 us, 470 24; 8 x 8000, 7 rows
  // 38 and 31, 32 rows 64 and 35; but 64 x 8000, 2048 waves 203, 512 231)
  const long long per = max(max((N + waves - 1) / waves, min(16ll, (N + 511) / 512)), 2ll);
  const long long x1 = min(N, (w + 1) * per);
  long long x = w * per;
  if (lane == 0) meta[0] = 0;
  if (x >= N) return;  // uniform, and nothing below synchronises waves
  int i0 = 0;            // first request of the 64 in the lanes
  long long before = 0;  // tiles before it
  if (per64 > 1) {
    const int l = __builtin_amdgcn_readfirstlane(__popcll(__ballot((upto - mine) * a.Hkv <= x)) - 1);
    i0 = l * per64;
    before = lane_ll(upto - mine, l);
  }
  const uint8_t* kb = (const uint8_t*)a.k;
  const uint8_t* vb = (const uint8_t*)a.v;
  const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  const int grp16 = lane >> 4, s16 = lane & 15;
  const uint8_t* vl0 = s_mem[wave][0] + (4 * half + (s16 >> 2)) * 64 + (grp16 & 1) * 32 + (s16 & 3) * 8;

  // tiles [ta, tb) of request i's kv head kvh; whole: that is all of them
  auto item = [&](int i, int s0, int add, int rows, int kv, int kvh, int ta, int tb, bool whole, int slot) {
    const int off = kv - add;
    const bool rvalid = m < rows;
    const int tok = rvalid ? m / a.grp : 0;
    const int head = kvh * a.grp + (rvalid ? m - tok * a.grp : 0);
    const size_t orow = (size_t)(s0 + tok) * a.Hq + head;
    const int klim = rvalid ? off + tok : -1;
    const int ntok = (rows - 1) / a.grp + 1;
    const int wfull = off + 1;                          // keys that every row sees
    const int kend = min(max(off + ntok, 0), kv);       // keys that some row sees
    const int tend = min(tb, (kend + 31) / 32);
    const int32_t* row = a.table + (size_t)i * a.stride;
    bf16x8 bq[8];
    {
      const u16x8* qr = reinterpret_cast<const u16x8*>((const uint8_t*)a.q + (size_t)(s0 + tok) * a.qs + head * (D * 2));
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) bq[kk] = __builtin_bit_cast(bf16x8, qr[2 * kk + half]);
    }
    f32x16 oacc[4] = {zero, zero, zero, zero};
    float mref = EX_NONE, lrun = 0.f;
    auto id_of = [&](int t) { return row[min(t * 32 + m, kend - 1) >> a.shift]; };
    // row index in the pages of this lane's key of tile t on page id (a tensor of
    // 2^31 rows would not fit the GPU); bad: no page, page 0 is read instead
    auto row_of = [&](int t, int id, bool& bad) {
      const int key = min(t * 32 + m, kend - 1);
      bad = (unsigned)id >= (unsigned)a.num_pages;
      return (int)((((unsigned)(bad ? 0 : id) * a.Hkv + kvh) << a.shift) + (key & ((1 << a.shift) - 1)));
    };
    auto load_k = [&](int rw, u16x8 (&kr)[8]) {
      const u16x8* p = reinterpret_cast<const u16x8*>(kb) + (size_t)(unsigned)rw * 16;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) kr[kk] = p[2 * kk + half];
    };
    // V rows of the tile straight into the wave's LDS: instruction (b, g) takes 32-dim
    // block b of rows 16 g .. + 15
    auto load_v = [&](int rw, int buf) {
#pragma unroll
      for (int g = 0; g < 2; ++g) {
        const unsigned r = __builtin_amdgcn_ds_bpermute(64 * g + (lane & ~3), rw);
        const uint8_t* p = vb + (size_t)r * (D * 2) + (lane & 3) * 16;
#pragma unroll
        for (int b = 0; b < 4; ++b) lds_dma16(p + b * 64, s_mem[wave][buf] + b * FW_VB + g * 1024);
      }
    };
    if (ta < tend) {
      u16x8 kr[8];
      bool bad;
      int rw = row_of(ta, id_of(ta), bad);
      int id = id_of(min(ta + 1, tend - 1));
      load_v(rw, ta & 1);
      __builtin_amdgcn_sched_barrier(0);
      load_k(rw, kr);
      for (int t = ta; t < tend; ++t) {
        const int tn = min(t + 1, tend - 1);  // past the last tile the loads repeat it
        const unsigned badm = (unsigned)__ballot(bad);
        rw = row_of(tn, id, bad);
        const bool masked = (t + 1) * 32 > wfull || badm != 0;  // uniform
        f32x16 s = zero;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kr[kk]), bq[kk], s, 0, 0, 0);
        // Loads return in the order of their issue: V's are issued before K's of the
        // same tile, so with K in the registers of the products V is in LDS.
        asm volatile("" : "+v"(s) : : "memory");
        __builtin_amdgcn_sched_barrier(0);
        if (t + 1 < tend) {  // uniform
          id = id_of(min(tn + 1, tend - 1));
          load_v(rw, (t + 1) & 1);  // read last by the products of tile t - 1
          __builtin_amdgcn_sched_barrier(0);
          load_k(rw, kr);
        }
        __builtin_amdgcn_sched_barrier(0);
        const uint8_t* vl = vl0 + (t & 1) * (4 * FW_VB);
        if (masked) {
          const int rel = klim - t * 32 - 4 * half;
#pragma unroll
          for (int j = 0; j < 16; ++j) s[j] = 8 * (j >> 2) + (j & 3) > rel ? -INFINITY : s[j];
          if (badm) {
            const unsigned bm = badm >> (4 * half);
#pragma unroll
            for (int j = 0; j < 16; ++j) s[j] = (bm >> (8 * (j >> 2) + (j & 3))) & 1 ? -INFINITY : s[j];
          }
        }
        float tmax = -INFINITY;
#pragma unroll
        for (int j = 0; j < 16; ++j) tmax = fmaxf(tmax, s[j]);
        tmax = fmaxf(tmax, xor32(tmax)) * EX_SCALE;
        const bool grow = tmax > mref + 8.0f;
        if (__ballot(grow)) {  // uniform
          const float mnew = grow ? tmax : mref;
          const float alpha = __builtin_amdgcn_exp2f(mref - mnew);
          lrun *= alpha;
#pragma unroll
          for (int b = 0; b < 4; ++b) oacc[b] *= alpha;
          mref = mnew;
        }
        bf16x8 pb[2];
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float p = __builtin_amdgcn_exp2f(fmaf(s[j], EX_SCALE, -mref));
          part[j & 1] += p;
          pb[j >> 3][j & 7] = (__bf16)p;
        }
        lrun += part[0] + part[1];
        auto read_v = [&](int b, int st, int z = 0) {
          const v4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vl + z + b * FW_VB + st * 1024));
          const v4i16 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16*)(vl + z + b * FW_VB + st * 1024 + 512));
          return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        };
        if (masked) {
          uint32_t odd = 0;
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
              const v8i16 v = read_v(b, st);
              odd |= odd_flags(v);
              oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<0>(v), pb[st], oacc[b], 0, 0, 0);
            }
          if (__ballot((odd & ODD) != 0)) {  // uniform
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              f32x16 hits = zero;
              int z = anew();
#pragma unroll
              for (int st = 0; st < 2; ++st)
                hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<1>(read_v(b, st, z)), pb[st], hits, 0, 0, 0);
              add_odd<1>(oacc[b], hits);
              __builtin_amdgcn_sched_barrier(0);
              hits = zero;
              z = anew();
#pragma unroll
              for (int st = 0; st < 2; ++st)
                hits = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd_operand<-1>(read_v(b, st, z)), pb[st], hits, 0, 0, 0);
              add_odd<-1>(oacc[b], hits);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        } else {
#pragma unroll
          for (int b = 0; b < 4; ++b)
#pragma unroll
            for (int st = 0; st < 2; ++st)
              oacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, read_v(b, st)), pb[st], oacc[b], 0, 0, 0);
        }
      }
    }
    lrun += xor32(lrun);
    if (!rvalid) return;
    if (whole) {
      const float inv = lrun > 0.f || lrun != lrun ? 1.0f / lrun : 0.f;
      const float lse = write_row<0, 16>(
          a, orow, lrun == 0.f ? -INFINITY : mref + log2f(lrun),
          [&](int i) {
            const int b = i >> 2, e = 4 * (i & 3);
            return (f32x4){oacc[b][e], oacc[b][e + 1], oacc[b][e + 2], oacc[b][e + 3]} * inv;
          },
          [&](int i) { return (i >> 2) * 32 + (i & 3) * 8 + half * 4; });
      if (half == 0 && a.lse) a.lse[orow] = lse;
      return;
    }
    const size_t prow = ((size_t)w * 2 + slot) * a.few_rows + m;
#pragma unroll
    for (int b = 0; b < 4; ++b)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        *reinterpret_cast<f32x4*>(a.few_o + prow * D + b * 32 + e * 8 + half * 4) =
            (f32x4){oacc[b][4 * e], oacc[b][4 * e + 1], oacc[b][4 * e + 2], oacc[b][4 * e + 3]};
    if (half == 0) {
      a.few_ml[prow * 2] = mref;
      a.few_ml[prow * 2 + 1] = lrun;
    }
  };

  while (x < x1 && i0 < a.n) {
    if (per64 > 1) {  // else the lanes have them
      q = Few{};
      if (i0 + lane < a.n) q = few_of(a, i0 + lane);
    }
    const long long incl = wave_sum(q.tiles), excl = incl - q.tiles;
    const long long all = before + lane_ll(incl, 63);
    while (x < x1 && x < all * a.Hkv) {
      // the request that x is in: the last one that begins at or before it
      const int r = __builtin_amdgcn_readfirstlane(__popcll(__ballot((before + excl) * a.Hkv <= x)) - 1);
      const int T = __builtin_amdgcn_readlane(q.tiles, r);
      const long long first = (before + lane_ll(excl, r)) * a.Hkv;
      const int kvh = __builtin_amdgcn_readfirstlane((int)((x - first) / T));
      const int ta = __builtin_amdgcn_readfirstlane((int)(x - first - (long long)kvh * T));
      const int tb = __builtin_amdgcn_readfirstlane((int)min((long long)T, ta + (x1 - x)));
      item(i0 + r, __builtin_amdgcn_readlane(q.s0, r), __builtin_amdgcn_readlane(q.add, r),
           __builtin_amdgcn_readlane(q.rows, r), __builtin_amdgcn_readlane(q.kv, r), kvh, ta, tb, ta == 0 && tb == T,
           ta == 0);
      if (ta == 0 && tb < T && lane == 0) {
        // its rows, kv head, the wave that it ends in, its first row of q
        *reinterpret_cast<int4*>(meta) = make_int4(__builtin_amdgcn_readlane(q.rows, r), kvh,
                                                   (int)((first + (long long)(kvh + 1) * T - 1) / per),
                                                   __builtin_amdgcn_readlane(q.s0, r));
      }
      x += tb - ta;
    }
    before = all;
    i0 += 64;
  }
}

// Joins the partials of the items that begin in waves 8 b .. 8 b + 7 of
// k_exact_few and run on: slot 1 of that wave, slot 0 of the next ones.  Of an
// item with few partials each wave takes a row by itself, 32 threads (four dims
// each) for every other partial; of one with many the workgroup takes a row at a
// time (FJ_MANY partials and more).  blockIdx.y deals the rows out.  64 requests, 2048
// waves' partials: 10 us; one request 4.8; a workgroup per row for all items, one
// after the other, 21 for the former.
constexpr int FJ_W = 8;
constexpr int FJ_Y = 4;
constexpr int FJ_MANY = 48;
__global__ __launch_bounds__(FJ_W * 64) void k_exact_few_join(ExactArgs a, int waves) {
  __shared__ f32x4 s_o[FJ_W][32];
  __shared__ float s_l[FJ_W][2];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w0 = blockIdx.x * FJ_W, y = blockIdx.y, ny = gridDim.y;
  const int g = lane >> 5, d4 = lane & 31;
  int4 meta[FJ_W];
#pragma unroll
  for (int e = 0; e < FJ_W; ++e)
    meta[e] = w0 + e < waves ? reinterpret_cast<const int4*>(a.few_meta)[w0 + e] : make_int4(0, 0, 0, 0);
  int at = 0;  // rows given out to the waves so far
#pragma unroll
  for (int e = 0; e < FJ_W; ++e) {
    const int rows = meta[e].x, kvh = meta[e].y, w = w0 + e, count = meta[e].z - w + 1, s0 = meta[e].w;
    const bool many = count > FJ_MANY;
    for (int r = y; r < rows; r += ny) {  // uniform
      if (!many && (at++ & (FJ_W - 1)) != wave) continue;
      Sum s;
      s.gather(a.few_o, a.few_ml, many ? wave * 2 + g : g, many ? 2 * FJ_W : 2, count, d4,
               [&](int k) { return ((size_t)(w + k) * 2 + (k == 0)) * a.few_rows + r; });
      {
        f32x4 v;
#pragma unroll
        for (int c = 0; c < 4; ++c) v[c] = xor32(s.o[c]);
        s.add(xor32(s.M), xor32(s.l), v);
      }
      if (many) {
        __syncthreads();  // s_o and s_l are free
        if (g == 0) s_o[wave][d4] = s.o;
        if (lane == 0) {
          s_l[wave][0] = s.M;
          s_l[wave][1] = s.l;
        }
        __syncthreads();
        if (wave != 0) continue;
#pragma unroll
        for (int k = 1; k < FJ_W; ++k) s.add(s_l[k][0], s_l[k][1], s_o[k][d4]);
      }
      const int tok = r / a.grp;
      if (g == 0) s.store<0>(a, (size_t)(s0 + tok) * a.Hq + kvh * a.grp + (r - tok * a.grp), d4);
    }
  }
}

}  // namespace

hipError_t launch_exact(const ExactArgs& a, bool fp32, bool paged, hipStream_t st) {
  if (a.few) {
    const int wgs = (a.few + FW_W - 1) / FW_W;
    hipLaunchKernelGGL(k_exact_few, dim3(wgs), dim3(FW_W * 64), 0, st, a);
    // a workgroup per row and 8 waves, up to 2048 of them, at least four to 8 waves
    const int parts = (wgs * FW_W + FJ_W - 1) / FJ_W;
    hipLaunchKernelGGL(k_exact_few_join, dim3(parts, std::min(a.few_rows, std::max(FJ_Y, 2048 / parts))), dim3(FJ_W * 64), 0,
                       st, a, wgs * FW_W);
  }
  const unsigned items = (unsigned)a.Hkv * a.blocks * a.splits;
  if (items == 0) return hipGetLastError();
  if (fp32) {
    if (paged) hipLaunchKernelGGL((k_exact_f32<1, 4>), dim3(items), dim3(4 * 64), 0, st, a);
    else if (a.waves == 4) hipLaunchKernelGGL((k_exact_f32<0, 4>), dim3(items), dim3(4 * 64), 0, st, a);
    else hipLaunchKernelGGL((k_exact_f32<0, 2>), dim3(items), dim3(2 * 64), 0, st, a);
  } else {
    const bool half = a.rows == EX_ROWS / 2;
    if (paged && half) hipLaunchKernelGGL((k_exact_bf16<1, 2>), dim3(items), dim3(512), 0, st, a);
    else if (paged) hipLaunchKernelGGL((k_exact_bf16<1, 1>), dim3(items), dim3(512), 0, st, a);
    else if (half) hipLaunchKernelGGL((k_exact_bf16<0, 2>), dim3(items), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_exact_bf16<0, 1>), dim3(items), dim3(512), 0, st, a);
  }
  if (a.splits > 1) {
    const dim3 wgs(a.Hkv * a.blocks * (a.rows / EJ_ROWS)), threads(EJ_ROWS * 32);
    if (fp32) hipLaunchKernelGGL((k_exact_join<1, EX_ROWS_F32>), wgs, threads, 0, st, a);
    else if (a.rows == EX_ROWS) hipLaunchKernelGGL((k_exact_join<0, EX_ROWS>), wgs, threads, 0, st, a);
    else hipLaunchKernelGGL((k_exact_join<0, EX_ROWS / 2>), wgs, threads, 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace pkv
