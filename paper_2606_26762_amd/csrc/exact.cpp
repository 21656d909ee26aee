// Host side of the handle-free calls: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <initializer_list>

#include "exact.h"
#include "pkv_internal.h"

using namespace pkv;

namespace {

protokv_status fail(protokv_status s, const char* who, const char* why) {
  call_error() = std::string(who) + ": " + why;
  return s;
}

protokv_status device(hipError_t e, const char* who) {
  if (e == hipSuccess) return PROTOKV_OK;
  return fail(PROTOKV_E_DEVICE, who, hipGetErrorString(e));
}

bool off4(const void* p) { return (uintptr_t)p % 4 != 0; }
bool off16(const void* p) { return (uintptr_t)p % 16 != 0; }
bool pow2(int x) { return x > 0 && (x & (x - 1)) == 0; }
int log2i(int x) { return 31 - __builtin_clz((unsigned)x); }

// Head counts and type of a call's rows.
struct Heads {
  int q, kv, dim, dtype;
  int es() const { return dtype == PROTOKV_KV_FP32 ? 4 : 2; }
};

protokv_status check_heads(const Heads& h, const char* who) {
  if (h.dtype != PROTOKV_KV_BF16 && h.dtype != PROTOKV_KV_FP32) return fail(PROTOKV_E_INVALID, who, "kv_dtype unknown");
  if (h.kv < 1 || h.q < h.kv || h.q % h.kv)
    return fail(PROTOKV_E_INVALID, who, "num_q_heads must be a positive multiple of num_kv_heads");
  if (h.dim != D) return fail(PROTOKV_E_UNSUPPORTED, who, "head_dim must be 128");
  if (h.q / h.kv > 256) return fail(PROTOKV_E_UNSUPPORTED, who, "num_q_heads / num_kv_heads above 256");
  if (h.q > 65536) return fail(PROTOKV_E_UNSUPPORTED, who, "num_q_heads above 65536");
  return PROTOKV_OK;
}

// Rows of `heads` heads at p, `stride` elements from row to row.
protokv_status check_rows(const void* p, int64_t stride, int heads, const Heads& h, const char* who, const char* name) {
  const std::string n(name);
  if (!p) return fail(PROTOKV_E_INVALID, who, (n + " is NULL").c_str());
  if (off16(p)) return fail(PROTOKV_E_INVALID, who, (n + " must be aligned to 16 bytes").c_str());
  if (stride < (int64_t)heads * D || stride > (1ll << 32))
    return fail(PROTOKV_E_INVALID, who, (n + "_stride must hold the row's heads (and be at most 2^32)").c_str());
  if (stride * h.es() % 16) return fail(PROTOKV_E_INVALID, who, (n + "_stride must be a multiple of 16 bytes").c_str());
  return PROTOKV_OK;
}

protokv_status check_page_rows(const protokv_pages& p, const char* who) {
  if (!p.k || !p.v || off16(p.k) || off16(p.v))
    return fail(PROTOKV_E_INVALID, who, "pages: k and v must be non-NULL and aligned to 16 bytes");
  return PROTOKV_OK;
}

protokv_status check_page_sizes(int num_pages, int page_size, const char* who) {
  if (num_pages < 1) return fail(PROTOKV_E_INVALID, who, "num_pages must be >= 1");
  if (!pow2(page_size) || page_size > 1024)
    return fail(PROTOKV_E_UNSUPPORTED, who, "page_size must be a power of two in [1, 1024]");
  if ((int64_t)num_pages * page_size >= (1ll << 31))
    return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages * page_size must be below 2^31");
  return PROTOKV_OK;
}

protokv_status check_pages4(const protokv_pages4& p, int heads, const char* who) {
  // (a page's row is found in 32 bits)
  if ((int64_t)p.num_pages * p.page_size * heads >= (1ll << 32))
    return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages * page_size * num_kv_heads must be below 2^32");
  if (!p.k || !p.v || off16(p.k) || off16(p.v))
    return fail(PROTOKV_E_INVALID, who, "pages: k and v must be non-NULL and aligned to 16 bytes");
  if (!p.k_scale || !p.v_scale || off4(p.k_scale) || off4(p.v_scale))
    return fail(PROTOKV_E_INVALID, who, "pages: k_scale and v_scale must be non-NULL and aligned to 4 bytes");
  return PROTOKV_OK;
}

// Requests' block tables, as protokv_page_plan takes them.
protokv_status check_table(int requests, int num_pages, int page_size, int stride, const char* who) {
  if (requests < 1) return fail(PROTOKV_E_INVALID, who, "num_requests must be >= 1");
  if (requests > MAX_REQUESTS) return fail(PROTOKV_E_UNSUPPORTED, who, "num_requests above 8192");
  protokv_status s = check_page_sizes(num_pages, page_size, who);
  if (s != PROTOKV_OK) return s;
  if (num_pages > (1 << 29)) return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages above 2^29");
  if (stride < 1 || (int64_t)stride * page_size >= (1ll << 31))
    return fail(PROTOKV_E_INVALID, who, "table_stride must be >= 1 and table_stride * page_size below 2^31");
  return PROTOKV_OK;
}

// Arrays of int32: what a call needs, and outputs that are none of its inputs nor each other.
protokv_status check_arrays(std::initializer_list<const void*> need, std::initializer_list<const void*> maybe,
                            std::initializer_list<const void*> in, std::initializer_list<const void*> out, const char* who) {
  for (const void* p : need)
    if (!p || off4(p)) return fail(PROTOKV_E_INVALID, who, "arrays must be non-NULL and aligned to 4 bytes");
  for (const void* p : maybe)
    if (off4(p)) return fail(PROTOKV_E_INVALID, who, "arrays must be aligned to 4 bytes");
  for (auto q = out.begin(); q != out.end(); ++q) {
    for (const void* p : in)
      if (p && p == *q) return fail(PROTOKV_E_INVALID, who, "an output must not be one of the inputs");
    for (auto p = out.begin(); p != q; ++p)
      if (*p && *p == *q) return fail(PROTOKV_E_INVALID, who, "two outputs are the same array");
  }
  return PROTOKV_OK;
}

// Output, prior and row counts shared by the two attentions.
protokv_status check_result(const Heads& h, int n, int total, const int32_t* cu, const void* o, const float* lse,
                            const void* po, const float* pl, const char* who) {
  if (n < 0 || total < 0) return fail(PROTOKV_E_INVALID, who, "counts must be >= 0");
  if ((int64_t)total * h.q >= (1ll << 31) || n >= (1 << 24))
    return fail(PROTOKV_E_UNSUPPORTED, who, "total * num_q_heads must be below 2^31, the number of sequences below 2^24");
  if (n == 0 || total == 0) return PROTOKV_OK;
  if (!cu || off4(cu)) return fail(PROTOKV_E_INVALID, who, "cu must be non-NULL and aligned to 4 bytes");
  if (!o || off16(o)) return fail(PROTOKV_E_INVALID, who, "o must be non-NULL and aligned to 16 bytes");
  if (off4(lse)) return fail(PROTOKV_E_INVALID, who, "lse must be aligned to 4 bytes");
  if ((po == nullptr) != (pl == nullptr)) return fail(PROTOKV_E_INVALID, who, "prior_o and prior_lse go together");
  if (off16(po) || off4(pl)) return fail(PROTOKV_E_INVALID, who, "prior_o must be aligned to 16 bytes, prior_lse to 4");
  return PROTOKV_OK;
}

// Row blocks of R rows: sequence i has the indices floor(cu[i] grp / R) + i and on,
// which leaves room for its ceil(rows / R) whatever cu is.  R and, over pages, the
// most context splits of a block are those with the least time by this count, in
// tenths of a 64-key tile's time in the form of 256 rows (about 2 us): a tile takes
// 10 (128 rows, two waves to a row's keys: 6), a workgroup 40 to start and to end (50
// with the waves' merge), a split 60 more for its partial; `slots` workgroups run at a time.  Prompts see half their keys on
// average and take at least as long as the last rows of a sequence of mean length.  The
// lengths are on the device: the host knows the mean of a prompt's, not the longest,
// and of contexts the table's width, so that unequal prompts' last rows are counted
// short, and contexts that leave most of the table empty are split for keys that are not
// there (8 x 64 tokens over 2000, 28 / 4 heads: 52 us in a table of 2064 tokens, unsplit,
// 62 in one of 32 768).  Measured, 28 / 4 heads, tables as wide as the contexts: one
// prompt of 1500 tokens 43 us by 256 rows, 34 by 128; eight of 200 17 and 25; one of
// 4000 115 and 146; 4 x 512 tokens over 16 k in 3 splits 540, unsplit 484.
int64_t plan_blocks(ExactArgs& a, bool paged) {
  const int64_t slots = 256;
  const int64_t keys = paged ? (int64_t)a.stride << a.shift : ((int64_t)a.total + a.n - 1) / std::max(a.n, 1);
  const int64_t tiles = (keys + 63) / 64;
  int64_t best = INT64_MAX;
  for (int half = 0; half <= 1; ++half) {
    const int R = EX_ROWS >> half;
    const int blocks = (int)((int64_t)a.total * a.grp / R) + a.n;
    const int64_t items = (int64_t)blocks * a.Hkv, unit = half ? 6 : 10, ends = half ? 50 : 40;
    for (int s = 1; s <= (paged ? EX_MAX_SPLITS : 1) && (s == 1 || s <= tiles / EX_MIN_TILES); ++s) {
      const int64_t rounds = (items * s + slots - 1) / slots;
      const int64_t cost = paged ? rounds * ((tiles + s - 1) / s * unit + ends + (s > 1 ? 60 : 0))
                                 : std::max(tiles * unit + ends, rounds * (tiles * unit / 2 + ends));
      if (cost < best) {
        best = cost;
        a.rows = R;
        a.blocks = blocks;
        a.splits = s;
      }
    }
  }
  return best;
}

// Row blocks of float32: 32 rows, whose waves take the 32-key tiles in turn, a tile
// 20 tenths of the unit above by itself.  Two workgroups share a compute unit, and then
// its matrix cores.  Over pages the splits with the least time by this count (3 chunks of
// 20 tokens over 2500, 6 / 2 heads: nine tiles and more to a split 31 us, four 22; 8 single
// tokens over 2000, 28 / 4 heads: 252 workgroups 31 us, 288 37).  Prompts: four waves, or
// two, which leave less of a short row idle and merge less, where the launch lasts
// several times as long as the last rows of a sequence of mean length (32 of 200 tokens, 28 / 4 heads: four waves 205
// us, two 154; 4 of 800 223 and 214; but one of 1500 188 and 215, one of 200 20 and 27).
void plan_blocks_f32(ExactArgs& a, bool paged) {
  a.rows = EX_ROWS_F32;
  a.blocks = (int)((int64_t)a.total * a.grp / EX_ROWS_F32) + a.n;
  a.splits = 1;
  a.waves = 4;
  const int64_t items = (int64_t)a.blocks * a.Hkv;
  const int64_t keys = paged ? (int64_t)a.stride << a.shift : ((int64_t)a.total + a.n - 1) / std::max(a.n, 1);
  const int64_t tiles = (keys + 31) / 32;
  if (!paged) {
    if (items > 512 && items >= 50 * tiles) a.waves = 2;
    return;
  }
  int64_t best = INT64_MAX;
  for (int s = 1; s <= EX_MAX_SPLITS_F32 && (s == 1 || s <= tiles / EX_MIN_TILES); ++s) {
    const int64_t turns = ((tiles + s - 1) / s + 3) / 4;  // tiles of a wave
    const int64_t cost = (items * s + 255) / 256 * turns * 20 + (items * s + 511) / 512 * (s > 1 ? 80 : 40) + (s > 1 ? 25 + s / 2 : 0);
    if (cost < best) {
      best = cost;
      a.splits = s;
    }
  }
}

// A launch has fewer than 2^32 threads: of row blocks by 512, of their join 512 to 16 rows.
protokv_status check_grid(const ExactArgs& a, const char* who) {
  const int64_t wgs = (int64_t)a.blocks * a.Hkv * std::max(a.splits, a.splits > 1 ? a.rows / 16 : 1);
  if (wgs < (1ll << 32) / 512) return PROTOKV_OK;
  return fail(PROTOKV_E_UNSUPPORTED, who, "too many rows or sequences for one launch");
}

// The workspace's parts, from `base` on (may be null); its size.
size_t lay_out(ExactArgs& a, uint8_t* base) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base ? base + off : nullptr;
    off += (bytes + 255) & ~(size_t)255;
    return p;
  };
  if (a.few && !a.few_alone) {
    const size_t rows = (size_t)a.few * 2 * a.few_rows;
    a.few_o = (float*)take(rows * D * 4);
    a.few_ml = (float*)take(rows * 2 * 4);
    a.few_meta = (int32_t*)take((size_t)a.few * 4 * 4);
  }
  if (a.splits > 1) {
    const size_t rows = (size_t)a.Hkv * a.blocks * a.splits * a.rows;
    a.part_o = (float*)take(rows * D * 4);
    a.part_ml = (float*)take(rows * 2 * 4);
  }
  return off;
}

protokv_status page_attend_shape(const protokv_page_attend_args* p, ExactArgs& a, bool four, const char* who) {
  const Heads h{p->num_q_heads, p->num_kv_heads, p->head_dim, p->kv_dtype};
  protokv_status s = check_heads(h, who);
  if (s != PROTOKV_OK) return s;
  if (p->num_requests < 0 || p->total < 0) return fail(PROTOKV_E_INVALID, who, "counts must be >= 0");
  if ((int64_t)p->total * h.q >= (1ll << 31) || p->num_requests >= (1 << 24))
    return fail(PROTOKV_E_UNSUPPORTED, who, "total * num_q_heads must be below 2^31, the number of sequences below 2^24");
  if (p->max_add < 1) return fail(PROTOKV_E_INVALID, who, "max_add must be >= 1");
  s = check_page_sizes(p->pages.num_pages, p->pages.page_size, who);
  if (s != PROTOKV_OK) return s;
  // (the places of a few tiles behind the last token are formed in 32 bits)
  if (p->table_stride < 1 || (int64_t)p->table_stride * p->pages.page_size > (1ll << 31) - 2048)
    return fail(PROTOKV_E_INVALID, who, "table_stride must be >= 1 and table_stride * page_size at most 2^31 - 2048");
  a.n = p->num_requests;
  a.total = p->total;
  a.max_add = p->max_add;
  a.Hq = h.q;
  a.Hkv = h.kv;
  a.grp = h.q / h.kv;
  a.stride = p->table_stride;
  a.shift = log2i(p->pages.page_size);
  a.num_pages = p->pages.num_pages;
  const bool fp32 = h.dtype == PROTOKV_KV_FP32;
  // requests of few rows go to a kernel of their own, the others to row blocks.  Its two
  // launches take 9 us even if no request has few rows; where some may have more, row
  // blocks take them all if that costs little: blocks that fill a quarter of the GPU at
  // most (8 x 16 tokens over 2000, 28 / 4 heads: 39 us with them, 31 without; 7 single
  // tokens over 30 000, 32 / 8 heads, that might have been more: 177 and 156), or 256
  // rows to a request on average (4 x 512 over 4096: 149 and 140; 4000 and six single
  // ones over 16 k: 814 and 785).
  const bool many = (int64_t)a.max_add * a.grp > EX_FEW;
  const int64_t rows = (int64_t)a.total * a.grp;
  const bool alone = many && ((rows / EX_ROWS + a.n) * a.Hkv <= 64 || rows >= (int64_t)256 * a.n);
  const bool with_few = !fp32 && !alone;
  a.few_limit = EX_FEW;
  a.few_rows = (int)std::min<int64_t>(EX_FEW, (int64_t)a.max_add * a.grp);
  const int64_t span = (int64_t)a.stride << a.shift;
  auto few_waves = [&](int64_t runs) {
    a.few = a.n ? (int)std::min<int64_t>(EX_FEW_WAVES, (std::max<int64_t>(1, runs) + 3) / 4 * 4) : 0;
  };
  a.splits = 1;
  if (fp32) plan_blocks_f32(a, true);
  const int64_t cost = !fp32 && many ? plan_blocks(a, true) + (with_few ? 45 : 0) : 0;
  s = check_grid(a, who);
  if (s != PROTOKV_OK) return s;
  if (four && !fp32) {
    // Pages of 4 bits: the few-rows kernel takes requests of more rows too, in groups of
    // 32, if it takes all of them and that costs less: its waves go through equal runs of tiles
    // whatever the lengths, where a row block of few rows leaves most of its compute unit
    // idle and a long context among short ones holds one for its whole length.  A wave's tile of 64
    // keys counts 16 of plan_blocks' tenths where the waves fill the GPU, else 10, launches and join
    // 60, and a fifth on top, which the blocks' count is closer by.  Calls by row blocks and by groups, 28 / 4 heads: 64 x 16
    // tokens over 8000 328 and 207 us; 8 x 40 over 250 to 16 000, 32 / 8 heads, 105 and 55; but 8 x 512 over 16 000 890
    // and 1268, one chunk of 64 over 30 000 49 and 61.  Over 100 shapes of 1 to 64 requests this choice took
    // 1.8 % longer than the better of the two on average, 29 % at most.
    const int64_t groups = many ? rows / EX_FEW + a.n : a.n, tiles = a.Hkv * groups * ((span + 63) / 64);
    const int64_t run = std::max<int64_t>({(tiles + EX_FEW_WAVES - 1) / EX_FEW_WAVES, std::min<int64_t>(EX_FEW_RUN4, (tiles + 511) / 512), 1});
    const bool all = many && (run * (tiles > 1024 * run ? 16 : 10) + 60) * 6 / 5 <= cost;
    if (all) {
      a.few_limit = INT32_MAX;
      a.blocks = 0;
      a.splits = 1;
    }
    if (all || with_few) few_waves(tiles);
    a.few_alone = span <= 64 * EX_FEW_ALONE4;
  } else if (with_few) {
    few_waves(((int64_t)a.Hkv * a.n * ((span + 31) / 32) + 1) / 2);
  }
  return PROTOKV_OK;
}

protokv_status rotate(const protokv_rotate_args* a, const protokv_head_norm* norm, void* stream, const char* who) {
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  const Heads h{a->num_q_heads, a->num_kv_heads, a->head_dim, a->kv_dtype};
  protokv_status s = check_heads(h, who);
  if (s != PROTOKV_OK) return s;
  if (a->num_tokens < 0) return fail(PROTOKV_E_INVALID, who, "num_tokens must be >= 0");
  if (a->num_axes < 1 || a->num_axes > MAX_AXES) return fail(PROTOKV_E_INVALID, who, "num_axes must be in [1, 8]");
  if (!a->axes) return fail(PROTOKV_E_INVALID, who, "axes is NULL");
  for (int i = 0; i < D / 2; ++i)
    if (a->axes[i] >= a->num_axes) return fail(PROTOKV_E_INVALID, who, "axes: an entry is not below num_axes");
  if (!(a->theta > 1.0) || !std::isfinite(a->theta)) return fail(PROTOKV_E_INVALID, who, "theta must be a finite base > 1");
  if (a->position_stride < 0) return fail(PROTOKV_E_INVALID, who, "position_stride must be >= 0");
  if (a->num_tokens == 0) return PROTOKV_OK;  // (empty arrays may have no address)
  if (!a->q && !a->k) return fail(PROTOKV_E_INVALID, who, "neither q nor k");
  if ((a->q == nullptr) != (a->q_out == nullptr)) return fail(PROTOKV_E_INVALID, who, "q and q_out go together");
  if (a->k && !a->k_out && !a->pages) return fail(PROTOKV_E_INVALID, who, "k needs k_out or pages");
  if (!a->k && (a->k_out || a->pages)) return fail(PROTOKV_E_INVALID, who, "k_out and pages need k");
  if ((a->pages == nullptr) != (a->v == nullptr)) return fail(PROTOKV_E_INVALID, who, "v and pages go together");
  RotateArgs r;
  std::memset(&r, 0, sizeof(r));
  if (a->pages) {
    s = check_page_rows(*a->pages, who);
    if (s == PROTOKV_OK) s = check_page_sizes(a->pages->num_pages, a->pages->page_size, who);
    if (s != PROTOKV_OK) return s;
    r.kp = (uint8_t*)a->pages->k;
    r.vp = (uint8_t*)a->pages->v;
    r.shift = log2i(a->pages->page_size);
    r.nslots = a->pages->num_pages * a->pages->page_size;
  }
  if (!a->positions || off4(a->positions)) return fail(PROTOKV_E_INVALID, who, "positions must be non-NULL and aligned to 4 bytes");
  if (a->pages && (!a->slots || off4(a->slots))) return fail(PROTOKV_E_INVALID, who, "slots must be non-NULL and aligned to 4 bytes");
  const int es = h.es();
  if (a->q) {
    s = check_rows(a->q, a->q_stride, h.q, h, who, "q");
    if (s == PROTOKV_OK) s = check_rows(a->q_out, a->q_out_stride, h.q, h, who, "q_out");
    if (s == PROTOKV_OK && a->q_out == a->q && a->q_out_stride != a->q_stride)
      s = fail(PROTOKV_E_INVALID, who, "q_out is q with another stride");
    if (s != PROTOKV_OK) return s;
  }
  if (a->k) {
    s = check_rows(a->k, a->k_stride, h.kv, h, who, "k");
    if (s == PROTOKV_OK && a->k_out) s = check_rows(a->k_out, a->k_out_stride, h.kv, h, who, "k_out");
    if (s == PROTOKV_OK && a->k_out == a->k && a->k_out_stride != a->k_stride)
      s = fail(PROTOKV_E_INVALID, who, "k_out is k with another stride");
    if (s == PROTOKV_OK && a->v) s = check_rows(a->v, a->v_stride, h.kv, h, who, "v");
    if (s != PROTOKV_OK) return s;
  }
  r.q = (const uint8_t*)a->q;
  r.k = (const uint8_t*)a->k;
  r.v = (const uint8_t*)a->v;
  r.qo = (uint8_t*)a->q_out;
  r.ko = (uint8_t*)a->k_out;
  r.pos = a->positions;
  r.slots = a->slots;
  r.qs = a->q_stride * es;
  r.ks = a->k_stride * es;
  r.vs = a->v_stride * es;
  r.qos = a->q_out_stride * es;
  r.kos = a->k_out_stride * es;
  r.ps = a->position_stride;
  r.N = a->num_tokens;
  r.Hq = a->q ? h.q : 0;
  r.Hkv = a->k ? h.kv : 0;
  // a wave per token and eight heads (a wave per token, 40 000 tokens of 32 + 8 heads:
  // 156 us against 139)
  r.parts = (r.Hq + (r.nslots ? 2 : 1) * r.Hkv + 7) / 8;
  if (((int64_t)r.N * r.parts + 3) / 4 >= (1ll << 32) / 256)  // a launch has fewer than 2^32 threads, 256 to a workgroup
    return fail(PROTOKV_E_UNSUPPORTED, who, "num_tokens times heads above 2^29");
  std::memcpy(r.axis, a->axes, D / 2);
  for (int i = 0; i < D / 2; ++i) r.inv[i] = std::pow(a->theta, -2.0 * i / D);
  NormArgs n{};
  if (norm) n = NormArgs{(const uint8_t*)norm->q_weight, (const uint8_t*)norm->k_weight, norm->eps};
  return device(launch_rotate(r, norm ? &n : nullptr, h.dtype == PROTOKV_KV_FP32, (hipStream_t)stream), who);
}

protokv_status page_attend(const protokv_page_attend_args* p, const protokv_pages4* four, void* stream, const char* who) {
  ExactArgs a{};
  protokv_status s = page_attend_shape(p, a, four != nullptr, who);
  if (s != PROTOKV_OK) return s;
  const Heads h{p->num_q_heads, p->num_kv_heads, p->head_dim, p->kv_dtype};
  s = check_result(h, p->num_requests, p->total, p->cu, p->o, p->lse, p->prior_o, p->prior_lse, who);
  if (s != PROTOKV_OK || p->num_requests == 0 || p->total == 0) return s;
  s = four ? check_pages4(*four, h.kv, who) : check_page_rows(p->pages, who);
  if (s == PROTOKV_OK) s = check_rows(p->q, p->q_stride, h.q, h, who, "q");
  if (s != PROTOKV_OK) return s;
  if (!p->kv_len || !p->table || off4(p->kv_len) || off4(p->table))
    return fail(PROTOKV_E_INVALID, who, "kv_len and table must be non-NULL and aligned to 4 bytes");
  const bool fp32 = h.dtype == PROTOKV_KV_FP32;
  const size_t need = lay_out(a, nullptr);
  if (need) {
    if (!p->workspace) return fail(PROTOKV_E_WORKSPACE, who, "workspace is NULL");
    if ((uintptr_t)p->workspace % 256) return fail(PROTOKV_E_WORKSPACE, who, "workspace must be 256-byte aligned");
    if (p->workspace_bytes < need)
      return fail(PROTOKV_E_WORKSPACE, who, ("workspace too small: need " + std::to_string(need) + " bytes").c_str());
    lay_out(a, (uint8_t*)p->workspace);
  }
  a.q = p->q;
  a.k = p->pages.k;
  a.v = p->pages.v;
  a.o = p->o;
  a.lse = p->lse;
  a.po = p->prior_o;
  a.pl = p->prior_lse;
  a.cu = p->cu;
  a.kv_len = p->kv_len;
  a.table = p->table;
  a.qs = p->q_stride * h.es();
  if (four) {
    a.ksc = four->k_scale;
    a.vsc = four->v_scale;
  }
  return device(launch_exact(a, fp32, four ? Keys::PAGES4 : Keys::PAGES, (hipStream_t)stream), who);
}

// The same call over exact pages: sizes and addresses of everything but the pages' own.
protokv_page_attend_args as_page_attend(const protokv_page4_attend_args& p) {
  protokv_page_attend_args a;
  a.num_q_heads = p.num_q_heads;
  a.num_kv_heads = p.num_kv_heads;
  a.head_dim = p.head_dim;
  a.kv_dtype = p.kv_dtype;
  a.num_requests = p.num_requests;
  a.total = p.total;
  a.max_add = p.max_add;
  a.table_stride = p.table_stride;
  a.cu = p.cu;
  a.kv_len = p.kv_len;
  a.table = p.table;
  a.q = p.q;
  a.q_stride = p.q_stride;
  a.pages = protokv_pages{p.pages.k, p.pages.v, p.pages.num_pages, p.pages.page_size};
  a.o = p.o;
  a.lse = p.lse;
  a.prior_o = p.prior_o;
  a.prior_lse = p.prior_lse;
  a.workspace = p.workspace;
  a.workspace_bytes = p.workspace_bytes;
  return a;
}

protokv_status attend_workspace(const protokv_page_attend_args& p, bool four, size_t* bytes, const char* who) {
  ExactArgs a{};
  protokv_status s = page_attend_shape(&p, a, four, who);
  if (s == PROTOKV_OK) *bytes = lay_out(a, nullptr);
  return s;
}

protokv_status page4_rows(const protokv_page4_rows_args* a, bool store, void* stream, const char* who) {
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  const Heads h{a->num_kv_heads, a->num_kv_heads, a->head_dim, a->kv_dtype};
  protokv_status s = check_heads(h, who);
  if (s != PROTOKV_OK) return s;
  if (a->num_tokens < 0) return fail(PROTOKV_E_INVALID, who, "num_tokens must be >= 0");
  s = check_page_sizes(a->pages.num_pages, a->pages.page_size, who);
  if (s != PROTOKV_OK) return s;
  const int64_t rows = 2 * (int64_t)a->num_tokens * h.kv;
  if (rows >= (1ll << 27) - 8)  // up to 32 threads to a row, fewer than 2^32 to a launch in whole workgroups
    return fail(PROTOKV_E_UNSUPPORTED, who, "2 * num_tokens * num_kv_heads must be below 2^27 - 8");
  if (rows == 0) return PROTOKV_OK;  // (empty arrays may have no address)
  s = check_pages4(a->pages, h.kv, who);
  if (s == PROTOKV_OK) s = check_rows(a->k, a->k_stride, h.kv, h, who, "k");
  if (s == PROTOKV_OK) s = check_rows(a->v, a->v_stride, h.kv, h, who, "v");
  if (s != PROTOKV_OK) return s;
  if (!a->slots || off4(a->slots)) return fail(PROTOKV_E_INVALID, who, "slots must be non-NULL and aligned to 4 bytes");
  if (!store && a->k == a->v) return fail(PROTOKV_E_INVALID, who, "k and v are the same rows");
  if (store && (a->pages.k == a->pages.v || a->pages.k_scale == a->pages.v_scale))
    return fail(PROTOKV_E_INVALID, who, "pages: k and v are the same array");
  Page4Rows r{};
  r.k = (uint8_t*)a->k;
  r.v = (uint8_t*)a->v;
  r.slots = a->slots;
  r.pk = a->pages.k;
  r.pv = a->pages.v;
  r.ksc = a->pages.k_scale;
  r.vsc = a->pages.v_scale;
  r.ks = a->k_stride * h.es();
  r.vs = a->v_stride * h.es();
  r.rows = rows;
  r.Hkv = h.kv;
  r.shift = log2i(a->pages.page_size);
  r.nslots = a->pages.num_pages * a->pages.page_size;
  return device(launch_page4_rows(r, h.dtype == PROTOKV_KV_FP32, store, (hipStream_t)stream), who);
}

}  // namespace

// What a check or a message allocates may fail; nothing may leave a C entry.
#define PKV_GUARD(who, ...)                                      \
  try __VA_ARGS__ catch (...) {                                  \
    try { call_error() = who ": out of memory"; } catch (...) {} \
    return PROTOKV_E_DEVICE;                                     \
  }

extern "C" {

protokv_status protokv_page_plan(const protokv_page_plan_args* a, void* stream) PKV_GUARD("page_plan", {
  const char* who = "page_plan";
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  const protokv_status s = check_table(a->num_requests, a->num_pages, a->page_size, a->table_stride, who);
  if (s != PROTOKV_OK) return s;
  if (a->max_tokens < 1 || a->max_tokens > (1 << 29)) return fail(PROTOKV_E_INVALID, who, "max_tokens must be in [1, 2^29]");
  const void* need[] = {a->ctx, a->add, a->table, a->free_pages, a->free_count, a->free_count_out, a->cu, a->kv_len, a->slots};
  for (const void* p : need)
    if (!p || off4(p)) return fail(PROTOKV_E_INVALID, who, "arrays must be non-NULL and aligned to 4 bytes");
  if (off4(a->base) || off4(a->positions) || off4(a->refused))
    return fail(PROTOKV_E_INVALID, who, "arrays must be aligned to 4 bytes");
  // every workgroup reads the inputs while the first writes the outputs
  const void* in[] = {a->ctx, a->add, a->base, a->free_count};
  const void* out[] = {a->free_count_out, a->cu, a->kv_len, a->slots, a->positions, a->refused};
  for (const void* p : in)
    for (const void* q : out)
      if (p && p == q) return fail(PROTOKV_E_INVALID, who, "an output must not be one of ctx, add, base and free_count");
  return device(launch_page_plan(*a, (hipStream_t)stream), who);
})

protokv_status protokv_rotate(const protokv_rotate_args* a, void* stream) PKV_GUARD("rotate", {
  return rotate(a, nullptr, stream, "rotate");
})

protokv_status protokv_norm_rotate(const protokv_rotate_args* a, const protokv_head_norm* norm,
                                   void* stream) PKV_GUARD("norm_rotate", {
  const char* who = "norm_rotate";
  if (!norm) return fail(PROTOKV_E_INVALID, who, "norm is NULL");
  if (!(norm->eps >= 0.0) || !std::isfinite(norm->eps)) return fail(PROTOKV_E_INVALID, who, "eps must be finite and >= 0");
  if (off16(norm->q_weight) || off16(norm->k_weight))
    return fail(PROTOKV_E_INVALID, who, "q_weight and k_weight must be aligned to 16 bytes");
  return rotate(a, norm, stream, who);
})

protokv_status protokv_prompt_attend(const protokv_prompt_args* p, void* stream) PKV_GUARD("prompt_attend", {
  const char* who = "prompt_attend";
  if (!p) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  const Heads h{p->num_q_heads, p->num_kv_heads, p->head_dim, p->kv_dtype};
  protokv_status s = check_heads(h, who);
  if (s == PROTOKV_OK) s = check_result(h, p->num_seqs, p->total, p->cu, p->o, p->lse, p->prior_o, p->prior_lse, who);
  if (s != PROTOKV_OK || p->num_seqs == 0 || p->total == 0) return s;
  s = check_rows(p->q, p->q_stride, h.q, h, who, "q");
  if (s == PROTOKV_OK) s = check_rows(p->k, p->k_stride, h.kv, h, who, "k");
  if (s == PROTOKV_OK) s = check_rows(p->v, p->v_stride, h.kv, h, who, "v");
  if (s != PROTOKV_OK) return s;
  const bool fp32 = h.dtype == PROTOKV_KV_FP32;
  ExactArgs a{};
  a.q = p->q;
  a.k = p->k;
  a.v = p->v;
  a.o = p->o;
  a.lse = p->lse;
  a.po = p->prior_o;
  a.pl = p->prior_lse;
  a.cu = p->cu;
  a.qs = p->q_stride * h.es();
  a.ks = p->k_stride * h.es();
  a.vs = p->v_stride * h.es();
  a.n = p->num_seqs;
  a.total = p->total;
  a.max_add = p->total;
  a.Hq = h.q;
  a.Hkv = h.kv;
  a.grp = h.q / h.kv;
  if (fp32) plan_blocks_f32(a, false);
  else plan_blocks(a, false);
  s = check_grid(a, who);
  if (s != PROTOKV_OK) return s;
  return device(launch_exact(a, fp32, Keys::ROWS, (hipStream_t)stream), who);
})

protokv_status protokv_page_attend_workspace(const protokv_page_attend_args* p, size_t* bytes) PKV_GUARD("page_attend_workspace", {
  const char* who = "page_attend_workspace";
  if (!p || !bytes) return fail(PROTOKV_E_INVALID, who, "args and bytes must be non-NULL");
  return attend_workspace(*p, false, bytes, who);
})

protokv_status protokv_page_attend(const protokv_page_attend_args* p, void* stream) PKV_GUARD("page_attend", {
  const char* who = "page_attend";
  if (!p) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  return page_attend(p, nullptr, stream, who);
})

protokv_status protokv_page4_attend_workspace(const protokv_page4_attend_args* p, size_t* bytes) PKV_GUARD("page4_attend_workspace", {
  const char* who = "page4_attend_workspace";
  if (!p || !bytes) return fail(PROTOKV_E_INVALID, who, "args and bytes must be non-NULL");
  return attend_workspace(as_page_attend(*p), true, bytes, who);
})

protokv_status protokv_page4_attend(const protokv_page4_attend_args* p, void* stream) PKV_GUARD("page4_attend", {
  const char* who = "page4_attend";
  if (!p) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  const protokv_page_attend_args a = as_page_attend(*p);
  return page_attend(&a, &p->pages, stream, who);
})

protokv_status protokv_page4_store(const protokv_page4_rows_args* a, void* stream) PKV_GUARD("page4_store", {
  return page4_rows(a, true, stream, "page4_store");
})

protokv_status protokv_page4_read(const protokv_page4_rows_args* a, void* stream) PKV_GUARD("page4_read", {
  return page4_rows(a, false, stream, "page4_read");
})

protokv_status protokv_page_fork(const protokv_page_fork_args* a, void* stream) PKV_GUARD("page_fork", {
  const char* who = "page_fork";
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  if (a->num_forks < 1) return fail(PROTOKV_E_INVALID, who, "num_forks must be >= 1");
  if (a->num_forks > MAX_REQUESTS) return fail(PROTOKV_E_UNSUPPORTED, who, "num_forks above 8192");
  protokv_status s = check_table(a->num_requests, a->num_pages, a->page_size, a->table_stride, who);
  if (s == PROTOKV_OK)
    s = check_arrays({a->ctx, a->src, a->dst, a->table, a->shares, a->free_pages, a->free_count, a->free_count_out, a->ctx_out,
                      a->lens, a->copy_src, a->copy_dst, a->copy_rows},
                     {a->at, a->refused}, {a->ctx, a->src, a->dst, a->at, a->free_pages, a->free_count},
                     {a->table, a->shares, a->free_count_out, a->ctx_out, a->lens, a->copy_src, a->copy_dst, a->copy_rows, a->refused},
                     who);
  if (s != PROTOKV_OK) return s;
  return device(launch_page_fork(*a, (hipStream_t)stream), who);
})

protokv_status protokv_page_copy(const protokv_page_copy_args* a, void* stream) PKV_GUARD("page_copy", {
  const char* who = "page_copy";
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  if (a->num_copies < 0) return fail(PROTOKV_E_INVALID, who, "num_copies must be >= 0");
  if (a->num_kv_heads < 1 || a->num_kv_heads > 65536) return fail(PROTOKV_E_INVALID, who, "num_kv_heads must be in [1, 65536]");
  protokv_status s = check_page_sizes(a->num_pages, a->page_size, who);
  if (s != PROTOKV_OK) return s;
  if (a->num_arrays < 1 || a->num_arrays > MAX_ARRAYS || !a->arrays)
    return fail(PROTOKV_E_INVALID, who, "num_arrays must be in [1, 128] and arrays non-NULL");
  PageCopy c;
  std::memset(&c, 0, sizeof(c));
  int64_t layers = 0, most = 0;
  for (int i = 0; i < a->num_arrays; ++i) {
    const protokv_page_array& x = a->arrays[i];
    if (x.row_bytes < 4 || x.row_bytes > 4096 || x.row_bytes % 4)
      return fail(PROTOKV_E_INVALID, who, "arrays: row_bytes must be a multiple of 4 in [4, 4096]");
    if (x.layers < 1) return fail(PROTOKV_E_INVALID, who, "arrays: layers must be >= 1");
    const int64_t page = (int64_t)x.row_bytes * a->num_kv_heads * a->page_size;
    if (page >= (1ll << 31)) return fail(PROTOKV_E_UNSUPPORTED, who, "a page of 2^31 bytes or more");
    // rows of 16 bytes each are copied by 16, others by 4, whose layers, one behind the other, need no more alignment
    const bool gap = x.layers > 1 && x.layer_stride != page * a->num_pages, by4 = x.row_bytes % 16 && !gap;
    if (a->num_copies && (!x.base || (by4 ? off4(x.base) : off16(x.base))))
      return fail(PROTOKV_E_INVALID, who, "arrays: base must be non-NULL and aligned to 16 bytes (to 4 for rows that are no "
                  "multiple of 16, if layers follow one another)");
    if (gap && (x.layer_stride < page * a->num_pages || x.layer_stride % 16))
      return fail(PROTOKV_E_INVALID, who, "arrays: layer_stride must be a layer's bytes, or more and a multiple of 16");
    c.base[i] = (uint8_t*)x.base;
    c.layer_stride[i] = x.layers > 1 ? x.layer_stride : 0;
    c.row_bytes[i] = x.row_bytes;
    c.first[i] = (int)layers;
    layers += x.layers;
    if (layers > 65535) return fail(PROTOKV_E_UNSUPPORTED, who, "more than 65535 layers in all");
    most = std::max(most, x.row_bytes % 16 ? page / 4 : page / 16);
  }
  if (a->num_copies == 0) return PROTOKV_OK;
  if (!a->src || !a->dst || off4(a->src) || off4(a->dst) || off4(a->rows))
    return fail(PROTOKV_E_INVALID, who, "src and dst must be non-NULL, and they and rows aligned to 4 bytes");
  // a launch has fewer than 2^32 threads: fewer workgroups to a page where there are many pages, and
  // parts of the copies in launches of their own where that is not enough
  const int64_t most_wgs = (1ll << 32) / 256 - 1;
  if (layers * a->num_copies > most_wgs && a->num_copies > MAX_REQUESTS)
    return fail(PROTOKV_E_UNSUPPORTED, who, "more than 8192 copies, and num_copies times the layers not below 2^24");
  const int64_t each = std::min<int64_t>(a->num_copies, most_wgs / layers);  // (at least 256)
  // four units to a thread, up to 64 workgroups to a page
  const int64_t parts = std::min({(most + 1023) / 1024, (int64_t)64, most_wgs / (layers * each)});
  c.num_arrays = a->num_arrays;
  c.num_pages = a->num_pages;
  c.Hkv = a->num_kv_heads;
  c.shift = log2i(a->page_size);
  for (int64_t i = 0; i < a->num_copies; i += each) {
    c.src = a->src + i;
    c.dst = a->dst + i;
    c.rows = a->rows ? a->rows + i : nullptr;
    s = device(launch_page_copy(c, (int)std::min(each, a->num_copies - i), (int)layers, (unsigned)parts, (hipStream_t)stream), who);
    if (s != PROTOKV_OK) return s;
  }
  return PROTOKV_OK;
})

protokv_status protokv_page_release(const protokv_page_release_args* a, void* stream) PKV_GUARD("page_release", {
  const char* who = "page_release";
  if (!a) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  protokv_status s = check_table(a->num_requests, a->num_pages, a->page_size, a->table_stride, who);
  if (s == PROTOKV_OK)
    s = check_arrays({a->ctx, a->keep, a->table, a->shares, a->free_pages, a->free_count, a->free_count_out, a->ctx_out,
                      a->refused, a->scratch},
                     {}, {a->ctx, a->keep, a->table, a->free_count},
                     {a->shares, a->free_pages, a->free_count_out, a->ctx_out, a->refused, a->scratch}, who);
  if (s != PROTOKV_OK) return s;
  return device(launch_page_release(*a, (hipStream_t)stream), who);
})

}  // extern "C"
