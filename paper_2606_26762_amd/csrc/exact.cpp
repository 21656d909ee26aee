// Host side of the handle-free calls: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>

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

protokv_status check_page_sizes(const protokv_pages& p, const char* who) {
  if (p.num_pages < 1) return fail(PROTOKV_E_INVALID, who, "num_pages must be >= 1");
  if (!pow2(p.page_size) || p.page_size > 1024)
    return fail(PROTOKV_E_UNSUPPORTED, who, "page_size must be a power of two in [1, 1024]");
  if ((int64_t)p.num_pages * p.page_size >= (1ll << 31))
    return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages * page_size must be below 2^31");
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
void plan_blocks(ExactArgs& a, bool paged) {
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
  if (a.few) {
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

protokv_status page_attend_shape(const protokv_page_attend_args* p, ExactArgs& a, const char* who) {
  const Heads h{p->num_q_heads, p->num_kv_heads, p->head_dim, p->kv_dtype};
  protokv_status s = check_heads(h, who);
  if (s != PROTOKV_OK) return s;
  if (p->num_requests < 0 || p->total < 0) return fail(PROTOKV_E_INVALID, who, "counts must be >= 0");
  if ((int64_t)p->total * h.q >= (1ll << 31) || p->num_requests >= (1 << 24))
    return fail(PROTOKV_E_UNSUPPORTED, who, "total * num_q_heads must be below 2^31, the number of sequences below 2^24");
  if (p->max_add < 1) return fail(PROTOKV_E_INVALID, who, "max_add must be >= 1");
  s = check_page_sizes(p->pages, who);
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
  if (!fp32 && !alone) {
    const int64_t tiles = (((int64_t)a.stride << a.shift) + 31) / 32;
    const int64_t waves = std::max<int64_t>(1, ((int64_t)a.Hkv * a.n * tiles + 1) / 2);
    a.few = a.n ? (int)std::min<int64_t>(EX_FEW_WAVES, (waves + 3) / 4 * 4) : 0;
    a.few_rows = (int)std::min<int64_t>(EX_FEW, (int64_t)a.max_add * a.grp);
  }
  a.splits = 1;
  if (fp32) plan_blocks_f32(a, true);
  else if (many) plan_blocks(a, true);
  return check_grid(a, who);
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
  if (a->num_requests < 1) return fail(PROTOKV_E_INVALID, who, "num_requests must be >= 1");
  if (a->num_requests > MAX_REQUESTS) return fail(PROTOKV_E_UNSUPPORTED, who, "num_requests above 8192");
  if (a->num_pages < 1) return fail(PROTOKV_E_INVALID, who, "num_pages must be >= 1");
  if (!pow2(a->page_size) || a->page_size > 1024)
    return fail(PROTOKV_E_UNSUPPORTED, who, "page_size must be a power of two in [1, 1024]");
  if ((int64_t)a->num_pages * a->page_size >= (1ll << 31))
    return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages * page_size must be below 2^31");
  if (a->table_stride < 1 || (int64_t)a->table_stride * a->page_size >= (1ll << 31))
    return fail(PROTOKV_E_INVALID, who, "table_stride must be >= 1 and table_stride * page_size below 2^31");
  if (a->num_pages > (1 << 29)) return fail(PROTOKV_E_UNSUPPORTED, who, "num_pages above 2^29");
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
  const char* who = "rotate";
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
    if (s == PROTOKV_OK) s = check_page_sizes(*a->pages, who);
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
  return device(launch_rotate(r, h.dtype == PROTOKV_KV_FP32, (hipStream_t)stream), who);
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
  return device(launch_exact(a, fp32, false, (hipStream_t)stream), who);
})

protokv_status protokv_page_attend_workspace(const protokv_page_attend_args* p, size_t* bytes) PKV_GUARD("page_attend_workspace", {
  const char* who = "page_attend_workspace";
  if (!p || !bytes) return fail(PROTOKV_E_INVALID, who, "args and bytes must be non-NULL");
  ExactArgs a{};
  protokv_status s = page_attend_shape(p, a, who);
  if (s == PROTOKV_OK) *bytes = lay_out(a, nullptr);
  return s;
})

protokv_status protokv_page_attend(const protokv_page_attend_args* p, void* stream) PKV_GUARD("page_attend", {
  const char* who = "page_attend";
  if (!p) return fail(PROTOKV_E_INVALID, who, "args is NULL");
  ExactArgs a{};
  protokv_status s = page_attend_shape(p, a, who);
  if (s != PROTOKV_OK) return s;
  const Heads h{p->num_q_heads, p->num_kv_heads, p->head_dim, p->kv_dtype};
  s = check_result(h, p->num_requests, p->total, p->cu, p->o, p->lse, p->prior_o, p->prior_lse, who);
  if (s != PROTOKV_OK || p->num_requests == 0 || p->total == 0) return s;
  s = check_page_rows(p->pages, who);
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
  return device(launch_exact(a, fp32, true, (hipStream_t)stream), who);
})

}  // extern "C"
