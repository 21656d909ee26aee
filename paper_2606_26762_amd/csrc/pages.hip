// Pages of 4 bits (protokv_page4_store, protokv_page4_read) and pages that several
// requests hold (protokv_page_fork, protokv_page_copy, protokv_page_release) for gfx950.
#include "exact.h"
#include "page4.h"
#include "pkv_internal.h"

namespace pkv {

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------------------
// Rows into and out of 4 bits.  A thread takes 16 bytes of a row (token, head, k or v),
// so that a wave's accesses are whole rows: 4 dims of float32, eight threads to a block of
// 32, or 8 of bfloat16, four.  v_cvt_scalef32_pk_fp4_f32 divides by the power of two,
// rounds to the nearest code, ties to the even one, and ends at 6, which is the format's own rule
// (all bfloat16 values and the codes' borders checked against it); the way back is
// exact.  Bound by the rows' bytes.
// ---------------------------------------------------------------------------

// Row r of a call is k's or v's head r % Hkv of token r / (2 Hkv), k's first.
struct Row4 {
  int token, head;
  bool value;
};
__device__ __forceinline__ Row4 row4_of(const Page4Rows& a, unsigned r) {  // below 2^27
  const unsigned per = 2 * a.Hkv, t = r / per;
  const int j = (int)(r - t * per);
  return {(int)t, j >= a.Hkv ? j - a.Hkv : j, j >= a.Hkv};
}
__device__ __forceinline__ int slot4_of(const Page4Rows& a, const Row4& x) {
  const int s = a.slots[x.token];
  return (unsigned)s < (unsigned)a.nslots ? s : -1;
}
template <int FP32>
__device__ __forceinline__ uint4* row4_at(const Page4Rows& a, const Row4& x) {
  return reinterpret_cast<uint4*>((x.value ? a.v : a.k) + x.token * (x.value ? a.vs : a.ks) + (size_t)x.head * (D * (FP32 ? 4 : 2)));
}
// row of the pages that a slot's head is
__device__ __forceinline__ long long place4(const Page4Rows& a, const Row4& x, int slot) {
  return (((long long)(slot >> a.shift) * a.Hkv + x.head) << a.shift) + (slot & ((1 << a.shift) - 1));
}

// P4_U: pieces of a thread, a workgroup's width apart, all in flight
template <int FP32, int P4_U>
__global__ __launch_bounds__(256) void k_page4_store(Page4Rows a) {
  constexpr int W = FP32 ? 4 : 8;  // dims to a piece
  uint4 in[P4_U];
  Row4 x[P4_U];
  int slot[P4_U];
  const unsigned c = threadIdx.x % (D / W);
#pragma unroll
  for (int u = 0; u < P4_U; ++u) {
    const unsigned r = (blockIdx.x * P4_U + u) * (256u / (D / W)) + threadIdx.x / (D / W);
    slot[u] = -1;
    if (r < a.rows) {  // the threads of a row together
      x[u] = row4_of(a, r);
      slot[u] = slot4_of(a, x[u]);
      in[u] = row4_at<FP32>(a, x[u])[c];
    }
  }
#pragma unroll
  for (int u = 0; u < P4_U; ++u) {
    if (slot[u] < 0) continue;
    const uint32_t w[4] = {in[u].x, in[u].y, in[u].z, in[u].w};
    float v[W];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (FP32) {
        v[i] = __uint_as_float(w[i]);
      } else {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
      }
    }
    // the block's largest |x| by its bits, where infinities and NaN lie above every number
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) top = max(top, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xf, 0xf, false));  // lane ^ 1
    top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xf, 0xf, false));  // lane ^ 2
    if (FP32) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xf, 0xf, false));  // the other four of eight
    // least e with top <= 7 * 2^e: two below top's exponent, one more past 1.75
    const bool odd = top >= 0x7F800000u;
    const int s = odd ? 255 : min(max((int)((top + 0x1FFFFFu) >> 23) - 2, 2), 252);
    const float scale = __uint_as_float((uint32_t)s << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0], v[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2], v[3], scale, 1);
    if constexpr (!FP32) {
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[4], v[5], scale, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[6], v[7], scale, 3);
    }
    if (odd) codes = 0;
    const long long at = place4(a, x[u], slot[u]);
    uint8_t* out = (x[u].value ? a.pv : a.pk) + at * (D / 2);
    if constexpr (FP32) reinterpret_cast<uint16_t*>(out)[c] = (uint16_t)codes;
    else reinterpret_cast<uint32_t*>(out)[c] = codes;
    if (c % (32 / W) == 0) (x[u].value ? a.vsc : a.ksc)[at * (D / 32) + c / (32 / W)] = (uint8_t)s;
  }
}

template <int FP32, int P4_U>
__global__ __launch_bounds__(256) void k_page4_read(Page4Rows a) {
  constexpr int W = FP32 ? 4 : 8;
  Row4 x[P4_U];
  int slot[P4_U];
  uint32_t codes[P4_U], s[P4_U];
  const unsigned c = threadIdx.x % (D / W), r0 = blockIdx.x * P4_U * (256u / (D / W)) + threadIdx.x / (D / W);
#pragma unroll
  for (int u = 0; u < P4_U; ++u) {
    x[u] = row4_of(a, min(r0 + u * (256u / (D / W)), (unsigned)a.rows - 1));  // past the last row it is read again
    slot[u] = slot4_of(a, x[u]);
  }
#pragma unroll
  for (int u = 0; u < P4_U; ++u) {
    codes[u] = s[u] = 0;
    if (slot[u] < 0) continue;
    const long long at = place4(a, x[u], slot[u]);
    const uint8_t* in = (x[u].value ? a.pv : a.pk) + at * (D / 2);
    codes[u] = FP32 ? reinterpret_cast<const uint16_t*>(in)[c] : reinterpret_cast<const uint32_t*>(in)[c];
    s[u] = (x[u].value ? a.vsc : a.ksc)[at * (D / 32) + c / (32 / W)];
  }
#pragma unroll
  for (int u = 0; u < P4_U; ++u) {
    if (r0 + u * (256u / (D / W)) >= a.rows) break;
    const float scale = __uint_as_float(s[u] << 23);
    uint4 out;
    if constexpr (FP32) {
      const f32x2 lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 0);
      const f32x2 hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[u], scale, 1);
      out = make_uint4(__float_as_uint(lo[0]), __float_as_uint(lo[1]), __float_as_uint(hi[0]), __float_as_uint(hi[1]));
    } else {
      out = values4(codes[u], scale);
    }
    row4_at<FP32>(a, x[u])[c] = out;
  }
}

// ---------------------------------------------------------------------------
// Forks.  One workgroup decides who is refused and who gets which page.  Where the
// forks' table rows are short together (PG_FEW entries) it copies them and counts the owners as well,
// else a second launch does that, with workgroups to each fork.  Latency chains both.
// ---------------------------------------------------------------------------
constexpr int FK_NT = 1024;
// Table entries, and pages, that one workgroup goes through by itself.  Both sides, microseconds of kernels at 1024, 4096,
// 8192, 16 384 and 32 768 entries: forks of 64 requests, four each, 4.8, 7.9, 13.4, 26.6, 52.6 by one workgroup and 5.9,
// 6.6, 6.6, 6.7, 7.8 by two launches; a third of 256 requests released 4.6, 6.9, 12.3, 22.1, 43.3 and 7.4, 8.5, 8.8, 8.9,
// 9.4 by three; of 8 requests, which three waves go through there, 4.6, 7.1, 12.9, 23.6, 47.3 and 7.5, 11.5, 15.7, 25.2,
// 42.6.  The sides meet near 3500 entries for forks and between 5000 and 20 000 for releases: forks above that, and
// releases of many requests, would be faster with a lower limit.
constexpr int PG_FEW = 16384;
constexpr int PG_REQ = 2048;   // and requests

// Inclusive running sum over the workgroup's threads; total: of all.  s: FK_NT / 64
// words, free again after the next barrier.
__device__ __forceinline__ int block_sum(int x, int* s, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int y = __shfl_up(x, d, 64);
    if (lane >= d) x += y;
  }
  if (lane == 63) s[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < FK_NT / 64; ++w) {
    const int y = s[w];
    if (w < wave) before += y;
    total += y;
  }
  return before + x;
}

template <int ROWS>
__global__ __launch_bounds__(FK_NT) void k_page_fork(protokv_page_fork_args a, int shift) {
  __shared__ int4 s_fork[ROWS ? PG_REQ : 1];     // full pages, src, dst
  __shared__ uint32_t s_src[MAX_REQUESTS / 32];  // requests that are forked
  __shared__ int s_dst[MAX_REQUESTS];            // first fork that becomes request r; once granted -1 - its tokens
  __shared__ int s_sum[2][FK_NT / 64];
  __shared__ int s_refused;
  const int tid = threadIdx.x, n = a.num_forks, R = a.num_requests, P1 = (1 << shift) - 1;
  const int span = a.table_stride << shift;
  const int held = min(max(a.free_count[0], 0), a.num_pages);
  for (int r = tid; r < R; r += FK_NT) s_dst[r] = 0x7FFFFFFF;
  for (int w = tid; w < (R + 31) / 32; w += FK_NT) s_src[w] = 0;
  if (tid == 0) s_refused = 0;
  __syncthreads();
  for (int i = tid; i < n; i += FK_NT) {
    const int s = a.src[i], d = a.dst[i];
    if ((unsigned)s < (unsigned)R && (unsigned)d < (unsigned)R && s != d) {
      atomicOr(&s_src[s >> 5], 1u << (s & 31));
      atomicMin(&s_dst[d], i);
    }
  }
  __syncthreads();
  int asked = 0, refused = 0;
  for (int i0 = 0, turn = 0; i0 < n; i0 += FK_NT, turn ^= 1) {
    const int i = i0 + tid;
    int s = 0, d = 0, len = 0;
    bool ok = false;
    if (i < n) {
      s = a.src[i];
      d = a.dst[i];
      ok = (unsigned)s < (unsigned)R && (unsigned)d < (unsigned)R && s != d && !((s_src[d >> 5] >> (d & 31)) & 1) &&
           s_dst[d] == i && a.ctx[d] <= 0;
      if (ok) {
        len = min(max(a.ctx[s], 0), span);
        if (a.at) len = min(max(a.at[i], 0), len);
      }
    }
    const int part = len & P1, full = len >> shift;
    int total;
    const int upto = asked + block_sum(ok && part, s_sum[turn], total);
    asked += total;
    if (i < n) {
      const bool take = ok && part;
      if (take && upto > held) ok = false;
      int from = -1, to = -1;
      if (ok && part) {
        from = a.table[(size_t)s * a.table_stride + full];
        to = a.free_pages[held - upto];
        a.table[(size_t)d * a.table_stride + full] = to;
      }
      a.lens[i] = ok ? len : -1;
      a.copy_src[i] = from;
      a.copy_dst[i] = to;
      a.copy_rows[i] = ok ? part : 0;
      if (ok) s_dst[d] = -1 - len;  // no other thread's fork is i
      if constexpr (ROWS) s_fork[i] = make_int4(ok ? full : 0, s, d, 0);
      refused += !ok;
    }
  }
  if (refused) atomicAdd(&s_refused, refused);
  __syncthreads();
  for (int r = tid; r < R; r += FK_NT) a.ctx_out[r] = s_dst[r] < 0 ? -1 - s_dst[r] : a.ctx[r];
  if (tid == 0) {
    a.free_count_out[0] = held - min(asked, held);
    if (a.refused) a.refused[0] = s_refused;
  }
  if constexpr (ROWS) {
    // (no src is a dst, so that what is read here was not written above)
    const int all = n * a.table_stride;
    for (int x0 = tid; x0 < all; x0 += 4 * FK_NT) {
      int page[4], to[4];  // four entries in flight
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = x0 + k * FK_NT, i = x / a.table_stride, j = x - i * a.table_stride;
        const int4 f = x < all ? s_fork[i] : make_int4(0, 0, 0, 0);
        to[k] = j < f.x ? f.z * a.table_stride + j : -1;  // (at most 8192 rows of PG_FEW)
        if (to[k] >= 0) page[k] = a.table[f.y * a.table_stride + j];
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (to[k] < 0) continue;
        a.table[to[k]] = page[k];
        if ((unsigned)page[k] < (unsigned)a.num_pages) atomicAdd(&a.shares[page[k]], 1);
      }
    }
  }
}

__global__ __launch_bounds__(256) void k_page_fork_rows(protokv_page_fork_args a, int shift) {
  const int i = blockIdx.y, full = a.lens[i] >> shift;  // refused: -1
  const size_t from = (size_t)(full > 0 ? a.src[i] : 0) * a.table_stride, to = (size_t)(full > 0 ? a.dst[i] : 0) * a.table_stride;
  for (int j = blockIdx.x * 256 + threadIdx.x; j < full; j += gridDim.x * 256) {
    const int page = a.table[from + j];
    a.table[to + j] = page;
    if ((unsigned)page < (unsigned)a.num_pages) atomicAdd(&a.shares[page], 1);
  }
}

// ---------------------------------------------------------------------------
// Rows of pages to other pages: bound by their bytes.  A head's rows of a page lie
// together; a workgroup takes a part of one copy in one layer of one array.
// ---------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ void copy_rows_of(const uint8_t* from, uint8_t* to, int heads, size_t head_bytes, unsigned per) {
  const unsigned all = heads * per, step = gridDim.y * 256;  // units of T: below 2^31, as a page's bytes are
  for (unsigned u0 = blockIdx.y * 256 + threadIdx.x; u0 < all; u0 += 4 * step) {
    T x[4];  // four units in flight
    size_t at[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const unsigned u = min(u0 + k * step, all - 1), h = u / per;  // past the last unit it is read again
      at[k] = h * head_bytes + (size_t)(u - h * per) * sizeof(T);
      x[k] = *reinterpret_cast<const T*>(from + at[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (u0 + k * step < all) *reinterpret_cast<T*>(to + at[k]) = x[k];
  }
}
__global__ __launch_bounds__(256) void k_page_copy(PageCopy a) {
  const int layer = blockIdx.z;
  int e = 0;
  while (e + 1 < a.num_arrays && layer >= a.first[e + 1]) ++e;  // uniform
  const int i = blockIdx.x, src = a.src[i], dst = a.dst[i], P = 1 << a.shift;
  if ((unsigned)src >= (unsigned)a.num_pages || (unsigned)dst >= (unsigned)a.num_pages || src == dst) return;
  const int rows = a.rows ? min(max(a.rows[i], 0), P) : P;
  const size_t rb = a.row_bytes[e], head = rb << a.shift, page = head * a.Hkv;
  uint8_t* base = a.base[e] + (size_t)(layer - a.first[e]) * a.layer_stride[e];
  const unsigned bytes = (unsigned)(rows * rb);
  if (bytes == 0) return;
  if (rb % 16 == 0) copy_rows_of<u32x4>(base + src * page, base + dst * page, a.Hkv, head, bytes / 16);
  else copy_rows_of<uint32_t>(base + src * page, base + dst * page, a.Hkv, head, bytes / 4);
}

// ---------------------------------------------------------------------------
// Releases, in three steps: what each request keeps, from the owners as they are;
// an owner less for every page dropped, whose count then is below 0 exactly if none is
// left; those pages onto the stack in their order.  Each step needs the whole of the
// one before: one workgroup where entries and pages are few (PG_FEW), else a launch to each, with
// a wave to a request.  Latency chains.
// ---------------------------------------------------------------------------

// Tokens that request i of ctx tokens keeps; -1 if that is refused.
__device__ __forceinline__ int kept(const protokv_page_release_args& a, int i, int ctx, int shift) {
  const int keep = min(max(a.keep[i], 0), ctx);
  if (keep < ctx && (keep & ((1 << shift) - 1))) {
    const int page = a.table[(size_t)i * a.table_stride + (keep >> shift)];
    if ((unsigned)page < (unsigned)a.num_pages && a.shares[page] > 0) return -1;
  }
  return keep;
}
__device__ __forceinline__ int pages_of(int tokens, int shift) { return (int)(((long long)tokens + (1 << shift) - 1) >> shift); }

__global__ __launch_bounds__(1024) void k_release_few(protokv_page_release_args a, int shift) {
  __shared__ int2 s_drop[PG_REQ];  // pages first .. end - 1 of a request
  __shared__ int s_sum[16];
  __shared__ int s_refused;
  const int tid = threadIdx.x, span = a.table_stride << shift;
  if (tid == 0) s_refused = 0;
  __syncthreads();
  for (int i = tid; i < a.num_requests; i += 1024) {
    const int ctx = min(max(a.ctx[i], 0), span);
    int keep = kept(a, i, ctx, shift);
    if (keep < 0) {
      keep = ctx;
      atomicAdd(&s_refused, 1);
    }
    a.ctx_out[i] = keep;
    s_drop[i] = make_int2(pages_of(keep, shift), pages_of(ctx, shift));
  }
  __syncthreads();
  const int all = a.num_requests * a.table_stride;
  for (int x0 = tid; x0 < all; x0 += 4096) {
    int page[4];  // four entries in flight
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int x = x0 + 1024 * k, i = x / a.table_stride, j = x - i * a.table_stride;
      const int2 d = x < all ? s_drop[i] : make_int2(0, 0);
      page[k] = j >= d.x && j < d.y ? a.table[x] : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((unsigned)page[k] < (unsigned)a.num_pages) atomicSub(&a.shares[page[k]], 1);
  }
  wait_vm<0>();  // this wave's are done
  __syncthreads();
  // a thread's pages lie together; read past the L1, which may hold them as they were
  const int per = (a.num_pages + 1023) / 1024, p0 = tid * per;
  uint32_t freed = 0;
#pragma unroll
  for (int k = 0; k < PG_FEW / 1024; ++k)
    if (k < per && p0 + k < a.num_pages)
      freed |= (__hip_atomic_load(&a.shares[p0 + k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) < 0 ? 1u : 0u) << k;
  int total;
  const int held = min(max(a.free_count[0], 0), a.num_pages);
  int at = held + block_sum(__popc(freed), s_sum, total) - __popc(freed);
  for (; freed; freed &= freed - 1, ++at) {
    const int page = p0 + __ffs(freed) - 1;
    a.shares[page] = 0;
    if (at < a.num_pages) a.free_pages[at] = page;
  }
  if (tid == 0) {
    a.free_count_out[0] = min(held + total, a.num_pages);
    a.refused[0] = s_refused;
  }
}

// scratch[b]: pages freed of the RL_PAGES from RL_PAGES b on
__global__ __launch_bounds__(1024) void k_release_keep(protokv_page_release_args a, int shift) {
  __shared__ int s_refused;
  const int span = a.table_stride << shift;
  if (threadIdx.x == 0) s_refused = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < a.num_requests; i += 1024) {
    const int ctx = min(max(a.ctx[i], 0), span);
    int keep = kept(a, i, ctx, shift);
    if (keep < 0) {
      keep = ctx;
      atomicAdd(&s_refused, 1);
    }
    a.ctx_out[i] = keep;
  }
  for (int b = threadIdx.x; b < (a.num_pages + RL_PAGES - 1) / RL_PAGES; b += 1024) a.scratch[b] = 0;
  __syncthreads();
  if (threadIdx.x == 0) a.refused[0] = s_refused;
}

constexpr int RL_BINS = 256;  // entries of scratch that a workgroup counts in its LDS first
__global__ __launch_bounds__(256) void k_release_drop(protokv_page_release_args a, int shift) {
  __shared__ int s_freed[RL_BINS];
  const int lane = threadIdx.x & 63, i = blockIdx.x * 4 + (threadIdx.x >> 6), span = a.table_stride << shift;
  const bool few = (a.num_pages + RL_PAGES - 1) / RL_PAGES <= RL_BINS;  // uniform
  s_freed[threadIdx.x] = 0;
  __syncthreads();
  if (i < a.num_requests) {
    const int ctx = min(max(a.ctx[i], 0), span);
    const int first = pages_of(a.ctx_out[i], shift), end = pages_of(ctx, shift);
    const int32_t* row = a.table + (size_t)i * a.table_stride;
    for (int j0 = first + lane; j0 < end; j0 += 256) {
      int page[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) page[k] = j0 + 64 * k < end ? row[j0 + 64 * k] : -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        // of a page's drops the one that finds no owner beyond itself is one alone
        if ((unsigned)page[k] < (unsigned)a.num_pages && atomicSub(&a.shares[page[k]], 1) == 0) {
          if (few) atomicAdd(&s_freed[page[k] / RL_PAGES], 1);
          else atomicAdd(&a.scratch[page[k] / RL_PAGES], 1);
        }
      }
    }
  }
  __syncthreads();
  if (few && s_freed[threadIdx.x]) atomicAdd(&a.scratch[threadIdx.x], s_freed[threadIdx.x]);
}

__global__ __launch_bounds__(1024) void k_release_collect(protokv_page_release_args a) {
  __shared__ int s_sum[2][16];
  const int tid = threadIdx.x, b = blockIdx.x;
  int before = 0, all;
  for (int w = tid; w < b; w += 1024) before += a.scratch[w];
  block_sum(before, s_sum[0], all);
  const int held = min(max(a.free_count[0], 0), a.num_pages);
  const int p0 = b * RL_PAGES + tid * 4;
  int sh[4], mine = 0;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    sh[k] = p0 + k < a.num_pages ? a.shares[p0 + k] : 0;
    mine += sh[k] < 0;
  }
  int total;
  int at = held + all + block_sum(mine, s_sum[1], total) - mine;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (sh[k] < 0) {
      a.shares[p0 + k] = 0;
      if (at < a.num_pages) a.free_pages[at] = p0 + k;
      ++at;
    }
  }
  if (b == (int)gridDim.x - 1 && tid == 0) a.free_count_out[0] = min(held + all + total, a.num_pages);
}

}  // namespace

template <int FP32, int U>
static void page4_rows(const Page4Rows& a, bool store, hipStream_t st) {
  constexpr unsigned per = 256 / (FP32 ? 32 : 16) * U;  // rows of a workgroup
  const dim3 wgs((unsigned)((a.rows + per - 1) / per)), threads(256);
  if (store) hipLaunchKernelGGL((k_page4_store<FP32, U>), wgs, threads, 0, st, a);
  else hipLaunchKernelGGL((k_page4_read<FP32, U>), wgs, threads, 0, st, a);
}

hipError_t launch_page4_rows(const Page4Rows& a, bool fp32, bool store, hipStream_t st) {
  // four pieces to a thread where one would take more than 8192 workgroups.  A store and the read of the same rows behind it,
  // 8 heads, one, two and four pieces: 18 432 tokens 50.2, 45.3 and 44.6 us, float32 91.0, 84.6 and 84.2, 8000 of float32
  // (16 000 workgroups) 33.6, 31.2 and 31.0; fewer are as long as the host's part of the two calls.  The kernels of
  // small calls: 64 tokens of 4 heads 2.4 + 2.3 with one, 3.5 + 2.7 with four, 2048 of 8 (2048 workgroups) 5.2 + 4.8 and
  // 6.6 + 5.3, 4608 8.8 + 9.2 and 9.7 + 8.5, 8000 13.3 + 14.3 and 14.7 + 12.9 (their rows not in a cache; the store
  // alone has nothing from more pieces there, the read has from about 4000 workgroups on)
  const bool many = a.rows * (fp32 ? 32 : 16) > 8192 * 256;
  if (fp32 && many) page4_rows<1, 4>(a, store, st);
  else if (fp32) page4_rows<1, 1>(a, store, st);
  else if (many) page4_rows<0, 4>(a, store, st);
  else page4_rows<0, 1>(a, store, st);
  return hipGetLastError();
}

hipError_t launch_page_fork(const protokv_page_fork_args& a, hipStream_t st) {
  const int shift = 31 - __builtin_clz((unsigned)a.page_size);
  if (a.num_forks <= PG_REQ && (long long)a.num_forks * a.table_stride <= PG_FEW) {
    hipLaunchKernelGGL((k_page_fork<1>), dim3(1), dim3(FK_NT), 0, st, a, shift);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((k_page_fork<0>), dim3(1), dim3(FK_NT), 0, st, a, shift);
  const unsigned parts = std::min((a.table_stride + 255u) / 256u, 64u);
  hipLaunchKernelGGL(k_page_fork_rows, dim3(parts, a.num_forks), dim3(256), 0, st, a, shift);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PageCopy& a, int copies, int layers, unsigned parts, hipStream_t st) {
  hipLaunchKernelGGL(k_page_copy, dim3(copies, parts, layers), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_release(const protokv_page_release_args& a, hipStream_t st) {
  const int shift = 31 - __builtin_clz((unsigned)a.page_size);
  if (a.num_requests <= PG_REQ && (long long)a.num_requests * a.table_stride <= PG_FEW && a.num_pages <= PG_FEW) {
    hipLaunchKernelGGL(k_release_few, dim3(1), dim3(1024), 0, st, a, shift);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(k_release_keep, dim3(1), dim3(1024), 0, st, a, shift);
  hipLaunchKernelGGL(k_release_drop, dim3((a.num_requests + 3) / 4), dim3(256), 0, st, a, shift);
  hipLaunchKernelGGL(k_release_collect, dim3((a.num_pages + RL_PAGES - 1) / RL_PAGES), dim3(1024), 0, st, a);
  return hipGetLastError();
}

}  // namespace pkv
