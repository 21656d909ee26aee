// Rotary positions of several axes and block tables (protokv_rotate,
// protokv_page_plan) for gfx950.
#include "exact.h"
#include "pkv_internal.h"
#include "rope.h"

namespace pkv {

namespace {

// ---------------------------------------------------------------------------
// Rotary positions: bound by the rows' bytes.  One wave takes 1 / parts of a
// token's heads (4608 tokens of 32 + 8 + 8 bf16 heads, stored to pages: 20.4 us,
// 5.5 TB/s, float32 37.5 us, 6.0; one token 2.8 us): lane i
// forms the (cos, sin) of pair i once (angle and reduction in float64), hands
// them round through LDS, and then eight lanes at a time turn a head: lane c of
// eight holds dims 8 c .. + 7 and their partners 64 + 8 c .. + 7.  Heads are
// numbered queries, keys, values (copied to their slots).
// ---------------------------------------------------------------------------
template <int FP32>
struct Vec8;  // eight dims of kv dtype as loaded
template <>
struct Vec8<0> {
  uint4 w;
  __device__ __forceinline__ float get(int i) const {
    const uint32_t u = i < 2 ? w.x : i < 4 ? w.y : i < 6 ? w.z : w.w;
    return __uint_as_float(i & 1 ? u & 0xFFFF0000u : u << 16);
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(uint32_t, (bf16x2){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
    w = make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <>
struct Vec8<1> {
  float4 a, b;
  __device__ __forceinline__ float get(int i) const {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return x[i];
  }
  __device__ __forceinline__ void set(const float (&x)[8]) {
    a = make_float4(x[0], x[1], x[2], x[3]);
    b = make_float4(x[4], x[5], x[6], x[7]);
  }
};

template <int FP32>
__global__ __launch_bounds__(256) void k_rotate(RotateArgs a) {
  constexpr int ES = FP32 ? 4 : 2;
  typedef Vec8<FP32> V;
  __shared__ __attribute__((aligned(16))) float s_cs[4][D];  // (cos, sin) of every pair
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const long long item = (long long)blockIdx.x * 4 + wave;
  const int t = (int)(item / a.parts), part = (int)(item % a.parts);
  if (t >= a.N) return;  // uniform, and nothing below synchronises waves
  {
    float c, s;
    rope_cs((double)a.pos[a.axis[lane] * a.ps + t], a.inv[lane], c, s);
    s_cs[wave][2 * lane] = c;
    s_cs[wave][2 * lane + 1] = s;
  }
  const int c8 = lane & 7;
  long long slot = -1;
  if (a.nslots) {
    slot = a.slots[t];
    if (slot >= a.nslots) slot = -1;
  }
  const long long page = slot >> a.shift, off = slot & ((1 << a.shift) - 1);
  asm volatile("" ::: "memory");  // the wave's LDS operations run in order
  float cs[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) cs[i] = s_cs[wave][c8 * 16 + i];
  const int heads = a.Hq + a.Hkv + (slot >= 0 ? a.Hkv : 0);
  for (int h = part * 8 + (lane >> 3); h < heads; h += a.parts * 8) {
    const int kh = h - a.Hq, vh = kh - a.Hkv;
    const uint8_t* src = h < a.Hq ? a.q + t * a.qs + (size_t)h * (D * ES)
                         : vh < 0 ? a.k + t * a.ks + (size_t)kh * (D * ES)
                                  : a.v + t * a.vs + (size_t)vh * (D * ES);
    V lo = reinterpret_cast<const V*>(src)[c8], hi = reinterpret_cast<const V*>(src + D / 2 * ES)[c8];
    if (vh < 0) {
      float x[8], y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) rope_pair(lo.get(i), hi.get(i), cs[2 * i], cs[2 * i + 1], x[i], y[i]);
      lo.set(x);
      hi.set(y);
    }
    auto put = [&](uint8_t* dst) {
      reinterpret_cast<V*>(dst)[c8] = lo;
      reinterpret_cast<V*>(dst + D / 2 * ES)[c8] = hi;
    };
    if (h < a.Hq) {
      put(a.qo + t * a.qos + (size_t)h * (D * ES));
    } else {
      const int hk = vh < 0 ? kh : vh;
      if (vh < 0 && a.ko) put(a.ko + t * a.kos + (size_t)kh * (D * ES));
      if (slot >= 0)
        put((vh < 0 ? a.kp : a.vp) + ((((page * a.Hkv + hk) << a.shift) + off)) * (size_t)(D * ES));
    }
  }
}

// ---------------------------------------------------------------------------
// Block tables and slot maps.  Everything follows from three running sums over
// the requests: pages given back, rows, pages taken.  Each workgroup forms them
// for all requests in its LDS (a few us; no second launch, nothing to wait for),
// then the workgroups share the pages given back, the pages taken and the rows,
// each of which finds its request by a search in the sums.  Sums saturate at
// PL_MAX, which no valid total reaches.  What bounds it is the chain of loads,
// barriers and the search: 64 requests 3.5 us, 1500 11.2.
// ---------------------------------------------------------------------------
constexpr int PL_MAX = (1 << 30) - 1;  // two of them fit an int

__device__ __forceinline__ int sat_add(int x, int y) { return min(x + y, PL_MAX); }

// Inclusive running sums over the workgroup's threads of x and y (each 0 ..
// PL_MAX); tx, ty: of all.  s: 2 NT / 64 words, free again two calls later with
// another one in between.  One barrier.
template <int NT>
__device__ __forceinline__ void block_sums(int& x, int& y, int* s, int& tx, int& ty) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  // running sums of the wave: within rows of 16 lanes, then over the rows (row_bcast)
#define PL_STEP(ctrl, rows)                                                     \
  x = sat_add(x, __builtin_amdgcn_update_dpp(0, x, ctrl, rows, 0xf, false));    \
  y = sat_add(y, __builtin_amdgcn_update_dpp(0, y, ctrl, rows, 0xf, false));
  PL_STEP(0x111, 0xf)
  PL_STEP(0x112, 0xf)
  PL_STEP(0x114, 0xf)
  PL_STEP(0x118, 0xf)
  PL_STEP(0x142, 0xa)
  PL_STEP(0x143, 0xc)
#undef PL_STEP
  if (lane == 63) {
    s[2 * wave] = x;
    s[2 * wave + 1] = y;
  }
  __syncthreads();
  int bx = 0, by = 0;
  tx = ty = 0;
#pragma unroll
  for (int w = 0; w < NT / 64; ++w) {
    const int u = s[2 * w], v = s[2 * w + 1];
    if (w < wave) {
      bx = sat_add(bx, u);
      by = sat_add(by, v);
    }
    tx = sat_add(tx, u);
    ty = sat_add(ty, v);
  }
  x = sat_add(bx, x);
  y = sat_add(by, y);
}

// Largest i in [0, n) with s[i] <= x (s non-decreasing, s[0] <= x).
__device__ __forceinline__ int find_at(const int* s, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// NMAX: requests at most; KEEP: their lengths stay in LDS (else they are read anew).
template <int NMAX, int NT, bool KEEP>
__global__ __launch_bounds__(NT) void k_page_plan(protokv_page_plan_args a, int shift) {
  __shared__ int s_row[NMAX + 1];   // first row
  __shared__ int s_back[NMAX + 1];  // pages given back before request i
  __shared__ int s_take[NMAX + 1];  // pages asked for before request i
  __shared__ int s_ctx[KEEP ? NMAX : 1], s_add[KEEP ? NMAX : 1];
  __shared__ int s_sum[3][2 * NT / 64];
  const int tid = threadIdx.x, n = a.num_requests, P1 = (1 << shift) - 1;
  const int span = a.table_stride << shift;  // tokens of a table row
  const int free0 = min(max(a.free_count[0], 0), a.num_pages);
  auto read_ctx = [&](int i) { return min(max(a.ctx[i], 0), span); };
  auto ctx_of = [&](int i) { return KEEP ? s_ctx[i] : read_ctx(i); };
  auto add_of = [&](int i) { return KEEP ? s_add[i] : a.add[i]; };
  auto pages_of = [&](long long x) { return (int)((x + P1) >> shift); };
  // pages that a request lacks, or -1 if it cannot be granted whatever the stack holds
  auto lacks = [&](int ctx, int add, int end) {
    if ((long long)ctx + add > span || end > a.max_tokens) return -1;
    return pages_of((long long)ctx + add) - pages_of(ctx);
  };
  int rows = 0, back = 0, take = 0, turn = 0;  // of the requests so far
  for (int i0 = 0; i0 < n; i0 += NT) {
    const int i = i0 + tid;
    int add = 0, ctx = 0;
    if (i < n) {
      add = a.add[i];
      ctx = read_ctx(i);
    }
    int tx, ty;
    int end = min(max(add, 0), PL_MAX), gave = add < 0 ? pages_of(ctx) : 0;
    block_sums<NT>(end, gave, s_sum[turn], tx, ty);
    turn = turn == 2 ? 0 : turn + 1;
    end = sat_add(rows, end);
    gave = sat_add(back, gave);
    rows = sat_add(rows, tx);
    back = sat_add(back, ty);
    int upto = add > 0 ? max(lacks(ctx, add, end), 0) : 0, none = 0;
    block_sums<NT>(upto, none, s_sum[turn], tx, ty);
    turn = turn == 2 ? 0 : turn + 1;
    upto = sat_add(take, upto);
    take = sat_add(take, tx);
    if (i < n) {
      s_row[i + 1] = end;
      s_back[i + 1] = gave;
      s_take[i + 1] = upto;
      if constexpr (KEEP) {
        s_ctx[i] = ctx;
        s_add[i] = add;
      }
    }
  }
  if (tid == 0) s_row[0] = s_back[0] = s_take[0] = 0;
  __syncthreads();
  const int nfree = min(free0 + back, a.num_pages);  // on the stack once pages are back
  auto granted = [&](int i, int ctx, int add) {
    if (add == 0) return true;
    if (add < 0) return false;
    const int need = lacks(ctx, add, s_row[i + 1]);
    return need == 0 || (need > 0 && s_take[i + 1] <= nfree);
  };
  // page at place x of the stack once pages are back
  auto stacked = [&](int x) {
    if (x < free0) return a.free_pages[x];
    const int i = find_at(s_back, n, x - free0);
    return a.table[(size_t)i * a.table_stride + (x - free0 - s_back[i])];
  };
  // page j of request i, which lacks the pages from `held` on
  auto taken = [&](int i, int j, int held) { return stacked(nfree - 1 - (s_take[i] + j - held)); };

  // one row, one page taken or one page given back to a thread at a time
  const int ntake = min(take, nfree), nback = nfree - free0;
  const long long all = (long long)a.max_tokens + ntake + nback;
  for (long long w = (long long)blockIdx.x * NT + tid; w < all; w += (long long)gridDim.x * NT) {
    if (w < a.max_tokens) {
      const int t = (int)w;
      int slot = -1, pos = 0;
      if (t < rows) {
        const int i = find_at(s_row, n, t);
        const int ctx = ctx_of(i), held = pages_of(ctx);
        const long long p = (long long)ctx + (t - s_row[i]);
        pos = (int)(p + (a.base ? a.base[i] : 0));
        if (granted(i, ctx, add_of(i))) {
          const int j = (int)(p >> shift);
          const int page = j < held ? a.table[(size_t)i * a.table_stride + j] : taken(i, j, held);
          if ((unsigned)page < (unsigned)a.num_pages) slot = (page << shift) + (int)(p & P1);
        }
      }
      a.slots[t] = slot;
      if (a.positions) a.positions[t] = pos;
    } else if (w < (long long)a.max_tokens + ntake) {
      const int x = (int)(w - a.max_tokens), i = find_at(s_take, n, x);
      const int ctx = ctx_of(i), held = pages_of(ctx);
      if (granted(i, ctx, add_of(i))) {
        const int j = held + x - s_take[i];
        a.table[(size_t)i * a.table_stride + j] = taken(i, j, held);
      }
    } else {
      const int x = (int)(w - a.max_tokens - ntake);
      a.free_pages[free0 + x] = stacked(free0 + x);
    }
  }
  if (blockIdx.x != 0) return;
  // lengths; the pages of the granted requests and the count of the others.  Pages
  // are granted from the front: the largest running sum of a granted request with
  // pages of its own.
  __syncthreads();  // s_sum is free
  int* s_end = s_sum[0];
  if (tid < 2) s_end[tid] = 0;
  __syncthreads();
  int used = 0, refused = 0;
  for (int i = tid; i < n; i += NT) {
    const int ctx = ctx_of(i), add = add_of(i);
    const bool ok = granted(i, ctx, add);
    a.kv_len[i] = ok ? ctx + add : 0;
    a.cu[i + 1] = min(s_row[i + 1], a.max_tokens);
    if (ok && s_take[i + 1] > s_take[i]) used = max(used, s_take[i + 1]);
    refused += add > 0 && !ok;
  }
  if (used) atomicMax(&s_end[0], used);
  if (refused) atomicAdd(&s_end[1], refused);
  __syncthreads();
  if (tid == 0) {
    a.cu[0] = 0;
    a.free_count_out[0] = nfree - s_end[0];
    if (a.refused) a.refused[0] = s_end[1];
  }
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& a, bool fp32, hipStream_t st) {
  const unsigned blocks = (unsigned)(((long long)a.N * a.parts + 3) / 4);
  if (fp32) hipLaunchKernelGGL((k_rotate<1>), dim3(blocks), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_rotate<0>), dim3(blocks), dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_page_plan(const protokv_page_plan_args& a, hipStream_t st) {
  const int shift = 31 - __builtin_clz((unsigned)a.page_size);
  // about a row or page a thread (every request may take or give some), at most 64
  // workgroups (each forms the sums of all requests); for few requests a workgroup of
  // four waves, whose barriers are short
  auto blocks = [&](int threads) {
    const long long b = ((long long)a.max_tokens + 4ll * a.num_requests + threads - 1) / threads;
    return dim3((unsigned)(b < 64 ? b : 64));
  };
  if (a.num_requests <= 256)
    hipLaunchKernelGGL((k_page_plan<256, 256, true>), blocks(256), dim3(256), 0, st, a, shift);
  else if (a.num_requests <= 2048)
    hipLaunchKernelGGL((k_page_plan<2048, 1024, true>), blocks(1024), dim3(1024), 0, st, a, shift);
  else
    hipLaunchKernelGGL((k_page_plan<MAX_REQUESTS, 1024, false>), blocks(1024), dim3(1024), 0, st, a, shift);
  return hipGetLastError();
}

}  // namespace pkv
