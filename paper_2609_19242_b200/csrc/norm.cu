// Layer norm and root-mean-square norm of a residual stream, forward and backward (include/bdlm_norm.h).
//
// Both passes are streams over the [T, D] tensors, bound by memory: 4 T D elements each (x, residual, y, h; dy, h, dh, dx).  A row
// is in registers from its load to its store, so each element is read and written once, and the variance is the sum of squares
// around the mean that has been formed, not a difference of two large sums.  A row belongs to `tpr` threads: a whole CTA
// where it has more than 128 vectors of 16 bytes, otherwise a warp or a power-of-two part of one, so that short rows fill the lanes.
// Rows whose length is no multiple of a vector start anywhere and go element by element.
#include <math.h>

#include "../../include/bdlm_norm.h"
#include "elem_common.cuh"

namespace bdlm {
namespace {

struct NormArgs {
  const void *x, *res, *w, *b;     // forward; backward: dy, dh, weight
  const void* h_in;                // backward
  void *y, *h;                     // forward; backward: dx
  float *mean, *rstd;
  float* part;                     // backward: [dweight, dbias][groups][D], nullptr: neither is wanted
  int T, D, nvec, tpr, rms;
  float eps, inv_d;
};

constexpr int RED_FLOATS = 2 * 32 * 2;   // two buffers in turn, 32 warps, two sums

// Items a thread: few, so that weights, sums and the next row's vectors fit its registers beside the row's; for rows that would
// need more than 512 threads of those, most_items of them, weights read again for each row and the backward's sums in shared memory.
__host__ __device__ constexpr int mid_items(int V) { return V == 1 ? 4 : 2; }
__host__ __device__ constexpr int most_items(int V) { return V == 1 ? 16 : 4; }
__host__ __device__ constexpr bool big(int V, int items, bool wide) { return wide && items == most_items(V); }
__host__ __device__ constexpr int max_threads(int V, int items, bool wide) { return !wide ? 128 : big(V, items, wide) && V < 8 ? 1024 : 512; }

// Sums over the threads of a row; every thread gets them.  The order is fixed.
template <bool WIDE, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], int tpr, float* red, int& turn) {
  const int top = WIDE ? 16 : tpr / 2;
  for (int s = top; s > 0; s >>= 1) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], s);
  }
  if (!WIDE) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
  float* at = red + turn * 64;
  turn ^= 1;   // (a buffer is written again only after the barrier of the other one's use)
  if (lane == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) at[warp * 2 + n] = v[n];
  }
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = lane < warps ? at[lane * 2 + n] : 0.f;
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], s);
  }
}

template <class T, class W, int V, int ITEMS, bool WIDE>
__global__ void __launch_bounds__(max_threads(V, ITEMS, WIDE)) norm_fwd_kernel(const NormArgs a) {
  constexpr bool BIG = big(V, ITEMS, WIDE);
  __shared__ float red[RED_FLOATS];
  const int tpr = WIDE ? (int)blockDim.x : a.tpr, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x % tpr;
  const int rows = WIDE ? 1 : (int)blockDim.x / tpr, sub = WIDE ? 0 : (int)threadIdx.x / tpr;
  int turn = 0;
  const T *x = static_cast<const T*>(a.x), *res = static_cast<const T*>(a.res);
  T *y = static_cast<T*>(a.y), *h = static_cast<T*>(a.h);
  Raw<W, V> w[BIG ? 1 : ITEMS], b[BIG ? 1 : ITEMS];   // of this thread's columns, for all its rows
  auto load_weight = [&](int i, int at) {
    const int c = lane + i * tpr;
    w[at].clear(); b[at].clear();
    if (c < a.nvec && a.w != nullptr) w[at].load(static_cast<const W*>(a.w) + (int64_t)c * V);
    if (c < a.nvec && a.b != nullptr) b[at].load(static_cast<const W*>(a.b) + (int64_t)c * V);
  };
  if (!BIG) {
#pragma unroll
    for (int i = 0; i < (BIG ? 1 : ITEMS); ++i) load_weight(i, i);
  }
  for (int64_t r0 = (int64_t)blockIdx.x * rows; r0 < a.T; r0 += (int64_t)gridDim.x * rows) {
    const int64_t row = r0 + sub;
    const bool ok = row < a.T;
    float f[ITEMS][V], s[1] = {0.f};
    Raw<T, V> rx[ITEMS], rr[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = lane + i * tpr;
      rx[i].clear(); rr[i].clear();
      if (ok && c < a.nvec) {
        rx[i].load(x + row * a.D + (int64_t)c * V);
        if (res != nullptr) rr[i].load(res + row * a.D + (int64_t)c * V);
      }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = lane + i * tpr;
      rx[i].get(f[i]);
      if (res != nullptr) {   // the sum as it is stored is what is normalised
        float g[V];
        rr[i].get(g);
#pragma unroll
        for (int e = 0; e < V; ++e) f[i][e] += g[e];
        rx[i].put(f[i]);
        rx[i].get(f[i]);
        if (ok && c < a.nvec) rx[i].store(h + row * a.D + (int64_t)c * V);
      }
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += f[i][e];
    }
    float mean = 0.f;
    if (!a.rms) {
      row_sum<WIDE>(s, tpr, red, turn);
      mean = s[0] * a.inv_d;
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (lane + i * tpr < a.nvec) {
#pragma unroll
        for (int e = 0; e < V; ++e) { const float t = f[i][e] - mean; s[0] = fmaf(t, t, s[0]); }
      }
    }
    row_sum<WIDE>(s, tpr, red, turn);
    const float rstd = rsqrtf(fmaf(s[0], a.inv_d, a.eps));
    if (ok && lane == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = lane + i * tpr;
      float wf[V], bf[V];
      if (BIG) load_weight(i, 0);
      w[BIG ? 0 : i].get(wf);
      b[BIG ? 0 : i].get(bf);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float n = (f[i][e] - mean) * rstd;
        f[i][e] = a.w != nullptr ? fmaf(n, wf[e], bf[e]) : n;
      }
      rx[i].put(f[i]);
      if (ok && c < a.nvec) rx[i].store(y + row * a.D + (int64_t)c * V);
    }
  }
}

// A thread keeps the sums for dweight and dbias of its columns over all its rows, so the columns' sums cost no traffic but one
// row of partial sums per CTA.  These sums take the registers that would hold loads in flight, so where a CTA has a row, the
// rows to come are copied to shared memory asynchronously, RING of them; a thread reads what it has copied itself and
// needs no barrier for it.  Elsewhere the next row's vectors are requested into registers before this one's sums are joined.
constexpr int RING = 4;
__device__ __forceinline__ void copy16(void* to, const void* from) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end_row() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_wait_first() { asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory"); }
// (16-byte vectors of rows that take a CTA, as long as the ring fits)
__host__ __device__ constexpr bool ringed(int V, int items, bool wide) { return wide && V > 1 && !big(V, items, wide); }
template <class T, class W, int V, int ITEMS, bool WIDE>
__global__ void __launch_bounds__(max_threads(V, ITEMS, WIDE)) norm_bwd_kernel(const NormArgs a) {
  constexpr bool BIG = big(V, ITEMS, WIDE), RINGED = ringed(V, ITEMS, WIDE);
  constexpr int KEEP = BIG ? 1 : ITEMS;
  __shared__ float red[RED_FLOATS];
  // rows in flight: [row][dy, h, dh][item][thread] vectors;  short rows: the CTA's groups of rows join their sums here; long ones: the sums themselves, [dweight, dbias][item, element][thread]
  extern __shared__ float comb[];
  const int tpr = WIDE ? (int)blockDim.x : a.tpr, lane = WIDE ? (int)threadIdx.x : (int)threadIdx.x % tpr;
  const int rows = WIDE ? 1 : (int)blockDim.x / tpr, sub = WIDE ? 0 : (int)threadIdx.x / tpr;
  int turn = 0;
  const T *dy = static_cast<const T*>(a.x), *h = static_cast<const T*>(a.h_in), *dh = static_cast<const T*>(a.res);
  T* dx = static_cast<T*>(a.y);
  Raw<W, V> w[KEEP];
  auto load_weight = [&](int i, int at) {
    const int c = lane + i * tpr;
    w[at].clear();
    if (c < a.nvec && a.w != nullptr) w[at].load(static_cast<const W*>(a.w) + (int64_t)c * V);
  };
  float dw[KEEP][V], db[KEEP][V];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (!BIG) load_weight(i, BIG ? 0 : i);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if (!BIG) { dw[BIG ? 0 : i][e] = 0.f; db[BIG ? 0 : i][e] = 0.f; }
      else if (a.part != nullptr) {
        comb[(i * V + e) * tpr + lane] = 0.f;
        comb[((ITEMS + i) * V + e) * tpr + lane] = 0.f;
      }
    }
  }
  Raw<T, V> ry[ITEMS], rh[ITEMS], rd[KEEP];
  float mean = 0.f, rstd = 0.f;
  uint4* ring = reinterpret_cast<uint4*>(comb);
  auto ring_at = [&](int slot, int tensor, int i) { return ring + ((slot * 3 + tensor) * ITEMS + i) * tpr + lane; };
  auto copy_row = [&](int64_t row, int slot) {
    if (row < a.T) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int c = lane + i * tpr;
        if (c < a.nvec) {
          copy16(ring_at(slot, 0, i), dy + row * a.D + (int64_t)c * V);
          copy16(ring_at(slot, 1, i), h + row * a.D + (int64_t)c * V);
          if (dh != nullptr) copy16(ring_at(slot, 2, i), dh + row * a.D + (int64_t)c * V);
        }
      }
    }
    copies_end_row();   // (an empty group where there is no row: the groups count rows)
  };
  auto request = [&](int64_t row) {
    const bool ok = row < a.T;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (RINGED) continue;
      const int c = lane + i * tpr;
      ry[i].clear(); rh[i].clear();
      if (!BIG) rd[BIG ? 0 : i].clear();
      if (ok && c < a.nvec) {
        ry[i].load(dy + row * a.D + (int64_t)c * V);
        rh[i].load(h + row * a.D + (int64_t)c * V);
        if (!BIG && dh != nullptr) rd[BIG ? 0 : i].load(dh + row * a.D + (int64_t)c * V);
      }
    }
    mean = ok && a.mean != nullptr ? a.mean[row] : 0.f;
    rstd = ok ? a.rstd[row] : 0.f;
  };
  const int64_t step = (int64_t)gridDim.x * rows;
  int64_t r0 = (int64_t)blockIdx.x * rows;
  if (RINGED) {
    for (int k = 0; k < RING; ++k) copy_row(r0 + k * step, k);
  }
  request(r0 + sub);
  for (int slot = 0; r0 < a.T; r0 += step, slot = slot + 1 == RING ? 0 : slot + 1) {
    const int64_t row = r0 + sub;
    if (RINGED) {
      copies_wait_first();
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        ry[i].clear(); rh[i].clear(); rd[BIG ? 0 : i].clear();
        if (lane + i * tpr < a.nvec) {
          ry[i].load(reinterpret_cast<const T*>(ring_at(slot, 0, i)));
          rh[i].load(reinterpret_cast<const T*>(ring_at(slot, 1, i)));
          if (dh != nullptr) rd[BIG ? 0 : i].load(reinterpret_cast<const T*>(ring_at(slot, 2, i)));
        }
      }
      copy_row(row + RING * step, slot);   // (after this thread's own reads of the slot)
    }
    const bool ok = row < a.T;
    const float mu = mean, rs = rstd;
    // g and n of an item, formed twice: as vectors of the element type they take half the registers across the joining of the sums
    Raw<T, V> cy[ITEMS], ch[ITEMS], cd[KEEP];
    auto form = [&](int i, float (&y)[V], float (&g)[V], float (&n)[V]) {
      float wf[V];
      if (BIG) load_weight(i, 0);
      cy[i].get(y);
      ch[i].get(n);
      w[BIG ? 0 : i].get(wf);
      const bool in = lane + i * tpr < a.nvec;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        n[e] = in ? (n[e] - mu) * rs : 0.f;
        g[e] = a.w != nullptr ? y[e] * wf[e] : y[e];
      }
    };
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float y[V], g[V], n[V];
      cy[i] = ry[i]; ch[i] = rh[i];
      if (!BIG) cd[BIG ? 0 : i] = rd[BIG ? 0 : i];
      form(i, y, g, n);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        s[0] = fmaf(g[e], n[e], s[0]);
        s[1] += g[e];
        if (!BIG) {
          dw[BIG ? 0 : i][e] = fmaf(y[e], n[e], dw[BIG ? 0 : i][e]);
          db[BIG ? 0 : i][e] += y[e];
        } else if (a.part != nullptr) {
          float *at = comb + (i * V + e) * tpr + lane, *at_b = at + ITEMS * V * tpr;
          *at = fmaf(y[e], n[e], *at);
          *at_b += y[e];
        }
      }
    }
    if (!BIG) request(row + step);
    row_sum<WIDE>(s, tpr, red, turn);
    const float c2 = s[0] * a.inv_d, c1 = a.rms ? 0.f : s[1] * a.inv_d;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = lane + i * tpr;
      float y[V], g[V], n[V], d[V];
      form(i, y, g, n);
      if (BIG) {
        cd[0].clear();
        if (dh != nullptr && c < a.nvec) cd[0].load(dh + row * a.D + (int64_t)c * V);
      }
      cd[BIG ? 0 : i].get(d);
#pragma unroll
      for (int e = 0; e < V; ++e) d[e] = fmaf(rs, g[e] - c1 - n[e] * c2, d[e]);
      Raw<T, V> o;
      o.put(d);
      if (ok && c < a.nvec) o.store(dx + row * a.D + (int64_t)c * V);
    }
    if (BIG) request(row + step);
  }
  if (a.part == nullptr) return;
  if (WIDE) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = lane + i * tpr;
      if (c < a.nvec) {
        float* at = a.part + (int64_t)blockIdx.x * a.D + (int64_t)c * V;
        float* at_b = at + (int64_t)gridDim.x * a.D;
#pragma unroll
        for (int e = 0; e < V; ++e) {
          at[e] = BIG ? comb[(i * V + e) * tpr + lane] : dw[BIG ? 0 : i][e];
          at_b[e] = BIG ? comb[((ITEMS + i) * V + e) * tpr + lane] : db[BIG ? 0 : i][e];
        }
      }
    }
  } else {
    const int cols = tpr * ITEMS * V;   // of which D are there
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) comb[sub * cols + (lane + i * tpr) * V + e] = which ? db[BIG ? 0 : i][e] : dw[BIG ? 0 : i][e];
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += blockDim.x) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += comb[r * cols + c];
        a.part[((int64_t)which * gridDim.x + blockIdx.x) * a.D + c] = s;
      }
    }
  }
}

// dweight and dbias from the CTAs' partial sums (blockIdx.y: which of the two): 32 columns a CTA, its warps take the groups in turn.
constexpr int WG_WARPS = 16;
template <class W>
__global__ void __launch_bounds__(WG_WARPS * 32) norm_wgrad_kernel(const float* part, int groups, int D, W* dweight, W* dbias) {
  __shared__ float sums[WG_WARPS][33];
  wait_for_predecessor();
  W* out = blockIdx.y == 0 ? dweight : dbias;
  if (out == nullptr) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = blockIdx.x * 32 + lane;
  const float* at = part + (int64_t)blockIdx.y * groups * D + c;
  float s = 0.f;
  if (c < D) {
#pragma unroll 8
    for (int g = warp; g < groups; g += WG_WARPS) s += at[(int64_t)g * D];
  }
  sums[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < D) {
#pragma unroll
    for (int k = 1; k < WG_WARPS; ++k) s += sums[k][lane];
    out[c] = W(s);
  }
}

// ------------------------------------------------------------------------------------------------ host
constexpr int MAX_GROUPS = 592;   // CTAs of a backward: four on each of 148 SMs

// How a row is laid over threads: V elements a vector, `items` vectors a thread.
struct Layout { int vec, nvec, items, tpr, threads; bool wide; };
Layout layout(const bdlm_norm_params* p) {
  const int full = p->dtype == BDLM_FP32 ? 4 : 8;
  Layout l;
  l.vec = p->D % full == 0 ? full : 1;
  l.nvec = p->D / l.vec;
  const int most = most_items(l.vec), mid = mid_items(l.vec);
  l.wide = l.nvec > 128;
  if (!l.wide) {
    l.tpr = 1;
    while (l.tpr < 32 && l.tpr < l.nvec) l.tpr *= 2;
    l.items = l.nvec <= 32 ? 1 : l.nvec <= 32 * mid ? mid : most;
    l.threads = 128;
  } else {
    l.items = l.nvec <= 512 * mid ? mid : most;
    l.threads = l.tpr = ((l.nvec + l.items - 1) / l.items + 31) / 32 * 32;
  }
  return l;
}
int64_t blocks_for_rows(const bdlm_norm_params* p, const Layout& l) {
  const int rows = l.wide ? 1 : l.threads / l.tpr;
  return ((int64_t)p->T + rows - 1) / rows;
}
int bwd_groups(const bdlm_norm_params* p, const Layout& l) {
  const int per_sm = l.threads <= 128 ? 4 : l.threads <= 256 ? 2 : 1;
  const int64_t want = blocks_for_rows(p, l), cap = MAX_GROUPS / 4 * per_sm;
  return (int)(want < cap ? want : cap);
}

int check(const bdlm_norm_params* p) {
  if (p == nullptr || p->T < 0 || p->D <= 0) return BDLM_ERR_INVALID_ARG;
  if (p->dtype < BDLM_BF16 || p->dtype > BDLM_FP32 || (p->wdtype != p->dtype && p->wdtype != BDLM_FP32)) return BDLM_ERR_INVALID_ARG;
  if (p->kind != BDLM_NORM_LAYER && p->kind != BDLM_NORM_RMS) return BDLM_ERR_INVALID_ARG;
  if (!(p->eps >= 0.f) || isinf(p->eps) || p->reserved[0] != 0 || p->reserved[1] != 0) return BDLM_ERR_INVALID_ARG;
  if (p->D > BDLM_NORM_MAX_D) return BDLM_ERR_UNSUPPORTED;
  return BDLM_OK;
}
bool al(const void* x, unsigned bytes) { return (reinterpret_cast<uintptr_t>(x) & (bytes - 1)) == 0; }
bool sm100() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  return cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess && major == 10;
}

// Calls f(T, W, V, ITEMS, WIDE) with the call's types and layout as template arguments.
template <int N> using Int = std::integral_constant<int, N>;
template <class T> struct Type { using type = T; };
template <class F>
void by_layout(const bdlm_norm_params* p, const Layout& l, F f) {
  auto by_items = [&](auto t, auto w, auto v) {
    constexpr int M = decltype(v)::value == 1 ? 4 : 2;
    auto by_width = [&](auto items) {
      if (l.wide) f(t, w, v, items, std::true_type{});
      else f(t, w, v, items, std::false_type{});
    };
    if (l.items == 1) f(t, w, v, Int<1>{}, std::false_type{});
    else if (l.items == M) by_width(Int<M>{});
    else by_width(Int<4 * (M / 2) * (M / 2)>{});
  };
  auto by_vec = [&](auto t, auto w) {
    constexpr int FULL = sizeof(typename decltype(t)::type) == 4 ? 4 : 8;
    if (l.vec == 1) by_items(t, w, Int<1>{});
    else by_items(t, w, Int<FULL>{});
  };
  auto by_weight = [&](auto t) {
    if (p->wdtype == BDLM_FP32) by_vec(t, Type<float>{});
    else by_vec(t, t);
  };
  if (p->dtype == BDLM_BF16) by_weight(Type<bf16_t>{});
  else if (p->dtype == BDLM_FP16) by_weight(Type<__half>{});
  else by_vec(Type<float>{}, Type<float>{});
}

}  // namespace
}  // namespace bdlm

using namespace bdlm;

extern "C" {

size_t bdlm_norm_workspace_bytes(const bdlm_norm_params* p) {
  if (check(p) != BDLM_OK) return 0;
  const size_t groups = (size_t)bwd_groups(p, layout(p));
  return 2 * groups * p->D * sizeof(float);
}

int bdlm_norm_fwd(const bdlm_norm_params* p, const void* x, const void* residual, const void* weight, const void* bias,
                  void* y, void* h, float* mean, float* rstd, void* cuda_stream) {
  const int rc = check(p);
  if (rc != BDLM_OK) return rc;
  if (p->T > 0 && (x == nullptr || y == nullptr)) return BDLM_ERR_INVALID_ARG;
  if (p->T > 0 && (residual != nullptr) != (h != nullptr)) return BDLM_ERR_INVALID_ARG;
  if ((bias != nullptr && weight == nullptr) || (mean != nullptr && p->kind == BDLM_NORM_RMS)) return BDLM_ERR_INVALID_ARG;
  const void* ptrs[] = {x, residual, weight, bias, y, h};
  for (const void* q : ptrs) if (!al(q, 16)) return BDLM_ERR_INVALID_ARG;
  if (!al(mean, 4) || !al(rstd, 4)) return BDLM_ERR_INVALID_ARG;
  if (!sm100()) return BDLM_ERR_UNSUPPORTED;
  if (p->T == 0) return BDLM_OK;
  const Layout l = layout(p);
  NormArgs a = {};
  a.x = x; a.res = residual; a.w = weight; a.b = bias; a.y = y; a.h = h; a.mean = mean; a.rstd = rstd;
  a.T = p->T; a.D = p->D; a.nvec = l.nvec; a.tpr = l.tpr; a.rms = p->kind == BDLM_NORM_RMS; a.eps = p->eps;
  a.inv_d = (float)(1.0 / p->D);
  const int64_t want = blocks_for_rows(p, l), cap = (int64_t)device_sm_count() * (2048 / l.threads);
  const unsigned blocks = (unsigned)(want < cap ? want : cap);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  by_layout(p, l, [&](auto t, auto w, auto v, auto items, auto wide) {
    norm_fwd_kernel<typename decltype(t)::type, typename decltype(w)::type, decltype(v)::value, decltype(items)::value, decltype(wide)::value>
        <<<blocks, l.threads, 0, st>>>(a);
  });
  return cudaGetLastError() == cudaSuccess ? BDLM_OK : BDLM_ERR_CUDA;
}

int bdlm_norm_bwd(const bdlm_norm_params* p, const void* dy, const void* h, const void* weight, const float* mean,
                  const float* rstd, const void* dh, void* dx, void* dweight, void* dbias,
                  void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check(p);
  if (rc != BDLM_OK) return rc;
  if (p->T > 0) {
    const void* need[] = {dy, h, rstd, dx};
    for (const void* q : need) if (q == nullptr) return BDLM_ERR_INVALID_ARG;
    if ((mean != nullptr) != (p->kind == BDLM_NORM_LAYER)) return BDLM_ERR_INVALID_ARG;
  }
  if (weight == nullptr && (dweight != nullptr || dbias != nullptr)) return BDLM_ERR_INVALID_ARG;
  const void* ptrs[] = {dy, h, weight, dh, dx, dweight, dbias, workspace};
  for (const void* q : ptrs) if (!al(q, 16)) return BDLM_ERR_INVALID_ARG;
  if (!al(mean, 4) || !al(rstd, 4)) return BDLM_ERR_INVALID_ARG;
  const bool grads = dweight != nullptr || dbias != nullptr;
  if (grads && p->T > 0 && workspace == nullptr) return BDLM_ERR_INVALID_ARG;
  if (grads && workspace_bytes < bdlm_norm_workspace_bytes(p)) return BDLM_ERR_WORKSPACE_TOO_SMALL;
  if (!sm100()) return BDLM_ERR_UNSUPPORTED;
  const Layout l = layout(p);
  const int groups = bwd_groups(p, l);
  NormArgs a = {};
  a.x = dy; a.res = dh; a.w = weight; a.h_in = h; a.y = dx;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = grads ? static_cast<float*>(workspace) : nullptr;
  a.T = p->T; a.D = p->D; a.nvec = l.nvec; a.tpr = l.tpr; a.rms = p->kind == BDLM_NORM_RMS;
  a.inv_d = (float)(1.0 / p->D);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  if (groups > 0) {
    by_layout(p, l, [&](auto t, auto w, auto v, auto items, auto wide) {
      constexpr int V = decltype(v)::value, I = decltype(items)::value;
      constexpr bool WIDE = decltype(wide)::value, BIG = big(V, I, WIDE);
      auto kern = norm_bwd_kernel<typename decltype(t)::type, typename decltype(w)::type, V, I, WIDE>;
      constexpr bool RINGED = ringed(V, I, WIDE);
      const int smem = RINGED ? RING * 3 * I * l.threads * 16 : !grads ? 0 : (int)((BIG ? 2 : WIDE ? 0 : 1) * l.threads * V * I * sizeof(float));
      e = !BIG && !RINGED ? cudaSuccess : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
      if (e != cudaSuccess) return;
      kern<<<groups, l.threads, smem, st>>>(a);
      e = cudaGetLastError();
    });
    if (e != cudaSuccess) return BDLM_ERR_CUDA;
  }
  if (!grads) return BDLM_OK;
  const unsigned bx = (unsigned)((p->D + 31) / 32);
  auto finish = [&](auto w) {
    using W = typename decltype(w)::type;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(bx, 2);
    cfg.blockDim = dim3(WG_WARPS * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = groups > 0 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, norm_wgrad_kernel<W>, (const float*)a.part, groups, p->D, static_cast<W*>(dweight), static_cast<W*>(dbias));
  };
  e = p->wdtype == BDLM_FP32 ? finish(Type<float>{}) : p->wdtype == BDLM_BF16 ? finish(Type<bf16_t>{}) : finish(Type<__half>{});
  return e == cudaSuccess ? BDLM_OK : BDLM_ERR_CUDA;
}

}  // extern "C"
