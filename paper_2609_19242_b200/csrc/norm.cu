// Layer norm and root-mean-square norm of a residual stream, forward and backward (include/bdlm_norm.h).
//
// Both passes are streams over the [T, D] tensors, bound by memory: 4 T D elements each (x, residual, y, h; dy, h, dh, dx).  A row
// is read once and in registers until it is written, and the variance is the sum of squares around the mean that has been
// formed, not a difference of two large sums.
//
// A row belongs to a part of a warp (a power of two of lanes) or a warp, to warps of a CTA, or, where those are not enough, to a
// cluster of two to five CTAs that exchange their sums.
//   forward    loads go straight into registers, several CTAs of an SM lie under one another
//   backward   one CTA an SM, of as many rows as 512 threads hold at 16 elements each: a thread keeps its columns for all its
//              rows, and with them the weight and the sums for dweight and dbias in registers, so that the columns' sums cost one row
//              of partial sums per CTA and a small reduction.  These sums leave no registers for loads in flight: the rows to
//              come are copied to shared memory asynchronously, a ring of them, and a thread reads what it has copied itself,
//              without a barrier.
// Bound by memory, the backward nearly as much by instruction issue (61 % of the slots at 8192 x 4096).  Measured, bf16 with
// residual, of the copy rate's floor, calls one after the other into outputs that are there:
// 16384 x 4096 forward 89 us (92 %), backward 92 (89 %); 32768 x 2048 87 (94 %), 90 (91 %);
// 8192 x 8192 93 (88 %), 102 (80 %); 4096 x 16384 102 (80 %), 128 (64 %: the cluster's exchange).  Without a residual the forward
// moves half the bytes but has as many barriers and nearly as many instructions: 16384 x 4096 64 us, 64 % (57 as a root-mean-square
// norm, which has one sum instead of two).  Tried and slower or no faster: in the forward the next row requested ahead where there is no residual
// (68: the registers do not hold it), products packed two to an instruction (87 and 62, but 65536 x 512 51 for 46), a ring
// (101); in both passes 1024 threads at 64 registers that read everything again from shared memory (105 and 168 us), 32 elements a
// thread (106 and 162); in the backward vectors in registers across the row's sums without a ring (101).
//
// Rows of a length that is no whole number of 16-byte vectors begin anywhere in a vector.  They are read as the vectors that cover
// them, shifted by `shift` elements; a thread's rows are P apart, P the number of rows after which the shift repeats, so that
// its columns stay its own.  (16384 x 4100: 142 us forward, 206 backward; element by element 462 and 1353.)  Part of what is left is the
// layout, which counts a row with the largest shift: 4095 elements have 513 vectors, one more than 256 threads take, so the backward's CTA
// has one row of 288 threads where 4096 elements give it two of 256.
#include <math.h>

#include "../../include/bdlm_norm.h"
#include "elem_common.cuh"
#include "tc_common.cuh"

namespace bdlm {
namespace {

using tc::add_f32x2;
using tc::fma_f32x2;
using tc::mul_f32x2;
using tc::pack_f32x2;
using tc::unpack_f32x2;

enum Span { NARROW, WIDE, TEAM };   // a row's threads: part of a warp or a warp; warps of a CTA; a cluster
// Vectors of a row that a thread has.  Backward: 16 elements, or one vector of short rows.  Forward: 16 elements too where a row takes
// more than a warp, or four vectors of 32-bit elements: with four, a row's weights are read again instead of kept, which costs long
// 16-bit rows more than the barriers of more threads do (8192 x 8191 279 us with four, 172 with two; 4096 x 16383 391,
// 239, with the fences below 214; 6144 x 10240 122, 114).  32-bit rows lose: 2048 x 16384 90 with four, 132 with two.
__host__ __device__ constexpr int bwd_items(int V) { return 16 / V; }
__host__ __device__ constexpr bool fwd_long(int items, Span s) { return s != NARROW && items == 4; }
constexpr int NARROW_THREADS = 128, BWD_THREADS = 512;   // of a CTA, at most
__host__ __device__ constexpr int fwd_threads(int V, int items, Span s) { return s == NARROW ? NARROW_THREADS : V == 4 && items == 2 ? 512 : 1024; }
// (64 registers where a row takes a CTA: 16384 x 4095 forward 242 us with 99, 144 with these)
__host__ __device__ constexpr int fwd_ctas(int V, int items, Span s) { return s == NARROW ? (items == 4 ? 4 : 8) : V == 4 && items == 2 ? 2 : 1; }
// One CTA an SM, said outright (0: not) where a thread has one vector: the compiler otherwise keeps to 64 registers and spills (262144 x 128
// 69 us, 58 so; with more vectors it does not, and 16384 x 4096 is 92 us without, 93 with).
__host__ __device__ constexpr int bwd_ctas(int items) { return items == 1 ? 1 : 0; }
// Rows in flight in the backward: the same number of bytes for 16- and 32-bit elements.
__host__ __device__ constexpr int ring_of(int V) { return V == 8 ? 4 : 2; }

struct NormArgs {
  const void *x, *res, *w, *b;     // forward; backward: dy, dh, weight
  const void* h_in;                // backward
  void *y, *h;                     // forward; backward: dx
  float *mean, *rstd;
  float* part;                     // backward: [dweight, dbias][groups][D]
  void *dw, *db;                   // backward in one CTA: where they go instead; all three nullptr: neither is wanted
  int T, D, tpr, rms, period, team;
  float eps, inv_d;
};

// The rows and columns of a thread.  SHIFT: rows may begin inside a vector.
template <int V, int ITEMS, Span S, bool SHIFT>
struct Place {
  int lane, sub, tpr, D;       // thread of the row's, which of the CTA's rows, and how many threads of it there are in this CTA
  bool first;                  // the row's first thread
  int64_t row, step;           // its first row, and how far apart they are
  int col[ITEMS];              // of each vector's first element; negative where the vector begins before the row
  bool has[ITEMS], whole[ITEMS];   // a vector there is; one that lies in the row altogether
  __device__ __forceinline__ Place(const NormArgs& a) {
    tpr = a.tpr;
    sub = (int)threadIdx.x / tpr;
    lane = (int)threadIdx.x - sub * tpr;
    const int rows = (int)blockDim.x / tpr, period = SHIFT ? a.period : 1;
    const int team = S == TEAM ? a.team : 1, rank = S == TEAM ? (int)tc::cluster_rank() : 0;
    const int64_t seq = (int64_t)(blockIdx.x / team) * rows + sub;
    row = seq;
    step = (int64_t)gridDim.x / team * rows;   // a multiple of the period
    D = a.D;
    const int shift = SHIFT ? (int)((seq % period) * D % V) : 0;
    const int all = (shift + D + V - 1) / V, share = (all + team - 1) / team;
    const int begin = min(all, rank * share), vecs = min(share, all - begin);
    first = lane == 0 && rank == 0;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      has[i] = lane + i * tpr < vecs;
      col[i] = (begin + lane + i * tpr) * V - shift;
      whole[i] = has[i] && (!SHIFT || (col[i] >= 0 && col[i] + V <= D));
    }
  }
  __device__ __forceinline__ bool in(int i, int e) const { return has[i] && (unsigned)(col[i] + e) < (unsigned)D; }
  template <class T, class R>
  __device__ __forceinline__ void store(int i, T* row_of, const R& r) const {   // row_of: the row's first element
    T* to = row_of + col[i];
    if (whole[i]) r.store(to);
    else if (SHIFT && has[i]) {
      const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
      for (int k = 0; k < V; ++k) if (in(i, k)) to[k] = e[k];
    }
  }
  // weight or bias of the thread's columns, zeros outside the row
  template <class W>
  __device__ __forceinline__ void columns(int i, const W* from, Raw<W, V>& r) const {
    r.clear();
    if (from == nullptr || !has[i]) return;
    if (!SHIFT) { r.load(from + col[i]); return; }
    W* e = reinterpret_cast<W*>(&r);
#pragma unroll
    for (int k = 0; k < V; ++k) if (in(i, k)) e[k] = from[col[i] + k];
  }
};
__device__ __forceinline__ void copies_end_row() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int RING>
__device__ __forceinline__ void copies_wait_first() { asm volatile("cp.async.wait_group %0;" ::"n"(RING - 1) : "memory"); }
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// The vectors of the rows to come: [row][tensor][item][thread].
template <class T, int TENSORS, int V, int ITEMS, Span S, bool SHIFT>
struct Ring {
  uint4* base;
  const Place<V, ITEMS, S, SHIFT>& at;
  int64_t elements;   // of the tensors
  uint4* masks;       // SHIFT: [item][thread], zero bits where a vector's elements are not the row's
  __device__ __forceinline__ void set_masks() const {
    if (!SHIFT) return;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      uint4 m;
      uint32_t* w = reinterpret_cast<uint32_t*>(&m);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) w[k] = at.in(i, k) ? ~0u : 0u;
        else w[k] = (at.in(i, 2 * k) ? 0xffffu : 0u) | (at.in(i, 2 * k + 1) ? 0xffff0000u : 0u);
      }
      masks[i * blockDim.x + threadIdx.x] = m;   // (read by this thread alone)
    }
  }
  __device__ __forceinline__ uint4* slot(int k, int tensor, int i) const { return base + ((k * TENSORS + tensor) * ITEMS + i) * blockDim.x + threadIdx.x; }
  __device__ __forceinline__ void copy(int k, int tensor, const T* from, int64_t row) const {
    const int64_t start = row * at.D;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (!at.has[i]) continue;
      const uint32_t to = (uint32_t)__cvta_generic_to_shared(slot(k, tensor, i));
      const int64_t left = elements - (start + at.col[i]);
      if (SHIFT && left < V) {   // the tensor ends inside its last vector
        const int bytes = (int)left * (int)sizeof(T);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from + start + at.col[i]), "r"(bytes) : "memory");
      } else {
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from + start + at.col[i]) : "memory");
      }
    }
  }
  // ok: there is such a row.  Elements of a vector that are not the row's become zeros.
  __device__ __forceinline__ void read(int k, int tensor, int i, bool ok, Raw<T, V>& r) const {
    r.clear();
    if (ok && at.has[i]) r.load(reinterpret_cast<const T*>(slot(k, tensor, i)));
    if (SHIFT && !at.whole[i]) {
      const uint4 m = masks[i * blockDim.x + threadIdx.x];
      r.q[0].x &= m.x; r.q[0].y &= m.y; r.q[0].z &= m.z; r.q[0].w &= m.w;
    }
  }
};

// A cluster's barrier that orders shared memory alone, which is where the sums are: a release of everything waits for the threads' stores
// to global memory too (backward 4096 x 16384 157 us, 136 with these fences, 128 with the exchange under the next row's products as well).
// The release covers this CTA's own sums, written before the others read them.  The other way round, a buffer is written again after
// others have read it, because a reader's next arrival comes after its loads have returned: every loaded sum goes through the
// shuffles that follow it, and those stand before that arrival.
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("fence.release.sync_restrict::shared::cta.cluster;\n\tbarrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;\n\tfence.acquire.sync_restrict::shared::cluster.cluster;" ::: "memory");
}
// Sums over the threads of a row; every thread gets them.  The order is fixed, and the same in all CTAs of a cluster.
template <Span S, int N>
__device__ __forceinline__ void row_sum(float (&v)[N], int tpr, int sub, int team, float* red, int& turn) {
  for (int s = S == NARROW ? tpr / 2 : 16; s > 0; s >>= 1) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], s);
  }
  if (S == NARROW) return;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = tpr >> 5;
  float* at = red + turn * 64;
  turn ^= 1;   // (a buffer is written again only after the barrier of the other one's use)
  if (lane == 0) {
#pragma unroll
    for (int n = 0; n < N; ++n) at[warp * 2 + n] = v[n];
  }
  if (S == TEAM) { cluster_arrive(); cluster_wait(); }
  else asm volatile("bar.sync %0, %1;" ::"r"(sub + 1), "r"(tpr) : "memory");   // the row's warps
  at += sub * warps * 2;
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = S == WIDE && lane < warps ? at[lane * 2 + n] : 0.f;
  if (S == TEAM && lane < warps) {
    for (int c = 0; c < team; ++c) {   // (its own among them)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        float u;
        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(u) : "r"(tc::peer_addr(tc::smem_u32(at + lane * 2 + n), c)) : "memory");
        v[n] += u;
      }
    }
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] += __shfl_xor_sync(0xffffffffu, v[n], s);
  }
}
constexpr int RED_FLOATS = 2 * 32 * 2;   // two buffers in turn, 32 warps, two sums
// The same over a cluster in two steps: a CTA's warps put their sums down before the cluster's barrier, every warp gets all of them after it.
__device__ __forceinline__ void team_put(float (&v)[2], float* red) {
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], s);
    v[1] += __shfl_xor_sync(0xffffffffu, v[1], s);
  }
  if ((threadIdx.x & 31) == 0) *reinterpret_cast<float2*>(red + (threadIdx.x >> 5) * 2) = make_float2(v[0], v[1]);
}
__device__ __forceinline__ void team_get(float (&v)[2], const float* red, int warps, int team) {
  const int lane = threadIdx.x & 31;
  v[0] = v[1] = 0.f;
  if (lane < warps) {
    const uint32_t at = tc::smem_u32(red + lane * 2);
    for (int c = 0; c < team; ++c) {
      float p, q;
      asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(p), "=f"(q) : "r"(tc::peer_addr(at, c)) : "memory");
      v[0] += p;
      v[1] += q;
    }
  }
#pragma unroll
  for (int s = 16; s > 0; s >>= 1) {
    v[0] += __shfl_xor_sync(0xffffffffu, v[0], s);
    v[1] += __shfl_xor_sync(0xffffffffu, v[1], s);
  }
}

// The forward loads a row's vectors straight into registers: a thread has nothing else to keep, so four CTAs of a 4096-element
// row share an SM and their loads lie under one another.  (The backward's ring took 101 us here instead of 89, 16384 x 4096.)
template <class T, class W, int V, int ITEMS, Span S, bool SHIFT>
__global__ void __launch_bounds__(fwd_threads(V, ITEMS, S), fwd_ctas(V, ITEMS, S)) norm_fwd_kernel(const NormArgs a) {
  constexpr bool LONG = fwd_long(ITEMS, S);
  __shared__ float red[RED_FLOATS];
  const int tpr = S == NARROW ? a.tpr : (int)blockDim.x, lane = S == NARROW ? (int)threadIdx.x % tpr : (int)threadIdx.x;
  const int rows = S == NARROW ? NARROW_THREADS / tpr : 1, sub = S == NARROW ? (int)threadIdx.x / tpr : 0;
  const int team = S == TEAM ? a.team : 1;
  const int seq = blockIdx.x / team * rows + sub, step = gridDim.x / team * rows;
  const int shift = SHIFT ? (int)((int64_t)(seq % a.period) * a.D % V) : 0;
  int begin = 0, vecs = (shift + a.D + V - 1) / V;
  if (S == TEAM) {
    const int share = (vecs + team - 1) / team;
    begin = min(vecs, (int)tc::cluster_rank() * share);
    vecs = min(vecs, begin + share);
  }
  const int first = begin + lane;
  int turn = 0;
  // element e of vector c is column c V - shift + e; only a row's first and last vectors can be partly outside it
  auto in = [&](int c, int e) { return c < vecs && (unsigned)(c * V - shift + e) < (unsigned)a.D; };
  auto whole = [&](int c) { return c < vecs && (!SHIFT || (c * V >= shift && c * V - shift + V <= a.D)); };
  auto load = [&](int c, const T* from, int row, Raw<T, V>& r) {
    r.clear();
    if (c >= vecs) return;
    const int64_t at = (int64_t)row * a.D - shift + (int64_t)c * V;
    if (!SHIFT || at + V <= (int64_t)a.T * a.D) r.load(from + at);   // (the tensor may end inside its last vector)
    else {
      T* e = reinterpret_cast<T*>(&r);
#pragma unroll
      for (int k = 0; k < V; ++k) if (in(c, k)) e[k] = from[at + k];
    }
  };
  auto store = [&](int c, T* to, int row, const Raw<T, V>& r) {
    const int64_t at = (int64_t)row * a.D - shift + (int64_t)c * V;
    if (whole(c)) r.store(to + at);
    else if (SHIFT) {
      const T* e = reinterpret_cast<const T*>(&r);
#pragma unroll
      for (int k = 0; k < V; ++k) if (in(c, k)) to[at + k] = e[k];
    }
  };
  auto columns = [&](int c, const void* p, Raw<W, V>& r) {
    const W* from = static_cast<const W*>(p);
    r.clear();
    if (from == nullptr || c >= vecs) return;
    if (!SHIFT) { r.load(from + (int64_t)c * V); return; }
    W* e = reinterpret_cast<W*>(&r);
#pragma unroll
    for (int k = 0; k < V; ++k) if (in(c, k)) e[k] = from[c * V - shift + k];
  };
  const T *x = static_cast<const T*>(a.x), *res = static_cast<const T*>(a.res);
  T *y = static_cast<T*>(a.y), *h = static_cast<T*>(a.h);
  Raw<W, V> w[LONG ? 1 : ITEMS], b[LONG ? 1 : ITEMS];   // of this thread's columns, for all its rows
  if (!LONG) {
#pragma unroll
    for (int i = 0; i < (LONG ? 1 : ITEMS); ++i) { columns(first + i * tpr, a.w, w[i]); columns(first + i * tpr, a.b, b[i]); }
  }
  for (int r0 = blockIdx.x / team * rows; r0 < a.T; r0 += step) {
    const int row = r0 + sub;
    const bool ok = row < a.T;
    float f[ITEMS][V], s[1] = {0.f};
    Raw<T, V> rx[ITEMS], rr[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      rx[i].clear(); rr[i].clear();
      if (ok) {
        load(first + i * tpr, x, row, rx[i]);
        if (res != nullptr) load(first + i * tpr, res, row, rr[i]);
      }
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = first + i * tpr;
      rx[i].get(f[i]);
      if (res != nullptr) {   // the sum as it is stored is what is normalised
        float g[V];
        rr[i].get(g);
#pragma unroll
        for (int e = 0; e < V; ++e) f[i][e] += g[e];
        rx[i].put(f[i]);
        rx[i].get(f[i]);
        if (ok) store(c, h, row, rx[i]);
      }
      if (SHIFT && !whole(c)) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[i][e] = in(c, e) ? f[i][e] : 0.f;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) s[0] += f[i][e];
    }
    float mean = 0.f;
    if (!a.rms) {
      row_sum<S>(s, tpr, 0, team, red, turn);
      mean = s[0] * a.inv_d;
    }
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = first + i * tpr;
      if (whole(c)) {
#pragma unroll
        for (int e = 0; e < V; ++e) { const float t = f[i][e] - mean; s[0] = fmaf(t, t, s[0]); }
      } else if (SHIFT) {
#pragma unroll
        for (int e = 0; e < V; ++e) { const float t = in(c, e) ? f[i][e] - mean : 0.f; s[0] = fmaf(t, t, s[0]); }
      }
    }
    row_sum<S>(s, tpr, 0, team, red, turn);
    const float rstd = rsqrtf(fmaf(s[0], a.inv_d, a.eps));
    if (ok && first == 0) {
      if (a.mean != nullptr) a.mean[row] = mean;
      if (a.rstd != nullptr) a.rstd[row] = rstd;
    }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int c = first + i * tpr;
      float wf[V], bf[V];
      if (LONG) { columns(c, a.w, w[0]); columns(c, a.b, b[0]); }
      w[LONG ? 0 : i].get(wf);
      b[LONG ? 0 : i].get(bf);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float n = (f[i][e] - mean) * rstd;
        f[i][e] = a.w != nullptr ? fmaf(n, wf[e], bf[e]) : n;
      }
      rx[i].put(f[i]);
      if (ok) store(c, y, row, rx[i]);
    }
  }
  if (S == TEAM) tc::cluster_sync();   // no CTA leaves while another one may still read its sums
}

// The products of a row's elements are packed two to an instruction: at 20 instructions an element, which they took one by one,
// their issue took as long as the memory does (16384 x 4096 bf16: 101 us, now 93 with the reduction, of which the memory's
// rate would allow 82).
// n is formed as the forward forms it, (h - mean) rstd: h rstd - mean rstd as one fused operation saves an instruction in each of the two
// places, but the rounding of mean rstd then stands in every n of a row (3e-5 at a mean of 1000 deviations; the subtraction is exact
// there).  It costs nothing that shows (16384 x 4096 92 us either way).
template <class T, class W, int V, int ITEMS, Span S, bool SHIFT>
__global__ void __launch_bounds__(BWD_THREADS, bwd_ctas(ITEMS)) norm_bwd_kernel(const NormArgs a) {
  constexpr int RING = ring_of(V);
  __shared__ __align__(8) float red[S == TEAM ? 2 * RED_FLOATS : RED_FLOATS];
  extern __shared__ uint4 ring_mem[];
  const Place<V, ITEMS, S, SHIFT> at(a);
  const Ring<T, 3, V, ITEMS, S, SHIFT> ring{ring_mem, at, (int64_t)a.T * a.D, ring_mem + RING * 3 * ITEMS * blockDim.x};
  ring.set_masks();
  const T *dy = static_cast<const T*>(a.x), *h = static_cast<const T*>(a.h_in), *dh = static_cast<const T*>(a.res);
  T* dx = static_cast<T*>(a.y);
  float next_mean = 0.f, next_rstd = 0.f;
  auto copy_row = [&](int k, int64_t row) {
    if (row < a.T) {
      ring.copy(k, 0, dy, row);
      ring.copy(k, 1, h, row);
      if (dh != nullptr) ring.copy(k, 2, dh, row);
    }
    copies_end_row();   // (an empty group where there is no row: the groups count rows)
  };
  auto request_stats = [&](int64_t row) {
    next_mean = row < a.T && !a.rms ? a.mean[row] : 0.f;
    next_rstd = row < a.T ? a.rstd[row] : 0.f;
  };
  for (int k = 0; k < RING; ++k) copy_row(k, at.row + k * at.step);
  request_stats(at.row);
  constexpr int H = V / 2;
  Raw<W, V> weight[ITEMS];
  uint64_t dw[ITEMS][H], db[ITEMS][H];   // pairs of columns
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    at.columns(i, static_cast<const W*>(a.w), weight[i]);
#pragma unroll
    for (int e = 0; e < H; ++e) dw[i][e] = db[i][e] = 0ull;
  }
  // the products that a row's two sums are made of, and the columns' sums; `y` and `h` of the row stay in ry, rh
  auto products = [&](int k, bool ok, float rs, float mean, Raw<T, V> (&ry)[ITEMS], Raw<T, V> (&rh)[ITEMS], float (&s)[2]) {
    const uint64_t rs2 = pack_f32x2(rs, rs), minus2 = pack_f32x2(-mean, -mean);
    uint64_t s0 = 0ull, s1 = 0ull;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float y[V], u[V], w[V];
      ring.read(k, 0, i, ok, ry[i]);
      ring.read(k, 1, i, ok, rh[i]);
      weight[i].get(w);
      ry[i].get(y);
      rh[i].get(u);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const uint64_t y2 = pack_f32x2(y[2 * e], y[2 * e + 1]), n2 = mul_f32x2(add_f32x2(pack_f32x2(u[2 * e], u[2 * e + 1]), minus2), rs2);
        const uint64_t g2 = a.w != nullptr ? mul_f32x2(y2, pack_f32x2(w[2 * e], w[2 * e + 1])) : y2;
        s0 = fma_f32x2(g2, n2, s0);
        s1 = add_f32x2(g2, s1);
        dw[i][e] = fma_f32x2(y2, n2, dw[i][e]);
        db[i][e] = add_f32x2(y2, db[i][e]);
      }
    }
    float p, q;
    unpack_f32x2(s0, p, q);
    s[0] = p + q;
    unpack_f32x2(s1, p, q);
    s[1] = p + q;
  };
  auto finish = [&](int k, int64_t row, bool ok, float rs, float mean, const Raw<T, V> (&ry)[ITEMS], const Raw<T, V> (&rh)[ITEMS], const float (&s)[2]) {
    const uint64_t rs2 = pack_f32x2(rs, rs), minus2 = pack_f32x2(-mean, -mean);
    const float c2 = -s[0] * a.inv_d * rs, c1 = a.rms ? 0.f : -s[1] * a.inv_d * rs;
    const uint64_t c22 = pack_f32x2(c2, c2), c12 = pack_f32x2(c1, c1);
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float y[V], u[V], w[V], d[V];
      Raw<T, V> rd, o;
      rd.clear();
      if (dh != nullptr) ring.read(k, 2, i, ok, rd);
      rd.get(d);
      weight[i].get(w);
      ry[i].get(y);
      rh[i].get(u);
#pragma unroll
      for (int e = 0; e < H; ++e) {
        const uint64_t n2 = mul_f32x2(add_f32x2(pack_f32x2(u[2 * e], u[2 * e + 1]), minus2), rs2);
        uint64_t g2 = pack_f32x2(y[2 * e], y[2 * e + 1]);
        if (a.w != nullptr) g2 = mul_f32x2(g2, pack_f32x2(w[2 * e], w[2 * e + 1]));
        const uint64_t t2 = add_f32x2(fma_f32x2(n2, c22, c12), pack_f32x2(d[2 * e], d[2 * e + 1]));
        unpack_f32x2(fma_f32x2(g2, rs2, t2), d[2 * e], d[2 * e + 1]);
      }
      o.put(d);
      if (ok) at.store(i, dx + row * a.D, o);
    }
    copy_row(k, row + RING * at.step);   // (after this thread's reads of the slot)
  };
  Raw<T, V> ry[ITEMS], rh[ITEMS];   // (as vectors of the element type they take half the registers across the joining of the sums)
  int64_t row = at.row;
  if constexpr (S == TEAM && RING == 4) {
    // The cluster's exchange of one row lies under the products of the next: arrive(r), then row r - 1 is finished, then the products of
    // row r + 1, and only then wait(r).  Four buffers of sums: one is written again when every CTA has arrived once more after its last
    // reads of it.
    float was_rs = 0.f, was_mean = 0.f;
    int n = 0;
    for (int64_t done = 0;; done += at.step, row += at.step, ++n) {
      const bool more = done < a.T;   // (the same in all CTAs of a cluster)
      const float rs = next_rstd, mean = next_mean;
      float s[2];
      if (more) {
        request_stats(row + at.step);
        copies_wait_first<RING - 1>();   // row n's: RING + n - 1 have been asked for, RING at first
        products(n % RING, row < a.T, rs, mean, ry, rh, s);
        team_put(s, red + n % 4 * 64);
      }
      if (n > 0) cluster_wait();
      if (more) cluster_arrive();
      if (n > 0) {
        const int k = (n - 1) % RING;
        const int64_t was = row - at.step;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) { ring.read(k, 0, i, was < a.T, ry[i]); ring.read(k, 1, i, was < a.T, rh[i]); }
        team_get(s, red + (n - 1) % 4 * 64, at.tpr >> 5, a.team);
        finish(k, was, was < a.T, was_rs, was_mean, ry, rh, s);
      }
      if (!more) break;
      was_rs = rs;
      was_mean = mean;
    }
  } else {
    int turn = 0, k = 0;
    for (int64_t done = 0; done < a.T; done += at.step, row += at.step, k = k + 1 == RING ? 0 : k + 1) {
      const bool ok = row < a.T;
      const float rs = next_rstd, mean = next_mean;
      float s[2];
      request_stats(row + at.step);
      copies_wait_first<RING>();
      products(k, ok, rs, mean, ry, rh, s);
      row_sum<S>(s, at.tpr, at.sub, a.team, red, turn);
      finish(k, row, ok, rs, mean, ry, rh, s);
    }
  }
  copies_wait_all();
  if (S == TEAM) tc::cluster_sync();   // no CTA leaves while the other one may still read its sums
  if (a.part == nullptr && a.dw == nullptr && a.db == nullptr) return;
  float* comb = reinterpret_cast<float*>(ring_mem);   // the CTA's rows join their sums here
  const int rows = blockDim.x / at.tpr, group = blockIdx.x / a.team, groups = gridDim.x / a.team;
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    W* out = static_cast<W*>(which ? a.db : a.dw);
    float* part = a.part + ((int64_t)which * groups + group) * a.D;
    float* to = rows > 1 ? comb + (int64_t)at.sub * a.D : part;
    __syncthreads();   // all rows' copies have landed, and the first sums have been read
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
      for (int e = 0; e < H; ++e) {
        float p, q;
        unpack_f32x2(which ? db[i][e] : dw[i][e], p, q);
        const int c = at.col[i] + 2 * e;
        if (rows > 1 || a.part != nullptr) {
          if (at.in(i, 2 * e)) to[c] = p;
          if (at.in(i, 2 * e + 1)) to[c + 1] = q;
        } else if (out != nullptr) {
          if (at.in(i, 2 * e)) out[c] = W(p);
          if (at.in(i, 2 * e + 1)) out[c + 1] = W(q);
        }
      }
    }
    if (rows > 1) {
      __syncthreads();
      for (int c = threadIdx.x; c < a.D; c += blockDim.x) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += comb[(int64_t)r * a.D + c];
        if (a.part != nullptr) part[c] = s;
        else if (out != nullptr) out[c] = W(s);
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
// Elements of a call whose backward one CTA does in a few rounds, in less time than a call takes the host (5 x 200 elements, back to
// back: 19.4 -> 14.1 us a call).
constexpr int ONE_CTA = 32768;
constexpr int SMS = 148;   // what the launch shapes, and with them the workspace, count on: the device has them

// How the rows are laid over threads: `rows` of them in a CTA (a CTA's share of one in a team), tpr threads each.
struct Layout { Span span; int vec, nvec, items, tpr, rows, period, team; };
Layout vectors_of(const bdlm_norm_params* p) {
  Layout l = {};
  l.vec = p->dtype == BDLM_FP32 ? 4 : 8;
  l.period = 1;
  while ((int64_t)p->D * l.period % l.vec != 0) l.period *= 2;
  l.nvec = l.period == 1 ? p->D / l.vec : (p->D + 2 * l.vec - 2) / l.vec;   // with the largest shift
  return l;
}
int up32(int n) { return (n + 31) / 32 * 32; }
int narrow_tpr(int nvec, int items) {
  int tpr = 1;
  while (tpr * items < nvec) tpr *= 2;
  return tpr;
}
Layout fwd_layout(const bdlm_norm_params* p) {
  Layout l = vectors_of(p);
  l.team = 1;
  if (l.nvec <= 128) {
    l.span = NARROW;
    l.items = l.nvec <= 32 ? 1 : l.nvec <= 64 ? 2 : 4;
    l.tpr = narrow_tpr(l.nvec, l.items);
    l.rows = NARROW_THREADS / l.tpr;
    return l;
  }
  l.items = l.vec == 8 || l.nvec <= 2 * fwd_threads(l.vec, 2, WIDE) ? 2 : 4;
  const int most = l.items * fwd_threads(l.vec, l.items, WIDE);
  l.team = (l.nvec + most - 1) / most;
  l.span = l.team > 1 ? TEAM : WIDE;
  l.tpr = up32(((l.nvec + l.team - 1) / l.team + l.items - 1) / l.items);
  l.rows = 1;
  return l;
}
// The backward's CTAs have as many rows as fit, because those share partial sums, but none that leaves SMs without rows; whole
// warps of NARROW ones, and a barrier of its own for each WIDE one, of 15 that there are.
Layout bwd_layout(const bdlm_norm_params* p) {
  Layout l = vectors_of(p);
  l.items = l.nvec <= 32 ? 1 : bwd_items(l.vec);
  l.team = (l.nvec + BWD_THREADS * l.items - 1) / (BWD_THREADS * l.items);
  const int own = ((l.nvec + l.team - 1) / l.team + l.items - 1) / l.items;   // threads a CTA needs for a row
  l.span = l.team > 1 ? TEAM : own > 32 ? WIDE : NARROW;
  l.tpr = own > 32 ? up32(own) : narrow_tpr(own, 1);
  const bool one = (int64_t)p->T * p->D <= ONE_CTA;
  const int64_t even = one ? p->T : ((int64_t)p->T + SMS - 1) / SMS;
  l.rows = l.span == TEAM ? 1 : BWD_THREADS / l.tpr;
  if (l.span == WIDE && l.rows > 15) l.rows = 15;
  if (l.rows > even) l.rows = even > 0 ? (int)even : 1;
  if (l.span == NARROW) { const int per_warp = 32 / l.tpr; l.rows = (l.rows + per_warp - 1) / per_warp * per_warp; }
  if (one) {   // whole periods of rows, some of them without a row if need be
    const int up = (l.rows + l.period - 1) / l.period * l.period;
    if (up * l.tpr <= BWD_THREADS && (l.span != WIDE || up <= 15)) l.rows = up;
    else if (l.rows > l.period) l.rows = l.rows / l.period * l.period;
  }
  return l;
}
// CTAs, or clusters, of a launch: as many as have rows, at most `per_sm` an SM, and sequences of rows in whole periods.
int groups_of(const bdlm_norm_params* p, const Layout& l, int per_sm) {
  int unit = 1;
  while (unit * l.rows % l.period != 0) unit *= 2;
  const int64_t want = ((int64_t)p->T + l.rows - 1) / l.rows, cap = SMS * per_sm / l.team;
  return (int)(want < cap ? (want + unit - 1) / unit * unit : cap / unit * unit);
}
int fwd_groups(const bdlm_norm_params* p, const Layout& l) { return groups_of(p, l, 2048 / (l.rows * l.tpr)); }
// One CTA for the smallest calls, if its rows are a whole period: it needs no partial sums, no workspace and no second launch.
int bwd_groups(const bdlm_norm_params* p, const Layout& l) {
  if (p->T > 0 && (int64_t)p->T * p->D <= ONE_CTA && l.span != TEAM && l.rows % l.period == 0) return 1;
  return groups_of(p, l, 1);
}

int check(const bdlm_norm_params* p) {
  if (p == nullptr || p->T < 0 || p->T > (1 << 30) || p->D <= 0) return BDLM_ERR_INVALID_ARG;
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

// Calls f(T, W, V, SHIFT) with the call's types and vectors as template arguments.
template <int N> using Int = std::integral_constant<int, N>;
template <class T> struct Type { using type = T; };
template <class F>
void by_types(const bdlm_norm_params* p, const Layout& l, F f) {
  auto by_shift = [&](auto t, auto w) {
    using V = Int<sizeof(typename decltype(t)::type) == 4 ? 4 : 8>;
    if (l.period > 1) f(t, w, V{}, std::true_type{});
    else f(t, w, V{}, std::false_type{});
  };
  auto by_weight = [&](auto t) {
    if (p->wdtype == BDLM_FP32) by_shift(t, Type<float>{});
    else by_shift(t, t);
  };
  if (p->dtype == BDLM_BF16) by_weight(Type<bf16_t>{});
  else if (p->dtype == BDLM_FP16) by_weight(Type<__half>{});
  else by_shift(Type<float>{}, Type<float>{});
}
// smem: bytes a thread.  The limit that is set is the one of the largest CTA, the same in every call: the attribute is the function's,
// and another host thread may set it between this call's setting and its launch.
template <class K>
cudaError_t launch_rows(K kern, const Layout& l, int groups, int smem, cudaStream_t st, const NormArgs& a) {
  if (smem > 0) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem * BWD_THREADS);
    if (e != cudaSuccess) return e;
  }
  return launch_chained(kern, false, (unsigned)(groups * l.team), l.rows * l.tpr, smem * l.rows * l.tpr, st, l.team, a);
}

}  // namespace
}  // namespace bdlm

using namespace bdlm;

extern "C" {

size_t bdlm_norm_workspace_bytes(const bdlm_norm_params* p) {
  if (check(p) != BDLM_OK) return 0;
  const size_t groups = (size_t)bwd_groups(p, bwd_layout(p));
  return groups == 1 ? 0 : 2 * groups * p->D * sizeof(float);
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
  const Layout l = fwd_layout(p);
  NormArgs a = {};
  a.x = x; a.res = residual; a.w = weight; a.b = bias; a.y = y; a.h = h; a.mean = mean; a.rstd = rstd;
  a.T = p->T; a.D = p->D; a.tpr = l.tpr; a.rms = p->kind == BDLM_NORM_RMS; a.period = l.period; a.team = l.team; a.eps = p->eps;
  a.inv_d = (float)(1.0 / p->D);
  cudaError_t e = cudaSuccess;
  by_types(p, l, [&](auto t, auto w, auto v, auto shift) {
    using X = typename decltype(t)::type;
    using Wt = typename decltype(w)::type;
    constexpr int V = decltype(v)::value;
    constexpr bool SH = decltype(shift)::value;
    constexpr int MOST = V == 8 ? 2 : 4;
    void (*kern)(NormArgs) = l.span == TEAM  ? norm_fwd_kernel<X, Wt, V, MOST, TEAM, SH>
                             : l.span == WIDE ? (l.items == 2 ? norm_fwd_kernel<X, Wt, V, 2, WIDE, SH> : norm_fwd_kernel<X, Wt, V, MOST, WIDE, SH>)
                             : l.items == 1   ? norm_fwd_kernel<X, Wt, V, 1, NARROW, SH>
                             : l.items == 2   ? norm_fwd_kernel<X, Wt, V, 2, NARROW, SH>
                                              : norm_fwd_kernel<X, Wt, V, 4, NARROW, SH>;
    e = launch_rows(kern, l, fwd_groups(p, l), 0, static_cast<cudaStream_t>(cuda_stream), a);
  });
  return e == cudaSuccess ? BDLM_OK : BDLM_ERR_CUDA;
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
  const size_t need_ws = grads ? bdlm_norm_workspace_bytes(p) : 0;
  if (need_ws > 0 && workspace == nullptr) return BDLM_ERR_INVALID_ARG;
  if (workspace_bytes < need_ws) return BDLM_ERR_WORKSPACE_TOO_SMALL;
  if (!sm100()) return BDLM_ERR_UNSUPPORTED;
  const Layout l = bwd_layout(p);
  const int groups = bwd_groups(p, l);
  NormArgs a = {};
  a.x = dy; a.res = dh; a.w = weight; a.h_in = h; a.y = dx;
  a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
  a.part = need_ws > 0 ? static_cast<float*>(workspace) : nullptr;
  if (groups == 1) { a.dw = dweight; a.db = dbias; }
  a.T = p->T; a.D = p->D; a.tpr = l.tpr; a.rms = p->kind == BDLM_NORM_RMS; a.period = l.period; a.team = l.team;
  a.inv_d = (float)(1.0 / p->D);
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  cudaError_t e = cudaSuccess;
  if (groups > 0) {
    by_types(p, l, [&](auto t, auto w, auto v, auto shift) {
      using X = typename decltype(t)::type;
      using Wt = typename decltype(w)::type;
      constexpr int V = decltype(v)::value, I = bwd_items(V);
      constexpr bool SH = decltype(shift)::value;
      void (*kern)(NormArgs) = l.span == TEAM   ? norm_bwd_kernel<X, Wt, V, I, TEAM, SH>
                               : l.span == WIDE ? norm_bwd_kernel<X, Wt, V, I, WIDE, SH>
                               : l.items == 1   ? norm_bwd_kernel<X, Wt, V, 1, NARROW, SH>
                                                : norm_bwd_kernel<X, Wt, V, I, NARROW, SH>;
      e = launch_rows(kern, l, groups, (ring_of(V) * 3 + (SH ? 1 : 0)) * l.items * 16, st, a);
    });
    if (e != cudaSuccess) return BDLM_ERR_CUDA;
  }
  if (!grads || groups == 1) return BDLM_OK;
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
