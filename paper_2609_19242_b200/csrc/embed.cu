// Token embedding (include/bdlm_embed.h): rows of the table looked up and scaled, and the table's gradient over sorted tokens.
//
// The lookup is a copy of T rows: 2 T D elements, bound by memory.
//
// The gradient has to read T D elements and write V D of them, most of the latter zeros (a batch holds a few thousand of
// 128256 tokens).  Three launches, chained (one, up to FEW_TOKENS tokens, which every CTA of the sum then sorts itself):
//   sort    up to RANK_MOST tokens by counting: a token's place is how many come before it.  More: one cluster sorts (id, position) by id, a stable radix sort whose CTAs exchange their digits' counts through
//           distributed shared memory; the pairs ping-pong through the workspace, which stays in L2
//   sum     zeros the rows of tokens that do not occur -- it finds them in the ids themselves, so this runs beside the sort --
//           and then, once the sort is done, sums the sorted tokens' rows in pieces of `piece` tokens.  A run of equal ids is
//           finished by the piece it begins in, into the next one if need be; of one that covers a whole further piece, each
//           piece leaves an fp32 part.  (With parts of every run that crosses a border, a third of the borders of 16384 tokens
//           over 32008 ids had some, and joining them took 25 us of 85.)
//   join    adds the parts of such long runs (the mask token's covers hundreds of pieces)
// Every sum runs in the tokens' order inside a piece, and a long run's over its pieces in order, or in
// sixteen interleaved shares that are added in order: the ids alone fix the order, and no atomics meet in a sum.
#include <math.h>

#include "../../include/bdlm_embed.h"
#include "elem_common.cuh"

namespace bdlm {
namespace {

__device__ __forceinline__ uint32_t cta_of_cluster() { uint32_t n; asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(n)); return n; }
// Also orders the CTAs' writes to global memory before the others' reads of it (release and acquire at cluster scope).
__device__ __forceinline__ void whole_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int ld_cluster_int(const int* own, int rank) {
  const uint32_t at = (uint32_t)__cvta_generic_to_shared(own);
  int v;
  asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.u32 %0, [a];\n\t}" : "=r"(v) : "r"(at), "r"(rank) : "memory");
  return v;
}
__device__ __forceinline__ void wait_for_sort() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// What a thread of a group of `tpr` has of a row's slab: a vector, or, where rows are no whole number of those, S single elements
// tpr apart.
template <class T, int V, int S>
struct Slice {
  static constexpr int C = V > 1 ? V : S;
  Raw<T, V> q[V > 1 ? 1 : S];
  __device__ __forceinline__ static int first(int slab, int tpr, int lane) { return V > 1 ? (slab * tpr + lane) * V : slab * S * tpr + lane; }   // its first column
  __device__ __forceinline__ void load(const T* row, int at, int tpr, int D) {
    if (V > 1) { q[0].load(row + at); return; }
#pragma unroll
    for (int e = 0; e < C / (V > 1 ? V : 1); ++e) {
      const int c = at + e * tpr;
      q[e].clear();
      if (c < D) q[e].load(row + c);
    }
  }
  __device__ __forceinline__ void store(T* row, int at, int tpr, int D) const {
    if (V > 1) { q[0].store(row + at); return; }
#pragma unroll
    for (int e = 0; e < C / (V > 1 ? V : 1); ++e) {
      const int c = at + e * tpr;
      if (c < D) q[e].store(row + c);
    }
  }
  __device__ __forceinline__ void get(float (&f)[C]) const {
#pragma unroll
    for (int e = 0; e < C / V; ++e) q[e].get(reinterpret_cast<float (&)[V]>(f[e * V]));
  }
  __device__ __forceinline__ void put(const float (&f)[C]) {
#pragma unroll
    for (int e = 0; e < C / V; ++e) q[e].put(reinterpret_cast<const float (&)[V]>(f[e * V]));
  }
};

// ------------------------------------------------------------------------------------------------ lookup
// `tpr` threads (a power of two) share a row, four vectors or eight elements of it in flight in each.
template <class E, class O, int V>
__global__ void __launch_bounds__(256) embed_fwd_kernel(const E* table, const int* ids, O* out, int T, int D, int vocab, int tpr, float scale) {
  const int rows = 256 / tpr, lane = threadIdx.x % tpr;
  const int64_t row = (int64_t)blockIdx.x * rows + threadIdx.x / tpr;
  if (row >= T) return;
  const int id = ids[row];
  const bool real = id >= 0 && id < vocab;
  const int nvec = D / V;
  const E* src = table + (int64_t)(real ? id : 0) * D;
  O* dst = out + row * D;
  constexpr int U = V > 1 ? 4 : 8;
  for (int c0 = lane; c0 < nvec; c0 += U * tpr) {
    Raw<E, V> r[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      r[u].clear();
      if (real && c0 + u * tpr < nvec) r[u].load(src + (int64_t)(c0 + u * tpr) * V);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (c0 + u * tpr < nvec) {
        float f[V];
        Raw<O, V> o;
        r[u].get(f);
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] *= scale;
        o.put(f);
        o.store(dst + (int64_t)(c0 + u * tpr) * V);
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ sort
constexpr int SORT_CTAS = 8, SORT_WARPS = 32, DIGIT_BITS = 9, BINS = 1 << DIGIT_BITS;
constexpr int SORT_SMEM = (SORT_WARPS + 2) * BINS * (int)sizeof(int) + 32 * (int)sizeof(int);

// Pairs (key, position), sorted by key with positions ascending among equal keys; key = id, or V where the id is no token.
// A warp owns a run of `seg` consecutive pairs.  A pass counts each warp's digits, turns the counts into the places where
// each warp's pairs of each digit begin (over the bins, then the CTAs, then the warps), and moves the pairs; equal digits
// inside a group of 32 are ranked by a vote.  The last pass writes `sorted`.
__global__ void __launch_bounds__(SORT_WARPS * 32) embed_sort_kernel(const int* ids, int T, int V, int passes, int bits, int2* sorted, int2* other) {
  extern __shared__ int sm[];
  int* hist = sm;                               // [warp][bin]
  int* total = sm + SORT_WARPS * BINS;          // this CTA's count of each bin, read by the others
  int* base = total + BINS;                     // where this CTA's pairs of each bin begin
  int* scan = base + BINS;
  let_next_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, bins = 1 << bits;
  const int rank = (int)cta_of_cluster();
  constexpr int warps = SORT_CTAS * SORT_WARPS;
  const int64_t seg = (((int64_t)T + warps - 1) / warps + 31) / 32 * 32;
  const int64_t first = min((int64_t)T, (int64_t)(rank * SORT_WARPS + warp) * seg), last = min((int64_t)T, first + seg);
  int* mine = hist + warp * BINS;
  constexpr int HELD = 8;   // pairs a thread has in flight; a short run stays in registers between counting and moving
  int2 held[HELD];
  const bool few = last - first <= 32 * HELD;
  for (int pass = 0; pass < passes; ++pass) {
    // which of the two buffers this pass writes: the last one writes `sorted`
    int2* dst = (passes - 1 - pass) % 2 == 0 ? sorted : other;
    const int2* src = dst == sorted ? other : sorted;
    const int shift = pass * bits;
    auto pair_at = [&](int64_t i) {
      if (i >= last) return make_int2(-1, 0);
      if (pass > 0) return __ldcg(src + i);
      const int id = ids[i];
      return make_int2(id >= 0 && id < V ? id : V, (int)i);
    };
    auto request = [&](int64_t i) {
#pragma unroll
      for (int k = 0; k < HELD; ++k) held[k] = pair_at(i + 32 * k + lane);
    };
    if (few) request(first);
    for (int b = threadIdx.x; b < SORT_WARPS * BINS / 4; b += SORT_WARPS * 32) reinterpret_cast<int4*>(hist)[b] = make_int4(0, 0, 0, 0);
    __syncthreads();
    for (int64_t i = first; i < last; i += 32 * HELD) {
      if (!few) request(i);
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
        const int2 p = held[k];
        const int digit = p.x < 0 ? bins : (p.x >> shift) & (bins - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        if (p.x >= 0 && lane == __ffs(same) - 1) mine[digit] += __popc(same);
        __syncwarp();
      }
    }
    __syncthreads();
    int sum = 0;
    if ((int)threadIdx.x < bins) {
#pragma unroll
      for (int w = 0; w < SORT_WARPS; ++w) {
        const int n = hist[w * BINS + threadIdx.x];
        hist[w * BINS + threadIdx.x] = sum;
        sum += n;
      }
      total[threadIdx.x] = sum;
    }
    whole_cluster_sync();
    // exclusive sums over the bins of all CTAs, and the lower CTAs' pairs of the same bin
    int all = 0, lower = 0;
    if ((int)threadIdx.x < bins) {
      int n[SORT_CTAS];   // all on their way at once
#pragma unroll
      for (int c = 0; c < SORT_CTAS; ++c) n[c] = ld_cluster_int(total + threadIdx.x, c);
#pragma unroll
      for (int c = 0; c < SORT_CTAS; ++c) { all += n[c]; lower += c < rank ? n[c] : 0; }
    }
    int up = all;
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
      const int n = __shfl_up_sync(0xffffffffu, up, s);
      if (lane >= s) up += n;
    }
    if (lane == 31) scan[warp] = up;
    __syncthreads();
    if (warp == 0) {
      int n = scan[lane];
#pragma unroll
      for (int s = 1; s < 32; s <<= 1) {
        const int m = __shfl_up_sync(0xffffffffu, n, s);
        if (lane >= s) n += m;
      }
      scan[lane] = n;
    }
    __syncthreads();
    if ((int)threadIdx.x < bins) base[threadIdx.x] = (warp > 0 ? scan[warp - 1] : 0) + up - all + lower;
    __syncthreads();
    for (int64_t i = first; i < last; i += 32 * HELD) {
      if (!few) request(i);
#pragma unroll
      for (int k = 0; k < HELD; ++k) {
        const int2 p = held[k];
        const int digit = p.x < 0 ? bins : (p.x >> shift) & (bins - 1);
        const unsigned same = __match_any_sync(0xffffffffu, digit);
        int at = 0;
        if (p.x >= 0) at = base[digit] + mine[digit];
        __syncwarp();
        if (p.x >= 0) {
          dst[at + __popc(same & ((1u << lane) - 1))] = p;
          if (lane == __ffs(same) - 1) mine[digit] += __popc(same);
        }
        __syncwarp();
      }
    }
    __threadfence();
    whole_cluster_sync();   // the pairs have arrived, and the counts have been read
  }
}

// The same pairs for few tokens: a token's place is the number of tokens that come before it, counted over all of them.  T^2
// comparisons over the whole chip and no exchange, where the radix sort is a chain of barriers in one cluster.
constexpr int RANK_WARPS = 8, RANK_TOKENS = 4, RANK_MOST = 8192;   // RANK_TOKENS tokens a warp at a time; keys in shared memory
__global__ void __launch_bounds__(RANK_WARPS * 32) embed_rank_kernel(const int* ids, int T, int V, int2* sorted) {
  __shared__ int keys[RANK_MOST];
  let_next_start();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, padded = (T + 31) / 32 * 32;
#pragma unroll 8
  for (int t = threadIdx.x; t < padded; t += RANK_WARPS * 32) {
    const int id = t < T ? ids[t] : -1;
    keys[t] = t >= T ? 0x7fffffff : id >= 0 && id < V ? id : V;
  }
  __syncthreads();
  const int t0 = (blockIdx.x * RANK_WARPS + warp) * RANK_TOKENS;   // RANK_TOKENS divides 32: they stand in one group of 32
  if (t0 >= T) return;
  int key[RANK_TOKENS], count[RANK_TOKENS];
#pragma unroll
  for (int n = 0; n < RANK_TOKENS; ++n) { key[n] = keys[min(t0 + n, T - 1)]; count[n] = 0; }
  const int own = t0 / 32 * 32;
#pragma unroll 4
  for (int j = 0; j < own; j += 32) {   // earlier tokens come first among equals
    const int k = keys[j + lane];
#pragma unroll
    for (int n = 0; n < RANK_TOKENS; ++n) count[n] += k <= key[n];
  }
  {
    const int k = keys[own + lane];
#pragma unroll
    for (int n = 0; n < RANK_TOKENS; ++n) count[n] += own + lane < t0 + n ? k <= key[n] : k < key[n];
  }
#pragma unroll 4
  for (int j = own + 32; j < padded; j += 32) {
    const int k = keys[j + lane];
#pragma unroll
    for (int n = 0; n < RANK_TOKENS; ++n) count[n] += k < key[n];
  }
#pragma unroll
  for (int n = 0; n < RANK_TOKENS; ++n) {
    count[n] = __reduce_add_sync(0xffffffffu, count[n]);
    if (lane == 0 && t0 + n < T) sorted[count[n]] = make_int2(key[n], t0 + n);
  }
}

// ------------------------------------------------------------------------------------------------ sum
struct SumArgs {
  const void* dout;
  const int* ids;
  const int2* sorted;
  void* dtable;
  float* parts;    // [pieces][2][D]: of a run that comes from the piece before, of one that begins here and goes on
  int T, D, V, piece, pieces, slabs, tpr;
  float scale;
  int accumulate;
  int spread;      // neighbouring pieces in different CTAs
};

constexpr int SUM_THREADS = 512, GROUP_THREADS = 128;   // threads of a CTA; of a piece's slab, at most
constexpr int FILL_WORDS = 4096;                        // rows a CTA looks up at a time: a bit each

// A warp zeros a row, wherever it begins: whole 16-byte vectors, and elements before and after them.
template <class E>
__device__ __forceinline__ void zero_row(E* row, int D) {
  constexpr int PER = 16 / (int)sizeof(E);
  const int lane = threadIdx.x & 31, head = min(D, (int)((16u - ((uintptr_t)row & 15u)) & 15u) / (int)sizeof(E));
  const int vecs = (D - head) / PER, tail = head + vecs * PER;
  if (lane < head) row[lane] = E(0.f);
  uint4* at = reinterpret_cast<uint4*>(row + head);
  for (int c = lane; c < vecs; c += 32) at[c] = make_uint4(0u, 0u, 0u, 0u);
  if (tail + lane < D) row[tail + lane] = E(0.f);
}

// The same for n short rows that lie one after the other, of which absent(r) says whether row r is to be zeroed: by the vectors that
// cover them, a thread each, where a warp to a row would leave most of its lanes idle.  (91650 rows of 154 bytes: the call 17 us instead
// of 27, in part by more tokens in flight; 128256 rows of 384 bytes 32 instead of 29.)
constexpr int SHORT_ROW = 256;   // bytes
template <class E, class F>
__device__ __forceinline__ void zero_short_rows(E* rows, int n, int D, F absent) {
  constexpr int PER = 16 / (int)sizeof(E);
  const int shift = (int)((uintptr_t)rows & 15u) / (int)sizeof(E), total = n * D;
  for (int v = threadIdx.x; v * PER < total + shift; v += blockDim.x) {
    const int first = v * PER - shift, lo = max(first, 0), hi = min(first + PER, total);
    int r = lo / D;
    const int last = (hi - 1) / D;
    bool all = hi - lo == PER;
    for (int q = r; q <= last; ++q) all = all && absent(q);
    if (all) { *reinterpret_cast<uint4*>(rows + first) = make_uint4(0u, 0u, 0u, 0u); continue; }
    int end = (r + 1) * D;   // of the element's row
    for (int e = lo; e < hi; ++e) {
      if (e == end) { ++r; end += D; }
      if (absent(r)) rows[e] = E(0.f);
    }
  }
}

// E: table, O: tokens' rows.  A group of `tpr` threads takes a piece and a slab of columns, a Slice of it each.
// FEW: no more than FEW_TOKENS of them, one piece: each CTA sorts them itself, and this is the only launch.
constexpr int FEW_TOKENS = 32;
__host__ __device__ constexpr int singles(bool few) { return few ? 2 : 8; }   // of a Slice: few tokens are a chain of loads, and threads there are enough
template <class E, class O, int V, bool ADD, bool FEW>
__global__ void __launch_bounds__(SUM_THREADS, 2) embed_sum_kernel(const SumArgs a) {
  __shared__ uint32_t present[FILL_WORDS];
  E* dtable = static_cast<E*>(a.dtable);
  if (!ADD) {
    const int64_t share = ((int64_t)a.V + gridDim.x - 1) / gridDim.x;
    const int64_t begin = min((int64_t)a.V, blockIdx.x * share), end = min((int64_t)a.V, begin + share);
    for (int64_t v0 = begin; v0 < end; v0 += FILL_WORDS * 32) {
      const int n = (int)min((int64_t)FILL_WORDS * 32, end - v0);
      for (int i = threadIdx.x; i < (n + 31) / 32; i += SUM_THREADS) present[i] = 0u;
      __syncthreads();
#pragma unroll 16
      for (int t = threadIdx.x; t < a.T; t += SUM_THREADS) {
        const int64_t at = (int64_t)a.ids[t] - v0;
        if (at >= 0 && at < n) atomicOr(&present[at >> 5], 1u << (at & 31));
      }
      __syncthreads();
      auto absent = [&](int r) { return !((present[r >> 5] >> (r & 31)) & 1u); };
      if (a.D <= SHORT_ROW / (int)sizeof(E)) zero_short_rows(dtable + v0 * a.D, n, a.D, absent);
      else
        for (int r = threadIdx.x >> 5; r < n; r += SUM_THREADS / 32)
          if (absent(r)) zero_row(dtable + (v0 + r) * a.D, a.D);
      __syncthreads();
    }
  }
  __shared__ int2 few[FEW ? FEW_TOKENS : 1];
  if (FEW) {
    const int lane = threadIdx.x, id = lane < a.T ? a.ids[lane] : -1, key = lane >= a.T ? 0x7fffffff : id >= 0 && id < a.V ? id : a.V;
    if (lane < 32) {
      int rank = 0;
#pragma unroll
      for (int t = 0; t < 32; ++t) {
        const int k = __shfl_sync(0xffffffffu, key, t);
        rank += k < key || (k == key && t < lane);
      }
      few[rank] = make_int2(key, lane);
    }
    __syncthreads();
  } else {
    wait_for_sort();
    let_next_start();
  }
  auto pair = [&](int64_t i) { return FEW ? few[FEW ? i : 0] : __ldcg(a.sorted + i); };
  const O* dout = static_cast<const O*>(a.dout);
  const int groups = SUM_THREADS / a.tpr, lane = threadIdx.x % a.tpr;
  const int64_t items = (int64_t)a.pieces * a.slabs;
  const int group = threadIdx.x / a.tpr;
  const int64_t begin_item = a.spread ? (int64_t)group * gridDim.x + blockIdx.x : (int64_t)blockIdx.x * groups + group;
  for (int64_t item = begin_item; item < items; item += (int64_t)gridDim.x * groups) {
    using Row = Slice<O, V, singles(FEW)>;
    using Out = Slice<E, V, singles(FEW)>;
    constexpr int N = Row::C;
    const int p = (int)(item / a.slabs), col = Row::first((int)(item % a.slabs), a.tpr, lane);
    const int64_t first = (int64_t)p * a.piece, last = min((int64_t)a.T, first + a.piece);
    const bool in = col < a.D;
    auto key = [&](int64_t i) { return i >= 0 && i < a.T ? pair(i).x : -1; };
    const int before = key(first - 1), after = key(last), end = key(last - 1), far_before = key(first - a.piece - 1), far_after = key(last + a.piece);
    // the run at the piece's front came from before: a long one leaves its part here, a short one is the piece before's
    const bool skip = far_before != before && after != before;
    // and the run at its end goes on: a short one that begins here is followed to its end
    const bool follow = end == after && end != before && far_after != end;
    float acc[N];
    int run = -1;
    // tokens in flight: what 64 registers hold, but for single elements, whose addresses spill 60 to 128 bytes a thread (not the adding of
    // few tokens).  (32 tokens of 1001 elements, added: 43 us, with more of them 16; vectors, which would
    // have to spill for it, lose: 14 tokens of 6864 11 us, 16.)
    constexpr int U = FEW && V == 1 ? (ADD ? 4 : 8) : V == 1 || ADD ? 2 : 4;
    const int64_t most = follow ? min((int64_t)a.T, last + a.piece) : last;
    for (int64_t i = first; i < most; i += U) {
      int2 pr[U + 1];
      Row r[U];
      Out old[U];
#pragma unroll
      for (int u = 0; u <= U; ++u) pr[u] = i + u < a.T ? pair(i + u) : make_int2(a.V, 0);
      if (i >= last && pr[0].x != end) break;
      bool real[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        // (padding stands last)
        real[u] = in && pr[u].x < a.V && (i + u < last ? !(skip && pr[u].x == before) : i + u < most && pr[u].x == end);
        if (real[u]) r[u].load(dout + (int64_t)pr[u].y * a.D, col, a.tpr, a.D);
        // what the sum is added to, where the run ends here as a whole: requested with the rows, not after them
        if (ADD && real[u] && pr[u + 1].x != pr[u].x && pr[u].x != before)
          old[u].load(dtable + (int64_t)pr[u].x * a.D, col, a.tpr, a.D);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (!real[u]) continue;
        float f[N];
        r[u].get(f);
        const bool begins = pr[u].x != run;
        run = pr[u].x;
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] = begins ? f[e] : acc[e] + f[e];
        const bool goes_on = pr[u + 1].x == run, came = run == before;
        if (goes_on && (follow || i + u + 1 != last)) continue;
        if (came || goes_on) {
          float* at = a.parts + ((int64_t)p * 2 + (came ? 0 : 1)) * a.D;
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int c = V > 1 ? col + e : col + e * a.tpr;
            if (V > 1 || c < a.D) at[c] = acc[e];
          }
        } else {
          float g[N];
          if (ADD) old[u].get(g);
#pragma unroll
          for (int e = 0; e < N; ++e) g[e] = ADD ? fmaf(acc[e], a.scale, g[e]) : acc[e] * a.scale;
          Out o;
          o.put(g);
          o.store(dtable + (int64_t)run * a.D, col, a.tpr, a.D);
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ join
// Long runs.  The piece in which such a run begins has it in its second part, the ones after it in their first.
// A CTA takes 32 C columns of the runs that begin in every gridDim.y-th piece.  Words of a text occur so unevenly that a batch has dozens of
// them, most of a few pieces: each of those is one warp's, so that they are added beside one another.  A longer one's parts are added
// by all warps in turn.  (8192 x 4096, the ids' logarithms even: the call 101 us with all warps for every run, 89 so.)
constexpr int JOIN_WARPS = 16, JOIN_Y = 16, JOIN_CTAS = 256, WARP_PARTS = 10;   // JOIN_Y or more CTAs share the pieces, JOIN_CTAS in all where columns are few
template <class E, int C>
__global__ void __launch_bounds__(JOIN_WARPS * 32) embed_join_kernel(const SumArgs a) {
  __shared__ float sums[JOIN_WARPS][32 * C + 1];
  __shared__ int2 runs[JOIN_WARPS * 32];   // id, first piece
  __shared__ int ends[JOIN_WARPS * 32];    // and its last
  __shared__ int count;
  if (threadIdx.x == 0) count = 0;
  wait_for_predecessor();
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (blockIdx.x * 32 + lane) * C;
  E* dtable = static_cast<E*>(a.dtable);
  auto key = [&](int64_t i) { return __ldcg(a.sorted + i).x; };
  {   // all of this CTA's pieces at once: one that a run begins in and goes on from
    const int p = blockIdx.y + threadIdx.x * gridDim.y;
    if (p + 1 < a.pieces) {
      const int64_t first = (int64_t)p * a.piece, end = first + a.piece;
      const int run = key(end - 1), far = end + a.piece < a.T ? key(end + a.piece) : -1, before = p > 0 ? key(first - 1) : -1;
      if (run < a.V && far == run && before != run) {
        runs[atomicAdd(&count, 1)] = make_int2(run, p);   // (in any order: no sum depends on it)
      }
    }
  }
  __syncthreads();
  auto add = [&](float (&s)[C], int64_t part) {
    Raw<float, C> r;
    float f[C];
    r.load(a.parts + part * a.D + c);
    r.get(f);
#pragma unroll
    for (int e = 0; e < C; ++e) s[e] += f[e];
  };
  // A warp to a run: the last piece that begins with it, in two looks (every 32nd piece, then 32 pieces), and the sum of one of few parts.
  for (int i = warp; i < count; i += JOIN_WARPS) {
    const int2 run = runs[i];
    auto begins = [&](int q) { return q < a.pieces && key((int64_t)q * a.piece) == run.x; };
    int last = run.y + 32 * __popc(__ballot_sync(0xffffffffu, begins(run.y + 32 * (lane + 1))));
    last += __popc(__ballot_sync(0xffffffffu, begins(last + 1 + lane)));
    if (lane == 0) ends[i] = last;
    if (last - run.y > WARP_PARTS || c >= a.D) continue;
    float s[C], g[C];
#pragma unroll
    for (int e = 0; e < C; ++e) s[e] = 0.f;
    E* at = dtable + (int64_t)run.x * a.D + c;
    Raw<E, C> old, o;
    if (a.accumulate) old.load(at);
    add(s, (int64_t)run.y * 2 + 1);
#pragma unroll 8
    for (int q = run.y + 1; q <= last; ++q) add(s, (int64_t)q * 2);
    if (a.accumulate) old.get(g);
#pragma unroll
    for (int e = 0; e < C; ++e) s[e] = a.accumulate ? fmaf(s[e], a.scale, g[e]) : s[e] * a.scale;
    o.put(s);
    o.store(at);
  }
  __syncthreads();
  for (int i = 0; i < count; ++i) {   // the longer ones, by all warps
    const int2 run = runs[i];
    const int last = ends[i];
    if (last - run.y <= WARP_PARTS) continue;
    float s[C];
#pragma unroll
    for (int e = 0; e < C; ++e) s[e] = 0.f;
    if (c < a.D) {
      if (warp == 0) add(s, (int64_t)run.y * 2 + 1);
#pragma unroll 8
      for (int q = run.y + 1 + warp; q <= last; q += JOIN_WARPS) add(s, (int64_t)q * 2);
    }
#pragma unroll
    for (int e = 0; e < C; ++e) sums[warp][lane * C + e] = s[e];
    __syncthreads();
    for (int k = threadIdx.x; k < 32 * C; k += JOIN_WARPS * 32) {
      const int col = blockIdx.x * 32 * C + k;
      if (col >= a.D) break;
      float t = sums[0][k];
#pragma unroll
      for (int w = 1; w < JOIN_WARPS; ++w) t += sums[w][k];
      E* at = dtable + (int64_t)run.x * a.D + col;
      *at = E(a.accumulate ? fmaf(t, a.scale, (float)*at) : t * a.scale);
    }
    __syncthreads();
  }
}

// ------------------------------------------------------------------------------------------------ host
// (D: columns are counted in 32 bits, and steps of a few thousand go past the last one)
int check(const bdlm_embed_params* p) {
  if (p == nullptr || p->T < 0 || p->D <= 0 || p->V <= 0 || p->T > (1 << 30) || p->V > (1 << 30) || p->D > (1 << 30)) return BDLM_ERR_INVALID_ARG;
  if (p->table_dtype < BDLM_BF16 || p->table_dtype > BDLM_FP32 || p->out_dtype < BDLM_BF16 || p->out_dtype > BDLM_FP32) return BDLM_ERR_INVALID_ARG;
  if (p->out_dtype != p->table_dtype && p->table_dtype != BDLM_FP32) return BDLM_ERR_INVALID_ARG;
  if (!isfinite(p->scale) || (p->accumulate != 0 && p->accumulate != 1) || p->reserved != 0) return BDLM_ERR_INVALID_ARG;
  return BDLM_OK;
}
bool al(const void* x, unsigned bytes) { return (reinterpret_cast<uintptr_t>(x) & (bytes - 1)) == 0; }
bool sm100() {
  int dev = 0, major = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  return cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) == cudaSuccess && major == 10;
}
size_t align256(size_t x) { return (x + 255) / 256 * 256; }

constexpr int MAX_PIECES = 1024, MIN_PIECE = 8;
static_assert(MAX_PIECES <= JOIN_Y * JOIN_WARPS * 32 && MAX_PIECES <= 32 * 33, "a thread of the join per piece; two looks find a run's end");
int piece_of(int T) {
  if (T <= FEW_TOKENS) return FEW_TOKENS;
  const int n = (T + MAX_PIECES - 1) / MAX_PIECES; return n < MIN_PIECE ? MIN_PIECE : n;
}
int pieces_of(int T) { return (T + piece_of(T) - 1) / piece_of(T); }
size_t pairs_bytes(int T) { return align256((size_t)T * sizeof(int2)); }

// Elements a thread takes at a time: 16 bytes of the table, where rows are whole numbers of those.  (32 bytes of an fp32 table in two
// stores left half-written sectors: 45452 x 3224 took 174 us, now 106.)
template <class E> constexpr int vector_of() { return 16 / (int)sizeof(E); }
int vector_of(const bdlm_embed_params* p) {
  const int v = p->table_dtype == BDLM_FP32 ? vector_of<float>() : vector_of<bf16_t>();
  return p->D % v == 0 ? v : 1;
}
template <class T> struct Type { using type = T; };
// Calls f(table type, row type).
template <class F>
void by_types(const bdlm_embed_params* p, F f) {
  if (p->table_dtype == BDLM_BF16) f(Type<bf16_t>{}, Type<bf16_t>{});
  else if (p->table_dtype == BDLM_FP16) f(Type<__half>{}, Type<__half>{});
  else if (p->out_dtype == BDLM_BF16) f(Type<float>{}, Type<bf16_t>{});
  else if (p->out_dtype == BDLM_FP16) f(Type<float>{}, Type<__half>{});
  else f(Type<float>{}, Type<float>{});
}
int pow2_at_least(int n, int most) {
  int p = 1;
  while (p < n && p < most) p *= 2;
  return p;
}

}  // namespace
}  // namespace bdlm

using namespace bdlm;

extern "C" {

size_t bdlm_embed_workspace_bytes(const bdlm_embed_params* p) {
  if (check(p) != BDLM_OK) return 0;
  if (p->T <= FEW_TOKENS) return 0;
  return 2 * pairs_bytes(p->T) + align256((size_t)pieces_of(p->T) * 2 * p->D * sizeof(float));
}

int bdlm_embed_fwd(const bdlm_embed_params* p, const void* table, const int32_t* ids, void* out, void* cuda_stream) {
  const int rc = check(p);
  if (rc != BDLM_OK) return rc;
  if (table == nullptr || (p->T > 0 && (ids == nullptr || out == nullptr))) return BDLM_ERR_INVALID_ARG;
  if (!al(table, 16) || !al(out, 16) || !al(ids, 4)) return BDLM_ERR_INVALID_ARG;
  if (!sm100()) return BDLM_ERR_UNSUPPORTED;
  if (p->T == 0) return BDLM_OK;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  const int V = vector_of(p), nvec = p->D / V, tpr = pow2_at_least(V > 1 ? (nvec + 3) / 4 : (nvec + 7) / 8, 256), rows = 256 / tpr;
  const unsigned blocks = (unsigned)(((int64_t)p->T + rows - 1) / rows);
  by_types(p, [&](auto e, auto o) {
    using E = typename decltype(e)::type;
    using O = typename decltype(o)::type;
    auto kern = V > 1 ? embed_fwd_kernel<E, O, vector_of<E>()> : embed_fwd_kernel<E, O, 1>;
    kern<<<blocks, 256, 0, st>>>(static_cast<const E*>(table), ids, static_cast<O*>(out), p->T, p->D, p->V, tpr, p->scale);
  });
  return cudaGetLastError() == cudaSuccess ? BDLM_OK : BDLM_ERR_CUDA;
}

int bdlm_embed_bwd(const bdlm_embed_params* p, const void* dout, const int32_t* ids, void* dtable,
                   void* workspace, size_t workspace_bytes, void* cuda_stream) {
  const int rc = check(p);
  if (rc != BDLM_OK) return rc;
  if (dtable == nullptr || (p->T > 0 && (dout == nullptr || ids == nullptr))) return BDLM_ERR_INVALID_ARG;
  const bool few = p->T <= FEW_TOKENS;
  if (!few && workspace == nullptr) return BDLM_ERR_INVALID_ARG;
  if (!al(dout, 16) || !al(dtable, 16) || !al(workspace, 16) || !al(ids, 4)) return BDLM_ERR_INVALID_ARG;
  if (workspace_bytes < bdlm_embed_workspace_bytes(p)) return BDLM_ERR_WORKSPACE_TOO_SMALL;
  if (!sm100()) return BDLM_ERR_UNSUPPORTED;
  if (p->T == 0 && p->accumulate) return BDLM_OK;
  cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  char* ws = static_cast<char*>(workspace);
  int2 *sorted = reinterpret_cast<int2*>(ws), *other = reinterpret_cast<int2*>(ws + pairs_bytes(p->T));
  cudaError_t e = cudaSuccess;
  if (!few) {
    int key_bits = 1;
    while ((1ll << key_bits) <= p->V) ++key_bits;   // keys 0 .. V
    const int passes = (key_bits + DIGIT_BITS - 1) / DIGIT_BITS, bits = (key_bits + passes - 1) / passes;
    if (p->T <= RANK_MOST) {
      constexpr int PER = RANK_WARPS * RANK_TOKENS;
      e = launch_chained(embed_rank_kernel, false, (p->T + PER - 1) / PER, RANK_WARPS * 32, 0, st, 1, ids, p->T, p->V, sorted);
    } else {
      e = cudaFuncSetAttribute(embed_sort_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SORT_SMEM);
      if (e == cudaSuccess)
        e = launch_chained(embed_sort_kernel, false, SORT_CTAS, SORT_WARPS * 32, SORT_SMEM, st, SORT_CTAS, ids, p->T, p->V, passes, bits, sorted, other);
    }
    if (e != cudaSuccess) return BDLM_ERR_CUDA;
  }
  const int V = vector_of(p), slices = V > 1 ? p->D / V : (p->D + singles(few) - 1) / singles(few);
  SumArgs a = {};
  a.dout = dout; a.ids = ids; a.sorted = sorted; a.dtable = dtable;
  a.parts = reinterpret_cast<float*>(ws + 2 * pairs_bytes(p->T));
  a.T = p->T; a.D = p->D; a.V = p->V; a.piece = piece_of(p->T); a.pieces = pieces_of(p->T);
  // Where a warp would hold many pieces, which diverge, and few CTAs all of them: a warp to a piece, and pieces spread over the CTAs.
  // (8000 tokens of 7 elements 63 us, so 32; 4000 of 320, no longer so, 30, so 33.)
  a.spread = slices < 8;
  a.tpr = a.spread ? 32 : pow2_at_least(slices, GROUP_THREADS);
  a.slabs = (slices + a.tpr - 1) / a.tpr;
  a.scale = p->scale; a.accumulate = p->accumulate;
  const int64_t items = (int64_t)a.pieces * a.slabs, groups = SUM_THREADS / a.tpr;
  int64_t want = a.spread ? items : (items + groups - 1) / groups;
  if (!a.accumulate && want < ((int64_t)p->V + 15) / 16) want = ((int64_t)p->V + 15) / 16;
  const int64_t cap = (int64_t)device_sm_count() * 2;
  const unsigned blocks = (unsigned)(want < cap ? want : cap);
  by_types(p, [&](auto te, auto to) {
    using E = typename decltype(te)::type;
    using O = typename decltype(to)::type;
    auto by_add = [&](auto v, auto is_few) {
      constexpr int VEC = decltype(v)::value;
      constexpr bool FEW = decltype(is_few)::value;
      return a.accumulate ? embed_sum_kernel<E, O, VEC, true, FEW> : embed_sum_kernel<E, O, VEC, false, FEW>;
    };
    auto by_few = [&](auto v) { return few ? by_add(v, std::true_type{}) : by_add(v, std::false_type{}); };
    auto sum = V > 1 ? by_few(std::integral_constant<int, vector_of<E>()>{}) : by_few(std::integral_constant<int, 1>{});
    e = launch_chained(sum, !few, blocks, SUM_THREADS, 0, st, 1, a);
    if (e != cudaSuccess || a.pieces < 2) return;
    const int cols = p->D % 4 == 0 ? 128 : 32;
    cudaLaunchConfig_t cfg = {};
    const int gx = (p->D + cols - 1) / cols, gy = JOIN_CTAS / gx > JOIN_Y ? JOIN_CTAS / gx : JOIN_Y;
    cfg.gridDim = dim3((unsigned)gx, (unsigned)(a.pieces - 1 < gy ? a.pieces - 1 : gy));
    cfg.blockDim = dim3(JOIN_WARPS * 32);
    cfg.stream = st;
    cudaLaunchAttribute attr = {};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, cols == 128 ? embed_join_kernel<E, 4> : embed_join_kernel<E, 1>, (const SumArgs)a);
  });
  return e == cudaSuccess ? BDLM_OK : BDLM_ERR_CUDA;
}

}  // extern "C"
