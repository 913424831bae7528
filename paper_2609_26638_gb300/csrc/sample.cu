// sample.cu -- temperature, min-p, top-k and top-p, and the draw of a token
// from a given uniform number, in one launch and one pass over the logits.
//
//   w_i = exp((l_i - M) / T),  q_i = floor(w_i 2^40),  order: l falling, i rising
//
// Every step is a search for the token at which a running total of that order
// passes a target: top-k in the count, top-p in the mass, the draw in the mass
// that is left.  No row is sorted for it.  A row's logits stay in the shared
// memory of a cluster of blocks (a slice each); one pass puts mass and count
// into 2048 bins of equal width in d = (l - M) / T, which the blocks add up;
// prefix sums over the bins give the bin in which a target is passed, and only
// the tokens of that bin (typically 20 to 200) are gathered, ranked by counting
// and searched.  Where the bins up to it hold few tokens in all, they are
// gathered together and serve the later searches too.  A bin too full for the
// list (equal logits, a hot row) is divided further by the bits of the logit.
//
// Masses are integers of 40 bits, so sums are exact and the result does not
// depend on the order of atomics, the slices or the cluster.  (A 64-bit add in
// shared memory is a compare-and-swap loop: the low and the high word are added
// apart, the high one only when it changes.)
//
// Bound: the row is read once; what is left is the exponential and two or three
// shared-memory adds per logit, which is what the time goes into for many rows,
// and the chain of cluster barriers for few.
#include <cmath>

#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kThreads = 512;
constexpr int kBins = 2048;                 // four per thread
constexpr int kList = 512;                  // gathered tokens
constexpr float kBinsPerNat = 73.f;         // 2^-40 is at 27.73 nats: bin 2024
constexpr int kMostVocab = 262144;
constexpr int kMostCluster = 8;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int vocab, slice;                         // tokens of a block's slice, a multiple of 16
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  const float* u;
  int32_t* token;
  float* logprob;
  int32_t* kept;
};

struct Entry {
  uint32_t key, idx;
  unsigned long long mass, before;          // own mass, mass of the list's entries ahead of it
};

// The place where a running total passed its target: the token, and the totals
// up to and with it.
struct Cut {
  uint32_t idx;
  uint32_t count;
  unsigned long long mass;
};

struct Shared {
  uint32_t lo[kBins], hi[kBins], cnt[kBins];
  Entry list[kList];
  uint32_t rank[kList];                     // list entries ahead of each entry
  int list_n;
  float block_max;
  unsigned long long warp_mass[kThreads / 32];
  uint32_t warp_cnt[kThreads / 32];
  float warp_max[kThreads / 32];
  int best;                                 // lowest index of the largest logit
  // the crossing bin of a search: totals ahead of it, and its count
  int bin;
  unsigned long long bin_mass;
  uint32_t bin_before, bin_cnt;
  uint32_t tie_cnt;                         // tokens of the crossing key in this block's slice
  Cut cut;
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// Generic address of a peer block's copy of a shared-memory object.
template <class T>
__device__ __forceinline__ T* peer(T* p, uint32_t rank) {
  uint64_t g;
  asm volatile("mapa.u64 %0, %1, %2;" : "=l"(g) : "l"(reinterpret_cast<uint64_t>(p)), "r"(rank));
  return reinterpret_cast<T*>(g);
}

__device__ __forceinline__ void cluster_barrier() {
  __syncwarp();              // the barrier is a warp-aligned instruction
  cluster_sync_all();
}

// What a row's logits are measured with.
struct Scale {
  float top, inv_t;
  // d = (l - M) / T, the same two roundings everywhere
  __device__ __forceinline__ float d(float x) const {
    return x == top ? 0.f : __fmul_rn(__fsub_rn(x, top), inv_t);
  }
  __device__ __forceinline__ static float weight(float x, float d) {
    return x == -INFINITY ? 0.f : expf(d);
  }
  // floor(w 2^40) from the bits of w (0 <= w <= 1)
  __device__ __forceinline__ static unsigned long long mass(float w) {
    const uint32_t u = __float_as_uint(w);
    const int s = static_cast<int>(u >> 23) - 110;        // exponent - 127 + 40 - 23
    const uint32_t m = (u & 0x7FFFFFu) | 0x800000u;
    if (s < 0) return s < -23 ? 0ull : m >> -s;
    return static_cast<unsigned long long>(m) << s;
  }
  // bins rise as the logit falls; rounded by adding 1.5 * 2^23
  __device__ __forceinline__ static int bin(float d) {
    const float y = fminf(-d * kBinsPerNat, static_cast<float>(kBins - 1));
    return static_cast<int>(__float_as_uint(y + 12582912.f) & 0xFFFFu);
  }
};

template <int TYPE> struct Elem;             // GS_F16, GS_BF16, GS_F32
template <> struct Elem<GS_F16> { static constexpr int kBytes = 2, kVec = 8; };
template <> struct Elem<GS_BF16> { static constexpr int kBytes = 2, kVec = 8; };
template <> struct Elem<GS_F32> { static constexpr int kBytes = 4, kVec = 4; };

// A logit as it counts: NaN is -inf, -0 is 0.
__device__ __forceinline__ float as_logit(float x) { return x != x ? -INFINITY : x + 0.f; }

template <int TYPE>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  if constexpr (TYPE == GS_F32)
    return as_logit(static_cast<const float*>(p)[i]);
  else if constexpr (TYPE == GS_F16)
    return as_logit(__half2float(static_cast<const __half*>(p)[i]));
  else
    return as_logit(__bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]));
}

template <int TYPE>
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[Elem<TYPE>::kVec]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == GS_F32) {
      x[i] = as_logit(__uint_as_float(w[i]));
    } else {
      const float2 f = unpack2<TYPE == GS_BF16>(w[i]);
      x[2 * i] = as_logit(f.x);
      x[2 * i + 1] = as_logit(f.y);
    }
  }
}

template <int TYPE>
__device__ __forceinline__ uint4 all_empty() {   // a vector of -inf
  const uint32_t w = TYPE == GS_F32 ? 0xFF800000u : (TYPE == GS_BF16 ? 0xFF80FF80u : 0xFC00FC00u);
  return make_uint4(w, w, w, w);
}

// Inclusive prefix sum over the block's threads of (mass, count); totals too.
__device__ __forceinline__ void block_scan(Shared& sh, unsigned long long& m, uint32_t& c,
                                           unsigned long long& total_m, uint32_t& total_c) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int s = 1; s < 32; s *= 2) {
    const unsigned long long pm = __shfl_up_sync(0xFFFFFFFFu, m, s);
    const uint32_t pc = __shfl_up_sync(0xFFFFFFFFu, c, s);
    if (lane >= s) {
      m += pm;
      c += pc;
    }
  }
  __syncthreads();
  if (lane == 31) {
    sh.warp_mass[warp] = m;
    sh.warp_cnt[warp] = c;
  }
  __syncthreads();
  total_m = 0;
  total_c = 0;
  unsigned long long before_m = 0;
  uint32_t before_c = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w == warp) {
      before_m = total_m;
      before_c = total_c;
    }
    total_m += sh.warp_mass[w];
    total_c += sh.warp_cnt[w];
  }
  m += before_m;
  c += before_c;
}

// A histogram of the whole row, four bins to a thread: exclusive totals ahead
// of the thread's first bin, and the bins.
struct Histogram {
  unsigned long long before_m, m[4];
  uint32_t before_c, c[4];
};

// Adds up the cluster's bins (every block gets all of them).
__device__ void merge_bins(Shared& sh, Histogram& h, unsigned long long& total_m, uint32_t& total_c) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    h.m[i] = 0;
    h.c[i] = 0;
  }
  const uint32_t n = cluster_size();
  for (uint32_t r = 0; r < n; ++r) {
    const Shared* p = peer(&sh, r);
    const uint4 lo = reinterpret_cast<const uint4*>(p->lo)[threadIdx.x];
    const uint4 hi = reinterpret_cast<const uint4*>(p->hi)[threadIdx.x];
    const uint4 c = reinterpret_cast<const uint4*>(p->cnt)[threadIdx.x];
    const uint32_t l4[4] = {lo.x, lo.y, lo.z, lo.w}, h4[4] = {hi.x, hi.y, hi.z, hi.w},
                   c4[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      h.m[i] += (static_cast<unsigned long long>(h4[i]) << 32) + l4[i];
      h.c[i] += c4[i];
    }
  }
  unsigned long long m = h.m[0] + h.m[1] + h.m[2] + h.m[3];
  uint32_t c = h.c[0] + h.c[1] + h.c[2] + h.c[3];
  const unsigned long long own_m = m;
  const uint32_t own_c = c;
  block_scan(sh, m, c, total_m, total_c);
  h.before_m = m - own_m;
  h.before_c = c - own_c;
}

// The bin in which base + running total passes `target` (in the count or the
// mass): the first with a total above it.  Writes sh.bin, bin_mass, ...
__device__ void find_bin(Shared& sh, const Histogram& h, bool by_count, unsigned long long target,
                         unsigned long long base_m, uint32_t base_c) {
  unsigned long long m = base_m + h.before_m;
  uint32_t c = base_c + h.before_c;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool before = (by_count ? c : m) <= target;
    const bool after = (by_count ? c + h.c[i] : m + h.m[i]) > target;
    if (before && after) {
      sh.bin = static_cast<int>(threadIdx.x) * 4 + i;
      sh.bin_mass = m;
      sh.bin_before = c;
      sh.bin_cnt = h.c[i];
    }
    m += h.m[i];
    c += h.c[i];
  }
  __syncthreads();
}

template <int TYPE>
struct Row {
  static constexpr int V = Elem<TYPE>::kVec;
  const uint4* vecs;      // the slice in shared memory, padded with -inf to whole vectors
  int n_vecs;
  int first;              // index in the row of the first vector's first element
  Scale sc;
  float min_p;

  // f(x, index) for every logit of the slice, vectors dealt to the threads in turn
  template <class F>
  __device__ __forceinline__ void each(F f) const {
    for (int v = threadIdx.x; v < n_vecs; v += kThreads) {
      float x[V];
      unpack<TYPE>(vecs[v], x);
#pragma unroll
      for (int e = 0; e < V; ++e) f(x[e], first + v * V + e);
    }
  }
  // the same, a run of neighbouring vectors to each thread, in index order
  template <class F>
  __device__ __forceinline__ void each_in_order(F f) const {
    const int per = (n_vecs + kThreads - 1) / kThreads, v0 = threadIdx.x * per;
    for (int v = v0; v < min(n_vecs, v0 + per); ++v) {
      float x[V];
      unpack<TYPE>(vecs[v], x);
#pragma unroll
      for (int e = 0; e < V; ++e) f(x[e], first + v * V + e);
    }
  }
  // mass of a logit, 0 if min-p drops it
  __device__ __forceinline__ unsigned long long mass(float x, float d) const {
    const float w = Scale::weight(x, d);
    return w >= min_p ? Scale::mass(w) : 0ull;
  }
};

__device__ __forceinline__ void add_to_bin(Shared& sh, int b, unsigned long long m) {
  const uint32_t lo = static_cast<uint32_t>(m);
  uint32_t hi = static_cast<uint32_t>(m >> 32);
  hi += atomicAdd(&sh.lo[b], lo) > 0xFFFFFFFFu - lo ? 1u : 0u;
  if (hi) atomicAdd(&sh.hi[b], hi);
  atomicAdd(&sh.cnt[b], 1u);
}

__device__ __forceinline__ void clear_bins(Shared& sh) {
  const uint4 z = make_uint4(0, 0, 0, 0);
  reinterpret_cast<uint4*>(sh.lo)[threadIdx.x] = z;
  reinterpret_cast<uint4*>(sh.hi)[threadIdx.x] = z;
  reinterpret_cast<uint4*>(sh.cnt)[threadIdx.x] = z;
}

// Tokens that a search still has in view: of bins first_bin .. bin, those with
// a key in [key_lo, key_hi].
struct View {
  int first_bin, bin;
  uint32_t key_lo, key_hi;
  __device__ __forceinline__ bool has(int b, uint32_t key) const {
    return b >= first_bin && b <= bin && key >= key_lo && key <= key_hi;
  }
};

// Gathers the view's tokens in block 0's list.
template <int TYPE>
__device__ void gather(Shared& sh, const Row<TYPE>& row, const View& view) {
  Shared* home = peer(&sh, 0);
  // a logit whose d is this far below is in no bin of the view (half a bin of slack)
  const float least = -(static_cast<float>(view.bin) + 1.f) / kBinsPerNat;
  row.each([&](float x, int i) {
    const float d = row.sc.d(x);
    if (d < least) return;
    const uint32_t key = float_order_key(x);
    if (!view.has(Scale::bin(d), key)) return;
    const unsigned long long m = row.mass(x, d);
    if (m == 0) return;
    const int at = atomicAdd(&home->list_n, 1);
    if (at < kList) {
      Entry e;
      e.key = key;
      e.idx = static_cast<uint32_t>(i);
      e.mass = m;
      e.before = 0;
      home->list[at] = e;
    }
  });
  cluster_barrier();
}

// Block 0: each entry's rank, and the mass ahead of it, by counting.
__device__ void rank_list(Shared& sh) {
  const int n = sh.list_n;
  for (int e = threadIdx.x; e < n; e += kThreads) {
    const uint32_t key = sh.list[e].key, idx = sh.list[e].idx;
    unsigned long long before = 0;
    uint32_t rank = 0;
    for (int k = 0; k < n; ++k) {
      const Entry& o = sh.list[k];
      if (o.key > key || (o.key == key && o.idx < idx)) {
        before += o.mass;
        ++rank;
      }
    }
    sh.list[e].before = before;
    sh.rank[e] = rank;
  }
  __syncthreads();
}

// Block 0: the list's entry at which the total passes the target.
__device__ void cut_list(Shared& sh, bool by_count, unsigned long long target,
                         unsigned long long base_m, uint32_t base_c) {
  for (int e = threadIdx.x; e < sh.list_n; e += kThreads) {
    const unsigned long long m = base_m + sh.list[e].before, own = sh.list[e].mass;
    const uint32_t c = base_c + sh.rank[e];
    const bool here = by_count ? c == target : m <= target && target < m + own;
    if (here) sh.cut = {sh.list[e].idx, c + 1, m + own};
  }
  __syncthreads();
}

// One row's searches.  Every block of the cluster takes the same branches: the
// merged totals are the same in all of them.
template <int TYPE>
struct Search {
  Shared& sh;
  const Row<TYPE>& row;
  const Histogram& bins;     // of the row
  bool listed = false;       // block 0's list is the order's first tokens
  bool clean = true;         // list_n is 0

  // The cut at which the total passes `target`; valid in every block.
  __device__ Cut cross(bool by_count, unsigned long long target) {
    const uint32_t rank = cluster_rank();
    if (listed) {            // the list covers every later target: it only gets smaller
      if (rank == 0) cut_list(sh, by_count, target, 0, 0);
      return share();
    }
    find_bin(sh, bins, by_count, target, 0, 0);
    View view = {sh.bin, sh.bin, 0u, 0xFFFFFFFFu};
    unsigned long long base_m = sh.bin_mass;
    uint32_t base_c = sh.bin_before, count = sh.bin_cnt;
    if (base_c + count <= kList) {
      view.first_bin = 0;
      base_m = 0;
      base_c = 0;
      listed = true;
    }
    __syncthreads();         // sh.bin .. have been read
    if (!listed && count > kList) {
      // divide the bin by the logits' bits, eleven at a time
      for (int shift = 21; count > kList; shift = shift > 11 ? shift - 11 : 0) {
        clear_bins(sh);
        __syncthreads();
        row.each([&](float x, int) {
          const float d = row.sc.d(x);
          const uint32_t key = float_order_key(x);
          if (!view.has(Scale::bin(d), key)) return;
          const unsigned long long m = row.mass(x, d);
          if (m) add_to_bin(sh, (view.key_hi - key) >> shift, m);
        });
        cluster_barrier();
        Histogram h;
        unsigned long long total_m;
        uint32_t total_c;
        merge_bins(sh, h, total_m, total_c);
        find_bin(sh, h, by_count, target, base_m, base_c);
        const uint32_t bin = static_cast<uint32_t>(sh.bin);
        view.key_hi -= bin << shift;
        view.key_lo = view.key_hi - ((1u << shift) - 1u);
        base_m = sh.bin_mass;
        base_c = sh.bin_before;
        count = sh.bin_cnt;
        cluster_barrier();  // the peers have read this block's bins
        if (shift == 0) break;
      }
      if (count > kList) return cross_ties(view.key_hi, by_count, target, base_m, base_c);
    }
    if (!clean) {
      if (rank == 0 && threadIdx.x == 0) sh.list_n = 0;
      cluster_barrier();
    }
    clean = false;
    gather(sh, row, view);
    if (rank == 0) {
      rank_list(sh);
      cut_list(sh, by_count, target, base_m, base_c);
    }
    return share();
  }

 private:
  // Block 0's cut to all of them.
  __device__ Cut share() {
    cluster_barrier();
    const Cut c = peer(&sh, 0)->cut;
    cluster_barrier();      // and it may be written again
    return c;
  }

  // More than kList tokens of one logit: all have the same mass, and the one in
  // question is found by its place among them in index order.
  __device__ Cut cross_ties(uint32_t key, bool by_count, unsigned long long target,
                            unsigned long long base_m, uint32_t base_c) {
    const float x = __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
    const unsigned long long own = row.mass(x, row.sc.d(x));
    const uint32_t want =
        static_cast<uint32_t>(by_count ? target - base_c : (target - base_m) / own);
    uint32_t c = 0;
    row.each_in_order([&](float y, int) { c += float_order_key(y) == key; });
    unsigned long long unused = 0, total_m;
    uint32_t upto = c, total;
    block_scan(sh, unused, upto, total_m, total);
    if (threadIdx.x == 0) sh.tie_cnt = total;
    cluster_barrier();
    uint32_t before = upto - c;
    for (uint32_t r = 0; r < cluster_rank(); ++r) before += peer(&sh, r)->tie_cnt;
    if (want >= before && want < before + c) {
      uint32_t at = before;
      row.each_in_order([&](float y, int i) {
        if (float_order_key(y) != key) return;
        if (at++ == want)
          peer(&sh, 0)->cut = {static_cast<uint32_t>(i), base_c + want + 1,
                               base_m + own * (want + 1ull)};
      });
    }
    return share();
  }
};

template <int TYPE>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleArgs a) {
  constexpr int V = Elem<TYPE>::kVec, B = Elem<TYPE>::kBytes;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  uint4* vecs = reinterpret_cast<uint4*>(smem + (sizeof(Shared) + 15) / 16 * 16);
  const uint32_t rank = cluster_rank(), n_blocks = cluster_size();
  const int r = blockIdx.x / n_blocks;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  // ---- the slice into shared memory.  Global vectors are aligned: the slice
  // begins `skew` elements into its first vector, and what a vector holds of
  // other slices or of beyond the row counts as -inf.
  const int begin = min(a.vocab, static_cast<int>(rank) * a.slice);
  const int end = min(a.vocab, begin + a.slice);
  const uintptr_t addr = reinterpret_cast<uintptr_t>(a.logits) + (r * a.ld + begin) * B;
  const int skew = static_cast<int>(addr % 16) / B;
  const uint4* src = reinterpret_cast<const uint4*>(addr - addr % 16);
  const int n_vecs = end > begin ? (end - begin + skew + V - 1) / V : 0;
  float top = -INFINITY;
#pragma unroll 4
  for (int v = threadIdx.x; v < n_vecs; v += kThreads) {
    const int e0 = v * V - skew;
    uint4 x = all_empty<TYPE>();
    if (e0 >= 0 && e0 + V <= end - begin) {
      x = src[v];
    } else {                 // the first or the last vector: its own elements only
      uint8_t* to = reinterpret_cast<uint8_t*>(&x);
      const uint8_t* from = reinterpret_cast<const uint8_t*>(src + v);
      for (int e = 0; e < V; ++e)
        if (e0 + e >= 0 && e0 + e < end - begin)
          for (int k = 0; k < B; ++k) to[e * B + k] = from[e * B + k];
    }
    vecs[v] = x;
    float f[V];
    unpack<TYPE>(x, f);
#pragma unroll
    for (int e = 0; e < V; ++e) top = fmaxf(top, f[e]);
  }
  clear_bins(sh);
#pragma unroll
  for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
  if (lane == 0) sh.warp_max[warp] = top;
  if (threadIdx.x == 0) {
    sh.list_n = 0;
    sh.best = kMostVocab;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) top = fmaxf(top, sh.warp_max[w]);
  if (threadIdx.x == 0) sh.block_max = top;
  cluster_barrier();
  for (uint32_t p = 0; p < n_blocks; ++p) top = fmaxf(top, peer(&sh, p)->block_max);

  const float t = a.temperature ? a.temperature[r] : 1.f;
  const bool greedy = !(t > 0.f);
  Row<TYPE> row;
  row.vecs = vecs;
  row.n_vecs = n_vecs;
  row.first = begin - skew;
  row.sc = {top, greedy ? 0.f : __fdiv_rn(1.f, t)};
  row.min_p = a.min_p ? a.min_p[r] : 0.f;
  row.min_p = row.min_p > 0.f ? fminf(row.min_p, 1.f) : 0.f;   // NaN: none

  int token = -1;
  float logprob = -INFINITY;
  uint32_t kept = 0;
  if (top == -INFINITY) {
    cluster_barrier();       // nothing to draw from; the peers have read block_max
  } else if (greedy) {
    row.each([&](float x, int i) {
      if (x == top) atomicMin(&peer(&sh, 0)->best, i);
    });
    cluster_barrier();
    token = sh.best;         // block 0 writes it
    logprob = 0.f;
    kept = 1;
  } else {
    row.each([&](float x, int) {
      const float d = row.sc.d(x);
      const unsigned long long m = row.mass(x, d);
      if (m) add_to_bin(sh, Scale::bin(d), m);
    });
    cluster_barrier();
    Histogram bins;
    unsigned long long mass;
    merge_bins(sh, bins, mass, kept);
    cluster_barrier();      // before any block clears its bins again
    Search<TYPE> search{sh, row, bins};
    const int k = a.top_k ? a.top_k[r] : 0;
    if (k > 0 && static_cast<uint32_t>(k) < kept) {
      const Cut c = search.cross(true, static_cast<unsigned long long>(k - 1));
      mass = c.mass;
      kept = c.count;
    }
    const float p = a.top_p ? a.top_p[r] : 1.f;
    if (p < 1.f) {
      const double need = ceil(static_cast<double>(p) * static_cast<double>(mass));
      const Cut c = search.cross(false, need > 1.0 ? static_cast<unsigned long long>(need) - 1 : 0);
      mass = c.mass;
      kept = c.count;
    }
    float u = a.u[r];
    u = u > 0.f ? fminf(u, 1.f) : 0.f;
    unsigned long long at =
        static_cast<unsigned long long>(static_cast<double>(u) * static_cast<double>(mass));
    if (at >= mass) at = mass - 1;
    const Cut c = search.cross(false, at);
    token = static_cast<int>(c.idx);
    if (rank == 0 && threadIdx.x == 0)       // from d: the integer weight of an unlikely token is coarse
      logprob = static_cast<float>(row.sc.d(load_logit<TYPE>(a.logits, r * a.ld + token)) -
                                   log(static_cast<double>(mass) * 0x1p-40));
  }
  if (rank == 0 && threadIdx.x == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = logprob;
    if (a.kept) a.kept[r] = static_cast<int32_t>(kept);
  }
}

// Blocks that share a row: as many as keep one wave of the GPU busy (three
// blocks fit an SM while a slice is at most 32 KB), at least what holds the
// row in shared memory.
constexpr int kSliceBytes = 96 * 1024;
int cluster_for(int rows, int vocab, int bytes) {
  int n = 1;
  while (n < kMostCluster &&
         (static_cast<int64_t>(vocab) * bytes > static_cast<int64_t>(n) * kSliceBytes ||
          (rows * static_cast<int64_t>(n) < 2 * kNumSMs && vocab > n * 4096)))
    n *= 2;
  return n;
}

template <int TYPE>
cudaError_t launch_sample(SampleArgs a, int rows, cudaStream_t s) {
  constexpr int B = Elem<TYPE>::kBytes;
  constexpr size_t head = (sizeof(Shared) + 15) / 16 * 16;
  constexpr int wide = kMostVocab / kMostCluster * B, most = wide > kSliceBytes ? wide : kSliceBytes;
  static DeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(sample_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(head) + most + 64);
  });
  if (e != cudaSuccess) return e;
  const int n = cluster_for(rows, a.vocab, B);
  a.slice = ((a.vocab + n - 1) / n + 15) / 16 * 16;
  const size_t smem = head + static_cast<size_t>(a.slice) * B + 32;
  return launch_ex(sample_kernel<TYPE>, dim3(rows * n), dim3(kThreads), smem, s, false, dim3(n, 1, 1),
                   a);
}

}  // namespace
}  // namespace gs

extern "C" int gs_sample(const void* logits, int64_t ld, int rows, int vocab, int dtype,
                         const gs_sample_params* params, const float* u, int32_t* token,
                         float* logprob, int32_t* kept, void* stream) {
  using namespace gs;
  if (!logits || !params || !u || !token || rows < 0 || vocab < 1 || ld < vocab)
    return GS_ERR_INVALID_ARG;
  if (dtype != GS_F16 && dtype != GS_BF16 && dtype != GS_F32) return GS_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(logits) % (dtype == GS_F32 ? 4 : 2)) return GS_ERR_INVALID_ARG;
  if (vocab > kMostVocab || rows > (1 << 24)) return GS_ERR_UNSUPPORTED;
  if (rows == 0) return GS_OK;
  SampleArgs a;
  a.logits = logits;
  a.ld = ld;
  a.vocab = vocab;
  a.temperature = params->temperature;
  a.top_p = params->top_p;
  a.min_p = params->min_p;
  a.top_k = params->top_k;
  a.u = u;
  a.token = token;
  a.logprob = logprob;
  a.kept = kept;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  const cudaError_t e = dtype == GS_F16    ? launch_sample<GS_F16>(a, rows, s)
                        : dtype == GS_BF16 ? launch_sample<GS_BF16>(a, rows, s)
                                           : launch_sample<GS_F32>(a, rows, s);
  return e == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
