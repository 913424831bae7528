// sample.cu -- temperature, min-p, top-k and top-p, and the draw of a token
// from a given uniform number, in one launch.
//
//   w_i = exp((l_i - M) / T),  q_i = floor(w_i 2^40),  order: l falling, i rising
//
// Every step is a search for the token at which a running total of that order
// passes a target: top-k in the count, top-p in the mass, the draw in the mass
// that is left.  No row is sorted for it.  A row is one block's, or, where there
// are few, a cluster's, a slice each.  The first pass finds the largest logit
// and, from the maxima of the threads' first logits, a level that about 3500
// logits of the row exceed, if logits do not depend on their place (see below).
// The second (the row is in L2 by then) notes these, the head, in shared memory and adds up the
// weights of the others.  The head goes into 512 bins of equal width in
// d = (l - M) / T; the blocks add up their bins; prefix sums over them give the
// bin in which a target is passed, and only the tokens of that bin are gathered
// in block 0, ranked by counting and searched.  Where the bins up to it hold few
// tokens in all, they are gathered together and serve the later searches too.  A
// target behind the head takes a pass for each 8 nats; a bin too full for the
// list (equal logits, a hot row) is divided further by the bits of the logit,
// and a logit too frequent for it by index.
//
// Masses are integers of 40 bits, so sums are exact and the result does not
// depend on the order of atomics, the slices or the cluster.  (A 64-bit add in
// shared memory is a compare-and-swap loop: the low and the high word are added
// apart, the high one only when it changes.)
//
// Many rows are bound by instruction issue, about 59 a logit, half of them for
// its weight: 544 rows of 59,392 (bf16, top-p) take 81 us, 12% of the copy rate
// (98 us with a head of 3000 tokens instead of 3500: more rows end behind it).
// Few rows are bound by the chain of passes and barriers: one row of 4096 takes
// 9 us, 32 rows of 59,392 (fp32, mixed settings) 17 us.
//
// The level is sampled at the start of each slice, and a slice without a finite
// logit leaves the row without one: nearly all of it is head then.  Where logits
// do depend on their place, draws are the same and take longer: the 544 rows
// above 80 us shuffled, 199 rising, 120 falling, 153 with the first half at -inf, 71 with
// the second; 32 rows of that kind (fp32) 17.5 us, and 31 to 32 for any of these.
// A draw far behind the head costs the same: without top-p the 544 rows take 172.
#include <cmath>
#include <cstddef>

#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kThreads = 512;
constexpr int kBins = kThreads;             // one per thread
constexpr int kBinBits = 9;
constexpr float kNats = 8.f;                // of a window behind the head
constexpr float kBinsPerNat = kBins / kNats;
constexpr int kWindows = 5;                 // the head, and 32 nats: 2^-40 is at 27.73
constexpr int kList = 256;                  // gathered tokens
constexpr int kPrefix = 64;                 // of which the order's first ones, kept for later searches
constexpr int kHead = 4096;                 // head tokens that a block notes
constexpr double kTarget = 3500.;           // head tokens of a row that the level aims at,
constexpr double kShare = 0.125;            // or this share of a smaller vocabulary;
constexpr int kSmall = 512;                 // one of so few tokens is all head
constexpr int kMostVocab = 262144;
constexpr int kMostCluster = 8;

struct SampleArgs {
  const void* logits;
  int64_t ld;
  int vocab, slice;                         // tokens of a block's slice, a multiple of 16
  // of 32 threads' maxima over their first level_vecs vectors, which sets the level
  int level_vecs, level_rank;
  const float *temperature, *top_p, *min_p;
  const int32_t* top_k;
  const float* u;
  int32_t* token;
  float* logprob;
  int32_t* kept;
};

struct alignas(16) Entry {
  unsigned long long mass;
  uint32_t key, idx;
};

// The place where a running total passed its target: the token, and the totals
// up to and with it.
struct Cut {
  uint32_t idx;
  uint32_t count;
  unsigned long long mass;
};

// A row's settings, read once: all blocks of its cluster take the same branches
// whatever happens to the arrays meanwhile.
struct Settings {
  float t, top_p, min_p, u;
  int top_k;
};

struct Shared {
  Entry list[kList];
  unsigned long long before[kList];         // mass of the list's entries ahead of each
  uint32_t rank[kList];                     // and their number
  alignas(16) uint32_t lo[kBins], hi[kBins], cnt[kBins];    // read four at a time
  unsigned long long head_upto_m[kBins];    // the head's merged bins: totals up to and with each
  uint32_t head_upto_c[kBins];
  float2 head[kHead];                       // the slice's logits in the head, and (as bits) their places
  alignas(16) uint4 edge[2];                // the slice's first and last vector
  unsigned long long warp_mass[kThreads / 32];
  // of every block, written by it: the mass and number of its other tokens
  unsigned long long tail_mass[kMostCluster];
  uint32_t tail_cnt[kMostCluster];
  float block_max[kMostCluster], block_level[kMostCluster];
  unsigned long long own_tail_mass;
  uint32_t own_tail_cnt;
  uint32_t warp_cnt[kThreads / 32];
  float warp_max[kThreads / 32], warp_level[kThreads / 32];
  int head_n;                               // may pass kHead: then the list is not used
  int list_n;
  int best;                                 // lowest index of the largest logit
  // the crossing bin of a search: totals ahead of it, and its count
  int bin;
  uint32_t bin_before, bin_cnt;
  unsigned long long bin_mass;
  uint32_t tie_cnt;                         // tokens of the crossing key in this block's slice
  Settings set;
  Cut cut[3];                               // of each search
};

static_assert(offsetof(Shared, lo) % 16 == 0 && offsetof(Shared, hi) % 16 == 0 &&
                  offsetof(Shared, cnt) % 16 == 0 && offsetof(Shared, edge) % 16 == 0 &&
                  sizeof(Entry) == 16 && offsetof(Shared, list) % 16 == 0,
              "read as vectors");

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

template <int TYPE> struct Elem;             // GS_F16, GS_BF16, GS_F32
template <> struct Elem<GS_F16> { static constexpr int kBytes = 2, kVec = 8; };
template <> struct Elem<GS_BF16> { static constexpr int kBytes = 2, kVec = 8; };
template <> struct Elem<GS_F32> { static constexpr int kBytes = 4, kVec = 4; };

template <int TYPE>
__device__ __forceinline__ float load_logit(const void* p, int64_t i) {
  if constexpr (TYPE == GS_F32)
    return static_cast<const float*>(p)[i];
  else if constexpr (TYPE == GS_F16)
    return __half2float(static_cast<const __half*>(p)[i]);
  else
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

template <int TYPE>
__device__ __forceinline__ void unpack(const uint4& v, float (&x)[Elem<TYPE>::kVec]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if constexpr (TYPE == GS_F32) {
      x[i] = __uint_as_float(w[i]);
    } else {
      const float2 f = unpack2<TYPE == GS_BF16>(w[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
}

// Elementwise maximum of packed logits (a NaN gives the other operand).
template <int TYPE>
__device__ __forceinline__ uint32_t max_packed(uint32_t a, uint32_t b) {
  uint32_t r;
  if constexpr (TYPE == GS_F32) {
    r = __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
  } else if constexpr (TYPE == GS_F16) {
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  } else {
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  }
  return r;
}
// The larger half of a packed pair.
template <int TYPE>
__device__ __forceinline__ float widest(uint32_t v) {
  if constexpr (TYPE == GS_F32) {
    return __uint_as_float(v);
  } else {
    const float2 f = unpack2<TYPE == GS_BF16>(v);
    return fmaxf(f.x, f.y);
  }
}
template <int TYPE>
constexpr uint32_t kEmpty = TYPE == GS_F32 ? 0xFF800000u : (TYPE == GS_BF16 ? 0xFF80FF80u : 0xFC00FC00u);

// What a row's logits are weighed with.  1 / T is kept within fp32's normal
// range, so that a logit of -inf is at d = -inf for every T.
struct Scale {
  float top, inv_t, min_p;
  float edge, per_nat;       // the head: d >= edge, and its bins
  // d = (l - M) / T, the same two roundings everywhere
  __device__ __forceinline__ float d(float x) const { return __fmul_rn(__fsub_rn(x, top), inv_t); }
  // the weight, 0 if min-p drops it
  __device__ __forceinline__ float weight(float d) const {
    const float w = expf(d);
    return w >= min_p ? w : 0.f;
  }
  // floor(w 2^40) from the bits of w (0 <= w <= 1)
  __device__ __forceinline__ static unsigned long long mass(float w) {
    const uint32_t u = __float_as_uint(w);
    const int s = static_cast<int>(u >> 23) - 110;        // exponent - 127 + 40 - 23
    const uint32_t m = (u & 0x7FFFFFu) | 0x800000u;
    if (s < 0) return s < -23 ? 0ull : m >> -s;
    return static_cast<unsigned long long>(m) << s;
  }
  // The windows: 0 is the head, w >= 1 the w-th 8 nats behind it.
  __device__ __forceinline__ float end_of(int w) const { return fmaf(-kNats, w, edge); }
  __device__ __forceinline__ bool in(int w, float d) const {
    return d >= end_of(w) && (w == 0 || d < end_of(w - 1));
  }
  // bins rise as the logit falls; rounded by adding 1.5 * 2^23
  __device__ __forceinline__ int bin(int w, float d) const {
    const float y = w == 0 ? -d * per_nat : (end_of(w - 1) - d) * kBinsPerNat;
    return static_cast<int>(
        __float_as_uint(fminf(fmaxf(y, 0.f), static_cast<float>(kBins - 1)) + 12582912.f) & 0xFFFFu);
  }
  __device__ __forceinline__ static uint32_t key(float x) { return float_order_key(x + 0.f); }
};

// floor(p Z) for 0 <= p <= 1, exactly; `whole` if nothing is cut off.  (In
// integers: this GPU's 64-bit floating-point units are few, and a block's 16
// warps would queue for them.)
__device__ __forceinline__ unsigned long long share_of(float p, unsigned long long z, bool& whole) {
  const uint32_t u = __float_as_uint(p), e = u >> 23;
  if (e < 23) {              // below 2^-104: p Z < 1
    whole = p == 0.f;
    return 0;
  }
  const unsigned long long m = (u & 0x7FFFFFu) | 0x800000u;
  const int s = 150 - static_cast<int>(e);      // p = m 2^-s, 23 <= s <= 127
  const unsigned long long lo = z * m, hi = __umul64hi(z, m);
  if (s < 64) {
    whole = lo << (64 - s) == 0;
    return hi << (64 - s) | lo >> s;
  }
  whole = lo == 0 && (s == 64 || hi << (128 - s) == 0);
  return hi >> (s - 64);
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

// The whole row's bins, one to a thread: totals up to and with it, and its own.
struct Bins {
  unsigned long long upto_m, m, total_m;
  uint32_t upto_c, c, total_c;
};

// Adds up the cluster's bins (every block gets all of them).
__device__ __forceinline__ Bins merge_bins(Shared& sh) {
  Bins h;
  const uint32_t n = cluster_size();
  unsigned long long m = 0;
  uint32_t c = 0;
  if (n == 1) {
    __syncthreads();
    m = (static_cast<unsigned long long>(sh.hi[threadIdx.x]) << 32) + sh.lo[threadIdx.x];
    c = sh.cnt[threadIdx.x];
  } else {
    // Four neighbouring threads take the same four bins, 16 bytes a load, of
    // every fourth peer, and exchange sums: one round trip through the cluster.
    const int quad = threadIdx.x / 4, part = threadIdx.x % 4;
    unsigned long long ms[4] = {};
    uint32_t cs[4] = {};
#pragma unroll
    for (int k = 0; k < kMostCluster / 4; ++k) {
      const uint32_t p = part + 4 * k;
      if (p >= n) continue;
      const Shared* from = peer(&sh, p);
      const uint4 lo = reinterpret_cast<const uint4*>(from->lo)[quad];
      const uint4 hi = reinterpret_cast<const uint4*>(from->hi)[quad];
      const uint4 cn = reinterpret_cast<const uint4*>(from->cnt)[quad];
      const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, u[4] = {hi.x, hi.y, hi.z, hi.w},
                     w[4] = {cn.x, cn.y, cn.z, cn.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        ms[i] += (static_cast<unsigned long long>(u[i]) << 32) + l[i];
        cs[i] += w[i];
      }
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int s = 1; s < 4; s *= 2) {
        ms[i] += __shfl_xor_sync(0xFFFFFFFFu, ms[i], s);
        cs[i] += __shfl_xor_sync(0xFFFFFFFFu, cs[i], s);
      }
      if (i == part) {
        m = ms[i];
        c = cs[i];
      }
    }
  }
  h.m = m;
  h.c = c;
  block_scan(sh, m, c, h.total_m, h.total_c);
  h.upto_m = m;
  h.upto_c = c;
  return h;
}

// The bin in which base + running total passes `target` (in the count or the
// mass).  Writes sh.bin, bin_mass, bin_before, bin_cnt.
__device__ __forceinline__ void find_bin(Shared& sh, const Bins& h, bool by_count,
                                         unsigned long long target, unsigned long long base_m,
                                         uint32_t base_c) {
  const unsigned long long m = base_m + h.upto_m - h.m;
  const uint32_t c = base_c + h.upto_c - h.c;
  __syncthreads();           // the last search's numbers have been read
  if (by_count ? c <= target && c + h.c > target : m <= target && m + h.m > target) {
    sh.bin = static_cast<int>(threadIdx.x);
    sh.bin_mass = m;
    sh.bin_before = c;
    sh.bin_cnt = h.c;
  }
  __syncthreads();
}

__device__ __forceinline__ void add_to_bin(Shared& sh, int b, unsigned long long m) {
  const uint32_t lo = static_cast<uint32_t>(m);
  uint32_t hi = static_cast<uint32_t>(m >> 32);
  hi += atomicAdd(&sh.lo[b], lo) > 0xFFFFFFFFu - lo ? 1u : 0u;
  if (hi) atomicAdd(&sh.hi[b], hi);
  atomicAdd(&sh.cnt[b], 1u);
}

__device__ __forceinline__ void clear_bins(Shared& sh) {
  sh.lo[threadIdx.x] = 0;
  sh.hi[threadIdx.x] = 0;
  sh.cnt[threadIdx.x] = 0;
}

// Tokens that a search still has in view: of a window's bins first .. last,
// those with a key in [key_lo, key_hi].
struct View {
  int window, first, last;
  uint32_t key_lo, key_hi;
};

// A block's slice of a row, as aligned vectors.  What the first and the last
// vector hold of other slices, or of beyond the row, counts as -inf: these two
// are in shared memory, the others are read where they are.
template <int TYPE>
struct Slice {
  static constexpr int V = Elem<TYPE>::kVec;
  const uint4* vecs;
  const uint4* edge;
  int n_vecs, v0, v1;     // vectors v0 .. v1 - 1 are whole
  int first;              // index in the row of the first vector's first element
  Scale sc;

  __device__ __forceinline__ uint4 load(int v) const {
    const uint4* p = v >= v0 && v < v1 ? vecs + v : edge + (v == 0 ? 0 : 1);
    return *p;
  }
  // NaN as -inf
  __device__ __forceinline__ static uint4 no_nan(uint4 x) {
    x.x = max_packed<TYPE>(x.x, kEmpty<TYPE>);
    x.y = max_packed<TYPE>(x.y, kEmpty<TYPE>);
    x.z = max_packed<TYPE>(x.z, kEmpty<TYPE>);
    x.w = max_packed<TYPE>(x.w, kEmpty<TYPE>);
    return x;
  }
  // f(vector's first element, its logits), vectors dealt to the threads in
  // turn; the next two are on their way meanwhile
  template <class F>
  __device__ __forceinline__ void each_vec(F f) const {
    int v = threadIdx.x;
    uint4 q0 = {}, q1 = {};
    if (v < n_vecs) q0 = load(v);
    if (v + kThreads < n_vecs) q1 = load(v + kThreads);
#pragma unroll 1
    for (; v < n_vecs; v += kThreads) {
      uint4 q2 = {};
      if (v + 2 * kThreads < n_vecs) q2 = load(v + 2 * kThreads);
      float x[V];
      unpack<TYPE>(no_nan(q0), x);
      f(v * V, x);
      q0 = q1;
      q1 = q2;
    }
  }
  // a logit by its place, which is one of the slice's own
  __device__ __forceinline__ float at(int i) const {
    const float x = load_logit<TYPE>(vecs, i);
    return x == x ? x : -INFINITY;
  }
  // f(x, d, element) for the logits with d in [least, most): few of them, so a
  // vector's are marked first and then taken one by one, and a warp goes
  // through f as often as its fullest lane, not once per element.
  template <class F>
  __device__ __forceinline__ void each_within(float least, float most, F f) const {
    each_vec([&](int i, const float (&x)[V]) {
      uint32_t marked = 0;
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const float d = sc.d(x[e]);
        if (d >= least && d < most) marked |= 1u << e;
      }
      while (marked) {
        const int k = i + __ffs(marked) - 1;
        marked &= marked - 1;
        const float y = at(k);
        f(y, sc.d(y), k);
      }
    });
  }
  // f(key, mass, element) for the tokens of a view that have a weight
  template <class F>
  __device__ __forceinline__ void each_in(const Shared& sh, const View& view, F f) const {
    auto take = [&](float x, float d, int i) {
      if (!sc.in(view.window, d)) return;
      const int b = sc.bin(view.window, d);
      const uint32_t key = Scale::key(x);
      if (b < view.first || b > view.last || key < view.key_lo || key > view.key_hi) return;
      const unsigned long long m = Scale::mass(sc.weight(d));
      if (m) f(key, m, i);
    };
    if (view.window == 0 && sh.head_n <= kHead) {
      for (int k = threadIdx.x; k < sh.head_n; k += kThreads) {
        const float2 h = sh.head[k];
        take(h.x, sc.d(h.x), __float_as_int(h.y));
      }
    } else {
      // half a bin and more on either side; the bin itself decides
      const float from = view.window == 0 ? 0.f : sc.end_of(view.window - 1);
      const float width = view.window == 0 ? 1.f / sc.per_nat : 1.f / kBinsPerNat;
      const float least = from - (static_cast<float>(view.last) + 1.f) * width;
      const float most =
          view.first == 0 ? INFINITY : from - (static_cast<float>(view.first) - 1.f) * width;
      each_within(view.last == kBins - 1 ? sc.end_of(view.window) : least, most, take);
    }
  }
  // f(element) for the tokens of this key in the thread's run of neighbouring
  // vectors, in index order
  template <class F>
  __device__ __forceinline__ void each_tie(uint32_t key, F f) const {
    const int per = (n_vecs + kThreads - 1) / kThreads, begin = threadIdx.x * per;
#pragma unroll 1
    for (int v = begin; v < min(n_vecs, begin + per); ++v) {
      float x[V];
      unpack<TYPE>(no_nan(load(v)), x);
#pragma unroll
      for (int e = 0; e < V; ++e)
        if (Scale::key(x[e]) == key) f(v * V + e);
    }
  }
};

// One row's searches.  Every block of the cluster takes the same branches: the
// merged totals are the same in all of them.  Everything is inlined: a call that
// takes `this` puts the whole state into local memory (544 rows 92 us instead of
// 83, 32 rows 21 instead of 17.5).
template <int TYPE>
struct Search {
  Shared& sh;
  const Slice<TYPE>& row;
  Bins bins;                 // of the window below, and the totals ahead of it
  unsigned long long ahead_m = 0;
  uint32_t ahead_c = 0;
  int window = 0;
  bool dirty = false;        // peers may still be reading this block's bins
  bool listed = false;       // block 0's list is the order's first tokens
  int n_cuts = 0;

  // The cut at which the total passes `target`, in every block, or in block 0
  // alone if it is the last one.
  __device__ Cut cross(bool by_count, unsigned long long target, bool last) {
    const uint32_t rank = cluster_rank();
    if (listed) {            // the list covers every later target: they only get smaller
      if (rank == 0) cut_list(by_count, target, last);
      return share(last);
    }
    move_window(by_count, target);
    find_bin(sh, bins, by_count, target, ahead_m, ahead_c);
    View view = {window, sh.bin, sh.bin, 0u, 0xFFFFFFFFu};
    unsigned long long base_m = sh.bin_mass;
    uint32_t base_c = sh.bin_before, count = sh.bin_cnt;
    if (window == 0 && base_c + count <= kPrefix) {
      view.first = 0;
      base_m = 0;
      base_c = 0;
      listed = true;
    } else if (count > kList) {
      // divide the bin by the logits' bits
      for (int shift = 32 - kBinBits;; shift = shift > kBinBits ? shift - kBinBits : 0) {
        const Bins part = fill_bins([&] {
          row.each_in(sh, view, [&](uint32_t key, unsigned long long m, int) {
            add_to_bin(sh, (view.key_hi - key) >> shift, m);
          });
        });
        find_bin(sh, part, by_count, target, base_m, base_c);
        view.key_hi -= static_cast<uint32_t>(sh.bin) << shift;
        view.key_lo = view.key_hi - ((1u << shift) - 1u);
        base_m = sh.bin_mass;
        base_c = sh.bin_before;
        count = sh.bin_cnt;
        if (count <= kList || shift == 0) break;
      }
      if (count > kList) return cross_ties(view.key_hi, by_count, target, base_m, base_c, last);
    }
    gather(view);
    if (rank == 0) {
      rank_list(by_count, target, base_m, base_c, last);
      if (!listed && threadIdx.x == 0) sh.list_n = 0;
    }
    return share(last);
  }

 private:
  // The whole row's bins, filled anew.
  template <class F>
  __device__ Bins fill_bins(F fill) {
    if (dirty) cluster_barrier();
    dirty = true;
    clear_bins(sh);
    __syncthreads();
    fill();
    cluster_barrier();
    return merge_bins(sh);
  }

  // Brings the target into the window's bins.
  __device__ void move_window(bool by_count, unsigned long long target) {
    if (target < (by_count ? ahead_c : ahead_m)) {       // back to the head
      window = 0;
      ahead_m = 0;
      ahead_c = 0;
      const int i = threadIdx.x;
      bins = {sh.head_upto_m[i], sh.head_upto_m[i] - (i ? sh.head_upto_m[i - 1] : 0),
              sh.head_upto_m[kBins - 1], sh.head_upto_c[i],
              sh.head_upto_c[i] - (i ? sh.head_upto_c[i - 1] : 0), sh.head_upto_c[kBins - 1]};
    }
    while (window + 1 < kWindows &&
           target >= (by_count ? ahead_c + bins.total_c : ahead_m + bins.total_m)) {
      if (window == 0) {     // to come back to
        sh.head_upto_m[threadIdx.x] = bins.upto_m;
        sh.head_upto_c[threadIdx.x] = bins.upto_c;
      }
      ahead_m += bins.total_m;
      ahead_c += bins.total_c;
      ++window;
      bins = fill_bins([&] {
        row.each_within(row.sc.end_of(window), row.sc.end_of(window - 1), [&](float, float d, int) {
          const unsigned long long m = Scale::mass(row.sc.weight(d));
          if (m) add_to_bin(sh, row.sc.bin(window, d), m);
        });
      });
    }
  }

  // Gathers the view's tokens in block 0's list.
  __device__ void gather(const View& view) {
    Shared* home = peer(&sh, 0);
    row.each_in(sh, view, [&](uint32_t key, unsigned long long m, int i) {
      const int to = atomicAdd(&home->list_n, 1);
      if (to < kList) home->list[to] = {m, key, static_cast<uint32_t>(row.first + i)};
    });
    cluster_barrier();
    dirty = false;           // all blocks are past their merges
  }

  // Block 0: each entry's rank, and the mass ahead of it, by counting; an
  // entry's comparisons are shared by as many neighbouring threads as there are.
  // The one at which the total passes the target is told.
  __device__ void rank_list(bool by_count, unsigned long long target, unsigned long long base_m,
                            uint32_t base_c, bool last) {
    const int n = min(sh.list_n, kList);
    int share = 32;
    while (share > 1 && share * n > kThreads) share /= 2;
    const int e = threadIdx.x / share, part = threadIdx.x % share;
    unsigned long long before = 0;
    uint32_t rank = 0;
    const Entry own = sh.list[min(e, kList - 1)];
    for (int k = part; k < n; k += share) {
      const Entry o = sh.list[k];
      if (o.key > own.key || (o.key == own.key && o.idx < own.idx)) {
        before += o.mass;
        ++rank;
      }
    }
    __syncwarp();
    for (int s = 1; s < share; s *= 2) {
      before += __shfl_xor_sync(0xFFFFFFFFu, before, s);
      rank += __shfl_xor_sync(0xFFFFFFFFu, rank, s);
    }
    if (e < n && part == 0) {
      sh.before[e] = before;
      sh.rank[e] = rank;
      cut_at(own, base_m + before, base_c + rank, by_count, target, last);
    }
    __syncthreads();
  }

  // Block 0: the same from ranks that are known, in a list from the order's start.
  __device__ void cut_list(bool by_count, unsigned long long target, bool last) {
    const int e = threadIdx.x;
    if (e < min(sh.list_n, kList))
      cut_at(sh.list[e], sh.before[e], sh.rank[e], by_count, target, last);
  }
  __device__ __forceinline__ void cut_at(const Entry& e, unsigned long long m, uint32_t c,
                                         bool by_count, unsigned long long target, bool last) {
    if (by_count ? c == target : m <= target && target < m + e.mass)
      tell({e.idx, c + 1, m + e.mass}, last);
  }

  // Every block has the cut once all are past the barrier.  Each search has a
  // place of its own for it, so the next one's does not overwrite what a peer
  // still reads; the last one's is block 0's alone.
  __device__ void tell(const Cut& c, bool last) {
    const uint32_t n = last ? 1 : cluster_size();        // the peers may have ended
    for (uint32_t p = 0; p < n; ++p) peer(&sh, p)->cut[n_cuts] = c;
  }
  __device__ Cut share(bool last) {
    const int i = n_cuts++;
    if (last)
      __syncthreads();
    else
      cluster_barrier();
    return sh.cut[i];
  }

  // More than kList tokens of one logit: all have the same mass, and the one in
  // question is found by its place among them in index order.
  __device__ __forceinline__ Cut cross_ties(uint32_t key, bool by_count, unsigned long long target,
                                         unsigned long long base_m, uint32_t base_c, bool last) {
    const float x = __uint_as_float((key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key);
    const unsigned long long own = Scale::mass(row.sc.weight(row.sc.d(x)));
    const uint32_t want =
        static_cast<uint32_t>(by_count ? target - base_c : (target - base_m) / own);
    uint32_t c;
    uint32_t at = count_ties(key, c);
    if (want >= at && want < at + c)
      row.each_tie(key, [&](int i) {
        if (at++ == want)
          tell({static_cast<uint32_t>(row.first + i), base_c + want + 1,
                base_m + own * (want + 1ull)}, last);
      });
    cluster_barrier();       // the cut is there, and every peer's count has been read
    return share(last);
  }

  // Tokens of this key in the thread's run, and in the row ahead of it.
  __device__ __forceinline__ uint32_t count_ties(uint32_t key, uint32_t& c) {
    c = 0;
    row.each_tie(key, [&](int) { ++c; });
    unsigned long long none = 0, total_m;
    uint32_t upto = c, total;
    block_scan(sh, none, upto, total_m, total);
    if (threadIdx.x == 0) sh.tie_cnt = total;
    cluster_barrier();
    uint32_t at = upto - c;
    for (uint32_t r = 0; r < cluster_rank(); ++r) at += peer(&sh, r)->tie_cnt;
    return at;
  }

 public:
  // A row with infinite logits: a draw between these, which weigh the same.
  __device__ __forceinline__ Cut draw_infinite(const Settings& set) {
    const uint32_t key = Scale::key(INFINITY);
    uint32_t c;
    uint32_t at = count_ties(key, c), kept = 0;
    for (uint32_t r = 0; r < cluster_size(); ++r) kept += peer(&sh, r)->tie_cnt;
    if (set.top_k > 0) kept = min(kept, static_cast<uint32_t>(set.top_k));
    bool whole;
    if (set.top_p < 1.f) {
      const uint32_t n = static_cast<uint32_t>(share_of(fmaxf(set.top_p, 0.f), kept, whole));
      kept = max(n + (whole ? 0u : 1u), 1u);
    }
    const uint32_t want = min(
        static_cast<uint32_t>(share_of(set.u > 0.f ? fminf(set.u, 1.f) : 0.f, kept, whole)), kept - 1);
    if (want >= at && want < at + c)
      row.each_tie(key, [&](int i) {
        if (at++ == want) tell({static_cast<uint32_t>(row.first + i), kept, 0}, true);
      });
    cluster_barrier();
    return sh.cut[0];
  }
};

// One pass over the slice.  HEAD: the elements at or above the edge are noted.
// TAIL: the mass of the others, and (COUNT) their number.  A weight's 40 bits
// are taken as two sums: adding 8 (then 2^-17, to the rest) with rounding toward
// zero leaves floor(w 2^20) (then the next 20 bits) in the low bits of the result.
template <int TYPE, bool HEAD, bool TAIL, bool COUNT>
__device__ __forceinline__ void weigh(Shared& sh, const Slice<TYPE>& row) {
  constexpr int V = Elem<TYPE>::kVec;
  uint32_t hi = 0, lo = 0, n = 0;            // at most 528 elements a thread: below 2^30
  row.each_vec([&](int i, const float (&x)[V]) {
    uint32_t head = 0;
    const F32x2 top = join2(-row.sc.top, -row.sc.top), inv = join2(row.sc.inv_t, row.sc.inv_t);
    const F32x2 eight = join2(8.f, 8.f), low = join2(0x1p-17f, 0x1p-17f), minus = join2(-1.f, -1.f);
#pragma unroll
    for (int e = 0; e < V; e += 2) {
      const float2 d = split2(mul2(add2(join2(x[e], x[e + 1]), top), inv));
      const bool is0 = d.x >= row.sc.edge, is1 = d.y >= row.sc.edge;
      if (is0) head |= 1u << e;
      if (is1) head |= 2u << e;
      if constexpr (TAIL) {
        const float w0 = is0 ? 0.f : row.sc.weight(d.x), w1 = is1 ? 0.f : row.sc.weight(d.y);
        const F32x2 w = join2(w0, w1), h = add2_rz(w, eight);
        const F32x2 l = add2_rz(add2(w, fma2(h, minus, eight)), low);
        const float2 hf = split2(h), lf = split2(l);
        hi += __float_as_uint(hf.x) + __float_as_uint(hf.y) - 2u * 0x41000000u;
        lo += __float_as_uint(lf.x) + __float_as_uint(lf.y) - 2u * 0x37000000u;
        if constexpr (COUNT) n += (w0 >= 0x1p-40f) + (w1 >= 0x1p-40f);
      }
    }
    if (HEAD && head) {
      int to = atomicAdd(&sh.head_n, __popc(head));
      do {
        if (to < kHead) sh.head[to].y = __int_as_float(i + __ffs(head) - 1);
        ++to;
        head &= head - 1;
      } while (head);
    }
  });
  if constexpr (TAIL) {
    unsigned long long m = (static_cast<unsigned long long>(hi) << 20) + lo;
#pragma unroll
    for (int s = 16; s; s >>= 1) {
      m += __shfl_xor_sync(0xFFFFFFFFu, m, s);
      n += __shfl_xor_sync(0xFFFFFFFFu, n, s);
    }
    if ((threadIdx.x & 31) == 0) {
      atomicAdd(&sh.own_tail_mass, m);
      atomicAdd(&sh.own_tail_cnt, n);
    }
  }
  __syncthreads();
  if (TAIL && threadIdx.x < cluster_size()) {
    Shared* to = peer(&sh, threadIdx.x);
    to->tail_mass[cluster_rank()] = sh.own_tail_mass;
    to->tail_cnt[cluster_rank()] = sh.own_tail_cnt;
  }
}

// The head into the block's bins: from the noted elements, or, if there were
// too many, from all of the slice.
template <int TYPE>
__device__ __forceinline__ void bin_head(Shared& sh, const Slice<TYPE>& row) {
  auto take = [&](float d) {
    const unsigned long long m = Scale::mass(row.sc.weight(d));
    if (m) add_to_bin(sh, row.sc.bin(0, d), m);
  };
  if (sh.head_n <= kHead) {
#pragma unroll 4
    for (int k = threadIdx.x; k < sh.head_n; k += kThreads) {
      const float x = row.at(__float_as_int(sh.head[k].y));
      sh.head[k].x = x;
      take(row.sc.d(x));
    }
  } else {
    row.each_within(row.sc.edge, INFINITY, [&](float, float d, int) { take(d); });
  }
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleArgs a) {
  constexpr int V = Elem<TYPE>::kVec, B = Elem<TYPE>::kBytes;
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  cluster_arrive_relaxed();
  const uint32_t rank = cluster_rank(), n_blocks = cluster_size();
  const int r = blockIdx.x / n_blocks;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;

  // ---- the slice: its first and last vector, which may hold other slices'
  // logits or lie beyond the row, are put together from its own elements
  const int begin = min(a.vocab, static_cast<int>(rank) * a.slice);
  const int len = min(a.vocab, begin + a.slice) - begin;
  const uintptr_t addr = reinterpret_cast<uintptr_t>(a.logits) + (r * a.ld + begin) * B;
  const int skew = static_cast<int>(addr % 16) / B;       // elements ahead of the slice's first
  Slice<TYPE> row;
  row.vecs = reinterpret_cast<const uint4*>(addr - addr % 16);
  row.edge = sh.edge;
  row.n_vecs = (len + skew + V - 1) / V;
  row.v0 = skew ? 1 : 0;
  row.v1 = (len + skew) / V;
  row.first = begin - skew;
  if (threadIdx.x == 0) {
    sh.head_n = 0;
    sh.list_n = 0;
    sh.best = kMostVocab;
    sh.bin = 0;
    sh.bin_mass = 0;
    sh.bin_before = 0;
    sh.bin_cnt = 0;
    for (Cut& c : sh.cut) c = {0u, 0u, 0ull};
    sh.own_tail_mass = 0;
    sh.own_tail_cnt = 0;
    if (rank == 0)           // the others' copies are written below
      sh.set = {a.temperature ? a.temperature[r] : 1.f, a.top_p ? a.top_p[r] : 1.f,
                a.min_p ? a.min_p[r] : 0.f, a.u[r], a.top_k ? a.top_k[r] : 0};
  }
  if (threadIdx.x < kMostCluster) {
    sh.tail_mass[threadIdx.x] = 0;
    sh.tail_cnt[threadIdx.x] = 0;
  }
  if (threadIdx.x < 2 * V) {
    const int at = (threadIdx.x < V ? 0 : (row.n_vecs - 1) * V) + threadIdx.x % V;
    const bool own = at >= skew && at - skew < len;
    const int64_t i = r * a.ld + begin + (at - skew);
    if constexpr (B == 4)
      reinterpret_cast<uint32_t*>(sh.edge)[threadIdx.x] =
          own ? static_cast<const uint32_t*>(a.logits)[i] : kEmpty<TYPE>;
    else
      reinterpret_cast<uint16_t*>(sh.edge)[threadIdx.x] =
          own ? static_cast<const uint16_t*>(a.logits)[i] : static_cast<uint16_t>(kEmpty<TYPE>);
  }
  clear_bins(sh);
  __syncthreads();

  // ---- the largest logit
  uint32_t best = kEmpty<TYPE>, early = best;             // early: of the thread's first vectors
  const int early_end = a.level_vecs * kThreads;
#pragma unroll 4
  for (int v = threadIdx.x; v < row.n_vecs; v += kThreads) {
    const uint4 x = Slice<TYPE>::no_nan(row.load(v));
    best = max_packed<TYPE>(best, max_packed<TYPE>(max_packed<TYPE>(x.x, x.y), max_packed<TYPE>(x.z, x.w)));
    if (v < early_end) early = best;
  }
  float top = widest<TYPE>(best);
  // ---- the row's largest logit, and a level that a given share of the threads'
  // maxima exceed: each warp's value of that rank, averaged
  {
    const float mine = widest<TYPE>(early);
    int before = 0;          // lanes of larger maximum
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float o = __shfl_sync(0xFFFFFFFFu, mine, i);
      before += o > mine || (o == mine && i < lane) ? 1 : 0;
    }
    if (before == a.level_rank) sh.warp_level[warp] = mine;
#pragma unroll
    for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, m));
    if (lane == 0) sh.warp_max[warp] = top;
  }
  __syncthreads();
  float level = 0.f;
  int levels = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    top = fmaxf(top, sh.warp_max[w]);
    if (fabsf(sh.warp_level[w]) < INFINITY) {
      level += sh.warp_level[w];
      ++levels;
    }
  }
  level = levels ? level / levels : -INFINITY;
  __syncwarp();
  cluster_wait();            // every block runs
  if (threadIdx.x < n_blocks) {
    Shared* to = peer(&sh, threadIdx.x);
    to->block_max[rank] = top;
    to->block_level[rank] = level;
    if (rank == 0) to->set = sh.set;
  }
  cluster_barrier();
  level = 0.f;
  for (uint32_t p = 0; p < n_blocks; ++p) {
    top = fmaxf(top, sh.block_max[p]);
    level += sh.block_level[p];              // -inf if a block has none
  }
  level /= n_blocks;
  const Settings set = sh.set;

  row.sc = {top, 0.f, set.min_p > 0.f ? fminf(set.min_p, 1.f) : 0.f, 0.f, 0.f};   // a NaN min_p: none
  int token = -1;
  float logprob = -INFINITY;
  uint32_t kept = 0;
  if (top == -INFINITY) {
    // nothing to draw from
  } else if (!(set.t > 0.f)) {
    row.each_vec([&](int i, const float (&x)[V]) {
      int e = V;
#pragma unroll
      for (int k = V - 1; k >= 0; --k)
        if (x[k] == top) e = k;
      if (e < V) atomicMin(&peer(&sh, 0)->best, row.first + i + e);
    });
    cluster_barrier();
    token = sh.best;         // block 0 writes it
    logprob = 0.f;
    kept = 1;
  } else if (top == INFINITY) {
    Search<TYPE> search{sh, row};
    const Cut c = search.draw_infinite(set);
    token = static_cast<int>(c.idx);
    kept = c.count;
    logprob = -logf(static_cast<float>(kept));
  } else {
    row.sc.inv_t = fminf(fmaxf(__fdiv_rn(1.f, set.t), 1.17549435e-38f), 3.40282347e38f);
    // ---- the head; the others' total, if it can matter (min-p and top-k mostly
    // end a row within the head)
    row.sc.edge = a.vocab <= kSmall ? -28.f : fminf(row.sc.d(level), -1e-6f);
    row.sc.edge = fmaxf(row.sc.edge, -28.f);             // nothing behind it has a weight
    row.sc.per_nat = (kBins - 1) / -row.sc.edge;
    const bool tail = !(row.sc.min_p > 1.001f * expf(row.sc.edge));
    if (!tail || set.top_k > 0)
      weigh<TYPE, true, false, false>(sh, row);
    else if (set.top_p < 1.f)                            // which ends in a count of its own
      weigh<TYPE, true, true, false>(sh, row);
    else
      weigh<TYPE, true, true, true>(sh, row);
    bin_head(sh, row);
    cluster_barrier();
    Search<TYPE> search{sh, row};
    search.dirty = true;
    search.bins = merge_bins(sh);
    if (tail && set.top_k > 0 && static_cast<uint32_t>(set.top_k) > search.bins.total_c) {
      weigh<TYPE, false, true, true>(sh, row);
      cluster_barrier();
    }
    unsigned long long mass = search.bins.total_m;
    kept = search.bins.total_c;
    for (uint32_t p = 0; p < n_blocks; ++p) {
      mass += sh.tail_mass[p];
      kept += sh.tail_cnt[p];
    }
    Cut c;
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {   // top-k, top-p, the draw
      unsigned long long target;
      if (step == 0) {
        if (!(set.top_k > 0 && static_cast<uint32_t>(set.top_k) < kept)) continue;
        target = static_cast<unsigned long long>(set.top_k - 1);
      } else if (step == 1) {
        if (!(set.top_p < 1.f)) continue;
        // passed where the total reaches ceil(p Z): where it passes ceil(p Z) - 1
        bool whole;
        target = share_of(fmaxf(set.top_p, 0.f), mass, whole);
        if (whole && target > 0) --target;
      } else {
        bool whole;
        target = share_of(set.u > 0.f ? fminf(set.u, 1.f) : 0.f, mass, whole);
        if (target >= mass) target = mass - 1;
      }
      c = search.cross(step == 0, target, step == 2);
      if (step < 2) {
        mass = c.mass;
        kept = c.count;
      }
    }
    if (rank == 0 && threadIdx.x == 0) {
      // (a row that someone writes meanwhile may give any index: not beyond it)
      token = min(static_cast<int>(c.idx), a.vocab - 1);
      // from d, as the integer weight of an unlikely token is coarse; the best
      // token's 2^40 is always part of the mass
      const float d = row.sc.d(load_logit<TYPE>(a.logits, r * a.ld + token));
      logprob = d - log1pf(__ull2float_rn(mass - (1ull << 40)) * 0x1p-40f);
    }
  }
  if (rank == 0 && threadIdx.x == 0) {
    a.token[r] = token;
    if (a.logprob) a.logprob[r] = logprob;
    if (a.kept) a.kept[r] = static_cast<int32_t>(kept);
  }
}

// Blocks that share a row: more while the GPU has an SM for each and each still
// has a few thousand logits; eight only for a few rows, as clusters of eight wait
// for room in one GPC (17 rows of 59,392: 16.4 us with four blocks, 18.8 with
// eight; 64 rows of 32,001: 12.4 us with two, 13.8 with four).
int cluster_for(int rows, int vocab) {
  int n = 1;
  while (n < kMostCluster && vocab > n * 4096 &&
         rows * 2 * static_cast<int64_t>(n) <= (n == 4 ? kNumSMs / 2 : kNumSMs))
    n *= 2;
  return n;
}

template <int TYPE>
cudaError_t launch_sample(SampleArgs a, int rows, cudaStream_t s) {
  constexpr size_t smem = sizeof(Shared);
  static DeviceOnce once;
  cudaError_t e = once.run([] {
    return cudaFuncSetAttribute(sample_kernel<TYPE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                static_cast<int>(sizeof(Shared)));
  });
  if (e != cudaSuccess) return e;
  const int n = cluster_for(rows, a.vocab);
  a.slice = ((a.vocab + n - 1) / n + 15) / 16 * 16;
  // The head's size, no more than the blocks can note, and the sample that finds
  // its level: with `each` of its tokens among so many vectors of a thread, a
  // share of 1 - exp(-each) of the threads has one.
  constexpr int V = Elem<TYPE>::kVec;
  const double want = fmin(fmin(kTarget, kShare * a.vocab), 0.88 * kHead * n), per_vec = V * want / a.vocab;
  a.level_vecs = per_vec > 1.0 ? 1 : static_cast<int>(1.0 / per_vec + 0.5);
  const double each = per_vec * a.level_vecs;
  a.level_rank = static_cast<int>(fmin(32.0 * (1.0 - exp(-each)), 31.0) - 0.5);
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
  if (!aligned4(params->temperature, params->top_p, params->min_p, params->top_k, u, token, logprob,
                kept))
    return GS_ERR_INVALID_ARG;
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
