// tree.cu -- what follows the verification of drafted trees: the accepted path
// (gs_tree_accept) and the move of its keys and values (gs_tree_commit).
#include "internal.h"
#include "step_common.cuh"

namespace gs {
namespace {

constexpr int kMostNodes = 64;       // two per lane of a warp

// ---------------------------------------------------------------- acceptance
// Child c of node p matches where its token is p's choice and no earlier child
// of p matches.  A node is on the path if it and all its ancestors but the root
// match.  A parent comes before its children, so the path is the nodes on it by
// rising number, and a node's place is the number of those before it.
//
// One warp per tree, two nodes per lane: choices and flags pass between lanes by
// shuffles, and the ancestors are joined by pointer doubling (six steps for 64
// nodes, where a walk takes as many as the path is long).  A few hundred bytes
// per tree: latency bounds it (one tree 1.7 us, 256 trees of 64 nodes 2.0 us, of which
// the launch is most).
constexpr int kAcceptWarps = 4;

struct AcceptArgs {
  const int32_t *parent, *token, *choice, *count, *most;
  int eos, trees, nodes;
  int32_t *path, *next, *length;
  int* err;
};

// Element i of an array that holds two values per lane, i and i + 32.
__device__ __forceinline__ int pick(const int (&v)[2], int i) {
  const int a = __shfl_sync(0xFFFFFFFFu, v[0], i & 31), b = __shfl_sync(0xFFFFFFFFu, v[1], i & 31);
  return i & 32 ? b : a;
}

__global__ void __launch_bounds__(kAcceptWarps * 32) tree_accept_kernel(const AcceptArgs a) {
  const int tree = blockIdx.x * kAcceptWarps + (threadIdx.x >> 5), lane = threadIdx.x & 31;
  if (tree >= a.trees) return;
  const int64_t at = static_cast<int64_t>(tree) * a.nodes;
  int count = a.count ? a.count[tree] : a.nodes;
  const int most = a.most ? a.most[tree] : a.nodes;
  bool bad = count < 0 || count > a.nodes;
  count = min(max(count, 0), a.nodes);
  int parent[2], token[2], choice[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    const bool in = i < count;
    parent[h] = in && i > 0 ? a.parent[at + i] : 0;
    token[h] = in && i > 0 ? a.token[at + i] : -1;
    choice[h] = in ? a.choice[at + i] : -1;
    if (in && i > 0 && (parent[h] < 0 || parent[h] >= i)) {
      bad = true;
      parent[h] = 0;
      token[h] = -1;                     // never matches
    }
  }
  if (bad) atomicExch(a.err, kErrBounds);
  // matches; of several children of a node the first
  int state[2];                          // the ancestor so far, and 64 while all match
  uint32_t had = 0;                      // nodes with a matching child below 32 (they are below 32)
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int want = pick(choice, parent[h]);
    const bool match = token[h] >= 0 && token[h] == want && want != a.eos;
    const uint32_t peers = __match_any_sync(0xFFFFFFFFu, match ? parent[h] : 64 + lane);
    bool first = match && __ffs(peers) - 1 == lane;
    if (h == 0) {
      had = __reduce_or_sync(0xFFFFFFFFu, first ? 1u << parent[0] : 0u);
    } else {
      first = first && !(parent[1] < 32 && ((had >> parent[1]) & 1));
    }
    const bool root = h == 0 && lane == 0 && count > 0;
    state[h] = root ? 64 : first ? 64 | parent[h] : 0;
  }
#pragma unroll
  for (int step = 0; step < 6; ++step) {
    const int u = pick(state, state[0] & 63), v = pick(state, state[1] & 63);
    state[0] = state[0] & 64 & u ? u : 0;
    state[1] = state[1] & 64 & v ? v : 0;
  }
  const uint32_t on0 = __ballot_sync(0xFFFFFFFFu, state[0] & 64),
                 on1 = __ballot_sync(0xFFFFFFFFu, state[1] & 64);
  const int length = min(__popc(on0) + __popc(on1), max(most, 0));
  if (lane == 0) a.length[tree] = length;
  const uint32_t before = (1u << lane) - 1;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    const int place = h == 0 ? __popc(on0 & before) : __popc(on0) + __popc(on1 & before);
    if ((state[h] & 64) && place < length) {
      a.path[at + place] = i;
      a.next[at + place] = choice[h];
    }
    if (i >= length && i < a.nodes) {
      a.path[at + i] = -1;
      a.next[at + i] = -1;
    }
  }
}

// -------------------------------------------------------------------- commit
// Place i of a path takes the key and value of node path[i]: slot n + path[i]
// goes to slot n + i.  A path rises, so path[i] >= i, and from the first place
// where they differ on, every one moves.  The slots overlap: a thread block reads
// all that it moves before it writes any of it.
//
// A block moves the keys, or the values, of one KV head of one tree in one
// layer.  A key is a row of D elements, moved in 16-byte pieces.  Values lie
// transposed, so a moved token is one element of each of D rows of 64: lanes
// are dealt to the (row, token) pairs, and reads and writes are sectors of 32
// bytes for elements of 2.  These sectors bound it: 64 trees, 12 layers, 8 heads of 128, paths
// of up to 16 tokens 38 us, for which DRAM reads 120 MB and writes 27, and 35 more stay in L2,
// where 51 MB are moved.  (Blocks that take 2, 4 or 12 layers each, so that paths and pages are
// looked up less often: 38, 40 and 50 us.)
constexpr int kCommitThreads = 128;
constexpr int kCommitWarps = kCommitThreads / 32;

struct CommitArgs {
  CacheView cache;
  int64_t layer_elems;
  const int32_t *seq, *n, *path, *length;
  int nodes;
  int* err;
};

template <int D>
__global__ void __launch_bounds__(kCommitThreads) tree_commit_kernel(const CommitArgs a) {
  __shared__ int s_length, s_n, s_seq, s_first;
  __shared__ int64_t s_from[kMostNodes], s_to[kMostNodes];   // element offsets in the pool
  const int tree = blockIdx.z, which = blockIdx.x & 1, head = blockIdx.x >> 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t at = static_cast<int64_t>(tree) * a.nodes;
  int path = tid < a.nodes ? a.path[at + tid] : 0;           // (its place may lie beyond the length)
  if (tid == 0) {
    s_length = a.length[tree];
    s_n = a.n[tree];
    s_seq = a.seq ? a.seq[tree] : tree;
    s_first = kMostNodes;
  }
  __shared__ int s_path[kMostNodes];
  if (tid < kMostNodes) s_path[tid] = path;
  __syncthreads();
  const int length = s_length, n = s_n, seq = s_seq;
  if (length == 0) return;
  bool bad = length < 0 || length > a.nodes || seq < 0 || seq >= a.cache.n_seq || n < 0;
  if (!bad && tid < length) {
    bad = path < 0 || path >= a.nodes || path >= a.cache.pt_stride * kPageTokens - n ||
          (tid > 0 && path <= s_path[tid - 1]);
    if (!bad && path != tid) {
      atomicMin(&s_first, tid);
      const int32_t* table = a.cache.page_table + static_cast<int64_t>(seq) * a.cache.pt_stride;
      const int src = n + path, dst = n + tid;
      const int p = table[src / kPageTokens], r = table[dst / kPageTokens];
      bad = p < 0 || p >= a.cache.n_pages || r < 0 || r >= a.cache.n_pages;
      const int64_t page = 2ll * a.cache.Hkv * kPageTokens * D;
      const int64_t block = (static_cast<int64_t>(which) * a.cache.Hkv + head) * kPageTokens * D;
      const int step = which ? 1 : D;    // a token's first element within its page's block
      s_from[tid] = p * page + block + static_cast<int64_t>(src % kPageTokens) * step;
      s_to[tid] = r * page + block + static_cast<int64_t>(dst % kPageTokens) * step;
    }
  }
  if (__syncthreads_or(bad)) {           // nothing of this tree is moved
    if (tid == 0) atomicExch(a.err, kErrBounds);
    return;
  }
  const int first = s_first, moved = length - first;
  if (moved <= 0) return;
  uint16_t* kv = a.cache.kv + blockIdx.y * a.layer_elems;
  if (which == 0) {
    constexpr int C = D / 8, NG = kCommitThreads / C, MOST = (kMostNodes + NG - 1) / NG;
    const int c = tid % C, grp = tid / C;
    uint4 r[MOST];
#pragma unroll
    for (int u = 0; u < MOST; ++u)
      if (grp + u * NG < moved)
        r[u] = *reinterpret_cast<const uint4*>(kv + s_from[first + grp + u * NG] + 8 * c);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < MOST; ++u)
      if (grp + u * NG < moved)
        *reinterpret_cast<uint4*>(kv + s_to[first + grp + u * NG] + 8 * c) = r[u];
    return;
  }
  // `width` lanes take the tokens of a row, the warp 32 / width rows at a time;
  // only one warp works on a row
  const int width = moved > 16 ? 32 : moved > 8 ? 16 : moved > 4 ? 8 : moved > 2 ? 4 : moved;
  const int i = lane % width, sub = lane / width, per = 32 / width;
  constexpr int U = 4;
  const bool one = i < moved, two = i + 32 < moved;
  const uint16_t *from0 = one ? kv + s_from[first + i] : nullptr,
                 *from1 = two ? kv + s_from[first + i + 32] : nullptr;
  uint16_t *to0 = one ? kv + s_to[first + i] : nullptr, *to1 = two ? kv + s_to[first + i + 32] : nullptr;
  for (int d0 = warp * per * U; d0 < D; d0 += kCommitWarps * per * U) {
    uint16_t x[U], y[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int d = d0 + u * per + sub;
      if (one && d < D) x[u] = from0[d * kPageTokens];
      if (two && d < D) y[u] = from1[d * kPageTokens];
    }
    __syncwarp();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int d = d0 + u * per + sub;
      if (one && d < D) to0[d * kPageTokens] = x[u];
      if (two && d < D) to1[d * kPageTokens] = y[u];
    }
    __syncwarp();
  }
}

}  // namespace
}  // namespace gs

extern "C" int gs_tree_accept(const int32_t* parent, const int32_t* token, const int32_t* choice,
                              const int32_t* count, const int32_t* most, int eos, int trees, int nodes,
                              int32_t* path, int32_t* next, int32_t* length, int32_t* err,
                              void* stream) {
  using namespace gs;
  if (!parent || !token || !choice || !path || !next || !length || !err || trees < 0 || nodes < 1)
    return GS_ERR_INVALID_ARG;
  if (!aligned4(parent, token, choice, count, most, path, next, length, err)) return GS_ERR_INVALID_ARG;
  if (nodes > kMostNodes) return GS_ERR_UNSUPPORTED;
  if (trees == 0) return GS_OK;
  const AcceptArgs a = {parent, token, choice, count, most, eos, trees, nodes, path, next, length, err};
  tree_accept_kernel<<<(trees + kAcceptWarps - 1) / kAcceptWarps, kAcceptWarps * 32, 0,
                       static_cast<cudaStream_t>(stream)>>>(a);
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}

extern "C" int gs_tree_commit(const gs_cache* cache, int n_layers, const int32_t* seq, const int32_t* n,
                              const int32_t* path, const int32_t* length, int trees, int nodes,
                              int32_t* err, void* stream) {
  using namespace gs;
  if (const int rc = check_cache(cache)) return rc;
  if (!n || !path || !length || !err || n_layers < 1 || trees < 0 || nodes < 1)
    return GS_ERR_INVALID_ARG;
  if (!aligned4(seq, n, path, length, err)) return GS_ERR_INVALID_ARG;
  // layers and trees are grid dimensions
  if (nodes > kMostNodes || n_layers > 65535 || trees > 65535) return GS_ERR_UNSUPPORTED;
  if (trees == 0) return GS_OK;
  CommitArgs a;
  a.cache = cache_view(*cache);
  a.layer_elems = static_cast<int64_t>(cache->n_pages) * 2 * cache->n_kv_heads * kPageTokens *
                  cache->head_dim;
  a.seq = seq;
  a.n = n;
  a.path = path;
  a.length = length;
  a.nodes = nodes;
  a.err = err;
  const dim3 grid(2 * cache->n_kv_heads, n_layers, trees);
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (cache->head_dim == 64)
    tree_commit_kernel<64><<<grid, kCommitThreads, 0, s>>>(a);
  else
    tree_commit_kernel<128><<<grid, kCommitThreads, 0, s>>>(a);
  return cudaGetLastError() == cudaSuccess ? GS_OK : GS_ERR_CUDA;
}
