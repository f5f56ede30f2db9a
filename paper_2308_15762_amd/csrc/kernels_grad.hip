// The gradients of a whole model as one vector: its squared 2-norm over any number of tensors, and the tensors scaled so
// that the norm does not exceed a limit.
//
//   S = sum over all tensors and elements of x^2,   norm = sqrt(S),   out = x * (norm > max_norm ? max_norm / norm : 1)
//
// Both passes are bound by HBM: the first reads every gradient once, the second reads and writes it.  Squares are formed
// and added in 64 bits: the largest and smallest fp32 gradients neither overflow nor vanish, and 2^40 of them add up with
// an error far below the fp32 result's last bit; the pass reads 4 bytes per conversion and addition, which the 64-bit rate of the vector
// units covers many times over.  Tensors are cut into tiles, and a launch's tiles go round its workgroups in turn; which
// partial sum holds what depends on the sizes, and inside a tile on where the tensor lies modulo 16 bytes; the partial sums are added
// in order.  So results repeat bit for bit for tensors that stay where they are, and may differ in the last of 53 bits where they do not.
#include <type_traits>

#include "clip.h"
#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

namespace {

constexpr unsigned kTileBytes = 32768;  // of a tensor: eight 16-byte loads a thread, all in flight at once
constexpr int kMaxBlocks = 2048;        // workgroups of a launch at most: 8 on every CU, one partial sum each
constexpr int kLoads = kTileBytes / 16 / 256;
// The pass that forms the norm leaves the first 192 MiB of a call's tensors in the 256 MB cache and reads the rest past it, so that the pass
// that scales or uses them finds that part there; that pass reads and writes past the cache.  Variants in turn on one card,
// norm and clipping of 403 MB / norm and Adam on 609 MB (30 bytes an element): 181 / 852 us; with ordinary loads and stores everywhere
// 238 / 1046, the rest past the cache in the first pass only 200 / 1043, nothing kept 214 / 1013.  Cards differ: others take 185 / 924 to 937.
constexpr unsigned kKeepTiles = 192u * (1 << 20) / kTileBytes;

// Up to so many tiles one workgroup forms the sum alone, without the launch that adds up partial sums (norm and clipping of one fp32 tensor,
// whole calls: 1 tile 8.8 us against 14.0, 4 tiles 10.6 against 14.0, 8 tiles 10.7 against 11.2 to 13.8, 16 tiles 12.8 against 11.3 to 13.6).
constexpr unsigned kAloneTiles = 8;

// A launch's tensors.  The table travels in the kernel's arguments: nothing to copy to the device first, so that a call can be
// captured into a graph, and nothing to keep alive.
struct GradEntry {
  const void* in;
  void* out;
  size_t count;
  unsigned first;  // the tensor's first tile
  int bf16;
};
constexpr int kEntries = 100;  // 3.2 KB; kernel arguments end at 4 KB
struct GradTable {
  GradEntry e[kEntries];
  int n;
  unsigned tiles, keep;  // keep: the first of them, that the norm's pass leaves in the cache
};

// Which tensor a tile lies in.  The lanes of a wavefront hold the tensors' first tiles, two each, and vote: one trip to memory
// for the whole launch in place of one for each step of a search.
struct TensorFinder {
  unsigned lo, hi;
  __device__ __forceinline__ TensorFinder(const GradTable& t) {
    static_assert(kEntries <= 128, "two tensors a lane");
    const int lane = threadIdx.x & 63;
    lo = lane < t.n ? t.e[lane].first : 0xffffffffu;
    hi = lane + 64 < t.n ? t.e[lane + 64].first : 0xffffffffu;
  }
  __device__ __forceinline__ int operator()(unsigned tile) const {
    return __popcll(__ballot(lo <= tile)) + __popcll(__ballot(hi <= tile)) - 1;
  }
};

template <int WAVES>
__device__ __forceinline__ double workgroup_sum(double v, double* red) {  // red: [WAVES]; the same sum in every thread
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, kWave);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < WAVES; ++w) v += red[w];
  return v;
}

// Elements of a tile before its first 16-byte boundary, and whole vectors behind that; a thread takes vector `thread + 256 u`.
template <typename T>
struct TileSplit {
  static constexpr unsigned kVec = 16 / sizeof(T);
  size_t begin;
  unsigned n, head, vecs;
  __device__ __forceinline__ TileSplit(const GradEntry& e, unsigned tile) {
    constexpr unsigned kTile = kTileBytes / sizeof(T);
    begin = (size_t)(tile - e.first) * kTile;
    n = e.count - begin < kTile ? (unsigned)(e.count - begin) : kTile;
    head = (16u - (unsigned)(reinterpret_cast<uintptr_t>(e.in) & 15u)) % 16u / sizeof(T);  // a tile is a whole number of vectors
    if (head > n) head = n;
    vecs = (n - head) / kVec;
  }
  // The elements that belong to no vector: fewer than two vectors' worth, one each for the first threads; n: none.
  __device__ __forceinline__ unsigned loose(unsigned thread) const {
    const unsigned i = thread < head ? thread : thread + vecs * kVec;
    return i < n ? i : n;
  }
};

template <typename T, bool KEEP>
__device__ __forceinline__ double tile_sumsq(const GradEntry& e, unsigned tile) {
  using Vec = typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type;
  const TileSplit<T> s(e, tile);
  const T* in = static_cast<const T*>(e.in) + s.begin;
  double acc = 0.0;
  if (s.vecs) {  // uniform; loads behind the last vector read it again and count as nothing: no branch between the loads
    Vec v[kLoads];
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      v[u] = fetch<!KEEP>(reinterpret_cast<const Vec*>(in + s.head + min(threadIdx.x + 256u * u, s.vecs - 1) * s.kVec));
#pragma unroll
    for (int u = 0; u < kLoads; ++u) {
      double part = 0.0;
#pragma unroll
      for (unsigned j = 0; j < s.kVec; ++j) {
        const double x = (float)v[u][j];
        part += x * x;
      }
      acc += threadIdx.x + 256u * u < s.vecs ? part : 0.0;
    }
  }
  const unsigned i = s.loose(threadIdx.x);
  if (i < s.n) {
    const double x = ld(in + i);
    acc += x * x;
  }
  return acc;
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradTable t, double* __restrict__ partial) {
  __shared__ double red[4];
  const TensorFinder find(t);
  double acc = 0.0;
  for (unsigned tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
    const GradEntry& e = t.e[find(tile)];
    if (tile < t.keep) acc += e.bf16 ? tile_sumsq<bf16, true>(e, tile) : tile_sumsq<float, true>(e, tile);
    else acc += e.bf16 ? tile_sumsq<bf16, false>(e, tile) : tile_sumsq<float, false>(e, tile);
  }
  acc = workgroup_sum<4>(acc, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

__global__ __launch_bounds__(1024) void grad_finish_kernel(const double* __restrict__ partial, size_t n, double* __restrict__ sumsq) {
  __shared__ double red[16];
  double acc = 0.0;
#pragma unroll 2
  for (size_t i = threadIdx.x; i < n; i += 1024) acc += partial[i];  // a launch leaves at most 2048
  acc = workgroup_sum<16>(acc, red);
  if (threadIdx.x == 0) sumsq[0] = acc;
}

template <typename T>
__device__ __forceinline__ void tile_scale(const GradEntry& e, unsigned tile, const ClipScale& k) {
  using Vec = typename std::conditional<sizeof(T) == 2, bf16x8, f32x4>::type;
  const TileSplit<T> s(e, tile);
  const T* in = static_cast<const T*>(e.in) + s.begin;
  T* out = static_cast<T*>(e.out) + s.begin;
  if ((reinterpret_cast<uintptr_t>(e.in) ^ reinterpret_cast<uintptr_t>(e.out)) & 15u) {  // no boundary in common
    for (unsigned i = threadIdx.x; i < s.n; i += 256) st(out + i, k(ld(in + i)));
    return;
  }
  Vec v[kLoads];
  if (s.vecs) {
#pragma unroll
    for (int u = 0; u < kLoads; ++u)
      v[u] = fetch<true>(reinterpret_cast<const Vec*>(in + s.head + min(threadIdx.x + 256u * u, s.vecs - 1) * s.kVec));
  }
#pragma unroll
  for (int u = 0; u < kLoads; ++u) {
    const unsigned at = threadIdx.x + 256u * u;
    if (at >= s.vecs) break;
    Vec o;
#pragma unroll
    for (unsigned j = 0; j < s.kVec; ++j) o[j] = (T)k((float)v[u][j]);
    put<true>(reinterpret_cast<Vec*>(out + s.head + at * s.kVec), o);
  }
  const unsigned i = s.loose(threadIdx.x);
  if (i < s.n) st(out + i, k(ld(in + i)));
}

__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, ClipArgs c) {
  const TensorFinder find(t);
  const ClipScale s = clip_scale(c);
  if (c.norm && blockIdx.x == 0 && threadIdx.x == 0) c.norm[0] = s.norm;
  for (unsigned tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
    const GradEntry& e = t.e[find(tile)];
    if (s.one() && e.in == e.out) continue;
    if (e.bf16) tile_scale<bf16>(e, tile, s);
    else tile_scale<float>(e, tile, s);
  }
}

// Fills the table with tensors from `at` on; returns how many it took.
size_t fill_table(const hanayo_grad* grads, size_t n, size_t at, GradTable& t) {
  t.n = 0;
  t.tiles = t.keep = 0;
  size_t taken = 0;
  while (at + taken < n && t.n < kEntries) {
    const hanayo_grad& g = grads[at + taken];
    ++taken;
    if (!g.count) continue;
    t.e[t.n++] = GradEntry{g.grad, g.out ? g.out : const_cast<void*>(g.grad), g.count, t.tiles, g.dtype == HANAYO_BF16};
    const size_t each = kTileBytes / (g.dtype == HANAYO_BF16 ? 2 : 4);
    t.tiles += (unsigned)((g.count + each - 1) / each);  // at most 2^40 elements together (kGradMaxElements): 2^27 tiles
  }
  return taken;
}

}  // namespace

size_t grad_workspace_bytes(size_t n) { return ((n + kEntries - 1) / kEntries + (n == 0)) * kMaxBlocks * sizeof(double); }

int grad_sumsq(const hanayo_grad* grads, size_t n, double* sumsq, double* workspace, hipStream_t stream) {
  size_t partials = 0;
  unsigned keep = kKeepTiles;
  for (size_t at = 0; at < n;) {
    GradTable t;
    at += fill_table(grads, n, at, t);
    if (!t.tiles) continue;
    t.keep = keep < t.tiles ? keep : t.tiles;
    keep -= t.keep;
    if (!partials && at == n && t.tiles <= kAloneTiles) {  // its one partial sum is the sum
      launch_kernel(grad_sumsq_kernel, dim3(1), dim3(256), 0, stream, t, sumsq);
      return check_launch("grad_sumsq");
    }
    const unsigned blocks = t.tiles < (unsigned)kMaxBlocks ? t.tiles : kMaxBlocks;
    launch_kernel(grad_sumsq_kernel, dim3(blocks), dim3(256), 0, stream, t, workspace + partials);
    if (const int rc = check_launch("grad_sumsq")) return rc;
    partials += blocks;
  }
  launch_kernel(grad_finish_kernel, dim3(1), dim3(1024), 0, stream, workspace, partials, sumsq);
  return check_launch("grad_sumsq (finish)");
}

int grad_clip(const hanayo_grad* grads, size_t n, const ClipArgs& clip, hipStream_t stream) {
  ClipArgs c = clip;
  size_t at = 0;
  do {
    GradTable t;
    at += fill_table(grads, n, at, t);
    if (!t.tiles && !c.norm) continue;
    const unsigned blocks = t.tiles < 1 ? 1 : t.tiles < (unsigned)kMaxBlocks ? t.tiles : kMaxBlocks;
    launch_kernel(grad_clip_kernel, dim3(blocks), dim3(256), 0, stream, t, c);
    if (const int rc = check_launch("grad_clip")) return rc;
    c.norm = nullptr;  // the first launch has written it
  } while (at < n);
  return HANAYO_OK;
}

}  // namespace k
}  // namespace hanayo
