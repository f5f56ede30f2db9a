// The gradients of a whole model as one vector: its squared 2-norm over any number of tensors, and the tensors scaled so
// that the norm does not exceed a limit.
//
//   S = sum over all tensors and elements of x^2,   norm = sqrt(S),   out = x * (norm > max_norm ? max_norm / norm : 1)
//
// Both passes are bound by HBM: the first reads every gradient once, the second reads and writes it.  Squares are formed
// and added in 64 bits: the largest and smallest fp32 gradients neither overflow nor vanish, and 2^40 of them add up with
// an error far below the fp32 result's last bit; the pass reads 4 bytes per conversion and addition, which the 64-bit rate of the vector
// units covers many times over.  Tensors are cut into tiles, and a launch's tiles go round its workgroups in turn; which
// partial sum holds what depends on the sizes alone, and the partial sums are added in order, so results repeat bit for bit.
#include "clip.h"
#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

namespace {

constexpr unsigned kTile = 8192;     // elements of a tile
constexpr int kMaxBlocks = 2048;     // workgroups of a launch at most: 8 on every CU, one partial sum each

// A launch's tensors.  The table travels in the kernel's arguments: nothing to copy to the device first, so that a call can be
// captured into a graph, and nothing to keep alive.  Entry `n` holds the number of tiles.
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
  unsigned tiles;
};

// The tensor that holds `tile` (tensors without elements hold none).
__device__ __forceinline__ int find_tensor(const GradTable& t, unsigned tile) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (t.e[mid].first <= tile) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
  red[threadIdx.x] = v;
  __syncthreads();
  for (int o = 128; o > 0; o >>= 1) {
    if ((int)threadIdx.x < o) red[threadIdx.x] += red[threadIdx.x + o];
    __syncthreads();
  }
  return red[0];
}

__global__ __launch_bounds__(256) void grad_sumsq_kernel(GradTable t, double* __restrict__ partial) {
  __shared__ double red[256];
  double acc = 0.0;
  for (unsigned tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
    const GradEntry& e = t.e[find_tensor(t, tile)];
    const size_t begin = (size_t)(tile - e.first) * kTile, end = begin + kTile < e.count ? begin + kTile : e.count;
    for (size_t i = begin + threadIdx.x; i < end; i += 256) {
      const double x = e.bf16 ? ld(static_cast<const bf16*>(e.in) + i) : ld(static_cast<const float*>(e.in) + i);
      acc += x * x;
    }
  }
  acc = block_sum(acc, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = acc;
}

__global__ __launch_bounds__(256) void grad_finish_kernel(const double* __restrict__ partial, size_t n, double* __restrict__ sumsq) {
  __shared__ double red[256];
  double acc = 0.0;
  for (size_t i = threadIdx.x; i < n; i += 256) acc += partial[i];
  acc = block_sum(acc, red);
  if (threadIdx.x == 0) sumsq[0] = acc;
}

__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, ClipArgs c) {
  const ClipScale s = clip_scale(c);
  if (c.norm && blockIdx.x == 0 && threadIdx.x == 0) c.norm[0] = s.norm;
  for (unsigned tile = blockIdx.x; tile < t.tiles; tile += gridDim.x) {
    const GradEntry& e = t.e[find_tensor(t, tile)];
    if (s.scale == 1.f && e.in == e.out) continue;
    const size_t begin = (size_t)(tile - e.first) * kTile, end = begin + kTile < e.count ? begin + kTile : e.count;
    for (size_t i = begin + threadIdx.x; i < end; i += 256) {
      if (e.bf16) st(static_cast<bf16*>(e.out) + i, ld(static_cast<const bf16*>(e.in) + i) * s.scale);
      else st(static_cast<float*>(e.out) + i, ld(static_cast<const float*>(e.in) + i) * s.scale);
    }
  }
}

// Fills the table with tensors from `at` on; returns how many it took.
size_t fill_table(const hanayo_grad* grads, size_t n, size_t at, GradTable& t) {
  t.n = 0;
  t.tiles = 0;
  size_t taken = 0;
  while (at + taken < n && t.n < kEntries) {
    const hanayo_grad& g = grads[at + taken];
    ++taken;
    if (!g.count) continue;
    t.e[t.n++] = GradEntry{g.grad, g.out ? g.out : const_cast<void*>(g.grad), g.count, t.tiles, g.dtype == HANAYO_BF16};
    t.tiles += (unsigned)((g.count + kTile - 1) / kTile);  // at most 2^40 elements together (kGradMaxElements): 2^27 tiles
  }
  return taken;
}

}  // namespace

size_t grad_workspace_bytes(size_t n) { return ((n + kEntries - 1) / kEntries + (n == 0)) * kMaxBlocks * sizeof(double); }

int grad_sumsq(const hanayo_grad* grads, size_t n, double* sumsq, double* workspace, hipStream_t stream) {
  size_t partials = 0;
  for (size_t at = 0; at < n;) {
    GradTable t;
    at += fill_table(grads, n, at, t);
    if (!t.tiles) continue;
    const unsigned blocks = t.tiles < (unsigned)kMaxBlocks ? t.tiles : kMaxBlocks;
    launch_kernel(grad_sumsq_kernel, dim3(blocks), dim3(256), 0, stream, t, workspace + partials);
    if (const int rc = check_launch("grad_sumsq")) return rc;
    partials += blocks;
  }
  launch_kernel(grad_finish_kernel, dim3(1), dim3(256), 0, stream, workspace, partials, sumsq);
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
