// Embedding lookup with a scale, and its gradient by sorted tokens.
//
//   out[t] = scale * table[token[t]],    d_table[v] (+)= scale * sum over t with token[t] = v of dout[t]
//
// Both are bound by HBM where they are large and by their launches where they are small.  The gradient first sorts the rows by
// token (ties in row order), so that the rows of a token follow each other and are added in a fixed order without
// atomics, whatever the distribution of the tokens.
#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

namespace {

constexpr int kRowsPerBlock = 4;  // wavefronts per 256-thread block

template <typename T>
__global__ __launch_bounds__(256) void embedding_fwd_kernel(const T* __restrict__ table, const int32_t* __restrict__ tokens,
                                                            float scale, T* __restrict__ out, int rows, int H, int vocab) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRowsPerBlock + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int tok = tokens[row];
  const bool known = tok >= 0 && tok < vocab;
  const T* src = table + (size_t)(known ? tok : 0) * H;
  for (int c = lane * 8; c < H; c += 64 * 8) {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (known) {
      load8(src + c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] *= scale;
    }
    store8(out + (size_t)row * H + c, v);
  }
}

// Where each row goes: the number of rows that sort before it, by token and, among equal tokens, by row.  A workgroup places 64
// rows, a row per lane; its 16 wavefronts compare them with a sixteenth of all rows each, whose tokens are uniform over the
// wavefront and come through scalar loads.  Tokens outside [0, vocab) count as `vocab` and go to the end.
__global__ __launch_bounds__(1024) void token_rank_kernel(const int32_t* __restrict__ tokens, int rows, int vocab,
                                                          int32_t* __restrict__ order, int32_t* __restrict__ sorted) {
  __shared__ int part[16][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * 64, t = first + lane;
  auto key = [&](int s) { return (int)min((unsigned)tokens[s], (unsigned)vocab); };
  const int mine = t < rows ? key(t) : 0;
  const int each = (rows + 15) / 16, begin = wave * each, end = min(begin + each, rows);
  int before = 0;
  for (int s = begin; s < min(end, first); ++s) before += key(s) <= mine;
  for (int s = max(begin, first); s < min(end, first + 64); ++s) {
    const int other = key(s);
    before += other < mine || (other == mine && s < t);
  }
  for (int s = max(begin, first + 64); s < end; ++s) before += key(s) < mine;
  part[wave][lane] = before;
  __syncthreads();
  if (wave == 0 && t < rows) {
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) at += part[w][lane];
    order[at] = t;
    sorted[at] = mine;
  }
}

__global__ __launch_bounds__(256) void zero_kernel(f32x4* __restrict__ out, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// A wavefront per sorted position and 512 columns: the one at the start of a token's run adds up the run.
template <typename T>
__global__ __launch_bounds__(256) void embedding_bwd_kernel(const int32_t* __restrict__ order, const int32_t* __restrict__ sorted,
                                                            const T* __restrict__ dout, float scale, float* __restrict__ d_table,
                                                            int rows, int H, int vocab) {
  const int lane = threadIdx.x & 63;
  const int p = blockIdx.x * kRowsPerBlock + (threadIdx.x >> 6), c = (blockIdx.y * 64 + lane) * 8;
  if (p >= rows) return;
  const int tok = sorted[p];
  if (tok >= vocab || (p > 0 && sorted[p - 1] == tok) || c >= H) return;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  for (int q = p; q < rows && sorted[q] == tok; ++q) {
    float v[8];
    load8(dout + (size_t)order[q] * H + c, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += v[j];
  }
  float* dst = d_table + (size_t)tok * H + c;
  float old[8];
  load8(dst, old);
#pragma unroll
  for (int j = 0; j < 8; ++j) old[j] += scale * acc[j];
  store8(dst, old);
}

}  // namespace

int embedding_forward(int dtype, const void* table, const int32_t* tokens, float scale, void* out, int rows, int H, int vocab,
                      hipStream_t stream) {
  if (rows == 0) return HANAYO_OK;
  const dim3 grid((rows + kRowsPerBlock - 1) / kRowsPerBlock);
  if (dtype == HANAYO_BF16)
    launch_kernel(embedding_fwd_kernel<bf16>, grid, dim3(256), 0, stream, (const bf16*)table, tokens, scale, (bf16*)out, rows, H, vocab);
  else
    launch_kernel(embedding_fwd_kernel<float>, grid, dim3(256), 0, stream, (const float*)table, tokens, scale, (float*)out, rows, H, vocab);
  return check_launch("embedding_forward");
}

size_t embedding_workspace_bytes(int rows, int H) { return align_up((size_t)rows * 8 + 256, 256); }

int embedding_backward(int dtype, const int32_t* tokens, const void* dout, float scale, float* d_table, int rows, int H, int vocab,
                       bool accumulate, void* workspace, hipStream_t stream) {
  if (!accumulate) {
    const size_t n = (size_t)vocab * H / 4, want = (n + 255) / 256;
    launch_kernel(zero_kernel, dim3((unsigned)(want < 4096 ? want : 4096)), dim3(256), 0, stream, (f32x4*)d_table, n);
    if (const int rc = check_launch("embedding_backward (zero)")) return rc;
  }
  if (rows == 0) return HANAYO_OK;
  int32_t* order = static_cast<int32_t*>(workspace);
  int32_t* sorted = order + rows;
  launch_kernel(token_rank_kernel, dim3((rows + 63) / 64), dim3(1024), 0, stream, tokens, rows, vocab, order, sorted);
  if (const int rc = check_launch("embedding_backward (sort)")) return rc;
  const dim3 grid((rows + kRowsPerBlock - 1) / kRowsPerBlock, (H + 511) / 512);
  if (dtype == HANAYO_BF16)
    launch_kernel(embedding_bwd_kernel<bf16>, grid, dim3(256), 0, stream, order, sorted, (const bf16*)dout, scale, d_table, rows, H, vocab);
  else
    launch_kernel(embedding_bwd_kernel<float>, grid, dim3(256), 0, stream, order, sorted, (const float*)dout, scale, d_table, rows, H, vocab);
  return check_launch("embedding_backward");
}

}  // namespace k
}  // namespace hanayo
