// The join between two sub-layers of a residual stack, forward and backward in one pass over its rows each:
//
//   u = Npost(branch),   x_out = x_scale x + branch_scale gate * u,   h = Npre(x_out)
//
// N is LayerNorm (gamma, beta), RMSNorm (gamma) or nothing; the gate is a number per channel, per element or nothing.
// With D = the gradient of x_out, vhat a normed row before gamma, <.> the mean over a row and q = branch_scale D gate:
//
//   D  = dx_out + rstd (a - <a> - xhat <a xhat>),  a = dh gamma          (RMSNorm: without <a>)
//   dx = x_scale D,   dbranch = rstd (b - <b> - fhat <b fhat>),  b = q gamma_post
//   d_pre  = sum over rows of dh xhat, dh;   d_post = of q fhat, q;   dgate = branch_scale D u (per channel: summed over rows)
//
// Everything streams its [rows][H] tensors once and is bound by HBM.
#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

namespace {

constexpr int kRowsPerBlock = 4;     // wavefronts per 256-thread block
constexpr int kPartialRows = 256;    // workgroups of the backward pass at most = partial rows of column sums

// Mean (LayerNorm; RMSNorm has none) and reciprocal deviation of a row that a wavefront holds in NV vectors per lane.  The
// squares are those of the deviations, formed in a second pass over the registers.
template <int NV, bool FULL>
__device__ __forceinline__ void row_moments(const float (&v)[NV][8], int kind, int lane, int H, float eps, float& mean, float& rstd) {
  mean = 0.f;
  rstd = 1.f;
  if (kind == HANAYO_NORM_NONE) return;
  if (kind == HANAYO_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
      if (FULL || (i * 64 + lane) * 8 < H) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[i][j];
      }
    mean = wave_sum(sum) / (float)H;
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (FULL || (i * 64 + lane) * 8 < H) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float d = v[i][j] - mean;
        sq += d * d;
      }
    }
  rstd = rsqrtf(wave_sum(sq) / (float)H + eps);
}

// v = (v - mean) rstd gamma (+ beta)
template <typename T>
__device__ __forceinline__ void apply_norm(float (&v)[8], const T* w, int kind, int c, int H, float mean, float rstd) {
  if (kind == HANAYO_NORM_NONE) return;
  float g[8];
  load8(w + c, g);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = (v[j] - mean) * rstd * g[j];
  if (kind == HANAYO_NORM_LAYER) {
    load8(w + H + c, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += g[j];
  }
}

// One wavefront per row, NV vectors of 8 per lane; FULL: H == 512 NV.  h is formed from x_out before its rounding.
template <typename T, int NV, bool FULL>
__global__ __launch_bounds__(256) void residual_fwd_kernel(ResidualArgs a) {
  const int lane = threadIdx.x & 63;
  const int row = blockIdx.x * kRowsPerBlock + (threadIdx.x >> 6), H = a.H;
  if (row >= a.rows) return;
  const size_t base = (size_t)row * H;
  float v[NV][8], x[NV][8];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * 64 + lane) * 8;
    if (FULL || c < H) {
      load8(static_cast<const T*>(a.branch) + base + c, v[i]);
      load8(static_cast<const T*>(a.x) + base + c, x[i]);
    }
  }
  float m1, r1, m2, r2;
  row_moments<NV, FULL>(v, a.post, lane, H, a.eps, m1, r1);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * 64 + lane) * 8;
    if (FULL || c < H) {
      apply_norm(v[i], static_cast<const T*>(a.w_post), a.post, c, H, m1, r1);
      if (a.gate_kind != HANAYO_GATE_NONE) {
        float g[8];
        load8(static_cast<const T*>(a.gate) + (a.gate_kind == HANAYO_GATE_CHANNEL ? 0 : base) + c, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] *= g[j];
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) x[i][j] = a.x_scale * x[i][j] + a.branch_scale * v[i][j];
      store8(static_cast<T*>(a.x_out) + base + c, x[i]);
    }
  }
  row_moments<NV, FULL>(x, a.pre, lane, H, a.eps, m2, r2);
  if (a.stats && lane == 0) a.stats[row] = make_float4(m1, r1, m2, r2);
  if (a.pre == HANAYO_NORM_NONE) return;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = (i * 64 + lane) * 8;
    if (FULL || c < H) {
      apply_norm(x[i], static_cast<const T*>(a.w_pre), a.pre, c, H, m2, r2);
      store8(static_cast<T*>(a.h) + base + c, x[i]);
    }
  }
}

// The sum over a row of two numbers: over the lanes, and over the RS wavefronts that share the row through `slot` (RS entries
// of the row group).  One barrier; parts are added in order.
template <int RS>
__device__ __forceinline__ void row_sums(float& s1, float& s2, float2* slot, int part, int lane) {
  s1 = wave_sum(s1);
  s2 = wave_sum(s2);
  if (RS > 1) {
    if (lane == 0) slot[part] = make_float2(s1, s2);
    __syncthreads();
    s1 = s2 = 0.f;
#pragma unroll
    for (int p = 0; p < RS; ++p) {
      const float2 t = slot[p];
      s1 += t.x;
      s2 += t.y;
    }
  }
}

// A row is shared by RS wavefronts, a lane owns 8 columns; a workgroup walks RG rows at a time.  The column sums
// (dh xhat, dh, q' fhat, q' with q' = q without a gate per channel, which the finaliser multiplies in) stay in registers over the
// rows and leave as one partial row of 4 H numbers per workgroup.
template <typename T, int RS, int RG>
__global__ __launch_bounds__(RS * RG * 64) void residual_bwd_kernel(ResidualArgs a) {
  extern __shared__ float red[];                 // [RG][2 * H] for the column sums; before that the row-sum exchange
  float2* xch = reinterpret_cast<float2*>(red);  // [2 steps][2][RG][RS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rg = wave / RS, part = wave % RS, H = a.H;
  const int col = (part * 64 + lane) * 8;
  const bool inside = col < H;
  const bool pre = a.pre != HANAYO_NORM_NONE, post = a.post != HANAYO_NORM_NONE, element = a.gate_kind == HANAYO_GATE_ELEMENT;
  float acc[4][8], w_pre[8], w_post[8], b_post[8], gate[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    acc[0][j] = acc[1][j] = acc[2][j] = acc[3][j] = 0.f;
    w_pre[j] = w_post[j] = gate[j] = 1.f;
    b_post[j] = 0.f;
  }
  if (inside) {
    if (pre) load8(static_cast<const T*>(a.w_pre) + col, w_pre);
    if (post) load8(static_cast<const T*>(a.w_post) + col, w_post);
    if (a.post == HANAYO_NORM_LAYER) load8(static_cast<const T*>(a.w_post) + H + col, b_post);
    if (a.gate_kind == HANAYO_GATE_CHANNEL) load8(static_cast<const T*>(a.gate) + col, gate);
  }
  int it = 0;
  for (int first = blockIdx.x * RG; first < a.rows; first += gridDim.x * RG, ++it) {  // the same trip count for every wavefront
    const int row = first + rg;
    const bool valid = row < a.rows && inside;
    const size_t at = (size_t)row * H + col;
    float4 st = make_float4(0.f, 1.f, 0.f, 1.f);
    float d[8], f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = f[j] = 0.f;
    if (valid) {
      st = a.stats[row];
      if (a.dx_out) load8(static_cast<const T*>(a.dx_out) + at, d);
      load8(static_cast<const T*>(a.branch) + at, f);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = (f[j] - st.x) * st.y;
    }
    float2* slot = xch + ((it & 1) * RG + rg) * RS;
    if (pre) {
      float xh[8], dy[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) xh[j] = dy[j] = 0.f;
      if (valid) {
        load8(static_cast<const T*>(a.x_out) + at, xh);
        load8(static_cast<const T*>(a.dh) + at, dy);
#pragma unroll
        for (int j = 0; j < 8; ++j) xh[j] = (xh[j] - st.z) * st.w;
      }
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        acc[0][j] += dy[j] * xh[j];
        acc[1][j] += dy[j];
        dy[j] *= w_pre[j];
        s1 += dy[j];
        s2 += dy[j] * xh[j];
      }
      row_sums<RS>(s1, s2, slot, part, lane);
      const float c1 = a.pre == HANAYO_NORM_LAYER ? s1 / (float)H : 0.f, c2 = s2 / (float)H;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] += st.w * (dy[j] - c1 - xh[j] * c2);
    }
    if (valid) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = a.x_scale * d[j];
      store8(static_cast<T*>(a.dx) + at, o);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) d[j] = valid ? d[j] * a.branch_scale : 0.f;
    if (element && valid) {
      float g[8], o[8];
      load8(static_cast<const T*>(a.gate) + at, g);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = d[j] * (f[j] * w_post[j] + b_post[j]);
        d[j] *= g[j];
      }
      store8(static_cast<T*>(a.dgate) + at, o);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[2][j] += d[j] * f[j];
      acc[3][j] += d[j];
      d[j] *= gate[j] * w_post[j];
      s1 += d[j];
      s2 += d[j] * f[j];
    }
    if (post) {
      row_sums<RS>(s1, s2, slot + 2 * RG * RS, part, lane);
      const float c1 = a.post == HANAYO_NORM_LAYER ? s1 / (float)H : 0.f, c2 = s2 / (float)H;
#pragma unroll
      for (int j = 0; j < 8; ++j) d[j] = st.y * (d[j] - c1 - f[j] * c2);
    }
    if (valid) store8(static_cast<T*>(a.dbranch) + at, d);
  }
  // the row groups' column sums, two of the four at a time (64 KiB of LDS)
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    __syncthreads();
    if (inside) {
      float* mine = red + (size_t)rg * 2 * H + col;
      store8(mine, acc[2 * half]);
      store8(mine + H, acc[2 * half + 1]);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * H; c += RS * RG * 64) {
      float t = 0.f;
#pragma unroll
      for (int g = 0; g < RG; ++g) t += red[g * 2 * H + c];
      a.scratch[((size_t)blockIdx.x * 2 + half) * 2 * H + c] = t;
    }
  }
}

// Adds up the partial rows and turns them into the parameters' gradients.  blockIdx.y: 0 the pre-norm's two sums, 1 the
// post-norm's and the gate's.  A workgroup owns 32 columns; 32 row groups run down every 32nd partial row and are added in order.
template <typename T>
__global__ __launch_bounds__(1024) void residual_finalize_kernel(ResidualArgs a, int partials) {
  __shared__ float red[2][32][32];
  const int cl = threadIdx.x & 31, rg = threadIdx.x >> 5, H = a.H, c = blockIdx.x * 32 + cl;
  const int half = blockIdx.y;
  if (half == 0 ? !a.d_pre : !a.d_post && a.gate_kind != HANAYO_GATE_CHANNEL) return;
  float t0 = 0.f, t1 = 0.f;
  if (c < H) {
    for (int r = rg; r < partials; r += 32) {
      const float* p = a.scratch + ((size_t)r * 2 + half) * 2 * H + c;
      t0 += p[0];
      t1 += p[H];
    }
  }
  red[0][rg][cl] = t0;
  red[1][rg][cl] = t1;
  __syncthreads();
  if (rg || c >= H) return;
  t0 = t1 = 0.f;
#pragma unroll
  for (int g = 0; g < 32; ++g) {
    t0 += red[0][g][cl];
    t1 += red[1][g][cl];
  }
  auto put = [&](float* out, float v) { *out = a.accumulate ? *out + v : v; };
  if (half == 0) {
    put(a.d_pre + c, t0);
    if (a.pre == HANAYO_NORM_LAYER) put(a.d_pre + H + c, t1);
    return;
  }
  const bool channel = a.gate_kind == HANAYO_GATE_CHANNEL;
  const float g = channel ? ld(static_cast<const T*>(a.gate) + c) : 1.f;
  if (a.post != HANAYO_NORM_NONE) put(a.d_post + c, g * t0);
  if (a.post == HANAYO_NORM_LAYER) put(a.d_post + H + c, g * t1);
  if (channel) {
    const T* w = static_cast<const T*>(a.w_post);
    float v = t0;
    if (a.post != HANAYO_NORM_NONE) v *= ld(w + c);
    if (a.post == HANAYO_NORM_LAYER) v += ld(w + H + c) * t1;
    put(static_cast<float*>(a.dgate) + c, v);
  }
}

template <typename T>
int residual_forward_t(const ResidualArgs& a, hipStream_t stream) {
  const dim3 grid((a.rows + kRowsPerBlock - 1) / kRowsPerBlock), block(256);
  const int nv = (a.H + 511) / 512;
#define LAUNCH(NV)                                                                                     \
  do {                                                                                                 \
    if (a.H == 512 * NV) launch_kernel((residual_fwd_kernel<T, NV, true>), grid, block, 0, stream, a); \
    else launch_kernel((residual_fwd_kernel<T, NV, false>), grid, block, 0, stream, a);                \
  } while (0)
  if (nv <= 1) LAUNCH(1);
  else if (nv <= 2) LAUNCH(2);
  else if (nv <= 4) LAUNCH(4);
  else LAUNCH(8);
#undef LAUNCH
  return check_launch("residual_forward");
}

// Workgroups of the backward pass, and the rows that each walks at a time.
int backward_blocks(int rows, int H) {
  const int rg = 16 / ((H + 511) / 512), blocks = (rows + rg - 1) / rg;
  return blocks < kPartialRows ? blocks : kPartialRows;
}

template <typename T>
int residual_backward_t(const ResidualArgs& a, hipStream_t stream) {
  const int rs = (a.H + 511) / 512, rg = 16 / rs, blocks = backward_blocks(a.rows, a.H);
  size_t lds = (size_t)rg * 2 * a.H * sizeof(float);  // at most 64 KiB
  if (lds < 1024) lds = 1024;                         // the row-sum exchange: 4 * 16 slots
  if (blocks > 0) {
#define LAUNCH(RS, RG) launch_kernel((residual_bwd_kernel<T, RS, RG>), dim3(blocks), dim3(RS * RG * 64), lds, stream, a)
    switch (rs) {
      case 1: LAUNCH(1, 16); break;
      case 2: LAUNCH(2, 8); break;
      case 3: LAUNCH(3, 5); break;
      case 4: LAUNCH(4, 4); break;
      case 5: LAUNCH(5, 3); break;
      case 6: LAUNCH(6, 2); break;
      case 7: LAUNCH(7, 2); break;
      default: LAUNCH(8, 2); break;
    }
#undef LAUNCH
    if (const int rc = check_launch("residual_backward")) return rc;
  }
  if (!a.d_pre && !a.d_post && a.gate_kind != HANAYO_GATE_CHANNEL) return HANAYO_OK;
  launch_kernel((residual_finalize_kernel<T>), dim3((a.H + 31) / 32, 2), dim3(1024), 0, stream, a, blocks);
  return check_launch("residual_backward (finalize)");
}

}  // namespace

int residual_forward(int dtype, const ResidualArgs& a, hipStream_t stream) {
  if (a.rows == 0) return HANAYO_OK;
  return dtype == HANAYO_BF16 ? residual_forward_t<bf16>(a, stream) : residual_forward_t<float>(a, stream);
}

size_t residual_scratch_bytes(int rows, int H) { return align_up((size_t)backward_blocks(rows, H) * 4 * H * sizeof(float) + 1, 256); }

int residual_backward(int dtype, const ResidualArgs& a, hipStream_t stream) {
  return dtype == HANAYO_BF16 ? residual_backward_t<bf16>(a, stream) : residual_backward_t<float>(a, stream);
}

}  // namespace k
}  // namespace hanayo
