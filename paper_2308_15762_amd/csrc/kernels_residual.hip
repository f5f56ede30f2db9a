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
// Everything streams its [rows][H] tensors once and is bound by HBM.  MI355X, bf16, calls one behind another: 4096 rows of 1024
// forward 8.3 us (34 MB), backward 17.0 us (50 MB); 8192 rows of 4096 with a gate per element backward 107 us (537 MB, 5.0 TB/s, what
// a large copy reaches).  A kernel by itself takes longer than its share of that, since starting and draining do not overlap with a
// neighbour's: 9.5 us, and 15.1 with 3.9 for the finaliser.
#include "device_util.h"
#include "kernels.h"

namespace hanayo {
namespace k {

namespace {

constexpr int kPartialRows = 256;  // workgroups of the backward pass at most = partial rows of column sums

// Operands that a call does not have (a norm's parameters, a gate) are read all the same, from a tensor that is there, and replaced
// by 1 or 0 behind the load: a load inside a branch would have to be waited for where the branch ends, and the loads of a row
// would come one after another.
template <typename T>
struct NormParams {
  const T* gamma;
  const T* beta;
  bool scale, shift;
  __device__ __forceinline__ NormParams(const void* w, int kind, const void* there, int H)
      : gamma(static_cast<const T*>(kind != HANAYO_NORM_NONE ? w : there)),
        beta(kind == HANAYO_NORM_LAYER ? gamma + H : gamma), scale(kind != HANAYO_NORM_NONE), shift(kind == HANAYO_NORM_LAYER) {}
};

// The sum over a row that W wavefronts share, parts added in order: one barrier where W > 1.  slot: [W], used again only
// behind another barrier.
template <int W>
__device__ __forceinline__ float row_sum(float v, float* slot, int part, int lane) {
  v = wave_sum(v);
  if constexpr (W > 1) {
    if (lane == 0) slot[part] = v;
    __syncthreads();
    v = slot[0];
#pragma unroll
    for (int p = 1; p < W; ++p) v += slot[p];
  }
  return v;
}

// Mean (LayerNorm; RMSNorm has none) and reciprocal deviation of a row, NV vectors per lane, zeros behind the row's end.  The
// squares are those of the deviations, formed in a second pass over the registers.  slots: [2][W]
template <int NV, int W, bool FULL>
__device__ __forceinline__ void row_moments(const float (&v)[NV][8], int kind, int c0, int H, float eps, float* slots, int part, int lane,
                                            float& mean, float& rstd) {
  mean = 0.f;
  rstd = 1.f;
  if (kind == HANAYO_NORM_NONE) return;
  if (kind == HANAYO_NORM_LAYER) {
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += v[i][j];
    mean = row_sum<W>(sum, slots, part, lane) / (float)H;
  }
  float sq = 0.f;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const bool in = FULL || c0 + i * 512 < H;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float d = v[i][j] - mean;
      sq += in ? d * d : 0.f;
    }
  }
  rstd = rsqrtf(row_sum<W>(sq, slots + W, part, lane) / (float)H + eps);
}

// W wavefronts per row, NV vectors of 8 per lane; FULL: H == 512 NV W.  Lanes behind the row's end read its last vector again.
// Everything that a row needs is asked for before its first sum; a wavefront that walks several rows keeps the parameters and
// asks for the next row before it works on the current one.  h is formed from x_out before its rounding.
template <typename T, int NV, int W, bool FULL>
__global__ __launch_bounds__(256) void residual_fwd_kernel(ResidualArgs a) {
  constexpr int kRows = 4 / W;  // that a workgroup works on at a time
  __shared__ float slots[2][kRows][4 * W];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rg = wave / W, part = wave % W, H = a.H;
  const int c0 = (part * NV * 64 + lane) * 8;
  const T *x = static_cast<const T*>(a.x), *branch = static_cast<const T*>(a.branch);
  const NormParams<T> post(a.w_post, a.post, branch, H), pre(a.w_pre, a.pre, branch, H);
  const bool gated = a.gate_kind != HANAYO_GATE_NONE, element = a.gate_kind == HANAYO_GATE_ELEMENT;
  const T* gate = gated ? static_cast<const T*>(a.gate) : branch;
  Raw8<T> w1[NV], b1[NV], w2[NV], b2[NV];
  struct Row {
    Raw8<T> v[NV], x[NV], g[NV];
  } next;
  auto at = [&](int i) { return FULL || c0 + i * 512 < H ? c0 + i * 512 : H - 8; };
  auto fetch_row = [&](int r) {
    const size_t base = (size_t)min(r, a.rows - 1) * H;
#pragma unroll
    for (int i = 0; i < NV; ++i) next.v[i].load(branch + base + at(i));
#pragma unroll
    for (int i = 0; i < NV; ++i) next.x[i].load(x + base + at(i));
#pragma unroll
    for (int i = 0; i < NV; ++i) next.g[i].load(gate + (element ? base : 0) + at(i));
  };
  fetch_row(blockIdx.x * kRows + rg);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w1[i].load(post.gamma + at(i));
    b1[i].load(post.beta + at(i));
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    w2[i].load(pre.gamma + at(i));
    b2[i].load(pre.beta + at(i));
  }
  int it = 0;
  for (int first = blockIdx.x * kRows; first < a.rows; first += gridDim.x * kRows, ++it) {  // the same trip count for every wavefront
    const int row = first + rg;
    const bool valid = row < a.rows;
    const size_t base = (size_t)row * H;
    const Row now = next;
    if (first + (int)gridDim.x * kRows < a.rows) fetch_row(row + gridDim.x * kRows);
    float v[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const bool in = FULL || c0 + i * 512 < H;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = in ? now.v[i].get(j) : 0.f;
    }
    float* slot = slots[it & 1][rg];
    float m1, r1, m2, r2;
    row_moments<NV, W, FULL>(v, a.post, c0, H, a.eps, slot, part, lane, m1, r1);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = c0 + i * 512;
      const bool in = FULL || c < H;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        float u = (v[i][j] - m1) * r1;
        u = (post.scale ? u * w1[i].get(j) : u) + (post.shift ? b1[i].get(j) : 0.f);
        if (gated) u *= now.g[i].get(j);
        v[i][j] = in ? a.x_scale * now.x[i].get(j) + a.branch_scale * u : 0.f;
      }
      if (in && valid) store8(static_cast<T*>(a.x_out) + base + c, v[i]);
    }
    row_moments<NV, W, FULL>(v, a.pre, c0, H, a.eps, slot + 2 * W, part, lane, m2, r2);
    if (a.stats && lane == 0 && part == 0 && valid) a.stats[row] = make_float4(m1, r1, m2, r2);
    if (a.pre == HANAYO_NORM_NONE) continue;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = c0 + i * 512;
#pragma unroll
      for (int j = 0; j < 8; ++j) v[i][j] = (v[i][j] - m2) * r2 * w2[i].get(j) + (pre.shift ? b2[i].get(j) : 0.f);
      if ((FULL || c < H) && valid) store8(static_cast<T*>(a.h) + base + c, v[i]);
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

// A row is shared by RS wavefronts, a lane owns 8 columns; a workgroup walks RG rows at a time, and each wavefront asks for its part of
// the next row (in storage form) before it works on the current one.  The column sums (dh xhat, dh, q' fhat, q' with q' = q without
// a gate per channel, which the finaliser multiplies in) stay in registers over the rows and leave as one partial row of 4 H numbers per
// workgroup.  PRE: there is a pre-norm; ELEMENT: a gate per element.  Lanes behind the row's end read its last vector again and
// count as zeros; wavefronts behind the last row read the last row.
template <typename T, int RS, int RG, bool PRE, bool ELEMENT>
__global__ __launch_bounds__(RS * RG * 64) void residual_bwd_kernel(ResidualArgs a) {
  extern __shared__ float red[];                 // [RG][2 * H] for the column sums; before that the row-sum exchange
  float2* xch = reinterpret_cast<float2*>(red);  // [2 steps][2][RG][RS]
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int rg = wave / RS, part = wave % RS, H = a.H;
  const int col = (part * 64 + lane) * 8;
  const bool inside = col < H, post = a.post != HANAYO_NORM_NONE;
  const size_t lane_at = inside ? col : H - 8;
  const NormParams<T> post_w(a.w_post, a.post, a.branch, H), pre_w(a.w_pre, a.pre, a.branch, H);
  const bool channel = a.gate_kind == HANAYO_GATE_CHANNEL;
  float acc[4][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[0][j] = acc[1][j] = acc[2][j] = acc[3][j] = 0.f;
  Raw8<T> w_pre, w_post, b_post, gate;  // parameters stay in storage form: registers
  if (PRE) w_pre.load(pre_w.gamma + lane_at);
  w_post.load(post_w.gamma + lane_at);
  if (ELEMENT) b_post.load(post_w.beta + lane_at);
  else gate.load((channel ? static_cast<const T*>(a.gate) : static_cast<const T*>(a.branch)) + lane_at);
  const bool given = !PRE || a.dx_out;  // a gradient from elsewhere
  const T* dx_out = static_cast<const T*>(given ? a.dx_out : a.branch);
  struct Row {
    Raw8<T> branch, dx_out, x_out, dh, gate;
    float4 stats;
  } next;
  auto fetch = [&](int row) {
    const size_t r = (size_t)min(row, a.rows - 1), at = r * H + lane_at;
    next.stats = a.stats[r];
    if (PRE) {
      next.x_out.load(static_cast<const T*>(a.x_out) + at);
      next.dh.load(static_cast<const T*>(a.dh) + at);
    }
    next.dx_out.load(dx_out + at);
    next.branch.load(static_cast<const T*>(a.branch) + at);
    if (ELEMENT) next.gate.load(static_cast<const T*>(a.gate) + at);
  };
  fetch(blockIdx.x * RG + rg);
  int it = 0;
  for (int first = blockIdx.x * RG; first < a.rows; first += gridDim.x * RG, ++it) {  // the same trip count for every wavefront
    const int row = first + rg;
    const bool valid = row < a.rows && inside;
    const size_t at = (size_t)row * H + col;
    const Row now = next;
    const float4 st = now.stats;
    if (first + gridDim.x * RG < a.rows) fetch(row + gridDim.x * RG);
    float d[8], f[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      d[j] = given ? now.dx_out.get(j) : 0.f;
      f[j] = valid ? (now.branch.get(j) - st.x) * st.y : 0.f;
    }
    float2* slot = xch + ((it & 1) * RG + rg) * RS;
    if (PRE) {
      float xh[8], dy[8];
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        xh[j] = valid ? (now.x_out.get(j) - st.z) * st.w : 0.f;
        dy[j] = valid ? now.dh.get(j) : 0.f;
        acc[0][j] += dy[j] * xh[j];
        acc[1][j] += dy[j];
        dy[j] *= w_pre.get(j);
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
    if (ELEMENT) {
      float o[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        o[j] = d[j] * ((post ? f[j] * w_post.get(j) : f[j]) + (post_w.shift ? b_post.get(j) : 0.f));
        d[j] = valid ? d[j] * now.gate.get(j) : 0.f;
      }
      if (valid) store8(static_cast<T*>(a.dgate) + at, o);
    }
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      acc[2][j] += d[j] * f[j];
      acc[3][j] += d[j];
      if (!ELEMENT) d[j] = channel ? d[j] * gate.get(j) : d[j];
      d[j] = post ? d[j] * w_post.get(j) : d[j];
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
#pragma unroll 8
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

// Rows of up to 5 KB (their operands and parameters in registers) take one wavefront, from 4 KB on no more workgroups than CUs, which walk
// the rows; wider ones take the four wavefronts of a workgroup, two workgroups a CU.  us, bf16 unless said otherwise:
//   width (rows)            1 wavefront, 256 workgroups / 512 / one a row; 4 wavefronts, 256 workgroups / 512 / one a row
//   1024 (16384)            33.4 / 27.4 / 27.2;  -
//   1536 (10922)            -    / 28.2 / 29.3;  -
//   2048 (8192)             27.6 / 31.8 / 40.6 (with two wavefronts 27.6 at best);  -
//   2560 (6553)             32.4 / 33.9 / - (with two 35.5);  66.3 / 41.4 / 39.8
//   4096 (4096)             36.9 / 39.9 / - (with two 31.5);  37.5 / 28.7 / 29.9
//   fp32 2048 (8192)        53.5 / 55.8 / -;  63.0 / 51.4 / 62.1
//   fp32 4096 (4096)        -  ;  55.8 / 52.0 / 61.6
constexpr int kAloneBytes = 5120;  // of a row that one wavefront takes
template <typename T>
int residual_forward_t(const ResidualArgs& a, hipStream_t stream) {
  const int row_bytes = a.H * (int)sizeof(T);
  const bool shared = row_bytes > kAloneBytes;
  const int nv = (a.H + (shared ? 2047 : 511)) / (shared ? 2048 : 512), want = shared ? a.rows : (a.rows + 3) / 4;
  const int most = shared ? 512 : row_bytes >= 4096 ? 256 : 1 << 20;  // the last: what a grid can hold
  const dim3 grid(want < most ? want : most), block(256);
#define LAUNCH(NV, W)                                                                    \
  do {                                                                                   \
    if constexpr (W > 1 || 512 * NV * (int)sizeof(T) <= kAloneBytes) {                   \
      if (a.H == 512 * NV * W) {                                                         \
        launch_kernel((residual_fwd_kernel<T, NV, W, true>), grid, block, 0, stream, a); \
        break;                                                                           \
      }                                                                                  \
    }                                                                                    \
    launch_kernel((residual_fwd_kernel<T, NV, W, false>), grid, block, 0, stream, a);    \
  } while (0)
  if (shared) {
    if constexpr (sizeof(T) == 4) {  // bf16 rows that are shared have more than 2560 numbers
      if (nv == 1) LAUNCH(1, 4);
    }
    if (nv == 2) LAUNCH(2, 4);
  } else if (nv == 1) LAUNCH(1, 1);
  else if (nv == 2) LAUNCH(2, 1);
  else if (nv == 3) LAUNCH(3, 1);
  else if constexpr (sizeof(T) == 2) {  // fp32 rows of more than 1536 numbers are over 5 KB
    if (nv == 4) LAUNCH(4, 1);
    else LAUNCH(5, 1);
  }
#undef LAUNCH
  return check_launch("residual_forward");
}

// Rows that a workgroup of the backward pass walks at a time, RS wavefronts each.  With a pre-norm a wavefront needs more than the 128
// registers that sixteen on a CU have: eight (8192 rows of 4096, bf16, RMS norms and a gate per element: 107 us against 157 with
// sixteen and what does not fit in memory; 4096 rows of 1024: 17.0 against 21.8); without one sixteen (fp32, 1527 rows of 2560: 18.1 against 19.7).
// Rows that 3, 5, 6 or 7 wavefronts share leave some of the eight out (6, 5, 6, 7 of them).  16.8 M numbers, LayerNorm and RMSNorm, a gate per
// channel, us in bf16 / fp32: 1024 columns 46.3 / 82.0, 1536 47.9 / 83.2, 2048 46.8 / 83.8, 2560 52.1 / 83.0, 3584 48.8 / 86.6, 4096 49.1 / 87.1
// (4.3 / 4.9 TB/s at 1024, 3.9 / 4.9 at 2560); a second workgroup on a CU, for which there are registers at 5, is not tried.
constexpr int row_groups(bool pre, int rs) { return (pre ? 8 : 16) / rs; }
int backward_blocks(bool pre, int rows, int H) {
  const int rg = row_groups(pre, (H + 511) / 512), blocks = (rows + rg - 1) / rg;
  return blocks < kPartialRows ? blocks : kPartialRows;
}

template <typename T>
int residual_backward_t(const ResidualArgs& a, hipStream_t stream) {
  const bool pre = a.pre != HANAYO_NORM_NONE, element = a.gate_kind == HANAYO_GATE_ELEMENT;
  const int rs = (a.H + 511) / 512, rg = row_groups(pre, rs), blocks = backward_blocks(pre, a.rows, a.H);
  size_t lds = (size_t)rg * 2 * a.H * sizeof(float);  // at most 64 KiB
  if (lds < 1024) lds = 1024;                         // the row-sum exchange: 4 * 16 slots
  if (blocks > 0) {
#define LAUNCH(RS)                                                                                                          \
  do {                                                                                                                      \
    constexpr int P = row_groups(true, RS), N = row_groups(false, RS);                                                      \
    auto kern = pre ? element ? residual_bwd_kernel<T, RS, P, true, true> : residual_bwd_kernel<T, RS, P, true, false>      \
                    : element ? residual_bwd_kernel<T, RS, N, false, true> : residual_bwd_kernel<T, RS, N, false, false>;   \
    launch_kernel(kern, dim3(blocks), dim3(rs * rg * 64), lds, stream, a);                                                  \
  } while (0)
    switch (rs) {
      case 1: LAUNCH(1); break;
      case 2: LAUNCH(2); break;
      case 3: LAUNCH(3); break;
      case 4: LAUNCH(4); break;
      case 5: LAUNCH(5); break;
      case 6: LAUNCH(6); break;
      case 7: LAUNCH(7); break;
      default: LAUNCH(8); break;
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

size_t residual_scratch_bytes(int rows, int H) { return align_up((size_t)backward_blocks(true, rows, H) * 4 * H * sizeof(float) + 1, 256); }

int residual_backward(int dtype, const ResidualArgs& a, hipStream_t stream) {
  return dtype == HANAYO_BF16 ? residual_backward_t<bf16>(a, stream) : residual_backward_t<float>(a, stream);
}

}  // namespace k
}  // namespace hanayo
