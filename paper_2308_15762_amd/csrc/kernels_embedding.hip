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

// ------------------------------------------------------------------ rows sorted by token
// Keys are tokens; one outside [0, vocab) counts as `vocab` and goes to the end.  Two ways to the same order:
// few rows: every row counts the rows before it (one launch); many rows: radix sort (two launches for every 9 bits of the vocabulary).
__device__ __forceinline__ int token_key(const int32_t* tokens, int t, int vocab) { return (int)min((unsigned)tokens[t], (unsigned)vocab); }

// The table's gradient is cleared by workgroups of the first launch, beside those that sort.
__device__ __forceinline__ void clear_share(f32x4* out, size_t n, int share, int shares, int threads) {
  for (size_t i = (size_t)share * threads + threadIdx.x; i < n; i += (size_t)shares * threads) out[i] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// Where each row goes: the number of rows that sort before it, by token and, among equal tokens, by row.  A workgroup places 64
// rows, a row per lane; its 16 wavefronts compare them with a sixteenth of all rows each, whose tokens are uniform over the
// wavefront and come through scalar loads.
__global__ __launch_bounds__(1024) void token_rank_kernel(const int32_t* __restrict__ tokens, int rows, int vocab,
                                                          int32_t* __restrict__ order, int32_t* __restrict__ sorted, int sorters,
                                                          f32x4* __restrict__ clear, size_t clear_n) {
  __shared__ int part[16][64];
  if ((int)blockIdx.x >= sorters) {
    clear_share(clear, clear_n, blockIdx.x - sorters, gridDim.x - sorters, 1024);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int first = blockIdx.x * 64, t = first + lane;
  const int mine = t < rows ? token_key(tokens, t, vocab) : 0;
  const int each = (rows + 15) / 16, begin = wave * each, end = min(begin + each, rows);
  int before = 0;
#pragma unroll 16
  for (int s = begin; s < min(end, first); ++s) before += token_key(tokens, s, vocab) <= mine;
  for (int s = max(begin, first); s < min(end, first + 64); ++s) {
    const int other = token_key(tokens, s, vocab);
    before += other < mine || (other == mine && s < t);
  }
#pragma unroll 16
  for (int s = max(begin, first + 64); s < end; ++s) before += token_key(tokens, s, vocab) < mine;
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

// Radix sort by one digit: workgroup b owns the b-th run of `each` keys.  `counts` [workgroups][bins]: how often each digit occurs in each run.
constexpr int kMaxBins = 512, kMaxSorters = 256, kSortWaves = 4;
struct SortArgs {
  const int32_t* tokens;  // the first pass: keys from the tokens, rows in order; later passes: nullptr
  const int32_t *order_in, *sorted_in;
  int32_t *order_out, *sorted_out, *counts;
  int rows, vocab, each, sorters, shift, bits;
};
__device__ __forceinline__ int sort_key(const SortArgs& a, int i) { return a.tokens ? token_key(a.tokens, i, a.vocab) : a.sorted_in[i]; }

__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a, f32x4* __restrict__ clear, size_t clear_n) {
  __shared__ int hist[kMaxBins];
  if ((int)blockIdx.x >= a.sorters) {
    clear_share(clear, clear_n, blockIdx.x - a.sorters, gridDim.x - a.sorters, 256);
    return;
  }
  const int bins = 1 << a.bits, begin = blockIdx.x * a.each, end = min(begin + a.each, a.rows);
  for (int d = threadIdx.x; d < bins; d += 256) hist[d] = 0;
  __syncthreads();
  for (int i = begin + threadIdx.x; i < end; i += 256) atomicAdd(&hist[sort_key(a, i) >> a.shift & (bins - 1)], 1);
  __syncthreads();
  for (int d = threadIdx.x; d < bins; d += 256) a.counts[blockIdx.x * bins + d] = hist[d];
}

// Moves a run's keys to their places: behind the keys of smaller digits and those of the same digit in earlier runs and earlier
// wavefronts (a wavefront owns a quarter of the run), in order.  64 keys at a time: a ballot for each bit of the digit finds the
// lanes with the same one.
__global__ __launch_bounds__(kSortWaves * 64) void sort_place_kernel(SortArgs a) {
  __shared__ int at[kSortWaves][kMaxBins];  // where the wavefront's next key of a digit goes
  __shared__ int scan[kSortWaves * 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << a.bits;
  const int begin = blockIdx.x * a.each, end = min(begin + a.each, a.rows);
  const int quarter = (a.each / kSortWaves), w0 = min(begin + wave * quarter, end), w1 = min(w0 + quarter, end);
  for (int d = threadIdx.x; d < kSortWaves * kMaxBins; d += 256) at[d / kMaxBins][d % kMaxBins] = 0;
  __syncthreads();
  for (int i = w0 + lane; i < w1; i += 64) atomicAdd(&at[wave][sort_key(a, i) >> a.shift & (bins - 1)], 1);
  // a thread owns two neighbouring digits: their totals, and their counts in earlier runs
  const int d0 = threadIdx.x * 2;
  int total[2] = {0, 0}, earlier[2] = {0, 0};
  if (d0 < bins) {
#pragma unroll 16
    for (int b = 0; b < a.sorters; ++b) {
      const int2 c = *reinterpret_cast<const int2*>(a.counts + b * bins + d0);
      total[0] += c.x;
      total[1] += c.y;
      if (b < (int)blockIdx.x) {
        earlier[0] += c.x;
        earlier[1] += c.y;
      }
    }
  }
  int sum = total[0] + total[1];
  scan[threadIdx.x] = sum;
  __syncthreads();
  for (int o = 1; o < kSortWaves * 64; o <<= 1) {
    const int add = (int)threadIdx.x >= o ? scan[threadIdx.x - o] : 0;
    __syncthreads();
    scan[threadIdx.x] += add;
    __syncthreads();
  }
  if (d0 < bins) {
    int base = scan[threadIdx.x] - sum;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      int next = base + earlier[k];
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) {
        const int n = at[w][d0 + k];
        at[w][d0 + k] = next;
        next += n;
      }
      base += total[k];
    }
  }
  __syncthreads();
  for (int i0 = w0; i0 < w1; i0 += 64) {
    const int i = i0 + lane;
    const bool have = i < w1;
    const int key = have ? sort_key(a, i) : 0, digit = key >> a.shift & (bins - 1);
    unsigned long long same = __ballot(have);
    for (int b = 0; b < a.bits; ++b) {
      const bool bit = digit >> b & 1;
      const unsigned long long set = __ballot(bit);
      same &= bit ? set : ~set;
    }
    const int before = __popcll(same & ((1ull << lane) - 1ull));
    if (have) {
      const int to = at[wave][digit] + before;  // the wavefront's own counters, read before the first of the lanes moves them on
      a.order_out[to] = a.tokens ? i : a.order_in[i];
      a.sorted_out[to] = key;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (have && before == 0) at[wave][digit] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ------------------------------------------------------------------ sums over the runs of equal tokens
// The sorted rows are cut into pieces of `R` (16 .. 64), a wavefront per piece and 512 columns, so that the work is even whatever the tokens: a token's
// run that lies within a piece is added up and written; of one that crosses a border the piece leaves its part as a partial sum (slot 0: the
// run comes from the piece before; slot 1: it starts here), and the kernel below adds those.  The piece's tokens and rows lie in
// the lanes; eight rows, and the old sums of the runs that end among them, are loaded at a time.
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void embedding_sum_kernel(const int32_t* __restrict__ order, const int32_t* __restrict__ sorted,
                                                            const T* __restrict__ dout, float scale, float* __restrict__ d_table,
                                                            float* __restrict__ partial, int rows, int H, int vocab, int R) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = blockIdx.x * 4 + wave, c = (blockIdx.y * 64 + lane) * 8;
  const long p0 = (long)piece * R;
  if (p0 >= rows) return;
  const int n = min(R, (int)(rows - p0));
  const int tok = lane < n ? sorted[p0 + lane] : -1, row = lane < n ? order[p0 + lane] : 0;
  const int before = p0 > 0 ? sorted[p0 - 1] : -1, after = p0 + n < rows ? sorted[p0 + n] : -1;
  const int live = __popcll(__ballot(lane < n && tok < vocab));
  if (live == 0) return;
  const int next = __shfl_down(tok, 1);
  const unsigned long long ends = __ballot(lane < n && (lane == n - 1 || tok != next));  // the last rows of runs
  unsigned long long whole = ends;                                                       // of runs that lie in the piece
  bool head = before == __builtin_amdgcn_readfirstlane(tok);                             // the first run comes from before
  if (head) whole &= whole - 1;
  if (after == __builtin_amdgcn_readlane(tok, n - 1)) whole &= ~(1ull << (n - 1));
  const bool inside = c < H;
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  constexpr int U = 8;
  for (int i0 = 0; i0 < live; i0 += U) {
    float v[U][8], old[U][8];
    if (inside) {
#pragma unroll
      for (int u = 0; u < U; ++u)
        load8(dout + (size_t)__builtin_amdgcn_readlane(row, min(i0 + u, live - 1)) * H + c, v[u]);
      if constexpr (ADD) {
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i0 + u < live && (whole >> (i0 + u) & 1))
            load8(d_table + (size_t)__builtin_amdgcn_readlane(tok, i0 + u) * H + c, old[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u;
      if (i >= live) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[u][j];
      if (ends >> i & 1) {
        if (whole >> i & 1) {
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = ADD ? old[u][j] + scale * acc[j] : scale * acc[j];
          if (inside) store8(d_table + (size_t)__builtin_amdgcn_readlane(tok, i) * H + c, acc);
        } else if (inside) {
          store8(partial + ((size_t)piece * 2 + (head ? 0 : 1)) * H + c, acc);
        }
        head = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = 0.f;
      }
    }
  }
}

// The runs that cross a piece's end, each by the workgroup of the piece that it starts in: that piece's slot 1 and slot 0 of
// the pieces behind it, every kJoinWaves-th by one wavefront, and the wavefronts' sums in order.
constexpr int kJoinWaves = 8;
template <bool ADD>
__global__ __launch_bounds__(kJoinWaves * 64) void embedding_join_kernel(const int32_t* __restrict__ sorted, const float* __restrict__ partial,
                                                                         float scale, float* __restrict__ d_table, int rows, int H,
                                                                         int vocab, int R) {
  __shared__ float part[kJoinWaves][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = blockIdx.x, col = lane * 8, c = blockIdx.y * 512 + col;
  const long p0 = (long)piece * R, p1 = p0 + R;
  if (p1 >= rows) return;
  const int tok = sorted[p1 - 1];
  if (tok >= vocab || sorted[p1] != tok || (p0 > 0 && sorted[p0] == tok && sorted[p0 - 1] == tok)) return;
  int n = 1;  // partial sums of the run
  for (;; n += 64) {
    const long q = (long)(piece + n + lane) * R;
    const unsigned long long in = __ballot(q < rows && sorted[min(q, (long)rows - 1)] == tok);
    if (in != ~0ull) {
      n += __popcll(in);  // pieces of a run follow each other: the set bits are the lowest
      break;
    }
  }
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < H) {
#pragma unroll 8
    for (int k = wave; k < n; k += kJoinWaves) {
      float v[8];
      load8(partial + ((size_t)(piece + k) * 2 + (k == 0 ? 1 : 0)) * H + c, v);
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[j];
    }
  }
  store8(part[wave] + col, acc);
  __syncthreads();
  if (wave || c >= H) return;
  const int waves = min(n, kJoinWaves);
  for (int w = 1; w < waves; ++w) {
    float v[8];
    load8(part[w] + col, v);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc[j] += v[j];
  }
  float* dst = d_table + (size_t)tok * H + c;
  float old[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if constexpr (ADD) load8(dst, old);
#pragma unroll
  for (int j = 0; j < 8; ++j) old[j] += scale * acc[j];
  store8(dst, old);
}

__global__ __launch_bounds__(256) void clear_kernel(f32x4* __restrict__ out, size_t n) { clear_share(out, n, blockIdx.x, gridDim.x, 256); }

// Up to so many rows the comparison of all pairs is the faster sort.
constexpr int kRankRows = 16384;

// Rows of a piece: enough pieces for four wavefronts on every SIMD where the rows allow it.
int piece_rows(int rows, int H) {
  const long slabs = (H + 511) / 512;
  for (int r = 64; r > 16; r /= 2)
    if ((long)rows / r * slabs >= 4096) return r;
  return 16;
}

struct EmbeddingLayout {
  size_t order[2], sorted[2], counts, partial, bytes;
};
EmbeddingLayout embedding_layout(int rows, int H) {
  EmbeddingLayout L{};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += align_up(bytes, 256);
    return here;
  };
  const bool radix = rows > kRankRows;
  for (int i = 0; i < (radix ? 2 : 1); ++i) {
    L.order[i] = take((size_t)rows * 4);
    L.sorted[i] = take((size_t)rows * 4);
  }
  L.counts = take(radix ? (size_t)kMaxSorters * kMaxBins * 4 : 0);
  const int r = piece_rows(rows, H);
  L.partial = take(((size_t)rows + r - 1) / r * 2 * H * sizeof(float));
  L.bytes = at;
  return L;
}

template <typename T, bool ADD>
int embedding_sums(const int32_t* order, const int32_t* sorted, const void* dout, float scale, float* d_table, float* partial, int rows,
                   int H, int vocab, hipStream_t stream) {
  const int r = piece_rows(rows, H), pieces = (rows + r - 1) / r, slabs = (H + 511) / 512;
  launch_kernel((embedding_sum_kernel<T, ADD>), dim3((pieces + 3) / 4, slabs), dim3(256), 0, stream, order, sorted, (const T*)dout, scale,
                d_table, partial, rows, H, vocab, r);
  if (const int rc = check_launch("embedding_backward (sums)")) return rc;
  if (pieces < 2) return HANAYO_OK;  // no border to cross
  launch_kernel((embedding_join_kernel<ADD>), dim3(pieces - 1, slabs), dim3(kJoinWaves * 64), 0, stream, sorted, partial, scale, d_table,
                rows, H, vocab, r);
  return check_launch("embedding_backward (join)");
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

size_t embedding_workspace_bytes(int rows, int H) { return embedding_layout(rows, H).bytes + 256; }

int embedding_backward(int dtype, const int32_t* tokens, const void* dout, float scale, float* d_table, int rows, int H, int vocab,
                       bool accumulate, void* workspace, hipStream_t stream) {
  f32x4* clear = reinterpret_cast<f32x4*>(d_table);
  const size_t clear_n = accumulate ? 0 : (size_t)vocab * H / 4;
  auto clearers = [&](int threads) {
    const size_t want = (clear_n + threads - 1) / threads;
    return (int)(want < 4096 ? want : 4096);
  };
  if (rows == 0) {
    if (!clear_n) return HANAYO_OK;
    launch_kernel(clear_kernel, dim3(clearers(256)), dim3(256), 0, stream, clear, clear_n);
    return check_launch("embedding_backward (clear)");
  }
  char* ws = static_cast<char*>(workspace);
  const EmbeddingLayout L = embedding_layout(rows, H);
  auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  int32_t *order = ints(L.order[0]), *sorted = ints(L.sorted[0]);
  if (rows <= kRankRows) {
    const int sorters = (rows + 63) / 64;
    launch_kernel(token_rank_kernel, dim3(sorters + clearers(1024)), dim3(1024), 0, stream, tokens, rows, vocab, order, sorted, sorters,
                  clear, clear_n);
    if (const int rc = check_launch("embedding_backward (sort)")) return rc;
  } else {
    int bits = 1;
    while (bits < 31 && (vocab >> bits)) ++bits;  // the keys are 0 .. vocab
    const int passes = (bits + 8) / 9;
    SortArgs a{};
    a.tokens = tokens; a.rows = rows; a.vocab = vocab; a.counts = ints(L.counts);
    const int unit = kSortWaves * 64;  // each wavefront's share is whole rounds of 64
    a.each = ((rows + kMaxSorters - 1) / kMaxSorters + unit - 1) / unit * unit;
    if (a.each < 1024) a.each = 1024;
    a.sorters = (rows + a.each - 1) / a.each;
    for (int pass = 0; pass < passes; ++pass) {
      a.shift = pass * bits / passes;
      a.bits = (pass + 1) * bits / passes - a.shift;
      const int to = pass & 1;
      a.order_out = ints(L.order[to]); a.sorted_out = ints(L.sorted[to]);
      launch_kernel(sort_count_kernel, dim3(a.sorters + (pass ? 0 : clearers(256))), dim3(256), 0, stream, a, clear, clear_n);
      if (const int rc = check_launch("embedding_backward (sort, count)")) return rc;
      launch_kernel(sort_place_kernel, dim3(a.sorters), dim3(kSortWaves * 64), 0, stream, a);
      if (const int rc = check_launch("embedding_backward (sort, place)")) return rc;
      a.tokens = nullptr;
      a.order_in = a.order_out; a.sorted_in = a.sorted_out;
    }
    order = a.order_out;
    sorted = a.sorted_out;
  }
  float* partial = reinterpret_cast<float*>(ws + L.partial);
  if (dtype == HANAYO_BF16)
    return accumulate ? embedding_sums<bf16, true>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, stream)
                      : embedding_sums<bf16, false>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, stream);
  return accumulate ? embedding_sums<float, true>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, stream)
                    : embedding_sums<float, false>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, stream);
}

}  // namespace k
}  // namespace hanayo
