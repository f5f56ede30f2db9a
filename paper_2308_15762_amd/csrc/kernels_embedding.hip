// Embedding lookup with a scale, and its gradient by sorted tokens.
//
//   out[t] = scale * table[token[t]],    d_table[v] (+)= scale * sum over t with token[t] = v of dout[t]
//
// Both are bound by HBM where they are large and by their launches where they are small.  The gradient first sorts the rows by
// token (ties in row order), so that the rows of a token follow each other and are added in a fixed order without
// atomics, whatever the distribution of the tokens.  MI355X, bf16: lookup of 4096 rows of 1024 4.0 us; 65521 rows 44.3 us (fp32 93.9);
// gradient of 65521 such rows, a quarter of them padding, 30592 tokens, written whole: sort 24 us in four launches, sums and clearing 47 us
// (226 MB, 4.8 TB/s; rows in random order alone cost 13 % of a copy's rate), borders 6.9 us.
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

typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(4), aligned(4))) int i32x4_any;  // four tokens, on any token's boundary

// ------------------------------------------------------------------ rows sorted by token
// Keys are tokens; one outside [0, vocab) counts as `vocab` and goes to the end.  Two ways to the same order: every row counts the
// rows before it (few rows, one launch), or a radix sort (many rows, two launches for every 9 bits of the vocabulary).
__device__ __forceinline__ int token_key(const int32_t* tokens, int t, int vocab) { return (int)min((unsigned)tokens[t], (unsigned)vocab); }

// Memory cleared by workgroups of a launch beside those that sort.
__device__ __forceinline__ void clear_share(f32x4* out, size_t n, int share, int shares, int threads) {
  const size_t step = (size_t)shares * threads;
#pragma unroll 4
  for (size_t i = (size_t)share * threads + threadIdx.x; i < n; i += step)
    put<true>(out + i, f32x4{0.f, 0.f, 0.f, 0.f});
}

// Where each row goes: the number of rows that sort before it, by token and, among equal tokens, by row.  A workgroup places 16
// rows: a lane compares row lane % 16 with four tokens of every sixteen that its wavefront takes from LDS, so that the comparisons
// spread over four times the CUs that a row per lane would use.  Tokens before the 16 rows count where they are at most the row's,
// tokens behind them where they are less.
__global__ __launch_bounds__(1024) void token_rank_kernel(const int32_t* __restrict__ tokens, int rows, int vocab,
                                                          int32_t* __restrict__ order, int32_t* __restrict__ sorted, int sorters,
                                                          f32x4* __restrict__ clear, size_t clear_n) {
  __shared__ int part[16][16];
  extern __shared__ i32x4 keys[];  // all rows' keys, behind the last row ones that sort behind everything
  if ((int)blockIdx.x >= sorters) {
    clear_share(clear, clear_n, blockIdx.x - sorters, gridDim.x - sorters, 1024);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int own = blockIdx.x, t = own * 16 + (lane & 15), quad = lane >> 4;
  const int spans = (rows + 15) / 16;
  for (int q = threadIdx.x; q < spans * 4; q += 1024) {
    i32x4 v;
    if (q * 4 + 4 <= rows) {
      v = *reinterpret_cast<const i32x4_any*>(tokens + q * 4);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = q * 4 + k < rows ? tokens[q * 4 + k] : -1;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = q * 4 + k < rows ? (int)min((unsigned)v[k], (unsigned)vocab) : -1;
    keys[q] = v;
  }
  __syncthreads();
  const unsigned mine = (unsigned)reinterpret_cast<const int*>(keys)[t];
  int before = 0;
#pragma unroll 8
  for (int span = wave; span < spans; span += 16) {
    const i32x4 v = keys[span * 4 + quad];
    const unsigned below = span < own ? mine + 1 : mine;  // mine is at most 2^31 - 1 where it counts
#pragma unroll
    for (int k = 0; k < 4; ++k) before += (unsigned)v[k] < below;
  }
  if (wave == own % 16) {
    const i32x4 v = keys[own * 4 + quad];
#pragma unroll
    for (int k = 0; k < 4; ++k) before += (unsigned)v[k] == mine && quad * 4 + k < (lane & 15);
  }
  before += __shfl_xor(before, 16);
  before += __shfl_xor(before, 32);
  if (lane < 16) part[wave][lane] = before;
  __syncthreads();
  if (threadIdx.x < 16 && t < rows) {
    int at = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) at += part[w][lane];
    order[at] = t;
    sorted[at] = (int)mine;
  }
}

// Radix sort by one digit: workgroup b owns the b-th run of `each` keys.  `counts` [workgroups][bins]: how often each digit occurs in
// each run.
constexpr int kMaxBins = 512, kMaxSorters = 256, kSortWaves = 16;
struct SortArgs {
  const int32_t* tokens;  // the first pass: keys from the tokens, rows in order; later passes: nullptr
  const int32_t *order_in, *sorted_in;
  int32_t *order_out, *sorted_out, *counts;
  unsigned char* present;  // the last pass: [vocab], 1 for every token that occurs; else nullptr
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
// wavefronts (a wavefront owns a sixteenth of the run), in order.  64 keys at a time: a ballot for each bit of the digit finds the
// lanes with the same one.  The counts of all runs are read by all 1024 threads: two digits each, every fourth run.
__global__ __launch_bounds__(kSortWaves * 64) void sort_place_kernel(SortArgs a) {
  __shared__ int at[kSortWaves][kMaxBins];  // where the wavefront's next key of a digit goes
  __shared__ int2 sums[2][4][kMaxBins / 2];  // of each group of runs: keys of a digit in all runs, in earlier runs
  __shared__ int wave_total[kSortWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, bins = 1 << a.bits;
  const int begin = blockIdx.x * a.each, end = min(begin + a.each, a.rows);
  const int share = a.each / kSortWaves, w0 = min(begin + wave * share, end), w1 = min(w0 + share, end);
  for (int d = lane; d < bins; d += 64) at[wave][d] = 0;  // its own counters: no other wavefront sees them yet
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  for (int i = w0 + lane; i < w1; i += 64) atomicAdd(&at[wave][sort_key(a, i) >> a.shift & (bins - 1)], 1);
  const int pair = threadIdx.x % (kMaxBins / 2), group = threadIdx.x / (kMaxBins / 2);
  int2 total = make_int2(0, 0), earlier = make_int2(0, 0);
  if (2 * pair < bins) {
#pragma unroll 16
    for (int b = group; b < a.sorters; b += 4) {
      const int2 c = *reinterpret_cast<const int2*>(a.counts + b * bins + 2 * pair);
      const int mine = b < (int)blockIdx.x ? -1 : 0;
      total.x += c.x;
      total.y += c.y;
      earlier.x += c.x & mine;
      earlier.y += c.y & mine;
    }
  }
  sums[0][group][pair] = total;
  sums[1][group][pair] = earlier;
  __syncthreads();
  // a thread per digit: the keys of smaller digits (a running sum over the lanes and the wavefronts before), then the places of the
  // digit's keys in this run, wavefront by wavefront
  const int d = threadIdx.x;
  const int* all = reinterpret_cast<const int*>(sums);
  int n = 0, ahead = 0;
  if (d < bins) {
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      n += all[g * kMaxBins + d];
      ahead += all[(4 + g) * kMaxBins + d];
    }
  }
  int upto = n;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int add = __shfl_up(upto, o);
    if (lane >= o) upto += add;
  }
  if (lane == 63) wave_total[wave] = upto;
  __syncthreads();
  if (d < bins) {
    int next = upto - n + ahead;
    for (int w = 0; w < wave; ++w) next += wave_total[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      const int c = at[w][d];
      at[w][d] = next;
      next += c;
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
      const int to = at[wave][digit] + before;  // read by all lanes before the first of them moves the counter on
      a.order_out[to] = a.tokens ? i : a.order_in[i];
      a.sorted_out[to] = key;
      if (a.present && key < a.vocab) a.present[key] = 1;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (have && before == 0) at[wave][digit] += __popcll(same);
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

// ------------------------------------------------------------------ sums over the runs of equal tokens
// The sorted rows are cut into pieces of R (8 .. 64), a wavefront per piece and 512 columns, so that the work is even whatever the
// tokens: a run of a token that lies within a piece is added up and written; of one that crosses a border the piece leaves its part
// in LDS (slot 0: the run comes from the piece before; slot 1: it starts here).  The workgroup then goes through its eight pieces'
// parts in order: runs that lie within the workgroup's rows are written, and of those that cross its border it leaves its part in
// memory, in two slots again, which the kernel below adds up.  A piece's tokens and rows lie in the lanes; eight rows are loaded
// while the eight before them are added.
// Where the table is written whole (`present`), workgroups behind those clear the rows of the tokens that do not occur, a wavefront
// sixteen tokens.
constexpr int kPieces = 8, kClearTokens = 16;  // of a workgroup; of a wavefront
template <typename T, bool ADD>
__global__ __launch_bounds__(kPieces * 64) void embedding_sum_kernel(const int32_t* __restrict__ order, const int32_t* __restrict__ sorted,
                                                                     const T* __restrict__ dout, float scale,
                                                                     float* __restrict__ d_table, float* __restrict__ partial, int rows,
                                                                     int H, int vocab, int R, int slabs, int groups,
                                                                     const unsigned char* __restrict__ present) {
  __shared__ float parts[kPieces][2][512];
  __shared__ int left[kPieces];  // what a piece left: bit 0 slot 0, bit 1 slot 1, bit 2: the run of slot 0 ends in the piece
  __shared__ int run_of[kPieces];  // the token of the piece's first row, that of slot 0
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (!ADD && (int)blockIdx.x >= groups * slabs) {
    const long v0 = ((long)(blockIdx.x - groups * slabs) * kPieces + wave) * kClearTokens;
    unsigned long long absent = __ballot(lane < kClearTokens && v0 + lane < vocab && !present[min(v0 + lane, (long)vocab - 1)]);
    for (; absent; absent &= absent - 1) {
      f32x4* out = reinterpret_cast<f32x4*>(d_table + (size_t)(v0 + __builtin_ctzll(absent)) * H);
#pragma unroll 4
      for (int i = lane; i < H / 4; i += 64) put<true>(out + i, f32x4{0.f, 0.f, 0.f, 0.f});
    }
    return;
  }
  // the slabs of a group of pieces follow each other, so that their rows are read at one time
  const int group = blockIdx.x / slabs, slab = blockIdx.x - group * slabs;
  const int c = (slab * 64 + lane) * 8;
  const bool inside = c < H;
  const long p0 = ((long)group * kPieces + wave) * R;
  const int n = p0 < rows ? min(R, (int)(rows - p0)) : 0;
  const int tok = lane < n ? sorted[p0 + lane] : -1, row = lane < n ? order[p0 + lane] : 0;
  const int before = p0 > 0 && n ? sorted[p0 - 1] : -1, after = p0 + n < rows ? sorted[p0 + n] : -1;
  const int live = __popcll(__ballot(lane < n && tok < vocab));
  if (lane == 0) left[wave] = 0;
  if (live) {
    const int first = __builtin_amdgcn_readfirstlane(tok);
    const int next = __shfl_down(tok, 1);
    const unsigned long long ends = __ballot(lane < n && (lane == n - 1 || tok != next));  // the last rows of runs
    unsigned long long whole = ends;                                                       // of runs that lie in the piece
    bool head = before == first;                                                           // the first run comes from before
    const bool tail = live == n && after == __builtin_amdgcn_readlane(tok, n - 1);         // the last one goes on
    if (lane == 0) {
      const bool one = (ends & (ends - 1)) == 0;  // a single run
      left[wave] = (head ? 1 | (one && tail ? 0 : 4) : 0) | (tail && !(one && head) ? 2 : 0);
      run_of[wave] = first;
    }
    if (head) whole &= whole - 1;
    if (tail) whole &= ~(1ull << (n - 1));
    float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    constexpr int U = sizeof(T) == 2 ? 8 : 4;
    Raw8<T> rows_now[U], rows_next[U];
    auto fetch_rows = [&](Raw8<T>(&v)[U], int i0) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].load(dout + (size_t)__builtin_amdgcn_readlane(row, min(i0 + u, live - 1)) * H + c);
    };
    if (inside) fetch_rows(rows_next, 0);
    for (int i0 = 0; i0 < live; i0 += U) {
      float old[U][8];
      if (inside) {
        if constexpr (ADD) {
#pragma unroll
          for (int u = 0; u < U; ++u)
            if (i0 + u < live && (whole >> (i0 + u) & 1))
              load8(d_table + (size_t)__builtin_amdgcn_readlane(tok, i0 + u) * H + c, old[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) rows_now[u] = rows_next[u];
        if (i0 + U < live) fetch_rows(rows_next, i0 + U);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u;
        if (i >= live) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += rows_now[u].get(j);
        if (ends >> i & 1) {
          if (whole >> i & 1) {
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] = ADD ? old[u][j] + scale * acc[j] : scale * acc[j];
            if (inside) store8(d_table + (size_t)__builtin_amdgcn_readlane(tok, i) * H + c, acc);
          } else {
            store8(&parts[wave][head ? 0 : 1][lane * 8], acc);
          }
          head = false;
#pragma unroll
          for (int j = 0; j < 8; ++j) acc[j] = 0.f;
        }
      }
    }
  }
  __syncthreads();
  // a thread per column
  const int col = threadIdx.x, gc = slab * 512 + col;
  static_assert(kPieces * 64 == 512, "a thread per column");
  if (gc >= H) return;
  float* mine = partial + (size_t)group * 2 * H + gc;
  float run = 0.f;
  bool open = false, ours = false;  // a run goes on; it starts in these pieces
  for (int w = 0; w < kPieces; ++w) {
    const int what = left[w];
    if (what & 1) {
      run = open ? run + parts[w][0][col] : parts[w][0][col];
      open = true;
      if (what & 4) {
        if (ours) {
          float* dst = d_table + (size_t)run_of[w] * H + gc;
          *dst = ADD ? *dst + scale * run : scale * run;
        } else {
          mine[0] = run;
        }
        open = ours = false;
      }
    }
    if (what & 2) {
      run = parts[w][1][col];
      open = ours = true;
    }
  }
  if (open) mine[ours ? H : 0] = run;
}

// The runs that cross a border between workgroups of the kernel above, whose rows are a piece here (R of them), each by the
// wavefront of the piece that it starts in: that piece's slot 1 and slot 0 of the pieces behind it.  Runs over many pieces are listed
// and then added by all wavefronts of the workgroup, every eighth partial sum each, whose sums are added in order.
constexpr int kJoinWaves = 8, kJoinAlone = 16;
struct JoinArgs {
  const int32_t* sorted;
  const float* partial;
  float scale;
  float* d_table;
  int rows, H, vocab, R;
};
__device__ __forceinline__ void join_partials(const JoinArgs& a, int piece, int first, int n, int step, int c, float (&acc)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) acc[j] = 0.f;
  constexpr int U = 16;  // loads in flight; behind the last one it is read again and not added
  for (int k0 = first; k0 < n; k0 += U * step) {
    float v[U][8];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(k0 + u * step, n - 1);
      load8(a.partial + ((size_t)(piece + k) * 2 + (k == 0 ? 1 : 0)) * a.H + c, v[u]);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * step >= n) break;
#pragma unroll
      for (int j = 0; j < 8; ++j) acc[j] += v[u][j];
    }
  }
}
template <bool ADD>
__device__ __forceinline__ void join_store(const JoinArgs& a, int tok, int c, float (&acc)[8]) {
  float* dst = a.d_table + (size_t)tok * a.H + c;
  float old[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if constexpr (ADD) load8(dst, old);
#pragma unroll
  for (int j = 0; j < 8; ++j) old[j] += a.scale * acc[j];
  store8(dst, old);
}
template <bool ADD>
__global__ __launch_bounds__(kJoinWaves * 64) void embedding_join_kernel(JoinArgs a) {
  __shared__ float part[kJoinWaves][512];
  __shared__ int runs[kJoinWaves][3];  // piece, token, partial sums (0: nothing for the workgroup)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int piece = blockIdx.x * kJoinWaves + wave, c = (blockIdx.y * 64 + lane) * 8;
  const long p0 = (long)piece * a.R, p1 = p0 + a.R;
  int n = 0, tok = 0;
  if (p1 < a.rows) {
    tok = a.sorted[p1 - 1];
    if (tok < a.vocab && a.sorted[p1] == tok && !(p0 > 0 && a.sorted[p0] == tok && a.sorted[p0 - 1] == tok)) {
      // pieces of a run follow each other: among 256 looked at together, those that hold the token are the first
      for (n = 1;; n += 256) {
        int in = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const long q = (long)(piece + n + 64 * k + lane) * a.R;
          in += __popcll(__ballot(q < a.rows && a.sorted[min(q, (long)a.rows - 1)] == tok));
        }
        if (in < 256) {
          n += in;
          break;
        }
      }
    }
  }
  if (lane == 0) {
    runs[wave][0] = piece;
    runs[wave][1] = tok;
    runs[wave][2] = n > kJoinAlone ? n : 0;
  }
  float acc[8];
  if (n > 0 && n <= kJoinAlone && c < a.H) {
    join_partials(a, piece, 0, n, 1, c, acc);
    join_store<ADD>(a, tok, c, acc);
  }
  __syncthreads();
  for (int r = 0; r < kJoinWaves; ++r) {
    const int many = runs[r][2];  // the same for the whole workgroup
    if (!many) continue;
    if (c < a.H) join_partials(a, runs[r][0], wave, many, kJoinWaves, c, acc);
    store8(part[wave] + lane * 8, acc);
    __syncthreads();
    if (wave == 0 && c < a.H) {
      for (int w = 1; w < kJoinWaves; ++w) {
        float v[8];
        load8(part[w] + lane * 8, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[j];
      }
      join_store<ADD>(a, runs[r][1], c, acc);
    }
    __syncthreads();
  }
}

// Few rows and a small table: a workgroup per token and 512 columns lists the token's rows, in order, and adds them up, every
// fourth row by one wavefront; no sort, no second launch, and tokens that do not occur are cleared on the way.  512 columns: 128 rows
// of 512 to 4096 tokens 6.8 us against 12.7 with the sort, 8192 tokens 7.6, 16384 tokens 12.2 against 13.4; 1024 rows of 4096 tokens
// 8.9 against 14.1, 8192 tokens 13.1 against 15.0, 16384 tokens 23.2 against 17.0.
constexpr int kDirectRows = 1024, kDirectGroups = 8192;
template <typename T, bool ADD>
__global__ __launch_bounds__(256) void embedding_direct_kernel(const int32_t* __restrict__ tokens, const T* __restrict__ dout,
                                                               float scale, float* __restrict__ d_table, int rows, int H) {
  __shared__ int list[kDirectRows];
  __shared__ int counts[kDirectRows / 64];
  __shared__ float part[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tok = blockIdx.x, c = (blockIdx.y * 64 + lane) * 8;
  const int groups = (rows + 63) / 64;
  bool hit[kDirectRows / 256];
  unsigned long long mask[kDirectRows / 256];
#pragma unroll
  for (int k = 0; k < kDirectRows / 256; ++k) {
    const int t = k * 256 + threadIdx.x;
    hit[k] = t < rows && tokens[t] == tok;
    mask[k] = __ballot(hit[k]);
    if (lane == 0) counts[k * 4 + wave] = __popcll(mask[k]);
  }
  __syncthreads();
  int n = 0;
#pragma unroll
  for (int g = 0; g < kDirectRows / 64; ++g) {
    if (g >= groups) break;
    if ((g & 3) == wave && hit[g >> 2]) list[n + __popcll(mask[g >> 2] & ((1ull << lane) - 1ull))] = g * 64 + lane;
    n += counts[g];
  }
  if (ADD && n == 0) return;
  __syncthreads();
  float acc[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (c < H) {
    constexpr int U = 8;
    for (int i0 = wave; i0 < n; i0 += 4 * U) {
      Raw8<T> v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) v[u].load(dout + (size_t)list[min(i0 + 4 * u, n - 1)] * H + c);
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (i0 + 4 * u >= n) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] += v[u].get(j);
      }
    }
  }
  if (n > 1) {
    store8(part[wave] + lane * 8, acc);
    __syncthreads();
  }
  if (wave || c >= H) return;
  for (int w = 1; w < min(n, 4); ++w) {
    float v[8];
    load8(part[w] + lane * 8, v);
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

template <typename T>
int embedding_direct(const int32_t* tokens, const void* dout, float scale, float* d_table, int rows, int H, int vocab, bool accumulate,
                     hipStream_t stream) {
  const dim3 grid(vocab, (H + 511) / 512);
  if (accumulate)
    launch_kernel((embedding_direct_kernel<T, true>), grid, dim3(256), 0, stream, tokens, (const T*)dout, scale, d_table, rows, H);
  else
    launch_kernel((embedding_direct_kernel<T, false>), grid, dim3(256), 0, stream, tokens, (const T*)dout, scale, d_table, rows, H);
  return check_launch("embedding_backward (direct)");
}

// Up to so many rows the comparison of all pairs is the faster sort, and its keys fit the LDS (512 columns, whole call: 4096 rows
// 15.5 us against 25.5 with the radix sort, 8192 rows 22.6 against 30.8, 12288 rows 30.0 against 32.1).
constexpr int kRankRows = 12288;

// Rows of a piece: as many as leave 4096 pieces, two workgroups of eight for every CU; eight rows where there are too few (whole call, 65521
// rows of 1024, table written: 16 rows 76.8 us, 8 rows 77.9, 32 rows 85, 64 rows 98; 4096 rows, added: 8 rows 17.5, 16 rows 20.2, 32 rows
// 27.8).  Two workgroups of the written form (115 registers) fit a CU together, one of the added form (bf16: 180 registers).  4096 rows of 1024 are
// 128 workgroups: half of the CUs have none.
int piece_rows(int rows, int H) {
  const long slabs = (H + 511) / 512;
  for (int r = 64; r > 8; r /= 2)
    if ((long)rows / r * slabs >= 4096) return r;
  return 8;
}

struct EmbeddingLayout {
  size_t order[2], sorted[2], counts, present, partial, bytes;
};
EmbeddingLayout embedding_layout(int rows, int H, int vocab) {
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
  L.present = take(radix ? (size_t)vocab : 0);
  const int each = piece_rows(rows, H) * kPieces;
  L.partial = take(((size_t)rows + each - 1) / each * 2 * H * sizeof(float));
  L.bytes = at;
  return L;
}

template <typename T, bool ADD>
int embedding_sums(const int32_t* order, const int32_t* sorted, const void* dout, float scale, float* d_table, float* partial, int rows,
                   int H, int vocab, const unsigned char* present, hipStream_t stream) {
  const int r = piece_rows(rows, H), each = r * kPieces, groups = (rows + each - 1) / each, slabs = (H + 511) / 512;
  const long clearers = present ? ((long)vocab + kPieces * kClearTokens - 1) / (kPieces * kClearTokens) : 0;
  launch_kernel((embedding_sum_kernel<T, ADD>), dim3((unsigned)((long)groups * slabs + clearers)), dim3(kPieces * 64), 0, stream, order, sorted,
                (const T*)dout, scale, d_table, partial, rows, H, vocab, r, slabs, groups, present);
  if (const int rc = check_launch("embedding_backward (sums)")) return rc;
  if (groups < 2) return HANAYO_OK;  // no border to cross
  launch_kernel((embedding_join_kernel<ADD>), dim3((groups - 1 + kJoinWaves - 1) / kJoinWaves, slabs), dim3(kJoinWaves * 64), 0, stream,
                JoinArgs{sorted, partial, scale, d_table, rows, H, vocab, each});
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

size_t embedding_workspace_bytes(int rows, int H, int vocab) { return embedding_layout(rows, H, vocab).bytes + 256; }

int embedding_backward(int dtype, const int32_t* tokens, const void* dout, float scale, float* d_table, int rows, int H, int vocab,
                       bool accumulate, void* workspace, hipStream_t stream) {
  f32x4* clear = reinterpret_cast<f32x4*>(d_table);
  const size_t clear_n = accumulate ? 0 : (size_t)vocab * H / 4;
  auto clearers = [&](size_t n, int threads) {
    const size_t want = (n + threads - 1) / threads, most = (size_t)(1 << 20) / threads;
    return (int)(want < most ? want : most);
  };
  if (rows == 0) {
    if (!clear_n) return HANAYO_OK;
    launch_kernel(clear_kernel, dim3(clearers(clear_n, 256)), dim3(256), 0, stream, clear, clear_n);
    return check_launch("embedding_backward (clear)");
  }
  if (rows <= kDirectRows && (long)vocab * ((H + 511) / 512) <= kDirectGroups)
    return dtype == HANAYO_BF16 ? embedding_direct<bf16>(tokens, dout, scale, d_table, rows, H, vocab, accumulate, stream)
                                : embedding_direct<float>(tokens, dout, scale, d_table, rows, H, vocab, accumulate, stream);
  char* ws = static_cast<char*>(workspace);
  const EmbeddingLayout L = embedding_layout(rows, H, vocab);
  auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(ws + at); };
  int32_t *order = ints(L.order[0]), *sorted = ints(L.sorted[0]);
  unsigned char* present = nullptr;
  if (rows <= kRankRows) {
    // few rows touch little of the table: all of it is cleared beside the sort
    const int sorters = (rows + 15) / 16;
    launch_kernel(token_rank_kernel, dim3(sorters + clearers(clear_n, 1024)), dim3(1024), (size_t)sorters * 64, stream, tokens, rows,
                  vocab, order, sorted, sorters, clear, clear_n);
    if (const int rc = check_launch("embedding_backward (sort)")) return rc;
  } else {
    if (!accumulate) present = reinterpret_cast<unsigned char*>(ws + L.present);
    const size_t present_n = accumulate ? 0 : ((size_t)vocab + 15) / 16;  // the layout rounds up to 256 bytes
    int bits = 1;
    while (bits < 31 && (vocab >> bits)) ++bits;  // the keys are 0 .. vocab
    const int passes = (bits + 8) / 9;
    SortArgs a{};
    a.tokens = tokens; a.rows = rows; a.vocab = vocab; a.counts = ints(L.counts);
    const int unit = kSortWaves * 64;  // each wavefront's share is whole rounds of 64
    a.each = ((rows + kMaxSorters - 1) / kMaxSorters + unit - 1) / unit * unit;
    a.sorters = (rows + a.each - 1) / a.each;
    for (int pass = 0; pass < passes; ++pass) {
      a.shift = pass * bits / passes;
      a.bits = (pass + 1) * bits / passes - a.shift;
      const int to = pass & 1;
      a.order_out = ints(L.order[to]); a.sorted_out = ints(L.sorted[to]);
      a.present = pass == passes - 1 ? present : nullptr;
      const size_t n = pass == 0 ? present_n : 0;
      launch_kernel(sort_count_kernel, dim3(a.sorters + clearers(n, 256)), dim3(256), 0, stream, a, reinterpret_cast<f32x4*>(present), n);
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
    return accumulate ? embedding_sums<bf16, true>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, nullptr, stream)
                      : embedding_sums<bf16, false>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, present, stream);
  return accumulate ? embedding_sums<float, true>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, nullptr, stream)
                    : embedding_sums<float, false>(order, sorted, dout, scale, d_table, partial, rows, H, vocab, present, stream);
}

}  // namespace k
}  // namespace hanayo
