// Tokens to rows in expert order and back, as operators of their own: row order from the experts of the pairs, dispatch of the
// tokens' rows, combine with the weights, their gradients, and the gate's gradient.
//
// With pairs q = t*k + j and e(q) the expert of pair q, the row of q is the number of pairs of lower experts plus the number of
// its own expert's pairs before it; pairs without an expert have no row.  All of it is data movement: a row is read once and
// written once (but a token's row for every slot in the gradient of a combine of more than 8), sums over a token's k rows and over a
// row's columns are fp32 in a fixed order.
#include "row_vector.h"

namespace moe {

constexpr int kSortChunk = 1024;        // pairs of a workgroup
constexpr int kBuckets = kMaxExperts + 1;   // the last one, number E, takes the pairs without an expert
constexpr int kMaxGateTopK = 64;
constexpr int kMinRowColumns = 8, kMaxRowColumns = 65536;

__device__ __forceinline__ int bucket_of(const int32_t* ids, int q, int E) {
  const int e = ids[q];
  return (unsigned)e < (unsigned)E ? e : E;
}

// Lanes of the wavefront with the same bucket (up to 9 bits) as this one, among the valid ones.
__device__ __forceinline__ uint64_t same_bucket(int e, bool valid) {
  uint64_t same = __ballot(valid);
#pragma unroll
  for (int bit = 0; bit < 9; bit++) {
    const uint64_t b = __ballot((e >> bit) & 1);
    same &= ((e >> bit) & 1) ? b : ~b;
  }
  return same;
}

// Exclusive prefix sum over kBuckets values in LDS, by the first wavefront.
__device__ __forceinline__ void scan_buckets(const int32_t* count, int32_t* first) {
  constexpr int kEach = (kBuckets + 63) / 64;
  if (threadIdx.x >= 64) return;
  const int lane = threadIdx.x;
  int v[kEach], sum = 0;
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    const int e = lane * kEach + i;
    v[i] = e < kBuckets ? count[e] : 0;
    sum += v[i];
  }
  int incl = sum;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int o = __shfl_up(incl, d);
    if (lane >= d) incl += o;
  }
  int at = incl - sum;
#pragma unroll
  for (int i = 0; i < kEach; i++) {
    const int e = lane * kEach + i;
    if (e < kBuckets) first[e] = at;
    at += v[i];
  }
}

// Up to RUNS * 64 pairs in one workgroup: a run of 64 pairs a wavefront, ranks inside it by ballots, prefix sums over the runs.  us for 32
// pairs with one run / as one of the chunks below 2.2 / 2.8, 192 with four 2.3 / 2.9, 1024 with sixteen 3.0 / 3.1.
template <int RUNS>
__global__ __launch_bounds__(RUNS * 64) void k_sort_one(const int32_t* __restrict__ ids, int R, int E, int32_t* __restrict__ offsets,
                                                        int32_t* __restrict__ perm, int32_t* __restrict__ inv) {
  constexpr int kThreads = RUNS * 64;
  __shared__ int32_t run_cnt[RUNS][kBuckets];
  __shared__ int32_t count[kBuckets], first[kBuckets];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, q = threadIdx.x;
  const int e = q < R ? bucket_of(ids, q, E) : -1;
  for (int i = threadIdx.x; i < RUNS * kBuckets; i += kThreads) (&run_cnt[0][0])[i] = 0;
  __syncthreads();
  const uint64_t same = same_bucket(e, e >= 0), below = same & ((1ull << lane) - 1ull);
  const int rank = __popcll(below);
  if (e >= 0 && below == 0) run_cnt[wave][e] = __popcll(same);
  __syncthreads();
  for (int i = threadIdx.x; i < kBuckets; i += kThreads) {
    int acc = 0;
#pragma unroll
    for (int r = 0; r < RUNS; r++) {
      const int c = run_cnt[r][i];
      run_cnt[r][i] = acc;
      acc += c;
    }
    count[i] = acc;
  }
  __syncthreads();
  scan_buckets(count, first);
  __syncthreads();
  if (e >= 0) {
    const int pos = first[e] + run_cnt[wave][e] + rank;
    perm[pos] = e < E ? q : -1;
    inv[q] = e < E ? pos : -1;
  }
  for (int i = threadIdx.x; i <= E; i += kThreads) offsets[i] = first[i];
}

// Pairs of each bucket in each chunk.
__global__ __launch_bounds__(1024) void k_sort_hist(const int32_t* __restrict__ ids, int R, int E, int32_t* __restrict__ hist) {
  __shared__ int32_t count[kBuckets];
  for (int e = threadIdx.x; e <= E; e += 1024) count[e] = 0;
  __syncthreads();
  const int q = blockIdx.x * kSortChunk + threadIdx.x;
  if (q < R) atomicAdd(&count[bucket_of(ids, q, E)], 1);
  __syncthreads();
  for (int e = threadIdx.x; e <= E; e += 1024) hist[(size_t)blockIdx.x * (E + 1) + e] = count[e];
}

// Many chunks: one workgroup per bucket turns its counts into prefix sums over the chunks, and leaves the total.
__global__ __launch_bounds__(1024) void k_sort_scan(int32_t* __restrict__ hist, int n_chunks, int E, int32_t* __restrict__ total) {
  __shared__ int32_t wave_sum_[16];
  const int e = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int at = 0;
  for (int b0 = 0; b0 < n_chunks; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    const int v = b < n_chunks ? hist[(size_t)b * (E + 1) + e] : 0;
    int incl = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int o = __shfl_up(incl, d);
      if (lane >= d) incl += o;
    }
    if (lane == 63) wave_sum_[wave] = incl;
    __syncthreads();
    int before = at, sum = 0;
#pragma unroll
    for (int w = 0; w < 16; w++) {
      const int c = wave_sum_[w];
      if (w < wave) before += c;
      sum += c;
    }
    if (b < n_chunks) hist[(size_t)b * (E + 1) + e] = before + incl - v;
    at += sum;
    __syncthreads();
  }
  if (threadIdx.x == 0) total[e] = at;
}

// Stable scatter of a chunk: a pair's row is the first one of its bucket, plus the bucket's pairs in the chunks before, in the runs of
// 64 before, and in the lanes before.  Where the bucket's pairs in other chunks come from:
// OWN: the workgroup counts all pairs itself, in 16 copies (by lane) of the counters, so that lanes with the same bucket seldom meet (us with 4 / 8 /
// 16 copies, 32768 pairs of 8 experts 8.2 / 7.4 / 6.8, of popular ones 10.7 / 7.6 / 6.4, of 64 6.5 / 6.6 / 6.5);
// otherwise from hist, as prefix sums over the chunks with their total, or as counts (total == nullptr), summed here by a thread per
// bucket and part of the chunks.
template <bool OWN>
__global__ __launch_bounds__(1024) void k_sort_scatter(const int32_t* __restrict__ ids, int R, int E, const int32_t* __restrict__ hist,
                                                       int n_chunks, const int32_t* __restrict__ total, int32_t* __restrict__ offsets,
                                                       int32_t* __restrict__ perm, int32_t* __restrict__ inv) {
  constexpr int kRuns = kSortChunk / 64, kCopies = 16;
  __shared__ int32_t run_cnt[kRuns][kBuckets];
  __shared__ int32_t count[kBuckets], first[kBuckets], before[kBuckets];
  __shared__ int32_t own[OWN ? 2 : 1][OWN ? kCopies : 1][OWN ? kBuckets : 1];   // pairs of earlier chunks, and of this and later ones
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = E + 1;
  const int q = blockIdx.x * kSortChunk + threadIdx.x;
  const int e = q < R ? bucket_of(ids, q, E) : -1;
  for (int i = threadIdx.x; i < kRuns * kBuckets; i += 1024) (&run_cnt[0][0])[i] = 0;
  if constexpr (OWN)
    for (int i = threadIdx.x; i < 2 * kCopies * kBuckets; i += 1024) (&own[0][0][0])[i] = 0;
  for (int i = threadIdx.x; i < kBuckets; i += 1024) {
    count[i] = !OWN && total != nullptr && i < n ? total[i] : 0;
    before[i] = !OWN && total != nullptr && i < n ? hist[(size_t)blockIdx.x * n + i] : 0;
  }
  __syncthreads();
  if constexpr (OWN) {
    const int copy = lane & (kCopies - 1), fours = R / 4;
    auto one = [&](int id, int later) { atomicAdd(&own[later][copy][(unsigned)id < (unsigned)E ? id : E], 1); };
#pragma unroll 4
    for (int i = threadIdx.x; i < fours; i += 1024) {
      const int4 v = ((const int4*)ids)[i];
      const int later = i * 4 >= (int)blockIdx.x * kSortChunk;   // (four pairs never lie in two chunks)
      one(v.x, later);
      one(v.y, later);
      one(v.z, later);
      one(v.w, later);
    }
    if (fours * 4 + (int)threadIdx.x < R) one(ids[fours * 4 + threadIdx.x], 1);   // up to three, in the last chunk
  } else if (total == nullptr) {
    const int parts = n <= 1024 / 16 ? 16 : n <= 1024 / 8 ? 8 : 3;
    const int b = threadIdx.x % n, part = threadIdx.x / n;
    if (part < parts) {
      int all = 0, mine = 0;
#pragma unroll 8
      for (int c = part; c < n_chunks; c += parts) {
        const int v = hist[(size_t)c * n + b];
        all += v;
        mine += c < (int)blockIdx.x ? v : 0;
      }
      atomicAdd(&count[b], all);   // (whole numbers: the order does not show)
      atomicAdd(&before[b], mine);
    }
  }
  const uint64_t same = same_bucket(e, e >= 0), below = same & ((1ull << lane) - 1ull);
  const int rank = __popcll(below);
  if (e >= 0 && below == 0) run_cnt[wave][e] = __popcll(same);
  __syncthreads();
  if constexpr (OWN) {
    for (int i = threadIdx.x; i < n; i += 1024) {
      int b = 0, a = 0;
#pragma unroll
      for (int c = 0; c < kCopies; c++) {
        b += own[0][c][i];
        a += own[1][c][i];
      }
      before[i] = b;
      count[i] = a + b;
    }
    __syncthreads();
  }
  scan_buckets(count, first);
  for (int i = threadIdx.x - 64; i >= 0 && i < n; i += 1024 - 64) {   // (the first wavefront is scanning)
    int acc = before[i];
#pragma unroll
    for (int r = 0; r < kRuns; r++) {
      const int c = run_cnt[r][i];
      run_cnt[r][i] = acc;
      acc += c;
    }
  }
  __syncthreads();
  if (e >= 0) {
    const int pos = first[e] + run_cnt[wave][e] + rank;
    perm[pos] = e < E ? q : -1;
    inv[q] = e < E ? pos : -1;
  }
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i <= E; i += 1024) offsets[i] = first[i];
}

__global__ void k_sort_none(int E, int32_t* __restrict__ offsets) {
  for (int e = threadIdx.x; e <= E; e += blockDim.x) offsets[e] = 0;
}

// ---------------------------------------------------------------------------------------------
// Rows.  LP lanes work on a token (64, or fewer where a row has few pieces of 16 bytes); with 64 everything about the
// token is the same in every lane and stays in scalar registers.
// ---------------------------------------------------------------------------------------------
template <int LP>
struct Unit {
  int wave, t, lane, span;
  __device__ __forceinline__ Unit(int spans) {
    wave = uniform((int)(threadIdx.x >> 6));
    const int u = blockIdx.x * 4 + wave;
    lane = threadIdx.x & (LP - 1);
    if constexpr (LP == 64) {
      t = u / spans;
      span = u - t * spans;
    } else {
      t = u * (64 / LP) + (int)((threadIdx.x & 63) / LP);
      span = 0;
    }
  }
};

// rows[inv[t][j]] = x[t]: a token's row is read once and written k times.
template <int LP, int NV>
__global__ __launch_bounds__(256) void k_dispatch(const char* x, const int32_t* __restrict__ inv, char* rows, int T, int k, int R,
                                                  uint32_t row_bytes, int spans) {
  constexpr int kGroup = 4;
  const Unit<LP> at(spans);
  if (at.t >= T) return;
  const char* src = x + (size_t)at.t * row_bytes;
  const uint32_t start = (uint32_t)at.span * (64 * 16 * NV) + at.lane * 16;
  u32x4 v[NV];
#pragma unroll
  for (int i = 0; i < NV; i++) v[i] = load_piece(src, start + i * (LP * 16), row_bytes);
  for (int j0 = 0; j0 < k; j0 += kGroup) {
    int pos[kGroup];
#pragma unroll
    for (int j = 0; j < kGroup; j++) pos[j] = j0 + j < k ? inv[(size_t)at.t * k + j0 + j] : -1;
#pragma unroll
    for (int j = 0; j < kGroup; j++) {
      if ((unsigned)pos[j] >= (unsigned)R) continue;   // no row
      char* dst = rows + (size_t)pos[j] * row_bytes;
#pragma unroll
      for (int i = 0; i < NV; i++) store_once(dst, start + i * (LP * 16), row_bytes, v[i]);
    }
  }
}

// out[t] = sum_j w[t][j] * rows[inv[t][j]] in the order of j, without weights the plain sum.  K > 0: up to K slots, the rows of
// all requested before the first is used; K == 0: any number, slot after slot.
template <int DT, int K, int LP, int NV>
__global__ __launch_bounds__(256) void k_combine_rows(const char* rows, const int32_t* __restrict__ inv, const float* __restrict__ w,
                                                      char* out, int T, int k, int R, uint32_t row_bytes, int spans) {
  using V = Row<DT>;
  constexpr int N = V::kVec, KK = K > 0 ? K : 1;
  const Unit<LP> at(spans);
  if (at.t >= T) return;
  const uint32_t start = (uint32_t)at.span * (64 * 16 * NV) + at.lane * 16;
  float acc[NV][N];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int c = 0; c < N; c++) acc[i][c] = 0.f;
  for (int j0 = 0; j0 < (K > 0 ? 1 : k); j0++) {
    int pos[KK];
    float wj[KK];
    u32x4 v[KK][NV];
#pragma unroll
    for (int j = 0; j < KK; j++) {
      const bool there = K == 0 || j < k;
      pos[j] = there ? inv[(size_t)at.t * k + j0 + j] : -1;
      wj[j] = there && w != nullptr ? w[(size_t)at.t * k + j0 + j] : 1.f;
    }
#pragma unroll
    for (int j = 0; j < KK; j++)
      if ((unsigned)pos[j] < (unsigned)R)
#pragma unroll
        for (int i = 0; i < NV; i++) v[j][i] = load_once(rows + (size_t)pos[j] * row_bytes, start + i * (LP * 16), row_bytes);
#pragma unroll
    for (int j = 0; j < KK; j++)
      if ((unsigned)pos[j] < (unsigned)R)
#pragma unroll
        for (int i = 0; i < NV; i++) {
          float f[N];
          V::unpack(v[j][i], f);
#pragma unroll
          for (int c = 0; c < N; c++) acc[i][c] = fmaf(wj[j], f[c], acc[i][c]);
        }
  }
  char* dst = out + (size_t)at.t * row_bytes;
#pragma unroll
  for (int i = 0; i < NV; i++) store_piece(dst, start + i * (LP * 16), row_bytes, V::pack(acc[i]));
}

// grad_rows[inv[t][j]] = w[t][j] * g[t], grad_w[t][j] = <g[t], rows[inv[t][j]]>, 0 for a slot without a row.  A token belongs to
// the wavefronts of a workgroup (LP == 64), which take its pieces in turn and add their sums up in LDS, or to LP lanes.
// rows == nullptr: no grad_w.
constexpr int kGradWaves = 8;
template <int DT, int K, int LP, int NV>
__global__ __launch_bounds__(LP == 64 ? kGradWaves * 64 : 256) void k_combine_grad(const char* g, const char* rows, const int32_t* __restrict__ inv,
                                                      const float* __restrict__ w, char* grad_rows, float* __restrict__ grad_w, int T,
                                                      int k, int R, uint32_t row_bytes) {
  using V = Row<DT>;
  constexpr int N = V::kVec, KK = K > 0 ? K : 1;
  constexpr bool kWhole = LP == 64;   // a workgroup has one token
  __shared__ float part[kWhole ? KK : 1][kGradWaves];
  Unit<LP> at(1);
  if constexpr (kWhole) at.t = blockIdx.x;
  if (at.t >= T) return;   // (kWhole: nobody)
  const uint32_t step = kWhole ? blockDim.x * (16 * NV) : LP * 16 * NV;
  const char* src = g + (size_t)at.t * row_bytes;
  const bool exact = row_bytes % step == 0;
  for (int j0 = 0; j0 < k; j0 += K > 0 ? k : 1) {
    int pos[KK];
    float wj[KK], dot[KK];
#pragma unroll
    for (int j = 0; j < KK; j++) {
      const bool there = K == 0 || j < k;
      pos[j] = there ? inv[(size_t)at.t * k + j0 + j] : -1;
      wj[j] = there && w != nullptr ? w[(size_t)at.t * k + j0 + j] : 1.f;
      dot[j] = 0.f;
    }
    for (uint32_t base = kWhole ? at.wave * (64 * 16 * NV) : 0; base < row_bytes; base += step) {
      const uint32_t start = base + at.lane * 16;
      u32x4 gv[NV], rv[KK][NV];
#pragma unroll
      for (int i = 0; i < NV; i++) gv[i] = load_once(src, start + i * (LP * 16), row_bytes);
      if (rows != nullptr) {
#pragma unroll
        for (int j = 0; j < KK; j++)
          if ((unsigned)pos[j] < (unsigned)R)
#pragma unroll
            for (int i = 0; i < NV; i++) rv[j][i] = load_once(rows + (size_t)pos[j] * row_bytes, start + i * (LP * 16), row_bytes);
      }
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const int from = exact ? 0 : counted<V::kBytes>(start + i * (LP * 16), row_bytes);
        float gf[N];
        V::unpack(gv[i], gf);
#pragma unroll
        for (int j = 0; j < KK; j++) {
          if ((unsigned)pos[j] >= (unsigned)R) continue;
          if (rows != nullptr) {
            float rf[N];
            V::unpack(rv[j][i], rf);
            if (exact) {
#pragma unroll
              for (int c = 0; c < N; c++) dot[j] = fmaf(gf[c], rf[c], dot[j]);
            } else {
#pragma unroll
              for (int c = 0; c < N; c++) dot[j] = c >= from ? fmaf(gf[c], rf[c], dot[j]) : dot[j];
            }
          }
          float o[N];
#pragma unroll
          for (int c = 0; c < N; c++) o[c] = wj[j] * gf[c];
          store_once(grad_rows + (size_t)pos[j] * row_bytes, start + i * (LP * 16), row_bytes, V::pack(o));
        }
      }
    }
    if (rows == nullptr) continue;
#pragma unroll
    for (int j = 0; j < KK; j++) {
      if constexpr (LP == 64) {
        dot[j] = wave_sum(dot[j]);
      } else {
#pragma unroll
        for (int off = LP / 2; off >= 1; off >>= 1) dot[j] += __shfl_xor(dot[j], off);
      }
      if constexpr (!kWhole) {
        if (at.lane == 0 && (K == 0 || j < k)) grad_w[(size_t)at.t * k + j0 + j] = dot[j];
      } else {
        if (at.lane == 0) part[j][at.wave] = dot[j];
      }
    }
    if constexpr (kWhole) {
      __syncthreads();
      const int j = threadIdx.x;
      if (j < KK && j0 + j < k) {
        float sum = part[j][0];
        for (int w = 1; w < (int)(blockDim.x >> 6); w++) sum += part[j][w];
        grad_w[(size_t)at.t * k + j0 + j] = sum;
      }
      if constexpr (K == 0) __syncthreads();   // part is written again
    }
  }
}

// The weights of a token are the softmax of its kept logits, so d w_i / d logit_j = w_i (delta_ij - w_j) among them:
// grad_logits[t][e] = sum over the slots j with expert e of w_j (g_j - sum_i g_i w_i).  A workgroup takes up to 1024 logits of whole tokens,
// adds the slots in LDS, a thread a token in the order of j, and writes them in one piece.  (Every thread going through its token's slots
// for 4 experts: 28.4 us for 65536 tokens of 256 experts, k = 8, so 20.7; 32768 of 64, k = 8 6.2 / 4.9; 32768 of 8, k = 2 2.6 / 3.0.  These
// find their inputs in the caches; where other work has run over them so takes 24.6, 5.7 and 4.6 to 5.1.)
constexpr int kGateLogits = 1024;
__global__ __launch_bounds__(256) void k_route_topk_grad(const int32_t* __restrict__ ids, const float* __restrict__ w,
                                                         const float* __restrict__ gw, int T, int E, int k, int tokens,
                                                         float* __restrict__ out) {
  __shared__ float tile[kGateLogits], wj[kGateLogits], gj[kGateLogits];   // (k <= E: no more slots than logits)
  __shared__ int32_t id[kGateLogits];
  const int t0 = blockIdx.x * tokens, n = min(tokens, T - t0), tid = threadIdx.x;
  const size_t slot0 = (size_t)t0 * k;
#pragma unroll
  for (int i = 0; i < kGateLogits / 256; i++) {
    const int s = i * 256 + tid;
    if (s < n * k) {
      id[s] = ids[slot0 + s];
      wj[s] = w[slot0 + s];
      gj[s] = gw[slot0 + s];
    }
    tile[s] = 0.f;
  }
  __syncthreads();
  for (int t = tid; t < n; t += 256) {
    float sum = 0.f;
    for (int j = 0; j < k; j++) sum = fmaf(gj[t * k + j], wj[t * k + j], sum);
    for (int j = 0; j < k; j++) {
      const int e = id[t * k + j];
      if ((unsigned)e < (unsigned)E) tile[t * E + e] += wj[t * k + j] * (gj[t * k + j] - sum);
    }
  }
  __syncthreads();
  float* dst = out + (size_t)t0 * E;
#pragma unroll
  for (int i = 0; i < kGateLogits / 256; i++) {
    const int s = i * 256 + tid;
    if (s < n * E) dst[s] = tile[s];
  }
}

namespace {

struct RowCall {
  int T, k, R;
  uint32_t row_bytes;
  hipStream_t st;
  size_t token_bytes() const { return (size_t)T * row_bytes; }
  size_t rows_bytes() const { return (size_t)R * row_bytes; }
  size_t pair_bytes() const { return (size_t)R * 4; }
};

// Lanes of a token, as many as a row has pieces.  us for 32768 tokens of 64 columns, k = 2, with 8 lanes / 64: combine 3.9 / 8.6, its gradient
// 5.9 / 11.6; of 256 columns with 32 / 64: 11.6 / 12.2, 16.7 / 18.3.
int lanes_of(const RowCall& c) { return c.row_bytes <= 8 * 16 ? 8 : c.row_bytes <= 32 * 16 ? 32 : 64; }

template <int LP, int NV>
dim3 row_grid(const RowCall& c, int* spans) {
  *spans = LP == 64 ? (int)((c.row_bytes + 64 * 16 * NV - 1) / (64 * 16 * NV)) : 1;
  const int64_t waves = LP == 64 ? (int64_t)c.T * *spans : ((int64_t)c.T * LP + 63) / 64;
  return dim3((unsigned)((waves + 3) / 4));
}

template <int LP, int NV>
hipError_t dispatch_as(const RowCall& c, const void* x, const int32_t* inv, void* rows) {
  int spans;
  const dim3 grid = row_grid<LP, NV>(c, &spans);
  hipLaunchKernelGGL((k_dispatch<LP, NV>), grid, dim3(256), 0, c.st, (const char*)x, inv, (char*)rows, c.T, c.k, c.R, c.row_bytes, spans);
  return hipGetLastError();
}
hipError_t launch_dispatch(const RowCall& c, const void* x, const int32_t* inv, void* rows) {
  switch (lanes_of(c)) {
    case 8: return dispatch_as<8, 1>(c, x, inv, rows);
    case 32: return dispatch_as<32, 1>(c, x, inv, rows);
    default: return dispatch_as<64, 4>(c, x, inv, rows);
  }
}

template <int DT, int K, int LP, int NV>
hipError_t combine_as(const RowCall& c, const void* rows, const int32_t* inv, const float* w, void* out) {
  int spans;
  const dim3 grid = row_grid<LP, NV>(c, &spans);
  hipLaunchKernelGGL((k_combine_rows<DT, K, LP, NV>), grid, dim3(256), 0, c.st, (const char*)rows, inv, w, (char*)out, c.T, c.k, c.R, c.row_bytes, spans);
  return hipGetLastError();
}
template <int DT, int K>
hipError_t combine_k(const RowCall& c, const void* rows, const int32_t* inv, const float* w, void* out) {
  switch (lanes_of(c)) {
    case 8: return combine_as<DT, K, 8, 1>(c, rows, inv, w, out);
    case 32: return combine_as<DT, K, 32, 1>(c, rows, inv, w, out);
    default: return combine_as<DT, K, 64, 2>(c, rows, inv, w, out);   // 1 or 4 pieces a lane are up to 5 % slower at one size or another
  }
}
// Slots whose rows are requested together: 1, 2, up to 4 or up to 8, whose two pieces a lane are 64 registers; more of them slot after slot
// (K == 0).  us so / slot after slot, 16384 tokens of 2048 columns: k = 1 22.6 / 23.8, 2 32.6 / 32.9, 3
// 43.5 / 44.8, 4 54.8 / 56.8, 5 67.0 / 68.6, 8 102 / 103; 48 tokens 2.5 / 2.7, 2.7 / 3.1, 2.6 / 3.2, 2.8 / 3.4, 3.3 / 3.8, 3.6 / 4.5.  Beyond 8: k = 9
// 116, 10 128, 16 196, 32 376 (5.8 to 5.9 TB/s); 48 tokens 4.9, 5.4, 7.6, 16.2, an index and a row of latency a slot.
template <int DT>
hipError_t combine_type(const RowCall& c, const void* rows, const int32_t* inv, const float* w, void* out) {
  if (c.k == 1) return combine_k<DT, 1>(c, rows, inv, w, out);
  if (c.k == 2) return combine_k<DT, 2>(c, rows, inv, w, out);
  if (c.k <= 4) return combine_k<DT, 4>(c, rows, inv, w, out);
  if (c.k <= 8) return combine_k<DT, 8>(c, rows, inv, w, out);
  return combine_k<DT, 0>(c, rows, inv, w, out);
}
hipError_t launch_combine_rows(int dtype, const RowCall& c, const void* rows, const int32_t* inv, const float* w, void* out) {
  switch (dtype) {
    case MOE_BF16: return combine_type<MOE_BF16>(c, rows, inv, w, out);
    case MOE_FP16: return combine_type<MOE_FP16>(c, rows, inv, w, out);
    default: return combine_type<MOE_FP32>(c, rows, inv, w, out);
  }
}

// A token has up to 8 wavefronts with a piece a lane each, two where that is too few, so that its pieces are requested together.  us with one
// wavefront a token and 1 / 2 / 4 pieces a lane, which takes longer rows in turns: 32768 tokens of 4096 columns, k = 2 284 / 287 / 268; so: 232.  With
// always four: 12000 of 300 15.2, so 10.7, of 1500, k = 1 20.8 / 22.1, of 2600, k = 3 90.9 / 82.3, of 2339 in fp32, k = 5 280 / 256; 2048 of 3584, k = 8
// 47.9 / 46.5.  Two pieces a lane from 2048 / 4096 / 8192 bytes a row: 12000 of 2600 91.5 / 92.3 / 82.3, 12000 of 2048, k = 4 80.9 / 76.8 / 76.2.
template <int DT, int K, int LP, int NV>
hipError_t combine_grad_as(const RowCall& c, const void* g, const void* rows, const int32_t* inv, const float* w, void* grad_rows, float* grad_w) {
  int waves = LP == 64 ? (int)((c.row_bytes + 1024 * NV - 1) / (1024 * NV)) : 4;
  if (waves > kGradWaves) waves = kGradWaves;
  const int64_t blocks = LP == 64 ? c.T : (((int64_t)c.T * LP + 63) / 64 + 3) / 4;
  hipLaunchKernelGGL((k_combine_grad<DT, K, LP, NV>), dim3((unsigned)blocks), dim3(waves * 64), 0, c.st, (const char*)g, (const char*)rows, inv, w,
                     (char*)grad_rows, grad_w, c.T, c.k, c.R, c.row_bytes);
  return hipGetLastError();
}
template <int DT, int K>
hipError_t combine_grad_k(const RowCall& c, const void* g, const void* rows, const int32_t* inv, const float* w, void* grad_rows, float* grad_w) {
  switch (lanes_of(c)) {
    case 8: return combine_grad_as<DT, K, 8, 1>(c, g, rows, inv, w, grad_rows, grad_w);
    case 32: return combine_grad_as<DT, K, 32, 1>(c, g, rows, inv, w, grad_rows, grad_w);
    default:
      if (c.row_bytes <= kGradWaves * 1024) return combine_grad_as<DT, K, 64, 1>(c, g, rows, inv, w, grad_rows, grad_w);
      return combine_grad_as<DT, K, 64, 2>(c, g, rows, inv, w, grad_rows, grad_w);
  }
}
// Slots as in the combine; the token's row is loaded once for those that go together, and again for each of the others, with two barriers.
// us so / slot after slot, 16384 tokens of 2048 columns: k = 1 37.0 / 37.3, 2 58.4 / 67.5, 3 86.6 / 105, 4 112 / 141, 5 138 / 176, 8 216 / 281; 48
// tokens 3.1 / 3.2, 3.4 / 4.1, 3.8 / 4.9, 3.7 / 5.6, 4.5 / 6.6, 4.5 / 8.7.  Beyond 8: k = 9 326, 10 354, 16 567, 32 1117 (3.9 TB/s, against 5.3 with 8);
// 48 tokens 9.7, 10.8, 16.9, 35.5.
template <int DT>
hipError_t combine_grad_type(const RowCall& c, const void* g, const void* rows, const int32_t* inv, const float* w, void* grad_rows, float* grad_w) {
  if (c.k == 1) return combine_grad_k<DT, 1>(c, g, rows, inv, w, grad_rows, grad_w);
  if (c.k == 2) return combine_grad_k<DT, 2>(c, g, rows, inv, w, grad_rows, grad_w);
  if (c.k <= 4) return combine_grad_k<DT, 4>(c, g, rows, inv, w, grad_rows, grad_w);
  if (c.k <= 8) return combine_grad_k<DT, 8>(c, g, rows, inv, w, grad_rows, grad_w);
  return combine_grad_k<DT, 0>(c, g, rows, inv, w, grad_rows, grad_w);
}

int n_chunks_of(int64_t R) { return (int)((R + kSortChunk - 1) / kSortChunk); }
// Where a chunk's workgroup has the counts of the others from.  us, it counts all pairs itself / counts by a launch of their own:
// 16384 pairs of 64 experts 5.4 / 6.8, 32768 6.5 / 7.2, 65536 8.7 / 7.1, of 8 experts 12.4 / 6.7; a launch also takes 2.6 us of the host.
constexpr int kSortOwnCounts = 32;
// It sums the counts of the chunks itself while they are few.  us of the scatter, itself / prefix sums by a launch of their own and the
// scatter: 256 chunks of 65 buckets 6.9 / -, 512 of 257 28 / 5 + 7, 1024 of 9 14.4 / 3.4 + 8.8.
constexpr int kSortOwnSums = 32768, kSortOwnSumChunks = 512;   // chunks x buckets, chunks

// Checks that the row operators share; *c is set where there is something to do.
int row_call(int32_t T, int32_t H, int32_t k, int32_t dtype, void* hip_stream, RowCall* c) {
  if (T < 0 || H <= 0 || k <= 0 || element_bytes(dtype) == 0) return MOE_ERR_INVALID_ARG;
  if (k > kMaxGateTopK || H < kMinRowColumns || H > kMaxRowColumns || (int64_t)T * k >= (1 << 24)) return MOE_ERR_UNSUPPORTED;
  if ((int64_t)T * H * element_bytes(dtype) >= (1ll << 35)) return MOE_ERR_UNSUPPORTED;   // threads of a launch: 32 bits
  c->T = T;
  c->k = k;
  c->R = T * k;
  c->row_bytes = (uint32_t)(H * element_bytes(dtype));
  c->st = (hipStream_t)hip_stream;
  return MOE_OK;
}

int sort_shape(int32_t T, int32_t E, int32_t k) {
  if (T < 0 || E <= 0 || k <= 0) return MOE_ERR_INVALID_ARG;
  if (E > kMaxExperts || k > kMaxGateTopK || (int64_t)T * k >= (1 << 24)) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}

int status_of(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" {

size_t moe_sort_workspace_bytes(int32_t T, int32_t E, int32_t k) {
  if (sort_shape(T, E, k) != MOE_OK) return 0;
  return ((size_t)n_chunks_of((int64_t)T * k) + 1) * (E + 1) * 4;
}

int moe_sort_tokens(const int32_t* topk_ids, int32_t T, int32_t E, int32_t k, int32_t* expert_offsets, int32_t* perm,
                    int32_t* inv_perm, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = sort_shape(T, E, k);
  if (rc != MOE_OK) return rc;
  hipStream_t st = (hipStream_t)hip_stream;
  if (!expert_offsets || !aligned16(expert_offsets)) return MOE_ERR_INVALID_ARG;
  const int R = T * k;
  if (R == 0) {
    hipLaunchKernelGGL(k_sort_none, dim3(1), dim3(256), 0, st, E, expert_offsets);
    return status_of(hipGetLastError());
  }
  if (!topk_ids || !perm || !inv_perm || !workspace) return MOE_ERR_INVALID_ARG;
  if (!aligned16(topk_ids) || !aligned16(perm) || !aligned16(inv_perm) || !aligned16(workspace)) return MOE_ERR_INVALID_ARG;
  const size_t need = moe_sort_workspace_bytes(T, E, k), pairs = (size_t)R * 4;
  if (workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
  if (!apart({{expert_offsets, (size_t)(E + 1) * 4}, {perm, pairs}, {inv_perm, pairs}, {workspace, need}}, {{topk_ids, pairs}})) return MOE_ERR_INVALID_ARG;
  int32_t* hist = (int32_t*)workspace;
  const int n_chunks = n_chunks_of(R);
  if (R <= kSortChunk) {
    auto kernel = R <= 64 ? k_sort_one<1> : R <= 256 ? k_sort_one<4> : k_sort_one<16>;
    hipLaunchKernelGGL(kernel, dim3(1), dim3(R <= 64 ? 64 : R <= 256 ? 256 : 1024), 0, st, topk_ids, R, E, expert_offsets, perm, inv_perm);
    return status_of(hipGetLastError());
  }
  if (n_chunks <= kSortOwnCounts) {
    hipLaunchKernelGGL(k_sort_scatter<true>, dim3(n_chunks), dim3(1024), 0, st, topk_ids, R, E, nullptr, n_chunks, nullptr, expert_offsets, perm, inv_perm);
    return status_of(hipGetLastError());
  }
  int32_t* total = n_chunks > kSortOwnSumChunks || n_chunks * (E + 1) > kSortOwnSums ? hist + (size_t)n_chunks * (E + 1) : nullptr;
  hipLaunchKernelGGL(k_sort_hist, dim3(n_chunks), dim3(1024), 0, st, topk_ids, R, E, hist);
  if (total) hipLaunchKernelGGL(k_sort_scan, dim3(E + 1), dim3(1024), 0, st, hist, n_chunks, E, total);
  hipLaunchKernelGGL(k_sort_scatter<false>, dim3(n_chunks), dim3(1024), 0, st, topk_ids, R, E, hist, n_chunks, total, expert_offsets, perm, inv_perm);
  return status_of(hipGetLastError());
}

int moe_dispatch(const void* x, const int32_t* inv_perm, int32_t T, int32_t H, int32_t k, int32_t dtype, void* rows,
                 void* hip_stream) {
  RowCall c;
  const int rc = row_call(T, H, k, dtype, hip_stream, &c);
  if (rc != MOE_OK) return rc;
  if (T == 0) return MOE_OK;
  if (!x || !inv_perm || !rows || !aligned16(x) || !aligned16(inv_perm) || !aligned16(rows)) return MOE_ERR_INVALID_ARG;
  if (!apart({{rows, c.rows_bytes()}}, {{x, c.token_bytes()}, {inv_perm, c.pair_bytes()}})) return MOE_ERR_INVALID_ARG;
  return status_of(launch_dispatch(c, x, inv_perm, rows));
}

int moe_combine(const void* rows, const int32_t* inv_perm, const float* topk_weights, int32_t T, int32_t H, int32_t k,
                int32_t dtype, void* out, void* hip_stream) {
  RowCall c;
  const int rc = row_call(T, H, k, dtype, hip_stream, &c);
  if (rc != MOE_OK) return rc;
  if (T == 0) return MOE_OK;
  if (!rows || !inv_perm || !out || !aligned16(rows) || !aligned16(inv_perm) || !aligned16(out) || !aligned16(topk_weights))
    return MOE_ERR_INVALID_ARG;
  if (!apart({{out, c.token_bytes()}}, {{rows, c.rows_bytes()}, {inv_perm, c.pair_bytes()}, {topk_weights, c.pair_bytes()}})) return MOE_ERR_INVALID_ARG;
  return status_of(launch_combine_rows(dtype, c, rows, inv_perm, topk_weights, out));
}

int moe_dispatch_backward(const void* grad_rows, const int32_t* inv_perm, int32_t T, int32_t H, int32_t k, int32_t dtype,
                          void* grad_x, void* hip_stream) {
  return moe_combine(grad_rows, inv_perm, nullptr, T, H, k, dtype, grad_x, hip_stream);
}

int moe_combine_backward(const void* grad_out, const void* rows, const int32_t* inv_perm, const float* topk_weights, int32_t T,
                         int32_t H, int32_t k, int32_t dtype, void* grad_rows, float* grad_weights, void* hip_stream) {
  RowCall c;
  const int rc = row_call(T, H, k, dtype, hip_stream, &c);
  if (rc != MOE_OK) return rc;
  if (T == 0) return MOE_OK;
  if (!grad_out || !inv_perm || !grad_rows || (grad_weights && !rows)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(grad_out) || !aligned16(rows) || !aligned16(inv_perm) || !aligned16(topk_weights) || !aligned16(grad_rows) ||
      !aligned16(grad_weights))
    return MOE_ERR_INVALID_ARG;
  if (!apart({{grad_rows, c.rows_bytes()}, {grad_weights, c.pair_bytes()}},
             {{grad_out, c.token_bytes()}, {rows, c.rows_bytes()}, {inv_perm, c.pair_bytes()}, {topk_weights, c.pair_bytes()}}))
    return MOE_ERR_INVALID_ARG;
  if (!grad_weights) rows = nullptr;
  switch (dtype) {
    case MOE_BF16: return status_of(combine_grad_type<MOE_BF16>(c, grad_out, rows, inv_perm, topk_weights, grad_rows, grad_weights));
    case MOE_FP16: return status_of(combine_grad_type<MOE_FP16>(c, grad_out, rows, inv_perm, topk_weights, grad_rows, grad_weights));
    default: return status_of(combine_grad_type<MOE_FP32>(c, grad_out, rows, inv_perm, topk_weights, grad_rows, grad_weights));
  }
}

int moe_route_topk_backward(const int32_t* topk_ids, const float* topk_weights, const float* grad_weights, int32_t T, int32_t E,
                            int32_t k, float* grad_logits, void* hip_stream) {
  if (T < 0 || E <= 0 || k <= 0 || k > E) return MOE_ERR_INVALID_ARG;
  if (E > kMaxExperts || k > kMaxGateTopK || (int64_t)T * k >= (1 << 24)) return MOE_ERR_UNSUPPORTED;
  if (T == 0) return MOE_OK;
  if (!topk_ids || !topk_weights || !grad_weights || !grad_logits) return MOE_ERR_INVALID_ARG;
  if (!aligned16(topk_ids) || !aligned16(topk_weights) || !aligned16(grad_weights) || !aligned16(grad_logits)) return MOE_ERR_INVALID_ARG;
  const size_t pairs = (size_t)T * k * 4;
  if (!apart({{grad_logits, (size_t)T * E * 4}}, {{topk_ids, pairs}, {topk_weights, pairs}, {grad_weights, pairs}})) return MOE_ERR_INVALID_ARG;
  const int tokens = kGateLogits / E;
  hipLaunchKernelGGL(k_route_topk_grad, dim3((unsigned)((T + tokens - 1) / tokens)), dim3(256), 0, (hipStream_t)hip_stream, topk_ids, topk_weights,
                     grad_weights, T, E, k, tokens, grad_logits);
  return status_of(hipGetLastError());
}

}  // extern "C"
