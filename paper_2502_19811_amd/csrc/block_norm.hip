// The norms on either side of the block, with the residual stream: sum and norm in front of it, norm, gate and residual sum
// behind it, and their gradients.
//
// A row stays in registers between its loads and its stores: one wavefront or a workgroup of up to MW hold it, NV pieces of 16 bytes a
// lane, so that every input is read once and every output written once.  Sums over a row are fp32, in a fixed order: lanes by DPP, wavefronts
// through LDS.
//
// A "layer" norm is as good where a row's mean is large against its deviation: m, the sum over the row divided by H, is off by a few roundings
// of the mean, so the differences d = v - m, which lose next to nothing, are summed along with their squares, and what they come to
// corrects both (the corrected two-pass sums of Chan, Golub and LeVeque, 1983): v - mean = d - S(d) / H, H var = S(d d) - S(d)^2 / H.  The
// correction goes into the constant of the operation that makes n from d.  A row of one value has d = 0.  us without / with it, 8192 rows of
// 4096 columns: before 44.2 / 44.7, its gradient 68.6 / 69.8, behind with a token's gate 34.7 / 35.5, its gradient 44.4 / 46.9 (RMS: as it was).
#include "row_vector.h"

// Fused operations are written out, and no others made: a result does not depend on which variant computes it.
#pragma clang fp contract(off)

namespace moe {

constexpr int kMinNormColumns = 8, kMaxNormColumns = 16384;

struct NormParams {
  const char* residual;   // before: the stream; after: the stream or nullptr
  const char* branch;     // before: what is added to the stream or nullptr; after: the block's output
  const char* gamma;
  const char* beta;       // or nullptr
  const char* gate;
  char* sum;              // before: the new stream or nullptr
  char* out;
  int32_t gate_kind, layer, T;
  int32_t in_place;       // an output lies in the place of an input
  uint32_t row_bytes;
  float scale, eps, h, inv_h;
};

struct NormColumnParams {
  const float* part_a;
  const float* part_b;    // or nullptr
  const char* gamma;
  const char* beta;       // or nullptr
  const char* gate;       // a channel gate, or nullptr
  float* grad_gamma;      // each or nullptr
  float* grad_beta;
  float* grad_gate;
  int32_t groups, H;      // rows of part_a and part_b, columns
};

// What becomes of a column's sums.  Without rows (groups == 0) they are 0, whatever the factors are.
template <int DT>
__device__ __forceinline__ void finish_column(const NormColumnParams& p, int col, float sa, float sb) {
  auto value = [&](const char* v) -> float {
    if constexpr (DT == MOE_BF16) return __uint_as_float((uint32_t)((const uint16_t*)v)[col] << 16);
    else if constexpr (DT == MOE_FP16) return (float)((const _Float16*)v)[col];
    else return ((const float*)v)[col];
  };
  const bool rows = p.groups > 0;
  const float gate = p.gate != nullptr && rows ? value(p.gate) : 1.f;
  if (p.grad_gamma != nullptr) p.grad_gamma[col] = sa * gate;
  if (p.grad_beta != nullptr) p.grad_beta[col] = sb * gate;
  if (p.grad_gate != nullptr) p.grad_gate[col] = rows ? fmaf(value(p.gamma), sa, p.beta != nullptr ? value(p.beta) * sb : 0.f) : 0.f;
}

template <int N>
__device__ __forceinline__ void store_sums(float* to, const float (&v)[N]) {
  typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
  for (int c = 0; c < N; c += 4) *(f32x4_any*)(to + c) = f32x4_any{v[c], v[c + 1], v[c + 2], v[c + 3]};
}
// The same for the columns of a piece.
template <int DT, int N>
__device__ __forceinline__ void finish_piece(const NormColumnParams& p, uint32_t start, uint32_t row_bytes, float (&sa)[N], float (&sb)[N]) {
  using V = Row<DT>;
  const int col = (int)(piece_at(start, row_bytes) / V::kBytes);
  float gamma[N], beta[N], gate[N], o[N];
  V::unpack(load_piece(p.gamma, start, row_bytes), gamma);
  if (p.beta != nullptr) V::unpack(load_piece(p.beta, start, row_bytes), beta);
  if (p.gate != nullptr) V::unpack(load_piece(p.gate, start, row_bytes), gate);
  if (p.grad_gate != nullptr) {
#pragma unroll
    for (int c = 0; c < N; c++) o[c] = fmaf(gamma[c], sa[c], p.beta != nullptr ? beta[c] * sb[c] : 0.f);
    store_sums(p.grad_gate + col, o);
  }
#pragma unroll
  for (int c = 0; c < N; c++) {
    sa[c] *= p.gate != nullptr ? gate[c] : 1.f;
    sb[c] *= p.gate != nullptr ? gate[c] : 1.f;
  }
  if (p.grad_gamma != nullptr) store_sums(p.grad_gamma + col, sa);
  if (p.grad_beta != nullptr) store_sums(p.grad_beta + col, sb);
}

struct NormGradParams {
  const char* v;          // the rows that were normed
  const char* g;          // gradient of the outputs
  const char* gamma;
  const char* beta;       // after: or nullptr
  const char* gate;
  const char* more;       // before: gradient that the stream has by itself, or nullptr
  char* grad_v;
  char* grad_other;       // before: scale * grad_v, or nullptr; after: gradient of a full gate, or nullptr
  float* grad_token_gate; // after: gradient of a token gate, or nullptr
  float* part_a;          // [workgroups][H] sums over the rows of a workgroup, or nullptr
  float* part_b;
  int32_t gate_kind, layer, T, H, groups;
  int32_t in_place;       // an output lies in the place of an input
  uint32_t row_bytes;
  float scale, eps, h, inv_h;
  NormColumnParams columns;   // one workgroup: it finishes its sums itself
};

// Workgroups: MW == 1 four wavefronts with a row each, otherwise a row for up to MW wavefronts, as many as the launch has.
template <int MW> constexpr int threads_of() { return MW == 1 ? 256 : MW * 64; }
template <int MW> __device__ __forceinline__ int row_waves() { return MW == 1 ? 1 : (int)(blockDim.x >> 6); }

// What the wavefronts of a row tell each other: four places, each for up to 4 sums, which take turns -- a wavefront may write the next
// sums while another still reads the last ones.  The places of wavefronts that the workgroup does not have hold zeros.
constexpr int kRowSums = 4;
template <int MW> struct RowSums { float part[4][kRowSums][MW]; };
template <int MW>
__device__ __forceinline__ void clear_absent(RowSums<MW>& sums) {
  if constexpr (MW > 1) {
    const int w = threadIdx.x % MW, at = threadIdx.x / MW;
    if (w >= row_waves<MW>() && at < 4 * kRowSums) (&sums.part[0][0][0])[at * MW + w] = 0.f;   // (MW <= 8: 2 wavefronts at least, 16: 9)
  }
}
// The sum of squares of v - mean, from that of d = v - m, where m is off from the mean by mean_d = sum_d / H.
__device__ __forceinline__ float corrected_squares(float sum_dd, float sum_d, float mean_d) {
  const float s = fmaf(-sum_d, mean_d, sum_dd);
  return s < 0.f ? 0.f : s;   // (a sum that is no number stays one)
}

// Sums over the wavefronts of a row, in every lane of them.
// ragged: the last pieces of a row share bytes, perhaps across two wavefronts, and an output lies in an input's place: what was
// requested has to be there before any wavefront goes on to its stores.
template <int MW, int N>
__device__ __forceinline__ void row_sums(RowSums<MW>& sums, float (&v)[N], int place, bool ragged) {
  if (ragged) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; i++) v[i] = wave_sum(v[i]);
  if constexpr (MW > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
      for (int i = 0; i < N; i++) sums.part[place][i][wave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; i++) {
      float s = 0.f;
#pragma unroll
      for (int w = 0; w < MW; w += 4) s += (sums.part[place][i][w] + sums.part[place][i][w + 1]) + (sums.part[place][i][w + 2] + sums.part[place][i][w + 3]);
      v[i] = s;
    }
  }
}

// A lane's pieces of a row.  EXACT: the row has as many as its wavefronts' lanes have places, one for everybody.  Otherwise the last
// ones may lie behind its end, for some wavefronts: whether a wavefront has any of a piece, and all of it, is the same in its lanes, and
// what is not there is neither loaded nor computed (8192 rows of 4104 columns, behind the block: 49 us with all of them, 41 without).
// The launch takes no more wavefronts than it needs, so that all of them have any of their first pieces, and with NV > 1 all of the
// first half of them.
template <int DT, int MW, int NV, bool EXACT>
struct Pieces {
  static constexpr int N = Row<DT>::kVec;
  uint32_t at[NV], first, step, row_bytes;
  __device__ __forceinline__ Pieces(int wave, int lane, uint32_t bytes)
      : first(MW == 1 ? 0u : (uint32_t)wave * 1024), step((uint32_t)row_waves<MW>() * 1024), row_bytes(bytes) {
#pragma unroll
    for (int i = 0; i < NV; i++) at[i] = i * step + first + lane * 16;
  }
  __device__ __forceinline__ bool any(int i) const { return EXACT || NV == 1 || i < NV / 2 || (MW == 1 && NV <= 2) || i * step + first < row_bytes; }
  __device__ __forceinline__ bool all(int i) const { return EXACT || i < NV / 2 || i * step + first + 1024 <= row_bytes; }
  __device__ __forceinline__ void store(char* row, int i, const u32x4& v) const {
    if constexpr (EXACT) *(u32x4*)(row + at[i]) = v;
    else store_piece(row, at[i], row_bytes, v);
  }
  __device__ __forceinline__ void store_rarely_read(char* row, int i, const u32x4& v) const {
    if constexpr (EXACT) __builtin_nontemporal_store(v, (u32x4*)(row + at[i]));
    else store_once(row, at[i], row_bytes, v);
  }
  // body(piece) for the pieces that are there
  template <typename F>
  __device__ __forceinline__ void each(F body) const {
#pragma unroll
    for (int i = 0; i < NV; i++)
      if (any(i)) body(i);
  }
  // body(piece, column, counts) for their elements; counts is false for those that another lane has, too
  template <typename F>
  __device__ __forceinline__ void each_element(F body) const {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if (all(i)) {
#pragma unroll
        for (int c = 0; c < N; c++) body(i, c, true);
      } else if (any(i)) {
        const int from = counted<Row<DT>::kBytes>(at[i], row_bytes);
#pragma unroll
        for (int c = 0; c < N; c++) body(i, c, c >= from);
      }
    }
  }
};

// n = d * r - mean_d * r (RMS: d = v, mean_d = 0), one fused operation an element whatever the norm: at 16 lanes a cycle and SIMD an operation
// on every element of 16384 x 4096 takes 1.7 us, so the gradients, which read three rows, have room for about 30.
template <int DT, int MW, int NV, bool AFTER, bool EXACT>
__global__ __launch_bounds__(threads_of<MW>()) void k_norm(NormParams p) {
  using V = Row<DT>;
  constexpr int N = V::kVec;
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int t = MW == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  if (t >= p.T) return;   // (MW > 1: the whole workgroup or nobody)
  __shared__ RowSums<MW> sums;
  clear_absent(sums);
  const size_t row = (size_t)t * p.row_bytes;
  const bool ragged = !EXACT && p.in_place && p.row_bytes % 16 != 0;
  const Pieces<DT, MW, NV, EXACT> mine(wave, lane, p.row_bytes);
  u32x4 rv[NV], bv[NV], gv[NV], hv[NV];
  if (!AFTER || p.residual != nullptr)
    mine.each([&](int i) { rv[i] = load_once(p.residual + row, mine.at[i], p.row_bytes); });
  if (AFTER || p.branch != nullptr)
    mine.each([&](int i) { bv[i] = load_once(p.branch + row, mine.at[i], p.row_bytes); });
  float scale = p.scale;
  const bool gated = AFTER && (p.gate_kind == MOE_GATE_CHANNEL || p.gate_kind == MOE_GATE_FULL);
  if constexpr (AFTER) {
    if (gated) {
      const char* gate = p.gate + (p.gate_kind == MOE_GATE_FULL ? row : 0);
      mine.each([&](int i) { hv[i] = load_piece(gate, mine.at[i], p.row_bytes); });
    } else if (p.gate_kind == MOE_GATE_TOKEN) {
      scale *= ((const float*)p.gate)[t];
    }
  }
  mine.each([&](int i) { gv[i] = load_piece(p.gamma, mine.at[i], p.row_bytes); });
  float v[NV][N];
#pragma unroll
  for (int i = 0; i < NV; i++) {
    if (!mine.any(i)) continue;
    if constexpr (AFTER) {
      V::unpack(bv[i], v[i]);
    } else {
      V::unpack(rv[i], v[i]);
      if (p.branch != nullptr) {
        float b[N];
        V::unpack(bv[i], b);
#pragma unroll
        for (int c = 0; c < N; c++) v[i][c] = fmaf(p.scale, b[c], v[i][c]);
      }
    }
  }
  float squares, m = 0.f, mean_d = 0.f;
  if (p.layer) {
    float s[1] = {0.f}, d[2] = {0.f, 0.f};   // d: sums of the squares, of the differences
    mine.each_element([&](int i, int c, bool counts) { s[0] += counts ? v[i][c] : 0.f; });
    row_sums<MW>(sums, s, 0, false);
    m = s[0] / p.h;
    mine.each_element([&](int i, int c, bool counts) {
      const float one = counts ? v[i][c] - m : 0.f;
      d[0] = fmaf(one, one, d[0]);
      d[1] += one;
    });
    row_sums<MW>(sums, d, 1, ragged);
    mean_d = d[1] * p.inv_h;
    squares = corrected_squares(d[0], d[1], mean_d);
  } else {
    float s[1] = {0.f};
    mine.each_element([&](int i, int c, bool counts) {
      const float one = counts ? v[i][c] : 0.f;
      s[0] = fmaf(one, one, s[0]);
    });
    row_sums<MW>(sums, s, 1, ragged);
    squares = s[0];
  }
  const float r = 1.f / sqrtf(fmaf(squares, p.inv_h, p.eps)), minus = p.layer ? -mean_d * r : 0.f;
  if constexpr (!AFTER)
    if (p.sum != nullptr) mine.each([&](int i) { mine.store_rarely_read(p.sum + row, i, V::pack(v[i])); });
#pragma unroll
  for (int i = 0; i < NV; i++) {
    if (!mine.any(i)) continue;
    float o[N], f[N];
    V::unpack(gv[i], f);
#pragma unroll
    for (int c = 0; c < N; c++) o[c] = fmaf(v[i][c] - m, r, minus) * f[c];
    if (p.beta != nullptr) {
      V::unpack(load_piece(p.beta, mine.at[i], p.row_bytes), f);
#pragma unroll
      for (int c = 0; c < N; c++) o[c] += f[c];
    }
    if constexpr (AFTER) {
      if (gated) {
        V::unpack(hv[i], f);
#pragma unroll
        for (int c = 0; c < N; c++) o[c] *= f[c];
      }
#pragma unroll
      for (int c = 0; c < N; c++) f[c] = 0.f;
      if (p.residual != nullptr) V::unpack(rv[i], f);
#pragma unroll
      for (int c = 0; c < N; c++) o[c] = fmaf(scale, o[c], f[c]);
    }
    mine.store(p.out + row, i, V::pack(o));
  }
}

// Gradients.  With n the normed row, e the gradient of n and r the reciprocal deviation, the gradient of the row is
//   r * (e - mean(e) - n * mean(e * n))           (without the mean of e where no mean was taken off),
// which is c1 * (e - mean(e)) + c2 * d + c0 with four numbers a row, d = v - m as above.  The scale and a token's gate are factors of c1, c2, c0.
// A group, the wavefronts that hold a row, takes rows group, group + groups, ... and keeps, in registers, its columns' sums over them: A of
// f * n and B of f, f the gradient of gamma * n + beta but for the scale and a channel gate, which are factors of the sums; they go
// to part_a and part_b, a row for each workgroup, which k_norm_columns adds up in a fixed order.  The next row is requested before the present one
// is summed up (PRE), which the largest rows have no registers for.  Its loads are waited for by counting what was requested after them,
// which takes that nothing is conditional: ALL says that the row is exact and that every optional row is given.
// Rows of more than eight wavefronts leave a lane 128 registers, fewer than its sums, gamma and rows are in most variants for more than 8192
// columns: those keep up to 248 bytes a lane in scratch memory, with four pieces up to 392.  us for 4096 rows of 8192 / 12288 / 16384 columns, without the sums of
// columns: bf16 before 59 / 97 / 128 (5.7, 5.2, 5.3 TB/s), behind with a channel gate 35 / 64 / 80, with a full one 61 / 102 / 136, that with mean and
// bias 63 / 177 / 230 (5.3, 2.8, 2.9 TB/s); fp32 before 123 / 220 / 346, channel 77 / 111 / 157, full 122 / 219 / 327, with mean and bias 134 / 359 / 459.
enum { GRAD_BEFORE = 0, GRAD_AFTER = 1, GRAD_AFTER_TOKEN = 2, GRAD_AFTER_FULL = 3 };   // AFTER: no gate or a channel gate
template <int DT, int MW, int NV, int MODE, bool WITH_B, bool PRE, bool ALL>
__global__ __launch_bounds__(threads_of<MW>()) void k_norm_grad(NormGradParams p) {
  using V = Row<DT>;
  constexpr int N = V::kVec;
  constexpr bool kToken = MODE == GRAD_AFTER_TOKEN, kFull = MODE == GRAD_AFTER_FULL;
  const int wave = uniform((int)(threadIdx.x >> 6)), lane = threadIdx.x & 63;
  const int group = MW == 1 ? blockIdx.x * 4 + wave : blockIdx.x;
  __shared__ RowSums<MW> sums;
  clear_absent(sums);
  const bool ragged = !ALL && p.in_place && p.row_bytes % 16 != 0;
  const Pieces<DT, MW, NV, ALL> mine(wave, lane, p.row_bytes);
  float gamma[NV][N];   // with a channel gate multiplied in
  u32x4 beta[NV];
  const bool has_beta = (kToken || kFull) && p.beta != nullptr;
#pragma unroll
  for (int i = 0; i < NV; i++) {
    if (!mine.any(i)) continue;
    V::unpack(load_piece(p.gamma, mine.at[i], p.row_bytes), gamma[i]);
    if constexpr (MODE == GRAD_AFTER)
      if (p.gate_kind == MOE_GATE_CHANNEL) {
        float h[N];
        V::unpack(load_piece(p.gate, mine.at[i], p.row_bytes), h);
#pragma unroll
        for (int c = 0; c < N; c++) gamma[i][c] *= h[c];
      }
    if (has_beta) beta[i] = load_piece(p.beta, mine.at[i], p.row_bytes);
  }
  float acc_a[NV][N], acc_b[WITH_B ? NV : 1][N];
#pragma unroll
  for (int i = 0; i < NV; i++)
#pragma unroll
    for (int c = 0; c < N; c++) {
      acc_a[i][c] = 0.f;
      if constexpr (WITH_B) acc_b[i][c] = 0.f;
    }
  // A third row is read: the gate, or the stream's own gradient, which is needed last.  Requested with the others, a row ahead (LATE: when
  // its turn begins), it takes registers and saves a wait where waits are for everything: 10000 rows of 4104 columns 109 us / 80 a row
  // ahead, 16384 of 4096 121 / 126.
  constexpr bool kThird = kFull || MODE == GRAD_BEFORE, kLate = MODE == GRAD_BEFORE && ALL;
  const char* third = kFull ? p.gate : p.more;
  const bool has_third = kThird && (ALL || third != nullptr);
  u32x4 vv[NV], gg[NV], hh[kThird ? NV : 1];
  auto request = [&](int t) {
    const size_t row = (size_t)t * p.row_bytes;
    mine.each([&](int i) { vv[i] = load_once(p.v + row, mine.at[i], p.row_bytes); });
    mine.each([&](int i) { gg[i] = load_once(p.g + row, mine.at[i], p.row_bytes); });
    if constexpr (kThird && !kLate)
      if (has_third) mine.each([&](int i) { hh[i] = load_once(third + row, mine.at[i], p.row_bytes); });
  };
  int flip = 0;
  const int begin = group < p.groups ? group : p.T;   // (a wavefront beyond the groups has no rows)
  if constexpr (PRE)
    if (begin < p.T) request(begin);
  for (int t = begin; t < p.T; t += p.groups) {
    const size_t row = (size_t)t * p.row_bytes;
    if constexpr (!PRE) request(t);
    u32x4 more[MODE == GRAD_BEFORE ? NV : 1];
    if constexpr (kLate) mine.each([&](int i) { more[i] = load_once(third + row, mine.at[i], p.row_bytes); });
    float v[NV][N], f[NV][N], g[kFull ? NV : 1][N];   // f: gradient of gamma * n + beta, but for the factors said above
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if (!mine.any(i)) continue;
      V::unpack(vv[i], v[i]);
      V::unpack(gg[i], f[i]);
      if constexpr (MODE == GRAD_BEFORE && !kLate) more[i] = hh[i];
      if constexpr (kFull) {
        float h[N];
        V::unpack(hh[i], h);
#pragma unroll
        for (int c = 0; c < N; c++) {
          g[i][c] = f[i][c];
          f[i][c] *= h[c];
        }
      }
    }
    if constexpr (PRE)
      if (t + p.groups < p.T) request(t + p.groups);
    const float gate_t = kToken ? ((const float*)p.gate)[t] : 1.f;
    // sums of the squares, of e * d, with a token's gate of f * beta, with a mean of d
    constexpr int kBeta = 2, kSums = kToken ? 3 : 2;
    float squares, sum_ed, sum_b = 0.f, mean = 0.f, mean_e = 0.f, mean_d = 0.f;
    auto sum_of_beta = [&](float& sum) {
      if constexpr (kToken)
        if (has_beta) {
          float b[NV][N];
#pragma unroll
          for (int i = 0; i < NV; i++) V::unpack(beta[i], b[i]);
          mine.each_element([&](int i, int c, bool counts) { sum = fmaf(counts ? f[i][c] : 0.f, counts ? b[i][c] : 0.f, sum); });
        }
    };
    if (p.layer) {
      float m[2] = {0.f, 0.f}, s[kSums + 1] = {};
      mine.each_element([&](int i, int c, bool counts) {
        m[0] += counts ? v[i][c] : 0.f;
        m[1] = fmaf(counts ? f[i][c] : 0.f, counts ? gamma[i][c] : 0.f, m[1]);
      });
      row_sums<MW>(sums, m, 2 + flip, false);
      mean = m[0] / p.h;
      mean_e = m[1] / p.h;
      mine.each_element([&](int i, int c, bool counts) {
        const float d = counts ? v[i][c] - mean : 0.f;
        s[0] = fmaf(d, d, s[0]);
        s[1] = fmaf(counts ? f[i][c] * gamma[i][c] : 0.f, d, s[1]);
        s[kSums] += d;
      });
      if constexpr (kToken) sum_of_beta(s[kBeta]);
      row_sums<MW>(sums, s, flip, ragged);
      mean_d = s[kSums] * p.inv_h;
      squares = corrected_squares(s[0], s[kSums], mean_d);
      sum_ed = fmaf(-mean_d, m[1], s[1]);
      if constexpr (kToken) sum_b = s[kBeta];
    } else {
      float s[kSums] = {};
      mine.each_element([&](int i, int c, bool counts) {
        const float d = counts ? v[i][c] : 0.f;
        s[0] = fmaf(d, d, s[0]);
        s[1] = fmaf(counts ? f[i][c] * gamma[i][c] : 0.f, d, s[1]);
      });
      if constexpr (kToken) sum_of_beta(s[kBeta]);
      row_sums<MW>(sums, s, flip, ragged);
      squares = s[0];
      sum_ed = s[1];
      if constexpr (kToken) sum_b = s[kBeta];
    }
    flip ^= 1;
    const float r = 1.f / sqrtf(fmaf(squares, p.inv_h, p.eps)), minus = p.layer ? -mean_d * r : 0.f;
    const float en = sum_ed * r;   // sum of e * n
    if constexpr (kToken)
      if (p.grad_token_gate != nullptr && lane == 0 && (MW == 1 || wave == 0)) p.grad_token_gate[t] = p.scale * (en + sum_b);
    const float c1 = MODE == GRAD_BEFORE ? r : r * p.scale * gate_t;
    const float c2 = -c1 * r * (en * p.inv_h);
    const float c0 = p.layer ? -c2 * mean_d : 0.f, minus_e = -mean_e;
    const float rt = kToken ? r * gate_t : r, minus_t = kToken ? minus * gate_t : minus;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if (!mine.any(i)) continue;
      float o[N], x[N];
      if constexpr (MODE == GRAD_BEFORE) {
#pragma unroll
        for (int c = 0; c < N; c++) x[c] = 0.f;
        if (has_third) V::unpack(more[i], x);
      }
#pragma unroll
      for (int c = 0; c < N; c++) {
        const float d = v[i][c] - mean;
        acc_a[i][c] = fmaf(f[i][c], fmaf(d, rt, minus_t), acc_a[i][c]);
        if constexpr (WITH_B) acc_b[i][c] = fmaf(f[i][c], gate_t, acc_b[i][c]);
        o[c] = fmaf(c1, fmaf(f[i][c], gamma[i][c], minus_e), fmaf(c2, d, c0));
        if constexpr (MODE == GRAD_BEFORE) o[c] += x[c];
      }
      mine.store(p.grad_v + row, i, V::pack(o));
      if constexpr (MODE == GRAD_BEFORE) {
        if (ALL || p.grad_other != nullptr) {
#pragma unroll
          for (int c = 0; c < N; c++) o[c] *= p.scale;
          mine.store(p.grad_other + row, i, V::pack(o));
        }
      }
      if constexpr (kFull) {
        if (ALL || p.grad_other != nullptr) {
#pragma unroll
          for (int c = 0; c < N; c++) x[c] = 0.f;
          if (has_beta) V::unpack(beta[i], x);
#pragma unroll
          for (int c = 0; c < N; c++) o[c] = p.scale * g[i][c] * fmaf(fmaf(v[i][c] - mean, r, minus), gamma[i][c], x[c]);
          mine.store(p.grad_other + row, i, V::pack(o));
        }
      }
    }
  }
  if (p.part_a == nullptr) return;
  const float scale = MODE == GRAD_BEFORE ? 1.f : p.scale;
  if constexpr (MW > 1) {
#pragma unroll
    for (int i = 0; i < NV; i++) {
      if (mine.at[i] >= p.row_bytes) continue;
      const int col = (int)(piece_at(mine.at[i], p.row_bytes) / V::kBytes);
      float sa[N], sb[N];
#pragma unroll
      for (int c = 0; c < N; c++) {
        sa[c] = acc_a[i][c] * scale;
        sb[c] = WITH_B ? acc_b[WITH_B ? i : 0][c] * scale : 0.f;
      }
      if (gridDim.x == 1) {
        finish_piece<DT>(p.columns, mine.at[i], p.row_bytes, sa, sb);
      } else {
        store_sums(p.part_a + (size_t)blockIdx.x * p.H + col, sa);
        if constexpr (WITH_B) store_sums(p.part_b + (size_t)blockIdx.x * p.H + col, sb);
      }
    }
  } else {
    // the four groups of the workgroup meet in LDS, a quarter of the columns a wavefront
    __shared__ float all[4][NV * N][64];
    constexpr int kMine = NV * N / 4;
    float a[kMine], b[kMine];
    auto meet = [&](float (&sum)[kMine], auto& acc) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int c = 0; c < N; c++) all[wave][i * N + c][lane] = acc[i][c];
      __syncthreads();
#pragma unroll
      for (int q = 0; q < kMine; q++) {
        const int ic = wave * kMine + q;
        sum[q] = ((all[0][ic][lane] + all[1][ic][lane]) + (all[2][ic][lane] + all[3][ic][lane])) * scale;
      }
    };
    meet(a, acc_a);
    if constexpr (WITH_B) meet(b, acc_b);
#pragma unroll
    for (int q = 0; q < kMine; q++) {
      const int ic = wave * kMine + q;
      const uint32_t start = (uint32_t)(ic / N * 64 + lane) * 16;
      if (start >= p.row_bytes) continue;
      const int col = (int)(piece_at(start, p.row_bytes) / V::kBytes) + ic % N;
      if (gridDim.x == 1) {
        finish_column<DT>(p.columns, col, a[q], WITH_B ? b[q] : 0.f);
      } else {
        p.part_a[(size_t)blockIdx.x * p.H + col] = a[q];
        if constexpr (WITH_B) p.part_b[(size_t)blockIdx.x * p.H + col] = b[q];
      }
    }
  }
}

// Column sums over the groups: a workgroup takes 32 columns, 32 threads each, which go down the groups in turn and meet in LDS.
template <int DT>
__global__ __launch_bounds__(1024) void k_norm_columns(NormColumnParams p) {
  __shared__ float a[32][33], b[32][33];
  const int c = threadIdx.x & 31, part = threadIdx.x >> 5;
  const int col = blockIdx.x * 32 + c;
  float sa = 0.f, sb = 0.f;
  if (col < p.H) {
#pragma unroll 8
    for (int g = part; g < p.groups; g += 32) sa += p.part_a[(size_t)g * p.H + col];
    if (p.part_b != nullptr)
#pragma unroll 8
      for (int g = part; g < p.groups; g += 32) sb += p.part_b[(size_t)g * p.H + col];
  }
  a[part][c] = sa;
  b[part][c] = sb;
  __syncthreads();
  if (part != 0 || col >= p.H) return;
#pragma unroll
  for (int i = 1; i < 32; i++) {
    sa += a[i][c];
    sb += b[i][c];
  }
  finish_column<DT>(p, col, sa, sb);
}

namespace {

uint32_t pieces_of(uint32_t row_bytes) { return (row_bytes + 15) / 16; }

// Pieces a lane and wavefronts of a row.  One wavefront up to 128 pieces; then one piece a lane, or two where that makes rows of up to 512
// pieces come out even; two beyond, four beyond 2048.  us in front of the block for 1 / 512 / 16384 rows: 2048 columns (256 pieces) one
// wavefront of four pieces 2.2 / 3.8 / 42.0, four of one 1.9 / 3.4 / 42.6, two of two, which is taken, 2.1 / 3.5 / 41.8; 4096 columns one of eight
// 3.4 / 5.7 / 94.1, eight of one 2.1 / 4.8 / 89.6, four of two, which is taken, 2.1 / 4.7 / 88.3 (8192 rows 41.5, eight of one 43.7).  The gradient
// with the sums of columns: 2048 columns two of two 3.0 / 9.6 / 66.9, four of one 2.5 / 9.4 / 68.2; 4096 columns four of two 3.1 / 12.0 / 125, eight of
// one 2.8 / 10.8 / 121; 4096 rows of 3584 columns four of two pieces, some of them empty, 30.0, seven of one 26.8.
struct RowShape { int nv, waves; };
RowShape shape_of(uint32_t pieces) {
  if (pieces <= 128) return {pieces <= 64 ? 1 : 2, 1};
  const int nv = pieces > 2048 ? 4 : pieces > 512 || pieces % 128 == 0 ? 2 : 1;
  return {nv, (int)((pieces + 64 * nv - 1) / (64 * nv))};
}

// Groups of rows of the gradients: per compute unit about 14 wavefronts with one piece a lane, 8 with two, which keeps enough rows on the
// way and leaves few sums of columns to write and read; then as few as have as many rows each.  us for 10000 rows, before the block, sums of
// columns included: 2049 columns (5 wavefronts of a piece) 1 / 2 / 4 groups a unit 82 / 58 / 53, behind it with a full gate 85 / 63 / 84; 4104
// columns (5 of two) 1 / 2 85 / 90, 88 / 97; 3584 columns (7 of one) 4096 rows, 292 groups of 14 or 15 rows 36, 256 of 16 rows 31.
// Few rows are one workgroup's, which finishes the sums itself; us a call, so / with a launch for the sums: 4 rows of 4096 columns 8.6 / 10.6, with a
// channel gate and a bias 9.6 / 11.7, 8 rows 9.5 / 10.6 and 12.5 / 11.7; one wavefront a row, 32 rows of 1000 columns 10.2 / 11.7, 64 17.7 / 11.9.
constexpr int kOneWorkgroupNarrow = 32, kOneWorkgroupWide = 4;
constexpr int kGroups1 = 4096;   // one wavefront a row: us for 30000 rows of 1024 columns with 4096 / 6144 groups 65 / 67
int most_groups(uint32_t pieces) {
  const RowShape s = shape_of(pieces);
  const int a_unit = (s.nv == 1 ? 14 : 8) / s.waves;
  return s.waves == 1 ? kGroups1 : kDefaultCus * (a_unit > 0 ? a_unit : 1);
}
int groups_of(int T, uint32_t pieces) {
  const bool narrow = shape_of(pieces).waves == 1;
  const int side = narrow ? 4 : 1, most = most_groups(pieces);   // side: groups of a workgroup
  if (T <= (narrow ? kOneWorkgroupNarrow : kOneWorkgroupWide)) return T < side ? T : side;
  if (T <= most) return T;
  const int each = (T + most - 1) / most;
  return (T + each - 1) / each;
}
// Workgroups of the gradients, each of which leaves a row of column sums; and the most that this or a smaller batch has, which is what a
// workspace is for (more rows may come out in fewer groups).
int workgroups_of(int T, uint32_t pieces) {
  const int groups = groups_of(T, pieces);
  return shape_of(pieces).waves == 1 ? (groups + 3) / 4 : groups;
}
int most_workgroups(int T, uint32_t pieces) {
  const bool narrow = shape_of(pieces).waves == 1;
  const int most = most_groups(pieces), groups = T <= (narrow ? kOneWorkgroupNarrow : kOneWorkgroupWide) ? 1 : T < most ? T : most;
  return narrow ? (groups + 3) / 4 : groups;
}

template <int DT, bool AFTER, int MW, int NV>
hipError_t norm_as(const NormParams& p, int waves, hipStream_t st) {
  auto kernel = p.row_bytes == (uint32_t)waves * NV * 1024 ? k_norm<DT, MW, NV, AFTER, true> : k_norm<DT, MW, NV, AFTER, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(MW == 1 ? (p.T + 3) / 4 : p.T)), dim3(MW == 1 ? 256 : waves * 64), 0, st, p);
  return hipGetLastError();
}
template <int DT, bool AFTER>
hipError_t norm_type(const NormParams& p, hipStream_t st) {
  const RowShape s = shape_of(pieces_of(p.row_bytes));
  if (s.waves == 1) return s.nv == 1 ? norm_as<DT, AFTER, 1, 1>(p, 1, st) : norm_as<DT, AFTER, 1, 2>(p, 1, st);
  if (s.waves <= 8 && s.nv <= 2) return s.nv == 1 ? norm_as<DT, AFTER, 8, 1>(p, s.waves, st) : norm_as<DT, AFTER, 8, 2>(p, s.waves, st);
  if (s.nv == 2) return norm_as<DT, AFTER, 16, 2>(p, s.waves, st);
  if constexpr (DT == MOE_FP32) return norm_as<DT, AFTER, 16, 4>(p, s.waves, st);
  return hipErrorInvalidValue;   // (no row of two-byte elements is that long)
}
template <bool AFTER>
hipError_t launch_norm(int dtype, const NormParams& p, hipStream_t st) {
  switch (dtype) {
    case MOE_BF16: return norm_type<MOE_BF16, AFTER>(p, st);
    case MOE_FP16: return norm_type<MOE_FP16, AFTER>(p, st);
    default: return norm_type<MOE_FP32, AFTER>(p, st);
  }
}

template <int DT, int MODE, bool WITH_B, int MW, int NV>
hipError_t norm_grad_as(const NormGradParams& p, int waves, hipStream_t st) {
  constexpr bool PRE = MW <= 8;
  const bool given = MODE == GRAD_BEFORE ? p.more != nullptr && p.grad_other != nullptr : MODE != GRAD_AFTER_FULL || p.grad_other != nullptr;
  auto kernel = given && p.row_bytes == (uint32_t)waves * NV * 1024 ? k_norm_grad<DT, MW, NV, MODE, WITH_B, PRE, true> : k_norm_grad<DT, MW, NV, MODE, WITH_B, PRE, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)workgroups_of(p.T, pieces_of(p.row_bytes))), dim3(MW == 1 ? 256 : waves * 64), 0, st, p);
  return hipGetLastError();
}
template <int DT, int MODE, bool WITH_B>
hipError_t norm_grad_b(const NormGradParams& p, hipStream_t st) {
  const RowShape s = shape_of(pieces_of(p.row_bytes));
  if (s.waves == 1) return s.nv == 1 ? norm_grad_as<DT, MODE, WITH_B, 1, 1>(p, 1, st) : norm_grad_as<DT, MODE, WITH_B, 1, 2>(p, 1, st);
  if (s.waves <= 8 && s.nv <= 2) return s.nv == 1 ? norm_grad_as<DT, MODE, WITH_B, 8, 1>(p, s.waves, st) : norm_grad_as<DT, MODE, WITH_B, 8, 2>(p, s.waves, st);
  if (s.nv == 2) return norm_grad_as<DT, MODE, WITH_B, 16, 2>(p, s.waves, st);
  if constexpr (DT == MOE_FP32) return norm_grad_as<DT, MODE, WITH_B, 16, 4>(p, s.waves, st);
  return hipErrorInvalidValue;   // (no row of two-byte elements is that long)
}
template <int DT>
hipError_t norm_grad_type(int mode, const NormGradParams& p, const NormColumnParams& cp, hipStream_t st) {
  if (p.groups > 0) {
    const bool b = p.part_b != nullptr;
    hipError_t e;
    switch (mode) {
      case GRAD_BEFORE: e = b ? norm_grad_b<DT, GRAD_BEFORE, true>(p, st) : norm_grad_b<DT, GRAD_BEFORE, false>(p, st); break;
      case GRAD_AFTER: e = b ? norm_grad_b<DT, GRAD_AFTER, true>(p, st) : norm_grad_b<DT, GRAD_AFTER, false>(p, st); break;
      case GRAD_AFTER_TOKEN: e = b ? norm_grad_b<DT, GRAD_AFTER_TOKEN, true>(p, st) : norm_grad_b<DT, GRAD_AFTER_TOKEN, false>(p, st); break;
      default: e = b ? norm_grad_b<DT, GRAD_AFTER_FULL, true>(p, st) : norm_grad_b<DT, GRAD_AFTER_FULL, false>(p, st); break;
    }
    if (e != hipSuccess) return e;
  }
  if (!cp.grad_gamma && !cp.grad_beta && !cp.grad_gate) return hipSuccess;
  if (cp.groups == 1) return hipSuccess;   // the workgroup has done it
  hipLaunchKernelGGL(k_norm_columns<DT>, dim3((unsigned)((cp.H + 31) / 32)), dim3(1024), 0, st, cp);
  return hipGetLastError();
}
hipError_t launch_norm_grad(int dtype, int mode, const NormGradParams& p, const NormColumnParams& cp, hipStream_t st) {
  switch (dtype) {
    case MOE_BF16: return norm_grad_type<MOE_BF16>(mode, p, cp, st);
    case MOE_FP16: return norm_grad_type<MOE_FP16>(mode, p, cp, st);
    default: return norm_grad_type<MOE_FP32>(mode, p, cp, st);
  }
}

int norm_shape(int32_t T, int32_t H) {
  if (T < 0 || H <= 0) return MOE_ERR_INVALID_ARG;
  if (H < kMinNormColumns || H > kMaxNormColumns || T >= (1 << 24)) return MOE_ERR_UNSUPPORTED;
  return MOE_OK;
}
int norm_call(int32_t T, int32_t H, int32_t dtype, int32_t norm, float eps, float scale) {
  if (element_bytes(dtype) == 0 || (norm != MOE_NORM_RMS && norm != MOE_NORM_LAYER)) return MOE_ERR_INVALID_ARG;
  if (!(eps >= 0.f) || !(eps < 1e30f) || !(scale > -1e30f && scale < 1e30f)) return MOE_ERR_INVALID_ARG;
  const int rc = norm_shape(T, H);
  if (rc != MOE_OK) return rc;
  return (int64_t)T * H * element_bytes(dtype) < (1ll << 35) ? MOE_OK : MOE_ERR_UNSUPPORTED;   // threads of a launch: 32 bits
}
bool gate_ok(const void* gate, int32_t gate_kind, bool rows) {
  if (gate_kind < MOE_GATE_NONE || gate_kind > MOE_GATE_FULL) return false;
  if (gate_kind == MOE_GATE_NONE) return gate == nullptr;
  return (gate != nullptr || (!rows && gate_kind != MOE_GATE_CHANNEL)) && aligned16(gate);
}
// An output may lie in the place of an input of the same rows, not across it.
bool in_place_or_apart(const void* out, std::initializer_list<const void*> ins, size_t bytes) {
  for (const void* in : ins)
    if (out != in && overlap({out, bytes}, {in, bytes})) return false;
  return true;
}

bool in_place(std::initializer_list<const void*> outs, std::initializer_list<const void*> ins) {
  for (const void* out : outs)
    for (const void* in : ins)
      if (out && out == in) return true;
  return false;
}

int status_of(hipError_t e) { return e == hipSuccess ? MOE_OK : MOE_ERR_HIP; }

}  // namespace

}  // namespace moe

using namespace moe;

extern "C" {

int moe_norm_before(const void* residual, const void* update, float residual_scale, const void* gamma, const void* beta,
                    int32_t norm, float eps, int32_t T, int32_t H, int32_t dtype, void* sum, void* x, void* hip_stream) {
  const int rc = norm_call(T, H, dtype, norm, eps, residual_scale);
  if (rc != MOE_OK) return rc;
  if (T == 0) return MOE_OK;
  if (!residual || !gamma || !x) return MOE_ERR_INVALID_ARG;
  if (!aligned16(residual) || !aligned16(update) || !aligned16(gamma) || !aligned16(beta) || !aligned16(sum) || !aligned16(x))
    return MOE_ERR_INVALID_ARG;
  const size_t row_bytes = (size_t)H * element_bytes(dtype), bytes = T * row_bytes;
  if (!in_place_or_apart(sum, {residual, update}, bytes) || !in_place_or_apart(x, {residual, update}, bytes) ||
      !apart({{sum, bytes}, {x, bytes}}, {{gamma, row_bytes}, {beta, row_bytes}}))
    return MOE_ERR_INVALID_ARG;
  NormParams p = {};
  p.residual = (const char*)residual;
  p.branch = (const char*)update;
  p.gamma = (const char*)gamma;
  p.beta = (const char*)beta;
  p.sum = (char*)sum;
  p.out = (char*)x;
  p.in_place = in_place({sum, x}, {residual, update});
  p.layer = norm == MOE_NORM_LAYER;
  p.T = T;
  p.row_bytes = (uint32_t)row_bytes;
  p.scale = residual_scale;
  p.eps = eps;
  p.h = (float)H;
  p.inv_h = 1.0f / (float)H;
  return status_of(launch_norm<false>(dtype, p, (hipStream_t)hip_stream));
}

int moe_norm_after(const void* residual, const void* y, const void* gamma, const void* beta, const void* gate, int32_t gate_kind,
                   float residual_scale, int32_t norm, float eps, int32_t T, int32_t H, int32_t dtype, void* out, void* hip_stream) {
  const int rc = norm_call(T, H, dtype, norm, eps, residual_scale);
  if (rc != MOE_OK) return rc;
  if (!gate_ok(gate, gate_kind, T > 0)) return MOE_ERR_INVALID_ARG;
  if (T == 0) return MOE_OK;
  if (!y || !gamma || !out) return MOE_ERR_INVALID_ARG;
  if (!aligned16(residual) || !aligned16(y) || !aligned16(gamma) || !aligned16(beta) || !aligned16(out)) return MOE_ERR_INVALID_ARG;
  const size_t row_bytes = (size_t)H * element_bytes(dtype), bytes = T * row_bytes;
  const bool full = gate_kind == MOE_GATE_FULL;
  const Span small_gate = {full ? nullptr : gate, gate_kind == MOE_GATE_TOKEN ? (size_t)T * 4 : row_bytes};
  if (!in_place_or_apart(out, {residual, y, full ? gate : nullptr}, bytes) || !apart({{out, bytes}}, {{gamma, row_bytes}, {beta, row_bytes}, small_gate}))
    return MOE_ERR_INVALID_ARG;
  NormParams p = {};
  p.residual = (const char*)residual;
  p.branch = (const char*)y;
  p.gamma = (const char*)gamma;
  p.beta = (const char*)beta;
  p.gate = (const char*)gate;
  p.gate_kind = gate_kind;
  p.out = (char*)out;
  p.in_place = in_place({out}, {residual, y, gate});
  p.layer = norm == MOE_NORM_LAYER;
  p.T = T;
  p.row_bytes = (uint32_t)row_bytes;
  p.scale = residual_scale;
  p.eps = eps;
  p.h = (float)H;
  p.inv_h = 1.0f / (float)H;
  return status_of(launch_norm<true>(dtype, p, (hipStream_t)hip_stream));
}

size_t moe_norm_workspace_bytes(int32_t T, int32_t H) {
  if (norm_shape(T, H) != MOE_OK) return 0;
  const int two = most_workgroups(T, pieces_of((uint32_t)H * 2)), four = most_workgroups(T, pieces_of((uint32_t)H * 4));
  const size_t rows = two > four ? two : four;
  return 2 * rows * (size_t)H * 4;
}

int moe_norm_before_backward(const void* sum, const void* gamma, const void* grad_x, const void* grad_sum, float residual_scale,
                             int32_t norm, float eps, int32_t T, int32_t H, int32_t dtype, void* grad_residual, void* grad_update,
                             float* grad_gamma, float* grad_beta, void* workspace, size_t workspace_bytes, void* hip_stream) {
  const int rc = norm_call(T, H, dtype, norm, eps, residual_scale);
  if (rc != MOE_OK) return rc;
  const size_t row_bytes = (size_t)H * element_bytes(dtype), bytes = T * row_bytes;
  const bool columns = grad_gamma || grad_beta;
  if (!gamma || (T > 0 && (!sum || !grad_x || !grad_residual)) || (columns && !workspace)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(sum) || !aligned16(gamma) || !aligned16(grad_x) || !aligned16(grad_sum) || !aligned16(grad_residual) ||
      !aligned16(grad_update) || !aligned16(grad_gamma) || !aligned16(grad_beta) || !aligned16(workspace))
    return MOE_ERR_INVALID_ARG;
  const size_t scratch = columns ? moe_norm_workspace_bytes(T, H) : 0, sums = (size_t)H * 4;
  if (workspace_bytes < scratch) return MOE_ERR_WORKSPACE_TOO_SMALL;
  const Span small[3] = {{grad_gamma, sums}, {grad_beta, sums}, {columns ? workspace : nullptr, scratch}};
  if (!in_place_or_apart(grad_residual, {sum, grad_x, grad_sum}, bytes) || !in_place_or_apart(grad_update, {sum, grad_x, grad_sum}, bytes) ||
      !apart({{grad_residual, bytes}, {grad_update, bytes}, small[0], small[1], small[2]}, {{gamma, row_bytes}}) ||
      !apart({small[0], small[1], small[2]}, {{sum, bytes}, {grad_x, bytes}, {grad_sum, bytes}}))
    return MOE_ERR_INVALID_ARG;
  NormGradParams p = {};
  p.v = (const char*)sum;
  p.g = (const char*)grad_x;
  p.gamma = (const char*)gamma;
  p.more = (const char*)grad_sum;
  p.grad_v = (char*)grad_residual;
  p.grad_other = (char*)grad_update;
  p.in_place = in_place({grad_residual, grad_update}, {sum, grad_x, grad_sum});
  p.layer = norm == MOE_NORM_LAYER;
  p.T = T;
  p.H = H;
  p.row_bytes = (uint32_t)row_bytes;
  p.groups = groups_of(T, pieces_of(p.row_bytes));
  p.part_a = columns ? (float*)workspace : nullptr;
  p.part_b = grad_beta ? p.part_a + (size_t)workgroups_of(T, pieces_of(p.row_bytes)) * H : nullptr;
  p.scale = residual_scale;
  p.eps = eps;
  p.h = (float)H;
  p.inv_h = 1.0f / (float)H;
  NormColumnParams cp = {};
  cp.part_a = p.part_a;
  cp.part_b = p.part_b;
  cp.gamma = p.gamma;
  cp.grad_gamma = grad_gamma;
  cp.grad_beta = grad_beta;
  cp.groups = workgroups_of(T, pieces_of(p.row_bytes));
  cp.H = H;
  p.columns = cp;
  return status_of(launch_norm_grad(dtype, GRAD_BEFORE, p, cp, (hipStream_t)hip_stream));
}

int moe_norm_after_backward(const void* y, const void* gamma, const void* beta, const void* gate, int32_t gate_kind,
                            float residual_scale, const void* grad_out, int32_t norm, float eps, int32_t T, int32_t H, int32_t dtype,
                            void* grad_y, float* grad_gamma, float* grad_beta, void* grad_gate, void* workspace,
                            size_t workspace_bytes, void* hip_stream) {
  const int rc = norm_call(T, H, dtype, norm, eps, residual_scale);
  if (rc != MOE_OK) return rc;
  if (!gate_ok(gate, gate_kind, T > 0) || (gate_kind == MOE_GATE_NONE && grad_gate)) return MOE_ERR_INVALID_ARG;
  const size_t row_bytes = (size_t)H * element_bytes(dtype), bytes = T * row_bytes;
  const bool channel = gate_kind == MOE_GATE_CHANNEL, columns = grad_gamma || grad_beta || (channel && grad_gate);
  if (!gamma || (T > 0 && (!y || !grad_out || !grad_y)) || (columns && !workspace)) return MOE_ERR_INVALID_ARG;
  if (!aligned16(y) || !aligned16(gamma) || !aligned16(beta) || !aligned16(grad_out) || !aligned16(grad_y) || !aligned16(grad_gamma) ||
      !aligned16(grad_beta) || !aligned16(grad_gate) || !aligned16(workspace))
    return MOE_ERR_INVALID_ARG;
  const size_t scratch = columns ? moe_norm_workspace_bytes(T, H) : 0, sums = (size_t)H * 4;
  if (workspace_bytes < scratch) return MOE_ERR_WORKSPACE_TOO_SMALL;
  const bool full = gate_kind == MOE_GATE_FULL, token = gate_kind == MOE_GATE_TOKEN;
  const Span small[4] = {{grad_gamma, sums}, {grad_beta, sums}, {columns ? workspace : nullptr, scratch}, {full ? nullptr : grad_gate, token ? (size_t)T * 4 : sums}};
  const void *full_gate = full ? gate : nullptr, *grad_full = full ? grad_gate : nullptr;
  if (!in_place_or_apart(grad_y, {y, grad_out, full_gate}, bytes) || !in_place_or_apart(grad_full, {y, grad_out, full_gate}, bytes) ||
      !apart({{grad_y, bytes}, {grad_full, bytes}, small[0], small[1], small[2], small[3]},
             {{gamma, row_bytes}, {beta, row_bytes}, {full ? nullptr : gate, token ? (size_t)T * 4 : row_bytes}}) ||
      !apart({small[0], small[1], small[2], small[3]}, {{y, bytes}, {grad_out, bytes}, {full_gate, bytes}}))
    return MOE_ERR_INVALID_ARG;
  NormGradParams p = {};
  p.v = (const char*)y;
  p.g = (const char*)grad_out;
  p.gamma = (const char*)gamma;
  p.beta = (const char*)beta;
  p.gate = (const char*)gate;
  p.gate_kind = gate_kind;
  p.grad_v = (char*)grad_y;
  p.grad_other = full ? (char*)grad_gate : nullptr;
  p.in_place = in_place({grad_y, grad_full}, {y, grad_out, full_gate});
  p.grad_token_gate = token ? (float*)grad_gate : nullptr;
  p.layer = norm == MOE_NORM_LAYER;
  p.T = T;
  p.H = H;
  p.row_bytes = (uint32_t)row_bytes;
  p.groups = groups_of(T, pieces_of(p.row_bytes));
  p.part_a = columns ? (float*)workspace : nullptr;
  p.part_b = grad_beta || (channel && grad_gate && beta) ? p.part_a + (size_t)workgroups_of(T, pieces_of(p.row_bytes)) * H : nullptr;
  p.scale = residual_scale;
  p.eps = eps;
  p.h = (float)H;
  p.inv_h = 1.0f / (float)H;
  NormColumnParams cp = {};
  cp.part_a = p.part_a;
  cp.part_b = p.part_b;
  cp.gamma = p.gamma;
  cp.beta = p.beta;
  cp.gate = channel ? p.gate : nullptr;
  cp.grad_gamma = grad_gamma;
  cp.grad_beta = grad_beta;
  cp.grad_gate = channel ? (float*)grad_gate : nullptr;
  cp.groups = workgroups_of(T, pieces_of(p.row_bytes));
  cp.H = H;
  const int mode = full ? GRAD_AFTER_FULL : token ? GRAD_AFTER_TOKEN : GRAD_AFTER;
  p.columns = cp;
  return status_of(launch_norm_grad(dtype, mode, p, cp, (hipStream_t)hip_stream));
}

}  // extern "C"
