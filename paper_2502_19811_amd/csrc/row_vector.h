// Rows of bf16, fp16 or fp32 in 16-byte pieces, for the operators around the experts.
//
// A row of H >= 8 elements starts at a multiple of its element's size only (H may be odd), so a piece is loaded and stored with
// the alignment of its element: global memory instructions of gfx950 take any.  The last piece of a row that is not a multiple
// of 16 bytes lies over the one before it, which needs no code of its own for what is left.
#pragma once
#include <initializer_list>

#include "moe_device.h"

namespace moe {

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <int DT> struct Row;
template <> struct Row<MOE_BF16> {
  static constexpr int kBytes = 2, kVec = 8;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&f)[8]) {
#pragma unroll
    for (int c = 0; c < 4; c++) {
      f[2 * c] = __uint_as_float(v[c] << 16);
      f[2 * c + 1] = __uint_as_float(v[c] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const bf16x2 pr = {(__bf16)f[2 * c], (__bf16)f[2 * c + 1]};
      v[c] = __builtin_bit_cast(uint32_t, pr);
    }
    return v;
  }
};
template <> struct Row<MOE_FP16> {
  static constexpr int kBytes = 2, kVec = 8;
  typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&f)[8]) {
#pragma unroll
    for (int c = 0; c < 4; c++) {
      const f16x2 pr = __builtin_bit_cast(f16x2, (uint32_t)v[c]);
      f[2 * c] = (float)pr[0];
      f[2 * c + 1] = (float)pr[1];
    }
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[8]) {
    u32x4 v;
#pragma unroll
    for (int c = 0; c < 4; c++) {
      // The conversion stays apart from what computed the value: where the compiler joins it to a fused operation, the sum is rounded
      // to 16 bits at once and not to 32 before, and whether it does depends on the code around.
      float lo = f[2 * c], hi = f[2 * c + 1];
      asm("" : "+v"(lo), "+v"(hi));
      const f16x2 pr = {(_Float16)lo, (_Float16)hi};
      v[c] = __builtin_bit_cast(uint32_t, pr);
    }
    return v;
  }
};
template <> struct Row<MOE_FP32> {
  static constexpr int kBytes = 4, kVec = 4;
  static __device__ __forceinline__ void unpack(const u32x4& v, float (&f)[4]) {
#pragma unroll
    for (int c = 0; c < 4; c++) f[c] = __uint_as_float(v[c]);
  }
  static __device__ __forceinline__ u32x4 pack(const float (&f)[4]) {
    u32x4 v;
#pragma unroll
    for (int c = 0; c < 4; c++) v[c] = __float_as_uint(f[c]);
    return v;
  }
};

// A thread's piece of a row is meant to start at byte `start`; it is taken from where a whole piece still fits.  Elements that
// two pieces then hold are computed twice, alike, and stored twice; sums leave them out of the later one: counted() tells.
__device__ __forceinline__ uint32_t piece_at(uint32_t start, uint32_t row_bytes) { return min(start, row_bytes - 16); }
__device__ __forceinline__ u32x4 load_piece(const char* row, uint32_t start, uint32_t row_bytes) {
  return *(const u32x4_any*)(row + piece_at(start, row_bytes));
}
__device__ __forceinline__ void store_piece(char* row, uint32_t start, uint32_t row_bytes, const u32x4& v) {
  if (start < row_bytes) *(u32x4_any*)(row + piece_at(start, row_bytes)) = v;
}
// The same with the non-temporal hint, which leaves little behind in the caches: for inputs, whose next reader, if there is one, comes
// much later, and for the outputs of which that is true (rows for the experts' products, the residual stream).  An output that the next
// operator reads (the normed rows, the combined tokens, their gradients) does without it.  us of the forward / backward calls of a block
// (H = 4096, k = 2, the caches run over where the experts' products are), without any hints, with these, with the hint on all
// loads and stores: 1024 tokens 31 / 48, 27 / 47, 26 / 45; 4096 84 / 111, 77 / 110, 83 / 115; 8192 162 / 222, 143 / 215, 155 / 225; 32768
// 613 / 835, 529 / 798, 582 / 806.
__device__ __forceinline__ u32x4 load_once(const char* row, uint32_t start, uint32_t row_bytes) {
  return __builtin_nontemporal_load((const u32x4_any*)(row + piece_at(start, row_bytes)));
}
__device__ __forceinline__ void store_once(char* row, uint32_t start, uint32_t row_bytes, const u32x4& v) {
  if (start < row_bytes) __builtin_nontemporal_store((u32x4_any)v, (u32x4_any*)(row + piece_at(start, row_bytes)));
}
// First element of the piece that counts in a sum over the row (0: all of them; kVec and more: none).
template <int UNIT>
__device__ __forceinline__ int counted(uint32_t start, uint32_t row_bytes) { return (int)((start - piece_at(start, row_bytes)) / UNIT); }

// Sum over the wavefront in a fixed order, in every lane.
__device__ __forceinline__ float wave_sum(float v) {
  auto step = [&](auto ctrl, auto rows) {   // lanes the control does not reach add 0
    v += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value, 0xf, true));
  };
  step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr 1, 2, 4, 8: the last lane of
  step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});   // every 16 has their sum
  step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});
  step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast 15, 31: the last lane of all
  step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Bytes of an element, 0: no such type.
inline int element_bytes(int dtype) { return dtype == MOE_BF16 || dtype == MOE_FP16 ? 2 : dtype == MOE_FP32 ? 4 : 0; }

inline bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Whether two buffers share bytes; a buffer that is not given shares none.
struct Span { const void* at; size_t bytes; };
inline bool overlap(const Span& a, const Span& b) {
  return a.at && b.at && (uintptr_t)a.at < (uintptr_t)b.at + b.bytes && (uintptr_t)b.at < (uintptr_t)a.at + a.bytes;
}
// Whether no output shares bytes with another output or with an input.
inline bool apart(std::initializer_list<Span> outs, std::initializer_list<Span> ins) {
  for (const Span* a = outs.begin(); a != outs.end(); a++) {
    for (const Span* b = outs.begin(); b != a; b++)
      if (overlap(*a, *b)) return false;
    for (const Span& b : ins)
      if (overlap(*a, b)) return false;
  }
  return true;
}

}  // namespace moe
