// Rows of an 8-bit cache: e4m3 codes and one power of two for each (token, KV head).
//
// A row x is held as codes c and a byte e, x_i ~ c_i 2^(e - 127), with e the smallest in [1, 254] for which the largest
// |x_i| is at most 448 * 2^(e - 127): 448 is the largest code.  Scaling by a power of two is exact, so a value is rounded
// once, by the code, to 2^-4 of itself at most (2^-10 of 2^(e-127) where the code is below 2^-6).  (A scale of 32 bits would use the codes' range up to 448 in every row, which gains
// nothing: the codes are floating-point numbers, their relative steps are the same everywhere but at the bottom.)
// A row with an element that is infinite or no number is held as NaN codes with e = 255, which stands for NaN.
#pragma once

#include "paged.cuh"

namespace tkphi {

// What scale byte e stands for: 2^(e-127), 255: NaN.
__device__ __forceinline__ float held_scale(uint32_t e) {
  const uint32_t w = e == 0 ? 0x00400000u : e << 23;
  return __uint_as_float(e == 255u ? 0x7fc00000u : w);
}
// Scale byte of a row whose largest magnitude has these bits (sign bit clear; NaN's are the largest of all).
__device__ __forceinline__ uint32_t held_byte(uint32_t magnitude) {
  if (magnitude >= 0x7f800000u) return 255u;
  const int e = (int)((magnitude + 0x1fffffu) >> 23) - 8;      // a fraction above 1.75 goes to the next power
  return e < 1 ? 1u : (uint32_t)e;
}
// 2^(127 - e) for e of a finite row (1 .. 247).
__device__ __forceinline__ float held_inverse(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// Four values (already scaled) as codes, the first in the lowest byte.
__device__ __forceinline__ uint32_t pack_codes(float a, float b, float c, float d) {
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(b), "f"(a));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(d), "f"(c));
  return (uint32_t)lo | (uint32_t)hi << 16;
}
// The two low and the two high codes of w as pairs of fp16 numbers (exact).
__device__ __forceinline__ void unpack_codes(uint32_t w, uint32_t& lo, uint32_t& hi) {
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.rn.f16x2.e4m3x2 %0, l;\n cvt.rn.f16x2.e4m3x2 %1, h;\n}"
      : "=r"(lo), "=r"(hi) : "r"(w));
}
// The element type as what comes out of an 8-bit cache is rounded to it: finite fp16 numbers from 63488 on are held as 65536, which
// fp16 does not have, so what is finite becomes its largest number, not infinite.
struct Fp16Held : Fp16 {
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    uint32_t r;
    asm("cvt.rn.satfinite.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
  }
};
template <typename T> struct OutOfHeld { using type = T; };
template <> struct OutOfHeld<Fp16> { using type = Fp16Held; };

// Four codes times a scale, as two pairs of the element type.
template <typename T>
__device__ __forceinline__ uint2 held_values(uint32_t w, float scale) {
  uint32_t lo, hi;
  unpack_codes(w, lo, hi);
  using Out = typename OutOfHeld<T>::type;
  return make_uint2(Out::pack(Fp16::lo(lo) * scale, Fp16::hi(lo) * scale), Out::pack(Fp16::lo(hi) * scale, Fp16::hi(hi) * scale));
}

// ---------------------------------------------------------------- launches (host)
struct HeldCache {
  uint8_t* k_scales; uint8_t* v_scales;      // [n_pages][hkv][page_size]
};
// Append with head norms and / or to an 8-bit cache.
struct WriteProblem {
  AppendProblem a;                           // (8-bit cache: strides in bytes)
  const float* q_weight; long long q_weight_head;      // null: not normed; elements between heads, 0: one for all
  const float* k_weight; long long k_weight_head;
  float eps;
  HeldCache held;                            // k_scales null: a 16-bit cache
  bool wide;                                 // all 16-bit rows that are written lie on 32-byte boundaries (set by the launch)
};
cudaError_t launch_paged_write(const WriteProblem& p, bool bf16, cudaStream_t st);

struct ReadProblem {
  int batch, hkv, d;
  int page_shift, n_pages, max_pages;
  const int* table;
  const long long* kv_lens;
  long long max_kv;
  const uint8_t* k; const uint8_t* v;
  long long stride_page, stride_head, stride_token;    // bytes
  HeldCache held;
  const long long* cu_rows;                  // [batch + 1]
  const long long* first;                    // [batch] or null: 0
  void* k_out; void* v_out;                  // either may be null
  long long k_row, k_head, v_row, v_head;    // elements
  long long total_rows;
  int* status;
  int heads;                                 // KV heads of a CTA (set by the launch)
};
constexpr int kReadRows = 64;                // rows of a CTA
cudaError_t launch_paged_read(const ReadProblem& p, bool bf16, cudaStream_t st);

constexpr int kExpandRows = 128;             // rows of an expanded page
struct ExpandProblem {
  const uint8_t* k; const uint8_t* v;
  long long stride_page, stride_head, stride_token;    // bytes
  HeldCache held;
  void* k_out; void* v_out;                  // [pages][hkv][128][d]
  int* table; int max_pages;                 // [batch][max_pages] written for the sequences with many rows
  int heads;                                 // KV heads of a CTA (set by the launch)
};
cudaError_t launch_paged_expand(const PagedProblem& p, const ExpandProblem& x, int d, bool bf16, int pages, cudaStream_t st);

constexpr int kHeldKeys = 128;               // keys of one tile of the row kernel
int paged8_row_ctas(int d, int max_rows);    // its CTAs per multiprocessor where units are dealt out as a line
cudaError_t launch_paged8_rows(const PagedProblem& p, const HeldCache& held, const CUtensorMap& tk, const CUtensorMap& tv, int d,
                               bool bf16, bool block, bool split, int max_rows, int grid, cudaStream_t st);
cudaError_t launch_paged8_rows_merge(const PagedProblem& p, int d, bool bf16, bool block, int units, int max_rows, cudaStream_t st);

}  // namespace tkphi
