// Matrices of 4-bit blocks as kernels see them (kernels_mx4.hip), and the launches of the operators around them.
#pragma once

#include "kv4.hpp"

namespace dllmc {

// codes [rows][Kp / 2]; scales [ceil(rows / 32)][Kp / 256][64 lanes][4]: lane l, byte j has block 8 c + 2 j + l / 32 of row 32 g + l % 32, so
// that a lane of the 32 x 32 x 64 product has the scales of its four products of a 256-element line in one register.
struct Mx4Tensor {
  uint8_t* codes;
  uint8_t* scales;
  int rows, Kp;
};
inline int mx4_width(int K) { return (K + 255) / 256 * 256; }
inline size_t mx4_code_bytes(int rows, int K) { return (static_cast<size_t>(rows) * (mx4_width(K) / 2) + 255) / 256 * 256; }
inline size_t mx4_bytes(int rows, int K) {
  return mx4_code_bytes(rows, K) + (static_cast<size_t>(rows) + 31) / 32 * 32 * (mx4_width(K) / 32);
}
inline Mx4Tensor mx4_tensor(const void* p, int rows, int K) {
  uint8_t* codes = static_cast<uint8_t*>(const_cast<void*>(p));
  return Mx4Tensor{codes, codes + mx4_code_bytes(rows, K), rows, mx4_width(K)};
}
// where the scale of the block of element t of row r lies
__device__ __forceinline__ size_t mx4_scale_at(int r, int t, int Kp) {
  return ((static_cast<size_t>(r >> 5) * (Kp >> 8) + (t >> 8)) * 64 + (t >> 5 & 1) * 32 + (r & 31)) * 4 + (t >> 6 & 3);
}

// Eight neighbouring elements as codes (zeros where the block is not finite), element e in bits 4 e.
__device__ __forceinline__ uint32_t mx4_codes(const float (&v)[8], uint32_t scale) {
  uint32_t w = 0;
  if (scale != 255) {
    const float s = __uint_as_float(scale << 23);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
  }
  return w;
}
// Bits of the largest magnitude of a block, four lanes of a quad with eight elements each.
__device__ __forceinline__ uint32_t block32_top(const float (&v)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);  // (magnitudes order as integers, NaN last)
  top = max(top, __float_as_uint(dpp_xor1(__uint_as_float(top))));
  return max(top, __float_as_uint(dpp_xor2(__uint_as_float(top))));
}

// Elements t .. t + 7 of a row of `len`, zeros behind it.  Rows start at any element: the vector memory instructions take 16 bytes at any address
// that is a multiple of the element's size.  WHOLE: len is a multiple of 8.
typedef uint32_t u32x4_at2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_at4 __attribute__((ext_vector_type(4), aligned(4)));
template <bool WHOLE = false> __device__ __forceinline__ void load8(const bf16_t* row, int t, int len, float (&v)[8]) {
  if (t + 8 <= len) {
    const u32x4_at2 a = *reinterpret_cast<const u32x4_at2*>(row + t);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e % 2 ? a[e / 2] & 0xffff0000u : a[e / 2] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = !WHOLE && t + e < len ? ldf(row + t + e) : 0.f;
  }
}
template <bool WHOLE = false> __device__ __forceinline__ void load8(const float* row, int t, int len, float (&v)[8]) {
  if (t + 8 <= len) {
    const u32x4_at4 a = *reinterpret_cast<const u32x4_at4*>(row + t), b = *reinterpret_cast<const u32x4_at4*>(row + t + 4);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e < 4 ? a[e % 4] : b[e % 4]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = !WHOLE && t + e < len ? ldf(row + t + e) : 0.f;
  }
}
__device__ __forceinline__ void store_pieces(bf16_t* p, const float (&v)[8]) {
  *reinterpret_cast<u32x4_at2*>(p) = u32x4_at2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
}
__device__ __forceinline__ void store_pieces(float* p, const float (&v)[8]) {
#pragma unroll
  for (int h = 0; h < 8; h += 4)
    *reinterpret_cast<u32x4_at4*>(p + h) =
        u32x4_at4{__float_as_uint(v[h]), __float_as_uint(v[h + 1]), __float_as_uint(v[h + 2]), __float_as_uint(v[h + 3])};
}
template <bool WHOLE = false, typename T> __device__ __forceinline__ void store8(T* row, int t, int len, const float (&v)[8]) {
  if (t + 8 <= len) {
    store_pieces(row + t, v);
  } else if (!WHOLE) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (t + e < len) stf(row + t + e, v[e]);
  }
}

// rows of x in 4-bit blocks, and back
void launch_quant_mx4(int dtype, const void* x, int x_rows, const int* rows, int M, int K, Mx4Tensor out, hipStream_t st);
void launch_mx4_load(int dtype, Mx4Tensor in, const int* rows, int M, int K, void* out, hipStream_t st);
void launch_load8(int dtype, const int8_t* q, const float* scale, int q_rows, int K, const int* rows, int M, void* out, hipStream_t st);
struct Mx4Plan { int wide, bm, bn, S, per; };  // wide: tile kernel; else ring of bm x bn and S slices of `per` lines of 256 elements
Mx4Plan plan_mx4(int M, int N, int Kp);
size_t linear_mx4_scratch_bytes(const Mx4Plan& p, int M, int N);
void launch_linear_mx4(const Mx4Plan& p, int dtype, Mx4Tensor a, Mx4Tensor w, void* out, void* scratch, hipStream_t st);

// Norm of stream + x in few bits (kernels_norm8.hip): 8-bit rows (q, scale) or 4-bit ones (mx).
struct NormRows {
  const void* x;       // [M, d] or null
  const void* stream;  // [stream_rows, d]
  const int* rows;     // or null
  const void* gain;
  void* sum_out;       // [M, d] or null
  int stream_rows, M, d;
  float eps;
};
void launch_norm_quant8(int dtype, int stream_dtype, const NormRows& n, int8_t* q, float* scale, hipStream_t st);
void launch_norm_mx4(int dtype, int stream_dtype, const NormRows& n, Mx4Tensor out, hipStream_t st);

// What rows of logits say about tokens (kernels_logprobs.hip).
constexpr int kMaxTop = 64;
struct LogprobRows {
  const void* logits;
  int ld, M, vocab;
  const int* tokens;  // [M, n_given]
  int n_given, top_k;
  float* logp;        // [M, n_given]
  float* entropy;     // [M] or null
  int* top_ids;       // [M, top_k]
  float* top_logp;
};
size_t logprobs_scratch_bytes(int dtype, int M, int vocab, int top_k);
void launch_logprobs(int dtype, const LogprobRows& r, void* scratch, hipStream_t st);

}  // namespace dllmc
