// K/V cache tensors held in 4 bits, and the attention that reads them.
//
// A block is 32 neighbouring elements of a head: codes of 4 bits (sign, and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) times one power of
// two, the smallest that holds the block's largest magnitude.  What a code stands for is exact in bf16 (two significant bits,
// exponents of +-125 clamped so that nothing is subnormal), so the matrix cores get a cached value with one conversion
// instruction and no rounding.  A tensor is head-major, [H][rows][d_h / 2] bytes of codes, then [H][rows][d_h / 32] of scales: what an
// attention workgroup reads, the keys of one head, is one contiguous run (one per page in a paged cache).
#include "common.hpp"
#include "kv4.hpp"

namespace dllmc {

namespace {

// ---- rows in and out -------------------------------------------------------------------------------
// Four lanes take a block, eight elements each: one 16-byte load of bf16 (two of float32), a maximum over the quad
// by lane moves, four bytes of codes.  Bound by the bytes: 64.5 bits an element in and out of a bf16 row.
template <typename T>
__global__ __launch_bounds__(256) void k_kv4_store(const T* __restrict__ x, long long pieces, int width,
                                                   const int* __restrict__ rows, Kv4Tensor c, int cache_rows, int d_h) {
  // a piece is eight elements (their number is a multiple of 4: whole quads leave)
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < pieces; p += static_cast<long long>(gridDim.x) * 256) {
  const int per_row = width / 8;
  const int i = static_cast<int>(p / per_row), t = static_cast<int>(p % per_row) * 8;
  float v[8];
  Eight<T>::load(x + p * 8, v);
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);  // (magnitudes order as integers, NaN last)
  top = max(top, __float_as_uint(dpp_xor1(__uint_as_float(top))));
  top = max(top, __float_as_uint(dpp_xor2(__uint_as_float(top))));
  const int row = rows ? rows[i] : i;
  if (static_cast<unsigned>(row) >= static_cast<unsigned>(cache_rows)) continue;
  const uint32_t scale = kv4_scale_byte(top);
  uint32_t w = 0;
  if (scale != 255) {
    const float s = __uint_as_float(scale << 23);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
  }
  const size_t at = static_cast<size_t>(t / d_h) * cache_rows + row;
  *reinterpret_cast<uint32_t*>(c.codes + at * (d_h / 2) + t % d_h / 2) = w;
  if (t % 32 == 0) c.scales[at * (d_h / 32) + t % d_h / 32] = static_cast<uint8_t>(scale);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_kv4_load(Kv4Tensor c, int cache_rows, int d_h, const int* __restrict__ rows,
                                                  long long pieces, int width, T* __restrict__ out) {
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < pieces; p += static_cast<long long>(gridDim.x) * 256) {
  const int per_row = width / 8;
  const int i = static_cast<int>(p / per_row), t = static_cast<int>(p % per_row) * 8;
  const int row = rows ? rows[i] : i;
  uint32_t w = 0, scale = 127;
  if (static_cast<unsigned>(row) < static_cast<unsigned>(cache_rows)) {
    const size_t at = static_cast<size_t>(t / d_h) * cache_rows + row;
    w = *reinterpret_cast<const uint32_t*>(c.codes + at * (d_h / 2) + t % d_h / 2);
    scale = c.scales[at * (d_h / 32) + t % d_h / 32];
  }
  const uint4 b = __builtin_bit_cast(uint4, kv4_expand(w, scale));
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint4*>(out + p * 8) = b;
  } else {
    const uint32_t u[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<float4*>(out + p * 8 + 4 * h) =
          make_float4(__uint_as_float(u[2 * h] << 16), __uint_as_float(u[2 * h] & 0xffff0000u),
                      __uint_as_float(u[2 * h + 1] << 16), __uint_as_float(u[2 * h + 1] & 0xffff0000u));
  }
  }
}

inline unsigned groups(long long items) {
  const long long g = (items + 255) / 256;
  return static_cast<unsigned>(g < (1 << 20) ? g : 1 << 20);
}

}  // namespace

void launch_kv4_store(int dtype, const void* x, int M, int width, const int* rows, Kv4Tensor c, int cache_rows, int d_h,
                      hipStream_t st) {
  const long long pieces = static_cast<long long>(M) * (width / 8);
  if (dtype == 1)
    hipLaunchKernelGGL(k_kv4_store<bf16_t>, dim3(groups(pieces)), dim3(256), 0, st, static_cast<const bf16_t*>(x), pieces,
                       width, rows, c, cache_rows, d_h);
  else
    hipLaunchKernelGGL(k_kv4_store<float>, dim3(groups(pieces)), dim3(256), 0, st, static_cast<const float*>(x), pieces,
                       width, rows, c, cache_rows, d_h);
}

void launch_kv4_load(int dtype, Kv4Tensor c, int cache_rows, int d_h, const int* rows, int M, int width, void* out,
                     hipStream_t st) {
  const long long pieces = static_cast<long long>(M) * (width / 8);
  if (dtype == 1)
    hipLaunchKernelGGL(k_kv4_load<bf16_t>, dim3(groups(pieces)), dim3(256), 0, st, c, cache_rows, d_h, rows, pieces, width,
                       static_cast<bf16_t*>(out));
  else
    hipLaunchKernelGGL(k_kv4_load<float>, dim3(groups(pieces)), dim3(256), 0, st, c, cache_rows, d_h, rows, pieces, width,
                       static_cast<float*>(out));
}

}  // namespace dllmc
