// K/V cache tensors held in 4 bits: rows in and out.
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
// by lane moves, four bytes of codes.  Bound by the bytes: 20.25 bits an element in and out of a bf16 row.
// A thread takes kTrips pieces of eight elements, a workgroup's 256 apart, all loaded before the first is used.
constexpr int kTrips = 4;
// Sixteen workgroups that follow each other run on one XCD: a head's rows lie 64 bytes of codes and 4 of scales apart, so neighbouring rows
// share lines, which an L2 sees whole.  12288 x 4096 in bf16 to the codes 32.2 to 31.0 us, back 22.6 to 21.0 (four workgroups 30.4 and
// 22.0, 64 of them 30.5 and 20.7 but smaller tensors slower).  Non-temporal loads and stores: alone 3 to 27 % quicker, with a
// reader behind them to 17 % slower; not taken.
constexpr int kNear = 16;

template <typename T>
__global__ __launch_bounds__(256) void k_kv4_store(const T* __restrict__ x, uint32_t pieces, uint32_t per_row,
                                                   const int* __restrict__ rows, int row0, Kv4Tensor c, int cache_rows, int d_h) {
  const uint32_t p0 = xcd_group_item(blockIdx.x, gridDim.x, kNear) * (256 * kTrips) + threadIdx.x;
  float v[kTrips][8];
  int row[kTrips];
#pragma unroll
  for (int u = 0; u < kTrips; ++u) {
    const uint32_t p = min(p0 + u * 256, pieces - 1);  // (whole quads stay together: their number is a multiple of 4, and so is 256)
    const int i = static_cast<int>(p / per_row);
    row[u] = rows ? rows[i] : row0 + i;
    Eight<T>::load(x + static_cast<size_t>(p) * 8, v[u]);
  }
#pragma unroll
  for (int u = 0; u < kTrips; ++u) {
    const uint32_t p = p0 + u * 256;
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[u][e]) & 0x7fffffffu);  // (magnitudes order as integers, NaN last)
    top = max(top, __float_as_uint(dpp_xor1(__uint_as_float(top))));
    top = max(top, __float_as_uint(dpp_xor2(__uint_as_float(top))));
    if (p >= pieces || static_cast<unsigned>(row[u]) >= static_cast<unsigned>(cache_rows)) continue;
    const uint32_t scale = kv4_scale_byte(top);
    uint32_t w = 0;
    if (scale != 255) {
      const float s = __uint_as_float(scale << 23);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][0], v[u][1], s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][2], v[u][3], s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][4], v[u][5], s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[u][6], v[u][7], s, 3);
    }
    const uint32_t t = p % per_row * 8, h = t / d_h, e = t % d_h;
    const size_t at = static_cast<size_t>(h) * cache_rows + row[u];
    *reinterpret_cast<uint32_t*>(c.codes + at * (d_h / 2) + e / 2) = w;
    if (t % 32 == 0) c.scales[at * (d_h / 32) + e / 32] = static_cast<uint8_t>(scale);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_kv4_load(Kv4Tensor c, int cache_rows, int d_h, const int* __restrict__ rows, int row0,
                                                  uint32_t pieces, uint32_t per_row, T* __restrict__ out) {
  const uint32_t p0 = xcd_group_item(blockIdx.x, gridDim.x, kNear) * (256 * kTrips) + threadIdx.x;
  uint32_t w[kTrips], scale[kTrips];
#pragma unroll
  for (int u = 0; u < kTrips; ++u) {
    const uint32_t p = min(p0 + u * 256, pieces - 1), t = p % per_row * 8, h = t / d_h, e = t % d_h;
    const int i = static_cast<int>(p / per_row), r = rows ? rows[i] : row0 + i;
    const bool ok = static_cast<unsigned>(r) < static_cast<unsigned>(cache_rows);
    const size_t at = static_cast<size_t>(h) * cache_rows + (ok ? r : 0);
    w[u] = *reinterpret_cast<const uint32_t*>(c.codes + at * (d_h / 2) + e / 2);
    scale[u] = c.scales[at * (d_h / 32) + e / 32];
    if (!ok) {
      w[u] = 0;
      scale[u] = 127;
    }
  }
#pragma unroll
  for (int u = 0; u < kTrips; ++u) {
    const uint32_t p = p0 + u * 256;
    if (p >= pieces) continue;
    const uint4 b = __builtin_bit_cast(uint4, kv4_expand(w[u], scale[u]));
    if constexpr (sizeof(T) == 2) {
      *reinterpret_cast<uint4*>(out + static_cast<size_t>(p) * 8) = b;
    } else {
      const uint32_t f[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int h = 0; h < 2; ++h)
        *reinterpret_cast<float4*>(out + static_cast<size_t>(p) * 8 + 4 * h) =
            make_float4(__uint_as_float(f[2 * h] << 16), __uint_as_float(f[2 * h] & 0xffff0000u),
                        __uint_as_float(f[2 * h + 1] << 16), __uint_as_float(f[2 * h + 1] & 0xffff0000u));
    }
  }
}

}  // namespace

// Pieces are counted in 32 bits: at most 2^30 a launch, in whole rows.
template <typename F> void in_parts(int M, int width, F&& f) {
  const int per_row = width / 8, most = (1 << 30) / per_row;
  for (int i0 = 0; i0 < M; i0 += most) {
    const uint32_t pieces = static_cast<uint32_t>(M - i0 < most ? M - i0 : most) * per_row;
    f(i0, pieces, static_cast<uint32_t>(per_row), dim3((pieces + 256 * kTrips - 1) / (256 * kTrips)));
  }
}

void launch_kv4_store(int dtype, const void* x, int M, int width, const int* rows, Kv4Tensor c, int cache_rows, int d_h,
                      hipStream_t st) {
  in_parts(M, width, [&](int i0, uint32_t pieces, uint32_t per_row, dim3 grid) {
    const int* r = rows ? rows + i0 : nullptr;
    const size_t at = static_cast<size_t>(i0) * width;
    if (dtype == 1)
      hipLaunchKernelGGL(k_kv4_store<bf16_t>, grid, dim3(256), 0, st, static_cast<const bf16_t*>(x) + at, pieces, per_row, r, i0, c,
                         cache_rows, d_h);
    else
      hipLaunchKernelGGL(k_kv4_store<float>, grid, dim3(256), 0, st, static_cast<const float*>(x) + at, pieces, per_row, r, i0, c, cache_rows,
                         d_h);
  });
}

void launch_kv4_load(int dtype, Kv4Tensor c, int cache_rows, int d_h, const int* rows, int M, int width, void* out,
                     hipStream_t st) {
  in_parts(M, width, [&](int i0, uint32_t pieces, uint32_t per_row, dim3 grid) {
    const int* r = rows ? rows + i0 : nullptr;
    const size_t at = static_cast<size_t>(i0) * width;
    if (dtype == 1)
      hipLaunchKernelGGL(k_kv4_load<bf16_t>, grid, dim3(256), 0, st, c, cache_rows, d_h, r, i0, pieces, per_row,
                         static_cast<bf16_t*>(out) + at);
    else
      hipLaunchKernelGGL(k_kv4_load<float>, grid, dim3(256), 0, st, c, cache_rows, d_h, r, i0, pieces, per_row, static_cast<float*>(out) + at);
  });
}

}  // namespace dllmc
