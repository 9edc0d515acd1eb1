// Matrices of 4-bit blocks: rows in and out, and their product.
//
// A block is 32 neighbouring elements of a row: codes of 4 bits (sign, and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) times one power of two, as
// in a 4-bit cache.  The scaled matrix instructions multiply codes exactly and take both blocks' powers of two along, so the only roundings of
// out[i][j] = sum_k a[i][k] w[j][k] are those of float32 sums and of the result.
#include "mx4.hpp"

namespace dllmc {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---- rows in and out --------------------------------------------------------------------------------------
// A workgroup per row; four lanes take a block.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_store(const T* __restrict__ x, int x_rows, const int* __restrict__ rows, int K, Mx4Tensor out) {
  const int i = blockIdx.x;
  const int row = rows ? rows[i] : i, len = static_cast<unsigned>(row) < static_cast<unsigned>(x_rows) ? K : 0;  // (no row: zeros)
  const T* r = x + static_cast<size_t>(len ? row : 0) * K;
  for (int t = threadIdx.x * 8; t < out.Kp; t += 2048) {
    float v[8];
    load8<VEC>(r, t, len, v);
    const uint32_t scale = kv4_scale_byte(block32_top(v));
    *reinterpret_cast<uint32_t*>(out.codes + static_cast<size_t>(i) * (out.Kp / 2) + t / 2) = mx4_codes(v, scale);
    if (t % 32 == 0) out.scales[mx4_scale_at(i, t, out.Kp)] = static_cast<uint8_t>(scale);
  }
}

template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_mx4_load(Mx4Tensor in, const int* __restrict__ rows, int K, T* __restrict__ out) {
  const int i = blockIdx.x, r = rows ? rows[i] : i;
  const bool ok = static_cast<unsigned>(r) < static_cast<unsigned>(in.rows);
  T* o = out + static_cast<size_t>(i) * K;
  for (int t = threadIdx.x * 8; t < K; t += 2048) {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (ok) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(in.codes + static_cast<size_t>(r) * (in.Kp / 2) + t / 2);
      const uint4 b = __builtin_bit_cast(uint4, kv4_expand(w, in.scales[mx4_scale_at(r, t, in.Kp)]));
      const uint32_t f[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        v[2 * h] = __uint_as_float(f[h] << 16);
        v[2 * h + 1] = __uint_as_float(f[h] & 0xffff0000u);
      }
    }
    store8<VEC>(o, t, K, v);
  }
}

// 8-bit rows back: q * scale, rounded to T
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void k_load8(const int8_t* __restrict__ q, const float* __restrict__ scale, int q_rows, int K, int Kp,
                                               const int* __restrict__ rows, T* __restrict__ out) {
  const int i = blockIdx.x, r = rows ? rows[i] : i;
  const bool ok = static_cast<unsigned>(r) < static_cast<unsigned>(q_rows);
  T* o = out + static_cast<size_t>(i) * K;
  const float s = ok ? scale[r] : 0.f;
  for (int t = threadIdx.x * 8; t < K; t += 2048) {
    const uint2 w = ok ? *reinterpret_cast<const uint2*>(q + static_cast<size_t>(r) * Kp + t) : make_uint2(0, 0);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(static_cast<int8_t>((e < 4 ? w.x : w.y) >> (e % 4 * 8))) * s;
    store8<VEC>(o, t, K, v);
  }
}

// ---- the product ------------------------------------------------------------------------------------------
// A wavefront per 32 x 32 results, operands from memory straight into registers.  The product is taken as W A^T, so that a lane holds
// four neighbouring columns of a row; lane l has row l % 32 of either operand, elements 32 (l / 32) .. + 31 of a step of 64.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_plain(Mx4Tensor a, Mx4Tensor w, T* __restrict__ out) {
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, ln = lane % 32, lg = lane / 32;
  const int M = a.rows, N = w.rows, Kp = a.Kp;
  const int nt = (N + 127) / 128;
  const int m0 = blockIdx.x / nt * 32, n0 = (blockIdx.x % nt * 4 + wave) * 32;
  if (n0 >= N) return;
  const uint8_t* ar = a.codes + static_cast<size_t>(min(m0 + ln, M - 1)) * (Kp / 2) + lg * 16;
  const uint8_t* wr = w.codes + static_cast<size_t>(min(n0 + ln, N - 1)) * (Kp / 2) + lg * 16;
  const uint32_t* as = reinterpret_cast<const uint32_t*>(a.scales) + static_cast<size_t>(m0 / 32) * (Kp / 256) * 64 + lane;
  const uint32_t* ws = reinterpret_cast<const uint32_t*>(w.scales) + static_cast<size_t>(n0 / 32) * (Kp / 256) * 64 + lane;
  f32x16 acc = {0.f};
  for (int c = 0; c < Kp / 256; ++c) {
    const int sa = static_cast<int>(as[c * 64]), sw = static_cast<int>(ws[c * 64]);
    i32x8 x[4], y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint4 u = *reinterpret_cast<const uint4*>(ar + c * 128 + j * 32), v = *reinterpret_cast<const uint4*>(wr + c * 128 + j * 32);
      x[j] = i32x8{static_cast<int>(u.x), static_cast<int>(u.y), static_cast<int>(u.z), static_cast<int>(u.w), 0, 0, 0, 0};
      y[j] = i32x8{static_cast<int>(v.x), static_cast<int>(v.y), static_cast<int>(v.z), static_cast<int>(v.w), 0, 0, 0, 0};
    }
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y[0], x[0], acc, 4, 4, 0, sw, 0, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y[1], x[1], acc, 4, 4, 1, sw, 1, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y[2], x[2], acc, 4, 4, 2, sw, 2, sa);
    acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(y[3], x[3], acc, 4, 4, 3, sw, 3, sa);
  }
  const int m = m0 + ln;
  if (m >= M) return;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int n = n0 + e / 4 * 8 + lg * 4 + e % 4;
    if (n < N) stf(out + static_cast<size_t>(m) * N + n, acc[e]);
  }
}

inline bool whole_pieces(const void* p, int K) { return K % 8 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0; }

}  // namespace

#define DLLMC_BY_TYPE(dtype, vec, CALL)      \
  do {                                       \
    if ((dtype) == 1 && (vec)) CALL(bf16_t, true);   \
    else if ((dtype) == 1) CALL(bf16_t, false);      \
    else if (vec) CALL(float, true);                 \
    else CALL(float, false);                         \
  } while (0)

void launch_quant_mx4(int dtype, const void* x, int x_rows, const int* rows, int M, int K, Mx4Tensor out, hipStream_t st) {
#define DLLMC_CALL(T, V) \
  hipLaunchKernelGGL((k_mx4_store<T, V>), dim3(M), dim3(256), 0, st, static_cast<const T*>(x), x_rows, rows, K, out)
  DLLMC_BY_TYPE(dtype, whole_pieces(x, K), DLLMC_CALL);
#undef DLLMC_CALL
}

void launch_mx4_load(int dtype, Mx4Tensor in, const int* rows, int M, int K, void* out, hipStream_t st) {
#define DLLMC_CALL(T, V) hipLaunchKernelGGL((k_mx4_load<T, V>), dim3(M), dim3(256), 0, st, in, rows, K, static_cast<T*>(out))
  DLLMC_BY_TYPE(dtype, whole_pieces(out, K), DLLMC_CALL);
#undef DLLMC_CALL
}

void launch_load8(int dtype, const int8_t* q, const float* scale, int q_rows, int K, const int* rows, int M, void* out, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
#define DLLMC_CALL(T, V) \
  hipLaunchKernelGGL((k_load8<T, V>), dim3(M), dim3(256), 0, st, q, scale, q_rows, K, Kp, rows, static_cast<T*>(out))
  DLLMC_BY_TYPE(dtype, whole_pieces(out, K), DLLMC_CALL);
#undef DLLMC_CALL
}

size_t linear_mx4_scratch_bytes(int, int, int) { return 0; }

void launch_linear_mx4(int dtype, Mx4Tensor a, Mx4Tensor w, void* out, void*, hipStream_t st) {
  const dim3 grid(((w.rows + 127) / 128) * ((a.rows + 31) / 32));
  if (dtype == 1) hipLaunchKernelGGL(k_mx4_plain<bf16_t>, grid, dim3(256), 0, st, a, w, static_cast<bf16_t*>(out));
  else hipLaunchKernelGGL(k_mx4_plain<float>, grid, dim3(256), 0, st, a, w, static_cast<float*>(out));
}

}  // namespace dllmc
