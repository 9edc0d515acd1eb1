// Linear maps in 8-bit integers: rows quantised with a scale each, integer products on the matrix cores, scales of row and
// column multiplied in at the end.
#include "kv4.hpp"

namespace dllmc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Rows below this largest magnitude count as zeros: 127 / it stays finite.
constexpr float kTiny = 1.17549435e-38f * 256.f;

// q = rint(x * (127 / max|x|)), scale = max|x| / 127; one workgroup per row.  A row with an infinity or NaN gets the scale NaN.
template <typename T>
__global__ __launch_bounds__(256) void k_quant8(const T* __restrict__ x, const int* __restrict__ rows, int K, int Kp,
                                                int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const int i = blockIdx.x;
  const T* r = x + static_cast<size_t>(rows ? rows[i] : i) * K;
  uint32_t top = 0;
  for (int t = threadIdx.x; t < K; t += 256) top = max(top, __float_as_uint(ldf(r + t)) & 0x7fffffffu);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), o, 64)));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = top;
  __syncthreads();
  top = max(max(red[0], red[1]), max(red[2], red[3]));
  const float m = __uint_as_float(top);
  const bool finite = top < 0x7f800000u;
  const float f = finite && m >= kTiny ? 127.f / m : 0.f;
  if (threadIdx.x == 0) scale[i] = !finite ? __uint_as_float(0x7fc00000u) : m >= kTiny ? m / 127.f : 0.f;
  int8_t* o = q + static_cast<size_t>(i) * Kp;
  for (int t = threadIdx.x; t < Kp; t += 256) o[t] = static_cast<int8_t>(finite && t < K ? static_cast<int>(rintf(ldf(r + t) * f)) : 0);
}

// a wavefront per 16 x 16 results, operands from memory
template <typename T>
__global__ __launch_bounds__(64) void k_i8_simple(const int8_t* __restrict__ a, const float* __restrict__ sa, int M,
                                                  const int8_t* __restrict__ w, const float* __restrict__ sw, int N, int Kp,
                                                  T* __restrict__ out) {
  const int ln = threadIdx.x % 16, lg = threadIdx.x / 16;
  const int m0 = blockIdx.y * 16, n0 = blockIdx.x * 16;
  const int8_t* ar = a + static_cast<size_t>(min(m0 + ln, M - 1)) * Kp + lg * 16;
  const int8_t* wr = w + static_cast<size_t>(min(n0 + ln, N - 1)) * Kp + lg * 16;
  i32x4 acc = {0, 0, 0, 0};
  for (int k = 0; k < Kp; k += 64)
    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4*>(ar + k), *reinterpret_cast<const i32x4*>(wr + k), acc, 0,
                                                0, 0);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int m = m0 + lg * 4 + e, n = n0 + ln;
    if (m < M && n < N) stf(out + static_cast<size_t>(m) * N + n, static_cast<float>(acc[e]) * sa[m] * sw[n]);
  }
}

}  // namespace

void launch_quant8(int dtype, const void* x, const int* rows, int M, int K, int8_t* q, float* scale, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
  if (dtype == 1)
    hipLaunchKernelGGL(k_quant8<bf16_t>, dim3(M), dim3(256), 0, st, static_cast<const bf16_t*>(x), rows, K, Kp, q, scale);
  else
    hipLaunchKernelGGL(k_quant8<float>, dim3(M), dim3(256), 0, st, static_cast<const float*>(x), rows, K, Kp, q, scale);
}

size_t linear_i8_scratch_bytes(int, int, int) { return 0; }

void launch_linear_i8(int dtype, const int8_t* a, const float* a_scale, int M, const int8_t* w, const float* w_scale, int N, int K,
                      void* out, void*, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
  const dim3 grid((N + 15) / 16, (M + 15) / 16);
  if (dtype == 1)
    hipLaunchKernelGGL(k_i8_simple<bf16_t>, grid, dim3(64), 0, st, a, a_scale, M, w, w_scale, N, Kp, static_cast<bf16_t*>(out));
  else
    hipLaunchKernelGGL(k_i8_simple<float>, grid, dim3(64), 0, st, a, a_scale, M, w, w_scale, N, Kp, static_cast<float*>(out));
}

}  // namespace dllmc
