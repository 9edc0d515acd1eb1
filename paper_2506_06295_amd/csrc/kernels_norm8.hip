// A sublayer's output added to the residual stream and the sum's RMS norm as 8- or 4-bit rows, what the maps in few bits take.
//
//   s = stream[r] + x[i], rounded to the stream's type;  h = (s * rstd) * g, rstd = 1 / sqrt(mean s^2 + eps);  h in few bits.
//
// Squares are summed in 64 bits: every finite row has a norm (squares of float32 or bf16 numbers pass float32's range), and the order in which a
// kernel adds them does not reach the codes.  Everything else is float32.
#include <cmath>

#include "mx4.hpp"

namespace dllmc {

namespace {

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
template <int NW> __device__ __forceinline__ double block_sum64(double v, double* red) {
  v = wave_sum64(v);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += red[w];
  return v;
}

// eight elements as 8-bit integers
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float f) {
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e) w[e / 4] |= (static_cast<uint32_t>(static_cast<int>(rintf(v[e] * f))) & 255u) << (e % 4 * 8);
  return make_uint2(w[0], w[1]);
}
__device__ __forceinline__ uint32_t top_of(const float (&v)[8], uint32_t top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[e]) & 0x7fffffffu);
  return top;
}
__device__ __forceinline__ void store_mx4(const float (&v)[8], int i, int t, const Mx4Tensor& mx) {
  const uint32_t byte = kv4_scale_byte(block32_top(v));
  *reinterpret_cast<uint32_t*>(mx.codes + static_cast<size_t>(i) * (mx.Kp / 2) + t / 2) = mx4_codes(v, byte);
  if (t % 32 == 0) mx.scales[mx4_scale_at(i, t, mx.Kp)] = static_cast<uint8_t>(byte);
}

// A workgroup per row.  PC > 0: the row, at most 2048 PC wide, stays in registers, PC pieces of eight elements a thread, and the gain is
// requested with it: one trip to memory.  PC = 0, wider ones: its elements are read again for the norm, from the sum where it is kept (the thread's
// own writes: the sum may have taken the stream's place).
template <typename T, typename S, bool I8, bool VEC, int PC>
__global__ __launch_bounds__(256) void k_norm_rows(NormRows n, int8_t* __restrict__ q, float* __restrict__ scale, Mx4Tensor mx) {
  __shared__ double red[4];
  __shared__ uint32_t redu[4];
  const int i = blockIdx.x, d = n.d;
  const int row = n.rows ? n.rows[i] : i;
  const int len = static_cast<unsigned>(row) < static_cast<unsigned>(n.stream_rows) ? d : 0;  // (no row: zeros, and no sum)
  const S* s = static_cast<const S*>(n.stream) + static_cast<size_t>(len ? row : 0) * d;
  const T* x = n.x ? static_cast<const T*>(n.x) + static_cast<size_t>(i) * d : nullptr;
  const T* gain = static_cast<const T*>(n.gain);
  S* sum = n.sum_out ? static_cast<S*>(n.sum_out) + static_cast<size_t>(i) * d : nullptr;
  const int Kp = I8 ? (d + 127) / 128 * 128 : mx.Kp;
  auto add = [&](float (&v)[8], const float (&y)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = roundf_to<S>(v[e] + y[e]);
  };
  double ss = 0.0;
  auto squares = [&](const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += static_cast<double>(v[e]) * v[e];
  };
  auto root = [&] {  // (an infinity or NaN makes the whole row NaN, in either form)
    ss = block_sum64<4>(ss, red);
    return ss < INFINITY ? static_cast<float>(1.0 / sqrt(ss / d + static_cast<double>(n.eps))) : NAN;
  };
  if constexpr (PC > 0) {
    float v[PC][8], y[PC][8], g[PC][8];
#pragma unroll
    for (int p = 0; p < PC; ++p) load8<VEC>(s, (p * 256 + threadIdx.x) * 8, len, v[p]);
    if (x) {
#pragma unroll
      for (int p = 0; p < PC; ++p) load8<VEC>(x, (p * 256 + threadIdx.x) * 8, len, y[p]);
    }
#pragma unroll
    for (int p = 0; p < PC; ++p) load8<VEC>(gain, (p * 256 + threadIdx.x) * 8, len, g[p]);
#pragma unroll
    for (int p = 0; p < PC; ++p) {
      if (x) add(v[p], y[p]);
      if (sum) store8<VEC>(sum, (p * 256 + threadIdx.x) * 8, len, v[p]);
      squares(v[p]);
    }
    const float rstd = root();
#pragma unroll
    for (int p = 0; p < PC; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] = v[p][e] * rstd * g[p][e];
    if constexpr (I8) {
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < PC; ++p) top = top_of(v[p], top);
      const RowScale rs = row_scale(len ? block_max<4>(top, redu) : 0);
      if (threadIdx.x == 0) scale[i] = rs.scale;
#pragma unroll
      for (int p = 0; p < PC; ++p) {
        const int t = (p * 256 + threadIdx.x) * 8;
        if (t < Kp) *reinterpret_cast<uint2*>(q + static_cast<size_t>(i) * Kp + t) = rs.finite ? codes8(v[p], rs.f) : make_uint2(0, 0);
      }
    } else {
#pragma unroll
      for (int p = 0; p < PC; ++p) {
        const int t = (p * 256 + threadIdx.x) * 8;
        if (t + 7 >= len) {  // (behind the row, where zero times a NaN or an infinity may stand)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[p][e] = t + e < len ? v[p][e] : 0.f;
        }
        if (t < Kp) store_mx4(v[p], i, t, mx);
      }
    }
  } else {
    auto total = [&](int t, float (&v)[8]) {
      load8<VEC>(s, t, len, v);
      if (x) {
        float y[8];
        load8<VEC>(x, t, len, y);
        add(v, y);
      }
    };
    for (int t = threadIdx.x * 8; t < len; t += 2048) {
      float v[8];
      total(t, v);
      if (sum) store8<VEC>(sum, t, len, v);
      squares(v);
    }
    const float rstd = root();
    auto normed = [&](int t, float (&v)[8]) {
      float g[8];
      if (sum) load8<VEC>(sum, t, len, v);
      else total(t, v);
      load8<VEC>(gain, t, len, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = t + e < len ? v[e] * rstd * g[e] : 0.f;
    };
    if constexpr (I8) {
      uint32_t top = 0;
      for (int t = threadIdx.x * 8; t < len; t += 2048) {
        float v[8];
        normed(t, v);
        top = top_of(v, top);
      }
      const RowScale rs = row_scale(block_max<4>(top, redu));
      if (threadIdx.x == 0) scale[i] = rs.scale;
      for (int t = threadIdx.x * 8; t < Kp; t += 2048) {
        float v[8];
        normed(t, v);
        *reinterpret_cast<uint2*>(q + static_cast<size_t>(i) * Kp + t) = rs.finite ? codes8(v, rs.f) : make_uint2(0, 0);
      }
    } else {
      for (int t = threadIdx.x * 8; t < Kp; t += 2048) {
        float v[8];
        normed(t, v);
        store_mx4(v, i, t, mx);
      }
    }
  }
}

template <bool I8>
void launch(int dtype, int stream_dtype, const NormRows& n, int8_t* q, float* scale, Mx4Tensor mx, hipStream_t st) {
  const uintptr_t low = reinterpret_cast<uintptr_t>(n.x) | reinterpret_cast<uintptr_t>(n.stream) | reinterpret_cast<uintptr_t>(n.gain) |
                        reinterpret_cast<uintptr_t>(n.sum_out);
  const bool vec = n.d % 8 == 0 && low % 16 == 0;
#define DLLMC_N(T, S, V, PC) hipLaunchKernelGGL((k_norm_rows<T, S, I8, V, PC>), dim3(n.M), dim3(256), 0, st, n, q, scale, mx)
#define DLLMC_NV(T, S) \
  if (!vec && n.d <= 4096) DLLMC_N(T, S, false, 2); \
  else if (!vec) DLLMC_N(T, S, false, 0); \
  else if (n.d <= 2048) DLLMC_N(T, S, true, 1); \
  else if (n.d <= 4096) DLLMC_N(T, S, true, 2); \
  else if (n.d <= 8192) DLLMC_N(T, S, true, 4); \
  else DLLMC_N(T, S, true, 0)
  if (dtype == 0) { DLLMC_NV(float, float); }
  else if (stream_dtype == 0) { DLLMC_NV(bf16_t, float); }
  else { DLLMC_NV(bf16_t, bf16_t); }
#undef DLLMC_NV
#undef DLLMC_N
}

}  // namespace

void launch_norm_quant8(int dtype, int stream_dtype, const NormRows& n, int8_t* q, float* scale, hipStream_t st) {
  launch<true>(dtype, stream_dtype, n, q, scale, Mx4Tensor{}, st);
}
void launch_norm_mx4(int dtype, int stream_dtype, const NormRows& n, Mx4Tensor out, hipStream_t st) {
  launch<false>(dtype, stream_dtype, n, nullptr, nullptr, out, st);
}

}  // namespace dllmc
