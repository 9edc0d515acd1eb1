// A sublayer's output added to the residual stream and the sum's RMS norm as 8- or 4-bit rows, what the maps in few bits take.
//
//   s = stream[r] + x[i], rounded to the stream's type;  h = (s * rstd) * g, rstd = 1 / sqrt(mean s^2 + eps);  h in few bits.
//
// Squares are summed in 64 bits: every finite row has a norm (squares of float32 or bf16 numbers pass float32's range), and the order in which a
// kernel adds them does not reach the codes.  Everything else is float32.  rstd can pass float32's range too (rows of subnormals
// with eps = 0) and fall below its normal numbers (rows near its largest): then s takes a power of two first and rstd goes without it.
//
// Bound by the bytes with many rows: x, stream, sum and codes of 12288 rows of 4096 (bf16, 8 bits) in 70.9 us, 5.0 TB/s; by two trips to memory and a
// launch with few: 64 rows 4.1 us.  (Times here: the median or best of several means of 20 launches behind one another.)
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
  if (NW == 1) return v;
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v += red[w];
  return v;
}

// Eight elements as 8-bit integers: a float32 number of at most 127 and 1.5 * 2^23 add up to the integer nearest to it, ties to even, in the low byte.
__device__ __forceinline__ uint2 codes8(const float (&v)[8], float f) {
#pragma clang fp contract(off)  // (the product is a float32 number before it is rounded to an integer)
  uint32_t b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(v[e] * f + 12582912.f);
  auto four = [](uint32_t a, uint32_t c, uint32_t d, uint32_t e) {
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(e, d, 0x0c0c0400u), __builtin_amdgcn_perm(c, a, 0x0c0c0400u), 0x05040100u);
  };
  return make_uint2(four(b[0], b[1], b[2], b[3]), four(b[4], b[5], b[6], b[7]));
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

// A workgroup of TR threads per row.  PC > 0: the row, at most 8 TR PC wide, stays in registers, PC pieces of eight elements a thread, and the
// gain is requested with it: one trip to memory.  PC = 0, wider ones: its elements are read again for the norm, from the sum where it is kept (the thread's
// own writes: the sum may have taken the stream's place).
template <typename T, typename S, bool I8, bool WHOLE, int TR, int PC>
__global__ __launch_bounds__(TR) void k_norm_rows(NormRows n, int8_t* __restrict__ q, float* __restrict__ scale, Mx4Tensor mx) {
  __shared__ double red[TR / 64];
  __shared__ uint32_t redu[TR / 64];
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
    for (int e = 0; e < 8; e += 2) {
      v[e] += y[e];
      v[e + 1] += y[e + 1];
      if (sizeof(S) == 2) {
        const uint32_t w = pack_bf16x2(v[e], v[e + 1]);
        v[e] = __uint_as_float(w << 16);
        v[e + 1] = __uint_as_float(w & 0xffff0000u);
      }
    }
  };
  double ss = 0.0;
  auto squares = [&](const float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) ss += static_cast<double>(v[e]) * v[e];
  };
  // (An infinity or NaN makes the whole row NaN, in either form; zeros with eps = 0 do as well.)
  auto root = [&] {
    ss = block_sum64<TR / 64>(ss, red);
    return ss < INFINITY ? 1.0 / sqrt(ss / d + static_cast<double>(n.eps)) : static_cast<double>(NAN);
  };
  // h = ((s * pre) * (rstd / pre)) * g, the second factor a normal float32 number.  pre = 1 but at both ends, where a root mean square lies under 2^-126
  // (rstd at most 2^157.5: one element of 2^-149 in 131072) or over 2^126 (rstd at least 2^-128).  What s * pre loses there is far
  // below what the products keep.
  auto inside = [](float rstd) { return rstd >= 0x1p-126f && rstd <= 0x1p126f; };
  auto at_an_end = [](double r, float& rstd) {
    const bool low = r < 1.0;
    rstd = static_cast<float>(r * (low ? 0x1p4 : 0x1p-32));
    return low ? 0x1p-4f : 0x1p32f;
  };
  if constexpr (PC > 0) {
    float v[PC][8], y[PC][8], g[PC][8];
#pragma unroll
    for (int p = 0; p < PC; ++p) load8<WHOLE>(s, (p * TR + threadIdx.x) * 8, len, v[p]);
    if (x) {
#pragma unroll
      for (int p = 0; p < PC; ++p) load8<WHOLE>(x, (p * TR + threadIdx.x) * 8, len, y[p]);
    }
#pragma unroll
    for (int p = 0; p < PC; ++p) load8<WHOLE>(gain, (p * TR + threadIdx.x) * 8, len, g[p]);
#pragma unroll
    for (int p = 0; p < PC; ++p) {
      if (x) add(v[p], y[p]);
      if (sum) store8<WHOLE>(sum, (p * TR + threadIdx.x) * 8, len, v[p]);
      squares(v[p]);
    }
    const double r = root();
    float rstd = static_cast<float>(r);
    if (!inside(rstd)) {
      const float pre = at_an_end(r, rstd);
#pragma unroll
      for (int p = 0; p < PC; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[p][e] *= pre;
    }
#pragma unroll
    for (int p = 0; p < PC; ++p)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] = v[p][e] * rstd * g[p][e];
    if constexpr (I8) {
      uint32_t top = 0;
#pragma unroll
      for (int p = 0; p < PC; ++p) top = top_of(v[p], top);
      const RowScale rs = row_scale(len ? block_max<TR / 64>(top, redu) : 0);
      if (threadIdx.x == 0) scale[i] = rs.scale;
#pragma unroll
      for (int p = 0; p < PC; ++p) {
        const int t = (p * TR + threadIdx.x) * 8;
        if (t < Kp) *reinterpret_cast<uint2*>(q + static_cast<size_t>(i) * Kp + t) = rs.finite ? codes8(v[p], rs.f) : make_uint2(0, 0);
      }
    } else {
#pragma unroll
      for (int p = 0; p < PC; ++p) {
        const int t = (p * TR + threadIdx.x) * 8;
        if (t + 7 >= len) {  // (behind the row, where zero times a NaN or an infinity may stand)
#pragma unroll
          for (int e = 0; e < 8; ++e) v[p][e] = t + e < len ? v[p][e] : 0.f;
        }
        if (t < Kp) store_mx4(v[p], i, t, mx);
      }
    }
  } else {
    auto total = [&](int t, float (&v)[8]) {
      load8<WHOLE>(s, t, len, v);
      if (x) {
        float y[8];
        load8<WHOLE>(x, t, len, y);
        add(v, y);
      }
    };
    for (int t = threadIdx.x * 8; t < len; t += 8 * TR) {
      float v[8];
      total(t, v);
      if (sum) store8<WHOLE>(sum, t, len, v);
      squares(v);
    }
    const double r = root();
    float rstd = static_cast<float>(r);
    const float pre = inside(rstd) ? 1.f : at_an_end(r, rstd);
    auto normed = [&](int t, float (&v)[8]) {
      float g[8];
      if (sum) load8<WHOLE>(sum, t, len, v);
      else total(t, v);
      load8<WHOLE>(gain, t, len, g);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = t + e < len ? v[e] * pre * rstd * g[e] : 0.f;
    };
    if constexpr (I8) {
      uint32_t top = 0;
      for (int t = threadIdx.x * 8; t < len; t += 8 * TR) {
        float v[8];
        normed(t, v);
        top = top_of(v, top);
      }
      const RowScale rs = row_scale(block_max<TR / 64>(top, redu));
      if (threadIdx.x == 0) scale[i] = rs.scale;
      for (int t = threadIdx.x * 8; t < Kp; t += 8 * TR) {
        float v[8];
        normed(t, v);
        *reinterpret_cast<uint2*>(q + static_cast<size_t>(i) * Kp + t) = rs.finite ? codes8(v, rs.f) : make_uint2(0, 0);
      }
    } else {
      for (int t = threadIdx.x * 8; t < Kp; t += 8 * TR) {
        float v[8];
        normed(t, v);
        store_mx4(v, i, t, mx);
      }
    }
  }
}

// Rows over 12288 are read two (4 bits) or three times (8 bits): 4096 x 18944 in bf16 117 and 139 us, their bytes 102 and 110 at 4.95 TB/s.
// Threads of a row and pieces of a thread by width.  Rows of up to 1024 go to a wavefront each, which waits for nobody (12288 x 256: 10.7 us, 23 with a
// workgroup of four per row).  2049 to 4096 wide, us for 12288 rows of 4096; 3584; 4049: a bf16 stream 70.7; 57.8; 85 with 256 threads of two pieces and
// 68.3; 62.5; 95 with 512 of one; a float32 one 105; 97; 116 and 100; 87; 119.  The bytes of 4096 wide take 71 and 112 at 4.95 TB/s, a copy of 4 GB's.
template <bool I8>
void launch(int dtype, int stream_dtype, const NormRows& n, int8_t* q, float* scale, Mx4Tensor mx, hipStream_t st) {
#define DLLMC_N(T, S, TR, PC)                                                                                                     \
  do {                                                                                                                          \
    if (n.d % 8 == 0) hipLaunchKernelGGL((k_norm_rows<T, S, I8, true, TR, PC>), dim3(n.M), dim3(TR), 0, st, n, q, scale, mx);     \
    else hipLaunchKernelGGL((k_norm_rows<T, S, I8, false, TR, PC>), dim3(n.M), dim3(TR), 0, st, n, q, scale, mx);                 \
  } while (0)
#define DLLMC_BY_WIDTH(T, S)               \
  if (n.d <= 512) DLLMC_N(T, S, 64, 1);        \
  else if (n.d <= 1024) DLLMC_N(T, S, 64, 2);  \
  else if (n.d <= 2048) DLLMC_N(T, S, 256, 1); \
  else if (n.d <= 4096) DLLMC_N(T, S, (sizeof(S) == 4 ? 512 : 256), (sizeof(S) == 4 ? 1 : 2)); \
  else if (n.d <= 8192) DLLMC_N(T, S, 512, 2); \
  else if (n.d <= 12288) DLLMC_N(T, S, 512, 3); \
  else DLLMC_N(T, S, 512, 0)
  if (dtype == 0) { DLLMC_BY_WIDTH(float, float); }
  else if (stream_dtype == 0) { DLLMC_BY_WIDTH(bf16_t, float); }
  else { DLLMC_BY_WIDTH(bf16_t, bf16_t); }
#undef DLLMC_BY_WIDTH
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
