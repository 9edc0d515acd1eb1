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
template <typename T> struct Eight;
template <> struct Eight<float> {
  static __device__ __forceinline__ void load(const float* p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
};
template <> struct Eight<bf16_t> {
  static __device__ __forceinline__ void load(const bf16_t* p, float (&x)[8]) {
    const uint4 a = *reinterpret_cast<const uint4*>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      x[2 * t] = __uint_as_float(w[t] << 16);
      x[2 * t + 1] = __uint_as_float(w[t] & 0xffff0000u);
    }
  }
};

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

// ---- attention, one wavefront per query and head --------------------------------------------------------
// Scores twice: once for the maximum and the sum, once for the probabilities of 64 keys at a time.
template <typename T, typename C>
__device__ __forceinline__ float score(const float* qs, const CacheView& c, int h, int row, int d_h) {
  float s = 0.f;
  for (int t = 0; t < d_h; ++t) s = fmaf(qs[t], cache_at<C>(c, h, row, t, d_h), s);
  return s;
}

template <typename T, typename C>
__global__ __launch_bounds__(64) void k_attend_simple(const T* __restrict__ q, int Mq, CacheView kc, CacheView vc, Keys keys,
                                                      int H_q, int H_kv, int d_h, T* __restrict__ out, float* __restrict__ lse) {
  extern __shared__ float sm[];
  float* qs = sm;
  float* ps = sm + d_h;
  const int lane = threadIdx.x;
  const long long w = blockIdx.x;
  const int a = static_cast<int>(w % H_q), i = static_cast<int>(w / H_q % Mq), b = static_cast<int>(w / H_q / Mq);
  const int h = a / (H_q / H_kv), len = keys.length(b);
  const T* qr = q + w * d_h;
  const float scale = 1.0f / sqrtf(static_cast<float>(d_h));
  for (int t = lane; t < d_h; t += 64) qs[t] = ldf(qr + t) * scale;
  __syncthreads();
  float m = -INFINITY, l = 0.f;
  for (int j = lane; j < len; j += 64) {
    const int row = keys.row(b, j);
    if (row < 0) continue;
    const float s = score<T, C>(qs, kc, h, row, d_h), top = fmaxf(m, s);
    const float u = top == -INFINITY ? 0.f : top;
    l = l * expf(m - u) + expf(s - u);
    m = top;
  }
  const float M = wave_max(m), U = M == -INFINITY ? 0.f : M;
  const float L = wave_sum(l * expf(m - U));
  if (lse != nullptr && lane == 0) lse[w] = M + logf(L);
  if (out == nullptr) return;
  float o[4] = {0.f, 0.f, 0.f, 0.f};
  for (int j0 = 0; j0 < len; j0 += 64) {
    const int j = j0 + lane, mine = j < len ? keys.row(b, j) : -1;
    __syncthreads();
    ps[lane] = mine >= 0 ? expf(score<T, C>(qs, kc, h, mine, d_h) - U) : 0.f;
    __syncthreads();
    for (int e = 0; e < 64 && j0 + e < len; ++e) {
      const int row = keys.row(b, j0 + e);
      if (row < 0) continue;
#pragma unroll
      for (int t = 0; t < 4; ++t)
        if (lane + 64 * t < d_h) o[t] = fmaf(ps[e], cache_at<C>(vc, h, row, lane + 64 * t, d_h), o[t]);
    }
  }
#pragma unroll
  for (int t = 0; t < 4; ++t)
    if (lane + 64 * t < d_h) stf(out + w * d_h + lane + 64 * t, L == 0.f ? 0.f : o[t] / L);
  (void)i;
}

// acc_out[b][j] = acc_in[b][j] + sum over queries and heads of exp(s - lse): a wavefront takes 64 keys
template <typename T, typename C>
__global__ __launch_bounds__(64) void k_weigh_simple(const T* __restrict__ q, int Mq, CacheView kc, Keys keys, int H_q, int H_kv,
                                                     int d_h, const float* __restrict__ lse, const float* __restrict__ acc_in,
                                                     float* __restrict__ acc_out) {
  extern __shared__ float sm[];
  const int tiles = (keys.n + 63) / 64, lane = threadIdx.x;
  const int b = blockIdx.x / tiles, j = blockIdx.x % tiles * 64 + lane;
  const int row = j < keys.length(b) ? keys.row(b, j) : -1;
  const float scale = 1.0f / sqrtf(static_cast<float>(d_h));
  float sum = 0.f;
  for (int r = 0; r < Mq * H_q; ++r) {
    const long long w = static_cast<long long>(b) * Mq * H_q + r;
    __syncthreads();
    for (int t = lane; t < d_h; t += 64) sm[t] = ldf(q + w * d_h + t) * scale;
    __syncthreads();
    if (row >= 0) sum += expf(score<T, C>(sm, kc, r % H_q / (H_q / H_kv), row, d_h) - lse[w]);
  }
  if (j < keys.n) {
    const size_t at = static_cast<size_t>(b) * keys.n + j;
    acc_out[at] = (acc_in ? acc_in[at] : 0.f) + sum;
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

size_t attention_weights_scratch_bytes(int, int, int B, int Mq, int, int H_q, int, int) {
  return static_cast<size_t>(B) * Mq * H_q * sizeof(float);
}

void launch_attention_weights(int dtype, int format, const void* q, int B, int Mq, const CacheView& k, const Keys& keys, int H_q,
                              int H_kv, int d_h, const float* lse, const float* acc_in, float* acc_out, void* scratch,
                              hipStream_t st) {
  const dim3 rows(static_cast<unsigned>(static_cast<long long>(B) * Mq * H_q)), tiles(B * ((keys.n + 63) / 64));
  const size_t lds = (d_h + 64) * sizeof(float);
  float* own = static_cast<float*>(scratch);
  auto go = [&](auto t, auto c) {
    typedef decltype(t) T;
    typedef decltype(c) C;
    if (lse == nullptr)
      hipLaunchKernelGGL((k_attend_simple<T, C>), rows, dim3(64), lds, st, static_cast<const T*>(q), Mq, k, k, keys, H_q, H_kv, d_h,
                         static_cast<T*>(nullptr), own);
    hipLaunchKernelGGL((k_weigh_simple<T, C>), tiles, dim3(64), lds, st, static_cast<const T*>(q), Mq, k, keys, H_q, H_kv, d_h,
                       lse ? lse : own, acc_in, acc_out);
  };
  if (format == 2) {
    if (dtype == 1) go(bf16_t(), Kv4Tensor());
    else go(float(), Kv4Tensor());
  } else if (dtype == 1) {
    go(bf16_t(), bf16_t());
  } else {
    go(float(), float());
  }
}

}  // namespace dllmc
