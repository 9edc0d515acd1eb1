// 4-bit cache tensors as kernels see them, and which cached keys of a sequence there are.
#pragma once

#include "common.hpp"

namespace dllmc {

// codes [H][rows][d_h / 2], scales [H][rows][d_h / 32]
struct Kv4Tensor {
  uint8_t* codes;
  uint8_t* scales;
};
inline size_t kv4_code_bytes(int cache_rows, int H, int d_h) {
  return (static_cast<size_t>(cache_rows) * H * (d_h / 2) + 255) / 256 * 256;
}
inline size_t kv4_bytes(int cache_rows, int H, int d_h) {
  return kv4_code_bytes(cache_rows, H, d_h) + static_cast<size_t>(cache_rows) * H * (d_h / 32);
}
inline Kv4Tensor kv4_tensor(const void* p, int cache_rows, int H, int d_h) {
  uint8_t* codes = static_cast<uint8_t*>(const_cast<void*>(p));
  return Kv4Tensor{codes, codes + kv4_code_bytes(cache_rows, H, d_h)};
}

// A cache tensor of one of the formats: `rows` is [cache_rows][H][d_h] of the model dtype, or `kv4`.
struct CacheView {
  const void* rows;
  Kv4Tensor kv4;
  int cache_rows, H;
};

// Which keys a sequence has: position j < min(lens[b], n) whose cache row, row_map[b * n + j] or b * n + j, lies in the cache.
struct Keys {
  const int* lens;
  const int* row_map;
  int n, cache_rows;
  __device__ __forceinline__ int length(int b) const { return lens ? max(0, min(lens[b], n)) : n; }
  // cache row of position j < n, negative if it is not there
  __device__ __forceinline__ int row(int b, int j) const {
    const int r = row_map ? row_map[static_cast<size_t>(b) * n + j] : b * n + j;
    return static_cast<unsigned>(r) < static_cast<unsigned>(cache_rows) ? r : -1;
  }
};

// Workgroups are handed to the 8 XCDs round-robin and each XCD has its own L2: the i-th of `all` workgroups takes the item below, such
// that the `group` items that follow each other and read the same memory run on one XCD.  A bijection for any `all`, a multiple of
// `group`; groups beyond the last multiple of 8 go as they come.
__device__ __forceinline__ int xcd_group_item(int i, int all, int group) {
  const int n8 = all / group & ~7;
  if (group == 1 || i >= n8 * group) return i;
  const int idx = i >> 3;
  return (idx / group * 8 + (i & 7)) * group + idx % group;
}

// sum over the 16 lanes of a row of lanes, in all of them
__device__ __forceinline__ float row16_sum(float v) {
  v += dpp_xor1(v);
  v += dpp_xor2(v);
  v += dpp_half_mirror(v);
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, false));  // (lane 15 - l of the 16)
}

// Maximum and sum over lanes l, l ^ 16, l ^ 32, l ^ 48, in all of them: two exchanges of rows of lanes between registers, no trip through LDS.
template <typename F> __device__ __forceinline__ float over_groups(float v, F&& f) {
  typedef uint32_t pair_t __attribute__((ext_vector_type(2)));
  uint32_t u = __float_as_uint(v);
  const pair_t a = __builtin_bit_cast(pair_t, __builtin_amdgcn_permlane16_swap(u, u, false, false));
  u = __float_as_uint(f(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const pair_t b = __builtin_bit_cast(pair_t, __builtin_amdgcn_permlane32_swap(u, u, false, false));
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float groups_max(float v) {
  return over_groups(v, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float groups_sum(float v) {
  return over_groups(v, [](float a, float b) { return a + b; });
}

// Scale byte of a block whose largest magnitude has the bits `top`: 127 + the smallest e with top <= 6 * 2^e = 1.5 * 2^(e + 2), so
// that nothing saturates; at least 2 (no value below 2^-126), at most 252 (6 * 2^125 is finite: above it values do saturate).
__device__ __forceinline__ uint32_t kv4_scale_byte(uint32_t top) {
  if (top >= 0x7f800000u) return 255;
  const int e = static_cast<int>(top >> 23) - 2 + ((top & 0x7fffffu) > 0x400000u ? 1 : 0);
  return static_cast<uint32_t>(max(2, min(252, e)));
}

// eight codes times 2^(scale - 127), exact; NaN for scale 255 (the conversion takes the exponent bits of its scale)
__device__ __forceinline__ bf16x8 kv4_expand(uint32_t w, uint32_t scale) {
  typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
  const float s = __uint_as_float(scale << 23);
  const uint4 r = make_uint4(__builtin_bit_cast(uint32_t, bf16x2_t(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 0))),
                             __builtin_bit_cast(uint32_t, bf16x2_t(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 1))),
                             __builtin_bit_cast(uint32_t, bf16x2_t(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 2))),
                             __builtin_bit_cast(uint32_t, bf16x2_t(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, 3))));
  return __builtin_bit_cast(bf16x8, r);
}

// eight neighbouring elements of a 16-byte aligned row as float32
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

// ---- 8-bit rows
// Rows below this largest magnitude count as zeros: 127 times its reciprocal stays finite.
constexpr float kTiny = 1.17549435e-38f * 256.f;

struct RowScale {
  float f, scale;  // q = rint(x * f)
  bool finite;
};
__device__ __forceinline__ RowScale row_scale(uint32_t top) {
  const float m = __uint_as_float(top);
  const bool finite = top < 0x7f800000u, some = finite && m >= kTiny;
  return {some ? 127.f * (1.f / m) : 0.f, !finite ? __uint_as_float(0x7fc00000u) : some ? m / 127.f : 0.f, finite};
}
template <int NW> __device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, static_cast<uint32_t>(__shfl_xor(static_cast<int>(v), o, 64)));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = v;
  __syncthreads();
  v = red[0];
#pragma unroll
  for (int w = 1; w < NW; ++w) v = max(v, red[w]);
  return v;
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

template <typename T> struct Parts;  // bf16 parts of a query element and of a probability
template <> struct Parts<bf16_t> { static constexpr int kQ = 1, kP = 2; };
template <> struct Parts<float> { static constexpr int kQ = 3, kP = 3; };

// Eight query elements as bf16 parts: x = part 0 + part 1 + part 2, each what is left rounded (what rounds to an infinity leaves NaN).
__device__ __forceinline__ void load_query(const bf16_t* p, bf16x8 (&f)[1]) {
  f[0] = *reinterpret_cast<const bf16x8*>(p);
}
__device__ __forceinline__ void split_query(const uint4& lo, const uint4& hi, bf16x8 (&f)[3]) {
  float x[8] = {__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w),
                __uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w)};
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    uint32_t w[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      w[t] = pack_bf16x2(x[2 * t], x[2 * t + 1]);
      x[2 * t] -= __uint_as_float(w[t] << 16);
      x[2 * t + 1] -= __uint_as_float(w[t] & 0xffff0000u);
    }
    f[u] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
  }
}
__device__ __forceinline__ void load_query(const float* p, bf16x8 (&f)[3]) {
  split_query(reinterpret_cast<const uint4*>(p)[0], reinterpret_cast<const uint4*>(p)[1], f);
}

void launch_kv4_store(int dtype, const void* x, int M, int width, const int* rows, Kv4Tensor c, int cache_rows, int d_h,
                      hipStream_t st);
void launch_kv4_load(int dtype, Kv4Tensor c, int cache_rows, int d_h, const int* rows, int M, int width, void* out,
                     hipStream_t st);

// A plan is a function of sizes alone; the thread's last one is kept with its sizes, which a model's layers ask for again and again
// (attention's takes 1.2 us to choose, a tenth of a short call).
template <typename Plan, int N, typename F> inline Plan last_plan(const int (&sizes)[N], F&& choose) {
  thread_local int of[N];  // (zeros: no valid sizes)
  thread_local Plan plan;
  bool same = true;
  for (int i = 0; i < N; ++i) same &= of[i] == sizes[i];
  if (!same) {
    plan = choose();
    for (int i = 0; i < N; ++i) of[i] = sizes[i];
  }
  return plan;
}

// Attention over a 4-bit cache, and the weights that cached positions get; scratch as large as the functions say.
// rows of an item (16, 32: few; 128, 256: tile), wavefronts, and how many items are not cut
struct AttendPlan { int rows, waves, tiles, whole, KS, per; long long items; };
AttendPlan plan_attend(int dtype, int B, int Mq, int n, int H_q, int H_kv, int d_h);
size_t attention_kv4_scratch_bytes(const AttendPlan& p, int d_h);
void launch_attention_kv4(const AttendPlan& p, int dtype, const void* q, int Mq, const CacheView& k, const CacheView& v, const Keys& keys,
                          int H_q, int H_kv, int d_h, void* out, float* lse, void* scratch, hipStream_t st);
struct WeighShape {
  int Mq, H_q, H_kv, G, NR;  // NR = Mq * G rows of a KV head
  int tiles, KS, per;        // stats: tiles of 16 QB rows, key ranges, 32-key blocks per range
  int blocks, RS, share;     // columns: workgroups of 64 KB keys per head, row shares, stages (brief: 16-row tiles) per share
};
struct WeighPlan { int QB, KB; bool brief; WeighShape s; };
WeighPlan plan_weigh(int dtype, int format, int B, int Mq, int n, int H_q, int H_kv, int d_h);
size_t attention_weights_scratch_bytes(const WeighPlan& p, int B, int Mq, int n, int H_q, int H_kv);
void launch_attention_weights(const WeighPlan& p, int dtype, int format, const void* q, int B, int Mq, const CacheView& k, const Keys& keys,
                              int H_q, int H_kv, int d_h, const float* lse, const float* acc_in, float* acc_out, void* scratch,
                              hipStream_t st);

// Which positions stay (kernels_evict.hip), and rows moved: dst row i = src row rows[i] for i < M where that is one.
void launch_evict(const float* acc, int B, const Keys& keys, int keep, int first, int last, int* kept, int* kept_rows,
                  int* new_lens, float* acc_out, hipStream_t st);
void launch_compact(int format, const int* rows, int M, int src_rows, int dst_rows, int H, int d_h, const void* k_src, void* k_dst,
                    const void* v_src, void* v_dst, hipStream_t st);

// 8-bit rows of K rounded up to 128 bytes (kernels_i8.hip)
inline size_t i8_row_bytes(int K) { return (static_cast<size_t>(K) + 127) / 128 * 128; }
void launch_quant8(int dtype, const void* x, int x_rows, const int* rows, int M, int K, int8_t* q, float* scale, hipStream_t st);
struct I8Plan { int wide, bm, bn, S, per; };  // wide: tile kernel; else ring of bm x bn and S slices of `per` bytes
I8Plan plan_i8(int M, int N, int Kp);
size_t linear_i8_scratch_bytes(const I8Plan& p, int M, int N);
void launch_linear_i8(const I8Plan& p, int dtype, const int8_t* a, const float* a_scale, int M, const int8_t* w, const float* w_scale,
                      int N, int K, void* out, void* scratch, hipStream_t st);

}  // namespace dllmc
