// Attention weight of every cached position: column sums of softmax(Q K^T / sqrt(d_h)) over queries and heads.
//
// A row's probabilities need its maximum and sum before any column can be added up, so scores are formed twice: k_weigh_stats
// reduces every row over ranges of keys to (m, l), k_weigh_cols holds a block of keys in registers, walks the rows, and adds exp2(s -
// m) / l per key; k_weigh_sum adds what heads and row shares left, in their order.  Where the caller has the rows'
// log-sum-exp the first launch and its pass over the keys fall away.  No value is read and no probability leaves a register.
#include <type_traits>

#include "kv4.hpp"

namespace dllmc {

namespace {

// Key operand of 16 keys of a head: as loaded, and as the matrix cores take it.  at(): first element of contraction piece c, eight
// elements (four in float32) a lane; queries are loaded in the same deal.
template <typename F, typename T, int D> struct KeyOperand;
template <typename T, int D> struct KeyOperand<Kv4Tensor, T, D> {
  static constexpr int kC = D / 32, kQ = Parts<T>::kQ;
  struct Raw { uint32_t w[kC], s; };
  typedef bf16x8 Frag[kC];
  typedef bf16x8 Query[kC][kQ];
  static __device__ __forceinline__ int at(int lg, int c) { return lg * (D / 4) + 8 * c; }
  static __device__ __forceinline__ void load(const CacheView& v, int h, int row, int lg, Raw& r) {
    const size_t i = static_cast<size_t>(h) * v.cache_rows + row;
    const uint8_t* p = v.kv4.codes + i * (D / 2) + lg * (D / 8);
    if constexpr (D == 64) {
      const uint2 w = *reinterpret_cast<const uint2*>(p);
      r.w[0] = w.x; r.w[1] = w.y;
    } else {
#pragma unroll
      for (int t = 0; t < D / 128; ++t) {
        const uint4 w = reinterpret_cast<const uint4*>(p)[t];
        r.w[4 * t] = w.x; r.w[4 * t + 1] = w.y; r.w[4 * t + 2] = w.z; r.w[4 * t + 3] = w.w;
      }
    }
    const uint8_t* q = v.kv4.scales + i * (D / 32);
    r.s = D == 64 ? q[lg / 2] : D == 128 ? q[lg] : reinterpret_cast<const uint16_t*>(q)[lg];
  }
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = kv4_expand(r.w[c], D == 256 ? (r.s >> (c / 4 * 8)) & 255u : r.s);
  }
  static __device__ __forceinline__ void query(const T* row, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) load_query(row + at(lg, c), q[c]);
  }
  static __device__ __forceinline__ f32x4 scores(const Frag& k, const Query& q) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int u = kQ - 1; u >= 0; --u)
#pragma unroll
      for (int c = 0; c < kC; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c], q[c][u], s, 0, 0, 0);
    return s;
  }
};
template <int D> struct KeyOperand<bf16_t, bf16_t, D> {
  static constexpr int kC = D / 32;
  struct Raw { bf16x8 w[kC]; };
  typedef bf16x8 Frag[kC];
  typedef bf16x8 Query[kC];
  static __device__ __forceinline__ int at(int lg, int c) { return 32 * c + 8 * lg; }
  static __device__ __forceinline__ void load(const CacheView& v, int h, int row, int lg, Raw& r) {
    const bf16_t* p = static_cast<const bf16_t*>(v.rows) + (static_cast<size_t>(row) * v.H + h) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) r.w[c] = *reinterpret_cast<const bf16x8*>(p + at(lg, c));
  }
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = r.w[c];
  }
  static __device__ __forceinline__ void query(const bf16_t* row, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) q[c] = *reinterpret_cast<const bf16x8*>(row + at(lg, c));
  }
  static __device__ __forceinline__ f32x4 scores(const Frag& k, const Query& q) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kC; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c], q[c], s, 0, 0, 0);
    return s;
  }
};
template <int D> struct KeyOperand<float, float, D> {
  static constexpr int kC = D / 16;
  struct Raw { f32x4 w[kC]; };
  typedef f32x4 Frag[kC];
  typedef f32x4 Query[kC];
  static __device__ __forceinline__ int at(int lg, int c) { return 16 * c + 4 * lg; }
  static __device__ __forceinline__ void load(const CacheView& v, int h, int row, int lg, Raw& r) {
    const float* p = static_cast<const float*>(v.rows) + (static_cast<size_t>(row) * v.H + h) * D;
#pragma unroll
    for (int c = 0; c < kC; ++c) r.w[c] = *reinterpret_cast<const f32x4*>(p + at(lg, c));
  }
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = r.w[c];
  }
  static __device__ __forceinline__ void query(const float* row, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) q[c] = *reinterpret_cast<const f32x4*>(row + at(lg, c));
  }
  static __device__ __forceinline__ f32x4 scores(const Frag& k, const Query& q) {
    f32x4 s0 = f32x4{0.f, 0.f, 0.f, 0.f}, s1 = s0;  // (two chains: an instruction may not wait for its predecessor)
#pragma unroll
    for (int c = 0; c < kC; c += 2)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c][e], q[c][e], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(k[c + 1][e], q[c + 1][e], s1, 0, 0, 0);
      }
    return s0 + s1;
  }
};

struct WeighShape {
  int Mq, H_q, H_kv, G, NR;  // NR = Mq * G rows of a KV head
  int tiles, KS, per;        // stats: tiles of 16 QB rows, key ranges, 32-key blocks per range
  int blocks, RS, share;     // columns: workgroups of 64 KB keys per head, row shares, 16-row tiles per share
};
__device__ __forceinline__ size_t row_of(const WeighShape& s, int b, int h, int r) {
  const int i = s.G == 1 ? r : r / s.G;
  return (static_cast<size_t>(b) * s.Mq + i) * s.H_q + h * s.G + (r - i * s.G);
}

// (m, l) of 16 QB rows over a range of keys, base 2; the wavefronts deal the range's blocks of 32 keys, the next one in flight.
template <typename F, typename T, int D, int QB>
__global__ __launch_bounds__(256, D == 256 ? (sizeof(T) == 4 ? 1 : 2) : QB == 1 && sizeof(T) == 2 ? 3 : 2) void k_weigh_stats(const T* __restrict__ q, WeighShape s, CacheView k, Keys keys,
                                                                     float2* __restrict__ ml) {
  typedef KeyOperand<F, T, D> Op;
  __shared__ float2 hand[4][16 * QB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  int x = blockIdx.x;
  const int tile = x % s.tiles; x /= s.tiles;
  const int range = x % s.KS; x /= s.KS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const int len = keys.length(b), r0 = tile * 16 * QB;
  const int nblk = (len + 31) / 32, blk1 = min(nblk, (range + 1) * s.per);
  int blk = range * s.per + wave;
  const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
  float m[QB], l[QB];
#pragma unroll
  for (int i = 0; i < QB; ++i) { m[i] = -INFINITY; l[i] = 0.f; }
  struct Block { typename Op::Raw k[2]; uint32_t there; };
  auto rows_of = [&](int blk_, int (&r)[2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const int j = blk_ * 32 + t * 16 + ln;
      r[t] = j < len ? keys.row(b, j) : -1;
    }
  };
  auto fetch = [&](const int (&r)[2], Block& kb) {
    kb.there = static_cast<uint32_t>(__ballot(r[0] >= 0) & 0xffffu) | static_cast<uint32_t>(__ballot(r[1] >= 0) & 0xffffu) << 16;
#pragma unroll
    for (int t = 0; t < 2; ++t) Op::load(k, h, max(r[t], 0), lg, kb.k[t]);
  };
  if (blk < blk1) {
    typename Op::Query qf[QB];
    auto use = [&](const Block& kb) {
      if (kb.there == 0) return;
      f32x4 st[2][QB];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        typename Op::Frag f;
        Op::expand(kb.k[t], f);
#pragma unroll
        for (int i = 0; i < QB; ++i) st[t][i] = Op::scores(f, qf[i]);
      }
      if (kb.there != 0xffffffffu) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (((kb.there >> (t * 16 + 4 * lg + e)) & 1) == 0) {
#pragma unroll
              for (int i = 0; i < QB; ++i) st[t][i][e] = -INFINITY;
            }
      }
      // (every lane has a maximum and sum of its own quarter of the keys, joined at the end)
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        float mx = st[0][i][0];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, st[t][i][e]);
        const float top = fmaxf(m[i], mx * sl2e), u = top == -INFINITY ? 0.f : top;
        float sum = l[i] * __builtin_amdgcn_exp2f(m[i] - u);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(fmaf(st[t][i][e], sl2e, -u));
        l[i] = sum;
        m[i] = top;
      }
    };
    Block b0, b1;
    int r[2];
    rows_of(blk, r);
    fetch(r, b0);
    rows_of(min(blk + 4, blk1 - 1), r);
#pragma unroll
    for (int i = 0; i < QB; ++i) Op::query(q + row_of(s, b, h, min(r0 + i * 16 + ln, s.NR - 1)) * D, lg, qf[i]);
    for (; blk + 4 < blk1; blk += 8) {
      fetch(r, b1);
      rows_of(min(blk + 8, blk1 - 1), r);
      use(b0);
      fetch(r, b0);
      rows_of(min(blk + 12, blk1 - 1), r);
      use(b1);
    }
    if (blk < blk1) use(b0);
  }
  auto join = [](float2 a, float2 c) {  // (sums may be NaN beside a maximum of minus infinity)
    const float M = fmaxf(a.x, c.x), u = M == -INFINITY ? 0.f : M;
    const float fa = a.y != a.y ? 1.f : __builtin_amdgcn_exp2f(a.x - u), fc = c.y != c.y ? 1.f : __builtin_amdgcn_exp2f(c.x - u);
    return make_float2(M, a.y * fa + c.y * fc);
  };
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    float2 v = make_float2(m[i], l[i]);
    v = join(v, make_float2(__shfl_xor(v.x, 16, 64), __shfl_xor(v.y, 16, 64)));
    v = join(v, make_float2(__shfl_xor(v.x, 32, 64), __shfl_xor(v.y, 32, 64)));
    if (lg == 0) hand[wave][i * 16 + ln] = v;
  }
  __syncthreads();
  if (threadIdx.x < 16 * QB && r0 + static_cast<int>(threadIdx.x) < s.NR) {
    float2 v = hand[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < 4; ++w) v = join(v, hand[w][threadIdx.x]);
    ml[row_of(s, b, h, r0 + threadIdx.x) * s.KS + range] = v;
  }
}

// Column sums: a wavefront holds 16 KB keys of one KV head and walks its share of the head's rows, 16 at a time, the next 16 in
// flight.  part[(share * B + b) * H_kv + h][n].
template <typename F, typename T, int D, int KB>
__global__ __launch_bounds__(256, D == 256 && sizeof(T) == 4 ? 1 : 2) void k_weigh_cols(const T* __restrict__ q, WeighShape s, CacheView k, Keys keys,
                                                       const float* __restrict__ lse, const float2* __restrict__ ml,
                                                       float* __restrict__ part) {
  typedef KeyOperand<F, T, D> Op;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  int x = blockIdx.x;
  const int blk = x % s.blocks; x /= s.blocks;
  const int share = x % s.RS; x /= s.RS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const int key0 = (blk * 4 + wave) * 16 * KB, len = keys.length(b);
  const int B = gridDim.x / (s.blocks * s.RS * s.H_kv);
  if (key0 >= keys.n) return;
  float* out = part + (static_cast<size_t>(share * B + b) * s.H_kv + h) * keys.n;
  f32x4 sum[KB];
#pragma unroll
  for (int t = 0; t < KB; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t there[KB];
  if (key0 < len) {
    typename Op::Frag kf[KB];
    {
      int r[KB];
      typename Op::Raw raw[KB];
#pragma unroll
      for (int t = 0; t < KB; ++t) r[t] = key0 + t * 16 + ln < len ? keys.row(b, key0 + t * 16 + ln) : -1;
#pragma unroll
      for (int t = 0; t < KB; ++t) {
        there[t] = static_cast<uint32_t>(__ballot(r[t] >= 0));
        Op::load(k, h, max(r[t], 0), lg, raw[t]);
      }
#pragma unroll
      for (int t = 0; t < KB; ++t) Op::expand(raw[t], kf[t]);
    }
    const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
    const int t1 = min((s.NR + 15) / 16, (share + 1) * s.share);
    struct Rows { typename Op::Query q; float z; };
    auto fetch = [&](int t, Rows& v) {
      const int r = t * 16 + ln;
      const size_t w = row_of(s, b, h, min(r, s.NR - 1));
      Op::query(q + w * D, lg, v.q);
      if (lse != nullptr) {
        v.z = lse[w] * kLog2e;
      } else {  // the ranges' (m, l), a quarter of them per group of lanes
        float m = -INFINITY, l = 0.f;
        for (int i = lg; i < s.KS; i += 4) {
          const float2 c = ml[w * s.KS + i];
          const float M = fmaxf(m, c.x), u = M == -INFINITY ? 0.f : M;
          l = l * __builtin_amdgcn_exp2f(m - u) + (c.y != c.y ? c.y : c.y * __builtin_amdgcn_exp2f(c.x - u));
          m = M;
        }
#pragma unroll
        for (int o = 16; o < 64; o <<= 1) {
          const float m2 = __shfl_xor(m, o, 64), l2 = __shfl_xor(l, o, 64), M = fmaxf(m, m2), u = M == -INFINITY ? 0.f : M;
          const float f1 = __builtin_amdgcn_exp2f(m - u), f2 = __builtin_amdgcn_exp2f(m2 - u);
          l = (l != l ? l : l * f1) + (l2 != l2 ? l2 : l2 * f2);
          m = M;
        }
        v.z = m + __builtin_amdgcn_logf(l);  // (base 2)
      }
      if (r >= s.NR) v.z = INFINITY;  // rows past the last one weigh nothing
    };
    auto use = [&](const Rows& v) {
#pragma unroll
      for (int t = 0; t < KB; ++t) {
        const f32x4 st = Op::scores(kf[t], v.q);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[t][e] += __builtin_amdgcn_exp2f(fmaf(st[e], sl2e, -v.z));
      }
    };
    int t = share * s.share;
    if (t < t1) {
      Rows v0, v1;
      fetch(t, v0);
      for (; t + 1 < t1; t += 2) {
        fetch(t + 1, v1);
        use(v0);
        fetch(min(t + 2, t1 - 1), v0);
        use(v1);
      }
      if (t < t1) use(v0);
    }
  } else {
#pragma unroll
    for (int t = 0; t < KB; ++t) there[t] = 0;
  }
#pragma unroll
  for (int t = 0; t < KB; ++t) {
#pragma unroll
    for (int o = 1; o < 16; o <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[t][e] += __shfl_xor(sum[t][e], o, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = key0 + t * 16 + 4 * lg + e;
      if (ln == 0 && j < keys.n) out[j] = (there[t] >> (4 * lg + e)) & 1 ? sum[t][e] : 0.f;
    }
  }
}

// acc_out[b][j] = acc_in[b][j] + the parts of all shares and heads, 16 wavefronts that take every 16th of them
__global__ __launch_bounds__(1024) void k_weigh_sum(const float* __restrict__ part, int shares, int B, int H, int n,
                                                    const float* __restrict__ acc_in, float* __restrict__ acc_out) {
  __shared__ float red[16][64];
  const int per = (n + 63) / 64, b = blockIdx.x / per, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int j = blockIdx.x % per * 64 + lane;
  float sum = 0.f;
  if (j < n)
    for (int p = wave; p < shares * H; p += 16) sum += part[(static_cast<size_t>(p / H * B + b) * H + p % H) * n + j];
  red[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || j >= n) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += red[w][lane];
  const size_t at = static_cast<size_t>(b) * n + j;
  acc_out[at] = (acc_in != nullptr ? acc_in[at] : 0.f) + sum;
}

struct WeighPlan { int QB, KB; WeighShape s; };
WeighPlan plan_weigh(int dtype, int format, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  WeighPlan p{};
  WeighShape& s = p.s;
  s.Mq = Mq; s.H_q = H_q; s.H_kv = H_kv; s.G = H_q / H_kv; s.NR = Mq * s.G;
  p.QB = s.NR <= 16 || dtype == 0 || d_h == 256 ? 1 : s.NR <= 32 ? 2 : 4;
  s.tiles = (s.NR + 16 * p.QB - 1) / (16 * p.QB);
  const int nblk = (n + 31) / 32;
  const long long items = static_cast<long long>(B) * H_kv * s.tiles;
  long long KS = items >= 512 ? 1 : 512 / items;
  const int most = (nblk + 7) / 8;
  KS = KS > most ? most : KS;
  KS = KS > 64 ? 64 : KS < 1 ? 1 : KS;
  s.per = static_cast<int>((nblk + KS - 1) / KS);
  s.KS = (nblk + s.per - 1) / s.per;
  p.KB = (format == 0 || d_h == 256) ? 2 : 4;
  s.blocks = (n + 64 * p.KB - 1) / (64 * p.KB);
  const int rt = (s.NR + 15) / 16;
  const long long groups = static_cast<long long>(B) * H_kv * s.blocks;
  long long RS = groups >= 512 ? 1 : 512 / groups;
  if (RS > rt) RS = rt;
  s.share = static_cast<int>((rt + RS - 1) / RS);
  s.RS = (rt + s.share - 1) / s.share;
  return p;
}

}  // namespace

size_t attention_weights_scratch_bytes(int dtype, int format, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  const WeighShape s = plan_weigh(dtype, format, B, Mq, n, H_q, H_kv, d_h).s;
  return static_cast<size_t>(B) * Mq * H_q * s.KS * sizeof(float2) + static_cast<size_t>(s.RS) * B * H_kv * n * sizeof(float);
}

void launch_attention_weights(int dtype, int format, const void* q, int B, int Mq, const CacheView& k, const Keys& keys, int H_q,
                              int H_kv, int d_h, const float* lse, const float* acc_in, float* acc_out, void* scratch,
                              hipStream_t st) {
  const WeighPlan p = plan_weigh(dtype, format, B, Mq, keys.n, H_q, H_kv, d_h);
  const WeighShape& s = p.s;
  float2* ml = static_cast<float2*>(scratch);
  float* part = reinterpret_cast<float*>(ml + static_cast<size_t>(B) * Mq * H_q * s.KS);
  const dim3 rows(static_cast<unsigned>(static_cast<long long>(B) * H_kv * s.tiles * s.KS));
  const dim3 cols(static_cast<unsigned>(static_cast<long long>(B) * H_kv * s.blocks * s.RS));
  auto go = [&](auto f, auto t, auto d) {
    typedef decltype(f) F;
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    const T* qt = static_cast<const T*>(q);
    if (lse == nullptr) {
      if constexpr (sizeof(T) == 4 || D == 256) {
        hipLaunchKernelGGL((k_weigh_stats<F, T, D, 1>), rows, dim3(256), 0, st, qt, s, k, keys, ml);
      } else {
        if (p.QB == 1) hipLaunchKernelGGL((k_weigh_stats<F, T, D, 1>), rows, dim3(256), 0, st, qt, s, k, keys, ml);
        else if (p.QB == 2) hipLaunchKernelGGL((k_weigh_stats<F, T, D, 2>), rows, dim3(256), 0, st, qt, s, k, keys, ml);
        else hipLaunchKernelGGL((k_weigh_stats<F, T, D, 4>), rows, dim3(256), 0, st, qt, s, k, keys, ml);
      }
    }
    constexpr int KB = std::is_same<F, float>::value || D == 256 ? 2 : 4;
    hipLaunchKernelGGL((k_weigh_cols<F, T, D, KB>), cols, dim3(256), 0, st, qt, s, k, keys, lse, ml, part);
  };
  auto with_d = [&](auto f, auto t) {
    if (d_h == 64) go(f, t, std::integral_constant<int, 64>{});
    else if (d_h == 128) go(f, t, std::integral_constant<int, 128>{});
    else go(f, t, std::integral_constant<int, 256>{});
  };
  if (format == 2) {
    if (dtype == 1) with_d(Kv4Tensor(), bf16_t());
    else with_d(Kv4Tensor(), float());
  } else if (dtype == 1) {
    with_d(bf16_t(), bf16_t());
  } else {
    with_d(float(), float());
  }
  hipLaunchKernelGGL(k_weigh_sum, dim3(static_cast<unsigned>(B * ((keys.n + 63) / 64))), dim3(1024), 0, st, part, s.RS, B, H_kv, keys.n,
                     acc_in, acc_out);
}

}  // namespace dllmc
