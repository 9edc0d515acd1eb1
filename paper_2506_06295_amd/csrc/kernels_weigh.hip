// Attention weight of every cached position: column sums of softmax(Q K^T / sqrt(d_h)) over queries and heads.
//
// A row's probabilities need its maximum and sum before any column can be added up.  Up to 1024 keys k_weigh_short holds a head's
// keys in the registers of one workgroup and forms every score once.  Beyond, scores are formed twice: k_weigh_stats reduces every row over
// ranges of keys to (m, l), k_weigh_join joins those, and k_weigh_cols holds a block of keys in registers, walks the rows and
// adds exp2(s - m) / l per key (exp2(s - m - log2 l) would round an exponent of 10 to 2^-21); where the caller has the rows'
// log-sum-exp, the first two and their pass over the keys fall away.  k_weigh_sum adds what heads and row shares left, in their order.
// No value is read and no probability leaves a register.
#include <type_traits>

#include "kv4.hpp"

namespace dllmc {

namespace {

// Key operand of 16 keys of a head: as loaded, and as the matrix cores take it.  at(): first element of contraction piece c, eight
// elements (four in float32) a lane; queries are read in the same deal.  A row is kCh pieces of 16 bytes, of which lane (ln, lg) wants
// chunk(lg, i) of row ln.  Read like that from global memory, neighbouring lanes have different rows and a CU takes in 16 bytes a
// cycle; read along the rows (load_keys16) and turned in LDS (turn_keys16), 64: 768 keys of 128 in bf16 by a CU 6.7 and 3.0 us.  A key
// in 4 bits is 64 bytes, and turning it costs the instructions that it saves: 4608 rows x 4608 keys x 32 heads 264 us as it is, 277 turned.
template <typename F, typename T, int D> struct KeyOperand;
template <typename T, int D> struct KeyOperand<Kv4Tensor, T, D> {
  static constexpr int kC = D / 32, kQ = Parts<T>::kQ, kCh = D / 32;
  static constexpr bool kAlong = false;
  struct Raw { uint4 w[(kC + 3) / 4]; uint32_t s; };
  typedef bf16x8 Frag[kC];
  typedef bf16x8 Query[kC][kQ];
  static __device__ __forceinline__ int at(int lg, int c) { return lg * (D / 4) + 8 * c; }
  static __device__ __forceinline__ const uint4* row(const CacheView& v, int h, int row) {
    // (a head's codes end below 2^24 * 128 bytes: a scalar base and a 32-bit offset)
    return reinterpret_cast<const uint4*>(v.kv4.codes + static_cast<size_t>(h) * v.cache_rows * (D / 2) + static_cast<uint32_t>(row) * (D / 2));
  }
  // what does not come along the rows
  static __device__ __forceinline__ void load(const CacheView& v, int h, int row_, int lg, Raw& r) {
    if constexpr (D == 64) {
      const uint2 w = reinterpret_cast<const uint2*>(row(v, h, row_))[lg];
      r.w[0].x = w.x; r.w[0].y = w.y;
    } else {
#pragma unroll
      for (int t = 0; t < kC / 4; ++t) r.w[t] = row(v, h, row_)[lg * (kC / 4) + t];
    }
    const uint8_t* q = v.kv4.scales + static_cast<size_t>(h) * v.cache_rows * (D / 32);
    const uint32_t at = static_cast<uint32_t>(row_) * (D / 32);
    r.s = D == 64 ? q[at + lg / 2] : D == 128 ? q[at + lg] : *reinterpret_cast<const uint16_t*>(q + (at + 2 * lg));
  }
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      const uint4 w = r.w[c / 4];
      f[c] = kv4_expand(c % 4 == 0 ? w.x : c % 4 == 1 ? w.y : c % 4 == 2 ? w.z : w.w, D == 256 ? (r.s >> (c / 4 * 8)) & 255u : r.s);
    }
  }
  template <typename P> static __device__ __forceinline__ void query_pieces(P&& piece, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) {
      if constexpr (sizeof(T) == 2) q[c][0] = __builtin_bit_cast(bf16x8, piece(at(lg, c) / 8));
      else split_query(piece(at(lg, c) / 4), piece(at(lg, c) / 4 + 1), q[c]);
    }
  }
  static __device__ __forceinline__ f32x4 scores(const Frag& k, const Query& q) {
    f32x4 s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[0], q[0][kQ - 1], f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
    for (int u = kQ - 1; u >= 0; --u)
#pragma unroll
      for (int c = u == kQ - 1 ? 1 : 0; c < kC; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c], q[c][u], s, 0, 0, 0);
    return s;
  }
};
template <int D> struct KeyOperand<bf16_t, bf16_t, D> {
  static constexpr int kC = D / 32, kCh = 4 * kC;
  static constexpr bool kAlong = true;
  struct Raw { uint4 w[kC]; };
  typedef bf16x8 Frag[kC];
  typedef bf16x8 Query[kC];
  static __device__ __forceinline__ int at(int lg, int c) { return 32 * c + 8 * lg; }
  static __device__ __forceinline__ int chunk(int lg, int i) { return 4 * i + lg; }
  static __device__ __forceinline__ const uint4* row(const CacheView& v, int h, int row) {
    return reinterpret_cast<const uint4*>(static_cast<const bf16_t*>(v.rows) + (static_cast<size_t>(row) * v.H + h) * D);
  }
  static __device__ __forceinline__ void load(const CacheView&, int, int, int, Raw&) {}
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = __builtin_bit_cast(bf16x8, r.w[c]);
  }
  template <typename P> static __device__ __forceinline__ void query_pieces(P&& piece, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) q[c] = __builtin_bit_cast(bf16x8, piece(at(lg, c) / 8));
  }
  static __device__ __forceinline__ f32x4 scores(const Frag& k, const Query& q) {
    f32x4 s = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < kC; ++c) s = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c], q[c], s, 0, 0, 0);
    return s;
  }
};
template <int D> struct KeyOperand<float, float, D> {
  static constexpr int kC = D / 16, kCh = 4 * kC;
  static constexpr bool kAlong = true;
  struct Raw { uint4 w[kC]; };
  typedef f32x4 Frag[kC];
  typedef f32x4 Query[kC];
  static __device__ __forceinline__ int at(int lg, int c) { return 16 * c + 4 * lg; }
  static __device__ __forceinline__ int chunk(int lg, int i) { return 4 * i + lg; }
  static __device__ __forceinline__ const uint4* row(const CacheView& v, int h, int row) {
    return reinterpret_cast<const uint4*>(static_cast<const float*>(v.rows) + (static_cast<size_t>(row) * v.H + h) * D);
  }
  static __device__ __forceinline__ void load(const CacheView&, int, int, int, Raw&) {}
  static __device__ __forceinline__ void expand(const Raw& r, Frag& f) {
#pragma unroll
    for (int c = 0; c < kC; ++c) f[c] = __builtin_bit_cast(f32x4, r.w[c]);
  }
  template <typename P> static __device__ __forceinline__ void query_pieces(P&& piece, int lg, Query& q) {
#pragma unroll
    for (int c = 0; c < kC; ++c) q[c] = __builtin_bit_cast(f32x4, piece(at(lg, c) / 4));
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

__device__ __forceinline__ size_t row_of(const WeighShape& s, int b, int h, int r) {
  const int i = s.G == 1 ? r : r / s.G;
  return (static_cast<size_t>(b) * s.Mq + i) * s.H_q + h * s.G + (r - i * s.G);
}

// Cache rows of the N keys key0, key0 + 16, .., negative where there is none.  (the lookups are made for keys in range whether they
// are there or not: none waits for a branch)
template <int N> __device__ __forceinline__ void key_rows(const Keys& keys, int b, int key0, int len, int (&r)[N]) {
  int at[N];
#pragma unroll
  for (int t = 0; t < N; ++t) at[t] = min(key0 + t * 16, keys.n - 1);
  if (keys.row_map != nullptr) {
    const int* map = keys.row_map + static_cast<size_t>(b) * keys.n;
#pragma unroll
    for (int t = 0; t < N; ++t) r[t] = map[at[t]];
  } else {
#pragma unroll
    for (int t = 0; t < N; ++t) r[t] = b * keys.n + at[t];
  }
#pragma unroll
  for (int t = 0; t < N; ++t)
    if (key0 + t * 16 >= len || static_cast<unsigned>(r[t]) >= static_cast<unsigned>(keys.cache_rows)) r[t] = -1;
}

// ROWS query rows for all NW wavefronts of a workgroup, loaded along the rows into LDS (in a fragment's order by every wavefront for itself,
// 64 rows of 128 in bf16 by eight of them would keep a CU's address unit for 3.9 us).
template <typename T, int D, int ROWS, int NW> struct QueryTile {
  static constexpr int kCh = D * static_cast<int>(sizeof(T)) / 16, kMix = kCh < 16 ? kCh : 16, kVecs = ROWS * kCh;
  // row(r): address of row r.  Wait for the loads and for each other before piece().
  template <typename Row> static __device__ __forceinline__ void issue(Row&& row, uint4* lds, int wave, int lane) {
#pragma unroll
    for (int j = 0; j < (kVecs / 64 + NW - 1) / NW; ++j) {
      const int i = wave + j * NW;
      if (i >= kVecs / 64) break;
      const int v = i * 64 + lane, r = v / kCh, c = (v % kCh) ^ (r % kMix);
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(row(r)) + c, &lds[i * 64], 16, 0, 0);
    }
  }
  // 16 bytes c of row r
  static __device__ __forceinline__ uint4 piece(const uint4* lds, int r, int c) { return lds[r * kCh + (c ^ (r % kMix))]; }
};

constexpr float kLowest = -3.4028234663852886e38f;

// 16 keys of a head; lane ln (and ln + 16, ..) names the cache row of key ln
template <typename Op> struct KeyTurn {
  static constexpr int kWide = Op::kCh < 32 ? Op::kCh : 32, kVecs = Op::kAlong ? 16 * kWide : 0;  // a wavefront's 16-byte slots of LDS
  static __device__ __forceinline__ int mix(int r) { return r % (kWide < 16 ? kWide : 16); }
};
template <typename Op> __device__ __forceinline__ void load_keys16(const CacheView& v, int h, int row, int lane, typename Op::Raw& raw) {
  constexpr int W = KeyTurn<Op>::kWide;
  if constexpr (Op::kAlong) {
#pragma unroll
    for (int u = 0; u < Op::kCh / W; ++u)
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const int x = i * 64 + lane;
        raw.w[u * (W / 4) + i] = Op::row(v, h, __shfl(row, x / W, 64))[u * W + x % W];
      }
  }
  Op::load(v, h, row, lane / 16, raw);
}
// (`lds` is the wavefront's own, and the LDS keeps a wavefront's order by itself)
template <typename Op> __device__ __forceinline__ void turn_keys16(typename Op::Raw& raw, uint4* lds, int lane) {
  typedef KeyTurn<Op> K;
  constexpr int W = K::kWide;
  if constexpr (Op::kAlong) {
#pragma unroll
    for (int u = 0; u < Op::kCh / W; ++u) {
#pragma unroll
      for (int i = 0; i < W / 4; ++i) {
        const int x = i * 64 + lane, r = x / W;
        lds[r * W + ((x % W) ^ K::mix(r))] = raw.w[u * (W / 4) + i];
      }
      asm volatile("" ::: "memory");
#pragma unroll
      for (int i = 0; i < W / 4; ++i)
        raw.w[u * (W / 4) + i] = lds[lane % 16 * W + ((Op::chunk(lane / 16, u * (W / 4) + i) - u * W) ^ K::mix(lane % 16))];
      asm volatile("" ::: "memory");
    }
  }
}

// 1 / l of a row; 0 where the sum is empty (no key, or every score minus infinity): such a row weighs nothing
__device__ __forceinline__ float reciprocal(float l) { return l == 0.f ? 0.f : 1.f / l; }

// (m, l) of 16 QB rows over a range of keys, base 2, or m and 1 / l where the range is all of them; the eight wavefronts deal the range's blocks
// of 32 keys, the next one in flight.  Bound by vector instructions: 4.6 a score, one per 6 cycles with two wavefronts per SIMD (an
// exponential 12); with four of them, queries read from LDS again for every block, the same.  512 rows x 4608 keys x 32 heads in 4 bits
// 33 us, 4608 rows 264, of which the products alone would take 129.  512 rows x 4608 keys x 32 heads, all launches, us (with the log-sum-exp given):
// bf16 cache 78 (45), 4 bits 65 (33); float32 queries over 4 bits 119 (66), over float32 402 (180; 146 a pass at the float32 matrix rate).
constexpr int kSW = 8;
template <typename F, typename T, int D, int QB>
__global__ __launch_bounds__(64 * kSW) __attribute__((amdgpu_waves_per_eu(2))) void k_weigh_stats(const T* __restrict__ q, WeighShape s, CacheView k,
                                                                                            Keys keys, float2* __restrict__ ml,
                                                                                            float* __restrict__ m_out,
                                                                                            float* __restrict__ il_out) {
  typedef KeyOperand<F, T, D> Op;
  typedef QueryTile<T, D, 16 * QB, kSW> Rows;
  __shared__ float2 hand[kSW][16 * QB];
  __shared__ __attribute__((aligned(1024))) uint4 lds[Rows::kVecs + kSW * KeyTurn<Op>::kVecs];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  int x = xcd_group_item(blockIdx.x, gridDim.x, s.tiles);  // tiles of one head and range read the same keys
  const int tile = x % s.tiles; x /= s.tiles;
  const int range = x % s.KS; x /= s.KS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const int len = keys.length(b), r0 = tile * 16 * QB;
  const int nblk = (len + 31) / 32, blk1 = min(nblk, (range + 1) * s.per);
  int blk = range * s.per + wave;
  const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
  float m[QB], ref[QB], l[QB];  // l: sum of exp2(sl2e s - ref)
#pragma unroll
  for (int i = 0; i < QB; ++i) { m[i] = -INFINITY; ref[i] = kLowest; l[i] = 0.f; }
  struct Block { typename Op::Raw k[2]; uint32_t there; };
  auto rows_of = [&](int blk_, int (&r)[2]) { key_rows(keys, b, blk_ * 32 + ln, len, r); };
  auto fetch = [&](const int (&r)[2], Block& kb) {
    kb.there = static_cast<uint32_t>(__ballot(r[0] >= 0) & 0xffffu) | static_cast<uint32_t>(__ballot(r[1] >= 0) & 0xffffu) << 16;
#pragma unroll
    for (int t = 0; t < 2; ++t) load_keys16<Op>(k, h, max(r[t], 0), lane, kb.k[t]);
  };
  Rows::issue([&](int r) { return q + row_of(s, b, h, min(r0 + r, s.NR - 1)) * D; }, lds, wave, lane);
  Block b0, b1;
  int r[2];
  if (blk < blk1) {
    rows_of(blk, r);
    fetch(r, b0);
    rows_of(min(blk + kSW, blk1 - 1), r);
  }
  wait_vmcnt_lds<0>();
  __syncthreads();
  if (blk < blk1) {
    typename Op::Query qf[QB];
#pragma unroll
    for (int i = 0; i < QB; ++i) Op::query_pieces([&](int c) { return Rows::piece(lds, i * 16 + ln, c); }, lg, qf[i]);
    auto use = [&](Block& kb) {
      if (kb.there == 0) return;
      f32x4 st[2][QB];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        typename Op::Frag f;
        turn_keys16<Op>(kb.k[t], lds + Rows::kVecs + wave * KeyTurn<Op>::kVecs, lane);
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
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) m[i] = fmaxf(m[i], st[t][i][e]);
        const float u = fmaxf(m[i] * sl2e, kLowest);  // finite: no key, no NaN
        float sum = l[i] * __builtin_amdgcn_exp2f(ref[i] - u);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) sum += __builtin_amdgcn_exp2f(fmaf(st[t][i][e], sl2e, -u));
        l[i] = sum;
        ref[i] = u;
      }
    };
    if constexpr (sizeof(typename Op::Raw) >= 256) {  // (two of them do not fit in the registers)
      while (true) {
        use(b0);
        blk += kSW;
        if (blk >= blk1) break;
        fetch(r, b0);
        rows_of(min(blk + kSW, blk1 - 1), r);
      }
      blk = blk1;
    }
    for (; blk + kSW < blk1; blk += 2 * kSW) {
      fetch(r, b1);
      rows_of(min(blk + 2 * kSW, blk1 - 1), r);
      use(b0);
      fetch(r, b0);
      rows_of(min(blk + 3 * kSW, blk1 - 1), r);
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
    float2 v = make_float2(m[i] * sl2e, l[i]);
    v = join(v, make_float2(__shfl_xor(v.x, 16, 64), __shfl_xor(v.y, 16, 64)));
    v = join(v, make_float2(__shfl_xor(v.x, 32, 64), __shfl_xor(v.y, 32, 64)));
    if (lg == 0) hand[wave][i * 16 + ln] = v;
  }
  __syncthreads();
  if (threadIdx.x < 16 * QB && r0 + static_cast<int>(threadIdx.x) < s.NR) {
    float2 v = hand[0][threadIdx.x];
#pragma unroll
    for (int w = 1; w < kSW; ++w) v = join(v, hand[w][threadIdx.x]);
    const size_t w = row_of(s, b, h, r0 + threadIdx.x);
    if (s.KS == 1) {
      m_out[w] = v.x;
      il_out[w] = reciprocal(v.y);
    } else {
      ml[w * s.KS + range] = v;
    }
  }
}

// m and 1 / l over the ranges, one thread per row
__global__ __launch_bounds__(256) void k_weigh_join(const float2* __restrict__ ml, int KS, int rows, float* __restrict__ m_out,
                                                    float* __restrict__ il_out) {
  const int w = blockIdx.x * 256 + threadIdx.x;
  if (w >= rows) return;
  float m = -INFINITY, l = 0.f;
  for (int i = 0; i < KS; ++i) {
    const float2 c = ml[static_cast<size_t>(w) * KS + i];
    const float M = fmaxf(m, c.x), u = M == -INFINITY ? 0.f : M;
    l = (l != l ? l : l * __builtin_amdgcn_exp2f(m - u)) + (c.y != c.y ? c.y : c.y * __builtin_amdgcn_exp2f(c.x - u));
    m = M;
  }
  m_out[w] = m;
  il_out[w] = reciprocal(l);
}

// 16 KB column sums of a wavefront leave for part[j], zero where there is no key; `there`: keys of each 16
template <int KB>
__device__ __forceinline__ void store_columns(f32x4 (&sum)[KB], const uint32_t (&there)[KB], int key0, int n, int ln, int lg, float* out) {
#pragma unroll
  for (int t = 0; t < KB; ++t) {
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[t][e] = row16_sum(sum[t][e]);
    // lane ln < 4 of each 16 takes key 4 lg + ln
    const float v = ln == 0 ? sum[t][0] : ln == 1 ? sum[t][1] : ln == 2 ? sum[t][2] : sum[t][3];
    const int j = key0 + t * 16 + 4 * lg + ln;
    if (ln < 4 && j < n) out[j] = (there[t] >> (4 * lg + ln)) & 1 ? v : 0.f;
  }
}
template <typename Op, int KB>
__device__ __forceinline__ void load_keys(const CacheView& k, const Keys& keys, int b, int h, int key0, int len, int lane, uint4* lds,
                                          typename Op::Frag (&f)[KB], uint32_t (&there)[KB]) {
  const int ln = lane % 16;
  int r[KB];
  typename Op::Raw raw[KB];
  key_rows(keys, b, key0 + ln, len, r);
#pragma unroll
  for (int t = 0; t < KB; ++t) {
    there[t] = static_cast<uint32_t>(__ballot(r[t] >= 0));  // (lanes 0 .. 15: the keys)
    load_keys16<Op>(k, h, max(r[t], 0), lane, raw[t]);  // what is not there: row 0, counts for nothing
  }
#pragma unroll
  for (int t = 0; t < KB; ++t) {
    turn_keys16<Op>(raw[t], lds, lane);
    Op::expand(raw[t], f[t]);
  }
}

// Column sums: a wavefront holds 16 KB keys of one KV head and walks its share of the head's rows; rows come in stages of 8 KB (16
// rows at least) through a ring in LDS that the four wavefronts share, with their m and 1 / l (lse: mul * m, no l).  part[(share * B + b) * H_kv + h][n].
// With every wavefront fetching its rows by itself, 16 ahead, a launch of 512 rows x 4608 keys x 32 heads waited on trips to the L2: 60 us.
template <typename T, int D> struct WeighStage {
  static constexpr int kRow = D * static_cast<int>(sizeof(T)), kRows = kRow >= 512 ? 16 : 8192 / kRow;
  static constexpr int kVecs = kRows * kRow / 16, kLoads = kVecs / 256, kStages = 4;
};
template <typename F, typename T, int D, int KB>
__device__ __forceinline__ void weigh_cols_body(const T* __restrict__ q, const WeighShape& s, const CacheView& k, const Keys& keys,
                                                const float* __restrict__ m, const float* __restrict__ il, float mul,
                                                float* __restrict__ part) {
  typedef KeyOperand<F, T, D> Op;
  typedef WeighStage<T, D> St;
  constexpr int kIssued = St::kLoads + 2;
  constexpr int NS = St::kStages, kChunks = St::kRow / 16, kMix = kChunks < 16 ? kChunks : 16;
  __shared__ __attribute__((aligned(1024))) uint4 lds[NS * St::kVecs + NS * 4 * 32 + 4 * KeyTurn<Op>::kVecs];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  int x = xcd_group_item(blockIdx.x, gridDim.x, s.blocks);  // key blocks of one head and share read the same rows
  const int blk = x % s.blocks; x /= s.blocks;
  const int share = x % s.RS; x /= s.RS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const int key0 = (blk * 4 + wave) * 16 * KB, len = keys.length(b);
  const int B = gridDim.x / (s.blocks * s.RS * s.H_kv);
  float* out = part + (static_cast<size_t>(share * B + b) * s.H_kv + h) * keys.n;
  const int t0 = share * s.share, t1 = min((s.NR + St::kRows - 1) / St::kRows, t0 + s.share);

  // loader: instruction j of a stage copies 1 KB, wavefront w issues kLoads w .. + kLoads - 1 and its own copy of m and 1 / l.  Rows
  // are walked, not computed: at[] is the row of q (of this sequence) of the next stage, g[] its head in the group, a stage further
  // is kRows / G queries and kRows % G heads (rows past the last one: the last one)
  const float* second = il != nullptr ? il : m;
  const size_t seq = static_cast<size_t>(b) * s.Mq * s.H_q;
  const T* qb = q + seq * D;
  const float *mb = m + seq, *sb = second + seq;
  const int over = St::kRows % s.G, step = St::kRows / s.G * s.H_q + over, last = (s.Mq - 1) * s.H_q + h * s.G + s.G - 1;
  int at[St::kLoads + 1], g[St::kLoads + 1];
#pragma unroll
  for (int j = 0; j <= St::kLoads; ++j) {
    const int r = t0 * St::kRows + (j < St::kLoads ? ((wave * St::kLoads + j) * 64 + lane) / kChunks : lane % St::kRows);
    g[j] = r % s.G;
    at[j] = r / s.G * s.H_q + h * s.G + g[j];
  }
  auto issue = [&](int slot) {
#pragma unroll
    for (int j = 0; j < St::kLoads; ++j) {
      const int v = (wave * St::kLoads + j) * 64 + lane, c = (v % kChunks) ^ (v / kChunks % kMix);
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(qb) + (static_cast<size_t>(min(at[j], last)) * kChunks + c),
                                       &lds[slot * St::kVecs + (wave * St::kLoads + j) * 64], 16, 0, 0);
    }
    const int w = min(at[St::kLoads], last);
    __builtin_amdgcn_global_load_lds(mb + w, &lds[NS * St::kVecs + (slot * 4 + wave) * 32], 4, 0, 0);
    __builtin_amdgcn_global_load_lds(sb + w, &lds[NS * St::kVecs + (slot * 4 + wave) * 32 + 16], 4, 0, 0);
#pragma unroll
    for (int j = 0; j <= St::kLoads; ++j) {
      const int next = g[j] + over;
      const bool wrap = next >= s.G;
      g[j] = wrap ? next - s.G : next;
      at[j] += wrap ? step + s.H_q - s.G : step;
    }
  };
#pragma unroll
  for (int t = 0; t < NS - 1; ++t)
    if (t0 + t < t1) issue(t);
  f32x4 sum[KB];
  uint32_t there[KB];
  typename Op::Frag kf[KB];
#pragma unroll
  for (int t = 0; t < KB; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  load_keys<Op, KB>(k, keys, b, h, key0, len, lane, lds + NS * (St::kVecs + 4 * 32) + wave * KeyTurn<Op>::kVecs, kf, there);
  const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
  int slot = 0;
  for (int t = t0; t < t1; ++t) {
    const int rem = t1 - 1 - t;
    if (rem >= NS - 2) wait_vmcnt_lds<(NS - 2) * kIssued>();
    else if (rem == 1) wait_vmcnt_lds<kIssued>();
    else wait_vmcnt_lds<0>();
    __builtin_amdgcn_s_barrier();  // stage t is there for everybody, and everybody has read stage t - 1, which is filled next
    if (t + NS - 1 < t1) issue(slot == 0 ? NS - 1 : slot - 1);
    if (key0 < len) {
#pragma unroll
      for (int g = 0; g < St::kRows / 16; ++g) {
        const int r = g * 16 + ln;
        const float* row = reinterpret_cast<const float*>(&lds[NS * St::kVecs + (slot * 4 + wave) * 32]) + r;
        float mr = row[0] * mul;
        const float ir = il != nullptr ? row[64] : 1.f;
        // rows past the last one weigh nothing, nor do those whose every score is minus infinity (which minus itself would be NaN)
        if (t * St::kRows + r >= s.NR || mr == -INFINITY) mr = INFINITY;
        typename Op::Query qf;
        Op::query_pieces([&](int c) { return lds[slot * St::kVecs + r * kChunks + (c ^ (r % kMix))]; }, lg, qf);
#pragma unroll
        for (int u = 0; u < KB; ++u) {
          const f32x4 st = Op::scores(kf[u], qf);
#pragma unroll
          for (int e = 0; e < 4; ++e) sum[u][e] = fmaf(__builtin_amdgcn_exp2f(fmaf(st[e], sl2e, -mr)), ir, sum[u][e]);
        }
      }
    }
    slot = slot + 1 < NS ? slot + 1 : 0;
  }
  if (key0 < keys.n) store_columns<KB>(sum, there, key0, keys.n, ln, lg, out);
}
template <typename F, typename T, int D, int KB>
__global__ __launch_bounds__(256, D == 256 && sizeof(T) == 4 ? 1 : 2) void k_weigh_cols(const T* __restrict__ q, WeighShape s, CacheView k,
                                                                                 Keys keys, const float* __restrict__ m,
                                                                                 const float* __restrict__ il, float mul,
                                                                                 float* __restrict__ part) {
  weigh_cols_body<F, T, D, KB>(q, s, k, keys, m, il, mul, part);
}

// Up to 128 KB keys: the eight wavefronts of a workgroup hold them all, 16 KB each, and walk a share of the head's rows 16 at a time.
// Scores stay in registers while the wavefronts exchange their maxima and sums; no second pass.  Bound by a wavefront's instructions:
// KB follows the keys in steps of two (768 keys by eight wavefronts of 96 11.1 us with the sum, by six of 128 12.7, of 64 rows x 32 heads).
template <typename F, typename T, int D, int KB>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void k_weigh_short(const T* __restrict__ q, WeighShape s, CacheView k,
                                                                                         Keys keys, float* __restrict__ part) {
  typedef KeyOperand<F, T, D> Op;
  typedef QueryTile<T, D, 16, 8> Rows;
  __shared__ float2 ml[2][8][16];
  __shared__ __attribute__((aligned(1024))) uint4 lds[2 * Rows::kVecs + 8 * KeyTurn<Op>::kVecs];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  int x = xcd_group_item(blockIdx.x, gridDim.x, s.RS);  // shares of one head read the same keys
  const int share = x % s.RS; x /= s.RS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const int key0 = wave * 16 * KB, len = keys.length(b);
  const int B = gridDim.x / (s.RS * s.H_kv);
  f32x4 sum[KB];
  uint32_t there[KB];
  typename Op::Frag kf[KB];
  typename Op::Query qf;
  const int t0 = share * s.share, t1 = min((s.NR + 15) / 16, t0 + s.share);
  auto issue = [&](int t) {
    Rows::issue([&](int r) { return q + row_of(s, b, h, min(t * 16 + r, s.NR - 1)) * D; }, lds + (t & 1) * Rows::kVecs, wave, lane);
  };
  issue(t0);
#pragma unroll
  for (int t = 0; t < KB; ++t) sum[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  load_keys<Op, KB>(k, keys, b, h, key0, len, lane, lds + 2 * Rows::kVecs + wave * KeyTurn<Op>::kVecs, kf, there);
  uint32_t mine = 0;  // bit 4 t + e: this lane's key e of the 16 t-th is there
#pragma unroll
  for (int t = 0; t < KB; ++t) mine |= ((there[t] >> (4 * lg)) & 15u) << (4 * t);
  bool all = true;  // wavefront-uniform
#pragma unroll
  for (int t = 0; t < KB; ++t) all &= (there[t] & 0xffffu) == 0xffffu;
  const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
  wait_vmcnt_lds<0>();
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    if (t + 1 < t1) issue(t + 1);  // (all have read tile t - 1: they have met since)
    Op::query_pieces([&](int c) { return Rows::piece(lds + (t & 1) * Rows::kVecs, ln, c); }, lg, qf);
    f32x4 st[KB];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int u = 0; u < KB; ++u) st[u] = Op::scores(kf[u], qf);
    if (!all) {
#pragma unroll
      for (int u = 0; u < KB; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (((mine >> (4 * u + e)) & 1) == 0) st[u][e] = -INFINITY;
    }
#pragma unroll
    for (int u = 0; u < KB; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) m = fmaxf(m, st[u][e]);
    m = groups_max(m) * sl2e;
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < KB; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        st[u][e] = __builtin_amdgcn_exp2f(fmaf(st[u][e], sl2e, -ref));
        l += st[u][e];
      }
    l = groups_sum(l);
    if (lg == 0) ml[t & 1][wave][ln] = make_float2(m, l);
    wait_vmcnt_lds<0>();
    __syncthreads();
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < 8; ++w) M = fmaxf(M, ml[t & 1][w][ln].x);
#pragma unroll
    for (int w = 0; w < 8; ++w) {  // (a sum may be NaN beside a maximum of minus infinity)
      const float2 c = ml[t & 1][w][ln];
      L += c.y != c.y ? c.y : c.x == -INFINITY ? 0.f : c.y * __builtin_amdgcn_exp2f(c.x - M);
    }
    // what this wavefront's exponentials are short of; nothing for rows past the last one (they repeat it: where they are NaN, so is it)
    // and wavefronts without keys
    float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - M) / L;
    if (L != L) f = L;
    if (t * 16 + ln >= s.NR) f = 0.f;
#pragma unroll
    for (int u = 0; u < KB; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[u][e] = fmaf(st[u][e], f, sum[u][e]);
  }
  if (key0 < keys.n)
    store_columns<KB>(sum, there, key0, keys.n, ln, lg, part + (static_cast<size_t>(share * B + b) * s.H_kv + h) * keys.n);
}

// acc_out[b][j] = acc_in[b][j] + the parts of all shares and heads, 16 wavefronts that take every 16th of them
__global__ __launch_bounds__(1024) void k_weigh_sum(const float* __restrict__ part, int shares, int B, int H, int n,
                                                    const float* __restrict__ acc_in, float* __restrict__ acc_out) {
  __shared__ float red[16][64];
  const int per = (n + 63) / 64, b = blockIdx.x / per, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
  const int j = blockIdx.x % per * 64 + lane;
  const int at = min(j, n - 1), parts = shares * H;
  auto load = [&](int p) { return part[(static_cast<size_t>(p / H * B + b) * H + p % H) * n + at]; };
  float sum = 0.f;
  int p = wave;
  for (; p + 112 < parts; p += 128) {  // (eight loads in flight: of 128 parts one after the other a microsecond)
    float v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = load(p + 16 * u);
#pragma unroll
    for (int u = 0; u < 8; ++u) sum += v[u];
  }
  for (; p < parts; p += 16) sum += load(p);
  red[wave][lane] = sum;
  __syncthreads();
  if (wave != 0 || j >= n) return;
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < 16; ++w) sum += red[w][lane];
  const size_t to = static_cast<size_t>(b) * n + j;
  acc_out[to] = (acc_in != nullptr ? acc_in[to] : 0.f) + sum;
}

// most 16s of keys a wavefront's registers hold: fragments of at most 128 of them
constexpr int short_blocks(bool f32_keys, bool f32, int D) { return (f32_keys ? 512 : f32 ? 512 : 1024) / D < 8 ? (f32_keys ? 512 : f32 ? 512 : 1024) / D : 8; }

}  // namespace

WeighPlan plan_weigh(int dtype, int format, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  WeighPlan p{};
  WeighShape& s = p.s;
  s.Mq = Mq; s.H_q = H_q; s.H_kv = H_kv; s.G = H_q / H_kv; s.NR = Mq * s.G;
  const long long heads = static_cast<long long>(B) * H_kv;
  const int most = short_blocks(format == 0, dtype == 0, d_h);
  if (n <= 128 * most) {
    p.brief = true;
    p.KB = n <= 256 || most == 2 ? 2 : n <= 512 || most == 4 ? 4 : n <= 768 ? 6 : 8;
    const int rt = (s.NR + 15) / 16;
    // A workgroup per CU, two where the registers leave room for more: 3 % from the quickest share count on average (40 shapes; half as many
    // workgroups 8 %, in the worst 2 times as long: a tile of rows is a chain of loads, products, two exchanges and a barrier)
    const long long target = dtype == 1 && p.KB == 2 ? 512 : 256;
    long long RS = heads >= target ? 1 : target / heads;
    if (RS > rt) RS = rt;
    s.share = static_cast<int>((rt + RS - 1) / RS);
    s.RS = (rt + s.share - 1) / s.share;
    return p;
  }
  p.QB = s.NR <= 16 || dtype == 0 || d_h == 256 ? 1 : s.NR <= 32 ? 2 : 4;
  s.tiles = (s.NR + 16 * p.QB - 1) / (16 * p.QB);
  const int nblk = (n + 31) / 32;
  const long long items = heads * s.tiles;
  long long KS = items >= 256 ? 1 : 256 / items;
  const int split = (nblk + 2 * kSW - 1) / (2 * kSW);  // two blocks a wavefront at least
  KS = KS > split ? split : KS;
  KS = KS > 64 ? 64 : KS < 1 ? 1 : KS;
  s.per = static_cast<int>((nblk + KS - 1) / KS);
  s.KS = (nblk + s.per - 1) / s.per;
  p.KB = (format == 0 || d_h == 256) ? 2 : 4;
  s.blocks = (n + 64 * p.KB - 1) / (64 * p.KB);
  const int row = d_h * (dtype == 1 ? 2 : 4), stage = row >= 512 ? 16 : 8192 / row, st = (s.NR + stage - 1) / stage;
  const long long groups = heads * s.blocks;
  double best = 1e300;
  for (int RS = 1; RS <= 16 && RS <= st; ++RS) {
    const int share = (st + RS - 1) / RS, used = (st + share - 1) / share;
    const double t = static_cast<double>((groups * used + 511) / 512) * (3 + share) + 0.1 * used;
    if (t < best) {
      best = t;
      s.share = share;
      s.RS = used;
    }
  }
  return p;
}

size_t attention_weights_scratch_bytes(const WeighPlan& p, int B, int Mq, int n, int H_q, int H_kv) {
  const size_t rows = static_cast<size_t>(B) * Mq * H_q;
  return (p.brief ? 0 : rows * (2 * p.s.KS + 2) * sizeof(float)) + static_cast<size_t>(p.s.RS) * B * H_kv * n * sizeof(float);
}

void launch_attention_weights(const WeighPlan& p, int dtype, int format, const void* q, int B, int Mq, const CacheView& k, const Keys& keys,
                              int H_q, int H_kv, int d_h, const float* lse, const float* acc_in, float* acc_out, void* scratch, hipStream_t st) {
  const WeighShape& s = p.s;
  const size_t count = static_cast<size_t>(B) * Mq * H_q;
  float2* ml = static_cast<float2*>(scratch);
  float* m = static_cast<float*>(scratch) + 2 * s.KS * count;
  float* il = m + count;
  float* part = static_cast<float*>(scratch) + (p.brief ? 0 : count * (2 * s.KS + 2));
  auto go = [&](auto f, auto t, auto d) {
    typedef decltype(f) F;
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    constexpr bool f32_keys = std::is_same<F, float>::value, f32 = sizeof(T) == 4;
    const T* qt = static_cast<const T*>(q);
    if (p.brief) {
      const dim3 grid(static_cast<unsigned>(static_cast<long long>(B) * H_kv * s.RS));
      constexpr int most = short_blocks(f32_keys, f32, D);
      if (p.KB == 2) hipLaunchKernelGGL((k_weigh_short<F, T, D, 2>), grid, dim3(512), 0, st, qt, s, k, keys, part);
      if constexpr (most >= 4) {
        if (p.KB == 4) hipLaunchKernelGGL((k_weigh_short<F, T, D, 4>), grid, dim3(512), 0, st, qt, s, k, keys, part);
      }
      if constexpr (most >= 8) {
        if (p.KB == 6) hipLaunchKernelGGL((k_weigh_short<F, T, D, 6>), grid, dim3(512), 0, st, qt, s, k, keys, part);
        if (p.KB == 8) hipLaunchKernelGGL((k_weigh_short<F, T, D, 8>), grid, dim3(512), 0, st, qt, s, k, keys, part);
      }
      return;
    }
    if (lse == nullptr) {
      const dim3 rows(static_cast<unsigned>(static_cast<long long>(B) * H_kv * s.tiles * s.KS));
      if constexpr (f32 || D == 256) {
        hipLaunchKernelGGL((k_weigh_stats<F, T, D, 1>), rows, dim3(64 * kSW), 0, st, qt, s, k, keys, ml, m, il);
      } else {
        if (p.QB == 1) hipLaunchKernelGGL((k_weigh_stats<F, T, D, 1>), rows, dim3(64 * kSW), 0, st, qt, s, k, keys, ml, m, il);
        else if (p.QB == 2) hipLaunchKernelGGL((k_weigh_stats<F, T, D, 2>), rows, dim3(64 * kSW), 0, st, qt, s, k, keys, ml, m, il);
        else hipLaunchKernelGGL((k_weigh_stats<F, T, D, 4>), rows, dim3(64 * kSW), 0, st, qt, s, k, keys, ml, m, il);
      }
      if (s.KS > 1)
        hipLaunchKernelGGL(k_weigh_join, dim3(static_cast<unsigned>((count + 255) / 256)), dim3(256), 0, st, ml, s.KS, static_cast<int>(count),
                           m, il);
    }
    constexpr int KB = f32_keys || D == 256 ? 2 : 4;
    hipLaunchKernelGGL((k_weigh_cols<F, T, D, KB>), dim3(static_cast<unsigned>(static_cast<long long>(B) * H_kv * s.blocks * s.RS)),
                       dim3(256), 0, st, qt, s, k, keys, lse ? lse : m, lse ? nullptr : il, lse ? kLog2e : 1.f, part);
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
