// Attention over a K/V cache held in 4 bits.
//
// A KV head's query rows -- Mq queries times the G = H_q / H_kv heads that share it, row r = query r / G, head r % G of the group
// -- are one set: cached keys are read once for all of them, and grouped heads fill the matrix cores' 16 columns where
// single queries would not.  Scores are computed transposed (S^T = K Q^T, 16 x 16 x 32 bf16), so that a lane holds, for one row, the
// keys 4 lg .. + 3 of each 16, which is the operand layout of O^T = V^T P^T.  Cached values are exact in bf16, so a bf16 model's products
// are what they would be over a bf16 cache of the same values; float32 queries and probabilities go in three bf16 parts (24 bits).
#include <type_traits>

#include "kv4.hpp"

namespace dllmc {

namespace {

constexpr float kLazyMax = 8.0f;
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));

// A block of 32 keys as a wavefront loads it.  K: lane (ln, lg) has elements lg D/4 .. + D/4 of keys ln and 16 + ln (any deal of
// the elements to the contraction will do that the queries share; this one makes a load of 16 keys one run of memory).  V: piece
// t 64 + lane of 32 elements, of key piece / (D / 32).
template <int D> struct KeyBlock {
  static constexpr int kW = D / 32, kV = D / 64, kKS = D == 256 ? 2 : 1;
  uint32_t k[2][kW];
  uint32_t ks[2];
  uint4 v[kV];
  uint32_t vs[kV];
  uint32_t there;  // bit j: key j of the block is there
};

template <int D, bool PAGED> struct KeyLoader {
  const uint8_t *kc, *ks, *vc, *vs;  // of this head
  const int* map;                    // of this sequence
  int seq0, len, cache_rows, lane;
  // cache row of key `key0 + lane % 32`, negative if it is not there (paged: one lookup per key of the block)
  __device__ __forceinline__ int lookup(int key0) const {
    const int j = key0 + lane % 32;
    if (j >= len) return -1;
    const int r = map[j];
    return static_cast<unsigned>(r) < static_cast<unsigned>(cache_rows) ? r : -1;
  }
  __device__ __forceinline__ void fetch(int key0, int rk, KeyBlock<D>& b) const {
    typedef KeyBlock<D> B;
    const int ln = lane % 16, lg = lane / 16;
    int krow[2], vrow[B::kV];
    if (PAGED) {
      b.there = static_cast<uint32_t>(__ballot(rk >= 0));
      const int safe = max(rk, 0);  // (what is not there reads row 0 and counts for nothing)
#pragma unroll
      for (int s = 0; s < 2; ++s) krow[s] = __shfl(safe, s * 16 + ln, 64);
#pragma unroll
      for (int t = 0; t < B::kV; ++t) vrow[t] = __shfl(safe, (t * 64 + lane) / (D / 32), 64);
    } else {
      const int left = len - key0;
      b.there = left >= 32 ? 0xffffffffu : (1u << max(left, 0)) - 1u;
#pragma unroll
      for (int s = 0; s < 2; ++s) krow[s] = seq0 + max(min(key0 + s * 16 + ln, len - 1), 0);
#pragma unroll
      for (int t = 0; t < B::kV; ++t) vrow[t] = seq0 + max(min(key0 + (t * 64 + lane) / (D / 32), len - 1), 0);
    }
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const uint8_t* p = kc + static_cast<size_t>(krow[s]) * (D / 2) + lg * (D / 8);
      if constexpr (D == 64) {
        const uint2 w = *reinterpret_cast<const uint2*>(p);
        b.k[s][0] = w.x; b.k[s][1] = w.y;
      } else {
#pragma unroll
        for (int h = 0; h < D / 128; ++h) {
          const uint4 w = reinterpret_cast<const uint4*>(p)[h];
          b.k[s][4 * h] = w.x; b.k[s][4 * h + 1] = w.y; b.k[s][4 * h + 2] = w.z; b.k[s][4 * h + 3] = w.w;
        }
      }
      const uint8_t* q = ks + static_cast<size_t>(krow[s]) * (D / 32);
      b.ks[s] = D == 64 ? q[lg / 2] : D == 128 ? q[lg] : reinterpret_cast<const uint16_t*>(q)[lg];
    }
#pragma unroll
    for (int t = 0; t < B::kV; ++t) {
      const int pc = (t * 64 + lane) % (D / 32);
      b.v[t] = *reinterpret_cast<const uint4*>(vc + static_cast<size_t>(vrow[t]) * (D / 2) + pc * 16);
      b.vs[t] = vs[static_cast<size_t>(vrow[t]) * (D / 32) + pc];
    }
  }
};

struct AttendShape {
  int Mq, H_q, H_kv, G, NR;  // NR = Mq * G rows of a KV head
  int tiles, KS, per;        // row tiles, key ranges, 32-key blocks per range
};

// ---- few rows -----------------------------------------------------------------------------------------
// k_attend_few<T, D, QB>: 16 QB rows of one KV head against a range of keys.  The four wavefronts deal the range's 32-key blocks
// among themselves; each carries all the rows, keeps the next block in registers while it works on this one, and meets the
// others in LDS at the end.  V is expanded into a tile of the wavefront's own in LDS and comes back transposed.
// Ranges: results of more than one go to `part` ([row][range][D], then [row][range] (m, l)) and k_attend_merge joins them.
template <typename T, int D, int QB, bool PAGED>
__device__ __forceinline__ void attend_few_body(const T* __restrict__ q, const AttendShape& s, KeyLoader<D, PAGED> ld, int b, int h,
                                                int tile, int range, T* __restrict__ out, float* __restrict__ lse,
                                                float* __restrict__ part, float2* __restrict__ part_ml) {
  constexpr int NQ = Parts<T>::kQ, NP = Parts<T>::kP, C = D / 32, DB = D / 16;
  constexpr int kSlots = D / 8, kMix = kSlots < 16 ? kSlots : 16;
  constexpr int kOS = D + 4;
  constexpr int kTile = 32 * kSlots;                        // 16-byte slots of a wavefront's V tile
  constexpr int kHand = (4 * 16 * kOS + 2 * 4 * 16) / 4;    // the hand-over of 16 rows
  __shared__ __attribute__((aligned(1024))) uint4 smem[4 * kTile > kHand ? 4 * kTile : kHand];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  uint4* vt = smem + wave * kTile;
  const int r0 = tile * 16 * QB;
  auto row_at = [&](int r) {  // (rows past the last one repeat it and are dropped)
    r = min(r, s.NR - 1);
    return (static_cast<size_t>(b) * s.Mq + r / s.G) * s.H_q + h * s.G + r % s.G;
  };

  const int nblk = (ld.len + 31) / 32;
  const int blk1 = min(nblk, (range + 1) * s.per);
  int blk = range * s.per + wave;

  const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
  float m_run[QB], l_run[QB];
  f32x4 o_acc[QB][DB];
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    m_run[i] = -INFINITY;
    l_run[i] = 0.f;
#pragma unroll
    for (int d = 0; d < DB; ++d) o_acc[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const int krow = 4 * lg + ln / 4;  // transposing reads, see k_attn_tile
  int voff[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) voff[d] = (krow * kSlots + ((2 * d + (ln % 4) / 2) ^ (krow % kMix))) * 16 + (ln % 2) * 8;

  bf16x8 qf[QB][C][NQ];

  auto use = [&](KeyBlock<D>& kb) {
    if (kb.there == 0) return;
    // V first: its way through LDS is under the scores
    typedef KeyBlock<D> B;
#pragma unroll
    for (int t = 0; t < B::kV; ++t) {
      const int x = t * 64 + lane, key = x / (D / 32), pc = x % (D / 32);
      const bool ok = (kb.there >> key) & 1;  // (a NaN times a probability of 0 would count)
      const uint32_t sc = ok ? kb.vs[t] : 127u;
      const uint32_t w[4] = {ok ? kb.v[t].x : 0u, ok ? kb.v[t].y : 0u, ok ? kb.v[t].z : 0u, ok ? kb.v[t].w : 0u};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        vt[key * kSlots + ((4 * pc + u) ^ (key % kMix))] = __builtin_bit_cast(uint4, kv4_expand(w[u], sc));
    }
    f32x4 st[2][QB];
#pragma unroll
    for (int sb = 0; sb < 2; ++sb) {
      bf16x8 kf[C];
#pragma unroll
      for (int c = 0; c < C; ++c)
        kf[c] = kv4_expand(kb.k[sb][c], D == 256 ? (kb.ks[sb] >> (c / 4 * 8)) & 255u : kb.ks[sb]);
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int u = NQ - 1; u >= 0; --u)
#pragma unroll
          for (int c = 0; c < C; ++c) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qf[i][c][u], acc, 0, 0, 0);
        st[sb][i] = acc;
      }
    }
    if (kb.there != 0xffffffffu) {  // wavefront-uniform
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (((kb.there >> (sb * 16 + 4 * lg + e)) & 1) == 0) {
#pragma unroll
            for (int i = 0; i < QB; ++i) st[sb][i][e] = -INFINITY;
          }
    }
    // running softmax (base 2); the reference point follows the maximum lazily: only when it has grown by more than 8
    float m_use[QB], m_new[QB];
    bool moved = false;
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      float mx = -INFINITY;
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, st[sb][i][e]);
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mb = mx * sl2e;
      m_new[i] = mb > m_run[i] + kLazyMax ? mb : m_run[i];
      m_use[i] = m_new[i] == -INFINITY ? 0.f : m_new[i];
      moved |= m_new[i] != m_run[i];
    }
    if (__builtin_amdgcn_ballot_w64(moved) != 0) {
#pragma unroll
      for (int i = 0; i < QB; ++i) {
        const float alpha = __builtin_amdgcn_exp2f(m_run[i] - m_use[i]);
        l_run[i] *= alpha;
        m_run[i] = m_new[i];
#pragma unroll
        for (int d = 0; d < DB; ++d) o_acc[i][d] *= alpha;
      }
    }
    // probabilities in parts: bf16 models as value + remainder (16 bits, as over the framework's other caches), float32 ones in three
    bf16x8 pf[QB][NP];
#pragma unroll
    for (int i = 0; i < QB; ++i)
#pragma unroll
      for (int sb = 0; sb < 2; ++sb)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float e0 = __builtin_amdgcn_exp2f(fmaf(st[sb][i][e], sl2e, -m_use[i]));
          float e1 = __builtin_amdgcn_exp2f(fmaf(st[sb][i][e + 1], sl2e, -m_use[i]));
          l_run[i] += e0;
          l_run[i] += e1;
#pragma unroll
          for (int u = 0; u < NP; ++u) {
            const uint32_t w = pack_bf16x2(e0, e1);
            reinterpret_cast<uint32_t*>(&pf[i][u])[sb * 2 + e / 2] = w;
            e0 -= __uint_as_float(w << 16);
            e1 -= __uint_as_float(w & 0xffff0000u);
          }
        }
    asm volatile("" ::: "memory");  // the tile is written (the LDS keeps a wavefront's order by itself)
#pragma unroll
    for (int d = 0; d < DB; ++d) {
      typedef v4s __attribute__((address_space(3))) * lds_v4;
      const char* at = reinterpret_cast<const char*>(vt) + voff[d];
      const v4s a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(at));
      const v4s a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(at + 16 * kSlots * 16));
      const bf16x8 vf = __builtin_bit_cast(bf16x8, v8s{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]});
#pragma unroll
      for (int i = 0; i < QB; ++i)
#pragma unroll
        for (int u = NP - 1; u >= 0; --u) o_acc[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[i][u], o_acc[i][d], 0, 0, 0);
    }
    asm volatile("" ::: "memory");
  };

  if (blk < blk1) {
    KeyBlock<D> b0, b1;
    int rk = PAGED ? ld.lookup(blk * 32) : 0;
    ld.fetch(blk * 32, rk, b0);
    if (PAGED) rk = ld.lookup(min(blk + 4, blk1 - 1) * 32);
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      const T* p = q + row_at(r0 + i * 16 + ln) * D + lg * (D / 4);
#pragma unroll
      for (int c = 0; c < C; ++c) load_query(p + 8 * c, qf[i][c]);
    }
    for (; blk + 4 < blk1; blk += 8) {
      ld.fetch((blk + 4) * 32, rk, b1);
      if (PAGED) rk = ld.lookup(min(blk + 8, blk1 - 1) * 32);
      use(b0);
      ld.fetch(min(blk + 8, blk1 - 1) * 32, rk, b0);
      if (PAGED) rk = ld.lookup(min(blk + 12, blk1 - 1) * 32);
      use(b1);
    }
    if (blk < blk1) use(b0);
  }

  // the wavefronts' parts, 16 rows at a time
  float* hand = reinterpret_cast<float*>(smem);  // [wavefront][row][kOS]
  float* ml = hand + 4 * 16 * kOS;               // [wavefront][row] m, then l
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    l_run[i] += __shfl_xor(l_run[i], 16, 64);
    l_run[i] += __shfl_xor(l_run[i], 32, 64);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(&hand[(wave * 16 + ln) * kOS + d * 16 + 4 * lg]) = o_acc[i][d];
    if (lg == 0) {
      ml[wave * 16 + ln] = m_run[i];
      ml[64 + wave * 16 + ln] = l_run[i];
    }
    __syncthreads();
    // 16 threads per row, D / 16 elements each
    constexpr int E = D / 16;
    const int rl = threadIdx.x / 16, t = (threadIdx.x % 16) * E, r = r0 + i * 16 + rl;
    if (r >= s.NR) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) M = fmaxf(M, ml[w * 16 + rl]);
    float L = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float mw = ml[w * 16 + rl], f = mw == -INFINITY ? 0.f : exp2f(mw - M);
      // (a wavefront that saw nothing but NaN scores has the maximum of one that saw nothing, and a NaN for a sum)
      const float lw = ml[64 + w * 16 + rl];
      L += lw != lw ? lw : lw * f;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(&hand[(w * 16 + rl) * kOS + t + e]);
#pragma unroll
        for (int z = 0; z < 4; ++z) o[e + z] += x[z] * f;
      }
    }
    const size_t w = row_at(r);
    if (s.KS == 1) {
      const float inv = L == 0.f ? 0.f : 1.0f / L;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<uint2*>(out + w * D + t + e) =
              make_uint2(pack_bf16x2(o[e] * inv, o[e + 1] * inv), pack_bf16x2(o[e + 2] * inv, o[e + 3] * inv));
      } else {
#pragma unroll
        for (int e = 0; e < E; e += 4)
          *reinterpret_cast<float4*>(out + w * D + t + e) = make_float4(o[e] * inv, o[e + 1] * inv, o[e + 2] * inv, o[e + 3] * inv);
      }
      if (lse != nullptr && t == 0) lse[w] = (M + log2f(L)) * kLn2;
    } else {
#pragma unroll
      for (int e = 0; e < E; e += 4)
        *reinterpret_cast<float4*>(part + (w * s.KS + range) * D + t + e) = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
      if (t == 0) part_ml[w * s.KS + range] = make_float2(M, L);
    }
  }
}

// workgroups per CU that its registers leave room for without spilling
constexpr int few_groups(bool f32, int D, int QB) { return D == 256 ? (f32 ? 1 : 2) : QB == 1 ? (f32 ? 2 : 3) : QB == 2 ? 2 : 1; }
template <typename T, int D, int QB, bool PAGED>
__global__ __launch_bounds__(256, few_groups(sizeof(T) == 4, D, QB)) void k_attend_few(const T* __restrict__ q, AttendShape s, CacheView k, CacheView v,
                                                                          Keys keys, T* __restrict__ out, float* __restrict__ lse,
                                                                          float* __restrict__ part, float2* __restrict__ part_ml) {
  // row tiles of one head and range run side by side: they read the same keys
  int x = blockIdx.x;
  const int tile = x % s.tiles; x /= s.tiles;
  const int range = x % s.KS; x /= s.KS;
  const int h = x % s.H_kv, b = x / s.H_kv;
  const size_t head = static_cast<size_t>(h) * k.cache_rows;
  KeyLoader<D, PAGED> ld{k.kv4.codes + head * (D / 2), k.kv4.scales + head * (D / 32), v.kv4.codes + head * (D / 2),
                         v.kv4.scales + head * (D / 32), PAGED ? keys.row_map + static_cast<size_t>(b) * keys.n : nullptr, b * keys.n,
                         keys.length(b), keys.cache_rows, static_cast<int>(threadIdx.x % 64)};
  attend_few_body<T, D, QB, PAGED>(q, s, ld, b, h, tile, range, out, lse, part, part_ml);
}

// One wavefront per row: its ranges in order.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_attend_merge(const float* __restrict__ part, const float2* __restrict__ part_ml, int KS,
                                                      long long rows, T* __restrict__ out, float* __restrict__ lse) {
  constexpr int E = D / 64;
  const long long w = static_cast<long long>(blockIdx.x) * 4 + threadIdx.x / 64;
  if (w >= rows) return;
  const int lane = threadIdx.x % 64;
  const float2 mine = lane < KS ? part_ml[w * KS + lane] : make_float2(-INFINITY, 0.f);
  const float M = wave_max(mine.x);
  float f = mine.x == -INFINITY ? 0.f : exp2f(mine.x - M);
  const float L = wave_sum(mine.y != mine.y ? mine.y : mine.y * f);
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  const float* p = part + w * KS * D + lane * E;
  for (int k = 0; k < KS; ++k) {
    const float fk = __shfl(f, k, 64);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += p[static_cast<size_t>(k) * D + e] * fk;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
  for (int e = 0; e < E; ++e) stf(out + w * D + lane * E + e, o[e] * inv);
  if (lse != nullptr && lane == 0) lse[w] = (M + log2f(L)) * kLn2;
}

struct AttendPlan { int QB, tiles, KS, per; };
AttendPlan plan_attend(int dtype, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  const int NR = Mq * (H_q / H_kv), nblk = (n + 31) / 32;
  AttendPlan p{};
  p.QB = NR <= 16 || dtype == 0 || d_h == 256 ? 1 : NR <= 32 ? 2 : 4;
  p.tiles = (NR + 16 * p.QB - 1) / (16 * p.QB);
  const long long items = static_cast<long long>(B) * H_kv * p.tiles;
  const long long want = p.QB == 4 ? 256 : 512;
  int KS = static_cast<int>(items >= want ? 1 : want / items);
  const int most = (nblk + 7) / 8;  // two blocks a wavefront at least
  KS = KS > most ? most : KS;
  KS = KS > 64 ? 64 : KS < 1 ? 1 : KS;
  p.per = (nblk + KS - 1) / KS;
  p.KS = (nblk + p.per - 1) / p.per;
  return p;
}

}  // namespace

size_t attention_kv4_scratch_bytes(int dtype, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  const AttendPlan p = plan_attend(dtype, B, Mq, n, H_q, H_kv, d_h);
  return p.KS == 1 ? 0 : static_cast<size_t>(B) * Mq * H_q * p.KS * (d_h + 2) * sizeof(float);
}

void launch_attention_kv4(int dtype, const void* q, int B, int Mq, const CacheView& k, const CacheView& v, const Keys& keys, int H_q,
                          int H_kv, int d_h, void* out, float* lse, void* scratch, hipStream_t st) {
  const AttendPlan p = plan_attend(dtype, B, Mq, keys.n, H_q, H_kv, d_h);
  const AttendShape s{Mq, H_q, H_kv, H_q / H_kv, Mq * (H_q / H_kv), p.tiles, p.KS, p.per};
  const long long rows = static_cast<long long>(B) * Mq * H_q;
  float* part = static_cast<float*>(scratch);
  float2* part_ml = reinterpret_cast<float2*>(part + (p.KS == 1 ? 0 : rows * p.KS * d_h));
  const dim3 grid(static_cast<unsigned>(static_cast<long long>(B) * H_kv * p.tiles * p.KS));
  auto go = [&](auto t, auto d, auto qb, auto paged) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value, QB = decltype(qb)::value;
    constexpr bool PAGED = decltype(paged)::value;
    hipLaunchKernelGGL((k_attend_few<T, D, QB, PAGED>), grid, dim3(256), 0, st, static_cast<const T*>(q), s, k, v, keys,
                       static_cast<T*>(out), lse, part, part_ml);
    if (p.KS > 1)
      hipLaunchKernelGGL((k_attend_merge<T, D>), dim3(static_cast<unsigned>((rows + 3) / 4)), dim3(256), 0, st, part, part_ml, p.KS,
                         rows, static_cast<T*>(out), lse);
  };
  auto with_qb = [&](auto t, auto d, auto paged) {
    if constexpr (sizeof(t) == 4 || decltype(d)::value == 256) go(t, d, std::integral_constant<int, 1>{}, paged);
    else if (p.QB == 1) go(t, d, std::integral_constant<int, 1>{}, paged);
    else if (p.QB == 2) go(t, d, std::integral_constant<int, 2>{}, paged);
    else go(t, d, std::integral_constant<int, 4>{}, paged);
  };
  auto with_d = [&](auto t, auto paged) {
    if (d_h == 64) with_qb(t, std::integral_constant<int, 64>{}, paged);
    else if (d_h == 128) with_qb(t, std::integral_constant<int, 128>{}, paged);
    else with_qb(t, std::integral_constant<int, 256>{}, paged);
  };
  if (keys.row_map != nullptr) {
    if (dtype == 1) with_d(bf16_t(), std::true_type{});
    else with_d(float(), std::true_type{});
  } else {
    if (dtype == 1) with_d(bf16_t(), std::false_type{});
    else with_d(float(), std::false_type{});
  }
}

}  // namespace dllmc
