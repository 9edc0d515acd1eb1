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
  static constexpr int kW = D / 32, kV = D / 64;
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
      // (a head's codes end below 2^24 * 128 bytes: a scalar base and a 32-bit offset)
      const uint8_t* p = kc + (static_cast<uint32_t>(krow[s]) * (D / 2) + lg * (D / 8));
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
      const uint32_t q = static_cast<uint32_t>(krow[s]) * (D / 32);
      b.ks[s] = D == 64 ? ks[q + lg / 2] : D == 128 ? ks[q + lg] : *reinterpret_cast<const uint16_t*>(ks + (q + 2 * lg));
    }
#pragma unroll
    for (int t = 0; t < B::kV; ++t) {
      const int pc = (t * 64 + lane) % (D / 32);
      b.v[t] = *reinterpret_cast<const uint4*>(vc + (static_cast<uint32_t>(vrow[t]) * (D / 2) + pc * 16));
      b.vs[t] = vs[static_cast<uint32_t>(vrow[t]) * (D / 32) + pc];
    }
  }
};

// An item is a tile of rows of one (sequence, KV head), items ordered by those.  The first `whole` items walk all keys; the others are
// cut into KS ranges of `per` blocks of keys, whose results go to `part` [item - whole][row][range][D] and `part_ml` (m, l), and
// k_attend_merge joins them.
struct AttendShape {
  int Mq, H_q, H_kv, G, NR;  // NR = Mq * G rows of a KV head
  int tiles, whole, KS, per;
  __device__ __forceinline__ size_t row_at(int b, int h, int r) const {  // row of q and out
    const int i = G == 1 ? r : r / G;
    return (static_cast<size_t>(b) * Mq + i) * H_q + h * G + (r - i * G);
  }
};
struct AttendItem { int b, h, tile, range, local; };  // range < 0: all keys


// ---- few rows -----------------------------------------------------------------------------------------
// k_attend_few<T, D, QB, NW>: 16 QB rows of one KV head against a range of keys.  The NW wavefronts deal the range's 32-key blocks
// among themselves; each carries all the rows, keeps the next block in registers while it works on this one, and meets the
// others in LDS at the end.  V is expanded into a tile of the wavefront's own in LDS and comes back transposed.
// Bound by the sum of its instructions with two wavefronts per SIMD (51 rows x 4608 keys: vector ALU 56 % of the time, matrix pipes 21 %,
// LDS 45 %), then the first loads and the hand-over.  Keys loaded along the rows and turned in LDS, queries loaded once for all wavefronts,
// scalar addresses for whole blocks: each within 4 % either way; sixteen wavefronts (128 registers): 21 to 32 us.
template <typename T, int D, int QB, int NW, bool PAGED>
__device__ __forceinline__ void attend_few_body(const T* __restrict__ q, const AttendShape& s, KeyLoader<D, PAGED> ld,
                                                const AttendItem& it, T* __restrict__ out, float* __restrict__ lse,
                                                float* __restrict__ part, float2* __restrict__ part_ml) {
  constexpr int NQ = Parts<T>::kQ, NP = Parts<T>::kP, C = D / 32, DB = D / 16;
  constexpr int kSlots = D / 8, kMix = kSlots < 16 ? kSlots : 16;
  constexpr int kOS = D + 4;
  constexpr int kTile = 32 * kSlots;                        // 16-byte slots of a wavefront's V tile
  constexpr int kHand = (NW * 16 * kOS + 2 * NW * 16) / 4;  // the hand-over of 16 rows
  __shared__ __attribute__((aligned(1024))) uint4 smem[NW * kTile > kHand ? NW * kTile : kHand];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  uint4* vt = smem + wave * kTile;
  const int r0 = it.tile * 16 * QB;

  const int nblk = (ld.len + 31) / 32;
  const int blk1 = it.range < 0 ? nblk : min(nblk, (it.range + 1) * s.per);
  int blk = (it.range < 0 ? 0 : it.range * s.per) + wave;

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
      if (kb.there != 0xffffffffu && ((kb.there >> key) & 1) == 0) {  // (a NaN times a probability of 0 would count)
        kb.vs[t] = 127;
        kb.v[t] = make_uint4(0, 0, 0, 0);
      }
      const uint32_t w[4] = {kb.v[t].x, kb.v[t].y, kb.v[t].z, kb.v[t].w};
#pragma unroll
      for (int u = 0; u < 4; ++u)
        vt[key * kSlots + ((4 * pc + u) ^ (key % kMix))] = __builtin_bit_cast(uint4, kv4_expand(w[u], kb.vs[t]));
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
      float mx = fmaxf(fmaxf(st[0][i][0], st[0][i][1]), st[0][i][2]);
#pragma unroll
      for (int x = 3; x < 8; ++x) mx = fmaxf(mx, st[x / 4][i][x % 4]);
      const float mb = groups_max(mx) * sl2e;
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
    if (PAGED) rk = ld.lookup(min(blk + NW, blk1 - 1) * 32);
#pragma unroll
    for (int i = 0; i < QB; ++i) {
      // (rows past the last one repeat it and are dropped)
      const T* p = q + s.row_at(it.b, it.h, min(r0 + i * 16 + ln, s.NR - 1)) * D + lg * (D / 4);
#pragma unroll
      for (int c = 0; c < C; ++c) load_query(p + 8 * c, qf[i][c]);
    }
    for (; blk + NW < blk1; blk += 2 * NW) {
      ld.fetch((blk + NW) * 32, rk, b1);
      if (PAGED) rk = ld.lookup(min(blk + 2 * NW, blk1 - 1) * 32);
      use(b0);
      ld.fetch(min(blk + 2 * NW, blk1 - 1) * 32, rk, b0);
      if (PAGED) rk = ld.lookup(min(blk + 3 * NW, blk1 - 1) * 32);
      use(b1);
    }
    if (blk < blk1) use(b0);
  }

  // the wavefronts' parts, 16 rows at a time
  float* hand = reinterpret_cast<float*>(smem);  // [wavefront][row][kOS]
  float* ml = hand + NW * 16 * kOS;              // [wavefront][row] m, then l
#pragma unroll
  for (int i = 0; i < QB; ++i) {
    l_run[i] += __shfl_xor(l_run[i], 16, 64);
    l_run[i] += __shfl_xor(l_run[i], 32, 64);
    __syncthreads();
#pragma unroll
    for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(&hand[(wave * 16 + ln) * kOS + d * 16 + 4 * lg]) = o_acc[i][d];
    if (lg == 0) {
      ml[wave * 16 + ln] = m_run[i];
      ml[NW * 16 + wave * 16 + ln] = l_run[i];
    }
    __syncthreads();
    // 4 NW threads per row, E elements each
    constexpr int TR = 4 * NW, E = D / TR;
    typedef float vec_t __attribute__((ext_vector_type(E < 4 ? E : 4)));
    constexpr int VE = E < 4 ? E : 4;
    const int rl = threadIdx.x / TR, t = (threadIdx.x % TR) * E, r = r0 + i * 16 + rl;
    if (r >= s.NR) continue;
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < NW; ++w) M = fmaxf(M, ml[w * 16 + rl]);
    float L = 0.f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.f;
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const float mw = ml[w * 16 + rl], f = mw == -INFINITY ? 0.f : exp2f(mw - M);
      // (a wavefront that saw nothing but NaN scores has the maximum of one that saw nothing, and a NaN for a sum)
      const float lw = ml[NW * 16 + w * 16 + rl];
      L += lw != lw ? lw : lw * f;
#pragma unroll
      for (int e = 0; e < E; e += VE) {
        const vec_t x = *reinterpret_cast<const vec_t*>(&hand[(w * 16 + rl) * kOS + t + e]);
#pragma unroll
        for (int z = 0; z < VE; ++z) o[e + z] += x[z] * f;
      }
    }
    if (it.range < 0) {
      const size_t w = s.row_at(it.b, it.h, r);
      const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
      for (int e = 0; e < E; e += VE) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int z = 0; z < VE; z += 2)
            *reinterpret_cast<uint32_t*>(out + w * D + t + e + z) = pack_bf16x2(o[e + z] * inv, o[e + z + 1] * inv);
        } else {
          vec_t x;
#pragma unroll
          for (int z = 0; z < VE; ++z) x[z] = o[e + z] * inv;
          *reinterpret_cast<vec_t*>(out + w * D + t + e) = x;
        }
      }
      if (lse != nullptr && t == 0) lse[w] = (M + log2f(L)) * kLn2;
    } else {
      const size_t at = (static_cast<size_t>(it.local) * (16 * QB) + i * 16 + rl) * s.KS + it.range;
#pragma unroll
      for (int e = 0; e < E; e += VE) {
        vec_t x;
#pragma unroll
        for (int z = 0; z < VE; ++z) x[z] = o[e + z];
        *reinterpret_cast<vec_t*>(part + at * D + t + e) = x;
      }
      if (t == 0) part_ml[at] = make_float2(M, L);
    }
  }
}

// Wavefronts per SIMD that the registers leave room for.  One alone issues a vector instruction every 9.7 cycles, two every 5: a
// workgroup of 16 rows has four or eight, one of 32 rows eight.
constexpr int few_waves(bool f32, int D, int QB) { return D == 256 ? (f32 ? 1 : 2) : QB == 1 ? (f32 ? 2 : 3) : 2; }
template <typename T, int D, int QB, int NW, bool PAGED>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(few_waves(sizeof(T) == 4, D, QB)))) void k_attend_few(
    const T* __restrict__ q, AttendShape s, CacheView k, CacheView v, Keys keys, T* __restrict__ out, float* __restrict__ lse,
    float* __restrict__ part, float2* __restrict__ part_ml) {
  // the row tiles of a head and range, which read the same keys, on one XCD
  AttendItem it;
  int x = xcd_group_item(blockIdx.x, gridDim.x, s.tiles);
  it.tile = x % s.tiles; x /= s.tiles;
  it.range = s.KS > 1 ? x % s.KS : -1; x /= s.KS;
  it.local = x * s.tiles + it.tile;
  it.h = x % s.H_kv;
  it.b = x / s.H_kv;
  const size_t head = static_cast<size_t>(it.h) * k.cache_rows;
  KeyLoader<D, PAGED> ld{k.kv4.codes + head * (D / 2), k.kv4.scales + head * (D / 32), v.kv4.codes + head * (D / 2),
                         v.kv4.scales + head * (D / 32), PAGED ? keys.row_map + static_cast<size_t>(it.b) * keys.n : nullptr,
                         it.b * keys.n, keys.length(it.b), keys.cache_rows, static_cast<int>(threadIdx.x % 64)};
  attend_few_body<T, D, QB, NW, PAGED>(q, s, ld, it, out, lse, part, part_ml);
}

// ---- many rows ----------------------------------------------------------------------------------------
// k_attend_tile<D, WV>: 32 WV rows of one KV head, 32 a wavefront; keys in blocks of 64, expanded once for the workgroup into
// bf16 tiles in LDS (slot = chunk ^ key % 16) that all wavefronts read, K as it lies, V transposed.  Two stages: while block i is
// multiplied, the codes of block i + 1, loaded a block earlier, are expanded into the other stage.
template <int D, int WV, bool PAGED>
__device__ __forceinline__ void attend_tile_body(const bf16_t* __restrict__ q, const AttendShape& s, const CacheView& k,
                                                 const CacheView& v, const Keys& keys, const AttendItem& it, bf16_t* __restrict__ out,
                                                 float* __restrict__ lse, float* __restrict__ part, float2* __restrict__ part_ml) {
  constexpr int C = D / 32, DB = D / 16, kSlots = D / 8, kMix = kSlots < 16 ? kSlots : 16;
  constexpr int kThreads = 64 * WV, kPieces = 4 * D / kThreads;  // 16-byte pieces of codes per thread, K's before V's
  static_assert(kPieces * kThreads == 4 * D && kThreads <= 4 * D, "whole pieces");
  __shared__ __attribute__((aligned(1024))) uint4 tiles[2][2][64 * kSlots];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  const int r0 = it.tile * 32 * WV + wave * 32;
  const int len = keys.length(it.b), nblk = (len + 63) / 64;
  const int blk0 = it.range < 0 ? 0 : min(nblk, it.range * s.per), blk1 = it.range < 0 ? nblk : min(nblk, (it.range + 1) * s.per);

  float m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
  f32x4 o_acc[2][DB];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int d = 0; d < DB; ++d) o_acc[i][d] = f32x4{0.f, 0.f, 0.f, 0.f};

  if (blk0 < blk1) {
    bf16x8 qf[2][C];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const bf16_t* p = q + s.row_at(it.b, it.h, min(r0 + i * 16 + ln, s.NR - 1)) * D + lg * 8;
#pragma unroll
      for (int c = 0; c < C; ++c) qf[i][c] = *reinterpret_cast<const bf16x8*>(p + 32 * c);
    }
    const size_t head = static_cast<size_t>(it.h) * k.cache_rows;
    // piece t of this thread: tensor, key of the block, piece of the key
    int pkey[kPieces], ppc[kPieces];
    const uint8_t *pc[kPieces], *ps[kPieces];
    bool pv[kPieces];
#pragma unroll
    for (int t = 0; t < kPieces; ++t) {
      const int x = t * kThreads + threadIdx.x;
      pv[t] = x >= 2 * D;
      pkey[t] = x % (2 * D) / (D / 32);
      ppc[t] = x % (D / 32);
      const Kv4Tensor& c = pv[t] ? v.kv4 : k.kv4;
      pc[t] = c.codes + head * (D / 2) + ppc[t] * 16;
      ps[t] = c.scales + head * (D / 32) + ppc[t];
    }
    // cache row of key lane of a block, negative if it is not there
    auto lookup = [&](int blk) {
      const int j = blk * 64 + lane;
      return j < len ? keys.row(it.b, j) : -1;
    };
    uint4 code[kPieces];
    uint32_t scale[kPieces];
    uint64_t there;  // of the block whose codes are in registers
    auto fetch = [&](int blk, int rk) {
      if (PAGED) there = __ballot(rk >= 0);
      else there = len - blk * 64 >= 64 ? ~0ull : (1ull << (len - blk * 64)) - 1;
#pragma unroll
      for (int t = 0; t < kPieces; ++t) {
        const int row = PAGED ? __shfl(max(rk, 0), pkey[t], 64) : it.b * keys.n + min(blk * 64 + pkey[t], len - 1);
        code[t] = *reinterpret_cast<const uint4*>(pc[t] + static_cast<uint32_t>(row) * (D / 2));
        scale[t] = ps[t][static_cast<uint32_t>(row) * (D / 32)];
      }
    };
    auto expand = [&](int stage) {
#pragma unroll
      for (int t = 0; t < kPieces; ++t) {
        const bool ok = (there >> pkey[t]) & 1;  // (a NaN times a probability of 0 would count)
        const uint32_t sc = ok ? scale[t] : 127u;
        const uint32_t w[4] = {ok ? code[t].x : 0u, ok ? code[t].y : 0u, ok ? code[t].z : 0u, ok ? code[t].w : 0u};
        uint4* dst = tiles[stage][pv[t] ? 1 : 0] + pkey[t] * kSlots;
#pragma unroll
        for (int u = 0; u < 4; ++u) dst[(4 * ppc[t] + u) ^ (pkey[t] % kMix)] = __builtin_bit_cast(uint4, kv4_expand(w[u], sc));
      }
    };
    const float sl2e = kLog2e / sqrtf(static_cast<float>(D));
    const int krow = 4 * lg + ln / 4;  // transposing reads, see k_attn_tile
    int voff[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) voff[d] = (krow * kSlots + ((2 * d + (ln % 4) / 2) ^ (krow % kMix))) * 16 + (ln % 2) * 8;

    int rk = PAGED ? lookup(blk0) : 0;
    fetch(blk0, rk);
    if (PAGED) rk = lookup(min(blk0 + 1, blk1 - 1));
    expand(0);
    uint64_t now = there;
    fetch(min(blk0 + 1, blk1 - 1), rk);
    if (PAGED) rk = lookup(min(blk0 + 2, blk1 - 1));
    for (int blk = blk0; blk < blk1; ++blk) {
      const int stage = (blk - blk0) & 1;
      __syncthreads();  // this stage is written, the other one read
      const uint64_t next = there;
      if (blk + 1 < blk1) {
        expand(stage ^ 1);
        fetch(min(blk + 2, blk1 - 1), rk);
        if (PAGED) rk = lookup(min(blk + 3, blk1 - 1));
      }
      const uint4* kt = tiles[stage][0];
      const char* vt = reinterpret_cast<const char*>(tiles[stage][1]);
      f32x4 st[4][2];
#pragma unroll
      for (int sb = 0; sb < 4; ++sb) {
        bf16x8 kf[C];
#pragma unroll
        for (int c = 0; c < C; ++c) kf[c] = __builtin_bit_cast(bf16x8, kt[(sb * 16 + ln) * kSlots + ((4 * c + lg) ^ (ln % kMix))]);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int c = 0; c < C; ++c) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[c], qf[i][c], acc, 0, 0, 0);
          st[sb][i] = acc;
        }
      }
      if (now != ~0ull) {  // wavefront-uniform
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (((now >> (sb * 16 + 4 * lg + e)) & 1) == 0) st[sb][0][e] = st[sb][1][e] = -INFINITY;
      }
      float m_use[2], m_new[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        float mx = -INFINITY;
#pragma unroll
        for (int sb = 0; sb < 4; ++sb)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, st[sb][i][e]);
        // (heads of 128: the exchange competes with the products' neighbours, 4608 rows x 4608 keys x 32 heads 448 us through LDS, 454 without;
        // of 64, 512 rows x 2048 keys x 8 heads 10.6 and 10.3)
        if (D == 64) {
          mx = groups_max(mx);
        } else {
          mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
          mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        }
        const float mb = mx * sl2e;
        m_new[i] = mb > m_run[i] + kLazyMax ? mb : m_run[i];
        m_use[i] = m_new[i] == -INFINITY ? 0.f : m_new[i];
      }
      if (__builtin_amdgcn_ballot_w64(m_new[0] != m_run[0] || m_new[1] != m_run[1]) != 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float alpha = __builtin_amdgcn_exp2f(m_run[i] - m_use[i]);
          l_run[i] *= alpha;
          m_run[i] = m_new[i];
#pragma unroll
          for (int d = 0; d < DB; ++d) o_acc[i][d] *= alpha;
        }
      }
      // probabilities as value + remainder, see k_attn_tile; the second 32 keys' exponentials between the first's products
      bf16x8 pf[2][2], pl[2][2];
      float psum[2] = {0.f, 0.f};
      auto exp_piece = [&](int i, int sb, int e) {
        const float e0 = __builtin_amdgcn_exp2f(fmaf(st[sb][i][e], sl2e, -m_use[i]));
        const float e1 = __builtin_amdgcn_exp2f(fmaf(st[sb][i][e + 1], sl2e, -m_use[i]));
        psum[i] += e0;
        psum[i] += e1;
        const uint32_t hi = pack_bf16x2(e0, e1);
        reinterpret_cast<uint32_t*>(&pf[i][sb / 2])[(sb % 2) * 2 + e / 2] = hi;
        reinterpret_cast<uint32_t*>(&pl[i][sb / 2])[(sb % 2) * 2 + e / 2] =
            pack_bf16x2(e0 - __uint_as_float(hi << 16), e1 - __uint_as_float(hi & 0xffff0000u));
      };
      auto pv_piece = [&](int d, int half) {
        typedef v4s __attribute__((address_space(3))) * lds_v4;
        const char* at = vt + voff[d] + half * (32 * kSlots * 16);
        const v4s a0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(at));
        const v4s a1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4)(at + 16 * kSlots * 16));
        const bf16x8 vf = __builtin_bit_cast(bf16x8, v8s{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]});
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          o_acc[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[i][half], o_acc[i][d], 0, 0, 0);
          o_acc[i][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[i][half], o_acc[i][d], 0, 0, 0);
        }
      };
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int sb = 0; sb < 2; ++sb)
#pragma unroll
          for (int e = 0; e < 4; e += 2) exp_piece(i, sb, e);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        pv_piece(d, 0);
        if (d * 8 % DB == 0) {
          const int x = d * 8 / DB;
          exp_piece(x / 4, 2 + (x / 2) % 2, (x % 2) * 2);
          if (DB < 8) exp_piece((x + 1) / 4, 2 + ((x + 1) / 2) % 2, ((x + 1) % 2) * 2);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int d = 0; d < DB; ++d) pv_piece(d, 1);
      l_run[0] += psum[0];
      l_run[1] += psum[1];
      now = next;
    }
  }
  // a lane: row ln of block i, elements 16 d + 4 lg .. + 3
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l_run[i] += __shfl_xor(l_run[i], 16, 64);
    l_run[i] += __shfl_xor(l_run[i], 32, 64);
    const int r = r0 + i * 16 + ln;
    if (r >= s.NR) continue;
    if (it.range < 0) {
      const size_t w = s.row_at(it.b, it.h, r);
      const float inv = l_run[i] == 0.f ? 0.f : 1.0f / l_run[i];
#pragma unroll
      for (int d = 0; d < DB; ++d)
        *reinterpret_cast<uint2*>(out + w * D + d * 16 + 4 * lg) =
            make_uint2(pack_bf16x2(o_acc[i][d][0] * inv, o_acc[i][d][1] * inv), pack_bf16x2(o_acc[i][d][2] * inv, o_acc[i][d][3] * inv));
      if (lse != nullptr && lg == 0) lse[w] = (m_run[i] + log2f(l_run[i])) * kLn2;
    } else {
      const size_t at = (static_cast<size_t>(it.local) * (32 * WV) + wave * 32 + i * 16 + ln) * s.KS + it.range;
#pragma unroll
      for (int d = 0; d < DB; ++d) *reinterpret_cast<f32x4*>(part + at * D + d * 16 + 4 * lg) = o_acc[i][d];
      if (lg == 0) part_ml[at] = make_float2(m_run[i], l_run[i]);
    }
  }
}

template <int D, int WV, bool PAGED>
__global__ __launch_bounds__(64 * WV, 2) void k_attend_tile(const bf16_t* __restrict__ q, AttendShape s, CacheView k, CacheView v, Keys keys,
                                                         bf16_t* __restrict__ out, float* __restrict__ lse, float* __restrict__ part,
                                                         float2* __restrict__ part_ml) {
  // Whole items first, an XCD (workgroups x, x + 8, ...) taking a contiguous piece of their order: its workgroups share keys.
  AttendItem it;
  int x = blockIdx.x;
  if (x < s.whole) {
    const int xcd = x & 7;
    x = xcd * (s.whole >> 3) + min(xcd, s.whole & 7) + (x >> 3);
    it.range = -1;
    it.local = 0;
  } else {
    x -= s.whole;
    it.range = x % s.KS;
    it.local = x / s.KS;
    x = s.whole + it.local;
  }
  it.tile = x % s.tiles; x /= s.tiles;
  it.h = x % s.H_kv;
  it.b = x / s.H_kv;
  attend_tile_body<D, WV, PAGED>(q, s, k, v, keys, it, out, lse, part, part_ml);
}

// ---- ranges joined -------------------------------------------------------------------------------------
// One wavefront per row of the items that were cut (`rows` of an item): its ranges in order, each loaded when the one before it has
// been added (the compiler does not unroll a loop of unknown length with a shuffle in it).  Bound by those trips to memory, behind that
// for the maxima and sums: 4 us with two ranges.
template <typename T, int D>
__global__ __launch_bounds__(256) void k_attend_merge(const float* __restrict__ part, const float2* __restrict__ part_ml, AttendShape s,
                                                      int rows, T* __restrict__ out, float* __restrict__ lse) {
  constexpr int E = D / 64;
  const int at = blockIdx.x * 4 + threadIdx.x / 64, lane = threadIdx.x % 64;  // (rows is a multiple of 4)
  int x = s.whole + at / rows;
  const int tile = x % s.tiles; x /= s.tiles;
  const int r = tile * rows + at % rows;
  if (r >= s.NR) return;
  const size_t w = s.row_at(x / s.H_kv, x % s.H_kv, r);
  const float2 mine = lane < s.KS ? part_ml[static_cast<size_t>(at) * s.KS + lane] : make_float2(-INFINITY, 0.f);
  const float M = wave_max(mine.x);
  // (a range of nothing but NaN scores has the maximum of an empty one, and a NaN for a sum)
  const float f = mine.x == -INFINITY ? 0.f : exp2f(mine.x - M);
  const float L = wave_sum(mine.y != mine.y ? mine.y : mine.y * f);
  float o[E];
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = 0.f;
  const float* p = part + static_cast<size_t>(at) * s.KS * D + lane * E;
  for (int i = 0; i < s.KS; ++i) {
    const float fk = __shfl(f, i, 64);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += p[static_cast<size_t>(i) * D + e] * fk;
  }
  const float inv = L == 0.f ? 0.f : 1.0f / L;
#pragma unroll
  for (int e = 0; e < E; ++e) stf(out + w * D + lane * E + e, o[e] * inv);
  if (lse != nullptr && lane == 0) lse[w] = (M + log2f(L)) * kLn2;
}

// Kernel, ranges and items that are not cut with the lowest estimate, us: start + rounds over the CUs x round + blocks that a
// wavefront walks x block (one after the other) and x share (per workgroup of a CU) + MB of the caches x mb; and where items are cut
// the joining launch: cut + MB of partial results x part + ranges x range.  Fitted (5 to 13 % rms) to 5600 launches of 419 shapes, 1 to
// 4608 rows, 96 to 16384 keys, 1 to 16 sequences; the choices are 1.3 % from the quickest on average.  Us (heads of 128): one row x 4608
// keys x 32 heads 12.5, 51 rows 19 to 21 (by what the caches hold), 16 sequences x 1 row x 4099 keys x 28 / 4 heads in pages 16.7, 4608 rows
// x 4608 keys x 32 heads 448 (0.78 PFLOP/s, 1.17 with the remainders' products): two and a quarter rounds of 256 workgroups, of which the
// quarter is cut in four.  Float32 and heads of 256 have one kernel, 16 rows by four wavefronts: 51 rows x 4608 keys x 32 heads in float32
// 25.5, 576 rows x 28 / 4 heads 127, 4608 rows x 32 heads 986 (773 at the bf16 rate of its six products); 16 heads of 256 in bf16: one row 15.1, 51
// rows 29, 512 rows 104, 4608 rows 823 (386): every 16 rows expand all keys again.
struct AttendCost { int d, f32, rows, waves, groups; double start, round, block, share, mb, cut, part, range; };
constexpr AttendCost kAttendCosts[] = {
    {64, 1, 16, 4, 5, 2.78, 0.56, 0.258, 0.406, 0, 2.68, 0.521, 0.268},
    {64, 0, 16, 4, 5, 3, 0, 0.481, 0.169, 0.00441, 2.75, 0.753, 0.249},
    {64, 0, 16, 8, 2, 2.97, 0.313, 0.037, 0.816, 0.0305, 2.7, 0.467, 0.244},
    {64, 0, 32, 8, 1, 2.09, 2.35, 1.21, 0, 0.0626, 2.69, 0.342, 0.229},
    {64, 0, 128, 4, 3, 2.97, 0, 0, 1.26, 0, 3, 0.309, 0.203},
    {128, 0, 16, 4, 3, 2.76, 1.12, 0.45, 0.42, 0.0316, 3.09, 0.329, 0.202},
    {128, 0, 16, 8, 1, 1.54, 2.52, 1.25, 0, 0.0309, 2.98, 0.114, 0.228},
    {128, 0, 32, 8, 1, 1.62, 4.3, 1.66, 0, 0.0375, 3.18, 0.171, 0.216},
    {128, 0, 128, 4, 2, 4.78, 0, 0.947, 0.852, 0, 3.87, 0.32, 0.105},
    {128, 0, 256, 8, 1, 4.46, 0, 2.52, 0, 0, 4.24, 0.239, 0.127},
    // not fitted, nothing to choose from but the ranges: blocks as long as the head and the parts make them
    {128, 1, 16, 4, 2, 2.78, 1.12, 0.6, 0.8, 0.03, 2.68, 0.521, 0.268},
    {256, 0, 16, 4, 2, 2.76, 1.5, 0.9, 0.84, 0.03, 3.09, 0.329, 0.202},
    {256, 1, 16, 4, 1, 2.78, 1.5, 2.4, 0, 0.03, 2.68, 0.521, 0.268},
};
}  // namespace

static AttendPlan choose_attend(int dtype, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  const int NR = Mq * (H_q / H_kv);
  const double mb = 2.0 * B * n * H_kv * (d_h / 2 + d_h / 32) / 1e6;
  AttendPlan best{};
  double best_t = 1e300;
  for (const AttendCost& c : kAttendCosts) {
    if (c.d != d_h || c.f32 != (dtype == 0)) continue;
    AttendPlan p{};
    const bool tile = c.rows >= 128;
    p.rows = c.rows;
    p.waves = c.waves;
    p.tiles = (NR + c.rows - 1) / c.rows;
    p.items = static_cast<long long>(B) * H_kv * p.tiles;
    const int blocks = (n + (tile ? 63 : 31)) / (tile ? 64 : 32), deal = tile ? 1 : c.waves;
    const long long slots = 256ll * c.groups;
    auto up = [](long long x, long long y) { return static_cast<double>((x + y - 1) / y); };
    for (const int ks : {1, 2, 3, 4, 6, 8, 10, 12, 16, 24, 32, 48, 64}) {
      if (ks > blocks) break;
      const int per = (blocks + ks - 1) / ks, used = (blocks + per - 1) / per;
      if (used != ks) continue;
      // all items whole; all cut; tiles: those beyond the last whole round cut
      for (int w = 0; w < (ks == 1 ? 1 : tile ? 2 : 1); ++w) {
        const long long whole = ks == 1 ? p.items : w == 0 ? 0 : p.items / slots * slots, cut = p.items - whole;
        if (ks > 1 && cut == 0) continue;
        const double steps = up(blocks, deal), part_steps = up(per, deal);
        double t = c.start + (up(whole, slots) + up(cut * ks, slots)) * c.round +
                   (up(whole, slots) * steps + up(cut * ks, slots) * part_steps) * c.block +
                   (up(whole, 256) * steps + up(cut * ks, 256) * part_steps) * c.share + mb * c.mb;
        if (cut > 0) t += c.cut + static_cast<double>(cut) * c.rows * ks * (d_h + 2) * 4e-6 * c.part + ks * c.range;
        if (t < best_t) {
          best_t = t;
          best = p;
          best.whole = static_cast<int>(whole);
          best.KS = ks;
          best.per = per;
        }
      }
    }
  }
  return best;
}

AttendPlan plan_attend(int dtype, int B, int Mq, int n, int H_q, int H_kv, int d_h) {
  return last_plan<AttendPlan>({dtype, B, Mq, n, H_q, H_kv, d_h}, [&] { return choose_attend(dtype, B, Mq, n, H_q, H_kv, d_h); });
}

size_t attention_kv4_scratch_bytes(const AttendPlan& p, int d_h) {
  return static_cast<size_t>(p.items - p.whole) * p.rows * p.KS * (d_h + 2) * sizeof(float);
}

void launch_attention_kv4(const AttendPlan& p, int dtype, const void* q, int Mq, const CacheView& k, const CacheView& v, const Keys& keys,
                          int H_q, int H_kv, int d_h, void* out, float* lse, void* scratch, hipStream_t st) {
  const AttendShape s{Mq, H_q, H_kv, H_q / H_kv, Mq * (H_q / H_kv), p.tiles, p.whole, p.KS, p.per};
  const long long cut = p.items - p.whole;
  float* part = static_cast<float*>(scratch);
  float2* part_ml = reinterpret_cast<float2*>(part + cut * p.rows * p.KS * d_h);
  const dim3 grid(static_cast<unsigned>(p.whole + cut * p.KS));
  auto go = [&](auto t, auto d, auto paged) {
    typedef decltype(t) T;
    constexpr int D = decltype(d)::value;
    constexpr bool PAGED = decltype(paged)::value;
    const T* qt = static_cast<const T*>(q);
    T* o = static_cast<T*>(out);
#define DLLMC_F(QB, NW) hipLaunchKernelGGL((k_attend_few<T, D, QB, NW, PAGED>), grid, dim3(64 * NW), 0, st, qt, s, k, v, keys, o, lse, part, part_ml)
#define DLLMC_T(WV) hipLaunchKernelGGL((k_attend_tile<D, WV, PAGED>), grid, dim3(64 * WV), 0, st, qt, s, k, v, keys, o, lse, part, part_ml)
    if constexpr (sizeof(T) == 2 && D <= 128) {
      if (p.rows == 16 && p.waves == 4) DLLMC_F(1, 4);
      else if (p.rows == 16) DLLMC_F(1, 8);
      else if (p.rows == 32) DLLMC_F(2, 8);
      else if (D == 64 || p.rows == 128) DLLMC_T(4);
      else if constexpr (D == 128) DLLMC_T(8);
    } else {
      DLLMC_F(1, 4);
    }
#undef DLLMC_F
#undef DLLMC_T
    if (cut > 0)
      hipLaunchKernelGGL((k_attend_merge<T, D>), dim3(static_cast<unsigned>(cut * p.rows / 4)), dim3(256), 0, st, part, part_ml, s, p.rows, o,
                         lse);
  };
  auto with_d = [&](auto t, auto paged) {
    if (d_h == 64) go(t, std::integral_constant<int, 64>{}, paged);
    else if (d_h == 128) go(t, std::integral_constant<int, 128>{}, paged);
    else go(t, std::integral_constant<int, 256>{}, paged);
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
