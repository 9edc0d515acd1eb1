// What a row of logits says about tokens: log probabilities of given ones, the entropy, and the likeliest tokens with theirs.
//
//   m = max l, z = sum e^(l - m), y = sum e^(l - m) (l - m);  log p(t) = (l_t - m) - log z, H = log z - y / z.
//
// One pass over the logits: every thread keeps its own m, z and y and takes them along when its maximum grows; they meet at the end of the row.
// A logit of minus infinity adds nothing to any of these; a NaN or plus infinity leaves z NaN, which marks the row.
//
// The likeliest tokens come from the same pass.  A block is the 32 logits that a thread takes at a time; their maximum is at hand and stays in LDS.
// At the end the k-th largest of the threads' 256 maxima bounds the k-th logit from below, the few blocks that reach it are read once more
// (k of 32 logits: they are in a cache), and what reaches it there is ranked by counting.  Where that is too many logits (rows of
// equal ones) the row is walked once per alternative.
//
// Rows are cut into slices where there are few of them; a second launch adds the slices.
#include <cmath>

#include "mx4.hpp"

namespace dllmc {

namespace {

typedef unsigned long long u64;

constexpr int kBlock = 32;                // logits of a block
constexpr int kChunk = 256 * kBlock;      // of a workgroup
constexpr int kMaxChunks = 32;            // of a slice: the blocks' maxima in LDS, 32 KB (one more for 2^24 logits)
constexpr int kFlagged = 256, kFound = 1024;

struct Soft {
  float m, z, y;
};
// Sums over either part, about the larger maximum.  (m = -inf: nothing yet, zeros, or NaN.  Differences so large that their exponential is
// zero are held where they can be multiplied.)
constexpr float kFar = -1e30f;
__device__ __forceinline__ Soft soft_join(const Soft& a, const Soft& b) {
  const float m = fmaxf(a.m, b.m);
  const float da = a.m == -INFINITY ? 0.f : a.m - m, db = b.m == -INFINITY ? 0.f : b.m - m;
  const float sa = expf(da), sb = expf(db);
  return {m, sa * a.z + sb * b.z, sa * (a.y + fmaxf(da, kFar) * a.z) + sb * (b.y + fmaxf(db, kFar) * b.z)};
}

// a float32's bits in the order that integers have, both zeros alike; 0 is below all
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderedLowest = 0x007fffffu;  // minus infinity's
// a token's place: its logit, then the lower id; 0: none
__device__ __forceinline__ u64 token_key(float v, int id) { return static_cast<u64>(ordered(v)) << 32 | (0xffffffffu - static_cast<uint32_t>(id)); }
__device__ __forceinline__ int key_token(u64 key) { return key ? static_cast<int>(0xffffffffu - static_cast<uint32_t>(key)) : -1; }

// total over 256 threads in every one, lanes and wavefronts in a fixed order
__device__ __forceinline__ Soft block_soft(Soft t, Soft* red) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) t = soft_join(t, {__shfl_xor(t.m, o, 64), __shfl_xor(t.z, o, 64), __shfl_xor(t.y, o, 64)});
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = t;
  __syncthreads();
  return soft_join(soft_join(red[0], red[1]), soft_join(red[2], red[3]));
}

// Of 256 threads' numbers in tops the largest that k of them reach, its lower 16 bits zero; tops complete, the same in every thread.
__device__ __forceinline__ uint32_t reached_by(const uint32_t* tops, int k) {
  const uint4 four = reinterpret_cast<const uint4*>(tops)[threadIdx.x % 64];
  uint32_t bound = 0;
#pragma unroll 1
  for (int bit = 31; bit >= 16; --bit) {
    const uint32_t b = bound | 1u << bit;
    const int reach = __popcll(__ballot(four.x >= b)) + __popcll(__ballot(four.y >= b)) + __popcll(__ballot(four.z >= b)) +
                      __popcll(__ballot(four.w >= b));
    if (reach >= k) bound = b;
  }
  return bound;
}

// keys[0 .. count) ranked, the k first to best (0 behind them); all of a workgroup's threads, keys complete and followed by room for seven more
__device__ __forceinline__ void rank_keys(u64* keys, int count, int k, u64* best) {
  for (int i = threadIdx.x; i < k; i += 256)
    if (i >= count) best[i] = 0;
  if (threadIdx.x < 7) keys[count + threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < count; i += 256) {
    const u64 own = keys[i];
    int rank = 0;
    for (int j = 0; j < count; j += 8)
#pragma unroll
      for (int e = 0; e < 8; ++e) rank += keys[j + e] > own;
    if (rank < k) best[rank] = own;
  }
  __syncthreads();
}

// the row's results from its sums and, in LDS, its k best keys
template <typename T>
__device__ __forceinline__ void finish_row(const LogprobRows& r, int i, const T* l, const Soft& t, const u64* best) {
  const bool bad = !(t.z >= 0.f), none = t.m == -INFINITY;
  const float logz = logf(t.z), off = bad ? NAN : -INFINITY;  // (off: what a row without a distribution gives)
  if (threadIdx.x == 0 && r.entropy) r.entropy[i] = bad ? NAN : none ? 0.f : logz - t.y / t.z;
  for (int c = threadIdx.x; c < r.n_given; c += 256) {
    const size_t at = static_cast<size_t>(i) * r.n_given + c;
    const int id = r.tokens[at];
    const bool in = static_cast<unsigned>(id) < static_cast<unsigned>(r.vocab);
    r.logp[at] = bad || none ? off : in ? ldf(l + id) - t.m - logz : -INFINITY;
  }
  for (int c = threadIdx.x; c < r.top_k; c += 256) {
    const size_t at = static_cast<size_t>(i) * r.top_k + c;
    const int id = bad || none ? -1 : key_token(best[c]);
    r.top_ids[at] = id;
    r.top_logp[at] = id < 0 ? off : ldf(l + id) - t.m - logz;
  }
}

template <typename T> struct Granule {  // 16 aligned bytes
  static constexpr int N = 16 / sizeof(T), Loads = kBlock / N;
};

// ALIGNED: rows start at multiples of 16 bytes and hold whole granules.  Otherwise a row starts `head` logits into its first granule, and the first
// and last granules' logits are loaded one by one.
template <typename T, bool ALIGNED>
__global__ __launch_bounds__(256) void k_logprobs(LogprobRows r, int slices, int per, Soft* __restrict__ part, u64* __restrict__ part_keys) {
  typedef Granule<T> G;
  extern __shared__ __attribute__((aligned(16))) float top_of[];  // [per][256] blocks' maxima
  __shared__ Soft red[4];
  __shared__ __attribute__((aligned(16))) uint32_t tops[256];
  __shared__ int flagged[kFlagged], count[2];
  __shared__ __attribute__((aligned(16))) u64 found[kFound + 8];
  __shared__ u64 best[kMaxTop], redk[4];
  const int i = blockIdx.x / slices, slice = blockIdx.x % slices, tid = threadIdx.x;
  const T* l = static_cast<const T*>(r.logits) + static_cast<size_t>(i) * r.ld;
  const int head = ALIGNED ? 0 : static_cast<int>(reinterpret_cast<uintptr_t>(l) % 16 / sizeof(T));
  const T* base = l - head;                                    // (a multiple of 16 bytes; nothing before l is read)
  const int granules = (r.vocab + head + G::N - 1) / G::N;     // the row's, partial ones among them
  const int whole0 = head ? 1 : 0, whole1 = (r.vocab + head) / G::N;
  const int g0 = slice * per * G::Loads * 256;
  const int chunks = min(per, (granules - g0 + G::Loads * 256 - 1) / (G::Loads * 256));
  if (tid < 2) count[tid] = 0;

  Soft t{-INFINITY, 0.f, 0.f};
  for (int c = 0; c < chunks; ++c) {
    float x[kBlock];
    const int gc = g0 + c * G::Loads * 256;
    if (ALIGNED || (gc >= whole0 && gc + G::Loads * 256 <= whole1)) {
      uint4 w[G::Loads];
#pragma unroll
      for (int u = 0; u < G::Loads; ++u) w[u] = reinterpret_cast<const uint4*>(base)[min(gc + u * 256 + tid, granules - 1)];
#pragma unroll
      for (int u = 0; u < G::Loads; ++u) {
        const bool in = !ALIGNED || gc + u * 256 + tid < granules;
        const uint32_t q[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int e = 0; e < G::N; ++e) {
          const float v = sizeof(T) == 4 ? __uint_as_float(q[e % 4]) : __uint_as_float(e % 2 ? q[e / 2 % 4] & 0xffff0000u : q[e / 2 % 4] << 16);
          x[u * G::N + e] = in ? v : -INFINITY;
        }
      }
    } else {
#pragma unroll
      for (int u = 0; u < G::Loads; ++u)
#pragma unroll
        for (int e = 0; e < G::N; ++e) {
          const int id = (gc + u * 256 + tid) * G::N + e - head;
          x[u * G::N + e] = id >= 0 && id < r.vocab ? ldf(l + id) : -INFINITY;
        }
    }
    float top = x[0];
#pragma unroll
    for (int e = 1; e < kBlock; ++e) top = fmaxf(top, x[e]);
    if (r.top_k) top_of[c * 256 + tid] = top;
    const float m = fmaxf(t.m, top), mu = m == -INFINITY ? 0.f : m;
    const float d = t.m == -INFINITY ? 0.f : t.m - m, s = __builtin_amdgcn_exp2f(d * kLog2e);
    float z = 0.f, y = 0.f;
#pragma unroll
    for (int e = 0; e < kBlock; ++e) {
      const float v = x[e] - mu, p = __builtin_amdgcn_exp2f(v * kLog2e);
      z += p;
      y = fmaf(p, fmaxf(v, kFar), y);  // (minus infinity times zero)
    }
    t.y = fmaf(s, fmaf(fmaxf(d, kFar), t.z, t.y), y);
    t.z = fmaf(s, t.z, z);
    t.m = m;
  }
  const float own_top = t.m;
  t = block_soft(t, red);

  if (r.top_k) {
    // a lower bound of the k-th largest logit
    tops[tid] = ordered(own_top);
    __syncthreads();
    const uint32_t bound = max(reached_by(tops, r.top_k), kOrderedLowest + 1);  // (minus infinity is no alternative)
    for (int c = 0; c < chunks; ++c)
      if (ordered(top_of[c * 256 + tid]) >= bound) {
        const int at = atomicAdd(&count[0], 1);
        if (at < kFlagged) flagged[at] = c * 256 + tid;
      }
    __syncthreads();
    const int blocks = count[0];
    if (blocks <= kFlagged)
      for (int b = tid / kBlock; b < blocks; b += 256 / kBlock) {
        const int c = flagged[b] / 256, th = flagged[b] % 256, u = tid % kBlock / G::N, e = tid % G::N;
        const int id = (g0 + (c * G::Loads + u) * 256 + th) * G::N + e - head;
        const float v = id >= 0 && id < r.vocab ? ldf(l + id) : -INFINITY;
        if (ordered(v) >= bound && v <= INFINITY) {
          const int at = atomicAdd(&count[1], 1);
          if (at < kFound) found[at] = token_key(v, id);
        }
      }
    __syncthreads();
    if (blocks <= kFlagged && count[1] <= kFound) {
      rank_keys(found, count[1], r.top_k, best);
    } else {
      // too many: a walk over the slice for every alternative
      const int id0 = max(0, g0 * G::N - head), id1 = min(r.vocab, (g0 + chunks * G::Loads * 256) * G::N - head);
      u64 last = ~0ull;
      for (int k = 0; k < r.top_k; ++k) {
        u64 top = 0;
        if (last)
          for (int id = id0 + tid; id < id1; id += 256) {
            const float v = ldf(l + id);
            const u64 key = token_key(v, id);
            if (v > -INFINITY && key < last && key > top) top = key;
          }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const u64 q = __shfl_xor(top, o, 64);
          top = top > q ? top : q;
        }
        if (tid % 64 == 0) redk[tid / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) top = top > redk[w] ? top : redk[w];
        if (tid == 0) best[k] = top;
        last = top;
        __syncthreads();
      }
    }
  }
  if (slices == 1) {
    finish_row(r, i, l, t, best);
  } else {
    if (tid == 0) part[blockIdx.x] = t;
    for (int c = tid; c < r.top_k; c += 256) part_keys[static_cast<size_t>(blockIdx.x) * r.top_k + c] = best[c];
  }
}

// slices of a row added: their sums in a fixed order, and the best of their keys as in a slice
constexpr int kMaxSlices = 64;
template <typename T>
__global__ __launch_bounds__(256) void k_logprobs_join(LogprobRows r, int slices, const Soft* __restrict__ part, const u64* __restrict__ part_keys) {
  __shared__ Soft red[4];
  __shared__ __attribute__((aligned(16))) uint32_t tops[256];
  __shared__ __attribute__((aligned(16))) u64 keys[kMaxSlices * kMaxTop + 8];
  __shared__ u64 best[kMaxTop];
  __shared__ int count;
  const int i = blockIdx.x, tid = threadIdx.x;
  const int all = slices * r.top_k;
  const u64* from = part_keys + static_cast<size_t>(i) * all;
  if (tid == 0) count = 0;
  u64 top = 0;
  for (int c = tid; c < all; c += 256) top = top > from[c] ? top : from[c];
  tops[tid] = static_cast<uint32_t>(top >> 32);
  const Soft t = block_soft(tid < slices ? part[static_cast<size_t>(i) * slices + tid] : Soft{-INFINITY, 0.f, 0.f}, red);
  if (r.top_k) {  // (keys of 0 are none)
    const uint32_t bound = max(reached_by(tops, r.top_k), kOrderedLowest + 1);
    for (int c = tid; c < all; c += 256) {
      const u64 key = from[c];
      if (static_cast<uint32_t>(key >> 32) >= bound) keys[atomicAdd(&count, 1)] = key;
    }
    __syncthreads();
    rank_keys(keys, count, r.top_k, best);
  }
  finish_row(r, i, static_cast<const T*>(r.logits) + static_cast<size_t>(i) * r.ld, t, best);
}

struct Cut { int slices, per; };
// Slices of whole chunks: enough workgroups for every CU where there are few rows, and no more chunks than the maxima's room.
Cut cut_rows(int M, int vocab) {
  const int chunks = (vocab + 8 + kChunk - 1) / kChunk;  // (a row that starts inside a granule may need one more)
  int slices = M >= 1024 ? 1 : (1024 + M - 1) / M;
  slices = slices < chunks ? slices : chunks;
  int per = (chunks + slices - 1) / slices;
  per = per < kMaxChunks ? per : kMaxChunks;
  const int least = (chunks + kMaxSlices - 1) / kMaxSlices;  // (at most 33)
  per = per > least ? per : least;
  return {(chunks + per - 1) / per, per};
}

template <typename T>
void launch(const LogprobRows& r, void* scratch, hipStream_t st) {
  const Cut c = cut_rows(r.M, r.vocab);
  Soft* part = static_cast<Soft*>(scratch);
  u64* keys = reinterpret_cast<u64*>(static_cast<char*>(scratch) + (static_cast<size_t>(r.M) * c.slices * sizeof(Soft) + 15) / 16 * 16);
  const bool aligned = reinterpret_cast<uintptr_t>(r.logits) % 16 == 0 && r.vocab % Granule<T>::N == 0 &&
                       (r.M == 1 || r.ld % Granule<T>::N == 0);
  const dim3 grid(static_cast<unsigned>(r.M) * c.slices);
  const size_t lds = r.top_k ? static_cast<size_t>(c.per) * 1024 : 0;
  if (aligned) hipLaunchKernelGGL((k_logprobs<T, true>), grid, dim3(256), lds, st, r, c.slices, c.per, part, keys);
  else hipLaunchKernelGGL((k_logprobs<T, false>), grid, dim3(256), lds, st, r, c.slices, c.per, part, keys);
  if (c.slices > 1) hipLaunchKernelGGL(k_logprobs_join<T>, dim3(r.M), dim3(256), 0, st, r, c.slices, part, keys);
}

}  // namespace

size_t logprobs_scratch_bytes(int, int M, int vocab, int top_k) {
  const Cut c = cut_rows(M, vocab);
  if (c.slices == 1) return 0;
  const size_t parts = static_cast<size_t>(M) * c.slices;
  return (parts * sizeof(Soft) + 15) / 16 * 16 + parts * top_k * sizeof(u64);
}

void launch_logprobs(int dtype, const LogprobRows& r, void* scratch, hipStream_t st) {
  if (dtype == 1) launch<bf16_t>(r, scratch, st);
  else launch<float>(r, scratch, st);
}

}  // namespace dllmc
