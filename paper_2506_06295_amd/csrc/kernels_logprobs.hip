// What a row of logits says about tokens: log probabilities of given ones, the entropy, and the likeliest tokens with theirs.
//
//   m = max l, z = sum e^(l - m), y = sum e^(l - m) (l - m);  log p(t) = (l_t - m) - log z, H = log z - y / z.
//
// One pass over the logits: every thread keeps its own m, z and y and takes them along when its maximum grows; they meet at the end of the row.
// A logit of minus infinity adds nothing to any of these; a NaN or plus infinity leaves z NaN, which marks the row.
//
// The likeliest tokens come from the same pass.  A block is the 32 logits that a thread takes at a time; their maximum is at hand and stays in LDS.
// At the end the k-th largest of the threads' maxima bounds the k-th logit from below, the few blocks that reach it are read once more
// (k of 32 logits: they are in a cache), and what reaches it there is ranked by counting.  Where that is too many logits the row is
// walked once per alternative: rows of equal ones (1024 of 126464 in bf16, k = 8: 1420 us), float32 logits so far from zero that the bound's 16 bits
// tell few of them apart (1024 x 126464, k = 8, deviation 2: 93 us about 0, 108 about 500, 2110 about 1000).
//
// k_logprobs takes a row, or where there are few rows a slice of one, with a workgroup; a second launch joins slices.  k_logprobs_short takes
// rows of up to 2048 logits with a wavefront each.
//
// Bound by the bytes where there are many: 4096 rows of 152064 bf16 logits, the eight likeliest of each, 229 us (5.4 TB/s; a logit costs 9 vector
// instructions and an exponential, 200 us of the card's), 1024 rows of 126464 in float32 93 (5.6).  Few rows are two dependent launches: 64 rows of
// 126464 15.8 us (13.3 with logits from the memory-side cache), one row 10.7 (the second launch 4.5 of it).  Times here: the best of several means of
// launches behind one another.
#include <cmath>
#include <type_traits>

#include "mx4.hpp"

namespace dllmc {

namespace {

typedef unsigned long long u64;

constexpr int kBlock = 32;                // logits of a block
constexpr int kChunk = 256 * kBlock;      // of a workgroup
constexpr int kMaxChunks = 32;            // of a slice: the blocks' maxima in LDS, 16 KB (one more for 2^24 logits)
constexpr int kFlagged = 256, kFound = 512;

struct Soft {
  float m, z, y;
};
// Sums about the larger maximum m of all.  (Own maximum -inf: nothing yet, zeros, or NaN.  Differences so large that their exponential is zero are held
// where they can be multiplied.)
constexpr float kFar = -1e30f;
__device__ __forceinline__ void about(Soft& t, float m) {
  const float d = t.m == -INFINITY ? 0.f : t.m - m, s = __builtin_amdgcn_exp2f(d * kLog2e);
  t.y = s * fmaf(fmaxf(d, kFar), t.z, t.y);
  t.z *= s;
  t.m = m;
}
__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_xor1(v));
  v = fmaxf(v, dpp_xor2(v));
  v = fmaxf(v, dpp_half_mirror(v));
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xF, 0xF, false)));  // (lane 15 - l of the 16)
}

// a float32's bits in the order that integers have, both zeros alike; 0 is below all
__device__ __forceinline__ uint32_t ordered(float v) {
  const uint32_t b = __float_as_uint(v + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t kOrderedLowest = 0x007fffffu;  // minus infinity's
__device__ __forceinline__ float unordered(uint32_t b) { return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b); }
// a token's place: its logit, then the lower id; 0: none
__device__ __forceinline__ u64 token_key(float v, int id) { return static_cast<u64>(ordered(v)) << 32 | (0xffffffffu - static_cast<uint32_t>(id)); }
__device__ __forceinline__ int key_token(u64 key) { return key ? static_cast<int>(0xffffffffu - static_cast<uint32_t>(key)) : -1; }

// Maximum of 256 threads, whose maxima tops holds in the order above (complete), in every thread.
__device__ __forceinline__ float max_of(const uint32_t* tops) {
  const uint4 four = reinterpret_cast<const uint4*>(tops)[threadIdx.x % 64];
  const uint32_t t = max(max(four.x, four.y), max(four.z, four.w));
  return groups_max(row16_max(unordered(t)));
}
// z and y over 256 threads, lanes and wavefronts in a fixed order; all about the same maximum
__device__ __forceinline__ void block_sums(Soft& t, float2* red) {
  t.z = groups_sum(row16_sum(t.z));
  t.y = groups_sum(row16_sum(t.y));
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = make_float2(t.z, t.y);
  __syncthreads();
  t.z = (red[0].x + red[1].x) + (red[2].x + red[3].x);
  t.y = (red[0].y + red[1].y) + (red[2].y + red[3].y);
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
template <int THREADS = 256, typename T>
__device__ __forceinline__ void finish_row(const LogprobRows& r, int i, const T* l, const Soft& t, const u64* best) {
  const int tid = threadIdx.x % THREADS;
  const bool bad = !(t.z >= 0.f), none = t.m == -INFINITY;
  const float logz = logf(t.z), off = bad ? NAN : -INFINITY;  // (off: what a row without a distribution gives)
  if (tid == 0 && r.entropy) r.entropy[i] = bad ? NAN : none ? 0.f : logz - t.y / t.z;
  for (int c = tid; c < r.n_given; c += THREADS) {
    const size_t at = static_cast<size_t>(i) * r.n_given + c;
    const int id = r.tokens[at];
    const bool in = static_cast<unsigned>(id) < static_cast<unsigned>(r.vocab);
    r.logp[at] = bad || none ? off : in ? ldf(l + id) - t.m - logz : -INFINITY;
  }
  for (int c = tid; c < r.top_k; c += THREADS) {
    const size_t at = static_cast<size_t>(i) * r.top_k + c;
    const int id = bad || none ? -1 : key_token(best[c]);
    r.top_ids[at] = id;
    r.top_logp[at] = id < 0 ? off : ldf(l + id) - t.m - logz;
  }
}

// A row as granules of 16 aligned bytes, counted from the 128-byte line that it starts in, so that a wavefront's loads are whole lines (4096 rows of
// 152013 bf16 logits: with granules counted from the row's own start 285 us, 241 so).  Granule g has logits g N - off ..; those from first on and
// before end are the row's alone, of `part0` and `part1` (-1: there is none) it has some.
template <typename T> struct Row {
  static constexpr int N = 16 / sizeof(T), Loads = kBlock / N;
  const T* l;
  int off, vocab, first, end, part0, part1;
  __device__ __forceinline__ Row(const LogprobRows& r, int i) {
    l = static_cast<const T*>(r.logits) + static_cast<size_t>(i) * r.ld;
    off = static_cast<int>(reinterpret_cast<uintptr_t>(l) % 128 / sizeof(T));
    vocab = r.vocab;
    first = (off + N - 1) / N;
    end = (off + vocab) / N;
    part0 = off % N ? off / N : -1;
    part1 = (off + vocab) % N && end != part0 ? end : -1;
  }
  __device__ __forceinline__ int granules() const { return (off + vocab + N - 1) / N; }
  // Logits of granules g, g + 256, ..: Loads of them, PITCH apart.  INSIDE: all are the row's alone.
  template <int PITCH, bool INSIDE> __device__ __forceinline__ void load(int g, float (&x)[kBlock]) const {
    uint4 w[Loads];
    if (INSIDE || first < end) {
#pragma unroll
      for (int u = 0; u < Loads; ++u) {
        const int at = INSIDE ? g + u * PITCH : max(first, min(g + u * PITCH, end - 1));
        w[u] = *reinterpret_cast<const uint4*>(l + (static_cast<ptrdiff_t>(at) * N - off));
      }
    }
#pragma unroll
    for (int u = 0; u < Loads; ++u) {
      const uint32_t q[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
      const bool in = INSIDE || (g + u * PITCH >= first && g + u * PITCH < end);
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float v = sizeof(T) == 4 ? __uint_as_float(q[e % 4]) : __uint_as_float(e % 2 ? q[e / 2 % 4] & 0xffff0000u : q[e / 2 % 4] << 16);
        x[u * N + e] = in ? v : -INFINITY;
      }
    }
    if (!INSIDE && (part0 >= 0 || part1 >= 0)) {
#pragma unroll
      for (int u = 0; u < Loads; ++u) {
        const int at = g + u * PITCH;
        if (at == part0 || at == part1) {
#pragma unroll
          for (int e = 0; e < N; ++e) {
            const int id = at * N + e - off;
            if (id >= 0 && id < vocab) x[u * N + e] = ldf(l + id);
          }
        }
      }
    }
  }
  __device__ __forceinline__ float logit(int id) const { return id >= 0 && id < vocab ? ldf(l + id) : -INFINITY; }
};

// A block joins a thread's sums; its maximum.
__device__ __forceinline__ float take_block(Soft& t, const float (&x)[kBlock]) {
  float top = x[0];
#pragma unroll
  for (int e = 1; e < kBlock; ++e) top = fmaxf(top, x[e]);
  const float m = fmaxf(t.m, top), mu = m == -INFINITY ? 0.f : m;
  about(t, m);
  float z = 0.f, y = 0.f;
#pragma unroll
  for (int e = 0; e < kBlock; ++e) {
    const float v = x[e] - mu, p = __builtin_amdgcn_exp2f(v * kLog2e);
    z += p;
    y = fmaf(p, fmaxf(v, kFar), y);  // (minus infinity times zero)
  }
  t.y += y;
  t.z += z;
  return top;
}

template <typename T>
__global__ __launch_bounds__(256) void k_logprobs(LogprobRows r, int slices, int per, Soft* __restrict__ part, u64* __restrict__ part_keys) {
  typedef Row<T> R;
  extern __shared__ __attribute__((aligned(16))) uint16_t top_of[];  // [per][256] blocks' maxima, upper half of their place in the order
  __shared__ float2 red[4];
  __shared__ __attribute__((aligned(16))) uint32_t tops[256];
  __shared__ int flagged[kFlagged], count[2];
  __shared__ __attribute__((aligned(16))) u64 found[kFound + 8];
  __shared__ u64 best[kMaxTop], redk[4];
  const int i = blockIdx.x / slices, slice = blockIdx.x % slices, tid = threadIdx.x;
  const R row(r, i);
  constexpr int kStep = R::Loads * 256;  // granules of a chunk
  const int g0 = slice * per * kStep;
  const int chunks = min(per, (row.granules() - g0 + kStep - 1) / kStep);
  if (tid < 2) count[tid] = 0;

  Soft t{-INFINITY, 0.f, 0.f};
  for (int c = 0; c < chunks; ++c) {
    float x[kBlock];
    const int gc = g0 + c * kStep;
    if (gc >= row.first && gc + kStep <= row.end) row.template load<256, true>(gc + tid, x);
    else row.template load<256, false>(gc + tid, x);
    const float top = take_block(t, x);
    if (r.top_k) top_of[c * 256 + tid] = static_cast<uint16_t>(ordered(top) >> 16);
  }
  tops[tid] = ordered(t.m);
  __syncthreads();
  about(t, max_of(tops));
  block_sums(t, red);

  if (r.top_k) {
    // a lower bound of the k-th largest logit
    const uint32_t bound = max(reached_by(tops, r.top_k), kOrderedLowest + 1);  // (its lower half is zero; minus infinity is no alternative)
    const float least = unordered(bound);
    for (int c = 0; c < chunks; ++c)
      if (top_of[c * 256 + tid] >= bound >> 16) {
        const int at = atomicAdd(&count[0], 1);
        if (at < kFlagged) flagged[at] = c * 256 + tid;
      }
    __syncthreads();
    const int blocks = count[0];
    if (blocks <= kFlagged)
      for (int b0 = tid / kBlock; b0 < blocks; b0 += 4 * 256 / kBlock) {
        float v[4];  // (four in flight)
        int id[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int b = b0 + q * 256 / kBlock, f = flagged[min(b, blocks - 1)];
          const int c = f / 256, th = f % 256, u = tid % kBlock / R::N, e = tid % R::N;
          id[q] = (g0 + (c * R::Loads + u) * 256 + th) * R::N + e - row.off;
          v[q] = b < blocks ? row.logit(id[q]) : -INFINITY;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (v[q] >= least) {
            const int at = atomicAdd(&count[1], 1);
            if (at < kFound) found[at] = token_key(v[q], id[q]);
          }
      }
    __syncthreads();
    if (blocks <= kFlagged && count[1] <= kFound) {
      rank_keys(found, count[1], r.top_k, best);
    } else {
      // too many: a walk over the slice for every alternative
      const int id0 = max(0, g0 * R::N - row.off), id1 = min(r.vocab, (g0 + chunks * kStep) * R::N - row.off);
      u64 last = ~0ull;
      for (int k = 0; k < r.top_k; ++k) {
        u64 top = 0;
        if (last)
          for (int id = id0 + tid; id < id1; id += 256) {
            const float v = ldf(row.l + id);
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
    finish_row(r, i, row.l, t, best);
  } else {
    if (tid == 0) part[blockIdx.x] = t;
    for (int c = tid; c < r.top_k; c += 256) part_keys[static_cast<size_t>(blockIdx.x) * r.top_k + c] = best[c];
  }
}

// slices of a row added: their sums in a fixed order, and the best of their keys as in a slice
constexpr int kMaxSlices = 64;
template <typename T>
__global__ __launch_bounds__(256) void k_logprobs_join(LogprobRows r, int slices, const Soft* __restrict__ part, const u64* __restrict__ part_keys) {
  __shared__ float2 red[4];
  __shared__ __attribute__((aligned(16))) uint32_t tops[2][256];
  __shared__ __attribute__((aligned(16))) u64 keys[kMaxSlices * kMaxTop + 8];
  __shared__ u64 best[kMaxTop];
  __shared__ int count;
  const int i = blockIdx.x, tid = threadIdx.x;
  const int all = slices * r.top_k;
  const u64* from = part_keys + static_cast<size_t>(i) * all;
  if (tid == 0) count = 0;
  u64 top = 0;
  for (int c = tid; c < all; c += 256) top = top > from[c] ? top : from[c];
  Soft t = tid < slices ? part[static_cast<size_t>(i) * slices + tid] : Soft{-INFINITY, 0.f, 0.f};
  tops[0][tid] = ordered(t.m);
  tops[1][tid] = static_cast<uint32_t>(top >> 32);
  __syncthreads();
  about(t, max_of(tops[0]));
  block_sums(t, red);
  if (r.top_k) {  // (keys of 0 are none)
    const uint32_t bound = max(reached_by(tops[1], r.top_k), kOrderedLowest + 1);
    for (int c = tid; c < all; c += 256) {
      const u64 key = from[c];
      if (static_cast<uint32_t>(key >> 32) >= bound) keys[atomicAdd(&count, 1)] = key;
    }
    __syncthreads();
    rank_keys(keys, count, r.top_k, best);
  }
  finish_row(r, i, static_cast<const T*>(r.logits) + static_cast<size_t>(i) * r.ld, t, best);
}

// ---- short rows -------------------------------------------------------------------------------------------
// A wavefront per row of up to 2048 logits (with what lies before it in its first line), a lane's 32 in registers; no wavefront waits for another
// (16384 x 1024 in bf16, k = 8: 22.4 us, 64 with a workgroup per row).  The bound is the k-th of 64 lanes' maxima, a weak one for k near 64: some 43
// logits reach it at k = 32 and 160 at 60; at 63 and 64 there are more than the list takes in one of six rows and in half of them, and those rows are
// walked (the same rows, k = 0; 8; 32; 48; 60; 63; 64: 13.3; 22.4; 27.7; 37.8; 69; 191; 291 us; rows of equal logits, k = 8: 66).
constexpr int kShort = 64 * kBlock, kShortFound = 256;
template <typename T>
__global__ __launch_bounds__(256) void k_logprobs_short(LogprobRows r) {
  typedef Row<T> R;
  __shared__ u64 found_[4][kShortFound], best_[4][kMaxTop];
  const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  const int i = blockIdx.x * 4 + wave;
  if (i >= r.M) return;
  u64 *found = found_[wave], *best = best_[wave];
  const R row(r, i);
  float x[kBlock];
  row.template load<64, false>(lane, x);
  Soft t{-INFINITY, 0.f, 0.f};
  take_block(t, x);
  const uint32_t top = ordered(t.m);
  about(t, groups_max(row16_max(t.m)));
  t.z = groups_sum(row16_sum(t.z));
  t.y = groups_sum(row16_sum(t.y));
  if (r.top_k) {
    uint32_t bound = 0;
#pragma unroll 1
    for (int bit = 31; bit >= 16; --bit) {
      const uint32_t b = bound | 1u << bit;
      if (__popcll(__ballot(top >= b)) >= r.top_k) bound = b;
    }
    const float least = unordered(max(bound, kOrderedLowest + 1));
    auto key_of = [&](int e) { return token_key(x[e], (e / R::N * 64 + lane) * R::N + e % R::N - row.off); };
    int count = 0;
#pragma unroll
    for (int e = 0; e < kBlock; ++e) {
      const bool hit = x[e] >= least;
      const unsigned long long hits = __ballot(hit);
      if (hits) {
        const int at = count + __popcll(hits & ((1ull << lane) - 1));
        if (hit && at < kShortFound) found[at] = key_of(e);
        count += __popcll(hits);
      }
    }
    if (lane < r.top_k) best[lane] = 0;
    if (count <= kShortFound) {
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      for (int a = lane; a < count; a += 64) {
        const u64 own = found[a];
        int rank = 0;
        for (int j = 0; j < count; ++j) rank += found[j] > own;
        if (rank < r.top_k) best[rank] = own;
      }
    } else {  // too many: the best behind the last one, once per alternative
      u64 last = ~0ull;
      for (int k = 0; k < r.top_k && last; ++k) {
        u64 next = 0;
#pragma unroll
        for (int e = 0; e < kBlock; ++e) {
          const u64 key = x[e] > -INFINITY ? key_of(e) : 0;
          if (key < last && key > next) next = key;
        }
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
          const u64 q = __shfl_xor(next, o, 64);
          next = next > q ? next : q;
        }
        if (lane == 0) best[k] = next;
        last = next;
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  }
  finish_row<64>(r, i, row.l, t, best);
}

struct Cut { int slices, per; };
// Slices of whole chunks: four workgroups for every CU where there are fewer rows than CUs, one launch beyond, and no more chunks than the maxima's
// room.  One slice and some 1024 workgroups, us, logits of 126464 from memory: float32 64 rows 22.3 and 15.8, 128 27.3 and 21.2, 200 29.1 and 28.9, 256
// 30.7 and 32.4, 500 50.8 and 54.0; bf16 128 rows 25.4 and 17.1, 256 32.7 and 23.7, 300 35.2 and 26.6, 500 37.1 and 36.2, 700 43.8 and 46.0.  The
// limit is float32's: bf16 rows of half the bytes would do better with slices up to some 500 rows.
Cut cut_rows(int dtype, int M, int vocab) {
  const int before = (dtype == 1 ? 64 : 32) - 1;  // (logits that a row's first line may hold before it)
  if (vocab + before <= kShort) return {0, 0};
  const int chunks = (vocab + before + kChunk - 1) / kChunk;
  int slices = M >= 256 ? 1 : (1024 + M - 1) / M;
  slices = slices < chunks ? slices : chunks;
  int per = (chunks + slices - 1) / slices;
  per = per < kMaxChunks ? per : kMaxChunks;
  const int least = (chunks + kMaxSlices - 1) / kMaxSlices;
  per = per > least ? per : least;
  return {(chunks + per - 1) / per, per};
}

template <typename T>
void launch(const LogprobRows& r, void* scratch, hipStream_t st) {
  const Cut c = cut_rows(sizeof(T) == 2, r.M, r.vocab);
  if (c.slices == 0) {
    hipLaunchKernelGGL(k_logprobs_short<T>, dim3((r.M + 3) / 4), dim3(256), 0, st, r);
    return;
  }
  Soft* part = static_cast<Soft*>(scratch);
  u64* keys = reinterpret_cast<u64*>(static_cast<char*>(scratch) + (static_cast<size_t>(r.M) * c.slices * sizeof(Soft) + 15) / 16 * 16);
  const dim3 grid(static_cast<unsigned>(r.M) * c.slices);
  const size_t lds = r.top_k ? static_cast<size_t>(c.per) * 512 : 0;
  hipLaunchKernelGGL(k_logprobs<T>, grid, dim3(256), lds, st, r, c.slices, c.per, part, keys);
  if (c.slices > 1) hipLaunchKernelGGL(k_logprobs_join<T>, dim3(r.M), dim3(256), 0, st, r, c.slices, part, keys);
}

}  // namespace

size_t logprobs_scratch_bytes(int dtype, int M, int vocab, int top_k) {
  const Cut c = cut_rows(dtype, M, vocab);
  if (c.slices <= 1) return 0;
  const size_t parts = static_cast<size_t>(M) * c.slices;
  return (parts * sizeof(Soft) + 15) / 16 * 16 + parts * top_k * sizeof(u64);
}

void launch_logprobs(int dtype, const LogprobRows& r, void* scratch, hipStream_t st) {
  if (dtype == 1) launch<bf16_t>(r, scratch, st);
  else launch<float>(r, scratch, st);
}

}  // namespace dllmc
