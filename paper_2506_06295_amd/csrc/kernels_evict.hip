// Eviction from a cache: the positions that stay under a budget, by accumulated attention weight, and their rows moved together.
#include "kv4.hpp"

namespace dllmc {

namespace {

// What positions are ordered by: 0 not there, then NaN, then the weights ascending (-0 as 0), then those always kept.
__device__ __forceinline__ uint32_t keep_key(float w, bool there, bool always) {
  w += 0.f;
  const uint32_t u = __float_as_uint(w);
  const uint32_t order = w != w ? 1 : (u >> 31) ? ~u : u | 0x80000000u;
  return !there ? 0 : always ? 0xffffffffu : order;
}

// One workgroup of W wavefronts per sequence.  Wavefront w takes the positions [w P, (w + 1) P), P = 64 KPT, 64 neighbours at a time, so
// that the order of positions is the order of (wavefront, trip, lane) and places come from ballots.  The k-th largest key by
// up to four passes over its bytes, fewer where a pass ends between two bins; each counts the keys that agree with the bytes found so far in
// a histogram with a column per lane (weights of one sequence share their exponents: in a single column most of a wavefront's
// adds would meet).  KPT > 0: keys, weights and rows in registers; 0: loaded again in every pass (beyond 16384 positions, whose trips would
// need more registers than sixteen wavefronts have: with their keys alone in them 29606 positions took 40 us, so 44 and 60000 80).  The
// loads of all trips, or of sixteen, go out before the first is looked at: behind conditions, each waiting for its predecessor, 16 sequences
// of 4608 took 13.1 us, now 9.8 to 10.9 (4.4 of them the search), one of 16384 18.6 and 14 to 16.
template <int W, int KPT>
__global__ __launch_bounds__(64 * W) void k_evict(const float* __restrict__ acc, Keys keys, int keep, int first, int last,
                                                  int* __restrict__ kept, int* __restrict__ kept_rows, int* __restrict__ new_lens,
                                                  float* __restrict__ acc_out) {
  constexpr int kThreads = 64 * W;
  __shared__ __attribute__((aligned(16))) uint32_t hist[256 * 64];
  __shared__ __attribute__((aligned(16))) int bins[256];  // (read as int4)
  __shared__ int found[3], counts[2][W];
  const int b = blockIdx.x, wave = threadIdx.x / 64, lane = threadIdx.x % 64;
  constexpr int kBatch = 16;  // trips whose loads go out together where not all do
  const int trips = KPT > 0 ? KPT : (keys.n + kBatch * kThreads - 1) / (kBatch * kThreads) * kBatch;
  const int len = keys.length(b), j0 = wave * trips * 64 + lane;
  const char* weight = reinterpret_cast<const char*>(acc + static_cast<size_t>(b) * keys.n);
  const char* map = keys.row_map != nullptr ? reinterpret_cast<const char*>(keys.row_map + static_cast<size_t>(b) * keys.n) : nullptr;
  auto at = [&](int i) { return static_cast<uint32_t>(min(j0 + i * 64, keys.n - 1)) * 4; };  // (bytes: a scalar base and a 32-bit offset)
  auto order = [&](int i, float w, int r) {
    const int j = j0 + i * 64;
    return keep_key(w, j < len && static_cast<unsigned>(r) < static_cast<unsigned>(keys.cache_rows), j < first || j >= len - last);
  };
  // weights and rows of trips i0 .. + N - 1
  auto load = [&](int i0, auto& w, auto& r) {
    constexpr int N = sizeof(w) / sizeof(w[0]);
#pragma unroll
    for (int u = 0; u < N; ++u) w[u] = *reinterpret_cast<const float*>(weight + at(i0 + u));
    if (map != nullptr) {
#pragma unroll
      for (int u = 0; u < N; ++u) r[u] = *reinterpret_cast<const int*>(map + at(i0 + u));
    } else {
#pragma unroll
      for (int u = 0; u < N; ++u) r[u] = b * keys.n + j0 + (i0 + u) * 64;
    }
  };
  uint32_t held[KPT > 0 ? KPT : 1];
  float held_w[KPT > 0 ? KPT : 1];
  int held_r[KPT > 0 ? KPT : 1];
  // f(trip, key, weight, row) for all trips
  auto each_whole = [&](auto&& f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) f(i, held[i], held_w[i], held_r[i]);
    } else {
      for (int i0 = 0; i0 < trips; i0 += kBatch) {
        float w[kBatch];
        int r[kBatch];
        load(i0, w, r);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) f(i0 + u, order(i0 + u, w[u], r[u]), w[u], r[u]);
      }
    }
  };
  auto each = [&](auto&& f) {
    if constexpr (KPT > 0) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) f(held[i]);
    } else {
      each_whole([&](int, uint32_t u, float, int) { f(u); });
    }
  };
  auto clear = [&] {
    for (int t = threadIdx.x; t < 256 * 16; t += kThreads) reinterpret_cast<uint4*>(hist)[t] = make_uint4(0, 0, 0, 0);
  };
  if constexpr (KPT > 0) {
    load(0, held_w, held_r);
#pragma unroll
    for (int i = 0; i < KPT; ++i) held[i] = order(i, held_w[i], held_r[i]);
  }
  clear();
  int mine = 0;
  each([&](uint32_t u) { mine += __popcll(__ballot(u != 0)); });
  if (lane == 0) counts[0][wave] = mine;
  __syncthreads();
  int there = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) there += counts[0][w];
  const int k = min(keep, there);

  // threshold: keys above it all stay, `quota` of those equal to it, the lowest positions
  uint32_t threshold = 0;
  int quota = 0;
  if (there > keep) {
    int want = k;  // of the keys that agree with the bytes found so far
    for (int shift = 24; shift >= 0; shift -= 8) {
      each([&](uint32_t u) {
        if (u != 0 && (shift == 24 || (u >> (shift + 8)) == (threshold >> (shift + 8)))) atomicAdd(&hist[((u >> shift) & 255) * 64 + lane], 1u);
      });
      __syncthreads();
      {
        constexpr int kParts = kThreads / 256;  // threads per bin
        const int bin = threadIdx.x / kParts, part = threadIdx.x % kParts;
        int sum = 0;
#pragma unroll
        for (int t = 0; t < 16 / kParts; ++t) {  // (the 16 pieces of a bin start elsewhere in every bin: other banks)
          const uint4 v = reinterpret_cast<const uint4*>(hist)[bin * 16 + (part + t * kParts + bin) % 16];
          sum += v.x + v.y + v.z + v.w;
        }
        if (kParts >= 2) sum += __shfl_xor(sum, 1, 64);
        if (kParts >= 4) sum += __shfl_xor(sum, 2, 64);
        if (part == 0) bins[bin] = sum;
      }
      __syncthreads();
      if (wave == 0) {
        const int4 v = reinterpret_cast<const int4*>(bins)[lane];
        const int c[4] = {v.x, v.y, v.z, v.w};
        const int own = c[0] + c[1] + c[2] + c[3];
        int above = own;
        for (int o = 1; o < 64; o <<= 1) {
          const int d = __shfl_down(above, o, 64);
          if (lane + o < 64) above += d;
        }
        above -= own;  // keys in the bins of the lanes after this one
#pragma unroll
        for (int t = 3; t >= 0; --t) {
          if (above < want && above + c[t] >= want) {
            found[0] = lane * 4 + t;
            found[1] = above;
            found[2] = c[t];
          }
          above += c[t];
        }
      }
      if (shift > 0) clear();  // (everybody has read its bins)
      __syncthreads();
      threshold |= static_cast<uint32_t>(found[0]) << shift;
      want -= found[1];
      if (want == found[2]) {  // all of the bin: everything from its lowest key on
        threshold -= threshold > 0 ? 1 : 0;
        want = 0;
        break;
      }
    }
    quota = want;
  }
  // places: of a position that stays, the number of those before it
  int above = 0, equal = 0;
  each([&](uint32_t u) {
    above += __popcll(__ballot(u > threshold));
    equal += __popcll(__ballot(u == threshold && u != 0));
  });
  __syncthreads();
  if (lane == 0) {
    counts[0][wave] = above;
    counts[1][wave] = equal;
  }
  __syncthreads();
  above = equal = 0;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    above += w < wave ? counts[0][w] : 0;
    equal += w < wave ? counts[1][w] : 0;
  }
  const size_t out0 = static_cast<size_t>(b) * keep;
  each_whole([&](int i, uint32_t u, float w, int r) {
    const uint64_t hi = __ballot(u > threshold), eq = __ballot(u == threshold && u != 0);
    const uint64_t below = (1ull << lane) - 1;
    const int hb = above + __popcll(hi & below), eb = equal + __popcll(eq & below);
    if (u > threshold || (u == threshold && u != 0 && eb < quota)) {
      const size_t at = out0 + hb + min(eb, quota);
      kept[at] = j0 + i * 64;
      kept_rows[at] = r;
      if (acc_out != nullptr) acc_out[at] = w;
    }
    above += __popcll(hi);
    equal += __popcll(eq);
  });
  for (int t = k + threadIdx.x; t < keep; t += kThreads) {
    kept[out0 + t] = -1;
    kept_rows[out0 + t] = -1;
    if (acc_out != nullptr) acc_out[out0 + t] = 0.f;
  }
  if (threadIdx.x == 0) new_lens[b] = k;
}

// dst row i = src row rows[i]: rows of `pieces` units
template <typename U>
__global__ __launch_bounds__(256) void k_compact_rows(const int* __restrict__ rows, int M, int src_rows, long long pieces,
                                                      const U* __restrict__ k_src, U* __restrict__ k_dst,
                                                      const U* __restrict__ v_src, U* __restrict__ v_dst) {
  const long long all = M * pieces;
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < all; p += static_cast<long long>(gridDim.x) * 256) {
    const int row = rows[p / pieces];
    if (static_cast<unsigned>(row) >= static_cast<unsigned>(src_rows)) continue;
    const size_t from = static_cast<size_t>(row) * pieces + p % pieces;
    const U k = k_src[from];
    if (v_src != nullptr) v_dst[p] = v_src[from];
    k_dst[p] = k;
  }
}

// the same for 4-bit tensors: a piece is 32 elements, 16 bytes of codes and a scale
__global__ __launch_bounds__(256) void k_compact_kv4(const int* __restrict__ rows, int M, int src_rows, int dst_rows, int H,
                                                     int blocks, Kv4Tensor ks, Kv4Tensor kd, Kv4Tensor vs, Kv4Tensor vd) {
  const long long all = static_cast<long long>(M) * H * blocks;
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < all; p += static_cast<long long>(gridDim.x) * 256) {
    const int g = static_cast<int>(p % blocks), i = static_cast<int>(p / blocks % M), h = static_cast<int>(p / blocks / M);
    const int row = rows[i];
    if (static_cast<unsigned>(row) >= static_cast<unsigned>(src_rows)) continue;
    const size_t from = (static_cast<size_t>(h) * src_rows + row) * blocks + g, to = (static_cast<size_t>(h) * dst_rows + i) * blocks + g;
    reinterpret_cast<uint4*>(kd.codes)[to] = reinterpret_cast<const uint4*>(ks.codes)[from];
    kd.scales[to] = ks.scales[from];
    if (vs.codes != nullptr) {
      reinterpret_cast<uint4*>(vd.codes)[to] = reinterpret_cast<const uint4*>(vs.codes)[from];
      vd.scales[to] = vs.scales[from];
    }
  }
}

inline unsigned groups(long long items) {
  const long long g = (items + 255) / 256;
  return static_cast<unsigned>(g < (1 << 20) ? g : 1 << 20);
}

}  // namespace

void launch_evict(const float* acc, int B, const Keys& keys, int keep, int first, int last, int* kept, int* kept_rows,
                  int* new_lens, float* acc_out, hipStream_t st) {
#define DLLMC_E(W, KPT) \
  hipLaunchKernelGGL((k_evict<W, KPT>), dim3(B), dim3(64 * W), 0, st, acc, keys, keep, first, last, kept, kept_rows, new_lens, acc_out)
  const int n = keys.n;
  if (n <= 256) DLLMC_E(4, 1);
  else if (n <= 1024) DLLMC_E(4, 4);
  else if (n <= 4096) DLLMC_E(16, 4);
  else if (n <= 8192) DLLMC_E(16, 8);
  else if (n <= 16384) DLLMC_E(16, 16);
  else DLLMC_E(16, 0);
#undef DLLMC_E
}

void launch_compact(int format, const int* rows, int M, int src_rows, int dst_rows, int H, int d_h, const void* k_src, void* k_dst,
                    const void* v_src, void* v_dst, hipStream_t st) {
  if (format == 2) {
    const Kv4Tensor none{nullptr, nullptr};
    hipLaunchKernelGGL(k_compact_kv4, dim3(groups(static_cast<long long>(M) * H * (d_h / 32))), dim3(256), 0, st, rows, M, src_rows,
                       dst_rows, H, d_h / 32, kv4_tensor(k_src, src_rows, H, d_h), kv4_tensor(k_dst, dst_rows, H, d_h),
                       v_src ? kv4_tensor(v_src, src_rows, H, d_h) : none, v_src ? kv4_tensor(v_dst, dst_rows, H, d_h) : none);
    return;
  }
  const size_t bytes = static_cast<size_t>(H) * d_h * (format == 1 ? 2 : 4);
  const uintptr_t any = reinterpret_cast<uintptr_t>(k_src) | reinterpret_cast<uintptr_t>(k_dst) | reinterpret_cast<uintptr_t>(v_src) |
                        reinterpret_cast<uintptr_t>(v_dst) | bytes;
  auto go = [&](auto u) {
    typedef decltype(u) U;
    const long long pieces = static_cast<long long>(bytes / sizeof(U));
    hipLaunchKernelGGL(k_compact_rows<U>, dim3(groups(M * pieces)), dim3(256), 0, st, rows, M, src_rows, pieces,
                       static_cast<const U*>(k_src), static_cast<U*>(k_dst), static_cast<const U*>(v_src), static_cast<U*>(v_dst));
  };
  if (any % 16 == 0) go(uint4());
  else go(uint16_t());
}

}  // namespace dllmc
