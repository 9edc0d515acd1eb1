// What a row of logits says about tokens: log probabilities of given ones, the entropy, and the likeliest tokens with theirs.
//
//   m = max l, z = sum e^(l - m), log p(t) = (l_t - m) - log z, H = log z - (sum e^(l - m) (l - m)) / z.
//
// A logit of minus infinity adds nothing to any of these.
#include <cmath>

#include "mx4.hpp"

namespace dllmc {

namespace {

// A workgroup per row: the maximum, the sums, then one walk per alternative for the best token behind the last one.
template <typename T>
__global__ __launch_bounds__(256) void k_logprobs(LogprobRows r) {
  __shared__ float red[4];
  __shared__ unsigned long long redk[4];
  const int i = blockIdx.x;
  const T* l = static_cast<const T*>(r.logits) + static_cast<size_t>(i) * r.ld;
  float m = -INFINITY;
  bool bad = false;
  for (int t = threadIdx.x; t < r.vocab; t += 256) {
    const float v = ldf(l + t);
    bad |= !(v < INFINITY);
    m = fmaxf(m, v);
  }
  m = wave_max(m);
  if (threadIdx.x % 64 == 0) red[threadIdx.x / 64] = m;
  bad = __syncthreads_or(bad);
  m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  const bool none = m == -INFINITY;
  float z = 0.f, y = 0.f;
  if (!bad && !none)
    for (int t = threadIdx.x; t < r.vocab; t += 256) {
      const float v = ldf(l + t) - m, p = expf(v);
      z += p;
      if (p > 0.f) y += p * v;
    }
  __syncthreads();
  z = block_sum<4>(z, red);
  y = block_sum<4>(y, red);
  const float logz = logf(z);
  const float off = bad ? NAN : -INFINITY;  // what a row without a distribution gives
  const bool fine = !bad && !none;
  if (threadIdx.x == 0 && r.entropy) r.entropy[i] = bad ? NAN : none ? 0.f : logz - y / z;
  for (int t = threadIdx.x; t < r.n_given; t += 256) {
    const int id = r.tokens[static_cast<size_t>(i) * r.n_given + t];
    const bool in = static_cast<unsigned>(id) < static_cast<unsigned>(r.vocab);
    r.logp[static_cast<size_t>(i) * r.n_given + t] = !fine ? off : in ? ldf(l + id) - m - logz : -INFINITY;
  }
  // key of a token: its logit in an order that integers have (both zeros alike), then the lower id
  unsigned long long last = ~0ull;
  for (int k = 0; k < r.top_k; ++k) {
    unsigned long long best = 0;
    if (fine)
      for (int t = threadIdx.x; t < r.vocab; t += 256) {
        const float v = ldf(l + t);
        uint32_t b = __float_as_uint(v == 0.f ? 0.f : v);
        b = b & 0x80000000u ? ~b : b | 0x80000000u;
        const unsigned long long key = static_cast<unsigned long long>(b) << 32 | (0xffffffffu - t);
        if (v > -INFINITY && key < last && key > best) best = key;
      }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const unsigned long long u = __shfl_xor(best, o, 64);
      best = best > u ? best : u;
    }
    __syncthreads();
    if (threadIdx.x % 64 == 0) redk[threadIdx.x / 64] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) best = best > redk[w] ? best : redk[w];
    if (threadIdx.x == 0) {
      const int id = best ? static_cast<int>(0xffffffffu - static_cast<uint32_t>(best)) : -1;
      r.top_ids[static_cast<size_t>(i) * r.top_k + k] = id;
      r.top_logp[static_cast<size_t>(i) * r.top_k + k] = id >= 0 ? ldf(l + id) - m - logz : off;
    }
    last = best;
  }
}

}  // namespace

size_t logprobs_scratch_bytes(int, int, int, int) { return 0; }

void launch_logprobs(int dtype, const LogprobRows& r, void*, hipStream_t st) {
  if (dtype == 1) hipLaunchKernelGGL(k_logprobs<bf16_t>, dim3(r.M), dim3(256), 0, st, r);
  else hipLaunchKernelGGL(k_logprobs<float>, dim3(r.M), dim3(256), 0, st, r);
}

}  // namespace dllmc
