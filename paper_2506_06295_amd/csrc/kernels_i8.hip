// Linear maps in 8-bit integers: rows quantised with a scale each, integer products on the matrix cores, scales of row and
// column multiplied in at the end.
//
// out[i][j] = sa[i] sw[j] sum_k a[i][k] w[j][k].  Integer sums are exact whatever their order (|sum| <= 127^2 K < 2^31), so slices of
// the contraction, wavefronts that share it and tiles of any shape give the same bits; the only roundings are the sum's to float32,
// two products and the result's to its type.
//
// Rows are K bytes padded to 128 with zeros: every load is a whole 128-byte line and no kernel knows a ragged K.  Rows past M and N
// repeat the last one and are dropped at the store.
#include <type_traits>

#include "kv4.hpp"

namespace dllmc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// ---- quantising rows --------------------------------------------------------------------------------------
// q = rint(x * (127 * (1 / max|x|))) in float32 (what 127 / tensor is where a tensor's reciprocal is multiplied: the same codes as a
// plain program's), scale = max|x| / 127; one workgroup per row, the row in registers (PC pieces of eight elements a
// thread).  Bound by the bytes with many rows, by two trips to memory with few.
template <typename T, int PC>
__global__ __launch_bounds__(256) void k_quant8(const T* __restrict__ x, int x_rows, const int* __restrict__ rows, int K, int Kp,
                                                int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const int i = blockIdx.x;
  const int row = rows ? rows[i] : i, len = static_cast<unsigned>(row) < static_cast<unsigned>(x_rows) ? K : 0;  // (no row: zeros)
  const T* r = x + static_cast<size_t>(len ? row : 0) * K;
  float v[PC][8];
#pragma unroll
  for (int p = 0; p < PC; ++p) {
    const int t = (p * 256 + threadIdx.x) * 8;
    if (t < len) {
      Eight<T>::load(r + t, v[p]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) v[p][e] = 0.f;
    }
  }
  uint32_t top = 0;
#pragma unroll
  for (int p = 0; p < PC; ++p)
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(v[p][e]) & 0x7fffffffu);
  const RowScale s = row_scale(block_max<4>(top, red));
  if (threadIdx.x == 0) scale[i] = s.scale;
#pragma unroll
  for (int p = 0; p < PC; ++p) {
    const int t = (p * 256 + threadIdx.x) * 8;
    if (t >= Kp) continue;
    uint32_t w[2] = {0, 0};
    if (s.finite) {
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e / 4] |= (static_cast<uint32_t>(static_cast<int>(rintf(v[p][e] * s.f))) & 255u) << (e % 4 * 8);
    }
    *reinterpret_cast<uint2*>(q + static_cast<size_t>(i) * Kp + t) = make_uint2(w[0], w[1]);
  }
}

// any K and alignment, the row read twice
template <typename T>
__global__ __launch_bounds__(256) void k_quant8_any(const T* __restrict__ x, int x_rows, const int* __restrict__ rows, int K, int Kp,
                                                    int8_t* __restrict__ q, float* __restrict__ scale) {
  __shared__ uint32_t red[4];
  const int i = blockIdx.x;
  const int row = rows ? rows[i] : i, len = static_cast<unsigned>(row) < static_cast<unsigned>(x_rows) ? K : 0;  // (no row: zeros)
  const T* r = x + static_cast<size_t>(len ? row : 0) * K;
  uint32_t top = 0;
  for (int t = threadIdx.x; t < len; t += 256) top = max(top, __float_as_uint(ldf(r + t)) & 0x7fffffffu);
  const RowScale s = row_scale(block_max<4>(top, red));
  if (threadIdx.x == 0) scale[i] = s.scale;
  uint32_t* o = reinterpret_cast<uint32_t*>(q + static_cast<size_t>(i) * Kp);
  for (int t = threadIdx.x; t < Kp / 4; t += 256) {
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (s.finite && 4 * t + e < len) w |= (static_cast<uint32_t>(static_cast<int>(rintf(ldf(r + 4 * t + e) * s.f))) & 255u) << (e * 8);
    o[t] = w;
  }
}

// four neighbouring results of a row, n0 + 4 <= N or element by element
template <typename T>
__device__ __forceinline__ void store4(T* p, int n, int N, bool whole, float a, float b, float c, float d) {
  if (whole) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(c, d));
    else *reinterpret_cast<float4*>(p) = make_float4(a, b, c, d);
  } else {
    if (n < N) stf(p, a);
    if (n + 1 < N) stf(p + 1, b);
    if (n + 2 < N) stf(p + 2, c);
    if (n + 3 < N) stf(p + 3, d);
  }
}

// ---- few rows -----------------------------------------------------------------------------------------
// k_i8_ring<RG, RB, NB>: tile = 16 RG RB rows x 16 NB weight rows, one workgroup of eight wavefronts per CU.  Both operands go
// from global memory straight into LDS through a ring of stages.  RG wavefronts take 16 RB rows each, 8 / RG share
// the contraction: a stage is 64 * 8 / RG bytes of every row, and a wavefront multiplies its own 64 of them.  Their sums meet in
// LDS at the end.  The products are taken as W A^T, so that a lane holds four neighbouring columns of a row.
// Slice blockIdx.z of the contraction; with one slice results leave scaled, else as int32 sums for k_i8_sum.
template <int RG, int RB, int NB> struct I8Ring {
  static constexpr int KW = 8 / RG, SS = KW / 2;  // wavefronts along the contraction, 128-byte columns of a stage
  static constexpr int BM = 16 * RG * RB, R = BM + 16 * NB;
  static constexpr int kStage = R * 8 * SS;       // 16-byte slots
  static constexpr int kFit = (152 * 1024) / (kStage * 16), NST = kFit > 8 ? 8 : kFit;
  static constexpr int T = R / 8 * SS, L = T / 8, LR = T % 8;  // load instructions of a stage, per wavefront, one more for the first LR
};

template <typename T, int RG, int RB, int NB>
__device__ __forceinline__ void i8_ring_body(const int8_t* __restrict__ A, const float* __restrict__ sa, int M,
                                             const int8_t* __restrict__ W, const float* __restrict__ sw, int N, int Kp, int per_slice,
                                             T* __restrict__ out, int* __restrict__ sums) {
  typedef I8Ring<RG, RB, NB> S;
  constexpr int NST = S::NST, SS = S::SS, R = S::R, BM = S::BM;
  static_assert(SS >= 1 && NST >= 2, "");
  __shared__ __attribute__((aligned(1024))) uint4 lds[NST][S::kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  const int wr = wave % RG, kk = wave / RG;
  int col_tile, row_tile;
  xcd_tile_map(col_tile, row_tile);
  const int m0 = row_tile * BM, n0 = col_tile * 16 * NB;
  const int kbeg = blockIdx.z * per_slice, lines = (min(Kp, kbeg + per_slice) - kbeg) / 128;  // 128-byte columns
  const int nkt = (lines + SS - 1) / SS;

  // loader: instruction q of a stage copies rows 8 (q % (R/8)) .. + 7 of column q / (R/8); lane: row lane/8, slot lane%8, chunk
  // slot ^ row % 8
  const int8_t* src[S::L + 1];
  int sub[S::L + 1];
#pragma unroll
  for (int j = 0; j < S::L + 1; ++j) {
    const int q = min(wave + 8 * j, S::T - 1);
    const int r = q % (R / 8) * 8 + lane / 8;
    const int8_t* row = r < BM ? A + static_cast<size_t>(min(m0 + r, M - 1)) * Kp : W + static_cast<size_t>(min(n0 + r - BM, N - 1)) * Kp;
    src[j] = row + kbeg + ((lane % 8) ^ (lane / 8)) * 16;
    sub[j] = q / (R / 8);
  }
  // the walk starts at a stage that depends on the column tile: unrotated every load in flight has the same address bits
  // below the row pitch
  const int rot = (col_tile % 8 * 8 + col_tile / 8) % nkt;
  auto issue_one = [&](int stage, int kt, int j) {
    const int q = wave + 8 * j;
    const int line = min(kt * SS + sub[j], lines - 1);  // (columns past the last one repeat it and are not multiplied)
    __builtin_amdgcn_global_load_lds(src[j] + line * 128, &lds[stage][q * 64], 16, 0, 0);
  };
  auto issue = [&](int stage, int kt) {
    const int k = kt + rot < nkt ? kt + rot : kt + rot - nkt;
#pragma unroll
    for (int j = 0; j < S::L; ++j) issue_one(stage, k, j);
    if (S::LR > 0 && wave < S::LR) issue_one(stage, k, S::L);
  };
  auto wait_steps = [&](auto steps) {
    constexpr int n = decltype(steps)::value;
    if (S::LR > 0 && wave < S::LR) wait_vmcnt_lds<n * (S::L + 1)>();
    else wait_vmcnt_lds<n * S::L>();
  };

  i32x4 acc[RB][NB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
#pragma unroll
  for (int s = 0; s < NST - 1; ++s)
    if (s < nkt) issue(s, s);
  int stage = 0;
  for (int kt = 0; kt < nkt; ++kt) {
    // the loads of stage kt have landed; the younger stages, at most NST - 2, stay in flight
    const int rem = nkt - 1 - kt;
    if (rem >= NST - 2) wait_steps(std::integral_constant<int, NST - 2>{});
    else if (NST > 7 && rem == 5) wait_steps(std::integral_constant<int, 5>{});
    else if (NST > 6 && rem == 4) wait_steps(std::integral_constant<int, 4>{});
    else if (NST > 5 && rem == 3) wait_steps(std::integral_constant<int, 3>{});
    else if (NST > 4 && rem == 2) wait_steps(std::integral_constant<int, 2>{});
    else if (NST > 3 && rem == 1) wait_steps(std::integral_constant<int, 1>{});
    else wait_steps(std::integral_constant<int, 0>{});
    __builtin_amdgcn_s_barrier();
    const int nxt = stage == 0 ? NST - 1 : stage - 1;
    if (kt + NST - 1 < nkt) issue(nxt, kt + NST - 1);
    const int k = kt + rot < nkt ? kt + rot : kt + rot - nkt;
    if (k * SS + kk / 2 < lines) {  // (wavefront-uniform)
      const uint4* base = &lds[stage][kk / 2 * R * 8];
      const int c = kk % 2 * 4 + lg;
      i32x4 af[RB], bf[NB];
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int r = (wr * RB + i) * 16 + ln;
        af[i] = __builtin_bit_cast(i32x4, base[r * 8 + (c ^ (r % 8))]);
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int r = BM + j * 16 + ln;
        bf[j] = __builtin_bit_cast(i32x4, base[r * 8 + (c ^ (r % 8))]);
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < RB; ++i) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(bf[j], af[i], acc[i][j], 0, 0, 0);
    }
    stage = stage + 1 < NST ? stage + 1 : 0;
  }
  // hand-over: the sums of the wavefronts that shared a row group, added by RG * RB * NB / 8 blocks per wavefront
  __syncthreads();
  i32x4* red = reinterpret_cast<i32x4*>(&lds[0][0]);
  static_assert(8 * RB * NB * 64 <= NST * S::kStage, "hand-over fits the ring");
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) red[((kk * RG + wr) * RB * NB + i * NB + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int x = wave; x < RG * RB * NB; x += 8) {  // block x = (row group, i, j)
    i32x4 sum = red[x * 64 + lane];
#pragma unroll
    for (int w = 1; w < S::KW; ++w) sum += red[(w * RG * RB * NB + x) * 64 + lane];
    const int j = x % NB, rb = x / NB;
    const int m = m0 + rb * 16 + ln, n = n0 + j * 16 + lg * 4;
    if (m >= M || n >= N) continue;
    const bool whole = n + 4 <= N && N % 4 == 0;
    if (gridDim.z == 1) {
      const float a = sa[m];
      float v[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = static_cast<float>(sum[e]) * a * sw[min(n + e, N - 1)];
      store4(out + static_cast<size_t>(m) * N + n, n, N, whole, v[0], v[1], v[2], v[3]);
    } else {
      int* o = sums + (static_cast<size_t>(blockIdx.z) * M + m) * N + n;
      if (whole) {
        *reinterpret_cast<i32x4*>(o) = sum;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (n + e < N) o[e] = sum[e];
      }
    }
  }
}

template <typename T, int RG, int RB, int NB>
__global__ __launch_bounds__(512) void k_i8_ring(const int8_t* __restrict__ A, const float* __restrict__ sa, int M,
                                                 const int8_t* __restrict__ W, const float* __restrict__ sw, int N, int Kp,
                                                 int per_slice, T* __restrict__ out, int* __restrict__ sums) {
  i8_ring_body<T, RG, RB, NB>(A, sa, M, W, sw, N, Kp, per_slice, out, sums);
}

// out = scaled sum of S slices
template <typename T>
__global__ __launch_bounds__(256) void k_i8_sum(const int* __restrict__ sums, int S, int M, int N, const float* __restrict__ sa,
                                                const float* __restrict__ sw, T* __restrict__ out) {
  const long long all = static_cast<long long>(M) * N;
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < all; p += static_cast<long long>(gridDim.x) * 256) {
    int v = 0;
    for (int s = 0; s < S; ++s) v += sums[s * all + p];
    stf(out + p, static_cast<float>(v) * sa[p / N] * sw[p % N]);
  }
}

// ---- many rows ----------------------------------------------------------------------------------------
// k_i8_wide<WM, WN, MI, NJ>: tile = 16 WM MI rows x 16 WN NJ columns, four wavefronts, one per SIMD, 16 MI x 16 NJ results
// each.  Operands, ring and the order of reads and loads are k_gemm_wide's (a step is 128 bytes of every row; 64 of
// them are one 16 x 16 x 64 product).  The accumulators are pinned to the accumulation registers by asm statements, the last
// product of a step waits for its own result.
template <int BM, int BN> struct I8Rings {
  static constexpr int kWhole = 1280 / (BM + BN);
  static constexpr int kLeft = 1280 - kWhole * (BM + BN);
  static constexpr int DA = kWhole + (kLeft >= BM && (BM >= BN || kLeft < BN) ? 1 : 0);
  static constexpr int DB = kWhole + (DA == kWhole && kLeft >= BN ? 1 : 0);
};

template <typename T, int WM, int WN, int MI, int NJ>
__device__ __forceinline__ void i8_wide_body(const int8_t* __restrict__ A, const float* __restrict__ sa, int M,
                                             const int8_t* __restrict__ W, const float* __restrict__ sw, int N, int Kp,
                                             T* __restrict__ out) {
  constexpr int BM = WM * MI * 16, BN = WN * NJ * 16, LA = BM / 32, LB = BN / 32;
  static_assert(WM * WN == 4 && BM % 32 == 0 && BN % 32 == 0, "four wavefronts, whole load instructions");
  typedef I8Rings<BM, BN> Ring;
  // X, the operand with the shallower ring, has its next block loaded in the second half of a step, Y in the first half of the
  // next one; the barrier stands between the halves
  constexpr int DA = Ring::DA < 5 ? Ring::DA : 5, DB = Ring::DB < 5 ? Ring::DB : 5;
  constexpr bool XB = DA >= DB;
  constexpr int DX = XB ? DB : DA, DY = XB ? DA : DB, LX = XB ? LB : LA, LY = XB ? LA : LB;
  constexpr int kSlotA = BM * 8, kSlotB = BN * 8;
  static_assert((DA * kSlotA + DB * kSlotB) * sizeof(uint4) <= 160 * 1024 && DX >= 2, "LDS of one CU");
  __shared__ __attribute__((aligned(1024))) uint4 lds[DA * kSlotA + DB * kSlotB];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  const int wm = wave / WN, wn = wave % WN;
  int col_tile, row_tile;
  xcd_tile_map_blocked(col_tile, row_tile);
  const int m0 = row_tile * BM, n0 = col_tile * BN, nkt = Kp / 128;

  // loader: wavefront w issues instructions L w .. L w + L - 1 of an operand, 8 rows each: a scalar base and a lane offset
  // (rows past the last one: the last one)
  const char *abase[LA], *bbase[LB];
  uint32_t aoff[LA], boff[LB];
  const int chunk = ((lane % 8) ^ (lane / 8)) * 16;
#pragma unroll
  for (int j = 0; j < LA; ++j) {
    const int r = min(m0 + 8 * (LA * wave + j), M - 1);
    abase[j] = wave_uniform_ptr(reinterpret_cast<const char*>(A + static_cast<size_t>(r) * Kp));
    aoff[j] = static_cast<uint32_t>(min(lane / 8, M - 1 - r) * Kp + chunk);
  }
#pragma unroll
  for (int j = 0; j < LB; ++j) {
    const int r = min(n0 + 8 * (LB * wave + j), N - 1);
    bbase[j] = wave_uniform_ptr(reinterpret_cast<const char*>(W + static_cast<size_t>(r) * Kp));
    boff[j] = static_cast<uint32_t>(min(lane / 8, N - 1 - r) * Kp + chunk);
  }
  const int rot = (((blockIdx.x + gridDim.x * blockIdx.y) & 7) * nkt) >> 3;  // the walk starts at a step that depends on the XCD
  auto kof = [&](int kt) { const int k = kt + rot; return (k < nkt ? k : k - nkt) * 128; };
  auto issue_a = [&](int slot, int ko, int j) {
    uint32_t o = aoff[j];
    asm volatile("" : "+v"(o));
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(wave_uniform_ptr(abase[j] + ko) + o),
                                     &lds[slot * kSlotA + (LA * wave + j) * 64], 16, 0, 0);
  };
  auto issue_b = [&](int slot, int ko, int j) {
    uint32_t o = boff[j];
    asm volatile("" : "+v"(o));
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(wave_uniform_ptr(bbase[j] + ko) + o),
                                     &lds[DA * kSlotA + slot * kSlotB + (LB * wave + j) * 64], 16, 0, 0);
  };
  auto issue_x = [&](int slot, int ko, int j) { if (XB) issue_b(slot, ko, j); else issue_a(slot, ko, j); };
  auto issue_y = [&](int slot, int ko, int j) { if (XB) issue_a(slot, ko, j); else issue_b(slot, ko, j); };
  auto block_x = [&](int t) {
    if (t >= nkt) return;
    const int ko = kof(t);
#pragma unroll
    for (int j = 0; j < LX; ++j) issue_x(t, ko, j);
  };
  auto block_y = [&](int t) {
    if (t >= nkt) return;
    const int ko = kof(t);
#pragma unroll
    for (int j = 0; j < LY; ++j) issue_y(t, ko, j);
  };
  // in the order of the main loop: X(t), Y(t + DY - DX); Y(DY - 1) goes out in step 0
#pragma unroll
  for (int t = 0; t < DY - DX; ++t) block_y(t);
#pragma unroll
  for (int t = 0; t < DX - 1; ++t) {
    block_x(t);
    block_y(t + DY - DX);
  }
  block_x(DX - 1);
  i32x4 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  i32x4 af[2][MI], bf[2][NJ];
  auto read = [&](int slot_a, int slot_b, int kk, int q) {
    const int c = kk * 4 + lg;
    if (q < NJ) {
      const int r = wn * (NJ * 16) + q * 16 + ln;
      bf[kk][q] = __builtin_bit_cast(i32x4, lds[DA * kSlotA + slot_b * kSlotB + r * 8 + (c ^ (r % 8))]);
    } else {
      const int r = wm * (MI * 16) + (q - NJ) * 16 + ln;
      af[kk][q - NJ] = __builtin_bit_cast(i32x4, lds[slot_a * kSlotA + r * 8 + (c ^ (r % 8))]);
    }
  };
  // The compiler does not know how long the results of an asm statement take: the last one of a step waits itself (8 wait
  // states), and nothing but these statements touches the accumulators inside the loop.
  auto half = [&](auto kk_, auto&& between) {
    constexpr int kk = decltype(kk_)::value;
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        if (kk == 1 && i * NJ + j == MI * NJ - 1)
          asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0\n\ts_nop 7" : "+a"(acc[i][j]) : "v"(bf[kk][j]), "v"(af[kk][i]));
        else
          asm volatile("v_mfma_i32_16x16x64_i8 %0, %1, %2, %0" : "+a"(acc[i][j]) : "v"(bf[kk][j]), "v"(af[kk][i]));
        __builtin_amdgcn_sched_barrier(0);
        between(i * NJ + j);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
  constexpr int kSpan = MI * NJ >= 64 ? MI * NJ * 5 / 8 : MI * NJ * 3 / 4;  // MFMAs that reads and loads are spread over
  if (nkt >= DY) wait_vmcnt_lds<(DX - 1) * LX + (DY > DX ? DX - 1 : DX - 2) * LY>();
  else wait_vmcnt_lds<0>();
  __builtin_amdgcn_s_barrier();
#pragma unroll
  for (int q = 0; q < MI + NJ; ++q) read(0, 0, 0, q);
  int s_a = 0, s_b = 0, s_y = DY - 1;
  // step kt with `left` steps to come (DX: that many or more)
  auto step = [&](int kt, auto left_) {
    constexpr int left = decltype(left_)::value;
    constexpr int kFly = left == 0 ? 0 : (DX - 2 < left - 1 ? DX - 2 : left - 1) * LX + (DY - 2 < left - 1 ? DY - 2 : left - 1) * LY;
    const int a1 = s_a + 1 < DA ? s_a + 1 : 0, b1 = s_b + 1 < DB ? s_b + 1 : 0;
    const int ky = left >= DY - 1 ? kof(kt + DY - 1) : 0, kx = left >= DX ? kof(kt + DX) : 0;
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    half(std::integral_constant<int, 0>{}, [&](int t) {
#pragma unroll
      for (int q = 0; q < MI + NJ; ++q)
        if (1 + q * kSpan / (MI + NJ) == t) read(s_a, s_b, 1, q);
#pragma unroll
      for (int l = 0; l < LY; ++l)
        if (left >= DY - 1 && l * kSpan / LY == t) issue_y(s_y, ky, l);
    });
    wait_vmcnt_lds<kFly>();
    if (left > 0) __builtin_amdgcn_s_barrier();
    half(std::integral_constant<int, 1>{}, [&](int t) {
#pragma unroll
      for (int q = 0; q < MI + NJ; ++q)
        if (left > 0 && 1 + q * kSpan / (MI + NJ) == t) read(a1, b1, 0, q);
#pragma unroll
      for (int l = 0; l < LX; ++l)
        if (left >= DX && l * kSpan / LX == t) issue_x(XB ? s_b : s_a, kx, l);
    });
    s_y = XB ? s_a : s_b;
    s_a = a1;
    s_b = b1;
  };
  int kt = 0;
  for (; kt < nkt - DX; ++kt) step(kt, std::integral_constant<int, DX>{});
  if constexpr (DX > 4) { if (nkt - kt > 4) step(kt++, std::integral_constant<int, 4>{}); }
  if constexpr (DX > 3) { if (nkt - kt > 3) step(kt++, std::integral_constant<int, 3>{}); }
  if constexpr (DX > 2) { if (nkt - kt > 2) step(kt++, std::integral_constant<int, 2>{}); }
  if (nkt - kt > 1) step(kt++, std::integral_constant<int, 1>{});
  step(kt, std::integral_constant<int, 0>{});
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
  __builtin_amdgcn_sched_barrier(0);
  // a lane: row ln of block i, columns 4 lg .. + 3 of block j
  float cs[NJ][4], rs[MI];
#pragma unroll
  for (int j = 0; j < NJ; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) cs[j][e] = sw[min(n0 + wn * (NJ * 16) + j * 16 + lg * 4 + e, N - 1)];
#pragma unroll
  for (int i = 0; i < MI; ++i) rs[i] = sa[min(m0 + wm * (MI * 16) + i * 16 + ln, M - 1)];
#pragma unroll
  for (int i = 0; i < MI; ++i) {
    const int m = m0 + wm * (MI * 16) + i * 16 + ln;
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int n = n0 + wn * (NJ * 16) + j * 16 + lg * 4;
      const i32x4 v = acc[i][j];
      if (m < M && n < N)
        store4(out + static_cast<size_t>(m) * N + n, n, N, N % 4 == 0, static_cast<float>(v[0]) * rs[i] * cs[j][0],
               static_cast<float>(v[1]) * rs[i] * cs[j][1], static_cast<float>(v[2]) * rs[i] * cs[j][2],
               static_cast<float>(v[3]) * rs[i] * cs[j][3]);
    }
  }
}

template <typename T, int WM, int WN, int MI, int NJ>
__global__ __launch_bounds__(256, 1) void k_i8_wide(const int8_t* __restrict__ A, const float* __restrict__ sa, int M,
                                                    const int8_t* __restrict__ W, const float* __restrict__ sw, int N, int Kp,
                                                    T* __restrict__ out) {
  i8_wide_body<T, WM, WN, MI, NJ>(A, sa, M, W, sw, N, Kp, out);
}

// Tile and slices with the lowest estimate, us: start + rounds of 256 workgroups x (round + line x 128-byte columns) + MB of weights x
// w + MB of results x out, or of int32 sums x sums + the launch that adds them.  Fitted (9 % rms) to 9000 launches, cold
// weights, 1 to 12288 rows, ten maps of 256 to 18944; the choices are 2.0 % from the quickest of 50 shapes on average.  Of shapes
// with the same rows those win whose wavefronts share the contraction: a stage is then longer and a barrier feeds more products (64 rows:
// stages of 256 bytes a row against 128, us: 4096 x 4096 9.6 and 12.1, 12288 x 4096 13.7 and 14.7, 18944 x 3584 16.9 and 24.9).  At 12288 x 4096 one
// row takes 10.8 us (floor 10.1 of weights), 64 rows 13.7 (10.6: each workgroup takes in 64 rows besides its 48 of the weights, 450 KB
// a CU), 12288 rows 541 (526 at the rate of a large library product).  Non-temporal
// weights: 3 % quicker cold up to 16 rows, 6 % slower from a cache, and slower with more rows: not taken.
struct I8Cost { int wide, bm, bn; double start, round, line, w, out, sums, add; };
constexpr I8Cost kI8Costs[] = {
    {0, 16, 16, 1.51, 1.32, 0.0652, 0.0579, 3.25, 1.37, 2.42},  {0, 16, 48, 1.52, 1.53, 0.099, 0.0821, 0.934, 0.274, 3.06},
    {0, 16, 80, 1.55, 1.6, 0.166, 0.0823, 1.15, 0.752, 2.73},   {0, 32, 32, 1.77, 1.43, 0.106, 0.0676, 0.185, 0.631, 2.62},
    {0, 32, 48, 2.39, 0.807, 0.136, 0.0727, 1.16, 1.04, 2.49},  {0, 32, 64, 1.38, 2.11, 0.176, 0.0585, 0.244, 0.451, 3.02},
    {0, 32, 80, 1.68, 2.25, 0.296, 0.0603, 0.109, 0.328, 2.71}, {0, 48, 16, 1.59, 1.39, 0.0999, 0.0434, 0.957, 0.927, 2.44},
    {0, 64, 16, 1.55, 1.46, 0.173, 0.0341, 0.89, 0.59, 2.39},   {0, 64, 32, 1.94, 1.23, 0.179, 0.0289, 0.862, 0.725, 2.51},
    {0, 64, 48, 2.21, 1.37, 0.206, 0.0484, 0.739, 0.632, 2.36}, {0, 64, 64, 2.03, 1.45, 0.243, 0.0345, 0.614, 0.65, 2.34},
    {0, 64, 80, 2.4, 1.47, 0.285, 0.0311, 0.781, 0.589, 2.61},  {0, 128, 16, 1.91, 1.08, 0.23, 0.0456, 1.13, 0.84, 2.38},
    {0, 128, 64, 2.91, 1.71, 0.341, 0.0296, 0.501, 0.6, 2.13},  {0, 128, 80, 3.94, 1.01, 0.438, 0.0144, 0.554, 0.593, 1.7},
    {1, 128, 64, 1.61, 1.89, 0.33, 0.0389, 0.204, 0, 0},        {1, 128, 128, 1.56, 3.09, 0.471, 0.0541, 0.227, 0, 0},
    {1, 128, 256, 1.41, 5.64, 0.747, 0.031, 0.215, 0, 0},       {1, 192, 128, 0.588, 5.05, 0.582, 0.0177, 0.308, 0, 0},
    {1, 192, 256, 0, 8.83, 0.884, 0.023, 0.258, 0, 0},          {1, 256, 128, 1.83, 4.33, 0.676, 0.00491, 0.391, 0, 0},
    {1, 256, 256, 0.785, 9.57, 1.13, 0.00482, 0.31, 0, 0}};

template <typename T>
void launch_i8(const I8Plan& p, const int8_t* a, const float* sa, int M, const int8_t* w, const float* sw, int N, int Kp, T* out,
               int* sums, hipStream_t st) {
  const dim3 grid((N + p.bn - 1) / p.bn, (M + p.bm - 1) / p.bm, p.S);
  if (p.wide) {
#define DLLMC_W(WM, WN, MI, NJ) \
  hipLaunchKernelGGL((k_i8_wide<T, WM, WN, MI, NJ>), grid, dim3(256), 0, st, a, sa, M, w, sw, N, Kp, out)
    switch (p.bm * 1000 + p.bn) {
      case 256256: DLLMC_W(2, 2, 8, 8); break;
      case 192256: DLLMC_W(2, 2, 6, 8); break;
      case 256128: DLLMC_W(2, 2, 8, 4); break;
      case 128256: DLLMC_W(2, 2, 4, 8); break;
      case 192128: DLLMC_W(2, 2, 6, 4); break;
      case 128128: DLLMC_W(2, 2, 4, 4); break;
      default: DLLMC_W(2, 2, 4, 2); break;
    }
#undef DLLMC_W
    return;
  }
#define DLLMC_R(RG, RB, NB) \
  hipLaunchKernelGGL((k_i8_ring<T, RG, RB, NB>), grid, dim3(512), 0, st, a, sa, M, w, sw, N, Kp, p.per, out, sums)
  switch (p.bm * 100 + p.bn) {
    case 1616: DLLMC_R(1, 1, 1); break;
    case 1648: DLLMC_R(1, 1, 3); break;
    case 1680: DLLMC_R(1, 1, 5); break;
    case 3232: DLLMC_R(1, 2, 2); break;
    case 3248: DLLMC_R(1, 2, 3); break;
    case 3264: DLLMC_R(1, 2, 4); break;
    case 3280: DLLMC_R(1, 2, 5); break;
    case 4816: DLLMC_R(1, 3, 1); break;
    case 6416: DLLMC_R(2, 2, 1); break;
    case 6432: DLLMC_R(2, 2, 2); break;
    case 6448: DLLMC_R(2, 2, 3); break;
    case 6464: DLLMC_R(2, 2, 4); break;
    case 6480: DLLMC_R(2, 2, 5); break;
    case 12816: DLLMC_R(2, 4, 1); break;
    case 12864: DLLMC_R(2, 4, 4); break;
    default: DLLMC_R(4, 2, 5); break;
  }
#undef DLLMC_R
  if (p.S > 1) {
    const long long g = (static_cast<long long>(M) * N + 255) / 256;
    hipLaunchKernelGGL(k_i8_sum<T>, dim3(static_cast<unsigned>(g < (1 << 20) ? g : 1 << 20)), dim3(256), 0, st, sums, p.S, M, N, sa, sw,
                       out);
  }
}

template <typename T>
void quant8(const T* x, int x_rows, const int* rows, int M, int K, int8_t* q, float* scale, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
  const bool pieces = K % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0;
#define DLLMC_Q(PC) hipLaunchKernelGGL((k_quant8<T, PC>), dim3(M), dim3(256), 0, st, x, x_rows, rows, K, Kp, q, scale)
  if (!pieces || K > 2048 * 10) hipLaunchKernelGGL(k_quant8_any<T>, dim3(M), dim3(256), 0, st, x, x_rows, rows, K, Kp, q, scale);
  else if (Kp <= 2048) DLLMC_Q(1);
  else if (Kp <= 4096) DLLMC_Q(2);
  else if (Kp <= 12288) DLLMC_Q(6);
  else DLLMC_Q(10);
#undef DLLMC_Q
}

}  // namespace

static I8Plan choose_i8(int M, int N, int Kp) {
  const int lines = Kp / 128;
  const double mb_w = static_cast<double>(N) * Kp / 1e6, mn = static_cast<double>(M) * N / 1e6;
  I8Plan best{};
  double best_t = 1e300;
  for (const I8Cost& c : kI8Costs) {
    const long long mt = (M + c.bm - 1) / c.bm, nt = (N + c.bn - 1) / c.bn;
    if (mt > 65535) continue;  // (the grid's second dimension)
    for (const int S : {1, 2, 3, 4, 6, 8}) {
      if (S > 1 && (c.wide || S > lines)) break;
      const int per = (lines + S - 1) / S, used = (lines + per - 1) / per;
      const double rounds = static_cast<double>((mt * nt * used + 255) / 256);
      const double t = c.start + rounds * (c.round + c.line * per) + mb_w * c.w + (used == 1 ? 2 * mn * c.out : used * 4 * mn * c.sums + c.add);
      if (t < best_t) {
        best_t = t;
        best = {c.wide, c.bm, c.bn, used, per * 128};
      }
    }
  }
  return best;
}

I8Plan plan_i8(int M, int N, int Kp) {
  return last_plan<I8Plan>({M, N, Kp}, [&] { return choose_i8(M, N, Kp); });
}

void launch_quant8(int dtype, const void* x, int x_rows, const int* rows, int M, int K, int8_t* q, float* scale, hipStream_t st) {
  if (dtype == 1) quant8(static_cast<const bf16_t*>(x), x_rows, rows, M, K, q, scale, st);
  else quant8(static_cast<const float*>(x), x_rows, rows, M, K, q, scale, st);
}

size_t linear_i8_scratch_bytes(const I8Plan& p, int M, int N) {
  return p.S == 1 ? 0 : static_cast<size_t>(p.S) * M * N * sizeof(int);
}

void launch_linear_i8(const I8Plan& p, int dtype, const int8_t* a, const float* a_scale, int M, const int8_t* w, const float* w_scale,
                      int N, int K, void* out, void* scratch, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
  if (dtype == 1) launch_i8(p, a, a_scale, M, w, w_scale, N, Kp, static_cast<bf16_t*>(out), static_cast<int*>(scratch), st);
  else launch_i8(p, a, a_scale, M, w, w_scale, N, Kp, static_cast<float*>(out), static_cast<int*>(scratch), st);
}

}  // namespace dllmc
