// Matrices of 4-bit blocks: rows in and out, and their product.
//
// A block is 32 neighbouring elements of a row: codes of 4 bits (sign, and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6) times one power of two, as
// in a 4-bit cache.  The scaled matrix instructions multiply codes exactly and take both blocks' powers of two along, so the only roundings of
// out[i][j] = sum_k a[i][k] w[j][k] are those of float32 sums and of the result.
//
// Times here: the best of several means of 20 launches behind one another.
#include <type_traits>

#include "mx4.hpp"

namespace dllmc {

namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---- rows in and out --------------------------------------------------------------------------------------
// A workgroup per row; four lanes take a block.  Bound by the bytes: 12288 x 4096 bf16 into blocks 24.8 us (5.1 TB/s), back 21.9 (5.8); 12288 x 4049
// 27.1 and 23.4.
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_store(const T* __restrict__ x, int x_rows, const int* __restrict__ rows, int K, Mx4Tensor out) {
  const int i = blockIdx.x;
  const int row = rows ? rows[i] : i, len = static_cast<unsigned>(row) < static_cast<unsigned>(x_rows) ? K : 0;  // (no row: zeros)
  const T* r = x + static_cast<size_t>(len ? row : 0) * K;
  for (int t = threadIdx.x * 8; t < out.Kp; t += 2048) {
    float v[8];
    load8(r, t, len, v);
    const uint32_t scale = kv4_scale_byte(block32_top(v));
    *reinterpret_cast<uint32_t*>(out.codes + static_cast<size_t>(i) * (out.Kp / 2) + t / 2) = mx4_codes(v, scale);
    if (t % 32 == 0) out.scales[mx4_scale_at(i, t, out.Kp)] = static_cast<uint8_t>(scale);
  }
}

template <typename T>
__global__ __launch_bounds__(256) void k_mx4_load(Mx4Tensor in, const int* __restrict__ rows, int K, T* __restrict__ out) {
  const int i = blockIdx.x, r = rows ? rows[i] : i;
  const bool ok = static_cast<unsigned>(r) < static_cast<unsigned>(in.rows);
  T* o = out + static_cast<size_t>(i) * K;
  for (int t = threadIdx.x * 8; t < K; t += 2048) {
    float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (ok) {
      const uint32_t w = *reinterpret_cast<const uint32_t*>(in.codes + static_cast<size_t>(r) * (in.Kp / 2) + t / 2);
      const uint4 b = __builtin_bit_cast(uint4, kv4_expand(w, in.scales[mx4_scale_at(r, t, in.Kp)]));
      const uint32_t f[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        v[2 * h] = __uint_as_float(f[h] << 16);
        v[2 * h + 1] = __uint_as_float(f[h] & 0xffff0000u);
      }
    }
    store8(o, t, K, v);
  }
}

// 8-bit rows back: q * scale, rounded to T
template <typename T>
__global__ __launch_bounds__(256) void k_load8(const int8_t* __restrict__ q, const float* __restrict__ scale, int q_rows, int K, int Kp,
                                               const int* __restrict__ rows, T* __restrict__ out) {
  const int i = blockIdx.x, r = rows ? rows[i] : i;
  const bool ok = static_cast<unsigned>(r) < static_cast<unsigned>(q_rows);
  T* o = out + static_cast<size_t>(i) * K;
  const float s = ok ? scale[r] : 0.f;
  for (int t = threadIdx.x * 8; t < K; t += 2048) {
    const uint2 w = ok ? *reinterpret_cast<const uint2*>(q + static_cast<size_t>(r) * Kp + t) : make_uint2(0, 0);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = static_cast<float>(static_cast<int8_t>((e < 4 ? w.x : w.y) >> (e % 4 * 8))) * s;
    store8(o, t, K, v);
  }
}

// ---- the product ------------------------------------------------------------------------------------------
// Products are taken as W A^T, so that a lane holds neighbouring columns of a row.  Rows past M and N repeat the last one (their scales are those
// of the last rows' group) and are dropped at the store.
// (A 4-bit operand is the first four registers.  LDS is read as i32x4: before a copied struct the compiler waits for every load into LDS.)
__device__ __forceinline__ i32x8 operand(const i32x4& u) { return i32x8{u[0], u[1], u[2], u[3], 0, 0, 0, 0}; }

typedef const __attribute__((address_space(1))) int* global_int_ptr;  // (a pointer put together from registers: a flat load otherwise)

// four neighbouring results of a row at any address, those before column N
typedef uint32_t u32x2_at2 __attribute__((ext_vector_type(2), aligned(2)));
template <typename T>
__device__ __forceinline__ void store4(T* p, int n, int N, float a, float b, float c, float d) {
  if (n + 4 <= N) {
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_at2*>(p) = u32x2_at2{pack_bf16x2(a, b), pack_bf16x2(c, d)};
    else *reinterpret_cast<u32x4_at4*>(p) = u32x4_at4{__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d)};
  } else {
    if (n < N) stf(p, a);
    if (n + 1 < N) stf(p + 1, b);
    if (n + 2 < N) stf(p + 2, c);
  }
}

// ---- few rows -----------------------------------------------------------------------------------------
// k_mx4_ring<RG, RB, NB>: tile = 16 RG RB rows x 16 NB weight rows, one workgroup of eight wavefronts per CU.  Codes and scales of both operands go
// from global memory straight into LDS through a ring of stages.  RG wavefronts take 16 RB rows each, 8 / RG share the
// contraction: a stage is 64 * 8 / RG bytes of every row's codes, and a wavefront multiplies its own 64 of them, 128 elements, with one 16 x 16 x 128
// product a block.  Their sums meet in LDS at the end, in one order.  Slice blockIdx.z of the contraction; with one slice results leave
// rounded, else as float32 sums for k_mx4_sum.  One row of 12288 x 4096 takes 7.5 us with weights from memory, 16 rows the same, 64 rows 10.1 (6.9, 7.0 and
// 8.8 with weights from the memory-side cache); the weights' bytes are 5.4 at a copy's rate, a launch alone some 2.
template <int RG, int RB, int NB> struct Mx4Ring {
  static constexpr int KW = 8 / RG, SS = KW / 2;  // wavefronts along the contraction, 128-byte lines of a stage
  static constexpr int BM = 16 * RG * RB, R = BM + 16 * NB;
  static constexpr int kUnits = R / 16, UL = (kUnits + 7) / 8;  // 16 rows' scales of a line (128 bytes), loads of eight of them
  static constexpr int kCodes = R * 8 * SS, kStage = kCodes + UL * SS * 64;  // 16-byte slots
  static constexpr int kFit = (160 * 1024) / (kStage * 16), NST = kFit > 8 ? 8 : kFit;
  static constexpr int TC = R / 8 * SS, T = TC + UL * SS;  // load instructions of a stage, those of the codes first
  static constexpr int L = T / 8, LR = T % 8;              // per wavefront, one more for the first LR
};

template <typename T, int RG, int RB, int NB>
__device__ __forceinline__ void mx4_ring_body(const Mx4Tensor& a, const Mx4Tensor& w, int per_slice, T* __restrict__ out,
                                              float* __restrict__ sums) {
  typedef Mx4Ring<RG, RB, NB> S;
  constexpr int NST = S::NST, SS = S::SS, R = S::R, BM = S::BM;
  static_assert(SS >= 1 && NST >= 2, "");
  __shared__ __attribute__((aligned(1024))) uint4 lds[NST][S::kStage];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 16, lg = lane / 16;
  const int wr = wave % RG, kk = wave / RG;
  const int M = a.rows, N = w.rows, row_bytes = a.Kp / 2, all_lines = a.Kp / 256;
  int col_tile, row_tile;
  xcd_tile_map(col_tile, row_tile);
  const int m0 = row_tile * BM, n0 = col_tile * 16 * NB;
  const int line0 = blockIdx.z * per_slice, lines = min(all_lines, line0 + per_slice) - line0;
  const int nkt = (lines + SS - 1) / SS;

  // loader: instruction q < TC of a stage copies the codes of rows 8 (q % (R/8)) .. + 7 of line q / (R/8) (lane: row lane/8, slot lane%8, chunk
  // slot ^ row % 8), the others the scales of eight units of a line (lane: unit lane/8, and of its [2][16] rows' four bytes the lane%8-th 16)
  const uint8_t* src[S::L + 1];
  int sub[S::L + 1], step[S::L + 1];
#pragma unroll
  for (int j = 0; j < S::L + 1; ++j) {
    const int q = min(wave + 8 * j, S::T - 1);
    if (q < S::TC) {
      const int r = q % (R / 8) * 8 + lane / 8;
      const uint8_t* row = r < BM ? a.codes + static_cast<size_t>(min(m0 + r, M - 1)) * row_bytes
                                  : w.codes + static_cast<size_t>(min(n0 + r - BM, N - 1)) * row_bytes;
      src[j] = row + static_cast<size_t>(line0) * 128 + ((lane % 8) ^ (lane / 8)) * 16;
      sub[j] = q / (R / 8);
      step[j] = 128;
    } else {
      const int u = min((q - S::TC) % S::UL * 8 + lane / 8, S::kUnits - 1);
      const Mx4Tensor& t = u < BM / 16 ? a : w;
      const int r = min(u < BM / 16 ? m0 + u * 16 : n0 + u * 16 - BM, (t.rows - 1) / 16 * 16);  // (a unit's first row)
      src[j] = t.scales + (static_cast<size_t>(r / 32) * all_lines + line0) * 256 + lane % 8 / 4 * 128 + r % 32 * 4 + lane % 4 * 16;
      sub[j] = (q - S::TC) / S::UL;
      step[j] = 256;
    }
  }
  // the walk starts at a stage that depends on the column tile: unrotated every load in flight has the same address bits
  // below the row pitch
  const int rot = (col_tile % 8 * 8 + col_tile / 8) % nkt;
  auto issue_one = [&](int stage, int kt, int j) {
    const int q = wave + 8 * j;
    const int line = min(kt * SS + sub[j], lines - 1);  // (lines past the last one repeat it and are not multiplied)
    __builtin_amdgcn_global_load_lds(src[j] + static_cast<size_t>(line) * step[j], &lds[stage][q * 64], 16, 0, 0);
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

  f32x4 acc[RB][NB];
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
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
      // the scale of block kk % 2 * 4 + lg of a line's eight: bytes [lg % 2][row][kk % 2 * 2 + lg / 2] of its unit
      const uint8_t* scale = reinterpret_cast<const uint8_t*>(&lds[stage][S::kCodes + kk / 2 * S::UL * 64]) + lg % 2 * 64 + ln * 4 + kk % 2 * 2 + lg / 2;
      const int c = kk % 2 * 4 + lg;
      i32x8 af[RB], bf[NB];
      int as[RB], bs[NB];
#pragma unroll
      for (int i = 0; i < RB; ++i) {
        const int r = (wr * RB + i) * 16 + ln;
        af[i] = operand(__builtin_bit_cast(i32x4, base[r * 8 + (c ^ (r % 8))]));
        as[i] = scale[(wr * RB + i) * 128];
      }
#pragma unroll
      for (int j = 0; j < NB; ++j) {
        const int r = BM + j * 16 + ln;
        bf[j] = operand(__builtin_bit_cast(i32x4, base[r * 8 + (c ^ (r % 8))]));
        bs[j] = scale[(BM / 16 + j) * 128];
      }
#pragma unroll
      for (int j = 0; j < NB; ++j)
#pragma unroll
        for (int i = 0; i < RB; ++i)
          acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bf[j], af[i], acc[i][j], 4, 4, 0, bs[j], 0, as[i]);
    }
    stage = stage + 1 < NST ? stage + 1 : 0;
  }
  // hand-over: the sums of the wavefronts that shared a row group, added by RG * RB * NB / 8 blocks per wavefront
  __syncthreads();
  f32x4* red = reinterpret_cast<f32x4*>(&lds[0][0]);
  static_assert(8 * RB * NB * 64 <= NST * S::kStage, "hand-over fits the ring");
#pragma unroll
  for (int i = 0; i < RB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) red[((kk * RG + wr) * RB * NB + i * NB + j) * 64 + lane] = acc[i][j];
  __syncthreads();
  for (int x = wave; x < RG * RB * NB; x += 8) {  // block x = (row group, i, j)
    f32x4 sum = red[x * 64 + lane];
#pragma unroll
    for (int v = 1; v < S::KW; ++v) sum += red[(v * RG * RB * NB + x) * 64 + lane];
    const int j = x % NB, rb = x / NB;
    const int m = m0 + rb * 16 + ln, n = n0 + j * 16 + lg * 4;
    if (m >= M || n >= N) continue;
    if (gridDim.z == 1) store4(out + static_cast<size_t>(m) * N + n, n, N, sum[0], sum[1], sum[2], sum[3]);
    else store4(sums + (static_cast<size_t>(blockIdx.z) * M + m) * N + n, n, N, sum[0], sum[1], sum[2], sum[3]);
  }
}

template <typename T, int RG, int RB, int NB>
__global__ __launch_bounds__(512) void k_mx4_ring(Mx4Tensor a, Mx4Tensor w, int per_slice, T* __restrict__ out, float* __restrict__ sums) {
  mx4_ring_body<T, RG, RB, NB>(a, w, per_slice, out, sums);
}

// out = sum of S slices, in their order
template <typename T>
__global__ __launch_bounds__(256) void k_mx4_sum(const float* __restrict__ sums, int S, long long all, T* __restrict__ out) {
  for (long long p = static_cast<long long>(blockIdx.x) * 256 + threadIdx.x; p < all; p += static_cast<long long>(gridDim.x) * 256) {
    float v = sums[p];
    for (int s = 1; s < S; ++s) v += sums[s * all + p];
    stf(out + p, v);
  }
}

// ---- many rows ----------------------------------------------------------------------------------------
// k_mx4_wide<MI, NJ>: tile = 64 MI rows x 64 NJ columns, four wavefronts, one per SIMD, of 32 MI x 32 NJ results each, in 32 x 32 x 64
// products (9.3 PFLOP/s on zeros with a wavefront per SIMD, 6.6 on random operands; 16 x 16 x 128 5.3 and 5.0: their issue takes longer).
// A step is 128 bytes, 256 elements, of every row.  Operands, rings and the order of reads and loads are k_gemm_wide's.  A step's scales
// are one more load of every wavefront (16 groups of 32 rows' 256 bytes, of rows first, then columns) and travel with the ring of X; the tile of
// 256 x 256 fills LDS (two stages of each operand instead would leave Y half a step to land), and its wavefronts load their own blocks' scales
// into registers, a step ahead.
// What bounds it is the card's power: 12288 x 12288 x 4096 takes 297 us (4.2 PFLOP/s), of zeros 206; a step of random operands 1.6 us at 1.8 GHz (bare
// products 1.24), of zeros 1.0 (0.88).  MFMAs run in 60 % of the launch's cycles, in 73 % of those of a copy that ends with its main loop and takes
// 260 us: the results cost 37, less than a fill of as many bytes alone (43); delaying half of the CUs, so that some store while others
// multiply, gave 2 % at this size.
template <int BM, int BN> struct Mx4Rings {
  static constexpr bool kInLds = BM + BN < 512;
  static constexpr int kRoom = kInLds ? 1280 - 4 * 32 : 1280;  // rows of 128 bytes, beside four stages of scales
  static constexpr int kWhole = kRoom / (BM + BN);
  static constexpr int kLeft = kRoom - kWhole * (BM + BN);
  static constexpr int DA0 = kWhole + (kLeft >= BM && (BM >= BN || kLeft < BN) ? 1 : 0);
  static constexpr int DB0 = kWhole + (DA0 == kWhole && kLeft >= BN ? 1 : 0);
  static constexpr int DA = DA0 < 4 ? DA0 : 4, DB = DB0 < 4 ? DB0 : 4;
};

template <typename T, int MI, int NJ>
__device__ __forceinline__ void mx4_wide_body(const Mx4Tensor& a, const Mx4Tensor& w, T* __restrict__ out) {
  constexpr int BM = 64 * MI, BN = 64 * NJ, LA = BM / 32, LB = BN / 32;
  typedef Mx4Rings<BM, BN> Ring;
  // X, the operand with the shallower ring, has its next block loaded in the second half of a step, Y in the first half of the
  // next one; the barrier stands between the halves
  constexpr int DA = Ring::DA, DB = Ring::DB;
  constexpr bool XB = DA >= DB, kInLds = Ring::kInLds;
  constexpr int DX = XB ? DB : DA, DY = XB ? DA : DB, LX = (XB ? LB : LA) + (kInLds ? 1 : 0), LY = XB ? LA : LB;
  constexpr int kSlotA = BM * 8, kSlotB = BN * 8, kScales = DA * kSlotA + DB * kSlotB, kLds = kScales + (kInLds ? DX * 256 : 0);
  static_assert(kLds * sizeof(uint4) <= 160 * 1024 && DX >= 2 && DY <= DX + 1, "LDS of one CU");
  __shared__ __attribute__((aligned(1024))) uint4 lds[kLds];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64;
  const int ln = lane % 32, lg = lane / 32;
  const int wm = wave / 2, wn = wave % 2;
  const int M = a.rows, N = w.rows, row_bytes = a.Kp / 2, nkt = a.Kp / 256;
  int col_tile, row_tile;
  xcd_tile_map_blocked(col_tile, row_tile);
  const int m0 = row_tile * BM, n0 = col_tile * BN;

  // Chunk c of a tile's row r lies in slot c ^ turn(r): rows 0 .. 7 and 16 .. 23 of 32, whose reads share a cycle, meet in no bank (4 cycles a read; with
  // r % 8 in its place 8, counted).
  auto turn = [](int r) { return (r >> 1 & 3) | (r >> 2 & 4); };
  // loader: wavefront v issues instructions L v .. L v + L - 1 of an operand, 8 rows each: a scalar base and a lane offset
  // (rows past the last one: the last one; groups of scales likewise)
  const char *abase[LA], *bbase[LB], *asbase[MI], *bsbase[NJ];
  uint32_t aoff[LA], boff[LB];
#pragma unroll
  for (int j = 0; j < LA; ++j) {
    const int r = min(m0 + 8 * (LA * wave + j), M - 1);
    abase[j] = wave_uniform_ptr(reinterpret_cast<const char*>(a.codes + static_cast<size_t>(r) * row_bytes));
    aoff[j] = static_cast<uint32_t>(min(lane / 8, M - 1 - r) * row_bytes + (lane % 8 ^ turn(8 * (LA * wave + j) + lane / 8)) * 16);
  }
#pragma unroll
  for (int j = 0; j < LB; ++j) {
    const int r = min(n0 + 8 * (LB * wave + j), N - 1);
    bbase[j] = wave_uniform_ptr(reinterpret_cast<const char*>(w.codes + static_cast<size_t>(r) * row_bytes));
    boff[j] = static_cast<uint32_t>(min(lane / 8, N - 1 - r) * row_bytes + (lane % 8 ^ turn(8 * (LB * wave + j) + lane / 8)) * 16);
  }
  // scales: in LDS one load of four groups a wavefront, else one of a group for each of its blocks
  const int group = min(wave * 4 + lane / 16, (BM + BN) / 32 - 1);
  const bool of_a = group < BM / 32;
  const int g32 = min(of_a ? m0 / 32 + group : n0 / 32 + group - BM / 32, ((of_a ? M : N) - 1) / 32);
  const uint8_t* ssrc = (of_a ? a.scales : w.scales) + static_cast<size_t>(g32) * nkt * 256 + lane % 16 * 16;
#pragma unroll
  for (int i = 0; i < MI; ++i)
    asbase[i] = wave_uniform_ptr(reinterpret_cast<const char*>(a.scales) + static_cast<size_t>(min(m0 / 32 + wm * MI + i, (M - 1) / 32)) * nkt * 256);
#pragma unroll
  for (int j = 0; j < NJ; ++j)
    bsbase[j] = wave_uniform_ptr(reinterpret_cast<const char*>(w.scales) + static_cast<size_t>(min(n0 / 32 + wn * NJ + j, (N - 1) / 32)) * nkt * 256);
  const int rot = (((blockIdx.x + gridDim.x * blockIdx.y) & 7) * nkt) >> 3;  // the walk starts at a step that depends on the XCD
  auto kof = [&](int kt) { const int k = kt + rot; return k < nkt ? k : k - nkt; };
  auto issue_a = [&](int slot, int k, int j) {
    uint32_t o = aoff[j];
    asm volatile("" : "+v"(o));
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(wave_uniform_ptr(abase[j] + k * 128) + o),
                                     &lds[slot * kSlotA + (LA * wave + j) * 64], 16, 0, 0);
  };
  auto issue_b = [&](int slot, int k, int j) {
    uint32_t o = boff[j];
    asm volatile("" : "+v"(o));
    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(wave_uniform_ptr(bbase[j] + k * 128) + o),
                                     &lds[DA * kSlotA + slot * kSlotB + (LB * wave + j) * 64], 16, 0, 0);
  };
  auto issue_x = [&](int slot, int k, int j) {
    if (kInLds && j == LX - 1)
      __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4*>(ssrc + k * 256), &lds[kInLds ? kScales + slot * 256 + wave * 64 : 0], 16, 0, 0);
    else if (XB) issue_b(slot, k, j);
    else issue_a(slot, k, j);
  };
  auto issue_y = [&](int slot, int k, int j) { if (XB) issue_a(slot, k, j); else issue_b(slot, k, j); };
  int as[2][MI], bs[2][NJ];  // scales of this step and of the next one
  auto read_scales = [&](int slot_x, int to) {
    const int* s = reinterpret_cast<const int*>(&lds[kInLds ? kScales + slot_x * 256 : 0]) + lane;
#pragma unroll
    for (int i = 0; i < MI; ++i) as[to][i] = s[(wm * MI + i) * 64];
#pragma unroll
    for (int j = 0; j < NJ; ++j) bs[to][j] = s[(2 * MI + wn * NJ + j) * 64];
  };
  auto load_scales = [&](int to, int k) {
#pragma unroll
    for (int i = 0; i < MI; ++i) as[to][i] = reinterpret_cast<global_int_ptr>(reinterpret_cast<uintptr_t>(wave_uniform_ptr(asbase[i] + k * 256)))[lane];
#pragma unroll
    for (int j = 0; j < NJ; ++j) bs[to][j] = reinterpret_cast<global_int_ptr>(reinterpret_cast<uintptr_t>(wave_uniform_ptr(bsbase[j] + k * 256)))[lane];
  };
  // The first blocks in the order of the main loop: X(t), Y(t + DY - DX); Y(DY - 1) goes out in step 0.  Straight code, whatever nkt is (a
  // step that there is not: the last one's block again, which nobody reads): over loads that may or may not have been issued the
  // compiler would wait for the scales in every step.
  auto block_x = [&](int t) {
    const int k = kof(min(t, nkt - 1));
#pragma unroll
    for (int j = 0; j < LX; ++j) issue_x(t, k, j);
  };
  auto block_y = [&](int t) {
    const int k = kof(min(t, nkt - 1));
#pragma unroll
    for (int j = 0; j < LY; ++j) issue_y(t, k, j);
  };
  if constexpr (!kInLds) {
    load_scales(0, kof(0));
    load_scales(1, kof(min(1, nkt - 1)));
    __builtin_amdgcn_sched_barrier(0);
  }
#pragma unroll
  for (int t = 0; t < DY - DX; ++t) block_y(t);
#pragma unroll
  for (int t = 0; t < DX - 1; ++t) {
    block_x(t);
    block_y(t + DY - DX);
  }
  block_x(DX - 1);
  wait_vmcnt_lds<(DX - 1) * LX + (DY > DX ? DX - 1 : DX - 2) * LY>();
  __builtin_amdgcn_s_barrier();
  f32x16 acc[MI][NJ];
#pragma unroll
  for (int i = 0; i < MI; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
  i32x4 af[2][2][MI], bf[2][2][NJ];  // fragments of a half step: two products' 64 elements each
  auto read = [&](int slot_a, int slot_b, int half, int q) {
    const int s = q / (MI + NJ), x = q % (MI + NJ), c = (half * 2 + s) * 2 + lg;
    if (x < NJ) {
      const int r = wn * (NJ * 32) + x * 32 + ln;
      bf[half][s][x] = __builtin_bit_cast(i32x4, lds[DA * kSlotA + slot_b * kSlotB + r * 8 + (c ^ turn(r))]);
    } else {
      const int r = wm * (MI * 32) + (x - NJ) * 32 + ln;
      af[half][s][x - NJ] = __builtin_bit_cast(i32x4, lds[slot_a * kSlotA + r * 8 + (c ^ turn(r))]);
    }
  };
  constexpr int kReads = 2 * (MI + NJ), kMfma = 2 * MI * NJ;
  constexpr int kSpan = kMfma * 3 / 4;  // MFMAs that reads and loads are spread over
  auto half_step = [&](auto half_, auto&& between) {
    constexpr int half = decltype(half_)::value;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#define DLLMC_MFMA(B) \
  __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(bf[half][s][j]), operand(af[half][s][i]), acc[i][j], 4, 4, B, bs[0][j], B, as[0][i])
          acc[i][j] = half * 2 + s == 0 ? DLLMC_MFMA(0) : half * 2 + s == 1 ? DLLMC_MFMA(1) : half * 2 + s == 2 ? DLLMC_MFMA(2) : DLLMC_MFMA(3);
#undef DLLMC_MFMA
          __builtin_amdgcn_sched_barrier(0);
          between((s * MI + i) * NJ + j);
          __builtin_amdgcn_sched_barrier(0);
        }
  };
#pragma unroll
  for (int q = 0; q < kReads; ++q) read(0, 0, 0, q);
  if constexpr (kInLds) read_scales(0, 0);
  int s_a = 0, s_b = 0, s_y = DY - 1;
  // step kt with `left` steps to come (DX: that many or more)
  auto step = [&](int kt, auto left_) {
    constexpr int left = decltype(left_)::value;
    // (the loads of scales are not counted: those behind what has to have landed only make the wait a longer one)
    constexpr int kFly = left == 0 ? 0 : (DX - 2 < left - 1 ? DX - 2 : left - 1) * LX + (DY - 2 < left - 1 ? DY - 2 : left - 1) * LY;
    const int a1 = s_a + 1 < DA ? s_a + 1 : 0, b1 = s_b + 1 < DB ? s_b + 1 : 0;
    const int ky = left >= DY - 1 ? kof(kt + DY - 1) : 0, kx = left >= DX ? kof(kt + DX) : 0;
    __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
    __builtin_amdgcn_sched_barrier(0);
    half_step(std::integral_constant<int, 0>{}, [&](int t) {
#pragma unroll
      for (int q = 0; q < kReads; ++q)
        if (1 + q * kSpan / kReads == t) read(s_a, s_b, 1, q);
#pragma unroll
      for (int l = 0; l < LY; ++l)
        if (left >= DY - 1 && l * kSpan / LY == t) issue_y(s_y, ky, l);
    });
    wait_vmcnt_lds<kFly>();
    if (left > 0) __builtin_amdgcn_s_barrier();
    half_step(std::integral_constant<int, 1>{}, [&](int t) {
      if (kInLds && left > 0 && t == 0) read_scales(XB ? b1 : a1, 1);
#pragma unroll
      for (int q = 0; q < kReads; ++q)
        if (left > 0 && 1 + q * kSpan / kReads == t) read(a1, b1, 0, q);
#pragma unroll
      for (int l = 0; l < LX; ++l)
        if (left >= DX && l * kSpan / LX == t) issue_x(XB ? s_b : s_a, kx, l);
    });
    if (left > 0) {
#pragma unroll
      for (int i = 0; i < MI; ++i) {
        as[0][i] = as[1][i];
        if (!kInLds) asm volatile("" : "+v"(as[0][i]));  // (the copy first: then the loads go to the registers that the copy has left)
      }
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        bs[0][j] = bs[1][j];
        if (!kInLds) asm volatile("" : "+v"(bs[0][j]));
      }
      if (!kInLds) {
        __builtin_amdgcn_sched_barrier(0);
        if (left > 1) load_scales(1, kof(kt + 2));
      }
    }
    s_y = XB ? s_a : s_b;
    s_a = a1;
    s_b = b1;
  };
  int kt = 0;
  for (; kt < nkt - DX; ++kt) step(kt, std::integral_constant<int, DX>{});
  if constexpr (DX > 3) { if (nkt - kt > 3) step(kt++, std::integral_constant<int, 3>{}); }
  if constexpr (DX > 2) { if (nkt - kt > 2) step(kt++, std::integral_constant<int, 2>{}); }
  if (nkt - kt > 1) step(kt++, std::integral_constant<int, 1>{});
  step(kt, std::integral_constant<int, 0>{});
  // A lane: row ln of block i, columns 8 q + 4 lg .. + 3 of block j.  Stored as they are, 16 bytes of every row at a time, they cost more than
  // a trip through LDS, 32 rows of the wavefront's columns at a time, that makes whole lines of them (12288 x 12288 x 4096: 45 us of
  // 320 for the direct stores).  Rows are 16 bytes further apart than they are long: no two lanes meet in a bank.
  constexpr int kPer = 16 / sizeof(T), kRow = NJ * 32 / kPer;  // elements and slots of 16 bytes
  constexpr int kPitch = kRow + 1;
  static_assert(4 * 32 * kPitch <= DA * kSlotA + DB * kSlotB, "results fit the ring");
  __syncthreads();
  uint4* mine = lds + wave * 32 * kPitch;
#pragma unroll
  for (int i = 0; i < MI; ++i) {
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x16& v = acc[i][j];
        T* to = reinterpret_cast<T*>(mine + ln * kPitch) + j * 32 + q * 8 + lg * 4;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(v[4 * q], v[4 * q + 1]), pack_bf16x2(v[4 * q + 2], v[4 * q + 3]));
        else *reinterpret_cast<float4*>(to) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
    for (int s = 0; s < 32 * kRow / 64; ++s) {
      const int at = s * 64 + lane, r = at / kRow, c = at % kRow;
      const int m = m0 + wm * (MI * 32) + i * 32 + r, n = n0 + wn * (NJ * 32) + c * kPer;
      const i32x4 v = __builtin_bit_cast(i32x4, mine[r * kPitch + c]);
      T* to = out + static_cast<size_t>(m) * N + n;
      if (m >= M) continue;
      if (n + kPer <= N) {
        *reinterpret_cast<typename std::conditional<sizeof(T) == 2, u32x4_at2, u32x4_at4>::type*>(to) = __builtin_bit_cast(u32x4_at4, v);
      } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
          if (n + e < N) {
            const uint32_t w = static_cast<uint32_t>(v[e * sizeof(T) / 4]);
            if constexpr (sizeof(T) == 2) to[e] = static_cast<bf16_t>(e % 2 ? w >> 16 : w);
            else to[e] = __uint_as_float(w);
          }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_sched_barrier(0);  // (no addresses of later rows beside the accumulators)
  }
}

template <typename T, int MI, int NJ>
__global__ __launch_bounds__(256, 1) void k_mx4_wide(Mx4Tensor a, Mx4Tensor w, T* __restrict__ out) {
  mx4_wide_body<T, MI, NJ>(a, w, out);
}

}  // namespace

void launch_quant_mx4(int dtype, const void* x, int x_rows, const int* rows, int M, int K, Mx4Tensor out, hipStream_t st) {
  if (dtype == 1) hipLaunchKernelGGL(k_mx4_store<bf16_t>, dim3(M), dim3(256), 0, st, static_cast<const bf16_t*>(x), x_rows, rows, K, out);
  else hipLaunchKernelGGL(k_mx4_store<float>, dim3(M), dim3(256), 0, st, static_cast<const float*>(x), x_rows, rows, K, out);
}

void launch_mx4_load(int dtype, Mx4Tensor in, const int* rows, int M, int K, void* out, hipStream_t st) {
  if (dtype == 1) hipLaunchKernelGGL(k_mx4_load<bf16_t>, dim3(M), dim3(256), 0, st, in, rows, K, static_cast<bf16_t*>(out));
  else hipLaunchKernelGGL(k_mx4_load<float>, dim3(M), dim3(256), 0, st, in, rows, K, static_cast<float*>(out));
}

void launch_load8(int dtype, const int8_t* q, const float* scale, int q_rows, int K, const int* rows, int M, void* out, hipStream_t st) {
  const int Kp = static_cast<int>(i8_row_bytes(K));
  if (dtype == 1) hipLaunchKernelGGL(k_load8<bf16_t>, dim3(M), dim3(256), 0, st, q, scale, q_rows, K, Kp, rows, static_cast<bf16_t*>(out));
  else hipLaunchKernelGGL(k_load8<float>, dim3(M), dim3(256), 0, st, q, scale, q_rows, K, Kp, rows, static_cast<float*>(out));
}

namespace {

// Tile and slices with the lowest estimate, us: start + rounds of 256 workgroups x (round + line x 128-byte lines) + MB of weights x w + MB of
// results x out, or of float32 sums x sums + the launch that adds them.  Fitted (4 to 9 % rms) to 2300 launches, weights from memory, 1 to 12288 rows of
// thirteen maps of 256 to 126464 outputs; the choices are 1.6 % from the quickest on average.  The shapes are those of 24 without which they
// would be further: 64 x 12288 x 4096 10.4 us (64 x 64; 9.7 of 128 x 64, 12.0 of 128 x 128, 14.4 of 32 x 64), 1280 x 18944 x 3584 53.1 in two rounds of
// 256 x 192 (58.2 of 256 x 256, 65.2 of 192 x 256, a third round for six tiles), 1 x 12288 x 4096 7.8 (16 x 48) and 11.6 (16 x 16, three rounds).
// All launches had bf16 results, and the estimate knows no type: float32 results, twice the bytes, take the same plan (12288 x 12288 x 4096 329 us for
// 297, 1280 x 18944 x 3584 56.7 for 52.6, 512 x 12288 x 4096 21.6 for 20.4).
struct Mx4Cost { int wide, bm, bn; double start, round, line, w, out, sums, add; };
constexpr Mx4Cost kMx4Costs[] = {
    {0, 16, 16, 2.44, 1.23, 0.0843, 0.0361, 0.372, 0, 2.5}, {0, 16, 48, 2.1, 1.46, 0.113, 0.0464, 0.698, 0.608, 2.37},
    {0, 16, 80, 1.38, 2.33, 0.17, 0.0594, 0, 0.377, 2.23}, {0, 32, 32, 1.99, 1.76, 0.122, 0, 0.144, 0.338, 2.4},
    {0, 32, 64, 1.16, 2.67, 0.182, 0.0382, 0, 0.439, 2.15}, {0, 64, 64, 1.02, 2.72, 0.269, 0.0261, 0.162, 0.496, 2.39},
    {0, 64, 80, 1.25, 2.88, 0.299, 0.0406, 0.274, 0.553, 2.26}, {1, 128, 64, 1.52, 1.83, 0.353, 0.0323, 0.0719, 0, 0},
    {1, 128, 128, 1.56, 1.96, 0.491, 0.0494, 0.156, 0, 0}, {1, 192, 128, 0.989, 3.06, 0.589, 0.0324, 0.139, 0, 0},
    {1, 192, 256, 0.525, 5, 0.893, 0.0587, 0.156, 0, 0}, {1, 256, 128, 0.236, 4.26, 0.694, 0.0403, 0.131, 0, 0},
    {1, 256, 192, 0.65, 4.97, 0.88, 0.0502, 0.163, 0, 0}, {1, 256, 256, 0, 6.1, 1.1, 0.0514, 0.177, 0, 0}};

template <typename T>
void launch_product(const Mx4Plan& p, Mx4Tensor a, Mx4Tensor w, T* out, float* sums, hipStream_t st) {
  const dim3 grid((w.rows + p.bn - 1) / p.bn, (a.rows + p.bm - 1) / p.bm, p.S);
  if (p.wide) {
#define DLLMC_W(MI, NJ) hipLaunchKernelGGL((k_mx4_wide<T, MI, NJ>), grid, dim3(256), 0, st, a, w, out)
    switch (p.bm * 1000 + p.bn) {
      case 256256: DLLMC_W(4, 4); break;
      case 192256: DLLMC_W(3, 4); break;
      case 256128: DLLMC_W(4, 2); break;
      case 256192: DLLMC_W(4, 3); break;
      case 192128: DLLMC_W(3, 2); break;
      case 128128: DLLMC_W(2, 2); break;
      default: DLLMC_W(2, 1); break;
    }
#undef DLLMC_W
    return;
  }
#define DLLMC_R(RG, RB, NB) hipLaunchKernelGGL((k_mx4_ring<T, RG, RB, NB>), grid, dim3(512), 0, st, a, w, p.per, out, sums)
  switch (p.bm * 100 + p.bn) {
    case 1616: DLLMC_R(1, 1, 1); break;
    case 1648: DLLMC_R(1, 1, 3); break;
    case 1680: DLLMC_R(1, 1, 5); break;
    case 3232: DLLMC_R(1, 2, 2); break;
    case 3264: DLLMC_R(1, 2, 4); break;
    case 6464: DLLMC_R(2, 2, 4); break;
    default: DLLMC_R(2, 2, 5); break;
  }
#undef DLLMC_R
  if (p.S > 1) {
    const long long all = static_cast<long long>(a.rows) * w.rows, g = (all + 255) / 256;
    hipLaunchKernelGGL(k_mx4_sum<T>, dim3(static_cast<unsigned>(g < (1 << 20) ? g : 1 << 20)), dim3(256), 0, st, sums, p.S, all, out);
  }
}

Mx4Plan choose_mx4(int M, int N, int Kp) {
  const int lines = Kp / 256;
  const double mb_w = static_cast<double>(N) * Kp / 2e6, mn = static_cast<double>(M) * N / 1e6;
  Mx4Plan best{};
  double best_t = 1e300;
  for (const Mx4Cost& c : kMx4Costs) {
    const long long mt = (M + c.bm - 1) / c.bm, nt = (N + c.bn - 1) / c.bn;
    if (mt > 65535) continue;  // (the grid's second dimension)
    for (const int S : {1, 2, 3, 4, 6, 8}) {
      if (S > 1 && (c.wide || S > lines)) break;
      const int per = (lines + S - 1) / S, used = (lines + per - 1) / per;
      const double rounds = static_cast<double>((mt * nt * used + 255) / 256);
      const double t = c.start + rounds * (c.round + c.line * per) + mb_w * c.w + (used == 1 ? 2 * mn * c.out : used * 4 * mn * c.sums + c.add);
      if (t < best_t) {
        best_t = t;
        best = {c.wide, c.bm, c.bn, used, per};
      }
    }
  }
  return best;
}

}  // namespace

Mx4Plan plan_mx4(int M, int N, int Kp) {
  return last_plan<Mx4Plan>({M, N, Kp}, [&] { return choose_mx4(M, N, Kp); });
}

size_t linear_mx4_scratch_bytes(const Mx4Plan& p, int M, int N) {
  return p.S == 1 ? 0 : static_cast<size_t>(p.S) * M * N * sizeof(float);
}

void launch_linear_mx4(const Mx4Plan& p, int dtype, Mx4Tensor a, Mx4Tensor w, void* out, void* scratch, hipStream_t st) {
  if (dtype == 1) launch_product(p, a, w, static_cast<bf16_t*>(out), static_cast<float*>(scratch), st);
  else launch_product(p, a, w, static_cast<float*>(out), static_cast<float*>(scratch), st);
}

}  // namespace dllmc
