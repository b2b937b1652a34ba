// Matrix products of 8-bit codes with a scale for each token (row of A) and
// each channel (row of B):
//
//   C[m, n] = f( sa[m] sb[n] sum_k A[m, k] B[n, k] + bias[n] )
//   f: none, GELU (tanh form), or res[row(m), n] + gate[n] * (.) in fp32
//
// The sums are exact in int32 (127^2 * 65536 < 2^31), so neither the tile nor
// the order of a split changes a result; the sum, rounded to fp32 once, is
// scaled by the token's and then the channel's factor.  Both operands are
// rows of codes whose pitch is a multiple of 128 bytes with zeros behind the
// last column (quantize_rows), so the depth has no tail.  M and N are
// arbitrary: rows past the end re-read the last one and are not stored.
//
// Tiles.  v_mfma_i32_16x16x64_i8 takes 16 codes of one row per lane, the
// bytes of v_mfma_f32_16x16x32_bf16 at twice its depth.  A workgroup of four
// waves (2 x 2) owns BM x BN outputs; k-steps of 128 bytes go through a
// two-stage LDS ring of direct copies, 16-byte chunks XOR-swizzled by
// (row >> 1) & 7 so that the 16 rows of one LDS cycle hit distinct banks.
// The channels are the instruction's first operand, so a lane's accumulators
// are four consecutive channels of one token and leave as one store.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int B, int E, typename F>
__device__ __forceinline__ void i8_for(F&& f) {
  if constexpr (B < E) {
    f(std::integral_constant<int, B>{});
    i8_for<B + 1, E>(f);
  }
}

// 0.5 z (1 + tanh u) = z / (1 + 2^(z (k1 + k2 z^2))), as in the bf16 products
__device__ __forceinline__ float i8_gelu(float z) {
  constexpr double kU = 0.7978845608028654 * 1.4426950408889634;
  constexpr float k1 = static_cast<float>(-2.0 * kU), k2 = static_cast<float>(-2.0 * kU * 0.044715);
  const float e = __builtin_amdgcn_exp2f(z * fmaf(k2, z * z, k1));
  return z * __builtin_amdgcn_rcpf(1.0f + e);
}

__device__ __forceinline__ float i8_load(const void* p, int bf, int64_t i) {
  return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// Scale and bias (and gate) of the four channels n .. n + 3 (past N: channel N - 1).
struct I8Cols {
  float sb[4], bias[4], gate[4];
};
template <int EPI>
__device__ __forceinline__ void i8_cols(const GemmI8Args& p, int n, I8Cols& c) {
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    const int i = n + r < p.N ? n + r : p.N - 1;
    c.sb[r] = p.sb[i];
    c.bias[r] = p.bias != nullptr ? i8_load(p.bias, p.bias_bf16, i) : 0.0f;
    c.gate[r] = EPI == EPI_GATE_RES ? p.gate[i] : 0.0f;
  }
}

// The outputs of four consecutive channels n .. n + 3 of row m.  vec: rows of
// C and of the residual are aligned for four values and N % 4 == 0.
template <int EPI>
__device__ __forceinline__ void i8_store4(const GemmI8Args& p, int m, int n, const int* acc, float sa,
                                          const I8Cols& c, bool vec) {
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) v[r] = fmaf(static_cast<float>(acc[r]) * sa, c.sb[r], c.bias[r]);
  if constexpr (EPI == EPI_GELU) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = i8_gelu(v[r]);
  }
  if constexpr (EPI == EPI_GATE_RES) {
    int64_t rr = m;
    float res[4];
    bool ok = true;
    if (p.res_rows != nullptr) {
      rr = p.res_rows[m];
      ok = rr >= 0 && rr < p.res_nrows;  // no such row: NaN
      rr = ok ? rr : 0;
    }
    if (vec && p.res_bf16) {
      const uint2 raw = ldg8_nt(static_cast<const bf16_t*>(p.res) + rr * p.ldr + n);
      res[0] = __uint_as_float(raw.x << 16);
      res[1] = __uint_as_float(raw.x & 0xffff0000u);
      res[2] = __uint_as_float(raw.y << 16);
      res[3] = __uint_as_float(raw.y & 0xffff0000u);
    } else if (vec) {
      unpack16(ldg16_nt(static_cast<const float*>(p.res) + rr * p.ldr + n), res, static_cast<const float*>(nullptr));
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) res[r] = n + r < p.N ? i8_load(p.res, p.res_bf16, rr * p.ldr + n + r) : 0.0f;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] = ok ? fmaf(c.gate[r], v[r], res[r]) : __uint_as_float(0x7fc00000u);
  }
  const int64_t at = static_cast<int64_t>(m) * p.ldc + n;
  if (vec) {
    if (p.c_bf16)
      *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.C) + at) =
          make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    else
      stg16(static_cast<float*>(p.C) + at, pack16(v, static_cast<const float*>(nullptr)));
  } else {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if (n + r >= p.N) break;
      if (p.c_bf16)
        Elem<bf16_t>::store(static_cast<bf16_t*>(p.C), at + r, v[r]);
      else
        static_cast<float*>(p.C)[at + r] = v[r];
    }
  }
}

__device__ __forceinline__ bool i8_vec(const GemmI8Args& p) {
  const uintptr_t ca = reinterpret_cast<uintptr_t>(p.C), ra = reinterpret_cast<uintptr_t>(p.res);
  const int ce = p.c_bf16 ? 2 : 4, re = p.res_bf16 ? 2 : 4;
  return (p.N & 3) == 0 && (p.ldc & 3) == 0 && (ca & (4 * ce - 1)) == 0 &&
         (p.res == nullptr || ((p.ldr & 3) == 0 && (ra & (4 * re - 1)) == 0));
}

// Grouped order: 8 tile-rows at a time, down the rows first.
__device__ __forceinline__ void i8_tile_of(int pid, int tm, int tn, int& tile_m, int& tile_n) {
  constexpr int GROUP = 8;
  const int group_size = GROUP * tn;
  const int first_m = (pid / group_size) * GROUP;
  const int gm = (tm - first_m) < GROUP ? (tm - first_m) : GROUP;
  tile_m = first_m + (pid % group_size) % gm;
  tile_n = (pid % group_size) / gm;
}

template <int BM, int BN, int EPI>
__global__ void __launch_bounds__(256, (BM + BN <= 256 ? 2 : 1)) gemm_i8_tile(GemmI8Args p) {
  constexpr int kStage = (BM + BN) * 128;
  constexpr int WM = BM / 2, WN = BN / 2, TI = WM / 16, TJ = WN / 16;
  constexpr int NM = TI * TJ, NR = TI + TJ;
  constexpr int CA = BM / 32, CB = BN / 32, NCP = CA + CB;
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
  const int wm = wave >> 1, wn = wave & 1;
  const int l16 = lane & 15, lq = lane >> 4;

  // XCD x takes a contiguous range of the grouped order (of the pieces, where
  // tiles are split along k: the ranges of a tile are neighbours)
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const int nb = gridDim.x, per = nb / 8, rem = nb % 8, xcd = blockIdx.x % 8;
  const int piece = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
  const int pid = piece / p.nsplit, ks = piece % p.nsplit;
  int tile_m, tile_n;
  i8_tile_of(pid, tm, tn, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int nk_all = p.K / 128, kt0 = ks * p.kps;
  const int nk = nk_all - kt0 < p.kps ? nk_all - kt0 : p.kps;  // >= 1

  // copy c of a wave fills the 8 rows 8 (wave + 4 c) .. of the (A ++ B) stage;
  // lane i takes row i / 8, slot i % 8, which holds chunk (i % 8) ^ ((row >> 1) & 7)
  const int chunk = ((lane % 8) ^ (((8 * wave + lane / 8) >> 1) & 7)) * 16;
  uint32_t voff[NCP];
#pragma unroll
  for (int c = 0; c < NCP; ++c) {
    const int r = 8 * (wave + 4 * (c < CA ? c : c - CA)) + lane / 8;
    const int last = (c < CA ? p.M - m0 : p.N - n0) - 1;
    voff[c] = static_cast<uint32_t>(r < last ? r : last) * static_cast<uint32_t>(c < CA ? p.lda : p.ldb) + chunk;
  }
  const int8_t* a0 = p.A + static_cast<int64_t>(m0) * p.lda + static_cast<int64_t>(kt0) * 128;
  const int8_t* b0 = p.B + static_cast<int64_t>(n0) * p.ldb + static_cast<int64_t>(kt0) * 128;
  const uint32_t dst0 = lds_offset(smem) + wave * 1024;
  const int8_t* src_a = a0;
  const int8_t* src_b = b0;
  uint32_t dst_stage = 0;
  auto set_fill = [&](int kt) __attribute__((always_inline)) {
    const int kf = kt < nk ? kt : nk - 1;  // past the last k-step: re-fetched, never used
    src_a = a0 + static_cast<int64_t>(kf) * 128;
    src_b = b0 + static_cast<int64_t>(kf) * 128;
    dst_stage = dst0 + (kt & 1) * kStage;
  };
  auto copy = [&](auto c_c) __attribute__((always_inline)) {
    constexpr int c = decltype(c_c)::value;
    lds_copy16_s(c < CA ? src_a : src_b, voff[c], dst_stage + c * 4096);
  };

  const int rd_a = (wm * WM + l16) * 128, rd_b = (BM + wn * WN + l16) * 128;
  const int ch0 = (lq ^ (l16 >> 1)) * 16, ch1 = ((4 + lq) ^ (l16 >> 1)) * 16;
  i32x4 fa[2][TI], fb[2][TJ], acc[TI][TJ];
  auto read = [&](auto set_c, auto q_c, const char* st) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value, Q = decltype(q_c)::value;
    const int ch = SET ? ch1 : ch0;
    if constexpr (Q == 0)
      fa[SET][0] = *reinterpret_cast<const i32x4*>(st + rd_a + ch);
    else if constexpr (Q <= TJ)
      fb[SET][Q - 1] = *reinterpret_cast<const i32x4*>(st + rd_b + (Q - 1) * 2048 + ch);
    else
      fa[SET][Q - TJ] = *reinterpret_cast<const i32x4*>(st + rd_a + (Q - TJ) * 2048 + ch);
  };
#pragma unroll
  for (int i = 0; i < TI; ++i)
#pragma unroll
    for (int j = 0; j < TJ; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto mma = [&](auto set_c, auto t0_c, auto t1_c) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value;
    i8_for<decltype(t0_c)::value, decltype(t1_c)::value>([&](auto t_c) __attribute__((always_inline)) {
      constexpr int T = decltype(t_c)::value;
      acc[T / TJ][T % TJ] =
          __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[SET][T % TJ], fa[SET][T / TJ], acc[T / TJ][T % TJ], 0, 0, 0);
    });
  };
  typedef std::integral_constant<int, 0> S0;
  typedef std::integral_constant<int, 1> S1;
  typedef std::integral_constant<int, NM / 2> Mid;
  // A k-step: the first half's MFMAs with the second half's reads between
  // them; half of the second half's; the wait for this wave's copies of the
  // next k-step and the barrier; the rest, with the next k-step's first reads
  // and the copies of the k-step after next into the stage just released.
  auto phase0 = [&](const char* st) __attribute__((always_inline)) {
    i8_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      constexpr int Q = decltype(q_c)::value;
      __builtin_amdgcn_sched_barrier(0);
      read(S1{}, q_c, st);
      mma(S0{}, std::integral_constant<int, Q * NM / NR>{}, std::integral_constant<int, (Q + 1) * NM / NR>{});
    });
    __builtin_amdgcn_sched_barrier(0);
    mma(S1{}, S0{}, Mid{});
    __builtin_amdgcn_sched_barrier(0);
  };
  set_fill(0);
  i8_for<0, NCP>(copy);
  set_fill(1);
  i8_for<0, NCP>(copy);
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(NCP));
  __syncthreads();
  i8_for<0, NR>([&](auto q_c) __attribute__((always_inline)) { read(S0{}, q_c, smem); });
  phase0(smem);
  for (int kt = 0; kt + 1 < nk; ++kt) {
    const char* nxt = smem + ((kt & 1) ^ 1) * kStage;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // this wave's copies of k-step kt + 1
    __syncthreads();
    set_fill(kt + 2);
    i8_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      constexpr int Q = decltype(q_c)::value, M1 = NM - Mid::value;
      __builtin_amdgcn_sched_barrier(0);
      read(S0{}, q_c, nxt);
      i8_for<Q * NCP / NR, (Q + 1) * NCP / NR>(copy);
      mma(S1{}, std::integral_constant<int, Mid::value + Q * M1 / NR>{},
          std::integral_constant<int, Mid::value + (Q + 1) * M1 / NR>{});
    });
    __builtin_amdgcn_sched_barrier(0);
    phase0(nxt);
  }
  mma(S1{}, Mid{}, std::integral_constant<int, NM>{});
  __builtin_amdgcn_s_waitcnt(0);  // re-fetched k-steps still landing in LDS

  // lane: channels n0 + wn WN + 16 j + 4 lq .. + 3 of token m0 + wm WM + 16 i + l16
  if (p.nsplit > 1) {
    int32_t* out = p.part + static_cast<int64_t>(piece) * BM * BN;
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        *reinterpret_cast<i32x4*>(out + (wm * WM + i * 16 + l16) * BN + wn * WN + j * 16 + 4 * lq) = acc[i][j];
    return;
  }
  const bool vec = i8_vec(p);
  float sa[TI];
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    const int m = m0 + wm * WM + i * 16 + l16;
    sa[i] = p.sa[m < p.M ? m : p.M - 1];
  }
  // one block of channels at a time (the fences keep the loads of all of them
  // from being gathered in registers in front)
  i8_for<0, TJ>([&](auto j_c) __attribute__((always_inline)) {
    constexpr int j = decltype(j_c)::value;
    const int n = n0 + wn * WN + j * 16 + 4 * lq;
    I8Cols cols;
    i8_cols<EPI>(p, n, cols);
    i8_for<0, TI>([&](auto i_c) __attribute__((always_inline)) {
      constexpr int i = decltype(i_c)::value;
      const int m = m0 + wm * WM + i * 16 + l16;
      if (m < p.M && n < p.N) {
        const int a4[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
        i8_store4<EPI>(p, m, n, a4, sa[i], cols, vec);
      }
    });
    __builtin_amdgcn_sched_barrier(0);
  });
}

// The k-ranges of every tile added (exact) and the epilogue; a thread takes
// four channels of a token.
template <int BM, int BN, int EPI>
__global__ void __launch_bounds__(256) gemm_i8_reduce(GemmI8Args p) {
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int c4 = static_cast<int>(e % (BN / 4)), r = static_cast<int>((e / (BN / 4)) % BM);
  const int pid = static_cast<int>(e / (static_cast<int64_t>(BM) * (BN / 4)));
  if (pid >= tm * tn) return;
  int tile_m, tile_n;
  i8_tile_of(pid, tm, tn, tile_m, tile_n);
  const int m = tile_m * BM + r, n = tile_n * BN + 4 * c4;
  if (m >= p.M || n >= p.N) return;
  int acc[4] = {0, 0, 0, 0};
  for (int s = 0; s < p.nsplit; ++s) {
    const i32x4 v = *reinterpret_cast<const i32x4*>(
        p.part + (static_cast<int64_t>(pid) * p.nsplit + s) * BM * BN + r * BN + 4 * c4);
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[j] += v[j];
  }
  I8Cols cols;
  i8_cols<EPI>(p, n, cols);
  i8_store4<EPI>(p, m, n, acc, p.sa[m], cols, i8_vec(p));
}

// ---- few tokens.  At most 16 MT tokens need every weight once and little
// else, so the weights go from memory straight to the matrix instruction's
// first operand: a workgroup takes 16 channels, its waves take turns of 64
// bytes along the depth, and their sums meet in LDS.
template <int MT, int WAVES, int EPI>
__global__ void __launch_bounds__(WAVES * 64) gemm_i8_few(GemmI8Args p) {
  __shared__ __attribute__((aligned(16))) int part[WAVES][MT][256];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int l16 = lane & 15, lq = lane >> 4;
  const int n0 = blockIdx.x * 16;
  const int nr = n0 + l16 < p.N ? n0 + l16 : p.N - 1;
  const int8_t* w = p.B + static_cast<int64_t>(nr) * p.ldb + 16 * lq;
  const int8_t* a[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = 16 * t + l16 < p.M ? 16 * t + l16 : p.M - 1;
    a[t] = p.A + static_cast<int64_t>(m) * p.lda + 16 * lq;
  }
  i32x4 acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = i32x4{0, 0, 0, 0};
#pragma unroll 4
  for (int k = wave * 64; k < p.K; k += WAVES * 64) {
    const u32x4_t raw = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(w + k));
    const i32x4 wf = __builtin_bit_cast(i32x4, raw);
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const i32x4 af = *reinterpret_cast<const i32x4*>(a[t] + k);
      acc[t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf, af, acc[t], 0, 0, 0);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) *reinterpret_cast<i32x4*>(&part[wave][t][lane * 4]) = acc[t];
  __syncthreads();
  // thread: channels n0 + 4 (lane / 16) .. + 3 of token 16 t + lane % 16
  for (int e = tid; e < MT * 64; e += WAVES * 64) {
    const int t = e / 64, l = e % 64;
    const int m = 16 * t + (l & 15), n = n0 + 4 * (l >> 4);
    if (m >= p.M || n >= p.N) continue;
    int sum[4] = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < WAVES; ++v)
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += part[v][t][l * 4 + j];
    I8Cols cols;
    i8_cols<EPI>(p, n, cols);
    i8_store4<EPI>(p, m, n, sum, p.sa[m], cols, i8_vec(p));
  }
}

namespace {

constexpr int kFewMax = 64;  // tokens that go to gemm_i8_few

struct I8Plan {
  int bm, bn, nsplit, kps;
  size_t bytes;
};

I8Plan i8_plan(int M, int N, int K) {
  const int ncu = device_cu_count();
  auto tiles = [&](int bm, int bn) {
    return static_cast<int64_t>((M + bm - 1) / bm) * ((N + bn - 1) / bn);
  };
  I8Plan p{64, 64, 1, K / 128, 0};
  if (tiles(256, 256) >= ncu)
    p.bm = p.bn = 256;
  else if (tiles(128, 128) >= ncu)
    p.bm = p.bn = 128;
  return p;
}

template <int BM, int BN>
hipError_t launch_tile(int epi, const GemmI8Args& a, hipStream_t stream) {
  const int tm = (a.M + BM - 1) / BM, tn = (a.N + BN - 1) / BN;
  const dim3 grid(static_cast<unsigned>(tm * tn * a.nsplit));
  auto go = [&](auto epi_c) -> hipError_t {
    constexpr int EPI = decltype(epi_c)::value;
    hipError_t e = ECHO_LAUNCH("gemm_int8", (gemm_i8_tile<BM, BN, EPI>), grid, dim3(256), 0, stream, a);
    if (e != hipSuccess || a.nsplit == 1) return e;
    const int64_t n = static_cast<int64_t>(tm) * tn * BM * (BN / 4);
    return ECHO_LAUNCH("gemm_int8_reduce", (gemm_i8_reduce<BM, BN, EPI>), dim3(static_cast<unsigned>((n + 255) / 256)),
                       dim3(256), 0, stream, a);
  };
  if (epi == EPI_GELU) return go(std::integral_constant<int, EPI_GELU>{});
  if (epi == EPI_GATE_RES) return go(std::integral_constant<int, EPI_GATE_RES>{});
  return go(std::integral_constant<int, EPI_BIAS>{});
}

template <int MT>
hipError_t launch_few(int epi, const GemmI8Args& a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.N + 15) / 16));
  auto go = [&](auto epi_c) -> hipError_t {
    constexpr int EPI = decltype(epi_c)::value;
    return ECHO_LAUNCH("gemm_int8_few", (gemm_i8_few<MT, 4, EPI>), grid, dim3(256), 0, stream, a);
  };
  if (epi == EPI_GELU) return go(std::integral_constant<int, EPI_GELU>{});
  if (epi == EPI_GATE_RES) return go(std::integral_constant<int, EPI_GATE_RES>{});
  return go(std::integral_constant<int, EPI_BIAS>{});
}

}  // namespace

size_t gemm_i8_partial_bytes(int M, int N, int K) { return M <= kFewMax ? 0 : i8_plan(M, N, K).bytes; }

hipError_t launch_gemm_i8(int epi, const GemmI8Args& args, hipStream_t stream) {
  GemmI8Args a = args;
  if (a.M <= 16) return launch_few<1>(epi, a, stream);
  if (a.M <= 32) return launch_few<2>(epi, a, stream);
  if (a.M <= kFewMax) return launch_few<4>(epi, a, stream);
  const I8Plan plan = i8_plan(a.M, a.N, a.K);
  a.nsplit = plan.nsplit;
  a.kps = plan.kps;
  if (plan.bm == 256) return launch_tile<256, 256>(epi, a, stream);
  if (plan.bm == 128) return launch_tile<128, 128>(epi, a, stream);
  return launch_tile<64, 64>(epi, a, stream);
}

}  // namespace echo
