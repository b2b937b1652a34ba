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
// are four consecutive channels of one token and are staged as one LDS write.
// Few tokens have kernels of their own (gemm_i8_row, gemm_i8_few).
#include <type_traits>

#include "common.h"
#include "gemm_rows.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

typedef int i32x4 __attribute__((ext_vector_type(4)));

// Four outputs of one token by themselves, vec or not (n < N).
template <int EPI, bool CBF>
__device__ __forceinline__ void i8_put4(const GemmI8Args& p, int m, int n, const i32x4& acc) {
  const float sa = p.sa[m];
  f32x4 za;
#pragma unroll
  for (int r = 0; r < 4; ++r) za[r] = static_cast<float>(acc[r]) * sa;
  out_put4<EPI, CBF>(p, m, n, za);
}

// RBF: the residual is bf16
template <int BM, int BN, int EPI, bool CBF, bool RBF>
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

  // Workgroups [0, npieces) are k-ranges of the tiles from tile_base on (a
  // tile's ranges are neighbours); the rest take the tiles before it whole.
  // Workgroup g runs on XCD g % 8.  Whole tiles go out so that the tiles which
  // run together, 256 of them (or 512, two to a CU), form one block of 8
  // tile-rows of the grouped order and the eight L2s work on the same rows of
  // A at the same time; a last partial wave of them keeps the plain order.
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const bool split = static_cast<int>(blockIdx.x) < p.npieces;
  int pid, ks = 0;
  if (split) {
    pid = p.tile_base + blockIdx.x / p.nsplit;
    ks = blockIdx.x % p.nsplit;
  } else {
    constexpr int XW = BM + BN > 256 ? 32 : 64;  // tiles of an XCD that run together
    const int g = blockIdx.x - p.npieces, xcd = g % 8, loc = g / 8;
    const int full_waves = (static_cast<int>(gridDim.x) - p.npieces) / (8 * XW);
    pid = loc < XW * full_waves ? (loc / XW) * 8 * XW + xcd * XW + loc % XW : g;
  }
  int tile_m, tile_n;
  gemm_tile_of(pid, tm, tn, tile_m, tile_n);
  const int m0 = tile_m * BM, n0 = tile_n * BN;
  const int nk_all = p.K / 128, kt0 = ks * p.kps;
  const int nk = split && nk_all - kt0 >= p.kps ? p.kps : nk_all - kt0;  // >= 1

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
    static_for<decltype(t0_c)::value, decltype(t1_c)::value>([&](auto t_c) __attribute__((always_inline)) {
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
    static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
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
  static_for<0, NCP>(copy);
  set_fill(1);
  static_for<0, NCP>(copy);
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(NCP));
  __syncthreads();
  static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) { read(S0{}, q_c, smem); });
  phase0(smem);
  for (int kt = 0; kt + 1 < nk; ++kt) {
    const char* nxt = smem + ((kt & 1) ^ 1) * kStage;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // this wave's copies of k-step kt + 1
    __syncthreads();
    set_fill(kt + 2);
    static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      constexpr int Q = decltype(q_c)::value, M1 = NM - Mid::value;
      __builtin_amdgcn_sched_barrier(0);
      read(S0{}, q_c, nxt);
      static_for<Q * NCP / NR, (Q + 1) * NCP / NR>(copy);
      mma(S1{}, std::integral_constant<int, Mid::value + Q * M1 / NR>{},
          std::integral_constant<int, Mid::value + (Q + 1) * M1 / NR>{});
    });
    __builtin_amdgcn_sched_barrier(0);
    phase0(nxt);
  }
  mma(S1{}, Mid{}, std::integral_constant<int, NM>{});
  __builtin_amdgcn_s_waitcnt(0);  // re-fetched k-steps still landing in LDS

  // lane: channels n0 + wn WN + 16 j + 4 lq .. + 3 of token m0 + wm WM + 16 i + l16
  if (split) {
    int32_t* out = p.part + static_cast<int64_t>(blockIdx.x) * BM * BN;
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
        *reinterpret_cast<i32x4*>(out + (wm * WM + i * 16 + l16) * BN + wn * WN + j * 16 + 4 * lq) = acc[i][j];
    return;
  }
  // Sixteen tokens of the wave's part at a time, scaled by their factor, are
  // staged in the wave's own piece of LDS and read back as four consecutive
  // channels a lane, whole rows a store (the accumulators go to LDS from where
  // they are; kept for direct stores they spilled, and an epilogue of 16 rows
  // by 32 bytes a store took 32 us of a 92 us round).  Residuals are fetched
  // before the staging they wait for.
  constexpr int LD = WN + 4, CPL = WN / 4, RPP = kWave / CPL, NQ = 16 / RPP;
  static_assert(4 * 16 * LD * 4 <= 2 * kStage, "staging fits the ring");
  __syncthreads();  // every wave's copies have landed and its last reads are done
  float* ep = reinterpret_cast<float*>(smem) + wave * 16 * LD;
  const bool vec = out_vec(p);
  const int cl = lane % CPL * 4, rl = lane / CPL;
  const int n = n0 + wn * WN + cl;
  OutCols cols;
  if (vec) out_cols4<EPI>(p, n < p.N ? n : p.N - 4, cols);
  float sa[TI];
#pragma unroll
  for (int i = 0; i < TI; ++i) {
    const int m = m0 + wm * WM + i * 16 + l16;
    sa[i] = p.sa[m < p.M ? m : p.M - 1];
  }
  // residuals of group g, raw, two groups ahead of their use
  constexpr bool RES = EPI == EPI_GATE_RES;
  constexpr int NPF = 2, NS = NPF + 1;
  ResRaw<RBF> raw[RES ? NS : 1][RES ? NQ : 1];
  bool miss[RES ? NS : 1][RES ? NQ : 1];
  auto fetch = [&](auto g_c) __attribute__((always_inline)) {
    constexpr int g = decltype(g_c)::value;
    if constexpr (RES && g < TI) {
      if (vec) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          const int m = m0 + wm * WM + g * 16 + rl + q * RPP;
          const int rr = out_res_row(p, m < p.M ? m : p.M - 1);
          miss[g % NS][q] = rr < 0;
          raw[g % NS][q].load(p.res, static_cast<int64_t>(rr < 0 ? 0 : rr) * p.ldr + (n < p.N ? n : p.N - 4));
        }
      }
    }
  };
  static_for<0, NPF>(fetch);
  static_for<0, TI>([&](auto i_c) __attribute__((always_inline)) {
    constexpr int i = decltype(i_c)::value;
    const int mi = m0 + wm * WM + i * 16 + rl;
    fetch(std::integral_constant<int, i + NPF>{});
    static_for<0, TJ>([&](auto j_c) __attribute__((always_inline)) {
      constexpr int j = decltype(j_c)::value;
      // (the empty asm keeps the compiler from moving all accumulators into
      // vector registers at once ahead of the epilogue: 29 to 77 spilled)
      if constexpr (BM * BN == 256 * 256) asm volatile("" : "+a"(acc[i][j]));
      f32x4 z;
#pragma unroll
      for (int r = 0; r < 4; ++r) z[r] = static_cast<float>(acc[i][j][r]) * sa[i];
      *reinterpret_cast<f32x4*>(ep + l16 * LD + j * 16 + 4 * lq) = z;
    });
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));  // this wave's staged rows are in LDS
    if (vec) {
#pragma unroll
      for (int q = 0; q < NQ; ++q) {
        const f32x4 z = *reinterpret_cast<const f32x4*>(ep + (rl + q * RPP) * LD + cl);
        float res[4];
        if constexpr (RES) raw[i % NS][q].unpack(miss[i % NS][q], res);
        if (mi + q * RPP < p.M && n < p.N) out_store4<EPI, CBF>(p, mi + q * RPP, n, z, cols, res);
      }
    } else {
      for (int e = lane; e < 16 * WN; e += kWave) {
        const int m = m0 + wm * WM + i * 16 + e / WN, nn = n0 + wn * WN + e % WN;
        if (m < p.M && nn < p.N) out_store1<EPI, CBF>(p, m, nn, ep[e / WN * LD + e % WN]);
      }
    }
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(63));  // and read, before the next rows replace them
    __builtin_amdgcn_sched_barrier(0);
  });
}

// The k-ranges of every split tile added (exact) and the epilogue; a thread takes
// four channels of a token.
template <int BM, int BN, int EPI, bool CBF>
__global__ void __launch_bounds__(256) gemm_i8_reduce(GemmI8Args p) {
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int c4 = static_cast<int>(e % (BN / 4)), r = static_cast<int>((e / (BN / 4)) % BM);
  const int t = static_cast<int>(e / (static_cast<int64_t>(BM) * (BN / 4)));
  if (p.tile_base + t >= tm * tn) return;
  int tile_m, tile_n;
  gemm_tile_of(p.tile_base + t, tm, tn, tile_m, tile_n);
  const int m = tile_m * BM + r, n = tile_n * BN + 4 * c4;
  if (m >= p.M || n >= p.N) return;
  i32x4 acc = {0, 0, 0, 0};
  for (int s = 0; s < p.nsplit; ++s)
    acc += *reinterpret_cast<const i32x4*>(p.part + (static_cast<int64_t>(t) * p.nsplit + s) * BM * BN + r * BN +
                                           4 * c4);
  i8_put4<EPI, CBF>(p, m, n, acc);
}

// ---- nine to sixteen tokens: as few tokens as one matrix instruction takes.
// The weights go from memory straight to its first operand: a workgroup takes
// 16 NT channels, its four waves take turns of 128 bytes along the depth with
// U turns in flight, and their sums meet in LDS.
template <int NT, int EPI, bool CBF>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 4))) gemm_i8_few(GemmI8Args p) {
  constexpr int WAVES = 4, U = NT == 1 ? 5 : NT == 2 ? 4 : 2;
  __shared__ __attribute__((aligned(16))) int part[WAVES][NT][256];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  const int l16 = lane & 15, lq = lane >> 4;
  const int n0 = blockIdx.x * 16 * NT;
  const int8_t* w[NT];
#pragma unroll
  for (int c = 0; c < NT; ++c) {
    const int n = n0 + 16 * c + l16 < p.N ? n0 + 16 * c + l16 : p.N - 1;
    w[c] = p.B + static_cast<int64_t>(n) * p.ldb + 16 * lq;
  }
  const int8_t* a = p.A + static_cast<int64_t>(l16 < p.M ? l16 : p.M - 1) * p.lda + 16 * lq;
  i32x4 acc[NT];
#pragma unroll
  for (int c = 0; c < NT; ++c) acc[c] = i32x4{0, 0, 0, 0};
  const int nk = p.K / 128;
  for (int k0 = wave; k0 < nk; k0 += WAVES * U) {
    i32x4 wf[U][2][NT], af[U][2];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * WAVES < nk ? k0 + u * WAVES : nk - 1;  // past the depth: read, multiplied by zeros
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int c = 0; c < NT; ++c)
          wf[u][h][c] = __builtin_bit_cast(
              i32x4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(w[c] + k * 128 + h * 64)));
        af[u][h] = *reinterpret_cast<const i32x4*>(a + k * 128 + h * 64);
      }
    }
    __builtin_amdgcn_sched_barrier(0);  // all loads of the turns are out before the first is used
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool in = k0 + u * WAVES < nk;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const i32x4 f = in ? af[u][h] : i32x4{0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < NT; ++c)
          acc[c] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wf[u][h][c], f, acc[c], 0, 0, 0);
      }
    }
  }
#pragma unroll
  for (int c = 0; c < NT; ++c) *reinterpret_cast<i32x4*>(&part[wave][c][lane * 4]) = acc[c];
  __syncthreads();
  // thread: channels n0 + 16 c + 4 (l / 16) .. + 3 of token l % 16
  for (int e = tid; e < NT * 64; e += WAVES * 64) {
    const int c = e / 64, l = e % 64;
    const int m = l & 15, n = n0 + 16 * c + 4 * (l >> 4);
    if (m >= p.M || n >= p.N) continue;
    i32x4 sum = {0, 0, 0, 0};
#pragma unroll
    for (int v = 0; v < WAVES; ++v) sum += *reinterpret_cast<const i32x4*>(&part[v][c][l * 4]);
    i8_put4<EPI, CBF>(p, m, n, sum);
  }
}

// ---- one to eight tokens: every weight meets as many products as there are
// tokens, so the read of the weights is all there is.  A wave takes R channels
// and reads each in pieces of 1 KB, 16 contiguous bytes a lane, U pieces of
// every channel in flight; v_dot4 adds four products of a lane at a time, and
// the lanes' sums (exact) meet in registers.  One token of depth 5120 to 30720
// channels: 25.3 us, 6.2 TB/s of weights (with 16 rows of 64 bytes to a load, as
// the matrix instruction takes them, 37.4 us).
template <int MT, int R, int U, int EPI, bool CBF>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 4))) gemm_i8_row(GemmI8Args p) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int n0 = (blockIdx.x * 4 + wave) * R;
  if (n0 >= p.N) return;
  const int8_t* w[R];
#pragma unroll
  for (int r = 0; r < R; ++r) w[r] = p.B + static_cast<int64_t>(n0 + r < p.N ? n0 + r : p.N - 1) * p.ldb;
  int acc[R][MT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[r][t] = 0;
  for (int k0 = 0; k0 < p.K; k0 += 1024 * U) {
    u32x4_t wf[U][R], af[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * 1024 + lane * 16, kc = k < p.K ? k : 0;  // past the depth: zeros of the token
#pragma unroll
      for (int r = 0; r < R; ++r) wf[u][r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(w[r] + kc));
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        af[u][t] = *reinterpret_cast<const u32x4_t*>(p.A + static_cast<int64_t>(t < p.M ? t : p.M - 1) * p.lda + kc);
        if (k >= p.K) af[u][t] = u32x4_t{0, 0, 0, 0};
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[r][t] = __builtin_amdgcn_sdot4(static_cast<int>(wf[u][r][j]), static_cast<int>(af[u][t][j]), acc[r][t],
                                               false);
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const float sum = wave_reduce(__uint_as_float(static_cast<uint32_t>(acc[r][t])), [](float x, float y) {
        return __uint_as_float(__float_as_uint(x) + __float_as_uint(y));  // integers in the lanes' registers
      });
      acc[r][t] = static_cast<int>(__float_as_uint(sum));
    }
  // lane l of pass s stores output 64 s + l = r MT + t: channel n0 + r of token t
#pragma unroll
  for (int s = 0; s < (R * MT + 63) / 64; ++s) {
    int mine = 0;
#pragma unroll
    for (int i = 64 * s; i < R * MT && i < 64 * s + 64; ++i) mine = lane == i - 64 * s ? acc[i / MT][i % MT] : mine;
    const int i = 64 * s + lane, n = n0 + i / MT, m = i % MT;
    if (i < R * MT && n < p.N && m < p.M) out_store1<EPI, CBF>(p, m, n, static_cast<float>(mine) * p.sa[m]);
  }
}

namespace {

constexpr int kRowMax = 8, kFewMax = 16;  // most tokens of gemm_i8_row and gemm_i8_few

enum I8Tile { I8_256, I8_128, I8_64 };
constexpr int kTileEdge[] = {256, 128, 64};

// Estimated time of a plan, us, fitted to 172 products of 17 .. 32760 tokens, 64
// .. 30720 channels and depths 128 .. 13824 in every tile and split (1531 times;
// 11 to 13% off on average; the choice by them is 3% slower than the fastest plan on
// average).  A CU holds `resident` workgroups of a tile; a k-step takes it `lat`
// at least and `thr` for each of them.
struct I8Cost {
  int resident;
  float start, lat, thr;  // launch and first loads; a k-step
  float store;            // epilogue, for a workgroup on every CU
  float join, piece;      // the second launch of a split product; 1 MB of partial sums
  float cold;             // a k-step's loads with the weights beyond the L2s (32 MB)
};
constexpr I8Cost kI8Cost[] = {{1, 7.28f, 1.431f, 1.431f, 7.86f, 3.42f, 0.146f, 0.0f},
                              {2, 4.52f, 0.288f, 0.432f, 2.01f, 2.40f, 0.215f, 0.043f},
                              {4, 3.26f, 0.225f, 0.175f, 0.57f, 2.73f, 0.228f, 0.076f}};

struct I8Plan {
  int tile;
  int base, nsplit, kps;  // tiles from `base` on are split in nsplit ranges of kps k-steps
  float us;
};

int64_t i8_tiles(int tile, int M, int N) {
  const int64_t e = kTileEdge[tile];
  return ((M + e - 1) / e) * ((N + e - 1) / e);
}
size_t i8_part_bytes(const I8Plan& p, int M, int N) {
  const size_t e = kTileEdge[p.tile];
  return p.nsplit < 2 ? 0 : sizeof(int32_t) * e * e * (i8_tiles(p.tile, M, N) - p.base) * p.nsplit;
}

float i8_us(const I8Plan& p, int M, int N, int K, int ncu) {
  const I8Cost& c = kI8Cost[p.tile];
  const int nk = K / 128;
  auto run = [&](int64_t pieces, int steps) {
    const int64_t n = (pieces + ncu - 1) / ncu;  // workgroups on the busiest CU
    const float full = c.resident * c.thr > c.lat ? c.resident * c.thr : c.lat;
    const int rest = static_cast<int>(n % c.resident);
    const float last = rest == 0 ? 0.0f : rest * c.thr > c.lat ? rest * c.thr : c.lat;
    return (n / c.resident * full + last) * steps + c.store * static_cast<float>(pieces) / ncu;
  };
  const float beyond = static_cast<float>(N) * K / 32e6f;
  float us = c.start + c.cold * (beyond < 1.0f ? beyond : 1.0f) * nk;
  if (p.base > 0) us += run(p.base, nk);
  const int64_t tail = i8_tiles(p.tile, M, N) - p.base;
  if (tail > 0) us += run(tail * p.nsplit, p.kps) + c.join + c.piece * 1e-6f * i8_part_bytes(p, M, N);
  return us;
}

// Every tile whole; or the tiles beyond the last whole round of the device, or
// all of them where they are less than a round, split along the depth.  The
// fastest by the estimate: 13104 x 5120 x 5120 (16 tiles beyond the fourth round)
// 322 us whole, 297 split; 100 x 5120 x 5120 21 and 16; 1950 x 1536 x 8960 46 and 41.
// (Sums are exact: the choice does not show in the results.)
I8Plan i8_plan(int M, int N, int K) {
  const int ncu = device_cu_count(), nk = K / 128;
  constexpr size_t kMostPartial = size_t(64) << 20;
  I8Plan best{-1, 0, 1, nk, 0.0f};
  auto consider = [&](int tile, int64_t base, int ns) {
    const int kps = (nk + ns - 1) / ns;
    I8Plan p{tile, static_cast<int>(base), (nk + kps - 1) / kps, kps, 0.0f};  // every range non-empty
    if (i8_part_bytes(p, M, N) > kMostPartial) return;
    p.us = i8_us(p, M, N, K, ncu);
    if (best.tile < 0 || p.us < best.us) best = p;
  };
  for (int tile = I8_256; tile <= I8_64; ++tile) {
    const int64_t tiles = i8_tiles(tile, M, N), round = static_cast<int64_t>(ncu) * kI8Cost[tile].resident;
    consider(tile, tiles, 1);
    for (const int ns : {2, 3, 4, 6, 8, 12, 16})
      if (nk / ns >= 2 && tiles % round != 0 && tiles < round * 64) consider(tile, tiles / round * round, ns);
  }
  return best;
}

template <int E>
hipError_t launch_tile(int epi, GemmI8Args a, const I8Plan& plan, hipStream_t stream) {
  const int tiles = static_cast<int>(i8_tiles(plan.tile, a.M, a.N)), tail = plan.nsplit > 1 ? tiles - plan.base : 0;
  a.tile_base = tiles - tail;
  a.nsplit = plan.nsplit;
  a.kps = plan.kps;
  a.npieces = tail * plan.nsplit;
  return with_epilogue(epi, a.c_bf16, a.res_bf16, [&](auto epi_c, auto bf_c, auto res_c) -> hipError_t {
    constexpr int EPI = decltype(epi_c)::value;
    constexpr bool CBF = decltype(bf_c)::value, RBF = decltype(res_c)::value;
    hipError_t e = ECHO_LAUNCH("gemm_int8", (gemm_i8_tile<E, E, EPI, CBF, RBF>),
                               dim3(static_cast<unsigned>(a.npieces + a.tile_base)), dim3(256), 0, stream, a);
    if (e != hipSuccess || tail == 0) return e;
    const int64_t n = static_cast<int64_t>(tail) * E * (E / 4);
    return ECHO_LAUNCH("gemm_int8_reduce", (gemm_i8_reduce<E, E, EPI, CBF>),
                       dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, a);
  });
}

template <int NT>
hipError_t launch_few(int epi, const GemmI8Args& a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.N + 16 * NT - 1) / (16 * NT)));
  return with_epilogue(epi, a.c_bf16, 1, [&](auto epi_c, auto bf_c, auto) -> hipError_t {
    return ECHO_LAUNCH("gemm_int8_few", (gemm_i8_few<NT, decltype(epi_c)::value, decltype(bf_c)::value>), grid,
                       dim3(256), 0, stream, a);
  });
}
template <int MT, int R, int U>
hipError_t launch_row(int epi, const GemmI8Args& a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.N + 4 * R - 1) / (4 * R)));
  return with_epilogue(epi, a.c_bf16, 1, [&](auto epi_c, auto bf_c, auto) -> hipError_t {
    return ECHO_LAUNCH("gemm_int8_row", (gemm_i8_row<MT, R, U, decltype(epi_c)::value, decltype(bf_c)::value>), grid,
                       dim3(256), 0, stream, a);
  });
}

}  // namespace

size_t gemm_i8_partial_bytes(int M, int N, int K) {
  return M <= kFewMax ? 0 : i8_part_bytes(i8_plan(M, N, K), M, N);
}

hipError_t launch_gemm_i8(int epi, const GemmI8Args& a, hipStream_t stream) {
  // two channels a wave and 5 KB of each in flight; with 5 to 8 tokens, whose
  // codes take the registers, four channels and 1 KB (one token, 5120 x 5120 and
  // 30720 x 5120 x 5: 6.2 and 25.3 us; two channels and 2 KB 6.7 and 28.5, eight and 1 KB
  // 7.5 and 25.7; eight tokens: 11.5 and 38.0; 16 channels a workgroup as below 12.3
  // and 45.9)
  if (a.M == 1) return launch_row<1, 2, 5>(epi, a, stream);
  if (a.M == 2) return launch_row<2, 2, 5>(epi, a, stream);
  if (a.M <= 4) return launch_row<4, 2, 5>(epi, a, stream);
  if (a.M <= kRowMax) return launch_row<8, 4, 1>(epi, a, stream);
  if (a.M <= kFewMax) {
    // more channels to a workgroup read the tokens less often and leave CUs idle
    // (16 tokens, 16 / 32 / 64 channels: 30720 x 5120 53 / 54 / 44 us, 5120 x 13824
    // 34 / 27 / 45, 5120 x 5120 14.2 / 14.6 / 21)
    if (a.N >= 64 * device_cu_count()) return launch_few<4>(epi, a, stream);
    return a.K >= 8192 ? launch_few<2>(epi, a, stream) : launch_few<1>(epi, a, stream);
  }
  const I8Plan plan = i8_plan(a.M, a.N, a.K);
  if (i8_part_bytes(plan, a.M, a.N) > a.part_bytes) return hipErrorInvalidValue;
  switch (plan.tile) {
    case I8_256: return launch_tile<256>(epi, a, plan, stream);
    case I8_128: return launch_tile<128>(epi, a, plan, stream);
    default: return launch_tile<64>(epi, a, plan, stream);
  }
}

}  // namespace echo
