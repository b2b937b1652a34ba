// Matrix products of rows in 4 bits (quant_fp4.hip: codes of one sign, two exponent
// and one fraction bit, a power of two for every 32 of them):
//
//   C[m, n] = f( sum_b 2^(ea[m, b] + eb[n, b]) sum_{k in b} A[m, k] B[n, k] + bias[n] )
//   f: none, GELU (tanh form), or res[row(m), n] + gate[n] * (.) in fp32
//
// v_mfma_scale_f32_16x16x128_f8f6f4 takes 32 codes of one row per lane (16 bytes,
// one block) and the block's scale byte from another register, multiplies and
// adds in fp32, and makes a scale of 255 a NaN: nothing is converted on the way.
// In bytes it is the 8-bit instruction (v_mfma_i32_16x16x64_i8: 16 bytes of a row
// a lane, 16 cycles), so the tiles, the LDS ring and the epilogue are those of
// gemm_int8.hip at twice the depth per byte, and the scales are added: a k-step
// of 128 bytes has 8 of them a row.  They go through a ring of their own, 16
// bytes a row for two k-steps (a sixteenth of the codes' bytes).
//
// Rows of codes have a pitch of whole 128 bytes and rows of scales of whole 16,
// with zeros behind the last column in one operand at least, so the depth has no
// tail.  M and N are arbitrary: rows past the end re-read the last one and are
// not stored.
#include <type_traits>

#include "common.h"
#include "gemm_rows.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kFp4 = 4;  // the instruction's name for the type (cbsz, blgp)

// c + a b, with byte SEL of sa and of sb the lanes' scales
template <int SEL>
__device__ __forceinline__ f32x4 mfma_fp4(const i32x4& a, int sa, const i32x4& b, int sb, const f32x4& c) {
  const i32x8 a8 = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, b8 = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a8, b8, c, kFp4, kFp4, SEL, sa, SEL, sb);
}

// An accumulator's value.  Written out so that the accumulators' own registers are all
// that ever holds them: left to the compiler, 240 to 460 registers were spilled.  The
// matrix instructions in front have to be done (acc_settled).
__device__ __forceinline__ float from_acc(float acc) {
  float v;
  asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc));
  return v;
}
__device__ __forceinline__ void acc_settled(f32x4& last) {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_nop 15\n\ts_nop 15" : "+a"(last));
  __builtin_amdgcn_sched_barrier(0);
}

// RBF: the residual is bf16.  STREAM: a workgroup goes from tile to tile without
// draining its copies, and stores from its accumulators (rows aligned to 16 bytes).
template <int BM, int BN, int EPI, bool CBF, bool RBF, bool STREAM>
__global__ void __launch_bounds__(256, (BM + BN <= 256 ? 2 : 1)) gemm_fp4_tile(GemmFp4Args p) {
  constexpr int kStage = (BM + BN) * 128, kScales = (BM + BN) * 16;
  constexpr int WM = BM / 2, WN = BN / 2, TI = WM / 16, TJ = WN / 16;
  constexpr int NM = TI * TJ, NR = TI + TJ;
  constexpr int CA = BM / 32, CB = BN / 32, NCP = CA + CB;
  constexpr int NSC = (BM + BN) / 64;  // copies of 64 rows' scales
  constexpr int kCols = STREAM ? 4 * WN * 8 : 0;  // the waves' bias and gate
  __shared__ __attribute__((aligned(1024))) char smem[2 * kStage + 2 * kScales + kCols];
  const int tid = threadIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave), lane = tid % kWave;
  const int wm = wave >> 1, wn = wave & 1;
  const int l16 = lane & 15, lq = lane >> 4;

  // Work items: [0, npieces) are k-ranges of the tiles from tile_base on, the rest
  // the tiles before it, whole, in the order of gemm_int8.hip; workgroup g takes
  // items g, g + grid, ...
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const int nk_all = p.K / 128, nitems = p.npieces + p.tile_base;
  auto item_at = [&](int item, int& m0, int& n0, int& kt0, int& nk) __attribute__((always_inline)) {
    int pid, ks = 0;
    if (item < p.npieces) {
      pid = p.tile_base + item / p.nsplit;
      ks = item % p.nsplit;
    } else {
      constexpr int XW = BM + BN > 256 ? 32 : 64;  // tiles of an XCD that run together
      const int g = item - p.npieces, xcd = g % 8, loc = g / 8;
      const int full_waves = p.tile_base / (8 * XW);
      pid = loc < XW * full_waves ? (loc / XW) * 8 * XW + xcd * XW + loc % XW : g;
    }
    int tile_m, tile_n;
    gemm_tile_of(pid, tm, tn, tile_m, tile_n);
    m0 = tile_m * BM, n0 = tile_n * BN;
    kt0 = ks * p.kps;  // kps is even: a range starts with a pair's scales
    nk = item < p.npieces && nk_all - kt0 >= p.kps ? p.kps : nk_all - kt0;  // >= 1
  };

  // The copies: two k-steps ahead of the products, over the ends of items.  Copy c of
  // a wave fills the 8 rows 8 (wave + 4 c) .. of the (A ++ B) stage; lane i takes row
  // i / 8, slot i % 8, which holds chunk (i % 8) ^ ((row >> 1) & 7).  Scale copy c of
  // wave w: rows 64 (w + 4 c) .. of A ++ B, a row a lane.
  constexpr int NSW = (NSC + 3) / 4;
  const int chunk = ((lane % 8) ^ (((8 * wave + lane / 8) >> 1) & 7)) * 16;
  const uint32_t dst0 = lds_offset(smem) + wave * 1024, sdst0 = lds_offset(smem) + 2 * kStage + wave * 1024;
  uint32_t voff[NCP], soff[NSW];
  const uint8_t *src_a, *src_b, *src_sa, *src_sb;
  int f_kt = 0, f_nk = 0, f_slot = 0;
  auto fill_item = [&](int item) __attribute__((always_inline)) {
    int m0, n0, kt0;
    item_at(item, m0, n0, kt0, f_nk);
#pragma unroll
    for (int c = 0; c < NCP; ++c) {
      const int r = 8 * (wave + 4 * (c < CA ? c : c - CA)) + lane / 8;
      const int last = (c < CA ? p.M - m0 : p.N - n0) - 1;
      voff[c] = static_cast<uint32_t>(r < last ? r : last) * static_cast<uint32_t>(c < CA ? p.lda : p.ldb) + chunk;
    }
#pragma unroll
    for (int c = 0; c < NSW; ++c) {
      const int s = wave + 4 * c, r = (s * 64 < BM ? s * 64 : s * 64 - BM) + lane;
      const int last = (s * 64 < BM ? p.M - m0 : p.N - n0) - 1;
      soff[c] = static_cast<uint32_t>(r < last ? r : last) * static_cast<uint32_t>(s * 64 < BM ? p.ldsa : p.ldsb);
    }
    src_a = p.A + static_cast<int64_t>(m0) * p.lda + static_cast<int64_t>(kt0) * 128;
    src_b = p.B + static_cast<int64_t>(n0) * p.ldb + static_cast<int64_t>(kt0) * 128;
    src_sa = p.sa + static_cast<int64_t>(m0) * p.ldsa + static_cast<int64_t>(kt0) * 8;
    src_sb = p.sb + static_cast<int64_t>(n0) * p.ldsb + static_cast<int64_t>(kt0) * 8;
    f_kt = 0;
  };
  // the next k-step to copy, of parity PAR: its stage, and with an even one the scales
  // of two; past an item's last k-step the same again, never used
  uint32_t dst_stage = 0;
  auto fill_start = [&](auto par_c) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_c)::value;
    dst_stage = dst0 + PAR * kStage;
    if constexpr (PAR == 0) {
#pragma unroll
      for (int c = 0; c < NSW; ++c) {
        const int s = wave + 4 * c;
        if (NSC % 4 == 0 || s < NSC)
          lds_copy16_s(s * 64 < BM ? src_sa : src_sb, soff[c], sdst0 + f_slot * kScales + c * 4096);
      }
      f_slot ^= 1;
    }
  };
  auto copy = [&](auto c_c) __attribute__((always_inline)) {
    constexpr int c = decltype(c_c)::value;
    lds_copy16_s(c < CA ? src_a : src_b, voff[c], dst_stage + c * 4096);
  };
  auto fill_done = [&](auto par_c) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_c)::value;
    const bool more = ++f_kt < f_nk;
    src_a += more ? 128 : 0;
    src_b += more ? 128 : 0;
    if constexpr (PAR == 1) {
      src_sa += more ? 16 : 0;
      src_sb += more ? 16 : 0;
    }
  };

  const int rd_a = (wm * WM + l16) * 128, rd_b = (BM + wn * WN + l16) * 128;
  // the halves of a k-step are its even and its odd blocks, so that a lane's two
  // scales are neighbours; in this order lanes of lq 0 and 1 (2 and 3) share banks, four
  // cycles more for each read of 16 bytes, which the order of gemm_int8.hip does not have
  const int rd_sa = (wm * WM + l16) * 16 + 2 * lq, rd_sb = (BM + wn * WN + l16) * 16 + 2 * lq;
  const int ch0 = ((2 * lq) ^ (l16 >> 1)) * 16, ch1 = ((2 * lq + 1) ^ (l16 >> 1)) * 16;
  i32x4 fa[2][TI], fb[2][TJ];
  int sa[2][TI], sb[2][TJ];  // of even and odd k-steps; two bytes each: the halves' scales
  f32x4 acc[TI][TJ];
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
  auto read_scale = [&](auto par_c, auto q_c, const char* st) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_c)::value, Q = decltype(q_c)::value;
    if constexpr (Q == 0)
      sa[PAR][0] = *reinterpret_cast<const uint16_t*>(st + rd_sa + PAR * 8);
    else if constexpr (Q <= TJ)
      sb[PAR][Q - 1] = *reinterpret_cast<const uint16_t*>(st + rd_sb + (Q - 1) * 256 + PAR * 8);
    else
      sa[PAR][Q - TJ] = *reinterpret_cast<const uint16_t*>(st + rd_sa + (Q - TJ) * 256 + PAR * 8);
  };
  auto mma = [&](auto par_c, auto set_c, auto t0_c, auto t1_c) __attribute__((always_inline)) {
    constexpr int SET = decltype(set_c)::value, PAR = decltype(par_c)::value;
    static_for<decltype(t0_c)::value, decltype(t1_c)::value>([&](auto t_c) __attribute__((always_inline)) {
      constexpr int T = decltype(t_c)::value;
      acc[T / TJ][T % TJ] =
          mfma_fp4<SET>(fb[SET][T % TJ], sb[PAR][T % TJ], fa[SET][T / TJ], sa[PAR][T / TJ], acc[T / TJ][T % TJ]);
    });
  };
  typedef std::integral_constant<int, 0> S0;
  typedef std::integral_constant<int, 1> S1;

  int item = blockIdx.x, m0, n0, kt0, nk, slot = 0;
  item_at(item, m0, n0, kt0, nk);
  fill_item(item);
  fill_start(S0{});
  static_for<0, NCP>(copy);
  fill_done(S0{});
  fill_start(S1{});
  static_for<0, NCP>(copy);
  fill_done(S1{});
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(NCP));  // the first k-step and its scales
  __syncthreads();
  auto first_reads = [&]() __attribute__((always_inline)) {
    static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      read(S0{}, q_c, smem);
      read_scale(S0{}, q_c, smem + 2 * kStage + slot * kScales);
    });
  };
  first_reads();
  // A k-step: the first half's MFMAs with the second half's reads between them; the
  // wait for this wave's copies of the next k-step and the barrier; the second half's
  // MFMAs with the next k-step's first reads and the copies of the k-step after next
  // into the stage just released.  (The wait in the middle of the second half, as the
  // 8-bit product has it, leaves 32 MFMAs for 64 KB of copies and all reads: 16384^3
  // 3.99 and 4.56 PFLOP/s.)
  auto first_half = [&](auto par_c) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_c)::value;
    static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      constexpr int Q = decltype(q_c)::value;
      __builtin_amdgcn_sched_barrier(0);
      read(S1{}, q_c, smem + PAR * kStage);
      mma(par_c, S0{}, std::integral_constant<int, Q * NM / NR>{}, std::integral_constant<int, (Q + 1) * NM / NR>{});
    });
    __builtin_amdgcn_sched_barrier(0);
  };
  auto step = [&](auto par_c) __attribute__((always_inline)) {
    constexpr int PAR = decltype(par_c)::value;
    typedef std::integral_constant<int, PAR ^ 1> Next;
    first_half(par_c);
    if constexpr (PAR == 1) slot ^= 1;
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // this wave's copies of the next k-step
    __syncthreads();
    fill_start(par_c);
    static_for<0, NR>([&](auto q_c) __attribute__((always_inline)) {
      constexpr int Q = decltype(q_c)::value;
      __builtin_amdgcn_sched_barrier(0);
      read(S0{}, q_c, smem + (PAR ^ 1) * kStage);
      read_scale(Next{}, q_c, smem + 2 * kStage + slot * kScales);
      static_for<Q * NCP / NR, (Q + 1) * NCP / NR>(copy);
      mma(par_c, S1{}, std::integral_constant<int, Q * NM / NR>{}, std::integral_constant<int, (Q + 1) * NM / NR>{});
    });
    __builtin_amdgcn_sched_barrier(0);
    fill_done(par_c);
  };
  for (;;) {
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    int kt = 0;
    for (; kt + 2 < nk; kt += 2) {
      step(S0{});
      step(S1{});
    }
    // The last two k-steps; with STREAM they copy the first two of the next item.  Of an
    // odd number the second is the last once more (fill_done stays there), with scales
    // of 2^-127: its products are zeros.
    if (STREAM && item + static_cast<int>(gridDim.x) < nitems) fill_item(item + gridDim.x);
    step(S0{});
    const int keep = kt + 1 < nk ? -1 : 0;
#pragma unroll
    for (int i = 0; i < TI; ++i) sa[1][i] &= keep;
#pragma unroll
    for (int j = 0; j < TJ; ++j) sb[1][j] &= keep;
    if constexpr (STREAM) {
      step(S1{});
    } else {
      first_half(S1{});
      mma(S1{}, S1{}, S0{}, std::integral_constant<int, NM>{});
    }

    // lane: channels n0 + wn WN + 16 j + 4 lq .. + 3 of token m0 + wm WM + 16 i + l16
    if (item < p.npieces) {
      float* out = p.part + static_cast<int64_t>(item) * BM * BN;
#pragma unroll
      for (int i = 0; i < TI; ++i)
#pragma unroll
        for (int j = 0; j < TJ; ++j)
          *reinterpret_cast<f32x4*>(out + (wm * WM + i * 16 + l16) * BN + wn * WN + j * 16 + 4 * lq) = acc[i][j];
    } else if constexpr (STREAM) {
      // The columns' vectors, then the row groups in batches, the residuals of a batch on
      // their way before the stores of the one before it: memory operations end in order,
      // so a load behind a store waits for it (a row group a batch: 513 us for 13104 x 5120
      // x 13824 with a bf16 residual, three 491).
      constexpr bool RES = EPI == EPI_GATE_RES;
      constexpr int BATCH = RBF ? 3 : 2, NB = (TI + BATCH - 1) / BATCH;
      const int nc = n0 + wn * WN + 4 * lq;
      // (the columns' vectors in the wave's own piece of LDS: 64 registers otherwise)
      float* const bias = reinterpret_cast<float*>(smem + 2 * kStage + 2 * kScales) + wave * 2 * WN;
      float* const gate = bias + WN;
      for (int c = lane; c < WN; c += kWave) {
        const int n = n0 + wn * WN + c < p.N ? n0 + wn * WN + c : p.N - 1;
        bias[c] = p.bias != nullptr ? out_load(p.bias, p.bias_bf16, n) : 0.0f;
        if constexpr (RES) gate[c] = p.gate[n];
      }
      ResRaw<RBF> raw[RES ? 2 * BATCH : 1][RES ? TJ : 1];
      bool miss[2 * BATCH];
      auto fetch = [&](auto b_c) __attribute__((always_inline)) {
        constexpr int b = decltype(b_c)::value;
        if constexpr (RES && b < NB) {
#pragma unroll
          for (int i = b * BATCH; i < (b + 1) * BATCH && i < TI; ++i) {
            const int at = i % (2 * BATCH), m = m0 + wm * WM + i * 16 + l16;
            const int rr = out_res_row(p, m < p.M ? m : p.M - 1);
            miss[at] = rr < 0;
#pragma unroll
            for (int j = 0; j < TJ; ++j)
              raw[at][j].load(p.res, static_cast<int64_t>(rr < 0 ? 0 : rr) * p.ldr +
                                         (nc + 16 * j < p.N ? nc + 16 * j : p.N - 4));
          }
        }
      };
      acc_settled(acc[TI - 1][TJ - 1]);
      fetch(S0{});
      static_for<0, TI>([&](auto i_c) __attribute__((always_inline)) {
        constexpr int i = decltype(i_c)::value, at_i = i % (2 * BATCH);
        if constexpr (i % BATCH == 0) fetch(std::integral_constant<int, i / BATCH + 1>{});
        const int m = m0 + wm * WM + i * 16 + l16;
        static_for<0, TJ / 2>([&](auto j_c) __attribute__((always_inline)) {
          constexpr int j = decltype(j_c)::value * 2;
          float z[2][4];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            float res[4];
            if constexpr (RES) raw[at_i][j + h].unpack(miss[at_i], res);
            const f32x4 cb = *reinterpret_cast<const f32x4*>(bias + 16 * (j + h) + 4 * lq);
            f32x4 cg = {};
            if constexpr (RES) cg = *reinterpret_cast<const f32x4*>(gate + 16 * (j + h) + 4 * lq);
#pragma unroll
            for (int r = 0; r < 4; ++r)
              z[h][r] = out_finish<EPI>(from_acc(acc[i][j + h][r]) + cb[r], cg[r], res[r]);
          }
          const int64_t row = m * p.ldc;
          const int at = n0 + wn * WN + 16 * j;
          if (CBF) {
            // (every lane takes part in the swaps)
            const uint32_t a0 = pack_bf16x2(z[0][0], z[0][1]), a1 = pack_bf16x2(z[0][2], z[0][3]);
            const uint32_t b0 = pack_bf16x2(z[1][0], z[1][1]), b1 = pack_bf16x2(z[1][2], z[1][3]);
            const auto s0 = __builtin_amdgcn_permlane32_swap(a0, b0, false, false);
            const auto s1 = __builtin_amdgcn_permlane32_swap(a1, b1, false, false);
            const auto t0 = __builtin_amdgcn_permlane16_swap(s0[0], s0[1], false, false);
            const auto t1 = __builtin_amdgcn_permlane16_swap(s1[0], s1[1], false, false);
            if (m < p.M && at + 8 * lq < p.N)
              stg16(static_cast<bf16_t*>(p.C) + row + at + 8 * lq, make_uint4(t0[0], t1[0], t0[1], t1[1]));
          } else {
#pragma unroll
            for (int h = 0; h < 2; ++h)
              if (m < p.M && at + 16 * h + 4 * lq < p.N)
                stg16(static_cast<float*>(p.C) + row + at + 16 * h + 4 * lq, pack16(z[h], static_cast<const float*>(nullptr)));
          }
        });
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    if constexpr (STREAM) {
      item += gridDim.x;
      if (item < nitems) {
        item_at(item, m0, n0, kt0, nk);
        // the first reads again: held through the stores they cost 80 registers
        first_reads();
        continue;
      }
    }
    break;
  }
  __builtin_amdgcn_s_waitcnt(0);  // re-fetched k-steps still landing in LDS
  if (STREAM || item < p.npieces) return;
  // The epilogue of gemm_int8.hip: sixteen tokens of the wave's part at a time
  // through the wave's own piece of LDS, whole rows a store, residuals ahead.
  constexpr int LD = WN + 4, CPL = WN / 4, RPP = kWave / CPL, NQ = 16 / RPP;
  static_assert(4 * 16 * LD * 4 <= 2 * kStage, "staging fits the ring");
  __syncthreads();  // every wave's copies have landed and its last reads are done
  float* ep = reinterpret_cast<float*>(smem) + wave * 16 * LD;
  const bool vec = out_vec(p);
  const int cl = lane % CPL * 4, rl = lane / CPL;
  const int n = n0 + wn * WN + cl;
  OutCols cols;
  if (vec) out_cols4<EPI>(p, n < p.N ? n : p.N - 4, cols);
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
      // (as there: keeps the accumulators where they are until their turn)
      if constexpr (BM * BN == 256 * 256) asm volatile("" : "+a"(acc[i][j]));
      *reinterpret_cast<f32x4*>(ep + l16 * LD + j * 16 + 4 * lq) = acc[i][j];
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

// The k-ranges of every split tile added in order, in fp32, and the epilogue; a
// thread takes four channels of a token.
template <int BM, int BN, int EPI, bool CBF>
__global__ void __launch_bounds__(256) gemm_fp4_reduce(GemmFp4Args p) {
  const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int c4 = static_cast<int>(e % (BN / 4)), r = static_cast<int>((e / (BN / 4)) % BM);
  const int t = static_cast<int>(e / (static_cast<int64_t>(BM) * (BN / 4)));
  if (p.tile_base + t >= tm * tn) return;
  int tile_m, tile_n;
  gemm_tile_of(p.tile_base + t, tm, tn, tile_m, tile_n);
  const int m = tile_m * BM + r, n = tile_n * BN + 4 * c4;
  if (m >= p.M || n >= p.N) return;
  f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < p.nsplit; ++s)
    acc += *reinterpret_cast<const f32x4*>(p.part + (static_cast<int64_t>(t) * p.nsplit + s) * BM * BN + r * BN +
                                           4 * c4);
  out_put4<EPI, CBF>(p, m, n, acc);
}

// ---- one to eight tokens: the read of the weights is all there is.  A wave
// takes R channels and reads each in pieces of 1 KB, 16 contiguous bytes (a
// block) a lane, U pieces of every channel in flight.  The matrix instruction's
// sixteen rows are then sixteen blocks of ONE channel and its sixteen columns the
// same blocks of one token: the sums of corresponding blocks, which are wanted,
// lie on the diagonal of its result and the other 240 are dropped.  At a
// sixteenth of its rate the instruction is still several times faster than the
// memory (an MFMA of 16 cycles takes 1 KB, 256 bytes a cycle and CU, where the
// memory delivers 11), and it needs no conversion of the codes.
template <int MT, int R, int U, int EPI, bool CBF>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 4))) gemm_fp4_row(GemmFp4Args p) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  const int n0 = (blockIdx.x * 4 + wave) * R;
  if (n0 >= p.N) return;
  const uint8_t *w[R], *ws[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t n = n0 + r < p.N ? n0 + r : p.N - 1;
    w[r] = p.B + n * p.ldb;
    ws[r] = p.sb + n * p.ldsb;
  }
  f32x4 acc[R][MT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int k0 = 0; k0 < p.K; k0 += 1024 * U) {
    i32x4 wf[U][R], af[U][MT];
    int wsc[U][R], asc[U][MT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * 1024 + lane * 16, kc = k < p.K ? k : 0;  // past the depth: zeros of the token
#pragma unroll
      for (int r = 0; r < R; ++r) {
        wf[u][r] = __builtin_bit_cast(i32x4, __builtin_nontemporal_load(reinterpret_cast<const u32x4_t*>(w[r] + kc)));
        wsc[u][r] = ws[r][kc / 16];
      }
#pragma unroll
      for (int t = 0; t < MT; ++t) {
        const int64_t m = t < p.M ? t : p.M - 1;
        af[u][t] = *reinterpret_cast<const i32x4*>(p.A + m * p.lda + kc);
        asc[u][t] = p.sa[m * p.ldsa + kc / 16];
        if (k >= p.K) af[u][t] = i32x4{0, 0, 0, 0};
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < MT; ++t) acc[r][t] = mfma_fp4<0>(wf[u][r], wsc[u][r], af[u][t], asc[u][t], acc[r][t]);
  }
  // lane (q, i): rows 4 q .. 4 q + 3 of column i; the diagonal's element of column
  // i lies in lane (i / 4, i), at i % 4
  const int i = lane & 15;
  const bool diag = i / 4 == lane / 16;
  float sum[R][MT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const f32x4 a = acc[r][t];
      const float v = i % 4 < 2 ? (i % 4 == 0 ? a[0] : a[1]) : (i % 4 == 2 ? a[2] : a[3]);
      sum[r][t] = wave_sum(diag ? v : 0.0f);
    }
  // lane l of pass s stores output 64 s + l = r MT + t: channel n0 + r of token t
#pragma unroll
  for (int s = 0; s < (R * MT + 63) / 64; ++s) {
    float mine = 0.0f;
#pragma unroll
    for (int e = 64 * s; e < R * MT && e < 64 * s + 64; ++e) mine = lane == e - 64 * s ? sum[e / MT][e % MT] : mine;
    const int e = 64 * s + lane, n = n0 + e / MT, m = e % MT;
    if (e < R * MT && n < p.N && m < p.M) out_store1<EPI, CBF>(p, m, n, mine);
  }
}

// ---- three to 32 tokens: one launch of many small workgroups, where a tile's stages
// and a second launch to join the depth's pieces would be most of the time.  A workgroup
// takes R times sixteen channels, and its waves share the depth: a wave reads 256 codes
// of every channel at a time, U such pieces in flight, and the same codes of the tokens,
// sixteen to an instruction's columns.  The waves' sums meet in LDS and are added in the
// waves' order.  The fragments are read as the instruction holds them, neighbouring lanes
// in different rows, which the first-level cache serves at an eighth of its rate: that
// bounds it (8 tokens on 1536 x 1536 codes 2.8 us where tiles and rows of 4.8 are, on
// 5120 x 5120 7.2 and 9.7, but on 30720 x 5120 22.7 and 15.1).
template <int TT, int R, int U, int EPI, bool CBF>
__global__ void __launch_bounds__(1024) gemm_fp4_few(GemmFp4Args p) {
  extern __shared__ f32x4 sums[];  // [wave][R][TT][lane]
  const int lane = threadIdx.x % kWave, waves = blockDim.x / kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int l16 = lane & 15, lq = lane / 16, n0 = blockIdx.x * 16 * R, units = p.K / 128;
  const uint8_t *w[R], *ws[R], *a[TT], *as[TT];  // (rows past the last one: the last one, not stored)
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int64_t n = n0 + 16 * r + l16 < p.N ? n0 + 16 * r + l16 : p.N - 1;
    w[r] = p.B + n * p.ldb + lq * 32;
    ws[r] = p.sb + n * p.ldsb + lq * 2;
  }
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int64_t m = 16 * t + l16 < p.M ? 16 * t + l16 : p.M - 1;
    a[t] = p.A + m * p.lda + lq * 32;
    as[t] = p.sa + m * p.ldsa + lq * 2;
  }
  f32x4 acc[R][TT];
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int u0 = wave * U; u0 < units; u0 += waves * U) {
    i32x4 wf[U][R][2], af[U][TT][2];
    int wsc[U][R], asc[U][TT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = u0 + u < units ? u0 + u : u0;  // (past the depth: read again, not used)
#pragma unroll
      for (int r = 0; r < R; ++r) {
        const u32x4_t* q = reinterpret_cast<const u32x4_t*>(w[r] + k * 128);
        wf[u][r][0] = __builtin_bit_cast(i32x4, q[0]);
        wf[u][r][1] = __builtin_bit_cast(i32x4, q[1]);
        wsc[u][r] = *reinterpret_cast<const uint16_t*>(ws[r] + k * 8);
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const i32x4* q = reinterpret_cast<const i32x4*>(a[t] + k * 128);
        af[u][t][0] = q[0];
        af[u][t][1] = q[1];
        asc[u][t] = *reinterpret_cast<const uint16_t*>(as[t] + k * 8);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (u0 + u >= units) break;
#pragma unroll
      for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < TT; ++t) {
          acc[r][t] = mfma_fp4<0>(wf[u][r][0], wsc[u][r], af[u][t][0], asc[u][t], acc[r][t]);
          acc[r][t] = mfma_fp4<1>(wf[u][r][1], wsc[u][r], af[u][t][1], asc[u][t], acc[r][t]);
        }
    }
  }
#pragma unroll
  for (int r = 0; r < R; ++r)
#pragma unroll
    for (int t = 0; t < TT; ++t) sums[((wave * R + r) * TT + t) * kWave + lane] = acc[r][t];
  __syncthreads();
  for (int e = threadIdx.x; e < R * TT * kWave; e += blockDim.x) {
    f32x4 z = sums[e];
    for (int v = 1; v < waves; ++v) z += sums[v * R * TT * kWave + e];
    const int l = e % kWave, rt = e / kWave, m = rt % TT * 16 + l % 16, n = n0 + rt / TT * 16 + l / 16 * 4;
    if (m < p.M && n < p.N) out_put4<EPI, CBF>(p, m, n, z);
  }
}

namespace {

constexpr int kRowMax = 8;   // most tokens of gemm_fp4_row
constexpr int kFewMax = 32;  // and of gemm_fp4_few

enum Fp4Tile { FP4_256, FP4_128, FP4_64 };
constexpr int kTileEdge[] = {256, 128, 64};

// Estimated time of a plan, us, in the form of gemm_int8.hip's estimate: fitted to
// 166 products of 1 .. 32760 tokens, 64 .. 30720 channels and depths 128 .. 13824 in
// every tile and split (1789 times; 5 to 9% off on average; the choice by them is 1%
// slower than the fastest plan on average, 2 and 3% with GELU or gate and residual).
// k-steps run in pairs.
struct Fp4Cost {
  int resident;
  float start, lat, thr;  // launch and first loads; a k-step
  float store[3];         // each epilogue, for a workgroup on every CU
  float join, piece;      // the second launch of a split product; 1 MB of partial sums
  float cold;             // a k-step's loads with the weights beyond the L2s (32 MB)
};
constexpr Fp4Cost kFp4Cost[] = {{1, 5.96f, 1.385f, 0.902f, {11.58f, 15.70f, 29.66f}, 7.28f, 0.100f, 0.007f},
                                {2, 4.25f, 0.725f, 0.550f, {2.77f, 3.31f, 4.72f}, 2.13f, 0.249f, 0.060f},
                                {4, 2.66f, 0.551f, 0.216f, {0.67f, 0.75f, 1.26f}, 2.43f, 0.357f, 0.093f}};

struct Fp4Plan {
  int tile;
  int base, nsplit, kps;  // tiles from `base` on are split in nsplit ranges of kps k-steps
  float us;
};

int64_t fp4_tiles(int tile, int M, int N) {
  const int64_t e = kTileEdge[tile];
  return ((M + e - 1) / e) * ((N + e - 1) / e);
}
size_t fp4_part_bytes(const Fp4Plan& p, int M, int N) {
  const size_t e = kTileEdge[p.tile];
  return p.nsplit < 2 ? 0 : sizeof(float) * e * e * (fp4_tiles(p.tile, M, N) - p.base) * p.nsplit;
}

float fp4_us(const Fp4Plan& p, int M, int N, int K, int epi, int ncu) {
  const Fp4Cost& c = kFp4Cost[p.tile];
  const int nk = K / 128;
  auto run = [&](int64_t pieces, int steps) {
    const int64_t n = (pieces + ncu - 1) / ncu;  // workgroups on the busiest CU
    const float full = c.resident * c.thr > c.lat ? c.resident * c.thr : c.lat;
    const int rest = static_cast<int>(n % c.resident);
    const float last = rest == 0 ? 0.0f : rest * c.thr > c.lat ? rest * c.thr : c.lat;
    return (n / c.resident * full + last) * ((steps + 1) / 2 * 2) + c.store[epi] * static_cast<float>(pieces) / ncu;
  };
  const float beyond = static_cast<float>(N) * K / 32e6f;
  float us = c.start + c.cold * (beyond < 1.0f ? beyond : 1.0f) * nk;
  if (p.base > 0) us += run(p.base, nk);
  const int64_t tail = fp4_tiles(p.tile, M, N) - p.base;
  if (tail > 0) us += run(tail * p.nsplit, p.kps) + c.join + c.piece * 1e-6f * fp4_part_bytes(p, M, N);
  return us;
}

// Every tile whole; or the tiles beyond the last whole round of the device, or
// all of them where they are less than a round, split along the depth: the
// fastest by the estimate.
Fp4Plan fp4_plan(int M, int N, int K, int epi) {
  const int ncu = device_cu_count(), nk = K / 128;
  constexpr size_t kMostPartial = size_t(64) << 20;
  Fp4Plan best{-1, 0, 1, nk, 0.0f};
  auto consider = [&](int tile, int64_t base, int ns) {
    const int even = (nk + ns - 1) / ns, kps = ns > 1 ? (even + 1) / 2 * 2 : even;
    Fp4Plan p{tile, static_cast<int>(base), (nk + kps - 1) / kps, kps, 0.0f};  // every range non-empty
    if (fp4_part_bytes(p, M, N) > kMostPartial) return;
    p.us = fp4_us(p, M, N, K, epi, ncu);
    if (best.tile < 0 || p.us < best.us) best = p;
  };
  for (int tile = FP4_256; tile <= FP4_64; ++tile) {
    const int64_t tiles = fp4_tiles(tile, M, N), round = static_cast<int64_t>(ncu) * kFp4Cost[tile].resident;
    consider(tile, tiles, 1);
    for (const int ns : {2, 3, 4, 6, 8, 12, 16})
      if (nk / ns >= 2 && tiles % round != 0 && tiles < round * 64) consider(tile, tiles / round * round, ns);
  }
  return best;
}

// whether rows of C, of the residual and the vectors over the channels are aligned
// for 16-byte stores of four fp32 or eight bf16 outputs
bool stream_fits(const GemmFp4Args& a) {
  auto at = [](const void* q, int bytes) { return reinterpret_cast<uintptr_t>(q) % bytes == 0; };
  const int per = a.c_bf16 ? 8 : 4;
  return a.N % per == 0 && a.ldc % per == 0 && at(a.C, 16) && at(a.bias, a.bias_bf16 ? 8 : 16) && at(a.gate, 16) &&
         at(a.res, a.res_bf16 ? 8 : 16) && a.ldr % 4 == 0;
}

template <int E>
hipError_t launch_tile(int epi, GemmFp4Args a, const Fp4Plan& plan, hipStream_t stream) {
  const int tiles = static_cast<int>(fp4_tiles(plan.tile, a.M, a.N)), tail = plan.nsplit > 1 ? tiles - plan.base : 0;
  a.tile_base = tiles - tail;
  a.nsplit = plan.nsplit;
  a.kps = plan.kps;
  a.npieces = tail * plan.nsplit;
  const int items = a.npieces + a.tile_base;
  return with_epilogue(epi, a.c_bf16, a.res_bf16, [&](auto epi_c, auto bf_c, auto res_c) -> hipError_t {
    constexpr int EPI = decltype(epi_c)::value;
    constexpr bool CBF = decltype(bf_c)::value, RBF = decltype(res_c)::value;
    constexpr const char* kName = E == 256 ? "gemm_fp4_256" : E == 128 ? "gemm_fp4_128" : "gemm_fp4_64";
    hipError_t e;
    // (the smaller tiles have several workgroups to a CU, whose ends overlap)
    if (E == 256 && stream_fits(a)) {
      const int wgs = items < device_cu_count() ? items : device_cu_count();
      e = ECHO_LAUNCH("gemm_fp4_256_stream", (gemm_fp4_tile<E, E, EPI, CBF, RBF, E == 256>),
                      dim3(static_cast<unsigned>(wgs)), dim3(256), 0, stream, a);
    } else {
      e = ECHO_LAUNCH(kName, (gemm_fp4_tile<E, E, EPI, CBF, RBF, false>), dim3(static_cast<unsigned>(items)),
                      dim3(256), 0, stream, a);
    }
    if (e != hipSuccess || tail == 0) return e;
    const int64_t n = static_cast<int64_t>(tail) * E * (E / 4);
    return ECHO_LAUNCH("gemm_fp4_reduce", (gemm_fp4_reduce<E, E, EPI, CBF>),
                       dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256), 0, stream, a);
  });
}

template <int MT, int R, int U>
hipError_t launch_row(int epi, const GemmFp4Args& a, hipStream_t stream) {
  const dim3 grid(static_cast<unsigned>((a.N + 4 * R - 1) / (4 * R)));
  return with_epilogue(epi, a.c_bf16, 1, [&](auto epi_c, auto bf_c, auto) -> hipError_t {
    return ECHO_LAUNCH("gemm_fp4_row", (gemm_fp4_row<MT, R, U, decltype(epi_c)::value, decltype(bf_c)::value>), grid,
                       dim3(256), 0, stream, a);
  });
}

template <int TT, int R, int U>
hipError_t launch_few(int epi, const GemmFp4Args& a, hipStream_t stream) {
  // as many waves as the depth keeps busy, up to 16, with equal shares
  const int pieces = (a.K / 128 + U - 1) / U, rounds = (pieces + 15) / 16, waves = (pieces + rounds - 1) / rounds;
  const dim3 grid(static_cast<unsigned>((a.N + 16 * R - 1) / (16 * R)));
  return with_epilogue(epi, a.c_bf16, 1, [&](auto epi_c, auto bf_c, auto) -> hipError_t {
    return ECHO_LAUNCH("gemm_fp4_few", (gemm_fp4_few<TT, R, U, decltype(epi_c)::value, decltype(bf_c)::value>), grid,
                       dim3(waves * kWave), static_cast<unsigned>(waves * R * TT * kWave * 16), stream, a);
  });
}

}  // namespace

// How a product is done.  Of few tokens by rows: that reads the weights at the memory's
// rate, but the tokens' codes again for every two channels, through the same path
// (1 / 2 / 4 / 8 tokens on 5120 x 5120 codes 5.0 / 5.7 / 6.5 / 9.7 us, tiles 11.3; on
// 30720 x 5120 15.9 / 16.9 / 23.1 / 35.5, tiles 20.2); or by groups of 16 or 32
// channels, whose time is their rounds on the device by the depth (16 tokens on 1536 x
// 1536 / 5120 x 5120 3.0 / 7.9, tiles 4.2 / 10.5); else in tiles.
enum Fp4Way { FP4_TILES, FP4_ROWS, FP4_FEW16, FP4_FEW32 };
static Fp4Way fp4_way(int M, int N, int K, const Fp4Plan& plan) {
  if (M <= 2) return FP4_ROWS;
  Fp4Way way = FP4_TILES;
  float us = plan.us;  // (up to a sixth too long for 9 to 32 tokens on deep rows: `margin`)
  auto consider = [&](Fp4Way w, float t) {
    if (t < us) us = t, way = w;
  };
  const float margin = M <= kRowMax ? 1.0f : 1.17f;
  const float depth = K / 512.0f;  // 1024 codes
  auto rounds = [&](int channels) {
    const int ncu = device_cu_count(), wgs = (N + channels - 1) / channels;
    return static_cast<float>((wgs + ncu - 1) / ncu);
  };
  if (M <= kRowMax) consider(FP4_ROWS, 2.9f + (0.15f + 0.031f * M) * 1e-6f * N * K);
  if (M <= kFewMax) consider(FP4_FEW16, margin * (2.2f + rounds(16) * depth * (0.42f + 0.0185f * M)));
  if (M <= kFewMax) consider(FP4_FEW32, margin * (2.4f + rounds(32) * depth * (0.82f + 0.0185f * M)));
  return way;
}

size_t gemm_fp4_partial_bytes(int M, int N, int K, int epi) {
  if (M <= 2) return 0;
  const Fp4Plan plan = fp4_plan(M, N, K, epi);
  return fp4_way(M, N, K, plan) != FP4_TILES ? 0 : fp4_part_bytes(plan, M, N);
}

hipError_t launch_gemm_fp4(int epi, const GemmFp4Args& a, hipStream_t stream) {
  // two channels a wave and 3 KB of each in flight (one token on 30720 x 5120 and 5120 x
  // 5120 codes 15.9 and 5.0 us; four channels 15.5 and 5.4, 5 KB 17.6 and 5.6)
  if (a.M == 1) return launch_row<1, 2, 3>(epi, a, stream);
  if (a.M == 2) return launch_row<2, 2, 3>(epi, a, stream);
  const Fp4Plan plan = fp4_plan(a.M, a.N, a.K, epi);
  switch (fp4_way(a.M, a.N, a.K, plan)) {
    case FP4_ROWS: return a.M <= 4 ? launch_row<4, 2, 3>(epi, a, stream) : launch_row<8, 2, 3>(epi, a, stream);
    case FP4_FEW16: return a.M <= 16 ? launch_few<1, 1, 2>(epi, a, stream) : launch_few<2, 1, 2>(epi, a, stream);
    case FP4_FEW32: return a.M <= 16 ? launch_few<1, 2, 2>(epi, a, stream) : launch_few<2, 2, 2>(epi, a, stream);
    case FP4_TILES: break;
  }
  if (fp4_part_bytes(plan, a.M, a.N) > a.part_bytes) return hipErrorInvalidValue;
  switch (plan.tile) {
    case FP4_256: return launch_tile<256>(epi, a, plan, stream);
    case FP4_128: return launch_tile<128>(epi, a, plan, stream);
    default: return launch_tile<64>(epi, a, plan, stream);
  }
}

}  // namespace echo
