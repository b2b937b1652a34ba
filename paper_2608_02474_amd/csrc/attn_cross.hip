// Attention of Lq queries to the Lk states of an encoder, B elements, H query
// heads over Hkv state heads (G = H / Hkv queries heads share one):
//
//   o[b, i, h] = sum_j softmax_j(scale q[b, i, h] . k[b, j, h / G]) v[b, j, h / G]
//
// over the states j < k_len[b] that key_mask[b] leaves; a query with no state
// left, or none of any weight, gets zeros.  Masked states are never read into
// a product, so what lies in them (infinities, NaN, uninitialised memory) has
// no effect: a mask is compacted to a list of the states it leaves, in order
// (cross_keys), and the kernels walk that list; without a mask they walk the
// first k_len[b].  Work follows the states that are left.
//
// Rows.  The G Lq queries that share a state head are rows r = g Lq + i of one
// problem, so a tile of 128 rows is as full for one query of 8 shared heads as
// for many queries.  A workgroup of four waves takes 128 rows (32 a wave) and
// walks tiles of states; where the rows do not fill the device the tiles are
// split over nsplit workgroups, whose partial sums, maxima and outputs (fp32)
// are joined by cross_combine.
//
// bf16 (cross_bf16): tiles of 64 states, K and V through a two-stage LDS ring
// of direct copies (swizzled as in the block's attention), S^T = K q^T and
// O^T += V^T P^T on v_mfma_f32_32x32x16_bf16; the K rows enter permuted so that
// a lane's scores are, once rounded to bf16, the operand of the second product.
// fp32 (cross_f32): tiles of 32 states on v_mfma_f32_32x32x2_f32, whose score
// registers are the second product's operand as they are.
// Softmax: running maximum and sum in fp32, in units of log2.  The maximum moves
// only when it has grown by so much that the weights against it (which stay
// below 2^8) need it: in fp32 by more than 2^8, in bf16 once a lane's 16 weights
// of a half tile sum to more, so that a rescale is rare.
#include <math.h>

#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

typedef short xv4i16 __attribute__((ext_vector_type(4)));
typedef __bf16 xbf16x2 __attribute__((ext_vector_type(2)));

constexpr int X_ROWS = 128;                 // rows of a workgroup, 32 a wave
constexpr int X_KT = 64;                    // states of a bf16 tile
constexpr int X_KT32 = 32;                  // states of an fp32 tile
constexpr int X_RING = 4;                   // LDS reads ahead of the matrix cores
constexpr float X_GROW = 8.0f;              // log2 of the growth that moves the maximum (fp32)
constexpr float X_GROW_SUM = 256.0f;        // sum of 16 weights that does (bf16)
constexpr float X_LOW = -3.402823466e38f;   // the maximum before any state: the lowest finite value

__device__ __forceinline__ int x_swap23(int r) { return (r & ~12) | ((r & 4) << 1) | ((r & 8) >> 1); }

// K row r (2 DH bytes in chunks of 16): chunk c lives in slot c ^ x_kx(r); the 16
// rows that one LDS cycle reads at one chunk then hit distinct bank groups.
template <int DH>
__device__ __forceinline__ int x_kx(int r) {
  return DH == 128 ? x_swap23(r & 15) : (r >> 1) & 7;
}
// V row r (in blocks of 32 bytes): block c lives in c ^ x_vx(r); a transpose read
// takes blocks 2 d, 2 d + 1 of four consecutive rows from distinct banks.
template <int DH>
__device__ __forceinline__ int x_vx(int r) {
  return DH == 128 ? (r & 3) << 1 : r & 2;
}

// ---- where a workgroup works
struct XItem {
  int b, hk, tile, split;  // element, state head, tile of rows, range of the states' tiles
  int t0, t1;              // tiles of states [t0, t1)
  int n;                   // states left
};
// Consecutive items share K and V, and an XCD takes a contiguous range of them.
// The (element, head) groups go by their number modulo 8 first, so that every
// XCD gets its share of each element, whatever their lengths (elements one after
// the other, of 512 and of 64 states: 305 us, now 228).
__device__ __forceinline__ XItem x_item(const CrossArgs& p, int tiles, int kt) {
  const int nb = gridDim.x, per = nb / 8, rem = nb % 8, xcd = blockIdx.x % 8;
  int i = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
  XItem x;
  x.tile = i % tiles;
  i /= tiles;
  x.split = i % p.nsplit;
  i /= p.nsplit;
  const int groups = p.B * p.Hkv, most = groups / 8, more = groups % 8;  // `more` residues have most + 1 groups
  const int first = more * (most + 1);
  const int group = i < first ? i % (most + 1) * 8 + i / (most + 1)
                              : (i - first) % most * 8 + more + (i - first) / most;
  x.hk = group % p.Hkv;
  x.b = group / p.Hkv;
  if (p.key_mask != nullptr) {
    x.n = p.key_count[x.b];
  } else {
    x.n = p.k_len != nullptr ? p.k_len[x.b] : p.Lk;
    x.n = x.n < 0 ? 0 : (x.n < p.Lk ? x.n : p.Lk);
  }
  x.n = __builtin_amdgcn_readfirstlane(x.n);
  const int nt = (x.n + kt - 1) / kt;
  x.t0 = static_cast<int>(static_cast<int64_t>(nt) * x.split / p.nsplit);
  x.t1 = static_cast<int>(static_cast<int64_t>(nt) * (x.split + 1) / p.nsplit);
  return x;
}

// row r = g Lq + i of the queries that share a state head
__device__ __forceinline__ void x_row(const CrossArgs& p, int r, int& g, int& i) {
  if (p.H == p.Hkv) {
    g = 0;
    i = r;
  } else if (p.Lq == 1) {
    g = r;
    i = 0;
  } else {
    g = r / p.Lq;
    i = r - g * p.Lq;
  }
}

// ---- partial results of a range: for the row's unit u, DH outputs, then all
// units' maxima and sums
__device__ __forceinline__ int64_t x_unit(const CrossArgs& p, const XItem& x, int tiles, int row) {
  return ((static_cast<int64_t>(x.b * p.Hkv + x.hk) * p.nsplit + x.split) * tiles + x.tile) * X_ROWS + row;
}
__device__ __forceinline__ int64_t x_units(const CrossArgs& p, int tiles) {
  return static_cast<int64_t>(p.B) * p.Hkv * p.nsplit * tiles * X_ROWS;
}

// ---- states that the mask leaves, in order; a workgroup per element (it goes on
// to others where there are more elements than workgroups), eight states a
// thread and turn
__global__ void __launch_bounds__(1024) cross_keys(CrossArgs p) {
  __shared__ int wave_n[16];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
    int n = p.k_len != nullptr ? p.k_len[b] : p.Lk;
    n = n < 0 ? 0 : (n < p.Lk ? n : p.Lk);
    const uint8_t* mask = p.key_mask + static_cast<int64_t>(b) * p.Lk;
    int32_t* list = p.key_list + static_cast<int64_t>(b) * p.Lk;
    int base = 0;
    for (int64_t j0 = 0; j0 < n; j0 += 8192) {
      const int64_t j = j0 + 8 * tid;
      uint32_t bits = 0;
#pragma unroll
      for (int e = 0; e < 8; ++e) bits |= (j + e < n && mask[j + e] != 0 ? 1u : 0u) << e;
      const int mine = __popc(bits);
      int upto = mine;  // of this lane and those before it
#pragma unroll
      for (int d = 1; d < kWave; d *= 2) {
        const int other = __shfl_up(upto, d);
        upto += lane >= d ? other : 0;
      }
      if (lane == kWave - 1) wave_n[wave] = upto;
      __syncthreads();
      int at = base + upto - mine, total = 0;
#pragma unroll
      for (int w = 0; w < 16; ++w) {
        at += w < wave ? wave_n[w] : 0;
        total += wave_n[w];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (bits >> e & 1u) list[at++] = static_cast<int32_t>(j) + e;
      base += total;
      __syncthreads();
    }
    if (tid == 0) p.key_count[b] = base;
  }
}

// ------------------------------------------------------------------- bf16
template <int DH, bool MASK>
__global__ void __launch_bounds__(256, 2) cross_bf16(CrossArgs p) {
  constexpr int ND = DH / 32, NS = DH / 16;      // 32-wide output blocks, 16-deep score steps
  constexpr int RB = 2 * DH;                     // bytes of a K or V row
  constexpr int TILE = X_KT * RB;                // bytes of a K or V tile
  constexpr int RPP = 1024 / RB;                 // rows of a 1 KB copy
  constexpr int NP = TILE / 1024 / 4;            // K (and V) copies of a wave and tile
  constexpr int OS = DH + 8;                     // staged output row
  // two stages of K, then three of V: 80 KB at dh 128, two workgroups to a CU
  constexpr int VB = 2 * TILE;
  static_assert(5 * TILE >= X_ROWS * OS * 2, "the output's rows fit the ring");
  __shared__ __attribute__((aligned(1024))) char smem[5 * TILE];
  const int tid = threadIdx.x, lane = tid % kWave, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int rows = p.H / p.Hkv * p.Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
  const XItem x = x_item(p, tiles, X_KT);
  const bf16_t* kb = static_cast<const bf16_t*>(p.k) + x.b * p.kb + x.hk * p.kh;
  const bf16_t* vb = static_cast<const bf16_t*>(p.v) + x.b * p.vb + x.hk * p.vh;
  const int32_t* list = MASK ? p.key_list + static_cast<int64_t>(x.b) * p.Lk : nullptr;

  // ---- copies.  Copy m of this wave is rows RPP (wave + 4 m) .. of the tile;
  // the lane lands in row lr of them, slot ls, and fetches the chunk that lives
  // there.  Whole tiles without a list take a uniform base and offsets that are
  // the same for every tile; the last tile and listed states an address each.
  const int lr = lane / (RB / 16), ls = lane % (RB / 16);
  const uint32_t lds0 = lds_offset(smem) + wave * 1024;
  uint32_t koff[NP], voff[NP];
#pragma unroll
  for (int m = 0; m < NP; ++m) {
    const int r = RPP * (wave + 4 * m) + lr;
    koff[m] = (static_cast<uint32_t>(r) * static_cast<uint32_t>(p.kr) + (ls ^ x_kx<DH>(r)) * 8) * 2;
    voff[m] = (static_cast<uint32_t>(r) * static_cast<uint32_t>(p.vr) +
               ((((ls >> 1) ^ x_vx<DH>(r)) << 1) + (ls & 1)) * 8) * 2;
  }
  // the list's entries for this lane's rows of a tile, a tile ahead
  int listed[NP];
  auto look = [&](int u) __attribute__((always_inline)) {
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int key = (x.t0 + u) * X_KT + RPP * (wave + 4 * m) + lr;
      listed[m] = list[key < x.n ? key : x.n - 1];
    }
  };
  auto issue = [&](int u) __attribute__((always_inline)) {  // the u-th tile of the range
    const int t = x.t0 + u;
    const uint32_t kd = lds0 + (u & 1) * TILE, vd = lds0 + VB + u % 3 * TILE;
    if (!MASK && (t + 1) * X_KT <= x.n) {
      const bf16_t* ks = kb + static_cast<int64_t>(t) * X_KT * p.kr;
      const bf16_t* vs = vb + static_cast<int64_t>(t) * X_KT * p.vr;
#pragma unroll
      for (int m = 0; m < NP; ++m) lds_copy16_s(ks, koff[m], kd + m * 4096);
#pragma unroll
      for (int m = 0; m < NP; ++m) lds_copy16_s(vs, voff[m], vd + m * 4096);
      return;
    }
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int r = RPP * (wave + 4 * m) + lr;
      int key = t * X_KT + r < x.n ? t * X_KT + r : x.n - 1;  // past the end: the last state again, never used
      if constexpr (MASK) key = listed[m];
      const int64_t at = static_cast<int64_t>(key) - r;
      lds_copy16(reinterpret_cast<const char*>(kb + at * p.kr) + koff[m], kd + m * 4096);
      lds_copy16(reinterpret_cast<const char*>(vb + at * p.vr) + voff[m], vd + m * 4096);
    }
    if constexpr (MASK) look(u + 1);
  };
  const int nt = x.t1 - x.t0;
  if constexpr (MASK)
    if (nt > 0) look(0);
  if (nt > 0) issue(0);

  // ---- the wave's 32 queries, through LDS as well (whole rows a load; straight
  // to registers a row came as 32-byte pieces of 8 loads and the L1 did not hold
  // them): they lie where the values of tiles 1 and 2 will, swizzled as K
  const int row0 = x.tile * X_ROWS + wave * 32;
  const bool idle = row0 >= rows;  // no row in this wave: it copies and waits with the others
  char* qs = smem + VB + TILE + wave * 32 * RB;
  if (!idle && nt > 0) {
    const bf16_t* qb = static_cast<const bf16_t*>(p.q) + x.b * p.qb + static_cast<int64_t>(x.hk) * (p.H / p.Hkv) * p.qh;
#pragma unroll
    for (int m = 0; m < 32 / RPP; ++m) {
      const int rl = RPP * m + lr;
      int g, i;
      x_row(p, row0 + rl < rows ? row0 + rl : rows - 1, g, i);
      lds_copy16(qb + i * p.qr + g * p.qh + (ls ^ x_kx<DH>(rl)) * 8, lds_offset(qs) + m * 1024);
    }
  }
  // ---- fragment addresses in a stage
  int k_rd[NS], v_rd[ND];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int r = x_swap23(l32);
    k_rd[s] = r * RB + ((2 * s + hi) ^ x_kx<DH>(r)) * 16;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    const int g16 = lane >> 4, i16 = lane & 15;
    const int r = 8 * (g16 >> 1) + (i16 >> 2);
    v_rd[d] = VB + r * RB + ((2 * d + (g16 & 1)) ^ x_vx<DH>(r)) * 32 + 8 * (i16 & 3);
  }
  bf16x8 qf[NS];
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mc = X_LOW, l_run = 0.0f;
  const f32x16 zero16 = {};
  const xbf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};

  // The states pass in halves of 32: while the matrix cores compute the scores
  // of one half, the vector units turn those of the half before it into
  // probabilities, which then weigh V.  LDS reads are issued
  // X_RING MFMAs ahead.  The probabilities enter the second product in bf16, the
  // type its instruction takes: an output is then within 0.0022 to 0.0024 of the
  // 64-bit one in the 2-norm, 0.0017 of it the output's own rounding.  Kept to
  // more bits, as a second bf16 number each, they would take that product twice.
  bf16x8 pf[2];
  float psum;
  auto weigh = [&](const f32x16& sc, int c) __attribute__((always_inline)) {  // scores 2 c, 2 c + 1
    const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[2 * c], p.scale_log2, -mc));
    const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[2 * c + 1], p.scale_log2, -mc));
    const int j = 2 * (c % 4);
    pf[c / 4][j] = static_cast<__bf16>(e0);
    pf[c / 4][j + 1] = static_cast<__bf16>(e1);
    // the sum is of the rounded probabilities, those that weigh V
    const xbf16x2 pair = {pf[c / 4][j], pf[c / 4][j + 1]};
    psum = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, psum, false);
  };
  // scores of half h of the u-th tile, with work(c), c < 8, spread between its MFMAs
  auto scores = [&](int u, int h, f32x16& sc, auto&& work) __attribute__((always_inline)) {
    const char* ks = smem + (u & 1) * TILE + h * 32 * RB;
    auto read = [&](int s) __attribute__((always_inline)) {
      return *reinterpret_cast<const bf16x8*>(ks + k_rd[s]);
    };
    bf16x8 ring[X_RING];
#pragma unroll
    for (int i = 0; i < X_RING; ++i) ring[i] = read(i);
#pragma unroll
    for (int s = 0; s < NS; ++s) {
      sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[s % X_RING], qf[s], s == 0 ? zero16 : sc, 0, 0, 0);
      if (s + X_RING < NS) ring[s % X_RING] = read(s + X_RING);
#pragma unroll
      for (int c = s * 8 / NS; c < (s + 1) * 8 / NS; ++c) work(c);
      __builtin_amdgcn_sched_barrier(0);
    }
    const int left = x.n - (x.t0 + u) * X_KT - 32 * h;  // states of the half and after it
    if (left < 32) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 16 * (r >> 3) + 8 * hi + (r & 7) < left ? sc[r] : -INFINITY;
    }
  };
  // The half's probabilities are against the maximum so far.  None can exceed
  // 2^8 unless the lane's sum does, so the half's own maximum is looked for only
  // then (always in the first), and every row that has grown takes it.  A row
  // that has brought the wave here then has weights of at most 1 and does not do
  // so again before one of them is above 16 (a maximum left where it was until a
  // growth of 2^8, and exceeded by 2^5 to 2^7 ever after, had every half computed
  // twice: 3900 queries x 4096 states x 16 heads, dh 64, 127 us, now 77).  Rows
  // that have not grown get the same probabilities again.
  auto settle = [&](const f32x16& sc) __attribute__((always_inline)) {
    if (__builtin_expect(__ballot(psum > X_GROW_SUM) != 0ull, 0)) {
      float mx = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[r]);
      mx = pair_max(mx) * p.scale_log2;
      const bool grow = mx > mc;
      const float alpha = grow ? __builtin_amdgcn_exp2f(mc - mx) : 1.0f;
      mc = grow ? mx : mc;
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      psum = 0.0f;
#pragma unroll
      for (int c = 0; c < 8; ++c) weigh(sc, c);
    }
    l_run += psum;
  };
  auto values = [&](int u, int h) __attribute__((always_inline)) {  // O += V^T P^T of a half
    const char* vs = smem + u % 3 * TILE + h * 32 * RB;
    auto read = [&](int i) __attribute__((always_inline)) {
      const char* at = vs + i / ND * 16 * RB + v_rd[i % ND];
      const xv4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) xv4i16*)(at));
      const xv4i16 up =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) xv4i16*)(at + 4 * RB));
      return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    bf16x8 ring[X_RING];
#pragma unroll
    for (int i = 0; i < X_RING; ++i) ring[i] = read(i);
#pragma unroll
    for (int i = 0; i < 2 * ND; ++i) {
      o[i % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % X_RING], pf[i / ND], o[i % ND], 0, 0, 0);
      if (i + X_RING < 2 * ND) ring[i % X_RING] = read(i + X_RING);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  // Tile u has landed for every wave and every wave is done with the scores of
  // tile u - 1 and the values of tile u - 2, whose stages the next copies refill.
  auto arrive = [&](int u) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    if (u == 0) {
#pragma unroll
      for (int s = 0; s < NS; ++s)
        qf[s] = *reinterpret_cast<const bf16x8*>(qs + l32 * RB + ((2 * s + hi) ^ x_kx<DH>(l32)) * 16);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));  // read, before another wave's copies replace them
    }
    __syncthreads();
    if (u + 1 < nt) issue(u + 1);
    const int left = x.n - (x.t0 + u) * X_KT;
    if (left < X_KT) {
      // V rows past the last state: zeros, so that their zero weights meet no infinity
      for (int e = tid; e < (X_KT - left) * (RB / 16); e += 256)
        *reinterpret_cast<uint4*>(smem + VB + u % 3 * TILE + left * RB + e * 16) = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
    }
  };
  if (idle) {
    for (int u = 0; u < nt; ++u) arrive(u);
  } else if (nt > 0) {
    f32x16 s0, s1;
    arrive(0);
    scores(0, 0, s0, [](int) {});
    for (int u = 0; u < nt; ++u) {
      // The two workgroups of a CU start together and would load and compute
      // together; the one past its middle goes first, so that they come apart and
      // one's loads and stores run under the other's products (13104 x 2 queries:
      // 240 -> 232 us; 3276 queries x 32760 states: 2314 -> 2202)
      if (2 * u >= nt) __builtin_amdgcn_s_setprio(2);
      psum = 0.0f;
      scores(u, 1, s1, [&](int c) __attribute__((always_inline)) { weigh(s0, c); });
      settle(s0);
      values(u, 0);
      psum = 0.0f;
      if (u + 1 < nt) {
        arrive(u + 1);
        scores(u + 1, 0, s0, [&](int c) __attribute__((always_inline)) { weigh(s1, c); });
      } else {
#pragma unroll
        for (int c = 0; c < 8; ++c) weigh(s1, c);
      }
      settle(s1);
      values(u, 1);
    }
  }
  const float lsum = pair_sum(l_run);
  if (p.nsplit > 1) {
    if (idle) return;
    if (row0 + l32 >= rows) return;
    const int64_t units = x_units(p, tiles), u = x_unit(p, x, tiles, wave * 32 + l32);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(p.part + u * DH + d * 32 + 8 * c + 4 * hi) =
            make_float4(o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]);
    if (hi == 0) *reinterpret_cast<float2*>(p.part + units * DH + 2 * u) = make_float2(mc, lsum);
    return;
  }
  // rows through LDS, so that stores are 16-byte pieces of whole rows
  __syncthreads();  // every wave is done with the last tile
  bf16_t* os = reinterpret_cast<bf16_t*>(smem);
  const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const uint2 w = make_uint2(pack_bf16x2(o[d][4 * c] * inv, o[d][4 * c + 1] * inv),
                                 pack_bf16x2(o[d][4 * c + 2] * inv, o[d][4 * c + 3] * inv));
      *reinterpret_cast<uint2*>(os + (wave * 32 + l32) * OS + d * 32 + 8 * c + 4 * hi) = w;
    }
  __syncthreads();
  bf16_t* ob = static_cast<bf16_t*>(p.out) + x.b * p.ob;
  for (int e = tid; e < X_ROWS * (DH / 8); e += 256) {
    const int rl = e / (DH / 8), ch = e % (DH / 8), r = x.tile * X_ROWS + rl;
    if (r >= rows) break;
    int g, i;
    x_row(p, r, g, i);
    stg16(ob + static_cast<int64_t>(i) * p.orow + static_cast<int64_t>(x.hk * (p.H / p.Hkv) + g) * p.oh + ch * 8,
          *reinterpret_cast<const uint4*>(os + rl * OS + ch * 8));
  }
}

// ------------------------------------------------------------------- fp32
// DHP: dh rounded up to 32, 64 or 128; columns past dh are zeros.
template <int DHP>
__global__ void __launch_bounds__(256) cross_f32(CrossArgs p) {
  constexpr int ND = DHP / 32, NS = DHP / 2, LD = DHP + 1;
  __shared__ float ks[X_KT32 * LD], vs[X_KT32 * DHP];
  const int tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave, l32 = lane & 31, hi = lane >> 5;
  const int rows = p.H / p.Hkv * p.Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
  const XItem x = x_item(p, tiles, X_KT32);
  const float* kb = static_cast<const float*>(p.k) + x.b * p.kb + x.hk * p.kh;
  const float* vb = static_cast<const float*>(p.v) + x.b * p.vb + x.hk * p.vh;
  const int32_t* list = p.key_mask != nullptr ? p.key_list + static_cast<int64_t>(x.b) * p.Lk : nullptr;
  const int row0 = x.tile * X_ROWS + wave * 32;
  const bool idle = row0 >= rows;
  int r = row0 + l32;
  const bool mine = r < rows;
  r = mine ? r : rows - 1;
  const int g = r / p.Lq, i = r % p.Lq;
  const int64_t head = x.hk * (p.H / p.Hkv) + g;
  float qf[NS];  // the lane's half of its query: elements 2 s + hi
  {
    const float* src = static_cast<const float*>(p.q) + x.b * p.qb + static_cast<int64_t>(i) * p.qr + head * p.qh;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = 2 * s + hi < p.dh ? src[2 * s + hi] : 0.0f;
  }
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.0f;
  float mc = X_LOW, l_run = 0.0f;
  // the next tile is on its way to registers while this one is worked on
  constexpr int NV = X_KT32 * (DHP / 4) / 256 > 0 ? X_KT32 * (DHP / 4) / 256 : 1;
  static_assert(X_KT32 * (DHP / 4) == NV * 256, "whole passes of the workgroup");
  float4 kv[NV], vv[NV];
  auto fetch = [&](int t) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int e = tid + 256 * u, kr = e / (DHP / 4), c = e % (DHP / 4) * 4;
      kv[u] = vv[u] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);  // no state, no column: zeros
      if (t * X_KT32 + kr < x.n && c < p.dh) {
        int key = t * X_KT32 + kr;
        if (list != nullptr) key = list[key];
        kv[u] = *reinterpret_cast<const float4*>(kb + static_cast<int64_t>(key) * p.kr + c);
        vv[u] = *reinterpret_cast<const float4*>(vb + static_cast<int64_t>(key) * p.vr + c);
      }
    }
  };
  if (x.t0 < x.t1) fetch(x.t0);
  for (int t = x.t0; t < x.t1; ++t) {
    const int left = x.n - t * X_KT32;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int e = tid + 256 * u, kr = e / (DHP / 4), c = e % (DHP / 4) * 4;
      ks[kr * LD + c] = kv[u].x;
      ks[kr * LD + c + 1] = kv[u].y;
      ks[kr * LD + c + 2] = kv[u].z;
      ks[kr * LD + c + 3] = kv[u].w;
      *reinterpret_cast<float4*>(vs + kr * DHP + c) = vv[u];
    }
    __syncthreads();
    if (t + 1 < x.t1) fetch(t + 1);
    if (!idle) {
      // lane: scores of its query with states 8 (e / 4) + 4 hi + e % 4
      f32x16 sc = {};
#pragma unroll
      for (int s = 0; s < NS; ++s)
        sc = __builtin_amdgcn_mfma_f32_32x32x2f32(ks[l32 * LD + 2 * s + hi], qf[s], sc, 0, 0, 0);
      float mx = -INFINITY;
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        if (8 * (e / 4) + 4 * hi + e % 4 >= left) sc[e] = -INFINITY;
        mx = fmaxf(mx, sc[e]);
      }
      mx = pair_max(mx) * p.scale_log2;
      const bool grow = mx - mc > X_GROW;
      if (__ballot(grow) != 0ull) {
        const float alpha = grow ? __builtin_amdgcn_exp2f(mc - mx) : 1.0f;
        mc = grow ? mx : mc;
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[d][e] *= alpha;
      }
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        sc[e] = __builtin_amdgcn_exp2f(fmaf(sc[e], p.scale_log2, -mc));
        l_run += sc[e];
      }
      // step e takes the states that register e holds: 8 (e / 4) + e % 4, and 4 more for the upper lanes
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(vs[(8 * (e / 4) + 4 * hi + e % 4) * DHP + d * 32 + l32], sc[e],
                                                      o[d], 0, 0, 0);
    }
    __syncthreads();
  }
  const float lsum = pair_sum(l_run);
  if (p.nsplit > 1) {
    if (!mine) return;
    const int64_t units = x_units(p, tiles), u = x_unit(p, x, tiles, wave * 32 + l32);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<float4*>(p.part + u * DHP + d * 32 + 8 * c + 4 * hi) =
            make_float4(o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]);
    if (hi == 0) *reinterpret_cast<float2*>(p.part + units * DHP + 2 * u) = make_float2(mc, lsum);
    return;
  }
  if (!mine) return;
  const float inv = lsum == 0.0f ? 0.0f : 1.0f / lsum;
  float* dst = static_cast<float*>(p.out) + x.b * p.ob + static_cast<int64_t>(i) * p.orow + head * p.oh;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const int at = d * 32 + 8 * c + 4 * hi;
      if (at < p.dh)
        *reinterpret_cast<float4*>(dst + at) = make_float4(o[d][4 * c] * inv, o[d][4 * c + 1] * inv,
                                                           o[d][4 * c + 2] * inv, o[d][4 * c + 3] * inv);
    }
}

// ---- o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s, m = max_s m_s, ranges in
// order; a thread takes four outputs of a row
template <typename T, int DHP>
__global__ void __launch_bounds__(256) cross_combine(CrossArgs p) {
  const int rows = p.H / p.Hkv * p.Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
  const int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
  const int c = static_cast<int>(e % (DHP / 4)) * 4;
  const int64_t rg = e / (DHP / 4);
  const int r = static_cast<int>(rg % rows), bh = static_cast<int>(rg / rows);
  if (bh >= p.B * p.Hkv || c >= p.dh) return;
  const int b = bh / p.Hkv, hk = bh % p.Hkv;
  const int64_t units = x_units(p, tiles), step = static_cast<int64_t>(tiles) * X_ROWS;
  const int64_t u0 = static_cast<int64_t>(bh) * p.nsplit * step + r;
  const float* ml = p.part + units * DHP;
  float m = X_LOW;
  for (int s = 0; s < p.nsplit; ++s) m = fmaxf(m, ml[2 * (u0 + s * step)]);
  float l = 0.0f, a[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int s = 0; s < p.nsplit; ++s) {
    const int64_t u = u0 + s * step;
    const float2 z = *reinterpret_cast<const float2*>(ml + 2 * u);
    if (z.y == 0.0f) continue;  // a range without states or weight
    const float w = __builtin_amdgcn_exp2f(z.x - m);
    const float4 v = *reinterpret_cast<const float4*>(p.part + u * DHP + c);
    l = fmaf(w, z.y, l);
    a[0] = fmaf(w, v.x, a[0]);
    a[1] = fmaf(w, v.y, a[1]);
    a[2] = fmaf(w, v.z, a[2]);
    a[3] = fmaf(w, v.w, a[3]);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int g = r / p.Lq, i = r % p.Lq;
  T* dst = static_cast<T*>(p.out) + b * p.ob + static_cast<int64_t>(i) * p.orow +
           static_cast<int64_t>(hk * (p.H / p.Hkv) + g) * p.oh + c;
#pragma unroll
  for (int j = 0; j < 4; ++j) a[j] *= inv;
  if constexpr (std::is_same<T, float>::value)
    *reinterpret_cast<float4*>(dst) = make_float4(a[0], a[1], a[2], a[3]);
  else
    *reinterpret_cast<uint2*>(dst) = make_uint2(pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3]));
}

namespace {

constexpr size_t kXAlign = 256;
// workgroups that compact masks: with 1024 threads each, far below the 2^32
// threads of a launch, which one for each of up to 2^24 elements would pass
constexpr int kXListGroups = 1 << 16;
size_t x_up(size_t n) { return (n + kXAlign - 1) / kXAlign * kXAlign; }
int x_pad(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : 128; }

// Ranges of the states, by estimated time (us).  A workgroup's tile of states
// takes `one` alone on its CU and `all` with the CU full (in between by their
// number), and no less than its K and V take from memory where no other
// workgroup shares them; a round has 4 or 6 us beside its tiles for queries and
// outputs; a split adds the second launch and its partial results, written and
// read.  With several elements, which have several lengths, rounds before the
// last count for three quarters.  Measured (us): 40 groups of one query x 32760
// states 623 whole, 134 in 12 ranges; 1040 workgroups x 512 tiles 2638 and 2286
// (5); 488 x 94 tiles 190 and 211 (2), at dh 64 121 and 126 (3); 384 x 8 tiles 24
// and 44 (2).
int x_splits(int bf16, int B, int Lq, int Lk, int H, int Hkv, int dh) {
  const int64_t rows = static_cast<int64_t>(H / Hkv) * Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
  const int64_t wgs = tiles * B * Hkv;
  const int kt = bf16 ? X_KT : X_KT32, nt = (Lk + kt - 1) / kt, dhp = x_pad(dh), ncu = device_cu_count();
  const int per = bf16 ? (dhp == 64 ? 3 : 2) : (dhp == 128 ? 1 : dhp == 64 ? 2 : 3);  // workgroups of a CU
  float one = bf16 ? (dhp == 64 ? 0.86f : 1.2f) : 0.045f * dhp;
  float all = bf16 ? (dhp == 64 ? 1.8f : 1.9f) : 0.045f * dhp * (per > 1 ? 1.5f : 1.0f);
  if (tiles == 1) {
    const float mem = 2.0f * kt * dhp * (bf16 ? 2 : 4) * ncu / 6.2e6f;  // a tile on every CU
    one = one > mem ? one : mem;
    all = all > per * mem ? all : per * mem;
  }
  const int64_t slots = static_cast<int64_t>(ncu) * per;
  int best = 1;
  float best_us = 0.0f;
  for (const int ns : {1, 2, 3, 4, 5, 6, 8, 12, 16, 24, 32}) {
    if (ns > 1 && nt < 2 * ns) break;
    if (ns > 1 && wgs * ns * X_ROWS * (dhp + 2) * 4 > (int64_t(512) << 20)) break;  // partial results
    const int steps = (nt + ns - 1) / ns;
    const int64_t pieces = wgs * ns, full = pieces / slots, rest = pieces % slots;
    const float round = steps * all + 6.0f;
    const int n = static_cast<int>((rest + ncu - 1) / ncu);  // workgroups on the busiest CU of the last round
    float us = rest == 0 ? round : n == 1 ? steps * one + 4.0f : steps * (one + (all - one) * (n - 1) / (per - 1)) + 6.0f;
    us += (B > 1 ? 0.75f : 1.0f) * (rest == 0 ? full - 1 : full) * round;
    if (ns > 1) {
      us += 6.0f + static_cast<int64_t>(B) * Hkv * ns * rows * (dhp + 2) * 8.0f / 4e6f;
    }
    if (ns == 1 || us < best_us) {
      best = ns;
      best_us = us;
    }
  }
  return best;
}

template <int DH>
hipError_t launch_x_bf16(const CrossArgs& a, unsigned grid, hipStream_t stream) {
  return a.key_mask != nullptr
             ? ECHO_LAUNCH("cross_bf16", (cross_bf16<DH, true>), dim3(grid), dim3(256), 0, stream, a)
             : ECHO_LAUNCH("cross_bf16", (cross_bf16<DH, false>), dim3(grid), dim3(256), 0, stream, a);
}

template <typename T, int DHP>
hipError_t launch_x_combine(const CrossArgs& a, hipStream_t stream) {
  const int64_t n = static_cast<int64_t>(a.B) * a.H * a.Lq * (DHP / 4);
  return ECHO_LAUNCH("cross_combine", (cross_combine<T, DHP>), dim3(static_cast<unsigned>((n + 255) / 256)), dim3(256),
                     0, stream, a);
}

}  // namespace

size_t cross_workspace_bytes(int bf16, int B, int Lq, int Lk, int H, int Hkv, int dh, bool masked) {
  size_t n = 0;
  if (masked) n = x_up(sizeof(int32_t) * static_cast<size_t>(B) * Lk) + x_up(sizeof(int32_t) * B);
  const int ns = x_splits(bf16, B, Lq, Lk, H, Hkv, dh);
  if (ns > 1) {
    const size_t rows = static_cast<size_t>(H / Hkv) * Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
    n += x_up(sizeof(float) * (x_pad(dh) + 2) * static_cast<size_t>(B) * Hkv * ns * tiles * X_ROWS);
  }
  return n;
}

hipError_t launch_cross(int bf16, CrossArgs a, void* workspace, hipStream_t stream) {
  char* ws = static_cast<char*>(workspace);
  hipError_t e;
  if (a.key_mask != nullptr) {
    a.key_list = reinterpret_cast<int32_t*>(ws);
    ws += x_up(sizeof(int32_t) * static_cast<size_t>(a.B) * a.Lk);
    a.key_count = reinterpret_cast<int32_t*>(ws);
    ws += x_up(sizeof(int32_t) * a.B);
    const int groups = a.B < kXListGroups ? a.B : kXListGroups;
    if ((e = ECHO_LAUNCH("cross_keys", cross_keys, dim3(groups), dim3(1024), 0, stream, a)) != hipSuccess) return e;
  }
  a.part = reinterpret_cast<float*>(ws);
  a.nsplit = x_splits(bf16, a.B, a.Lq, a.Lk, a.H, a.Hkv, a.dh);
  const int64_t rows = static_cast<int64_t>(a.H / a.Hkv) * a.Lq;
  const unsigned grid =
      static_cast<unsigned>((rows + X_ROWS - 1) / X_ROWS * a.B * a.Hkv * a.nsplit);
  const int dhp = x_pad(a.dh);
  if (bf16)
    e = dhp == 64 ? launch_x_bf16<64>(a, grid, stream) : launch_x_bf16<128>(a, grid, stream);
  else if (dhp == 32)
    e = ECHO_LAUNCH("cross_f32", cross_f32<32>, dim3(grid), dim3(256), 0, stream, a);
  else if (dhp == 64)
    e = ECHO_LAUNCH("cross_f32", cross_f32<64>, dim3(grid), dim3(256), 0, stream, a);
  else
    e = ECHO_LAUNCH("cross_f32", cross_f32<128>, dim3(grid), dim3(256), 0, stream, a);
  if (e != hipSuccess || a.nsplit == 1) return e;
  if (bf16) return dhp == 64 ? launch_x_combine<bf16_t, 64>(a, stream) : launch_x_combine<bf16_t, 128>(a, stream);
  if (dhp == 32) return launch_x_combine<float, 32>(a, stream);
  return dhp == 64 ? launch_x_combine<float, 64>(a, stream) : launch_x_combine<float, 128>(a, stream);
}

}  // namespace echo
