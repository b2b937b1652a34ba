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
// Softmax: running maximum and sum in fp32, in units of log2; the maximum moves
// only when a tile's exceeds it by more than 2^8, so that probabilities stay
// below 2^8 and a rescale is rare.
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
constexpr float X_GROW = 8.0f;              // log2 of the growth that moves the maximum
constexpr float X_LOW = -3.402823466e38f;   // the maximum before any state: the lowest finite value

// maximum and sum over lanes l and l ^ 32
__device__ __forceinline__ float x_pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float x_pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

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
__device__ __forceinline__ XItem x_item(const CrossArgs& p, int tiles, int kt) {
  const int nb = gridDim.x, per = nb / 8, rem = nb % 8, xcd = blockIdx.x % 8;
  int i = xcd * per + (xcd < rem ? xcd : rem) + blockIdx.x / 8;
  XItem x;
  x.tile = i % tiles;
  i /= tiles;
  x.split = i % p.nsplit;
  i /= p.nsplit;
  x.hk = i % p.Hkv;
  x.b = i / p.Hkv;
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

// ---- partial results of a range: for the row's unit u, DH outputs, then all
// units' maxima and sums
__device__ __forceinline__ int64_t x_unit(const CrossArgs& p, const XItem& x, int tiles, int row) {
  return ((static_cast<int64_t>(x.b * p.Hkv + x.hk) * p.nsplit + x.split) * tiles + x.tile) * X_ROWS + row;
}
__device__ __forceinline__ int64_t x_units(const CrossArgs& p, int tiles) {
  return static_cast<int64_t>(p.B) * p.Hkv * p.nsplit * tiles * X_ROWS;
}

// ---- states that the mask leaves, in order; one workgroup per element
__global__ void __launch_bounds__(1024) cross_keys(CrossArgs p) {
  __shared__ int wave_n[16];
  const int b = blockIdx.x, tid = threadIdx.x, wave = tid / kWave, lane = tid % kWave;
  int n = p.k_len != nullptr ? p.k_len[b] : p.Lk;
  n = n < 0 ? 0 : (n < p.Lk ? n : p.Lk);
  const uint8_t* mask = p.key_mask + static_cast<int64_t>(b) * p.Lk;
  int32_t* list = p.key_list + static_cast<int64_t>(b) * p.Lk;
  int base = 0;
  for (int j0 = 0; j0 < n; j0 += 1024) {
    const int j = j0 + tid;
    const bool in = j < n && mask[j] != 0;
    const uint64_t bits = __ballot(in);
    if (lane == 0) wave_n[wave] = __popcll(bits);
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
      before += w < wave ? wave_n[w] : 0;
      total += wave_n[w];
    }
    if (in) list[base + before + __popcll(bits & ((1ull << lane) - 1ull))] = j;
    base += total;
    __syncthreads();
  }
  if (tid == 0) p.key_count[b] = base;
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
  constexpr int LDS = 4 * TILE > X_ROWS * OS * 2 ? 4 * TILE : X_ROWS * OS * 2;
  __shared__ __attribute__((aligned(1024))) char smem[LDS];  // stage s: K at 2 s TILE, V behind it
  const int tid = threadIdx.x, lane = tid % kWave, l32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int rows = p.H / p.Hkv * p.Lq, tiles = (rows + X_ROWS - 1) / X_ROWS;
  const XItem x = x_item(p, tiles, X_KT);
  const bf16_t* kb = static_cast<const bf16_t*>(p.k) + x.b * p.kb + x.hk * p.kh;
  const bf16_t* vb = static_cast<const bf16_t*>(p.v) + x.b * p.vb + x.hk * p.vh;
  const int32_t* list = MASK ? p.key_list + static_cast<int64_t>(x.b) * p.Lk : nullptr;

  // ---- this lane's query: row r = g Lq + i
  const int row0 = x.tile * X_ROWS + wave * 32;
  const bool idle = row0 >= rows;  // no row in this wave: it copies and waits with the others
  bf16x8 qf[NS];
  {
    int r = row0 + l32;
    r = r < rows ? r : rows - 1;
    const int g = r / p.Lq, i = r % p.Lq;
    const bf16_t* src = static_cast<const bf16_t*>(p.q) + x.b * p.qb + static_cast<int64_t>(i) * p.qr +
                        static_cast<int64_t>(x.hk * (p.H / p.Hkv) + g) * p.qh + 8 * hi;
#pragma unroll
    for (int s = 0; s < NS; ++s) qf[s] = __builtin_bit_cast(bf16x8, ldg16(src + 16 * s));
  }
  // the loads above are waited for here: later waits count the copies alone
  __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));

  // ---- copies.  Copy m of this wave is rows RPP (wave + 4 m) .. of the tile;
  // the lane lands in row lr of them, slot ls, and fetches the chunk that lives there.
  const int lr = lane / (RB / 16), ls = lane % (RB / 16);
  const uint32_t lds0 = lds_offset(smem);
  auto issue = [&](int t, int stage) __attribute__((always_inline)) {
    const int key0 = t * X_KT;
#pragma unroll
    for (int m = 0; m < NP; ++m) {
      const int r = RPP * (wave + 4 * m) + lr;
      int key = key0 + r < x.n ? key0 + r : x.n - 1;  // past the end: the last state again, never used
      if constexpr (MASK) key = list[key];
      const int kc = (ls ^ x_kx<DH>(r)) * 8, vc = ((((ls >> 1) ^ x_vx<DH>(r)) << 1) + (ls & 1)) * 8;
      const uint32_t dst = lds0 + 2 * stage * TILE + (wave + 4 * m) * 1024;
      lds_copy16(kb + static_cast<int64_t>(key) * p.kr + kc, dst);
      lds_copy16(vb + static_cast<int64_t>(key) * p.vr + vc, dst + TILE);
    }
  };
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
    v_rd[d] = TILE + r * RB + ((2 * d + (g16 & 1)) ^ x_vx<DH>(r)) * 32 + 8 * (i16 & 3);
  }
  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
  float mc = X_LOW, l_run = 0.0f;
  const f32x16 zero16 = {};
  const xbf16x2 ones = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};

  if (x.t0 < x.t1) issue(x.t0, 0);
  for (int t = x.t0; t < x.t1; ++t) {
    const int stage = (t - x.t0) & 1;
    if (t + 1 < x.t1) {
      issue(t + 1, stage ^ 1);
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(2 * NP));  // this wave's copies of tile t
    } else {
      __builtin_amdgcn_s_waitcnt(waitcnt_vm(0));
    }
    __syncthreads();
    char* st = smem + 2 * stage * TILE;
    const int left = x.n - t * X_KT;  // states of the tile and after it
    if (left < X_KT) {
      // V rows past the last state: zeros, so that their zero weights meet no infinity
      for (int e = tid; e < (X_KT - left) * (RB / 16); e += 256)
        *reinterpret_cast<uint4*>(st + TILE + left * RB + e * 16) = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
    }
    if (!idle) {
      f32x16 sc[2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int s = 0; s < NS; ++s) {
          const bf16x8 a = *reinterpret_cast<const bf16x8*>(st + h * 32 * RB + k_rd[s]);
          sc[h] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[s], s == 0 ? zero16 : sc[h], 0, 0, 0);
        }
      if (left < X_KT) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            sc[h][r] = 32 * h + 16 * (r >> 3) + 8 * hi + (r & 7) < left ? sc[h][r] : -INFINITY;
      }
      float mx = sc[0][0];
#pragma unroll
      for (int r = 1; r < 32; ++r) mx = fmaxf(mx, sc[r / 16][r % 16]);
      mx = x_pair_max(mx) * p.scale_log2;
      const bool grow = mx - mc > X_GROW;
      if (__ballot(grow) != 0ull) {
        const float alpha = grow ? __builtin_amdgcn_exp2f(mc - mx) : 1.0f;
        mc = grow ? mx : mc;
        l_run *= alpha;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) o[d][r] *= alpha;
      }
      bf16x8 pf[2][2];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(sc[h][2 * c], p.scale_log2, -mc));
          const float e1 = __builtin_amdgcn_exp2f(fmaf(sc[h][2 * c + 1], p.scale_log2, -mc));
          const int j = 2 * (c % 4);
          pf[h][c / 4][j] = static_cast<__bf16>(e0);
          pf[h][c / 4][j + 1] = static_cast<__bf16>(e1);
          // the sum is of the rounded probabilities, those that weigh V
          const xbf16x2 pair = {pf[h][c / 4][j], pf[h][c / 4][j + 1]};
          l_run = __builtin_amdgcn_fdot2_f32_bf16(pair, ones, l_run, false);
        }
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const char* vs = st + (32 * h + 16 * a) * RB + v_rd[d];
            const xv4i16 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) xv4i16*)(vs));
            const xv4i16 up = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (__attribute__((address_space(3))) xv4i16*)(vs + 4 * RB));
            const bf16x8 va = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, up, 0, 1, 2, 3, 4, 5, 6, 7));
            o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, pf[h][a], o[d], 0, 0, 0);
          }
    }
    __syncthreads();  // every wave is done with the stage that the next tile's copies refill
  }
  const float lsum = x_pair_sum(l_run);
  if (p.nsplit > 1) {
    if (idle) return;
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
    const int g = r / p.Lq, i = r % p.Lq;
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
  for (int t = x.t0; t < x.t1; ++t) {
    const int left = x.n - t * X_KT32;
    for (int e = tid; e < X_KT32 * (DHP / 4); e += 256) {
      const int kr = e / (DHP / 4), c = e % (DHP / 4) * 4;
      float4 kv = make_float4(0.0f, 0.0f, 0.0f, 0.0f), vv = kv;
      if (kr < left && c < p.dh) {
        int key = t * X_KT32 + kr;
        if (list != nullptr) key = list[key];
        kv = *reinterpret_cast<const float4*>(kb + static_cast<int64_t>(key) * p.kr + c);
        vv = *reinterpret_cast<const float4*>(vb + static_cast<int64_t>(key) * p.vr + c);
      }
      ks[kr * LD + c] = kv.x;
      ks[kr * LD + c + 1] = kv.y;
      ks[kr * LD + c + 2] = kv.z;
      ks[kr * LD + c + 3] = kv.w;
      *reinterpret_cast<float4*>(vs + kr * DHP + c) = vv;
    }
    __syncthreads();
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
      mx = x_pair_max(mx) * p.scale_log2;
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
  const float lsum = x_pair_sum(l_run);
  if (p.nsplit > 1) {
    if (idle) return;
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
size_t x_up(size_t n) { return (n + kXAlign - 1) / kXAlign * kXAlign; }
int x_pad(int dh) { return dh <= 32 ? 32 : dh <= 64 ? 64 : 128; }

// ranges of the states: enough workgroups for two to each CU, each with four
// tiles of states at least (of the longest element)
int x_splits(int bf16, int B, int Lq, int Lk, int H, int Hkv) {
  const int64_t rows = static_cast<int64_t>(H / Hkv) * Lq;
  const int64_t wgs = (rows + X_ROWS - 1) / X_ROWS * B * Hkv;
  const int kt = bf16 ? X_KT : X_KT32, nt = (Lk + kt - 1) / kt;
  const int64_t want = (2ll * device_cu_count() + wgs - 1) / wgs;
  const int64_t most = nt / 4;
  const int64_t n = want < most ? want : most;
  return n < 1 ? 1 : static_cast<int>(n);
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
  const int ns = x_splits(bf16, B, Lq, Lk, H, Hkv);
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
    if ((e = ECHO_LAUNCH("cross_keys", cross_keys, dim3(a.B), dim3(1024), 0, stream, a)) != hipSuccess) return e;
  }
  a.part = reinterpret_cast<float*>(ws);
  a.nsplit = x_splits(bf16, a.B, a.Lq, a.Lk, a.H, a.Hkv);
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
