// Rows held in 4 bits: microscaled floating point, every 32 values of a row with a
// power of two of their own, for the products of gemm_fp4.hip.
//
//   e_b = max(floor(log2 max_{j in b} |a_ij|) - 2, -127),   c_ij = rn(a_ij / 2^e_b)
//   a_ij = x[rows(i)]_j                 or LN(x[rows(i)])_j (1 + scale_j) + shift_j
//
// c of one sign, two exponent and one fraction bit (0, 0.5, 1, 1.5, 2, 3, 4, 6),
// halves to the even code, magnitudes above 6 to 6; the scale is the byte e_b +
// 127, 255 (NaN) for a block that is not finite.  The quotient is exact, so the
// code is the value rounded once, by v_cvt_scalef32_pk_fp4_f32.  The instruction
// takes its scale as an fp32 number, of which 2^-127 is a denormal one: such
// blocks are multiplied by 2^64 first.
//
// A lane takes 8 values, four lanes a block, whose maximum is two DPP moves, and 16
// lanes a set of 128 values: 64 bytes of codes and one word of scales.  Without
// LayerNorm the sets of all rows are one list, which the lanes go through with four
// of them in flight: bound by memory.  With it a row is a group of lanes that fits it
// (gated_norm.hip), which holds the modulation for its rows.  A row's last set
// writes the zeros up to the row's pitches.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

// The 4-bit codes of a lane's 8 values, packed, and the scales of the four blocks of
// its set of 16 lanes as one word.  bad: the row is not there.  live: the lane's block has
// columns; one behind the last column is zeros also where the row is NaN.
__device__ __forceinline__ uint32_t codes8_fp4(const float* v, bool bad, bool live, uint32_t& scales) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(v[j]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0xb1, 0xf, 0xf, false)));
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(top), 0x4e, 0xf, 0xf, false)));
  bad = bad || top >= 0x7f800000u;
  const uint32_t e = top >> 23, byte = e > 2 ? e - 2 : 0;
  uint32_t w = 0;
  if (byte > 0) {
    const float s = __uint_as_float(byte << 23);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], s, 3);
  } else {
    constexpr float k = 0x1p64f, s = 0x1p-63f;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0] * k, v[1] * k, s, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2] * k, v[3] * k, s, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4] * k, v[5] * k, s, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6] * k, v[7] * k, s, 3);
  }
  scales = (!live ? 0u : bad ? 255u : byte) << (threadIdx.x / 4 % 4 * 8);
  scales |= dpp_ror<4>(scales);
  scales |= dpp_ror<8>(scales);
  return bad || !live ? 0u : w;
}

// Set `set` of a row: lane i of its 16 has the codes w and the scales' word.
__device__ __forceinline__ void put_set(const QuantizeArgs& p, int64_t row, int set, uint32_t w, uint32_t scales) {
  const int i = threadIdx.x % 16, sets = (p.D + 127) / 128;
  int8_t* codes = p.codes + row * p.ldq + set * 64;
  uint8_t* sc = p.scales + row * p.lds + set * 4;
  *reinterpret_cast<uint32_t*>(codes + 4 * i) = w;
  if (i == 0) *reinterpret_cast<uint32_t*>(sc) = scales;
  if (set == sets - 1) {  // zeros up to whole 128 bytes of codes and whole 16 of scales
    if (sets % 2 == 1) *reinterpret_cast<uint32_t*>(codes + 64 + 4 * i) = 0;
    if (i > 0 && i <= 3 - (sets - 1) % 4) *reinterpret_cast<uint32_t*>(sc + 4 * i) = 0;
  }
}

// whether the lane's block of a set has columns
__device__ __forceinline__ bool live_block(const QuantizeArgs& p, int set) {
  return set * 128 + static_cast<int>(threadIdx.x / 4 % 4) * 32 < p.D;
}

__device__ __forceinline__ int64_t row_of(const QuantizeArgs& p, int64_t row, bool& bad) {
  bad = false;
  if (p.rows == nullptr) return row;
  const int32_t r = p.rows[row];
  bad = r < 0 || r >= p.x_rows;  // no such row: as a row that is not finite
  return bad ? 0 : r;
}

// The sets of all rows: those g, g + G, ... of the list for group g of G groups of 16
// lanes (step_row and step_set: G in rows and sets of one).
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) quantize_fp4_k(QuantizeArgs p, int64_t step_row, int step_set) {
  constexpr int U = 4;
  const int sets = (p.D + 127) / 128, lane = threadIdx.x % 16;
  const int64_t g = static_cast<int64_t>(blockIdx.x) * 16 + threadIdx.x / 16;
  int64_t row = g / sets;
  int set = static_cast<int>(g % sets);
  while (row < p.M) {
    int64_t rows[U];
    int at[U];
    bool bad[U];
    Raw8<T> raw[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      rows[u] = row;
      at[u] = set;
      const int c = set * 128 + lane * 8;
      const T* x = static_cast<const T*>(p.x);
      bad[u] = false;
      if (row < p.M) x += row_of(p, row, bad[u]) * p.ldx;
      // (blocks behind the last column hold zeros here, so a row that is not there is all that makes them NaN)
      if (p.rows != nullptr) bad[u] = bad[u] && live_block(p, set);
      load_chunk<VEC, true>(raw[u], x, c, p.D);
      row += step_row;
      set += step_set;
      if (set >= sets) set -= sets, ++row;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (rows[u] >= p.M) break;
      float f[8];
      unpack_chunk<VEC>(raw[u], at[u] * 128 + lane * 8, p.D, f);
      uint32_t scales;
      const uint32_t w = codes8_fp4(f, bad[u], true, scales);
      put_set(p, rows[u], at[u], w, scales);
    }
  }
}

// With LayerNorm: a row to `threads` threads (16 if NARROW, one wave or the whole
// workgroup), NV chunks of 8 values each; a workgroup takes consecutive rows, the next
// row's values on their way and the modulation in registers (HOLD: where they leave room
// for a second workgroup on the CU; of wider rows both are read when they are due).
template <typename T, int MAXT, int NV, bool VEC, bool NARROW>
__global__ void __launch_bounds__(MAXT) quantize_fp4_ln_k(QuantizeArgs p, int threads, int rows_per_wg) {
  constexpr bool HOLD = MAXT <= 256 || NV <= 2, AHEAD = HOLD;
  __shared__ float red[2][2][MAXT / kWave];
  const int t = threadIdx.x % threads, D = p.D, rpb = blockDim.x / threads, waves = threads / kWave;
  int turn = 0;
  // as in gated_norm.hip: a piece of LDS for each reduction, two sets in turn
  auto total = [&](float v, int slot) __attribute__((always_inline)) {
    if constexpr (NARROW) return sum16(v);
    v = wave_sum(v);
    if (waves > 1) {
      if (t % kWave == 0) red[turn][slot][t / kWave] = v;
      __syncthreads();
      const int w = t & 15;
      v = sum16(w < waves ? red[turn][slot][w] : 0.0f);
    }
    return v;
  };
  // 1 + scale and shift of chunk u; 0 and 0 past the last column, so that the values
  // there come out as zeros
  auto modulation = [&](int u, float* sc, float* sh) __attribute__((always_inline)) {
    const int c = (t + u * threads) * 8;
    Raw8<float> rs, rh;
    load_chunk<VEC, false>(rs, p.scale, c, D);
    load_chunk<VEC, false>(rh, p.shift, c, D);
    unpack_chunk<VEC>(rs, c, D, sc);
    unpack_chunk<VEC>(rh, c, D, sh);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      sc[j] = (VEC ? c < D : c + j < D) ? 1.0f + sc[j] : 0.0f;
    }
  };
  float sc[HOLD ? NV : 1][8], sh[HOLD ? NV : 1][8];
  if constexpr (HOLD) {
#pragma unroll
    for (int u = 0; u < NV; ++u) modulation(u, sc[u], sh[u]);
  }
  Raw8<T> next[AHEAD ? NV : 1];
  bool next_bad = false;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    const T* x = static_cast<const T*>(p.x) + row_of(p, row, next_bad) * p.ldx;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      load_chunk<VEC, true>(next[AHEAD ? u : 0], x, (t + u * threads) * 8, D);
    }
  };
  const int64_t base = static_cast<int64_t>(blockIdx.x) * rows_per_wg;
  const int64_t end = base + rows_per_wg < p.M ? base + rows_per_wg : p.M;
  int64_t row = base + threadIdx.x / threads;
  if constexpr (AHEAD)
    if (row < end) fetch(row);
  // (a group that reaches a barrier is the whole workgroup, so the loop is uniform for its waves)
  for (; row < end; row += rpb) {
    bool bad = next_bad;
    float v[NV][8];
    const T* x = nullptr;
    if constexpr (!AHEAD) x = static_cast<const T*>(p.x) + row_of(p, row, bad) * p.ldx;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      if constexpr (AHEAD) {
        unpack_chunk<VEC>(next[u], (t + u * threads) * 8, D, v[u]);
      } else {
        Raw8<T> raw;
        load_chunk<VEC, true>(raw, x, (t + u * threads) * 8, D);
        unpack_chunk<VEC>(raw, (t + u * threads) * 8, D, v[u]);
      }
    }
    if constexpr (AHEAD)
      if (row + rpb < end) fetch(row + rpb);
    float sum = 0.0f, sq = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) sum += v[u][j];
    const float mean = total(sum, 0) / static_cast<float>(D);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * threads) * 8;
      const float m = c < D ? mean : 0.0f;  // (what lies past the last column stays zero)
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[u][j] -= VEC || c + j < D ? m : 0.0f;
        sq = fmaf(v[u][j], v[u][j], sq);
      }
    }
    const float rstd = 1.0f / sqrtf(total(sq, 1) / static_cast<float>(D) + p.ln_eps);
    turn ^= 1;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int set = (t + u * threads) / 16;
      if (set * 128 >= D) continue;  // (for 16 lanes together)
      float c8[8], h8[8];
      if constexpr (!HOLD) modulation(u, c8, h8);
#pragma unroll
      for (int j = 0; j < 8; ++j)
        v[u][j] = fmaf(v[u][j] * rstd, HOLD ? sc[HOLD ? u : 0][j] : c8[j], HOLD ? sh[HOLD ? u : 0][j] : h8[j]);
      uint32_t scales;
      const uint32_t w = codes8_fp4(v[u], bad, live_block(p, set), scales);
      put_set(p, row, set, w, scales);
    }
  }
}

// y_ij = cast(2^e_b c_ij), exact in both types; a thread takes 8 values
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) dequantize_fp4_k(DequantizeArgs p) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const int nch = (p.D + 7) / 8;
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < static_cast<int64_t>(p.M) * nch;
       e += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = e / nch;
    const int c = static_cast<int>(e % nch) * 8;
    const uint32_t w = *reinterpret_cast<const uint32_t*>(p.codes + row * p.ldq + c / 2);
    const uint32_t b = p.scales[row * p.lds + c / 32];
    // 2^-127 is a denormal number, 255 a NaN
    const float s = __uint_as_float(b == 255u ? 0x7fc00000u : b == 0u ? 0x00400000u : b << 23);
    const f32x2 u0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
    const f32x2 u1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
    const f32x2 u2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
    const f32x2 u3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
    const float v[8] = {s * u0[0], s * u0[1], s * u1[0], s * u1[1], s * u2[0], s * u2[1], s * u3[0], s * u3[1]};
    store_chunk<VEC, true>(static_cast<T*>(p.y) + row * p.ldy, c, p.D, v);
  }
}

namespace {

constexpr int64_t kMaxGroups = 1 << 20;  // workgroups of a launch; more rows than that loop

template <typename T, bool VEC>
hipError_t launch_plain(const QuantizeArgs& p, hipStream_t stream) {
  const int sets = (p.D + 127) / 128;
  // four sets to 16 lanes, one where there are few (300 x 1536: 2.3 us, 3.2 with four)
  const int64_t all = static_cast<int64_t>(p.M) * sets;
  const int64_t n = all <= static_cast<int64_t>(device_cu_count()) * 32 ? (all + 15) / 16 : (all + 63) / 64;
  const int64_t wgs = n < kMaxGroups ? n : kMaxGroups;
  return ECHO_LAUNCH("quantize_rows_fp4", (quantize_fp4_k<T, VEC>), dim3(static_cast<unsigned>(wgs)), dim3(256), 0,
                     stream, p, wgs * 16 / sets, static_cast<int>(wgs * 16 % sets));
}

template <typename T, int MAXT, int NV, bool VEC, bool NARROW = false>
hipError_t launch_ln(const QuantizeArgs& p, int threads, hipStream_t stream) {
  const int block = threads <= kWave ? 256 : threads, rpb = block / threads;
  // consecutive rows of a workgroup share one read of the modulation
  const int64_t want = static_cast<int64_t>(device_cu_count()) * 4096 / block;
  int64_t per = (p.M + want - 1) / want;
  per = (per + rpb - 1) / rpb * rpb;
  return ECHO_LAUNCH("quantize_rows_fp4", (quantize_fp4_ln_k<T, MAXT, NV, VEC, NARROW>),
                     dim3(static_cast<unsigned>((p.M + per - 1) / per)), dim3(block), 0, stream, p, threads,
                     static_cast<int>(per));
}

// What a reduction costs a wave is shared by its chunks, what it waits for by the
// workgroups of a CU: up to 512 columns 16 lanes with up to four chunks a row, up to
// 1024 a wave, then up to 256 threads with up to three chunks and no more threads than
// that takes (32760 x 5120: three chunks to 256 threads 106 us, two to 320 142; 100000 x
// 1024: two to a wave 60, one to 128 threads 73; 16000 x 8192: two to 512 threads 84, four
// to 256 102; 13104 x 13824: four to 448 threads 149, two to 896 172, 181 if they hold the
// modulation).  Rows of more than 16384 columns are more than 1024 threads hold: 71 to 85
// registers spill (5120 x 32768: 341 us, 1.25 TB/s; 10240 x 16384 without: 134, 3.2).
template <typename T, bool VEC>
hipError_t launch_ln_width(const QuantizeArgs& p, hipStream_t stream) {
  auto threads = [&](int chunks) { return (p.D + 8 * chunks * kWave - 1) / (8 * chunks * kWave) * kWave; };
  if (p.D <= 128) return launch_ln<T, 256, 1, VEC, true>(p, 16, stream);
  if (p.D <= 256) return launch_ln<T, 256, 2, VEC, true>(p, 16, stream);
  if (p.D <= 512) return launch_ln<T, 256, 4, VEC, true>(p, 16, stream);
  if (p.D <= 1024) return launch_ln<T, 256, 2, VEC>(p, kWave, stream);
  if (p.D <= 2048) return launch_ln<T, 256, 1, VEC>(p, threads(1), stream);
  if (p.D <= 4096) return launch_ln<T, 256, 2, VEC>(p, threads(2), stream);
  if (p.D <= 6144) return launch_ln<T, 256, 3, VEC>(p, threads(3), stream);
  if (p.D <= 8192) return launch_ln<T, 512, 2, VEC>(p, threads(2), stream);
  if (p.D <= 16384) return launch_ln<T, 512, 4, VEC>(p, threads(4), stream);
  return launch_ln<T, 1024, 8, VEC>(p, threads(8), stream);  // 65536 values
}

template <typename T>
hipError_t launch_type(const QuantizeArgs& p, hipStream_t stream) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p.x) | reinterpret_cast<uintptr_t>(p.shift) |
                       reinterpret_cast<uintptr_t>(p.scale);
  const bool vec = p.D % 8 == 0 && p.ldx % Elem<T>::kPerVec == 0 && at % 16 == 0;
  if (p.shift != nullptr) return vec ? launch_ln_width<T, true>(p, stream) : launch_ln_width<T, false>(p, stream);
  return vec ? launch_plain<T, true>(p, stream) : launch_plain<T, false>(p, stream);
}

}  // namespace

hipError_t launch_quantize_rows_fp4(int dtype_bf16, const QuantizeArgs& p, hipStream_t stream) {
  return dtype_bf16 ? launch_type<bf16_t>(p, stream) : launch_type<float>(p, stream);
}

hipError_t launch_dequantize_rows_fp4(int dtype_bf16, const DequantizeArgs& p, hipStream_t stream) {
  const int64_t n = (static_cast<int64_t>(p.M) * ((p.D + 7) / 8) + 255) / 256;
  const dim3 grid(static_cast<unsigned>(n < kMaxGroups ? n : kMaxGroups));
  auto go = [&](auto t) -> hipError_t {
    typedef decltype(t) T;
    return p.D % 8 == 0 && p.ldy % Elem<T>::kPerVec == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0
               ? ECHO_LAUNCH("dequantize_rows_fp4", (dequantize_fp4_k<T, true>), grid, dim3(256), 0, stream, p)
               : ECHO_LAUNCH("dequantize_rows_fp4", (dequantize_fp4_k<T, false>), grid, dim3(256), 0, stream, p);
  };
  return dtype_bf16 ? go(bf16_t{}) : go(0.0f);
}

}  // namespace echo
