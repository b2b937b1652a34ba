// Rows held in 8 bits: codes in [-127, 127] with one scale per row, for the
// matrix products in 8-bit integers (gemm_int8.hip) and for states kept in a
// quarter or half of their bytes.
//
//   a_ij = x[rows(i)]_j                 or LN(x[rows(i)])_j (1 + scale_j) + shift_j
//   s_i  = fp32(max_j |a_ij| / 127),   c_ij = rint(127 a_ij / max_j |a_ij|)
//
// The code is the real quotient rounded once (ties to even), for every value
// of x: 127 x / amax of 16-bit values meets halves often (x = amax / 2 gives
// 63.5), and a quotient with two roundings falls to either side of them.  The
// fp32 product x * fl(127 / amax) is within 127 * 2^-23 of the quotient, so
// its rounding is the quotient's unless it lies within 2^-14 of a half; those
// few, and rows whose maximum is so small that 127 / amax overflows, are
// decided in fp64, whose quotient cannot cross a half: 254 x and an odd
// multiple of amax are multiples of a common unit that is at least 2^-32 of
// either.
//
// A row whose values are not all finite has scale NaN and codes 0, so that a
// product with it is NaN in that row and no other.  Rows are written up to
// their pitch (a multiple of 128 bytes), zeros behind the last column: the
// products then need no tail in their depth.
//
// One pass: a row stays in the registers of its wave (or of a workgroup, for
// longer rows) between the maximum and the codes.
#include <type_traits>

#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The codes of 8 values, packed.  q + 1.5 * 2^23 holds the whole number nearest
// to q in its low bits, ties to even (and a byte of it is the code).  `exact`:
// decide every value in fp64.
__device__ __forceinline__ uint2 codes8(const float* v, float amax, float inv, bool exact) {
  constexpr float kMagic = 12582912.0f, kNear = 0.5f - 0x1p-14f;
  float f[8], off = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float q = v[j] * inv;
    f[j] = q + kMagic;
    off = fmaxf(off, fabsf(q - (f[j] - kMagic)));
  }
  if (exact || off > kNear) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (exact || fabsf(v[j] * inv - (f[j] - kMagic)) > kNear)
        f[j] = kMagic + static_cast<float>(rint(static_cast<double>(v[j]) * 127.0 / static_cast<double>(amax)));
  }
  uint32_t w[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(f[4 * h + 1]), __float_as_uint(f[4 * h]), 0x0c0c0400u);
    const uint32_t up = __builtin_amdgcn_perm(__float_as_uint(f[4 * h + 3]), __float_as_uint(f[4 * h + 2]), 0x0c0c0400u);
    w[h] = __builtin_amdgcn_perm(up, lo, 0x05040100u);
  }
  return make_uint2(w[0], w[1]);
}

// One row per group of THREADS threads, NV chunks of 8 values per thread; a
// group goes from row to row, the next row's values on their way while one is
// worked on (VEC).  With LN (NV <= 4) the modulation stays in registers for all
// its rows: read again for each it was four times the bytes of a bf16 row.
template <typename T, int THREADS, int NV, bool VEC, bool LN>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS)
quantize_rows_k(QuantizeArgs p) {
  constexpr int BLOCK = THREADS < 256 ? 256 : THREADS, RPB = BLOCK / THREADS, NW = THREADS / kWave;
  constexpr bool HOLD = LN && NV <= 4, AHEAD = VEC && NV <= 4;
  __shared__ float red[3][NW > 1 ? NW : 1];
  const int t = threadIdx.x % THREADS;
  // reduction `slot` of a row over its group: each has its own piece of LDS, so
  // one barrier is enough (the others of a row lie between two uses of a piece;
  // without LN, whose single reduction uses pieces 0 and 1 in turn, one does)
  auto all = [&](float v, int slot, auto op) __attribute__((always_inline)) {
    if constexpr (THREADS == 16) {  // a row to every 16 lanes
      v = op(v, __uint_as_float(dpp_ror<8>(__float_as_uint(v))));
      v = op(v, __uint_as_float(dpp_ror<4>(__float_as_uint(v))));
      v = op(v, __uint_as_float(dpp_ror<2>(__float_as_uint(v))));
      return op(v, __uint_as_float(dpp_ror<1>(__float_as_uint(v))));
    }
    v = wave_reduce(v, op);
    if constexpr (NW > 1) {
      if (t % kWave == 0) red[slot][t / kWave] = v;
      __syncthreads();
      v = red[slot][0];
#pragma unroll
      for (int w = 1; w < NW; ++w) v = op(v, red[slot][w]);
    }
    return v;
  };
  const int D = p.D, nch = static_cast<int>(p.ldq / 8);
  auto source = [&](int64_t row, bool& bad) __attribute__((always_inline)) {
    int64_t src = row;
    bad = false;
    if (p.rows != nullptr) {
      const int32_t r = p.rows[row];
      bad = r < 0 || r >= p.x_rows;  // no such row: as a row that is not finite
      src = bad ? 0 : r;
    }
    return static_cast<const T*>(p.x) + src * p.ldx;
  };
  // 1 + scale and shift of chunk c; 0 and 0 past the last column, so that the
  // values there come out as zeros
  auto modulation = [&](int c, float* sc, float* sh) __attribute__((always_inline)) {
    if (VEC) {
      const int k = c < D ? c : 0;
      unpack16(ldg16(p.scale + k), sc, static_cast<const float*>(nullptr));
      unpack16(ldg16(p.scale + k + 4), sc + 4, static_cast<const float*>(nullptr));
      unpack16(ldg16(p.shift + k), sh, static_cast<const float*>(nullptr));
      unpack16(ldg16(p.shift + k + 4), sh + 4, static_cast<const float*>(nullptr));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool in = VEC ? c < D : c + j < D;
      if (!VEC) {
        sc[j] = in ? p.scale[c + j] : 0.0f;
        sh[j] = in ? p.shift[c + j] : 0.0f;
      }
      sc[j] = in ? 1.0f + sc[j] : 0.0f;
      sh[j] = in ? sh[j] : 0.0f;
    }
  };
  float sc[HOLD ? NV : 1][8], sh[HOLD ? NV : 1][8];
  if constexpr (HOLD) {
#pragma unroll
    for (int u = 0; u < NV; ++u) modulation((t + u * THREADS) * 8, sc[u], sh[u]);
  }
  Raw8<T> next[AHEAD ? NV : 1];
  bool next_bad = false;
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    const T* xr = source(row, next_bad);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * THREADS) * 8;
      next[u].load_nt(xr + (c < D ? c : 0));
    }
  };
  const int64_t first = static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / THREADS,
                step = static_cast<int64_t>(gridDim.x) * RPB;
  if constexpr (AHEAD)
    if (first < p.M) fetch(first);
  int turn = 0;
  // (where there are barriers a row is a whole workgroup's, so the loop is uniform for its waves)
  for (int64_t row = first; row < p.M; row += step) {
    bool bad;
    float v[NV][8];
    if constexpr (AHEAD) {
      bad = next_bad;
#pragma unroll
      for (int u = 0; u < NV; ++u) next[u].unpack(v[u]);
      if (row + step < p.M) fetch(row + step);
    } else {
      const T* xr = source(row, bad);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int c = (t + u * THREADS) * 8;
        if constexpr (VEC) {
          Raw8<T> raw;
          raw.load_nt(xr + (c < D ? c : 0));
          raw.unpack(v[u]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[u][j] = c + j < D ? Elem<T>::load(xr, c + j) : 0.0f;
        }
      }
    }
    if constexpr (VEC) {  // chunks past the last column (a chunk is in or out: D % 8 == 0)
#pragma unroll
      for (int u = 0; u < NV; ++u)
        if ((t + u * THREADS) * 8 >= D) {
#pragma unroll
          for (int j = 0; j < 8; ++j) v[u][j] = 0.0f;
        }
    }
    if constexpr (LN) {
      auto add = [](float a, float b) { return a + b; };
      float sum = 0.0f, sq = 0.0f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[u][j];
      const float mean = all(sum, 0, add) / static_cast<float>(D);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          v[u][j] -= mean;
          const float d = VEC || (t + u * THREADS) * 8 + j < D ? v[u][j] : 0.0f;
          part += d * d;
        }
        sq += !VEC || (t + u * THREADS) * 8 < D ? part : 0.0f;
      }
      const float rstd = 1.0f / sqrtf(all(sq, 1, add) / static_cast<float>(D) + p.ln_eps);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float c8[8], h8[8];
        if constexpr (!HOLD) modulation((t + u * THREADS) * 8, c8, h8);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[u][j] = fmaf(v[u][j] * rstd, HOLD ? sc[HOLD ? u : 0][j] : c8[j], HOLD ? sh[HOLD ? u : 0][j] : h8[j]);
      }
    }
    // the largest magnitude as bits: those of infinities and NaN are above every number's
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, abs_bits(v[u][j]));
    top = __float_as_uint(all(__uint_as_float(top), LN ? 2 : turn, [](float a, float b) {
      return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
    }));
    turn ^= 1;
    const float amax = __uint_as_float(top);
    bad = bad || top >= 0x7f800000u;
    const bool none = bad || top == 0;
    const bool tiny = amax < 0x1p-100f;
    const float inv = none || tiny ? 0.0f : 127.0f / amax;
    int8_t* crow = p.codes + row * p.ldq;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = t + u * THREADS;
      if (c < nch) {
        const uint2 w = codes8(v[u], amax, inv, tiny && !none);
        *reinterpret_cast<uint2*>(crow + c * 8) = none ? make_uint2(0u, 0u) : w;
      }
    }
    if (t == 0) p.row_scale[row] = bad ? __uint_as_float(0x7fc00000u) : amax / 127.0f;
  }
}

// y_ij = cast(fp32(s_i c_ij)); a thread takes 8 values
template <typename T>
__global__ void __launch_bounds__(256) dequantize_rows_k(DequantizeArgs p, int vec) {
  const int nch = (p.D + 7) / 8;
  for (int64_t e = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; e < static_cast<int64_t>(p.M) * nch;
       e += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t row = e / nch;
    const int c = static_cast<int>(e % nch) * 8;
    const uint2 w = *reinterpret_cast<const uint2*>(p.codes + row * p.ldq + c);
    const float s = p.row_scale[row];
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j)
      v[j] = s * static_cast<float>(static_cast<int8_t>((j < 4 ? w.x : w.y) >> (8 * (j % 4))));
    T* y = static_cast<T*>(p.y) + row * p.ldy + c;
    if (vec) {
      constexpr int PV = Elem<T>::kPerVec;
#pragma unroll
      for (int h = 0; h < 8 / PV; ++h) stg16_nt(y + h * PV, pack16(v + h * PV, static_cast<const T*>(nullptr)));
    } else {
      for (int j = 0; j < 8 && c + j < p.D; ++j) Elem<T>::store(y, j, v[j]);
    }
  }
}

namespace {

constexpr int kMaxGroups = 1 << 20;  // workgroups of a launch; more rows than that loop

template <typename T, int THREADS, int NV, bool VEC, bool LN>
hipError_t launch_q(const QuantizeArgs& p, hipStream_t stream) {
  constexpr int BLOCK = THREADS < 256 ? 256 : THREADS, RPB = BLOCK / THREADS;
  // With LN a group takes several rows for one read of the modulation; without,
  // rows of their own start sooner (32760 x 5120 bf16: 81 us against 91 with 16
  // groups a CU; with LN 137 and 150).
  const int64_t groups = (int64_t(p.M) + RPB - 1) / RPB, most = LN ? 16 * device_cu_count() : kMaxGroups;
  return ECHO_LAUNCH("quantize_rows", (quantize_rows_k<T, THREADS, NV, VEC, LN>),
                     dim3(static_cast<unsigned>(groups < most ? groups : most)), dim3(BLOCK), 0, stream, p);
}

// The shortest form whose registers hold the row.  (5120 wide: a row to 256
// threads 81 us, to a wave 99, to 512 threads 101; 13824 wide: 1024 threads 101,
// 256 threads 108; with LN and its registers 7800 x 1536: 256 threads 17.6, a wave
// 20.6.)
template <typename T, bool VEC, bool LN>
hipError_t launch_q_width(const QuantizeArgs& p, hipStream_t stream) {
  const int64_t w = p.ldq;  // values to write, the padding included
  if (w <= 16 * 8) return launch_q<T, 16, 1, VEC, LN>(p, stream);
  if (w <= 64 * 8) return launch_q<T, 64, 1, VEC, LN>(p, stream);
  if (w <= 64 * 8 * 4) {
    if constexpr (LN) return launch_q<T, 256, 1, VEC, LN>(p, stream);
    return launch_q<T, 64, 4, VEC, LN>(p, stream);
  }
  if (w <= 256 * 8 * 3) return launch_q<T, 256, 3, VEC, LN>(p, stream);
  if (w <= 1024 * 8 * 2) return launch_q<T, 1024, 2, VEC, LN>(p, stream);
  return launch_q<T, 1024, 8, VEC, LN>(p, stream);  // 65536 values
}

template <typename T>
hipError_t launch_q_type(const QuantizeArgs& p, hipStream_t stream) {
  const bool vec = p.D % 8 == 0 && p.ldx % Elem<T>::kPerVec == 0 && reinterpret_cast<uintptr_t>(p.x) % 16 == 0;
  if (p.shift != nullptr)
    return vec ? launch_q_width<T, true, true>(p, stream) : launch_q_width<T, false, true>(p, stream);
  return vec ? launch_q_width<T, true, false>(p, stream) : launch_q_width<T, false, false>(p, stream);
}

}  // namespace

hipError_t launch_quantize_rows(int dtype_bf16, const QuantizeArgs& p, hipStream_t stream) {
  return dtype_bf16 ? launch_q_type<bf16_t>(p, stream) : launch_q_type<float>(p, stream);
}

hipError_t launch_dequantize_rows(int dtype_bf16, const DequantizeArgs& p, hipStream_t stream) {
  const int64_t n = static_cast<int64_t>(p.M) * ((p.D + 7) / 8);
  const dim3 grid(static_cast<unsigned>((n + 255) / 256 < kMaxGroups ? (n + 255) / 256 : kMaxGroups));
  const int per = dtype_bf16 ? 8 : 4;
  const int vec = p.D % 8 == 0 && p.ldy % per == 0 && reinterpret_cast<uintptr_t>(p.y) % 16 == 0;
  return dtype_bf16
             ? ECHO_LAUNCH("dequantize_rows", dequantize_rows_k<bf16_t>, grid, dim3(256), 0, stream, p, vec)
             : ECHO_LAUNCH("dequantize_rows", dequantize_rows_k<float>, grid, dim3(256), 0, stream, p, vec);
}

}  // namespace echo
