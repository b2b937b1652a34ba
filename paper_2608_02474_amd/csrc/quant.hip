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

// `exact`: decide every element in fp64
__device__ __forceinline__ int code_of(float a, float amax, float inv, bool exact) {
  const float q = a * inv;
  float n = rintf(q);
  if (exact || fabsf(q - n) > 0.5f - 0x1p-14f)
    n = static_cast<float>(rint(static_cast<double>(a) * 127.0 / static_cast<double>(amax)));
  return static_cast<int>(n);
}

// One row per group of THREADS threads, NV chunks of 8 values per thread.
template <typename T, int THREADS, int NV, bool VEC, bool LN>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS)
quantize_rows_k(QuantizeArgs p) {
  constexpr int BLOCK = THREADS < 256 ? 256 : THREADS, RPB = BLOCK / THREADS, NW = THREADS / kWave;
  __shared__ float red[NW > 1 ? NW : 1];
  const int t = threadIdx.x % THREADS;
  auto all = [&](float v, auto op) __attribute__((always_inline)) {
    v = wave_reduce(v, op);
    if constexpr (NW > 1) {
      __syncthreads();
      if (t % kWave == 0) red[t / kWave] = v;
      __syncthreads();
      v = red[0];
#pragma unroll
      for (int w = 1; w < NW; ++w) v = op(v, red[w]);
    }
    return v;
  };
  // (a workgroup's waves share its row where there are barriers, so the loop is uniform for them)
  for (int64_t row = static_cast<int64_t>(blockIdx.x) * RPB + threadIdx.x / THREADS; row < p.M;
       row += static_cast<int64_t>(gridDim.x) * RPB) {
    int64_t src = row;
    bool bad = false;
    if (p.rows != nullptr) {
      const int32_t r = p.rows[row];
      bad = r < 0 || r >= p.x_rows;  // no such row: as a row that is not finite
      src = bad ? 0 : r;
    }
    const T* xr = static_cast<const T*>(p.x) + src * p.ldx;
    const int D = p.D, nch = static_cast<int>(p.ldq / 8);

    float v[NV][8];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * THREADS) * 8;
      if constexpr (VEC) {  // D % 8 == 0 and aligned rows
        Raw8<T> raw;
        raw.load_nt(xr + (c < D ? c : 0));
        raw.unpack(v[u]);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = c < D ? v[u][j] : 0.0f;
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = c + j < D ? Elem<T>::load(xr, c + j) : 0.0f;
      }
    }
    if constexpr (LN) {
      auto add = [](float a, float b) { return a + b; };
      float sum = 0.0f, sq = 0.0f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += v[u][j];
      const float mean = all(sum, add) / static_cast<float>(D);
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float d = (t + u * THREADS) * 8 + j < D ? v[u][j] - mean : 0.0f;
          v[u][j] = d;
          sq += d * d;
        }
      const float rstd = 1.0f / sqrtf(all(sq, add) / static_cast<float>(D) + p.ln_eps);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int c = (t + u * THREADS) * 8;
        float sc[8], sh[8];
        if (VEC && c < D) {
          unpack16(ldg16(p.scale + c), sc, static_cast<const float*>(nullptr));
          unpack16(ldg16(p.scale + c + 4), sc + 4, static_cast<const float*>(nullptr));
          unpack16(ldg16(p.shift + c), sh, static_cast<const float*>(nullptr));
          unpack16(ldg16(p.shift + c + 4), sh + 4, static_cast<const float*>(nullptr));
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            sc[j] = c + j < D ? p.scale[c + j] : 0.0f;
            sh[j] = c + j < D ? p.shift[c + j] : 0.0f;
          }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = v[u][j] * rstd * (1.0f + sc[j]) + sh[j];
      }
    }
    // the largest magnitude as bits: those of infinities and NaN are above every number's
    uint32_t top = 0;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, abs_bits(v[u][j]));
    top = __float_as_uint(all(__uint_as_float(top), [](float a, float b) {
      return __uint_as_float(max(__float_as_uint(a), __float_as_uint(b)));
    }));
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
        uint32_t w[2] = {0u, 0u};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int n = none ? 0 : code_of(v[u][j], amax, inv, tiny);
          w[j / 4] |= (static_cast<uint32_t>(n) & 0xffu) << (8 * (j % 4));
        }
        *reinterpret_cast<uint2*>(crow + c * 8) = make_uint2(w[0], w[1]);
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
  const int groups = (p.M + RPB - 1) / RPB;
  return ECHO_LAUNCH("quantize_rows", (quantize_rows_k<T, THREADS, NV, VEC, LN>),
                     dim3(groups < kMaxGroups ? groups : kMaxGroups), dim3(BLOCK), 0, stream, p);
}

// the shortest form whose registers hold the row
template <typename T, bool VEC, bool LN>
hipError_t launch_q_width(const QuantizeArgs& p, hipStream_t stream) {
  const int64_t w = p.ldq;  // values to write, the padding included
  if (w <= 64 * 8) return launch_q<T, 64, 1, VEC, LN>(p, stream);
  if (w <= 64 * 8 * 4) return launch_q<T, 64, 4, VEC, LN>(p, stream);
  if (w <= 256 * 8 * 3) return launch_q<T, 256, 3, VEC, LN>(p, stream);
  if (w <= 256 * 8 * 8) return launch_q<T, 256, 8, VEC, LN>(p, stream);
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
