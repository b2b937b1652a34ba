// Outputs of the products of quantized rows (gemm_int8.hip, gemm_fp4.hip):
//
//   C[m, n] = f( za[m, n] sb[n] + bias[n] )     (without sb where Args::kScaled is false)
//   f: none, GELU (tanh form), or res[row(m), n] + gate[n] * (.) in fp32
//
// Args has N, bias, bias_bf16, C, c_bf16, ldc, gate, res, res_bf16, ldr, res_rows and
// res_nrows (RowsOut in kernels.h), and sb where it is scaled.
#pragma once

#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace echo {

__device__ __forceinline__ float out_load(const void* p, int bf, int64_t i) {
  return bf ? bf16_to_f32(static_cast<const bf16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}

// z -> f(z), res being the residual and gate the channel's gate
template <int EPI>
__device__ __forceinline__ float out_finish(float z, float gate, float res) {
  if constexpr (EPI == EPI_GELU) return gelu_tanh_fast(z);
  if constexpr (EPI == EPI_GATE_RES) return fmaf(gate, z, res);
  return z;
}

// the residual row of output row m; -1: no such row
template <typename Args>
__device__ __forceinline__ int out_res_row(const Args& p, int m) {
  if (p.res_rows == nullptr) return m;
  const int r = p.res_rows[m];
  return r >= 0 && r < p.res_nrows ? r : -1;
}

// One output; za = the sum, rounded to fp32, times the token's factor.
template <int EPI, bool CBF, typename Args>
__device__ __forceinline__ void out_store1(const Args& p, int m, int n, float za) {
  const float bias = p.bias != nullptr ? out_load(p.bias, p.bias_bf16, n) : 0.0f;
  float z = za + bias;
  if constexpr (Args::kScaled) z = fmaf(za, p.sb[n], bias);
  float res = 0.0f, gate = 0.0f;
  if constexpr (EPI == EPI_GATE_RES) {
    const int rr = out_res_row(p, m);
    gate = p.gate[n];
    res = rr < 0 ? __uint_as_float(0x7fc00000u) : out_load(p.res, p.res_bf16, rr * p.ldr + n);
  }
  const float v = out_finish<EPI>(z, gate, res);
  const int64_t at = m * p.ldc + n;
  if constexpr (CBF)
    Elem<bf16_t>::store(static_cast<bf16_t*>(p.C), at, v);
  else
    static_cast<float*>(p.C)[at] = v;
}

// ---- four consecutive channels at a time, where rows of C, of the residual,
// and the vectors over the channels are aligned for that and N % 4 == 0 (vec)
template <typename Args>
__device__ __forceinline__ bool out_vec(const Args& p) {
  const uintptr_t ca = reinterpret_cast<uintptr_t>(p.C), ra = reinterpret_cast<uintptr_t>(p.res),
                  ba = reinterpret_cast<uintptr_t>(p.bias);
  uintptr_t fa = reinterpret_cast<uintptr_t>(p.gate);
  if constexpr (Args::kScaled) fa |= reinterpret_cast<uintptr_t>(p.sb);
  const int ce = p.c_bf16 ? 8 : 16, re = p.res_bf16 ? 8 : 16, be = p.bias_bf16 ? 8 : 16;
  return (p.N & 3) == 0 && (p.ldc & 3) == 0 && (ca & (ce - 1)) == 0 && (p.ldr & 3) == 0 && (ra & (re - 1)) == 0 &&
         (ba & (be - 1)) == 0 && (fa & 15) == 0;
}
__device__ __forceinline__ void out_load4(const void* p, int bf, int64_t i, float* v) {
  if (bf) {
    const uint2 raw = *reinterpret_cast<const uint2*>(static_cast<const bf16_t*>(p) + i);
    v[0] = __uint_as_float(raw.x << 16);
    v[1] = __uint_as_float(raw.x & 0xffff0000u);
    v[2] = __uint_as_float(raw.y << 16);
    v[3] = __uint_as_float(raw.y & 0xffff0000u);
  } else {
    unpack16(ldg16(static_cast<const float*>(p) + i), v, static_cast<const float*>(nullptr));
  }
}
// four residuals as loaded, bf16 or fp32; `miss`: NaN in their place
template <bool BF>
struct ResRaw {
  uint2 v;
  __device__ void load(const void* p, int64_t i) { v = ldg8_nt(static_cast<const bf16_t*>(p) + i); }
  __device__ void unpack(bool miss, float* o) const {
    const uint32_t w[2] = {miss ? 0x7fc07fc0u : v.x, miss ? 0x7fc07fc0u : v.y};
    o[0] = __uint_as_float(w[0] << 16);
    o[1] = __uint_as_float(w[0] & 0xffff0000u);
    o[2] = __uint_as_float(w[1] << 16);
    o[3] = __uint_as_float(w[1] & 0xffff0000u);
  }
};
template <>
struct ResRaw<false> {
  uint4 v;
  __device__ void load(const void* p, int64_t i) { v = ldg16_nt(static_cast<const float*>(p) + i); }
  __device__ void unpack(bool miss, float* o) const {
    unpack16(v, o, static_cast<const float*>(nullptr));
    if (miss) o[0] = o[1] = o[2] = o[3] = __uint_as_float(0x7fc00000u);
  }
};

// scale, bias and gate of channels n .. n + 3
struct OutCols {
  float sb[4], bias[4], gate[4];
};
template <int EPI, typename Args>
__device__ __forceinline__ void out_cols4(const Args& p, int n, OutCols& c) {
  if constexpr (Args::kScaled) out_load4(p.sb, 0, n, c.sb);
  if (p.bias != nullptr)
    out_load4(p.bias, p.bias_bf16, n, c.bias);
  else
    c.bias[0] = c.bias[1] = c.bias[2] = c.bias[3] = 0.0f;
  if constexpr (EPI == EPI_GATE_RES) out_load4(p.gate, 0, n, c.gate);
}
template <int EPI, bool CBF, typename Args>
__device__ __forceinline__ void out_store4(const Args& p, int m, int n, const f32x4& za, const OutCols& c,
                                           const float* res) {
  float v[4];
#pragma unroll
  for (int r = 0; r < 4; ++r)
    v[r] = out_finish<EPI>(Args::kScaled ? fmaf(za[r], c.sb[r], c.bias[r]) : za[r] + c.bias[r], c.gate[r], res[r]);
  const int64_t at = m * p.ldc + n;
  if constexpr (CBF)
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(p.C) + at) =
        make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else
    stg16(static_cast<float*>(p.C) + at, pack16(v, static_cast<const float*>(nullptr)));
}

// Four outputs of one token by themselves, vec or not (n < N).
template <int EPI, bool CBF, typename Args>
__device__ __forceinline__ void out_put4(const Args& p, int m, int n, const f32x4& za) {
  if (!out_vec(p)) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
      if (n + r < p.N) out_store1<EPI, CBF>(p, m, n + r, za[r]);
    return;
  }
  OutCols cols;
  out_cols4<EPI>(p, n, cols);
  float res[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (EPI == EPI_GATE_RES) {
    const int rr = out_res_row(p, m);
    out_load4(p.res, p.res_bf16, static_cast<int64_t>(rr < 0 ? 0 : rr) * p.ldr + n, res);
    if (rr < 0) res[0] = res[1] = res[2] = res[3] = __uint_as_float(0x7fc00000u);
  }
  out_store4<EPI, CBF>(p, m, n, za, cols, res);
}

// f(epilogue, whether C, whether the residual is bf16) as compile-time constants
template <typename F>
inline hipError_t with_epilogue(int epi, int c_bf16, int res_bf16, F&& f) {
  auto go = [&](auto epi_c, auto res_c) -> hipError_t {
    return c_bf16 ? f(epi_c, std::true_type{}, res_c) : f(epi_c, std::false_type{}, res_c);
  };
  if (epi == EPI_GELU) return go(std::integral_constant<int, EPI_GELU>{}, std::true_type{});
  if (epi != EPI_GATE_RES) return go(std::integral_constant<int, EPI_BIAS>{}, std::true_type{});
  return res_bf16 ? go(std::integral_constant<int, EPI_GATE_RES>{}, std::true_type{})
                  : go(std::integral_constant<int, EPI_GATE_RES>{}, std::false_type{});
}

}  // namespace echo
