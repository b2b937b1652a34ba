// The norms on both sides of a sub-layer with its gate and residual, in one pass:
//
//   y_i = a x_r(i) + gate_g * (N1(z_i) * w1),   h_i = N2(y_i) * w2 * (1 + scale_g) + shift_g
//
// z: the sub-layer's output, x: the residual stream (its rows picked by r), g:
// the row's modulation.  N1 and N2 are root-mean-square or layer norms (biased
// variance, two passes over registers) in fp32, N1 may be left out.  y and h are
// rounded once, h from the y that is not rounded.
//
// Apart, these are three kernels that write and read the stream between them;
// here z and x are read and y and h written once, and the kernel is bound by
// that: 26208 x 5120 with x and y in fp32 (1.6 GB) 335 us, 4.8 TB/s where a copy
// moves 5.1.  A row lies in the registers of 16 lanes, a wave or a workgroup; a
// workgroup takes consecutive rows with the vectors over the channels (gate w1,
// w2 (1 + scale), shift) in registers, and the next row's values on their way
// behind the first norm (during it too, they took the registers of a second
// workgroup on the CU).  Rows of more than 8192 columns do neither (they would
// leave 1024 threads no registers).  Unaligned rows take vector accesses at any
// element (7524 x 7341: 166 us where single elements took 769).
#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

// A row to `threads` threads (16 if NARROW, one wave or the whole workgroup), NV chunks
// of 8 values each.  VEC: every row of every tensor is aligned to 16 bytes and D % 8 == 0.
// HOLD: the vectors over the channels stay in registers for a workgroup's rows, and the
// next row is fetched ahead.
template <int MAXT, int NV, bool VEC, bool HOLD, bool NARROW, typename TZ, typename TX>
__global__ void __launch_bounds__(MAXT) gated_norm_k(GatedNormArgs p, int threads, int rows_per_wg) {
  __shared__ float red[2][4][MAXT / kWave];
  const int t = threadIdx.x % threads, D = p.D, rpb = blockDim.x / threads, waves = threads / kWave;
  int turn = 0;
  // reduction `slot` of a row: a piece of LDS each, of two sets in turn, so that
  // one barrier is enough
  auto total = [&](float v, int slot) __attribute__((always_inline)) {
    if constexpr (NARROW) return sum16(v);
    v = wave_sum(v);
    if (waves > 1) {
      if (t % kWave == 0) red[turn][slot][t / kWave] = v;
      __syncthreads();
      // (at most 16 waves: a partial sum to each lane of 16, and four steps)
      const int w = t & 15;
      v = sum16(w < waves ? red[turn][slot][w] : 0.0f);
    }
    return v;
  };
  auto in = [&](int u, int j) __attribute__((always_inline)) {
    const int c = (t + u * threads) * 8;
    return VEC ? c < D : c + j < D;
  };
  // v becomes its norm; what lies past the last column stays zero
  auto norm = [&](float (&v)[NV][8], int kind, int slot) __attribute__((always_inline)) {
    if (kind == NORM_LAYER) {
      float s = 0.0f;
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[u][j];
      const float mean = total(s, slot) / static_cast<float>(D);
#pragma unroll
      for (int u = 0; u < NV; ++u)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[u][j] = in(u, j) ? v[u][j] - mean : 0.0f;
    }
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) s = fmaf(v[u][j], v[u][j], s);
    const float r = 1.0f / sqrtf(total(s, slot + 1) / static_cast<float>(D) + p.eps);
#pragma unroll
    for (int u = 0; u < NV; ++u)
#pragma unroll
      for (int j = 0; j < 8; ++j) v[u][j] *= r;
  };
  // a vector over the channels, `none` where it is not given (past the last column 0)
  auto vector = [&](const float* w, int u, float none, float* o) __attribute__((always_inline)) {
    const int c = (t + u * threads) * 8;
    if (w != nullptr && (!VEC || c < D)) {  // (VEC: a branch 1 us shorter for one row than selects)
      Raw8<float> r;
      load_chunk<VEC, false>(r, w, c, D);
      if constexpr (VEC)
        r.unpack(o);
      else
        unpack_chunk<false>(r, c, D, o);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) o[j] = none;
    }
  };
  auto gate_of = [&](int g, int u, float* o) __attribute__((always_inline)) {  // gate w1
    float w[8];
    vector(p.gate != nullptr ? p.gate + g * p.ldgate : nullptr, u, 1.0f, o);
    vector(p.w1, u, 1.0f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= w[j];
  };
  auto scale_of = [&](int g, int u, float* o) __attribute__((always_inline)) {  // w2 (1 + scale)
    float w[8];
    vector(p.scale != nullptr ? p.scale + g * p.ldscale : nullptr, u, 0.0f, o);
    vector(p.w2, u, 1.0f, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = w[j] * (1.0f + o[j]);
  };
  auto shift_of = [&](int g, int u, float* o) __attribute__((always_inline)) {
    vector(p.shift != nullptr ? p.shift + g * p.ldshift : nullptr, u, 0.0f, o);
  };
  float ga[HOLD ? NV : 1][8], sc[HOLD ? NV : 1][8], sh[HOLD ? NV : 1][8];
  Raw8<TZ> nz[NV];
  Raw8<TX> nx[NV];
  bool nbad = false;
  auto source = [&](int64_t row, bool& bad) __attribute__((always_inline)) -> int64_t {
    bad = false;
    if (p.x_rows == nullptr) return row;
    const int32_t r = p.x_rows[row];
    bad = r < 0 || r >= p.x_nrows;  // no such row: NaN
    return bad ? 0 : r;
  };
  auto fetch = [&](int64_t row) __attribute__((always_inline)) {
    const int64_t xr = source(row, nbad);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int c = (t + u * threads) * 8;
      const TZ* z = static_cast<const TZ*>(p.z) + row * p.ldz;
      const TX* x = static_cast<const TX*>(p.x) + xr * p.ldx;
      load_chunk<VEC, true>(nz[u], z, c, D);
      load_chunk<VEC, true>(nx[u], x, c, D);
    }
  };
  const int64_t base = static_cast<int64_t>(blockIdx.x) * rows_per_wg;
  const int64_t end = base + rows_per_wg < p.M ? base + rows_per_wg : p.M;
  int64_t row = base + threadIdx.x / threads;
  int have = -1;
  if constexpr (HOLD)
    if (row < end) fetch(row);
  // (a group that reaches a barrier is the whole workgroup, so the loop is uniform for its waves)
  for (; row < end; row += rpb) {
    const int g = p.groups != nullptr ? p.groups[row] : static_cast<int>(row / p.rows_per_group);
    const bool no_group = g < 0 || g >= p.G;
    if constexpr (HOLD) {
      if (!no_group && g != have) {
        have = g;
#pragma unroll
        for (int u = 0; u < NV; ++u) gate_of(g, u, ga[u]), scale_of(g, u, sc[u]), shift_of(g, u, sh[u]);
      }
    }
    const int gm = no_group ? 0 : g;
    if constexpr (!HOLD) fetch(row);
    float v[NV][8];
    bool bad = nbad;
#pragma unroll
    for (int u = 0; u < NV; ++u) unpack_chunk<VEC>(nz[u], (t + u * threads) * 8, D, v[u]);
    bad = bad || no_group;
    if (p.after != NORM_NONE) norm(v, p.after, 0);
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      float m[8], x[8];
      if constexpr (!HOLD) gate_of(gm, u, m);
      if constexpr (VEC)
        nx[u].unpack(x);  // (zeroed past the row's end below)
      else
        unpack_chunk<false>(nx[u], (t + u * threads) * 8, D, x);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        v[u][j] = fmaf(v[u][j], HOLD ? ga[HOLD ? u : 0][j] : m[j], p.alpha * x[j]);
        if (bad) v[u][j] = __uint_as_float(0x7fc00000u);
        if (!in(u, j)) v[u][j] = 0.0f;
      }
    }
    // the next row's values, on their way through the stores and the second norm
    if constexpr (HOLD)
      if (row + rpb < end) fetch(row + rpb);
    auto put = [&](void* out, int bf, int64_t ld) __attribute__((always_inline)) {
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        const int c = (t + u * threads) * 8;
        if (bf)
          store_chunk<VEC, false>(static_cast<bf16_t*>(out) + row * ld, c, D, v[u]);
        else
          store_chunk<VEC, false>(static_cast<float*>(out) + row * ld, c, D, v[u]);
      }
    };
    put(p.y, p.y_bf16, p.ldy);
    if (p.before != NORM_NONE) {
      norm(v, p.before, 2);
#pragma unroll
      for (int u = 0; u < NV; ++u) {
        float m[8], a[8];
        if constexpr (!HOLD) scale_of(gm, u, m), shift_of(gm, u, a);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[u][j] = fmaf(v[u][j], HOLD ? sc[HOLD ? u : 0][j] : m[j], HOLD ? sh[HOLD ? u : 0][j] : a[j]);
      }
      put(p.h, p.h_bf16, p.ldh);
    }
    turn ^= 1;
  }
}

namespace {

template <int MAXT, int NV, bool VEC, bool HOLD, bool NARROW = false>
hipError_t launch_w(const GatedNormArgs& p, int threads, hipStream_t stream) {
  const int block = threads <= kWave ? 256 : threads, rpb = block / threads;
  // consecutive rows of a workgroup share one read of the vectors; of few rows each has a
  // workgroup of its own, which reads them all (1950 x 1536, five vectors: 10.6 us, 60 MB of
  // vectors from the L2s beside 36 MB of rows)
  // (a whole number of workgroups to a CU: 9000 x 13824 takes 431 us with 7/3 of them)
  const int64_t want = static_cast<int64_t>(device_cu_count()) * (2048 / block);
  int64_t per = (p.M + want - 1) / want;
  per = (per + rpb - 1) / rpb * rpb;
  const dim3 grid(static_cast<unsigned>((p.M + per - 1) / per));
  auto go = [&](auto z, auto x) -> hipError_t {
    return ECHO_LAUNCH("gated_norm", (gated_norm_k<MAXT, NV, VEC, HOLD, NARROW, decltype(z), decltype(x)>), grid, dim3(block), 0,
                       stream, p, threads, static_cast<int>(per));
  };
  if (p.z_bf16) return p.x_bf16 ? go(bf16_t{}, bf16_t{}) : go(bf16_t{}, 0.0f);
  return p.x_bf16 ? go(0.0f, bf16_t{}) : go(0.0f, 0.0f);
}
// The fewest chunks a thread that 256 threads hold the row with, and no more threads
// than that takes (26208 x 5120: three chunks to 256 threads 335 us, two to 320 390;
// 400000 x 64: 16 lanes to a row 67, a wave 193).  Wider rows, and unaligned ones whose
// bounds would take the registers of a second chunk, go to up to 1024 threads with one
// chunk, two from 8192 columns on (16000 x 8192: 327, four to 256 threads 354; 9000 x
// 13824: 359, four to 448 threads 395; 7524 x 7341: 166, four to 256 threads 617).
template <bool VEC>
hipError_t launch_v(const GatedNormArgs& p, hipStream_t stream) {
  auto threads = [&](int chunks) { return (p.D + 8 * chunks * kWave - 1) / (8 * chunks * kWave) * kWave; };
  if (p.D <= 128) return launch_w<256, 1, VEC, true, true>(p, 16, stream);
  if (p.D <= 2048) return launch_w<256, 1, VEC, true>(p, threads(1), stream);
  if constexpr (VEC) {  // (the bounds of unaligned rows take the registers that would hold the vectors)
    if (p.D <= 4096) return launch_w<256, 2, VEC, true>(p, threads(2), stream);
    if (p.D <= 6144) return launch_w<256, 3, VEC, true>(p, threads(3), stream);
  }
  if (p.D <= 8192) return launch_w<1024, 1, VEC, true>(p, threads(1), stream);
  return launch_w<1024, 2, VEC, false>(p, threads(2), stream);
}

}  // namespace

hipError_t launch_gated_norm(const GatedNormArgs& p, hipStream_t stream) {
  auto rows = [](const void* q, int bf, int64_t ld) {
    return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % (bf ? 8 : 4) == 0;
  };
  auto vec = [](const float* q, int64_t ld) { return reinterpret_cast<uintptr_t>(q) % 16 == 0 && ld % 4 == 0; };
  const bool aligned = p.D % 8 == 0 && rows(p.z, p.z_bf16, p.ldz) && rows(p.x, p.x_bf16, p.ldx) &&
                       rows(p.y, p.y_bf16, p.ldy) && (p.before == NORM_NONE || rows(p.h, p.h_bf16, p.ldh)) &&
                       vec(p.w1, 0) && vec(p.w2, 0) && vec(p.gate, p.ldgate) && vec(p.scale, p.ldscale) &&
                       vec(p.shift, p.ldshift);
  return aligned ? launch_v<true>(p, stream) : launch_v<false>(p, stream);
}

}  // namespace echo
