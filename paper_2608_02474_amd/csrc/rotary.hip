// Rotary positions: the first `dims` channels of every head turn in pairs by an
// angle of the token's position,
//
//   (u, v) -> m (u cos t - v sin t, u sin t + v cos t),   t = pos f_j,
//
// pair j being channels (2j, 2j + 1) or (j, j + dims / 2); the other channels pass.
// pos is the token's number, its entry in `positions`, or, with a grid, its frame,
// row or column there (one of the three for each pair).  m scales for contexts
// longer than the frequencies were made for.
//
// The angle is the product of the position and the frequency in fp64 (a position
// of a million turns a fast pair 160000 times: fp32 would keep 6 bits of the
// angle), brought to an eighth of a turn in fp64, and its sine and cosine are
// taken in fp32.  A workgroup takes these once for all heads of its tokens, into
// LDS, and then turns its tokens' heads, 2 P channels a thread: the kernel is
// bound by the read and the write of the heads (bytes are touched once).
#include "common.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

// N consecutive elements as one access of at most 16 bytes each
template <typename T, int N>
struct RawN {
  static constexpr int kBytes = N * static_cast<int>(sizeof(T));
  static constexpr int kWords = kBytes < 4 ? 1 : kBytes / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i) {
        const uint4 v = ldg16_nt(reinterpret_cast<const char*>(p) + 16 * i);
        w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
      }
    } else if constexpr (kBytes == 8) {
      const uint2 v = ldg8_nt(p);
      w[0] = v.x, w[1] = v.y;
    } else if constexpr (kBytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
      w[0] = *reinterpret_cast<const uint16_t*>(p);
    }
  }
  __device__ __forceinline__ void store(T* p) const {
    if constexpr (kBytes >= 16) {
#pragma unroll
      for (int i = 0; i < kBytes / 16; ++i)
        stg16_nt(reinterpret_cast<char*>(p) + 16 * i, make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]));
    } else if constexpr (kBytes == 8) {
      *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (kBytes == 4) {
      *reinterpret_cast<uint32_t*>(p) = w[0];
    } else {
      *reinterpret_cast<uint16_t*>(p) = static_cast<uint16_t>(w[0]);
    }
  }
  __device__ __forceinline__ void unpack(float* o) const {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = __uint_as_float(w[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) o[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
  }
  __device__ __forceinline__ void pack(const float* o) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(o[i]);
    } else {
#pragma unroll
      for (int i = 0; i < (N + 1) / 2; ++i) w[i] = pack_bf16x2(o[2 * i], 2 * i + 1 < N ? o[2 * i + 1] : 0.0f);
    }
  }
};

constexpr int kRotThreads = 256;
constexpr int kRotPairs = 256;  // (cos, sin) of a workgroup's tokens in LDS

// cosine and sine of pos f, times m
__device__ __forceinline__ float2 turn_of(int pos, double f, float m) {
  constexpr double kTurns = 0.15915494309189533577;  // 1 / 2 pi
  const double t = static_cast<double>(pos) * f * kTurns;
  const double q = rint(4.0 * t);  // quarter turns
  float s, c;
  sincospif(static_cast<float>(2.0 * (t - 0.25 * q)), &s, &c);
  const int quarter = static_cast<int>(static_cast<int64_t>(q)) & 3;
  const float co = quarter == 0 ? c : quarter == 1 ? -s : quarter == 2 ? -c : s;
  const float si = quarter == 0 ? s : quarter == 1 ? c : quarter == 2 ? -s : -c;
  return make_float2(m * co, m * si);
}

// A unit is P pairs of one head, or as many passing channels; U units of a thread in
// flight.  Threads hold one unit number each and go over (token, head).  The pairs of a
// unit are one access (interleaved) or two (half), so that neighbouring threads' accesses
// are neighbours: two of 16 bytes each for 32 of interleaved pairs took 368 us where one
// of 16 takes 258 (32760 tokens x 80 heads of 128, bf16).
template <typename T, int P, bool HALF>
__global__ void __launch_bounds__(kRotThreads) rotary_k(RotaryArgs p, int tokens, int units, int turned) {
  constexpr int U = 4;
  __shared__ __attribute__((aligned(16))) float2 cs[kRotPairs];
  __shared__ int64_t at_token[4][kRotPairs];  // of q, its output, k, its output
  const int n = p.dims / 2, heads = p.H + p.Hk;
  const int64_t first = static_cast<int64_t>(blockIdx.x) * tokens, total = static_cast<int64_t>(p.B) * p.L;
  const int here = static_cast<int>(total - first < tokens ? total - first : tokens);
  if (static_cast<int>(threadIdx.x) < here) {
    const uint32_t tok = static_cast<uint32_t>(first) + threadIdx.x;  // B L < 2^24
    const int64_t b = tok / static_cast<uint32_t>(p.L), i = tok % static_cast<uint32_t>(p.L);
    at_token[0][threadIdx.x] = b * p.qb + i * p.qr;
    at_token[1][threadIdx.x] = b * p.qob + i * p.qor;
    at_token[2][threadIdx.x] = b * p.kb + i * p.kr;
    at_token[3][threadIdx.x] = b * p.kob + i * p.kor;
  }
  for (int e = threadIdx.x; e < here * n; e += kRotThreads) {
    const uint32_t tok = static_cast<uint32_t>(first) + e / n;
    const int j = e % n;
    const uint32_t b = tok / static_cast<uint32_t>(p.L), i = tok % static_cast<uint32_t>(p.L);
    int pos = p.positions != nullptr ? p.positions[b * p.pos_batch + i] : static_cast<int>(i);
    if (p.grid_w > 0) {
      const int col = pos % p.grid_w, rest = pos / p.grid_w;
      pos = j < p.pairs_t ? rest / p.grid_h : j < p.pairs_t + p.pairs_r ? rest % p.grid_h : col;
    }
    cs[e] = turn_of(pos, p.freq[j], p.magnitude);
  }
  __syncthreads();
  const int slots = kRotThreads / units;  // (token, head) items side by side
  const int unit = threadIdx.x % units, slot = threadIdx.x / units;
  if (slot >= slots) return;
  const bool pass = unit >= turned;
  const int at = pass ? p.dims + (unit - turned) * 2 * P : HALF ? unit * P : unit * 2 * P;
  // the second access of a unit: of half layouts, and of single pairs, whose last passing
  // unit may have one channel only
  constexpr bool TWO = HALF || P == 1;
  constexpr int N = TWO ? P : 2 * P;
  const int at2 = at + (!pass && HALF ? n : P);
  const bool second = TWO && at2 < p.dh;
  const int step_t = slots / heads, step_h = slots % heads;
  int tok = slot / heads, head = slot % heads;
  while (tok < here) {
    RawN<T, N> a[U], b[U];
    T* dst[U];
    int of[U];
    bool live[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      live[u] = tok < here;
      of[u] = live[u] ? tok : here - 1;
      const bool is_q = head < p.H;
      const int h = is_q ? head : head - p.H;
      const T* src = static_cast<const T*>(is_q ? p.q : p.k) + at_token[is_q ? 0 : 2][of[u]] + h * (is_q ? p.qh : p.kh);
      dst[u] = static_cast<T*>(is_q ? p.qo : p.ko) + at_token[is_q ? 1 : 3][of[u]] + h * (is_q ? p.qoh : p.koh);
      if (live[u]) {
        a[u].load(src + at);
        if (second) b[u].load(src + at2);
      }
      tok += step_t;
      head += step_h;
      if (head >= heads) head -= heads, ++tok;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (!live[u]) break;
      if (!pass) {
        float x[2 * P], y[2 * P];
        a[u].unpack(x);
        if constexpr (TWO) b[u].unpack(x + P);
        const float2* c = cs + of[u] * n + unit * P;
#pragma unroll
        for (int j = 0; j < P; ++j) {
          const int iu = HALF ? j : 2 * j, iv = HALF ? P + j : 2 * j + 1;
          const float2 r = c[j];
          y[iu] = x[iu] * r.x - x[iv] * r.y;
          y[iv] = x[iu] * r.y + x[iv] * r.x;
        }
        a[u].pack(y);
        if constexpr (TWO) b[u].pack(y + P);
      }
      a[u].store(dst[u] + at);
      if (second) b[u].store(dst[u] + at2);
    }
  }
}

namespace {

template <typename T, int P, bool HALF>
hipError_t launch_p(const RotaryArgs& p, hipStream_t stream) {
  const int n = p.dims / 2, turned = n / P;
  const bool in_place = p.q == p.qo && (p.Hk == 0 || p.k == p.ko);  // (then with the same strides)
  const int units = turned + (in_place ? 0 : (p.dh - p.dims + 2 * P - 1) / (2 * P));
  const int64_t total = static_cast<int64_t>(p.B) * p.L;
  // tokens to a workgroup: as many as it has threads for their pairs, one where
  // the device is not filled by that
  int tokens = kRotThreads / n > 1 ? kRotThreads / n : 1;
  while (tokens > 1 && (total + tokens - 1) / tokens < 4 * device_cu_count()) tokens /= 2;
  const dim3 grid(static_cast<unsigned>((total + tokens - 1) / tokens));
  return ECHO_LAUNCH("rotary", (rotary_k<T, P, HALF>), grid, dim3(kRotThreads), 0, stream, p, tokens, units, turned);
}

// the widest unit that divides the channels and to whose accesses every tensor is
// aligned: 16 bytes, or less
template <typename T>
hipError_t launch_t(const RotaryArgs& p, hipStream_t stream) {
  auto fits = [&](int pairs) {
    const int64_t el = p.half || pairs == 1 ? pairs : 2 * pairs, bytes = el * static_cast<int>(sizeof(T));
    auto at = [&](const void* q, int64_t b, int64_t r, int64_t h) {
      return reinterpret_cast<uintptr_t>(q) % bytes == 0 && b % el == 0 && r % el == 0 && h % el == 0;
    };
    return p.dims % (2 * pairs) == 0 && (p.dh - p.dims) % (2 * pairs) == 0 && at(p.q, p.qb, p.qr, p.qh) &&
           at(p.qo, p.qob, p.qor, p.qoh) &&
           (p.Hk == 0 || (at(p.k, p.kb, p.kr, p.kh) && at(p.ko, p.kob, p.kor, p.koh)));
  };
  constexpr int W = 16 / static_cast<int>(sizeof(T));  // elements of 16 bytes
  if (p.half) {
    if (fits(W)) return launch_p<T, W, true>(p, stream);
    if (fits(W / 2)) return launch_p<T, W / 2, true>(p, stream);
    if constexpr (W / 4 > 1)
      if (fits(W / 4)) return launch_p<T, W / 4, true>(p, stream);
    return launch_p<T, 1, true>(p, stream);
  }
  if (fits(W / 2)) return launch_p<T, W / 2, false>(p, stream);
  if constexpr (W / 4 > 1)
    if (fits(W / 4)) return launch_p<T, W / 4, false>(p, stream);
  return launch_p<T, 1, false>(p, stream);
}

}  // namespace

hipError_t launch_rotary(int bf16, const RotaryArgs& p, hipStream_t stream) {
  return bf16 ? launch_t<bf16_t>(p, stream) : launch_t<float>(p, stream);
}

}  // namespace echo
