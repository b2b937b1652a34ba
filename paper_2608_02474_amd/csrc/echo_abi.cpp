// C ABI of libecho: argument validation, workspace carving and the launch
// sequence of each call.  Every check runs before the first HIP call, so a
// rejected call touches neither the device nor the stream.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <cmath>
#include <mutex>
#include <vector>

#include "../../include/echo.h"
#include "kernels.h"
#include "launch.h"

namespace echo {

// ---- per-thread error and timing state
static thread_local int g_last_hip_error = 0;

struct TimingRecord {
  const char* name;
  hipEvent_t start, stop;
};
static thread_local bool g_profile = false;
static thread_local std::vector<TimingRecord> g_records;
static thread_local std::vector<hipEvent_t> g_event_pool;

bool profile_enabled() { return g_profile; }
void profile_set(bool on) { g_profile = on; }

static hipEvent_t take_event() {
  if (!g_event_pool.empty()) {
    hipEvent_t e = g_event_pool.back();
    g_event_pool.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  if (hipEventCreate(&e) != hipSuccess) return nullptr;
  return e;
}

TimedLaunch::TimedLaunch(const char* name, hipStream_t s) : slot(-1), stream(s) {
  if (!g_profile) return;
  TimingRecord r{name, take_event(), take_event()};
  if (r.start == nullptr || r.stop == nullptr || hipEventRecord(r.start, s) != hipSuccess) {
    if (r.start) g_event_pool.push_back(r.start);
    if (r.stop) g_event_pool.push_back(r.stop);
    return;
  }
  g_records.push_back(r);
  slot = static_cast<int>(g_records.size()) - 1;
}
TimedLaunch::~TimedLaunch() {
  if (slot >= 0) (void)hipEventRecord(g_records[slot].stop, stream);
}

int device_cu_count() {
  static const int n = [] {
    int dev = 0, cu = 0;
    if (hipGetDevice(&dev) != hipSuccess ||
        hipDeviceGetAttribute(&cu, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cu <= 0)
      cu = 256;
    return cu;
  }();
  return n;
}

size_t gemm_partial_bytes() { return sizeof(float) * 256 * 256 * 256; }

}  // namespace echo

using namespace echo;

namespace {

constexpr size_t kAlign = 256;
constexpr size_t align_up(size_t n) { return (n + kAlign - 1) / kAlign * kAlign; }
inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline bool ok_ptr(const void* p) { return p != nullptr && aligned16(p); }
inline size_t esize(int dtype) { return dtype == ECHO_BF16 ? 2 : 4; }
inline bool ok_dtype(int dtype) { return dtype == ECHO_F32 || dtype == ECHO_BF16; }

int device_status(hipError_t e) {
  if (e == hipSuccess) return ECHO_OK;
  g_last_hip_error = static_cast<int>(e);
  return ECHO_EDEVICE;
}

// ---- energy
bool energy_cfg_ok(const echo_energy_cfg* c, int64_t n_samples) {
  return c != nullptr && c->T >= 1 && c->T <= 65535 && n_samples >= c->T && c->n_fft >= 16 &&
         c->n_fft <= 2048 && (c->n_fft % 2) == 0 && c->hop >= 1 && c->n_bands >= 1 &&
         c->n_bands <= 64 && c->sample_rate > 0;
}
size_t energy_ws(const echo_energy_cfg* c, int64_t n_samples) {
  const int mf = energy_max_frames(n_samples, c->T, c->n_fft, c->hop);
  // per-frame band energies, then per-segment energies and band sums
  return align_up(sizeof(double) * static_cast<size_t>(c->T) * mf * c->n_bands) +
         align_up(sizeof(double) * static_cast<size_t>(c->T) * (1 + c->n_bands));
}

// ---- select
bool select_cfg_ok(const echo_select_cfg* c) {
  if (c == nullptr || c->T < 1 || c->N < 1 || c->D < 8 || (c->D % 8) != 0 || !ok_dtype(c->dtype))
    return false;
  const int64_t L = static_cast<int64_t>(c->T) * c->N;
  if (L >= (int64_t(1) << 31)) return false;
  if (c->k > L) return false;
  if (!(c->xi >= 0.0) || isnan(c->threshold)) return false;
  return true;
}
size_t select_ws(const echo_select_cfg* c) {
  const size_t L = static_cast<size_t>(c->T) * c->N;
  return align_up(L * sizeof(float)) + 2 * align_up(L * sizeof(double));
}

int select_args_status(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                       const int32_t* idx, const uint8_t* mask, const int32_t* n_sel, const float* saliency,
                       const double* step_delta) {
  if (!select_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!ok_ptr(x) || !ok_ptr(xref) || !ok_ptr(frame_weight) || !ok_ptr(idx) || !ok_ptr(mask) ||
      n_sel == nullptr)
    return ECHO_EINVAL;
  if ((saliency != nullptr && !aligned16(saliency)) ||
      (step_delta != nullptr && (reinterpret_cast<uintptr_t>(step_delta) & 7u)))
    return ECHO_EINVAL;
  return ECHO_OK;
}
int select_launch(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                  int32_t* idx, uint8_t* mask, int32_t* n_sel, float* saliency, double* step_delta,
                  void* workspace, void* stream);

// ---- allocation-free selection: the workspace of echo_select for up to
// ECHO_SELECT_NOALLOC_MAX_TOKENS tokens as a static device array.  Each GPU
// holds its own copy; its address is looked up once per device (with that
// device current) and kept, and only that address is handed to kernels: in
// host code the array's name is not a device address.
constexpr size_t kNoAllocScratchBytes =
    align_up(ECHO_SELECT_NOALLOC_MAX_TOKENS * sizeof(float)) + 2 * align_up(ECHO_SELECT_NOALLOC_MAX_TOKENS * sizeof(double));
__device__ __align__(256) char scratch[kNoAllocScratchBytes];

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
void* g_scratch_ptr[kMaxDevices] = {};

// Device address of the current device's scratch array (ECHO_EDEVICE if the
// lookup fails).
int noalloc_scratch(void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return device_status(e);
  if (dev < 0 || dev >= kMaxDevices) return ECHO_EUNSUPPORTED;
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (g_scratch_ptr[dev] == nullptr) {
    void* p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess) return device_status(e);
    if (p == nullptr) return ECHO_EDEVICE;
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return ECHO_OK;
}

// ---- block
bool block_cfg_ok(const echo_block_cfg* c) {
  return c != nullptr && c->L >= 1 && c->D >= 8 && c->H >= 1 && c->F >= 8 && ok_dtype(c->dtype) &&
         c->D <= 16384 && c->F <= 65536 && (c->D % c->H) == 0 && (c->D % 8) == 0 &&
         (c->F % 8) == 0 && c->ln_eps >= 0.0f && (c->flags & ~ECHO_BLOCK_BATCH_INVARIANT) == 0;
}
bool block_supported(const echo_block_cfg* c) {
  const int dh = c->D / c->H;
  // bf16 GEMM tiles address their operands through 32-bit byte offsets
  if (c->dtype == ECHO_BF16)
    return dh == 128 && (c->D % 256) == 0 && (c->F % 256) == 0 &&
           int64_t(c->L) * c->D < (int64_t(1) << 30) && int64_t(c->F) * c->D < (int64_t(1) << 30);
  return dh <= 128;
}
struct BlockWs {
  void *a, *kv, *q, *o, *b, *h;
  float* x1;
  float* part;        // bf16 path: partial results of the GEMM and attention tails
  size_t part_bytes;  // its size: the larger of the two needs
  size_t bytes;
};
size_t max_size(size_t a, size_t b) { return a > b ? a : b; }
BlockWs block_ws_layout(const echo_block_cfg* c, int64_t n, char* base) {
  const size_t es = esize(c->dtype);
  const size_t L = c->L, D = c->D, F = c->F, m = static_cast<size_t>(n);
  BlockWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += align_up(bytes);
    return p;
  };
  w.a = take(L * D * es);
  w.kv = take(L * 2 * D * es);
  w.q = take(m * D * es);
  w.o = take(m * D * es);
  w.x1 = reinterpret_cast<float*>(take(m * D * 4));
  w.b = take(m * D * es);
  w.h = take(m * F * es);
  if (c->dtype == ECHO_BF16) {
    w.part_bytes = max_size(gemm_partial_bytes(), attn_partial_bytes(static_cast<int>(n), c->L, c->H));
    w.part = reinterpret_cast<float*>(take(w.part_bytes));
  }
  w.bytes = off;
  return w;
}
bool weights_ok(const echo_block_weights* w) {
  return w != nullptr && ok_ptr(w->wq) && ok_ptr(w->wk) && ok_ptr(w->wv) && ok_ptr(w->wo) &&
         ok_ptr(w->w1) && ok_ptr(w->w2) && ok_ptr(w->bq) && ok_ptr(w->bk) && ok_ptr(w->bv) &&
         ok_ptr(w->bo) && ok_ptr(w->b1) && ok_ptr(w->b2) && ok_ptr(w->mod);
}

}  // namespace

namespace {
bool refcache_cfg_ok(const echo_refcache_cfg* c) {
  return c != nullptr && c->L >= 1 && c->D >= 8 && (c->D % 8) == 0 && c->D <= 16384 && ok_dtype(c->dtype) &&
         c->chain_len >= 1 && (c->L % c->chain_len) == 0 && std::isfinite(c->tau) &&
         static_cast<int64_t>(c->capacity) >= static_cast<int64_t>(c->L) + c->L / c->chain_len;
}
bool refcache_state_ok(const echo_refcache_state* s) {
  return s != nullptr && ok_ptr(s->pool) && ok_ptr(s->refcount) && ok_ptr(s->free_list) && ok_ptr(s->free_top) &&
         ok_ptr(s->chain_ref) && ok_ptr(s->ent_slot) && ok_ptr(s->ent_kind) && ok_ptr(s->codes) &&
         ok_ptr(s->scale);
}
}  // namespace

namespace {
bool wan_cfg_ok(const echo_wan_block_cfg* c) {
  return c != nullptr && c->B >= 1 && c->L >= 1 && c->D >= 8 && c->H >= 1 && c->F >= 8 && c->Lc >= 1 &&
         c->T >= 1 && c->gh >= 1 && c->gw >= 1 && int64_t(c->T) * c->gh * c->gw == c->L &&
         ok_dtype(c->dtype) && c->D <= 16384 && c->F <= 65536 && (c->D % c->H) == 0 && (c->D % 8) == 0 &&
         (c->F % 8) == 0 && c->ln_eps >= 0.0f && c->rms_eps >= 0.0f && std::isfinite(c->rope_base) &&
         c->rope_base > 0.0 && (c->flags & ~ECHO_BLOCK_BATCH_INVARIANT) == 0;
}
bool wan_supported(const echo_wan_block_cfg* c) {
  const int64_t lim = int64_t(1) << 30;
  return c->dtype == ECHO_BF16 && c->D / c->H == 128 && (c->D % 256) == 0 && (c->F % 256) == 0 &&
         int64_t(c->B) * c->L * c->D < lim && int64_t(c->B) * c->Lc * c->D < lim && int64_t(c->F) * c->D < lim;
}
struct WanWs {
  void *a, *kv, *kvc, *q, *o, *b, *h;
  float *x1, *x2, *part, *ones, *g3m1;
  float2* tab;
  size_t part_bytes;
  size_t bytes;
};
WanWs wan_ws_layout(const echo_wan_block_cfg* c, int64_t n, char* base) {
  const size_t es = esize(c->dtype);
  const size_t BL = size_t(c->B) * c->L, BLc = size_t(c->B) * c->Lc, D = c->D, F = c->F, m = size_t(n);
  WanWs w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += align_up(bytes);
    return p;
  };
  w.a = take(BL * D * es);
  w.kv = take(BL * 2 * D * es);
  w.kvc = take(BLc * 2 * D * es);
  w.q = take(m * D * es);
  w.o = take(m * D * es);
  w.b = take(m * D * es);
  w.h = take(m * F * es);
  w.x1 = reinterpret_cast<float*>(take(m * D * 4));
  w.x2 = reinterpret_cast<float*>(take(m * D * 4));
  // the attention runs per batch element, with at most n selected rows
  w.part_bytes = max_size(gemm_partial_bytes(),
                          max_size(attn_partial_bytes(static_cast<int>(n), c->L, c->H),
                                   attn_partial_bytes(static_cast<int>(n), c->Lc, c->H)));
  w.part = reinterpret_cast<float*>(take(w.part_bytes));
  w.ones = reinterpret_cast<float*>(take(D * 4));
  w.g3m1 = reinterpret_cast<float*>(take(D * 4));
  w.tab = reinterpret_cast<float2*>(take(sizeof(float2) * size_t(rope_table_entries(c->T, c->gh, c->gw,
                                                                                     c->D / c->H))));
  w.bytes = off;
  return w;
}
bool wan_weights_ok(const echo_wan_block_weights* w) {
  return w != nullptr && weights_ok(&w->self) && ok_ptr(w->wqc) && ok_ptr(w->wkc) && ok_ptr(w->wvc) &&
         ok_ptr(w->woc) && ok_ptr(w->bqc) && ok_ptr(w->bkc) && ok_ptr(w->bvc) && ok_ptr(w->boc) &&
         ok_ptr(w->gq) && ok_ptr(w->gk) && ok_ptr(w->gqc) && ok_ptr(w->gkc) && ok_ptr(w->g3) && ok_ptr(w->b3);
}
}  // namespace

namespace {
// ---- rows in 8 bits
bool elem_aligned(const void* p, size_t es) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) % es) == 0; }
bool quantize_cfg_ok(const echo_quantize_cfg* c) {
  return c != nullptr && c->M >= 0 && c->D >= 1 && c->D <= 65536 && ok_dtype(c->dtype) && c->ldx >= c->D &&
         c->ldq >= echo_int8_pitch(c->D) && c->ldq <= 65536 && (c->ldq % 128) == 0 && c->ln_eps >= 0.0f;
}
bool linear_cfg_ok(const echo_linear_int8_cfg* c) {
  return c != nullptr && c->M >= 0 && c->N >= 1 && c->K >= 1 && c->K <= 65536 && ok_dtype(c->out_dtype) &&
         ok_dtype(c->bias_dtype) && ok_dtype(c->residual_dtype) &&
         (c->epilogue == ECHO_LINEAR_NONE || c->epilogue == ECHO_LINEAR_GELU_TANH ||
          c->epilogue == ECHO_LINEAR_GATE_RESIDUAL) &&
         c->lda >= echo_int8_pitch(c->K) && (c->lda % 128) == 0 && c->ldw >= echo_int8_pitch(c->K) &&
         (c->ldw % 128) == 0 && c->lda <= 65536 && c->ldw <= 65536 && c->ldc >= c->N &&
         (c->epilogue != ECHO_LINEAR_GATE_RESIDUAL || c->ldr >= c->N);
}
// a launch holds fewer than 2^32 threads: 2^24 workgroups of 256
constexpr int64_t kMaxGroups = int64_t(1) << 24;
bool linear_supported(const echo_linear_int8_cfg* c) {
  return c->N <= (1 << 22) && ((int64_t(c->M) + 63) / 64) * ((int64_t(c->N) + 63) / 64) < kMaxGroups;
}

// ---- rows in 4 bits
bool fp4_rows_ok(int64_t ld, int64_t lds, int32_t D) {
  return ld >= echo_fp4_pitch(D) && ld <= 65536 && ld % 128 == 0 && lds >= echo_fp4_scale_pitch(D) && lds <= 65536 &&
         lds % 16 == 0;
}
bool quantize_fp4_cfg_ok(const echo_quantize_fp4_cfg* c) {
  return c != nullptr && c->M >= 0 && c->D >= 1 && c->D <= 65536 && ok_dtype(c->dtype) && c->ldx >= c->D &&
         fp4_rows_ok(c->ldq, c->lds, c->D) && c->ln_eps >= 0.0f;
}
bool linear_fp4_cfg_ok(const echo_linear_fp4_cfg* c) {
  return c != nullptr && c->M >= 0 && c->N >= 1 && c->K >= 1 && c->K <= 65536 && ok_dtype(c->out_dtype) &&
         ok_dtype(c->bias_dtype) && ok_dtype(c->residual_dtype) &&
         (c->epilogue == ECHO_LINEAR_NONE || c->epilogue == ECHO_LINEAR_GELU_TANH ||
          c->epilogue == ECHO_LINEAR_GATE_RESIDUAL) &&
         fp4_rows_ok(c->lda, c->ldsa, c->K) && fp4_rows_ok(c->ldw, c->ldsw, c->K) && c->ldc >= c->N &&
         (c->epilogue != ECHO_LINEAR_GATE_RESIDUAL || c->ldr >= c->N);
}
bool linear_fp4_supported(const echo_linear_fp4_cfg* c) {
  return c->N <= (1 << 22) && ((int64_t(c->M) + 63) / 64) * ((int64_t(c->N) + 63) / 64) < kMaxGroups;
}

// ---- rotary positions
bool rotary_strides_ok(const echo_strides& s) { return s.batch >= 0 && s.row >= 0 && s.head >= 0; }
bool rotary_cfg_ok(const echo_rotary_cfg* c) {
  return c != nullptr && c->B >= 0 && c->L >= 0 && c->H >= 1 && c->Hk >= 0 && c->dims >= 2 && c->dims % 2 == 0 &&
         c->dims <= c->dh && (c->layout == ECHO_ROTARY_INTERLEAVED || c->layout == ECHO_ROTARY_HALF) &&
         ok_dtype(c->dtype) && c->grid_h >= 0 && c->grid_w >= 0 && (c->grid_h > 0) == (c->grid_w > 0) &&
         c->pairs_t >= 0 && c->pairs_r >= 0 && int64_t(c->pairs_t) + c->pairs_r <= c->dims / 2 &&
         std::isfinite(c->magnitude) && c->pos_batch >= 0 && rotary_strides_ok(c->q) && rotary_strides_ok(c->q_out) &&
         (c->Hk == 0 || (rotary_strides_ok(c->k) && rotary_strides_ok(c->k_out)));
}
bool rotary_supported(const echo_rotary_cfg* c) {
  return c->dh <= 512 && int64_t(c->H) + c->Hk <= 65536 && int64_t(c->B) * c->L < (int64_t(1) << 24);
}
bool same_strides(const echo_strides& a, const echo_strides& b) {
  return a.batch == b.batch && a.row == b.row && a.head == b.head;
}
// an output's rows: in the place of a repeated input row they would be turned once each
bool rows_apart(const echo_strides& s, int32_t B, int32_t L, int32_t H) {
  return (B == 1 || s.batch > 0) && (L == 1 || s.row > 0) && (H == 1 || s.head > 0);
}

// ---- norms on both sides of a sub-layer
bool norm_ok(int n) { return n == ECHO_NORM_NONE || n == ECHO_NORM_RMS || n == ECHO_NORM_LAYER; }
bool gated_norm_cfg_ok(const echo_gated_norm_cfg* c) {
  auto mod = [&](int64_t ld) { return ld == 0 || ld >= c->D; };
  return c != nullptr && c->M >= 0 && c->D >= 1 && c->n_groups >= 1 && norm_ok(c->after) && norm_ok(c->before) &&
         ok_dtype(c->z_dtype) && ok_dtype(c->residual_dtype) && ok_dtype(c->y_dtype) && ok_dtype(c->h_dtype) &&
         std::isfinite(c->residual_scale) && c->eps >= 0.0f && std::isfinite(c->eps) && c->ldz >= c->D &&
         c->ldr >= c->D && c->ldy >= c->D && (c->before == ECHO_NORM_NONE || c->ldh >= c->D) && mod(c->ldgate) &&
         mod(c->ldscale) && mod(c->ldshift);
}

// ---- cross attention
constexpr int32_t kMaxStates = INT32_MAX - 127;  // 2^31 - 128: two tiles of 64 short of overflow
bool strides_ok(const echo_strides& s, int per16) {
  return s.batch >= 0 && s.row >= 0 && s.head >= 0 && s.batch % per16 == 0 && s.row % per16 == 0 &&
         s.head % per16 == 0;
}
bool cross_cfg_ok(const echo_cross_attention_cfg* c) {
  if (c == nullptr || c->B < 0 || c->Lq < 0 || c->Lk < 0 || c->H < 1 || c->Hkv < 1 || c->H % c->Hkv != 0 ||
      c->dh < 1 || !ok_dtype(c->dtype) || !std::isfinite(c->scale) || !(c->scale > 0.0f))
    return false;
  const int per16 = c->dtype == ECHO_BF16 ? 8 : 4;
  return strides_ok(c->q, per16) && strides_ok(c->k, per16) && strides_ok(c->v, per16) && strides_ok(c->out, per16);
}
bool cross_supported(const echo_cross_attention_cfg* c) {
  if (c->dtype == ECHO_BF16 ? (c->dh != 64 && c->dh != 128) : (c->dh % 4 != 0 || c->dh > 128)) return false;
  if (!std::isfinite(c->scale * 1.4426950408889634f)) return false;  // the scale in units of log2
  // a tile of states is addressed by 32-bit offsets
  if (c->k.row >= (int64_t(1) << 24) || c->v.row >= (int64_t(1) << 24)) return false;
  // states are numbered in 32 bits, up to the end of the tile after the last one
  if (c->Lk > kMaxStates) return false;
  const int64_t rows = int64_t(c->H / c->Hkv) * c->Lq, groups = int64_t(c->B) * c->Hkv;
  return rows < (int64_t(1) << 31) - 128 && groups < kMaxGroups && groups * ((rows + 127) / 128) < kMaxGroups;
}
CrossArgs cross_args(const echo_cross_attention_cfg* c) {
  CrossArgs a{};
  a.qb = c->q.batch; a.qr = c->q.row; a.qh = c->q.head;
  a.kb = c->k.batch; a.kr = c->k.row; a.kh = c->k.head;
  a.vb = c->v.batch; a.vr = c->v.row; a.vh = c->v.head;
  a.ob = c->out.batch; a.orow = c->out.row; a.oh = c->out.head;
  a.B = c->B; a.Lq = c->Lq; a.Lk = c->Lk; a.H = c->H; a.Hkv = c->Hkv; a.dh = c->dh;
  a.scale_log2 = static_cast<float>(c->scale * 1.4426950408889634);
  return a;
}
}  // namespace

extern "C" {

const char* echo_status_str(int status) {
  switch (status) {
    case ECHO_OK: return "ok";
    case ECHO_EINVAL: return "invalid argument";
    case ECHO_EUNSUPPORTED: return "unsupported shape or dtype";
    case ECHO_EWORKSPACE: return "workspace missing or too small";
    case ECHO_EDEVICE: return "HIP device error";
    case ECHO_ELIMIT: return "size above the allocation-free limit";
    default: return "unknown status";
  }
}

int echo_last_hip_error(void) { return g_last_hip_error; }

const char* echo_version(void) { return "0.1.0"; }

size_t echo_energy_workspace(const echo_energy_cfg* cfg, int64_t n_samples) {
  if (!energy_cfg_ok(cfg, n_samples)) return 0;
  return energy_ws(cfg, n_samples);
}

int echo_energy(const echo_energy_cfg* cfg, const float* audio, int64_t n_samples, float* band_energy,
                float* frame_energy, float* frame_weight, void* workspace, size_t workspace_bytes,
                void* stream) {
  if (!energy_cfg_ok(cfg, n_samples)) return ECHO_EINVAL;
  if (!ok_ptr(audio) || !ok_ptr(band_energy) || !ok_ptr(frame_energy) || !ok_ptr(frame_weight))
    return ECHO_EINVAL;
  const size_t need = energy_ws(cfg, n_samples);
  if (!ok_ptr(workspace) || workspace_bytes < need) return ECHO_EWORKSPACE;
  const int mf = energy_max_frames(n_samples, cfg->T, cfg->n_fft, cfg->hop);
  double* part = static_cast<double*>(workspace);
  double* e_scr = reinterpret_cast<double*>(
      static_cast<char*>(workspace) +
      align_up(sizeof(double) * static_cast<size_t>(cfg->T) * mf * cfg->n_bands));
  return device_status(launch_energy(audio, n_samples, cfg->T, cfg->sample_rate, cfg->n_fft, cfg->hop,
                                     cfg->n_bands, band_energy, frame_energy, frame_weight, part,
                                     e_scr, static_cast<hipStream_t>(stream)));
}

size_t echo_select_workspace(const echo_select_cfg* cfg) {
  if (!select_cfg_ok(cfg)) return 0;
  return select_ws(cfg);
}

int echo_select(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                int32_t* idx, uint8_t* mask, int32_t* n_sel, float* saliency, double* step_delta,
                void* workspace, size_t workspace_bytes, void* stream) {
  const int bad = select_args_status(cfg, x, xref, frame_weight, idx, mask, n_sel, saliency, step_delta);
  if (bad != ECHO_OK) return bad;
  const size_t need = select_ws(cfg);
  if (!ok_ptr(workspace) || workspace_bytes < need) return ECHO_EWORKSPACE;
  return select_launch(cfg, x, xref, frame_weight, idx, mask, n_sel, saliency, step_delta, workspace, stream);
}

int echo_select_noalloc(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                        int32_t* idx, uint8_t* mask, int32_t* n_sel, float* saliency, double* step_delta,
                        void* stream) {
  const int bad = select_args_status(cfg, x, xref, frame_weight, idx, mask, n_sel, saliency, step_delta);
  if (bad != ECHO_OK) return bad;
  if (static_cast<int64_t>(cfg->T) * cfg->N > ECHO_SELECT_NOALLOC_MAX_TOKENS) return ECHO_ELIMIT;
  void* ws = nullptr;
  const int st = noalloc_scratch(&ws);
  if (st != ECHO_OK) return st;
  return select_launch(cfg, x, xref, frame_weight, idx, mask, n_sel, saliency, step_delta, ws, stream);
}

}  // extern "C"

namespace {
int select_launch(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                  int32_t* idx, uint8_t* mask, int32_t* n_sel, float* saliency, double* step_delta,
                  void* workspace, void* stream) {
  const int L = cfg->T * cfg->N;
  char* ws = static_cast<char*>(workspace);
  float* s_ws = reinterpret_cast<float*>(ws);
  double* num = reinterpret_cast<double*>(ws + align_up(L * sizeof(float)));
  double* den = reinterpret_cast<double*>(ws + align_up(L * sizeof(float)) + align_up(L * sizeof(double)));
  float* s = saliency ? saliency : s_ws;
  const int threshold_mode = cfg->k < 0 ? 1 : 0;
  return device_status(launch_select(cfg->dtype == ECHO_BF16, x, xref, frame_weight, L, cfg->N, cfg->D,
                                     cfg->xi, threshold_mode ? 0 : cfg->k, threshold_mode,
                                     cfg->threshold, s, num, den, idx, mask, n_sel, step_delta,
                                     static_cast<hipStream_t>(stream)));
}
}  // namespace

extern "C" {

size_t echo_saliency_workspace(const echo_select_cfg* cfg) {
  if (!select_cfg_ok(cfg)) return 0;
  const size_t L = static_cast<size_t>(cfg->T) * cfg->N;
  return 2 * align_up(L * sizeof(double));
}

int echo_saliency(const echo_select_cfg* cfg, const void* x, const void* xref, const float* frame_weight,
                  float* saliency, double* step_delta, void* workspace, size_t workspace_bytes, void* stream) {
  if (!select_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!ok_ptr(x) || !ok_ptr(xref) || !ok_ptr(frame_weight) || !ok_ptr(saliency)) return ECHO_EINVAL;
  if (step_delta != nullptr && (reinterpret_cast<uintptr_t>(step_delta) & 7u)) return ECHO_EINVAL;
  const size_t need = echo_saliency_workspace(cfg);
  if (!ok_ptr(workspace) || workspace_bytes < need) return ECHO_EWORKSPACE;
  const int L = cfg->T * cfg->N;
  double* num = static_cast<double*>(workspace);
  double* den = reinterpret_cast<double*>(static_cast<char*>(workspace) + align_up(L * sizeof(double)));
  return device_status(launch_saliency(cfg->dtype == ECHO_BF16, x, xref, frame_weight, L, cfg->N, cfg->D,
                                       cfg->xi, saliency, num, den, step_delta,
                                       static_cast<hipStream_t>(stream)));
}

int echo_topk(const echo_select_cfg* cfg, const float* saliency, int32_t* idx, uint8_t* mask, int32_t* n_sel,
              void* stream) {
  if (!select_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!ok_ptr(saliency) || !ok_ptr(idx) || !ok_ptr(mask) || n_sel == nullptr) return ECHO_EINVAL;
  const int L = cfg->T * cfg->N;
  const int threshold_mode = cfg->k < 0 ? 1 : 0;
  return device_status(launch_topk(saliency, L, threshold_mode ? 0 : cfg->k, threshold_mode, cfg->threshold,
                                   idx, mask, n_sel, static_cast<hipStream_t>(stream)));
}

int echo_anchors(const float* keys, int32_t T, int32_t k, int32_t mode, uint8_t* anchors, void* stream) {
  if (T < 1 || T > max_anchor_segments() || k < 0 || k > T) return ECHO_EINVAL;
  if (mode != ECHO_ANCHOR_TOPK && mode != ECHO_ANCHOR_UNIFORM) return ECHO_EINVAL;
  if (anchors == nullptr || (mode == ECHO_ANCHOR_TOPK && !ok_ptr(keys))) return ECHO_EINVAL;
  return device_status(launch_anchors(keys, T, k, mode, anchors, static_cast<hipStream_t>(stream)));
}

int echo_topk_segments(const float* saliency, const uint8_t* anchors, int32_t T, int32_t N, int32_t k,
                       int32_t* idx, uint8_t* mask, int32_t* n_sel, void* stream) {
  if (T < 1 || T > 65535 || N < 1 || k < 0) return ECHO_EINVAL;
  if (static_cast<int64_t>(T) * N >= (int64_t(1) << 31)) return ECHO_EINVAL;
  if (!ok_ptr(saliency) || anchors == nullptr || !ok_ptr(idx) || !ok_ptr(mask) || n_sel == nullptr)
    return ECHO_EINVAL;
  return device_status(
      launch_topk_segments(saliency, anchors, T, N, k, idx, mask, n_sel, static_cast<hipStream_t>(stream)));
}

int32_t echo_topk_count(double ratio, int32_t L) {
  if (L < 1 || !(ratio >= 0.0 && ratio <= 1.0)) return -ECHO_EINVAL;
  const double kk = std::ceil(ratio * L - 1e-9);
  return kk < 0.0 ? 0 : (kk > L ? L : static_cast<int32_t>(kk));
}

int32_t echo_segments_count(int32_t n_anchors, int32_t N, int32_t k) {
  if (n_anchors < 0 || N < 1 || k < 0) return -ECHO_EINVAL;
  const int64_t n = static_cast<int64_t>(n_anchors) * (k < N ? k : N);
  return n >= (int64_t(1) << 31) ? -ECHO_EINVAL : static_cast<int32_t>(n);
}

int32_t echo_schedule_next(const echo_schedule_cfg* cfg, echo_schedule_state* st, double delta_t, int32_t L,
                           int32_t* full) {
  if (cfg == nullptr || st == nullptr || full == nullptr || L < 1 || cfg->n_full < 0 ||
      !(cfg->r_min >= 0.0) || !(cfg->r_max <= 1.0) || !(cfg->r_min <= cfg->r_max) || !std::isfinite(cfg->alpha) ||
      std::isnan(cfg->refresh_delta) || std::isnan(delta_t))
    return -ECHO_EINVAL;
  const int32_t step = st->step++;
  if (step < cfg->n_full) {
    st->delta_acc = 0.0;
    *full = 1;
    return L;
  }
  st->delta_acc += delta_t;
  if (cfg->refresh_delta > 0.0 && st->delta_acc > cfg->refresh_delta) {
    st->delta_acc = 0.0;
    *full = 1;
    return L;
  }
  st->delta_max = delta_t > st->delta_max ? delta_t : st->delta_max;
  const double dhat = st->delta_max > 0.0 ? delta_t / st->delta_max : 0.0;
  double r = cfg->r_min + cfg->alpha * dhat;
  r = r < cfg->r_min ? cfg->r_min : (r > cfg->r_max ? cfg->r_max : r);
  *full = 0;
  return echo_topk_count(r, L);
}

size_t echo_block_workspace(const echo_block_cfg* cfg, int32_t n_sel_max) {
  if (!block_cfg_ok(cfg) || n_sel_max < 0) return 0;
  return block_ws_layout(cfg, n_sel_max, nullptr).bytes;
}

int echo_block_partial(const echo_block_cfg* cfg, const echo_block_weights* w, const void* x,
                       const int32_t* idx, int32_t n_sel, float* y_sel, void* workspace,
                       size_t workspace_bytes, void* stream) {
  if (!block_cfg_ok(cfg) || !weights_ok(w) || n_sel < 0) return ECHO_EINVAL;
  if (!block_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (n_sel == 0) return ECHO_OK;
  if (cfg->dtype == ECHO_BF16 && int64_t(n_sel) * cfg->F >= (int64_t(1) << 30)) return ECHO_EUNSUPPORTED;
  if (!ok_ptr(x) || !ok_ptr(idx) || !ok_ptr(y_sel)) return ECHO_EINVAL;
  const size_t need = block_ws_layout(cfg, n_sel, nullptr).bytes;
  if (!ok_ptr(workspace) || workspace_bytes < need) return ECHO_EWORKSPACE;
  const BlockWs ws = block_ws_layout(cfg, n_sel, static_cast<char*>(workspace));
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int L = cfg->L, D = cfg->D, H = cfg->H, F = cfg->F, n = n_sel;
  const float* mod = w->mod;
  const bool bf = cfg->dtype == ECHO_BF16;
  hipError_t e = launch_modln_input(bf, x, L, D, mod + 0 * D, mod + 1 * D, cfg->ln_eps, ws.a, st);
  if (e != hipSuccess) return device_status(e);
  if (bf) {
    typedef const bf16_t* P;
    GemmBf16Args g{};
    // partial results of the split tails (none when every row must be batch-invariant)
    float* part = (cfg->flags & ECHO_BLOCK_BATCH_INVARIANT) ? nullptr : ws.part;
    auto with_part = [&](GemmBf16Args a) {
      a.part = part;
      a.part_bytes = ws.part_bytes;
      return a;
    };
    // q = a[idx] Wq^T + bq
    const GemmBf16Args gq{static_cast<P>(ws.a), D, idx, L, static_cast<P>(w->wq), static_cast<P>(w->wq), D, D,
                          static_cast<P>(w->bq), static_cast<P>(w->bq), n, D, D, ws.q, D,
                          nullptr, nullptr, 0, nullptr, 0};
    // [k | v] = a [Wk; Wv]^T + [bk; bv], one N = 2D GEMM over all L rows
    g = GemmBf16Args{static_cast<P>(ws.a), D, nullptr, L, static_cast<P>(w->wk), static_cast<P>(w->wv), D,
                     D, static_cast<P>(w->bk), static_cast<P>(w->bv), L, 2 * D, D, ws.kv, 2 * D,
                     nullptr, nullptr, 0, nullptr, 0};
    if ((e = launch_gemm_bf16_pair("gemm_qkv_bf16", "gemm_q_bf16", "gemm_kv_bf16", with_part(gq), with_part(g), st)) !=
        hipSuccess)
      return device_status(e);
    const bf16_t* kvp = static_cast<const bf16_t*>(ws.kv);
    if ((e = launch_attn_bf16(static_cast<P>(ws.q), D, kvp, kvp + D, 2 * D, n, L, H,
                              static_cast<bf16_t*>(ws.o), D,
                              part, ws.part_bytes, st)) !=
        hipSuccess)
      return device_status(e);
    // x1 = x[idx] + gate1 * (o Wo^T + bo)
    g = GemmBf16Args{static_cast<P>(ws.o), D, nullptr, n, static_cast<P>(w->wo), static_cast<P>(w->wo), D,
                     D, static_cast<P>(w->bo), static_cast<P>(w->bo), n, D, D, ws.x1, D,
                     mod + 2 * D, x, D, idx, 1};
    if ((e = launch_gemm_bf16("gemm_o_bf16", 2, with_part(g), st)) != hipSuccess) return device_status(e);
    if ((e = launch_modln_x1(1, ws.x1, n, D, mod + 3 * D, mod + 4 * D, cfg->ln_eps, ws.b, st)) !=
        hipSuccess)
      return device_status(e);
    // h = GELU(b W1^T + b1)
    g = GemmBf16Args{static_cast<P>(ws.b), D, nullptr, n, static_cast<P>(w->w1), static_cast<P>(w->w1), F,
                     D, static_cast<P>(w->b1), static_cast<P>(w->b1), n, F, D, ws.h, F,
                     nullptr, nullptr, 0, nullptr, 0};
    if ((e = launch_gemm_bf16("gemm_ffn_up_bf16", 1, with_part(g), st)) != hipSuccess) return device_status(e);
    // y_sel = x1 + gate2 * (h W2^T + b2)
    g = GemmBf16Args{static_cast<P>(ws.h), F, nullptr, n, static_cast<P>(w->w2), static_cast<P>(w->w2), D,
                     F, static_cast<P>(w->b2), static_cast<P>(w->b2), n, D, F, y_sel, D,
                     mod + 5 * D, ws.x1, D, nullptr, 0};
    if ((e = launch_gemm_bf16("gemm_ffn_down_bf16", 2, with_part(g), st)) != hipSuccess) return device_status(e);
    return ECHO_OK;
  }
  typedef const float* P;
  const int dh = D / H;
  const GemmF32Args gq{static_cast<P>(ws.a), D, idx, static_cast<P>(w->wq), static_cast<P>(w->wq), D, D,
                  static_cast<P>(w->bq), static_cast<P>(w->bq), n, D, D, static_cast<float*>(ws.q), D,
                  nullptr, nullptr, 0, nullptr};
  GemmF32Args g{static_cast<P>(ws.a), D, nullptr, static_cast<P>(w->wk), static_cast<P>(w->wv), D, D,
                  static_cast<P>(w->bk), static_cast<P>(w->bv), L, 2 * D, D,
                  static_cast<float*>(ws.kv), 2 * D, nullptr, nullptr, 0, nullptr};
  if ((e = launch_gemm_f32_pair("gemm_qkv_f32", gq, g, st)) != hipSuccess) return device_status(e);
  const float* kvp = static_cast<const float*>(ws.kv);
  if ((e = launch_attn_f32(static_cast<P>(ws.q), D, kvp, kvp + D, 2 * D, n, L, H, dh,
                           static_cast<float*>(ws.o), D, st)) != hipSuccess)
    return device_status(e);
  g = GemmF32Args{static_cast<P>(ws.o), D, nullptr, static_cast<P>(w->wo), static_cast<P>(w->wo), D, D,
                  static_cast<P>(w->bo), static_cast<P>(w->bo), n, D, D, ws.x1, D, mod + 2 * D,
                  static_cast<P>(x), D, idx};
  if ((e = launch_gemm_f32("gemm_o_f32", 2, g, st)) != hipSuccess) return device_status(e);
  if ((e = launch_modln_x1(0, ws.x1, n, D, mod + 3 * D, mod + 4 * D, cfg->ln_eps, ws.b, st)) !=
      hipSuccess)
    return device_status(e);
  g = GemmF32Args{static_cast<P>(ws.b), D, nullptr, static_cast<P>(w->w1), static_cast<P>(w->w1), F, D,
                  static_cast<P>(w->b1), static_cast<P>(w->b1), n, F, D, static_cast<float*>(ws.h), F,
                  nullptr, nullptr, 0, nullptr};
  if ((e = launch_gemm_f32("gemm_ffn_up_f32", 1, g, st)) != hipSuccess) return device_status(e);
  g = GemmF32Args{static_cast<P>(ws.h), F, nullptr, static_cast<P>(w->w2), static_cast<P>(w->w2), D, F,
                  static_cast<P>(w->b2), static_cast<P>(w->b2), n, D, F, y_sel, D, mod + 5 * D, ws.x1,
                  D, nullptr};
  if ((e = launch_gemm_f32("gemm_ffn_down_f32", 2, g, st)) != hipSuccess) return device_status(e);
  return ECHO_OK;
}


size_t echo_wan_block_workspace(const echo_wan_block_cfg* cfg, int32_t n_total_max) {
  if (!wan_cfg_ok(cfg) || n_total_max < 0) return 0;
  return wan_ws_layout(cfg, n_total_max, nullptr).bytes;
}

int echo_wan_block_partial(const echo_wan_block_cfg* cfg, const echo_wan_block_weights* w, const void* x,
                           const void* ctx, const int32_t* idx, const int32_t* n_sel, float* y_sel,
                           void* workspace, size_t workspace_bytes, void* stream) {
  if (!wan_cfg_ok(cfg) || !wan_weights_ok(w) || n_sel == nullptr) return ECHO_EINVAL;
  int64_t tot = 0;
  for (int b = 0; b < cfg->B; ++b) {
    if (n_sel[b] < 0 || n_sel[b] > cfg->L) return ECHO_EINVAL;
    tot += n_sel[b];
  }
  if (!wan_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (tot == 0) return ECHO_OK;
  if (tot * cfg->F >= (int64_t(1) << 30)) return ECHO_EUNSUPPORTED;
  if (!ok_ptr(x) || !ok_ptr(ctx) || !ok_ptr(idx) || !ok_ptr(y_sel)) return ECHO_EINVAL;
  const size_t need = wan_ws_layout(cfg, tot, nullptr).bytes;
  if (!ok_ptr(workspace) || workspace_bytes < need) return ECHO_EWORKSPACE;
  const WanWs ws = wan_ws_layout(cfg, tot, static_cast<char*>(workspace));
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int B = cfg->B, L = cfg->L, D = cfg->D, H = cfg->H, F = cfg->F, Lc = cfg->Lc, n = static_cast<int>(tot);
  const int BL = B * L, BLc = B * Lc, dh = D / H;
  const float* mod = w->self.mod;
  typedef const bf16_t* P;
  float* part = (cfg->flags & ECHO_BLOCK_BATCH_INVARIANT) ? nullptr : ws.part;
  auto with_part = [&](GemmBf16Args a) {
    a.part = part;
    a.part_bytes = ws.part_bytes;
    return a;
  };
  hipError_t e;
#define ECHO_TRY(call)                              \
  if ((e = (call)) != hipSuccess) return device_status(e);
  // constants: rotary table, the unit gate of the cross-attention output, g3 - 1
  ECHO_TRY(launch_wan_constants(cfg->T, cfg->gh, cfg->gw, dh, cfg->rope_base, ws.tab, w->g3, ws.ones, ws.g3m1, D, st));
  // self-attention
  ECHO_TRY(launch_modln_input(1, x, BL, D, mod + 0 * D, mod + 1 * D, cfg->ln_eps, ws.a, st));
  const GemmBf16Args gq{static_cast<P>(ws.a), D, idx, BL, static_cast<P>(w->self.wq), static_cast<P>(w->self.wq), D, D,
                        static_cast<P>(w->self.bq), static_cast<P>(w->self.bq), n, D, D, ws.q, D,
                        nullptr, nullptr, 0, nullptr, 0};
  GemmBf16Args g{static_cast<P>(ws.a), D, nullptr, BL, static_cast<P>(w->self.wk), static_cast<P>(w->self.wv), D,
                   D, static_cast<P>(w->self.bk), static_cast<P>(w->self.bv), BL, 2 * D, D, ws.kv, 2 * D,
                   nullptr, nullptr, 0, nullptr, 0};
  ECHO_TRY(launch_gemm_bf16_pair("gemm_qkv_bf16", "gemm_q_bf16", "gemm_kv_bf16", with_part(gq), with_part(g), st));
  ECHO_TRY(launch_qk_norm_rope(QkRows{static_cast<bf16_t*>(ws.q), D, n, w->gq, idx},
                               QkRows{static_cast<bf16_t*>(ws.kv), 2 * D, BL, w->gk, nullptr}, D, cfg->rms_eps,
                               ws.tab, L, cfg->T, cfg->gh, cfg->gw, dh, st));
  {
    const bf16_t* kvp = static_cast<const bf16_t*>(ws.kv);
    int64_t o = 0;
    for (int b = 0; b < B; ++b) {
      const bf16_t* kb = kvp + int64_t(b) * L * 2 * D;
      ECHO_TRY(launch_attn_bf16(static_cast<P>(ws.q) + o * D, D, kb, kb + D, 2 * D, n_sel[b], L, H,
                                static_cast<bf16_t*>(ws.o) + o * D, D, part, ws.part_bytes, st));
      o += n_sel[b];
    }
  }
  g = GemmBf16Args{static_cast<P>(ws.o), D, nullptr, n, static_cast<P>(w->self.wo), static_cast<P>(w->self.wo), D,
                   D, static_cast<P>(w->self.bo), static_cast<P>(w->self.bo), n, D, D, ws.x1, D,
                   mod + 2 * D, x, D, idx, 1};
  ECHO_TRY(launch_gemm_bf16("gemm_o_bf16", 2, with_part(g), st));
  // cross-attention: c = LN(x1) * g3 + b3 = LN(x1) * (1 + (g3 - 1)) + b3
  ECHO_TRY(launch_modln_x1(1, ws.x1, n, D, w->b3, ws.g3m1, cfg->ln_eps, ws.b, st));
  const GemmBf16Args gqc{static_cast<P>(ws.b), D, nullptr, n, static_cast<P>(w->wqc), static_cast<P>(w->wqc), D, D,
                         static_cast<P>(w->bqc), static_cast<P>(w->bqc), n, D, D, ws.q, D,
                         nullptr, nullptr, 0, nullptr, 0};
  g = GemmBf16Args{static_cast<P>(ctx), D, nullptr, BLc, static_cast<P>(w->wkc), static_cast<P>(w->wvc), D, D,
                   static_cast<P>(w->bkc), static_cast<P>(w->bvc), BLc, 2 * D, D, ws.kvc, 2 * D,
                   nullptr, nullptr, 0, nullptr, 0};
  ECHO_TRY(launch_gemm_bf16_pair("gemm_qkvc_bf16", "gemm_qc_bf16", "gemm_kvc_bf16", with_part(gqc), with_part(g), st));
  ECHO_TRY(launch_qk_norm_rope(QkRows{static_cast<bf16_t*>(ws.q), D, n, w->gqc, nullptr},
                               QkRows{static_cast<bf16_t*>(ws.kvc), 2 * D, BLc, w->gkc, nullptr}, D, cfg->rms_eps,
                               nullptr, L, cfg->T, cfg->gh, cfg->gw, dh, st));
  {
    const bf16_t* kvp = static_cast<const bf16_t*>(ws.kvc);
    int64_t o = 0;
    for (int b = 0; b < B; ++b) {
      const bf16_t* kb = kvp + int64_t(b) * Lc * 2 * D;
      ECHO_TRY(launch_attn_bf16(static_cast<P>(ws.q) + o * D, D, kb, kb + D, 2 * D, n_sel[b], Lc, H,
                                static_cast<bf16_t*>(ws.o) + o * D, D, part, ws.part_bytes, st,
                                true));
      o += n_sel[b];
    }
  }
  // x2 = x1 + 1 * (oc Woc^T + boc)
  g = GemmBf16Args{static_cast<P>(ws.o), D, nullptr, n, static_cast<P>(w->woc), static_cast<P>(w->woc), D, D,
                   static_cast<P>(w->boc), static_cast<P>(w->boc), n, D, D, ws.x2, D,
                   ws.ones, ws.x1, D, nullptr, 0};
  ECHO_TRY(launch_gemm_bf16("gemm_oc_bf16", 2, with_part(g), st));
  // FFN
  ECHO_TRY(launch_modln_x1(1, ws.x2, n, D, mod + 3 * D, mod + 4 * D, cfg->ln_eps, ws.b, st));
  g = GemmBf16Args{static_cast<P>(ws.b), D, nullptr, n, static_cast<P>(w->self.w1), static_cast<P>(w->self.w1), F,
                   D, static_cast<P>(w->self.b1), static_cast<P>(w->self.b1), n, F, D, ws.h, F,
                   nullptr, nullptr, 0, nullptr, 0};
  ECHO_TRY(launch_gemm_bf16("gemm_ffn_up_bf16", 1, with_part(g), st));
  g = GemmBf16Args{static_cast<P>(ws.h), F, nullptr, n, static_cast<P>(w->self.w2), static_cast<P>(w->self.w2), D,
                   F, static_cast<P>(w->self.b2), static_cast<P>(w->self.b2), n, D, F, y_sel, D,
                   mod + 5 * D, ws.x2, D, nullptr, 0};
  ECHO_TRY(launch_gemm_bf16("gemm_ffn_down_bf16", 2, with_part(g), st));
#undef ECHO_TRY
  return ECHO_OK;
}

int echo_cache_update(const echo_cache_cfg* cfg, const void* x, const int32_t* idx, const uint8_t* mask,
                      int32_t n_sel, const float* y_sel, void* xref, int8_t* codes, float* scale,
                      void* y, void* stream) {
  if (cfg == nullptr || cfg->L < 1 || cfg->D < 8 || (cfg->D % 8) != 0 || cfg->D > 16384 ||
      !ok_dtype(cfg->dtype))
    return ECHO_EINVAL;
  if (n_sel < 0 || n_sel > cfg->L) return ECHO_EINVAL;
  if (!ok_ptr(x) || !ok_ptr(mask) || !ok_ptr(xref) || !ok_ptr(codes) || !ok_ptr(scale) || !ok_ptr(y))
    return ECHO_EINVAL;
  if (n_sel > 0 && (!ok_ptr(idx) || !ok_ptr(y_sel))) return ECHO_EINVAL;
  return device_status(launch_cache_update(cfg->dtype == ECHO_BF16, x, idx, mask, n_sel, cfg->L, cfg->D,
                                           y_sel, xref, codes, scale, y,
                                           static_cast<hipStream_t>(stream)));
}

int echo_cache_update_codec(const echo_cache_cfg* cfg, int32_t codec, const void* x, const int32_t* idx,
                            const uint8_t* mask, int32_t n_sel, const float* y_sel, void* xref, void* store,
                            int8_t* codes, float* scale, void* y, void* stream) {
  if (cfg == nullptr || cfg->L < 1 || cfg->D < 8 || (cfg->D % 8) != 0 || cfg->D > 16384 ||
      !ok_dtype(cfg->dtype))
    return ECHO_EINVAL;
  if (codec != ECHO_CODEC_RESIDUAL_INT8 && codec != ECHO_CODEC_FULL && codec != ECHO_CODEC_NAIVE_INT8)
    return ECHO_EINVAL;
  if (n_sel < 0 || n_sel > cfg->L) return ECHO_EINVAL;
  if (!ok_ptr(x) || !ok_ptr(mask) || !ok_ptr(xref) || !ok_ptr(y)) return ECHO_EINVAL;
  if (codec == ECHO_CODEC_FULL ? !ok_ptr(store) : (!ok_ptr(codes) || !ok_ptr(scale))) return ECHO_EINVAL;
  if (n_sel > 0 && (!ok_ptr(idx) || !ok_ptr(y_sel))) return ECHO_EINVAL;
  return device_status(launch_cache_codec(cfg->dtype == ECHO_BF16, codec, x, idx, mask, n_sel, cfg->L, cfg->D,
                                          y_sel, xref, store, codes, scale, y, static_cast<hipStream_t>(stream)));
}


int echo_refcache_init(const echo_refcache_cfg* cfg, const echo_refcache_state* st, void* stream) {
  if (!refcache_cfg_ok(cfg) || !refcache_state_ok(st)) return ECHO_EINVAL;
  return device_status(launch_refcache_init(cfg->L, cfg->L / cfg->chain_len, cfg->capacity, st->refcount,
                                            st->free_list, st->free_top, st->chain_ref, st->ent_slot,
                                            st->ent_kind, st->scale, static_cast<hipStream_t>(stream)));
}

int echo_refcache_update(const echo_refcache_cfg* cfg, const echo_refcache_state* st, const void* x,
                         const int32_t* idx, const uint8_t* mask, int32_t n_sel, const float* y_sel,
                         void* xref, void* y, void* stream) {
  if (!refcache_cfg_ok(cfg) || !refcache_state_ok(st)) return ECHO_EINVAL;
  if (n_sel < 0 || n_sel > cfg->L) return ECHO_EINVAL;
  if (!ok_ptr(x) || !ok_ptr(mask) || !ok_ptr(xref) || !ok_ptr(y)) return ECHO_EINVAL;
  if (n_sel > 0 && (!ok_ptr(idx) || !ok_ptr(y_sel))) return ECHO_EINVAL;
  return device_status(launch_refcache_update(
      cfg->dtype == ECHO_BF16, x, idx, mask, n_sel, cfg->L, cfg->D, cfg->chain_len, cfg->tau, y_sel, st->pool,
      st->refcount, st->free_list, st->free_top, st->chain_ref, st->ent_slot, st->ent_kind, st->codes,
      st->scale, xref, y, static_cast<hipStream_t>(stream)));
}

int64_t echo_int8_pitch(int32_t D) { return D < 1 || D > 65536 ? 0 : (int64_t(D) + 127) / 128 * 128; }

int echo_quantize_rows(const echo_quantize_cfg* cfg, const void* x, const int32_t* rows, const float* shift,
                       const float* scale, int8_t* codes, float* row_scale, void* stream) {
  if (!quantize_cfg_ok(cfg) || (shift == nullptr) != (scale == nullptr)) return ECHO_EINVAL;
  if (cfg->M == 0) return ECHO_OK;
  if (!elem_aligned(x, esize(cfg->dtype)) || !ok_ptr(codes) || !elem_aligned(row_scale, 4) ||
      (rows != nullptr ? !elem_aligned(rows, 4) || cfg->x_rows < 1 : cfg->x_rows < cfg->M) ||
      (shift != nullptr && (!ok_ptr(shift) || !ok_ptr(scale))))
    return ECHO_EINVAL;
  const QuantizeArgs a{x,    cfg->ldx, rows,  cfg->x_rows, cfg->M, cfg->D, shift, scale, cfg->ln_eps,
                       codes, cfg->ldq, row_scale, nullptr, 0};
  return device_status(launch_quantize_rows(cfg->dtype == ECHO_BF16, a, static_cast<hipStream_t>(stream)));
}

int echo_dequantize_rows(const echo_quantize_cfg* cfg, const int8_t* codes, const float* row_scale, void* x,
                         void* stream) {
  if (!quantize_cfg_ok(cfg)) return ECHO_EINVAL;
  if (cfg->M == 0) return ECHO_OK;
  if (!ok_ptr(codes) || !elem_aligned(row_scale, 4) || !elem_aligned(x, esize(cfg->dtype))) return ECHO_EINVAL;
  const DequantizeArgs a{codes, cfg->ldq, row_scale, cfg->M, cfg->D, x, cfg->ldx, nullptr, 0};
  return device_status(launch_dequantize_rows(cfg->dtype == ECHO_BF16, a, static_cast<hipStream_t>(stream)));
}

size_t echo_linear_int8_workspace(const echo_linear_int8_cfg* cfg) {
  if (!linear_cfg_ok(cfg) || !linear_supported(cfg) || cfg->M == 0) return 0;
  return gemm_i8_partial_bytes(cfg->M, cfg->N, static_cast<int>(echo_int8_pitch(cfg->K)));
}

int echo_linear_int8(const echo_linear_int8_cfg* cfg, const int8_t* a, const float* a_scale, const int8_t* w,
                     const float* w_scale, const void* bias, const float* gate, const void* residual,
                     const int32_t* residual_rows, void* c, void* workspace, size_t workspace_bytes, void* stream) {
  if (!linear_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!linear_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (cfg->M == 0) return ECHO_OK;
  const bool gated = cfg->epilogue == ECHO_LINEAR_GATE_RESIDUAL;
  if (!ok_ptr(a) || !elem_aligned(a_scale, 4) || !ok_ptr(w) || !elem_aligned(w_scale, 4) || !elem_aligned(c, esize(cfg->out_dtype)) ||
      (bias != nullptr && !elem_aligned(bias, esize(cfg->bias_dtype))))
    return ECHO_EINVAL;
  if (gated ? (!elem_aligned(gate, 4) || !elem_aligned(residual, esize(cfg->residual_dtype)) ||
               (residual_rows != nullptr ? !elem_aligned(residual_rows, 4) || cfg->residual_nrows < 1
                                         : cfg->residual_nrows < cfg->M))
            : (gate != nullptr || residual != nullptr || residual_rows != nullptr))
    return ECHO_EINVAL;
  const size_t need = echo_linear_int8_workspace(cfg);
  if (need > 0 && (!ok_ptr(workspace) || workspace_bytes < need)) return ECHO_EWORKSPACE;
  GemmI8Args g{};
  g.A = a; g.lda = cfg->lda; g.sa = a_scale;
  g.B = w; g.ldb = cfg->ldw; g.sb = w_scale;
  g.M = cfg->M; g.N = cfg->N; g.K = static_cast<int>(echo_int8_pitch(cfg->K));
  g.bias = bias; g.bias_bf16 = cfg->bias_dtype == ECHO_BF16;
  g.C = c; g.c_bf16 = cfg->out_dtype == ECHO_BF16; g.ldc = cfg->ldc;
  g.gate = gate; g.res = residual; g.res_bf16 = cfg->residual_dtype == ECHO_BF16; g.ldr = cfg->ldr;
  g.res_rows = residual_rows; g.res_nrows = cfg->residual_nrows;
  g.part = static_cast<int32_t*>(workspace); g.part_bytes = workspace_bytes;
  return device_status(launch_gemm_i8(cfg->epilogue, g, static_cast<hipStream_t>(stream)));
}

int64_t echo_fp4_pitch(int32_t D) { return D < 1 || D > 65536 ? 0 : (int64_t(D) + 255) / 256 * 128; }
int64_t echo_fp4_scale_pitch(int32_t D) { return D < 1 || D > 65536 ? 0 : (int64_t(D) + 511) / 512 * 16; }

int echo_quantize_rows_fp4(const echo_quantize_fp4_cfg* cfg, const void* x, const int32_t* rows, const float* shift,
                           const float* scale, uint8_t* codes, uint8_t* scales, void* stream) {
  if (!quantize_fp4_cfg_ok(cfg) || (shift == nullptr) != (scale == nullptr)) return ECHO_EINVAL;
  if (cfg->M == 0) return ECHO_OK;
  if (!elem_aligned(x, esize(cfg->dtype)) || !ok_ptr(codes) || !ok_ptr(scales) ||
      (rows != nullptr ? !elem_aligned(rows, 4) || cfg->x_rows < 1 : cfg->x_rows < cfg->M) ||
      (shift != nullptr && (!elem_aligned(shift, 4) || !elem_aligned(scale, 4))))
    return ECHO_EINVAL;
  QuantizeArgs a{};
  a.x = x; a.ldx = cfg->ldx; a.rows = rows; a.x_rows = cfg->x_rows; a.M = cfg->M; a.D = cfg->D;
  a.shift = shift; a.scale = scale; a.ln_eps = cfg->ln_eps;
  a.codes = reinterpret_cast<int8_t*>(codes); a.ldq = cfg->ldq;
  a.scales = scales; a.lds = cfg->lds;
  return device_status(launch_quantize_rows_fp4(cfg->dtype == ECHO_BF16, a, static_cast<hipStream_t>(stream)));
}

int echo_dequantize_rows_fp4(const echo_quantize_fp4_cfg* cfg, const uint8_t* codes, const uint8_t* scales, void* x,
                             void* stream) {
  if (!quantize_fp4_cfg_ok(cfg)) return ECHO_EINVAL;
  if (cfg->M == 0) return ECHO_OK;
  if (!ok_ptr(codes) || !ok_ptr(scales) || !elem_aligned(x, esize(cfg->dtype))) return ECHO_EINVAL;
  DequantizeArgs a{};
  a.codes = reinterpret_cast<const int8_t*>(codes); a.ldq = cfg->ldq;
  a.scales = scales; a.lds = cfg->lds;
  a.M = cfg->M; a.D = cfg->D; a.y = x; a.ldy = cfg->ldx;
  return device_status(launch_dequantize_rows_fp4(cfg->dtype == ECHO_BF16, a, static_cast<hipStream_t>(stream)));
}

size_t echo_linear_fp4_workspace(const echo_linear_fp4_cfg* cfg) {
  if (!linear_fp4_cfg_ok(cfg) || !linear_fp4_supported(cfg) || cfg->M == 0) return 0;
  return gemm_fp4_partial_bytes(cfg->M, cfg->N, static_cast<int>(echo_fp4_pitch(cfg->K)), cfg->epilogue);
}

int echo_linear_fp4(const echo_linear_fp4_cfg* cfg, const uint8_t* a, const uint8_t* a_scales, const uint8_t* w,
                    const uint8_t* w_scales, const void* bias, const float* gate, const void* residual,
                    const int32_t* residual_rows, void* c, void* workspace, size_t workspace_bytes, void* stream) {
  if (!linear_fp4_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!linear_fp4_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (cfg->M == 0) return ECHO_OK;
  const bool gated = cfg->epilogue == ECHO_LINEAR_GATE_RESIDUAL;
  if (!ok_ptr(a) || !ok_ptr(a_scales) || !ok_ptr(w) || !ok_ptr(w_scales) || !elem_aligned(c, esize(cfg->out_dtype)) ||
      (bias != nullptr && !elem_aligned(bias, esize(cfg->bias_dtype))))
    return ECHO_EINVAL;
  if (gated ? (!elem_aligned(gate, 4) || !elem_aligned(residual, esize(cfg->residual_dtype)) ||
               (residual_rows != nullptr ? !elem_aligned(residual_rows, 4) || cfg->residual_nrows < 1
                                         : cfg->residual_nrows < cfg->M))
            : (gate != nullptr || residual != nullptr || residual_rows != nullptr))
    return ECHO_EINVAL;
  const size_t need = echo_linear_fp4_workspace(cfg);
  if (need > 0 && (!ok_ptr(workspace) || workspace_bytes < need)) return ECHO_EWORKSPACE;
  GemmFp4Args g{};
  g.A = a; g.lda = cfg->lda; g.sa = a_scales; g.ldsa = cfg->ldsa;
  g.B = w; g.ldb = cfg->ldw; g.sb = w_scales; g.ldsb = cfg->ldsw;
  g.M = cfg->M; g.N = cfg->N; g.K = static_cast<int>(echo_fp4_pitch(cfg->K));
  g.bias = bias; g.bias_bf16 = cfg->bias_dtype == ECHO_BF16;
  g.C = c; g.c_bf16 = cfg->out_dtype == ECHO_BF16; g.ldc = cfg->ldc;
  g.gate = gate; g.res = residual; g.res_bf16 = cfg->residual_dtype == ECHO_BF16; g.ldr = cfg->ldr;
  g.res_rows = residual_rows; g.res_nrows = cfg->residual_nrows;
  g.part = static_cast<float*>(workspace); g.part_bytes = workspace_bytes;
  return device_status(launch_gemm_fp4(cfg->epilogue, g, static_cast<hipStream_t>(stream)));
}

int echo_rotary(const echo_rotary_cfg* cfg, const void* q, const void* k, const int32_t* positions, const double* freq,
                void* q_out, void* k_out, void* stream) {
  if (!rotary_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!rotary_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (cfg->B == 0 || cfg->L == 0) return ECHO_OK;
  const size_t es = esize(cfg->dtype);
  const bool keys = cfg->Hk > 0;
  if (!elem_aligned(q, es) || !elem_aligned(q_out, es) || !elem_aligned(freq, 8) ||
      (positions != nullptr && !elem_aligned(positions, 4)) ||
      (keys && (!elem_aligned(k, es) || !elem_aligned(k_out, es))) ||
      !rows_apart(cfg->q_out, cfg->B, cfg->L, cfg->H) || (keys && !rows_apart(cfg->k_out, cfg->B, cfg->L, cfg->Hk)) ||
      (q == q_out && !same_strides(cfg->q, cfg->q_out)) ||
      (keys && k == k_out && !same_strides(cfg->k, cfg->k_out)))
    return ECHO_EINVAL;
  RotaryArgs a{};
  auto st = [](const echo_strides& s, int64_t& b, int64_t& r, int64_t& h) { b = s.batch, r = s.row, h = s.head; };
  a.q = q; a.qo = q_out;
  st(cfg->q, a.qb, a.qr, a.qh);
  st(cfg->q_out, a.qob, a.qor, a.qoh);
  if (keys) {
    a.k = k; a.ko = k_out;
    st(cfg->k, a.kb, a.kr, a.kh);
    st(cfg->k_out, a.kob, a.kor, a.koh);
  }
  a.B = cfg->B; a.L = cfg->L; a.H = cfg->H; a.Hk = cfg->Hk; a.dh = cfg->dh; a.dims = cfg->dims;
  a.half = cfg->layout == ECHO_ROTARY_HALF;
  a.grid_h = cfg->grid_h; a.grid_w = cfg->grid_w; a.pairs_t = cfg->pairs_t; a.pairs_r = cfg->pairs_r;
  a.magnitude = cfg->magnitude;
  a.positions = positions; a.pos_batch = cfg->pos_batch; a.freq = freq;
  return device_status(launch_rotary(cfg->dtype == ECHO_BF16, a, static_cast<hipStream_t>(stream)));
}

int echo_rotary_frequencies(const echo_rotary_freq_cfg* cfg, double* freq, float* magnitude) {
  constexpr double kTwoPi = 6.283185307179586476925;
  if (cfg == nullptr || freq == nullptr || magnitude == nullptr) return ECHO_EINVAL;
  const int n = cfg->dims / 2, s = cfg->scaling;
  const bool grid = cfg->pairs_t != 0 || cfg->pairs_r != 0, mixed = s == ECHO_ROTARY_RAMP || s == ECHO_ROTARY_BANDS;
  if (cfg->dims < 2 || cfg->dims > 512 || cfg->dims % 2 != 0 || cfg->pairs_t < 0 || cfg->pairs_r < 0 ||
      int64_t(cfg->pairs_t) + cfg->pairs_r > n || !std::isfinite(cfg->base) || !(cfg->base > 1.0) ||
      s < ECHO_ROTARY_PLAIN || s > ECHO_ROTARY_BANDS || (grid && s > ECHO_ROTARY_LINEAR) ||
      (s == ECHO_ROTARY_BASE && cfg->dims <= 2))
    return ECHO_EINVAL;
  if (s != ECHO_ROTARY_PLAIN && (!std::isfinite(cfg->factor) || !(cfg->factor >= 1.0))) return ECHO_EINVAL;
  if (mixed && (!std::isfinite(cfg->original_length) || !(cfg->original_length >= 1.0) || !(cfg->low > 0.0) ||
                !std::isfinite(cfg->high) || !(cfg->high > cfg->low)))
    return ECHO_EINVAL;
  const double base = s == ECHO_ROTARY_BASE ? cfg->base * std::pow(cfg->factor, cfg->dims / (cfg->dims - 2.0)) : cfg->base;
  if (!std::isfinite(base)) return ECHO_EINVAL;
  const auto clamp = [](double v, double lo, double hi) { return v < lo ? lo : v > hi ? hi : v; };
  const auto pair_of = [&](double turns) {
    return n * std::log(cfg->original_length / (kTwoPi * turns)) / std::log(base);
  };
  double from = 0.0, to = 0.0;
  if (s == ECHO_ROTARY_RAMP) {
    from = clamp(std::floor(pair_of(cfg->high)), 0.0, cfg->dims - 1.0);
    to = clamp(std::ceil(pair_of(cfg->low)), 0.0, cfg->dims - 1.0);
    if (!(to > from)) to = from + 0.001;
  }
  for (int j = 0; j < n; ++j) {
    int at = j, of = n;
    if (grid) {
      const int t = cfg->pairs_t, r = cfg->pairs_r;
      at = j < t ? j : j < t + r ? j - t : j - t - r;
      of = j < t ? t : j < t + r ? r : n - t - r;
    }
    const double f = std::pow(base, -static_cast<double>(at) / of);
    double keep = 1.0;
    if (s == ECHO_ROTARY_LINEAR) keep = 0.0;
    if (s == ECHO_ROTARY_RAMP) keep = 1.0 - clamp((j - from) / (to - from), 0.0, 1.0);
    if (s == ECHO_ROTARY_BANDS)
      keep = clamp((cfg->original_length * f / kTwoPi - cfg->low) / (cfg->high - cfg->low), 0.0, 1.0);
    freq[j] = keep == 1.0 ? f : keep * f + (1.0 - keep) * f / cfg->factor;
  }
  *magnitude = s == ECHO_ROTARY_RAMP ? static_cast<float>(1.0 + 0.1 * std::log(cfg->factor)) : 1.0f;
  return ECHO_OK;
}

int echo_gated_norm(const echo_gated_norm_cfg* cfg, const void* z, const void* residual, const int32_t* residual_rows,
                    const float* after_weight, const float* gate, const float* before_weight, const float* scale,
                    const float* shift, const int32_t* groups, void* y, void* h, void* stream) {
  if (!gated_norm_cfg_ok(cfg)) return ECHO_EINVAL;
  if (cfg->D > 16384) return ECHO_EUNSUPPORTED;
  if (cfg->M == 0) return ECHO_OK;
  const bool next = cfg->before != ECHO_NORM_NONE;
  auto opt = [](const void* p) { return p == nullptr || elem_aligned(p, 4); };
  if (!elem_aligned(z, esize(cfg->z_dtype)) || !elem_aligned(residual, esize(cfg->residual_dtype)) ||
      !elem_aligned(y, esize(cfg->y_dtype)) || !opt(residual_rows) || !opt(after_weight) || !opt(gate) ||
      !opt(before_weight) || !opt(scale) || !opt(shift) || !opt(groups) ||
      (residual_rows != nullptr ? cfg->residual_nrows < 1 : cfg->residual_nrows < cfg->M) ||
      (groups == nullptr && cfg->M % cfg->n_groups != 0))
    return ECHO_EINVAL;
  if (next ? !elem_aligned(h, esize(cfg->h_dtype))
           : (h != nullptr || before_weight != nullptr || scale != nullptr || shift != nullptr))
    return ECHO_EINVAL;
  // an output in an input's place has to be written where that row alone was read
  if ((y == residual && (residual_rows != nullptr || cfg->y_dtype != cfg->residual_dtype || cfg->ldy != cfg->ldr)) ||
      (next && h == z && (cfg->h_dtype != cfg->z_dtype || cfg->ldh != cfg->ldz)))
    return ECHO_EINVAL;
  GatedNormArgs a{};
  a.M = cfg->M; a.D = cfg->D; a.G = cfg->n_groups; a.after = cfg->after; a.before = cfg->before;
  a.alpha = cfg->residual_scale; a.eps = cfg->eps;
  a.z = z; a.z_bf16 = cfg->z_dtype == ECHO_BF16; a.ldz = cfg->ldz;
  a.x = residual; a.x_bf16 = cfg->residual_dtype == ECHO_BF16; a.ldx = cfg->ldr;
  a.x_rows = residual_rows; a.x_nrows = cfg->residual_nrows;
  a.w1 = after_weight; a.w2 = before_weight;
  a.gate = gate; a.scale = scale; a.shift = shift;
  a.ldgate = cfg->ldgate; a.ldscale = cfg->ldscale; a.ldshift = cfg->ldshift;
  a.groups = groups; a.rows_per_group = groups != nullptr ? 1 : cfg->M / cfg->n_groups;
  a.y = y; a.y_bf16 = cfg->y_dtype == ECHO_BF16; a.ldy = cfg->ldy;
  a.h = h; a.h_bf16 = cfg->h_dtype == ECHO_BF16; a.ldh = cfg->ldh;
  return device_status(launch_gated_norm(a, static_cast<hipStream_t>(stream)));
}

size_t echo_cross_attention_workspace(const echo_cross_attention_cfg* cfg, int32_t masked) {
  if (!cross_cfg_ok(cfg) || !cross_supported(cfg) || cfg->B == 0 || cfg->Lq == 0) return 0;
  return cross_workspace_bytes(cfg->dtype == ECHO_BF16, cfg->B, cfg->Lq, cfg->Lk, cfg->H, cfg->Hkv, cfg->dh,
                               masked != 0 && cfg->Lk > 0);
}

int echo_cross_attention(const echo_cross_attention_cfg* cfg, const void* q, const void* k, const void* v,
                         const int32_t* k_len, const uint8_t* key_mask, void* out, void* workspace,
                         size_t workspace_bytes, void* stream) {
  if (!cross_cfg_ok(cfg)) return ECHO_EINVAL;
  if (!cross_supported(cfg)) return ECHO_EUNSUPPORTED;
  if (cfg->B == 0 || cfg->Lq == 0) return ECHO_OK;
  const bool states = cfg->Lk > 0;  // without any, k, v and the masks are not looked at
  if (!ok_ptr(q) || !ok_ptr(out) || (states && (!ok_ptr(k) || !ok_ptr(v) || (k_len != nullptr && !elem_aligned(k_len, 4)))))
    return ECHO_EINVAL;
  const size_t need = echo_cross_attention_workspace(cfg, key_mask != nullptr);
  if (need > 0 && (!ok_ptr(workspace) || workspace_bytes < need)) return ECHO_EWORKSPACE;
  CrossArgs a = cross_args(cfg);
  a.q = q; a.k = k; a.v = v; a.out = out;
  a.k_len = states ? k_len : nullptr;
  a.key_mask = states ? key_mask : nullptr;
  return device_status(launch_cross(cfg->dtype == ECHO_BF16, a, workspace, static_cast<hipStream_t>(stream)));
}

int echo_mfma_ceiling(int32_t pattern, int32_t data, double seconds, double* tflops, void* stream) {
  if ((pattern != ECHO_MFMA_ATTENTION && pattern != ECHO_MFMA_GEMM) ||
      (data != ECHO_OPERANDS_CONSTANT && data != ECHO_OPERANDS_GAUSSIAN) || !(seconds > 0.0 && seconds <= 60.0) ||
      tflops == nullptr)
    return ECHO_EINVAL;
  const hipError_t e = run_mfma_ceiling(pattern, data == ECHO_OPERANDS_GAUSSIAN, seconds, tflops,
                                        static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ECHO_OK : device_status(e);
}

int echo_profile_enable(int on) {
  profile_set(on != 0);
  return ECHO_OK;
}

int echo_profile_read(echo_kernel_time* out, int32_t max) {
  if (max < 0 || (max > 0 && out == nullptr)) return -ECHO_EINVAL;
  int n = 0;
  int status = ECHO_OK;
  for (const TimingRecord& r : g_records) {
    float ms = 0.0f;
    hipError_t e = hipEventSynchronize(r.stop);
    if (e == hipSuccess) e = hipEventElapsedTime(&ms, r.start, r.stop);
    if (e != hipSuccess) {
      g_last_hip_error = static_cast<int>(e);
      status = ECHO_EDEVICE;
    }
    int slot = -1;
    for (int i = 0; i < n; ++i)
      if (strcmp(out[i].name, r.name) == 0) slot = i;
    if (slot < 0 && n < max) {
      slot = n++;
      out[slot].name = r.name;
      out[slot].launches = 0;
      out[slot].total_ms = 0.0;
    }
    if (slot >= 0) {
      out[slot].launches += 1;
      out[slot].total_ms += ms;
    }
    g_event_pool.push_back(r.start);
    g_event_pool.push_back(r.stop);
  }
  g_records.clear();
  return status == ECHO_OK ? n : -status;
}

}  // extern "C"
