// adamw.hip -- one AdamW step over a list of tensors.
//
// g' = s g, m = b1 m + (1 - b1) g', v = b2 v + (1 - b2) g'^2,
// p = p (1 - lr wd) - lr / (1 - b1^t) m / (sqrt(v) / sqrt(1 - b2^t) + eps).
// Every value is read and written once, so the step is bound by memory (28 bytes a parameter with 32-bit
// states and fp32 parameters, 16 with 8-bit states).  The list travels in the kernel's arguments, 40 tensors
// a launch: no table in device memory, no copy, nothing to wait for, and a captured launch holds all it
// needs.  A workgroup takes CHUNK values of one tensor; it finds the tensor by bisecting the first chunk
// of each.
//
// 8-bit states: blocks of 256 values (one wave, 4 a lane), a code each in e4m3 (v_cvt_pk_fp8_f32, to nearest
// even) and a scale in fp32, the block's largest magnitude / 448, so the largest value is exact and the
// scale, not only the codes, follows a decaying block (steps of b2 = 0.999 are far below a code's 6%).
// The step itself uses the m and v it has just computed; only what is kept is rounded.  A second moment
// above 0 is kept as the smallest code at least: as 0 it would turn the next step into m / eps.
#include "layers.hpp"
#include "units.hpp"

#include <math.h>

namespace svmx {

namespace {

constexpr int AB = 256, AR = 4;                 // threads, blocks of 256 values a wave takes
constexpr int64_t SBLOCK = 256;                 // values of one scale
constexpr int64_t CHUNK = SBLOCK * (AB / 64) * AR;
constexpr int LIST = 40;                        // tensors of a launch
constexpr float F8_MAX = 448.f, F8_MIN = 0x1p-9f, F8_FLUSH = 0x1p-100f;

struct AdamItem {
  void *p, *master;
  const void *g;
  void *m, *v;
  float *ms, *vs;
  int64_t n;
  uint32_t first;  // its first chunk
  float keep;      // 1 - lr wd
  int32_t p_type, g_type;
};

struct AdamList {
  AdamItem t[LIST];
  const float *gs_dev;  // device factor on the gradients, or NULL
  float gs, b1, c1, b2, c2, step, inv_bc2, eps;  // c = 1 - b; step = lr / (1 - b1^t); inv_bc2 = 1 / sqrt(1 - b2^t)
  int32_t count, pad;
};
static_assert(sizeof(AdamList) <= 4000, "kernel arguments");

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

__device__ __forceinline__ uint32_t f8_pack(const float (&r)[4]) {
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(r[0], r[1], 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(r[2], r[3], u, true);
}

// b x + y, rounded as written.  A code is a step function of what is kept, so which of two neighbours a value near
// the step becomes is settled by its last bit: nothing here is contracted, and another implementation
// that rounds every operation reaches the same codes.
__device__ __forceinline__ float moment(float b, float x, float y) {
#pragma clang fp contract(off)
  const float t = b * x;
  return t + y;
}

// The codes of a wave's block of x and its scale.  Infinities count for nothing in the scale and are kept
// as NaN.  POS: values >= 0.
template <bool POS>
__device__ __forceinline__ uint32_t f8_encode(const float (&x)[4], float &scale) {
  float top = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) top = fmaxf(top, __builtin_isfinite(x[e]) ? fabsf(x[e]) : 0.f);
  top = wave_max(top);
  if (top < F8_FLUSH) top = 0.f;
  const float inv = top > 0.f ? (1.0f / top) * F8_MAX : 0.f;
  float r[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const float s = x[e] * inv;
    r[e] = s > F8_MAX ? F8_MAX : s < -F8_MAX ? -F8_MAX : s;
    if (POS && r[e] > 0.f && r[e] < F8_MIN) r[e] = F8_MIN;
    if (!__builtin_isfinite(x[e])) r[e] = __builtin_nanf("");
  }
  scale = top * (1.0f / F8_MAX);
  return f8_pack(r);
}

__device__ __forceinline__ void f8_decode(uint32_t u, float scale, float (&x)[4]) {
  x[0] = __builtin_amdgcn_cvt_f32_fp8((int)u, 0) * scale;
  x[1] = __builtin_amdgcn_cvt_f32_fp8((int)u, 1) * scale;
  x[2] = __builtin_amdgcn_cvt_f32_fp8((int)u, 2) * scale;
  x[3] = __builtin_amdgcn_cvt_f32_fp8((int)u, 3) * scale;
}

// Four codes at p, `left` of them in the tensor.
__device__ __forceinline__ uint32_t load_codes(const uint8_t *p, int64_t left) {
  if (left >= 4) {
    typedef uint32_t u32u __attribute__((aligned(1)));
    return *reinterpret_cast<const u32u *>(p);
  }
  uint32_t u = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) u |= (uint32_t)p[e] << (8 * e);
  return u;
}

__device__ __forceinline__ void store_codes(uint8_t *p, int64_t left, uint32_t u) {
  if (left >= 4) {
    typedef uint32_t u32u __attribute__((aligned(1)));
    *reinterpret_cast<u32u *>(p) = u;
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < left) p[e] = (uint8_t)(u >> (8 * e));
}

template <bool F8>
__global__ void __launch_bounds__(AB) adamw_k(AdamList L) {
  int lo = 0, hi = L.count;  // the last tensor whose first chunk is not past this one
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (L.t[mid].first <= blockIdx.x)
      lo = mid;
    else
      hi = mid;
  }
  const AdamItem &t = L.t[lo];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t b0 = (int64_t)(blockIdx.x - t.first) * (CHUNK / SBLOCK) + w;  // block of this wave, then every 4th
  void *const p_at = t.master ? t.master : t.p;
  const int32_t p_type = t.master ? SVM_F32 : t.p_type;
  float p[AR][4], g[AR][4], m[AR][4], v[AR][4];
#pragma unroll
  for (int r = 0; r < AR; ++r) {
    const int64_t b = b0 + r * (AB / 64), at = b * SBLOCK + 4 * lane, left = t.n - at;
    load_any<4>(p_at, p_type, at, left, p[r]);
    load_any<4>(t.g, t.g_type, at, left, g[r]);
    if (F8) {
      const bool in = b * SBLOCK < t.n;
      f8_decode(load_codes(static_cast<const uint8_t *>(t.m) + at, left), in ? t.ms[b] : 0.f, m[r]);
      f8_decode(load_codes(static_cast<const uint8_t *>(t.v) + at, left), in ? t.vs[b] : 0.f, v[r]);
    } else {
      load_n<4>(static_cast<const float *>(t.m) + at, left, m[r]);
      load_n<4>(static_cast<const float *>(t.v) + at, left, v[r]);
    }
  }
  const float gs = L.gs_dev ? L.gs * *L.gs_dev : L.gs;
#pragma unroll
  for (int r = 0; r < AR; ++r) {
    const int64_t b = b0 + r * (AB / 64), at = b * SBLOCK + 4 * lane, left = t.n - at;
    if (b * SBLOCK >= t.n) break;  // the wave's: blocks are whole waves
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float gr = g[r][e] * gs;
      m[r][e] = moment(L.b1, m[r][e], L.c1 * gr);
      v[r][e] = moment(L.b2, v[r][e], (L.c2 * gr) * gr);
      const float den = __builtin_fmaf(__builtin_sqrtf(v[r][e]), L.inv_bc2, L.eps);
      p[r][e] = __builtin_fmaf(p[r][e], t.keep, -(L.step * m[r][e]) / den);
      if (e >= left) m[r][e] = v[r][e] = 0.f;
    }
    store_any<4>(p_at, p_type, at, left, p[r]);
    if (t.master) store_any<4>(t.p, t.p_type, at, left, p[r]);
    if (F8) {
      float ms, vs;
#pragma unroll
      for (int e = 0; e < 4; ++e)  // a finite gradient's square past fp32: as large as fp32 goes
        if (__builtin_isfinite(m[r][e]) && v[r][e] > 3.402823466e38f) v[r][e] = 3.402823466e38f;
      const uint32_t mc = f8_encode<false>(m[r], ms), vc = f8_encode<true>(v[r], vs);
      store_codes(static_cast<uint8_t *>(t.m) + at, left, mc);
      store_codes(static_cast<uint8_t *>(t.v) + at, left, vc);
      if (lane == 0) {
        t.ms[b] = ms;
        t.vs[b] = vs;
      }
    } else {
      store_n<4>(static_cast<float *>(t.m) + at, left, m[r]);
      store_n<4>(static_cast<float *>(t.v) + at, left, v[r]);
    }
  }
}

}  // namespace

hipError_t launch_adamw(const svm_adamw_tensor *tensors, int64_t count, const svm_adamw_params &p, hipStream_t s) {
  AdamList L;
  L.gs_dev = p.grad_scale_device;
  L.gs = (float)p.grad_scale;
  L.b1 = (float)p.beta1;
  L.c1 = (float)(1.0 - p.beta1);
  L.b2 = (float)p.beta2;
  L.c2 = (float)(1.0 - p.beta2);
  L.step = (float)(p.lr / (1.0 - pow(p.beta1, (double)p.step)));
  L.inv_bc2 = (float)(1.0 / sqrt(1.0 - pow(p.beta2, (double)p.step)));
  L.eps = (float)p.eps;
  L.pad = 0;
  for (const int32_t state : {(int32_t)SVM_F32, (int32_t)SVM_F8}) {
    L.count = 0;
    uint64_t chunks = 0;
    const auto flush = [&]() -> hipError_t {
      if (!L.count) return hipSuccess;
      if (state == SVM_F8)
        hipLaunchKernelGGL(adamw_k<true>, dim3((unsigned)chunks), dim3(AB), 0, s, L);
      else
        hipLaunchKernelGGL(adamw_k<false>, dim3((unsigned)chunks), dim3(AB), 0, s, L);
      L.count = 0;
      chunks = 0;
      return hipGetLastError();
    };
    for (int64_t i = 0; i < count; ++i) {
      const svm_adamw_tensor &t = tensors[i];
      if (t.count == 0 || t.state_type != state) continue;
      const uint64_t c = (uint64_t)((t.count + CHUNK - 1) / CHUNK);
      if (L.count == LIST || chunks + c > 0x7fffffffULL) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      if (c > 0x7fffffffULL) return hipErrorInvalidValue;
      AdamItem &o = L.t[L.count++];
      o.p = t.param;
      o.master = t.master;
      o.g = t.grad;
      o.m = t.m;
      o.v = t.v;
      o.ms = t.m_scale;
      o.vs = t.v_scale;
      o.n = t.count;
      o.first = (uint32_t)chunks;
      o.keep = (float)(1.0 - p.lr * t.weight_decay);
      o.p_type = t.param_type;
      o.g_type = t.grad_type;
      chunks += c;
    }
    const hipError_t e = flush();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace svmx
