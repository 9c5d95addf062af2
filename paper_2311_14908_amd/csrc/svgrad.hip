// svgrad.hip -- the gradient of decision values in their test samples, and of the objective in the rows.
//
// out_q = u_q 2 gamma sum_j c_j K(x_j, x_q) (x_j - x_q), c_j = a_j y_j.  The objective's gradient is the same
// sum with the rows themselves as samples and u_q = -c_q (a_j y_j a_q y_q K is symmetric, which cancels the
// 1/2), zero where a_q = 0; the pair j = q adds nothing and is left out.
#include "layers.hpp"
#include "rbf_d2.hpp"
#include "units.hpp"

namespace svmx {

namespace {

constexpr int GB = 256, GQ = 4, GL = 256;  // threads, samples of a workgroup, rows looked at in one go

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Chunks of training rows: about 1,024 workgroups in all, 64 rows a chunk at least.
int64_t grad_chunks(int64_t n, int64_t d, int64_t m) {
  const int64_t wide = div_up(m, GQ) * div_up(d, 4 * GB), most = div_up(n, 64);
  const int64_t c = wide >= 1024 ? 1 : 1024 / wide;
  return c > most ? most : c > 256 ? 256 : c;
}

// Workgroup (x, y, z): samples 4 x .., columns 1024 y .., chunk z of the training rows.  The chunk's support
// vectors are listed in LDS 256 rows at a time; a wave takes one after the other, adds up the squared
// differences of the four samples in fp64 and leaves c K; then the threads, a unit of four columns each,
// add c K (x_j - x_q) over the listed rows.
__global__ void __launch_bounds__(GB) sv_grad_k(SvGradCall c, double cexp, int64_t chunks, float *__restrict__ part) {
  __shared__ int32_t rows[GL];
  __shared__ double coefs[GL];
  __shared__ float wt[GL][GQ];
  __shared__ int cnt[GB / 64];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const bool objective = c.Q == nullptr;
  const float *Q = objective ? c.X : c.Q;
  const int64_t q0 = (int64_t)blockIdx.x * GQ, at = ((int64_t)blockIdx.y * GB + threadIdx.x) * 4;
  const int64_t per = (c.n + chunks - 1) / chunks, j1 = min(c.n, (blockIdx.z + 1) * per);
  const float *t[GQ];
  double up[GQ];
  bool any = false;
#pragma unroll
  for (int q = 0; q < GQ; ++q) {
    const int64_t i = min(q0 + q, c.m - 1);
    t[q] = Q + i * c.d;
    const double a = objective ? c.alpha[i] : 0.0;
    up[q] = objective ? (a > 0.0 ? -a * (double)c.y[i] : 0.0) : c.up ? c.up[i] : 1.0;
    any = any || !objective || a > 0.0;
  }
  float acc[GQ][4] = {};
  for (int64_t j0 = blockIdx.z * per; any && j0 < j1; j0 += GL) {
    const int64_t j = j0 + threadIdx.x;
    const double a = j < j1 ? c.alpha[j] : 0.0;
    const unsigned long long mask = __ballot(a > 0.0);
    if (lane == 0) cnt[w] = __popcll(mask);
    __syncthreads();
    int off = __popcll(mask & ((1ull << lane) - 1ull)), nsv = 0;
#pragma unroll
    for (int q = 0; q < GB / 64; ++q) {
      off += q < w ? cnt[q] : 0;
      nsv += cnt[q];
    }
    if (a > 0.0) {
      rows[off] = (int32_t)j;
      coefs[off] = a * (double)c.y[j];
    }
    __syncthreads();
    for (int r = w; r < nsv; r += GB / 64) {
      const float *x = c.X + (int64_t)rows[r] * c.d;
      double s[GQ] = {};
      for (int64_t k = 4 * lane; k < c.d; k += 256) {
        float xv[4];
        load_n<4>(x + k, c.d - k, xv);
#pragma unroll
        for (int q = 0; q < GQ; ++q) {
          float tv[4];
          load_n<4>(t[q] + k, c.d - k, tv);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const double f = (double)(xv[e] - tv[e]);
            s[q] = __builtin_fma(f, f, s[q]);
          }
        }
      }
#pragma unroll
      for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int q = 0; q < GQ; ++q) s[q] += __shfl_xor(s[q], o);
      if (lane < GQ) {
        double d2 = s[0];
#pragma unroll
        for (int q = 1; q < GQ; ++q) d2 = lane == q ? s[q] : d2;
        wt[r][lane] = objective && q0 + lane == rows[r] ? 0.f : (float)(coefs[r] * rbf_of_d2(cexp, d2));
      }
    }
    __syncthreads();
    if (at < c.d) {
      float tv[GQ][4];
#pragma unroll
      for (int q = 0; q < GQ; ++q) load_n<4>(t[q] + at, c.d - at, tv[q]);
#pragma unroll 4
      for (int r = 0; r < nsv; ++r) {
        float xv[4];
        load_n<4>(c.X + (int64_t)rows[r] * c.d + at, c.d - at, xv);
#pragma unroll
        for (int q = 0; q < GQ; ++q)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[q][e] = __builtin_fmaf(wt[r][q], xv[e] - tv[q][e], acc[q][e]);
      }
    }
    __syncthreads();
  }
  if (at >= c.d) return;
#pragma unroll
  for (int q = 0; q < GQ; ++q) {
    if (q0 + q >= c.m) break;
    const float f = chunks == 1 ? (float)(2.0 * c.gamma * up[q]) : 1.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[q][e] *= f;
    float *o = chunks == 1 ? c.out + (q0 + q) * c.d : part + ((int64_t)blockIdx.z * c.m + q0 + q) * c.d;
    store_n<4>(o + at, c.d - at, acc[q]);
  }
}

// The chunks' sums in their order, times u_q 2 gamma.
__global__ void __launch_bounds__(GB) sv_grad_join_k(SvGradCall c, int64_t chunks, const float *__restrict__ part) {
  const int64_t i = ((int64_t)blockIdx.x * GB + threadIdx.x) * 4, total = c.m * c.d;
  if (i >= total) return;
  float s[4] = {};
#pragma unroll 8
  for (int64_t k = 0; k < chunks; ++k) {
    float v[4];
    load_n<4>(part + k * total + i, total - i, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) s[e] += v[e];
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int64_t q = min((i + e) / c.d, c.m - 1);
    const double a = c.Q ? 0.0 : c.alpha[q];
    const double up = c.Q ? (c.up ? c.up[q] : 1.0) : (a > 0.0 ? -a * (double)c.y[q] : 0.0);
    s[e] *= (float)(2.0 * c.gamma * up);
  }
  store_n<4>(c.out + i, total - i, s);
}

}  // namespace

int64_t sv_grad_scratch_bytes(int64_t n, int64_t d, int64_t m, bool) {
  if (m == 0) return 0;
  const int64_t chunks = grad_chunks(n, d, m);
  return chunks == 1 ? 0 : 4 * chunks * m * d + 256;
}

hipError_t launch_sv_grad(const SvGradCall &c, void *ws, hipStream_t s) {
  const int64_t chunks = grad_chunks(c.n, c.d, c.m), groups = div_up(c.m, GQ);
  float *part = reinterpret_cast<float *>((reinterpret_cast<uintptr_t>(ws) + 255) & ~(uintptr_t)255);
  hipLaunchKernelGGL(sv_grad_k, dim3((unsigned)groups, (unsigned)div_up(c.d, 4 * GB), (unsigned)chunks), dim3(GB), 0, s, c,
                     -c.gamma * 1.4426950408889634, chunks, part);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (chunks > 1) {
    hipLaunchKernelGGL(sv_grad_join_k, dim3((unsigned)div_up(c.m * c.d, 4 * GB)), dim3(GB), 0, s, c, chunks, part);
    return hipGetLastError();
  }
  return hipSuccess;
}

}  // namespace svmx
