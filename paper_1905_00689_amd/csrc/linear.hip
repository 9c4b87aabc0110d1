// The gated linear recurrence on gfx950: the LSTM cell whose gates depend on the
// input alone,
//
//   c_t = sigmoid(f_t) c_{t-1} + sigmoid(i_t) tanh(g_t),   h_t = sigmoid(o_t) tanh(c_t),
//
// and its gradients.  Every (sequence, unit) is a recurrence of its own.
#include <algorithm>

#include "device_common.hpp"
#include "gated.hpp"

namespace alstm {

namespace {

constexpr int kWalkThreads = 256;

template <class T>
__device__ __forceinline__ float to_f32(T v) { return (float)v; }

__device__ __forceinline__ float sig(float x) { return __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }
__device__ __forceinline__ float tnh(float x) { return __builtin_fmaf(-2.0f, __builtin_amdgcn_rcpf(1.0f + __expf(2.0f * x)), 1.0f); }

template <class T>
__global__ void __launch_bounds__(kWalkThreads) linear_walk_kernel(LinearArgs a) {
  const size_t i = (size_t)blockIdx.x * kWalkThreads + threadIdx.x, BH = (size_t)a.B * a.H;
  if (i >= BH) return;
  const int b = (int)(i / a.H), r = (int)(i % a.H), H = a.H;
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  float bi = 0.f, bf = 0.f, bg = 0.f, bo = 0.f;
  if (a.bias) bi = a.bias[r], bf = a.bias[H + r], bg = a.bias[2 * H + r], bo = a.bias[3 * H + r];
  float c = a.c0 ? a.c0[i] : 0.f;
  for (int t = 0; t < a.T; ++t) {
    if (a.c_save && t % kLinearSave == 0) a.c_save[(size_t)(t / kLinearSave) * BH + i] = c;
    float h = 0.f;
    if (t < len) {
      const T* p = (const T*)a.p + ((size_t)t * a.B + b) * 4 * H + r;
      c = __builtin_fmaf(sig((float)p[H] + bf), c, sig((float)p[0] + bi) * tnh((float)p[2 * H] + bg));
      h = sig((float)p[3 * H] + bo) * tnh(c);
    }
    ((T*)a.h)[(size_t)t * BH + i] = (T)h;
  }
  if (a.c_out) a.c_out[i] = c;
}

template <class T>
__global__ void __launch_bounds__(kWalkThreads) linear_back_kernel(LinearArgs a) {
  const size_t i = (size_t)blockIdx.x * kWalkThreads + threadIdx.x, BH = (size_t)a.B * a.H;
  if (i >= BH) return;
  const int b = (int)(i / a.H), r = (int)(i % a.H), H = a.H;
  const int len = a.lengths ? min(max(a.lengths[b], 0), a.T) : a.T;
  float bi = 0.f, bf = 0.f, bg = 0.f, bo = 0.f;
  if (a.bias) bi = a.bias[r], bf = a.bias[H + r], bg = a.bias[2 * H + r], bo = a.bias[3 * H + r];
  float e = a.dc_out ? a.dc_out[i] : 0.f;
  float si = 0.f, sf = 0.f, sg = 0.f, so = 0.f;
  for (int t0 = (a.T - 1) / kLinearSave * kLinearSave; t0 >= 0; t0 -= kLinearSave) {
    float cs[kLinearSave + 1];
    cs[0] = a.c_save[(size_t)(t0 / kLinearSave) * BH + i];
#pragma unroll
    for (int k = 0; k < kLinearSave; ++k) {
      cs[k + 1] = cs[k];
      if (t0 + k < len) {
        const T* p = (const T*)a.p + ((size_t)(t0 + k) * a.B + b) * 4 * H + r;
        cs[k + 1] = __builtin_fmaf(sig((float)p[H] + bf), cs[k], sig((float)p[0] + bi) * tnh((float)p[2 * H] + bg));
      }
    }
#pragma unroll
    for (int k = kLinearSave - 1; k >= 0; --k) {
      const int t = t0 + k;
      if (t >= a.T) continue;
      float di = 0.f, df = 0.f, dg = 0.f, dO = 0.f;
      if (t < len) {
        const T* p = (const T*)a.p + ((size_t)t * a.B + b) * 4 * H + r;
        const float vi = sig((float)p[0] + bi), vf = sig((float)p[H] + bf), vg = tnh((float)p[2 * H] + bg),
                    vo = sig((float)p[3 * H] + bo), tc = tnh(cs[k + 1]);
        const float dh = (float)((const T*)a.dh)[(size_t)t * BH + i];
        const float d = __builtin_fmaf(dh * vo, 1.f - tc * tc, e);
        di = d * vg * (vi * (1.f - vi));
        df = d * cs[k] * (vf * (1.f - vf));
        dg = d * vi * (1.f - vg * vg);
        dO = dh * tc * (vo * (1.f - vo));
        e = vf * d;
      }
      T* dp = (T*)a.dp + ((size_t)t * a.B + b) * 4 * H + r;
      dp[0] = (T)di, dp[H] = (T)df, dp[2 * H] = (T)dg, dp[3 * H] = (T)dO;
      si += di, sf += df, sg += dg, so += dO;
    }
  }
  if (a.dc0) a.dc0[i] = e;
  if (a.dbias) {
    float* s = a.dpart + (size_t)b * 4 * H + r;
    s[0] = si, s[H] = sf, s[2 * H] = sg, s[3 * H] = so;
  }
}

// dbias[k] = the sum of the rows of dpart, in order
__global__ void __launch_bounds__(64) linear_dbias_kernel(const float* dpart, int rows, int n, float* dbias) {
  const int k = blockIdx.x * 64 + threadIdx.x;
  if (k >= n) return;
  float s = 0.f;
  for (int r = 0; r < rows; ++r) s += dpart[(size_t)r * n + k];
  dbias[k] = s;
}

}  // namespace

size_t linear_workspace(int T, int B, int H, int num_cu, int backward) {
  (void)T;
  (void)num_cu;
  return backward == 2 ? ((size_t)B * 4 * H * 4 + 255) / 256 * 256 : 0;
}

hipError_t launch_linear(const LinearArgs& a, void* ws, hipStream_t stream) {
  (void)ws;
  const unsigned blocks = (unsigned)(((size_t)a.B * a.H + kWalkThreads - 1) / kWalkThreads);
  if (a.bf16) linear_walk_kernel<__bf16><<<blocks, kWalkThreads, 0, stream>>>(a);
  else linear_walk_kernel<float><<<blocks, kWalkThreads, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_linear_backward(const LinearArgs& a0, void* ws, hipStream_t stream) {
  LinearArgs a = a0;
  a.dpart = (float*)ws;
  const unsigned blocks = (unsigned)(((size_t)a.B * a.H + kWalkThreads - 1) / kWalkThreads);
  if (a.bf16) linear_back_kernel<__bf16><<<blocks, kWalkThreads, 0, stream>>>(a);
  else linear_back_kernel<float><<<blocks, kWalkThreads, 0, stream>>>(a);
  if (a.dbias) linear_dbias_kernel<<<(4 * a.H + 63) / 64, 64, 0, stream>>>(a.dpart, a.B, 4 * a.H, a.dbias);
  return hipGetLastError();
}

}  // namespace alstm
