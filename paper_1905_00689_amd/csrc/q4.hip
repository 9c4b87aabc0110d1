// Products with a matrix of 4-bit levels on gfx950:
//
//   y[n][r] = bias[r] + sum_d s[r][d / G] (q[r][d] - z[r][d / G]) x[n][d].
#include <algorithm>

#include "device_common.hpp"
#include "gated.hpp"

namespace alstm {

namespace {

__global__ void __launch_bounds__(256) q4_layout_kernel(Q4Matrix m, const uint8_t* q, const float* scale,
                                                        const uint8_t* zero, int* bad) {
  const size_t nq = (size_t)m.R * ((m.D + 1) / 2), ns = (size_t)m.R * m.groups;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < nq; i += (size_t)gridDim.x * 256) m.q[i] = q[i];
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < ns; i += (size_t)gridDim.x * 256) {
    m.s[i] = scale[i];
    const int z = zero ? zero[i] : 8;
    m.z[i] = (float)z;
    if (z > 15) *bad = 1;
  }
}

__global__ void __launch_bounds__(256) q4_unpack_kernel(Q4Matrix m, uint8_t* q, float* scale, uint8_t* zero) {
  const size_t nq = (size_t)m.R * ((m.D + 1) / 2), ns = (size_t)m.R * m.groups;
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < nq; i += (size_t)gridDim.x * 256) q[i] = m.q[i];
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < ns; i += (size_t)gridDim.x * 256) {
    scale[i] = m.s[i];
    zero[i] = (uint8_t)m.z[i];
  }
}

// One wave per row and four rows of x: lane l takes every 64th column.
template <class T>
__global__ void __launch_bounds__(256) q4_row_kernel(Q4Matrix m, const T* x, int N, const float* bias, T* y) {
  const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int n0 = blockIdx.y * 4;
  if (r >= m.R) return;
  const uint8_t* q = m.q + (size_t)r * ((m.D + 1) / 2);
  float acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int d = lane; d < m.D; d += 64) {
    const size_t g = (size_t)r * m.groups + d / m.G;
    const float w = m.s[g] * ((float)((q[d / 2] >> (4 * (d & 1))) & 15) - m.z[g]);
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + j < N) acc[j] = __builtin_fmaf(w, (float)x[(size_t)(n0 + j) * m.D + d], acc[j]);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float s = wave_sum(acc[j]);
    if (lane == 0 && n0 + j < N) y[(size_t)(n0 + j) * m.R + r] = (T)(s + (bias ? bias[r] : 0.f));
  }
}

}  // namespace

size_t q4_bytes(int R, int D, int G) {
  const size_t groups = (size_t)(D + G - 1) / G;
  return ((size_t)R * ((D + 1) / 2) + 255) / 256 * 256 + 2 * (((size_t)R * groups * 4 + 255) / 256 * 256);
}

void q4_place(Q4Matrix& m, uint8_t* store) {
  m.q = store;
  store += ((size_t)m.R * ((m.D + 1) / 2) + 255) / 256 * 256;
  m.s = reinterpret_cast<float*>(store);
  store += ((size_t)m.R * m.groups * 4 + 255) / 256 * 256;
  m.z = reinterpret_cast<float*>(store);
}

hipError_t launch_q4_layout(const Q4Matrix& m, const uint8_t* q, const float* scale, const uint8_t* zero, int* bad,
                            hipStream_t stream) {
  q4_layout_kernel<<<1024, 256, 0, stream>>>(m, q, scale, zero, bad);
  return hipGetLastError();
}

hipError_t launch_q4_unpack(const Q4Matrix& m, uint8_t* q, float* scale, uint8_t* zero, hipStream_t stream) {
  q4_unpack_kernel<<<1024, 256, 0, stream>>>(m, q, scale, zero);
  return hipGetLastError();
}

hipError_t launch_q4(const Q4Matrix& m, const void* x, int N, int bf16, const float* bias, void* y, int num_cu,
                     hipStream_t stream) {
  (void)num_cu;
  const dim3 grid((m.R + 3) / 4, (N + 3) / 4);
  if (bf16) q4_row_kernel<__bf16><<<grid, 256, 0, stream>>>(m, (const __bf16*)x, N, bias, (__bf16*)y);
  else q4_row_kernel<float><<<grid, 256, 0, stream>>>(m, (const float*)x, N, bias, (float*)y);
  return hipGetLastError();
}

}  // namespace alstm
