// Linear layers with 8-bit integer operands: the per-token quantiser of the
// activations and the int8 x int8 GEMM with a scale per token and channel.
#include "device_common.h"

namespace {

// ---------------------------------------------------------------------------
// Per-token quantiser: r = max(max|x|, 1e-5), q = rne(x * fl(127 / r)), in fp32
// with a correctly rounded divide.  A row with a NaN or an infinity (seen as
// the largest |x| by its bits, which order non-negative floats and put NaN
// last) gets codes 0 and r = NaN.

// Any alignment: one value at a time, two passes over the row.
template <int F32>
__global__ __launch_bounds__(256) void quant_tok_any(QuantTokArgs a) {
  __shared__ uint32_t red[4];
  const int m = blockIdx.x;
  const char* row = reinterpret_cast<const char*>(a.x) + (size_t)m * a.ldx * (F32 ? 4 : 2);
  auto at = [&](int k) {
    return F32 ? reinterpret_cast<const float*>(row)[k] : bf2f(reinterpret_cast<const bf16_t*>(row)[k]);
  };
  uint32_t top = 0;
  for (int k = threadIdx.x; k < a.K; k += 256) top = max(top, __float_as_uint(at(k)) & 0x7FFFFFFFu);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  top = max(max(red[0], red[1]), max(red[2], red[3]));
  const bool finite = top < 0x7F800000u;
  const float r = fmaxf(__uint_as_float(top), 1e-5f);
  const float inv = __fdiv_rn(127.0f, r);
  int8_t* q = a.q + (size_t)m * a.ldq;
  for (int k = threadIdx.x; k < a.K; k += 256) q[k] = finite ? (int8_t)(int)rintf(__fmul_rn(at(k), inv)) : 0;
  if (threadIdx.x == 0) a.r[m] = finite ? r : __uint_as_float(0x7FC00000u);
}

// ---------------------------------------------------------------------------
// int8 GEMM, one wave per 32 x 32 output tile, operands straight from memory.
// W rows are the A operand, token rows B: a lane holds four consecutive
// columns of one token row.  Lane group g (= lane / 16) of a 64-deep step
// holds k = 16 g .. 16 g + 15.
__global__ __launch_bounds__(256) void int8_direct(Int8Args a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, g4 = lane >> 4;
  const int M = a.M, N = a.N, K = a.K;
  const long long unit = (long long)blockIdx.x * 4 + wave;
  const int mt = (int)(unit / a.n_tiles), nt = (int)(unit - (long long)mt * a.n_tiles);
  if (mt >= a.m_tiles) return;
  const int m0 = mt * 32, n0 = nt * 32;
  i32x4 acc[2][2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  for (int k0 = 0; k0 < K; k0 += 64) {
    const int k = k0 + 16 * g4;
    uint4 xf[2], wf[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int m = m0 + 16 * i + r16, n = n0 + 16 * i + r16;
      xf[i] = m < M && k < K ? ldg16(a.x + (size_t)m * a.ldx + k) : make_uint4(0, 0, 0, 0);
      wf[i] = n < N && k < K ? ldg16(a.w + (size_t)n * a.ldw + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[j]),
                                                          __builtin_bit_cast(i32x4, xf[i]), acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int m = m0 + 16 * i + r16;
    if (m >= M) continue;
    const float r = a.r[m];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * j + 4 * g4 + e;
        if (n >= N) continue;
        const float y = (float)acc[i][j][e] * (a.wscale[n] * r / 127.0f) + (a.bias ? a.bias[n] : 0.0f);
        if (a.out_f32) reinterpret_cast<float*>(a.y)[(size_t)m * a.ldy + n] = y;
        else reinterpret_cast<bf16_t*>(a.y)[(size_t)m * a.ldy + n] = f2bf(y);
      }
  }
}

}  // namespace

hipError_t launch_quantize_tokens(int f32, const QuantTokArgs& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (f32) hipLaunchKernelGGL(quant_tok_any<1>, dim3(a.M), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(quant_tok_any<0>, dim3(a.M), dim3(256), 0, s, a);
  return hipGetLastError();
}

hipError_t launch_int8_gemm(const Int8Args& a0, hipStream_t s) {
  Int8Args a = a0;
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  a.m_tiles = (a.M + 31) / 32;
  a.n_tiles = (a.N + 31) / 32;
  const long long units = (long long)a.m_tiles * a.n_tiles;
  hipLaunchKernelGGL(int8_direct, dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}
