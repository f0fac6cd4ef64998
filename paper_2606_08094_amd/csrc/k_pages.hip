// The paged K/V cache: rows of new tokens into their pages, quantised to int8
// or e4m3 where the pages hold 8 bits, and rows back out of them.
//
// Both are bound by memory: a row (one token, one K/V head, K or V) is read
// and written once.  A row is shared by as many lanes as it has 16-byte
// vectors of source (write) or 16-value pieces (read).
#include "paged.h"

namespace {

// fp32 values of 16 bytes of row: 4 (fp32) or 8 (bf16) of them.
template <int F32>
VLA_DEV void row_vec(uint4 u, float* v) {
  if constexpr (F32) unpack16(u, v, float());
  else unpack16(u, v, bf16_t());
}

// One row per LPR lanes (LPR a power of two, 8 .. 64), NV values per lane.
// Rows are numbered (token, K or V, head), heads fastest.
template <int F32, int TYPE, int HD>
__global__ __launch_bounds__(256) void pages_write(PageRowsArgs a) {
  constexpr int NV = F32 ? 4 : 8, LPR = HD / NV;
  const PageArgs& p = a.p;
  const int lane = threadIdx.x & 63;
  const long long rows = (long long)p.T * 2 * p.G;
  const long long row = ((long long)blockIdx.x * 256 + threadIdx.x) / LPR;
  const bool live = row < rows;
  const int t = live ? (int)(row / (2 * p.G)) : 0;
  const int kv = live ? (int)(row / p.G) & 1 : 0, g = live ? (int)(row % p.G) : 0;
  const int c = (lane & (LPR - 1)) * NV;
  uint4 u = make_uint4(0, 0, 0, 0);
  // (a padding token's row is not read: its request is looked up first)
  const int b = request_of(p, t);
  const int s0 = p.starts[b], s1 = p.starts[b + 1];
  const bool mine = live && t >= s0 && t < s1;
  const long long pos = (long long)max(p.lens[b], 0) - s1 + t;
  const int pid = mine ? page_of(p, b, pos) : -1;
  const bool ok = pid >= 0;
  if (ok) {
    const long long off = (long long)t * a.tstride + (long long)g * a.hstride + c;
    u = ldg16(reinterpret_cast<const char*>(kv ? a.v : a.k) + off * (F32 ? 4 : 2));
  }
  float x[NV];
  row_vec<F32>(u, x);
  const size_t at = ((size_t)max(pid, 0) * p.G + g) * ((size_t)1 << p.lg) + (size_t)(pos & ((1 << p.lg) - 1));
  void* dst = kv ? p.v : p.k;
  if constexpr (TYPE == VLA_KV_F32 || TYPE == VLA_KV_BF16) {
    if (!ok) return;
    if constexpr (TYPE == VLA_KV_F32) {
      float* d = reinterpret_cast<float*>(dst) + at * HD + c;
#pragma unroll
      for (int i = 0; i < NV; i += 4) *reinterpret_cast<float4*>(d + i) = make_float4(x[i], x[i + 1], x[i + 2], x[i + 3]);
    } else {
      bf16_t* d = reinterpret_cast<bf16_t*>(dst) + at * HD + c;
#pragma unroll
      for (int i = 0; i < NV; i += 4) *reinterpret_cast<uint2*>(d + i) = make_uint2(pack_bf16x2(x[i], x[i + 1]), pack_bf16x2(x[i + 2], x[i + 3]));
    }
  } else {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (!ok) return;
    constexpr float TOP = TYPE == VLA_KV_I8 ? 127.0f : 448.0f;
    const bool finite = top < 0x7F800000u;
    const float r = fmaxf(__uint_as_float(top), 1e-5f);
    const float inv = __fdiv_rn(TOP, r);
    uint32_t w[NV / 4];
#pragma unroll
    for (int i = 0; i < NV / 4; ++i) {
      float y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) y[e] = finite ? __fmul_rn(x[4 * i + e], inv) : 0.0f;
      w[i] = pack_codes<TYPE>(y);
    }
    uint8_t* d = reinterpret_cast<uint8_t*>(dst) + at * HD + c;
    if constexpr (NV == 8) *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[NV / 4 - 1]);
    else *reinterpret_cast<uint32_t*>(d) = w[0];
    if ((lane & (LPR - 1)) == 0) (kv ? p.vs : p.ks)[at] = finite ? __fdiv_rn(r, TOP) : __uint_as_float(0x7FC00000u);
  }
}

// 16 values of a row per thread; rows are numbered (request, head, row of the
// request), K in blockIdx.y 0 and V in 1.
template <int F32, int TYPE, int HD>
__global__ __launch_bounds__(256) void pages_read(PageRowsArgs a) {
  constexpr int TPR = HD / 16;
  const PageArgs& p = a.p;
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  const long long rows = (long long)p.B * p.G * a.rows;
  const long long row = idx / TPR;
  if (row >= rows) return;
  const int c = (int)(idx % TPR) * 16;
  const long long bg = row / a.rows;
  const int j = (int)(row - bg * a.rows), b = (int)(bg / p.G), g = (int)(bg - (long long)b * p.G);
  if (j >= p.lens[b]) return;
  const int pid = page_of(p, b, j);
  const size_t at = ((size_t)max(pid, 0) * p.G + g) * ((size_t)1 << p.lg) + (size_t)(j & ((1 << p.lg) - 1));
  const bool v = blockIdx.y != 0;
  float x[16];
  if (pid < 0) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(0x7FC00000u);
  } else {
    const char* src = reinterpret_cast<const char*>(v ? p.v : p.k) + (at * HD + c) * type_bytes(TYPE);
    if constexpr (TYPE == VLA_KV_F32) {
#pragma unroll
      for (int i = 0; i < 4; ++i) unpack16(ldg16(src + 16 * i), x + 4 * i, float());
    } else if constexpr (TYPE == VLA_KV_BF16) {
#pragma unroll
      for (int i = 0; i < 2; ++i) unpack16(ldg16(src + 16 * i), x + 8 * i, bf16_t());
    } else {
      const uint4 u = ldg16(src);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
      const float s = (v ? p.vs : p.ks)[at];
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i] = code_f<TYPE>(w[i >> 2], i & 3) * s;
    }
  }
  void* out = v ? a.vo : a.ko;
  if constexpr (F32) {
    float* d = reinterpret_cast<float*>(out) + (size_t)row * HD + c;
#pragma unroll
    for (int i = 0; i < 4; ++i) stg16(d + 4 * i, pack16(x + 4 * i, float()));
  } else {
    bf16_t* d = reinterpret_cast<bf16_t*>(out) + (size_t)row * HD + c;
#pragma unroll
    for (int i = 0; i < 2; ++i) stg16(d + 8 * i, pack16(x + 8 * i, bf16_t()));
  }
}

template <int F32, int TYPE, int HD>
hipError_t write_hd(const PageRowsArgs& a, hipStream_t s) {
  constexpr int LPR = HD / (F32 ? 4 : 8);
  const long long rows = (long long)a.p.T * 2 * a.p.G, per = 256 / LPR;
  hipLaunchKernelGGL((pages_write<F32, TYPE, HD>), dim3((unsigned)((rows + per - 1) / per)), dim3(256), 0, s, a);
  return hipGetLastError();
}
template <int F32, int TYPE, int HD>
hipError_t read_hd(const PageRowsArgs& a, hipStream_t s) {
  const long long rows = (long long)a.p.B * a.p.G * a.rows, per = 256 / (HD / 16);
  hipLaunchKernelGGL((pages_read<F32, TYPE, HD>), dim3((unsigned)((rows + per - 1) / per), 2), dim3(256), 0, s, a);
  return hipGetLastError();
}

// f(element type, page type, head dimension), each as an integral_constant
template <typename F>
hipError_t by_type(int f32, int type, int hd, F f) {
  auto h = [&](auto e, auto t) {
    constexpr int T = decltype(t)::value;
    switch (hd) {
      case 64: return f(e, t, std::integral_constant<int, 64>{});
      case 128: return f(e, t, std::integral_constant<int, 128>{});
      case 256: if constexpr (T != VLA_KV_F32) return f(e, t, std::integral_constant<int, 256>{});
    }
    return hipErrorInvalidValue;
  };
  auto g = [&](auto e) {
    switch (type) {
      case VLA_KV_F32: return h(e, std::integral_constant<int, VLA_KV_F32>{});
      case VLA_KV_BF16: return h(e, std::integral_constant<int, VLA_KV_BF16>{});
      case VLA_KV_I8: return h(e, std::integral_constant<int, VLA_KV_I8>{});
      case VLA_KV_E4M3: return h(e, std::integral_constant<int, VLA_KV_E4M3>{});
    }
    return hipErrorInvalidValue;
  };
  return f32 ? g(std::integral_constant<int, 1>{}) : g(std::integral_constant<int, 0>{});
}

}  // namespace

hipError_t launch_pages_write(const PageRowsArgs& a, hipStream_t s) {
  if (a.p.T <= 0 || a.p.B <= 0) return hipSuccess;
  return by_type(a.f32, a.p.type, a.p.hd, [&](auto e, auto t, auto d) {
    return write_hd<decltype(e)::value, decltype(t)::value, decltype(d)::value>(a, s);
  });
}

hipError_t launch_pages_read(const PageRowsArgs& a, hipStream_t s) {
  if (a.rows <= 0 || a.p.B <= 0) return hipSuccess;
  return by_type(a.f32, a.p.type, a.p.hd, [&](auto e, auto t, auto d) {
    return read_hd<decltype(e)::value, decltype(t)::value, decltype(d)::value>(a, s);
  });
}
