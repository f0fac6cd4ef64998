// The paged K/V cache: rows of new tokens into their pages, quantised to int8
// or e4m3 where the pages hold 8 bits, and rows back out of them.
//
// Both are bound by memory: a row (one token, one K/V head, K or V) is read
// and written once, and where it lies is known after two or three dependent
// loads, which are made for many rows at once.
#include "paged.h"

namespace {

// fp32 values of 16 bytes of row: 4 (fp32) or 8 (bf16) of them.
template <int F32>
VLA_DEV void row_vec(uint4 u, float* v) {
  if constexpr (F32) unpack16(u, v, float());
  else unpack16(u, v, bf16_t());
}

// A wave writes the rows of NT consecutive tokens of one head of K or of V, a
// row per LPR lanes (8 .. 64) of NV values each.  Where the tokens go is found
// for all of them at once, lane i for token i: the request from one load of 64
// starts and a ballot per token, then its length, then its page, while the rows
// are on their way.
template <int F32, int TYPE, int HD, int NT>
__global__ __launch_bounds__(256) void pages_write(PageRowsArgs a) {
  constexpr int NV = F32 ? 4 : 8, LPR = HD / NV, RPS = 64 / LPR, NS = (NT + RPS - 1) / RPS;   // rows per step, steps
  const PageArgs& p = a.p;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const unsigned unit = blockIdx.x * 4 + wave, groups = (unsigned)(p.T + NT - 1) / NT;
  const unsigned kvg = unit / groups;          // K or V and head
  if (kvg >= 2u * p.G) return;
  const int t0 = (int)(unit - kvg * groups) * NT;
  const int kv = kvg >= (unsigned)p.G, g = (int)kvg - (kv ? p.G : 0);
  const int c = (lane & (LPR - 1)) * NV, rs = lane / LPR;
  const char* src = reinterpret_cast<const char*>(kv ? a.v : a.k) + ((long long)g * a.hstride + c) * (F32 ? 4 : 2);
  uint4 u[NS];
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int i = s * RPS + rs, t = min(t0 + i, p.T - 1);
    u[s] = ldg16(src + (long long)t * a.tstride * (F32 ? 4 : 2));
  }

  int cnt = 0;                                 // lane i < NT: requests that begin at or before token t0 + i
  for (int base = 0; base < p.B; base += 64) {
    const int first = p.starts[min(base + lane, p.B - 1)];
    int more = 0;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const int n = __popcll(__ballot(base + lane < p.B && first <= t0 + i));
      if (lane == i) cnt += n;
      more = n;
    }
    if (more < 64) break;
  }
  long long at = -1;                           // row of the pool, -1: not written
  if (lane < NT && cnt > 0) {
    const int b = cnt - 1, t = t0 + lane;
    const int s0 = p.starts[b], s1 = p.starts[b + 1];
    const long long pos = (long long)max(p.lens[b], 0) - s1 + t;
    const int pid = t < p.T && t >= s0 && t < s1 ? page_of(p, b, pos) : -1;
    if (pid >= 0) at = (((long long)pid * p.G + g) << p.lg) + (pos & ((1 << p.lg) - 1));
  }

  char* dst = reinterpret_cast<char*>(kv ? p.v : p.k);
  float* scales = kv ? p.vs : p.ks;
#pragma unroll
  for (int s = 0; s < NS; ++s) {
    const int i = s * RPS + rs;
    const int lo = __shfl((int)at, min(i, NT - 1), 64), hi = __shfl((int)(at >> 32), min(i, NT - 1), 64);
    const bool ok = i < NT && hi >= 0;
    const size_t row = ((size_t)(unsigned)hi << 32) | (unsigned)lo;
    float x[NV];
    row_vec<F32>(u[s], x);
    if constexpr (TYPE == VLA_KV_F32 || TYPE == VLA_KV_BF16) {
      if (!ok) continue;
      if constexpr (TYPE == VLA_KV_F32) {
        float* d = reinterpret_cast<float*>(dst) + row * HD + c;
#pragma unroll
        for (int e = 0; e < NV; e += 4) *reinterpret_cast<float4*>(d + e) = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
      } else if constexpr (F32) {
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(dst) + row * HD + c) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
      } else {
        stg16(reinterpret_cast<bf16_t*>(dst) + row * HD + c, u[s]);
      }
    } else {
      uint32_t top = 0;
#pragma unroll
      for (int e = 0; e < NV; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
      if (!ok) continue;
      constexpr float TOP = TYPE == VLA_KV_I8 ? 127.0f : 448.0f;
      const bool finite = top < 0x7F800000u;
      const float r = fmaxf(__uint_as_float(top), 1e-5f);
      const float inv = __fdiv_rn(TOP, r);
      uint32_t w[NV / 4];
#pragma unroll
      for (int e = 0; e < NV / 4; ++e) {
        float y[4];
#pragma unroll
        for (int f = 0; f < 4; ++f) y[f] = finite ? __fmul_rn(x[4 * e + f], inv) : 0.0f;
        w[e] = pack_codes<TYPE>(y);
      }
      char* d = dst + row * HD + c;
      if constexpr (NV == 8) *reinterpret_cast<uint2*>(d) = make_uint2(w[0], w[NV / 4 - 1]);
      else *reinterpret_cast<uint32_t*>(d) = w[0];
      if ((lane & (LPR - 1)) == 0) scales[row] = finite ? __fdiv_rn(r, TOP) : __uint_as_float(0x7FC00000u);
    }
  }
}

// A workgroup reads RB rows of one request and head, of K or of V.  A thread
// makes 16 bytes of each of U rows, so that a wave's store is one contiguous
// KB; the rows' page ids, then the rows, are all in flight.
template <int F32, int HD>
struct ReadShape {
  static constexpr int NV = F32 ? 4 : 8, TPR = HD / NV, U = 8, RS = 256 / TPR, RB = RS * U;   // rows of a step, of a workgroup
};
template <int F32, int TYPE, int HD>
__global__ __launch_bounds__(256) void pages_read(PageRowsArgs a) {
  using R = ReadShape<F32, HD>;
  constexpr int U = R::U, NV = R::NV, NB = NV * type_bytes(TYPE), NW = NB / 4;   // bytes and dwords stored of NV values
  const PageArgs& p = a.p;
  const unsigned nblk = (unsigned)(a.rows + R::RB - 1) / R::RB;
  unsigned u = blockIdx.x / nblk;
  const int j0 = (int)(blockIdx.x - u * nblk) * R::RB + threadIdx.x / R::TPR, c = threadIdx.x % R::TPR * NV;
  const bool v = u & 1;
  u >>= 1;
  const int b = (int)(u / (unsigned)p.G), g = (int)(u - (unsigned)b * p.G);
  const int end = min(p.lens[b], a.rows);
  int pid[U];
#pragma unroll
  for (int i = 0; i < U; ++i) pid[i] = j0 + i * R::RS < end ? page_of(p, b, j0 + i * R::RS) : -1;
  const char* src = reinterpret_cast<const char*>(v ? p.v : p.k);
  uint32_t raw[U][NW];
  float sc[U];
#pragma unroll
  for (int i = 0; i < U; ++i) {      // (without branches: what is not there is read from page 0 and not used)
    const size_t at = (((size_t)max(pid[i], 0) * p.G + g) << p.lg) + ((j0 + i * R::RS) & ((1 << p.lg) - 1));
    const char* row = src + (at * HD + c) * type_bytes(TYPE);
    if constexpr (NB >= 16) {
#pragma unroll
      for (int l = 0; l < NB / 16; ++l) {
        const uint4 x = ldg16(row + 16 * l);
        raw[i][4 * l] = x.x; raw[i][4 * l + 1] = x.y; raw[i][4 * l + 2] = x.z; raw[i][4 * l + 3] = x.w;
      }
    } else if constexpr (NB == 8) {
      const uint2 x = *reinterpret_cast<const uint2*>(row);
      raw[i][0] = x.x; raw[i][1] = x.y;
    } else {
      raw[i][0] = *reinterpret_cast<const uint32_t*>(row);
    }
    sc[i] = type_bytes(TYPE) == 1 ? (v ? p.vs : p.ks)[at] : 1.0f;
  }
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int j = j0 + i * R::RS;
    if (j >= end) break;
    float x[NV];
#pragma unroll
    for (int e = 0; e < NV; ++e) {
      if constexpr (TYPE == VLA_KV_F32) x[e] = __uint_as_float(raw[i][e]);
      else if constexpr (TYPE == VLA_KV_BF16) x[e] = __uint_as_float(e & 1 ? raw[i][e >> 1] & 0xFFFF0000u : raw[i][e >> 1] << 16);
      else x[e] = code_f<TYPE>(raw[i][e >> 2], e & 3) * sc[i];
      if (pid[i] < 0) x[e] = __uint_as_float(0x7FC00000u);
    }
    const size_t o = (((size_t)b * p.G + g) * a.rows + j) * HD + c;
    if constexpr (F32) stg16(reinterpret_cast<float*>(v ? a.vo : a.ko) + o, pack16(x, float()));
    else stg16(reinterpret_cast<bf16_t*>(v ? a.vo : a.ko) + o, pack16(x, bf16_t()));
  }
}

template <int F32, int TYPE, int HD, int NT>
void write_nt(const PageRowsArgs& a, hipStream_t s) {
  const long long units = (long long)((a.p.T + NT - 1) / NT) * 2 * a.p.G;
  hipLaunchKernelGGL((pages_write<F32, TYPE, HD, NT>), dim3((unsigned)((units + 3) / 4)), dim3(256), 0, s, a);
}
template <int F32, int TYPE, int HD>
hipError_t write_hd(const PageRowsArgs& a, hipStream_t s) {
  // As many tokens per wave as leave some rounds of waves, whose lookups then
  // overlap with others' rows (16 x 2048 rows of 256 at most, int8: 11.4 us with
  // 16 tokens, 10.2 with 8; 16 x 4096 x 8 heads of 128: the same).
  const long long rows = (long long)a.p.T * 2 * a.p.G;
  if (rows >= 64 * 2048) write_nt<F32, TYPE, HD, 16>(a, s);
  else if (rows >= 16 * 2048) write_nt<F32, TYPE, HD, 8>(a, s);
  else if (rows >= 4 * 2048) write_nt<F32, TYPE, HD, 4>(a, s);
  else write_nt<F32, TYPE, HD, 1>(a, s);
  return hipGetLastError();
}
template <int F32, int TYPE, int HD>
hipError_t read_hd(const PageRowsArgs& a, hipStream_t s) {
  constexpr int RB = ReadShape<F32, HD>::RB;
  const long long blocks = (long long)a.p.B * a.p.G * 2 * ((a.rows + RB - 1) / RB);
  hipLaunchKernelGGL((pages_read<F32, TYPE, HD>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  return hipGetLastError();
}

// f(element type, page type, head dimension), each as an integral_constant
template <typename F>
hipError_t by_type(int f32, int type, int hd, F f) {
  auto h = [&](auto e, auto t) {
    switch (hd) {
      case 64: return f(e, t, std::integral_constant<int, 64>{});
      case 128: return f(e, t, std::integral_constant<int, 128>{});
      case 256: return f(e, t, std::integral_constant<int, 256>{});
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
