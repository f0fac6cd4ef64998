// Linear layers with 8-bit integer operands: the per-token quantiser of the
// activations and the int8 x int8 GEMM with a scale per token and channel.
#include <algorithm>
#include <utility>

#include "device_common.h"

namespace {

// ---------------------------------------------------------------------------
// Per-token quantiser: r = max(max|x|, 1e-5), q = rne(x * fl(127 / r)), in fp32
// with a correctly rounded divide.  A row with a NaN or an infinity (seen as
// the largest |x| by its bits, which order non-negative floats and put NaN
// last) gets codes 0 and r = NaN.
struct TokScale {
  bool finite;
  float r, inv;
};
VLA_DEV TokScale tok_scale(uint32_t top) {
  const float r = fmaxf(__uint_as_float(top), 1e-5f);
  return {top < 0x7F800000u, r, __fdiv_rn(127.0f, r)};
}
VLA_DEV uint32_t wave_umax(uint32_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v = max(v, (uint32_t)__shfl_xor((int)v, o, 64));
  return v;
}

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
  top = wave_umax(top);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
  const TokScale s = tok_scale(max(max(red[0], red[1]), max(red[2], red[3])));
  int8_t* q = a.q + (size_t)m * a.ldq;
  for (int k = threadIdx.x; k < a.K; k += 256) q[k] = s.finite ? (int8_t)(int)rintf(__fmul_rn(at(k), s.inv)) : 0;
  if (threadIdx.x == 0) a.r[m] = s.finite ? s.r : __uint_as_float(0x7FC00000u);
}

// Rows of whole aligned vectors that fit the registers of TPR threads (NV
// 16-byte vectors each), every load in flight before the first use.
template <int F32, int TPR, int NV>
__global__ __launch_bounds__(256) void quant_tok_vec(QuantTokArgs a) {
  constexpr int VE = F32 ? 4 : 8;
  __shared__ uint32_t red[4];
  const int m = blockIdx.x * (256 / TPR) + threadIdx.x / TPR, t = threadIdx.x % TPR;
  const bool live = m < a.M;
  const char* row = reinterpret_cast<const char*>(a.x) + (size_t)(live ? m : 0) * a.ldx * (F32 ? 4 : 2);
  float f[NV][VE];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = VE * (t + TPR * i);
    const uint4 u = live && c < a.K ? ldg16(row + (size_t)c * (F32 ? 4 : 2)) : make_uint4(0, 0, 0, 0);
    if constexpr (F32) unpack16(u, f[i], float());
    else unpack16(u, f[i], bf16_t());
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int e = 0; e < VE; ++e) top = max(top, __float_as_uint(f[i][e]) & 0x7FFFFFFFu);
  top = wave_umax(top);
  if constexpr (TPR > 64) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = max(max(red[0], red[1]), max(red[2], red[3]));
  }
  if (!live) return;
  const TokScale s = tok_scale(top);
  int8_t* q = a.q + (size_t)m * a.ldq;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int c = VE * (t + TPR * i);
    if (c >= a.K) continue;
    uint32_t w[VE / 4];
#pragma unroll
    for (int j = 0; j < VE / 4; ++j) {
      w[j] = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[j] |= ((uint32_t)(int)rintf(__fmul_rn(f[i][4 * j + e], s.inv)) & 0xFFu) << (8 * e);
      if (!s.finite) w[j] = 0;
    }
    if constexpr (VE == 8) *reinterpret_cast<uint2*>(q + c) = make_uint2(w[0], w[VE / 4 - 1]);
    else *reinterpret_cast<uint32_t*>(q + c) = w[0];
  }
  if (t == 0) a.r[m] = s.finite ? s.r : __uint_as_float(0x7FC00000u);
}

template <int F32, int TPR, int NV>
void quant_vec_launch(const QuantTokArgs& a, hipStream_t s) {
  constexpr int RPB = 256 / TPR;
  hipLaunchKernelGGL((quant_tok_vec<F32, TPR, NV>), dim3((a.M + RPB - 1) / RPB), dim3(256), 0, s, a);
}

template <int F32>
void quant_launch(const QuantTokArgs& a, hipStream_t s) {
  constexpr int VE = F32 ? 4 : 8;
  const int nv = (a.K + VE - 1) / VE;      // vectors of a row
  if (a.K % VE || a.ldx % VE || a.ldq % VE || nv > 8 * 256) {
    hipLaunchKernelGGL(quant_tok_any<F32>, dim3(a.M), dim3(256), 0, s, a);
    return;
  }
  // Few rows: a workgroup each, so that a row's loads are spread wide.  Rows
  // enough to fill the chip with one wave each: no barrier.
  if (a.M < 1024 || nv > 8 * 64) {
    if (nv <= 256) quant_vec_launch<F32, 256, 1>(a, s);
    else if (nv <= 512) quant_vec_launch<F32, 256, 2>(a, s);
    else if (nv <= 1024) quant_vec_launch<F32, 256, 4>(a, s);
    else quant_vec_launch<F32, 256, 8>(a, s);
  } else if (nv <= 128) quant_vec_launch<F32, 64, 2>(a, s);
  else if (nv <= 256) quant_vec_launch<F32, 64, 4>(a, s);
  else quant_vec_launch<F32, 64, 8>(a, s);
}

// ---------------------------------------------------------------------------
// int8 GEMM.  W rows are the A operand of v_mfma_i32_16x16x64_i8, token rows B,
// so a lane ends up with four consecutive columns of one token row.  Lane group
// g (= lane / 16) of a 64-deep step holds k = 16 g .. 16 g + 15.

// Four columns n .. n+3 (n % 4 == 0) of token row m; rr = r[m] / 127.
VLA_DEV void store4(const Int8Args& a, int m, int n, i32x4 acc, float rr) {
  const int N = a.N;
  if (n + 3 < N) {
    const float4 ws = *reinterpret_cast<const float4*>(a.wscale + n);
    float4 b = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.bias) b = *reinterpret_cast<const float4*>(a.bias + n);
    const float y0 = (float)acc[0] * (ws.x * rr) + b.x, y1 = (float)acc[1] * (ws.y * rr) + b.y;
    const float y2 = (float)acc[2] * (ws.z * rr) + b.z, y3 = (float)acc[3] * (ws.w * rr) + b.w;
    const size_t at = (size_t)m * a.ldy + n;
    if (a.ldy % 4 == 0) {
      if (a.out_f32) *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.y) + at) = make_float4(y0, y1, y2, y3);
      else *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.y) + at) = make_uint2(pack_bf16x2(y0, y1), pack_bf16x2(y2, y3));
    } else if (a.out_f32) {
      float* y = reinterpret_cast<float*>(a.y) + at;
      y[0] = y0; y[1] = y1; y[2] = y2; y[3] = y3;
    } else {
      bf16_t* y = reinterpret_cast<bf16_t*>(a.y) + at;
      y[0] = f2bf(y0); y[1] = f2bf(y1); y[2] = f2bf(y2); y[3] = f2bf(y3);
    }
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n + e >= N) break;
    const float y = (float)acc[e] * (a.wscale[n + e] * rr) + (a.bias ? a.bias[n + e] : 0.0f);
    if (a.out_f32) reinterpret_cast<float*>(a.y)[(size_t)m * a.ldy + n + e] = y;
    else reinterpret_cast<bf16_t*>(a.y)[(size_t)m * a.ldy + n + e] = f2bf(y);
  }
}

// int8_skinny: at most 64 token rows, where W's bytes set the pace.  A
// workgroup owns 16 NSUB rows of W and every token row; its eight waves split
// K into contiguous ranges of 64-deep steps, U steps' loads in flight at a
// time, straight into the MFMA operands.  The waves' exact int32 sums are added
// through LDS.
constexpr int SKW = 8;
template <int MS, int NSUB>
__global__ __launch_bounds__(64 * SKW) void int8_skinny(Int8Args a) {
  constexpr int U = MS == 1 ? 8 : 4;
  __shared__ i32x4 red[SKW][MS * NSUB][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, g4 = lane >> 4;
  const int M = a.M, N = a.N, K = a.K;
  const int n0 = blockIdx.x * 16 * NSUB;
  const int nst = (K + 63) / 64, per = (nst + SKW - 1) / SKW;
  const int st0 = wave * per, st1 = min(nst, st0 + per);

  const int8_t *wp[NSUB], *xp[MS];
  bool wok[NSUB], xok[MS];
#pragma unroll
  for (int s = 0; s < NSUB; ++s) {
    const int n = n0 + s * 16 + r16;
    wok[s] = n < N;
    wp[s] = a.w + (size_t)(wok[s] ? n : 0) * a.ldw + 16 * g4;
  }
#pragma unroll
  for (int i = 0; i < MS; ++i) {
    const int m = i * 16 + r16;
    xok[i] = m < M;
    xp[i] = a.x + (size_t)(xok[i] ? m : 0) * a.ldx + 16 * g4;
  }
  i32x4 acc[MS][NSUB];
#pragma unroll
  for (int i = 0; i < MS; ++i)
#pragma unroll
    for (int s = 0; s < NSUB; ++s) acc[i][s] = i32x4{0, 0, 0, 0};
  for (int st = st0; st < st1; st += U) {
    uint4 wf[U][NSUB], xf[U][MS];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int k = (st + j) * 64;
      const bool kok = st + j < st1 && k + 16 * g4 < K;
#pragma unroll
      for (int s = 0; s < NSUB; ++s) wf[j][s] = kok && wok[s] ? ldg16(wp[s] + k) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < MS; ++i) xf[j][i] = kok && xok[i] ? ldg16(xp[i] + k) : make_uint4(0, 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
#pragma unroll
      for (int i = 0; i < MS; ++i)
#pragma unroll
        for (int s = 0; s < NSUB; ++s)
          acc[i][s] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[j][s]),
                                                            __builtin_bit_cast(i32x4, xf[j][i]), acc[i][s], 0, 0, 0);
  }
#pragma unroll
  for (int i = 0; i < MS; ++i)
#pragma unroll
    for (int s = 0; s < NSUB; ++s) red[wave][i * NSUB + s][lane] = acc[i][s];
  __syncthreads();
  if (wave >= MS * NSUB) return;
  const int i = wave / NSUB, s = wave % NSUB;
  const int m = i * 16 + r16, n = n0 + s * 16 + 4 * g4;
  if (m >= M || n >= N) return;
  i32x4 sum = red[0][wave][lane];
#pragma unroll
  for (int w = 1; w < SKW; ++w) sum += red[w][wave][lane];
  store4(a, m, n, sum, a.r[m] / 127.0f);
}

// ---------------------------------------------------------------------------
// int8_tile: a (16 MR) x (32 NS) output tile on eight waves.  128-byte K-slices
// of both operands (BM token rows, BN rows of W) stream into a ring of NST LDS
// stages by direct-to-LDS loads, NST - 1 slices ahead of the MFMAs.  A load
// instruction of a wave fills 1 KB (eight rows); 16-byte chunk c of row r lies
// at slot c ^ (r % 8), so the 16 rows of an operand read are spread over the
// banks.  Chunks past K come from a vector of zeros, rows past M or N from the
// last row (not stored).
//
// KG = 2: the waves are two groups of four that take alternate K-slices, each
// with a ring of its own, and add their exact sums through LDS at the end.  A
// wave's share of the tile is then twice as large, and so is what it does with
// every operand byte it reads from LDS; for tiles so small that the LDS reads
// of eight separate shares would set the pace.
__device__ const v4u kZero16 = {0, 0, 0, 0};

template <int MR, int NS, int KG, bool PAIR>
struct I8Tile {
  static constexpr int BM = 16 * MR, BN = 32 * NS, ROWS = BM + BN;
  static constexpr int SB = ROWS * 8;                                // 16-byte slots per stage
  // PAIR: two stages only, so that two workgroups share a compute unit and one
  // computes while the other begins or writes its output.
  static constexpr int NST = PAIR ? 2 : std::min(4, 144 * 1024 / (SB * 16 * KG));
  static constexpr int WV = 8 / KG, WN = WV / 2;                     // waves of a group, along N (two along M)
  static constexpr int MSW = MR / 2, NSW = 2 * NS / WN;              // 16-row subtiles of a wave
  static constexpr int LPT = ROWS / 8 / WV;                          // load instructions of a wave per slice
  // 16-row subtiles of a wave that a pass of the output takes through the ring
  template <int ES>
  static constexpr int ipp() {
    int n = MSW;
    while (n > 1 && (32 * n * (BN * ES + 16) > KG * NST * SB * 16 || MSW % n)) --n;
    return n;
  }
  static_assert(MR % 2 == 0 && (2 * NS) % WN == 0 && LPT * 8 * WV == ROWS && BM % (8 * WV) == 0 && NST >= 2, "tile");
};

// Scales the sums and writes the tile through LDS in passes of 32 IPP rows, so
// that whole cache lines of a row leave at once: the accumulators' own pieces
// are 8 or 16 bytes.
template <typename T, typename R>
VLA_DEV void tile_out(const Int8Args& a, const i32x4 (&acc)[R::MSW][R::NSW], v4u* lds, int m0, int n0, int wm, int wn,
                      bool has_sums) {
  constexpr int MSW = R::MSW, NSW = R::NSW, BN = R::BN, V = 16 / sizeof(T);
  constexpr int PITCH = BN + V;                    // elements; the extra 16 bytes spread the rows over the banks
  constexpr int IPP = R::template ipp<sizeof(T)>();   // 16-row subtiles of a wave per pass
  constexpr int TPR = BN / V, RPI = 512 / TPR;     // threads per row, rows per step
  T* out = reinterpret_cast<T*>(lds);
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, g4 = lane >> 4;
  const int M = a.M, N = a.N;
  float ws[NSW][4], bs[NSW][4];
#pragma unroll
  for (int j = 0; j < NSW; ++j)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int n = min(n0 + (wn * NSW + j) * 16 + 4 * g4 + e, N - 1);
      ws[j][e] = a.wscale[n];
      bs[j][e] = a.bias ? a.bias[n] : 0.0f;
    }
  const bool vec = a.ldy % V == 0;
#pragma unroll
  for (int ip = 0; ip < MSW / IPP; ++ip) {
    if (ip > 0) lds_barrier();
    if (has_sums) {
#pragma unroll
      for (int ii = 0; ii < IPP; ++ii) {
        const int i = ip * IPP + ii;
        const float rr = a.r[min(m0 + (wm * MSW + i) * 16 + r16, M - 1)] / 127.0f;
        T* row = out + (size_t)((wm * IPP + ii) * 16 + r16) * PITCH + wn * NSW * 16 + 4 * g4;
#pragma unroll
        for (int j = 0; j < NSW; ++j) {
          float y[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) y[e] = (float)acc[i][j][e] * (ws[j][e] * rr) + bs[j][e];
          if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(row + 16 * j) = make_float4(y[0], y[1], y[2], y[3]);
          else *reinterpret_cast<uint2*>(row + 16 * j) = make_uint2(pack_bf16x2(y[0], y[1]), pack_bf16x2(y[2], y[3]));
        }
      }
    }
    lds_barrier();
#pragma unroll
    for (int k = 0; k < 32 * IPP / RPI; ++k) {
      const int pr = k * RPI + tid / TPR, c = tid % TPR * V;      // row of the pass: [wm][ii][16]
      const int m = m0 + (pr / (16 * IPP) * MSW + ip * IPP) * 16 + pr % (16 * IPP), n = n0 + c;
      if (m >= M || n >= N) continue;
      T* y = reinterpret_cast<T*>(a.y) + (size_t)m * a.ldy + n;
      const T* v = out + (size_t)pr * PITCH + c;
      if (vec && n + V <= N) {
        stg16(y, *reinterpret_cast<const uint4*>(v));
      } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
          if (n + e < N) y[e] = v[e];
      }
    }
  }
}

template <int MR, int NS, int KG, bool PAIR>
__global__ __launch_bounds__(512, PAIR ? 4 : 2) void int8_tile(Int8Args a) {
  using R = I8Tile<MR, NS, KG, PAIR>;
  constexpr int BM = R::BM, BN = R::BN, SB = R::SB, NST = R::NST, D = NST - 1, LPT = R::LPT, MSW = R::MSW, NSW = R::NSW;
  __shared__ v4u ring[KG][NST][SB];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = KG == 1 ? 0 : wave / R::WV, wl = wave % R::WV;
  const int r16 = lane & 15, g4 = lane >> 4;
  const int wm = wl / R::WN, wn = wl % R::WN;
  const int M = a.M, N = a.N, K = a.K;
  const int per = gridDim.x >> 3;
  const int u = (blockIdx.x & 7) * per + (blockIdx.x >> 3);   // consecutive units on one XCD
  if (u >= a.m_tiles * a.n_tiles) return;
  // Tiles in bands of eight tile rows, so that the 32 that run at a time on an
  // XCD are about 8 x 4 and share their operands in its L2.
  const int band = u / (8 * a.n_tiles), in = u - band * 8 * a.n_tiles;
  const int high = min(8, a.m_tiles - 8 * band);
  const int m0 = (8 * band + in % high) * BM, n0 = in / high * BN;
  const int nsl = (K + 127) / 128;

  const int8_t* src[LPT];
  const int chunk = (lane & 7) ^ (lane >> 3);   // row % 8 = lane / 8
#pragma unroll
  for (int i = 0; i < LPT; ++i) {
    const int row = (i * R::WV + wl) * 8 + (lane >> 3);
    src[i] = (row < BM ? a.x + (size_t)min(m0 + row, M - 1) * a.ldx : a.w + (size_t)min(n0 + row - BM, N - 1) * a.ldw) + chunk * 16;
  }
  const bool past = (nsl - 1) * 128 + chunk * 16 >= K;   // this lane's chunk of the last slice
  auto issue = [&](auto j, int sl) {
    v4u* b = ring[grp][decltype(j)::value];
    const bool z = sl == nsl - 1 && past;
#pragma unroll
    for (int i = 0; i < LPT; ++i)
      dma16(z ? reinterpret_cast<const int8_t*>(&kZero16) : src[i] + (size_t)sl * 128, b + (i * R::WV + wl) * 64);
  };

  i32x4 acc[MSW][NSW];
#pragma unroll
  for (int i = 0; i < MSW; ++i)
#pragma unroll
    for (int j = 0; j < NSW; ++j) acc[i][j] = i32x4{0, 0, 0, 0};
  auto compute = [&](const v4u* b) {
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
      v4u xf[MSW], wf[NSW];
      const int c = kk * 4 + g4;
#pragma unroll
      for (int i = 0; i < MSW; ++i) {
        const int row = (wm * MSW + i) * 16 + r16;
        xf[i] = b[row * 8 + (c ^ (row & 7))];
      }
#pragma unroll
      for (int j = 0; j < NSW; ++j) {
        const int row = BM + (wn * NSW + j) * 16 + r16;
        wf[j] = b[row * 8 + (c ^ (row & 7))];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int i = 0; i < MSW; ++i)
#pragma unroll
        for (int j = 0; j < NSW; ++j)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, wf[j]), __builtin_bit_cast(i32x4, xf[i]),
                                                            acc[i][j], 0, 0, 0);
    }
  };

  // slices grp, grp + KG, ... are this group's: its it-th is KG it + grp
  const int mine = (nsl - grp + KG - 1) / KG, most = (nsl + KG - 1) / KG;
  [&]<int... J>(std::integer_sequence<int, J...>) {
    ((J < mine ? issue(std::integral_constant<int, J>{}, KG * J + grp) : void()), ...);
  }(std::make_integer_sequence<int, D>{});
  for (int it0 = 0; it0 < most; it0 += NST) {
    [&]<int... J>(std::integer_sequence<int, J...>) {
      (
          [&] {
            const int it = it0 + J;
            if (it >= most) return;
            // slice `it` has landed once at most the D - 1 later ones are pending
            if (it + D - 1 < mine) __builtin_amdgcn_s_waitcnt(vm_wait((D - 1) * LPT));
            else __builtin_amdgcn_s_waitcnt(vm_wait(0));
            lds_barrier();
            if (it + D < mine) issue(std::integral_constant<int, (J + D) % NST>{}, KG * (it + D) + grp);
            if (it < mine) compute(ring[grp][J]);
          }(),
          ...);
    }(std::make_integer_sequence<int, NST>{});
  }

  lds_barrier();   // every wave is past its operand reads, and no load is in flight
  if constexpr (KG == 2) {
    i32x4* red = reinterpret_cast<i32x4*>(&ring[0][0][0]);
    static_assert((size_t)R::WV * MSW * NSW * 64 <= (size_t)KG * NST * SB, "sums in the ring");
    if (grp == 1) {
#pragma unroll
      for (int i = 0; i < MSW; ++i)
#pragma unroll
        for (int j = 0; j < NSW; ++j) red[((wl * MSW + i) * NSW + j) * 64 + lane] = acc[i][j];
    }
    lds_barrier();
    if (grp == 0) {
#pragma unroll
      for (int i = 0; i < MSW; ++i)
#pragma unroll
        for (int j = 0; j < NSW; ++j) acc[i][j] += red[((wl * MSW + i) * NSW + j) * 64 + lane];
    }
    lds_barrier();
  }
  if (a.out_f32) tile_out<float, R>(a, acc, &ring[0][0][0], m0, n0, wm, wn, grp == 0);
  else tile_out<bf16_t, R>(a, acc, &ring[0][0][0], m0, n0, wm, wn, grp == 0);
}

template <int MR, int NS, int KG, bool PAIR>
void tile_launch(Int8Args a, hipStream_t s) {
  a.m_tiles = (a.M + 16 * MR - 1) / (16 * MR);
  a.n_tiles = (a.N + 32 * NS - 1) / (32 * NS);
  const int tiles = a.m_tiles * a.n_tiles;
  hipLaunchKernelGGL((int8_tile<MR, NS, KG, PAIR>), dim3((tiles + 7) / 8 * 8), dim3(512), 0, s, a);
}

template <int MS, int NSUB>
void skinny_launch(const Int8Args& a, hipStream_t s) {
  hipLaunchKernelGGL((int8_skinny<MS, NSUB>), dim3((a.N + 16 * NSUB - 1) / (16 * NSUB)), dim3(64 * SKW), 0, s, a);
}

}  // namespace

hipError_t launch_quantize_tokens(int f32, const QuantTokArgs& a, hipStream_t s) {
  if (a.M <= 0) return hipSuccess;
  if (f32) quant_launch<1>(a, s);
  else quant_launch<0>(a, s);
  return hipGetLastError();
}

hipError_t launch_int8_gemm(const Int8Args& a, hipStream_t s) {
  if (a.M <= 0 || a.N <= 0) return hipSuccess;
  // The tile whose rounds over 256 compute units cost least.  Microseconds per
  // 128-deep slice and per round beside the slices (first loads, output),
  // measured at 8192 x 16384 x 1024 .. 4096: a CU takes in about 45 GB/s (256 x
  // 256) to 71 GB/s (64 x 128), so large tiles win where they fill the chip
  // (816 x 16384 x 2048: 33.7 us, 46.4 us on 128 x 128) and small ones where
  // they would not (816 x 2048 x 16384: 44 us on 64 x 128, 179 us on 256 x 256).
  // Where there are more than 256 tiles of 128 x 128, two of their workgroups can
  // share a unit, and a last round may be half a one (8192 x 16384 x 1024: 222 us,
  // 290 one at a time; 1000 x 5000 x 8192: 51 us, 59 on 128 x 256).  Not for rows
  // that do not begin with a cache line: the smaller the tile, the more lines
  // they touch in vain (5000 x 2000 x 6000: 103 us, 79 on 256 x 256).
  struct Cost { int bm, bn; bool pair; float slice, round; void (*launch)(Int8Args, hipStream_t); };
  static const Cost costs[] = {
      {256, 256, false, 1.50f, 9.8f, tile_launch<16, 8, 1, false>}, {128, 256, false, 0.88f, 7.3f, tile_launch<8, 8, 1, false>},
      {128, 128, false, 0.57f, 4.5f, tile_launch<8, 4, 1, false>},  {128, 128, true, 0.51f, 3.0f, tile_launch<8, 4, 1, true>},
      {64, 128, false, 0.34f, 3.2f, tile_launch<4, 4, 2, false>},   {64, 64, false, 0.24f, 2.3f, tile_launch<4, 2, 2, false>}};
  const bool lines = a.ldx % 128 == 0 && a.ldw % 128 == 0;
  const Cost* best = nullptr;
  float least = 0.0f;
  for (const Cost& c : costs) {
    const long long tiles = ((a.M + c.bm - 1LL) / c.bm) * ((a.N + c.bn - 1LL) / c.bn);
    if (c.pair && (tiles <= 256 || !lines)) continue;
    const float rounds = c.pair ? 0.5f * (float)((tiles + 127) / 128) : (float)((tiles + 255) / 256);
    const float t = rounds * ((float)((a.K + 127) / 128) * c.slice + c.round);
    if (!best || t < least) best = &c, least = t;
  }
  // Up to 64 tokens the skinny kernel, which spreads K, is ahead where there are
  // few columns (a workgroup takes in about 36 GB/s of its rows of W and the
  // tokens'): 36 x 20 x 13120 in 16 us, 1 x 2560 x 2560 in 4.4, but 64 x 16384 x
  // 8192 in 60 us against 32 on tiles.
  const bool two = a.N >= 16 * 2 * 256 && a.M <= 32;
  const float wide = two ? 32.0f : 16.0f, rounds = (float)(((long long)(a.N + (int)wide - 1) / (int)wide + 255) / 256);
  if (a.M <= 64 && rounds * (wide + (float)a.M) * (float)a.K / 36e3f + 3.0f < least) {
    switch ((a.M <= 16 ? 10 : a.M <= 32 ? 20 : 40) + two) {
      case 10: skinny_launch<1, 1>(a, s); break;
      case 11: skinny_launch<1, 2>(a, s); break;
      case 20: skinny_launch<2, 1>(a, s); break;
      case 21: skinny_launch<2, 2>(a, s); break;
      default: skinny_launch<4, 1>(a, s); break;
    }
  } else {
    best->launch(a, s);
  }
  return hipGetLastError();
}
