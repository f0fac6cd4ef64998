// Attention of new tokens over the paged K/V cache of their requests.
//
// One pass over the keys with a running maximum and sum (softmax in base 2).
// The R = H / G query heads that share a K/V head are rows of one tile: row rr
// of a request's group is head rr % R of token rr / R, so a key serves every
// row of the tile from one load whatever R and the number of tokens are.
//
// Scores are computed transposed, S^T = K Q^T on MFMA: a lane's column is one
// row of the tile and the softmax statistics live in the lane.  Row rho of
// score tile t holds key 8 (rho / 4) + 4 t + rho % 4 of a block of 32, so lane
// group g (= lane / 16) ends up with keys 8 g .. 8 g + 7, which are the k
// slots of its B operand P^T in O^T += V^T P^T.
#include <algorithm>

#include "paged.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Over the four 16-lane groups of the wave, per lane % 16 (row swaps).
template <typename F>
VLA_DEV float over_groups(float v, F f) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
VLA_DEV float groups_max(float v) { return over_groups(v, [](float x, float y) { return fmaxf(x, y); }); }
VLA_DEV float groups_sum(float v) { return over_groups(v, [](float x, float y) { return x + y; }); }

// The tile of one workgroup.  Request b owns tile slots floor(starts[b] R / ROWS)
// + b and up: the next request's begin no earlier than its ceil(n R / ROWS)
// tiles end, and there are floor(T R / ROWS) + B slots in all, so the host
// needs no lengths to size the grid and a workgroup no prefix sum to find its
// tile, only the last request whose first slot is not past its own.
struct Tile {
  int b, s0, n;        // request, its first new token and their number
  int row0;            // first row of the tile in the request's group
  int len;             // rows of the request, at most what its page table holds
  int pos0;            // position of its first new token
  bool beyond;         // kv_len is past the page table
};
template <int ROWS>
VLA_DEV bool paged_tile_of(const PagedAttnArgs& a, int slot, Tile& t) {
  const PageArgs& p = a.p;
  auto first = [&](int b) { return (int)((long long)p.starts[b] * a.R / ROWS) + b; };
  const int lane = threadIdx.x & 63;
  int cnt = 0;
  for (int base = 0; base < p.B; base += 64) {
    const int i = base + lane;
    const unsigned long long in = __ballot(i < p.B && first(min(i, p.B - 1)) <= slot);
    cnt += __popcll(in);
    if (in != ~0ull) break;
  }
  if (cnt == 0) return false;
  t.b = cnt - 1;
  t.s0 = p.starts[t.b];
  const int s1 = p.starts[t.b + 1];
  t.n = s1 - t.s0;
  if (t.s0 < 0 || s1 > p.T || t.n <= 0) return false;
  t.row0 = (slot - first(t.b)) * ROWS;
  if (t.row0 < 0 || t.row0 >= t.n * a.R) return false;
  const int kv = p.lens[t.b];
  const int cap = p.max_pages << p.lg;
  t.beyond = kv > cap;
  t.len = min(max(kv, 0), cap);
  t.pos0 = max(kv, 0) - t.n;
  return true;
}

// Keys [lo, hi) that some row of the tile may see, of them those of one split
// (none if lo >= hi); lo is rounded down to a block of 32.
VLA_DEV void tile_keys(const PagedAttnArgs& a, const Tile& t, int rows, int split, int& lo, int& hi) {
  const int i0 = t.row0 / a.R, i1 = min(t.n - 1, (t.row0 + rows - 1) / a.R);
  hi = a.causal ? min(t.len, t.pos0 + i1 + 1) : t.len;
  lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + i0 - a.window + 1) : 0;
  const long long base = (lo & ~31) + (long long)split * a.chunk;
  if (split + 1 < a.nsplit) hi = (int)min((long long)hi, base + a.chunk);
  lo = (int)min(base, 0x7fffff00LL);
}

// How a lane's share of a K or V row is laid out, by page type and head
// dimension.  K: 16-byte pieces, lane group g takes piece 4 c + g, c < NK.
// V: VE values of piece h at dimension h 16 VE + (lane % 16) VE, h < NH.
template <int TYPE, int HD>
struct Lay {
  static constexpr int ES = type_bytes(TYPE);
  static constexpr int NK = HD * ES / 64;                    // 16-byte vectors of K per lane and key
  static constexpr int DT = HD / 16;                         // 16-dimension tiles of O^T
  static constexpr int VE = 16 / ES < DT ? 16 / ES : DT;     // values per V load
  static constexpr int NH = DT / VE;                         // V loads per key
  static constexpr int VB = VE * ES;                         // their bytes: 4, 8 or 16
  static constexpr bool F32 = TYPE == VLA_KV_F32;
  static constexpr int QK = F32 ? HD / 16 : HD / 32;         // 16-byte vectors of Q per lane
  // first dimension of a lane's Q vector c
  static VLA_DEV int qdim(int c, int g4) {
    if constexpr (F32) return 16 * c + 4 * g4;
    else if constexpr (TYPE == VLA_KV_BF16) return 32 * c + 8 * g4;
    else return 64 * (c >> 1) + 16 * g4 + 8 * (c & 1);
  }
};

template <int B> struct VecOf;
template <> struct VecOf<4> { uint32_t w[1]; };
template <> struct VecOf<8> { uint32_t w[2]; };
template <> struct VecOf<16> { uint32_t w[4]; };
template <int B>
VLA_DEV VecOf<B> ldgv(const void* p) {
  VecOf<B> r;
  if constexpr (B == 16) {
    const uint4 u = ldg16(p);
    r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
  } else if constexpr (B == 8) {
    typedef unsigned v2u __attribute__((ext_vector_type(2)));
    const v2u u = *(const __attribute__((address_space(1))) v2u*)(p);
    r.w[0] = u.x; r.w[1] = u.y;
  } else {
    r.w[0] = *(const __attribute__((address_space(1))) unsigned*)(p);
  }
  return r;
}

// Eight codes (two dwords) as a bf16 MFMA operand vector (exact).
template <int TYPE>
VLA_DEV uint4 codes_bf16(uint32_t lo, uint32_t hi) {
  return make_uint4(pack_bf16x2(code_f<TYPE>(lo, 0), code_f<TYPE>(lo, 1)), pack_bf16x2(code_f<TYPE>(lo, 2), code_f<TYPE>(lo, 3)),
                    pack_bf16x2(code_f<TYPE>(hi, 0), code_f<TYPE>(hi, 1)), pack_bf16x2(code_f<TYPE>(hi, 2), code_f<TYPE>(hi, 3)));
}

// Value e of a V vector, and whether any of its values is NaN or infinite.
template <int TYPE, int B>
VLA_DEV float v_value(const VecOf<B>& v, int e) {
  if constexpr (TYPE == VLA_KV_F32) return __uint_as_float(v.w[e]);
  else if constexpr (TYPE == VLA_KV_BF16) return __uint_as_float(e & 1 ? v.w[e >> 1] & 0xFFFF0000u : v.w[e >> 1] << 16);
  else return code_f<TYPE>(v.w[e >> 2], e & 3);
}
VLA_DEV bool not_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) == 0x7F800000u; }

// ---------------------------------------------------------------------------
// paged_stream: a tile of 16 rows per workgroup, the keys of a split dealt to
// four waves in blocks of 32.  K goes straight from memory into the MFMA A
// operand.  So does V: lane group g loads keys 8 g .. 8 g + 7, each lane the
// same dimensions of all eight, so the V^T operand (eight keys of a dimension)
// is a permutation of the lane's own registers; which of the head's dimensions
// a row of an O^T tile stands for is free.  No LDS until the waves' results
// are joined, no barrier among the loads.
template <int TYPE, int HD>
__global__ __launch_bounds__(256) void paged_stream(PagedAttnArgs a) {
  using L = Lay<TYPE, HD>;
  using E = std::conditional_t<L::F32, float, bf16_t>;
  constexpr int DT = L::DT, VE = L::VE, NH = L::NH, W = 4;
  __shared__ float so[W][DT][64][4];
  __shared__ float sm[W][16], sl[W][16];

  const PageArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, g4 = lane >> 4;
  const int units = a.slots * p.G * a.nsplit;
  int u = (int)(blockIdx.x % 8u) * (int)(gridDim.x / 8u) + (int)(blockIdx.x / 8u);
  if (u >= units) return;
  const int slot = u % a.slots;
  u /= a.slots;
  const int split = u % a.nsplit, g = u / a.nsplit;
  Tile t;
  if (!paged_tile_of<16>(a, slot, t)) return;
  int k_lo, k_hi;
  tile_keys(a, t, 16, split, k_lo, k_hi);

  // this lane's row of the tile
  const int rr = t.row0 + r16;
  const bool rok = rr < t.n * a.R;
  const int tok = rok ? rr / a.R : 0, h = g * a.R + (rok ? rr % a.R : 0);
  const int pos = t.pos0 + tok;
  // it sees keys [see_lo, see_hi)
  const int see_hi = rok ? (a.causal ? min(t.len, pos + 1) : t.len) : 0;
  const int see_lo = a.window > 0 ? (int)max(0LL, (long long)pos - a.window + 1) : 0;
  uint4 qf[L::QK];
  const E* qp = reinterpret_cast<const E*>(a.q) + (size_t)(t.s0 + tok) * a.ldq + (size_t)h * HD;
#pragma unroll
  for (int c = 0; c < L::QK; ++c) qf[c] = rok ? ldg16(qp + L::qdim(c, g4)) : make_uint4(0, 0, 0, 0);
  // every row of the tile sees every key in [all_lo, all_hi)
  const int i1 = min(t.n - 1, (t.row0 + 15) / a.R);
  const int all_hi = a.causal ? min(t.len, t.pos0 + t.row0 / a.R + 1) : t.len;
  const int all_lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + i1 - a.window + 1) : 0;

  f32x4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mrun = -INFINITY, lrun = 0.0f;
  const float sc = a.scale * kLog2e;
  const size_t pagerows = (size_t)1 << p.lg;
  const int mask = (1 << p.lg) - 1;

  for (int kb = k_lo + 32 * wave; kb < k_hi; kb += 32 * W) {
    // pages of the keys whose K (group r16 / 4) and V (group g4) this lane loads
    const int kk0 = kb + 8 * (r16 >> 2), vk0 = kb + 8 * g4;
    const int kpid = kk0 < k_hi ? page_of(p, t.b, kk0) : -1;
    const int vpid = vk0 < k_hi ? page_of(p, t.b, vk0) : -1;
    const size_t krow = ((size_t)max(kpid, 0) * p.G + g) * pagerows + (size_t)(kk0 & mask);
    const size_t vrow = ((size_t)max(vpid, 0) * p.G + g) * pagerows + (size_t)(vk0 & mask);
    uint4 kf[2][L::NK];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int kr = 4 * tt + (r16 & 3);
      const bool ok = kpid >= 0 && kk0 + kr < k_hi;
      const char* kp = reinterpret_cast<const char*>(p.k) + (krow + kr) * (HD * L::ES) + 16 * g4;
#pragma unroll
      for (int c = 0; c < L::NK; ++c) kf[tt][c] = ok ? ldg16(kp + 64 * c) : make_uint4(0, 0, 0, 0);
    }
    VecOf<L::VB> vf[8][NH];
    float ks[8], vs[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool ok = vpid >= 0 && vk0 + j < k_hi;
      const char* vp = reinterpret_cast<const char*>(p.v) + (vrow + j) * (HD * L::ES) + r16 * L::VB;
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) vf[j][hh] = ok ? ldgv<L::VB>(vp + 16 * L::VB * hh) : VecOf<L::VB>{};
      ks[j] = L::ES == 1 && ok ? p.ks[vrow + j] : 1.0f;
      vs[j] = L::ES == 1 && ok ? p.vs[vrow + j] : 1.0f;
    }
    f32x4 s[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      s[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < L::NK; ++c) {
        if constexpr (L::ES == 1) {
          mma16(s[tt], codes_bf16<TYPE>(kf[tt][c].x, kf[tt][c].y), qf[2 * c], bf16_t());
          mma16(s[tt], codes_bf16<TYPE>(kf[tt][c].z, kf[tt][c].w), qf[2 * c + 1], bf16_t());
        } else {
          mma16(s[tt], kf[tt][c], qf[c], E());
        }
      }
    }
    // lane: keys vk0 + j of row r16.  A key on a page outside the pool is NaN
    // where it is seen.
    float x[8];
    float bmax = -INFINITY;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int key = vk0 + j;
      const bool vis = key < see_hi && key >= see_lo && key < k_hi;
      const float sv = s[j >> 2][j & 3] * (L::ES == 1 ? ks[j] * sc : sc);
      x[j] = vis ? (vpid < 0 ? NAN : sv) : -INFINITY;
      bmax = fmaxf(bmax, x[j]);
    }
    bmax = groups_max(bmax);
    const float mnew = fmaxf(mrun, bmax);
    const float mref = mnew == -INFINITY ? 0.0f : mnew;   // no visible key so far: weight 0
    const float corr = __builtin_amdgcn_exp2f(mrun - mref);
    float psum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const bool hidden = x[j] == -INFINITY;
      x[j] = __builtin_amdgcn_exp2f(x[j] - mref);
      psum += x[j];
      if constexpr (L::ES == 1) x[j] = hidden ? 0.0f : x[j] * vs[j];   // (the scale may be NaN)
    }
    lrun = lrun * corr + groups_sum(psum);
    mrun = mnew;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d] *= corr;

    if constexpr (TYPE != VLA_KV_I8) {
      // A NaN or an infinity in V must not reach the rows that do not see its
      // key, and 0 times it would: where rows see different keys, such values
      // are taken out of the product and added to the rows that see them.
      if (!(kb >= all_lo && min(kb + 32, k_hi) <= all_hi)) {
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int hh = 0; hh < NH; ++hh)
#pragma unroll
            for (int e = 0; e < VE; ++e) bad |= not_finite(v_value<TYPE>(vf[j][hh], e));
        if (__any(bad)) {
#pragma unroll 1
          for (int gk = 0; gk < 4; ++gk)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int key = kb + 8 * gk + j;
              const float pk = __shfl(x[j], 16 * gk + r16, 64);
              const bool vis = key < see_hi && key >= see_lo && key < k_hi;
#pragma unroll
              for (int hh = 0; hh < NH; ++hh)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                  const float own = v_value<TYPE>(vf[j][hh], e);
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    const float val = __shfl(own, 16 * gk + 4 * g4 + i, 64);
                    if (vis && not_finite(val)) o[hh * VE + e][i] += pk * val;
                  }
                }
            }
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int hh = 0; hh < NH; ++hh)
#pragma unroll
              for (int e = 0; e < VE; ++e)
                if (not_finite(v_value<TYPE>(vf[j][hh], e))) {
                  if constexpr (TYPE == VLA_KV_F32) vf[j][hh].w[e] = 0;
                  else if constexpr (TYPE == VLA_KV_BF16) vf[j][hh].w[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
                  else vf[j][hh].w[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
                }
        }
      }
    }

    // O^T += V^T P^T
    if constexpr (L::F32) {
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int e = 0; e < VE; ++e)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            o[hh * VE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vf[j][hh].w[e]), x[j], o[hh * VE + e], 0, 0, 0);
    } else {
      const uint4 pb = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          uint32_t w[4];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            if constexpr (TYPE == VLA_KV_BF16)
              w[jj] = __builtin_amdgcn_perm(vf[2 * jj + 1][hh].w[e >> 1], vf[2 * jj][hh].w[e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
            else
              w[jj] = pack_bf16x2(v_value<TYPE>(vf[2 * jj][hh], e), v_value<TYPE>(vf[2 * jj + 1][hh], e));
          }
          mma16(o[hh * VE + e], make_uint4(w[0], w[1], w[2], w[3]), pb, bf16_t());
        }
    }
  }

  // Join the waves: tile d, row 4 g4 + i, column r16 of each.
  if (t.beyond) lrun = NAN;
  if (g4 == 0) {
    sm[wave][r16] = mrun;
    sl[wave][r16] = lrun;
  }
#pragma unroll
  for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(so[wave][d][lane]) = o[d];
  __syncthreads();
  float mx = -INFINITY;
#pragma unroll
  for (int w = 0; w < W; ++w) mx = fmaxf(mx, sm[w][r16]);
  const float mref = mx == -INFINITY ? 0.0f : mx;
  float f[W], tot = 0.0f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    f[w] = __builtin_amdgcn_exp2f(sm[w][r16] - mref);
    tot += sl[w][r16] * f[w];
  }
  if (!rok) return;
  const size_t th = (size_t)(t.s0 + tok) * a.H + h;
  const bool whole = a.nsplit == 1;
  if (g4 == 0 && wave == 0) {
    if (!whole) *reinterpret_cast<float2*>(a.stats + ((size_t)split * p.T * a.H + th) * 2) = make_float2(mx, tot);
    else if (a.lse) a.lse[th] = (mx + __log2f(tot)) * kLn2;
  }
  const float inv = whole ? (tot == 0.0f ? 0.0f : 1.0f / tot) : 1.0f;
#pragma unroll
  for (int dd = 0; dd < DT / W; ++dd) {
    const int d = wave * (DT / W) + dd;
    f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w) v += *reinterpret_cast<const f32x4*>(so[w][d][lane]) * f[w];
    v *= inv;
    // rows 4 g4 + i of tile (hh, e): dimension hh 16 VE + (4 g4 + i) VE + e
    const int hh = d / VE, e = d % VE;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int dim = hh * 16 * VE + (4 * g4 + i) * VE + e;
      if (!whole) a.part[((size_t)split * p.T * a.H + th) * HD + dim] = v[i];
      else reinterpret_cast<E*>(a.o)[(size_t)(t.s0 + tok) * a.ldo + (size_t)h * HD + dim] = ElemTraits<E>::from_f(v[i]);
    }
  }
}

// Joins the splits of one (token, head) per wave: o = sum_s 2^(m_s - m) o_s / sum_s 2^(m_s - m) l_s.
template <int F32>
__global__ __launch_bounds__(256) void paged_join(PagedAttnArgs a) {
  using E = std::conditional_t<F32, float, bf16_t>;
  const PageArgs& p = a.p;
  const long long th = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  const long long all = (long long)p.T * a.H;
  if (th >= all) return;
  const int t = (int)(th / a.H), h = (int)(th - (long long)t * a.H);
  if (t < p.starts[0] || t >= p.starts[p.B]) return;   // padding
  float mx = -INFINITY;
  for (int s = 0; s < a.nsplit; ++s) {
    const float2 st = *reinterpret_cast<const float2*>(a.stats + ((size_t)s * all + th) * 2);
    if (st.y != 0.0f) mx = fmaxf(mx, st.x);
  }
  const float mref = mx == -INFINITY ? 0.0f : mx;
  float tot = 0.0f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  const int c = lane * (p.hd / 64);
  for (int s = 0; s < a.nsplit; ++s) {
    const float2 st = *reinterpret_cast<const float2*>(a.stats + ((size_t)s * all + th) * 2);
    if (st.y == 0.0f) continue;   // a split without keys
    const float f = __builtin_amdgcn_exp2f(st.x - mref);
    tot += st.y * f;
    const float* src = a.part + ((size_t)s * all + th) * p.hd + c;
    for (int i = 0; i < p.hd / 64; ++i) acc[i] += src[i] * f;
  }
  const float inv = tot == 0.0f ? 0.0f : 1.0f / tot;
  E* dst = reinterpret_cast<E*>(a.o) + (size_t)t * a.ldo + (size_t)h * p.hd + c;
  for (int i = 0; i < p.hd / 64; ++i) dst[i] = ElemTraits<E>::from_f(acc[i] * inv);
  if (lane == 0 && a.lse) a.lse[th] = (mx + __log2f(tot)) * kLn2;
}

template <int TYPE, int HD>
hipError_t stream_launch(const PagedAttnArgs& a, hipStream_t s) {
  const long long units = (long long)a.slots * a.p.G * a.nsplit;
  hipLaunchKernelGGL((paged_stream<TYPE, HD>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int TYPE>
hipError_t stream_hd(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.hd) {
    case 64: return stream_launch<TYPE, 64>(a, s);
    case 128: return stream_launch<TYPE, 128>(a, s);
    case 256: if constexpr (TYPE != VLA_KV_F32) return stream_launch<TYPE, 256>(a, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

void paged_attention_plan(PagedAttnArgs& a, long long span) {
  a.slots = (int)((long long)a.p.T * a.R / 16) + a.p.B;
  const long long base = std::max(1LL, (long long)a.slots * a.p.G);
  const long long want = (512 + base - 1) / base, most = std::max(1LL, (span + 127) / 128);
  a.nsplit = (int)std::max(1LL, std::min({want, most, 64LL}));
  a.chunk = (int)std::min<long long>(((span + a.nsplit - 1) / a.nsplit + 127) / 128 * 128, 1 << 30);
  if (a.chunk < 128) a.chunk = 128;
}

size_t paged_attention_bytes(const PagedAttnArgs& a) {
  if (a.nsplit <= 1) return 0;
  return (size_t)a.nsplit * a.p.T * a.H * (a.p.hd + 2) * sizeof(float);
}

hipError_t launch_paged_attention(const PagedAttnArgs& a, hipStream_t s) {
  if (a.p.T <= 0 || a.p.B <= 0) return hipSuccess;
  hipError_t e = hipErrorInvalidValue;
  switch (a.p.type) {
    case VLA_KV_F32: e = stream_hd<VLA_KV_F32>(a, s); break;
    case VLA_KV_BF16: e = stream_hd<VLA_KV_BF16>(a, s); break;
    case VLA_KV_I8: e = stream_hd<VLA_KV_I8>(a, s); break;
    case VLA_KV_E4M3: e = stream_hd<VLA_KV_E4M3>(a, s); break;
  }
  if (e != hipSuccess || a.nsplit == 1) return e;
  const long long rows = (long long)a.p.T * a.H;
  if (a.p.type == VLA_KV_F32) hipLaunchKernelGGL(paged_join<1>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(paged_join<0>, dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}
