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
#include <cmath>

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

// x / R and x % R for 0 <= x < 2^28 (rdiv = ceil(2^32 / R), R <= 16).
VLA_DEV int by_r(const PagedAttnArgs& a, int x) { return (int)(((unsigned long long)(unsigned)x * a.rdiv) >> 32); }
VLA_DEV int mod_r(const PagedAttnArgs& a, int x) { return x - by_r(a, x) * a.R; }

// The scores' factor (base 2) is kept positive, so that a maximum of scores can
// be taken before it is applied; one that is not positive turns the scores
// themselves.
VLA_DEV float score_factor(const PagedAttnArgs& a) { return a.scale == 0.0f ? 1.0f : fabsf(a.scale) * kLog2e; }
template <int N>
VLA_DEV void turn_scores(const PagedAttnArgs& a, float (&w)[N]) {
  if (a.scale <= 0.0f) {
    const float f = a.scale < 0.0f ? -1.0f : 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] *= f;
  }
}

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
  const int lane = threadIdx.x & 63;
  int found = -1, s0 = 0, s1 = 0, kv = 0, at = 0;
  for (int base = 0; base < p.B; base += 64) {   // 64 requests at a time, all that is needed of them in one go
    const int i = min(base + lane, p.B - 1);
    const int si = p.starts[i], ei = p.starts[i + 1], li = p.lens[i];
    const int fi = (int)((long long)si * a.R / ROWS) + i;
    const unsigned long long in = __ballot(base + lane < p.B && fi <= slot);
    if (in) {
      const int l = __popcll(in) - 1;
      found = base + l;
      s0 = __builtin_amdgcn_readlane(si, l);
      s1 = __builtin_amdgcn_readlane(ei, l);
      kv = __builtin_amdgcn_readlane(li, l);
      at = __builtin_amdgcn_readlane(fi, l);
    }
    if (in != ~0ull) break;
  }
  if (found < 0) return false;
  t.b = found;
  t.s0 = s0;
  t.n = s1 - s0;
  if (s0 < 0 || s1 > p.T || t.n <= 0) return false;
  t.row0 = (slot - at) * ROWS;
  if (t.row0 < 0 || t.row0 >= t.n * a.R) return false;
  const int cap = p.max_pages << p.lg;
  t.beyond = kv > cap;
  t.len = min(max(kv, 0), cap);
  t.pos0 = max(kv, 0) - t.n;
  return true;
}

// Keys [lo, hi) that some row of the tile may see, of them those of one split
// (none if lo >= hi); lo is rounded down to a block of 32.  A request uses as
// many splits as it has multiples of a.chunk keys, of equal length.
VLA_DEV void tile_keys(const PagedAttnArgs& a, const Tile& t, int rows, int split, int& lo, int& hi) {
  const int i0 = by_r(a, t.row0), i1 = min(t.n - 1, by_r(a, t.row0 + rows - 1));
  hi = a.causal ? min(t.len, t.pos0 + i1 + 1) : t.len;
  lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + i0 - a.window + 1) : 0;
  lo &= ~31;
  if (a.nsplit == 1) return;
  const int span = max(hi - lo, 0);
  const int ns = min((span + a.chunk - 1) / a.chunk, a.nsplit);
  int each = ns > 0 ? (span + ns - 1) / ns : 0;
  if (rows > 16) each = (each + 63) & ~63;                    // blocks of the tile kernel
  else each = each > 64 ? (each + 127) & ~127 : (each + 31) & ~31;   // whole rounds of four waves, or one or two waves
  if (split >= ns) {
    hi = lo;
    return;
  }
  lo += split * each;
  if (split + 1 < ns) hi = min(hi, lo + each);
}

// A split without keys only says so: its output is not read.
VLA_DEV bool empty_split(const PagedAttnArgs& a, const Tile& t, int rows, int g, int split, int lo, int hi) {
  if (a.nsplit == 1 || lo < hi) return false;
  const int rr = t.row0 + threadIdx.x;
  if ((int)threadIdx.x < rows && rr < t.n * a.R) {
    const size_t th = (size_t)(t.s0 + by_r(a, rr)) * a.H + g * a.R + mod_r(a, rr);
    *reinterpret_cast<float2*>(a.stats + ((size_t)split * a.p.T * a.H + th) * 2) = make_float2(-INFINITY, t.beyond ? NAN : 0.0f);
  }
  return true;
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

// Eight codes (two dwords) as a bf16 MFMA operand vector (exact; e4m3 two at a
// time, with a scale of one).
template <bool HI>
VLA_DEV uint32_t e4m3_pair(uint32_t w) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)w, 1.0f, HI));
}
template <int TYPE>
VLA_DEV uint4 codes_bf16(uint32_t lo, uint32_t hi) {
  if constexpr (TYPE == VLA_KV_E4M3)
    return make_uint4(e4m3_pair<false>(lo), e4m3_pair<true>(lo), e4m3_pair<false>(hi), e4m3_pair<true>(hi));
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

// Whether some value of a V vector is NaN or infinite; and the vector with
// those set to zero.
template <int TYPE, int B>
VLA_DEV bool v_bad(const VecOf<B>& v) {
  bool bad = false;
#pragma unroll
  for (int e = 0; e < B / type_bytes(TYPE); ++e) bad |= not_finite(v_value<TYPE>(v, e));
  return bad;
}
template <int TYPE, int B>
VLA_DEV void v_clean(VecOf<B>& v) {
#pragma unroll
  for (int e = 0; e < B / type_bytes(TYPE); ++e)
    if (not_finite(v_value<TYPE>(v, e))) {
      if constexpr (TYPE == VLA_KV_F32) v.w[e] = 0;
      else if constexpr (TYPE == VLA_KV_BF16) v.w[e >> 1] &= e & 1 ? 0x0000FFFFu : 0xFFFF0000u;
      else v.w[e >> 2] &= ~(0xFFu << (8 * (e & 3)));
    }
}
// N (1, 2 or 4) neighbouring values.
template <typename T, int N>
VLA_DEV void put(T* d, const float* x) {
  if constexpr (N == 1) *d = ElemTraits<T>::from_f(x[0]);
  else if constexpr (sizeof(T) == 2 && N == 2) *reinterpret_cast<uint32_t*>(d) = pack_bf16x2(x[0], x[1]);
  else if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(d) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
  else if constexpr (N == 2) *reinterpret_cast<float2*>(d) = make_float2(x[0], x[1]);
  else *reinterpret_cast<float4*>(d) = make_float4(x[0], x[1], x[2], x[3]);
}
// One stored value (dimension dim of a row) as fp32, without its scale.
template <int TYPE>
VLA_DEV float stored(const void* row, int dim) {
  if constexpr (TYPE == VLA_KV_F32) return reinterpret_cast<const float*>(row)[dim];
  else if constexpr (TYPE == VLA_KV_BF16) return bf2f(reinterpret_cast<const bf16_t*>(row)[dim]);
  else return code_f<TYPE>(reinterpret_cast<const uint8_t*>(row)[dim], 0);
}

// Adds the NaNs and infinities among the V values of keys [k0, k1) to the
// outputs of the row that sees them ([see_lo, see_hi)); o[d][i] is dimension
// dim(d, i).  The weights are positive, and such a sum is what it is whatever
// they are.
template <int TYPE, int HD, int DT, typename F>
VLA_DEV void add_not_finite(const PageArgs& p, const int* table, int g, int k0, int k1, int see_lo, int see_hi, f32x4 (&o)[DT], F dim) {
#pragma unroll 1
  for (int key = k0; key < k1; ++key) {
    const int pid = table[key >> p.lg];
    if ((unsigned)pid >= (unsigned)p.n_pages) continue;
    const size_t at = (((size_t)pid * p.G + g) << p.lg) + (key & ((1 << p.lg) - 1));
    const char* row = reinterpret_cast<const char*>(p.v) + at * (HD * type_bytes(TYPE));
    const bool vis = key < see_hi && key >= see_lo;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float val = stored<TYPE>(row, dim(d, i));
        if (vis && not_finite(val)) o[d][i] += val;
      }
  }
}

// ---------------------------------------------------------------------------
// paged_stream: a tile of 16 rows per workgroup, the keys of a split dealt to
// four waves in blocks of 32.  V goes straight from memory into the MFMA A
// operand: lane group g loads keys 8 g .. 8 g + 7, each lane the same dimensions
// of all eight, so the V^T operand (eight keys of a dimension) is a permutation
// of the lane's own registers; which of the head's dimensions a row of an O^T
// tile stands for is free.  K goes by way of LDS, or directly (see KRows).  No
// barrier until the waves' results are joined.
//
// Bound by the cache's bytes: with the arithmetic taken out it takes the same
// time.  The waves of a SIMD hide each other's waits (a second block of both in
// flight per wave leaves room for half the waves: 64 requests of up to 8192 rows
// of int8, 117 us instead of 113 at the time).  Loads have no branches: a key
// that does not exist is read from page 0 and not used.
// Workgroups per compute unit that the registers have to allow: as many as
// they do without spilling.
constexpr int stream_occupancy(int type, int hd) {
  return type == VLA_KV_F32 ? (hd == 64 ? 3 : hd == 128 ? 2 : 1) : type == VLA_KV_BF16 ? (hd == 64 ? 4 : 3) : (hd == 256 ? 2 : hd == 128 ? 3 : 4);
}
// K by way of LDS.  A K operand has sixteen rows in sixteen neighbouring lanes, so
// a load straight into it touches a cache line per lane (some 40 per load
// instruction, and their number is what the cache keeps up with).  Instead whole
// rows go to LDS by direct loads, piece c (16 bytes) of row `key` at slot
// c ^ slot(key), so that the sixteen rows of an operand read lie in different
// banks.  The next block's are under way while a block is worked on.  64 requests
// of up to 8192 rows of 128: int8 96.0 -> 93.0 us, bf16 161 -> 150; fp32, 22 x 50
// tokens over 9737 rows of 128: 345 -> 297.  Not where it does not pay: rows of 64
// bytes, of which four lanes read all (54 us, 57 by LDS), fp32 rows of 256, whose
// registers are full (180, 203), and of 64 (the same at size, a short call 0.2 us
// more).
// A wave's share of LDS also takes its outputs in the end.
template <int TYPE, int HD>
struct KRows {
  static constexpr int RB = HD * type_bytes(TYPE), VPR = RB / 16;   // bytes and pieces of a row
  static constexpr bool USED = TYPE == VLA_KV_F32 ? HD == 128 : RB >= 128;
  static constexpr int RPI = 64 / VPR, NI = 32 / RPI;               // rows of a load, loads of a block
  static constexpr int BYTES = std::max(USED ? 32 * RB : 0, HD / 16 * 1024);
  static VLA_DEV int slot(int key) {
    if constexpr (VPR == 8) return key >> 3 | (key & 2) << 1;
    else return key >> 3 | (key & 3) << 2;
  }
};

template <int TYPE, int HD>
struct KvBlock {           // one lane's share of a block of 32 keys
  using L = Lay<TYPE, HD>;
  uint4 k[2][L::NK];
  VecOf<L::VB> v[8][L::NH];
  float4 ks[2], vs[2];     // 8-bit types: scales of keys 8 g4 .. 8 g4 + 7
  int vpid;
};

template <int TYPE, int HD>
__global__ __launch_bounds__(256, stream_occupancy(TYPE, HD)) void paged_stream(PagedAttnArgs a) {
  using L = Lay<TYPE, HD>;
  using E = std::conditional_t<L::F32, float, bf16_t>;
  constexpr int DT = L::DT, VE = L::VE, NH = L::NH, W = 4;
  using KR = KRows<TYPE, HD>;
  __shared__ __align__(16) unsigned char lds[W][KR::BYTES];
  __shared__ float sm[W][16], sl[W][16];

  const PageArgs& p = a.p;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
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
  if (empty_split(a, t, 16, g, split, k_lo, k_hi)) return;

  // Pages of the keys whose K (group r16 / 4 of eight) and V (group g4) this lane loads.
  const int* table = p.table + (size_t)t.b * p.max_pages;
  const size_t pagerows = (size_t)1 << p.lg;
  const int mask = (1 << p.lg) - 1;
  auto pids = [&](int kb, int& kp, int& vp) {   // -1: past the split's keys
    const int kk = kb + 8 * (r16 >> 2), vk = kb + 8 * g4;
    kp = kk < k_hi ? table[kk >> p.lg] : -1;
    vp = vk < k_hi ? table[vk >> p.lg] : -1;
  };
  unsigned char* const mine = lds[wave];
  auto issue_k = [&](int kb, int kp) {          // K rows of a block on their way into LDS
    const int p0 = __builtin_amdgcn_readlane(kp, 0), p1 = __builtin_amdgcn_readlane(kp, 8);   // its halves' pages
#pragma unroll
    for (int j = 0; j < KR::NI; ++j) {
      const int r = j * KR::RPI, key = r + lane / KR::VPR, p16 = r < 16 ? p0 : p1;
      const size_t row = ((size_t)((unsigned)p16 < (unsigned)p.n_pages ? p16 : 0) * p.G + g) * pagerows + ((kb + r) & mask);
      const char* src = reinterpret_cast<const char*>(p.k) + row * KR::RB + lane / KR::VPR * KR::RB + 16 * (lane % KR::VPR ^ KR::slot(key));
      dma16(src, reinterpret_cast<v4u*>(mine + 1024 * j));
    }
  };
  auto load_k = [&](int kb, int kp, KvBlock<TYPE, HD>& x) {
    const size_t krow = ((size_t)((unsigned)kp < (unsigned)p.n_pages ? kp : 0) * p.G + g) * pagerows + ((kb + 8 * (r16 >> 2)) & mask) + (r16 & 3);
    const char* ka = reinterpret_cast<const char*>(p.k) + krow * (HD * L::ES) + 16 * g4;
#pragma unroll
    for (int tt = 0; tt < 2; ++tt)
#pragma unroll
      for (int c = 0; c < L::NK; ++c) x.k[tt][c] = ldg16(ka + tt * 4 * (HD * L::ES) + 64 * c);
  };
  auto load_v = [&](int kb, int vp, KvBlock<TYPE, HD>& x) {   // and the scales
    x.vpid = (unsigned)vp < (unsigned)p.n_pages ? vp : -1;
    const size_t vrow = ((size_t)max(x.vpid, 0) * p.G + g) * pagerows + ((kb + 8 * g4) & mask);
    const char* va = reinterpret_cast<const char*>(p.v) + vrow * (HD * L::ES) + r16 * L::VB;
    if constexpr (L::ES == 1) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x.ks[i] = __builtin_bit_cast(float4, ldg16(p.ks + vrow + 4 * i));
        x.vs[i] = __builtin_bit_cast(float4, ldg16(p.vs + vrow + 4 * i));
      }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
      for (int hh = 0; hh < NH; ++hh) x.v[j][hh] = ldgv<L::VB>(va + j * (HD * L::ES) + 16 * L::VB * hh);
  };
  constexpr int STEP = 32 * W;
  const int kb0 = k_lo + 32 * wave;
  KvBlock<TYPE, HD> buf;
  int kp = -1, vp = -1, kp1 = -1, vp1 = -1;     // pages of this block and (K by LDS) of the next one
  pids(kb0, kp, vp);
  if constexpr (KR::USED) {
    pids(kb0 + STEP, kp1, vp1);
    if (kb0 < k_hi) issue_k(kb0, kp);
  }

  // this lane's row of the tile
  const int rr = t.row0 + r16;
  const bool rok = rr < t.n * a.R;
  const int tok = rok ? by_r(a, rr) : 0, h = g * a.R + (rok ? mod_r(a, rr) : 0);
  const int pos = t.pos0 + tok;
  // it sees keys [see_lo, see_hi)
  const int see_hi = rok ? (a.causal ? min(t.len, pos + 1) : t.len) : 0;
  const int see_lo = a.window > 0 ? (int)max(0LL, (long long)pos - a.window + 1) : 0;
  uint4 qf[L::QK];
  const E* qp = reinterpret_cast<const E*>(a.q) + (size_t)(t.s0 + tok) * a.ldq + (size_t)h * HD;
#pragma unroll
  for (int c = 0; c < L::QK; ++c) qf[c] = rok ? ldg16(qp + L::qdim(c, g4)) : make_uint4(0, 0, 0, 0);
  // every row of the tile sees every key in [all_lo, all_hi)
  const int i1 = min(t.n - 1, by_r(a, t.row0 + 15));
  const int all_hi = min(k_hi, a.causal ? min(t.len, t.pos0 + by_r(a, t.row0) + 1) : t.len);
  const int all_lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + i1 - a.window + 1) : 0;

  f32x4 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x4{0.f, 0.f, 0.f, 0.f};
  float mrun = -INFINITY, lrun = 0.0f;
  bool rare = false;   // V values that are not finite were taken out of a product
  const float sc = score_factor(a);

  auto block = [&](int kb, KvBlock<TYPE, HD>& x) {
    const int vk0 = kb + 8 * g4;
    // some row does not see some key, or a page is not there
    const bool part = !(kb >= all_lo && kb + 32 <= all_hi) || __any(x.vpid < 0);
    f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < L::NK; ++c) {
      if constexpr (L::ES == 1) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) mma16(s[tt], codes_bf16<TYPE>(x.k[tt][c].x, x.k[tt][c].y), qf[2 * c], bf16_t());
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) mma16(s[tt], codes_bf16<TYPE>(x.k[tt][c].z, x.k[tt][c].w), qf[2 * c + 1], bf16_t());
      } else {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) mma16(s[tt], x.k[tt][c], qf[c], E());
      }
    }
    // lane: keys vk0 + j of row r16
    const float ks[8] = {x.ks[0].x, x.ks[0].y, x.ks[0].z, x.ks[0].w, x.ks[1].x, x.ks[1].y, x.ks[1].z, x.ks[1].w};
    const float vs[8] = {x.vs[0].x, x.vs[0].y, x.vs[0].z, x.vs[0].w, x.vs[1].x, x.vs[1].y, x.vs[1].z, x.vs[1].w};
    float w[8];
    unsigned hid = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = L::ES == 1 ? s[j >> 2][j & 3] * ks[j] : s[j >> 2][j & 3];
    turn_scores(a, w);
    if (part) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = vk0 + j;
        const bool vis = key < see_hi && key >= see_lo && key < k_hi;
        // a key on a page outside the pool is NaN where it is seen
        w[j] = vis ? (x.vpid < 0 ? NAN : w[j]) : -INFINITY;
        hid |= vis ? 0u : 1u << j;
      }
    }
    float bmax = w[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) bmax = fmaxf(bmax, w[j]);
    bmax *= sc;
    // The reference moves only when a score exceeds it by more than 2^8: the
    // exponentials stay below 256, most blocks need no rescaling, and until
    // then no lane needs the others' maximum.
    if (__any(bmax > mrun + 8.0f)) {
      bmax = groups_max(bmax);
      const bool move = bmax > mrun + 8.0f;
      const float mnew = move ? bmax : mrun;
      const float corr = move ? __builtin_amdgcn_exp2f(mrun - mnew) : 1.0f;
      lrun *= corr;
      mrun = mnew;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= corr;
    }
    const float mref = mrun == -INFINITY ? 0.0f : mrun;   // no visible key so far: weight 0
    float psum = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = __builtin_amdgcn_exp2f(fmaf(w[j], sc, -mref));
      psum += w[j];
    }
    if constexpr (L::ES == 1) {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[j] *= vs[j];
      if (part) {   // a hidden key's scale may be NaN
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = hid >> j & 1 ? 0.0f : w[j];
      }
    }
    lrun += psum;   // this lane's keys
    if (part) {
      // Keys past the split or without a page are not what their registers hold.
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (x.vpid < 0 || vk0 + j >= k_hi) {
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) x.v[j][hh] = VecOf<L::VB>{};
        }
      if constexpr (TYPE != VLA_KV_I8) {
        // A NaN or an infinity in V must not reach the rows that do not see its
        // key, and 0 times it would: such values are taken out of the product
        // and added to the rows that see them at the end (see add_not_finite).
        bool bad = false;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
          for (int hh = 0; hh < NH; ++hh) bad |= v_bad<TYPE>(x.v[j][hh]);
        if (__any(bad)) {
          rare = true;
#pragma unroll
          for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int hh = 0; hh < NH; ++hh) v_clean<TYPE>(x.v[j][hh]);
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
            o[hh * VE + e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[j][hh].w[e]), w[j], o[hh * VE + e], 0, 0, 0);
    } else {
      const uint4 pb = make_uint4(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7]));
#pragma unroll
      for (int hh = 0; hh < NH; ++hh)
#pragma unroll
        for (int e = 0; e < VE; ++e) {
          uint32_t vt[4];
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) {
            if constexpr (TYPE == VLA_KV_BF16)
              vt[jj] = __builtin_amdgcn_perm(x.v[2 * jj + 1][hh].w[e >> 1], x.v[2 * jj][hh].w[e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
            else
              vt[jj] = pack_bf16x2(v_value<TYPE>(x.v[2 * jj][hh], e), v_value<TYPE>(x.v[2 * jj + 1][hh], e));
          }
          mma16(o[hh * VE + e], make_uint4(vt[0], vt[1], vt[2], vt[3]), pb, bf16_t());
        }
    }
  };

  for (int kb = kb0; kb < k_hi; kb += STEP) {
    if constexpr (KR::USED) {
      // This block's K rows have landed: they were loaded before the last block's V.
      __builtin_amdgcn_s_waitcnt(vm_wait(0));
      asm volatile("" : : : "memory");
#pragma unroll
      for (int tt = 0; tt < 2; ++tt)
#pragma unroll
        for (int c = 0; c < L::NK; ++c) {
          const int key = 8 * (r16 >> 2) + 4 * tt + (r16 & 3);
          buf.k[tt][c] = *reinterpret_cast<const uint4*>(mine + key * KR::RB + 16 * ((4 * c + g4) ^ KR::slot(key)));
        }
      asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");   // before the next ones overwrite them
      if (kb + STEP < k_hi) issue_k(kb + STEP, kp1);
      const int vnow = vp;
      vp = vp1;
      pids(kb + 2 * STEP, kp1, vp1);
      load_v(kb, vnow, buf);
    } else {
      load_k(kb, kp, buf);
      load_v(kb, vp, buf);
      pids(kb + STEP, kp, vp);
    }
    block(kb, buf);
  }

  if constexpr (TYPE != VLA_KV_I8) {
    if (rare) {
      for (int kb = kb0; kb < k_hi; kb += STEP)
        if (!(kb >= all_lo && kb + 32 <= all_hi))
          add_not_finite<TYPE, HD>(p, table, g, kb, min(kb + 32, k_hi), see_lo, see_hi, o,
                                   [&](int d, int i) { return d / VE * 16 * VE + (4 * g4 + i) * VE + d % VE; });
    }
  }

  // Join the waves that had keys: tile d, row 4 g4 + i, column r16 of each.
  const int nact = max(1, min(W, (k_hi - k_lo + 31) / 32));
  lrun = t.beyond ? NAN : groups_sum(lrun);
  if (g4 == 0) {
    sm[wave][r16] = mrun;
    sl[wave][r16] = lrun;
  }
  if (wave < nact) {
#pragma unroll
    for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(mine + 1024 * d + 16 * lane) = o[d];
  }
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
  // Row 4 g4 + i of tile (hh, e) is dimension hh 16 VE + (4 g4 + i) VE + e: a
  // wave's DW = DT / 4 tiles are DW neighbouring dimensions, for each i.
  constexpr int DW = DT / W;
  const int d0 = wave * DW, dim0 = d0 / VE * 16 * VE + d0 % VE;
  f32x4 v[DW];
#pragma unroll
  for (int d = 0; d < DW; ++d) {
    v[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < W; ++w)
      if (w < nact) v[d] += *reinterpret_cast<const f32x4*>(lds[w] + 1024 * (d0 + d) + 16 * lane) * f[w];
    v[d] *= inv;
  }
  float* pd = a.part + ((size_t)split * p.T * a.H + th) * HD + dim0;
  E* od = reinterpret_cast<E*>(a.o) + (size_t)(t.s0 + tok) * a.ldo + (size_t)h * HD + dim0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float x[DW];
#pragma unroll
    for (int d = 0; d < DW; ++d) x[d] = v[d][i];
    if (!whole) put<float, DW>(pd + (4 * g4 + i) * VE, x);
    else put<E, DW>(od + (4 * g4 + i) * VE, x);
  }
}

// ---------------------------------------------------------------------------
// paged_tile: many rows per request (prompts, action chunks).  A workgroup of
// NW waves takes 16 RS NW rows, RS subtiles of 16 per wave, and walks its keys
// in blocks of 64 that are staged in LDS as bf16 (8-bit codes are widened once
// for all rows) and serve every row:
//   K [64 keys][HD]  16-byte chunk c of key k at slot kslot(c, k)
//   V [64 keys][HD]  16-byte chunk c of key k at slot vslot(c, k)
// The slots keep apart modulo 16 (the 64 banks of LDS) the sixteen keys of a
// score operand (8 i + j, i, j < 4, one chunk), the sixteen pieces of a
// transposing read (keys 8 i + j, i < 2, j < 4, two chunks), and what sixteen
// lanes write: chunks of bf16 rows, or the even (odd) chunks of 8-bit rows.
// V^T operands come from ds_read_b64_tr_b16: within 16 lanes, lane i receives
// element i % 4 of the 8-byte blocks addressed by lanes i / 4, i / 4 + 4, + 8
// and + 12, so lane p of group g addresses key 8 g + p / 4 (+ 4 for the second
// read) at dimensions 16 d + 4 (p % 4) and gets four consecutive keys of
// dimension 16 d + p; vswz puts the four keys of a read in disjoint banks.
// An operand from LDS feeds RS MFMAs.  The next block's rows are on their way
// in registers, and the page ids of the one after that, while a block is
// worked on; LDS is double-buffered, one barrier per block.
template <int HD>
VLA_DEV int kslot(int c, int k) {
  if constexpr (HD == 64) return c ^ ((k >> 1 & 1) | (k >> 2 & 6));   // (two rows to 256 bytes)
  return c ^ (c >> 4) ^ ((k & 3) | (k >> 1 & 12));
}
template <int HD>
VLA_DEV int vslot(int c, int k) {
  if constexpr (HD == 64) return c ^ ((k >> 1 & 1) * 3 | (k >> 1 & 4));
  return c ^ (c >> 4) ^ ((k & 1) | (k & 3) << 1 | (k & 8));
}

constexpr int TKB = 64;   // keys per block

template <int TYPE, int HD, int RS, int NW>
struct TileShape {
  static constexpr int ROWS = 16 * RS * NW, THR = 64 * NW;
  static constexpr int ES = type_bytes(TYPE);
  static constexpr int VPR = HD * ES / 16;            // 16-byte vectors of a stored row
  static constexpr int LD = TKB * VPR / THR;          // of them per thread and block (K; V the same)
  static constexpr int KPW = 64 / VPR, KPL = THR / VPR;   // keys of a wave's load, keys of all waves' load
  static constexpr int CPR = HD / 8;                  // 16-byte chunks of a staged row
  static constexpr int BUF = 2 * TKB * CPR;           // chunks per buffer: K, then V
  static_assert(LD * THR == TKB * VPR && KPW <= 16, "staging");
};

template <int TYPE, int HD, int RS, int NW, int OCC>
__global__ __launch_bounds__(64 * NW, OCC) void paged_tile(PagedAttnArgs a) {
  using S = TileShape<TYPE, HD, RS, NW>;
  constexpr int LD = S::LD, CPR = S::CPR, NQV = HD / 32, DT = HD / 16, ES = S::ES;
  __shared__ uint4 st[2][S::BUF];
  __shared__ __align__(16) float scl[2][2][TKB];   // 8-bit types: scales of the block's keys, K (times sc) and V
  __shared__ int rare;                         // V values that are not finite were taken out of a product

  const PageArgs& p = a.p;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, g4 = lane >> 4;
  const int units = a.slots * p.G * a.nsplit;
  int u = a.by_xcd ? (int)(blockIdx.x % 8u) * (int)(gridDim.x / 8u) + (int)(blockIdx.x / 8u) : (int)blockIdx.x;
  if (u >= units) return;
  const int inner = a.by_xcd ? a.slots : p.G, i0 = u % inner;
  u /= inner;
  const int split = u % a.nsplit, outer = u / a.nsplit;
  const int slot = a.by_xcd ? i0 : outer, g = a.by_xcd ? outer : i0;
  Tile t;
  if (!paged_tile_of<S::ROWS>(a, slot, t)) return;
  int k_lo, k_hi;
  tile_keys(a, t, S::ROWS, split, k_lo, k_hi);
  if (empty_split(a, t, S::ROWS, g, split, k_lo, k_hi)) return;

  const int* table = p.table + (size_t)t.b * p.max_pages;
  const size_t pagerows = (size_t)1 << p.lg;
  const int mask = (1 << p.lg) - 1;
  const float sc = a.scale * kLog2e;
  // rows of the tile that see every key in [all_lo, all_hi): of tokens i0 .. i1
  auto all_of = [&](int row, int rows, int& lo, int& hi) {
    const int i0 = by_r(a, row), i1 = min(t.n - 1, by_r(a, row + rows - 1));
    hi = a.causal ? min(t.len, t.pos0 + i0 + 1) : t.len;
    lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + i1 - a.window + 1) : 0;
  };
  int tile_lo, tile_hi;   // every row of the tile sees these
  all_of(t.row0, S::ROWS, tile_lo, tile_hi);

  // Pages of a block's four groups of 16 keys, group lane / 16 in each lane: -1
  // past the split, -2 outside the pool.
  auto pages = [&](int kb) {
    const int key = kb + 16 * g4;
    int pid = -1;
    if (key < k_hi) {
      pid = table[key >> p.lg];
      if ((unsigned)pid >= (unsigned)p.n_pages) pid = -2;
    }
    return pid;
  };
  // The keys that load i of this wave brings are of one group.
  const int key0 = wave * S::KPW, lkey = lane / S::VPR, lvec = lane % S::VPR;
  auto page_of_load = [&](int pg, int i) { return __builtin_amdgcn_readlane(pg, (key0 + S::KPL * i) & 48); };
  const unsigned pstride = (unsigned)p.G << p.lg;   // rows of a page (of all heads); times the row's bytes below 2^29
  const char* kbase = reinterpret_cast<const char*>(p.k) + ((size_t)g << p.lg) * (HD * ES) + lane * 16;
  const char* vbase = reinterpret_cast<const char*>(p.v) + ((size_t)g << p.lg) * (HD * ES) + lane * 16;
  uint4 kr[LD], vr[LD];
  float sreg = 0.0f;           // one scale of the block in the registers: thread key (K) or 64 + key (V)
  auto load = [&](int kb, int pg) {
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int key = kb + key0 + S::KPL * i;
      const size_t off = (size_t)(unsigned)max(page_of_load(pg, i), 0) * (pstride * (HD * ES)) + (unsigned)(key & mask) * (HD * ES);
      kr[i] = ldg16(kbase + off);
      vr[i] = ldg16(vbase + off);
    }
    if constexpr (ES == 1) {
      if (wave < 2) {          // lane: key kb + lane, of page group lane / 16
        const size_t row = ((size_t)max(pg, 0) * p.G + g) * pagerows + ((kb + lane) & mask);
        sreg = (wave == 0 ? p.ks : p.vs)[row];
        if (wave == 0) sreg = pg == -2 ? NAN : sreg * sc;
        else if (pg < 0) sreg = 0.0f;
      }
    }
  };
  // registers -> LDS buffer b
  auto stage = [&](int kb, int b, int pg) {
    // some row does not see some key, or a page is not there
    const bool part = !(kb >= tile_lo && kb + TKB <= min(tile_hi, k_hi)) || __any(pg < 0);
    bool bad = false;
#pragma unroll
    for (int i = 0; i < LD; ++i) {
      const int k = key0 + S::KPL * i + lkey;    // key of the block
      uint4 v = vr[i];
      if (part && (page_of_load(pg, i) < 0 || kb + k >= k_hi)) v = make_uint4(0, 0, 0, 0);   // not what the registers hold
      if constexpr (TYPE != VLA_KV_I8) {
        if (part) {
          VecOf<16> x{{v.x, v.y, v.z, v.w}};
          if (v_bad<TYPE>(x)) {
            bad = true;
            v_clean<TYPE>(x);
            v = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
          }
        }
      }
      uint4* kl = st[b] + k * CPR;
      uint4* vl = st[b] + (TKB + k) * CPR;
      if constexpr (ES == 1) {
        kl[kslot<HD>(2 * lvec, k)] = codes_bf16<TYPE>(kr[i].x, kr[i].y);
        kl[kslot<HD>(2 * lvec + 1, k)] = codes_bf16<TYPE>(kr[i].z, kr[i].w);
        vl[vslot<HD>(2 * lvec, k)] = codes_bf16<TYPE>(v.x, v.y);
        vl[vslot<HD>(2 * lvec + 1, k)] = codes_bf16<TYPE>(v.z, v.w);
      } else {
        kl[kslot<HD>(lvec, k)] = kr[i];
        vl[vslot<HD>(lvec, k)] = v;
      }
    }
    if constexpr (ES == 1) {
      if (wave < 2) scl[b][wave][lane] = sreg;
    }
    if constexpr (TYPE != VLA_KV_I8) {
      if (part && __any(bad) && lane == 0) rare = 1;
    }
  };

  // this lane's rows
  int see_lo[RS], see_hi[RS];
  uint4 qf[RS][NQV];
  const int wrow = t.row0 + wave * 16 * RS;
  int wave_lo, wave_hi;   // every row of the wave sees these
  all_of(wrow, 16 * RS, wave_lo, wave_hi);
  // and none sees a key from here on, or before
  const int w1 = min(t.n - 1, by_r(a, wrow + 16 * RS - 1)), w0 = by_r(a, wrow);
  const int none_hi = wrow >= t.n * a.R ? 0 : a.causal ? min(t.len, t.pos0 + w1 + 1) : t.len;
  const int none_lo = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + w0 - a.window + 1) : 0;
#pragma unroll
  for (int s = 0; s < RS; ++s) {
    const int rr = wrow + 16 * s + r16;
    const bool rok = rr < t.n * a.R;
    const int tok = rok ? by_r(a, rr) : 0, h = g * a.R + (rok ? mod_r(a, rr) : 0);
    see_hi[s] = rok ? (a.causal ? min(t.len, t.pos0 + tok + 1) : t.len) : 0;
    see_lo[s] = a.window > 0 ? (int)max(0LL, (long long)t.pos0 + tok - a.window + 1) : 0;
    const bf16_t* qp = reinterpret_cast<const bf16_t*>(a.q) + (size_t)(t.s0 + tok) * a.ldq + (size_t)h * HD + g4 * (HD / 4);
#pragma unroll
    for (int c = 0; c < NQV; ++c) qf[s][c] = rok ? ldg16(qp + 8 * c) : make_uint4(0, 0, 0, 0);
  }
  // LDS operand places of this lane: score row r16 is key 32 kk + 4 tt + 8 (r16
  // / 4) + r16 % 4 (the slots of a chunk do not depend on kk and tt), and chunk
  // g4 NQV + c of it.
  const int kkey = 8 * (r16 >> 2) + (r16 & 3);
  int kat[NQV];
#pragma unroll
  for (int c = 0; c < NQV; ++c) kat[c] = kkey * CPR + kslot<HD>(g4 * NQV + c, kkey);
  // V^T reads of dim tile d: key 8 g4 + r16 / 4 (+ 4, + 32: the same slots), chunk 2 d + (r16 % 4) / 2
  int vat[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) {
    const int k = 8 * g4 + (r16 >> 2);
    vat[d] = k * HD * 2 + vslot<HD>(2 * d + ((r16 & 3) >> 1), k) * 16 + (r16 & 1) * 8;
  }

  f32x4 o[RS][DT];
  float mref[RS], limit[RS], lrun[RS];   // reference of the exponentials; how far above it a score may be
#pragma unroll
  for (int s = 0; s < RS; ++s) {
    mref[s] = 0.0f;
    limit[s] = -INFINITY;
    lrun[s] = 0.0f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[s][d] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // this lane's keys' scales (32 kk + 8 g4 + j of the block)
  auto scales = [&](const float* from, float (&to)[16]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float4 v = *reinterpret_cast<const float4*>(from + 32 * (q >> 1) + 8 * g4 + 4 * (q & 1));
      to[4 * q] = v.x; to[4 * q + 1] = v.y; to[4 * q + 2] = v.z; to[4 * q + 3] = v.w;
    }
  };
  auto block = [&](int kb, int b, int pg) {
    if (kb >= none_hi || kb + TKB <= none_lo) return;
    const uint4* kl = st[b];
    const unsigned char* vl = reinterpret_cast<const unsigned char*>(st[b] + TKB * CPR);
    f32x4 s[RS][2][2];
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) s[r][kk][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < NQV; ++c)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const uint4 kv = kl[kat[c] + (32 * kk + 4 * tt) * CPR];
#pragma unroll
          for (int r = 0; r < RS; ++r) mma16(s[r][kk][tt], kv, qf[r][c], bf16_t());
        }
    // some row of the wave does not see some key, or a page is not there
    const bool part = !(kb >= wave_lo && kb + TKB <= min(wave_hi, k_hi)) || __any(pg < 0);
    uint4 pb[RS][2];
    float w[RS][16], kv[16];
    unsigned hid[RS];
    // scores less the reference (base 2): one operation each
    if constexpr (ES == 1) scales(scl[b][0], kv);
#pragma unroll
    for (int r = 0; r < RS; ++r)
#pragma unroll
      for (int i = 0; i < 16; ++i) w[r][i] = fmaf(s[r][i >> 3][i >> 2 & 1][i & 3], ES == 1 ? kv[i] : sc, -mref[r]);
    if (part) {
      int gp[2];      // pages of this lane's keys
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) gp[kk] = __shfl(pg, 16 * (2 * kk + (g4 >> 1)), 64);
#pragma unroll
      for (int r = 0; r < RS; ++r) {
        hid[r] = 0;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = kb + 32 * (i >> 3) + 8 * g4 + (i & 7);
          const bool vis = key < see_hi[r] && key >= see_lo[r] && key < k_hi;
          w[r][i] = vis ? (gp[i >> 3] == -2 ? NAN : w[r][i]) : -INFINITY;
          hid[r] |= vis ? 0u : 1u << i;
        }
      }
    }
    if constexpr (ES == 1) scales(scl[b][1], kv);
#pragma unroll
    for (int r = 0; r < RS; ++r) {
      float bmax = w[r][0];
#pragma unroll
      for (int i = 1; i < 16; ++i) bmax = fmaxf(bmax, w[r][i]);
      // The reference moves as in paged_stream, and from the first visible key on
      // (limit is 8, before that -infinity); until then no lane needs the others'
      // maximum.
      if (__any(bmax > limit[r])) {
        bmax = groups_max(bmax);
        if (bmax > limit[r]) {
          const float corr = limit[r] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(-bmax);
          limit[r] = 8.0f;
          mref[r] += bmax;
          lrun[r] *= corr;
#pragma unroll
          for (int d = 0; d < DT; ++d) o[r][d] *= corr;
#pragma unroll
          for (int i = 0; i < 16; ++i) w[r][i] -= bmax;
        }
      }
      float psum = 0.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        w[r][i] = __builtin_amdgcn_exp2f(w[r][i]);
        psum += w[r][i];
      }
      lrun[r] += psum;   // this lane's keys
      if constexpr (ES == 1) {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[r][i] *= kv[i];
        if (part) {   // a hidden key's scale may be NaN
#pragma unroll
          for (int i = 0; i < 16; ++i) w[r][i] = hid[r] >> i & 1 ? 0.0f : w[r][i];
        }
      }
#pragma unroll
      for (int kk = 0; kk < 2; ++kk)
        pb[r][kk] = make_uint4(pack_bf16x2(w[r][8 * kk], w[r][8 * kk + 1]), pack_bf16x2(w[r][8 * kk + 2], w[r][8 * kk + 3]),
                               pack_bf16x2(w[r][8 * kk + 4], w[r][8 * kk + 5]), pack_bf16x2(w[r][8 * kk + 6], w[r][8 * kk + 7]));
    }
    typedef short v4s_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4s_t lds_v4s;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        const unsigned char* ap = vl + vat[d] + kk * 32 * HD * 2;
        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(ap)));
        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(ap + 4 * HD * 2)));
#pragma unroll
        for (int r = 0; r < RS; ++r) mma16(o[r][d], make_uint4(lo.x, lo.y, hi.x, hi.y), pb[r][kk], bf16_t());
      }
  };

  if (tid == 0) rare = 0;
  int pg0 = pages(k_lo), pg1 = pages(k_lo + TKB);   // of the block in LDS, of the next one
  load(k_lo, pg0);
  __syncthreads();
  stage(k_lo, 0, pg0);
  for (int kb = k_lo, b = 0; kb < k_hi; kb += TKB, b ^= 1) {
    const bool more = kb + TKB < k_hi;
    if (more) load(kb + TKB, pg1);
    const int pg2 = pages(kb + 2 * TKB);
    __syncthreads();          // buffer b is staged, and b ^ 1 no longer read
    block(kb, b, pg0);
    if (more) stage(kb + TKB, b ^ 1, pg1);
    pg0 = pg1;
    pg1 = pg2;
  }

  if constexpr (TYPE != VLA_KV_I8) {
    __syncthreads();
    if (rare) {
      for (int kb = k_lo; kb < k_hi; kb += TKB)
        if (!(kb >= tile_lo && kb + TKB <= min(tile_hi, k_hi))) {
#pragma unroll
          for (int s = 0; s < RS; ++s)
            add_not_finite<TYPE, HD>(p, table, g, kb, min(kb + TKB, k_hi), see_lo[s], see_hi[s], o[s],
                                     [&](int d, int i) { return 16 * d + 4 * g4 + i; });
        }
    }
  }

  float lsum[RS], mrun[RS];
#pragma unroll
  for (int s = 0; s < RS; ++s) {
    lsum[s] = groups_sum(lrun[s]);
    mrun[s] = limit[s] == -INFINITY ? -INFINITY : mref[s];
  }
  // lane holds O^T[dim 16 d + 4 g4 + i][row r16] of each subtile
  const bool whole = a.nsplit == 1;
#pragma unroll
  for (int s = 0; s < RS; ++s) {
    const int rr = wrow + 16 * s + r16;
    if (rr >= t.n * a.R) continue;
    const int tok = by_r(a, rr), h = g * a.R + mod_r(a, rr);
    const size_t th = (size_t)(t.s0 + tok) * a.H + h;
    const float tot = t.beyond ? NAN : lsum[s];
    if (g4 == 0) {
      if (!whole) *reinterpret_cast<float2*>(a.stats + ((size_t)split * p.T * a.H + th) * 2) = make_float2(mrun[s], tot);
      else if (a.lse) a.lse[th] = (mrun[s] + __log2f(tot)) * kLn2;
    }
    const float inv = whole ? (tot == 0.0f ? 0.0f : 1.0f / tot) : 1.0f;
    float* pd = a.part + ((size_t)split * p.T * a.H + th) * HD + 4 * g4;
    bf16_t* od = reinterpret_cast<bf16_t*>(a.o) + (size_t)(t.s0 + tok) * a.ldo + (size_t)h * HD + 4 * g4;
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const float x[4] = {o[s][d][0] * inv, o[s][d][1] * inv, o[s][d][2] * inv, o[s][d][3] * inv};
      if (!whole) put<float, 4>(pd + 16 * d, x);
      else put<bf16_t, 4>(od + 16 * d, x);
    }
  }
}

// Joins the splits of one (token, head) per wave: o = sum_s 2^(m_s - m) o_s /
// sum_s 2^(m_s - m) l_s.  Lane s weighs split s; the outputs of a split that
// saw no key are not read (they may not have been written).
template <int F32, int HD>
__global__ __launch_bounds__(256) void paged_join(PagedAttnArgs a) {
  using E = std::conditional_t<F32, float, bf16_t>;
  constexpr int V = HD / 64;   // values per lane
  const PageArgs& p = a.p;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const long long th = (long long)blockIdx.x * 4 + wave;
  const long long all = (long long)p.T * a.H;
  if (th >= all) return;
  const int t = (int)(th / a.H), h = (int)(th - (long long)t * a.H);
  const float2 st = lane < a.nsplit ? *reinterpret_cast<const float2*>(a.stats + ((size_t)lane * all + th) * 2)
                                    : make_float2(-INFINITY, 0.0f);
  if (t < p.starts[0] || t >= p.starts[p.B]) return;   // padding
  const bool any = st.y != 0.0f;
  const float mx = wave_max(any ? st.x : -INFINITY);
  const float mref = mx == -INFINITY ? 0.0f : mx;
  const float f = any ? __builtin_amdgcn_exp2f(st.x - mref) : 0.0f;
  const float tot = wave_sum(any ? st.y * f : 0.0f);
  const unsigned long long live = __ballot(any);
  float acc[V] = {};
  constexpr int U = 8;
  for (int s0 = 0; s0 < a.nsplit; s0 += U) {
    float v[U][V];
#pragma unroll
    for (int j = 0; j < U; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) v[j][i] = 0.0f;
      if (s0 + j < 64 && (live >> (s0 + j) & 1)) {
        const VecOf<4 * V> x = ldgv<4 * V>(a.part + ((size_t)(s0 + j) * all + th) * HD + lane * V);
#pragma unroll
        for (int i = 0; i < V; ++i) v[j][i] = __uint_as_float(x.w[i]);
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), min(s0 + j, 63)));
#pragma unroll
      for (int i = 0; i < V; ++i) acc[i] += v[j][i] * w;
    }
  }
  const float inv = tot == 0.0f ? 0.0f : 1.0f / tot;
  E* dst = reinterpret_cast<E*>(a.o) + (size_t)t * a.ldo + (size_t)h * HD + lane * V;
#pragma unroll
  for (int i = 0; i < V; ++i) dst[i] = ElemTraits<E>::from_f(acc[i] * inv);
  if (lane == 0 && a.lse) a.lse[th] = (mx + __log2f(tot)) * kLn2;
}

template <int TYPE, int HD>
hipError_t stream_launch(const PagedAttnArgs& a, hipStream_t s) {
  const long long units = (long long)a.slots * a.p.G * a.nsplit;
  hipLaunchKernelGGL((paged_stream<TYPE, HD>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <int TYPE, int HD, int RS, int NW, int OCC>
hipError_t tile_launch(const PagedAttnArgs& a, hipStream_t s) {
  const long long units = (long long)a.slots * a.p.G * a.nsplit;
  hipLaunchKernelGGL((paged_tile<TYPE, HD, RS, NW, OCC>), dim3((unsigned)((units + 7) / 8 * 8)), dim3(64 * NW), 0, s, a);
  return hipGetLastError();
}

template <int TYPE>
hipError_t tile_hd(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.hd) {
    case 64: return tile_launch<TYPE, 64, 2, 4, 2>(a, s);
    case 128: return tile_launch<TYPE, 128, 2, 4, 2>(a, s);
    case 256: return tile_launch<TYPE, 256, 1, 8, 2>(a, s);
  }
  return hipErrorInvalidValue;
}

template <int TYPE>
hipError_t stream_hd(const PagedAttnArgs& a, hipStream_t s) {
  switch (a.p.hd) {
    case 64: return stream_launch<TYPE, 64>(a, s);
    case 128: return stream_launch<TYPE, 128>(a, s);
    case 256: if constexpr (TYPE != VLA_KV_BF16) return stream_launch<TYPE, 256>(a, s);   // (bf16: tiles, see the plan)
  }
  return hipErrorInvalidValue;
}

}  // namespace

// The split counts that are tried: all up to 8, then in steps of a fourth, and the last.
static long long next_split(long long k, long long end) {
  return k == end ? end + 1 : std::min(end, k + (k < 8 ? 1 : k / 4));
}

void paged_attention_plan(PagedAttnArgs& a, long long span, int most) {
  a.rdiv = ((1ull << 32) + a.R - 1) / a.R;
  const long long rows = (long long)a.p.T * a.R, B = std::max(1, a.p.B), G = a.p.G;
  // The 128-row tile reads a key once for all rows, but a request with few rows
  // leaves most of its waves without work: from 32 rows per request where the
  // tiles are a round of the chip at most (8 requests, 38 rows over 2000 keys:
  // 22.6 us against 24.0), else from 96 (64 requests over 4000 keys of 128: 66
  // rows 165 us against 139, 104 rows 185 against 192).  bf16 rows of 256 take a
  // stream wave's registers twice over; the tile is faster at any number (16 x 1
  // token of 8 heads over 16000 keys: 57 us against 87).
  const long long tiles = (rows / 128 + B) * G, fit = a.p.hd == 256 ? 256 : 512;
  const bool tile = a.p.type != VLA_KV_F32 && ((a.p.type == VLA_KV_BF16 && a.p.hd == 256) || rows >= (2 * tiles <= fit ? 32 : 96) * B);
  a.rows = tile ? 128 : 16;
  a.slots = (int)(rows / a.rows) + a.p.B;
  const long long base = std::max(1LL, a.slots * G);
  long long n;
  if (!tile) {
    // The splits of least estimated time.  A workgroup begins and ends in some 6 us
    // and takes 0.5 us and its bytes' time for each 128 keys (fp32: its products'
    // time), one after the other; together they take as long as memory needs, the
    // longest ones' last third, when they do not fill it any more, and 3.5 us per
    // workgroup of a full chip; a join is a launch of 6.5 us.  64 requests of up to
    // 8192 rows of int8: 114 us whole, 93 in four splits, 96 in eight, 130 in 32; one:
    // 66 whole, 13 in 24; 32 of 1000 rows: 14 whole, 16 in four.
    const double bytes = a.p.hd * (a.p.type == VLA_KV_BF16 ? 4.0 : a.p.type == VLA_KV_F32 ? 8.0 : 2.0) + (a.p.type >= VLA_KV_I8 ? 8.0 : 0.0);
    const double chain = span / 128.0 * (a.p.type == VLA_KV_F32 ? a.p.hd * 0.02 : 0.5 + 0.0018 * bytes);
    const double memory = (B == 1 ? 1.0 : 0.6) * span * B * G * bytes / 4.2e6, out_us = (double)rows * G * a.p.hd * 8 / 5e6;
    const double fit = 256.0 * stream_occupancy(a.p.type, a.p.hd), units = std::max((double)B, rows / 16.0 + 0.5 * B) * G;
    const long long end = std::min((span + 31) / 32, (long long)most);
    double least = 0.0;
    n = 1;
    for (long long k = 1; k <= end; k = next_split(k, end)) {
      const double load = units * k / fit, alone = std::max(1.0, B == 1 ? load : 0.75 * load) * (chain / k + 6.0);
      const double us = std::max(alone, memory + 0.35 * chain / k + 3.5 * load) + (k > 1 ? 6.5 + k * (0.05 + out_us) : 0.0);
      if (k == 1 || us < least) n = k, least = us;
    }
  } else {
    // The splits of least estimated time: rounds of the workgroups that fit, each
    // of its blocks of 64 keys (measured: 1.75, 2.5, 3 us at 64, 128, 256) and what
    // it begins and ends with, then the splits' outputs, written and read in fp32
    // (about 5 TB/s), and a launch.  The tiles of one request are alike and take
    // whole rounds (2048 tokens over 8192 rows, 325 tiles: 321 us whole, 294 in two
    // splits, 236 in three, 263 in four); of several, some 75% of the tiles' keys
    // are there, and half a round passes at the end (three prompts of up to 10007
    // rows, 715 tiles: 600 us whole, 520 in three or four; 24 of 21 tokens over 9787
    // rows of 64: 265 whole, 151 in two, 98 in eight; 8 x 50 tokens of 8 heads over
    // 866 rows of 256: 36 whole, 23 in five to seven, 31 in eight).
    const double block_us = a.p.hd == 64 ? 1.75 : a.p.hd == 128 ? 2.5 : 3.0, ends_us = a.p.hd == 256 ? 6.0 : 2.0;
    const double out_us = (double)rows * G * a.p.hd * 8 / 5e6;
    const double tiles_of_all = std::max((double)B, rows / 128.0 + 0.5 * B) * G;   // (a tile slot may be empty)
    const long long end = std::min({std::max(8LL, fit / base), (span + 63) / 64, (long long)most});
    double least = 0.0;
    n = 1;
    const long long blocks = (span + 63) / 64;
    for (long long t = 1; t <= end; t = next_split(t, end)) {
      const long long each = (blocks + t - 1) / t, k = each > 0 ? (blocks + each - 1) / each : 1;   // splits of whole blocks
      const double load = tiles_of_all * k / fit;
      const double rounds = load <= 1.0 ? 1.0 : B == 1 ? std::ceil(load) : 0.75 * load + 0.5;
      const double us = rounds * (each * block_us + ends_us) + (k > 1 ? k * out_us + 3.0 : 0.0);
      if (t == 1 || us < least) n = k, least = us;
    }
  }
  a.nsplit = (int)n;
  // Tile kernel: consecutive tiles on one XCD read the same keys through its L2
  // (4 x 600 tokens over 4000 keys: 95 us, in turn over all XCDs 102).  In more
  // rounds, or more than one of whole tiles, which differ most in length, all
  // heads of the first requests go first, in turn over all XCDs (8 x 800 tokens
  // over 866 rows of 256: 146 us against 125; 6 x 1000 over 4000: 243, 220).
  a.by_xcd = a.nsplit > 1 ? base * a.nsplit <= 2 * fit : base <= fit;
  a.chunk = (int)((span + a.nsplit - 1) / a.nsplit + 31) & ~31;
  if (a.chunk < 32) a.chunk = 32;
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
    case VLA_KV_BF16: e = a.rows == 16 ? stream_hd<VLA_KV_BF16>(a, s) : tile_hd<VLA_KV_BF16>(a, s); break;
    case VLA_KV_I8: e = a.rows == 16 ? stream_hd<VLA_KV_I8>(a, s) : tile_hd<VLA_KV_I8>(a, s); break;
    case VLA_KV_E4M3: e = a.rows == 16 ? stream_hd<VLA_KV_E4M3>(a, s) : tile_hd<VLA_KV_E4M3>(a, s); break;
  }
  if (e != hipSuccess || a.nsplit == 1) return e;
  const long long rows = (long long)a.p.T * a.H;
  const dim3 grid((unsigned)((rows + 3) / 4));
  if (a.p.type == VLA_KV_F32) {
    if (a.p.hd == 64) hipLaunchKernelGGL((paged_join<1, 64>), grid, dim3(256), 0, s, a);
    else if (a.p.hd == 128) hipLaunchKernelGGL((paged_join<1, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_join<1, 256>), grid, dim3(256), 0, s, a);
  } else {
    if (a.p.hd == 64) hipLaunchKernelGGL((paged_join<0, 64>), grid, dim3(256), 0, s, a);
    else if (a.p.hd == 128) hipLaunchKernelGGL((paged_join<0, 128>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_join<0, 256>), grid, dim3(256), 0, s, a);
  }
  return hipGetLastError();
}
