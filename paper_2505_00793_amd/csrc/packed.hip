// Causal dual attention over packed sequences with grouped heads, for bf16 and
// float32 operands and head dimensions up to 128.
//
// Attention of one query head with scores S = s Q K^T over the tokens of its own
// sequence, causal mask, P = softmax(S) by rows, O = P V, and its tangent along
// (Qd, Kd, Vd) (the forward-mode half of the forward-over-reverse HVP, Section 2.2):
//   Sd = s (Qd K^T + Q Kd^T),  c = rowsum(P Sd),  Od = (P Sd) V + P Vd - c O.
// The forward keeps a running row maximum and sums over key blocks and saves
// log2 sum exp2 and c per query row.  The backward recomputes P and
// Pd = P (Sd - c) from them:
//   dP = dO V^T,  dPd = dOd V^T + dO Vd^T,
//   r = <dO, O>,  rd = <dOd, O> + <dO, Od>,
//   dS = s P (dP - r),  dSd = s (Pd (dP - r) + P (dPd - rd)),
//   dQ = dS K,  dQd = dSd K + dS Kd,  dK = dS^T Q,  dKd = dSd^T Q + dS^T Qd,
//   dV = P^T dO,  dVd = Pd^T dO + P^T dOd,
// in two passes, one per query tile (dQ, dQd; it also writes r and rd) and one per key
// tile (dK, dV and tangents, summed over the query heads that share the key head), so
// every output has one writer and every sum a fixed order.
//
// Tiles never straddle sequences: rows past a sequence's end are read as its last
// row and masked, so nothing of another sequence or of unused rows enters a product.
//
// Fragments.  A wave owns R = 16 or 32 rows (queries, or keys in the dK/dV pass) and
// lane l = R g + i holds row i; NG = 64 / R lane groups g.  Products are formed as
// C[a][b] = sum_k A[a][k] B[b][k] with b the lane's row: an operand fragment is the 8
// elements k = 8 g + 0..7 of 8 NG, and of R x R results the lane holds a =
// 4 NG (t / 4) + 4 g + t % 4 of its row.  So the scores of a 64-row block leave a lane
// with the values at 64-block rows idx(t) = 4 NG (t / 4) + 4 g + t % 4, eight of which
// are a fragment of the next product, over rows in that order; its other operand is
// read from the tile in the same order (tfrag), and probabilities never leave registers.
#include "packed.h"

#include <algorithm>

namespace mfmg {

namespace {

constexpr int KB = 64;   // rows of a block staged in LDS
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int R> struct AccT;
template <> struct AccT<16> { typedef f32x4 V; };
template <> struct AccT<32> { typedef f32x16 V; };

struct f32x8 {
  float v[8];
};
template <typename T> struct FragT;
template <> struct FragT<bf16_t> { typedef bf16x8 V; };
template <> struct FragT<float> { typedef f32x8 V; };

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const bf16x8& a, const bf16x8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// float32: element t of every lane group's eight is one instruction's contraction
__device__ __forceinline__ f32x4 mma(const f32x8& a, const f32x8& b, f32x4 c) {
#pragma unroll
  for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.v[t], b.v[t], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x16 mma(const f32x8& a, const f32x8& b, f32x16 c) {
#pragma unroll
  for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.v[t], b.v[t], c, 0, 0, 0);
  return c;
}

// LDS tile of KB rows of DH elements in 16-byte chunks, the chunk index XOR-swizzled by
// the row: sixteen rows read at one chunk, and four rows read at four neighbouring
// chunks (the transposing reads), fall on different banks.
template <typename T, int DH>
struct Tile {
  static constexpr int VE = Elem<T>::VE, NC = DH / VE;   // chunks of a row
  static constexpr int ELEMS = KB * DH;
  __device__ static __forceinline__ int at(int row, int chunk) {
    const int f = NC >= 16 ? ((row & 3) << 2) | ((row >> 2) & 3)
                           : (((row >> 1) & 1) << 2) | ((row >> 2) & 3);
    return row * DH + ((chunk ^ f) * VE);
  }
};

// KB rows starting at row0 (rows past `last` read as row `last`), columns past dh zero.
template <typename T, int DH, int NT>
__device__ __forceinline__ void stage(T* lds, const T* __restrict__ g, long ld, int row0, int last,
                                      int dh, int tid) {
  typedef Tile<T, DH> L;
#pragma unroll
  for (int k = 0; k < KB * L::NC / NT; ++k) {
    const int i = tid + NT * k, r = i / L::NC, ch = i % L::NC;
    uint4 v = make_uint4(0, 0, 0, 0);
    if (ch * L::VE < dh)
      v = *reinterpret_cast<const uint4*>(g + (long)min(row0 + r, last) * ld + ch * L::VE);
    *reinterpret_cast<uint4*>(lds + L::at(r, ch)) = v;
  }
}

// Fragment c of a row in global memory: elements 8 NG c + 8 g .. + 7, zero past dh.
template <int NG>
__device__ __forceinline__ bf16x8 gfrag(const bf16_t* p, int g, int c, int dh) {
  const int d = 8 * NG * c + 8 * g;
  if (d < dh) return *reinterpret_cast<const bf16x8*>(p + d);
  bf16x8 z;
#pragma unroll
  for (int t = 0; t < 8; ++t) z[t] = (__bf16)0.f;
  return z;
}
template <int NG>
__device__ __forceinline__ f32x8 gfrag(const float* p, int g, int c, int dh) {
  const int d = 8 * NG * c + 8 * g;
  f32x8 z;
#pragma unroll
  for (int t = 0; t < 8; ++t) z.v[t] = d < dh ? p[d + t] : 0.f;
  return z;
}

// The same of a row of an LDS tile.
template <int DH, int NG>
__device__ __forceinline__ bf16x8 frag(const bf16_t* lds, int row, int g, int c) {
  return *reinterpret_cast<const bf16x8*>(lds + Tile<bf16_t, DH>::at(row, NG * c + g));
}
template <int DH, int NG>
__device__ __forceinline__ f32x8 frag(const float* lds, int row, int g, int c) {
  typedef Tile<float, DH> L;
  f32x8 v;
  const f32x4 a = *reinterpret_cast<const f32x4*>(lds + L::at(row, 2 * (NG * c + g)));
  const f32x4 b = *reinterpret_cast<const f32x4*>(lds + L::at(row, 2 * (NG * c + g) + 1));
#pragma unroll
  for (int t = 0; t < 4; ++t) { v.v[t] = a[t]; v.v[4 + t] = b[t]; }
  return v;
}

// Fragment c of column R e + (lane % R) of an LDS tile: rows 8 NG c + idx(t), t = 0..7.
// ds_read_b64_tr_b16 works on groups of 16 lanes: lane i reads 4 elements at its own
// address and lane j gets element j % 4 of lanes j / 4, j / 4 + 4, + 8, + 12, so with
// lane i at row i / 4 and columns 4 (i % 4) .. + 3, lane j holds 4 rows of column j.
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
template <int DH, int R>
__device__ __forceinline__ bf16x8 tfrag(const bf16_t* lds, int e, int lane, int c) {
  constexpr int NG = 64 / R;
  const int g = lane / R, i = lane & 15, sub = (lane % R) >> 4;
  const int row = 8 * NG * c + 4 * g + (i >> 2);
  const int ch = (e * R + 16 * sub) / 8 + ((i >> 1) & 1);
  const bf16_t* p = lds + Tile<bf16_t, DH>::at(row, ch) + (i & 1) * 4;
  const bf16_t* q = lds + Tile<bf16_t, DH>::at(row + 4 * NG, ch) + (i & 1) * 4;
  union {
    v4s h[2];
    bf16x8 v;
  } x;
  x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)p);
  x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)q);
  return x.v;
}
template <int DH, int R>
__device__ __forceinline__ f32x8 tfrag(const float* lds, int e, int lane, int c) {
  constexpr int NG = 64 / R;
  typedef Tile<float, DH> L;
  const int g = lane / R, col = e * R + lane % R;
  f32x8 v;
#pragma unroll
  for (int t = 0; t < 8; ++t)
    v.v[t] = lds[L::at(8 * NG * c + 4 * NG * (t / 4) + 4 * g + t % 4, col / 4) + (col & 3)];
  return v;
}

// Fragment c from the lane's own values (flat index 8 c .. 8 c + 7).  bf16 rounds P and
// the score cotangents to nearest even: the products take bf16 operands, and the sums
// of the softmax are taken from the float32 values before that.
template <typename V>
__device__ __forceinline__ void pack(const V* s, int c, bf16x8& f) {
  constexpr int AV = sizeof(V) / 4;
#pragma unroll
  for (int t = 0; t < 8; ++t) f[t] = (__bf16)s[(8 * c + t) / AV][(8 * c + t) % AV];
}
template <typename V>
__device__ __forceinline__ void pack(const V* s, int c, f32x8& f) {
  constexpr int AV = sizeof(V) / 4;
#pragma unroll
  for (int t = 0; t < 8; ++t) f.v[t] = s[(8 * c + t) / AV][(8 * c + t) % AV];
}

template <int R>
__device__ __forceinline__ float sum_groups(float v) {
  if (R == 16) v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
template <int R>
__device__ __forceinline__ float max_groups(float v) {
  if (R == 16) v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}

template <typename V>
__device__ __forceinline__ void zero(V& v) {
#pragma unroll
  for (int i = 0; i < (int)(sizeof(V) / 4); ++i) v[i] = 0.f;
}

// A row's dims from the lane's accumulators (dim idx(t)), scaled, columns past dh left out.
template <int R, int NE, typename T, typename V>
__device__ __forceinline__ void store_row(T* row, const V (&acc)[NE], float f, int g, int dh) {
  constexpr int NG = 64 / R, AV = sizeof(V) / 4;
#pragma unroll
  for (int t = 0; t < NE * AV; t += 4) {
    const int d = 4 * NG * (t / 4) + 4 * g;
    const V& v = acc[t / AV];
    if (d < dh)
      store4(row + d, v[t % AV] * f, v[t % AV + 1] * f, v[t % AV + 2] * f, v[t % AV + 3] * f);
  }
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Tile and head of this workgroup: heads vary slowest, and when the grid divides
// evenly each XCD (workgroups go to the 8 of them round-robin) is given a contiguous
// run, so the tiles that share keys meet in one L2.
__device__ __forceinline__ void tile_of(int& tile, int& head) {
  const int L = blockIdx.x + gridDim.x * blockIdx.y;
  const int N = gridDim.x * gridDim.y;
  const int i = (N & 7) == 0 ? (L & 7) * (N >> 3) + (L >> 3) : L;
  head = i / gridDim.x;
  tile = i - head * gridDim.x;
}

// ---------------------------------------------------------------- forward
template <typename T, int DH, int R, bool DUAL>
__global__ void __launch_bounds__(64 * PK_TILE / R) packed_fwd_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * PK_TILE / R, NG = 64 / R, NS = KB / R, NE = DH / R, NC = DH / (8 * NG);
  constexpr int AV = R * R / 64, NK = KB / (8 * NG);
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sK[L::ELEMS], sV[L::ELEMS], sKd[DUAL ? L::ELEMS : 8],
      sVd[DUAL ? L::ELEMS : 8];
  int ti, h;
  tile_of(ti, h);
  const int nt = a.p.head[0];
  if (ti >= nt) return;
  const int4 tile = a.p.tile[nt - 1 - ti];
  const int lo = tile.y, hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane % R, g = lane / R;
  const int q0 = tile.x + w * R, q = q0 + lr, qc = min(q, hi - 1);
  const int kh = h / (a.H / a.K), dh = a.dh;
  const T* K = a.k + (long)kh * dh;
  const T* Vp = a.v + (long)kh * dh;
  const T* Kd = DUAL ? a.kd + (long)kh * dh : nullptr;
  const T* Vd = DUAL ? a.vd + (long)kh * dh : nullptr;
  F qf[NC], qdf[DUAL ? NC : 1];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    qf[c] = gfrag<NG>(a.q + qc * a.ldq + (long)h * dh, g, c, dh);
    if constexpr (DUAL) qdf[c] = gfrag<NG>(a.qd + qc * a.ldqd + (long)h * dh, g, c, dh);
  }
  const float s2 = a.scale * 1.44269504088896341f;
  float m = -INFINITY, l = 0.f, cs = 0.f;
  V o[NE], od[DUAL ? NE : 1];
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    zero(o[e]);
    if constexpr (DUAL) zero(od[e]);
  }
  const int qlast = min(tile.x + PK_TILE, hi) - 1;
  for (int k0 = lo; k0 <= qlast; k0 += KB) {
    __syncthreads();
    stage<T, DH, NT>(sK, K, a.ldk, k0, hi - 1, dh, tid);
    stage<T, DH, NT>(sV, Vp, a.ldv, k0, hi - 1, dh, tid);
    if constexpr (DUAL) {
      stage<T, DH, NT>(sKd, Kd, a.ldkd, k0, hi - 1, dh, tid);
      stage<T, DH, NT>(sVd, Vd, a.ldvd, k0, hi - 1, dh, tid);
    }
    __syncthreads();
    if (k0 > q0 + R - 1 || q0 >= hi) continue;   // nothing of the block is visible to the wave
    V s[NS], sd[DUAL ? NS : 1];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      zero(s[n]);
      if constexpr (DUAL) zero(sd[n]);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const F kf = frag<DH, NG>(sK, n * R + lr, g, c);
        s[n] = mma(kf, qf[c], s[n]);
        if constexpr (DUAL) {
          sd[n] = mma(kf, qdf[c], sd[n]);
          sd[n] = mma(frag<DH, NG>(sKd, n * R + lr, g, c), qf[c], sd[n]);
        }
      }
    }
    const bool diag = k0 + KB - 1 > q0;
    float mx = -INFINITY;
#pragma unroll
    for (int t = 0; t < NS * AV; ++t) {
      float v = s[t / AV][t % AV] * s2;
      if (diag && k0 + 4 * NG * (t / 4) + 4 * g + t % 4 > q) v = -INFINITY;
      s[t / AV][t % AV] = v;
      mx = fmaxf(mx, v);
    }
    // block lo holds a visible key of every query, so m is finite from the first block on
    const float mn = fmaxf(m, max_groups<R>(mx));
    const float al = exp2_(m - mn);
    m = mn;
    float ls = 0.f, lc = 0.f;
#pragma unroll
    for (int t = 0; t < NS * AV; ++t) {
      const float sv = s[t / AV][t % AV];
      const float p = exp2_(sv - mn);
      s[t / AV][t % AV] = p;
      ls += p;
      if constexpr (DUAL) {
        const float pd = sv == -INFINITY ? 0.f : p * (sd[t / AV][t % AV] * a.scale);
        sd[t / AV][t % AV] = pd;
        lc += pd;
      }
    }
    l = l * al + ls;
    if constexpr (DUAL) cs = cs * al + lc;
#pragma unroll
    for (int e = 0; e < NE; ++e) {
      o[e] *= al;
      if constexpr (DUAL) od[e] *= al;
    }
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      F pf, pdf;
      pack(s, c, pf);
      if constexpr (DUAL) pack(sd, c, pdf);
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const F vf = tfrag<DH, R>(sV, e, lane, c);
        o[e] = mma(vf, pf, o[e]);
        if constexpr (DUAL) {
          od[e] = mma(vf, pdf, od[e]);
          od[e] = mma(tfrag<DH, R>(sVd, e, lane, c), pf, od[e]);
        }
      }
    }
  }
  if (q >= hi) return;   // (lanes of one row leave together; q0 < hi has l > 0)
  const float lt = sum_groups<R>(l), inv = 1.0f / lt;
  const float c = DUAL ? sum_groups<R>(cs) * inv : 0.f;
  if (g == 0) {
    a.lse[(long)h * a.p.n + q] = m + __log2f(lt);
    if constexpr (DUAL) a.cst[(long)h * a.p.n + q] = c;
  }
  if constexpr (DUAL) {
#pragma unroll
    for (int e = 0; e < NE; ++e) od[e] = od[e] - c * o[e];
    store_row<R, NE>(a.od + q * a.ldod + (long)h * dh, od, inv, g, dh);
  }
  store_row<R, NE>(a.o + q * a.ldo + (long)h * dh, o, inv, g, dh);
}

// ---------------------------------------------------------------- backward: dQ
__device__ __forceinline__ float dot(const bf16x8& a, const bf16x8& b) {
  float s = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) s += (float)a[t] * (float)b[t];
  return s;
}
__device__ __forceinline__ float dot(const f32x8& a, const f32x8& b) {
  float s = 0.f;
#pragma unroll
  for (int t = 0; t < 8; ++t) s += a.v[t] * b.v[t];
  return s;
}

template <typename T, int DH, int R, bool DUAL>
__global__ void __launch_bounds__(64 * PK_TILE / R) packed_dq_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * PK_TILE / R, NG = 64 / R, NS = KB / R, NE = DH / R, NC = DH / (8 * NG);
  constexpr int AV = R * R / 64, NK = KB / (8 * NG);
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sK[L::ELEMS], sV[L::ELEMS], sKd[DUAL ? L::ELEMS : 8],
      sVd[DUAL ? L::ELEMS : 8];
  int ti, h;
  tile_of(ti, h);
  const int nt = a.p.head[0];
  if (ti >= nt) return;
  const int4 tile = a.p.tile[nt - 1 - ti];
  const int lo = tile.y, hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane % R, g = lane / R;
  const int q0 = tile.x + w * R, q = q0 + lr, qc = min(q, hi - 1);
  const int kh = h / (a.H / a.K), dh = a.dh;
  const T* K = a.k + (long)kh * dh;
  const T* Vp = a.v + (long)kh * dh;
  const T* Kd = DUAL ? a.kd + (long)kh * dh : nullptr;
  const T* Vd = DUAL ? a.vd + (long)kh * dh : nullptr;
  F qf[NC], gf[NC], qdf[DUAL ? NC : 1], gdf[DUAL ? NC : 1];
  float r = 0.f, rd = 0.f;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    qf[c] = gfrag<NG>(a.q + qc * a.ldq + (long)h * dh, g, c, dh);
    gf[c] = gfrag<NG>(a.g + qc * a.ldg + (long)h * dh, g, c, dh);
    const F of = gfrag<NG>((const T*)a.o + qc * a.ldo + (long)h * dh, g, c, dh);
    r += dot(gf[c], of);
    if constexpr (DUAL) {
      qdf[c] = gfrag<NG>(a.qd + qc * a.ldqd + (long)h * dh, g, c, dh);
      gdf[c] = gfrag<NG>(a.gd + qc * a.ldgd + (long)h * dh, g, c, dh);
      rd += dot(gdf[c], of) +
            dot(gf[c], gfrag<NG>((const T*)a.od + qc * a.ldod + (long)h * dh, g, c, dh));
    }
  }
  r = sum_groups<R>(r);
  if constexpr (DUAL) rd = sum_groups<R>(rd);
  const long row = (long)h * a.p.n + qc;
  if (g == 0 && q < hi) {
    a.r[row] = r;
    if constexpr (DUAL) a.rd[row] = rd;
  }
  const float lse = a.lse[row], cst = DUAL ? a.cst[row] : 0.f;
  const float s2 = a.scale * 1.44269504088896341f;
  V dq[NE], dqd[DUAL ? NE : 1];
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    zero(dq[e]);
    if constexpr (DUAL) zero(dqd[e]);
  }
  const int qlast = min(tile.x + PK_TILE, hi) - 1;
  for (int k0 = lo; k0 <= qlast; k0 += KB) {
    __syncthreads();
    stage<T, DH, NT>(sK, K, a.ldk, k0, hi - 1, dh, tid);
    stage<T, DH, NT>(sV, Vp, a.ldv, k0, hi - 1, dh, tid);
    if constexpr (DUAL) {
      stage<T, DH, NT>(sKd, Kd, a.ldkd, k0, hi - 1, dh, tid);
      stage<T, DH, NT>(sVd, Vd, a.ldvd, k0, hi - 1, dh, tid);
    }
    __syncthreads();
    if (k0 > q0 + R - 1 || q0 >= hi) continue;
    const bool diag = k0 + KB - 1 > q0;
    V ds[NS], dsd[DUAL ? NS : 1];
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      V s, sd, dp, dpd;
      zero(s); zero(sd); zero(dp); zero(dpd);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const F kf = frag<DH, NG>(sK, n * R + lr, g, c), vf = frag<DH, NG>(sV, n * R + lr, g, c);
        s = mma(kf, qf[c], s);
        dp = mma(vf, gf[c], dp);
        if constexpr (DUAL) {
          sd = mma(kf, qdf[c], sd);
          sd = mma(frag<DH, NG>(sKd, n * R + lr, g, c), qf[c], sd);
          dpd = mma(vf, gdf[c], dpd);
          dpd = mma(frag<DH, NG>(sVd, n * R + lr, g, c), gf[c], dpd);
        }
      }
#pragma unroll
      for (int t = 0; t < AV; ++t) {
        const bool ok = !diag || k0 + n * R + 4 * NG * (t / 4) + 4 * g + t % 4 <= q;
        const float p = exp2_(s[t] * s2 - lse);
        const float x = dp[t] - r;
        ds[n][t] = ok ? a.scale * p * x : 0.f;
        if constexpr (DUAL) {
          const float pd = p * (sd[t] * a.scale - cst);
          dsd[n][t] = ok ? a.scale * (pd * x + p * (dpd[t] - rd)) : 0.f;
        }
      }
    }
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      F df, ddf;
      pack(ds, c, df);
      if constexpr (DUAL) pack(dsd, c, ddf);
#pragma unroll
      for (int e = 0; e < NE; ++e) {
        const F kt = tfrag<DH, R>(sK, e, lane, c);
        dq[e] = mma(kt, df, dq[e]);
        if constexpr (DUAL) {
          dqd[e] = mma(kt, ddf, dqd[e]);
          dqd[e] = mma(tfrag<DH, R>(sKd, e, lane, c), df, dqd[e]);
        }
      }
    }
  }
  if (q >= hi) return;
  store_row<R, NE>(a.dq + q * a.lddq + (long)h * dh, dq, 1.f, g, dh);
  if constexpr (DUAL) store_row<R, NE>(a.dqd + q * a.lddqd + (long)h * dh, dqd, 1.f, g, dh);
}

// ---------------------------------------------------------------- backward: dK, dV
template <typename T, int DH, int R, bool DUAL>
__global__ void __launch_bounds__(64 * PK_TILE / R) packed_dkv_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * PK_TILE / R, NG = 64 / R, NS = KB / R, NE = DH / R, NC = DH / (8 * NG);
  constexpr int AV = R * R / 64, NK = KB / (8 * NG);
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sQ[L::ELEMS], sG[L::ELEMS], sQd[DUAL ? L::ELEMS : 8],
      sGd[DUAL ? L::ELEMS : 8];
  __shared__ __attribute__((aligned(16))) float sL[KB], sR[KB], sC[KB], sRd[KB];
  int ti, kh;
  tile_of(ti, kh);
  if (ti >= a.p.head[0]) return;
  const int4 tile = a.p.tile[ti];
  const int hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lr = lane % R, g = lane / R;
  const int k0 = tile.x + w * R, k = k0 + lr, kc = min(k, hi - 1);
  const int G = a.H / a.K, dh = a.dh;
  F kf[NC], vf[NC], kdf[DUAL ? NC : 1], vdf[DUAL ? NC : 1];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    kf[c] = gfrag<NG>(a.k + kc * a.ldk + (long)kh * dh, g, c, dh);
    vf[c] = gfrag<NG>(a.v + kc * a.ldv + (long)kh * dh, g, c, dh);
    if constexpr (DUAL) {
      kdf[c] = gfrag<NG>(a.kd + kc * a.ldkd + (long)kh * dh, g, c, dh);
      vdf[c] = gfrag<NG>(a.vd + kc * a.ldvd + (long)kh * dh, g, c, dh);
    }
  }
  const float s2 = a.scale * 1.44269504088896341f;
  V dk[NE], dv[NE], dkd[DUAL ? NE : 1], dvd[DUAL ? NE : 1];
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    zero(dk[e]);
    zero(dv[e]);
    if constexpr (DUAL) {
      zero(dkd[e]);
      zero(dvd[e]);
    }
  }
  for (int h = kh * G; h < (kh + 1) * G; ++h) {
    const T* Q = a.q + (long)h * dh;
    const T* Gp = a.g + (long)h * dh;
    const T* Qd = DUAL ? a.qd + (long)h * dh : nullptr;
    const T* Gd = DUAL ? a.gd + (long)h * dh : nullptr;
    for (int q0 = tile.x; q0 < hi; q0 += KB) {
      __syncthreads();
      stage<T, DH, NT>(sQ, Q, a.ldq, q0, hi - 1, dh, tid);
      stage<T, DH, NT>(sG, Gp, a.ldg, q0, hi - 1, dh, tid);
      if constexpr (DUAL) {
        stage<T, DH, NT>(sQd, Qd, a.ldqd, q0, hi - 1, dh, tid);
        stage<T, DH, NT>(sGd, Gd, a.ldgd, q0, hi - 1, dh, tid);
      }
      if (tid < KB) {
        const long i = (long)h * a.p.n + min(q0 + tid, hi - 1);
        sL[tid] = a.lse[i];
        sR[tid] = a.r[i];
        if constexpr (DUAL) {
          sC[tid] = a.cst[i];
          sRd[tid] = a.rd[i];
        }
      }
      __syncthreads();
      if (q0 + KB - 1 < k0 || k0 >= hi) continue;   // every query of the block precedes the wave's keys
      const bool mask = q0 < k0 + R - 1 || q0 + KB > hi;
      V p[NS], ds[NS], pd[DUAL ? NS : 1], dsd[DUAL ? NS : 1];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        V s, sd, dp, dpd;
        zero(s); zero(sd); zero(dp); zero(dpd);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const F qq = frag<DH, NG>(sQ, n * R + lr, g, c), gg = frag<DH, NG>(sG, n * R + lr, g, c);
          s = mma(qq, kf[c], s);
          dp = mma(gg, vf[c], dp);
          if constexpr (DUAL) {
            sd = mma(qq, kdf[c], sd);
            sd = mma(frag<DH, NG>(sQd, n * R + lr, g, c), kf[c], sd);
            dpd = mma(gg, vdf[c], dpd);
            dpd = mma(frag<DH, NG>(sGd, n * R + lr, g, c), vf[c], dpd);
          }
        }
#pragma unroll
        for (int t = 0; t < AV; ++t) {
          const int i = n * R + 4 * NG * (t / 4) + 4 * g + t % 4;
          const bool ok = !mask || (q0 + i >= k && q0 + i < hi);
          const float pv = ok ? exp2_(s[t] * s2 - sL[i]) : 0.f;
          const float x = dp[t] - sR[i];
          p[n][t] = pv;
          ds[n][t] = ok ? a.scale * pv * x : 0.f;
          if constexpr (DUAL) {
            const float pdv = ok ? pv * (sd[t] * a.scale - sC[i]) : 0.f;
            pd[n][t] = pdv;
            dsd[n][t] = ok ? a.scale * (pdv * x + pv * (dpd[t] - sRd[i])) : 0.f;
          }
        }
      }
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        F pf, df, pdf, ddf;
        pack(p, c, pf);
        pack(ds, c, df);
        if constexpr (DUAL) {
          pack(pd, c, pdf);
          pack(dsd, c, ddf);
        }
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const F gt = tfrag<DH, R>(sG, e, lane, c), qt = tfrag<DH, R>(sQ, e, lane, c);
          dv[e] = mma(gt, pf, dv[e]);
          dk[e] = mma(qt, df, dk[e]);
          if constexpr (DUAL) {
            dvd[e] = mma(gt, pdf, dvd[e]);
            dvd[e] = mma(tfrag<DH, R>(sGd, e, lane, c), pf, dvd[e]);
            dkd[e] = mma(qt, ddf, dkd[e]);
            dkd[e] = mma(tfrag<DH, R>(sQd, e, lane, c), df, dkd[e]);
          }
        }
      }
    }
  }
  if (k >= hi) return;
  store_row<R, NE>(a.dk + k * a.lddk + (long)kh * dh, dk, 1.f, g, dh);
  store_row<R, NE>(a.dv + k * a.lddv + (long)kh * dh, dv, 1.f, g, dh);
  if constexpr (DUAL) {
    store_row<R, NE>(a.dkd + k * a.lddkd + (long)kh * dh, dkd, 1.f, g, dh);
    store_row<R, NE>(a.dvd + k * a.lddvd + (long)kh * dh, dvd, 1.f, g, dh);
  }
}

// ---------------------------------------------------------------- plan
// Bounds made ascending (running maximum of the clamped offsets) and the tiles before
// each sequence, by one workgroup over chunks of its size.
constexpr int SCAN = 1024;
__global__ void __launch_bounds__(SCAN) plan_scan_kernel(SeqPlanArgs a) {
  __shared__ int sv[SCAN], carry[2];
  const int tid = threadIdx.x, m = a.p.m, n = (int)a.p.n;
  auto raw = [&](int j) {
    if (!a.cu) return (int)min((long)j * a.len, (long)n);
    if (!a.cover) return min(max(a.cu[j], 0), n);
    return j == 0 ? 0 : j == m ? n : min(max(a.cu[j - 1], 0), n);
  };
  if (tid == 0) carry[0] = carry[1] = 0;
  __syncthreads();
  for (int j0 = 0; j0 <= m; j0 += SCAN) {
    const int j = j0 + tid;
    sv[tid] = j <= m ? raw(j) : 0;
    __syncthreads();
    for (int o = 1; o < SCAN; o <<= 1) {
      const int x = tid >= o ? sv[tid - o] : 0;
      __syncthreads();
      sv[tid] = max(sv[tid], x);
      __syncthreads();
    }
    if (j <= m) a.p.bound[j] = max(sv[tid], carry[0]);
    __syncthreads();
    if (tid == 0) carry[0] = max(carry[0], sv[SCAN - 1]);
    __syncthreads();
  }
  for (int j0 = 0; j0 <= m; j0 += SCAN) {
    const int j = j0 + tid;
    const int t = j < m ? (a.p.bound[j + 1] - a.p.bound[j] + PK_TILE - 1) / PK_TILE : 0;
    sv[tid] = t;
    __syncthreads();
    for (int o = 1; o < SCAN; o <<= 1) {
      const int x = tid >= o ? sv[tid - o] : 0;
      __syncthreads();
      sv[tid] += x;
      __syncthreads();
    }
    if (j <= m) a.p.tstart[j] = carry[1] + sv[tid] - t;
    __syncthreads();
    if (tid == 0) carry[1] += sv[SCAN - 1];
    __syncthreads();
  }
  if (tid == 0) {
    a.p.head[0] = carry[1];
    a.p.head[1] = a.p.bound[0];
    a.p.head[2] = a.p.bound[m];
    a.p.head[3] = 0;
  }
}

// Index j of the last entry of x[0 .. m] that is <= v (x[0] <= v).
__device__ __forceinline__ int last_le(const int* x, int m, int v) {
  int lo = 0, hi = m + 1;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (x[mid] <= v) lo = mid; else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(256) plan_fill_kernel(SeqPlanArgs a) {
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const int m = a.p.m;
  if (i < a.p.head[0]) {
    const int j = last_le(a.p.tstart, m, (int)i);
    a.p.tile[i] = make_int4(a.p.bound[j] + ((int)i - a.p.tstart[j]) * PK_TILE, a.p.bound[j],
                            a.p.bound[j + 1], 0);
  }
  if (i < a.p.n) {
    int pos = 0;
    if (a.positions)
      pos = a.positions[i];
    else if (i >= a.p.bound[0] && i < a.p.bound[m])
      pos = (int)i - a.p.bound[last_le(a.p.bound, m, (int)i)];
    a.p.pos[i] = pos;
  }
}

// Rows a wave owns: 32 where the accumulators of the pass leave a wave its registers.
template <typename T, int DH, bool DUAL>
constexpr int rows_of() { return sizeof(T) == 2 && !DUAL ? 32 : 16; }

template <typename T, int DH, bool DUAL>
void launch_fwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  constexpr int R = rows_of<T, DH, DUAL>();
  hipLaunchKernelGGL((packed_fwd_kernel<T, DH, R, DUAL>), dim3(a.p.max_tiles, a.H),
                     dim3(64 * PK_TILE / R), 0, s, a);
}
template <typename T, int DH, bool DUAL>
hipError_t launch_bwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  constexpr int R = rows_of<T, DH, DUAL>();
  hipLaunchKernelGGL((packed_dq_kernel<T, DH, R, DUAL>), dim3(a.p.max_tiles, a.H),
                     dim3(64 * PK_TILE / R), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((packed_dkv_kernel<T, DH, R, DUAL>), dim3(a.p.max_tiles, a.K),
                     dim3(64 * PK_TILE / R), 0, s, a);
  return hipGetLastError();
}

template <typename T>
bool shapes_ok(const PackedAttnArgs<T>& a) {
  return a.dh >= 8 && a.dh <= PK_MAX_DH && a.dh % 8 == 0 && a.K >= 1 && a.H >= a.K &&
         a.H % a.K == 0 && a.H <= PK_MAX_HEADS && a.p.n >= 0 && a.p.n <= PK_MAX_TOKENS;
}

}  // namespace

SeqPlan seq_plan_at(char* base, long n, int m, size_t* bytes) {
  SeqPlan p;
  size_t off = 0;
  auto take = [&](size_t b) {
    char* r = base ? base + off : nullptr;
    off += (b + 255) / 256 * 256;
    return r;
  };
  p.n = n;
  p.m = m;
  p.max_tiles = (int)(n / PK_TILE + std::min((long)m, n));
  p.head = (int*)take(16);
  p.bound = (int*)take(4 * ((size_t)m + 1));
  p.tstart = (int*)take(4 * ((size_t)m + 1));
  p.tile = (int4*)take(16 * (size_t)p.max_tiles);
  p.pos = (int*)take(4 * (size_t)n);
  if (bytes) *bytes = off;
  return p;
}

hipError_t seq_plan_make(const SeqPlanArgs& a, hipStream_t s) {
  if (a.p.n < 1) return hipSuccess;
  hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(SCAN), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long items = std::max((long)a.p.max_tiles, a.p.n);
  hipLaunchKernelGGL(plan_fill_kernel, dim3((unsigned)((items + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t packed_attn_fwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  if (!shapes_ok(a)) return hipErrorInvalidValue;
  if (a.p.max_tiles < 1) return hipSuccess;
  if (a.dh <= 64) {
    if (a.dual) launch_fwd<T, 64, true>(a, s); else launch_fwd<T, 64, false>(a, s);
  } else {
    if (a.dual) launch_fwd<T, 128, true>(a, s); else launch_fwd<T, 128, false>(a, s);
  }
  return hipGetLastError();
}

template <typename T>
hipError_t packed_attn_bwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  if (!shapes_ok(a)) return hipErrorInvalidValue;
  if (a.p.max_tiles < 1) return hipSuccess;
  if (a.dh <= 64) return a.dual ? launch_bwd<T, 64, true>(a, s) : launch_bwd<T, 64, false>(a, s);
  return a.dual ? launch_bwd<T, 128, true>(a, s) : launch_bwd<T, 128, false>(a, s);
}

template hipError_t packed_attn_fwd<bf16_t>(const PackedAttnArgs<bf16_t>&, hipStream_t);
template hipError_t packed_attn_fwd<float>(const PackedAttnArgs<float>&, hipStream_t);
template hipError_t packed_attn_bwd<bf16_t>(const PackedAttnArgs<bf16_t>&, hipStream_t);
template hipError_t packed_attn_bwd<float>(const PackedAttnArgs<float>&, hipStream_t);

}  // namespace mfmg
