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
// C[a][b] = sum_k A[a][k] B[b][k] with b the lane's row: an operand fragment is the FE
// elements k = FE g + 0 .. FE - 1 of FE NG (FE = 8 for bf16, 4 for float32), and of R x R
// results the lane holds a = idx(t) = 4 NG (t / 4) + 4 g + t % 4 of its row.  So the
// scores of a block leave a lane with the values at block rows idx(t), FE of which are a
// fragment of the next product, over rows in that order; its other operand is read from
// the tile in the same order (tfrag), and probabilities never leave registers.
//
// What bounds it.  The matrix instructions: 2 and 6 products a visible pair in the primal
// and dual forward, 3 and 9 in the dQ pass, 4 and 12 in the dK/dV pass, where S and dP
// are formed again so that no sum needs atomics (a single pass would take 5 and 15 for
// the backward, not 7 and 21).  They are fed from LDS, one fragment read a product and R
// rows, by two or three waves a SIMD, whose exponentials run beside another's products.
// Counters at 16384 tokens of 16 heads of 128: matrix units busy 64% of the cycles at the
// 1.7 GHz the card then holds, vector units 50%, no bank conflicts.
#include "packed.h"

#include <algorithm>
#include <cfloat>
#include <type_traits>

namespace mfmg {

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));

template <int R> struct AccT;
template <> struct AccT<16> { typedef f32x4 V; };
template <> struct AccT<32> { typedef f32x16 V; };

// Operand fragments: FE elements of a row.
template <typename T> struct FragT;
template <> struct FragT<bf16_t> { typedef bf16x8 V; static constexpr int FE = 8; };
template <> struct FragT<float> { typedef f32x4 V; static constexpr int FE = 4; };

__device__ __forceinline__ f32x4 mma(const bf16x8& a, const bf16x8& b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(const bf16x8& a, const bf16x8& b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// float32: element t of every lane group's four is one instruction's contraction
__device__ __forceinline__ f32x4 mma(const f32x4& a, const f32x4& b, f32x4 c) {
#pragma unroll
  for (int t = 0; t < 4; ++t) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[t], b[t], c, 0, 0, 0);
  return c;
}

// LDS tile of rows of DH elements in 16-byte chunks, the chunk index XOR-swizzled by the
// row.  A fragment read's 16-byte lanes are served in sets of 0-3, 12-15, 20-23, 24-27 (and
// so on): both with 16 rows at two neighbouring chunks and with 32 rows at one, their
// 16 addresses cover all 64 banks; so do the 32 lanes of a transposing read (8 rows of
// two chunks, or 4 rows of four), and for float32 the four rows of a column read.
// (SQ_LDS_BANK_CONFLICT 0; with row bits 2 and 3 unmixed 42% of the LDS cycles of
// 64-dim tiles were conflicts.)
template <typename T, int DH>
struct Tile {
  static constexpr int P = DH <= 64 ? 64 : 128;          // row pitch
  static constexpr int VE = Elem<T>::VE, NC = P / VE;    // chunks of a row
  __device__ static __forceinline__ int chunk(int row, int place) {   // and the place of a chunk
    const int x = (row >> 2) & 3, h = ((x ^ (x >> 1)) & 1) << 1 | x >> 1;   // 0, 2, 3, 1
    const int f = sizeof(T) == 4 ? row & 15 : NC >= 16 ? (row & 3) << 2 | h : ((row >> 1) & 1) << 2 | h;
    return place ^ f;
  }
  __device__ static __forceinline__ int at(int row, int c) { return row * P + chunk(row, c) * VE; }
};

// A block of KB rows on its way to an LDS tile: the NT threads of a workgroup load 16 bytes
// each, straight to LDS, where a wave's 64 chunks land behind one another: a thread's chunk
// is the one that the swizzle puts at its place.  No registers hold the data, and the next
// block travels during the current one's products.  The compiler lets LDS reads pass such
// loads only where it knows them to be of different variables, so a tile's two buffers
// are two variables.  A thread's chunks are STEP rows apart (leading dimensions are below
// 2^22: 32-bit offsets in a block, below 2^30).  Rows past `last` and columns past dh are out of
// the descriptor's range and land as zeros.
typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ void load_lds16(__amdgpu_buffer_rsrc_t rsrc, void* lds, unsigned off) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)lds, 16, off, 0, 0, 0);
}
template <typename T, int DH, int KB, int NT>
struct Block {
  typedef Tile<T, DH> L;
  static constexpr int N = KB * L::NC / NT, STEP = NT / L::NC, NO = STEP % 16 ? 2 : 1;
  static_assert(KB * L::NC % NT == 0 && NT % L::NC == 0 && STEP % 8 == 0, "chunks of a thread");
  unsigned off[NO];   // byte offset of the thread's chunk in the block's first (NO) STEP rows
  unsigned ldb;
  __device__ __forceinline__ void init(long ld, int dh, int tid) {
    ldb = (unsigned)ld * sizeof(T);
#pragma unroll
    for (int k = 0; k < NO; ++k) {   // (the swizzle repeats every 16 rows)
      const int r = tid / L::NC + k * STEP, c = L::chunk(r, tid % L::NC);
      off[k] = c < dh / L::VE ? r * ldb + c * 16 : 1u << 31;
    }
  }
  // rows row0 .. of g to the tile at lds, by wave w
  __device__ __forceinline__ void load(const T* __restrict__ g, int row0, int last, T* lds, int w) const {
    const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(
        const_cast<char*>(reinterpret_cast<const char*>(g) + (long)row0 * ldb), 0,
        (int)(min(last - row0 + 1, KB) * ldb), 0x00020000);
#pragma unroll
    for (int k = 0; k < N; ++k)
      load_lds16(rsrc, lds + (k * NT + w * 64) * L::VE, off[k % NO] + k / NO * NO * STEP * ldb);
  }
};
// Every wave's loads have landed, and nobody reads the other buffers any more.
__device__ __forceinline__ void landed() {
  __builtin_amdgcn_s_waitcnt(7 << 4);   // vmcnt(0) lgkmcnt(0)
  __syncthreads();
}

// Fragment c of a row in global memory: elements FE (NG c + g) .. + FE - 1, zero past dh.
template <int NG>
__device__ __forceinline__ bf16x8 gfrag(const bf16_t* p, int g, int c, int dh) {
  const int d = 8 * (NG * c + g);
  if (d < dh) return *reinterpret_cast<const bf16x8*>(p + d);
  bf16x8 z;
#pragma unroll
  for (int t = 0; t < 8; ++t) z[t] = (__bf16)0.f;
  return z;
}
template <int NG>
__device__ __forceinline__ f32x4 gfrag(const float* p, int g, int c, int dh) {
  const int d = 4 * (NG * c + g);
  return d < dh ? *reinterpret_cast<const f32x4*>(p + d) : f32x4{0.f, 0.f, 0.f, 0.f};
}

// Where a lane finds its parts of an LDS tile.  frag: fragment c of row row0 + lane % R
// (row0 a multiple of 16, which leaves the swizzle alone).  tfrag: fragment c of column
// R e + lane % R, rows idx(FE c + t), t < FE.  The chunk indices are XORed with the
// swizzle, so the address of another c or e is one XOR away from the first: `pin` hides
// the bases from the compiler, which would otherwise keep every address in a register
// of its own through the whole loop.
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;
template <typename T, int DH, int R>
struct Lane;
template <int DH, int R>
struct Lane<bf16_t, DH, R> {
  typedef Tile<bf16_t, DH> L;
  static constexpr int NG = 64 / R;
  int f, t0, t1;
  // ds_read_b64_tr_b16 works on groups of 16 lanes: lane i reads 4 elements at its own
  // address and lane j gets element j % 4 of lanes j / 4, j / 4 + 4, + 8, + 12, so with
  // lane i at row i / 4 and columns 4 (i % 4) .. + 3, lane j holds 4 rows of column j.
  __device__ __forceinline__ Lane(int lane) {
    const int g = lane / R, i = lane & 15, sub = (lane % R) >> 4;
    const int row = 4 * g + (i >> 2), ch = 2 * sub + ((i >> 1) & 1);
    f = L::at(lane % R, g);
    t0 = L::at(row, ch) + (i & 1) * 4;
    t1 = L::at(row + 4 * NG, ch) + (i & 1) * 4;
  }
  __device__ __forceinline__ void pin() { asm volatile("" : "+v"(f), "+v"(t0), "+v"(t1)); }
  __device__ __forceinline__ bf16x8 frag(const bf16_t* lds, int row0, int c) const {
    return *reinterpret_cast<const bf16x8*>(lds + (f ^ (8 * NG * c)) + row0 * L::P);
  }
  __device__ __forceinline__ bf16x8 tfrag(const bf16_t* lds, int e, int c) const {
    union {
      v4s h[2];
      bf16x8 v;
    } x;
    x.h[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(lds + (t0 ^ (R * e)) + 8 * NG * c * L::P));
    x.h[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(lds + (t1 ^ (R * e)) + 8 * NG * c * L::P));
    return x.v;
  }
};
template <int DH, int R>
struct Lane<float, DH, R> {
  typedef Tile<float, DH> L;
  static constexpr int NG = 64 / R;
  int f, t0, t1, t2, t3;   // (a lane's four rows of a column are swizzled differently)
  __device__ __forceinline__ Lane(int lane) {
    const int g = lane / R, r = lane % R;
    f = L::at(r, g);
    t0 = L::at(4 * g, r / 4) + (r & 3);
    t1 = L::at(4 * g + 1, r / 4) + (r & 3);
    t2 = L::at(4 * g + 2, r / 4) + (r & 3);
    t3 = L::at(4 * g + 3, r / 4) + (r & 3);
  }
  __device__ __forceinline__ void pin() {
    asm volatile("" : "+v"(f), "+v"(t0), "+v"(t1), "+v"(t2), "+v"(t3));
  }
  __device__ __forceinline__ f32x4 frag(const float* lds, int row0, int c) const {
    return *reinterpret_cast<const f32x4*>(lds + (f ^ (4 * NG * c)) + row0 * L::P);
  }
  __device__ __forceinline__ f32x4 tfrag(const float* lds, int e, int c) const {
    const float* p = lds + 4 * NG * c * L::P;
    return f32x4{p[t0 ^ (R * e)], p[t1 ^ (R * e)], p[t2 ^ (R * e)], p[t3 ^ (R * e)]};
  }
};

// Fragment c from the lane's own values (flat index FE c .. + FE - 1).  bf16 rounds P and
// the score cotangents to nearest even: the products take bf16 operands, and the softmax
// sums are taken from the float32 values before that.
template <typename V>
__device__ __forceinline__ void pack(const V* s, int c, bf16x8& f) {
  constexpr int AV = sizeof(V) / 4;
#pragma unroll
  for (int t = 0; t < 8; ++t) f[t] = (__bf16)s[(8 * c + t) / AV][(8 * c + t) % AV];
}
template <typename V>
__device__ __forceinline__ void pack(const V* s, int c, f32x4& f) {
  constexpr int AV = sizeof(V) / 4;
#pragma unroll
  for (int t = 0; t < 4; ++t) f[t] = s[(4 * c + t) / AV][(4 * c + t) % AV];
}

// Sum and maximum over the lane groups (the lanes of one row).
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

// KS waves that own the same rows and every KS-th sub-block of the other side join their
// sums in LDS, lane by lane and in order, in the first of them.  All waves call this
// together; `lds` is free for it.
template <int R, int NE, int KS>
struct Merge {
  static constexpr int AV = R * R / 64, LANE = NE * AV;   // floats of a lane
  float* p;
  int rank;   // 0 .. KS - 1
  __device__ __forceinline__ Merge(float* lds, int w, int lane)
      : p(lds + w / KS * LANE * 64 + lane), rank(w % KS) {}
  __device__ __forceinline__ float& scalar(int i) { return p[i * 64]; }
  // from wave j: v of the first wave becomes v f0 + v_j f1
  template <typename V>
  __device__ __forceinline__ void add(int j, V (&v)[NE], float f0, float f1) {
    __syncthreads();
    if (rank == j) {
#pragma unroll
      for (int t = 0; t < NE * AV; ++t) p[t * 64] = v[t / AV][t % AV];
    }
    __syncthreads();
    if (rank == 0) {
#pragma unroll
      for (int t = 0; t < NE * AV; ++t) v[t / AV][t % AV] = v[t / AV][t % AV] * f0 + p[t * 64] * f1;
    }
  }
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Rank (0 = most work) and head of this workgroup: ranks vary slowest, so the longest
// tiles of all heads start first, and where the heads divide by 8 each XCD (workgroups
// go to the 8 of them round-robin) has neighbouring heads, which share keys in its L2.
__device__ __forceinline__ void tile_of(int heads, int& rank, int& head) {
  const int L = blockIdx.x;
  rank = L / heads;
  const int i = L - rank * heads;
  head = (heads & 7) == 0 ? (i & 7) * (heads >> 3) + (i >> 3) : i;
}

// ---------------------------------------------------------------- forward
// 16384 tokens of 16 heads of 128 over 2 key heads, bf16: 1.00 ms, 1.10 PFLOP/s (a bf16
// product of 8192^3 reaches 1.21); dual, 2 x 4096 tokens of 8 heads of 64: 112 us, 0.92.
// A workgroup owns NW R / KS queries of one head.  Scores are formed for SB keys at a time
// and consumed before the next SB, which bounds the registers they need.  The running
// maximum is only raised, and the accumulators rescaled, when a score exceeds it by
// more than 2^8: until then exp2 stays below 2^8 times its usual range, far from
// float32's, and a factor common to numerator and denominator changes neither's
// relative error.
template <typename T, int DH, int R, int NW, int KS, int KB, int SB, int MW, bool PIN, bool DUAL>
__global__ void __launch_bounds__(64 * NW, MW) packed_fwd_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * NW, NG = 64 / R, NS = SB / R, NE = DH / R, FE = FragT<T>::FE, NC = DH / (FE * NG);
  constexpr int AV = R * R / 64, NK = SB / (FE * NG), ROWS = NW * R / KS;
  static_assert(SB % R == 0, "a wave that takes a sub-block sees its first row");
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sK0[KB * L::P], sK1[KB * L::P], sV0[KB * L::P], sV1[KB * L::P],
      sKd0[DUAL ? KB * L::P : 8], sKd1[DUAL ? KB * L::P : 8], sVd0[DUAL ? KB * L::P : 8], sVd1[DUAL ? KB * L::P : 8];
  int rank, h;
  tile_of(a.H, rank, h);
  const TileList tl = a.p.list[tile_kind(ROWS)];
  const int4 tile = tl.byq[rank];   // (its load does not wait for the count)
  if (rank >= a.p.head[tile_kind(ROWS)]) return;
  const int lo = tile.y, hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane % R, g = lane / R;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Lane<T, DH, R> at(lane);
  const int q0 = tile.x + w / KS * R, q = q0 + lr, qc = min(q, hi - 1);
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
  float m = -FLT_MAX, l = 0.f, cs = 0.f;   // (finite: scores of -inf are weights of 0 from the start)
  V o[NE], od[DUAL ? NE : 1];
#pragma unroll
  for (int e = 0; e < NE; ++e) {
    zero(o[e]);
    if constexpr (DUAL) zero(od[e]);
  }
  Block<T, DH, KB, NT> rK, rV, rKd, rVd;
  rK.init(a.ldk, dh, tid);
  rV.init(a.ldv, dh, tid);
  if constexpr (DUAL) {
    rKd.init(a.ldkd, dh, tid);
    rVd.init(a.ldvd, dh, tid);
  }
  auto load = [&](int k0, auto buffer) {
    constexpr bool b = decltype(buffer)::value;
    rK.load(K, k0, hi - 1, b ? sK1 : sK0, w);
    rV.load(Vp, k0, hi - 1, b ? sV1 : sV0, w);
    if constexpr (DUAL) {
      rKd.load(Kd, k0, hi - 1, b ? sKd1 : sKd0, w);
      rVd.load(Vd, k0, hi - 1, b ? sVd1 : sVd0, w);
    }
  };
  const int nb = (min(tile.x + ROWS, hi) - 1 - lo) / KB + 1;
  load(lo, std::false_type());
  auto block = [&](int kb, auto buffer) {
    constexpr bool b = decltype(buffer)::value;
    const T *sK = b ? sK1 : sK0, *sV = b ? sV1 : sV0, *sKd = b ? sKd1 : sKd0, *sVd = b ? sVd1 : sVd0;
    landed();   // block kb is in its buffer
    const int k0 = lo + kb * KB;
    if (kb + 1 < nb) load(k0 + KB, std::bool_constant<!b>());
#pragma unroll
    for (int sb = 0; sb < KB / SB; ++sb) {
      const int ks = k0 + sb * SB;
      if (KS > 1 && sb % KS != w % KS) continue;
      if (ks > q0 + R - 1 || q0 >= hi) break;   // nothing further is visible to the wave
      if constexpr (PIN) at.pin();
      V s[NS], sd[DUAL ? NS : 1];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        zero(s[n]);
        if constexpr (DUAL) zero(sd[n]);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const F kf = at.frag(sK, sb * SB + n * R, c);
          s[n] = mma(kf, qf[c], s[n]);
          if constexpr (DUAL) {
            sd[n] = mma(kf, qdf[c], sd[n]);
            sd[n] = mma(at.frag(sKd, sb * SB + n * R, c), qf[c], sd[n]);
          }
        }
      }
      if (ks + SB - 1 > q0) {   // some key may follow some query
#pragma unroll
        for (int t = 0; t < NS * AV; ++t)
          if (ks + 4 * NG * (t / 4) + 4 * g + t % 4 > q) {
            s[t / AV][t % AV] = -INFINITY;
            if constexpr (DUAL) sd[t / AV][t % AV] = 0.f;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < NS * AV; ++t) mx = fmaxf(mx, s[t / AV][t % AV]);
      if (__any(mx * s2 > m + 8.f)) {
        const float mn = fmaxf(m, max_groups<R>(mx) * s2), al = exp2_(m - mn);
        m = mn;
        l *= al;
        if constexpr (DUAL) cs *= al;
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          o[e] *= al;
          if constexpr (DUAL) od[e] *= al;
        }
      }
#pragma unroll
      for (int t = 0; t < NS * AV; ++t) {
        const float p = exp2_(fmaf(s[t / AV][t % AV], s2, -m));
        s[t / AV][t % AV] = p;
        l += p;
        if constexpr (DUAL) {
          const float pd = p * (sd[t / AV][t % AV] * a.scale);
          sd[t / AV][t % AV] = pd;
          cs += pd;
        }
      }
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        F pf, pdf;
        pack(s, c, pf);
        if constexpr (DUAL) pack(sd, c, pdf);
#pragma unroll
        for (int e = 0; e < NE; ++e) {
          const F vf = at.tfrag(sV, e, sb * NK + c);
          o[e] = mma(vf, pf, o[e]);
          if constexpr (DUAL) {
            od[e] = mma(vf, pdf, od[e]);
            od[e] = mma(at.tfrag(sVd, e, sb * NK + c), pf, od[e]);
          }
        }
      }
    }
  };
  for (int kb = 0; kb < nb; kb += 2) {   // (buffers at constant addresses)
    block(kb, std::false_type());
    if (kb + 1 < nb) block(kb + 1, std::true_type());
  }
  if constexpr (KS > 1) {
    // the other waves' keys join in, at the larger maximum
    Merge<R, NE, KS> M(reinterpret_cast<float*>(sK0), w, lane);
    static_assert(NW / KS * M.LANE * 256 <= sizeof(sK0), "merge buffer");
#pragma unroll
    for (int j = 1; j < KS; ++j) {
      __syncthreads();
      if (M.rank == j) {
        M.scalar(0) = m;
        M.scalar(1) = l;
        M.scalar(2) = cs;
      }
      __syncthreads();
      float f0 = 1.f, f1 = 1.f;
      if (M.rank == 0) {
        const float m1 = M.scalar(0), mn = fmaxf(m, m1);
        f0 = exp2_(m - mn);
        f1 = exp2_(m1 - mn);
        m = mn;
        l = l * f0 + M.scalar(1) * f1;
        cs = cs * f0 + M.scalar(2) * f1;
      }
      M.add(j, o, f0, f1);
      if constexpr (DUAL) M.add(j, od, f0, f1);
    }
    if (M.rank) return;
  }
  if (q >= hi) return;   // (lanes of one row leave together)
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
__device__ __forceinline__ float dot(const f32x4& a, const f32x4& b) {
  return a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3];
}

// 40 sequences of 16001 tokens in all, 16 heads of 128 over 2: 152 us, 0.61 PFLOP/s; dual, 2 x 4096
// tokens of 8 heads of 64: 142 us, 1.08.  Score cotangents are formed without the scale s,
// which the sums take at the end.
template <typename T, int DH, int R, int NW, int KS, int KB, int SB, int MW, bool PIN, bool DUAL>
__global__ void __launch_bounds__(64 * NW, MW) packed_dq_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * NW, NG = 64 / R, NS = SB / R, NE = DH / R, FE = FragT<T>::FE, NC = DH / (FE * NG);
  constexpr int AV = R * R / 64, NK = SB / (FE * NG), ROWS = NW * R / KS;
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sK0[KB * L::P], sK1[KB * L::P], sV0[KB * L::P], sV1[KB * L::P],
      sKd0[DUAL ? KB * L::P : 8], sKd1[DUAL ? KB * L::P : 8], sVd0[DUAL ? KB * L::P : 8], sVd1[DUAL ? KB * L::P : 8];
  int rank, h;
  tile_of(a.H, rank, h);
  const TileList tl = a.p.list[tile_kind(ROWS)];
  const int4 tile = tl.byq[rank];   // (its load does not wait for the count)
  if (rank >= a.p.head[tile_kind(ROWS)]) return;
  const int lo = tile.y, hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane % R, g = lane / R;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Lane<T, DH, R> at(lane);
  const int q0 = tile.x + w / KS * R, q = q0 + lr, qc = min(q, hi - 1);
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
  Block<T, DH, KB, NT> rK, rV, rKd, rVd;
  rK.init(a.ldk, dh, tid);
  rV.init(a.ldv, dh, tid);
  if constexpr (DUAL) {
    rKd.init(a.ldkd, dh, tid);
    rVd.init(a.ldvd, dh, tid);
  }
  auto load = [&](int k0, auto buffer) {
    constexpr bool b = decltype(buffer)::value;
    rK.load(K, k0, hi - 1, b ? sK1 : sK0, w);
    rV.load(Vp, k0, hi - 1, b ? sV1 : sV0, w);
    if constexpr (DUAL) {
      rKd.load(Kd, k0, hi - 1, b ? sKd1 : sKd0, w);
      rVd.load(Vd, k0, hi - 1, b ? sVd1 : sVd0, w);
    }
  };
  const int nb = (min(tile.x + ROWS, hi) - 1 - lo) / KB + 1;
  load(lo, std::false_type());
  auto block = [&](int kb, auto buffer) {
    constexpr bool b = decltype(buffer)::value;
    const T *sK = b ? sK1 : sK0, *sV = b ? sV1 : sV0, *sKd = b ? sKd1 : sKd0, *sVd = b ? sVd1 : sVd0;
    landed();
    const int k0 = lo + kb * KB;
    if (kb + 1 < nb) load(k0 + KB, std::bool_constant<!b>());
#pragma unroll
    for (int sb = 0; sb < KB / SB; ++sb) {
      const int ks = k0 + sb * SB;
      if (KS > 1 && sb % KS != w % KS) continue;
      if (ks > q0 + R - 1 || q0 >= hi) break;
      if constexpr (PIN) at.pin();
      const bool diag = ks + SB - 1 > q0;
      V ds[NS], dsd[DUAL ? NS : 1];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        V s, sd, dp, dpd;
        zero(s); zero(sd); zero(dp); zero(dpd);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int kr = sb * SB + n * R;
          const F kf = at.frag(sK, kr, c), vf = at.frag(sV, kr, c);
          s = mma(kf, qf[c], s);
          dp = mma(vf, gf[c], dp);
          if constexpr (DUAL) {
            sd = mma(kf, qdf[c], sd);
            sd = mma(at.frag(sKd, kr, c), qf[c], sd);
            dpd = mma(vf, gdf[c], dpd);
            dpd = mma(at.frag(sVd, kr, c), gf[c], dpd);
          }
        }
        if (diag) {   // some key may follow some query: its weight is 2^-inf = 0
#pragma unroll
          for (int t = 0; t < AV; ++t)
            if (ks + n * R + 4 * NG * (t / 4) + 4 * g + t % 4 > q) s[t] = -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < AV; ++t) {
          const float p = exp2_(fmaf(s[t], s2, -lse));
          const float x = dp[t] - r;
          ds[n][t] = p * x;
          if constexpr (DUAL) {
            const float pd = p * fmaf(sd[t], a.scale, -cst);
            dsd[n][t] = fmaf(pd, x, p * (dpd[t] - rd));
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
          const F kt = at.tfrag(sK, e, sb * NK + c);
          dq[e] = mma(kt, df, dq[e]);
          if constexpr (DUAL) {
            dqd[e] = mma(kt, ddf, dqd[e]);
            dqd[e] = mma(at.tfrag(sKd, e, sb * NK + c), df, dqd[e]);
          }
        }
      }
    }
  };
  for (int kb = 0; kb < nb; kb += 2) {   // (buffers at constant addresses)
    block(kb, std::false_type());
    if (kb + 1 < nb) block(kb + 1, std::true_type());
  }
  if constexpr (KS > 1) {
    Merge<R, NE, KS> M(reinterpret_cast<float*>(sK0), w, lane);
    static_assert(NW / KS * M.LANE * 256 <= sizeof(sK0), "merge buffer");
#pragma unroll
    for (int j = 1; j < KS; ++j) {
      M.add(j, dq, 1.f, 1.f);
      if constexpr (DUAL) M.add(j, dqd, 1.f, 1.f);
    }
    if (M.rank) return;
  }
  if (q >= hi) return;
  store_row<R, NE>(a.dq + q * a.lddq + (long)h * dh, dq, a.scale, g, dh);
  if constexpr (DUAL) store_row<R, NE>(a.dqd + q * a.lddqd + (long)h * dh, dqd, a.scale, g, dh);
}

// ---------------------------------------------------------------- backward: dK, dV
// The same calls: 163 us and 23 to add the parts, 0.66 PFLOP/s; dual 194 us, 1.06.
// A workgroup owns NW R / KS keys of one key head and goes through the queries of some of the
// head's query heads (all, or one part of `parts`, whose float32 sums dkv_sum_kernel
// adds in order).
template <typename T, int DH, int R, int NW, int KS, int KB, int SB, int MW, bool PIN, bool DUAL>
__global__ void __launch_bounds__(64 * NW, MW) packed_dkv_kernel(PackedAttnArgs<T> a) {
  constexpr int NT = 64 * NW, NG = 64 / R, NS = SB / R, NE = DH / R, FE = FragT<T>::FE, NC = DH / (FE * NG);
  constexpr int AV = R * R / 64, NK = SB / (FE * NG), ROWS = NW * R / KS;
  typedef typename AccT<R>::V V;
  typedef typename FragT<T>::V F;
  typedef Tile<T, DH> L;
  __shared__ __attribute__((aligned(16))) T sQ0[KB * L::P], sQ1[KB * L::P], sG0[KB * L::P], sG1[KB * L::P],
      sQd0[DUAL ? KB * L::P : 8], sQd1[DUAL ? KB * L::P : 8], sGd0[DUAL ? KB * L::P : 8], sGd1[DUAL ? KB * L::P : 8];
  __shared__ __attribute__((aligned(16))) float sL[2][KB], sR[2][KB], sC[2][KB], sRd[2][KB];
  int rank, hp;
  tile_of(a.K * a.parts, rank, hp);
  const TileList tl = a.p.list[tile_kind(ROWS)];
  const int4 tile = tl.byk[rank];
  if (rank >= a.p.head[tile_kind(ROWS)]) return;
  const int kh = hp / a.parts, part = hp - kh * a.parts, hi = tile.z;
  const int tid = threadIdx.x, lane = tid & 63, lr = lane % R, g = lane / R;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  Lane<T, DH, R> at(lane);
  const int k0 = tile.x + w / KS * R, k = k0 + lr, kc = min(k, hi - 1);
  const int GP = a.H / a.K / a.parts, dh = a.dh;   // query heads of a part
  const int h0 = (kh * a.parts + part) * GP;
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
  Block<T, DH, KB, NT> rQ, rG, rQd, rGd;
  rQ.init(a.ldq, dh, tid);
  rG.init(a.ldg, dh, tid);
  if constexpr (DUAL) {
    rQd.init(a.ldqd, dh, tid);
    rGd.init(a.ldgd, dh, tid);
  }
  float xL = 0.f, xR = 0.f, xC = 0.f, xRd = 0.f;   // a query's row values (threads 0 .. 63)
  const int nq = (hi - tile.x + KB - 1) / KB, nb = nq * GP;
  auto load = [&](int i, auto buffer) {   // block i: query head i / nq, its block i % nq
    constexpr bool b = decltype(buffer)::value;
    const int hq = i / nq, h = h0 + hq, r0 = tile.x + (i - hq * nq) * KB;
    rQ.load(a.q + (long)h * dh, r0, hi - 1, b ? sQ1 : sQ0, w);
    rG.load(a.g + (long)h * dh, r0, hi - 1, b ? sG1 : sG0, w);
    if constexpr (DUAL) {
      rQd.load(a.qd + (long)h * dh, r0, hi - 1, b ? sQd1 : sQd0, w);
      rGd.load(a.gd + (long)h * dh, r0, hi - 1, b ? sGd1 : sGd0, w);
    }
    const long x = (long)h * a.p.n + min(r0 + (tid & (KB - 1)), hi - 1);
    xL = a.lse[x];
    xR = a.r[x];
    if constexpr (DUAL) {
      xC = a.cst[x];
      xRd = a.rd[x];
    }
  };
  auto store = [&](int b) {
    if (tid < KB) {
      sL[b][tid] = xL;
      sR[b][tid] = xR;
      if constexpr (DUAL) {
        sC[b][tid] = xC;
        sRd[b][tid] = xRd;
      }
    }
  };
  load(0, std::false_type());
  store(0);
  int r0 = tile.x;   // first query of the block
  auto block = [&](int i, auto buffer) {
    constexpr bool b = decltype(buffer)::value;
    const T *sQ = b ? sQ1 : sQ0, *sG = b ? sG1 : sG0, *sQd = b ? sQd1 : sQd0, *sGd = b ? sGd1 : sGd0;
    landed();
    if (i + 1 < nb) load(i + 1, std::bool_constant<!b>());
#pragma unroll
    for (int sb = 0; sb < KB / SB; ++sb) {
      const int qs = r0 + sb * SB;
      if (KS > 1 && sb % KS != w % KS) continue;
      if (qs + SB - 1 < k0 || k0 >= hi || qs >= hi) continue;   // no query of these sees the wave's keys
      if constexpr (PIN) at.pin();
      const bool mask = qs < k0 + R - 1 || qs + SB > hi;
      V p[NS], ds[NS], pd[DUAL ? NS : 1], dsd[DUAL ? NS : 1];
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        V s, sd, dp, dpd;
        zero(s); zero(sd); zero(dp); zero(dpd);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const int qr = sb * SB + n * R;
          const F qq = at.frag(sQ, qr, c), gg = at.frag(sG, qr, c);
          s = mma(qq, kf[c], s);
          dp = mma(gg, vf[c], dp);
          if constexpr (DUAL) {
            sd = mma(qq, kdf[c], sd);
            sd = mma(at.frag(sQd, qr, c), kf[c], sd);
            dpd = mma(gg, vdf[c], dpd);
            dpd = mma(at.frag(sGd, qr, c), vf[c], dpd);
          }
        }
        if (mask) {   // (weight 0, as above)
#pragma unroll
          for (int t = 0; t < AV; ++t) {
            const int i1 = qs + n * R + 4 * NG * (t / 4) + 4 * g + t % 4;
            if (i1 < k || i1 >= hi) s[t] = -INFINITY;
          }
        }
#pragma unroll
        for (int t4 = 0; t4 < AV; t4 += 4) {
          const int i4 = sb * SB + n * R + NG * t4 + 4 * g;   // four queries of the block
          const f32x4 Lq = *reinterpret_cast<const f32x4*>(&sL[b][i4]);
          const f32x4 Rq = *reinterpret_cast<const f32x4*>(&sR[b][i4]);
          f32x4 Cq, Dq;
          if constexpr (DUAL) {
            Cq = *reinterpret_cast<const f32x4*>(&sC[b][i4]);
            Dq = *reinterpret_cast<const f32x4*>(&sRd[b][i4]);
          }
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int t = t4 + u;
            const float pv = exp2_(fmaf(s[t], s2, -Lq[u])), x = dp[t] - Rq[u];
            p[n][t] = pv;
            ds[n][t] = pv * x;
            if constexpr (DUAL) {
              const float pdv = pv * fmaf(sd[t], a.scale, -Cq[u]);
              pd[n][t] = pdv;
              dsd[n][t] = fmaf(pdv, x, pv * (dpd[t] - Dq[u]));
            }
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
          const F gt = at.tfrag(sG, e, sb * NK + c);
          const F qt = at.tfrag(sQ, e, sb * NK + c);
          dv[e] = mma(gt, pf, dv[e]);
          dk[e] = mma(qt, df, dk[e]);
          if constexpr (DUAL) {
            dvd[e] = mma(gt, pdf, dvd[e]);
            dvd[e] = mma(at.tfrag(sGd, e, sb * NK + c), pf, dvd[e]);
            dkd[e] = mma(qt, ddf, dkd[e]);
            dkd[e] = mma(at.tfrag(sQd, e, sb * NK + c), df, dkd[e]);
          }
        }
      }
    }
    r0 += KB;
    if (r0 >= hi) r0 = tile.x;
    if (i + 1 < nb) store(!b);
  };
  for (int i = 0; i < nb; i += 2) {
    block(i, std::false_type());
    if (i + 1 < nb) block(i + 1, std::true_type());
  }
  if constexpr (KS > 1) {
    Merge<R, NE, KS> M(reinterpret_cast<float*>(sQ0), w, lane);
    static_assert(NW / KS * M.LANE * 256 <= sizeof(sQ0), "merge buffer");
#pragma unroll
    for (int j = 1; j < KS; ++j) {
      M.add(j, dk, 1.f, 1.f);
      M.add(j, dv, 1.f, 1.f);
      if constexpr (DUAL) {
        M.add(j, dkd, 1.f, 1.f);
        M.add(j, dvd, 1.f, 1.f);
      }
    }
    if (M.rank) return;
  }
  if (k >= hi) return;
  if (a.parts > 1) {
    float* P = a.partial + (((long)part * a.p.n + k) * a.K + kh) * (DUAL ? 4 : 2) * dh;
    store_row<R, NE>(P, dk, a.scale, g, dh);
    store_row<R, NE>(P + dh, dv, 1.f, g, dh);
    if constexpr (DUAL) {
      store_row<R, NE>(P + 2 * dh, dkd, a.scale, g, dh);
      store_row<R, NE>(P + 3 * dh, dvd, 1.f, g, dh);
    }
    return;
  }
  store_row<R, NE>(a.dk + k * a.lddk + (long)kh * dh, dk, a.scale, g, dh);
  store_row<R, NE>(a.dv + k * a.lddv + (long)kh * dh, dv, 1.f, g, dh);
  if constexpr (DUAL) {
    store_row<R, NE>(a.dkd + k * a.lddkd + (long)kh * dh, dkd, a.scale, g, dh);
    store_row<R, NE>(a.dvd + k * a.lddvd + (long)kh * dh, dvd, 1.f, g, dh);
  }
}

// dK, dV (and tangents) as the sums of their parts, four dims a thread.
template <typename T>
__global__ void __launch_bounds__(256) dkv_sum_kernel(PackedAttnArgs<T> a) {
  const int na = a.dual ? 4 : 2, d4 = a.dh / 4;
  const long i = (long)blockIdx.x * 256 + threadIdx.x;
  const int per = a.K * na * d4;   // fours of a token
  const long tok = i / per;
  if (tok < a.p.head[PLAN_FIRST] || tok >= a.p.head[PLAN_LAST]) return;
  const int j = (int)(i - tok * per), d = 4 * (j % d4), k = j / d4 % na, kh = j / d4 / na;
  const float* P = a.partial + ((tok * a.K + kh) * na + k) * a.dh + d;
  f32x4 s = *reinterpret_cast<const f32x4*>(P);
  for (int p = 1; p < a.parts; ++p)
    s += *reinterpret_cast<const f32x4*>(P + (long)p * a.p.n * a.K * na * a.dh);
  T* out = k == 0 ? a.dk + tok * a.lddk : k == 1 ? a.dv + tok * a.lddv
         : k == 2 ? a.dkd + tok * a.lddkd : a.dvd + tok * a.lddvd;
  store4(out + (long)kh * a.dh + d, s[0], s[1], s[2], s[3]);
}

// ---------------------------------------------------------------- plan
// Once a batch: 6 us for the scan, 5 to 10 for the lists and positions at up to 16384 tokens.
// Bounds made ascending (running maximum of the clamped offsets) and, for every tile
// size, the tiles before each sequence, by one workgroup over chunks of its size.
constexpr int SCAN = 1024, SCAN_WAVES = SCAN / 64;

// Inclusive scan over the workgroup (and the total): in waves by shuffles, then over the
// waves' totals in `lds`.
template <typename Op>
__device__ __forceinline__ int scan(int v, Op op, int* lds, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(v, o, 64);
    if (lane >= o) v = op(v, x);
  }
  __syncthreads();   // (lds may still be read by the last scan)
  if (lane == 63) lds[w] = v;
  __syncthreads();
  total = lds[0];
#pragma unroll
  for (int i = 1; i < SCAN_WAVES; ++i) {
    if (w == i) v = op(v, total);
    total = op(total, lds[i]);
  }
  return v;
}

__global__ void __launch_bounds__(SCAN) plan_scan_kernel(SeqPlanArgs a) {
  __shared__ int lds[SCAN_WAVES];
  const int tid = threadIdx.x, m = a.p.m, n = (int)a.p.n;
  auto raw = [&](int j) {
    if (!a.cu) return (int)min((long)j * a.len, (long)n);
    if (!a.cover) return min(max(a.cu[j], 0), n);
    return j == 0 ? 0 : j == m ? n : min(max(a.cu[j - 1], 0), n);
  };
  int carry = 0, total;
  for (int j0 = 0; j0 <= m; j0 += SCAN) {
    const int j = j0 + tid;
    const int v = scan(j <= m ? raw(j) : 0, [](int x, int y) { return max(x, y); }, lds, total);
    if (j <= m) a.p.bound[j] = max(v, carry);
    carry = max(carry, total);
  }
  __syncthreads();
  for (int kind = 0; kind < TILE_KINDS; ++kind) {
    const int rows = tile_rows(kind);
    carry = 0;
    for (int j0 = 0; j0 <= m; j0 += SCAN) {
      const int j = j0 + tid;
      const int t = j < m ? (a.p.bound[j + 1] - a.p.bound[j] + rows - 1) / rows : 0;
      const int v = scan(t, [](int x, int y) { return x + y; }, lds, total);
      if (j <= m) a.p.list[kind].tstart[j] = carry + v - t;
      carry += total;
    }
    if (tid == 0) a.p.head[kind] = carry;
  }
  if (tid == 0) {
    a.p.head[PLAN_FIRST] = a.p.bound[0];
    a.p.head[PLAN_LAST] = a.p.bound[m];
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

// The first workgroups write the tile lists (of each size, by the keys a query tile sees and
// by the queries that see a key tile), longest first, by counting into SCAN classes of
// length; the order inside a class is free, since every tile's results are its own.
// The others write the positions.
constexpr int PLAN_LISTS = 2 * TILE_KINDS;
__global__ void __launch_bounds__(SCAN) plan_fill_kernel(SeqPlanArgs a) {
  const int m = a.p.m, tid = threadIdx.x;
  if (blockIdx.x >= PLAN_LISTS) {
    const long i = (long)(blockIdx.x - PLAN_LISTS) * SCAN + tid;
    if (i >= a.p.n) return;
    int pos = 0;
    if (a.positions)
      pos = a.positions[i];
    else if (i >= a.p.bound[0] && i < a.p.bound[m])
      pos = (int)i - a.p.bound[last_le(a.p.bound, m, (int)i)];
    a.p.pos[i] = pos;
    return;
  }
  __shared__ int count[SCAN], longest, lds[SCAN_WAVES];
  const int kind = blockIdx.x >> 1, byk = blockIdx.x & 1, rows = tile_rows(kind);
  const TileList l = a.p.list[kind];
  const int nt = a.p.head[kind];
  count[tid] = 0;
  if (tid == 0) longest = 1;
  __syncthreads();
  auto length = [&](int i, int4& t) {   // tiles i's rows meet
    const int j = last_le(l.tstart, m, i), k = i - l.tstart[j], lo = a.p.bound[j], hi = a.p.bound[j + 1];
    t = make_int4(lo + k * rows, lo, hi, 0);
    return byk ? (hi - lo + rows - 1) / rows - k : k + 1;
  };
  int4 t;
  for (int i = tid; i < nt; i += SCAN) atomicMax(&longest, length(i, t));
  __syncthreads();
  const int step = longest / SCAN + 1;
  for (int i = tid; i < nt; i += SCAN) atomicAdd(&count[SCAN - 1 - length(i, t) / step], 1);
  __syncthreads();
  const int own = count[tid];
  int total;
  const int before = scan(own, [](int x, int y) { return x + y; }, lds, total) - own;
  count[tid] = before;   // (every thread's own class)
  __syncthreads();
  int4* out = byk ? l.byk : l.byq;
  for (int i = tid; i < nt; i += SCAN) {
    const int c = SCAN - 1 - length(i, t) / step;
    out[atomicAdd(&count[c], 1)] = t;
  }
}

// Parts the query heads of a key head are split into for the dK/dV pass: while there are
// too few key tiles to fill the chip.
int dkv_parts(long n, int H, int K) {
  const int G = H / K;
  const long tiles = n / 128 + 1;
  for (int p = 1; p < G; ++p)
    if (G % p == 0 && tiles * K * p >= 1024) return p;
  return G;
}

// Rows a wave owns, waves of a workgroup, waves that share rows, rows of a staged block, rows
// of it that a wave forms and consumes scores of at a time, waves a SIMD holds, addresses
// pinned (Lane).  What they were chosen by, in us (the longer differences were measured
// with blocks staged through registers, which cost all of them a tenth more):
//  forward and dQ, 128 dims, bf16 (16001 tokens in 40 sequences of 16 heads | 16384 in one):
//   32 rows a wave, 4 waves, 104 | 1160 and 170; 16 rows, 4 waves 115 | 1380 and 178 (twice
//   the LDS reads a product); 16 rows, 8 waves 110 | 1200 and 200; blocks of 32 rows in the
//   forward 1003, of 64 1048;
//  dK/dV, 128 dims: 16 rows, 4 waves 209; 16 rows, 8 waves 246; 32 rows need more registers
//   than two waves a SIMD have: with the V fragments in LDS 4 x 4096 tokens take 950 us for
//   the whole backward, 1000 with 16 rows, but the 40 short sequences 368 and 340, whose
//   tiles they fill less;
//  dual, 64 dims (2 x 4096 tokens of 8 heads): 16 rows, 8 waves 112 and 344 (both backward
//   passes); 4 waves, blocks of 32 109 and 359; 32 rows 145 and 509;
//  dual, 128 dims (8191 tokens of 12 heads): dK/dV 16 rows, 4 waves, blocks of 64 and one wave
//   a SIMD, the backward 558; blocks of 32 and two waves a SIMD 640 (spills), with fragments
//   of the own rows in LDS 575; unpinned 580;
//  float32: 16 rows, one wave a SIMD (dual 64 dims: 32 rows take twice the time), but dual
//   up to 64 dims two waves and blocks of 32 (2 x 2048 tokens of 16 heads of 64: forward
//   456 -> 430, backward 1537 -> 1495);
//  few rows (bf16: 16 x 256 tokens of 8 heads, 64-row tiles 8.1, 9.6, 10.5, 128-row tiles 9.0,
//   11.4, 15.4; float32: 1531 tokens of 6 heads, pairs of waves sharing 32 rows 62, 79, 105,
//   64-row tiles 118, 166, 229).
enum Pass { FWD, DQ, DKV };
template <typename T, int DH, bool DUAL, int PASS, int SMALL>
struct Shape {
  static constexpr bool F32 = sizeof(T) == 4, BIG = DH > 64;
  static constexpr int R = !F32 && !DUAL && PASS != DKV && !SMALL ? 32 : 16;
  static constexpr int NW = !F32 && DUAL && !BIG && !SMALL ? 8 : 4;
  static constexpr int KS = F32 && SMALL ? 2 * SMALL : 1;
  static constexpr bool FEW = F32 && DUAL && !BIG && PASS != DKV && !SMALL;
  static constexpr int KB = FEW || (BIG && (DUAL ? F32 || PASS != DKV : !F32 && PASS == FWD)) ? 32 : 64;
  static constexpr int SB = F32 && KB < 32 * KS ? 16 : 32;
  static constexpr int MW = FEW ? 2 : F32 || (DUAL && BIG && PASS == DKV) ? 1 : 2;
  static constexpr bool PIN = DUAL && BIG && (F32 || PASS != FWD);
  static constexpr int KIND = tile_kind(NW * R / KS);
};

template <typename T, int DH, bool DUAL, int SMALL>
void launch_fwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  typedef Shape<T, DH, DUAL, FWD, SMALL> S;
  hipLaunchKernelGGL((packed_fwd_kernel<T, DH, S::R, S::NW, S::KS, S::KB, S::SB, S::MW, S::PIN, DUAL>),
                     dim3(a.p.max_tiles[S::KIND] * a.H), dim3(64 * S::NW), 0, s, a);
}
template <typename T, int DH, bool DUAL, int SMALL>
hipError_t launch_bwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  typedef Shape<T, DH, DUAL, DQ, SMALL> Q;
  typedef Shape<T, DH, DUAL, DKV, SMALL> S;
  hipLaunchKernelGGL((packed_dq_kernel<T, DH, Q::R, Q::NW, Q::KS, Q::KB, Q::SB, Q::MW, Q::PIN, DUAL>),
                     dim3(a.p.max_tiles[Q::KIND] * a.H), dim3(64 * Q::NW), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((packed_dkv_kernel<T, DH, S::R, S::NW, S::KS, S::KB, S::SB, S::MW, S::PIN, DUAL>),
                     dim3(a.p.max_tiles[S::KIND] * a.K * a.parts), dim3(64 * S::NW), 0, s, a);
  e = hipGetLastError();
  if (e != hipSuccess || a.parts == 1) return e;
  const long fours = a.p.n * a.K * (a.dual ? 4 : 2) * (a.dh / 4);
  hipLaunchKernelGGL(dkv_sum_kernel<T>, dim3((unsigned)((fours + 255) / 256)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// Few rows: smaller tiles, so that more workgroups share the work.  2, float32 only: four
// waves a 16-row tile, where sequences are long enough to divide (primal 1500 tokens of 8
// heads in 3 sequences 141 -> 110 us, dual 1531 of 6 in 4 257 -> 208; but dual 2000 of 8
// in 3 432 -> 484, 200 of 8 in 30 43 -> 60) and a staged block holds four sub-blocks.
template <typename T, int DH>
int small(const PackedAttnArgs<T>& a) {
  const long rows = a.p.n * a.H;
  if (sizeof(T) == 2) return rows < 512 * 128;
  if (rows < 192 * 64 && a.p.n >= 256L * a.p.m && !(DH > 64 && a.dual)) return 2;
  return rows < 512 * 64;
}
template <typename T, int DH, int SMALL>
hipError_t run_at(const PackedAttnArgs<T>& a, bool bwd, hipStream_t s) {
  if (bwd) return a.dual ? launch_bwd<T, DH, true, SMALL>(a, s) : launch_bwd<T, DH, false, SMALL>(a, s);
  if (a.dual) launch_fwd<T, DH, true, SMALL>(a, s); else launch_fwd<T, DH, false, SMALL>(a, s);
  return hipGetLastError();
}
template <typename T, int DH>
hipError_t run(const PackedAttnArgs<T>& a, bool bwd, hipStream_t s) {
  const int level = small<T, DH>(a);
  if constexpr (sizeof(T) == 4) {
    if (level == 2) {
      if constexpr (DH <= 64) return run_at<T, DH, 2>(a, bwd, s);
      if (bwd) return launch_bwd<T, DH, false, 2>(a, s);   // (primal: see small)
      launch_fwd<T, DH, false, 2>(a, s);
      return hipGetLastError();
    }
  }
  return level ? run_at<T, DH, 1>(a, bwd, s) : run_at<T, DH, 0>(a, bwd, s);
}
// The products' head dimension: dh rounded up to one that is compiled (columns past dh are
// zero, and not stored).
template <typename T>
hipError_t run_dh(const PackedAttnArgs<T>& a, bool bwd, hipStream_t s) {
  if (a.dh <= 32) return run<T, 32>(a, bwd, s);
  if constexpr (sizeof(T) == 4)
    if (a.dh <= 48) return run<T, 48>(a, bwd, s);
  if (a.dh <= 64) return run<T, 64>(a, bwd, s);
  if (a.dh <= 96) return run<T, 96>(a, bwd, s);
  return run<T, 128>(a, bwd, s);
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
  p.head = (int*)take(4 * (TILE_KINDS + 2));
  p.bound = (int*)take(4 * ((size_t)m + 1));
  p.pos = (int*)take(4 * (size_t)n);
  for (int k = 0; k < TILE_KINDS; ++k) {
    p.max_tiles[k] = (int)(n / tile_rows(k) + std::min((long)m, n));
    p.list[k].tstart = (int*)take(4 * ((size_t)m + 1));
    p.list[k].byq = (int4*)take(16 * (size_t)p.max_tiles[k]);
    p.list[k].byk = (int4*)take(16 * (size_t)p.max_tiles[k]);
  }
  if (bytes) *bytes = off;
  return p;
}

hipError_t seq_plan_make(const SeqPlanArgs& a, hipStream_t s) {
  if (a.p.n < 1) return hipSuccess;
  hipLaunchKernelGGL(plan_scan_kernel, dim3(1), dim3(SCAN), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(plan_fill_kernel, dim3((unsigned)(PLAN_LISTS + (a.p.n + SCAN - 1) / SCAN)),
                     dim3(SCAN), 0, s, a);
  return hipGetLastError();
}

size_t packed_attn_ws_floats(long n, int H, int K, int dh) {
  const int parts = dkv_parts(n, H, K);
  return 2 * (size_t)H * n + (parts > 1 ? (size_t)parts * n * K * 4 * dh : 0);
}
template <typename T>
void packed_attn_ws(PackedAttnArgs<T>& a, float* ws) {
  a.r = ws;
  a.rd = ws + (long)a.H * a.p.n;
  a.parts = dkv_parts(a.p.n, a.H, a.K);
  a.partial = a.rd + (long)a.H * a.p.n;
}

template <typename T>
hipError_t packed_attn_fwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  if (!shapes_ok(a)) return hipErrorInvalidValue;
  if (a.p.n < 1 || a.p.m < 1) return hipSuccess;
  return run_dh(a, false, s);
}

template <typename T>
hipError_t packed_attn_bwd(const PackedAttnArgs<T>& a, hipStream_t s) {
  if (!shapes_ok(a)) return hipErrorInvalidValue;
  if (a.p.n < 1 || a.p.m < 1) return hipSuccess;
  return run_dh(a, true, s);
}

template hipError_t packed_attn_fwd<bf16_t>(const PackedAttnArgs<bf16_t>&, hipStream_t);
template hipError_t packed_attn_fwd<float>(const PackedAttnArgs<float>&, hipStream_t);
template hipError_t packed_attn_bwd<bf16_t>(const PackedAttnArgs<bf16_t>&, hipStream_t);
template hipError_t packed_attn_bwd<float>(const PackedAttnArgs<float>&, hipStream_t);

template void packed_attn_ws<bf16_t>(PackedAttnArgs<bf16_t>&, float*);
template void packed_attn_ws<float>(PackedAttnArgs<float>&, float*);

}  // namespace mfmg
