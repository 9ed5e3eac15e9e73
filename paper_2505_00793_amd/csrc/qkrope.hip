// RMS norms of query and key heads and rotary positions, in one pass over the rows of
// a QKV product, forwards and backwards, with tangents.
//
// One head x of n = head_dim values with gain g, at position pos:
//   r = (mean(x^2) + eps)^(-1/2),  xh = r x,  y = g xh,  z = R(pos) y,
// where R turns pair j by the angle pos * theta_j (and scales the rotated dims by
// mscale); without norms y = x.  Its tangent, with c = mean(xh xd):
//   xhd = r (xd - c xh),  yd = gd xh + g xhd,  zd = R yd.
// Backward from dz: dy = R^T dz, e = g dy, m = mean(xh e),
//   dx = r (e - xh m),  dg = sum dy xh,
// and along the tangent, with ed = gd dy + g dyd and md = mean(xhd e + xh ed),
//   dxd = -r^2 c (e - xh m) + r (ed - xhd m - xh md),  dgd = sum dyd xh + dy xhd.
// The norm is recomputed from x in the backward (nothing is saved).  Value heads pass
// through.
//
// Bound by memory.  Lanes of a wave hold 4 consecutive dims of a head; a wave goes
// through the heads of one token, so its angles are formed once.  They are formed in
// double precision down to a fraction of a quarter turn (exact to 2^-22 turns at
// position 2^31, 2^-38 at 2^15), then in float32: no table, and no limit on positions.
#include "packed.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace mfmg {

namespace {

constexpr int WAVES = 4;          // of a workgroup
constexpr int MAX_PARTS = 1024;   // workgroups of a backward that sums gains

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
               __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const bf16_t* p) { return bf2f(*p); }

template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
#pragma unroll
  for (int o = LPH / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
__device__ __forceinline__ float sum4(const f32x4& v) { return (v[0] + v[1]) + (v[2] + v[3]); }

// Rotation of a lane's dims d .. d + 3 of a head at one position: z_k = y_k c_k + y'_k s_k
// with y' the pairs' other members (back: the transpose has -s).
struct Rot {
  f32x4 c, s;
  int other;    // first dim of y' where the four are consecutive and 4-aligned, else -1
  int odd[4];   // else their dims

  __device__ __forceinline__ void make(const RopeFreqs& f, int d, int pos) {
    const int half = f.dims >> 1;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = d + k;
      c[k] = 1.f;
      s[k] = 0.f;
      odd[k] = j;
      if (j < f.dims) {
        const bool first = f.interleaved ? !(j & 1) : j < half;
        const int pair = f.interleaved ? j >> 1 : first ? j : j - half;
        odd[k] = f.interleaved ? j ^ 1 : first ? j + half : j - half;
        // the angle in quarter turns: k of them and t in [-1/2, 1/2]
        const double a = (double)pos * f.f4[pair], q = rint(a);
        float sn, cs;
        sincospif(0.5f * (float)(a - q), &sn, &cs);
        const int n = (int)(long long)q & 3;
        const float cc = n & 1 ? -sn : cs, ss = n & 1 ? cs : sn;
        const float m = n & 2 ? -f.mscale : f.mscale;
        c[k] = cc * m;
        s[k] = first ? -(ss * m) : ss * m;
      }
    }
    other = (odd[0] & 3) == 0 && odd[3] == odd[0] + 3 ? odd[0] : -1;
  }
  // the pairs' other members of a head in memory
  template <typename T>
  __device__ __forceinline__ f32x4 pairs(const T* head, const f32x4& own, const RopeFreqs& f) const {
    if (f.interleaved) {   // (a lane's dims are whole pairs; s is 0 past the rotated dims)
      return f32x4{own[1], own[0], own[3], own[2]};
    }
    if ((f.dims & 7) == 0) return load4(head + other);
    f32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = load1(head + odd[k]);
    return v;
  }
};

__device__ __forceinline__ void put4(float* p, const f32x4& v) { store4(p, v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void put4(bf16_t* p, const f32x4& v) { store4(p, v[0], v[1], v[2], v[3]); }

// ---------------------------------------------------------------- forward
// A wave takes every splits-th group of 64 / LPH heads of one token.  Lanes past the
// head (head dims that are no power of two) hold zeros.
template <typename T, int LPH, bool NORM, bool DUAL>
__global__ void __launch_bounds__(64 * WAVES) qk_rope_fwd_kernel(QkRopeArgs<T> a, int splits) {
  constexpr int HP = 64 / LPH;
  const int lane = threadIdx.x & 63, sub = lane / LPH, d = 4 * (lane % LPH);
  const long item = (long)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const long tok = item / splits;
  if (tok < a.p.head[PLAN_FIRST] || tok >= a.p.head[PLAN_LAST]) return;
  const int dh = a.dh, nrot = a.H + a.K, nh = a.H + 2 * a.K;
  const bool live = d < dh;
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  Rot rot;
  rot.make(a.f, d, a.p.pos[tok]);
  f32x4 g[2], gp[2], gd[2], gdp[2];   // q, k gains and those of the pairs' other members
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      g[k] = live ? load4(a.gain + k * dh + d) : none;
      gp[k] = live ? rot.pairs(a.gain + k * dh, g[k], a.f) : none;
      if constexpr (DUAL) {
        gd[k] = live ? load4(a.gaind + k * dh + d) : none;
        gdp[k] = live ? rot.pairs(a.gaind + k * dh, gd[k], a.f) : none;
      }
    }
  }
  const float inv = 1.0f / dh;
  for (int h = (int)(item % splits) * HP + sub; h < nh; h += splits * HP) {
    const float* x = a.x + tok * a.ldx + (long)h * dh;
    const float* xd = DUAL ? a.xd + tok * a.ldxd + (long)h * dh : nullptr;
    f32x4 v = live ? load4(x + d) : none, vd = none;
    if constexpr (DUAL) vd = live ? load4(xd + d) : none;
    if (h < nrot) {
      f32x4 p = live ? rot.pairs(x, v, a.f) : none, pd = none;
      if constexpr (DUAL) pd = live ? rot.pairs(xd, vd, a.f) : none;
      if constexpr (NORM) {
        const int k = h >= a.H;
        const float r = rsqrtf(head_sum<LPH>(sum4(v * v)) * inv + a.eps);
        if constexpr (DUAL) {
          const float c = r * head_sum<LPH>(sum4(v * vd)) * inv;
          vd = gd[k] * (r * v) + g[k] * (r * (vd - c * (r * v)));
          pd = gdp[k] * (r * p) + gp[k] * (r * (pd - c * (r * p)));
        }
        v = g[k] * (r * v);
        p = gp[k] * (r * p);
      }
      v = v * rot.c + p * rot.s;
      if constexpr (DUAL) vd = vd * rot.c + pd * rot.s;
    }
    if (live) {
      put4(a.y + tok * a.ldy + (long)h * dh + d, v);
      if constexpr (DUAL) put4(a.yd + tok * a.ldyd + (long)h * dh + d, vd);
    }
  }
}

// ---------------------------------------------------------------- backward
// A workgroup's waves take items (token, split) strided by the grid; with norms each
// lane sums its dims' gain gradients on the way, and the workgroup adds its lanes' in a
// fixed order into its own partial.
template <typename T, int LPH, bool NORM, bool DUAL>
__global__ void __launch_bounds__(64 * WAVES) qk_rope_bwd_kernel(QkRopeArgs<T> a, int splits) {
  constexpr int HP = 64 / LPH, NA = NORM ? (DUAL ? 4 : 2) : 0;
  __shared__ float red[NORM ? WAVES * HP * 4 * 4 * LPH : 1];
  const int lane = threadIdx.x & 63, sub = lane / LPH, i = lane % LPH, d = 4 * i;
  const int w = threadIdx.x >> 6;
  const int dh = a.dh, nrot = a.H + a.K, nh = a.H + 2 * a.K;
  const bool live = d < dh;
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  f32x4 acc[NORM ? 4 : 1];   // q, k gains' gradients, then their tangents
  f32x4 g[2], gd[2];
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[k] = none;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      g[k] = live ? load4(a.gain + k * dh + d) : none;
      if constexpr (DUAL) gd[k] = live ? load4(a.gaind + k * dh + d) : none;
    }
  }
  const float inv = 1.0f / dh;
  const long first = a.p.head[PLAN_FIRST], last = a.p.head[PLAN_LAST];
  for (long item = (long)blockIdx.x * WAVES + w; item < a.p.n * splits;
       item += (long)gridDim.x * WAVES) {
    const long tok = item / splits;
    if (tok < first || tok >= last) continue;
    Rot rot;
    rot.make(a.f, d, a.p.pos[tok]);
    for (int h = (int)(item % splits) * HP + sub; h < nh; h += splits * HP) {
      const long col = (long)h * dh;
      const T* y = a.y + tok * a.ldy + col;
      const T* yd = DUAL ? a.yd + tok * a.ldyd + col : nullptr;
      f32x4 v = live ? load4(y + d) : none, vd = none;
      if constexpr (DUAL) vd = live ? load4(yd + d) : none;
      if (h < nrot) {
        v = v * rot.c - (live ? rot.pairs(y, v, a.f) : none) * rot.s;
        if constexpr (DUAL) vd = vd * rot.c - (live ? rot.pairs(yd, vd, a.f) : none) * rot.s;
        if constexpr (NORM) {
          const int k = h >= a.H;
          const f32x4 x = live ? load4(a.x + tok * a.ldx + col + d) : none;
          const f32x4 e = g[k] * v;
          const float r = rsqrtf(head_sum<LPH>(sum4(x * x)) * inv + a.eps);
          const float m = r * head_sum<LPH>(sum4(x * e)) * inv;
          const f32x4 xh = r * x;
          const f32x4 u = e - m * xh;
          acc[k] += v * xh;
          if constexpr (DUAL) {
            const f32x4 xd = live ? load4(a.xd + tok * a.ldxd + col + d) : none;
            const f32x4 ed = gd[k] * v + g[k] * vd;
            const float c = r * head_sum<LPH>(sum4(x * xd)) * inv;
            const f32x4 xhd = r * (xd - c * xh);
            const float md = head_sum<LPH>(sum4(xhd * e + xh * ed)) * inv;
            acc[2 + k] += vd * xh + v * xhd;
            vd = (-r * r * c) * u + r * (ed - m * xhd - md * xh);
          }
          v = r * u;
        }
      }
      if (live) {
        put4(a.dx + tok * a.lddx + col + d, v);
        if constexpr (DUAL) put4(a.dxd + tok * a.lddxd + col + d, vd);
      }
    }
  }
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < NA; ++k)
#pragma unroll
      for (int t = 0; t < 4; ++t) red[((w * HP + sub) * 4 + k) * 4 * LPH + d + t] = acc[k][t];
    __syncthreads();
    for (int j = threadIdx.x; j < 4 * dh; j += 64 * WAVES) {
      const int k = j / dh, c = j % dh;
      float sum = 0.f;
      if (k < NA)
        for (int q = 0; q < WAVES * HP; ++q) sum += red[(q * 4 + k) * 4 * LPH + c];
      a.partial[(long)blockIdx.x * 4 * dh + j] = sum;
    }
  }
}

int lanes_per_head(int dh) { return dh <= 32 ? 8 : dh <= 64 ? 16 : 32; }

// Waves of one token: its groups of heads are dealt to more waves while there are too
// few tokens to fill the chip.
int splits_of(long n, int H, int K, int dh) {
  const int hp = 64 / lanes_per_head(dh), groups = (H + 2 * K + hp - 1) / hp;
  int s = 1;
  while (s < groups && n * s < 8192) s *= 2;
  return std::min(s, groups);
}
int bwd_blocks(long n, int H, int K, int dh) {
  const long items = n * splits_of(n, H, K, dh);
  return (int)std::min((long)MAX_PARTS, std::max(1L, (items + WAVES - 1) / WAVES));
}

template <typename T, int LPH, bool NORM, bool DUAL>
hipError_t launch(const QkRopeArgs<T>& a, bool bwd, hipStream_t s) {
  const int splits = splits_of(a.p.n, a.H, a.K, a.dh);
  if (bwd) {
    hipLaunchKernelGGL((qk_rope_bwd_kernel<T, LPH, NORM, DUAL>),
                       dim3(bwd_blocks(a.p.n, a.H, a.K, a.dh)), dim3(64 * WAVES), 0, s, a, splits);
  } else {
    const long blocks = (a.p.n * splits + WAVES - 1) / WAVES;
    hipLaunchKernelGGL((qk_rope_fwd_kernel<T, LPH, NORM, DUAL>), dim3((unsigned)blocks),
                       dim3(64 * WAVES), 0, s, a, splits);
  }
  return hipGetLastError();
}
template <typename T, int LPH>
hipError_t launch_kind(const QkRopeArgs<T>& a, bool bwd, hipStream_t s) {
  if (a.gain)
    return a.dual ? launch<T, LPH, true, true>(a, bwd, s) : launch<T, LPH, true, false>(a, bwd, s);
  return a.dual ? launch<T, LPH, false, true>(a, bwd, s) : launch<T, LPH, false, false>(a, bwd, s);
}
template <typename T>
hipError_t launch_heads(const QkRopeArgs<T>& a, bool bwd, hipStream_t s) {
  if (a.p.n < 1) return hipSuccess;
  if (a.dh < 8 || a.dh > PK_MAX_DH || a.dh % 8 || a.f.dims < 2 || a.f.dims > a.dh || a.f.dims % 2 ||
      a.K < 1 || a.H < 1 || a.p.n > PK_MAX_TOKENS)
    return hipErrorInvalidValue;
  switch (lanes_per_head(a.dh)) {
    case 8: return launch_kind<T, 8>(a, bwd, s);
    case 16: return launch_kind<T, 16>(a, bwd, s);
    default: return launch_kind<T, 32>(a, bwd, s);
  }
}

}  // namespace

const char* attn_desc_error(const mfmg_attn_desc& d) {
  if (d.heads < 1 || d.heads > PK_MAX_HEADS || d.kv_heads < 1 || d.kv_heads > d.heads ||
      d.heads % d.kv_heads)
    return "heads must be in [1, 1024] and a multiple of kv_heads";
  if (d.head_dim < 8 || d.head_dim > PK_MAX_DH || d.head_dim % 8)
    return "head_dim must be a multiple of 8 in [8, 128]";
  if (d.precision != MFMG_PREC_FP32 && d.precision != MFMG_PREC_BF16) return "unknown precision";
  if (!std::isfinite(d.scale) || d.scale < 0.f) return "scale must be finite and >= 0";
  if (d.qk_norm != 0 && d.qk_norm != 1) return "qk_norm must be 0 or 1";
  if (d.qk_norm && !(d.norm_eps > 0.f && std::isfinite(d.norm_eps))) return "norm_eps must be > 0";
  if (d.rope_dims < 0 || d.rope_dims > d.head_dim || d.rope_dims % 2)
    return "rope_dims must be even and in [0, head_dim]";
  if (d.rope_interleaved != 0 && d.rope_interleaved != 1) return "rope_interleaved must be 0 or 1";
  if (!(d.rope_base > 0.f) || !std::isfinite(d.rope_base)) return "rope_base must be > 0";
  if (!std::isfinite(d.rope_mscale) || d.rope_mscale < 0.f) return "rope_mscale must be finite and >= 0";
  if (d.rope_scaling < MFMG_ROPE_PLAIN || d.rope_scaling > MFMG_ROPE_PARTS)
    return "unknown rope_scaling";
  if (d.rope_scaling != MFMG_ROPE_PLAIN && !(d.rope_factor >= 1.f && std::isfinite(d.rope_factor)))
    return "rope_factor must be >= 1";
  if (d.rope_scaling == MFMG_ROPE_BASE && d.rope_dims == 2) return "MFMG_ROPE_BASE needs rope_dims >= 4";
  if (d.rope_scaling == MFMG_ROPE_PARTS &&
      (!(d.rope_train_len > 0.f) || !std::isfinite(d.rope_train_len) || !std::isfinite(d.rope_slow) ||
       !std::isfinite(d.rope_fast) || !(d.rope_fast > d.rope_slow)))
    return "MFMG_ROPE_PARTS needs rope_train_len > 0 and rope_fast > rope_slow";
  return nullptr;
}

RopeFreqs rope_freqs(const mfmg_attn_desc& d) {
  RopeFreqs f;
  std::memset(&f, 0, sizeof(f));
  const double pi = 3.14159265358979323846;
  const int D = d.rope_dims ? d.rope_dims : d.head_dim;
  double base = d.rope_base;
  if (d.rope_scaling == MFMG_ROPE_BASE) base *= std::pow((double)d.rope_factor, D / (D - 2.0));
  f.dims = D;
  f.interleaved = d.rope_interleaved;
  f.mscale = d.rope_mscale != 0.f ? d.rope_mscale : 1.f;
  for (int j = 0; j < D / 2; ++j) {
    double th = std::pow(base, -2.0 * j / D);
    if (d.rope_scaling == MFMG_ROPE_LINEAR) th /= d.rope_factor;
    if (d.rope_scaling == MFMG_ROPE_PARTS) {
      const double turns = d.rope_train_len * th / (2.0 * pi);
      const double w = std::min(1.0, std::max(0.0, (turns - d.rope_slow) /
                                                       ((double)d.rope_fast - d.rope_slow)));
      th *= (1.0 - w) / d.rope_factor + w;
    }
    f.f4[j] = th * 2.0 / pi;
  }
  return f;
}

int qk_rope_parts(long n, int H, int K, int dh) { return bwd_blocks(n, H, K, dh); }

template <typename T>
hipError_t qk_rope_fwd(const QkRopeArgs<T>& a, hipStream_t s) { return launch_heads(a, false, s); }
template <typename T>
hipError_t qk_rope_bwd(const QkRopeArgs<T>& a, hipStream_t s) { return launch_heads(a, true, s); }

template hipError_t qk_rope_fwd<bf16_t>(const QkRopeArgs<bf16_t>&, hipStream_t);
template hipError_t qk_rope_fwd<float>(const QkRopeArgs<float>&, hipStream_t);
template hipError_t qk_rope_bwd<bf16_t>(const QkRopeArgs<bf16_t>&, hipStream_t);
template hipError_t qk_rope_bwd<float>(const QkRopeArgs<float>&, hipStream_t);

}  // namespace mfmg
