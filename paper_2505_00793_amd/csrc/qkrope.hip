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
// Bound by memory: 65536 tokens of 32 + 8 + 8 heads of 128, bf16, 460 us forwards (5.2 TB/s)
// and 600 us backwards (4.9), where a large copy reaches 4.9.  Lanes of a wave hold 4 consecutive dims of a head; a wave goes
// through the heads of one token, so its angles are formed once.  They are formed in
// double precision down to a fraction of a quarter turn (exact to 2^-22 turns at
// position 2^31, 2^-38 at 2^15), then in float32: no table, and no limit on positions.
#include "packed.h"

#include <algorithm>
#include <cmath>
#include <cstring>

namespace mfmg {

namespace {

constexpr int WAVES = 4;   // of a workgroup
// Workgroups of a backward that sums gains: what its registers let the 256 CUs hold at once
// (5 and 3 waves a SIMD), so that all go through the rows together.  Dual, 8191 tokens of
// 16 + 2 heads of 128: 512 132, 768 117, 1024 128 us with the forward; primal, 65536
// tokens of 32 + 8: 768 1106, 1024 1054, 1280 1050.  (Fewer workgroups of 12 and 10 waves
// leave fewer partial sums, but wait for each other: 119 and 1200.)
constexpr int max_parts(bool dual) { return dual ? 768 : 1280; }

__device__ __forceinline__ f32x4 load4(const float* p) { return *reinterpret_cast<const f32x4*>(p); }
__device__ __forceinline__ f32x4 load4(const bf16_t* p) {
  const uint2 v = *reinterpret_cast<const uint2*>(p);
  return f32x4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u),
               __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xffff0000u)};
}
// Sum over the LPH lanes of a head, in all of them: quads, halves and rows of 16 lanes by
// DPP (each step adds what the mirrored lane holds of the other half), row pairs by
// exchanging rows.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
  return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// Lanes 0-15 and 16-31 of each half exchanged.
__device__ __forceinline__ float swap16(float v) {
  const unsigned u = __builtin_bit_cast(unsigned, v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(float, (threadIdx.x & 16) ? r[0] : r[1]);
}
template <int LPH>
__device__ __forceinline__ float head_sum(float v) {
  v += dpp<0xb1>(v);    // quad_perm 1 0 3 2
  v += dpp<0x4e>(v);    // quad_perm 2 3 0 1
  v += dpp<0x141>(v);   // row_half_mirror
  if (LPH >= 16) v += dpp<0x140>(v);   // row_mirror
  if (LPH >= 32) v += swap16(v);
  return v;
}
__device__ __forceinline__ float sum4(const f32x4& v) { return (v[0] + v[1]) + (v[2] + v[3]); }

__device__ __forceinline__ void put4(float* p, const f32x4& v) { store4(p, v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void put4(bf16_t* p, const f32x4& v) { store4(p, v[0], v[1], v[2], v[3]); }

// Rotation of a lane's dims d .. d + 3 of a head: z_k = y_k c_k + y'_k s_k with y' the
// pairs' other members (back: the transpose has -s), which the lane or another of the
// head's holds.
template <int LPH>
struct Rot {
  f32x4 c, s;
  double f4[4];   // quarter turns per position (0 past the rotated dims)
  int how;        // where y' is: 0 in the lane (interleaved), 1 in the lane LPH / 2 away
                  // (the whole head, LPH lanes), 2 in one other lane, 3 in any
  int rotated;    // dims of the lane's (first ones) that rotate: < 1 none, > 3 all; the others'
                  // y' is 0, so that an infinity passes as one
  int half;
  unsigned first; // bit k: dim k is its pair's first member

  __device__ __forceinline__ void init(const RopeFreqs& f, int d) {
    half = f.dims >> 1;
    how = f.interleaved ? 0 : LPH >= 16 && f.dims == 4 * LPH ? 1 : (f.dims & 7) == 0 ? 2 : 3;
    rotated = f.dims - d;
    first = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = d + k;
      f4[k] = 0.0;
      if (j < f.dims) {
        const bool one = f.interleaved ? !(j & 1) : j < half;
        f4[k] = f.f4[f.interleaved ? j >> 1 : one ? j : j - half];
        first |= (unsigned)one << k;
      }
    }
  }
  __device__ __forceinline__ void at(const RopeFreqs& f, int d, int pos) {
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      // the angle in quarter turns: q of them and the rest, t in [-pi/4, pi/4], by the
      // power series of sine (to t^9) and cosine (to t^10), exact to 2e-9 there
      const double a = (double)pos * f4[k], q = rint(a);
      const float t = (float)(a - q) * 1.57079632679489662f, t2 = t * t;
      const float sn = t * fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), 1.f);
      const float cs = fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, fmaf(t2, -1.f / 3628800, 1.f / 40320), -1.f / 720),
                                             1.f / 24), -0.5f), 1.f);
      const int n = (int)fma(-4.0, floor(0.25 * q), q);   // q mod 4
      const float cc = n & 1 ? -sn : cs, ss = n & 1 ? cs : sn;
      const float m = d + k >= f.dims ? 1.f : n & 2 ? -f.mscale : f.mscale;
      c[k] = cc * m;
      s[k] = first >> k & 1 ? -(ss * m) : ss * m;
    }
  }
  __device__ __forceinline__ f32x4 pairs(const f32x4& own) const {
    const auto keep = [](float v, int m) { return __builtin_bit_cast(float, __builtin_bit_cast(int, v) & m); };
    if (how == 0) {
      const int a = rotated > 0 ? -1 : 0, b = rotated > 2 ? -1 : 0;
      return f32x4{keep(own[1], a), keep(own[0], a), keep(own[3], b), keep(own[2], b)};
    }
    f32x4 v;
    if (how == 1) {
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = LPH == 32 ? swap16(own[k]) : dpp<0x128>(own[k]);   // row_ror 8
      return v;
    }
    const auto of = [](int lane, float x) {
      return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute(4 * lane, __builtin_bit_cast(int, x)));
    };
    const int lane = threadIdx.x & 63;
    if (how == 2) {   // (half is a multiple of 4, and the lane's dims rotate all or none)
      const int m = rotated > 0 ? -1 : 0, l = lane + ((first ? half >> 2 : -(half >> 2)) & m);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = keep(of(l, own[k]), m);
      return v;
    }
    const auto at = [&](int e) { e &= 3; return e == 0 ? own[0] : e == 1 ? own[1] : e == 2 ? own[2] : own[3]; };
#pragma unroll
    for (int k = 0; k < 4; ++k) {   // element k + half of a later lane, or k - half of an earlier one
      const float x = of(k < rotated ? lane + ((k + half) >> 2) : lane, at(k + half));
      const float y = of(k < rotated ? lane + ((k - half) >> 2) : lane, at(k - half));
      v[k] = k >= rotated ? 0.f : first >> k & 1 ? x : y;
    }
    return v;
  }
};

// ---------------------------------------------------------------- forward
// A wave takes every splits-th group of 64 / LPH heads of one token, the next group's
// values requested before the current one's arithmetic.  Lanes past the head (head dims
// that are no power of two) hold zeros.
template <typename T, int LPH, bool NORM, bool DUAL>
__global__ void __launch_bounds__(64 * WAVES) qk_rope_fwd_kernel(QkRopeArgs<T> a, int splits) {
  constexpr int HP = 64 / LPH;
  const int lane = threadIdx.x & 63, sub = lane / LPH, d = 4 * (lane % LPH);
  const long item = (long)blockIdx.x * WAVES + (threadIdx.x >> 6);
  const long tok = item / splits;
  if (tok < a.p.head[PLAN_FIRST] || tok >= a.p.head[PLAN_LAST]) return;
  const int dh = a.dh, nrot = a.H + a.K, nh = a.H + 2 * a.K, step = splits * HP;
  const bool live = d < dh;
  const f32x4 none = {0.f, 0.f, 0.f, 0.f};
  Rot<LPH> rot;
  rot.init(a.f, d);
  struct Row {
    f32x4 v, vd;
  };
  auto load = [&](int h) {
    Row r = {none, none};
    if (live && h < nh) {
      r.v = load4(a.x + tok * a.ldx + (long)h * dh + d);
      if constexpr (DUAL) r.vd = load4(a.xd + tok * a.ldxd + (long)h * dh + d);
    }
    return r;
  };
  int h = (int)(item % splits) * HP + sub;
  Row cur = load(h);
  rot.at(a.f, d, a.p.pos[tok]);
  f32x4 g[2], gd[2];   // q, k gains
  if constexpr (NORM) {
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      g[k] = live ? load4(a.gain + k * dh + d) : none;
      if constexpr (DUAL) gd[k] = live ? load4(a.gaind + k * dh + d) : none;
    }
  }
  const float inv = 1.0f / dh;
  for (; h < nh; h += step) {
    const Row next = load(h + step);
    f32x4 v = cur.v, vd = cur.vd;
    if (h < nrot) {
      if constexpr (NORM) {
        const bool k = h >= a.H;
        const f32x4 w = k ? g[1] : g[0];
        const float r = rsqrtf(head_sum<LPH>(sum4(v * v)) * inv + a.eps);
        if constexpr (DUAL) {
          const float c = r * head_sum<LPH>(sum4(v * vd)) * inv;
          vd = (k ? gd[1] : gd[0]) * (r * v) + w * (r * (vd - c * (r * v)));
        }
        v = w * (r * v);
      }
      v = v * rot.c + rot.pairs(v) * rot.s;
      if constexpr (DUAL) vd = vd * rot.c + rot.pairs(vd) * rot.s;
    }
    if (live) {
      put4(a.y + tok * a.ldy + (long)h * dh + d, v);
      if constexpr (DUAL) put4(a.yd + tok * a.ldyd + (long)h * dh + d, vd);
    }
    cur = next;
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
  const int lane = threadIdx.x & 63, sub = lane / LPH, d = 4 * (lane % LPH);
  const int w = threadIdx.x >> 6;
  const int dh = a.dh, nrot = a.H + a.K, nh = a.H + 2 * a.K, step = splits * HP;
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
  Rot<LPH> rot;
  rot.init(a.f, d);
  struct Row {
    f32x4 v, vd, x, xd;
  };
  for (long item = (long)blockIdx.x * WAVES + w; item < a.p.n * splits;
       item += (long)gridDim.x * WAVES) {
    const long tok = item / splits;
    if (tok < first || tok >= last) continue;
    auto load = [&](int h) {
      Row r = {none, none, none, none};
      if (live && h < nh) {
        r.v = load4(a.y + tok * a.ldy + (long)h * dh + d);
        if constexpr (DUAL) r.vd = load4(a.yd + tok * a.ldyd + (long)h * dh + d);
        if constexpr (NORM) {
          if (h < nrot) {
            r.x = load4(a.x + tok * a.ldx + (long)h * dh + d);
            if constexpr (DUAL) r.xd = load4(a.xd + tok * a.ldxd + (long)h * dh + d);
          }
        }
      }
      return r;
    };
    int h = (int)(item % splits) * HP + sub;
    Row cur = load(h);
    rot.at(a.f, d, a.p.pos[tok]);
    for (; h < nh; h += step) {
      const Row next = load(h + step);
      f32x4 v = cur.v, vd = cur.vd;
      if (h < nrot) {
        v = v * rot.c - rot.pairs(v) * rot.s;
        if constexpr (DUAL) vd = vd * rot.c - rot.pairs(vd) * rot.s;
        if constexpr (NORM) {
          const bool k = h >= a.H;
          const f32x4 e = (k ? g[1] : g[0]) * v;
          const float r = rsqrtf(head_sum<LPH>(sum4(cur.x * cur.x)) * inv + a.eps);
          const float m = r * head_sum<LPH>(sum4(cur.x * e)) * inv;
          const f32x4 xh = r * cur.x, u = e - m * xh, dg = v * xh;
          if (k) acc[1] += dg; else acc[0] += dg;
          if constexpr (DUAL) {
            const f32x4 ed = (k ? gd[1] : gd[0]) * v + (k ? g[1] : g[0]) * vd;
            const float c = r * head_sum<LPH>(sum4(cur.x * cur.xd)) * inv;
            const f32x4 xhd = r * (cur.xd - c * xh), dgd = vd * xh + v * xhd;
            const float md = head_sum<LPH>(sum4(xhd * e + xh * ed)) * inv;
            if (k) acc[3] += dgd; else acc[2] += dgd;
            vd = (-r * r * c) * u + r * (ed - m * xhd - md * xh);
          }
          v = r * u;
        }
      }
      if (live) {
        put4(a.dx + tok * a.lddx + (long)h * dh + d, v);
        if constexpr (DUAL) put4(a.dxd + tok * a.lddxd + (long)h * dh + d, vd);
      }
      cur = next;
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

// Partials in groups of GROUP consecutive ones, added in order: [parts][4][dh] ->
// [cdiv(parts, GROUP)][4][dh] behind them.
constexpr int GROUP = 32;
__global__ void __launch_bounds__(256) gain_group_kernel(const float* __restrict__ partial, int parts,
                                                         int cols, float* __restrict__ out) {
  __shared__ float red[4][64];
  const int c = threadIdx.x & 63, ph = threadIdx.x >> 6, j = blockIdx.x * 64 + c;
  const int p0 = blockIdx.y * GROUP + ph * (GROUP / 4);
  float v[GROUP / 4];
#pragma unroll
  for (int k = 0; k < GROUP / 4; ++k)
    v[k] = j < cols && p0 + k < parts ? partial[(long)(p0 + k) * cols + j] : 0.f;
  float s = 0.f;
#pragma unroll
  for (int k = 0; k < GROUP / 4; ++k) s += v[k];
  red[ph][c] = s;
  __syncthreads();
  if (ph == 0 && j < cols) out[(long)blockIdx.y * cols + j] = (red[0][c] + red[1][c]) + (red[2][c] + red[3][c]);
}

int lanes_per_head(int dh) { return dh <= 32 ? 8 : dh <= 64 ? 16 : 32; }

// Waves of one token: its groups of heads are dealt evenly to more waves while there are too
// few tokens to fill the chip (999 tokens of 10 + 5 heads of 80, dual: up to 8192 waves 31 us,
// 4096 27.5, 2048 27.1, where each forms the angles anew; 256 tokens the same either way).
int splits_of(long n, int H, int K, int dh) {
  const int hp = 64 / lanes_per_head(dh), groups = (H + 2 * K + hp - 1) / hp;
  int s = 1;
  while (s < groups && n * s < 2048) s *= 2;
  const int per = (groups + s - 1) / s;
  return (groups + per - 1) / per;
}
int bwd_blocks(long n, int H, int K, int dh, bool dual) {   // (with norms)
  const long items = n * splits_of(n, H, K, dh);
  return (int)std::min((long)max_parts(dual), std::max(1L, (items + WAVES - 1) / WAVES));
}

// Few partials are left as they are.
int gain_groups(int parts) { return parts <= GROUP ? parts : (parts + GROUP - 1) / GROUP; }

template <typename T, int LPH, bool NORM, bool DUAL>
hipError_t launch(const QkRopeArgs<T>& a, bool bwd, hipStream_t s) {
  const int splits = splits_of(a.p.n, a.H, a.K, a.dh);
  if (bwd) {
    const int blocks = NORM ? bwd_blocks(a.p.n, a.H, a.K, a.dh, DUAL)
                            : (int)((a.p.n * splits + WAVES - 1) / WAVES);
    hipLaunchKernelGGL((qk_rope_bwd_kernel<T, LPH, NORM, DUAL>), dim3(blocks), dim3(64 * WAVES), 0,
                       s, a, splits);
    const int groups = gain_groups(blocks);
    if (NORM && groups < blocks) {
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(gain_group_kernel, dim3((4 * a.dh + 63) / 64, groups), dim3(256), 0, s,
                         a.partial, blocks, 4 * a.dh, a.partial + (long)blocks * 4 * a.dh);
    }
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

int qk_rope_partials(long n, int H, int K, int dh) {
  const int parts = bwd_blocks(n, H, K, dh, false);
  return parts + gain_groups(parts);
}
const float* qk_rope_sums(const float* partial, long n, int H, int K, int dh, bool dual, int* count) {
  const int parts = bwd_blocks(n, H, K, dh, dual);
  *count = gain_groups(parts);
  return *count < parts ? partial + (long)parts * 4 * dh : partial;
}

template <typename T>
hipError_t qk_rope_fwd(const QkRopeArgs<T>& a, hipStream_t s) { return launch_heads(a, false, s); }
template <typename T>
hipError_t qk_rope_bwd(const QkRopeArgs<T>& a, hipStream_t s) { return launch_heads(a, true, s); }

template hipError_t qk_rope_fwd<bf16_t>(const QkRopeArgs<bf16_t>&, hipStream_t);
template hipError_t qk_rope_fwd<float>(const QkRopeArgs<float>&, hipStream_t);
template hipError_t qk_rope_bwd<bf16_t>(const QkRopeArgs<bf16_t>&, hipStream_t);
template hipError_t qk_rope_bwd<float>(const QkRopeArgs<float>&, hipStream_t);

}  // namespace mfmg
