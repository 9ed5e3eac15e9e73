// Interfaces of the packed-sequence attention operators (packed.hip, qkrope.hip).
#pragma once

#include "kernels.h"
#include "mfmg.h"

namespace mfmg {

// Attention tiles of four sizes: 16, 32, 64 and 128 rows (queries or keys).
constexpr int TILE_KINDS = 4;
__host__ __device__ constexpr int tile_rows(int kind) { return 16 << kind; }
__host__ __device__ constexpr int tile_kind(int rows) {
  return rows == 128 ? 3 : rows == 64 ? 2 : rows == 32 ? 1 : 0;
}
constexpr int PLAN_FIRST = TILE_KINDS, PLAN_LAST = TILE_KINDS + 1;   // of SeqPlan::head
constexpr int PK_MAX_DH = 128;      // largest head dimension
// A grid is at most 2^32 threads: 64 a token for the rotation, and what attn_grid_fits says.
constexpr long PK_MAX_TOKENS = (1L << 26) - 1;
constexpr int PK_MAX_SEQS = 1 << 20;
constexpr int PK_MAX_HEADS = 1024;
constexpr int ROPE_MAX_PAIRS = PK_MAX_DH / 2;

// What the kernels need to know of a batch's sequences, in device memory.
// Sequences are [b[j], b[j + 1]), j < m; tokens outside [b[0], b[m]) are unused rows.
// A tile is (first row, b[j], b[j + 1], 0) of its sequence j; the lists are longest first.
struct TileList {
  int* tstart;    // [m + 1] tiles before sequence j
  int4* byq;      // [max_tiles] as query tiles, by the keys they see
  int4* byk;      // [max_tiles] as key tiles, by the queries that see them
};
struct SeqPlan {
  int* head;      // [TILE_KINDS + 2] tiles of each size, then b[0], b[m]
  int* bound;     // [m + 1] b
  int* pos;       // [n] rotary position of each token
  TileList list[TILE_KINDS];
  long n;
  int m, max_tiles[TILE_KINDS];
};
// Whether the attention grids of `heads` heads over n tokens and m sequences can be launched
// (256 threads a tile of 64 rows, 512 one of 128).
inline bool attn_grid_fits(long n, int m, int heads) {
  return (n / 64 + 2 * (m < n ? (long)m : n) + 1) * heads * 256 < (1L << 32);
}
// Layout of a plan over n tokens and m sequences at `base` (null: measure);
// *bytes receives its size.
SeqPlan seq_plan_at(char* base, long n, int m, size_t* bytes);

// Fills a plan.  cu: m + 1 ascending offsets (clamped to ascending values within
// 0 .. n), or with `cover` m - 1 inner ones, the first and last bound being 0 and n;
// null: sequences of `len` tokens each.  positions: null for the index within the
// sequence.
struct SeqPlanArgs {
  const int* cu;
  const int* positions;
  int cover, len;
  SeqPlan p;
};
hipError_t seq_plan_make(const SeqPlanArgs& a, hipStream_t s);

// Causal attention over the plan's sequences.  Row pointers are T rows by token,
// head h at columns h * dh; dual: the tangents' are set.
template <typename T>
struct PackedAttnArgs {
  const T *q, *k, *v;
  const T *qd, *kd, *vd;
  T *o, *od;                      // backward: read
  const T *g, *gd;                // cotangent of o (and its tangent)
  T *dq, *dk, *dv;
  T *dqd, *dkd, *dvd;
  long ldq, ldk, ldv, ldqd, ldkd, ldvd, ldo, ldod, ldg, ldgd;
  long lddq, lddk, lddv, lddqd, lddkd, lddvd;
  float* lse;                     // [H][n] log2 of the softmax denominators, scaled scores' base 2
  float* cst;                     // [H][n] <P, Sd> (dual)
  float *r, *rd;                  // [H][n] backward workspace: <dO, O>, <dOd, O> + <dO, Od>
  float* partial;                 // [parts][n][K][2 or 4][dh] backward workspace: dK, dV (and
  int parts;                      //   tangents) of parts of the query heads (parts > 1)
  SeqPlan p;
  int H, K, dh, dual;
  float scale;
};
// Floats of the backward's workspace, and its parts (r, rd, partial, parts of a, whose n, H,
// K are set) at `ws`.
size_t packed_attn_ws_floats(long n, int H, int K, int dh);
template <typename T>
void packed_attn_ws(PackedAttnArgs<T>& a, float* ws);
template <typename T>
hipError_t packed_attn_fwd(const PackedAttnArgs<T>& a, hipStream_t s);
template <typename T>
hipError_t packed_attn_bwd(const PackedAttnArgs<T>& a, hipStream_t s);

// Rotation (and RMS norm) of the query and key heads of QKV rows.
// Returns nullptr for a description the operators take, else what is wrong with it.
const char* attn_desc_error(const mfmg_attn_desc& d);

struct RopeFreqs {
  double f4[ROPE_MAX_PAIRS];      // quarter turns per position of each pair
  float mscale;
  int dims, interleaved;
};
RopeFreqs rope_freqs(const mfmg_attn_desc& d);

template <typename T>
struct QkRopeArgs {
  const float *x, *xd;            // rows q | k | v (backward with norms: the forward's input)
  const float *gain, *gaind;      // [2][dh] q, k gains; null: no norms
  T *y, *yd;                      // forward: out.  Backward: y, yd = the cotangent (in),
  T *dx, *dxd;                    //   dx, dxd = the input's gradient (out)
  long ldx, ldxd, ldy, ldyd, lddx, lddxd;
  float* partial;                 // backward with norms: [qk_rope_partials][4][dh]
  SeqPlan p;
  int H, K, dh, dual;
  float eps;
  RopeFreqs f;
};
template <typename T>
hipError_t qk_rope_fwd(const QkRopeArgs<T>& a, hipStream_t s);
// Writes dx (dxd) and, with norms, partial sums of the gains' gradients (q, k, and their
// tangents): qk_rope_partials rows of [4][dh] (dual: no more), of which qk_rope_sums says which `count`
// gain_param finishes.
int qk_rope_partials(long n, int H, int K, int dh);
const float* qk_rope_sums(const float* partial, long n, int H, int K, int dh, bool dual, int* count);
template <typename T>
hipError_t qk_rope_bwd(const QkRopeArgs<T>& a, hipStream_t s);
// The parameter epilogue on column sums of partial [parts][4][d] (transformer.hip).
template <typename T>
hipError_t gain_param(const float* partial, int parts, int d, long off0, long off1,
                      const ParamArgs<T>& P, float* out0, float* out1, hipStream_t s);

}  // namespace mfmg
