// Queries and keys before the attention: RMS norm of every head's row and rotation by the token's position, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * weight
//   pair i of the first rot_dim channels, turned by the angle t = position[axis(i)] * turns[i] (in full turns):
//     (a, b) -> magnitude * (a cos t - b sin t, a sin t + b cos t)
// in fp32 from bf16 rows, rounded once.  The angle is formed in 64 bits and reduced to (-1/2, 1/2] turns before it is rounded to 32:
// at position 2^20 the fastest pair's angle in 32 bits would be off by 1/16 of a radian.  Sines and cosines in 32 bits then err by less
// than 1e-6, far below the rounding of the result (2^-8 relative).
//
// Bound: HBM, every row is read and written once.  A wave takes one token (or some of its heads, where tokens are few): its lanes work
// the token's cosines and sines out once, one pair each, and all heads of the token share them; a row is D / 8 lanes wide, and a
// lane holds whole pairs in either layout (eight neighbouring channels, or four of each half), so that nothing crosses lanes but the sum of squares.
// 88920 tokens of 24 heads of 128: 190 us, 5.7 TB/s read and written; torch's copy of the same bytes takes 203, this kernel without norm and
// rotation 199 and with the rotation alone 185, so the vector ALU, which its counters show as busy all the time, does not bind.
#include <math.h>
#include <type_traits>
#include "pf_internal.h"

typedef __attribute__((ext_vector_type(4))) __bf16 rope_quad;     // four channels
typedef __attribute__((ext_vector_type(4))) float rope_f4;

constexpr int ROPE_THREADS = 256;
constexpr int ROPE_WAVES = ROPE_THREADS / 64;
// A token's heads are dealt out to several waves until there are so many, 32 per compute unit: 4680 tokens of 24 heads 12.8 us (with 16384 15.3, with
// 32768 21.0: the angles are worked out once per wave)
constexpr int ROPE_MIN_WAVES = 8192;
constexpr int ROPE_MAX_TOKENS = ((1 << 24) - 1) * ROPE_WAVES;      // a launch has fewer than 2^32 threads
constexpr int ROPE_AHEAD = 3;                                     // groups of rows in flight per wave (2: 199.6 us for 88920 tokens, 3: 190, 4: 213)

struct RopeParams {
  const __bf16 *x[2], *weight[2];                                 // queries, keys
  __bf16 *out[2];
  long long x_tok[2], x_head[2], out_tok[2], out_head[2];
  const int32_t *positions;                                       // [axes][tokens]
  int n_tokens, n_q, n_rows;                                      // query heads; heads in all
  int rows_per_wave, n_parts;                                     // a token's rows are cut into n_parts
  int rot, pairs_end0, pairs_end1, norm;
  float eps, magnitude;
  double turns[PF_ROPE_MAX_PAIRS];
};

// sum over the 16 (or 8) lanes of a row
template <int CTRL>
__device__ __forceinline__ float rope_add_lane(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float rope_row_sum(float x) {
  x = rope_add_lane<0xB1>(x);                                     // quad_perm 1 0 3 2
  x = rope_add_lane<0x4E>(x);                                     // quad_perm 2 3 0 1
  x = rope_add_lane<0x141>(x);                                    // mirror inside 8 lanes
  return LANES == 16 ? rope_add_lane<0x140>(x) : x;               // mirror inside 16 lanes
}

// PART: the channels from P.rot on are not turned (as a test at run time it costs calls that turn them all: 4680 tokens 12.8 -> 13.2 us)
template <int D, bool INTERLEAVED, bool PART>
__global__ __launch_bounds__(ROPE_THREADS) void pf_qk_norm_rope_kernel(RopeParams P) {
  constexpr int LANES = D / 8, ROWS = 64 / LANES;                 // lanes of a row, rows that a wave holds side by side
  __shared__ float2 s_turn[ROPE_WAVES][PF_ROPE_MAX_PAIRS];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int job = blockIdx.x * ROPE_WAVES + wave;
  const int token = job / P.n_parts;
  if (token >= P.n_tokens) return;
  const int row0 = (job - token * P.n_parts) * P.rows_per_wave;
  const int row1 = pf_min(row0 + P.rows_per_wave, P.n_rows);
  const int j = lane % LANES, sub = lane / LANES;

  // this lane's channels: a quad at `at_a` and one at `at_b`
  int at_a, at_b;
  const bool turned = !PART || 8 * j < P.rot;
  if (INTERLEAVED || !turned) {
    at_a = 8 * j;
    at_b = 8 * j + 4;
  } else {
    at_a = 4 * j;
    at_b = P.rot / 2 + 4 * j;
  }

  // the first rows travel while the angles are worked out
  rope_quad a[ROPE_AHEAD], b[ROPE_AHEAD];
  auto load = [&](int i, int r) __attribute__((always_inline)) {
    const int row = pf_min(r, row1 - 1);
    const bool is_k = row >= P.n_q;
    const __bf16 *x = (is_k ? P.x[1] : P.x[0]) + token * (is_k ? P.x_tok[1] : P.x_tok[0]) +
                      (is_k ? row - P.n_q : row) * (is_k ? P.x_head[1] : P.x_head[0]);
    a[i] = *(const rope_quad *)(x + at_a);
    b[i] = *(const rope_quad *)(x + at_b);
  };
#pragma unroll
  for (int i = 0; i < ROPE_AHEAD; ++i) load(i, row0 + i * ROWS + sub);

  float cs[4] = {1.0f, 1.0f, 1.0f, 1.0f}, sn[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (P.rot > 0) {
    if (lane < P.rot / 2) {
      const int axis = (lane >= P.pairs_end0) + (lane >= P.pairs_end1);
      const double t = (double)P.positions[(long long)axis * P.n_tokens + token] * P.turns[lane];
      const float f = (float)(t - rint(t));
      float si, co;
      sincospif(2.0f * f, &si, &co);
      s_turn[wave][lane] = make_float2(co * P.magnitude, si * P.magnitude);
    }
    __builtin_amdgcn_wave_barrier();                              // a wave reads what it wrote itself: LDS operations of a wave keep their order
    if (turned) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float2 v = s_turn[wave][4 * j + i];
        cs[i] = v.x;
        sn[i] = v.y;
      }
    }
  }
  rope_f4 w[2][2];
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    w[t][0] = w[t][1] = rope_f4{1.0f, 1.0f, 1.0f, 1.0f};
    if (P.weight[t]) {
      w[t][0] = __builtin_convertvector(*(const rope_quad *)(P.weight[t] + at_a), rope_f4);
      w[t][1] = __builtin_convertvector(*(const rope_quad *)(P.weight[t] + at_b), rope_f4);
    }
  }

  for (int r0 = row0; r0 < row1; r0 += ROPE_AHEAD * ROWS) {
#pragma unroll
    for (int i = 0; i < ROPE_AHEAD; ++i) {
      const int row = r0 + i * ROWS + sub;
      rope_f4 x = __builtin_convertvector(a[i], rope_f4), y = __builtin_convertvector(b[i], rope_f4);
      const bool is_k = row >= P.n_q;
      if (P.norm) {
        float sq = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sq = fmaf(x[e], x[e], fmaf(y[e], y[e], sq));
        const float inv = 1.0f / sqrtf(rope_row_sum<LANES>(sq) * (1.0f / D) + P.eps);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] *= inv * (is_k ? w[1][0][e] : w[0][0][e]);
          y[e] *= inv * (is_k ? w[1][1][e] : w[0][1][e]);
        }
      }
      rope_quad to_a, to_b;
      if (INTERLEAVED) {                                          // pairs (0, 1) (2, 3) of either quad
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          to_a[e] = (__bf16)(x[e] * cs[e / 2] - x[e + 1] * sn[e / 2]);
          to_a[e + 1] = (__bf16)(x[e] * sn[e / 2] + x[e + 1] * cs[e / 2]);
          to_b[e] = (__bf16)(y[e] * cs[2 + e / 2] - y[e + 1] * sn[2 + e / 2]);
          to_b[e + 1] = (__bf16)(y[e] * sn[2 + e / 2] + y[e + 1] * cs[2 + e / 2]);
        }
      } else {                                                    // pair: the same place of either quad
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          to_a[e] = (__bf16)(x[e] * cs[e] - y[e] * sn[e]);
          to_b[e] = (__bf16)(x[e] * sn[e] + y[e] * cs[e]);
        }
      }
      if (!turned) {                                              // an infinity beside a channel must not reach it by 0 * inf
        to_a = __builtin_convertvector(x, rope_quad);
        to_b = __builtin_convertvector(y, rope_quad);
      }
      if (row < row1) {
        __bf16 *o = (is_k ? P.out[1] : P.out[0]) + token * (is_k ? P.out_tok[1] : P.out_tok[0]) +
                    (is_k ? row - P.n_q : row) * (is_k ? P.out_head[1] : P.out_head[0]);
        *(rope_quad *)(o + at_a) = to_a;
        *(rope_quad *)(o + at_b) = to_b;
      }
    }
    const int next = r0 + ROPE_AHEAD * ROWS;
    if (next < row1) {
#pragma unroll
      for (int i = 0; i < ROPE_AHEAD; ++i) load(i, next + i * ROWS + sub);
    }
  }
}

extern "C" int pf_rope_init(pf_rope *rope, int head_dim, int rot_dim, int interleaved, int n_axes, const int32_t *axis_pairs,
                            double base, const pf_rope_scaling *scaling) {
  if (!rope) return PF_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return PF_ERR_UNSUPPORTED;
  if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 8 || (interleaved != 0 && interleaved != 1)) return PF_ERR_INVALID_ARG;
  if (n_axes < 1 || n_axes > 3 || !axis_pairs || !(base > 0.0) || !(base < 1e300)) return PF_ERR_INVALID_ARG;
  int pairs = 0;
  for (int a = 0; a < n_axes; ++a) {
    if (axis_pairs[a] < 0 || axis_pairs[a] > PF_ROPE_MAX_PAIRS) return PF_ERR_INVALID_ARG;
    pairs += axis_pairs[a];
  }
  if (pairs != rot_dim / 2) return PF_ERR_INVALID_ARG;
  if (scaling && scaling->reserved) return PF_ERR_INVALID_ARG;
  const int kind = scaling ? scaling->kind : PF_ROPE_SCALE_NONE;
  if (kind != PF_ROPE_SCALE_NONE && kind != PF_ROPE_SCALE_LINEAR && kind != PF_ROPE_SCALE_BY_WAVELENGTH) return PF_ERR_INVALID_ARG;
  const double factor = kind == PF_ROPE_SCALE_NONE ? 1.0 : scaling->factor;
  if (!(factor >= 1.0) || !(factor < 1e300)) return PF_ERR_INVALID_ARG;
  if (kind == PF_ROPE_SCALE_BY_WAVELENGTH && !(scaling->original_positions > 0.0 && scaling->original_positions < 1e300 && scaling->slow_turns >= 0.0 &&
                                               scaling->fast_turns > scaling->slow_turns && scaling->fast_turns < 1e300)) return PF_ERR_INVALID_ARG;
  const double magnitude = scaling && scaling->magnitude != 0.0 ? scaling->magnitude : 1.0;
  if (!(fabs(magnitude) < 1e30)) return PF_ERR_INVALID_ARG;
  pf_rope r = {};
  r.head_dim = head_dim;
  r.rot_dim = rot_dim;
  r.interleaved = interleaved;
  r.n_axes = n_axes;
  r.magnitude = (float)magnitude;
  int i = 0;
  for (int a = 0; a < n_axes; ++a) {
    r.axis_pairs[a] = axis_pairs[a];
    for (int m = 0; m < axis_pairs[a]; ++m, ++i) {
      double turns = pow(base, -(double)m / axis_pairs[a]) / 6.283185307179586476925;
      if (kind == PF_ROPE_SCALE_LINEAR) turns /= factor;
      if (kind == PF_ROPE_SCALE_BY_WAVELENGTH) {
        // how often the pair turns over the context that was trained on: often -> as it is, hardly -> stretched, a ramp between
        const double often = turns * scaling->original_positions;
        double keep = (often - scaling->slow_turns) / (scaling->fast_turns - scaling->slow_turns);
        keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
        turns = keep * turns + (1.0 - keep) * turns / factor;
      }
      r.turns[i] = turns;
    }
  }
  *rope = r;
  return PF_OK;
}

static int rope_rows_ok(const pf_rope_rows *t, int n_tokens, int head_dim) {
  if (t->n_heads < 0 || t->n_heads > PF_MAX_HEADS || t->reserved) return PF_ERR_INVALID_ARG;
  if (t->n_heads == 0) return t->x || t->out || t->weight ? PF_ERR_INVALID_ARG : PF_OK;
  if (n_tokens > 0 && (!t->x || !t->out)) return PF_ERR_INVALID_ARG;
  if ((((uintptr_t)t->x) | ((uintptr_t)t->out) | ((uintptr_t)t->weight)) & 15u) return PF_ERR_INVALID_ARG;
  for (const pf_chunk_layout *l : {&t->x_layout, &t->out_layout})
    if ((l->token_stride || l->head_stride) && !pf_chunk_layout_ok(l, t->n_heads, n_tokens, head_dim)) return PF_ERR_INVALID_ARG;
  return PF_OK;
}

extern "C" int pf_qk_norm_rope(const pf_rope *rope, int n_tokens, const int32_t *positions, const pf_rope_rows *q, const pf_rope_rows *k,
                               float eps, void *stream) {
  if (!rope || !q || !k || n_tokens < 0 || n_tokens > ROPE_MAX_TOKENS) return PF_ERR_INVALID_ARG;
  const int D = rope->head_dim;
  if (D != 64 && D != 128) return PF_ERR_UNSUPPORTED;
  if (rope->rot_dim < 0 || rope->rot_dim > D || rope->rot_dim % 8 || rope->n_axes < 1 || rope->n_axes > 3) return PF_ERR_INVALID_ARG;
  int pairs = 0;
  for (int a = 0; a < rope->n_axes; ++a) {
    if (rope->axis_pairs[a] < 0 || rope->axis_pairs[a] > PF_ROPE_MAX_PAIRS) return PF_ERR_INVALID_ARG;
    pairs += rope->axis_pairs[a];
  }
  if (pairs != rope->rot_dim / 2) return PF_ERR_INVALID_ARG;
  if (!(eps >= 0.0f) || !(eps < 1.0e30f)) return PF_ERR_INVALID_ARG;
  if (eps == 0.0f && (q->weight || k->weight)) return PF_ERR_INVALID_ARG;   // a weight belongs to the norm
  if (q->n_heads + k->n_heads < 1) return PF_ERR_INVALID_ARG;
  for (const pf_rope_rows *t : {q, k}) {
    const int rc = rope_rows_ok(t, n_tokens, D);
    if (rc != PF_OK) return rc;
  }
  if (rope->rot_dim > 0 && ((n_tokens > 0 && !positions) || ((uintptr_t)positions & 3u))) return PF_ERR_INVALID_ARG;
  if (n_tokens == 0) return PF_OK;
  RopeParams P = {};
  const pf_rope_rows *t[2] = {q, k};
  for (int i = 0; i < 2; ++i) {
    P.x[i] = (const __bf16 *)t[i]->x;
    P.out[i] = (__bf16 *)t[i]->out;
    P.weight[i] = (const __bf16 *)t[i]->weight;
    const bool xs = t[i]->x_layout.token_stride != 0, os = t[i]->out_layout.token_stride != 0;
    P.x_tok[i] = xs ? t[i]->x_layout.token_stride : D;
    P.x_head[i] = xs ? t[i]->x_layout.head_stride : (long long)n_tokens * D;
    P.out_tok[i] = os ? t[i]->out_layout.token_stride : D;
    P.out_head[i] = os ? t[i]->out_layout.head_stride : (long long)n_tokens * D;
  }
  P.positions = positions;
  P.n_tokens = n_tokens;
  P.n_q = q->n_heads;
  P.n_rows = q->n_heads + k->n_heads;
  // A wave takes a whole token's rows where tokens are many (its cosines and sines then serve all of them), and where waves would be
  // too few to hide each other's memory latency, as few rows as it holds side by side
  const int side = 64 * 8 / D, groups = pf_ceil_div(P.n_rows, side);
  const int parts = (int)(ROPE_MIN_WAVES / n_tokens < groups ? ROPE_MIN_WAVES / n_tokens : groups);
  P.rows_per_wave = pf_ceil_div(groups, parts < 1 ? 1 : parts) * side;
  P.n_parts = pf_ceil_div(P.n_rows, P.rows_per_wave);
  P.rot = rope->rot_dim;
  P.pairs_end0 = rope->axis_pairs[0];
  P.pairs_end1 = rope->n_axes > 1 ? rope->axis_pairs[0] + rope->axis_pairs[1] : PF_ROPE_MAX_PAIRS;
  if (rope->n_axes == 1) P.pairs_end0 = PF_ROPE_MAX_PAIRS;
  P.norm = eps > 0.0f;
  P.eps = eps;
  P.magnitude = rope->magnitude;
  for (int i = 0; i < PF_ROPE_MAX_PAIRS; ++i) P.turns[i] = i < pairs ? rope->turns[i] : 0.0;
  const long long jobs = (long long)n_tokens * P.n_parts;
  const dim3 grid((unsigned)((jobs + ROPE_WAVES - 1) / ROPE_WAVES));
  hipStream_t st = (hipStream_t)stream;
  auto launch = [&](auto part) {
    constexpr bool PART = decltype(part)::value;
    if (D == 128 && rope->interleaved) hipLaunchKernelGGL((pf_qk_norm_rope_kernel<128, true, PART>), grid, dim3(ROPE_THREADS), 0, st, P);
    else if (D == 128) hipLaunchKernelGGL((pf_qk_norm_rope_kernel<128, false, PART>), grid, dim3(ROPE_THREADS), 0, st, P);
    else if (rope->interleaved) hipLaunchKernelGGL((pf_qk_norm_rope_kernel<64, true, PART>), grid, dim3(ROPE_THREADS), 0, st, P);
    else hipLaunchKernelGGL((pf_qk_norm_rope_kernel<64, false, PART>), grid, dim3(ROPE_THREADS), 0, st, P);
  };
  if (rope->rot_dim < D) launch(std::true_type());
  else launch(std::false_type());
  PF_HIP_CHECK(hipGetLastError());
  return PF_OK;
}
