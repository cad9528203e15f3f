// Attention of packed sequences: whole prompts, causal by blocks, with grouped heads, alone or behind a prefix whose keys and values all
// sequences share (and that are read once for all of them).
//
//   out[i, h] = sum_j softmax_j(scale * q[i, h] . k[j, h / group]) v[j, h / group]
// over the prefix's keys and the keys j of i's own sequence with j / block <= p / block, p = i's place among those keys (the last query
// stands at the last key); a query that sees no key gets zeros.
//
// The rows of a key head are the queries of its group: row r of a sequence is query r / group of head kv_head * group + r % group, so that
// a group reads its keys and values once.  A line of rows is one sequence's; its keys are the prefix's tiles and then its own.  Sequences
// of few rows (single tokens) would each read the prefix for a tile of which they fill little: in front of the prefix they are stacked,
// neighbours in one line, and each has its own keys as another line.  A work item is a tile of rows against a run of key tiles of its
// line: the host cuts the work into items and orders them (pf_packed_plan), heaviest first.  Rows whose keys are cut into several items
// park unnormalised partial results (O, m, l) in fp32, one plane per item, and they are joined plane by plane in a fixed order: by a second
// kernel, or, where a head has a few rows only, by the head's last workgroup to finish (no spinning).  Planes hold the rows that park and no
// others: they are numbered, head by head, and say themselves which row of the result they are.
//
// Three kinds of items.  Full: 128 rows, four waves, two workgroups per compute unit (four at head_dim 64) that fill each other's gaps.  Wide
// (pf_packed_wide.h): 256 rows, eight waves that alternate between matrix and vector work, one workgroup per compute unit; a whole batch is
// laid out with one or the other, whichever the planner finds faster (one head_dim-128 prompt of 16 heads: 1200 tokens 24 us either way,
// 4800 tokens 109 full and 101 wide, 9600 tokens 340 and 319).  Thin: at most 32 rows, among the full ones.
// Bound: prompts by the matrix pipe and the power it may draw (14040 tokens of 12 heads 1130 to 1210 TFLOP/s, 666 to 712 us from card to card,
// where a plain product of 8192^3 reached 1214; head_dim 64 by the vector ALU too: 910 to 966), single tokens by HBM (64 answers behind 16384
// tokens: 4.6 TB/s, a plain copy 4.9), short launches by what an item costs whatever its length: some 3 us to its first tile and 1.5 for its results.
//
// Scores, softmax and value products as in the ragged-cache kernels: S^T = K Q^T and O^T += V^T P^T on 32x32x16 bf16 MFMAs with fp32
// accumulation, one query row per lane; weights are rounded to bf16 for the second product (2^-8 relative at most each, the sum is
// taken in fp32 before that rounding).
#include <math.h>
#include <string.h>
#include <algorithm>
#include <functional>
#include <new>
#include <queue>
#include <vector>
#include "pf_packed_steps.h"
#ifndef PF_STRICT_FENCES
#define PF_STRICT_FENCES 0   // 1: release and acquire fences around the arrival counters (the memory model's own form)
#endif

// ---- plan ------------------------------------------------------------------------------------------------------------

struct PackedItem {
  int32_t q_base;      // first token of the line of rows (queries of one sequence, or of all of them in front of the prefix)
  int32_t row0;        // first row of the tile in that line
  int32_t n_rows;      // rows of the whole line
  int32_t k_base;      // token of the line's first key
  int32_t n_keys;      // keys of the line behind the prefix
  int32_t kt0, kt1;    // key tiles of this item: the prefix's (if the line has it), then the line's own
  int32_t head;        // key head | the line has the prefix << 12 | (plane + 1) << 13 (0: unsplit) | further planes without an item << 22 | thin << 31
  int32_t park;        // row r of the line is the key head's parked row park + r (of an item with a plane)
};
constexpr int PACKED_MAX_PLANES = 256;
constexpr int PACKED_JOIN_BATCHES = PACKED_MAX_PLANES / 64;
constexpr int PACKED_FEW_PLANES = 4;                              // joined by groups of lanes (118 and 50 us where a wave for every row takes 126 and 55)
constexpr int PACKED_PREFIX_BIT = 12;
PF_HD int packed_head(const PackedItem &it) { return it.head & 0xfff; }
PF_HD bool packed_has_prefix(const PackedItem &it) { return (it.head >> PACKED_PREFIX_BIT) & 1; }
PF_HD int packed_plane(const PackedItem &it) { return ((it.head >> 13) & 0x1ff) - 1; }
PF_HD bool packed_is_thin(const PackedItem &it) { return it.head < 0; }
PF_HD int packed_missing(const PackedItem &it) { return (it.head >> 22) & 0x1ff; }

// In front of the items: which plan this is.  Every workgroup looks it up with its item: a buffer that has been planned in anew, or not yet, by
// the time a call or a replay comes to it would lead outside the call's tensors.  A prompt of 14040 tokens 690 -> 693 us, 13 questions behind a
// prefix of 5003 tokens 28.9 -> 29.3.
struct __attribute__((aligned(32))) PackedHead {
  uint64_t planned_for;
};

// Items reach the device as kernel arguments: the call neither allocates nor waits, and can be captured.
constexpr int PACKED_UPLOAD = 108;                                // kernel arguments end at 4096 bytes
struct PackedUpload {
  PackedItem item[PACKED_UPLOAD];
};
__global__ void pf_packed_upload_kernel(PackedUpload U, int n, PackedItem *to, int32_t *arrivals, int n_arrivals, PackedHead *head, uint64_t planned_for) {
  const int i = threadIdx.x;
  if (i == 0) head->planned_for = planned_for;
  if (i < n) to[i] = U.item[i];
  for (int j = i; j < n_arrivals; j += blockDim.x) arrivals[j] = 0;
}

constexpr int PACKED_WAVES = 4;
constexpr int PACKED_ROWS = 32 * PACKED_WAVES;                    // rows of a full item
constexpr int PACKED_WIDE_ROWS = 256;                             // ... and of a wide one (pf_packed_wide.h)
// Rows that a head may have for its last workgroup to join them.  It saves the host the second launch (8 tokens behind 2048: 12.0 us a call, 14.9
// with it) and costs the GPU the last arrival and round trips to memory one after the other: 12 heads behind 4096 keys, replayed from a graph, take
// 10.7, 11.9, 15.4 and 31.6 us for 1, 8, 16 and 32 rows, with a second launch 9.6, 10.7, 13.8 and 17.3.
constexpr int PACKED_ARRIVE_ROWS = 8;
// Lines of at most so many rows are thin items: 16 sequences of 8 to 32 rows against 2000 keys of 8 heads 24 to 25 us, as full items 28 to 29;
// head_dim 64: 15 and 18 (of 2 rows: 19 and 18).
constexpr int PACKED_THIN_ROWS = 32;

struct PackedParams {
  const __bf16 *q, *k, *v, *k_prefix, *v_prefix;
  __bf16 *out;
  const PackedItem *items;
  float *part_o;                                                  // [planes][part_rows][D]
  float2 *part_ml;                                                // [planes][part_rows]: reference maximum, sum of weights
  int32_t *part_row;                                              // [part_rows]: token x heads + head
  long long q_tok, q_head, out_tok, out_head, kv_tok, kv_head, pre_tok, pre_head;    // element strides
  int n_rows, n_heads, group, block;                              // n_rows: tokens x heads
  int32_t *arrivals;                                              // [key heads] workgroups of the head that are done; null: a second kernel joins
  int items_per_head;
  int head_rows, part_rows;                                       // parked rows of a key head, of all
  int planes, prefix_tokens, prefix_tiles;
  unsigned group_mul, group_shift;                                // n / group = (n * group_mul) >> 32 >> group_shift
  float scale_log2;
  unsigned long long planned_for;                                 // the plan that this launch is under
};

template <class T>
__device__ __forceinline__ T *packed_global(T *p) {
  return (T *)(__attribute__((address_space(1))) T *)(unsigned long long)p;
}
// The parameters, read again from the kernel-argument segment at every call (a few scalar loads): held in registers through the loop over the
// key tiles they would crowd out its own scalars, which the copies need as such.
__device__ __forceinline__ PackedParams packed_params() {
  static_assert(sizeof(PackedParams) % 8 == 0, "parameters are copied as 8-byte words");
  struct Words {
    unsigned long long w[sizeof(PackedParams) / 8];
  };
  int zero = 0;                                                   // hides from the compiler that every call reads the same words
  asm volatile("" : "+s"(zero));
  const __attribute__((address_space(4))) unsigned long long *arg =
      (const __attribute__((address_space(4))) unsigned long long *)__builtin_amdgcn_kernarg_segment_ptr() + __builtin_amdgcn_readfirstlane(zero);
  Words words;
#pragma unroll
  for (int i = 0; i < (int)(sizeof(PackedParams) / 8); ++i) words.w[i] = arg[i];
  PackedParams P = __builtin_bit_cast(PackedParams, words);
  P.q = packed_global(P.q), P.k = packed_global(P.k), P.v = packed_global(P.v), P.k_prefix = packed_global(P.k_prefix);
  P.v_prefix = packed_global(P.v_prefix), P.out = packed_global(P.out), P.items = packed_global(P.items);
  P.part_o = packed_global(P.part_o), P.part_ml = packed_global(P.part_ml), P.part_row = packed_global(P.part_row), P.arrivals = packed_global(P.arrivals);
  return P;
}

// The plan was written before this launch and is constant during it: scalar loads, so that what follows from an item is scalar too.
typedef const __attribute__((address_space(4))) unsigned *packed_words_t;
__device__ __forceinline__ bool packed_is_there(const PackedParams &P) {
  return *(const __attribute__((address_space(4))) uint64_t *)((const PackedHead *)P.items - 1) == P.planned_for;
}
// This workgroup's item; is it one of the call's plan?
__device__ __forceinline__ PackedItem packed_item(bool &there) {
  struct Words {
    unsigned w[sizeof(PackedItem) / 4];
  } words;
  const PackedParams P = packed_params();
  const packed_words_t from = (packed_words_t)(P.items + blockIdx.x);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(PackedItem) / 4); ++i) words.w[i] = from[i];
  there = packed_is_there(P);
  PackedItem it = __builtin_bit_cast(PackedItem, words);
  asm volatile("" : "+v"(it.park));                               // through the loop over the key tiles it would be one scalar too many
  return it;
}
// It is not: the launch says so in every row of the result, and touches nothing else.
template <int D>
__device__ __forceinline__ void packed_no_plan(int tid, int threads) {
  const PackedParams P = packed_params();
  constexpr int LANES = D / 8;
  for (int id = (int)blockIdx.x * (threads / LANES) + tid / LANES; id < P.n_rows; id += (int)gridDim.x * (threads / LANES))
    *(u32x4 *)(P.out + id / P.n_heads * P.out_tok + id % P.n_heads * P.out_head + tid % LANES * 8) = u32x4{0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
}

template <int D>
struct PackedTile {
  static constexpr int ROW_BYTES = D * 2;
  static constexpr int TENSOR_BYTES = PF_BK * ROW_BYTES;
  static constexpr int STAGE_BYTES = 2 * TENSOR_BYTES;
  static constexpr int CHUNKS = ROW_BYTES / 16;                   // 16-byte chunks of a row
  static constexpr int COPY_ROWS = 1024 / ROW_BYTES;              // rows of one copy instruction
  static constexpr int NKS = D / 16, NDB = D / 32;
  static constexpr int LD = D + 4;                                // row stride of the staged result
  // 16-byte chunk c of row r sits at c ^ swz(r): the reads of K (32 rows x one chunk) and of V^T (64 bytes of four rows) then cover all banks
  static __device__ constexpr int swz_k(int r) { return D == 128 ? r & 15 : (r >> 1) & 7; }
  static __device__ constexpr int swz_v(int r) { return D == 128 ? (r & 3) << 2 : ((r >> 1) & 1) << 2; }
};

// n / group by multiplication (n < 2^31; the factors are worked out in pf_packed_attn_fwd): divisions by a number known at run time are some 25 instructions each, and there
// are several for every row of a tile
__device__ __forceinline__ int packed_div_group(const PackedParams &P, int n) {
  return P.group == 1 ? n : (int)(__umulhi((unsigned)n, P.group_mul) >> P.group_shift);
}

// keys behind the prefix that row r of the item's line may see
__device__ __forceinline__ int packed_limit(const PackedParams &P, const PackedItem &it, int r) {
  if (P.block == 0) return it.n_keys;
  const int place = it.n_keys - packed_div_group(P, it.n_rows) + packed_div_group(P, r);
  if (place < 0) return 0;
  if (P.block == 1) return place + 1;
  // the last key of the row's block; the block's number and its end stay below 2^31 for any block size (a sequence has at most 2^30 keys)
  const unsigned number = (unsigned)place / (unsigned)P.block;
  return (int)min((unsigned)it.n_keys, number * (unsigned)P.block + (unsigned)P.block);
}

// Where the keys of an item's tiles sit: one key head of the prefix, and of the line's own keys behind it.
struct PackedKeys {
  const __bf16 *k, *v, *k_pre, *v_pre;
  int pre;             // tiles of the prefix
};
__device__ __forceinline__ PackedKeys packed_keys(const PackedParams &P, const PackedItem &it) {
  PackedKeys K;
  const int h = packed_head(it);
  const long long own = (long long)it.k_base * P.kv_tok + h * P.kv_head;
  K.pre = packed_has_prefix(it) ? P.prefix_tiles : 0;
  K.k = P.k + own;
  K.v = P.v + own;
  K.k_pre = P.k_prefix + h * P.pre_head;
  K.v_pre = P.v_prefix + h * P.pre_head;
  return K;
}
// Send the copies of ROWS rows of key tile kt, from row r0 on (a multiple of 8), of K (V) into `to`, that row's place in the tile.
template <int D, bool IS_V, int ROWS>
__device__ __forceinline__ void packed_copy(const PackedParams &P, const PackedItem &it, const PackedKeys &K, int kt, int r0, char *to, int lane) {
  typedef PackedTile<D> C;
  typedef __attribute__((address_space(3))) void *lptr_t;
  const bool in_prefix = kt < K.pre;
  const long long tok = in_prefix ? P.pre_tok : P.kv_tok;
  const int key0 = (in_prefix ? kt : kt - K.pre) * PF_BK + r0;
  const __bf16 *b = (in_prefix ? (IS_V ? K.v_pre : K.k_pre) : (IS_V ? K.v : K.k)) + key0 * tok;
  const unsigned rb = (unsigned)(tok * 2);                        // bytes between key rows (below 2^25: checked on the host)
  const int last = (in_prefix ? P.prefix_tokens : it.n_keys) - 1 - key0;
  const int rr = lane / C::CHUNKS, p = lane % C::CHUNKS;
  const unsigned low = (unsigned)((p ^ (IS_V ? C::swz_v(rr) : C::swz_k(rr) ^ C::swz_k(r0 & 15))) << 4);
  const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)b, 0, -1, 0x00020000u);
  if (__builtin_expect(last >= ROWS - 1, 1)) {
    const unsigned at = (unsigned)rr * rb;
    static_for<0, ROWS / C::COPY_ROWS>([&](auto gi) {
      constexpr int G = decltype(gi)::value;
      constexpr unsigned flip = (unsigned)((IS_V ? C::swz_v(G * C::COPY_ROWS) : C::swz_k(G * C::COPY_ROWS)) << 4);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)(to + G * 1024), 16, at + (low ^ flip), G * C::COPY_ROWS * rb, 0, 0);
    });
  } else {                                                        // rows past the end repeat the last key (or, past a whole step, the one before)
    int lane_l = lane;
    asm volatile("" : "+v"(lane_l));                              // rare: its lane offsets are not held in registers through the loop
    const unsigned low_l = (unsigned)((lane_l % C::CHUNKS ^ (IS_V ? C::swz_v(lane_l / C::CHUNKS) : C::swz_k(lane_l / C::CHUNKS) ^ C::swz_k(r0 & 15))) << 4);
    const __amdgpu_buffer_rsrc_t e = __builtin_amdgcn_make_buffer_rsrc((void *)(b + (long long)pf_min(last, 0) * tok), 0, -1, 0x00020000u);
    static_for<0, ROWS / C::COPY_ROWS>([&](auto gi) {
      constexpr int G = decltype(gi)::value;
      constexpr unsigned flip = (unsigned)((IS_V ? C::swz_v(G * C::COPY_ROWS) : C::swz_k(G * C::COPY_ROWS)) << 4);
      const unsigned at = (unsigned)pf_min(G * C::COPY_ROWS + lane_l / C::CHUNKS, pf_max(last, 0)) * rb;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(e, (lptr_t)(to + G * 1024), 16, at + (low_l ^ flip), 0, 0, 0);
    });
  }
}

// One row's softmax state.  The reference maximum starts below every score; its multiple is kept finite, so that a masked key's weight against
// it is 0 and not NaN.  Where it starts says whether the row sees a key of the item at all: one that does and has no weight in the end saw
// scores of minus infinity only, of which alone there is no softmax (its maximum becomes minus infinity then, see packed_to).
struct PackedRow {
  float m, l, mc;
};
constexpr float PACKED_SEES = -3.0e38f, PACKED_SEES_NONE = -3.1e38f;
__device__ __forceinline__ float packed_mc(float m, float c) { return fmaxf(m * c, -3.0e38f); }
// limit: keys behind the prefix that the row sees; pre: the prefix's tiles
__device__ __forceinline__ PackedRow packed_row(const PackedItem &it, int pre, int limit, float c) {
  const bool sees = it.kt0 < pf_min(it.kt1, pre) || (it.kt1 > pre && limit > (pf_max(it.kt0, pre) - pre) * PF_BK);
  const float m = sees ? PACKED_SEES : PACKED_SEES_NONE;
  return {m, 0.0f, packed_mc(m, c)};
}

// Scores of NKB blocks of 32 keys (accumulators of K Q^T: register i of block kb is key 32 kb + 8 (i / 4) + 4 g + i % 4) -> weights in bf16,
// the row's state and O moved on.  first: an item's first tile, whose rows have no reference yet.
template <int D, int NKB>
__device__ __forceinline__ void packed_softmax(f32x16 (&s)[NKB], bf16x8 (&pf)[2 * NKB], f32x16 (&o)[D / 32], PackedRow &R, float c, bool first) {
  float ts[2];
  auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; i += 2) {
        const float e0 = fast_exp2(fmaf(s[kb][i], c, -R.mc)), e1 = fast_exp2(fmaf(s[kb][i + 1], c, -R.mc));
        ts[0] = kb + i == 0 ? e0 : ts[0] + e0;
        ts[1] = kb + i == 0 ? e1 : ts[1] + e1;
        pf[kb * 2 + (i >> 3)][i & 7] = (__bf16)e0;
        pf[kb * 2 + (i >> 3)][(i & 7) + 1] = (__bf16)e1;
      }
  };
  if (__builtin_expect(!first, 1)) {
    weights();
  } else {                                                        // as if they had been formed against no reference at all
    ts[0] = ts[1] = INFINITY;
#pragma unroll
    for (int i = 0; i < 2 * NKB; ++i) pf[i] = bf16x8{};
  }
#pragma unroll
  for (int i = 0; i < 2 * NKB; ++i) asm volatile("" : "+v"(pf[i]));   // rounded here: sunk past the branch, all weights would stay in registers
  if (__builtin_expect(tile_sum_too_large(ts[0] + ts[1]), 0)) {
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb][i]);
    // only rows that need it move, so that no row's bits depend on what its neighbours hold
    const float over = partner_max(ts[0] + ts[1] <= PACKED_MAX_TILE_SUM ? 0.0f : 1.0f);
    const float m_new = over > 0.0f ? fmaxf(R.m, partner_max(mx)) : R.m;
    const float alpha = fast_exp2((R.m - m_new) * c);
    R.m = m_new;
    R.mc = packed_mc(m_new, c);
    R.l *= alpha;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
    weights();
  }
  R.l += ts[0] + ts[1];
}
// keys of the tile (or step) at t0 that a row with this limit does not see
template <int NKB>
__device__ __forceinline__ void packed_mask(f32x16 (&s)[NKB], int valid, int g) {
  asm volatile("" : "+v"(g));                                     // rare: per-lane constants are not held in registers through the loop
#pragma unroll
  for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (kb * 32 + 8 * (i >> 2) + 4 * g + (i & 3) >= valid) s[kb][i] = -INFINITY;
}
// O^T += V^T P^T over NS16 groups of 16 keys: fragment s16 * NDB + db = 16 keys, channel block db (two transpose reads each), four ahead
template <int D, int NS16>
__device__ __forceinline__ void packed_pv(f32x16 (&o)[D / 32], const bf16x8 (&pf)[NS16], unsigned av) {
  typedef PackedTile<D> C;
  constexpr int N = NS16 * C::NDB, AHEAD = N < 4 ? N : 4;
  u32x2 vl[N], vh[N];
  auto vread = [&](auto i) {
    constexpr int I = decltype(i)::value, OFF = (I / C::NDB) * 16 * C::ROW_BYTES;
    const unsigned a = av ^ (unsigned)((I % C::NDB) << 6);
    read_vt<OFF>(vl[I], a);
    read_vt<OFF + 8 * C::ROW_BYTES>(vh[I], a);
  };
  static_for<0, AHEAD>([&](auto i) { vread(i); });
  static_for<0, N>([&](auto i) {
    constexpr int I = decltype(i)::value;
    wait_lds<2 * (I + AHEAD - 1 < N - 1 ? AHEAD - 1 : N - 1 - I)>();
    const u32x4 a4 = __builtin_shufflevector(vl[I], vh[I], 0, 1, 2, 3);
    o[I % C::NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a4), pf[I / C::NDB], o[I % C::NDB], 0, 0, 0);
    if constexpr (I + AHEAD < N) vread(IntC<I + AHEAD>());
    __builtin_amdgcn_sched_barrier(0);
  });
}
// S^T = K Q^T: fragment NKB * ks + kb = key block kb, k-step ks, four ahead
template <int D, int NKB>
__device__ __forceinline__ void packed_qk(f32x16 (&s)[NKB], const bf16x8 (&qf)[D / 16], unsigned ak) {
  typedef PackedTile<D> C;
  constexpr int N = NKB * C::NKS;
  u32x4 kf[N];
  auto kread = [&](auto i) {
    constexpr int I = decltype(i)::value;
    read_k<(I % NKB) * 32 * C::ROW_BYTES>(kf[I], ak ^ (unsigned)((I / NKB) << 5));
  };
  static_for<0, 4>([&](auto i) { kread(i); });
  static_for<0, N>([&](auto i) {
    constexpr int I = decltype(i)::value, KB = I % NKB, KSTEP = I / NKB;
    wait_lds<(I + 3 < N - 1 ? 3 : N - 1 - I)>();
    const f32x16 zero = {};
    s[KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[I]), qf[KSTEP], KSTEP == 0 ? zero : s[KB], 0, 0, 0);
    if constexpr (I + 4 < N) kread(IntC<I + 4>());
    __builtin_amdgcn_sched_barrier(0);
  });
}
// LDS addresses of this lane's fragments: K row l32, chunk (2 ks + g) ^ swz -> ak ^ (ks << 5); V^T rows 4 g + (lane & 15) / 4 (+ 8, 16 ..), channel
// block db -> av ^ (db << 6)
template <int D>
__device__ __forceinline__ void packed_lds(const char *k, const char *v, int lane, unsigned &ak, unsigned &av) {
  typedef PackedTile<D> C;
  const int l32 = lane & 31, g = lane >> 5, rowv = 4 * g + ((lane & 15) >> 2), c0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
  ak = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char *)k + l32 * C::ROW_BYTES + ((g ^ C::swz_k(l32)) << 4);
  av = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char *)v + rowv * C::ROW_BYTES + ((c0 ^ C::swz_v(rowv)) << 4) + 8 * (lane & 1);
}
// Q^T fragments of a row: lane (l32, g) holds channels 16 ks + 8 g .. + 7
template <int D>
__device__ __forceinline__ void packed_load_q(const PackedParams &P, const PackedItem &it, int row, int g, bf16x8 (&qf)[D / 16]) {
  const int t = packed_div_group(P, row), h = packed_head(it) * P.group + row - t * P.group;
  const __bf16 *q = P.q + (it.q_base + t) * P.q_tok + h * P.q_head + 8 * g;
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) qf[ks] = *(const bf16x8 *)(q + ks * 16);
}
// The same of a wave's 32 rows, through 32 rows of LDS that are its own: a load of Q^T fragments from memory touches 32 rows (64 cycles for 1 KB), a
// copy of whole rows 4 or 8.  First the copies, ...
template <int D>
__device__ __forceinline__ void packed_send_q(const PackedParams &P, const PackedItem &it, int wrow0, char *stage, int lane) {
  typedef PackedTile<D> C;
  typedef __attribute__((address_space(3))) void *lptr_t;
  typedef const __attribute__((address_space(1))) void *gptr_t;
  asm volatile("" : "+v"(lane));
  const int row = pf_min(wrow0 + (lane & 31), it.n_rows - 1), t = packed_div_group(P, row), h = packed_head(it) * P.group + row - t * P.group;
  const unsigned long long q = (unsigned long long)(P.q + (it.q_base + t) * P.q_tok + h * P.q_head);
  const int r0 = lane / C::CHUNKS, p = lane % C::CHUNKS;
  static_for<0, 32 / C::COPY_ROWS>([&](auto gi) {
    constexpr int G = decltype(gi)::value;
    const int r = G * C::COPY_ROWS + r0;
    const unsigned lo = __builtin_amdgcn_ds_bpermute(r * 4, (int)(unsigned)q), hi = __builtin_amdgcn_ds_bpermute(r * 4, (int)(unsigned)(q >> 32));
    __builtin_amdgcn_global_load_lds((gptr_t)(((unsigned long long)hi << 32 | lo) + ((p ^ C::swz_k(r)) << 4)), (lptr_t)(stage + G * 1024), 16, 0, 0);
  });
}
// ... and once they have landed, the fragments.
template <int D>
__device__ __forceinline__ void packed_read_q(const char *stage, int lane, bf16x8 (&qf)[D / 16]) {
  typedef PackedTile<D> C;
  unsigned aq, unused;
  packed_lds<D>(stage, stage, lane, aq, unused);
  u32x4 x[C::NKS];
  static_for<0, C::NKS>([&](auto i) { read_k<0>(x[decltype(i)::value], aq ^ (unsigned)(decltype(i)::value << 5)); });
  wait_lds<0>();
#pragma unroll
  for (int ks = 0; ks < C::NKS; ++ks) {
    asm volatile("" : "+v"(x[ks]));
    qf[ks] = __builtin_bit_cast(bf16x8, x[ks]);
  }
}
// Partial results that the head's last workgroup joins cross workgroups on different dies, each with an L2 of its own: they are written and read
// at device scope, 8 bytes at a time, past the L2; the wait for the stores before the arrival is all that stands between.  With the memory model's
// own fences (PF_STRICT_FENCES), which write back and drop whole L2s, one row of 12 heads behind 4096 keys takes 13.9 us and not 10.6.
__device__ __forceinline__ void packed_st8(void *p, float a, float b) {
  __hip_atomic_store((unsigned long long *)p, (unsigned long long)__float_as_uint(a) | (unsigned long long)__float_as_uint(b) << 32, __ATOMIC_RELAXED,
                     __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 packed_ld8(const void *p) {
  const unsigned long long x = __hip_atomic_load((const unsigned long long *)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)x), __uint_as_float((unsigned)(x >> 32)));
}

// Where a row of an item goes: the result, or a plane's share of it.
template <int D>
struct PackedTo {
  __bf16 *out;
  float *part;         // null: the result
  float inv;
  bool past_l2;
};
__device__ __forceinline__ float packed_inverse(float sum, bool lost) { return sum > 0.0f ? 1.0f / sum : lost ? __builtin_nanf("") : sum; }   // (a sum that is NaN stays NaN)
// note: this lane also notes the row's maximum and sum, and with plane 0, of which every parked row has one item, which row of the result it is
template <int D>
__device__ __forceinline__ PackedTo<D> packed_to(const PackedParams &P, const PackedItem &it, int row, float2 ml, bool note) {
  const int t = packed_div_group(P, row), h = packed_head(it) * P.group + row - t * P.group, plane = packed_plane(it);
  PackedTo<D> to = {nullptr, nullptr, 1.0f, P.arrivals != nullptr};
  if (ml.y == 0.0f && ml.x == PACKED_SEES) ml.x = -INFINITY;
  if (plane >= 0) {
    const int id = packed_head(it) * P.head_rows + it.park + row;
    auto put_ml = [&](int p, float2 x) __attribute__((always_inline)) {
      float2 *at = P.part_ml + (long long)p * P.part_rows + id;
      if (to.past_l2) packed_st8(at, x.x, x.y);
      else *at = x;
    };
    to.part = P.part_o + ((long long)plane * P.part_rows + id) * D;
    if (note) {
      put_ml(plane, ml);
      for (int i = 1; i <= packed_missing(it); ++i) put_ml(plane + i, make_float2(PACKED_SEES_NONE, 0.0f));
      if (plane == 0) __hip_atomic_store(P.part_row + id, (it.q_base + t) * P.n_heads + h, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  } else {
    to.out = P.out + (it.q_base + t) * P.out_tok + h * P.out_head;
    to.inv = packed_inverse(ml.y, ml.x == -INFINITY);
  }
  return to;
}
// eight channels from d0 on
template <int D>
__device__ __forceinline__ void packed_put(const PackedTo<D> &to, int d0, const f32x4 &a, const f32x4 &b) {
  if (to.part) {
    if (to.past_l2) {
      packed_st8(to.part + d0, a[0], a[1]);
      packed_st8(to.part + d0 + 2, a[2], a[3]);
      packed_st8(to.part + d0 + 4, b[0], b[1]);
      packed_st8(to.part + d0 + 6, b[2], b[3]);
    } else {
      *(f32x4 *)(to.part + d0) = a;
      *(f32x4 *)(to.part + d0 + 4) = b;
    }
    return;
  }
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = (__bf16)(a[i] * to.inv), w[i + 4] = (__bf16)(b[i] * to.inv);
  *(bf16x8 *)(to.out + d0) = w;
}
// The workgroup is done with its item.  Where there is no second kernel, the last one of its head joins the planes of the head's rows (see
// pf_packed_join_few_kernel): D / 8 lanes take a row, four planes in flight.  Bound: the round trips to memory, one per four planes.
template <int D>
__device__ __forceinline__ void packed_arrive(const PackedItem &it, int32_t *s_last, int tid) {
  const PackedParams P = packed_params();
  if (P.arrivals == nullptr) return;
  __builtin_amdgcn_s_waitcnt(0);                                  // this wave's partial stores have completed
#if PF_STRICT_FENCES
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "agent");
#endif
  __syncthreads();
  const int head = packed_head(it);
  if (tid == 0) {
#if PF_STRICT_FENCES
    const int before = __hip_atomic_fetch_add(&P.arrivals[head], 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT);
#else
    const int before = __hip_atomic_fetch_add(&P.arrivals[head], 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#endif
    *s_last = before == P.items_per_head - 1;
    if (*s_last) __hip_atomic_store(&P.arrivals[head], 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);   // ready for the next launch of the plan
  }
  __syncthreads();
  if (!*s_last) return;
#if PF_STRICT_FENCES
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "agent");
#endif
  constexpr int LANES = D / 8, AHEAD = 4;
  const int d0 = tid % LANES * 8;
  for (int r = tid / LANES; r < P.head_rows; r += PACKED_WAVES * 64 / LANES) {
    const int id = head * P.head_rows + r, row = __hip_atomic_load(P.part_row + id, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    float top = PACKED_SEES_NONE, sum = 0.0f, acc[8] = {};
    bool lost = false;
    for (int p0 = 0; p0 < P.planes; p0 += AHEAD) {
      float2 ml[AHEAD], x[AHEAD][4];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {                           // (the last plane again once they run out)
        const long long at = (long long)pf_min(p0 + i, P.planes - 1) * P.part_rows + id;
        ml[i] = packed_ld8(P.part_ml + at);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[i][e] = packed_ld8(P.part_o + at * D + d0 + 2 * e);
      }
      float new_top = top;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) new_top = fmaxf(new_top, ml[i].x), lost |= ml[i].x == -INFINITY;
      const float keep = fast_exp2((top - new_top) * P.scale_log2);
      top = new_top;
      sum *= keep;
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] *= keep;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if (p0 + i >= P.planes || ml[i].y == 0.0f) continue;      // a plane that saw no key (or has no item) counts nothing
        const float w = fast_exp2((ml[i].x - top) * P.scale_log2);
        sum += w * ml[i].y;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[2 * e] += w * x[i][e].x, acc[2 * e + 1] += w * x[i][e].y;
      }
    }
    const float inv = packed_inverse(sum, lost);
    bf16x8 w;
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = (__bf16)(acc[e] * inv);
    *(bf16x8 *)(P.out + row / P.n_heads * P.out_tok + row % P.n_heads * P.out_head + d0) = w;
  }
}
// A wave's O^T (lane = row l32) as rows of LDS.
template <int D>
__device__ __forceinline__ void packed_stage(float *row, const f32x16 (&o)[D / 32], int g) {
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      *(f32x4 *)(row + db * 32 + 8 * i4 + 4 * g) = f32x4{o[db][i4 * 4], o[db][i4 * 4 + 1], o[db][i4 * 4 + 2], o[db][i4 * 4 + 3]};
}

// A wave's results, through 32 rows of D * 2 bytes of LDS that are its own: a lane of the accumulators has one row, so that a store straight from
// them would touch 64 cache lines, and as full rows it touches 8 or 16.  Partial results, twice as wide, go in two halves.  No barrier; chunks
// are permuted as K's.  A prompt of 14040 tokens 680 -> 672 us; short launches are as they were.
template <int D>
__device__ __forceinline__ void packed_results(const PackedItem &it, int wrow0, const f32x16 (&o)[D / 32], const PackedRow &R, char *stage, int lane) {
  typedef PackedTile<D> C;
  asm volatile("" : "+v"(lane));                                  // what follows from it is not held in registers through the loop over the tiles
  const int l32 = lane & 31, g = lane >> 5;
  const float lsum = partner_sum(R.l);
  const PackedTo<D> to = packed_to<D>(packed_params(), it, pf_min(wrow0 + l32, it.n_rows - 1), make_float2(R.m, lsum), wrow0 + l32 < it.n_rows && g == 0);
  char *const mine = stage + l32 * C::ROW_BYTES;
  const unsigned swz = C::swz_k(l32);
  // the staged rows to where lanes 0 .. 31 say, 16 bytes a lane
  auto store = [&](const void *where) __attribute__((always_inline)) {
    const unsigned long long w = (unsigned long long)where;
    const int r0 = lane / C::CHUNKS, p = lane % C::CHUNKS;
#pragma unroll
    for (int i = 0; i < 32 / C::COPY_ROWS; ++i) {
      const int r = i * C::COPY_ROWS + r0;
      const u32x4 x = *(const u32x4 *)(stage + r * C::ROW_BYTES + ((p ^ C::swz_k(r)) << 4));
      const unsigned lo = __builtin_amdgcn_ds_bpermute(r * 4, (int)(unsigned)w), hi = __builtin_amdgcn_ds_bpermute(r * 4, (int)(unsigned)(w >> 32));
      if (wrow0 + r < it.n_rows) *(u32x4 *)packed_global((char *)((unsigned long long)hi << 32 | lo) + 16 * p) = x;
    }
  };
  if (packed_plane(it) < 0) {
    // a lane holds four channels of every eight, the other half of the wave the other four: pairs of quads are exchanged, after which a lane
    // has eight channels side by side
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int pair = 0; pair < 2; ++pair) {
        bf16x8 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const auto r = __builtin_amdgcn_permlane32_swap(__float_as_int(o[db][pair * 8 + i]), __float_as_int(o[db][pair * 8 + 4 + i]), false, false);
          w[i] = (__bf16)(__int_as_float(r[0]) * to.inv);
          w[i + 4] = (__bf16)(__int_as_float(r[1]) * to.inv);
        }
        *(bf16x8 *)(mine + (((unsigned)(db * 4 + 2 * pair + g) ^ swz) << 4)) = w;
      }
    store(to.out);
  } else {
    constexpr int HALF = D / 64;                                  // channel blocks of a half
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
      for (int db = 0; db < HALF; ++db)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
          const f32x16 &x = o[h * HALF + db];
          *(f32x4 *)(mine + (((unsigned)(db * 8 + 2 * i4 + g) ^ swz) << 4)) = f32x4{x[i4 * 4], x[i4 * 4 + 1], x[i4 * 4 + 2], x[i4 * 4 + 3]};
        }
      store(to.part + h * (D / 2));
    }
  }
}

// ---- a full item: 128 rows, 32 a wave; the waves share every key tile, two stages of tiles copied global -> LDS directly ----
template <int D>
__device__ __forceinline__ void packed_full(const PackedItem &it, char *smem, int tid) {
  typedef PackedTile<D> C;
  typedef __attribute__((address_space(3))) void *lptr_t;
  constexpr int WROWS = PF_BK / PACKED_WAVES, NC = WROWS / C::COPY_ROWS;   // tile rows that one wave copies, in so many copies a tensor
  static_assert(WROWS % 16 == 0, "a wave's rows start at a multiple of the chunk permutations' period");
  static_assert(C::swz_v(C::COPY_ROWS) == 0 && C::swz_v(2 * C::COPY_ROWS) == 0, "all groups of a wave's rows permute V's chunks alike");
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5, n_tiles = it.kt1 - it.kt0;
  const int wrow0 = it.row0 + wave * 32;
  const bool has_rows = wrow0 < it.n_rows;
  char *const stage_q = smem + C::STAGE_BYTES + wave * (32 * C::ROW_BYTES);   // in the second tile's stage, whose copies go out behind a barrier
  bf16x8 qf[C::NKS];
  int pre, prefix_tokens, limit;                                  // the prefix's tiles and keys, if the line has it; this lane's row sees so many own keys
  float c;
  {
    const PackedParams P = packed_params();
    const int row = pf_min(wrow0 + l32, it.n_rows - 1);
    packed_send_q<D>(P, it, wrow0, stage_q, lane);
    pre = packed_has_prefix(it) ? P.prefix_tiles : 0;
    prefix_tokens = P.prefix_tokens;
    limit = packed_limit(P, it, row);
    c = P.scale_log2;
  }
  PackedRow R = packed_row(it, pre, limit, c);
  // Copies go by runs of whole tiles (of the prefix, of the line's own keys): from tile to tile only one scalar offset moves on, and a ragged last
  // tile goes row by row.  With base and offsets worked out for every tile a prompt of 14040 tokens took 757 us instead of 728.
  __amdgpu_buffer_rsrc_t run_k = __builtin_amdgcn_make_buffer_rsrc(nullptr, 0, 0, 0x00020000u), run_v = run_k;
  unsigned run_soff = 0, run_tile = 0, run_group = 0, run_vk[NC], run_vv = 0;
  int run_n = 0;                                                  // tiles left in the run
  asm volatile("" : "+s"(run_soff), "+s"(run_tile), "+s"(run_group), "+s"(run_n));   // scalars from the start (a zero shared with a vector register would keep them there)
#pragma unroll
  for (int i = 0; i < NC; ++i) run_vk[i] = 0;
  char *const mine = smem + wave * (WROWS * C::ROW_BYTES);
  auto copy_tile = [&](int u) __attribute__((always_inline)) {
    char *to = mine + (u & 1) * C::STAGE_BYTES;
    if (__builtin_expect(run_n <= 0, 0)) {
      if (u >= n_tiles) return;
      const PackedParams P = packed_params();
      const PackedKeys K = packed_keys(P, it);
      const int kt = it.kt0 + u;
      const bool in_prefix = kt < K.pre;
      const long long tok = in_prefix ? P.pre_tok : P.kv_tok;
      const int key0 = (in_prefix ? kt : kt - K.pre) * PF_BK;
      const int whole = ((in_prefix ? P.prefix_tokens : it.n_keys) - key0) / PF_BK;
      int lane_l = lane;
      asm volatile("" : "+v"(lane_l));                            // lane offsets are worked out here, not held in registers through the loop
      if (whole == 0) {
        packed_copy<D, false, WROWS>(P, it, K, kt, wave * WROWS, to, lane_l);
        packed_copy<D, true, WROWS>(P, it, K, kt, wave * WROWS, to + C::TENSOR_BYTES, lane_l);
        return;
      }
      const unsigned rb = (unsigned)(tok * 2);                    // bytes between key rows (below 2^25: checked on the host)
      run_tile = PF_BK * rb;
      run_n = __builtin_amdgcn_readfirstlane(pf_min(pf_min(whole, n_tiles - u), 1 << (__builtin_clz(run_tile) - 1)));   // offsets stay below 2^31
      run_soff = 0;
      run_group = C::COPY_ROWS * rb;
      const long long e = (long long)(key0 + wave * WROWS) * tok;
      run_k = __builtin_amdgcn_make_buffer_rsrc((void *)((in_prefix ? K.k_pre : K.k) + e), 0, -1, 0x00020000u);
      run_v = __builtin_amdgcn_make_buffer_rsrc((void *)((in_prefix ? K.v_pre : K.v) + e), 0, -1, 0x00020000u);
      const int rr = lane_l / C::CHUNKS, p = lane_l % C::CHUNKS;
#pragma unroll
      for (int i = 0; i < NC; ++i) run_vk[i] = (unsigned)((p ^ C::swz_k(rr) ^ C::swz_k(i * C::COPY_ROWS)) << 4) + (unsigned)rr * rb;
      run_vv = (unsigned)((p ^ C::swz_v(rr)) << 4) + (unsigned)rr * rb;
    }
    --run_n;
    static_for<0, NC>([&](auto gi) {
      constexpr int G = decltype(gi)::value;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(run_k, (lptr_t)(to + G * 1024), 16, run_vk[G], run_soff + G * run_group, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(run_v, (lptr_t)(to + C::TENSOR_BYTES + G * 1024), 16, run_vv, run_soff + G * run_group, 0, 0);
    });
    run_soff += run_tile;
  };
  copy_tile(0);
  // the limit grows with the row: the wave's first lane has the least, its 32nd the most
  const int lim_first = __builtin_amdgcn_readlane(limit, 0), lim_last = __builtin_amdgcn_readlane(limit, 31);
  if (n_tiles > 0) wait_vm<2 * NC>();                             // the first tile may still travel
  else wait_vm<0>();
  packed_read_q<D>(stage_q, lane, qf);
  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
  unsigned ak, av;
  packed_lds<D>(smem, smem + C::TENSOR_BYTES, lane, ak, av);
  for (int u = 0; u < n_tiles; ++u) {
    const unsigned stage = (u & 1) * C::STAGE_BYTES;
    wait_vm<0>();                                                 // this wave's share of tile u has landed
    __builtin_amdgcn_s_barrier();                                 // ... everyone's has, and everyone is done with tile u-1
    copy_tile(u + 1);
    const int kt = it.kt0 + u, t0 = (kt < pre ? kt : kt - pre) * PF_BK;
    if (!has_rows || (kt >= pre && t0 >= lim_last)) continue;     // none of this wave's rows sees the tile
    f32x16 s[2];
    packed_qk<D, 2>(s, qf, ak + stage);
    if (__builtin_expect((kt < pre ? prefix_tokens : lim_first) - t0 < PF_BK, 0))   // some row does not see the whole tile
      packed_mask<2>(s, (kt < pre ? prefix_tokens : limit) - t0, g);
    bf16x8 pf[4];
    packed_softmax<D, 2>(s, pf, o, R, c, u == 0);
    packed_pv<D, 4>(o, pf, av + stage);
  }
  // the stage of the tile before the last: every wave is done with it
  packed_results<D>(it, wrow0, o, R, smem + (n_tiles & 1) * C::STAGE_BYTES + wave * (32 * C::ROW_BYTES), lane);
}

// ---- a thin item: 32 rows that all waves hold, the keys split over the waves.  Each streams steps of 32 keys through a place of its own in
// LDS, without barriers: K of the next step is sent once this step's K fragments are in registers, V of the next once its V^T fragments
// are.  The waves' results are joined in LDS.  For lines of few rows (single tokens), where three waves of a full item would have nothing
// but copies to do and a tile would take as long. ----
template <int D>
__device__ __forceinline__ void packed_thin(const PackedItem &it, char *smem, float2 *s_ml, int tid) {
  typedef PackedTile<D> C;
  const PackedParams P = packed_params();
  constexpr int KEYS = 32, NC = KEYS / C::COPY_ROWS;              // of a step; its copies of one tensor
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5;
  const float c = P.scale_log2;
  const PackedKeys K = packed_keys(P, it);
  const int row = pf_min(it.row0 + l32, it.n_rows - 1);
  const int steps = 2 * (it.kt1 - it.kt0), j0 = steps * wave / PACKED_WAVES, j1 = steps * (wave + 1) / PACKED_WAVES;
  char *mine_k = smem + wave * (2 * KEYS * C::ROW_BYTES), *mine_v = mine_k + KEYS * C::ROW_BYTES;
  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
  const int limit = packed_limit(P, it, row);
  PackedRow R = packed_row(it, K.pre, limit, c);
  if (j0 < j1) {
    bf16x8 qf[C::NKS];
    packed_load_q<D>(P, it, row, g, qf);
    packed_copy<D, false, KEYS>(P, it, K, it.kt0 + j0 / 2, j0 % 2 * KEYS, mine_k, lane);
    packed_copy<D, true, KEYS>(P, it, K, it.kt0 + j0 / 2, j0 % 2 * KEYS, mine_v, lane);
    const int lim_first = __builtin_amdgcn_readlane(limit, 0);
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) asm volatile("" : "+v"(qf[ks]));
    unsigned ak, av;
    packed_lds<D>(mine_k, mine_v, lane, ak, av);
    for (int j = j0; j < j1; ++j) {
      const bool more = j + 1 < j1;
      const int kt = it.kt0 + j / 2, t0 = (kt < K.pre ? kt : kt - K.pre) * PF_BK + j % 2 * KEYS;
      wait_vm<NC>();                                              // K of this step has landed (its V may still travel)
      f32x16 s[1];
      packed_qk<D, 1>(s, qf, ak);
      if (more) packed_copy<D, false, KEYS>(P, it, K, it.kt0 + (j + 1) / 2, (j + 1) % 2 * KEYS, mine_k, lane);
      if (__builtin_expect((kt < K.pre ? P.prefix_tokens : lim_first) - t0 < KEYS, 0))
        packed_mask<1>(s, (kt < K.pre ? P.prefix_tokens : limit) - t0, g);
      bf16x8 pf[2];
      packed_softmax<D, 1>(s, pf, o, R, c, j == j0);
      if (more) wait_vm<NC>();                                    // V of this step has landed (K of the next may still travel)
      else wait_vm<0>();
      packed_pv<D, 2>(o, pf, av);
      if (more) packed_copy<D, true, KEYS>(P, it, K, it.kt0 + (j + 1) / 2, (j + 1) % 2 * KEYS, mine_v, lane);
    }
  }
  __syncthreads();
  float *sO = (float *)smem;
  const float lsum = partner_sum(R.l);
  packed_stage<D>(sO + (wave * 32 + l32) * C::LD, o, g);
  if (g == 0) s_ml[wave * 32 + l32] = make_float2(R.m, lsum);
  __syncthreads();
  for (int e = tid; e < 32 * (D / 8); e += PACKED_WAVES * 64) {
    const int r = e / (D / 8), d0 = (e % (D / 8)) * 8;
    float2 ml[PACKED_WAVES], all = make_float2(PACKED_SEES_NONE, 0.0f);
#pragma unroll
    for (int w = 0; w < PACKED_WAVES; ++w) ml[w] = s_ml[w * 32 + r], all.x = fmaxf(all.x, ml[w].x);
    f32x4 a = {0.0f, 0.0f, 0.0f, 0.0f}, b = a;
#pragma unroll
    for (int w = 0; w < PACKED_WAVES; ++w) {
      const float f = fast_exp2((ml[w].x - all.x) * c);
      const f32x4 x = *(const f32x4 *)(sO + (w * 32 + r) * C::LD + d0), y = *(const f32x4 *)(sO + (w * 32 + r) * C::LD + d0 + 4);
      all.y += f * ml[w].y;
#pragma unroll
      for (int i = 0; i < 4; ++i) a[i] += f * x[i], b[i] += f * y[i];
    }
    if (it.row0 + r < it.n_rows) packed_put<D>(packed_to<D>(P, it, it.row0 + r, all, d0 == 0), d0, a, b);
  }
}

template <int D>
__global__ __launch_bounds__(PACKED_WAVES * 64, 2 * 128 / D) void pf_packed_attn_kernel(PackedParams) {
  typedef PackedTile<D> C;
  constexpr int THIN_STAGE = PACKED_WAVES * 32 * C::LD * 4;       // where a thin item joins its waves' results
  __shared__ __attribute__((aligned(1024))) char smem[2 * C::STAGE_BYTES > THIN_STAGE ? 2 * C::STAGE_BYTES : THIN_STAGE];
  __shared__ float2 s_ml[PACKED_WAVES * 32];
  __shared__ int32_t s_last;
  bool there;
  const PackedItem it = packed_item(there);
  if (__builtin_expect(!there, 0)) {
    packed_no_plan<D>(threadIdx.x, PACKED_WAVES * 64);
    return;
  }
  if (!packed_is_thin(it)) {
    packed_full<D>(it, smem, threadIdx.x);
    return;
  }
  packed_thin<D>(it, smem, s_ml, threadIdx.x);
  packed_arrive<D>(it, &s_last, threadIdx.x);                     // (a head of few rows has thin items only)
}
static_assert(PACKED_ARRIVE_ROWS <= PACKED_THIN_ROWS, "full and wide items have no arrivals");

#include "pf_packed_wide.h"


// Joins the planes of every parked row: out = sum_p 2^((m_p - M) c) O_p / sum_p 2^((m_p - M) c) l_p.
//
// Few planes: D / 8 lanes take a row, eight channels each, plane after plane.
template <int D>
__global__ __launch_bounds__(256) void pf_packed_join_few_kernel(PackedParams P) {
  constexpr int LANES = D / 8;
  const int id = blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (id >= P.part_rows) return;
  const bool there = packed_is_there(P);
  const int d0 = threadIdx.x % LANES * 8, row = P.part_row[id];
  float2 ml[PACKED_FEW_PLANES];
#pragma unroll
  for (int p = 0; p < PACKED_FEW_PLANES; ++p) ml[p] = p < P.planes ? P.part_ml[(long long)p * P.part_rows + id] : make_float2(PACKED_SEES_NONE, 0.0f);
  float top = PACKED_SEES_NONE, sum = 0.0f, acc[8] = {};
  bool lost = false;
#pragma unroll
  for (int p = 0; p < PACKED_FEW_PLANES; ++p) top = fmaxf(top, ml[p].x), lost |= ml[p].x == -INFINITY;
  f32x4 x[PACKED_FEW_PLANES][2];
#pragma unroll
  for (int p = 0; p < PACKED_FEW_PLANES; ++p) {
    x[p][0] = x[p][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (ml[p].y == 0.0f) continue;                                // a plane that saw no key (or has no item) counts nothing
    const float *o = P.part_o + ((long long)p * P.part_rows + id) * D + d0;
    x[p][0] = *(const f32x4 *)o;
    x[p][1] = *(const f32x4 *)(o + 4);
  }
#pragma unroll
  for (int p = 0; p < PACKED_FEW_PLANES; ++p) {
    if (ml[p].y == 0.0f) continue;
    const float w = fast_exp2((ml[p].x - top) * P.scale_log2);
    sum += w * ml[p].y;
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += w * x[p][0][e], acc[e + 4] += w * x[p][1][e];
  }
  if (!there) return;
  const float inv = packed_inverse(sum, lost);
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)(acc[i] * inv);
  *(bf16x8 *)(P.out + row / P.n_heads * P.out_tok + row % P.n_heads * P.out_head + d0) = r;
}
// Many planes: a wave takes a row: its lanes look at a
// plane's maximum and sum each, then groups of D / 8 lanes (eight channels a lane) add up every 64 / (D / 8)-th plane and the groups'
// sums are added in a fixed order.  Bound: with few rows two round trips to memory, with many the planes' bytes.
__device__ __forceinline__ float packed_lane(float x, int lane) { return __int_as_float(__builtin_amdgcn_ds_bpermute(lane * 4, __float_as_int(x))); }
template <int D>
__global__ __launch_bounds__(256) void pf_packed_join_kernel(PackedParams P) {
  constexpr int LANES = D / 8, GROUPS = 64 / LANES;
  const int lane = threadIdx.x & 63;
  const int id = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (id >= P.part_rows) return;
  const bool there = packed_is_there(P);
  const int d0 = lane % LANES * 8, grp = lane / LANES, row = P.part_row[id];
  float2 ml[PACKED_JOIN_BATCHES];
  float top = PACKED_SEES_NONE;
  bool lost = false;
#pragma unroll
  for (int b = 0; b < PACKED_JOIN_BATCHES; ++b) {
    ml[b] = make_float2(PACKED_SEES_NONE, 0.0f);
    if (b * 64 + lane < P.planes) ml[b] = P.part_ml[(long long)(b * 64 + lane) * P.part_rows + id];
  }
#pragma unroll
  for (int b = 0; b < PACKED_JOIN_BATCHES; ++b) top = fmaxf(top, ml[b].x), lost |= __ballot(ml[b].x == -INFINITY) != 0;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) top = fmaxf(top, packed_lane(top, lane ^ step));
  float w[PACKED_JOIN_BATCHES], sum = 0.0f;
#pragma unroll
  for (int b = 0; b < PACKED_JOIN_BATCHES; ++b) {
    w[b] = ml[b].y == 0.0f ? 0.0f : fast_exp2((ml[b].x - top) * P.scale_log2);   // a plane that saw no key (or has no item) counts nothing
    sum += w[b] * ml[b].y;
  }
#pragma unroll
  for (int step = 1; step < 64; step *= 2) sum += packed_lane(sum, lane ^ step);
  float acc[8] = {};
#pragma unroll
  for (int b = 0; b < PACKED_JOIN_BATCHES; ++b) {
    for (int p0 = 0; p0 < 64 && b * 64 + p0 < P.planes; p0 += 2 * GROUPS) {
      f32x4 x[2][2];
      float f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {                               // two planes of every group in flight
        const int p = p0 + i * GROUPS + grp;
        f[i] = packed_lane(w[b], pf_min(p, 63));
        if (p > 63) f[i] = 0.0f;
        x[i][0] = x[i][1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (f[i] != 0.0f) {
          const float *o = P.part_o + ((long long)(b * 64 + p) * P.part_rows + id) * D + d0;
          x[i][0] = *(const f32x4 *)o;
          x[i][1] = *(const f32x4 *)(o + 4);
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] += f[i] * x[i][0][e], acc[e + 4] += f[i] * x[i][1][e];
    }
  }
#pragma unroll
  for (int step = LANES; step < 64; step *= 2)
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += packed_lane(acc[e], lane ^ step);
  if (grp != 0 || !there) return;
  const float inv = packed_inverse(sum, lost);
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = (__bf16)(acc[i] * inv);
  *(bf16x8 *)(P.out + row / P.n_heads * P.out_tok + row % P.n_heads * P.out_head + d0) = r;
}

// ---- host ------------------------------------------------------------------------------------------------------------

static int packed_check(const pf_packed *p) {
  if (!p || p->reserved) return PF_ERR_INVALID_ARG;
  if (p->head_dim != 64 && p->head_dim != 128) return PF_ERR_UNSUPPORTED;
  if (p->n_heads < 1 || p->n_heads > PF_MAX_HEADS || p->n_kv_heads < 1 || p->n_heads % p->n_kv_heads) return PF_ERR_INVALID_ARG;
  if (p->n_seqs < 1 || p->n_seqs > (1 << 20) || p->block < 0 || p->prefix_tokens < 0 || p->prefix_tokens > (1 << 24)) return PF_ERR_INVALID_ARG;
  if (!p->cu_q || !p->cu_k || p->cu_q[0] != 0 || p->cu_k[0] != 0) return PF_ERR_INVALID_ARG;
  for (int s = 0; s < p->n_seqs; ++s)
    if (p->cu_q[s + 1] < p->cu_q[s] || p->cu_k[s + 1] < p->cu_k[s]) return PF_ERR_INVALID_ARG;
  if (p->cu_q[p->n_seqs] > (1 << 24) || p->cu_k[p->n_seqs] > (1 << 30)) return PF_ERR_INVALID_ARG;
  if ((long long)p->cu_q[p->n_seqs] * p->n_heads > (1ll << 30)) return PF_ERR_INVALID_ARG;
  return PF_OK;
}

// A row tile's keys on the host: those that its last row sees.
static int packed_host_limit(const pf_packed *p, int lq, int lk, int query) {
  if (p->block == 0) return lk;
  const long long place = (long long)lk - lq + query;
  if (place < 0) return 0;
  return (int)std::min<long long>(lk, (place / p->block + 1) * p->block);
}

// Plan in pf_packed.work: its head, items, then the heads' arrival counters.
static size_t packed_plan_bytes(size_t items, int kv_heads) {
  return pf_align_up(sizeof(PackedHead) + items * sizeof(PackedItem) + (size_t)kv_heads * sizeof(int32_t), sizeof(PackedHead));
}
static PackedItem *packed_items(const pf_packed *p) { return (PackedItem *)((PackedHead *)p->work + 1); }
// Room for the plan of any lengths with so many row tiles: theirs and those of stacked lines uncut, and as many items again as several rounds of
// every place on the chip.  The planner looks at no cut that has more (it would pay for their set-up 16 times over).
constexpr long long PACKED_CUT_ITEMS = 8192;
constexpr long long PACKED_MAX_ITEMS = (1 << 23) - 1;             // a launch has fewer than 2^32 threads, an item up to 512
static long long packed_most_items(const pf_packed *p) {
  const int G = p->n_heads / p->n_kv_heads;
  long long tiles = 0;
  for (int s = 0; s < p->n_seqs; ++s) tiles += pf_ceil_div((long long)(p->cu_q[s + 1] - p->cu_q[s]) * G, PACKED_ROWS);
  return (p->prefix_tokens > 0 ? 2 : 1) * tiles * p->n_kv_heads + PACKED_CUT_ITEMS;
}
// Few rows a head: its last workgroup joins them and there is no second launch.
static bool packed_by_arrival(const pf_packed *p) { return (long long)p->cu_q[p->n_seqs] * (p->n_heads / p->n_kv_heads) <= PACKED_ARRIVE_ROWS; }

struct PackedPlan {
  std::vector<PackedItem> items;
  int planes = 0, head_rows = 0;   // a key head's rows that park
  bool wide = false;           // items of 256 rows (head_dim 128)
};

// Rows that share their keys: one sequence's, or in front of the prefix those of neighbouring sequences.
struct PackedLine {
  int q_base, n_rows, k_base, n_keys;
  bool prefix;                 // has the prefix's tiles
  int stack;                   // >= 0: the line that has the prefix in this one's place; -1: this line has all of its rows' keys; -2: it is such a line
  bool thin;                   // goes by thin items
};
struct PackedRowTile {
  int line, row0, n_kt;
  bool thin;
  int load;                    // its time, where all places are taken, in key tiles of a full item
};

// What the planner knows of the time that things take, in microseconds, measured on launches of 32 to 1024 items of 1 to 32 key tiles.  All
// places taken: a full item's key tile, and a key tile that no other row tile reads from memory; few taken: a key tile of a full and of a thin item.
// An item's set-up and end; the second launch; a row of a plane written and read.
struct PackedCosts {
  int rows, thin_rows, places; // of a full item; of a thin one at most; workgroups on the chip at once
  double tile, tile_alone, tile_few, tile_thin, item, join, plane_row;
};
static PackedCosts packed_costs(int head_dim, bool wide) {
  if (wide) return {PACKED_WIDE_ROWS, 0, 256, 1.8, 1.8, 1.5, 0.35, 5.0, 6.0, 2.3e-4};
  if (head_dim == 128) return {PACKED_ROWS, PACKED_THIN_ROWS, 512, 1.95, 3.4, 1.15, 0.42, 3.0, 6.0, 2.3e-4};
  return {PACKED_ROWS, PACKED_THIN_ROWS, 1024, 2.3, 3.4, 0.85, 0.32, 3.0, 6.0, 1.2e-4};
}

static int packed_line_tiles(const pf_packed *p, const PackedLine &l, int row0, int rows, int pre_kt) {
  const int G = p->n_heads / p->n_kv_heads, last = pf_min(row0 + rows, l.n_rows) - 1;
  const int own = l.n_keys > 0 ? pf_ceil_div(packed_host_limit(p, l.n_rows / G, l.n_keys, last / G), PF_BK) : 0;
  return own + (l.prefix ? pre_kt : 0);
}

// How a batch's row tiles (heaviest first) are cut: the first `whole` not at all, the others into runs of at most seg full key tiles' time.
struct PackedCut {
  int whole, seg;
  int of(int i, const PackedRowTile &t) const { return i < whole ? 1 : std::max(1, std::min(pf_ceil_div(t.load, seg), t.n_kt)); }
};

// Time that the launch takes under a cut; more than `limit` is not worked out.
static double packed_time(const std::vector<PackedRowTile> &tiles, int heads, const PackedCut &cut, const PackedCosts &C, double limit) {
  long long n = 0;
  int longest = 0;
  double work = 0.0, few = 0.0;
  for (size_t i = 0; i < tiles.size(); ++i) {
    const int cuts = cut.of((int)i, tiles[i]);
    n += (long long)cuts * heads;
    longest = std::max(longest, pf_ceil_div(tiles[i].load, cuts));
    few = std::max(few, pf_ceil_div(tiles[i].n_kt, cuts) * (tiles[i].thin ? C.tile_thin : C.tile_few));
    work += tiles[i].load * (double)heads;
  }
  if (n <= C.places / 2) return C.item + few;
  if ((work * C.tile + n * C.item) / C.places > limit) return 1e300;
  std::vector<int> count(longest + 1, 0);
  for (size_t i = 0; i < tiles.size(); ++i) {
    const int cuts = cut.of((int)i, tiles[i]);
    count[pf_ceil_div(tiles[i].load, cuts)] += cuts * heads;      // (a run may be a tile shorter)
  }
  // heaviest first, each to the place that is free first; places that become free together go on together
  typedef std::pair<double, int> Free;
  std::priority_queue<Free, std::vector<Free>, std::greater<Free>> free_at;
  free_at.push({0.0, C.places});
  double end = C.item + few;
  for (int t = longest; t >= 0; --t)
    for (int left = count[t]; left > 0;) {
      const Free first = free_at.top();
      const int n_taken = std::min(left, first.second);
      const double at = first.first + C.item + t * C.tile;
      free_at.pop();
      if (first.second > n_taken) free_at.push({first.first, first.second - n_taken});
      free_at.push({at, n_taken});
      left -= n_taken;
      end = std::max(end, at);
      if (end > limit) return 1e300;
    }
  return end;
}

// The batch's lines and how their keys are cut, as fast as the costs above say.  take_all: every sequence has the prefix in its own line;
// otherwise those whose tiles would stay mostly empty in front of it are stacked.  Returns the time.
struct PackedLayout {
  std::vector<PackedLine> lines;
  std::vector<PackedRowTile> tiles;
  std::vector<int> cuts, first, park;  // of every row tile: into how many items its keys are cut, the plane of the first, where its line's row 0 parks
  int planes = 0, head_rows = 0;
};
// Partial results: O, and the row's maximum and sum, a plane; and which row it is.  Cuts may bring them to this; two planes of the rows that are
// stacked, all in front of the prefix and all behind it, are there without any cut.
constexpr double PACKED_PART_BYTES = 1e9;
static size_t packed_part_bytes(const pf_packed *p, int planes, long long head_rows) {
  return planes == 0 ? 0 : (size_t)head_rows * p->n_kv_heads * ((size_t)planes * ((size_t)p->head_dim * 4 + 8) + 4);
}
static double packed_lay_out(const pf_packed *p, const PackedCosts &C, bool take_all, PackedLayout &L) {
  const int G = p->n_heads / p->n_kv_heads, KV = p->n_kv_heads, BQ = C.rows;
  const int pre_kt = pf_ceil_div(p->prefix_tokens, PF_BK);
  std::vector<PackedLine> &lines = L.lines;
  std::vector<PackedRowTile> &tiles = L.tiles;
  int stack = -1;
  bool any_stack = false;
  for (int s = 0; s < p->n_seqs; ++s) {
    const int lq = p->cu_q[s + 1] - p->cu_q[s], r = lq * G;
    if (lq == 0) continue;
    // the rows that its tiles would leave empty in front of the prefix, against parking its rows' partial results
    const double empty = r <= C.thin_rows ? 1.0 : pf_ceil_div(r, BQ) - (double)r / BQ;
    const bool own = pre_kt == 0 || take_all || empty * pre_kt * C.tile / C.places < 2.0 * r * C.plane_row;
    if (own) {
      stack = -1;
    } else {
      if (stack < 0) {
        stack = (int)lines.size();
        lines.push_back({p->cu_q[s], 0, 0, 0, true, -2, false});
      }
      lines[stack].n_rows += r;
      any_stack = true;
    }
    lines.push_back({p->cu_q[s], r, p->cu_k[s], p->cu_k[s + 1] - p->cu_k[s], pre_kt > 0 && own, stack, false});
  }
  for (PackedLine &l : lines) l.thin = l.n_rows <= C.thin_rows;
  long long with_prefix = 0;
  for (const PackedLine &l : lines)
    if (l.prefix) with_prefix += pf_ceil_div(l.n_rows, BQ);
  // a key tile's time in full tiles: what its bytes take where row tiles that read them are few, if that is more
  auto load_of = [&](int n_pre, int n_own, const PackedLine &l) {
    const double least = l.thin ? C.tile_thin / C.tile_few : 1.0, alone = C.tile_alone / C.tile;
    const double pre = std::max(least, alone / std::max(1ll, with_prefix)), own = std::max(least, alone / pf_ceil_div(l.n_rows, BQ));
    return (int)ceil(n_pre * pre + n_own * own - 1e-9);
  };
  for (size_t l = 0; l < lines.size(); ++l)
    for (int r0 = 0; r0 < lines[l].n_rows; r0 += BQ) {
      const int n_kt = packed_line_tiles(p, lines[l], r0, BQ, pre_kt), pre = lines[l].prefix ? pre_kt : 0;
      tiles.push_back({(int)l, r0, n_kt, lines[l].thin, load_of(pre, n_kt - pre, lines[l])});
    }
  std::stable_sort(tiles.begin(), tiles.end(), [](const PackedRowTile &a, const PackedRowTile &b) { return a.load > b.load; });
  const int longest = tiles.empty() ? 1 : std::max(1, tiles[0].load);
  // A row's planes: its stacked line's first, then its own line's (every tile of a stacked line is cut alike, so that own planes start at one place).
  std::vector<int> stack_load(lines.size(), 0);
  for (size_t l = 0; l < lines.size(); ++l)
    if (lines[l].stack == -2) stack_load[l] = load_of(pre_kt, 0, lines[l]);
  auto stack_cuts = [&](int line, int seg) { return std::max(1, std::min(pf_ceil_div(stack_load[line], seg), pre_kt)); };
  auto cuts_of = [&](const PackedCut &cut, size_t i) {
    return lines[tiles[i].line].stack == -2 ? stack_cuts(tiles[i].line, cut.seg) : cut.of((int)i, tiles[i]);
  };
  long long n_items = 0, head_rows = 0;
  auto planes_of = [&](const PackedCut &cut, double *parked) {
    int most = 0;
    *parked = 0.0;
    n_items = head_rows = 0;
    for (size_t i = 0; i < tiles.size(); ++i) {
      const PackedLine &l = lines[tiles[i].line];
      const int n = cuts_of(cut, i), before = l.stack >= 0 ? stack_cuts(l.stack, cut.seg) : 0;
      n_items += (long long)n * KV;
      if (l.stack == -1 && n == 1) continue;
      most = std::max(most, before + n);
      if (l.stack != -2) head_rows += pf_min(BQ, l.n_rows - tiles[i].row0);
      *parked += (double)n * pf_min(BQ, l.n_rows - tiles[i].row0);
    }
    return most;
  };
  const long long most_items = packed_most_items(p);
  PackedCut best = {0, longest};
  double parked = 0.0, least = 1e300;
  if ((long long)tiles.size() * KV <= 8ll * C.places) {
    const int rounds = (int)((long long)tiles.size() * KV / C.places);
    for (int whole_rounds = any_stack ? 0 : rounds; whole_rounds >= 0; whole_rounds = whole_rounds > 0 ? 0 : -1) {
      const int whole = whole_rounds * C.places / KV;
      const int most = whole < (int)tiles.size() ? std::max(1, tiles[whole].load) : 1;   // the longest that is cut
      for (int n : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64, 80, 96, 120}) {
        const PackedCut cut = {whole, pf_ceil_div(most, n)};
        const int planes = planes_of(cut, &parked);
        if (planes > PACKED_MAX_PLANES || n_items > most_items || (n > 1 && (double)packed_part_bytes(p, planes, head_rows) > PACKED_PART_BYTES)) break;
        const double rest = planes ? (packed_by_arrival(p) ? 1.0 + 0.3 * planes : C.join) + parked * KV * C.plane_row : 0.0;
        if (rest >= least) break;
        // a plan with partial results has to be a good deal faster: whole launches run at their power limit, where idle places at the end
        // leave the others a higher clock
        const double handicap = planes && !any_stack ? 1.1 : 1.0;
        const double t = (packed_time(tiles, KV, cut, C, least / handicap - rest) + rest) * handicap;
        if (t < least) {
          least = t;
          best = cut;
        }
        if (cut.seg == 1) break;
      }
    }
  } else {
    double work = 0.0;
    for (const PackedRowTile &t : tiles) work += (double)t.load * KV;
    least = work * C.tile / C.places;
  }
  L.planes = planes_of(best, &parked);
  for (size_t i = 0; i < tiles.size(); ++i) {
    const int st = lines[tiles[i].line].stack;
    L.cuts.push_back(cuts_of(best, i));
    L.first.push_back(st >= 0 ? stack_cuts(st, best.seg) : 0);
  }
  // parked rows: those of stacked lines, in which the sequences behind them have theirs, then the other cut tiles'
  std::vector<int> line_park(lines.size(), 0);
  for (size_t l = 0; l < lines.size(); ++l) {
    const PackedLine &x = lines[l];
    if (x.stack == -2) line_park[l] = L.head_rows, L.head_rows += x.n_rows;
    if (x.stack >= 0) line_park[l] = line_park[x.stack] + (x.q_base - lines[x.stack].q_base) * G;
  }
  for (size_t i = 0; i < tiles.size(); ++i) {
    const PackedLine &x = lines[tiles[i].line];
    L.park.push_back(x.stack == -1 ? L.head_rows - tiles[i].row0 : line_park[tiles[i].line]);
    if (x.stack == -1 && L.cuts[i] > 1) L.head_rows += pf_min(BQ, x.n_rows - tiles[i].row0);
  }
  return least;
}

static void packed_make(const pf_packed *p, PackedPlan &plan) {
  PackedLayout L;
  double least = 1e300;
  for (int wide = 0; wide < (p->head_dim == 128 && !packed_by_arrival(p) ? 2 : 1); ++wide)
    for (int take_all = 0; take_all < (p->prefix_tokens > 0 ? 2 : 1); ++take_all) {
      PackedLayout other;
      const double t = packed_lay_out(p, packed_costs(p->head_dim, wide != 0), take_all != 0, other);
      if (t < least) {
        least = t;
        L = std::move(other);
        plan.wide = wide != 0;
      }
    }
  plan.planes = L.planes;
  plan.head_rows = L.head_rows;
  struct Loaded {
    PackedItem item;
    int load;
  };
  std::vector<Loaded> items;
  for (int h = 0; h < p->n_kv_heads; ++h)
    for (size_t t = 0; t < L.tiles.size(); ++t) {
      const PackedRowTile &tile = L.tiles[t];
      const PackedLine &l = L.lines[tile.line];
      const int n = L.cuts[t];
      for (int i = 0; i < n; ++i) {
        PackedItem it = {l.q_base, tile.row0, l.n_rows, l.k_base, l.n_keys, pf_seg_begin(tile.n_kt, n, i), pf_seg_begin(tile.n_kt, n, i + 1), h, L.park[t]};
        if (l.prefix) it.head |= 1 << PACKED_PREFIX_BIT;
        if (tile.thin) it.head |= (int)(1u << 31);
        if (!(l.stack == -1 && n == 1)) {
          it.head |= (L.first[t] + i + 1) << 13;
          if (i == n - 1 && l.stack != -2) it.head |= (L.planes - L.first[t] - n) << 22;
        }
        items.push_back({it, tile.load / n});
      }
    }
  // Heaviest first.  Workgroup i runs on die i % 8, and every die has an L2 of its own: among items of one load, which have no order to keep,
  // the heads are dealt out to the dies in runs, so that a die's workgroups read the keys of one head or two.
  std::stable_sort(items.begin(), items.end(), [](const Loaded &a, const Loaded &b) { return a.load > b.load; });
  plan.items.resize(items.size());
  for (size_t a = 0, b; a < items.size(); a = b) {
    for (b = a + 1; b < items.size() && items[b].load == items[a].load;) ++b;
    size_t from = a;
    for (size_t d = 0; d < PF_NUM_XCD; ++d)
      for (size_t i = a + (d + PF_NUM_XCD - a % PF_NUM_XCD) % PF_NUM_XCD; i < b; i += PF_NUM_XCD) plan.items[i] = items[from++].item;
  }
}

// What a plan is for: with anything else its items would point outside the tensors.
static uint64_t packed_checksum(const pf_packed *p) {
  uint64_t h = 1469598103934665603ull;                            // FNV-1a, a word at a time
  auto add = [&](int32_t x) { h = (h ^ (uint32_t)x) * 1099511628211ull; };
  for (const int32_t x : {p->n_seqs, p->n_heads, p->n_kv_heads, p->head_dim, p->block, p->prefix_tokens, p->n_items, p->n_planes, p->kernel}) add(x);
  for (int s = 1; s <= p->n_seqs; ++s) add(p->cu_q[s]), add(p->cu_k[s]);
  if (p->n_unparked) add(p->n_unparked);
  return h;
}
static bool packed_is_planned(const pf_packed *p) {
  return p->total_q == p->cu_q[p->n_seqs] && p->total_k == p->cu_k[p->n_seqs] && p->planned_for == packed_checksum(p);
}

// rows of a key head that park under the batch's plan
static int packed_head_rows(const pf_packed *p) { return p->cu_q[p->n_seqs] * (p->n_heads / p->n_kv_heads) - p->n_unparked; }

// Runs f; memory that the plan needs on the host and does not get is an error, not an exception.
template <class F>
static int packed_guard(F &&f) {
  try {
    return f();
  } catch (const std::bad_alloc &) {
    return PF_ERR_CAPACITY;
  } catch (...) {
    return PF_ERR_INVALID_ARG;
  }
}

extern "C" size_t pf_packed_work_bytes(const pf_packed *packed) {
  if (packed_check(packed) != PF_OK) return 0;
  const long long items = packed_most_items(packed);
  return items > PACKED_MAX_ITEMS ? 0 : packed_plan_bytes((size_t)items, packed->n_kv_heads);
}

extern "C" int pf_packed_plan(pf_packed *packed, void *stream) {
  return packed_guard([&]() {
    const int rc = packed_check(packed);
    if (rc != PF_OK) return rc;
    if (!packed->work || ((uintptr_t)packed->work & 31u)) return (int)PF_ERR_INVALID_ARG;
    const size_t need = pf_packed_work_bytes(packed);
    if (need == 0) return (int)PF_ERR_UNSUPPORTED;
    if (packed->work_bytes < need) return (int)PF_ERR_CAPACITY;
    PackedPlan plan;
    packed_make(packed, plan);
    if (plan.items.size() > (size_t)packed_most_items(packed)) return (int)PF_ERR_UNSUPPORTED;
    pf_packed planned = *packed;
    planned.n_items = (int32_t)plan.items.size();
    planned.n_planes = plan.planes;
    planned.kernel = plan.wide ? 1 : 0;
    planned.n_unparked = 0;
    if (plan.planes > 0) planned.n_unparked = packed_head_rows(&planned) - plan.head_rows;
    planned.total_q = packed->cu_q[packed->n_seqs];
    planned.total_k = packed->cu_k[packed->n_seqs];
    planned.planned_for = packed_checksum(&planned);
    planned.planned_in = packed->work;
    PackedItem *to = packed_items(packed);
    for (size_t i = 0; i < plan.items.size(); i += PACKED_UPLOAD) {
      PackedUpload U;
      const int n = (int)std::min<size_t>(PACKED_UPLOAD, plan.items.size() - i);
      memcpy(U.item, &plan.items[i], n * sizeof(PackedItem));
      if (n < PACKED_UPLOAD) memset(U.item + n, 0, (PACKED_UPLOAD - n) * sizeof(PackedItem));
      const bool last = i + n == plan.items.size();               // there is no plan before its last item
      hipLaunchKernelGGL(pf_packed_upload_kernel, dim3(1), dim3(128), 0, (hipStream_t)stream, U, n, to + i, (int32_t *)(to + plan.items.size()),
                         i == 0 ? packed->n_kv_heads : 0, (PackedHead *)packed->work, last ? planned.planned_for : 0);
      PF_HIP_CHECK(hipGetLastError());
    }
    *packed = planned;
    return (int)PF_OK;
  });
}

extern "C" size_t pf_packed_workspace_bytes(const pf_packed *packed) {
  if (packed_check(packed) != PF_OK || !packed_is_planned(packed)) return 0;
  return pf_align_up(packed_part_bytes(packed, packed->n_planes, packed_head_rows(packed)) + 256, 256);
}

extern "C" int pf_packed_attn_fwd(const pf_packed *packed, const void *q, const pf_chunk_layout *q_layout, const void *k, const void *v,
                                  const pf_chunk_layout *kv_layout, const void *k_prefix, const void *v_prefix,
                                  const pf_chunk_layout *prefix_layout, void *out, const pf_chunk_layout *out_layout,
                                  float softmax_scale, void *workspace, size_t workspace_bytes, void *stream) {
  const int rc = packed_check(packed);
  if (rc != PF_OK) return rc;
  const int tq = packed->cu_q[packed->n_seqs], tk = packed->cu_k[packed->n_seqs], D = packed->head_dim;
  if (!packed_is_planned(packed)) return PF_ERR_INVALID_ARG;
  if (!packed->work || ((uintptr_t)packed->work & 31u) || packed->work_bytes < packed_plan_bytes(packed->n_items, packed->n_kv_heads)) return PF_ERR_INVALID_ARG;
  if (!(softmax_scale >= 0.0f) || softmax_scale > 1.0e6f) return PF_ERR_INVALID_ARG;
  if (tq > 0 && (!q || !out)) return PF_ERR_INVALID_ARG;
  if (tk > 0 && (!k || !v)) return PF_ERR_INVALID_ARG;
  if (packed->prefix_tokens > 0 ? !k_prefix || !v_prefix : k_prefix || v_prefix) return PF_ERR_INVALID_ARG;
  if ((((uintptr_t)q) | ((uintptr_t)k) | ((uintptr_t)v) | ((uintptr_t)out) | ((uintptr_t)k_prefix) | ((uintptr_t)v_prefix) | ((uintptr_t)workspace)) & 15u)
    return PF_ERR_INVALID_ARG;
  if (!pf_chunk_layout_ok(q_layout, packed->n_heads, tq, D) || !pf_chunk_layout_ok(out_layout, packed->n_heads, tq, D) ||
      !pf_chunk_layout_ok(kv_layout, packed->n_kv_heads, tk, D) ||
      !pf_chunk_layout_ok(prefix_layout, packed->n_kv_heads, packed->prefix_tokens, D))
    return PF_ERR_INVALID_ARG;
  const size_t need = packed_part_bytes(packed, packed->n_planes, packed_head_rows(packed));
  if (need > 0 && (!workspace || workspace_bytes < need)) return PF_ERR_INVALID_ARG;
  if (tq == 0) return PF_OK;
  if (packed->planned_in != packed->work) return PF_ERR_INVALID_ARG;   // the plan stands in another buffer
  PackedParams P = {};
  P.q = (const __bf16 *)q;
  P.k = (const __bf16 *)k;
  P.v = (const __bf16 *)v;
  P.k_prefix = (const __bf16 *)k_prefix;
  P.v_prefix = (const __bf16 *)v_prefix;
  P.out = (__bf16 *)out;
  P.items = packed_items(packed);
  P.planned_for = packed->planned_for;
  P.n_rows = tq * packed->n_heads;
  P.n_heads = packed->n_heads;
  P.group = packed->n_heads / packed->n_kv_heads;
  P.block = packed->block;
  {
    // with 2^(s-1) < group <= 2^s and mul = ceil(2^(31+s) / group) < 2^32 the quotient is exact for n < 2^31: mul * group exceeds 2^(31+s) by
    // less than group <= 2^s, and n times that by less than 2^(31+s)
    int s = 0;
    while ((1 << s) < P.group) ++s;
    P.group_mul = (unsigned)(((1ull << (31 + s)) + P.group - 1) / P.group);
    P.group_shift = s > 0 ? s - 1 : 0;
  }
  P.planes = packed->n_planes;
  P.prefix_tokens = packed->prefix_tokens;
  P.prefix_tiles = pf_ceil_div(packed->prefix_tokens, PF_BK);
  if (P.planes > 0 && packed_by_arrival(packed)) P.arrivals = (int32_t *)(packed_items(packed) + packed->n_items);
  P.items_per_head = packed->n_items / packed->n_kv_heads;
  P.part_o = (float *)workspace;
  P.head_rows = packed_head_rows(packed);
  P.part_rows = P.head_rows * packed->n_kv_heads;
  P.part_ml = (float2 *)((char *)workspace + (size_t)P.planes * P.part_rows * D * 4);
  P.part_row = (int32_t *)(P.part_ml + (size_t)P.planes * P.part_rows);
  P.q_tok = q_layout ? q_layout->token_stride : D;
  P.q_head = q_layout ? q_layout->head_stride : (long long)tq * D;
  P.out_tok = out_layout ? out_layout->token_stride : D;
  P.out_head = out_layout ? out_layout->head_stride : (long long)tq * D;
  P.kv_tok = kv_layout ? kv_layout->token_stride : D;
  P.kv_head = kv_layout ? kv_layout->head_stride : (long long)tk * D;
  P.pre_tok = prefix_layout ? prefix_layout->token_stride : D;
  P.pre_head = prefix_layout ? prefix_layout->head_stride : (long long)packed->prefix_tokens * D;
  const float scale = softmax_scale > 0.0f ? softmax_scale : 1.0f / sqrtf((float)D);
  P.scale_log2 = scale * 1.4426950408889634f;
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid(packed->n_items), block(PACKED_WAVES * 64);
  if (packed->kernel == 1) hipLaunchKernelGGL(pf_packed_wide_kernel, grid, dim3(WIDE_WAVES * 64), 0, st, P);
  else if (D == 128) hipLaunchKernelGGL((pf_packed_attn_kernel<128>), grid, block, 0, st, P);
  else hipLaunchKernelGGL((pf_packed_attn_kernel<64>), grid, block, 0, st, P);
  PF_HIP_CHECK(hipGetLastError());
  if (P.planes > 0 && !P.arrivals) {
    const bool few = P.planes <= PACKED_FEW_PLANES;
    const dim3 rows((unsigned)pf_ceil_div(P.part_rows, few ? 256 / (D / 8) : 4));
    if (D == 128 && few) hipLaunchKernelGGL((pf_packed_join_few_kernel<128>), rows, block, 0, st, P);
    else if (D == 128) hipLaunchKernelGGL((pf_packed_join_kernel<128>), rows, block, 0, st, P);
    else if (few) hipLaunchKernelGGL((pf_packed_join_few_kernel<64>), rows, block, 0, st, P);
    else hipLaunchKernelGGL((pf_packed_join_kernel<64>), rows, block, 0, st, P);
    PF_HIP_CHECK(hipGetLastError());
  }
  return PF_OK;
}
