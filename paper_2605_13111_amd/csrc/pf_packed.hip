// Attention of packed sequences: whole prompts, causal by blocks, with grouped heads, alone or behind a prefix whose keys and values all
// sequences share (and that are read once for all of them).
//
//   out[i, h] = sum_j softmax_j(scale * q[i, h] . k[j, h / group]) v[j, h / group]
// over the prefix's keys and the keys j of i's own sequence with j / block <= p / block, p = i's place among those keys (the last query
// stands at the last key); a query that sees no key gets zeros.
//
// The rows of a key head are the queries of its group: row r of a sequence is query r / group of head kv_head * group + r % group, so that
// a group reads its keys and values once.  In front of the prefix all sequences' queries make one long line of rows.  A work item is a tile of
// rows against a run of key tiles: the host cuts the work into items and orders them (pf_packed_plan), heaviest first.  A row tile whose
// keys are cut into several items, or that has a prefix in front, parks unnormalised partial results (O, m, l) in fp32, one plane per
// item, row by row; a second kernel joins them in a fixed order.  A launch boundary stands between: no counters, no waiting.
//
// Scores, softmax and value products as in the ragged-cache kernels: S^T = K Q^T and O^T += V^T P^T on 32x32x16 bf16 MFMAs with fp32
// accumulation, one query row per lane; weights are rounded to bf16 for the second product (2^-8 relative at most each, the sum is
// taken in fp32 before that rounding).
#include <math.h>
#include <string.h>
#include <algorithm>
#include <new>
#include <vector>
#include "pf_packed_steps.h"

// ---- plan ------------------------------------------------------------------------------------------------------------

struct __attribute__((aligned(32))) PackedItem {
  int32_t q_base;      // first token of the line of rows (queries of one sequence, or of all of them in front of the prefix)
  int32_t row0;        // first row of the tile in that line
  int32_t n_rows;      // rows of the whole line
  int32_t k_base;      // token of the line's first key
  int32_t n_keys;      // keys of the line
  int32_t kt0, kt1;    // key tiles of this item
  int32_t head;        // key head | prefix flag << 12 | (plane + 1) << 13 (0: unsplit) | further planes without an item << 22
};
constexpr int PACKED_MAX_PLANES = 256;
constexpr int PACKED_PREFIX_BIT = 12;
PF_HD int packed_head(const PackedItem &it) { return it.head & 0xfff; }
PF_HD bool packed_is_prefix(const PackedItem &it) { return (it.head >> PACKED_PREFIX_BIT) & 1; }
PF_HD int packed_plane(const PackedItem &it) { return ((it.head >> 13) & 0x1ff) - 1; }
PF_HD int packed_missing(const PackedItem &it) { return (it.head >> 22) & 0x1ff; }

// Items reach the device as kernel arguments: the call neither allocates nor waits, and can be captured.
constexpr int PACKED_UPLOAD = 120;
struct PackedUpload {
  PackedItem item[PACKED_UPLOAD];
};
__global__ void pf_packed_upload_kernel(PackedUpload U, int n, PackedItem *to) {
  const int i = threadIdx.x;
  if (i < n) to[i] = U.item[i];
}

constexpr int PACKED_ROWS = 128;                                  // rows of an item: 4 waves x 32

struct PackedParams {
  const __bf16 *q, *k, *v, *k_prefix, *v_prefix;
  __bf16 *out;
  const PackedItem *items;
  float *part_o;                                                  // [planes][rows][D]
  float2 *part_ml;                                                // [planes][rows]: reference maximum, sum of weights; a sum of -1 in plane 0: the row is done
  long long q_tok, q_head, out_tok, out_head, kv_tok, kv_head, pre_tok, pre_head;    // element strides
  int n_rows, n_heads, group, block;                              // n_rows: tokens x heads
  int planes;
  float scale_log2;
};

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

// keys that row r of the item's line may see
__device__ __forceinline__ int packed_limit(const PackedParams &P, const PackedItem &it, int r) {
  if (packed_is_prefix(it) || P.block == 0) return it.n_keys;
  const int place = it.n_keys - it.n_rows / P.group + r / P.group;
  if (place < 0) return 0;
  // the last key of the row's block; the block's number and its end stay below 2^31 for any block size (a sequence has at most 2^30 keys)
  const unsigned number = (unsigned)place / (unsigned)P.block;
  return (int)min((unsigned)it.n_keys, number * (unsigned)P.block + (unsigned)P.block);
}

template <int D>
__global__ __launch_bounds__(256, D == 128 ? 2 : 4) void pf_packed_attn_kernel(PackedParams P) {
  typedef PackedTile<D> C;
  typedef __attribute__((address_space(3))) void *lptr_t;
  constexpr int WAVES = 4, WROWS = PF_BK / WAVES;                 // tile rows that one wave copies
  constexpr int NC = WROWS / C::COPY_ROWS;
  constexpr int SMEM = 2 * C::STAGE_BYTES > PACKED_ROWS * C::LD * 4 ? 2 * C::STAGE_BYTES : PACKED_ROWS * C::LD * 4;
  __shared__ __attribute__((aligned(1024))) char smem[SMEM];
  __shared__ float2 s_ml[PACKED_ROWS];
  const PackedItem it = P.items[blockIdx.x];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, g = lane >> 5;
  const bool prefix = packed_is_prefix(it);
  const int kvh = packed_head(it);
  const float c = P.scale_log2;
  const long long tok = prefix ? P.pre_tok : P.kv_tok;
  const long long k0 = (long long)(it.k_base + it.kt0 * PF_BK) * tok + kvh * (prefix ? P.pre_head : P.kv_head);
  const __bf16 *kb = (prefix ? P.k_prefix : P.k) + k0, *vb = (prefix ? P.v_prefix : P.v) + k0;
  const int key0 = it.kt0 * PF_BK, n_tiles = it.kt1 - it.kt0;
  const unsigned rb = (unsigned)(tok * 2);                        // bytes between key rows (below 2^25: checked on the host)

  // this lane's query row
  const int wrow0 = it.row0 + wave * 32;
  const bool has_rows = wrow0 < it.n_rows;
  const int row = pf_min(wrow0 + l32, it.n_rows - 1);
  const int limit = packed_limit(P, it, row);
  const int lim_first = __builtin_amdgcn_readlane(limit, 0), lim_last = __builtin_amdgcn_readlane(limit, 31);

  const int rr = lane / C::CHUNKS, p = lane % C::CHUNKS;
  const unsigned low_k = (unsigned)((p ^ C::swz_k(rr)) << 4), low_v = (unsigned)((p ^ C::swz_v(rr)) << 4);
  char *const mine = smem + wave * (WROWS * C::ROW_BYTES);
  auto copy_tile = [&](int u) __attribute__((always_inline)) {
    if (u >= n_tiles) return;
    char *to = mine + (u & 1) * C::STAGE_BYTES;
    const long long e = (long long)u * PF_BK * tok;
    const __amdgpu_buffer_rsrc_t rk = __builtin_amdgcn_make_buffer_rsrc((void *)(kb + e), 0, -1, 0x00020000u);
    const __amdgpu_buffer_rsrc_t rv = __builtin_amdgcn_make_buffer_rsrc((void *)(vb + e), 0, -1, 0x00020000u);
    const int last = it.n_keys - 1 - key0 - u * PF_BK;            // rows past the sequence's end repeat its last key
    static_for<0, NC>([&](auto gi) {
      constexpr int G = decltype(gi)::value;
      const unsigned at = (unsigned)pf_min(wave * WROWS + G * C::COPY_ROWS + rr, last) * rb;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rk, (lptr_t)(to + G * 1024), 16, at + (low_k ^ (unsigned)(C::swz_k(G * C::COPY_ROWS) << 4)), 0, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rv, (lptr_t)(to + C::TENSOR_BYTES + G * 1024), 16, at + (low_v ^ (unsigned)(C::swz_v(G * C::COPY_ROWS) << 4)), 0, 0, 0);
    });
  };
  copy_tile(0);

  bf16x8 qf[C::NKS];
  const int qt = it.q_base + row / P.group, qh = kvh * P.group + row % P.group;
  {
    const __bf16 *q = P.q + (long long)qt * P.q_tok + (long long)qh * P.q_head + 8 * g;
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) qf[ks] = *(const bf16x8 *)(q + ks * 16);
#pragma unroll
    for (int ks = 0; ks < C::NKS; ++ks) asm volatile("" : "+v"(qf[ks]));   // the compiler waits here, not inside the loop
  }
  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
  // The reference maximum starts below every score; its multiple is kept finite, so that a masked key's weight against it is 0 and not NaN
  float m_run = -3.0e38f, l_run = 0.0f, mc = fmaxf(m_run * c, -3.0e38f);
  const unsigned lds0 = (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char *)smem;
  const unsigned ak = lds0 + l32 * C::ROW_BYTES + ((g ^ C::swz_k(l32)) << 4);
  unsigned av;
  {
    const int rowv = 4 * g + ((lane & 15) >> 2);
    const int c0 = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    av = lds0 + C::TENSOR_BYTES + rowv * C::ROW_BYTES + ((c0 ^ C::swz_v(rowv)) << 4) + 8 * (lane & 1);
  }
  for (int u = 0; u < n_tiles; ++u) {
    const unsigned stage = (u & 1) * C::STAGE_BYTES;
    wait_vm<0>();                                            // this wave's share of tile u has landed
    __builtin_amdgcn_s_barrier();                                 // ... everyone's has, and everyone is done with tile u-1
    copy_tile(u + 1);
    const int t0 = key0 + u * PF_BK;
    if (!has_rows || t0 >= lim_last) continue;                    // none of this wave's rows sees the tile
    // ---- S^T = K Q^T: fragment 2 ks + kb = key block kb, k-step ks, four ahead ----
    f32x16 s[2];
    {
      u32x4 kf[2 * C::NKS];
      auto kread = [&](auto i) {
        constexpr int I = decltype(i)::value, KB = I & 1, KSTEP = I >> 1;
        read_k<KB * 32 * C::ROW_BYTES>(kf[I], (ak + stage) ^ (unsigned)(KSTEP << 5));
      };
      static_for<0, 4>([&](auto i) { kread(i); });
      static_for<0, 2 * C::NKS>([&](auto i) {
        constexpr int I = decltype(i)::value, KB = I & 1, KSTEP = I >> 1, N = 2 * C::NKS;
        wait_lds<(I + 3 < N - 1 ? 3 : N - 1 - I)>();
        const f32x16 zero = {};
        s[KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[I]), qf[KSTEP], KSTEP == 0 ? zero : s[KB], 0, 0, 0);
        if constexpr (I + 4 < N) kread(IntC<I + 4>());
        __builtin_amdgcn_sched_barrier(0);
      });
    }
    if (__builtin_expect(lim_first - t0 < PF_BK, 0)) {            // some row does not see the whole tile
      int g_l = g;
      asm volatile("" : "+v"(g_l));                               // its per-lane constants are not held in registers through the loop
      const int valid = limit - t0;
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (kb2 * 32 + 8 * (i >> 2) + 4 * g_l + (i & 3) >= valid) s[kb2][i] = -INFINITY;
    }
    // ---- online softmax, one query row per lane ----
    bf16x8 pf[4];
    float ts[2];
    auto weights = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
          const float e0 = fast_exp2(fmaf(s[kb2][i], c, -mc)), e1 = fast_exp2(fmaf(s[kb2][i + 1], c, -mc));
          ts[0] = kb2 + i == 0 ? e0 : ts[0] + e0;
          ts[1] = kb2 + i == 0 ? e1 : ts[1] + e1;
          pf[kb2 * 2 + (i >> 3)][i & 7] = (__bf16)e0;
          pf[kb2 * 2 + (i >> 3)][(i & 7) + 1] = (__bf16)e1;
        }
    };
    weights();
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(pf[i]));   // rounded here: sunk past the branch, all 32 weights would stay in registers
    if (__builtin_expect(tile_sum_too_large(ts[0] + ts[1]), 0)) {
      float mx = s[0][0];
#pragma unroll
      for (int kb2 = 0; kb2 < 2; ++kb2)
#pragma unroll
        for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[kb2][i]);
      // only rows that need it move, so that no row's bits depend on what its neighbours hold
      const float over = partner_max(ts[0] + ts[1] <= PACKED_MAX_TILE_SUM ? 0.0f : 1.0f);
      const float m_new = over > 0.0f ? fmaxf(m_run, partner_max(mx)) : m_run;
      const float alpha = fast_exp2((m_run - m_new) * c);
      m_run = m_new;
      mc = fmaxf(m_new * c, -3.0e38f);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < C::NDB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= alpha;
      weights();
    }
    l_run += ts[0] + ts[1];
    // ---- O^T += V^T P^T: fragment s16 * NDB + db = 16 keys, channel block db (two transpose reads each), four ahead ----
    {
      constexpr int N = 4 * C::NDB;
      u32x2 vl[N], vh[N];
      auto vread = [&](auto i) {
        constexpr int I = decltype(i)::value, OFF = (I / C::NDB) * 16 * C::ROW_BYTES;
        const unsigned a = (av + stage) ^ (unsigned)((I % C::NDB) << 6);
        read_vt<OFF>(vl[I], a);
        read_vt<OFF + 8 * C::ROW_BYTES>(vh[I], a);
      };
      static_for<0, 4>([&](auto i) { vread(i); });
      static_for<0, N>([&](auto i) {
        constexpr int I = decltype(i)::value;
        wait_lds<2 * (I + 3 < N - 1 ? 3 : N - 1 - I)>();
        const u32x4 a4 = __builtin_shufflevector(vl[I], vh[I], 0, 1, 2, 3);
        o[I % C::NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a4), pf[I / C::NDB], o[I % C::NDB], 0, 0, 0);
        if constexpr (I + 4 < N) vread(IntC<I + 4>());
        __builtin_amdgcn_sched_barrier(0);
      });
    }
  }
  __syncthreads();
  // ---- result rows through LDS, so that they are written as full rows ----
  float *sO = (float *)smem;
  const float lsum = partner_sum(l_run);
#pragma unroll
  for (int db = 0; db < C::NDB; ++db)
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4)
      *(f32x4 *)(sO + (wave * 32 + l32) * C::LD + db * 32 + 8 * i4 + 4 * g) = f32x4{o[db][i4 * 4], o[db][i4 * 4 + 1], o[db][i4 * 4 + 2], o[db][i4 * 4 + 3]};
  if (g == 0) s_ml[wave * 32 + l32] = make_float2(m_run, lsum);
  __syncthreads();
  const int plane = packed_plane(it), n_valid = pf_min(PACKED_ROWS, it.n_rows - it.row0);
  for (int e = tid; e < n_valid * (D / 8); e += 256) {
    const int r = e / (D / 8), d0 = (e % (D / 8)) * 8;
    const int lr = it.row0 + r, t = it.q_base + lr / P.group, h = kvh * P.group + lr % P.group;
    const f32x4 a = *(const f32x4 *)(sO + r * C::LD + d0), b = *(const f32x4 *)(sO + r * C::LD + d0 + 4);
    const float2 ml = s_ml[r];
    const long long id = (long long)t * P.n_heads + h;
    if (plane >= 0) {
      float *po = P.part_o + ((long long)plane * P.n_rows + id) * D + d0;
      *(f32x4 *)po = a;
      *(f32x4 *)(po + 4) = b;
      if (d0 == 0) {
        P.part_ml[(long long)plane * P.n_rows + id] = ml;
        for (int i = 1; i <= packed_missing(it); ++i) P.part_ml[(long long)(plane + i) * P.n_rows + id] = make_float2(-3.0e38f, 0.0f);
      }
    } else {
      const float inv = ml.y > 0.0f ? 1.0f / ml.y : ml.y;         // no key seen: zeros (a sum that is NaN stays NaN)
      bf16x8 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = (__bf16)(a[i] * inv), w[i + 4] = (__bf16)(b[i] * inv);
      *(bf16x8 *)(P.out + (long long)t * P.out_tok + (long long)h * P.out_head + d0) = w;
      if (P.planes > 0 && d0 == 0) P.part_ml[id] = make_float2(0.0f, -1.0f);
    }
  }
}

// Joins the planes of every row: out = sum_p 2^((m_p - M) c) O_p / sum_p 2^((m_p - M) c) l_p, planes in order.
template <int D>
__global__ __launch_bounds__(256) void pf_packed_join_kernel(PackedParams P) {
  constexpr int LANES = D / 8;                                    // of a row, eight channels each
  const long long id = (long long)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
  if (id >= P.n_rows) return;
  const int d0 = threadIdx.x % LANES * 8;
  const float2 first = P.part_ml[id];
  if (first.y == -1.0f) return;                                   // written by its only item
  float top = first.x;
  for (int p = 1; p < P.planes; ++p) top = fmaxf(top, P.part_ml[(long long)p * P.n_rows + id].x);
  float acc[8] = {}, sum = 0.0f;
  for (int p = 0; p < P.planes; ++p) {
    const float2 ml = P.part_ml[(long long)p * P.n_rows + id];
    if (ml.y == 0.0f) continue;                                   // saw no key (nothing was written for a plane without an item)
    const float w = fast_exp2((ml.x - top) * P.scale_log2);
    sum += w * ml.y;
    const float *o = P.part_o + ((long long)p * P.n_rows + id) * D + d0;
    const f32x4 a = *(const f32x4 *)o, b = *(const f32x4 *)(o + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += w * a[i], acc[i + 4] += w * b[i];
  }
  const float inv = sum > 0.0f ? 1.0f / sum : sum;
  bf16x8 w;
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = (__bf16)(acc[i] * inv);
  *(bf16x8 *)(P.out + id / P.n_heads * P.out_tok + id % P.n_heads * P.out_head + d0) = w;
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

struct PackedPlan {
  std::vector<PackedItem> items;
  int planes = 0;
};

// Key tiles per item: where whole row tiles are fewer than the places that workgroups find on the chip, their keys are cut until about as
// many items are there.
static constexpr int PACKED_PLACES = 512, PACKED_MIN_SEG = 8;

static void packed_cut(PackedPlan &plan, PackedItem it, int n_kt, int seg, int first_plane, int planes_of_line, bool alone) {
  const int n = std::max(1, pf_ceil_div(n_kt, seg));
  for (int i = 0; i < n; ++i) {
    PackedItem x = it;
    x.kt0 = pf_seg_begin(n_kt, n, i);
    x.kt1 = pf_seg_begin(n_kt, n, i + 1);
    if (!(alone && n == 1)) {
      x.head |= (first_plane + i + 1) << 13;
      if (i == n - 1) x.head |= (planes_of_line - n) << 22;
    }
    plan.items.push_back(x);
  }
}

static void packed_make(const pf_packed *p, PackedPlan &plan) {
  const int G = p->n_heads / p->n_kv_heads, KV = p->n_kv_heads, BQ = PACKED_ROWS;
  const long long total_rows = (long long)p->cu_q[p->n_seqs] * G;
  const int pre_kt = pf_ceil_div(p->prefix_tokens, PF_BK);
  // the work in key tiles, the longest line
  long long work = (total_rows + BQ - 1) / BQ * pre_kt, longest = pre_kt;
  for (int s = 0; s < p->n_seqs; ++s) {
    const int lq = p->cu_q[s + 1] - p->cu_q[s], lk = p->cu_k[s + 1] - p->cu_k[s];
    const long long rows = (long long)lq * G;
    for (long long r0 = 0; r0 < rows; r0 += BQ)
      work += pf_ceil_div(packed_host_limit(p, lq, lk, (int)((std::min(r0 + BQ, rows) - 1) / G)), PF_BK);
    longest = std::max<long long>(longest, pf_ceil_div(lk, PF_BK));
  }
  work *= KV;
  const int seg = (int)std::max<long long>(std::max<long long>(PACKED_MIN_SEG, (work + PACKED_PLACES - 1) / PACKED_PLACES), (longest + 120) / 120);
  const int pre_planes = pre_kt ? pf_ceil_div(pre_kt, seg) : 0;
  int own_planes = 0;
  for (int s = 0; s < p->n_seqs; ++s) {
    const int lq = p->cu_q[s + 1] - p->cu_q[s], lk = p->cu_k[s + 1] - p->cu_k[s];
    if (lq > 0) own_planes = std::max(std::max(own_planes, 1), pf_ceil_div(pf_ceil_div(packed_host_limit(p, lq, lk, lq - 1), PF_BK), seg));
  }
  if (pre_planes == 0 && own_planes <= 1) own_planes = 0;
  plan.planes = pre_planes + own_planes;
  for (long long r0 = 0; pre_kt && r0 < total_rows; r0 += BQ)
    for (int h = 0; h < KV; ++h) {
      const PackedItem it = {0, (int)r0, (int)total_rows, 0, p->prefix_tokens, 0, 0, h | 1 << PACKED_PREFIX_BIT};
      packed_cut(plan, it, pre_kt, seg, 0, pre_planes, false);
    }
  for (int s = 0; s < p->n_seqs; ++s) {
    const int lq = p->cu_q[s + 1] - p->cu_q[s], lk = p->cu_k[s + 1] - p->cu_k[s];
    const int rows = lq * G;
    for (int r0 = 0; r0 < rows; r0 += BQ) {
      const int n_kt = pf_ceil_div(packed_host_limit(p, lq, lk, (pf_min(r0 + BQ, rows) - 1) / G), PF_BK);
      for (int h = 0; h < KV; ++h) {
        const PackedItem it = {p->cu_q[s], r0, rows, p->cu_k[s], lk, 0, 0, h};
        packed_cut(plan, it, n_kt, seg, pre_planes, own_planes, pre_planes == 0);
      }
    }
  }
  std::stable_sort(plan.items.begin(), plan.items.end(), [](const PackedItem &a, const PackedItem &b) { return a.kt1 - a.kt0 > b.kt1 - b.kt0; });
}

static size_t packed_part_bytes(const pf_packed *p, int planes) {
  return (size_t)planes * p->cu_q[p->n_seqs] * p->n_heads * ((size_t)p->head_dim * 4 + 8);
}

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
  size_t n = 0;
  packed_guard([&]() {
    const int rc = packed_check(packed);
    if (rc != PF_OK) return rc;
    PackedPlan plan;
    packed_make(packed, plan);
    n = std::max<size_t>(1, plan.items.size()) * sizeof(PackedItem);
    return PF_OK;
  });
  return n;
}

extern "C" int pf_packed_plan(pf_packed *packed, void *stream) {
  return packed_guard([&]() {
    const int rc = packed_check(packed);
    if (rc != PF_OK) return rc;
    if (!packed->work || ((uintptr_t)packed->work & 31u)) return (int)PF_ERR_INVALID_ARG;
    PackedPlan plan;
    packed_make(packed, plan);
    if (packed->work_bytes < std::max<size_t>(1, plan.items.size()) * sizeof(PackedItem)) return (int)PF_ERR_CAPACITY;
    PackedItem *to = (PackedItem *)packed->work;
    for (size_t i = 0; i < plan.items.size(); i += PACKED_UPLOAD) {
      PackedUpload U;
      const int n = (int)std::min<size_t>(PACKED_UPLOAD, plan.items.size() - i);
      memcpy(U.item, &plan.items[i], n * sizeof(PackedItem));
      if (n < PACKED_UPLOAD) memset(U.item + n, 0, (PACKED_UPLOAD - n) * sizeof(PackedItem));
      hipLaunchKernelGGL(pf_packed_upload_kernel, dim3(1), dim3(128), 0, (hipStream_t)stream, U, n, to + i);
      PF_HIP_CHECK(hipGetLastError());
    }
    packed->n_items = (int32_t)plan.items.size();
    packed->n_planes = plan.planes;
    packed->total_q = packed->cu_q[packed->n_seqs];
    packed->total_k = packed->cu_k[packed->n_seqs];
    return (int)PF_OK;
  });
}

extern "C" size_t pf_packed_workspace_bytes(const pf_packed *packed) {
  if (packed_check(packed) != PF_OK || packed->n_planes < 0 || packed->n_planes > PACKED_MAX_PLANES) return 0;
  return pf_align_up(packed_part_bytes(packed, packed->n_planes) + 256, 256);
}

extern "C" int pf_packed_attn_fwd(const pf_packed *packed, const void *q, const pf_chunk_layout *q_layout, const void *k, const void *v,
                                  const pf_chunk_layout *kv_layout, const void *k_prefix, const void *v_prefix,
                                  const pf_chunk_layout *prefix_layout, void *out, const pf_chunk_layout *out_layout,
                                  float softmax_scale, void *workspace, size_t workspace_bytes, void *stream) {
  const int rc = packed_check(packed);
  if (rc != PF_OK) return rc;
  const int tq = packed->cu_q[packed->n_seqs], tk = packed->cu_k[packed->n_seqs], D = packed->head_dim;
  if (packed->n_items < 0 || packed->n_planes < 0 || packed->n_planes > PACKED_MAX_PLANES || packed->total_q != tq || packed->total_k != tk)
    return PF_ERR_INVALID_ARG;                                    // not planned, or planned for other lengths
  if (tq > 0 && packed->n_items == 0) return PF_ERR_INVALID_ARG;
  if (!packed->work || ((uintptr_t)packed->work & 31u) || packed->work_bytes < (size_t)packed->n_items * sizeof(PackedItem)) return PF_ERR_INVALID_ARG;
  if (!(softmax_scale >= 0.0f) || softmax_scale > 1.0e6f) return PF_ERR_INVALID_ARG;
  if (tq > 0 && (!q || !out)) return PF_ERR_INVALID_ARG;
  if (tk > 0 && (!k || !v)) return PF_ERR_INVALID_ARG;
  if (packed->prefix_tokens > 0 && (!k_prefix || !v_prefix)) return PF_ERR_INVALID_ARG;
  if ((((uintptr_t)q) | ((uintptr_t)k) | ((uintptr_t)v) | ((uintptr_t)out) | ((uintptr_t)k_prefix) | ((uintptr_t)v_prefix) | ((uintptr_t)workspace)) & 15u)
    return PF_ERR_INVALID_ARG;
  if (!pf_chunk_layout_ok(q_layout, packed->n_heads, tq, D) || !pf_chunk_layout_ok(out_layout, packed->n_heads, tq, D) ||
      !pf_chunk_layout_ok(kv_layout, packed->n_kv_heads, tk, D) ||
      !pf_chunk_layout_ok(prefix_layout, packed->n_kv_heads, packed->prefix_tokens, D))
    return PF_ERR_INVALID_ARG;
  const size_t need = packed_part_bytes(packed, packed->n_planes);
  if (need > 0 && (!workspace || workspace_bytes < need)) return PF_ERR_INVALID_ARG;
  if (tq == 0) return PF_OK;
  PackedParams P = {};
  P.q = (const __bf16 *)q;
  P.k = (const __bf16 *)k;
  P.v = (const __bf16 *)v;
  P.k_prefix = (const __bf16 *)k_prefix;
  P.v_prefix = (const __bf16 *)v_prefix;
  P.out = (__bf16 *)out;
  P.items = (const PackedItem *)packed->work;
  P.n_rows = tq * packed->n_heads;
  P.n_heads = packed->n_heads;
  P.group = packed->n_heads / packed->n_kv_heads;
  P.block = packed->block;
  P.planes = packed->n_planes;
  P.part_o = (float *)workspace;
  P.part_ml = (float2 *)((char *)workspace + (size_t)P.planes * P.n_rows * D * 4);
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
  if (D == 128) hipLaunchKernelGGL((pf_packed_attn_kernel<128>), dim3(packed->n_items), dim3(256), 0, st, P);
  else hipLaunchKernelGGL((pf_packed_attn_kernel<64>), dim3(packed->n_items), dim3(256), 0, st, P);
  PF_HIP_CHECK(hipGetLastError());
  if (P.planes > 0) {
    const int rows = 256 / (D / 8);
    const dim3 grid((unsigned)((P.n_rows + rows - 1) / rows));
    if (D == 128) hipLaunchKernelGGL((pf_packed_join_kernel<128>), grid, dim3(256), 0, st, P);
    else hipLaunchKernelGGL((pf_packed_join_kernel<64>), grid, dim3(256), 0, st, P);
    PF_HIP_CHECK(hipGetLastError());
  }
  return PF_OK;
}
