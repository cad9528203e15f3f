// Wide items of the packed attention, head_dim 128: 256 rows, 8 waves x 32, one workgroup per compute unit.  Included by pf_packed.hip (whose
// copies, masks, softmax and results it shares).
//
// Waves w and w + 4 share a SIMD; they belong to two groups, and group 1 runs one phase behind group 0, so that while one wave of a SIMD
// issues the 32 MFMAs of a tile (O^T += V^T P^T of the tile before, then S^T = K Q^T of this one) the other works its softmax out on the
// vector ALU.  A barrier ends every phase:
//   matrix phase u   reads K of tile u and V of tile u - 1, requests the first V^T fragments of tile u for the next matrix phase, waits for this
//                    wave's copies of tile u + 1; its barrier stands in front of the last MFMA
//   vector phase u   sends the copies of tile u + 3 to where tiles u - 1 (K) and u - 2 (V) were (their last readers, both groups' matrix phases
//                    u - 1, are two barriers back), then scores of tile u -> weights
// Bound: both kinds of phase (1260 cycles of the 992 that 31 MFMAs take: vector instructions of the other wave hold their issue up; 960 of
// weights and 255 of copies), at the clock that the power leaves (1.7 GHz).  A prompt of 14040 tokens of 12 heads takes 666 to 712 us from card to
// card (1210 to 1130 TFLOP/s); as 128-row items, two workgroups per compute unit, it took 741 when this form took 695: there a key tile is copied
// into LDS twice for 256 rows, and the matrix pipe waits for softmaxes.  Not better, each measured on that prompt at 700: copies sent between the MFMAs (744), the barrier 3, 4 or 6 MFMAs early (757, 764,
// 782; 2: the same), matrix phases without priority (713).  Workgroups that stay resident and take items, with the copies of the next one under
// way: 740 from lists made beforehand (the dies do not run at one speed), 713 by tickets.
#ifndef PF_PACKED_WIDE_H
#define PF_PACKED_WIDE_H

constexpr int WIDE_WAVES = 8;
constexpr int WIDE_KSTAGES = 4;                                   // K of tile u is read in matrix phase u
constexpr int WIDE_VSTAGES = 5;                                   // V of tile u is read one phase later
constexpr int WIDE_TILE = PF_BK * 256;                            // bytes of one tensor's tile
constexpr int WIDE_RING = 5;                                      // fragments requested ahead of their MFMA
constexpr int WIDE_EARLY = 1;                                     // MFMAs of a matrix phase behind its barrier
static_assert(PACKED_WIDE_ROWS == 32 * WIDE_WAVES, "a wave's rows");
// LDS reads that fragments i + 1 .. last of a matrix phase take: V^T fragments (0 .. 15, and from 32 on the next tile's) two, K one
constexpr int wide_reads_between(int i, int last) {
  int n = 0;
  for (int j = i + 1; j <= last; ++j) n += j >= 16 && j < 32 ? 1 : 2;
  return n;
}

__device__ __forceinline__ void packed_wide(const PackedItem &it, char *smem, int tid) {
  constexpr int D = 128;
  typedef PackedTile<D> C;
  typedef __attribute__((address_space(3))) void *lptr_t;
  constexpr int WROWS = PF_BK / WIDE_WAVES, NC = WROWS / C::COPY_ROWS;   // tile rows that one wave copies, in so many copies a tensor
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), grp = wave >> 2;
  const int l32 = lane & 31, g = lane >> 5, n_tiles = it.kt1 - it.kt0;
  const int wrow0 = it.row0 + wave * 32;
  char *const ring_k = smem + wave * (WROWS * C::ROW_BYTES), *const ring_v = ring_k + WIDE_KSTAGES * WIDE_TILE;
  // where its queries are staged: what K of tiles 2 and 3 and V of tiles 3 and 4 will take
  char *const stage_q = smem + (wave < 4 ? 2 * WIDE_TILE : (WIDE_KSTAGES + 1) * WIDE_TILE) + wave * (32 * C::ROW_BYTES);
  static_assert(WIDE_WAVES == 8 && WIDE_KSTAGES == 4 && WIDE_VSTAGES == 5, "two stages of K and of V hold four waves' queries each");
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
  asm volatile("" : "+v"(R.m), "+v"(R.mc));                       // worked out here (put off by the compiler a prompt of 14040 tokens took 700 us, so 696)
  // ---- copies, by runs of whole tiles (see packed_full) ----
  __amdgpu_buffer_rsrc_t run_k = __builtin_amdgcn_make_buffer_rsrc(nullptr, 0, 0, 0x00020000u), run_v = run_k;
  unsigned run_soff = 0, run_tile = 0, run_group = 0, run_vk[NC], run_vv = 0;
  int run_n = 0;                                                  // tiles left in the run
  asm volatile("" : "+s"(run_soff), "+s"(run_tile), "+s"(run_group), "+s"(run_n));   // scalars from the start
#pragma unroll
  for (int i = 0; i < NC; ++i) run_vk[i] = 0;
  // tile u of the item, K to ring offset dk and V to dv; settle: fragment reads that are in flight have landed (the compiler takes their
  // registers as written, and on the rare path, which needs many, it may move them)
  auto copy_tile = [&](int u, unsigned dk, unsigned dv, auto settle) __attribute__((always_inline)) {
    if (__builtin_expect(run_n <= 0, 0)) {
      if (u >= n_tiles) return;
      settle();
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
        packed_copy<D, false, WROWS>(P, it, K, kt, wave * WROWS, ring_k + dk, lane_l);
        packed_copy<D, true, WROWS>(P, it, K, kt, wave * WROWS, ring_v + dv, lane_l);
        return;
      }
      const unsigned rb = (unsigned)(tok * 2);
      run_tile = PF_BK * rb;
      run_n = __builtin_amdgcn_readfirstlane(pf_min(pf_min(whole, n_tiles - u), 1 << (__builtin_clz(run_tile) - 1)));   // offsets stay below 2^31
      run_soff = 0;
      run_group = C::COPY_ROWS * rb;
      const long long e = (long long)(key0 + wave * WROWS) * tok;
      run_k = __builtin_amdgcn_make_buffer_rsrc((void *)((in_prefix ? K.k_pre : K.k) + e), 0, -1, 0x00020000u);
      run_v = __builtin_amdgcn_make_buffer_rsrc((void *)((in_prefix ? K.v_pre : K.v) + e), 0, -1, 0x00020000u);
      const int rr = lane_l / C::CHUNKS, p = lane_l % C::CHUNKS;
#pragma unroll
      for (int i = 0; i < NC; ++i) run_vk[i] = (unsigned)((p ^ C::swz_k(rr) ^ C::swz_k(i * C::COPY_ROWS) ^ C::swz_k(wave * WROWS & 15)) << 4) + (unsigned)rr * rb;
      run_vv = (unsigned)((p ^ C::swz_v(rr)) << 4) + (unsigned)rr * rb;
    }
    --run_n;
    static_for<0, NC>([&](auto gi) {
      constexpr int G = decltype(gi)::value;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(run_k, (lptr_t)(ring_k + dk + G * 1024), 16, run_vk[G], run_soff + G * run_group, 0, 0);
      __builtin_amdgcn_raw_ptr_buffer_load_lds(run_v, (lptr_t)(ring_v + dv + G * 1024), 16, run_vv, run_soff + G * run_group, 0, 0);
    });
    run_soff += run_tile;
  };
  // the copies of every vector phase but the last have landed: a phase sends one tile's, or none behind the item's end
  auto wait_copies = [&](int u) __attribute__((always_inline)) {
    if (__builtin_expect(u < n_tiles, 1)) wait_vm<2 * NC>();
    else wait_vm<0>();
  };
#pragma unroll 1
  for (int i = 0; i < 3; ++i) {
    if (i == 2) {                                                 // some of its place holds queries until here
      if (n_tiles > 1) wait_vm<2 * NC>();                         // queries and the first tile have landed
      else wait_vm<0>();
      packed_read_q<D>(stage_q, lane, qf);
      __builtin_amdgcn_s_barrier();
    }
    copy_tile(i, i * WIDE_TILE, i * WIDE_TILE, []() {});
  }

  // the limit grows with the row: the wave's first lane has the least, its 32nd the most.  A wave computes its tiles up to the last that one of
  // its rows sees; behind it it sends its copies and meets the barriers, and does nothing else.
  const int lim_first = __builtin_amdgcn_readlane(limit, 0), lim_last = __builtin_amdgcn_readlane(limit, 31);
  const int mine = wrow0 < it.n_rows ? pf_max(0, pf_min(n_tiles, pre + pf_ceil_div(lim_last, PF_BK) - it.kt0)) : 0;
  f32x16 o[C::NDB];
#pragma unroll
  for (int db = 0; db < C::NDB; ++db)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[db][i] = 0.0f;
  unsigned ak, av;
  packed_lds<D>(smem, smem + WIDE_KSTAGES * WIDE_TILE, lane, ak, av);
  if (grp == 1) __builtin_amdgcn_s_barrier();                     // group 1 trails by one phase

  // ---- a matrix phase consumes 32 operand fragments from LDS, one per MFMA:
  //   0..15   V^T of the tile before: 16-key group i / 4, channel block i % 4 (two 8-byte transpose reads)
  //   16..31  K of this tile: key block (i - 16) % 2, k-step (i - 16) / 2 (one 16-byte read)
  // requested WIDE_RING ahead (at most 15 LDS reads of a wave may be in flight) and waited for with counted waits ----
  f32x16 s[2];
  bf16x8 pf[4];
  u32x2 vl[16], vh[16];
  u32x4 kf[16];
  auto m_phase = [&](auto has_pv, auto has_qk, unsigned off_k, unsigned off_v, unsigned off_v_next, auto end) __attribute__((always_inline)) {
    constexpr bool PV = decltype(has_pv)::value != 0, QK = decltype(has_qk)::value != 0;
    constexpr int FIRST = PV ? 0 : 16, LAST = QK ? 31 : 15, LAST_SENT = QK ? LAST + WIDE_RING : LAST;
    auto request = [&](auto f) __attribute__((always_inline)) {
      constexpr int F = decltype(f)::value, I = F > LAST ? F - LAST - 1 : F;
      if constexpr (I < 16) {
        const unsigned a = (av + (F > LAST ? off_v_next : off_v)) ^ (unsigned)((I % 4) << 6);
        read_vt<(I / 4) * 16 * C::ROW_BYTES>(vl[I], a);
        read_vt<(I / 4) * 16 * C::ROW_BYTES + 8 * C::ROW_BYTES>(vh[I], a);
      } else {
        constexpr int J = I - 16;
        read_k<(J & 1) * 32 * C::ROW_BYTES>(kf[J], (ak + off_k) ^ (unsigned)((J >> 1) << 5));
      }
    };
    __builtin_amdgcn_s_setprio(3);                                // the matrix phase goes first on its SIMD
    if constexpr (!PV) static_for<16, 16 + WIDE_RING>([&](auto f) { request(f); });
    static_for<FIRST, LAST + 1>([&](auto f) {
      constexpr int I = decltype(f)::value;
      constexpr int NEWEST = I + WIDE_RING - 1 < LAST_SENT ? I + WIDE_RING - 1 : LAST_SENT;
      wait_lds<wide_reads_between(I, NEWEST)>();
      if constexpr (I < 16) {
        const u32x4 a4 = __builtin_shufflevector(vl[I], vh[I], 0, 1, 2, 3);
        o[I % 4] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a4), pf[I / 4], o[I % 4], 0, 0, 0);
      } else {
        constexpr int J = I - 16, KB = J & 1, KSTEP = J >> 1;
        const f32x16 zero = {};
        s[KB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[J]), qf[KSTEP], KSTEP == 0 ? zero : s[KB], 0, 0, 0);
      }
      if constexpr (I + WIDE_RING <= LAST_SENT) request(IntC<I + WIDE_RING>());
      __builtin_amdgcn_sched_barrier(0);                          // keep the hand-made order: wait, MFMA, next request
      if constexpr (I == LAST - WIDE_EARLY) {
        end();
        __builtin_amdgcn_sched_barrier(0);
      }
    });
    __builtin_amdgcn_s_setprio(0);
  };
  auto settle = [&]() __attribute__((always_inline)) {
    asm volatile("s_waitcnt lgkmcnt(0)" : "+v"(vl[0]), "+v"(vh[0]), "+v"(vl[1]), "+v"(vh[1]), "+v"(vl[2]), "+v"(vh[2]), "+v"(vl[3]), "+v"(vh[3]), "+v"(vl[4]), "+v"(vh[4]));
  };
  static_assert(WIDE_RING == 5, "settle names the fragments in flight");
  auto weights = [&](int u, bool first) __attribute__((always_inline)) {
    const int kt = it.kt0 + u, t0 = (kt < pre ? kt : kt - pre) * PF_BK;
    if (__builtin_expect((kt < pre ? prefix_tokens : lim_first) - t0 < PF_BK, 0))   // some row does not see the whole tile
      packed_mask<2>(s, (kt < pre ? prefix_tokens : limit) - t0, g);
    packed_softmax<D, 2>(s, pf, o, R, c, first);
  };
  // ring offsets of tile u (ok, ov) and of the V tiles before it (ov1, ov2)
  unsigned ok = 0, ov = 0, ov1 = (WIDE_VSTAGES - 1) * WIDE_TILE, ov2 = (WIDE_VSTAGES - 2) * WIDE_TILE;
  auto rings_on = [&]() __attribute__((always_inline)) {
    ok = (ok + WIDE_TILE) & (WIDE_KSTAGES * WIDE_TILE - 1);
    ov2 = ov1;
    ov1 = ov;
    ov = ov + WIDE_TILE == WIDE_VSTAGES * WIDE_TILE ? 0 : ov + WIDE_TILE;
  };
  auto copy_next = [&](int u, auto settle) __attribute__((always_inline)) {
    copy_tile(u + 3, (ok + 3 * WIDE_TILE) & (WIDE_KSTAGES * WIDE_TILE - 1), ov2, settle);
  };
  int u = 1;
  if (__builtin_expect(mine > 0, 1)) {
    m_phase(IntC<0>(), IntC<1>(), 0, 0, 0, [&]() __attribute__((always_inline)) {
      wait_copies(2);
      __builtin_amdgcn_s_barrier();
    });
    copy_next(0, settle);
    weights(0, true);
    __builtin_amdgcn_s_barrier();
    for (; u < mine; ++u) {
      rings_on();
      // this wave's copies of tile u + 1 have landed once only those of its last vector phase are outstanding
      m_phase(IntC<1>(), IntC<1>(), ok, ov1, ov, [&]() __attribute__((always_inline)) {
        wait_copies(u + 2);
        __builtin_amdgcn_s_barrier();
      });
      copy_next(u, settle);
      weights(u, false);
      __builtin_amdgcn_s_barrier();
    }
    // the values of the wave's last tile: its matrix phase of the tile behind it, or the item's last
    m_phase(IntC<1>(), IntC<0>(), 0, ov, 0, [&]() __attribute__((always_inline)) {
      if (u < n_tiles) wait_copies(u + 2);
      __builtin_amdgcn_s_barrier();
    });
  } else {
    wait_copies(2);
    __builtin_amdgcn_s_barrier();
    u = 0;
  }
  // Behind them: the same copies and barriers, and nothing else.  A wave without tiles comes here from its first matrix phase, the others
  // from that of tile u = mine; one that has all of the item's tiles is done.
  if (u < n_tiles) {
    run_soff = __builtin_amdgcn_readfirstlane(run_soff);          // scalars, here too
    run_tile = __builtin_amdgcn_readfirstlane(run_tile);
    run_group = __builtin_amdgcn_readfirstlane(run_group);
    run_n = __builtin_amdgcn_readfirstlane(run_n);
    if (u > 0) rings_on();
    while (true) {
      copy_next(u, []() {});
      __builtin_amdgcn_s_barrier();
      if (++u >= n_tiles) break;
      rings_on();
      wait_copies(u + 2);
      __builtin_amdgcn_s_barrier();
    }
    __builtin_amdgcn_s_barrier();                                 // the others' last matrix phase
  }
  // K's ring: the last phase, in which group 1 may still be, reads V only
  packed_results<D>(it, wrow0, o, R, smem + wave * (32 * C::ROW_BYTES), lane);
  if (grp == 0) __builtin_amdgcn_s_barrier();                     // group 1's last phase has one more
}

__global__ __launch_bounds__(WIDE_WAVES * 64, 2) void pf_packed_wide_kernel(PackedParams) {
  __shared__ __attribute__((aligned(1024))) char smem[(WIDE_KSTAGES + WIDE_VSTAGES) * WIDE_TILE];
  bool there;
  const PackedItem it = packed_item(there);
  if (__builtin_expect(!there, 0)) packed_no_plan<128>(threadIdx.x, WIDE_WAVES * 64);
  else packed_wide(it, smem, threadIdx.x);
}

#endif  // PF_PACKED_WIDE_H
