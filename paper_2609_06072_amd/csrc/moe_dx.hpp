// Input gradient of the expert projection, many rows per expert (included by
// moe_gemm.hip behind what both share): y[p] = W_e^T x[p] per pair, W_e [K][N]
// row-major, so the contraction runs over W_e's rows.
//
// bf16, tiles of 256 rows x 256 columns, four waves of 128 x 128 as in
// moe_gemm_large_kernel, with its ring of five 32 KB slots and its half-steps.
// Two things differ:
//   - A W unit is 64 contraction rows x 64 columns for each wx, and W fragments
//     are transposed reads (two of 8 bytes in the place of one of 16).
//   - A block stays and takes tile after tile, and the ring runs through:
//     the last half-steps of a tile copy and read the first units of the next
//     one, and a tile's results go from the accumulators to memory while these
//     land.  (One block per tile spent about 14 us per tile outside its loop of
//     14 to 28 us, with the matrix units and HBM busy in turns.)
// A block's tiles are every 32nd of its XCD's run, so the blocks of an XCD work
// on neighbouring tiles at a time.  Where the run's last round would occupy half
// of the XCD's CUs or fewer, its tiles are cut into two or four column parts, which
// as many blocks of a second set (launched behind the first) take.  With splits,
// that many blocks share a tile's contraction (a tile below is then one of these
// parts).  Where a sum follows (of these parts, of a token's slots, with what dx
// holds) the fp32 sums go to a.part as they are, for moe_dx_join_kernel, so that a
// result is rounded once.
// 8192 x 8192 with a contraction of 1024 131 us, of 2048 228 us (the library's dense
// products of these sizes 129 and 220): 1.44 us a stage on a full card, 1.24 for a
// block alone, of which the matrix units are busy for 0.9, and 8 us a tile for its
// results and the next one's start.
#pragma once

namespace ace {
namespace {

// Chunk swizzle of a 128-byte W^T row: pairs of chunks trade places, so that the
// 32 bytes that a transposed read takes of the rows 8 g + (0..3) (+ 4) spread
// over the banks for the lanes of one g and of two.
__device__ inline int lt_swz(int r) { return 2 * ((r & 3) ^ ((r >> 3) & 1)); }

// Fragments of W^T.  A stage holds contraction rows of BN columns; fragment:
// columns n .. n + 15 (lane c16), contraction rows PER*g .. PER*g + PER - 1 of a
// K-block (lane group g), as in Tr<T>::frag.
// bf16: ds_read_b64_tr_b16 hands lane i of 16 the element i & 3 of the 8 bytes
// that lanes 4 j + (i >> 2), j = 0..3, address.  fp32: four words of four rows.
typedef __attribute__((ext_vector_type(4))) short s16x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

// Chunk swizzle of a row of 256 bytes and more (lt_swz for those of 128): bf16
// spreads the rows 8 g + (0..3) of a transposed read, fp32 the rows 4 g + i.
template <typename T, int BN>
__device__ inline int wt_swz(int r) {
  if (sizeof(T) == 4) return 4 * ((r >> 2) & 3);
  return BN == 64 ? lt_swz(r) : 2 * ((r & 3) | (((r >> 3) & 1) << 2));
}

template <typename T, int BN>
__device__ inline typename Tr<T>::frag wt_frag(const char* S, int n, int lane) {
  constexpr int ROWB = BN * (int)sizeof(T);
  const int c16 = lane & 15, g = lane >> 4;
  if constexpr (sizeof(T) == 2) {
    const int r = 8 * g + (c16 >> 2);   // and 4 on: the same swizzle
    const char* p = S + r * ROWB + ((((n >> 3) + ((c16 & 3) >> 1)) ^ wt_swz<T, BN>(r)) << 4) + ((c16 & 1) << 3);
    s16x4 h2[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) h2[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * h * ROWB));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(h2[0], h2[1], 0, 1, 2, 3, 4, 5, 6, 7));
  } else {
    const char* p = S + 4 * g * ROWB + ((((n >> 2) + (c16 >> 2)) ^ wt_swz<T, BN>(4 * g)) << 4) + ((c16 & 3) << 2);
    f32x4 f;
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = *reinterpret_cast<const float*>(p + i * ROWB);
    return f;
  }
}

// mfma_acc without its wait: for operands that no vector instruction wrote just
// before (here LDS reads did; the test of these kernels looks for any).  The two
// wait states of each of 128 instructions a stage were 5% of its time.
__device__ inline void mfma_ready(f32x4& d, bf16x8 a, bf16x8 b) {
  asm("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(d) : "v"(a), "v"(b));
}

// Four values rounded to bf16, as two words.
__device__ inline u32x2 round4(f32x4 v) {
  return __builtin_bit_cast(u32x2, bf16x4{(__bf16)v[0], (__bf16)v[1], (__bf16)v[2], (__bf16)v[3]});
}

// Columns 4 g .. 4 g + 3 of a row's two neighbouring 16-column blocks (lane (c16,
// g)) as bf16: the lanes of a row trade their 8-byte pieces until lane g holds the 16
// bytes 8 g .. 8 g + 7 of the 32 columns.
__device__ inline u32x4 trade4(f32x4 a, f32x4 b) {
  const u32x2 lo = round4(a), hi = round4(b);
  u32x4 o;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    u32x2 s = __builtin_amdgcn_permlane32_swap(lo[i], hi[i], false, false);
    s = __builtin_amdgcn_permlane16_swap(s[0], s[1], false, false);
    o[i] = s[0];
    o[2 + i] = s[1];
  }
  return o;
}

// The lane's number, computed where it is asked for.
__device__ inline int lane_id() {
  int l;
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(l));
  return l;
}

// RAGGED: K is no multiple of two stages; the copies of chunks past it read
// zeros instead (both operands': an infinity times zero is no zero).  Zeroing the
// fragments instead cost 0.6 of 1.8 us a stage on the one wave of a SIMD.
// K >= kDxLargeK, so that the copies never run ahead by more than a tile.
constexpr int kDxLargeK = 256;
__device__ const u32x4 kZeros = {0u, 0u, 0u, 0u};

//
// One block's tiles: NB 16-column blocks a wave (8: whole tiles, item, item + step,
// ... below items; 4 or 2: part `item` of the halves or quarters of the tiles from
// `items` on).  before, upto: see the kernel.
template <bool RAGGED, int NB>
__device__ inline void moe_dx_large_block(const MoeArgs& a, char* smem, int before, int upto, int first, int item,
                                          int step, int items) {
  using C = Large;
  using F = bf16x8;
  constexpr int ROWB = C::ROWB, NC = C::COPIES, KPL = kMaxKeys / 64, CW = 16 * NB;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  const int wy = wave >> 1, wx = wave & 1;
  const int K = a.d_in, N = a.d_out;
  // stages of a tile (an even number; RAGGED: those past the contraction are zeros)
  const int nst2 = 2 * ((K + 2 * C::KC * a.splits - 1) / (2 * C::KC * a.splits));

  struct Tile {
    int e, n0, u0, hi;   // expert, first column (a part's may lie past the last),
                         // first row, end of the expert's rows
    int split;
  };
  // (offsets through the constant address space: scalar loads, which the copies
  // in flight do not hold up); within an expert, groups of up to eight row tiles
  // walk the columns together.  The search goes on from the last tile's key, q.
  const auto soff = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)a.offsets;
  auto tile_of = [&](int it) { return first + (NB == 8 ? it : items + it / (8 / NB)); };
  const int owner = __builtin_ctzll(__ballot(tile_of(item) >= before && tile_of(item) < upto));
  int q = owner * KPL, key0 = __builtin_amdgcn_readlane(before, owner);   // the key's first tile
  int lo = soff[q], hi = soff[min(q + 1, a.E)];
  auto locate = [&](int it) {
    int rem = tile_of(it) - key0;
    for (;;) {   // ends: the tile is one of the offsets' tiles
      const int n = (hi - lo + C::BM - 1) / C::BM * a.nt * a.splits;
      if (rem < n) break;
      rem -= n;
      key0 += n;
      ++q;
      lo = hi;
      hi = soff[min(q + 1, a.E)];
    }
    const int m_e = (hi - lo + C::BM - 1) / C::BM;
    const int split = rem / (m_e * a.nt);
    rem -= split * m_e * a.nt;
    int gtiles = kRowGroup * a.nt;
    asm volatile("" : "+s"(gtiles));   // (its reciprocal, kept, would be spilled)
    const int grp = rem / gtiles, gsz = min(kRowGroup, m_e - grp * kRowGroup);
    const int ing = rem - grp * gtiles;
    const int n0 = ing / gsz * C::BN + (NB == 8 ? 0 : it % (8 / NB) * 2 * CW);
    return Tile{q, n0, lo + (grp * kRowGroup + ing % gsz) * C::BM, hi, split};
  };
  // pairs of the wave's rows 128 wy + lane and + 64 (past the segment: its last)
  auto pairs = [&](const Tile& t, int (&p)[2]) {
    const int r = t.u0 + 128 * wy + lane_id();
#pragma unroll
    for (int i = 0; i < 2; ++i) p[i] = a.pair_list[min(r + 64 * i, t.hi - 1)];
  };
  Tile cur = locate(item), nxt = cur;
  int pc[2], pn[2];      // pairs of the current and the next tile
  pairs(cur, pc);
  bool more = NB == 8 && item + step < items;
  if (more) nxt = locate(item + step);
  pairs(nxt, pn);
  asm volatile("" : "+v"(pn[0]), "+v"(pn[1]));   // waits here, and not in the loop

  // ---- copies: the waves wx = 0 copy the x rows of their wy, the others the W
  // columns of the half wy: of a slot eight 8-row copies, lane l the chunk at
  // position l & 7 of row l >> 3.  Offsets count 16-byte chunks.
  const int crl = lane >> 3, cpos = lane & 7;
  const bool xwave = wx == 0;
  const int xmask = xwave ? -1 : 0;
  const int col[2] = {cpos ^ l_swz(crl), cpos ^ l_swz(8 + crl)};
  uint32_t roff[2][NC];    // slots P[v] of even and of odd v
  const char* base;        // x, or the tile's first column of W_e
  int st0;                 // the tile's first stage of the contraction
  auto set_tile = [&](const Tile& t, const int (&p)[2]) {
    const int n0 = min(t.n0, N - 8);
    st0 = t.split * nst2;
    base = xwave ? static_cast<const char*>(a.x)
                 : static_cast<const char*>(a.W) + ((size_t)t.e * K * N + n0) * 2;
#pragma unroll
    for (int par = 0; par < 2; ++par)
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        const int h = xwave ? 1 - par : par;   // x unit v + 1, W unit v + 2
        const int c = CW / 8 * wy + 8 * h + (cpos ^ lt_swz(8 * i + crl));
        const uint32_t w = (uint32_t)(8 * i + crl) * (uint32_t)(N / 8) + min(c, (N - n0) / 8 - 1);
        // (p[h], as an indexed array would lie in memory)
        const uint32_t x = (uint32_t)__shfl(p[par] ^ ((p[0] ^ p[1]) & xmask), 8 * i + crl, 64) * (uint32_t)(K / 8);
        roff[par][i] = xwave ? x : w;
      }
  };
  set_tile(cur, pc);
  const uint32_t cbase = lds_addr(smem) + (xwave ? 0 : C::UNIT) + wy * (C::UNIT / 2);
  uint32_t cslot = cbase;      // where this wave's copies of the next slot go
  int cst = -1;                // stage that this wave copies (x starts half a stage early)
  const char* sbase = base;    // of that stage
  uint32_t colb[2] = {0, 0};   // x: chunk of the lane's column, by copy parity
  // RAGGED: copy i reads zeros where key + i wmul >= K / 8 (x: the chunk; W: the
  // 8-row group of the stage); one form for both, so that nothing branches
  uint32_t key[2] = {0, 0};
  const int wmul = xwave ? 0 : 1;
  uint64_t zeros = reinterpret_cast<uint64_t>(&kZeros);
  asm("" : "+s"(zeros));
  // ENDS: the stage may be the first one past the tile (then it is the next
  // tile's first, or the last one again)
  auto begin_copies = [&](int par, bool ends) {
    if (par == (xwave ? 1 : 0)) ++cst;
    if (ends && cst == nst2 && more) {
      cst = 0;
      set_tile(nxt, pn);
    }
    // (a block without a next tile repeats its last stage)
    const int st = st0 + max(0, min(cst, nst2 - 1));
    if (xwave) {
      sbase = base;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        colb[c] = key[c] = st * (C::KC / 8) + col[c];
      }
    } else {
      sbase = base + (size_t)st * (C::KC * 2) * N;
      key[0] = key[1] = st * (C::KC / 8);
    }
  };
  auto copy = [&](int par, int i) {
    uint64_t p = reinterpret_cast<uint64_t>(sbase) + (uint64_t)(roff[par][i] + colb[i & 1]) * 16;
    if (RAGGED) p = (int)key[i & 1] >= K / 8 - i * wmul ? zeros : p;
    dma16(reinterpret_cast<const void*>(p), __builtin_amdgcn_readfirstlane(cslot + i * 1024));
  };
  auto end_copies = [&]() {
    cslot += C::SLOT;
    if (cslot >= cbase + C::SLOTS * C::SLOT) cslot = cbase;
  };
#pragma unroll
  for (int v = -2; v < 2; ++v) {
    begin_copies(v & 1, false);
#pragma unroll
    for (int i = 0; i < NC; ++i) copy(v & 1, i);
    end_copies();
  }

  F x0[4], x1a[4], x1b[4], wa[16], wb[16];   // x: K-block 0 and 1 of a half, W: [nb + 8 kh]
  f32x4 acc[NB][8];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int mb = 0; mb < 8; ++mb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};

  // ---- fragment reads.  x rows 64 wy + 16 mb + c16 of a unit, as in the
  // forward.  W fragment nb of K-block kh: 8 bytes of the rows 32 kh + 8 g + 4 h +
  // (c16 >> 2) of the unit's wx half, at chunk 2 nb + (c16 & 3) / 2; the swizzle
  // depends on the lane only, and moves nb.
  const int xl = (64 * wy + c16) * ROWB + ((g ^ l_swz(c16)) << 4);
  int wtl[4];
#pragma unroll
  for (int nb = 0; nb < 4; ++nb) {
    const int r = 8 * g + (c16 >> 2);
    wtl[nb] = C::UNIT + (64 * wx + r) * ROWB + (((2 * nb + ((c16 & 3) >> 1)) ^ lt_swz(r)) << 4) + ((c16 & 1) << 3);
  }
  int rslot = 0;     // slot that the half-step reads
  auto wt_read = [&](int nb, int kh) {
    s16x4 h2[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      h2[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(smem + rslot + wtl[nb] + (32 * kh + 4 * h) * ROWB));
    return __builtin_bit_cast(F, __builtin_shufflevector(h2[0], h2[1], 0, 1, 2, 3, 4, 5, 6, 7));
  };
  // Half-step h = PAR of a stage: matrix work on (x0, xc, wc) for the wave's row
  // blocks 4 h .. 4 h + 3; reads the next half's x fragments and half of the next
  // stage's W fragments; copies the slot after next but three.
  // The copies come to the end of the tile in its last stage but two, an odd one.
  // drained: the first four half-steps behind a tile whose 32 stores were all
  // issued.  The slots they read were copied before the stores, which may all be
  // under way beside the 24 copies behind the needed ones.  (As compiled they have
  // ended by then: set_tile reloads spilled chunk numbers, behind all of them.)
  auto half = [&](auto par_c, auto mma_c, auto odd_c, bool drained, F (&x1)[4], F (&wc)[16], F (&x1n)[4], F (&wn)[16]) {
    constexpr int PAR = decltype(par_c)::value;
    constexpr bool MMA = decltype(mma_c)::value;
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    if (drained) wait_vmcnt<56>();
    else wait_vmcnt<24>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const char* xs = smem + rslot + xl;
    const char* xs1 = smem + rslot + (xl ^ 64);
    begin_copies(PAR, decltype(odd_c)::value);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (i < 8) {
        if (i < 4) x1n[i] = *reinterpret_cast<const F*>(xs1 + i * 16 * ROWB);
        if (4 * PAR + (i & 3) < NB) wn[4 * PAR + (i & 3) + 8 * (i >> 2)] = wt_read(i & 3, i >> 2);
        copy(PAR, i);
      }
      if (i >= 8 && i < 12) x0[i - 8] = *reinterpret_cast<const F*>(xs + (i - 8) * 16 * ROWB);
      if (MMA && (i & 7) < NB) {
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) {
          const int nb = i & 7, kh = i >> 3;
          mfma_ready(acc[nb][4 * PAR + mb], wc[nb + 8 * kh], kh ? x1[mb] : x0[mb]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    end_copies();
    rslot = rslot == (C::SLOTS - 1) * C::SLOT ? 0 : rslot + C::SLOT;
  };
  using P0 = std::integral_constant<int, 0>;
  using P1 = std::integral_constant<int, 1>;
  using Yes = std::true_type;
  using No = std::false_type;
  __bf16* Y = static_cast<__bf16*>(a.y);
  half(P0{}, No{}, No{}, false, x1a, wb, x1b, wa);
  half(P1{}, No{}, No{}, false, x1b, wb, x1a, wa);
  bool drained = false;
  for (;;) {
    for (int st = 0; st < nst2; st += 2) {   // two stages: the W fragments change registers
      half(P0{}, Yes{}, No{}, drained, x1a, wa, x1b, wb);
      half(P1{}, Yes{}, No{}, drained, x1b, wa, x1a, wb);
      half(P0{}, Yes{}, Yes{}, drained, x1a, wb, x1b, wa);
      half(P1{}, Yes{}, Yes{}, drained, x1b, wb, x1a, wa);
      drained = false;
    }
    // ---- the tile after next, then this tile's results: lane (c16, g) holds
    const bool last = !more;
    Tile nn = nxt;
    int pnn[2];
    item += step;
    more = NB == 8 && item + step < items;
    if (more) nn = locate(item + step);
    pairs(nn, pnn);
    mfma_done();
    __builtin_amdgcn_sched_barrier(0);
    // columns 4 g .. 4 g + 3 of a 16-column block of row c16.  Of two neighbouring
    // blocks the lanes of a row trade their 8-byte pieces until lane g holds the
    // 16 bytes g: a store covers 64 bytes of each of 16 rows (32 bytes of them:
    // 35 us more for 134 MB of results).  fp32 sums go out as they are.
    // full: all 32 stores are issued, in a straight line, so that the compiler can
    // count them where it waits for the loads above, which are older.
    // (the lane's number anew: kept, it and what follows from it would be spilled
    // too)
    const int ln = lane_id(), lc16 = ln & 15, lg = ln >> 4;
    const int col0 = cur.n0 + CW * wx + 8 * lg, col1 = cur.n0 + CW * wx + 4 * lg, row0 = cur.u0 + 128 * wy + lc16;
    auto store = [&](auto full_c, int mb) {
      constexpr bool FULL = decltype(full_c)::value;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) asm volatile("" : "+a"(acc[nb][mb]));   // read behind mfma_done
      u32x4 o[NB / 2];
#pragma unroll
      for (int nb = 0; nb < NB; nb += 2) o[nb / 2] = trade4(acc[nb][mb], acc[nb + 1][mb]);
      const int p = __shfl(pc[mb >> 2], 16 * (mb & 3) + lc16, 64);
      if (!FULL && a.part) {
        if (row0 + 16 * mb < cur.hi) {
          float* row = a.part + ((size_t)cur.split * a.pairs + p) * N + col1;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            if (col1 + 16 * nb < N) *reinterpret_cast<f32x4*>(row + 16 * nb) = acc[nb][mb];
        }
      } else if (FULL || row0 + 16 * mb < cur.hi) {
        __bf16* row = Y + (size_t)p * N + col0;
#pragma unroll
        for (int nb = 0; nb < NB; nb += 2)
          if (FULL || col0 + 16 * nb < N) *reinterpret_cast<u32x4*>(row + 16 * nb) = o[nb / 2];
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
    };
    drained = NB == 8 && !a.part && cur.u0 + C::BM <= cur.hi && cur.n0 + C::BN <= N;
    if (drained) {
#pragma unroll
      for (int mb = 0; mb < 8; ++mb) store(Yes{}, mb);
      asm volatile("" : "+v"(pnn[0]), "+v"(pnn[1]));
    } else {
#pragma unroll
      for (int mb = 0; mb < 8; ++mb) store(No{}, mb);
      asm volatile("" : "+v"(pnn[0]), "+v"(pnn[1]));
    }
    if (last) break;
    cur = nxt;
    nxt = nn;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      pc[i] = pn[i];
      pn[i] = pnn[i];
    }
  }
  wait_vmcnt<0>();   // copies past the last tile (repeats of its last stage)
}

template <bool RAGGED>
__global__ __launch_bounds__(Large::THREADS, 1) void moe_dx_large_kernel(MoeArgs a) {
  using C = Large;
  constexpr int KPL = kMaxKeys / 64;
  __shared__ __attribute__((aligned(16))) char smem[C::SLOTS * C::SLOT];
  // Lane l keeps the number of tiles before and up to the end of the keys KPL l ..
  // KPL l + KPL - 1.
  const int lane = threadIdx.x & 63;
  int cnt = 0, off[KPL + 1];
#pragma unroll
  for (int i = 0; i <= KPL; ++i) off[i] = a.offsets[min(lane * KPL + i, a.E)];
#pragma unroll
  for (int i = 0; i < KPL; ++i) cnt += (off[i + 1] - off[i] + C::BM - 1) / C::BM * a.nt * a.splits;
  int upto = cnt;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o, 64);
    if (lane >= o) upto += v;
  }
  const int before = upto - cnt;
  // the XCD's run of tiles, and how many of them form a last round that is cut up
  const int n_tiles = __builtin_amdgcn_readfirstlane(__shfl(upto, 63, 64));
  const int per_xcd = (n_tiles + kXcds - 1) / kXcds;
  const int step = gridDim.x / (2 * kXcds);     // blocks of each set per XCD
  const int first = blockIdx.x % kXcds * per_xcd, mine = max(0, min(per_xcd, n_tiles - first));
  const int over = mine % step, whole = 2 * over <= step ? mine - over : mine;
  const int b = blockIdx.x / kXcds;
  if (b < step) {
    if (b < whole) moe_dx_large_block<RAGGED, 8>(a, smem, before, upto, first, b, step, whole);
  } else if (4 * over <= step) {
    if (b - step < 4 * (mine - whole)) moe_dx_large_block<RAGGED, 2>(a, smem, before, upto, first, b - step, step, whole);
  } else {
    if (b - step < 2 * (mine - whole)) moe_dx_large_block<RAGGED, 4>(a, smem, before, upto, first, b - step, step, whole);
  }
}

// ---- few rows per expert: the weights bound the call, and a block streams them.
//
// A block takes up to 16 NRB rows of one expert and BN columns (128 to 256 bytes
// of a W row).  Its four waves split the contraction: wave w takes the K-blocks w, w +
// 4, ..., each through a ring of its own in LDS (the K-block's W rows and the same
// columns of the x rows), so no barrier stands in the loop; the four sums meet in
// LDS at the end, in wave order.  Where even the smallest tiles leave CUs idle,
// several blocks share a tile's K-blocks in the same way (a.splits) and moe_dx_join_kernel
// adds their sums, in order.  A third buffer per wave gained nothing (fewer
// streams at a time serve HBM better).  64 experts of 2048 x 1024 with 4 rows
// each: 44 us, 5.9 TB/s of weights.
template <typename T, int NRB, int BN_>
struct DxStream {
  static constexpr int KB = Tr<T>::KB, BM = 16 * NRB, BN = BN_, NBUF = 2, NCB = BN / 16;
  static constexpr int WBYTES = KB * BN * (int)sizeof(T), STAGE = WBYTES + BM * kGRowBytes;
  static constexpr int NS = WBYTES / 1024;                  // W copies of a stage
  static constexpr int WCH = BN * (int)sizeof(T) / 16;      // chunks of a W row
  static constexpr int CST = BN + 4;                        // row stride of the sums
  static constexpr int RING = 4 * NBUF * STAGE, SUMS = 4 * BM * CST * 4;
};

// RUNS (several row tiles per expert on average): each XCD walks a contiguous run
// of items (expert, columns, rows, split), so that the row tiles that read the same
// W columns share an L2 (fp32, 3380 x 2852, 16 experts of 80 rows: 485 -> 335 us).
// Otherwise the items (expert, rows, columns, split) go round, and W bypasses the
// caches: it is read once (8 uneven experts of 4096 x 4096, 32 rows on average: 69
// us, in runs 82).
template <typename T, int NRB, int BN, bool RUNS>
__global__ __launch_bounds__(256) void moe_dx_stream_kernel(MoeArgs a) {
  using C = DxStream<T, NRB, BN>;
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER, KB = C::KB, NCB = C::NCB, NBUF = C::NBUF;
  __shared__ __attribute__((aligned(16))) char smem[C::RING > C::SUMS ? C::RING : C::SUMS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  int e, u0, u_end, n0, split;   // (the returns are block-uniform)
  if constexpr (RUNS) {
    const int n_items = count_tiles(a.offsets, a.E, C::BM) * a.nt * a.splits;
    const int per_xcd = (n_items + kXcds - 1) / kXcds, bi = blockIdx.x / kXcds;
    const int item = (blockIdx.x % kXcds) * per_xcd + bi;
    if (bi >= per_xcd || item >= n_items) return;
    int lo, rem;
    if (!locate_key(a.offsets, a.E, C::BM, a.nt, item / a.splits, &e, &lo, &u_end, &rem)) return;
    split = item % a.splits;
    const int m_e = (u_end - lo + C::BM - 1) / C::BM;
    n0 = rem / m_e * C::BN;
    u0 = lo + rem % m_e * C::BM;
  } else {
    const int tile = blockIdx.x / a.splits;
    split = blockIdx.x % a.splits;
    n0 = tile % a.nt * C::BN;
    if (!locate_tile(a.offsets, a.E, C::BM, tile / a.nt, &e, &u0, &u_end)) return;
    e = __builtin_amdgcn_readfirstlane(e);
  }
  const int K = a.d_in, N = a.d_out;
  const T* X = static_cast<const T*>(a.x);
  const T* Wt = static_cast<const T*>(a.W) + (size_t)e * K * N + n0;
  // x copies: lane l takes the chunk at position l & 3 of row l >> 2 of 16; only
  // those that hold rows of the tile
  const int nx = __builtin_amdgcn_readfirstlane(min(NRB, (u_end - u0 + 15) / 16));
  const T* xsrc[NRB];
#pragma unroll
  for (int i = 0; i < NRB; ++i)
    xsrc[i] = X + (size_t)a.pair_list[min(u0 + 16 * i + (lane >> 2), u_end - 1)] * K;
  const int xcol = PER * ((lane & 3) ^ g_swz(lane >> 2));
  // W copies: 64 chunks each, of rows of WCH
  const int wrow = lane / C::WCH;
  constexpr int RPC = 64 / C::WCH;
  auto col_of = [&](int i) { return min(PER * ((lane % C::WCH) ^ wt_swz<T, BN>(RPC * i + wrow)), N - PER - n0); };
  const int nst = (K + KB - 1) / KB;
  // K-blocks of this wave: first, first + stride, ...
  const int stride = 4 * a.splits, first = 4 * split + wave;
  const int mine = max(0, (nst - first + stride - 1) / stride);
  char* ring = smem + wave * NBUF * C::STAGE;
  auto issue = [&](int i) {
    const int k0 = (first + stride * i) * KB;
    const uint32_t buf = lds_addr(ring) + (i % NBUF) * C::STAGE;
    const T* Wk = Wt + (size_t)k0 * N;
#pragma unroll
    for (int c = 0; c < C::NS; ++c) {
      const int col = col_of(c);
      const int row = min(RPC * c + wrow, K - 1 - k0);
      const T* src = Wk + ((uint32_t)row * (uint32_t)N + (uint32_t)col);
      const uint32_t dst = __builtin_amdgcn_readfirstlane(buf + c * 1024);
      if constexpr (RUNS) dma16(src, dst);
      else dma16_nt(src, dst);
    }
#pragma unroll
    for (int r = 0; r < NRB; ++r)
      if (r < nx)
        dma16(xsrc[r] + min(k0 + xcol, K - PER), __builtin_amdgcn_readfirstlane(buf + C::WBYTES + r * 1024));
  };
  f32x4 acc[NCB][NRB];
#pragma unroll
  for (int nb = 0; nb < NCB; ++nb)
#pragma unroll
    for (int ib = 0; ib < NRB; ++ib) acc[nb][ib] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NBUF - 1; ++i)
    if (i < mine) issue(i);
  for (int i = 0; i < mine; ++i) {
    // K-block i - 1 is in registers: its buffer takes K-block i + NBUF - 1
    __builtin_amdgcn_s_waitcnt(0xc07f);   // lgkmcnt(0)
    asm volatile("" ::: "memory");
    if (i + NBUF - 1 < mine) issue(i + NBUF - 1);
    wait_vmcnt_upto<(NBUF - 1) * (C::NS + NRB)>(min(NBUF - 1, mine - 1 - i) * (C::NS + nx));
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    const char* S = ring + (i % NBUF) * C::STAGE;
    const bool past = (first + stride * i) * KB + PER * g >= K;
    F wf[NCB], xf[NRB];
#pragma unroll
    for (int nb = 0; nb < NCB; ++nb) {
      wf[nb] = wt_frag<T, BN>(S, 16 * nb, lane);
      if (past) wf[nb] = Tr<T>::zero();
    }
#pragma unroll
    for (int ib = 0; ib < NRB; ++ib) {
      xf[ib] = *reinterpret_cast<const F*>(S + C::WBYTES + (16 * ib + c16) * kGRowBytes + ((g ^ g_swz(c16)) << 4));
      if (past || ib >= nx) xf[ib] = Tr<T>::zero();
    }
#pragma unroll
    for (int ib = 0; ib < NRB; ++ib)
#pragma unroll
      for (int nb = 0; nb < NCB; ++nb) acc[nb][ib] = Tr<T>::mma(wf[nb], xf[ib], acc[nb][ib]);   // D[column][row]
  }
  // ---- the waves' sums
  __syncthreads();
  float* sums = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int ib = 0; ib < NRB; ++ib)
#pragma unroll
    for (int nb = 0; nb < NCB; ++nb)
      *reinterpret_cast<f32x4*>(sums + (wave * C::BM + 16 * ib + c16) * C::CST + 16 * nb + 4 * g) = acc[nb][ib];
  __syncthreads();
  typedef __attribute__((ext_vector_type(4))) T T4;
  T* Y = static_cast<T*>(a.y);
#pragma unroll
  for (int i = 0; i < NRB * BN / 64; ++i) {
    const int it = 256 * i + threadIdx.x, row = it / (BN / 4), col = 4 * (it % (BN / 4));
    f32x4 v = *reinterpret_cast<const f32x4*>(sums + row * C::CST + col);
#pragma unroll
    for (int w = 1; w < 4; ++w) v += *reinterpret_cast<const f32x4*>(sums + (w * C::BM + row) * C::CST + col);
    if (u0 + row < u_end && n0 + col < N) {
      const size_t at = (size_t)a.pair_list[u0 + row] * N + n0 + col;
      if (a.part) *reinterpret_cast<f32x4*>(a.part + (size_t)split * a.pairs * N + at) = v;
      else *reinterpret_cast<T4*>(Y + at) = T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]};
    }
  }
}

// dx (four columns per thread) from the fp32 sums of the splits: of one pair, or of a
// token's routed slots in slot order, added to what dx holds where accumulate asks for
// it, and rounded once.
// The loads of G sums are under way at a time, without branches between them (one
// token, 8 experts of 2048 x 1024: the call 16.3 -> 13.0 us).
template <typename T, int G>
__global__ __launch_bounds__(kThreads) void moe_dx_join_kernel(DxJoinArgs a) {
  typedef __attribute__((ext_vector_type(4))) T T4;
  const uint32_t idx = blockIdx.x * kThreads + threadIdx.x;
  if (idx >= a.pieces) return;
  const uint32_t t = a.per_row.div(idx), col = 4 * (idx - t * a.per_row.d);
  f32x4 v = {0.f, 0.f, 0.f, 0.f};
  bool routed = false;
  const int n = a.k * a.splits;
  for (int i0 = 0, j = 0, s = 0; i0 < n; i0 += G) {
    int row[G];
    f32x4 f[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
      const size_t p = (size_t)t * a.k + j;
      row[g] = a.pair_row[p];
      f[g] = Tr<float>::load_nt(a.part + ((size_t)s * a.pairs + p) * a.d + col);
      if (i0 + g + 1 < n && ++s == a.splits) {
        s = 0;
        ++j;
      }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) {
      asm volatile("" : "+v"(f[g]));   // loaded above, not behind the branch
      if (i0 + g >= n || row[g] < 0) continue;
      routed = true;
      v += f[g];
    }
  }
  if (!routed && (a.keep || a.accumulate)) return;   // (a sum with 0 would lose a zero's sign)
  T4* out = reinterpret_cast<T4*>(static_cast<T*>(a.out) + (size_t)t * a.d + col);
  if (a.accumulate) {
    const T4 o = *out;
    v += f32x4{(float)o[0], (float)o[1], (float)o[2], (float)o[3]};
  }
  __builtin_nontemporal_store(T4{(T)v[0], (T)v[1], (T)v[2], (T)v[3]}, out);
}

// Sums under way: as many as there are, up to eight.
template <typename T>
void moe_dx_join(const DxJoinArgs& a, unsigned grid, hipStream_t stream) {
  const int n = a.k * a.splits;
  if (n == 1) moe_dx_join_kernel<T, 1><<<grid, kThreads, 0, stream>>>(a);
  else if (n == 2) moe_dx_join_kernel<T, 2><<<grid, kThreads, 0, stream>>>(a);
  else if (n <= 4) moe_dx_join_kernel<T, 4><<<grid, kThreads, 0, stream>>>(a);
  else moe_dx_join_kernel<T, 8><<<grid, kThreads, 0, stream>>>(a);
}

// ---- tiles of 128 rows x 128 columns, four waves of 64 x 64, one K-block a stage
// in a ring in LDS, several blocks per CU (while one waits or stores, the others use
// the matrix units): fp32 with many rows per expert, bf16 where the large tiles leave
// CUs idle.  Tile order, splits and fp32 sums as in the large tiles.
template <typename T>
struct DxTile {
  static constexpr int KB = Tr<T>::KB, BM = 128, BN = 128, NBUF = sizeof(T) == 4 ? 3 : 4, PER_CU = sizeof(T) == 4 ? 3 : 2;
  static constexpr int XBYTES = BM * kGRowBytes, STAGE = XBYTES + KB * BN * (int)sizeof(T), COPIES = 2;
  static constexpr int WCH = BN * (int)sizeof(T) / 16, RPC = 64 / WCH;   // chunks of a W row, rows of a copy
};

template <typename T>
__global__ __launch_bounds__(256, DxTile<T>::PER_CU) void moe_dx_tile_kernel(MoeArgs a) {
  using C = DxTile<T>;
  using F = typename Tr<T>::frag;
  constexpr int PER = Tr<T>::PER;
  __shared__ __attribute__((aligned(16))) char smem[C::NBUF * C::STAGE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c16 = lane & 15, g = lane >> 4;
  const int wy = wave >> 1, wx = wave & 1;
  const int n_items = count_tiles(a.offsets, a.E, C::BM) * a.nt * a.splits;
  const int per_xcd = (n_items + kXcds - 1) / kXcds;
  const int bi = blockIdx.x / kXcds;
  const int item = (blockIdx.x % kXcds) * per_xcd + bi;
  if (bi >= per_xcd || item >= n_items) return;
  int e, lo, hi, rem;
  if (!locate_key(a.offsets, a.E, C::BM, a.nt, item / a.splits, &e, &lo, &hi, &rem)) return;
  const int split = item % a.splits;
  const int m_e = (hi - lo + C::BM - 1) / C::BM;
  const int grp = rem / (kRowGroup * a.nt), gsz = min(kRowGroup, m_e - grp * kRowGroup);
  const int ing = rem - grp * kRowGroup * a.nt;
  const int n0 = ing / gsz * C::BN;
  const int u0 = lo + (grp * kRowGroup + ing % gsz) * C::BM;
  const int K = a.d_in, N = a.d_out;
  const T* X = static_cast<const T*>(a.x);
  const T* Wt = static_cast<const T*>(a.W) + (size_t)e * K * N + n0;
  // copies of wave w: x rows 32 w + 16 i + (lane >> 2), W rows RPC (2 w + i) + lane / WCH
  const int wrow = C::RPC * 2 * wave + lane / C::WCH;
  const T* xsrc[C::COPIES];
  int wcol[C::COPIES];
#pragma unroll
  for (int i = 0; i < C::COPIES; ++i) {
    xsrc[i] = X + (size_t)a.pair_list[min(u0 + 32 * wave + 16 * i + (lane >> 2), hi - 1)] * K;
    wcol[i] = min(PER * ((lane % C::WCH) ^ wt_swz<T, C::BN>(wrow + C::RPC * i)), N - PER - n0);
  }
  const int xcol = PER * ((lane & 3) ^ g_swz(lane >> 2));
  // K-blocks st0 .. st0 + nst - 1
  const int all = (K + C::KB - 1) / C::KB, share = (all + a.splits - 1) / a.splits;
  const int st0 = split * share, nst = max(0, min(share, all - st0));
  const uint32_t sbase = lds_addr(smem);
  auto issue = [&](int st) {
    const uint32_t buf = sbase + (st % C::NBUF) * C::STAGE;
    const int k0 = (st0 + st) * C::KB;
    const T* Wk = Wt + (size_t)k0 * N;
#pragma unroll
    for (int i = 0; i < C::COPIES; ++i) {
      dma16(xsrc[i] + min(k0 + xcol, K - PER), __builtin_amdgcn_readfirstlane(buf + (32 * wave + 16 * i) * kGRowBytes));
      const int row = min(wrow + C::RPC * i, K - 1 - k0);
      dma16(Wk + ((uint32_t)row * (uint32_t)N + (uint32_t)wcol[i]),
            __builtin_amdgcn_readfirstlane(buf + C::XBYTES + (2 * wave + i) * 1024));
    }
  };
  f32x4 acc[4][4];
#pragma unroll
  for (int nb = 0; nb < 4; ++nb)
#pragma unroll
    for (int mb = 0; mb < 4; ++mb) acc[nb][mb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int s = 0; s < C::NBUF - 1; ++s)
    if (s < nst) issue(s);
  for (int st = 0; st < nst; ++st) {
    wait_vmcnt_upto<(C::NBUF - 2) * 2 * C::COPIES>(min(C::NBUF - 2, nst - 1 - st) * 2 * C::COPIES);
    __syncthreads();
    if (st + C::NBUF - 1 < nst) issue(st + C::NBUF - 1);
    const char* S = smem + (st % C::NBUF) * C::STAGE;
    const bool past = (st0 + st) * C::KB + PER * g >= K;
    F xf[4], wf[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      xf[i] = *reinterpret_cast<const F*>(S + (64 * wy + 16 * i + c16) * kGRowBytes + ((g ^ g_swz(c16)) << 4));
      wf[i] = wt_frag<T, C::BN>(S + C::XBYTES, 64 * wx + 16 * i, lane);
      if (past) xf[i] = wf[i] = Tr<T>::zero();
    }
    if constexpr (sizeof(T) == 4) {
#pragma unroll
      for (int i = 0; i < 4; ++i)   // the four products of an accumulator block apart
#pragma unroll
        for (int nb = 0; nb < 4; ++nb)
#pragma unroll
          for (int mb = 0; mb < 4; ++mb)   // D[column][row]
            acc[nb][mb] = __builtin_amdgcn_mfma_f32_16x16x4f32(wf[nb][i], xf[mb][i], acc[nb][mb], 0, 0, 0);
    } else {
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
#pragma unroll
        for (int mb = 0; mb < 4; ++mb) acc[nb][mb] = Tr<T>::mma(wf[nb], xf[mb], acc[nb][mb]);
    }
  }
  T* Y = static_cast<T*>(a.y);
  const int col0 = n0 + 64 * wx + 4 * g, col8 = n0 + 64 * wx + 8 * g;
#pragma unroll
  for (int mb = 0; mb < 4; ++mb) {
    const int u = u0 + 64 * wy + 16 * mb + c16;
    const size_t at = (size_t)a.pair_list[min(u, hi - 1)] * N;
    if (sizeof(T) == 4 || a.part) {
      float* row = (a.part ? a.part + (size_t)split * a.pairs * N : reinterpret_cast<float*>(Y)) + at + col0;
#pragma unroll
      for (int nb = 0; nb < 4; ++nb)
        if (u < hi && col0 + 16 * nb < N) *reinterpret_cast<f32x4*>(row + 16 * nb) = acc[nb][mb];
    } else {
#pragma unroll
      for (int nb = 0; nb < 4; nb += 2) {   // (before the branch: lanes trade pieces)
        const u32x4 o = trade4(acc[nb][mb], acc[nb + 1][mb]);
        if (u < hi && col8 + 16 * nb < N) *reinterpret_cast<u32x4*>(Y + at + col8 + 16 * nb) = o;
      }
    }
  }
}

}  // namespace
}  // namespace ace
