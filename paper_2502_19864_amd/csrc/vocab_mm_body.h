// The body of a workgroup of the vocabulary head's bf16 products, in vocab_mm_k and, twice, in vocab_mm_grads_k (k_vocab_mm.hip).  As text: as a
// function that both call, the arguments are kept in registers over the products, and 2048 x 32000 logits of d 4096 take 463 us instead of 445.
// In scope: BM, BN, WM, WN, KA, KB, E; a, p; smem; wg() of wgs() workgroups.
  constexpr int NW = WM * WN, TM = BM / WM, TN = BN / WN, FM = TM / 32, FN = TN / 32, BK = 64, NS = 2, KS = BK / 16;
  using OA = Operand<BM, BK, NW, KA>;
  using OB = Operand<BN, BK, NW, KB>;
  constexpr int LPT = OA::L + OB::L, STAGE = (BM + BN) * BK * 2;
  constexpr int ND = FM * (KA ? 1 : 2) + FN * (KB ? 1 : 2);
  static_assert(FM * 32 * WM == BM && FN * 32 * WN == BN, "tile");
  static_assert(NS * STAGE + NW * 4096 == MM_LDS<BM, BN, WM, WN> && MM_LDS<BM, BN, WM, WN> <= 160 * 1024, "LDS");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave / WN, wn = wave % WN;
  const int wave_u = __builtin_amdgcn_readfirstlane(wave);
  const int cnt = __builtin_amdgcn_readfirstlane(piece_rows(a));
  const int M = E == Prod::Dw ? p.M : cnt, N = p.N;
  constexpr bool SHARED = E == Prod::Dh || E == Prod::Dw;
  const bool two = SHARED && two_parts(cnt);
  const int K = E == Prod::Dw ? (two ? 2 * TWO_PARTS : cnt) : p.K;
  const int ntm = (M + BM - 1) / BM, ntn = (N + BN - 1) / BN, tiles = ntm * ntn;
  const int splits = SHARED && tiles ? __builtin_amdgcn_readfirstlane(k_shares(p.slots, tiles, K, MM_LEAST, MM_LONGEST)) : 1;
  const int nk_all = (K + BK - 1) / BK;
  int m0 = 0, n0 = 0, split = 0, kt0 = 0, nk = 0, tile = 0;
  // the g-th piece of work, or none
  auto locate = [&](int g) {
    if (g >= tiles * splits) return false;
    if constexpr (SHARED) split = __builtin_amdgcn_readfirstlane(g / tiles);
    int tm, tn;
    vocab_tile<4>(g - split * tiles, ntm, ntn, tm, tn);
    tile = __builtin_amdgcn_readfirstlane(tm * ntn + tn);
    m0 = __builtin_amdgcn_readfirstlane(tm * BM);
    n0 = __builtin_amdgcn_readfirstlane(tn * BN);
    kt0 = (int)((long)nk_all * split / splits);
    nk = (int)((long)nk_all * (split + 1) / splits) - kt0;
    return true;
  };
  const float unit = SHARED ? dloss_unit(a) : 1.f;
  OA oa;
  OB ob;
  // part q of `of` of k-tile kt's DMA instructions.  A (hc in the logits, P) has zeros up to whole k-tiles; B has not.
  auto issue = [&](int kt, int slot, int q, int of) {
    const uint32_t l0 = lds_addr(smem) + slot * STAGE;
    const bool again = E == Prod::Dw && two;  // the second part meets the same rows of hc
    const int kb = again ? 0 : kt0 + kt, left = again ? cnt : min(BK, K - kb * BK);
#pragma unroll
    for (int i = LPT * q / of; i < LPT * (q + 1) / of; ++i) {
      if (i < OA::L) oa.dma(i, kt0 + kt, BK, l0, wave, wave_u, lane);
      else ob.dma(i - OA::L, kb, left, l0 + BM * BK * 2, wave, wave_u, lane);
    }
  };
  auto begin = [&] {
    oa.init(p.A, p.lda, m0, E == Prod::Dh && two ? 2 * TWO_PARTS : M, wave, lane);
    ob.init(p.B, p.ldb, n0, N, wave, lane);
#pragma unroll
    for (int t = 0; t < NS; ++t)
      if (t < nk) issue(t, t, 0, 1);
  };
  Frags<BM, BK, FM, KA> ra;
  Frags<BN, BK, FN, KB> rb;
  ra.init(wm * TM, lane);
  rb.init(wn * TN, lane);
  bf16x8 fa[2][FM], fb[2][FN];
  auto read_frags = [&](int slot, int ks, int buf) {
    ra.read(smem + slot * STAGE, ks, lane, fa[buf]);
    rb.read(smem + slot * STAGE + BM * BK * 2, ks, lane, fb[buf]);
  };
  f32x16 acc[FM][FN];
  // A finished stage is refilled in pieces, the first right after the barrier that frees it.  The first NS k-tiles of a tile
  // had landed before the stores of the last one were issued: they are not waited for, so neither are the stores.
  constexpr int PARTS = 2;
  auto step = [&](auto S, int kt) {
    constexpr int s = decltype(S)::value, other = 1 - s;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (ks + 1 < KS) {
        if (ks + 1 < PARTS && kt > 0 && kt + 1 < nk) issue(kt + 1, other, ks + 1, PARTS);
        read_frags(s, ks + 1, (ks + 1) & 1);
      } else if (kt + 1 < nk) {
        if (kt + 1 >= NS) wait_dma<0>();
        else __builtin_amdgcn_s_waitcnt(0xF | (0x7 << 4) | (0x3 << 14));  // lgkmcnt == 0
        wg_barrier();
        if (kt + NS < nk) issue(kt + NS, s, 0, PARTS);
        read_frags(other, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = mfma32(fb[ks & 1][j], fa[ks & 1][i], acc[i][j]);
      spread_reads<ND, FM * FN>(std::make_integer_sequence<int, FM * FN>{});
    }
  };

  if (!locate(wg())) return;
  begin();
  wait_dma<0>();
  for (int g = wg();;) {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    wg_barrier();
    if (nk > 0) {
      read_frags(0, 0, 0);
      for (int kt = 0; kt < nk; kt += NS) {
        step(std::integral_constant<int, 0>{}, kt);
        if (kt + 1 < nk) step(std::integral_constant<int, 1>{}, kt + 1);
      }
    }
    const int em0 = m0 + wm * TM, en0 = n0 + wn * TN, etile = tile, esplit = split;
    g += wgs();
    const bool more = locate(g);
    __builtin_amdgcn_s_waitcnt(0xF | (0x7 << 4) | (0x3 << 14));  // lgkmcnt == 0
    wg_barrier();  // every wave is done with the stages
    if constexpr (E == Prod::Dh) {
      static_assert(TM == TWO_PARTS && TWO_PARTS == BK && WN * TM * TN * 4 <= NS * STAGE, "a wave's rows are a part");
      if (two) {  // the second part's sums to the first's
        float* x = reinterpret_cast<float*>(smem) + wn * TM * TN + lane;
        if (wm == 1) {
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) x[((i * FN + j) * 16 + r) * 64] = acc[i][j][r];
        }
        __builtin_amdgcn_s_waitcnt(0xF | (0x7 << 4) | (0x3 << 14));  // lgkmcnt == 0
        wg_barrier();
        if (wm == 0) {
#pragma unroll
          for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
              for (int r = 0; r < 16; ++r) acc[i][j][r] += x[((i * FN + j) * 16 + r) * 64];
        }
        __builtin_amdgcn_s_waitcnt(0xF | (0x7 << 4) | (0x3 << 14));
        wg_barrier();
      }
    }
    if (more) begin();

    // Lane l holds of each 32x32 block row l % 32, columns 8 g + 4 (l / 32) + 0..3, g = 0..3.
    int at = lane;
    asm volatile("" : "+v"(at));  // what follows is worked out here, not kept over the products
    const int l32 = at & 31, half = at >> 5;
    if constexpr (E == Prod::Stats || E == Prod::Logits) {
      const int c0 = en0 + 4 * half;
      auto col = [&](int j, int r) { return c0 + j * 32 + 8 * (r / 4) + r % 4; };
      if (en0 + TN > N) {  // columns past the vocabulary
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const bool past = col(j, r) >= N;
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[i][j][r] = past ? -INFINITY : acc[i][j][r];
          }
      }
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int row = em0 + i * 32 + l32;
        const int lab = a.lab_c && row < M ? a.lab_c[a.row0 + row] : -1;
        const int mine = lab - c0;  // 32 j + 8 (r / 4) + r % 4 where the label is among this lane's columns
        if (mine >= 0 && lab < en0 + TN && !(mine & 4)) {
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) t = mine == j * 32 + 8 * (r / 4) + r % 4 ? acc[i][j][r] : t;
          a.target[a.row0 + row] = t;
        }
        float m = -INFINITY;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) m = fmaxf(m, acc[i][j][r]);
        m = fmaxf(m, __shfl_xor(m, 32));
        const float z = m == -INFINITY ? 0.f : m;
        float l = 0.f;
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            if constexpr (E == Prod::Logits) {  // stored so; differences beside the sums would not fit the registers
              acc[i][j][r] -= z;
              l += exp_below(acc[i][j][r]);
            } else {
              l += exp_below(acc[i][j][r] - z);
            }
          }
        l += __shfl_xor(l, 32);
        if (half == 0 && row < M && en0 < N) a.part[(long)row * a.tiles + en0 / TN] = make_float2(m, l);
        if (a.part_at) {
          int lowest = INT32_MAX;
#pragma unroll
          for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r)
              lowest = acc[i][j][r] == m ? min(lowest, col(j, r)) : lowest;
          lowest = min(lowest, __shfl_xor(lowest, 32));
          if (half == 0 && row < M && en0 < N) a.part_at[(long)row * a.tiles + en0 / TN] = min(lowest, N - 1);
        }
      }
    }
    wait_dma<0>();  // the next tile's first k-tiles; then come the stores
    if constexpr (E != Prod::Stats) {
      char* mine = smem + NS * STAGE + wave * 4096;
      const int limit = E == Prod::Logits ? a.Vp : N;
      // 16-bit results, 64 columns of 32 rows at a time; else fp32 sums, 32 columns
      const bool packed = E == Prod::Logits || (splits == 1 && (E == Prod::Dh || (a.first && a.last)));
#pragma unroll
      for (int i = 0; i < FM; ++i) {
        const int mb = em0 + i * 32;
        if (mb >= M) continue;  // wave-uniform
        float left = 0.f;       // dh, not in shares: of this lane's row, for its label's row of w.  Asked for where it is needed: before the
                                // wait above it took as long, and 256 x 256 tiles have no registers for it
        const bf16* own = nullptr;
        if constexpr (E == Prod::Dh)
          if (packed) {
            const int m = min(mb + l32, M - 1);
            left = row_left(a, m);
            own = p.B + (long)a.lab_c[a.row0 + m] * p.ldb;
          }
        if (packed) {
#pragma unroll
          for (int j = 0; j < FN; j += 2) {
            const int nb = en0 + j * 32;
            if (nb >= limit) continue;
            uint2 c[8];
            if constexpr (E == Prod::Dh)
#pragma unroll
              for (int q = 0; q < 8; ++q) c[q] = *reinterpret_cast<const uint2*>(own + min(nb + 8 * q + 4 * half, N - 4));
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              float v[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) v[e] = acc[i][j + q / 4][q % 4 * 4 + e];
              if constexpr (E == Prod::Dh) {
                v[0] += left * __uint_as_float(c[q].x << 16);
                v[1] += left * __uint_as_float(c[q].x & 0xffff0000u);
                v[2] += left * __uint_as_float(c[q].y << 16);
                v[3] += left * __uint_as_float(c[q].y & 0xffff0000u);
              }
              uint2 w;
              if constexpr (E == Prod::Logits) {
                const half4 h = {(_Float16)v[0], (_Float16)v[1], (_Float16)v[2], (_Float16)v[3]};
                w = __builtin_bit_cast(uint2, h);
              } else {
                w = make_uint2(f2bf2(v[0] * unit, v[1] * unit), f2bf2(v[2] * unit, v[3] * unit));
              }
              *reinterpret_cast<uint2*>(mine + l32 * 128 + ((q ^ (l32 & 7)) << 4) + half * 8) = w;
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int row = 8 * q + (at >> 3), c = at & 7, m = mb + row, n = nb + 8 * c;
              const bf16x8 v = *reinterpret_cast<const bf16x8*>(mine + row * 128 + ((c ^ (row & 7)) << 4));
              if (m >= M || n >= limit) continue;
              bf16* o;
              if constexpr (E == Prod::Logits) o = static_cast<bf16*>(a.logits) + (long)m * a.Vp + n;
              else if constexpr (E == Prod::Dh) o = static_cast<bf16*>(a.dh) + (long)a.idx[a.row0 + m] * a.lddh + n;
              else o = static_cast<bf16*>(a.dw) + (long)m * a.lddw + n;
              *reinterpret_cast<bf16x8*>(o) = v;
            }
          }
        } else if constexpr (SHARED) {
#pragma unroll
          for (int j = 0; j < FN; ++j) {
            const int nb = en0 + j * 32;
            if (nb >= N) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q)
              *reinterpret_cast<float4*>(mine + l32 * 128 + (((2 * q + half) ^ (l32 & 7)) << 4)) =
                  make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int row = 8 * q + (at >> 3), c = at & 7, m = mb + row, n = nb + 4 * c;
              const f32x4 v = *reinterpret_cast<const f32x4*>(mine + row * 128 + ((c ^ (row & 7)) << 4));
              if (m >= M || n >= N) continue;
              if (splits > 1)
                *reinterpret_cast<f32x4*>(a.shares + ((long)esplit * tiles + etile) * (BM * BN) + (wm * TM + i * 32 + row) * BN + wn * TN + j * 32 + 4 * c) = v;
              else
                add_dw(a, m, n, unit, v);
            }
          }
        }
      }
    }
    if (!more) return;
  }
