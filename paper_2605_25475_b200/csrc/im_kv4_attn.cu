// Attention over the paged 4-bit KV cache (include/indexmem.h, im_kv4_attention).
//
// k_kv4_stream: the few query rows of a (sequence, KV head) against its entries.  The floor is one pass over the cache,
// 1.125 head_dim bytes per entry and KV head; next to it stands the work of unpacking: every code has to become an f16 in a
// register before a tensor core takes it, two per conversion instruction and two per multiplication with the block's scale.
//   split    The line of tiles (im_kv4_attn.cuh) in tiles of 32 entries; the workers are the warps of a persistent grid.
//   copies   Each warp has a ring of tiles of its own in shared memory, filled by one bulk copy per tile: the 16-token groups
//            of a page lie side by side with keys, values and scales.  No barrier but the warp's own.
//   scores   S^T = K Q^T with mma.m16n8k16: 16 entries on M, 8 rows on N.  The contraction's order is free, so a lane takes
//            the 16 bytes of its row as they lie (32 channels, two blocks) and Q is loaded in the same order once per run.
//            q is scaled by a power of two per row so that bf16 fits f16: K and Q are exact, S differs from the exact
//            scores by float32 summation alone.
//   values   O^T += V^T P^T, 16 channels on M: a register of A holds one channel of two entries, whose codes come
//            together by merging the nibbles of two rows before the conversion, so that one multiplication applies both
//            scales.  P comes from the score accumulators through movmatrix; it is kept relative to a reference maximum that is raised
//            only when a score exceeds it by 2^8, and 2^7 times as large, for f16's sake.  f16 inputs or float32
//            outputs take P as two f16 terms (2^-22), bf16 outputs one (2^-12, an eighth of their own step).
//   bound    Issue slots and the ALU pipe (302 warp instructions per 16 entries of a head; 64 and 56 % busy): 476,398 entries of 8
//            heads of 128, 549 MB, 112 us, 115 with the join (4.8 TB/s, 73 % of a copy).  20 warps with
//            shorter rings, or 12, were no faster.  One sequence of 513: 7.6 us alone, all round trips.
#include <math.h>

#include "im_kv4_attn.cuh"

namespace {

constexpr int TILE = 32;            // entries per tile: two groups
constexpr int RING_BYTES = 221184;  // shared memory of a CTA's rings

constexpr int warps_of(int d, int nt) { return d == 256 ? (nt == 1 ? 12 : 8) : nt == 1 ? 16 : 12; }
constexpr int stages_of(int d, int nt) { return RING_BYTES / (warps_of(d, nt) * 2 * kv4_group_bytes(d)); }

// bounded; the whole warp waits, and gets one answer
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
  uint32_t done = 0;
#pragma unroll 1
  for (uint32_t it = 0; it < IM_WAIT_LIMIT && !done; ++it)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
  return __all_sync(0xffffffffu, done);
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the first step of a sum: c = a b
__device__ __forceinline__ void mma_f16_first(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

template <int D, int NT, bool TWO, typename T, typename OutT>
__global__ void __launch_bounds__(warps_of(D, NT) * 32, 1)
k_kv4_stream(const AttnArgs a, const T* __restrict__ q, OutT* __restrict__ out, float* __restrict__ lse) {
  constexpr int WARPS = warps_of(D, NT), THREADS = WARPS * 32, STAGES = stages_of(D, NT), ROWS = 8 * NT;
  constexpr int GROUP = 18 * D, STAGE = 2 * GROUP;
  constexpr int KSTEPS = D / 16, MT = D / 16;   // MMA steps over the channels; channel tiles of O
  extern __shared__ __align__(128) uint8_t s_ring[];
  __shared__ long long s_cum[THREADS + 1];      // tiles ahead of a run of sequences
  __shared__ long long s_scan[WARPS];
  __shared__ __align__(8) unsigned long long s_bar[WARPS][STAGES];
  const Kv4& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, cq = lane & 3;
  pdl_release();
  if (lane < STAGES) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&s_bar[warp][lane])));
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  int workers, per;
  const Deal deal = deal_line<ROWS, TILE, THREADS>(a, s_cum, s_scan, (long long)gridDim.x * WARPS, &workers, &per);
  const int worker = warp * gridDim.x + blockIdx.x;  // neighbours in the line sit on different SMs
  const long long t0 = worker * deal.q + min((long long)worker, deal.rest), t1 = t0 + deal.q + (worker < deal.rest ? 1 : 0);
  if (worker >= workers || t0 >= t1) {
    empty_rows<D>(a, out, lse, warp, WARPS);
    return;
  }
  long long off;
  const int i0 = find_tile<ROWS, TILE, THREADS>(a, s_cum, per, t0, &off);
  // ---- the copies' side: sequence pi, KV head ph, row block pr, tile p_tile
  const Seq first = seq_of<ROWS, TILE>(a, i0);
  const int item0 = (off >> 31) == 0 ? (int)((unsigned)off / (unsigned)first.tiles) : (int)(off / first.tiles), tile0 = (int)(off - (long long)item0 * first.tiles);
  Seq sq = first;
  int pi = i0, ph = item0 / first.rb, pr = item0 % first.rb, p_tile = tile0;
  int left = (int)(t1 - t0);           // tiles still to be requested
  int win_base = 0, win_end = 0, win = 0;  // lane j: page of tile win_base + j (page_size 16: of group 2 win_base + j)
  uint32_t bad = 0;                    // bit 2 s + k: group k of stage s has no page
  uint8_t* ring = s_ring + warp * (STAGES * STAGE);
  const uint32_t bar0 = smem_u32(&s_bar[warp][0]), ring0 = smem_u32(ring);
  const size_t head_bytes = (size_t)(c.ps >> 4) * GROUP, page_bytes = head_bytes * c.Hkv;
  auto request = [&](int s) {
    if (p_tile >= win_end) {
      const int e = c.ps == 16 ? 2 * p_tile + lane : (int)(((long long)(p_tile + lane) * TILE) / c.ps);
      win = (long long)e * c.ps < sq.L ? a.table[(size_t)pi * c.max_pages + e] : -1;
      win_base = p_tile;
      win_end = p_tile + (c.ps == 16 ? 16 : 32);
    }
    const uint32_t bar = bar0 + 8 * s, dst = ring0 + s * STAGE;
    const uint8_t* src = c.pool + ph * head_bytes;
    bad &= ~(3u << (2 * s));
    if (c.ps == 16) {
      const int a0 = __shfl_sync(0xffffffffu, win, 2 * (p_tile - win_base)), a1 = __shfl_sync(0xffffffffu, win, 2 * (p_tile - win_base) + 1);
      const bool ok0 = (unsigned)a0 < (unsigned)c.n_pages, ok1 = (unsigned)a1 < (unsigned)c.n_pages;
      bad |= ((ok0 ? 0u : 1u) | (ok1 ? 0u : 2u)) << (2 * s);
      if (lane == 0) {
        if (!ok0 || (!ok1 && p_tile * TILE + 16 < sq.L)) atomicOr(c.status, IM_KV4_BAD_MAP);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)((ok0 + ok1) * GROUP)) : "memory");
        if (ok0) bulk_load(dst, src + a0 * page_bytes, GROUP, bar);
        if (ok1) bulk_load(dst + GROUP, src + a1 * page_bytes, GROUP, bar);
      }
    } else {
      const int page = __shfl_sync(0xffffffffu, win, p_tile - win_base);
      const bool ok = (unsigned)page < (unsigned)c.n_pages;
      if (!ok) bad |= 3u << (2 * s);
      if (lane == 0) {
        if (!ok) atomicOr(c.status, IM_KV4_BAD_MAP);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)(ok ? STAGE : 0)) : "memory");
        if (ok) bulk_load(dst, src + page * page_bytes + ((p_tile * TILE & (c.ps - 1)) >> 4) * GROUP, STAGE, bar);
      }
    }
    --left;
    if (++p_tile == sq.tiles) {  // on to the next item, if there is one in the run
      p_tile = win_end = 0;
      if (++pr == sq.rb) {
        pr = 0;
        if (++ph == c.Hkv && left > 0) {
          ph = 0;
          do sq = seq_of<ROWS, TILE>(a, ++pi);
          while (sq.tiles == 0);
        }
      }
    }
  };
  // row 8 nt + g of Q, channels in the order the keys' lanes take them (the first segment's are asked for ahead of the tiles: a
  // round trip less before the first product)
  uint32_t raw[NT][D / 8];
  auto load_q = [&](const Seq& sq_, int item_) {
    const int h = item_ / sq_.rb, row0 = (item_ % sq_.rb) * ROWS, rows = min(ROWS, sq_.nq * a.G - row0);
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int r = row0 + 8 * nt + g;
      const bool there = 8 * nt + g < rows;
      const T* src = q + (size_t)(sq_.first + (there ? r / a.G : 0)) * a.q_stride + (size_t)(h * a.G + (there ? r % a.G : 0)) * D;
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {  // 8 channels each
        const int at = D == 64 ? 16 * cq + 8 * b : 128 * (b / 4) + 32 * cq + 8 * (b % 4);
        const uint4 v = there ? *reinterpret_cast<const uint4*>(src + at) : make_uint4(0u, 0u, 0u, 0u);
        raw[nt][4 * b] = v.x, raw[nt][4 * b + 1] = v.y, raw[nt][4 * b + 2] = v.z, raw[nt][4 * b + 3] = v.w;
      }
    }
  };
  load_q(first, item0);
#pragma unroll 1
  for (int s = 0; s < STAGES && left > 0; ++s) request(s);

  // ---- the arithmetic's side
  Seq cs = first;
  int ci = i0, item = item0, tile = tile0, todo = (int)(t1 - t0), stage = 0;
  uint32_t parity = 0;
  bool fine = true;
  while (todo > 0 && fine) {
    // one segment: tiles [tile, end) of item
    const int end = min(cs.tiles, tile + todo);
    const int h = item / cs.rb, row0 = (item % cs.rb) * ROWS, rows = min(ROWS, cs.nq * a.G - row0);
    const long long base = t1 - todo - tile;  // first tile of the item in the line
    uint32_t qf[NT][KSTEPS][2];
    float f[NT][2], mref[NT][2], l[NT][2];
    int lim[NT][2];
    int lim_min = cs.L;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      float amax = 0.f;
      int ex = 0;
      if constexpr (std::is_same<T, bf16>::value) {
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const float2 x = two_of((const bf16*)nullptr, raw[nt][k]);
          amax = fmaxf(amax, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        ex = row_exponent(amax);
        const float by = exp2i(ex);
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const float2 x = two_of((const bf16*)nullptr, raw[nt][k]);
          raw[nt][k] = pack_f16(x.x * by, x.y * by);
        }
      }
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) {
        qf[nt][k][0] = raw[nt][2 * k];
        qf[nt][k][1] = raw[nt][2 * k + 1];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // columns 2 cq + k of the scores
        const int col = 8 * nt + 2 * cq + k;
        const int e = __shfl_sync(0xffffffffu, ex, (2 * cq + k) * 4);
        f[nt][k] = row_factor(a, h, e);
        mref[nt][k] = NO_MAX;
        l[nt][k] = 0.f;
        const int j = (row0 + col) / a.G;
        lim[nt][k] = col >= rows ? 0 : a.causal ? max(0, min(cs.L, cs.L - cs.nq + j + 1)) : cs.L;
        if (col < rows) lim_min = min(lim_min, lim[nt][k]);
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) lim_min = min(lim_min, __shfl_xor_sync(0xffffffffu, lim_min, o));
    constexpr int FLUSH_TILES = std::is_same<OutT, float>::value ? FLUSH_STEPS / (TWO ? 4 : 2) : 1 << 30;
    float* const place = a.ws.part + (size_t)(2 * worker + (t0 <= base ? 1 : 0)) * ROWS * (D + 4);  // of the segment's partial result
    int fresh = 0, flushed = 0;  // tiles since the accumulators were emptied; how often they were
    float fref[NT][2];           // reference maximum of what lies there
    float o[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[m][nt][k] = 0.f;

    // what lies in the segment's place, brought to the present reference maximum and added to the accumulators
    auto add_flushed = [&](auto store) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int col = 8 * nt + 2 * cq + k;
          if (col >= rows) continue;
          float* p = place + (size_t)col * (D + 4) + g * (D / 8);
          const float by = flushed ? ex2(fref[nt][k] - mref[nt][k]) : 0.f;
#pragma unroll
          for (int m = 0; m < MT; m += 2) {
            if (flushed) {
              const float4 y = *reinterpret_cast<const float4*>(p + 2 * m);
              o[m][nt][k] = fmaf(y.x, by, o[m][nt][k]), o[m][nt][k + 2] = fmaf(y.y, by, o[m][nt][k + 2]);
              o[m + 1][nt][k] = fmaf(y.z, by, o[m + 1][nt][k]), o[m + 1][nt][k + 2] = fmaf(y.w, by, o[m + 1][nt][k + 2]);
            }
            if constexpr (decltype(store)::value) {
              *reinterpret_cast<float4*>(p + 2 * m) = make_float4(o[m][nt][k], o[m][nt][k + 2], o[m + 1][nt][k], o[m + 1][nt][k + 2]);
              o[m][nt][k] = o[m][nt][k + 2] = o[m + 1][nt][k] = o[m + 1][nt][k + 2] = 0.f;
            }
          }
          fref[nt][k] = mref[nt][k];
        }
    };
    for (; tile < end; ++tile) {
      if (FLUSH_TILES < (1 << 30) && fresh == FLUSH_TILES) {
        add_flushed(std::true_type{});
        fresh = 0;
        ++flushed;
      }
      ++fresh;
      if (!mbar_wait(bar0 + 8 * stage, parity)) {
        fine = false;
        break;
      }
      const uint8_t* st = ring + stage * STAGE;
      const uint32_t no_page = (bad >> (2 * stage)) & 3u;
      const int e0 = tile * TILE;
      // (one body for the tiles that every row sees whole, one for the others)
      auto compute = [&](auto whole) {
        constexpr bool WHOLE = decltype(whole)::value;
        // entry of MMA row i within a group: i ^ (i >> 1 & 1), so that the lanes of a V load see both halves of the banks
        const int ra = g ^ ((g >> 1) & 1);
        float sc[2][NT][4];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* gp = st + u * GROUP;
#pragma unroll
          for (int half = 0; half < (D == 256 ? 2 : 1); ++half) {
            constexpr int W = D == 64 ? 2 : 4;  // words of a lane: 8 channels each
            uint32_t ka[W], kb[W], sa, sb;
            const int at = ra * (D / 2) + half * 64 + cq * 4 * W;
            if constexpr (W == 4) {
              const uint4 x = *reinterpret_cast<const uint4*>(gp + at), y = *reinterpret_cast<const uint4*>(gp + at + 4 * D);
              ka[0] = x.x, ka[1] = x.y, ka[2] = x.z, ka[3] = x.w;
              kb[0] = y.x, kb[1] = y.y, kb[2] = y.z, kb[3] = y.w;
              sa = *reinterpret_cast<const uint16_t*>(gp + 8 * D + ra * (D / 16) + half * 8 + 2 * cq);
              sb = *reinterpret_cast<const uint16_t*>(gp + 8 * D + (ra + 8) * (D / 16) + half * 8 + 2 * cq);
            } else {
              const uint2 x = *reinterpret_cast<const uint2*>(gp + at), y = *reinterpret_cast<const uint2*>(gp + at + 4 * D);
              ka[0] = x.x, ka[1] = x.y;
              kb[0] = y.x, kb[1] = y.y;
              sa = gp[8 * D + ra * (D / 16) + cq];
              sb = gp[8 * D + (ra + 8) * (D / 16) + cq];
            }
            sa = kv4_f16x2_e4m3(sa);
            sb = kv4_f16x2_e4m3(sb);
            const uint32_t fa[2] = {__byte_perm(sa, sa, 0x1010), __byte_perm(sa, sa, 0x3232)};
            const uint32_t fb[2] = {__byte_perm(sb, sb, 0x1010), __byte_perm(sb, sb, 0x3232)};
#pragma unroll
            for (int w = 0; w < W; ++w) {
              uint32_t x[4], y[4];
              kv4_f16_e2m1(ka[w], x);
              kv4_f16_e2m1(kb[w], y);
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                x[k] = mul2(x[k], fa[w / 2]);
                y[k] = mul2(y[k], fb[w / 2]);
              }
#pragma unroll
              for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                  const int step = half * 8 + 2 * w + k;
                  if (step == 0) mma_f16_first(sc[u][nt], x[0], y[0], x[1], y[1], qf[nt][0][0], qf[nt][0][1]);
                  else mma_f16(sc[u][nt], x[2 * k], y[2 * k], x[2 * k + 1], y[2 * k + 1], qf[nt][step][0], qf[nt][step][1]);
                }
            }
          }
        }
        if constexpr (!WHOLE) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int e = e0 + 16 * u + ra + 8 * (k >> 1);
              const bool gone = (no_page >> u) & 1u;
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                if (gone || e >= lim[nt][k & 1]) sc[u][nt][k] = NEG_INF;
            }
        }
        // softmax in base 2, relative to mref (7 below the reference maximum)
        float x[2][NT][4], top = NEG_INF;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 4; k += 2) {
              const float2 e = fma2(make_float2(sc[u][nt][k], sc[u][nt][k + 1]), make_float2(f[nt][0], f[nt][1]), make_float2(-mref[nt][0], -mref[nt][1]));
              x[u][nt][k] = e.x;
              x[u][nt][k + 1] = e.y;
              top = max3(top, e.x, e.y);
            }
        if (__any_sync(0xffffffffu, top > 15.0f)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float m = fmaxf(fmaxf(sc[0][nt][k], sc[0][nt][k + 2]), fmaxf(sc[1][nt][k], sc[1][nt][k + 2])) * f[nt][k];
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
              const float next = m - mref[nt][k] > 15.0f ? m - 7.0f : mref[nt][k];
              const float corr = ex2(mref[nt][k] - next);
              mref[nt][k] = next;
              l[nt][k] *= corr;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                o[mt][nt][k] *= corr;
                o[mt][nt][k + 2] *= corr;
              }
#pragma unroll
              for (int v = 0; v < 4; ++v) x[v >> 1][nt][k + 2 * (v & 1)] = fmaf(sc[v >> 1][nt][k + 2 * (v & 1)], f[nt][k], -next);
            }
        }
        uint32_t pb[2][NT][2], pl[2][NT][2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            float p[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) p[k] = ex2(x[u][nt][k]);
            const float2 sum = add2(make_float2(l[nt][0], l[nt][1]), add2(make_float2(p[0], p[1]), make_float2(p[2], p[3])));
            l[nt][0] = sum.x;
            l[nt][1] = sum.y;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t hi = pack_f16(p[2 * k], p[2 * k + 1]);
              pb[u][nt][k] = transpose8x8(hi);
              if constexpr (TWO) {
                const float2 back = kv4_unpack_f16(hi);
                pl[u][nt][k] = transpose8x8(pack_f16(p[2 * k] - back.x, p[2 * k + 1] - back.y));
              }
            }
          }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const uint8_t* gp = st + u * GROUP + 9 * D;
          // the lane's entries: MMA columns 2 cq, 2 cq + 1, and 8 further
          const int ta = 2 * cq + (cq & 1), tb = 2 * cq + 1 - (cq & 1);
          constexpr int VW = D / 64;  // words of 8 channels per entry and lane: channels 8 VW g ..
          uint32_t code[4][VW];
          uint32_t s[2][D == 256 ? 2 : 1];  // scales of (ta, tb) and (ta + 8, tb + 8), per block of the lane
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint8_t* p = gp + ((k & 1 ? tb : ta) + 8 * (k >> 1)) * (D / 2) + g * 4 * VW;
            if constexpr (VW == 1) code[k][0] = *reinterpret_cast<const uint32_t*>(p);
            if constexpr (VW == 2) {
              const uint2 v = *reinterpret_cast<const uint2*>(p);
              code[k][0] = v.x, code[k][1] = v.y;
            }
            if constexpr (VW == 4) {
              const uint4 v = *reinterpret_cast<const uint4*>(p);
              code[k][0] = v.x, code[k][1] = v.y, code[k][2] = v.z, code[k][3] = v.w;
            }
          }
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint8_t* p = gp + 8 * D + (D == 64 ? g >> 1 : D == 128 ? g : 2 * g);
            uint32_t sa, sb;
            if constexpr (D == 256) {
              sa = *reinterpret_cast<const uint16_t*>(p + (ta + 8 * k) * (D / 16));
              sb = *reinterpret_cast<const uint16_t*>(p + (tb + 8 * k) * (D / 16));
            } else {
              sa = p[(ta + 8 * k) * (D / 16)];
              sb = p[(tb + 8 * k) * (D / 16)];
            }
            if constexpr (!WHOLE) {  // what lies behind the sequence may be anything, a scale's NaN too
              const int e = e0 + 16 * u + 8 * k;
              if (((no_page >> u) & 1u) || e + ta >= cs.L) sa = 0;
              if (((no_page >> u) & 1u) || e + tb >= cs.L) sb = 0;
            }
            s[k][0] = kv4_f16x2_e4m3(D == 256 ? __byte_perm(sa, sb, 0x0040) : sa | sb << 8);
            if constexpr (D == 256) s[k][1] = kv4_f16x2_e4m3(__byte_perm(sa, sb, 0x0051));
          }
#pragma unroll
          for (int w = 0; w < VW; ++w) {
            uint32_t lo[2][4], hi[2][4];  // even and odd channels of the word, entries (ta, tb) / (ta + 8, tb + 8)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint32_t p = code[2 * k][w], r = code[2 * k + 1][w];
              kv4_f16_e2m1((p & 0x0f0f0f0fu) | ((r << 4) & 0xf0f0f0f0u), lo[k]);
              kv4_f16_e2m1(((p >> 4) & 0x0f0f0f0fu) | (r & 0xf0f0f0f0u), hi[k]);
              const uint32_t by = s[k][D == 256 ? w / 2 : 0];
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                lo[k][b] = mul2(lo[k][b], by);
                hi[k][b] = mul2(hi[k][b], by);
              }
            }
#pragma unroll
            for (int b = 0; b < 4; ++b)
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) {
                mma_f16(o[4 * w + b][nt], lo[0][b], hi[0][b], lo[1][b], hi[1][b], pb[u][nt][0], pb[u][nt][1]);
                if constexpr (TWO) mma_f16(o[4 * w + b][nt], lo[0][b], hi[0][b], lo[1][b], hi[1][b], pl[u][nt][0], pl[u][nt][1]);
              }
          }
        }
      };
      if (__all_sync(0xffffffffu, e0 + TILE <= lim_min && no_page == 0)) compute(std::true_type{});
      else compute(std::false_type{});
      __syncwarp();  // every lane is through with the stage
      if (left > 0) request(stage);
      if (++stage == STAGES) {
        stage = 0;
        parity ^= 1u;
      }
      --todo;
    }
    if (!fine) break;
    // ---- the segment's result
    if (FLUSH_TILES < (1 << 30) && flushed) add_flushed(std::false_type{});
    const bool complete = base >= t0 && end == cs.tiles;  // the item begins and ends here
    const float vup = kv4_pow2(kv4_exp(c.v_exp, h));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[nt][k] += __shfl_xor_sync(0xffffffffu, l[nt][k], x);
        const int col = 8 * nt + 2 * cq + k;
        if (col >= rows) continue;
        if (complete) {
          const int r = row0 + col;
          const size_t at = (size_t)(cs.first + r / a.G) * a.H + h * a.G + r % a.G;
          const float inv = l[nt][k] == 0.f ? 0.f : vup / l[nt][k];
          OutT* dst = out + at * D + g * (D / 8);
#pragma unroll
          for (int m = 0; m < MT; m += 4) {
            float v[8];
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              v[2 * b] = o[m + b][nt][k] * inv;
              v[2 * b + 1] = o[m + b][nt][k + 2] * inv;
            }
            put8(dst + 2 * m, v);
          }
          if (lse && g == 0) lse[at] = l[nt][k] == 0.f ? NEG_INF : (mref[nt][k] + log2f(l[nt][k])) * LN2;
        } else {
          float* dst = place + (size_t)col * (D + 4);
#pragma unroll
          for (int m = 0; m < MT; m += 2)
            *reinterpret_cast<float4*>(dst + g * (D / 8) + 2 * m) = make_float4(o[m][nt][k], o[m][nt][k + 2], o[m + 1][nt][k], o[m + 1][nt][k + 2]);
          if (g == 0) *reinterpret_cast<float2*>(dst + D) = make_float2(mref[nt][k], l[nt][k]);
        }
      }
    // ---- next item
    if (todo > 0) {
      tile = 0;
      if (++item == cs.rb * c.Hkv) {
        item = 0;
        do cs = seq_of<ROWS, TILE>(a, ++ci);
        while (cs.tiles == 0);
      }
      load_q(cs, item);
    }
  }
  if (!fine) {
    // a wait gave up: report it, and give the copies in flight time to land (with a limit) before the block's memory is handed on
    if (lane == 0) atomicOr(c.status, IM_KV4_TIMEOUT);
    for (int k = 0; k < 64; ++k) __nanosleep(1000);
  }
  empty_rows<D>(a, out, lse, warp, WARPS);
}

// ------------------------------------------------------------------ host side
size_t workspace(const Kv4& c, long long rows, int nt, uint8_t* base, AttnWs* ws) {
  // no more workers than tiles
  const double tiles = (double)c.n_seqs * ((double)c.max_pages * c.ps / TILE + 1) * c.Hkv * (double)((rows + 8 * nt - 1) / (8 * nt));
  const int most = MOST_SMS * warps_of(c.d, nt);
  const size_t workers = tiles < most ? (size_t)tiles : (size_t)most;
  const size_t cum = 256, part = cum + kv4_align(8 * (size_t)c.n_seqs);
  if (ws) *ws = {(Deal*)base, (long long*)(base + cum), nullptr, (float*)(base + part), (int)workers};
  return part + kv4_align(2 * workers * 8 * nt * (c.d + 4) * 4);
}

template <int D, int NT, bool TWO, typename T, typename OutT>
cudaError_t launch(const AttnArgs& a, const void* q, void* out, float* lse, int grid, int rows, cudaStream_t s) {
  static bool flags[64] = {};
  bool* done = im_device_flag(flags);
  constexpr int smem = stages_of(D, NT) * warps_of(D, NT) * 2 * kv4_group_bytes(D);
  if (!done) return cudaErrorInvalidDevice;
  if (!*done) {
    const cudaError_t e = cudaFuncSetAttribute(k_kv4_stream<D, NT, TWO, T, OutT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    *done = true;
  }
  cudaError_t e = kv4_launch(k_kv4_stream<D, NT, TWO, T, OutT>, dim3(grid), warps_of(D, NT) * 32, smem, s, false, a, (const T*)q, (OutT*)out, lse);
  if (e == cudaSuccess)
    e = kv4_launch(k_kv4_join_seqs<D, 8 * NT, TILE, 4, OutT>, dim3(a.c.n_seqs, a.c.Hkv, rows < 32 ? (rows + 1) / 2 : 16), JOIN_WARPS * 32, 0, s, true, a, (OutT*)out, lse);
  return e;
}

template <int D, int NT>
cudaError_t launch_types(const AttnArgs& a, int dtype, int out_f32, const void* q, void* out, float* lse, int grid, int rows, cudaStream_t s) {
  if (dtype == IM_BF16)
    return out_f32 ? launch<D, NT, true, bf16, float>(a, q, out, lse, grid, rows, s) : launch<D, NT, false, bf16, bf16>(a, q, out, lse, grid, rows, s);
  return out_f32 ? launch<D, NT, true, __half, float>(a, q, out, lse, grid, rows, s) : launch<D, NT, true, __half, __half>(a, q, out, lse, grid, rows, s);
}

// query rows of a KV head in the longest sequence
long long rows_of(const Kv4& c, bool ragged, int max_q, int n_q_heads) { return (long long)(ragged ? (max_q > 0 ? max_q : 1) : 1) * (n_q_heads / c.Hkv); }
// Which kernel.  The streaming kernel unpacks the cache again for every 16 rows (two column tiles), the other one once for up to
// 256, at a higher price per tile, and higher again where P has two terms.  8 sequences of 12000 entries, 8 KV heads of 128,
// streaming / other: 24 rows 85 / 106 us, 36 rows 117 / 107 (float32 outputs 149 / 143), 52 rows 143 / 108 (187 / 145); 4 KV
// heads, 35 rows, 5 tokens of 7 heads each, 100,484 entries: 72 / 82 with float32 outputs.
bool by_chunks(const Kv4& c, long long rows, bool two_terms) { return rows > (two_terms ? 48 : 32) && c.d != 256; }

}  // namespace

int kv4_sm_count() {
  static int counts[64] = {};  // (threads that look it up at the same time store the same value)
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (!counts[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    counts[dev] = n < MOST_SMS ? n : MOST_SMS;
  }
  return counts[dev];
}

size_t kv4_attention_workspace(const Kv4& c, int max_q, int n_q_heads) {
  const long long rows = rows_of(c, true, max_q, n_q_heads);
  const size_t stream = workspace(c, rows, rows <= 8 ? 1 : 2, nullptr, nullptr);
  if (!by_chunks(c, rows, false)) return stream;
  const size_t chunk = kv4_chunk_workspace(c, nullptr, nullptr);
  return by_chunks(c, rows, true) || chunk > stream ? chunk : stream;
}

extern "C" int im_kv4_attention(const im_kv4* cache, const im_kv4_map* map, int dtype, const void* q, long long q_stride, int n_tokens,
                                const int32_t* cu_q, int max_q, int n_q_heads, float softmax_scale, int causal, void* out, int out_f32,
                                float* lse, void* workspace_, size_t workspace_bytes, void* cuda_stream) {
  const char* fn = "im_kv4_attention";
  Kv4 c;
  int rc = kv4_describe(cache, fn, &c);
  if (rc == IM_OK) rc = kv4_check_map(map, fn);
  if (rc != IM_OK) return rc;
  if (dtype != IM_BF16 && dtype != IM_F16) return kv4_fail(IM_ERR_ARG, fn, "queries are bf16 or f16");
  if (n_q_heads < 1 || n_q_heads % c.Hkv || n_q_heads > 65535) return kv4_fail(IM_ERR_ARG, fn, "n_q_heads must be a multiple of n_kv_heads");
  if (n_tokens < 0 || max_q < 0 || (!cu_q && n_tokens != c.n_seqs)) return kv4_fail(IM_ERR_ARG, fn, "bad token count");
  if (n_tokens && (!q || !out)) return kv4_fail(IM_ERR_ARG, fn, "null tensor");
  const long long dense = (long long)n_q_heads * c.d;
  if (!q_stride) q_stride = dense;
  if (q_stride < dense || q_stride % 8 || (((uintptr_t)q | (uintptr_t)out) & 15) || ((uintptr_t)lse & 3))
    return kv4_fail(IM_ERR_ARG, fn, "the token stride must be a multiple of 8 elements, no shorter than a token; bases 16-byte aligned");
  if (!(softmax_scale >= 0.f) || isinf(softmax_scale)) return kv4_fail(IM_ERR_ARG, fn, "softmax_scale must be positive (0: 1/sqrt(head_dim))");
  if (!workspace_ || ((uintptr_t)workspace_ & 255) || workspace_bytes < kv4_attention_workspace(c, cu_q ? max_q : 1, n_q_heads))
    return kv4_fail(IM_ERR_CAPACITY, fn, "workspace missing, misaligned or too small");
  if (!n_tokens) return IM_OK;
  const int grid = kv4_sm_count();
  if (grid < 1) return kv4_fail(IM_ERR_CUDA, fn, "no usable CUDA device");
  AttnArgs a = {c, map->table, map->lens, cu_q, q_stride, n_tokens, n_q_heads, n_q_heads / c.Hkv, causal ? 1 : 0,
                softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)c.d), {}};
  const long long rows = rows_of(c, cu_q != nullptr, max_q, n_q_heads);
  cudaStream_t s = (cudaStream_t)cuda_stream;
  if (by_chunks(c, rows, out_f32 || dtype == IM_F16)) {
    kv4_chunk_workspace(c, (uint8_t*)workspace_, &a.ws);
    const cudaError_t e = kv4_launch_chunk(a, dtype, out_f32, q, out, lse, grid, s);
    return e == cudaSuccess ? IM_OK : im_fail_message(IM_ERR_CUDA, cudaGetErrorString(e));
  }
  const int nt = rows <= 8 ? 1 : 2, few = rows < 32 ? (int)rows : 32;
  workspace(c, rows, nt, (uint8_t*)workspace_, &a.ws);
  auto go = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    return nt == 1 ? launch_types<D, 1>(a, dtype, out_f32, q, out, lse, grid, few, s) : launch_types<D, 2>(a, dtype, out_f32, q, out, lse, grid, few, s);
  };
  const cudaError_t e = c.d == 64    ? go(std::integral_constant<int, 64>{})
                        : c.d == 128 ? go(std::integral_constant<int, 128>{})
                                     : go(std::integral_constant<int, 256>{});
  return e == cudaSuccess ? IM_OK : im_fail_message(IM_ERR_CUDA, cudaGetErrorString(e));
}
