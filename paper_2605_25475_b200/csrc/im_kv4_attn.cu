// Attention over the paged 4-bit KV cache (include/indexmem.h, im_kv4_attention).
//
// k_kv4_stream: the few query rows of a (sequence, KV head) against its entries.  The floor is one pass over the cache,
// 1.125 head_dim bytes per entry and KV head; next to it stands the work of unpacking: every code has to become an f16 in a
// register before a tensor core takes it, two per conversion instruction and two per multiplication with the block's scale.
//   split    The entries of all (sequence, KV head, row block) items form one line of tiles of 32; every warp of a
//            persistent grid gets an equal run of it, whatever the lengths are (they are known to the device alone).  A run that
//            does not cover an item writes (sum of p v, reference maximum, sum of p) to the workspace, and k_kv4_merge adds those up
//            in order of the warps: results do not depend on timing.
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
#include <math.h>

#include <type_traits>

#include "im_kv4.cuh"

namespace {

constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float NO_MAX = -1e30f;         // reference maximum of a row that has seen nothing
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int TILE = 32;                 // entries per tile: two groups
constexpr int RING_BYTES = 221184;       // shared memory of a CTA's rings
constexpr int MERGE_THREADS = 128;

constexpr int warps_of(int d, int nt) { return d == 256 ? (nt == 1 ? 12 : 8) : nt == 1 ? 16 : 12; }
constexpr int stages_of(int d, int nt) { return RING_BYTES / (warps_of(d, nt) * 2 * kv4_group_bytes(d)); }

// how a call's tiles are dealt to the warps (written by CTA 0 of k_kv4_stream for k_kv4_merge)
struct Deal {
  long long q, rest;  // the first `rest` workers get q + 1 tiles, the others q
};
struct AttnWs {
  Deal* deal;
  long long* cum;  // [n_seqs] tiles ahead of the sequence
  float* part;     // [2 * workers][8 NT][D + 2]
};

struct AttnArgs {
  Kv4 c;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
  long long q_stride;
  int n_tokens, H, G, causal;
  float scale;
  AttnWs ws;
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity) {
  for (uint32_t it = 0; it < IM_WAIT_LIMIT; ++it) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    if (done) return true;
  }
  return false;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float2 two_of(const bf16*, uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack_two(const bf16*, float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t pack_two(const __half*, float a, float b) { return pack_f16(a, b); }

// query tokens of sequence i, clipped to the tensors
__device__ __forceinline__ void queries_of(const AttnArgs& a, int i, int* first, int* count) {
  if (!a.cu) {
    *first = i;
    *count = 1;
    return;
  }
  const int s = max(0, min(a.n_tokens, a.cu[i])), e = max(s, min(a.n_tokens, a.cu[i + 1]));
  *first = s;
  *count = e - s;
}
__device__ __forceinline__ int length_of(const AttnArgs& a, int i) {
  return (int)max(0ll, min((long long)a.lens[i], (long long)a.c.max_pages * a.c.ps));
}

// the line of tiles: sequence-major, then KV head, then row block
struct Seq {
  int L, first, nq, tiles, rb;  // rb: row blocks
};
template <int ROWS>
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int i) {
  Seq s;
  s.L = length_of(a, i);
  queries_of(a, i, &s.first, &s.nq);
  s.rb = (int)(((long long)s.nq * a.G + ROWS - 1) / ROWS);
  s.tiles = s.nq ? (s.L + TILE - 1) / TILE : 0;
  return s;
}
__device__ __forceinline__ long long work_of(const AttnArgs& a, const Seq& s) { return (long long)s.tiles * s.rb * a.c.Hkv; }

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
  // ---- the line of tiles: every CTA adds the sequences up for itself
  const int per = (c.n_seqs + THREADS - 1) / THREADS;
  {
    long long mine = 0;
    for (int i = tid * per; i < min(c.n_seqs, tid * per + per); ++i) mine += work_of(a, seq_of<ROWS>(a, i));
    long long incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, incl, o);
      if (lane >= o) incl += u;
    }
    if (lane == 31) s_scan[warp] = incl;
    if (lane < STAGES) asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(smem_u32(&s_bar[warp][lane])));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    long long before = 0;
    for (int w = 0; w < warp; ++w) before += s_scan[w];
    s_cum[tid] = before + incl - mine;
    if (tid == THREADS - 1) s_cum[THREADS] = before + incl;
    __syncthreads();
  }
  const long long total = s_cum[THREADS];
  const int workers = (int)min((long long)gridDim.x * WARPS, max(1ll, total));
  const long long quo = total / workers, rest = total % workers;
  if (blockIdx.x == 0) {
    if (tid == 0) *a.ws.deal = {quo, rest};
    long long at = s_cum[tid];
    for (int i = tid * per; i < min(c.n_seqs, tid * per + per); ++i) {
      a.ws.cum[i] = at;
      at += work_of(a, seq_of<ROWS>(a, i));
    }
  }
  const int worker = warp * gridDim.x + blockIdx.x;  // neighbours in the line sit on different SMs
  if (worker >= workers) return;
  const long long t0 = worker * quo + min((long long)worker, rest), t1 = t0 + quo + (worker < rest ? 1 : 0);
  if (t0 >= t1) return;
  // ---- where the run starts
  int i0;
  long long off;
  {
    int lo = 0, hi = THREADS;  // s_cum[lo] <= t0 < s_cum[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (s_cum[mid] <= t0) lo = mid;
      else hi = mid;
    }
    i0 = lo * per;
    off = t0 - s_cum[lo];
    while (true) {
      const long long w = work_of(a, seq_of<ROWS>(a, i0));
      if (off < w) break;
      off -= w;
      ++i0;
    }
  }
  // ---- the copies' side: sequence pi, item (head, row block) of it, tile pt of its tiles
  int pi = i0, p_item, p_tile;
  Seq ps_ = seq_of<ROWS>(a, i0);
  p_item = (int)(off / ps_.tiles);
  p_tile = (int)(off % ps_.tiles);
  int left = (int)(t1 - t0);           // tiles still to be requested
  int win_base = -1, win = 0;          // lane j: page of tile win_base + j (page_size 16: of group 2 win_base + j)
  const int win_tiles = c.ps == 16 ? 16 : 32;
  uint32_t bad = 0;                    // bit 2 s + k: group k of stage s has no page
  uint8_t* ring = s_ring + warp * (STAGES * STAGE);
  const uint32_t bar0 = smem_u32(&s_bar[warp][0]), ring0 = smem_u32(ring);
  auto request = [&](int s) {
    const int h = p_item / ps_.rb;
    if (win_base < 0 || p_tile >= win_base + win_tiles || p_tile < win_base) {
      win_base = p_tile;
      const int e = c.ps == 16 ? 2 * win_base + lane : (int)(((long long)(win_base + lane) * TILE) / c.ps);
      const int pages = (ps_.L + c.ps - 1) / c.ps;
      win = e < pages ? a.table[(size_t)pi * c.max_pages + e] : -1;
    }
    const uint32_t bar = bar0 + 8 * s, dst = ring0 + s * STAGE;
    bad &= ~(3u << (2 * s));
    if (c.ps == 16) {
      const int a0 = __shfl_sync(0xffffffffu, win, 2 * (p_tile - win_base)), a1 = __shfl_sync(0xffffffffu, win, 2 * (p_tile - win_base) + 1);
      const bool ok0 = a0 >= 0 && a0 < c.n_pages, ok1 = a1 >= 0 && a1 < c.n_pages;
      bad |= ((ok0 ? 0u : 1u) | (ok1 ? 0u : 2u)) << (2 * s);
      if (lane == 0) {
        if (!ok0 || (!ok1 && p_tile * TILE + 16 < ps_.L)) atomicOr(c.status, IM_KV4_BAD_MAP);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)((ok0 + ok1) * GROUP)) : "memory");
        if (ok0) bulk_load(dst, kv4_group(c, a0, h, 0), GROUP, bar);
        if (ok1) bulk_load(dst + GROUP, kv4_group(c, a1, h, 0), GROUP, bar);
      }
    } else {
      const int page = __shfl_sync(0xffffffffu, win, p_tile - win_base);
      const bool ok = page >= 0 && page < c.n_pages;
      bad |= (ok ? 0u : 3u) << (2 * s);
      if (lane == 0) {
        if (!ok) atomicOr(c.status, IM_KV4_BAD_MAP);
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"((uint32_t)(ok ? STAGE : 0)) : "memory");
        if (ok) bulk_load(dst, kv4_group(c, page, h, (p_tile * TILE & (c.ps - 1)) >> 4), STAGE, bar);
      }
    }
    if (++p_tile == ps_.tiles) {
      p_tile = 0;
      win_base = -1;
      if (++p_item == ps_.rb * c.Hkv && left > 1) {
        p_item = 0;
        do ps_ = seq_of<ROWS>(a, ++pi);
        while (ps_.tiles == 0);  // (there is work ahead: left > 1)
      }
    }
    --left;
  };
#pragma unroll 1
  for (int s = 0; s < STAGES && left > 0; ++s) request(s);

  // ---- the arithmetic's side
  int ci = i0, item, tile;
  Seq cs = seq_of<ROWS>(a, i0);
  item = (int)(off / cs.tiles);
  tile = (int)(off % cs.tiles);
  long long todo = t1 - t0;
  int stage = 0;
  uint32_t parity = 0;
  bool fine = true;
  while (todo > 0 && fine) {
    // one segment: tiles [tile, end) of item
    const int end = (int)min((long long)cs.tiles, tile + todo);
    const int h = item / cs.rb, row0 = (item % cs.rb) * ROWS, rows = min(ROWS, cs.nq * a.G - row0);
    const long long base = t1 - todo - tile;  // first tile of the item in the line
    uint32_t qf[NT][KSTEPS][2];
    float f[NT][2], mref[NT][2], l[NT][2];
    int lim[NT][2];
    int lim_min = cs.L;
    const float up = a.scale * LOG2E * kv4_pow2(kv4_exp(c.k_exp, h));
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      // row 8 nt + g: channels in the order the keys' lanes take them
      const int r = row0 + 8 * nt + g;
      const bool there = 8 * nt + g < rows;
      const T* src = q + (size_t)(cs.first + (there ? r / a.G : 0)) * a.q_stride + (size_t)(h * a.G + (there ? r % a.G : 0)) * D;
      float amax = 0.f;
      uint32_t raw[D / 8];
#pragma unroll
      for (int b = 0; b < D / 32; ++b) {  // 8 channels each
        const int at = D == 64 ? 16 * cq + 8 * b : 128 * (b / 4) + 32 * cq + 8 * (b % 4);
        const uint4 v = there ? *reinterpret_cast<const uint4*>(src + at) : make_uint4(0u, 0u, 0u, 0u);
        raw[4 * b] = v.x, raw[4 * b + 1] = v.y, raw[4 * b + 2] = v.z, raw[4 * b + 3] = v.w;
      }
      int ex = 0;
      if constexpr (std::is_same<T, bf16>::value) {
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const float2 x = two_of(src, raw[k]);
          amax = fmaxf(amax, fmaxf(fabsf(x.x), fabsf(x.y)));
        }
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
        ex = max(-114, min(100, 13 - ((int)(__float_as_uint(amax) >> 23) - 127)));  // largest value to [2^13, 2^14)
        const float by = __uint_as_float((uint32_t)(127 + ex) << 23);
#pragma unroll
        for (int k = 0; k < D / 8; ++k) {
          const float2 x = two_of(src, raw[k]);
          raw[k] = pack_f16(x.x * by, x.y * by);
        }
      }
#pragma unroll
      for (int k = 0; k < KSTEPS; ++k) {
        qf[nt][k][0] = raw[2 * k];
        qf[nt][k][1] = raw[2 * k + 1];
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {  // columns 2 cq + k of the scores
        const int col = 8 * nt + 2 * cq + k;
        const int e = __shfl_sync(0xffffffffu, ex, (2 * cq + k) * 4);
        f[nt][k] = up * __uint_as_float((uint32_t)(127 - e) << 23);
        mref[nt][k] = NO_MAX;
        l[nt][k] = 0.f;
        const int j = (row0 + col) / a.G;
        lim[nt][k] = col >= rows ? 0 : a.causal ? max(0, min(cs.L, cs.L - cs.nq + j + 1)) : cs.L;
        if (col < rows) lim_min = min(lim_min, lim[nt][k]);
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) lim_min = min(lim_min, __shfl_xor_sync(0xffffffffu, lim_min, o));
    float o[MT][NT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) o[m][nt][k] = 0.f;

    for (; tile < end; ++tile) {
      if (!mbar_wait(bar0 + 8 * stage, parity)) {
        fine = false;
        break;
      }
      const uint8_t* st = ring + stage * STAGE;
      const uint32_t no_page = (bad >> (2 * stage)) & 3u;
      const int e0 = tile * TILE;
      const bool whole = e0 + TILE <= lim_min && no_page == 0;
      // entry of MMA row i within a group: i ^ (i >> 1 & 1), so that the lanes of a V load see both halves of the banks
      const int ra = g ^ ((g >> 1) & 1);
      float sc[2][NT][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* gp = st + u * GROUP;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[u][nt][k] = 0.f;
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
              for (int nt = 0; nt < NT; ++nt)
                mma_f16(sc[u][nt], x[2 * k], y[2 * k], x[2 * k + 1], y[2 * k + 1], qf[nt][half * 8 + 2 * w + k][0], qf[nt][half * 8 + 2 * w + k][1]);
          }
        }
      }
      if (!whole) {
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
      bool raise = false;
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int k = 0; k < 4; ++k) raise |= fmaf(sc[u][nt][k], f[nt][k & 1], -mref[nt][k & 1]) > 15.0f;
      if (__any_sync(0xffffffffu, raise)) {
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
          }
      }
      uint32_t pb[2][NT][2], pl[2][NT][2];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float p[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) p[k] = ex2(fmaf(sc[u][nt][k], f[nt][k & 1], -mref[nt][k & 1]));
          l[nt][0] += p[0] + p[2];
          l[nt][1] += p[1] + p[3];
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
        uint32_t x[4][VW];
        uint32_t s[2][D == 256 ? 2 : 1];  // scales of (ta, tb) and (ta + 8, tb + 8), per block of the lane
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint8_t* p = gp + ((k & 1 ? tb : ta) + 8 * (k >> 1)) * (D / 2) + g * 4 * VW;
          if constexpr (VW == 1) x[k][0] = *reinterpret_cast<const uint32_t*>(p);
          if constexpr (VW == 2) {
            const uint2 v = *reinterpret_cast<const uint2*>(p);
            x[k][0] = v.x, x[k][1] = v.y;
          }
          if constexpr (VW == 4) {
            const uint4 v = *reinterpret_cast<const uint4*>(p);
            x[k][0] = v.x, x[k][1] = v.y, x[k][2] = v.z, x[k][3] = v.w;
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
          if (!whole) {  // what lies behind the sequence may be anything, a scale's NaN too
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
            const uint32_t p = x[2 * k][w], r = x[2 * k + 1][w];
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
            if constexpr (sizeof(OutT) == 2) {
              *reinterpret_cast<uint4*>(dst + 2 * m) =
                  make_uint4(pack_two(dst, v[0], v[1]), pack_two(dst, v[2], v[3]), pack_two(dst, v[4], v[5]), pack_two(dst, v[6], v[7]));
            } else {
              *reinterpret_cast<float4*>(dst + 2 * m) = make_float4(v[0], v[1], v[2], v[3]);
              *reinterpret_cast<float4*>(dst + 2 * m + 4) = make_float4(v[4], v[5], v[6], v[7]);
            }
          }
          if (lse && g == 0) lse[at] = l[nt][k] == 0.f ? NEG_INF : (mref[nt][k] + log2f(l[nt][k])) * LN2;
        } else {
          float* dst = a.ws.part + ((size_t)(2 * worker + (t0 <= base ? 1 : 0)) * ROWS + col) * (D + 4);
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
        do cs = seq_of<ROWS>(a, ++ci);
        while (cs.tiles == 0);
      }
    }
  }
  if (!fine) {
    // a wait gave up: report it, and give the copies in flight time to land (with a limit) before the block's memory is handed on
    if (lane == 0) atomicOr(c.status, IM_KV4_TIMEOUT);
    for (int k = 0; k < 64; ++k) __nanosleep(1000);
  }
}

// Joins the partial results of the items that several warps share, and writes the rows that see nothing.  Block = (query token,
// query head); its warps take the partial results in turn, so that all of them are asked for at once.
template <int D, int NT, typename OutT>
__global__ void __launch_bounds__(MERGE_THREADS) k_kv4_merge(const AttnArgs a, OutT* __restrict__ out, float* __restrict__ lse) {
  constexpr int ROWS = 8 * NT, CH = D / 32, WARPS = MERGE_THREADS / 32;
  __shared__ float s_acc[WARPS][D], s_m[WARPS], s_l[WARPS];
  const int t = blockIdx.x, head = blockIdx.y, h = head / a.G, j = head % a.G, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int i = kv4_find(a.cu, a.c.n_seqs, t);
  if (i < 0) return;
  const Seq s = seq_of<ROWS>(a, i);
  const float vup = kv4_pow2(kv4_exp(a.c.v_exp, h));
  const int r = (t - s.first) * a.G + j;
  float acc[CH], total = 0.f, m = NO_MAX;
#pragma unroll
  for (int k = 0; k < CH; ++k) acc[k] = 0.f;
  pdl_wait();
  if (s.tiles) {
    const Deal deal = *a.ws.deal;
    const long long base = a.ws.cum[i] + ((long long)h * s.rb + r / ROWS) * s.tiles;
    auto worker_of = [&](long long x) {
      const long long big = deal.rest * (deal.q + 1);
      if (((big | x) >> 31) == 0) {
        const unsigned q = (unsigned)deal.q;
        return x < big ? (int)((unsigned)x / (q + 1)) : (int)deal.rest + (int)((unsigned)(x - big) / q);
      }
      return (int)(x < big ? x / (deal.q + 1) : deal.rest + (x - big) / deal.q);
    };
    const int w0 = worker_of(base), w1 = worker_of(base + s.tiles - 1);
    if (w0 == w1) return;  // written where it was computed
    // worker w's result: its run began ahead of the item, but for the first one's
    const float* part = a.ws.part + (size_t)(r % ROWS) * (D + 4);
    for (int b = w0 + warp * 32; b <= w1; b += MERGE_THREADS) {
      const int mine = b + lane;
      float2 ml = make_float2(NO_MAX, 0.f);
      if (mine <= w1) ml = *reinterpret_cast<const float2*>(part + (size_t)(2 * mine + (mine == w0 ? 1 : 0)) * (ROWS * (D + 4)) + D);
      float mb = ml.x;
#pragma unroll
      for (int x = 1; x < 32; x <<= 1) mb = fmaxf(mb, __shfl_xor_sync(0xffffffffu, mb, x));
      mb = fmaxf(mb, m);
      const float corr = ex2(m - mb), e = ex2(ml.x - mb);
      m = mb;
      float le = ml.y * e;
#pragma unroll
      for (int x = 1; x < 32; x <<= 1) le += __shfl_xor_sync(0xffffffffu, le, x);
      total = fmaf(total, corr, le);
#pragma unroll
      for (int k = 0; k < CH; ++k) acc[k] *= corr;
      const int n = min(32, w1 + 1 - b);
#pragma unroll 8
      for (int x = 0; x < n; ++x) {
        const int w = b + x;
        const float by = __shfl_sync(0xffffffffu, e, x);
        const float* p = part + (size_t)(2 * w + (w == w0 ? 1 : 0)) * (ROWS * (D + 4));
        if constexpr (CH == 2) {
          const float2 v = *reinterpret_cast<const float2*>(p + 2 * lane);
          acc[0] = fmaf(v.x, by, acc[0]), acc[1] = fmaf(v.y, by, acc[1]);
        } else {
#pragma unroll
          for (int k = 0; k < CH; k += 4) {
            const float4 v = *reinterpret_cast<const float4*>(p + CH * lane + k);
            acc[k] = fmaf(v.x, by, acc[k]), acc[k + 1] = fmaf(v.y, by, acc[k + 1]);
            acc[k + 2] = fmaf(v.z, by, acc[k + 2]), acc[k + 3] = fmaf(v.w, by, acc[k + 3]);
          }
        }
      }
    }
    if (w1 - w0 >= 32) {  // (the same for the whole block)
#pragma unroll
      for (int k = 0; k < CH; ++k) s_acc[warp][CH * lane + k] = acc[k];
      if (lane == 0) s_m[warp] = m, s_l[warp] = total;
      __syncthreads();
      if (warp) return;
#pragma unroll
      for (int w = 1; w < WARPS; ++w) m = fmaxf(m, s_m[w]);
      total = 0.f;
#pragma unroll
      for (int k = 0; k < CH; ++k) acc[k] = 0.f;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        const float by = ex2(s_m[w] - m);
        total = fmaf(s_l[w], by, total);
#pragma unroll
        for (int k = 0; k < CH; ++k) acc[k] = fmaf(s_acc[w][CH * lane + k], by, acc[k]);
      }
    }
  }
  if (warp) return;
  const size_t at = (size_t)t * a.H + head;
  const float inv = total == 0.f ? 0.f : vup / total;
  OutT* dst = out + at * D + CH * lane;
#pragma unroll
  for (int k = 0; k < CH; k += 2) {
    if constexpr (sizeof(OutT) == 2) *reinterpret_cast<uint32_t*>(dst + k) = pack_two(dst, acc[k] * inv, acc[k + 1] * inv);
    else *reinterpret_cast<float2*>(dst + k) = make_float2(acc[k] * inv, acc[k + 1] * inv);
  }
  if (lse && lane == 0) lse[at] = total == 0.f ? NEG_INF : (m + log2f(total)) * LN2;
}

int sm_count() {
  static int counts[64] = {};  // (threads that look it up at the same time store the same value)
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
  if (!counts[dev]) {
    int n = 0;
    if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
    counts[dev] = n;
  }
  return counts[dev];
}
constexpr int MOST_SMS = 160;  // workspaces are sized for this many; the grid never has more CTAs

size_t workspace(const Kv4& c, int rows, int d, int nt, uint8_t* base, AttnWs* ws) {
  const size_t cum = 256, part = cum + kv4_align(8 * (size_t)c.n_seqs);
  if (ws) *ws = {(Deal*)base, (long long*)(base + cum), (float*)(base + part)};
  // no more workers than tiles
  const double tiles = (double)c.n_seqs * ((double)c.max_pages * c.ps / TILE + 1) * c.Hkv * ((rows + 8 * nt - 1) / (8 * nt));
  const size_t workers = (size_t)(tiles < MOST_SMS * warps_of(d, nt) ? tiles : MOST_SMS * warps_of(d, nt));
  return part + kv4_align(2 * workers * 8 * nt * (d + 4) * 4);
}

template <int D, int NT, bool TWO, typename T, typename OutT>
cudaError_t launch(const AttnArgs& a, const void* q, void* out, float* lse, int grid, cudaStream_t s) {
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
  if (e == cudaSuccess) e = kv4_launch(k_kv4_merge<D, NT, OutT>, dim3(a.n_tokens, a.H), MERGE_THREADS, 0, s, true, a, (OutT*)out, lse);
  return e;
}

template <int D, int NT>
cudaError_t launch_types(const AttnArgs& a, int dtype, int out_f32, const void* q, void* out, float* lse, int grid, cudaStream_t s) {
  if (dtype == IM_BF16)
    return out_f32 ? launch<D, NT, true, bf16, float>(a, q, out, lse, grid, s) : launch<D, NT, false, bf16, bf16>(a, q, out, lse, grid, s);
  return out_f32 ? launch<D, NT, true, __half, float>(a, q, out, lse, grid, s) : launch<D, NT, true, __half, __half>(a, q, out, lse, grid, s);
}

}  // namespace

size_t kv4_attention_workspace(const Kv4& c, int n_tokens, int n_q_heads) {
  // (rows: what the longest sequence could bring; both row-block sizes are covered)
  const long long rows = (long long)n_tokens * (n_q_heads / c.Hkv);
  const int r = (int)(rows < (1 << 20) ? rows : 1 << 20);
  const size_t x = workspace(c, r, c.d, 1, nullptr, nullptr), y = workspace(c, r, c.d, 2, nullptr, nullptr);
  return x > y ? x : y;
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
  if (!workspace_ || ((uintptr_t)workspace_ & 255) || workspace_bytes < kv4_attention_workspace(c, n_tokens, n_q_heads))
    return kv4_fail(IM_ERR_CAPACITY, fn, "workspace missing, misaligned or too small");
  if (!n_tokens) return IM_OK;
  const int sms = sm_count();
  if (sms < 1) return kv4_fail(IM_ERR_CUDA, fn, "no usable CUDA device");
  AttnArgs a = {c, map->table, map->lens, cu_q, q_stride, n_tokens, n_q_heads, n_q_heads / c.Hkv, causal ? 1 : 0,
                softmax_scale > 0.f ? softmax_scale : 1.0f / sqrtf((float)c.d), {}};
  const long long rows = (long long)(cu_q ? max_q : 1) * a.G;
  const int nt = rows <= 8 ? 1 : 2;
  workspace(c, 1, c.d, nt, (uint8_t*)workspace_, &a.ws);
  const int grid = sms < MOST_SMS ? sms : MOST_SMS;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  auto go = [&](auto dim) {
    constexpr int D = decltype(dim)::value;
    return nt == 1 ? launch_types<D, 1>(a, dtype, out_f32, q, out, lse, grid, s) : launch_types<D, 2>(a, dtype, out_f32, q, out, lse, grid, s);
  };
  const cudaError_t e = c.d == 64    ? go(std::integral_constant<int, 64>{})
                        : c.d == 128 ? go(std::integral_constant<int, 128>{})
                                     : go(std::integral_constant<int, 256>{});
  return e == cudaSuccess ? IM_OK : im_fail_message(IM_ERR_CUDA, cudaGetErrorString(e));
}
