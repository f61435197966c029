// Attention over the paged 4-bit KV cache for many query rows (a prompt's chunk behind cached tokens, drafted tokens): the
// products on the 5th-generation tensor cores, for head_dim 64 and 128.  With hundreds of rows per KV head the work is the
// two products, 4 head_dim flops per (row, entry); unpacking is paid once per 256 rows.
//
// Items are (sequence, KV head, block of 256 rows): two Q tiles of 128 rows, row r = query token r / G, head r % G of the group;
// the workers that share the line of tiles (im_kv4_attn.cuh, 64 entries a tile) are the CTAs, one per SM.  Per tile:
//   warp 8       asks for the packed groups of the tile (bulk copies into a ring of RAW tiles)
//   warps 9-12   unpack them: a lane turns a word (8 channels) into 16 bytes of f16, exactly (code times scale has 6 significant
//                bits), and stores them in the layout of an MMA operand (128-byte swizzle; neighbouring lanes write neighbouring
//                16-byte chunks of a row, so that the stores of a quarter warp cover all banks)
//   warps 13, 14 S_g = Q_g K^T and O_g += P_g V (tcgen05.mma, M = 128, accumulators and P in tensor memory), a warp per Q tile g;
//                the whole warp runs the loop and one elected lane issues
//   warps 0-7    softmax: thread (g, r) owns row r of tile g and reads its 64 scores with tcgen05.ld.  P is formed relative to a
//                reference maximum that is raised only by jumps of more than 2^8, kept 2^7 times as large (f16's range), and
//                written to tensor memory in f16: one term for bf16 outputs, two otherwise, as in im_kv4_attn.cu.  q is scaled
//                by a power of two per row so that bf16 fits f16.
// Tensor memory (512 columns): S_g at 64 g, P_g at 128 + 64 g (32 columns a term; one term: two buffers), O_g at 256 + 128 g.
// With two buffers P needs no wait: S(j) is issued behind the product of tile j - 2, so who has seen S(j) may overwrite P(j - 2).
// Where outputs are float32 the accumulators are emptied every FLUSH_STEPS steps (im_kv4_attn.cuh).  Every wait is bounded
// (IM_KV4_TIMEOUT).
// 2048 queries x 16384 entries, 32 heads on 8 of 128: 554 us, 930 TF, 56 % of the measured bf16 rate.  A tile of 256 rows takes
// 2100 cycles: 1024 of exponentials (16 per clock), 1280 of products, overlapped but for the chain barrier, load, maximum,
// exponentials, store that every softmax thread runs through.  Tiles of 128 entries with P over S took 634 us.
#include <math.h>

#include "im_kv4_attn.cuh"

namespace {

constexpr int KT = 64, ROWS = 128, QT = 2, BLOCK_ROWS = QT * ROWS;
constexpr int UNPACK_WARPS = 4, UNPACK = UNPACK_WARPS * 32;
constexpr int W_COPY = 8, W_UNPACK = 9, W_MMA = W_UNPACK + UNPACK_WARPS, THREADS = (W_MMA + QT) * 32;
constexpr int STAGES = 3, RAW = 5;
constexpr int HALF_BYTES = KT * 128;  // 64 rows x 128 bytes (64 channels)
template <bool TWO, typename OutT>  // tiles between two emptyings of the accumulators
constexpr int flush_tiles() { return std::is_same<OutT, float>::value ? FLUSH_STEPS / (KT / 16 * (TWO ? 2 : 1)) : 1 << 30; }
constexpr int S_COL = 0, P_COL = 128, O_COL = 256, TMEM_COLS = 512;

template <int D>
struct Sizes {
  static constexpr int Q = ROWS * D * 2, KV = KT * D * 2, STAGE = 2 * KV, GROUP = kv4_group_bytes(D), TILE = 4 * GROUP;
  static constexpr int BYTES = QT * Q + STAGES * STAGE + RAW * TILE + 1024;
};

struct Shared {
  unsigned long long raw_full[RAW], raw_empty[RAW], full[STAGES], empty[STAGES], qfull[QT], sfull[QT], sempty[QT], pfull[QT][2], pvdone[QT], odone[QT], ofree[QT];
  long long cum[THREADS + 1], scan[THREADS / 32];
  int no_page[RAW];   // groups of a raw tile that have no page (bits)
  int hidden[STAGES]; // the same for the unpacked tile
  uint32_t tmem;
  int abort;
};

__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count)); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Bounded; the whole warp waits, and gets one answer (what follows is collective).  NAP: nanoseconds between attempts, for
// the warps that work ahead of the others: attempts take issue slots from the softmax warps (a third of all instructions
// when every warp polled without a pause).
__device__ __forceinline__ uint32_t mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(done)
      : "r"(bar), "r"(parity)
      : "memory");
  return done;
}
template <int NAP = 0>
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  if (__all_sync(0xffffffffu, mbar_try(bar, parity))) return true;
  uint32_t done = 0;
#pragma unroll 1
  for (uint32_t it = 0; it < IM_WAIT_LIMIT / 16; ++it) {
#pragma unroll 1
    for (int k = 0; k < 16 && !done; ++k) {
      if (NAP) __nanosleep(NAP);
      done = mbar_try(bar, parity);
    }
    if (done || *abort_flag) break;
  }
  return __all_sync(0xffffffffu, done);
}
// shared-memory operand descriptor, 128-byte swizzle: lbo / sbo in bytes
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr, uint32_t lbo, uint32_t sbo) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(sbo >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ void mma_ss(uint32_t d_tmem, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
// the A operand in tensor memory: row = lane, two f16 per 32-bit column along K
__device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\t"
      "elect.sync _|q, 0xffffffff;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar)
      : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float* v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(r[k]);
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr),
      "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
      "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
      : "memory");
}

__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t* y) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(y[0]), "=r"(y[1]), "=r"(y[2]), "=r"(y[3]), "=r"(y[4]), "=r"(y[5]), "=r"(y[6]), "=r"(y[7]), "=r"(y[8]), "=r"(y[9]),
        "=r"(y[10]), "=r"(y[11]), "=r"(y[12]), "=r"(y[13]), "=r"(y[14]), "=r"(y[15])
      : "r"(taddr)
      : "memory");
}
// One segment of a worker's run: tiles [tile, end) of an item.  Every role walks the run by itself.
struct Walk {
  Seq s;
  int i, h, rb, tile, todo;
};
struct Segment {
  int h, row0, rows, tile, end, L, first, nq;
  long long base;  // first tile of the item in the line
  bool complete;
};
__device__ __forceinline__ bool next_segment(const AttnArgs& a, Walk& w, long long t0, long long t1, Segment* g) {
  if (w.todo <= 0) return false;
  g->h = w.h;
  g->row0 = w.rb * BLOCK_ROWS;
  g->rows = min(BLOCK_ROWS, w.s.nq * a.G - g->row0);
  g->tile = w.tile;
  g->end = min(w.s.tiles, w.tile + w.todo);
  g->L = w.s.L;
  g->first = w.s.first;
  g->nq = w.s.nq;
  g->base = t1 - w.todo - w.tile;
  g->complete = g->base >= t0 && g->end == w.s.tiles;
  w.todo -= g->end - w.tile;
  w.tile = 0;
  if (w.todo > 0 && ++w.rb == w.s.rb) {
    w.rb = 0;
    if (++w.h == a.c.Hkv) {
      w.h = 0;
      do w.s = seq_of<BLOCK_ROWS, KT>(a, ++w.i);
      while (w.s.tiles == 0);
    }
  }
  return true;
}

template <int D, bool TWO, typename T, typename OutT>
__global__ void __launch_bounds__(THREADS, 1) k_kv4_chunk(const AttnArgs a, const T* __restrict__ q, OutT* __restrict__ out, float* __restrict__ lse) {
  using Z = Sizes<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ Shared sh;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint8_t* s_q = smem;                                // [QT][D / 64 halves][128 rows][128 bytes]
  uint8_t* s_kv = smem + QT * Z::Q;                   // [STAGES][K | V][D / 64 halves][64 rows][128 bytes]
  uint8_t* s_packed = s_kv + STAGES * Z::STAGE;       // [RAW][4 groups]
  const Kv4& c = a.c;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int* abort_flag = &sh.abort;
  pdl_release();
  if (tid == 0) {
    for (int s = 0; s < RAW; ++s) {
      mbar_init(smem_u32(&sh.raw_full[s]), 1);
      mbar_init(smem_u32(&sh.raw_empty[s]), UNPACK_WARPS);
    }
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&sh.full[s]), UNPACK);
      mbar_init(smem_u32(&sh.empty[s]), QT);
    }
    for (int g = 0; g < QT; ++g) {
      mbar_init(smem_u32(&sh.qfull[g]), ROWS);
      mbar_init(smem_u32(&sh.sfull[g]), 1);
      mbar_init(smem_u32(&sh.sempty[g]), ROWS);
      mbar_init(smem_u32(&sh.pfull[g][0]), ROWS);
      mbar_init(smem_u32(&sh.pfull[g][1]), ROWS);
      mbar_init(smem_u32(&sh.pvdone[g]), 1);
      mbar_init(smem_u32(&sh.odone[g]), 1);
      mbar_init(smem_u32(&sh.ofree[g]), ROWS);
    }
    sh.abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"((uint32_t)TMEM_COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  }
  int workers, per;
  const Deal deal = deal_line<BLOCK_ROWS, KT, THREADS>(a, sh.cum, sh.scan, gridDim.x, &workers, &per);  // (a block barrier inside)
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh.tmem;
  const int worker = blockIdx.x;
  const long long t0 = worker * deal.q + min((long long)worker, deal.rest), t1 = t0 + deal.q + (worker < deal.rest ? 1 : 0);
  bool ok = true;
  if (worker < workers && t0 < t1) {
    Walk w;
    long long off;
    w.i = find_tile<BLOCK_ROWS, KT, THREADS>(a, sh.cum, per, t0, &off);
    w.s = seq_of<BLOCK_ROWS, KT>(a, w.i);
    w.tile = (int)(off % w.s.tiles);
    const int item = (int)(off / w.s.tiles);
    w.h = item / w.s.rb;
    w.rb = item % w.s.rb;
    w.todo = (int)(t1 - t0);
    Segment g;
    if (tid == 0) {  // what the run begins with
      Walk v = w;
      next_segment(a, v, t0, t1, &g);
      a.ws.piece[worker] = {g.base < t0 ? g.base : -1, w.s.tiles, g.rows, g.row0, g.first, g.h, 0};
    }

    if (warp == W_COPY) {
      // ---- packed tiles: 64 entries are 4, 2 or 1 pieces of pages
      const size_t head_bytes = (size_t)(c.ps >> 4) * Z::GROUP, page_bytes = head_bytes * c.Hkv;
      const int piece = min(c.ps, KT), pieces = KT / piece;  // entries per piece; a window of 32 lanes holds 32 / pieces tiles
      int n = 0;
      while (ok) {
        const int i = w.i;
        if (!next_segment(a, w, t0, t1, &g)) break;
        const uint8_t* src = c.pool + g.h * head_bytes;
        int win = 0, win_base = 0, win_end = 0;
        for (int t = g.tile; t < g.end; ++t, ++n) {
          if (t >= win_end) {
            const long long e = ((long long)t * pieces + lane) * piece;
            win = e < g.L ? a.table[(size_t)i * c.max_pages + e / c.ps] : -1;
            win_base = t;
            win_end = t + 32 / pieces;
          }
          const int r = n % RAW;
          if (n >= RAW && !mbar_wait<200>(smem_u32(&sh.raw_empty[r]), (uint32_t)((n / RAW - 1) & 1), abort_flag)) { ok = false; break; }
          const int page = __shfl_sync(0xffffffffu, win, min(31, (t - win_base) * pieces + min(lane, pieces - 1)));
          const bool has = lane < pieces && (unsigned)page < (unsigned)c.n_pages;
          const int at = t * KT + lane * piece;
          if (lane < pieces && !has && at < g.L) atomicOr(c.status, IM_KV4_BAD_MAP);
          const unsigned mask = __ballot_sync(0xffffffffu, has);
          const uint32_t bytes = (uint32_t)(piece >> 4) * Z::GROUP;
          const uint32_t bar = smem_u32(&sh.raw_full[r]);
          if (lane == 0) {
            int none = 0;
            for (int p = 0; p < pieces; ++p)
              if (!((mask >> p) & 1)) none |= ((1 << (piece >> 4)) - 1) << (p * (piece >> 4));
            sh.no_page[r] = none;
            asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes * __popc(mask)) : "memory");
          }
          __syncwarp();
          if (has)
            bulk_load(smem_u32(s_packed + r * Z::TILE) + lane * bytes, src + page * page_bytes + ((at & (c.ps - 1)) >> 4) * Z::GROUP, bytes, bar);
        }
      }
    } else if (warp >= W_UNPACK && warp < W_MMA) {
      // ---- packed tile -> f16 operand tiles
      constexpr int WORDS = D / 8, STEP = UNPACK / WORDS;  // words of a row; rows apart
      const int ut = tid - W_UNPACK * 32, word = ut % WORDS, r0 = ut / WORDS;
      int n = 0;
      while (ok && next_segment(a, w, t0, t1, &g)) {
        for (int t = g.tile; t < g.end; ++t, ++n) {
          const int r = n % RAW, s = n % STAGES;
          if (!mbar_wait(smem_u32(&sh.raw_full[r]), (uint32_t)((n / RAW) & 1), abort_flag)) { ok = false; break; }
          if (n >= STAGES && !mbar_wait<40>(smem_u32(&sh.empty[s]), (uint32_t)((n / STAGES - 1) & 1), abort_flag)) { ok = false; break; }
          const uint8_t* codes = s_packed + r * Z::TILE + r0 * (D / 2) + 4 * word;
          const uint8_t* scales = s_packed + r * Z::TILE + 8 * D + r0 * (D / 16) + (word >> 1);
          uint8_t* dst = s_kv + s * Z::STAGE + (word >> 3) * HALF_BYTES + r0 * 128 + (((word & 7) ^ (r0 & 7)) << 4);
          const int none = *(volatile int*)&sh.no_page[r], seen = g.L - t * KT;  // rows from `seen` on hold anything
          const bool whole = __all_sync(0xffffffffu, seen >= KT && none == 0);
          if (ut == 0) sh.hidden[s] = none;
          // (every offset below is a constant but for those of the lane)
          // The loads of a batch stand ahead of its stores, which the compiler could not know to be elsewhere.
          auto unpack = [&](auto all) {
            constexpr int ROUNDS = KT / STEP, BATCH = 8;  // words of a thread: 2 ROUNDS, keys then values
#pragma unroll
            for (int y0 = 0; y0 < 2 * ROUNDS; y0 += BATCH) {
              uint32_t code[BATCH], by[BATCH];
#pragma unroll
              for (int y = 0; y < BATCH; ++y) {
                const int v = (y0 + y) / ROUNDS, p = (y0 + y) % ROUNDS;
                const int group = p * STEP / 16, up = p * STEP % 16;  // row r0 + p STEP = row r0 + up of the group
                code[y] = *reinterpret_cast<const uint32_t*>(codes + group * Z::GROUP + v * 9 * D + up * (D / 2));
                by[y] = scales[group * Z::GROUP + v * 9 * D + up * (D / 16)];
                if (!decltype(all)::value && (r0 + p * STEP >= seen || ((none >> group) & 1))) by[y] = 0;
              }
#pragma unroll
              for (int y = 0; y < BATCH; ++y) {
                by[y] = kv4_f16x2_e4m3(by[y]);
                by[y] = __byte_perm(by[y], by[y], 0x1010);
              }
#pragma unroll
              for (int y = 0; y < BATCH; ++y) {
                const int v = (y0 + y) / ROUNDS, p = (y0 + y) % ROUNDS;
                uint32_t x[4];
                kv4_f16_e2m1(code[y], x);
                *reinterpret_cast<uint4*>(dst + v * Z::KV + p * STEP * 128) = make_uint4(mul2(x[0], by[y]), mul2(x[1], by[y]), mul2(x[2], by[y]), mul2(x[3], by[y]));
              }
            }
          };
          if (whole) unpack(std::true_type{});
          else unpack(std::false_type{});
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(smem_u32(&sh.full[s]));
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&sh.raw_empty[r]));
        }
      }
    } else if (warp >= W_MMA) {
      // ---- products: a warp per Q tile, so that neither waits for the other's softmax.  The scores of the next tile are issued
      // as soon as the softmax threads have read the last, ahead of the product that waits for their P.
      const int x = warp - W_MMA;
      const uint32_t idesc_s = (1u << 4) | ((uint32_t)(KT >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
      const uint32_t idesc_o = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(ROWS >> 4) << 24);
      const uint32_t qa = smem_u32(s_q) + x * Z::Q, kv = smem_u32(s_kv);
      int n = 0, cnt = 0, segs = 0;  // tiles so far; tiles and segments of this Q tile
      auto scores = [&](int m, int k, bool first) -> bool {  // tile m of the run, k of this Q tile
        if (!mbar_wait(smem_u32(&sh.full[m % STAGES]), (uint32_t)((m / STAGES) & 1), abort_flag)) return false;
        if (first && !mbar_wait(smem_u32(&sh.qfull[x]), (uint32_t)(segs & 1), abort_flag)) return false;
        if (k >= 1 && !mbar_wait(smem_u32(&sh.sempty[x]), (uint32_t)((k - 1) & 1), abort_flag)) return false;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const uint32_t ka = kv + (m % STAGES) * Z::STAGE;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
          mma_ss(tmem + (uint32_t)(S_COL + x * KT), desc_sw128(qa + (ks >> 2) * (ROWS * 128) + (ks & 3) * 32, 16, 1024),
                 desc_sw128(ka + (ks >> 2) * HALF_BYTES + (ks & 3) * 32, 16, 1024), idesc_s, ks ? 1u : 0u);
        mma_commit(smem_u32(&sh.sfull[x]));
        return true;
      };
      while (ok && next_segment(a, w, t0, t1, &g)) {
        const int nt = g.end - g.tile;
        if (x * ROWS >= g.rows) {  // no rows: hand the stages on as they come
          for (int j = 0; j < nt && ok; ++j, ++n) {
            ok = mbar_wait(smem_u32(&sh.full[n % STAGES]), (uint32_t)((n / STAGES) & 1), abort_flag);
            if (ok && lane == 0) mbar_arrive(smem_u32(&sh.empty[n % STAGES]));
          }
          continue;
        }
        ok = scores(n, cnt, true);
        for (int j = 0; j < nt && ok; ++j, ++n, ++cnt) {
          if (j + 1 < nt && !scores(n + 1, cnt + 1, false)) { ok = false; break; }
          if (!mbar_wait(smem_u32(&sh.pfull[x][cnt & 1]), (uint32_t)((cnt >> 1) & 1), abort_flag)) { ok = false; break; }
          if (j == 0 && segs > 0 && !mbar_wait(smem_u32(&sh.ofree[x]), (uint32_t)((segs - 1) & 1), abort_flag)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t va = kv + (n % STAGES) * Z::STAGE + Z::KV;
#pragma unroll
          for (int term = 0; term < (TWO ? 2 : 1); ++term)
#pragma unroll
            for (int ks = 0; ks < KT / 16; ++ks)
              mma_ts(tmem + (uint32_t)(O_COL + x * 128), tmem + (uint32_t)(P_COL + 64 * x + 32 * (TWO ? term : cnt & 1) + 8 * ks),
                     desc_sw128(va + ks * 2048, HALF_BYTES, 1024), idesc_o, (j % flush_tiles<TWO, OutT>() | term | ks) ? 1u : 0u);
          mma_commit(smem_u32(&sh.pvdone[x]));
          if (j + 1 == nt) mma_commit(smem_u32(&sh.odone[x]));
          mma_commit(smem_u32(&sh.empty[n % STAGES]));
        }
        ++segs;
      }
      // (the last arrivals land before the block's memory is handed on)
      if (ok) ok = mbar_wait(smem_u32(&sh.empty[(n - 1) % STAGES]), (uint32_t)(((n - 1) / STAGES) & 1), abort_flag);
    } else if (warp < 8) {
      // ---- softmax: warps 4 x .. 4 x + 3 own Q tile x, thread = row = lane of tensor memory
      const int x = warp >> 2, r = tid & (ROWS - 1);
      const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
      const uint32_t t_s = tmem + lane_addr + (uint32_t)(S_COL + x * KT);
      const uint32_t t_p = tmem + lane_addr + (uint32_t)(P_COL + 64 * x);
      const uint32_t t_o = tmem + lane_addr + (uint32_t)(O_COL + 128 * x);
      int n0 = 0, cnt = 0, segs = 0;
      while (ok && next_segment(a, w, t0, t1, &g)) {
        const int nt = g.end - g.tile;
        if (x * ROWS >= g.rows) {  // nothing for this Q tile
          n0 += nt;
          continue;
        }
        const bool there = x * ROWS + r < g.rows;
        const int row = g.row0 + x * ROWS + r, token = there ? row / a.G : 0, head = g.h * a.G + (there ? row % a.G : 0);
        const int lim = !there ? 0 : a.causal ? max(0, min(g.L, g.L - g.nq + token + 1)) : g.L;
        int ex = 0;
        {  // the row of Q (the products that read the last one are complete: their scores have been waited for)
          const uint4* src = reinterpret_cast<const uint4*>(q + (size_t)(g.first + token) * a.q_stride + (size_t)head * D);
          uint4 v[D / 8];
#pragma unroll
          for (int k = 0; k < D / 8; ++k) v[k] = there ? src[k] : make_uint4(0u, 0u, 0u, 0u);
          if constexpr (std::is_same<T, bf16>::value) {
            float amax = 0.f;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
              const uint32_t u[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const float2 y = two_of((const bf16*)nullptr, u[b]);
                amax = max3(amax, fabsf(y.x), fabsf(y.y));
              }
            }
            ex = row_exponent(amax);
            const float by = exp2i(ex);
#pragma unroll
            for (int k = 0; k < D / 8; ++k) {
              uint32_t u[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
              for (int b = 0; b < 4; ++b) {
                const float2 y = two_of((const bf16*)nullptr, u[b]);
                u[b] = pack_f16(y.x * by, y.y * by);
              }
              v[k] = make_uint4(u[0], u[1], u[2], u[3]);
            }
          }
#pragma unroll
          for (int k = 0; k < D / 8; ++k)
            *reinterpret_cast<uint4*>(s_q + x * Z::Q + (k >> 3) * (ROWS * 128) + (r >> 3) * 1024 + (r & 7) * 128 + (((k & 7) ^ (r & 7)) << 4)) = v[k];
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(smem_u32(&sh.qfull[x]));
        }
        const float f = row_factor(a, g.h, ex);
        const int lim_min = __reduce_min_sync(0xffffffffu, there ? lim : g.L);
        constexpr int FLUSH = flush_tiles<TWO, OutT>();
        float* pp = a.ws.part + ((size_t)(2 * worker + (t0 <= g.base ? 1 : 0)) * BLOCK_ROWS + x * ROWS + r) * (D + 4);
        float mref = NO_MAX, fref = NO_MAX;  // fref: of what has been flushed to pp
        float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};  // the sum of p, in four parts
        for (int j = 0; j < nt; ++j) {
          const int k = cnt + j;
          if (!mbar_wait(smem_u32(&sh.sfull[x]), (uint32_t)(k & 1), abort_flag)) { ok = false; break; }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const int none = *(volatile int*)&sh.hidden[(n0 + j) % STAGES];
          float sv[KT];
          tmem_ld32(t_s, sv);
          tmem_ld32(t_s + 32, sv + 32);
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          mbar_arrive(smem_u32(&sh.sempty[x]));
          const int e0 = (g.tile + j) * KT;
          if (e0 + KT > lim_min || none) {  // (the same for the whole warp; the tiles that need it are few)
#pragma unroll
            for (int b = 0; b < KT; ++b)
              if (e0 + b >= lim || ((none >> (b >> 4)) & 1)) sv[b] = NEG_INF;
          }
          float m0 = sv[0], m1 = sv[1], m2 = sv[2], m3 = sv[3];
#pragma unroll
          for (int b = 4; b < KT - 4; b += 8) {
            m0 = max3(m0, sv[b], sv[b + 1]);
            m1 = max3(m1, sv[b + 2], sv[b + 3]);
            m2 = max3(m2, sv[b + 4], sv[b + 5]);
            m3 = max3(m3, sv[b + 6], sv[b + 7]);
          }
          m0 = max3(m0, sv[KT - 4], sv[KT - 3]);
          m1 = max3(m1, sv[KT - 2], sv[KT - 1]);
          const float top = max3(m0, m1, fmaxf(m2, m3)) * f;
          const bool raise = top - mref > 15.0f;
          bool pv_waited = false;
          if (FLUSH < (1 << 30) && j > 0 && j % FLUSH == 0) {  // empty the accumulators, which the product of this tile then overwrites
            if (!mbar_wait(smem_u32(&sh.pvdone[x]), (uint32_t)((k - 1) & 1), abort_flag)) { ok = false; break; }
            pv_waited = true;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const float by = j > FLUSH ? ex2(fref - mref) : 0.f;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 16) {
              uint32_t y[16];
              tmem_ld16(t_o + (uint32_t)c0, y);
              if (there) {
#pragma unroll
                for (int b = 0; b < 16; b += 4) {
                  float4 p = make_float4(__uint_as_float(y[b]), __uint_as_float(y[b + 1]), __uint_as_float(y[b + 2]), __uint_as_float(y[b + 3]));
                  if (j > FLUSH) {
                    const float4 q = *reinterpret_cast<const float4*>(pp + c0 + b);
                    p = make_float4(fmaf(q.x, by, p.x), fmaf(q.y, by, p.y), fmaf(q.z, by, p.z), fmaf(q.w, by, p.w));
                  }
                  *reinterpret_cast<float4*>(pp + c0 + b) = p;
                }
              }
            }
            fref = mref;
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          }
          if (__any_sync(0xffffffffu, raise)) {
            const float next = raise ? top - 7.0f : mref;
            const float corr = ex2(mref - next);
            mref = next;
#pragma unroll
            for (int b = 0; b < 2; ++b) l2[b].x *= corr, l2[b].y *= corr;
            if (j % FLUSH) {  // O holds the products up to tile j - 1 (that of j - 2 is complete): wait for the last one, then scale the row
              if (!mbar_wait(smem_u32(&sh.pvdone[x]), (uint32_t)((k - 1) & 1), abort_flag)) { ok = false; break; }
              pv_waited = true;
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll
              for (int c0 = 0; c0 < D; c0 += 16) {
                uint32_t y[16];
                tmem_ld16(t_o + (uint32_t)c0, y);
#pragma unroll
                for (int b = 0; b < 16; ++b) y[b] = __float_as_uint(__uint_as_float(y[b]) * corr);
                tmem_st16(t_o + (uint32_t)c0, y);
              }
              asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
              asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            }
          }
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            uint32_t hi[16], lo[16];
#pragma unroll
            for (int b = 0; b < 16; ++b) {
              const float2 e = fma2(make_float2(sv[32 * hf + 2 * b], sv[32 * hf + 2 * b + 1]), make_float2(f, f), make_float2(-mref, -mref));
              const float2 p = make_float2(ex2(e.x), ex2(e.y));
              l2[b & 1] = add2(l2[b & 1], p);
              hi[b] = pack_f16(p.x, p.y);
              if constexpr (TWO) {
                const float2 back = kv4_unpack_f16(hi[b]);
                lo[b] = pack_f16(p.x - back.x, p.y - back.y);
              }
            }
            if (TWO && hf == 0 && j >= 1 && !pv_waited) {  // one buffer: the product of tile j - 1 has to be through with it
              if (!mbar_wait(smem_u32(&sh.pvdone[x]), (uint32_t)((k - 1) & 1), abort_flag)) { ok = false; break; }
              asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            }
            tmem_st16(t_p + (uint32_t)(16 * hf + (TWO ? 0 : 32 * (k & 1))), hi);
            if constexpr (TWO) tmem_st16(t_p + (uint32_t)(32 + 16 * hf), lo);
          }
          if (!ok) break;
          asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
          mbar_arrive(smem_u32(&sh.pfull[x][k & 1]));  // (a barrier per parity: a warp may be a tile ahead of the others)
        }
        if (!ok) break;
        cnt += nt;
        n0 += nt;
        // (a barrier of its own: with two buffers up to two products are outstanding here, and pvdone's parity cannot tell them apart)
        if (!mbar_wait(smem_u32(&sh.odone[x]), (uint32_t)(segs & 1), abort_flag)) { ok = false; break; }
        ++segs;
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        // ---- the segment's result
        const float l = (l2[0].x + l2[1].x) + (l2[0].y + l2[1].y);
        const size_t at = (size_t)(g.first + token) * a.H + head;
        const float inv = l == 0.f ? 0.f : kv4_pow2(kv4_exp(c.v_exp, g.h)) / l;
        OutT* op = out + at * D;
        const bool flushed = FLUSH < (1 << 30) && nt > FLUSH;
        const float fby = flushed ? ex2(fref - mref) : 0.f;
#pragma unroll
        for (int c0 = 0; c0 < D; c0 += 32) {
          float v[32];
          tmem_ld32(t_o + (uint32_t)c0, v);  // (warp-collective: rows that are not there load too, and store nothing)
          if (flushed && there) {
#pragma unroll
            for (int b = 0; b < 32; ++b) v[b] = fmaf(pp[c0 + b], fby, v[b]);
          }
          if (there && g.complete) {
#pragma unroll
            for (int b = 0; b < 32; ++b) v[b] *= inv;
#pragma unroll
            for (int b = 0; b < 32; b += 8) put8(op + c0 + b, v + b);
          } else if (there) {
#pragma unroll
            for (int b = 0; b < 32; b += 8) put8(pp + c0 + b, v + b);
          }
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        mbar_arrive(smem_u32(&sh.ofree[x]));
        if (there && g.complete) {
          if (lse) lse[at] = l == 0.f ? NEG_INF : (mref + log2f(l)) * LN2;
        } else if (there) {
          *reinterpret_cast<float2*>(pp + D) = make_float2(mref, l);
        }
      }
    }
    if (!ok && lane == 0) {
      sh.abort = 1;
      atomicOr(c.status, IM_KV4_TIMEOUT);
      // copies that this CTA still has in flight write into its shared memory: give them time to land (bounded)
      for (int k = 0; k < 64; ++k) __nanosleep(1000);
    }
  }
  empty_rows<D>(a, out, lse, warp, THREADS / 32);
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == W_MMA) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"((uint32_t)TMEM_COLS) : "memory");
  }
}

template <int D, bool TWO, typename T, typename OutT>
cudaError_t launch(const AttnArgs& a, const void* q, void* out, float* lse, int grid, cudaStream_t s) {
  static bool flags[64] = {};
  bool* done = im_device_flag(flags);
  if (!done) return cudaErrorInvalidDevice;
  if (!*done) {
    const cudaError_t e = cudaFuncSetAttribute(k_kv4_chunk<D, TWO, T, OutT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sizes<D>::BYTES);
    if (e != cudaSuccess) return e;
    *done = true;
  }
  cudaError_t e = kv4_launch(k_kv4_chunk<D, TWO, T, OutT>, dim3(grid), THREADS, Sizes<D>::BYTES, s, false, a, (const T*)q, (OutT*)out, lse);
  if (e == cudaSuccess && grid > 1)
    e = kv4_launch(k_kv4_join_workers<D, BLOCK_ROWS, OutT>, dim3(grid - 1, BLOCK_ROWS / JOIN_WARPS), JOIN_WARPS * 32, 0, s, true, a, (OutT*)out, lse);
  return e;
}
template <int D>
cudaError_t launch_types(const AttnArgs& a, int dtype, int out_f32, const void* q, void* out, float* lse, int grid, cudaStream_t s) {
  if (dtype == IM_BF16) return out_f32 ? launch<D, true, bf16, float>(a, q, out, lse, grid, s) : launch<D, false, bf16, bf16>(a, q, out, lse, grid, s);
  return out_f32 ? launch<D, true, __half, float>(a, q, out, lse, grid, s) : launch<D, true, __half, __half>(a, q, out, lse, grid, s);
}

}  // namespace

size_t kv4_chunk_workspace(const Kv4& c, uint8_t* base, AttnWs* ws) {
  const size_t piece = 256, part = piece + kv4_align(sizeof(Piece) * MOST_SMS);
  if (ws) *ws = {(Deal*)base, nullptr, (Piece*)(base + piece), (float*)(base + part), MOST_SMS};
  return part + kv4_align(2 * (size_t)MOST_SMS * BLOCK_ROWS * (c.d + 4) * 4);
}
cudaError_t kv4_launch_chunk(const AttnArgs& a, int dtype, int out_f32, const void* q, void* out, float* lse, int grid, cudaStream_t s) {
  return a.c.d == 64 ? launch_types<64>(a, dtype, out_f32, q, out, lse, grid, s) : launch_types<128>(a, dtype, out_f32, q, out, lse, grid, s);
}
