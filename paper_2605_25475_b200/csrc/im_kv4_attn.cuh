// Shared by the kernels of im_kv4_attention (im_kv4_attn.cu: few query rows; im_kv4_chunk.cu: many): how a call's work is dealt to
// workers of equal share, and how their partial results are joined.
//
// The entries of all items (sequence, KV head, row block) form one line of tiles, sequence-major; a worker gets an equal run
// of it whatever the lengths are, which the device alone knows.  An item that one worker runs through is written by it; of
// the others the workers leave (sum of p v, reference maximum, sum of p) in the workspace, and the joining kernels add those up in
// order of the workers: results do not depend on timing.
#pragma once
#include <type_traits>

#include "im_kv4.cuh"

struct Deal {
  long long q, rest;  // the first `rest` workers get q + 1 tiles, the others q
  int workers;
};
// Tensor cores cut off what does not fit their float32 accumulators: 1e-8 of the sum per step, always towards zero.  Where
// outputs are float32 the accumulators are therefore emptied into the workspace (the place of the segment's partial result,
// float32 additions) every FLUSH_STEPS steps; for 16-bit outputs the loss is far below their own rounding.
constexpr int FLUSH_STEPS = 128;

struct Piece {  // of a worker whose run begins inside an item: that item
  long long base;  // its first tile in the line; -1: the run begins with an item
  int tiles, rows;
  int first_row, seq_first, h, pad;  // row block's first row, the sequence's first query token, KV head
};
struct AttnWs {
  Deal* deal;
  long long* cum;  // [n_seqs] tiles ahead of the sequence (few rows: joined by query token), or
  Piece* piece;    // [workers] (many rows: joined by worker)
  float* part;     // [2 * workers][ROWS][D + 4]
  int workers;     // what the workspace has room for: the call may hold more tiles than its max_q says
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

// many query rows (head_dim 64 or 128): workspace (ws, if not null, is set up in `base`), launch
size_t kv4_chunk_workspace(const Kv4& c, uint8_t* base, AttnWs* ws);
cudaError_t kv4_launch_chunk(const AttnArgs& a, int dtype, int out_f32, const void* q, void* out, float* lse, int grid, cudaStream_t s);

namespace {

constexpr float NEG_INF = -__builtin_huge_valf();
constexpr float NO_MAX = -1e30f;  // reference maximum of a row that has seen nothing
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int MOST_SMS = 160;     // workspaces are sized for this many; a grid never has more CTAs

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
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
// two float32 operations in one instruction, and the largest of three
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  unsigned long long d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;"
      : "=l"(d)
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)), "l"(*reinterpret_cast<unsigned long long*>(&c)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  unsigned long long d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return *reinterpret_cast<float2*>(&d);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
__device__ __forceinline__ float2 two_of(const bf16*, uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
__device__ __forceinline__ uint32_t pack_two(const bf16*, float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
__device__ __forceinline__ uint32_t pack_two(const __half*, float a, float b) { return pack_f16(a, b); }
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}
// eight values of a row to `dst`, in its type
template <typename OutT>
__device__ __forceinline__ void put8(OutT* dst, const float* v) {
  if constexpr (sizeof(OutT) == 2) {
    *reinterpret_cast<uint4*>(dst) = make_uint4(pack_two(dst, v[0], v[1]), pack_two(dst, v[2], v[3]), pack_two(dst, v[4], v[5]), pack_two(dst, v[6], v[7]));
  } else {
    reinterpret_cast<float4*>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
  }
}

// power of two that brings a row's largest bf16 value to [2^13, 2^14): the row then fits f16, values down to 2^-29 of the
// largest exactly
__device__ __forceinline__ int row_exponent(float amax) { return max(-114, min(100, 13 - ((int)(__float_as_uint(amax) >> 23) - 127))); }
__device__ __forceinline__ float exp2i(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// scores times this: base-2 exponents (kept finite and above zero, so that -inf stays -inf)
__device__ __forceinline__ float row_factor(const AttnArgs& a, int h, int e) {
  return fmaxf(1e-37f, fminf(1e37f, a.scale * LOG2E * kv4_pow2(kv4_exp(a.c.k_exp, h)) * exp2i(-e)));
}

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

struct Seq {
  int L, first, nq, tiles, rb;  // rb: row blocks
};
template <int ROWS, int TILE>
__device__ __forceinline__ Seq seq_of(const AttnArgs& a, int i) {
  Seq s;
  s.L = (int)max(0ll, min((long long)a.lens[i], (long long)a.c.max_pages * a.c.ps));
  queries_of(a, i, &s.first, &s.nq);
  s.rb = (int)(((long long)s.nq * a.G + ROWS - 1) / ROWS);
  s.tiles = s.nq ? (s.L + TILE - 1) / TILE : 0;
  return s;
}
__device__ __forceinline__ long long work_of(const AttnArgs& a, const Seq& s) { return (long long)s.tiles * s.rb * a.c.Hkv; }

// Adds the sequences up (every CTA for itself) and deals the line to at most `most` workers, and no more than the workspace holds.  s_cum [THREADS + 1]: tiles
// ahead of each thread's run of `per` sequences.  Ends with a block barrier.
template <int ROWS, int TILE, int THREADS>
__device__ __forceinline__ Deal deal_line(const AttnArgs& a, long long* s_cum, long long* s_scan, long long most, int* workers, int* per_) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, n = a.c.n_seqs;
  const int per = (n + THREADS - 1) / THREADS;
  long long mine = 0;
  for (int i = tid * per; i < min(n, tid * per + per); ++i) mine += work_of(a, seq_of<ROWS, TILE>(a, i));
  long long incl = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, incl, o);
    if (lane >= o) incl += u;
  }
  if (lane == 31) s_scan[warp] = incl;
  __syncthreads();
  long long before = 0;
  for (int w = 0; w < warp; ++w) before += s_scan[w];
  s_cum[tid] = before + incl - mine;
  if (tid == THREADS - 1) s_cum[THREADS] = before + incl;
  __syncthreads();
  const long long total = s_cum[THREADS];
  *workers = (int)min(min(most, (long long)a.ws.workers), max(1ll, total));
  *per_ = per;
  Deal d;
  d.workers = *workers;
  if ((total >> 31) == 0) {  // (a 64-bit division costs 0.1 us)
    d.q = (unsigned)total / (unsigned)*workers;
    d.rest = (unsigned)total % (unsigned)*workers;
  } else {
    d.q = total / *workers;
    d.rest = total % *workers;
  }
  if (blockIdx.x == 0) {
    if (tid == 0) *a.ws.deal = d;
    long long at = s_cum[tid];
    if (a.ws.cum)
      for (int i = tid * per; i < min(n, tid * per + per); ++i) {
        a.ws.cum[i] = at;
        at += work_of(a, seq_of<ROWS, TILE>(a, i));
      }
  }
  return d;
}
// Rows of sequences that hold nothing: zeros, and no sum.  The sequences go round the CTAs, here to one warp of this CTA's.
template <int D, typename OutT>
__device__ __forceinline__ void empty_rows(const AttnArgs& a, OutT* out, float* lse, int warp, int warps) {
  const int lane = threadIdx.x & 31;
  for (int i = blockIdx.x + warp * gridDim.x; i < a.c.n_seqs; i += gridDim.x * warps) {
    if (a.lens[i] > 0) continue;
    int first, nq;
    queries_of(a, i, &first, &nq);
    const size_t at = (size_t)first * a.H, n = (size_t)nq * a.H;
    for (size_t x = lane; x < n * (D / 8); x += 32) {
      const float zero[8] = {};
      put8(out + at * D + 8 * x, zero);
    }
    if (lse)
      for (size_t x = lane; x < n; x += 32) lse[at + x] = NEG_INF;
  }
}
// the sequence that tile t (< total) of the line lies in, and the tile's place in it
template <int ROWS, int TILE, int THREADS>
__device__ __forceinline__ int find_tile(const AttnArgs& a, const long long* s_cum, int per, long long t, long long* off) {
  int lo = 0, hi = THREADS;  // s_cum[lo] <= t < s_cum[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (s_cum[mid] <= t) lo = mid;
    else hi = mid;
  }
  int i = lo * per;
  *off = t - s_cum[lo];
  while (per > 1) {
    const long long w = work_of(a, seq_of<ROWS, TILE>(a, i));
    if (*off < w) return i;
    *off -= w;
    ++i;
  }
  return i;
}

// ---- joining the partial results of an item that workers w0 .. w1 share
constexpr int JOIN_WARPS = 8;
__device__ __forceinline__ int worker_of(const Deal& d, long long x) {  // (of tile x)
  const long long big = d.rest * (d.q + 1);
  if (((big | x) >> 31) == 0) {
    const unsigned q = (unsigned)d.q;
    return x < big ? (int)((unsigned)x / (q + 1)) : (int)d.rest + (int)((unsigned)(x - big) / q);
  }
  return (int)(x < big ? x / (d.q + 1) : d.rest + (x - big) / d.q);
}
// Row r of the item, by PER warps of the block, which take its results in turn; `at`: the row of out and lse.  The whole block calls it
// with the same w0, w1 where PER > 1.  Sums and vectors of a round are asked for together: one round trip for up to 8 PER results.
template <int D, int ROWS, int PER, typename OutT>
__device__ __forceinline__ void join_row(const AttnArgs& a, int w0, int w1, int r, bool there, int h, size_t at, OutT* out, float* lse) {
  constexpr int CH = D / 32, ROUND = CH == 8 ? 4 : 8;
  __shared__ float s_acc[JOIN_WARPS][D], s_m[JOIN_WARPS], s_l[JOIN_WARPS];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % PER;
  float acc[CH], total = 0.f, m = NO_MAX;
#pragma unroll
  for (int k = 0; k < CH; ++k) acc[k] = 0.f;
  if (there) {
    // worker w's result: its run began ahead of the item, but for the first one's
    const float* part = a.ws.part + (size_t)r * (D + 4);
    auto result = [&](int w) { return part + (size_t)(2 * w + (w == w0 ? 1 : 0)) * (ROWS * (D + 4)); };
    for (int b = w0 + sub; b <= w1; b += PER * ROUND) {
      float v[ROUND][CH];
      float2 ml[ROUND];
#pragma unroll
      for (int x = 0; x < ROUND; ++x) {
        const int w = b + x * PER;
        const float* q = result(min(w, w1));
        ml[x] = *reinterpret_cast<const float2*>(q + D);
        if (w > w1) ml[x] = make_float2(NO_MAX, 0.f);
        if constexpr (CH == 2) {
          const float2 y = *reinterpret_cast<const float2*>(q + 2 * lane);
          v[x][0] = y.x, v[x][1] = y.y;
        } else {
#pragma unroll
          for (int k = 0; k < CH; k += 4) {
            const float4 y = *reinterpret_cast<const float4*>(q + CH * lane + k);
            v[x][k] = y.x, v[x][k + 1] = y.y, v[x][k + 2] = y.z, v[x][k + 3] = y.w;
          }
        }
      }
      float top = m;
#pragma unroll
      for (int x = 0; x < ROUND; ++x) top = fmaxf(top, ml[x].x);
      const float corr = ex2(m - top);
      m = top;
      total *= corr;
#pragma unroll
      for (int k = 0; k < CH; ++k) acc[k] *= corr;
#pragma unroll
      for (int x = 0; x < ROUND; ++x) {
        if (b + x * PER > w1) continue;
        const float by = ex2(ml[x].x - top);
        total = fmaf(ml[x].y, by, total);
#pragma unroll
        for (int k = 0; k < CH; ++k) acc[k] = fmaf(v[x][k], by, acc[k]);
      }
    }
  }
  if (PER > 1) {
#pragma unroll
    for (int k = 0; k < CH; ++k) s_acc[warp][CH * lane + k] = acc[k];
    if (lane == 0) s_m[warp] = m, s_l[warp] = total;
    __syncthreads();
    if (sub == 0) {
#pragma unroll
      for (int x = 1; x < PER; ++x) m = fmaxf(m, s_m[warp + x]);
      total = 0.f;
#pragma unroll
      for (int k = 0; k < CH; ++k) acc[k] = 0.f;
#pragma unroll
      for (int x = 0; x < PER; ++x) {
        const float by = ex2(s_m[warp + x] - m);
        total = fmaf(s_l[warp + x], by, total);
#pragma unroll
        for (int k = 0; k < CH; ++k) acc[k] = fmaf(s_acc[warp + x][CH * lane + k], by, acc[k]);
      }
    }
  }
  if (!there || sub) return;
  const float inv = total == 0.f ? 0.f : kv4_pow2(kv4_exp(a.c.v_exp, h)) / total;
  OutT* dst = out + at * D + CH * lane;
#pragma unroll
  for (int k = 0; k < CH; k += 2) {
    if constexpr (sizeof(OutT) == 2) *reinterpret_cast<uint32_t*>(dst + k) = pack_two(dst, acc[k] * inv, acc[k + 1] * inv);
    else *reinterpret_cast<float2*>(dst + k) = make_float2(acc[k] * inv, acc[k + 1] * inv);
  }
  if (lse && lane == 0) lse[at] = total == 0.f ? NEG_INF : (m + log2f(total)) * LN2;
}

// Few rows: block = (sequence, KV head, rows by z), PER warps per row.  A row that sees nothing is written where it was found.
// A chain of two round trips (the deal, then up to 8 PER results at once): 3 us behind the streaming kernel.
template <int D, int ROWS, int TILE, int PER, typename OutT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) k_kv4_join_seqs(const AttnArgs a, OutT* __restrict__ out, float* __restrict__ lse) {
  const int i = blockIdx.x, h = blockIdx.y;
  const Seq s = seq_of<ROWS, TILE>(a, i);
  pdl_wait();
  const Deal deal = *a.ws.deal;
  const long long cum = a.ws.cum[i];
  if (!s.tiles) return;
  for (int r0 = blockIdx.z * (JOIN_WARPS / PER); r0 < s.nq * a.G; r0 += gridDim.z * (JOIN_WARPS / PER)) {  // (rows of a block lie in one item)
    const int r = r0 + (threadIdx.x >> 5) / PER;
    const long long base = cum + ((long long)h * s.rb + r0 / ROWS) * s.tiles;
    const int w0 = worker_of(deal, base), w1 = worker_of(deal, base + s.tiles - 1);
    if (w0 == w1) continue;  // written where it was computed
    join_row<D, ROWS, PER>(a, w0, w1, r % ROWS, r < s.nq * a.G, h, (size_t)(s.first + r / a.G) * a.H + h * a.G + r % a.G, out, lse);
    __syncthreads();  // (its shared memory is used again)
  }
}
// Many rows: block (w, y) = the item that worker w + 1's run begins inside, if w + 1 is the second worker on it (each shared item
// has one); a warp per row, JOIN_WARPS rows by y.  31 us alone, with cold caches, for 147 items of 256 rows (up to
// 40 MB of partial results): 5 % of that call.
template <int D, int ROWS, typename OutT>
__global__ void __launch_bounds__(JOIN_WARPS * 32) k_kv4_join_workers(const AttnArgs a, OutT* __restrict__ out, float* __restrict__ lse) {
  const int w = blockIdx.x + 1, r = blockIdx.y * JOIN_WARPS + (threadIdx.x >> 5);
  pdl_wait();
  const Deal deal = *a.ws.deal;
  if (w >= deal.workers || deal.q == 0) return;
  const Piece p = a.ws.piece[w];
  if (p.base < 0 || (w - 1) * deal.q + min((long long)w - 1, deal.rest) > p.base || r >= p.rows) return;
  const int row = p.first_row + r;
  join_row<D, ROWS, 1>(a, w - 1, worker_of(deal, p.base + p.tiles - 1), r, true, p.h, (size_t)(p.seq_first + row / a.G) * a.H + p.h * a.G + row % a.G, out, lse);
}

}  // namespace
