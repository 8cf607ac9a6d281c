// Attention of one new token per sequence over a paged cache (a3_paged_attention), split over the keys and joined.
//
//   o[s][h] = sum_t softmax_t(scale q[s][h] . k[s][t][h/G]) v[s][t][h/G],   t < len[s]
//
// Every key and value is read once and used by the G query heads of its KV head: bound by HBM.  The lengths are known on the
// device only, so the kernel divides the work itself: the keys of all sequences, cut into tiles of KT keys, form one line
// per KV head; a CTA takes an equal stretch of it (where it is long, one more short stretch for who is done early) and each of
// its warps an equal part of that, whatever sequences lie there.  Few and short sequences have CTAs of their own instead.  A warp
// streams its tiles through a ring of its own with 16-byte asynchronous copies (two tiles under way while
// the third is computed, no barrier between warps) and keeps the running maximum and sum of the softmax, fp32, in registers.
// Products: S^T = K Q^T and O^T = V^T P^T with warp-level MMAs, keys (head dimensions) on the 16-row side and the heads that share
// them on the 8-column side: the query heads of a group fill the narrow side of the instruction, and what they need of the
// tensor pipe is a few percent, so nothing is gained by the wide one.  Where a sequence lies in one warp's part the result is
// written at once; a CTA merges what its warps hold of a sequence; what several CTAs hold goes to the workspace as (maximum, sum,
// unnormalised output) and a second kernel merges it in the order of the keys.  The division depends on the lengths and
// the device only: results do not depend on timing.
//
// Measured, 32 query heads over 8 of 128, bf16: 128 sequences of up to 8 191 slots, 2.0 GB, in 298-312 us, 6.4-6.7 TB/s, as fast as a copy; one of 5 153 slots,
// 21 MB, in 10.2 us by eight CTAs for each KV head, nearly all of them lengths, pages and keys one after the other and the two merges; where a
// second launch joins, that is 2 us more; one of 32 801 in 8 bits, 67 MB, in 21.3-21.9 us.  28 heads over 4, 8 bits, 16 sequences of up to 15 675 slots, 157 MB, in 34.3-36.3 us: the
// widening and the products of 8-bit tiles take as long as their way from HBM, and the SM with the slowest way to it 32.6 us where the median takes 25.
//
// P is kept to 16 bits for bf16 values (two bf16 terms): with one, its rounding is as large as that of the output itself.  8-bit keys
// and values are widened to fp16, which holds them exactly; the query is scaled by a power of two per head so that fp16 holds all of
// its bits down to 2^-29 of its largest element.  P as one fp16 term is off by 2^-11 of itself, an eighth of the output's rounding, or by 2^-32 of
// the reference's weight where it is far below it; a second term would be half as many products again.
#include <cuda_fp16.h>

#include <type_traits>

#include "a3_internal.cuh"
#include "a3_paged.cuh"

namespace a3 {

constexpr int PD_WARPS = 8;      // of a CTA, one per SM
constexpr int PD_STAGE = 8192;   // bytes of a tile: keys in the lower half, values in the upper
constexpr float LN2 = 0.693147180559945309f;
// A sequence (of a unit of heads) has CTAs to itself, without a second launch, where that leaves a warp PD_ALONE tiles at most if the page table's row is full:
// the host does not know the lengths.  So one sequence of 600 slots takes 6.2 us behind a table of 38 pages of 16 and 8.9 behind one of 8 192, of 5 153 9.9 and
// 11.6, 16 of 760 9.6 and 14.5 (keys in L2).  As many CTAs, up to PD_CTAS in a cluster, as run at once, but no more once a warp has PD_FEW.  On the device, 32 query heads over 8, with CTAs of its own and on
// the line: one sequence of 600 slots 6.3 us and 9.1, 2 500 7.6 and 9.7, 5 100 9.5 and 10.3; 8 of 1 200 10.5 and 12.7; 4 of 2 500 11.5 and 13.6;
// 16 of 760, a CTA and 6 tiles a warp each, 11.5 and 16.2; in 8 bits, whose tiles are twice the slots and the work, one of 1 200 6.9 and 10.5,
// of 5 100 10.8 and 11.6, and of 9 000 with more than PD_ALONE_E4M3 tiles a warp 12.8 and 12.1.  With no more CTAs than PD_ALONE asks for: 600
// slots 7.4, 2 500 8.9, 1 200 in 8 bits 9.4.
constexpr int PD_CTAS = 8;
constexpr int PD_ALONE = 6, PD_ALONE_E4M3 = 3;
constexpr int PD_FEW = 2, PD_FEW_E4M3 = 1;
// From so many tiles for each warp on, one tile in PD_LATE goes to late parts: 128 sequences of up to 8 191 slots (213 tiles a warp) 321 -> 300 us,
// 32 of them (57) 93.3 -> 89.7, 32 of 28 heads over 4 (40) 70.3 -> 71.8.  One in 20: 307 and 91.1.
constexpr int PD_MANY = 48, PD_LATE = 10;
constexpr int PD_LEAST = 2;  // tiles of a warp, before another part is begun
constexpr float PD_SLACK = 8.f;  // see the running softmax
// Weights beside 8-bit values are 2^PD_LIFT times as large as their logits say, up to 2^15: fp16 keeps 11 bits of a weight down to 2^-21 of the reference's, and
// half a step of what is below is 2^-32 of it.
constexpr float PD_LIFT = 7.f;

struct PagedAttnArgs {
  const char *k_pages, *v_pages;
  long long page_stride;
  int n_pages, page_size;
  const float *k_scale, *v_scale;
  const int32_t *table, *lens;
  int n_seqs, max_pages;
  const bf16* q;
  long long q_stride;
  float scale_log2;  // scale * log2(e)
  bf16* out;
  float* lse;
  int q_heads, kv_heads, group, groups;  // groups: CTAs' head units per KV head, of `unit` query heads at most
  int unit, parts;        // parts: that run at once
  int most_parts;         // with late ones, where the page table is wide enough for so many tiles
  int by_seq;             // CTAs that have one sequence (of a unit) to themselves, a cluster where more than one; 0: parts of the line
  // workspace
  int4* meta;             // [parts]: what the join of part p does, see there
  float* part_o;          // [parts][units][2][unit][D]
  float2* part_ml;        // [parts][units][2][unit]
  float* first_o;         // [parts][units][warps][unit][D]: see below
  uint32_t* status;
};
// A line cut into `n` parts, the first ones a tile longer where it does not divide.
struct Parts {
  unsigned size, more;  // tiles of a part; parts that have one more
  __device__ Parts(unsigned total, unsigned n) : size(total / n), more(total - size * n) {}
  __device__ unsigned begin(unsigned p) const { return p * size + min(p, more); }
  __device__ unsigned of(unsigned tile) const {
    const unsigned longer = more * (size + 1);
    return tile < longer ? tile / (size + 1) : more + (tile - longer) / size;
  }
};
// The line of all tiles: its parts at first, which run at once, and behind them late parts, which the SMs take up as they finish.  SMs that share
// a way to memory with more others are slower by a third: with equal parts alone the others wait for them.
struct Line {
  unsigned firsts, early, active;  // first parts, the tiles that they have together, parts in all
  Parts first, late;
  __device__ Line(unsigned total, unsigned parts, unsigned warps)
      : firsts(min((total + PD_LEAST * warps - 1) / (PD_LEAST * warps), parts)),
        early(total >= parts * warps * PD_MANY ? total - total / PD_LATE : total),
        active(early < total ? 2 * parts : firsts),
        first(early, firsts > 0 ? firsts : 1),
        late(total - early, parts) {}
  __device__ unsigned begin(unsigned p) const { return p < firsts ? first.begin(p) : early + late.begin(p - firsts); }
  __device__ int of(unsigned tile) const { return tile < early ? first.of(tile) : firsts + late.of(tile - early); }
};

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
// D(16x8, fp32) += A(16x16, row) * B(16x8, col), fp16 or bf16; not volatile: the compiler may place it among the loads
template <bool H>
__device__ __forceinline__ void mma_any(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if constexpr (H)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"((unsigned short)two));
  return y;
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;\n" ::"r"(dst), "l"(src));
}
__device__ __forceinline__ void prefetch_l2(const void* p) { asm volatile("prefetch.global.L2 [%0];" ::"l"(p)); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Where a variable of this CTA's shared memory lies in CTA `rank` of the cluster.
template <typename V>
__device__ __forceinline__ const V* of_rank(const V* p, unsigned rank) {
  const V* q;
  asm("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(rank));
  return q;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();  // a warp's lanes arrive as one, wherever a loop before has left them
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Two bf16, neither above its number (of numbers from 0 on).
__device__ __forceinline__ uint32_t pack2_down(float a, float b) {
  uint32_t y;
  asm("cvt.rz.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(b), "f"(a));
  return y;
}
__device__ __forceinline__ uint32_t pack2h(float a, float b) {
  __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&t);
}

template <int D, bool F8, int NT>
struct PagedCfg {
  static constexpr int ROWB = D * (F8 ? 1 : 2), CH = ROWB / 16, HN = 8 * NT;
  static constexpr int WARPS = PD_WARPS, THREADS = 32 * WARPS;
  static constexpr int STAGE = PD_STAGE, HALF = STAGE / 2;
  static constexpr int KT = HALF / ROWB, STAGES = 3, RING = STAGES * STAGE;
  static constexpr int SMEM = WARPS * RING;
  static_assert(HN * D * 4 <= RING, "a warp's last partial output lies in its ring");
  __device__ static uint32_t at(int row, int chunk) {  // swizzled so that eight rows of one chunk column cover all banks
    return row * ROWB + ((CH == 4 ? chunk ^ ((row >> 1) & 3) : chunk ^ (row & 7)) << 4);
  }
  __device__ static int out_at(int h, int d) { return h * D + (d ^ (h >> 1 & 3) << 3); }  // the four heads of a store in banks of their own
};

struct SlotInfo {
  unsigned first, tiles;  // of the sequence, on the line
  int seq;                // -1: empty
};

// An SM's memory is divided in steps: with no more than 196 KiB for a CTA (its static memory and 1 KiB of the system's included) it keeps 60 KiB of L1,
// above that 28, with which 32 801 slots in 8 bits took 23.7 us instead of 21.9.
// WHOLE: a tile never crosses a page (page_size is a multiple of KT), so that its rows lie at one distance from each other.
template <int D, bool F8, int NT, bool WHOLE>
__global__ void __launch_bounds__(PagedCfg<D, F8, NT>::THREADS, 1)
paged_attention_kernel(const PagedAttnArgs a) {
  using C = PagedCfg<D, F8, NT>;
  constexpr int KT = C::KT, CH = C::CH, HN = C::HN, SUB = KT / 16, MT = D / 16, WARPS = C::WARPS;
  constexpr float LIFT = F8 ? PD_LIFT : 0.f;
  extern __shared__ __align__(1024) char smem[];
  __shared__ unsigned s_scan[WARPS], s_warp_first[WARPS];
  __shared__ int s_warp_seq[WARPS], s_warp_len[WARPS];
  constexpr int TILES = 8, PAGES = 4, KEYS = WHOLE ? 1 : KT;
  __shared__ int4 s_tile[WARPS][TILES];  // of the tiles looked up, not yet computed: sequence, its length, tile in it, its first entry in its page
  __shared__ int s_page[WARPS][PAGES][KEYS], s_ent[WARPS][PAGES][KEYS];  // page of a tile or, where it may cross pages, page and entry of each key
  __shared__ SlotInfo s_info[2 * WARPS];
  __shared__ float s_m[2 * WARPS][HN], s_l[2 * WARPS][HN];
  __shared__ float2 s_whole[HN];  // (m, l) of the CTA's share of a cluster's sequence; l -1: it has none
  static_assert(!WHOLE || NT > 1 || C::SMEM + sizeof(s_scan) + sizeof(s_warp_first) + sizeof(s_warp_seq) + sizeof(s_warp_len) + sizeof(s_tile) + sizeof(s_page) +
                                        sizeof(s_ent) + sizeof(s_info) + sizeof(s_m) + sizeof(s_l) + sizeof(s_whole) <= 195 * 1024, "see above");
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int units = a.kv_heads * a.groups, ctas = max(a.by_seq, 1), rank = blockIdx.x % ctas, hu = blockIdx.x / ctas % units, part = blockIdx.x / ctas / units;
  const int kvh = hu / a.groups, h0 = kvh * a.group + hu % a.groups * a.unit, hn = min(a.unit, (kvh + 1) * a.group - h0);
  char* ring = smem + warp * C::RING;
  const uint32_t ring_u = smem_u32(ring);
  // A warp's first piece of a sequence, where it is partial and others follow it, waits in the workspace for the others' end.
  float* first_o = a.first_o + (long long)blockIdx.x * WARPS * a.unit * D;
  if (threadIdx.x < 2 * WARPS) s_info[threadIdx.x].seq = -1;

  // What a warp will want once it knows its place is sent for into L2 before anything is known - a launch
  // before this one may still be writing there -: every thread of the device one line of the page table and one of the queries.
  {
    const unsigned line = blockIdx.x * C::THREADS + threadIdx.x, per_seq = a.q_heads * (D / 64), s = line / per_seq;
    if (line < (unsigned long long)a.n_seqs * a.max_pages / 32) prefetch_l2(a.table + line * 32ull);
    if (s < (unsigned)a.n_seqs) prefetch_l2(a.q + s * a.q_stride + (line - s * per_seq) * 64);
  }

  pdl_wait();
  const float k_by = F8 ? __ldcg(a.k_scale + kvh) : 1.f, vs = F8 ? __ldcg(a.v_scale + kvh) : 1.f;

  // ---- the line: every thread adds up the tiles of a stretch of sequences; each warp for itself or, where they are many, all together
  const long long cap = (long long)a.max_pages * a.page_size;
  // Each length is read several times.  Should another stream write them meanwhile, results are meaningless, but every loop still ends and every
  // access stays where it may be.
  auto length = [&](int s) {
    const int n = __ldcg(a.lens + s);
    return n < 0 || n > cap ? 0 : n;
  };
  auto nothing = [&](int s) {  // a sequence with nothing to attend to: no weight anywhere
    if (__ldcg(a.lens + s) != 0 && hu == 0) atomicOr(a.status, A3_DEV_BAD_POSITION);
    for (int h = h0; h < h0 + hn; ++h) {
      uint4* o = reinterpret_cast<uint4*>(a.out + ((long long)s * a.q_heads + h) * D);
      for (int i = 0; i < D / 8; ++i) o[i] = make_uint4(0, 0, 0, 0);
      if (a.lse) a.lse[(long long)s * a.q_heads + h] = -INFINITY;
    }
  };
  Line parts(0, 1, WARPS);
  unsigned c0 = 0, c1, w0;  // this part's tiles of the line; the first of this warp's
  auto warp_begin = [&](int w) { return c0 + (unsigned)((unsigned long long)(c1 - c0) * w / WARPS); };
  // the sequence that this warp's stretch begins in: its number, its length, its first tile
  int seq0 = 0, len0 = 0;
  unsigned first0 = 0;
  if (a.by_seq) {  // a sequence and head unit has CTAs of its own, each an equal stretch
    seq0 = part, len0 = length(part);
    if (len0 == 0) {
      if (threadIdx.x == 0 && rank == 0) nothing(part);
      if (ctas == 1) return;  // in a cluster nobody leaves alone
    }
    const unsigned total = (len0 + KT - 1) / KT;
    c0 = total * (unsigned)rank / ctas, c1 = total * (unsigned)(rank + 1) / ctas;
    w0 = warp_begin(warp);
  } else {
    const bool alone = a.n_seqs <= 32;
    const int me = alone ? lane : threadIdx.x, per = (a.n_seqs + (alone ? 31 : C::THREADS - 1)) / (alone ? 32 : C::THREADS);
    const int s0 = min(a.n_seqs, me * per), s1 = min(a.n_seqs, s0 + per);
    unsigned mine = 0;
    int n0 = 0;  // the first of them
    for (int s = s0; s < s1; ++s) {
      const int n = length(s);
      if (s == s0) n0 = n;
      mine += (n + KT - 1) / KT;
    }
    unsigned upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned t = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += t;
    }
    unsigned total = __shfl_sync(0xffffffffu, upto, 31), before = upto - mine;
    if (!alone) {
      if (lane == 31) s_scan[warp] = upto, s_warp_seq[warp] = s_warp_len[warp] = 0, s_warp_first[warp] = 0;
      __syncthreads();
      total = 0;
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        if (w < warp) before += s_scan[w];
        total += s_scan[w];
      }
    }
    if (part == 0 && (!alone || warp == 0))
      for (int s = s0; s < s1; ++s)
        if ((s == s0 ? n0 : length(s)) == 0) nothing(s);
    parts = Line(total, a.parts, WARPS);
    if (part >= parts.active) {
      if (hu == 0 && threadIdx.x == 0) a.meta[part] = make_int4(0, 0, 0, 0);
      return;
    }
    c0 = parts.begin(part), c1 = parts.begin(part + 1);
    w0 = warp_begin(warp);
    if (alone) {
      for (int s = s0; s < s1; ++s) {
        const int n = s == s0 ? n0 : length(s);
        const unsigned tiles = (n + KT - 1) / KT;
        if (w0 >= before && w0 < before + tiles) seq0 = s, len0 = n, first0 = before;
        before += tiles;
      }
      const int who = __ffs(__ballot_sync(0xffffffffu, len0 > 0)) - 1;  // none where the stretch is empty and at the line's end
      seq0 = __shfl_sync(0xffffffffu, seq0, who & 31), len0 = __shfl_sync(0xffffffffu, len0, who & 31), first0 = __shfl_sync(0xffffffffu, first0, who & 31);
    } else {
      for (int s = s0; s < s1; ++s) {
        const int n = s == s0 ? n0 : length(s);
        const unsigned tiles = (n + KT - 1) / KT;
        for (int w = 0; w < WARPS; ++w) {
          const unsigned b = warp_begin(w);
          if (b >= before && b < before + tiles) s_warp_seq[w] = s, s_warp_first[w] = before, s_warp_len[w] = n;
        }
        before += tiles;
      }
      __syncthreads();
      seq0 = s_warp_seq[warp], len0 = s_warp_len[warp], first0 = s_warp_first[warp];
    }
  }
  const int count = (int)(warp_begin(warp + 1) - w0);
  __syncthreads();  // s_info

  // ---- this warp's stretch
  if (count > 0) {
    const long long entry = (long long)a.kv_heads * C::ROWB;
    const char *k_base = a.k_pages + (long long)kvh * C::ROWB + lane % CH * 16, *v_base = a.v_pages + (long long)kvh * C::ROWB + lane % CH * 16;
    const long long step = 32 / CH * entry;
    constexpr int RPI = 32 / CH;            // rows that a warp copies with one instruction
    unsigned cfirst = first0;               // first tile of the sequence that is computed

    // Queries of a sequence, one head in eight for each group of four lanes, raw.  Those of the next one are fetched while a sequence is
    // computed (where the registers suffice), the first ones before any key: behind the copies under way a load takes 2 us.
    uint32_t qf[MT][NT][2], qn[MT][NT][2];
    uint32_t(&qr)[MT][NT][2] = NT == 1 ? qn : qf;
    int q_seq = seq0;
    auto load_q = [&] {
      const bf16* q = a.q + q_seq * a.q_stride;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        const int h = nt * 8 + lane / 4;
        const uint32_t* row = reinterpret_cast<const uint32_t*>(q + (h0 + h) * D);
#pragma unroll
        for (int ks = 0; ks < MT; ++ks)
#pragma unroll
          for (int e = 0; e < 2; ++e) qr[ks][nt][e] = h < hn ? __ldcg(row + 8 * ks + (F8 ? 2 * (lane % 4) + e : lane % 4 + 4 * e)) : 0u;
      }
    };

    // Three steps of a tile, each in its own turn: its pages are looked up, three turns later its rows are copied, two turns after that it
    // is computed.  Pages and rows come by asynchronous copies, so that no turn waits for an access that it makes itself.
    int xs = seq0, xn = len0, xt = (int)min(w0 - first0, (unsigned)cap / KT), xp = xt * KT / a.page_size, xe = xt * KT - xp * a.page_size;
    // lengths of the 32 sequences behind the first one, of the 32 behind those once they are done with, a lane for each
    int x_left = count, x_base = xs + 1, x_len = 0;
    auto lengths = [&] { x_len = x_base + lane < a.n_seqs ? length(x_base + lane) : 0; };
    if (x_left > (xn + KT - 1) / KT - xt) lengths();  // the stretch goes on there
    auto next_length = [&] {
      if (xs == a.n_seqs - 1) return xn = 0, true;
      if (++xs == x_base + 32) {
        x_base = xs;
        lengths();
      }
      xn = __shfl_sync(0xffffffffu, x_len, xs - x_base);
      return xn > 0;
    };
    auto look_up = [&](int j) {
      if (x_left <= 0) return;
      const int32_t* row = a.table + (long long)xs * a.max_pages;
      if (lane == 0) s_tile[warp][j % TILES] = make_int4(xs, xn, xt, xe);
      if constexpr (WHOLE) {
        if (lane == 0) cp_async4(smem_u32(&s_page[warp][j % PAGES][0]), row + min(xp, a.max_pages - 1));
      } else {
#pragma unroll
        for (int i = lane; i < KT; i += 32) {
          const int key = xt * KT + i, p = key / a.page_size;
          if (key < xn) cp_async4(smem_u32(&s_page[warp][j % PAGES][i]), row + p);
          s_ent[warp][j % PAGES][i] = key < xn ? key - p * a.page_size : -1;
        }
      }
      if (--x_left == 0) return;
      if (++xt * KT >= xn) {
        xt = xp = xe = 0;
        while (!next_length()) {}
      } else if (WHOLE && (xe += KT) == a.page_size) {
        xe = 0;
        ++xp;
      }
    };
    auto copy = [&](int j) {  // rows that are not there are filled with zeros: nothing behind a sequence is read
      if (j >= count) return;
      const uint32_t dst = ring_u + j % C::STAGES * C::STAGE;
      const int r0 = lane / CH;
      if constexpr (WHOLE) {
        const int4 x = s_tile[warp][j % TILES];
        const int page = s_page[warp][j % PAGES][0];
        const bool good = (unsigned)page < (unsigned)a.n_pages;
        if (!good) atomicOr(a.status, A3_DEV_BAD_POSITION);
        const int left = good ? x.y - x.z * KT : 0;
        long long at = (good ? page * a.page_stride : 0) + (x.w + r0) * entry;
        if (left >= KT) {
#pragma unroll
          for (int i = 0; i < KT / RPI; ++i, at += step) {
            cp_async16(dst + C::at(r0 + i * RPI, lane % CH), k_base + at, true);
            cp_async16(dst + C::HALF + C::at(r0 + i * RPI, lane % CH), v_base + at, true);
          }
        } else {
#pragma unroll
          for (int i = 0; i < KT / RPI; ++i, at += step) {
            const bool there = r0 + i * RPI < left;
            cp_async16(dst + C::at(r0 + i * RPI, lane % CH), k_base + (there ? at : 0), there);
            cp_async16(dst + C::HALF + C::at(r0 + i * RPI, lane % CH), v_base + (there ? at : 0), there);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < KT / RPI; ++i) {
          const int page = s_page[warp][j % PAGES][r0 + i * RPI], ent = s_ent[warp][j % PAGES][r0 + i * RPI];
          const bool good = (unsigned)page < (unsigned)a.n_pages, there = ent >= 0 && good;
          if (ent >= 0 && !good) atomicOr(a.status, A3_DEV_BAD_POSITION);
          const long long at = there ? page * a.page_stride + ent * entry : 0;
          cp_async16(dst + C::at(r0 + i * RPI, lane % CH), k_base + at, there);
          cp_async16(dst + C::HALF + C::at(r0 + i * RPI, lane % CH), v_base + at, there);
        }
      }
    };

    float o[MT][NT][4], m[NT][2], l[NT][2], cq[NT][2];
#pragma unroll 1
    for (int j = 0; j < 3; ++j) look_up(j);
    cp_async_commit();
    load_q();
    cp_async_wait<0>();
    __syncwarp();
    static_assert(C::STAGES == 3, "two turns between the copy and its use, three between look-up and copy");
    bool fresh = true;
    int piece0 = 0;
    // the first two turns only copy: what runs once should not be there a second time, its instructions come cold from L2
    for (int i = -2; i < count; ++i) {
      copy(i + 2);
      look_up(i + 5);
      cp_async_commit();
      if (i < 0) {
        __syncwarp();  // a look-up may take the place of the page that another lane has just read
        continue;
      }
      const int4 tile = s_tile[warp][i % TILES];
      const int cs = tile.x, cn = tile.y, ct = tile.z;
      if (fresh) {  // a sequence, or what is left of one, begins
        fresh = false;
        piece0 = ct;
        if (q_seq != cs) {
          q_seq = cs;
          load_q();
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
          for (int ks = 0; ks < MT; ++ks)
#pragma unroll
            for (int e = 0; e < 2; ++e) qf[ks][nt][e] = qr[ks][nt][e];
          float up = a.scale_log2;
          if (F8) {
            float most = 0.f;
#pragma unroll
            for (int ks = 0; ks < MT; ++ks)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&qf[ks][nt][e]));
                most = fmaxf(most, fmaxf(fabsf(f.x), fabsf(f.y)));
              }
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
            most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
            // 2^(14 - e) brings the largest element to [2^14, 2^15); kept where both it and its inverse are normal numbers
            int ex = most > 0.f && most < INFINITY ? ilogbf(most) - 14 : 0;
            ex = max(-120, min(120, ex));
            const float down = __int_as_float((127 - ex) << 23);
            up *= __int_as_float((127 + ex) << 23) * k_by;
#pragma unroll
            for (int ks = 0; ks < MT; ++ks)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const float2 f = __bfloat1622float2(*reinterpret_cast<__nv_bfloat162*>(&qf[ks][nt][e]));
                qf[ks][nt][e] = pack2h(f.x * down, f.y * down);
              }
          }
          // columns of the accumulators are heads 2 (lane % 4) and the one after it
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            cq[nt][e] = F8 ? __shfl_sync(0xffffffffu, up, (2 * (lane % 4) + e) * 4) : up;
            m[nt][e] = -INFINITY;
            l[nt][e] = 0.f;
          }
#pragma unroll
          for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[mt][nt][e] = 0.f;
        }
        if (NT == 1 && cs + 1 < a.n_seqs && count - i > (cn + KT - 1) / KT - ct) {  // more sequences follow: of the next one, unless it is empty
          ++q_seq;
          load_q();
        }
      }
      cp_async_wait<C::STAGES - 1>();
      __syncwarp();
      const uint32_t kt_u = ring_u + i % C::STAGES * C::STAGE, vt_u = kt_u + C::HALF;

      // ---- S^T = K Q^T; all loads of 16 keys first, two sums of each product (a chain of eight would take 8 x 22 clocks)
      float s[SUB][NT][4];
      constexpr int KL = F8 ? MT / 2 : MT;  // ldmatrix instructions for 16 rows
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
        uint32_t k[KL][4];
        const int row = sub * 16 + (lane >> 3 & 1) * 8 + (lane & 7);
#pragma unroll
        for (int j = 0; j < KL; ++j) ldmatrix_x4(kt_u + C::at(row, 2 * j + (lane >> 4)), k[j][0], k[j][1], k[j][2], k[j][3]);
        float odd[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][nt][e] = odd[nt][e] = 0.f;
#pragma unroll
        for (int j = 0; j < KL; ++j) {
          if constexpr (!F8) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
              mma_any<false>(j & 1 ? odd[nt] : s[sub][nt], k[j][0], k[j][1], k[j][2], k[j][3], qf[j][nt][0], qf[j][nt][1]);
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t x = k[j][2 * e], y = k[j][2 * e + 1];
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_any<true>(e ? odd[nt] : s[sub][nt], e4m3x2_to_f16x2(x), e4m3x2_to_f16x2(y), e4m3x2_to_f16x2(x >> 16), e4m3x2_to_f16x2(y >> 16),
                              qf[2 * j + e][nt][0], qf[2 * j + e][nt][1]);
            }
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][nt][e] += odd[nt][e];
      }
      // values of the first 16 keys, on their way while the weights are formed
      uint32_t v[KL][4];
      auto load_v = [&](int sub) {
        const int row = sub * 16 + (F8 ? lane >> 3 & 1 : lane >> 4) * 8 + (lane & 7);
#pragma unroll
        for (int j = 0; j < KL; ++j) ldmatrix_x4_trans(vt_u + C::at(row, 2 * j + (F8 ? lane >> 4 : lane >> 3 & 1)), v[j][0], v[j][1], v[j][2], v[j][3]);
      };
      load_v(0);

      // ---- running softmax: the reference need not be the maximum, it only has to be near it.  It is raised, over the lanes that
      // share a head and with everything rescaled, when a logit's weight is more than 2^8 of its.  m is the logit of weight 1, LIFT below it.
      const int left = cn - ct * KT;  // keys from here on
      bool grew = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float t = s[sub][nt][e] * cq[nt][e & 1];
            s[sub][nt][e] = t;
            grew |= t > m[nt][e & 1] + (PD_SLACK + LIFT);
          }
      if (left < KT) {  // the sequence ends in this tile; what `grew` made of the rows behind it only raises the reference needlessly
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (sub * 16 + (e >> 1) * 8 + lane / 4 >= left) s[sub][nt][e] = -INFINITY;
      }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float now = -INFINITY;
#pragma unroll
            for (int sub = 0; sub < SUB; ++sub) now = fmaxf(now, fmaxf(s[sub][nt][e], s[sub][nt][e + 2]));
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, x));
            now = fmaxf(m[nt][e], now - LIFT);
            const float f = now == -INFINITY ? 1.f : ex2(m[nt][e] - now);
            m[nt][e] = now;
            l[nt][e] *= f;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) o[mt][nt][e] *= f, o[mt][nt][e + 2] *= f;
          }
      }
      uint32_t hi[SUB][NT][2], lo[SUB][NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        // all logits -inf so far: no weight, not NaN
        const float r0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0], r1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1];
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p0 = ex2(s[sub][nt][2 * e] - r0), p1 = ex2(s[sub][nt][2 * e + 1] - r1);
            l[nt][0] += p0;
            l[nt][1] += p1;
            if constexpr (F8) {
              hi[sub][nt][e] = movmatrix(pack2h(p0, p1));
            } else {
              // the upper term is rounded down and the lower one is 2^-20 of the weight at least: an infinite value times either is that infinity
              const uint32_t h = pack2_down(p0, p1);
              const float2 back = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&h));
              hi[sub][nt][e] = movmatrix(h);
              lo[sub][nt][e] = movmatrix(pack2(fmaxf(p0 - back.x, p0 * 0x1p-20f), fmaxf(p1 - back.y, p1 * 0x1p-20f)));
            }
          }
      }

      // ---- O^T += V^T P^T
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
        for (int j = 0; j < KL; ++j) {
          if constexpr (!F8) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_any<false>(o[j][nt], v[j][0], v[j][1], v[j][2], v[j][3], hi[sub][nt][0], hi[sub][nt][1]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_any<false>(o[j][nt], v[j][0], v[j][1], v[j][2], v[j][3], lo[sub][nt][0], lo[sub][nt][1]);
          } else {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // a register holds dimensions (2i, 2i+1) of one key, then of the next: rows i and i + 8 of the product are those two
              const uint32_t x = __byte_perm(v[j][2 * e], 0, 0x3120), y = __byte_perm(v[j][2 * e + 1], 0, 0x3120);
#pragma unroll
              for (int nt = 0; nt < NT; ++nt)
                mma_any<true>(o[2 * j + e][nt], e4m3x2_to_f16x2(x), e4m3x2_to_f16x2(x >> 16), e4m3x2_to_f16x2(y), e4m3x2_to_f16x2(y >> 16), hi[sub][nt][0],
                              hi[sub][nt][1]);
            }
          }
        }
        if (sub + 1 < SUB) load_v(sub + 1);
      }
      __syncwarp();

      // ---- the end of a sequence, or of the stretch
      const int tiles = (cn + KT - 1) / KT;
      if (ct == tiles - 1 || i == count - 1) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], x);
        if (piece0 == 0 && ct == tiles - 1 && ctas == 1) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = nt * 8 + 2 * (lane % 4) + e;
              if (h < hn) {
                const float f = l[nt][e] == 0.f ? 0.f : vs / l[nt][e];
                const long long at = (long long)cs * a.q_heads + h0 + h;
                if constexpr (F8) {
#pragma unroll
                  for (int mt = 0; mt < MT; ++mt)
                    *reinterpret_cast<uint32_t*>(a.out + at * D + mt * 16 + 2 * (lane / 4)) = pack2(o[mt][nt][e] * f, o[mt][nt][e + 2] * f);
                }
                if (a.lse && lane / 4 == 0) a.lse[at] = l[nt][e] == 0.f ? -INFINITY : (m[nt][e] + log2f(l[nt][e])) * LN2;
              }
            }
          if constexpr (!F8) {
            // Lanes 4 apart hold neighbouring dimensions of the same two heads: one takes the first head's pair, the other the second's.
            const int odd = lane >> 2 & 1;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const float f0 = l[nt][0] == 0.f ? 0.f : vs / l[nt][0], f1 = l[nt][1] == 0.f ? 0.f : vs / l[nt][1];
              const int h = nt * 8 + 2 * (lane % 4) + odd;
              bf16* dst = a.out + ((long long)cs * a.q_heads + h0 + h) * D + (lane / 8) * 2;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                  const float x = o[mt][nt][2 * half] * f0, y = o[mt][nt][2 * half + 1] * f1;
                  const float got = __shfl_xor_sync(0xffffffffu, odd ? x : y, 4);
                  if (h < hn) *reinterpret_cast<uint32_t*>(dst + mt * 16 + half * 8) = odd ? pack2(got, y) : pack2(x, got);
                }
            }
          }
        } else {
          const int which = i == count - 1, info = 2 * warp + which;  // partial and not the last: the first
          float* dst = which == 0 ? first_o + warp * a.unit * D : reinterpret_cast<float*>(ring);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = nt * 8 + 2 * (lane % 4) + e;
              if (which == 0 && h >= hn) continue;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                const int d = mt * 16 + (F8 ? 2 * (lane / 4) : lane / 4);
                dst[C::out_at(h, d)] = o[mt][nt][e] * vs;
                dst[C::out_at(h, d + (F8 ? 1 : 8))] = o[mt][nt][e + 2] * vs;
              }
              if (lane / 4 == 0) s_m[info][h] = m[nt][e], s_l[info][h] = l[nt][e];
            }
          if (lane == 0) s_info[info] = SlotInfo{cfirst, (unsigned)tiles, cs};
        }
        fresh = true;
        if (ct == tiles - 1) cfirst += tiles;
      }
    }
  }
  // The join, or the next launch, is let in here and by the join once its loads are out: call after call, 16 sequences in 8 bits take 35.1 us so and
  // took 36.7 with both at the start, one of 5 153 slots 11.0 and 11.6, one of 32 801 in 8 bits 22.5 and 22.7.
  pdl_launch_dependents();
  if (!a.by_seq && hu == 0 && threadIdx.x == 0) {  // first0 and len0 are of the sequence that the part begins with
    const int from = first0 < c0 ? parts.of(first0) : part;
    const unsigned to = min((unsigned)parts.of(first0 + (unsigned)(len0 + KT - 1) / KT - 1), parts.active - 1);
    a.meta[part] = make_int4(seq0, from, from == part - 1 ? (int)to - from + 1 : 0, 0);
  }
  __syncthreads();

  // ---- what the warps hold of one sequence, merged
  if (ctas > 1 && threadIdx.x < HN) s_whole[threadIdx.x] = make_float2(-INFINITY, -1.f);
  if (ctas > 1) __syncthreads();
  int seqs[2 * WARPS];
#pragma unroll
  for (int i = 0; i < 2 * WARPS; ++i) seqs[i] = s_info[i].seq;
  unsigned left = 0;
#pragma unroll
  for (int i = 0; i < 2 * WARPS; ++i) left |= (seqs[i] >= 0) << i;
  while (left) {
    const SlotInfo info = s_info[__ffs(left) - 1];
    unsigned members = 0;
#pragma unroll
    for (int i = 0; i < 2 * WARPS; ++i) members |= (seqs[i] == info.seq) << i;
    left &= ~members;
    const bool began = info.first < c0, goes_on = info.first + info.tiles > c1;
    const long long slot = ((long long)part * units + hu) * 2 + (began ? 0 : 1);
    for (int x = threadIdx.x; x < hn * (D / 4); x += C::THREADS) {
      const int h = x / (D / 4), d = x % (D / 4) * 4;
      // the warps' last pieces lie in shared memory, all read at once whether they belong to this sequence or not; first pieces are rare
      float f[WARPS], mm = -INFINITY, ll = 0.f;
      float4 v[WARPS];
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        f[w] = s_m[2 * w + 1][h];
        v[w] = *reinterpret_cast<const float4*>(smem + w * C::RING + C::out_at(h, d) * 4);
      }
#pragma unroll
      for (int w = 0; w < WARPS; ++w) {
        if (!(members >> (2 * w + 1) & 1)) f[w] = -INFINITY;
        mm = fmaxf(mm, f[w]);
      }
      for (unsigned b = members & 0x55555555u; b; b &= b - 1) mm = fmaxf(mm, s_m[__ffs(b) - 1][h]);
      const float ref = mm == -INFINITY ? 0.f : mm;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
      auto add = [&](float g, float l, const float4& y) {
        ll += g * l;
        o.x += g * y.x, o.y += g * y.y, o.z += g * y.z, o.w += g * y.w;
      };
#pragma unroll
      for (int w = 0; w < WARPS; ++w)
        if (members >> (2 * w + 1) & 1) add(ex2(f[w] - ref), s_l[2 * w + 1][h], v[w]);
      for (unsigned b = members & 0x55555555u; b; b &= b - 1) {
        const int i = __ffs(b) - 1;
        add(ex2(s_m[i][h] - ref), s_l[i][h], *reinterpret_cast<const float4*>(first_o + i / 2 * a.unit * D + C::out_at(h, d)));
      }
      if (ctas > 1) {  // in the place of warp 0's, which nobody else reads
        *reinterpret_cast<float4*>(smem + C::out_at(h, d) * 4) = o;
        if (d == 0) s_whole[h] = make_float2(mm, ll);
      } else if (!began && !goes_on) {
        const float g = ll == 0.f ? 0.f : 1.f / ll;
        const long long at = (long long)info.seq * a.q_heads + h0 + h;
        *reinterpret_cast<uint2*>(a.out + at * D + d) = make_uint2(pack2(o.x * g, o.y * g), pack2(o.z * g, o.w * g));
        if (a.lse && d == 0) a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * LN2;
      } else {
        *reinterpret_cast<float4*>(a.part_o + (slot * a.unit + h) * D + d) = o;
        if (d == 0) a.part_ml[slot * a.unit + h] = make_float2(mm, ll);
      }
    }
  }

  // ---- what the CTAs of a cluster hold of it, merged by the first
  if (ctas == 1) return;
  cluster_sync();
  if (rank == 0) {
    for (int x = threadIdx.x; x < hn * (D / 4); x += C::THREADS) {
      const int h = x / (D / 4), d = x % (D / 4) * 4;
      float2 ml[PD_CTAS];
      float4 v[PD_CTAS];
#pragma unroll
      for (int i = 0; i < PD_CTAS; ++i) {
        ml[i] = make_float2(-INFINITY, -1.f);
        if (i < ctas) {
          ml[i] = *of_rank(&s_whole[h], i);
          v[i] = *of_rank(reinterpret_cast<const float4*>(smem + C::out_at(h, d) * 4), i);
        }
      }
      float mm = -INFINITY, ll = 0.f;
#pragma unroll
      for (int i = 0; i < PD_CTAS; ++i) mm = fmaxf(mm, ml[i].x);
      const float ref = mm == -INFINITY ? 0.f : mm;
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < PD_CTAS; ++i) {
        if (ml[i].y == -1.f) continue;
        const float g = ex2(ml[i].x - ref);
        ll += g * ml[i].y;
        o.x += g * v[i].x, o.y += g * v[i].y, o.z += g * v[i].z, o.w += g * v[i].w;
      }
      const float g = ll == 0.f ? 0.f : 1.f / ll;
      const long long at = (long long)part * a.q_heads + h0 + h;
      *reinterpret_cast<uint2*>(a.out + at * D + d) = make_uint2(pack2(o.x * g, o.y * g), pack2(o.z * g, o.w * g));
      if (a.lse && d == 0) a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * LN2;
    }
  }
  cluster_sync();  // the others' memory is there until it has been read
}

// Block (p, unit, head): the sequence that part p begins with, if it began in the part before, from all parts that hold some of it:
// meta[p] = (sequence, first of those parts, how many, -), none where there is nothing to join.  A warp's lanes cover the head dimension;
// the warps take parts in turn.
constexpr int PJ_WARPS = 4;
template <int D>
__global__ void __launch_bounds__(32 * PJ_WARPS)
paged_join_kernel(const PagedAttnArgs a) {
  constexpr int V = D / 32;
  extern __shared__ float s_f[];  // [parts] weights
  __shared__ float s_red[2][PJ_WARPS], s_o[PJ_WARPS][D];
  const int p = blockIdx.x + 1, hu = blockIdx.y, g = blockIdx.z, units = a.kv_heads * a.groups, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int kvh = hu / a.groups, h0 = kvh * a.group + hu % a.groups * a.unit, hn = min(a.unit, (kvh + 1) * a.group - h0);
  pdl_wait();
  if (g >= hn) return;
  const int4 meta = __ldcg(a.meta + p);
  const int seq = meta.x, from = meta.y, n = meta.z;
  if (n == 0) return;
  constexpr int EARLY = 8;  // parts of a warp whose outputs are sent for before their weights are known
  // the first part holds the sequence's beginning in its second place, the others hold it in their first
  const int at0 = (from * units + hu) * 2 * a.unit + g, stride = units * 2 * a.unit;
  auto slot = [&](int i) { return at0 + i * stride + (i == 0 ? a.unit : 0); };
  using Vec = std::conditional_t<V == 4, float4, float2>;
  Vec early[EARLY];
#pragma unroll
  for (int k = 0; k < EARLY; ++k)
    if (warp + k * PJ_WARPS < n) early[k] = __ldcg(reinterpret_cast<const Vec*>(a.part_o + (long long)slot(warp + k * PJ_WARPS) * D + lane * V));
  float most = -INFINITY;
  float2 mine = make_float2(-INFINITY, 0.f);
  for (int i = threadIdx.x; i < n; i += 32 * PJ_WARPS) {
    const float2 ml = __ldcg(a.part_ml + slot(i));
    if (i == (int)threadIdx.x) mine = ml;
    most = fmaxf(most, ml.x);
  }
#pragma unroll
  for (int x = 16; x; x >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, x));
  if (lane == 0) s_red[0][warp] = most;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < PJ_WARPS; ++w) most = fmaxf(most, s_red[0][w]);
  const float ref = most == -INFINITY ? 0.f : most;
  float ll = 0.f;
  for (int i = threadIdx.x; i < n; i += 32 * PJ_WARPS) {
    const float2 ml = i == (int)threadIdx.x ? mine : __ldcg(a.part_ml + slot(i));
    const float f = ex2(ml.x - ref);
    s_f[i] = f;
    ll += f * ml.y;
  }
#pragma unroll
  for (int x = 16; x; x >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, x);
  if (lane == 0) s_red[1][warp] = ll;
  __syncthreads();
  ll = 0.f;
#pragma unroll
  for (int w = 0; w < PJ_WARPS; ++w) ll += s_red[1][w];
  pdl_launch_dependents();
  float o[V] = {};
  auto add = [&](const Vec& v, float f) {
    o[0] += f * v.x, o[1] += f * v.y;
    if constexpr (V == 4) o[2] += f * v.z, o[3] += f * v.w;
  };
#pragma unroll
  for (int k = 0; k < EARLY; ++k)
    if (warp + k * PJ_WARPS < n) add(early[k], s_f[warp + k * PJ_WARPS]);
#pragma unroll 4
  for (int i = warp + EARLY * PJ_WARPS; i < n; i += PJ_WARPS) add(__ldcg(reinterpret_cast<const Vec*>(a.part_o + (long long)slot(i) * D + lane * V)), s_f[i]);
#pragma unroll
  for (int v = 0; v < V; ++v) s_o[warp][lane * V + v] = o[v];
  __syncthreads();
  if (threadIdx.x < D / 2) {
    const int d = threadIdx.x * 2;
    float x = 0.f, y = 0.f;
#pragma unroll
    for (int w = 0; w < PJ_WARPS; ++w) x += s_o[w][d], y += s_o[w][d + 1];
    const float f = ll == 0.f ? 0.f : 1.f / ll;
    const long long at = (long long)seq * a.q_heads + h0 + g;
    *reinterpret_cast<uint32_t*>(a.out + at * D + d) = pack2(x * f, y * f);
    if (a.lse && d == 0) a.lse[at] = ll == 0.f ? -INFINITY : (most + log2f(ll)) * LN2;
  }
}

struct PagedPlan {
  int unit, groups, parts;
  size_t meta, ml, o, bytes;
};
static PagedPlan paged_plan(const a3_handle* h) {
  PagedPlan p;
  const int group = h->m.n_q_heads / h->m.n_kv_heads;
  p.unit = group <= 8 ? group : 16;  // query heads that one pass over the keys serves
  p.groups = cdiv(group, p.unit);
  const int units = h->m.n_kv_heads * p.groups;
  p.parts = h->sm_count / units;
  if (p.parts < 1) p.parts = 1;
  const size_t slots = (size_t)2 * p.parts * units * 2 * p.unit;
  p.meta = align_up(sizeof(int4) * 2 * p.parts, 256);
  p.ml = align_up(slots * sizeof(float2), 256);
  p.o = align_up(slots * h->m.head_dim * 4, 256);
  p.bytes = p.meta + p.ml + p.o + (size_t)2 * p.parts * units * PD_WARPS * p.unit * h->m.head_dim * 4;
  return p;
}

// CTAs for each sequence and head unit, 0 where the line has them; whatever the lengths turn out to be within the page table's width.
static int paged_alone(const a3_handle* h, const PagedPlan& plan, const a3_paged_cache* cache, int n_seqs, int max_pages) {
  const bool f8 = cache->type == A3_CACHE_E4M3;
  const long long slots = (long long)max_pages * cache->page_size, seqs = (long long)n_seqs * h->m.n_kv_heads * plan.groups;
  const long long round = (long long)PD_WARPS * (PD_STAGE / 2 / (h->m.head_dim * (f8 ? 1 : 2)));  // slots of a CTA whose warps have a tile each
  // clusters leave SMs unused: 12 of eight CTAs run at once, 16 do not (8 sequences of 5 100 17.2 us and on the line 12.6)
  auto fit = [&](int ctas) { return seqs * ctas <= h->sm_count - (ctas == 1 ? 0 : ctas < 8 ? h->sm_count / 8 : h->sm_count / 4); };
  int ctas = 1;
  while (ctas < PD_CTAS && slots > (f8 ? PD_FEW_E4M3 : PD_FEW) * round * ctas && fit(2 * ctas)) ctas *= 2;
  return slots <= (f8 ? PD_ALONE_E4M3 : PD_ALONE) * round * ctas && fit(ctas) ? ctas : 0;
}

template <int D, bool F8, int NT, bool WHOLE>
static int paged_launch(const a3_handle* h, const PagedAttnArgs& a, int units, cudaStream_t st) {
  static SmemAttrOnce once;
  using C = PagedCfg<D, F8, NT>;
  A3_TRY(smem_attr_once(once, h->device, paged_attention_kernel<D, F8, NT, WHOLE>, C::SMEM));
  {
    ProfScope prof(h, A3_K_PAGED_ATTENTION, st);
    A3_CUDA(launch_pdl_cluster(a.by_seq > 1 ? a.by_seq : 1, paged_attention_kernel<D, F8, NT, WHOLE>, dim3((a.by_seq ? a.n_seqs * a.by_seq : a.most_parts) * units),
                               dim3(C::THREADS), C::SMEM, st, a));
    A3_LAUNCHED();
  }
  if (a.by_seq || a.most_parts == 1) return A3_OK;  // every sequence ends in the part that it begins in
  ProfScope prof(h, A3_K_PAGED_ATTENTION, st);
  A3_CUDA(launch_pdl(paged_join_kernel<D>, dim3(a.most_parts - 1, units, a.unit), dim3(32 * PJ_WARPS), a.most_parts * sizeof(float), st, a));
  return launched();
}

}  // namespace a3

using namespace a3;

extern "C" size_t a3_paged_attention_workspace_bytes(const a3_handle* h, const a3_paged_cache* cache, int n_seqs, int max_pages) {
  if (!h || !cache || n_seqs <= 0 || max_pages < 0) return 0;
  const PagedPlan plan = paged_plan(h);
  return paged_alone(h, plan, cache, n_seqs, max_pages) > 0 ? 0 : plan.bytes;
}

extern "C" int a3_paged_attention(const a3_handle* h, const a3_paged_cache* cache, const a3_paged_queries* queries, a3_stream stream) {
  if (!h || !cache || !queries) return A3_EINVAL;
  const a3_paged_queries& p = *queries;
  if (p.n_seqs < 0 || p.max_pages < 0 || !isfinite(p.scale)) return A3_EINVAL;
  A3_TRY(paged_cache_check(h, cache));
  // slots of a sequence and tiles of all sequences (16 slots at least) are counted in 32 bits
  const unsigned long long slots = (unsigned long long)p.max_pages * cache->page_size;
  if (slots > 0x7fff0000ull || (p.n_seqs > 0 && slots > (1ull << 34) / p.n_seqs)) return A3_ETOOLARGE;
  if (p.n_seqs == 0) return A3_OK;
  if ((!p.page_table && p.max_pages > 0) || !p.cache_len || !p.q_rows || !p.out) return A3_EINVAL;
  if (((uintptr_t)p.q_rows | (uintptr_t)p.out) & 15) return A3_EINVAL;
  const a3_model_desc& m = h->m;
  if (p.q_stride < (uint64_t)m.n_q_heads * m.head_dim || p.q_stride % 8 || p.q_stride > (uint64_t)1 << 31) return A3_EINVAL;
  const PagedPlan plan = paged_plan(h);
  const int alone = paged_alone(h, plan, cache, p.n_seqs, p.max_pages);
  if (!alone && (!p.ws || (uintptr_t)p.ws & 255)) return A3_EINVAL;
  if (!alone && p.ws_bytes < plan.bytes) return A3_EWORKSPACE;
  PagedAttnArgs a{};
  a.k_pages = (const char*)cache->k_pages, a.v_pages = (const char*)cache->v_pages;
  a.page_stride = (long long)cache->page_stride, a.n_pages = cache->n_pages, a.page_size = cache->page_size;
  a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
  a.table = p.page_table, a.lens = p.cache_len, a.n_seqs = p.n_seqs, a.max_pages = p.max_pages;
  a.q = (const bf16*)p.q_rows, a.q_stride = (long long)p.q_stride;
  a.scale_log2 = p.scale * 1.44269504088896341f;
  a.out = (bf16*)p.out, a.lse = p.lse_out;
  a.q_heads = m.n_q_heads, a.kv_heads = m.n_kv_heads, a.group = m.n_q_heads / m.n_kv_heads;
  a.unit = plan.unit, a.groups = plan.groups, a.parts = plan.parts, a.by_seq = alone;
  const int tile = PD_STAGE / 2 / (m.head_dim * (cache->type == A3_CACHE_E4M3 ? 1 : 2));
  a.most_parts = (slots / tile + 1) * p.n_seqs >= (unsigned long long)plan.parts * PD_WARPS * PD_MANY ? 2 * plan.parts : plan.parts;
  if (!alone) {
    a.meta = (int4*)p.ws;
    a.part_ml = (float2*)((char*)p.ws + plan.meta);
    a.part_o = (float*)((char*)p.ws + plan.meta + plan.ml);
    a.first_o = (float*)((char*)p.ws + plan.meta + plan.ml + plan.o);
  }
  a.status = h->dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  const int units = m.n_kv_heads * plan.groups;
  const bool f8 = cache->type == A3_CACHE_E4M3;
  auto heads = [&](auto d, auto nt) {
    constexpr int DD = decltype(d)::value, N = decltype(nt)::value;
    if (f8) return a.page_size % PagedCfg<DD, true, N>::KT ? paged_launch<DD, true, N, false>(h, a, units, st) : paged_launch<DD, true, N, true>(h, a, units, st);
    return a.page_size % PagedCfg<DD, false, N>::KT ? paged_launch<DD, false, N, false>(h, a, units, st) : paged_launch<DD, false, N, true>(h, a, units, st);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (m.head_dim == 64) return plan.unit <= 8 ? heads(D64{}, One{}) : heads(D64{}, Two{});
  return plan.unit <= 8 ? heads(D128{}, One{}) : heads(D128{}, Two{});
}
