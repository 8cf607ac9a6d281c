// Attention of one new token per sequence over a paged cache (a3_paged_attention), split over the keys and joined.
//
//   o[s][h] = sum_t softmax_t(scale q[s][h] . k[s][t][h/G]) v[s][t][h/G],   t < len[s]
//
// Every key and value is read once and used by the G query heads of its KV head: bound by HBM.  The lengths are known on the
// device only, so the kernel divides the work itself: the keys of all sequences, cut into tiles of KT keys, form one line
// per KV head; a CTA takes an equal stretch of it and each of its warps an equal part of that, whatever sequences
// lie there.  A warp streams its tiles through a ring of its own with 16-byte asynchronous copies (two tiles under way while
// the third is computed, no barrier between warps) and keeps the running maximum and sum of the softmax, fp32, in registers.
// Products: S^T = K Q^T and O^T = V^T P^T with warp-level MMAs, keys (head dimensions) on the 16-row side and the heads that share
// them on the 8-column side: the query heads of a group fill the narrow side of the instruction, and what they need of the
// tensor pipe is a few percent, so nothing is gained by the wide one.  Where a sequence lies in one warp's part the result is
// written at once; a CTA merges what its warps hold of a sequence; what several CTAs hold goes to the workspace as (maximum, sum,
// unnormalised output) and a second kernel merges it in the order of the keys.  The division depends on the lengths and
// the device only: results do not depend on timing.
//
// P is kept to 16 bits for bf16 values (two bf16 terms): with one, its rounding is as large as that of the output itself.  8-bit keys
// and values are widened to fp16, which holds them exactly; the query is scaled by a power of two per head so that fp16 holds all of
// its bits down to 2^-29 of its largest element, and P as fp16 is off by 2^-12 at most.
#include <cuda_fp16.h>

#include <type_traits>

#include "a3_internal.cuh"
#include "a3_paged.cuh"

namespace a3 {

constexpr int PD_WARPS = 4, PD_THREADS = 32 * PD_WARPS;
constexpr int PD_STAGE = 8192;                 // bytes of a tile: keys in the lower half, values in the upper
constexpr int PD_CTAS = 2;                     // per SM

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
  int unit, parts;
  // workspace
  struct PartMeta* meta;  // [parts]
  float* part_o;          // [parts][units][2][unit][D]
  float2* part_ml;        // [parts][units][2][unit]
  uint32_t* status;
};
// The sequence that a part begins with: its number, its first tile on the line and its tiles; the tiles on the line, the parts that share them.
struct PartMeta {
  long long first, tiles, total;
  int seq, active;
};

__device__ __forceinline__ long long part_begin(long long p, long long total, long long active) { return p * total / active; }
__device__ __forceinline__ long long part_of(long long tile, long long total, long long active) { return ((tile + 1) * active - 1) / total; }

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};\n"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t y;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(y) : "h"((unsigned short)two));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2h(float a, float b) {
  __half2 t = __floats2half2_rn(a, b);
  return *reinterpret_cast<uint32_t*>(&t);
}

template <int D, bool F8, int NT>
struct PagedCfg {
  static constexpr int ROWB = D * (F8 ? 1 : 2), CH = ROWB / 16, KT = PD_STAGE / 2 / ROWB, HN = 8 * NT;
  static constexpr int STAGES = D == 128 && NT == 2 ? 2 : 3;  // what leaves room for two CTAs per SM
  static constexpr int SLOT = HN * D * 4;  // bytes of one partial output in shared memory
  static constexpr int RING = STAGES * PD_STAGE, SMEM = PD_WARPS * (RING + SLOT);
  static_assert(SLOT <= RING, "a warp's second partial output lies in its ring");
  __device__ static uint32_t at(int row, int chunk) {  // swizzled so that eight rows of one chunk column cover all banks
    return row * ROWB + ((CH == 4 ? chunk ^ ((row >> 1) & 3) : chunk ^ (row & 7)) << 4);
  }
  __device__ static int out_at(int h, int d) { return h * D + (d ^ (h >> 1 & 3) << 3); }  // the four heads of a store in banks of their own
};

struct SlotInfo {
  long long first, tiles;  // of the sequence, on the line
  int seq;                 // -1: empty
};

template <int D, bool F8, int NT>
__global__ void __launch_bounds__(PD_THREADS, PD_CTAS)
paged_attention_kernel(const PagedAttnArgs a) {
  using C = PagedCfg<D, F8, NT>;
  constexpr int KT = C::KT, CH = C::CH, HN = C::HN, SUB = KT / 16, MT = D / 16;
  extern __shared__ __align__(1024) char smem[];
  __shared__ long long s_scan[PD_WARPS], s_warp_first[PD_WARPS], s_warp_seqtile[PD_WARPS];
  __shared__ int s_warp_seq[PD_WARPS];
  __shared__ SlotInfo s_info[2 * PD_WARPS];
  __shared__ float s_m[2 * PD_WARPS][HN], s_l[2 * PD_WARPS][HN];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int units = a.kv_heads * a.groups, hu = blockIdx.x % units, part = blockIdx.x / units;
  const int kvh = hu / a.groups, h0 = kvh * a.group + hu % a.groups * a.unit, hn = min(a.unit, (kvh + 1) * a.group - h0);
  char* ring = smem + warp * C::RING;
  const uint32_t ring_u = smem_u32(ring);
  float* slot0 = reinterpret_cast<float*>(smem + PD_WARPS * C::RING + warp * C::SLOT);
  if (threadIdx.x < 2 * PD_WARPS) s_info[threadIdx.x].seq = -1;

  pdl_wait();
  pdl_launch_dependents();

  // ---- the line: every thread adds up the tiles of a stretch of sequences
  const long long cap = (long long)a.max_pages * a.page_size;
  auto length = [&](int s) {
    const int n = __ldcg(a.lens + s);
    return n < 0 || n > cap ? 0 : n;
  };
  const int per = (a.n_seqs + PD_THREADS - 1) / PD_THREADS, s0 = min(a.n_seqs, (int)threadIdx.x * per), s1 = min(a.n_seqs, s0 + per);
  long long mine = 0;
  for (int s = s0; s < s1; ++s) {
    const int n = length(s);
    mine += (n + KT - 1) / KT;
    if (n == 0 && part == 0) {  // nothing to attend to: no weight anywhere
      if (__ldcg(a.lens + s) != 0 && hu == 0) atomicOr(a.status, A3_DEV_BAD_POSITION);
      for (int h = h0; h < h0 + hn; ++h) {
        uint4* o = reinterpret_cast<uint4*>(a.out + ((long long)s * a.q_heads + h) * D);
        for (int i = 0; i < D / 8; ++i) o[i] = make_uint4(0, 0, 0, 0);
        if (a.lse) a.lse[(long long)s * a.q_heads + h] = -INFINITY;
      }
    }
  }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long t = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += t;
  }
  if (lane == 31) s_scan[warp] = upto;
  __syncthreads();
  long long total = 0, before = upto - mine;
#pragma unroll
  for (int w = 0; w < PD_WARPS; ++w) {
    if (w < warp) before += s_scan[w];
    total += s_scan[w];
  }
  const long long wanted = (total + PD_WARPS - 1) / PD_WARPS;  // a tile for each warp at least
  const int active = (int)(wanted < a.parts ? wanted : a.parts);
  if (total == 0 && blockIdx.x == 0 && threadIdx.x == 0) a.meta[0].active = 0;
  if (part >= active) return;
  const long long c0 = part_begin(part, total, active), c1 = part_begin(part + 1, total, active);
  auto warp_begin = [&](int w) { return c0 + (c1 - c0) * w / PD_WARPS; };
  if (mine > 0) {
    for (int s = s0; s < s1; ++s) {
      const long long n = (length(s) + KT - 1) / KT;
      for (int w = 0; w < PD_WARPS; ++w) {
        const long long b = warp_begin(w);
        if (b >= before && b < before + n) s_warp_seq[w] = s, s_warp_first[w] = before;
      }
      before += n;
    }
  }
  __syncthreads();

  // ---- this warp's stretch
  const long long w0 = warp_begin(warp), w1 = warp_begin(warp + 1);
  const int count = (int)(w1 - w0);
  if (hu == 0 && threadIdx.x == 0) {
    const int s = s_warp_seq[0];
    a.meta[part] = PartMeta{s_warp_first[0], (length(s) + KT - 1) / KT, total, s, active};
  }
  if (count > 0) {
    const long long kv_off = (long long)kvh * C::ROWB, entry = (long long)a.kv_heads * C::ROWB;
    // where the copies are: sequence, its length, tile in it
    int ls = s_warp_seq[warp], ln = length(ls), lt = (int)(w0 - s_warp_first[warp]);
    // and the computation
    int cs = ls, cn = ln, ct = lt;
    long long cfirst = s_warp_first[warp];
    constexpr int KPL = (KT + 31) / 32;
    int page[KPL], ent[KPL];
    auto look_up = [&] {  // the pages of the next tile, one lane for each key
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        const int key = lt * KT + 32 * i + lane;
        const bool there = 32 * i + lane < KT && key < ln;
        page[i] = -1, ent[i] = -1;
        if (there) {
          const int p = key / a.page_size;
          ent[i] = key - p * a.page_size;
          page[i] = __ldcg(a.table + (long long)ls * a.max_pages + p);
        }
      }
    };
    auto next_tile = [&](int& s, int& n, int& t) {
      if (++t * KT >= n) {
        t = 0;
        do n = length(++s);
        while (n == 0);
      }
    };
    auto issue = [&](int stage) {
      const uint32_t dst = ring_u + stage * PD_STAGE;
      long long off[KPL];
#pragma unroll
      for (int i = 0; i < KPL; ++i) {
        off[i] = -1;
        if (ent[i] >= 0) {
          if (page[i] >= 0 && page[i] < a.n_pages) off[i] = page[i] * a.page_stride + ent[i] * entry + kv_off;
          else atomicOr(a.status, A3_DEV_BAD_POSITION);
        }
      }
      constexpr int RPI = 32 / CH;  // rows a warp copies with one instruction
#pragma unroll
      for (int i = 0; i < KT / RPI; ++i) {
        const int r = i * RPI + lane / CH, c = lane % CH;
        const long long o = __shfl_sync(0xffffffffu, off[i * RPI / 32], r & 31);
        const bool there = o >= 0;  // rows that are not there are filled with zeros: nothing behind a sequence is read
        const long long src = there ? o + c * 16 : 0;
        cp_async16(dst + C::at(r, c), a.k_pages + src, there);
        cp_async16(dst + PD_STAGE / 2 + C::at(r, c), a.v_pages + src, there);
      }
    };

    uint32_t qf[MT][NT][2];
    float o[MT][NT][4], m[NT][2], l[NT][2], cq[NT][2];
    int left_ld = count;
    look_up();
    auto advance = [&](int stage) {  // one more tile under way
      if (left_ld > 0) {
        issue(stage);
        if (--left_ld > 0) {
          next_tile(ls, ln, lt);
          look_up();
        }
      }
      cp_async_commit();
    };
#pragma unroll
    for (int i = 0; i < C::STAGES - 1; ++i) advance(i);
    bool fresh = true;
    int piece0 = ct, n_pieces = 0;
    for (int i = 0; i < count; ++i) {
      advance((i + C::STAGES - 1) % C::STAGES);
      if (fresh) {  // queries of the sequence
        fresh = false;
        piece0 = ct;
        const bf16* q = a.q + cs * a.q_stride;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          const int h = nt * 8 + lane / 4;
          const uint32_t* row = reinterpret_cast<const uint32_t*>(q + (h0 + h) * D);
#pragma unroll
          for (int ks = 0; ks < MT; ++ks) {
#pragma unroll
            for (int e = 0; e < 2; ++e)
              qf[ks][nt][e] = h < hn ? __ldcg(row + 8 * ks + (F8 ? 2 * (lane % 4) + e : lane % 4 + 4 * e)) : 0u;
          }
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
            up *= __int_as_float((127 + ex) << 23) * a.k_scale[kvh];
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
      }
      cp_async_wait<C::STAGES - 1>();
      __syncwarp();
      const uint32_t kt_u = ring_u + i % C::STAGES * PD_STAGE, vt_u = kt_u + PD_STAGE / 2;

      // ---- S^T = K Q^T
      float s[SUB][NT][4];
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[sub][nt][e] = 0.f;
        const int row = sub * 16 + (lane >> 3 & 1) * 8 + (lane & 7);
        if constexpr (!F8) {
#pragma unroll
          for (int ks = 0; ks < MT; ++ks) {
            uint32_t k[4];
            ldmatrix_x4(kt_u + C::at(row, 2 * ks + (lane >> 4)), k[0], k[1], k[2], k[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mma_bf16(s[sub][nt], k, qf[ks][nt][0], qf[ks][nt][1]);
          }
        } else {
#pragma unroll
          for (int ks = 0; ks < MT; ks += 2) {
            uint32_t r[4];
            ldmatrix_x4(kt_u + C::at(row, ks + (lane >> 4)), r[0], r[1], r[2], r[3]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t k[4] = {e4m3x2_to_f16x2(r[2 * e]), e4m3x2_to_f16x2(r[2 * e + 1]), e4m3x2_to_f16x2(r[2 * e] >> 16),
                                     e4m3x2_to_f16x2(r[2 * e + 1] >> 16)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(s[sub][nt], k, qf[ks + e][nt][0], qf[ks + e][nt][1]);
            }
          }
        }
      }

      // ---- running softmax
      const int left = cn - ct * KT;  // keys from here on
      float top[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
        for (int sub = 0; sub < SUB; ++sub)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float t = s[sub][nt][e] * cq[nt][e & 1];
            if (left < KT && sub * 16 + (e >> 1) * 8 + lane / 4 >= left) t = -INFINITY;
            s[sub][nt][e] = t;
            top[nt][e & 1] = fmaxf(top[nt][e & 1], t);
          }
      }
      bool grew = false;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) top[nt][e] = fmaxf(top[nt][e], __shfl_xor_sync(0xffffffffu, top[nt][e], x));
          grew |= top[nt][e] > m[nt][e];
        }
      if (__any_sync(0xffffffffu, grew)) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float now = fmaxf(m[nt][e], top[nt][e]);
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
              const uint32_t h = pack2(p0, p1);
              const float2 back = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&h));
              hi[sub][nt][e] = movmatrix(h);
              lo[sub][nt][e] = movmatrix(pack2(p0 - back.x, p1 - back.y));
            }
          }
      }

      // ---- O^T += V^T P^T
#pragma unroll
      for (int sub = 0; sub < SUB; ++sub) {
        if constexpr (!F8) {
          const int row = sub * 16 + (lane >> 4) * 8 + (lane & 7);
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            uint32_t v[4];
            ldmatrix_x4_trans(vt_u + C::at(row, 2 * mt + (lane >> 3 & 1)), v[0], v[1], v[2], v[3]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              mma_bf16(o[mt][nt], v, hi[sub][nt][0], hi[sub][nt][1]);
              mma_bf16(o[mt][nt], v, lo[sub][nt][0], lo[sub][nt][1]);
            }
          }
        } else {
          const int row = sub * 16 + (lane >> 3 & 1) * 8 + (lane & 7);
#pragma unroll
          for (int mt = 0; mt < MT; mt += 2) {
            uint32_t r[4];
            ldmatrix_x4_trans(vt_u + C::at(row, mt + (lane >> 4)), r[0], r[1], r[2], r[3]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // a register holds dimensions (2i, 2i+1) of one key, then of the next: rows i and i + 8 of the product are those two
              const uint32_t x = __byte_perm(r[2 * e], 0, 0x3120), y = __byte_perm(r[2 * e + 1], 0, 0x3120);
              const uint32_t v[4] = {e4m3x2_to_f16x2(x), e4m3x2_to_f16x2(x >> 16), e4m3x2_to_f16x2(y), e4m3x2_to_f16x2(y >> 16)};
#pragma unroll
              for (int nt = 0; nt < NT; ++nt) mma_f16(o[mt + e][nt], v, hi[sub][nt][0], hi[sub][nt][1]);
            }
          }
        }
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
        const float vs = F8 ? a.v_scale[kvh] : 1.f;
        if (piece0 == 0 && ct == tiles - 1) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = nt * 8 + 2 * (lane % 4) + e;
              if (h < hn) {
                const float f = l[nt][e] == 0.f ? 0.f : vs / l[nt][e];
                const long long at = (long long)cs * a.q_heads + h0 + h;
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                  const int d = mt * 16 + (F8 ? 2 * (lane / 4) : lane / 4);
                  a.out[at * D + d] = __float2bfloat16(o[mt][nt][e] * f);
                  a.out[at * D + d + (F8 ? 1 : 8)] = __float2bfloat16(o[mt][nt][e + 2] * f);
                }
                if (a.lse && lane / 4 == 0) a.lse[at] = l[nt][e] == 0.f ? -INFINITY : (m[nt][e] + log2f(l[nt][e])) * 0.693147180559945309f;
              }
            }
        } else {
          const int which = n_pieces == 0 ? 0 : 1, info = 2 * warp + which;
          float* dst = which == 0 ? slot0 : reinterpret_cast<float*>(ring);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int h = nt * 8 + 2 * (lane % 4) + e;
#pragma unroll
              for (int mt = 0; mt < MT; ++mt) {
                const int d = mt * 16 + (F8 ? 2 * (lane / 4) : lane / 4);
                dst[C::out_at(h, d)] = o[mt][nt][e] * vs;
                dst[C::out_at(h, d + (F8 ? 1 : 8))] = o[mt][nt][e + 2] * vs;
              }
              if (lane / 4 == 0) s_m[info][h] = m[nt][e], s_l[info][h] = l[nt][e];
            }
          if (lane == 0) s_info[info] = SlotInfo{cfirst, tiles, cs};
        }
        ++n_pieces;
        fresh = true;
        if (ct == tiles - 1) cfirst += tiles;
      }
      if (i + 1 < count) next_tile(cs, cn, ct);
    }
  }
  __syncthreads();

  // ---- what the warps hold of one sequence, merged
  for (int i0 = 0; i0 < 2 * PD_WARPS; ++i0) {
    const SlotInfo info = s_info[i0];
    if (info.seq < 0) continue;
    bool first_of = true;
    for (int i = 0; i < i0; ++i) first_of = first_of && s_info[i].seq != info.seq;
    if (!first_of) continue;
    const bool began = info.first < c0, goes_on = info.first + info.tiles > c1;
    const long long slot = ((long long)part * units + hu) * 2 + (began ? 0 : 1);
    for (int x = threadIdx.x; x < hn * (D / 2); x += PD_THREADS) {
      const int h = x / (D / 2), d = x % (D / 2) * 2;
      float mm = -INFINITY;
      for (int i = i0; i < 2 * PD_WARPS; ++i)
        if (s_info[i].seq == info.seq) mm = fmaxf(mm, s_m[i][h]);
      const float ref = mm == -INFINITY ? 0.f : mm;
      float ll = 0.f, ox = 0.f, oy = 0.f;
      for (int i = i0; i < 2 * PD_WARPS; ++i)
        if (s_info[i].seq == info.seq) {
          const float f = ex2(s_m[i][h] - ref);
          const float* src = reinterpret_cast<const float*>(i & 1 ? smem + i / 2 * C::RING : smem + PD_WARPS * C::RING + i / 2 * C::SLOT) + C::out_at(h, d);
          ll += f * s_l[i][h];
          ox += f * src[0];
          oy += f * src[1];
        }
      if (!began && !goes_on) {
        const float f = ll == 0.f ? 0.f : 1.f / ll;
        const long long at = (long long)info.seq * a.q_heads + h0 + h;
        *reinterpret_cast<uint32_t*>(a.out + at * D + d) = pack2(ox * f, oy * f);
        if (a.lse && d == 0) a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.693147180559945309f;
      } else {
        *reinterpret_cast<float2*>(a.part_o + (slot * a.unit + h) * D + d) = make_float2(ox, oy);
        if (d == 0) a.part_ml[slot * a.unit + h] = make_float2(mm, ll);
      }
    }
  }
}

// Block (p, unit, head): the sequence that part p begins with, if it began in the part before, from all parts that hold some of it.
template <int D>
__global__ void __launch_bounds__(D / 2)
paged_join_kernel(const PagedAttnArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  const int p = blockIdx.x + 1, hu = blockIdx.y, g = blockIdx.z, units = a.kv_heads * a.groups;
  const int kvh = hu / a.groups, h0 = kvh * a.group + hu % a.groups * a.unit, hn = min(a.unit, (kvh + 1) * a.group - h0);
  if (g >= hn) return;
  const int active = __ldcg(&a.meta[0].active);
  if (p >= active) return;
  const long long total = __ldcg(&a.meta[p].total), first = __ldcg(&a.meta[p].first), tiles = __ldcg(&a.meta[p].tiles);
  if (first >= part_begin(p, total, active)) return;
  const int from = (int)part_of(first, total, active), to = (int)part_of(first + tiles - 1, total, active);
  if (from != p - 1) return;
  const int d = threadIdx.x * 2;
  float mm = -INFINITY, ll = 0.f, ox = 0.f, oy = 0.f;
  for (int i = from; i <= to; ++i) {
    const long long slot = ((long long)i * units + hu) * 2 + (i == from ? 1 : 0);
    const float2 ml = __ldcg(a.part_ml + slot * a.unit + g);
    const float2 v = __ldcg(reinterpret_cast<const float2*>(a.part_o + (slot * a.unit + g) * D + d));
    const float now = fmaxf(mm, ml.x), ref = now == -INFINITY ? 0.f : now;
    const float f = ex2(mm - ref), e = ex2(ml.x - ref);
    mm = now;
    ll = ll * f + ml.y * e;
    ox = ox * f + v.x * e;
    oy = oy * f + v.y * e;
  }
  const float f = ll == 0.f ? 0.f : 1.f / ll;
  const long long at = (long long)__ldcg(&a.meta[p].seq) * a.q_heads + h0 + g;
  *reinterpret_cast<uint32_t*>(a.out + at * D + d) = pack2(ox * f, oy * f);
  if (a.lse && d == 0) a.lse[at] = ll == 0.f ? -INFINITY : (mm + log2f(ll)) * 0.693147180559945309f;
}

struct PagedPlan {
  int unit, groups, parts;
  size_t meta, ml, bytes;
};
static PagedPlan paged_plan(const a3_handle* h) {
  PagedPlan p;
  const int group = h->m.n_q_heads / h->m.n_kv_heads;
  p.unit = group <= 8 ? group : 16;  // query heads that one pass over the keys serves
  p.groups = cdiv(group, p.unit);
  const int units = h->m.n_kv_heads * p.groups;
  p.parts = h->sm_count * PD_CTAS / units;
  if (p.parts < 1) p.parts = 1;
  const size_t slots = (size_t)p.parts * units * 2 * p.unit;
  p.meta = align_up(sizeof(PartMeta) * p.parts, 256);
  p.ml = align_up(slots * sizeof(float2), 256);
  p.bytes = p.meta + p.ml + slots * h->m.head_dim * 4;
  return p;
}

template <int D, bool F8, int NT>
static int paged_launch(const a3_handle* h, const PagedAttnArgs& a, int units, cudaStream_t st) {
  static SmemAttrOnce once;
  using C = PagedCfg<D, F8, NT>;
  A3_TRY(smem_attr_once(once, h->device, paged_attention_kernel<D, F8, NT>, C::SMEM));
  A3_CUDA(launch_pdl(paged_attention_kernel<D, F8, NT>, dim3(a.parts * units), dim3(PD_THREADS), C::SMEM, st, a));
  A3_LAUNCHED();
  if (a.parts == 1) return A3_OK;  // every sequence ends in the part that it begins in
  A3_CUDA(launch_pdl(paged_join_kernel<D>, dim3(a.parts - 1, units, a.unit), dim3(D / 2), 0, st, a));
  return launched();
}

}  // namespace a3

using namespace a3;

extern "C" size_t a3_paged_attention_workspace_bytes(const a3_handle* h) { return h ? paged_plan(h).bytes : 0; }

extern "C" int a3_paged_attention(const a3_handle* h, const a3_paged_cache* cache, const int32_t* page_table, int n_seqs, int max_pages,
                                  const int32_t* cache_len, const void* q_rows, size_t q_stride, float scale, void* out, float* lse_out,
                                  void* ws, size_t ws_bytes, a3_stream stream) {
  if (!h || !cache || n_seqs < 0 || max_pages < 0 || !isfinite(scale)) return A3_EINVAL;
  A3_TRY(paged_cache_check(h, cache));
  if (n_seqs == 0) return A3_OK;
  if ((!page_table && max_pages > 0) || !cache_len || !q_rows || !out || !ws) return A3_EINVAL;
  if (((uintptr_t)q_rows | (uintptr_t)out) & 15 || (uintptr_t)ws & 255) return A3_EINVAL;
  const a3_model_desc& m = h->m;
  if (q_stride < (size_t)m.n_q_heads * m.head_dim || q_stride % 8 || q_stride > (size_t)1 << 40) return A3_EINVAL;
  const PagedPlan plan = paged_plan(h);
  if (ws_bytes < plan.bytes) return A3_EWORKSPACE;
  PagedAttnArgs a{};
  a.k_pages = (const char*)cache->k_pages, a.v_pages = (const char*)cache->v_pages;
  a.page_stride = (long long)cache->page_stride, a.n_pages = cache->n_pages, a.page_size = cache->page_size;
  a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
  a.table = page_table, a.lens = cache_len, a.n_seqs = n_seqs, a.max_pages = max_pages;
  a.q = (const bf16*)q_rows, a.q_stride = (long long)q_stride;
  a.scale_log2 = scale * 1.44269504088896341f;
  a.out = (bf16*)out, a.lse = lse_out;
  a.q_heads = m.n_q_heads, a.kv_heads = m.n_kv_heads, a.group = m.n_q_heads / m.n_kv_heads;
  a.unit = plan.unit, a.groups = plan.groups, a.parts = plan.parts;
  a.meta = (PartMeta*)ws;
  a.part_ml = (float2*)((char*)ws + plan.meta);
  a.part_o = (float*)((char*)ws + plan.meta + plan.ml);
  a.status = h->dev_status;
  cudaStream_t st = (cudaStream_t)stream;
  const int units = m.n_kv_heads * plan.groups;
  ProfScope prof(h, A3_K_ATTENTION, st);
  const bool f8 = cache->type == A3_CACHE_E4M3;
  auto heads = [&](auto d, auto nt) {
    constexpr int DD = decltype(d)::value, N = decltype(nt)::value;
    return f8 ? paged_launch<DD, true, N>(h, a, units, st) : paged_launch<DD, false, N>(h, a, units, st);
  };
  using One = std::integral_constant<int, 1>;
  using Two = std::integral_constant<int, 2>;
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (m.head_dim == 64) return plan.unit <= 8 ? heads(D64{}, One{}) : heads(D64{}, Two{});
  return plan.unit <= 8 ? heads(D128{}, One{}) : heads(D128{}, Two{});
}
