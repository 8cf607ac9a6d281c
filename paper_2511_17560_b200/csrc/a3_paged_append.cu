// Rows into a paged cache (a3_paged_append): keys rotated to their positions, values as they are, queries rotated beside them.
//
// A row is cut into units of 16 elements of one head: the two 16-byte vectors at 8j and 8j + D/2, which with pairs (i, i + D/2) rotate
// among themselves and with pairs (2i, 2i+1) each within itself.  One thread moves the units j of `HEADS` heads of a row, which share
// the cosines and sines: its loads do not depend on where the row goes, so they are on their way while the page is looked up.
//
// Bound by HBM where rows are many, by latency where they are few.  Measured on heads of 128: 17 871 rows of 28 heads over 4, bf16, 342 MB, in
// 57.5 us, 5.9 TB/s; 32 768 rows of 8 KV heads into 8 bits, 202 MB, in 39.5 us, 5.1 TB/s (rotation and conversion issue for half of
// the time); 256 rows of a batch 2.4 us, one row 1.7 us.
#include <cuda_fp8.h>

#include "a3_internal.cuh"
#include "a3_paged.cuh"

namespace a3 {

constexpr int PA_THREADS = 128;
// CTAs per SM: 96 registers hold the four heads and their cosines.  The rows in 8 bits above 39.5 us with 5, 44 with 4 or 6; those in bf16 57.5, 58.7
// and 61.7.  Two heads for each thread and 7 CTAs 44.5 and 60.7.
constexpr int PA_MIN = 5;
constexpr int PA_HEADS = 4;  // of a thread where rows are many
// Units per SM up to which a thread moves one head, three CTAs: 128 rows of 32 heads over 8, bf16 (332 units per SM), 2.42 us with one
// head and 2.52 with four, 160 rows (415) 2.95 and 2.61, 2 048 rows 16.3 and 10.7.
constexpr int PA_ONE = 3 * PA_THREADS;

struct AppendArgs {
  char *k_pages, *v_pages;
  long long page_stride;  // bytes
  int n_pages, page_size;
  const float *k_scale, *v_scale;
  const int32_t *table, *row_seq, *row_slot, *row_pos;
  int n_seqs, max_pages;
  const bf16 *q, *k, *v;
  long long q_stride, k_stride, v_stride, q_out_stride;  // elements
  bf16* q_out;
  int M, q_heads, kv_heads;  // q_heads 0: no queries
  const float2* tab;
  int max_pos;
  bool rotate;
  uint32_t* status;
};

// One rounding to 8 bits, from the rotated fp32 value by the reciprocal of the scale (2^-23 off the quotient at most: a true division of every
// element would take more instructions than all else); beyond the largest value: the largest value.
__device__ __forceinline__ uint2 pack8_e4m3(const float* f, float by) {
  uint32_t h[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) h[i] = __nv_cvt_float2_to_fp8x2(make_float2(f[2 * i] * by, f[2 * i + 1] * by), __NV_SATFINITE, __NV_E4M3);
  return make_uint2(h[0] | h[1] << 16, h[2] | h[3] << 16);
}

template <int D, int LAYOUT, bool F8, int HEADS>
__global__ void __launch_bounds__(PA_THREADS, PA_MIN)
paged_append_kernel(const AppendArgs a) {
  pdl_wait();
  pdl_launch_dependents();
  constexpr int UPH = D / 16;  // units per head
  const int heads = a.q_heads + 2 * a.kv_heads, stride = (heads + HEADS - 1) / HEADS;  // of the thread's heads
  const unsigned upr = (unsigned)stride * UPH, threads = gridDim.x * PA_THREADS;       // a thread's items are `threads` apart
  const unsigned step_r = threads / upr, step_u = threads - step_r * upr;
  unsigned r = (blockIdx.x * PA_THREADS + threadIdx.x) / upr, u = blockIdx.x * PA_THREADS + threadIdx.x - r * upr;
  if (r >= (unsigned)a.M) return;
  // Where a row goes is looked up while the row before it is moved: the chain from its slot over the page to the store is as long as two
  // loads of the row itself.  A launch before this one may have written the indices: past L1.
  int seq, slot, pos, page;
  auto read_row = [&](unsigned row) {
    seq = __ldcg(a.row_seq + row), slot = __ldcg(a.row_slot + row);
    pos = a.row_pos ? __ldcg(a.row_pos + row) : slot;
  };
  unsigned turn, entry;
  auto look_up = [&] {  // page: -2 for padding, -1 where the row leads nowhere
    turn = !a.rotate ? 0u : pos < 0 ? 0u - (unsigned)pos : (unsigned)pos;
    const unsigned nth = (unsigned)slot / (unsigned)a.page_size;
    entry = (unsigned)slot - nth * a.page_size;
    const bool good = seq >= 0 && seq < a.n_seqs && slot >= 0 && nth < (unsigned)a.max_pages && turn < (unsigned)a.max_pos;
    page = good ? __ldcg(a.table + (long long)seq * a.max_pages + nth) : seq < 0 ? -2 : -1;
  };
  read_row(r);
  look_up();
  for (;;) {
    const int j = u % UPH, h0 = u / UPH;
    const bf16 *q = a.q + r * a.q_stride + 8 * j, *k = a.k + r * a.k_stride + 8 * j - a.q_heads * D;
    const bf16* v = a.v + r * a.v_stride + 8 * j - (a.q_heads + a.kv_heads) * D;
    uint4 x[HEADS][2];
    float scale[HEADS];
#pragma unroll
    for (int i = 0; i < HEADS; ++i) {
      const int h = h0 + i * stride;
      if (h < heads) {
        const bf16* src = (h < a.q_heads ? q : h < a.q_heads + a.kv_heads ? k : v) + h * D;
        x[i][0] = __ldcs(reinterpret_cast<const uint4*>(src));
        x[i][1] = __ldcs(reinterpret_cast<const uint4*>(src + D / 2));
        if (F8 && h >= a.q_heads) scale[i] = __ldca(h < a.q_heads + a.kv_heads ? a.k_scale + (h - a.q_heads) : a.v_scale + (h - a.q_heads - a.kv_heads));
      }
    }
    const bool turned = a.rotate && pos < 0, live = page != -2;
    const int this_page = page, this_entry = entry;
    const unsigned this_r = r, this_u = u;
    // (cos, sin) of two frequencies each: 8j.. for pairs (i, i + D/2); 4j.. and 4j + D/4.. for pairs (2i, 2i+1)
    float4 cs[4];
    if (a.rotate && turn < (unsigned)a.max_pos) {
      const float4* tr = reinterpret_cast<const float4*>(a.tab + (size_t)turn * (D / 2));
#pragma unroll
      for (int e = 0; e < 4; ++e) cs[e] = __ldg(tr + (LAYOUT == 0 ? 4 * j + e : 2 * j + e % 2 + e / 2 * (D / 8)));
    }
    r += step_r;
    if ((u += step_u) >= upr) u -= upr, ++r;
    const bool more = r < (unsigned)a.M;
    if (more) read_row(r);
    if (live && (this_page < 0 || this_page >= a.n_pages)) {
      if (this_u == 0) atomicOr(a.status, A3_DEV_BAD_POSITION);
    } else if (live) {
      const long long place = this_page * a.page_stride + (long long)this_entry * a.kv_heads * (D * (F8 ? 1 : 2)) + 8 * j * (F8 ? 1 : 2);
      if (turned) {
#pragma unroll
        for (int e = 0; e < 4; ++e) cs[e].y = -cs[e].y, cs[e].w = -cs[e].w;
      }
#pragma unroll
      for (int i = 0; i < HEADS; ++i) {
        const int h = h0 + i * stride;
        if (h >= heads) break;
        const bool is_v = h >= a.q_heads + a.kv_heads;
        float f[16];
        unpack8(x[i][0], f);
        unpack8(x[i][1], f + 8);
        if (!is_v && a.rotate) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int p = LAYOUT == 0 ? 2 * e : 4 * e, step = LAYOUT == 0 ? 1 : 2, mate = LAYOUT == 0 ? 8 : 1;
            const float a0 = f[p], b0 = f[p + mate], a1 = f[p + step], b1 = f[p + step + mate];
            f[p] = a0 * cs[e].x - b0 * cs[e].y;
            f[p + mate] = a0 * cs[e].y + b0 * cs[e].x;
            f[p + step] = a1 * cs[e].z - b1 * cs[e].w;
            f[p + step + mate] = a1 * cs[e].w + b1 * cs[e].z;
          }
        }
        if (h < a.q_heads) {
          bf16* dst = a.q_out + this_r * a.q_out_stride + h * D + 8 * j;
          *reinterpret_cast<uint4*>(dst) = pack8(f);
          *reinterpret_cast<uint4*>(dst + D / 2) = pack8(f + 8);
          continue;
        }
        const int kh = h - a.q_heads - (is_v ? a.kv_heads : 0);
        char* dst = (is_v ? a.v_pages : a.k_pages) + place + kh * (D * (F8 ? 1 : 2));
        if (F8) {
          const float by = __frcp_rn(scale[i]);
          *reinterpret_cast<uint2*>(dst) = pack8_e4m3(f, by);
          *reinterpret_cast<uint2*>(dst + D / 2) = pack8_e4m3(f + 8, by);
        } else {
          *reinterpret_cast<uint4*>(dst) = pack8(f);
          *reinterpret_cast<uint4*>(dst + D) = pack8(f + 8);
        }
      }
    }
    if (!more) return;
    look_up();
  }
}

int paged_cache_check(const a3_handle* h, const a3_paged_cache* c) {
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != h->device) return A3_EINVAL;
  if (!c->k_pages || !c->v_pages || c->n_pages <= 0 || c->page_size <= 0) return A3_EINVAL;
  if (c->type != A3_CACHE_BF16 && c->type != A3_CACHE_E4M3) return A3_EUNSUPPORTED;
  if (c->type == A3_CACHE_E4M3 && (!c->k_scale || !c->v_scale)) return A3_EINVAL;
  if (((uintptr_t)c->k_pages | (uintptr_t)c->v_pages | c->page_stride) & 15) return A3_EINVAL;
  const unsigned long long entry = (unsigned long long)h->m.n_kv_heads * h->m.head_dim * (c->type == A3_CACHE_BF16 ? 2 : 1);
  if (c->page_stride < entry * c->page_size || c->page_stride > (1ull << 62) / (unsigned)c->n_pages) return A3_EINVAL;
  return A3_OK;
}

}  // namespace a3

using namespace a3;

extern "C" int a3_paged_append(const a3_handle* h, const a3_paged_cache* cache, const a3_paged_rows* rows, a3_stream stream) {
  if (!h || !cache || !rows) return A3_EINVAL;
  const a3_paged_rows& p = *rows;
  if (p.M < 0 || p.n_seqs < 0 || p.max_pages < 0) return A3_EINVAL;
  A3_TRY(paged_cache_check(h, cache));
  if (p.M == 0) return A3_OK;
  if (!p.page_table || !p.row_seq || !p.row_slot || !p.k_rows || !p.v_rows || !p.q_rows != !p.q_out) return A3_EINVAL;
  if (((uintptr_t)p.q_rows | (uintptr_t)p.k_rows | (uintptr_t)p.v_rows | (uintptr_t)p.q_out) & 15) return A3_EINVAL;
  const a3_model_desc& m = h->m;
  const uint64_t qd = (uint64_t)m.n_q_heads * m.head_dim, kvd = (uint64_t)m.n_kv_heads * m.head_dim;
  if (p.k_stride < kvd || p.v_stride < kvd || (p.q_rows && (p.q_stride < qd || p.q_out_stride < qd))) return A3_EINVAL;
  if ((p.k_stride | p.v_stride | (p.q_rows ? p.q_stride | p.q_out_stride : 0)) % 8) return A3_EINVAL;
  const uint64_t most = (uint64_t)1 << 31;  // elements between rows: offsets stay inside 63 bits
  if (p.k_stride > most || p.v_stride > most || (p.q_rows && (p.q_stride > most || p.q_out_stride > most))) return A3_EINVAL;
  AppendArgs a{};
  a.k_pages = (char*)cache->k_pages, a.v_pages = (char*)cache->v_pages;
  a.page_stride = (long long)cache->page_stride, a.n_pages = cache->n_pages, a.page_size = cache->page_size;
  a.k_scale = cache->k_scale, a.v_scale = cache->v_scale;
  a.table = p.page_table, a.row_seq = p.row_seq, a.row_slot = p.row_slot, a.row_pos = p.row_pos;
  a.n_seqs = p.n_seqs, a.max_pages = p.max_pages;
  a.q = (const bf16*)p.q_rows, a.k = (const bf16*)p.k_rows, a.v = (const bf16*)p.v_rows;
  a.q_stride = (long long)p.q_stride, a.k_stride = (long long)p.k_stride, a.v_stride = (long long)p.v_stride, a.q_out_stride = (long long)p.q_out_stride;
  a.q_out = (bf16*)p.q_out;
  a.M = p.M, a.q_heads = p.q_rows ? m.n_q_heads : 0, a.kv_heads = m.n_kv_heads;
  a.tab = h->rope_tab, a.max_pos = m.max_positions, a.rotate = p.rotate != 0, a.status = h->dev_status;
  // one head for each thread while rows are few, then four
  const int all = a.q_heads + 2 * a.kv_heads, uph = m.head_dim / 16;
  const bool many = (unsigned long long)p.M * all * uph > (unsigned long long)h->sm_count * PA_ONE;
  const int heads = many ? PA_HEADS : 1;
  const unsigned long long need = ((unsigned long long)p.M * cdiv(all, heads) * uph + PA_THREADS - 1) / PA_THREADS;
  const unsigned blocks = (unsigned)(need < (unsigned long long)h->sm_count * PA_MIN ? need : (unsigned long long)h->sm_count * PA_MIN);
  cudaStream_t st = (cudaStream_t)stream;
  ProfScope prof(h, A3_K_PAGED_APPEND, st);
  const bool f8 = cache->type == A3_CACHE_E4M3;
  auto go = [&](auto one, auto four) { return launch_pdl(many ? four : one, dim3(blocks), dim3(PA_THREADS), 0, st, a); };
  auto pick = [&](auto d, auto layout) {
    constexpr int DD = decltype(d)::value, L = decltype(layout)::value;
    if (f8) return go(paged_append_kernel<DD, L, true, 1>, paged_append_kernel<DD, L, true, PA_HEADS>);
    return go(paged_append_kernel<DD, L, false, 1>, paged_append_kernel<DD, L, false, PA_HEADS>);
  };
  auto shape = [&](auto d) { return m.rope_layout == 0 ? pick(d, std::integral_constant<int, 0>{}) : pick(d, std::integral_constant<int, 1>{}); };
  A3_CUDA(m.head_dim == 64 ? shape(std::integral_constant<int, 64>{}) : shape(std::integral_constant<int, 128>{}));
  return launched();
}
