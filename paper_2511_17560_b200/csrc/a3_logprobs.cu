// Log probabilities of given tokens, entropy and the best alternatives (a3_token_logprobs), from rows of logits.
//
//   M = max x,  s = sum exp(x - M),  w = sum exp(x - M) (x - M)
//   logprob = x_t - M - log s,   entropy = log s - w / s
//
// The logits are read once: bound by HBM where rows are many, by latency where they are few.  A row belongs to one CTA or, where rows
// are fewer than the device holds, to a cluster whose CTAs join their parts through distributed shared memory.  Each thread keeps the
// running (M, s, w) of its own elements.  From the warps' sums on, s is carried without the 1 of one largest element, and ends in log1p: where one
// token has nearly all of the probability, what it lacks of 1 and the entropy come from the other tokens alone.  The thread that holds it has
// added its other elements to that 1; in such a row, and in no other, they are added up once more without it.
//
// The alternatives come from the same pass: the n-th largest of the threads' maxima (of the 32 that are left when each warp gives its largest), exactly, is
// a bound that at least n elements reach, and only the threads whose own maximum reaches it - little more than n of them - are gone
// through again, in the ring where that still holds the row, else from L2, a warp together on one thread's elements.  What reaches the
// bound, usually 1-2 n elements, is ranked by counting.
//
// Measured, bf16: 2 048 rows of 128 256, 525 MB, one alternative each, 87 us while the clock holds (6.0 TB/s) and 102-105 us repeated without a pause,
// when the power limit lowers it to 1.6 GHz: an exponential and some seven other instructions for each element fill the SM as the way from HBM does; with 20
// alternatives 129 us, the search and the ranking of a row with no load under way.  65 rows of 152 064 with 20 alternatives each 12.4 us, one row of
// 128 256 in fp32 7.2 us: latency, the ranking after the pass among it.  With a nearly certain token in every row 13.0, 7.6 and 89 us.
#include <cuda_fp16.h>

#include "a3_internal.cuh"

namespace a3 {

constexpr int LP_U = 4, LP_CAP = 512, LP_PARTS = 8, LP_TOP = A3_LOGPROBS_MAX_TOP;
constexpr int LP_STAGES = 3;  // batches of LP_U vectors that a thread's ring holds
// A CTA of so many threads, which has a row alone or as one of PARTS at most.
template <int THREADS, int PARTS>
struct LpCfg {
  static constexpr int WARPS = THREADS / 32, BATCH = THREADS * LP_U, RING = LP_STAGES * BATCH * 16, MIN = 1024 / THREADS;
  static constexpr int KEPT = 32 / WARPS;  // largest maxima of a warp's lanes that the bound is taken from: 32 in all
};
static_assert(LP_TOP <= 32, "the bound is the n-th largest of them");
constexpr float LOG2E = 1.44269504088896341f;
// Where the other elements of the warp that has the largest one come to an eighth of it or more, an addition to a sum that holds its 1 is off by
// 9 x 2^-24 of theirs at most; below, the largest one's thread adds its elements up once more.
constexpr float LP_CERTAIN = 0.125f;
constexpr float LP_FAR = -200.f;  // exp of it is 0 in fp32, and unlike that of -inf or of the lowest value its product with that 0 is 0 too

struct LogprobArgs {
  const void* logits;
  long long row_stride;
  int M, vocab;
  const int32_t* targets;
  int n_top;
  float *logprob, *entropy;
  int32_t* top_ids;
  float* top_logprobs;
  uint32_t* status;
};

// Pairs of fp32 in one 64-bit register: additions and products of two at once.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pack_f2(float x, float y) {
  f32x2 z;
  asm("mov.b64 %0, {%1, %2};" : "=l"(z) : "f"(x), "f"(y));
  return z;
}
__device__ __forceinline__ float2 unpack_f2(f32x2 z) {
  float2 v;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(v.x), "=f"(v.y) : "l"(z));
  return v;
}
__device__ __forceinline__ f32x2 add_f2(f32x2 a, f32x2 b) {
  f32x2 z;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(a), "l"(b));
  return z;
}
__device__ __forceinline__ f32x2 mul_f2(f32x2 a, f32x2 b) {
  f32x2 z;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(z) : "l"(a), "l"(b));
  return z;
}
__device__ __forceinline__ f32x2 fma_f2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 z;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(z) : "l"(a), "l"(b), "l"(c));
  return z;
}

// VE values of a 16-byte vector, W words of it that hold them: the largest number of vectors, word by word (`max_of`, then `largest`), and the
// values of a word as pairs, those of -inf as the type's lowest number (NaN stays); next to a maximum above ORDINARY that number's exponential is 0.
template <typename T>
struct Logit;
template <>
struct Logit<float> {
  static constexpr int VE = 4;
  static constexpr float LOWEST = -3.40282347e38f, ORDINARY = LOWEST;
  static constexpr uint32_t NONE = 0xff800000u;
  static constexpr int LAST_BIT = 0;
  __device__ static uint4 max_of(uint4 a, uint4 b) { return make_uint4(two(a.x, b.x), two(a.y, b.y), two(a.z, b.z), two(a.w, b.w)); }
  __device__ static uint32_t two(uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }
  __device__ static float largest(uint4 v) { return __uint_as_float(two(two(v.x, v.y), two(v.z, v.w))); }
  __device__ static void pairs(const uint4& v, f32x2* p) { p[0] = pack_f2(finite(v.x), finite(v.y)), p[1] = pack_f2(finite(v.z), finite(v.w)); }
  __device__ static float finite(uint32_t x) {
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(__uint_as_float(x)), "f"(LOWEST));
    return y;
  }
  __device__ static void unpack(const uint4& v, float* f) {
    f[0] = __uint_as_float(v.x), f[1] = __uint_as_float(v.y), f[2] = __uint_as_float(v.z), f[3] = __uint_as_float(v.w);
  }
  __device__ static float one(const float* p) { return *p; }
};
template <>
struct Logit<bf16> {
  static constexpr int VE = 8;
  static constexpr float LOWEST = -3.38953139e38f, ORDINARY = LOWEST;
  static constexpr uint32_t NONE = 0xff80ff80u;  // a word of -inf
  static constexpr int LAST_BIT = 16;            // of a value's bits in fp32
  __device__ static uint4 max_of(uint4 a, uint4 b) { return make_uint4(two(a.x, b.x), two(a.y, b.y), two(a.z, b.z), two(a.w, b.w)); }
  __device__ static uint32_t two(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
  }
  __device__ static float largest(uint4 v) {
    const uint32_t x = two(two(v.x, v.y), two(v.z, v.w));
    return fmaxf(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
  __device__ static f32x2 pair(uint32_t x) {
    asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(x) : "r"(0xff7fff7fu));
    return pack_f2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
  __device__ static void pairs(const uint4& v, f32x2* p) { p[0] = pair(v.x), p[1] = pair(v.y), p[2] = pair(v.z), p[3] = pair(v.w); }
  __device__ static void unpack(const uint4& v, float* f) { unpack8(v, f); }
  __device__ static float one(const bf16* p) { return __bfloat162float(*p); }
};
template <>
struct Logit<__half> {
  static constexpr int VE = 8;
  static constexpr float LOWEST = -65504.f, ORDINARY = LOWEST - LP_FAR;
  static constexpr uint32_t NONE = 0xfc00fc00u;
  static constexpr int LAST_BIT = 13;
  __device__ static uint4 max_of(uint4 a, uint4 b) { return make_uint4(two(a.x, b.x), two(a.y, b.y), two(a.z, b.z), two(a.w, b.w)); }
  __device__ static uint32_t two(uint32_t a, uint32_t b) {
    uint32_t y;
    asm("max.f16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
    return y;
  }
  __device__ static float2 floats(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
  __device__ static float largest(uint4 v) {
    const float2 t = floats(two(two(v.x, v.y), two(v.z, v.w)));
    return fmaxf(t.x, t.y);
  }
  __device__ static f32x2 pair(uint32_t x) {
    asm("max.NaN.f16x2 %0, %0, %1;" : "+r"(x) : "r"(0xfbfffbffu));
    const float2 t = floats(x);
    return pack_f2(t.x, t.y);
  }
  __device__ static void pairs(const uint4& v, f32x2* p) { p[0] = pair(v.x), p[1] = pair(v.y), p[2] = pair(v.z), p[3] = pair(v.w); }
  __device__ static void unpack(const uint4& v, float* f) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 t = floats(w[i]);
      f[2 * i] = t.x, f[2 * i + 1] = t.y;
    }
  }
  __device__ static float one(const __half* p) { return __half2float(*p); }
};

__device__ __forceinline__ float lp_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}
// Whole numbers in the order of the values: NaN 0, -inf LP_NONE; both zeros alike.
constexpr uint32_t LP_NONE = 0x007fffffu;
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x + 0.f);
  return x != x ? 0u : u ^ ((int32_t)u < 0 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k) { return k == 0 ? NAN : __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// larger is better: the value, then the lower id
__device__ __forceinline__ unsigned long long lp_key(uint32_t o, int id) { return (unsigned long long)o << 32 | (0xffffffffu - (uint32_t)id); }
__device__ __forceinline__ int key_id(unsigned long long k) { return (int)(0xffffffffu - (uint32_t)k); }

struct LpStats {
  float m, s, w;  // s without the 1 of one largest element
};
// Clusters: this CTA's place, the barrier in halves (all threads arrive; what was written before is seen behind the wait), and the place of
// a variable of this CTA in the first one of its cluster.
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t x;
  asm("mov.u32 %0, %cluster_nctaid.x;" : "=r"(x));
  return x;
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t x;
  asm("mov.u32 %0, %cluster_ctarank;" : "=r"(x));
  return x;
}
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();  // a warp's lanes arrive, and wait, as one, wherever a loop before has left them
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename V>
__device__ __forceinline__ V* in_first(V* p, int parts) {
  if (parts == 1) return p;
  V* q;
  asm("mapa.u64 %0, %1, %2;" : "=l"(q) : "l"(p), "r"(0));
  return q;
}
__device__ __forceinline__ float warp_max(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}

template <typename T, int THREADS, int PARTS>
__global__ void __launch_bounds__(THREADS, LpCfg<THREADS, PARTS>::MIN)
logprobs_kernel(const LogprobArgs a) {
  using C = LpCfg<THREADS, PARTS>;
  constexpr int WARPS = C::WARPS;
  constexpr int VE = Logit<T>::VE;
  extern __shared__ __align__(16) uint4 ring[];
  __shared__ float s_red[3][WARPS];
  __shared__ __align__(16) uint32_t s_kept[32];
  __shared__ unsigned long long s_cand[LP_CAP], s_best[WARPS];
  __shared__ int s_count, s_n_found;
  __shared__ uint8_t s_found[THREADS];
  // of the row, in its first CTA: every CTA's statistics and best elements (in descending order, 0 where there are fewer), and the row's
  __shared__ LpStats s_stats[PARTS];
  __shared__ unsigned long long s_lists[PARTS][LP_TOP], s_top[LP_TOP];
  const int parts = PARTS == 1 ? 1 : (int)cluster_size(), rank = PARTS == 1 ? 0 : (int)cluster_rank();
  if (parts > 1) cluster_arrive();  // waited for before the first access to another CTA's memory: it has to be there
  // The launch behind is let in as CTAs end, not before: let in when the last rows had been read, it took their places unevenly (calls one after the
  // other, 65 rows of 152 064 17.7 us and 12.6 so, 400 of 128 256 29.1 and 25.4, 858 of 21 870 in fp16 16.1 and 12.4).
  pdl_wait();
  const int row = blockIdx.x / parts, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const T* x = reinterpret_cast<const T*>(a.logits) + row * a.row_stride;
  // 16-byte vectors from the first boundary on, the few elements before and behind them one by one
  const int head = min(a.vocab, (int)((16 - ((uintptr_t)x & 15)) % 16 / sizeof(T)));
  const int n_vec = (a.vocab - head) / VE, tail0 = head + n_vec * VE;
  const int v0 = (int)((long long)n_vec * rank / parts), v1 = (int)((long long)n_vec * (rank + 1) / parts);
  const uint4* xv = reinterpret_cast<const uint4*>(x + head);
  // this thread's single element: of the head in the first CTA, of the tail in the last
  int single = -1;
  if (rank == 0 && tid < head) single = tid;
  if (rank == parts - 1 && tid >= 32 && tid - 32 < a.vocab - tail0) single = tail0 + tid - 32;

  // the given token's logit, on its way from here on
  const int target = rank == 0 && a.targets ? __ldcg(a.targets + row) : -1;
  const float target_logit = tid == 0 && target >= 0 && target < a.vocab ? Logit<T>::one(x + target) : 0.f;

  float m = -INFINITY, s = 0.f, w = 0.f;
  f32x2 s2 = 0, w2 = 0;  // the vectors' share of s and w, two sums each
  auto raise = [&](float most) {
    if (most > m) {
      if (m > -INFINITY) {
        const float d = fmaxf(m - most, LP_FAR), g = lp_ex2(d * LOG2E);
        w = g * (w + s * d);
        s *= g;
        const f32x2 gg = pack_f2(g, g);
        w2 = mul_f2(gg, fma_f2(s2, pack_f2(d, d), w2));
        s2 = mul_f2(gg, s2);
      }
      m = most;
    }
  };
  auto add = [&](const float* f, int n) {  // any values
    if (m > -INFINITY) {
#pragma unroll
      for (int i = 0; i < n; ++i) {
        const float d = max_nan(f[i] - m, LP_FAR), e = lp_ex2(d * LOG2E);  // NaN goes into s
        s += e;
        w += e * d;
      }
    } else {
#pragma unroll
      for (int i = 0; i < n; ++i)
        if (f[i] != f[i]) s = NAN;
    }
  };
  // LP_U vectors at once (at, at + THREADS, ...; from the n-th on -inf): one look at whether the maximum rises.  With a maximum in the
  // ordinary range -inf may stand as the type's lowest number: its exponential is 0 and the product of the two is.  Others take the slow way.
  auto take = [&](const uint4* at, int n) {
    uint4 raw[LP_U];
#pragma unroll
    for (int u = 0; u < LP_U; ++u) raw[u] = at[u * THREADS];
    if (n < LP_U) {
#pragma unroll
      for (int u = 0; u < LP_U; ++u)
        if (u >= n) raw[u] = make_uint4(Logit<T>::NONE, Logit<T>::NONE, Logit<T>::NONE, Logit<T>::NONE);
    }
    uint4 top = raw[0];
#pragma unroll
    for (int u = 1; u < LP_U; ++u) top = Logit<T>::max_of(top, raw[u]);
    raise(Logit<T>::largest(top));
    if (m > Logit<T>::ORDINARY && m < 1e30f) {
      const f32x2 ref = pack_f2(-m, -m), log2e = pack_f2(LOG2E, LOG2E);
#pragma unroll
      for (int u = 0; u < LP_U; ++u) {
        f32x2 p[VE / 2];
        Logit<T>::pairs(raw[u], p);
#pragma unroll
        for (int i = 0; i < VE / 2; ++i) {
          const f32x2 d = add_f2(p[i], ref);
          const float2 t = unpack_f2(mul_f2(d, log2e));
          const f32x2 e = pack_f2(lp_ex2(t.x), lp_ex2(t.y));
          s2 = add_f2(s2, e);
          w2 = fma_f2(e, d, w2);
        }
      }
    } else {
#pragma unroll 1
      for (int u = 0; u < n; ++u) {
        float f[VE];
        Logit<T>::unpack(at[u * THREADS], f);
        add(f, VE);
      }
    }
  };
  {
    // Each thread's vectors come through a ring of its own in shared memory, LP_STAGES - 1 batches under way while one is computed: what the
    // registers of all threads hold is too little to cover the way from HBM.
    constexpr int BATCH = C::BATCH;
    const uint32_t ring_u = smem_u32(ring + tid);
    const uint4* from = xv + v0 + tid;
    int to_fetch = v1 - v0, left = v1 - v0;  // vectors of the CTA
    uint32_t put = 0, get = 0;               // batches of the ring, in bytes
    auto turn = [](uint32_t& at) { at = at == (LP_STAGES - 1) * BATCH * 16 ? 0 : at + BATCH * 16; };
    auto fetch = [&] {
      if (to_fetch >= BATCH) {
#pragma unroll
        for (int u = 0; u < LP_U; ++u) cp_async16(ring_u + put + u * THREADS * 16, from + u * THREADS, true);
      } else {
#pragma unroll
        for (int u = 0; u < LP_U; ++u)
          if (tid + u * THREADS < to_fetch) cp_async16(ring_u + put + u * THREADS * 16, from + u * THREADS, true);
      }
      cp_async_commit();
      from += BATCH, to_fetch -= BATCH;
      turn(put);
    };
#pragma unroll 1
    for (int b = 0; b < LP_STAGES - 1; ++b) fetch();
    for (; left > 0; left -= BATCH) {
      fetch();
      cp_async_wait<LP_STAGES - 1>();
      take(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(ring + tid) + get), left >= BATCH ? LP_U : (left - tid + THREADS - 1) / THREADS);
      turn(get);
    }
  }
  {
    const float2 ss = unpack_f2(s2), ww = unpack_f2(w2);
    s += ss.x + ss.y;
    w += ww.x + ww.y;
    s2 = w2 = 0;
  }
  const uint32_t mine = ordered(m);  // of the vectors alone; LP_NONE: nothing above -inf
  if (single >= 0) {
    const float f = Logit<T>::one(x + single);
    raise(f);
    add(&f, 1);
  }

  // ---- the CTA's statistics; its largest elements' bound
  if (tid == 0) s_count = s_n_found = 0;
  const int n = a.n_top;
  {
    const float top = warp_max(m);
    if (lane == 0) s_red[0][warp] = top;
    if (n > 1) {
      uint32_t o = mine;
#pragma unroll
      for (int k = 0; k < C::KEPT; ++k) {
        const uint32_t best = __reduce_max_sync(0xffffffffu, o);
        if (lane == 0) s_kept[warp * C::KEPT + k] = best;
        if (lane == __ffs(__ballot_sync(0xffffffffu, o == best)) - 1) o = 0;
      }
    }
  }
  __syncthreads();
  float most = s_red[0][0];
  int holder = 0;  // the warp of one largest element, which s leaves out
#pragma unroll
  for (int i = 1; i < WARPS; ++i)
    if (s_red[0][i] > most) most = s_red[0][i], holder = i;
  {
    const uint32_t these = __ballot_sync(0xffffffffu, m == most);
    const int who = __ffs(these) - 1;
    const float d = fmaxf(m - most, LP_FAR), g = m > -INFINITY ? lp_ex2(d * LOG2E) : 0.f;
    float ps = warp_sum(g * (warp == holder && lane == who ? s - 1.f : s));
    const float pw = warp_sum(m > -INFINITY ? g * (w + s * d) : 0.f);
    // What the holder's other elements add beside its 1 is lost below 2^-24: where that is much of what all others add, the warp goes through
    // them again and leaves the 1 out.
    if (warp == holder && most > -INFINITY && ps < LP_CERTAIN) {
      const bool kept = v1 - v0 <= LP_STAGES * LP_U * THREADS;  // all of the CTA's vectors are still in the ring
      float others = lane == who ? 0.f : g * s;
      int ones = 0;  // elements that are as large
      auto count = [&](float f) {
        if (f == most)
          ++ones;
        else
          others += lp_ex2(fmaxf(f - most, LP_FAR) * LOG2E);
      };
      for (int v = warp * 32 + who + lane * THREADS; v < v1 - v0; v += 32 * THREADS) {
        float f[VE];
        Logit<T>::unpack(kept ? ring[v] : __ldcg(xv + v0 + v), f);
#pragma unroll
        for (int e = 0; e < VE; ++e) count(f[e]);
      }
      if (lane == who && single >= 0) count(Logit<T>::one(x + single));
      ps = warp_sum(others) + (float)((int)__reduce_add_sync(0xffffffffu, ones) - 1);
    }
    if (lane == 0) s_red[1][warp] = ps, s_red[2][warp] = pw;
  }

  // ---- the CTA's best elements above -inf
  uint32_t bound = 0;
  // one thread's elements, a warp together: `use(value, id)` for each
  auto again = [&](int t, auto use) {
    for (int v = v0 + t + lane * THREADS; v < v1; v += 32 * THREADS) {
      float f[VE];
      Logit<T>::unpack(__ldcg(xv + v), f);
#pragma unroll
      for (int e = 0; e < VE; ++e) use(f[e], head + v * VE + e);
    }
  };
  if (n > 0) {
    // The n-th largest of the threads' maxima that were kept, or of all where not every thread has a vector: n elements reach it.  To the last bit of the
    // type: of logits far from zero, whose spread is a small part of them, nearly all would reach a bound of fewer.  Of one element alone, it is it.
    if (n == 1) {
      bound = ordered(most);
    } else if (v1 - v0 >= THREADS) {
      // an element's place is how many are better: a lane for each of the 32
      const uint32_t kept = s_kept[lane];
      int better = 0;
#pragma unroll
      for (int i = 0; i < 32; i += 4) {
        const uint4 other = *reinterpret_cast<const uint4*>(s_kept + i);
        better += (other.x > kept) + (other.y > kept) + (other.z > kept) + (other.w > kept);
      }
      bound = __reduce_min_sync(0xffffffffu, better < n ? kept : 0xffffffffu);
    } else {
#pragma unroll 1
      for (int bit = 31; bit >= Logit<T>::LAST_BIT; --bit) {
        const uint32_t c = bound | 1u << bit;
        if (__syncthreads_count(mine >= c) >= n) bound = c;
      }
    }
    if (bound <= LP_NONE) bound = LP_NONE + 1;
    const float least = unordered(bound);
    auto offer = [&](float f, int id) {
      if (f >= least) {
        const int at = atomicAdd(&s_count, 1);
        if (at < LP_CAP) s_cand[at] = lp_key(ordered(f), id);
      }
    };
    if (v1 - v0 <= LP_STAGES * LP_U * THREADS) {  // all of the CTA's vectors are still in the ring, each thread's at its hand
      if (mine >= bound) {
#pragma unroll 1
        for (int v = v0 + tid, i = tid; v < v1; v += THREADS, i += THREADS) {
          const uint4 raw = ring[i];
          if (!(Logit<T>::largest(raw) >= least)) continue;
          float f[VE];
          Logit<T>::unpack(raw, f);
#pragma unroll
          for (int e = 0; e < VE; ++e) offer(f[e], head + v * VE + e);
        }
      }
    } else {  // from L2, a warp together on one thread's vectors, four threads at a time
      if (mine >= bound) s_found[atomicAdd(&s_n_found, 1)] = (uint8_t)tid;
      __syncthreads();
      const int found = s_n_found;
      for (int i = warp; i < found; i += 4 * WARPS) {
        for (int k = lane * THREADS; k < v1 - v0; k += 32 * THREADS) {
          uint4 raw[4];
          int v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int at = i + q * WARPS;
            v[q] = at < found ? v0 + k + s_found[at] : v1;
            if (v[q] < v1) raw[q] = __ldcg(xv + v[q]);
          }
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (v[q] < v1 && Logit<T>::largest(raw[q]) >= least) {
              float f[VE];
              Logit<T>::unpack(raw[q], f);
#pragma unroll
              for (int e = 0; e < VE; ++e) offer(f[e], head + v[q] * VE + e);
            }
          }
        }
      }
    }
    if (single >= 0) offer(Logit<T>::one(x + single), single);
  }
  __syncthreads();
  if (parts > 1) cluster_wait();
  if (warp == WARPS - 1) {
    const float ps = warp_sum(lane < WARPS ? s_red[1][lane % WARPS] : 0.f), pw = warp_sum(lane < WARPS ? s_red[2][lane % WARPS] : 0.f);
    if (lane == 0) *in_first(&s_stats[rank], parts) = LpStats{most, ps, pw};
  }
  unsigned long long* list = in_first(s_lists[rank], parts);
  if (n > 0) {
    const int count = s_count;
    if (count <= LP_CAP) {
      for (int i = tid; i < count; i += THREADS) {
        const unsigned long long k = s_cand[i];
        int better = 0;
#pragma unroll 4
        for (int j = 0; j < count; ++j) better += s_cand[j] > k;
        if (better < (n + 3) / 4 * 4) list[better] = k;
      }
      if (tid >= count && tid < (n + 3) / 4 * 4) list[tid] = 0;  // in fours, as they are compared
    } else {
      // More elements at the bound than there is room for (a row of equal values): the best of all, n times, where each time only
      // the thread that had it looks for its next.
      unsigned long long best = 0, last = ~0ull;
      auto next_of = [&](int t) {  // of thread t, below `last`
        unsigned long long k = 0;
        again(t, [&](float f, int id) {
          const uint32_t o = ordered(f);
          const unsigned long long c = o > LP_NONE ? lp_key(o, id) : 0;
          if (c < last && c > k) k = c;
        });
#pragma unroll
        for (int o = 16; o; o >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
        return k;
      };
      for (int t = 0; t < 32; ++t) {
        const unsigned long long k = next_of(warp * 32 + t);
        if (lane == t) best = k;
      }
      unsigned long long extra = 0;
      if (single >= 0) {
        const uint32_t o = ordered(Logit<T>::one(x + single));
        extra = o > LP_NONE ? lp_key(o, single) : 0;
      }
      for (int i = 0; i < n; ++i) {
        unsigned long long k = max(best, extra);
#pragma unroll
        for (int o = 16; o; o >>= 1) k = max(k, __shfl_xor_sync(0xffffffffu, k, o));
        if (lane == 0) s_best[warp] = k;
        __syncthreads();
        for (int j = 0; j < WARPS; ++j) k = max(k, s_best[j]);
        if (tid == 0) {
          list[i] = k;
          if (i == n - 1)
            for (int j = n; j % 4; ++j) list[j] = 0;
        }
        last = k;
        if (extra == k) extra = 0;
        const uint32_t whose = __ballot_sync(0xffffffffu, best == k && k != 0);
        if (whose) {
          const int t = __ffs(whose) - 1;
          const unsigned long long nk = next_of(warp * 32 + t);
          if (lane == t) best = nk;
        }
        __syncthreads();
      }
    }
  }

  // ---- the parts of the row, joined by the first CTA
  if (parts > 1) {
    cluster_arrive();
    cluster_wait();
    if (rank != 0) return;  // nobody reads this CTA's memory
  } else {
    __syncthreads();
  }
  if (warp == 0) {
    const bool have = lane < parts;
    const LpStats o = have ? s_stats[lane % PARTS] : LpStats{-INFINITY, 0.f, 0.f};
    const float top = warp_max(o.m);
    const uint32_t these = __ballot_sync(0xffffffffu, have && o.m == top);
    const float d = fmaxf(o.m - top, LP_FAR), g = o.m > -INFINITY ? lp_ex2(d * LOG2E) : 0.f, full = 1.f + o.s;
    // a CTA with nothing above -inf still says whether it met a NaN
    const float s_all = warp_sum(o.m > -INFINITY ? g * (lane == __ffs(these) - 1 ? o.s : full) : o.s == o.s ? 0.f : o.s);
    const float w_all = warp_sum(o.m > -INFINITY ? g * (o.w + full * d) : 0.f);
    const bool sound = top > -INFINITY && top < INFINITY && s_all == s_all;
    const float log_s = sound ? log1pf(s_all) : NAN;
    if (lane == 0) {
      bool bad_target = false;
      if (a.targets) {
        bad_target = target >= a.vocab;
        a.logprob[row] = target < 0 ? 0.f : bad_target ? NAN : (target_logit - top) - log_s;
      }
      if (a.entropy) a.entropy[row] = sound ? log_s - w_all / (1.f + s_all) : NAN;
      if (!sound || bad_target) atomicOr(a.status, (sound ? 0u : A3_DEV_NONFINITE_SCORE) | (bad_target ? A3_DEV_BAD_POSITION : 0u));
      s_red[0][0] = top;
      s_red[1][0] = log_s;
    }
  }
  if (n == 0) return;
  if (tid < n) s_top[tid] = parts == 1 ? s_lists[0][tid] : 0;
  __syncthreads();
  const float top = s_red[0][0], log_s = s_red[1][0];  // log_s: NaN where there is no distribution
  if (parts > 1) {  // an element's place is how many are better: all of them compared, which needs no branch
    for (int i = tid; i < parts * n; i += THREADS) {
      const unsigned long long k = s_lists[i / n][i % n];
      int better = k == 0 ? n : 0;
#pragma unroll 1
      for (int l = 0; l < parts; ++l)
#pragma unroll 1
        for (int j = 0; j < n; j += 4)
#pragma unroll
          for (int e = 0; e < 4; ++e) better += s_lists[l][j + e] > k;
      if (better < n) s_top[better] = k;
    }
    __syncthreads();
  }
  if (warp == 0) {
    // fewer elements above -inf than asked for: the lowest ids of those at -inf, then of NaNs
    int have = __popc(__ballot_sync(0xffffffffu, lane < n && s_top[lane] != 0));
    for (int pass = 0; pass < 2 && have < n; ++pass) {
      for (int i0 = 0; i0 < a.vocab && have < n; i0 += 32) {
        const int i = i0 + lane;
        const uint32_t o = i < a.vocab ? ordered(Logit<T>::one(x + i)) : 0xffffffffu;
        const uint32_t these = __ballot_sync(0xffffffffu, o == (pass == 0 ? LP_NONE : 0u));
        const int at = have + __popc(these & ((1u << lane) - 1));
        if ((these >> lane & 1) && at < n) s_top[at] = lp_key(o, i);
        have = min(n, have + __popc(these));
        __syncwarp();
      }
    }
    __syncwarp();
    if (lane < n) {
      const unsigned long long k = s_top[lane];
      a.top_ids[(long long)row * n + lane] = key_id(k);
      a.top_logprobs[(long long)row * n + lane] = log_s == log_s ? (unordered((uint32_t)(k >> 32)) - top) - log_s : NAN;
    }
  }
}

template <typename T, int THREADS, int PARTS>
static int logprobs_rows(const a3_handle* h, const LogprobArgs& a, int parts, cudaStream_t st) {
  static SmemAttrOnce once;
  using C = LpCfg<THREADS, PARTS>;
  const dim3 grid((unsigned)(a.M * parts));
  A3_TRY(smem_attr_once(once, h->device, logprobs_kernel<T, THREADS, PARTS>, C::RING));
  A3_CUDA(launch_pdl_cluster(parts, logprobs_kernel<T, THREADS, PARTS>, grid, dim3(THREADS), C::RING, st, a));
  return launched();
}

template <typename T>
static int logprobs_launch(const a3_handle* h, const LogprobArgs& a, cudaStream_t st) {
  // CTAs of a row: up to two for each SM (65 rows of 152 064 in bf16, of which 20 each: 4 CTAs a row 12.4 us, 8 16.5), no fewer than 2 048
  // elements for each.
  int parts = 1;
  while (parts < LP_PARTS && (long long)a.M * parts * 2 <= 2 * h->sm_count && a.vocab / (2 * parts) >= 2048) parts *= 2;
  if (parts > 1) return logprobs_rows<T, 256, LP_PARTS>(h, a, parts, st);
  // Short rows in small CTAs, of which more are at work at once.  With 64, 128 and 256 threads and 5 alternatives: 858 rows of 21 870 in fp16 14.7 us, 14.8
  // and 19.8; 2 500 of 24 000 in bf16 37.9, 33.6 and 42.2, of 32 000 48.1, 39.2 and 42.7; 1 500 of 48 000 43.7, 36.0 and 35.8, of 65 536 61.1, 47.0
  // and 42.6; 1 000 of 128 256 in fp32 144, 114 and 94.  The lines could lie a little lower, near 44 and 96 KiB.
  const long long bytes = (long long)a.vocab * sizeof(T);
  if (bytes <= 52 << 10) return logprobs_rows<T, 64, 1>(h, a, 1, st);
  if (bytes <= 128 << 10) return logprobs_rows<T, 128, 1>(h, a, 1, st);
  return logprobs_rows<T, 256, 1>(h, a, 1, st);
}

}  // namespace a3

using namespace a3;

extern "C" int a3_token_logprobs(const a3_handle* h, const a3_logit_rows* rows, a3_stream stream) {
  if (!h || !rows) return A3_EINVAL;
  const a3_logit_rows& p = *rows;
  if (p.M < 0 || p.vocab <= 0 || p.n_top < 0 || p.n_top > p.vocab) return A3_EINVAL;
  if (p.n_top > A3_LOGPROBS_MAX_TOP || p.type < A3_LOGITS_FP32 || p.type > A3_LOGITS_FP16) return A3_EUNSUPPORTED;
  int device = -1;
  if (cudaGetDevice(&device) != cudaSuccess || device != h->device) return A3_EINVAL;
  if (p.M == 0) return A3_OK;
  if (!p.targets != !p.logprob_out || !p.top_ids_out != (p.n_top == 0) || !p.top_logprobs_out != (p.n_top == 0)) return A3_EINVAL;
  if (!p.logits || (uintptr_t)p.logits % (p.type == A3_LOGITS_FP32 ? 4 : 2)) return A3_EINVAL;
  if ((p.M > 1 && p.row_stride < (uint64_t)p.vocab) || p.row_stride > (uint64_t)1 << 31) return A3_EINVAL;
  const LogprobArgs a{p.logits, (long long)p.row_stride, p.M, p.vocab, p.targets, p.n_top, p.logprob_out, p.entropy_out, p.top_ids_out, p.top_logprobs_out, h->dev_status};
  cudaStream_t st = (cudaStream_t)stream;
  ProfScope prof(h, A3_K_TOKEN_LOGPROBS, st);
  return p.type == A3_LOGITS_FP32 ? logprobs_launch<float>(h, a, st) : p.type == A3_LOGITS_BF16 ? logprobs_launch<bf16>(h, a, st)
                                                                                                : logprobs_launch<__half>(h, a, st);
}
