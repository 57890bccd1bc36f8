// Log probabilities of given tokens from bf16 logits, one row per token:
//
//   m = max_v x_v,  S = sum_v exp(x_v - m),  A = sum_v exp(x_v - m) (x_v - m)
//   lse = m + log S,  logp = x_t - lse,  entropy = log S - A / S
//   the k largest x_v (equal ones by the lowest index) and their x_v - lse
//
// and the gradient of the logits for upstream dlogp and dentropy:
//   dx_v = dlogp ([v = t] - p_v) - dentropy p_v (log p_v + entropy)
//
// Both are bound by memory: one pass over the logits forward (2 bytes a
// logit), one read and one write backward (4 bytes).  All sums are fp32; dx is rounded to bf16 as its
// logits are.  16384 x 32000: 155 us, 6.7 TB/s (99 % of a copy's), and with eight alternatives 203 us, whose
// search is a chain of some 3 us at the end of a block; 4099 x 50257: 70 us, 5.9 TB/s, and backward
// 119 us, 6.9 TB/s (caches clean; after a write of all of the L2 each takes some 15 us more).  5 rows of 32000, five alternatives: 7 us, a launch and that chain.
#include <cuda_bf16.h>

#include "dqt_internal.h"

namespace dqt {

namespace {

constexpr int kUnroll = 4;  // 16-byte vectors in flight per thread
constexpr int kCandidates = 1024;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
// Below this x - m an exponential is 0 in fp32; distances are held there, so that a logit
// of -inf adds 0 and not 0 * inf.
constexpr float kFar = -200.0f;

__device__ __forceinline__ float bf16f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The larger of two pairs of bf16, NaN where either is.
__device__ __forceinline__ uint32_t max2(uint32_t a, uint32_t b) {
  uint32_t d;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
  return d;
}

// (m, S, A) of part of a row (m = -inf, S = A = 0 for no logit above -inf).
struct Part {
  float m, s, a;
};

// S and A as for a maximum of m (>= p.m).
__device__ __forceinline__ Part shifted(Part p, float m) {
  const float d = fmaxf(p.m - m, kFar);
  const float e = exp2_approx(d * kLog2e);
  return {m, p.s * e, e * (p.a + p.s * d)};
}
__device__ __forceinline__ Part join(Part p, Part q) {
  const float m = fmaxf(p.m, q.m);
  p = shifted(p, m);
  q = shifted(q, m);
  return {m, p.s + q.s, p.a + q.a};
}
// One more logit.  An infinite maximum leaves S = 0 and so gives NaN in the end.
__device__ __forceinline__ void add(Part& p, float x) {
  const float d = fmaxf(x - p.m, kFar);
  const float e = exp2_approx(d * kLog2e);
  p.s += e;
  p.a = fmaf(e, d, p.a);
}

// Orders bf16 values as integers: larger value, larger key; -0 as 0, NaN above all; 0 is
// below every value.
__device__ __forceinline__ uint32_t order_key(uint32_t w) {
  if ((w & 0x7FFFu) > 0x7F80u) return 0xFFFFu;
  if (w == 0x8000u) w = 0;
  return (w & 0x8000u) ? 0xFFFFu & ~w : w | 0x8000u;
}
// The value of a key (0 for -0, some NaN for NaN).
__device__ __forceinline__ uint32_t key_value(uint32_t key) {
  return (key & 0x8000u) ? key & 0x7FFFu : 0xFFFFu & ~key;
}
// Key of value and index: larger value first, then lower index.
__device__ __forceinline__ unsigned long long entry(uint32_t w, int64_t v) {
  return (static_cast<unsigned long long>(order_key(w)) << 32) | (0xFFFFFFFFu - static_cast<uint32_t>(v));
}

// A row as its 16-byte vectors and what stands before and after them.
struct Row {
  const uint16_t* x;
  const uint4* vec;
  int head;       // logits before the vectors
  int64_t nv, V;  // vectors, logits
  __device__ __forceinline__ Row(const uint16_t* row, int64_t V_) : x(row), V(V_) {
    head = static_cast<int>(((16u - (reinterpret_cast<uintptr_t>(row) & 15u)) & 15u) / 2);
    if (head > V) head = static_cast<int>(V);
    nv = (V - head) / 8;
    vec = reinterpret_cast<const uint4*>(row + head);
  }
  // The index of the i-th logit outside the vectors (up to 14 of them), or -1
  __device__ __forceinline__ int64_t outside(int i) const {
    const int64_t v = i < head ? i : head + 8 * nv + (i - head);
    return v < V ? v : -1;
  }
  // Every logit of this thread's share of NT, f(bits, index)
  template <int NT, typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int64_t o = outside(threadIdx.x);
    if (threadIdx.x < 16 && o >= 0) f(static_cast<uint32_t>(x[o]), o);
    for (int64_t i = threadIdx.x; i < nv; i += NT) {
      const uint4 q = vec[i];
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int e = 0; e < 8; ++e) f((e & 1) ? w[e / 2] >> 16 : w[e / 2] & 0xFFFFu, head + 8 * i + e);
    }
  }
  // The same for the share of thread t by its warp (all lanes): four lanes to a vector
  template <int NT, typename F>
  __device__ __forceinline__ void each_of(int t, int lane, F&& f) const {
    const int64_t o = lane == 0 ? outside(t) : -1;
    if (t < 16 && o >= 0) f(static_cast<uint32_t>(x[o]), o);
    for (int64_t j = lane >> 2; t + (j - (lane >> 2)) * NT < nv; j += 16) {  // (all lanes together)
      const int64_t i[2] = {t + j * NT, t + (j + 8) * NT};
      uint32_t w[2];
#pragma unroll
      for (int e = 0; e < 2; ++e)
        w[e] = i[e] < nv ? reinterpret_cast<const uint32_t*>(vec + i[e])[lane & 3] : 0u;
#pragma unroll
      for (int e = 0; e < 2; ++e)
        if (i[e] < nv) {
          const int64_t v = head + 8 * i[e] + 2 * (lane & 3);
          f(w[e] & 0xFFFFu, v);
          f(w[e] >> 16, v + 1);
        }
    }
  }
};

// The k-th largest of the threads' keys of 16 bits, given the largest (0: fewer than k
// are above 0).  Mostly the k-th is within 256 of it.
template <int NT>
__device__ __forceinline__ uint32_t kth_key(uint32_t key, uint32_t largest, int k) {
  uint32_t lo = largest > 255u ? largest - 255u : 1u;
  int bit = 7;
  if (__syncthreads_count(key >= lo) < k) {
    lo = 0;
    bit = 15;
  }
#pragma unroll 1
  for (; bit >= 0; --bit)
    if (__syncthreads_count(key >= lo + (1u << bit)) >= k) lo += 1u << bit;
  return lo;
}

// One block per row.  A thread keeps (m, S, A) of its own logits, 32 at a time
// against their common maximum, and the block joins them.
//
// Alternatives: at least k logits reach the k-th largest of the threads' maxima, and
// only threads whose maxima reach it own such logits: their warps read those
// threads' logits again into a list, whose k first are the answer.  A list that runs over (many equal
// logits) is made again with a bound on value and index, the k-th largest of
// the threads' first largest; one that still does (a thread with hundreds of logits and
// most of the largest) is left for k rounds over the row.
//
// NT threads: a row's loads are few and its end is a chain of short steps, which fall
// beside other rows' loads where an SM has many blocks: 64 up to 4096 logits, 128 up to 32768, 256
// above, and 1024 where there are no more rows than SMs.  16384 rows with eight alternatives, us with
// 64, 128 and 256 threads: 4000 logits 61, 72, 115; 16000: 158, 127, 152; 4000 rows of 128256: 436, 264, 211.
template <int NT>
__global__ void __launch_bounds__(NT)
    token_logprob_kernel(const uint16_t* __restrict__ x, int64_t ld, const int64_t* __restrict__ tgt,
                         int64_t V, int top, float* __restrict__ logp, float* __restrict__ entropy,
                         float* __restrict__ lse, int64_t* __restrict__ top_ids,
                         float* __restrict__ top_logp) {
  dep_wait();
  constexpr int kWarps = NT / 32;
  __shared__ Part parts[kWarps];
  __shared__ unsigned long long list[kCandidates];
  __shared__ unsigned long long bound;
  __shared__ uint32_t listed;
  const int64_t r = blockIdx.x;
  const Row row(x + r * ld, V);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Part p = {-INFINITY, 0.0f, 0.0f};
  bool nan = false;
  // (asked for ahead: thread 0 would wait for it while all others wait for thread 0)
  int64_t target = 0;
  uint32_t at_target = 0;
  if (threadIdx.x == 0) {
    target = tgt[r];
    if (target >= 0 && target < V) at_target = row.x[target];
  }
  for (int64_t i0 = threadIdx.x; i0 < row.nv; i0 += kUnroll * NT) {
    uint32_t w[kUnroll][4];
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * NT;
      // (past the end: -inf, which adds nothing)
      const uint4 q = i < row.nv ? row.vec[i] : make_uint4(0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u);
      w[u][0] = q.x;
      w[u][1] = q.y;
      w[u][2] = q.z;
      w[u][3] = q.w;
    }
    uint32_t mx[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      mx[e] = w[0][e];
#pragma unroll
      for (int u = 1; u < kUnroll; ++u) mx[e] = max2(mx[e], w[u][e]);
    }
    const uint32_t mm = max2(max2(mx[0], mx[1]), max2(mx[2], mx[3]));
    const float g = fmaxf(bf16f(mm), bf16_hi(mm));
    nan |= bf16f(mm) != bf16f(mm) || bf16_hi(mm) != bf16_hi(mm);
    if (g > p.m) p = shifted(p, g);
    f32x2 s = pack2(p.s, 0.0f), a = pack2(p.a, 0.0f);
    const f32x2 nm = pack2(-p.m, -p.m), l2e = pack2(kLog2e, kLog2e);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        // (x log2 e - m log2 e as one operation was 2 % faster, and wrong for logits of 1e30)
        const float2 x = unpack2(add2(pack2(bf16f(w[u][e]), bf16_hi(w[u][e])), nm));
        const f32x2 d = pack2(fmaxf(x.x, kFar), fmaxf(x.y, kFar));
        const f32x2 v = exp2_approx2(mul2(d, l2e));
        s = add2(s, v);
        a = fma2(v, d, a);
      }
    p.s = unpack2(s).x + unpack2(s).y;
    p.a = unpack2(a).x + unpack2(a).y;
  }
  if (threadIdx.x < 16) {
    const int64_t o = row.outside(threadIdx.x);
    if (o >= 0) {
      const float f = bf16f(row.x[o]);
      nan |= f != f;
      if (f > p.m) p = shifted(p, f);
      add(p, f);
    }
  }
  const bool any = threadIdx.x < row.nv || (threadIdx.x < 16 && row.outside(threadIdx.x) >= 0);
  const uint32_t key = !any ? 0u : nan ? 0xFFFFu : order_key(__float_as_uint(p.m) >> 16);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1)
    p = join(p, {__shfl_xor_sync(~0u, p.m, off), __shfl_xor_sync(~0u, p.s, off),
                 __shfl_xor_sync(~0u, p.a, off)});
  if (lane == 0) parts[warp] = p;
  if (threadIdx.x == 0) listed = 0;
  const bool nans = __syncthreads_or(nan);
  p = parts[lane % kWarps];
#pragma unroll
  for (int off = kWarps / 2; off > 0; off >>= 1)
    p = join(p, {__shfl_xor_sync(~0u, p.m, off), __shfl_xor_sync(~0u, p.s, off),
                 __shfl_xor_sync(~0u, p.a, off)});
  // (the two sides of a join may round differently: everyone takes lane 0's)
  p = {__shfl_sync(~0u, p.m, 0), __shfl_sync(~0u, p.s, 0), __shfl_sync(~0u, p.a, 0)};
  const bool none = p.m == -INFINITY && !nans;  // no logit above -inf
  const float log_s = nans ? __uint_as_float(0x7FC00000u) : kLn2 * log2f(p.s);
  auto logprob = [&](uint32_t w) { return none ? -INFINITY : (bf16f(w) - p.m) - log_s; };
  if (threadIdx.x == 0) {
    lse[r] = none ? -INFINITY : p.m + log_s;
    entropy[r] = none ? 0.0f : log_s - p.a / p.s;
    logp[r] = target >= 0 && target < V ? logprob(at_target) : 0.0f;
  }
  if (top == 0) return;

  const uint32_t kth =
      kth_key<NT>(key, nans ? 0xFFFFu : order_key(__float_as_uint(p.m) >> 16), top);
  const bool reach = any && key >= kth;
  // the entries from b on of the threads in `who`, by their warp
  auto gather = [&](unsigned who, unsigned long long b) {
    for (; who; who &= who - 1)
      row.each_of<NT>(warp * 32 + __ffs(who) - 1, lane, [&](uint32_t w, int64_t v) {
        const unsigned long long e = entry(w, v);
        if (e >= b) {
          const uint32_t i = atomicAdd(&listed, 1u);
          if (i < kCandidates) list[i] = e;
        }
      });
  };
  gather(__ballot_sync(~0u, reach), static_cast<unsigned long long>(kth) << 32);
  __syncthreads();
  uint32_t n = listed;
  if (n > kCandidates) {
    unsigned long long first = 0;
    if (reach)
      row.each<NT>([&](uint32_t w, int64_t v) {
        const unsigned long long e = entry(w, v);
        first = e > first ? e : first;
      });
    __syncthreads();
    if (threadIdx.x == 0) listed = 0;
    if (threadIdx.x == 0) bound = 0;
    __syncthreads();
    if (reach) list[atomicAdd(&listed, 1u)] = first;
    __syncthreads();
    const uint32_t nf = listed;
    int rank = 0;
    if (reach)
      for (uint32_t i = 0; i < nf; ++i) rank += list[i] > first;
    if (reach && rank == top - 1) bound = first;
    __syncthreads();
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
    const unsigned long long b = bound;
    gather(__ballot_sync(~0u, reach && first >= b), b);
    __syncthreads();
    n = listed;
  }
  if (n <= kCandidates) {
    for (uint32_t i = threadIdx.x; i < n; i += NT) {
      const unsigned long long e = list[i];
      int rank = 0;
      for (uint32_t k = 0; k < n; ++k) rank += list[k] > e;
      if (rank < top) {
        const int64_t v = 0xFFFFFFFFu - static_cast<uint32_t>(e);
        top_ids[r * top + rank] = v;
        top_logp[r * top + rank] = logprob(key_value(static_cast<uint32_t>(e >> 32)));
      }
    }
    return;
  }
  unsigned long long last = ~0ull;
  for (int k = 0; k < top; ++k) {
    unsigned long long best = 0;
    row.each<NT>([&](uint32_t w, int64_t v) {
      const unsigned long long e = entry(w, v);
      if (e < last && e > best) best = e;
    });
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      const unsigned long long o = __shfl_xor_sync(~0u, best, off);
      best = o > best ? o : best;
    }
    __syncthreads();
    if (lane == 0) list[warp] = best;
    __syncthreads();
    best = list[0];
    for (int w = 1; w < kWarps; ++w) best = list[w] > best ? list[w] : best;
    last = best;
    if (threadIdx.x == 0) {
      const int64_t v = 0xFFFFFFFFu - static_cast<uint32_t>(best);
      top_ids[r * top + k] = v;
      top_logp[r * top + k] = logprob(key_value(static_cast<uint32_t>(best >> 32)));
    }
  }
}

// The gradient of a logit
struct Grad {
  float l, c, de, dl;  // lse, dlogp + dentropy * entropy, dentropy, dlogp
  __device__ __forceinline__ float operator()(float x, bool target) const { return of(x - l, target); }
  __device__ __forceinline__ float of(float logp, bool target) const {
    // (held off -inf, so that a logit without probability gets 0; a NaN in c reaches all)
    const float lp = fmaxf(logp, kFar);
    const float d = -exp2_approx(lp * kLog2e) * fmaf(de, lp, c);
    return target ? d + dl : d;
  }
};

// Beyond this |lse|, half a step of which puts 2^-15 into p, a row's lse may say too little about
// its log S: a row of bf16's lowest value alone has lse = max in fp32, and p = 1 from it.
constexpr float kLseLimit = 1024.0f;

// Such a row: max and log S found anew, one logit at a time.
template <int NT>
__device__ __forceinline__ void far_row(const Row& row, const Grad& g, int64_t t, uint16_t* out) {
  __shared__ Part parts[NT / 32];
  Part p = {-INFINITY, 0.0f, 0.0f};
  auto joined = [&] {
#pragma unroll 1
    for (int off = 16; off > 0; off >>= 1)
      p = join(p, {__shfl_xor_sync(~0u, p.m, off), __shfl_xor_sync(~0u, p.s, off), 0.0f});
  };
#pragma unroll 1
  for (int64_t v = threadIdx.x; v < row.V; v += NT) {
    const float f = bf16f(row.x[v]);
    if (f > p.m) p = shifted(p, f);
    add(p, f);
  }
  joined();
  if ((threadIdx.x & 31) == 0) parts[threadIdx.x >> 5] = p;
  __syncthreads();
  p = (threadIdx.x & 31) < NT / 32 ? parts[threadIdx.x & 31] : Part{-INFINITY, 0.0f, 0.0f};
  joined();
  const float m = __shfl_sync(~0u, p.m, 0), log_s = kLn2 * log2f(__shfl_sync(~0u, p.s, 0));
#pragma unroll 1
  for (int64_t v = threadIdx.x; v < row.V; v += NT)
    out[v] = __bfloat16_as_ushort(__float2bfloat16_rn(g.of((bf16f(row.x[v]) - m) - log_s, v == t)));
}

// One block per row; 16-byte vectors where the rows of logits and gradient
// stand alike to a 16-byte boundary (VEC), else single values.  NT threads: 128 up to 8192 logits,
// 256 up to 32768, 512 above and where there are no more rows than SMs (us with 128, 256 and 512, 16384
// rows of 4000: 45, 53, 72; of 24000: 244, 238, 240; 4000 rows of 128256: 330, 324, 311).
template <int NT, bool VEC>
__global__ void __launch_bounds__(NT)
    token_logprob_bwd_kernel(const uint16_t* __restrict__ x, int64_t ld, const int64_t* __restrict__ tgt,
                             const float* __restrict__ lse, const float* __restrict__ entropy,
                             const float* __restrict__ dlogp, const float* __restrict__ dent, int64_t V,
                             uint16_t* __restrict__ dx) {
  dep_wait();
  const int64_t r = blockIdx.x;
  const Row row(x + r * ld, V);
  uint4 q[kUnroll];
  auto fetch = [&](int64_t i0) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u)
      if (i0 + u * NT < row.nv) q[u] = __ldcs(row.vec + i0 + u * NT);
  };
  if (VEC) fetch(threadIdx.x);
  const int64_t t = tgt[r];
  Grad g;
  g.l = lse[r];
  g.de = dent[r];
  g.dl = dlogp[r];
  if (t < 0 || t >= V) g.dl = 0.0f;
  g.c = fmaf(g.de, entropy[r], g.dl);
  const bool none = g.l == -INFINITY;  // a row of -inf alone
  if (none) g = {0.0f, 0.0f, 0.0f, 0.0f};
  uint16_t* out = dx + r * V;
  if (fabsf(g.l) > kLseLimit) {  // (not a NaN)
    far_row<NT>(row, g, t, out);
    return;
  }
  auto one = [&](int64_t v) {
    out[v] = none ? 0 : __bfloat16_as_ushort(__float2bfloat16_rn(g(bf16f(row.x[v]), v == t)));
  };
  if (!VEC) {
    for (int64_t v = threadIdx.x; v < V; v += NT) one(v);
    return;
  }
  uint4* ov = reinterpret_cast<uint4*>(out + row.head);
  for (int64_t i0 = threadIdx.x; i0 < row.nv; i0 += kUnroll * NT) {
    if (i0 != threadIdx.x) fetch(i0);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int64_t i = i0 + u * NT;
      if (i >= row.nv) break;
      const uint32_t w[4] = {q[u].x, q[u].y, q[u].z, q[u].w};
      // the target's place in this vector, if it is there
      const int64_t at = t - row.head - 8 * i;
      uint32_t o[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        o[e] = none ? 0u : pack_bf16x2(g(bf16f(w[e]), at == 2 * e), g(bf16_hi(w[e]), at == 2 * e + 1));
      __stcs(ov + i, make_uint4(o[0], o[1], o[2], o[3]));
    }
  }
  if (threadIdx.x < 16) {
    const int64_t o = row.outside(threadIdx.x);
    if (o >= 0) one(o);
  }
}

}  // namespace

int launch_token_logprob(const uint16_t* logits, int64_t ld, const int64_t* targets, int64_t M, int64_t V,
                         int top, float* logp, float* entropy, float* lse, int64_t* top_ids,
                         float* top_logp, cudaStream_t stream) {
  const int nt = M <= sm_count() ? 1024 : V <= 4096 ? 64 : V <= 32768 ? 128 : 256;
  return launch_dep(nt == 1024  ? token_logprob_kernel<1024>
                    : nt == 256 ? token_logprob_kernel<256>
                    : nt == 128 ? token_logprob_kernel<128>
                                : token_logprob_kernel<64>,
                    dim3(static_cast<unsigned>(M)), nt, 0, stream, logits, ld, targets, V, top, logp, entropy,
                    lse, top_ids, top_logp);
}

int launch_token_logprob_bwd(const uint16_t* logits, int64_t ld, const int64_t* targets, const float* lse,
                             const float* entropy, const float* dlogp, const float* dent, int64_t M,
                             int64_t V, uint16_t* dlogits, cudaStream_t stream) {
  // every row alike: the same boundary at the first, and strides that differ by whole vectors
  const bool vec = ((reinterpret_cast<uintptr_t>(logits) ^ reinterpret_cast<uintptr_t>(dlogits)) & 15u) == 0 &&
                   (M == 1 || (ld - V) % 8 == 0);
  const int nt = M <= sm_count() || V > 32768 ? 512 : V > 8192 ? 256 : 128;
  return launch_dep(!vec        ? token_logprob_bwd_kernel<512, false>
                    : nt == 512 ? token_logprob_bwd_kernel<512, true>
                    : nt == 256 ? token_logprob_bwd_kernel<256, true>
                                : token_logprob_bwd_kernel<128, true>,
                    dim3(static_cast<unsigned>(M)), vec ? nt : 512, 0, stream, logits, ld, targets, lse, entropy,
                    dlogp, dent, V, dlogits);
}

}  // namespace dqt
