// Causal attention of packed documents with grouped heads.
//
//   s_ij = scale q_i . k_j  (j <= i in one document),  lse_i = log sum_j exp s_ij,
//   p_ij = exp(s_ij - lse_i),  o_i = sum_j p_ij v_j
//   delta_i = do_i . o_i,  ds_ij = p_ij (do_i . v_j - delta_i)
//   dq_i = scale sum_j ds_ij k_j,  dk_j = scale sum ds_ij q_i,  dv_j = sum p_ij do_i
//   (dk and dv over the q heads that share the k and v head)
//
// Work comes as tiles of rows of one document, in the order of a table that
// dqt_attn_plan fills: the longest first.
//
// Scores, their maxima and sums, delta and all accumulators are fp32.  Rounded to bf16, because the
// tensor cores take no wider operands at this rate: p (its sum l is taken before), and ds.  So o,
// dv, dq and dk carry a rounding of each term next to that of the result: 0.0025 relative
// rms for dq and dk, where rounding the result alone gives 0.0017.
//
// Masked places: what a row does not see of its own tile of 128 is multiplied by a p or ds of 0, so a
// value there that is not finite makes the row's sums NaN, as a matrix product with the zeros written out
// does.  Rows of other documents, and of tiles that a row does not see, reach it in no way.
#include <cuda_bf16.h>

#include <type_traits>

#include "dqt_internal.h"

namespace dqt {

namespace {

constexpr uint64_t kDrainNs = 1000000000ull;  // wait for in-flight copies and products when giving up

constexpr uint32_t kRowBytes = 128;               // a tile's row of 64 columns
constexpr uint32_t kAtomBytes = 128 * kRowBytes;  // 128 rows of 64 columns

__device__ __forceinline__ uint8_t* align1024(uint8_t* p) {
  const uint32_t s = smem_u32(p);
  return p + ((1024u - (s & 1023u)) & 1023u);
}
// The waits of a role whose warps stay together: once one has run out the rest
// do not wait, and the role runs on to its end (its outputs are undefined then, its
// accesses stay where they are) and says so.  Control flow never depends on it.
struct Waits {
  uint64_t limit_ns;
  bool late = false;
  __device__ __forceinline__ void operator()(uint64_t* bar, uint32_t parity) {
    if (!late) late = !mbar_wait(bar, parity, limit_ns);
  }
  // Two phases, asked for together: an answer takes 150 clk
  __device__ __forceinline__ void operator()(uint64_t* a, uint32_t pa, uint64_t* b, uint32_t pb) {
    if (!mbar_test2(a, pa, b, pb)) {
      (*this)(a, pa);
      (*this)(b, pb);
    }
  }
};
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ f32x2 f2(uint32_t a, uint32_t b) {
  return pack2(__uint_as_float(a), __uint_as_float(b));
}
__device__ __forceinline__ uint32_t pack_bf16x2(f32x2 v) {
  const float2 x = unpack2(v);
  return pack_bf16x2(x.x, x.y);
}
// c plus the products of two pairs of bf16
__device__ __forceinline__ f32x2 dot2(uint32_t a, uint32_t b, f32x2 c) {
  return fma2(f2(a << 16, a & 0xFFFF0000u), f2(b << 16, b & 0xFFFF0000u), c);
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t sel) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %1, %2;" : "=r"(d) : "r"(a), "r"(sel));
  return d;
}
__device__ __forceinline__ uint64_t first_bits(int n) {
  return n <= 0 ? 0 : n >= 64 ? ~0ull : (1ull << n) - 1;
}
// A copying role's wait for a buffer of round ph - 1 to be empty.  It was full before,
// unless a role that ran out of time let it go early: its copies must have landed, or the
// next round's would count on the same phase.
__device__ __forceinline__ bool buffer_wait(uint64_t* empty, uint64_t* full, uint32_t ph, uint64_t ns) {
  return mbar_test2(empty, ph, full, ph) || (mbar_wait(empty, ph, ns) && mbar_wait(full, ph, ns));
}
// A place in a ring of N and the parity of its present round.
template <int N>
struct Ring {
  int i = 0;
  uint32_t ph = 0;
  __device__ __forceinline__ void next() {
    if (++i == N) {
      i = 0;
      ph ^= 1u;
    }
  }
};
// n / d for n < 2^31 as a product: magic = ceil(2^(32 + s) / d) with 2^s < d <= 2^(s + 1), so
// magic d - 2^(32 + s) < 2^(s + 1) and the quotient is exact.  (Divisions were most of the 1000
// clk that a warp took to find its next item.)
struct Div {
  uint32_t d = 1, magic = 0, shift = 0;
  Div() = default;
  explicit Div(int64_t by) : d(static_cast<uint32_t>(by)) {
    if (d == 1) return;
    while ((2ull << shift) < d) ++shift;
    magic = static_cast<uint32_t>(((1ull << (32 + shift)) + d - 1) / d);
  }
  __device__ __forceinline__ int of(int n) const {
    return d == 1 ? n : static_cast<int>(__umulhi(static_cast<uint32_t>(n), magic) >> shift);
  }
};
// Descriptor of shared memory at addr, of the kind whose halves are hi and lo.
__device__ __forceinline__ uint64_t desc_at(uint32_t hi, uint32_t lo, uint32_t addr) {
  return (static_cast<uint64_t>(hi) << 32) | (lo + (addr >> 4));
}
// Descriptor of rows of 16 columns without a swizzle: the first eight at lo, 16 bytes a
// row, and the others at hi (above lo).
__device__ __forceinline__ uint64_t sdesc_pieces(uint32_t lo, uint32_t hi) {
  return static_cast<uint64_t>((lo & 0x3FFFFu) >> 4) | static_cast<uint64_t>((hi - lo) >> 4) << 16 |
         static_cast<uint64_t>(128 >> 4) << 32 | 1ull << 46;
}
// v as a sum of three bf16: 24 bits of it
__device__ __forceinline__ void pieces(float v, uint32_t (&w)[3]) {
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    const __nv_bfloat16 b = __float2bfloat16_rn(v);
    w[i] = __bfloat16_as_ushort(b);
    v -= __bfloat162float(b);
  }
}
// 32 columns of a warp's 32 rows (a row per lane, fp32 bits in v, times f) to bf16 in
// memory: through 2 KB of shared memory, so that a store instruction writes 8 rows' 64
// bytes and not 16 bytes of 32 rows.  out: this lane's own row's first column; valid: the
// rows that are there.
__device__ __forceinline__ void store_rows(uint4* buf, const uint32_t (&v)[32], float f, uint16_t* out,
                                           int64_t row_stride, int valid, int lane) {
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e)
      w[e] = pack_bf16x2(__uint_as_float(v[8 * k + 2 * e]) * f, __uint_as_float(v[8 * k + 2 * e + 1]) * f);
    buf[lane * 4 + (k ^ ((lane >> 1) & 3))] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __syncwarp();
  uint16_t* first = out - lane * row_stride;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int r = 8 * k + (lane >> 2);
    const uint4 w = buf[r * 4 + ((lane & 3) ^ ((r >> 1) & 3))];
    if (r < valid) *reinterpret_cast<uint4*>(first + r * row_stride + 8 * (lane & 3)) = w;
  }
  __syncwarp();
}
// Zeros in rows [from, to) of an atom (64 columns of any rows) in shared memory, by a warp.
__device__ __forceinline__ void zero_rows(uint8_t* atom, int from, int to, int lane) {
  for (int i = lane; i < (to - from) * 8; i += 32)
    *reinterpret_cast<uint4*>(atom + (from + i / 8) * kRowBytes + (i % 8) * 16) = make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <int N>
__device__ __forceinline__ void regs_inc() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_dec() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
// Copies bytes (a multiple of 16, both addresses too) to shared memory, counted on bar.
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile(
      "cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(
          smem_u32(dst)),
      "l"(src), "r"(bytes), "r"(smem_u32(bar))
      : "memory");
}
// Items in falling order of work, dealt out to and fro.
__device__ __forceinline__ int deal(int round) {
  const int b = static_cast<int>(blockIdx.x), g = static_cast<int>(gridDim.x);
  return round * g + ((round & 1) ? g - 1 - b : b);
}
// The tile of an item that may be one past the last (any tile then): for loads ahead.
__device__ __forceinline__ dqt_attn_tile_t tile_of(const dqt_attn_tile_t* tiles, int it, int items,
                                                   const Div& per) {
  const int4 v = __ldg(reinterpret_cast<const int4*>(tiles) + per.of(it < items ? it : 0));
  return {v.x, v.y, v.z, v.w};
}

// A tile that lies in the tensors, and its slot in the workspace; others are left out.  (Rows start
// at multiples of 128: the slots of a document's other rows are counted from that.)
__device__ __forceinline__ bool tile_ok(const dqt_attn_tile_t& t, const dqt_attn_layout_t& L) {
  return t.start >= 0 && t.row >= 0 && (t.row & 127) == 0 && t.row < t.len && t.start + static_cast<int64_t>(t.len) <= L.tokens &&
         t.slot >= t.row >> 7 && t.slot + static_cast<int64_t>((t.len - t.row + 127) >> 7) <= L.tiles;
}

// ---------------------------------------------------------------------------
// Forward on the tensor cores: a CTA has an SM to itself and goes from one pair of tiles to the
// next; two tiles of 128 queries in flight that read the same keys and values, so that one
// tile's softmax runs beside the other's matrix products.
//
//   warps 0-3, 4-7  softmax of tile 0 and tile 1: a thread has a query
//   warp 8          the items, copies (TMA): queries, and a ring of key and value tiles
//   warp 9          products (tcgen05) S = Q K^T
//   warp 10         products O += P V
//   warp 11         none
//   warps 12-15     outputs of either tile, while the softmax is at the next item
//
// S (fp32) and P (bf16, over S's own columns) stay in tensor memory; P is the
// A operand of the second product from there.  The blocks of both tiles take
// the S buffers in turn: three of them where tensor memory has room (dim 64), so
// that the next S is there when a softmax ends.  O is rescaled in place by the
// softmax warps, once the last product into it is done, and only when a row's maximum has
// grown by 2^8 (P then stays below 2^8, which bf16 holds as well).
//
// The two tiles are two heads of a group at the same rows where the group has
// an even number of heads (the same blocks for both: nothing idles), else 256
// rows of one head (32 heads over 8: 16 documents of 1 to 4093 168 and 176 us, one of 16384 866 and 872).
//
// The grid has a block for each pair of tiles, longest first; a block that is done takes over the
// next that has not started (cluster launch control), so that few uneven pairs fill the SMs: 6063 tokens in 4
// documents, 16 heads over 2 of 128, 59 us, and 68 with the pairs dealt out in advance.
//
// A document of 16384, 32 q heads over 8 of 64: 869 us, 1.27 PFLOP/s, 66 % of the rate of a large matrix
// product.  A pair of blocks takes 1960 clk, in which the exponentials take 1024 of the SM's (32 a clk)
// and the products 1024: a warp's own chain bounds it (a wait of 150 to 400 clk, the maximum 450, exponentials
// and sums 950), two warps to a scheduler.  Measured and left: turns for the two warps' exponentials 897 us, a P
// beside S with S freed once read 1050, S read twice in a rolled loop 1110.
// ---------------------------------------------------------------------------
// Four groups of four warps (two of them for the mathematics), and their registers of the
// 512 * 128 that a block is launched with.
constexpr int kThreads = 512, kRegsLaunch = 128;
struct FwdRegs {
  static constexpr int kMath = 176, kFeed = 80, kItems = 80;
};
struct BwdRegs {
  static constexpr int kMath = 168, kFeed = 72, kItems = 104;
};
static_assert(2 * FwdRegs::kMath + FwdRegs::kFeed + FwdRegs::kItems <= 4 * kRegsLaunch, "registers");
static_assert(2 * BwdRegs::kMath + BwdRegs::kFeed + BwdRegs::kItems <= 4 * kRegsLaunch, "registers");
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int D>
struct FwdSmem {
  static constexpr int ATOMS = D / 64;
  static constexpr int TILE = ATOMS * kAtomBytes;  // 128 rows of Q, K or V
  static constexpr int QBUF = D == 64 ? 2 : 1;     // buffers of two query tiles
  static constexpr int RING = D == 64 ? 8 : 4;     // K and V tiles
  static constexpr int RING_OFF = QBUF * 2 * TILE;
  static constexpr int OUT_OFF = RING_OFF + RING * TILE;  // 2 KB for each warp that writes outputs
  static constexpr int SUM_OFF = OUT_OFF + 4 * 2048;      // maximum and sum of the tiles' rows
  static constexpr int QUEUE_OFF = SUM_OFF + 2 * 128 * 8;
  static constexpr int BAR_OFF = QUEUE_OFF + 160;
  static constexpr int BYTES = BAR_OFF + 512 + 1024;  // alignment of the swizzle's 1024 bytes
  static_assert(BYTES <= 232448, "shared memory per CTA");
  static constexpr int NS = D == 64 ? 3 : 2;          // S buffers
  static_assert(NS * 128 + 2 * D <= 512, "tensor memory");
  static_assert((2 * RING + 2 * QBUF + 2 * NS + 22) * 8 + 4 <= 512, "barriers");
};

struct FwdParams {
  dqt_attn_layout_t L;
  const dqt_attn_tile_t* tiles;
  int items;      // pairs of tiles
  Div pairs;      // of them per table entry
  Div group;      // q heads to a k and v head
  bool by_heads;  // a pair is two heads (else two halves of 256 rows)
  float scale_log2;
  uint16_t* o;
  float* lse;
  uint64_t wait_ns;
  unsigned int* status;
};

// The items of a block in turn: its own, then such as other blocks of the grid have not begun
// (which come in the same order, longest first).  The copying lane finds them and gives them to the
// other roles' warps through four places in shared memory.
struct Queue {
  int4 item[4];
  int4 answer;
  uint64_t full[4], empty[4], answered;
};
// What a role knows of an item.
struct FwdItem {
  int start, len, row, head;
};
__device__ __forceinline__ FwdItem fwd_item(const FwdParams& p, int it, const dqt_attn_tile_t& t) {
  const int j = it - p.pairs.of(it) * static_cast<int>(p.pairs.d);
  FwdItem x{t.start, t.len, t.row, p.by_heads ? 2 * j : j};
  if (!tile_ok(t, p.L)) x = {0, 0, 0, x.head};
  return x;
}
// Key blocks of 128 that tile t of the item sees (0: the tile has no rows).
__device__ __forceinline__ int fwd_blocks(const FwdParams& p, const FwdItem& x, int t) {
  const int row = x.row + (p.by_heads ? 0 : 128 * t);
  return row < x.len ? (row >> 7) + 1 : 0;
}
// The next item for a role's warp; false: there are no more, or a wait has run out (of the whole warp).
__device__ __forceinline__ bool take(Queue* q, Ring<4>& at, Waits& wait, int lane, FwdItem& x) {
  wait(&q->full[at.i], at.ph);
  if (__any_sync(~0u, wait.late)) return false;
  const int4 v = q->item[at.i];
  __syncwarp();
  if (lane == 0) mbar_arrive(&q->empty[at.i]);
  at.next();
  x = {v.x, v.y, v.z, v.w};
  return x.start >= 0;
}
template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    attn_fwd_kernel(const __grid_constant__ CUtensorMap mq, const __grid_constant__ CUtensorMap mk,
                    const __grid_constant__ CUtensorMap mv, const __grid_constant__ FwdParams p) {
  using S = FwdSmem<D>;
  constexpr uint32_t kIdescS = idesc_bf16(128, 128, false, false);
  constexpr uint32_t kIdescO = idesc_bf16(128, D, false, true);
  constexpr uint32_t kO = S::NS * 128;  // tensor memory: the S buffers, O of both tiles

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);
  uint64_t* kv_empty = kv_full + S::RING;
  uint64_t* q_full = kv_empty + S::RING;
  uint64_t* q_empty = q_full + S::QBUF;
  uint64_t* p_full = q_empty + S::QBUF;  // [NS]
  uint64_t* s_free = p_full + S::NS;     // [NS]
  // Of either tile's blocks, in turns of four: S, and the product into O.  A parity wait
  // is good only for who knows the phase before complete: a tile's softmax waits
  // for each S of its own, and when it has S of block i the product of block i - 4 is done (S is
  // issued after the product of the block NS before it, of either tile).
  uint64_t* s_full = s_free + S::NS;     // [2][4]
  uint64_t* o_done = s_full + 8;         // [2][4]
  uint64_t* sum_full = o_done + 8;       // [2]: a tile's item is through the softmax
  uint64_t* o_free = sum_full + 2;       // [2]: its O is read, and the sums
  uint64_t* drain = o_free + 2;          // [2]
  uint32_t* slot = reinterpret_cast<uint32_t*>(drain + 2);
  Queue* queue = reinterpret_cast<Queue*>(smem + S::QUEUE_OFF);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::RING; ++i) {
      mbar_init(&kv_full[i], 1);
      mbar_init(&kv_empty[i], 1);
    }
    for (int i = 0; i < S::QBUF; ++i) {
      mbar_init(&q_full[i], 1);
      mbar_init(&q_empty[i], 1);
    }
    for (int i = 0; i < S::NS; ++i) {
      mbar_init(&p_full[i], 4);
      mbar_init(&s_free[i], 1);
    }
    for (int i = 0; i < 8; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&o_done[i], 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(&sum_full[t], 4);
      mbar_init(&o_free[t], 4);
      mbar_init(&drain[t], 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(&queue->full[i], 1);
      mbar_init(&queue->empty[i], 14);  // S and PV, eight softmax warps, four for outputs
    }
    mbar_init(&queue->answered, 1);
    fence_mbarrier_init();
    tma_prefetch_desc(&mq);
    tma_prefetch_desc(&mk);
    tma_prefetch_desc(&mv);
  }
  if (warp == 9) tmem_alloc(slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *slot;
  dep_wait();
  dep_trigger();

  if (warp >= 12) {
    regs_dec<FwdRegs::kItems>();
    // ---------------- outputs ----------------
    const int row = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    uint4* buf = reinterpret_cast<uint4*>(smem + S::OUT_OFF) + quad * 128;
    const float2* sums = reinterpret_cast<const float2*>(smem + S::SUM_OFF) + row;
    Waits wait{p.wait_ns};
    uint32_t ns[2] = {0, 0}, ni[2] = {0, 0};  // blocks and items of either tile so far
    Ring<4> from;
    FwdItem x;
    while (take(queue, from, wait, lane, x)) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int blocks = fwd_blocks(p, x, t);
        if (blocks == 0) continue;
        wait(&sum_full[t], ni[t] & 1u);
        ++ni[t];
        ns[t] += blocks;
        wait(&o_done[4 * t + ((ns[t] - 1) & 3)], ((ns[t] - 1) >> 2) & 1u);
        tc_fence_after();
        const float2 ml = sums[128 * t];
        const int head = x.head + (p.by_heads ? t : 0);
        const int i = x.row + (p.by_heads ? 0 : 128 * t) + row;
        const int64_t token = static_cast<int64_t>(x.start) + i;
        const float inv = 1.0f / ml.y;
        uint16_t* out = p.o + (token * p.L.heads + head) * D;
#pragma unroll
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(tmem + lanes + kO + t * D + c, o);
          tmem_ld_wait();
          if (c + 32 == D) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&o_free[t]);
          }
          store_rows(buf, o, inv, out + c, p.L.heads * D, x.len - i + lane, lane);
        }
        if (i < x.len) p.lse[head * p.L.tokens + token] = (ml.x + log2f(ml.y)) * kLn2;
      }
    }
    if (wait.late) record_timeout(p.status);
  } else if (warp >= 8) {
    regs_dec<FwdRegs::kFeed>();
    if (warp == 8) {
      if (lane == 0) {
        // ---------------- copies ----------------
        int n = 0, nq = 0;  // ring entries and query buffers filled so far
        bool ok = true;
        int it = blockIdx.x;
        uint32_t asked = 0;
        Ring<4> to;
        // gives the other roles an item
        auto give = [&](const FwdItem& x, int r) {
          if (r >= 4 && !mbar_wait(&queue->empty[to.i], to.ph ^ 1u, p.wait_ns)) return false;
          queue->item[to.i] = make_int4(x.start, x.len, x.row, x.head);
          mbar_arrive(&queue->full[to.i]);
          to.next();
          return true;
        };
        for (int r = 0; ok; ++r) {
          if (it < 0) {
            ok = give({-1, 0, 0, 0}, r);
            break;
          }
          const FwdItem x = fwd_item(p, it, tile_of(p.tiles, it, p.items, p.pairs));
          if (!give(x, r)) {
            ok = false;
            break;
          }
          const int b0 = fwd_blocks(p, x, 0), b1 = fwd_blocks(p, x, 1), blocks = max(b0, b1);
          const int hk = p.group.of(x.head);
          for (int j = 0; ok && j < blocks; ++j) {
            if (j == 0) {
              const int b = nq % S::QBUF;
              if (nq >= S::QBUF && !buffer_wait(&q_empty[b], &q_full[b], (nq / S::QBUF - 1) & 1u, p.wait_ns)) {
                ok = false;
                break;
              }
              mbar_arrive_expect_tx(&q_full[b], 2 * S::TILE);
              for (int t = 0; t < 2; ++t)
                for (int a = 0; a < S::ATOMS; ++a)
                  tma_load_3d(&mq, &q_full[b], smem + (2 * b + t) * S::TILE + a * kAtomBytes, 64 * a,
                              x.head + (p.by_heads ? t : 0), x.start + x.row + (p.by_heads ? 0 : 128 * t));
              ++nq;
            }
            for (int kv = 0; kv < 2; ++kv, ++n) {
              const int s = n % S::RING;
              if (n >= S::RING && !buffer_wait(&kv_empty[s], &kv_full[s], (n / S::RING - 1) & 1u, p.wait_ns)) {
                ok = false;
                break;
              }
              mbar_arrive_expect_tx(&kv_full[s], S::TILE);
              for (int a = 0; a < S::ATOMS; ++a)
                tma_load_3d(kv ? &mv : &mk, &kv_full[s], smem + S::RING_OFF + s * S::TILE + a * kAtomBytes,
                            64 * a, hk, x.start + 128 * j);
            }
          }
          clc_ask(&queue->answer, &queue->answered);
          if (!mbar_wait(&queue->answered, asked & 1u, kDrainNs)) {
            ok = false;
            break;
          }
          ++asked;
          it = clc_answer(&queue->answer);
          fence_async_shared();
        }
        if (!ok) record_timeout(p.status);
        // the copies in flight land before the CTA exits, whoever gave up
        for (int i = n > S::RING ? n - S::RING : 0; i < n; ++i)
          mbar_wait(&kv_full[i % S::RING], (i / S::RING) & 1u, kDrainNs);
        for (int i = nq > S::QBUF ? nq - S::QBUF : 0; i < nq; ++i)
          mbar_wait(&q_full[i % S::QBUF], (i / S::QBUF) & 1u, kDrainNs);
      }
    } else if (warp == 9) {
      // ---------------- S = Q K^T ----------------
      const uint64_t desc = sdesc_sw128(0, 16, 1024);
      const uint32_t hi = static_cast<uint32_t>(desc >> 32), lo = static_cast<uint32_t>(desc);
      const uint32_t base = smem_u32(smem);
      Waits wait{p.wait_ns};
      int n = 0, nq = 0, nk = 0;  // S blocks, query buffers and key blocks so far
      uint32_t nt[2] = {0, 0};    // S blocks of either tile
      Ring<4> from;
      FwdItem x;
      while (take(queue, from, wait, lane, x)) {
        const int nb[2] = {fwd_blocks(p, x, 0), fwd_blocks(p, x, 1)}, blocks = max(nb[0], nb[1]);
        if (blocks == 0) continue;
        const int qb = nq % S::QBUF;
        wait(&q_full[qb], (nq / S::QBUF) & 1u);
        ++nq;
        for (int j = 0; j < blocks; ++j, ++nk) {
          const int ks = (2 * nk) % S::RING;
          const uint32_t k0 = base + S::RING_OFF + ks * S::TILE;
          wait(&kv_full[ks], (2 * nk / S::RING) & 1u);
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (j >= nb[t]) continue;
            const int buf = n % S::NS;
            if (n >= S::NS) wait(&s_free[buf], (n / S::NS - 1) & 1u);
            ++n;
            tc_fence_after();
            const uint32_t q0 = base + (2 * qb + t) * S::TILE;
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < D / 16; ++k) {
                const uint32_t off = (k / 4) * kAtomBytes + (k % 4) * 32;
                umma_bf16(tmem + buf * 128, desc_at(hi, lo, q0 + off), desc_at(hi, lo, k0 + off), kIdescS,
                          k > 0 ? 1u : 0u);
              }
              umma_commit(&s_full[4 * t + (nt[t] & 3)]);
            }
            __syncwarp();
            ++nt[t];
          }
          if (elect_one()) {
            umma_commit(&kv_empty[ks]);
            if (j == blocks - 1) umma_commit(&q_empty[qb]);
          }
          __syncwarp();
        }
      }
      if (wait.late) record_timeout(p.status);
      // every product issued is done before tensor memory is freed
      if (elect_one()) umma_commit(&drain[0]);
      mbar_wait(&drain[0], 0, kDrainNs);
    } else if (warp == 10) {
      // ---------------- O += P V ----------------
      const uint64_t desc = sdesc_sw128(0, kAtomBytes, 1024);
      const uint32_t hi = static_cast<uint32_t>(desc >> 32), lo = static_cast<uint32_t>(desc);
      const uint32_t base = smem_u32(smem);
      Waits wait{p.wait_ns};
      int n = 0, nk = 0;  // P blocks and value blocks so far
      uint32_t nt[2] = {0, 0}, ni[2] = {0, 0};  // P blocks and items of either tile
      Ring<4> from;
      FwdItem x;
      while (take(queue, from, wait, lane, x)) {
        const int nb[2] = {fwd_blocks(p, x, 0), fwd_blocks(p, x, 1)}, blocks = max(nb[0], nb[1]);
        for (int j = 0; j < blocks; ++j, ++nk) {
          const int vs = (2 * nk + 1) % S::RING, rows = min(128, x.len - 128 * j), steps = (rows + 15) / 16;
          const uint32_t v0 = base + S::RING_OFF + vs * S::TILE;
          wait(&kv_full[vs], (2 * nk / S::RING) & 1u);
          if (rows % 16) {
            // V's keys beyond the document: their probabilities are 0, but what
            // stands there may not be finite
            for (int a = 0; a < S::ATOMS; ++a)
              zero_rows(smem + S::RING_OFF + vs * S::TILE + a * kAtomBytes, rows, 16 * steps, lane);
            fence_async_shared();
            __syncwarp();
          }
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            if (j >= nb[t]) continue;
            const int buf = n % S::NS;
            if (j == 0 && ni[t]++ > 0) wait(&o_free[t], ni[t] & 1u);
            wait(&p_full[buf], (n / S::NS) & 1u);
            ++n;
            tc_fence_after();
            if (elect_one()) {
#pragma unroll
              for (int k = 0; k < 8; ++k)
                if (k < steps)
                  umma_bf16_ts(tmem + kO + t * D, tmem + buf * 128 + 8 * k, desc_at(hi, lo, v0 + 2048 * k),
                               kIdescO, k > 0 || j > 0 ? 1u : 0u);
              umma_commit(&s_free[buf]);
              umma_commit(&o_done[4 * t + (nt[t] & 3)]);
            }
            __syncwarp();
            ++nt[t];
          }
          if (elect_one()) umma_commit(&kv_empty[vs]);
          __syncwarp();
        }
      }
      if (wait.late) record_timeout(p.status);
      if (elect_one()) umma_commit(&drain[1]);
      mbar_wait(&drain[1], 0, kDrainNs);
    }
  } else {
    regs_inc<FwdRegs::kMath>();
    // ---------------- softmax ----------------
    const int t = warp >> 2, row = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    const uint32_t to = tmem + lanes + kO + t * D;
    const float sl = p.scale_log2;
    const f32x2 sl2 = pack2(sl, sl);
    Waits wait{p.wait_ns};
    int n0 = 0;       // S blocks of both tiles in the items so far
    uint32_t ns = 0;  // of this tile
    float m = 0.0f, l = 0.0f;  // the row's shift (in log2 units) and sum
    // the product of this tile's last block
    auto o_wait = [&] { wait(&o_done[4 * t + ((ns - 1) & 3)], ((ns - 1) >> 2) & 1u); };
    // The row's shift for a block's maximum mx.  (l = 0: no score above -inf so far, m is no
    // maximum.)  Each row goes by its own scores: what other documents' rows hold changes nothing in it.
    auto shift = [&](float mx, bool first) {
      const bool grown = mx > (l > 0.0f ? m + 8.0f : -INFINITY);
      if (__any_sync(~0u, grown)) {
        const float mn = grown ? mx : m;
        const float a = !grown ? 1.0f : l > 0.0f ? exp2_approx(m - mn) : 0.0f;
        m = mn;
        l *= a;
        if (!first) {
          o_wait();
          tc_fence_after();
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_ld_32x32b_x16(to + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
            tmem_st_32x32b_x16(to + c, o);
          }
        }
      }
    };
    // 32 scores to probabilities, and into the sums
    auto probs = [&](const uint32_t (&s)[32], f32x2 (&sum)[2], f32x2 ml2, uint32_t (&pk)[16]) {
#pragma unroll
      for (int i = 0; i < 32; i += 2) {
        const f32x2 pp = exp2_approx2(fma2(f2(s[i], s[i + 1]), sl2, ml2));
        sum[(i / 2) & 1] = add2(sum[(i / 2) & 1], pp);
        pk[i / 2] = pack_bf16x2(pp);
      }
    };
    auto largest = [&](const uint32_t (&s)[32], float (&mx4)[4]) {
#pragma unroll
      for (int i = 0; i < 32; i += 2)
        mx4[(i / 2) & 3] = max3(mx4[(i / 2) & 3], __uint_as_float(s[i]), __uint_as_float(s[i + 1]));
    };
    auto close = [&](f32x2 (&sum)[2]) {
      const float2 both = unpack2(add2(sum[0], sum[1]));
      l = both.x + both.y;
      tmem_st_wait();
    };
    auto block = [&](uint32_t ts, bool first) {
      uint32_t s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld_32x32b_x32(ts + 32 * c, s[c]);
      tmem_ld_wait();
      float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int c = 0; c < 4; ++c) largest(s[c], mx4);
      shift(max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * sl, first);
      const f32x2 ml2 = pack2(-m, -m);
      f32x2 sum[2] = {pack2(l, 0.0f), 0};
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t pk[16];
        probs(s[c], sum, ml2, pk);
        tmem_st_32x32b_x16(ts + 16 * c, pk);
      }
      close(sum);
    };
    // The block on the diagonal, where a row sees the columns up to its own: 32 columns at a
    // time, up to the warp's rows'.  (Rolled, and S read twice: with selections for every column
    // among the code of all blocks the others lost what these gained.)
    auto diagonal = [&](uint32_t ts, bool first) {
      uint32_t s[32];
      auto load = [&](int c) {
        tmem_ld_32x32b_x32(ts + 32 * c, s);
        tmem_ld_wait();
        if (c == quad) {
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (i > lane) s[i] = 0xFF800000u;
        }
      };
      float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll 1
      for (int c = 0; c <= quad; ++c) {
        load(c);
        largest(s, mx4);
      }
      shift(max3(fmaxf(mx4[0], mx4[1]), mx4[2], mx4[3]) * sl, first);
      const f32x2 ml2 = pack2(-m, -m);
      f32x2 sum[2] = {pack2(l, 0.0f), 0};
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        uint32_t pk[16] = {};
        if (c <= quad) {
          load(c);
          probs(s, sum, ml2, pk);
        }
        tmem_st_32x32b_x16(ts + 16 * c, pk);
      }
      close(sum);
    };
    uint32_t ni = 0;  // items of this tile so far
    Ring<4> from;
    FwdItem x;
    while (take(queue, from, wait, lane, x)) {
      const int b0 = fwd_blocks(p, x, 0), b1 = fwd_blocks(p, x, 1), blocks = t ? b1 : b0;
      m = l = 0.0f;
      for (int j = 0; j < blocks; ++j, ++ns) {
        // (blocks come as tile 0's, tile 1's, tile 0's, ... while either has some)
        const int n = n0 + j + (t ? min(j + 1, b0) : min(j, b1)), buf = n % S::NS;
        const uint32_t ts = tmem + lanes + buf * 128;
        wait(&s_full[4 * t + (ns & 3)], (ns >> 2) & 1u);
        tc_fence_after();
        if (j < blocks - 1)
          block(ts, j == 0);
        else
          diagonal(ts, j == 0);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_full[buf]);
      }
      n0 += b0 + b1;
      if (blocks == 0) continue;
      if (ni++ > 0) wait(&o_free[t], ni & 1u);  // the sums of the item before are read
      reinterpret_cast<float2*>(smem + S::SUM_OFF)[128 * t + row] = make_float2(m, l);
      __syncwarp();
      if (lane == 0) mbar_arrive(&sum_full[t]);
    }
    if (wait.late) record_timeout(p.status);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// ---------------------------------------------------------------------------
// Backward on the tensor cores, as two kernels of one shape: dQ over tiles of
// 128 queries, dK and dV over tiles of 128 keys.  Each forms the scores and dP
// anew: two products more than one kernel would need, but every sum is taken in one
// place, in one order (no atomics on dQ, and the q heads of a group add into the
// same accumulators), and dQ never exists in fp32 in memory.
//
//   resident tiles  R0, R1 (128 rows):   Q, dO       |  K, V
//   streamed blocks S0, S1 (W rows):     K, V        |  Q, dO
//   X = R0 S0^T, Y = R1 S1^T             S, dP       |  S^T - lse / scale, dP^T - delta  (tensor memory)
//   p = exp2(scale log2 e X - lse log2 e), ds = p (Y - delta)  |  p = exp2(scale log2 e X), ds = p Y
//   dq += ds S0 (= K)                                |  dv += p S1 (= dO), dk += ds S0 (= Q)
//
// p and ds go back to tensor memory as bf16, over X (so that Y's columns are free once
// read), and are the A operands of the last products from there; the streamed block serves both as
// B^T of the first and as B of the last.
//
//   warps 0-3, 4-7  p and ds: a row to a thread, half of a step's columns to a group
//   warp 8          copies
//   warps 9, 10     the products X, and Y
//   warp 11         the accumulations
//   warps 12-15     the items: what the math warps are to know of the next, its delta, and
//                   the outputs of the one before
//
// lse and delta belong to lanes in the dQ kernel, which takes delta from do and o and writes both for the
// other kernel, whose columns they belong to: as three bf16 each (24 bits), which a product of 16 columns with
// ones adds to X and Y.  Each has a row of its own, so that a delta that is not finite meets no zero in X
// (dv does not depend on it).  Read from shared memory instead, 8 bytes for each of a thread's columns, they were
// as much traffic there as the operands (dk and dv of 8 x 2048, 32 heads, in a form before this one: 286 us, and
// 254 so).
//
// W is 128 for dim 64: with steps of 64 rows the warps' waits alone took 635 clk a step of
// 980.  For dim 128 shared and tensor memory hold 64.
//
// 8 x 2048, 32 heads of 64: dq 195 us, dk and dv 222 (215 with lse and delta in one row, of which the stamps
// that follow are).  A step of dk and dv (128 x 128) takes 1530 clk, and its
// products keep the tensor cores for 1410 of them (1150 if nothing else used shared memory, which their operands
// take at the full 128 bytes a clk); one of dq 1400, 1100 of them products.  Dim 128 (6063 tokens, 16 heads
// over 2): 73 and 109 us, a step of 64 columns 1130 and 1600 clk, products 1020 and 1380 (64 columns take 48 clk
// for 16 of dim, 128 take 64).  Measured and left: X and Y freed once read and p and ds in columns of their
// own (dk and dv 250 us, beside 214), Y in a half for each group (269, beside 254), four groups for p and ds, resident tiles in
// tensor memory, heads in sets that fit the L2 (2 % of this case, and 3 % lost to uneven ends of others).
// ---------------------------------------------------------------------------
template <int D, bool KV>
struct BwdSmem {
  static constexpr int ATOMS = D / 64;
  static constexpr int RES = ATOMS * kAtomBytes;        // one resident tile
  static constexpr int W = D == 64 ? 128 : 64;          // rows of a streamed block, columns of a step
  static constexpr int ATOM = W * kRowBytes;            // a block's 64 columns of dim
  static constexpr int BLK = ATOMS * ATOM;              // one streamed block
  static constexpr int NR = 2;                          // resident tiles
  static constexpr int RBUF = D == 64 ? 2 : 1;          // buffers of them
  static constexpr int RING = 4;                        // stages of two blocks
  static constexpr int RING_OFF = RBUF * NR * RES;
  // KV: the stages' lse and delta, ones, zeros; dQ: lse and delta of two items
  static constexpr int STAT_OFF = RING_OFF + RING * 2 * BLK;
  static constexpr int STAT = W * 16;  // lse, or delta, of a stage
  static constexpr int ONES_OFF = STAT_OFF + RING * 2 * STAT;
  static constexpr int ZERO_OFF = ONES_OFF + 2048;
  static constexpr int OUT_OFF = KV ? ZERO_OFF + 2048 : STAT_OFF + 2 * 2 * 512;
  static constexpr int INFO_OFF = OUT_OFF + 4 * 2048;  // what the math warps know of two items
  static constexpr int BAR_OFF = INFO_OFF + 2 * 32;
  static constexpr int BYTES = BAR_OFF + 384 + 1024;
  static_assert(BYTES <= 232448, "shared memory per CTA");
  // Tensor memory: W columns for X and for Y of some steps, and the accumulators, two sets of
  // them where there is room (dq of dim 64).  A step's X is held until its
  // accumulation, which also empties its stage: RING >= NX.  Its Y only until it is read.
  static constexpr int ACC = KV ? 2 * D : D;
  static constexpr int NXY = (512 - ACC) / W < 6 ? (512 - ACC) / W : 6;
  static constexpr int NX = (NXY + 1) / 2, NY = NXY / 2;
  static constexpr uint32_t Y_COL = NX * W, ACC_COL = NXY * W;
  static constexpr int NA = (512 - NXY * W) / ACC < 2 ? 1 : 2;
  static_assert(NX >= 2 && NY >= 1 && RING >= NX, "tensor memory");
  static_assert((2 * RING + 2 * RBUF + 2 * NX + 2 * NY + 2 * NA + 2 + 3) * 8 + 4 <= 384, "barriers");
  static constexpr uint32_t STAGE_TX = 2 * BLK + (KV ? 2 * STAT : 0);
};

struct BwdParams {
  dqt_attn_layout_t L;
  const dqt_attn_tile_t* tiles;
  int items;
  Div per;    // items to a table entry
  Div split;  // KV: parts of an item's steps (1: none)
  Div group;  // q heads to a k and v head
  float* part;
  float scale, inv_scale, scale_log2;
  const float* lse;      // dQ
  const uint16_t* o;     // dQ
  uint4* stat;           // [2, heads, tiles * 128], lse and delta: dQ writes, KV reads
  uint16_t* out0;  // dq, or dv
  uint16_t* out1;  // dk
  uint64_t wait_ns;
  unsigned int* status;
};

// An item of either kernel: its tile, its head (of q, or of k and v), its blocks of W
// streamed rows [b0, b1) per q head; its steps, of which the first is block b of the
// group's q head h.
struct BwdItem {
  dqt_attn_tile_t t;
  int head, part, b0, b1, steps, b, h;
};
// Steps [from, to) of part i of n
__device__ __forceinline__ int2 steps_of(int steps, int i, int n) {
  return n == 1 ? make_int2(0, steps)
                : make_int2(static_cast<int>(static_cast<int64_t>(steps) * i / n),
                            static_cast<int>(static_cast<int64_t>(steps) * (i + 1) / n));
}
template <int W, bool KV>
__device__ __forceinline__ BwdItem bwd_item(const BwdParams& p, int it, const dqt_attn_tile_t& t) {
  BwdItem x;
  x.t = t;
  constexpr int LOG = W == 128 ? 7 : 6;
  const int j = it - p.per.of(it) * static_cast<int>(p.per.d);
  x.head = KV ? p.split.of(j) : j;
  x.part = KV ? j - x.head * static_cast<int>(p.split.d) : 0;
  x.b0 = KV ? t.row >> LOG : 0;
  x.b1 = ((KV ? t.len : min(t.row + 128, t.len)) + W - 1) >> LOG;
  const int blocks = x.b1 - x.b0;
  const int2 r = KV ? steps_of(blocks * static_cast<int>(p.group.d), x.part, static_cast<int>(p.split.d))
                    : make_int2(0, blocks);
  x.steps = r.y - r.x;
  x.h = r.x == 0 ? 0 : r.x / blocks;
  x.b = x.b0 + r.x - x.h * blocks;
  if (!tile_ok(t, p.L)) x.steps = 0;
  return x;
}

// First column of a part's sums for dv (w 0) or dk (w 1) of a head's tile, in units of 128 rows.
template <int D>
__device__ __forceinline__ int64_t part_at(const BwdParams& p, int w, int part, int head, int slot) {
  return (((static_cast<int64_t>(w) * p.split.d + part) * p.L.kv_heads + head) * p.L.tiles + slot) * D;
}

// dv and dk from the parts' sums, added up in order: a block per tile, head, output and
// 16 columns, a thread per row and eight of them (half of all columns to a
// thread left the loads waiting for one another: 47 us and not 23 at 6063 tokens, 2 heads of 128).
template <int D>
__global__ void __launch_bounds__(256) attn_bwd_join_kernel(const BwdParams p) {
  dep_wait();
  constexpr int W = BwdSmem<D, true>::W, CHUNKS = D / 16;
  const int it = blockIdx.x / (2 * CHUNKS), w = blockIdx.x / CHUNKS & 1;
  const dqt_attn_tile_t t = p.tiles[it / p.L.kv_heads];
  const int head = it % p.L.kv_heads, row = threadIdx.x & 127;
  const int c = blockIdx.x % CHUNKS * 16 + (threadIdx.x >> 7) * 8;
  if (!tile_ok(t, p.L) || t.row + row >= t.len) return;
  const int steps = ((t.len + W - 1) / W - t.row / W) * static_cast<int>(p.group.d);
  float v[8] = {};
  const int split = static_cast<int>(p.split.d);
#pragma unroll 4
  for (int i = 0; i < split; ++i) {
    const int2 r = steps_of(steps, i, split);
    if (r.x == r.y) continue;  // an empty part wrote nothing
    const float* from = p.part + (part_at<D>(p, w, i, head, t.slot) + c) * 128 + row;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] += __ldcs(from + e * 128);
  }
  const float f = w ? p.scale : 1.0f;
  uint32_t o[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) o[e] = pack_bf16x2(v[2 * e] * f, v[2 * e + 1] * f);
  uint16_t* out = (w ? p.out1 : p.out0) +
                  ((static_cast<int64_t>(t.start) + t.row + row) * p.L.kv_heads + head) * D + c;
  *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
}

template <int D, bool KV>
__global__ void __launch_bounds__(kThreads, 1)
    attn_bwd_kernel(const __grid_constant__ CUtensorMap mr0, const __grid_constant__ CUtensorMap mr1,
                    const __grid_constant__ CUtensorMap ms0, const __grid_constant__ CUtensorMap ms1,
                    const __grid_constant__ BwdParams p) {
  using S = BwdSmem<D, KV>;
  constexpr uint32_t kIdescXY = idesc_bf16(128, S::W, false, false);
  constexpr uint32_t kIdescAcc = idesc_bf16(128, D, false, true);

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = align1024(smem_raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::BAR_OFF);
  uint64_t* empty = full + S::RING;
  uint64_t* r_full = empty + S::RING;
  uint64_t* r_empty = r_full + S::RBUF;
  uint64_t* x_full = r_empty + S::RBUF;  // [NX]
  uint64_t* pd_full = x_full + S::NX;    // [NX]: p and ds in X's place
  uint64_t* y_full = pd_full + S::NX;    // [NY]
  uint64_t* y_free = y_full + S::NY;     // [NY]: read
  uint64_t* acc_full = y_free + S::NY;   // [NA]
  uint64_t* acc_empty = acc_full + S::NA;
  uint64_t* info_full = acc_empty + S::NA;  // [2]
  uint64_t* drain = info_full + 2;          // [3]
  uint32_t* slot = reinterpret_cast<uint32_t*>(drain + 3);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < S::RING; ++i) {
      mbar_init(&full[i], 1);
      mbar_init(&empty[i], 1);
    }
    for (int i = 0; i < S::RBUF; ++i) {
      mbar_init(&r_full[i], 1);
      mbar_init(&r_empty[i], KV ? 2 : 2 + 4);  // the issuing warps; the items' warps for delta
    }
    for (int i = 0; i < S::NX; ++i) {
      mbar_init(&x_full[i], 1);
      mbar_init(&pd_full[i], 8);
    }
    for (int i = 0; i < S::NY; ++i) {
      mbar_init(&y_full[i], 1);
      mbar_init(&y_free[i], 8);
    }
    for (int i = 0; i < S::NA; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], 4);
    }
    for (int i = 0; i < 2; ++i) mbar_init(&info_full[i], 4);
    for (int i = 0; i < 3; ++i) mbar_init(&drain[i], 1);
    fence_mbarrier_init();
    tma_prefetch_desc(&mr0);
    tma_prefetch_desc(&mr1);
    tma_prefetch_desc(&ms0);
    tma_prefetch_desc(&ms1);
  }
  if (KV && threadIdx.x < 128) {
    uint4* at = reinterpret_cast<uint4*>(smem + S::ONES_OFF) + threadIdx.x;
    at[0] = make_uint4(0x3F803F80u, 0x00003F80u, 0, 0);
    at[128] = make_uint4(0, 0, 0, 0);
    fence_async_shared();
  }
  if (warp == 9) tmem_alloc(slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *slot;
  dep_wait();
  dep_trigger();

  if (warp >= 12) {
    regs_dec<BwdRegs::kItems>();
    // ---------------- the items: lse and delta, outputs ----------------
    const int row = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    const int64_t heads = KV ? p.L.kv_heads : p.L.heads;
    uint4* obuf = reinterpret_cast<uint4*>(smem + S::OUT_OFF) + quad * 128;
    Waits wait{p.wait_ns};
    Ring<2> info;
    Ring<S::RBUF> res;
    Ring<S::NA> acc;
    BwdItem done;  // the item whose outputs are to be written
    done.steps = 0;
    dqt_attn_tile_t ahead = tile_of(p.tiles, deal(0), p.items, p.per);
    // dQ: the lse of this lane's row of an item's tile
    auto read_lse = [&](int it, const dqt_attn_tile_t& t) {
      return !KV && it < p.items && tile_ok(t, p.L) && t.row + row < t.len
                 ? p.lse[(it - p.per.of(it) * static_cast<int>(p.per.d)) * p.L.tokens + t.start + t.row + row]
                 : 0.0f;
    };
    float lse_ahead = read_lse(deal(0), ahead);
    for (int r = 0;; ++r) {
      const bool more = deal(r) < p.items;  // (a last round says that there are no more)
      BwdItem x = bwd_item<S::W, KV>(p, deal(r), ahead);
      const float lse = lse_ahead;
      if (more) {
        ahead = tile_of(p.tiles, deal(r + 1), p.items, p.per);
        lse_ahead = read_lse(deal(r + 1), ahead);
        if (x.steps == 0) continue;
      } else {
        x.steps = 0;
      }
      // The math warps are done with the item before the last one, whose outputs are
      // written: its place is free.
      int4* to = reinterpret_cast<int4*>(smem + S::INFO_OFF) + 2 * info.i;
      if (threadIdx.x == 384) {
        to[0] = make_int4(x.t.row, x.t.len, x.steps, x.b);
        to[1] = make_int4(x.b0, x.b1, 0, 0);
      }
      if (!KV && more) {
        // delta = do . o of this lane's row, do from the resident tile (16-byte pieces of a
        // row of 64 columns stand at piece ^ (row % 8): the swizzle of the copies)
        const bool in = x.t.row + row < x.t.len;
        uint4 ov[8];
        const uint4* o = reinterpret_cast<const uint4*>(
            p.o + ((static_cast<int64_t>(x.t.start) + x.t.row + row) * p.L.heads + x.head) * D);
#pragma unroll
        for (int k = 0; k < 8; ++k) ov[k] = in ? o[k] : make_uint4(0, 0, 0, 0);
        wait(&r_full[res.i], res.ph);
        const uint8_t* tile = smem + (S::NR * res.i + 1) * S::RES + row * kRowBytes;
        f32x2 d[2] = {};
#pragma unroll
        for (int h = 0; h < S::ATOMS; ++h) {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const uint4 u = *reinterpret_cast<const uint4*>(tile + h * kAtomBytes + ((k ^ (row & 7)) * 16));
            d[0] = dot2(u.x, ov[k].x, d[0]);
            d[1] = dot2(u.y, ov[k].y, d[1]);
            d[0] = dot2(u.z, ov[k].z, d[0]);
            d[1] = dot2(u.w, ov[k].w, d[1]);
            if (h + 1 < S::ATOMS) ov[k] = in ? o[8 + k] : make_uint4(0, 0, 0, 0);
          }
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&r_empty[res.i]);
        res.next();
        const float2 sum = unpack2(add2(d[0], d[1]));
        const float nd = in ? -(sum.x + sum.y) : 0.0f;
        float* stat = reinterpret_cast<float*>(smem + S::STAT_OFF) + info.i * 256 + row;
        stat[0] = -lse * kLog2e;
        stat[128] = nd;
        uint32_t a[3], e[3];
        pieces(-lse * p.inv_scale, a);
        pieces(nd, e);
        const int64_t of_row = (static_cast<int64_t>(x.head) * p.L.tiles + x.t.slot) * 128 + row;
        p.stat[of_row] = make_uint4(a[0] | a[1] << 16, a[2], 0, 0);
        p.stat[p.L.heads * p.L.tiles * 128 + of_row] = make_uint4(e[0] | e[1] << 16, e[2], 0, 0);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&info_full[info.i]);
      info.next();
      if (done.steps > 0) {
        wait(&acc_full[acc.i], acc.ph);
        tc_fence_after();
        const int io = done.t.row + row;
        const uint32_t from = tmem + lanes + S::ACC_COL + acc.i * S::ACC;
        auto freed = [&] {
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&acc_empty[acc.i]);
          acc.next();
        };
        if (KV && p.split.d > 1) {
          // a part's sums, columns of 128 rows: attn_bwd_join_kernel adds the parts up
#pragma unroll 1
          for (int c = 0; c < S::ACC; c += 32) {
            uint32_t o[32];
            tmem_ld_32x32b_x32(from + c, o);
            tmem_ld_wait();
            if (c + 32 == S::ACC) freed();
            float* to = p.part + (part_at<D>(p, c / D, done.part, done.head, done.t.slot) + c % D) * 128 + row;
#pragma unroll
            for (int e = 0; e < 32; ++e) to[e * 128] = __uint_as_float(o[e]);
          }
        } else {
          // 64 columns at once, so that the accumulators are soon free
#pragma unroll
          for (int c = 0; c < S::ACC; c += 64) {
            const int w = c / D;  // dv, dk
            uint32_t o[2][32];
            tmem_ld_32x32b_x32(from + c, o[0]);
            tmem_ld_32x32b_x32(from + c + 32, o[1]);
            tmem_ld_wait();
            if (c + 64 == S::ACC) freed();
            uint16_t* out = (KV && w ? p.out1 : p.out0) +
                            ((static_cast<int64_t>(done.t.start) + io) * heads + done.head) * D + c % D;
#pragma unroll
            for (int e = 0; e < 2; ++e)
              store_rows(obuf, o[e], KV && w == 0 ? 1.0f : p.scale, out + 32 * e, heads * D,
                         done.t.len - io + lane, lane);
          }
        }
      }
      if (!more) break;
      done = x;
    }
    if (wait.late) record_timeout(p.status);
  } else if (warp >= 8) {
    regs_dec<BwdRegs::kFeed>();
    if (warp == 8) {
      if (lane == 0) {
        // ---------------- copies ----------------
        int n = 0, nr = 0;  // stages and resident buffers filled so far
        bool ok = true;
        dqt_attn_tile_t ahead = tile_of(p.tiles, deal(0), p.items, p.per);
        for (int r = 0; ok && deal(r) < p.items; ++r) {
          const BwdItem x = bwd_item<S::W, KV>(p, deal(r), ahead);
          ahead = tile_of(p.tiles, deal(r + 1), p.items, p.per);
          if (x.steps == 0) continue;
          const int rb = nr % S::RBUF;
          if (nr >= S::RBUF && !buffer_wait(&r_empty[rb], &r_full[rb], (nr / S::RBUF - 1) & 1u, p.wait_ns)) {
            ok = false;
            break;
          }
          mbar_arrive_expect_tx(&r_full[rb], S::NR * S::RES);
          for (int m = 0; m < S::NR; ++m)
            for (int a = 0; a < S::ATOMS; ++a)
              tma_load_3d(m ? &mr1 : &mr0, &r_full[rb],
                          smem + (S::NR * rb + m) * S::RES + a * kAtomBytes, 64 * a, x.head,
                          x.t.start + x.t.row);
          ++nr;
          int b = x.b, h = KV ? x.head * static_cast<int>(p.group.d) + x.h : p.group.of(x.head);
          for (int st = 0; st < x.steps; ++st, ++n) {
            const int s = n % S::RING;
            if (n >= S::RING && !buffer_wait(&empty[s], &full[s], (n / S::RING - 1) & 1u, p.wait_ns)) {
              ok = false;
              break;
            }
            mbar_arrive_expect_tx(&full[s], S::STAGE_TX);
            for (int m = 0; m < 2; ++m)
              for (int a = 0; a < S::ATOMS; ++a)
                tma_load_3d(m ? &ms1 : &ms0, &full[s],
                            smem + S::RING_OFF + (2 * s + m) * S::BLK + a * S::ATOM, 64 * a, h,
                            x.t.start + S::W * b);
            if (KV) {
              // the block's rows in the slots of its document
              const int64_t at = static_cast<int64_t>(h) * p.L.tiles * 128 +
                                 (static_cast<int64_t>(x.t.slot) - x.t.row / 128) * 128 + S::W * b;
              for (int m = 0; m < 2; ++m)
                bulk_load(smem + S::STAT_OFF + (2 * s + m) * S::STAT, p.stat + m * p.L.heads * p.L.tiles * 128 + at,
                          S::STAT, &full[s]);
            }
            if (++b == x.b1) {
              b = x.b0;
              ++h;
            }
          }
        }
        if (!ok) record_timeout(p.status);
        // the copies in flight land before the CTA exits, whoever gave up
        for (int i = n > S::RING ? n - S::RING : 0; i < n; ++i)
          mbar_wait(&full[i % S::RING], (i / S::RING) & 1u, kDrainNs);
        for (int i = nr > S::RBUF ? nr - S::RBUF : 0; i < nr; ++i)
          mbar_wait(&r_full[i % S::RBUF], (i / S::RBUF) & 1u, kDrainNs);
      }
    } else if (warp < 11) {
      // ---------------- X, and Y ----------------
      const int m = warp - 9, cols = m ? S::NY : S::NX;
      const uint64_t desc = sdesc_sw128(0, 16, 1024);
      const uint32_t hi = static_cast<uint32_t>(desc >> 32), lo = static_cast<uint32_t>(desc);
      const uint32_t base = smem_u32(smem) + m * S::RES, ring = smem_u32(smem) + S::RING_OFF + m * S::BLK;
      const uint32_t d0 = tmem + (m ? S::Y_COL : 0);
      uint64_t* done_bar = m ? y_full : x_full;
      const uint64_t ones = sdesc_pieces(smem_u32(smem) + S::ONES_OFF, smem_u32(smem) + S::ZERO_OFF);
      Waits wait{p.wait_ns};
      Ring<S::RING> stage, before;  // the step's stage, and that of the step whose columns X takes
      Ring<S::RBUF> res;
      int col = 0;
      uint32_t ph = 0;
      bool reused = false;
      dqt_attn_tile_t ahead = tile_of(p.tiles, deal(0), p.items, p.per);
      for (int r = 0; deal(r) < p.items; ++r) {
        const BwdItem x = bwd_item<S::W, KV>(p, deal(r), ahead);
        ahead = tile_of(p.tiles, deal(r + 1), p.items, p.per);
        if (x.steps == 0) continue;
        wait(&r_full[res.i], res.ph);
        for (int st = 0; st < x.steps; ++st) {
          // X's columns are free with the accumulation of NX steps before, which also empties
          // that step's stage; Y's once they are read
          if (reused)
            wait(&full[stage.i], stage.ph, m ? &y_free[col] : &empty[before.i], m ? ph ^ 1u : before.ph);
          else
            wait(&full[stage.i], stage.ph);
          tc_fence_after();
          const uint32_t d = d0 + col * S::W, s0 = ring + 2 * stage.i * S::BLK;
          const uint32_t r0 = base + S::NR * res.i * S::RES;
          if (elect_one()) {
#pragma unroll
            for (int k = 0; k < D / 16; ++k)
              umma_bf16(d, desc_at(hi, lo, r0 + (k / 4) * kAtomBytes + (k % 4) * 32),
                        desc_at(hi, lo, s0 + (k / 4) * S::ATOM + (k % 4) * 32), kIdescXY,
                        k > 0 ? 1u : 0u);
            if (KV)
              umma_bf16(d, ones,
                        sdesc_pieces(smem_u32(smem) + S::STAT_OFF + (2 * stage.i + m) * S::STAT,
                                     smem_u32(smem) + S::ZERO_OFF),
                        kIdescXY, 1u);
            umma_commit(&done_bar[col]);
            if (st == x.steps - 1) umma_commit(&r_empty[res.i]);
          }
          __syncwarp();
          stage.next();
          if (reused) before.next();
          if (++col == cols) {
            col = 0;
            ph ^= 1u;
            reused = true;
          }
        }
        res.next();
      }
      if (wait.late) record_timeout(p.status);
      // every product issued is done before tensor memory is freed
      if (elect_one()) umma_commit(&drain[m]);
      mbar_wait(&drain[m], 0, kDrainNs);
    } else {
      // ---------------- the accumulators ----------------
      const uint64_t desc = sdesc_sw128(0, S::ATOM, 1024);
      const uint32_t hi = static_cast<uint32_t>(desc >> 32), lo = static_cast<uint32_t>(desc);
      const uint32_t ring = smem_u32(smem) + S::RING_OFF;
      Waits wait{p.wait_ns};
      Ring<S::NX> col;
      Ring<S::RING> stage;
      Ring<S::NA> acc;
      int items = 0;
      dqt_attn_tile_t ahead = tile_of(p.tiles, deal(0), p.items, p.per);
      for (int r = 0; deal(r) < p.items; ++r) {
        const BwdItem x = bwd_item<S::W, KV>(p, deal(r), ahead);
        ahead = tile_of(p.tiles, deal(r + 1), p.items, p.per);
        if (x.steps == 0) continue;
        if (items >= S::NA) wait(&acc_empty[acc.i], acc.ph ^ 1u);
        ++items;
        const uint32_t d0 = tmem + S::ACC_COL + acc.i * S::ACC;
        int b = x.b;
        for (int st = 0; st < x.steps; ++st) {
          const int rows = min(S::W, x.t.len - S::W * b), steps = (rows + 15) / 16;
          if (++b == x.b1) b = x.b0;
          wait(&pd_full[col.i], col.ph);
          if (rows % 16) {
            // the block's rows beyond the document: p and ds are 0 there, but what
            // stands there may not be finite
            for (int a = 0; a < (KV ? 2 : 1) * S::ATOMS; ++a)
              zero_rows(smem + S::RING_OFF + 2 * stage.i * S::BLK + a * S::ATOM, rows, 16 * steps, lane);
            fence_async_shared();
            __syncwarp();
          }
          tc_fence_after();
          const uint32_t s0 = ring + 2 * stage.i * S::BLK, s1 = s0 + S::BLK, pc = tmem + col.i * S::W;
          if (elect_one()) {
            // either group's p and ds stand side by side in its half of X's columns
#pragma unroll
            for (int k = 0; k < S::W / 16; ++k)
              if (k < steps) {
                constexpr int K = S::W / 32;  // products of a group's half
                const uint32_t on = k > 0 || st > 0 ? 1u : 0u, a = pc + (k / K) * (S::W / 2) + 8 * (k % K);
                if (KV) umma_bf16_ts(d0, a, desc_at(hi, lo, s1 + 2048 * k), kIdescAcc, on);
                umma_bf16_ts(d0 + (KV ? D : 0), a + S::W / 4, desc_at(hi, lo, s0 + 2048 * k), kIdescAcc, on);
              }
            umma_commit(&empty[stage.i]);
            if (st == x.steps - 1) umma_commit(&acc_full[acc.i]);
          }
          __syncwarp();
          stage.next();
          col.next();
        }
        acc.next();
      }
      if (wait.late) record_timeout(p.status);
      if (elect_one()) umma_commit(&drain[2]);
      mbar_wait(&drain[2], 0, kDrainNs);
    }
  } else {
    regs_inc<BwdRegs::kMath>();
    // ---------------- p and ds ----------------
    const int g = warp >> 2, row = threadIdx.x & 127, quad = warp & 3;
    const uint32_t lanes = static_cast<uint32_t>(quad * 32) << 16;
    const f32x2 sl2 = pack2(p.scale_log2, p.scale_log2);
    Waits wait{p.wait_ns};
    constexpr int C = S::W / 2;  // this group's columns of a step
    Ring<2> info;
    Ring<S::NX> xcol;
    Ring<S::NY> ycol;
    while (true) {
      wait(&info_full[info.i], info.ph);
      // (what is there would be no item)
      if (__any_sync(~0u, wait.late)) break;
      const int4* from = reinterpret_cast<const int4*>(smem + S::INFO_OFF) + 2 * info.i;
      const int4 it = from[0], bl = from[1];
      const int t_row = it.x, t_len = it.y, steps = it.z, b0 = bl.x, b1 = bl.y;
      if (steps == 0) break;
      const float* stat = reinterpret_cast<const float*>(smem + S::STAT_OFF) + info.i * 256 + row;
      const float nl = KV ? 0.0f : stat[0], nd = KV ? 0.0f : stat[128];
      info.next();
      const int i = t_row + row;  // this lane's row in the document
      int b = it.w;
      for (int st = 0; st < steps; ++st) {
        wait(&x_full[xcol.i], xcol.ph, &y_full[ycol.i], ycol.ph);
        tc_fence_after();
        // columns [lo, hi) of the group's count: queries from this key on, in the
        // document | keys up to this query
        const int c0 = S::W * b + g * C;
        const int lo = KV ? i - c0 : 0, hi = KV ? t_len - c0 : i - c0 + 1;
        const bool masked = KV ? c0 < t_row + 128 || c0 + C > t_len : c0 + C > t_row;
        const uint32_t tx = tmem + lanes + xcol.i * S::W + g * C;
        const uint32_t ty = tmem + lanes + S::Y_COL + ycol.i * S::W + g * C;
        const f32x2 nl2 = pack2(nl, nl), nd2 = pack2(nd, nd);
        uint32_t X[C / 32][32], Y[C / 32][32], P[C / 32][16], G[C / 32][16];
#pragma unroll
        for (int h = 0; h < C / 32; ++h) {
          tmem_ld_32x32b_x32(tx + 32 * h, X[h]);
          tmem_ld_32x32b_x32(ty + 32 * h, Y[h]);
        }
        tmem_ld_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&y_free[ycol.i]);
#pragma unroll
        for (int c = 0; c < C; c += 2) {
          const f32x2 xv = f2(X[c / 32][c % 32], X[c / 32][c % 32 + 1]);
          const f32x2 yv = f2(Y[c / 32][c % 32], Y[c / 32][c % 32 + 1]);
          // (KV: lse and delta are in X and Y)
          const f32x2 pp = exp2_approx2(KV ? mul2(xv, sl2) : fma2(xv, sl2, nl2));
          if (KV) P[c / 32][c % 32 / 2] = pack_bf16x2(pp);
          G[c / 32][c % 32 / 2] = pack_bf16x2(mul2(pp, KV ? yv : add2(yv, nd2)));
        }
        if (masked) {
          // (selected, not multiplied: what stands there may not be finite)
          const uint64_t in = first_bits(hi) & ~first_bits(lo);
#pragma unroll
          for (int c = 0; c < C; c += 4) {
            // the four columns' bits to the signs of four bytes, and these to halves of words
            const uint32_t four = static_cast<uint32_t>(in >> c) & 15u;
            const uint32_t bytes = four * 0x10204080u & 0x80808080u;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t keep = prmt(bytes, e ? 0xBBAAu : 0x9988u);
              if (KV) P[c / 32][c % 32 / 2 + e] &= keep;
              G[c / 32][c % 32 / 2 + e] &= keep;
            }
          }
        }
#pragma unroll
        for (int h = 0; h < C / 32; ++h) {
          if (KV) tmem_st_32x32b_x16(tx + 16 * h, P[h]);
          tmem_st_32x32b_x16(tx + C / 2 + 16 * h, G[h]);
        }
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&pd_full[xcol.i]);
        xcol.next();
        ycol.next();
        if (++b == b1) b = b0;
      }
    }
    if (wait.late) record_timeout(p.status);
  }

  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

// Shared memory and registers of a kernel, once per device and kernel: the
// groups' shares of the registers must not exceed what the block is launched with.
template <typename K>
bool ready(K kern, int smem, int regs, PerDevice& set) {
  int dev = 0, done = 0;
  return cudaGetDevice(&dev) == cudaSuccess && set.get(dev, done, [&](int& n) {
    n = 1;
    cudaFuncAttributes at;
    return cudaFuncGetAttributes(&at, kern) == cudaSuccess && at.numRegs >= regs &&
           cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) == cudaSuccess;
  });
}

unsigned ctas(int items) {
  const int sms = sm_count();
  return static_cast<unsigned>(items < sms ? items : sms);
}

template <int D>
int fwd(const uint16_t* q, const uint16_t* k, const uint16_t* v, const dqt_attn_layout_t& L,
        const dqt_attn_tile_t* tiles, float scale, uint16_t* o, float* lse, cudaStream_t stream) {
  auto kern = attn_fwd_kernel<D>;
  static PerDevice set;  // per template instance
  if (!ready(kern, FwdSmem<D>::BYTES, kRegsLaunch, set)) return 3;
  CUtensorMap mq, mk, mv;
  if (!encode_heads_map(&mq, q, L.tokens, L.heads, D, L.q_row, L.q_head, 128) ||
      !encode_heads_map(&mk, k, L.tokens, L.kv_heads, D, L.k_row, L.k_head, 128) ||
      !encode_heads_map(&mv, v, L.tokens, L.kv_heads, D, L.v_row, L.v_head, 128))
    return 3;
  FwdParams p = {};
  p.L = L;
  p.by_heads = (L.heads / L.kv_heads) % 2 == 0;
  p.tiles = p.by_heads ? tiles : tiles + 2 * L.tiles;
  p.pairs = Div(p.by_heads ? L.heads / 2 : L.heads);
  p.group = Div(L.heads / L.kv_heads);
  p.items = static_cast<int>((p.by_heads ? L.tiles : L.tiles256) * p.pairs.d);
  p.scale_log2 = scale * kLog2e;
  p.o = o;
  p.lse = lse;
  p.wait_ns = wait_limit_ns();
  p.status = status_word();
  if (!p.status) return 3;
  return launch_dep(kern, dim3(p.items), kThreads, FwdSmem<D>::BYTES, stream, mq, mk, mv, p);
}

// Parts that the keys' kernel cuts its items into.  An item is a tile of keys with all queries of its
// group that see it: where tiles or heads are few the longest item takes longer than an SM's share of all,
// and is cut into as many parts as it has shares (a part's sums go through memory, and
// attn_bwd_join_kernel).  The share takes one document as the longest, the others' tiles as half as long.
// Both kernels uncut, in 2, 3 and 4 parts, us: 6063 tokens in 4 documents, 16 heads over 2 of 128 (4
// shares) 376, 240, 194, 196; a document of 4096, 4 heads of 64 (2.3) 64, 58, 62, 63, 8 heads (1.2) 66, 76, 79,
// 83; 8 heads over 1 (9) 238, 142, and 73 in 8.
int bwd_split(const dqt_attn_layout_t& L) {
  const double longest = static_cast<double>((L.longest + 127) / 128), group = L.heads / L.kv_heads;
  const double rest = L.tiles > longest ? L.tiles - longest : 0.0;
  const double blocks = longest * (longest + 1) / 2 + rest * (longest + 3) / 4;
  const double shares = longest * group * sm_count() / (blocks * L.heads);
  const int n = static_cast<int>(shares < longest * group / 8 ? shares : longest * group / 8);
  return n < 1 ? 1 : n > 8 ? 8 : n;
}

template <int D>
int bwd(const uint16_t* dout, const uint16_t* q, const uint16_t* k, const uint16_t* v, const uint16_t* o,
        const float* lse, const dqt_attn_layout_t& L, const dqt_attn_tile_t* tiles, float scale,
        float* ws, uint16_t* dq, uint16_t* dk, uint16_t* dv, cudaStream_t stream) {
  auto kq = attn_bwd_kernel<D, false>;
  auto kkv = attn_bwd_kernel<D, true>;
  static PerDevice set_q, set_kv;  // per template instance
  if (!ready(kq, BwdSmem<D, false>::BYTES, kRegsLaunch, set_q) ||
      !ready(kkv, BwdSmem<D, true>::BYTES, kRegsLaunch, set_kv))
    return 3;
  constexpr int W = BwdSmem<D, true>::W;
  CUtensorMap rq, rdo, rk, rv, sq, sdo, sk, sv;  // boxes of 128 rows and of W
  auto maps = [&](CUtensorMap* big, CUtensorMap* small, const uint16_t* t, int64_t heads, int64_t row,
                  int64_t head) {
    return encode_heads_map(big, t, L.tokens, heads, D, row, head, 128) &&
           encode_heads_map(small, t, L.tokens, heads, D, row, head, W);
  };
  if (!maps(&rq, &sq, q, L.heads, L.q_row, L.q_head) || !maps(&rdo, &sdo, dout, L.heads, L.heads * D, D) ||
      !maps(&rk, &sk, k, L.kv_heads, L.k_row, L.k_head) || !maps(&rv, &sv, v, L.kv_heads, L.v_row, L.v_head))
    return 3;
  BwdParams p = {};
  p.L = L;
  p.tiles = tiles;
  p.items = static_cast<int>(L.tiles * L.heads);
  p.per = Div(L.heads);
  p.split = Div(1);
  p.group = Div(L.heads / L.kv_heads);
  p.scale = scale;
  // (below 1e-36 an lse over it might be above fp32: such scores are 0 to fp32)
  const float sc = scale > 1e-36f ? scale : 1e-36f;
  p.inv_scale = 1.0f / sc;
  p.scale_log2 = sc * kLog2e;
  p.lse = lse;
  p.o = o;
  p.stat = reinterpret_cast<uint4*>(ws);
  p.out0 = dq;
  p.wait_ns = wait_limit_ns();
  p.status = status_word();
  if (!p.status) return 3;
  const int rc = launch_dep(kq, dim3(ctas(p.items)), kThreads, BwdSmem<D, false>::BYTES, stream, rq, rdo, sk,
                            sv, p);
  if (rc) return rc;
  p.tiles = tiles + L.tiles;
  p.items = static_cast<int>(L.tiles * L.kv_heads);
  p.out0 = dv;
  p.out1 = dk;
  p.split = Div(bwd_split(L));
  p.per = Div(L.kv_heads * p.split.d);
  p.part = ws + L.heads * L.tiles * 1024;
  p.items *= static_cast<int>(p.split.d);
  const int rc2 = launch_dep(kkv, dim3(ctas(p.items)), kThreads, BwdSmem<D, true>::BYTES, stream, rk, rv, sq,
                             sdo, p);
  if (rc2 || p.split.d == 1) return rc2;
  return launch_dep(attn_bwd_join_kernel<D>, dim3(static_cast<unsigned>(L.tiles * L.kv_heads * 2 * (D / 16))),
                    256, 0, stream, p);
}

}  // namespace

int launch_attn_fwd(const uint16_t* q, const uint16_t* k, const uint16_t* v, const dqt_attn_layout_t& L,
                    const dqt_attn_tile_t* tiles, float scale, uint16_t* o, float* lse,
                    cudaStream_t stream) {
  return L.dim == 64 ? fwd<64>(q, k, v, L, tiles, scale, o, lse, stream)
                     : fwd<128>(q, k, v, L, tiles, scale, o, lse, stream);
}

size_t attn_bwd_ws(const dqt_attn_layout_t& L) {
  const int split = bwd_split(L);
  const size_t rows = static_cast<size_t>(L.tiles) * 128;
  return (rows * L.heads * 8 + (split > 1 ? rows * L.kv_heads * L.dim * 2 * split : 0)) * sizeof(float);
}

int launch_attn_bwd(const uint16_t* dout, const uint16_t* q, const uint16_t* k, const uint16_t* v,
                    const uint16_t* o, const float* lse, const dqt_attn_layout_t& L,
                    const dqt_attn_tile_t* tiles, float scale, void* ws, uint16_t* dq, uint16_t* dk,
                    uint16_t* dv, cudaStream_t stream) {
  float* w = static_cast<float*>(ws);
  return L.dim == 64 ? bwd<64>(dout, q, k, v, o, lse, L, tiles, scale, w, dq, dk, dv, stream)
                     : bwd<128>(dout, q, k, v, o, lse, L, tiles, scale, w, dq, dk, dv, stream);
}

}  // namespace dqt
