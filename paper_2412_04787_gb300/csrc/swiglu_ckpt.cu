// The SwiGLU gate of the decoder's MLP with an 8-bit checkpoint of its inputs.
//
//   forward   h = silu(g) u, and for each row and 128 columns of g and of u
//             amax = max |x|, scale = amax / 127, code = rint(127 x / amax)
//   backward  dg = dh u s (1 + g (1 - s)), du = dh g s with s = sigmoid(g),
//             g and u the values code * scale
//
// Both move 8.06 bytes per element and are bound by that (forward: 4 read, 2 + 2
// written; backward: 2 + 2 read, 4 written; 0.06 for the scales), next to some 35
// instructions.  Half a warp has the 128 columns that share a scale, a 16-byte
// vector of g and of u per lane, so that the maximum is four shuffles; a half-warp
// takes kItems blocks at once to keep that many loads in flight.  16384 x 5632: 117 us, 6.4 TB/s (94 %
// of a copy's), and backward 102 us, 7.3 TB/s; 3001 x 2744: 14 and 10.9 us.
//
// The checkpoint is the one rounding of g and u that the backward sees: half a scale, 1 / 254 of
// the block's largest.  h, dg and du are rounded to bf16 as g and u are; all between is fp32.
#include <cuda_bf16.h>

#include "dqt_internal.h"

namespace dqt {

namespace {

constexpr int kThreads = 256;
constexpr int kItems = 2;                              // blocks of 128 columns per half-warp
constexpr int kPerBlock = kThreads / 16 * kItems;      // and per thread block

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

__device__ __forceinline__ uint16_t bf16(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

// 1 / (1 + exp(-x)) for |x| < 80, to 2^-17 relative (x log2 e of 64 and more is off by 2^-17 in fp32),
// beside the 2^-9 of the results' rounding.  (Exactly rounded functions took the forward from 110 to
// 161 us at 16384 x 5632: it was bound by their instructions.)
__device__ __forceinline__ f32x2 sigmoid2(f32x2 x) {
  const f32x2 e = mul2(x, pack2(-1.4426950408889634f, -1.4426950408889634f));
  const float2 d = unpack2(add2(exp2_approx2(e), pack2(1.0f, 1.0f)));
  return pack2(rcp_approx(d.x), rcp_approx(d.y));
}

// Blocks with a g of 80 and more take these: for large g 1 - s loses what g multiplies, and for g < -87
// s leaves the normal numbers, but s u need not.  With e = exp(-|g| / 2), r = 1 / (1 + e^2):
// s = r, 1 - s = e^2 r above 0 and the other way round below, and e is multiplied in twice.
// One value at a time from memory, so that the other blocks' registers stay as few.
struct Far {
  float x, e, r;
  __device__ __forceinline__ explicit Far(float x_) : x(x_), e(expf(-0.5f * fabsf(x_))), r(1.0f / (1.0f + e * e)) {}
  // s x f
  __device__ __forceinline__ float silu(float f) const { return x < 0.0f ? x * e * r * f * e : x * r * f; }
  // s (1 + x (1 - s)) f d
  __device__ __forceinline__ float slope(float f, float d) const {
    return x < 0.0f ? (1.0f + x * r) * e * r * f * d * e : (1.0f + x * (e * e * r)) * r * f * d;
  }
};
constexpr uint32_t kFarBits = 0x42A0u;       // 80 as bf16
constexpr float kFarScale = 80.0f / 127.0f;  // and the scale of its block

// Blocks of 128 columns per row, and n / nb for n < 2^31 as a product (magic = ceil(2^(32 + s) / nb)
// with 2^s < nb <= 2^(s + 1), so magic nb - 2^(32 + s) < 2^(s + 1) and the quotient is exact).
struct Cols {
  int64_t F;
  uint32_t nb, magic, shift, items;
  __device__ __forceinline__ uint32_t row_of(uint32_t n) const {
    return nb == 1 ? n : __umulhi(n, magic) >> shift;
  }
};

Cols cols_of(int64_t M, int64_t F) {
  Cols c = {};
  c.F = F;
  c.nb = static_cast<uint32_t>((F + 127) / 128);
  c.items = static_cast<uint32_t>(M * c.nb);
  if (c.nb > 1) {
    while ((2ull << c.shift) < c.nb) ++c.shift;
    c.magic = static_cast<uint32_t>(((1ull << (32 + c.shift)) + c.nb - 1) / c.nb);
  }
  return c;
}

// Where a lane's eight columns are: row, block of columns, first column, and whether
// the item and the columns exist.
struct Place {
  uint32_t row, b;
  int col;
  bool item, in;
};
__device__ __forceinline__ Place place(const Cols& c, int k) {
  const int lane = threadIdx.x & 15;
  const uint32_t n = (blockIdx.x * kItems + k) * (kThreads / 16) + (threadIdx.x >> 4);
  Place p;
  p.item = n < c.items;
  p.row = c.row_of(n);
  p.b = n - p.row * c.nb;
  p.col = static_cast<int>(p.b * 128) + lane * 8;
  p.in = p.item && p.col < c.F;
  return p;
}

// The largest |x| of the half-warp as bf16 bits (0x7F80 and more: not finite).
__device__ __forceinline__ uint32_t amax_bits(const uint4& v) {
  // (as integers: without their signs bf16 values are ordered like their bits, NaN above all)
  uint32_t a = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu),
                        __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
#pragma unroll
  for (int off = 8; off > 0; off >>= 1) a = __vmaxu2(a, __shfl_xor_sync(~0u, a, off));
  return max(a & 0xFFFFu, a >> 16);
}

// The eight codes of v, and the scale.  127 x and amax have 15 and 8 significant
// bits, so that the quotient is a tie exactly or off one by more than 2^-10 relative to
// its last place: its product with the rounded reciprocal, corrected once by the exact remainder, rounds
// like the quotient itself.  (The power of two keeps 127 x and the reciprocal in range.)
__device__ __forceinline__ uint2 encode(const uint4& v, uint32_t bits, float* scale) {
  const float amax = __uint_as_float(bits << 16);
  if (bits >= 0x7F80u) {
    *scale = __uint_as_float(0x7FC00000u);
    return make_uint2(0, 0);
  }
  *scale = __fdiv_rn(amax, 127.0f);
  if (bits == 0) return make_uint2(0, 0);
  const float pw = amax < 1e-30f ? 18446744073709551616.0f : amax > 1e30f ? 5.421010862427522e-20f : 1.0f;
  const float a = amax * pw, r = __frcp_rn(a), f = 127.0f * pw;
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
  const f32x2 f2 = pack2(f, f), r2 = pack2(r, r), na = pack2(-a, -a);
  // + 1.5 2^23: the integer nearest (ties to even) in the low bits
  const f32x2 magic = pack2(12582912.0f, 12582912.0f);
  uint32_t c[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x2 x = mul2(pack2(bf16_lo(w[j]), bf16_hi(w[j])), f2);
    const f32x2 t = mul2(x, r2);
    const float2 q = unpack2(add2(fma2(fma2(t, na, x), r2, t), magic));
    c[2 * j] = __float_as_uint(q.x);
    c[2 * j + 1] = __float_as_uint(q.y);
  }
  return make_uint2(__byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410),
                    __byte_perm(__byte_perm(c[4], c[5], 0x0040), __byte_perm(c[6], c[7], 0x0040), 0x5410));
}

__global__ void __launch_bounds__(kThreads)
    swiglu_ckpt_kernel(const uint16_t* __restrict__ g, const uint16_t* __restrict__ u, const Cols c,
                       uint16_t* __restrict__ h, int8_t* __restrict__ codes, float* __restrict__ scales) {
  dep_wait();
  Place p[kItems];
  uint4 gv[kItems], uv[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    p[k] = place(c, k);
    gv[k] = uv[k] = make_uint4(0, 0, 0, 0);
    if (p[k].in) {
      const int64_t at = static_cast<int64_t>(p[k].row) * c.F + p[k].col;
      gv[k] = __ldcs(reinterpret_cast<const uint4*>(g + at));
      uv[k] = __ldcs(reinterpret_cast<const uint4*>(u + at));
    }
  }
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    const uint32_t ag = amax_bits(gv[k]), au = amax_bits(uv[k]);
    if (!p[k].item) continue;
    float sg, su;
    const uint2 cg = encode(gv[k], ag, &sg), cu = encode(uv[k], au, &su);
    const int64_t row = p[k].row;
    if ((threadIdx.x & 15) == 0) {
      scales[row * 2 * c.nb + p[k].b] = sg;
      scales[(row * 2 + 1) * c.nb + p[k].b] = su;
    }
    if (!p[k].in) continue;
    __stcs(reinterpret_cast<uint2*>(codes + row * 2 * c.F + p[k].col), cg);
    __stcs(reinterpret_cast<uint2*>(codes + (row * 2 + 1) * c.F + p[k].col), cu);
    if (ag >= kFarBits) {
      const int64_t at = row * c.F + p[k].col;
#pragma unroll 1
      for (int j = 0; j < 8; ++j) h[at + j] = bf16(Far(bf16_lo(g[at + j])).silu(bf16_lo(u[at + j])));
      continue;
    }
    const uint32_t gw[4] = {gv[k].x, gv[k].y, gv[k].z, gv[k].w}, uw[4] = {uv[k].x, uv[k].y, uv[k].z, uv[k].w};
    uint32_t o[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 x = pack2(bf16_lo(gw[j]), bf16_hi(gw[j]));
      const float2 y = unpack2(mul2(mul2(x, sigmoid2(x)), pack2(bf16_lo(uw[j]), bf16_hi(uw[j]))));
      o[j] = pack_bf16x2(y.x, y.y);
    }
    *reinterpret_cast<uint4*>(h + row * c.F + p[k].col) = make_uint4(o[0], o[1], o[2], o[3]);
  }
}

// Code j (a signed byte) of w as a float
__device__ __forceinline__ float code(const uint2& w, int j) {
  const uint32_t v = j < 4 ? w.x : w.y;
  return static_cast<float>(static_cast<int32_t>(v << (24 - 8 * (j & 3))) >> 24);
}

__global__ void __launch_bounds__(kThreads)
    swiglu_ckpt_bwd_kernel(const uint16_t* __restrict__ dh, const int8_t* __restrict__ codes,
                           const float* __restrict__ scales, const Cols c, uint16_t* __restrict__ dg,
                           uint16_t* __restrict__ du) {
  dep_wait();
  Place p[kItems];
  uint4 dv[kItems];
  uint2 cg[kItems], cu[kItems];
  float sg[kItems], su[kItems];
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    p[k] = place(c, k);
    if (p[k].in) {
      const int64_t row = p[k].row;
      dv[k] = __ldcs(reinterpret_cast<const uint4*>(dh + row * c.F + p[k].col));
      cg[k] = __ldcs(reinterpret_cast<const uint2*>(codes + row * 2 * c.F + p[k].col));
      cu[k] = __ldcs(reinterpret_cast<const uint2*>(codes + (row * 2 + 1) * c.F + p[k].col));
      sg[k] = __ldg(scales + row * 2 * c.nb + p[k].b);
      su[k] = __ldg(scales + (row * 2 + 1) * c.nb + p[k].b);
    }
  }
#pragma unroll
  for (int k = 0; k < kItems; ++k) {
    if (!p[k].in) continue;
    const int64_t at = static_cast<int64_t>(p[k].row) * c.F + p[k].col;
    if (!(sg[k] < kFarScale)) {
      const int8_t* cr = codes + at + p[k].row * c.F;
#pragma unroll 1
      for (int j = 0; j < 8; ++j) {
        const Far x(cr[j] * sg[k]);
        const float d = bf16_lo(dh[at + j]);
        dg[at + j] = bf16(x.slope(cr[c.F + j] * su[k], d));
        du[at + j] = bf16(x.silu(d));
      }
      continue;
    }
    const uint32_t dw[4] = {dv[k].x, dv[k].y, dv[k].z, dv[k].w};
    uint32_t og[4], ou[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x2 d = pack2(bf16_lo(dw[j]), bf16_hi(dw[j])), one = pack2(1.0f, 1.0f);
      const f32x2 x = mul2(pack2(code(cg[k], 2 * j), code(cg[k], 2 * j + 1)), pack2(sg[k], sg[k]));
      const f32x2 y = mul2(pack2(code(cu[k], 2 * j), code(cu[k], 2 * j + 1)), pack2(su[k], su[k]));
      const f32x2 s = sigmoid2(x), ds = mul2(d, s);
      const f32x2 rest = fma2(s, pack2(-1.0f, -1.0f), one);
      const float2 rg = unpack2(mul2(mul2(ds, y), fma2(x, rest, one))), ru = unpack2(mul2(ds, x));
      og[j] = pack_bf16x2(rg.x, rg.y);
      ou[j] = pack_bf16x2(ru.x, ru.y);
    }
    __stcs(reinterpret_cast<uint4*>(dg + at), make_uint4(og[0], og[1], og[2], og[3]));
    __stcs(reinterpret_cast<uint4*>(du + at), make_uint4(ou[0], ou[1], ou[2], ou[3]));
  }
}

unsigned blocks_of(const Cols& c) { return (c.items + kPerBlock - 1) / kPerBlock; }

}  // namespace

int launch_swiglu_ckpt(const uint16_t* g, const uint16_t* u, int64_t M, int64_t F, uint16_t* h,
                       int8_t* codes, float* scales, cudaStream_t stream) {
  const Cols c = cols_of(M, F);
  return launch_dep(swiglu_ckpt_kernel, dim3(blocks_of(c)), kThreads, 0, stream, g, u, c, h, codes, scales);
}

int launch_swiglu_ckpt_bwd(const uint16_t* dh, const int8_t* codes, const float* scales, int64_t M,
                           int64_t F, uint16_t* dg, uint16_t* du, cudaStream_t stream) {
  const Cols c = cols_of(M, F);
  return launch_dep(swiglu_ckpt_bwd_kernel, dim3(blocks_of(c)), kThreads, 0, stream, dh, codes, scales, c,
                    dg, du);
}

}  // namespace dqt
