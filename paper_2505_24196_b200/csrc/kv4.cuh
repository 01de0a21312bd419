// Key/value cache held in 4 bits (CLASP_FLAG_KV4): rows quantised into it, rows read back, attention over it.
//
// A block is 16 consecutive dims of one (position, kv head) row of K or V:
//   value = (c - 8) * s        c: 4 bits, 1..15;   s: one byte b, the half-precision number with the bits b << 7
// s is the smallest such number with 7 s >= max |x| (at most 896, then |x| > 6272 saturates), c - 8 = x / s to the
// nearest, ties to even.  Every step of that is exact in fp32 (7 s has 7 significant bits, a border (k + 1/2) s has 8, a
// correctly rounded quotient never reaches a border that x / s does not), so the bytes are a function of the row alone.  A
// value has at most 8 significant bits: exact in bf16 and in half precision.  Sixteen dims per scale: uniform steps of
// a seventh of a block's largest magnitude leave a Gaussian row 9.3 % of its standard deviation as error (4-bit floating point
// with the same scale byte 10.0 %).  A block that holds an infinity or NaN gets the byte 0xFF and reads back as NaN throughout; one
// whose largest magnitude is 2^-18 or less, half the smallest scale, becomes zeros.
//
// One layer's array (keys or values): codes [n_kv, capacity, hd / 2], low nibble first, then scale bytes
// [n_kv, capacity, hd / 16].  Head-major: what one CTA of the attention reads is contiguous.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gemm_tc.cuh"
#include "wide.cuh"

namespace clasp {
namespace kv4 {

using bf16 = __nv_bfloat16;
constexpr int BLOCK = 16;
constexpr uint32_t TOP_SCALE = 0xC6;   // 896: 72 s, which the code-to-half conversion needs, stays finite
constexpr uint32_t NAN_SCALE = 0xFF;
constexpr uint32_t INF_SCALE = 0xF8;   // half precision's infinity; never written here

// One layer's array as the kernels see it.
struct View {
  uint8_t* codes;
  uint8_t* scales;
  long long head_codes;    // bytes from one kv head to the next
  long long head_scales;
};
inline View view(void* p, int n_kv, int hd, long long capacity) {
  View v;
  v.codes = (uint8_t*)p;
  v.head_codes = capacity * (hd / 2);
  v.head_scales = capacity * (hd / BLOCK);
  v.scales = v.codes + v.head_codes * n_kv;
  return v;
}
inline size_t array_bytes(int n_kv, int hd, long long capacity) {
  return (size_t)n_kv * (size_t)capacity * (size_t)(hd / 2 + hd / BLOCK);
}

__device__ __forceinline__ float scale_of(uint32_t b) { return __half2float(__ushort_as_half((unsigned short)(b << 7))); }

// Sixteen values -> eight bytes of codes and the scale byte.
__device__ __forceinline__ uint2 quantise(float (&x)[BLOCK], uint32_t& byte) {
  float a = 0.f;
#pragma unroll
  for (int i = 0; i < BLOCK; ++i) asm("max.NaN.f32 %0, %0, %1;" : "+f"(a) : "f"(fabsf(x[i])));
  if (!(a <= 3.402823466e38f)) {         // an infinity or NaN
    byte = NAN_SCALE;
    return make_uint2(0x88888888u, 0x88888888u);
  }
  if (a > 6272.f) {
#pragma unroll
    for (int i = 0; i < BLOCK; ++i) x[i] = fminf(fmaxf(x[i], -6272.f), 6272.f);
    a = 6272.f;
  }
  // candidate: a / 7 cut to three mantissa bits (the product errs by less than one step of them); the next one if that is
  // too small
  const uint32_t h = (uint32_t)__half_as_ushort(__float2half_rz(a * (1.0f / 7.0f))) >> 7;
  byte = h + (7.f * scale_of(h) < a ? 1u : 0u);
  const float s = scale_of(byte);
  const float r = byte ? __frcp_rn(s) : 0.f;
  // x / s, correctly rounded: reciprocal to the nearest, then one residual step (Markstein's division); at most 7.  Added to
  // 1.5 x 2^23 + 8 its integer (ties to even) plus 8 is the sum's low bits; what stands above them is taken off the word at once.
  constexpr uint32_t BIAS = 0x4B400000u;
  uint32_t w[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < BLOCK; ++i) {
    const float q0 = x[i] * r;
    const float q = fmaf(fmaf(-q0, s, x[i]), r, q0) + 12582920.f;
    w[i >> 3] += (__float_as_uint(q) - BIAS) << ((i & 7) * 4);
  }
  return make_uint2(w[0], w[1]);
}

__device__ __forceinline__ void load16(const float* p, float (&x)[BLOCK]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 v = reinterpret_cast<const float4*>(p)[i];
    x[4 * i] = v.x; x[4 * i + 1] = v.y; x[4 * i + 2] = v.z; x[4 * i + 3] = v.w;
  }
}
__device__ __forceinline__ void store16(float* p, const float (&x)[BLOCK]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void store16(bf16* p, const float (&x)[BLOCK]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    reinterpret_cast<uint4*>(p)[i] = make_uint4(pack_bf16(x[8 * i], x[8 * i + 1]), pack_bf16(x[8 * i + 2], x[8 * i + 3]),
                                                pack_bf16(x[8 * i + 4], x[8 * i + 5]), pack_bf16(x[8 * i + 6], x[8 * i + 7]));
}

// ------------------------------------------------------------------ rows into the cache and back
// lanes of a 32-bit logic operation: (x & m) | o
__device__ __forceinline__ uint32_t and_or(uint32_t x, uint32_t m, uint32_t o) {
  uint32_t y;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(y) : "r"(x), "r"(m), "r"(o));
  return y;
}
// Two codes, the low four bits of each half, as bf16 values (c - 8) s: four low mantissa bits of 128 make 128 + c without an integer
// conversion, then (128 + c) s - 136 s in one step, exact (136 s has 8 significant bits).  s2, m136: s and -136 s in both halves.
__device__ __forceinline__ uint32_t nib_bf16(uint32_t w, uint32_t s2, uint32_t m136) {
  uint32_t y;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(y) : "r"(and_or(w, 0x000F000Fu, 0x43004300u)), "r"(s2), "r"(m136));
  return y;
}

// 32 bytes at a time where the addresses allow it (al32): two 16-byte accesses of a lane leave every sector half done twice.
__device__ __forceinline__ void ld32(const void* p, uint32_t (&w)[8], bool al32) {
  if (al32) {
    asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
  } else {
    const uint4 a = __ldg((const uint4*)p), b = __ldg((const uint4*)p + 1);
    w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
  }
}
__device__ __forceinline__ void st32(void* p, const uint32_t (&w)[8], bool al32) {
  if (al32) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]),
                 "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
  } else {
    ((uint4*)p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
    ((uint4*)p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
  }
}
__device__ __forceinline__ void load_block(const bf16* p, float (&x)[BLOCK], bool al32) {
  uint32_t w[8];
  ld32(p, w, al32);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void load_block(const float* p, float (&x)[BLOCK], bool al32) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[8];
    ld32(p + 8 * h, w, al32);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[8 * h + i] = __uint_as_float(w[i]);
  }
}
__device__ __forceinline__ void store_block(float* p, const float (&x)[BLOCK], bool al32) {
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = __float_as_uint(x[8 * h + i]);
    st32(p + 8 * h, w, al32);
  }
}

// A CTA takes one kv head of K or of V (blockIdx.y), a thread one block.  Neighbours take the blocks of a row, then of the next
// row: a warp's codes and scales lie side by side in the cache, whole sectors of both.
//
// Measured, bf16, eight heads of 128, write + read of 8192 rows together, us: 24.8 with the heads of a row side by side and 16-byte
// accesses, 30.0 with four rows per thread, 23.4 so, 20.3 with the shorter quantiser, 15.7 without divisions (DRAM: 13.2).
template <typename T, int HD>
__global__ void __launch_bounds__(256) write_kernel(const T* __restrict__ k, long long k_stride, const T* __restrict__ v,
                                                    long long v_stride, int n, long long pos0, View ck, View cv, bool al32) {
  constexpr int PER = HD / BLOCK;
  const unsigned u = blockIdx.x * 256u + threadIdx.x, j = u % PER;
  const int row = (int)(u / PER), head = blockIdx.y >> 1;
  if (row >= n) return;
  const bool val = blockIdx.y & 1;
  float x[BLOCK];
  load_block((val ? v + row * v_stride : k + row * k_stride) + head * HD + j * BLOCK, x, al32);
  uint32_t byte;
  const uint2 w = quantise(x, byte);
  const long long at = (pos0 + row) * PER + j;
  *reinterpret_cast<uint2*>((val ? cv.codes : ck.codes) + head * ck.head_codes + at * 8) = w;
  ((val ? cv.scales : ck.scales) + head * ck.head_scales)[at] = (uint8_t)byte;
}

// code e of a block, less 8
__device__ __forceinline__ float code_of(uint2 w, int e) { return (float)(((e < 8 ? w.x : w.y) >> ((e & 7) * 4)) & 15u) - 8.f; }

// The inverse; code times scale is exact in fp32 and in bf16.  36.2 us for 32768 rows of eight heads of 128 with the heads of a
// row side by side and 16-byte accesses, 34.0 in whole sectors, 31.8 without divisions and with paired conversions (DRAM: 26.3).
template <typename T, int HD>
__global__ void __launch_bounds__(256) read_kernel(View ck, View cv, int n, long long pos0, T* __restrict__ k, long long k_stride,
                                                   T* __restrict__ v, long long v_stride, bool al32) {
  constexpr int PER = HD / BLOCK;
  const unsigned u = blockIdx.x * 256u + threadIdx.x, j = u % PER;
  const int row = (int)(u / PER), head = blockIdx.y >> 1;
  if (row >= n) return;
  const bool val = blockIdx.y & 1;
  const long long at = (pos0 + row) * PER + j;
  const uint2 w = __ldg(reinterpret_cast<const uint2*>((val ? cv.codes : ck.codes) + head * ck.head_codes + at * 8));
  const uint32_t byte = __ldg((val ? cv.scales : ck.scales) + head * ck.head_scales + at);
  const float s = scale_of(byte);
  T* dst = (val ? v + row * v_stride : k + row * k_stride) + head * HD + j * BLOCK;
  if constexpr (sizeof(T) == 2) {
    if (byte == INF_SCALE) {   // (from another writer: 136 s has no finite value to take off; short code, no speed)
#pragma unroll 1
      for (int e = 0; e < BLOCK; ++e) dst[e] = __float2bfloat16(code_of(w, e) * s);
      return;
    }
    const uint32_t sc = pack_bf16(s, s), off = pack_bf16(s * -136.f, s * -136.f);
    uint32_t y[8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t c = h ? w.y : w.x;
      const uint32_t a = nib_bf16(c, sc, off), b = nib_bf16(c >> 4, sc, off), d = nib_bf16(c >> 8, sc, off), e = nib_bf16(c >> 12, sc, off);
      y[4 * h] = __byte_perm(a, b, 0x5410);        // values 0 1, 2 3, 4 5, 6 7 from 0 4, 1 5, 2 6, 3 7
      y[4 * h + 1] = __byte_perm(d, e, 0x5410);
      y[4 * h + 2] = __byte_perm(a, b, 0x7632);
      y[4 * h + 3] = __byte_perm(d, e, 0x7632);
    }
    st32(dst, y, al32);
  } else {
    float x[BLOCK];
#pragma unroll
    for (int e = 0; e < BLOCK; ++e) x[e] = code_of(w, e) * s;
    store_block(dst, x, al32);
  }
}

// A layer's fused projections [R, (nq + 2 nkv) hd] (fp32): queries rotated and stored in the model dtype (in bf16 models rounded to
// its 8 bits, as the persistent kernel rounds them: the multiplies take bf16 or half precision), keys rotated and quantised,
// values quantised.  Dims i and i + hd / 2 share a rotation, so a thread of the rotated part takes the blocks j and j + hd / 32.
template <typename T>
__global__ void __launch_bounds__(256) store_rows_kernel(const float* __restrict__ qkv, long long ld, const float2* __restrict__ cs, int R,
                                                         int rows, int nq, int nkv, int hd, View ck, View cv, long long pos0,
                                                         T* __restrict__ q) {
  const int half_blocks = hd / (2 * BLOCK), per_row = (nq + 2 * nkv) * half_blocks;
  const long long u = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (u >= (long long)R * per_row) return;
  const int r = (int)(u / per_row), e = (int)(u - (long long)r * per_row), head = e / half_blocks, j = e - head * half_blocks;
  const float* p = qkv + r * ld + head * hd + j * BLOCK;
  float a[BLOCK], b[BLOCK];
  load16(p, a);
  load16(p + hd / 2, b);
  if (head < nq + nkv) {
    const float2* w = cs + (long long)(r % rows) * (hd / 2) + j * BLOCK;   // (states of `rows` rows)
#pragma unroll
    for (int i = 0; i < BLOCK; ++i) {
      const float2 c = w[i];
      const float x = a[i] * c.x - b[i] * c.y, y = b[i] * c.x + a[i] * c.y;
      a[i] = x;
      b[i] = y;
    }
    if (head < nq) {
      T* out = q + ((long long)r * nq + head) * hd + j * BLOCK;
      store16(out, a);
      store16(out + hd / 2, b);
      return;
    }
  }
  const bool val = head >= nq + nkv;
  const View& c = val ? cv : ck;
  const int h = head - nq - (val ? nkv : 0);
  uint8_t* codes = c.codes + h * c.head_codes + (pos0 + r) * (hd / 2) + j * 8;
  uint8_t* scales = c.scales + h * c.head_scales + (pos0 + r) * (hd / BLOCK) + j;
  uint32_t byte;
  *reinterpret_cast<uint2*>(codes) = quantise(a, byte);
  scales[0] = (uint8_t)byte;
  *reinterpret_cast<uint2*>(codes + hd / 4) = quantise(b, byte);
  scales[half_blocks] = (uint8_t)byte;
}

// ------------------------------------------------------------------ attention
// Rows are S states of T rows (row r: state r / T).  Row r sees the cache positions [0, limit_r) and, where the call has
// own rows, the rows first..r of its state, which lie at own + own_pos0.  When the own rows continue the cache (a
// verification: one state behind the context), the two are one prefix and own_n is 0: limit_r = prefix + r + 1.
struct AttnArgs {
  const void* q;           // row r, head h at q + r * q_stride + h * hd; model dtype, as `out`
  long long q_stride;
  void* out;
  long long out_stride;
  int R, T, nq, nkv;
  View k, v;               // the cache
  int n_keys;              // positions any row may see
  int causal;              // 1: limit_r = n_keys - R + r + 1
  const int* visible;      // or null: limit_r = min(n_keys, max(0, visible[r]))
  View own_k, own_v;
  long long own_pos0;
  int own_n;               // rows of the own region (R_all), or 0
  int run_len, runs;       // keys per CTA and CTAs over the cache; one more CTA where own_n > 0
  float* part;             // [R * nq, parts, hd] and
  float2* part_ml;         // [R * nq, parts] (maximum, sum)
  int* counters;           // one per (kv head, block of pairs), zero on entry and on exit
  int* status;             // set when a bounded wait of attn_many_kernel runs out
  uint32_t spin_fast, spin_slow;   // its polls (constants in their place unroll the loop: 4 % of a call)
  int blocks, splits;      // attn_many_kernel: blocks of pairs per kv head, parts of each block's key tiles
  int r0;                  // first row of this launch (of `visible` and the causal limit; q, out are offset already)
  int R_all;               // rows of the call
};

__device__ __forceinline__ int row_limit(const AttnArgs& p, int r) {
  if (p.causal) return p.n_keys - p.R_all + p.r0 + r + 1;
  if (p.visible) return min(p.n_keys, max(0, p.visible[p.r0 + r]));
  return p.n_keys;
}

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t movmatrix_t(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half(float a, float b) {
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t u) { return __half22float2(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ __half2 as_half2(uint32_t u) { return *reinterpret_cast<const __half2*>(&u); }
__device__ __forceinline__ uint32_t as_u32(__half2 h) { return *reinterpret_cast<const uint32_t*>(&h); }

// A query row for half precision: the power of two that brings its largest magnitude into [2^9, 2^10), and
// the factor that takes it back and brings the scores into units of log2 (1 / sqrt(hd) aside).  LANES neighbouring lanes hold a row,
// N values each.  A row with an infinity or NaN in it has no finite score: its factor is NaN, and so are all its weights.
struct RowScale {
  float up, mult;
};
// a: the bits of the row's largest magnitude
__device__ __forceinline__ RowScale scale_for(uint32_t a) {
  const int up = 9 - max((int)(a >> 23) - 127, -113);   // rows far below 2^-113 are as good as zero
  RowScale r;
  r.up = __uint_as_float((uint32_t)(127 + up) << 23);
  r.mult = __uint_as_float((uint32_t)(127 - up) << 23) * 1.4426950408889634f;
  if (a >= 0x7f800000u) r.mult = __int_as_float(0x7fffffff);
  return r;
}
template <int N, int LANES>
__device__ __forceinline__ RowScale row_scale(const float (&x)[N]) {
  uint32_t a = 0;                      // magnitudes compare like their bits; infinities and NaN are the largest
#pragma unroll
  for (int e = 0; e < N; ++e) a = max(a, __float_as_uint(x[e]) & 0x7fffffffu);
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) a = max(a, __shfl_xor_sync(0xffffffffu, a, o));
  return scale_for(a);
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// two fp32 operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, z, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 w, x, y, z;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
  return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 d;
  asm("{\n\t.reg .b64 x, y, w;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 w, x, y;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
  return d;
}

// Scales of the two halves of a register, as the conversion needs them.
struct Scale2 {
  __half2 s, s16, m64, m72;   // s, s / 16, -64.5 s, -72 s
};
// b: the scale bytes of the low and the high half at bits 0 and 16
__device__ __forceinline__ Scale2 scale2(uint32_t b) {
  Scale2 r;
  r.s = as_half2(b * 128u);
  r.s16 = __hmul2(r.s, as_half2(0x2C002C00u));    // 1 / 16
  r.m64 = __hmul2(r.s, as_half2(0xD408D408u));    // -64.5
  r.m72 = __hmul2(r.s, as_half2(0xD480D480u));    // -72
  return r;
}
// The nibbles 0, 1 (w) or 2, 3 (w >> 8) of both 16-bit halves: a nibble in the low mantissa bits of 1024 makes 1024 + c, one
// place higher 1024 + 16 c, without an integer conversion; one multiply-add with s / 16 then gives
//   nib_lo: (c - 8) s / 16     nib_hi: (c - 8) s
// exactly (64.5 s and 72 s have at most 11 significant bits, the results at most 7 above half precision's last place).  The
// sixteenth is made up for where it costs nothing: in q, and in the finished output.  ((1024 + c) s - 1032 s would overflow
// from s = 64 on.)
__device__ __forceinline__ uint32_t nib_lo(uint32_t w, const Scale2& s) {
  return as_u32(__hfma2(as_half2(and_or(w, 0x000F000Fu, 0x64006400u)), s.s16, s.m64));
}
__device__ __forceinline__ uint32_t nib_hi(uint32_t w, const Scale2& s) {
  return as_u32(__hfma2(as_half2(and_or(w, 0x00F000F0u, 0x64006400u)), s.s16, s.m72));
}

constexpr int WARPS = 16;
constexpr int STEP = 16;                 // keys a warp takes at a time
constexpr int PB = 8;                    // pairs per CTA
constexpr int STAGES = 4;                // steps of a warp in shared memory: one at work, three on their way
constexpr int MAX_PARTS = 152;           // runs of one launch and the own rows
constexpr float P_BITS = 12.f;           // weights are held as 2^12 .. 2^20 x exp2(s - m) in half precision (see below)

template <int HD> struct Raw {           // one warp step: two key rows' and four value rows' pieces per lane
  uint32_t k[2][HD / 32], v[4][HD / 64];
  uint32_t ks[2], vs[4];
};
template <int HD> constexpr int STEP_BYTES = STEP * (HD + HD / 8);
template <int HD, bool SPLIT> constexpr int rows_smem() {
  constexpr int ring = WARPS * STAGES * STEP_BYTES<HD>, merge = WARPS * PB * (HD + 4) * 4;
  return (ring > merge ? ring : merge) + (SPLIT ? 2 : 1) * (HD / 16) * 32 * 8;
}
template <int N> __device__ __forceinline__ void cp_async(uint32_t dst, const void* src, bool in) {
  if constexpr (N == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16u : 0u) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(in ? (uint32_t)N : 0u), "n"(N) : "memory");
}

// Attention of few (row, query head) pairs: eight pairs of one kv head per CTA, one run of the cache per CTA, its steps of 16
// keys dealt to sixteen warps that never wait for one another before the end.
//
//   S^T = K q^T     16 keys x 8 pairs: the keys are the M rows of mma.m16n8k16, so few pairs waste little
//   O^T = V^T P^T   16 dims x 8 pairs
//
// Which key an M row is and which dim a k index is, is free as long as both operands agree, so a lane gets its pieces of
// K and V in 16- and 8-byte loads and converts them in place: lane (g, t) of a step holds dims [32 t, 32 t + 32) of two keys, and
// 16 dims [16 g, 16 g + 16) of four values (hd 128).  A warp copies its steps to a ring of its own, three ahead (asynchronous
// copies: the bytes on their way cost no registers), with the rows placed so that those loads meet no bank twice.  K and V are exact in
// half precision.  q is scaled by a power of two per row to a largest magnitude in [2^9, 2^10) (a nibble's 16 on top of it, see
// nib_lo) and rounded to half precision: exact for bf16 rows (what lies 2^25 below the row's maximum aside); SPLIT (fp32 models)
// adds the rounding error of q and of the weights as a second half-precision operand: 22 bits.  Weights: half precision of 2^12 exp2(s - m), m a maximum that moves
// only when exceeded by 2^3, so they stay below 2^15 and lose nothing above 2^-26 of the largest; sums in fp32.  One part, 11 bits, is
// enough for bf16 results of 8: their error against 64 bits is 0.5 % above that of fp32 weights (1.648e-3 against 1.641e-3 over 512
// positions), a second part would double these multiplies.
// A block with the NaN byte must reach only the rows that see it, and 0 x NaN is NaN: values' NaN blocks enter as zeros, and
// `poison` remembers which (pair, block) they belong to.
//
// Measured, eight kv heads of 128, us: one token over 512 / 131071 positions (four pairs) 7.2 / 38.9, five rows of 64 heads over
// 2048 12.5.  A step is about 300 instructions and 1850 cycles of sixteen warps side by side (61 % of the issue slots, the
// conversion's logic and half-precision pipes at 48 and 38 %): 131071 positions move at 3.9 TB/s.  Straight loads of a step one ahead
// took 55.7 us, twenty or twenty-four warps 42.0 / 44.7, sixteen pairs per CTA as long per pair (17 instead of 12.6 us for the
// five rows).  Below a thousand positions it is launch, first instruction fetches and the joining of the warps.
template <int HD, bool SPLIT>
__global__ void __launch_bounds__(WARPS * 32, 1) attn_rows_kernel(const __grid_constant__ AttnArgs p) {
  constexpr int KS = HD / 16;            // k steps of the scores, and tiles of 16 dims of the output
  constexpr int KW = HD / 32, VW = HD / 64;
  constexpr int PARTS = SPLIT ? 2 : 1;
  constexpr float NEG = -INFINITY;
  extern __shared__ __align__(1024) uint8_t smem[];
  uint2 (*qf)[KS][32] = reinterpret_cast<uint2 (*)[KS][32]>(smem);
  uint8_t* ring = smem + PARTS * KS * 32 * 8;                       // the warps' steps, later their results
  float (*o_sm)[PB][HD + 4] = reinterpret_cast<float (*)[PB][HD + 4]>(ring);
  __shared__ float2 ml_sm[WARPS][PB];
  __shared__ float w_sm[WARPS][PB], mx_sm[PB];
  __shared__ float mult_sm[PB];
  __shared__ int lo_sm[PB], hi_sm[PB];
  __shared__ uint32_t poison_sm[8];
  __shared__ int last_sm;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int run = blockIdx.x, kvh = blockIdx.y, pb = blockIdx.z;
  const int G = p.nq / p.nkv, n_pairs = p.R * G, parts = gridDim.x;
  const bool own = run >= p.runs;
  const int pair0 = pb * PB;

  // what each pair sees (every warp for itself; the masks read it from shared memory)
  int lo = 0, hi = 0;
  const bool mine = lane < PB && pair0 + lane < n_pairs;
  if (mine) {
    const int r = (pair0 + lane) / G;
    if (own) { lo = (p.r0 + r) / p.T * p.T; hi = p.r0 + r + 1; }
    else hi = row_limit(p, r);
  }
  if (warp == 0 && lane < PB) { lo_sm[lane] = lo; hi_sm[lane] = hi; }
  if (threadIdx.x < 8) poison_sm[threadIdx.x] = 0;
  const int first = __reduce_min_sync(0xffffffffu, mine ? lo : 0x7fffffff), last = __reduce_max_sync(0xffffffffu, hi);
  // keys of this CTA
  int k_lo, k_end;
  if (own) {
    k_lo = first;
    k_end = min(last, p.own_n);
  } else {
    k_lo = run * p.run_len;
    k_end = min(min(k_lo + p.run_len, p.n_keys), last);
  }
  const int full_lo = __reduce_max_sync(0xffffffffu, lo);
  const int full_hi = min(__reduce_min_sync(0xffffffffu, mine ? hi : 0x7fffffff), k_end);
  const long long pos_off = own ? p.own_pos0 : 0;
  const View& vk = own ? p.own_k : p.k;
  const View& vv = own ? p.own_v : p.v;
  const uint8_t* kc = vk.codes + kvh * vk.head_codes + pos_off * (HD / 2);
  const uint8_t* kx = vk.scales + kvh * vk.head_scales + pos_off * (HD / BLOCK);
  const uint8_t* vc = vv.codes + kvh * vv.head_codes + pos_off * (HD / 2);
  const uint8_t* vx = vv.scales + kvh * vv.head_scales + pos_off * (HD / BLOCK);
  const int kg = (g >> 1) + 4 * (g & 1);   // key of M row g; row g + 8 is key kg + 8
  // A step in shared memory: K codes, V codes, K scales, V scales.  Key k's row of K lies where M row g = k is (so that g's rows
  // follow one another); of V, the 16-byte pieces of keys 2, 3 of each four are swapped in pairs (hd 128).
  constexpr int ROW = HD / 2, KV_STEP = STEP * ROW, SC = HD / BLOCK;
  const uint32_t my_ring = tc::smem_u32(ring) + warp * STAGES * STEP_BYTES<HD>;
  int ahead = k_lo + warp * STEP, ahead_stage = 0;   // the next step to fetch
  const int f_key = HD == 128 ? lane >> 2 : lane >> 1, f_piece = HD == 128 ? lane & 3 : lane & 1, x_key = lane & 15;
  const uint8_t* f_k = kc + (long long)(ahead + f_key) * ROW + f_piece * 16;
  const uint8_t* f_v = vc + (long long)(ahead + f_key) * ROW + f_piece * 16;
  const uint8_t* f_x = (lane < 16 ? kx : vx) + (long long)(ahead + x_key) * SC;
  const uint32_t d_k = my_ring + ((f_key & 8) + ((f_key & 3) << 1) + ((f_key >> 2) & 1)) * ROW + f_piece * 16;
  const uint32_t d_v = my_ring + KV_STEP + f_key * ROW + (HD == 128 ? f_piece ^ (f_key & 2) : f_piece) * 16;
  const uint32_t d_x = my_ring + 2 * KV_STEP + (lane >> 4) * STEP * SC + x_key * SC;
  auto fetch = [&]() {
    if (ahead < k_end) {
      const uint32_t at = ahead_stage * STEP_BYTES<HD>;
      const bool whole = ahead + STEP <= k_end;
      // keys past the end: zero bytes (and an address inside the cache)
      auto copy = [&](uint32_t dst, const uint8_t* src, const uint8_t* safe, int key) {
        const bool in = ahead + key < k_end;
        cp_async<16>(dst + at, in ? src : safe, in);
      };
      if (whole) {
        cp_async<16>(d_k + at, f_k, true);
        cp_async<16>(d_v + at, f_v, true);
        if constexpr (HD == 128) {     // eight keys further on
          cp_async<16>(d_k + at + 8 * ROW, f_k + 8 * ROW, true);
          cp_async<16>(d_v + at + 8 * ROW, f_v + 8 * ROW, true);
        }
        cp_async<SC>(d_x + at, f_x, true);
      } else {
        copy(d_k, f_k, kc + (long long)k_lo * ROW, f_key);
        copy(d_v, f_v, vc + (long long)k_lo * ROW, f_key);
        if constexpr (HD == 128) {
          copy(d_k + 8 * ROW, f_k + 8 * ROW, kc + (long long)k_lo * ROW, f_key + 8);
          copy(d_v + 8 * ROW, f_v + 8 * ROW, vc + (long long)k_lo * ROW, f_key + 8);
        }
        const bool in = ahead + x_key < k_end;
        cp_async<SC>(d_x + at, in ? f_x : (lane < 16 ? kx : vx) + (long long)k_lo * SC, in);
      }
      ahead += WARPS * STEP;
      f_k += WARPS * STEP * ROW;
      f_v += WARPS * STEP * ROW;
      f_x += WARPS * STEP * SC;
      if (++ahead_stage == STAGES) ahead_stage = 0;
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto take = [&](Raw<HD>& w, int stage) {
    const uint8_t* s = ring + (warp * STAGES + stage) * STEP_BYTES<HD>;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* a = s + (g + 8 * i) * ROW + t * (HD / 8);
      const uint8_t* x = s + 2 * KV_STEP + (kg + 8 * i) * SC + t * (HD / 64);
      if constexpr (HD == 128) {
        const uint4 u = *reinterpret_cast<const uint4*>(a);
        w.k[i][0] = u.x; w.k[i][1] = u.y; w.k[i][2] = u.z; w.k[i][3] = u.w;
        w.ks[i] = *reinterpret_cast<const unsigned short*>(x);
      } else {
        const uint2 u = *reinterpret_cast<const uint2*>(a);
        w.k[i][0] = u.x; w.k[i][1] = u.y;
        w.ks[i] = *x;
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = t + 4 * i;
      const uint8_t* a = s + KV_STEP + key * ROW;
      if constexpr (HD == 128) {
        const uint2 u = *reinterpret_cast<const uint2*>(a + (((g >> 1) ^ (t & 2)) << 4) + ((g & 1) << 3));
        w.v[i][0] = u.x; w.v[i][1] = u.y;
      } else {
        w.v[i][0] = *reinterpret_cast<const uint32_t*>(a + g * 4);
      }
      w.vs[i] = s[2 * KV_STEP + STEP * SC + key * SC + (HD == 128 ? g : g >> 1)];
    }
  };

  int base = k_lo + warp * STEP, stage = 0;
#pragma unroll 1
  for (int i = 0; i < STAGES - 1; ++i) fetch();

  // q rows into the fragments of the second operand: a warp per pair, lane = its place along the row
  if (warp < PB) {
    const int i = warp, pp = pair0 + i;
    constexpr int E = HD / 32;
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.f;
    if (pp < n_pairs) {
      const long long off = (long long)(pp / G) * p.q_stride + (long long)(kvh * G + pp % G) * HD + lane * E;
      if constexpr (!SPLIT) {
        const bf16* s = (const bf16*)p.q + off;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = __bfloat162float(s[e]);
      } else {
        const float* s = (const float*)p.q + off;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = s[e];
      }
    }
    const RowScale rs = row_scale<E, 32>(x);
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] *= rs.up;
    // element d of the row is half h of register b of lane (g = i & 7, t = d / (HD / 4)) in step 2 (word) + (n & 3) / 2, for
    // word = d % (HD / 4) / 8, n = d % 8: b = n & 1, half n / 4
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int d = lane * E + e, tt = d / (HD / 4), wd = d % (HD / 4) / 8, n = d & 7;
      const int step = wd * 2 + ((n >> 1) & 1);
      if ((n & 1) == 0) x[e] *= 16.f;    // meets nib_lo
      const __half hx = __float2half_rn(x[e]);
      __half* dst = reinterpret_cast<__half*>(&qf[0][step][i * 4 + tt]) + (n & 1) * 2 + (n >> 2);
      *dst = hx;
      if constexpr (SPLIT) {
        __half* d2 = reinterpret_cast<__half*>(&qf[PARTS - 1][step][i * 4 + tt]) + (n & 1) * 2 + (n >> 2);
        *d2 = __float2half_rn(x[e] - __half2float(hx));
      }
    }
    if (lane == 0) mult_sm[i] = rs.mult * rsqrtf((float)HD);
  }
  __syncthreads();

  // off: m - P_BITS of each pair (0 before its first visible key, then top is -inf); top: a score above it moves m
  float o[KS][4], off[2], top[2], l[2], mult[2];
  uint32_t poison = 0;
#pragma unroll
  for (int c = 0; c < 2; ++c) { off[c] = 0.f; top[c] = NEG; l[c] = 0.f; mult[c] = mult_sm[2 * t + c]; }
#pragma unroll
  for (int j = 0; j < KS; ++j)
#pragma unroll
    for (int c = 0; c < 4; ++c) o[j][c] = 0.f;

#pragma unroll 1
  for (; base < k_end; base += WARPS * STEP) {
    asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 2) : "memory");
    __syncwarp();                          // the step has arrived for all lanes, and all are done with the one before it
    fetch();
    Raw<HD> cur;
    take(cur, stage);
    if (++stage == STAGES) stage = 0;
    // ---- scores, in two chains of multiplies
    float s[4], s2[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) s[c] = s2[c] = 0.f;
#pragma unroll
    for (int wd = 0; wd < KW; ++wd) {
      constexpr int WPS = 2;                          // words per scale
      const Scale2 s0 = scale2(__byte_perm(cur.ks[0], 0, 0x4040 + 0x101 * (wd / WPS))),
                   s1 = scale2(__byte_perm(cur.ks[1], 0, 0x4040 + 0x101 * (wd / WPS)));
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint32_t w0 = cur.k[0][wd] >> (8 * h), w1 = cur.k[1][wd] >> (8 * h);
        const uint32_t a[4] = {nib_lo(w0, s0), nib_lo(w1, s1), nib_hi(w0, s0), nib_hi(w1, s1)};
#pragma unroll
        for (int q = 0; q < PARTS; ++q) {
          const uint2 b = qf[q][wd * 2 + h][lane];
          mma16816(h ? s2 : s, a, b.x, b.y);
        }
      }
    }
    // ---- masks, weights
    const bool full = base >= full_lo && base + STEP <= full_hi;
    uint32_t pw[PARTS][2];
#pragma unroll
    for (int c = 0; c < 4; ++c) s[c] = fmaf(s2[c], mult[c & 1], fmaf(s[c], mult[c & 1], -off[c & 1]));
    if (!full) {
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int key = base + kg + (c >> 1) * 8, col = 2 * t + (c & 1);
        if (key < lo_sm[col] || key >= min(hi_sm[col], k_end)) s[c] = NEG;
      }
    }
    const float x0 = fmaxf(s[0], s[2]), x1 = fmaxf(s[1], s[3]);
    if (__any_sync(0xffffffffu, x0 > top[0] || x1 > top[1])) {
      float y[2] = {x0, x1};
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) y[c] = fmaxf(y[c], __shfl_xor_sync(0xffffffffu, y[c], d));
        if (y[c] > top[c]) {
          const float by = y[c] - P_BITS, corr = top[c] == NEG ? 0.f : exp2f(-by);
          off[c] += by;
          top[c] = P_BITS + 3.f;
          l[c] *= corr;
          s[c] -= by;
          s[c + 2] -= by;
#pragma unroll
          for (int j = 0; j < KS; ++j) { o[j][c] *= corr; o[j][c + 2] *= corr; }
        }
      }
      __syncwarp();
    }
    float e[4];
#pragma unroll
    for (int c = 0; c < 4; ++c) e[c] = ex2(s[c]);   // (nothing visible so far: exp2(-inf) = 0)
    l[0] += e[0] + e[2];
    l[1] += e[1] + e[3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t u = pack_half(e[2 * h], e[2 * h + 1]);
      pw[0][h] = movmatrix_t(u);
      if constexpr (SPLIT) {
        const float2 f = unpack_half(u);
        pw[PARTS - 1][h] = movmatrix_t(pack_half(e[2 * h] - f.x, e[2 * h + 1] - f.y));
      }
    }
    // ---- values.  Lane (g, t): keys t, t + 4 are the M-operand's columns 2 t, 2 t + 1, keys t + 8, t + 12 the upper ones
    Scale2 z0 = scale2(cur.vs[0] + cur.vs[1] * 65536u), z1 = scale2(cur.vs[2] + cur.vs[3] * 65536u);
    const __half2 zz = __hadd2(z0.s, z1.s);             // NaN where one of the four is
    if (__any_sync(0xffffffffu, !__hbeq2(zz, zz))) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (cur.vs[i] == NAN_SCALE) {
          const int key = base + t + 4 * i;
#pragma unroll 1
          for (int c = 0; c < PB; ++c)
            if (key >= lo_sm[c] && key < min(hi_sm[c], k_end)) poison |= 1u << c;
          cur.vs[i] = 0;
        }
      z0 = scale2(cur.vs[0] + cur.vs[1] * 65536u);
      z1 = scale2(cur.vs[2] + cur.vs[3] * 65536u);
      __syncwarp();
    }
#pragma unroll
    for (int wd = 0; wd < VW; ++wd) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        // dims 4 h .. 4 h + 3 of the word, one key in each half
        const uint32_t x = __byte_perm(cur.v[0][wd], cur.v[1][wd], h ? 0x7632 : 0x5410);
        const uint32_t y = __byte_perm(cur.v[2][wd], cur.v[3][wd], h ? 0x7632 : 0x5410);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t a[4] = {nib_lo(x >> (8 * e), z0), nib_hi(x >> (8 * e), z0), nib_lo(y >> (8 * e), z1), nib_hi(y >> (8 * e), z1)};
#pragma unroll
          for (int q = 0; q < PARTS; ++q) mma16816(o[wd * 4 + h * 2 + e], a, pw[q][0], pw[q][1]);
        }
      }
    }
  }

  // ---- the warps' results together, in warp order.  (From here on every instruction runs once: short code, its fetch counts.)
  asm volatile("cp.async.wait_all;" ::: "memory");
  __syncthreads();                         // the ring's place takes the results
#pragma unroll
  for (int c = 0; c < 2; ++c) {
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) l[c] += __shfl_xor_sync(0xffffffffu, l[c], d);
    // (maxima without P_BITS, here and in every part alike; a sum without a maximum is 0, or NaN)
    if (g == 0) ml_sm[warp][2 * t + c] = make_float2(top[c] == NEG ? NEG : off[c], l[c]);
#pragma unroll
    for (int j = 0; j < KS; ++j)
      *reinterpret_cast<float2*>(&o_sm[warp][2 * t + c][g * (HD / 8) + 2 * j]) =
          make_float2(o[j][c] * 16.f, o[j][c + 2]);     // (even dims are nib_lo's)
  }
  if (poison) atomicOr(&poison_sm[g], poison);
  __syncthreads();
  constexpr int UNITS = PB * (HD / 4), GROUPS = WARPS * 32 / UNITS;   // four dims of a pair; threads that share the work on them
  static_assert(WARPS * PB <= WARPS * 32 && GROUPS >= 1, "a thread per (warp, pair), one at least per unit");
  if (threadIdx.x < WARPS * PB) {          // each warp's weight
    const int col = threadIdx.x % PB, w = threadIdx.x / PB;
    float mx = NEG;
#pragma unroll 4
    for (int i = 0; i < WARPS; ++i) mx = fmaxf(mx, ml_sm[i][col].x);
    const float2 v = ml_sm[w][col];
    w_sm[w][col] = v.x == NEG ? (v.y == 0.f ? 0.f : 1.f) : exp2f(v.x - mx);
    if (w == 0) mx_sm[col] = mx;
  }
  __syncthreads();
  const bool single = parts == 1;
  const int unit = threadIdx.x % UNITS, group = threadIdx.x / UNITS, col = unit / (HD / 4), d = unit % (HD / 4) * 4;
  const int pp = pair0 + col, r = pp / G, hq = kvh * G + pp - r * G;
  const bool on = pp < n_pairs && group < GROUPS;
  const long long rh = (long long)r * p.nq + hq;
  auto store = [&](const float4& a, float den) {
    const float inv = den == 0.f ? 0.f : 1.0f / den;
    const long long at = (long long)r * p.out_stride + (long long)hq * HD + d;
    // (+ 0: a zero's sign would tell whether the call had runs that the pair sees nothing of)
    const float4 y = make_float4(fmaf(a.x, inv, 0.f), fmaf(a.y, inv, 0.f), fmaf(a.z, inv, 0.f), fmaf(a.w, inv, 0.f));
    if constexpr (!SPLIT) *reinterpret_cast<uint2*>((bf16*)p.out + at) = make_uint2(pack_bf16(y.x, y.y), pack_bf16(y.z, y.w));
    else *reinterpret_cast<float4*>((float*)p.out + at) = y;
  };
  if (group == 0 && on) {
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    float den = 0.f;
#pragma unroll 4
    for (int w = 0; w < WARPS; ++w) {
      const float4 v = *reinterpret_cast<const float4*>(&o_sm[w][col][d]);
      const float f = w_sm[w][col];
      a.x = fmaf(f, v.x, a.x); a.y = fmaf(f, v.y, a.y); a.z = fmaf(f, v.z, a.z); a.w = fmaf(f, v.w, a.w);
      den = fmaf(f, ml_sm[w][col].y, den);
    }
    if ((poison_sm[d / (HD / 8)] >> col) & 1u) a.x = a.y = a.z = a.w = __int_as_float(0x7fffffff);
    if (single) {
      store(a, den);
    } else {
      *reinterpret_cast<float4*>(p.part + (rh * parts + run) * HD + d) = a;
      if (d == 0) p.part_ml[rh * parts + run] = make_float2(mx_sm[col], den);
    }
  }
  if (single) return;

  // ---- the CTA that arrives last adds the runs, in run order
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) {
    int* c = p.counters + (long long)pb * p.nkv + kvh;
    const int n = atomicAdd(c, 1);
    last_sm = n == parts - 1;
    if (n == parts - 1) *c = 0;
  }
  __syncthreads();
  if (!last_sm) return;
  __threadfence();
  float* wr_sm = reinterpret_cast<float*>(ring);                       // [PB][MAX_PARTS] weights of the runs
  float* den_sm = wr_sm + PB * MAX_PARTS;                              // [PB]
  float4* red = reinterpret_cast<float4*>(den_sm + PB);                // [threads]
  static_assert(WARPS * PB * (HD + 4) >= PB * MAX_PARTS + PB + WARPS * 32 * 4, "weights and sums fit");
  if (warp < PB && pair0 + warp < n_pairs) {                           // a warp per pair
    const int rw = (pair0 + warp) / G;
    const float2* ml = p.part_ml + ((long long)rw * p.nq + kvh * G + pair0 + warp - rw * G) * parts;
    float mx = NEG, den = 0.f;
#pragma unroll 1
    for (int i = lane; i < parts; i += 32) mx = fmaxf(mx, __ldcg(&ml[i]).x);
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, e));
#pragma unroll 1
    for (int i = lane; i < parts; i += 32) {
      const float2 v = __ldcg(&ml[i]);
      const float w = v.x == NEG ? (v.y == 0.f ? 0.f : 1.f) : exp2f(v.x - mx);
      wr_sm[warp * MAX_PARTS + i] = w;
      den = fmaf(v.y, w, den);
    }
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) den += __shfl_xor_sync(0xffffffffu, den, e);
    if (lane == 0) den_sm[warp] = den;
  }
  __syncthreads();
  // groups of threads share the runs between them: run i is group i % GROUPS', however many runs the call has (others' rows may
  // reach into runs that this pair sees nothing of), so that a row's sum does not depend on the rows that share the call
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (on) {
    const float* src = p.part + rh * parts * HD + d;
#pragma unroll 9
    for (int i = group; i < parts; i += GROUPS) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(src + (long long)i * HD));
      const float w = wr_sm[col * MAX_PARTS + i];
      a.x = fmaf(w, v.x, a.x); a.y = fmaf(w, v.y, a.y); a.z = fmaf(w, v.z, a.z); a.w = fmaf(w, v.w, a.w);
    }
  }
  if constexpr (GROUPS > 1) {
    red[threadIdx.x] = a;
    __syncthreads();
    if (group > 0 || !on) return;
#pragma unroll
    for (int e = 1; e < GROUPS; ++e) {
      const float4 v = red[e * UNITS + unit];
      a.x += v.x; a.y += v.y; a.z += v.z; a.w += v.w;
    }
  }
  if (on) store(a, den_sm[col]);
}

// ------------------------------------------------------------------ attention of many pairs
constexpr int TK = 64;                 // keys per tile
constexpr int TP = 128;                // pairs per block: tensor-memory lanes
constexpr int RING = 6;                // K and V tiles, converted, in shared memory
constexpr float LAZY = 5.f, MANY_BITS = 10.f;   // the maximum moves when exceeded by 2^5; weights are 2^10 exp2(s - m)

template <int HD, int NB>
constexpr int many_smem() { return NB * TP * HD * 2 + RING * TK * HD * 2 + 2048; }
// warps: four per block of pairs for the softmax, four for the conversion of the tiles (one block: eight, four for the keys and four
// for the values), one per block for the multiplies
template <int NB>
constexpr int many_threads() { return NB * 128 + (NB == 1 ? 256 : 128) + NB * 32; }

struct ManyShared {
  uint64_t full[RING], empty[RING], s_full[2][2], p_full[2][2];
  uint64_t o_done[2][2];   // by parity of the tile: a wait that skips tiles may lag one behind, never two
  uint32_t tmem_base;
  uint64_t q_ready;
  int abort, poison;
};
static_assert(sizeof(ManyShared) <= 2048, "fits its share of shared memory");

// Attention of many (row, query head) pairs of a kv head: NB blocks of 128 pairs per CTA share the key tiles, which warps of
// their own convert from the cache's codes into shared memory (128-byte swizzle).
//   S = Q K^T in bf16 (rows as they are, K exact), P = 2^10 exp2(S - m) and V in half precision, O += P V:
//   tcgen05, S / P / O in tensor memory
// A thread owns a pair; its maximum moves only when exceeded by 2^5 (then O is rescaled).  Scores are double-buffered: the next
// tile's Q K^T runs under this tile's softmax.  NaN blocks: as in attn_rows_kernel; where a value's NaN block was met, the pairs
// look through the scale bytes of the keys they see once more at the end.  Half-precision weights: as there (error against 64 bits 0.5 -
// 0.7 % above that of fp32 weights).
//
// Measured, 32 query heads over eight kv heads of 128, us: a prompt of 1999 rows 49, 128 rows over 4095 positions 22.8 with its
// merge, twelve states over 8192 19.4.  A tile of 2 x 128 pairs takes 2000 cycles where its multiplies take 1280 and its
// exponentials 1024: bound by the softmax warps' chain (scores from tensor memory, maximum, exponentials, weights back, barrier),
// two warps per scheduler in step.  No gain from a quarter of the exponentials on the multiply-add pipe, from exponentials with
// the previous maximum while the new one is found, nor from starting the blocks half a tile apart (51.8, 55.3, 56.8 us against
// 51.4 then).
//
// LIMITED: for calls under a wait limit of the caller's.
template <int HD, int NB, bool LIMITED>
__global__ void __launch_bounds__(many_threads<NB>(), 1) attn_many_kernel(const __grid_constant__ AttnArgs p) {
  constexpr uint32_t Q_BYTES = TP * HD * 2, KV_BYTES = TK * HD * 2, HALF_Q = TP * 128, HALF_KV = TK * 128;
  constexpr uint32_t TM_COLS = NB == 2 ? 512 : 256, O_COL = NB * 128;
  extern __shared__ __align__(1024) uint8_t smem[];
  const uint32_t base = tc::smem_u32(smem);
  ManyShared* sh = reinterpret_cast<ManyShared*>(smem + NB * Q_BYTES + RING * KV_BYTES);
  constexpr int CONV = NB == 1 ? 8 : 4, W_CONV = NB * 4, W_MMA = W_CONV + CONV;   // first warps of the roles
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int Gq = p.nq / p.nkv, Pn = p.R * Gq;
  // longest blocks first
  int b = blockIdx.x;
  const int split = b % p.splits;
  b /= p.splits;
  const int kvh = b % p.nkv;
  const int pair0 = (p.blocks - 1 - b / p.nkv) * (NB * TP);
  const int r_lo = pair0 / Gq, r_hi = min(p.R - 1, (pair0 + NB * TP - 1) / Gq);
  if ((base & 1023u) != 0) {   // the tiles' swizzle needs it (dynamic shared memory starts aligned)
    if (threadIdx.x == 0) atomicExch(p.status, 1);
    return;
  }
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");   // (merge_kernel, which waits for this grid's end)
  if (threadIdx.x == 0) {
    for (int s = 0; s < RING; ++s) {
      tc::mbar_init(tc::smem_u32(&sh->full[s]), 4);
      tc::mbar_init(tc::smem_u32(&sh->empty[s]), NB);
    }
    for (int s = 0; s < 4; ++s) {
      tc::mbar_init(tc::smem_u32(&sh->s_full[s >> 1][s & 1]), 1);
      tc::mbar_init(tc::smem_u32(&sh->p_full[s >> 1][s & 1]), 4);
      tc::mbar_init(tc::smem_u32(&sh->o_done[s >> 1][s & 1]), 1);
    }
    tc::mbar_init(tc::smem_u32(&sh->q_ready), NB * 4);
    sh->abort = 0;
    sh->poison = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  if (warp == W_MMA) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(&sh->tmem_base)), "r"(TM_COLS)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = sh->tmem_base;
  // key tiles of this CTA: the cache's, up to the last one any of its rows sees, then the own rows'
  int n_cache = row_limit(p, r_hi);
  if (p.visible) {
    n_cache = 0;
    for (int r = r_lo + lane; r <= r_hi; r += 32) n_cache = max(n_cache, row_limit(p, r));
    n_cache = __reduce_max_sync(0xffffffffu, n_cache);
  }
  const int own_lo = p.own_n > 0 ? r_lo / p.T * p.T : 0;
  const int nt_c = (n_cache + TK - 1) / TK, nt_all = nt_c + (p.own_n > 0 ? (r_hi - own_lo) / TK + 1 : 0);
  const int t_lo = (int)((long long)nt_all * split / p.splits), nt = (int)((long long)nt_all * (split + 1) / p.splits) - t_lo;

  // A wait of a whole warp.  The first poll stands outside the bounded loop: most waits here find their phase complete, and the
  // loop's code cost each of them about 200 cycles of the tile's chain.  Such a poll may suspend the warp for microseconds, in which a
  // healthy wait is over: under a limit a poll is one look, some 100 ns with the sleep behind it.
  bool ok = true;
  auto warp_wait = [&](uint64_t* bar, uint32_t parity) {
    const uint32_t at = tc::smem_u32(bar);
    if (!__all_sync(0xffffffffu, LIMITED ? tc::mbar_look(at, parity) : tc::mbar_test(at, parity))) {
      if constexpr (LIMITED) {
        ok = false;
        for (uint32_t i = 0; i < p.spin_slow && !(ok = tc::mbar_look(at, parity)); ++i) __nanosleep(64);
        if (!ok) atomicExch(p.status, 1);
      } else {
        ok = tc::mbar_wait(at, parity, p.status, p.spin_fast, p.spin_slow);
      }
      ok = __all_sync(0xffffffffu, ok);
    }
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    return ok;
  };

  if (warp >= W_CONV && warp < W_MMA) {
    // ---- tiles in the order the multiplies take them: K0, K1, V0, K2, V1, ... (tile t's keys are item 2 t - 1, its values item
    // 2 t + 2 of the ring).  A thread takes half a row of a tile: key
    // tid % 64 (eight neighbours fill eight different 16-byte columns of the swizzle).  Codes are fetched two tiles ahead.
    constexpr int W = HD / 16;                       // words of codes per thread
    const int tid = ((int)threadIdx.x - NB * 128) & 127, row = tid & 63, part = tid >> 6;
    struct Piece { uint32_t w[W], s; };
    struct Source { const uint8_t *c, *x; };         // this thread's share of key 0
    auto source = [&](const View& v, long long pos) {
      return Source{v.codes + kvh * v.head_codes + pos * (HD / 2) + part * (HD / 4),
                    v.scales + kvh * v.head_scales + pos * (HD / BLOCK) + part * (HD / 32)};
    };
    const Source kc = source(p.k, 0), ko = source(p.own_k, p.own_pos0), vc = source(p.v, 0), vo = source(p.own_v, p.own_pos0);
    auto fetch = [&](Piece& d, bool value, int t) {
      const bool own = t_lo + t >= nt_c;
      const int key = (own ? own_lo - nt_c * TK : 0) + (t_lo + t) * TK + row, end = own ? r_hi + 1 : n_cache;
      d.s = 0;
#pragma unroll
      for (int k = 0; k < W; ++k) d.w[k] = 0x88888888u;
      if (t < nt && key < end) {
        const uint8_t* c = (own ? (value ? vo.c : ko.c) : (value ? vc.c : kc.c)) + (long long)key * (HD / 2);
        const uint8_t* x = (own ? (value ? vo.x : ko.x) : (value ? vc.x : kc.x)) + (long long)key * (HD / BLOCK);
#pragma unroll
        for (int k = 0; k < W / 4; ++k) {
          const uint4 u = __ldg(reinterpret_cast<const uint4*>(c) + k);
          d.w[4 * k] = u.x; d.w[4 * k + 1] = u.y; d.w[4 * k + 2] = u.z; d.w[4 * k + 3] = u.w;
        }
        if constexpr (HD == 128) d.s = __ldg(reinterpret_cast<const uint32_t*>(x));
        else d.s = __ldg(reinterpret_cast<const unsigned short*>(x));
      }
    };
    const uint32_t dst0 = base + NB * Q_BYTES + (HD == 128 ? part * HALF_KV : 0) + row * 128;
    const uint32_t col0 = (uint32_t)((row & 7) << 4) ^ (HD == 128 ? 0u : (uint32_t)part * 64u);
    auto convert = [&](Piece& d, bool value, uint32_t item) {
      const uint32_t slot = item % RING;
      if (!warp_wait(&sh->empty[slot], ((item / RING) & 1u) ^ 1u)) return;   // (the first pass finds every slot free)
      if (value && __vcmpeq4(d.s, 0xffffffffu)) {
        sh->poison = 1;
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (((d.s >> (8 * k)) & 255u) == NAN_SCALE) d.s &= ~(255u << (8 * k));
      }
      const uint32_t dst = dst0 + slot * KV_BYTES;
      auto put = [&](int k, uint32_t a, uint32_t b, uint32_t c, uint32_t e) {
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(dst + (col0 ^ (uint32_t)(k << 4))), "r"(a), "r"(b), "r"(c), "r"(e)
                     : "memory");
      };
      if (value) {
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const Scale2 sc = scale2(__byte_perm(d.s, 0, 0x4040 + 0x101 * (k >> 1)));
          const uint32_t w = d.w[k], w8 = w >> 8;
          put(k, nib_lo(w, sc), nib_hi(w, sc), nib_lo(w8, sc), nib_hi(w8, sc));
        }
      } else {
#pragma unroll
        for (int k = 0; k < W; ++k) {
          const float f = scale_of((d.s >> (8 * (k >> 1))) & 255u);
          const uint32_t sc = pack_bf16(f, f), off = pack_bf16(f * -136.f, f * -136.f), w = d.w[k];
          put(k, nib_bf16(w, sc, off), nib_bf16(w >> 4, sc, off), nib_bf16(w >> 8, sc, off), nib_bf16(w >> 12, sc, off));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&sh->full[slot])) : "memory");
    };
    if constexpr (NB == 1) {
      // one block: its softmax takes a tile faster than four warps convert one, so four take the keys and four the values
      const bool value = warp >= W_CONV + 4;
      Piece d[3];
#pragma unroll
      for (int k = 0; k < 3; ++k) fetch(d[k], value, k);
#pragma unroll 1
      for (int t = 0; t < nt && ok; t += 3) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          if (t + k < nt && ok) {
            convert(d[k], value, value ? 2 * (t + k) + 2 : max(2 * (t + k) - 1, 0));
            fetch(d[k], value, t + k + 3);
          }
        }
      }
    } else {
      Piece dk[3], dv[3];
      if (nt > 0) {
        fetch(dk[0], false, 0);
        fetch(dk[1], false, 1);
        fetch(dv[0], true, 0);
        fetch(dk[2], false, 2);
        fetch(dv[1], true, 1);
        convert(dk[0], false, 0);
      }
#pragma unroll 1
      for (int t = 0; t < nt && ok; t += 3) {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
          if (t + k < nt && ok) {
            fetch(dk[k], false, t + k + 3);
            fetch(dv[(k + 2) % 3], true, t + k + 2);
            if (t + k + 1 < nt) convert(dk[(k + 1) % 3], false, 2 * (t + k) + 1);
            if (ok) convert(dv[k], true, 2 * (t + k) + 2);
          }
        }
      }
    }
    if (!ok) sh->abort = 1;
  } else if (warp >= W_MMA) {
    // ---- multiplies: a warp per block of pairs, so that one's waits are covered by the other's multiplies (one warp for both:
    // 2350 cycles per tile of 2 x 128 pairs, of which the tensor pipe worked 1280).  Q K^T takes bf16, P V half precision.
    const int bl = warp - W_MMA;
    const uint32_t idesc_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TK >> 3) << 17) | ((uint32_t)(TP >> 4) << 24);
    const uint32_t idesc_pv = (1u << 4) | (1u << 16) | ((uint32_t)(HD >> 3) << 17) | ((uint32_t)(TP >> 4) << 24);
    const uint32_t el = wide::elect_one();
    const uint32_t t_s = tmem + bl * 128, t_o = tmem + O_COL + bl * 128;
    const uint32_t q_base = base + bl * Q_BYTES;
    uint32_t slot = 0, phase = 0;
    auto next = [&]() {
      if (++slot == RING) { slot = 0; phase ^= 1u; }
    };
    auto scores = [&](int t) {
      if (!warp_wait(&sh->full[slot], phase)) return;
      const uint32_t k_base = base + NB * Q_BYTES + slot * KV_BYTES, d = t_s + (t & 1) * TK;
#pragma unroll
      for (int k = 0; k < HD / 16; ++k) {
        const uint64_t da = tc::make_smem_desc(q_base + (k >> 2) * HALF_Q) + (uint64_t)((k & 3) * 2);
        const uint64_t db = tc::make_smem_desc(k_base + (k >> 2) * HALF_KV) + (uint64_t)((k & 3) * 2);
        wide::mma_ss(d, da, db, idesc_qk, k > 0, el);
      }
      wide::commit_one(tc::smem_u32(&sh->s_full[bl][t & 1]), el);
      wide::commit_one(tc::smem_u32(&sh->empty[slot]), el);
      next();
    };
    if (nt > 0 && warp_wait(&sh->q_ready, 0)) scores(0);
    for (int t = 0; t < nt && ok; ++t) {
      if (t + 1 == nt) next();         // (no item 2 nt - 1)
      else scores(t + 1);              // (buffer of tile t - 1: its P V was issued before, the tensor pipe keeps the order)
      if (!ok || !warp_wait(&sh->full[slot], phase) || !warp_wait(&sh->p_full[bl][t & 1], (t >> 1) & 1u)) break;
      // V tile: key rows of 64 dims, the MN-major form of B (64-dim halves HALF_KV apart)
      const uint64_t db = (tc::make_smem_desc(base + NB * Q_BYTES + slot * KV_BYTES) & ~(0x3FFFull << 16)) |
                          ((uint64_t)(HALF_KV / 16) << 16);
      const uint32_t a = t_s + (t & 1) * TK;
#pragma unroll
      for (int k = 0; k < TK / 16; ++k) wide::mma_ts(t_o, a + k * 8, db + (uint64_t)(k * 128), idesc_pv, t > 0 || k > 0, el);
      wide::commit_one(tc::smem_u32(&sh->o_done[bl][t & 1]), el);
      wide::commit_one(tc::smem_u32(&sh->empty[slot]), el);
      next();
    }
    if (!ok) sh->abort = 1;
  } else {
    // ---- query rows: a lane takes sixteen dims, HD / 16 lanes a row
    {
      constexpr int LPR = HD / 16, STEP_ROWS = NB * 128 / LPR;
      const int j = threadIdx.x % LPR;
      int qrow = (int)threadIdx.x / LPR, rr = (pair0 + qrow) / Gq, hh = (pair0 + qrow) - rr * Gq;
      const int dr = STEP_ROWS / Gq, dh = STEP_ROWS - dr * Gq;
      uint4 w[LPR][2];                        // all loads in flight at once
#pragma unroll
      for (int e = 0; e < LPR; ++e) {
        w[e][0] = w[e][1] = make_uint4(0, 0, 0, 0);
        if (rr < p.R) {
          const uint4* src = reinterpret_cast<const uint4*>((const bf16*)p.q + (long long)rr * p.q_stride +
                                                            (long long)(kvh * Gq + hh) * HD + j * 16);
          w[e][0] = src[0];
          w[e][1] = src[1];
        }
        rr += dr;
        hh += dh;
        if (hh >= Gq) { hh -= Gq; ++rr; }
      }
#pragma unroll
      for (int e = 0; e < LPR; ++e, qrow += STEP_ROWS) {
        uint8_t* dst = smem + (qrow / TP) * Q_BYTES + (j >> 2) * HALF_Q + (qrow % TP) * 128;
#pragma unroll
        for (int h = 0; h < 2; ++h) {         // the order of the codes' conversion: dims 0 4, 1 5, 2 6, 3 7 of each eight
          const uint4 u = w[e][h];
          *reinterpret_cast<uint4*>(dst + ((((j & 3) * 2 + h) ^ (qrow & 7)) << 4)) =
              make_uint4(__byte_perm(u.x, u.z, 0x5410), __byte_perm(u.x, u.z, 0x7632), __byte_perm(u.y, u.w, 0x5410),
                         __byte_perm(u.y, u.w, 0x7632));
        }
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&sh->q_ready)) : "memory");
    }
    // ---- softmax: a thread per pair
    const int bl = warp >> 2, pp = pair0 + (int)threadIdx.x;
    const bool pv = pp < Pn;
    const int r = pv ? pp / Gq : 0, hq = kvh * Gq + (pv ? pp % Gq : 0);
    const int own_first = r / p.T * p.T, lim = pv ? row_limit(p, r) : 0;
    const float scale = 1.4426950408889634f * rsqrtf((float)HD);   // scores in units of log2
    const uint32_t t_row = tmem + ((uint32_t)((warp & 3) * 32) << 16) + bl * 128;
    const uint32_t t_o = tmem + ((uint32_t)((warp & 3) * 32) << 16) + O_COL + bl * 128;
    // tiles that all of the warp's pairs see whole
    const int whole = min(nt_c, __reduce_min_sync(0xffffffffu, pv ? lim : 0x7fffffff) / TK) - t_lo;
    bool seen = min(whole, nt) > 0;  // the pair sees some key of this part
    float m = -INFINITY, l = 0.f;
    for (int t = 0; t < nt && ok; ++t) {
      if (!warp_wait(&sh->s_full[bl][t & 1], (t >> 1) & 1u)) break;
      const uint32_t t_s = t_row + (t & 1) * TK;
      float s[TK];
      {
        float a[32], c[32];
        wide::tmem_ld<32>(t_s, a);
        wide::tmem_ld<32>(t_s + 32, c);
        wide::tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 32; ++k) { s[k] = a[k]; s[32 + k] = c[k]; }
      }
      if (t >= whole) {   // visible keys of the tile: [lo, hi)
        const int tt = t_lo + t;
        int lo = 0, hi = TK;
        if (tt < nt_c) {
          hi = lim - tt * TK;
        } else {
          const int y = own_lo + (tt - nt_c) * TK;
          lo = own_first - y;
          hi = r + 1 - y;
        }
        if (!pv) { lo = 0; hi = TK; }   // (nothing of these pairs is stored)
        seen |= min(hi, TK) > max(lo, 0);
        if (__any_sync(0xffffffffu, hi < TK)) {
#pragma unroll
          for (int k = 0; k < TK; ++k)
            if (k >= hi) s[k] = -INFINITY;
        }
        if (__any_sync(0xffffffffu, lo > 0)) {
#pragma unroll
          for (int k = 0; k < TK; ++k)
            if (k < lo) s[k] = -INFINITY;
        }
      }
      float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int k = 0; k < TK; k += 2) m4[(k >> 1) & 3] = max3(m4[(k >> 1) & 3], s[k], s[k + 1]);
      const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])) * scale;
      const bool grow = t > 0 && mx > m + LAZY;       // (also the first visible key of the row: m = -inf)
      if (t == 0) {
        m = mx;
      } else if (__any_sync(0xffffffffu, grow)) {
        // the outputs so far are rescaled: every P V issued so far (tile t - 1 is the last) has to be done
        if (!warp_wait(&sh->o_done[bl][(t - 1) & 1], ((t - 1) >> 1) & 1u)) break;
        const float corr = grow ? exp2f(m - mx) : 1.f;
        if (grow) { l *= corr; m = mx; }
#pragma unroll 1
        for (int c = 0; c < HD; c += 32) {
          float o[32];
          wide::tmem_ld<32>(t_o + c, o);
          wide::tmem_wait_ld();
          uint32_t u[32];
#pragma unroll
          for (int k = 0; k < 32; ++k) u[k] = __float_as_uint(o[k] * corr);
          wide::tmem_st32(t_o + c, u);
        }
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      }
      const float mm = m == -INFINITY ? 0.f : m - MANY_BITS;   // no visible key so far: all weights are exp2(-inf) = 0
      const float2 scale2v = make_float2(scale, scale), off2 = make_float2(-mm, -mm);
      float2 r2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
      uint32_t ph[32];
#pragma unroll
      for (int k = 0; k < TK; k += 2) {
        const float2 x = fma2(make_float2(s[k], s[k + 1]), scale2v, off2);
        const float2 e = make_float2(ex2(x.x), ex2(x.y));
        r2[(k >> 1) & 1] = add2(r2[(k >> 1) & 1], e);
        ph[k >> 1] = pack_half(e.x, e.y);
      }
      l += (r2[0].x + r2[0].y) + (r2[1].x + r2[1].y);
      wide::tmem_st32(t_s, ph);
      asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(tc::smem_u32(&sh->p_full[bl][t & 1])) : "memory");
    }
    if (ok && nt > 0) warp_wait(&sh->o_done[bl][(nt - 1) & 1], ((nt - 1) >> 1) & 1u);
    if (!ok) sh->abort = 1;
    if (ok) {
      // scores of minus infinity alone: a query with an infinity in it
      if (seen && l == 0.f) l = __int_as_float(0x7fffffff);
      // (poison was written before the last tile's barrier; NaN blocks among the keys this pair sees)
      uint32_t bad = 0;
      if (*(volatile int*)&sh->poison && pv) {
        const uint8_t* xc = p.v.scales + kvh * p.v.head_scales;
        const uint8_t* xo = p.own_v.scales + kvh * p.own_v.head_scales;
        const int k0 = t_lo * TK, k1 = min(lim, (t_lo + nt) * TK);
        for (int k = k0; k < k1; ++k)
#pragma unroll 1
          for (int j = 0; j < HD / BLOCK; ++j) bad |= (uint32_t)(xc[(long long)k * (HD / BLOCK) + j] == NAN_SCALE) << j;
        if (t_lo + nt > nt_c && p.own_n > 0)
          for (int k = max(own_first, own_lo + max(0, t_lo - nt_c) * TK); k <= min(r, own_lo + (t_lo + nt - nt_c) * TK - 1); ++k)
#pragma unroll 1
            for (int j = 0; j < HD / BLOCK; ++j)
              bad |= (uint32_t)(xo[(p.own_pos0 + k) * (HD / BLOCK) + j] == NAN_SCALE) << j;
      }
      const bool part = p.splits > 1;
      const float inv = part ? 1.f : (l == 0.f ? 0.f : 1.0f / l);
      // part: [item, split][dim][pair], neighbouring lanes side by side
      float* dst_part = p.part + (long long)blockIdx.x * HD * (NB * TP) + threadIdx.x;
      // out: a warp's 32 rows through shared memory (the queries' place: every multiply is done), so that whole rows go out
      constexpr int CPR = HD / 8;      // 16-byte pieces of a row
      uint8_t* stage = smem + warp * 32 * HD * 2;
#pragma unroll 1
      for (int c = 0; c < HD; c += 32) {
        float o[32];
        if (nt > 0) {
          wide::tmem_ld<32>(t_o + c, o);
          wide::tmem_wait_ld();
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = 0.f;
        }
        float f[32];
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          const int dim = (k & ~7) + ((k & 1) << 2) + ((k & 7) >> 1);   // columns hold dims 0 4 1 5 2 6 3 7 of each eight, 0 4 2 6 as sixteenths
          f[dim] = ((bad >> ((c + k) >> 4)) & 1u) ? __int_as_float(0x7fffffff) : o[k] * ((k & 2) ? inv : inv * 16.f);
        }
        if (part) {
#pragma unroll
          for (int k = 0; k < 32; ++k) dst_part[(c + k) * (NB * TP)] = f[k];
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            *reinterpret_cast<uint4*>(stage + lane * HD * 2 + (((c / 8 + k) ^ (lane & (CPR - 1))) << 4)) =
                make_uint4(pack_bf16(f[8 * k], f[8 * k + 1]), pack_bf16(f[8 * k + 2], f[8 * k + 3]),
                           pack_bf16(f[8 * k + 4], f[8 * k + 5]), pack_bf16(f[8 * k + 6], f[8 * k + 7]));
        }
      }
      if (part) {
        p.part_ml[(long long)blockIdx.x * (NB * TP) + threadIdx.x] = make_float2(m, l);
      } else {
        __syncwarp();
        const long long mine = pv ? (long long)r * p.out_stride + (long long)hq * HD : -1;
        const int col = lane & (CPR - 1);
#pragma unroll 4
        for (int i = 0; i < 32; i += 32 / CPR) {
          const int row = i + lane / CPR;
          const long long off = __shfl_sync(0xffffffffu, mine, row);
          const uint4 v = *reinterpret_cast<const uint4*>(stage + row * HD * 2 + ((col ^ (row & (CPR - 1))) << 4));
          if (off >= 0) *reinterpret_cast<uint4*>((bf16*)p.out + off + col * 8) = v;
        }
      }
    }
  }

  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (sh->abort)
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  if (warp == W_MMA) {
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TM_COLS) : "memory");
  }
}

// The parts of each pair of attn_many_kernel, in their order: eight pairs per CTA (whole sectors of the parts, where pairs lie side
// by side), a thread takes HD / 32 dims of one -- two where the parts are many and the pairs few --, and the rows go out through
// shared memory.  (A thread per four dims of a pair, pairs
// on neighbouring lanes, left an eighth of a sector per store: 28 us where 400 rows of 32 heads were cut in two.)  All parts are fetched
// at once up to BATCH of them: 3, 9 or 18, since what is not there costs its instructions too (400 rows in two parts 18 / 20 / 27 us
// with the attention, twelve states in 18 parts 24.7 / 21.5 / 19.2).
constexpr int MAX_SPLITS = 148;
template <int HD, int BATCH> constexpr int merge_dims = BATCH > 9 ? 64 : HD;
template <int HD, int NB, int BATCH>
__global__ void __launch_bounds__(256) merge_kernel(const __grid_constant__ AttnArgs p) {
  constexpr int PAIRS = NB * TP, GROUP = 8, DIMS = merge_dims<HD, BATCH>, E = DIMS / 32, PER = PAIRS / GROUP * (HD / DIMS);
  __shared__ float w_sm[MAX_SPLITS][GROUP], den_sm[GROUP];
  __shared__ __align__(16) float o_sm[GROUP][DIMS + 4];
  const int item = blockIdx.x / PER, first = blockIdx.x % PER / (HD / DIMS) * GROUP, dim0 = blockIdx.x % (HD / DIMS) * DIMS;
  const int Gq = p.nq / p.nkv;
  const int kvh = item % p.nkv, pair0 = (p.blocks - 1 - item / p.nkv) * PAIRS + first;
  asm volatile("griddepcontrol.wait;" ::: "memory");   // (launched while the parts are still being made)
  if (pair0 >= p.R * Gq) return;
  const int pair = threadIdx.x % GROUP, d0 = threadIdx.x / GROUP;
  const float* src = p.part + ((long long)item * p.splits * HD + dim0 + d0) * PAIRS + first + pair;
  float x[BATCH][E];                       // the parts on their way, BATCH at a time
  auto load = [&](int i0) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b)
#pragma unroll
      for (int e = 0; e < E; ++e) x[b][e] = i0 + b < p.splits ? __ldcg(src + ((long long)(i0 + b) * HD + e * 32) * PAIRS) : 0.f;
  };
  load(0);
  {                                        // the parts' weights: a warp per pair, a lane per part
    const int w = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const float2* ml = p.part_ml + (long long)item * p.splits * PAIRS + first + w;
    float mx = -INFINITY, sum = 0.f;
#pragma unroll 1
    for (int i = lane; i < p.splits; i += 32) mx = fmaxf(mx, __ldcg(ml + i * PAIRS).x);
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, e));
#pragma unroll 1
    for (int i = lane; i < p.splits; i += 32) {
      const float2 v = __ldcg(ml + i * PAIRS);
      const float f = v.x == -INFINITY ? (v.y == v.y ? 0.f : 1.f) : exp2f(v.x - mx);   // (a sum without a maximum is 0, or NaN)
      w_sm[i][w] = f;
      sum = fmaf(v.y, f, sum);
    }
#pragma unroll
    for (int e = 16; e > 0; e >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, e);
    if (lane == 0) den_sm[w] = sum;
  }
  __syncthreads();
  const float den = den_sm[pair];
  float a[E];
#pragma unroll
  for (int e = 0; e < E; ++e) a[e] = 0.f;
#pragma unroll 1
  for (int i0 = 0; i0 < p.splits; i0 += BATCH) {
    if (i0 > 0) load(i0);
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const float f = i0 + b < p.splits ? w_sm[i0 + b][pair] : 0.f;
#pragma unroll
      for (int e = 0; e < E; ++e) a[e] = fmaf(f, x[b][e], a[e]);
    }
  }
  const float inv = den == 0.f ? 0.f : 1.0f / den;
#pragma unroll
  for (int e = 0; e < E; ++e) o_sm[pair][d0 + e * 32] = a[e] * inv;
  __syncthreads();
  const int row = threadIdx.x / (DIMS / 8), c = threadIdx.x % (DIMS / 8) * 8, pp = pair0 + row;
  if (row >= GROUP || pp >= p.R * Gq) return;
  const float4 u = *reinterpret_cast<const float4*>(&o_sm[row][c]), v = *reinterpret_cast<const float4*>(&o_sm[row][c + 4]);
  const int r = pp / Gq;
  *reinterpret_cast<uint4*>((bf16*)p.out + (long long)r * p.out_stride + (long long)(kvh * Gq + pp - r * Gq) * HD + dim0 + c) =
      make_uint4(pack_bf16(u.x, u.y), pack_bf16(u.z, u.w), pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}

}  // namespace kv4
}  // namespace clasp
