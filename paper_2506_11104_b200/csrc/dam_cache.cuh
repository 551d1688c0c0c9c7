// The KV cache held in 8 bits: how the kernels see it, and the arithmetic of its codes and scales (dam.h states the rule).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "dam_internal.cuh"

// dam_cache_t as the kernels take it, by value.  The scales of block j of sequence b stand in row cu[b] / block + b + j.
struct DamCacheView {
  const int32_t* cu;
  int32_t num_seqs, Hkv;
  int32_t shift;                 // log2 of block_tokens
  unsigned char *k, *v;
  float *ks, *vs;
  int64_t kst, ksh, vst, vsh;    // bytes
};

inline DamCacheView dam_cache_view(const dam_cache_t* c) {
  DamCacheView v;
  v.cu = c->cu_seqlens_dev; v.num_seqs = c->num_seqs; v.Hkv = c->num_kv_heads;
  v.shift = 0;
  while ((1 << v.shift) < c->block_tokens) ++v.shift;
  v.k = reinterpret_cast<unsigned char*>(c->k_codes); v.v = reinterpret_cast<unsigned char*>(c->v_codes);
  v.ks = c->k_scales; v.vs = c->v_scales;
  v.kst = c->k_stride_tok; v.ksh = c->k_stride_head; v.vst = c->v_stride_tok; v.vsh = c->v_stride_head;
  return v;
}

// ---- codes -> values ----------------------------------------------------------------------------
// Two e4m3 codes (low byte first) as two fp16 numbers: exact, fp16 has more exponent and mantissa bits.
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t codes16) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)codes16));
  return h;
}
// Two int8 codes that were XORed with 0x80 (so they read c + 128) and placed under the byte 0x64, i.e. the fp16 numbers
// 1024 + 128 + c, whose spacing is 1: minus 1152 is c, exactly.
__device__ __forceinline__ uint32_t biased_to_half2(uint32_t h) {
  uint32_t r;
  asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(h), "r"(0x64806480u));
  return r;
}
// Two fp32 numbers at a time.
struct F2 {
  uint64_t v;
  __device__ __forceinline__ F2() {}
  __device__ __forceinline__ F2(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y)); }
  __device__ __forceinline__ void get(float& x, float& y) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
};
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v)); return r; }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v)); return r; }

// The values of the four codes of a word under the scale s.
template <int CODE>
__device__ __forceinline__ void code_values(uint32_t w, float s, float* f) {
  F2 lo, hi;
  if constexpr (CODE == DAM_CODE_INT8) {
    // 2^23 + 128 + c as fp32 bits, minus 2^23 + 128
    w ^= 0x80808080u;
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) u[k] = __byte_perm(w, 0x4B000000u, 0x7440 | k);
    const F2 bias(-8388736.f, -8388736.f);
    lo = add2(F2(__uint_as_float(u[0]), __uint_as_float(u[1])), bias);
    hi = add2(F2(__uint_as_float(u[2]), __uint_as_float(u[3])), bias);
  } else {
    const uint32_t a = e4m3x2_to_half2(w & 0xFFFFu), b = e4m3x2_to_half2(w >> 16);
    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&a)), y = __half22float2(*reinterpret_cast<const __half2*>(&b));
    lo = F2(x.x, x.y); hi = F2(y.x, y.y);
  }
  const F2 scale(s, s);
  mul2(lo, scale).get(f[0], f[1]);
  mul2(hi, scale).get(f[2], f[3]);
}

// ---- values -> codes ----------------------------------------------------------------------------
__device__ __forceinline__ float dam_cache_nan() { return __uint_as_float(0x7FC00000u); }

// The scale of a block whose largest magnitude has the bits `amax` (sign bit clear).  A block with an infinity or a NaN has
// none: its scale is a NaN, and so is every value read back from it.
template <int CODE>
__device__ __forceinline__ float cache_scale(uint32_t amax) {
  if (amax >= 0x7F800000u) return dam_cache_nan();
  if constexpr (CODE == DAM_CODE_INT8) {
    return fmaxf(__fdiv_rn(__uint_as_float(amax), 127.f), 1.17549435e-38f);
  } else {
    // amax = M 2^E: the least k with M 2^E <= 1.75 * 2^8 * 2^k is E - 8, plus 1 when M > 1.75 (mantissa bits above 0x600000)
    const int e = (int)((amax + 0x1FFFFFu) >> 23) - 8;
    return __uint_as_float((uint32_t)(e < 1 ? 1 : e) << 23);
  }
}

// What makes codes of values under one scale.
template <int CODE>
struct Coder {
  float s;
  F2 lo, hi;                     // int8: 1 / s, a little less and a little more; e4m3: 1 / s
  __device__ __forceinline__ explicit Coder(float scale) : s(scale) {
    const float inv = 1.f / scale;
    if constexpr (CODE == DAM_CODE_INT8) {
      const float a = inv * (1.f - 2.3841858e-7f), b = inv * (1.f + 2.3841858e-7f);      // (2^-22)
      lo = F2(a, a);
      hi = F2(b, b);
    } else {
      lo = F2(inv, inv);
    }
  }
  // The codes of eight values.
  __device__ __forceinline__ uint2 eight(const float* x) const {
    uint32_t w[2];
    if constexpr (CODE == DAM_CODE_INT8) {
      // The nearest integer to x / s, ties to even, of the exact quotient: x times a little less and a little more than 1 / s
      // enclose it (1 / s and the two factors are off by 2^-23 together), so where both round to the same integer (the sum with
      // 1.5 * 2^23 does that; its low byte is the code), the quotient does.  Otherwise x is next to a border of two codes.
      constexpr float kMagic = 12582912.f;
      const F2 magic(kMagic, kMagic);
      float t[8];
      uint32_t differ = 0u;
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        const F2 v(x[k], x[k + 1]);
        float a, b;
        fma2(v, lo, magic).get(t[k], t[k + 1]);
        fma2(v, hi, magic).get(a, b);
        differ |= __float_as_uint(t[k]) ^ __float_as_uint(a);
        differ |= __float_as_uint(t[k + 1]) ^ __float_as_uint(b);
      }
      if (differ) {                      // (of bf16 values: one that is an exact tie, or amax / 2)
        // x - q s is s / 2 there, or next to it, and the difference is exact: a multiple of half an ulp of s.  Twice the difference
        // is compared with s: half of an s below 2^-125 may be no fp32 number.
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float q = t[k] - kMagic, twice = 2.f * fmaf(-q, s, x[k]);
          const bool odd = (__float_as_uint(t[k]) & 1u) != 0;
          const float far = fabsf(twice);
          // (the next float is the next integer there)
          if (far > s || (far == s && odd)) t[k] = __uint_as_float(__float_as_uint(t[k]) + (twice < 0.f ? -1 : 1));
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t a = __byte_perm(__float_as_uint(t[4 * i]), __float_as_uint(t[4 * i + 1]), 0x0040);
        const uint32_t b = __byte_perm(__float_as_uint(t[4 * i + 2]), __float_as_uint(t[4 * i + 3]), 0x0040);
        w[i] = __byte_perm(a, b, 0x5410);
      }
    } else {
      // (the scale is a power of two: x / s is exact, or so small that its code is zero)
      uint16_t h[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float a, b;
        mul2(F2(x[2 * i], x[2 * i + 1]), lo).get(a, b);
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(h[i]) : "f"(b), "f"(a));
      }
      w[0] = (uint32_t)h[0] | (uint32_t)h[1] << 16;
      w[1] = (uint32_t)h[2] | (uint32_t)h[3] << 16;
    }
    return make_uint2(w[0], w[1]);
  }
};

// ---- which sequence -----------------------------------------------------------------------------
// The work of a packed batch is cut into slots: sequence b owns the slots (cu[b] >> shift) + extra * b onwards, up to the next
// sequence's.  Returns the sequence of a slot (whole warp; a step looks at 32 places at once).
__device__ __forceinline__ int cache_seq_of_slot(const int32_t* __restrict__ cu, int n, int shift, int extra, int64_t slot) {
  int lo = 0, hi = n;
  const int lane = threadIdx.x & 31;
  while (hi - lo > 1) {
    const int step = (hi - lo + 31) >> 5, b = lo + lane * step;
    const bool here = b < hi && (int64_t)(__ldg(cu + b) >> shift) + (int64_t)extra * b <= slot;
    const int cnt = __popc(__ballot_sync(0xFFFFFFFFu, here));
    lo += (cnt - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// ---- host: dispatch ----------------------------------------------------------------------------
// FN<T, D, CODE>(...) for the types at hand
#define DAM_CACHE_DISPATCH(FN, dtype, dim, code, ...)                                                                          \
  (dtype == DAM_BF16 ? (dim == 128 ? (code == DAM_CODE_INT8 ? FN<__nv_bfloat16, 128, DAM_CODE_INT8>(__VA_ARGS__)               \
                                                            : FN<__nv_bfloat16, 128, DAM_CODE_E4M3>(__VA_ARGS__))              \
                                   : (code == DAM_CODE_INT8 ? FN<__nv_bfloat16, 64, DAM_CODE_INT8>(__VA_ARGS__)                \
                                                            : FN<__nv_bfloat16, 64, DAM_CODE_E4M3>(__VA_ARGS__)))              \
                     : (dim == 128 ? (code == DAM_CODE_INT8 ? FN<float, 128, DAM_CODE_INT8>(__VA_ARGS__)                       \
                                                            : FN<float, 128, DAM_CODE_E4M3>(__VA_ARGS__))                      \
                                   : (code == DAM_CODE_INT8 ? FN<float, 64, DAM_CODE_INT8>(__VA_ARGS__)                        \
                                                            : FN<float, 64, DAM_CODE_E4M3>(__VA_ARGS__))))

// ---- launch entry points ------------------------------------------------------------------------
cudaError_t dam_launch_cache_write(const void* K, const void* V, const dam_shape_t* tokens, const int32_t* starts, const dam_cache_t* cache,
                                   void* scratch, cudaStream_t st);
cudaError_t dam_launch_cache_read(const dam_cache_t* cache, const dam_shape_t* tokens, const int32_t* starts, void* K, void* V,
                                  void* scratch, cudaStream_t st);
// bytes of scratch that the attention over a cache wants (partial results of sequences that several blocks share)
size_t dam_cache_scratch_bytes(int head_dim);
cudaError_t dam_launch_cache_decode(const void* q, const dam_cache_t* cache, const void* mask, const int32_t* positions, int Hq, int dtype,
                                    float scale, void* O, float* lse, void* scratch, cudaStream_t st);
