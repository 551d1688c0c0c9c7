// Writing K and V rows into a cache held in 8 bits, and reading them back.
//
// Write: x -> code, with one scale per block of tokens and KV head, s = amax / 127 (int8) or the least power of two that
// brings amax to 448 (e4m3).  A block of threads takes one (block of tokens, KV head) of K or of V: it holds the rows in
// registers from the one time they are read, finds their largest magnitude, and writes the codes; nothing is read twice.
// Where the block of tokens was begun by an earlier call its scale can only grow, and when it does the tokens that are
// there are read back and quantised again.  Read: value = code * scale.  Both move bytes and do little else: HBM bounds them
// (2 + 1 bytes per element of a bf16 write, 1 + 2 of a read).
#include "dam_cache.cuh"

namespace {

constexpr int kCThreads = 256;
constexpr int kReadTokens = 64;        // packed tokens of a read's slot

// 8 consecutive elements as fp32
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float* x) {
  const uint4 a = __ldcs(reinterpret_cast<const uint4*>(p));
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void load8(const float* p, float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p) + i);
    x[4 * i] = a.x; x[4 * i + 1] = a.y; x[4 * i + 2] = a.z; x[4 * i + 3] = a.w;
  }
}
__device__ __forceinline__ void store8(__nv_bfloat16* p, const float* x) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float* p, const float* x) {
#pragma unroll
  for (int i = 0; i < 2; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
}
template <int CODE>
__device__ __forceinline__ uint2 codes8(const float* x, float s, float inv) {
  uint32_t w[2];
#pragma unroll
  for (int i = 0; i < 2; ++i)
    w[i] = cache_code<CODE>(x[4 * i], s, inv) | cache_code<CODE>(x[4 * i + 1], s, inv) << 8 | cache_code<CODE>(x[4 * i + 2], s, inv) << 16 |
           cache_code<CODE>(x[4 * i + 3], s, inv) << 24;
  return make_uint2(w[0], w[1]);
}

// start of sequence b's range, and whether the range [start, start + n) lies inside its capacity (an empty one always does)
__device__ __forceinline__ bool range_fits(const DamCacheView& c, const int32_t* starts, int b, int n, int* start) {
  *start = starts ? __ldg(starts + b) : 0;
  return n == 0 || (*start >= 0 && *start <= __ldg(c.cu + b + 1) - __ldg(c.cu + b) - n);
}
// the scratch block of the whole call, its status word included (one block of threads looks at every sequence)
__device__ __forceinline__ void report_ranges(const DamCacheView& c, const int32_t* tok_cu, const int32_t* starts, uint32_t* scratch) {
  bool bad = false;
  for (int b = threadIdx.x; b < c.num_seqs; b += kCThreads) {
    int start;
    bad |= !range_fits(c, starts, b, __ldg(tok_cu + b + 1) - __ldg(tok_cu + b), &start);
  }
  const int st = __syncthreads_or(bad) ? (int)DAM_ERR_INVALID_ARGUMENT : 0;
  if (threadIdx.x < 64) scratch[threadIdx.x] = threadIdx.x == 1 ? (uint32_t)st : 0u;
}

struct CacheRows {               // K and V rows of the packed tokens
  const void *K, *V;
  int64_t kst, ksh, vst, vsh;    // elements
  const int32_t* cu;
};

// grid: (slot, K or V, KV head), the head fastest.  PASSES: rows of a block of tokens that a thread holds 8 elements of.
template <typename T, int D, int CODE, int PASSES>
__global__ void __launch_bounds__(kCThreads)
cache_write_kernel(CacheRows src, const int32_t* __restrict__ starts, DamCacheView c, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  constexpr int TPR = D / 8, RPP = kCThreads / TPR;          // threads of a row, rows of a pass
  __shared__ uint32_t warp_max[kCThreads / 32];
  if (blockIdx.x == 0) report_ranges(c, src.cu, starts, scratch);
  const int h = blockIdx.x % c.Hkv, kv = blockIdx.x / c.Hkv & 1;
  const int64_t slot = blockIdx.x / (2 * c.Hkv);
  const int b = cache_seq_of_slot(src.cu, c.num_seqs, c.shift, 2, slot);
  const int t0 = __ldg(src.cu + b), n = __ldg(src.cu + b + 1) - t0, cap0 = __ldg(c.cu + b);
  int start;
  if (!range_fits(c, starts, b, n, &start) || n == 0) return;
  const int first = start >> c.shift;
  const int64_t j64 = first + (slot - ((t0 >> c.shift) + 2ll * b));
  if (j64 > (start + n - 1) >> c.shift) return;
  const int j = (int)j64, p0 = j << c.shift, p1 = min(p0 + (1 << c.shift), start + n), lo = max(p0, start);
  const T* x = reinterpret_cast<const T*>(kv ? src.V : src.K) + (int64_t)t0 * (kv ? src.vst : src.kst) + (int64_t)h * (kv ? src.vsh : src.ksh);
  const int64_t xst = kv ? src.vst : src.kst, cst = kv ? c.vst : c.kst;
  unsigned char* codes = (kv ? c.v : c.k) + (int64_t)cap0 * cst + (int64_t)h * (kv ? c.vsh : c.ksh);
  float* scale = (kv ? c.vs : c.ks) + (int64_t)((cap0 >> c.shift) + b + j) * c.Hkv + h;
  const int tid = threadIdx.x, r0 = tid / TPR, e = tid % TPR * 8;
  const float before = lo > p0 ? *scale : 0.f;
  float v[PASSES][8];
  uint32_t top = 0u;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int p = p0 + r0 + i * RPP;
#pragma unroll
    for (int k = 0; k < 8; ++k) v[i][k] = 0.f;
    if (p >= lo && p < p1) load8(x + (int64_t)(p - start) * xst + e, v[i]);
  }
  // the largest magnitude, as bits: an infinity or a NaN is larger than any number
#pragma unroll
  for (int i = 0; i < PASSES; ++i)
#pragma unroll
    for (int k = 0; k < 8; ++k) top = max(top, __float_as_uint(v[i][k]) & 0x7FFFFFFFu);
  top = __reduce_max_sync(0xFFFFFFFFu, top);
  if ((tid & 31) == 0) warp_max[tid >> 5] = top;
  __syncthreads();                                           // (every thread has read the old scale, too)
#pragma unroll
  for (int w = 0; w < kCThreads / 32; ++w) top = max(top, warp_max[w]);
  float s = cache_scale<CODE>(top);
  if (lo > p0) s = s != s || before != before ? dam_cache_nan() : fmaxf(before, s);
  const bool ok = s == s;
  const float inv = ok ? 1.f / s : 0.f;
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int p = p0 + r0 + i * RPP;
    if (p >= lo && p < p1)
      *reinterpret_cast<uint2*>(codes + (int64_t)p * cst + e) = ok ? codes8<CODE>(v[i], s, inv) : make_uint2(0u, 0u);
  }
  if (lo > p0 && s > before) {
    // the scale grew: the tokens that are there are read back and quantised again (every thread its own 8 elements)
    for (int p = p0 + r0; p < lo; p += RPP) {
      uint2* at = reinterpret_cast<uint2*>(codes + (int64_t)p * cst + e);
      const uint2 old = *at;
      float f[8];
      codes_to_float<CODE>(old.x, f);
      codes_to_float<CODE>(old.y, f + 4);
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] *= before;
      *at = codes8<CODE>(f, s, inv);
    }
  }
  if (tid == 0) *scale = s;
}

// grid: (slot of kReadTokens packed tokens, K or V, KV head), the head fastest
template <typename T, int D, int CODE>
__global__ void __launch_bounds__(kCThreads)
cache_read_kernel(CacheRows dst, const int32_t* __restrict__ starts, DamCacheView c, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  constexpr int TPR = D / 8, RPP = kCThreads / TPR, PASSES = kReadTokens / RPP;
  if (blockIdx.x == 0) report_ranges(c, dst.cu, starts, scratch);
  const int h = blockIdx.x % c.Hkv, kv = blockIdx.x / c.Hkv & 1;
  const int64_t slot = blockIdx.x / (2 * c.Hkv);
  constexpr int kShift = 6;
  static_assert(1 << kShift == kReadTokens, "slots are counted by a shift");
  const int b = cache_seq_of_slot(dst.cu, c.num_seqs, kShift, 1, slot);
  const int t0 = __ldg(dst.cu + b), n = __ldg(dst.cu + b + 1) - t0, cap0 = __ldg(c.cu + b);
  int start;
  const bool fits = range_fits(c, starts, b, n, &start);
  const int64_t base64 = (slot - ((t0 >> kShift) + (int64_t)b)) * kReadTokens;
  if (base64 >= n) return;
  const int base = (int)base64;
  const int tid = threadIdx.x, r0 = tid / TPR, e = tid % TPR * 8;
  const int64_t xst = kv ? dst.vst : dst.kst, cst = kv ? c.vst : c.kst;
  T* x = reinterpret_cast<T*>(const_cast<void*>(kv ? dst.V : dst.K)) + (int64_t)t0 * xst + (int64_t)h * (kv ? dst.vsh : dst.ksh) + e;
  if (!fits) {                                               // nothing of this sequence can be read: zeros
    const float zero[8] = {};
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int t = base + r0 + i * RPP;
      if (t < n) store8(x + (int64_t)t * xst, zero);
    }
    return;
  }
  const unsigned char* codes = (kv ? c.v : c.k) + ((int64_t)cap0 + start) * cst + (int64_t)h * (kv ? c.vsh : c.ksh) + e;
  const float* scales = (kv ? c.vs : c.ks) + (int64_t)((cap0 >> c.shift) + b) * c.Hkv + h;
  uint2 w[PASSES];
  float s[PASSES];
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int t = base + r0 + i * RPP;
    w[i] = make_uint2(0u, 0u);
    s[i] = 0.f;
    if (t < n) {
      w[i] = __ldcs(reinterpret_cast<const uint2*>(codes + (int64_t)t * cst));
      s[i] = __ldg(scales + (int64_t)((start + t) >> c.shift) * c.Hkv);
    }
  }
#pragma unroll
  for (int i = 0; i < PASSES; ++i) {
    const int t = base + r0 + i * RPP;
    float f[8];
    codes_to_float<CODE>(w[i].x, f);
    codes_to_float<CODE>(w[i].y, f + 4);
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] *= s[i];
    if (t < n) store8(x + (int64_t)t * xst, f);
  }
}

CacheRows rows_of(const void* K, const void* V, const dam_shape_t* t) {
  return {K, V, t->k_stride_tok, t->k_stride_head, t->v_stride_tok, t->v_stride_head, t->cu_seqlens_dev};
}

template <typename T, int D, int CODE>
cudaError_t launch_write(const CacheRows& src, const int32_t* starts, const DamCacheView& c, int64_t grid, uint32_t* scratch, cudaStream_t st) {
  const int passes = ((1 << c.shift) * (D / 8) + kCThreads - 1) / kCThreads;
  void (*k)(CacheRows, const int32_t*, DamCacheView, uint32_t*) =
      passes <= 1 ? cache_write_kernel<T, D, CODE, 1> : passes == 2 ? cache_write_kernel<T, D, CODE, 2>
      : passes == 4 ? cache_write_kernel<T, D, CODE, 4> : cache_write_kernel<T, D, CODE, 8>;
  return dam_launch_chained(k, dim3((unsigned)grid), dim3(kCThreads), 0, st, src, starts, c, scratch);
}

template <typename T, int D, int CODE>
cudaError_t launch_read(const CacheRows& dst, const int32_t* starts, const DamCacheView& c, int64_t grid, uint32_t* scratch, cudaStream_t st) {
  return dam_launch_chained(cache_read_kernel<T, D, CODE>, dim3((unsigned)grid), dim3(kCThreads), 0, st, dst, starts, c, scratch);
}

}  // namespace

cudaError_t dam_launch_cache_write(const void* K, const void* V, const dam_shape_t* tokens, const int32_t* starts, const dam_cache_t* cache,
                                   void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  // a sequence's tokens touch at most (n - 2) / block + 2 blocks: its slots are two more than the difference of cu / block
  const int64_t slots = (tokens->total_tokens >> c.shift) + 2ll * c.num_seqs, grid = slots * 2 * c.Hkv;
  if (grid > 0x7FFFFFFF) return cudaErrorNotSupported;
  return DAM_CACHE_DISPATCH(launch_write, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c, grid,
                            reinterpret_cast<uint32_t*>(scratch), st);
}

cudaError_t dam_launch_cache_read(const dam_cache_t* cache, const dam_shape_t* tokens, const int32_t* starts, void* K, void* V,
                                  void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  const int64_t slots = tokens->total_tokens / kReadTokens + (int64_t)c.num_seqs, grid = slots * 2 * c.Hkv;
  if (grid > 0x7FFFFFFF) return cudaErrorNotSupported;
  return DAM_CACHE_DISPATCH(launch_read, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c, grid,
                            reinterpret_cast<uint32_t*>(scratch), st);
}
