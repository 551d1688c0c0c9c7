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

// 8 consecutive elements as they are in memory, and as fp32
template <typename T> struct Eight;
template <> struct Eight<__nv_bfloat16> {
  uint4 a;
  __device__ __forceinline__ void clear() { a = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { a = __ldcs(reinterpret_cast<const uint4*>(p)); }
  __device__ __forceinline__ void floats(float* x) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(w[i] << 16); x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
  }
  // largest magnitudes so far, two at a time: as bits, where an infinity or a NaN is larger than any number
  __device__ __forceinline__ void top(uint32_t& t) const {
    t = __vmaxu2(__vmaxu2(t, a.x & 0x7FFF7FFFu), a.y & 0x7FFF7FFFu);
    t = __vmaxu2(__vmaxu2(t, a.z & 0x7FFF7FFFu), a.w & 0x7FFF7FFFu);
  }
  static __device__ __forceinline__ uint32_t joined(uint32_t t) { return max(t << 16, t & 0xFFFF0000u); }
  static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* x) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
  }
};
template <> struct Eight<float> {
  float4 a, b;
  __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void load(const float* p) { a = __ldcs(reinterpret_cast<const float4*>(p)); b = __ldcs(reinterpret_cast<const float4*>(p) + 1); }
  __device__ __forceinline__ void floats(float* x) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ __forceinline__ void top(uint32_t& t) const {
    float x[8];
    floats(x);
#pragma unroll
    for (int k = 0; k < 8; ++k) t = max(t, __float_as_uint(x[k]) & 0x7FFFFFFFu);
  }
  static __device__ __forceinline__ uint32_t joined(uint32_t t) { return t; }
  static __device__ __forceinline__ void store(float* p, const float* x) {
#pragma unroll
    for (int i = 0; i < 2; ++i) reinterpret_cast<float4*>(p)[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
  }
};

// The scale of a block from its new tokens' largest magnitude, and, where it was begun before, from the scale it has.
template <int CODE>
__device__ __forceinline__ float block_scale(uint32_t top, bool begun, float before) {
  const float s = cache_scale<CODE>(top);
  if (!begun) return s;
  return s != s || before != before ? dam_cache_nan() : fmaxf(before, s);
}
// eight elements of a token that is there already, from the scale `before` to the scale s
template <int CODE>
__device__ __forceinline__ void requantise(unsigned char* p, float before, float s, float inv) {
  uint2* at = reinterpret_cast<uint2*>(p);
  const uint2 old = *at;
  float f[8];
  codes_to_float<CODE>(old.x, f);
  codes_to_float<CODE>(old.y, f + 4);
#pragma unroll
  for (int k = 0; k < 8; ++k) f[k] *= before;
  *at = cache_codes8<CODE>(f, s, inv);
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

// One (block of tokens, K or V, KV head) of a write.
template <typename T>
struct WriteUnit {
  const T* x;                    // row of token `start`
  unsigned char* codes;          // row of token 0
  float* scale;
  int64_t xst, cst;
  int p0, lo, p1, start;         // the block's first token; its new tokens lo .. p1 - 1
  // unit u of the grid's list: (slot, K or V, KV head), the head fastest.  False: nothing to do there.  (whole warp)
  __device__ __forceinline__ bool find(const CacheRows& src, const int32_t* starts, const DamCacheView& c, uint32_t u) {
    const int h = u % c.Hkv, kv = u / c.Hkv & 1;
    const int64_t slot = u / (2 * c.Hkv);
    const int b = cache_seq_of_slot(src.cu, c.num_seqs, c.shift, 2, slot);
    const int t0 = __ldg(src.cu + b), n = __ldg(src.cu + b + 1) - t0, cap0 = __ldg(c.cu + b);
    if (!range_fits(c, starts, b, n, &start) || n == 0) return false;
    const int64_t j = (start >> c.shift) + (slot - ((t0 >> c.shift) + 2ll * b));
    if (j > (start + n - 1) >> c.shift) return false;
    p0 = (int)j << c.shift; p1 = min(p0 + (1 << c.shift), start + n); lo = max(p0, start);
    xst = kv ? src.vst : src.kst; cst = kv ? c.vst : c.kst;
    x = reinterpret_cast<const T*>(kv ? src.V : src.K) + (int64_t)t0 * xst + (int64_t)h * (kv ? src.vsh : src.ksh);
    codes = (kv ? c.v : c.k) + (int64_t)cap0 * cst + (int64_t)h * (kv ? c.vsh : c.ksh);
    scale = (kv ? c.vs : c.ks) + ((cap0 >> c.shift) + b + j) * c.Hkv + h;
    return true;
  }
};

// PASSES: rows of a block of tokens that a thread holds 8 elements of.  The blocks of threads stay and take one unit after
// another; the rows of the next are on their way while this one's are quantised.
template <typename T, int D, int CODE, int PASSES>
__global__ void __launch_bounds__(kCThreads, PASSES * sizeof(T) <= 8 ? 5 : PASSES * sizeof(T) <= 16 ? 3 : 2)
cache_write_kernel(CacheRows src, const int32_t* __restrict__ starts, DamCacheView c, uint32_t units, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  constexpr int TPR = D / 8, RPP = kCThreads / TPR;          // threads of a row, rows of a pass
  __shared__ uint32_t warp_max[2][kCThreads / 32];
  if (blockIdx.x == 0) report_ranges(c, src.cu, starts, scratch);
  const int tid = threadIdx.x, r0 = tid / TPR, e = tid % TPR * 8;
  WriteUnit<T> cur, nxt;
  Eight<T> v[PASSES], w[PASSES];
  float before = 0.f, before_next = 0.f;
  auto load = [&](const WriteUnit<T>& y, Eight<T>* r, float& b) {
    b = y.lo > y.p0 ? *reinterpret_cast<const volatile float*>(y.scale) : 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int p = y.p0 + r0 + i * RPP;
      r[i].clear();
      if (p >= y.lo && p < y.p1) r[i].load(y.x + (int64_t)(p - y.start) * y.xst + e);
    }
  };
  uint32_t u = blockIdx.x;
  bool have = false;
  while (u < units && !(have = cur.find(src, starts, c, u))) u += gridDim.x;
  if (have) load(cur, v, before);
  int turn = 0;
  while (have) {
    bool more = false;
    u += gridDim.x;                                          // (units and the grid together stay below 2^32)
    while (u < units && !(more = nxt.find(src, starts, c, u))) u += gridDim.x;
    if (more) load(nxt, w, before_next);
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) v[i].top(top);
    top = __reduce_max_sync(0xFFFFFFFFu, Eight<T>::joined(top));
    if ((tid & 31) == 0) warp_max[turn][tid >> 5] = top;
    __syncthreads();                                         // (every thread has read the old scale, too)
#pragma unroll
    for (int k = 0; k < kCThreads / 32; ++k) top = max(top, warp_max[turn][k]);
    const float s = block_scale<CODE>(top, cur.lo > cur.p0, before);
    const bool ok = s == s;
    const float inv = ok ? 1.f / s : 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int p = cur.p0 + r0 + i * RPP;
      if (p >= cur.lo && p < cur.p1) {
        float x[8];
        v[i].floats(x);
        *reinterpret_cast<uint2*>(cur.codes + (int64_t)p * cur.cst + e) = ok ? cache_codes8<CODE>(x, s, inv) : make_uint2(0u, 0u);
      }
    }
    // where the scale grew the tokens that are there are read back and quantised again (every thread its own 8 elements)
    if (cur.lo > cur.p0 && s > before) {
#pragma unroll 1
      for (int p = cur.p0 + r0; p < cur.lo; p += RPP) requantise<CODE>(cur.codes + (int64_t)p * cur.cst + e, before, s, inv);
    }
    if (tid == 0) *cur.scale = s;
    cur = nxt; before = before_next; have = more; turn ^= 1;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) v[i] = w[i];
  }
}

// One token per sequence at most (a generation step): a warp per (sequence, K or V, KV head).
template <typename T, int D, int CODE>
__global__ void __launch_bounds__(128)
cache_write_one_kernel(CacheRows src, const int32_t* __restrict__ starts, DamCacheView c, uint32_t units, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  if (blockIdx.x == 0) {
    bool bad = false;
    for (int b = threadIdx.x; b < c.num_seqs; b += 128) {
      int start;
      bad |= !range_fits(c, starts, b, __ldg(src.cu + b + 1) - __ldg(src.cu + b), &start);
    }
    const int st = __syncthreads_or(bad) ? (int)DAM_ERR_INVALID_ARGUMENT : 0;
    if (threadIdx.x < 64) scratch[threadIdx.x] = threadIdx.x == 1 ? (uint32_t)st : 0u;
  }
  const uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (u >= units) return;
  constexpr int TPR = D / 8;
  const int lane = threadIdx.x & 31, r0 = lane / TPR, e = lane % TPR * 8;
  const int h = u % c.Hkv, kv = u / c.Hkv & 1, b = u / (2 * c.Hkv);
  const int t0 = __ldg(src.cu + b), n = __ldg(src.cu + b + 1) - t0, cap0 = __ldg(c.cu + b);
  int start;
  if (!range_fits(c, starts, b, n, &start) || n == 0) return;
  const int p0 = start >> c.shift << c.shift;
  const int64_t cst = kv ? c.vst : c.kst;
  unsigned char* codes = (kv ? c.v : c.k) + (int64_t)cap0 * cst + (int64_t)h * (kv ? c.vsh : c.ksh) + e;
  float* scale = (kv ? c.vs : c.ks) + (int64_t)((cap0 >> c.shift) + b + (start >> c.shift)) * c.Hkv + h;
  const float before = start > p0 ? *scale : 0.f;
  Eight<T> v;
  v.load(reinterpret_cast<const T*>(kv ? src.V : src.K) + (int64_t)t0 * (kv ? src.vst : src.kst) + (int64_t)h * (kv ? src.vsh : src.ksh) + e);
  uint32_t top = 0u;
  v.top(top);
  top = __reduce_max_sync(0xFFFFFFFFu, Eight<T>::joined(top));
  const float s = block_scale<CODE>(top, start > p0, before);
  const bool ok = s == s;
  const float inv = ok ? 1.f / s : 0.f;
  if (r0 == 0) {
    float x[8];
    v.floats(x);
    *reinterpret_cast<uint2*>(codes + (int64_t)start * cst) = ok ? cache_codes8<CODE>(x, s, inv) : make_uint2(0u, 0u);
  }
  if (start > p0 && s > before) {
#pragma unroll 4
    for (int p = p0 + r0; p < start; p += 32 / TPR) requantise<CODE>(codes + (int64_t)p * cst, before, s, inv);
  }
  __syncwarp();                                              // (every lane has read the old scale)
  if (lane == 0) *scale = s;
}

// One (slot of kReadTokens packed tokens, K or V, KV head) of a read.
template <typename T>
struct ReadUnit {
  T* x;                          // row of the slot's first token
  const unsigned char* codes;
  const float* scales;           // of block 0 of the sequence
  int64_t xst, cst;
  int p, n;                      // the first token's place in its sequence; tokens left from it on (n < 0: to be zeros)
  __device__ __forceinline__ bool find(const CacheRows& dst, const int32_t* starts, const DamCacheView& c, uint32_t u) {
    constexpr int kShift = 6;
    static_assert(1 << kShift == kReadTokens, "slots are counted by a shift");
    const int h = u % c.Hkv, kv = u / c.Hkv & 1;
    const int64_t slot = u / (2 * c.Hkv);
    const int b = cache_seq_of_slot(dst.cu, c.num_seqs, kShift, 1, slot);
    const int t0 = __ldg(dst.cu + b), all = __ldg(dst.cu + b + 1) - t0, cap0 = __ldg(c.cu + b);
    int start;
    const bool fits = range_fits(c, starts, b, all, &start);
    const int64_t base = (slot - ((t0 >> kShift) + (int64_t)b)) * kReadTokens;
    if (base >= all) return false;
    n = all - (int)base;
    xst = kv ? dst.vst : dst.kst; cst = kv ? c.vst : c.kst;
    x = reinterpret_cast<T*>(const_cast<void*>(kv ? dst.V : dst.K)) + (t0 + base) * xst + (int64_t)h * (kv ? dst.vsh : dst.ksh);
    if (!fits) { n = -n; return true; }                      // nothing of this sequence can be read
    p = start + (int)base;
    codes = (kv ? c.v : c.k) + ((int64_t)cap0 + p) * cst + (int64_t)h * (kv ? c.vsh : c.ksh);
    scales = (kv ? c.vs : c.ks) + (int64_t)((cap0 >> c.shift) + b) * c.Hkv + h;
    return true;
  }
};

template <typename T, int D, int CODE>
__global__ void __launch_bounds__(kCThreads, 5)
cache_read_kernel(CacheRows dst, const int32_t* __restrict__ starts, DamCacheView c, uint32_t units, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  constexpr int TPR = D / 8, RPP = kCThreads / TPR, PASSES = kReadTokens / RPP;
  if (blockIdx.x == 0) report_ranges(c, dst.cu, starts, scratch);
  const int tid = threadIdx.x, r0 = tid / TPR, e = tid % TPR * 8;
  ReadUnit<T> cur, nxt;
  uint2 v[PASSES], w[PASSES];
  float s[PASSES], z[PASSES];
  auto load = [&](const ReadUnit<T>& y, uint2* r, float* f) {
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int t = r0 + i * RPP;
      r[i] = make_uint2(0u, 0u);
      f[i] = 0.f;
      if (t < y.n) {
        r[i] = __ldcs(reinterpret_cast<const uint2*>(y.codes + (int64_t)t * y.cst + e));
        f[i] = __ldg(y.scales + (int64_t)((y.p + t) >> c.shift) * c.Hkv);
      }
    }
  };
  uint32_t u = blockIdx.x;
  bool have = false;
  while (u < units && !(have = cur.find(dst, starts, c, u))) u += gridDim.x;
  if (have) load(cur, v, s);
  while (have) {
    bool more = false;
    u += gridDim.x;
    while (u < units && !(more = nxt.find(dst, starts, c, u))) u += gridDim.x;
    if (more) load(nxt, w, z);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      const int t = r0 + i * RPP;
      float f[8];
      codes_to_float<CODE>(v[i].x, f);
      codes_to_float<CODE>(v[i].y, f + 4);
      // (the rows of a sequence that cannot be read become zeros: int8 code 0 of scale 0, or the e4m3 zero)
#pragma unroll
      for (int k = 0; k < 8; ++k) f[k] *= s[i];
      if (t < abs(cur.n)) Eight<T>::store(cur.x + (int64_t)t * cur.xst + e, f);
    }
    cur = nxt; have = more;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) { v[i] = w[i]; s[i] = z[i]; }
  }
}

CacheRows rows_of(const void* K, const void* V, const dam_shape_t* t) {
  return {K, V, t->k_stride_tok, t->k_stride_head, t->v_stride_tok, t->v_stride_head, t->cu_seqlens_dev};
}

template <typename T, int D, int CODE>
cudaError_t launch_write(const CacheRows& src, const int32_t* starts, const DamCacheView& c, int64_t units, bool one, int sms, uint32_t* scratch,
                         cudaStream_t st) {
  if (one) {
    return dam_launch_chained(cache_write_one_kernel<T, D, CODE>, dim3((unsigned)((units + 3) / 4)), dim3(128), 0, st, src, starts, c,
                              (uint32_t)units, scratch);
  }
  const int passes = ((1 << c.shift) * (D / 8) + kCThreads - 1) / kCThreads;
  void (*k)(CacheRows, const int32_t*, DamCacheView, uint32_t, uint32_t*) =
      passes <= 1 ? cache_write_kernel<T, D, CODE, 1> : passes == 2 ? cache_write_kernel<T, D, CODE, 2>
      : passes == 4 ? cache_write_kernel<T, D, CODE, 4> : cache_write_kernel<T, D, CODE, 8>;
  const int per_sm = passes * (int)sizeof(T) <= 8 ? 5 : passes * (int)sizeof(T) <= 16 ? 3 : 2;
  const int64_t grid = units < (int64_t)sms * per_sm ? units : (int64_t)sms * per_sm;
  return dam_launch_chained(k, dim3((unsigned)grid), dim3(kCThreads), 0, st, src, starts, c, (uint32_t)units, scratch);
}

template <typename T, int D, int CODE>
cudaError_t launch_read(const CacheRows& dst, const int32_t* starts, const DamCacheView& c, int64_t units, int sms, uint32_t* scratch,
                        cudaStream_t st) {
  const int64_t grid = units < 5ll * sms ? units : 5ll * sms;
  return dam_launch_chained(cache_read_kernel<T, D, CODE>, dim3((unsigned)grid), dim3(kCThreads), 0, st, dst, starts, c, (uint32_t)units,
                            scratch);
}

cudaError_t sm_count(int* sms) {
  int dev = 0;
  DamDeviceInfo di;
  const cudaError_t e = dam_current_device(&dev, &di);
  *sms = di.sm_count;
  return e;
}

}  // namespace

cudaError_t dam_launch_cache_write(const void* K, const void* V, const dam_shape_t* tokens, const int32_t* starts, const dam_cache_t* cache,
                                   void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  // a sequence's tokens touch at most (n - 2) / block + 2 blocks: its slots are two more than the difference of cu / block
  bool one = true;
  for (int b = 0; b < c.num_seqs; ++b) one &= tokens->cu_seqlens_host[b + 1] - tokens->cu_seqlens_host[b] <= 1;
  const int64_t slots = one ? c.num_seqs : (tokens->total_tokens >> c.shift) + 2ll * c.num_seqs, units = slots * 2 * c.Hkv;
  if (units > 0x7FFFFFFF) return cudaErrorNotSupported;
  return DAM_CACHE_DISPATCH(launch_write, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c, units, one, sms,
                            reinterpret_cast<uint32_t*>(scratch), st);
}

cudaError_t dam_launch_cache_read(const dam_cache_t* cache, const dam_shape_t* tokens, const int32_t* starts, void* K, void* V,
                                  void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  const int64_t slots = tokens->total_tokens / kReadTokens + (int64_t)c.num_seqs, units = slots * 2 * c.Hkv;
  if (units > 0x7FFFFFFF) return cudaErrorNotSupported;
  return DAM_CACHE_DISPATCH(launch_read, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c, units, sms,
                            reinterpret_cast<uint32_t*>(scratch), st);
}
