// Writing K and V rows into a cache held in 8 bits, and reading them back.
//
// Write: x -> code, with one scale per block of tokens and KV head, s = amax / 127 (int8) or the least power of two that
// brings amax to 448 (e4m3).  A block of threads takes one (block of tokens, KV head) of K or of V: it holds the rows in
// registers from the one time they are read, finds their largest magnitude, and writes the codes; nothing is read twice.
// Where the block of tokens was begun by an earlier call its scale can only grow, and when it does the tokens that are
// there are read back and quantised again.  Read: value = code * scale.  Both move bytes and do little else: HBM bounds them
// (2 + 1 bytes per element of a bf16 write, 1 + 2 of a read; 128k tokens of 8 KV heads of 128, 805 MB either way: written in 133 us,
// read in 131, 6.0 and 6.1 TB/s), once the instructions per element are few enough (two fused multiply-adds that enclose the
// quotient instead of a division or a rounding instruction: the first form of the write took 240 us).
#include <type_traits>

#include "dam_cache.cuh"

namespace {

constexpr int kRThreads = 256, kRPasses = 4, kRBlocks = 4;   // of a read: threads, 8-element pieces per thread, blocks per SM
constexpr int kRPieces = kRThreads * kRPasses;

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
  // largest magnitudes so far, two at a time; as bits an infinity or a NaN is larger than any number
  __device__ __forceinline__ void top(uint32_t& t) const {
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 m = __hmax2_nan(*reinterpret_cast<const __nv_bfloat162*>(&t), __habs2(*reinterpret_cast<const __nv_bfloat162*>(&w[i])));
      t = *reinterpret_cast<const uint32_t*>(&m);
    }
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
// eight elements of a token that is there already, from the scale `before` to the coder's
template <int CODE>
__device__ __forceinline__ void requantise(unsigned char* p, float before, const Coder<CODE>& coder) {
  uint2* at = reinterpret_cast<uint2*>(p);
  const uint2 old = *at;
  float f[8];
  code_values<CODE>(old.x, before, f);
  code_values<CODE>(old.y, before, f + 4);
  *at = coder.eight(f);
}

// start of sequence b's range, and whether the range [start, start + n) lies inside its capacity (an empty one always does)
__device__ __forceinline__ bool range_fits(const DamCacheView& c, const int32_t* starts, int b, int n, int* start) {
  *start = starts ? __ldg(starts + b) : 0;
  return n == 0 || (*start >= 0 && *start <= __ldg(c.cu + b + 1) - __ldg(c.cu + b) - n);
}
// the scratch block of the whole call, its status word included (one block of threads looks at every sequence)
__device__ __forceinline__ void report_ranges(const DamCacheView& c, const int32_t* tok_cu, const int32_t* starts, uint32_t* scratch) {
  bool bad = false;
  for (int b = threadIdx.x; b < c.num_seqs; b += blockDim.x) {
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

// A block of threads' way through the slots: its KV head and its side (K or V) stay, its slots are `step` apart, so that blocks
// that run side by side read the heads of the same tokens (contiguous in memory).  SLOT finds a slot's tokens; its search of the
// sequence runs only where the next slot is another sequence's (whole warp, the same in all warps).
template <typename SLOT>
struct Slots {
  SLOT at;
  uint32_t slot, until, step;    // until: first slot of the next sequence
  int h, kv;
  __device__ __forceinline__ Slots(const DamCacheView& c) : until(0) {
    const uint32_t lane = blockIdx.x % (2 * c.Hkv);          // (the grid is a multiple of 2 Hkv)
    kv = lane >= (uint32_t)c.Hkv;
    h = (int)lane - (kv ? c.Hkv : 0);
    slot = blockIdx.x / (2 * c.Hkv);
    step = gridDim.x / (2 * c.Hkv);
  }
  // to the first slot from this one on that holds tokens
  __device__ __forceinline__ bool seek(const DamCacheView& c, const CacheRows& rows, const int32_t* starts, uint32_t slots) {
    for (; slot < slots; slot += step) {
      if (slot >= until) until = at.enter(c, rows, starts, slot);
      if (at.place(c, slot)) {
        at.aim(c, rows, kv, h, step);
        return true;
      }
    }
    return false;
  }
  __device__ __forceinline__ bool next(const DamCacheView& c, const CacheRows& rows, const int32_t* starts, uint32_t slots) {
    slot += step;
    if (slot < until && at.place(c, slot)) {
      at.go_on();
      return true;
    }
    return seek(c, rows, starts, slots);
  }
};

// Slot of a write: one block of tokens of a sequence.  The pointers are a thread's own: row r0 of the block, element e.
template <typename T, int D>
struct WriteSlot {
  int b, t0, cap0, start, end;   // sequence; its packed and its cache row; its new tokens start .. end - 1 (none: start == end)
  int zero;                      // slot `x` is block x - zero of the sequence
  const T* x;
  unsigned char* codes;
  float* scale;
  int64_t xst, cst;
  int64_t dx, dc, ds;            // to the next slot of the same sequence
  int p0, first, last;           // the block's first token; its new tokens: rows first .. last - 1 of it
  __device__ __forceinline__ uint32_t enter(const DamCacheView& c, const CacheRows& src, const int32_t* starts, uint32_t slot) {
    b = cache_seq_of_slot(src.cu, c.num_seqs, c.shift, 2, slot);
    t0 = __ldg(src.cu + b);
    cap0 = __ldg(c.cu + b);
    const int t1 = __ldg(src.cu + b + 1);
    end = range_fits(c, starts, b, t1 - t0, &start) ? start + (t1 - t0) : start;
    zero = (t0 >> c.shift) + 2 * b - (start >> c.shift);
    return (uint32_t)(t1 >> c.shift) + 2u * (uint32_t)(b + 1);
  }
  __device__ __forceinline__ bool place(const DamCacheView& c, uint32_t slot) {
    const int64_t p = ((int64_t)(int)slot - zero) << c.shift;
    if (p >= end || start == end) return false;
    p0 = (int)p;
    first = max(start - p0, 0);
    last = min(1 << c.shift, end - p0);
    return true;
  }
  __device__ __forceinline__ void aim(const DamCacheView& c, const CacheRows& src, int kv, int h, uint32_t step) {
    constexpr int TPR = D / 8;
    const int r0 = threadIdx.x / TPR, e = threadIdx.x % TPR * 8;
    xst = kv ? src.vst : src.kst; cst = kv ? c.vst : c.kst;
    const int64_t tokens = (int64_t)step << c.shift;
    dx = tokens * xst; dc = tokens * cst; ds = (int64_t)step * c.Hkv;
    // (row t0 + p0 - start may lie before the sequence's where the block was begun before; it is not read then)
    x = reinterpret_cast<const T*>(kv ? src.V : src.K) + ((int64_t)t0 + p0 - start + r0) * xst + (int64_t)h * (kv ? src.vsh : src.ksh) + e;
    codes = (kv ? c.v : c.k) + ((int64_t)cap0 + p0 + r0) * cst + (int64_t)h * (kv ? c.vsh : c.ksh) + e;
    scale = (kv ? c.vs : c.ks) + (int64_t)((cap0 >> c.shift) + b + (p0 >> c.shift)) * c.Hkv + h;
  }
  __device__ __forceinline__ void go_on() { x += dx; codes += dc; scale += ds; }
};

// PASSES: rows of a block of tokens that a thread holds 8 elements of.  Enough blocks of threads share an SM that some wait for their
// rows while others quantise theirs (a prompt of 128k tokens 133 us; with the next slot's rows requested ahead, at twice the
// registers and four blocks, 160).
template <typename T, int D, int CODE, int THREADS, int PASSES, int BLOCKS>
__global__ void __launch_bounds__(THREADS, BLOCKS)
cache_write_kernel(CacheRows src, const int32_t* __restrict__ starts, DamCacheView c, uint32_t slots, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  constexpr int TPR = D / 8, RPP = THREADS / TPR;            // threads of a row, rows of a pass
  __shared__ uint32_t warp_max[2][THREADS / 32];
  if (blockIdx.x == 0) report_ranges(c, src.cu, starts, scratch);
  const int tid = threadIdx.x, r0 = tid / TPR;
  constexpr int whole = PASSES * RPP;                        // = block_tokens
  Slots<WriteSlot<T, D>> it(c);
  Eight<T> v[PASSES];
  float before = 0.f;
  auto load = [&](const WriteSlot<T, D>& y, Eight<T>* r, float& b) {
    if (y.first == 0 && y.last == whole) {
#pragma unroll
      for (int i = 0; i < PASSES; ++i) r[i].load(y.x + i * RPP * y.xst);
      return;
    }
    b = y.first > 0 ? *reinterpret_cast<const volatile float*>(y.scale) : 0.f;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
      r[i].clear();
      if (r0 + i * RPP >= y.first && r0 + i * RPP < y.last) r[i].load(y.x + i * RPP * y.xst);
    }
  };
  bool have = it.seek(c, src, starts, slots);
  int turn = 0;
  while (have) {
    load(it.at, v, before);
    unsigned char* const codes = it.at.codes;
    float* const scale = it.at.scale;
    const int64_t cst = it.at.cst;
    const int first = it.at.first, last = it.at.last;
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) v[i].top(top);
    top = __reduce_max_sync(0xFFFFFFFFu, Eight<T>::joined(top));
    if ((tid & 31) == 0) warp_max[turn][tid >> 5] = top;
    __syncthreads();                                         // (every thread has read the old scale, too)
#pragma unroll
    for (int k = 0; k < THREADS / 32; ++k) top = max(top, warp_max[turn][k]);
    const float s = block_scale<CODE>(top, first > 0, before);
    if (s == s) {
      const Coder<CODE> coder(s);
      if (first == 0 && last == whole) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          float x[8];
          v[i].floats(x);
          *reinterpret_cast<uint2*>(codes + i * RPP * cst) = coder.eight(x);
        }
      } else {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) {
          if (r0 + i * RPP >= first && r0 + i * RPP < last) {
            float x[8];
            v[i].floats(x);
            *reinterpret_cast<uint2*>(codes + i * RPP * cst) = coder.eight(x);
          }
        }
        // where the scale grew the tokens that are there are read back and quantised again (every thread its own 8 elements)
        if (first > 0 && s > before) {
#pragma unroll 1
          for (int r = r0; r < first; r += RPP) requantise<CODE>(codes + (int64_t)(r - r0) * cst, before, coder);
        }
      }
    } else {
#pragma unroll 1
      for (int r = r0; r < last; r += RPP)
        if (r >= first) *reinterpret_cast<uint2*>(codes + (int64_t)(r - r0) * cst) = make_uint2(0u, 0u);
    }
    if (tid == 0) *scale = s;
    turn ^= 1; have = it.next(c, src, starts, slots);
  }
}

// One token per sequence at most (a generation step): a warp per (sequence, K or V, KV head).
template <typename T, int D, int CODE>
__global__ void __launch_bounds__(128)
cache_write_one_kernel(CacheRows src, const int32_t* __restrict__ starts, DamCacheView c, uint32_t rows, uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  if (blockIdx.x == 0) report_ranges(c, src.cu, starts, scratch);
  const uint32_t u = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (u >= rows) return;
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
  const Coder<CODE> coder(s);
  if (r0 == 0) {
    float x[8];
    v.floats(x);
    *reinterpret_cast<uint2*>(codes + (int64_t)start * cst) = s == s ? coder.eight(x) : make_uint2(0u, 0u);
  }
  if (start > p0 && s > before) {
#pragma unroll 4
    for (int p = p0 + r0; p < start; p += 32 / TPR) requantise<CODE>(codes + (int64_t)p * cst, before, coder);
  }
  __syncwarp();                                              // (every lane has read the old scale)
  if (lane == 0) *scale = s;
}

// 8 floats to a 32-byte boundary in one piece: a warp's store covers whole sectors, not one half of each after the other.
__device__ __forceinline__ void store32(float* p, const float* x) {
  asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}

// A read's slot is 2^shift packed tokens of a sequence, all heads of K or of V: up to kRPieces pieces of 8 elements, which lie one after
// the other in memory where the rows are dense, however many heads share a row (a slot of one head left every other head's bytes of
// a row to another block: 128k fp32 tokens of 4 heads of 64, 64 us instead of 58; 64 short reads 7.2 instead of 4.1).  Tokens of more pieces than that are cut into `cuts`.
// DENSE: codes and rows are [token][head][d] without gaps, and fp32 rows begin on a 32-byte boundary.  grid: (slot, K or V, cut), the cut fastest.
template <typename T, int D, int CODE, bool DENSE>
__global__ void __launch_bounds__(kRThreads, kRBlocks)
cache_read_kernel(CacheRows dst, const int32_t* __restrict__ starts, DamCacheView c, uint32_t slots, int shift, uint32_t cuts,
                  uint32_t* __restrict__ scratch) {
  dam_chain_prologue();
  if (blockIdx.x == 0) report_ranges(c, dst.cu, starts, scratch);
  const uint32_t side = blockIdx.x / cuts, cut = blockIdx.x - side * cuts, step = gridDim.x / (2 * cuts);
  const bool kv = side & 1u;
  uint32_t slot = side >> 1, until = 0u;                     // until: first slot of the next sequence
  const int64_t xst = kv ? dst.vst : dst.kst, cst = kv ? c.vst : c.kst;
  T* const X = reinterpret_cast<T*>(const_cast<void*>(kv ? dst.V : dst.K));
  const unsigned char* const C = kv ? c.v : c.k;
  const float* const S = kv ? c.vs : c.ks;
  // this thread's pieces: token of the slot (none: beyond every slot), head, and where they stand in codes and rows
  int r[kRPasses], h[kRPasses];
  int64_t co[kRPasses], xo[kRPasses];                        // (DENSE: known when compiled, but for a start)
  const int64_t mine = 8 * ((int64_t)threadIdx.x + cut * kRPieces);
#pragma unroll
  for (int i = 0; i < kRPasses; ++i) {
    const int per = c.Hkv * (D / 8), f = (int)threadIdx.x + kRThreads * i + (int)cut * kRPieces;
    r[i] = f / per;
    const int piece = f - r[i] * per, e = piece % (D / 8) * 8;
    h[i] = piece / (D / 8);
    co[i] = DENSE ? 8 * kRThreads * i : r[i] * cst + h[i] * (kv ? c.vsh : c.ksh) + e;
    xo[i] = DENSE ? 8 * kRThreads * i : r[i] * xst + h[i] * (kv ? dst.vsh : dst.ksh) + e;
    if (r[i] >> shift) r[i] = 0x7FFFFFFF;
  }
  int b = 0, t0 = 0, cap0 = 0, start = 0, all = 0, zero = 0;  // the sequence of the slot: see WriteSlot; `all`: its tokens
  bool fits = false;
  // the present slot: its first token's place among `all`, and the tokens from it on
  int base = 0;
  auto seek = [&]() -> bool {
    for (; slot < slots; slot += step) {
      if (slot >= until) {
        b = cache_seq_of_slot(dst.cu, c.num_seqs, shift, 1, slot);
        t0 = __ldg(dst.cu + b);
        cap0 = __ldg(c.cu + b);
        const int t1 = __ldg(dst.cu + b + 1);
        all = t1 - t0;
        fits = range_fits(c, starts, b, all, &start);
        zero = (t0 >> shift) + b;
        until = (uint32_t)(t1 >> shift) + (uint32_t)(b + 1);
      }
      const int64_t at = (int64_t)((int)slot - zero) << shift;
      if (at < all) {
        base = (int)at;
        return true;
      }
    }
    return false;
  };
  uint2 v[kRPasses], w[kRPasses];
  float s[kRPasses], z[kRPasses];
  auto load = [&](uint2* to, float* scale) {
    const unsigned char* codes = C + ((int64_t)cap0 + start + base) * cst + (DENSE ? mine : 0);
    const float* scales = S + (int64_t)((cap0 >> c.shift) + b) * c.Hkv;
#pragma unroll
    for (int i = 0; i < kRPasses; ++i) {
      to[i] = make_uint2(0u, 0u);                            // (a sequence that cannot be read: code 0 of scale 0)
      scale[i] = 0.f;
      if (fits && r[i] < all - base) {
        to[i] = __ldcs(reinterpret_cast<const uint2*>(codes + co[i]));
        scale[i] = __ldg(scales + (int64_t)((start + base + r[i]) >> c.shift) * c.Hkv + h[i]);
      }
    }
  };
  bool have = seek();
  if (have) load(v, s);
  while (have) {
    // the next slot's codes are on their way while this one's values are written
    T* const x = X + ((int64_t)t0 + base) * xst + (DENSE ? mine : 0);
    const int n = all - base;
    slot += step;
    have = seek();
    if (have) load(w, z);
#pragma unroll
    for (int i = 0; i < kRPasses; ++i) {
      float f[8];
      code_values<CODE>(v[i].x, s[i], f);
      code_values<CODE>(v[i].y, s[i], f + 4);
      if (r[i] < n) {
        if constexpr (DENSE && sizeof(T) == 4) store32(x + xo[i], f);
        else Eight<T>::store(x + xo[i], f);
      }
    }
#pragma unroll
    for (int i = 0; i < kRPasses; ++i) { v[i] = w[i]; s[i] = z[i]; }
  }
}

CacheRows rows_of(const void* K, const void* V, const dam_shape_t* t) {
  return {K, V, t->k_stride_tok, t->k_stride_head, t->v_stride_tok, t->v_stride_head, t->cu_seqlens_dev};
}

template <int N> using Int = std::integral_constant<int, N>;

// Threads, rows per thread and blocks per SM of a write, by the elements of a block of tokens: 8 rows per thread (fp32: 4) keep what
// a slot costs beside its rows small.
template <typename T, int D, typename F>
cudaError_t write_form(int block_tokens, F go) {
  const int rows = block_tokens * (D / 64);                  // (of 64 elements)
  if constexpr (sizeof(T) == 2) {
    if (rows <= 16) return go(Int<128>(), Int<1>(), Int<8>());
    if (rows == 32) return go(Int<128>(), Int<2>(), Int<8>());
    if (rows == 64) return go(Int<128>(), Int<4>(), Int<8>());
    if (rows == 128) return go(Int<128>(), Int<8>(), Int<7>());
    if constexpr (D == 128) return go(Int<256>(), Int<8>(), Int<3>());
  } else {
    if (rows <= 16) return go(Int<128>(), Int<1>(), Int<8>());
    if (rows == 32) return go(Int<128>(), Int<2>(), Int<8>());
    if (rows == 64) return go(Int<128>(), Int<4>(), Int<7>());
    if (rows == 128) return go(Int<256>(), Int<4>(), Int<3>());
    if constexpr (D == 128) return go(Int<512>(), Int<4>(), Int<1>());
  }
  return cudaErrorNotSupported;
}

// Blocks of a grid over `slots` of c: a multiple of 2 Hkv, no more than are resident at once (or one slot at a time).
unsigned slot_grid(int64_t slots, const DamCacheView& c, int resident) {
  const int64_t per = 2ll * c.Hkv, at_once = resident / per > 0 ? resident / per : 1;
  return (unsigned)(per * (slots < at_once ? slots : at_once));
}

template <typename T, int D, int CODE>
cudaError_t launch_write(const CacheRows& src, const int32_t* starts, const DamCacheView& c, int64_t slots, bool one, int sms, uint32_t* scratch,
                         cudaStream_t st) {
  if (one) {
    const int64_t rows = slots * 2 * c.Hkv;
    return dam_launch_chained(cache_write_one_kernel<T, D, CODE>, dim3((unsigned)((rows + 3) / 4)), dim3(128), 0, st, src, starts, c,
                              (uint32_t)rows, scratch);
  }
  auto go = [&](auto threads, auto passes, auto blocks) {
    constexpr int THREADS = decltype(threads)::value, PASSES = decltype(passes)::value, BLOCKS = decltype(blocks)::value;
    return dam_launch_chained(cache_write_kernel<T, D, CODE, THREADS, PASSES, BLOCKS>, dim3(slot_grid(slots, c, sms * BLOCKS)), dim3(THREADS),
                              0, st, src, starts, c, (uint32_t)slots, scratch);
  };
  return write_form<T, D>(1 << c.shift, go);
}

template <typename T, int D, int CODE>
cudaError_t launch_read(const CacheRows& dst, const int32_t* starts, const DamCacheView& c, int64_t tokens, int sms, uint32_t* scratch,
                        cudaStream_t st) {
  // as many tokens as have kRPieces pieces, at most 64; one token of more pieces is cut
  const int64_t per = (int64_t)c.Hkv * (D / 8), cuts = (per + kRPieces - 1) / kRPieces;
  int shift = 0;
  while (shift < 6 && (per << (shift + 1)) <= kRPieces) ++shift;
  const int64_t slots = (tokens >> shift) + c.num_seqs, at_once = (int64_t)sms * kRBlocks / (2 * cuts);
  const int64_t grid = 2 * cuts * (slots < at_once ? slots : at_once > 0 ? at_once : 1);
  if (slots > 0x3FFFFFFF || per > 0x3FFFFFFF || grid > 0x7FFFFFFF) return cudaErrorNotSupported;
  auto dense = [&](int64_t st, int64_t sh) { return sh == D && st == (int64_t)c.Hkv * D; };
  const bool aligned = sizeof(T) == 2 || (reinterpret_cast<uintptr_t>(dst.K) | reinterpret_cast<uintptr_t>(dst.V)) % 32 == 0;
  const bool all = aligned && dense(dst.kst, dst.ksh) && dense(dst.vst, dst.vsh) && dense(c.kst, c.ksh) && dense(c.vst, c.vsh);
  return dam_launch_chained(all ? cache_read_kernel<T, D, CODE, true> : cache_read_kernel<T, D, CODE, false>, dim3((unsigned)grid), dim3(kRThreads), 0, st, dst, starts, c, (uint32_t)slots, shift,
                            (uint32_t)cuts, scratch);
}

cudaError_t sm_count(int* sms) {
  int dev = 0;
  DamDeviceInfo di;
  const cudaError_t e = dam_current_device(&dev, &di);
  *sms = e == cudaSuccess ? di.sm_count : 0;
  return e;
}

}  // namespace

cudaError_t dam_launch_cache_write(const void* K, const void* V, const dam_shape_t* tokens, const int32_t* starts, const dam_cache_t* cache,
                                   void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  bool one = true;
  for (int b = 0; b < c.num_seqs; ++b) one &= tokens->cu_seqlens_host[b + 1] - tokens->cu_seqlens_host[b] <= 1;
  // a sequence's tokens touch at most (n - 2) / block + 2 blocks: its slots are two more than the difference of cu / block
  const int64_t slots = one ? c.num_seqs : (tokens->total_tokens >> c.shift) + 2ll * c.num_seqs;
  if (slots * 2 * c.Hkv > 0x7FFFFFFF) return cudaErrorNotSupported;
  return DAM_CACHE_DISPATCH(launch_write, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c, slots, one, sms,
                            reinterpret_cast<uint32_t*>(scratch), st);
}

cudaError_t dam_launch_cache_read(const dam_cache_t* cache, const dam_shape_t* tokens, const int32_t* starts, void* K, void* V,
                                  void* scratch, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  int sms = 0;
  const cudaError_t e = sm_count(&sms);
  if (e != cudaSuccess) return e;
  return DAM_CACHE_DISPATCH(launch_read, tokens->dtype, tokens->head_dim, cache->code, rows_of(K, V, tokens), starts, c,
                            (int64_t)tokens->total_tokens, sms, reinterpret_cast<uint32_t*>(scratch), st);
}
