// Generation over a KV cache held in 8 bits: one new token per sequence, against every key its sequence holds, or against the
// keys that the patterns of a mask blob keep (paper Sec. 4.3, Case 2).
//
// The logit of key j is scale * sK(j) * (q . codes of K_j), the output sum_j p_j sV(j) (codes of V_j) / sum_j p_j: the codes go
// through the warp-level tensor-core instruction as fp16 numbers, which hold every int8 and every e4m3 value exactly, and the
// scales are applied to the logits and to the probabilities, one multiplication per key and head instead of one per element.
// Both products are taken transposed, S^T = K q^T and O^T = V^T P^T: the 8 query heads of a KV head are the narrow side of the
// instruction's tile, so nothing of it is padding where a group has 8 heads.  fp16 operands: q is scaled by a power of two so
// that its largest element lies in [2^14, 2^15) (a bf16 q is then exact wherever it matters), and the weights, probability times sV,
// are held in units of their own for every head: a power of two that puts the largest weight of the head so far between 2^11 and
// 2^15.  A weight of a bf16 query is one fp16 number, 11 bits under a result of 8: the result's error against 64 bits grows by 1 to
// 2 % (1.69e-3 -> 1.72e-3, one sequence of 8000 tokens), and for more than four heads a second number would double the second
// product's instructions.  An fp32 q and its weights are each the sum of two fp16 numbers (22 bits), at the price of twice the
// instructions.  What fp16's last step of 2^-24 drops of a weight is 2^-36 of the head's largest, and 2^-47 where there is a second
// number, which is held 2^11 times larger than the first: a key that the head does not keep, or that has no probability, costs the
// others nothing however large its V is.
//
// A warp works on slices of 16 keys (two at a time where keys are contiguous: two independent chains of instructions), brought to
// shared memory by asynchronous copies ahead of their use, and keeps a running softmax and its share of O^T of its own; the warps of
// a block meet at the end of a sequence's share only.  The order of the dimensions inside the instructions' k side and of O^T's rows
// is free, and taken so that every lane reads its codes 16 bytes at a time and, with K, a register of four codes is two operand
// registers.
//
// Bound by HBM: 2 d bytes and two scales per key and KV head are read once.  64 sequences of 16k to 32k tokens (8 KV heads of 128,
// int8): 515 to 590 us by box and by how the batch repeats, 5.5 to 6.2 TB/s of codes and scales; one of 64k to 128k tokens 33 to 39 us with
// its 7 us of beginning and end.
// A slice costs about 330 warp instructions, a third of them the conversion of its codes (int8: exclusive or, byte permutation and
// one subtraction for two codes; e4m3: one conversion), and 175 cycles of its SM's share of the bandwidth: with the copies issued
// by the lanes (cp.async, 600 instructions in all) the same batch took 820 us.
#include <cooperative_groups.h>
#include <math_constants.h>

#include "dam_cache.cuh"
#include "dam_gather.cuh"
#include "sm100_ptx.cuh"

namespace {

constexpr int kSlice = 16;             // keys of a slice: the rows of the first instruction, the k side of the second
constexpr int kTile = 2;               // slices that a warp takes at a time where the keys are contiguous: two independent chains

constexpr int kGMaxGroup = 8;         // query heads a block takes: the narrow side of the instructions' tiles
constexpr int kPackGroup = 4;         // so many at most, and both numbers of an fp32 value fit into it

__device__ __forceinline__ void cp_async4_zfill(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 r;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
  return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 r;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
  return r;
}
__device__ __forceinline__ float lds_float(uint32_t a) {
  float r;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(r) : "r"(a));
  return r;
}
// D (16 x 8, fp32) += A (16 x 16, fp16, row-major) * B (16 x 8, fp16, column-major)
__device__ __forceinline__ void mma_f16(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// The second number of a weight is held kLow times larger (it is at most 2^4, half a step of 2^15), and so are its products, in columns
// or in an accumulator of their own.
constexpr float kLow = 2048.f;
// four codes in memory order -> two operand registers (codes 0, 1 and codes 2, 3)
template <int CODE>
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t* h) {
  if constexpr (CODE == DAM_CODE_INT8) {
    w ^= 0x80808080u;
    h[0] = biased_to_half2(__byte_perm(w, 0x64646464u, 0x4140));
    h[1] = biased_to_half2(__byte_perm(w, 0x64646464u, 0x4342));
  } else {
    h[0] = e4m3x2_to_half2(w & 0xFFFFu);
    h[1] = e4m3x2_to_half2(w >> 16);
  }
}

// Rows of N slices in shared memory: 16 N of K, 16 N of V, as a tiled copy with 128-byte (head_dim 64: 64-byte) swizzle leaves
// them.  The 16-byte piece p of row r stands at piece p ^ (r & 7) of the row, for head_dim 64 at p ^ (r / 2 & 3): the eight lanes
// that a 16-byte read is served for at a time find their pieces in different banks, given the order in which rows are taken.
template <int D, int N>
struct Rows {
  static constexpr int keys = kSlice * N, pieces = D / 16;
  static constexpr int v_off = keys * D, bytes = 2 * keys * D;
  static __device__ __forceinline__ uint32_t at(int r, int p) {
    if constexpr (D == 128) return r * 128 + ((p ^ (r & 7)) << 4);
    else return r * 64 + ((p ^ (r >> 1 & 3)) << 4);
  }
  // The key that stands for row i of the instructions' tiles (i + 8: that key + 8).  head_dim 64: 0 3 4 7 1 2 5 6, so that rows 2 j
  // and 2 j + 1 lie in different halves of 128 bytes (K), and rows 0 2 4 6, and 1 3 5 7, in different quarters (V).
  static __device__ __forceinline__ int key(int i) { return D == 128 ? i : (int)(0x65217430u >> (4 * (i & 7)) & 7u) + (i & 8); }
};

// What a warp carries through the keys of one (sequence, up to 8 query heads of one KV head).  Lane = 4 row + quad: the lane
// holds the logits of keys row and row + 8 against heads 2 quad and 2 quad + 1, and of O^T the dimensions D / 8 * row ... of the
// same two heads.
// PACK: of an fp32 q of at most four heads, the second numbers of q and P are columns 4 to 7 of the tiles; quads 2 and 3 stand for the
// heads of quads 0 and 1 then (six sequences of 16 heads over 4 KV heads of 64: 20.9 us with two instructions each).
template <typename T, int D, int CODE, bool PACK>
struct WarpState {
  static_assert(!PACK || sizeof(T) == 4, "one number has no second");
  static constexpr bool kSplit = sizeof(T) == 4 && !PACK;    // q and P as two fp16 numbers each, an instruction each
  static __device__ __forceinline__ int head_of(int column) { return PACK ? column & (kPackGroup - 1) : column; }
  static constexpr int KS = D / 16;
  uint32_t qh[KS][2], ql[kSplit ? KS : 1][2];
  float qs[2];                         // logits (log2 units) per product of codes and q as it is held, of the lane's heads
  float m[2], l[2];                    // reference (log2 units) and the lane's share of the sum
  float unit[2];                       // a weight p sV of the lane's heads is held times this power of two, 2^-116 to 2^120
  float o[KS][4];                      // [u][0..1]: dimension D / 8 * row + 2 u, the lane's heads; [u][2..3]: the next dimension

  __device__ __forceinline__ void reset() {
    m[0] = m[1] = -CUDART_INF_F;
    l[0] = l[1] = 0.f;
    unit[0] = unit[1] = 1.329227995784916e36f;               // 2^120: smaller weights than 2^-109 get no larger unit
#pragma unroll
    for (int u = 0; u < KS; ++u) o[u][0] = o[u][1] = o[u][2] = o[u][3] = 0.f;
  }

  // The lane's elements of head `row`: dimensions D / 4 * quad ..., as they are in memory.  q: row of the first of `heads` heads.
  struct Query { uint4 w[D / 4 * sizeof(T) / 16]; };
  static __device__ __forceinline__ Query fetch_q(const T* q, int heads) {
    const int lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
    const uint4* p = reinterpret_cast<const uint4*>(q + (int64_t)(head_of(row) < heads ? head_of(row) : 0) * D + D / 4 * quad);
    Query r;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r.w) / 16); ++i) r.w[i] = __ldg(p + i);
    return r;
  }
  __device__ __forceinline__ void set_q(const Query& q, int heads, float scale_log2) {
    const int lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
    constexpr int N = D / 4;
    float x[N];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(q.w) / 16); ++i) {
      const uint32_t w[4] = {q.w[i].x, q.w[i].y, q.w[i].z, q.w[i].w};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
          x[4 * i + k] = __uint_as_float(w[k]);
        } else {
          x[8 * i + 2 * k] = __uint_as_float(w[k] << 16); x[8 * i + 2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
      }
    }
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < N; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    // 2^(14 - exponent of the largest); an infinity or a NaN stays one
    const int f = min(268 - (int)(top >> 23), 253);
    const float mul = head_of(row) < heads ? __uint_as_float((uint32_t)f << 23) : 0.f;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float a = x[4 * s + 2 * k] * mul, b = x[4 * s + 2 * k + 1] * mul;
        qh[s][k] = pack_half2(a, b);
        if constexpr (kSplit || PACK) {
          const float2 hi = __half22float2(*reinterpret_cast<const __half2*>(&qh[s][k]));
          const uint32_t lo = pack_half2(a - hi.x, b - hi.y);
          if constexpr (kSplit) ql[s][k] = lo;
          else qh[s][k] = row < kPackGroup ? qh[s][k] : lo;
        }
      }
    }
    const float back = scale_log2 * __uint_as_float((uint32_t)(254 - f) << 23);
    qs[0] = __shfl_sync(0xFFFFFFFFu, back, 8 * quad);
    qs[1] = __shfl_sync(0xFFFFFFFFu, back, 8 * quad + 4);
  }

  // N slices: rows at `rows`, scales at `sc`, and which keys there are for whom.
  //   kAll    every head keeps all of them; the 16 of a slice share their scales (they lie in one block): K's and V's, slice by slice
  //   kFirst  the same for the first `arg` keys; the rows behind may hold anything
  //   kKeep   (one slice) bit e (e + 2) of arg: head head_of(2 quad + e) keeps key `row` (key `row + 8`), keys by Rows::key; 16 scales of K and
  //           16 of V
  // A key that a head does not keep has no part in it.
  enum Mode { kAll, kFirst, kKeep };
  template <Mode MODE, int N>
  __device__ __forceinline__ void step(uint32_t rows, uint32_t sc, uint32_t arg) {
    using RW = Rows<D, N>;
    constexpr bool ALL = MODE == kAll, UNIFORM = MODE != kKeep;
    static_assert(UNIFORM || N == 1, "keys of their own come one slice at a time");
    const int lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3, key = RW::key(row);
    uint32_t keep[N];
    float ks[N][2], vs[N][2];                                // of keys row and row + 8
#pragma unroll
    for (int n = 0; n < N; ++n) {
      keep[n] = arg;
      if constexpr (MODE == kFirst) keep[n] = (16 * n + key < (int)arg ? 3u : 0u) | (16 * n + key + 8 < (int)arg ? 12u : 0u);
      if constexpr (UNIFORM) {
        ks[n][0] = ks[n][1] = lds_float(sc + 8 * n);
        vs[n][0] = vs[n][1] = lds_float(sc + 8 * n + 4);
      } else {
        ks[n][0] = lds_float(sc + 4 * key); ks[n][1] = lds_float(sc + 32 + 4 * key);
        vs[n][0] = lds_float(sc + 64 + 4 * key); vs[n][1] = lds_float(sc + 96 + 4 * key);
      }
    }
    auto kept = [&](int n, int bit) { return ALL || (keep[n] >> bit & 1u); };
    // S^T = K q^T: k-step s takes the dimensions D / 4 * quad + 4 s ... of a lane
    float st[N][2][4] = {};                                  // (two chains of instructions per slice, half as long)
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const uint4 a = lds128(rows + RW::at(16 * n + key, D / 64 * quad + c)), b = lds128(rows + RW::at(16 * n + key + 8, D / 64 * quad + c));
        const uint32_t wa[4] = {a.x, a.y, a.z, a.w}, wb[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int s = 4 * c + i;
          uint32_t ha[2], hb[2];
          codes_to_half<CODE>(wa[i], ha);
          codes_to_half<CODE>(wb[i], hb);
          mma_f16(st[n][s & 1], ha[0], hb[0], ha[1], hb[1], qh[s][0], qh[s][1]);
          if constexpr (kSplit) mma_f16(st[n][s & 1], ha[0], hb[0], ha[1], hb[1], ql[s][0], ql[s][1]);
        }
      }
    }
    float x[N][4];
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float y = st[n][0][e] + st[n][1][e];
        if constexpr (PACK) y += __shfl_xor_sync(0xFFFFFFFFu, y, 2);
        x[n][e] = kept(n, e) ? y * (ks[n][e >> 1] * qs[e & 1]) : -CUDART_INF_F;
      }
    }
    // The reference of a head's logits moves when one lies more than 8 above it (probabilities stay below 2^8), its unit when a weight
    // passes 2^15: most steps move nothing.
    float top[2], sum[2], w[N][4], most;
    bool far = false;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      top[e] = fmaxf(x[0][e], x[0][2 + e]);
#pragma unroll
      for (int n = 1; n < N; ++n) top[e] = fmaxf(top[e], fmaxf(x[n][e], x[n][2 + e]));
      far |= top[e] > m[e] + 8.f;
    }
    // weights over the units, sums, and the largest weight; of no key, or of logits of -inf alone, nothing has a weight
    auto weigh = [&](float u0, float u1) {
      const float ref[2] = {m[0] == -CUDART_INF_F ? 0.f : m[0], m[1] == -CUDART_INF_F ? 0.f : m[1]}, u[2] = {u0, u1};
      most = sum[0] = sum[1] = 0.f;
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = g_ex2(x[n][e] - ref[e & 1]);
          sum[e & 1] += p;
          // (a key that is not kept may stand in a block without a scale: 0 * NaN is not 0.  p times the scale first: an unused
          // unit times a large scale is infinite)
          w[n][e] = kept(n, e) ? p * vs[n][e >> 1] * u[e & 1] : 0.f;
          most = fmaxf(most, w[n][e]);
        }
      }
    };
    weigh(unit[0], unit[1]);
    far |= most > 32768.f;
    if (__any_sync(0xFFFFFFFFu, far)) {
      float f[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float mx = top[e];
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
        const float mn = fmaxf(m[e], mx);
        f[e] = mn == -CUDART_INF_F ? 1.f : g_ex2(m[e] - mn);
        m[e] = mn;
        l[e] *= f[e];
      }
      weigh(1.f, 1.f);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        // the largest weight of the head so far (2^11 / unit at least was the largest when the unit was chosen) comes to [2^11, 2^12)
        float mx = 0.f;
#pragma unroll
        for (int n = 0; n < N; ++n) mx = fmaxf(mx, fmaxf(w[n][e], w[n][2 + e]));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 4));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 8));
        mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, 16));
        const float over = __uint_as_float(0x7F000000u - __float_as_uint(unit[e]));          // 1 / unit
        mx = fmaxf(mx, f[e] * (2048.f * over));
        const float now = __uint_as_float((uint32_t)min(265 - (int)(__float_as_uint(mx) >> 23), 247) << 23);
        f[e] = f[e] * now * over;                            // (at most 1: the unit grows no more than the weights before have shrunk)
        unit[e] = now;
      }
#pragma unroll
      for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) w[n][e] *= unit[e & 1];
      }
#pragma unroll
      for (int u = 0; u < KS; ++u) { o[u][0] *= f[0]; o[u][1] *= f[1]; o[u][2] *= f[0]; o[u][3] *= f[1]; }
    }
    l[0] += sum[0];
    l[1] += sum[1];
    uint32_t pb[N][2], pl[N][2];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      // P^T as operands (k = key, n = head): the transposes of the two 8 x 8 blocks [key][head]
      uint32_t h0 = pack_half2(w[n][0], w[n][1]), h1 = pack_half2(w[n][2], w[n][3]);
      if constexpr (PACK) {
        const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
        if (quad >= 2) {
          h0 = pack_half2((w[n][0] - f0.x) * kLow, (w[n][1] - f0.y) * kLow);
          h1 = pack_half2((w[n][2] - f1.x) * kLow, (w[n][3] - f1.y) * kLow);
        }
      }
      pb[n][0] = movmatrix_trans(h0);
      pb[n][1] = movmatrix_trans(h1);
      if constexpr (kSplit) {
        const float2 f0 = __half22float2(*reinterpret_cast<const __half2*>(&h0)), f1 = __half22float2(*reinterpret_cast<const __half2*>(&h1));
        pl[n][0] = movmatrix_trans(pack_half2((w[n][0] - f0.x) * kLow, (w[n][1] - f0.y) * kLow));
        pl[n][1] = movmatrix_trans(pack_half2((w[n][2] - f1.x) * kLow, (w[n][3] - f1.y) * kLow));
      }
    }
    // O^T += V^T P^T: the lane's rows are 2 quad, 2 quad + 1, 2 quad + 8, 2 quad + 9; their codes of one dimension are brought
    // together byte by byte
#pragma unroll
    for (int n = 0; n < N; ++n) {
      uint32_t vw[4][D / 32];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = 16 * n + RW::key(2 * quad + (r & 1)) + (r >> 1) * 8;
        if constexpr (D == 128) {
          const uint4 a = lds128(rows + RW::v_off + RW::at(at, row));
          vw[r][0] = a.x; vw[r][1] = a.y; vw[r][2] = a.z; vw[r][3] = a.w;
        } else {
          const uint2 a = lds64(rows + RW::v_off + RW::at(at, row >> 1) + (row & 1) * 8);
          vw[r][0] = a.x; vw[r][1] = a.y;
        }
        if constexpr (MODE == kFirst) {                      // (an e4m3 code behind the last key may be a NaN: 0 * NaN is not 0)
#pragma unroll
          for (int i = 0; i < D / 32; ++i) vw[r][i] = at < (int)arg ? vw[r][i] : 0u;
        }
      }
#pragma unroll
      for (int i = 0; i < D / 32; ++i) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          // (bytes 2 k, 2 k + 1 of either key: dimension 4 i + 2 k of both keys, then dimension 4 i + 2 k + 1)
          const uint32_t sel = k ? 0x7362u : 0x5140u;
          uint32_t a[2], b[2];
          codes_to_half<CODE>(__byte_perm(vw[0][i], vw[1][i], sel), a);
          codes_to_half<CODE>(__byte_perm(vw[2][i], vw[3][i], sel), b);
          const int u = 2 * i + k;
          mma_f16(o[u], a[0], a[1], b[0], b[1], pb[n][0], pb[n][1]);
          if constexpr (kSplit) {
            // (codes divided by kLow instead, four multiplications of halves: 64 x 1000 tokens of 64 heads of 128 38.6 us, this 33.9)
            float low[4] = {};
            mma_f16(low, a[0], a[1], b[0], b[1], pl[n][0], pl[n][1]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[u][e] = fmaf(low[e], 1.f / kLow, o[u][e]);
          }
        }
      }
    }
  }

  // The warp's state to shared memory: [head][kRow] floats, O at position 16 u + 2 row + (0, 1) for dimension D / 8 * row + 2 u +
  // (0, 1), then the reference and the sum.  (kRow: the lanes of a store fall into different banks.)
  static constexpr int kRow = D + 4;
  __device__ __forceinline__ void store(float* mg) {
    const int lane = threadIdx.x & 31, row = lane >> 2, quad = lane & 3;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const float back = __uint_as_float(0x7F000000u - __float_as_uint(unit[e]));            // 1 / unit
      float s = l[e];
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 4);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 8);
      s += __shfl_xor_sync(0xFFFFFFFFu, s, 16);
      float* dst = mg + (2 * quad + e) * kRow;               // (PACK: rows 4 to 7 hold copies)
#pragma unroll
      for (int u = 0; u < KS; ++u) {
        float2 y = make_float2(o[u][e] * back, o[u][2 + e] * back);
        if constexpr (PACK) {
          if (quad >= 2) { y.x *= 1.f / kLow; y.y *= 1.f / kLow; }
          y.x += __shfl_xor_sync(0xFFFFFFFFu, y.x, 2);
          y.y += __shfl_xor_sync(0xFFFFFFFFu, y.y, 2);
        }
        *reinterpret_cast<float2*>(dst + 16 * u + 2 * row) = y;
      }
      if (row == 0) { dst[D] = m[e]; dst[D + 1] = s; }
    }
  }
};

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put2(float* p, float a, float b) { *reinterpret_cast<float2*>(p) = make_float2(a, b); }
__device__ __forceinline__ void put2(__nv_bfloat16* p, float a, float b) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b); }
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.f ? -CUDART_INF_F : (m + log2f(l)) * 0.6931471805599453f; }
// weight of a partial result with reference m under the common reference mx (a partial result without a key has none)
__device__ __forceinline__ float weight(float m, float mx) { return m == -CUDART_INF_F ? 0.f : g_ex2(m - mx); }

// Four positions (p ... p + 3) of a row under a common reference.
struct Fold {
  float m, l;
  float4 o;
  // the rows of `n` warps, `stride` floats apart
  template <int N>
  __device__ __forceinline__ void warps(const float* row, int stride, int d, int p) {
    m = -CUDART_INF_F; l = 0.f;
    o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < N; ++w) m = fmaxf(m, row[w * stride + d]);
#pragma unroll
    for (int w = 0; w < N; ++w) {
      const float f = weight(row[w * stride + d], m);
      add(f, row[w * stride + d + 1], *reinterpret_cast<const float4*>(row + w * stride + p));
    }
  }
  __device__ __forceinline__ void add(float f, float sum, float4 x) {
    l += sum * f;
    o.x += x.x * f; o.y += x.y * f; o.z += x.z * f; o.w += x.w * f;
  }
  // the result: dimension D / 8 * row + 2 u + (0, 1) stands at position 16 u + 2 row + (0, 1)
  template <int D, typename T>
  __device__ __forceinline__ void write(T* O, float* lse, int p) const {
    const float inv = l == 0.f ? 0.f : 1.f / l;              // (no key: O is zero already; a NaN stays one)
    const int at = D / 8 * ((p & 15) >> 1) + 2 * (p >> 4);
    put2(O + at, o.x * inv, o.y * inv);
    put2(O + at + D / 8, o.z * inv, o.w * inv);
    if (p == 0) *lse = lse_of(m, l);
  }
};

// The blocks of a cluster join their results by pushing: element e of the `heads` rows belongs to block e / part; every block folds
// its warps' rows and stores them, and their references and sums, into the shared memory of the blocks they belong to, and after one
// barrier every block has what it needs.  (Blocks that pulled needed a second barrier, and waited for remote reads between the two.)
struct ClusterJoin {
  static constexpr int most = 16, bytes = kGMaxGroup * 128 * 4 + most * kGMaxGroup * 8;
  float* rows;                         // [block][part]
  float2* refs;                        // [block][head]: reference and sum
  __device__ __forceinline__ explicit ClusterJoin(unsigned char* at)
      : rows(reinterpret_cast<float*>(at)), refs(reinterpret_cast<float2*>(at + kGMaxGroup * 128 * 4)) {}
  // a first barrier, early: every block has begun before any is written to
  static __device__ __forceinline__ void begin() { asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory"); }
  template <int D, int WARPS, typename T>
  __device__ __forceinline__ void join(const float* mg, int stride, int heads, T* O, float* lse) const {
    cooperative_groups::cluster_group cl = cooperative_groups::this_cluster();
    const int blocks = (int)cl.num_blocks(), rank = (int)cl.block_rank(), part = heads * D / blocks;
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int e = 4 * threadIdx.x; e < heads * D; e += 4 * blockDim.x) {
      const int g = e / D, p = e % D, to = e / part, first = to * part;
      Fold f;
      f.template warps<WARPS>(mg + g * stride, kGMaxGroup * stride, D, p);
      *reinterpret_cast<float4*>(cl.map_shared_rank(rows, to) + rank * part + e - first) = f.o;
      if (p == 0 || e == first) cl.map_shared_rank(refs, to)[rank * kGMaxGroup + g] = make_float2(f.m, f.l);
    }
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    for (int i = 4 * threadIdx.x; i < part; i += 4 * blockDim.x) {
      const int e = rank * part + i, g = e / D;
      Fold f;
      f.m = -CUDART_INF_F; f.l = 0.f;
      f.o = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < blocks; ++k) f.m = fmaxf(f.m, refs[k * kGMaxGroup + g].x);
      for (int k = 0; k < blocks; ++k) {
        const float2 r = refs[k * kGMaxGroup + g];
        f.add(weight(r.x, f.m), r.y, *reinterpret_cast<const float4*>(rows + k * part + i));
      }
      f.template write<D>(O + g * D, lse + g, e % D);
    }
  }
};

struct CacheDecode {
  const void* q;
  const int32_t* pos;
  int Hq, G, NS;               // query heads, per KV head, and groups of 8 of them per KV head
  float scale_log2;
  void* O;
  float* lse;
  uint32_t* scratch;
  int side;                    // see the next section
};

// ---- every key ----------------------------------------------------------------------------------
// The keys of all sequences form one list of chunks (a tile of 32 keys per warp), and share s of S takes the chunks [total s / S,
// total (s + 1) / S): every SM reads the same number of bytes, however ragged the batch.  side > 1: that many (KV head, group of 8
// heads), all of them, are served side by side, a block for each in every share: the rows that neighbouring blocks read at about the
// same time are neighbours in memory.  side == 1: the list goes through the (KV head, group) of each sequence one after the other.
// Where a share ends inside a sequence's keys it leaves a partial result, and a second kernel joins those.
constexpr int kMaxSms = 148;           // of a B200
// Blocks per SM: one for head_dim 128 (two of four warps: one sequence of 65000 tokens 25.3 -> 26.6 us, 64 x 32k 549 -> 536), two for 64,
// where the ends of a sequence fall under the other's work (against one of 16 warps: 6 ragged fp32 sequences of 4 heads 20.7 -> 18.6 us, 64 x
// 8000 tokens of 8 bf16 heads 86 -> 82, 64 x 16000 143 -> 147; a third stage instead: 19.6 us for the 6).
template <int D> constexpr int kListBlocks = D == 128 ? 1 : 2;

// (EARLY: of the joining kernel, before it waits for the one before it: past the L1 cache, whose lines may be older than that wait)
template <bool EARLY = false>
__device__ __forceinline__ int chunks_of(const DamCacheView& c, const int32_t* pos, int b, int chunk) {
  const int p = EARLY ? __ldcg(pos + b) : __ldg(pos + b), room = __ldg(c.cu + b + 1) - __ldg(c.cu + b);
  return (unsigned)p >= (unsigned)room ? 0 : p / chunk + 1;
}

constexpr int kKeys = kTile * kSlice;    // keys of a warp's tile

// Chunks per head of all sequences, of those before sequence b, and whether some position lies outside its capacity (whole warp).
template <bool EARLY = false>
struct Survey {
  int total, before, mine;     // mine: chunks of sequence `lane`
  bool bad;
  __device__ __forceinline__ Survey(const DamCacheView& c, const int32_t* pos, int chunk, int b) : bad(false) {
    const int lane = threadIdx.x & 31;
    mine = lane < c.num_seqs ? chunks_of<EARLY>(c, pos, lane, chunk) : 0;
    bad = lane < c.num_seqs && mine == 0;
    total = mine;
    before = lane < b ? mine : 0;
    for (int x = 32 + lane; x < c.num_seqs; x += 32) {
      const int n = chunks_of<EARLY>(c, pos, x, chunk);
      bad |= n == 0;
      total += n;
      before += x < b ? n : 0;
    }
    total = __reduce_add_sync(0xFFFFFFFFu, total);
    before = __reduce_add_sync(0xFFFFFFFFu, before);
    bad = __any_sync(0xFFFFFFFFu, bad);
  }
};

// A place in the list of chunks.  Consumers and the copies that run ahead of them walk the list each on their own.
struct Place {
  int b, hg;                   // sequence; KV head and group of heads
  int n, left;                 // chunks of the sequence, and how many are left of this (KV head, group), this one included
  int live;                    // keys of the sequence from the warp's tile of this chunk on (may be none: <= 0)
  __device__ __forceinline__ void begin(const int32_t* pos, int chunk, int k) {
    left = n - k;
    live = __ldg(pos + b) + 1 - k * chunk - (int)(threadIdx.x >> 5) * kKeys;
  }
  // chunk `at` of the whole list (which has it); returns its number within the (KV head, group)
  __device__ __forceinline__ int locate(const DamCacheView& c, const int32_t* pos, const Survey<>& all, int chunk, int heads, int at) {
    const int lane = threadIdx.x & 31;
    int before = 0, mine = all.mine;
    b = hg = 0; n = left = 1; live = 0;
    for (int base = 0; base < c.num_seqs; base += 32) {
      if (base) mine = base + lane < c.num_seqs ? chunks_of(c, pos, base + lane, chunk) : 0;
      int incl = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int y = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += y;
      }
      const uint32_t past = __ballot_sync(0xFFFFFFFFu, (before + incl) * heads > at);
      if (past) {
        const int w = __ffs(past) - 1;
        b = base + w;
        n = __shfl_sync(0xFFFFFFFFu, mine, w);
        int k = at - (before + __shfl_sync(0xFFFFFFFFu, incl, w) - n) * heads;
        if (heads > 1) {
          hg = k / n;
          k -= hg * n;
        }
        begin(pos, chunk, k);
        return k;
      }
      before += __shfl_sync(0xFFFFFFFFu, incl, 31);
    }
    return 0;
  }
  // the next chunk (there is one); whether it is another (KV head, group)'s first
  __device__ __forceinline__ bool next(const DamCacheView& c, const int32_t* pos, int chunk, int heads) {
    if (--left > 0) {
      live -= chunk;
      return false;
    }
    if (++hg == heads) {
      hg = 0;
      do { n = chunks_of(c, pos, ++b, chunk); } while (n == 0 && b + 1 < c.num_seqs);
    }
    begin(pos, chunk, 0);
    return true;
  }
};

template <int D, int WARPS, int STAGES>
struct DenseLayout {
  static constexpr int chunk = WARPS * kKeys;
  static constexpr int ring = WARPS * STAGES * Rows<D, kTile>::bytes;
  static constexpr int merge_off = ring, merge = WARPS * kGMaxGroup * (D + 4) * 4;
  static constexpr int scale_off = merge_off + merge;                           // [warp][stage][slice] K scale, V scale
  static constexpr int bar_off = scale_off + WARPS * STAGES * kTile * 8;        // [warp][stage]
  static constexpr int flag_off = bar_off + WARPS * STAGES * 8;
  static constexpr int total = flag_off + 16 + 1024;                            // (the ring starts on a multiple of 1024)
};
// floats of one partial result: O of 8 heads, references, sums
template <int D> constexpr int kPartial = kGMaxGroup * (D + 2);

// The shares of `total` chunks (below 2^31: the host sees to it): the first `more` have one chunk more than the others.
struct Shares {
  int each, more;
  __device__ __forceinline__ Shares(int total, int shares) : each(total / shares), more(total % shares) {}
  __device__ __forceinline__ int begin(int s) const { return s * each + min(s, more); }
  __device__ __forceinline__ int of(int at) const {           // the share that has chunk `at`
    const int there = more * (each + 1);
    return at < there ? at / (each + 1) : more + (at - there) / each;
  }
};

// The end of a warp that has given up on a copy: those on their way (none otherwise) land before it leaves.
__device__ __forceinline__ void drain(uint32_t bars, int stages, uint32_t phases, uint32_t pending, volatile uint32_t* gave_up) {
  if (pending == 0u) return;
  for (int s = 0; s < stages; ++s)
    if (pending >> s & 1u) sm100::mbar_wait(bars + 8 * s, phases >> s & 1u, gave_up, sm100::kDrainPolls);
}

template <typename T, int D, int CODE, bool PACK, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32, kListBlocks<D>)
cache_decode_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, CacheDecode a, DamCacheView c,
                    float* __restrict__ partial) {
  using LY = DenseLayout<D, WARPS, STAGES>;
  using WS = WarpState<T, D, CODE, PACK>;
  extern __shared__ unsigned char sm_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int heads = a.side > 1 ? 1 : c.Hkv * a.NS;            // of the list
  const int share = blockIdx.x / a.side, beside = blockIdx.x - share * a.side;
  unsigned char* sm = sm_raw + (-sm100::smem_u32(sm_raw) & 1023u);
  float* mg = reinterpret_cast<float*>(sm + LY::merge_off);
  const uint32_t base = sm100::smem_u32(sm), ring = base + warp * (STAGES * Rows<D, kTile>::bytes);
  const uint32_t scales = base + LY::scale_off + warp * (STAGES * kTile * 8), bars = base + LY::bar_off + warp * (STAGES * 8);
  volatile uint32_t* const gave_up = reinterpret_cast<uint32_t*>(sm + LY::flag_off);
  if (lane < STAGES) sm100::mbar_init(bars + 8 * lane, 1);
  if (tid == 0) {
    *gave_up = 0u;
    sm100::tma_prefetch_desc(&kmap);
    sm100::tma_prefetch_desc(&vmap);
  }
  sm100::mbar_fence_init();
  __syncthreads();
  // The joining kernel may begin when this one has seen its predecessors' memory: it reads the positions before it waits for this.
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;");
  const Survey<> all(c, a.pos, LY::chunk, 0);
  // sequences whose position lies outside their capacity get zeros; block 0 says so in the status word
  if (blockIdx.x == 0 && tid < 64) a.scratch[tid] = tid == 1 && all.bad ? (uint32_t)DAM_ERR_INVALID_ARGUMENT : 0u;
  if (all.bad) {
    for (int b = blockIdx.x; b < c.num_seqs; b += gridDim.x) {
      if (chunks_of(c, a.pos, b, LY::chunk)) continue;
      for (int t = tid; t < a.Hq * D; t += WARPS * 32) put(reinterpret_cast<T*>(a.O) + (int64_t)b * a.Hq * D + t, 0.f);
      for (int t = tid; t < a.Hq; t += WARPS * 32) a.lse[(int64_t)b * a.Hq + t] = -CUDART_INF_F;
    }
  }
  const Shares sh(all.total * heads, gridDim.x / a.side);
  const int lo = sh.begin(share), todo = sh.begin(share + 1) - lo;
  if (todo == 0) return;
  Place in, cur;
  int key = in.locate(c, a.pos, all, LY::chunk, heads, lo) * LY::chunk + warp * kKeys;     // first key of the slice to be copied
  cur = in;

  // The copies: a tile of 32 rows of K, one of V, and the scales of its two slices.
  const float* sp;                     // scale of block 0 of the sequence
  int kvh, token;                      // KV head; packed row of the slice's first key
  auto aim = [&]() {
    kvh = a.NS == 1 ? in.hg + beside : (in.hg + beside) / a.NS;
    const int cu = __ldg(c.cu + in.b);
    token = cu + key;
    sp = (lane & 1 ? c.vs : c.ks) + (int64_t)((cu >> c.shift) + in.b) * c.Hkv + kvh;
  };
  uint32_t phases = 0u, pending = 0u;  // bit s: parity of the next copy into stage s; whether one is on its way
  auto issue = [&](int stage) {
    if (in.live <= 0) return;
    pending |= 1u << stage;
    // (16 keys from a multiple of 16 on lie in one block.  A tile may reach into the rows behind the last key, of this sequence
    // or of the next; rows beyond the cache read as zeros.  The scale of a slice without a key is the first slice's)
    if (lane < 2 * kTile) {
      const int at = key + (in.live > (lane >> 1) * kSlice ? (lane >> 1) * kSlice : 0);
      cp_async4_zfill(scales + 8 * kTile * stage + 4 * lane, sp + (int64_t)(at >> c.shift) * c.Hkv, 4u);
    }
    if (sm100::elect_one()) {
      const uint32_t dst = ring + stage * Rows<D, kTile>::bytes, bar = bars + 8 * stage;
      sm100::mbar_arrive_expect_tx(bar, Rows<D, kTile>::bytes);
      sm100::tma_load_3d(dst, &kmap, bar, 0, kvh, token);
      sm100::tma_load_3d(dst + Rows<D, kTile>::v_off, &vmap, bar, 0, kvh, token);
    }
  };
  auto advance = [&]() {
    if (in.next(c, a.pos, LY::chunk, heads)) {
      key = warp * kKeys;
      aim();
    } else {
      token += LY::chunk;
      key += LY::chunk;
    }
  };
  aim();
  // (a group is committed every time, so that "all but the newest STAGES - 1" always includes this chunk's scales)
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) {
    if (s < todo) {
      if (s) advance();
      issue(s);
    }
    cp_async_commit();
  }
  WS ws;
  int stage = 0, ahead = STAGES - 1, segment = 0, since = 0;  // `since`: chunks of the present (KV head, group) behind it
  int h0 = 0, nh = 0;
  bool lost = false;                   // a copy did not arrive: no more are asked for
#pragma unroll 1
  for (int it = 0; it < todo; ++it) {
    if (it + STAGES - 1 < todo) {
      advance();
      if (!lost) issue(ahead);
    }
    cp_async_commit();
    if (since == 0) {
      const int kv = a.NS == 1 ? cur.hg + beside : (cur.hg + beside) / a.NS, sub = cur.hg + beside - kv * a.NS;
      h0 = kv * a.G + sub * kGMaxGroup;
      nh = min(kGMaxGroup, a.G - sub * kGMaxGroup);
      ws.reset();
      ws.set_q(WS::fetch_q(reinterpret_cast<const T*>(a.q) + ((int64_t)cur.b * a.Hq + h0) * D, nh), nh, a.scale_log2);
    }
    cp_async_wait<STAGES - 1>();
    __syncwarp();
    if (cur.live > 0 && !lost) lost = !sm100::mbar_wait(bars + 8 * stage, phases >> stage & 1u, gave_up);
    if (cur.live > 0 && !lost) {
      phases ^= 1u << stage;
      pending ^= 1u << stage;
      const uint32_t rows = ring + stage * Rows<D, kTile>::bytes, sc = scales + 8 * kTile * stage;
      if (cur.live >= kKeys) ws.template step<WS::kAll, kTile>(rows, sc, 0u);
      else ws.template step<WS::kFirst, kTile>(rows, sc, (uint32_t)cur.live);
    }
    __syncwarp();                                            // the stage is free for the copy the next trip issues
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    ahead = ahead + 1 == STAGES ? 0 : ahead + 1;
    ++since;
    if (cur.left == 1 || it + 1 == todo) {
      // ---- the end of this block's share of (sequence, KV head, group): the warps meet
      const bool whole = cur.left == 1 && since == cur.n;
      ws.store(mg + warp * (kGMaxGroup * WS::kRow));
      __syncthreads();
      float* part = partial + (int64_t)(2 * blockIdx.x + (segment > 0)) * kPartial<D>;
      for (int e = 4 * tid; e < nh * D; e += WARPS * 128) {
        const int g = e / D, p = e % D;
        Fold f;
        f.template warps<WARPS>(mg + g * WS::kRow, kGMaxGroup * WS::kRow, D, p);
        if (whole) {
          const int64_t h = (int64_t)cur.b * a.Hq + h0 + g;
          f.template write<D>(reinterpret_cast<T*>(a.O) + h * D, a.lse + h, p);
        } else {
          *reinterpret_cast<float4*>(part + e) = f.o;
          if (p == 0) { part[kGMaxGroup * D + g] = f.m; part[kGMaxGroup * (D + 1) + g] = f.l; }
        }
      }
      __syncthreads();                                       // before the next end overwrites the rows
      ++segment;
      since = 0;
    }
    if (it + 1 < todo) cur.next(c, a.pos, LY::chunk, heads);
  }
  drain(bars, STAGES, phases, pending, gave_up);
  sm100::report_expired_wait(gave_up, a.scratch + 1, (uint32_t)DAM_ERR_DEVICE_TIMEOUT);
}

// Joins the partial results of one (sequence, KV head, group) and head; nothing to do where one block had all its keys.
// grid: head of the group fastest, then (KV head, group), then sequence.
template <typename T, int D>
__global__ void __launch_bounds__(256)
cache_join_kernel(CacheDecode a, DamCacheView c, const float* __restrict__ partial, int chunk, int shares) {
  constexpr int TD = D / 4, WAYS = 256 / TD;                 // threads of a row (4 positions each), partial results at a time
  __shared__ float4 red[WAYS][TD];
  __shared__ float sums[WAYS], refs[WAYS];
  // (before the wait: the positions, which the kernel before this one has read behind its own wait; it writes none)
  asm volatile("griddepcontrol.launch_dependents;");
  const int heads = c.Hkv * a.NS, per = min(a.G, kGMaxGroup);
  const int g = blockIdx.x % per, hg = blockIdx.x / per % heads, b = blockIdx.x / per / heads;
  const int sub = hg % a.NS, nh = min(kGMaxGroup, a.G - sub * kGMaxGroup);
  const int tid = threadIdx.x, way = tid / TD, col = tid % TD;
  const int n = chunks_of<true>(c, a.pos, b, chunk);
  const Survey<true> all(c, a.pos, chunk, b);
  const int list = a.side > 1 ? 1 : heads;
  const Shares sh(max(all.total * list, 1), shares);
  const int first = all.before * list + (a.side > 1 ? 0 : hg * n), s0 = sh.of(first), s1 = n ? sh.of(first + n - 1) : s0;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (g >= nh || n == 0 || s0 == s1) return;
  // (every share from s0 to s1 has chunks; where its first is an earlier (KV head, group)'s, this one's is its second result)
  auto row_of = [&](int s) -> const float* {
    const int block = a.side > 1 ? s * a.side + hg : s;
    return partial + (int64_t)(2 * block + (sh.begin(s) < first)) * kPartial<D>;
  };
  // every thread joins its share of them under a reference of its own
  Fold f;
  f.m = -CUDART_INF_F; f.l = 0.f;
  f.o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = s0 + way; s <= s1; s += 4 * WAYS) {
    float m[4], l[4], mx = f.m;
    float4 o[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float* r = row_of(min(s + k * WAYS, s1));
      m[k] = s + k * WAYS <= s1 ? r[kGMaxGroup * D + g] : -CUDART_INF_F;
      l[k] = r[kGMaxGroup * (D + 1) + g];
      o[k] = *reinterpret_cast<const float4*>(r + g * D + 4 * col);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) mx = fmaxf(mx, m[k]);
    const float w = weight(f.m, mx);
    f.m = mx;
    f.l *= w; f.o.x *= w; f.o.y *= w; f.o.z *= w; f.o.w *= w;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (s + k * WAYS <= s1) f.add(weight(m[k], mx), l[k], o[k]);
  }
  red[way][col] = f.o;
  if (col == 0) { sums[way] = f.l; refs[way] = f.m; }
  __syncthreads();
  if (way == 0) {
    Fold r;
    r.m = -CUDART_INF_F; r.l = 0.f;
    r.o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < WAYS; ++w) r.m = fmaxf(r.m, refs[w]);
#pragma unroll
    for (int w = 0; w < WAYS; ++w) r.add(weight(refs[w], r.m), sums[w], red[w][col]);
    const int64_t h = (int64_t)b * a.Hq + hg / a.NS * a.G + sub * kGMaxGroup + g;
    r.template write<D>(reinterpret_cast<T*>(a.O) + h * D, a.lse + h, 4 * col);
  }
}

// ---- every key of short sequences ---------------------------------------------------------------
// One block, or a cluster of up to sixteen, per (sequence, KV head, group of 8 heads): a single launch, and nothing to look up before
// the first copy but the sequence's own position and bounds.  The partial results of a cluster's blocks meet in shared memory.
// kAlone: blocks of eight warps, one per SM.  kPairs, kFours: two of eight or four of four warps per SM, whose beginnings and ends fall
// under one another's work; no clusters.
enum ShortForm { kAlone, kPairs, kFours };
template <int D, ShortForm FORM>
struct ShortLayout {
  static constexpr int warps = FORM == kFours ? 4 : 8, blocks = FORM == kAlone ? 1 : FORM == kPairs ? 2 : 4;   // blocks per SM
  static constexpr int stages = (FORM == kAlone ? 2 : 1) * (D == 128 ? 1 : 2);
  static constexpr int ring = warps * stages * Rows<D, kTile>::bytes;
  static constexpr int merge_off = ring, merge = warps * kGMaxGroup * (D + 4) * 4;
  static constexpr int join_off = merge_off + merge, scale_off = join_off + (FORM == kAlone ? ClusterJoin::bytes : 0);
  static constexpr int bar_off = scale_off + warps * stages * kTile * 8;
  static constexpr int flag_off = bar_off + warps * stages * 8;
  static constexpr int total = flag_off + 16 + 1024;
};

template <typename T, int D, int CODE, bool PACK, ShortForm FORM>
__global__ void __launch_bounds__(ShortLayout<D, FORM>::warps * 32, (ShortLayout<D, FORM>::blocks))
cache_decode_short_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, CacheDecode a, DamCacheView c) {
  using LY = ShortLayout<D, FORM>;
  using WS = WarpState<T, D, CODE, PACK>;
  constexpr int WARPS = LY::warps, STAGES = LY::stages, kThreads = WARPS * 32, kChunk = WARPS * kKeys;
  extern __shared__ unsigned char sm_raw[];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int blocks = FORM != kAlone ? 1 : (int)cooperative_groups::this_cluster().num_blocks();
  const int rank = FORM != kAlone ? 0 : (int)cooperative_groups::this_cluster().block_rank();
  const int heads = c.Hkv * a.NS, unit = blockIdx.x / blocks, b = unit / heads, hg = unit - b * heads;
  const int kvh = hg / a.NS, sub = hg - kvh * a.NS, h0 = kvh * a.G + sub * kGMaxGroup, nh = min(kGMaxGroup, a.G - sub * kGMaxGroup);
  unsigned char* sm = sm_raw + (-sm100::smem_u32(sm_raw) & 1023u);
  float* mg = reinterpret_cast<float*>(sm + LY::merge_off);
  const uint32_t base = sm100::smem_u32(sm), ring = base + warp * (STAGES * Rows<D, kTile>::bytes);
  const uint32_t scales = base + LY::scale_off + warp * (STAGES * kTile * 8), bars = base + LY::bar_off + warp * (STAGES * 8);
  volatile uint32_t* const gave_up = reinterpret_cast<uint32_t*>(sm + LY::flag_off);
  if (lane < STAGES) sm100::mbar_init(bars + 8 * lane, 1);
  if (tid == 0) {
    *gave_up = 0u;
    sm100::tma_prefetch_desc(&kmap);
    sm100::tma_prefetch_desc(&vmap);
  }
  sm100::mbar_fence_init();
  __syncthreads();
  if (blocks > 1) ClusterJoin::begin();
  dam_chain_prologue();
  const int pos = __ldg(a.pos + b), cu0 = __ldg(c.cu + b), cu1 = __ldg(c.cu + b + 1);
  const typename WS::Query q = WS::fetch_q(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + h0) * D, nh);
  T* O = reinterpret_cast<T*>(a.O) + ((int64_t)b * a.Hq + h0) * D;
  float* lse = a.lse + (int64_t)b * a.Hq + h0;
  const bool bad = (unsigned)pos >= (unsigned)(cu1 - cu0);
  // this block's chunks of the sequence, and the warp's slice in the first of them
  const int n = bad ? 0 : pos / kChunk + 1;
  const Shares sh(n, blocks);
  const int todo = sh.begin(rank + 1) - sh.begin(rank), key0 = sh.begin(rank) * kChunk + warp * kKeys, len = pos + 1;
  const float* sp = (lane & 1 ? c.vs : c.ks) + (int64_t)((cu0 >> c.shift) + b) * c.Hkv + kvh;
  uint32_t phases = 0u, pending = 0u;  // bit s: parity of the next copy into stage s; whether one is on its way
  auto issue = [&](int it, int stage) {
    const int key = key0 + it * kChunk;
    if (key >= len) return;
    pending |= 1u << stage;
    if (lane < 2 * kTile) {
      const int at = key + (key + (lane >> 1) * kSlice < len ? (lane >> 1) * kSlice : 0);
      cp_async4_zfill(scales + 8 * kTile * stage + 4 * lane, sp + (int64_t)(at >> c.shift) * c.Hkv, 4u);
    }
    if (sm100::elect_one()) {
      const uint32_t dst = ring + stage * Rows<D, kTile>::bytes, bar = bars + 8 * stage;
      sm100::mbar_arrive_expect_tx(bar, Rows<D, kTile>::bytes);
      sm100::tma_load_3d(dst, &kmap, bar, 0, kvh, cu0 + key);
      sm100::tma_load_3d(dst + Rows<D, kTile>::v_off, &vmap, bar, 0, kvh, cu0 + key);
    }
  };
#pragma unroll 1
  for (int s = 0; s < STAGES - 1; ++s) {
    if (s < todo) issue(s, s);
    cp_async_commit();
  }
  if (blockIdx.x == 0) {
    // the scratch block for the whole call, its status word included: this block looks at every sequence's position
    bool any = false;
    for (int x = tid; x < c.num_seqs; x += kThreads) any |= chunks_of(c, a.pos, x, kChunk) == 0;
    const int st = __syncthreads_or(any) ? (int)DAM_ERR_INVALID_ARGUMENT : 0;
    if (tid < 64) a.scratch[tid] = tid == 1 ? (uint32_t)st : 0u;
  }
  WS ws;
  ws.reset();
  ws.set_q(q, nh, a.scale_log2);
  int stage = 0, ahead = STAGES - 1;
  bool lost = false;                   // a copy did not arrive: no more are asked for
#pragma unroll 1
  for (int it = 0; it < todo; ++it) {
    if (it + STAGES - 1 < todo && !lost) issue(it + STAGES - 1, ahead);
    cp_async_commit();
    cp_async_wait<STAGES - 1>();
    __syncwarp();
    // (with one stage the copy has just been asked for, and the other warps of the SM cover the wait)
    const int live = len - (key0 + it * kChunk);
    if (live > 0 && !lost) lost = !sm100::mbar_wait(bars + 8 * stage, phases >> stage & 1u, gave_up);
    if (live > 0 && !lost) {
      phases ^= 1u << stage;
      pending ^= 1u << stage;
      const uint32_t rows = ring + stage * Rows<D, kTile>::bytes, sc = scales + 8 * kTile * stage;
      if (live >= kKeys) ws.template step<WS::kAll, kTile>(rows, sc, 0u);
      else ws.template step<WS::kFirst, kTile>(rows, sc, (uint32_t)live);
    }
    __syncwarp();                                            // the stage is free for the copy the next trip issues
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    ahead = ahead + 1 == STAGES ? 0 : ahead + 1;
  }
  // (a sequence whose position lies outside its capacity has no chunk: O = 0, LSE = -inf)
  ws.store(mg + warp * (kGMaxGroup * WS::kRow));
  __syncthreads();
  if (blocks > 1) {
    ClusterJoin(sm + LY::join_off).template join<D, WARPS>(mg, WS::kRow, nh, O, lse);
  } else {
    for (int e = 4 * tid; e < nh * D; e += 4 * kThreads) {
      Fold f;
      f.template warps<WARPS>(mg + e / D * WS::kRow, kGMaxGroup * WS::kRow, D, e % D);
      f.template write<D>(O + e / D * D, lse + e / D, e % D);
    }
  }
  drain(bars, STAGES, phases, pending, gave_up);
  sm100::report_expired_wait(gave_up, a.scratch + 1, (uint32_t)DAM_ERR_DEVICE_TIMEOUT);
}

// ---- the keys of the stored patterns ------------------------------------------------------------
// As decode_group_kernel (dam_decode_mma.cu): one block, or a cluster of two to eight, per (sequence, KV head, group of 8 heads)
// expands the patterns of its heads into one key list and deals its slices of 16 keys to the warps.  Rows are gathered by cp.async.
// 64 sequences of 16k to 32k tokens, window 1024 (440 keys a list, 48 MB): 19 us, of which 4 until the first rows are asked for
// (header and position, sequence record, words: three dependent reads; then the list), 10 of gathering, 1 to 2 of joining.  One
// sequence of 8000: 7.4 us.
constexpr int kMWarps = 5, kMStages = 2, kMBlocks = 4;
constexpr int kScales = 2 * kSlice * 4;         // bytes of the scales of a slice

constexpr int kRoundWords = 64;       // pattern words expanded per round (at most 2048 keys)

// A listed key: which of the group's heads keep it (bits 0 .. 7), and the column (bits 9 ...) or, with bit 8, the diagonal it is on
// (both lie below the window, whose map of L^2 bits fits a memory: far below 2^23).
__device__ __forceinline__ int listed_key(uint32_t entry, int pos) {
  const int at = (int)(entry >> 9);
  return entry & 256u ? pos - at : at;
}

// One round of the key list of `G` heads (h0, h0 + 1, ...): kRoundWords pattern words from word w0 on, a thread per word, the words
// of all heads OR-ed into `list`.  `words`: kGMaxGroup + 2 rows of kRoundWords words.  By all threads of the block; returns the number
// of listed keys.
template <int WARPS>
__device__ __forceinline__ int expand_round(const unsigned char* blob, const DamHeader* H, const DamSeq& sq, int h0, int G, bool in_window,
                                            int pos, int w0, int nwords, uint32_t* list, uint32_t* words, uint64_t keep_policy) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, W = sq.W;
  const int used = min(kRoundWords, nwords - w0);
  uint32_t* const unions = words + kGMaxGroup * kRoundWords;
  uint32_t* const begins = unions + kRoundWords;
  __syncthreads();                                        // the previous round's list is no longer read
  if (warp * 32 < kRoundWords) {
    uint32_t uni = 0u;
    if (warp * 32 < used) {
      const int wi = w0 + tid;
      const bool mine = tid < used;
      // The words of all heads are requested before any is looked at: one trip to memory, not one per head.  Below the window,
      // word wi >= W holds diagonals: diagonal r = 32 (wi - W) + k selects key pos - r; dropped when that key is a matched column
      // of the head (then it is in the list already): bit k of the reversed 32-bit window of V that ends at key pos - 32 (wi - W).
      const bool diagonals = mine && !in_window && wi >= W;
      const int own = pos - 32 * wi;                      // bit of the word that is the row's own position
      const uint32_t upto = own < 0 ? 0u : own >= 31 ? 0xFFFFFFFFu : (2u << own) - 1u;
      const DamHeadBits hb = dam_head_bits(blob, H, sq, h0);
      const uint32_t* word = in_window ? hb.M + (size_t)pos * W + wi : wi < W ? hb.V + wi : hb.D + (wi - W);
      const int64_t per_head = in_window ? (int64_t)sq.L * W : 3ll * W;
      const int x = pos - 32 * (wi - W) - 31, xw = x >> 5;
#pragma unroll
      for (int g0 = 0; g0 < kGMaxGroup; g0 += 4) {        // (four heads at a time: most groups have no more)
        uint32_t wh[4], lo[4], hi[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int g = g0 + i;
          wh[i] = lo[i] = hi[i] = 0u;
          if (g0 < G) {
            if (mine && g < G) wh[i] = ldg_keep(word + g * per_head, keep_policy);
            if (diagonals && g < G && xw >= 0 && xw < W) lo[i] = ldg_keep(hb.V + 3ll * W * g + xw, keep_policy);
            if (diagonals && g < G && xw + 1 >= 0 && xw + 1 < W) hi[i] = ldg_keep(hb.V + 3ll * W * g + xw + 1, keep_policy);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          wh[i] &= ~__brev(__funnelshift_r(lo[i], hi[i], x & 31));
          if (in_window) wh[i] &= upto;                   // (a map of the caller's may have cells above its diagonal)
          words[(g0 + i) * kRoundWords + tid] = wh[i];
          uni |= wh[i];
        }
      }
    }
    // where the keys of a word begin in the list: within the warp's words (the other warp's are added below)
    const int cnt = __popc(uni);
    int off = cnt;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(0xFFFFFFFFu, off, o);
      if (lane >= o) off += y;
    }
    unions[tid] = uni;
    begins[tid] = (uint32_t)(off - cnt);
  }
  __syncthreads();
  static_assert(kRoundWords == 64, "two warps have the words");
  const int first = (int)begins[31] + __popc(unions[31]), total = first + (int)begins[63] + __popc(unions[63]);
  // the words are spread to the warps, a lane per bit (a thread that took its own word's bits one by one needed up to 32 steps, and
  // the words of a band are full)
  for (int w = warp; w < used; w += WARPS) {
    const uint32_t uni = unions[w];
    if (uni >> lane & 1u) {
      uint32_t heads = 0u;
#pragma unroll
      for (int g = 0; g < kGMaxGroup; ++g)
        if (g < 4 || G > 4) heads |= (words[g * kRoundWords + w] >> lane & 1u) << g;
      const int wi = w0 + w;
      const uint32_t at = in_window || wi < W ? 32u * wi + lane : 32u * (wi - W) + lane;
      list[begins[w] + (w < 32 ? 0 : first) + __popc(uni & ((1u << lane) - 1u))] = at << 9 | (in_window || wi < W ? 0u : 256u) | heads;
    }
  }
  __syncthreads();
  return total;
}

template <int D, bool CLUSTER>
struct MaskedLayout {
  static constexpr int ring = kMWarps * kMStages * (Rows<D, 1>::bytes + kScales);
  static constexpr int merge = kMWarps * kGMaxGroup * (D + 4) * 4;              // the merge reuses the ring
  static constexpr int list_off = ring > merge ? ring : merge;
  static constexpr int words_off = list_off + kRoundWords * 32 * 4;
  static constexpr int join_off = words_off + (kGMaxGroup + 2) * kRoundWords * 4;
  static constexpr int total = join_off + (CLUSTER ? ClusterJoin::bytes : 0);
};

template <typename T, int D, int CODE, bool PACK, bool CLUSTER>
__global__ void __launch_bounds__(kMWarps * 32, CLUSTER || sizeof(T) == 4 ? 3 : kMBlocks)
cache_decode_masked_kernel(CacheDecode a, DamCacheView c, const unsigned char* __restrict__ blob) {
  dam_chain_prologue();
  using LY = MaskedLayout<D, CLUSTER>;
  using WS = WarpState<T, D, CODE, PACK>;
  constexpr int kThreads = kMWarps * 32;
  extern __shared__ __align__(128) unsigned char sm[];
  uint32_t* list = reinterpret_cast<uint32_t*>(sm + LY::list_off);
  uint32_t* words = reinterpret_cast<uint32_t*>(sm + LY::words_off);
  const int nsplit = CLUSTER ? (int)cooperative_groups::this_cluster().num_blocks() : 1;
  const int split = CLUSTER ? (int)cooperative_groups::this_cluster().block_rank() : 0;
  const int heads = c.Hkv * a.NS, unit = blockIdx.x / nsplit, hg = unit % heads, b = unit / heads;
  const int kvh = hg / a.NS, sub = hg % a.NS, h0 = kvh * a.G + sub * kGMaxGroup, nh = min(kGMaxGroup, a.G - sub * kGMaxGroup);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, row = lane >> 2, quad = lane & 3;
  const DamHeader* H = reinterpret_cast<const DamHeader*>(blob);
  // (the header, the position, the bounds and the queries are requested together: one round trip to memory)
  const int pos = __ldg(a.pos + b), cu0 = __ldg(c.cu + b), cu1 = __ldg(c.cu + b + 1);
  const typename WS::Query q = WS::fetch_q(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + h0) * D, nh);
  const bool bad_blob = H->magic != DAM_MAGIC || H->num_seqs != c.num_seqs || H->num_q_heads != a.Hq;
  const bool bad = bad_blob || pos < 0 || pos >= cu1 - cu0;
  T* O = reinterpret_cast<T*>(a.O) + ((int64_t)b * a.Hq + h0) * D;
  float* lse = a.lse + (int64_t)b * a.Hq + h0;
  if (blockIdx.x == 0) {
    bool any = bad_blob;
    for (int x = tid; x < c.num_seqs; x += kThreads) any |= chunks_of(c, a.pos, x, 1) == 0;
    const int st = __syncthreads_or(any) ? (int)DAM_ERR_INVALID_ARGUMENT : 0;
    if (tid < 64) a.scratch[tid] = tid == 1 ? (uint32_t)st : 0u;
  }
  if (bad) {
    if (split == 0) {
      for (int t = tid; t < nh * D; t += kThreads) put(O + t, 0.f);
      if (tid < nh) lse[tid] = -CUDART_INF_F;
    }
    return;                                                  // (all blocks of a cluster)
  }
  if constexpr (CLUSTER) ClusterJoin::begin();
  const DamSeq sq = reinterpret_cast<const DamSeq*>(blob + H->off_seq)[b];
  const int L = sq.L, W = sq.W;
  const bool in_window = pos < L;
  const int nwords = in_window ? W : 2 * W;
  const unsigned char* Kb = c.k + (int64_t)cu0 * c.kst + (int64_t)kvh * c.ksh;
  const unsigned char* Vb = c.v + (int64_t)cu0 * c.vst + (int64_t)kvh * c.vsh;
  const int64_t row0 = (cu0 >> c.shift) + b;
  WS ws;
  ws.reset();
  ws.set_q(q, nh, a.scale_log2);
  const uint32_t ring = static_cast<uint32_t>(__cvta_generic_to_shared(sm)) + warp * (kMStages * (Rows<D, 1>::bytes + kScales));
  const uint64_t stream_policy = l2_evict_first_policy(), keep_policy = l2_evict_last_policy();
  constexpr int P = Rows<D, 1>::pieces, kRowsAtOnce = 32 / P;
  const unsigned char *kp = Kb + lane % P * 16, *vp = Vb + lane % P * 16;
  const float* sp = (lane < 16 ? c.ks : c.vs) + row0 * c.Hkv + kvh;
  const int kst = (int)c.kst, vst = (int)c.vst;              // (the host has seen to it that they are 32-bit numbers)
  for (int w0 = 0; w0 < nwords; w0 += kRoundWords) {
    const int total = expand_round<kMWarps>(blob, H, sq, h0, nh, in_window, pos, w0, nwords, list, words, keep_policy);
    const int nslices = (total + kSlice - 1) / kSlice, first = split * kMWarps + warp, step = nsplit * kMWarps;
    auto issue = [&](int s, int stage) {
      const uint32_t dst = ring + stage * (Rows<D, 1>::bytes + kScales);
      // lane: key `lane & 15` of the slice (places past the end repeat the first key; nobody keeps them below)
      const int idx = s * kSlice + (lane & 15), j = listed_key(list[idx < total ? idx : s * kSlice], pos);
#pragma unroll
      for (int i = 0; i < kSlice / kRowsAtOnce; ++i) {
        const int r = lane / P + kRowsAtOnce * i, key = __shfl_sync(0xFFFFFFFFu, j, r);
        const uint32_t at = Rows<D, 1>::at(r, lane % P);
        cp_async16(dst + at, kp + (int64_t)key * kst, stream_policy);
        cp_async16(dst + Rows<D, 1>::v_off + at, vp + (int64_t)key * vst, stream_policy);
      }
      cp_async4_zfill(dst + Rows<D, 1>::bytes + 4 * lane, sp + (int64_t)(j >> c.shift) * c.Hkv, 4u);
    };
#pragma unroll
    for (int s = 0; s < kMStages - 1; ++s) {
      if (first + s * step < nslices) issue(first + s * step, s);
      cp_async_commit();
    }
    int it = 0;
    for (int s = first; s < nslices; s += step, ++it) {
      if (s + (kMStages - 1) * step < nslices) issue(s + (kMStages - 1) * step, (it + kMStages - 1) % kMStages);
      cp_async_commit();
      cp_async_wait<kMStages - 1>();
      __syncwarp();
      uint32_t keep = 0u;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int idx = s * kSlice + Rows<D, 1>::key(row) + 8 * k;
        if (idx < total) keep |= (list[idx] >> WS::head_of(2 * quad) & 3u) << (2 * k);
      }
      const uint32_t slice = ring + it % kMStages * (Rows<D, 1>::bytes + kScales);
      ws.template step<WS::kKeep, 1>(slice, slice + Rows<D, 1>::bytes, keep);
      __syncwarp();                                          // the stage is free for the copy the next trip issues
    }
    cp_async_wait<0>();                                      // (only empty groups are left; the merge reuses the ring)
  }
  // ---- merge: the warps of the block, then the blocks of the cluster
  __syncthreads();
  float* mg = reinterpret_cast<float*>(sm);
  ws.store(mg + warp * (kGMaxGroup * WS::kRow));
  __syncthreads();
  if constexpr (CLUSTER) {
    ClusterJoin(sm + LY::join_off).template join<D, kMWarps>(mg, WS::kRow, nh, O, lse);
  } else {
    for (int e = 4 * tid; e < nh * D; e += 4 * kThreads) {
      Fold f;
      f.template warps<kMWarps>(mg + e / D * WS::kRow, kGMaxGroup * WS::kRow, D, e % D);
      f.template write<D>(O + e / D * D, lse + e / D, e % D);
    }
  }
}

// Blocks per (sequence, KV head, group): a block spends 4 us before its first rows arrive and then streams its list, so sharing the
// list pays as long as all clusters are resident at once: 48 of 8 blocks (three per SM), 104 of 4, 222 of 2.  us a pass with 8 / 4 /
// 2 / 1 blocks (4 heads of one KV head, head_dim 128, 4000 tokens, window 1024):
//    40 units   8.5 /  8.6 /  9.5 / 13.1        104 units   20.2 / 10.1 / 10.9 / 13.2        222 units   36.2 / 22.6 / 12.8 / 17.3
//    56        13.5 /  9.6 /  9.7 / 13.1        112         21.1 / 14.4 / 11.3 / 13.2        240         37.8 / 23.5 / 17.3 / 18.4
int masked_split(int64_t units) { return units <= 48 ? 8 : units <= 104 ? 4 : units <= 222 ? 2 : 1; }

// the shared memory a kernel wants, asked for once per device (KEY: a set-up step of its own per instance)
template <auto KERNEL, int BYTES, bool LARGE_CLUSTER = false>
cudaError_t opt_in(int key, int* sm_count) {
  int dev = 0;
  DamDeviceInfo di;
  const cudaError_t e = dam_current_device(&dev, &di);
  if (e != cudaSuccess) return e;
  *sm_count = di.sm_count;
  if (di.smem_optin < BYTES) return cudaErrorNotSupported;
  return dam_device_table().once(dev, key, [](void) -> cudaError_t {
    const cudaError_t r = cudaFuncSetAttribute(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, BYTES);
    return r != cudaSuccess || !LARGE_CLUSTER ? r : cudaFuncSetAttribute(KERNEL, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  });
}

// instance number of <T, D, CODE, PACK>, one of 12
template <typename T, int D, int CODE, bool PACK> constexpr int kInstance = (PACK ? 8 : sizeof(T) == 4 ? 4 : 0) + (D == 128) * 2 + CODE;

// Short sequences get a cluster each: of so many blocks that all are resident at once, one per SM (148, 74, 33, 15 and 7 clusters
// of 1, 2, 4, 8 and 16 blocks: the SMs of a GPC are not a multiple), and no more than have a chunk.  0: there are too many of them.
int short_split(int64_t units, int64_t longest, int chunk) {
  static const struct { int split, resident; } sizes[] = {{16, 7}, {8, 15}, {4, 33}, {2, 74}, {1, 148}};
  for (const auto& s : sizes)
    if (units <= s.resident && (s.split == 1 || longest > (int64_t)s.split / 2 * chunk)) return s.split;
  return 0;
}
// capacity per block up to which they are short: large clusters leave more SMs without one
int64_t short_keys(int split) { return split >= 8 ? 1024 : 2048; }
// Batches of more (sequence, KV head, group) than SMs, in us a pass (capacities of equal length; 8 KV heads of 128, int8 / 4 of 64, fp32
// queries; one block each as kPairs, as kFours, or the list that all SMs share):
//    20 x 1000   13 / 20 / 16        64 x 1000   26 / 25 / 39        256 x 500   54 / 46 / 113        64 x 8000   145 / 152 / 135
//    40 x 3000   45 / 54 / 46        64 x 4000   76 / 80 / 80        64 x 1000 of 64  9 / 13 / 18     64 x 4000 of 64  25 / 41 / 32
// A block each, then, up to 4096 tokens, unless one sequence is longer than an SM's part of all of them.
constexpr int64_t kManyKeys = 4096;

template <typename T, int D, int CODE, bool PACK, ShortForm FORM>
cudaError_t launch_short(const CacheDecode& a, const DamCacheView& c, const CUtensorMap& kmap, const CUtensorMap& vmap, int64_t units, int split,
                         cudaStream_t st) {
  using LY = ShortLayout<D, FORM>;
  if (units * split > 0x7FFFFFFF) return cudaErrorNotSupported;
  int sms = 0;
  const cudaError_t e = opt_in<cache_decode_short_kernel<T, D, CODE, PACK, FORM>, LY::total, FORM == kAlone>(
      DAM_SETUP_CACHE_SMEM + 36 + 12 * FORM + kInstance<T, D, CODE, PACK>, &sms);
  if (e != cudaSuccess) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * split)); cfg.blockDim = dim3(LY::warps * 32); cfg.dynamicSmemBytes = LY::total; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = FORM == kAlone ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, cache_decode_short_kernel<T, D, CODE, PACK, FORM>, kmap, vmap, a, c);
}

template <typename T, int D, int CODE, bool PACK>
cudaError_t launch_dense(CacheDecode a, const DamCacheView& c, const dam_cache_t* cache, cudaStream_t st) {
  // (two stages, 128 KB per SM on their way or at work, for either head_dim: a third made 64 x 32k tokens 568 us instead of 549)
  constexpr int WARPS = 8, STAGES = 2;
  using LY = DenseLayout<D, WARPS, STAGES>;
  int sms = 0;
  cudaError_t e = opt_in<cache_decode_kernel<T, D, CODE, PACK, WARPS, STAGES>, LY::total>(DAM_SETUP_CACHE_SMEM + kInstance<T, D, CODE, PACK>, &sms);
  if (e != cudaSuccess) return e;
  const int64_t heads = (int64_t)c.Hkv * a.NS;
  int64_t most = 0, longest = 0;
  for (int b = 0; b < c.num_seqs; ++b) {
    const int64_t len = (int64_t)cache->cu_seqlens_host[b + 1] - cache->cu_seqlens_host[b];
    most += (len + LY::chunk - 1) / LY::chunk;
    longest = len > longest ? len : longest;
  }
  if (most * heads > 0x7FFFFFFF) return cudaErrorNotSupported;
  CUtensorMap kmap, vmap;
  if (!dam_make_tmap_codes(&kmap, c.k, D, c.Hkv, cache->total_tokens, c.kst, c.ksh, kKeys) ||
      !dam_make_tmap_codes(&vmap, c.v, D, c.Hkv, cache->total_tokens, c.vst, c.vsh, kKeys))
    return cudaErrorInvalidValue;
  const int blocks = sms < kMaxSms ? sms : kMaxSms;

  const int64_t units = heads * c.num_seqs;
  const int split = short_split(units, longest, ShortLayout<D, kAlone>::warps * kKeys);
  if (split && longest <= split * short_keys(split)) return launch_short<T, D, CODE, PACK, kAlone>(a, c, kmap, vmap, units, split, st);
  if (!split && longest <= kManyKeys && longest * blocks <= cache->total_tokens * heads)
    return units <= 4 * blocks ? launch_short<T, D, CODE, PACK, kPairs>(a, c, kmap, vmap, units, 1, st)
                               : launch_short<T, D, CODE, PACK, kFours>(a, c, kmap, vmap, units, 1, st);

  // all heads side by side where that leaves no more than an eighth of the blocks' places without work; and no more shares than
  // there can be chunks
  const int places = blocks * kListBlocks<D>;
  a.side = heads > 1 && heads <= places && places % heads * 8 <= places ? (int)heads : 1;
  int64_t shares = places / a.side;
  const int64_t list = a.side > 1 ? most : most * heads;
  if (list < shares) shares = list > 0 ? list : 1;
  float* partial = reinterpret_cast<float*>(a.scratch + 64);
  e = dam_launch_chained(cache_decode_kernel<T, D, CODE, PACK, WARPS, STAGES>, dim3((unsigned)(shares * a.side)), dim3(WARPS * 32), LY::total, st, kmap,
                         vmap, a, c, partial);
  if (e != cudaSuccess || shares == 1 || longest <= LY::chunk) return e;   // (then every sequence is whole in one block)
  const int64_t grid = heads * (a.G < kGMaxGroup ? a.G : kGMaxGroup) * c.num_seqs;
  if (grid > 0x7FFFFFFF) return cudaErrorNotSupported;
  return dam_launch_chained(cache_join_kernel<T, D>, dim3((unsigned)grid), dim3(256), 0, st, a, c, (const float*)partial, LY::chunk, (int)shares);
}

template <typename T, int D, int CODE, bool PACK>
cudaError_t launch_masked(const CacheDecode& a, const DamCacheView& c, const void* mask, cudaStream_t st) {
  constexpr int kOne = MaskedLayout<D, false>::total, kMany = MaskedLayout<D, true>::total;
  int sms = 0;
  cudaError_t e = opt_in<cache_decode_masked_kernel<T, D, CODE, PACK, false>, kOne>(DAM_SETUP_CACHE_SMEM + 12 + kInstance<T, D, CODE, PACK>, &sms);
  if (e == cudaSuccess) e = opt_in<cache_decode_masked_kernel<T, D, CODE, PACK, true>, kMany>(DAM_SETUP_CACHE_SMEM + 24 + kInstance<T, D, CODE, PACK>, &sms);
  if (e != cudaSuccess) return e;
  const int64_t units = (int64_t)c.num_seqs * c.Hkv * a.NS;
  const int split = masked_split(units);
  if (units * split > 0x7FFFFFFF) return cudaErrorNotSupported;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(units * split)); cfg.blockDim = dim3(kMWarps * 32); cfg.dynamicSmemBytes = split > 1 ? kMany : kOne; cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)split; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, split > 1 ? cache_decode_masked_kernel<T, D, CODE, PACK, true> : cache_decode_masked_kernel<T, D, CODE, PACK, false>, a, c,
                            reinterpret_cast<const unsigned char*>(mask));
}

template <typename T, int D, int CODE>
cudaError_t launch(const CacheDecode& a, const dam_cache_t* cache, const void* mask, cudaStream_t st) {
  const DamCacheView c = dam_cache_view(cache);
  if constexpr (sizeof(T) == 4)
    if (a.G <= kPackGroup) return mask ? launch_masked<T, D, CODE, true>(a, c, mask, st) : launch_dense<T, D, CODE, true>(a, c, cache, st);
  return mask ? launch_masked<T, D, CODE, false>(a, c, mask, st) : launch_dense<T, D, CODE, false>(a, c, cache, st);
}

}  // namespace

size_t dam_cache_scratch_bytes(int head_dim) {
  return 256 + 2ull * kMaxSms * 4 * (head_dim == 128 ? kListBlocks<128> * kPartial<128> : kListBlocks<64> * kPartial<64>);
}

cudaError_t dam_launch_cache_decode(const void* q, const dam_cache_t* cache, const void* mask, const int32_t* positions, int Hq, int dtype,
                                    float scale, void* O, float* lse, void* scratch, cudaStream_t st) {
  const int G = Hq / cache->num_kv_heads;
  const CacheDecode a = {q, positions, Hq, G, (G + kGMaxGroup - 1) / kGMaxGroup, scale * 1.4426950408889634f, O, lse,
                         reinterpret_cast<uint32_t*>(scratch), 1};
  return DAM_CACHE_DISPATCH(launch, dtype, cache->head_dim, cache->code, a, cache, mask, st);
}
