// What the generation kernels that serve a whole GQA group at once share: the expansion of the stored patterns into one key
// list per group, asynchronous copies, the transposition of a matrix fragment (dam_decode_mma.cu for a bf16 cache,
// dam_cache_decode.cu for a cache held in 8 bits).
#pragma once
#include "dam_internal.cuh"

namespace {

constexpr int kGRoundWords = 128;     // pattern words expanded per round (at most 4096 keys)
constexpr int kGMaxSplit = 8;         // blocks of a cluster (the largest portable size)
constexpr int kGMaxGroup = 8;         // query heads a block takes (one side of the warp-level instructions' tiles)

__device__ __forceinline__ float g_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// K / V rows are read once per launch: they are marked to leave L2 first, so that the few lines every launch reads
// again (blob header, sequence records, pattern words, queries) are still there next time
__device__ __forceinline__ uint64_t l2_evict_first_policy() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint64_t l2_evict_last_policy() {
  uint64_t p;
  asm volatile("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(p));
  return p;
}
__device__ __forceinline__ uint32_t ldg_keep(const uint32_t* ptr, uint64_t policy) {
  uint32_t v;
  asm volatile("ld.global.nc.L2::cache_hint.u32 %0, [%1], %2;" : "=r"(v) : "l"(ptr), "l"(policy));
  return v;
}
// bits [x, x + 32) of a bit array of nwords words, zero outside it (x may be negative)
__device__ __forceinline__ uint32_t window32_keep(const uint32_t* bits, int nwords, int x, uint64_t policy) {
  const int w = x >> 5, sh = x & 31;
  const uint32_t lo = (w >= 0 && w < nwords) ? ldg_keep(bits + w, policy) : 0u;
  const uint32_t hi = (w + 1 >= 0 && w + 1 < nwords) ? ldg_keep(bits + w + 1, policy) : 0u;
  return __funnelshift_r(lo, hi, sh);
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint64_t policy) {
  asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
// transpose of an 8 x 8 matrix of 16-bit elements held one row pair per lane (the accumulator layout of two columns)
__device__ __forceinline__ uint32_t movmatrix_trans(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// One round of the key list of `G` heads (h0, h0 + 1, ...): kGRoundWords pattern words from word w0 on, a thread per word, the
// words of all heads OR-ed.  A listed key is stored as (word, bit) of the round in `codes`; which heads keep it is read back
// from the round's words in `whs`, [head][word].  By all threads of the block (WARPS warps, at least kGRoundWords threads);
// returns the number of listed keys.
template <int WARPS>
__device__ __forceinline__ int expand_round(const unsigned char* blob, const DamHeader* H, const DamSeq& sq, int h0, int G, bool in_window,
                                            int pos, int w0, int nwords, unsigned short* codes, uint32_t* whs, int* warp_tot,
                                            uint64_t keep_policy) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, W = sq.W;
  const int wi = w0 + tid;                                // (threads beyond the round's words hold no word)
  uint32_t wh[kGMaxGroup], uni = 0u;
#pragma unroll
  for (int g = 0; g < kGMaxGroup; ++g) {
    wh[g] = 0u;
    if (g < G && tid < kGRoundWords && wi < nwords) {
      const DamHeadBits hb = dam_head_bits(blob, H, sq, h0 + g);
      if (in_window) {
        wh[g] = ldg_keep(hb.M + (size_t)pos * W + wi, keep_policy);
      } else if (wi < W) {
        wh[g] = ldg_keep(hb.V + wi, keep_policy);
      } else {
        // diagonal r = 32 (wi - W) + k selects key pos - r; dropped when that key is a matched column of the head
        // (then it is in the list already): bit k of the reversed 32-bit window of V that ends at key pos - 32 (wi - W)
        const int r0 = 32 * (wi - W);
        wh[g] = ldg_keep(hb.D + (wi - W), keep_policy) & ~__brev(window32_keep(hb.V, W, pos - r0 - 31, keep_policy));
      }
      uni |= wh[g];
    }
  }
  const int cnt = __popc(uni);
  int off = cnt;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(0xFFFFFFFFu, off, o);
    if (lane >= o) off += y;
  }
  __syncthreads();                                        // the previous round's list is no longer read
  if (lane == 31) warp_tot[warp] = off;
  if (tid < kGRoundWords) {
#pragma unroll
    for (int g = 0; g < kGMaxGroup; ++g) whs[g * kGRoundWords + tid] = wh[g];
  }
  __syncthreads();
  int total = 0, before = 0;
#pragma unroll
  for (int w = 0; w < WARPS; ++w) {
    const int wt = warp_tot[w];
    if (w < warp) before += wt;
    total += wt;
  }
  off += before - cnt;
  while (uni) {
    const int k = __ffs(uni) - 1;
    uni &= uni - 1u;
    codes[off++] = (unsigned short)(tid * 32 + k);
  }
  __syncthreads();
  return total;
}

}  // namespace
