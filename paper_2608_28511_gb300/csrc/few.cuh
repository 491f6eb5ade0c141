// Device code shared by the few-token layer's kernels (few.cu, few_tc.cu): the
// expert-grouped row lists and the grid barrier.  At most kFewT tokens, so all
// lists live in shared memory and every block builds them for itself from the
// router's choice.
#pragma once

#include <math_constants.h>

#include "common.cuh"
#include "launch.h"

namespace moe {
namespace few {

constexpr int kMaskWords = kFewT / 32;
static_assert(kMaskWords == 4, "an expert's token mask is one 16-byte vector");
constexpr int kMaxSlots = kFewT * kMaxK;
constexpr uint64_t kBarrierLimitNs = 4000000000ull;

// The routed slots of all tokens, in shared memory: row r (expert-grouped,
// stable in the token) is slot slot[r] of token tok[r]; expert active[i] owns
// rows off[e] .. off[e + 1].
struct Lists {
  uint16_t slot[kMaxSlots];
  uint8_t tok[kMaxSlots];
  int off[kMaxE + 1];
  uint8_t active[kMaxE];
  int nact;
};
// What building them takes: the tokens of every expert, one bit each, and the
// expert of every slot.
struct alignas(16) ListScratch {
  uint32_t mask[kMaxE][kMaskWords];
  uint8_t sel[kMaxSlots];
};

__device__ __forceinline__ uint32_t order_bits(float key) {
  if (key != key) key = -CUDART_INF_F;  // NaN counts as -inf
  if (key == 0.f) key = 0.f;            // -0 ties with +0
  const uint32_t b = __float_as_uint(key);
  return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ float order_value(uint32_t o) {
  return __uint_as_float((o & 0x80000000u) ? (o & 0x7fffffffu) : ~o);
}
__device__ __forceinline__ float sigmoid_rn(float z) { return __frcp_rn(1.0f + __expf(-z)); }

// Fills L from the T tokens' chosen experts (every thread of the block calls it).
__device__ __forceinline__ void build_lists(Lists& L, ListScratch& S, const int32_t* topk_idx, int T, int K) {
  const int tid = threadIdx.x, nt = blockDim.x, warp = tid >> 5, lane = tid & 31;
  const int first = tid < T * K ? __ldcg(topk_idx + tid) : 0;  // under the clearing
  for (int i = tid; i < kMaxE; i += nt) *reinterpret_cast<uint4*>(S.mask[i]) = make_uint4(0, 0, 0, 0);
  __syncthreads();
  for (int s = tid; s < T * K; s += nt) {
    const int e = s == tid ? first : __ldcg(topk_idx + s), t = s / K;
    S.sel[s] = (uint8_t)e;
    atomicOr(&S.mask[e][t >> 5], 1u << (t & 31));
  }
  __syncthreads();
  if (warp == 0) {
    // exclusive prefix over the experts of their row counts and of "has rows",
    // eight consecutive experts a lane, both in one 32-bit sum (rows < 2^16)
    uint32_t v[kMaxE / 32], sum = 0;
#pragma unroll
    for (int j = 0; j < kMaxE / 32; ++j) {
      const uint4 m = *reinterpret_cast<const uint4*>(S.mask[lane * (kMaxE / 32) + j]);
      const int n = __popc(m.x) + __popc(m.y) + __popc(m.z) + __popc(m.w);
      v[j] = (uint32_t)n | (n > 0 ? 0x10000u : 0u);
      sum += v[j];
    }
    uint32_t inc = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t u = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += u;
    }
    uint32_t at = inc - sum;
#pragma unroll
    for (int j = 0; j < kMaxE / 32; ++j) {
      const int e = lane * (kMaxE / 32) + j;
      L.off[e] = (int)(at & 0xffffu);
      if (v[j]) L.active[at >> 16] = (uint8_t)e;
      at += v[j];
    }
    if (lane == 31) {
      L.off[kMaxE] = (int)(at & 0xffffu);
      L.nact = (int)(at >> 16);
    }
  }
  __syncthreads();
  for (int s = tid; s < T * K; s += nt) {
    const int e = S.sel[s], t = s / K;
    int r = L.off[e];
    for (int w = 0; w < (t >> 5); ++w) r += __popc(S.mask[e][w]);
    r += __popc(S.mask[e][t >> 5] & ((1u << (t & 31)) - 1u));
    L.slot[r] = (uint16_t)s;
    L.tok[r] = (uint8_t)t;
  }
  __syncthreads();
}

__device__ __forceinline__ uint64_t timer_ns() {
  uint64_t t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
  return t;
}
__device__ __forceinline__ uint32_t ld_acquire(const uint32_t* p) {
  uint32_t v;
  asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
  return v;
}
__device__ __forceinline__ void red_release(uint32_t* p, uint32_t v) {
  asm volatile("red.release.gpu.global.add.u32 [%0], %1;" ::"l"(p), "r"(v) : "memory");
}
// Waits until *p reaches `target`; false (and the status bit) once the limit has passed.
__device__ __forceinline__ bool wait_count(const uint32_t* p, uint32_t target, uint32_t* err) {
  if (ld_acquire(p) >= target) return true;
  const uint64_t t0 = timer_ns();
  for (;;) {
    if (ld_acquire(p) >= target) return true;
    if (timer_ns() - t0 > kBarrierLimitNs) {
      set_error(err, kErrTimeout);
      return false;
    }
  }
}
// A barrier of the whole grid on a counter that was zero before the kernel.
// The launch is cooperative (all blocks resident); after an expired wait the
// block goes on, so that every block still arrives at every barrier.
__device__ __forceinline__ void grid_barrier(uint32_t* counter, uint32_t* err) {
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    red_release(counter, 1u);
    wait_count(counter, gridDim.x, err);
    __threadfence();
  }
  __syncthreads();
}

// bf16 keeps act as two terms up to 32 tokens: then y is rounded once, as from an
// fp32 act, where one term adds about 40 % to its error.  The second term's rows and
// products cost 2 to 5 % of the time (graph: 1 token 31.7 -> 32.8 us, 7 tokens
// 53.7 -> 54.8, 32 tokens of D = 2048, F = 1024, E = 64, K = 6 122.8 -> 129.4); above
// 32 tokens its rows would take stages from the ring, and more.
constexpr int kFewTerms(int T) { return T <= 32 ? 2 : 1; }

// bf16, up to kSplitT tokens: a product with few tiles has them cut along k into
// at most kSplitParts parts each, at most kSplitUnits in all (few_tc.cu).
constexpr int kSplitT = 8, kSplitParts = 4, kSplitUnits = 128;

struct Args {
  int T, D, E, K, F;
  const void* x;
  const void* w1;
  const void* w2;
  void* act;             // [T K, F] rows in expert-grouped order, storage type (bf16: kFewTerms of them)
  float* ypart;          // [T K, D] by slot, for each part of the second product's tiles
  float* hpart;          // bf16: parts of the first product's tiles, [kSplitUnits, kSplitT, 128]
  uint32_t* counters;    // zeroed by the router kernel
  const int32_t* topk_idx;
  const float* topk_prob;
  void* y;
  uint32_t* err;
};

// y[t] = sum_k p_tk ypart[t K + k] (of all its parts) in order of k, one rounding;
// the whole grid shares the T D / 4 groups of four columns.
template <typename TX, bool SPLIT>
__device__ __forceinline__ void combine_rows(const Args& a, int parts) {
  const int d4 = a.D >> 2;
  const int64_t part = (int64_t)a.T * a.K * d4;
  for (int i = blockIdx.x * blockDim.x + threadIdx.x; i < a.T * d4; i += gridDim.x * blockDim.x) {
    const int t = i / d4, c = i - t * d4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < a.K; k0 += 8) {  // eight rows' loads in flight, whatever K
      float p[8];
      float4 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int slot = t * a.K + k0 + j;
        const bool in = k0 + j < a.K;
        p[j] = in ? __ldg(a.topk_prob + slot) : 0.f;
        v[j] = in ? __ldcg(reinterpret_cast<const float4*>(a.ypart) + (int64_t)slot * d4 + c)
                  : make_float4(0.f, 0.f, 0.f, 0.f);
      }
      for (int u = 1; SPLIT && u < parts; ++u) {
        float4 w[8];
#pragma unroll
        for (int j = 0; j < 8; ++j)
          w[j] = k0 + j < a.K ? __ldcg(reinterpret_cast<const float4*>(a.ypart) + u * part +
                                       (int64_t)(t * a.K + k0 + j) * d4 + c)
                              : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int j = 0; j < 8; ++j)
          v[j] = make_float4(v[j].x + w[j].x, v[j].y + w[j].y, v[j].z + w[j].z, v[j].w + w[j].w);
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        s.x = fmaf(p[j], v[j].x, s.x);
        s.y = fmaf(p[j], v[j].y, s.y);
        s.z = fmaf(p[j], v[j].z, s.z);
        s.w = fmaf(p[j], v[j].w, s.w);
      }
    }
    if (sizeof(TX) == 4) {
      reinterpret_cast<float4*>(a.y)[i] = s;
    } else {
      __nv_bfloat162 lo = __floats2bfloat162_rn(s.x, s.y), hi = __floats2bfloat162_rn(s.z, s.w);
      reinterpret_cast<uint2*>(a.y)[i] =
          make_uint2(*reinterpret_cast<uint32_t*>(&lo), *reinterpret_cast<uint32_t*>(&hi));
    }
  }
}

cudaError_t launch_few_tc(const Ctx& c, const Args& a);  // bf16 (few_tc.cu)

}  // namespace few
}  // namespace moe
