// A whole routed MoE layer for at most 128 tokens (moe_few_tokens): generation
// with one or a few sequences, where reading the chosen experts' weights is
// the work and every launch and barrier counts.
//
// Two launches.  few_router chooses every token's experts (and zeroes the
// counters of the second launch's barriers).  few_layer (cooperative, one block
// per SM): every block builds the row lists for itself (few.cuh), then the grid
// computes act = silu(g) * u of every routed row and W2 act by slot, meets at a
// barrier and combines.  fp32 runs on the CUDA cores (here), with another barrier
// between the products; bf16 on the tensor cores, with a counter an expert there
// (few_tc.cu).
#include <algorithm>

#include "few.cuh"

namespace moe {
namespace few {
namespace {

constexpr int kTokens = 8;        // tokens that share one read of a weight row
constexpr int kRouterCtas = 8;    // blocks of a cluster: they share the experts, then take one token each
constexpr int kRouterThreads = 512;

// The sum over the warp's lanes of v[i] in lane i (32 / V) and its 32 / V - 1
// followers, for V values a lane.
template <int V>
__device__ __forceinline__ float transpose_sum(float (&v)[V], int lane) {
  int o = 16;
#pragma unroll
  for (int n = V / 2; n > 0; n >>= 1, o >>= 1) {
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const bool up = lane & o;
      const float keep = up ? v[j + n] : v[j], send = up ? v[j] : v[j + n];
      v[j] = keep + __shfl_xor_sync(0xffffffffu, send, o);
    }
  }
#pragma unroll
  for (; o > 0; o >>= 1) v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
  return v[0];
}

// acc[r * NT + i] += sum over this lane's k of w_r[k] x_i[k], for R rows of
// weights and NT of x.  Each lane takes every 32nd vector of 16 bytes.
template <typename T, int R, int NT, bool kWritten>  // kWritten: x was written by this kernel (no read-only path)
__device__ __forceinline__ void dot_rows(const uint4* const (&w)[R], const uint4* const (&x)[NT], int nvec, int lane,
                                         float (&acc)[R * NT]) {
  constexpr int NV = Vec<T>::N;
  // steps in flight: as many as 128 registers hold (graph times; 2 tokens of D = 1024,
  // F = 512, E = 64, K = 6: 27.0 us with two steps, 24.9 with four; 64 tokens of
  // D = F = 512, E = 32, K = 4: 46.3 with two, 44.3 with one)
  constexpr int kSteps = NT <= 2 ? 4 : NT == 4 ? 2 : 1;
#pragma unroll kSteps
  for (int v = lane; v < nvec; v += 32) {
    uint4 wr[R];
#pragma unroll
    for (int r = 0; r < R; ++r) wr[r] = ld_stream(w[r] + v);
    float wf[R][NV];
#pragma unroll
    for (int r = 0; r < R; ++r) unpack16<T>(wr[r], wf[r]);
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      float xf[NV];
      unpack16<T>(kWritten ? __ldcg(x[i] + v) : __ldg(x[i] + v), xf);
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int j = 0; j < NV; ++j) acc[r * NT + i] = fmaf(wf[r][j], xf[j], acc[r * NT + i]);
      }
    }
  }
}

__device__ __forceinline__ void st_cluster_f32(float* p, uint32_t rank, float v) {
  uint32_t a = static_cast<uint32_t>(__cvta_generic_to_shared(p)), r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(rank));
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(r), "f"(v) : "memory");
}

constexpr int kRouterWarps = kRouterThreads / 32;
constexpr int kRouterRows = kMaxE / kRouterCtas;  // experts of a block, at most

__device__ __forceinline__ void mma16816(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                         uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// part[row][split][token] = the partial logits of this block's `rows` experts
// (weights from w on) and the group's n tokens, k in windows dealt to `splits`
// warps; returns splits.  Rows and tokens past the last read the last one's
// data; their sums are not used.
//
// bf16: mma.sync m16n8k16, 16 experts by 8 tokens a warp (the work is a few
// MFLOP; what counts is that a warp needs three 16-byte loads for 32 k of all
// of them).  Lane (g, q) loads k = 32 j + 8 q .. + 7 of expert rows g and g + 8
// and of token g: its words 0, 1 and 2, 3 are the fragments of two products
// over 16 of those 32 k each, in the same order for both operands.
__device__ __forceinline__ int router_parts(const bf16* w, const bf16* x, int rows, int n, int Din, int warp, int lane,
                                            float (*part)[kRouterWarps][kTokens]) {
  const int tiles = (rows + 15) / 16, splits = kRouterWarps / tiles;
  if (warp < tiles * splits) {
    const int tile = warp / splits, split = warp % splits;
    const int g = lane >> 2, q = lane & 3;
    const uint4* a0 = reinterpret_cast<const uint4*>(w + (int64_t)min(tile * 16 + g, rows - 1) * Din) + q;
    const uint4* a1 = reinterpret_cast<const uint4*>(w + (int64_t)min(tile * 16 + g + 8, rows - 1) * Din) + q;
    const uint4* b = reinterpret_cast<const uint4*>(x + (int64_t)min(g, n - 1) * Din) + q;
    float c[4] = {0.f, 0.f, 0.f, 0.f};
    // eight windows' loads in flight, whatever their number
    constexpr int kBatch = 8;
    for (int j0 = split; j0 < Din / 32; j0 += kBatch * splits) {
      uint4 u[kBatch], v[kBatch], t[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        const int j = j0 + i * splits;
        u[i] = v[i] = t[i] = make_uint4(0, 0, 0, 0);
        if (j < Din / 32) {
          u[i] = ld_keep(a0 + 4 * j);
          v[i] = ld_keep(a1 + 4 * j);
          t[i] = ld_keep(b + 4 * j);
        }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        mma16816(c, u[i].x, v[i].x, u[i].y, v[i].y, t[i].x, t[i].y);
        mma16816(c, u[i].z, v[i].z, u[i].w, v[i].w, t[i].z, t[i].w);
      }
    }
    float* p = part[tile * 16 + g][split] + 2 * q;
    *reinterpret_cast<float2*>(p) = make_float2(c[0], c[1]);
    p = part[tile * 16 + g + 8][split] + 2 * q;
    *reinterpret_cast<float2*>(p) = make_float2(c[2], c[3]);
  }
  return splits;
}

// fp32: one expert by up to 8 tokens a warp, lanes along k.
__device__ __forceinline__ int router_parts(const float* w, const float* x, int rows, int n, int Din, int warp,
                                            int lane, float (*part)[kRouterWarps][kTokens]) {
  const int splits = rows > 8 ? 1 : rows > 4 ? 2 : rows > 2 ? 4 : 8;
  const int nvec = Din / 4, split = warp % splits;
  for (int r = warp / splits; r < rows; r += kRouterWarps / splits) {
    const float4* wr = reinterpret_cast<const float4*>(w + (int64_t)r * Din);
    float acc[kTokens];
#pragma unroll
    for (int i = 0; i < kTokens; ++i) acc[i] = 0.f;
#pragma unroll 2
    for (int v = split * 32 + lane; v < nvec; v += 32 * splits) {
      const float4 a = __ldg(wr + v);
#pragma unroll
      for (int i = 0; i < kTokens; ++i) {
        if (i < n) {
          const float4 b = __ldg(reinterpret_cast<const float4*>(x + (int64_t)i * Din) + v);
          acc[i] = fmaf(a.x, b.x, fmaf(a.y, b.y, fmaf(a.z, b.z, fmaf(a.w, b.w, acc[i]))));
        }
      }
    }
    const float z = transpose_sum<kTokens>(acc, lane);
    if (lane % 4 == 0) part[r][split][lane / 4] = z;
  }
  return splits;
}

// The router: a cluster of eight blocks takes eight tokens.  Each block forms
// its eighth of the experts' logits for all of them and sends every token's to
// the block that chooses for it, which ranks the E keys by counting the better
// ones (larger, or equal with a lower index) and forms the probabilities as
// moe_topk (softmax) and moe_topk_sigmoid (sigmoid) form them.  Bound by
// latency: one read of W_r's rows, one cluster barrier, the counting (one token
// of D = 2048, E = 128: 4.9 us, 2.8 of them for cold rows; 2.6 us warm).
template <typename T>
__global__ void __cluster_dims__(kRouterCtas, 1, 1) __launch_bounds__(kRouterThreads)
    few_router_kernel(const T* __restrict__ x, const T* __restrict__ w, const float* __restrict__ bias, int router,
                      int Tn, int E, int K, int Din, int32_t* __restrict__ topk_idx, float* __restrict__ topk_prob,
                      uint32_t* __restrict__ counters) {
  __shared__ float logit[kMaxE];
  __shared__ alignas(16) uint32_t key[kMaxE];
  __shared__ int better[kMaxE];
  __shared__ float score[kMaxK];
  __shared__ float part[kRouterRows][kRouterWarps][kTokens];
  // Bring this block's rows of W_r into L2 while the kernels before this one
  // end (no value is read yet): cold, their latency is most of this kernel.
  const int per = (E + kRouterCtas - 1) / kRouterCtas;
  const int e0 = (int)(blockIdx.x % kRouterCtas) * per, rows = max(0, min(per, E - e0));
  {
    const char* wb = reinterpret_cast<const char*>(w + (int64_t)e0 * Din);
    for (int i = threadIdx.x * 128; i < rows * Din * (int)sizeof(T); i += kRouterThreads * 128)
      asm volatile("prefetch.global.L2 [%0];" ::"l"(wb + i));
  }
  grid_dependency_wait();  // what came before has written x
  if (blockIdx.x == 0)
    for (int i = threadIdx.x; i < kFewCounters; i += kRouterThreads) counters[i] = 0u;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = blockIdx.x % kRouterCtas, t0 = (int)blockIdx.x / kRouterCtas * kTokens;
  const int n = min(kTokens, Tn - t0);
  const float my_bias = bias && tid < E ? __ldg(bias + tid) : 0.f;  // its latency under the products'
  for (int i = tid; i < kMaxE; i += kRouterThreads) better[i] = 0;
  // no block writes into another's shared memory before all of them run
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  int splits = 0;
  if (rows > 0)
    splits = router_parts(w + (int64_t)e0 * Din, x + (int64_t)t0 * Din, rows, n, Din, warp, lane, part);
  __syncthreads();
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
  if (tid < rows * kTokens) {
    const int r = tid / kTokens, i = tid % kTokens;
    float z = part[r][0][i];
    for (int s = 1; s < splits; ++s) z += part[r][s][i];
    if (i < n) st_cluster_f32(logit + e0 + r, (uint32_t)i, z);
  }
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  if (rank >= n) return;
  if (tid < kMaxE) {
    uint32_t k = 0u;  // below every key
    if (tid < E) {
      float v = logit[tid];
      if (router == MOE_ROUTER_SIGMOID) v = sigmoid_rn(v);
      k = order_bits(bias ? __fadd_rn(v, my_bias) : v);
    }
    key[tid] = k;
  }
  __syncthreads();
  // thread (e, part of the keys): the better ones among them
  {
    const int pe = E <= 128 ? 128 : 256, parts = kRouterThreads / pe;
    const int e = tid % pe, len = pe / parts, j0 = tid / pe * len;
    // a key from a lower expert is better already when it is equal
    const uint32_t mine = key[e], low = mine - 1u;
    int c = 0;
#pragma unroll 8
    for (int j = j0; j < j0 + len; j += 4) {
      const uint4 o = *reinterpret_cast<const uint4*>(key + j);
      c += (o.x > (j < e ? low : mine)) + (o.y > (j + 1 < e ? low : mine)) + (o.z > (j + 2 < e ? low : mine)) +
           (o.w > (j + 3 < e ? low : mine));
    }
    atomicAdd(&better[e], c);
  }
  __syncthreads();
  const int t = t0 + rank;
  if (tid < E && better[tid] < K) {
    topk_idx[t * K + better[tid]] = tid;
    score[better[tid]] = router == MOE_ROUTER_SIGMOID ? sigmoid_rn(logit[tid]) : order_value(key[tid]);
  }
  __syncthreads();
  if (warp == 0) {
    float v = 0.f;
    if (lane < K) v = router == MOE_ROUTER_SIGMOID ? score[lane] : expf(score[lane] - score[0]);
    float sum = 0.f;
    for (int k = 0; k < K; ++k) sum += __shfl_sync(0xffffffffu, v, k);
    if (lane < K) topk_prob[t * K + lane] = router == MOE_ROUTER_SIGMOID ? v * __frcp_rn(sum) : v * (1.0f / sum);
  }
}

template <typename T>
cudaError_t launch_router(const Ctx& c, const void* x, const void* w, const float* bias, int router, int Tn, int E,
                          int K, int Din, int32_t* topk_idx, float* topk_prob, uint32_t* counters) {
  KernelScope ks("few_router", c.stream);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((Tn + kTokens - 1) / kTokens * kRouterCtas, 1, 1);
  cfg.blockDim = dim3(kRouterThreads, 1, 1);
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, few_router_kernel<T>, (const T*)x, (const T*)w, bias, router, Tn, E, K, Din,
                            topk_idx, topk_prob, counters);
}

constexpr int kSimtThreads = 512;

// act of NT of an expert's rows from r0 on (n <= NT exist), features f and f + 1.
template <typename T, int NT>
__device__ __forceinline__ void first_unit(const Args& a, const Lists& L, const uint4* w, int r0, int n, int f,
                                           int lane) {
  const int nvec = a.D / Vec<T>::N;
  const uint4* const wr[4] = {w, w + nvec, w + 64 * (int64_t)nvec, w + 65 * (int64_t)nvec};
  const uint4* xr[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i)
    xr[i] = static_cast<const uint4*>(a.x) + (int64_t)L.tok[r0 + min(i, n - 1)] * nvec;
  float acc[4 * NT];
#pragma unroll
  for (int i = 0; i < 4 * NT; ++i) acc[i] = 0.f;
  dot_rows<T, 4, NT, false>(wr, xr, nvec, lane, acc);
  const float h = transpose_sum<4 * NT>(acc, lane);
  const float up = __shfl_down_sync(0xffffffffu, h, 16);
  const int j = lane / (32 / (4 * NT)), i = j % NT;
  if (lane < 16 && lane % (32 / (4 * NT)) == 0 && i < n)
    static_cast<T*>(a.act)[(int64_t)(r0 + i) * a.F + f + j / NT] = from_f32<T>(h * sigmoid_rn(h) * up);
}

// W2 act of the same rows, output columns d .. d + 3.
template <typename T, int NT>
__device__ __forceinline__ void second_unit(const Args& a, const Lists& L, const uint4* w, int r0, int n, int d,
                                            int lane) {
  const int nvec = a.F / Vec<T>::N;
  const uint4* const wr[4] = {w, w + nvec, w + 2 * nvec, w + 3 * nvec};
  const uint4* xr[NT];
#pragma unroll
  for (int i = 0; i < NT; ++i) xr[i] = static_cast<const uint4*>(a.act) + (int64_t)(r0 + min(i, n - 1)) * nvec;
  float acc[4 * NT];
#pragma unroll
  for (int i = 0; i < 4 * NT; ++i) acc[i] = 0.f;
  dot_rows<T, 4, NT, true>(wr, xr, nvec, lane, acc);
  const float s = transpose_sum<4 * NT>(acc, lane);
  const int j = lane / (32 / (4 * NT)), i = j % NT;
  if (lane % (32 / (4 * NT)) == 0 && i < n) a.ypart[(int64_t)L.slot[r0 + i] * a.D + d + j / NT] = s;
}

// The experts on the CUDA cores (fp32): a warp takes four weight rows of one
// expert (GEMM-1: the gate and up rows of two features; GEMM-2: four output
// columns) and up to eight of its tokens at a time, lanes along k, sums by a
// transposing shuffle reduction.  Bound by reading the weights: 13 tokens of
// D = F = 512, E = 64, K = 6 take 36.4 us as a graph, W1 at 6.2 and W2 at 6.4 TB/s,
// the rest the router, two barriers and the combine.  The rows of weights are
// split over warps and not over blocks, so every warp has loads of its own in
// flight; 16 warps an SM (24 spill, 39.4 us; 12: 37.6).  Experts with more than
// eight tokens have their rows walked again for every eight of them.
template <typename T>
__global__ void __launch_bounds__(kSimtThreads, 1) few_layer_kernel(const __grid_constant__ Args a) {
  constexpr int NV = Vec<T>::N;
  __shared__ Lists L;
  __shared__ ListScratch scratch;
  build_lists(L, scratch, a.topk_idx, a.T, a.K);
  const int lane = threadIdx.x & 31;
  const int wid = (threadIdx.x >> 5) * gridDim.x + blockIdx.x;  // neighbouring units on different SMs
  const int nw = gridDim.x * (kSimtThreads / 32);
  const int F = a.F, D = a.D;
  {
    const int per = F / 2, nvec = D / NV;
    for (int u = wid; u < L.nact * per; u += nw) {
      const int e = L.active[u / per], f = (u % per) * 2;
      const uint4* w = static_cast<const uint4*>(a.w1) + ((int64_t)e * 2 * F + (f / 64) * 128 + f % 64) * nvec;
      for (int r0 = L.off[e]; r0 < L.off[e + 1]; r0 += kTokens) {
        const int n = min(kTokens, L.off[e + 1] - r0);
        if (n == 1) first_unit<T, 1>(a, L, w, r0, n, f, lane);
        else if (n == 2) first_unit<T, 2>(a, L, w, r0, n, f, lane);
        else if (n <= 4) first_unit<T, 4>(a, L, w, r0, n, f, lane);
        else first_unit<T, 8>(a, L, w, r0, n, f, lane);
      }
    }
  }
  {
    // the rows of this warp's first unit of the second product come into L2
    // while the grid meets
    const int per = D / 4;
    if (wid < L.nact * per) {
      const char* w = reinterpret_cast<const char*>(
          static_cast<const T*>(a.w2) + ((int64_t)L.active[wid / per] * D + wid % per * 4) * F);
      for (int i = lane * 128; i < 4 * F * (int)sizeof(T); i += 32 * 128)
        asm volatile("prefetch.global.L2 [%0];" ::"l"(w + i));
    }
  }
  grid_barrier(a.counters, a.err);
  {
    const int per = D / 4, nvec = F / NV;
    for (int u = wid; u < L.nact * per; u += nw) {
      const int e = L.active[u / per], d = (u % per) * 4;
      const uint4* w = static_cast<const uint4*>(a.w2) + ((int64_t)e * D + d) * nvec;
      for (int r0 = L.off[e]; r0 < L.off[e + 1]; r0 += kTokens) {
        const int n = min(kTokens, L.off[e + 1] - r0);
        if (n == 1) second_unit<T, 1>(a, L, w, r0, n, d, lane);
        else if (n == 2) second_unit<T, 2>(a, L, w, r0, n, d, lane);
        else if (n <= 4) second_unit<T, 4>(a, L, w, r0, n, d, lane);
        else second_unit<T, 8>(a, L, w, r0, n, d, lane);
      }
    }
  }
  grid_barrier(a.counters + 1, a.err);
  grid_dependency_launch();
  combine_rows<T, false>(a, 1);
}

cudaError_t launch_few_simt(const Ctx& c, const Args& a) {
  const int64_t units = (int64_t)std::min(a.E, a.T * a.K) * (a.F / 2);
  const int grid = (int)std::min<int64_t>(c.num_sms, (units + kSimtThreads / 32 - 1) / (kSimtThreads / 32));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid, 1, 1);
  cfg.blockDim = dim3(kSimtThreads, 1, 1);
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  KernelScope ks("few_layer_simt", c.stream);
  return cudaLaunchKernelEx(&cfg, few_layer_kernel<float>, a);
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

// counters, act, ypart, hpart.  bf16 has room for two terms of act and, up to
// kSplitT tokens, for the tiles' parts, used or not: sizes grow with T, so one
// workspace serves every smaller call.
struct Carve {
  size_t act, ypart, hpart, total;
};
Carve carve(const ShapeInfo& d) {
  Carve w;
  const bool tc = d.dt == DType::BF16;
  const size_t few = std::min<size_t>(d.T, kSplitT);
  const size_t slots = tc ? std::max<size_t>(d.TK, kSplitParts * few * d.K) : d.TK;
  w.act = up256(kFewCounters * sizeof(uint32_t));
  w.ypart = w.act + up256((tc ? 2 : 1) * d.TK * d.F * d.bx);
  w.hpart = w.ypart + up256(slots * d.D * 4);
  w.total = w.hpart + (tc ? (size_t)kSplitUnits * kSplitT * 128 * 4 : 0);
  return w;
}

int check(const moe_shape_t* shape, ShapeInfo* d) {
  const int st = abi_check_shape(shape, d);
  if (st != MOE_OK) return st;
  return d->T > kFewT ? MOE_ERR_TOO_LARGE : MOE_OK;
}

}  // namespace

}  // namespace few
}  // namespace moe

using namespace moe;

extern "C" int moe_few_workspace_size(const moe_shape_t* shape, size_t* bytes) {
  ShapeInfo d;
  const int st = few::check(shape, &d);
  if (st != MOE_OK) return st;
  if (!bytes) return MOE_ERR_NULL;
  *bytes = few::carve(d).total;
  return MOE_OK;
}

extern "C" int moe_few_tokens(const moe_shape_t* shape, int32_t router, const void* x, const void* x_router,
                              const void* w_router, const float* bias, const void* w1, const void* w2,
                              int32_t* topk_idx, float* topk_prob, void* y, void* ws, size_t ws_bytes,
                              void* stream) {
  ShapeInfo d;
  int st = few::check(shape, &d);
  if (st != MOE_OK) return st;
  if (router != MOE_ROUTER_SOFTMAX && router != MOE_ROUTER_SIGMOID) return MOE_ERR_UNSUPPORTED;
  if (!x_router && !d.H) x_router = x;
  const void* need[] = {x, x_router, w_router, w1, w2, topk_idx, topk_prob, y, ws};
  for (const void* p : need)
    if (!p) return MOE_ERR_NULL;
  for (const void* p : need)
    if ((uintptr_t)p & 15u) return MOE_ERR_ALIGN;
  if ((uintptr_t)bias & 15u) return MOE_ERR_ALIGN;
  const few::Carve w = few::carve(d);
  if (ws_bytes < w.total) return MOE_ERR_WORKSPACE;
  Ctx c;
  st = abi_device_ctx(stream, &c);
  if (st != MOE_OK) return st;
  char* base = static_cast<char*>(ws);
  few::Args a;
  a.T = (int)d.T;
  a.D = d.D;
  a.E = d.E;
  a.K = d.K;
  a.F = d.F;
  a.x = x;
  a.w1 = w1;
  a.w2 = w2;
  a.act = base + w.act;
  a.ypart = reinterpret_cast<float*>(base + w.ypart);
  a.hpart = reinterpret_cast<float*>(base + w.hpart);
  a.counters = reinterpret_cast<uint32_t*>(base);
  a.topk_idx = topk_idx;
  a.topk_prob = topk_prob;
  a.y = y;
  a.err = c.err;
  auto launch = d.dt == DType::BF16 ? few::launch_router<bf16> : few::launch_router<float>;
  st = abi_cuda_status(
      launch(c, x_router, w_router, bias, router, a.T, a.E, a.K, d.Din, topk_idx, topk_prob, a.counters));
  if (st != MOE_OK) return st;
  return abi_cuda_status(d.dt == DType::BF16 ? few::launch_few_tc(c, a) : few::launch_few_simt(c, a));
}
