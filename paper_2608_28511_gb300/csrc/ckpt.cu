// 8-bit activation checkpoints (ckpt.cuh): the streaming kernels that write and
// read one, and the expert FFN that keeps nothing else between its forward and
// its backward pass.
#include <algorithm>

#include "ckpt.cuh"
#include "launch.h"

namespace moe {
namespace ckpt {
namespace {

constexpr int kTileRows = 32;
constexpr int kTileCols = 256;
constexpr int kTileBlocks = kTileCols / kBlock;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// 32 bytes of x; WIDE: in one load (x and its row pitch are multiples of 32 bytes).
template <bool WIDE>
__device__ __forceinline__ void load32(const void* p, uint32_t (&w)[8]) {
  if (WIDE) {
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p));
  } else {
    const uint4 a = ld_stream(static_cast<const uint4*>(p)), b = ld_stream(static_cast<const uint4*>(p) + 1);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  }
}
// The values of 32 bytes, and the largest magnitude's bits (fp32).
__device__ __forceinline__ uint32_t unpack32(const uint32_t (&w)[8], float (&f)[16]) {  // bf16
  uint32_t m = 0;  // two 16-bit magnitudes, ordered as unsigned integers
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[2 * i] = __uint_as_float(w[i] << 16);
    f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    m = __vmaxu2(m, w[i] & 0x7fff7fffu);
  }
  return max(m << 16, m & 0xffff0000u);
}
__device__ __forceinline__ uint32_t unpack32(const uint32_t (&w)[8], float (&f)[8]) {  // fp32
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    f[i] = __uint_as_float(w[i]);
    m = max(m, mag_bits(f[i]));
  }
  return m;
}

// A block takes 32 rows by 1 KB: a lane reads 32 bytes of a row (four rows'
// loads in flight), the two (bf16) or four lanes of a 32-column block share its
// maximum by shuffles, and the tile's scales go through shared memory so that
// they are written as lines of scale [cols / 32][rows].  HBM has b + 1.125 bytes
// an element to move, and a warp can spend about 9 instructions on one before
// it falls behind; half of a lane's go to the scale and its inverse, so a lane
// takes 16 bf16 elements (with 8: 15 instructions an element, 0.78 issued a
// cycle, 76 us for [65536, 2048]; now 66).
template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads) ckpt_pack_kernel(const T* __restrict__ x, int64_t ldx, int64_t rows,
                                                             int64_t cols, int tiles_c, uint8_t* __restrict__ codes,
                                                             float* __restrict__ scale) {
  constexpr int NV = 32 / sizeof(T);  // elements of a lane
  constexpr int NL = kBlock / NV;     // lanes of a 32-column block
  constexpr int NR = kTileRows / kWarps;
  constexpr int NB = 32 / NL;         // 32-column blocks of a tile
  __shared__ float s[NB][kTileRows + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * kTileRows + warp * NR;
  const int64_t c0 = (int64_t)(blockIdx.x % tiles_c) * (32 * NV), c = c0 + lane * NV;
  uint32_t w[NR][8];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    if (r0 + i < rows && c < cols) {
      load32<WIDE>(x + (r0 + i) * ldx + c, w[i]);
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) w[i][j] = 0u;
    }
  }
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    float f[NV];
    uint32_t m = unpack32(w[i], f);
#pragma unroll
    for (int o = 1; o < NL; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    const Scale sc = block_scale(m);
    if (lane % NL == 0) s[lane / NL][warp * NR + i] = sc.scale;
    if (r0 + i < rows && c < cols) {
      uint32_t q[NV / 4];
#pragma unroll
      for (int j = 0; j < NV / 4; ++j) q[j] = codes4(f[4 * j], f[4 * j + 1], f[4 * j + 2], f[4 * j + 3], sc.inv);
      uint8_t* out = codes + (r0 + i) * cols + c;
      if (NV == 16) __stcs(reinterpret_cast<uint4*>(out), make_uint4(q[0], q[1], q[NV / 4 - 2], q[NV / 4 - 1]));
      else __stcs(reinterpret_cast<uint2*>(out), make_uint2(q[0], q[1]));
    }
  }
  __syncthreads();
  const int64_t r = (int64_t)(blockIdx.x / tiles_c) * kTileRows + lane;
  for (int j = warp; j < NB; j += kWarps) {
    const int64_t blk = c0 / kBlock + j;
    if (blk < cols / kBlock && r < rows) scale[blk * rows + r] = s[j][lane];
  }
}

template <typename T>
void launch_pack(const Ctx& c, const void* x, int64_t ldx, int64_t rows, int64_t cols, uint8_t* codes, float* scale) {
  const int64_t tile = 1024 / sizeof(T), tc = (cols + tile - 1) / tile;
  const unsigned grid = (unsigned)(tc * ((rows + kTileRows - 1) / kTileRows));
  const bool wide = ((uintptr_t)x | (uintptr_t)(ldx * sizeof(T))) % 32 == 0;
  auto k = wide ? ckpt_pack_kernel<T, true> : ckpt_pack_kernel<T, false>;
  k<<<grid, kThreads, 0, c.stream>>>(static_cast<const T*>(x), ldx, rows, cols, (int)tc, codes, scale);
}

// The other way, a tile of 32 rows by 256 columns.  Bound by HBM: [65536, 2048] to
// bf16 62 us, 6.8 TB/s.
template <typename T>
__global__ void __launch_bounds__(kThreads) ckpt_unpack_kernel(const uint8_t* __restrict__ codes,
                                                               const float* __restrict__ scale, int64_t rows,
                                                               int64_t cols, int tiles_c, T* __restrict__ x,
                                                               int64_t ldx) {
  constexpr int NV = Vec<T>::N;
  constexpr int NL = kBlock / NV;
  constexpr int NC = kTileCols / (32 * NV);
  constexpr int NR = kTileRows / kWarps;
  __shared__ float s[kTileBlocks][kTileRows + 1];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t r0 = (int64_t)(blockIdx.x / tiles_c) * kTileRows, c0 = (int64_t)(blockIdx.x % tiles_c) * kTileCols;
  uint2 v[NR][NC];
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int64_t r = r0 + warp * NR + i;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int64_t c = c0 + (j * 32 + lane) * NV;
      v[i][j] = make_uint2(0, 0);
      if (r < rows && c < cols) {
        const uint8_t* in = codes + r * cols + c;
        if (NV == 8) v[i][j] = __ldcs(reinterpret_cast<const uint2*>(in));
        else v[i][j].x = __ldcs(reinterpret_cast<const uint32_t*>(in));
      }
    }
  }
  const int64_t blk = c0 / kBlock + warp;
  s[warp][lane] = blk < cols / kBlock && r0 + lane < rows ? __ldcs(scale + blk * rows + r0 + lane) : 0.f;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < NR; ++i) {
    const int64_t r = r0 + warp * NR + i;
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int64_t c = c0 + (j * 32 + lane) * NV;
      const float sc = s[(j * 32 + lane) / NL][warp * NR + i];
      float f[8];
      values4(v[i][j].x, sc, f);
      if (NV == 8) values4(v[i][j].y, sc, f + 4);
      if (r < rows && c < cols) st_stream(reinterpret_cast<uint4*>(x + r * ldx + c), pack16<T>(f));
    }
  }
}

// dprob[r] = sum over j of part[j][r], in order: the GEMM's warps leave one
// partial a row for every 128 columns of dA.  4.7 us for 49152 rows of 8 (latency).
__global__ void __launch_bounds__(256) ckpt_dprob_kernel(const float* __restrict__ part, int n, int64_t rows,
                                                         float* __restrict__ dprob) {
  grid_dependency_wait();
  grid_dependency_launch();
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r >= rows) return;
  float s = 0.f;
#pragma unroll 8
  for (int j = 0; j < n; ++j) s += __ldcs(part + j * rows + r);
  dprob[r] = s;
}

// The tensor maps in the workspace want 128-byte alignment, callers owe 16: the
// carve-up starts at the next multiple of 256, and the size leaves room for that.
constexpr size_t kWsAlign = 256;
size_t up256(size_t v) { return (v + kWsAlign - 1) & ~(kWsAlign - 1); }
char* ws_base(void* ws) { return reinterpret_cast<char*>(up256(reinterpret_cast<uintptr_t>(ws))); }

// act of the forward pass; and the backward pass's rows of dy and x, dH, p act,
// partial dprob sums and the two weight gradients' tensor maps.
struct Carve {
  size_t act_f, dy, x, dh, act, part, maps0, maps1, total;
  int parts;
};
Carve carve(const ShapeInfo& d) {
  Carve w;
  const size_t n = (size_t)d.TK;
  w.parts = 2 * ((d.F + 255) / 256);
  w.act_f = 0;
  w.dy = 0;
  w.x = w.dy + up256(n * d.D * 2);
  w.dh = w.x + up256(n * d.D * 2);
  w.act = w.dh + up256(n * 2 * d.F * 2);
  w.part = w.act + up256(n * d.F * 2);
  w.maps0 = w.part + up256(n * w.parts * 4);
  w.maps1 = w.maps0 + up256(gemm_tc_group_scratch_bytes(d.E));
  w.total = w.maps1 + up256(gemm_tc_group_scratch_bytes(d.E)) + kWsAlign - 1;
  return w;
}

int check_rows(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, const void* codes,
               const void* scale, int64_t* tiles) {
  if (dtype != MOE_BF16 && dtype != MOE_F32) return MOE_ERR_DTYPE;
  const int64_t vec = dtype == MOE_BF16 ? 8 : 4;
  const int64_t most = int64_t(1) << 40;
  if (rows <= 0 || cols <= 0 || cols % kBlock || ldx < cols || rows > most || cols > most || ldx > most)
    return MOE_ERR_SHAPE;
  const int64_t tc = (cols + kTileCols - 1) / kTileCols, tr = (rows + kTileRows - 1) / kTileRows;
  if (tc > INT32_MAX / tr) return MOE_ERR_SHAPE;  // one block a tile
  if (!x || !codes || !scale) return MOE_ERR_NULL;
  for (const void* p : {x, codes, scale})
    if ((uintptr_t)p & 15u) return MOE_ERR_ALIGN;
  if (ldx % vec) return MOE_ERR_ALIGN;
  *tiles = tc * tr;
  return MOE_OK;
}

int check_ffn(const moe_shape_t* shape, ShapeInfo* d) {
  const int st = abi_check_shape(shape, d);
  if (st != MOE_OK) return st;
  return d->dt == DType::BF16 ? MOE_OK : MOE_ERR_UNSUPPORTED;
}

int check_pointers(std::initializer_list<const void*> need) {
  for (const void* p : need)
    if (!p) return MOE_ERR_NULL;
  for (const void* p : need)
    if ((uintptr_t)p & 15u) return MOE_ERR_ALIGN;
  return MOE_OK;
}

// C(m, n) = sum_k A(m, k) B(n, k) over each expert's rows m, A K-major.
GemmDesc by_rows(Epi epi, const ShapeInfo& d, const int32_t* offsets, const void* A, int64_t K, const void* B,
                 int64_t N, bool b_mn, void* C, int64_t ldc) {
  GemmDesc g;
  g.group = Group::M;
  g.epi = epi;
  g.N = N;
  g.K = K;
  g.num_groups = d.E;
  g.offsets = offsets;
  g.max_rows = d.TK;
  g.A = A;
  g.sa_m = K;
  g.sa_k = 1;
  g.B = B;
  g.sb_n = b_mn ? 1 : K;
  g.sb_k = b_mn ? N : 1;
  g.sb_g = N * K;
  g.C = C;
  g.ldc = ldc;
  return g;
}

// C_e(m, n) = sum over expert e's rows r of A(r, m) B(r, n).
GemmDesc weight_grad(const ShapeInfo& d, const int32_t* offsets, const void* A, int64_t M, const void* B, int64_t N,
                     void* C, DType ct, void* maps) {
  GemmDesc g;
  g.group = Group::K;
  g.M = M;
  g.N = N;
  g.num_groups = d.E;
  g.offsets = offsets;
  g.max_rows = d.TK;
  g.A = A;
  g.sa_m = 1;
  g.sa_k = M;
  g.B = B;
  g.sb_n = 1;
  g.sb_k = N;
  g.scratch = maps;
  g.C = C;
  g.c_type = ct;
  g.ldc = N;
  g.sc_g = M * N;
  return g;
}

}  // namespace
}  // namespace ckpt
}  // namespace moe

using namespace moe;

#define CKPT_TRY(expr)             \
  do {                             \
    const int st_ = (expr);        \
    if (st_ != MOE_OK) return st_; \
  } while (0)

extern "C" int moe_ckpt_pack(int32_t dtype, int64_t rows, int64_t cols, const void* x, int64_t ldx, int8_t* codes,
                             float* scale, void* stream) {
  int64_t tiles;
  CKPT_TRY(ckpt::check_rows(dtype, rows, cols, x, ldx, codes, scale, &tiles));
  Ctx c;
  CKPT_TRY(abi_device_ctx(stream, &c));
  KernelScope ks("ckpt_pack", c.stream);
  (dtype == MOE_BF16 ? ckpt::launch_pack<bf16> : ckpt::launch_pack<float>)(c, x, ldx, rows, cols,
                                                                           reinterpret_cast<uint8_t*>(codes), scale);
  return abi_cuda_status(cudaGetLastError());
}

extern "C" int moe_ckpt_unpack(int32_t dtype, int64_t rows, int64_t cols, const int8_t* codes, const float* scale,
                               void* x, int64_t ldx, void* stream) {
  int64_t tiles;
  CKPT_TRY(ckpt::check_rows(dtype, rows, cols, x, ldx, codes, scale, &tiles));
  Ctx c;
  CKPT_TRY(abi_device_ctx(stream, &c));
  const int tc = (int)((cols + ckpt::kTileCols - 1) / ckpt::kTileCols);
  const uint8_t* q = reinterpret_cast<const uint8_t*>(codes);
  KernelScope ks("ckpt_unpack", c.stream);
  if (dtype == MOE_BF16)
    ckpt::ckpt_unpack_kernel<bf16><<<(unsigned)tiles, ckpt::kThreads, 0, c.stream>>>(q, scale, rows, cols, tc,
                                                                                    (bf16*)x, ldx);
  else
    ckpt::ckpt_unpack_kernel<float><<<(unsigned)tiles, ckpt::kThreads, 0, c.stream>>>(q, scale, rows, cols, tc,
                                                                                     (float*)x, ldx);
  return abi_cuda_status(cudaGetLastError());
}

extern "C" int moe_ckpt_workspace_size(const moe_shape_t* shape, size_t* bytes) {
  ShapeInfo d;
  CKPT_TRY(ckpt::check_ffn(shape, &d));
  if (!bytes) return MOE_ERR_NULL;
  *bytes = ckpt::carve(d).total;
  return MOE_OK;
}

extern "C" int moe_expert_ffn_ckpt(const moe_shape_t* shape, const void* x_perm, const int32_t* expert_offsets,
                                   const void* w1, const void* w2, int8_t* h_q, float* h_scale, void* y_perm,
                                   void* ws, size_t ws_bytes, void* stream) {
  ShapeInfo d;
  CKPT_TRY(ckpt::check_ffn(shape, &d));
  CKPT_TRY(ckpt::check_pointers({x_perm, expert_offsets, w1, w2, h_q, h_scale, y_perm, ws}));
  const ckpt::Carve w = ckpt::carve(d);
  if (ws_bytes < w.total) return MOE_ERR_WORKSPACE;
  Ctx c;
  CKPT_TRY(abi_device_ctx(stream, &c));
  void* act = ckpt::ws_base(ws) + w.act_f;
  // GEMM-1, its epilogue: act = silu(g) u and the codes and scales of h, which
  // is never written in 16 bits
  GemmDesc g1 = ckpt::by_rows(Epi::SwigluFwdQ8, d, expert_offsets, x_perm, d.D, w1, 2 * (int64_t)d.F, false, h_q,
                              2 * (int64_t)d.F);
  g1.aux = act;
  g1.qscale = h_scale;
  CKPT_TRY(abi_cuda_status(launch_gemm_tc(c, g1, "ffn1_swiglu_q8_tc")));
  const GemmDesc g2 = ckpt::by_rows(Epi::Store, d, expert_offsets, act, d.F, w2, d.D, false, y_perm, d.D);
  return abi_cuda_status(launch_gemm_tc(c, g2, "ffn2_tc"));
}

extern "C" int moe_expert_ffn_bwd_ckpt(const moe_shape_t* shape, const void* dy, const void* x, const float* prob_perm,
                                       const int32_t* row_of_slot, const int32_t* expert_offsets, const int8_t* h_q,
                                       const float* h_scale, const void* w1, const void* w2, void* dx_perm,
                                       int32_t dw_dtype, void* dw1, void* dw2, float* dprob_perm, void* ws,
                                       size_t ws_bytes, void* stream) {
  ShapeInfo d;
  CKPT_TRY(ckpt::check_ffn(shape, &d));
  if (dw_dtype != MOE_BF16 && dw_dtype != MOE_F32) return MOE_ERR_DTYPE;
  CKPT_TRY(ckpt::check_pointers({dy, x, prob_perm, row_of_slot, expert_offsets, h_q, h_scale, w1, w2, dx_perm, dw1,
                                 dw2, dprob_perm, ws}));
  const ckpt::Carve w = ckpt::carve(d);
  if (ws_bytes < w.total) return MOE_ERR_WORKSPACE;
  Ctx c;
  CKPT_TRY(abi_device_ctx(stream, &c));
  char* base = ckpt::ws_base(ws);
  void *dy_rows = base + w.dy, *x_rows = base + w.x, *dh = base + w.dh, *act = base + w.act;
  float* part = reinterpret_cast<float*>(base + w.part);
  const DType ct = dw_dtype == MOE_BF16 ? DType::BF16 : DType::F32;
  CKPT_TRY(abi_cuda_status(
      launch_dispatch_rows_pair(c, dy, x, row_of_slot, d.T, d.K, (int64_t)d.D * 2, dy_rows, x_rows)));
  // dA = dy W2 (of the unscaled dy); its epilogue reads the codes and writes
  // dH = p (SwiGLU backward of dA), p act, and each row's part of <dA, act>
  GemmDesc a = ckpt::by_rows(Epi::SwigluBwdQ8, d, expert_offsets, dy_rows, d.D, w2, d.F, true, dh, 2 * (int64_t)d.F);
  a.aux = const_cast<int8_t*>(h_q);
  a.aux2 = act;
  a.qscale = const_cast<float*>(h_scale);
  a.prob = prob_perm;
  a.part = part;
  CKPT_TRY(abi_cuda_status(launch_gemm_tc(c, a, "ffn2_dgrad_swiglu_q8_tc")));
  {
    KernelScope ks("ckpt_dprob", c.stream);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)((d.TK + 255) / 256), 1, 1);
    cfg.blockDim = dim3(256, 1, 1);
    cfg.stream = c.stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CKPT_TRY(abi_cuda_status(cudaLaunchKernelEx(&cfg, ckpt::ckpt_dprob_kernel, (const float*)part, w.parts,
                                                (int64_t)d.TK, dprob_perm)));
  }
  GemmDesc g2 = ckpt::weight_grad(d, expert_offsets, dy_rows, d.D, act, d.F, dw2, ct, base + w.maps0);
  GemmDesc g1 = ckpt::weight_grad(d, expert_offsets, dh, 2 * (int64_t)d.F, x_rows, d.D, dw1, ct, base + w.maps1);
  cudaError_t maps = cudaSuccess;
  if (gemm_tc_group_maps_pair(c, g2, g1, &maps)) {
    CKPT_TRY(abi_cuda_status(maps));
    g1.maps_ready = g2.maps_ready = true;
  }
  CKPT_TRY(abi_cuda_status(launch_gemm_tc(c, g2, "ffn2_wgrad_tc")));
  CKPT_TRY(abi_cuda_status(launch_gemm_tc(c, g1, "ffn1_wgrad_tc")));
  const GemmDesc dx = ckpt::by_rows(Epi::Store, d, expert_offsets, dh, 2 * (int64_t)d.F, w1, d.D, true, dx_perm, d.D);
  return abi_cuda_status(launch_gemm_tc(c, dx, "ffn1_dgrad_tc"));
}
