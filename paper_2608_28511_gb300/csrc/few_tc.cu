// The few-token layer on the tensor cores (bf16).  The weights are the wide
// operand: a tile is 128 rows of one expert's W1 (64 gate and the 64 up rows
// of the same features) or W2, the expert's tokens are the N columns, so every
// weight is read once by TMA and its 128 x 64 blocks feed tcgen05.mma straight
// from a ring that fills the shared memory.  Bound by that stream from HBM: 128
// tokens of D = 2048, F = 1024, E = 128, K = 8 read 1.6 GB in 251 us (graph, router
// included), 6.9 TB/s while it runs; one token 100 MB in 33 us, of which about 16
// are the router, its launch, the lists, the first loads, the hand-over between
// the products, the last barrier and the combine.
//
// One cooperative launch, one block per SM; warp roles (one lane each issues):
//   warps 0-1   weight blocks, in turn, of the first product's tiles and then,
//               without a stop, of the second's;
//   warps 2-3   the tokens' rows beside each weight block, in turn: rows of x
//               gathered by TMA four at a time, then act's, which are in order,
//               as soon as all tiles of that expert's first product are done
//               (a counter an expert, instead of a barrier between the two);
//   warps 4-7   MMA issue, in turn, each into an accumulator of its own;
//   warps 8-11  epilogue: act = silu(g) u, or W2 act by slot.
// A block's wait, its four products and its commit cost one thread about 600
// cycles, and HBM delivers a block every 590: one issuer alone was the bound,
// hence the turns.  Before the roles start, and after they end, all warps build
// the row lists and combine.
#include <algorithm>
#include <cstring>

#include "few.cuh"
#include "tc_ptx.cuh"

namespace moe {
namespace few {
namespace {

using namespace tc;

constexpr int kThreads = 384;
constexpr int kIssuers = 4;
constexpr int kRows = 128;  // weight rows of a tile
constexpr int kK = 64;      // depth of a block: 128 bytes, one swizzle row
constexpr int kABytes = kRows * kK * 2;
constexpr int kMaxStages = 12;
constexpr float kMaxBf16 = 0x1.fep127f;
constexpr int kXchg = 2 * 64 * 17 * 4;  // two buffers of 64 up rows x 16 columns, padded

struct TcArgs {
  Args a;
  CUtensorMap t1, t2, tx, ta, tb;  // W1, W2 in 128-row boxes; x, act in one-row boxes; act in 16-row boxes
  int ncap;    // columns of a stage's token block: a multiple of 16
  int terms;   // bf16 terms of act: 2 (its value and what that rounding left), or 1
  int nacc;    // issuing warps, and accumulators of a tile: 2 or 4
  int stages;  // a multiple of nacc
  int tmem_cols;
};

__device__ __forceinline__ void tmem_ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
}
// The registers of r are tied to the wait, so no use of them is scheduled before it.
__device__ __forceinline__ void tmem_ld16_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])
               :
               : "memory");
}
// Rows r[0] .. r[3] of a map with one-row boxes, columns x .. x + 63, as four
// consecutive 128-byte rows.
__device__ __forceinline__ void tma_gather4(uint32_t dst, const CUtensorMap* map, uint32_t bar, int x, const int (&r)[4]) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, "
      "%5, %6, %7}], [%2];" ::"r"(dst),
      "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3])
      : "memory");
}
// Generic-proxy accesses before it and copy-engine accesses after it (or the
// reverse) are ordered.
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async;" ::: "memory"); }

// The four epilogue warps' barrier; the second form also returns whether any
// thread passed true, the same answer to all of them.
__device__ __forceinline__ void epi_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool epi_any(bool x) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.or.pred q, 1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}\n"
      : "=r"(r)
      : "r"((uint32_t)x)
      : "memory");
  return r != 0;
}

// A tile of either product, or one of its parts along k: rows row0 .. row0 + 127
// of its weight map, blocks kb0 .. kb0 + nkb - 1, for expert rows r0 .. r0 + n of
// the lists.
struct Item {
  bool second;
  int e, tile, part, r0, n;
  int index;  // of the tile among its product's
  int64_t row0;
  int kb0, nkb;
};

// A block's tiles.  First product: cta, cta + ncta, ... (expert by expert).
// Second: all blocks in turn, after the blocks that have one tile less of the
// first have taken about as much of the second (33 tokens: 123.5 -> 122.2 us);
// with one wave or less of first tiles nothing is given ahead, because those
// blocks would all wait for the first product's end.
//
// Up to kSplitT tokens, a product with so few tiles that most blocks would have
// none has them cut along k into two or four units: one SM alone draws a
// seventieth of HBM's rate (one token, one of 64 experts of 2048 x 1024, 16 tiles
// each product: 27.8 us whole, 23.6 in four).  With a tile for more than a
// quarter of the blocks cutting loses (128 tiles: 34.0 us whole, 39.4 in two): a
// unit costs about 0.6 us beside its weights, and joining the parts of a tile of
// the first product two round trips to L2.
struct Walk {
  int i, step, lim;              // next unit of this phase
  int phase, n1, n2, per1, per2;
  int parts1, parts2;            // units a tile
  int r1, ahead;                 // second units that blocks r1 .. take first
};
__device__ __forceinline__ int split_parts(int tiles, int nkb) {
  int parts = 1;
  while (parts < kSplitParts && 4 * tiles * parts <= (int)gridDim.x && tiles * parts * 2 <= kSplitUnits &&
         nkb >= 8 * parts)
    parts *= 2;
  return parts;
}
template <bool SPLIT>
__device__ __forceinline__ Walk make_walk(const Args& a, const Lists& L) {
  Walk w;
  w.per1 = a.F / 64;
  w.per2 = (a.D + kRows - 1) / kRows;
  const int nkb1 = a.D / kK, nkb2 = a.F / kK;
  w.parts1 = SPLIT ? split_parts(L.nact * w.per1, nkb1) : 1;
  w.parts2 = SPLIT ? split_parts(L.nact * w.per2, nkb2) : 1;
  w.n1 = L.nact * w.per1 * w.parts1;
  w.n2 = L.nact * w.per2 * w.parts2;
  const int g = (int)gridDim.x;
  w.r1 = w.n1 % g;
  // second units as long as a first one
  const int more = (nkb1 * w.parts2 + nkb2 * w.parts1 / 2) / (nkb2 * w.parts1);
  w.ahead = w.n1 < g || w.r1 == 0 ? 0 : min(w.n2, more * (g - w.r1));
  w.phase = 0;
  w.i = blockIdx.x;
  w.step = g;
  w.lim = w.n1;
  return w;
}
template <bool SPLIT>
__device__ __forceinline__ bool next_item(Walk& w, const Args& a, const Lists& L, Item& it) {
  while (w.i >= w.lim) {
    const int g = (int)gridDim.x, c = (int)blockIdx.x;
    if (w.phase == 0) {  // those given ahead
      w.phase = 1;
      w.lim = c >= w.r1 ? w.ahead : 0;
      w.i = c >= w.r1 ? c - w.r1 : 0;
      w.step = g - w.r1;
    } else if (w.phase == 1) {  // the others; they go on where the first product's ended
      w.phase = 2;
      w.lim = w.n2;
      w.i = w.ahead + (w.ahead ? c : (c - w.r1 + g) % g);
      w.step = g;
    } else {
      return false;
    }
  }
  it.second = w.phase > 0;
  const int per = it.second ? w.per2 : w.per1, parts = !SPLIT ? 1 : it.second ? w.parts2 : w.parts1;
  it.index = w.i / parts;
  it.part = w.i % parts;
  it.e = L.active[it.index / per];
  it.tile = it.index % per;
  it.r0 = L.off[it.e];
  it.n = L.off[it.e + 1] - it.r0;
  it.row0 = (int64_t)it.e * (it.second ? a.D : 2 * a.F) + it.tile * kRows;
  const int nkb = (it.second ? a.F : a.D) / kK;
  it.kb0 = nkb * it.part / parts;
  it.nkb = nkb * (it.part + 1) / parts - it.kb0;
  w.i += w.step;
  return true;
}

// SPLIT: the products may be cut along k (kept out of the other instantiation:
// its code alone cost every call 0.5 to 0.8 us).
template <bool SPLIT>
__global__ void __launch_bounds__(kThreads, 1) few_layer_tc_kernel(const __grid_constant__ TcArgs p) {
  const Args& a = p.a;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ Lists L;
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], tfull[2], tempty[2], done;
  __shared__ uint32_t s_tmem;
  __shared__ bool s_last;
  __shared__ volatile int s_abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int stages = p.stages;
  const uint32_t stage_bytes = kABytes + p.terms * p.ncap * 128;
  const uint32_t ring = smem_u32(smem);
  float* xchg = reinterpret_cast<float*>(smem + stages * stage_bytes);

  const int nacc = p.nacc;
  if (tid == 0) {
    for (int s = 0; s < stages; ++s) {
      mbar_init(smem_u32(&full[s]), 2);  // the two producers
      mbar_init(smem_u32(&empty[s]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&tfull[i]), nacc);
      mbar_init(smem_u32(&tempty[i]), 4);
    }
    mbar_init(smem_u32(&done), nacc);
    fence_barrier_init();
    s_abort = 0;
    tma_prefetch_desc(&p.t1);
    tma_prefetch_desc(&p.t2);
    tma_prefetch_desc(&p.tx);
    tma_prefetch_desc(&p.ta);
    tma_prefetch_desc(&p.tb);
  }
  if (warp == 4) {
    tmem_alloc(smem_u32(&s_tmem), p.tmem_cols);
    tmem_relinquish();
  }
  build_lists(L, *reinterpret_cast<ListScratch*>(smem), a.topk_idx, a.T, a.K);  // scratch in the idle ring
  fence_proxy_async_smem();  // before the copy engine writes there
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;

  Walk wk = make_walk<SPLIT>(a, L);
  Item it;
  // Block b of this CTA (base: those of the items before) goes through stage
  // b % stages and is handled by warp b % (number of warps) of each role.  The
  // number of stages is a multiple of those numbers, so every use of a stage is
  // one warp's, in order: a wait on a barrier's parity is never a round behind.
  int base = 0;
  auto stage_of = [&](int b, uint32_t& phase) {
    phase = (b / stages) & 1;
    return b % stages;
  };
  if (warp < 4) {
    // ---------------------------------------------------------- weight blocks; token rows
    if (lane == 0) {
      const bool tokens = warp >= 2;
      const int turn = warp & 1;
      bool ok = true, all_ready = false;
      int issued = 0;  // this warp's last block, plus one
      for (; ok && next_item<SPLIT>(wk, a, L, it); base += it.nkb) {
        if (tokens && it.second && !all_ready) {
          // the expert's rows of act are written; once every tile of the first
          // product is done, no more items ask (the asking took 1.8 us an item)
          all_ready = ld_acquire(a.counters + 1) >= (uint32_t)(wk.n1 / wk.parts1);
          if (!all_ready && !wait_count(a.counters + kFewReady + it.e, wk.per1, a.err)) s_abort = 1;
          fence_proxy_async();
        }
        const CUtensorMap* map = it.second ? &p.t2 : &p.t1;
        // the expert's rows one by one below four (every block of a call may read
        // the same few lines then), else four at a time, or act's, which are
        // consecutive, sixteen at a time (128 tokens: 259 us with gathers, 254);
        // rows past the expert's own feed columns that nothing reads
        const CUtensorMap* rows = it.second ? &p.ta : &p.tx;
        const int terms = it.second ? p.terms : 1;
        auto row = [&](int u, int i) {
          return it.second ? u * a.T * a.K + it.r0 + i : (int)L.tok[it.r0 + i];
        };
        for (int kb = (turn - base) & 1; kb < it.nkb; kb += 2) {
          uint32_t phase;
          const int stage = stage_of(base + kb, phase);
          if (!wait_bounded(smem_u32(&empty[stage]), phase ^ 1u, &s_abort, a.err)) { ok = false; break; }
          const uint32_t fb = smem_u32(&full[stage]);
          const uint32_t sa = ring + stage * stage_bytes, sb = sa + kABytes;
          const int k0 = (it.kb0 + kb) * kK;
          if (!tokens) {
            mbar_expect_tx(fb, kABytes);
            tma_load_2d(sa, map, fb, k0, (int)it.row0);
          } else if (it.n < 4) {
            mbar_expect_tx(fb, terms * it.n * 128);
            for (int u = 0; u < terms; ++u)
              for (int i = 0; i < it.n; ++i)
                tma_load_2d(sb + (u * p.ncap + i) * 128, rows, fb, k0, row(u, i));
          } else if (it.second && it.n > 8) {
            const int groups = (it.n + 15) / 16;
            mbar_expect_tx(fb, terms * groups * 2048);
            for (int u = 0; u < terms; ++u)
              for (int j = 0; j < groups; ++j)
                tma_load_2d(sb + (u * p.ncap + 16 * j) * 128, &p.tb, fb, k0, row(u, 16 * j));
          } else {
            mbar_expect_tx(fb, terms * ((it.n + 3) / 4) * 512);
            for (int u = 0; u < terms; ++u)
              for (int j = 0; j < it.n; j += 4) {
                int r[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) r[i] = row(u, min(j + i, it.n - 1));
                tma_gather4(sb + (u * p.ncap + j) * 128, rows, fb, k0, r);
              }
          }
          issued = base + kb + 1;
        }
      }
      // this warp's last copies have landed before the block ends
      for (int b = issued - 1; b >= 0 && b >= issued - stages; b -= 2) {
        uint32_t phase;
        const int stage = stage_of(b, phase);
        wait_drain(smem_u32(&full[stage]), phase, 1000000000ull);
      }
    }
    __syncwarp();
  } else if (warp < 4 + kIssuers) {
    // ---------------------------------------------------------- MMA issue
    const int turn = warp - 4;
    if (lane == 0 && turn < nacc) {
      int acc = 0;
      uint32_t acc_phase = 0;
      bool ok = true;
      for (; ok && next_item<SPLIT>(wk, a, L, it); base += it.nkb) {
        if (!wait_bounded(smem_u32(&tempty[acc]), acc_phase ^ 1u, &s_abort, a.err)) break;
        tc_fence_after();
        const uint32_t d = tmem + (acc * nacc + turn) * p.ncap;
        const uint32_t idesc = make_idesc((it.n + 15) & ~15, kRows, false, false);
        const int first = (turn - base) & (nacc - 1);
        for (int kb = first; kb < it.nkb; kb += nacc) {
          uint32_t phase;
          const int stage = stage_of(base + kb, phase);
          if (!wait_bounded(smem_u32(&full[stage]), phase, &s_abort, a.err)) { ok = false; break; }
          tc_fence_after();
          const uint32_t sa = ring + stage * stage_bytes, sb = sa + kABytes;
#pragma unroll
          for (int k = 0; k < kK / 16; ++k)
            mma_bf16(d, make_sdesc(sa + k * 32, 16, 1024), make_sdesc(sb + k * 32, 16, 1024), idesc,
                     (kb > first || k > 0) ? 1u : 0u);
          if (it.second && p.terms == 2) {
            const uint32_t sl = sb + p.ncap * 128;
#pragma unroll
            for (int k = 0; k < kK / 16; ++k)
              mma_bf16(d, make_sdesc(sa + k * 32, 16, 1024), make_sdesc(sl + k * 32, 16, 1024), idesc, 1u);
          }
          mma_commit(smem_u32(&empty[stage]));
        }
        if (!ok) break;
        mma_commit(smem_u32(&tfull[acc]));  // at once if this warp had no block of the item
        if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
      }
      mma_commit(smem_u32(&done));
      wait_drain(smem_u32(&done), 0, 1000000000ull);  // every issuer's products are complete
    }
    __syncwarp();
  } else {
    // ---------------------------------------------------------- epilogue
    const int q = warp & 3;  // TMEM lane quarter: rows 32 q .. 32 q + 31 of the tile
    int acc = 0, buf = 0;
    uint32_t acc_phase = 0;
    bf16* act = static_cast<bf16*>(a.act);
    const int64_t low = (int64_t)a.T * a.K * a.F;  // act's second term
    for (; next_item<SPLIT>(wk, a, L, it); base += it.nkb) {
      // all four warps take the same decision: the barriers below need every one of them
      if (epi_any(!wait_bounded(smem_u32(&tfull[acc]), acc_phase, &s_abort, a.err))) break;
      tc_fence_after();
      const uint32_t t = tmem + ((uint32_t)(q * 32) << 16) + acc * nacc * p.ncap;
      const int used = min(nacc, it.nkb);  // accumulators that had a block
      bool whole = true;  // first product: this block finishes the tile
      for (int c0 = 0; c0 < it.n; c0 += 16) {
        const int n = min(16, it.n - c0);
        uint32_t part[kIssuers][16];
#pragma unroll
        for (int j = 0; j < kIssuers; ++j)
          if (j < used) tmem_ld16_issue(t + ((base + j) & (nacc - 1)) * p.ncap + c0, part[j]);
        float v[16];
#pragma unroll
        for (int j = 0; j < kIssuers; ++j) {
          if (j < used) {
            tmem_ld16_wait(part[j]);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = (j ? v[i] : 0.f) + __uint_as_float(part[j][i]);
          }
        }
        if (SPLIT && !it.second && wk.parts1 > 1) {
          // h's part goes to the workspace (n <= kSplitT columns); the block that
          // brings the tile's last one adds them, in order
          float* hp = a.hpart + (int64_t)it.index * wk.parts1 * (kSplitT * kRows) + q * 32 + lane;
#pragma unroll
          for (int i = 0; i < kSplitT; ++i)
            if (i < n) __stcg(hp + (it.part * kSplitT + i) * kRows, v[i]);
          epi_barrier();
          if (tid == kThreads - 128) {
            __threadfence();
            s_last = atomicAdd(a.counters + kFewTiles + it.index, 1u) == (uint32_t)wk.parts1 - 1u;
            __threadfence();
          }
          epi_barrier();
          whole = s_last;
          if (!whole) break;
#pragma unroll
          for (int i = 0; i < kSplitT; ++i) {
            if (i < n) {
              float h[kSplitParts];
#pragma unroll
              for (int j = 0; j < kSplitParts; ++j)
                h[j] = j < wk.parts1 ? __ldcg(hp + (j * kSplitT + i) * kRows) : 0.f;
              v[i] = (h[0] + h[1]) + (h[2] + h[3]);
            }
          }
        }
        if (!it.second) {
          float* xb = xchg + buf * (64 * 17);
          if (q >= 2) {
#pragma unroll
            for (int i = 0; i < 16; ++i) xb[((q - 2) * 32 + lane) * 17 + i] = v[i];
          }
          epi_barrier();
          if (q < 2) {
            const int f = it.tile * 64 + q * 32 + lane;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (i >= n) break;
              const float z = v[i] * sigmoid_rn(v[i]) * xb[(q * 32 + lane) * 17 + i];
              const int64_t at = (int64_t)(it.r0 + c0 + i) * a.F + f;
              if (p.terms == 2) {
                // the first term stays finite, so that the second is z's rest where z
                // rounds to infinity, and infinity or NaN where z is
                const bf16 hi = __float2bfloat16_rn(fminf(fmaxf(z, -kMaxBf16), kMaxBf16));
                act[at] = hi;
                act[at + low] = __float2bfloat16_rn(z - __bfloat162float(hi));
              } else {
                act[at] = __float2bfloat16_rn(z);
              }
            }
          }
          buf ^= 1;
        } else {
          const int d = it.tile * kRows + q * 32 + lane;
          if (d < a.D) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              if (i >= n) break;
              a.ypart[((int64_t)it.part * a.T * a.K + L.slot[it.r0 + c0 + i]) * a.D + d] = v[i];
            }
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&tempty[acc]));
      if (!it.second && whole) {  // these rows of act are written, and the copy engines may read them
        fence_proxy_async();
        epi_barrier();
        if (tid == kThreads - 128) {
          __threadfence();  // cumulative: the other warps' writes before the barrier too
          red_release(a.counters + kFewReady + it.e, 1u);
          red_release(a.counters + 1, 1u);
        }
      }
      if (++acc == 2) { acc = 0; acc_phase ^= 1u; }
    }
  }
  tc_fence_before();
  grid_barrier(a.counters, a.err);
  tc_fence_after();
  if (warp == 4) tmem_dealloc(tmem, p.tmem_cols);
  grid_dependency_launch();
  combine_rows<bf16, SPLIT>(a, wk.parts2);
}

}  // namespace

cudaError_t launch_few_tc(const Ctx& c, const Args& a) {
  TcArgs p;
  memset(&p, 0, sizeof(p));
  p.a = a;
  if (!make_map(&p.t1, a.w1, a.D, (uint64_t)a.E * 2 * a.F, (uint64_t)a.D * 2, kK, kRows) ||
      !make_map(&p.t2, a.w2, a.F, (uint64_t)a.E * a.D, (uint64_t)a.F * 2, kK, kRows) ||
      !make_map(&p.tx, a.x, a.D, a.T, (uint64_t)a.D * 2, kK, 1) ||
      !make_map(&p.ta, a.act, a.F, (uint64_t)kFewTerms(a.T) * a.T * a.K, (uint64_t)a.F * 2, kK, 1) ||
      !make_map(&p.tb, a.act, a.F, (uint64_t)kFewTerms(a.T) * a.T * a.K, (uint64_t)a.F * 2, kK, 16))
    return cudaErrorInvalidValue;
  // an expert has at most T tokens; the ring takes what the lists leave of the
  // 227 KB of shared memory
  p.ncap = (a.T + 15) & ~15;
  // two accumulators of ncap columns an issuer, in the 512 columns of TMEM
  p.nacc = p.ncap <= 64 ? kIssuers : kIssuers / 2;
  p.tmem_cols = 32;
  while (p.tmem_cols < 2 * p.nacc * p.ncap) p.tmem_cols *= 2;
  p.terms = kFewTerms(a.T);
  const int stage_bytes = kABytes + p.terms * p.ncap * 128;
  // Where even the fewest experts that T tokens can choose, K, have tiles for more
  // than a quarter of the blocks, nothing is cut.
  const bool split = a.T <= kSplitT && 4 * a.K * std::min(a.F / 64, (a.D + kRows - 1) / kRows) <= c.num_sms;
  auto kernel = split ? few_layer_tc_kernel<true> : few_layer_tc_kernel<false>;
  static PerDevice budgets[2];
  int budget = 0;  // bytes of dynamic shared memory
  const cudaError_t st = budgets[split].get(c.device, cudaSuccess, &budget, [&](int* v) {
    cudaFuncAttributes fa;
    cudaError_t e = cudaFuncGetAttributes(&fa, kernel);
    if (e != cudaSuccess) return e;
    *v = (227 * 1024 - (int)fa.sharedSizeBytes) & ~1023;
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, *v);
  });
  if (st != cudaSuccess) return st;
  p.stages = std::min(kMaxStages, (budget - 1024 - kXchg) / stage_bytes) / p.nacc * p.nacc;
  const int64_t items = (int64_t)std::min(a.E, a.T * a.K) * std::max(a.F / 64, (a.D + kRows - 1) / kRows) *
                        (split ? kSplitParts : 1);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)std::min<int64_t>(c.num_sms, items), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = p.stages * stage_bytes + kXchg + 1024;
  cfg.stream = c.stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeCooperative;
  attr[0].val.cooperative = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  KernelScope ks("few_layer_tc", c.stream);
  return cudaLaunchKernelEx(&cfg, kernel, p);
}

}  // namespace few
}  // namespace moe
