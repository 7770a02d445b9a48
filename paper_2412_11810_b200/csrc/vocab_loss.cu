// Soft-max cross entropy over a large vocabulary with the readout product inside, and its gradients (include/snn.h,
// "sequence-model operators").  The logits never reach memory: the forward pass reduces every 256 x 256 tile of them to a
// maximum and a sum per row while it leaves tensor memory, the backward pass recomputes the tiles, turns them into
// derivatives dz on the way out and multiplies those, one piece of the vocabulary at a time, by w and by x.
//
// Everything heavy is one persistent kernel on pairs of SMs (umma.cuh) with four epilogues:
//   STATS   z tile -> per row (maximum, sum of exponentials), the target's logit
//   GRAD    z tile -> dz tile, to memory through shared memory and TMA
//   DX      dz w^T, fp32, added to what earlier pieces left (the contraction may be split; parts are joined at the end)
//   DW      x^T dz, scaled and rounded
// Work per pass: 2 rows dim classes for STATS, three times that for the backward pass (one of them the recomputation).
//
// fp32 operands are split into three bf16 parts of 8 bits: all 24 bits of a value, whatever its magnitude beside the others'
// (bf16 has the exponents of fp32).  Six products of parts instead of one: those left out are below 2^-24 of the whole.  Two
// scaled fp16 parts need half of them, but what is 2^18 times smaller than the largest value of its tensor loses bits to the
// common scale: with one feature of x 10^9 times the others the others' rows of dw were off by 2e-3 of their norm.
#include <algorithm>
#include <cmath>
#include <mutex>

#include "seq_common.cuh"
#include "umma.cuh"

using namespace snnk;

namespace {

constexpr uint32_t VL_TIMEOUT = 1u;               // status bit: a bounded wait ran out
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int VL_RUN = 8;                                    // k-blocks per run (fp32 operands)
// Warps of the epilogue: one per quarter of tensor memory's lanes, or two with half of the tile's columns each.  Two hide
// the epilogue's latency where the contraction is short and the epilogue sets the pace (8192 x 64 x 65536 bf16 forward: 403
// us with four warps, 336 with eight); where it is long four leave more of the SM to the products (8192 x 2048 x 131072
// backward: 9.3 ms against 9.8).
constexpr int VL_SHORT = 16;                                 // k-blocks: eight warps below
constexpr uint32_t VL_STORE_BYTES = UM_HALF * 128;           // one staged block of dz per half: 128 rows x 64 values
constexpr size_t VL_SMEM = 1024 + (size_t)UM_STAGES * UM_STAGE_BYTES + 2 * VL_STORE_BYTES + 256;
// dz / (gradient of the row loss) lies in [-1, 1].  As an operand of the next two products it has the operands' type: of fp32
// three bf16 parts (nothing is lost), bf16 8 bits, fp16 11 bits down to 2^-28, after this scale, and steps of 2^-38 below.
// (The rounding adds 6e-4 to the 1.7e-3 that rounding the gradients themselves to bf16 costs: 4096 x 1024 x 50257, norms;
// two parts would double the time of two of the three products.)
constexpr float FP16_DZ_SCALE = 16384.f;
// The others have the range for the mean's factor, as a power of two, before the products, so that sums over the rows stay
// within fp32 wherever their mean does.
float dz_unit_of(int dtype, int rows) {
  float unit = 1.f;
  if (dtype == SNN_DTYPE_FP16) return FP16_DZ_SCALE;
  for (int64_t n = 1; n < rows; n *= 2) unit *= 0.5f;
  return unit;
}
// The kernels of a call follow one another closely: each is launched while the one before still runs, sets itself up, and
// waits here before it touches memory.  (Every kernel behind another one waits, so that their bodies never overlap.)
__device__ __forceinline__ void wait_for_kernel_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_kernel_start() { asm volatile("griddepcontrol.launch_dependents;"); }
constexpr size_t PIECE_BYTES = (size_t)512 << 20;            // dz held at a time
constexpr int MAX_SPLITS = 32;

enum Epilogue { STATS, GRAD, DX, DW };
// The tensor cores do not round a sum to nearest, and what they cut adds up over a long contraction: 5e-6 of the result
// after 8000 terms, where fp32 should have a tenth of that.  So for fp32 operands (RUNS) the epilogue takes over the
// accumulator after every VL_RUN k-blocks and adds it to sums in its registers; the other accumulator fills meanwhile.

struct ProductParams {
  CUtensorMap a, b, out;      // out: GRAD only
  int tiles_m, tiles_n;       // 256 x 256 tiles; m is the fastest in the order of work for STATS, GRAD and DX, n for DW
  int kblocks, splits;        // 64-deep blocks of the contraction; DX: parts of it
  int n_pairs;                // products of operand planes: 1, or 6 for fp32 operands in three bf16 planes
  uint32_t pair_a, pair_b;    // their planes, four bits each, the smallest products first
  int a0, b0, bk0;            // first row of A and of B, first k of B (A's k starts at 0)
  int m, n;                   // rows of A and of B that exist from there on
  bool bf16;
  bool behind;                // (host) another kernel of the call
  // STATS and GRAD
  const void* targets;
  int target_bits;
  int64_t ignore_index;
  int classes;
  float z_scale;              // times log2 e: exponents of 2
  float2* partial;            // [tile_n][halves][rows]
  float* target_z;            // [rows], in units of log 2
  const float* lse;
  float dz_unit;              // GRAD: what stands for a derivative of one, a power of two
  int planes;
  // DX and DW
  float* acc;                 // DX: [splits][m][n_pitch]
  int64_t acc_split;
  int acc_pitch;
  bool accumulate;
  void* dw;
  int64_t dw_stride;
  int dw_dtype;
  bool dw_vector;             // rows of dw are aligned to 16 bytes
  const float* alpha;         // DW: factor, from the device
  uint32_t* status;
  // WAIT_TESTS: limits of the waits.  The self-test lets them run out: no loads from a unit of work on, or one warp of the
  // epilogue that does not wait for it
  uint32_t polls;
  int loads_end, quits_at;
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The target of a row, or -1 if it does not count, -2 if it is not a class.
__device__ __forceinline__ int target_of(const void* targets, int bits, int64_t ignore, int classes, int row) {
  const int64_t t = bits == 64 ? reinterpret_cast<const int64_t*>(targets)[row] : (int64_t) reinterpret_cast<const int32_t*>(targets)[row];
  if (t == ignore) return -1;
  return t >= 0 && t < classes ? (int)t : -2;
}

struct Barriers {
  uint64_t full[UM_STAGES], empty[UM_STAGES];   // full: used in the even block only
  uint64_t acc_full[2], acc_empty[2];           // acc_empty: used in the even block only
  uint32_t tmem;
  uint32_t gave_up;
};

// A bounded wait that also ends when another role of this block gave up.
__device__ __forceinline__ bool wait_for(uint64_t* bar, uint32_t parity, Barriers& s, uint32_t* status, uint32_t limit) {
  for (uint32_t i = 0; i < limit; ++i) {
    if (mbar_try_wait(bar, parity)) return true;
    if ((i & 63u) == 63u && *reinterpret_cast<volatile uint32_t*>(&s.gave_up)) return false;
  }
  *reinterpret_cast<volatile uint32_t*>(&s.gave_up) = 1u;
  if (status) atomicOr(status, VL_TIMEOUT);
  return false;
}

// Whether all 128 threads at a named barrier say so.
__device__ __forceinline__ bool together(bool ok, int barrier) {
  uint32_t all;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %2, 0;\n\t"
      "barrier.cta.red.and.pred q, %1, 128, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all) : "r"(barrier), "r"((uint32_t)ok) : "memory");
  return all != 0;
}

template <bool MN_MAJOR>
__device__ __forceinline__ void load_operand(unsigned char* smem, const CUtensorMap* map, int row, int k, int plane, uint32_t bar) {
  if (MN_MAJOR) {
    tma_pair_load_3d(smem, map, row, k, plane, bar);
    tma_pair_load_3d(smem + UM_KB * 128, map, row + 64, k, plane, bar);
  } else {
    tma_pair_load_3d(smem, map, k, row, plane, bar);
  }
}

// the i-th unit of work of a pair: its tile and its part of the contraction
struct Unit {
  int m, n, split, kb0, kbs;
};
template <int EPI> __device__ __forceinline__ Unit unit_of(const ProductParams& p, int u) {
  Unit w;
  if (EPI == DW) {
    w.n = u % p.tiles_n; w.m = u / p.tiles_n; w.split = 0;
  } else {
    w.m = u % p.tiles_m;
    const int v = u / p.tiles_m;
    w.n = v % p.tiles_n; w.split = v / p.tiles_n;
  }
  w.kb0 = (int)((int64_t)p.kblocks * w.split / p.splits);
  w.kbs = (int)((int64_t)p.kblocks * (w.split + 1) / p.splits) - w.kb0;
  return w;
}

__device__ __forceinline__ void store_dw(const ProductParams& p, int64_t at, float f) {
  if (p.dw_dtype == SNN_DTYPE_FP32) ((float*)p.dw)[at] = f;
  else if (p.dw_dtype == SNN_DTYPE_BF16) ((__nv_bfloat16*)p.dw)[at] = __float2bfloat16_rn(f);
  else ((__half*)p.dw)[at] = __float2half_rn(f);
}

template <int EPI, bool A_MN, bool B_MN, int WARPS, bool RUNS>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(32 * (2 + WARPS), 1) product_kernel(const __grid_constant__ ProductParams p) {
  constexpr int HALVES = WARPS / 4, WIDTH = UM_TILE / HALVES;   // columns per warp of the epilogue
  static_assert(!RUNS || HALVES == 2, "a thread's sums fit its registers");
  extern __shared__ unsigned char s_raw[];
  unsigned char* const s_base = s_raw + ((1024u - (smem_u32(s_raw) & 1023u)) & 1023u);
  unsigned char* const s_store = s_base + (size_t)UM_STAGES * UM_STAGE_BYTES;
  Barriers& s = *reinterpret_cast<Barriers*>(s_store + 2 * VL_STORE_BYTES);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const uint32_t rank = cluster_rank();
  const int pair = blockIdx.x >> 1, n_pairs_sm = gridDim.x >> 1;
  const int units = p.tiles_m * p.tiles_n * p.splits;
  const uint32_t polls = WAIT_TESTS ? p.polls : MBAR_WAIT_LIMIT;
  let_next_kernel_start();

  if (tid == 0) {
    for (int i = 0; i < UM_STAGES; ++i) {
      mbar_init(&s.full[i], 1);
      mbar_init(&s.empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&s.acc_full[i], 1);
      mbar_init(&s.acc_empty[i], 2 * WARPS);
    }
    s.gave_up = 0;
    mbar_fence_init();
  }
  if (warp == 1) pair_tmem_alloc(&s.tmem, UM_TMEM_COLS);
  tcgen05_before_sync();
  cluster_sync_all();
  tcgen05_after_sync();
  const uint32_t tmem = s.tmem;
  wait_for_kernel_before();

  if (warp == 0) {
    if (lane == 0) {   // loads: this block's halves of A and B, announced to the even block's barrier
      int it = 0;
      bool ok = true;
      for (int u = pair; u < units && !(WAIT_TESTS && u >= p.loads_end) && ok; u += n_pairs_sm) {
        const Unit w = unit_of<EPI>(p, u);
        const int row_a = p.a0 + w.m * UM_TILE + (int)rank * UM_HALF, row_b = p.b0 + w.n * UM_TILE + (int)rank * UM_HALF;
        for (int q = 0; q < p.n_pairs && ok; ++q) {
          const int plane_a = (p.pair_a >> (4 * q)) & 15, plane_b = (p.pair_b >> (4 * q)) & 15;
          for (int kb = 0; kb < w.kbs; ++kb, ++it) {
            const int st = it % UM_STAGES;
            if (it >= UM_STAGES && !(ok = wait_for(&s.empty[st], (uint32_t)(it / UM_STAGES - 1) & 1u, s, p.status, polls))) break;
            unsigned char* const at = s_base + (size_t)st * UM_STAGE_BYTES;
            if (rank == 0) mbar_arrive_expect_tx(&s.full[st], 2 * UM_STAGE_BYTES);
            const uint32_t bar = peer_address(smem_u32(&s.full[st]), 0);
            const int k = (w.kb0 + kb) * UM_KB;
            load_operand<A_MN>(at, &p.a, row_a, k, plane_a, bar);
            load_operand<B_MN>(at + UM_OPERAND_BYTES, &p.b, row_b, p.bk0 + k, plane_b, bar);
          }
        }
      }
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {   // products, of both blocks
      const uint32_t idesc = f16_instruction(p.bf16, A_MN, B_MN);
      int it = 0, run = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += n_pairs_sm) {
        const Unit w = unit_of<EPI>(p, u);
        const int n_it = p.n_pairs * w.kbs;
        for (int i0 = 0; i0 < n_it && ok; i0 += RUNS ? VL_RUN : n_it, ++run) {   // a run of k-blocks into one accumulator
          const int buf = run & 1, end = RUNS ? min(i0 + VL_RUN, n_it) : n_it;
          if (run >= 2 && !(ok = wait_for(&s.acc_empty[buf], (uint32_t)(run / 2 - 1) & 1u, s, p.status, polls))) break;
          tcgen05_after_sync();
          const uint32_t acc = tmem + (uint32_t)buf * UM_TILE;
          for (int i = i0; i < end; ++i, ++it) {
            const int st = it % UM_STAGES;
            if (!(ok = wait_for(&s.full[st], (uint32_t)(it / UM_STAGES) & 1u, s, p.status, polls))) break;
            tcgen05_after_sync();
            const uint32_t at = smem_u32(s_base + (size_t)st * UM_STAGE_BYTES);
#pragma unroll
            for (int j = 0; j < UM_KB / 16; ++j)
              pair_mma_f16(acc, operand_descriptor<A_MN>(at + j * kstep_bytes<A_MN>()),
                           operand_descriptor<B_MN>(at + UM_OPERAND_BYTES + j * kstep_bytes<B_MN>()), idesc, i > i0 || j > 0);
            pair_commit(&s.empty[st]);
          }
          if (ok) pair_commit(&s.acc_full[buf]);
        }
      }
    }
  } else {
    // ---- epilogue: a thread has one row of this block's half of the tile
    const int quarter = warp & 3, row_in_block = quarter * 32 + lane, half = (warp - 2) / 4, half_col0 = half * WIDTH;
    const bool storer = threadIdx.x == 64 + 128 * half;   // of the half's dz blocks
    int store_buf = half;
    const float nan = __uint_as_float(0x7fc00000u);
    // (a wait that ran out in a kernel before: dz is not what it should be)
    const float alpha = EPI != DW ? 0.f : *p.status & VL_TIMEOUT ? nan : *p.alpha;
    int run = 0;
    bool ok = true;
    float sums[RUNS ? WIDTH : 1];
    // the run's accumulator is complete / may be filled again
    auto run_full = [&](int u) {
      const bool quits = WAIT_TESTS && warp == 2 && u >= p.quits_at;
      return (bool)__all_sync(0xffffffffu, wait_for(&s.acc_full[run & 1], (uint32_t)(run / 2) & 1u, s, p.status, quits ? 0u : polls));
    };
    auto run_read = [&]() {
      tcgen05_before_sync();
      __syncwarp();
      if (lane == 0) mbar_arrive_at(peer_address(smem_u32(&s.acc_empty[run & 1]), 0));
      ++run;
    };
    auto accumulator = [&]() { return tmem + (uint32_t)((run & 1) * UM_TILE + half_col0) + ((uint32_t)(32 * quarter) << 16); };
    for (int u = pair; u < units && ok; u += n_pairs_sm) {
      const Unit w = unit_of<EPI>(p, u);
      if constexpr (RUNS) {
        const int n_runs = (p.n_pairs * w.kbs + VL_RUN - 1) / VL_RUN;
#pragma unroll
        for (int j = 0; j < WIDTH; ++j) sums[j] = 0.f;
#pragma unroll 1
        for (int r = 0; r < n_runs && (ok = run_full(u)); ++r) {
          tcgen05_after_sync();
#pragma unroll
          for (int c = 0; c < WIDTH; c += 16) {
            float v[16];
            tmem_load_16(accumulator() + c, v);
#pragma unroll
            for (int j = 0; j < 16; ++j) sums[c + j] += v[j];
          }
          run_read();
        }
      } else {
        ok = run_full(u);
      }
      // Every warp decides for itself whether a wait ran out.  Those that share the buffers of dz meet at a barrier, where one
      // that left would be waited for without end: they go on together or not at all.
      if constexpr (EPI == GRAD) ok = together(ok, 1 + half);
      if (!ok) {
        if (EPI == STATS) {   // the rows' losses become NaN
          for (; u < units; u += n_pairs_sm) {
            const Unit left = unit_of<EPI>(p, u);
            const int row = left.m * UM_TILE + (int)rank * UM_HALF + row_in_block;
            if (row < p.m) p.partial[((int64_t)left.n * HALVES + half) * p.m + row] = make_float2(nan, nan);
          }
        }
        if (EPI == DW) {      // and the gradients of the tiles that are left
          for (; u < units; u += n_pairs_sm) {
            const Unit left = unit_of<EPI>(p, u);
            const int row = left.m * UM_TILE + (int)rank * UM_HALF + row_in_block, col0 = left.n * UM_TILE + half_col0;
            for (int c = 0; c < WIDTH && row < p.m && col0 + c < p.n; ++c) store_dw(p, (int64_t)row * p.dw_stride + col0 + c, nan);
          }
        }
        break;
      }
      tcgen05_after_sync();
      const uint32_t acc = accumulator();
      const int block_row0 = w.m * UM_TILE + (int)rank * UM_HALF;
      const int row = block_row0 + row_in_block;          // within A's rows
      const int col0 = w.n * UM_TILE + half_col0, cols = max(min(p.n - col0, WIDTH), 0);   // of this warp's half
      const bool row_on = row < p.m;
      // the j-th column from c on: in registers already, or loaded from tensor memory
#define V(j) (RUNS ? sums[RUNS ? c + (j) : 0] : loaded[RUNS ? 0 : (j)])
      if constexpr (EPI == STATS) {
        const int target = row_on ? target_of(p.targets, p.target_bits, p.ignore_index, p.classes, row) - (p.b0 + col0) : -1;
        float top = -INFINITY, sum = 0.f;
#pragma unroll(RUNS ? WIDTH / 32 : 1)
        for (int c = 0; c < WIDTH; c += 32) {
          if (c >= cols) continue;
          float loaded[RUNS ? 1 : 32];
          if constexpr (!RUNS) tmem_load_32(acc + c, loaded);
#pragma unroll
          for (int j = 0; j < 32; ++j) V(j) = V(j) * p.z_scale;
          if (target >= c && target < c + 32) {
            float z = 0.f;
#pragma unroll
            for (int j = 0; j < 32; ++j) z = c + j == target ? V(j) : z;
            p.target_z[row] = z;
          }
          if (cols - c < 32) {
#pragma unroll
            for (int j = 0; j < 32; ++j) V(j) = c + j < cols ? V(j) : -INFINITY;
          }
          float m = top;
#pragma unroll
          for (int j = 0; j < 32; ++j) m = fmaxf(m, V(j));
          const float at = m == -INFINITY ? 0.f : m;
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 32; ++j) part += exp2_fast(V(j) - at);
          sum = sum * exp2_fast(top - at) + part;
          top = m;
        }
        if (row_on) p.partial[((int64_t)w.n * HALVES + half) * p.m + row] = make_float2(top, sum);
      }
      if constexpr (EPI == GRAD) {
        const int target = row_on ? target_of(p.targets, p.target_bits, p.ignore_index, p.classes, row) : -1;
        const bool counts = target >= 0;
        const int target_col = target - (p.b0 + col0);
        // lse log2 e in two parts: the second, what rounding the first leaves, as a factor
        const double lse2_exact = counts ? (double)p.lse[row] * 1.4426950408889634074 : 0.;
        const float lse2 = (float)lse2_exact, rest = p.dz_unit * (1.f - (float)(lse2_exact - (double)lse2) * LN2);
#pragma unroll(RUNS ? WIDTH / 64 : 1)
        for (int c = 0; c < WIDTH; c += 64) {
          if (c >= cols) continue;
          float loaded[RUNS ? 1 : 64];
          if constexpr (!RUNS) {
            tmem_load_32(acc + c, *reinterpret_cast<float(*)[32]>(&loaded[0]));
            tmem_load_32(acc + c + 32, *reinterpret_cast<float(*)[32]>(&loaded[32]));
          }
#pragma unroll
          for (int j = 0; j < 64; ++j) V(j) = counts ? exp2_fast(fmaf(V(j), p.z_scale, -lse2)) * rest : 0.f;
          if (counts && target_col >= c && target_col < c + 64) {
#pragma unroll
            for (int j = 0; j < 64; ++j) V(j) = c + j == target_col ? V(j) - p.dz_unit : V(j);
          }
          for (int plane = 0; plane < p.planes; ++plane) {
            // the buffer's previous store has to have read it (there are two buffers: one per half, or both for all)
            if (storer) bulk_read_done<HALVES == 1 ? 1 : 0>();
            asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
            unsigned char* const out = s_store + store_buf * VL_STORE_BYTES + row_in_block * 128;
#pragma unroll
            for (int g = 0; g < 8; ++g) {   // 16-byte pieces, swizzled as the tensor map says
              uint32_t q[4];
#pragma unroll
              for (int h = 0; h < 4; ++h) {
                float &lo = V(8 * g + 2 * h), &hi = V(8 * g + 2 * h + 1);
                if (p.bf16) {
                  const __nv_bfloat162 r = __float22bfloat162_rn(make_float2(lo, hi));
                  q[h] = *reinterpret_cast<const uint32_t*>(&r);
                  if (p.planes > 1) {   // what is left for the next plane
                    const float2 f = __bfloat1622float2(r);
                    lo -= f.x;
                    hi -= f.y;
                  }
                } else {
                  const __half2 r = __float22half2_rn(make_float2(lo, hi));
                  q[h] = *reinterpret_cast<const uint32_t*>(&r);
                }
              }
              *reinterpret_cast<uint4*>(out + ((g ^ (row_in_block & 7)) << 4)) = make_uint4(q[0], q[1], q[2], q[3]);
            }
            fence_proxy_async_smem();
            asm volatile("bar.sync %0, 128;" ::"r"(1 + half) : "memory");
            if (storer && block_row0 < p.m) tma_store_3d(&p.out, col0 + c, block_row0, plane, s_store + store_buf * VL_STORE_BYTES);
            if (storer) bulk_commit();
            if (HALVES == 1) store_buf ^= 1;
          }
        }
      }
      if constexpr (EPI == DX) {
#pragma unroll(RUNS ? WIDTH / 32 : 1)
        for (int c = 0; c < WIDTH; c += 32) {
          if (c >= cols) continue;
          float loaded[RUNS ? 1 : 32];
          if constexpr (!RUNS) tmem_load_32(acc + c, loaded);
          if (row_on) {
            float* const out = p.acc + w.split * p.acc_split + (int64_t)row * p.acc_pitch + col0 + c;
#pragma unroll
            for (int j = 0; j < 32; j += 4) {   // acc_pitch is a multiple of 4: whole groups
              if (c + j < cols) {
                float4 f = make_float4(V(j), V(j + 1), V(j + 2), V(j + 3));
                if (p.accumulate) {
                  const float4 o = *reinterpret_cast<const float4*>(out + j);
                  f = make_float4(f.x + o.x, f.y + o.y, f.z + o.z, f.w + o.w);
                }
                *reinterpret_cast<float4*>(out + j) = f;
              }
            }
          }
        }
      }
      if constexpr (EPI == DW) {
#pragma unroll(RUNS ? WIDTH / 32 : 1)
        for (int c = 0; c < WIDTH; c += 32) {
          if (c >= cols) continue;
          float loaded[RUNS ? 1 : 32];
          if constexpr (!RUNS) tmem_load_32(acc + c, loaded);
#pragma unroll
          for (int j = 0; j < 32; ++j) V(j) *= alpha;
          if (!p.dw_vector || cols - c < 32) {
            // odd strides, the last columns: through shared memory, so that a warp stores along a row
            // (places exchanged within a row, so that both ways use all banks)
            float* const mine = reinterpret_cast<float*>(s_store) + (warp - 2) * (32 * 32);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; ++j) mine[lane * 32 + (j ^ lane)] = V(j);
            __syncwarp();
            const int first = block_row0 + quarter * 32, n_rows = min(p.m - first, 32);
            if (c + lane < cols) {
              const int64_t at = (int64_t)first * p.dw_stride + col0 + c + lane;
#pragma unroll 4
              for (int r = 0; r < n_rows; ++r) {
                const float f = mine[r * 32 + (lane ^ r)];
                store_dw(p, at + r * p.dw_stride, f);
              }
            }
            continue;
          }
          if (!row_on) continue;
          const int64_t at = (int64_t)row * p.dw_stride + col0 + c;
          if (p.dw_dtype == SNN_DTYPE_FP32) {
            float* const out = (float*)p.dw + at;
#pragma unroll
            for (int j = 0; j < 32; j += 4) *reinterpret_cast<float4*>(out + j) = make_float4(V(j), V(j + 1), V(j + 2), V(j + 3));
          } else {
            uint16_t* const out = (uint16_t*)p.dw + at;
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
              uint32_t q[4];
#pragma unroll
              for (int h = 0; h < 4; ++h) {
                if (p.dw_dtype == SNN_DTYPE_BF16) {
                  const __nv_bfloat162 r = __float22bfloat162_rn(make_float2(V(j + 2 * h), V(j + 2 * h + 1)));
                  q[h] = *reinterpret_cast<const uint32_t*>(&r);
                } else {
                  const __half2 r = __float22half2_rn(make_float2(V(j + 2 * h), V(j + 2 * h + 1)));
                  q[h] = *reinterpret_cast<const uint32_t*>(&r);
                }
              }
              *reinterpret_cast<uint4*>(out + j) = make_uint4(q[0], q[1], q[2], q[3]);
            }
          }
        }
      }
#undef V
      if constexpr (!RUNS) run_read();
    }
    if (EPI == GRAD && storer) bulk_done();
  }
  // After a wait that ran out, copies and products may still be under way: give them time to land.
  __syncwarp();
  if (*reinterpret_cast<volatile uint32_t*>(&s.gave_up))
    for (int i = 0; i < 100; ++i) __nanosleep(20000);
  tcgen05_before_sync();
  cluster_sync_all();
  if (warp == 1) pair_tmem_dealloc(tmem, UM_TMEM_COLS);
}

// ---- around the products ---------------------------------------------------------------------------------------

// An operand on its way to 16-bit planes: a copy with an aligned pitch, or fp32 values in three bf16 parts.  With `mask`, rows
// that do not count become zeros (what they hold must not reach the sums over rows).
struct StageJob {
  const void* src;
  int64_t stride;
  int rows, cols;
  uint16_t* dst;
  int64_t pitch, plane;
  bool mask;
};
struct StageParams {
  StageJob job[2];      // x and w; rows = 0 if there is nothing to do.  blockIdx.y selects one
  const void* targets;
  int bits;
  int64_t ignore;
  int classes;
  // the backward pass has blocks with blockIdx.y = 2: the first counts the rows and writes the gradients' factor
  float* alpha;
  float factor;
  const float* dloss;
  uint32_t* status;
  int rows;
};
constexpr int STAGE_COLS = 1024;   // columns of a row that a block takes at a time, four per thread

// To the nearest bf16 value; what is finite stays finite (fp32's largest values round to infinity).
__device__ __forceinline__ __nv_bfloat16 to_bf16_finite(float f) {
  const float top = largest_finite<__nv_bfloat16>();
  return __float2bfloat16_rn(fabsf(f) > top && isfinite(f) ? copysignf(top, f) : f);
}
// Sums of a block's values, the same in every thread; `warp_sums` has 32 entries.
__device__ __forceinline__ double block_sum(double v, double* warp_sums) {
#pragma unroll
  for (int o = 16; o > 0; o /= 2) v += __shfl_xor_sync(0xffffffffu, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0;
  for (int w = 0; w < (int)blockDim.x / 32; ++w) t += warp_sums[w];
  return t;
}
template <typename IO> __global__ void __launch_bounds__(256) stage_kernel(const __grid_constant__ StageParams p) {
  let_next_kernel_start();
  if (blockIdx.y == 2) {
    __shared__ double warp_sums[32];
    if (blockIdx.x != 0) return;
    int n = 0;
#pragma unroll 8
    for (int r = threadIdx.x; r < p.rows; r += 256) n += target_of(p.targets, p.bits, p.ignore, p.classes, r) >= 0;
    const double count = block_sum((double)n, warp_sums);
    if (threadIdx.x == 0) {
      *p.alpha = count > 0 ? (float)((double)p.factor * (p.dloss ? (double)*p.dloss : 1.) / count) : 0.f;
      *p.status = 0u;
    }
    return;
  }
  const StageJob& j = p.job[blockIdx.y];
  const int parts = (int)((j.pitch + STAGE_COLS - 1) / STAGE_COLS);
  for (int64_t i = blockIdx.x; i < (int64_t)j.rows * parts; i += gridDim.x) {
    const int row = (int)(i / parts), c0 = (int)(i % parts) * STAGE_COLS + 2 * threadIdx.x;
    const bool on = !j.mask || target_of(p.targets, p.bits, p.ignore, p.classes, row) >= 0;
    const IO* const src = (const IO*)j.src + row * j.stride;
    uint16_t* const dst = j.dst + row * j.pitch;
    IO v[2][2];
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q / 2][q % 2] = src[min(c0 + 512 * (q / 2) + q % 2, j.cols - 1)];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = c0 + 512 * q;
      if (c >= j.pitch) continue;
      if constexpr (sizeof(IO) == 4) {
        float2 f = make_float2(on && c < j.cols ? v[q][0] : 0.f, on && c + 1 < j.cols ? v[q][1] : 0.f);
#pragma unroll
        for (int part = 0; part < 3; ++part) {
          const __nv_bfloat162 r = __halves2bfloat162(to_bf16_finite(f.x), to_bf16_finite(f.y));
          *reinterpret_cast<__nv_bfloat162*>(dst + part * j.plane + c) = r;
          const float2 g = __bfloat1622float2(r);
          f = make_float2(f.x - g.x, f.y - g.y);   // exact
        }
      } else {
        const IO zero = from_f32<IO>(0.f);
        __half2 r;
        r.x = on && c < j.cols ? v[q][0] : zero;
        r.y = on && c + 1 < j.cols ? v[q][1] : zero;
        *reinterpret_cast<__half2*>(dst + c) = r;
      }
    }
  }
}

__device__ __forceinline__ float2 join_sums(float2 a, float2 b) {   // (maximum, sum of exponentials)
  const float m = a.x != a.x || b.x != b.x ? __uint_as_float(0x7fc00000u) : fmaxf(a.x, b.x), at = m == -INFINITY ? 0.f : m;
  return make_float2(m, a.y * exp2f(a.x - at) + b.y * exp2f(b.x - at));
}
// log-sum-exp of a row from its joined (maximum, sum), in units of 1
__device__ __forceinline__ double log_sum(float2 v) { return ((double)v.x + (double)log2f(v.y)) * 0.69314718055994530942; }
// The tiles' (maximum, sum) of a row joined: log-sum-exp and loss of the row.  32 rows per block, 32 threads per row.  If
// one block has all rows it takes the mean as well (loss != NULL).
__global__ void __launch_bounds__(1024) row_loss_kernel(const float2* partial, int tiles, const float* target_z, int rows, const void* targets,
                                                        int bits, int64_t ignore, int classes, float* lse, float* row_loss, float* row_out,
                                                        float* loss) {
  __shared__ float2 s_part[32][33];
  let_next_kernel_start();
  wait_for_kernel_before();
  const int in_block = threadIdx.x % 32, part = threadIdx.x / 32, row = blockIdx.x * 32 + in_block;
  float2 v = make_float2(-INFINITY, 0.f);
  if (row < rows)
    for (int t = part; t < tiles; t += 32) v = join_sums(v, partial[(int64_t)t * rows + row]);
  s_part[part][in_block] = v;
  __syncthreads();
  // warp `part` joins the 32 parts of row `part` of the block
  v = s_part[in_block][part];
#pragma unroll
  for (int o = 16; o > 0; o /= 2)
    v = join_sums(v, make_float2(__shfl_down_sync(0xffffffffu, v.x, o), __shfl_down_sync(0xffffffffu, v.y, o)));
  __syncthreads();
  if (in_block == 0) s_part[0][part] = v;
  __syncthreads();
  if (part != 0) return;
  float out = 0.f, count = 0.f;
  if (row < rows) {
    v = s_part[0][in_block];
    const int target = target_of(targets, bits, ignore, classes, row);
    const double exact = log_sum(v);
    float l = (float)exact;
    out = (float)(exact - (target >= 0 ? (double)target_z[row] * 0.69314718055994530942 : 0.));
    if (target < 0) l = 0.f, out = target == -1 ? 0.f : __uint_as_float(0x7fc00000u);
    count = target >= 0;
    lse[row] = l;
    row_loss[row] = out;
    if (row_out) row_out[row] = out;
  }
  if (loss) {
    double sum = out;
#pragma unroll
    for (int o = 16; o > 0; o /= 2) {
      sum += __shfl_xor_sync(0xffffffffu, sum, o);
      count += __shfl_xor_sync(0xffffffffu, count, o);
    }
    if (in_block == 0) *loss = (float)(sum / fmax((double)count, 1.));
  }
}

// One block.  The mean of row_loss over the rows that count.
__global__ void __launch_bounds__(1024) mean_kernel(const float* row_loss, int rows, const void* targets, int bits, int64_t ignore, int classes,
                                                    float* loss) {
  __shared__ double warp_sums[32];
  wait_for_kernel_before();
  double sum = 0, count = 0;
  for (int r = threadIdx.x; r < rows; r += blockDim.x) {
    sum += (double)row_loss[r];
    count += target_of(targets, bits, ignore, classes, r) >= 0;
  }
  sum = block_sum(sum, warp_sums);
  count = block_sum(count, warp_sums);
  if (threadIdx.x == 0) *loss = (float)(sum / fmax(count, 1.));
}

// The parts of dx joined, scaled and rounded; rows that do not count are zero.
template <typename IO>
__global__ void __launch_bounds__(256) join_dx_kernel(const float* acc, int splits, int64_t split_stride, int pitch, int rows, int cols,
                                                      const float* alpha, const void* targets, int bits, int64_t ignore, int classes, IO* dx,
                                                      int64_t stride, const uint32_t* status) {
  wait_for_kernel_before();
  const float a = (*status & VL_TIMEOUT) ? __uint_as_float(0x7fc00000u) : *alpha;
  for (int64_t row = blockIdx.y; row < rows; row += gridDim.y) {
    const bool on = target_of(targets, bits, ignore, classes, (int)row) >= 0;
    for (int c = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 4; c < cols; c += (int)(gridDim.x * blockDim.x) * 4) {
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int s = 0; s < splits; ++s) {
        const float4 o = *reinterpret_cast<const float4*>(acc + s * split_stride + row * pitch + c);
        f = make_float4(f.x + o.x, f.y + o.y, f.z + o.z, f.w + o.w);
      }
      const float v[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (c + j < cols) dx[row * stride + c + j] = from_f32<IO>(on ? v[j] * a : 0.f);
    }
  }
}

// ---- a few rows (scoring the last position of a sequence) ----------------------------------------------------------
// Up to FEW_ROWS rows the forward pass is one pass over w at HBM speed: plain fp32 arithmetic on what is loaded, every
// block a share of the classes.  (256 x 256 tiles would be nearly empty, and a wave and a half of them leaves SMs idle: 1 x
// 1024 x 32000 bf16 took 33 us with both kernels behind it.)
constexpr int FEW_ROWS = 4, FEW_BLOCKS = 148 * 4, FEW_WARPS = 8;
constexpr int FEW_VALUES = 7168;      // rows (as many as a kernel takes) x dim, as fp32 in shared memory

struct FewParams {
  const void *x, *w, *targets;
  int64_t x_stride, w_stride, ignore;
  int rows, dim, classes, bits;
  float z_scale;
  float2* partial;      // [gridDim.x][rows]
  float* target_z;
};
template <typename IO, int R> __device__ __forceinline__ void few_targets(const FewParams& p, int (&target)[R]) {
#pragma unroll
  for (int r = 0; r < R; ++r) target[r] = r < p.rows ? target_of(p.targets, p.bits, p.ignore, p.classes, r) : -1;
}
// The block's partial sums: those of its warps joined.
template <int R> __device__ __forceinline__ void few_finish(const FewParams& p, const float2 (&v)[R], float2 (*s_part)[R]) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  __syncthreads();
  if (lane == 0)
#pragma unroll
    for (int r = 0; r < R; ++r) s_part[warp][r] = v[r];
  __syncthreads();
  if (threadIdx.x < p.rows) {
    float2 t = s_part[0][threadIdx.x];
    for (int q = 1; q < FEW_WARPS; ++q) t = join_sums(t, s_part[q][threadIdx.x]);
    p.partial[(int64_t)blockIdx.x * p.rows + threadIdx.x] = t;
  }
}
template <typename IO> struct EightValues;
template <> struct EightValues<float> {
  float4 a, b;
  __device__ void get(float (&v)[8]) const { v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w; }
};
template <typename IO> struct alignas(16) EightHalfValues {
  typename Pair<IO>::raw q[4];
  __device__ void get(float (&v)[8]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = to_f32(q[i]);
      v[2 * i] = f.x, v[2 * i + 1] = f.y;
    }
  }
};
template <> struct EightValues<__nv_bfloat16> : EightHalfValues<__nv_bfloat16> {};
template <> struct EightValues<__half> : EightHalfValues<__half> {};

// w by class: a warp takes a run of classes, four at a time; its lanes share the features.  VEC: eight features per load
// (dim a multiple of 8, rows aligned to 16 bytes).
template <typename IO, int R, bool VEC> __global__ void __launch_bounds__(32 * FEW_WARPS) few_rows_by_class_kernel(const FewParams p) {
  let_next_kernel_start();
  extern __shared__ __align__(16) float s_x[];   // VEC: [R][2][dim / 8] float4, the halves of eight features apart; else [R][dim]
  __shared__ float2 s_part[FEW_WARPS][R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int r = 0; r < R; ++r)
    for (int d = threadIdx.x; d < p.dim; d += blockDim.x)
      s_x[r * p.dim + (VEC ? (d / 4 % 2) * (p.dim / 2) + d / 8 * 4 + d % 4 : d)] = r < p.rows ? to_f32(((const IO*)p.x)[r * p.x_stride + d]) : 0.f;
  __syncthreads();
  int target[R];
  few_targets<IO, R>(p, target);
  float2 sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) sum[r] = make_float2(-INFINITY, 0.f);
  const int64_t n = (int64_t)gridDim.x * FEW_WARPS, id = (int64_t)blockIdx.x * FEW_WARPS + warp;
  const int last = (int)(p.classes * (id + 1) / n);
  for (int v0 = (int)(p.classes * id / n); v0 < last; v0 += 4) {
    const IO* row[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) row[j] = (const IO*)p.w + min(v0 + j, last - 1) * p.w_stride;
    float acc[4][R] = {};
    if (VEC) {
      auto add = [&](const EightValues<IO> (&q)[4], int d) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const float4 xa = *reinterpret_cast<const float4*>(s_x + r * p.dim + d / 2);
          const float4 xb = *reinterpret_cast<const float4*>(s_x + r * p.dim + p.dim / 2 + d / 2);
          const float xs[8] = {xa.x, xa.y, xa.z, xa.w, xb.x, xb.y, xb.z, xb.w};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            float f[8];
            q[j].get(f);
#pragma unroll
            for (int k = 0; k < 8; ++k) acc[j][r] = fmaf(f[k], xs[k], acc[j][r]);
          }
        }
      };
      for (int d = lane * 8; d < p.dim; d += 512) {   // eight loads in flight per lane
        const bool two = d + 256 < p.dim;
        EightValues<IO> q[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int j = 0; j < 4; ++j) q[h][j] = *reinterpret_cast<const EightValues<IO>*>(row[j] + (h && two ? d + 256 : d));
        add(q[0], d);
        if (two) add(q[1], d + 256);
      }
    } else {
#pragma unroll 4
      for (int d = lane; d < p.dim; d += 32) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float f = to_f32(row[j][d]);
#pragma unroll
          for (int r = 0; r < R; ++r) acc[j][r] = fmaf(f, s_x[r * p.dim + d], acc[j][r]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (v0 + j >= last) break;
#pragma unroll
      for (int r = 0; r < R; ++r) {
        float z = acc[j][r];
#pragma unroll
        for (int o = 16; o > 0; o /= 2) z += __shfl_xor_sync(0xffffffffu, z, o);
        z *= p.z_scale;
        if (lane == 0 && target[r] == v0 + j) p.target_z[r] = z;
        sum[r] = join_sums(sum[r], make_float2(z, z == -INFINITY ? 0.f : 1.f));
      }
    }
  }
  few_finish<R>(p, sum, s_part);
}
// w by feature: a block takes 128 classes, four per lane; its warps share the features.
template <typename IO, int R> __global__ void __launch_bounds__(32 * FEW_WARPS) few_rows_by_feature_kernel(const FewParams p) {
  let_next_kernel_start();
  extern __shared__ __align__(16) float s_x[];   // [R][dim]
  __shared__ float s_acc[FEW_WARPS][R][128];
  __shared__ float2 s_part[FEW_WARPS][R];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int r = 0; r < R; ++r)
    for (int d = threadIdx.x; d < p.dim; d += blockDim.x) s_x[r * p.dim + d] = r < p.rows ? to_f32(((const IO*)p.x)[r * p.x_stride + d]) : 0.f;
  __syncthreads();
  int target[R];
  few_targets<IO, R>(p, target);
  const int v0 = blockIdx.x * 128;
  float acc[4][R] = {};
#pragma unroll 8
  for (int d = warp; d < p.dim; d += FEW_WARPS) {
    const IO* const row = (const IO*)p.w + d * p.w_stride;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float f = to_f32(row[min(v0 + 32 * j + lane, p.classes - 1)]);
#pragma unroll
      for (int r = 0; r < R; ++r) acc[j][r] = fmaf(f, s_x[r * p.dim + d], acc[j][r]);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int r = 0; r < R; ++r) s_acc[warp][r][32 * j + lane] = acc[j][r];
  __syncthreads();
  float2 sum[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    sum[r] = make_float2(-INFINITY, 0.f);
    const int c = warp * 16 + lane % 16, v = v0 + c;   // 16 classes per warp
    if (lane < 16 && v < p.classes) {
      float z = 0.f;
#pragma unroll
      for (int q = 0; q < FEW_WARPS; ++q) z += s_acc[q][r][c];
      z *= p.z_scale;
      if (target[r] == v) p.target_z[r] = z;
      sum[r] = make_float2(z, z == -INFINITY ? 0.f : 1.f);
    }
#pragma unroll
    for (int o = 16; o > 0; o /= 2)
      sum[r] = join_sums(sum[r], make_float2(__shfl_xor_sync(0xffffffffu, sum[r].x, o), __shfl_xor_sync(0xffffffffu, sum[r].y, o)));
  }
  few_finish<R>(p, sum, s_part);
}

// One block: the blocks' partial sums of a few rows to the rows' losses and their mean; lanes across the parts.
__global__ void __launch_bounds__(1024) few_loss_kernel(const float2* partial, int parts, const float* target_z, int rows, const void* targets,
                                                        int bits, int64_t ignore, int classes, float* lse, float* row_out, float* loss) {
  __shared__ float2 s_part[32];
  wait_for_kernel_before();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  double sum = 0.;
  int count = 0;
  for (int row = 0; row < rows; ++row) {
    float2 v = make_float2(-INFINITY, 0.f);
    for (int t = threadIdx.x; t < parts; t += blockDim.x) v = join_sums(v, partial[(int64_t)t * rows + row]);
#pragma unroll
    for (int o = 16; o > 0; o /= 2) v = join_sums(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
    if (lane == 0) s_part[warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = s_part[lane];
#pragma unroll
      for (int o = 16; o > 0; o /= 2) v = join_sums(v, make_float2(__shfl_xor_sync(0xffffffffu, v.x, o), __shfl_xor_sync(0xffffffffu, v.y, o)));
      const int target = target_of(targets, bits, ignore, classes, row);
      const double exact = log_sum(v);
      float l = (float)exact, out = (float)(exact - (target >= 0 ? (double)target_z[row] * 0.69314718055994530942 : 0.));
      if (target < 0) l = 0.f, out = target == -1 ? 0.f : __uint_as_float(0x7fc00000u);
      sum += out;
      count += target >= 0;
      if (lane == 0) {
        lse[row] = l;
        if (row_out) row_out[row] = out;
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) *loss = (float)(sum / (double)max(count, 1));
}

// ---- host --------------------------------------------------------------------------------------------------------
size_t align_up(size_t v) { return (v + 255) / 256 * 256; }
int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }
int64_t round_up(int64_t a, int64_t b) { return (a + b - 1) / b * b; }

// Pairs of SMs of the current device.
int sm_pairs() {
  static std::mutex mutex;
  static int known[64] = {};
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) { cudaGetLastError(); return 0; }
  std::lock_guard<std::mutex> lock(mutex);
  if (dev < 64 && known[dev]) return known[dev];
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) { cudaGetLastError(); return 0; }
  if (dev < 64) known[dev] = sms / 2;
  return sms / 2;
}

struct Operand {           // how a matrix of rows x cols is handed to the products
  bool staged;             // copied to the workspace first
  int planes;
  int64_t pitch, plane;    // in values
  size_t offset, bytes;    // in the workspace, if staged
};
struct Layout {
  Operand x, w;
  size_t status, alpha, partial, target_z, row_loss, dz, acc, total;
  int piece;               // classes per piece of the backward pass
  int64_t dz_pitch, dz_plane;
  int splits, acc_pitch;
  int64_t acc_split;
};

bool usable_directly(const void* p, int64_t stride, int dtype) {
  return dtype != SNN_DTYPE_FP32 && (uintptr_t)p % 16 == 0 && stride % 8 == 0;
}
// Parts of the contraction of dx: as many as fill the device best, in whole waves, each at least 8 k-blocks deep.
int dx_splits(int tiles, int kblocks, int pairs) {
  int best = 1;
  double best_cost = 1e30;
  for (int s = 1; s <= MAX_SPLITS && (s == 1 || kblocks / s >= 8); ++s) {
    const double cost = ceil_div((int64_t)tiles * s, pairs) / (double)s + 0.02 * s;   // waves of full depth, and the cost of joining
    if (cost < best_cost) best_cost = cost, best = s;
  }
  return best;
}
int few_kernel_rows(int rows) { return rows <= 2 ? rows : 4; }
bool few_rows(const snn_vocab_loss_args* a) { return a->rows > 0 && a->rows <= FEW_ROWS && (int64_t)few_kernel_rows(a->rows) * a->dim <= FEW_VALUES; }
int few_blocks(const snn_vocab_loss_args* a) {
  return a->w_layout == SNN_W_BY_CLASS ? std::min(FEW_BLOCKS, ceil_div(a->classes, 4 * FEW_WARPS)) : ceil_div(a->classes, 128);
}
Layout layout_of(const snn_vocab_loss_args* a, bool backward, int pairs) {
  Layout l{};
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes); return o; };
  const int planes = a->dtype == SNN_DTYPE_FP32 ? 3 : 1;
  auto operand = [&](const void* p, int64_t stride, int rows, int cols, bool always) {
    Operand o{};
    o.planes = planes;
    o.staged = always || !usable_directly(p, rows == 1 ? 0 : stride, a->dtype);
    o.pitch = o.staged || rows == 1 ? round_up(cols, 8) : stride;   // (the stride of a single row means nothing)
    o.plane = o.pitch * rows;
    if (o.staged) {
      o.bytes = (size_t)planes * o.plane * 2;
      o.offset = take(o.bytes);
    }
    return o;
  };
  l.status = take(256);
  l.alpha = l.status + 128;
  const bool by_class = a->w_layout == SNN_W_BY_CLASS;
  if (backward || !few_rows(a)) l.x = operand(a->x, a->x_stride, a->rows, a->dim, backward);
  if (backward || !few_rows(a)) l.w = operand(a->w, a->w_stride, by_class ? a->classes : a->dim, by_class ? a->dim : a->classes, false);
  if (!backward) {
    l.partial = take(sizeof(float2) * (size_t)a->rows * (few_rows(a) ? few_blocks(a) : 2 * ceil_div(a->classes, UM_TILE)));
    l.target_z = take(sizeof(float) * (size_t)a->rows);
    l.row_loss = take(sizeof(float) * (size_t)a->rows);
  } else {
    const int64_t fit = (int64_t)(PIECE_BYTES / (2 * (size_t)planes * std::max(a->rows, 1))) / UM_TILE * UM_TILE;
    l.piece = (int)std::min<int64_t>(std::max<int64_t>(fit, UM_TILE), round_up(a->classes, UM_TILE));
    // pieces of equal width
    l.piece = (int)round_up(ceil_div(a->classes, ceil_div(a->classes, l.piece)), UM_TILE);
    l.dz_pitch = l.piece;
    l.dz_plane = l.dz_pitch * a->rows;
    l.dz = take((size_t)planes * l.dz_plane * 2);
    l.splits = dx_splits(ceil_div(a->rows, UM_TILE) * ceil_div(a->dim, UM_TILE), l.piece / UM_KB, std::max(pairs, 1));
    l.acc_pitch = (int)round_up(a->dim, 4);
    l.acc_split = (int64_t)l.acc_pitch * a->rows;
    l.acc = take(sizeof(float) * (size_t)l.acc_split * l.splits);
  }
  l.total = at;
  return l;
}

snn_status check(const snn_vocab_loss_args* a) {
  constexpr int LIMIT = 1 << 30;
  if (!a || a->rows < 0 || a->dim < 1 || a->classes < 1 || a->rows >= LIMIT || a->dim >= LIMIT || a->classes >= LIMIT) return SNN_ERR_INVALID_ARG;
  if (a->dtype < SNN_DTYPE_FP32 || a->dtype > SNN_DTYPE_FP16) return SNN_ERR_INVALID_ARG;
  if (a->w_layout != SNN_W_BY_FEATURE && a->w_layout != SNN_W_BY_CLASS) return SNN_ERR_INVALID_ARG;
  if (a->target_bits != 32 && a->target_bits != 64) return SNN_ERR_INVALID_ARG;
  if (!(std::fabs(a->scale * LOG2E) < INFINITY)) return SNN_ERR_INVALID_ARG;   // (as it multiplies the logits)
  const int64_t w_cols = a->w_layout == SNN_W_BY_CLASS ? a->dim : a->classes, w_rows = a->w_layout == SNN_W_BY_CLASS ? a->classes : a->dim;
  if ((a->rows > 1 && a->x_stride < a->dim) || (w_rows > 1 && a->w_stride < w_cols)) return SNN_ERR_INVALID_ARG;
  if (!a->w || (a->rows > 0 && (!a->x || !a->targets))) return SNN_ERR_INVALID_ARG;
  return SNN_OK;
}
bool is_bf16(int dtype) { return dtype != SNN_DTYPE_FP16; }   // (fp32: bf16 planes)

// Launches a kernel; `behind` another one of the same call.
template <typename... P, typename... A>
snn_status launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, cudaStream_t stream, bool behind, const A&... args) {
  cudaLaunchConfig_t cfg{};
  cudaLaunchAttribute at{};
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = grid;
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cfg.attrs = &at;
  cfg.numAttrs = behind ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, P(args)...) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
}
template <int EPI, bool A_MN, bool B_MN, int WARPS, bool RUNS> snn_status launch_one(const ProductParams& p, int pairs, cudaStream_t stream) {
  const auto kernel = product_kernel<EPI, A_MN, B_MN, WARPS, RUNS>;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VL_SMEM) != cudaSuccess) return cudaGetLastError(), SNN_ERR_CUDA;
  const int64_t units = (int64_t)p.tiles_m * p.tiles_n * p.splits;
  if (units > INT32_MAX / 2) return SNN_ERR_UNSUPPORTED;
  return launch(kernel, dim3(2 * (unsigned)std::min<int64_t>(units, pairs)), 32 * (2 + WARPS), VL_SMEM, stream, p.behind, p);
}
bool eight_warps(const ProductParams& p) { return p.planes > 1 || p.kblocks < VL_SHORT; }
template <int EPI, bool A_MN, bool B_MN> snn_status launch_product(const ProductParams& p, int pairs, cudaStream_t stream) {
  if (p.planes > 1) return launch_one<EPI, A_MN, B_MN, 8, true>(p, pairs, stream);
  if constexpr (EPI == STATS || EPI == GRAD)
    if (eight_warps(p)) return launch_one<EPI, A_MN, B_MN, 8, false>(p, pairs, stream);
  return launch_one<EPI, A_MN, B_MN, 4, false>(p, pairs, stream);
}
// z products: B is w, by class (K-major) or by feature
template <int EPI> snn_status launch_z(const ProductParams& p, bool by_class, int pairs, cudaStream_t stream) {
  return by_class ? launch_product<EPI, false, false>(p, pairs, stream) : launch_product<EPI, false, true>(p, pairs, stream);
}

struct WaitTest {   // of snn_selftest_vocab_loss_wait
  int kernel, unit;
  bool quits;
  uint32_t polls;
};
struct Call {
  const snn_vocab_loss_args* a;
  const WaitTest* test;
  Layout l;
  char* ws;
  cudaStream_t stream;
  int pairs;
  uint32_t* status() const { return (uint32_t*)(ws + l.status); }
  float* alpha() const { return (float*)(ws + l.alpha); }

  snn_status begin(bool backward, void* s) {
    stream = (cudaStream_t)s;
    pairs = sm_pairs();
    if (pairs < 1) return SNN_ERR_CUDA;
    l = layout_of(a, backward, pairs);
    if (!a->workspace || (uintptr_t)a->workspace % 256 != 0) return SNN_ERR_INVALID_ARG;
    if (a->workspace_bytes < l.total) return SNN_ERR_WORKSPACE_TOO_SMALL;
    ws = (char*)a->workspace;
    return SNN_OK;   // (the status is cleared by the staging kernel)
  }
  // with `factor`, for the backward pass: alpha and the status as well
  snn_status stage_operands(const float* factor) const {
    const bool by_class = a->w_layout == SNN_W_BY_CLASS;
    StageParams p{};
    p.targets = a->targets; p.bits = a->target_bits; p.ignore = a->ignore_index; p.classes = a->classes;
    if (l.x.staged) p.job[0] = {a->x, a->x_stride, a->rows, a->dim, (uint16_t*)(ws + l.x.offset), l.x.pitch, l.x.plane, true};
    if (l.w.staged)
      p.job[1] = {a->w, a->w_stride, by_class ? a->classes : a->dim, by_class ? a->dim : a->classes, (uint16_t*)(ws + l.w.offset), l.w.pitch, l.w.plane, false};
    int64_t work = 0;
    for (const StageJob& j : p.job) work = std::max(work, j.rows * (j.pitch / STAGE_COLS + 1));
    if (factor) {
      p.alpha = alpha(); p.factor = *factor; p.dloss = a->dloss_device; p.status = status(); p.rows = a->rows;
      work = std::max<int64_t>(work, 1);
    }
    if (work == 0) return SNN_OK;
    const dim3 grid((unsigned)std::min<int64_t>(work, 148 * 8), factor ? 3 : 2);
    if (a->dtype == SNN_DTYPE_FP32) return launch(stage_kernel<float>, grid, 256, 0, stream, false, p);
    return launch(stage_kernel<__half>, grid, 256, 0, stream, false, p);   // 16 bits are copied, whatever they mean
  }
  const void* data(const Operand& o, const void* direct) const { return o.staged ? ws + o.offset : direct; }
  bool map(CUtensorMap* m, const Operand& o, const void* direct, int rows, int cols, bool mn_major) const {
    return make_tensor_map_16bit(m, data(o, direct), is_bf16(a->dtype), cols, rows, o.planes, o.pitch, o.plane, mn_major ? UM_KB : UM_HALF);
  }
  // partial sums of `tiles` parts of the vocabulary to the losses
  snn_status row_losses(const float2* partial, int tiles, const float* target_z) const {
    float* const row_loss = (float*)(ws + l.row_loss);
    const bool one = a->rows <= 32;
    const snn_status st = launch(row_loss_kernel, dim3(ceil_div(a->rows, 32)), 1024, 0, stream, true, partial, tiles, target_z, a->rows, a->targets,
                                 a->target_bits, a->ignore_index, a->classes, a->lse, row_loss, a->row_loss, one ? a->loss : nullptr);
    if (st != SNN_OK || one) return st;
    return launch(mean_kernel, dim3(1), 1024, 0, stream, true, row_loss, a->rows, a->targets, a->target_bits, a->ignore_index, a->classes, a->loss);
  }
  ProductParams base() const {
    ProductParams p{};
    p.bf16 = is_bf16(a->dtype);
    p.splits = 1;
    p.planes = l.x.planes;
    // fp32: (plane of a, plane of b) = (2, 0), (0, 2), (1, 1), (1, 0), (0, 1), (0, 0), plane 0 the leading part: the small products first
    p.n_pairs = p.planes == 3 ? 6 : 1;
    p.pair_a = p.planes == 3 ? 0x001102u : 0u;
    p.pair_b = p.planes == 3 ? 0x010120u : 0u;
    p.targets = a->targets; p.target_bits = a->target_bits; p.ignore_index = a->ignore_index; p.classes = a->classes;
    p.z_scale = a->scale * LOG2E;
    p.status = status();
    p.behind = true;
    p.polls = MBAR_WAIT_LIMIT;
    p.loads_end = p.quits_at = INT32_MAX;
    return p;
  }
  // the self-test's limits for the call's kernel of this number
  void limit(ProductParams& p, int kernel) const {
    if (!test || test->kernel != kernel) return;
    p.polls = test->polls;
    (test->quits ? p.quits_at : p.loads_end) = test->unit;
  }
};

// The forward pass of a few rows.
template <typename IO, int R> void launch_few(const Call& c, const FewParams& p) {
  const snn_vocab_loss_args* a = c.a;
  const unsigned blocks = (unsigned)few_blocks(a);
  const size_t smem = sizeof(float) * R * a->dim;   // at most 28 KB
  if (a->w_layout != SNN_W_BY_CLASS) few_rows_by_feature_kernel<IO, R><<<blocks, 32 * FEW_WARPS, smem, c.stream>>>(p);
  else if (a->dim % 8 == 0 && (uintptr_t)a->w % 16 == 0 && a->w_stride % 8 == 0) few_rows_by_class_kernel<IO, R, true><<<blocks, 32 * FEW_WARPS, smem, c.stream>>>(p);
  else few_rows_by_class_kernel<IO, R, false><<<blocks, 32 * FEW_WARPS, smem, c.stream>>>(p);
}
template <typename IO> snn_status forward_few(const Call& c) {
  const snn_vocab_loss_args* a = c.a;
  FewParams p{a->x, a->w, a->targets, a->x_stride, a->w_stride, a->ignore_index, a->rows, a->dim, a->classes, a->target_bits, a->scale * LOG2E,
              (float2*)(c.ws + c.l.partial), (float*)(c.ws + c.l.target_z)};
  if (a->rows == 1) launch_few<IO, 1>(c, p);
  else if (a->rows == 2) launch_few<IO, 2>(c, p);
  else launch_few<IO, 4>(c, p);
  if (cudaGetLastError() != cudaSuccess) return SNN_ERR_CUDA;
  return launch(few_loss_kernel, dim3(1), 1024, 0, c.stream, true, p.partial, few_blocks(a), p.target_z, a->rows, a->targets, a->target_bits,
                a->ignore_index, a->classes, a->lse, a->row_loss, a->loss);
}

#define VL_TRY(expr)                            \
  do {                                          \
    const snn_status st_ = (expr);              \
    if (st_ != SNN_OK) return st_;              \
  } while (0)

}  // namespace

extern "C" snn_status snn_vocab_loss_workspace(const snn_vocab_loss_args* a, int32_t backward, size_t* bytes) {
  VL_TRY(check(a));
  if (!bytes) return SNN_ERR_INVALID_ARG;
  int pairs = sm_pairs();
  *bytes = layout_of(a, backward != 0, pairs < 1 ? 74 : pairs).total;
  return SNN_OK;
}

namespace {
snn_status forward(const snn_vocab_loss_args* a, const WaitTest* test, void* stream) {
  VL_TRY(check(a));
  if (!a->loss || (a->rows > 0 && !a->lse)) return SNN_ERR_INVALID_ARG;
  Call c{a, test};
  VL_TRY(c.begin(false, stream));
  if (a->rows == 0) return cudaMemsetAsync(a->loss, 0, 4, c.stream) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
  if (few_rows(a))
    return a->dtype == SNN_DTYPE_FP32   ? forward_few<float>(c)
           : a->dtype == SNN_DTYPE_BF16 ? forward_few<__nv_bfloat16>(c)
                                        : forward_few<__half>(c);
  const bool by_class = a->w_layout == SNN_W_BY_CLASS;
  const int w_rows = by_class ? a->classes : a->dim, w_cols = by_class ? a->dim : a->classes;
  VL_TRY(c.stage_operands(nullptr));
  ProductParams p = c.base();
  p.behind = c.l.x.staged || c.l.w.staged;
  p.status = nullptr;   // (a wait that ran out shows in the losses)
  if (!c.map(&p.a, c.l.x, a->x, a->rows, a->dim, false) || !c.map(&p.b, c.l.w, a->w, w_rows, w_cols, !by_class)) return SNN_ERR_CUDA;
  p.tiles_m = ceil_div(a->rows, UM_TILE);
  p.tiles_n = ceil_div(a->classes, UM_TILE);
  p.kblocks = ceil_div(a->dim, UM_KB);
  p.m = a->rows;
  p.n = a->classes;
  p.partial = (float2*)(c.ws + c.l.partial);
  p.target_z = (float*)(c.ws + c.l.target_z);
  c.limit(p, 0);
  VL_TRY(launch_z<STATS>(p, by_class, c.pairs, c.stream));
  return c.row_losses(p.partial, (eight_warps(p) ? 2 : 1) * p.tiles_n, p.target_z);
}

snn_status backward(const snn_vocab_loss_args* a, const WaitTest* test, void* stream) {
  VL_TRY(check(a));
  const bool by_class = a->w_layout == SNN_W_BY_CLASS;
  const int w_rows = by_class ? a->classes : a->dim, w_cols = by_class ? a->dim : a->classes;
  if (!a->dw || (a->rows > 0 && (!a->dx || !a->lse))) return SNN_ERR_INVALID_ARG;
  if ((a->rows > 1 && a->dx_stride < a->dim) || (w_rows > 1 && a->dw_stride < w_cols)) return SNN_ERR_INVALID_ARG;
  Call c{a, test};
  VL_TRY(c.begin(true, stream));
  const size_t size = a->dtype == SNN_DTYPE_FP32 ? 4 : 2;
  if (a->rows == 0) {   // (the stride of a single row means nothing)
    const size_t width = w_cols * size, pitch = w_rows > 1 ? a->dw_stride * size : width;
    return cudaMemset2DAsync(a->dw, pitch, 0, width, w_rows, c.stream) == cudaSuccess ? SNN_OK : (cudaGetLastError(), SNN_ERR_CUDA);
  }
  const Layout& l = c.l;
  const ProductParams base = c.base();
  const float dz_unit = dz_unit_of(a->dtype, a->rows), factor = a->dloss * a->scale / dz_unit;
  VL_TRY(c.stage_operands(&factor));
  CUtensorMap x_k, x_mn, w_z, w_dx, dz_k, dz_mn;   // as operands that are contiguous along the contraction, and across it
  bool ok = c.map(&x_k, l.x, a->x, a->rows, a->dim, false) && c.map(&x_mn, l.x, a->x, a->rows, a->dim, true);
  ok = ok && c.map(&w_z, l.w, a->w, w_rows, w_cols, !by_class) && c.map(&w_dx, l.w, a->w, w_rows, w_cols, by_class);
  for (int v0 = 0; v0 < a->classes; v0 += l.piece) {
    const int width = std::min(l.piece, a->classes - v0);
    // (the maps end at the piece's width: columns beyond it arrive as zeros and are not stored)
    ok = ok && make_tensor_map_16bit(&dz_k, c.ws + l.dz, base.bf16, width, a->rows, base.planes, l.dz_pitch, l.dz_plane, UM_HALF) &&
         make_tensor_map_16bit(&dz_mn, c.ws + l.dz, base.bf16, width, a->rows, base.planes, l.dz_pitch, l.dz_plane, UM_KB);
    if (!ok) return SNN_ERR_CUDA;
    ProductParams p = base;   // dz of the piece
    p.a = x_k; p.b = w_z; p.out = dz_k;
    p.tiles_m = ceil_div(a->rows, UM_TILE); p.tiles_n = ceil_div(width, UM_TILE); p.kblocks = ceil_div(a->dim, UM_KB);
    p.m = a->rows; p.n = width; p.b0 = v0;
    p.lse = a->lse;
    p.dz_unit = dz_unit;
    c.limit(p, 0);
    VL_TRY(launch_z<GRAD>(p, by_class, c.pairs, c.stream));
    p = base;                 // dx += dz w^T
    p.a = dz_k; p.b = w_dx;
    p.tiles_m = ceil_div(a->rows, UM_TILE); p.tiles_n = ceil_div(a->dim, UM_TILE); p.kblocks = ceil_div(width, UM_KB);
    p.splits = std::min(l.splits, p.kblocks);
    p.bk0 = v0;
    p.m = a->rows; p.n = a->dim;
    p.acc = (float*)(c.ws + l.acc); p.acc_pitch = l.acc_pitch; p.acc_split = l.acc_split; p.accumulate = v0 > 0;
    c.limit(p, 1);
    VL_TRY((by_class ? launch_product<DX, false, true>(p, c.pairs, c.stream) : launch_product<DX, false, false>(p, c.pairs, c.stream)));
    p = base;                 // the piece's part of dw
    p.kblocks = ceil_div(a->rows, UM_KB);
    p.alpha = c.alpha();
    p.dw_stride = a->dw_stride; p.dw_dtype = a->dtype;
    if (by_class) {           // rows are classes
      p.a = dz_mn; p.b = x_mn;
      p.m = width; p.n = a->dim;
      p.dw = (char*)a->dw + (size_t)v0 * a->dw_stride * size;
    } else {
      p.a = x_mn; p.b = dz_mn;
      p.m = a->dim; p.n = width;
      p.dw = (char*)a->dw + (size_t)v0 * size;
    }
    p.dw_vector = (uintptr_t)p.dw % 16 == 0 && p.dw_stride * (int64_t)size % 16 == 0;
    p.tiles_m = ceil_div(p.m, UM_TILE); p.tiles_n = ceil_div(p.n, UM_TILE);
    c.limit(p, 2);
    VL_TRY((launch_product<DW, true, true>(p, c.pairs, c.stream)));
  }
  const int splits = std::min(l.splits, ceil_div(std::min(l.piece, a->classes), UM_KB));
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(a->dim, 1024), 64), (unsigned)std::min(a->rows, 16384));
  auto join = [&](auto io) {
    using IO = decltype(io);
    return launch(join_dx_kernel<IO>, grid, 256, 0, c.stream, true, (const float*)(c.ws + l.acc), splits, l.acc_split, l.acc_pitch, a->rows, a->dim,
                  c.alpha(), a->targets, a->target_bits, a->ignore_index, a->classes, (IO*)a->dx, a->dx_stride, c.status());
  };
  return a->dtype == SNN_DTYPE_FP32 ? join(float()) : a->dtype == SNN_DTYPE_BF16 ? join(__nv_bfloat16()) : join(__half());
}
}  // namespace

extern "C" snn_status snn_vocab_loss_forward(const snn_vocab_loss_args* a, void* stream) { return forward(a, nullptr, stream); }
extern "C" snn_status snn_vocab_loss_backward(const snn_vocab_loss_args* a, void* stream) { return backward(a, nullptr, stream); }

extern "C" snn_status snn_selftest_vocab_loss_wait(const snn_vocab_loss_args* a, int32_t is_backward, int32_t kernel, int32_t unit, int32_t quits,
                                                   uint32_t poll_limit, void* stream) {
  if (kernel < 0 || kernel > (is_backward ? 2 : 0) || unit < 0 || poll_limit == 0 || poll_limit > MBAR_WAIT_LIMIT) return SNN_ERR_INVALID_ARG;
  if (!WAIT_TESTS) return SNN_ERR_UNSUPPORTED;
  const WaitTest test{kernel, unit, quits != 0, poll_limit};
  return is_backward ? backward(a, &test, stream) : forward(a, &test, stream);
}
