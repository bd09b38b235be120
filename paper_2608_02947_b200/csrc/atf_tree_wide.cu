// The kernel of atf_decode_tree for many rows: 128 rows (nodes x heads of a KV head) a block, on the fifth-generation tensor cores.
//
// A step is 64 keys.  S = Q K^T (128 x 64, tcgen05, both operands in shared memory) over the pairs that are live for every row, the
// online softmax with one row a thread (S read from tensor memory, weights written back over it in 16 bits), O += P V
// (tcgen05, P from tensor memory).  The group-major tiles of the cache ARE the 32-byte-swizzled K-major operand: a group of 8 pairs
// is one 16-column step, so the live prefix of a tile is copied and multiplied as it stands; V rows come in 128-byte-swizzled
// boxes, read MN-major.  Codes of 8 bits are turned into f16 operands on the way (exactly; the scale of a key multiplies
// its column of S, that of a value its weight).  Weights are rounded to the type of V, which the product wants: bf16 beside bf16 values,
// f16 beside codes; their sum is that of the unrounded ones, in fp32.
//
// Roles of a block (12 warps, two blocks an SM): 0-3 softmax, 4-7 preparation of the operands: they zero what the window or the length
// leaves out of a step's K and V, or convert the codes; 8 copies, 9 issues the scores, 10 the values' products.  The scores of step
// t + 1 run under step t's softmax; the two blocks of an SM fill each other's waits.
//
// What bounds it: no one pipe.  131072 x 8 heads, 96 rows, e4m3: 133 us (memory would take 32, the exponentials 30, the products 25).  A block
// spends 6 us on Q and the tree, 3 until its first scores, 107 (the longest 121) on its 55 steps, 3 on its sums, two blocks an SM; the join
// is 9.  In a step K's conversion, the scores, the softmax, V's conversion and the product follow one another, and issue slots are 45 % busy.  4 x
// 64 nodes x 32768 in bf16, nothing to convert: 164 us, 576 blocks in two rounds, each 6, 1, 58 (81) and 3.  Blocks of one an SM with steps of
// 128 keys, with the scores in two or three buffers, with the softmax by halves of the keys or by alternate steps, and K's operands a step
// ahead were built and measured: 127 to 191 us where the first took 130, 183 to 222 where the second took 161, 67 to 77 where 8 x 16 nodes x
// 30011 (int8, heads of 64) took 65.  mma.sync with 32 rows a block: 1106 / 2300 / 355 us.
//
// A key's products take the pairs that are live for every row; a (key, pair) term that only some rows keep - where a window ends
// between the nearest and the farthest row of the tree, a few keys a pair - is added to S in tensor memory by the softmax warps.
#include <cmath>

#include "atf_tree.cuh"

namespace {

constexpr int TW_THREADS = 384, TW_KEYS = 64, TW_PREP = 4, TW_PREP_WARPS = 4, TW_PRODUCER = 8, TW_SCORES = 9, TW_VALUES = 10;
// Registers of a thread of the three warpgroups (softmax; operands; copies, both products and a warp that only keeps them company).
constexpr int TW_REGS = 80, TW_REGS_SOFTMAX = 128, TW_REGS_PREP = 80, TW_REGS_REST = 32;
static_assert(TW_REGS_SOFTMAX + TW_REGS_PREP + TW_REGS_REST <= 3 * TW_REGS, "setmaxnreg moves registers within what the block was launched with");
static_assert(TW_REGS_PREP <= TW_REGS && TW_REGS_REST <= TW_REGS && TW_REGS_SOFTMAX >= TW_REGS, "a decrement to more registers than a warp has is an illegal instruction");
constexpr int TW_AHEAD = 4;  // steps that are brought into L2 before the ring has room for them
constexpr int TW_LONE = 4;  // terms of one key that only some rows keep and that are handed to the softmax warps in shared memory
constexpr uint32_t TW_TMEM_COLS = 256;  // S of even steps, of odd steps (64 each, P over them), O (d)

template <int D, int FMT>
struct WideShape {
  static constexpr bool F16 = FMT != ATF_KV_BF16;
  static constexpr int H = D / 2, NG = D / 16, KT = atf_kv_tile_keys(D, !F16), EB = F16 ? 16 : 32;
  static constexpr int QBYTES = TW_ROWS * D * 2;
  static constexpr int KBYTES = TW_KEYS * D * (F16 ? 1 : 2), SCALES = F16 ? 2 * TW_KEYS * 4 : 0;
  static constexpr int KSTAGE = KBYTES + SCALES, VSTAGE = KBYTES;
  static constexpr int ST = F16 ? 2 : 32768 / KBYTES;
  static constexpr int OP = TW_KEYS * D * 2;  // K or V of a step as f16 operands
  static constexpr int K_OFF = QBYTES, V_OFF = K_OFF + ST * KSTAGE, C_OFF = V_OFF + ST * VSTAGE;
  static constexpr int SC_OFF = C_OFF + (F16 ? 2 * OP : 0);            // 8-bit: [2][key scales, value weights][64]
  static constexpr int X_OFF = SC_OFF + (F16 ? 2 * 2 * TW_KEYS * 4 : 0);  // lone terms, see TW_LONE
  static constexpr int XBUFS = ST, XSIZE = TW_KEYS * TW_LONE * 8 + TW_KEYS * 4;
  static constexpr int BAR_OFF = X_OFF + XBUFS * XSIZE;
  static constexpr int SMEM = BAR_OFF + 256 + 1024;
  static_assert(K_OFF % 1024 == 0 && V_OFF % 1024 == 0 && C_OFF % 256 == 0 && (!F16 || OP % 1024 == 0), "operands stand at their swizzle's period");
};

__host__ __device__ constexpr uint32_t wide_idesc(bool f16, int M, int N, int b_mn_major) {
  return (1u << 4) | (f16 ? 0u : (1u << 7) | (1u << 10)) | ((uint32_t)b_mn_major << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}
// K-major operand of 16 columns: rows of 32 bytes, 32-byte swizzle (the halves of rows with bit 2 set trade places).
__device__ __forceinline__ uint64_t desc_sw32(uint32_t addr) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | (1ull << 16) | ((uint64_t)(256 >> 4) << 32) | (1ull << 46) | (6ull << 61);
}
__device__ __forceinline__ void sts128(uint32_t a, uint4 v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void tc_ld4(uint32_t taddr, float (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0, %1, %2, %3}, [%4];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_st4(uint32_t taddr, const float (&r)[4]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x4.b32 [%0], {%1, %2, %3, %4};" ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]) : "memory");
}

__device__ __forceinline__ void tc_ld8(uint32_t taddr, float* r) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t taddr, const float (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"r"(taddr), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]) : "memory");
}
// Behind loads from tensor memory: nothing that uses the values moves in front of the wait.
template <int N>
__device__ __forceinline__ void tc_wait_ld_pin(float (&r)[N]) {
  tc_wait_ld();
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+f"(r[i]));
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ void prefetch_l2(const void* p, uint32_t bytes) {
  asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(p), "r"(bytes) : "memory");
}

// 8-bit, rare: the largest weight times scale of this thread's row (log2), cell by cell.  A function of its own: its code in the loop of the
// softmax costs the steps that do not need it (32 nodes of 131072, e4m3: 132 us, with it in the loop 136).
__device__ __noinline__ float row_top(uint32_t tS, const float* sc, float rs) {
  float top = -INFINITY;
#pragma unroll 1
  for (int c = 0; c < TW_KEYS; c += 8) {
    float x[8];
    tc_ld8(tS + c, x);
    tc_wait_ld_pin(x);
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, x[i] * sc[c + i] * rs + value_log2(sc[TW_KEYS + c + i]));
  }
  return top;
}

// A step of 64 keys: pairs live at its farthest distance, at its nearest key for every row, and there for some row.
struct StepPairs {
  int far, all, any;
  bool plain;  // every row sees every key
  template <int H>
  __device__ __forceinline__ StepPairs(const PairWidths<H>& W, int Wmax, int k0, int L, int dmin, int dmax) {
    const bool committed = k0 + TW_KEYS <= L;
    far = W.live(max(L - k0, 0) + dmax);
    all = W.live(committed ? L + dmax - (k0 + TW_KEYS - 1) : 0);
    any = W.live(committed ? L + dmin - (k0 + TW_KEYS - 1) : 0);
    plain = committed && L + dmax - k0 <= Wmax;
  }
};

template <int D, int FMT>
__global__ void __launch_bounds__(TW_THREADS, 2)
atf_tree_wide(const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams P, const __grid_constant__ AtfTable table) {
  using S = WideShape<D, FMT>;
  constexpr bool F16 = S::F16;
  constexpr int H = S::H, NG = S::NG, KT = S::KT, EB = S::EB, ST = S::ST;
  constexpr uint32_t IDESC_S = wide_idesc(F16, TW_ROWS, TW_KEYS, 0), IDESC_O = wide_idesc(F16, TW_ROWS, D, F16 ? 0 : 1);
  const float kScale = 1.4426950408889634f / sqrtf((float)D);

  extern __shared__ uint8_t dsm_raw[];
  __shared__ int sW[ATF_MAX_PAIRS];
  __shared__ TreeShared<TR_MAX_NODES> tr;
  __shared__ int s_depth[TW_ROWS];
  __shared__ float s_qs[TW_ROWS];
  __shared__ unsigned long long s_bad[ST][2];  // keys of a step (stage of V in bf16, of K in 8 bits) that make a row which sees them NaN
  __shared__ int s_groups[ST];              // groups of 8 pairs that the scores of a stage of K contract
  __shared__ int s_lone[ST];                // the step has terms that only some rows keep
  __shared__ float s_vtop[2];               // 8-bit, of even / odd steps: log2 of the largest scale of a value; -inf where they differ much
  __shared__ uint32_t s_tmem;
  __shared__ int s_near, s_far, s_abort;
  const uint32_t sbase = (smem_u32(dsm_raw) + 1023u) & ~1023u;
  uint8_t* sgen = dsm_raw + (sbase - smem_u32(dsm_raw));
  const uint32_t sQ = sbase, sK = sbase + S::K_OFF, sV = sbase + S::V_OFF, sC = sbase + S::C_OFF, sSc = sbase + S::SC_OFF,
                 bars = sbase + S::BAR_OFF;
  auto bar = [&](int kind, int st) { return bars + 8u * (uint32_t)(kind * ST + st); };
  enum { KFULL, KEMPTY, KREADY, VFULL, VEMPTY, VREADY, OTHERS };
  auto sdone = [&](int i) { return bars + 8u * (uint32_t)(OTHERS * ST + i); };
  auto pready = [&](int i) { return bars + 8u * (uint32_t)(OTHERS * ST + 2 + i); };
  // Even and odd steps have barriers of their own: a wait on one is told the right phase as long as no other than the step two before and
  // the step itself can have completed, and scores t follow product t - 2.
  auto odone = [&](int i) { return bars + 8u * (uint32_t)(OTHERS * ST + 4 + i); };
  auto drained = [&](int i) { return bars + 8u * (uint32_t)(OTHERS * ST + 6 + i); };
  static_assert((OTHERS * ST + 8) * 8 <= 256, "room for the barriers");

  const int split = blockIdx.x, hkv = blockIdx.y / P.rtiles, rt = blockIdx.y % P.rtiles, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = P.G, T = P.T, row0 = rt * TW_ROWS;
  const int64_t grp = (int64_t)b * P.Hkv + hkv;
  if (threadIdx.x < ATF_MAX_PAIRS) sW[threadIdx.x] = table.w[threadIdx.x];
  grid_dependency_launch();
  grid_dependency_wait();
  const int n = P.counts ? min(max(P.counts[b], 0), T) : T;
  const int L = P.lens ? min(max(P.lens[b], 0), P.max_len) : P.len;
  const int rows = min(n * G - row0, TW_ROWS);
  if (rows <= 0) return;  // the same for the whole block
  const int nactive = (rows + 31) / 32;
  if (warp == TW_PREP) {
    tmem_alloc(smem_u32(&s_tmem), TW_TMEM_COLS);
    tmem_relinquish();
  }
  if (threadIdx.x == 0) {
    s_abort = 0;
    s_near = 0x7fffffff;
    s_far = 0;
    for (int st = 0; st < ST; ++st) {
      mbar_init(bar(KFULL, st), 1);
      mbar_init(bar(VFULL, st), 1);
      mbar_init(bar(KEMPTY, st), F16 ? TW_PREP_WARPS : 1);  // the conversion is through with it, or the products are
      mbar_init(bar(VEMPTY, st), F16 ? TW_PREP_WARPS : 1);
      mbar_init(bar(KREADY, st), TW_PREP_WARPS);
      mbar_init(bar(VREADY, st), TW_PREP_WARPS);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(sdone(i), 1);
      mbar_init(pready(i), nactive);
      mbar_init(odone(i), 1);
      mbar_init(drained(i), 1);
    }
    mbar_fence_init();
    fence_proxy_async_smem();
    if (!F16) tma_prefetch_desc(&tmV);
  }
  const int Ltot = L + n;
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  const uint32_t tO = tmem + 2 * TW_KEYS;
  const int Wmax = sW[H - 1];
  const int nsteps = (Ltot + TW_KEYS - 1) / TW_KEYS;
  const int s_first = max(0, L - Wmax) / TW_KEYS + split;  // steps in front of it hold no key that any row reaches
  const int mine = s_first < nsteps ? (nsteps - s_first + P.nsplit - 1) / P.nsplit : 0;
  unsigned int fail_site = 0;
  volatile int* abortp = &s_abort;
  auto bounded_wait = [&](uint32_t bar_, uint32_t parity) { return tr_wait(bar_, parity, abortp); };
  // for a whole warp: all of it goes on or gives up
  auto warp_wait = [&](uint32_t bar_, uint32_t parity) { return __all_sync(0xffffffffu, bounded_wait(bar_, parity)) != 0; };
  const PairWidths<H> W(sW, lane);

  if (warp == TW_PRODUCER) {
    // =============================== copies ===============================
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TW_REGS_REST));
    // They start while the others still read the tree and Q, and so take a row to be as near as rows can be.
    // The bytes of a step stand in L2 some steps before a stage of the ring is free for them.
    auto prefetch = [&](int t) {
      if (t >= mine) return;
      const int k0 = (s_first + t * P.nsplit) * TW_KEYS, kin = k0 % KT;
      const int ngl = (W.live(k0 + TW_KEYS > L ? 0 : L - (k0 + TW_KEYS - 1)) + 7) >> 3;
      const int64_t tile = grp * P.ktiles + k0 / KT;
      if (lane < ngl) prefetch_l2(P.k + tile * 16384 + (lane * KT + kin) * EB, TW_KEYS * EB);
      if (lane == 16) {
        const int keys = min(TW_KEYS, Ltot - k0);
        if (F16) prefetch_l2(P.v + tile * 16384 + kin * D, (uint32_t)((keys + 15) / 16 * 16 * D));
        else prefetch_l2(P.v + ((grp * P.cap + k0) * D) * 2, (uint32_t)(keys * D * 2));
      }
    };
    for (int t = 0; t < TW_AHEAD; ++t) prefetch(t);
    int kissued = 0, vissued = 0;
    for (int t = 0; t < mine; ++t) {
      const int st = t % ST, k0 = (s_first + t * P.nsplit) * TW_KEYS, kin = k0 % KT;
      const int ngl = (W.live(k0 + TW_KEYS > L ? 0 : L - (k0 + TW_KEYS - 1)) + 7) >> 3;
      const int64_t tile = grp * P.ktiles + k0 / KT;
      const uint32_t kd = sK + st * S::KSTAGE, vd = sV + st * S::VSTAGE;
      if (t >= ST && !warp_wait(bar(KEMPTY, st), ((t / ST) - 1) & 1)) { fail_site = 70; break; }
      if (lane == 0) {
        mbar_expect_tx(bar(KFULL, st), (uint32_t)(ngl * TW_KEYS * EB + S::SCALES));
        if (F16) {
          bulk_load_1d(kd + S::KBYTES, P.scales + tile * (2 * KT) + kin, TW_KEYS * 4, bar(KFULL, st));
          bulk_load_1d(kd + S::KBYTES + TW_KEYS * 4, P.scales + tile * (2 * KT) + KT + kin, TW_KEYS * 4, bar(KFULL, st));
        }
        if (KT == TW_KEYS) {
          if (ngl) bulk_load_1d(kd, P.k + tile * 16384, (uint32_t)(ngl * TW_KEYS * EB), bar(KFULL, st));
        } else {
          for (int j = 0; j < ngl; ++j)
            bulk_load_1d(kd + j * TW_KEYS * EB, P.k + tile * 16384 + (j * KT + kin) * EB, TW_KEYS * EB, bar(KFULL, st));
        }
      }
      kissued = t + 1;
      if (t >= ST && !warp_wait(bar(VEMPTY, st), ((t / ST) - 1) & 1)) { fail_site = 71; break; }
      if (lane == 0) {
        const uint32_t vbytes = F16 ? (uint32_t)((min(TW_KEYS, Ltot - k0) + 15) / 16 * 16 * D) : (uint32_t)S::KBYTES;
        mbar_expect_tx(bar(VFULL, st), vbytes);
        if (F16) {
          bulk_load_1d(vd, P.v + tile * 16384 + kin * D, vbytes, bar(VFULL, st));
        } else {
#pragma unroll
          for (int vb = 0; vb < D / 64; ++vb) tma_load_3d(vd + vb * (TW_KEYS * 128), &tmV, bar(VFULL, st), vb * 64, k0, (int)grp);
        }
      }
      vissued = t + 1;
      prefetch(t + TW_AHEAD);
    }
    // no copy is in flight when the block ends, whatever the others gave up
    for (int t = max(0, kissued - ST); t < kissued; ++t)
      if (!mbar_wait(bar(KFULL, t % ST), (t / ST) & 1)) fail_site = 79;
    for (int t = max(0, vissued - ST); t < vissued; ++t)
      if (!mbar_wait(bar(VFULL, t % ST), (t / ST) & 1)) fail_site = 79;
  } else {
    // Q as the 32-byte-swizzled operand: group j of 8 pairs, row, pair p at ((p & 7) 4) ^ (16 where row has bit 2 set)
    const int parent = tree_parent(P, b, n, threadIdx.x);
    stage_rows<D, F16, TW_ROWS, TW_THREADS / 32 - 1, 3>(P, (int64_t)b * P.Hq + hkv * G, row0, rows, warp < TW_PRODUCER ? warp : warp - 1, lane, s_qs,
                                    [&](int rr, int p, uint32_t w) {
                                      *reinterpret_cast<uint32_t*>(sgen + (p >> 3) * (TW_ROWS * 32) + rr * 32 + (((p & 7) * 4) ^ ((rr & 4) << 2))) = w;
                                    });
    const int cur = build_tree<TW_THREADS - 32>(tr, parent, n, threadIdx.x);
    if (warp < nactive) {
      const int dep = tr.depth[cur][(row0 + min((int)threadIdx.x, rows - 1)) / G];
      s_depth[threadIdx.x] = dep;
      const int least = __reduce_min_sync(0xffffffffu, dep), most = __reduce_max_sync(0xffffffffu, dep);
      if (lane == 0) {
        atomicMin(&s_near, least);
        atomicMax(&s_far, most);
      }
    }
    fence_proxy_async_smem();
    group_barrier(TW_THREADS - 32);
    const int dmin = s_near, dmax = s_far;
    if (warp == TW_SCORES) {
      // =============================== S = Q K^T ===============================
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TW_REGS_REST));
      if (lane == 0) {
        const uint64_t dQ = desc_sw32(sQ);
        for (int t = 0; t < mine; ++t) {
          const int st = t % ST;
          // S of step t is written over the weights that the product of step t - 2 reads
          if ((t >= 2 && !bounded_wait(odone(t & 1), ((t - 2) >> 1) & 1)) || !bounded_wait(bar(KREADY, st), (t / ST) & 1)) { fail_site = 72; break; }
          const int ngl = *reinterpret_cast<volatile int*>(&s_groups[st]);
          const uint64_t dK = desc_sw32(F16 ? sC : sK + st * S::KSTAGE);
          const uint32_t tS = tmem + (t & 1) * TW_KEYS;
          tc_fence_after();
#pragma unroll
          for (int j = 0; j < NG; ++j)
            if (j < ngl) tc_mma_ss(tS, dQ + (uint64_t)(j * (TW_ROWS * 32 / 16)), dK + (uint64_t)(j * (TW_KEYS * 32 / 16)), IDESC_S, j > 0 ? 1u : 0u);
          tc_commit(sdone(t & 1));
          if (!F16) tc_commit(bar(KEMPTY, st));
        }
        if (fail_site) {  // products in flight end before tensor memory is given back
          tc_commit(drained(0));
          (void)mbar_wait(drained(0), 0);
        }
      }
    } else if (warp == TW_VALUES) {
      // =============================== O += P V ===============================
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TW_REGS_REST));
      if (lane == 0) {
        for (int t = 0; t < mine; ++t) {
          const int st = t % ST;
          if (!bounded_wait(bar(VREADY, st), (t / ST) & 1) || !bounded_wait(pready(t & 1), (t >> 1) & 1)) { fail_site = 80; break; }
          tc_fence_after();
          const uint64_t dV = F16 ? desc_sw32(sC + S::OP) : make_smem_desc_sw128(sV + st * S::VSTAGE, TW_KEYS * 128, 1024);
#pragma unroll
          for (int i = 0; i < TW_KEYS / 16; ++i)
            tc_mma_ts(tO, tmem + (t & 1) * TW_KEYS + 8 * i, dV + (uint64_t)((F16 ? D * 2 : 128) * i), IDESC_O, t > 0 || i > 0 ? 1u : 0u);
          tc_commit(odone(t & 1));
          if (!F16) tc_commit(bar(VEMPTY, st));
        }
        if (fail_site) {
          tc_commit(drained(1));
          (void)mbar_wait(drained(1), 0);
        }
      }
    } else if (warp > TW_VALUES) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TW_REGS_REST));
    } else if (warp >= TW_PREP) {
      // =============================== operands ===============================
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(TW_REGS_PREP));
      const int pt = threadIdx.x - TW_PREP * 32, i = pt & 63, part = pt >> 6;  // two threads a key
      float vtop = 0.f;  // see atf_tree_tiles
      for (int t = 0; t < mine; ++t) {
        const int st = t % ST, k0 = (s_first + t * P.nsplit) * TW_KEYS, key = k0 + i;
        const uint32_t kr = sK + st * S::KSTAGE, vr = sV + st * S::VSTAGE;
        const StepPairs sp(W, Wmax, k0, L, dmin, dmax);
        const bool plain = sp.plain, lone = sp.any != sp.far;
        int live = sp.far, some = sp.far;  // pairs of this thread's key that every row keeps, that some row keeps
        if (lone) {
          const int place = key < L ? key - L : key < Ltot ? tr.depth[cur][key - L] : 0;
          const int zm = key < Ltot ? dmax - place : 0x7fffffff, zl = key < L ? dmin - place : key < Ltot ? 0 : 0x7fffffff;
          some = pairs_reaching<H>(sW, zl);
          live = pairs_reaching<H>(sW, zm);
        }
        const int ngl = max(1, (sp.all + 7) >> 3);  // with no pair for every row, a group of zeros
        if (!warp_wait(bar(KFULL, st), (t / ST) & 1)) { fail_site = 73; break; }
        // lone terms of this thread's key, in the groups that it works on: the pair as the products take it, and where Q has it with the deepest row that keeps it
        uint2 term[TW_LONE];
        if (lone) {
          const int place = key < L ? key - L : key < Ltot ? tr.depth[cur][key - L] : 0;
#pragma unroll
          for (int e = 0; e < TW_LONE; ++e) {
            const int p = live + e;
            term[e] = make_uint2(0u, 0u);
            if (p < some && ((p >> 3) & 1) == part) {
              const uint32_t kw = F16 ? codes_f16<FMT>((lds32(kr + ((p >> 3) * TW_KEYS + i) * 16 + ((p & 7) >> 1) * 4) >> ((p & 1) * 16)) & 0xffffu)
                                      : lds32(kr + ((p >> 3) * TW_KEYS + i) * 32 + (((p & 7) * 4) ^ ((i & 4) << 2)));
              term[e] = make_uint2(kw, (uint32_t)((p >> 3) * (TW_ROWS * 32) + (p & 7) * 4) | ((uint32_t)(sW[H - 1 - p] + place) << 16));
            }
          }
        }
        auto hand_over = [&](int stage) {
          if (pt == 0) s_lone[stage] = lone;
          if (!lone) return;
          uint8_t* xb = sgen + S::X_OFF + stage * S::XSIZE;
#pragma unroll
          for (int e = 0; e < TW_LONE; ++e)
            if ((((live + e) >> 3) & 1) == part) reinterpret_cast<uint2*>(xb)[e * TW_KEYS + i] = term[e];
          if (part == 0) reinterpret_cast<uint32_t*>(xb + TW_KEYS * TW_LONE * 8)[i] = (uint32_t)(live | (some << 16));
        };
        if (!F16) {
          for (int j = (live >> 3) + (((live >> 3) ^ part) & 1); j < ngl; j += 2) {
            const int keep = live - 8 * j;  // pairs 0 .. keep - 1 of the group stay
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const uint32_t a = kr + (j * TW_KEYS + i) * 32 + ((hf * 16) ^ ((i & 4) << 2));
              if (keep >= 4 * hf + 4) continue;
              uint4 w = lds128(a);
              w.x = keep > 4 * hf ? w.x : 0u;
              w.y = keep > 4 * hf + 1 ? w.y : 0u;
              w.z = keep > 4 * hf + 2 ? w.z : 0u;
              w.w = 0u;
              sts128(a, w);
            }
          }
        } else {
          // the scores of the step before have left the buffer
          if (t > 0 && !warp_wait(sdone((t - 1) & 1), ((t - 1) >> 1) & 1)) { fail_site = 74; break; }
          const uint4* kraw = reinterpret_cast<const uint4*>(sgen + S::K_OFF + st * S::KSTAGE) + i;
          uint8_t* kop = sgen + S::C_OFF + i * 32;
          const int sw = (i & 4) << 2;
#pragma unroll 2
          for (int j = part; j < ngl; j += 2) {
            const uint4 c4 = kraw[j * TW_KEYS];
            const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
            uint32_t w[8];
#pragma unroll
            for (int q = 0; q < 4; ++q) codes4_f16<FMT>(c[q], w[2 * q], w[2 * q + 1]);
            if (8 * j + 8 > live) {
#pragma unroll
              for (int q = 0; q < 8; ++q)
                if (8 * j + q >= live) w[q] = 0u;
            }
            *reinterpret_cast<uint4*>(kop + j * (TW_KEYS * 32) + sw) = make_uint4(w[0], w[1], w[2], w[3]);
            *reinterpret_cast<uint4*>(kop + j * (TW_KEYS * 32) + (16 ^ sw)) = make_uint4(w[4], w[5], w[6], w[7]);
          }
          // scales of the keys; scales of the values (one that is not finite counts for nothing)
          float* sc = reinterpret_cast<float*>(sgen + S::SC_OFF) + (t & 1) * (2 * TW_KEYS);
          const float* raw = reinterpret_cast<const float*>(sgen + S::K_OFF + st * S::KSTAGE + S::KBYTES);
          float x = 0.f, v[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            v[e] = k0 + lane + 32 * e < Ltot ? raw[TW_KEYS + lane + 32 * e] : 0.f;
            x = fmaxf(x, v[e] < 3e38f ? v[e] : 0.f);
          }
          x = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
          const float mine_k = raw[i], even = x * (1.f / TR_V_EVEN);
          float mine_v = key < Ltot ? raw[TW_KEYS + i] : 0.f;
          bool uneven = false;
          if (__builtin_expect(__any_sync(0xffffffffu, even > vtop || (v[0] > 0.f && v[0] < even) || (v[1] > 0.f && v[1] < even)), 0)) {
            // They differ from before or from each other: rows of zeros, whose scale is 1 whatever the others are, do not count.
            if (!warp_wait(bar(VFULL, st), (t / ST) & 1)) { fail_site = 75; break; }
            float least = 3e38f;
            x = 0.f;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t zero = zero_rows<D, FMT>(sgen + S::V_OFF + st * S::VSTAGE + e * (32 * D), lane);
              const bool none = v[e] > 0.f && v[e] < 3e38f && (zero >> lane & 1u) != 0u;  // behind the last slot, what was there before
              uneven |= none;
              if (none) v[e] = 0.f;
              if (e == (i >> 5)) mine_v = v[e];  // lane = i & 31
              x = fmaxf(x, v[e] < 3e38f ? v[e] : 0.f);
              least = fminf(least, v[e] > 0.f ? v[e] : 3e38f);
            }
            x = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
            least = __uint_as_float(__reduce_min_sync(0xffffffffu, __float_as_uint(least)));
            uneven = __any_sync(0xffffffffu, uneven) || x > least * TR_V_EVEN;
            if (!uneven) vtop = fmaxf(vtop, x);  // a few large ones, that no row may see, are looked at again
          }
          const bool bad = key < Ltot && !(fabsf(mine_v) + fabsf(mine_k) < INFINITY);
          // Where some row does not see some key, that key's scales may be anything (a slot that was never written has zeros), but neither may
          // make a NaN of a score of -inf or of a weight of 0: the key's is positive and finite (the rows that see a key whose scale is zero
          // get its scores, zeros, from the smallest one), a value's finite, and the rows that do see a key with others are marked.
          if (part == 0) sc[i] = plain || (key < Ltot && !bad && mine_k > 0.f) ? mine_k : 1.17549435e-38f;
          else sc[TW_KEYS + i] = plain || !bad ? mine_v : 0.f;
          if (!plain) {
            const unsigned m = __ballot_sync(0xffffffffu, bad);
            if (lane == 0) reinterpret_cast<volatile uint32_t*>(&s_bad[st][part])[warp & 1] = m;
          }
          hand_over(st);  // the softmax warps have left step t - 2: the V part of step t - 1 has waited for its product
          if (pt == 0) s_vtop[t & 1] = uneven ? -INFINITY : value_log2(x);
        }
        if (pt == 0) s_groups[st] = ngl;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(KREADY, st));
          if (F16) mbar_arrive(bar(KEMPTY, st));
        }

        if (!warp_wait(bar(VFULL, st), (t / ST) & 1)) { fail_site = 75; break; }
        // 8-bit: the products of the step before have left the buffer.  From here on the softmax warps have left step t - ST, too.
        if (F16 && t > 0 && !warp_wait(odone((t - 1) & 1), ((t - 1) >> 1) & 1)) { fail_site = 75; break; }
        if (!F16) hand_over(st);
        if (!F16) {
          if (!plain) {  // a slot behind the last node, or values that some rows must not meet
            bool bad = false;
#pragma unroll 1
            for (int c = part; c < D / 8; c += 2) {
              const uint32_t a = vr + (c >> 3) * (TW_KEYS * 128) + sw128_offset(i, c & 7);
              const uint4 w4 = lds128(a);
              uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
              uint32_t odd = 0u;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t m = ((w[k] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) | ((w[k] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
                w[k] = key < Ltot ? w[k] & ~m : 0u;
                odd |= m;
              }
              if (odd != 0u || key >= Ltot) sts128(a, make_uint4(w[0], w[1], w[2], w[3]));
              bad |= odd != 0u && key < Ltot;
            }
            const unsigned m = __ballot_sync(0xffffffffu, bad);
            if (lane == 0) reinterpret_cast<volatile uint32_t*>(&s_bad[st][part])[warp & 1] = m;
          }
        } else {
          // V as a K-major operand: of each 16 keys, rows of 32 bytes.  Row i D/4 + c is dim 4 c + i, so that neighbouring lanes write
          // neighbouring rows; the columns of O stand in that order.
          uint8_t* vop = sgen + S::C_OFF + S::OP;
          constexpr int PARTS = TW_PREP_WARPS * 32 / D;  // threads that share 16 keys of four dims
          {
            const int u = pt % D, kb = u / (D / 4), c = u % (D / 4);
            uint32_t w[4][4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const uint4 c4 = *reinterpret_cast<const uint4*>(sgen + S::V_OFF + st * S::VSTAGE + kb * (16 * D) + v_chunk<D>(q, c));
              w[q][0] = c4.x;
              w[q][1] = c4.y;
              w[q][2] = c4.z;
              w[q][3] = c4.w;
            }
            if (!plain) {  // slots behind the last node, or that some row does not see, may hold anything, a NaN among it
#pragma unroll
              for (int q = 0; q < 4; ++q) {
                uint32_t m = 0u;
#pragma unroll
                for (int e = 0; e < 4; ++e) m |= k0 + kb * 16 + v_key(q, e) < Ltot ? 0xffu << (8 * e) : 0u;
#pragma unroll
                for (int d4 = 0; d4 < 4; ++d4) w[q][d4] = without_nan<FMT>(w[q][d4] & m);
              }
            }
#pragma unroll
            for (int dd = 0; dd < 4 / PARTS; ++dd) {
              const int d4 = dd * PARTS + pt / D;
              uint32_t lo[4], hi[4];
#pragma unroll
              for (int q = 0; q < 4; ++q) codes4_f16<FMT>(PARTS == 1 || pt < D ? w[q][dd * PARTS] : w[q][dd * PARTS + PARTS - 1], lo[q], hi[q]);
              const int nrow = d4 * (D / 4) + c;
              uint8_t* at = vop + kb * (D * 32) + nrow * 32;
              const int sw = (nrow & 4) << 2;
              *reinterpret_cast<uint4*>(at + sw) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
              *reinterpret_cast<uint4*>(at + (16 ^ sw)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(bar(VREADY, st));
          if (F16) mbar_arrive(bar(VEMPTY, st));
        }
      }
    } else {
      // =============================== softmax ===============================
      asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(TW_REGS_SOFTMAX));
      if (warp < nactive) {
      const int rr = threadIdx.x;  // row of the block = lane of tensor memory
      const int depth = rr < rows ? s_depth[rr] : dmax, node = min((row0 + rr) / G, n - 1);
      const float rs = F16 ? kScale * s_qs[rr] : kScale;
      const uint32_t lanes = (uint32_t)(warp * 32) << 16;
      float m_used = -INFINITY;
      float2 l2 = make_float2(0.f, 0.f);
      bool ok = true;
      for (int t = 0; t < mine; ++t) {
        const int st = t % ST, bf = t & 1, k0 = (s_first + t * P.nsplit) * TW_KEYS;
        const uint32_t tS = tmem + lanes + bf * TW_KEYS;
        const bool plain = k0 + TW_KEYS <= L && L + dmax - k0 <= Wmax;  // every row sees every key
        // What the operands' warps hand over comes with K in 8 bits, with V in bf16 (whose K may be a stage ahead of this step).
        ok = warp_wait(F16 ? bar(KREADY, st) : bar(VREADY, st), (t / ST) & 1) && warp_wait(sdone(bf), (t >> 1) & 1);
        if (!ok) { fail_site = 76; break; }
        tc_fence_after();

        // ---- terms that only some rows keep, into S where it stands ----
        if (s_lone[st]) {
          const uint8_t* xb = sgen + S::X_OFF + st * S::XSIZE;
          const uint32_t* xn = reinterpret_cast<const uint32_t*>(xb + TW_KEYS * TW_LONE * 8);
          const uint8_t* qrow = sgen + rr * 32;
          const int qsw = (rr & 4) << 2;
          const uint32_t c0n = xn[lane], c1n = xn[lane + 32];
          const int n0 = (int)(c0n >> 16) - (int)(c0n & 0xffffu), n1 = (int)(c1n >> 16) - (int)(c1n & 0xffffu);
          const int most = __reduce_max_sync(0xffffffffu, max(n0, n1));
#pragma unroll 1
          for (int e = 0; e < most; ++e) {  // the e-th lone term of every key, four keys at a time
            const unsigned long long have =
                (unsigned long long)__ballot_sync(0xffffffffu, n0 > e) | ((unsigned long long)__ballot_sync(0xffffffffu, n1 > e) << 32);
#pragma unroll 1
            for (int c = 0; c < TW_KEYS; c += 4) {
              if (((have >> c) & 15ull) == 0ull) continue;
              float x[4], add[4];
              tc_ld4(tS + c, x);
              uint2 w[4];
              if (e < TW_LONE) {
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                  const uint4 two = *reinterpret_cast<const uint4*>(xb + (e * TW_KEYS + c + k) * 8);
                  w[k] = make_uint2(two.x, two.y);
                  w[k + 1] = make_uint2(two.z, two.w);
                }
              } else {  // more than are handed over: from the cache
                const uint8_t* ktile = P.k + (grp * P.ktiles + k0 / KT) * 16384;
#pragma unroll 1
                for (int k = 0; k < 4; ++k) {
                  uint2 v = make_uint2(0u, 0u);
                  if (((have >> (c + k)) & 1ull) != 0ull) {
                    const int p = (int)(xn[c + k] & 0xffffu) + e, kk = k0 + c + k, kin = kk % KT;
                    const int place = kk < L ? kk - L : tr.depth[cur][kk - L];
                    v.x = F16 ? codes_f16<FMT>(*reinterpret_cast<const uint16_t*>(ktile + ((p >> 3) * KT + kin) * 16 + (p & 7) * 2))
                              : *reinterpret_cast<const uint32_t*>(ktile + ((p >> 3) * KT + kin) * 32 + (((p & 7) * 4) ^ ((kin & 4) << 2)));
                    v.y = (uint32_t)((p >> 3) * (TW_ROWS * 32) + (p & 7) * 4) | ((uint32_t)(sW[H - 1 - p] + place) << 16);
                  }
                  w[0] = k == 0 ? v : w[0];
                  w[1] = k == 1 ? v : w[1];
                  w[2] = k == 2 ? v : w[2];
                  w[3] = k == 3 ? v : w[3];
                }
              }
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const uint32_t qw = *reinterpret_cast<const uint32_t*>(qrow + ((w[k].y & 0xffffu) ^ qsw));
                const float2 q = F16 ? half2_to_f2(qw) : make_float2(bf16lo_to_f32(qw), bf16hi_to_f32(qw));
                const float2 kv = F16 ? half2_to_f2(w[k].x) : make_float2(bf16lo_to_f32(w[k].x), bf16hi_to_f32(w[k].x));
                const bool keeps = ((have >> (c + k)) & 1ull) != 0ull && depth <= (int)(int16_t)(w[k].y >> 16);
                add[k] = keeps ? fmaf(q.x, kv.x, q.y * kv.y) : 0.f;
              }
              tc_wait_ld_pin(x);
#pragma unroll
              for (int k = 0; k < 4; ++k) x[k] += add[k];
              tc_st4(tS + c, x);
            }
            tc_wait_st();
          }
        }

        // ---- keys that this row does not see ----
        if (!plain) {
          const unsigned long long l0 = tr.line[cur][node][0], l1 = tr.line[cur][node][1], bad = s_bad[st][0] | s_bad[st][1];
#pragma unroll 1
          for (int c = 0; c < TW_KEYS; c += 8) {
            float x[8];
            tc_ld8(tS + c, x);
            tc_wait_ld_pin(x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              const int key = k0 + c + i, j = key - L;
              bool seen = L + depth - key <= Wmax;
              if (key >= L) seen = j < n && (((j < 64 ? l0 : l1) >> (j & 63)) & 1ull) != 0ull && depth - tr.depth[cur][min(j, n - 1)] <= Wmax;
              x[i] = !seen ? -INFINITY : ((bad >> (c + i)) & 1ull) != 0ull ? __uint_as_float(0x7fc00000u) : x[i];
            }
            tc_st8(tS + c, x);
          }
          tc_wait_st();
        }

        // 8-bit, scales of the values that differ much: the reference needs the row's own largest weight times scale.  (Elsewhere the largest
        // score and the largest scale bound it well enough: an addition and a maximum a cell less.)
        float top = -INFINITY;
        if (F16 && __builtin_expect(s_vtop[bf] == -INFINITY, 0)) top = row_top(tS, reinterpret_cast<const float*>(sgen + S::SC_OFF) + bf * (2 * TW_KEYS), rs);

        float2 s[32];
        tc_ld32(tS, reinterpret_cast<uint32_t*>(s));
        tc_ld32(tS + 32, reinterpret_cast<uint32_t*>(s) + 32);
        const float4* sck = reinterpret_cast<const float4*>(sgen + S::SC_OFF) + bf * (2 * TW_KEYS / 4);  // scales of the keys, then weights of the values
        tc_wait_ld_pin64(reinterpret_cast<float(&)[64]>(s));
        if (F16) {
#pragma unroll
          for (int c = 0; c < 32; c += 2) {
            const float4 k4 = sck[c / 2];
            s[c] = __fmul2_rn(s[c], make_float2(k4.x, k4.y));
            s[c + 1] = __fmul2_rn(s[c + 1], make_float2(k4.z, k4.w));
          }
        }
        float mx0 = fmaxf(s[0].x, s[0].y), mx1 = fmaxf(s[1].x, s[1].y);
#pragma unroll
        for (int c = 2; c < 32; c += 2) {
          mx0 = max3(mx0, s[c].x, s[c].y);
          mx1 = max3(mx1, s[c + 1].x, s[c + 1].y);
        }
        const float mx = F16 ? fmaxf(fmaf(fmaxf(mx0, mx1), rs, s_vtop[bf]), top) : fmaxf(mx0, mx1) * rs;
        float fix = 1.f;
        bool moved = false;
        if (mx > m_used + (m_used == -INFINITY ? 0.f : TR_RESCALE)) {
          fix = m_used == -INFINITY ? 0.f : tr_ex2(F16 ? 0.5f * (m_used - mx) : m_used - mx);  // 8-bit: its root, since it may pass the range of a float
          m_used = mx;
          moved = true;
        }
        const float bias = F16 ? TR_P_SHIFT - (m_used == -INFINITY ? 0.f : m_used) : (m_used == -INFINITY ? 0.f : -m_used);
        if (__any_sync(0xffffffffu, moved)) {
          l2.x = F16 ? l2.x * fix * fix : l2.x * fix;
          l2.y = F16 ? l2.y * fix * fix : l2.y * fix;
          if (t > 0) {
            if (!warp_wait(odone((t - 1) & 1), ((t - 1) >> 1) & 1)) { fail_site = 77; ok = false; break; }
            tc_fence_after();
#pragma unroll 1
            for (int c = 0; c < D; c += 8) {
              float o[8];
              tc_ld8(tO + lanes + c, o);
              tc_wait_ld_pin(o);
#pragma unroll
              for (int k = 0; k < 8; ++k) o[k] = F16 ? o[k] * fix * fix : o[k] * fix;
              tc_st8(tO + lanes + c, o);
            }
          }
        }
        const float2 rs2 = make_float2(rs, rs), bias2 = make_float2(bias, bias);
        uint32_t p[32];
#pragma unroll
        for (int c = 0; c < 32; c += 2) {
          float4 v4 = make_float4(1.f, 1.f, 1.f, 1.f);
          if (F16) v4 = sck[TW_KEYS / 4 + c / 2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float2 x = __ffma2_rn(s[c + i], rs2, bias2);
            const float2 e = make_float2(tr_ex2(x.x), tr_ex2(x.y));
            l2 = __fadd2_rn(l2, e);
            if (F16) {
              const float2 w = __fmul2_rn(e, i ? make_float2(v4.z, v4.w) : make_float2(v4.x, v4.y));
              p[c + i] = pack_f16x2(w.x, w.y);
            } else {
              p[c + i] = pack_bf16x2(e.x, e.y);
            }
          }
        }
        tc_st32(tS, p);
        tc_wait_st();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(pready(bf));
      }
      // ---- the row's sums: the result, or this split's share of it ----
      if (ok && mine > 0 && !warp_wait(odone((mine - 1) & 1), ((mine - 1) >> 1) & 1)) { fail_site = 78; ok = false; }
      tc_fence_after();
      if (ok) {
        const float l = l2.x + l2.y;
        bool odd = false;
        const int row = row0 + rr;
        const int64_t o = ((int64_t)b * P.Hq + hkv * G + row % G) * T + row / G, at = (grp * P.nsplit + split) * (int64_t)(T * G) + row;
        const bool direct = P.nsplit == 1;
        const float f = direct || F16 ? (l > 0.f || l != l ? 1.f / l : 0.f) : 1.f;  // 8-bit: see the parts of atf_tree_tiles
        const float ref = F16 ? m_used + log2f(l) - TR_P_SHIFT : m_used;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          float x[32];  // dims c .. c + 31
          if (mine > 0) {
            if (F16) {
              float y[4][8];
#pragma unroll
              for (int i = 0; i < 4; ++i) tc_ld8(tO + lanes + i * (D / 4) + c / 4, y[i]);
#pragma unroll
              for (int i = 0; i < 4; ++i) tc_wait_ld_pin(y[i]);
#pragma unroll
              for (int k = 0; k < 32; ++k) x[k] = y[k & 3][k >> 2];
            } else {
              tc_ld32(tO + lanes + c, reinterpret_cast<uint32_t*>(x));
              tc_wait_ld_pin(x);
            }
          }
          if (rr < rows) {
#pragma unroll
            for (int k = 0; k < 32; ++k) x[k] = mine > 0 ? x[k] * f : 0.f;
            if (direct) {
#pragma unroll
              for (int k = 0; k < 32; k += 4) odd |= not_finite(x[k], x[k + 1], x[k + 2], x[k + 3]);
#pragma unroll
              for (int k = 0; k < 32; k += 8)
                *reinterpret_cast<uint4*>(P.O + o * D + c + k) = make_uint4(pack_bf16x2(x[k], x[k + 1]), pack_bf16x2(x[k + 2], x[k + 3]),
                                                                            pack_bf16x2(x[k + 4], x[k + 5]), pack_bf16x2(x[k + 6], x[k + 7]));
            } else {
#pragma unroll
              for (int k = 0; k < 32; k += 4) *reinterpret_cast<float4*>(P.outs + at * D + c + k) = make_float4(x[k], x[k + 1], x[k + 2], x[k + 3]);
            }
          }
        }
        if (direct && odd) {
#pragma unroll 1
          for (int c = 0; c < D; c += 8) *reinterpret_cast<uint4*>(P.O + o * D + c) = make_uint4(0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u);
        }
        if (rr < rows) {
          if (!direct) *reinterpret_cast<float2*>(P.sums + at * 2) = F16 ? make_float2(l == 0.f ? -INFINITY : ref, l == 0.f ? 0.f : 1.f) : make_float2(m_used, l);
          else if (P.lse) P.lse[o] = odd ? __uint_as_float(0x7fc00000u) : (F16 ? ref : m_used + log2f(l)) * 0.6931471805599453f;
        }
      }
      }
    }
  }
  if (fail_site) {
    atomicExch(P.status, 1u);
    atomicExch(P.status + 1, fail_site);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == TW_PREP) tmem_dealloc(tmem, TW_TMEM_COLS);
}

template <int D, int FMT>
atf_status launch_wide(const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, cudaStream_t s) {
  auto kern = atf_tree_wide<D, FMT>;
  constexpr int smem = WideShape<D, FMT>::SMEM;
  // a warpgroup that asks for registers which the block was not launched with would wait for good, and one that gives up what it does not have faults
  static const bool enough = [&] {
    cudaFuncAttributes a;
    return cudaFuncGetAttributes(&a, kern) == cudaSuccess && a.numRegs == TW_REGS;
  }();
  if (!enough) return atf_fail(ATF_ERR_CUDA, "atf_decode_tree: the kernel was built with other registers than it shares out");
  ATF_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  ATF_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
  ATF_CUDA_CHECK(atf_launch_overlapped(kern, dim3(P.nsplit, P.Hkv * P.rtiles, B), TW_THREADS, smem, s, tmV, P, t));
  return ATF_OK;
}

}  // namespace

atf_status atf_tree_wide_launch(int format, const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, int d, cudaStream_t s) {
  if (d == 64)
    return format == ATF_KV_BF16   ? launch_wide<64, ATF_KV_BF16>(tmV, P, t, B, s)
           : format == ATF_KV_E4M3 ? launch_wide<64, ATF_KV_E4M3>(tmV, P, t, B, s)
                                   : launch_wide<64, ATF_KV_INT8>(tmV, P, t, B, s);
  return format == ATF_KV_BF16   ? launch_wide<128, ATF_KV_BF16>(tmV, P, t, B, s)
         : format == ATF_KV_E4M3 ? launch_wide<128, ATF_KV_E4M3>(tmV, P, t, B, s)
                                 : launch_wide<128, ATF_KV_INT8>(tmV, P, t, B, s);
}
