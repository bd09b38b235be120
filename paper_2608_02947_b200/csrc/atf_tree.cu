// atf_decode_tree: windowed attention of a tree of T drafted tokens per sequence over a key/value cache (T = 1: a decode step),
// in bf16 or in 8 bits.
//
// The rows of a block are the nodes of the tree times the query heads that share a KV head; the cache is read once for all of
// them.  Node i stands at position L + depth_i behind the L committed tokens; it sees every committed key and the drafted keys
// of its ancestors and its own.  The pair predicate z <= W_r differs from row to row only where a window ends between the
// nearest and the farthest row of the tree, a few keys a pair: a key's products take the pairs that are live for EVERY row, and
// the few (key, pair) terms that only some rows keep are added one by one.
//
// Work split: grid = (splits, KV heads x tiles of rows, sequences).  Tiles of 16 KiB of K are dealt round-robin to the
// splits; one warp issues bulk copies of the live prefix of a K tile, its V tile and its scales into a ring, four warps take a
// quarter of the tile's keys each.  S^T = K Q^T and O^T += V^T P^T are mma.sync products (m16n8k16) with keys or dims as M and 8
// or 16 rows of the tree as N: bf16 for the bf16 cache, f16 for the 8-bit ones, whose codes f16 holds exactly (Q is shifted into
// its range row by row, which rounds nothing that 28 bits below the row's largest element keep; a weight times its value's
// scale is kept below 2^16 by a running reference of the row, see TR_P_SHIFT).  The scale of a key multiplies its row of S^T, in 32 bits.  Weights are rounded
// to the type of V, which the product wants; their sum is that of the unrounded ones, in fp32.
// More than 16 rows take the kernel of atf_tree_wide.cu.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <type_traits>

#include "atf_tree.cuh"

namespace {

constexpr int TR_WARPS = 4, TR_THREADS = (TR_WARPS + 1) * 32, TR_TILE = 16384;

template <int D, int FMT, int NB>
struct TreeShape {
  static constexpr bool F16 = FMT != ATF_KV_BF16;
  static constexpr int H = D / 2, KT = atf_kv_tile_keys(D, !F16), EB = F16 ? 16 : 32;  // bytes of a (key, group) entry
  static constexpr int KB = KT / TR_WARPS, SB = KB >= 32 ? 32 : 16;
  static constexpr int NKS = D / 16, NMT = D / 16, ROWS = 8 * NB, PS = D + 4;
  static constexpr int BLOCKS = NB == 1 ? 3 : 2;  // blocks an SM
  static constexpr int STAGES = NB == 1 ? 2 : 3;
  static constexpr int SCALE_BYTES = F16 ? 2 * KT * 4 : 0;
  static constexpr int STAGE = 2 * TR_TILE + SCALE_BYTES;
  static constexpr int QBYTES = NB * NKS * 256;
  static constexpr int SMEM = STAGES * STAGE + QBYTES + 1024 + 64;
  static_assert(BLOCKS * (SMEM + ROWS * 48 + 1024 + 1024) <= 228 * 1024, "that many blocks fit an SM, with what is declared in the kernel");
  static_assert(TR_WARPS * ROWS * PS * 4 <= STAGES * STAGE, "the warps' sums fit the ring");
};

template <int D, int FMT, int NB>
__global__ void __launch_bounds__(TR_THREADS, (TreeShape<D, FMT, NB>::BLOCKS))
atf_tree_tiles(const __grid_constant__ CUtensorMap tmV, const __grid_constant__ TreeParams P, const __grid_constant__ AtfTable table) {
  using S = TreeShape<D, FMT, NB>;
  constexpr bool F16 = S::F16;
  constexpr int H = S::H, KT = S::KT, EB = S::EB, KB = S::KB, SB = S::SB, NKS = S::NKS, NMT = S::NMT, ROWS = S::ROWS, PS = S::PS;
  constexpr int NK = SB / 16, STAGE = S::STAGE, ST = S::STAGES;
  const float kScale = 1.4426950408889634f / sqrtf((float)D);

  extern __shared__ uint8_t dsm_raw[];
  __shared__ int sW[ATF_MAX_PAIRS];
  __shared__ TreeShared<ROWS> tr;  // all the rows of a sequence are in one block, and a node has a row
  __shared__ int s_depth[ROWS];
  __shared__ float s_qs[ROWS];
  __shared__ int s_near, s_far, s_abort;
  const uint32_t sbase = (smem_u32(dsm_raw) + 1023u) & ~1023u;
  uint8_t* sgen = dsm_raw + (sbase - smem_u32(dsm_raw));
  const uint32_t bars = sbase + ST * STAGE + S::QBYTES;
  uint32_t* qfrag = reinterpret_cast<uint32_t*>(sgen + ST * STAGE);
  auto full_bar = [&](int st) { return bars + 8u * (uint32_t)st; };
  auto empty_bar = [&](int st) { return bars + 8u * (uint32_t)(ST + st); };

  const int split = blockIdx.x, hkv = blockIdx.y / P.rtiles, rt = blockIdx.y % P.rtiles, b = blockIdx.z;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t4 = lane & 3;
  const int G = P.G, T = P.T, row0 = rt * ROWS;
  const int64_t grp = (int64_t)b * P.Hkv + hkv;
  if (threadIdx.x < ATF_MAX_PAIRS) sW[threadIdx.x] = table.w[threadIdx.x];
  if (threadIdx.x == 0) {
    s_abort = 0;
    s_near = 0x7fffffff;
    s_far = 0;
    for (int st = 0; st < ST; ++st) {
      mbar_init(full_bar(st), 1);
      mbar_init(empty_bar(st), TR_WARPS);
    }
    mbar_fence_init();
    fence_proxy_async_smem();
    if (!F16) tma_prefetch_desc(&tmV);
  }
  grid_dependency_launch();
  grid_dependency_wait();
  const int n = P.counts ? min(max(P.counts[b], 0), T) : T;
  const int L = P.lens ? min(max(P.lens[b], 0), P.max_len) : P.len;
  const int rows = min(n * G - row0, ROWS);  // rows of this block that are somebody's
  if (rows <= 0) return;                     // the same for the whole block
  const int Ltot = L + n;
  __syncthreads();
  const int Wmax = sW[H - 1];
  const int ntiles = (Ltot + KT - 1) / KT;
  const int t_first = max(0, L - Wmax) / KT + split;  // tiles in front of it hold no key that any row reaches
  const PairWidths<H> W(sW, lane);
  unsigned int fail_site = 0;
  volatile int* abortp = &s_abort;
  auto bounded_wait = [&](uint32_t bar_, uint32_t parity) { return tr_wait(bar_, parity, abortp); };
  auto warp_wait = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, bounded_wait(bar, parity)) != 0; };

  // Both products are taken transposed: keys or dims fill the 16 rows of an mma, the 8 NB rows of the tree are its columns.
  float oacc[NB][NMT][4];  // two dims (see below) x rows 8 nb + 2 t4 + {0, 1}
  float m_used[NB][2], l_part[NB][2];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
    for (int mt = 0; mt < NMT; ++mt)
#pragma unroll
      for (int e = 0; e < 4; ++e) oacc[nb][mt][e] = 0.f;
    m_used[nb][0] = m_used[nb][1] = -INFINITY;
    l_part[nb][0] = l_part[nb][1] = 0.f;
  }
  float vtop = 0.f;  // 8-bit: up to where the values' scales are taken as they stand

  if (warp == TR_WARPS) {
    // =============================== producer ===============================
    // It starts while the others still read the tree and Q, and so takes a row to be as near as rows can be.
    int it = 0;
    for (int t = t_first; t < ntiles; t += P.nsplit, ++it) {
      const int st = it % ST, end = t * KT + KT;
      const int ngl = (W.live(end > L ? 0 : L - (end - 1)) + 7) >> 3;  // groups some key of the tile keeps for a row of any depth
      if (it >= ST && !warp_wait(empty_bar(st), ((it / ST) - 1) & 1)) { fail_site = 60; break; }
      if (lane == 0) {
        const uint32_t kdst = sbase + st * STAGE, vdst = kdst + TR_TILE;
        const uint32_t kbytes = (uint32_t)(ngl * KT * EB);
        const uint32_t vbytes = F16 ? (uint32_t)((min(KT, Ltot - t * KT) + 15) / 16 * 16 * D) : (uint32_t)TR_TILE;
        mbar_expect_tx(full_bar(st), kbytes + vbytes + S::SCALE_BYTES);
        const int64_t tile = grp * P.ktiles + t;
        if (kbytes) bulk_load_1d(kdst, P.k + tile * TR_TILE, kbytes, full_bar(st));
        if (F16) {
          bulk_load_1d(vdst, P.v + tile * TR_TILE, vbytes, full_bar(st));
          bulk_load_1d(vdst + TR_TILE, P.scales + tile * (2 * KT), S::SCALE_BYTES, full_bar(st));
        } else {
#pragma unroll
          for (int vb = 0; vb < D / 64; ++vb) tma_load_3d(vdst + vb * (KT * 128), &tmV, full_bar(st), vb * 64, t * KT, (int)grp);
        }
      }
    }
    // no copy is in flight when the sums go where the ring was and the block ends, whatever the others gave up
    for (int i = max(0, it - ST); i < it; ++i)
      if (!mbar_wait(full_bar(i % ST), (i / ST) & 1)) fail_site = 62;
  } else {
    // =============================== consumers ===============================
    // word ((row / 8) NKS + j) 32 + lane, register: pair 8 j + 2 t + c of row g is register c of lane 4 g + t
    const int parent = tree_parent(P, b, n, threadIdx.x);
    stage_rows<D, F16, ROWS, TR_WARPS, ROWS / TR_WARPS>(P, (int64_t)b * P.Hq + hkv * G, row0, rows, warp, lane, s_qs, [&](int rr, int p, uint32_t w) {
      qfrag[((((rr >> 3) * NKS + (p >> 3)) * 32 + (rr & 7) * 4 + ((p & 7) >> 1)) << 1) + (p & 1)] = w;
    });
    const int cur = build_tree<TR_WARPS * 32>(tr, parent, n, threadIdx.x);
    // ---- this block's rows: depth, and Q in the order of the products' B fragments ----
    if (threadIdx.x < ROWS) {
      const int dep = tr.depth[cur][min((row0 + (int)threadIdx.x) / G, n - 1)];
      s_depth[threadIdx.x] = dep;
      if (threadIdx.x < rows) {
        atomicMin(&s_near, dep);
        atomicMax(&s_far, dep);
      }
    }
    group_barrier(TR_WARPS * 32);
    const int dmin = s_near, dmax = s_far;
    uint32_t qb[NB][NKS][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int j = 0; j < NKS; ++j) *reinterpret_cast<uint2*>(qb[nb][j]) = reinterpret_cast<const uint2*>(qfrag)[(nb * NKS + j) * 32 + lane];
    float rs[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) rs[nb][e] = F16 ? kScale * s_qs[nb * 8 + 2 * t4 + e] : kScale;
    // One block of keys of a warp.  FAST: every row sees every key and keeps the same pairs of a key as the others do, as nearly all blocks
    // of a long context are; the form for the others, with its masks and lone terms, is code of its own that stays out of the way.
    // (One token, 32 x 8 x 16384, e4m3, with the general form wherever a window ends within a block: 135 us instead of 115.)
    auto step = [&](auto form, const uint8_t* ks, int t, int kin0, int kb0, bool committed, bool plain, int n_far, int n_all, int n_any) __attribute__((always_inline)) {
      constexpr bool FAST = decltype(form)::value;
      const bool uniform = n_any == n_far;
      const uint8_t* vs = ks + TR_TILE;
      const float* kscale = reinterpret_cast<const float*>(vs + TR_TILE);
      const float* vscale = kscale + KT;
      int live[NK][2], some[NK][2];  // pairs that this lane's keys g, g + 8 of each 16 keep for every row, and for some row
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) live[k][hf] = some[k][hf] = n_far;
      if (FAST || committed) {  // the windows that end within the block, mostly none or one
        const int last = FAST ? n_all : n_any, z0 = L - kb0 - g;
        for (int p = n_far; p < last; ++p) {
          const int w = sW[H - 1 - p];
#pragma unroll
          for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              const int z = z0 - k * 16 - hf * 8;
              live[k][hf] += w >= z + dmax ? 1 : 0;
              if (!FAST) some[k][hf] += w >= z + dmin ? 1 : 0;
            }
        }
      } else if (!uniform) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int key = kb0 + k * 16 + hf * 8 + g;
            const int place = key < L ? key - L : key < Ltot ? tr.depth[cur][key - L] : 0;
            live[k][hf] = key < Ltot ? pairs_reaching<H>(sW, dmax - place) : 0;
            some[k][hf] = key < L ? pairs_reaching<H>(sW, dmin - place) : key < Ltot ? H : 0;
          }
      }
      float sc[NK][NB][4];  // keys g + {0, 0, 8, 8}, rows 2 t4 + {0, 1, 0, 1}
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc[k][nb][e] = 0.f;

      // ---- S^T = K Q^T over the pairs that are live for every row ----
      const int ngl = (n_all + 7) >> 3, nwhole = FAST || uniform ? n_far >> 3 : 0;  // groups of which every key keeps all
#pragma unroll
      for (int j = 0; j < NKS; ++j) {
        if (j >= ngl) break;  // the same for the warp
        uint32_t a[NK][4];
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int key = kin0 + k * 16 + hf * 8 + g;
            if (F16) {
              codes4_f16<FMT>(*reinterpret_cast<const uint32_t*>(ks + (j * KT + key) * 16 + t4 * 4), a[k][hf], a[k][2 + hf]);
            } else {
              const uint2 w = *reinterpret_cast<const uint2*>(ks + (j * KT + key) * 32 + ((t4 * 8) ^ ((key & 4) << 2)));
              a[k][hf] = w.x;
              a[k][2 + hf] = w.y;
            }
          }
        if (j >= nwhole) {
#pragma unroll
          for (int k = 0; k < NK; ++k)
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
              if (8 * j + 2 * t4 >= live[k][hf]) a[k][hf] = 0u;
              if (8 * j + 2 * t4 + 1 >= live[k][hf]) a[k][2 + hf] = 0u;
            }
        }
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) tr_mma<F16>(sc[k][nb], a[k], qb[nb][j][0], qb[nb][j][1]);
      }

      // ---- terms that only some rows keep ----
      if (!FAST && !uniform) {
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int kin = kin0 + k * 16 + hf * 8 + g, key = t * KT + kin;
            const int place = key < L ? key - L : key < Ltot ? tr.depth[cur][key - L] : 0;  // relative to L, as the rows' depths are
            for (int p = live[k][hf]; p < some[k][hf]; ++p) {
              float2 kv;
              if (F16) {
                kv = half2_to_f2(codes_f16<FMT>(*reinterpret_cast<const uint16_t*>(ks + ((p >> 3) * KT + kin) * 16 + (p & 7) * 2)));
              } else {
                const uint32_t w = *reinterpret_cast<const uint32_t*>(ks + ((p >> 3) * KT + kin) * 32 + (((p & 7) * 4) ^ ((kin & 4) << 2)));
                kv = make_float2(bf16lo_to_f32(w), bf16hi_to_f32(w));
              }
              const int deepest = sW[H - 1 - p] + place;
#pragma unroll
              for (int nb = 0; nb < NB; ++nb)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const int rr = nb * 8 + 2 * t4 + e;
                  if (s_depth[rr] > deepest) continue;
                  const uint32_t w = qfrag[(((nb * NKS + (p >> 3)) * 32 + (2 * t4 + e) * 4 + ((p & 7) >> 1)) << 1) + (p & 1)];
                  const float2 qv = F16 ? half2_to_f2(w) : make_float2(bf16lo_to_f32(w), bf16hi_to_f32(w));
                  sc[k][nb][2 * hf + e] = fmaf(qv.x, kv.x, fmaf(qv.y, kv.y, sc[k][nb][2 * hf + e]));
                }
            }
          }
      }

      // ---- 8-bit: scales of the values ----
      float v2[NK][2], lv[NK][2];  // and log2 of them
      if (F16) {
        bool larger = false;
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) {
            const int i = k * 16 + hf * 8 + g;
            v2[k][hf] = FAST || kb0 + i < Ltot ? vscale[kin0 + i] : 0.f;
            larger |= v2[k][hf] > vtop;
          }
        if (__any_sync(0xffffffffu, larger)) {  // than before
          float x, least;
          bool one;
          auto range = [&]() {
            x = 0.f;
            least = 3e38f;
            one = false;
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf) {
                const float v = v2[k][hf];
                x = fmaxf(x, v < 3e38f ? v : 0.f);
                least = fminf(least, v > 0.f ? v : 3e38f);
                one |= v == 1.f;
              }
            x = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(x)));
            least = __uint_as_float(__reduce_min_sync(0xffffffffu, __float_as_uint(least)));
          };
          range();
          if (__any_sync(0xffffffffu, one) || x > least * TR_V_EVEN) {  // rows of zeros, whose scale is 1 whatever the others are, do not count
            const uint32_t zero = zero_rows<D, FMT>(vs + kin0 * D, lane);
#pragma unroll
            for (int k = 0; k < NK; ++k)
#pragma unroll
              for (int hf = 0; hf < 2; ++hf)
                if (v2[k][hf] < 3e38f && (zero >> (k * 16 + hf * 8 + g) & 1u) != 0u) v2[k][hf] = 0.f;
            range();
          }
          // up to 64 times as large is taken as it stands from now on; a few large ones, that no row may see, are looked at again
          if (x <= least * TR_V_EVEN) vtop = fmaxf(vtop, x * TR_V_EVEN);
        }
#pragma unroll
        for (int k = 0; k < NK; ++k)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) lv[k][hf] = value_log2(v2[k][hf]);
      }

      // ---- scaling, mask, online softmax (log2 domain) ----
      float mx[NB][2];
      uint32_t hidden = 0u;  // bf16: cells that their rows do not see, which a score of -inf alone does not tell (8-bit keys give none that is not masked)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) mx[nb][0] = mx[nb][1] = -INFINITY;
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const float k2 = F16 ? kscale[kin0 + k * 16 + hf * 8 + g] : 1.f;
          const int key = kb0 + k * 16 + hf * 8 + g;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              float& s = sc[k][nb][2 * hf + e];
              s *= F16 ? rs[nb][e] * k2 : rs[nb][e];
              if (!FAST && !plain) {
                const int rr = nb * 8 + 2 * t4 + e;
                bool seen;
                if (key < L) {
                  seen = L + s_depth[rr] - key <= Wmax;
                } else {
                  const int j = key - L, node = min((row0 + rr) / G, n - 1);
                  seen = j < n && ((tr.line[cur][node][(j >> 6) & 1] >> (j & 63)) & 1ull) != 0ull && tr.depth[cur][node] - tr.depth[cur][min(j, n - 1)] <= Wmax;
                }
                s = seen ? s : -INFINITY;
                if (!F16) hidden |= seen ? 0u : 1u << (((k * 2 + hf) * NB + nb) * 2 + e);
              }
              mx[nb][e] = fmaxf(mx[nb][e], F16 ? s + lv[k][hf] : s);
            }
        }
      bool moved = false;
      float fix[NB][2], bias[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = mx[nb][e];
#pragma unroll
          for (int off = 4; off < 32; off <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, off));
          float& m = m_used[nb][e];
          fix[nb][e] = 1.f;
          if (x > m + (m == -INFINITY ? 0.f : TR_RESCALE)) {
            fix[nb][e] = m == -INFINITY ? 0.f : tr_ex2(F16 ? 0.5f * (m - x) : m - x);  // 8-bit: its root, since it may pass the range of a float
            m = x;
            moved = true;
          }
          bias[nb][e] = (F16 ? TR_P_SHIFT : 0.f) - (m == -INFINITY ? 0.f : m);
        }
      if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int again = 0; again < (F16 ? 2 : 1); ++again) {
            l_part[nb][0] *= fix[nb][0];
            l_part[nb][1] *= fix[nb][1];
#pragma unroll
            for (int mt = 0; mt < NMT; ++mt)
#pragma unroll
              for (int e = 0; e < 4; ++e) oacc[nb][mt][e] *= fix[nb][e & 1];
          }
        }
      }
      uint32_t pb[NK][NB][2];  // B fragments: keys 2 t4 + {0, 1} (+ 8) of row g
#pragma unroll
      for (int k = 0; k < NK; ++k)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            float p[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float s = sc[k][nb][2 * hf + e];
              p[e] = tr_ex2(s + bias[nb][e]);
              l_part[nb][e] += p[e];
              if (F16) p[e] = FAST || plain || s != -INFINITY ? p[e] * v2[k][hf] : 0.f;  // a key that is not seen counts nothing, whatever it holds
            }
            pb[k][nb][hf] = tr_movmatrix(F16 ? pack_f16x2(p[0], p[1]) : pack_bf16x2(p[0], p[1]));
          }

      if (FMT == ATF_KV_E4M3 && !FAST && !plain) {  // where the codes stand: in the loop below it would cost the form without masks registers
        bool found = false;
#pragma unroll 1
        for (int o = lane * 16; o < SB * D; o += 512) {
          uint4* at = const_cast<uint4*>(reinterpret_cast<const uint4*>(vs + kin0 * D + o));
          const uint4 w = *at, x = make_uint4(without_nan<FMT>(w.x), without_nan<FMT>(w.y), without_nan<FMT>(w.z), without_nan<FMT>(w.w));
          if (w.x == x.x && w.y == x.y && w.z == x.z && w.w == x.w) continue;
          *at = x;
          found = true;
        }
        if (found) fence_proxy_async_smem();  // the next tile is copied over them
        __syncwarp();
      }
      // ---- O^T += V^T P^T ----
      const bool whole = FAST || kb0 + SB <= Ltot;  // slots behind the last node may hold anything
#pragma unroll
      for (int k = 0; k < NK; ++k) {
        uint32_t pm0 = 0xffffffffu, pm1 = 0xffffffffu;  // bf16: keys 2 t, 2 t + 1 and 8 further; 8-bit: bytes of a word
        if (!whole) {
          const int key = kb0 + k * 16 + 2 * t4;
          pm0 = (key < Ltot ? 0x0000ffffu : 0u) | (key + 1 < Ltot ? 0xffff0000u : 0u);
          pm1 = (key + 8 < Ltot ? 0x0000ffffu : 0u) | (key + 9 < Ltot ? 0xffff0000u : 0u);
        }
        if (F16) {
          if (!whole) pm0 = __byte_perm(pm0, pm1, 0x6420);
#pragma unroll
          for (int J = 0; J < D / 32; ++J) {
            const uint4 c4 = *reinterpret_cast<const uint4*>(vs + (kin0 / 16 + k) * (16 * D) + v_chunk<D>(t4, 8 * J + g));
            uint32_t w[4] = {c4.x, c4.y, c4.z, c4.w};
            if (!whole) {
#pragma unroll
              for (int i = 0; i < 4; ++i) w[i] &= pm0;
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {  // dims 32 J + 4 g + 2 i, + 1 as rows g, g + 8
              uint32_t a[4];
              codes4_f16<FMT>(w[2 * i], a[0], a[2]);
              codes4_f16<FMT>(w[2 * i + 1], a[1], a[3]);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) tr_mma<true>(oacc[nb][2 * J + i], a, pb[k][nb][0], pb[k][nb][1]);
            }
          }
        } else {
          const int lm_i = lane >> 3, lm_r = lane & 7, vrow = kin0 + k * 16 + (lm_i & 1) * 8 + lm_r;
          const uint32_t va = smem_u32(vs) + vrow * 128;
          uint32_t odd0 = 0u, odd1 = 0u;  // halves: this lane's keys whose values are not all finite
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) {
            const int chunk = 2 * mt + (lm_i >> 1);
            uint32_t bf[4];
            tr_ldsm_trans(va + (chunk >> 3) * (KT * 128) + (((chunk & 7) ^ lm_r) << 4), bf);
            if (!FAST && !plain) {  // a key that some row does not see has weight 0 there, which an infinity would not survive
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                bf[i] &= (i & 1) ? pm1 : pm0;
                const uint32_t lo = (bf[i] & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (bf[i] & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
                bf[i] &= ~(lo | hi);
                if (i & 1) odd1 |= lo | hi; else odd0 |= lo | hi;
              }
            }
            const uint32_t a[4] = {bf[0], bf[2], bf[1], bf[3]};
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) tr_mma<false>(oacc[nb][mt], a, pb[k][nb][0], pb[k][nb][1]);
          }
          if (!FAST && !plain) {  // the rows that do see it are NaN as a whole
            const uint32_t mine = ((odd0 & 1u) | ((odd0 >> 30) & 2u)) << (2 * t4) | ((odd1 & 1u) | ((odd1 >> 30) & 2u)) << (2 * t4 + 8);
            const uint32_t odd = __reduce_or_sync(0xffffffffu, mine);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb)
#pragma unroll
              for (int e = 0; e < 4; ++e)
                if (((odd >> (g + 8 * (e >> 1))) & 1u) != 0u && (hidden >> (((k * 2 + (e >> 1)) * NB + nb) * 2 + (e & 1)) & 1u) == 0u) l_part[nb][e & 1] = __uint_as_float(0x7fc00000u);
          }
        }
      }
          };
    int it = 0;
    for (int t = t_first; t < ntiles; t += P.nsplit, ++it) {
      const int st = it % ST;
      if (!warp_wait(full_bar(st), (it / ST) & 1)) { fail_site = 61; break; }
      const uint8_t* ks = sgen + st * STAGE;
#pragma unroll 1
      for (int sb = 0; sb < KB / SB; ++sb) {
        const int kin0 = warp * KB + sb * SB, kb0 = t * KT + kin0;
        if (kb0 >= Ltot) break;
        const bool committed = kb0 + SB <= L;
        const bool plain = committed && L + dmax - kb0 <= Wmax;  // every row sees every key
        // pairs live: at the farthest distance; at the nearest key for every row; there for some row
        const int n_far = W.live(max(L - kb0, 0) + dmax);
        const int n_all = W.live(committed ? L + dmax - (kb0 + SB - 1) : 0), n_any = W.live(committed ? L + dmin - (kb0 + SB - 1) : 0);
        if (plain && (n_any == n_far || dmin == dmax)) step(std::true_type(), ks, t, kin0, kb0, committed, plain, n_far, n_all, n_any);
        else step(std::false_type(), ks, t, kin0, kb0, committed, plain, n_far, n_all, n_any);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(st));
    }
  }

  // ---- the warps' sums meet in shared memory (the ring is free once everybody is here) ----
  if (fail_site) {
    atomicExch(P.status, 1u);
    atomicExch(P.status + 1, fail_site);
  }
  __syncthreads();
  float* sm = reinterpret_cast<float*>(sgen);  // [TR_WARPS][ROWS][PS]: outputs, reference, sum
  if (warp < TR_WARPS) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float l = l_part[nb][e];
#pragma unroll
        for (int off = 4; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
        float* dst = sm + (warp * ROWS + nb * 8 + 2 * t4 + e) * PS;
        // 8-bit: references lie apart as the scales do; the parts are joined by their weight in the row, and their outputs are averages
        const float inv = l == 0.f ? 0.f : __fdividef(1.f, l);
        if (g == 0) {
          dst[D] = F16 ? m_used[nb][e] + tr_lg2(l) - TR_P_SHIFT : m_used[nb][e];  // -inf for no weight
          dst[D + 1] = F16 ? l * inv : l;                                         // 1, 0, or a NaN
        }
        if (F16) {
#pragma unroll
          for (int J = 0; J < D / 32; ++J)
            *reinterpret_cast<float4*>(dst + 32 * J + 4 * g) = make_float4(oacc[nb][2 * J][e] * inv, oacc[nb][2 * J][2 + e] * inv,
                                                                           oacc[nb][2 * J + 1][e] * inv, oacc[nb][2 * J + 1][2 + e] * inv);
        } else {
#pragma unroll
          for (int mt = 0; mt < NMT; ++mt) {
            dst[16 * mt + g] = oacc[nb][mt][e];
            dst[16 * mt + 8 + g] = oacc[nb][mt][2 + e];
          }
        }
      }
  }
  __syncthreads();
  for (int i0 = warp * 32; i0 < rows * (D / 4); i0 += TR_THREADS) {  // four dims of a row a lane, D / 4 lanes a row
    const bool in = i0 + lane < rows * (D / 4);
    const int idx = in ? i0 + lane : i0, rr = idx / (D / 4), col = idx % (D / 4) * 4, row = row0 + rr;
    float m[TR_WARPS], M = -INFINITY;
#pragma unroll
    for (int w = 0; w < TR_WARPS; ++w) {
      m[w] = sm[(w * ROWS + rr) * PS + D];
      M = fmaxf(M, m[w]);
    }
    const float Ms = M == -INFINITY ? 0.f : M;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float lacc = 0.f;
#pragma unroll
    for (int w = 0; w < TR_WARPS; ++w) {
      const float* src = sm + (w * ROWS + rr) * PS;
      const float f = tr_ex2(m[w] - Ms);
      const float4 x = *reinterpret_cast<const float4*>(src + col);
      acc.x = fmaf(f, x.x, acc.x);
      acc.y = fmaf(f, x.y, acc.y);
      acc.z = fmaf(f, x.z, acc.z);
      acc.w = fmaf(f, x.w, acc.w);
      lacc = fmaf(f, src[D + 1], lacc);
    }
    if (P.nsplit == 1) {
      const unsigned odd = __ballot_sync(0xffffffffu, in && not_finite(acc.x, acc.y, acc.z, acc.w));
      if ((odd & (D == 64 ? 0xffffu << (lane & 16) : 0xffffffffu)) != 0u) lacc = __uint_as_float(0x7fc00000u);
      if (!in) continue;
      const int64_t o = ((int64_t)b * P.Hq + hkv * G + row % G) * T + row / G;
      const float inv = lacc > 0.f || lacc != lacc ? 1.f / lacc : 0.f;
      *reinterpret_cast<uint2*>(P.O + o * D + col) = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
      if (P.lse && col == 0) P.lse[o] = (M + log2f(lacc)) * 0.6931471805599453f;
    } else if (in) {
      const int64_t at = (grp * P.nsplit + split) * (int64_t)(T * G) + row;
      *reinterpret_cast<float4*>(P.outs + at * D + col) = acc;
      if (col == 0) *reinterpret_cast<float2*>(P.sums + at * 2) = make_float2(M, lacc);
    }
  }
}

// One warp a row: the partial sums of all splits by their references (lanes across the splits, then across the columns).
constexpr int TM_THREADS = 128;
template <int D, bool F16>
__global__ void __launch_bounds__(TM_THREADS) atf_tree_join(const __grid_constant__ TreeParams P, int64_t nrows) {
  constexpr int BATCH = 8;
  const int lane = threadIdx.x & 31;
  const int64_t o = (int64_t)blockIdx.x * (TM_THREADS / 32) + (threadIdx.x >> 5);  // (b Hq + hq) T + node
  grid_dependency_launch();
  grid_dependency_wait();
  if (o >= nrows) return;
  const int node = (int)(o % P.T), hq = (int)(o / P.T % P.Hq);
  const int64_t b = o / ((int64_t)P.T * P.Hq);
  if (P.counts && node >= P.counts[b]) return;  // a row that no node stands for is left as it is
  const int G = P.G, ns = P.nsplit;
  const int64_t step = (int64_t)P.T * G, at = (b * P.Hkv + hq / G) * ns * step + node * G + hq % G;
  const float2* sums = reinterpret_cast<const float2*>(P.sums) + at;
  const float* outs = P.outs + at * D + lane;
  float M = -INFINITY;
  for (int s = lane; s < ns; s += 32) M = fmaxf(M, __ldcg(sums + s * step).x);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, off));
  const float Ms = M == -INFINITY ? 0.f : M;
  float acc[D / 32], L = 0.f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) acc[c] = 0.f;
  for (int s0 = 0; s0 < ns; s0 += BATCH) {
    float2 f[BATCH];
    float x[BATCH][D / 32];
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const bool in = s0 + i < ns;
      f[i] = in ? __ldcg(sums + (s0 + i) * step) : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) x[i][c] = in ? __ldcg(outs + (s0 + i) * step * D + c * 32) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < BATCH; ++i) {
      const float w = tr_ex2(f[i].x - Ms);
      L = fmaf(w, f[i].y, L);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) acc[c] = fmaf(w, x[i][c], acc[c]);
    }
  }
  if (__any_sync(0xffffffffu, not_finite(acc[0], acc[1], acc[D / 32 - 2], acc[D / 32 - 1]))) L = __uint_as_float(0x7fc00000u);
  const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
#pragma unroll
  for (int c = 0; c < D / 32; ++c) P.O[o * D + c * 32 + lane] = __float2bfloat16_rn(acc[c] * inv);
  if (P.lse && lane == 0) P.lse[o] = (M + log2f(L)) * 0.6931471805599453f;
}

atf_status launch_join(int format, const TreeParams& P, int B, int d, cudaStream_t s) {
  if (P.nsplit == 1) return ATF_OK;
  const int64_t nrows = (int64_t)B * P.Hq * P.T;
  const bool f16 = format != ATF_KV_BF16;
  void (*kern)(TreeParams, int64_t) = d == 64 ? (f16 ? atf_tree_join<64, true> : atf_tree_join<64, false>)
                                              : (f16 ? atf_tree_join<128, true> : atf_tree_join<128, false>);
  ATF_CUDA_CHECK(atf_launch_overlapped(kern, dim3((unsigned)((nrows + TM_THREADS / 32 - 1) / (TM_THREADS / 32))), TM_THREADS, 0, s, P, nrows));
  return ATF_OK;
}

template <int D, int FMT, int NB>
atf_status launch_tree(const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, cudaStream_t s) {
  auto kern = atf_tree_tiles<D, FMT, NB>;
  constexpr int smem = TreeShape<D, FMT, NB>::SMEM;
  ATF_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
  ATF_CUDA_CHECK(cudaFuncSetAttribute(kern, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
  ATF_CUDA_CHECK(atf_launch_overlapped(kern, dim3(P.nsplit, P.Hkv * P.rtiles, B), TR_THREADS, smem, s, tmV, P, t));
  return launch_join(FMT, P, B, D, s);
}
template <int D, int FMT>
atf_status launch_tree(const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, int nb, cudaStream_t s) {
  return nb == 1 ? launch_tree<D, FMT, 1>(tmV, P, t, B, s) : launch_tree<D, FMT, 2>(tmV, P, t, B, s);
}
template <int D>
atf_status launch_tree(int format, const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, int nb, cudaStream_t s) {
  return format == ATF_KV_BF16   ? launch_tree<D, ATF_KV_BF16>(tmV, P, t, B, nb, s)
         : format == ATF_KV_E4M3 ? launch_tree<D, ATF_KV_E4M3>(tmV, P, t, B, nb, s)
                                 : launch_tree<D, ATF_KV_INT8>(tmV, P, t, B, nb, s);
}

struct TreePlan {
  bool wide;
  int nb, rtiles;
  int64_t ntiles, nsplit;
};
// Up to 8 rows (a decode step of up to 8 heads) and up to 16 on mma.sync, more on the tensor memory of a block of 128 rows.
// Splits: in units of the time an SM with all its blocks takes for one block's tile, a launch costs the tiles of a block, and a
// few for its start and end, for each round of blocks; blocks that share an SM with fewer others are faster, but not by as much.
TreePlan tree_plan(int format, int B, int Hq, int Hkv, int T, int64_t max_len, int d) {
  TreePlan p;
  const int64_t rows = (int64_t)T * (Hq / Hkv);
  p.wide = rows > 16;
  p.nb = rows <= 8 ? 1 : 2;
  const int block_rows = p.wide ? TW_ROWS : 8 * p.nb;
  p.rtiles = (int)((rows + block_rows - 1) / block_rows);
  const int kt = p.wide ? 64 : atf_kv_tile_keys(d, format == ATF_KV_BF16);
  p.ntiles = (max_len + T + kt - 1) / kt;
  const int64_t groups = (int64_t)B * Hkv * p.rtiles;
  const int slots = p.wide || p.nb == 2 ? 2 : 3;
  const double alone[3] = {0.0, slots == 3 ? 1.6 : 1.4, 2.3}, start = p.wide ? 4.0 : 10.0;
  double best = 0.0;
  p.nsplit = 0;
  for (int64_t ns = 1; ns <= p.ntiles && (ns == 1 || groups * ns <= 8 * slots * 148);) {
    const int64_t tiles = (p.ntiles + ns - 1) / ns, per_sm = (groups * ns + 147) / 148;
    const double cost = ((double)tiles + start) * ((double)(per_sm / slots) * slots + alone[per_sm % slots]) + 0.25 * (double)ns;
    if (p.nsplit == 0 || cost < best) {
      best = cost;
      p.nsplit = ns;
    }
    if (tiles == 1) break;
    ns = (p.ntiles + tiles - 2) / (tiles - 1);
  }
  return p;
}

size_t tree_sums_bytes(size_t rows) { return (rows * 2 * sizeof(float) + 255) & ~(size_t)255; }

atf_status tree_shape(const char* who, int B, int Hq, int Hkv, int T, int64_t max_len, int d) {
  if (d != 64 && d != 128) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: d must be 64 or 128 (got %d)", who, d);
  if (B < 1 || Hq < 1 || Hkv < 1 || T < 1 || max_len < 0) return atf_fail(ATF_ERR_INVALID_ARG, "%s: bad shape", who);
  if (Hq % Hkv) return atf_fail(ATF_ERR_INVALID_ARG, "%s: Hq must be a multiple of Hkv", who);
  if (T > TR_MAX_NODES) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: at most %d nodes (got %d)", who, TR_MAX_NODES, T);
  if (max_len >= (1ll << 30)) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: max_len must be below 2^30", who);
  if (B > 65535 || (int64_t)T * Hq > 65535ll * 16) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: too many rows", who);
  return ATF_OK;
}

}  // namespace

atf_status atf_validate_table(const char* who, const int64_t* table, int d, int64_t N, AtfTable* out);
atf_status atf_kvcache_check(const char* who, const atf_kvcache* c, int B, int Hkv, int d);

extern "C" size_t atf_decode_tree_scratch_bytes(int format, int B, int Hq, int Hkv, int T, int64_t max_len, int d) {
  if (tree_shape("atf_decode_tree", B, Hq, Hkv, T, max_len, d) != ATF_OK || atf_kvcache_tile_keys(format, d) == 0) return 0;
  const TreePlan p = tree_plan(format, B, Hq, Hkv, T, max_len, d);
  const size_t rows = (size_t)B * Hq * T * p.nsplit;
  return p.nsplit == 1 ? 256 : tree_sums_bytes(rows) + ((rows * d * sizeof(float) + 255) & ~(size_t)255);
}

extern "C" atf_status atf_decode_tree(const void* Q, const atf_kvcache* cache, const int32_t* lens, int64_t max_len, const int32_t* parents,
                                      int64_t parents_step, const int32_t* counts, void* O, float* lse, int B, int Hq, int Hkv, int T, int d,
                                      const int64_t* table, void* scratch, size_t scratch_bytes, void* stream) {
  const char* who = "atf_decode_tree";
  atf_status st = tree_shape(who, B, Hq, Hkv, T, max_len, d);
  if (st != ATF_OK) return st;
  if ((st = atf_kvcache_check(who, cache, B, Hkv, d)) != ATF_OK) return st;
  if (!Q || !O || !scratch) return atf_fail(ATF_ERR_INVALID_ARG, "%s: null pointer", who);
  if (((uintptr_t)Q | (uintptr_t)O) & 15) return atf_fail(ATF_ERR_INVALID_ARG, "%s: Q and O must be 16-byte aligned", who);
  if ((uintptr_t)scratch & 255) return atf_fail(ATF_ERR_INVALID_ARG, "%s: scratch must be 256-byte aligned", who);
  if (parents && parents_step != 0 && parents_step < T) return atf_fail(ATF_ERR_INVALID_ARG, "%s: parents_step must be 0 or at least T", who);
  if (max_len + T > cache->capacity)
    return atf_fail(ATF_ERR_INVALID_ARG, "%s: max_len + T is %lld, the cache holds %lld", who, (long long)(max_len + T), (long long)cache->capacity);
  AtfTable t;
  if ((st = atf_validate_table(who, table, d, max_len + T, &t)) != ATF_OK) return st;
  AtfWorkspace ws = atf_bound_workspace();
  if (!ws.ptr) return atf_fail(ATF_ERR_WORKSPACE, "%s: no workspace bound", who);
  const size_t need = atf_decode_tree_scratch_bytes(cache->format, B, Hq, Hkv, T, max_len, d);
  if (scratch_bytes < need) return atf_fail(ATF_ERR_WORKSPACE, "%s: scratch has %zu bytes, needs %zu", who, scratch_bytes, need);
  const TreePlan p = tree_plan(cache->format, B, Hq, Hkv, T, max_len, d);
  TreeParams P;
  P.q = (const __nv_bfloat16*)Q;
  P.k = (const uint8_t*)cache->k;
  P.v = (const uint8_t*)cache->v;
  P.scales = cache->scales;
  P.O = (__nv_bfloat16*)O;
  P.lse = lse;
  P.sums = (float*)scratch;
  P.outs = (float*)((char*)scratch + tree_sums_bytes((size_t)B * Hq * T * p.nsplit));
  P.status = (unsigned int*)ws.ptr;
  P.lens = lens;
  P.counts = counts;
  P.parents = parents;
  P.parents_step = parents_step;
  const int kt = atf_kv_tile_keys(d, cache->format == ATF_KV_BF16);
  P.ktiles = (cache->capacity + kt - 1) / kt;
  P.cap = cache->capacity;
  P.len = P.max_len = (int)max_len;
  P.Hq = Hq;
  P.Hkv = Hkv;
  P.G = Hq / Hkv;
  P.T = T;
  P.nsplit = (int)p.nsplit;
  P.rtiles = p.rtiles;
  if ((int64_t)Hkv * p.rtiles > 65535) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: too many rows", who);
  CUtensorMap tmV = {};
  if (cache->format == ATF_KV_BF16 &&
      (st = atf_make_tile_map(&tmV, cache->v, (int64_t)B * Hkv, cache->capacity, d, cache->capacity, p.wide ? 64 : kt)) != ATF_OK)
    return st;
  if (p.wide) {
    if ((st = atf_tree_wide_launch(cache->format, tmV, P, t, B, d, (cudaStream_t)stream)) != ATF_OK) return st;
    return launch_join(cache->format, P, B, d, (cudaStream_t)stream);
  }
  return d == 64 ? launch_tree<64>(cache->format, tmV, P, t, B, p.nb, (cudaStream_t)stream)
                 : launch_tree<128>(cache->format, tmV, P, t, B, p.nb, (cudaStream_t)stream);
}
