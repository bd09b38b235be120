// What the two kernels of atf_decode_tree share: parameters, the tree in shared memory, codes as f16, small wrappers.
#pragma once

#include <cuda_fp16.h>

#include "atf_kvcache.cuh"

constexpr int TR_MAX_NODES = 128;
constexpr float TR_RESCALE = 7.f;  // log2 units by which a row's maximum may outgrow its reference before sums are rescaled
// 8-bit: f16 holds a weight times its value's scale, 2^7 times as large, against a reference of the row: the largest such product among the keys
// that the row sees, so far.  2^-21 of it is still a full f16, and nothing that a row does not see moves its reference.  The row's sum of weights
// has the same reference: they are fp32 and may be as much smaller or larger than 1 as scales are.
constexpr float TR_P_SHIFT = 7.f;
constexpr float TR_V_EVEN = 64.f;  // scales of a block of keys within this factor are not told apart where that saves work

struct TreeParams {
  const __nv_bfloat16* q;  // [B, Hq, T, D]
  const uint8_t* k;
  const uint8_t* v;
  const float* scales;
  __nv_bfloat16* O;
  float* lse;       // may be null
  float* sums;      // [B Hkv][nsplit][T G][2]: reference and sum of each split; not used with one split
  float* outs;      // [B Hkv][nsplit][T G][D], 16-byte aligned
  unsigned int* status;
  const int32_t* lens;     // committed tokens of each sequence, or null: `len` for all
  const int32_t* counts;   // nodes of each sequence, or null: T
  const int32_t* parents;  // [T] or [B, T], or null: a chain
  int64_t parents_step;
  int64_t ktiles, cap;
  int len, max_len, Hq, Hkv, G, T, nsplit, rtiles;
};

__device__ __forceinline__ float tr_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
template <bool F16>
__device__ __forceinline__ void tr_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void tr_ldsm_trans(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t tr_movmatrix(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}

// How many pairs, from the lowest frequency, reach a distance: for a warp at once, the widths in its registers, two a lane.
template <int H>
struct PairWidths {
  int w0, w1;
  __device__ __forceinline__ PairWidths(const int* W, int lane) : w0(W[lane]), w1(H == 64 ? W[lane + 32] : -1) {}
  __device__ __forceinline__ int live(int z) const {
    const int c = __popc(__ballot_sync(0xffffffffu, w0 >= z));
    return H == 64 ? c + __popc(__ballot_sync(0xffffffffu, w1 >= z)) : c;
  }
};
// The same for a distance of each thread's own: the widths do not decrease with the pair's index.
template <int H>
__device__ __forceinline__ int pairs_reaching(const int* W, int z) {
  int first = 0;  // pairs in front of it do not reach z
#pragma unroll
  for (int step = H / 2; step > 0; step >>= 1) first += W[first + step - 1] < z ? step : 0;
  return H - (first + (W[first] < z ? 1 : 0));
}
// Four codes as two f16x2.
template <int FMT>
__device__ __forceinline__ void codes4_f16(uint32_t w, uint32_t& a, uint32_t& b) {
  if (FMT == ATF_KV_E4M3) {
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tcvt.rn.f16x2.e4m3x2 %0, l;\n\tcvt.rn.f16x2.e4m3x2 %1, h;\n\t}" : "=r"(a), "=r"(b) : "r"(w));
  } else {  // byte ^ 128 in the low bits of 1024: minus 1152
    const uint32_t x = w ^ 0x80808080u, u = __byte_perm(x, 0x64646464u, 0x4140), v = __byte_perm(x, 0x64646464u, 0x4342);
    const __half2 off = __floats2half2_rn(1152.f, 1152.f);
    const __half2 p = __hsub2(*reinterpret_cast<const __half2*>(&u), off), q = __hsub2(*reinterpret_cast<const __half2*>(&v), off);
    a = *reinterpret_cast<const uint32_t*>(&p);
    b = *reinterpret_cast<const uint32_t*>(&q);
  }
}
// Four codes with zeros in the place of NaN ones.  No row that is written has those, but a slot that was not may, and a key that some row
// does not see has weight 0 there, which a NaN would not survive.
template <int FMT>
__device__ __forceinline__ uint32_t without_nan(uint32_t w) {
  if (FMT != ATF_KV_E4M3) return w;
  const uint32_t nan = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;  // bytes 0x7f and 0xff
  return w & ~((nan >> 7) * 0xffu);
}
__device__ __forceinline__ float tr_lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// log2 of a value's scale, for references.  What is smaller than 2^-100, zeros among it, counts as that, so that a sum of weights against such a
// reference stays in the range of fp32.
__device__ __forceinline__ float value_log2(float scale) { return tr_lg2(fmaxf(scale, 7.8886091e-31f)); }
// The keys of two 16-key blocks of V whose codes are all zero, one bit a key.  Rows of zeros have scale 1, whatever the size of the others.
template <int D, int FMT>
__device__ __forceinline__ uint32_t zero_rows(const uint8_t* blocks, int lane) {
  const int t = lane >> 3;
  uint32_t keys = 0u;
#pragma unroll 1
  for (int kb = 0; kb < 32; kb += 16) {
    uint32_t any = 0u;
#pragma unroll 1
    for (int c = lane & 7; c < D / 4; c += 8) {
      const uint4 w = *reinterpret_cast<const uint4*>(blocks + kb * D + v_chunk<D>(t, c));
      any |= w.x | w.y | w.z | w.w;
    }
    if (FMT == ATF_KV_E4M3) any &= 0x7f7f7f7fu;  // a zero may have a sign
#pragma unroll
    for (int e = 0; e < 4; ++e) keys |= (any >> (8 * e) & 0xffu) != 0u ? 1u << (kb + v_key(t, e)) : 0u;
  }
  return ~__reduce_or_sync(0xffffffffu, keys);
}
// Two codes (the low 16 bits).
template <int FMT>
__device__ __forceinline__ uint32_t codes_f16(uint32_t two) {
  uint32_t a, b;
  codes4_f16<FMT>(two, a, b);
  return a;
}
__device__ __forceinline__ float2 half2_to_f2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Of a row's sums.  A row that has met a value which is not finite is NaN as a whole, its LSE with it: which of its elements an infinity or a
// NaN gets to depends on the block of keys that it stands in.
__device__ __forceinline__ bool not_finite(float a, float b, float c, float d) {
  const float z = fmaf(a, 0.f, b * 0.f) + fmaf(c, 0.f, d * 0.f);
  return z != z;
}

// Rows of Q (node, head of the KV head's group) into shared memory: warp `w` of NW takes every NW-th of ROWS rows, U of them in flight;
// store(row of the block, pair from the lowest frequency, its two dims) gets every word, zeros behind the last row.  A lane has two
// neighbouring pairs of a row.  8-bit caches: a row is stored as f16, multiplied by the power of two that brings its largest element
// into [2^14, 2^15) (its inverse goes to qs).  U of a block of 128 rows: three; with all twelve of a warp in flight its start is 2000
// clocks shorter, but what their registers push out is missing in every step (64 / 164 / 133 us with three, 66 / 168 / 140 with twelve).
template <int D, bool F16, int ROWS, int NW, int U, typename Store>
__device__ __forceinline__ void stage_rows(const TreeParams& P, int64_t head0, int row0, int rows, int w, int lane, float* qs, Store store) {
  constexpr int H = D / 2;
  const int l = lane & (H / 2 - 1);
  int node = (row0 + w) / P.G, head = row0 + w - node * P.G;
  const int dnode = NW / P.G, dhead = NW - dnode * P.G;
  for (int u0 = 0; u0 * NW < ROWS; u0 += U) {
    uint32_t lo[U], hi[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      lo[u] = hi[u] = 0u;
      if (w + (u0 + u) * NW < rows) {
        const __nv_bfloat16* src = P.q + ((head0 + head) * P.T + node) * D + H - 2 - 2 * l;
        lo[u] = *reinterpret_cast<const uint32_t*>(src);
        hi[u] = *reinterpret_cast<const uint32_t*>(src + H);
      }
      head += dhead;
      node += dnode;
      if (head >= P.G) {
        head -= P.G;
        ++node;
      }
    }
    uint32_t top[U];  // largest absolute bits of the row
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t a = lo[u], b = hi[u];
      lo[u] = __byte_perm(a, b, 0x7632), hi[u] = __byte_perm(a, b, 0x5410);  // pairs 2 l and 2 l + 1
      top[u] = max(max((lo[u] << 16) & 0x7fffffffu, lo[u] & 0x7fff0000u), max((hi[u] << 16) & 0x7fffffffu, hi[u] & 0x7fff0000u));
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int rr = w + (u0 + u) * NW;
      uint32_t a = lo[u], b = hi[u];
      if (F16) {
        const uint32_t amax = __reduce_max_sync(0xffffffffu, top[u]);
        const int e = amax == 0u || amax >= 0x7f800000u ? 0 : min(max(14 - ((int)(amax >> 23) - 127), -112), 126);
        const float mul = __uint_as_float((uint32_t)(e + 127) << 23);
        if (lane == 0 && rr < ROWS) qs[rr] = __uint_as_float((uint32_t)(127 - e) << 23);
        a = pack_f16x2(bf16lo_to_f32(a) * mul, bf16hi_to_f32(a) * mul);
        b = pack_f16x2(bf16lo_to_f32(b) * mul, bf16hi_to_f32(b) * mul);
      }
      if (lane < H / 2 && rr < ROWS) {
        store(rr, 2 * l, a);
        store(rr, 2 * l + 1, b);
      }
    }
  }
}

// Bounded wait of a thread for a phase of an mbarrier; `abort` (shared by the block) ends the waits of the others once one has given
// up.  (Tests that may suspend the thread for up to 20 us execute half as many instructions and take longer to answer: 64 x 4 x 32768
// in bf16 165.1 us where these take 164.2; 32 x 131072 in e4m3 138.4, 133.1.)
__device__ __forceinline__ bool tr_wait(uint32_t bar, uint32_t parity, volatile int* abort) {
  if (mbar_try_wait(bar, parity)) return true;
  const unsigned long long t0 = global_timer_ns();
  for (;;) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
      if (mbar_try_wait(bar, parity)) return true;
    if (*abort) return false;
    if (global_timer_ns() - t0 > ATF_WAIT_LIMIT_NS) {
      *abort = 1;
      return false;
    }
  }
}

// The tree of a sequence in shared memory: depth and ancestors (itself included) of each of up to NODES nodes.
template <int NODES>
struct TreeShared {
  unsigned long long line[2][NODES][2];
  int depth[2][NODES], jump[2][NODES];
};
// By doubling the jumps: after round k a node holds its nearest 2^k ancestors.  A parent that is not an earlier node stands for
// the committed text.  Returns which half of the buffers holds the result; ends with a barrier of the THREADS threads (whole
// warps, numbered by i) that take part: the warp that issues the copies starts without them.
__device__ __forceinline__ void group_barrier(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }
// parent: what thread i read of node i's (tree_parent), asked for long before it is needed.
__device__ __forceinline__ int tree_parent(const TreeParams& P, int b, int n, int i) {
  return i >= n ? -1 : P.parents ? P.parents[(int64_t)b * P.parents_step + i] : i - 1;
}
template <int THREADS, int NODES>
__device__ __forceinline__ int build_tree(TreeShared<NODES>& S, int parent, int n, int i) {
  if (i < n) {
    const bool node = parent >= 0 && parent < i;
    S.jump[0][i] = node ? parent : -1;
    S.depth[0][i] = node ? 1 : 0;
    S.line[0][i][0] = i < 64 ? 1ull << i : 0ull;
    S.line[0][i][1] = i < 64 ? 0ull : 1ull << (i - 64);
  }
  static_assert(THREADS >= NODES, "a thread a node");
  group_barrier(THREADS);
  int cur = 0;
  for (int span = 1; span < n; span *= 2) {
    if (i < n) {
      const int j = S.jump[cur][i];
      S.jump[cur ^ 1][i] = j < 0 ? -1 : S.jump[cur][j];
      S.depth[cur ^ 1][i] = S.depth[cur][i] + (j < 0 ? 0 : S.depth[cur][j]);
      S.line[cur ^ 1][i][0] = S.line[cur][i][0] | (j < 0 ? 0ull : S.line[cur][j][0]);
      S.line[cur ^ 1][i][1] = S.line[cur][i][1] | (j < 0 ? 0ull : S.line[cur][j][1]);
    }
    cur ^= 1;
    group_barrier(THREADS);
  }
  return cur;
}

// Launches of the kernel for many rows (atf_tree_wide.cu).
atf_status atf_tree_wide_launch(int format, const CUtensorMap& tmV, const TreeParams& P, const AtfTable& t, int B, int d, cudaStream_t s);
constexpr int TW_ROWS = 128;  // rows of one of its blocks
