// atf_qk_norm_rope: the RMS norm of every query and key head and the rotary embedding, in one pass, from the rows as the
// fused projection leaves them (token by token, strided) to the head-major rows that attention takes.
//
//   y = x / sqrt(mean(x^2) + eps) * w,  pair r of y turned by (position * theta_r).
//
// One read and one write of each row: bound by memory.  d/16 lanes hold a row, each the eight pairs of 16 bytes of either half,
// so that the sum of squares is a few shuffles and the rotation needs no other lane.  The angle is reduced to a fraction of a
// turn in 64 bits (positions past 2^20 keep their full accuracy), its sine and cosine, the norm and the rotation are fp32, and
// the result is rounded once.  A thread evaluates its eight angles once and walks the heads of its token.  Where a mean square comes near the ends
// of the range of 32 bits, the squares are taken again of a row that is shifted by a power of two: a vote a head, else.
#include <algorithm>
#include <cmath>

#include "atf_common.cuh"

namespace {

constexpr int NR_THREADS = 256;

struct NormRopeSide {
  const void* x;
  const void* w;  // may be null: ones
  void* o;
  int64_t batch, row, head;  // input strides, elements
  int H;
};
struct NormRopeParams {
  NormRopeSide side[2];  // queries, keys
  const int64_t* positions;  // [B, N], or null
  int64_t N, rows, pos0;     // rows = B N
  float eps, eps_up, eps_down;  // as it is, and for rows times 2^100 and times 2^-70
  double turn[ATF_MAX_PAIRS];  // theta / (2 pi)
};

// Eight consecutive elements as they stand in memory, and as floats.
struct Raw16 {
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void zero() { v = make_uint4(0u, 0u, 0u, 0u); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16lo_to_f32(u[i]);
      f[2 * i + 1] = bf16hi_to_f32(u[i]);
    }
  }
};
struct Raw32 {
  float4 a, b;
  __device__ __forceinline__ void load(const float* p) {
    a = *reinterpret_cast<const float4*>(p);
    b = *reinterpret_cast<const float4*>(p + 4);
  }
  __device__ __forceinline__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w;
    f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
  }
};
template <typename T>
struct RawOf;
template <>
struct RawOf<__nv_bfloat16> {
  using type = Raw16;
};
template <>
struct RawOf<float> {
  using type = Raw32;
};
__device__ __forceinline__ void store8f(__nv_bfloat16* p, const float (&v)[8]) {
  *reinterpret_cast<uint4*>(p) =
      make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ void store8f(float* p, const float (&v)[8]) {
  *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(v[4], v[5], v[6], v[7]);
}

// HL threads share the heads of a (token, segment); blockIdx.y deals the heads out further.  U heads of a thread are in flight.
template <int D, int HL, typename T, int U>
__global__ void __launch_bounds__(NR_THREADS, U * (int)sizeof(T) > 4 ? 2 : 3) atf_norm_rope_rows(const __grid_constant__ NormRopeParams P) {
  constexpr int H = D / 2, LPR = D / 16, SEGS = NR_THREADS / HL, ROWS = SEGS / LPR;
  using Raw = typename RawOf<T>::type;
  static_assert(SEGS % LPR == 0 && ROWS >= 1, "a row's lanes are neighbours");
  const int sg = threadIdx.x % SEGS, c = sg % LPR;
  const int64_t row = (int64_t)blockIdx.x * ROWS + sg / LPR;
  grid_dependency_launch();
  grid_dependency_wait();
  const bool in = row < P.rows;  // lanes of a row leave together, but the shuffles below name the whole warp
  const int64_t rc = in ? row : P.rows - 1, b = rc / P.N, n = rc - b * P.N;
  const int64_t pos = P.positions ? P.positions[rc] : P.pos0 + n;
  float cs[8], sn[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    double a = (double)pos * P.turn[c * 8 + i];
    a -= rint(a);
    sincospif(2.f * (float)a, &sn[i], &cs[i]);
  }
  const int lane_h = threadIdx.x / SEGS, step = HL * (int)gridDim.y;
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const NormRopeSide& S = P.side[k];
    const T* x = (const T*)S.x + b * S.batch + n * S.row + c * 8;
    T* o = (T*)S.o + (b * S.H * P.N + n) * D + c * 8;
    Raw wl, wh;  // the weights, as they stand
    const bool weighted = S.w != nullptr && S.H > 0;
    if (weighted) {
      wl.load((const T*)S.w + c * 8);
      wh.load((const T*)S.w + H + c * 8);
    } else {
      wl.zero();
      wh.zero();
    }
    // every thread of the warp takes the same number of turns: the shuffles need all lanes
    for (int h0 = (int)blockIdx.y * HL; h0 < S.H; h0 += U * step) {
      Raw lo[U], hi[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * step + lane_h;
        if (h < S.H) {
          lo[u].load(x + (int64_t)h * S.head);
          hi[u].load(x + (int64_t)h * S.head + H);
        } else {
          lo[u].zero();
          hi[u].zero();
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int h = h0 + u * step + lane_h;
        float f[8], g[8], ss = 0.f;
        lo[u].get(f);
        hi[u].get(g);
#pragma unroll
        for (int i = 0; i < 8; ++i) ss += f[i] * f[i] + g[i] * g[i];
#pragma unroll
        for (int off = 1; off < LPR; off <<= 1) ss += __shfl_xor_sync(0xffffffffu, ss, off);
        const float ms = ss * (1.f / D) + P.eps;
        float inv = rsqrtf(ms);
        constexpr uint32_t LEAST = 27u << 23, MOST = 227u << 23;  // 2^-100, 2^100
        const uint32_t bits = __float_as_uint(ms);
        if (__builtin_expect(__any_sync(0xffffffffu, bits - LEAST >= MOST - LEAST), 0)) {
          const bool up = bits < LEAST, down = bits >= MOST;
          const float by = up ? 1.2676506e30f : down ? 8.4703295e-22f : 1.f;  // 2^100, 2^-70: the squares of whatever is left stay in range
          float s2 = 0.f;
#pragma unroll
          for (int i = 0; i < 8; ++i) s2 += (f[i] * by) * (f[i] * by) + (g[i] * by) * (g[i] * by);
#pragma unroll
          for (int off = 1; off < LPR; off <<= 1) s2 += __shfl_xor_sync(0xffffffffu, s2, off);
          const float again = rsqrtf(s2 * (1.f / D) + (up ? P.eps_up : P.eps_down)) * by;
          if (up || down) inv = again;
        }
        float a[8], z[8], w[8], v[8];
        wl.get(w);
        wh.get(v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p = weighted ? f[i] * inv * w[i] : f[i] * inv, q = weighted ? g[i] * inv * v[i] : g[i] * inv;
          a[i] = p * cs[i] - q * sn[i];
          z[i] = q * cs[i] + p * sn[i];
        }
        if (in && h < S.H) {
          T* dst = o + (int64_t)h * P.N * D;
          store8f(dst, a);
          store8f(dst + H, z);
        }
      }
    }
  }
}

// A prompt gives a thread all heads of its token, eight of them (four in fp32) in flight: bound by memory (24/8 heads of 128 x 32768, bf16,
// 537 MB: two heads in flight 100 us, four 93, eight 89; 6.1 TB/s).  Fewer tokens have their heads dealt over blocks, two (one) at a
// time, since what a thread looks at behind the last head costs it as much as a head (8 tokens: 4.1 us, with eight at a time 6.6), and
// very few over the threads of a block as well (132 tokens of 28/4 heads: 4.5 us; 5001 of 14/2 heads of 64 in fp32: 9.7, and 11.0
// where the threads of a block share the heads although there are blocks enough).
template <int D, typename T>
cudaError_t launch_norm_rope(const NormRopeParams& P, cudaStream_t s) {
  constexpr int FEW = sizeof(T) == 2 ? 2 : 1;
  const int heads = std::max(P.side[0].H, P.side[1].H);
  const auto blocks = [&](int hl) { return (P.rows * (D / 16) + NR_THREADS / hl - 1) / (NR_THREADS / hl); };
  const int64_t want = 3 * 148;
  int hl = 1;
  while (hl < 8 && 2 * hl <= heads && blocks(hl) < 64) hl *= 2;
  const int64_t gx = blocks(hl);
  const unsigned gy = gx < want ? (unsigned)std::max<int64_t>(1, std::min<int64_t>((heads + hl - 1) / hl, (want + gx - 1) / gx)) : 1u;
  void (*kern)(NormRopeParams) = hl == 1 && gy == 1 && heads >= 8 ? atf_norm_rope_rows<D, 1, T, 4 * FEW>
                                 : hl == 1                        ? atf_norm_rope_rows<D, 1, T, FEW>
                                 : hl == 2                        ? atf_norm_rope_rows<D, 2, T, FEW>
                                 : hl == 4                        ? atf_norm_rope_rows<D, 4, T, FEW>
                                                                  : atf_norm_rope_rows<D, 8, T, FEW>;
  return atf_launch_overlapped(kern, dim3((unsigned)gx, gy), NR_THREADS, 0, s, P);
}

}  // namespace

extern "C" atf_status atf_qk_norm_rope(const void* Q, const atf_row_strides* q_strides, const void* K,
                                       const atf_row_strides* k_strides, const void* q_weight, const void* k_weight, double eps,
                                       void* Qo, void* Ko, int B, int Hq, int Hkv, int64_t N, int d, int dtype, const double* theta,
                                       int64_t pos0, const int64_t* positions, void* stream) {
  const char* who = "atf_qk_norm_rope";
  if (dtype != ATF_DTYPE_BF16 && dtype != ATF_DTYPE_F32) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: unknown dtype %d", who, dtype);
  if (d != 64 && d != 128) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: d must be 64 or 128 (got %d)", who, d);
  if (B < 1 || N < 1 || Hq < 0 || Hkv < 0 || Hq + Hkv < 1) return atf_fail(ATF_ERR_INVALID_ARG, "%s: bad shape", who);
  if (!theta || (Hq && (!Q || !Qo || !q_strides)) || (Hkv && (!K || !Ko || !k_strides)))
    return atf_fail(ATF_ERR_INVALID_ARG, "%s: null pointer", who);
  if (!(eps >= 0.0) || !std::isfinite(eps)) return atf_fail(ATF_ERR_INVALID_ARG, "%s: eps must be finite and not negative", who);
  if (N > (1ll << 40) / B / d) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: N too large", who);
  const int64_t unit = dtype == ATF_DTYPE_BF16 ? 8 : 4;  // elements of 16 bytes
  NormRopeParams P;
  const void* xs[2] = {Q, K};
  const void* ws[2] = {q_weight, k_weight};
  void* os[2] = {Qo, Ko};
  const atf_row_strides* st[2] = {q_strides, k_strides};
  const int hs[2] = {Hq, Hkv};
  for (int k = 0; k < 2; ++k) {
    P.side[k] = NormRopeSide{xs[k], ws[k], os[k], 0, 0, 0, hs[k]};
    if (!hs[k]) continue;
    if (((uintptr_t)xs[k] | (uintptr_t)os[k] | (uintptr_t)ws[k]) & 15)
      return atf_fail(ATF_ERR_INVALID_ARG, "%s: pointers must be 16-byte aligned", who);
    if (st[k]->batch % unit || st[k]->row % unit || st[k]->head % unit)
      return atf_fail(ATF_ERR_INVALID_ARG, "%s: strides must be multiples of 16 bytes", who);
    P.side[k].batch = st[k]->batch;
    P.side[k].row = st[k]->row;
    P.side[k].head = st[k]->head;
  }
  P.positions = positions;
  P.N = N;
  P.rows = (int64_t)B * N;
  P.pos0 = pos0;
  P.eps = (float)eps;
  P.eps_up = (float)std::ldexp(eps, 200);
  P.eps_down = (float)std::ldexp(eps, -140);
  for (int r = 0; r < ATF_MAX_PAIRS; ++r) {
    if (r < d / 2 && !std::isfinite(theta[r])) return atf_fail(ATF_ERR_INVALID_ARG, "%s: theta[%d] is not finite", who, r);
    P.turn[r] = r < d / 2 ? theta[r] / 6.283185307179586476925 : 0.0;
  }
  if (P.rows * (d / 16) / NR_THREADS >= 0x7FFFFFFF) return atf_fail(ATF_ERR_UNSUPPORTED, "%s: B*N too large", who);
  cudaStream_t s = (cudaStream_t)stream;
  ATF_CUDA_CHECK(dtype == ATF_DTYPE_BF16
                     ? (d == 64 ? launch_norm_rope<64, __nv_bfloat16>(P, s) : launch_norm_rope<128, __nv_bfloat16>(P, s))
                     : (d == 64 ? launch_norm_rope<64, float>(P, s) : launch_norm_rope<128, float>(P, s)));
  return ATF_OK;
}
