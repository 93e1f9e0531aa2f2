// Attention over a packed cache (packed.cuh): o = sum_j softmax_j(scale * q . k_j) v_j with k_j = s * code, v_j likewise, per group of
// 32 elements.  The I * g query rows that share a cache are the columns of
//     S^T = K Q^T          A = codes of 16 keys x 16 elements, B = queries (16 elements x 8 columns)
//     O^T = V^T P^T        A = codes of 16 elements x 16 keys, B = weights (16 keys x 8 columns)
// on mma.m16n8k16 with fp16 inputs and fp32 sums.  Rows are read once, 9 bytes for 16 elements, so a step of one token is bound by HBM
// as long as unpacking keeps up: about 1.1 instructions per element in place of the multiplications of 1 to 8 heads.
//
// Unpacking: the code + 8 is an integer u of 4 bits.  The word AND 0x000f000f holds two of them as the fp16 pair (u, u) * 2^-24
// (subnormals, which the multiplication takes as they are), AND 0x00f000f0 two as u * 2^-20; a shift by 8 gives the other four.  No
// addition takes the 8 away: sum u q = sum code q + 8 sum q, so the sums of Q.K start at -8 sum q, and P.V counts the sum of its own
// rounded weights with one more MMA per group.  What that costs is digits: sums of up to 23 times what remains, at fp32's step.  It
// is far below the rounding of bf16 outputs, and 30 times above that of fp32 ones (relative error 5e-6 measured), so fp32 caches take the
// codes themselves, one fp16 addition per pair, and join P.V's sums tile by tile outside the MMA.
//
// Numbers: a query row is brought to a largest magnitude of 2^10 .. 2^11 by a power of two, so that bf16 values are exact in fp16 (fp32
// values are two fp16 numbers, 22 bits, and two MMAs).  Weights are p * 2^12 (fp16, 11 bits; two numbers for fp32) times the
// value's scale, brought to 1 .. 8 by a power of two per group and warp (f below); softmax statistics and all sums are fp32.
//
// Every warp streams tiles of 32 rows of its own through its own ring of shared memory (cp.async.bulk, one mbarrier a slot) and keeps
// its own maximum, sums and outputs: warps wait for nobody until the end, where they meet in shared memory, and CTAs that share a
// cache in the workspace (packed_combine).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "packed.cuh"
#include "tc_common.cuh"

namespace bm {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kStages = 3;
constexpr float kShift = 12.f;                // weights are p * 2^12
constexpr int kMaxSplitCtas = 1184;           // CTAs of a call whose caches are shared (8 per SM)

__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, const float* c) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2*>(&x)); }
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ float exp2_approx(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127
__device__ __forceinline__ void bulk_load(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
               ::"r"(tc::smem_u32(dst)), "l"(src), "r"(bytes), "r"(tc::smem_u32(bar)) : "memory");
}
// Bounded wait for a slot's copies.  One that gives up records BM_ERR_TIMEOUT; its warp then takes no further tile.
__device__ __forceinline__ bool slot_full(uint64_t* b, uint32_t parity, int* status) {
  const uint32_t addr = tc::smem_u32(b);
#pragma unroll 1
  for (int left = tc::kWaitLimit; left > 0; --left) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(addr), "r"(parity), "r"(tc::kWaitSleepNs) : "memory");
    if (ok) return true;
  }
  *reinterpret_cast<volatile int*>(status) = tc::kErrTimeout;
  return false;
}
// n words of 32 bits at once
template <int N>
__device__ __forceinline__ void lds(const void* p, uint32_t* w) {
  if constexpr (N == 4) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
  } else if constexpr (N == 2) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Two codes of a word as an fp16 pair: kHigh takes bits 4 .. 7 of both halves, else bits 0 .. 3.
template <bool kSigned, bool kHigh>
__device__ __forceinline__ uint32_t codes(uint32_t w) {
  const uint32_t u = w & (kHigh ? 0x00f000f0u : 0x000f000fu);
  if constexpr (!kSigned) return u;
  const uint32_t x = u | 0x64006400u;   // 1024 + u, 1024 + 16 u
  const __half2 h = *reinterpret_cast<const __half2*>(&x);
  const __half2 y = kHigh ? __hfma2(h, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hsub2(h, __float2half2_rn(1032.f));
  return *reinterpret_cast<const uint32_t*>(&y);
}

struct AttendArgs {
  PackedView c;
  const void* q;
  int64_t q_sample, q_token;
  int32_t I;
  const int32_t* lens;
  const int32_t* first;
  void* out;
  float* partial;
  float mul;          // scale * log2(e)
  int32_t splits, query_tiles;
};

// One CTA's share of one cache, for a tile of 8 NT query rows: rows [lo, hi) of the cache.  PIECES fp16 numbers per query and weight.
template <typename T, int D, int NT>
struct Attend {
  static constexpr bool kSigned = sizeof(T) == 4;   // the MMAs take codes, not codes + 8
  static constexpr int G = D / kPackedGroup, kPieces = sizeof(T) == 4 ? 2 : 1, kCols = 8 * NT;
  static constexpr int kCodes = kPackedTile * D / 2, kScales = kPackedTile * G * 2, kSlot = 2 * (kCodes + kScales);
  static constexpr int kRing = kWarps * kStages * kSlot, kMerge = kWarps * 8 * D * 4;
  static constexpr int kQuery = NT > 1 ? NT * kPieces * G * 2 * 32 * 8 : 0;   // B fragments of Q, where registers do not hold them
  static constexpr int kSmem = (kRing > kMerge ? kRing : kMerge) + kQuery;
};

template <typename T, int D, int NT>
__global__ void __launch_bounds__(kThreads, NT == 1 ? (sizeof(T) == 4 ? 3 : 4) : 2) packed_attend_kernel(AttendArgs a) {
  using A = Attend<T, D, NT>;
  constexpr int G = A::G, P = A::kPieces;
  constexpr bool kSigned = A::kSigned;
  constexpr float kEven = kSigned ? 1.f : 0x1p24f, kOdd = kSigned ? 1.f : 0x1p20f;   // what a code of the MMA's has to be multiplied by
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ __align__(8) uint64_t bars[kWarps * kStages];
  __shared__ float stat_m[kWarps][A::kCols], stat_l[kWarps][A::kCols];
  const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32, r = lane / 4, c = lane % 4;
  if (tid == 0) {
    for (int i = 0; i < kWarps * kStages; ++i) tc::mbar_init(&bars[i], 1);
    tc::mbar_fence_init();
  }
  __syncthreads();
  pdl_wait();
  pdl_release();

  const int split = blockIdx.x % a.splits, qt = (blockIdx.x / a.splits) % a.query_tiles;
  const int unit = blockIdx.x / (a.splits * a.query_tiles);
  const int smp = unit / a.c.Hkv, head = unit % a.c.Hkv, g = a.c.g, cols = a.I * g;
  const int col0 = qt * A::kCols, cols_here = min(A::kCols, cols - col0);
  const int len = min(max(a.lens[smp], 0), a.c.capacity);
  const int lo = a.first != nullptr ? max(a.first[smp], 0) : 0;
  // query i sees the rows [lo, len - (I - 1 - i)); this tile's queries are (col0 / g) .. (col0 + cols_here - 1) / g
  const int i_last = (col0 + cols_here - 1) / g;
  const int least = len - (a.I - 1 - col0 / g), hi = len - (a.I - 1 - i_last);
  const int t_lo = lo / kPackedTile, tiles = hi > lo ? (hi + kPackedTile - 1) / kPackedTile - t_lo : 0;
  const int t0 = (int)((long long)tiles * split / a.splits), t1 = (int)((long long)tiles * (split + 1) / a.splits);
  const int mine = t1 - t0 > warp ? (t1 - t0 - warp + kWarps - 1) / kWarps : 0;   // tiles t0 + warp, + kWarps, ...

  unsigned char* ring = smem + warp * kStages * A::kSlot;
  uint64_t* bar = bars + warp * kStages;
  const size_t row_base = (size_t)unit * a.c.stride;
  auto issue = [&](int n) {   // the warp's n-th tile into slot n % kStages
    const size_t row = row_base + (size_t)(t_lo + t0 + warp + n * kWarps) * kPackedTile;
    unsigned char* slot = ring + (n % kStages) * A::kSlot;
    uint64_t* b = bar + n % kStages;
    tc::mbar_expect_tx(b, A::kSlot);
    bulk_load(slot, a.c.k_codes + row * (D / 2), A::kCodes, b);
    bulk_load(slot + A::kCodes, a.c.k_scales + row * G, A::kScales, b);
    bulk_load(slot + A::kCodes + A::kScales, a.c.v_scales + row * G, A::kScales, b);
    bulk_load(slot + A::kCodes + 2 * A::kScales, a.c.v_codes + row * (D / 2), A::kCodes, b);
  };
  if (lane == 0)
    for (int n = 0; n < kStages && n < mine; ++n) issue(n);

  // ---- queries: lane (r, c) has the elements 32 g + 8 c .. + 7 of column 8 nt + r -------------------------------------------
  uint32_t bq[NT == 1 ? P * G * 4 : 1];        // [piece][group][two k-steps][b0, b1]
  float start[NT][G][2], colmul[NT][2];        // of columns 8 nt + 2 c, + 1
  uint32_t* bq_smem = reinterpret_cast<uint32_t*>(smem + A::kSmem - A::kQuery);
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int col = col0 + 8 * nt + r;
    float x[G][8];
    float most = 0.f;
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[gi][j] = 0.f;
      if (col < cols) {
        const T* p = static_cast<const T*>(a.q) + smp * a.q_sample + (col / g) * a.q_token + ((size_t)head * g + col % g) * D + 32 * gi + 8 * c;
        if constexpr (sizeof(T) == 2) {
          Elem<T>::unpack(ld_global_16(p), x[gi]);
        } else {
          Elem<T>::unpack(ld_global_16(p), x[gi]);
          Elem<T>::unpack(ld_global_16(p + 4), x[gi] + 4);
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) most = fmaxf(most, fabsf(x[gi][j]));
    }
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 1));
    most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, 2));
    // the largest magnitude to 2^10 .. 2^11; an infinite row stays so, and its logits become NaN
    const int e = most > 0.f && most < INFINITY ? min(10 - (int)((__float_as_uint(most) >> 23) & 255u) + 127, 100) : 0;
    const float up = pow2(e);
    float mul = a.mul * kEven * pow2(-e);
    float sums[G];
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      float sum = 0.f;
      float v[2][8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = x[gi][j] * up;
        v[0][j] = __half2float(__float2half_rn(y));
        sum += v[0][j];
        if constexpr (P == 2) {
          v[1][j] = __half2float(__float2half_rn(y - v[0][j]));
          sum += v[1][j];
        }
      }
#pragma unroll
      for (int pc = 0; pc < P; ++pc) {
        // the k-steps take the elements (0, 4 | 1, 5) and (2, 6 | 3, 7); the codes of odd elements come 16 times as large
        constexpr float odd = kOdd / kEven;
        const uint32_t w[4] = {pack(v[pc][0], v[pc][4]), pack(v[pc][1] * odd, v[pc][5] * odd), pack(v[pc][2], v[pc][6]),
                               pack(v[pc][3] * odd, v[pc][7] * odd)};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          if constexpr (NT == 1) bq[(pc * G + gi) * 4 + k] = w[k];
          else if (warp == 0) bq_smem[((((nt * P + pc) * G + gi) * 2 + k / 2) * 32 + lane) * 2 + k % 2] = w[k];
        }
      }
      sum += __shfl_xor_sync(0xffffffffu, sum, 1);
      sum += __shfl_xor_sync(0xffffffffu, sum, 2);
      sums[gi] = kSigned ? 0.f * sum : sum * (-8.f / kEven);   // (a row that is not finite stays so)
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {   // from the column 8 nt + r of this lane to the columns 2 c + j of the sums
      const int from = 4 * (2 * c + j);
      colmul[nt][j] = __shfl_sync(0xffffffffu, mul, from);
#pragma unroll
      for (int gi = 0; gi < G; ++gi) start[nt][gi][j] = __shfl_sync(0xffffffffu, sums[gi], from);
    }
  }
  if constexpr (NT > 1) __syncthreads();

  float m[NT][2], l[NT][2], o[NT][G][2][4], ow[NT][4];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    m[nt][0] = m[nt][1] = -INFINITY;
    l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
    for (int k = 0; k < 4; ++k) ow[nt][k] = 0.f;
#pragma unroll
    for (int gi = 0; gi < G; ++gi)
#pragma unroll
      for (int k = 0; k < 8; ++k) o[nt][gi][k / 4][k % 4] = 0.f;
  }
  int f[G];                     // value scales are taken times 2^f
  uint32_t f2[G];               // 2^f as a pair
  float bound[G];               // the scales' magnitudes up to which f is good
#pragma unroll
  for (int gi = 0; gi < G; ++gi) { f[gi] = 15; f2[gi] = 0x78007800u; bound[gi] = 0x1p-12f; }

  auto tile = [&](auto masked_tag, int row0, const unsigned char* slot) {
    constexpr bool kMasked = decltype(masked_tag)::value;
    const unsigned char* kc = slot;
    const unsigned char* ks = slot + A::kCodes;
    const unsigned char* vs = ks + A::kScales;
    const unsigned char* vc = vs + A::kScales;

    // ---- logits, in units of log2 --------------------------------------------------------------------------------------
    float s[2][NT][4];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[sub][nt][k] = 0.f;
      // the MMA's row r is the key r / 2 + 4 (r % 2), so that a lane's four keys in P.V are c, c + 4, c + 8, c + 12
      const int key = sub * 16 + r / 2 + 4 * (r % 2);
      uint32_t w0[G], w1[G], sc[2][G / 2];
      lds<G>(kc + key * (D / 2) + c * 4 * G, w0);
      lds<G>(kc + (key + 8) * (D / 2) + c * 4 * G, w1);
      lds<G / 2>(ks + key * G * 2, sc[0]);
      lds<G / 2>(ks + (key + 8) * G * 2, sc[1]);
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        const uint32_t x0 = w0[gi] >> 8, x1 = w1[gi] >> 8;
        const uint32_t a0[4] = {codes<kSigned, false>(w0[gi]), codes<kSigned, false>(w1[gi]), codes<kSigned, true>(w0[gi]),
                                codes<kSigned, true>(w1[gi])};
        const uint32_t a1[4] = {codes<kSigned, false>(x0), codes<kSigned, false>(x1), codes<kSigned, true>(x0), codes<kSigned, true>(x1)};
        const float2 p0 = unpack(sc[0][gi / 2]), p1 = unpack(sc[1][gi / 2]);
        const float s0 = gi % 2 ? p0.y : p0.x, s1 = gi % 2 ? p1.y : p1.x;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          float acc[4] = {start[nt][gi][0], start[nt][gi][1], start[nt][gi][0], start[nt][gi][1]};
#pragma unroll
          for (int pc = 0; pc < P; ++pc) {
            if constexpr (NT == 1) {
              const uint32_t* b = bq + (pc * G + gi) * 4;
              mma(acc, a0, b[0], b[1], acc);
              mma(acc, a1, b[2], b[3], acc);
            } else {
              const uint32_t* b = bq_smem + ((((nt * P + pc) * G + gi) * 2) * 32 + lane) * 2;
              uint32_t b0[2], b1[2];
              lds<2>(b, b0);
              lds<2>(b + 64, b1);
              mma(acc, a0, b0[0], b0[1], acc);
              mma(acc, a1, b1[0], b1[1], acc);
            }
          }
          s[sub][nt][0] = fmaf(s0, acc[0], s[sub][nt][0]);
          s[sub][nt][1] = fmaf(s0, acc[1], s[sub][nt][1]);
          s[sub][nt][2] = fmaf(s1, acc[2], s[sub][nt][2]);
          s[sub][nt][3] = fmaf(s1, acc[3], s[sub][nt][3]);
        }
      }
    }

    // ---- softmax, running ----------------------------------------------------------------------------------------------
    bool grown = false;
    float top[NT][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = -INFINITY;
        const int seen = kMasked ? len - (a.I - 1 - (col0 + 8 * nt + 2 * c + j) / g) : 0;
#pragma unroll
        for (int sub = 0; sub < 2; ++sub)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float& x = s[sub][nt][2 * k + j];
            x *= colmul[nt][j];
            if constexpr (kMasked) {
              const int row = row0 + sub * 16 + 8 * k + r / 2 + 4 * (r % 2);
              if (row < lo || row >= seen) x = -INFINITY;
            }
            t = fmaxf(t, x);
          }
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
        t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
        top[nt][j] = fmaxf(m[nt][j], t);
        grown |= top[nt][j] > m[nt][j];
      }
    if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        float k[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          k[j] = m[nt][j] == top[nt][j] ? 1.f : exp2_approx(m[nt][j] - top[nt][j]);   // (both -inf: nothing seen yet)
          m[nt][j] = top[nt][j];
          l[nt][j] *= k[j];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) ow[nt][i] *= k[i % 2];
#pragma unroll
        for (int gi = 0; gi < G; ++gi)
#pragma unroll
          for (int i = 0; i < 8; ++i) o[nt][gi][i / 4][i % 4] *= k[i % 2];
      }
    }
    // weights p * 2^12: lane (r, c) ends with the query r and the keys c, c + 4 (b0) and c + 8, c + 12 (b1) of every 16
    uint32_t w[2][NT][P][2];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const float m0 = m[nt][0] == -INFINITY ? 0.f : m[nt][0] - kShift, m1 = m[nt][1] == -INFINITY ? 0.f : m[nt][1] - kShift;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const float p0 = exp2_approx(s[sub][nt][2 * k] - m0), p1 = exp2_approx(s[sub][nt][2 * k + 1] - m1);
          l[nt][0] += p0;
          l[nt][1] += p1;
          const uint32_t h = pack(p0, p1);
          w[sub][nt][0][k] = transpose8x8(h);
          if constexpr (P == 2) {
            const float2 back = unpack(h);
            w[sub][nt][P - 1][k] = transpose8x8(pack(p0 - back.x, p1 - back.y));
          }
        }
    }

    // ---- f: every lane looks at one row's scales -----------------------------------------------------------------------
    {
      uint32_t sc[G / 2];
      lds<G / 2>(vs + lane * G * 2, sc);
      bool over = false;
      float mag[G];
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        const float2 p = unpack(sc[gi / 2]);
        mag[gi] = fabsf(gi % 2 ? p.y : p.x);
        over |= !(mag[gi] <= bound[gi]);
      }
      if (__any_sync(0xffffffffu, over)) {
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          const uint32_t most = __reduce_max_sync(0xffffffffu, mag[gi] < INFINITY ? __float_as_uint(mag[gi]) : 0u);
          if (__uint_as_float(most) > bound[gi]) {
            const int next = max(-15, 127 - (int)(most >> 23));   // the largest scale to 1 .. 2
            const float k = pow2(next - f[gi]);
            f[gi] = next;
            f2[gi] = pack(pow2(next), pow2(next));
            bound[gi] = pow2(3 - next);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
              for (int i = 0; i < 8; ++i) o[nt][gi][i / 4][i % 4] *= k;
              if (r == gi) { ow[nt][0] *= k; ow[nt][1] *= k; }
            }
          }
          // A group whose scale is not finite is NaN for the queries that see it and nothing for the others: its scale becomes 0
          // in the slot, and the group's outputs of those queries NaN.
          const uint32_t bad = __ballot_sync(0xffffffffu, !(mag[gi] < INFINITY));
          if (bad != 0) {
            if (bad >> lane & 1) *reinterpret_cast<unsigned short*>(const_cast<unsigned char*>(vs) + (lane * G + gi) * 2) = 0;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int j = 0; j < 2; ++j) {
                const int seen = len - (a.I - 1 - (col0 + 8 * nt + 2 * c + j) / g);
                const int from = max(lo - row0, 0), to = min(seen - row0, 32);
                const uint32_t rows = to > from ? (0xffffffffu >> (32 - (to - from))) << from : 0u;
                if (bad & rows)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[nt][gi][i / 2][2 * (i % 2) + j] = __int_as_float(0x7fffffff);
              }
          }
        }
        tc::fence_async_smem();   // (the slot is filled by an asynchronous copy again)
        __syncwarp();
      }
    }

    // ---- outputs -------------------------------------------------------------------------------------------------------
    uint32_t v[2][4][G / 2], sv[2][4][G / 2];
#pragma unroll
    for (int sub = 0; sub < 2; ++sub)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int key = sub * 16 + 4 * k + c;
        lds<G / 2>(vc + key * (D / 2) + r * 2 * G, v[sub][k]);
        lds<G / 2>(vs + key * G * 2, sv[sub][k]);
      }
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const uint32_t half = gi % 2 ? 0x7632u : 0x5410u;
      float part[kSigned ? NT : 1][2][4];
      if constexpr (kSigned)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 8; ++i) part[nt][i / 4][i % 4] = 0.f;
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        const uint32_t x0 = __byte_perm(v[sub][0][gi / 2], v[sub][1][gi / 2], half), x1 = __byte_perm(v[sub][2][gi / 2], v[sub][3][gi / 2], half);
        const uint32_t y0 = x0 >> 8, y1 = x1 >> 8;
        const uint32_t a0[4] = {codes<kSigned, false>(x0), codes<kSigned, true>(x0), codes<kSigned, false>(x1), codes<kSigned, true>(x1)};
        const uint32_t a1[4] = {codes<kSigned, false>(y0), codes<kSigned, true>(y0), codes<kSigned, false>(y1), codes<kSigned, true>(y1)};
        [[maybe_unused]] const uint32_t ones = r == gi ? 0x3c003c00u : 0u;
        [[maybe_unused]] const uint32_t a2[4] = {ones, 0u, ones, 0u};   // row gi: the sum of the weights
        const uint32_t sc[2] = {mul2(__byte_perm(sv[sub][0][gi / 2], sv[sub][1][gi / 2], half), f2[gi]),
                                mul2(__byte_perm(sv[sub][2][gi / 2], sv[sub][3][gi / 2], half), f2[gi])};
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          uint32_t b[P][2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if constexpr (P == 1) {
              b[0][k] = mul2(w[sub][nt][0][k], sc[k]);
            } else {
              const float2 hi2 = unpack(w[sub][nt][0][k]), lo2 = unpack(w[sub][nt][P - 1][k]), s2 = unpack(sc[k]);
              const float y0f = (hi2.x + lo2.x) * s2.x, y1f = (hi2.y + lo2.y) * s2.y;
              b[0][k] = pack(y0f, y1f);
              const float2 back = unpack(b[0][k]);
              b[P - 1][k] = pack(y0f - back.x, y1f - back.y);
            }
          }
          float(&to)[2][4] = *(kSigned ? &part[kSigned ? nt : 0] : &o[nt][gi]);
#pragma unroll
          for (int pc = 0; pc < P; ++pc) {
            mma(to[0], a0, b[pc][0], b[pc][1], to[0]);
            mma(to[1], a1, b[pc][0], b[pc][1], to[1]);
            if constexpr (!kSigned) mma(ow[nt], a2, b[pc][0], b[pc][1], ow[nt]);
          }
        }
      }
      if constexpr (kSigned)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int i = 0; i < 8; ++i) o[nt][gi][i / 4][i % 4] += part[nt][i / 4][i % 4];
    }
  };

  int n = 0;
#pragma unroll 1
  for (; n < mine; ++n) {
    if (!slot_full(bar + n % kStages, (n / kStages) & 1, a.c.status)) break;
    const int row0 = (t_lo + t0 + warp + n * kWarps) * kPackedTile;
    const unsigned char* slot = ring + (n % kStages) * A::kSlot;
    if (row0 < lo || row0 + kPackedTile > least) tile(std::true_type{}, row0, slot);
    else tile(std::false_type{}, row0, slot);
    __syncwarp();
    if (lane == 0 && n + kStages < mine) issue(n + kStages);
  }
#pragma unroll 1
  for (int k = n + 1; k < min(n + kStages, mine); ++k) slot_full(bar + k % kStages, (k / kStages) & 1, a.c.status);   // a wait gave up: what is in flight lands first

  // ---- the warps' results meet ---------------------------------------------------------------------------------------------
#pragma unroll
  for (int nt = 0; nt < NT; ++nt)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float t = l[nt][j];
      t += __shfl_xor_sync(0xffffffffu, t, 4);
      t += __shfl_xor_sync(0xffffffffu, t, 8);
      t += __shfl_xor_sync(0xffffffffu, t, 16);
      if (r == 0) {
        stat_m[warp][8 * nt + 2 * c + j] = m[nt][j];
        stat_l[warp][8 * nt + 2 * c + j] = t;
      }
    }
  float* merge = reinterpret_cast<float*>(smem);   // [warp][8 columns][D], over the ring
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    __syncthreads();   // (the ring, or the columns before, have been read)
    float k[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int col = 8 * nt + 2 * c + j;
      float top = stat_m[0][col];
#pragma unroll
      for (int i = 1; i < kWarps; ++i) top = fmaxf(top, stat_m[i][col]);
      k[j] = m[nt][j] == top ? 1.f : exp2_approx(m[nt][j] - top);
    }
#pragma unroll
    for (int gi = 0; gi < G; ++gi) {
      const float down = pow2(-f[gi]) ;
      float sum[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) sum[j] = 8.f * __shfl_sync(0xffffffffu, ow[nt][j], 4 * gi + c);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const float by = k[j] * down;
        float4 x;
        x.x = (o[nt][gi][0][j] * kEven - sum[j]) * by;
        x.y = (o[nt][gi][0][2 + j] * kOdd - sum[j]) * by;
        x.z = (o[nt][gi][1][j] * kEven - sum[j]) * by;
        x.w = (o[nt][gi][1][2 + j] * kOdd - sum[j]) * by;
        *reinterpret_cast<float4*>(merge + (warp * 8 + 2 * c + j) * D + 32 * gi + 4 * r) = x;
      }
    }
    __syncthreads();
    for (int i = tid; i < 8 * D / 4; i += kThreads) {
      const int col = i / (D / 4), at = (i % (D / 4)) * 4, cc = 8 * nt + col;
      if (cc >= cols_here) continue;
      float top = stat_m[0][cc], sum = 0.f;
#pragma unroll
      for (int k2 = 1; k2 < kWarps; ++k2) top = fmaxf(top, stat_m[k2][cc]);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k2 = 0; k2 < kWarps; ++k2) {
        const float wm = stat_m[k2][cc];
        sum += stat_l[k2][cc] * (wm == top ? 1.f : exp2_approx(wm - top));
        const float4 y = *reinterpret_cast<const float4*>(merge + (k2 * 8 + col) * D + at);
        x.x += y.x; x.y += y.y; x.z += y.z; x.w += y.w;
      }
      if (a.splits == 1) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;   // (a query that sees no row has a row of zeros)
        T* p = static_cast<T*>(a.out) + (((size_t)smp * a.I + (col0 + cc) / g) * a.c.Hq + (size_t)head * g + (col0 + cc) % g) * D + at;
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(p) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
        } else {
          const __nv_bfloat162 y0 = __floats2bfloat162_rn(x.x * inv, x.y * inv), y1 = __floats2bfloat162_rn(x.z * inv, x.w * inv);
          *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
        }
      } else {   // [unit][query tile][split][column][D + 4]: the sums, then the maximum and the sum of the weights
        float* p = a.partial + ((size_t)blockIdx.x * A::kCols + cc) * (D + 4);
        *reinterpret_cast<float4*>(p + at) = x;
        if (at == 0) *reinterpret_cast<float2*>(p + D) = make_float2(top, sum);
      }
    }
  }
}

// Joins the shares of a cache that several CTAs had: a thread has four elements of a query row.
template <typename T, int D>
__global__ void __launch_bounds__(128) packed_combine_kernel(AttendArgs a, int cols_per_tile) {
  constexpr int kPerRow = D / 4;
  pdl_wait();
  const long long i = (long long)blockIdx.x * (128 / kPerRow) + threadIdx.x / kPerRow;   // (unit, column)
  const int g = a.c.g, cols = a.I * g, at = (threadIdx.x % kPerRow) * 4;
  if (i >= (long long)a.c.nsamples * a.c.Hkv * cols) return;
  const int unit = (int)(i / cols), col = (int)(i % cols), qt = col / cols_per_tile;
  const size_t step = (size_t)cols_per_tile * (D + 4);
  const float* p = a.partial + ((size_t)(unit * (long long)a.query_tiles + qt) * a.splits * cols_per_tile + col % cols_per_tile) * (D + 4);
  float top = -INFINITY, sum = 0.f;
  for (int k = 0; k < a.splits; ++k) top = fmaxf(top, p[k * step + D]);
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k = 0; k < a.splits; ++k) {
    const float2 st = *reinterpret_cast<const float2*>(p + k * step + D);
    if (st.y == 0.f) continue;   // nothing seen there
    const float by = st.x == top ? 1.f : exp2_approx(st.x - top);
    const float4 y = *reinterpret_cast<const float4*>(p + k * step + at);
    sum += st.y * by;
    x.x += y.x * by; x.y += y.y * by; x.z += y.z * by; x.w += y.w * by;
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  const int smp = unit / a.c.Hkv, head = unit % a.c.Hkv;
  T* out = static_cast<T*>(a.out) + (((size_t)smp * a.I + col / g) * a.c.Hq + (size_t)head * g + col % g) * D + at;
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(out) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
  } else {
    const __nv_bfloat162 y0 = __floats2bfloat162_rn(x.x * inv, x.y * inv), y1 = __floats2bfloat162_rn(x.z * inv, x.w * inv);
    *reinterpret_cast<uint2*>(out) = make_uint2(*reinterpret_cast<const uint32_t*>(&y0), *reinterpret_cast<const uint32_t*>(&y1));
  }
}

// Query rows that a CTA takes, in units of 8.
int column_tiles(int64_t cols) { return cols <= 8 ? 1 : cols <= 16 ? 2 : 4; }

int choose_splits(int64_t ctas, int max_len) {
  const int64_t most = (max_len + kWarps * kPackedTile - 1) / (kWarps * kPackedTile);   // a tile for every warp
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, kMaxSplitCtas / std::max<int64_t>(ctas, 1)));
}

template <typename T, int D, int NT>
cudaError_t launch_nt(const AttendArgs& args, int64_t units, int max_len, cudaStream_t st) {
  using A = Attend<T, D, NT>;
  AttendArgs a = args;
  const int64_t cols = (int64_t)a.I * a.c.g;
  const int64_t tiles = (cols + A::kCols - 1) / A::kCols;
  a.query_tiles = (int)tiles;
  a.splits = choose_splits(units * tiles, max_len);
  const int64_t ctas = units * tiles * a.splits;
  if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
  static SmemConfigured configured;
  if (cudaError_t err = configured.ensure(packed_attend_kernel<T, D, NT>, A::kSmem); err != cudaSuccess) return err;
  cudaError_t err = launch_dependent(packed_attend_kernel<T, D, NT>, dim3((unsigned)ctas), dim3(kThreads), A::kSmem, st, a);
  count_launch();
  if (err == cudaSuccess && a.splits > 1) {
    const int64_t per_block = 128 / (D / 4), blocks = (units * cols + per_block - 1) / per_block;
    err = launch_dependent(packed_combine_kernel<T, D>, dim3((unsigned)blocks), dim3(128), 0, st, a, (int)A::kCols);
    count_launch();
  }
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_t(const AttendArgs& a, int64_t units, int max_len, cudaStream_t st) {
  switch (column_tiles((int64_t)a.I * a.c.g)) {
    case 1: return launch_nt<T, D, 1>(a, units, max_len, st);
    case 2: return launch_nt<T, D, 2>(a, units, max_len, st);
    default: return launch_nt<T, D, 4>(a, units, max_len, st);
  }
}

}  // namespace

size_t packed_attend_workspace(int d, int g, int queries) {
  // CTAs that share caches, each with up to this many query rows
  return (size_t)kMaxSplitCtas * 8 * column_tiles((int64_t)queries * g) * (d + 4) * sizeof(float);
}

cudaError_t launch_packed_attend(int dtype, int d, const PackedView& c, const PackedAttend& p, cudaStream_t st) {
  AttendArgs a;
  a.c = c;
  a.q = p.q; a.q_sample = p.q_sample; a.q_token = p.q_token;
  a.I = p.I;
  a.lens = p.lens; a.first = p.first;
  a.out = p.out;
  a.partial = p.partial;
  a.mul = p.scale * 1.4426950408889634f;
  a.splits = a.query_tiles = 1;
  const int64_t units = (int64_t)c.nsamples * c.Hkv;
  if (dtype == 0) return d == 64 ? launch_t<float, 64>(a, units, p.max_len, st) : launch_t<float, 128>(a, units, p.max_len, st);
  return d == 64 ? launch_t<__nv_bfloat16, 64>(a, units, p.max_len, st) : launch_t<__nv_bfloat16, 128>(a, units, p.max_len, st);
}

}  // namespace bm
