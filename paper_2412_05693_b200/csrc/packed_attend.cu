// Attention over a packed cache (packed.cuh): o = sum_j softmax_j(scale * q . k_j) v_j with k_j = s * code, v_j likewise, per group of
// 32 elements.  The I * g query rows that share a cache are the columns of
//     S^T = K Q^T          A = codes of 16 keys x 16 elements, B = queries (16 elements x 8 columns)
//     O^T = V^T P^T        A = codes of 16 elements x 16 keys, B = weights (16 keys x 8 columns)
// on warp-level MMAs with fp32 sums.  Rows are read once, 9 bytes for 16 elements, so a step of one token is bound by HBM as long as
// unpacking keeps up, which is what everything here is about.  (Cycles a scheduler needs per operation, measured: logic on 32 bits, byte
// permutations, conversions and fp16 arithmetic 2; mma.m16n8k16 of fp16 and mma.m16n8k32 of 8-bit integers 8; the latter of e4m3 34, so
// that it seems to be made of conversions and fp16 MMAs; ex2 8.)
//
// Unpacking: the code + 8 is an integer u of 4 bits.  The word AND 0x000f000f holds two of them as the fp16 pair (u, u) * 2^-24
// (subnormals, which the multiplication takes as they are), AND 0x00f000f0 two as u * 2^-20; a shift by 8 gives the other four.  AND
// 0x0f0f0f0f it holds four bytes, shifted by 4 the other four: half the work, where the other side of the product can be 8-bit integers.
// It can for up to four query rows, as two numbers each in two of the eight columns: q = 256 hi + lo, 15 bits with the sign for the row's
// largest element; a row whose largest element stands out gets 8 more in products of their own (kUneven).  No addition takes the 8 away:
// sum u q = sum code q + 8 sum q, so integer sums start at -8 sum q, fp32 ones at the sum over the groups of s * (-8 sum q), one small MMA
// of the scales and the queries' sums; P.V counts the sum of its own rounded weights with one more MMA per group.  What that costs is
// digits: sums of up to 23 times what remains, at fp32's step.  It is far below the rounding of bf16 outputs, and 30 times above that of
// fp32 ones (relative error 5e-6 measured), so fp32 caches take the codes themselves as fp16 numbers, one fp16 addition per pair, and join
// P.V's sums tile by tile outside the MMA.
//
// Numbers: a query row is brought to a largest magnitude of 2^13 .. 2^14 by a power of two for the integers (an element is off by 1/2 at
// most, by 1/256 with the third number), of 2^14 .. 2^15 for fp16, where bf16 values are exact (fp32: two numbers, 22 bits).  Weights are
// p * 2^shift (fp16, 11 bits; two numbers for fp32) times the value's scale; shift is 12, less where a scale of 2 or more would pass fp16
// (fp32: it stays, and a group's scales are taken times 2^lift, so that the largest of a group so far is where it keeps both numbers).  Only
// rows that some query of the tile sees count there.  The maximum that p refers to follows when logits pass it by 2 (in log2), not sooner.
// Softmax statistics and all sums are fp32.
//
// Work: the tiles of all caches of the call, one after another, are cut into equal runs, so that samples of unequal length cost no idle
// SMs and few long caches are shared by all.  A run is one warp's, which streams it through a ring of shared memory (one
// cp.async.bulk and one mbarrier per tile) and waits for nobody.  A cache that lies in one run is written out by its warp; of the others
// the sums go to the workspace, and packed_combine_kernel joins them.
//
// Measured in bursts (us, both kernels; share of the copy bandwidth over the rows' bytes; seconds of such calls meet the power limit and
// take 10 to 20 % more): d = 128, bf16, 384 samples of 1535 rows, 8 kv-heads, 8 query heads 113 (92 %), 32 118 (88 %), 64 135 (77 %); 32
// samples of 2048, 40 heads without groups 66 (87 %); one sample of 131072 35 (67 %); 16 of 4096 21 (55 %); 16 of 1472 14; one of 1024 7.4.
// d = 64, 96 samples of 4096, 64 / 16 heads 94 (73 %).  fp32, 8 samples of 8192, 32 / 8 heads 36 (32 %).  What bounds it: bytes in the first
// case (433 instructions per 32 rows, schedulers 54 % busy); the instructions with eight columns, at d = 64 and in fp32 (two MMAs and two
// weights for one); below a few thousand rows the way in (2 us until a warp knows its run, 1 to 3 until its queries are ready) and out (5 us
// with packed_combine_kernel).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "packed.cuh"
#include "tc_common.cuh"

namespace bm {
namespace {

constexpr int kWarps = 2;                     // independent of each other; one per CTA would cost 1 KB of shared memory more for each
constexpr int kWarpsPerSm = 12;
constexpr int kMostSms = 148;                 // that the workspace is sized for
constexpr int kFullShift = 12;
// Queries as integers: a row whose largest element is more than this many times the mean of its magnitudes (3.6 for normal values) gets a
// third number of 8 bits.  Without it an element is off by 2^-14 of the largest at most, so by 2^-11 of the mean: what fp16 does to weights.
// Measured (us; 384 samples of 1535 rows, 32 / 8 heads, d = 128 | 96 of 4096, 64 / 16, d = 64): two numbers 117 | 94, this 118 | 95 and 167 | 139
// where every tile of queries has such a row, three for every row 127 | 97.  With both halves of a tile side by side on the way of such rows
// 121 | 94 and 148 | 118.
constexpr float kUneven = 8.f;

__device__ __forceinline__ void mma(float* d, const uint32_t* a, uint32_t b0, uint32_t b1, const float* c) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(c[0]), "f"(c[1]), "f"(c[2]), "f"(c[3]));
}
// a: bytes without sign, b: with
__device__ __forceinline__ void mma_u8s8(int* d, const uint32_t* a, uint32_t b0, uint32_t b1, const uint32_t* c) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%11,%12,%13};"
      : "=r"(d[0]), "=r"(d[1]), "=r"(d[2]), "=r"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "r"(c[0]), "r"(c[1]), "r"(c[2]), "r"(c[3]));
}
// d = a (16 x 8) * b (8 x 8)
__device__ __forceinline__ void mma_k8(float* d, uint32_t a0, uint32_t a1, uint32_t b) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5}, {%6}, {%7,%7,%7,%7};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(b), "f"(0.f));
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
__device__ __forceinline__ bool slot_full(uint64_t* b, uint32_t parity, int* status, int limit = tc::kWaitLimit) {
  const uint32_t addr = tc::smem_u32(b);
#pragma unroll 1
  for (; limit > 0; --limit) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\nselp.b32 %0, 1, 0, p;\n}\n"
                 : "=r"(ok) : "r"(addr), "r"(parity), "r"(tc::kWaitSleepNs) : "memory");
    if (ok) return true;
  }
  *reinterpret_cast<volatile int*>(status) = tc::kErrTimeout;
  return false;
}
template <int N>   // N words of 32 bits at once
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
  float mul;              // scale * log2(e)
  int32_t query_tiles;    // of 8 (PAIR: 4) query rows, per cache
  int32_t runs;           // the most there may be: one for each warp of the grid
  int32_t slot_cols;      // query rows of a share in the workspace
  FastDiv by_g, by_query_tiles, by_cols, by_heads;
  int32_t* before;        // workspace: [nsamples + 1] tiles (of one kv-head and query tile) of the samples before each
  float* partial;         // workspace: [runs][2][slot_cols][D + 4] sums of a cache's share, their maximum and sum of weights
};

// PAIR: up to four query rows as 8-bit integers, each with two columns in Q.K and one of two in P.V (the other's weights are 0); else eight.
// Wider tiles of query rows unpack less often and hold more: two and four times as many columns were no faster with bf16 at 16 rows of a
// cache (16 samples of 4096 rows, 8 kv-heads, d = 128: 40 us, 42 now) and slower at 32 (93 against 60; fp32 204 against 109).
template <typename T, int D, bool PAIR>
struct Attend {
  static constexpr bool kSigned = sizeof(T) == 4;   // fp32: the MMAs take codes, not codes + 8
  static constexpr int G = D / kPackedGroup, kPieces = kSigned ? 2 : 1, kCols = PAIR ? 4 : 8;
  // Slots of the ring, warps per SM.  us, 384 samples of 1535 rows, 32 / 8 heads, d = 128, with 16 warps of 128 registers 142, 14 167, 12 of 168
  // 122, 10 137; four slots 121 against 118.
  static constexpr int kStages = 3, kResident = kWarpsPerSm;
  static constexpr int kQueryWords = kSigned ? 8 * G : PAIR ? 2 * G : 4 * G;   // B fragments of Q, words of a lane
  static constexpr int kWarpBytes = kStages * PackedLayout<D>::kBytes;
  // Shared memory of PAIR beside the ring: words that a lane has for its queries' third numbers, [group][b0, b1] and -8 times their sums
  // [group]; per warp what the other integer sums start at, quads of an MMA's C [group][c] (which would take 16 registers).
  static constexpr int kThirdWords = PAIR ? (3 * G + 3) / 4 * 4 : 0, kThirdBytes = kThirdWords * 4 * 32, kStartBytes = PAIR ? G * 4 * 16 : 0;
  static constexpr int kSmem = kWarps * (kWarpBytes + kThirdBytes + kStartBytes);
  static_assert(!PAIR || !kSigned, "");
};

// Self-test of that wait: a warp waits for copies that nobody issues.
__global__ void packed_wait_selftest_kernel(int* status) {
  __shared__ __align__(8) uint64_t bar;
  if (threadIdx.x == 0) {
    tc::mbar_init(&bar, 1);
    tc::mbar_fence_init();
  }
  __syncwarp();
  if (slot_full(&bar, 0, status, 1 << 16)) *status = 0;   // (never)
}

// The rows of a sample that some query sees: tiles first .. first + n - 1 of its caches.
struct Tiles {
  int len, lo, first, n;
};
__device__ __forceinline__ Tiles sample_tiles(const AttendArgs& a, int smp) {
  Tiles t;
  t.len = min(max(a.lens[smp], 0), a.c.capacity);
  t.lo = a.first != nullptr ? max(a.first[smp], 0) : 0;
  t.first = t.lo / kPackedTile;
  t.n = t.len > t.lo ? (t.len + kPackedTile - 1) / kPackedTile - t.first : 0;
  return t;
}
template <typename N>
__device__ __forceinline__ N warp_inclusive_sum(N x, int lane) {
#pragma unroll
  for (int step = 1; step < 32; step *= 2) {
    const N y = __shfl_up_sync(0xffffffffu, x, step);
    if (lane >= step) x += y;
  }
  return x;
}
// v tiles in w <= v runs: run j has the tiles [start(j), start(j + 1)).
struct Runs {
  long long each;
  int more;   // the first runs have one tile more
  __device__ __forceinline__ Runs(long long v, int w) {
    each = (unsigned long long)v >> 32 ? v / w : (long long)((uint32_t)v / (uint32_t)w);
    more = (int)(v - each * w);
  }
  __device__ __forceinline__ long long start(int j) const { return j * each + min(j, more); }
  __device__ __forceinline__ int of(long long tile) const {
    const long long longer = (each + 1) * more;
    const bool in_longer = tile < longer;
    const long long x = in_longer ? tile : tile - longer, by = in_longer ? each + 1 : each;
    return (in_longer ? 0 : more) + (int)((unsigned long long)(x | by) >> 32 ? x / by : (long long)((uint32_t)x / (uint32_t)by));
  }
};

// A place in the order of the call's tiles: sample, kv-head, query tile, tile.
struct Walk {
  int smp, head, qt, t, n, first;
  __device__ __forceinline__ void next_cache(const AttendArgs& a) {
    t = 0;
    if (++qt < a.query_tiles) return;
    qt = 0;
    if (++head < a.c.Hkv) return;
    head = 0;
    do {
      const Tiles x = sample_tiles(a, ++smp);
      n = x.n;
      first = x.first;
    } while (n == 0 && smp + 1 < a.c.nsamples);
  }
};

template <typename T>
__device__ __forceinline__ void store4(T* p, float x, float y, float z, float w) {
  if constexpr (sizeof(T) == 4) {
    *reinterpret_cast<float4*>(p) = make_float4(x, y, z, w);
  } else {
    const __nv_bfloat162 a = __floats2bfloat162_rn(x, y), b = __floats2bfloat162_rn(z, w);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
  }
}

template <typename T, int D, bool PAIR>
__global__ void __launch_bounds__(kWarps * 32, Attend<T, D, PAIR>::kResident / kWarps) packed_attend_kernel(AttendArgs a) {
  using A = Attend<T, D, PAIR>;
  using L = PackedLayout<D>;
  constexpr int G = A::G, P = A::kPieces, kStages = A::kStages, C = PAIR ? 1 : 2;   // C: columns of the sums that a lane has
  constexpr bool kSigned = A::kSigned;
  constexpr float kEven = kSigned ? 1.f : 0x1p24f, kOdd = kSigned ? 1.f : 0x1p20f;   // what a code of the fp16 MMAs has to be multiplied by
  constexpr float kKey = PAIR ? 1.f : kEven;
  constexpr int kMagic = 0x4b400000;   // integers up to 2^22 on top of it are that much above the fp32 number 1.5 * 2^23
  extern __shared__ __align__(128) unsigned char smem[];
  __shared__ __align__(8) uint64_t bars[kWarps][kStages];
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, r = lane / 4, c = lane % 4, run = blockIdx.x * kWarps + warp;
  unsigned char* ring = smem + warp * A::kWarpBytes;
  uint64_t* bar = bars[warp];
  [[maybe_unused]] auto start_at = [&](int gi) {   // this lane's quad
    return reinterpret_cast<int4*>(smem + kWarps * (A::kWarpBytes + A::kThirdBytes)) + (warp * G + gi) * 4 + c;
  };
  [[maybe_unused]] auto third_at = [&](int i) {    // this lane's word i
    return reinterpret_cast<int*>(smem + kWarps * A::kWarpBytes) + ((i / 4) * kWarps * 32 + (int)threadIdx.x) * 4 + i % 4;
  };
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) tc::mbar_init(&bar[i], 1);
    tc::mbar_fence_init();
  }
  __syncwarp();
  pdl_wait();
  pdl_release();

  // ---- this warp's run ------------------------------------------------------------------------------------------------------
  const int cols = a.I * a.c.g, per_sample = a.c.Hkv * a.query_tiles;
  // Lane i has the samples [i q, (i + 1) q): their tiles in all, and those before them.
  const int ns = a.c.nsamples, each_lane = (ns + 31) / 32, mine0 = lane * each_lane;
  auto tiles_at = [&](int smp) { return smp < ns ? sample_tiles(a, smp).n : 0; };
  int tiles_of_lane = 0;
#pragma unroll 4
  for (int i = 0; i < each_lane; ++i) tiles_of_lane += tiles_at(mine0 + i);
  // (the tiles of one kv-head of all samples fit 32 bits: 2^31 of them are 8 TB)
  const int up_to_lane = warp_inclusive_sum(tiles_of_lane, lane), total = __shfl_sync(0xffffffffu, up_to_lane, 31);
  const long long all = (long long)total * per_sample;
  if (run == 0) {   // for packed_combine_kernel
    int sum = up_to_lane - tiles_of_lane;
    for (int smp = mine0; smp < min(mine0 + each_lane, ns); ++smp) {
      a.before[smp] = sum;
      sum += tiles_at(smp);
    }
    if (lane == 0) a.before[ns] = total;
  }
  const int runs = (int)min((long long)a.runs, all);
  if (run >= runs) return;
  const Runs cut(all, runs);
  const long long begin = cut.start(run);
  int left = (int)(cut.start(run + 1) - begin), to_issue = left;
  Walk at;
  {
    const int src = __ffs(__ballot_sync(0xffffffffu, begin < (long long)up_to_lane * per_sample)) - 1;   // the lane whose samples `begin` is in
    int before = __shfl_sync(0xffffffffu, up_to_lane - tiles_of_lane, src);
    at.smp = src;
    at.n = __shfl_sync(0xffffffffu, tiles_of_lane, src);
    if (each_lane > 1) {
      for (int s0 = src * each_lane;; s0 += 32) {
        const int n = s0 + lane < (src + 1) * each_lane ? tiles_at(s0 + lane) : 0, up_to = before + warp_inclusive_sum(n, lane);
        const unsigned hit = __ballot_sync(0xffffffffu, begin < (long long)up_to * per_sample);
        if (hit != 0) {
          const int k = __ffs(hit) - 1;
          at.smp = s0 + k;
          at.n = __shfl_sync(0xffffffffu, n, k);
          before = __shfl_sync(0xffffffffu, up_to - n, k);
          break;
        }
        before = __shfl_sync(0xffffffffu, up_to, 31);
      }
    }
    at.first = a.first != nullptr ? max(a.first[at.smp], 0) / kPackedTile : 0;
    const long long in = begin - (long long)before * per_sample;
    const int unit = (unsigned long long)in >> 32 ? (int)(in / at.n) : (int)((uint32_t)in / (uint32_t)at.n);
    at.t = (int)(in - (long long)unit * at.n);
    at.head = a.by_query_tiles(unit);
    at.qt = unit - at.head * a.query_tiles;
  }
  Walk ahead = at;   // the next tile to fetch
  const uint8_t* from = nullptr;
  auto cache_tiles = [&](const Walk& w) {
    return a.c.data + (((size_t)w.smp * a.c.Hkv + w.head) * a.c.tiles + w.first + w.t) * L::kBytes;
  };
  from = cache_tiles(ahead);
  auto issue = [&](int slot) {
    if (to_issue == 0) return;
    --to_issue;
    if (lane == 0) {
      tc::mbar_expect_tx(bar + slot, L::kBytes);
      bulk_load(ring + slot * L::kBytes, from, L::kBytes, bar + slot);
    }
    from += L::kBytes;
    if (++ahead.t == ahead.n && to_issue > 0) {
      ahead.next_cache(a);
      from = cache_tiles(ahead);
    }
  };
#pragma unroll
  for (int i = 0; i < kStages; ++i) issue(i);

  int slot = 0;
  uint32_t parity = 0;
#pragma unroll 1
  while (left > 0) {
    // ---- one cache's share: its queries, lane (r, c) has the elements 32 g + 8 c .. + 7 of its column -----------------------
    const Tiles sample = sample_tiles(a, at.smp);
    const int len = sample.len, lo = sample.lo, share = min(at.n - at.t, left), col0 = at.qt * A::kCols;
    const int cols_here = min(A::kCols, cols - col0);
    // query i sees the rows [lo, len - (I - 1 - i)); the first of this tile's the rows below `least`, the last those below `most_rows`
    const int least = len - (a.I - 1 - a.by_g(col0)), most_rows = len - (a.I - 1 - a.by_g(col0 + cols_here - 1));
    uint32_t bq[A::kQueryWords];                 // [number][group][two k-steps][b0, b1], integers: [group][b0, b1]
    uint32_t start = 0;                          // B fragment of the -8 sum q: two fp16 numbers for each group
    float colmul[C];                             // of this lane's columns
    [[maybe_unused]] float not_finite = 0.f;     // integers: NaN where the column's query is not finite
    [[maybe_unused]] bool third = false;         // integers: some query of the tile has a third number
    {
      const int col = col0 + (PAIR ? r / 2 : r), query = a.by_g(col);
      const T* q = static_cast<const T*>(a.q) + at.smp * a.q_sample + query * a.q_token + ((size_t)at.head * a.c.g + col - query * a.c.g) * D + 8 * c;
      float x[G][8];
      uint32_t most_bits = 0;   // magnitudes compare as integers, what is not finite above the rest
      [[maybe_unused]] float mean = 0.f;   // of the magnitudes
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[gi][j] = 0.f;
        if (col < cols) {
          Elem<T>::unpack(ld_global_16(q + 32 * gi), x[gi]);
          if constexpr (kSigned) Elem<T>::unpack(ld_global_16(q + 32 * gi + 4), x[gi] + 4);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) most_bits = max(most_bits, __float_as_uint(x[gi][j]) & 0x7fffffffu);
        if constexpr (PAIR) {   // (divided first, so that no sum is infinite)
          float part = 0.f;
#pragma unroll
          for (int j = 0; j < 8; ++j) part = fmaf(fabsf(x[gi][j]), 1.f / D, part);
          mean += part;
        }
      }
      most_bits = max(most_bits, __shfl_xor_sync(0xffffffffu, most_bits, 1));
      most_bits = max(most_bits, __shfl_xor_sync(0xffffffffu, most_bits, 2));
      if constexpr (PAIR) {
        mean += __shfl_xor_sync(0xffffffffu, mean, 1);
        mean += __shfl_xor_sync(0xffffffffu, mean, 2);
      }
      // the largest magnitude to its place; a row that is not finite has NaN logits
      const bool finite = most_bits < 0x7f800000u;
      const int e = finite && most_bits > 0 ? min((PAIR ? 13 : 14) - (int)(most_bits >> 23) + 127, 100) : 0;
      if constexpr (PAIR) not_finite = __shfl_sync(0xffffffffu, finite ? 0.f : __int_as_float(0x7fffffff), 8 * c);
      const float up = pow2(e);
      // Above 0: times -inf it stays -inf.  Finite: next to the largest queries it may be above fp32, where the codes' 2^-24 makes up for it; logits
      // are 2^50 apart then or equal, with the largest number in its place too.
      const float mul = fminf(fmaxf(a.mul * kKey * pow2(-e), 0x1p-126f), 0x1.fffffep127f);
      if constexpr (PAIR) {
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          // On top of kMagic the low 16 bits are the integer y; its low byte is lo, the second one of y + 128 is hi.  b0 takes the
          // elements 0, 2, 4, 6, b1 the others.
          const float magic = __int_as_float(r % 2 ? kMagic : kMagic + 128);
          const uint32_t two = r % 2 ? 0x0040u : 0x0051u;
          int sum = 0;
#pragma unroll
          for (int odd = 0; odd < 2; ++odd) {
            uint32_t y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) y[j] = __float_as_uint(fmaf(x[gi][2 * j + odd], up, magic));
            const uint32_t b = __byte_perm(__byte_perm(y[0], y[1], two), __byte_perm(y[2], y[3], two), 0x5410);
            bq[gi * 2 + odd] = b;
            sum = __dp4a((int)b, 0x01010101, sum);
          }
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          const int of_hi = -8 * __shfl_sync(0xffffffffu, sum, 8 * c), of_lo = -8 * __shfl_sync(0xffffffffu, sum, 8 * c + 4) + kMagic;
          if (r == 0) *start_at(gi) = make_int4(of_hi, of_lo, of_hi, of_lo);
        }
        third = __any_sync(0xffffffffu, finite && __uint_as_float(most_bits) * (1.f / kUneven) > mean);
        if (third) {
          // what rounding to integers left, in 256ths (a half would be 128 of them: 127)
#pragma unroll
          for (int gi = 0; gi < G; ++gi) {
            int sum = 0;
#pragma unroll
            for (int odd = 0; odd < 2; ++odd) {
              uint32_t y[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const float v = x[gi][2 * j + odd] * up, left = v - ((v + __int_as_float(kMagic)) - __int_as_float(kMagic));
                y[j] = __float_as_uint(fminf(left * 256.f, 127.f) + __int_as_float(kMagic));   // (its low byte)
              }
              const uint32_t b = __byte_perm(__byte_perm(y[0], y[1], 0x0040), __byte_perm(y[2], y[3], 0x0040), 0x5410);
              *third_at(2 * gi + odd) = r % 2 ? 0 : (int)b;
              sum = __dp4a((int)b, 0x01010101, sum);
            }
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            *third_at(2 * G + gi) = -8 * __shfl_sync(0xffffffffu, sum, 8 * c);
          }
        }
      } else {
        float sums[G];
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          float sum = 0.f;
          float v[2][8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            v[0][j] = x[gi][j] * up;
            sum += v[0][j];   // (of bf16 values fp16 has all digits that count)
            if constexpr (P == 2) v[1][j] = v[0][j] - __half2float(__float2half_rn(v[0][j]));
          }
#pragma unroll
          for (int pc = 0; pc < P; ++pc)   // the k-steps take the elements (0, 4 | 1, 5) and (2, 6 | 3, 7); codes of odd ones come 16 times as large
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const float by = k % 2 ? kOdd / kEven : 1.f;
              bq[(pc * G + gi) * 4 + k] = pack(v[pc][k] * by, v[pc][k + 4] * by);
            }
          sum += __shfl_xor_sync(0xffffffffu, sum, 1);
          sum += __shfl_xor_sync(0xffffffffu, sum, 2);
          sums[gi] = sum * (-8.f / kKey);
        }
        // k = 2 c, 2 c + 1 of the start's MMA: the groups 0 .. G - 1 of the first fp16 number, then those of the second
#pragma unroll
        for (int k = 0; k < 2 * G; k += 2) {
          float s0 = sums[k % G], s1 = sums[k % G + 1];
          if (k >= G) {
            s0 -= __half2float(__float2half_rn(s0));
            s1 -= __half2float(__float2half_rn(s1));
          }
          if (c == k / 2) start = pack(s0, s1);
        }
      }
#pragma unroll
      for (int j = 0; j < C; ++j) colmul[j] = __shfl_sync(0xffffffffu, mul, 4 * (2 * c + j));   // from this lane's column to the sums'
      __syncwarp();
    }
    auto column = [&](int j) { return PAIR ? c : 2 * c + j; };   // of the sums, from col0

    // Weights are 2^(logit + mneg), mneg = shift - m rounded down: where m leaves no room for the shift they are the smaller ones, and all that
    // was summed with another mneg follows by the difference of the two.
    float m[C], mneg[C], l[C], o[G][2][4], ow[4];
#pragma unroll
    for (int j = 0; j < C; ++j) {
      m[j] = -INFINITY;
      mneg[j] = l[j] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) ow[k] = 0.f;
#pragma unroll
    for (int gi = 0; gi < G; ++gi)
#pragma unroll
      for (int k = 0; k < 8; ++k) o[gi][k / 4][k % 4] = 0.f;
    int shift = kFullShift;
    // fp32: the shift stays, and every group's value scales are taken times a power of two of its own, so that small ones keep their second number
    [[maybe_unused]] int lift[G];
#pragma unroll
    for (int gi = 0; gi < G; ++gi) lift[gi] = kSigned ? 15 : 0;
    auto over_of = [](int total) { return 0x7fff7fffu - 0x00010001u * (((28 - total) << 10) - 1); };
    constexpr int kOvers = kSigned ? G / 2 : 1;
    uint32_t over_add[kOvers];                      // carries into bit 15 what is 2^(13 - shift - lift) or more (fp32: of the lane's words)
#pragma unroll
    for (int i = 0; i < kOvers; ++i) over_add[i] = over_of(shift + (kSigned ? 15 : 0));

    auto rescale = [&](const float* k) {   // everything that was summed with the weights
#pragma unroll
      for (int j = 0; j < C; ++j) {
        l[j] *= k[j];
        if constexpr (!kSigned) ow[j] *= k[j];
      }
#pragma unroll
      for (int gi = 0; gi < G; ++gi)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < C; ++j) o[gi][i / 2][2 * (i % 2) + j] *= k[j];
    };

    auto tile = [&](auto masked_tag, int row0, unsigned char* in) {
      constexpr bool kMasked = decltype(masked_tag)::value;

      // ---- value scales: too large for the shift, or not finite? -------------------------------------------------------------
      {
        uint32_t sc[G / 2], over = 0;
        lds<G / 2>(in + L::kValueScales + lane * 2 * G, sc);
#pragma unroll
        for (int i = 0; i < G / 2; ++i) over |= (sc[i] & 0x7fff7fffu) + over_add[i % kOvers];
        if (__any_sync(0xffffffffu, (over & 0x80008000u) != 0)) {
          uint32_t largest = 0;   // of rows that some query of this tile sees: the others may hold anything, and get weights of 0
          const bool counts = !kMasked || (row0 + lane >= lo && row0 + lane < most_rows);
#pragma unroll
          for (int gi = 0; gi < G; ++gi) {   // lane = row
            unsigned short* place = reinterpret_cast<unsigned short*>(in + L::value_scale(lane, gi));
            const uint32_t mag = *place & 0x7fffu;
            const uint32_t bad = __ballot_sync(0xffffffffu, mag >= 0x7c00u);
            const uint32_t mine = !counts || mag >= 0x7c00u ? 0u : mag;
            largest = max(largest, mine);
            if constexpr (kSigned) {
              const int next = min(shift + lift[gi], 12 - ((int)(__reduce_max_sync(0xffffffffu, mine) >> 10) - 15));
              if (next < shift + lift[gi]) {
                const float k = pow2(next - shift - lift[gi]);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[gi][i / 4][i % 4] *= k;
                lift[gi] = next - shift;
              }
            }
            // A group whose scale is not finite is NaN for the queries that see it and nothing for the others: its scale becomes 0 in
            // the slot, and the group's outputs of those queries NaN.
            if (bad != 0) {
              if (bad >> lane & 1) *place = 0;
#pragma unroll
              for (int j = 0; j < C; ++j) {
                const int seen = len - (a.I - 1 - a.by_g(col0 + column(j)));
                const int b0 = max(lo - row0, 0), b1 = min(seen - row0, 32);
                const uint32_t rows = b1 > b0 ? (0xffffffffu >> (32 - (b1 - b0))) << b0 : 0u;
                if (bad & rows)
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[gi][i / 2][2 * (i % 2) + j] = __int_as_float(0x7fffffff);
              }
            }
          }
          if constexpr (kSigned) {
            // the lane's words: of the groups lane % 2 * (G / 2) ..
#pragma unroll
            for (int i = 0; i < kOvers; ++i) over_add[i] = over_of(shift + (lane % 2 ? lift[G / 2 + i] : lift[i]));
          } else {
            largest = __reduce_max_sync(0xffffffffu, largest);
            const int next = min(shift, 12 - ((int)(largest >> 10) - 15));   // the largest scale is below 2^(13 - shift)
            if (next < shift) {
              float ks[C];
#pragma unroll
              for (int j = 0; j < C; ++j) {
                const float before = mneg[j];
                if (m[j] != -INFINITY) mneg[j] = __fsub_rd((float)next, m[j]);
                ks[j] = exp2_approx(mneg[j] - before);
              }
              rescale(ks);
              shift = next;
              over_add[0] = over_of(next);
            }
          }
          tc::fence_async_smem();   // (the slot is filled by an asynchronous copy again)
          __syncwarp();
        }
      }

      // ---- logits -------------------------------------------------------------------------------------------------------------
      float s[2][2][C];   // [16 keys][key + 8][column]
#pragma unroll
      for (int sub = 0; sub < 2; ++sub) {
        // the MMA's row r is the key r / 2 + 4 (r % 2), so that a lane's four keys in P.V are c, c + 4, c + 8, c + 12
        const int key = sub * 16 + r / 2 + 4 * (r % 2);
        uint32_t w0[G], w1[G], sc[2][G / 2];
        lds<G>(in + key * (D / 2) + c * 4 * G, w0);
        lds<G>(in + (key + 8) * (D / 2) + c * 4 * G, w1);
        lds<G / 2>(in + L::kKeyScales + key * G * 2, sc[0]);
        lds<G / 2>(in + L::kKeyScales + (key + 8) * G * 2, sc[1]);
        float first[4] = {0.f, 0.f, 0.f, 0.f};
        if constexpr (!kSigned && !PAIR) {   // (G = 2: lanes c >= 2 multiply by 0)
          mma_k8(first, G == 4 && (c & 1) ? sc[0][G / 2 - 1] : sc[0][0], G == 4 && (c & 1) ? sc[1][G / 2 - 1] : sc[1][0], start);
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int j = 0; j < C; ++j) s[sub][k][j] = first[2 * k + j];
#pragma unroll
        for (int gi = 0; gi < G; ++gi) {
          const float2 p0 = unpack(sc[0][gi / 2]), p1 = unpack(sc[1][gi / 2]);
          const float s0 = gi % 2 ? p0.y : p0.x, s1 = gi % 2 ? p1.y : p1.x;
          if constexpr (PAIR) {
            const uint32_t a0[4] = {w0[gi] & 0x0f0f0f0fu, w1[gi] & 0x0f0f0f0fu, w0[gi] >> 4 & 0x0f0f0f0fu, w1[gi] >> 4 & 0x0f0f0f0fu};
            int acc[4];
            uint32_t from8[4];
            lds<4>(start_at(gi), from8);
            mma_u8s8(acc, a0, bq[2 * gi], bq[2 * gi + 1], from8);
            // |sum code q| < 32 * 8 * 2^14 = 2^22
            s[sub][0][0] = fmaf(s0, __int_as_float(acc[0] * 256 + acc[1]) - __int_as_float(kMagic), s[sub][0][0]);
            s[sub][1][0] = fmaf(s1, __int_as_float(acc[2] * 256 + acc[3]) - __int_as_float(kMagic), s[sub][1][0]);
          } else {
            const uint32_t x0 = w0[gi] >> 8, x1 = w1[gi] >> 8;
            const uint32_t a0[4] = {codes<kSigned, false>(w0[gi]), codes<kSigned, false>(w1[gi]), codes<kSigned, true>(w0[gi]),
                                    codes<kSigned, true>(w1[gi])};
            const uint32_t a1[4] = {codes<kSigned, false>(x0), codes<kSigned, false>(x1), codes<kSigned, true>(x0), codes<kSigned, true>(x1)};
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int pc = 0; pc < P; ++pc) {
              const uint32_t* b = bq + (pc * G + gi) * 4;
              mma(acc, a0, b[0], b[1], acc);
              mma(acc, a1, b[2], b[3], acc);
            }
#pragma unroll
            for (int j = 0; j < C; ++j) {
              s[sub][0][j] = fmaf(s0, acc[j], s[sub][0][j]);
              s[sub][1][j] = fmaf(s1, acc[2 + j], s[sub][1][j]);
            }
          }
        }
      }

      // ---- softmax, running -----------------------------------------------------------------------------------------------------
      bool grown = PAIR && third;
      float top[C];
#pragma unroll
      for (int j = 0; j < C; ++j) {
        if constexpr (kMasked) {
          const int seen = len - (a.I - 1 - a.by_g(col0 + column(j)));
#pragma unroll
          for (int sub = 0; sub < 2; ++sub)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int row = row0 + sub * 16 + 8 * k + r / 2 + 4 * (r % 2);
              if (row < lo || row >= seen) s[sub][k][j] = -INFINITY;
            }
        }
        top[j] = fmaxf(fmaxf(s[0][0][j], s[0][1][j]), fmaxf(s[1][0][j], s[1][1][j])) * colmul[j];
        grown |= top[j] > m[j] + 2.f;
      }
      if (__any_sync(0xffffffffu, grown)) {
        if constexpr (PAIR) {
          if (third) {   // (rare: what this needs is fetched again, so that nothing is kept for it)
            uint32_t low[2 * G], from[G];
#pragma unroll
            for (int i = 0; i < 2 * G; i += 4) lds<4>(third_at(i), low + i);
            lds<G>(third_at(2 * G), from);
#pragma unroll 1   // (unrolled it costs the other rows registers)
            for (int sub = 0; sub < 2; ++sub) {
              const int key = sub * 16 + r / 2 + 4 * (r % 2);
              uint32_t w0[G], w1[G], sc[2][G / 2];
              lds<G>(in + key * (D / 2) + c * 4 * G, w0);
              lds<G>(in + (key + 8) * (D / 2) + c * 4 * G, w1);
              lds<G / 2>(in + L::kKeyScales + key * G * 2, sc[0]);
              lds<G / 2>(in + L::kKeyScales + (key + 8) * G * 2, sc[1]);
              float d0 = 0.f, d1 = 0.f;
#pragma unroll
              for (int gi = 0; gi < G; ++gi) {
                const uint32_t a0[4] = {w0[gi] & 0x0f0f0f0fu, w1[gi] & 0x0f0f0f0fu, w0[gi] >> 4 & 0x0f0f0f0fu, w1[gi] >> 4 & 0x0f0f0f0fu};
                const uint32_t from8[4] = {from[gi], 0u, from[gi], 0u};
                int acc[4];
                mma_u8s8(acc, a0, low[2 * gi], low[2 * gi + 1], from8);
                const float2 p0 = unpack(sc[0][gi / 2]), p1 = unpack(sc[1][gi / 2]);
                d0 = fmaf(gi % 2 ? p0.y : p0.x, (float)acc[0], d0);
                d1 = fmaf(gi % 2 ? p1.y : p1.x, (float)acc[2], d1);
              }
              // (hidden logits stay -inf, whatever the row's scale)
              if (sub == 0) {
                if (s[0][0][0] != -INFINITY) s[0][0][0] = fmaf(d0, 0x1p-8f, s[0][0][0]);
                if (s[0][1][0] != -INFINITY) s[0][1][0] = fmaf(d1, 0x1p-8f, s[0][1][0]);
              } else {
                if (s[1][0][0] != -INFINITY) s[1][0][0] = fmaf(d0, 0x1p-8f, s[1][0][0]);
                if (s[1][1][0] != -INFINITY) s[1][1][0] = fmaf(d1, 0x1p-8f, s[1][1][0]);
              }
            }
            top[0] = fmaxf(fmaxf(s[0][0][0], s[0][1][0]), fmaxf(s[1][0][0], s[1][1][0])) * colmul[0];
          }
        }
        float k[C];
#pragma unroll
        for (int j = 0; j < C; ++j) {
          float t = top[j];
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
          t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
          t = fmaxf(m[j], fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16)));
          const float next = t == -INFINITY ? 0.f : __fsub_rd((float)shift, t);
          k[j] = m[j] == -INFINITY ? 1.f : exp2_approx(next - mneg[j]);   // (nothing seen yet: nothing summed)
          m[j] = t;
          mneg[j] = next;
        }
        rescale(k);
      }
      // weights p * 2^shift: lane (r, c) ends with the column r and the keys c, c + 4 (b0) and c + 8, c + 12 (b1) of every 16
      uint32_t w[2][P][2];
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float p[2] = {0.f, 0.f};
#pragma unroll
          for (int j = 0; j < C; ++j) {
            // The logit is rounded before m is taken off, as m was: a largest one of 2^25 may be 2 above its rounded self, one of 2^30 64.  fp32
            // has its last digits of smaller ones without.
            const float rounded = __fadd_rn(__fmul_rn(s[sub][k][j], colmul[j]), mneg[j]);
            p[j] = exp2_approx(kSigned && fabsf(mneg[j]) < 0x1p18f ? fmaf(s[sub][k][j], colmul[j], mneg[j]) : rounded);
            l[j] += p[j];
          }
          const uint32_t h = pack(p[0], p[1]);
          w[sub][0][k] = transpose8x8(h);
          if constexpr (P == 2) {
            const float2 back = unpack(h);
            w[sub][P - 1][k] = transpose8x8(pack(p[0] - back.x, p[1] - back.y));
          }
        }

      // ---- outputs ---------------------------------------------------------------------------------------------------------------
      uint32_t v[2][2][G], sv[2][2][G];   // of the keys (c, c + 4) and (c + 8, c + 12) of every 16, a word per group
#pragma unroll
      for (int sub = 0; sub < 2; ++sub)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          lds<G>(in + L::kValueCodes + (((sub * 2 + k) * 8 + r) * 4 + c) * G * 4, v[sub][k]);
          lds<G>(in + L::kValueScales + ((sub * 4 + c) * 2 + k) * G * 4, sv[sub][k]);
        }
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        float part[2][4];
        [[maybe_unused]] const float lifted = pow2(lift[gi]);
        if constexpr (kSigned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) part[i / 4][i % 4] = 0.f;
        }
#pragma unroll
        for (int sub = 0; sub < 2; ++sub) {
          const uint32_t x0 = v[sub][0][gi], x1 = v[sub][1][gi], y0 = x0 >> 8, y1 = x1 >> 8;
          const uint32_t a0[4] = {codes<kSigned, false>(x0), codes<kSigned, true>(x0), codes<kSigned, false>(x1), codes<kSigned, true>(x1)};
          const uint32_t a1[4] = {codes<kSigned, false>(y0), codes<kSigned, true>(y0), codes<kSigned, false>(y1), codes<kSigned, true>(y1)};
          [[maybe_unused]] const uint32_t ones = r == gi ? 0x3c003c00u : 0u;
          [[maybe_unused]] const uint32_t a2[4] = {ones, 0u, ones, 0u};   // row gi: the sum of the weights
          uint32_t b[P][2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            if constexpr (P == 1) {
              b[0][k] = mul2(w[sub][0][k], sv[sub][k][gi]);
            } else {
              const float2 hi2 = unpack(w[sub][0][k]), lo2 = unpack(w[sub][P - 1][k]), s2 = unpack(sv[sub][k][gi]);
              const float y0f = (hi2.x + lo2.x) * (s2.x * lifted), y1f = (hi2.y + lo2.y) * (s2.y * lifted);
              b[0][k] = pack(y0f, y1f);
              const float2 back = unpack(b[0][k]);
              b[P - 1][k] = pack(y0f - back.x, y1f - back.y);
            }
          }
          float(&to)[2][4] = kSigned ? part : o[gi];
#pragma unroll
          for (int pc = 0; pc < P; ++pc) {
            mma(to[0], a0, b[pc][0], b[pc][1], to[0]);
            mma(to[1], a1, b[pc][0], b[pc][1], to[1]);
            if constexpr (!kSigned) mma(ow, a2, b[pc][0], b[pc][1], ow);
          }
        }
        if constexpr (kSigned) {
#pragma unroll
          for (int i = 0; i < 8; ++i) o[gi][i / 4][i % 4] += part[i / 4][i % 4];
        }
      }
    };

#pragma unroll 1
    for (int t = at.t; t < at.t + share; ++t) {
      if (!slot_full(bar + slot, parity, a.c.status)) {   // gave up: what is in flight lands first, then the warp ends
#pragma unroll 1
        for (int k = 0; k < min(kStages, left - (t - at.t)); ++k) {   // (this slot's copy among them)
          slot_full(bar + slot, parity, a.c.status);
          if (++slot == kStages) { slot = 0; parity ^= 1; }
        }
        return;
      }
      const int row0 = (at.first + t) * kPackedTile;
      unsigned char* in = ring + slot * L::kBytes;
      if (row0 >= lo && row0 + kPackedTile <= least) tile(std::false_type{}, row0, in);
      else if (row0 < most_rows) tile(std::true_type{}, row0, in);
      __syncwarp();
      issue(slot);
      if (++slot == kStages) { slot = 0; parity ^= 1; }
    }

    // ---- the cache's share is done ------------------------------------------------------------------------------------------------
    const bool whole = share == at.n;
    float* to = a.partial + ((size_t)run * 2 + (at.t == 0 ? 1 : 0)) * a.slot_cols * (D + 4);
#pragma unroll
    for (int j = 0; j < C; ++j) {
      l[j] += __shfl_xor_sync(0xffffffffu, l[j], 4);
      l[j] += __shfl_xor_sync(0xffffffffu, l[j], 8);
      l[j] += __shfl_xor_sync(0xffffffffu, l[j], 16);
      if constexpr (PAIR)
        if (l[j] != 0.f) l[j] += not_finite;   // (seen something)
      const int cc = column(j), col = col0 + cc, query = a.by_g(col);
      const float by_all = whole ? (l[j] == 0.f ? 0.f : 1.f / l[j]) : 1.f;   // (a query that sees no row has a row of zeros)
      T* out = static_cast<T*>(a.out) + (((size_t)at.smp * a.I + query) * a.c.Hq + (size_t)at.head * a.c.g + col - query * a.c.g) * D + 4 * r;
#pragma unroll
      for (int gi = 0; gi < G; ++gi) {
        const float sum = kSigned ? 0.f : 8.f * __shfl_sync(0xffffffffu, ow[j], 4 * gi + c);
        const float by = by_all * pow2(-lift[gi]);
        const float x0 = (o[gi][0][j] * kEven - sum) * by, x1 = (o[gi][0][2 + j] * kOdd - sum) * by;
        const float x2 = (o[gi][1][j] * kEven - sum) * by, x3 = (o[gi][1][2 + j] * kOdd - sum) * by;
        if (cc < cols_here) {
          if (whole) store4(out + 32 * gi, x0, x1, x2, x3);
          else store4(to + cc * (D + 4) + 32 * gi + 4 * r, x0, x1, x2, x3);
        }
      }
      // what the weights are relative to
      if (!whole && r == 0 && cc < cols_here)
        *reinterpret_cast<float2*>(to + cc * (D + 4) + D) = make_float2(m[j] == -INFINITY ? m[j] : -mneg[j], l[j]);
    }
    left -= share;
    if (left > 0) at.next_cache(a);
  }
}

// Joins the shares of the caches that several runs had, and writes the zeros of queries whose caches have no tiles.  A row is one
// (sample, kv-head, query row): D / 4 lanes have four elements each, kGroups of such lanes every kGroups-th share.
struct Joined {
  float top = -INFINITY, sum = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  __device__ __forceinline__ void add(float2 st, float4 v) {
    if (st.y == 0.f) return;   // nothing seen there
    const float next = fmaxf(top, st.x);
    const float k = top == next ? 1.f : exp2_approx(top - next), by = st.x == next ? 1.f : exp2_approx(st.x - next);
    top = next;
    sum = sum * k + st.y * by;
    o.x = o.x * k + v.x * by; o.y = o.y * k + v.y * by; o.z = o.z * k + v.z * by; o.w = o.w * k + v.w * by;
  }
};
template <typename T, int D, int kGroups>
__global__ void __launch_bounds__(kGroups == 1 ? 128 : kGroups * D / 4) packed_combine_kernel(AttendArgs a, int log_tile_cols) {
  constexpr int kPerRow = D / 4, kRows = kGroups == 1 ? 128 / kPerRow : 1, kBatch = 4;
  __shared__ float4 sums[kGroups][kPerRow];
  __shared__ float2 stats[kGroups];
  pdl_wait();
  const int x = threadIdx.x % kPerRow, y = threadIdx.x / kPerRow;
  const long long i = (long long)blockIdx.x * kRows + (kGroups == 1 ? y : 0);
  const int part = kGroups == 1 ? 0 : y;
  const int g = a.c.g, cols = a.I * g, at = x * 4;
  if (i >= (long long)a.c.nsamples * a.c.Hkv * cols) return;   // (uniform where kGroups > 1)
  const int unit = a.by_cols((int)i), col = (int)i - unit * cols, qt = col >> log_tile_cols, smp = a.by_heads(unit), head = unit - smp * a.c.Hkv;
  const int query = a.by_g(col);
  const long long per_sample = (long long)a.c.Hkv * a.query_tiles;
  const int before = a.before[smp], n = a.before[smp + 1] - before;
  const long long all = a.before[a.c.nsamples] * per_sample;
  T* out = static_cast<T*>(a.out) + (((size_t)smp * a.I + query) * a.c.Hq + (size_t)head * g + col - query * g) * D + at;
  if (n == 0) {
    if (part == 0) store4(out, 0.f, 0.f, 0.f, 0.f);
    return;
  }
  const Runs cut(all, (int)min((long long)a.runs, all));
  const long long begin = before * per_sample + ((long long)head * a.query_tiles + qt) * n;
  const int j0 = cut.of(begin), j1 = cut.of(begin + n - 1);
  if (j0 == j1) return;   // written out by its warp
  const size_t row = (size_t)a.slot_cols * (D + 4);
  const float* p = a.partial + (size_t)(col - (qt << log_tile_cols)) * (D + 4);
  Joined mine;
  for (int j = j0 + part; j <= j1; j += kBatch * kGroups) {
    float2 st[kBatch];
    float4 v[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int jb = j + b * kGroups;
      const float* q = p + (size_t)(2 * (long long)jb + (jb == j0 ? 1 : 0)) * row;   // the first share begins with the cache
      st[b] = make_float2(0.f, 0.f);
      v[b] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (jb <= j1) {
        st[b] = *reinterpret_cast<const float2*>(q + D);
        v[b] = *reinterpret_cast<const float4*>(q + at);
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) mine.add(st[b], v[b]);
  }
  if constexpr (kGroups > 1) {   // halves: a tree over the groups
    for (int half = kGroups / 2; half > 0; half /= 2) {
      if (y >= half && y < 2 * half) {
        sums[y][x] = mine.o;
        if (x == 0) stats[y] = make_float2(mine.top, mine.sum);
      }
      __syncthreads();
      if (y < half) mine.add(stats[y + half], sums[y + half][x]);
    }
    if (y != 0) return;
  }
  const float inv = mine.sum == 0.f ? 0.f : 1.f / mine.sum;
  store4(out, mine.o.x * inv, mine.o.y * inv, mine.o.z * inv, mine.o.w * inv);
}

size_t before_bytes(int nsamples) { return ((size_t)nsamples + 1 + 63) / 64 * 64 * sizeof(int32_t); }

template <typename T, int D, bool PAIR>
cudaError_t launch_columns(const AttendArgs& args, void* workspace, int max_len, cudaStream_t st) {
  using A = Attend<T, D, PAIR>;
  AttendArgs a = args;
  const int64_t units = (int64_t)a.c.nsamples * a.c.Hkv, cols = (int64_t)a.I * a.c.g;
  a.query_tiles = (int)((cols + A::kCols - 1) / A::kCols);
  const int64_t most_tiles = units * a.query_tiles * ((max_len + kPackedTile - 1) / kPackedTile);
  // From 256 tiles on a warp takes two at least, and there are fewer shares to join.  us with one / with two each: 128 tiles 6.8 / 7.7,
  // 256 7.7 / 7.1, 2048 11.3 / 10.0 (one sample) and 9.6 / 9.2 (four), 3200 8.2 / 7.8.
  const int64_t most_runs = most_tiles < 256 ? most_tiles : (most_tiles + 1) / 2;
  a.runs = (int)std::min<int64_t>(most_runs, std::min(sm_count(), kMostSms) * A::kResident);
  a.slot_cols = (int)std::min<int64_t>(A::kCols, cols);
  a.by_g = FastDiv((uint32_t)a.c.g);
  a.by_query_tiles = FastDiv((uint32_t)a.query_tiles);
  a.by_cols = FastDiv((uint32_t)cols);
  a.by_heads = FastDiv((uint32_t)a.c.Hkv);
  a.before = static_cast<int32_t*>(workspace);
  a.partial = reinterpret_cast<float*>(static_cast<char*>(workspace) + before_bytes(a.c.nsamples));
  static SmemConfigured configured;
  if (cudaError_t err = configured.ensure(packed_attend_kernel<T, D, PAIR>, A::kSmem); err != cudaSuccess) return err;
  cudaError_t err;
  {
    ProfileScope prof(kPacked, st);
    err = launch_dependent(packed_attend_kernel<T, D, PAIR>, dim3((a.runs + kWarps - 1) / kWarps), dim3(kWarps * 32), A::kSmem, st, a);
  }
  count_launch();
  if (err != cudaSuccess) return err;
  const int64_t rows = units * cols;
  const int64_t shares = a.runs / (units * a.query_tiles);   // of a cache, more or less
  ProfileScope prof(kPacked, st);
  constexpr int kLogCols = PAIR ? 2 : 3;
  static_assert(1 << kLogCols == A::kCols, "");
  if (shares >= 32) {
    constexpr int kGroups = 4096 / D;   // 1024 threads
    err = launch_dependent(packed_combine_kernel<T, D, kGroups>, dim3((unsigned)rows), dim3(1024), 0, st, a, kLogCols);
  } else if (shares >= 4) {
    constexpr int kGroups = 1024 / D;   // 256 threads
    err = launch_dependent(packed_combine_kernel<T, D, kGroups>, dim3((unsigned)rows), dim3(256), 0, st, a, kLogCols);
  } else {
    const int per_block = 128 / (D / 4);
    err = launch_dependent(packed_combine_kernel<T, D, 1>, dim3((unsigned)((rows + per_block - 1) / per_block)), dim3(128), 0, st, a,
                           kLogCols);
  }
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, int D>
cudaError_t launch_t(const AttendArgs& a, void* workspace, int max_len, cudaStream_t st) {
  // (five to eight query rows in two tiles of four would unpack everything twice)
  if constexpr (sizeof(T) == 2)
    if ((int64_t)a.I * a.c.g <= 4) return launch_columns<T, D, true>(a, workspace, max_len, st);
  return launch_columns<T, D, false>(a, workspace, max_len, st);
}

}  // namespace

cudaError_t launch_packed_wait_selftest(int32_t* status, cudaStream_t st) {
  packed_wait_selftest_kernel<<<1, 32, 0, st>>>(status);
  count_launch();
  return cudaGetLastError();
}

size_t packed_attend_workspace(int d, int batch, int Hkv, int g, int queries, int tiles) {
  // every run leaves two shares at most; calls of fewer samples, queries or rows take no more runs and no more columns
  const int64_t cols = (int64_t)queries * g;
  int64_t runs = 1;
  for (const int64_t factor : {(int64_t)batch, (int64_t)Hkv, (cols + 3) / 4, (int64_t)tiles})   // (their product may pass 64 bits)
    runs = std::min<int64_t>(runs * std::min<int64_t>(factor, kMostSms * kWarpsPerSm), kMostSms * kWarpsPerSm);
  const size_t most = (size_t)runs * 2 * std::min<int64_t>(8, cols) * (d + 4) * sizeof(float);
  return std::max(before_bytes(batch) + most, packed_block_workspace(batch, Hkv));
}

cudaError_t launch_packed_attend(int dtype, int d, const PackedView& c, const PackedAttend& p, cudaStream_t st) {
  g_last_packed_path = dtype == 1 && packed_block_pays(d, c, p.I, p.max_len) ? 1 : 0;
  if (g_last_packed_path == 1) return launch_packed_block(d, c, p, st);
  AttendArgs a;
  a.c = c;
  a.q = p.q; a.q_sample = p.q_sample; a.q_token = p.q_token;
  a.I = p.I;
  a.lens = p.lens; a.first = p.first;
  a.out = p.out;
  a.mul = p.scale * 1.4426950408889634f;
  a.query_tiles = a.runs = a.slot_cols = 1;
  a.before = nullptr;
  a.partial = nullptr;
  if (dtype == 0) return d == 64 ? launch_t<float, 64>(a, p.workspace, p.max_len, st) : launch_t<float, 128>(a, p.workspace, p.max_len, st);
  return d == 64 ? launch_t<__nv_bfloat16, 64>(a, p.workspace, p.max_len, st)
                 : launch_t<__nv_bfloat16, 128>(a, p.workspace, p.max_len, st);
}

}  // namespace bm
