// Attention of blocks of queries over a packed cache (packed.cuh) on the 5th-generation tensor cores: what packed_attend.cu computes, for
// calls whose query rows, I * g of a cache, fill tiles of 128.
//
// A CTA has two tiles of 128 query rows of one cache, A and B, and 128 keys at a time.  Eight warps turn the packed rows into fp16 tiles in
// shared memory (K as code * s, V likewise: exact, since a scale of bf16 rows has 8 bits and a code 3 more; rounded to 11 bits where a scale
// was held to 65504), one issues S = Q K^T of both, one each O += P V of A and of B, and four softmax warps per tile have a thread for every
// query row, which also brought its row of Q.  Tensor memory: O_A | O_B | P_A | P_B | S (one of 128 columns that the tiles use in turn at
// d = 128, one each at d = 64).  A group reads its row's 128 logits into registers at once and gives S back; P has columns of its own, so
// that the next Q K^T and the P V before run under the exponentials.
//
// fp16 has 40 binades: keys and values are taken times a power of two per cache (packed_scales_kernel finds the largest scale), queries per
// row, and what remains below fp16's smallest is 2^-38 of the largest.  Elements of every eight are kept in the order 0 4 1 5 2 6 3 7, in
// which two masked codes are neighbours, in Q as in K; outputs are put in order on their way out.
//
// A scale that is not finite: keys give NaN logits.  A weight of 0 times a NaN value would be NaN for queries that do not see the row, so such
// values are 0 in the tile, and the first such row of each group is kept: queries see a prefix of the rows, those that see it are NaN there.
//
// What bounds it: issue slots and latency of the softmax warps (exponentials 2048 cycles per pair of tiles and scheduler, the tensor pipe as
// many, of 4400) and, beside them on the same schedulers, the unpacking (a third of the instructions).  Measured in bursts, with
// packed_scales_kernel (4 us), 256 queries of 4 samples over 4352 rows, 32 / 8 heads, d = 128: 89 us, 793 TFLOP/s (128 CTAs, 2.5 us per 128
// keys), 16 samples of 4096 336, d = 64 74; one row tile, 32 queries of 16 samples of 4096, 68.  Other ways, before the last of these was
// found (us, in this order, 89, 331, 75, 66 then): addresses and scales worked out per element group 93, 345, 75, 69; four unpacking warps
// with twice the work each (512 threads) 95, 370, 74, 86; a mask at the rows' load, which waits for it, 101, 392, 77, 93; 64 keys per step,
// with logits of its own for either row tile, 98, 350, 87, 77 where 128 took 94, 349, 74, 69: a step's waits and reductions come twice.
#include <algorithm>
#include <cmath>

#include "packed.cuh"
#include "tc_common.cuh"

namespace bm {
using namespace tc;
namespace {

constexpr int kRows = 128, kKeys = 128, kThreads = 640, kLaunchRegs = 96;
constexpr int kScaleParts = 16;         // CTAs that look at a cache's scales
constexpr float kRescale = 8.f;         // the maximum follows when logits pass it by this much (log2): weights stay below 2^8

struct BlockArgs16 {
  PackedView c;
  const __nv_bfloat16* q;
  int64_t q_sample, q_token;
  int32_t I;
  const int32_t* lens;
  const int32_t* first;
  __nv_bfloat16* out;
  float mul;              // scale * log2(e)
  int32_t pairs;          // of row tiles, per cache
  FastDiv by_g, by_pairs, by_heads;
  uint32_t* largest;      // workspace: [units][kScaleParts][2] largest finite magnitudes of the key scales, the value scales (fp16 bits)
};

struct Seen {
  int len, lo;            // rows [lo, len) are seen by some query
};
__device__ __forceinline__ Seen seen_rows(const BlockArgs16& a, int smp) {
  Seen s;
  s.len = min(max(a.lens[smp], 0), a.c.capacity);
  s.lo = a.first != nullptr ? max(a.first[smp], 0) : 0;
  return s;
}

// The largest scales of a cache's rows that some query sees, in kScaleParts parts.
template <int D>
__global__ void __launch_bounds__(256) packed_scales_kernel(BlockArgs16 a) {
  using L = PackedLayout<D>;
  constexpr int kPieces = 2 * L::kScales / 16, kTilesPerStep = 256 / kPieces;   // 16-byte pieces of a tile's scales
  __shared__ uint32_t warp_max[8][2];
  pdl_wait();
  pdl_release();
  const int unit = blockIdx.x / kScaleParts, part = blockIdx.x % kScaleParts, smp = a.by_heads(unit);
  const Seen seen = seen_rows(a, smp);
  const int t0 = seen.lo / kPackedTile, t1 = seen.len > seen.lo ? (seen.len + kPackedTile - 1) / kPackedTile : t0;
  const uint8_t* base = a.c.data + (size_t)unit * a.c.tiles * L::kBytes;
  const int piece = threadIdx.x % kPieces;
  uint32_t most = 0;
#pragma unroll 4
  for (int t = t0 + part * kTilesPerStep + threadIdx.x / kPieces; t < t1; t += kScaleParts * kTilesPerStep) {
    const uint4 v = ld_global_16(base + (size_t)t * L::kBytes + L::kKeyScales + piece * 16);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    const int lo_row = seen.lo - t * kPackedTile, hi_row = seen.len - t * kPackedTile;   // rows [lo_row, hi_row) of the tile are seen
    if (lo_row > 0 || hi_row < kPackedTile) {
      // the others may hold anything: the scales (at most two rows to a word) of those are taken as 0
      auto kept = [&](int row) { return row >= lo_row && row < hi_row; };
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int word = (piece % (kPieces / 2)) * 4 + i;   // (of the key scales or of the value scales)
        if (piece < kPieces / 2) {
          if (!kept(word / (L::G / 2))) w[i] = 0;
        } else {
          const int row = word / (8 * L::G) * 16 + word / L::G % 2 * 8 + word / (2 * L::G) % 4;   // (value_scale the other way round)
          w[i] &= (kept(row) ? 0x0000ffffu : 0u) | (kept(row + 4) ? 0xffff0000u : 0u);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t lo = w[i] & 0x7fffu, hi = (w[i] >> 16) & 0x7fffu;
      most = max(most, max(lo < 0x7c00u ? lo : 0u, hi < 0x7c00u ? hi : 0u));
    }
  }
  const bool value = piece >= kPieces / 2;
  const uint32_t k = __reduce_max_sync(0xffffffffu, value ? 0u : most), v = __reduce_max_sync(0xffffffffu, value ? most : 0u);
  if (threadIdx.x % 32 == 0) {
    warp_max[threadIdx.x / 32][0] = k;
    warp_max[threadIdx.x / 32][1] = v;
  }
  __syncthreads();
  if (threadIdx.x < 2) {
    uint32_t m = 0;
    for (int i = 0; i < 8; ++i) m = max(m, warp_max[i][threadIdx.x]);
    a.largest[(size_t)blockIdx.x * 2 + threadIdx.x] = m;
  }
}

template <int D>
struct BlockSmem {
  static constexpr int kTile = kRows * D * 2;     // 128 rows of D fp16 numbers, in pieces of 64 elements: [piece][row][128 bytes, swizzled]
  static constexpr int kQ = 0, kK = 2 * kTile, kV = 4 * kTile, kBars = 6 * kTile, kTotal = kBars + 512 + 1024;
};

__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
// eight codes of a word times a scale (a pair), in the order 0 4 1 5 2 6 3 7
__device__ __forceinline__ uint4 unpack_scaled(uint32_t w, uint32_t s2) {
  uint32_t x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t u = ((i < 2 ? w : w >> 8) & (i % 2 ? 0x00f000f0u : 0x000f000fu)) | 0x64006400u;   // 1024 + u, 1024 + 16 u
    const __half2 h = *reinterpret_cast<const __half2*>(&u);
    const __half2 c = i % 2 ? __hfma2(h, __float2half2_rn(0.0625f), __float2half2_rn(-72.f)) : __hsub2(h, __float2half2_rn(1032.f));
    x[i] = hmul2(*reinterpret_cast<const uint32_t*>(&c), s2);
  }
  return make_uint4(x[0], x[1], x[2], x[3]);
}
__device__ __forceinline__ bool not_finite(uint32_t s) { return (s & 0x7c00u) == 0x7c00u; }   // of an fp16 number in the low half

template <int D>
__global__ void __launch_bounds__(kThreads, 1) packed_block_kernel(BlockArgs16 a) {
  using S = BlockSmem<D>;
  using L = PackedLayout<D>;
  constexpr int G = L::G, kQkWarp = 8, kPvWarp = 9 /* A; 10: B */, kUnpackWarp = 12, kUnpackWarps = 8;
  constexpr int NSB = D == 128 ? 1 : 2;   // logit buffers
  constexpr int B_Q = 0, B_KFULL = 2, B_KFREE = 4, B_VFULL = 6, B_VFREE = 8, B_SFULL = 10, B_SFREE = 12, B_P = 14 /* [half][group] */,
                B_PV = 18 /* likewise */, B_COUNT = 22;
  extern __shared__ unsigned char smem_raw[];
  unsigned char* sm = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint64_t* bars = reinterpret_cast<uint64_t*>(sm + S::kBars);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + B_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  int* nan_row = reinterpret_cast<int*>(tmem_slot + 2);   // [4]
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  pdl_wait();   // (before tensor memory is taken: a kernel before may have CTAs that wait for it)
  pdl_release();
  if (tid == 0) {
    *abort_flag = 0;
#pragma unroll 1
    for (int b = 0; b < B_COUNT; ++b)
      mbar_init(&bars[b], b < B_KFULL || (b >= B_SFREE && b < B_PV) ? 4
                          : b < B_KFREE || (b >= B_VFULL && b < B_VFREE) ? kUnpackWarps
                          : b >= B_VFREE && b < B_SFULL                  ? 2
                                                                         : 1);
    mbar_fence_init();
    for (int i = 0; i < 4; ++i) nan_row[i] = INT32_MAX;
  }
  if (warp == kQkWarp) tmem_alloc(tmem_slot, 512);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  const uint32_t tm_o0 = tmem, tm_p0 = tmem + 2 * D, tm_s0 = tmem + 2 * D + 128;   // group x: + D x, + 64 x, + 128 x (NSB = 2)
  auto wait = [&](int b, int n) { mbar_wait(&bars[b], (uint32_t)n & 1, abort_flag, a.c.status); };   // for the n-th completion

  const int unit = a.by_pairs(blockIdx.x), pair = a.pairs - 1 - (blockIdx.x - unit * a.pairs);   // (later rows see more keys: first)
  const int smp = a.by_heads(unit), head = unit - smp * a.c.Hkv;
  const Seen seen = seen_rows(a, smp);
  const int cols = a.I * a.c.g, t_first = seen.lo / kKeys;
  // key tiles that row tile x sees: up to its last row's limit
  auto key_tiles = [&](int x) {
    const int row0 = (2 * pair + x) * kRows;
    if (row0 >= cols) return 0;
    const int limit = seen.len - (a.I - 1 - a.by_g(min(row0 + kRows, cols) - 1));
    return limit > seen.lo ? (limit + kKeys - 1) / kKeys - t_first : 0;
  };
  const int n0 = key_tiles(0), n1 = key_tiles(1), T = max(n0, n1);
  // powers of two that bring the largest key and value scale to 2^11 .. 2^12 (times 8: below 2^15)
  int ek = 0, ev = 0;
  {
    const uint32_t* p = a.largest + (size_t)unit * kScaleParts * 2;
    uint32_t mk = 0, mv = 0;
#pragma unroll
    for (int i = 0; i < kScaleParts; ++i) { mk = max(mk, p[2 * i]); mv = max(mv, p[2 * i + 1]); }
    const float fk = __half2float(__ushort_as_half((unsigned short)mk)), fv = __half2float(__ushort_as_half((unsigned short)mv));
    if (mk > 0) ek = min(11 - ((int)(__float_as_uint(fk) >> 23) - 127), 30);
    if (mv > 0) ev = min(11 - ((int)(__float_as_uint(fv) >> 23) - 127), 30);   // -4 .. 30
  }
  auto pow2 = [](int e) { return __int_as_float((e + 127) << 23); };

  // 640 threads start with kLaunchRegs = 96 registers each: 256 x 160 + 128 x 32 + 256 x 64
  if (warp >= kQkWarp) {
    if (warp >= kUnpackWarp) {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
      // ------------------------------------------------------------------ packed rows -> fp16 tiles
      const int u = tid - kUnpackWarp * 32, d = u & 127, half = u >> 7;
      const uint8_t* base = a.c.data + (size_t)unit * a.c.tiles * L::kBytes;
      auto power = [&](int e) { return half2_bits(pow2(e), pow2(e)); };
      const uint32_t k1 = power(min(ek, 15)), k2 = power(max(ek - 15, 0)), v1 = power(min(ev, 15)), v2 = power(max(ev - 15, 0));
      // this thread's codes: of half of key row d; of the value rows vr and vr + 4, the elements 8 rp .. + 7 of each group
      uint4 kc[D / 64], vc[2];
      uint32_t ks[G / 2], vs[G];
      const int rp = u / 4 % 4, vr = u / 16 * 8 + u % 4;
      // where they go, in the tile: key row d's pieces 2 half, the others by flipping bits; the pieces rp of the value rows, the odd rp
      // the later row first (eight lanes write to all banks)
      const uint32_t k_at = S::kK + sw128_offset(d, 2 * half), v_at = S::kV + sw128_offset(vr + 4 * (rp & 1), rp);
      const uint32_t first_half = rp & 1 ? 0x7632 : 0x5410, first_scale = rp & 1 ? 0x3232 : 0x1010;
      // Rows that no query sees are read as they are (of the last tile that has such rows, if theirs is behind it) and get scales of 0, when
      // they are used: a mask at the load would wait for it.
      const int last_tile = (seen.len - 1) / kPackedTile;
      auto tile_at = [&](int row) { return base + (size_t)min(row / kPackedTile, last_tile) * L::kBytes; };
      auto load_keys = [&](int j) {
        const uint8_t* tile = tile_at((t_first + j) * kKeys + d);
        const int at = d % kPackedTile;
#pragma unroll
        for (int i = 0; i < D / 64; ++i) kc[i] = ld_global_16(tile + at * (D / 2) + (half * (D / 64) + i) * 16);
#pragma unroll
        for (int i = 0; i < G / 2; ++i) ks[i] = *reinterpret_cast<const uint32_t*>(tile + L::kKeyScales + at * G * 2 + i * 4);
      };
      auto load_values = [&](int j) {
        const uint8_t* tile = tile_at((t_first + j) * kKeys + vr);
        const int at = vr % kPackedTile;
        if constexpr (G == 4) {
          vc[0] = ld_global_16(tile + L::value_codes(at, 0, 2 * rp));
          vc[1] = ld_global_16(tile + L::value_codes(at, 0, 2 * rp + 1));
          const uint4 s = ld_global_16(tile + L::value_scale(at, 0));
          vs[0] = s.x; vs[1] = s.y; vs[G - 2] = s.z; vs[G - 1] = s.w;
        } else {
          const uint2 x = *reinterpret_cast<const uint2*>(tile + L::value_codes(at, 0, 2 * rp));
          const uint2 y = *reinterpret_cast<const uint2*>(tile + L::value_codes(at, 0, 2 * rp + 1));
          vc[0] = make_uint4(x.x, x.y, 0, 0);
          vc[1] = make_uint4(y.x, y.y, 0, 0);
          const uint2 s = *reinterpret_cast<const uint2*>(tile + L::value_scale(at, 0));
          vs[0] = s.x; vs[1] = s.y;
        }
      };
      if (T > 0) {
        load_keys(0);
        load_values(0);
      }
#pragma unroll 1
      for (int j = 0; j < T; ++j) {
        const int s = j & 1;
        if (j >= 2) wait(B_KFREE + s, j / 2 - 1);
        const int row0 = (t_first + j) * kKeys;
        auto seen_row = [&](int row) { return row >= seen.lo && row < seen.len; };
        if (!seen_row(row0 + d)) {
#pragma unroll
          for (int i = 0; i < G / 2; ++i) ks[i] = 0u;
        }
#pragma unroll
        for (int i = 0; i < G / 2; ++i) ks[i] = hmul2(hmul2(ks[i], k1), k2);
#pragma unroll
        for (int g4 = 0; g4 < G; ++g4) {
          const uint32_t s2 = __byte_perm(ks[g4 / 2], 0, g4 % 2 ? 0x3232 : 0x1010);
#pragma unroll
          for (int i = 0; i < 2; ++i) {   // the word (g4, c): word c G + g4 of the row
            const int at = i * G + g4;
            const uint4 four = kc[at / 4];
            const uint32_t w = at % 4 == 0 ? four.x : at % 4 == 1 ? four.y : at % 4 == 2 ? four.z : four.w;
            *reinterpret_cast<uint4*>(sm + ((k_at + s * S::kTile) ^ (4 * (g4 % 2) + i) << 4) + g4 / 2 * 16384) = unpack_scaled(w, s2);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_KFULL + s]);
        if (j + 1 < T) load_keys(j + 1);   // (on its way while the values are unpacked, and theirs during the next keys)
        if (j >= 2) wait(B_VFREE + s, j / 2 - 1);
        const uint32_t keep = (seen_row(row0 + vr) ? 0x0000ffffu : 0u) | (seen_row(row0 + vr + 4) ? 0xffff0000u : 0u);
        uint32_t bad = 0;   // bit 15 of a half: some exponent is all ones
#pragma unroll
        for (int g4 = 0; g4 < G; ++g4) {
          vs[g4] &= keep;
          bad |= (vs[g4] & 0x7c007c00u) + 0x04000400u;
        }
        if (bad & 0x80008000u) {
#pragma unroll
          for (int g4 = 0; g4 < G; ++g4) {
            if (not_finite(vs[g4] >> 16)) { atomicMin(&nan_row[g4], row0 + vr + 4); vs[g4] &= 0x0000ffffu; }
            if (not_finite(vs[g4])) { atomicMin(&nan_row[g4], row0 + vr); vs[g4] &= 0xffff0000u; }
          }
          __threadfence_block();
        }
#pragma unroll
        for (int g4 = 0; g4 < G; ++g4) {
          vs[g4] = hmul2(hmul2(vs[g4], v1), v2);
          const uint32_t x = g4 == 0 ? vc[0].x : g4 == 1 ? vc[0].y : g4 == 2 ? vc[0].z : vc[0].w;
          const uint32_t y = g4 == 0 ? vc[1].x : g4 == 1 ? vc[1].y : g4 == 2 ? vc[1].z : vc[1].w;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t words = h == 0 ? first_half : first_half ^ 0x2222;
            *reinterpret_cast<uint4*>(sm + ((v_at + s * S::kTile) ^ (h ^ g4 % 2) << 6 ^ h << 9) + g4 / 2 * 16384) =
                unpack_scaled(__byte_perm(x, y, words), __byte_perm(vs[g4], 0, h == 0 ? first_scale : first_scale ^ 0x2222));
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars[B_VFULL + s]);
        if (j + 1 < T) load_values(j + 1);
      }
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 32;");
      if (lane == 0) {
        const uint64_t dk_hi = smem_desc(0, 16, 1024) & 0xffffffff00000000ull;      // K-major operands (Q, K)
        const uint32_t dk_lo = (uint32_t)(smem_desc(0, 16, 1024) & 0xffffffffull);
        const uint64_t dv_hi = smem_desc(0, 16384, 1024) & 0xffffffff00000000ull;   // MN-major operand (V)
        const uint32_t dv_lo = (uint32_t)(smem_desc(0, 16384, 1024) & 0xffffffffull);
        constexpr uint32_t kBf16 = 1u << 7 | 1u << 10;                               // instr_desc's input formats: cleared, fp16
        if (warp == kQkWarp) {
          // ---------------------------------------------------------------- S = Q K^T of both tiles, in turn
          const uint32_t idesc = instr_desc(kRows, kKeys, 0, 0) & ~kBf16;
          const uint32_t q_lo = dk_lo + (smem_u32(sm + S::kQ) >> 4), k_base = dk_lo + (smem_u32(sm + S::kK) >> 4);
          int sc0 = 0, sc1 = 0, last = -1;
#pragma unroll 1
          for (int j = 0; j < T; ++j) {
            wait(B_KFULL + (j & 1), j / 2);
            const uint32_t k_lo = k_base + (uint32_t)(j & 1) * (S::kTile >> 4);
#pragma unroll 1
            for (int x = 0; x < 2; ++x) {
              if (j >= (x ? n1 : n0)) continue;
              if (j == 0) wait(B_Q + x, 0);
              const int before = NSB == 2 ? x : last, n = before == 0 ? sc0 : sc1;   // the logits that the buffer holds have been read
              if (before >= 0 && n > 0) wait(B_SFREE + before, n - 1);
              last = x;
              if (x == 0) ++sc0; else ++sc1;
              tc_fence_after();
              const uint32_t q = q_lo + x * (S::kTile >> 4);
#pragma unroll
              for (int step = 0; step < D / 16; ++step) {
                const uint32_t off = (step >> 2) * 1024 + (step & 3) * 2;   // (piece * 16384 + step * 32) / 16
                mma_ss(tm_s0 + (NSB == 2 ? 128 * x : 0), dk_hi | (q + off), dk_hi | (k_lo + off), idesc, step > 0 ? 1u : 0u);
              }
              mma_commit(&bars[B_SFULL + x]);
            }
            mma_commit(&bars[B_KFREE + (j & 1)]);
          }
        } else if (warp == kPvWarp || warp == kPvWarp + 1) {
          // ---------------------------------------------------------------- O += P V of tile x, 64 keys at a time
          const int x = warp - kPvWarp, n = x ? n1 : n0;
          const uint32_t idesc = instr_desc(kRows, D, 0, 1) & ~kBf16;   // V is MN-major: d contiguous, keys along K
          const uint32_t v_base = dv_lo + (smem_u32(sm + S::kV) >> 4);
          const uint32_t tm_o = tm_o0 + D * x, tm_p = tm_p0 + 64 * x;
#pragma unroll 1
          for (int j = 0; j < T; ++j) {
            wait(B_VFULL + (j & 1), j / 2);
            if (j >= n) { mbar_arrive(&bars[B_VFREE + (j & 1)]); continue; }
            const uint32_t v_lo = v_base + (uint32_t)(j & 1) * (S::kTile >> 4);
#pragma unroll 1
            for (int h = 0; h < 2; ++h) {
              wait(B_P + 2 * h + x, j);
              tc_fence_after();
#pragma unroll
              for (int q = 0; q < 4; ++q)
                mma_ts(tm_o, tm_p + (4 * h + q) * 8, dv_hi | (v_lo + (4 * h + q) * 128), idesc, j > 0 || h > 0 || q > 0 ? 1u : 0u);
              mma_commit(&bars[B_PV + 2 * h + x]);
            }
            mma_commit(&bars[B_VFREE + (j & 1)]);
          }
        }
      }
    }
  } else {
    // -------------------------------------------------------------------- a thread per query row
    asm volatile("setmaxnreg.inc.sync.aligned.u32 160;");
    const int x = warp >> 2, quad = warp & 3, r = quad * 32 + lane, n = x ? n1 : n0;
    const int col = (2 * pair + x) * kRows + r, query = a.by_g(min(col, cols - 1)), in_group = min(col, cols - 1) - query * a.c.g;
    const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
    const uint32_t tm_s = tm_s0 + (NSB == 2 ? 128 * x : 0) + lane_addr, tm_p = tm_p0 + 64 * x + lane_addr, tm_o = tm_o0 + D * x + lane_addr;
    const int limit = seen.len - (a.I - 1 - query);   // this row sees [seen.lo, limit)
    float row_mul = 0.f;
    if (n > 0) {   // the row of Q, to a largest magnitude of 2^14 .. 2^15
      const __nv_bfloat16* q = a.q + smp * a.q_sample + query * a.q_token + ((size_t)head * a.c.g + in_group) * D;
      uint4 raw[D / 8];
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        raw[i] = ld_global_16(q + 8 * i);
        const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) most = max(most, max(w[e] << 16 & 0x7fff0000u, w[e] & 0x7fff0000u));
      }
      const int e = most > 0 && most < 0x7f800000u ? min(14 - (int)(most >> 23) + 127, 100) : 0;
      const float up = pow2(e);
      row_mul = fminf(fmaxf(a.mul * pow2(-e) * pow2(-ek), 0x1p-126f), 0x1.fffffep127f);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        float f[8];
        Elem<__nv_bfloat16>::unpack(raw[i], f);
        uint32_t w[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = half2_bits(f[k] * up, f[k + 4] * up);
        *reinterpret_cast<uint4*>(sm + S::kQ + x * S::kTile + i / 8 * 16384 + sw128_offset(r, i % 8)) = make_uint4(w[0], w[1], w[2], w[3]);
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_Q + x]);
    }
    // tiles that every row of the warp sees whole
    const int full0 = seen.lo % kKeys ? 1 : 0, full1 = (__reduce_min_sync(0xffffffffu, limit) - t_first * kKeys) >> 7;
    float m_used = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int j = 0; j < n; ++j) {
      wait(B_SFULL + x, j);
      tc_fence_after();
      const int row0 = (t_first + j) * kKeys, v0 = max(seen.lo - row0, 0), v1 = min(limit - row0, kKeys);   // visible columns [v0, v1)
      if (j < full0 || j >= full1) {
        // hidden logits become -inf, in tensor memory and in a rolled loop: these tiles are few
#pragma unroll 1
        for (int cc = 0; cc < 8; ++cc) {
          uint32_t raw[16];
          tmem_ld16(tm_s + 16 * cc, raw);
          const int b0 = min(max(v0 - 16 * cc, 0), 16), b1 = min(max(v1 - 16 * cc, 0), 16);
          const uint32_t bits = ((1u << b1) - 1u) & ~((1u << b0) - 1u);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) raw[e] = (bits >> e) & 1 ? raw[e] : 0xff800000u;
          tmem_st16(tm_s + 16 * cc, raw);
        }
        tmem_wait_st();
      }
      uint32_t s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tmem_ld32(tm_s + 32 * c, s[c]);
      tmem_wait_ld();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&bars[B_SFREE + x]);
      float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int e = 0; e < 32; e += 2)
#pragma unroll
        for (int c = 0; c < 4; ++c) m4[c] = max3_nan(m4[c], __uint_as_float(s[c][e]), __uint_as_float(s[c][e + 1]));
      float mx = max3_nan(max3_nan(m4[0], m4[1], m4[2]), m4[3], -INFINITY) * row_mul;
      if (mx == INFINITY) mx = __uint_as_float(0x7fffffffu);   // an infinite logit makes its row NaN, as NaN does
      bool rescale = false;
      float alpha = 1.f;
      if (j == 0) m_used = mx;
      else if (!(mx <= m_used + kRescale)) { alpha = exp2f(m_used - mx); m_used = mx; rescale = true; }
      if (__any_sync(0xffffffffu, rescale)) {
        wait(B_PV + 2 + x, j - 1);
        tc_fence_after();
#pragma unroll 1
        for (int cc = 0; cc < D / 16; ++cc) {
          uint32_t raw[16];
          tmem_ld16(tm_o + cc * 16, raw);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 16; ++e) raw[e] = __float_as_uint(__uint_as_float(raw[e]) * alpha);
          tmem_st16(tm_o + cc * 16, raw);
        }
        l *= alpha;
      }
      const float neg_m = m_used == -INFINITY ? 0.f : -m_used;   // (no row seen so far)
      // Below, m_used is taken from the exact product of a logit and row_mul, which is up to 2^-24 of it away from the rounded one that m_used is:
      // where that is not next to nothing, logits are rounded first, as m_used was.
      float mul = row_mul;
      if (__any_sync(0xffffffffu, fabsf(neg_m) > 0x1p20f)) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
          for (int e = 0; e < 32; ++e) s[c][e] = __float_as_uint(__fmul_rn(__uint_as_float(s[c][e]), row_mul));
        mul = 1.f;
      }
      float pa0 = 0.f, pa1 = 0.f, pb0 = 0.f, pb1 = 0.f;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        uint32_t pk[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x0, x1;
          fma2(x0, x1, __uint_as_float(s[c][2 * e]), __uint_as_float(s[c][2 * e + 1]), mul, neg_m);
          const float p0 = ex2(x0), p1 = ex2(x1);
          if (e & 1) add2(pb0, pb1, p0, p1);
          else add2(pa0, pa1, p0, p1);
          pk[e] = half2_bits(p0, p1);
        }
        if (!(c & 1) && j > 0) wait(B_PV + c + x, j - 1);   // the columns' weights of the tile before are used up
        tmem_st16(tm_p + 16 * c, pk);
        if (c & 1) {                            // 64 keys may enter P V
          tmem_wait_st();
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(&bars[B_P + c - 1 + x]);
        }
      }
      l += (pa0 + pb0) + (pa1 + pb1);
    }
    // ---- O / l, out in order; a row that sees nothing is a row of zeros ---------------------------------------------------------
    __nv_bfloat16* out = a.out + (((size_t)smp * a.I + query) * a.c.Hq + (size_t)head * a.c.g + in_group) * D;
    const bool any = n > 0 && limit > seen.lo;
    if (n > 0) {
      wait(B_PV + 2 + x, n - 1);
      tc_fence_after();
    }
    const float by = any ? pow2(-ev) / l : 0.f;
#pragma unroll 1
    for (int g4 = 0; g4 < G; ++g4) {
      uint32_t raw[32];
      if (n > 0) {
        tmem_ld32(tm_o + 32 * g4, raw);
        tmem_wait_ld();
      }
      const float scale = any && *const_cast<volatile int*>(&nan_row[g4]) < limit ? __uint_as_float(0x7fffffffu) : by;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float f[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = any ? __uint_as_float(raw[8 * i + (k < 4 ? 2 * k : 2 * k - 7)]) * scale : 0.f;
        if (col < cols)
          st_global_16(out + 32 * g4 + 8 * i, make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7])));
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kQkWarp) tmem_dealloc(tmem, 512);
}

template <int D>
cudaError_t launch_d(const PackedView& c, const PackedAttend& p, cudaStream_t st) {
  BlockArgs16 a;
  a.c = c;
  a.q = static_cast<const __nv_bfloat16*>(p.q);
  a.q_sample = p.q_sample; a.q_token = p.q_token;
  a.I = p.I;
  a.lens = p.lens; a.first = p.first;
  a.out = static_cast<__nv_bfloat16*>(p.out);
  a.mul = p.scale * 1.4426950408889634f;
  a.largest = static_cast<uint32_t*>(p.workspace);
  const int64_t units = (int64_t)c.nsamples * c.Hkv, cols = (int64_t)p.I * c.g;
  a.pairs = (int)((cols + 2 * kRows - 1) / (2 * kRows));
  a.by_g = FastDiv((uint32_t)c.g);
  a.by_pairs = FastDiv((uint32_t)a.pairs);
  a.by_heads = FastDiv((uint32_t)c.Hkv);
  if (units * std::max<int64_t>(a.pairs, kScaleParts) > 0x7fffffff) return cudaErrorInvalidConfiguration;
  static SmemConfigured configured;
  if (cudaError_t err = configured.ensure(packed_block_kernel<D>, BlockSmem<D>::kTotal); err != cudaSuccess) return err;
  // its warps divide the registers among them anew: with fewer at the launch than that takes they would wait for good
  static const bool enough = [] {
    cudaFuncAttributes attr;
    return cudaFuncGetAttributes(&attr, packed_block_kernel<D>) == cudaSuccess && attr.numRegs >= kLaunchRegs;
  }();
  if (!enough) return cudaErrorInvalidConfiguration;
  cudaError_t err;
  {
    ProfileScope prof(kPacked, st);
    err = launch_dependent(packed_scales_kernel<D>, dim3((unsigned)(units * kScaleParts)), dim3(256), 0, st, a);
  }
  count_launch();
  if (err != cudaSuccess) return err;
  ProfileScope prof(kPacked, st);
  err = launch_dependent(packed_block_kernel<D>, dim3((unsigned)(units * a.pairs)), dim3(kThreads), BlockSmem<D>::kTotal, st, a);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

}  // namespace

// Which calls take this kernel: its time goes by rounds of one CTA per SM, 5 us and so much for 128 keys of one or of two row tiles; that of
// the warps' kernel by tiles of 32 keys x 8 query rows, shared evenly, and 5 us.  us, this kernel / the other: 32 / 8 heads, d = 128, 16
// samples of 4096 rows, 32 query rows of a cache 66 / 60, 64 rows 67 / 110, 128 rows 68 / 212; 4 samples, 64 rows 63 / 40, 128 rows 64 / 60,
// 256 rows 84 / 109, 1024 rows (4352) 89 / 431; 1 sample of 4352, 256 rows 87 / 41, 1024 rows 87 / 114; of 16384, 512 rows 291 / 203; 64
// samples of 1024, 32 rows 92 / 67, 64 rows 94 / 123; 32 samples of 2048, 32 heads without groups, 32 rows 261 / 223, 64 rows 266 / 430.
// 8 kv-heads, d = 64, 16 samples of 4096, 32 rows 59 / 45, 64 rows 59 / 74; 4 of 4352, 256 rows 74 / 75, 512 rows 74 / 140; 1, 1024 rows
// 73 / 72; short caches: 128 samples of 256, d = 128, 64 rows 95 / 87, 128 rows 105 / 163; 40 samples of 400 with 2 heads, d = 64, 257
// rows 30 / 28.
bool packed_block_pays(int d, const PackedView& c, int I, int max_len) {
  const double cols = (double)I * c.g, units = (double)c.nsamples * c.Hkv, pairs = std::ceil(cols / (2 * kRows));
  const double step = d == 64 ? (cols <= kRows ? 1.7 : 2.08) : (cols <= kRows ? 1.9 : 2.45);
  const double here = (5. + step * max_len / kKeys) * std::ceil(units * pairs / sm_count());
  const double warps = 5. + (d == 64 ? 0.81 : 1.36) * units * std::ceil(cols / 8) * max_len / kPackedTile / (12. * sm_count());
  return here < warps;
}

size_t packed_block_workspace(int batch, int Hkv) { return (size_t)batch * Hkv * kScaleParts * 2 * sizeof(uint32_t); }

cudaError_t launch_packed_block(int d, const PackedView& c, const PackedAttend& p, cudaStream_t st) {
  return d == 64 ? launch_d<64>(c, p, st) : launch_d<128>(c, p, st);
}

}  // namespace bm
