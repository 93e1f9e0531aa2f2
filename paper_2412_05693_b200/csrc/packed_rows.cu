// Writing rows into a packed cache, and reading them back (packed.cuh has the format).
//
// Both are bound by HBM: a row of d elements comes in as d * e bytes and goes out as d / 2 + d / 16, or the other way round.  A CTA has one
// tile of a cache, whose bytes meet in shared memory, so that global memory sees whole 16-byte pieces although a tile's bytes are ordered for
// the attention kernel.  A thread has eight consecutive elements of a row, four threads a group.
//
// Measured, 16 samples of 4096 rows, 8 heads, d = 128 (344 MB, 52.6 us at the copy bandwidth): bf16 written in 67 us, read in 57; d = 64, as
// many bytes, 74 and 58; fp32, half as many rows, 57 and 51 (46.8).  Reading is bound by HBM, writing bf16 by its instructions (16 per
// element's lane: schedulers 84 % busy, the logic pipe 70 %); with a CTA of 256 threads 77 and 61 where this took 70 and 56 (fp32 55 and 49).
#include <algorithm>

#include "packed.cuh"
#include "tc_common.cuh"

namespace bm {
namespace {

constexpr int kThreads = 128;
constexpr float kMagic = 12582912.f;   // 1.5 * 2^23: adding it rounds to integers, ties to even; the low bits are the integer

template <typename T>
__device__ __forceinline__ void unpack8(const uint4* raw, float* x) {
  Elem<T>::unpack(raw[0], x);
  if constexpr (sizeof(T) == 4) Elem<T>::unpack(raw[1], x + 4);
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float y;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
  return y;
}

__device__ __forceinline__ uint32_t max2_nan(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
__device__ __forceinline__ uint32_t min2_nan(uint32_t a, uint32_t b) {
  uint32_t y;
  asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(y) : "r"(a), "r"(b));
  return y;
}
// The largest element of the group and the largest of its negatives, NaN where one is NaN: four lanes with eight elements each.
template <typename T>
__device__ __forceinline__ void group_range(const uint4* raw, const float* x, float* top, float* low) {
  if constexpr (sizeof(T) == 2) {   // in pairs; then (top, low) as one
    const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
    constexpr uint32_t kSigns = 0x80008000u;
    const uint32_t t = max2_nan(max2_nan(w[0], w[1]), max2_nan(w[2], w[3]));
    const uint32_t l = min2_nan(min2_nan(w[0], w[1]), min2_nan(w[2], w[3])) ^ kSigns;
    uint32_t both = max2_nan(__byte_perm(t, l, 0x5410), __byte_perm(t, l, 0x7632));
    both = max2_nan(both, __shfl_xor_sync(0xffffffffu, both, 1));
    both = max2_nan(both, __shfl_xor_sync(0xffffffffu, both, 2));
    *top = __uint_as_float(both << 16);
    *low = __uint_as_float(both & 0xffff0000u);
  } else {
    *top = x[0];
    *low = -x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      *top = max_nan(*top, x[i]);
      *low = max_nan(*low, -x[i]);
    }
#pragma unroll
    for (int step = 1; step < 4; step *= 2) {
      *top = max_nan(*top, __shfl_xor_sync(0xffffffffu, *top, step));
      *low = max_nan(*low, __shfl_xor_sync(0xffffffffu, *low, step));
    }
  }
}

// The group's scale (quad: which of its four lanes this is).
template <typename T>
__device__ __forceinline__ __half group_scale(const uint4* raw, const float* x, int quad) {
  float top, low;
  group_range<T>(raw, x, &top, &low);
  float peak = top > low ? top : -low;
  if (__any_sync(0xffffffffu, top == low)) {   // largest magnitudes of both signs: the first one counts
    uint32_t first = 64;                       // 2 * place, + 1 where it is negative
#pragma unroll
    for (int i = 7; i >= 0; --i)
      if (fabsf(x[i]) == top) first = 2 * (8 * quad + i) + (x[i] < 0.f ? 1 : 0);
    first = min(first, __shfl_xor_sync(0xffffffffu, first, 1));
    first = min(first, __shfl_xor_sync(0xffffffffu, first, 2));
    if (top == low) peak = first & 1 ? -top : top;
  }
  if (!(fabsf(peak) < INFINITY)) return __ushort_as_half((unsigned short)0x7fff);
  return __float2half_rn(fminf(fmaxf(peak * -0.125f, -65504.f), 65504.f));
}

// Codes + 8 of eight elements, element i in bits 4 i: rint(x / s) of the exact quotient, ties to even.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(float* x, float s) {
  if (!(s != 0.f) || s != s) return 0x88888888u;   // (NaN: the codes do not matter, but are the same for the same rows)
  float inv;
  uint32_t m[8];
  if constexpr (sizeof(T) == 2) {
    // A quotient of 8 by 11 bits is a tie or at least 2^-12 away from one, and x * inv errs by less than 2^-19.  On top of 192 fp32 has
    // steps of 2^-16: there a tie is exact again, and everything else stays on its side.
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(inv) : "f"(s));
    if (!(fabsf(s) >= 0x1p-14f && fabsf(s) < 65504.f)) {   // a scale of fewer digits, or held: quotients may lie outside of -8 .. 8
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(x[i], -8.f * fabsf(s)), 8.f * fabsf(s));
    }
    constexpr float kStep = 192.f;
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float t0, t1, k0, k1;
      tc::fma2(t0, t1, x[i], x[i + 1], inv, kStep);
      tc::add2g(k0, k1, fminf(t0, kStep + 7.f), fminf(t1, kStep + 7.f), kMagic - kStep + 8.f, kMagic - kStep + 8.f);
      m[i] = __float_as_uint(k0);
      m[i + 1] = __float_as_uint(k1);
    }
  } else {
    // A quotient of 24 by 11 bits may be 2^-24 of itself away from a tie; x * inv errs by less than 2^-22 of itself.  Those within 2^-18 of a
    // half-integer are divided.
    inv = __frcp_rn(s);
    float worst = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float t = fminf(fmaxf(x[i] * inv, -8.f), 7.f), k = t + (kMagic + 8.f);
      worst = fmaxf(worst, fabsf(t - (k - (kMagic + 8.f))));
      m[i] = __float_as_uint(k);
    }
    if (worst > 0.5f - 0x1p-18f) {
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = __float_as_uint(fminf(fmaxf(__fdiv_rn(x[i], s), -8.f), 7.f) + (kMagic + 8.f));
    }
  }
  const uint32_t even = __byte_perm(__byte_perm(m[0], m[2], 0x0040), __byte_perm(m[4], m[6], 0x0040), 0x5410);
  const uint32_t odd = __byte_perm(__byte_perm(m[1], m[3], 0x0040), __byte_perm(m[5], m[7], 0x0040), 0x5410);
  return even + odd * 16;
}

// A CTA: the tokens of one sample and kv-head that fall into one tile.  Tiles of a sample: from the one that its first row lies in.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_write_kernel(PackedView c, RowSource src, int I, FastDiv by_heads,
                                                                FastDiv by_tiles, const int32_t* start, const int32_t* counts) {
  using L = PackedLayout<D>;
  constexpr int G = L::G, kPerRow = D / 8, kRows = kThreads / kPerRow, kSteps = kPackedTile / kRows, kVec = sizeof(T) / 2;
  __shared__ __align__(16) uint8_t image[L::kBytes];
  pdl_wait();
  const int rest = by_heads(blockIdx.x), head = blockIdx.x - rest * c.Hkv, smp = by_tiles(rest), tile_of_sample = rest - smp * (int)by_tiles.d;
  const int begin = start != nullptr ? start[smp] : 0, count = counts != nullptr ? min(counts[smp], I) : I;
  const long long row0 = ((long long)(begin >> 5) + tile_of_sample) * kPackedTile;   // of the tile
  const long long lo = max((long long)begin, row0), hi = min((long long)begin + count, row0 + kPackedTile);   // rows to store, [lo, hi)
  if (hi <= lo) return;
  if (lo < 0 || hi > c.capacity) {
    if (threadIdx.x == 0) atomicExch(c.status, kErrCapacity);
  }
  if (hi <= 0 || lo >= c.capacity) return;
  const int first = (int)(max(lo, 0ll) - row0), last = (int)(min(hi, (long long)c.capacity) - row0);   // rows of the tile, [first, last)
  const bool all_rows = first == 0 && last == kPackedTile;
  const int part = threadIdx.x % kPerRow, group = part / 4, quad = part % 4;
  const int in_cta = threadIdx.x / kPerRow;   // a step goes kRows rows further
  const long long token = row0 + in_cta - begin;
  const T* k = static_cast<const T*>(src.k) + smp * src.k_sample + head * src.k_head + token * src.k_token + part * 8;
  const T* v = static_cast<const T*>(src.v) + smp * src.v_sample + head * src.v_head + token * src.v_token + part * 8;
  uint4 raw[kSteps][2][kVec];
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = in_cta + i * kRows;
    const bool in = row >= first && row < last;
#pragma unroll
    for (int j = 0; j < kVec; ++j) {
      raw[i][0][j] = in ? ld_global_16(k + i * kRows * src.k_token + 4 * j) : make_uint4(0, 0, 0, 0);
      raw[i][1][j] = in ? ld_global_16(v + i * kRows * src.v_token + 4 * j) : make_uint4(0, 0, 0, 0);
    }
  }
  uint8_t* k_codes = image + in_cta * (D / 2) + quad * 4 * G + group * 4;
  uint8_t* v_codes = image + L::value_codes(in_cta, group, 2 * quad);
  uint8_t* k_scale = image + L::kKeyScales + (in_cta * G + group) * 2;
#pragma unroll
  for (int i = 0; i < kSteps; ++i) {
    const int row = in_cta + i * kRows;
    if (!all_rows && !__any_sync(0xffffffffu, row >= first && row < last)) continue;
    float x[8];
    unpack8<T>(raw[i][0], x);
    __half s = group_scale<T>(raw[i][0], x, quad);
    *reinterpret_cast<uint32_t*>(k_codes + i * kRows * (D / 2)) = quantise8<T>(x, __half2float(s));
    if (quad == 0) *reinterpret_cast<__half*>(k_scale + i * kRows * G * 2) = s;
    unpack8<T>(raw[i][1], x);
    s = group_scale<T>(raw[i][1], x, quad);
    const uint32_t w = quantise8<T>(x, __half2float(s));
    *reinterpret_cast<uint16_t*>(v_codes + i * kRows * (D / 2)) = (uint16_t)w;
    *reinterpret_cast<uint16_t*>(v_codes + i * kRows * (D / 2) + 16 * G) = (uint16_t)(w >> 16);
    if (quad == 0) *reinterpret_cast<__half*>(image + L::value_scale(row, group)) = s;
  }
  __syncthreads();
  uint8_t* tile = c.data + (((size_t)smp * c.Hkv + head) * c.tiles + (size_t)(row0 / kPackedTile)) * L::kBytes;
  if (all_rows) {
    for (int i = threadIdx.x; i < L::kBytes / 16; i += kThreads)
      reinterpret_cast<uint4*>(tile)[i] = reinterpret_cast<const uint4*>(image)[i];
    return;
  }
  // some rows only, the others are left as they were: rows of key codes and scales lie together, those of values do not
  for (int i = threadIdx.x; i < kPackedTile * D / 32; i += kThreads)
    if (i / (D / 32) >= first && i / (D / 32) < last) reinterpret_cast<uint4*>(tile)[i] = reinterpret_cast<const uint4*>(image)[i];
  static_assert(kPackedTile * G <= kThreads, "");
  if (threadIdx.x < kPackedTile * G) {
    const int row = threadIdx.x / G, g = threadIdx.x % G, ks = L::kKeyScales + threadIdx.x * 2, vs = L::value_scale(row, g);
    if (row >= first && row < last) {
      *reinterpret_cast<uint16_t*>(tile + ks) = *reinterpret_cast<const uint16_t*>(image + ks);
      *reinterpret_cast<uint16_t*>(tile + vs) = *reinterpret_cast<const uint16_t*>(image + vs);
    }
  }
  for (int i = threadIdx.x; i < kPackedTile * 8 * G; i += kThreads) {
    const int row = i % 2 * 4 + i / 2 / G % 4 + i / (64 * G) * 8;   // (value_codes the other way round)
    if (row >= first && row < last)
      reinterpret_cast<uint16_t*>(tile + L::kValueCodes)[i] = reinterpret_cast<const uint16_t*>(image + L::kValueCodes)[i];
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, uint32_t w, float s, bool wanted) {   // (by whole warps)
  // The code + 8 in the highest digits of an fp32 number is 16 + (code + 8); of 5 by 11 bits no product is rounded.
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    f[i] = fmaf(__uint_as_float(((i < 5 ? w << (19 - 4 * i) : w >> (4 * i - 19)) & 0x00780000u) | 0x41800000u), s, -24.f * s);
  if constexpr (sizeof(T) == 4) {
    // Two lanes' 64 bytes: each store has whole sectors of 32 bytes when the even lane has the first halves of both, the odd one the second.
    const bool odd = threadIdx.x & 1;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float other = __shfl_xor_sync(0xffffffffu, odd ? f[i] : f[i + 4], 1);
      (odd ? f[i] : f[i + 4]) = other;
    }
    if (!wanted) return;
    if (odd) p -= 4;   // even: its own first half, then the odd lane's; odd: the even lane's second half, then its own
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4*>(p + 8) = make_float4(f[4], f[5], f[6], f[7]);
  } else {
    if (!wanted) return;
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 pair = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      o[i] = *reinterpret_cast<const uint32_t*>(&pair);
    }
    st_global_16(p, make_uint4(o[0], o[1], o[2], o[3]));
  }
}

// A CTA: the rows of one sample and kv-head that one tile has of those asked for.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_read_kernel(PackedView c, int row0, int count, FastDiv by_heads,
                                                               FastDiv by_tiles, const int32_t* lens, T* k_out, T* v_out) {
  using L = PackedLayout<D>;
  constexpr int G = L::G, kPerRow = D / 8;
  __shared__ __align__(16) uint8_t image[L::kBytes];
  pdl_wait();
  const int rest = by_heads(blockIdx.x), head = blockIdx.x - rest * c.Hkv, smp = by_tiles(rest);
  const int t = row0 / kPackedTile + rest - smp * (int)by_tiles.d, base = t * kPackedTile;
  const int first = max(row0 - base, 0), last = min(row0 + count - base, kPackedTile);   // rows of the tile, [first, last)
  const int len = lens != nullptr ? min(max(lens[smp], 0), c.capacity) - base : kPackedTile;   // rows of the tile below the sample's length
  const uint8_t* tile = c.data + (((size_t)smp * c.Hkv + head) * c.tiles + t) * L::kBytes;
  for (int i = threadIdx.x; i < L::kBytes / 16; i += kThreads) {
    // pieces of key codes are of one row, those of value codes of eight
    const int piece = i * 16 - L::kValueCodes, row = piece >= 0 ? piece / (8 * D / 2) * 8 : i / (D / 32);
    const bool wanted = piece >= 0 ? row + 8 > first && row < last : i * 16 >= L::kCodes || (row >= first && row < last);
    if (wanted) reinterpret_cast<uint4*>(image)[i] = ld_global_16(tile + i * 16);
  }
  __syncthreads();
  constexpr int kRows = kThreads / kPerRow;
  const int part = threadIdx.x % kPerRow, group = part / 4, quad = part % 4, in_cta = threadIdx.x / kPerRow;
  const uint8_t* k_codes = image + in_cta * (D / 2) + quad * 4 * G + group * 4;
  const uint8_t* v_codes = image + L::value_codes(in_cta, group, 2 * quad);
  const uint8_t* k_scale = image + L::kKeyScales + (in_cta * G + group) * 2;
  const size_t out0 = (((size_t)smp * count + (base + in_cta - row0)) * c.Hkv + head) * D + part * 8, step = (size_t)kRows * c.Hkv * D;
#pragma unroll
  for (int i = 0; i < kPackedTile / kRows; ++i) {
    const int row = in_cta + i * kRows;
    const bool wanted = row >= first && row < last;
    if (!__any_sync(0xffffffffu, wanted)) continue;
    uint32_t wk = 0, wv = 0;
    float fk = 0.f, fv = 0.f;
    if (wanted && row < len) {
      wk = *reinterpret_cast<const uint32_t*>(k_codes + i * kRows * (D / 2));
      wv = *reinterpret_cast<const uint16_t*>(v_codes + i * kRows * (D / 2)) |
           ((uint32_t)*reinterpret_cast<const uint16_t*>(v_codes + i * kRows * (D / 2) + 16 * G) << 16);
      fk = __half2float(*reinterpret_cast<const __half*>(k_scale + i * kRows * G * 2));
      fv = __half2float(*reinterpret_cast<const __half*>(image + L::value_scale(row, group)));
    }
    store8(k_out + out0 + i * step, wk, fk, wanted);
    store8(v_out + out0 + i * step, wv, fv, wanted);
  }
}

template <typename T, int D>
cudaError_t write_t(const PackedView& c, const RowSource& src, int I, const int32_t* start, const int32_t* counts, cudaStream_t st) {
  const int tiles = start == nullptr ? (I + kPackedTile - 1) / kPackedTile : (I + 2 * kPackedTile - 2) / kPackedTile;   // that I rows may touch
  const long long blocks = (long long)c.nsamples * tiles * c.Hkv;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  ProfileScope prof(kPacked, st);
  const cudaError_t err = launch_dependent(packed_write_kernel<T, D>, dim3((unsigned)blocks), dim3(kThreads), 0, st, c, src, I,
                                           FastDiv((uint32_t)c.Hkv), FastDiv((uint32_t)tiles), start, counts);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, int D>
cudaError_t read_t(const PackedView& c, int row0, int count, const int32_t* lens, void* k_out, void* v_out, cudaStream_t st) {
  const int tiles = (row0 + count - 1) / kPackedTile - row0 / kPackedTile + 1;
  const long long blocks = (long long)c.nsamples * tiles * c.Hkv;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  ProfileScope prof(kPacked, st);
  const cudaError_t err = launch_dependent(packed_read_kernel<T, D>, dim3((unsigned)blocks), dim3(kThreads), 0, st, c, row0, count,
                                           FastDiv((uint32_t)c.Hkv), FastDiv((uint32_t)tiles), lens, static_cast<T*>(k_out), static_cast<T*>(v_out));
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

}  // namespace

cudaError_t launch_packed_write(int dtype, int d, const PackedView& c, const RowSource& src, int I, const int32_t* start,
                                const int32_t* counts, cudaStream_t st) {
  if (dtype == 0) return d == 64 ? write_t<float, 64>(c, src, I, start, counts, st) : write_t<float, 128>(c, src, I, start, counts, st);
  return d == 64 ? write_t<__nv_bfloat16, 64>(c, src, I, start, counts, st) : write_t<__nv_bfloat16, 128>(c, src, I, start, counts, st);
}

cudaError_t launch_packed_read(int dtype, int d, const PackedView& c, int row0, int rows, const int32_t* lens, void* k_out,
                               void* v_out, cudaStream_t st) {
  if (dtype == 0) return d == 64 ? read_t<float, 64>(c, row0, rows, lens, k_out, v_out, st)
                                 : read_t<float, 128>(c, row0, rows, lens, k_out, v_out, st);
  return d == 64 ? read_t<__nv_bfloat16, 64>(c, row0, rows, lens, k_out, v_out, st)
                 : read_t<__nv_bfloat16, 128>(c, row0, rows, lens, k_out, v_out, st);
}

}  // namespace bm
