// Writing rows into a packed cache, and reading them back (packed.cuh has the format).
//
// Both are bound by HBM: a row of d elements comes in as d * e bytes and goes out as d / 2 + d / 16, or the other way round.  A thread
// has eight consecutive elements (one 16-byte load in bf16), four threads a group: the group's peak takes two shuffles, and every
// word of a packed row is written by one thread.
#include <algorithm>

#include "packed.cuh"

namespace bm {
namespace {

constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ void load8(const T* p, float* x);
template <>
__device__ __forceinline__ void load8<float>(const float* p, float* x) {
  const uint4 a = ld_global_16(p), b = ld_global_16(p + 4);
  Elem<float>::unpack(a, x);
  Elem<float>::unpack(b, x + 4);
}
template <>
__device__ __forceinline__ void load8<__nv_bfloat16>(const __nv_bfloat16* p, float* x) {
  Elem<__nv_bfloat16>::unpack(ld_global_16(p), x);
}

// Code + 8 of every element: rint(x / s) of the exact quotient, ties to even.  x / s has at most 24 by 11 bits, so it is a tie or
// at least 2^-24 of itself away from one; x * (1 / s) errs by less than 2^-22 of itself, so only quotients within 2^-18 of a
// half-integer (|quotient| <= 8 where it is not clamped) have to be divided.
constexpr float kNearTie = 0.5f - 0x1p-18f;

__device__ __forceinline__ uint32_t quantise8(const float* x, float s) {
  constexpr float kMagic = 12582912.f + 8.f;   // 1.5 * 2^23 + 8: adding it rounds to integers, the low bits are the code + 8
  if (!(s != 0.f)) return 0x88888888u;
  const float inv = __frcp_rn(s);
  uint32_t w = 0;
  float worst = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float t = fminf(fmaxf(x[i] * inv, -8.f), 7.f);
    const float m = t + kMagic;
    worst = fmaxf(worst, fabsf(t - (m - kMagic)));
    w |= (__float_as_uint(m) & 15u) << (4 * i);
  }
  if (worst > kNearTie) {
    w = 0;
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
      const float m = fminf(fmaxf(__fdiv_rn(x[i], s), -8.f), 7.f) + kMagic;
      w |= (__float_as_uint(m) & 15u) << (4 * i);
    }
  }
  return w;
}

// The group's scale: four lanes with eight elements each, in order.
__device__ __forceinline__ __half group_scale(const float* x, int c) {
  float peak = x[0];
  uint32_t most = __float_as_uint(x[0]) & 0x7fffffffu;
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    const uint32_t m = __float_as_uint(x[i]) & 0x7fffffffu;   // magnitudes compare as integers, NaN and infinity above the rest
    if (m > most) { most = m; peak = x[i]; }
  }
#pragma unroll
  for (int step = 1; step < 4; step *= 2) {
    const float other = __shfl_xor_sync(0xffffffffu, peak, step);
    const uint32_t m = __float_as_uint(other) & 0x7fffffffu;
    if (m > most || (m == most && (c & step))) { most = m; peak = other; }   // equal: the lower elements' lane
  }
  if (most >= 0x7f800000u) return __ushort_as_half((unsigned short)0x7fff);
  return __float2half_rn(fminf(fmaxf(peak * -0.125f, -65504.f), 65504.f));
}

// One thread: eight elements of a key row and of the value row beside it.  Row index: ((sample * I + token) * Hkv + head).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_write_kernel(PackedView c, RowSource src, int I, long long rows,
                                                                const int32_t* start, const int32_t* counts) {
  constexpr int G = D / kPackedGroup, kPerRow = D / 8;
  pdl_wait();
  const long long row = ((long long)blockIdx.x * kThreads + threadIdx.x) / kPerRow;
  const int part = threadIdx.x % kPerRow, group = part / 4, quad = part % 4;
  const bool valid = row < rows;
  const long long token_row = valid ? row / c.Hkv : 0;
  const int head = valid ? (int)(row % c.Hkv) : 0, smp = (int)(token_row / I), token = (int)(token_row % I);
  bool kept = valid && (counts == nullptr || token < counts[smp]);
  const long long at = (long long)(start != nullptr ? start[smp] : 0) + token;
  if (kept && (at < 0 || at >= c.capacity)) {
    kept = false;
    if (part == 0) atomicExch(c.status, kErrCapacity);
  }
  if (!__any_sync(0xffffffffu, kept)) return;
  float x[2][8] = {};
  if (kept) {
    load8(static_cast<const T*>(src.k) + smp * src.k_sample + token * src.k_token + head * src.k_head + part * 8, x[0]);
    load8(static_cast<const T*>(src.v) + smp * src.v_sample + token * src.v_token + head * src.v_head + part * 8, x[1]);
  }
  const __half sk = group_scale(x[0], quad), sv = group_scale(x[1], quad);
  const float fk = __half2float(sk), fv = __half2float(sv);
  // a NaN scale: the codes do not matter, but are the same for the same rows
  const uint32_t wk = fk == fk ? quantise8(x[0], fk) : 0x88888888u, wv = fv == fv ? quantise8(x[1], fv) : 0x88888888u;
  if (!kept) return;
  using L = PackedLayout<D>;
  uint8_t* tile = c.data + (((size_t)smp * c.Hkv + head) * c.tiles + (size_t)at / kPackedTile) * L::kBytes;
  const int in = (int)(at % kPackedTile);
  uint8_t* kc = tile + in * (D / 2);
  *reinterpret_cast<uint32_t*>(kc + quad * 4 * G + group * 4) = wk;
  *reinterpret_cast<uint16_t*>(tile + L::value_codes(in, group, 2 * quad)) = (uint16_t)wv;
  *reinterpret_cast<uint16_t*>(tile + L::value_codes(in, group, 2 * quad + 1)) = (uint16_t)(wv >> 16);
  if (quad == 0) {
    *reinterpret_cast<__half*>(tile + L::kKeyScales + (in * G + group) * 2) = sk;
    *reinterpret_cast<__half*>(tile + L::value_scale(in, group)) = sv;
  }
}

template <typename T>
__device__ __forceinline__ void store8(T* p, uint32_t w, float s);
template <>
__device__ __forceinline__ void store8<float>(float* p, uint32_t w, float s) {
  float f[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (float)((int)((w >> (4 * i)) & 15u) - 8) * s;
  *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
template <>
__device__ __forceinline__ void store8<__nv_bfloat16>(__nv_bfloat16* p, uint32_t w, float s) {
  uint32_t o[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 pair = __floats2bfloat162_rn((float)((int)((w >> (8 * i)) & 15u) - 8) * s,
                                                      (float)((int)((w >> (8 * i + 4)) & 15u) - 8) * s);
    o[i] = *reinterpret_cast<const uint32_t*>(&pair);
  }
  st_global_16(p, make_uint4(o[0], o[1], o[2], o[3]));
}

// One thread: eight elements of a key row and of the value row beside it.  Row index: ((sample * count + row) * Hkv + head).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) packed_read_kernel(PackedView c, int row0, int count, long long rows, const int32_t* lens,
                                                               T* k_out, T* v_out) {
  constexpr int G = D / kPackedGroup, kPerRow = D / 8;
  pdl_wait();
  const long long row = ((long long)blockIdx.x * kThreads + threadIdx.x) / kPerRow;
  if (row >= rows) return;
  const int part = threadIdx.x % kPerRow, group = part / 4, quad = part % 4;
  const long long token_row = row / c.Hkv;
  const int head = (int)(row % c.Hkv), smp = (int)(token_row / count), at = row0 + (int)(token_row % count);
  uint32_t wk = 0x88888888u, wv = 0x88888888u;
  float fk = 0.f, fv = 0.f;
  if (lens == nullptr || at < lens[smp]) {
    using L = PackedLayout<D>;
    const uint8_t* tile = c.data + (((size_t)smp * c.Hkv + head) * c.tiles + at / kPackedTile) * L::kBytes;
    const int in = at % kPackedTile;
    wk = *reinterpret_cast<const uint32_t*>(tile + in * (D / 2) + quad * 4 * G + group * 4);
    wv = *reinterpret_cast<const uint16_t*>(tile + L::value_codes(in, group, 2 * quad)) |
         ((uint32_t)*reinterpret_cast<const uint16_t*>(tile + L::value_codes(in, group, 2 * quad + 1)) << 16);
    fk = __half2float(*reinterpret_cast<const __half*>(tile + L::kKeyScales + (in * G + group) * 2));
    fv = __half2float(*reinterpret_cast<const __half*>(tile + L::value_scale(in, group)));
  }
  store8(k_out + row * D + part * 8, wk, fk);
  store8(v_out + row * D + part * 8, wv, fv);
}

template <typename T, int D>
cudaError_t write_t(const PackedView& c, const RowSource& src, int I, const int32_t* start, const int32_t* counts, cudaStream_t st) {
  const long long rows = (long long)c.nsamples * I * c.Hkv, blocks = (rows * (D / 8) + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const cudaError_t err = launch_dependent(packed_write_kernel<T, D>, dim3((unsigned)blocks), dim3(kThreads), 0, st, c, src, I, rows,
                                           start, counts);
  count_launch();
  return err != cudaSuccess ? err : cudaGetLastError();
}

template <typename T, int D>
cudaError_t read_t(const PackedView& c, int row0, int count, const int32_t* lens, void* k_out, void* v_out, cudaStream_t st) {
  const long long rows = (long long)c.nsamples * count * c.Hkv, blocks = (rows * (D / 8) + kThreads - 1) / kThreads;
  if (blocks > 0x7fffffff) return cudaErrorInvalidConfiguration;
  const cudaError_t err = launch_dependent(packed_read_kernel<T, D>, dim3((unsigned)blocks), dim3(kThreads), 0, st, c, row0, count, rows,
                                           lens, static_cast<T*>(k_out), static_cast<T*>(v_out));
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
