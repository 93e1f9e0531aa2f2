// A cache held in 4 bits ("packed cache"): layout of its rows and the launchers of its kernels.
//
// A row (one key or one value, d elements) is cut into G = d / 32 groups.  Of a group, with x* its first element of the largest
// magnitude:  s = fp16(x* / -8) held to +-65504,  code = clamp(rint(x / s), -8, 7),  value = code * s.  All 16 codes are used: x*
// stands at -8 exactly (up to the rounding of s), which makes the step an eighth of the largest magnitude where codes of -7 .. 7
// have a seventh.  Stored is code + 8.  A group with a NaN or an infinity has a NaN for its scale.
//
// Rows are stored in tiles of 32 (a cache's rows are padded to whole tiles), each tile one piece of 32 * 2 * (d / 2 + d / 16) bytes that
// a single bulk copy fetches:
//     key codes [32][d / 2] | key scales [32][G] | value scales, see below | value codes [32][d / 2]
// The bytes are ordered for the fragments that mma.m16n8k16 wants, so that a lane fetches what it needs of a row at once and unpacks two
// codes by one AND (packed_attend.cu):
//   key codes:    the lane (r, c) of a warp, r = lane / 4, c = lane % 4, multiplies the elements 32 g + 8 c + (0 .. 7) of every group g: a
//                 32-bit word, element i in bits 4 i.  Its G words lie together at byte c * 4 G of the row.
//   value codes:  the lane (r, c) multiplies the elements 32 g + 4 r + (0 .. 3), a 16-bit half per row and group, of the rows
//                 16 t + 8 p + c and + 4 together: [t][p][r][c][g][which row], 16-bit halves.
//   value scales: of the same rows [t][c][p][g][which row].
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace bm {

constexpr int kPackedGroup = 32;     // elements that share a scale
constexpr int kPackedTile = 32;      // rows of a tile
constexpr int kErrCapacity = 3;      // BM_ERR_CAPACITY

// One layer's packed rows for a range of samples; unit = local sample * Hkv + kv-head, its tiles start at unit * tiles.
struct PackedView {
  uint8_t* data;        // [units][tiles][tile bytes]
  int32_t capacity;     // rows a cache may hold
  int32_t tiles;        // of 32 rows, per cache
  int32_t nsamples, Hq, Hkv, g;
  int32_t* status;      // device status word
};

// Bytes and places inside a tile.
template <int D>
struct PackedLayout {
  static constexpr int G = D / kPackedGroup;
  static constexpr int kCodes = kPackedTile * D / 2, kScales = kPackedTile * G * 2;
  static constexpr int kKeyScales = kCodes, kValueScales = kCodes + kScales, kValueCodes = kCodes + 2 * kScales;
  static constexpr int kBytes = 2 * (kCodes + kScales);
  // byte of the value scale of group g of the tile's row
  __host__ __device__ static constexpr int value_scale(int row, int g) {
    return kValueScales + 2 * ((((row / 16 * 4 + row % 4) * 2 + row % 16 / 8) * G + g) * 2 + row / 4 % 2);
  }
  // byte of the value codes of the elements 32 g + 4 r .. + 3 of the tile's row
  __host__ __device__ static constexpr int value_codes(int row, int g, int r) {
    return kValueCodes + 2 * ((((row / 8 * 8 + r) * 4 + row % 4) * G + g) * 2 + row / 4 % 2);
  }
};

// x / d for 0 <= x < 2^31, 1 <= d < 2^31: with 2^(s - 1) < d <= 2^s and m = floor(2^32 (2^s - d) / d) + 1 (the round-up method of Granlund and
// Montgomery, 1994), x / d = (mulhi(x, m) + x) >> s, which fits 32 bits for such x.
struct FastDiv {
  uint32_t d, m, s;
  FastDiv() = default;
  explicit FastDiv(uint32_t by) : d(by), m(0), s(0) {
    while ((1ull << s) < by) ++s;
    m = (uint32_t)(((((1ull << s) - by) << 32) / by) + 1);
  }
  __device__ __forceinline__ int operator()(int x) const { return (int)((__umulhi((uint32_t)x, m) + (uint32_t)x) >> s); }
};

// Rows to quantise: element (sample, token, head) of k starts at k + sample * sample_stride + token * token_stride + head * head_stride.
struct RowSource {
  const void *k, *v;
  int64_t k_sample, k_token, k_head, v_sample, v_token, v_head;   // strides in elements
};

cudaError_t launch_packed_write(int dtype, int d, const PackedView& c, const RowSource& src, int I, const int32_t* start,
                                const int32_t* counts, cudaStream_t st);
cudaError_t launch_packed_read(int dtype, int d, const PackedView& c, int row0, int rows, const int32_t* lens, void* k_out,
                               void* v_out, cudaStream_t st);

struct PackedAttend {
  const void* q;           // [nsamples][I][Hq][d], strides in elements
  int64_t q_sample, q_token;
  int32_t I;
  const int32_t* lens;     // [nsamples] rows of every sample's caches, its own I among them
  const int32_t* first;    // [nsamples] first row that counts, or null
  void* out;               // [nsamples][I][Hq][d] contiguous
  void* workspace;
  float scale;
  int32_t max_len;         // the longest length to expect
};
// Bytes for calls of up to this many samples, kv-heads and queries.
size_t packed_attend_workspace(int d, int batch, int Hkv, int g, int queries, int tiles);
cudaError_t launch_packed_wait_selftest(int32_t* status, cudaStream_t st);
extern thread_local int g_last_packed_path;   // (packed_api.cu) what bm_last_packed_path reports
// (packed_block.cu) the same for blocks of queries, bf16
size_t packed_block_workspace(int batch, int Hkv);
cudaError_t launch_packed_block(int d, const PackedView& c, const PackedAttend& a, cudaStream_t st);
bool packed_block_pays(int d, const PackedView& c, int I, int max_len);
cudaError_t launch_packed_attend(int dtype, int d, const PackedView& c, const PackedAttend& a, cudaStream_t st);

}  // namespace bm
