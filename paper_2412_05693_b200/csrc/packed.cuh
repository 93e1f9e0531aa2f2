// A cache held in 4 bits ("packed cache"): layout of its rows and the launchers of its kernels.
//
// A row (one key or one value, d elements) is cut into G = d / 32 groups.  Of a group, with x* its first element of the largest
// magnitude:  s = fp16(x* / -8) held to +-65504,  code = clamp(rint(x / s), -8, 7),  value = code * s.  All 16 codes are used: x*
// stands at -8 exactly (up to the rounding of s), which makes the step an eighth of the largest magnitude where codes of -7 .. 7
// have a seventh.  Stored is code + 8.  A group with a NaN or an infinity has a NaN for its scale.
//
// Four slabs, rows of a (layer, sample, kv-head) together: codes [rows][d / 2] and scales [rows][G] of the keys, the same of the
// values.  A row's code bytes are ordered for the fragments that mma.m16n8k16 wants of them, so that a lane fetches all its codes
// of a row at once and unpacks two by one AND (see packed_attend.cu):
//   keys:   the lane (r, c) of a warp, r = lane / 4, c = lane % 4, multiplies the elements 32 g + 8 c + (0 .. 7) of every group g:
//           a 32-bit word, element i in bits 4 i.  Its G words lie together at byte c * 4 G.
//   values: the lane (r, c) multiplies the elements 32 g + 4 r + (0 .. 3): a 16-bit half, its G halves together at byte r * 2 G.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace bm {

constexpr int kPackedGroup = 32;     // elements that share a scale
constexpr int kPackedTile = 32;      // rows of one step of the attention kernel; a cache's rows are padded to a multiple
constexpr int kErrCapacity = 3;      // BM_ERR_CAPACITY

// One layer's packed rows for a range of samples; unit = local sample * Hkv + kv-head, its rows start at unit * stride.
struct PackedView {
  uint8_t* k_codes;     // [units][stride][d / 2]
  uint8_t* v_codes;
  __half* k_scales;     // [units][stride][d / 32]
  __half* v_scales;
  int32_t capacity;     // rows a cache may hold
  int32_t stride;       // capacity, rounded up to kPackedTile
  int32_t nsamples, Hq, Hkv, g;
  int32_t* status;      // device status word
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
  float* partial;          // workspace
  float scale;
  int32_t max_len;         // what the work is split by
};
size_t packed_attend_workspace(int d, int g, int queries);   // bytes for calls of up to this many queries
cudaError_t launch_packed_attend(int dtype, int d, const PackedView& c, const PackedAttend& a, cudaStream_t st);

}  // namespace bm
