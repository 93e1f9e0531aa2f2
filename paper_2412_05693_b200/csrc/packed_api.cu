// Entry points of packed caches: memory model, arena, argument checks, launches (packed.cuh has the format).
#include <cmath>
#include <new>

#include "../../include/batchmax.h"
#include "packed.cuh"

namespace bm {
thread_local int g_last_packed_path = 0;
}  // namespace bm

using namespace bm;

struct bm_packed {
  bm_packed_config_t cfg;
  int tiles, g;
  float scale;
  int32_t* status;
  uint8_t* data;    // [L][b][Hkv][tiles] tiles of 32 rows
};

namespace {

constexpr size_t kHeader = 256;   // status word

bool config_ok(const bm_packed_config_t* c, bool need_batch) {
  if (c == nullptr) return false;
  if (need_batch && c->batch < 1) return false;
  if (c->n_layers < 1 || c->n_q_heads < 1 || c->n_kv_heads < 1 || c->n_q_heads % c->n_kv_heads != 0) return false;
  if (!(c->head_dim == 64 || c->head_dim == 128)) return false;
  if (c->capacity < 1 || c->capacity > (1 << 24)) return false;
  if (c->queries_max < 1 || c->queries_max > (1 << 24)) return false;
  if (!(c->dtype == BM_F32 || c->dtype == BM_BF16)) return false;
  if (!(c->softmax_scale >= 0.f) || std::isinf(c->softmax_scale)) return false;
  if (c->device < 0) return false;
  return true;
}

int tiles_of(const bm_packed_config_t* c) { return (c->capacity + kPackedTile - 1) / kPackedTile; }
size_t tile_bytes(const bm_packed_config_t* c) { return c->head_dim == 64 ? PackedLayout<64>::kBytes : PackedLayout<128>::kBytes; }

// false: more than a size holds
bool per_sample(const bm_packed_config_t* c, size_t* bytes) {
  return !__builtin_mul_overflow((size_t)c->n_layers * (size_t)c->n_kv_heads, (size_t)tiles_of(c) * tile_bytes(c), bytes);
}
bool arena_size(const bm_packed_config_t* c, size_t* bytes) {
  return per_sample(c, bytes) && !__builtin_mul_overflow(*bytes, (size_t)c->batch, bytes) && !__builtin_add_overflow(*bytes, kHeader, bytes);
}
size_t workspace_size(const bm_packed_config_t* c) {
  return packed_attend_workspace(c->head_dim, c->batch, c->n_kv_heads, c->n_q_heads / c->n_kv_heads, c->queries_max, tiles_of(c));
}

bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool strides_ok(const bm_packed_config_t& c, const int64_t* s, int n) {
  const int64_t unit = c.dtype == BM_BF16 ? 8 : 4;   // elements in 16 bytes
  for (int i = 0; i < n; ++i)
    if (s[i] < 0 || s[i] % unit != 0) return false;
  return true;
}

// The handle's device for the length of a call.
struct OnDevice {
  int before = -1;
  cudaError_t err;
  explicit OnDevice(int device) {
    err = cudaGetDevice(&before);
    if (err == cudaSuccess && before != device) err = cudaSetDevice(device);
    else before = -1;
  }
  ~OnDevice() {
    if (before >= 0) cudaSetDevice(before);
  }
};

bm_status_t status_of(cudaError_t e) { return e == cudaSuccess ? BM_OK : static_cast<bm_status_t>(note_cuda_error(e)); }

bool range_ok(const bm_packed* c, int layer, int sample0, int nsamples) {
  return c != nullptr && layer >= 0 && layer < c->cfg.n_layers && sample0 >= 0 && nsamples >= 1 &&
         (long long)sample0 + nsamples <= c->cfg.batch;
}

PackedView view_of(const bm_packed* c, int layer, int sample0, int nsamples) {
  PackedView v;
  v.data = c->data + ((size_t)layer * c->cfg.batch + sample0) * c->cfg.n_kv_heads * (size_t)c->tiles * tile_bytes(&c->cfg);
  v.capacity = c->cfg.capacity;
  v.tiles = c->tiles;
  v.nsamples = nsamples; v.Hq = c->cfg.n_q_heads; v.Hkv = c->cfg.n_kv_heads; v.g = c->g;
  v.status = c->status;
  return v;
}

}  // namespace

extern "C" {

bm_status_t bm_packed_bytes_per_sample(const bm_packed_config_t* cfg, size_t* bytes) {
  if (!config_ok(cfg, false) || bytes == nullptr) return BM_ERR_INVALID;
  return per_sample(cfg, bytes) ? BM_OK : BM_ERR_INVALID;
}

bm_status_t bm_packed_arena_bytes(const bm_packed_config_t* cfg, size_t* bytes) {
  if (!config_ok(cfg, true) || bytes == nullptr) return BM_ERR_INVALID;
  return arena_size(cfg, bytes) ? BM_OK : BM_ERR_INVALID;
}

bm_status_t bm_packed_max_batch(const bm_packed_config_t* cfg, size_t hbm_budget_bytes, int32_t* b) {
  size_t one = 0;
  if (!config_ok(cfg, false) || b == nullptr || !per_sample(cfg, &one)) return BM_ERR_INVALID;
  const size_t q = hbm_budget_bytes > kHeader ? (hbm_budget_bytes - kHeader) / one : 0;
  *b = (int32_t)(q > 0x7fffffff ? 0x7fffffff : q);
  return BM_OK;
}

bm_status_t bm_packed_workspace_bytes(const bm_packed_config_t* cfg, size_t* bytes) {
  size_t arena = 0;
  if (!config_ok(cfg, true) || bytes == nullptr || !arena_size(cfg, &arena)) return BM_ERR_INVALID;
  *bytes = workspace_size(cfg);
  return BM_OK;
}

bm_status_t bm_packed_create(const bm_packed_config_t* cfg, void* arena, size_t arena_bytes, void* cuda_stream, bm_packed_t** out) {
  size_t need = 0;
  if (!config_ok(cfg, true) || arena == nullptr || out == nullptr || !aligned(arena, 256) || !arena_size(cfg, &need)) return BM_ERR_INVALID;
  if (arena_bytes < need) return BM_ERR_OOM;
  const OnDevice on(cfg->device);
  if (on.err != cudaSuccess) return status_of(on.err);
  bm_packed* c = new (std::nothrow) bm_packed();
  if (c == nullptr) return BM_ERR_OOM;
  c->cfg = *cfg;
  c->tiles = tiles_of(cfg);
  c->g = cfg->n_q_heads / cfg->n_kv_heads;
  c->scale = cfg->softmax_scale > 0.f ? cfg->softmax_scale : 1.0f / std::sqrt((float)cfg->head_dim);
  c->status = static_cast<int32_t*>(arena);
  c->data = static_cast<uint8_t*>(arena) + kHeader;
  if (cudaError_t e = cudaMemsetAsync(arena, 0, need, static_cast<cudaStream_t>(cuda_stream)); e != cudaSuccess) {
    delete c;
    return status_of(e);
  }
  *out = c;
  return BM_OK;
}

bm_status_t bm_packed_destroy(bm_packed_t* cache) {
  if (cache == nullptr) return BM_ERR_INVALID;
  delete cache;
  return BM_OK;
}

bm_status_t bm_packed_write(bm_packed_t* c, int32_t layer, int32_t sample0, int32_t nsamples, const void* k, const void* v,
                            const int64_t* strides, int32_t I, const int32_t* start, const int32_t* counts, void* cuda_stream) {
  if (!range_ok(c, layer, sample0, nsamples) || k == nullptr || v == nullptr) return BM_ERR_INVALID;
  if (!aligned(k, 16) || !aligned(v, 16) || !aligned(start, 4) || !aligned(counts, 4)) return BM_ERR_INVALID;
  if (I < 1 || I > c->cfg.capacity || (strides != nullptr && !strides_ok(c->cfg, strides, 4))) return BM_ERR_INVALID;
  if ((long long)nsamples * c->cfg.n_kv_heads * I > 0x7fffffffLL) return BM_ERR_CAPACITY;
  const int64_t token = (int64_t)c->cfg.n_kv_heads * c->cfg.head_dim;
  RowSource src;
  src.k = k; src.v = v;
  src.k_sample = strides ? strides[0] : token * I; src.k_token = strides ? strides[1] : token;
  src.v_sample = strides ? strides[2] : token * I; src.v_token = strides ? strides[3] : token;
  src.k_head = src.v_head = c->cfg.head_dim;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(launch_packed_write(c->cfg.dtype, c->cfg.head_dim, view_of(c, layer, sample0, nsamples), src, I, start, counts,
                                       static_cast<cudaStream_t>(cuda_stream)));
}

bm_status_t bm_packed_write_from(bm_packed_t* c, int32_t layer, int32_t sample0, int32_t nsamples, const bm_cache_t* from,
                                 int32_t from_layer, int32_t from_sample0, void* cuda_stream) {
  if (!range_ok(c, layer, sample0, nsamples)) return BM_ERR_INVALID;
  CacheRows rows;
  if (int s = cache_range_rows(from, from_layer, from_sample0, nsamples, &rows); s != BM_OK) return static_cast<bm_status_t>(s);
  if (rows.dtype != c->cfg.dtype || rows.head_dim != c->cfg.head_dim || rows.n_kv_heads != c->cfg.n_kv_heads ||
      rows.device != c->cfg.device)
    return BM_ERR_INVALID;
  if (rows.padded) return BM_ERR_STATE;
  if (rows.n > c->cfg.capacity || (long long)nsamples * c->cfg.n_kv_heads * rows.n > 0x7fffffffLL) return BM_ERR_CAPACITY;
  if (rows.n == 0) return BM_OK;
  RowSource src;
  src.k = rows.k; src.v = rows.v;
  src.k_token = src.v_token = rows.head_dim;
  src.k_head = src.v_head = (int64_t)rows.cap * rows.head_dim;
  src.k_sample = src.v_sample = src.k_head * rows.n_kv_heads;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(launch_packed_write(c->cfg.dtype, c->cfg.head_dim, view_of(c, layer, sample0, nsamples), src, rows.n, nullptr, nullptr,
                                       static_cast<cudaStream_t>(cuda_stream)));
}

bm_status_t bm_packed_read(bm_packed_t* c, int32_t layer, int32_t sample0, int32_t nsamples, int32_t row0, int32_t rows,
                           const int32_t* lens, void* k_out, void* v_out, void* cuda_stream) {
  if (!range_ok(c, layer, sample0, nsamples) || k_out == nullptr || v_out == nullptr) return BM_ERR_INVALID;
  if (!aligned(k_out, 16) || !aligned(v_out, 16) || !aligned(lens, 4)) return BM_ERR_INVALID;
  if (row0 < 0 || rows < 1 || (long long)row0 + rows > c->cfg.capacity) return BM_ERR_INVALID;
  if ((long long)nsamples * c->cfg.n_kv_heads * rows > 0x7fffffffLL) return BM_ERR_CAPACITY;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(launch_packed_read(c->cfg.dtype, c->cfg.head_dim, view_of(c, layer, sample0, nsamples), row0, rows, lens, k_out, v_out,
                                      static_cast<cudaStream_t>(cuda_stream)));
}

bm_status_t bm_packed_attend(bm_packed_t* c, int32_t layer, int32_t sample0, int32_t nsamples, const void* q, const int64_t* strides,
                             int32_t I, const int32_t* lens, const int32_t* first, int32_t max_len, void* out, void* workspace,
                             size_t workspace_bytes, void* cuda_stream) {
  if (!range_ok(c, layer, sample0, nsamples) || q == nullptr || lens == nullptr || out == nullptr || workspace == nullptr)
    return BM_ERR_INVALID;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(workspace, 16) || !aligned(lens, 4) || !aligned(first, 4)) return BM_ERR_INVALID;
  if (I < 1 || I > c->cfg.queries_max || max_len < 0 || (strides != nullptr && !strides_ok(c->cfg, strides, 2))) return BM_ERR_INVALID;
  if (workspace_bytes < workspace_size(&c->cfg)) return BM_ERR_OOM;
  if ((long long)nsamples * c->cfg.n_q_heads * I > 0x7fffffffLL) return BM_ERR_CAPACITY;
  const int64_t token = (int64_t)c->cfg.n_q_heads * c->cfg.head_dim;
  PackedAttend a;
  a.q = q;
  a.q_sample = strides ? strides[0] : token * I; a.q_token = strides ? strides[1] : token;
  a.I = I;
  a.lens = lens; a.first = first;
  a.out = out;
  a.workspace = workspace;
  a.scale = c->scale;
  a.max_len = max_len > 0 && max_len < c->cfg.capacity ? max_len : c->cfg.capacity;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(launch_packed_attend(c->cfg.dtype, c->cfg.head_dim, view_of(c, layer, sample0, nsamples), a,
                                        static_cast<cudaStream_t>(cuda_stream)));
}

int32_t bm_last_packed_path(void) { return g_last_packed_path; }

bm_status_t bm_packed_status(bm_packed_t* c, int32_t* device_status, void* cuda_stream) {
  if (c == nullptr || device_status == nullptr) return BM_ERR_INVALID;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  int32_t w = 0;
  if (cudaError_t e = cudaMemcpyAsync(&w, c->status, sizeof(w), cudaMemcpyDeviceToHost, st); e != cudaSuccess) return status_of(e);
  if (cudaError_t e = cudaStreamSynchronize(st); e != cudaSuccess) return status_of(e);
  *device_status = w;
  return BM_OK;
}

bm_status_t bm_packed_clear_status(bm_packed_t* c, void* cuda_stream) {
  if (c == nullptr) return BM_ERR_INVALID;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(cudaMemsetAsync(c->status, 0, sizeof(int32_t), static_cast<cudaStream_t>(cuda_stream)));
}

bm_status_t bm_packed_selftest_wait_timeout(bm_packed_t* c, void* cuda_stream) {
  if (c == nullptr) return BM_ERR_INVALID;
  const OnDevice on(c->cfg.device);
  if (on.err != cudaSuccess) return status_of(on.err);
  return status_of(launch_packed_wait_selftest(c->status, static_cast<cudaStream_t>(cuda_stream)));
}

}  // extern "C"
