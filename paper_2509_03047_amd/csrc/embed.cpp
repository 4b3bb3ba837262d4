// The embedding's host side: validation against a plan's table, the scratch of
// its gradient and the C entry points' checks.
#include "embed.h"

#include <hip/hip_runtime_api.h>

#include <new>

#include "checks.h"
#include "fr_internal.h"

using namespace fr;

struct fr_embed {
  int device = -1;
  fr_embed_info info{};
  uint64_t offset = 0;       // of the table in the state
  uint64_t grad_offset = 0;
  void* mem = nullptr;       // the scratch below
  uint32_t *order = nullptr, *row_of = nullptr;
  Places* places = nullptr;
  float* runs = nullptr;
};

namespace {

uint64_t size_of(uint32_t dtype) { return dtype == FR_F32 ? 4 : 2; }

int validate(const fr_tensor_desc* table, uint32_t n_entries, uint64_t arena_bytes, const fr_embed_desc& d,
             uint64_t grad_bytes, fr_embed* e) {
  if (d.reserved[0] || d.reserved[1] || !d.rows || !d.cols) return FR_E_INVAL;
  if (d.grad_dtype != FR_F32 && d.grad_dtype != FR_BF16) return FR_E_INVAL;
  if (d.entry < 0 || uint32_t(d.entry) >= n_entries) return FR_E_INVAL;
  const uint64_t numel = uint64_t(d.rows) * d.cols;
  if (table[d.entry].numel != numel) return FR_E_INVAL;
  if (d.grad_offset % 16) return FR_E_ALIGN;
  if (d.rows > (1u << 30) || d.cols > (1u << 24) || numel >= (uint64_t(1) << 40) || d.max_tokens >= (1u << 30) ||
      d.first > INT64_MAX - int64_t(d.rows))
    return FR_E_RANGE;
  if (!embed_waves_fit(d.rows, d.cols) || !embed_waves_fit(embed_run_slots(d.max_tokens), d.cols)) return FR_E_RANGE;
  const uint64_t gb = numel * size_of(d.grad_dtype);
  if (d.max_tokens && (d.grad_offset > grad_bytes || gb > grad_bytes - d.grad_offset)) return FR_E_RANGE;
  e->offset = table[d.entry].src_offset;
  e->grad_offset = d.grad_offset;
  fr_embed_info& i = e->info;
  i.rows = d.rows;
  i.cols = d.cols;
  i.max_tokens = d.max_tokens;
  i.arena_bytes = arena_bytes;
  i.grad_arena_bytes = grad_bytes;
  i.first = d.first;
  i.device = -1;
  i.dtype = table[d.entry].dtype;
  i.grad_dtype = d.grad_dtype;
  return FR_OK;
}

int build(fr_embed* e) {
  const uint64_t T = e->info.max_tokens;
  if (!T) return FR_OK;
  const auto up = [](uint64_t x) { return (x + 255) & ~uint64_t(255); };
  const uint64_t order = up(T * 4), places = up((e->info.rows + 1) * sizeof(Places));
  const uint64_t runs = up(embed_run_slots(T) * e->info.cols * 4);
  const uint64_t total = 2 * order + places + runs;
  const hipError_t rc = hipMalloc(&e->mem, total);
  if (rc != hipSuccess) {
    e->mem = nullptr;
    (void)hipGetLastError();
    return rc == hipErrorOutOfMemory ? FR_E_NOMEM : device_error(rc);
  }
  uint8_t* p = static_cast<uint8_t*>(e->mem);
  e->order = reinterpret_cast<uint32_t*>(p);
  e->row_of = reinterpret_cast<uint32_t*>(p + order);
  e->places = reinterpret_cast<Places*>(p + 2 * order);
  e->runs = reinterpret_cast<float*>(p + 2 * order + places);
  e->info.device_bytes = total;
  return FR_OK;
}

// The checks of what both calls take.
int check_tokens(const fr_embed* e, const void* ids, uint32_t id_bytes, uint64_t n, const void* act, uint32_t dtype,
                 uint64_t stride, float scale, uint64_t* id_size, uint64_t* act_size) {
  if ((id_bytes != 4 && id_bytes != 8) || (dtype != FR_F32 && dtype != FR_BF16)) return FR_E_INVAL;
  if (stride < e->info.cols || !(scale - scale == 0)) return FR_E_INVAL;
  if (n >= (uint64_t(1) << 30) || stride > (uint64_t(1) << 30) || !embed_lanes_fit(n, uint32_t(e->info.cols)))
    return FR_E_RANGE;
  *id_size = n * id_bytes;
  *act_size = n ? ((n - 1) * stride + e->info.cols) * size_of(dtype) : 0;
  FR_TRY(check_buffer(e->device, ids, *id_size, id_bytes));
  return check_buffer(e->device, act, *act_size, size_of(dtype));
}

EmbedArgs args_of(const fr_embed* e, const void* ids, uint32_t id_bytes, uint64_t n, uint32_t dtype, uint64_t stride,
                  float scale) {
  EmbedArgs a;
  a.first = uint64_t(e->info.first);
  a.rows = uint32_t(e->info.rows);
  a.cols = uint32_t(e->info.cols);
  a.ids = ids;
  a.id_bytes = id_bytes;
  a.n = n;
  a.scale = scale;
  a.act_f32 = dtype == FR_F32;
  a.stride = stride;
  return a;
}

}  // namespace

extern "C" int fr_embed_create(const fr_plan* plan, const fr_embed_desc* desc, uint64_t grad_arena_bytes,
                               fr_embed** out) {
  if (!plan || !desc || !out) return FR_E_INVAL;
  fr_embed* e = new (std::nothrow) fr_embed();
  if (!e) return FR_E_NOMEM;
  int rc = validate(plan->table.data(), uint32_t(plan->table.size()), plan->src_arena_bytes, *desc, grad_arena_bytes, e);
  if (rc == FR_OK) rc = check_device_and_stream(plan->device, nullptr);
  if (rc == FR_OK) {
    e->device = plan->device;
    e->info.device = plan->device;
    rc = build(e);
  }
  if (rc != FR_OK) {
    fr_embed_destroy(e);
    return rc;
  }
  *out = e;
  return FR_OK;
}

extern "C" int fr_embed_get_info(const fr_embed* e, fr_embed_info* out) {
  if (!e || !out) return FR_E_INVAL;
  *out = e->info;
  return FR_OK;
}

extern "C" int fr_embed_destroy(fr_embed* e) {
  if (!e) return FR_OK;
  int prev = -1;
  bool switched = false;
  if (e->device >= 0 && hipGetDevice(&prev) == hipSuccess && prev != e->device)
    switched = hipSetDevice(e->device) == hipSuccess;
  if (e->mem) (void)hipFree(e->mem);
  if (switched) (void)hipSetDevice(prev);
  delete e;
  return FR_OK;
}

extern "C" int fr_embed_query(const fr_tensor_desc* table, uint32_t n_entries, uint64_t arena_bytes,
                              const fr_embed_desc* desc, uint64_t grad_arena_bytes, fr_embed_info* info) {
  if (!desc || !info) return FR_E_INVAL;
  try {
    Layout L;
    FR_TRY(validate_and_layout(table, n_entries, 4096, kDefaultSegmentAlign, arena_bytes, uint64_t(1) << 62, &L));
    fr_embed e;
    FR_TRY(validate(table, n_entries, arena_bytes, *desc, grad_arena_bytes, &e));
    *info = e.info;
  } catch (const std::bad_alloc&) {
    return FR_E_NOMEM;
  }
  return FR_OK;
}

extern "C" int fr_embed_lookup(const fr_embed* e, const void* state, const void* ids, uint32_t id_bytes,
                               uint64_t n_tokens, float scale, void* out, uint32_t out_dtype, uint64_t out_stride,
                               hipStream_t stream) {
  if (!e) return FR_E_INVAL;
  uint64_t ib = 0, ob = 0;
  FR_TRY(check_device_and_stream(e->device, stream));
  FR_TRY(check_tokens(e, ids, id_bytes, n_tokens, out, out_dtype, out_stride, scale, &ib, &ob));
  FR_TRY(check_buffer(e->device, state, e->info.arena_bytes, 16));
  const Region outs[] = {{out, ob}}, ins[] = {{state, e->info.arena_bytes}, {ids, ib}};
  FR_TRY(check_disjoint(outs, 1, ins, 2));
  EmbedArgs a = args_of(e, ids, id_bytes, n_tokens, out_dtype, out_stride, scale);
  a.table = static_cast<const uint8_t*>(state) + e->offset;
  a.table_f32 = e->info.dtype == FR_F32;
  a.out = out;
  return launch_result(launch_embed_lookup(a, stream));
}

extern "C" int fr_embed_grad(const fr_embed* e, const void* ids, uint32_t id_bytes, uint64_t n_tokens,
                             const void* dout, uint32_t dout_dtype, uint64_t dout_stride, float scale, void* grads,
                             uint32_t add, hipStream_t stream) {
  if (!e || add > 1 || !e->info.max_tokens) return FR_E_INVAL;
  if (n_tokens > e->info.max_tokens) return FR_E_RANGE;
  uint64_t ib = 0, db = 0;
  FR_TRY(check_device_and_stream(e->device, stream));
  FR_TRY(check_tokens(e, ids, id_bytes, n_tokens, dout, dout_dtype, dout_stride, scale, &ib, &db));
  FR_TRY(check_buffer(e->device, grads, e->info.grad_arena_bytes, 16));
  const Region outs[] = {{grads, e->info.grad_arena_bytes}}, ins[] = {{ids, ib}, {dout, db}};
  FR_TRY(check_disjoint(outs, 1, ins, 2));
  EmbedArgs a = args_of(e, ids, id_bytes, n_tokens, dout_dtype, dout_stride, scale);
  a.dout = dout;
  a.grad = static_cast<uint8_t*>(grads) + e->grad_offset;
  a.grad_f32 = e->info.grad_dtype == FR_F32;
  a.add = add != 0;
  a.order = e->order;
  a.row_of = e->row_of;
  a.places = e->places;
  a.runs = e->runs;
  return launch_result(launch_embed_grad(a, stream));
}
