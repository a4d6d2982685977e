// extern "C" entry points of libppas.so (declared in include/ppas.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>
#include <mutex>
#include <new>
#include <utility>
#include <vector>

#include "adapters.h"
#include "device.h"
#include "list_pool.h"
#include "logprobs.h"
#include "plan.h"
#include "ppas.h"
#include "rope.h"

namespace ppas {

hipError_t launch_kv_append(uint16_t* kp, uint16_t* vp, const uint16_t* kn, const uint16_t* vn,
                            const AppendItem* items, int32_t n_items, const int32_t* bt, int32_t bt_stride,
                            int32_t hkv, hipStream_t stream, hipEvent_t ev_start, hipEvent_t ev_stop);
hipError_t launch_rope_append(uint16_t* q, uint16_t* kp, uint16_t* vp, const uint16_t* kn, const uint16_t* vn,
                              const AppendItem* items, int32_t n_items, const int32_t* bt, int32_t bt_stride,
                              int32_t hq, int32_t hkv, double theta, hipStream_t stream, hipEvent_t ev_start,
                              hipEvent_t ev_stop);

namespace {

std::mutex g_dev_mu;
std::vector<DeviceInfo> g_dev;

}  // namespace

// Compute-unit count and architecture of the current device (cached). Without a
// usable device, reports 256 CUs and not-gfx950.
DeviceInfo current_device() {
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    return DeviceInfo{};
  }
  std::lock_guard<std::mutex> lk(g_dev_mu);
  if (dev >= int(g_dev.size())) g_dev.resize(size_t(dev) + 1);
  DeviceInfo& d = g_dev[size_t(dev)];
  if (!d.known) {
    hipDeviceProp_t prop;
    if (hipGetDeviceProperties(&prop, dev) == hipSuccess) {
      d.gfx950 = std::strncmp(prop.gcnArchName, "gfx950", 6) == 0;
      d.cus = prop.multiProcessorCount > 0 ? prop.multiProcessorCount : 256;
    } else {
      (void)hipGetLastError();
    }
    d.known = true;
  }
  return d;
}

bool capturing(void* hip_stream) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(static_cast<hipStream_t>(hip_stream), &st) != hipSuccess) {
    (void)hipGetLastError();
    return false;
  }
  return st != hipStreamCaptureStatusNone;
}

namespace {

// Work-item counts and partial-slot offsets travel as int32 (and the item count
// sets the launch grid): a step too large for that is refused.
bool plan_fits(const Plan& plan, size_t n_append) {
  return plan.items.size() + plan.rows.size() <= size_t(INT32_MAX) && plan.combine.size() <= size_t(INT32_MAX) &&
         n_append <= size_t(INT32_MAX) && plan.part_slots <= int64_t(INT32_MAX) - 64 * kGroup;
}

ppas_status check_opts(const ppas_plan_opts* o) {
  if (!o) return PPAS_OK;
  if (o->prefill_split < 0 || o->decode_split < 0 || o->num_cus < 0) return PPAS_EINVAL;
  if (o->tile_positions != 0 && o->tile_positions != kTilePosSmall && o->tile_positions != kTilePosLarge)
    return PPAS_EINVAL;
  return PPAS_OK;
}

PlanOpts to_opts(const ppas_plan_opts* o) {
  PlanOpts p;
  if (o) {
    p.prefill_split = o->prefill_split;
    p.decode_split = o->decode_split;
    p.tile_pos = o->tile_positions;
  }
  return p;
}

ppas_status check_events(const ppas_events* ev) {
  if (!ev) return PPAS_OK;
  if ((ev->start == nullptr) != (ev->stop == nullptr)) return PPAS_EINVAL;
  if ((ev->merge_start == nullptr) != (ev->merge_stop == nullptr)) return PPAS_EINVAL;
  return PPAS_OK;
}

hipEvent_t ev_of(const ppas_events* ev, int which) {
  if (!ev) return nullptr;
  void* const e[4] = {ev->start, ev->stop, ev->merge_start, ev->merge_stop};
  return static_cast<hipEvent_t>(e[which]);
}

// ---------------------------------------------------------------------------
// Pinned host buffers holding work lists. The kernels read their items straight
// from this memory: each workgroup reads its 32-byte item once, which costs less
// than a host-to-device copy on a separate engine and the two cross-engine
// waits around it. A buffer in use belongs to one plan; once released it is
// handed out again only after every launch that read it has completed (an event
// is recorded behind those launches, one per stream).
// ---------------------------------------------------------------------------
struct Pinned : ListBuffer<hipStream_t, hipEvent_t> {
  void* host = nullptr;
  char* dev = nullptr;      // the same memory as the device addresses it
};

constexpr size_t kPoolMax = 64;   // buffers kept; beyond that a call reuses a released one
std::mutex g_pool_mu;
std::vector<Pinned*> g_pool;

bool completed(hipEvent_t ev) {
  const hipError_t e = hipEventQuery(ev);
  if (e == hipErrorNotReady) return false;
  if (e != hipSuccess) (void)hipGetLastError();
  return true;
}

void drop_events(Pinned& b) {
  for (auto& u : b.uses) (void)hipEventDestroy(u.event);
  b.uses.clear();
}

ppas_status grow(Pinned& b, size_t bytes) {
  if (b.cap >= bytes) return PPAS_OK;
  if (b.host) (void)hipHostFree(b.host);
  b.host = nullptr;
  b.dev = nullptr;
  b.cap = 0;
  size_t cap = size_t(1) << 16;
  while (cap < bytes) cap <<= 1;
  if (hipHostMalloc(&b.host, cap, hipHostMallocDefault) != hipSuccess) {
    b.host = nullptr;
    return PPAS_EHIP;
  }
  void* d = nullptr;
  if (hipHostGetDevicePointer(&d, b.host, 0) != hipSuccess) {
    (void)hipHostFree(b.host);
    b.host = nullptr;
    return PPAS_EHIP;
  }
  b.dev = static_cast<char*>(d);
  b.cap = cap;
  return PPAS_OK;
}

// A buffer of at least `bytes`, marked in use.
ppas_status acquire(size_t bytes, Pinned*& out) {
  std::lock_guard<std::mutex> lk(g_pool_mu);
  Pinned* pick = idle_buffer(g_pool, bytes, completed);
  if (!pick && g_pool.size() < kPoolMax) {
    pick = new (std::nothrow) Pinned;
    if (!pick) return PPAS_EHIP;
    g_pool.push_back(pick);
  }
  if (!pick) pick = any_idle_buffer(g_pool, bytes, completed);   // the pool is full: a small one is grown
  if (!pick) {  // else wait for a released buffer whose launches are still running
    pick = oldest_buffer(g_pool);
    if (pick) {
      for (auto& u : pick->uses) {
        if (u.pending && hipEventSynchronize(u.event) != hipSuccess) return PPAS_EHIP;
        u.pending = false;
      }
    }
  }
  if (!pick) {  // every buffer belongs to a live plan: the pool grows past its cap
    pick = new (std::nothrow) Pinned;
    if (!pick) return PPAS_EHIP;
    g_pool.push_back(pick);
  }
  if (pick->uses.size() > 8) drop_events(*pick);
  const ppas_status st = grow(*pick, bytes);
  if (st != PPAS_OK) return st;
  pick->in_use = true;
  out = pick;
  return PPAS_OK;
}

// Records, behind the work just enqueued on `stream`, that the buffer was read.
// Without the event the stream is drained, so the buffer is never reused early.
bool note_use(Pinned* b, hipStream_t stream) {
  std::lock_guard<std::mutex> lk(g_pool_mu);
  auto use = std::find_if(b->uses.begin(), b->uses.end(), [&](const auto& u) { return u.stream == stream; });
  if (use == b->uses.end()) {
    hipEvent_t ev = nullptr;
    if (hipEventCreateWithFlags(&ev, hipEventDisableTiming) != hipSuccess) {
      (void)hipStreamSynchronize(stream);
      return false;
    }
    use = b->uses.insert(b->uses.end(), {stream, ev, false});
  }
  if (hipEventRecord(use->event, stream) != hipSuccess) {
    (void)hipStreamSynchronize(stream);
    return false;
  }
  use->pending = true;
  return true;
}

void release(Pinned* b) {
  if (!b) return;
  std::lock_guard<std::mutex> lk(g_pool_mu);
  b->in_use = false;
  const auto at = std::find(g_pool.begin(), g_pool.end(), b);
  if (at != g_pool.end()) std::rotate(at, at + 1, g_pool.end());   // the latest release is last
}

}  // namespace
}  // namespace ppas

using namespace ppas;

// The plan of one step: validated descriptors, the attention work list and the
// page-write list, staged in one pinned buffer.
struct ppas_step_plan {
  ppas_shape shape{};
  int32_t bt_stride = 0;
  int32_t n_seqs = 0;
  int64_t n_rows = 0;
  Plan plan;
  int32_t n_append = 0;
  size_t off_append = 0;
  int32_t n_desc = 0;            // the page-write list by request, where the step has few
  AppendDesc desc[kAppendInline];
  Pinned* buf = nullptr;
};

namespace {

// kWantInline: the page-write list, but only by request where that is enough
enum : int { kWantAttn = 1, kWantAppend = 2, kWantInline = 4 };

// Validate, plan and stage. On success p.buf holds the lists (nullptr for an empty step,
// and where a page-write list by request is all that is wanted).
ppas_status build_plan(ppas_step_plan& p, const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                       const int32_t* bt_host, int32_t bt_stride, const ppas_plan_opts* opts, int want,
                       bool check_overlap, const ppas_prefix* prefixes = nullptr, int32_t n_prefixes = 0) {
  ppas_status st = check_opts(opts);
  if (st != PPAS_OK) return st;
  st = validate(shape, seqs, n_seqs, bt_host, bt_stride, check_overlap);
  if (st != PPAS_OK) return st;
  st = validate_prefixes(seqs, n_seqs, bt_host, bt_stride, prefixes, n_prefixes);
  if (st != PPAS_OK) return st;
  p.shape = *shape;
  p.bt_stride = bt_stride;
  p.n_seqs = n_seqs;
  if (n_seqs == 0) return PPAS_OK;
  p.n_rows = int64_t(seqs[n_seqs - 1].query_start) + seqs[n_seqs - 1].n_query;
  const DeviceInfo dev = current_device();
  if (!dev.gfx950) return PPAS_EUNSUPPORTED;
  std::vector<AppendItem> app;
  if (want & kWantAttn)
    make_plan(*shape, seqs, n_seqs, (opts && opts->num_cus > 0) ? opts->num_cus : dev.cus, to_opts(opts), p.plan,
              prefixes, n_prefixes);
  const bool by_request = (want & (kWantAppend | kWantInline)) && n_seqs <= kAppendInline;
  if (by_request) {
    int32_t item = 0;   // at most a page per token row
    for (int32_t s = 0; s < n_seqs; ++s) {
      const ppas_seq& q = seqs[s];
      p.desc[s] = AppendDesc{item, q.query_start, q.n_query, q.cached_len};
      item += (q.cached_len + q.n_query - 1) / kPage - q.cached_len / kPage + 1;
    }
    p.n_desc = n_seqs;
    p.n_append = item;
    if (want == kWantInline) return PPAS_OK;
  }
  if (want & (kWantAppend | kWantInline)) make_append_items(seqs, n_seqs, app);
  if (!plan_fits(p.plan, app.size())) return PPAS_ERANGE;
  p.n_append = int32_t(app.size());
  const size_t list = (want & kWantAttn) ? p.plan.list_bytes : 0;
  p.off_append = (list + 255) / 256 * 256;
  const size_t bytes = p.off_append + app.size() * sizeof(AppendItem);
  st = acquire(std::max<size_t>(bytes, 256), p.buf);
  if (st != PPAS_OK) return st;
  char* host = static_cast<char*>(p.buf->host);
  if (!p.plan.items.empty()) std::memcpy(host, p.plan.items.data(), p.plan.items.size() * sizeof(WorkItem));
  if (!p.plan.rows.empty())
    std::memcpy(host + p.plan.off_rows, p.plan.rows.data(), p.plan.rows.size() * sizeof(WorkItem));
  if (!p.plan.combine.empty())
    std::memcpy(host + p.plan.off_combine, p.plan.combine.data(), p.plan.combine.size() * sizeof(CombineItem));
  if (!app.empty()) std::memcpy(host + p.off_append, app.data(), app.size() * sizeof(AppendItem));
  return PPAS_OK;
}

// Lists in host memory are staged per call or plan and reused once its launches have
// ended, which a graph's replays would read again: every call that reads one refuses a
// capturing stream, and does so before it asks the pool for a buffer (an allocation would
// end the capture). The appends refuse it also where few requests' list is in the arguments.
ppas_status run_append(const ppas_step_plan& p, bool rope, float theta, void* q, void* k_pages, void* v_pages,
                       const void* k_new, const void* v_new, const int32_t* bt_dev, const ppas_events* ev,
                       void* hip_stream) {
  if (p.n_seqs == 0) return PPAS_OK;
  if (!k_pages || !v_pages || !k_new || !v_new || !bt_dev || (rope && !q)) return PPAS_EINVAL;
  if (!p.buf || p.n_append == 0) return PPAS_EINVAL;   // a plan made without the page-write list
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  const AppendItem* items = reinterpret_cast<const AppendItem*>(p.buf->dev + p.off_append);
  hipError_t e;
  if (rope)
    e = launch_rope_append(static_cast<uint16_t*>(q), static_cast<uint16_t*>(k_pages), static_cast<uint16_t*>(v_pages),
                           static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), items, p.n_append,
                           bt_dev, p.bt_stride, p.shape.n_q_heads, p.shape.n_kv_heads, double(theta), stream,
                           ev_of(ev, 0), ev_of(ev, 1));
  else
    e = launch_kv_append(static_cast<uint16_t*>(k_pages), static_cast<uint16_t*>(v_pages),
                         static_cast<const uint16_t*>(k_new), static_cast<const uint16_t*>(v_new), items, p.n_append,
                         bt_dev, p.bt_stride, p.shape.n_kv_heads, stream, ev_of(ev, 0), ev_of(ev, 1));
  // the buffer is free again once the kernel that reads it has finished (also
  // after a failed launch: a kernel that did start may still read it)
  const bool noted = note_use(p.buf, stream);
  return (e == hipSuccess && noted) ? PPAS_OK : PPAS_EHIP;
}

// Bytes that T rows of `row` elements, `stride` apart, span.
uint64_t span_bytes(int64_t T, int64_t stride, int64_t row) { return 2 * (uint64_t(T - 1) * uint64_t(stride) + uint64_t(row)); }

bool overlap(const void* a, uint64_t a_bytes, const void* b, uint64_t b_bytes) {
  const uint64_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y ? y - x < a_bytes : x - y < b_bytes;
}

// Memory that a call reads or writes; of a pointer that is NULL, none.
struct Span {
  const void* at;
  uint64_t bytes;
};
bool over_any(const Span& s, std::initializer_list<Span> others) {
  if (!s.at || s.bytes == 0) return false;
  for (const Span& o : others)
    if (o.at && o.bytes > 0 && overlap(s.at, s.bytes, o.at, o.bytes)) return true;
  return false;
}

bool off(const void* p, uintptr_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// T: the step's token rows.
ppas_status check_qkv(const ppas_shape& s, const ppas_rope* rope, const ppas_qkv* r, const void* q_out,
                      const void* k_pages, const void* v_pages, const int32_t* bt_dev, int64_t T, RopeTable& table) {
  const ppas_status st = rope_table(rope, s.head_dim, table);
  if (st != PPAS_OK) return st;
  if (!r || !r->q || !r->k || !r->v || !q_out || !k_pages || !v_pages || !bt_dev) return PPAS_EINVAL;
  const int64_t q_row = int64_t(s.n_q_heads) * s.head_dim, kv_row = int64_t(s.n_kv_heads) * s.head_dim;
  if (r->q_stride < q_row || r->k_stride < kv_row || r->v_stride < kv_row) return PPAS_EINVAL;
  // a step's last row has to lie within 2^62 bytes, far past any device's memory
  const int64_t most = (int64_t(1) << 61) / T;
  if (r->q_stride > most || r->k_stride > most || r->v_stride > most) return PPAS_ERANGE;
  if (off(r->q, 2) || off(r->k, 2) || off(r->v, 2) || off(q_out, 2) || off(k_pages, 16) || off(v_pages, 16) ||
      off(bt_dev, 4))
    return PPAS_EINVAL;
  const uint64_t out_bytes = span_bytes(T, q_row, q_row);
  const bool in_place = q_out == r->q && r->q_stride == q_row;
  if ((!in_place && overlap(q_out, out_bytes, r->q, span_bytes(T, r->q_stride, q_row))) ||
      overlap(q_out, out_bytes, r->k, span_bytes(T, r->k_stride, kv_row)) ||
      overlap(q_out, out_bytes, r->v, span_bytes(T, r->v_stride, kv_row)))
    return PPAS_EINVAL;
  return PPAS_OK;
}

// The norms of a call's heads, where it has any.
struct Norms {
  const ppas_head_norm *q, *k;
};

ppas_status check_norm(const ppas_head_norm* n, int64_t heads, int32_t head_dim) {
  if (!n || !std::isfinite(n->eps) || !(n->eps >= 0x1p-100f) || !std::isfinite(n->offset)) return PPAS_EINVAL;
  if (!n->weight) return PPAS_OK;
  if (off(n->weight, 2) || (n->head_stride != 0 && n->head_stride < head_dim)) return PPAS_EINVAL;
  return n->head_stride > (int64_t(1) << 61) / heads ? PPAS_ERANGE : PPAS_OK;
}

Span weights_of(const ppas_head_norm& n, int64_t heads, int32_t head_dim) {
  return {n.weight, span_bytes(heads, n.head_stride, head_dim)};
}

HeadNorm norm_of(const ppas_head_norm& n) {
  return HeadNorm{static_cast<const uint16_t*>(n.weight), n.head_stride, n.eps, n.offset, n.center != 0};
}

ppas_status run_qkv_append(const ppas_step_plan& p, const RopeTable& table, const Norms* norms, const ppas_qkv& rows,
                           void* q_out, void* k_pages, void* v_pages, const int32_t* bt_dev, const ppas_events* ev,
                           void* hip_stream) {
  if (p.n_append == 0 || (p.n_desc == 0 && !p.buf)) return PPAS_EINVAL;   // a plan made without the page-write list
  if (p.n_append > kAppendMaxItems) return PPAS_ERANGE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  RopeAppend r;
  r.q = static_cast<const uint16_t*>(rows.q);
  r.k = static_cast<const uint16_t*>(rows.k);
  r.v = static_cast<const uint16_t*>(rows.v);
  r.q_stride = rows.q_stride;
  r.k_stride = rows.k_stride;
  r.v_stride = rows.v_stride;
  r.q_out = static_cast<uint16_t*>(q_out);
  r.k_pages = static_cast<uint16_t*>(k_pages);
  r.v_pages = static_cast<uint16_t*>(v_pages);
  if (p.n_desc == 0) r.items = reinterpret_cast<const AppendItem*>(p.buf->dev + p.off_append);
  r.bt = bt_dev;
  r.desc = p.desc;
  r.n_desc = p.n_desc;
  r.n_items = p.n_append;
  r.bt_stride = p.bt_stride;
  r.hq = p.shape.n_q_heads;
  r.hkv = p.shape.n_kv_heads;
  const hipError_t e =
      norms ? launch_norm_rope_qkv_append(r, norm_of(*norms->q), norm_of(*norms->k), table, stream, ev_of(ev, 0),
                                          ev_of(ev, 1))
            : launch_rope_qkv_append(r, table, stream, ev_of(ev, 0), ev_of(ev, 1));
  // a list by request travels in the kernel's arguments: no buffer is read
  const bool noted = p.n_desc > 0 || note_use(p.buf, stream);
  return (e == hipSuccess && noted) ? PPAS_OK : PPAS_EHIP;
}

ppas_status run_attn(const ppas_step_plan& p, void* out, const void* q, const void* k_pages, const void* v_pages,
                     const int32_t* bt_dev, void* workspace, size_t workspace_bytes, const ppas_events* ev,
                     void* hip_stream) {
  if (p.n_seqs == 0) return PPAS_OK;
  if (!out || !q || !k_pages || !v_pages || !bt_dev || !workspace) return PPAS_EINVAL;
  if (!p.buf || (p.plan.items.empty() && p.plan.rows.empty())) return PPAS_EINVAL;   // a plan made without the attention list
  if (workspace_bytes < p.plan.total) return PPAS_ENOSPACE;
  hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const Plan& plan = p.plan;
  const hipError_t e = launch_attn_step(
      static_cast<const uint16_t*>(q), static_cast<uint16_t*>(out), static_cast<const uint16_t*>(k_pages),
      static_cast<const uint16_t*>(v_pages), bt_dev, p.bt_stride, p.shape.n_q_heads, p.shape.n_kv_heads,
      p.shape.scale, reinterpret_cast<const WorkItem*>(p.buf->dev), int(plan.items.size()),
      reinterpret_cast<const WorkItem*>(p.buf->dev + plan.off_rows), int(plan.rows.size()),
      reinterpret_cast<const CombineItem*>(p.buf->dev + plan.off_combine), int(plan.combine.size()),
      plan.combine_pos, reinterpret_cast<float2*>(ws + plan.off_ml), reinterpret_cast<float*>(ws + plan.off_acc), plan.tile_pos,
      stream, ev_of(ev, 0), ev_of(ev, 1), ev_of(ev, 2), ev_of(ev, 3));
  const bool noted = note_use(p.buf, stream);
  return (e == hipSuccess && noted) ? PPAS_OK : PPAS_EHIP;
}

}  // namespace

extern "C" {

const char* ppas_status_string(ppas_status status) {
  switch (status) {
    case PPAS_OK: return "PPAS_OK";
    case PPAS_EINVAL: return "PPAS_EINVAL: invalid argument or step description";
    case PPAS_ERANGE: return "PPAS_ERANGE: block-table entry, length or step size out of range";
    case PPAS_ENOSPACE: return "PPAS_ENOSPACE: workspace too small";
    case PPAS_EHIP: return "PPAS_EHIP: HIP runtime error";
    case PPAS_EUNSUPPORTED: return "PPAS_EUNSUPPORTED: shape or device outside the compiled set";
  }
  return "PPAS: unknown status";
}

ppas_status ppas_validate_step(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                               const int32_t* block_table_host, int32_t bt_stride) {
  try {
    return validate(shape, seqs, n_seqs, block_table_host, bt_stride, true);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

int32_t ppas_plan_items(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs, const ppas_plan_opts* opts,
                        int32_t* items_out, int32_t capacity) {
  return ppas_plan_shared_items(shape, seqs, n_seqs, nullptr, 0, opts, items_out, capacity);
}

int32_t ppas_plan_shared_items(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                               const ppas_prefix* prefixes, int32_t n_prefixes, const ppas_plan_opts* opts,
                               int32_t* items_out, int32_t capacity) {
  try {
    ppas_status st = check_opts(opts);
    if (st != PPAS_OK) return st;
    st = validate(shape, seqs, n_seqs, nullptr, INT32_MAX, false);
    if (st != PPAS_OK) return st;
    st = validate_prefixes(seqs, n_seqs, nullptr, INT32_MAX, prefixes, n_prefixes);
    if (st != PPAS_OK) return st;
    Plan plan;
    make_plan(*shape, seqs, n_seqs, (opts && opts->num_cus > 0) ? opts->num_cus : 256, to_opts(opts), plan, prefixes,
              n_prefixes);
    if (!plan_fits(plan, 0)) return PPAS_ERANGE;
    const size_t n = plan.items.size() + plan.rows.size();
    for (size_t i = 0; items_out && i < n && int64_t(i) < capacity; ++i) {
      const bool row = i >= plan.items.size();
      const WorkItem& w = row ? plan.rows[i - plan.items.size()] : plan.items[i];
      const int32_t v[8] = {row ? 2 : w.npos_kind >> 16, w.seq,  w.kvh, w.row0, w.pos0, w.npos_kind & 0xffff,
                            w.key_lo,                    w.key_hi};
      std::copy(v, v + 8, items_out + 8 * i);
    }
    return int32_t(n);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

size_t ppas_attn_workspace_bytes(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs) {
  try {
    if (validate(shape, seqs, n_seqs, nullptr, INT32_MAX, false) != PPAS_OK) return 0;
    Plan plan;
    make_plan(*shape, seqs, n_seqs, current_device().cus, PlanOpts{}, plan);
    return plan_fits(plan, 0) ? plan.total : 0;
  } catch (...) {
    return 0;
  }
}

ppas_status ppas_step_plan_create(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                  const int32_t* block_table_host, int32_t bt_stride, const ppas_plan_opts* opts,
                                  ppas_step_plan** plan) {
  return ppas_step_plan_create_shared(shape, seqs, n_seqs, nullptr, 0, block_table_host, bt_stride, opts, plan);
}

ppas_status ppas_step_plan_create_shared(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                         const ppas_prefix* prefixes, int32_t n_prefixes,
                                         const int32_t* block_table_host, int32_t bt_stride,
                                         const ppas_plan_opts* opts, ppas_step_plan** plan) {
  if (!plan) return PPAS_EINVAL;
  *plan = nullptr;
  ppas_step_plan* p = nullptr;
  try {
    p = new ppas_step_plan;
    const ppas_status st =
        build_plan(*p, shape, seqs, n_seqs, block_table_host, bt_stride, opts, kWantAttn | kWantAppend, true, prefixes,
                   n_prefixes);
    if (st != PPAS_OK) {
      release(p->buf);
      delete p;
      return st;
    }
    *plan = p;
    return PPAS_OK;
  } catch (...) {
    if (p) {
      release(p->buf);
      delete p;
    }
    return PPAS_EINVAL;
  }
}

ppas_status ppas_step_plan_info(const ppas_step_plan* plan, ppas_plan_info* info) {
  if (!plan || !info) return PPAS_EINVAL;
  const size_t waves = plan->plan.tile_pos == kTilePosLarge ? 8 : 4;
  info->n_items = int32_t(plan->plan.items.size() + (plan->plan.rows.size() + waves - 1) / waves);
  info->n_merge = int32_t(plan->plan.combine.size());
  info->tile_positions = plan->plan.tile_pos;
  info->n_append = plan->n_append;
  info->workspace_bytes = plan->n_seqs ? uint64_t(plan->plan.total) : 256;
  return PPAS_OK;
}

void ppas_step_plan_destroy(ppas_step_plan* plan) {
  if (!plan) return;
  release(plan->buf);
  delete plan;
}

ppas_status ppas_kv_append_planned(const ppas_step_plan* plan, void* k_pages, void* v_pages, const void* k_new,
                                   const void* v_new, const int32_t* block_table_dev, const ppas_events* events,
                                   void* hip_stream) {
  if (!plan) return PPAS_EINVAL;
  const ppas_status st = check_events(events);
  if (st != PPAS_OK) return st;
  try {
    if (plan->n_seqs > 0 && capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    return run_append(*plan, false, 0.f, nullptr, k_pages, v_pages, k_new, v_new, block_table_dev, events,
                      hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_rope_kv_append_planned(const ppas_step_plan* plan, float rope_theta, void* q, void* k_pages,
                                        void* v_pages, const void* k_new, const void* v_new,
                                        const int32_t* block_table_dev, const ppas_events* events,
                                        void* hip_stream) {
  if (!plan) return PPAS_EINVAL;
  if (!std::isfinite(rope_theta) || !(rope_theta > 0.f)) return PPAS_EINVAL;
  const ppas_status st = check_events(events);
  if (st != PPAS_OK) return st;
  try {
    if (plan->n_seqs > 0 && capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    return run_append(*plan, true, rope_theta, q, k_pages, v_pages, k_new, v_new, block_table_dev, events,
                      hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

namespace {

ppas_status check_norms(const Norms* norms, const ppas_shape& s) {
  if (!norms) return PPAS_OK;
  const ppas_status st = check_norm(norms->q, s.n_q_heads, kHeadDim);
  return st != PPAS_OK ? st : check_norm(norms->k, s.n_kv_heads, kHeadDim);
}

// A step's outputs over the weights of its norms.
bool over_weights(const Norms* norms, const ppas_shape& s, const void* q_out, const void* k_pages, const void* v_pages,
                  int64_t T) {
  if (!norms) return false;
  const uint64_t pool = 2 * uint64_t(s.num_pages) * uint64_t(s.n_kv_heads) * uint64_t(s.page_size) * uint64_t(s.head_dim);
  const uint64_t q_row = uint64_t(s.n_q_heads) * uint64_t(s.head_dim);
  const Span q{q_out, 2 * uint64_t(T) * q_row}, k{k_pages, pool}, v{v_pages, pool};
  return over_any(weights_of(*norms->q, s.n_q_heads, s.head_dim), {q, k, v}) ||
         over_any(weights_of(*norms->k, s.n_kv_heads, s.head_dim), {q, k, v});
}

ppas_status qkv_append_planned(const ppas_step_plan* plan, const Norms* norms, const ppas_rope* rope,
                               const ppas_qkv* rows, void* q_out, void* k_pages, void* v_pages,
                               const int32_t* block_table_dev, const ppas_events* events, void* hip_stream) {
  if (!plan) return PPAS_EINVAL;
  ppas_status st = check_events(events);
  if (st != PPAS_OK) return st;
  try {
    st = check_norms(norms, plan->shape);
    if (st != PPAS_OK) return st;
    RopeTable table;
    if (plan->n_seqs == 0) return rope_table(rope, kHeadDim, table);
    st = check_qkv(plan->shape, rope, rows, q_out, k_pages, v_pages, block_table_dev, plan->n_rows, table);
    if (st != PPAS_OK) return st;
    if (over_weights(norms, plan->shape, q_out, k_pages, v_pages, plan->n_rows)) return PPAS_EINVAL;
    if (capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    return run_qkv_append(*plan, table, norms, *rows, q_out, k_pages, v_pages, block_table_dev, events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

}  // namespace

ppas_status ppas_rope_qkv_append_planned(const ppas_step_plan* plan, const ppas_rope* rope, const ppas_qkv* rows,
                                         void* q_out, void* k_pages, void* v_pages, const int32_t* block_table_dev,
                                         const ppas_events* events, void* hip_stream) {
  return qkv_append_planned(plan, nullptr, rope, rows, q_out, k_pages, v_pages, block_table_dev, events, hip_stream);
}

ppas_status ppas_norm_rope_qkv_append_planned(const ppas_step_plan* plan, const ppas_head_norm* q_norm,
                                              const ppas_head_norm* k_norm, const ppas_rope* rope,
                                              const ppas_qkv* rows, void* q_out, void* k_pages, void* v_pages,
                                              const int32_t* block_table_dev, const ppas_events* events,
                                              void* hip_stream) {
  const Norms norms{q_norm, k_norm};
  return qkv_append_planned(plan, &norms, rope, rows, q_out, k_pages, v_pages, block_table_dev, events, hip_stream);
}

ppas_status ppas_attn_step_planned(const ppas_step_plan* plan, void* out, const void* q, const void* k_pages,
                                   const void* v_pages, const int32_t* block_table_dev, void* workspace,
                                   size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  if (!plan) return PPAS_EINVAL;
  const ppas_status st = check_events(events);
  if (st != PPAS_OK) return st;
  try {
    if (plan->n_seqs > 0 && capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    return run_attn(*plan, out, q, k_pages, v_pages, block_table_dev, workspace, workspace_bytes, events,
                    hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

namespace {

ppas_status check_gateup(int32_t n_tokens, int32_t hidden, int32_t n_out) {
  if (n_tokens < 0 || hidden <= 0 || n_out <= 0) return PPAS_EINVAL;
  if (hidden % 64 != 0) return PPAS_EUNSUPPORTED;
  // tile origins and edges stay inside int32, and the grid inside its limit
  if (n_tokens > INT32_MAX - 512 || n_out > INT32_MAX - 512) return PPAS_ERANGE;
  if (gateup_tiles(n_tokens, n_out) > INT32_MAX) return PPAS_ERANGE;
  return PPAS_OK;
}

}  // namespace

size_t ppas_gateup_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_out) {
  try {
    if (check_gateup(n_tokens, hidden, n_out) != PPAS_OK || n_tokens == 0) return 0;
    return gateup_workspace_bytes(n_tokens, n_out, gateup_splits(n_tokens, hidden, n_out, current_device().cus));
  } catch (...) {
    return 0;
  }
}

namespace {

// The most splits of a call: the automatic number, reduced to what the workspace
// holds (no split needs none).
int allowed_splits(int32_t n_tokens, int32_t hidden, int32_t n_out, size_t workspace_bytes, int cus) {
  int splits = gateup_splits(n_tokens, hidden, n_out, cus);
  while (splits > 1 && gateup_workspace_bytes(n_tokens, n_out, splits) > workspace_bytes) --splits;
  return gateup_tiles(n_tokens, n_out) * splits > INT32_MAX ? 1 : splits;
}

// Both projection entry points: n_out weight rows; with `act` the output holds the
// gated activation of the two halves (n_out / 2 columns).
ppas_status gateup_call(const void* x, const void* w, void* y, int32_t n_tokens, int32_t hidden, int32_t n_out,
                        bool act, void* workspace, size_t workspace_bytes, const ppas_events* events,
                        void* hip_stream) {
  ppas_status st = check_gateup(n_tokens, hidden, n_out);
  if (st != PPAS_OK) return st;
  st = check_events(events);
  if (st != PPAS_OK) return st;
  if (n_tokens == 0) return PPAS_OK;
  if (!x || !w || !y || (workspace_bytes > 0 && !workspace)) return PPAS_EINVAL;
  const DeviceInfo dev = current_device();
  if (!dev.gfx950) return PPAS_EUNSUPPORTED;
  const int splits = allowed_splits(n_tokens, hidden, n_out, workspace_bytes, dev.cus);
  const hipError_t e = launch_gateup(static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w),
                                     static_cast<uint16_t*>(y), n_tokens, hidden, n_out, act, splits,
                                     static_cast<float*>(workspace), dev.cus, static_cast<hipStream_t>(hip_stream),
                                     ev_of(events, 0), ev_of(events, 1));
  return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
}

// weight rows of the activated projection (two per intermediate feature), or -1
int32_t act_rows(int32_t n_inter) { return (n_inter <= 0 || n_inter > (INT32_MAX - 512) / 2) ? -1 : 2 * n_inter; }

}  // namespace

ppas_status ppas_gateup_proj(const void* x, const void* w, void* y, int32_t n_tokens, int32_t hidden, int32_t n_out,
                             void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    return gateup_call(x, w, y, n_tokens, hidden, n_out, false, workspace, workspace_bytes, events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

size_t ppas_gateup_act_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_inter) {
  const int32_t n_out = act_rows(n_inter);
  return n_out < 0 ? 0 : ppas_gateup_workspace_bytes(n_tokens, hidden, n_out);
}

ppas_status ppas_gateup_act(const void* x, const void* w, void* y, int32_t n_tokens, int32_t hidden, int32_t n_inter,
                            void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    if (n_inter > (INT32_MAX - 512) / 2) return PPAS_ERANGE;
    const int32_t n_out = act_rows(n_inter);
    if (n_out < 0) return PPAS_EINVAL;
    return gateup_call(x, w, y, n_tokens, hidden, n_out, true, workspace, workspace_bytes, events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_gateup_choice(int32_t n_tokens, int32_t hidden, int32_t n_out, int32_t activation, int32_t aligned,
                               size_t workspace_bytes, int32_t num_cus, int32_t* choice) {
  const ppas_status st = check_gateup(n_tokens, hidden, n_out);
  if (st != PPAS_OK) return st;
  if (!choice || n_tokens == 0 || num_cus < 0 || (activation && n_out % 2 != 0)) return PPAS_EINVAL;
  const int cus = num_cus > 0 ? num_cus : 256;
  const GateupChoice c = gateup_choose(n_tokens, hidden, n_out, activation != 0, aligned != 0,
                                       allowed_splits(n_tokens, hidden, n_out, workspace_bytes, cus), cus);
  const int32_t v[8] = {c.kernel, c.rows, c.main_m, c.tail_m, c.g, c.wr, c.splits, c.block};
  std::copy(v, v + 8, choice);
  return PPAS_OK;
}

namespace {

// 8-bit rows: sums of up to 131,071 products of at most 128 x 128 fit int32.
constexpr int32_t kMaxHiddenI8 = 131071;

ppas_status check_gateup_i8(int32_t n_tokens, int32_t hidden, int32_t n_out, bool act) {
  if (n_tokens < 0 || hidden <= 0 || n_out <= 0) return PPAS_EINVAL;
  if (hidden > kMaxHiddenI8 || n_tokens > INT32_MAX - 512 || n_out > INT32_MAX - 512) return PPAS_ERANGE;
  if (gateup_tiles(n_tokens, n_out) > INT32_MAX || gateup_i8_any_tiles(n_tokens, n_out, act) > INT32_MAX)
    return PPAS_ERANGE;
  return PPAS_OK;
}

// The most splits of a call in whole 128-feature stages (1: the general kernel takes it).
int splits_i8(int32_t n_tokens, int32_t hidden, int32_t n_out, int cus) {
  return hidden % 128 ? 1 : gateup_splits(n_tokens, hidden / 2, n_out, cus);
}

// The most splits that the workspace holds.
int allowed_splits_i8(int32_t n_tokens, int32_t hidden, int32_t n_out, size_t workspace_bytes, int cus) {
  int splits = splits_i8(n_tokens, hidden, n_out, cus);
  while (splits > 1 && gateup_workspace_bytes(n_tokens, n_out, splits) > workspace_bytes) --splits;
  return gateup_tiles(n_tokens, n_out) * splits > INT32_MAX ? 1 : splits;
}

ppas_status gateup_i8_call(const void* x, const float* sx, const void* w, const float* sw, void* y, int32_t n_tokens,
                           int32_t hidden, int32_t n_out, bool act, void* workspace, size_t workspace_bytes,
                           const ppas_events* events, void* hip_stream) {
  ppas_status st = check_gateup_i8(n_tokens, hidden, n_out, act);
  if (st != PPAS_OK) return st;
  st = check_events(events);
  if (st != PPAS_OK) return st;
  if (n_tokens == 0) return PPAS_OK;
  if (!x || !sx || !w || !sw || !y || (workspace_bytes > 0 && !workspace)) return PPAS_EINVAL;
  if (off(sx, 4) || off(sw, 4) || off(y, 2) || off(workspace, 16)) return PPAS_EINVAL;
  const DeviceInfo dev = current_device();
  if (!dev.gfx950) return PPAS_EUNSUPPORTED;
  const int splits = allowed_splits_i8(n_tokens, hidden, n_out, workspace_bytes, dev.cus);
  const Int8Product p{static_cast<const int8_t*>(x), sx, static_cast<const int8_t*>(w), sw,
                      static_cast<uint16_t*>(y), n_tokens, hidden, n_out};
  const hipError_t e = launch_gateup_i8(p, act, splits, workspace, dev.cus, static_cast<hipStream_t>(hip_stream),
                                        ev_of(events, 0), ev_of(events, 1));
  return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
}

}  // namespace

ppas_status ppas_quant_i8(const void* x, int64_t x_stride, void* xq, float* scale, int32_t n_rows, int32_t hidden,
                          const ppas_events* events, void* hip_stream) {
  try {
    if (n_rows < 0 || hidden <= 0) return PPAS_EINVAL;
    const ppas_status st = check_events(events);
    if (st != PPAS_OK) return st;
    if (n_rows == 0) return PPAS_OK;
    if (!x || !xq || !scale || x_stride < hidden || off(x, 2) || off(scale, 4)) return PPAS_EINVAL;
    if (x_stride > (int64_t(1) << 61) / n_rows) return PPAS_ERANGE;
    if (!current_device().gfx950) return PPAS_EUNSUPPORTED;
    const hipError_t e = launch_quant_i8(static_cast<const uint16_t*>(x), x_stride, static_cast<int8_t*>(xq), scale,
                                         n_rows, hidden, static_cast<hipStream_t>(hip_stream), ev_of(events, 0),
                                         ev_of(events, 1));
    return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_gateup_proj_i8(const void* x, const float* x_scale, const void* w, const float* w_scale, void* y,
                                int32_t n_tokens, int32_t hidden, int32_t n_out, void* workspace,
                                size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    return gateup_i8_call(x, x_scale, w, w_scale, y, n_tokens, hidden, n_out, false, workspace, workspace_bytes,
                          events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_gateup_act_i8(const void* x, const float* x_scale, const void* w, const float* w_scale, void* y,
                               int32_t n_tokens, int32_t hidden, int32_t n_inter, void* workspace,
                               size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    if (n_inter > (INT32_MAX - 512) / 2) return PPAS_ERANGE;
    const int32_t n_out = act_rows(n_inter);
    if (n_out < 0) return PPAS_EINVAL;
    return gateup_i8_call(x, x_scale, w, w_scale, y, n_tokens, hidden, n_out, true, workspace, workspace_bytes,
                          events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

size_t ppas_gateup_i8_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_out) {
  try {
    if (check_gateup_i8(n_tokens, hidden, n_out, false) != PPAS_OK || n_tokens == 0) return 0;
    return gateup_workspace_bytes(n_tokens, n_out, splits_i8(n_tokens, hidden, n_out, current_device().cus));
  } catch (...) {
    return 0;
  }
}

size_t ppas_gateup_act_i8_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t n_inter) {
  const int32_t n_out = act_rows(n_inter);
  return n_out < 0 ? 0 : ppas_gateup_i8_workspace_bytes(n_tokens, hidden, n_out);
}

ppas_status ppas_gateup_i8_choice(int32_t n_tokens, int32_t hidden, int32_t n_out, int32_t activation, int32_t aligned,
                                  size_t workspace_bytes, int32_t num_cus, int32_t* choice) {
  const ppas_status st = check_gateup_i8(n_tokens, hidden, n_out, activation != 0);
  if (st != PPAS_OK) return st;
  if (!choice || n_tokens == 0 || num_cus < 0 || (activation && n_out % 2 != 0)) return PPAS_EINVAL;
  const int cus = num_cus > 0 ? num_cus : 256;
  gateup_i8_choice(n_tokens, hidden, n_out, activation != 0, aligned != 0,
                   allowed_splits_i8(n_tokens, hidden, n_out, workspace_bytes, cus), cus, choice);
  return PPAS_OK;
}

namespace {

constexpr int32_t kMaxAdapterRows = 1 << 24;   // token rows of an adapters' call

ppas_status check_adapter_rows(int32_t n_tokens, int32_t n_adapters) {
  if (n_tokens < 0 || n_adapters <= 0) return PPAS_EINVAL;
  if (n_adapters > kAdaptersMax) return PPAS_EUNSUPPORTED;
  return n_tokens > kMaxAdapterRows ? PPAS_ERANGE : PPAS_OK;
}

ppas_status check_adapter_sizes(int32_t n_tokens, int32_t hidden, int32_t rank, int32_t n_adapters) {
  const ppas_status st = check_adapter_rows(n_tokens, n_adapters);
  if (st != PPAS_OK) return st;
  if (hidden <= 0 || rank <= 0) return PPAS_EINVAL;
  if (rank > kAdapterMaxRank) return PPAS_EUNSUPPORTED;
  return hidden > INT32_MAX - 512 ? PPAS_ERANGE : PPAS_OK;
}

ppas_status adapter_call(const ppas_adapters* set, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                         void* out, int64_t out_stride, int32_t n_tokens, const void* rows, size_t rows_bytes, bool act,
                         void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  if (!set) return PPAS_EINVAL;
  ppas_status st = check_adapter_sizes(n_tokens, set->hidden, set->rank, set->n_adapters);
  if (st != PPAS_OK) return st;
  if (set->n_out <= 0 || (act && set->n_out % 2 != 0)) return PPAS_EINVAL;
  if (set->n_out > INT32_MAX - 512) return PPAS_ERANGE;
  st = check_events(events);
  if (st != PPAS_OK || n_tokens == 0) return st;
  const int64_t cols = act ? set->n_out / 2 : set->n_out, most = (int64_t(1) << 61) / n_tokens;
  if (!set->a || !set->b || !x || !y || !out || !rows || !workspace) return PPAS_EINVAL;
  if (x_stride < set->hidden || y_stride < set->n_out || out_stride < cols) return PPAS_EINVAL;
  if (x_stride > most || y_stride > most || out_stride > most) return PPAS_ERANGE;
  if (off(set->a, 2) || off(set->b, 2) || off(set->scale, 4) || off(x, 2) || off(y, 2) || off(out, 2) || off(rows, 16) ||
      off(workspace, 16))
    return PPAS_EINVAL;
  const uint64_t out_bytes = span_bytes(n_tokens, out_stride, cols);
  const bool in_place = !act && out == y && out_stride == y_stride;
  if ((!in_place && overlap(out, out_bytes, y, span_bytes(n_tokens, y_stride, set->n_out))) ||
      overlap(out, out_bytes, x, span_bytes(n_tokens, x_stride, set->hidden)))
    return PPAS_EINVAL;
  if (rows_bytes < AdapterOrder{n_tokens, set->n_adapters}.bytes()) return PPAS_ENOSPACE;
  // a buffer that is kept for steps of any size may hold fewer splits than this one would take
  const size_t fit = workspace_bytes / adapter_workspace_bytes(n_tokens, set->rank, 1);
  if (fit == 0) return PPAS_ENOSPACE;
  const DeviceInfo dev = current_device();
  const int splits = int(std::min<size_t>(fit, size_t(adapter_splits(n_tokens, set->hidden, set->n_adapters, dev.cus))));
  const uint64_t n = uint64_t(set->n_adapters), r = uint64_t(set->rank);
  const Span weights_a{set->a, 2 * n * r * uint64_t(set->hidden)}, weights_b{set->b, 2 * n * r * uint64_t(set->n_out)},
      scale{set->scale, 4 * n}, order{rows, AdapterOrder{n_tokens, set->n_adapters}.bytes()},
      work{workspace, adapter_workspace_bytes(n_tokens, set->rank, splits)}, result{out, out_bytes};
  if (over_any(result, {weights_a, weights_b, scale, order, work}) ||
      over_any(work, {weights_a, weights_b, scale, order, {x, span_bytes(n_tokens, x_stride, set->hidden)},
                      {y, span_bytes(n_tokens, y_stride, set->n_out)}}))
    return PPAS_EINVAL;
  if (!dev.gfx950) return PPAS_EUNSUPPORTED;
  const AdapterCall c{static_cast<const uint16_t*>(set->a), static_cast<const uint16_t*>(set->b), set->scale,
                      static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(y), static_cast<uint16_t*>(out),
                      x_stride, y_stride, out_stride, n_tokens, set->hidden, set->n_out, set->rank, set->n_adapters,
                      rows, static_cast<float*>(workspace), splits};
  const hipError_t e = launch_adapters(c, act, dev.cus, static_cast<hipStream_t>(hip_stream), ev_of(events, 0),
                                       ev_of(events, 1));
  return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
}

}  // namespace

size_t ppas_adapter_rows_bytes(int32_t n_tokens, int32_t n_adapters) {
  if (check_adapter_rows(n_tokens, n_adapters) != PPAS_OK || n_tokens == 0) return 0;
  return AdapterOrder{n_tokens, n_adapters}.bytes();
}

ppas_status ppas_adapter_rows(const int32_t* row_adapter_dev, int32_t n_tokens, int32_t n_adapters, void* rows,
                              size_t rows_bytes, const ppas_events* events, void* hip_stream) {
  try {
    ppas_status st = check_adapter_rows(n_tokens, n_adapters);
    if (st != PPAS_OK) return st;
    st = check_events(events);
    if (st != PPAS_OK || n_tokens == 0) return st;
    if (!row_adapter_dev || !rows || off(row_adapter_dev, 4) || off(rows, 16)) return PPAS_EINVAL;
    const AdapterOrder o{n_tokens, n_adapters};
    if (rows_bytes < o.bytes()) return PPAS_ENOSPACE;
    if (overlap(rows, o.bytes(), row_adapter_dev, 4 * uint64_t(n_tokens))) return PPAS_EINVAL;   // read twice
    if (!current_device().gfx950) return PPAS_EUNSUPPORTED;
    const hipError_t e = launch_adapter_rows(row_adapter_dev, o, rows, static_cast<hipStream_t>(hip_stream),
                                             ev_of(events, 0), ev_of(events, 1));
    return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
  } catch (...) {
    return PPAS_EINVAL;
  }
}

size_t ppas_adapter_workspace_bytes(int32_t n_tokens, int32_t hidden, int32_t rank, int32_t n_adapters) {
  if (check_adapter_sizes(n_tokens, hidden, rank, n_adapters) != PPAS_OK || n_tokens == 0) return 0;
  try {
    return adapter_workspace_bytes(n_tokens, rank, adapter_splits(n_tokens, hidden, n_adapters, current_device().cus));
  } catch (...) {
    return 0;
  }
}

ppas_status ppas_adapter_add(const ppas_adapters* set, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                             void* out, int64_t out_stride, int32_t n_tokens, const void* rows, size_t rows_bytes,
                             void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    return adapter_call(set, x, x_stride, y, y_stride, out, out_stride, n_tokens, rows, rows_bytes, false, workspace,
                        workspace_bytes, events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_adapter_act(const ppas_adapters* set, const void* x, int64_t x_stride, const void* y, int64_t y_stride,
                             void* out, int64_t out_stride, int32_t n_tokens, const void* rows, size_t rows_bytes,
                             void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    return adapter_call(set, x, x_stride, y, y_stride, out, out_stride, n_tokens, rows, rows_bytes, true, workspace,
                        workspace_bytes, events, hip_stream);
  } catch (...) {
    return PPAS_EINVAL;
  }
}

namespace {

// what bounds a call's logit rows: token numbers and vectors stay far inside int32
constexpr int32_t kMaxVocab = 1 << 30;

ppas_status check_logprobs(int32_t n_rows, int32_t vocab, int32_t top_k) {
  if (n_rows < 0 || vocab <= 0 || top_k < 0) return PPAS_EINVAL;
  if (top_k > kLogprobsMaxTop) return PPAS_EUNSUPPORTED;
  return vocab > kMaxVocab ? PPAS_ERANGE : PPAS_OK;
}

}  // namespace

size_t ppas_logprobs_workspace_bytes(int32_t n_rows, int32_t vocab, int32_t top_k) {
  if (check_logprobs(n_rows, vocab, top_k) != PPAS_OK || n_rows == 0) return 0;
  try {
    const int cus = current_device().cus;
    return std::max(logprob_workspace_bytes(n_rows, top_k, logprob_split(n_rows, vocab, false, cus).splits),
                    logprob_workspace_bytes(n_rows, top_k, logprob_split(n_rows, vocab, true, cus).splits));
  } catch (...) {
    return 0;
  }
}

ppas_status ppas_logprobs(const void* logits, int32_t type, int64_t row_stride, int32_t n_rows, int32_t vocab,
                          float scale, const int32_t* tokens_dev, int32_t top_k, const ppas_logprob_out* out,
                          void* workspace, size_t workspace_bytes, const ppas_events* events, void* hip_stream) {
  try {
    ppas_status st = check_logprobs(n_rows, vocab, top_k);
    if (st != PPAS_OK) return st;
    if (type != PPAS_BF16 && type != PPAS_F32) return PPAS_EINVAL;
    if (!(scale >= 0x1p-100f && scale <= 0x1p100f)) return PPAS_EINVAL;
    st = check_events(events);
    if (st != PPAS_OK || n_rows == 0) return st;
    if (!logits || !out || row_stride < vocab || (workspace_bytes > 0 && !workspace)) return PPAS_EINVAL;
    if (row_stride > (int64_t(1) << 60) / n_rows) return PPAS_ERANGE;
    const LogprobRows r{logits,          row_stride,   tokens_dev,    out->logprob,      out->rank,
                        out->entropy,    top_k ? out->top_ids : nullptr, top_k ? out->top_logprobs : nullptr,
                        scale,           n_rows,       vocab,         out->top_ids || out->top_logprobs ? top_k : 0,
                        type == PPAS_F32};
    if ((r.logprob || r.rank) && !r.tokens) return PPAS_EINVAL;
    if (off(logits, type == PPAS_F32 ? 4 : 2) || off(r.tokens, 4) || off(r.logprob, 4) || off(r.rank, 4) ||
        off(r.entropy, 4) || off(r.top_ids, 4) || off(r.top_logprobs, 4) || off(workspace, 16))
      return PPAS_EINVAL;
    // the rows are read until the last result is written
    const uint64_t logit_bytes = span_bytes(n_rows, row_stride, vocab) * (r.f32 ? 2 : 1), n = uint64_t(n_rows);
    if (overlap(logits, logit_bytes, r.logprob, 4 * n) || overlap(logits, logit_bytes, r.rank, 4 * n) ||
        overlap(logits, logit_bytes, r.entropy, 4 * n) || overlap(logits, logit_bytes, r.top_ids, 4 * n * r.top) ||
        overlap(logits, logit_bytes, r.top_logprobs, 4 * n * r.top))
      return PPAS_EINVAL;
    if (!r.logprob && !r.rank && !r.entropy && !r.top) return PPAS_OK;
    const DeviceInfo dev = current_device();
    if (!dev.gfx950) return PPAS_EUNSUPPORTED;
    LogprobSplit split = logprob_split(n_rows, vocab, r.f32, dev.cus);
    for (; split.splits > 1 && logprob_workspace_bytes(n_rows, r.top, split.splits) > workspace_bytes; --split.splits)
      split.held = 0;   // longer parts than lanes hold
    const hipError_t e = launch_logprobs(r, split, workspace, static_cast<hipStream_t>(hip_stream), ev_of(events, 0),
                                         ev_of(events, 1));
    return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_stream_read(const void* buf, size_t bytes, void* sink, const ppas_events* events,
                             void* hip_stream) {
  try {
    const ppas_status st = check_events(events);
    if (st != PPAS_OK) return st;
    if (!buf || !sink || bytes % 16 != 0 || reinterpret_cast<uintptr_t>(buf) % 16 != 0 ||
        reinterpret_cast<uintptr_t>(sink) % 4 != 0)
      return PPAS_EINVAL;
    if (bytes == 0) return PPAS_OK;
    const DeviceInfo dev = current_device();
    if (!dev.gfx950) return PPAS_EUNSUPPORTED;
    const hipError_t e = launch_stream_read(buf, bytes, static_cast<uint32_t*>(sink), dev.cus,
                                            static_cast<hipStream_t>(hip_stream), ev_of(events, 0),
                                            ev_of(events, 1));
    return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
  } catch (...) {
    return PPAS_EINVAL;
  }
}

ppas_status ppas_kv_append(const ppas_shape* shape, void* k_pages, void* v_pages, const void* k_new,
                           const void* v_new, const ppas_seq* seqs, int32_t n_seqs,
                           const int32_t* block_table_dev, int32_t bt_stride,
                           const int32_t* block_table_host, void* hip_stream) {
  ppas_step_plan p;
  try {
    ppas_status st = validate(shape, seqs, n_seqs, block_table_host, bt_stride, true);
    if (st != PPAS_OK) return st;
    if (n_seqs == 0) return PPAS_OK;
    if (!k_pages || !v_pages || !k_new || !v_new || !block_table_dev) return PPAS_EINVAL;
    if (capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    // validated above; build only the page-write list
    st = build_plan(p, shape, seqs, n_seqs, nullptr, bt_stride, nullptr, kWantAppend, false);
    if (st == PPAS_OK) st = run_append(p, false, 0.f, nullptr, k_pages, v_pages, k_new, v_new, block_table_dev,
                                       nullptr, hip_stream);
    release(p.buf);
    return st;
  } catch (...) {
    release(p.buf);
    return PPAS_EINVAL;
  }
}

ppas_status ppas_rope_kv_append(const ppas_shape* shape, float rope_theta, void* q, void* k_pages, void* v_pages,
                                const void* k_new, const void* v_new, const ppas_seq* seqs, int32_t n_seqs,
                                const int32_t* block_table_dev, int32_t bt_stride,
                                const int32_t* block_table_host, void* hip_stream) {
  ppas_step_plan p;
  try {
    if (!std::isfinite(rope_theta) || !(rope_theta > 0.f)) return PPAS_EINVAL;
    ppas_status st = validate(shape, seqs, n_seqs, block_table_host, bt_stride, true);
    if (st != PPAS_OK) return st;
    if (n_seqs == 0) return PPAS_OK;
    if (!q || !k_pages || !v_pages || !k_new || !v_new || !block_table_dev) return PPAS_EINVAL;
    if (capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    st = build_plan(p, shape, seqs, n_seqs, nullptr, bt_stride, nullptr, kWantAppend, false);
    if (st == PPAS_OK) st = run_append(p, true, rope_theta, q, k_pages, v_pages, k_new, v_new, block_table_dev,
                                       nullptr, hip_stream);
    release(p.buf);
    return st;
  } catch (...) {
    release(p.buf);
    return PPAS_EINVAL;
  }
}

ppas_status ppas_rope_frequencies(const ppas_rope* rope, int32_t head_dim, double* out) {
  double w[kRopeMaxPairs];
  const ppas_status st = rope_frequencies(rope, head_dim, w);
  if (st != PPAS_OK) return st;
  if (!out) return PPAS_EINVAL;
  std::copy(w, w + rope->rotary_dim / 2, out);
  return PPAS_OK;
}

namespace {

ppas_status rope_rows_call(const ppas_head_norm* norm, const ppas_rope* rope, const void* x, int64_t x_stride, void* y,
                           int64_t y_stride, const int32_t* positions_dev, int32_t n_rows, int32_t n_heads,
                           int32_t head_dim, bool transposed, const ppas_events* events, void* hip_stream) {
  try {
    if (n_rows < 0 || n_heads < 1 || n_heads > 65536 || head_dim < 2 || head_dim % 2 != 0) return PPAS_EINVAL;
    if (head_dim > 2 * kRopeMaxPairs) return PPAS_EUNSUPPORTED;
    RopeTable table;
    ppas_status st = rope_table(rope, head_dim, table);
    if (st != PPAS_OK) return st;
    st = check_events(events);
    if (st != PPAS_OK) return st;
    if (norm) st = check_norm(norm, n_heads, head_dim);
    if (st != PPAS_OK || n_rows == 0) return st;
    const int64_t row = int64_t(n_heads) * head_dim, most = (int64_t(1) << 61) / n_rows;
    if (!x || !y || !positions_dev || x_stride < row || y_stride < row) return PPAS_EINVAL;
    if (x_stride > most || y_stride > most) return PPAS_ERANGE;
    if (off(x, 2) || off(y, 2) || off(positions_dev, 4)) return PPAS_EINVAL;
    if (!(x == y && x_stride == y_stride) &&
        overlap(x, span_bytes(n_rows, x_stride, row), y, span_bytes(n_rows, y_stride, row)))
      return PPAS_EINVAL;
    if (norm && over_any(weights_of(*norm, n_heads, head_dim), {{y, span_bytes(n_rows, y_stride, row)}})) return PPAS_EINVAL;
    if (!current_device().gfx950) return PPAS_EUNSUPPORTED;
    const RopeRows r{static_cast<const uint16_t*>(x), static_cast<uint16_t*>(y), x_stride, y_stride, positions_dev,
                     n_rows, n_heads, head_dim, transposed};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const hipError_t e =
        norm ? launch_norm_rope_rows(r, norm_of(*norm), table, stream, ev_of(events, 0), ev_of(events, 1))
             : launch_rope_rows(r, table, stream, ev_of(events, 0), ev_of(events, 1));
    return e == hipSuccess ? PPAS_OK : PPAS_EHIP;
  } catch (...) {
    return PPAS_EINVAL;
  }
}

}  // namespace

ppas_status ppas_rope_rows(const ppas_rope* rope, const void* x, int64_t x_stride, void* y, int64_t y_stride,
                           const int32_t* positions_dev, int32_t n_rows, int32_t n_heads, int32_t head_dim,
                           int32_t transposed, const ppas_events* events, void* hip_stream) {
  return rope_rows_call(nullptr, rope, x, x_stride, y, y_stride, positions_dev, n_rows, n_heads, head_dim,
                        transposed != 0, events, hip_stream);
}

ppas_status ppas_norm_rope_rows(const ppas_head_norm* norm, const ppas_rope* rope, const void* x, int64_t x_stride,
                                void* y, int64_t y_stride, const int32_t* positions_dev, int32_t n_rows,
                                int32_t n_heads, int32_t head_dim, const ppas_events* events, void* hip_stream) {
  if (!norm) return PPAS_EINVAL;
  return rope_rows_call(norm, rope, x, x_stride, y, y_stride, positions_dev, n_rows, n_heads, head_dim, false, events,
                        hip_stream);
}

namespace {

ppas_status qkv_append(const ppas_shape* shape, const Norms* norms, const ppas_rope* rope, const ppas_qkv* rows,
                       void* q_out, void* k_pages, void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                       const int32_t* block_table_dev, int32_t bt_stride, const int32_t* block_table_host,
                       void* hip_stream) {
  ppas_step_plan p;
  try {
    ppas_status st = validate(shape, seqs, n_seqs, block_table_host, bt_stride, true);
    if (st != PPAS_OK) return st;
    st = check_norms(norms, *shape);
    if (st != PPAS_OK) return st;
    RopeTable table;
    if (n_seqs == 0) return rope_table(rope, kHeadDim, table);
    const int64_t T = int64_t(seqs[n_seqs - 1].query_start) + seqs[n_seqs - 1].n_query;
    st = check_qkv(*shape, rope, rows, q_out, k_pages, v_pages, block_table_dev, T, table);
    if (st != PPAS_OK) return st;
    if (over_weights(norms, *shape, q_out, k_pages, v_pages, T)) return PPAS_EINVAL;
    if (capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    // validated above; build only the page-write list
    st = build_plan(p, shape, seqs, n_seqs, nullptr, bt_stride, nullptr, kWantInline, false);
    if (st == PPAS_OK)
      st = run_qkv_append(p, table, norms, *rows, q_out, k_pages, v_pages, block_table_dev, nullptr, hip_stream);
    release(p.buf);
    return st;
  } catch (...) {
    release(p.buf);
    return PPAS_EINVAL;
  }
}

}  // namespace

ppas_status ppas_rope_qkv_append(const ppas_shape* shape, const ppas_rope* rope, const ppas_qkv* rows, void* q_out,
                                 void* k_pages, void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                                 const int32_t* block_table_dev, int32_t bt_stride,
                                 const int32_t* block_table_host, void* hip_stream) {
  return qkv_append(shape, nullptr, rope, rows, q_out, k_pages, v_pages, seqs, n_seqs, block_table_dev, bt_stride,
                    block_table_host, hip_stream);
}

ppas_status ppas_norm_rope_qkv_append(const ppas_shape* shape, const ppas_head_norm* q_norm,
                                      const ppas_head_norm* k_norm, const ppas_rope* rope, const ppas_qkv* rows,
                                      void* q_out, void* k_pages, void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                                      const int32_t* block_table_dev, int32_t bt_stride,
                                      const int32_t* block_table_host, void* hip_stream) {
  const Norms norms{q_norm, k_norm};
  return qkv_append(shape, &norms, rope, rows, q_out, k_pages, v_pages, seqs, n_seqs, block_table_dev, bt_stride,
                    block_table_host, hip_stream);
}

size_t ppas_attn_shared_workspace_bytes(const ppas_shape* shape, const ppas_seq* seqs, int32_t n_seqs,
                                        const ppas_prefix* prefixes, int32_t n_prefixes) {
  try {
    if (validate(shape, seqs, n_seqs, nullptr, INT32_MAX, false) != PPAS_OK ||
        validate_prefixes(seqs, n_seqs, nullptr, INT32_MAX, prefixes, n_prefixes) != PPAS_OK)
      return 0;
    Plan plan;
    make_plan(*shape, seqs, n_seqs, current_device().cus, PlanOpts{}, plan, prefixes, n_prefixes);
    return plan_fits(plan, 0) ? plan.total : 0;
  } catch (...) {
    return 0;
  }
}

ppas_status ppas_attn_step(const ppas_shape* shape, void* out, const void* q, const void* k_pages,
                           const void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                           const int32_t* block_table_dev, int32_t bt_stride, const int32_t* block_table_host,
                           void* workspace, size_t workspace_bytes, void* hip_stream) {
  return ppas_attn_step_shared(shape, out, q, k_pages, v_pages, seqs, n_seqs, nullptr, 0, block_table_dev, bt_stride,
                               block_table_host, workspace, workspace_bytes, hip_stream);
}

ppas_status ppas_attn_step_shared(const ppas_shape* shape, void* out, const void* q, const void* k_pages,
                                  const void* v_pages, const ppas_seq* seqs, int32_t n_seqs,
                                  const ppas_prefix* prefixes, int32_t n_prefixes, const int32_t* block_table_dev,
                                  int32_t bt_stride, const int32_t* block_table_host, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  ppas_step_plan p;
  try {
    ppas_status st = validate(shape, seqs, n_seqs, block_table_host, bt_stride, false);
    if (st != PPAS_OK) return st;
    st = validate_prefixes(seqs, n_seqs, block_table_host, bt_stride, prefixes, n_prefixes);
    if (st != PPAS_OK) return st;
    if (n_seqs == 0) return PPAS_OK;
    if (!out || !q || !k_pages || !v_pages || !block_table_dev || !workspace) return PPAS_EINVAL;
    if (capturing(hip_stream)) return PPAS_EUNSUPPORTED;
    // validated above
    st = build_plan(p, shape, seqs, n_seqs, nullptr, bt_stride, nullptr, kWantAttn, false, prefixes, n_prefixes);
    if (st == PPAS_OK)
      st = run_attn(p, out, q, k_pages, v_pages, block_table_dev, workspace, workspace_bytes, nullptr, hip_stream);
    release(p.buf);
    return st;
  } catch (...) {
    release(p.buf);
    return PPAS_EINVAL;
  }
}

}  // extern "C"
