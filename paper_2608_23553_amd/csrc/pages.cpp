// pages.cpp - the C ABI of the paged MXFP4 token store: validation, host
// bookkeeping (pages_book.h), the plans' way to the device and the order of
// calls on different streams.  The kernels are in k_pages.hip.
#include <atomic>
#include <cstdio>
#include <cstring>
#include <new>

#include "guards.h"
#include "internal.h"
#include "pages_handle.h"

namespace chimera {

// Whether s is being captured into a graph.  Elsewhere: s is the null stream, and
// a blocking stream is captured, which forbids work on it.
enum class Capture { none, here, elsewhere };
static Capture capture(hipStream_t s) {
  hipStreamCaptureStatus st = hipStreamCaptureStatusNone;
  if (hipStreamIsCapturing(s, &st) != hipSuccess) {
    (void)hipGetLastError();
    return Capture::elsewhere;
  }
  return st == hipStreamCaptureStatusNone ? Capture::none : Capture::here;
}
static int captured_elsewhere(const char *call) {
  return fail(CHIMERA_E_UNSUPPORTED, "%s: another stream's capture forbids work on the null stream", call);
}

int pages_not_captured(hipStream_t s, const char *call, const char *why) {
  switch (capture(s)) {
    case Capture::none: return CHIMERA_OK;
    case Capture::elsewhere: return captured_elsewhere(call);
    case Capture::here: break;
  }
  return fail(CHIMERA_E_UNSUPPORTED, "%s: cannot be captured into a graph (%s)", call, why);
}

int pages_order_before(chimera_pages *pg, hipStream_t s) {
  if (pg->on_null && s == nullptr) return CHIMERA_OK;
  if (pg->on_null) {
    if (capture(nullptr) != Capture::none) return captured_elsewhere("a call behind work on the null stream");
    CHIMERA_HIP(hipEventRecord(pg->done, nullptr));
    pg->pending = true;
    pg->on_null = false;
  }
  if (pg->pending) CHIMERA_HIP(hipStreamWaitEvent(s, pg->done, 0));
  return CHIMERA_OK;
}
int pages_order_after(chimera_pages *pg, hipStream_t s) {
  pg->on_null = s == nullptr;
  if (!pg->on_null) {
    CHIMERA_HIP(hipEventRecord(pg->done, s));
    pg->pending = true;
  }
  return CHIMERA_OK;
}

static int ring_make(PlanRing &r, size_t half) {
  for (int i = 0; i < 2; ++i) {
    if (!r.left[i]) CHIMERA_HIP(hipEventCreateWithFlags(&r.left[i], hipEventDisableTiming));
    r.pending[i] = false;
  }
  if (r.host) CHIMERA_HIP(hipHostFree(r.host));
  r.host = nullptr;
  if (r.dev) CHIMERA_HIP(hipFree(r.dev));
  r.dev = nullptr;
  r.half = r.used = 0;
  r.cur = 0;
  hipError_t e = hipHostMalloc((void **)&r.host, 2 * half, hipHostMallocDefault);
  if (e == hipSuccess) e = hipMalloc((void **)&r.dev, 2 * half);
  if (e != hipSuccess) {
    if (r.host) (void)hipHostFree(r.host);
    r.host = r.dev = nullptr;
    (void)hipGetLastError();
    return hip_fail(e, "plan buffer");
  }
  r.half = half;
  return CHIMERA_OK;
}

// Room for a call's plan; s is ordered behind every earlier call (pages_order_before).
static int ring_take(chimera_pages *pg, size_t bytes, hipStream_t s, char **out) {
  PlanRing &r = pg->ring;
  bytes = (bytes + 63) / 64 * 64;
  if (bytes > r.half) {  // the plans under way lie in the buffer that goes
    CHIMERA_HIP(hipDeviceSynchronize());
    size_t half = 512 << 10;
    while (half < 2 * bytes) half *= 2;
    if (int rc = ring_make(r, half)) return rc;
  }
  if (r.used + bytes > r.half) {
    CHIMERA_HIP(hipEventRecord(r.left[r.cur], s));
    r.pending[r.cur] = true;
    r.cur ^= 1;
    r.used = 0;
    if (r.pending[r.cur]) CHIMERA_HIP(hipEventSynchronize(r.left[r.cur]));
    r.pending[r.cur] = false;
  }
  *out = r.host + (size_t)r.cur * r.half + r.used;
  r.used += bytes;
  return CHIMERA_OK;
}

// Where the kernels read the first `bytes` of a plan: in place or, from 32 KB on,
// copied, which is one more launch for the host (2.7 us). On the device, 32 bytes
// a fork: 256 copied and read 5.4 us, in place 4.4; 512: 5.7 and 6.0; 1024: 6.3 and
// 9.0; 4096: 9.0 and 26.9; 36 bytes an append: 256: 5.8 and 5.5; 1024: 6.8 and 10.4.
static char *plan_for_device(chimera_pages *pg, char *plan, size_t bytes, hipStream_t s) {
  if (bytes < (32 << 10)) return plan;
  char *dev = pg->ring.dev + (plan - pg->ring.host);
  launch_pages_plan(plan, dev, (bytes + 15) / 16 * 16, s);
  return dev;
}

static int book_fail(BookError e, const char *call, const int64_t *ids, int64_t at) {
  const long long i = (long long)at, id = ids ? (long long)ids[at] : -1;
  switch (e) {
    case BookError::none: return CHIMERA_OK;
    case BookError::id: return fail(CHIMERA_E_INVAL, "%s: entry %lld: document id out of range", call, i);
    case BookError::repeated: return fail(CHIMERA_E_INVAL, "%s: entry %lld: document %lld named twice", call, i, id);
    case BookError::length:
      return fail(CHIMERA_E_INVAL, "%s: entry %lld: length below 0 or above the document's", call, i);
    case BookError::too_long: return fail(CHIMERA_E_INVAL, "%s: entry %lld: document longer than max_len", call, i);
    case BookError::busy_dst: return fail(CHIMERA_E_INVAL, "%s: entry %lld: document %lld is not empty", call, i, id);
    case BookError::src_is_dst:
      return fail(CHIMERA_E_INVAL, "%s: entry %lld: its source is written by the same call", call, i);
    case BookError::position:
      return fail(CHIMERA_E_INVAL, "%s: entry %lld: positions must ascend within the document", call, i);
    case BookError::pages: return fail(CHIMERA_E_NOMEM, "%s: not enough free pages", call);
  }
  return fail(CHIMERA_E_INVAL, "%s: internal error", call);
}

// What every call that changes or reads documents by a host list starts with.
static int check_list(const chimera_pages *pg, const void *ids, int64_t n, const char *call,
                      int64_t most = kPagesMaxItems) {
  if (!pg) return fail(CHIMERA_E_INVAL, "null pages");
  if (n < 0 || (n > 0 && !ids)) return fail(CHIMERA_E_INVAL, "%s: null ids or n < 0", call);
  if (n > most) return fail(CHIMERA_E_UNSUPPORTED, "%s: more than %lld documents in one call", call, (long long)most);
  return CHIMERA_OK;
}
static int check_stream(hipStream_t s, const char *call) {
  return pages_not_captured(s, call, "its host bookkeeping happens once");
}

// exact: the documents' tokens, which have to be as many as rows (below 0: they
// are only counted); null: at most as many.
static int read_common(chimera_pages *pg, const int64_t *doc_ids, int64_t n, void *out, int64_t rows, int dtype,
                       int64_t *exact, void *hip_stream) {
  if (int rc = check_list(pg, doc_ids, n, "read")) return rc;
  if (dtype != CHIMERA_F32 && dtype != CHIMERA_BF16) return fail(CHIMERA_E_INVAL, "dtype must be F32 or BF16");
  if ((uintptr_t)out % 16) return fail(CHIMERA_E_INVAL, "read: out must be 16-byte aligned");
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(pg);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  int64_t at = 0, items = 0, total = 0;
  if (exact && rows < 0) return book_fail(pg->book.count(doc_ids, n, &at, exact), "read", doc_ids, at);
  DeviceGuard dg(pg->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", pg->device);
  return guarded([&]() -> int {
    if (BookError e = pg->book.check_read(doc_ids, n, &at, &items, &total); e != BookError::none)
      return book_fail(e, "read", doc_ids, at);
    if (exact) *exact = total;
    if (total > rows || (exact && total < rows))
      return fail(CHIMERA_E_INVAL, "read: %lld tokens, out has %lld rows", (long long)total, (long long)rows);
    if (items == 0) return CHIMERA_OK;
    if (!out) return fail(CHIMERA_E_INVAL, "null output pointer");
    if (items > kPagesMaxItems) return fail(CHIMERA_E_UNSUPPORTED, "read: too many tokens in one call");
    if (int rc = check_stream(s, "read")) return rc;
    char *plan = nullptr;
    if (int rc = pages_order_before(pg, s)) return rc;
    if (int rc = ring_take(pg, (size_t)items * sizeof(PageItem), s, &plan)) return rc;
    pg->book.plan_read(doc_ids, n, (PageItem *)plan);
    const PageItem *it = (const PageItem *)plan_for_device(pg, plan, (size_t)items * sizeof(PageItem), s);
    launch_pages_read(it, items, pg->view.pool, pg->view.table, pg->view.stride, out, dtype, s);
    CHIMERA_HIP(hipGetLastError());
    return pages_order_after(pg, s);
  });
}

}  // namespace chimera

using namespace chimera;

extern "C" {

int chimera_pages_create(int hip_device, int64_t npages, int64_t ndocs, int32_t max_len, chimera_pages **out) {
  if (!out) return fail(CHIMERA_E_INVAL, "null argument");
  if (npages < 1 || ndocs < 1 || max_len < 1)
    return fail(CHIMERA_E_INVAL, "npages, ndocs and max_len must be >= 1");
  if (npages > kPagesMaxPages || ndocs > INT32_MAX || max_len > CHIMERA_PAGES_MAX_LEN)
    return fail(CHIMERA_E_UNSUPPORTED, "npages above %lld, ndocs above 2^31 - 1 or max_len above %d",
                (long long)kPagesMaxPages, CHIMERA_PAGES_MAX_LEN);
  int ndev = 0;
  if (hipGetDeviceCount(&ndev) != hipSuccess || ndev <= 0) {
    (void)hipGetLastError();
    return fail(CHIMERA_E_DEVICE, "no HIP device available");
  }
  if (hip_device < 0 || hip_device >= ndev)
    return fail(CHIMERA_E_INVAL, "device %d out of range (%d devices)", hip_device, ndev);
  DeviceGuard dg(hip_device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", hip_device);
  return guarded([&]() -> int {
    const size_t stride = (size_t)PageBook::row_pages(max_len);
    const size_t bytes[3] = {(size_t)npages * kPageBytes, (size_t)ndocs * stride * 4, (size_t)ndocs * 4};
    size_t free_b = 0, total_b = 0;
    if (hipMemGetInfo(&free_b, &total_b) == hipSuccess && bytes[0] + bytes[1] + bytes[2] > free_b)
      return fail(CHIMERA_E_NOMEM, "pages need %zu bytes, %zu free on device %d", bytes[0] + bytes[1] + bytes[2],
                  free_b, hip_device);
    chimera_pages *pg = new chimera_pages;
    pg->device = hip_device;
    int rc = guarded([&]() -> int {
      pg->book.init(npages, ndocs, max_len);
      void **ptr[3] = {(void **)&pg->view.pool, (void **)&pg->view.table, (void **)&pg->view.lens};
      for (int i = 0; i < 3; ++i) {
        hipError_t e = hipMalloc(ptr[i], bytes[i]);
        if (e == hipSuccess) e = hipMemset(*ptr[i], 0, bytes[i]);
        if (e != hipSuccess) {
          (void)hipGetLastError();
          return hip_fail(e, "page pool");
        }
      }
      CHIMERA_HIP(hipEventCreateWithFlags(&pg->done, hipEventDisableTiming));
      if (int rc = ring_make(pg->ring, 512 << 10)) return rc;
      CHIMERA_HIP(hipDeviceSynchronize());  // the clears above ran on the null stream
      return CHIMERA_OK;
    });
    if (rc) {
      chimera_pages_free(pg);
      return rc;
    }
    pg->view.ndocs = ndocs;
    pg->view.stride = (int)stride;
    pg->device_bytes = (int64_t)(bytes[0] + bytes[1] + bytes[2]);
    *out = pg;
    return CHIMERA_OK;
  });
}

void chimera_pages_free(chimera_pages *pg) {
  if (!pg) return;
  DeviceGuard dg(pg->device);
  (void)hipDeviceSynchronize();
  for (void *p : {(void *)pg->view.pool, (void *)pg->view.table, (void *)pg->view.lens})
    if (p) (void)hipFree(p);
  if (pg->ring.host) (void)hipHostFree(pg->ring.host);
  if (pg->ring.dev) (void)hipFree(pg->ring.dev);
  for (hipEvent_t e : pg->ring.left)
    if (e) (void)hipEventDestroy(e);
  if (pg->done) (void)hipEventDestroy(pg->done);
  delete pg;
}

int chimera_pages_info_get(const chimera_pages *pg, chimera_pages_info *out) {
  if (!pg || !out) return fail(CHIMERA_E_INVAL, "null argument");
  out->npages = pg->book.npages;
  out->free_pages = pg->book.free_pages();
  out->ndocs = pg->book.ndocs;
  out->ntokens = pg->book.ntok;
  out->device_bytes = pg->device_bytes;
  out->max_len = pg->book.max_len;
  out->device = pg->device;
  return CHIMERA_OK;
}

int chimera_pages_lengths(const chimera_pages *pg, const int64_t *doc_ids, int64_t n, int32_t *lens,
                          int64_t *total) {
  if (int rc = check_list(pg, doc_ids, n, "lengths", INT64_MAX)) return rc;
  for (int64_t i = 0; i < n; ++i)
    if (doc_ids[i] < 0 || doc_ids[i] >= pg->book.ndocs) return book_fail(BookError::id, "lengths", doc_ids, i);
  int64_t sum = 0;
  for (int64_t i = 0; i < n; ++i) {
    sum += pg->book.len[doc_ids[i]];
    if (lens) lens[i] = pg->book.len[doc_ids[i]];
  }
  if (total) *total = sum;
  return CHIMERA_OK;
}

int chimera_pages_append(chimera_pages *pg, const int64_t *doc_ids, const int32_t *lens, int64_t n, const void *X,
                         int x_dtype, int32_t d, int64_t ld, int64_t doc_stride, void *hip_stream) {
  if (int rc = check_list(pg, doc_ids, n, "append")) return rc;
  if (n > 0 && !lens) return fail(CHIMERA_E_INVAL, "append: null lens");
  if (x_dtype != CHIMERA_F32 && x_dtype != CHIMERA_BF16) return fail(CHIMERA_E_INVAL, "x_dtype must be F32 or BF16");
  if (d != CHIMERA_DIM) return fail(CHIMERA_E_INVAL, "token dim %d != %d", d, CHIMERA_DIM);
  const int64_t unit = x_dtype == CHIMERA_F32 ? 4 : 8;
  if (ld < CHIMERA_DIM || ld % unit || (uintptr_t)X % 16)
    return fail(CHIMERA_E_INVAL, "append: rows must be 16-byte aligned (X, and ld a multiple of %d that is >= %d)",
                (int)unit, CHIMERA_DIM);
  if (doc_stride < 0) return fail(CHIMERA_E_INVAL, "append: doc_stride must be >= 0");
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(pg);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  DeviceGuard dg(pg->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", pg->device);
  return guarded([&]() -> int {
    int64_t at = 0, items = 0, pages = 0;
    if (BookError e = pg->book.check_append(doc_ids, lens, n, &at, &items, &pages); e != BookError::none)
      return book_fail(e, "append", doc_ids, at);
    for (int64_t i = 0; doc_stride && i < n; ++i)
      if (lens[i] > doc_stride)
        return fail(CHIMERA_E_INVAL, "append: entry %lld: length %d above doc_stride", (long long)i, lens[i]);
    if (items == 0) return CHIMERA_OK;
    if (!X) return fail(CHIMERA_E_INVAL, "append: null token pointer");
    if (items > kPagesMaxItems) return fail(CHIMERA_E_UNSUPPORTED, "append: too many tokens in one call");
    if (int rc = check_stream(s, "append")) return rc;
    char *plan = nullptr;
    if (int rc = pages_order_before(pg, s)) return rc;
    const size_t bytes = (size_t)items * sizeof(PageItem) + (size_t)(pages + PageBook::kSlack) * 4;
    if (int rc = ring_take(pg, bytes, s, &plan)) return rc;
    pg->book.commit_append(doc_ids, lens, n, doc_stride, (PageItem *)plan, (int32_t *)((PageItem *)plan + items));
    const PageItem *it = (const PageItem *)plan_for_device(pg, plan, bytes, s);
    launch_pages_append(it, items, (const int32_t *)(it + items), X, x_dtype, ld, pg->view.pool, pg->view.table,
                        pg->view.stride, pg->view.lens, s);
    CHIMERA_HIP(hipGetLastError());
    return pages_order_after(pg, s);
  });
}

int chimera_pages_fork(chimera_pages *pg, const int64_t *src_ids, const int64_t *dst_ids, const int32_t *lens,
                       int64_t n, void *hip_stream) {
  if (int rc = check_list(pg, src_ids, n, "fork")) return rc;
  if (n > 0 && !dst_ids) return fail(CHIMERA_E_INVAL, "fork: null ids");
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(pg);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  DeviceGuard dg(pg->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", pg->device);
  return guarded([&]() -> int {
    int64_t at = 0;
    if (BookError e = pg->book.check_fork(src_ids, dst_ids, lens, n, &at); e != BookError::none)
      return book_fail(e, "fork", dst_ids, at);
    if (n == 0) return CHIMERA_OK;
    if (int rc = check_stream(s, "fork")) return rc;
    char *plan = nullptr;
    if (int rc = pages_order_before(pg, s)) return rc;
    if (int rc = ring_take(pg, (size_t)n * sizeof(PageItem), s, &plan)) return rc;
    pg->book.commit_fork(src_ids, dst_ids, lens, n, (PageItem *)plan);
    const PageItem *it = (const PageItem *)plan_for_device(pg, plan, (size_t)n * sizeof(PageItem), s);
    launch_pages_fork(it, n, pg->view.pool, pg->view.table, pg->view.stride, pg->view.lens, s);
    CHIMERA_HIP(hipGetLastError());
    return pages_order_after(pg, s);
  });
}

int chimera_pages_copy(chimera_pages *src, const int64_t *src_ids, chimera_pages *dst, const int64_t *dst_ids,
                       const int32_t *lens, const int32_t *positions, int64_t n, void *hip_stream) {
  if (int rc = check_list(src, src_ids, n, "copy")) return rc;
  if (int rc = check_list(dst, dst_ids, n, "copy")) return rc;
  if (src->device != dst->device) return fail(CHIMERA_E_INVAL, "copy: the two stores are on different devices");
  if (positions && !lens) return fail(CHIMERA_E_INVAL, "copy: positions without lens");
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(dst);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  BusyGuard<chimera_pages> bs(src != dst ? src : nullptr);
  if (!bs.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  DeviceGuard dg(dst->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", dst->device);
  return guarded([&]() -> int {
    int64_t at = 0, items = 0, pages = 0, npos = 0, turns = 0;
    bool in_place = false;
    if (BookError e = src->book.check_copy(src_ids, dst->book, dst_ids, lens, positions, n, &at, &items, &pages,
                                           &npos, &turns, &in_place);
        e != BookError::none)
      return book_fail(e, "copy", dst_ids, at);
    if (items == 0) return CHIMERA_OK;
    if (items > kPagesMaxItems) return fail(CHIMERA_E_UNSUPPORTED, "copy: too many tokens in one call");
    if (int rc = check_stream(s, "copy")) return rc;
    char *plan = nullptr;
    if (int rc = pages_order_before(dst, s)) return rc;
    if (src != dst)
      if (int rc = pages_order_before(src, s)) return rc;
    const bool short_pos = src->book.max_len <= 65536;  // positions in 16 bits
    const size_t ids_at = (size_t)items * sizeof(PageItem), pos_at = ids_at + (size_t)(pages + PageBook::kSlack) * 4;
    const size_t bytes = pos_at + (size_t)npos * (short_pos ? 2 : 4);
    if (int rc = ring_take(dst, bytes, s, &plan)) return rc;
    if (!(short_pos ? PageBook::take_positions(positions, npos, turns, (uint16_t *)(plan + pos_at))
                    : PageBook::take_positions(positions, npos, turns, (int32_t *)(plan + pos_at))))
      return book_fail(BookError::position, "copy", dst_ids, PageBook::falling(lens, positions, n));
    src->book.commit_copy(src_ids, dst->book, dst_ids, lens, positions, n, (PageItem *)plan,
                          (int32_t *)(plan + ids_at));
    const char *p = plan_for_device(dst, plan, bytes, s);
    launch_pages_copy((const PageItem *)p, items, (const int32_t *)(p + ids_at), positions ? p + pos_at : nullptr,
                      short_pos, src->view.pool, src->view.table, src->view.stride, dst->view.pool,
                      dst->view.table, dst->view.stride, dst->view.lens, in_place, s);
    CHIMERA_HIP(hipGetLastError());
    if (src != dst)
      if (int rc = pages_order_after(src, s)) return rc;
    return pages_order_after(dst, s);
  });
}

int chimera_pages_drop(chimera_pages *pg, const int64_t *doc_ids, int64_t n, void *hip_stream) {
  if (int rc = check_list(pg, doc_ids, n, "drop")) return rc;
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(pg);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  for (int64_t i = 0; i < n; ++i)
    if (doc_ids[i] < 0 || doc_ids[i] >= pg->book.ndocs) return book_fail(BookError::id, "drop", doc_ids, i);
  if (n == 0) return CHIMERA_OK;
  DeviceGuard dg(pg->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", pg->device);
  return guarded([&]() -> int {
    if (int rc = check_stream(s, "drop")) return rc;
    char *plan = nullptr;
    if (int rc = pages_order_before(pg, s)) return rc;
    if (int rc = ring_take(pg, (size_t)n * 8, s, &plan)) return rc;
    int64_t *ids = (int64_t *)plan, m = 0;
    for (int64_t i = 0; i < n; ++i) {
      if (pg->book.len[doc_ids[i]] == 0) continue;  // empty, or named before
      ids[m++] = doc_ids[i];
      pg->book.release(doc_ids[i]);
    }
    if (m == 0) return CHIMERA_OK;
    launch_pages_drop(ids, m, pg->view.lens, s);
    CHIMERA_HIP(hipGetLastError());
    return pages_order_after(pg, s);
  });
}

int chimera_pages_read(chimera_pages *pg, const int64_t *doc_ids, int64_t n, void *out, int64_t rows, int dtype,
                       void *hip_stream) {
  return read_common(pg, doc_ids, n, out, rows, dtype, nullptr, hip_stream);
}

int chimera_pages_read_all(chimera_pages *pg, const int64_t *doc_ids, int64_t n, void *out, int64_t rows, int dtype,
                           int64_t *total, void *hip_stream) {
  if (!total) return fail(CHIMERA_E_INVAL, "read: null total");
  return read_common(pg, doc_ids, n, out, rows, dtype, total, hip_stream);
}

int chimera_pages_score(chimera_pages *pg, const void *Q, int q_dtype, int64_t nq, int32_t Tq, int32_t d,
                        const int32_t *doc_ids, int64_t n, int64_t ld, float *scores, void *hip_stream) {
  if (!pg) return fail(CHIMERA_E_INVAL, "null pages");
  if (nq < 0 || n < 0) return fail(CHIMERA_E_INVAL, "nq and n must be >= 0");
  if (q_dtype != CHIMERA_F32 && q_dtype != CHIMERA_BF16) return fail(CHIMERA_E_INVAL, "q_dtype must be F32 or BF16");
  if (d != CHIMERA_DIM) return fail(CHIMERA_E_INVAL, "query dim %d != %d", d, CHIMERA_DIM);
  if (Tq < 1) return fail(CHIMERA_E_INVAL, "Tq must be >= 1");
  if (Tq > CHIMERA_MAX_TQ) return fail(CHIMERA_E_UNSUPPORTED, "Tq %d > %d", Tq, CHIMERA_MAX_TQ);
  if (n > CHIMERA_PAGES_MAX_SCORE)
    return fail(CHIMERA_E_UNSUPPORTED, "n %lld > %d", (long long)n, CHIMERA_PAGES_MAX_SCORE);
  if (!doc_ids && n > pg->book.ndocs) return fail(CHIMERA_E_INVAL, "n above ndocs without a list of documents");
  if (doc_ids && ld != 0 && ld < n) return fail(CHIMERA_E_INVAL, "ld must be 0 (one list for every query) or >= n");
  if (nq == 0 || n == 0) return CHIMERA_OK;
  if (!Q) return fail(CHIMERA_E_INVAL, "null query pointer");
  if (!scores) return fail(CHIMERA_E_INVAL, "null output pointer");
  if ((uintptr_t)Q % 16) return fail(CHIMERA_E_INVAL, "Q must be 16-byte aligned");
  hipStream_t s = (hipStream_t)hip_stream;
  BusyGuard<chimera_pages> bg(pg);
  if (!bg.ok) return fail(CHIMERA_E_BUSY, "pages in use by another thread");
  DeviceGuard dg(pg->device);
  if (!dg.ok) return fail(CHIMERA_E_DEVICE, "cannot select device %d", pg->device);
  const Capture c = capture(s);
  if (c == Capture::elsewhere) return captured_elsewhere("score");
  const bool graph = c == Capture::here;
  if (!graph)
    if (int rc = pages_order_before(pg, s)) return rc;
  launch_pages_score(Q, q_dtype, nq, Tq, Tq, doc_ids, ld, nullptr, n, pg->view, scores, false, s);
  CHIMERA_HIP(hipGetLastError());
  return graph ? CHIMERA_OK : pages_order_after(pg, s);
}

}  // extern "C"
