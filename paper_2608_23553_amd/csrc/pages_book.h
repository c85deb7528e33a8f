// pages_book.h - host bookkeeping of the paged token store (chimera_pages):
// which pages each document holds and how many documents hold each page.  No
// HIP in here: the plans below are what the kernels of k_pages.hip carry out.
//
// A document's token i is slot i % 16 of its page i / 16.  A page that several
// documents hold is full in all of them, so no call ever writes into a page
// that another document can see: a fork shares whole pages only and copies the
// partly filled one behind them.
#pragma once

#include <cstdint>
#include <cstring>
#include <vector>

namespace chimera {

constexpr int kPageTokens = 16;
// pages one work item of a plan covers at most: long documents are cut, so
// that no workgroup has much more to do than the others
constexpr int kItemPages = 16;

// One work item: pages first .. first + npages - 1 of document doc.
struct PageItem {
  int32_t doc = 0;      // document written (read: document read)
  int32_t first = 0;    // its first page here, as a page of the document
  int32_t pages = 0;    // position of their page ids in the plan's list
  int32_t len = -1;     // the document's length after the call; -1: another item sets it
  int64_t row = 0;      // append, read: first row of the tensor; copy: its place in the list of positions, or first token
  int32_t src = 0;      // copy, fork: the document read
  uint16_t ntok = 0;    // tokens to write (read) from there
  uint8_t npages = 0;
  uint8_t fill = 0;     // tokens that the first page holds already
};
static_assert(sizeof(PageItem) == 32 && kItemPages * kPageTokens <= 65535, "a plan is read across the bus");

// What the caller asked for that cannot be done (see the messages in pages.cpp).
enum class BookError { none, id, repeated, length, too_long, busy_dst, src_is_dst, pages, position };

struct PageBook {
  int64_t npages = 0, ndocs = 0, ntok = 0;
  int32_t max_len = 0, stride = 0;
  std::vector<int32_t> table;  // [ndocs][stride] page ids, kSlack more
  std::vector<int32_t> len;    // [ndocs] tokens
  std::vector<int32_t> more;   // [npages] documents that hold the page, beyond the first
  std::vector<int32_t> spare;  // free pages: the first `top` entries, the next one last
  int64_t top = 0, shared = 0;  // shared: sum of `more`
  std::vector<uint32_t> stamp;
  uint32_t epoch = 0;

  static int64_t pages_of(int64_t tokens) { return (tokens + kPageTokens - 1) / kPageTokens; }
  // Page ids are copied eight at a time, so that documents of a few pages take no
  // branch for each: rows of the table are whole eights, and what a copy reads or
  // writes beyond its n entries is nobody's.
  static int32_t row_pages(int32_t max_len) { return (int32_t)((pages_of(max_len) + 7) / 8 * 8); }
  static constexpr int kSlack = 8;
  static void copy8(int32_t *to, const int32_t *from, int64_t n) {
    for (int64_t i = 0; i < n; i += 8) std::memcpy(to + i, from + i, 32);
  }

  void init(int64_t npages_, int64_t ndocs_, int32_t max_len_) {
    npages = npages_;
    ndocs = ndocs_;
    max_len = max_len_;
    stride = row_pages(max_len);
    table.assign((size_t)ndocs * stride + kSlack, 0);
    len.assign((size_t)ndocs, 0);
    more.assign((size_t)npages, 0);
    stamp.assign((size_t)ndocs, 0);
    spare.assign((size_t)npages + kSlack, 0);
    for (int64_t i = 0; i < npages; ++i) spare[i] = (int32_t)(npages - 1 - i);  // lowest pages first
    top = npages;
  }

  int32_t *row(int64_t doc) { return table.data() + (size_t)doc * stride; }
  const int32_t *row(int64_t doc) const { return table.data() + (size_t)doc * stride; }

  // Marks every id; id where one is outside [0, ndocs), repeated (at: its place).
  BookError mark(const int64_t *ids, int64_t n, int64_t *at) {
    if (++epoch == 0) {
      stamp.assign(stamp.size(), 0);
      epoch = 1;
    }
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (ids[i] < 0 || ids[i] >= ndocs) return BookError::id;
      if (stamp[ids[i]] == epoch) return BookError::repeated;
      stamp[ids[i]] = epoch;
    }
    return BookError::none;
  }
  bool marked(int64_t id) const { return stamp[id] == epoch; }

  int64_t free_pages() const { return top; }
  // The next n free pages (there are as many).
  const int32_t *take(int64_t n) {
    top -= n;
    return spare.data() + top;
  }
  void release(int64_t doc) {
    const int32_t *r = row(doc);
    const int64_t n = pages_of(len[doc]);
    if (shared == 0) {
      copy8(spare.data() + top, r, n);
      top += n;
    } else {
      for (int64_t i = 0; i < n; ++i) {  // without a branch: shared or not is a coin's toss
        int32_t &m = more[r[i]];
        const bool last = m == 0;
        spare[top] = r[i];
        top += last;
        m -= !last;
        shared -= !last;
      }
    }
    ntok -= len[doc];
    len[doc] = 0;
  }

  // Every plan comes in two steps: a check that changes nothing and counts the
  // plan's items and page ids, and a commit that cannot fail and writes them (the
  // list of page ids has kSlack entries more).

  // ---- append: lens[i] tokens to the end of document ids[i]
  BookError check_append(const int64_t *ids, const int32_t *lens, int64_t n, int64_t *at, int64_t *items,
                         int64_t *pages) {
    if (BookError e = mark(ids, n, at); e != BookError::none) return e;
    int64_t fresh = 0;
    *items = *pages = 0;
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (lens[i] < 0) return BookError::length;
      const int64_t old = len[ids[i]], now = old + lens[i];
      if (now > max_len) return BookError::too_long;
      if (lens[i] == 0) continue;
      fresh += pages_of(now) - pages_of(old);
      const int64_t span = pages_of(now) - old / kPageTokens;
      *pages += span;
      *items += (span + kItemPages - 1) / kItemPages;
    }
    return fresh > free_pages() ? BookError::pages : BookError::none;
  }
  // row: first row of document i, i * doc_stride or, packed (0), behind document i - 1's.
  void commit_append(const int64_t *ids, const int32_t *lens, int64_t n, int64_t doc_stride, PageItem *item,
                     int32_t *page) {
    int64_t packed = 0;
    int32_t np = 0;
    for (int64_t i = 0; i < n; ++i) {
      int64_t r = doc_stride ? i * doc_stride : packed;
      packed += lens[i];
      if (lens[i] == 0) continue;
      const int64_t d = ids[i];
      int32_t *t = row(d);
      const int32_t old = len[d], now = old + lens[i];
      const int32_t p0 = old / kPageTokens;  // the first page written, there already if it is partly filled
      const int64_t fresh = pages_of(now) - pages_of(old);
      const int32_t *f = take(fresh);
      if (pages_of(old) + (fresh + 7) / 8 * 8 <= stride) copy8(t + pages_of(old), f, fresh);
      else std::memcpy(t + pages_of(old), f, (size_t)fresh * 4);
      copy8(page + np, t + p0, pages_of(now) - p0);
      for (int32_t p = p0, left = lens[i], fill = old % kPageTokens; left > 0; fill = 0) {
        const int32_t span = (int32_t)pages_of(fill + left);
        PageItem w;
        w.doc = (int32_t)d;
        w.first = p;
        w.npages = (uint8_t)(span < kItemPages ? span : kItemPages);
        w.pages = np;
        w.fill = (uint8_t)fill;
        w.ntok = (uint16_t)(left < w.npages * kPageTokens - fill ? left : w.npages * kPageTokens - fill);
        w.row = r;
        left -= w.ntok;
        r += w.ntok;
        if (left == 0) w.len = now;
        np += w.npages;
        p += w.npages;
        *item++ = w;
      }
      len[d] = now;
      ntok += lens[i];
    }
  }

  // ---- fork: document dst[i], empty until now, becomes the first lens[i] tokens of src[i]
  BookError check_fork(const int64_t *src, const int64_t *dst, const int32_t *lens, int64_t n, int64_t *at) {
    if (BookError e = mark(dst, n, at); e != BookError::none) return e;
    int64_t fresh = 0;
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (src[i] < 0 || src[i] >= ndocs) return BookError::id;
      if (len[dst[i]] != 0) return BookError::busy_dst;
      if (marked(src[i])) return BookError::src_is_dst;
      const int32_t l = lens ? lens[i] : len[src[i]];
      if (l < 0 || l > len[src[i]]) return BookError::length;
      fresh += l % kPageTokens != 0;
    }
    return fresh > free_pages() ? BookError::pages : BookError::none;
  }
  // An item a document: first = whole pages shared, ntok = tokens of the page
  // copied behind them, whose page is `pages` (itself, not a place in a list).
  void commit_fork(const int64_t *src, const int64_t *dst, const int32_t *lens, int64_t n, PageItem *item) {
    for (int64_t i = 0; i < n; ++i) {
      const int32_t l = lens ? lens[i] : len[src[i]];
      const int32_t *s = row(src[i]);
      int32_t *t = row(dst[i]);
      PageItem w;
      w.doc = (int32_t)dst[i];
      w.src = (int32_t)src[i];
      w.first = l / kPageTokens;
      w.ntok = (uint16_t)(l % kPageTokens);
      w.len = l;
      copy8(t, s, w.first);
      for (int32_t p = 0; p < w.first; ++p) ++more[s[p]];
      shared += w.first;
      if (w.ntok) w.pages = t[w.first] = *take(1);
      len[dst[i]] = l;
      ntok += l;
      item[i] = w;
    }
  }

  // ---- copy: document dst[i] of `to` becomes tokens pos (ascending; null: the
  // first lens[i]) of document src[i] of this store, in pages of its own.  dst[i]
  // is empty, or src[i] itself (compaction in place).  npos: positions in all;
  // turns: places where one document's follow another's without ascending
  // (take_positions completes the check).
  BookError check_copy(const int64_t *src, PageBook &to, const int64_t *dst, const int32_t *lens, const int32_t *pos,
                       int64_t n, int64_t *at, int64_t *items, int64_t *pages, int64_t *npos, int64_t *turns,
                       bool *in_place) {
    if (BookError e = to.mark(dst, n, at); e != BookError::none) return e;
    const bool same = &to == this;
    *items = *pages = *npos = *turns = 0;
    *in_place = false;
    // there are sum lens positions: as many as a document's length says only
    // where no other one is below zero, and else none is read (the call is refused)
    int32_t least = 0;
    for (int64_t i = 0; pos && i < n; ++i) least = lens[i] < least ? lens[i] : least;
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (src[i] < 0 || src[i] >= ndocs) return BookError::id;
      const bool self = same && src[i] == dst[i];
      if (!self && to.len[dst[i]] != 0) return BookError::busy_dst;
      if (same && !self && marked(src[i])) return BookError::src_is_dst;
      const int32_t have = len[src[i]], l = lens ? lens[i] : have;
      if (l < 0 || l > have) return BookError::length;
      if (l > to.max_len) return BookError::too_long;
      if (pos && l && least == 0) {
        const int32_t *q = pos + *npos;
        if (q[0] < 0 || q[l - 1] >= have) return BookError::position;
        *turns += *npos && q[0] <= q[-1];
        *npos += l;
      }
      *in_place |= self;
      *pages += pages_of(l);
      *items += l ? (pages_of(l) + kItemPages - 1) / kItemPages : self;
    }
    return *pages > to.free_pages() ? BookError::pages : BookError::none;
  }
  // The positions as the plan holds them, and whether they ascend but at `turns`
  // places: one pass without a branch for each document.
  template <class T>
  static bool take_positions(const int32_t *pos, int64_t npos, int64_t turns, T *out) {
    for (int64_t k = 0; k < npos;) {
      const int64_t stop = npos - k < 4096 ? npos : k + 4096;
      int32_t falls = 0;
      for (int64_t j = k ? k : 1; j < stop; ++j) falls += pos[j] <= pos[j - 1];
      turns -= falls;
      for (; k < stop; ++k) out[k] = (T)pos[k];
    }
    return turns == 0;
  }
  // The first document whose positions do not ascend.
  static int64_t falling(const int32_t *lens, const int32_t *pos, int64_t n) {
    int64_t k = 0;
    for (int64_t i = 0; i < n; ++i)
      for (const int64_t first = k, stop = k + lens[i]; k < stop; ++k)
        if (k > first && pos[k] <= pos[k - 1]) return i;
    return 0;
  }
  void commit_copy(const int64_t *src, PageBook &to, const int64_t *dst, const int32_t *lens, const int32_t *pos,
                   int64_t n, PageItem *item, int32_t *page) {
    // old pages of documents copied onto themselves are read by this plan: they
    // go back only after every new page is taken
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) all += pages_of(lens ? lens[i] : len[src[i]]);
    std::memcpy(page, to.take(all), (size_t)all * 4);
    int32_t np = 0;
    int64_t at = 0;
    for (int64_t i = 0; i < n; ++i) {
      const bool self = &to == this && src[i] == dst[i];
      const int32_t l = lens ? lens[i] : len[src[i]];
      const int32_t base = np;
      np += (int32_t)pages_of(l);
      if (self) release(src[i]);
      copy8(to.row(dst[i]), page + base, np - base);
      for (int32_t done = 0; done < l || (l == 0 && self);) {
        PageItem w;
        w.doc = (int32_t)dst[i];
        w.src = (int32_t)src[i];
        w.first = done / kPageTokens;
        w.ntok = (uint16_t)(l - done < kItemPages * kPageTokens ? l - done : kItemPages * kPageTokens);
        w.npages = (uint8_t)pages_of(w.ntok);
        w.pages = base + w.first;
        w.row = pos ? at + done : done;
        done += w.ntok;
        if (done == l) w.len = l;
        *item++ = w;
        if (l == 0) break;
      }
      at += l;
      to.len[dst[i]] = l;
      to.ntok += l;
    }
  }

  // ---- read: the tokens of ids[i], one document behind the other
  BookError count(const int64_t *ids, int64_t n, int64_t *at, int64_t *rows) const {
    int64_t sum = 0;
    for (int64_t i = 0; i < n; ++i) {
      if (ids[i] < 0 || ids[i] >= ndocs) {
        *at = i;
        return BookError::id;
      }
      sum += len[ids[i]];
    }
    *rows = sum;
    return BookError::none;
  }
  BookError check_read(const int64_t *ids, int64_t n, int64_t *at, int64_t *items, int64_t *rows) const {
    if (BookError e = count(ids, n, at, rows); e != BookError::none) return e;
    constexpr uint32_t kItemTokens = kItemPages * kPageTokens;
    int64_t sum = 0;
    for (int64_t i = 0; i < n; ++i) sum += (len[ids[i]] + kItemTokens - 1) / kItemTokens;
    *items = sum;
    return BookError::none;
  }
  void plan_read(const int64_t *ids, int64_t n, PageItem *item) const {
    int64_t r = 0;
    for (int64_t i = 0; i < n; ++i)
      for (int32_t done = 0, l = len[ids[i]]; done < l;) {
        PageItem w;
        w.doc = (int32_t)ids[i];
        w.first = done / kPageTokens;
        w.ntok = (uint16_t)(l - done < kItemPages * kPageTokens ? l - done : kItemPages * kPageTokens);
        w.npages = (uint8_t)pages_of(w.ntok);
        w.row = r;
        done += w.ntok;
        r += w.ntok;
        *item++ = w;
      }
  }
};

}  // namespace chimera
