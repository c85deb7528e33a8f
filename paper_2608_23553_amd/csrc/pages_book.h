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
  int32_t npages = 0;
  int32_t pages = 0;    // position of their page ids in the plan's list
  int32_t fill = 0;     // tokens that the first page holds already
  int32_t ntok = 0;     // tokens to write (read) from there
  int32_t len = -1;     // the document's length after the call; -1: another item sets it
  int32_t src = 0;      // copy, fork: the document read
  int64_t row = 0;      // append, read: first row of the tensor; copy: first position in the plan's list, or first token
};

// What the caller asked for that cannot be done (see the messages in pages.cpp).
enum class BookError { none, id, repeated, length, too_long, busy_dst, src_is_dst, pages, position };

struct PageBook {
  int64_t npages = 0, ndocs = 0, ntok = 0;
  int32_t max_len = 0, stride = 0;
  std::vector<int32_t> table;  // [ndocs][stride] page ids
  std::vector<int32_t> len;    // [ndocs] tokens
  std::vector<int32_t> ref;    // [npages] documents that hold the page
  std::vector<int32_t> spare;  // free pages, the next one last; never grows past npages
  std::vector<uint32_t> stamp;
  uint32_t epoch = 0;

  static int64_t pages_of(int64_t tokens) { return (tokens + kPageTokens - 1) / kPageTokens; }

  void init(int64_t npages_, int64_t ndocs_, int32_t max_len_) {
    npages = npages_;
    ndocs = ndocs_;
    max_len = max_len_;
    stride = (int32_t)pages_of(max_len);
    table.assign((size_t)ndocs * stride, 0);
    len.assign((size_t)ndocs, 0);
    ref.assign((size_t)npages, 0);
    stamp.assign((size_t)ndocs, 0);
    spare.resize((size_t)npages);
    for (int64_t i = 0; i < npages; ++i) spare[i] = (int32_t)(npages - 1 - i);  // lowest page first
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

  int32_t take() {
    const int32_t p = spare.back();
    spare.pop_back();
    ref[p] = 1;
    return p;
  }
  void release(int64_t doc) {
    const int32_t *r = row(doc);
    for (int64_t i = 0, n = pages_of(len[doc]); i < n; ++i)
      if (--ref[r[i]] == 0) spare.push_back(r[i]);
    ntok -= len[doc];
    len[doc] = 0;
  }

  // Every plan comes in two steps: a check that changes nothing and counts the
  // plan's items and page ids, and a commit that cannot fail and writes them.

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
    return fresh > (int64_t)spare.size() ? BookError::pages : BookError::none;
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
      for (int64_t p = pages_of(old); p < pages_of(now); ++p) t[p] = take();
      for (int32_t p = old / kPageTokens, left = lens[i], fill = old % kPageTokens; left > 0; fill = 0) {
        PageItem w;
        w.doc = (int32_t)d;
        w.first = p;
        w.npages = (int32_t)pages_of(fill + left) < kItemPages ? (int32_t)pages_of(fill + left) : kItemPages;
        w.pages = np;
        w.fill = fill;
        w.ntok = left < w.npages * kPageTokens - fill ? left : w.npages * kPageTokens - fill;
        w.row = r;
        left -= w.ntok;
        r += w.ntok;
        if (left == 0) w.len = now;
        for (int k = 0; k < w.npages; ++k) page[np++] = t[p + k];
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
    return fresh > (int64_t)spare.size() ? BookError::pages : BookError::none;
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
      w.ntok = l % kPageTokens;
      w.len = l;
      for (int32_t p = 0; p < w.first; ++p) {
        t[p] = s[p];
        ++ref[s[p]];
      }
      if (w.ntok) w.pages = t[w.first] = take();
      len[dst[i]] = l;
      ntok += l;
      item[i] = w;
    }
  }

  // ---- copy: document dst[i] of `to` becomes tokens pos (ascending; null: the
  // first lens[i]) of document src[i] of this store, in pages of its own.  dst[i]
  // is empty, or src[i] itself (compaction in place).
  BookError check_copy(const int64_t *src, PageBook &to, const int64_t *dst, const int32_t *lens, const int32_t *pos,
                       int64_t n, int64_t *at, int64_t *items, int64_t *pages, bool *in_place) {
    if (BookError e = to.mark(dst, n, at); e != BookError::none) return e;
    const bool same = &to == this;
    *items = *pages = 0;
    *in_place = false;
    const int32_t *q = pos;
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (src[i] < 0 || src[i] >= ndocs) return BookError::id;
      const bool self = same && src[i] == dst[i];
      if (!self && to.len[dst[i]] != 0) return BookError::busy_dst;
      if (same && !self && marked(src[i])) return BookError::src_is_dst;
      const int32_t have = len[src[i]], l = lens ? lens[i] : have;
      if (l < 0 || l > have) return BookError::length;
      if (l > to.max_len) return BookError::too_long;
      if (pos) {
        int32_t before = -1;
        for (int32_t k = 0; k < l; ++k, ++q) {
          if (*q <= before || *q >= have) return BookError::position;
          before = *q;
        }
      }
      *in_place |= self;
      *pages += pages_of(l);
      *items += l ? (pages_of(l) + kItemPages - 1) / kItemPages : self;
    }
    return *pages > (int64_t)to.spare.size() ? BookError::pages : BookError::none;
  }
  void commit_copy(const int64_t *src, PageBook &to, const int64_t *dst, const int32_t *lens, const int32_t *pos,
                   int64_t n, PageItem *item, int32_t *page) {
    // old pages of documents copied onto themselves are read by this plan: they
    // go back only after every new page is taken
    int32_t np = 0;
    for (int64_t i = 0; i < n; ++i)
      for (int64_t p = pages_of(lens ? lens[i] : len[src[i]]); p > 0; --p) page[np++] = to.take();
    int64_t at = 0;
    np = 0;
    for (int64_t i = 0; i < n; ++i) {
      const bool self = &to == this && src[i] == dst[i];
      const int32_t l = lens ? lens[i] : len[src[i]];
      const int32_t base = np;
      np += (int32_t)pages_of(l);
      if (self) release(src[i]);
      int32_t *t = to.row(dst[i]);
      for (int32_t p = 0; p < np - base; ++p) t[p] = page[base + p];
      for (int32_t done = 0; done < l || (l == 0 && self);) {
        PageItem w;
        w.doc = (int32_t)dst[i];
        w.src = (int32_t)src[i];
        w.first = done / kPageTokens;
        w.ntok = l - done < kItemPages * kPageTokens ? l - done : kItemPages * kPageTokens;
        w.npages = (int32_t)pages_of(w.ntok);
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
  BookError check_read(const int64_t *ids, int64_t n, int64_t *at, int64_t *items, int64_t *rows) const {
    *items = *rows = 0;
    for (int64_t i = 0; i < n; ++i) {
      *at = i;
      if (ids[i] < 0 || ids[i] >= ndocs) return BookError::id;
      *items += (pages_of(len[ids[i]]) + kItemPages - 1) / kItemPages;
      *rows += len[ids[i]];
    }
    return BookError::none;
  }
  void plan_read(const int64_t *ids, int64_t n, PageItem *item) const {
    int64_t r = 0;
    for (int64_t i = 0; i < n; ++i)
      for (int32_t done = 0, l = len[ids[i]]; done < l;) {
        PageItem w;
        w.doc = (int32_t)ids[i];
        w.first = done / kPageTokens;
        w.ntok = l - done < kItemPages * kPageTokens ? l - done : kItemPages * kPageTokens;
        w.npages = (int32_t)pages_of(w.ntok);
        w.row = r;
        done += w.ntok;
        r += w.ntok;
        *item++ = w;
      }
  }
};

}  // namespace chimera
