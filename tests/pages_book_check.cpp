// Random calls on the paged store's host bookkeeping, its plans carried out on
// an array as the kernels carry them out on the device, against documents kept
// as plain lists of numbers.  Prints "ok" or what went wrong.
#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../paper_2608_23553_amd/csrc/pages_book.h"

using namespace chimera;
typedef std::vector<int64_t> Ids;
typedef std::vector<int32_t> Lens;

#define CHECK(c)                                             \
  do {                                                       \
    if (!(c)) {                                              \
      std::printf("line %d: %s\n", __LINE__, #c);            \
      std::exit(1);                                          \
    }                                                        \
  } while (0)

constexpr int FREE = -1;

static int64_t bad_entry = 0;  // of the next call whose positions do not ascend

struct Store {
  PageBook book;
  std::vector<int> pool;                // [npages][16] token numbers, FREE where the scale is NaN
  std::vector<int32_t> table, len;      // the device's copies
  std::vector<std::vector<int>> plain;  // what each document holds

  Store(int64_t npages, int64_t ndocs, int32_t max_len) {
    book.init(npages, ndocs, max_len);
    pool.assign((size_t)npages * 16, 12345);
    table.assign((size_t)ndocs * book.stride, -7);
    len.assign((size_t)ndocs, 0);
    plain.resize((size_t)ndocs);
  }

  void check() const {
    std::vector<int> ref(book.npages, 0);
    int64_t ntok = 0;
    for (int64_t d = 0; d < book.ndocs; ++d) {
      CHECK(len[d] == (int)plain[d].size() && book.len[d] == len[d]);
      ntok += len[d];
      for (int64_t p = 0; p < PageBook::pages_of(len[d]); ++p) {
        const int32_t id = table[d * book.stride + p];
        CHECK(id >= 0 && id < book.npages && id == book.row(d)[p]);
        ++ref[id];
        for (int t = 0; t < 16; ++t)
          CHECK(pool[(size_t)id * 16 + t] == (p * 16 + t < len[d] ? plain[d][p * 16 + t] : FREE));
      }
    }
    CHECK(ntok == book.ntok);
    int64_t spare = 0, more = 0;
    for (int64_t p = 0; p < book.npages; ++p) {
      CHECK((ref[p] ? ref[p] - 1 : 0) == book.more[p]);
      spare += ref[p] == 0;
      more += book.more[p];
    }
    std::vector<int32_t> f(book.spare.begin(), book.spare.begin() + book.top);
    std::sort(f.begin(), f.end());
    CHECK(more == book.shared && (int64_t)f.size() == spare && std::unique(f.begin(), f.end()) == f.end());
    for (int32_t p : f) CHECK(ref[p] == 0);
  }

  BookError append(const Ids &ids, const Lens &lens, int64_t stride, int &next) {
    int64_t at, ni, np;
    if (BookError e = book.check_append(ids.data(), lens.data(), ids.size(), &at, &ni, &np); e != BookError::none)
      return e;
    std::vector<PageItem> it(ni + 1);
    Lens page(np + PageBook::kSlack);
    it[ni].doc = -99;
    std::vector<int> rows;  // the tensor
    for (size_t i = 0; i < ids.size(); ++i) {
      if (stride) rows.resize(i * stride, -2);
      for (int k = 0; k < lens[i]; ++k) {
        rows.push_back(next);
        plain[ids[i]].push_back(next++);
      }
    }
      book.commit_append(ids.data(), lens.data(), ids.size(), stride, it.data(), page.data());
    CHECK(it[ni].doc == -99);
    for (int64_t j = 0; j < ni; ++j) {
      const PageItem &w = it[j];
      CHECK(w.npages >= 1 && w.npages <= kItemPages && w.ntok >= 1 && w.pages + w.npages <= np);
      for (int p = 0; p < w.npages; ++p) {
        const int32_t id = page[w.pages + p];
        for (int t = 0; t < 16; ++t) {
          const int i = p * 16 + t - w.fill;
          int &slot = pool[(size_t)id * 16 + t];
          if (i >= 0 && i < w.ntok) slot = rows.at(w.row + i);
          else if (i >= w.ntok) slot = FREE;
        }
        table[(size_t)w.doc * book.stride + w.first + p] = id;
      }
      if (w.len >= 0) len[w.doc] = w.len;
    }
    return BookError::none;
  }

  BookError fork(const Ids &src, const Ids &dst, const Lens *lens) {
    int64_t at;
    const int32_t *l = lens ? lens->data() : nullptr;
    if (BookError e = book.check_fork(src.data(), dst.data(), l, src.size(), &at); e != BookError::none) return e;
    for (size_t i = 0; i < src.size(); ++i) {
      plain[dst[i]] = plain[src[i]];
      if (lens) plain[dst[i]].resize((*lens)[i]);
    }
    std::vector<PageItem> it(src.size());
    book.commit_fork(src.data(), dst.data(), l, src.size(), it.data());
    for (const PageItem &w : it) {
      const int32_t *s = &table[(size_t)w.src * book.stride];
      int32_t *d = &table[(size_t)w.doc * book.stride];
      for (int p = 0; p < w.first; ++p) d[p] = s[p];
      if (w.ntok) {
        for (int t = 0; t < 16; ++t)
          pool[(size_t)w.pages * 16 + t] = t < w.ntok ? pool[(size_t)s[w.first] * 16 + t] : FREE;
        d[w.first] = w.pages;
      }
      len[w.doc] = w.len;
    }
    return BookError::none;
  }

  BookError copy(const Ids &src, Store &to, const Ids &dst, const Lens *lens, const Lens *pos) {
    int64_t at, ni, np, npos, turns;
    bool in_place;
    const int32_t *l = lens ? lens->data() : nullptr, *q = pos ? pos->data() : nullptr;
    if (BookError e = book.check_copy(src.data(), to.book, dst.data(), l, q, src.size(), &at, &ni, &np, &npos, &turns,
                                      &in_place);
        e != BookError::none)
      return e;
    if (q) {
      std::vector<uint16_t> taken(npos);
      if (!PageBook::take_positions(q, npos, turns, taken.data())) {
        CHECK(PageBook::falling(l, q, src.size()) == bad_entry);
        return BookError::position;
      }
      CHECK(std::equal(taken.begin(), taken.end(), q));
    }
    std::vector<std::vector<int>> made;
    for (size_t i = 0, k = 0; i < src.size(); ++i) {
      const std::vector<int> &s = plain[src[i]];
      std::vector<int> v;
      for (int j = 0, n = l ? l[i] : (int)s.size(); j < n; ++j) v.push_back(s[q ? q[k++] : j]);
      made.push_back(v);
    }
    for (size_t i = 0; i < src.size(); ++i) to.plain[dst[i]] = made[i];
    std::vector<PageItem> it(ni + 1);
    Lens page(np + PageBook::kSlack);
    it[ni].doc = -99;
    book.commit_copy(src.data(), to.book, dst.data(), l, q, src.size(), it.data(), page.data());
    CHECK(it[ni].doc == -99);
    // every write before any read would show a page that is both; so do the items backwards too
    const std::vector<int> old = pool;
    for (int64_t j = ni - 1; j >= 0; --j) {
      const PageItem &w = it[j];
      for (int p = 0; p < w.npages; ++p)
        for (int t = 0; t < 16; ++t) {
          const int i = p * 16 + t;
          int v = FREE;
          if (i < w.ntok) {
            const int a = q ? q[w.row + i] : (int)w.row + i;
            const size_t slot = (size_t)table[(size_t)w.src * book.stride + a / 16] * 16 + a % 16;
            CHECK(pool[slot] == old[slot]);
            v = pool[slot];
          }
          to.pool[(size_t)page[w.pages + p] * 16 + t] = v;
        }
    }
    for (int64_t j = 0; j < ni; ++j) {
      const PageItem &w = it[j];
      for (int p = 0; p < w.npages; ++p) to.table[(size_t)w.doc * to.book.stride + w.first + p] = page[w.pages + p];
      if (w.len >= 0) to.len[w.doc] = w.len;
    }
    return BookError::none;
  }

  void drop(const Ids &ids) {
    for (int64_t d : ids) {
      book.release(d);
      len[d] = 0;
      plain[d].clear();
    }
  }

  void read(const Ids &ids) const {
    int64_t at, ni, rows;
    CHECK(book.check_read(ids.data(), ids.size(), &at, &ni, &rows) == BookError::none);
    std::vector<PageItem> it(ni);
    book.plan_read(ids.data(), ids.size(), it.data());
    std::vector<int> want, got(rows, -5);
    for (int64_t d : ids) want.insert(want.end(), plain[d].begin(), plain[d].end());
    for (const PageItem &w : it)
      for (int i = 0; i < w.ntok; ++i)
        got.at(w.row + i) = pool[(size_t)table[(size_t)w.doc * book.stride + w.first + i / 16] * 16 + i % 16];
    CHECK(got == want);
  }
};

static void random_calls(unsigned seed, int64_t npages, int64_t ndocs, int32_t max_len, int calls) {
  std::mt19937 g(seed);
  auto rnd = [&](int lo, int hi) { return (int)(lo + g() % (unsigned)(hi - lo + 1)); };
  Store a(npages, ndocs, max_len), b(npages / 2 + 1, ndocs, max_len);
  int next = 0, done[6] = {0};
  for (int c = 0; c < calls; ++c) {
    Ids all((size_t)ndocs);
    for (int64_t i = 0; i < ndocs; ++i) all[i] = i;
    std::shuffle(all.begin(), all.end(), g);
    const int n = rnd(0, (int)std::min<int64_t>(ndocs, 6));
    Ids ids(all.begin(), all.begin() + n);
    auto any = [&] { Ids v; for (int i = 0; i < n; ++i) v.push_back(rnd(0, (int)ndocs - 1)); return v; };
    Store &s = rnd(0, 3) ? a : b;
    BookError e = BookError::none;
    const int what = rnd(0, 5);
    if (what == 0) {
      Lens l;
      int longest = 0;
      for (int i = 0; i < n; ++i) {
        l.push_back(rnd(0, 2) ? rnd(0, 40) : rnd(0, max_len));
        longest = std::max(longest, l.back());
      }
      e = s.append(ids, l, rnd(0, 1) ? 0 : longest + rnd(0, 9), next);
    } else if (what == 1) {
      const Ids src = any();
      Lens l;
      for (int64_t d : src) l.push_back(rnd(0, s.book.len[d]));
      e = s.fork(src, ids, rnd(0, 1) ? &l : nullptr);
    } else if (what == 2 || what == 3) {
      Store &to = rnd(0, 1) ? s : (&s == &a ? b : a);
      const bool self = what == 3 && &to == &s;
      const Ids src = self ? ids : any();
      Lens l, pos;
      const bool some = rnd(0, 1);
      for (int64_t d : src) {
        int kept = 0;
        for (int t = 0; t < s.book.len[d]; ++t)
          if (rnd(0, 2)) pos.push_back(t), ++kept;
        l.push_back(some ? kept : rnd(0, s.book.len[d]));
      }
      e = s.copy(src, to, ids, &l, some ? &pos : nullptr);
    } else if (what == 4) {
      s.drop(any());
    } else {
      s.read(any());
    }
    done[what] += e == BookError::none;
    a.check();
    b.check();
  }
  for (int i = 0; i < 6; ++i) CHECK(done[i] > calls / 60);
}

static void refusals() {
  Store s(6, 4, 50);
  int next = 0;
  auto append = [&](Ids i, Lens l) { return s.append(i, l, 0, next); };
  CHECK(append({4}, {1}) == BookError::id && append({-1}, {1}) == BookError::id);
  CHECK(append({1, 2, 1}, {1, 1, 1}) == BookError::repeated);
  CHECK(append({0}, {-1}) == BookError::length && append({0}, {51}) == BookError::too_long);
  CHECK(append({0, 1, 2}, {50, 33, 1}) == BookError::pages);  // 4 + 3 + 1 pages of 6
  CHECK(append({0}, {33}) == BookError::none && append({0}, {18}) == BookError::too_long);
  const Lens l34{34}, l20{20}, l51{2, 5, 1}, l2{2}, back{5, 5}, down{6, 5}, far{32, 33};
  CHECK(s.fork({0}, {0}, nullptr) == BookError::busy_dst && s.fork({0}, {1}, &l34) == BookError::length);
  CHECK(s.fork({0, 0}, {1, 1}, nullptr) == BookError::repeated && s.fork({4}, {1}, nullptr) == BookError::id);
  CHECK(s.fork({0, 1}, {1, 2}, nullptr) == BookError::src_is_dst);
  CHECK(s.fork({0, 0}, {1, 2}, nullptr) == BookError::none);  // two pages shared by three, a third each
  CHECK(s.book.free_pages() == 1);
  CHECK(s.copy({1}, s, {3}, nullptr, nullptr) == BookError::pages);
  CHECK(s.copy({1}, s, {3}, &l2, &back) == BookError::position);
  CHECK(s.copy({1}, s, {3}, &l2, &down) == BookError::position);
  const Lens l23{2, 3}, second{7, 9, 0, 4, 4}, turn{7, 9, 0, 4, 5};
  bad_entry = 1;
  CHECK(s.copy({1, 2}, s, {3, 0}, &l23, &second) != BookError::none);
  s.drop({0});
  CHECK(s.copy({1, 2}, s, {3, 0}, &l23, &second) == BookError::position);
  CHECK(s.copy({1, 2}, s, {3, 0}, &l23, &turn) == BookError::none);
  s.check();
  s.drop({0, 3});
  CHECK(s.fork({1}, {0}, nullptr) == BookError::none);
  CHECK(s.copy({1}, s, {3}, &l2, &far) == BookError::position);
  CHECK(s.copy({0}, s, {1}, &l20, nullptr) == BookError::busy_dst);
  CHECK(s.copy({0, 0}, s, {0, 3}, &l51, nullptr) == BookError::src_is_dst);
  s.check();
  CHECK(s.copy({0}, s, {0}, &l2, nullptr) == BookError::none && s.book.free_pages() == 1);
  s.check();
  s.drop({0, 1, 1, 2});
  s.check();
  CHECK(s.book.free_pages() == 6 && s.book.ntok == 0);
}

int main() {
  refusals();
  random_calls(1, 40, 9, 70, 4000);
  random_calls(2, 400, 23, 1100, 1500);   // documents of more than one work item
  random_calls(3, 12, 30, 16, 3000);      // one page a document
  random_calls(4, 9, 5, 33, 3000);        // mostly out of pages
  std::printf("ok\n");
}
