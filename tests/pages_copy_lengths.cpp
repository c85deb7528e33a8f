// Copies by position whose lengths are out of range: refused before a position
// behind those that the lengths promise is looked at.  Such a position is marked
// here by a value that is out of range itself, in memory that is there, so a
// check that looks at it answers with the wrong refusal.  Prints "ok" or what
// went wrong.
#include <cstdio>
#include <vector>

#include "../paper_2608_23553_amd/csrc/pages_book.h"

using namespace chimera;

static int failed = 0;

static void expect(const char *name, BookError want, std::vector<int64_t> src, std::vector<int32_t> lens,
                   std::vector<int32_t> given, int64_t want_at) {
  PageBook book;
  book.init(300, 8, 1100);
  const int64_t ids[2] = {0, 1}, dst[4] = {4, 5, 6, 7};
  const int32_t have[2] = {1000, 20};
  int64_t at = -1, items = 0, pages = 0, npos = 0, turns = 0;
  bool in_place = false;
  std::vector<PageItem> item(16);
  std::vector<int32_t> page(100 + PageBook::kSlack);
  if (book.check_append(ids, have, 2, &at, &items, &pages) != BookError::none) failed = 1;
  book.commit_append(ids, have, 2, 0, item.data(), page.data());
  std::vector<int32_t> pos(4000, 1 << 20);  // behind what is given: no document's position
  for (size_t i = 0; i < given.size(); ++i) pos[1000 + i] = given[i];
  const int64_t free_pages = book.free_pages(), ntok = book.ntok;
  const BookError e = book.check_copy(src.data(), book, dst, lens.data(), pos.data() + 1000, (int64_t)src.size(), &at,
                                      &items, &pages, &npos, &turns, &in_place);
  if (e != want || at != want_at || book.free_pages() != free_pages || book.ntok != ntok) {
    std::printf("%s: error %d at entry %lld, not %d at %lld\n", name, (int)e, (long long)at, (int)want,
                (long long)want_at);
    failed = 1;
  }
}

int main() {
  expect("a length below zero behind a long one", BookError::length, {0, 0}, {1000, -999}, {0}, 1);
  expect("and between two", BookError::length, {0, 1, 0}, {500, -499, 1}, {0, 1}, 1);
  expect("first", BookError::length, {1, 0}, {-3, 4}, {5}, 0);
  expect("the lowest there is", BookError::length, {1, 1, 1}, {20, -2147483647 - 1, 20}, {}, 1);
  expect("a length above the document's", BookError::length, {1, 1}, {21, 0}, {}, 0);
  expect("behind sound ones", BookError::length, {1, 0, 1}, {2, 0, 21}, {3, 4}, 2);
  expect("no such document", BookError::id, {1, 9, 0}, {2, 5, -7}, {}, 1);
  expect("sound lengths, a position out of range", BookError::position, {1, 1}, {2, 1}, {3, 4, 20}, 1);
  expect("sound", BookError::none, {1, 0, 1}, {2, 1, 1}, {0, 19, 999, 5}, 2);
  if (!failed) std::printf("ok\n");
  return failed;
}
