// Host-side page bookkeeping for a paged KV cache shared by sequences that join and leave between
// steps (the serving setting of Sec. 4.3).  No device code: a free list of pages and one page
// list per slot.  Pages are handed out lowest index first from a stack of free pages, so that a
// test can predict them; nothing else depends on the order.  A page that forked slots share counts its
// holders and returns to the stack with the last of them.
#include "../../include/space.h"
#include <new>
#include <vector>

struct space_pager {
  int32_t n_pages, pages_per_seq, max_slots;
  std::vector<int32_t> free_pages;                 // stack: back() is handed out next
  std::vector<int32_t> table;                      // [max_slots][pages_per_seq], -1 = no page
  std::vector<int32_t> held;                       // pages a slot holds, -1 = slot not in use
  std::vector<int32_t> refs;                       // slots that hold a page, 0 = free
};

namespace {
bool slot_in_use(const space_pager* p, int32_t slot) {
  return slot >= 0 && slot < p->max_slots && p->held[slot] >= 0;
}
int32_t* row_of(space_pager* p, int32_t slot) { return p->table.data() + (size_t)slot * p->pages_per_seq; }
// (the stack never holds more than n_pages entries, which create has made room for: no push allocates)
int32_t take_page(space_pager* p) {
  const int32_t page = p->free_pages.back();
  p->free_pages.pop_back();
  p->refs[page] = 1;
  return page;
}
void drop_page(space_pager* p, int32_t page) {
  if (--p->refs[page] == 0) p->free_pages.push_back(page);
}
int64_t pages_for(int32_t n_rows) { return ((int64_t)n_rows + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE; }
}  // namespace

extern "C" {

int space_pager_create(int32_t n_pages, int32_t pages_per_seq, int32_t max_slots, space_pager** out) {
  if (!out || n_pages < 1 || pages_per_seq < 1 || max_slots < 1) return SPACE_E_INVALID_ARG;
  space_pager* p = new (std::nothrow) space_pager;
  if (!p) return SPACE_E_WORKSPACE;
  p->n_pages = n_pages; p->pages_per_seq = pages_per_seq; p->max_slots = max_slots;
  try {
    p->free_pages.resize(n_pages);
    for (int32_t i = 0; i < n_pages; ++i) p->free_pages[i] = n_pages - 1 - i;   // page 0 on top
    p->table.assign((size_t)max_slots * pages_per_seq, -1);
    p->held.assign(max_slots, -1);
    p->refs.assign(n_pages, 0);
  } catch (...) {                                          // no exception leaves a C entry
    delete p;
    return SPACE_E_WORKSPACE;
  }
  *out = p;
  return SPACE_OK;
}

void space_pager_destroy(space_pager* p) { delete p; }

int space_pager_admit(space_pager* p, int32_t* slot) {
  if (!p || !slot) return SPACE_E_INVALID_ARG;
  for (int32_t s = 0; s < p->max_slots; ++s) {
    if (p->held[s] < 0) { p->held[s] = 0; *slot = s; return SPACE_OK; }
  }
  return SPACE_E_WORKSPACE;
}

int space_pager_reserve(space_pager* p, int32_t slot, int32_t n_rows) {
  if (!p || !slot_in_use(p, slot) || n_rows < 0) return SPACE_E_INVALID_ARG;
  const int64_t want = pages_for(n_rows);
  if (want > p->pages_per_seq) return SPACE_E_INVALID_ARG;
  const int32_t have = p->held[slot];
  if (want <= have) return SPACE_OK;                               // pages are given back only by release
  if ((int64_t)p->free_pages.size() < want - have) return SPACE_E_WORKSPACE;
  for (int32_t j = have; j < (int32_t)want; ++j) row_of(p, slot)[j] = take_page(p);
  p->held[slot] = (int32_t)want;
  return SPACE_OK;
}

int space_pager_release(space_pager* p, int32_t slot) {
  if (!p || !slot_in_use(p, slot)) return SPACE_E_INVALID_ARG;
  space_pager_truncate(p, slot, 0);
  p->held[slot] = -1;
  return SPACE_OK;
}

int space_pager_truncate(space_pager* p, int32_t slot, int32_t n_rows) {
  if (!p || !slot_in_use(p, slot) || n_rows < 0) return SPACE_E_INVALID_ARG;
  const int64_t keep = pages_for(n_rows);
  int32_t* row = row_of(p, slot);
  while (p->held[slot] > keep) {
    int32_t& e = row[--p->held[slot]];
    drop_page(p, e);
    e = -1;
  }
  return SPACE_OK;
}

int space_pager_fork(space_pager* p, int32_t parent, int32_t n_rows, int32_t* slot) {
  if (!p || !slot || !slot_in_use(p, parent) || n_rows < 0) return SPACE_E_INVALID_ARG;
  const int64_t share = pages_for(n_rows);
  if (share > p->held[parent]) return SPACE_E_INVALID_ARG;
  int32_t child;
  const int rc = space_pager_admit(p, &child);
  if (rc != SPACE_OK) return rc;
  for (int32_t j = 0; j < (int32_t)share; ++j) {
    const int32_t page = row_of(p, parent)[j];
    row_of(p, child)[j] = page;
    ++p->refs[page];
  }
  p->held[child] = (int32_t)share;
  *slot = child;
  return SPACE_OK;
}

int space_pager_make_writable(space_pager* p, int32_t slot, int32_t first_row, int32_t n_rows, space_page_move* moves,
                              int32_t max_moves, int32_t* n_moves) {
  if (!p || !n_moves || !slot_in_use(p, slot) || first_row < 0 || n_rows < 0 || max_moves < 0 || (max_moves > 0 && !moves))
    return SPACE_E_INVALID_ARG;
  *n_moves = 0;
  if (n_rows == 0) return SPACE_OK;
  const int64_t end = (int64_t)first_row + n_rows;
  const int64_t j1 = (end + SPACE_PAGE_SIZE - 1) / SPACE_PAGE_SIZE;
  if (j1 > p->held[slot]) return SPACE_E_INVALID_ARG;
  const int32_t j0 = first_row / SPACE_PAGE_SIZE, kept = first_row % SPACE_PAGE_SIZE;
  int32_t* row = row_of(p, slot);
  int64_t fresh = 0;
  for (int32_t j = j0; j < (int32_t)j1; ++j) fresh += p->refs[row[j]] > 1;
  if (fresh > (int64_t)p->free_pages.size()) return SPACE_E_WORKSPACE;
  const bool move = kept > 0 && p->refs[row[j0]] > 1;      // only the first page holds rows that are kept
  if (move && max_moves < 1) return SPACE_E_WORKSPACE;
  for (int32_t j = j0; j < (int32_t)j1; ++j) {
    if (p->refs[row[j]] <= 1) continue;
    const int32_t old = row[j];
    row[j] = take_page(p);
    drop_page(p, old);
    if (j == j0 && move) { moves[0].src = old; moves[0].dst = row[j]; moves[0].rows = kept; *n_moves = 1; }
  }
  return SPACE_OK;
}

int space_pager_compact(space_pager* p, space_page_move* moves, int32_t max_moves, int32_t* n_moves) {
  if (!p || !n_moves || max_moves < 0 || (max_moves > 0 && !moves)) return SPACE_E_INVALID_ARG;
  *n_moves = 0;
  // the lowest free page and the highest one in use, towards each other: a page read is never one written
  int32_t lo = 0, hi = p->n_pages - 1, n = 0;
  while (n < max_moves) {
    while (lo < hi && p->refs[lo] > 0) ++lo;
    while (lo < hi && p->refs[hi] == 0) --hi;
    if (lo >= hi) break;
    moves[n].src = hi; moves[n].dst = lo; moves[n].rows = SPACE_PAGE_SIZE;
    ++n; ++lo; --hi;
  }
  if (n == 0) return SPACE_OK;
  // moves are in descending order of src: a table entry finds its move by halving
  for (int32_t s = 0; s < p->max_slots; ++s) {
    for (int32_t j = 0; j < p->held[s]; ++j) {
      int32_t& e = row_of(p, s)[j];
      if (e < moves[n - 1].src) continue;
      int32_t a = 0, b = n - 1;
      while (a < b) {
        const int32_t m = (a + b) / 2;
        if (moves[m].src > e) a = m + 1; else b = m;
      }
      if (moves[a].src == e) e = moves[a].dst;
    }
  }
  for (int32_t i = 0; i < n; ++i) { p->refs[moves[i].dst] = p->refs[moves[i].src]; p->refs[moves[i].src] = 0; }
  p->free_pages.clear();
  for (int32_t i = p->n_pages - 1; i >= 0; --i)
    if (p->refs[i] == 0) p->free_pages.push_back(i);        // the lowest on top again
  *n_moves = n;
  return SPACE_OK;
}

int32_t space_pager_page_refs(const space_pager* p, int32_t page) {
  return p && page >= 0 && page < p->n_pages ? p->refs[page] : -1;
}

int32_t space_pager_free_pages(const space_pager* p) { return p ? (int32_t)p->free_pages.size() : -1; }

int32_t space_pager_rows(const space_pager* p, int32_t slot) {
  if (!p || !slot_in_use(p, slot)) return -1;
  return p->held[slot] * SPACE_PAGE_SIZE;
}

int space_pager_batch_table(const space_pager* p, const int32_t* slots, int32_t n, int32_t* table_out) {
  if (!p || n < 0 || (n > 0 && (!slots || !table_out))) return SPACE_E_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i)
    if (!slot_in_use(p, slots[i])) return SPACE_E_INVALID_ARG;
  for (int32_t i = 0; i < n; ++i)
    for (int32_t j = 0; j < p->pages_per_seq; ++j)
      table_out[(size_t)i * p->pages_per_seq + j] = p->table[(size_t)slots[i] * p->pages_per_seq + j];
  return SPACE_OK;
}

}  // extern "C"
