// Which pages of a pool the sequences have: lists of pages, lengths, and how many sequences have each page.  Host code only.
//
// A sequence of n rows has ceil(n / page rows) pages, in order; its row i is row i mod page rows of page i / page rows.  Sequences
// may share pages (a fork), but rows are only written to pages that one sequence has: extending a sequence whose last page is
// shared gives it a copy of that page's rows.  The lowest free page is taken first, so the same calls give the same lists.
//
// Every call checks, then reserves what it will report, then changes the lists: an error leaves them as they were.  What it
// reports is what has to be done on the device: runs of entries of the table, pages to copy, rows to move.
#pragma once

#include <stdint.h>

#include <string>
#include <vector>

namespace fsx {

// Entries at .. at + count - 1 of a sequence's list: pages first, first + 1, ..; or, where first < 0, the same entries of sequence
// ~first.  And the sequence's length.
struct PageRun {
  int32_t seq, at, first, count, len;
};
// The first `rows` rows of page `to` become those of page `from`.
struct PageCopy {
  int32_t from, to, rows;
};
// Rows first .. first + count - 1 of a sequence, which stay.
struct PageRange {
  int32_t first, count;
};
// Ranges range .. range + n_ranges - 1 close up; rows `start` .. rows - 1 of the outcome are written, from a page's first row on.
struct PageMove {
  int32_t seq, range, n_ranges, start, rows;
};

class PageLists {
 public:
  enum { OK = 0, BAD = 1, FULL = 3 };  // as fsx_status

  const int32_t n_pages, max_seqs, most, P;  // most: pages of a sequence
  std::vector<int32_t> table, len, ref;
  int64_t n_free;
  std::string error;

  // What a call reports.
  std::vector<PageRun> runs;    // (keep: after the rows have moved)
  std::vector<PageRun> before;  // keep: the lists that rows move to, into a second table, where some page is replaced
  std::vector<PageCopy> copies;
  std::vector<PageRange> ranges;
  std::vector<PageMove> moves;

  PageLists(int32_t pages, int32_t seqs, int32_t seq_pages, int32_t page_rows)
      : n_pages(pages), max_seqs(seqs), most(seq_pages), P(page_rows), table((size_t)seqs * seq_pages, -1), len(seqs, 0),
        ref(pages, 0), n_free(pages), free_((pages + 63) / 64, ~0ull), named_(seqs, 0) {
    if (pages % 64) free_.back() = (1ull << pages % 64) - 1;
  }

  int pages_of(int64_t rows) const { return (int)((rows + P - 1) / P); }

  // Sequences 0 .. max_seqs - 1, none twice.
  int check(int n, const int32_t* seqs) {
    for (int i = 0; i < n; ++i)
      if (seqs[i] < 0 || seqs[i] >= max_seqs) return fail(BAD, "sequence " + std::to_string(seqs[i]) + " outside 0..max_seqs-1");
    int twice = -1;
    for (int i = 0; i < n; ++i) {
      if (named_[seqs[i]]) twice = seqs[i];
      named_[seqs[i]] = 1;
    }
    for (int i = 0; i < n; ++i) named_[seqs[i]] = 0;
    return twice < 0 ? (int)OK : fail(BAD, "sequence " + std::to_string(twice) + " is named twice");
  }

  int extend(int n, const int32_t* seqs, const int32_t* rows) {
    if (int rc = begin(n, seqs)) return rc;
    int64_t need = 0, n_copies = 0;
    for (int i = 0; i < n; ++i) {
      if (rows[i] < 0) return fail(BAD, "rows " + std::to_string(i) + " are negative");
      const int64_t now = (int64_t)len[seqs[i]] + rows[i];
      if (now > (int64_t)most * P)
        return fail(FULL, "sequence " + std::to_string(seqs[i]) + " would pass its " + std::to_string(most) + " pages");
      need += pages_of(now) - pages_of(len[seqs[i]]);
    }
    // the sharers that need a copy: each leaves the page to one less, so the last of them may keep it
    std::vector<char> copy(n);
    for (int i = 0; i < n; ++i) {
      const int32_t s = seqs[i];
      if (!rows[i] || len[s] % P == 0) continue;
      int32_t& r = ref[last(s)];
      if (r > 1) copy[i] = 1, ++n_copies, --r;
    }
    const auto undo = [&] {
      for (int i = 0; i < n; ++i)
        if (copy[i]) ++ref[last(seqs[i])];
    };
    need += n_copies;
    if (need > n_free) {
      undo();
      return fail(FULL, std::to_string(need) + " pages are needed, " + std::to_string(n_free) + " are free");
    }
    try {
      runs.reserve(n + need);
      copies.reserve(n_copies);
    } catch (...) {
      undo();
      throw;
    }
    for (int i = 0; i < n; ++i) {
      const int32_t s = seqs[i], had = pages_of(len[s]), now = len[s] + rows[i];
      if (!rows[i]) continue;
      int32_t* t = &table[(size_t)s * most];
      const int at = had - copy[i];
      if (copy[i]) {
        const int32_t p = take();
        copies.push_back({t[at], p, len[s] % P});
        t[at] = p;
      }
      for (int j = had; j < pages_of(now); ++j) t[j] = take();
      len[s] = now;
      list(runs, s, at, pages_of(now), t);
    }
    return OK;
  }

  // dst[i], which has no rows, gets the first rows[i] (rows NULL: all) of src[i].
  int fork(int n, const int32_t* src, const int32_t* dst, const int32_t* rows) {
    if (int rc = begin(n, dst)) return rc;
    for (int i = 0; i < n; ++i) {
      if (src[i] < 0 || src[i] >= max_seqs) return fail(BAD, "sequence " + std::to_string(src[i]) + " outside 0..max_seqs-1");
      if (len[dst[i]]) return fail(BAD, "sequence " + std::to_string(dst[i]) + " has rows: free it first");
      if (rows && (rows[i] < 0 || rows[i] > len[src[i]]))
        return fail(BAD, "rows " + std::to_string(i) + " outside 0.." + std::to_string(len[src[i]]));
    }
    bool both = false;
    for (int i = 0; i < n; ++i) named_[dst[i]] = 1;
    for (int i = 0; i < n; ++i) both |= named_[src[i]];
    for (int i = 0; i < n; ++i) named_[dst[i]] = 0;
    if (both) return fail(BAD, "a sequence is forked from and to");
    runs.reserve(n);
    for (int i = 0; i < n; ++i) {
      const int32_t m = rows ? rows[i] : len[src[i]], have = pages_of(m);
      const int32_t* from = &table[(size_t)src[i] * most];
      int32_t* to = &table[(size_t)dst[i] * most];
      for (int j = 0; j < have; ++j) ++ref[to[j] = from[j]];
      len[dst[i]] = m;
      if (m) runs.push_back({dst[i], 0, ~src[i], have, m});
    }
    return OK;
  }

  int free(int n, const int32_t* seqs) {
    if (int rc = begin(n, seqs)) return rc;
    runs.reserve(n);
    for (int i = 0; i < n; ++i) {
      if (!len[seqs[i]]) continue;
      drop(seqs[i], 0, pages_of(len[seqs[i]]));
      len[seqs[i]] = 0;
      runs.push_back({seqs[i], 0, 0, 0, 0});
    }
    return OK;
  }

  // Sequence seqs[i] keeps rows first[r] .. first[r] + count[r] - 1 of its n_ranges[i] ranges r, ascending, and no others.
  // Pages that it alone has are written in place, shared ones replaced; pages become free when all sequences are done.
  int keep(int n, const int32_t* seqs, const int32_t* n_ranges, const int32_t* first, const int32_t* count) {
    if (int rc = begin(n, seqs)) return rc;
    int64_t total = 0, entries = 0;
    for (int i = 0; i < n; ++i) {
      if (n_ranges[i] < 0) return fail(BAD, "ranges " + std::to_string(i) + " are negative");
      int64_t end = 0;
      for (int r = 0; r < n_ranges[i]; ++r, ++total) {
        if (first[total] < end || count[total] < 0 || (int64_t)first[total] + count[total] > len[seqs[i]])
          return fail(BAD, "range " + std::to_string(r) + " of sequence " + std::to_string(seqs[i]) +
                               ": ranges must ascend, apart, within its " + std::to_string(len[seqs[i]]) + " rows");
        end = (int64_t)first[total] + count[total];
      }
      entries += pages_of(len[seqs[i]]);
    }
    ranges.reserve(total);
    moves.reserve(n);
    runs.reserve(n + entries);
    before.reserve(n + entries);
    // the ranges, joined where they touch; what has to move; the pages that are replaced (shared ones, as they are at the start)
    int64_t need = 0, at = 0;
    std::vector<int32_t> now(n);
    for (int i = 0; i < n; ++i) {
      const int32_t s = seqs[i], begin = (int32_t)ranges.size();
      int32_t rows = 0, still = -1;  // still: rows before the first that moves
      for (int r = 0; r < n_ranges[i]; ++r, ++at) {
        if (!count[at]) continue;
        if ((int32_t)ranges.size() > begin && ranges.back().first + ranges.back().count == first[at]) ranges.back().count += count[at];
        else ranges.push_back({first[at], count[at]});
        if (still < 0 && first[at] != rows) still = rows;
        rows += count[at];
      }
      now[i] = rows;
      if (still < 0) {  // none moves
        ranges.resize(begin);
        continue;
      }
      const int32_t start = still / P * P;
      moves.push_back({s, begin, (int32_t)ranges.size() - begin, start, rows});
      for (int j = start / P; j < pages_of(rows); ++j) need += ref[table[(size_t)s * most + j]] > 1;
    }
    if (need > n_free) return fail(FULL, std::to_string(need) + " pages are needed, " + std::to_string(n_free) + " are free");
    std::vector<int32_t> gone;
    gone.reserve(need + entries);
    for (size_t m = 0, i = 0; i < (size_t)n; ++i) {
      const int32_t s = seqs[i], had = pages_of(len[s]), left = pages_of(now[i]);
      int32_t* t = &table[(size_t)s * most];
      if (m < moves.size() && moves[m].seq == s) {
        const int from = moves[m++].start / P;
        for (int j = from; j < left;) {  // stretches of entries that stay, and that are replaced
          int e = j;
          const bool shared = ref[t[j]] > 1;
          while (e < left && (ref[t[e]] > 1) == shared) ++e;
          if (shared) {
            for (int x = j; x < e; ++x) {
              gone.push_back(t[x]);
              t[x] = take();
            }
            list(runs, s, j, e, t, now[i]);
            list(before, s, j, e, t, now[i]);
          } else if (need) {
            before.push_back({s, j, ~s, e - j, now[i]});
          }
          j = e;
        }
      }
      runs.push_back({s, 0, 0, 0, now[i]});
      for (int j = left; j < had; ++j) {
        gone.push_back(t[j]);
        t[j] = -1;
      }
      len[s] = now[i];
    }
    for (const int32_t p : gone) release(p);
    return OK;
  }

  // Whether the last `rows` rows of s lie in pages that it alone has.
  bool writable(int32_t s, int64_t rows) const {
    for (int j = (int)((len[s] - rows) / P); rows > 0 && j < pages_of(len[s]); ++j)
      if (ref[table[(size_t)s * most + j]] > 1) return false;
    return true;
  }

  int fail(int code, const std::string& what) {
    error = what;
    return code;
  }

 private:
  std::vector<uint64_t> free_;  // a bit per page
  size_t low_ = 0;              // no word before has one
  std::vector<char> named_;

  int begin(int n, const int32_t* seqs) {
    runs.clear();
    before.clear();
    copies.clear();
    ranges.clear();
    moves.clear();
    return check(n, seqs);
  }
  int32_t last(int32_t s) const { return table[(size_t)s * most + pages_of(len[s]) - 1]; }
  int32_t take() {
    while (!free_[low_]) ++low_;
    const int b = __builtin_ctzll(free_[low_]);
    free_[low_] &= free_[low_] - 1;
    --n_free;
    const int32_t p = (int32_t)(low_ * 64 + b);
    ref[p] = 1;
    return p;
  }
  void release(int32_t p) {
    if (--ref[p]) return;
    free_[p / 64] |= 1ull << p % 64;
    if ((size_t)p / 64 < low_) low_ = p / 64;
    ++n_free;
  }
  void drop(int32_t s, int from, int to) {
    int32_t* t = &table[(size_t)s * most];
    for (int j = from; j < to; ++j) {
      release(t[j]);
      t[j] = -1;
    }
  }
  // Entries from .. to - 1 of t as runs.
  void list(std::vector<PageRun>& out, int32_t s, int from, int to, const int32_t* t, int32_t length = -1) {
    const int32_t n = length < 0 ? len[s] : length;
    if (from == to) out.push_back({s, from, 0, 0, n});
    for (int j = from; j < to;) {
      int e = j + 1;
      while (e < to && t[e] == t[e - 1] + 1) ++e;
      out.push_back({s, j, t[j], e - j, n});
      j = e;
    }
  }
};

}  // namespace fsx
