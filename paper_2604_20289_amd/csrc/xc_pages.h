// Page tables of the branching cache: host arithmetic without HIP, so that it
// can be compiled and checked on any host.
//
// Sequences share pages by reference.  The lowest free page and the lowest
// unused sequence number are always taken first, so the same calls give the
// same tables in every run.  Token i of a sequence lies at place first + i of
// its pages (first < page size: dropped leading tokens that share the first
// page with kept ones).
#pragma once

#include <algorithm>
#include <cstdint>
#include <unordered_map>
#include <vector>

namespace xc {

enum class PageStatus { ok, invalid, full };

struct PageCopy {
  int src, dst, rows;
};

struct PageSeq {
  bool used = false;
  int first = 0, tokens = 0;
  std::vector<int> pages;
  uint64_t version = 0;  // changes whenever the table does; never repeats
};

class PageBook {
 public:
  // shift: log2 of the tokens per page
  PageBook(int n_pages, int shift, int max_seqs) : shift_(shift), refs_(n_pages, 0), seqs_(max_seqs) {}

  int n_pages() const { return (int)refs_.size(); }
  int page() const { return 1 << shift_; }
  int shift() const { return shift_; }
  int live_pages() const { return live_; }
  int live_seqs() const { return used_; }
  int refs(int page) const { return refs_[page]; }
  bool valid(int s) const { return s >= 0 && s < (int)seqs_.size() && seqs_[s].used; }
  const PageSeq& seq(int s) const { return seqs_[s]; }

  // every seqs[i] valid and no number twice
  bool distinct(int n, const int32_t* seqs) const {
    std::vector<char> seen(seqs_.size(), 0);
    for (int i = 0; i < n; ++i) {
      if (!valid(seqs[i]) || seen[seqs[i]]) return false;
      seen[seqs[i]] = 1;
    }
    return true;
  }

  PageStatus create(int32_t* out) {
    if (used_ == (int)seqs_.size()) return PageStatus::full;
    *out = take_seq();
    return PageStatus::ok;
  }

  PageStatus fork(int src, int n, int32_t* out) {
    if (!valid(src) || n < 0) return PageStatus::invalid;
    if (n > (int)seqs_.size() - used_) return PageStatus::full;
    // everything that allocates comes first: after it nothing can fail
    std::vector<std::vector<int>> tables(n, seqs_[src].pages);
    for (int i = 0; i < n; ++i) {
      const int s = take_seq();
      seqs_[s].first = seqs_[src].first;
      seqs_[s].tokens = seqs_[src].tokens;
      seqs_[s].pages.swap(tables[i]);
      for (int p : seqs_[s].pages) ++refs_[p];
      out[i] = s;
    }
    return PageStatus::ok;
  }

  // Grows seqs[i] by tokens[i].  Where a sequence's last page is partly filled
  // and shared, it gets its own copy: copies receives (shared page, own page,
  // rows to copy).  All or nothing.
  PageStatus extend(int n, const int32_t* seqs, const int32_t* tokens, std::vector<PageCopy>* copies) {
    if (n < 0 || !distinct(n, seqs)) return PageStatus::invalid;
    std::unordered_map<int, int> left;  // references of the last pages, as the calls in turn leave them
    long long need = 0;
    for (int i = 0; i < n; ++i) {
      const PageSeq& q = seqs_[seqs[i]];
      if (tokens[i] < 0) return PageStatus::invalid;
      const long long end = (long long)q.first + q.tokens + tokens[i];
      // no table can hold more; also keeps every place in 32 bits
      if (end > (long long)n_pages() << shift_) return PageStatus::full;
      if (tokens[i] > 0 && partial(q)) {
        const int p = q.pages.back();
        const auto it = left.emplace(p, refs_[p]).first;
        if (it->second > 1) {
          --it->second;
          ++need;
        }
      }
      need += std::max(0ll, ((end + page() - 1) >> shift_) - (long long)q.pages.size());
    }
    if (need > n_pages() - live_) return PageStatus::full;
    copies->clear();
    copies->reserve(n);
    for (int i = 0; i < n; ++i) {
      PageSeq& q = seqs_[seqs[i]];
      q.pages.reserve((size_t)(((long long)q.first + q.tokens + tokens[i] + page() - 1) >> shift_));
    }
    for (int i = 0; i < n; ++i) {
      PageSeq& q = seqs_[seqs[i]];
      if (tokens[i] == 0) continue;
      if (partial(q) && refs_[q.pages.back()] > 1) {
        const int p = take_page();
        copies->push_back({q.pages.back(), p, (q.first + q.tokens) & (page() - 1)});
        --refs_[q.pages.back()];
        q.pages.back() = p;
      }
      q.tokens += tokens[i];
      while (((long long)q.pages.size() << shift_) < (long long)q.first + q.tokens) q.pages.push_back(take_page());
      q.version = ++versions_;
    }
    return PageStatus::ok;
  }

  // Drops the first `front` and the last `back` tokens; whole pages that hold
  // none of the sequence's tokens any more are released.
  PageStatus trim(int s, int front, int back) {
    if (!valid(s) || front < 0 || back < 0 || (long long)front + back > seqs_[s].tokens) return PageStatus::invalid;
    if (front == 0 && back == 0) return PageStatus::ok;
    PageSeq& q = seqs_[s];
    q.tokens -= front + back;
    const long long lo = (long long)q.first + front;
    const size_t skip = q.tokens ? (size_t)(lo >> shift_) : q.pages.size();
    const size_t end = q.tokens ? (size_t)((lo + q.tokens + page() - 1) >> shift_) : q.pages.size();
    for (size_t i = 0; i < q.pages.size(); ++i)
      if (i < skip || i >= end) release(q.pages[i]);
    q.pages.resize(end);
    q.pages.erase(q.pages.begin(), q.pages.begin() + skip);
    q.first = q.tokens ? (int)(lo & (page() - 1)) : 0;
    q.version = ++versions_;
    return PageStatus::ok;
  }

  PageStatus free(int n, const int32_t* seqs) {
    if (n < 0 || !distinct(n, seqs)) return PageStatus::invalid;
    for (int i = 0; i < n; ++i) {
      PageSeq& q = seqs_[seqs[i]];
      for (int p : q.pages) release(p);
      q.pages.clear();
      q.first = q.tokens = 0;
      q.used = false;
      q.version = ++versions_;
      --used_;
      seq_hint_ = std::min(seq_hint_, (int)seqs[i]);
    }
    return PageStatus::ok;
  }

  // Moves the live pages past the first live_pages() places into the free
  // pages below them, both in ascending order: sources and destinations are
  // disjoint, and no page moves that need not.
  void compact(std::vector<PageCopy>* moves) {
    moves->clear();
    std::vector<int> to(refs_.size(), -1);
    int hole = 0;
    for (int p = live_; p < n_pages(); ++p) {
      if (refs_[p] == 0) continue;
      while (refs_[hole] != 0) ++hole;
      to[p] = hole++;
      moves->push_back({p, to[p], page()});
    }
    if (moves->empty()) return;
    for (const PageCopy& m : *moves) {
      refs_[m.dst] = refs_[m.src];
      refs_[m.src] = 0;
    }
    page_hint_ = live_;
    for (PageSeq& q : seqs_) {
      bool moved = false;
      for (int& p : q.pages)
        if (to[p] >= 0) p = to[p], moved = true;
      if (moved) q.version = ++versions_;
    }
  }

 private:
  bool partial(const PageSeq& q) const { return ((q.first + (long long)q.tokens) & (page() - 1)) != 0; }
  int take_page() {
    while (refs_[page_hint_] != 0) ++page_hint_;
    refs_[page_hint_] = 1;
    ++live_;
    return page_hint_++;
  }
  void release(int p) {
    if (--refs_[p] == 0) {
      --live_;
      page_hint_ = std::min(page_hint_, p);
    }
  }
  int take_seq() {
    while (seqs_[seq_hint_].used) ++seq_hint_;
    PageSeq& q = seqs_[seq_hint_];
    q.used = true;
    q.version = ++versions_;
    ++used_;
    return seq_hint_++;
  }

  int shift_, live_ = 0, used_ = 0, page_hint_ = 0, seq_hint_ = 0;
  uint64_t versions_ = 0;
  std::vector<int> refs_;
  std::vector<PageSeq> seqs_;
};

}  // namespace xc
