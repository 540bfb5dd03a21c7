// Book of a paged key/value cache (host side, no HIP types): which pages each
// sequence holds, how many sequences share a page, and which pages are free.
//
// A sequence is a list of pages and a length; position p is in page p / P of
// the list. A page may be in several lists (forked sequences) as long as
// nobody writes to it: a sequence that is extended into a shared page first
// gets a copy of its own. Free pages are handed out lowest number first.
// Every call checks all it needs before it changes anything.
#pragma once

#include <stdint.h>

#include <set>
#include <string>
#include <vector>

#include "common.h"

namespace wmi {

struct PageCopy {
    int src, dst;
};

class PageBook {
   public:
    PageBook(int page_size, int n_pages, int max_seqs, int max_positions)
        : P_(page_size), max_pos_(max_positions), ref_(n_pages, 0), pages_(max_seqs), len_(max_seqs, 0) {
        for (int i = 0; i < n_pages; ++i) free_.insert(free_.end(), i);
    }
    int page_size() const { return P_; }
    int max_seqs() const { return (int)len_.size(); }
    int length(int s) const { return len_[s]; }
    int n_pages() const { return (int)ref_.size(); }
    int free_pages() const { return (int)free_.size(); }
    const std::vector<int>& pages(int s) const { return pages_[s]; }
    int max_list() const { return pages_for(max_pos_); }

    // Adds counts[i] positions to sequence seqs[i]. Pages that get their
    // first new position and are shared are replaced by a copy (appended to
    // `copies`); the last holder of a page writes in place.
    void extend(const int* seqs, const int* counts, int n, std::vector<PageCopy>& copies) {
        // the same page may be the partial page of several listed sequences:
        // every one but the last then needs a copy, counted on shadow counts
        long long need = 0;
        std::vector<std::pair<int, int>> taken;  // page, references given up by this call
        for (int i = 0; i < n; ++i) {
            const int s = seqs[i];
            if ((long long)len_[s] + counts[i] > max_pos_)
                throw ArgError(CAPACITY, "sequence " + std::to_string(s) + " would exceed max_positions (" +
                                                        std::to_string(max_pos_) + ")");
            need += pages_for(len_[s] + counts[i]) - (int)pages_[s].size();
            if (writes_partial(s, counts[i])) {
                const int pg = pages_[s].back();
                int given = 0;
                for (auto& t : taken)
                    if (t.first == pg) given = t.second;
                if (ref_[pg] - given > 1) {
                    ++need;
                    bool found = false;
                    for (auto& t : taken)
                        if (t.first == pg) { ++t.second; found = true; }
                    if (!found) taken.push_back({pg, 1});
                }
            }
        }
        require(need);
        for (int i = 0; i < n; ++i) {
            const int s = seqs[i];
            if (writes_partial(s, counts[i]) && ref_[pages_[s].back()] > 1) {
                const int old = pages_[s].back(), now = take();
                --ref_[old];
                pages_[s].back() = now;
                copies.push_back({old, now});
            }
            len_[s] += counts[i];
            while ((int)pages_[s].size() < pages_for(len_[s])) pages_[s].push_back(take());
        }
    }

    // Shortens sequence seqs[i] to lengths[i] positions; pages that nobody
    // holds any more are free again.
    void truncate(const int* seqs, const int* lengths, int n) {
        for (int i = 0; i < n; ++i) {
            const int s = seqs[i];
            len_[s] = lengths[i];
            while ((int)pages_[s].size() > pages_for(lengths[i])) {
                give_back(pages_[s].back());
                pages_[s].pop_back();
            }
        }
    }

    // Makes each (empty) sequence dst[i] a copy of src's first len positions:
    // whole pages are shared, a partly filled last page is copied.
    void fork(int src, int len, const int* dst, int n, std::vector<PageCopy>& copies) {
        const bool partial = len % P_ != 0;
        if (partial) require(n);
        const std::vector<int> from(pages_[src].begin(), pages_[src].begin() + pages_for(len));
        for (int i = 0; i < n; ++i) {
            const int d = dst[i];
            pages_[d] = from;
            len_[d] = len;
            if (partial) {
                pages_[d].back() = take();
                copies.push_back({from.back(), pages_[d].back()});
            }
            for (size_t k = 0; k + (partial ? 1 : 0) < pages_[d].size(); ++k) ++ref_[pages_[d][k]];
        }
    }

    // Makes sequence seqs[i] what sequence from[i] was before the call, all at
    // once: pages are shared, partly filled ones too (the next extend copies
    // those that still have several holders).
    void reorder(const int* seqs, const int* from, int n) {
        std::vector<std::vector<int>> lists(n);
        std::vector<int> lens(n);
        for (int i = 0; i < n; ++i) {
            lists[i] = pages_[from[i]];
            lens[i] = len_[from[i]];
        }
        for (auto& l : lists)
            for (int p : l) ++ref_[p];
        for (int i = 0; i < n; ++i) {
            for (int p : pages_[seqs[i]]) give_back(p);
            pages_[seqs[i]].swap(lists[i]);
            len_[seqs[i]] = lens[i];
        }
    }

    // Moves the pages in use to the lowest numbers: afterwards page numbers
    // from used() on are free. Sources and destinations are disjoint.
    void compact(std::vector<PageCopy>& copies) {
        std::vector<int> to(ref_.size(), -1);
        int hi = (int)ref_.size() - 1;
        for (;;) {
            while (hi >= 0 && ref_[hi] == 0) --hi;
            if (hi < 0 || free_.empty() || *free_.begin() > hi) break;
            const int lo = *free_.begin();
            free_.erase(free_.begin());
            free_.insert(hi);
            ref_[lo] = ref_[hi];
            ref_[hi] = 0;
            to[hi] = lo;
            copies.push_back({hi, lo});
        }
        if (copies.empty()) return;
        for (auto& l : pages_)
            for (int& p : l)
                if (to[p] >= 0) p = to[p];
    }
    int used() const { return (int)(ref_.size() - free_.size()); }

   private:
    static constexpr int CAPACITY = -4;  // WHISPER_E_CAPACITY
    int P_, max_pos_;
    std::vector<int> ref_;
    std::set<int> free_;
    std::vector<std::vector<int>> pages_;
    std::vector<int> len_;

    int pages_for(int n) const { return (int)(((long long)n + P_ - 1) / P_); }
    // whether new positions go into a page that already holds some
    bool writes_partial(int s, int count) const { return count > 0 && len_[s] % P_ != 0; }
    void require(long long n) const {
        if (n > (long long)free_.size())
            throw ArgError(CAPACITY, "the call needs " + std::to_string(n) + " free pages, the cache has " +
                                                    std::to_string(free_.size()));
    }
    int take() {
        const int p = *free_.begin();
        free_.erase(free_.begin());
        ref_[p] = 1;
        return p;
    }
    void give_back(int p) {
        if (--ref_[p] == 0) free_.insert(p);
    }
};

}  // namespace wmi
