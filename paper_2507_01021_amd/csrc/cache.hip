// The paged cache's device side: pages and page lists in device memory, the
// plan of a chunk of new tokens, and the launches.
#include <string.h>

#include <algorithm>

#include "cache.h"
#include "device.h"
#include "paged.h"

namespace wmi {

namespace {

// Workgroups that an attention call is cut into when its rows alone give
// fewer: four per CU (paged_attn_kernel has both sides' times).
constexpr int ATTN_WGS = 1024;
// Longest range that is never cut: four blocks of 32 positions per wave. Longer
// ones give equal parts of 384 positions or more, and a last one of what is left.
constexpr int ATTN_PART = 512;
// Rows of a sequence and key/value head from which the kernel of 128 rows per
// workgroup takes them (bf16), the workgroups it is cut into where the rows
// give fewer (one per CU), and the longest range that it never cuts: with 1024,
// two sequences of 100 tokens over 3000 positions, 32 / 8 heads of 128, took 45
// instead of 35 us, one of 30 tokens with 8 query heads 28 instead of 19.
// us of the 16-row kernel and of this one, 20 heads of 64, per rows of a sequence:
//                              32         64          96        128        256
//    1 sequence  over  200   4.5  8.3   5.2  9.8   5.1 10.0   5.4 11.3   6.4 13.7
//    1           over 4000    14   16    15   18    19   19    19   19    30   26
//    9 sequences over  200   5.2  8.3   6.6 10.0  10.9 10.3  12.7 11.9  25.5 17.6
//    9           over 1000    21   21    26   23    35   25    43   27   106   36
//   32           over 1000    52   38   102   36   152   45   206   47   430   84
// Rows alone do not say which is faster. From 128 on, the 16-row kernel would save
// some 7 us where it is faster (few sequences, short contexts) and lose several
// times the time where it is not; below, it loses with many sequences too.
constexpr int BIG_FROM = 128, BIG_WGS = 256, BIG_PART = 512;
// Most workgroups of a launch along its list (a grid holds fewer than 2^32
// threads): the kernels go through longer lists in strides.
constexpr int MOST_WGS = 1 << 22;

template <class T>
class PagedCacheT final : public PagedCache {
   public:
    PagedCacheT(const whisper_cache_params& p, int device)
        : P_(p), dev_(device), book_(p.page_size, p.n_pages, p.max_seqs, p.max_positions) {
        G_ = p.n_head / p.n_kv_head;
        // parts of cut ranges: ATTN_WGS / n_kv_head whole ones and a partial one for each of as many ranges
        max_parts_ = 2 * (ATTN_WGS / p.n_kv_head + 1);
        if (big_rows(p.max_tokens)) max_parts_ += BIG_ROWS / 16 * 2 * (BIG_WGS / p.n_kv_head + 1);
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        head_elems_ = (long long)p.page_size * p.head_size;
        page_bytes_ = 2LL * p.n_layer * p.n_kv_head * head_elems_ * sizeof(T);
        while ((1 << shift_) < p.page_size) ++shift_;
        pages_ = dalloc<unsigned char>((size_t)p.n_pages * page_bytes_);
        table_ = dalloc<int>((size_t)p.max_seqs * book_.max_list() + 1);
        odd_ = table_ + (size_t)p.max_seqs * book_.max_list();  // (the pages are cleared: all finite)
        // room for the longest plan, so that recorded launches keep their addresses
        const long long T0 = p.max_tokens, S0 = p.max_seqs;
        max_tiles_ = (int)std::min(T0, T0 / 32 + 2 * S0);
        plan_.cap = HEAD_INTS + 8 * (T0 * G_ / 16 + S0 + max_parts_) + 6LL * max_parts_ + 4LL * max_tiles_ +
                    2 * (std::min(T0, T0 / p.page_size + S0) + 2 * S0);
        plan_.dev = dalloc<int>(plan_.cap);
        parts_ = dalloc<float>((size_t)max_parts_ * p.n_kv_head * 16 * (p.head_size + 2));
        WMI_HIP(hipDeviceSynchronize());
    }
    ~PagedCacheT() override {
        if (dev_ == WHISPER_NO_DEVICE) return;
        int old = -1;
        (void)hipGetDevice(&old);
        (void)hipSetDevice(dev_);
        (void)hipStreamSynchronize(st_);
        for (auto& s : ring_) {
            if (s.ev) (void)hipEventDestroy(s.ev);
            if (s.host) (void)hipHostFree(s.host);
        }
        for (void* q : {(void*)pages_, (void*)table_, (void*)parts_, (void*)plan_.dev, (void*)list_.dev})
            if (q) (void)hipFree(q);
        if (old >= 0) (void)hipSetDevice(old);
    }

    const PageBook& book() const override { return book_; }
    int tokens() const override { return plan_ok_ ? tokens_ : 0; }

    void set_stream(void* s) override {
        if (dev_ == WHISPER_NO_DEVICE || s == st_) return;
        DeviceScope scope(dev_);
        no_capture();
        WMI_HIP(hipStreamSynchronize(st_));
        st_ = static_cast<hipStream_t>(s);
    }

    void extend(const int* seqs, const int* counts, int n) override {
        int total = 0;
        for (int i = 0; i < n; ++i) {
            if (counts[i] > P_.max_tokens - total)
                throw ArgError(WHISPER_E_CAPACITY, "the chunk has more than max_tokens (" + std::to_string(P_.max_tokens) +
                                                       ") new tokens");
            total += counts[i];
        }
        if (dev_ != WHISPER_NO_DEVICE) {
            DeviceScope scope(dev_);
            no_capture();
        }
        std::vector<PageCopy> copies;
        std::vector<int> before(n);
        for (int i = 0; i < n; ++i) before[i] = (int)book_.pages(seqs[i]).size();
        book_.extend(seqs, counts, n, copies);
        tokens_ = total;
        chunk_.assign(seqs, seqs + n);
        counts_.assign(counts, counts + n);
        plan_ok_ = append_ok_ = true;
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        // the plan, the changed entries of the page lists and the page copies in one list
        build_plan(seqs, counts, n);
        std::vector<int> upd;
        for (int i = 0; i < n; ++i) {
            const auto& pg = book_.pages(seqs[i]);
            // a partly filled page may have been replaced by a copy
            for (int k = std::max(0, before[i] - (copies.empty() ? 0 : 1)); k < (int)pg.size(); ++k) add_update(upd, seqs[i], k, pg[k]);
        }
        const size_t u0 = blob_.size(), c0 = u0 + upd.size();
        blob_.insert(blob_.end(), upd.begin(), upd.end());
        for (auto& c : copies) blob_.insert(blob_.end(), {c.src, c.dst});
        put(plan_, blob_, u0, (int)upd.size() / 2);
        copy_pages(plan_.dev + c0, (int)copies.size());
    }

    void append(int layer, const void* k, const void* v, int64_t k_ld, int64_t v_ld) override {
        need_chunk();
        if (!append_ok_)
            throw ArgError(WHISPER_E_STATE, "a sequence of the chunk was forked: its rows cannot be written any more");
        DeviceScope scope(dev_);
        // a recorded launch goes through whatever list is current at its replay in strides
        const int n = capturing(st_) ? std::min(max_tiles_, ATTN_WGS) : n_tiles_;
        if (n == 0) return;
        move<true>(layer, plan_.dev, n, k, v, k_ld, v_ld, tokens_);
    }

    void attend(int layer, const void* q, void* out, int64_t q_ld, int64_t out_ld, float scale) override {
        need_chunk();
        DeviceScope scope(dev_);
        const bool rec = capturing(st_);
        if (n_items_ + n_bigs_ == 0 && !rec) return;
        AttnArgs a{view(), layer, P_.n_head, G_, q, out, q_ld, out_ld, scale * 1.4426950408889634f, plan_.dev,
                   parts_};
        if (P_.head_size == 64) launch_attn<64>(a, rec);
        else launch_attn<128>(a, rec);
        WMI_HIP(hipGetLastError());
    }

    void truncate(const int* seqs, const int* lengths, int n) override {
        for (int i = 0; i < n; ++i)
            if (lengths[i] > book_.length(seqs[i]))
                throw ArgError(WHISPER_E_INVAL, "sequence " + std::to_string(seqs[i]) + " holds " +
                                                    std::to_string(book_.length(seqs[i])) + " positions, fewer than " +
                                                    std::to_string(lengths[i]));
        if (dev_ != WHISPER_NO_DEVICE) {
            DeviceScope scope(dev_);
            no_capture();
        }
        bool taken = false;
        for (int i = 0; i < n; ++i)
            taken = taken || (lengths[i] < book_.length(seqs[i]) && std::find(chunk_.begin(), chunk_.end(), seqs[i]) != chunk_.end());
        book_.truncate(seqs, lengths, n);
        if (!taken || !plan_ok_) return;
        plan_ok_ = false;
        if (dev_ == WHISPER_NO_DEVICE) return;
        // a replay must find no rows: the pages may soon be another sequence's
        DeviceScope scope(dev_);
        put(plan_, std::vector<int>(HEAD_INTS, 0), 0, 0);
    }

    void fork(int src, const int* dst, int n) override {
        for (int i = 0; i < n; ++i)
            if (book_.length(dst[i]) != 0)
                throw ArgError(WHISPER_E_STATE, "sequence " + std::to_string(dst[i]) + " is not empty");
        if (dev_ != WHISPER_NO_DEVICE) {
            DeviceScope scope(dev_);
            no_capture();
        }
        std::vector<PageCopy> copies;
        book_.fork(src, book_.length(src), dst, n, copies);
        if (dev_ == WHISPER_NO_DEVICE) return;
        std::vector<int> upd;
        for (int i = 0; i < n; ++i) {
            const auto& pg = book_.pages(dst[i]);
            for (int k = 0; k < (int)pg.size(); ++k) add_update(upd, dst[i], k, pg[k]);
        }
        apply(upd, copies);
        // pages of the chunk's new positions are shared now, or were copied as they
        // were: nothing more is written there, by replays either
        bool open = false;
        for (size_t i = 0; i < chunk_.size(); ++i) open = open || (chunk_[i] == src && counts_[i] > 0);
        if (n == 0 || !open || !plan_ok_ || !append_ok_) return;
        append_ok_ = false;
        DeviceScope scope(dev_);
        ListHead head = head_;
        head.tiles = 0;
        std::vector<int> h(HEAD_INTS);
        memcpy(h.data(), &head, sizeof(head));
        put(plan_, h, 0, 0);
    }

    void compact() override {
        if (dev_ != WHISPER_NO_DEVICE) {
            DeviceScope scope(dev_);
            no_capture();
        }
        std::vector<std::vector<int>> before(P_.max_seqs);
        for (int s = 0; s < P_.max_seqs; ++s) before[s] = book_.pages(s);
        std::vector<PageCopy> copies;
        book_.compact(copies);
        if (dev_ == WHISPER_NO_DEVICE || copies.empty()) return;
        std::vector<int> upd;
        for (int s = 0; s < P_.max_seqs; ++s) {
            const auto& pg = book_.pages(s);
            for (int k = 0; k < (int)pg.size(); ++k)
                if (pg[k] != before[s][k]) add_update(upd, s, k, pg[k]);
        }
        apply(upd, copies);
    }

    void read(int layer, const int* seqs, int n, void* k, void* v, int64_t k_ld, int64_t v_ld) override {
        if (dev_ == WHISPER_NO_DEVICE) throw ArgError(WHISPER_E_STATE, "the cache has no device");
        DeviceScope scope(dev_);
        no_capture();
        long long rows = 0;
        for (int i = 0; i < n; ++i) rows += book_.length(seqs[i]);
        if (rows > INT32_MAX) throw ArgError(WHISPER_E_INVAL, "more than 2^31 - 1 positions to read at once");
        std::vector<int> t(HEAD_INTS);
        int row = 0;
        for (int i = 0; i < n; ++i) row = add_tiles(t, seqs[i], 0, book_.length(seqs[i]), row);
        if (row == 0) return;
        const ListHead head{0, 0, (int)(t.size() - HEAD_INTS) / 4, 0, HEAD_INTS, 0, 0, 0};
        memcpy(t.data(), &head, sizeof(head));
        put(list_, t, 0, 0);
        move<false>(layer, list_.dev, head.tiles, k, v, k_ld, v_ld, row);
    }

   private:
    struct DevList {
        int* dev = nullptr;
        size_t cap = 0;
    };
    struct Stage {
        int* host = nullptr;
        size_t cap = 0;
        hipEvent_t ev = nullptr;
    };
    whisper_cache_params P_;
    int dev_, G_, shift_ = 0;
    long long head_elems_ = 0, page_bytes_ = 0;
    int max_parts_ = 0;
    PageBook book_;
    hipStream_t st_ = nullptr;  // the device's default stream unless one was chosen
    unsigned char* pages_ = nullptr;
    int *table_ = nullptr, *odd_ = nullptr;
    float* parts_ = nullptr;
    DevList plan_, list_;
    Stage ring_[8];
    int next_ = 0;
    // the chunk: its sequences, new tokens and the lengths of its lists
    std::vector<int> chunk_, counts_, blob_;
    ListHead head_{};
    bool plan_ok_ = false;    // there is a chunk
    bool append_ok_ = false;  // none of its sequences was forked since
    int tokens_ = 0, n_items_ = 0, n_bigs_ = 0, n_merges_ = 0, n_tiles_ = 0;
    int max_tiles_ = 0;

    template <class U>
    U* dalloc(size_t count) {
        void* q = nullptr;
        if (hipMalloc(&q, std::max<size_t>(count, 1) * sizeof(U)) != hipSuccess) {
            (void)hipGetLastError();
            for (void* x : {(void*)pages_, (void*)table_, (void*)plan_.dev})
                if (x) (void)hipFree(x);
            throw ArgError(WHISPER_E_NOMEM, "device allocation of " + std::to_string(count * sizeof(U)) + " bytes failed");
        }
        WMI_HIP(hipMemset(q, 0, std::max<size_t>(count, 1) * sizeof(U)));
        return static_cast<U*>(q);
    }
    void no_capture() const {
        if (capturing(st_))
            throw ArgError(WHISPER_E_STATE, "the stream is recording a graph: only append and attend may be recorded");
    }
    void need_chunk() const {
        if (dev_ == WHISPER_NO_DEVICE) throw ArgError(WHISPER_E_STATE, "the cache has no device");
        if (!plan_ok_) throw ArgError(WHISPER_E_STATE, "no chunk: call whisper_cache_extend first");
    }
    PagedView view() const {
        return PagedView{pages_, table_, book_.max_list(), shift_, P_.n_layer, P_.n_kv_head, head_elems_, odd_};
    }

    // Copies a list to the device, as a kernel argument if it is short, else
    // through pinned memory (a ring, so that the host rarely waits), and makes
    // the n changes of page lists that begin at upd.
    void put(DevList& d, const std::vector<int>& v, size_t upd, int n) {
        if (&d == &plan_ && v.size() > d.cap) throw DeviceError("paged cache: a longer plan than planned for");
        if (v.size() > d.cap) {
            WMI_HIP(hipStreamSynchronize(st_));
            if (d.dev) WMI_HIP(hipFree(d.dev));
            d.dev = nullptr;
            d.cap = 0;
            const size_t cap = std::max<size_t>(4096, v.size() + v.size() / 2);
            if (hipMalloc(reinterpret_cast<void**>(&d.dev), cap * sizeof(int)) != hipSuccess)
                throw DeviceError("device allocation of a list failed");
            d.cap = cap;
        }
        if (v.size() <= 2 * PUT_INTS) {
            const bool once = v.size() <= PUT_INTS;
            for (size_t i = 0; i < v.size(); i += PUT_INTS) {
                PutInts a;
                a.n = (int)std::min<size_t>(PUT_INTS, v.size() - i);
                memcpy(a.v, v.data() + i, a.n * sizeof(int));
                hipLaunchKernelGGL(put_ints_kernel, dim3(1), dim3(256), 0, st_, a, d.dev + i, (int)upd, once ? n : 0, table_);
            }
            WMI_HIP(hipGetLastError());
            if (!once) update_table(d.dev + upd, n);
            return;
        }
        Stage& s = ring_[next_];
        next_ = (next_ + 1) % 8;
        if (s.ev) WMI_HIP(hipEventSynchronize(s.ev));
        else WMI_HIP(hipEventCreateWithFlags(&s.ev, hipEventDisableTiming));
        if (v.size() > s.cap) {
            if (s.host) WMI_HIP(hipHostFree(s.host));
            s.host = nullptr;
            s.cap = 0;
            const size_t cap = std::max<size_t>(4096, v.size() + v.size() / 2);
            WMI_HIP(hipHostMalloc(reinterpret_cast<void**>(&s.host), cap * sizeof(int)));
            s.cap = cap;
        }
        memcpy(s.host, v.data(), v.size() * sizeof(int));
        WMI_HIP(hipMemcpyAsync(d.dev, s.host, v.size() * sizeof(int), hipMemcpyHostToDevice, st_));
        WMI_HIP(hipEventRecord(s.ev, st_));
        update_table(d.dev + upd, n);
    }

    void add_update(std::vector<int>& upd, int seq, int k, int page) const {
        upd.push_back(seq * book_.max_list() + k);
        upd.push_back(page);
    }
    void update_table(const int* upd, int n) {
        if (n == 0) return;
        hipLaunchKernelGGL(table_update_kernel, dim3((n + 255) / 256), dim3(256), 0, st_, upd, n, table_);
        WMI_HIP(hipGetLastError());
    }
    void copy_pages(const int* pairs, int n) {
        for (int i = 0; i < n; i += 32768) {
            hipLaunchKernelGGL(paged_copy_kernel, dim3((unsigned)((page_bytes_ + PAGE_RUN - 1) / PAGE_RUN), std::min(32768, n - i)),
                               dim3(256), 0, st_, pages_, pairs + 2 * i, page_bytes_);
            WMI_HIP(hipGetLastError());
        }
    }
    void apply(const std::vector<int>& upd, const std::vector<PageCopy>& copies) {
        std::vector<int> v = upd;
        for (auto& c : copies) v.insert(v.end(), {c.src, c.dst});
        if (v.empty()) return;
        DeviceScope scope(dev_);
        put(list_, v, 0, (int)upd.size() / 2);
        copy_pages(list_.dev + upd.size(), (int)copies.size());
    }

    // Whether a chunk's `count` tokens of one sequence go to the kernel of many rows.
    bool big_rows(int count) const { return sizeof(T) == 2 && (long long)count * G_ >= BIG_FROM; }
    bool max_bigs() const { return big_rows(P_.max_tokens); }

    // Positions [first, first + n) of a sequence as tiles; returns the row after its last.
    static int add_tiles(std::vector<int>& t, int seq, int first, int n, int row) {
        for (int p = first; p < first + n;) {
            const int m = std::min(32 - (p & 31), first + n - p);
            t.insert(t.end(), {seq, p, m, row});
            p += m;
            row += m;
        }
        return row;
    }

    // The chunk's lists: header, attention items, merges, append tiles.
    // Ranges of positions are cut where the rows alone give fewer workgroups
    // than ATTN_WGS, if they are longer than ATTN_PART, into parts of equal length
    // but for the last.
    void build_plan(const int* seqs, const int* counts, int n) {
        std::vector<AttnItem> items, cut;
        std::vector<MergeItem> merges;
        std::vector<int> tiles;
        int row = 0, np = 0;
        // items of `step` rows of the sequences that kernel `big` takes, cut
        // into about `wgs` workgroups, a part's positions a multiple of 128
        auto plan = [&](bool big, int step, int wgs, int least) {
            items.clear();
            cut.clear();
            long long work = 0;
            int tok0 = 0;
            for (int i = 0; i < n; tok0 += counts[i++]) {
                const int s = seqs[i], past = book_.length(s) - counts[i], rows = counts[i] * G_;
                if (big_rows(counts[i]) != big) continue;
                for (int j = 0; j < rows; j += step) {
                    const int end = past + (std::min(j + step, rows) - 1) / G_ + 1;
                    items.push_back(AttnItem{s, past, counts[i], tok0, j, 0, end, -1});
                    work += end;
                }
            }
            const long long part = std::max<long long>(least, (work * P_.n_kv_head / wgs + 127) / 128 * 128);
            for (const AttnItem& t : items) {
                const int k = (int)((t.kv1 + part - 1) / part);
                if (k < 2) {
                    cut.push_back(t);
                    continue;
                }
                const int len = ((t.kv1 + k - 1) / k + 127) / 128 * 128, slots = step / 16, first = np;
                for (int p = 0; p < t.kv1; p += len) {
                    AttnItem c = t;
                    c.kv0 = p;
                    c.kv1 = std::min(p + len, t.kv1);
                    c.part = np;
                    np += slots;
                    cut.push_back(c);
                }
                for (int g = 0; g < slots && t.j0 + 16 * g < t.count * G_; ++g)
                    merges.push_back(MergeItem{t.count, t.tok0, t.j0 + 16 * g, first + g, (np - first) / slots, slots});
            }
            if (np > max_parts_) throw DeviceError("paged cache: more parts than planned for");
            // long ranges first, so that none starts last
            std::stable_sort(cut.begin(), cut.end(),
                             [](const AttnItem& a, const AttnItem& b) { return a.kv1 - a.kv0 > b.kv1 - b.kv0; });
        };
        for (int i = 0; i < n; ++i) row = add_tiles(tiles, seqs[i], book_.length(seqs[i]) - counts[i], counts[i], row);
        plan(true, BIG_ROWS, BIG_WGS, BIG_PART);
        const std::vector<AttnItem> bigs = cut;
        plan(false, 16, ATTN_WGS, ATTN_PART);
        n_items_ = (int)cut.size();
        n_bigs_ = (int)bigs.size();
        n_merges_ = (int)merges.size();
        n_tiles_ = (int)tiles.size() / 4;
        blob_.assign(HEAD_INTS, 0);
        auto add = [&](const void* p, size_t ints) {
            const size_t at = blob_.size();
            blob_.resize(at + ints);
            if (ints) memcpy(blob_.data() + at, p, ints * sizeof(int));
            return at;
        };
        add(cut.data(), cut.size() * (sizeof(AttnItem) / sizeof(int)));
        const size_t ma = add(merges.data(), merges.size() * (sizeof(MergeItem) / sizeof(int)));
        const size_t ta = add(tiles.data(), tiles.size());
        const size_t ba = add(bigs.data(), bigs.size() * (sizeof(AttnItem) / sizeof(int)));
        head_ = ListHead{n_items_, n_merges_, n_tiles_, (int)ma, (int)ta, n_bigs_, (int)ba, 0};
        memcpy(blob_.data(), &head_, sizeof(head_));
    }

    template <int D>
    void launch_attn(const AttnArgs& a, bool rec) {
        // a recorded launch may meet a longer list at its replay: the kernels go through it in strides
        const unsigned ni = rec ? 2 * ATTN_WGS : std::min(n_items_ * P_.n_kv_head, MOST_WGS);
        const unsigned nm = rec ? ATTN_WGS : (unsigned)n_merges_ * P_.n_kv_head;
        if constexpr (sizeof(T) == 2) {
            const unsigned nb = rec ? (max_bigs() ? 2 * BIG_WGS : 0) : (unsigned)n_bigs_ * P_.n_kv_head;
            if (nb) hipLaunchKernelGGL(paged_attn_big_kernel<D>, dim3(nb), dim3(BIG_THREADS), 0, st_, a);
        }
        if (ni) hipLaunchKernelGGL((paged_attn_kernel<T, D, false>), dim3(ni), dim3(256), 0, st_, a);
        if (nm) hipLaunchKernelGGL((paged_merge_kernel<T, D, false>), dim3(nm), dim3(256), 0, st_, a);
    }

    // Rows of `n_rows` tokens into (IN) or out of the pages; layer -1: every
    // layer, rows of layer l at l * n_rows * ld.
    template <bool IN>
    void move(int layer, const int* list, int n, const void* k, const void* v, int64_t k_ld, int64_t v_ld, int n_rows) {
        if (P_.head_size == 64) move_d<IN, 64>(layer, list, n, k, v, k_ld, v_ld, n_rows);
        else move_d<IN, 128>(layer, list, n, k, v, k_ld, v_ld, n_rows);
        WMI_HIP(hipGetLastError());
    }
    template <bool IN, int D>
    void move_d(int layer, const int* list, int n, const void* k, const void* v, int64_t k_ld, int64_t v_ld, int n_rows) {
        const int l0 = layer < 0 ? 0 : layer, nl = layer < 0 ? P_.n_layer : 1;
        const long long kl = k_ld * n_rows, vl = v_ld * n_rows;
        constexpr int EL = 16 / sizeof(T);
        const bool vec = (reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16 == 0 && k_ld % EL == 0 &&
                         v_ld % EL == 0;
        const dim3 grid(std::min(n, MOST_WGS), P_.n_kv_head, nl), block(256);
        if constexpr (IN) {
            const T *kk = static_cast<const T*>(k), *vv = static_cast<const T*>(v);
            if (vec) hipLaunchKernelGGL((paged_append_kernel<T, D, true>), grid, block, 0, st_, view(), list, l0, kk, vv, k_ld, v_ld, kl, vl);
            else hipLaunchKernelGGL((paged_append_kernel<T, D, false>), grid, block, 0, st_, view(), list, l0, kk, vv, k_ld, v_ld, kl, vl);
        } else {
            T *kk = static_cast<T*>(const_cast<void*>(k)), *vv = static_cast<T*>(const_cast<void*>(v));
            if (vec) hipLaunchKernelGGL((paged_read_kernel<T, D, true>), grid, block, 0, st_, view(), list, l0, kk, vv, k_ld, v_ld, kl, vl);
            else hipLaunchKernelGGL((paged_read_kernel<T, D, false>), grid, block, 0, st_, view(), list, l0, kk, vv, k_ld, v_ld, kl, vl);
        }
    }
};

}  // namespace

std::unique_ptr<PagedCache> make_paged_cache(const whisper_cache_params& p, int device) {
    if (p.dtype == WHISPER_DTYPE_BF16) return std::unique_ptr<PagedCache>(new PagedCacheT<bf16>(p, device));
    return std::unique_ptr<PagedCache>(new PagedCacheT<float>(p, device));
}

}  // namespace wmi
