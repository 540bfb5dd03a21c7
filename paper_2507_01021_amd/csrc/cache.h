// Paged key/value cache (host interface, no HIP types): pages in device
// memory, the book of who holds which, and the calls that enqueue work on
// them. Arguments are checked by the C ABI layer, what depends on the cache's
// state (lengths, free pages) here.
#pragma once

#include <memory>

#include "../../include/whisper_mi355x.h"
#include "pages.h"

namespace wmi {

class PagedCache {
   public:
    virtual ~PagedCache() {}
    virtual void set_stream(void* hip_stream) = 0;
    virtual void extend(const int* seqs, const int* counts, int n) = 0;
    virtual void append(int layer, const void* k, const void* v, int64_t k_ld, int64_t v_ld) = 0;
    virtual void attend(int layer, const void* q, void* out, int64_t q_ld, int64_t out_ld, float scale) = 0;
    virtual void truncate(const int* seqs, const int* lengths, int n) = 0;
    virtual void fork(int src, const int* dst, int n) = 0;
    virtual void reorder(const int* seqs, const int* from, int n) = 0;
    virtual void compact() = 0;
    virtual void read(int layer, const int* seqs, int n, void* k, void* v, int64_t k_ld, int64_t v_ld) = 0;
    virtual const PageBook& book() const = 0;
    virtual int tokens() const = 0;  // new tokens of the current chunk
};

// bits 0: keys and values in p.dtype; 8 or 4: packed. device WHISPER_NO_DEVICE:
// the book alone. Throws ArgError or DeviceError.
std::unique_ptr<PagedCache> make_paged_cache(const whisper_cache_params& p, int bits, int device);

}  // namespace wmi
