// C ABI of the operators that work on a program's own device memory
// (include/whisper_mi355x.h): the paged key/value cache, the sampler and the
// choice of beams. Argument checks, error codes and messages; every check runs
// before any device work.
#include <hip/hip_runtime.h>

#include <memory>
#include <new>
#include <set>
#include <string>
#include <vector>

#include "beam.h"
#include "cache.h"
#include "sampler.h"

namespace {

thread_local std::string g_error;  // last failed create of this thread, calls with a NULL handle

}  // namespace

struct whisper_cache {
    whisper_cache_params p;
    std::unique_ptr<wmi::PagedCache> impl;
    std::string err;
    bool broken = false;
};

struct whisper_sampler {
    int n_vocab, max_rows;
    std::unique_ptr<wmi::Sampler> impl;
    std::string err;
    bool broken = false;
};

struct whisper_beam {
    int n_vocab, max_rows;
    std::unique_ptr<wmi::Beam> impl;
    std::string err;
    bool broken = false;
};

namespace {

template <class H>
whisper_status fail(H* h, whisper_status code, const std::string& msg) {
    if (h) {
        h->err = msg;
        if (code == WHISPER_E_DEVICE) h->broken = true;
    } else {
        g_error = msg;
    }
    return code;
}

// Runs f, turning exceptions into a status and a message.
template <class H, class F>
whisper_status guarded(H* h, F&& f) {
    try {
        return f();
    } catch (const wmi::ArgError& e) {
        return fail(h, e.code, e.what());
    } catch (const wmi::DeviceError& e) {
        return fail(h, WHISPER_E_DEVICE, e.what());
    } catch (const std::bad_alloc&) {
        return fail(h, WHISPER_E_NOMEM, "host allocation failed");
    } catch (const std::exception& e) {
        return fail(h, WHISPER_E_DEVICE, e.what());
    }
}

template <class H>
whisper_status usable(H* h) {
    if (!h) return fail(h, WHISPER_E_INVAL, "handle is NULL");
    if (h->broken) {
        h->err = "unusable after a device error";
        return WHISPER_E_DEVICE;
    }
    return WHISPER_OK;
}

whisper_status check_device(int device) {
    if (device == WHISPER_NO_DEVICE) return WHISPER_OK;
    int n = 0;
    if (hipGetDeviceCount(&n) != hipSuccess || device < 0 || device >= n)
        return fail<whisper_cache>(nullptr, WHISPER_E_DEVICE, "no HIP device " + std::to_string(device));
    return WHISPER_OK;
}

std::string check_cache(const whisper_cache_params& p) {
    if (p.dtype != WHISPER_DTYPE_F32 && p.dtype != WHISPER_DTYPE_BF16) return "dtype must be 0 (fp32) or 1 (bf16)";
    if (p.n_layer < 1 || p.n_layer > 256) return "n_layer must be in 1..256";
    if (p.n_kv_head < 1 || p.n_head < p.n_kv_head || p.n_head > 256 || p.n_head % p.n_kv_head)
        return "n_head must be a multiple of n_kv_head, 256 at most";
    if (p.head_size != 64 && p.head_size != 128) return "head_size must be 64 or 128";
    if (p.page_size != 32 && p.page_size != 64 && p.page_size != 128 && p.page_size != 256)
        return "page_size must be 32, 64, 128 or 256";
    if (p.n_pages < 1 || p.n_pages > (1 << 22)) return "n_pages must be in 1..4194304";
    if (p.max_seqs < 1 || p.max_seqs > 4096) return "max_seqs must be in 1..4096";
    if (p.max_positions < 1 || p.max_positions > (1 << 24)) return "max_positions must be in 1..16777216";
    if (p.max_tokens < 1 || p.max_tokens > (1 << 20)) return "max_tokens must be in 1..1048576";
    if ((int64_t)p.max_seqs * ((p.max_positions + p.page_size - 1) / p.page_size) > (1 << 28))
        return "max_seqs x max_positions / page_size must not exceed 268435456";
    return "";
}

// n distinct sequences of the cache (n >= 0), and one value >= 0 for each.
whisper_status check_seqs(whisper_cache* c, const int32_t* seqs, const int32_t* values, int32_t n, const char* what) {
    if (n < 0 || n > c->p.max_seqs) return fail(c, WHISPER_E_INVAL, "n must be in 0..max_seqs");
    if (n > 0 && (!seqs || !values)) return fail(c, WHISPER_E_INVAL, std::string("seqs and ") + what + " must not be NULL");
    std::vector<bool> seen(c->p.max_seqs, false);
    for (int i = 0; i < n; ++i) {
        if (seqs[i] < 0 || seqs[i] >= c->p.max_seqs)
            return fail(c, WHISPER_E_CAPACITY, "sequence " + std::to_string(seqs[i]) + " outside 0..max_seqs-1");
        if (seen[seqs[i]]) return fail(c, WHISPER_E_INVAL, "sequences must be distinct");
        seen[seqs[i]] = true;
        if (values[i] < 0) return fail(c, WHISPER_E_INVAL, std::string(what) + " must not be negative");
    }
    return WHISPER_OK;
}

// Row pointers of one call: not NULL if there are rows, row strides of a row
// at least (0: rows without gaps); *ld receives the stride.
whisper_status check_rows(whisper_cache* c, const void* p, int64_t given, int heads, bool any, int64_t* ld) {
    const int64_t row = (int64_t)heads * c->p.head_size;
    if (!p && any) return fail(c, WHISPER_E_INVAL, "device pointers must not be NULL");
    if (given != 0 && (given < row || given > ((int64_t)1 << 40)))
        return fail(c, WHISPER_E_INVAL, "a row stride must be 0 or at least " + std::to_string(row));
    *ld = given ? given : row;
    const size_t es = c->p.dtype == WHISPER_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(p) % es) return fail(c, WHISPER_E_INVAL, "a device pointer is not aligned to its type");
    return WHISPER_OK;
}

// Ids that are never chosen: in the vocabulary, and not all of it.
template <class H>
whisper_status check_suppressed(H* h, int n_vocab, const int32_t* suppress, int32_t n) {
    if (n < 0 || (n > 0 && !suppress)) return fail(h, WHISPER_E_INVAL, "suppress must not be NULL");
    std::set<int> ids;
    for (int i = 0; i < n; ++i) {
        if (suppress[i] < 0 || suppress[i] >= n_vocab) return fail(h, WHISPER_E_INVAL, "suppressed id out of range");
        ids.insert(suppress[i]);
    }
    if ((int)ids.size() >= n_vocab) return fail(h, WHISPER_E_INVAL, "every id would be suppressed");
    return WHISPER_OK;
}

whisper_status check_layer(whisper_cache* c, int32_t layer, bool all) {
    if (layer < (all ? -1 : 0) || layer >= c->p.n_layer)
        return fail(c, WHISPER_E_INVAL, "layer outside 0..n_layer-1" + std::string(all ? " and not -1" : ""));
    return WHISPER_OK;
}

}  // namespace

#define WMI_TRY(call)                                \
    do {                                             \
        const whisper_status st_ = (call);           \
        if (st_ != WHISPER_OK) return st_;           \
    } while (0)

extern "C" {

whisper_status whisper_cache_create(const whisper_cache_params* params, int device, whisper_cache** out) {
    return whisper_cache_create_packed(params, 0, device, out);
}

whisper_status whisper_cache_create_packed(const whisper_cache_params* params, int32_t bits, int device, whisper_cache** out) {
    whisper_cache* none = nullptr;
    if (!params || !out) return fail(none, WHISPER_E_INVAL, "params and out must not be NULL");
    const std::string bad = check_cache(*params);
    if (!bad.empty()) return fail(none, WHISPER_E_INVAL, bad);
    if (bits != 0 && bits != 4 && bits != 8) return fail(none, WHISPER_E_INVAL, "bits must be 0, 4 or 8");
    WMI_TRY(check_device(device));
    std::unique_ptr<whisper_cache> c(new (std::nothrow) whisper_cache());
    if (!c) return fail(none, WHISPER_E_NOMEM, "host allocation failed");
    c->p = *params;
    WMI_TRY(guarded(none, [&]() -> whisper_status {
        c->impl = wmi::make_paged_cache(*params, bits, device);
        return WHISPER_OK;
    }));
    *out = c.release();
    return WHISPER_OK;
}

void whisper_cache_destroy(whisper_cache* cache) { delete cache; }

const char* whisper_cache_error(const whisper_cache* cache) { return cache ? cache->err.c_str() : g_error.c_str(); }

whisper_status whisper_cache_set_stream(whisper_cache* cache, void* hip_stream) {
    WMI_TRY(usable(cache));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->set_stream(hip_stream);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_extend(whisper_cache* cache, const int32_t* seqs, const int32_t* counts, int32_t n) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_seqs(cache, seqs, counts, n, "counts"));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->extend(seqs, counts, n);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_append(whisper_cache* cache, int32_t layer, const void* k, const void* v, int64_t k_stride,
                                    int64_t v_stride) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_layer(cache, layer, true));
    const bool any = cache->impl->tokens() > 0;
    int64_t kl = 0, vl = 0;
    WMI_TRY(check_rows(cache, k, k_stride, cache->p.n_kv_head, any, &kl));
    WMI_TRY(check_rows(cache, v, v_stride, cache->p.n_kv_head, any, &vl));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->append(layer, k, v, kl, vl);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_attend(whisper_cache* cache, int32_t layer, const void* q, void* out, int64_t q_stride,
                                    int64_t out_stride, float scale) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_layer(cache, layer, false));
    const bool any = cache->impl->tokens() > 0;
    int64_t ql = 0, ol = 0;
    WMI_TRY(check_rows(cache, q, q_stride, cache->p.n_head, any, &ql));
    WMI_TRY(check_rows(cache, out, out_stride, cache->p.n_head, any, &ol));
    const int64_t el = cache->p.dtype == WHISPER_DTYPE_F32 ? 4 : 8;
    if (reinterpret_cast<uintptr_t>(q) % 16 || reinterpret_cast<uintptr_t>(out) % 16 || ql % el || ol % el)
        return fail(cache, WHISPER_E_INVAL, "queries and outputs must be 16-byte aligned, row strides multiples of 16 bytes");
    if (!(scale > 0.f && scale < 1e30f)) return fail(cache, WHISPER_E_INVAL, "scale must be positive and finite");
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->attend(layer, q, out, ql, ol, scale);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_truncate(whisper_cache* cache, const int32_t* seqs, const int32_t* lengths, int32_t n) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_seqs(cache, seqs, lengths, n, "lengths"));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->truncate(seqs, lengths, n);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_fork(whisper_cache* cache, int32_t src, const int32_t* dst, int32_t n) {
    WMI_TRY(usable(cache));
    if (src < 0 || src >= cache->p.max_seqs) return fail(cache, WHISPER_E_CAPACITY, "sequence outside 0..max_seqs-1");
    const std::vector<int32_t> none(n > 0 && n <= cache->p.max_seqs ? n : 0, 0);
    WMI_TRY(check_seqs(cache, dst, none.data() ? none.data() : dst, n, "dst"));
    for (int i = 0; i < n; ++i)
        if (dst[i] == src) return fail(cache, WHISPER_E_INVAL, "a sequence cannot be forked into itself");
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->fork(src, dst, n);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_reorder(whisper_cache* cache, const int32_t* seqs, const int32_t* from, int32_t n) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_seqs(cache, seqs, seqs, n, "from"));
    if (n > 0 && !from) return fail(cache, WHISPER_E_INVAL, "seqs and from must not be NULL");
    for (int i = 0; i < n; ++i)
        if (from[i] < 0 || from[i] >= cache->p.max_seqs)
            return fail(cache, WHISPER_E_CAPACITY, "sequence " + std::to_string(from[i]) + " outside 0..max_seqs-1");
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->reorder(seqs, from, n);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_compact(whisper_cache* cache) {
    WMI_TRY(usable(cache));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->compact();
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_read(whisper_cache* cache, int32_t layer, const int32_t* seqs, int32_t n, void* k, void* v,
                                  int64_t k_stride, int64_t v_stride) {
    WMI_TRY(usable(cache));
    WMI_TRY(check_layer(cache, layer, true));
    WMI_TRY(check_seqs(cache, seqs, seqs, n, "seqs"));
    bool any = false;
    for (int i = 0; i < n; ++i) any = any || cache->impl->book().length(seqs[i]) > 0;
    int64_t kl = 0, vl = 0;
    WMI_TRY(check_rows(cache, k, k_stride, cache->p.n_kv_head, any, &kl));
    WMI_TRY(check_rows(cache, v, v_stride, cache->p.n_kv_head, any, &vl));
    return guarded(cache, [&]() -> whisper_status {
        cache->impl->read(layer, seqs, n, k, v, kl, vl);
        return WHISPER_OK;
    });
}

whisper_status whisper_cache_info(whisper_cache* cache, int32_t seq, int32_t* length, int32_t* pages, int32_t* free_pages) {
    WMI_TRY(usable(cache));
    if (seq < 0 || seq >= cache->p.max_seqs) return fail(cache, WHISPER_E_CAPACITY, "sequence outside 0..max_seqs-1");
    const wmi::PageBook& b = cache->impl->book();
    if (length) *length = b.length(seq);
    if (pages) *pages = (int32_t)b.pages(seq).size();
    if (free_pages) *free_pages = b.free_pages();
    return WHISPER_OK;
}

whisper_status whisper_sampler_create(int32_t n_vocab, int32_t max_rows, int device, whisper_sampler** out) {
    whisper_sampler* none = nullptr;
    if (!out) return fail(none, WHISPER_E_INVAL, "out must not be NULL");
    if (n_vocab < 1 || n_vocab > (1 << 20)) return fail(none, WHISPER_E_INVAL, "n_vocab must be in 1..1048576");
    if (max_rows < 1 || max_rows > (1 << 16)) return fail(none, WHISPER_E_INVAL, "max_rows must be in 1..65536");
    WMI_TRY(check_device(device));
    std::unique_ptr<whisper_sampler> s(new (std::nothrow) whisper_sampler());
    if (!s) return fail(none, WHISPER_E_NOMEM, "host allocation failed");
    s->n_vocab = n_vocab;
    s->max_rows = max_rows;
    WMI_TRY(guarded(none, [&]() -> whisper_status {
        s->impl = wmi::make_sampler(n_vocab, max_rows, device);
        return WHISPER_OK;
    }));
    *out = s.release();
    return WHISPER_OK;
}

void whisper_sampler_destroy(whisper_sampler* sampler) { delete sampler; }

const char* whisper_sampler_error(const whisper_sampler* sampler) {
    return sampler ? sampler->err.c_str() : g_error.c_str();
}

whisper_status whisper_sampler_set_stream(whisper_sampler* sampler, void* hip_stream) {
    WMI_TRY(usable(sampler));
    return guarded(sampler, [&]() -> whisper_status {
        sampler->impl->set_stream(hip_stream);
        return WHISPER_OK;
    });
}

whisper_status whisper_sampler_options(whisper_sampler* sampler, const whisper_sampling* rows, int32_t n,
                                       const int32_t* suppress, int32_t n_suppress) {
    WMI_TRY(usable(sampler));
    if (n < 0 || n > sampler->max_rows) return fail(sampler, WHISPER_E_INVAL, "n must be in 0..max_rows");
    if (n > 0 && !rows) return fail(sampler, WHISPER_E_INVAL, "rows and suppress must not be NULL");
    for (int i = 0; i < n; ++i) {
        const char* bad = wmi::sampling_fault(rows[i]);
        if (bad) return fail(sampler, WHISPER_E_INVAL, "row " + std::to_string(i) + ": " + bad);
    }
    WMI_TRY(check_suppressed(sampler, sampler->n_vocab, suppress, n_suppress));
    return guarded(sampler, [&]() -> whisper_status {
        sampler->impl->options(rows, n, suppress, n_suppress);
        return WHISPER_OK;
    });
}

whisper_status whisper_sampler_run(whisper_sampler* sampler, const void* logits, int32_t dtype, int32_t n_rows,
                                   int64_t row_stride, const float* uniforms, int32_t* tokens, float* logprobs) {
    WMI_TRY(usable(sampler));
    if (dtype != WHISPER_DTYPE_F32 && dtype != WHISPER_DTYPE_BF16)
        return fail(sampler, WHISPER_E_INVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    if (n_rows < 0 || n_rows > sampler->max_rows) return fail(sampler, WHISPER_E_INVAL, "n_rows must be in 0..max_rows");
    if (row_stride != 0 && (row_stride < sampler->n_vocab || row_stride > ((int64_t)1 << 40)))
        return fail(sampler, WHISPER_E_INVAL, "row_stride must be 0 or at least n_vocab");
    if (n_rows == 0) return WHISPER_OK;
    if (!logits || !uniforms || !tokens) return fail(sampler, WHISPER_E_INVAL, "device pointers must not be NULL");
    const size_t es = dtype == WHISPER_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % es || reinterpret_cast<uintptr_t>(uniforms) % 4 ||
        reinterpret_cast<uintptr_t>(tokens) % 4 || reinterpret_cast<uintptr_t>(logprobs) % 4)
        return fail(sampler, WHISPER_E_INVAL, "a device pointer is not aligned to its type");
    return guarded(sampler, [&]() -> whisper_status {
        sampler->impl->run(logits, dtype, n_rows, row_stride ? row_stride : sampler->n_vocab, uniforms, tokens, logprobs);
        return WHISPER_OK;
    });
}

whisper_status whisper_beam_create(int32_t n_vocab, int32_t max_rows, int device, whisper_beam** out) {
    whisper_beam* none = nullptr;
    if (!out) return fail(none, WHISPER_E_INVAL, "out must not be NULL");
    if (n_vocab < 1 || n_vocab > (1 << 20)) return fail(none, WHISPER_E_INVAL, "n_vocab must be in 1..1048576");
    if (max_rows < 1 || max_rows > (1 << 16)) return fail(none, WHISPER_E_INVAL, "max_rows must be in 1..65536");
    WMI_TRY(check_device(device));
    std::unique_ptr<whisper_beam> b(new (std::nothrow) whisper_beam());
    if (!b) return fail(none, WHISPER_E_NOMEM, "host allocation failed");
    b->n_vocab = n_vocab;
    b->max_rows = max_rows;
    WMI_TRY(guarded(none, [&]() -> whisper_status {
        b->impl = wmi::make_beam(n_vocab, device);
        return WHISPER_OK;
    }));
    *out = b.release();
    return WHISPER_OK;
}

void whisper_beam_destroy(whisper_beam* beam) { delete beam; }

const char* whisper_beam_error(const whisper_beam* beam) { return beam ? beam->err.c_str() : g_error.c_str(); }

whisper_status whisper_beam_set_stream(whisper_beam* beam, void* hip_stream) {
    WMI_TRY(usable(beam));
    return guarded(beam, [&]() -> whisper_status {
        beam->impl->set_stream(hip_stream);
        return WHISPER_OK;
    });
}

whisper_status whisper_beam_options(whisper_beam* beam, const int32_t* suppress, int32_t n_suppress) {
    WMI_TRY(usable(beam));
    WMI_TRY(check_suppressed(beam, beam->n_vocab, suppress, n_suppress));
    return guarded(beam, [&]() -> whisper_status {
        beam->impl->options(suppress, n_suppress);
        return WHISPER_OK;
    });
}

whisper_status whisper_beam_run(whisper_beam* beam, const void* logits, int32_t dtype, int32_t n_groups, int32_t width,
                                int32_t n_best, int64_t row_stride, const float* scores, int32_t* parents, int32_t* tokens,
                                float* out_scores) {
    WMI_TRY(usable(beam));
    if (dtype != WHISPER_DTYPE_F32 && dtype != WHISPER_DTYPE_BF16)
        return fail(beam, WHISPER_E_INVAL, "dtype must be 0 (fp32) or 1 (bf16)");
    if (width < 1 || width > wmi::BEAM_WIDTH) return fail(beam, WHISPER_E_INVAL, "width must be in 1..32");
    if (n_best < 1 || n_best > wmi::BEAM_BEST) return fail(beam, WHISPER_E_INVAL, "n_best must be in 1..64");
    if (n_groups < 0 || n_groups > beam->max_rows / width)
        return fail(beam, WHISPER_E_INVAL, "n_groups x width must be in 0..max_rows");
    if (row_stride != 0 && (row_stride < beam->n_vocab || row_stride > ((int64_t)1 << 40)))
        return fail(beam, WHISPER_E_INVAL, "row_stride must be 0 or at least n_vocab");
    if (n_groups == 0) return WHISPER_OK;
    if (!logits || !scores || !parents || !tokens || !out_scores)
        return fail(beam, WHISPER_E_INVAL, "device pointers must not be NULL");
    const size_t es = dtype == WHISPER_DTYPE_F32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(logits) % es ||
        (reinterpret_cast<uintptr_t>(scores) | reinterpret_cast<uintptr_t>(parents) | reinterpret_cast<uintptr_t>(tokens) |
         reinterpret_cast<uintptr_t>(out_scores)) % 4)
        return fail(beam, WHISPER_E_INVAL, "a device pointer is not aligned to its type");
    return guarded(beam, [&]() -> whisper_status {
        beam->impl->run(logits, dtype, n_groups, width, n_best, row_stride ? row_stride : beam->n_vocab, scores, parents,
                        tokens, out_scores);
        return WHISPER_OK;
    });
}

}  // extern "C"
