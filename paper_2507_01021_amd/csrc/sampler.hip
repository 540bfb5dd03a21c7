// The sampler's device side: options in device memory and the launch.
#include <string.h>

#include <algorithm>
#include <vector>

#include "device.h"
#include "sampler.h"
#include "sampling.h"

namespace wmi {

namespace {

class SamplerImpl final : public Sampler {
   public:
    SamplerImpl(int n_vocab, int max_rows, int device) : V_(n_vocab), R_(max_rows), dev_(device) {
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        const size_t words = (size_t)V_ / 32 + 2;
        void* q = nullptr;
        const size_t head = (R_ * sizeof(SampleRow) + words * sizeof(unsigned) + 255) / 256 * 256;
        if (hipMalloc(&q, head + sample_ws_bytes(R_)) != hipSuccess) {
            (void)hipGetLastError();
            throw ArgError(WHISPER_E_NOMEM, "device allocation of the sampler's options failed");
        }
        rows_ = static_cast<SampleRow*>(q);
        never_ = reinterpret_cast<unsigned*>(rows_ + R_);
        ws_ = static_cast<unsigned char*>(q) + head;
        host_.assign(R_, SampleRow{1.f, 0, 1.f, 0.f});
        WMI_HIP(hipMemcpy(rows_, host_.data(), R_ * sizeof(SampleRow), hipMemcpyHostToDevice));
        const std::vector<unsigned> none(words, 0u);
        WMI_HIP(hipMemcpy(never_, none.data(), words * sizeof(unsigned), hipMemcpyHostToDevice));
    }
    ~SamplerImpl() override {
        if (dev_ == WHISPER_NO_DEVICE) return;
        int old = -1;
        (void)hipGetDevice(&old);
        (void)hipSetDevice(dev_);
        (void)hipStreamSynchronize(st_);
        if (rows_) (void)hipFree(rows_);
        if (old >= 0) (void)hipSetDevice(old);
    }
    void set_stream(void* s) override {
        if (dev_ == WHISPER_NO_DEVICE || s == st_) return;
        DeviceScope scope(dev_);
        if (capturing(st_)) throw ArgError(WHISPER_E_STATE, "the stream is recording a graph: only run may be recorded");
        WMI_HIP(hipStreamSynchronize(st_));
        st_ = static_cast<hipStream_t>(s);
    }
    // Waits for the work enqueued so far: options change between steps rarely.
    void options(const whisper_sampling* rows, int n, const int32_t* suppress, int n_suppress) override {
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        if (capturing(st_)) throw ArgError(WHISPER_E_STATE, "the stream is recording a graph: only run may be recorded");
        std::vector<SampleRow> h(n);
        for (int i = 0; i < n; ++i) h[i] = SampleRow{rows[i].temperature, rows[i].top_k, rows[i].top_p, rows[i].min_p};
        std::vector<unsigned> m((size_t)V_ / 32 + 2, 0u);
        for (int i = 0; i < n_suppress; ++i) m[suppress[i] >> 5] |= 1u << (suppress[i] & 31);
        WMI_HIP(hipStreamSynchronize(st_));
        if (n) WMI_HIP(hipMemcpy(rows_, h.data(), h.size() * sizeof(SampleRow), hipMemcpyHostToDevice));
        WMI_HIP(hipMemcpy(never_, m.data(), m.size() * sizeof(unsigned), hipMemcpyHostToDevice));
        use_never_ = n_suppress > 0;
        std::copy(h.begin(), h.end(), host_.begin());
        filters_ = false;
        for (const SampleRow& x : host_) filters_ = filters_ || (x.temperature > 0.f && (x.top_k > 0 || x.top_p < 1.f));
    }
    void run(const void* logits, int dtype, int n_rows, int64_t ld, const float* u, int32_t* tok, float* logp) override {
        if (dev_ == WHISPER_NO_DEVICE) throw ArgError(WHISPER_E_STATE, "the sampler has no device");
        DeviceScope scope(dev_);
        // a recorded run may meet other options and other suppressed ids at its replay
        const bool rec = capturing(st_), filters = filters_ || rec;
        const SampleArgs a{logits, ld, V_, rows_, use_never_ || rec ? never_ : nullptr, u, tok, logp, nullptr, nullptr, nullptr, nullptr, nullptr, ws_, 0};
        if (dtype == WHISPER_DTYPE_BF16) sample_rows<bf16>(a, n_rows, filters, st_);
        else sample_rows<float>(a, n_rows, filters, st_);
        WMI_HIP(hipGetLastError());
    }

   private:
    int V_, R_, dev_;
    hipStream_t st_ = nullptr;
    SampleRow* rows_ = nullptr;
    unsigned* never_ = nullptr;
    unsigned char* ws_ = nullptr;
    bool use_never_ = false, filters_ = false;
    std::vector<SampleRow> host_;  // the rows' options
};

}  // namespace

std::unique_ptr<Sampler> make_sampler(int n_vocab, int max_rows, int device) {
    return std::unique_ptr<Sampler>(new SamplerImpl(n_vocab, max_rows, device));
}

}  // namespace wmi
