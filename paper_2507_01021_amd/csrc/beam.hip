// The beam selection's device side: suppressed ids and workspace, the launch.
#include <vector>

#include "beam.h"
#include "beaming.h"
#include "device.h"

namespace wmi {

namespace {

class BeamImpl final : public Beam {
   public:
    BeamImpl(int n_vocab, int device) : V_(n_vocab), dev_(device) {
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        const std::vector<unsigned> none((size_t)V_ / 32 + 2, 0u);
        const size_t head = (none.size() * sizeof(unsigned) + 255) / 256 * 256;
        void* q = nullptr;
        if (hipMalloc(&q, head + beam_ws_bytes()) != hipSuccess) {
            (void)hipGetLastError();
            throw ArgError(WHISPER_E_NOMEM, "device allocation of the beam selection's workspace failed");
        }
        never_ = static_cast<unsigned*>(q);
        ws_ = static_cast<unsigned char*>(q) + head;
        WMI_HIP(hipMemcpy(never_, none.data(), none.size() * sizeof(unsigned), hipMemcpyHostToDevice));
    }
    ~BeamImpl() override {
        if (dev_ == WHISPER_NO_DEVICE) return;
        int old = -1;
        (void)hipGetDevice(&old);
        (void)hipSetDevice(dev_);
        (void)hipStreamSynchronize(st_);
        if (never_) (void)hipFree(never_);
        if (old >= 0) (void)hipSetDevice(old);
    }
    void set_stream(void* s) override {
        if (dev_ == WHISPER_NO_DEVICE || s == st_) return;
        DeviceScope scope(dev_);
        no_capture();
        WMI_HIP(hipStreamSynchronize(st_));
        st_ = static_cast<hipStream_t>(s);
    }
    // Waits for the work enqueued so far: the list changes rarely.
    void options(const int32_t* suppress, int n_suppress) override {
        if (dev_ == WHISPER_NO_DEVICE) return;
        DeviceScope scope(dev_);
        no_capture();
        std::vector<unsigned> m((size_t)V_ / 32 + 2, 0u);
        for (int i = 0; i < n_suppress; ++i) m[suppress[i] >> 5] |= 1u << (suppress[i] & 31);
        WMI_HIP(hipStreamSynchronize(st_));
        WMI_HIP(hipMemcpy(never_, m.data(), m.size() * sizeof(unsigned), hipMemcpyHostToDevice));
        use_never_ = n_suppress > 0;
    }
    void run(const void* logits, int dtype, int n_groups, int width, int n_best, int64_t ld, const float* scores,
             int32_t* parents, int32_t* tokens, float* out) override {
        if (dev_ == WHISPER_NO_DEVICE) throw ArgError(WHISPER_E_STATE, "the beam selection has no device");
        DeviceScope scope(dev_);
        // a recorded run may meet other suppressed ids at its replay
        const BeamArgs a{logits, ld, V_, width, n_best, use_never_ || capturing(st_) ? never_ : nullptr, scores,
                         parents, tokens, out, reinterpret_cast<BeamPiece*>(ws_),
                         reinterpret_cast<u64*>(ws_ + sizeof(BeamPiece) * BEAM_PIECES), 0, 0};
        if (dtype == WHISPER_DTYPE_BF16) beam_rows<bf16>(a, n_groups, st_);
        else beam_rows<float>(a, n_groups, st_);
        WMI_HIP(hipGetLastError());
    }

   private:
    int V_, dev_;
    hipStream_t st_ = nullptr;
    unsigned* never_ = nullptr;
    unsigned char* ws_ = nullptr;
    bool use_never_ = false;

    void no_capture() const {
        if (capturing(st_)) throw ArgError(WHISPER_E_STATE, "the stream is recording a graph: only run may be recorded");
    }
};

}  // namespace

std::unique_ptr<Beam> make_beam(int n_vocab, int device) {
    return std::unique_ptr<Beam>(new BeamImpl(n_vocab, device));
}

}  // namespace wmi
