// Sampler (host interface, no HIP types): per-row options and the ids never
// chosen in device memory, and the launch of the choice. Arguments are checked
// by the C ABI layer.
#pragma once

#include <memory>

#include "../../include/whisper_mi355x.h"

namespace wmi {

// What is wrong with a row's options, or null.
inline const char* sampling_fault(const whisper_sampling& o) {
    if (!(o.temperature >= 0.f && o.temperature <= 3.402823466e38f)) return "temperature must be finite and >= 0";
    if (o.top_k < 0) return "top_k must be >= 0";
    if (!(o.top_p > 0.f && o.top_p <= 1.f)) return "top_p must be in (0, 1]";
    if (!(o.min_p >= 0.f && o.min_p <= 1.f)) return "min_p must be in 0..1";
    return nullptr;
}

class Sampler {
   public:
    virtual ~Sampler() {}
    virtual void set_stream(void* hip_stream) = 0;
    virtual void options(const whisper_sampling* rows, int n, const int32_t* suppress, int n_suppress) = 0;
    virtual void run(const void* logits, int dtype, int n_rows, int64_t ld, const float* uniforms, int32_t* tokens,
                     float* logprobs) = 0;
};

// device WHISPER_NO_DEVICE: argument checks alone. Throws ArgError or DeviceError.
std::unique_ptr<Sampler> make_sampler(int n_vocab, int max_rows, int device);

}  // namespace wmi
