// Beam selection (host interface, no HIP types): the ids never chosen in
// device memory, and the launch of the choice. Arguments are checked by the C
// ABI layer.
#pragma once

#include <memory>

#include "../../include/whisper_mi355x.h"

namespace wmi {

constexpr int BEAM_WIDTH = 32, BEAM_BEST = 64;  // beams of a group, continuations of a group

class Beam {
   public:
    virtual ~Beam() {}
    virtual void set_stream(void* hip_stream) = 0;
    virtual void options(const int32_t* suppress, int n_suppress) = 0;
    virtual void run(const void* logits, int dtype, int n_groups, int width, int n_best, int64_t ld, const float* scores,
                     int32_t* parents, int32_t* tokens, float* out_scores) = 0;
};

// device WHISPER_NO_DEVICE: argument checks alone. Throws ArgError or DeviceError.
std::unique_ptr<Beam> make_beam(int n_vocab, int device);

}  // namespace wmi
