// The fp32 kernels of attention_forms.h.
#include "attention_forms.h"

namespace mslt {
hipError_t form_fwd_f32(const FormArgs& a, hipStream_t s) { return forms::fwd_t<float>(a, s); }
hipError_t form_bwd_f32(const FormArgs& a, hipStream_t s) { return forms::bwd_t<float>(a, s); }
}  // namespace mslt
