// Linear attention's chunked kernels, fp16 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_fp16(const Core& c, const Split& p, float* states, hipStream_t s) {
  return chunks_launch<f16_t>(c, p, states, s);
}

}  // namespace rn18
