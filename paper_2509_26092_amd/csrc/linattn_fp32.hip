// Linear attention's chunked kernels, fp32 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_fp32(const Core& c, const Split& p, float* states, hipStream_t s) {
  return chunks_launch<float>(c, p, states, s);
}

}  // namespace rn18
