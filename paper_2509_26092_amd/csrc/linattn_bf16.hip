// Linear attention's chunked kernels, bf16 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_bf16(const Core& c, const Split& p, float* states, hipStream_t s) {
  return chunks_launch<bf16_t>(c, p, states, s);
}

}  // namespace rn18
