// Linear attention's chunked kernels, fp16 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_fp16(const Cores& cs, const Split& p, hipStream_t s) { return chunks_launch<f16_t>(cs, p, s); }

}  // namespace rn18
