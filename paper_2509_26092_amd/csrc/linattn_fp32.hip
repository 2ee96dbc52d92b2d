// Linear attention's chunked kernels, fp32 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_fp32(const Cores& cs, const Split& p, hipStream_t s) { return chunks_launch<float>(cs, p, s); }

}  // namespace rn18
