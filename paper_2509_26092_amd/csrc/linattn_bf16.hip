// Linear attention's chunked kernels, bf16 storage.
#include "linattn.h"

namespace rn18 {

int chunks_launch_bf16(const Cores& cs, const Split& p, hipStream_t s) { return chunks_launch<bf16_t>(cs, p, s); }

}  // namespace rn18
