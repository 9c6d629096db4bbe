// Attention of many query tokens, heads of 128 elements (attention.cuh).
#include "attention.cuh"

namespace cake {
namespace serving {
namespace attn {

int launch_128(const Args& a, const Maps& m, int kind, const DeviceInfo& di, cudaStream_t s) { return launch_kind<128>(a, m, kind, di, s); }

}  // namespace attn
}  // namespace serving
}  // namespace cake
