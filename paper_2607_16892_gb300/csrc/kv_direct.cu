// The kernel for few rows, with prefixes in front of the requests' own tokens, on caches of 16 bits.
#include "kv_decode.cuh"

namespace kvdro {

cudaError_t kv_direct_prepare() { return prepare_all<false, true>(); }

cudaError_t launch_kv_direct(const AttendArgs& a, const KvMaps& maps, int rows, int sms, cudaStream_t s) {
    return launch_any<false, true>(a, maps, rows, false, sms, s);
}

}  // namespace kvdro
