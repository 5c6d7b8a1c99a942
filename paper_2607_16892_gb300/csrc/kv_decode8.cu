// The kernel for few rows on caches of 8 bits.
#include "kv_decode.cuh"

namespace kvdro {

cudaError_t kv_decode8_prepare() { return prepare_all<true, false>(); }

cudaError_t launch_kv_decode8(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s) {
    return launch_any<true, false>(a, maps, rows, early, sms, s);
}

}  // namespace kvdro
