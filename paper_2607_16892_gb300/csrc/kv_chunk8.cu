// The kernel for chunks on caches of 8 bits.
#include "kv_chunk.cuh"

namespace kvdro {

cudaError_t kv_chunk8_prepare() { return prepare_all<true>(); }

cudaError_t launch_kv_chunk8(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s) {
    return launch_any<true>(a, maps, after_few, sms, s);
}

}  // namespace kvdro
