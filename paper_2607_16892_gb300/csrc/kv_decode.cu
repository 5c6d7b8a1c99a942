// The kernel for few rows on caches of 16 bits.
#include "kv_decode.cuh"

namespace kvdro {

size_t kv_decode_piece_bytes(int sms) { return (size_t)sms * kMostCtas * 2 * kPieceFloats<128> * sizeof(float); }
int kv_decode_ctas(int sms) { return sms * kMostCtas; }

cudaError_t kv_decode_prepare() { return prepare_all<false, false>(); }

cudaError_t launch_kv_decode(const AttendArgs& a, const KvMaps& maps, int rows, bool early, int sms, cudaStream_t s) {
    return launch_any<false, false>(a, maps, rows, early, sms, s);
}

}  // namespace kvdro
