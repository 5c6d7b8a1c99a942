// The kernel for chunks on caches of 16 bits.
#include "kv_chunk.cuh"

namespace kvdro {

size_t kv_chunk_piece_bytes(int sms) { return (size_t)sms * 2 * Shape<128, false>::kPieceFloats * sizeof(float); }

// The launch for few tiles has kJoinCtas CTAs per SM, and a tile takes kJoinGroups of them at least.
bool kv_join_few(int64_t tiles, int sms) {
    return tiles <= kFewTiles && tiles * kJoinGroups <= (int64_t)sms * kJoinCtas && sms <= kJoinMost;
}

cudaError_t kv_chunk_prepare() { return prepare_all<false>(); }

cudaError_t launch_kv_chunk(const AttendArgs& a, const KvMaps& maps, bool after_few, int sms, cudaStream_t s) {
    return launch_any<false>(a, maps, after_few, sms, s);
}

}  // namespace kvdro
