// The few-row attention kernel and the join for calls of their own (kv4_few.cuh).
#define ACES_FILE 8  // site numbers of the checked build
#include "kv4_few.cuh"

namespace aces {

template cudaError_t launch_kv4_join<KV4_ALONE>(const Kv4Att &, const Kv4Ws &, int, int, cudaStream_t);
template cudaError_t launch_kv4_few<KV4_ALONE>(const Kv4Att &, void *, int, cudaStream_t);

size_t kv4_few_ws(int n, int G, int D, int nsm) { return kv4_ws_bytes(2 * nsm, 8 * few_tiles(n, G), D); }

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_few(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
