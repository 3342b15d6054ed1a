// The few-row attention kernel and the join over rows in two places, a shared prefix's
// and each sequence's own (kv4_few.cuh).
#define ACES_FILE 13  // site numbers of the checked build
#include "kv4_few.cuh"

namespace aces {

template cudaError_t launch_kv4_join<KV4_SPLIT>(const Kv4Att &, const Kv4Ws &, int, int, cudaStream_t);
template cudaError_t launch_kv4_few<KV4_SPLIT>(const Kv4Att &, void *, int, cudaStream_t);

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_few_split(unsigned long long out[3]) { return check_take(out); }
#endif

}  // namespace aces
