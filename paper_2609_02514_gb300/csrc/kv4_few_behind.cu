// The few-row attention kernel and the join over each sequence's own rows, behind a shared prefix (kv4_few.cuh).
#define ACES_FILE 12  // site numbers of the checked build
#include "kv4_few.cuh"

namespace aces {

template cudaError_t launch_kv4_join<KV4_BEHIND>(const Kv4Att &, const Kv4Ws &, int, int, cudaStream_t);
template cudaError_t launch_kv4_few<KV4_BEHIND>(const Kv4Att &, void *, int, cudaStream_t);

#ifdef ACES_CHECKED
cudaError_t check_take_kv4_few_behind(unsigned long long out[3]) { return check_take(out); }
cudaError_t check_set_late(int late) { return cudaMemcpyToSymbol(g_late, &late, sizeof(late)); }
#endif

}  // namespace aces
