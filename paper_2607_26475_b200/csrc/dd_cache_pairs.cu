// The kernels of attention over listed pages with two query tokens to a unit (dd_cache_sparse.cu), compiled by themselves.
#include "dd_cache_attn.cuh"

int dd_cache_pairs_launch(const char* who, ca_args& args, int format, int blocks, int head_dim, cudaStream_t stream) {
  return ca_launch(who, args, ca_pick<2>(format, head_dim, 1), 0, blocks, 1, head_dim, stream);
}
