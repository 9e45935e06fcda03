#include "kvq.cuh"
namespace wedlm {
bool kvq_tensor_supported(const wedlm_config_t*) { return false; }
KvqLayout plan_kvq_tensor(const wedlm_config_t*) { return KvqLayout{}; }
int launch_kvq_tensor(const Shape&, const KvqLayout&, const void*, const KvqView&, const int32_t*, const int32_t*, void*, void*, int32_t*, cudaStream_t) { return WEDLM_ERR_UNSUPPORTED; }
}
