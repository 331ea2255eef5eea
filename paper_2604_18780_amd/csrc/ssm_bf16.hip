// Scan kernels for activations stored as __bf16.
#include "ssm_bwd.inl"
#include "ssm_fwd.inl"

template int semicrf_enc::ssm_scan<__bf16>(bool, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_grad<__bf16>(const SsmArgs &, hipStream_t);
