// Scan kernels for activations stored as float.
#include "ssm_bwd.inl"
#include "ssm_fwd.inl"

template int semicrf_enc::ssm_scan<float>(bool, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_grad<float>(const SsmArgs &, hipStream_t);
