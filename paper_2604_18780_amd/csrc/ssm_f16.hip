// Scan kernels for activations stored as _Float16.
#include "ssm_bwd.inl"
#include "ssm_fwd.inl"

template int semicrf_enc::ssm_scan<_Float16>(bool, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_grad<_Float16>(const SsmArgs &, hipStream_t);
