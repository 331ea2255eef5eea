// Scan kernels for activations stored as __bf16.
#include "ssm_fwd.inl"
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<__bf16>(Use, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_scan<__bf16>(bool, bool, const SsmArgs &, hipStream_t);
