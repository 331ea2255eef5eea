// Scan kernels for activations stored as _Float16.
#include "ssm_fwd.inl"
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<_Float16>(Use, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_scan<_Float16>(bool, bool, const SsmArgs &, hipStream_t);
