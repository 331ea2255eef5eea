// Scan kernels for activations stored as float.
#include "ssm_fwd.inl"
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<float>(Use, bool, const SsmArgs &, hipStream_t);
template int semicrf_enc::ssm_scan<float>(bool, bool, const SsmArgs &, hipStream_t);
