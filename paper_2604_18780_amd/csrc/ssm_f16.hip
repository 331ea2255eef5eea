// Sweeps of the state space scan for activations stored as _Float16.
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<_Float16>(Use, bool, const SsmArgs &, hipStream_t);
