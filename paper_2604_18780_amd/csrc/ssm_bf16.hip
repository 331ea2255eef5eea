// Sweeps of the state space scan for activations stored as __bf16.
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<__bf16>(Use, bool, const SsmArgs &, hipStream_t);
