// Sweeps of the state space scan for activations stored as float.
#include "ssm_sweep.inl"

template int semicrf_enc::ssm_sweep<float>(Use, bool, const SsmArgs &, hipStream_t);
