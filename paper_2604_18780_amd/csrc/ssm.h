// Selective state space scan: arguments of the kernels, and how a call is cut into pieces.
//
//   delta_t = softplus(dt_t + dt_bias),   l_t = delta_t * rate,   u_t = delta_t x_t         (each head)
//   H_t = e^{l_t} H_{t-1} + u_t B_t^T     [P x N]                 y_t = H_t C_t + skip x_t
//
// With c_t = l_1 + ... + l_t the output is a masked product, y_i = sum_{j<=i} e^{c_i-c_j} (C_i . B_j) u_j, and so are the
// gradients: with G_t the gradient of H_t (G_t = e^{l_{t+1}} G_{t+1} + dy_t C_t^T),
//   dC_i = sum_{j<=i} e^{c_i-c_j} (dy_i . u_j) B_j      (forwards,  state H)
//   du_j = sum_{i>=j} e^{c_i-c_j} (B_j . C_i) dy_i      (backwards, state G)
//   dB_j = sum_{i>=j} e^{c_i-c_j} (u_j . dy_i) C_i      (backwards, state G)
// Blocks of positions go through the matrix cores, the state from block to block in registers.  Time is cut into segments so that
// there are workgroups enough for the chip; states at their boundaries come from a scan that keeps only the state, chained by
// k_ssm_chain.
#ifndef SEMICRF_SSM_H
#define SEMICRF_SSM_H

#include "encoder.h"

namespace semicrf_enc {

struct SsmArgs {
    const void *x, *b, *c, *dt, *gy;
    int64_t x_row, b_row, c_row, dt_row, gy_row;
    const float *rate, *skip, *dt_bias;
    const int32_t *lengths;
    const float *state;       // [B,H,P,N] or null: zeros
    const float *grad_last;   // [B,H,P,N] or null: gradient of the state after the last token
    int B, T, H, P, G, N;
    int seg, nseg;            // positions of a segment (a multiple of 64) and how many there are
    int heads, chunks;        // heads of a group that a workgroup of the gradient kernels takes, and how many such there are
    void *y;
    int64_t y_row;
    float *state_out;         // [B,H,P,N] or null
    void *gx, *gb, *gc, *gdt;
    int64_t gx_row, gb_row, gc_row, gdt_row;
    float *grate, *gskip, *gbias, *gstate;
    // workspace
    float *hs, *gs;           // [B*H][nseg+1][P][N] states, and gradients of states, at the segments' boundaries
    float *kept;              // [B*H][nseg] what a state keeps over a segment
    float *partc, *partb;     // [chunks][B*T][G][N] gradients of C and B by workgroup, where there are several
    float *rint, *dlin, *qint, *xdu;  // [B*H][T] see k_ssm_steps
    double *skipp;            // [B*H][nseg] sums for the skip
    double *cross;            // [B*H][nseg+1][P*N/256] pairs that cross a segment's boundary, by wave of k_ssm_chain
    double *headp;            // [B*H*nseg][2] sums for rate and bias
};

// Positions of a block of the gradient kernels.  Blocks of 64 read a state half as often, but want 250 registers, two waves to a SIMD,
// where blocks of 32 run three: gradients of 4 x 100 000 tokens, 8 heads of 64, 64 states, bfloat16 2365 us with blocks of 64 and
// 1713 with blocks of 32 (16 x 4000 tokens, 32 heads of 16, 32 states 765 and 568).
// Heads that a workgroup of the gradient kernels takes where B and C are shared: one needs fewer registers, but leaves a part of the
// gradients of B and C for each head (1814 us instead of 1713), four spill.
constexpr int GRAD_BLOCK = 32, GRAD_HEADS = 2;

// One instantiation per storage type, each in a translation unit of its own: outputs, or states alone (forwards, or both ways in
// one launch); and the gradient kernels.
template <class T> int ssm_scan(bool out, bool both, const SsmArgs &a, hipStream_t st);
extern template int ssm_scan<float>(bool, bool, const SsmArgs &, hipStream_t);
extern template int ssm_scan<_Float16>(bool, bool, const SsmArgs &, hipStream_t);
extern template int ssm_scan<__bf16>(bool, bool, const SsmArgs &, hipStream_t);
template <class T> int ssm_grad(const SsmArgs &a, hipStream_t st);
extern template int ssm_grad<float>(const SsmArgs &, hipStream_t);
extern template int ssm_grad<_Float16>(const SsmArgs &, hipStream_t);
extern template int ssm_grad<__bf16>(const SsmArgs &, hipStream_t);

}  // namespace semicrf_enc

#endif
