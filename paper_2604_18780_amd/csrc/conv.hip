// Short causal convolution along the sequence, one filter per channel, with SiLU; forwards, backwards, and continued from a
// ring of the last W tokens.
//
//   a[t,c] = bias[c] + sum_j w[c,j] u[t-W+1+j,c]        out = a * sigmoid(a)
//   da = g * silu'(a)     du[t] = sum_k w[W-1-k] da[t+k]     dw[j] = sum_t da[t] u[t-W+1+j]     dbias = sum_t da[t]
//
// Bound by memory: every input is read and every output written once (a run's first W-1 positions twice).  A thread owns 16 bytes
// of channels and walks a run of positions with the window in registers, the next four rows on their way while four are
// worked on; sixteen threads side by side make 256-byte rows.
// Measured, bfloat16, 4 x 100 000 positions of 640 channels, width 4: forwards 193 us (5.3 TB/s), backwards 371 us (4.1 TB/s; a sigmoid
// and fifteen multiply-adds for each element keep the vector units half busy, and 242 registers leave two waves a SIMD) and 15 us for the parameters' parts.
#include "encoder.h"

namespace semicrf_enc {

constexpr uint32_t OUTSIDE = 0x80000000u;  // an offset beyond any range

struct ConvArgs {
    const void *u, *gy, *ring;
    int64_t u_row, gy_row, y_row, gu_row;
    const float *weight, *bias;
    const int32_t *lengths, *seen;
    int B, T, C, W, run, runs;  // positions of a run (a multiple of 4), runs of a sequence
    unsigned cols;  // workgroups side by side over the channels
    bool linear;
    void *y, *ring_out, *gu;
    float *part;   // [blocks][C][W+1] sums for weight and bias
    int blocks;
    float *gw, *gb;
};

__device__ __forceinline__ float fast_sigmoid(float v)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504f * v));
}

template <class T, int W, int V> struct Filter {
    float w[W][V], b[V];
    __device__ __forceinline__ Filter(const ConvArgs &a, int c)
    {
#pragma unroll
        for (int e = 0; e < V; ++e) {
            b[e] = a.bias ? a.bias[c + e] : 0.0f;
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][e] = a.weight[(int64_t)(c + e) * W + j];
        }
    }
};

// Rows of a run behind one range check: those that lie before the first or behind the sequence's end read as zeros, and a
// thread's offsets are relative to the first row of its workgroup.
template <class T> struct RunRows {
    __amdgpu_buffer_rsrc_t rows;
    uint32_t first;  // of position 0 of this thread's run
    int bytes;
    __device__ __forceinline__ RunRows(const void *p, int64_t row, int64_t block_row, int64_t my_row, int c)
    {
        bytes = (int)row * (int)sizeof(T);
        rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>((const char *)p + block_row * bytes), 0, 0x7ffffff0, 0x00020000);
        first = (uint32_t)((my_row - block_row) * bytes) + (uint32_t)c * (uint32_t)sizeof(T);
    }
    __device__ __forceinline__ u4 load(int t, bool in) const
    {
        return __builtin_amdgcn_raw_buffer_load_b128(rows, in ? (int)(first + (uint32_t)(t * bytes)) : (int)OUTSIDE, 0, 0);
    }
    __device__ __forceinline__ void store(int t, bool in, u4 v) const
    {
        __builtin_amdgcn_raw_buffer_store_b128(v, rows, in ? (int)(first + (uint32_t)(t * bytes)) : (int)OUTSIDE, 0, 0);
    }
};
template <class T, int V> __device__ __forceinline__ void widen(u4 r, float (&o)[V])
{
    typedef T X __attribute__((ext_vector_type(V)));
    const X v = __builtin_bit_cast(X, r);
#pragma unroll
    for (int e = 0; e < V; ++e) o[e] = (float)v[e];
}
template <class T, int V> __device__ __forceinline__ u4 narrow(const float (&o)[V])
{
    typedef T X __attribute__((ext_vector_type(V)));
    typedef float F __attribute__((ext_vector_type(V)));
    F f;
#pragma unroll
    for (int e = 0; e < V; ++e) f[e] = o[e];
    return __builtin_bit_cast(u4, __builtin_convertvector(f, X));
}

template <class T, int W> __global__ __launch_bounds__(256) void k_conv_fwd(ConvArgs a)
{
    constexpr int V = PER16<T>;
    const int c = (int)(blockIdx.x % a.cols * 16 + threadIdx.x % 16) * V;
    const int64_t id0 = (int64_t)(blockIdx.x / a.cols) * 16, id = id0 + threadIdx.x / 16;
    if (c >= a.C || id >= (int64_t)a.B * a.runs) return;
    const int b = (int)(id / a.runs), t0 = (int)(id % a.runs) * a.run;
    const int64_t row0 = id0 / a.runs * a.T + id0 % a.runs * a.run, row = (int64_t)b * a.T + t0;
    const int seen = a.seen ? a.seen[b] : 0, L = seen < 0 ? 0 : length_of(a.lengths, b, a.T);
    const T *u = (const T *)a.u + (int64_t)b * a.T * a.u_row + c;
    const RunRows<T> in(a.u, a.u_row, row0, row, c), out(a.y, a.y_row, row0, row, c);
    const T *ring = a.ring ? (const T *)a.ring + ((int64_t)b * a.C + c) * W : nullptr;
    const int n = t0 + a.run < a.T ? a.run : a.T - t0, have = L - t0;  // rows to write, rows that exist
    u4 next[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) next[k] = in.load(k, k < have);
    const Filter<T, W, V> f(a, c);
    float win[W][V];  // win[j]: position t - W + 1 + j
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int t = t0 - W + 1 + j;
#pragma unroll
        for (int e = 0; e < V; ++e) win[j + 1][e] = 0.0f;
        if (t >= 0) {
            if (t < L) load_n<T, V>(u + t * a.u_row, win[j + 1]);
        } else if (ring && seen + t >= 0) {
#pragma unroll
            for (int e = 0; e < V; ++e) win[j + 1][e] = (float)ring[(int64_t)e * W + (seen + t) % W];
        }
    }
    for (int t = 0; t < n; t += 4) {
        u4 now[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) now[k] = next[k];
#pragma unroll
        for (int k = 0; k < 4; ++k) next[k] = in.load(t + 4 + k, t + 4 + k < have && t + 4 < n);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float o[V];
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) win[j][e] = win[j + 1][e];
            widen<T, V>(now[k], win[W - 1]);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                float v = f.b[e];
#pragma unroll
                for (int j = 0; j < W; ++j) v += f.w[j][e] * win[j][e];
                if (!a.linear) v *= fast_sigmoid(v);
                o[e] = t + k < have ? v : 0.0f;
            }
            out.store(t + k, t + k < n, narrow<T, V>(o));
        }
    }
    if (t0 == 0 && a.ring_out) {
        // the last W tokens, each at its position modulo W; this thread alone touches these channels' ring
        T *out = (T *)a.ring_out + ((int64_t)b * a.C + c) * W;
        if (L == 0 && (!ring || out == ring)) {
            if (!ring && out)
                for (int k = 0; k < V * W; ++k) out[k] = (T)0.0f;
            return;
        }
        const int n = (seen < 0 ? 0 : seen) + L;
        for (int j = 0; j < W; ++j) {
            int p = n - 1 - ((n - 1) % W - j + W) % W;  // newest position below n that is j mod W
            if (n == 0) p = -1;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                T v = (T)0.0f;
                if (L == 0) v = ring[(int64_t)e * W + j];
                else if (p >= seen) v = u[(int64_t)(p - seen) * a.u_row + e];
                else if (p >= 0 && ring) v = ring[(int64_t)e * W + j];
                out[(int64_t)e * W + j] = v;
            }
        }
    }
}

template <class T, int W> __global__ __launch_bounds__(256) void k_conv_bwd(ConvArgs a)
{
    constexpr int V = PER16<T>;
    __shared__ float part[4][16][V * (W + 1)];
    const int lane16 = threadIdx.x % 16, col0 = (int)(blockIdx.x % a.cols) * 16, c = (col0 + lane16) * V;
    const int64_t block = blockIdx.x / a.cols;
    float dw[W + 1][V];
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[j][e] = 0.0f;
    if (c < a.C) {
        const Filter<T, W, V> f(a, c);
        for (int64_t id = block * 16 + threadIdx.x / 16; id < (int64_t)a.B * a.runs; id += (int64_t)a.blocks * 16) {
            const int b = (int)(id / a.runs), t0 = (int)(id % a.runs) * a.run;
            const int64_t id0 = id - threadIdx.x / 16;
            const int64_t row0 = id0 / a.runs * a.T + id0 % a.runs * a.run, row = (int64_t)b * a.T + t0;
            const int L = length_of(a.lengths, b, a.T);
            const RunRows<T> in(a.u, a.u_row, row0, row, c), gin(a.gy, a.gy_row, row0, row, c), out(a.gu, a.gu_row, row0, row, c);
            const int n = t0 + a.run < a.T ? a.run : a.T - t0, have = L - t0;
            u4 nu[4], ng[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) nu[k] = in.load(k, k < have), ng[k] = gin.load(k, k < have);
            float win[W][V], da[W][V];
#pragma unroll
            for (int j = 0; j < W; ++j)
#pragma unroll
                for (int e = 0; e < V; ++e) win[j][e] = da[j][e] = 0.0f;
            const T *u = (const T *)a.u + (int64_t)b * a.T * a.u_row + c;
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int t = t0 - W + 1 + j;
                if (t >= 0 && t < L) load_n<T, V>(u + t * a.u_row, win[j + 1]);
            }
            // a gradient of u needs the W-1 positions behind it: rows n .. n+W-2 are looked at, and counted by the run they are in
            for (int t = 0; t < n + W - 1; t += 4) {
                u4 uu[4], gg[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) uu[k] = nu[k], gg[k] = ng[k];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const bool want = t + 4 + k < have && t + 4 < n + W - 1;
                    nu[k] = in.load(t + 4 + k, want), ng[k] = gin.load(t + 4 + k, want);
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float g[V];
#pragma unroll
                    for (int j = 0; j < W - 1; ++j)
#pragma unroll
                        for (int e = 0; e < V; ++e) win[j][e] = win[j + 1][e], da[j][e] = da[j + 1][e];
                    widen<T, V>(uu[k], win[W - 1]);
                    widen<T, V>(gg[k], g);
                    // rows that do not exist have g = 0, and so no share in anything
                    const float mine = t + k < n ? 1.0f : 0.0f;
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        float v = f.b[e];
#pragma unroll
                        for (int j = 0; j < W; ++j) v += f.w[j][e] * win[j][e];
                        const float s = fast_sigmoid(v);
                        const float d = a.linear ? g[e] : g[e] * s * (1.0f + v * (1.0f - s));
                        da[W - 1][e] = d;
                        const float m = d * mine;
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][e] += m * win[j][e];
                        dw[W][e] += m;
                    }
                    float o[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) {
                        o[e] = 0.0f;
#pragma unroll
                        for (int j = 0; j < W; ++j) o[e] += f.w[W - 1 - j][e] * da[j][e];
                    }
                    const int to = t + k - (W - 1);
                    out.store(to, to >= 0 && to < n, narrow<T, V>(o));
                }
            }
        }
    }
    // sixteen threads hold sums for the same channels: four in a wave, four waves
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int e = 0; e < V; ++e) {
            float s = dw[j][e];
            s += __shfl_xor(s, 16);
            s += __shfl_xor(s, 32);
            if (threadIdx.x % 64 < 16) part[threadIdx.x / 64][lane16][e * (W + 1) + j] = s;
        }
    __syncthreads();
    for (int k = threadIdx.x; k < 16 * V * (W + 1); k += 256) {
        const int col = k / (V * (W + 1)), at = k % (V * (W + 1));
        if ((col0 + col) * V < a.C) {
            const float s = part[0][col][at] + part[1][col][at] + part[2][col][at] + part[3][col][at];
            a.part[(block * a.C + (col0 + col) * V) * (W + 1) + at] = s;
        }
    }
}

// Sums over the workgroups' parts, in a fixed order: sixteen threads to an entry.
__global__ __launch_bounds__(256) void k_conv_params(ConvArgs a)
{
    const int per = a.W + 1, n = a.C * per, at = blockIdx.x * 16 + threadIdx.x / 16;
    double s = 0.0;
    if (at < n)
        for (int k = threadIdx.x % 16; k < a.blocks; k += 16) s += (double)a.part[(int64_t)k * n + at];
    for (int d = 1; d < 16; d *= 2) s += __shfl_xor(s, d);
    if (at < n && threadIdx.x % 16 == 0) {
        const int c = at / per, j = at % per;
        if (j < a.W) a.gw[(int64_t)c * a.W + j] = (float)s;
        else if (a.gb) a.gb[c] = (float)s;
    }
}

int conv_sizes(int B, int T, int C, int W)
{
    if (B < 1 || T < 1 || C < 1 || W < 1) return SEMICRF_EINVAL;
    if (C % 8 || W > 4 || T > (1 << 30) || (double)B * ((T + 7) / 8) * (C / 4) > 2e9) return SEMICRF_EUNSUPPORTED;
    return SEMICRF_OK;
}

// Positions of a run: 32, so that the W-1 positions read twice are a tenth, but as few as 8 where that leaves the chip (256
// compute units of 2048 threads) less than half filled.
int run_length(int B, int T, int C, int per16)
{
    const int64_t threads = (int64_t)B * T * (C / per16);
    int run = 32;
    while (run > 8 && threads / run < 256 * 1024) run /= 2;
    return run;
}

// Workgroups along the sequences in a backward call: two thousand in all keep the chip busy, and each leaves a row of sums.
int conv_blocks(int B, int T, int C, int per16)
{
    const int run = run_length(B, T, C, per16);
    const int64_t runs = (int64_t)B * ((T + run - 1) / run), cols = (C / per16 + 15) / 16;
    int64_t n = (runs + 15) / 16, most = 2048 / cols + 1;
    return (int)(n < most ? n : most);
}

template <class T, int W> void conv_launch(const ConvArgs &a, bool back, hipStream_t st)
{
    const unsigned rows = (unsigned)(((int64_t)a.B * a.runs + 15) / 16);
    if (!back) hipLaunchKernelGGL((k_conv_fwd<T, W>), dim3(a.cols * rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_conv_bwd<T, W>), dim3(a.cols * a.blocks), dim3(256), 0, st, a);
}
template <class T> void conv_launch_type(ConvArgs a, bool back, hipStream_t st)
{
    a.cols = (a.C / PER16<T> + 15) / 16;
    if (a.W == 1) conv_launch<T, 1>(a, back, st);
    else if (a.W == 2) conv_launch<T, 2>(a, back, st);
    else if (a.W == 3) conv_launch<T, 3>(a, back, st);
    else conv_launch<T, 4>(a, back, st);
}
int conv_run(const ConvArgs &a, int type, bool back, hipStream_t st)
{
    if (type == ACT_BF16) conv_launch_type<__bf16>(a, back, st);
    else if (type == ACT_F16) conv_launch_type<_Float16>(a, back, st);
    else conv_launch_type<float>(a, back, st);
    return launched();
}

}  // namespace semicrf_enc

using namespace semicrf_enc;

extern "C" {

int semicrf_conv_fwd(const void *u, int64_t u_row, const float *weight, const float *bias, const int32_t *lengths,
                     const int32_t *seen, const void *ring, int B, int T, int C, int W, unsigned flags, void *out,
                     int64_t out_row, void *ring_out, void *stream)
{
    if (int rc = conv_sizes(B, T, C, W)) return rc;
    const int type = act_type(flags);
    if (type < 0 || !weight || (ring && !seen) || u_row > (1 << 19) || out_row > (1 << 19) || !rows_ok(u, u_row, C, type) || !rows_ok(out, out_row, C, type))
        return SEMICRF_EINVAL;
    ConvArgs a = {};
    a.u = u; a.u_row = u_row; a.weight = weight; a.bias = bias; a.lengths = lengths; a.seen = seen; a.ring = ring;
    a.B = B; a.T = T; a.C = C; a.W = W; a.run = run_length(B, T, C, 16 / act_bytes(type));
    a.runs = (T + a.run - 1) / a.run;
    a.linear = (flags & SEMICRF_CONV_LINEAR) != 0;
    a.y = out; a.y_row = out_row; a.ring_out = ring_out;
    return conv_run(a, type, false, (hipStream_t)stream);
}

int semicrf_conv_bwd_workspace_bytes(int B, int T, int C, int W, size_t *bytes)
{
    if (!bytes) return SEMICRF_EINVAL;
    const int rc = conv_sizes(B, T, C, W);
    if (rc == SEMICRF_OK) {
        const int a = conv_blocks(B, T, C, 4), b = conv_blocks(B, T, C, 8);
        *bytes = align256((size_t)(a > b ? a : b) * C * (W + 1) * 4);
    }
    return rc;
}

int semicrf_conv_bwd(const void *u, int64_t u_row, const float *weight, const float *bias, const int32_t *lengths,
                     const void *grad_out, int64_t grad_out_row, int B, int T, int C, int W, unsigned flags,
                     void *workspace, size_t workspace_bytes, void *grad_u, int64_t grad_u_row, float *grad_weight,
                     float *grad_bias, void *stream)
{
    size_t need = 0;
    if (int rc = semicrf_conv_bwd_workspace_bytes(B, T, C, W, &need)) return rc;
    const int type = act_type(flags);
    if (type < 0 || !weight || !grad_weight || u_row > (1 << 19) || grad_out_row > (1 << 19) || grad_u_row > (1 << 19) || !rows_ok(u, u_row, C, type) ||
        !rows_ok(grad_out, grad_out_row, C, type) || !rows_ok(grad_u, grad_u_row, C, type))
        return SEMICRF_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < need) return SEMICRF_EWORKSPACE;
    ConvArgs a = {};
    a.u = u; a.u_row = u_row; a.weight = weight; a.bias = bias; a.lengths = lengths;
    a.gy = grad_out; a.gy_row = grad_out_row; a.gu = grad_u; a.gu_row = grad_u_row;
    a.B = B; a.T = T; a.C = C; a.W = W; a.run = run_length(B, T, C, 16 / act_bytes(type));
    a.runs = (T + a.run - 1) / a.run;
    a.linear = (flags & SEMICRF_CONV_LINEAR) != 0;
    a.part = (float *)workspace; a.gw = grad_weight; a.gb = grad_bias;
    a.blocks = conv_blocks(B, T, C, act_bytes(type) == 4 ? 4 : 8);
    const hipStream_t st = (hipStream_t)stream;
    if (int rc = conv_run(a, type, true, st)) return rc;
    hipLaunchKernelGGL(k_conv_params, dim3((C * (W + 1) + 15) / 16), dim3(256), 0, st, a);
    return launched();
}

}  // extern "C"
