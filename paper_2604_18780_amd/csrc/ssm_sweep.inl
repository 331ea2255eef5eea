// The sweep of the state space scan over one segment of one head: see ssm.h for the mathematics.
//
// One wave per (sequence, head, segment, tile of 64 value columns).  A block of 32 positions is staged in LDS row by row;
// what the products need with positions as the inner index is read from there transposed (ds_read_b64_tr_b16).
//   scores  M[j,i] = K_j . Q_i        rows j, columns i: a lane holds four keys of one query,
//   output  O[v,i] = sum_j V[j,v] M[j,i] w[j,i] + e^{c_i} sum_k S[k,v] Q[i,k]
//   state   S[k,v] = e^{c_32} S[k,v] + sum_j w_j K[j,k] V[j,v]
// The rows a lane holds of a 16 x 16 result are the inner indexes it holds of the next product's operand (4g..4g+3 of each
// of two tiles, g = lane / 16), so scores and state go from one product into the next without leaving registers.
#include "ssm_block.h"

namespace semicrf_enc {

// ---- staging ------------------------------------------------------------------------------------------------------

// One operand's rows: BLOCK rows of `dim` elements (W with padding columns of zeros), rows outside the sequence zeros.
template <class T, int W> struct Rows {
    static constexpr int E = PER16<T>, S = W + E, CH = BLOCK * W / E / 64, PR = W / E;
    const T *base;
    int64_t row;
    int dim;
    u4 r[CH];
    // row r holds position base_t + r, or base_t + BLOCK-1 - r
    template <bool REV> __device__ __forceinline__ void fetch(int base_t, int L, int lane)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = lane + 64 * i, k = at / PR, col = at % PR * E, t = base_t + (REV ? BLOCK - 1 - k : k);
            r[i] = t < L && col < dim ? *(const u4 *)(base + t * row + col) : (u4)0u;
        }
    }
    __device__ __forceinline__ void put(T *tile, int lane) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = lane + 64 * i;
            *(u4 *)(tile + at / PR * S + at % PR * E) = r[i];
        }
    }
};

struct Steps32 {  // of one block, by row of the staged tiles
    double c[BLOCK];      // log2 of what has been kept up to a query
    float out[BLOCK];     // e^c
    float in[BLOCK];      // what the state at the block's end keeps of a key, times the key's scale
    float key[BLOCK];     // the key's scale
    float query[BLOCK];   // the query's scale
};



template <class T, int DK, int DV, Use USE, bool REV>
__global__ __launch_bounds__(64) void k_ssm_sweep(SsmArgs a)
{
    constexpr int KT = DK / 16, VT = DV / 16, KS = DK / 32;
    constexpr int RAW = Parts<T>::raw, MADE = Parts<T>::made;
    constexpr bool OUT = USE != USE_STATE;
    constexpr bool EXTRA = USE == USE_DC || USE == USE_DU;   // a fourth operand, multiplied into the output
    constexpr int HELD = EXTRA ? 3 : MADE;                   // parts of the state: the steps' gradients are sums of both signs
    constexpr bool WIDE_N = USE == USE_DC || USE == USE_DB;  // values are rows of B or C
    constexpr int SK = DK + PER16<T>, SV = DV + PER16<T>;
    __shared__ __attribute__((aligned(16))) T sq[OUT ? BLOCK * SK : 8];
    __shared__ __attribute__((aligned(16))) T sk[BLOCK * SK];
    __shared__ __attribute__((aligned(16))) T sv[BLOCK * SV];
    __shared__ __attribute__((aligned(16))) T se[EXTRA ? BLOCK * SV : 8];
    __shared__ Steps32 ss;

    const int lane = threadIdx.x, g = lane >> 4, i16 = lane & 15;
    const int vdim = WIDE_N ? a.N : a.P, kdim = WIDE_N ? a.P : a.N;
    const int ntile = (vdim + DV - 1) / DV;
    // heads of one segment follow each other on one XCD (workgroups go round the eight in turn): they share B and C
    const int unit = (blockIdx.x % 8) + 8 * (blockIdx.x / 8 / (a.H * ntile)), within = blockIdx.x / 8 % (a.H * ntile);
    if (unit >= a.B * a.nseg) return;
    const int b = unit / a.nseg, seg = unit % a.nseg, h = within / ntile, tile = within % ntile, v0 = tile * DV;
    const int grp = h / (a.H / a.G);
    const int L = length_of(a.lengths, b, a.T);
    const int t0 = seg * a.seg, t1 = t0 + a.seg < a.T ? t0 + a.seg : a.T;
    const int used = (t1 < L ? t1 : L) - t0;              // positions of the segment that exist
    const int nblk = used > 0 ? (used + BLOCK - 1) / BLOCK : 0;
    const int bh = b * a.H + h;
    const size_t cells = (size_t)a.P * a.N;

    const int64_t rb = (int64_t)b * a.T;
    auto x_of = [&](int off) { return (const T *)a.x + rb * a.x_row + h * a.P + off; };
    auto gy_of = [&](int off) { return (const T *)a.gy + rb * a.gy_row + h * a.P + off; };
    auto b_of = [&](int off) { return (const T *)a.b + rb * a.b_row + grp * a.N + off; };
    auto c_of = [&](int off) { return (const T *)a.c + rb * a.c_row + grp * a.N + off; };
    Rows<T, DK> rq, rk;
    Rows<T, DV> rv, re;
    rq.dim = rk.dim = kdim;
    rv.dim = re.dim = vdim - v0;
    if constexpr (USE == USE_Y || (USE == USE_STATE && !REV)) {
        rq.base = c_of(0); rq.row = a.c_row; rk.base = b_of(0); rk.row = a.b_row; rv.base = x_of(v0); rv.row = a.x_row;
    } else if constexpr (USE == USE_DC) {
        rq.base = gy_of(0); rq.row = a.gy_row; rk.base = x_of(0); rk.row = a.x_row; rv.base = b_of(v0); rv.row = a.b_row;
        re.base = c_of(v0); re.row = a.c_row;
    } else if constexpr (USE == USE_DU || USE == USE_STATE) {
        rq.base = b_of(0); rq.row = a.b_row; rk.base = c_of(0); rk.row = a.c_row; rv.base = gy_of(v0); rv.row = a.gy_row;
        re.base = x_of(v0); re.row = a.x_row;
    } else {
        rq.base = x_of(0); rq.row = a.x_row; rk.base = gy_of(0); rk.row = a.gy_row; rv.base = c_of(v0); rv.row = a.c_row;
    }
    const float rate = a.rate[h], bias = a.dt_bias ? a.dt_bias[h] : 0.0f;
    const T *dts = (const T *)a.dt + rb * a.dt_row + h;

    // state: rows k (16 kt + 4g + r), column v (16 vt + lane % 16); memory is [P][N]
    f4 S[KT][VT];
    const float *from = nullptr;
    if constexpr (OUT) {
        if (REV) from = a.gs + ((size_t)bh * (a.nseg + 1) + seg + 1) * cells;
        else if (a.hs) from = a.hs + ((size_t)bh * (a.nseg + 1) + seg) * cells;
        else from = a.state ? a.state + bh * cells : nullptr;
    }
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
        for (int vt = 0; vt < VT; ++vt) {
            const int k = 16 * kt + 4 * g, v = v0 + 16 * vt + i16;
            S[kt][vt] = (f4)0.0f;
            if (from && k < kdim && v < vdim) {
                if constexpr (!WIDE_N) S[kt][vt] = *(const f4 *)(from + (size_t)v * a.N + k);
                else
#pragma unroll
                    for (int r = 0; r < 4; ++r) S[kt][vt][r] = from[(size_t)(k + r) * a.N + v];
            }
        }

    double gone = 0.0;     // log2 of what the segment keeps
    float skip_sum = 0.0f;
    auto at = [&](int n) { return t0 + BLOCK * (REV ? nblk - 1 - n : n); };
    auto step_of = [&](int base) {
        const int r = lane & 31, t = base + (REV ? BLOCK - 1 - r : r);
        return t < L ? (float)dts[t * a.dt_row] : -INFINITY;  // softplus gives 0 there
    };
    float dt_next = 0.0f;
    if (nblk) {
        const int base = at(0);
        dt_next = step_of(base);
        if constexpr (OUT) rq.template fetch<REV>(base, L, lane);
        rk.template fetch<REV>(base, L, lane);
        rv.template fetch<REV>(base, L, lane);
        if constexpr (EXTRA) re.template fetch<REV>(base, L, lane);
    }
    for (int n = 0; n < nblk; ++n) {
        const int base = at(n);
        __syncthreads();
        if constexpr (OUT) rq.put(sq, lane);
        rk.put(sk, lane);
        rv.put(sv, lane);
        if constexpr (EXTRA) re.put(se, lane);
        double total;
        {
            // a step beyond the sequence has delta = 0: nothing is kept from it and nothing forgotten
            const float raw = dt_next + bias, delta = raw == -INFINITY ? 0.0f : softplus(raw);
            const double l = (double)delta * (double)rate * 1.4426950408889634;
            double c = l;
#pragma unroll
            for (int d = 1; d < BLOCK; d *= 2) {
                const double o = __shfl_up(c, d, 32);
                if ((lane & 31) >= d) c += o;
            }
            total = __shfl(c, 31, 32);
            if (REV) c -= l;  // a state handed back in time has not passed the step it is handed to
            if (lane < 32) {
                constexpr bool SCALED = USE == USE_Y || USE == USE_DC || (USE == USE_STATE && !REV);
                const float key = SCALED ? delta : 1.0f;
                ss.c[lane] = c;
                ss.out[lane] = pow2(c);
                ss.in[lane] = pow2(total - c) * key;
                ss.key[lane] = key;
                ss.query[lane] = delta;
            }
        }
        __syncthreads();
        if (n + 1 < nblk) {
            const int next = at(n + 1);
            dt_next = step_of(next);
            if constexpr (OUT) rq.template fetch<REV>(next, L, lane);
            rk.template fetch<REV>(next, L, lane);
            rv.template fetch<REV>(next, L, lane);
            if constexpr (EXTRA) re.template fetch<REV>(next, L, lane);
        }
        Op<RAW> v[VT];
#pragma unroll
        for (int vt = 0; vt < VT; ++vt) v[vt] = col_op<T, SV>(sv, 16 * vt, lane);

        if constexpr (OUT) {
            Op<RAW> q[2][KS];
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) q[it][ks] = row_op<T>(sq + (16 * it + i16) * SK, 32 * ks, g);
            // what the state at the block's start gives
            f4 O[VT][2];
#pragma unroll
            for (int vt = 0; vt < VT; ++vt) {
                O[vt][0] = O[vt][1] = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const f4 lo = S[2 * ks][vt], hi = S[2 * ks + 1][vt];
                    const Op<HELD> s = split<HELD>(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
                    O[vt][0] = mma(O[vt][0], s, q[0][ks]);
                    O[vt][1] = mma(O[vt][1], s, q[1][ks]);
                }
            }
            const float out0 = ss.out[i16], out1 = ss.out[16 + i16];
            float from_state[2] = {0.0f, 0.0f};  // its part of the output times the extra operand, by query
#pragma unroll
            for (int vt = 0; vt < VT; ++vt) {
                O[vt][0] *= out0;
                O[vt][1] *= out1;
                if constexpr (EXTRA) {
#pragma unroll
                    for (int it = 0; it < 2; ++it) {
                        float e[4];
                        load_n<T, 4>(se + (16 * it + i16) * SV + 16 * vt + 4 * g, e);
#pragma unroll
                        for (int r = 0; r < 4; ++r) from_state[it] += O[vt][it][r] * e[r];
                    }
                }
            }
            // weighed scores of the block: tiles (keys 0-15, queries 0-15), (0-15, 16-31), (16-31, 16-31)
            f4 M[3], D[3];
#pragma unroll
            for (int m = 0; m < 3; ++m) M[m] = D[m] = (f4)0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Op<RAW> k0 = row_op<T>(sk + i16 * SK, 32 * ks, g), k1 = row_op<T>(sk + (16 + i16) * SK, 32 * ks, g);
                M[0] = mma(M[0], k0, q[0][ks]);
                M[1] = mma(M[1], k0, q[1][ks]);
                M[2] = mma(M[2], k1, q[1][ks]);
            }
            if constexpr (USE == USE_DC) {
                // C_i . B_j over this tile's columns, for the gradient of the steps
#pragma unroll
                for (int vs = 0; vs < DV / 32; ++vs) {
                    const Op<RAW> b0 = row_op<T>(sv + i16 * SV, 32 * vs, g), b1 = row_op<T>(sv + (16 + i16) * SV, 32 * vs, g);
                    const Op<RAW> c0 = row_op<T>(se + i16 * SV, 32 * vs, g), c1 = row_op<T>(se + (16 + i16) * SV, 32 * vs, g);
                    D[0] = mma(D[0], b0, c0);
                    D[1] = mma(D[1], b0, c1);
                    D[2] = mma(D[2], b1, c1);
                }
            }
#pragma unroll
            for (int m = 0; m < 3; ++m) {
                const int jt = m == 2, it = m > 0;
                const double ci = ss.c[16 * it + i16];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * jt + 4 * g + r, i = 16 * it + i16;
                    const float w = pow2(ci - ss.c[j]) * ss.key[j];
                    M[m][r] = j <= i ? M[m][r] * w : 0.0f;
                    D[m][r] *= M[m][r];
                }
            }
            {
                const f4 none = (f4)0.0f;
                const Op<MADE> m0 = split<MADE>(__builtin_shufflevector(M[0], none, 0, 1, 2, 3, 4, 5, 6, 7));
                const Op<MADE> m1 = split<MADE>(__builtin_shufflevector(M[1], M[2], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int vt = 0; vt < VT; ++vt) {
                    O[vt][0] = mma(O[vt][0], v[vt], m0);
                    O[vt][1] = mma(O[vt][1], v[vt], m1);
                }
            }
            // ---- what becomes of the output: a lane holds columns 16 vt + 4g .. +3 of queries i16, 16 + i16
            float whole[2] = {0.0f, 0.0f}, skips = 0.0f;
            const float skip = a.skip ? a.skip[h] : 0.0f;
#pragma unroll
            for (int it = 0; it < 2; ++it) {
                const int r = 16 * it + i16, t = base + (REV ? BLOCK - 1 - r : r);
#pragma unroll
                for (int vt = 0; vt < VT; ++vt) {
                    const int col = v0 + 16 * vt + 4 * g;
                    float o[4] = {O[vt][it][0], O[vt][it][1], O[vt][it][2], O[vt][it][3]};
                    if constexpr (USE == USE_Y) {
                        float x[4];
                        load_n<T, 4>(sv + r * SV + 16 * vt + 4 * g, x);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[e] += skip * x[e];
                        if (t < t1 && col < vdim) store_n<T, 4>((T *)a.y + (rb + t) * a.y_row + h * a.P + col, o);
                    } else if constexpr (USE == USE_DU) {
                        float x[4], dy[4];
                        load_n<T, 4>(se + r * SV + 16 * vt + 4 * g, x);
                        load_n<T, 4>(sv + r * SV + 16 * vt + 4 * g, dy);
                        const float delta = ss.query[r];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            whole[it] += x[e] * o[e];
                            skips += x[e] * dy[e];
                            o[e] = delta * o[e] + skip * dy[e];
                        }
                        if (t < t1 && col < vdim) store_n<T, 4>((T *)a.gx + (rb + t) * a.gx_row + h * a.P + col, o);
                    } else {
                        if constexpr (USE == USE_DB) {
                            const float delta = ss.query[r];
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] *= delta;
                        }
                        float *part = USE == USE_DC ? a.partc : a.partb;
                        if (t < t1 && col < vdim) store_n<float, 4>(part + ((rb + t) * a.H + h) * a.N + col, o);
                    }
                }
            }
            if constexpr (EXTRA) {
                const size_t line = ((size_t)tile * a.B * a.H + bh) * a.T;
#pragma unroll
                for (int it = 0; it < 2; ++it) {
                    const int r = 16 * it + i16, t = base + (REV ? BLOCK - 1 - r : r);
                    float s = from_state[it], w = whole[it];
                    s += __shfl_xor(s, 16);
                    s += __shfl_xor(s, 32);
                    if constexpr (USE == USE_DU) {
                        w += __shfl_xor(w, 16);
                        w += __shfl_xor(w, 32);
                        s *= ss.query[r];
                        if (g == 0 && t < t1) a.xdu[line + t] = w;
                    }
                    if (g == 0 && t < t1) (USE == USE_DC ? a.rint : a.qint)[line + t] = s;
                }
                skip_sum += skips;
            }
            if constexpr (USE == USE_DC) {
                // pairs of the block that span a step t: j < t <= i.  Sums over j < t as a product with a matrix of ones,
                // then over the lanes that hold i >= t: sums of prefix differences would lose what is small next to the block's largest
                const f4 none = (f4)0.0f;
                const Op<3> d0 = split<3>(__builtin_shufflevector(D[0], none, 0, 1, 2, 3, 4, 5, 6, 7));
                const Op<3> d1 = split<3>(__builtin_shufflevector(D[1], D[2], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    Op<1> ones;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        ones.p[0][e] = (__bf16)((e < 4 ? 4 * g + e : 12 + 4 * g + e) < 16 * tt + i16 ? 1.0f : 0.0f);
                    f4 z0 = (f4)0.0f, z1 = mma((f4)0.0f, ones, d1);
                    if (tt == 0) z0 = mma(z0, ones, d0);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int at = 4 * g + r;  // of this tile of steps
                        float s = tt == 0 ? (i16 >= at ? z0[r] : 0.0f) + z1[r] : (i16 >= at ? z1[r] : 0.0f);
                        for (int d = 1; d < 16; d *= 2) s += __shfl_xor(s, d);
                        const int t = base + 16 * tt + at;
                        if (i16 == 0 && t < t1) a.dlin[((size_t)tile * a.B * a.H + bh) * a.T + t] = s;
                    }
                }
            }
        }
        // the state at the block's end
        {
            const float keep = pow2(total);
            f8 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = ss.in[4 * g + e], w[4 + e] = ss.in[16 + 4 * g + e];
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) {
                const Op<MADE> k = split<MADE>(col_floats<T, SK>(sk, 16 * kt, lane) * w);
#pragma unroll
                for (int vt = 0; vt < VT; ++vt) S[kt][vt] = mma(S[kt][vt] * keep, k, v[vt]);
            }
            gone += total;
        }
    }

    if constexpr (USE == USE_STATE || USE == USE_Y) {
        float *to = nullptr;
        if constexpr (USE == USE_STATE) {
            to = (REV ? a.gs + ((size_t)bh * (a.nseg + 1) + seg) * cells : a.hs + ((size_t)bh * (a.nseg + 1) + seg + 1) * cells);
            if (lane == 0 && tile == 0) a.kept[(size_t)bh * a.nseg + seg] = pow2(gone);
        } else if (!a.hs) {
            to = a.state_out ? a.state_out + bh * cells : nullptr;
        }
        if (to) {
#pragma unroll
            for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                for (int vt = 0; vt < VT; ++vt) {
                    const int k = 16 * kt + 4 * g, v = v0 + 16 * vt + i16;
                    if (k < kdim && v < vdim) *(f4 *)(to + (size_t)v * a.N + k) = S[kt][vt];
                }
        }
    }
    if constexpr (USE == USE_DU) {
        for (int d = 1; d < 64; d *= 2) skip_sum += __shfl_xor(skip_sum, d);
        if (lane == 0) a.skipp[((size_t)tile * a.B * a.H + bh) * a.nseg + seg] = skip_sum;
    }
    // rows beyond the sequence's end that no block covered
    if constexpr (USE == USE_Y || USE == USE_DU) {
        T *out = (T *)(USE == USE_Y ? a.y : a.gx);
        const int64_t row = USE == USE_Y ? a.y_row : a.gx_row;
        const int first = t0 + nblk * BLOCK, wide = (vdim - v0 < DV ? vdim - v0 : DV) / 4;
        for (int k = lane; k < (t1 - first) * wide; k += 64) {
            const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            store_n<T, 4>(out + (rb + first + k / wide) * row + h * a.P + v0 + k % wide * 4, zero);
        }
    }
}

template <class T, int DK, int DV> int launch_sweep(Use use, bool rev, const SsmArgs &a, hipStream_t st)
{
    const int vdim = use == USE_DC || use == USE_DB ? a.N : a.P;
    const long units = ((long)a.B * a.nseg + 7) / 8 * 8, grid = units * a.H * ((vdim + DV - 1) / DV);
    if (grid > 0x7fffffffL) return SEMICRF_EUNSUPPORTED;
    const dim3 g((unsigned)grid), t(64);
    if (use == USE_STATE && !rev) hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_STATE, false>), g, t, 0, st, a);
    else if (use == USE_STATE) hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_STATE, true>), g, t, 0, st, a);
    else if (use == USE_Y) hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_Y, false>), g, t, 0, st, a);
    else if (use == USE_DC) hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_DC, false>), g, t, 0, st, a);
    else if (use == USE_DU) hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_DU, true>), g, t, 0, st, a);
    else hipLaunchKernelGGL((k_ssm_sweep<T, DK, DV, USE_DB, true>), g, t, 0, st, a);
    return launched();
}

template <class T> int ssm_sweep(Use use, bool rev, const SsmArgs &a, hipStream_t st)
{
    const bool wide_n = use == USE_DC || use == USE_DB;
    const int kdim = wide_n ? a.P : a.N, vdim = wide_n ? a.N : a.P;
    if (vdim <= 32) {
        if (kdim <= 32) return launch_sweep<T, 32, 32>(use, rev, a, st);
        if (kdim <= 64) return launch_sweep<T, 64, 32>(use, rev, a, st);
        return launch_sweep<T, 128, 32>(use, rev, a, st);
    }
    if (kdim <= 32) return launch_sweep<T, 32, 64>(use, rev, a, st);
    if (kdim <= 64) return launch_sweep<T, 64, 64>(use, rev, a, st);
    return launch_sweep<T, 128, 64>(use, rev, a, st);
}

}  // namespace semicrf_enc
