// Gradients of the scan: two kernels that walk a segment's blocks, one forwards (gradient of C), one backwards in time (gradients
// of x and B), each with what the gradients of the steps need on the way.
//
// A workgroup owns a segment and up to HB heads that share B and C; it takes a block's heads one after the other, so that rows of
// B and C are staged once for all of them, C_i . B_j is formed once, and the sum over heads is a sum in registers.  A wave owns
// sixteen of the 64 (32, 128) state columns: with P and N padded to the same DM, sixteen of N for the gradients of C and B,
// sixteen of P for that of x.  Products, operands and steps as in ssm_fwd.inl.
//
// Gradients of the steps: l_t multiplies every pair (i, j) with j < t <= i of W[i,j] = e^{c_i-c_j} (C_i . B_j) (dy_i . u_j).
//   dlin[t]  pairs within t's block: sums of prefix and suffix sums of tiles of W, nothing subtracted
//   rint[i]  pairs that begin before i's block: C_i . (its gradient from the state)
//   qint[j]  pairs that end behind j's block: u_j . (its gradient from the state)
// k_ssm_steps joins them.
#ifndef SEMICRF_SSM_BWD_INL
#define SEMICRF_SSM_BWD_INL

#include "ssm_block.h"

namespace semicrf_enc {

// What both kernels know of their workgroup.
template <class T> struct Place {
    int b, seg, grp, chunk, h0, nh, L, t0, t1, nblk;
    int64_t rb;
    bool any;
    __device__ __forceinline__ Place(const SsmArgs &a, int HB, int Q, int chunks)
    {
        // workgroups of one segment follow each other on one XCD: they share B and C
        const int per = a.G * chunks, unit = (blockIdx.x % 8) + 8 * (blockIdx.x / 8 / per), within = blockIdx.x / 8 % per;
        any = unit < a.B * a.nseg;
        b = unit / a.nseg;
        seg = unit % a.nseg;
        grp = within / chunks;
        chunk = within % chunks;
        const int hpg = a.H / a.G;
        h0 = grp * hpg + chunk * HB;
        nh = hpg - chunk * HB < HB ? hpg - chunk * HB : HB;
        L = any ? __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T)) : 0;
        t0 = seg * a.seg;
        t1 = t0 + a.seg < a.T ? t0 + a.seg : a.T;
        const int used = (t1 < L ? t1 : L) - t0;
        nblk = used > 0 ? (used + Q - 1) / Q : 0;
        rb = (int64_t)b * a.T;
    }
};

// Four columns of sixteen positions of a lane to a row of the gradient of B or C: at once in its type where one workgroup sums
// all heads, else to the workgroup's part.
template <class T> __device__ __forceinline__ void store_shared(const SsmArgs &a, void *out, int64_t out_row, float *part, const Place<T> &w,
                                                                int chunks, int t, int n, f4 v)
{
    if (t >= w.t1 || n >= a.N) return;
    const float o[4] = {v[0], v[1], v[2], v[3]};
    if (chunks == 1) store_n<T, 4>((T *)out + (w.rb + t) * out_row + w.grp * a.N + n, o);
    else store_n<float, 4>(part + (((size_t)w.chunk * a.B * a.T + w.rb + t) * a.G + w.grp) * a.N + n, o);
}

// Zeros in the rows [first, t1) of `width` columns.
template <class T> __device__ __forceinline__ void clear_rows(T *out, int64_t row, int first, int t1, int width, int tid, int nt)
{
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = tid; k < (t1 - first) * (width / 4); k += nt)
        store_n<T, 4>(out + (int64_t)(first + k / (width / 4)) * row + k % (width / 4) * 4, zero);
}

// ---- gradient of C ------------------------------------------------------------------------------------------------
//   dC_i = sum_h sum_{j<=i} e^{c_i-c_j} (dy_i . u_j) B_j:  queries dy, keys x (scaled by delta), values B; state H [P x N]
template <class T, int Q, int DM, int HB> __global__ __launch_bounds__(DM * 4, 2) void k_ssm_grad_c(SsmArgs a)
{
    constexpr int NT = DM * 4, NW = DM / 16, KT = DM / 16, KS = DM / 32, IT = Q / 16, QS = Q / 32;
    constexpr int RAW = Parts<T>::raw, MADE = Parts<T>::made, HELD = 3;
    typedef Tile<T, Q, DM, NT, false> TL;
    typedef Scores<Q, MADE> SC;
    constexpr int OWN = (SC::TILES + NW - 1) / NW;  // tiles of scores a wave makes at most
    __shared__ __attribute__((aligned(16))) __bf16 sx[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sy[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sb[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sc[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sm[SC::ELEMS];
    __shared__ __attribute__((aligned(16))) Steps<Q> ss[HB];
    __shared__ float rp[NW][Q];             // by wave: its columns' part of rint
    __shared__ float ends[SC::TILES][16];   // sums of a tile of W by its later positions (on the diagonal: dlin), ..
    __shared__ float starts[SC::TILES][16]; // .. and by its earlier ones

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const Place<T> at(a, HB, Q, a.c_chunks);
    if (!at.any) return;
    const size_t cells = (size_t)a.P * a.N;
    const int n0 = 16 * w + i16;  // this lane's column of the state

    TL rx, ry, rbt, rct;
    rbt.init((const T *)a.b + at.rb * a.b_row + at.grp * a.N, a.b_row, a.N, tid);
    rct.init((const T *)a.c + at.rb * a.c_row + at.grp * a.N, a.c_row, a.N, tid);
    const T *x0 = (const T *)a.x + at.rb * a.x_row, *y0 = (const T *)a.gy + at.rb * a.gy_row;
    rx.init(x0 + at.h0 * a.P, a.x_row, a.P, tid);
    ry.init(y0 + at.h0 * a.P, a.gy_row, a.P, tid);

    f4 S[HB][KT];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const float *from = a.hs + ((size_t)(at.b * a.H + at.h0 + k) * (a.nseg + 1) + at.seg) * cells;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            S[k][kt] = (f4)0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int p = 16 * kt + 4 * g + r;
                if (k < at.nh && at.nblk && p < a.P && n0 < a.N) S[k][kt][r] = from[(size_t)p * a.N + n0];
            }
        }
    }
    // steps: wave w makes those of heads w, w + NW, ..
    constexpr int MINE = (HB + NW - 1) / NW;
    float dt_next[MINE];
    auto fetch_dt = [&](int n) {
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const int head = w + NW * k, t = at.t0 + Q * n + lane % Q;
            dt_next[k] = head < at.nh && n < at.nblk && t < at.L ? (float)((const T *)a.dt)[(at.rb + t) * a.dt_row + at.h0 + head] : -INFINITY;
        }
    };
    fetch_dt(0);
    if (at.nblk) {
        rbt.fetch(at.t0, at.L);
        rct.fetch(at.t0, at.L);
        rx.fetch(at.t0, at.L);
        ry.fetch(at.t0, at.L);
        SC::clear(sm, tid, NT);
    }
    for (int n = 0; n < at.nblk; ++n) {
        const int base = at.t0 + Q * n;
        rbt.put(sb, tid);
        rct.put(sc, tid);
#pragma unroll
        for (int k = 0; k < MINE; ++k)
            if (w + NW * k < at.nh)
                make_steps<Q, false>(ss[w + NW * k], dt_next[k], a.dt_bias ? a.dt_bias[at.h0 + w + NW * k] : 0.0f, a.rate[at.h0 + w + NW * k], true, lane);
        fetch_dt(n + 1);
        Op<RAW> v[QS];
        f4 O[IT], D[OWN];
#pragma unroll
        for (int it = 0; it < IT; ++it) O[it] = (f4)0.0f;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            if (k >= at.nh) break;
            rx.put(sx, tid);
            ry.put(sy, tid);
            lds_barrier();
            {
                // the next head's rows, or the next block's
                const bool last = k + 1 >= at.nh;
                const int next = last ? base + Q : base;
                rx.base = x0 + (at.h0 + (last ? 0 : k + 1)) * a.P;
                ry.base = y0 + (at.h0 + (last ? 0 : k + 1)) * a.P;
                if (!last || n + 1 < at.nblk) {
                    rx.fetch(next, at.L);
                    ry.fetch(next, at.L);
                    if (last) {
                        rbt.fetch(next, at.L);
                        rct.fetch(next, at.L);
                    }
                }
            }
            if (k == 0) {
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) v[ks] = TL::by_col(sb, 32 * ks, 16 * w, lane);
                int own = 0;
#pragma unroll
                for (int m = 0; m < SC::TILES; ++m) {
                    if (SC::wave(m, NW) != w) continue;
                    f4 d = (f4)0.0f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        d = mma(d, TL::by_row(sb, 16 * SC::keys(m) + i16, 32 * ks, g), TL::by_row(sc, 16 * SC::query(m) + i16, 32 * ks, g));
#pragma unroll
                    for (int o = 0; o < OWN; ++o)
                        if (o == own) D[o] = d;
                    ++own;
                }
            }
            const Steps<Q> &s = ss[k];
            int own = 0;
#pragma unroll
            for (int m = 0; m < SC::TILES; ++m) {
                if (SC::wave(m, NW) != w) continue;
                const int it = SC::query(m), jt = SC::keys(m);
                f4 p = (f4)0.0f, d = D[0];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    p = mma(p, TL::by_row(sx, 16 * jt + i16, 32 * ks, g), TL::by_row(sy, 16 * it + i16, 32 * ks, g));
                p *= weights(s, it, jt, i16, g);
                SC::put(sm, it, jt, p, lane);
#pragma unroll
                for (int o = 1; o < OWN; ++o)
                    if (o == own) d = D[o];
                ++own;
                const f4 W = p * d;
                if (it == jt) {
                    // dlin[t] = sum over i >= t of sum over j < t; t = 4g + r
                    const float t1 = W[0], t2 = t1 + W[1], t3 = t2 + W[2], t4 = t3 + W[3];
                    const float g1 = __shfl_up(t4, 16), g2 = __shfl_up(t4, 32), g3 = __shfl_up(t4, 48);
                    const float below = (g >= 1 ? g1 : 0.0f) + (g >= 2 ? g2 : 0.0f) + (g >= 3 ? g3 : 0.0f);
                    const float z[4] = {below, below + t1, below + t2, below + t3};
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float sum = sum16(i16 >= 4 * g + r ? z[r] : 0.0f);
                        if (i16 == r) ends[m][4 * g + r] = sum;
                    }
                } else {
                    const float e = sum_rows(W[0] + W[1] + W[2] + W[3]);
                    if (g == 0) ends[m][i16] = e;
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const float sum = sum16(W[r]);
                        if (i16 == r) starts[m][4 * g + r] = sum;
                    }
                }
            }
            // what the state at the block's start gives
            f4 F[IT];
#pragma unroll
            for (int it = 0; it < IT; ++it) F[it] = (f4)0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Op<HELD> st = split<HELD>(__builtin_shufflevector(S[k][2 * ks], S[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int it = 0; it < IT; ++it) F[it] = mma(F[it], st, TL::by_row(sy, 16 * it + i16, 32 * ks, g));
            }
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                F[it] *= s.out[16 * it + i16];
                const f4 e = F[it] * TL::four(sc, 16 * it + i16, 16 * w + 4 * g);
                const float sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                if (g == 0) rp[w][16 * it + i16] = sum;
                O[it] += F[it];
            }
            // the state at the block's end
            {
                const float keep = pow2(s.total);
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) S[k][kt] *= keep;
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) {
                    const f4 lo = *(const f4 *)(s.in + 32 * ks + 4 * g), hi = *(const f4 *)(s.in + 32 * ks + 16 + 4 * g);
                    const Op<HELD> u = split<HELD>(values(v[ks]) * __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt) S[k][kt] = mma(S[k][kt], TL::by_col(sx, 32 * ks, 16 * kt, lane), u);
                }
            }
            lds_barrier();
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
                for (int ks = 0; ks <= it / 2; ++ks) O[it] = mma(O[it], v[ks], SC::get(sm, SC::op(it, ks), lane));
            if (w == k % NW) {
                // lane = position; its sixteen is tile K
                const int r = lane % Q, K = r >> 4, t = base + r;
                float ri = 0.0f, before = 0.0f, after = 0.0f, own_t = 0.0f;
                for (int x = 0; x < NW; ++x) ri += rp[x][r];
                float span = 0.0f;
#pragma unroll
                for (int m = 0; m < SC::TILES; ++m) {
                    const int it = SC::query(m), jt = SC::keys(m);
                    if (it == jt) {
                        if (K == it) own_t = ends[m][i16];
                    } else {
                        const float e = ends[m][i16], b = starts[m][i16];
                        if (K == it) after += e;
                        if (K == jt) before += b;
                        if (it - jt > 1) {
                            const float whole = sum16(e);
                            if (jt < K && K < it) span += whole;
                        }
                    }
                }
                const float tail = suffix16(after), head = moved<0x111>(prefix16(before));
                const size_t to = (size_t)(at.b * a.H + at.h0 + k) * a.T + t;
                if (lane < Q && t < at.t1) {
                    a.rint[to] = ri;
                    a.dlin[to] = own_t + tail + head + span;
                }
            }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) store_shared<T>(a, a.gc, a.gc_row, a.partc, at, a.c_chunks, base + 16 * it + i16, 16 * w + 4 * g, O[it]);
        // the first head's rows of the next block go where this block's last were read transposed by every wave: all have passed
        // the barrier behind that
    }
    if (a.c_chunks == 1)
        clear_rows<T>((T *)a.gc + at.rb * a.gc_row + at.grp * a.N, a.gc_row, at.t0 + at.nblk * Q, at.t1, a.N, tid, NT);
}

// ---- gradients of x and B -----------------------------------------------------------------------------------------
//   du_j = sum_{i>=j} e^{c_i-c_j} (B_j . C_i) dy_i     queries B, keys C, values dy; state G [N x P]     dx = delta du + skip dy
//   dB_j = sum_h delta_j sum_{i>=j} e^{c_i-c_j} (x_j . dy_i) C_i     queries x, keys dy, values C; state G^T [P x N]
// Rows run backwards in time.  G is held both ways round, sixteen columns of each to a wave: twice the products for its
// updates, and nothing to exchange.
template <class T, int Q, int DM, int HB> __global__ __launch_bounds__(DM * 4, 2) void k_ssm_grad_xb(SsmArgs a)
{
    constexpr int NT = DM * 4, NW = DM / 16, KT = DM / 16, KS = DM / 32, IT = Q / 16, QS = Q / 32;
    constexpr int RAW = Parts<T>::raw, MADE = Parts<T>::made, HELD = 3;
    typedef Tile<T, Q, DM, NT, true> TL;
    typedef Scores<Q, MADE> SC;
    constexpr int OWN = (SC::TILES + NW - 1) / NW;
    __shared__ __attribute__((aligned(16))) __bf16 sx[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sy[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sb[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sc[TL::ELEMS];
    __shared__ __attribute__((aligned(16))) __bf16 sm[2 * SC::ELEMS];
    __shared__ __attribute__((aligned(16))) Steps<Q> ss[HB];
    __shared__ float qp[NW][Q], xp[NW][Q];

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const Place<T> at(a, HB, Q, a.b_chunks);
    if (!at.any) return;
    const size_t cells = (size_t)a.P * a.N;
    const int c0 = 16 * w + i16;  // this lane's column: of P in G, of N in its transpose
    const bool has_p = 16 * w < a.P, has_n = 16 * w < a.N;

    TL rx, ry, rbt, rct;
    rbt.init((const T *)a.b + at.rb * a.b_row + at.grp * a.N, a.b_row, a.N, tid);
    rct.init((const T *)a.c + at.rb * a.c_row + at.grp * a.N, a.c_row, a.N, tid);
    const T *x0 = (const T *)a.x + at.rb * a.x_row, *y0 = (const T *)a.gy + at.rb * a.gy_row;
    rx.init(x0 + at.h0 * a.P, a.x_row, a.P, tid);
    ry.init(y0 + at.h0 * a.P, a.gy_row, a.P, tid);

    f4 S[HB][KT], R[HB][KT];  // G [n][p], and [p][n]
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const float *from = a.gs + ((size_t)(at.b * a.H + at.h0 + k) * (a.nseg + 1) + at.seg + 1) * cells;
        const bool live = k < at.nh && at.nblk;
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int row = 16 * kt + 4 * g;
            S[k][kt] = live && row < a.N && c0 < a.P ? *(const f4 *)(from + (size_t)c0 * a.N + row) : (f4)0.0f;
            R[k][kt] = (f4)0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (live && row + r < a.P && c0 < a.N) R[k][kt][r] = from[(size_t)(row + r) * a.N + c0];
        }
    }
    constexpr int MINE = (HB + NW - 1) / NW;
    float dt_next[MINE];
    auto base_of = [&](int n) { return at.t0 + Q * (at.nblk - 1 - n); };
    auto fetch_dt = [&](int n) {
#pragma unroll
        for (int k = 0; k < MINE; ++k) {
            const int head = w + NW * k, t = base_of(n) + Q - 1 - lane % Q;
            dt_next[k] = head < at.nh && n < at.nblk && t < at.L ? (float)((const T *)a.dt)[(at.rb + t) * a.dt_row + at.h0 + head] : -INFINITY;
        }
    };
    fetch_dt(0);
    if (at.nblk) {
        const int base = base_of(0);
        rbt.fetch(base, at.L);
        rct.fetch(base, at.L);
        rx.fetch(base, at.L);
        ry.fetch(base, at.L);
        SC::clear(sm, tid, NT);
        SC::clear(sm + SC::ELEMS, tid, NT);
    }
    float skip_sum[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) skip_sum[k] = 0.0f;
    for (int n = 0; n < at.nblk; ++n) {
        const int base = base_of(n);
        rbt.put(sb, tid);
        rct.put(sc, tid);
#pragma unroll
        for (int k = 0; k < MINE; ++k)
            if (w + NW * k < at.nh)
                make_steps<Q, true>(ss[w + NW * k], dt_next[k], a.dt_bias ? a.dt_bias[at.h0 + w + NW * k] : 0.0f, a.rate[at.h0 + w + NW * k], false, lane);
        fetch_dt(n + 1);
        Op<RAW> vc[QS];
        f4 O[IT], D[OWN];
#pragma unroll
        for (int it = 0; it < IT; ++it) O[it] = (f4)0.0f;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            if (k >= at.nh) break;
            rx.put(sx, tid);
            ry.put(sy, tid);
            lds_barrier();
            {
                const bool last = k + 1 >= at.nh;
                const int next = last ? base - Q : base;
                rx.base = x0 + (at.h0 + (last ? 0 : k + 1)) * a.P;
                ry.base = y0 + (at.h0 + (last ? 0 : k + 1)) * a.P;
                if (!last || n + 1 < at.nblk) {
                    rx.fetch(next, at.L);
                    ry.fetch(next, at.L);
                    if (last) {
                        rbt.fetch(next, at.L);
                        rct.fetch(next, at.L);
                    }
                }
            }
            if (k == 0) {
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) vc[ks] = TL::by_col(sc, 32 * ks, 16 * w, lane);
                int own = 0;
#pragma unroll
                for (int m = 0; m < SC::TILES; ++m) {
                    if (SC::wave(m, NW) != w) continue;
                    f4 d = (f4)0.0f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks)
                        d = mma(d, TL::by_row(sc, 16 * SC::keys(m) + i16, 32 * ks, g), TL::by_row(sb, 16 * SC::query(m) + i16, 32 * ks, g));
#pragma unroll
                    for (int o = 0; o < OWN; ++o)
                        if (o == own) D[o] = d;
                    ++own;
                }
            }
            const Steps<Q> &s = ss[k];
            int own = 0;
#pragma unroll
            for (int m = 0; m < SC::TILES; ++m) {
                if (SC::wave(m, NW) != w) continue;
                const int it = SC::query(m), jt = SC::keys(m);
                f4 p = (f4)0.0f, d = D[0];
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    p = mma(p, TL::by_row(sy, 16 * jt + i16, 32 * ks, g), TL::by_row(sx, 16 * it + i16, 32 * ks, g));
                if (it == jt) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) skip_sum[k] += 4 * g + r == i16 ? p[r] : 0.0f;
                }
#pragma unroll
                for (int o = 1; o < OWN; ++o)
                    if (o == own) d = D[o];
                ++own;
                const f4 f = weights(s, it, jt, i16, g);
                SC::put(sm, it, jt, d * f, lane);
                SC::put(sm + SC::ELEMS, it, jt, p * (f * s.delta[16 * it + i16]), lane);
            }
            // what the state behind the block gives to the gradient of B ..
            if (has_n) {
                f4 F[IT];
#pragma unroll
                for (int it = 0; it < IT; ++it) F[it] = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const Op<MADE> st = split<MADE>(__builtin_shufflevector(R[k][2 * ks], R[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int it = 0; it < IT; ++it) F[it] = mma(F[it], st, TL::by_row(sx, 16 * it + i16, 32 * ks, g));
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) O[it] += F[it] * (s.out[16 * it + i16] * s.delta[16 * it + i16]);
            }
            // .. and to that of u
            f4 U[IT];
            Op<RAW> vy[QS];
            if (has_p) {
#pragma unroll
                for (int it = 0; it < IT; ++it) U[it] = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const Op<HELD> st = split<HELD>(__builtin_shufflevector(S[k][2 * ks], S[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int it = 0; it < IT; ++it) U[it] = mma(U[it], st, TL::by_row(sb, 16 * it + i16, 32 * ks, g));
                }
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) vy[ks] = TL::by_col(sy, 32 * ks, 16 * w, lane);
            }
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                float sum = 0.0f;
                if (has_p) {
                    U[it] *= s.out[16 * it + i16];
                    const f4 e = U[it] * TL::four(sx, 16 * it + i16, 16 * w + 4 * g);
                    sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                }
                if (g == 0) qp[w][16 * it + i16] = sum * s.delta[16 * it + i16];
            }
            // the state before the block, both ways round
            {
                const float keep = pow2(s.total);
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) {
                    const f4 lo = *(const f4 *)(s.in + 32 * ks + 4 * g), hi = *(const f4 *)(s.in + 32 * ks + 16 + 4 * g);
                    const f8 in = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    if (has_p) {
                        const Op<HELD> u = split<HELD>(values(vy[ks]) * in);
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) {
                            if (ks == 0) S[k][kt] *= keep;
                            S[k][kt] = mma(S[k][kt], TL::by_col(sc, 32 * ks, 16 * kt, lane), u);
                        }
                    }
                    if (has_n) {
                        const Op<MADE> u = split<MADE>(values(vc[ks]) * in);
#pragma unroll
                        for (int kt = 0; kt < KT; ++kt) {
                            if (ks == 0) R[k][kt] *= keep;
                            R[k][kt] = mma(R[k][kt], TL::by_col(sy, 32 * ks, 16 * kt, lane), u);
                        }
                    }
                }
            }
            const float skip = a.skip ? a.skip[at.h0 + k] : 0.0f;
            lds_barrier();
            if (has_n) {
#pragma unroll
                for (int it = 0; it < IT; ++it)
#pragma unroll
                    for (int ks = 0; ks <= it / 2; ++ks) O[it] = mma(O[it], vc[ks], SC::get(sm + SC::ELEMS, SC::op(it, ks), lane));
            }
            if (has_p) {
                const int col = 16 * w + 4 * g;
#pragma unroll
                for (int it = 0; it < IT; ++it) {
#pragma unroll
                    for (int ks = 0; ks <= it / 2; ++ks) U[it] = mma(U[it], vy[ks], SC::get(sm, SC::op(it, ks), lane));
                    const int r = 16 * it + i16, t = base + Q - 1 - r;
                    const f4 e = U[it] * TL::four(sx, r, 16 * w + 4 * g), o = U[it] * s.delta[r] + TL::four(sy, r, 16 * w + 4 * g) * skip;
                    const float sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                    if (g == 0) xp[w][r] = sum;
                    const float out[4] = {o[0], o[1], o[2], o[3]};
                    if (t < at.t1 && col < a.P) store_n<T, 4>((T *)a.gx + (at.rb + t) * a.gx_row + (at.h0 + k) * a.P + col, out);
                }
            } else {
#pragma unroll
                for (int it = 0; it < IT; ++it)
                    if (g == 0) xp[w][16 * it + i16] = 0.0f;
            }
            lds_barrier();
            if (w == k % NW) {
                const int r = lane % Q, t = base + Q - 1 - r;
                float q = 0.0f, x = 0.0f;
                for (int y = 0; y < NW; ++y) q += qp[y][r], x += xp[y][r];
                const size_t to = (size_t)(at.b * a.H + at.h0 + k) * a.T + t;
                if (lane < Q && t < at.t1) {
                    a.qint[to] = q;
                    a.xdu[to] = x;
                }
            }
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) store_shared<T>(a, a.gb, a.gb_row, a.partb, at, a.b_chunks, base + Q - 1 - 16 * it - i16, 16 * w + 4 * g, O[it]);
    }
    // sums for the skip: by wave in LDS, then over the waves in order
    lds_barrier();
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        for (int d = 1; d < 64; d *= 2) skip_sum[k] += __shfl_xor(skip_sum[k], d);
        if (lane == 0) qp[w][k] = skip_sum[k];
    }
    lds_barrier();
    if (tid < at.nh) {
        float s = 0.0f;
        for (int y = 0; y < NW; ++y) s += qp[y][tid];
        a.skipp[(size_t)(at.b * a.H + at.h0 + tid) * a.nseg + at.seg] = s;
    }
    clear_rows<T>((T *)a.gx + at.rb * a.gx_row + at.h0 * a.P, a.gx_row, at.t0 + at.nblk * Q, at.t1, at.nh * a.P, tid, NT);
    if (a.b_chunks == 1)
        clear_rows<T>((T *)a.gb + at.rb * a.gb_row + at.grp * a.N, a.gb_row, at.t0 + at.nblk * Q, at.t1, a.N, tid, NT);
}

template <class T, int Q, int DM> int launch_grad(const SsmArgs &a, hipStream_t st)
{
    const long units = ((long)a.B * a.nseg + 7) / 8 * 8 * a.G;
    if (units * a.b_chunks > 0x7fffffffL) return SEMICRF_EUNSUPPORTED;
    const dim3 gc((unsigned)(units * a.c_chunks)), gx((unsigned)(units * a.b_chunks)), t(DM * 4);
    if constexpr (DM <= 64) {
        if (a.c_heads > 1) hipLaunchKernelGGL((k_ssm_grad_c<T, Q, DM, 4>), gc, t, 0, st, a);
        else hipLaunchKernelGGL((k_ssm_grad_c<T, Q, DM, 1>), gc, t, 0, st, a);
        if (a.b_heads > 1) hipLaunchKernelGGL((k_ssm_grad_xb<T, Q, DM, 2>), gx, t, 0, st, a);
        else hipLaunchKernelGGL((k_ssm_grad_xb<T, Q, DM, 1>), gx, t, 0, st, a);
    } else {
        hipLaunchKernelGGL((k_ssm_grad_c<T, Q, DM, 1>), gc, t, 0, st, a);
        hipLaunchKernelGGL((k_ssm_grad_xb<T, Q, DM, 1>), gx, t, 0, st, a);
    }
    return launched();
}
template <class T> int ssm_grad(const SsmArgs &a, hipStream_t st)
{
    constexpr int R = Parts<T>::raw;
    const int most = a.P > a.N ? a.P : a.N;
    if (most <= 32) return launch_grad<T, grad_block(R, 32), 32>(a, st);
    if (most <= 64) return launch_grad<T, grad_block(R, 64), 64>(a, st);
    return launch_grad<T, grad_block(R, 128), 128>(a, st);
}

}  // namespace semicrf_enc

#endif
