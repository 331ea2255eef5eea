// The scan over one segment of one head, forwards (outputs, or the state alone) and backwards in time (the state alone): see ssm.h
// for the mathematics.
//
// A workgroup owns a segment of one head and takes it in blocks of Q positions; a wave owns sixteen channels: their columns of
// the state (N x 16, in registers from block to block) and of the output.  Rows of the block are staged in LDS as they lie in
// memory, the next block's already on their way; what the products need with positions as the inner index is read transposed
// (ds_read_b64_tr_b16).
//   scores  M[j,i] = (B_j . C_i) e^{c_i-c_j} delta_j, j <= i, skip added where j = i; each wave makes some, all read them
//   output  O[p,i] = sum_j x[j,p] M[j,i] + e^{c_i} sum_n S[n,p] C[i,n]
//   state   S[n,p] = e^{c_Q} S[n,p] + sum_j B[j,n] (e^{c_Q-c_j} delta_j x[j,p])
// Steps (delta, c) are made for four blocks at a time, one by each wave.
//
// Measured, bfloat16, 400 000 positions of 8 heads, 64 channels, 64 states: outputs 318 us, 922 MB (2.9 TB/s); states alone 125 us, 461 MB
// (3.7 TB/s).  Bound by no unit: of the outputs' time the vector units are busy 48 %, LDS 50 % and the matrix cores 33 %; what is
// left is the latency from one to the next with three waves on a SIMD (157 registers).
#ifndef SEMICRF_SSM_FWD_INL
#define SEMICRF_SSM_FWD_INL

#include "ssm_block.h"

namespace semicrf_enc {

// LDS of a workgroup.
template <class T, int Q, int DK, int PV, bool OUT> struct ScanShared {
    static constexpr int NW = PV / 16, AHEAD = NW < 4 ? NW : 4;  // blocks whose steps are made together, one by each wave
    typedef Tile<T, Q, DK, PV * 4, false> TK;
    typedef Tile<T, Q, PV, PV * 4, false> TV;
    // one array, so that operands' places differ by constants
    alignas(16) __bf16 pool[(OUT ? 2 : 1) * TK::ELEMS + TV::ELEMS + (OUT ? Scores<Q>::ELEMS : 0)];
    Steps<Q> ss[AHEAD];
};

template <class T, int Q, int DK, int PV, bool OUT, bool REV>
__device__ __forceinline__ void scan_segment(const SsmArgs &a, unsigned block, ScanShared<T, Q, DK, PV, OUT> &sh)
{
    constexpr int NT = PV * 4, NW = PV / 16, KT = DK / 16, KS = DK / 32, IT = Q / 16, QS = Q / 32;
    constexpr int AHEAD = ScanShared<T, Q, DK, PV, OUT>::AHEAD;
    constexpr int RAW = Parts<T>::raw;
    // queries are kept from the scores to the output, except where they would take 96 registers (float32, 128 states: 488 us so, 303
    // read again; bfloat16 144 us kept, 174 read again; 16 x 4000 positions of 8 heads of 64)
    constexpr bool HOLD = IT * KS * RAW <= 16;
    typedef Tile<T, Q, DK, NT, REV> TK;
    typedef Tile<T, Q, PV, NT, REV> TV;
    typedef Scores<Q> SC;
    __bf16 *const sk = sh.pool, *const sv = sk + TK::ELEMS, *const sq = sv + TV::ELEMS, *const sm = sq + (OUT ? TK::ELEMS : 0);
    Steps<Q> *const ss = sh.ss;

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
    // heads of one segment follow each other on one XCD (workgroups go round the eight in turn): they share B and C
    const int unit = (block % 8) + 8 * (block / 8 / a.H), h = block / 8 % a.H;
    if (unit >= a.B * a.nseg) return;
    const int b = unit / a.nseg, seg = unit % a.nseg, grp = h / (a.H / a.G), bh = b * a.H + h;
    const int L = __builtin_amdgcn_readfirstlane(length_of(a.lengths, b, a.T));
    const int t0 = seg * a.seg, t1 = t0 + a.seg < a.T ? t0 + a.seg : a.T;
    const int used = (t1 < L ? t1 : L) - t0, nblk = used > 0 ? (used + Q - 1) / Q : 0;
    const size_t cells = (size_t)a.P * a.N;
    const int64_t rb = (int64_t)b * a.T;

    TK rq, rk;
    TV rv;
    const typename TK::Lane lk(lane, 0);
    const typename TV::Lane lv(lane, w);
    const typename TK::Place pk(tid);
    const typename TV::Place pv(tid);
    // rows from the first block on; each block moves on (back) by Q of them
    const int qk_bytes = (int)(a.c_row * (int64_t)sizeof(T)), b_bytes = (int)(a.b_row * (int64_t)sizeof(T));
    const int v_bytes = (int)((REV ? a.gy_row : a.x_row) * (int64_t)sizeof(T)), dt_bytes = (int)(a.dt_row * (int64_t)sizeof(T));
    const int y_bytes = (int)(a.y_row * (int64_t)sizeof(T)), k_bytes = REV ? qk_bytes : b_bytes;
    const int64_t start = rb + t0 + (REV && nblk ? Q * (nblk - 1) : 0);
    const char *cs = (const char *)a.c + start * qk_bytes + grp * a.N * (int)sizeof(T);
    const char *kb = REV ? cs : (const char *)a.b + start * b_bytes + grp * a.N * (int)sizeof(T);
    const char *vs = (const char *)(REV ? a.gy : a.x) + start * v_bytes + h * a.P * (int)sizeof(T);
    const char *dts = (const char *)a.dt + (rb + t0) * dt_bytes + h * (int)sizeof(T);
    char *ys = (char *)a.y + (rb + t0) * y_bytes + h * a.P * (int)sizeof(T);
    constexpr int DIR = REV ? -Q : Q;
    if constexpr (OUT) rq.init(qk_bytes, a.N, tid);
    rk.init(k_bytes, a.N, tid);
    rv.init(v_bytes, a.P, tid);
    const float rate = a.rate[h], bias = a.dt_bias ? a.dt_bias[h] : 0.0f, skip = OUT && a.skip ? a.skip[h] : 0.0f;

    // state: rows n (16 kt + 4g + r), column p = 16 w + lane % 16; memory is [P][N]
    const int p = 16 * w + i16;
    f4 S[KT];
    const float *from = !OUT ? nullptr : a.hs ? a.hs + ((size_t)bh * (a.nseg + 1) + seg) * cells
                                              : a.state ? a.state + bh * cells : nullptr;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt) {
        const int n = 16 * kt + 4 * g;
        S[kt] = from && n < a.N && p < a.P ? *(const f4 *)(from + (size_t)p * a.N + n) : (f4)0.0f;
    }

    double gone = 0.0;
    auto at = [&](int n) { return t0 + Q * (REV ? nblk - 1 - n : n); };
    Dt<T> dt_next;  // of the block this wave makes the steps of
    auto fetch_dt = [&](int n) {
        const int r = lane % Q, first = at(n) - t0;
        dt_next.fetch(dts + (int64_t)first * dt_bytes, dt_bytes, REV ? Q - 1 - r : r, n < nblk ? L - at(n) : 0);
    };
    auto fetch = [&](int n) {
        const int left = L - at(n);
        if constexpr (OUT) rq.fetch(rows_at(cs, left, Q, qk_bytes), 0);
        rk.fetch(rows_at(kb, left, Q, k_bytes), 0);
        rv.fetch(rows_at(vs, left, Q, v_bytes), 0);
        cs += (int64_t)DIR * qk_bytes;
        kb += (int64_t)DIR * k_bytes;
        vs += (int64_t)DIR * v_bytes;
    };
    const uint32_t y_off = 16 * w + 4 * g < a.P ? (uint32_t)(i16 * y_bytes + (16 * w + 4 * g) * (int)sizeof(T)) : OUTSIDE;
    f4 skips;  // on the diagonal of the scores
#pragma unroll
    for (int r = 0; r < 4; ++r) skips[r] = 4 * g + r == i16 ? skip : 0.0f;
    fetch_dt(w);
    if (nblk) fetch(0);
    for (int n = 0; n < nblk; ++n) {
        const int base = at(n);
        const Steps<Q> &s = ss[n % AHEAD];
        if (n % AHEAD == 0 && w < AHEAD) {
            make_steps<Q, REV>(ss[w], dt_next.value(), bias, rate, lane);
            fetch_dt(n + AHEAD + w);
        }
        if constexpr (OUT) rq.put(sq, pk, tid);
        rk.put(sk, pk, tid);
        rv.template put<!OUT>(sv, pv, tid);
        lds_barrier();
        if (n + 1 < nblk) fetch(n + 1);
        f4 O[IT];
        if constexpr (OUT) {
            Op<RAW> held[HOLD ? IT : 1][HOLD ? KS : 1];
            if constexpr (HOLD) {
#pragma unroll
                for (int it = 0; it < IT; ++it)
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) held[it][ks] = TK::by_row(sq, lk, it, ks);
            }
            auto q = [&](int it, int ks) -> Op<RAW> {
                if constexpr (HOLD) return held[it][ks];
                else return TK::by_row(sq, lk, it, ks);
            };
#pragma unroll
            for (int k = 0; k < SC::TILES; ++k) {
                if (SC::wave(k, NW) != w) continue;
                const int it = SC::query(k), jt = SC::keys(k);
                f4 m = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) m = mma_inputs(m, TK::by_row(sk, lk, jt, ks), q(it, ks));
                m *= weights<Q, REV>(s, it, jt, i16, g);
                if (it == jt) m += skips;
                SC::put(sm, it, jt, m, lane);
            }
            // what the state at the block's start gives
#pragma unroll
            for (int it = 0; it < IT; ++it) O[it] = (f4)0.0f;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const Op<HELD> st = split<HELD>(__builtin_shufflevector(S[2 * ks], S[2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int it = 0; it < IT; ++it) O[it] = mma(O[it], st, q(it, ks));
            }
#pragma unroll
            for (int it = 0; it < IT; ++it) O[it] *= s.out[16 * it + i16];
        }
        Op<RAW> v[QS];
#pragma unroll
        for (int ks = 0; ks < QS; ++ks) v[ks] = TV::own_col(sv, lv, ks);
        // the state at the block's end
        {
            const float keep = pow2(s.total);
#pragma unroll
            for (int kt = 0; kt < KT; ++kt) S[kt] *= keep;
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) {
                const f4 lo = *(const f4 *)(s.in + 32 * ks + 4 * g), hi = *(const f4 *)(s.in + 32 * ks + 16 + 4 * g);
                const Op<HELD> u = split<HELD>(values(v[ks]) * __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                for (int kt = 0; kt < KT; ++kt) S[kt] = mma(S[kt], TK::by_col(sk, lk, ks, kt), u);
            }
            gone += s.total;
        }
        lds_barrier();
        if constexpr (OUT) {
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
                for (int ks = 0; ks <= it / 2; ++ks) O[it] = SC::product(O[it], v[ks], sm, it, ks, lane);
            // a lane holds channels 16 w + 4g .. +3 of positions i16, 16 + i16, ..
            const __amdgpu_buffer_rsrc_t rows = rows_at(ys, t1 - base, Q, y_bytes);
            ys += (int64_t)Q * y_bytes;
#pragma unroll
            for (int it = 0; it < IT; ++it) store_four<T>(rows, y_off, 16 * it * y_bytes, O[it]);
        }
    }

    float *to;
    if constexpr (!OUT) {
        to = REV ? a.gs + ((size_t)bh * (a.nseg + 1) + seg) * cells : a.hs + ((size_t)bh * (a.nseg + 1) + seg + 1) * cells;
        if (!REV && tid == 0) a.kept[(size_t)bh * a.nseg + seg] = pow2(gone);
    } else {
        to = !a.hs && a.state_out ? a.state_out + bh * cells : nullptr;
    }
    if (to) {
#pragma unroll
        for (int kt = 0; kt < KT; ++kt) {
            const int n = 16 * kt + 4 * g;
            if (n < a.N && p < a.P) *(f4 *)(to + (size_t)p * a.N + n) = !OUT && (i16 & 1) ? -S[kt] : S[kt];
        }
    }
    if constexpr (OUT) {
        // rows beyond the sequence's end that no block covered
        const int first = t0 + nblk * Q, wide = a.P / 4;
        for (int k = tid; k < (t1 - first) * wide; k += NT) {
            const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            store_n<T, 4>((T *)a.y + (rb + first + k / wide) * a.y_row + h * a.P + k % wide * 4, zero);
        }
    }
}

template <class T, int Q, int DK, int PV> __global__ __launch_bounds__(PV * 4, 2) void k_ssm_scan(SsmArgs a)
{
    __shared__ __attribute__((aligned(16))) ScanShared<T, Q, DK, PV, true> sh;
    scan_segment<T, Q, DK, PV, true, false>(a, blockIdx.x, sh);
}
// States alone, forwards or (the second half of a launch of twice as many workgroups) backwards.
template <class T, int Q, int DK, int PV> __global__ __launch_bounds__(PV * 4, 2) void k_ssm_states(SsmArgs a, unsigned half)
{
    __shared__ __attribute__((aligned(16))) ScanShared<T, Q, DK, PV, false> sh;
    if (blockIdx.x < half) scan_segment<T, Q, DK, PV, false, false>(a, blockIdx.x, sh);
    else scan_segment<T, Q, DK, PV, false, true>(a, blockIdx.x - half, sh);
}

template <class T, int Q, int DK, int PV> int launch_scan(bool out, bool both, const SsmArgs &a, hipStream_t st)
{
    const long grid = ((long)a.B * a.nseg + 7) / 8 * 8 * a.H;
    if (grid > 0x3fffffffL) return SEMICRF_EUNSUPPORTED;
    const dim3 t(PV * 4);
    if (out) hipLaunchKernelGGL((k_ssm_scan<T, Q, DK, PV>), dim3((unsigned)grid), t, 0, st, a);
    else hipLaunchKernelGGL((k_ssm_states<T, Q, DK, PV>), dim3((unsigned)(both ? 2 * grid : grid)), t, 0, st, a, (unsigned)grid);
    return launched();
}
// Positions of a block: 64 as long as the staged parts leave room for two workgroups on a compute unit, and the rows on their way
// take few of a thread's registers (narrow heads have few threads for as many rows of B and C).  16 x 4000 positions of 512
// channels, with blocks of 64 and of 32: float32, heads of 32, 32 states 238 and 165 us; float16, heads of 16, 64 states 588 and
// 327; bfloat16, heads of 32, 128 states 246 and 181, heads of 16, 64 states 217 and 246.
template <class T> constexpr int scan_block(int DK, int PV)
{
    constexpr int R = Parts<T>::raw;
    const int rows = 4 * (2 * DK + PV) * (int)sizeof(T) / PV;  // registers
    return R * (2 * DK + PV) <= 448 && rows <= (R == 1 && DK <= 64 ? 72 : 40) ? 64 : 32;
}
template <class T, int DK> int launch_scan_p(bool out, bool both, const SsmArgs &a, hipStream_t st)
{
    if (a.P <= 16) return launch_scan<T, scan_block<T>(DK, 16), DK, 16>(out, both, a, st);
    if (a.P <= 32) return launch_scan<T, scan_block<T>(DK, 32), DK, 32>(out, both, a, st);
    if (a.P <= 64) return launch_scan<T, scan_block<T>(DK, 64), DK, 64>(out, both, a, st);
    return launch_scan<T, scan_block<T>(DK, 128), DK, 128>(out, both, a, st);
}
template <class T> int ssm_scan(bool out, bool both, const SsmArgs &a, hipStream_t st)
{
    if (a.N <= 32) return launch_scan_p<T, 32>(out, both, a, st);
    if (a.N <= 64) return launch_scan_p<T, 64>(out, both, a, st);
    return launch_scan_p<T, 128>(out, both, a, st);
}

}  // namespace semicrf_enc

#endif
