// Gradients of the scan: two kernels that walk a segment's blocks, one forwards (gradient of C), one backwards in time (gradients
// of x and B), each with what the gradients of the steps need on the way.
//
// A workgroup owns a segment and up to HB heads that share B and C; it takes a block's heads one after the other, so that rows of
// B and C are staged once for all of them, C_i . B_j is formed once, and the sum over heads is a sum in registers.  P and N are
// padded to PP and NN (32, 64, 128), and there is a wave to every sixteen of the wider: it owns sixteen columns of N for the
// gradients of C and B, sixteen of P for that of x, where there are as many.  Products, operands and steps as in ssm_fwd.inl.
//
// Gradients of the steps: l_t multiplies every pair (i, j) with j < t <= i of W[i,j] = e^{c_i-c_j} (C_i . B_j) (dy_i . u_j).
//   dlin[t]  pairs within t's block: sums of prefix and suffix sums of tiles of W, nothing subtracted
//   rint[i]  pairs that begin before i's block: C_i . (its gradient from the state)
//   qint[j]  pairs that end behind j's block: u_j . (its gradient from the state)
// k_ssm_steps joins them.
//
// Measured, bfloat16, 4 x 100 000 positions of 8 heads, 64 channels, 64 states: gradient of C 569 us, gradients of x and B 716 us
// under a trace.  Bound by the instructions around the products: of the latter's time the vector units are busy 49 %, LDS 45 %, the
// matrix cores 21 %, at three waves on a SIMD.
#ifndef SEMICRF_SSM_BWD_INL
#define SEMICRF_SSM_BWD_INL

#include "ssm_block.h"

namespace semicrf_enc {

// Waves to a SIMD that the registers are cut for (16 x 4000 positions, 8 heads of 64, 64 states, float16: 501 us with two, 452 with
// three, though its gradients of x and B get two either way, for 70 KB of LDS; what is wider spills).
constexpr int waves_for(int raw, int most) { return most <= 64 && raw <= 2 ? 3 : 2; }

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

// Rows of the gradient of B or C: in its type where one workgroup sums all heads, else the workgroup's part.
template <class T> struct SharedOut {
    char *first;
    int row;  // bytes
    bool whole;
    __device__ __forceinline__ SharedOut(const SsmArgs &a, void *out, int64_t out_row, float *part, int chunks, const Place<T> &w)
    {
        whole = chunks == 1;
        row = whole ? (int)(out_row * (int64_t)sizeof(T)) : a.G * a.N * 4;
        first = whole ? (char *)((T *)out + w.rb * out_row + w.grp * a.N)
                      : (char *)(part + (((size_t)w.chunk * a.B * a.T + w.rb) * a.G + w.grp) * a.N);
    }
    // row r of a block from position `base`, `above` rows further down; columns n.. of N
    template <int Q> __device__ __forceinline__ void put(int base, int r, int above, int n, int N, int t1, f4 v) const
    {
        const __amdgpu_buffer_rsrc_t rows = rows_at(first + (int64_t)base * row, t1 - base, Q, row);
        const uint32_t off = n < N ? (uint32_t)(r * row + n * (whole ? (int)sizeof(T) : 4)) : OUTSIDE;
        if (whole) store_four<T>(rows, off, above * row, v);
        else store_four<float>(rows, off, above * row, v);
    }
};

// A value for position base + r of a head's line, r >= 0.  Stores are never skipped by a branch, here and below: the wait for the
// rows that are on their way could not tell how many stores came after them, and would wait for all.
template <int Q> __device__ __forceinline__ void put_line(float *line, int base, int t1, int r, float v)
{
    __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, v), rows_at(line + base, t1 - base, Q, 4), r >= 0 ? 4 * r : (int)OUTSIDE, 0, 0);
}

// The operands' rows: where the block that is fetched next begins, at the first head's (the group's) columns.
template <class T> struct Sources {
    const char *x, *y, *b, *c, *dt;
    int x_bytes, y_bytes, b_bytes, c_bytes, dt_bytes;
    __device__ __forceinline__ Sources(const SsmArgs &a, const Place<T> &w, int64_t first)
    {
        constexpr int e = (int)sizeof(T);
        x_bytes = (int)a.x_row * e, y_bytes = (int)a.gy_row * e, b_bytes = (int)a.b_row * e, c_bytes = (int)a.c_row * e;
        dt_bytes = (int)a.dt_row * e;
        const int64_t at = w.rb + first;
        x = (const char *)a.x + at * x_bytes + w.h0 * a.P * e;
        y = (const char *)a.gy + at * y_bytes + w.h0 * a.P * e;
        b = (const char *)a.b + at * b_bytes + w.grp * a.N * e;
        c = (const char *)a.c + at * c_bytes + w.grp * a.N * e;
        dt = (const char *)a.dt + at * dt_bytes + w.h0 * e;
    }
    __device__ __forceinline__ void move(int rows)
    {
        x += (int64_t)rows * x_bytes, y += (int64_t)rows * y_bytes, b += (int64_t)rows * b_bytes, c += (int64_t)rows * c_bytes;
    }
};

// Zeros in the rows [first, t1) of `width` columns.
template <class T> __device__ __forceinline__ void clear_rows(T *out, int64_t row, int first, int t1, int width, int tid, int nt)
{
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k = tid; k < (t1 - first) * (width / 4); k += nt)
        store_n<T, 4>(out + (int64_t)(first + k / (width / 4)) * row + k % (width / 4) * 4, zero);
}

// ---- gradient of C ------------------------------------------------------------------------------------------------
//   dC_i = sum_h sum_{j<=i} e^{c_i-c_j} (dy_i . u_j) B_j:  queries dy, keys x (scaled by delta), values B; state H [P x N]
template <class T, int PP, int NN, int HB> __global__ __launch_bounds__((PP > NN ? PP : NN) * 4, waves_for(Parts<T>::raw, PP > NN ? PP : NN)) void k_ssm_grad_c(SsmArgs a)
{
    constexpr int Q = GRAD_BLOCK, MOST = PP > NN ? PP : NN, NT = MOST * 4, NW = MOST / 16, IT = Q / 16, QS = Q / 32;
    constexpr int KTP = PP / 16, KTN = NN / 16, KSP = PP / 32, KSN = NN / 32;
    constexpr int RAW = Parts<T>::raw, E = (int)sizeof(T);
    typedef Tile<T, Q, PP, NT, false> TP;
    typedef Tile<T, Q, NN, NT, false> TN;
    typedef Scores<Q> SC;
    constexpr int OWN = (SC::TILES + NW - 1) / NW;  // tiles of scores a wave makes at most
    constexpr int TURNS = (IT + NW - 1) / NW;       // sixteens of positions whose sums a wave makes
    // one array, so that operands' places differ by constants
    __shared__ __attribute__((aligned(16))) __bf16 pool[2 * TP::ELEMS + 2 * TN::ELEMS + SC::ELEMS];
    __bf16 *const sx = pool, *const sy = sx + TP::ELEMS, *const sb = sy + TP::ELEMS, *const sc = sb + TN::ELEMS, *const sm = sc + TN::ELEMS;
    __shared__ Steps<Q> ss[2];  // of this head and the next
    __shared__ float skips[HB][NT];         // by thread: sums for the skip, of at most 32 blocks
    __shared__ __attribute__((aligned(16))) float rp[NW][Q];  // by wave: its columns' part of rint
    __shared__ float ends[SC::TILES][16];   // sums of a tile of W by its later positions (on the diagonal: dlin), ..
    __shared__ float starts[SC::TILES][16]; // .. and by its earlier ones

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const Place<T> at(a, HB, Q, a.chunks);
    if (!at.any) return;
    const size_t cells = (size_t)a.P * a.N;
    const int n0 = 16 * w + i16;  // this lane's column of the state
    const bool own_n = NN == MOST || 16 * w < NN;

    Sources<T> src(a, at, at.t0);
    TP rx, ry;
    TN rbt, rct;
    const typename TP::Lane lp(lane, w);
    const typename TN::Lane ln(lane, w);
    const typename TP::Place plp(tid);
    const typename TN::Place pln(tid);
    rx.init(src.x_bytes, a.P, tid);
    ry.init(src.y_bytes, a.P, tid);
    rbt.init(src.b_bytes, a.N, tid);
    rct.init(src.c_bytes, a.N, tid);

    f4 S[HB][KTP];
    float rate[HB], bias[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const int head = k < at.nh ? at.h0 + k : at.h0;
        rate[k] = a.rate[head];
        bias[k] = a.dt_bias ? a.dt_bias[head] : 0.0f;
        skips[k][tid] = 0.0f;
        const float *from = a.hs + ((size_t)(at.b * a.H + head) * (a.nseg + 1) + at.seg) * cells;
#pragma unroll
        for (int kt = 0; kt < KTP; ++kt) {
            S[k][kt] = (f4)0.0f;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int p = 16 * kt + 4 * g + r;
                if (at.nblk && p < a.P && n0 < a.N) S[k][kt][r] = from[(size_t)p * a.N + n0];
            }
        }
    }
    // Steps are made a head ahead, by the last wave, which has the fewest scores to make; dt comes another head ahead.
    Dt<T> dt;
    const bool two = HB > 1 && at.nh > 1;  // heads in turn
    auto fetch_dt = [&](int n, int k) {
        dt.fetch(src.dt + (int64_t)Q * n * src.dt_bytes + k * E, src.dt_bytes, lane % Q, n < at.nblk ? at.L - at.t0 - Q * n : 0);
    };
    if (at.nblk) {
        rbt.fetch(rows_at(src.b, at.L - at.t0, Q, src.b_bytes), 0);
        rct.fetch(rows_at(src.c, at.L - at.t0, Q, src.c_bytes), 0);
        rx.fetch(rows_at(src.x, at.L - at.t0, Q, src.x_bytes), 0);
        ry.fetch(rows_at(src.y, at.L - at.t0, Q, src.y_bytes), 0);
        fetch_dt(0, 0);
        if (w == 0) make_steps<Q, false>(ss[0], dt.value(), bias[0], rate[0], lane);
        fetch_dt(two ? 0 : 1, two ? 1 : 0);
    }
    int turn = 0;  // counts heads
    const SharedOut<T> out(a, a.gc, a.gc_row, a.partc, a.chunks, at);
    for (int n = 0; n < at.nblk; ++n) {
        const int base = at.t0 + Q * n;
        rbt.put(sb, pln, tid);
        rct.put(sc, pln, tid);
        Op<RAW> v[QS];
        f4 O[IT], D[OWN];
#pragma unroll
        for (int it = 0; it < IT; ++it) O[it] = (f4)0.0f;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            if (HB > 1 && k >= at.nh) break;
            rx.put(sx, plp, tid);
            ry.put(sy, plp, tid);
            skips[k][tid] += rx.dot(ry);
            lds_barrier();
            // the next head's rows, or the next block's
            {
                const bool last = HB == 1 || k + 1 >= at.nh;
                if (last) src.move(Q);
                const int left = last ? at.L - base - Q : at.L - base, col = last ? 0 : (k + 1) * a.P * E;
                rx.fetch(rows_at(src.x, left, Q, src.x_bytes), col);
                ry.fetch(rows_at(src.y, left, Q, src.y_bytes), col);
                if (last) {
                    rbt.fetch(rows_at(src.b, left, Q, src.b_bytes), 0);
                    rct.fetch(rows_at(src.c, left, Q, src.c_bytes), 0);
                }
            }
            if (k == 0) {
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) v[ks] = TN::own_col(sb, ln, ks);
                int own = 0;
#pragma unroll
                for (int m = 0; m < SC::TILES; ++m) {
                    if (SC::wave(m, NW) != w) continue;
                    f4 d = (f4)0.0f;
#pragma unroll
                    for (int ks = 0; ks < KSN; ++ks)
                        d = mma_inputs(d, TN::by_row(sb, ln, SC::keys(m), ks), TN::by_row(sc, ln, SC::query(m), ks));
#pragma unroll
                    for (int o = 0; o < OWN; ++o)
                        if (o == own) D[o] = d;
                    ++own;
                }
            }
            const Steps<Q> &s = ss[turn & 1];
            int own = 0;
#pragma unroll
            for (int m = 0; m < SC::TILES; ++m) {
                if (SC::wave(m, NW) != w) continue;
                const int it = SC::query(m), jt = SC::keys(m);
                f4 p = (f4)0.0f, d = D[0];
#pragma unroll
                for (int ks = 0; ks < KSP; ++ks)
                    p = mma_inputs(p, TP::by_row(sx, lp, jt, ks), TP::by_row(sy, lp, it, ks));
                p *= weights<Q, false>(s, it, jt, i16, g);
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
            if (w == NW - 1) {
                const int next = k + 1 < HB ? k + 1 : 0;
                const bool same = two && k == 0;
                make_steps<Q, false>(ss[(turn + 1) & 1], dt.value(), same ? bias[next] : bias[0], same ? rate[next] : rate[0], lane);
            }
            fetch_dt(two ? n + 1 : n + 2, two ? k : 0);
            if (own_n) {
                // what the state at the block's start gives
                f4 F[IT];
#pragma unroll
                for (int it = 0; it < IT; ++it) F[it] = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KSP; ++ks) {
                    const Op<HELD> st = split<HELD>(__builtin_shufflevector(S[k][2 * ks], S[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int it = 0; it < IT; ++it) F[it] = mma(F[it], st, TP::by_row(sy, lp, it, ks));
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) {
                    F[it] *= s.out[16 * it + i16];
                    const f4 e = F[it] * TN::four(sc, ln, it);
                    const float sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                    if (g == 0) rp[w][16 * it + i16] = sum;
                    O[it] += F[it];
                }
                // the state at the block's end
                {
                    const float keep = pow2(s.total);
#pragma unroll
                    for (int kt = 0; kt < KTP; ++kt) S[k][kt] *= keep;
#pragma unroll
                    for (int ks = 0; ks < QS; ++ks) {
                        const f4 lo = *(const f4 *)(s.in + 32 * ks + 4 * g), hi = *(const f4 *)(s.in + 32 * ks + 16 + 4 * g);
                        const Op<HELD> u = split<HELD>(values(v[ks]) * __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                        for (int kt = 0; kt < KTP; ++kt) S[k][kt] = mma(S[k][kt], TP::by_col(sx, lp, ks, kt), u);
                    }
                }
            }
            lds_barrier();
#pragma unroll
            for (int it = 0; it < IT; ++it)
#pragma unroll
                for (int ks = 0; ks <= it / 2; ++ks)
                    if (own_n) O[it] = SC::product(O[it], v[ks], sm, it, ks, lane);
            // sums over waves and tiles: each wave those of its sixteens, lane = position
            const size_t line = (size_t)(at.b * a.H + at.h0 + k) * a.T;
#pragma unroll
            for (int turn = 0; turn < TURNS; ++turn) {
                const int K = w + NW * turn, at16 = 16 * K + i16;
                float ri = 0.0f, dl = 0.0f;
                if (K < IT) {
                    float before = 0.0f, after = 0.0f;
                    for (int x = 0; x < KTN; ++x) ri += rp[x][at16];
#pragma unroll
                    for (int m = 0; m < SC::TILES; ++m) {
                        const int it = SC::query(m), jt = SC::keys(m);
                        if (it == jt) {
                            if (K == it) dl += ends[m][i16];
                        } else {
                            if (K == it) after += ends[m][i16];
                            if (K == jt) before += starts[m][i16];
                            if (jt < K && K < it) dl += sum16(ends[m][i16]);
                        }
                    }
                    dl += suffix16(after) + moved<0x111>(prefix16(before));
                }
                put_line<Q>(a.rint + line, base, at.t1, K < IT && g == 0 ? at16 : -1, ri);
                put_line<Q>(a.dlin + line, base, at.t1, K < IT && g == 0 ? at16 : -1, dl);
            }
            ++turn;
        }
#pragma unroll
        for (int it = 0; it < IT; ++it) out.template put<Q>(base, i16, 16 * it, 16 * w + 4 * g, a.N, at.t1, O[it]);
    }
    // sums for the skip: by wave in LDS, then over the waves in order
    lds_barrier();
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        double s = skips[k][tid];
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        if (lane == 0) ((double *)rp[w])[k] = s;
    }
    lds_barrier();
    if (tid < at.nh) {
        double s = 0.0;
        for (int y = 0; y < NW; ++y) s += ((const double *)rp[y])[tid];
        a.skipp[(size_t)(at.b * a.H + at.h0 + tid) * a.nseg + at.seg] = s;
    }
    if (a.chunks == 1)
        clear_rows<T>((T *)a.gc + at.rb * a.gc_row + at.grp * a.N, a.gc_row, at.t0 + at.nblk * Q, at.t1, a.N, tid, NT);
}

// ---- gradients of x and B -----------------------------------------------------------------------------------------
//   du_j = sum_{i>=j} e^{c_i-c_j} (B_j . C_i) dy_i     queries B, keys C, values dy; state G [N x P]     dx = delta du + skip dy
//   dB_j = sum_h delta_j sum_{i>=j} e^{c_i-c_j} (x_j . dy_i) C_i     queries x, keys dy, values C; state G^T [P x N]
// Rows run backwards in time.  A wave holds sixteen columns p of G; its parts, which the product with B needs anyway, go through
// LDS, from where they are read transposed for the product with x.  Only float32 and float16 at 128 x 128 have no room for that
// (98 KB): there a wave holds sixteen columns n of the transpose as well, at twice the products for the updates.
template <class T, int PP, int NN, int HB> __global__ __launch_bounds__((PP > NN ? PP : NN) * 4, waves_for(Parts<T>::raw, PP > NN ? PP : NN)) void k_ssm_grad_xb(SsmArgs a)
{
    constexpr int Q = GRAD_BLOCK, MOST = PP > NN ? PP : NN, NT = MOST * 4, NW = MOST / 16, IT = Q / 16, QS = Q / 32;
    constexpr int KTP = PP / 16, KTN = NN / 16, KSP = PP / 32, KSN = NN / 32;
    constexpr int RAW = Parts<T>::raw, E = (int)sizeof(T);
    typedef Tile<T, Q, PP, NT, true> TP;
    typedef Tile<T, Q, NN, NT, true> TN;
    typedef Scores<Q> SC;
    constexpr int OWN = (SC::TILES + NW - 1) / NW, TURNS = (IT + NW - 1) / NW;
    constexpr bool TWICE = RAW >= 2 && PP == 128 && NN == 128;
    // one array, so that operands' places differ by constants
    __shared__ __attribute__((aligned(16))) __bf16 pool[2 * TP::ELEMS + 2 * TN::ELEMS + 2 * SC::ELEMS + (TWICE ? 0 : HELD * PP * NN)];
    __bf16 *const sx = pool, *const sy = sx + TP::ELEMS, *const sb = sy + TP::ELEMS, *const sc = sb + TN::ELEMS, *const su = sc + TN::ELEMS,
        *const sm = su + SC::ELEMS, *const sg = sm + SC::ELEMS;  // sg: G [p][n]
    __shared__ Steps<Q> ss[2];  // of this head and the next
    __shared__ __attribute__((aligned(16))) float qp[2][NW][Q], xp[NW][Q];  // by wave: its columns' part of qint (of this head and the one before) and of x . du

    const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane >> 4, i16 = lane & 15;
    const Place<T> at(a, HB, Q, a.chunks);
    if (!at.any) return;
    const size_t cells = (size_t)a.P * a.N;
    // Where there are more waves than columns of P, some hold the same ones, and only the first of them write: without a branch the
    // compiler finds the registers (8 x 4000 positions, 8 heads of 64, 128 states: bfloat16 391 us, with one an eighth more, and with P
    // padded to 128 as well a twelfth).  Columns of N are few enough to be branched on.
    const int wp = w % KTP, c0 = 16 * wp + i16, n0 = 16 * w + i16;  // this lane's columns
    const bool own_n = NN == MOST || 16 * w < NN;

    auto base_of = [&](int n) { return at.t0 + Q * (at.nblk - 1 - n); };
    Sources<T> src(a, at, at.nblk ? base_of(0) : at.t0);
    TP rx, ry;
    TN rbt, rct;
    const typename TP::Lane lp(lane, wp);
    const typename TN::Lane ln(lane, w);
    const typename TP::Place plp(tid);
    const typename TN::Place pln(tid);
    rx.init(src.x_bytes, a.P, tid);
    ry.init(src.y_bytes, a.P, tid);
    rbt.init(src.b_bytes, a.N, tid);
    rct.init(src.c_bytes, a.N, tid);

    f4 S[HB][KTN];               // G: rows n, this lane's column p (odd ones negated, here, in LDS and in U)
    f4 R[TWICE ? HB : 1][TWICE ? KTP : 1];  // its transpose: rows p (odd ones negated), this lane's column n
    float rate[HB], bias[HB], skip[HB];
#pragma unroll
    for (int k = 0; k < HB; ++k) {
        const int head = k < at.nh ? at.h0 + k : at.h0;
        rate[k] = a.rate[head];
        bias[k] = a.dt_bias ? a.dt_bias[head] : 0.0f;
        skip[k] = a.skip ? a.skip[head] : 0.0f;
        const float *from = a.gs + ((size_t)(at.b * a.H + head) * (a.nseg + 1) + at.seg + 1) * cells;
#pragma unroll
        for (int kt = 0; kt < KTN; ++kt) {
            const int row = 16 * kt + 4 * g;
            S[k][kt] = at.nblk && row < a.N && c0 < a.P ? *(const f4 *)(from + (size_t)c0 * a.N + row) : (f4)0.0f;
            if (c0 & 1) S[k][kt] = -S[k][kt];
            if constexpr (TWICE) {
                R[k][kt] = (f4)0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (at.nblk && row + r < a.P && n0 < a.N) R[k][kt][r] = (r & 1 ? -1.0f : 1.0f) * from[(size_t)(row + r) * a.N + n0];
            }
        }
    }
    Dt<T> dt;
    const bool two = HB > 1 && at.nh > 1;  // heads in turn
    auto fetch_dt = [&](int n, int k) {
        dt.fetch(src.dt + k * E - (int64_t)Q * n * src.dt_bytes, src.dt_bytes, Q - 1 - lane % Q, n < at.nblk ? at.L - base_of(n) : 0);
    };
    if (at.nblk) {
        const int left = at.L - base_of(0);
        rbt.fetch(rows_at(src.b, left, Q, src.b_bytes), 0);
        rct.fetch(rows_at(src.c, left, Q, src.c_bytes), 0);
        rx.fetch(rows_at(src.x, left, Q, src.x_bytes), 0);
        ry.fetch(rows_at(src.y, left, Q, src.y_bytes), 0);
        fetch_dt(0, 0);
        if (w == 0) make_steps<Q, true>(ss[0], dt.value(), bias[0], rate[0], lane);
        fetch_dt(two ? 0 : 1, two ? 1 : 0);
    }
    const SharedOut<T> out(a, a.gb, a.gb_row, a.partb, a.chunks, at);
    const int gx_bytes = (int)a.gx_row * E;
    char *gxs = (char *)a.gx + (at.rb + (at.nblk ? base_of(0) : at.t0)) * gx_bytes + at.h0 * a.P * E;
    const uint32_t gx_off = 16 * w + 4 * g < a.P ? (uint32_t)((15 - i16) * gx_bytes + (16 * w + 4 * g) * E) : OUTSIDE;
    // The sums of a head over the waves are made while the next one is worked on, until its second barrier; `turn` counts heads.
    int turn = 0;
    auto join = [&](int n, int k, bool any) {
        const size_t line = (size_t)(at.b * a.H + at.h0 + k) * a.T;
        const int base = base_of(n);
#pragma unroll
        for (int x = 0; x < TURNS; ++x) {
            const int K = w + NW * x, at16 = 16 * K + i16;
            float q = 0.0f, s = 0.0f;
            if (K < IT)
                for (int y = 0; y < KTP; ++y) q += qp[(turn & 1) ^ 1][y][at16], s += xp[y][at16];
            put_line<Q>(a.qint + line, base, at.t1, any && K < IT && g == 0 ? Q - 1 - at16 : -1, q);
            put_line<Q>(a.xdu + line, base, at.t1, any && K < IT && g == 0 ? Q - 1 - at16 : -1, s);
        }
    };
    for (int n = 0; n < at.nblk; ++n) {
        const int base = base_of(n);
        rbt.put(sb, pln, tid);
        rct.put(sc, pln, tid);
        Op<RAW> vc[QS];
        f4 O[IT], D[OWN];
#pragma unroll
        for (int it = 0; it < IT; ++it) O[it] = (f4)0.0f;
#pragma unroll
        for (int k = 0; k < HB; ++k) {
            if (k >= at.nh) break;
            rx.template put<true>(sx, plp, tid);
            ry.template put<true>(sy, plp, tid);
            Op<HELD> st[KSN];
            {
#pragma unroll
                for (int ks = 0; ks < KSN; ++ks) {
                    st[ks] = split<HELD>(__builtin_shufflevector(S[k][2 * ks], S[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
                    for (int part = 0; part < (TWICE ? 0 : HELD); ++part) {
                        const u4 v = __builtin_bit_cast(u4, st[ks].p[part]);
                        __bf16 *to = sg + part * PP * NN + 16 * wp * NN + ks / 2 * 64;
                        *(u2 *)(to + ln.row[NN >= 64 ? ks % 2 * 2 : 0]) = (u2){v[0], v[1]};
                        *(u2 *)(to + ln.row[NN >= 64 ? ks % 2 * 2 + 1 : 1]) = (u2){v[2], v[3]};
                    }
                }
            }
            lds_barrier();
            {
                const bool last = k + 1 >= at.nh;
                if (last) src.move(-Q);
                const int left = last ? Q : at.L - base, col = last ? 0 : (k + 1) * a.P * E;
                if (!last || n + 1 < at.nblk) {
                    rx.fetch(rows_at(src.x, left, Q, src.x_bytes), col);
                    ry.fetch(rows_at(src.y, left, Q, src.y_bytes), col);
                    if (last) {
                        rbt.fetch(rows_at(src.b, left, Q, src.b_bytes), 0);
                        rct.fetch(rows_at(src.c, left, Q, src.c_bytes), 0);
                    }
                }
            }
            if (k == 0) join(n > 0 ? n - 1 : 0, at.nh - 1, n > 0);
            else join(n, k - 1, true);
            if (k == 0) {
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) vc[ks] = TN::own_col(sc, ln, ks);
                int own = 0;
#pragma unroll
                for (int m = 0; m < SC::TILES; ++m) {
                    if (SC::wave(m, NW) != w) continue;
                    f4 d = (f4)0.0f;
#pragma unroll
                    for (int ks = 0; ks < KSN; ++ks)
                        d = mma_inputs(d, TN::by_row(sc, ln, SC::keys(m), ks), TN::by_row(sb, ln, SC::query(m), ks));
#pragma unroll
                    for (int o = 0; o < OWN; ++o)
                        if (o == own) D[o] = d;
                    ++own;
                }
            }
            const Steps<Q> &s = ss[turn & 1];
            f4 U[IT];
#pragma unroll
            for (int it = 0; it < IT; ++it) U[it] = (f4)0.0f;
#pragma unroll
            for (int ks = 0; ks < KSN; ++ks)
#pragma unroll
                for (int it = 0; it < IT; ++it) U[it] = mma(U[it], st[ks], TN::by_row(sb, ln, it, ks));
            int own = 0;
#pragma unroll
            for (int m = 0; m < SC::TILES; ++m) {
                if (SC::wave(m, NW) != w) continue;
                const int it = SC::query(m), jt = SC::keys(m);
                f4 p = (f4)0.0f, d = D[0];
#pragma unroll
                for (int ks = 0; ks < KSP; ++ks)
                    p = mma_inputs(p, TP::by_row(sy, lp, jt, ks), TP::by_row(sx, lp, it, ks));
#pragma unroll
                for (int o = 1; o < OWN; ++o)
                    if (o == own) d = D[o];
                ++own;
                const f4 f = weights<Q, true>(s, it, jt, i16, g);
                SC::put(su, it, jt, d * f, lane);
                SC::put(sm, it, jt, p * (f * s.delta[16 * it + i16]), lane);
            }
            if (w == NW - 1) {
                const int next = k + 1 < HB ? k + 1 : 0;
                const bool same = two && k == 0;
                make_steps<Q, true>(ss[(turn + 1) & 1], dt.value(), same ? bias[next] : bias[0], same ? rate[next] : rate[0], lane);
            }
            fetch_dt(two ? n + 1 : n + 2, two ? k : 0);
            // what the state behind the block gives to the gradient of B ..
            if (own_n) {
                f4 F[IT];
#pragma unroll
                for (int it = 0; it < IT; ++it) F[it] = (f4)0.0f;
#pragma unroll
                for (int ks = 0; ks < KSP; ++ks) {
                    Op<HELD> gt;
                    if constexpr (TWICE) gt = split<HELD>(__builtin_shufflevector(R[k][2 * ks], R[k][2 * ks + 1], 0, 1, 2, 3, 4, 5, 6, 7));
                    else gt = TN::template transposed<HELD>(sg, ln.own, 32 * ks * NN, PP * NN);
#pragma unroll
                    for (int it = 0; it < IT; ++it) F[it] = mma(F[it], gt, TP::by_row(sx, lp, it, ks));
                }
#pragma unroll
                for (int it = 0; it < IT; ++it) O[it] += F[it] * (s.out[16 * it + i16] * s.delta[16 * it + i16]);
            }
            // .. and to that of u
            f4 xv[IT], yv[IT];
            Op<RAW> vy[QS];
#pragma unroll
            for (int ks = 0; ks < QS; ++ks) vy[ks] = TP::own_col(sy, lp, ks);
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                U[it] *= s.out[16 * it + i16];
                xv[it] = TP::four(sx, lp, it);
                yv[it] = TP::four(sy, lp, it);
                const f4 e = U[it] * xv[it];
                const float sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                if (g == 0) qp[turn & 1][w][16 * it + i16] = sum * s.delta[16 * it + i16];
            }
            // the state before the block
            {
                const float keep = pow2(s.total);
#pragma unroll
                for (int kt = 0; kt < KTN; ++kt) S[k][kt] *= keep;
#pragma unroll
                for (int ks = 0; ks < QS; ++ks) {
                    const f4 lo = *(const f4 *)(s.in + 32 * ks + 4 * g), hi = *(const f4 *)(s.in + 32 * ks + 16 + 4 * g);
                    const f8 in = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                    const Op<HELD> u = split<HELD>(values(vy[ks]) * in);
#pragma unroll
                    for (int kt = 0; kt < KTN; ++kt) S[k][kt] = mma(S[k][kt], TN::by_col(sc, ln, ks, kt), u);
                    if constexpr (TWICE) {
                        const Op<HELD> v = split<HELD>(values(vc[ks]) * in);
#pragma unroll
                        for (int kt = 0; kt < KTP; ++kt) R[k][kt] = mma(ks ? R[k][kt] : R[k][kt] * keep, TP::by_col(sy, lp, ks, kt), v);
                    }
                }
            }
            lds_barrier();
            if (own_n) {
#pragma unroll
                for (int it = 0; it < IT; ++it)
#pragma unroll
                    for (int ks = 0; ks <= it / 2; ++ks) O[it] = SC::product(O[it], vc[ks], sm, it, ks, lane);
            }
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const int r = 16 * it + i16;
#pragma unroll
                for (int ks = 0; ks <= it / 2; ++ks) U[it] = SC::product(U[it], vy[ks], su, it, ks, lane);
                const f4 e = U[it] * xv[it], o = (U[it] * s.delta[r] + yv[it] * skip[k]) * (f4){1.0f, -1.0f, 1.0f, -1.0f};
                const float sum = sum_rows(e[0] + e[1] + e[2] + e[3]);
                if (g == 0) xp[w][r] = sum;
                store_four<T>(rows_at(gxs, at.t1 - base, Q, gx_bytes), gx_off, 16 * (IT - 1 - it) * gx_bytes + k * a.P * E, o);
            }
            ++turn;
        }
        gxs -= (int64_t)Q * gx_bytes;
#pragma unroll
        for (int it = 0; it < IT; ++it) out.template put<Q>(base, 15 - i16, 16 * (IT - 1 - it), 16 * w + 4 * g, a.N, at.t1, O[it]);
    }
    lds_barrier();
    if (at.nblk) join(at.nblk - 1, at.nh - 1, true);
    clear_rows<T>((T *)a.gx + at.rb * a.gx_row + at.h0 * a.P, a.gx_row, at.t0 + at.nblk * Q, at.t1, at.nh * a.P, tid, NT);
    if (a.chunks == 1)
        clear_rows<T>((T *)a.gb + at.rb * a.gb_row + at.grp * a.N, a.gb_row, at.t0 + at.nblk * Q, at.t1, a.N, tid, NT);
}

template <class T, int PP, int NN> int launch_grad(const SsmArgs &a, hipStream_t st)
{
    constexpr int MOST = PP > NN ? PP : NN, HB = MOST <= 64 ? GRAD_HEADS : 1;
    const long grid = ((long)a.B * a.nseg + 7) / 8 * 8 * a.G * a.chunks;
    if (grid > 0x7fffffffL) return SEMICRF_EUNSUPPORTED;
    const dim3 g((unsigned)grid), t(MOST * 4);
    if (a.heads > 1) {
        hipLaunchKernelGGL((k_ssm_grad_c<T, PP, NN, HB>), g, t, 0, st, a);
        hipLaunchKernelGGL((k_ssm_grad_xb<T, PP, NN, HB>), g, t, 0, st, a);
    } else {
        hipLaunchKernelGGL((k_ssm_grad_c<T, PP, NN, 1>), g, t, 0, st, a);
        hipLaunchKernelGGL((k_ssm_grad_xb<T, PP, NN, 1>), g, t, 0, st, a);
    }
    return launched();
}
template <class T, int NN> int launch_grad_p(const SsmArgs &a, hipStream_t st)
{
    if (a.P <= 32) return launch_grad<T, 32, NN>(a, st);
    if (a.P <= 64) return launch_grad<T, 64, NN>(a, st);
    return launch_grad<T, 128, NN>(a, st);
}
template <class T> int ssm_grad(const SsmArgs &a, hipStream_t st)
{
    if (a.N <= 32) return launch_grad_p<T, 32>(a, st);
    if (a.N <= 64) return launch_grad_p<T, 64>(a, st);
    return launch_grad_p<T, 128>(a, st);
}

}  // namespace semicrf_enc

#endif
