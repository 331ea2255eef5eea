// Selective state space scan: the small kernels around the scans, the single-token form, and the entry points.
#include "ssm.h"

namespace semicrf_enc {

// States at the segments' boundaries from what each segment adds: H_{s+1} = kept_s H_s + added_s forwards, and with `grad` the
// same backwards for gradients of states, and the pairs of positions that cross each boundary: <G, H> there, by wave.  A
// thread owns four entries, and a workgroup is a wave, so that few heads still reach most of the chip.  Bound by the states, read and
// written: 32 heads' 98 boundaries of 16 KB both ways 53 us.
template <bool REV> __device__ __forceinline__ void chain_line(const SsmArgs &a, size_t bh, size_t at, bool mine, double *cross, size_t parts)
{
    const size_t cells = (size_t)a.P * a.N;
    float *line = (REV ? a.gs : a.hs) + bh * (a.nseg + 1) * cells + at;
    const float *first = REV ? a.grad_last : a.state, *states = a.hs ? a.hs + bh * (a.nseg + 1) * cells + at : nullptr;
    float *last = REV ? a.gstate : a.state_out;
    const float *kept = a.kept + bh * a.nseg;
    constexpr int AHEAD = 8;
    f4 h = first && mine ? *(const f4 *)(first + bh * cells + at) : (f4)0.0f;
    // the next eight segments' loads are on their way while eight are worked on
    f4 added[AHEAD], there[REV ? AHEAD : 1], next[AHEAD], next_there[REV ? AHEAD : 1];
    float k[AHEAD], next_k[AHEAD];
    auto fetch = [&](int s0) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            next[i] = (f4)0.0f;
            if constexpr (REV) next_there[i] = (f4)0.0f;
            next_k[i] = 0.0f;
            if (s0 + i < a.nseg && mine) {
                const int s = REV ? a.nseg - 1 - s0 - i : s0 + i;
                next[i] = *(const f4 *)(line + (size_t)(REV ? s : s + 1) * cells);
                if constexpr (REV) next_there[i] = *(const f4 *)(states + (size_t)s * cells);
                next_k[i] = kept[s];
            }
        }
    };
    fetch(0);
    auto product = [&](f4 g, f4 h) { return (double)g[0] * h[0] + (double)g[1] * h[1] + (double)g[2] * h[2] + (double)g[3] * h[3]; };
    if constexpr (REV) {
        double s = mine ? product(h, *(const f4 *)(states + (size_t)a.nseg * cells)) : 0.0;
        for (int d = 1; d < 64; d *= 2) s += __shfl_xor(s, d);
        if (threadIdx.x == 0) cross[(bh * (a.nseg + 1) + a.nseg) * parts] = s;
    }
    if (mine) *(f4 *)(line + (REV ? (size_t)a.nseg * cells : 0)) = h;
    for (int s0 = 0; s0 < a.nseg; s0 += AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            added[i] = next[i], k[i] = next_k[i];
            if constexpr (REV) there[i] = next_there[i];
        }
        if (s0 + AHEAD < a.nseg) fetch(s0 + AHEAD);
        double pairs[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            pairs[i] = 0.0;
            if (s0 + i < a.nseg) {
                const int s = REV ? a.nseg - 1 - s0 - i : s0 + i;
                h = k[i] * h + added[i];
                if (mine) *(f4 *)(line + (size_t)(REV ? s : s + 1) * cells) = h;
                if constexpr (REV) pairs[i] = product(h, there[i]);
            }
        }
        if constexpr (REV) {
#pragma unroll
            for (int d = 1; d < 64; d *= 2)
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) pairs[i] += __shfl_xor(pairs[i], d);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (s0 + i < a.nseg && threadIdx.x == 0) cross[(bh * (a.nseg + 1) + a.nseg - 1 - s0 - i) * parts] = pairs[i];
        }
    }
    if (last && mine) *(f4 *)(last + bh * cells + at) = h;
}

__global__ __launch_bounds__(64) void k_ssm_chain(SsmArgs a, bool grad)
{
    const size_t cells = (size_t)a.P * a.N;
    const unsigned parts = (unsigned)((cells / 4 + 63) / 64);
    const size_t at = (size_t)(blockIdx.x % parts * 64 + threadIdx.x) * 4, bh = blockIdx.x / parts;
    const bool mine = at < cells;
    chain_line<false>(a, bh, at, mine, nullptr, 0);
    if (grad) chain_line<true>(a, bh, at, mine, a.cross + blockIdx.x % parts, parts);
}

// Gradients of the steps.  l_t multiplies everything that passes step t: pairs (i, j) with j < t <= i, of four kinds by block:
//   dlin[t]  both ends in t's block,
//   rint[i]  from before the block to i in it; those with i >= t count,
//   qint[j]  from j in the block to behind it; those with j < t count,
//   across   from before the block to behind it.
// The pairs that cross a boundary are known at a segment's ends (k_ssm_chain).  From the later one backwards, taking off those that
// begin in a block leaves its `across`, and adding those that end in it gives what crosses its start.  Rounding adds up along that
// walk, and all positions of a block share it.  What the walk is off by at the segment's start is therefore taken back: each value
// by the share that its variance has of the difference's, both ends' included, with the squares of what has been added up
// (all of it rounded alike) as variances.  Where a block keeps less than 2^-30, nothing is left of the difference but rounding:
// `across` is 0, and the walk begins anew.  One wave per (sequence, head, segment); bound by latency, 60 to 80 us of the 2110 that
// training on 4 x 100 000 positions of 8 heads takes.
constexpr int MOST_BLOCKS = 32;  // of a segment of 1024

template <class T> __global__ __launch_bounds__(64) void k_ssm_steps(SsmArgs a)
{
    // variances in 64 bits: squares of float32 values need not fit in 32
    __shared__ double over[MOST_BLOCKS], qs[MOST_BLOCKS], rs[MOST_BLOCKS], q2[MOST_BLOCKS], r2[MOST_BLOCKS], var[MOST_BLOCKS];
    __shared__ float ks[MOST_BLOCKS];
    constexpr int Q = GRAD_BLOCK;
    const int lane = threadIdx.x, r = lane & (Q - 1);
    const int seg = blockIdx.x % a.nseg, bh = blockIdx.x / a.nseg, h = bh % a.H, b = bh / a.H;
    const int L = length_of(a.lengths, b, a.T);
    const int t0 = seg * a.seg, t1 = t0 + a.seg < a.T ? t0 + a.seg : a.T;
    const int used = (t1 < L ? t1 : L) - t0, nblk = used > 0 ? (used + Q - 1) / Q : 0, end = t0 + (used > 0 ? used : 0);
    T *gdt = (T *)a.gdt + (int64_t)b * a.T * a.gdt_row + h;
    const T *dts = (const T *)a.dt + (int64_t)b * a.T * a.dt_row + h;
    const float rate = a.rate[h], bias = a.dt_bias ? a.dt_bias[h] : 0.0f;
    // sums of each block, two blocks at a time
    for (int i = t0; i < end; i += 64) {
        const int t = i + lane;
        const bool in = t < end;
        const size_t at = (size_t)bh * a.T + t;
        double q = in ? (double)a.qint[at] : 0.0, ri = in ? (double)a.rint[at] : 0.0;
        float kept = in ? softplus((float)dts[t * a.dt_row] + bias) : 0.0f;
        double qq = q * q, rr = ri * ri;
        for (int d = 1; d < Q; d *= 2) {
            q += __shfl_xor(q, d), ri += __shfl_xor(ri, d), kept += __shfl_xor(kept, d);
            qq += __shfl_xor(qq, d), rr += __shfl_xor(rr, d);
        }
        const int n = (i - t0 + lane) / Q;
        if (r == 0 && n < nblk) qs[n] = q, rs[n] = ri, ks[n] = kept, q2[n] = qq, r2[n] = rr;
    }
    double cross[2] = {0.0, 0.0};
    {
        const int parts = (a.P * a.N / 4 + 63) / 64;
        const double *from = a.cross + ((size_t)bh * (a.nseg + 1) + seg) * parts;
        for (int e = 0; e < 2; ++e) {
            if (lane < parts) cross[e] = from[(size_t)e * parts + lane];
            for (int d = 1; d < 64; d *= 2) cross[e] += __shfl_xor(cross[e], d);
        }
    }
    __syncthreads();
    {
        double across = cross[1];
        double spread = cross[1] * cross[1];  // the walk's variance
        int first = nblk;                     // its blocks: up to here
        for (int n = nblk - 1; n >= 0; --n) {
            const double qi = qs[n], ri = rs[n];
            const bool gone = ks[n] * rate * 1.44269504f < -30.0f;
            across -= qi;
            spread += q2[n];
            if (lane == 0) over[n] = across, var[n] = spread;
            if (gone || n == 0) {
                const double off = gone ? across : across + ri - cross[0];
                const double all = gone ? spread : spread + r2[n] + cross[0] * cross[0];
                __syncthreads();
                if (lane < first - n && all > 0.0) over[n + lane] -= off * (var[n + lane] / all);
                __syncthreads();
                if (gone && lane == 0) over[n] = 0.0;
                first = n;
                across = 0.0;
                spread = 0.0;
            }
            across += ri;
            spread += r2[n];
        }
    }
    __syncthreads();
    double grate = 0.0, gbias = 0.0;
    for (int i = t0; i < end; i += 64) {
        const int t = i + lane;
        const bool in = t < end;
        const size_t at = (size_t)bh * a.T + t;
        float tail = 0.0f, qi = 0.0f, own = 0.0f, dx = 0.0f, raw = 0.0f;
        if (in) {
            tail = a.rint[at], own = a.dlin[at], qi = a.qint[at], dx = a.xdu[at];
            raw = (float)dts[t * a.dt_row] + bias;
        }
        float head = __shfl_up(qi, 1);
        if (r == 0) head = 0.0f;
        for (int d = 1; d < Q; d *= 2) {
            const float o = __shfl_down(tail, d), p = __shfl_up(head, d);
            if (r + d < Q) tail += o;
            if (r >= d) head += p;
        }
        if (in) {
            const float dl = own + tail + head + (float)over[(t - t0) / Q], g = (dx + rate * dl) * sigmoid(raw);
            const float one[1] = {g};
            store_n<T, 1>(gdt + t * a.gdt_row, one);
            grate += (double)dl * softplus(raw);
            gbias += (double)g;
        }
    }
    for (int t = (used > 0 ? t0 + used : t0) + lane; t < t1; t += 64) gdt[t * a.gdt_row] = (T)0.0f;
    for (int d = 1; d < 64; d *= 2) grate += __shfl_xor(grate, d), gbias += __shfl_xor(gbias, d);
    if (lane == 0) {
        a.headp[2 * (size_t)blockIdx.x] = grate;
        a.headp[2 * (size_t)blockIdx.x + 1] = gbias;
    }
}

// Sums over sequences and segments, in a fixed order.  One workgroup per head.
__global__ __launch_bounds__(256) void k_ssm_params(SsmArgs a)
{
    __shared__ double s[3][256];
    const int h = blockIdx.x, tid = threadIdx.x;
    double rate = 0.0, bias = 0.0, skip = 0.0;
    const int n = a.B * a.nseg;
    for (int k = tid; k < n; k += 256) {
        const size_t at = ((size_t)(k / a.nseg) * a.H + h) * a.nseg + k % a.nseg;
        rate += a.headp[2 * at];
        bias += a.headp[2 * at + 1];
        skip += a.skipp[at];
    }
    s[0][tid] = rate, s[1][tid] = bias, s[2][tid] = skip;
    for (int d = 128; d > 0; d /= 2) {
        __syncthreads();
        if (tid < d)
            for (int k = 0; k < 3; ++k) s[k][tid] += s[k][tid + d];
    }
    if (tid == 0) {
        a.grate[h] = (float)s[0][0];
        if (a.gbias) a.gbias[h] = (float)s[1][0];
        if (a.gskip) a.gskip[h] = (float)s[2][0];
    }
}

// Gradients of B and C where several workgroups have parts: their sum, in order.  A thread owns four columns of a row.  Bound by the
// parts: four of 400 000 rows of 64 and 64 columns, 922 MB in 157 us (5.9 TB/s; 181 where the parts
// are read through the caches).
template <class T> __global__ __launch_bounds__(256) void k_ssm_heads(SsmArgs a)
{
    const int quads = a.N / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, rows = (int64_t)a.B * a.T;
    if (at >= rows * a.G * quads) return;
    const int64_t row = at / quads / a.G, col = at % (quads * a.G) * 4;
    const int b = (int)(row / a.T), t = (int)(row % a.T);
    const float *part = blockIdx.y ? a.partc : a.partb;
    f4 s = (f4)0.0f;
    if (t < length_of(a.lengths, b, a.T))
        for (int k = 0; k < a.chunks; ++k) s += __builtin_nontemporal_load((const f4 *)(part + ((int64_t)k * rows + row) * a.G * a.N + col));
    const float o[4] = {s[0], s[1], s[2], s[3]};
    store_n<T, 4>((T *)(blockIdx.y ? a.gc : a.gb) + row * (blockIdx.y ? a.gc_row : a.gb_row) + col, o);
}

// ---- one more token of each stream --------------------------------------------------------------------------------

struct StepArgs {
    const void *u, *dt, *ring;
    int64_t u_row, dt_row;
    const float *weight, *bias, *rate, *skip, *dt_bias, *state;
    const int32_t *seen;
    int B, H, P, G, N, W;
    void *y, *ring_out;
    float *state_out;
    bool linear;
};

// One launch for the whole step: a workgroup owns 16 R rows of one head's [P x N] state (16 lanes to a row), and convolves what it
// needs for them: its channels of x and its group's B and C, again in every workgroup of the group (2 N W multiply-adds)
// rather than in a launch before this one.  The ring holds the last W tokens at slot (position mod W), so the one slot that
// is written is the one nobody reads.
// Bound by the state, read and written once and past the caches (51 us through them); its loads are on their way before the
// convolution starts: 192 streams of 16 heads of 64 x 128 take 39 us (206 MB, 5.3 TB/s).  One stream takes 5 us, a launch and
// three loads that wait for one another.  Sixteen rows to a workgroup spread one stream over the chip; where there are
// workgroups enough, 64 rows convolve B and C a quarter as often.
template <class T, int R> __global__ __launch_bounds__(256) void k_ssm_step(StepArgs a)
{
    constexpr int ROWS = 16 * R;
    __shared__ __attribute__((aligned(16))) float sb[128], sc[128];  // read four at a time
    __shared__ float sx[ROWS];
    const int tid = threadIdx.x, tiles = (a.P + ROWS - 1) / ROWS;
    const int tile = blockIdx.x % tiles, h = blockIdx.x / tiles % a.H, b = blockIdx.x / tiles / a.H;
    const int grp = h / (a.H / a.G), channels = a.H * a.P + 2 * a.G * a.N;
    const int p0 = tile * ROWS + tid / 16, q = tid % 16;
    const size_t cell = (((size_t)b * a.H + h) * a.P + p0) * a.N;  // rows p0, p0 + 16, ..
    f4 s[R][2];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int n = 4 * (q + 16 * k);
            if (p0 + 16 * r < a.P && n < a.N) s[r][k] = __builtin_nontemporal_load((const f4 *)(a.state + cell + (size_t)16 * r * a.N + n));
        }
    const int seen = a.seen[b], W = a.W;
    const bool live = seen >= 0;
    const float raw = live ? (float)((const T *)a.dt)[b * a.dt_row + h] + (a.dt_bias ? a.dt_bias[h] : 0.0f) : 0.0f;
    const int slot = live ? seen % W : -1;
    for (int k = tid; k < ROWS + 2 * a.N; k += 256) {
        int ch;
        float *to;
        bool mine = true;  // whether this workgroup writes the channel's ring
        if (k < ROWS) {
            if (tile * ROWS + k >= a.P) continue;
            ch = h * a.P + tile * ROWS + k;
            to = sx + k;
        } else {
            const int which = k - ROWS >= a.N, n = k - ROWS - which * a.N;
            ch = a.H * a.P + (which * a.G + grp) * a.N + n;
            to = (which ? sc : sb) + n;
            mine = tile == 0 && h % (a.H / a.G) == 0;
        }
        const T *ring = (const T *)a.ring + ((size_t)b * channels + ch) * W;
        T *ring_out = (T *)a.ring_out + ((size_t)b * channels + ch) * W;
        const T fresh = live ? ((const T *)a.u)[b * a.u_row + ch] : (T)0.0f;
        float v = a.bias ? a.bias[ch] : 0.0f;
        for (int j = 0; j < W; ++j) {
            // slot j holds the newest position up to `seen` that is j mod W
            const int back = !live ? 0 : slot >= j ? slot - j : slot - j + W;
            const T held = j == slot ? fresh : ring[j];
            if (live && back <= seen) v += a.weight[ch * W + W - 1 - back] * (float)held;
            if (mine && (ring_out != ring || j == slot)) ring_out[j] = held;
        }
        *to = a.linear ? v : v * sigmoid(v);
    }
    __syncthreads();
    const float delta = softplus(raw), keep = expf(delta * a.rate[h]), skip = a.skip ? a.skip[h] : 0.0f;
    f4 vb[2], vc[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int n = 4 * (q + 16 * k);
        vb[k] = vc[k] = (f4)0.0f;
        if (n < a.N) vb[k] = *(const f4 *)(sb + n), vc[k] = *(const f4 *)(sc + n);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int p = p0 + 16 * r;
        const bool in = p < a.P;
        const float x = in ? sx[tid / 16 + 16 * r] : 0.0f, u = delta * x;
        float y = 0.0f;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int n = 4 * (q + 16 * k);
            if (in && n < a.N) {
                if (live) {
                    s[r][k] = s[r][k] * keep + u * vb[k];
                    const f4 m = s[r][k] * vc[k];
                    y += m[0] + m[1] + m[2] + m[3];
                }
                if (live || a.state_out != a.state) __builtin_nontemporal_store(s[r][k], (f4 *)(a.state_out + cell + (size_t)16 * r * a.N + n));
            }
        }
#pragma unroll
        for (int d = 1; d < 16; d *= 2) y += __shfl_xor(y, d);
        if (q == 0 && in) {
            const float o[1] = {live ? y + skip * x : 0.0f};
            store_n<T, 1>((T *)a.y + ((size_t)b * a.H + h) * a.P + p, o);
        }
    }
}

template <class T> void launch_step(const StepArgs &a, hipStream_t st)
{
    const int64_t whole = (int64_t)a.B * a.H * ((a.P + 63) / 64);
    if (whole >= 1024) hipLaunchKernelGGL((k_ssm_step<T, 4>), dim3((unsigned)whole), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_ssm_step<T, 1>), dim3((unsigned)(a.B * a.H * ((a.P + 15) / 16))), dim3(256), 0, st, a);
}

// ---- planning -----------------------------------------------------------------------------------------------------

struct SsmPlan {
    int seg, nseg, heads, chunks;
    size_t hs, gs, kept, partc, partb, rint, dlin, qint, xdu, skipp, cross, headp, total;
};

// Positions of a segment, by sequences and what a workgroup takes of each: as many segments as make three workgroups to a compute
// unit, which is what the registers of most kernels let run at once; more would only add states to hand on (twice as many:
// training on 32 x 1999 positions of 8 heads 438 us instead of 411, 400 000 positions of 8 heads forwards 493 instead of 465),
// and shorter ones than 256 positions cost more than their share of the states.
int segment_length(int B, int T, int H)
{
    const long groups = (long)B * H, want = 768;
    long seg = ((long)T * groups + want - 1) / want;
    if (seg < 256) seg = 256;
    const long whole = ((long)T + 63) / 64 * 64;
    seg = (seg + 63) / 64 * 64;
    return (int)(seg < whole ? seg : whole);
}

int make_ssm_plan(int B, int T, int H, int P, int G, int N, bool grad, SsmPlan *p)
{
    if (B < 1 || T < 1 || H < 1 || P < 1 || G < 1 || N < 1 || H % G) return SEMICRF_EINVAL;
    if (P % 8 || N % 8 || P > 128 || N > 128 || T > (1 << 30) || (double)B * T * H > 2e9) return SEMICRF_EUNSUPPORTED;
    p->seg = segment_length(B, T, H);
    p->heads = p->chunks = 1;
    if (grad) {
        // two heads to a workgroup of the gradient kernels where that leaves two workgroups for each compute unit
        const int hpg = H / G;
        const long groups = (long)B * ((T + 255) / 256) * G;
        const bool room = P <= 64 && N <= 64 && hpg > 1;
        p->heads = room && groups * ((hpg + GRAD_HEADS - 1) / GRAD_HEADS) >= 512 ? GRAD_HEADS : 1;
        p->chunks = (hpg + p->heads - 1) / p->heads;
        p->seg = segment_length(B, T, G * p->chunks);
        if (p->seg > 32 * MOST_BLOCKS) p->seg = 32 * MOST_BLOCKS;
    }
    p->nseg = (T + p->seg - 1) / p->seg;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    const size_t bh = (size_t)B * H, cells = (size_t)P * N, rows = (size_t)B * T;
    const bool chain = grad || p->nseg > 1;
    p->hs = take(chain ? bh * (p->nseg + 1) * cells * 4 : 0);
    p->kept = take(chain ? bh * p->nseg * 4 : 0);
    if (grad) {
        p->gs = take(bh * (p->nseg + 1) * cells * 4);
        p->partc = take(p->chunks > 1 ? p->chunks * rows * G * N * 4 : 0);
        p->partb = take(p->chunks > 1 ? p->chunks * rows * G * N * 4 : 0);
        p->rint = take(rows * H * 4);
        p->dlin = take(rows * H * 4);
        p->qint = take(rows * H * 4);
        p->xdu = take(rows * H * 4);
        p->skipp = take(bh * p->nseg * 8);
        p->cross = take(bh * (p->nseg + 1) * ((cells / 4 + 63) / 64) * 8);
        p->headp = take(bh * p->nseg * 16);
    }
    p->total = at;
    return SEMICRF_OK;
}

int grad(int type, const SsmArgs &a, hipStream_t st)
{
    if (type == ACT_BF16) return ssm_grad<__bf16>(a, st);
    if (type == ACT_F16) return ssm_grad<_Float16>(a, st);
    return ssm_grad<float>(a, st);
}

int scan(int type, bool out, bool both, const SsmArgs &a, hipStream_t st)
{
    if (type == ACT_BF16) return ssm_scan<__bf16>(out, both, a, st);
    if (type == ACT_F16) return ssm_scan<_Float16>(out, both, a, st);
    return ssm_scan<float>(out, both, a, st);
}

int chain(bool grad, const SsmArgs &a, hipStream_t st)
{
    hipLaunchKernelGGL(k_ssm_chain, dim3((unsigned)((a.P * a.N / 4 + 63) / 64 * a.B * a.H)), dim3(64), 0, st, a, grad);
    return launched();
}

int ssm_inputs(SsmArgs &a, int type, const void *x, int64_t x_row, const void *b, int64_t b_row, const void *c,
               int64_t c_row, const void *dt, int64_t dt_row, const float *rate, const float *skip,
               const float *dt_bias, const int32_t *lengths, const float *state, int B, int T, int H, int P, int G, int N)
{
    if (type < 0 || !dt || !rate || dt_row < H || dt_row > (1 << 22) || ((uintptr_t)state & 15)) return SEMICRF_EINVAL;
    if (!rows_ok(x, x_row, (int64_t)H * P, type) || !rows_ok(b, b_row, (int64_t)G * N, type) ||
        !rows_ok(c, c_row, (int64_t)G * N, type))
        return SEMICRF_EINVAL;
    a.x = x; a.b = b; a.c = c; a.dt = dt;
    a.x_row = x_row; a.b_row = b_row; a.c_row = c_row; a.dt_row = dt_row;
    a.rate = rate; a.skip = skip; a.dt_bias = dt_bias; a.lengths = lengths; a.state = state;
    a.B = B; a.T = T; a.H = H; a.P = P; a.G = G; a.N = N;
    return SEMICRF_OK;
}

}  // namespace semicrf_enc

using namespace semicrf_enc;

extern "C" {

int semicrf_ssm_workspace_bytes(int B, int T, int H, int P, int G, int N, int want_grad, size_t *bytes)
{
    if (!bytes) return SEMICRF_EINVAL;
    SsmPlan p = {};
    const int rc = make_ssm_plan(B, T, H, P, G, N, want_grad != 0, &p);
    if (rc == SEMICRF_OK) *bytes = p.total;
    return rc;
}

int semicrf_ssm_fwd(const void *x, int64_t x_row, const void *b, int64_t b_row, const void *c, int64_t c_row,
                    const void *dt, int64_t dt_row, const float *rate, const float *skip, const float *dt_bias,
                    const int32_t *lengths, const float *state, int B, int T, int H, int P, int G, int N,
                    unsigned flags, void *workspace, size_t workspace_bytes, void *y, int64_t y_row,
                    float *state_out, void *stream)
{
    SsmPlan p = {};
    if (int rc = make_ssm_plan(B, T, H, P, G, N, false, &p)) return rc;
    const int type = act_type(flags);
    SsmArgs a = {};
    if (int rc = ssm_inputs(a, type, x, x_row, b, b_row, c, c_row, dt, dt_row, rate, skip, dt_bias, lengths, state, B, T, H,
                            P, G, N))
        return rc;
    if (!rows_ok(y, y_row, (int64_t)H * P, type) || ((uintptr_t)state_out & 15)) return SEMICRF_EINVAL;
    if (p.total && (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.total)) return SEMICRF_EWORKSPACE;
    a.y = y; a.y_row = y_row; a.state_out = state_out;
    a.seg = p.seg; a.nseg = p.nseg;
    const hipStream_t st = (hipStream_t)stream;
    if (p.nseg > 1) {
        a.hs = (float *)((char *)workspace + p.hs);
        a.kept = (float *)((char *)workspace + p.kept);
        if (int rc = scan(type, false, false, a, st)) return rc;
        if (int rc = chain(false, a, st)) return rc;
    }
    return scan(type, true, false, a, st);
}

int semicrf_ssm_bwd(const void *x, int64_t x_row, const void *b, int64_t b_row, const void *c, int64_t c_row,
                    const void *dt, int64_t dt_row, const float *rate, const float *skip, const float *dt_bias,
                    const int32_t *lengths, const float *state, const void *grad_y, int64_t grad_y_row,
                    const float *grad_state_out, int B, int T, int H, int P, int G, int N, unsigned flags,
                    void *workspace, size_t workspace_bytes, void *grad_x, int64_t grad_x_row, void *grad_b,
                    int64_t grad_b_row, void *grad_c, int64_t grad_c_row, void *grad_dt, int64_t grad_dt_row,
                    float *grad_rate, float *grad_skip, float *grad_dt_bias, float *grad_state, void *stream)
{
    SsmPlan p = {};
    if (int rc = make_ssm_plan(B, T, H, P, G, N, true, &p)) return rc;
    const int type = act_type(flags);
    SsmArgs a = {};
    if (int rc = ssm_inputs(a, type, x, x_row, b, b_row, c, c_row, dt, dt_row, rate, skip, dt_bias, lengths, state, B, T, H,
                            P, G, N))
        return rc;
    if (!rows_ok(grad_y, grad_y_row, (int64_t)H * P, type) || !rows_ok(grad_x, grad_x_row, (int64_t)H * P, type) ||
        !rows_ok(grad_b, grad_b_row, (int64_t)G * N, type) || !rows_ok(grad_c, grad_c_row, (int64_t)G * N, type) ||
        !grad_dt || grad_dt_row < H || !grad_rate || ((uintptr_t)grad_state_out & 15) || ((uintptr_t)grad_state & 15))
        return SEMICRF_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.total) return SEMICRF_EWORKSPACE;
    a.gy = grad_y; a.gy_row = grad_y_row; a.grad_last = grad_state_out;
    a.gx = grad_x; a.gx_row = grad_x_row; a.gb = grad_b; a.gb_row = grad_b_row; a.gc = grad_c; a.gc_row = grad_c_row;
    a.gdt = grad_dt; a.gdt_row = grad_dt_row;
    a.grate = grad_rate; a.gskip = grad_skip; a.gbias = grad_dt_bias; a.gstate = grad_state;
    a.seg = p.seg; a.nseg = p.nseg;
    char *w = (char *)workspace;
    a.hs = (float *)(w + p.hs); a.gs = (float *)(w + p.gs); a.kept = (float *)(w + p.kept);
    a.partc = (float *)(w + p.partc); a.partb = (float *)(w + p.partb);
    a.rint = (float *)(w + p.rint); a.dlin = (float *)(w + p.dlin); a.qint = (float *)(w + p.qint);
    a.xdu = (float *)(w + p.xdu); a.skipp = (double *)(w + p.skipp); a.headp = (double *)(w + p.headp);
    a.cross = (double *)(w + p.cross);
    const hipStream_t st = (hipStream_t)stream;
    a.heads = p.heads; a.chunks = p.chunks;
    if (int rc = scan(type, false, true, a, st)) return rc;
    if (int rc = chain(true, a, st)) return rc;
    if (int rc = grad(type, a, st)) return rc;
    const dim3 steps(B * H * p.nseg), heads((unsigned)(((int64_t)B * T * G * (N / 4) + 255) / 256), 2);
    if (type == ACT_BF16) {
        hipLaunchKernelGGL((k_ssm_steps<__bf16>), steps, dim3(64), 0, st, a);
        if (p.chunks > 1) hipLaunchKernelGGL((k_ssm_heads<__bf16>), heads, dim3(256), 0, st, a);
    } else if (type == ACT_F16) {
        hipLaunchKernelGGL((k_ssm_steps<_Float16>), steps, dim3(64), 0, st, a);
        if (p.chunks > 1) hipLaunchKernelGGL((k_ssm_heads<_Float16>), heads, dim3(256), 0, st, a);
    } else {
        hipLaunchKernelGGL((k_ssm_steps<float>), steps, dim3(64), 0, st, a);
        if (p.chunks > 1) hipLaunchKernelGGL((k_ssm_heads<float>), heads, dim3(256), 0, st, a);
    }
    hipLaunchKernelGGL(k_ssm_params, dim3(H), dim3(256), 0, st, a);
    return launched();
}

int semicrf_ssm_step(const void *u, int64_t u_row, const float *weight, const float *bias, const void *dt, int64_t dt_row,
                     const float *rate, const float *skip, const float *dt_bias, const int32_t *seen, const void *ring,
                     const float *state, int B, int H, int P, int G, int N, int W, unsigned flags, void *y,
                     void *ring_out, float *state_out, void *stream)
{
    if (B < 1 || H < 1 || P < 1 || G < 1 || N < 1 || H % G || W < 1) return SEMICRF_EINVAL;
    const int64_t channels = (int64_t)H * P + 2 * (int64_t)G * N;
    const int type = act_type(flags);
    if (P % 8 || N % 8 || P > 128 || N > 128 || W > 4 || (double)B * H * ((P + 15) / 16) > 2e9 || channels > 1e8)
        return SEMICRF_EUNSUPPORTED;
    if (type < 0 || !u || u_row < channels || !weight || !dt || dt_row < H || !rate || !seen || !ring || !state || !y ||
        !ring_out || !state_out || (((uintptr_t)state | (uintptr_t)state_out) & 15))
        return SEMICRF_EINVAL;
    StepArgs a = {u, dt, ring, u_row, dt_row, weight, bias, rate, skip, dt_bias, state, seen, B, H, P, G, N, W,
                  y, ring_out, state_out, (flags & SEMICRF_CONV_LINEAR) != 0};
    const hipStream_t st = (hipStream_t)stream;
    if (type == ACT_BF16) launch_step<__bf16>(a, st);
    else if (type == ACT_F16) launch_step<_Float16>(a, st);
    else launch_step<float>(a, st);
    return launched();
}

}  // extern "C"
