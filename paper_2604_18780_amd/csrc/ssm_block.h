// Blocks of positions in LDS: staging of operands' rows, their fragments, and the steps of a block.
#ifndef SEMICRF_SSM_BLOCK_H
#define SEMICRF_SSM_BLOCK_H

#include <stddef.h>

#include "ssm_ops.h"

namespace semicrf_enc {

// Rows of one sequence behind a range check: of the Q rows from `first`, `bytes` apart, those from the `left`-th on read as zeros
// and are not written.  An offset that a scalar adds (a head's columns) counts in the range, as it does within a row.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const void *first, int left, int Q, int bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(first), 0, left >= Q ? 0x7ffffff0 : left > 0 ? left * bytes : 0, 0x00020000);
}
constexpr uint32_t OUTSIDE = 0x80000000u;  // an offset beyond any range

// Four columns of a row to memory, by range: `off` is the lane's, in bytes, from the rows' first.
template <class T> __device__ __forceinline__ void store_four(__amdgpu_buffer_rsrc_t rows, uint32_t off, int from_row, f4 v)
{
    typedef T T4 __attribute__((ext_vector_type(4)));
    const T4 o = __builtin_convertvector(v, T4);
    if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, o), rows, (int)off, from_row, 0);
    else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u2, o), rows, (int)off, from_row, 0);
}

// dt of a block's positions, one a lane.  The raw value is kept until it is used: a load that is converted at once waits for
// every load before it.
template <class T> struct Dt {
    uint32_t raw;
    bool in;
    // row r of the block whose rows at the head's column begin at `first`, `bytes` apart; `left` positions exist
    __device__ __forceinline__ void fetch(const char *first, int bytes, int r, int left)
    {
        in = r < left;
        const __amdgpu_buffer_rsrc_t from = rows_at(first, left > 0 ? 64 : 0, 64, bytes);
        const int off = in ? r * bytes : (int)OUTSIDE;
        if constexpr (sizeof(T) == 4) raw = __builtin_amdgcn_raw_buffer_load_b32(from, off, 0, 0);
        else raw = (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(from, off, 0, 0);
    }
    __device__ __forceinline__ float value() const
    {
        float v;
        if constexpr (sizeof(T) == 4) v = __builtin_bit_cast(float, raw);
        else v = (float)__builtin_bit_cast(T, (uint16_t)raw);
        return in ? v : -INFINITY;
    }
};

// One operand's rows of a block: Q rows of `dim` elements, staged as bfloat16 parts W wide (padding columns zeros), by NT
// threads.  REV: row r is the block's position Q-1-r.
// A row is W/4 cells of 8 bytes; cell c lies at c ^ mix(row), so that neither the sixteen rows a row-wise read takes side by side
// nor the four rows by four cells of a transposed one meet in a bank.
template <class T, int Q, int W, int NT, bool REV> struct Tile {
    static constexpr int RAW = Parts<T>::raw, E = PER16<T>, PART = Q * W, ELEMS = RAW * PART;
    static constexpr int PR = W / E, ALL = Q * PR, CH = (ALL + NT - 1) / NT;
    uint32_t off[CH];
    u4 r[CH];
    static __device__ __forceinline__ int mix(int rw)
    {
        const int low = (rw >> 2) & 3;
        return W >= 64 ? ((rw & 3) << 2) | low : W == 32 ? ((rw & 2) << 1) | low : low;
    }
    // element `col` (a multiple of 4) of row rw
    static __device__ __forceinline__ int cell(int rw, int col) { return rw * W + (((col >> 2) ^ mix(rw)) << 2); }
    // rows `bytes` apart
    __device__ __forceinline__ void init(int bytes, int dim, int tid)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const int at = tid + NT * i, k = at / PR, col = at % PR * E;
            off[i] = k < Q && col < dim ? (uint32_t)((REV ? Q - 1 - k : k) * bytes + col * (int)sizeof(T)) : OUTSIDE;
        }
    }
    __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t rows, int columns)
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) r[i] = __builtin_amdgcn_raw_buffer_load_b128(rows, (int)off[i], columns, 0);
    }
    // where this thread's chunks lie in a tile: the same for all operands of one shape
    struct Place {
        int a[CH], b[CH];
        __device__ __forceinline__ Place(int tid)
        {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const int at = tid + NT * i, k = at / PR % Q, col = at % PR * E;
                a[i] = cell(k, col);
                b[i] = E == 8 ? cell(k, col + 4) : 0;
            }
        }
    };
    // TURN: odd columns negated
    template <bool TURN = false> __device__ __forceinline__ void put(__bf16 *tile, const Place &to, int tid) const
    {
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            if (ALL % NT != 0 && tid + NT * i >= ALL) break;
            u4 raw = r[i];
            if constexpr (TURN) raw ^= E == 8 ? (u4)0x80000000u : (u4){0u, 0x80000000u, 0u, 0x80000000u};
            if constexpr (RAW == 1) {
                *(u2 *)(tile + to.a[i]) = (u2){raw[0], raw[1]};
                *(u2 *)(tile + to.b[i]) = (u2){raw[2], raw[3]};
            } else if constexpr (RAW == 2) {
                typedef _Float16 h8 __attribute__((ext_vector_type(8)));
                const Op<2> o = split<2>(__builtin_convertvector(__builtin_bit_cast(h8, raw), f8));
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const u4 v = __builtin_bit_cast(u4, o.p[j]);
                    *(u2 *)(tile + to.a[i] + j * PART) = (u2){v[0], v[1]};
                    *(u2 *)(tile + to.b[i] + j * PART) = (u2){v[2], v[3]};
                }
            } else {
                const f4 v = __builtin_bit_cast(f4, raw);
                float x[4] = {v[0], v[1], v[2], v[3]};
                uint32_t p[3][2];
                split_pairs<3, 2>(x, p);
#pragma unroll
                for (int j = 0; j < 3; ++j) *(u2 *)(tile + to.a[i] + j * PART) = (u2){p[j][0], p[j][1]};
            }
        }
    }
    // Sum of the products of this thread's elements of two operands, for sums over a text, which the matrix cores' rounding spoils
    // (3e-5 of a sum over 800 000 positions in float32).
    __device__ __forceinline__ float dot(const Tile &o) const
    {
        typedef T X __attribute__((ext_vector_type(E)));
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const X a = __builtin_bit_cast(X, r[i]), b = __builtin_bit_cast(X, o.r[i]);
#pragma unroll
            for (int e = 0; e < E; ++e) s = __builtin_fmaf((float)a[e], (float)b[e], s);
        }
        return s;
    }
    // Where a lane reads.  Of a cell's number the mix changes its low four bits (three where a row is 32 wide), so the places of
    // all operands of a tile are four (two) numbers of the lane's and constants: the reads' own offsets.
    struct Lane {
        int row[4], col[4];  // of row lane % 16 / of row lane / 4: by bits 2 and 3 of the cell
        int own, four;       // columns 16 w..: read transposed; four of row lane % 16
        __device__ __forceinline__ Lane(int lane, int w)
        {
            const int g = lane >> 4, i16 = lane & 15;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                row[k] = cell(i16, W >= 64 ? 16 * k + 4 * g : 16 * (k & 1) + 4 * g);
                col[k] = cell(lane >> 2, W >= 64 ? 16 * k + 4 * (lane & 3) : 16 * (k & 1) % W + 4 * (lane & 3));
            }
            own = cell(lane >> 2, 16 * w + 4 * (lane & 3));
            four = cell(i16, 16 * w + 4 * g);
        }
    };
    // inner index = column: columns 32 ks + 4g.., + 16 + 4g.. of rows 16 it + lane % 16
    static __device__ __forceinline__ Op<RAW> by_row(const __bf16 *tile, const Lane &at, int it, int ks)
    {
        Op<RAW> o;
        const int more = 16 * it * W + ks / 2 * 64, k0 = W >= 64 ? ks % 2 * 2 : 0;
#pragma unroll
        for (int k = 0; k < RAW; ++k)
            o.p[k] = __builtin_shufflevector(*(const bf4 *)(tile + at.row[k0] + (more + k * PART)),
                                             *(const bf4 *)(tile + at.row[k0 + 1] + (more + k * PART)), 0, 1, 2, 3, 4, 5, 6, 7);
        return o;
    }
    template <int n> static __device__ __forceinline__ Op<n> transposed(const __bf16 *tile, int from, int more, int part)
    {
        typedef __attribute__((address_space(3))) s4 *lds;
        Op<n> o;
        __bf16 *p = const_cast<__bf16 *>(tile) + from;
#pragma unroll
        for (int k = 0; k < n; ++k) {
            const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + (more + k * part)));
            const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds)(p + (more + k * part + 16 * W)));
            o.p[k] = __builtin_shufflevector(__builtin_bit_cast(bf4, lo), __builtin_bit_cast(bf4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return o;
    }
    // inner index = row: rows 32 ks + 4g.., + 16 + 4g.. of column 16 kt + lane % 16 / of the wave's own sixteen columns
    static __device__ __forceinline__ Op<RAW> by_col(const __bf16 *tile, const Lane &at, int ks, int kt)
    {
        return transposed<RAW>(tile, at.col[W >= 64 ? kt % 4 : kt], 32 * ks * W + (W >= 64 ? kt / 4 * 64 : 0), PART);
    }
    static __device__ __forceinline__ Op<RAW> own_col(const __bf16 *tile, const Lane &at, int ks) { return transposed<RAW>(tile, at.own, 32 * ks * W, PART); }
    // columns 16 w + 4g.. of row 16 it + lane % 16
    static __device__ __forceinline__ f4 four(const __bf16 *tile, const Lane &at, int it)
    {
        const __bf16 *p = tile + at.four + 16 * it * W;
        f4 v = __builtin_convertvector(*(const bf4 *)(p + (RAW - 1) * PART), f4);
#pragma unroll
        for (int k = RAW - 2; k >= 0; --k) v += __builtin_convertvector(*(const bf4 *)(p + k * PART), f4);
        return v;
    }
};

// The values an operand's parts stand for.
template <int n> __device__ __forceinline__ f8 values(const Op<n> &o)
{
    f8 v = __builtin_convertvector(o.p[n - 1], f8);
#pragma unroll
    for (int k = n - 2; k >= 0; --k) v += __builtin_convertvector(o.p[k], f8);
    return v;
}

__device__ __forceinline__ float pow2(double v) { return __builtin_amdgcn_exp2f((float)v); }

// Steps of a block of Q positions.  c is log2 of what is kept from the block's start to a position (REV: from its far end in
// time, without the position's own step).  What is kept between two positions is 2^(c_i - c_j): between different sixteens it is
// taken as query[i] * from[j], the two sides of the query's sixteen's first c, neither of which overflows where their product does not.  A position's
// term is scaled by its delta forwards, and by 1 backwards.
// Four positions are read at once, of any element of an array of these: the size is a multiple of 16 bytes.
template <int Q> struct alignas(16) Steps {
    double c[Q];
    float out[Q];               // 2^c
    float in[Q];                // what the state at the block's other end keeps of a position's term, times its scale
    float delta[Q];
    float step[Q];              // what is kept from the position before
    float query[Q - 16];        // of position 16 + i: 2^(c_i - c of the first of its sixteen)
    float from[Q / 16 * (Q / 16 - 1) * 8];  // 2^(c of the first of sixteen k+1 - c_j), scaled, for the 16 k + 16 earlier j: a line for each k
    double total;               // log2 of what the block keeps
    static constexpr __device__ __host__ int line(int k) { return 8 * k * (k + 1); }
};
template <int Q> constexpr bool steps_aligned()
{
    return sizeof(Steps<Q>) % 16 == 0 && offsetof(Steps<Q>, in) % 16 == 0 && offsetof(Steps<Q>, delta) % 16 == 0 &&
           offsetof(Steps<Q>, step) % 16 == 0 && offsetof(Steps<Q>, from) % 16 == 0;
}
static_assert(steps_aligned<32>() && steps_aligned<64>(), "four positions of any element are read as 16 bytes");

// The value of another lane of the wave, by a fixed pattern; 0 where the pattern or the mask of rows of sixteen names none.
template <int CTRL, int ROWS> __device__ __forceinline__ double other(double v)
{
    const u2 x = __builtin_bit_cast(u2, v);
    const u2 y = {(uint32_t)__builtin_amdgcn_update_dpp(0, (int)x[0], CTRL, ROWS, 0xf, true),
                  (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x[1], CTRL, ROWS, 0xf, true)};
    return __builtin_bit_cast(double, y);
}
__device__ __forceinline__ double of_lane(double v, int lane)
{
    const u2 x = __builtin_bit_cast(u2, v);
    const u2 y = {(uint32_t)__builtin_amdgcn_readlane((int)x[0], lane), (uint32_t)__builtin_amdgcn_readlane((int)x[1], lane)};
    return __builtin_bit_cast(double, y);
}

// One wave; lane = row (Q = 32: the upper half of the wave repeats nothing and writes nothing).
template <int Q, bool REV> __device__ __forceinline__ void make_steps(Steps<Q> &s, float dt, float bias, float rate, int lane)
{
    // a step beyond the sequence's end has delta = 0: nothing comes in and nothing is forgotten
    const float raw = dt + bias, delta = raw == -INFINITY ? 0.0f : softplus(raw);
    const double l = (double)delta * (double)rate * 1.4426950408889634;
    double c = l, step = l;
    if (REV) step = other<0x138, 0xf>(l);  // of the lane below: handed back in time, a state passes the later step
    c += other<0x111, 0xf>(c);  // from 1, 2, 4, 8 lanes below in a row of sixteen
    c += other<0x112, 0xf>(c);
    c += other<0x114, 0xf>(c);
    c += other<0x118, 0xf>(c);
    c += other<0x142, 0xa>(c);  // the last of the row before, for rows 1 and 3
    if (Q == 64) c += other<0x143, 0xc>(c);  // lane 31, for rows 2 and 3
    const double total = of_lane(c, Q - 1);
    if (REV) c -= l;
    const float key = REV ? 1.0f : delta;
    double first = of_lane(c, 0);
    float from[Q / 16 - 1];
#pragma unroll
    for (int k = 0; k < Q / 16 - 1; ++k) {
        const double ref = of_lane(c, 16 * (k + 1));
        if (lane >= 16 * (k + 1)) first = ref;
        from[k] = lane < 16 * (k + 1) ? pow2(ref - c) * key : 0.0f;
    }
    if (lane < Q) {
        s.c[lane] = c;
        s.out[lane] = pow2(c);
        s.in[lane] = pow2(total - c) * key;
        s.delta[lane] = delta;
        s.step[lane] = pow2(step);
        if (lane >= 16) s.query[lane - 16] = pow2(c - first);
#pragma unroll
        for (int k = 0; k < Q / 16 - 1; ++k)
            if (lane < 16 * (k + 1)) s.from[Steps<Q>::line(k) + lane] = from[k];
        if (lane == 0) s.total = total;
    }
}

// Weights of scores: sixteen queries `it`, sixteen keys `jt` <= it, as four keys of one query in a lane; 0 where the key lies
// behind the query.  Where the two are the same sixteen, only the last of a lane's keys takes a power; the earlier ones
// multiply what is kept on the way to it.
template <int Q, bool REV> __device__ __forceinline__ f4 weights(const Steps<Q> &s, int it, int jt, int i16, int g)
{
    if (jt < it) return *(const f4 *)(s.from + Steps<Q>::line(it - 1) + 16 * jt + 4 * g) * s.query[16 * (it - 1) + i16];
    const f4 step = *(const f4 *)(s.step + 16 * it + 4 * g);
    const float last = (float)(s.c[16 * it + i16] - s.c[16 * it + 4 * g + 3]);
    f4 e;
    e[3] = i16 >= 4 * g + 3 ? __builtin_amdgcn_exp2f(last) : 0.0f;
#pragma unroll
    for (int r = 2; r >= 0; --r) e[r] = i16 == 4 * g + r ? 1.0f : e[r + 1] * step[r + 1];
    return REV ? e : e * *(const f4 *)(s.delta + 16 * it + 4 * g);
}

// Where scores are handed from the wave that makes them to those that multiply with them: operands of queries 16 it.., keys
// 32 ks.., ks <= it / 2; each is two tiles of sixteen keys, of which the second, where it lies behind the queries (keys from
// 16 it on, it even), is not stored but zeros.
template <int Q> struct Scores {
    static constexpr int IT = Q / 16, TILES = IT * (IT + 1) / 2, ELEMS = TILES * HELD * 64 * 4;
    static constexpr __device__ __host__ bool half(int it, int ks) { return 2 * ks == it; }
    static constexpr __device__ __host__ int first(int it, int ks) { return (it * (it + 1) / 2 + 2 * ks) * HELD * 64 * 4; }
    // tile k of the block, and the wave of NW that makes it: with four waves three, three, two and two, sixteen keys each
    static constexpr __device__ int query(int k) { return IT == 2 ? (k > 0) : k == 0 ? 0 : k == 1 || k == 3 ? 1 : k == 4 || k == 6 || k == 9 ? 2 : 3; }
    static constexpr __device__ int keys(int k) { return IT == 2 ? k / 2 : k < 3 || k == 9 ? 0 : k < 6 ? 1 : k < 8 ? 2 : 3; }
    static constexpr __device__ int wave(int k, int nw) { return IT == 4 && nw == 4 ? (k == 9 ? 3 : keys(k)) : k % nw; }
    static __device__ __forceinline__ void put(__bf16 *sm, int it, int jt, f4 v, int lane)
    {
        float x[4] = {v[0], v[1], v[2], v[3]};
        uint32_t p[HELD][2];
        split_pairs<HELD, 2>(x, p);
        const int wide = half(it, jt / 2) ? 4 : 8;
#pragma unroll
        for (int k = 0; k < HELD; ++k) *(u2 *)(sm + first(it, jt / 2) + (k * 64 + lane) * wide + 4 * (jt & 1)) = (u2){p[k][0], p[k][1]};
    }
    // acc + v * the scores of queries 16 it.. and keys 32 ks..
    template <int n> static __device__ __forceinline__ f4 product(f4 acc, const Op<n> &v, const __bf16 *sm, int it, int ks, int lane)
    {
        const __bf16 *p = sm + first(it, ks) + lane * (half(it, ks) ? 4 : 8);
        Op<HELD> s;
#pragma unroll
        for (int k = 0; k < HELD; ++k) {
            if (half(it, ks)) s.p[k] = __builtin_shufflevector(*(const bf4 *)(p + k * 64 * 4), (bf4)(__bf16)0.0f, 0, 1, 2, 3, 4, 5, 6, 7);
            else s.p[k] = *(const bf8 *)(p + k * 64 * 8);
        }
        return mma(acc, v, s);
    }
};

// Sums over a row of sixteen lanes, and over the four rows of a wave.
template <int CTRL> __device__ __forceinline__ float moved(float v)
{
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float sum16(float v)  // in every lane
{
    v += moved<0x128>(v);  // rotated by 8, 4, 2, 1
    v += moved<0x124>(v);
    v += moved<0x122>(v);
    return v + moved<0x121>(v);
}
__device__ __forceinline__ float prefix16(float v)
{
    v += moved<0x111>(v);
    v += moved<0x112>(v);
    v += moved<0x114>(v);
    return v + moved<0x118>(v);
}
__device__ __forceinline__ float suffix16(float v)
{
    v += moved<0x101>(v);
    v += moved<0x102>(v);
    v += moved<0x104>(v);
    return v + moved<0x108>(v);
}
__device__ __forceinline__ float sum_rows(float v)
{
    // the two operands of a swap have to be two registers, or the compiler takes its two results for one
    uint32_t x = __builtin_bit_cast(uint32_t, v), y = x;
    asm("" : "+v"(y));
    const auto a = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    x = __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, (uint32_t)a[0]) + __builtin_bit_cast(float, (uint32_t)a[1]));
    y = x;
    asm("" : "+v"(y));
    const auto b = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    return __builtin_bit_cast(float, (uint32_t)b[0]) + __builtin_bit_cast(float, (uint32_t)b[1]);
}

__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

}  // namespace semicrf_enc

#endif
