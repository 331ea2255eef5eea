// Token embedding with scaling, and the gradient of its table.
//
//   out[b,t,:] = scale * table[token[b,t],:]           grad_table[v,:] = scale * sum over positions that hold v of g[b,t,:]
//
// The gradient has no atomics: positions are sorted by token (stable radix sort, 8 bits a pass), and rows are added up in that
// order, in 32 bits.  Texts are skewed, so the sorted positions are cut into chunks of equal length instead of one piece of work
// for each token: a chunk writes the tokens that lie in it whole, and leaves a partial row where one enters from the chunk
// before or goes on in the next; those are joined in chunk order.  Zeros for tokens that do not occur are written while the
// positions are sorted, which keeps few workgroups busy.  Bound by g read once and the table written once; for few tokens by the
// launches: the sort's one, or two to three a pass, and two.
// Measured, bfloat16: 4 x 100 000 tokens, table 4101 x 512, forwards 72 us (410 MB written, 5.7 TB/s), gradient 130 us, of which 80
// add up rows (5.1 TB/s); 64 x 256 tokens, table 32000 x 512, gradient 40 us (65 MB of it zeros and sums).
#include "encoder.h"

namespace semicrf_enc {

constexpr int RADIX = 256;

struct EmbedArgs {
    const int32_t *tokens, *lengths;
    const void *table, *g;
    float scale;
    int B, T, V, D, lanes;  // lanes of a row in k_embed_fwd, as a power of two
    void *out;
    float *grad;
    int n, tiles, chunk, chunks, fills;  // fills: launches that share the zeros
    uint32_t *key[2], *pos[2], *count, *digit;
    float *part;  // [chunks][2][D]
};

// A row is 16 bytes a lane over a power of two of lanes (some idle where a row is none), four rows to a lane at once; a workgroup
// stays within one sequence, so that no position is divided by anything.
constexpr int ROWS = 4;
template <class T> __global__ __launch_bounds__(256) void k_embed_fwd(EmbedArgs a)
{
    constexpr int E = PER16<T>;
    typedef T X __attribute__((ext_vector_type(E)));
    const int side = 256 >> a.lanes, tiles = (a.T + ROWS * side - 1) / (ROWS * side);  // rows side by side in a workgroup
    const int b = blockIdx.x / tiles, t0 = blockIdx.x % tiles * (ROWS * side) + (threadIdx.x >> a.lanes);
    const int L = length_of(a.lengths, b, a.T), first = (threadIdx.x & ((1 << a.lanes) - 1)) * E;
    int32_t v[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
        const int t = t0 + k * side;
        v[k] = t < L ? a.tokens[(int64_t)b * a.T + t] : -1;
    }
    for (int col = first; col < a.D; col += E << a.lanes) {
        X x[ROWS];
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            x[k] = (X)(T)0.0f;
            if (v[k] >= 0 && v[k] < a.V) x[k] = *(const X *)((const T *)a.table + (int64_t)v[k] * a.D + col);
        }
#pragma unroll
        for (int k = 0; k < ROWS; ++k) {
            X o;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = (T)((float)x[k][e] * (v[k] >= 0 && v[k] < a.V ? a.scale : 0.0f));
            if (t0 + k * side < a.T) __builtin_nontemporal_store(o, (X *)((T *)a.out + ((int64_t)b * a.T + t0 + k * side) * a.D + col));
        }
    }
}

// The key of position i: its token, or V where it holds none (sorted to the end, never added).
__device__ __forceinline__ uint32_t key_of(const EmbedArgs &a, int i)
{
    const int b = i / a.T, t = i % a.T;
    const int32_t v = t < length_of(a.lengths, b, a.T) ? a.tokens[i] : -1;
    return v >= 0 && v < a.V ? (uint32_t)v : (uint32_t)a.V;
}

// The workgroups of a sorting launch beyond its tiles clear a share of the gradient.
constexpr int CLEAR = 512;
__device__ __forceinline__ bool clear_share(const EmbedArgs &a, int launch)
{
    if ((int)blockIdx.x < a.tiles) return false;
    const int64_t all = (int64_t)a.V * a.D / 4, from = all * launch / a.fills, to = all * (launch + 1) / a.fills;
    for (int64_t k = from + (int64_t)(blockIdx.x - a.tiles) * 256 + threadIdx.x; k < to; k += CLEAR * 256) *(f4 *)(a.grad + 4 * k) = (f4)0.0f;
    return true;
}

// Where the launch that puts positions in their places adds up the tiles' counts by itself: count[tile][digit] then, count[digit][tile]
// where k_sort_offsets does.  Up to 64 tiles that saves a launch a pass: 16384 positions of 250 tokens, 256 columns, take 18 us
// instead of 21, 32000 positions (63 tiles) as long with as without.
constexpr int FEW_TILES = 64;

// How often each digit occurs in each tile of 256 * ROUNDS positions.
template <int ROUNDS> __global__ __launch_bounds__(256) void k_sort_count(EmbedArgs a, int shift)
{
    __shared__ uint32_t c[RADIX];
    if (clear_share(a, shift / 4)) return;
    c[threadIdx.x] = 0;
    __syncthreads();
    const int first = blockIdx.x * 256 * ROUNDS + threadIdx.x;
    uint32_t key[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k)
        if (first + 256 * k < a.n) key[k] = shift ? a.key[(shift / 8) & 1][first + 256 * k] : key_of(a, first + 256 * k);
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k)
        if (first + 256 * k < a.n) atomicAdd(&c[(key[k] >> shift) % RADIX], 1u);
    __syncthreads();
    a.count[a.tiles <= FEW_TILES ? blockIdx.x * RADIX + threadIdx.x : threadIdx.x * a.tiles + blockIdx.x] = c[threadIdx.x];
}

// Prefix sum of a wave's values, exclusive; `all` is their sum.
__device__ __forceinline__ uint32_t before_lane(uint32_t v, uint32_t &all)
{
    uint32_t run = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(run, d);
        if ((int)(threadIdx.x & 63) >= d) run += o;
    }
    all = __shfl(run, 63);
    return run - v;
}

// For each digit, what earlier tiles hold of it, and how often it occurs in all.  One wave to a digit.
__global__ __launch_bounds__(64) void k_sort_offsets(EmbedArgs a)
{
    uint32_t base = 0, all;
    for (int k = threadIdx.x; k - (int)threadIdx.x < a.tiles; k += 64) {
        uint32_t *c = a.count + (size_t)blockIdx.x * a.tiles + k;
        const uint32_t v = k < a.tiles ? *c : 0, at = base + before_lane(v, all);
        if (k < a.tiles) *c = at;
        base += all;
    }
    if (threadIdx.x == 0) a.digit[blockIdx.x] = base;
}

// Lanes of the wave that hold the same digit as this one, of those that are `in`.
__device__ __forceinline__ uint64_t same_digit(uint32_t d, bool in)
{
    uint64_t same = __ballot(in);
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
        const uint64_t set = __ballot((d >> bit) & 1);
        same &= (d >> bit) & 1 ? set : ~set;
    }
    return same;
}

// Puts a tile's positions in their places.  A wave takes 64 positions at a time, in order; a position's place among equal digits
// is what earlier tiles, waves, rounds and lower lanes hold, so equal keys keep their order.
template <int ROUNDS> __global__ __launch_bounds__(256) void k_sort_scatter(EmbedArgs a, int shift)
{
    __shared__ uint32_t c[4][RADIX], wave[4];
    if (clear_share(a, shift / 4 + 1)) return;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64, pass = shift / 8;
    for (int k = 0; k < 4; ++k) c[k][threadIdx.x] = 0;
    uint32_t all, earlier = 0, here = 0;  // of the digit `threadIdx.x`: in earlier tiles, in all
    if (a.tiles <= FEW_TILES) {
#pragma unroll 8
        for (int k = 0; k < a.tiles; ++k) {
            const uint32_t n = a.count[k * RADIX + threadIdx.x];
            here += n;
            earlier += k < (int)blockIdx.x ? n : 0;
        }
    } else {
        earlier = a.count[threadIdx.x * a.tiles + blockIdx.x], here = a.digit[threadIdx.x];
    }
    uint32_t base = before_lane(here, all);
    if (lane == 63) wave[w] = all;
    const int first = blockIdx.x * 256 * ROUNDS + w * 64 * ROUNDS + lane;
    uint32_t key[ROUNDS], pos[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int i = first + 64 * k;
        key[k] = i >= a.n ? 0 : pass ? a.key[pass & 1][i] : key_of(a, i);
        pos[k] = i >= a.n ? 0 : pass ? a.pos[pass & 1][i] : (uint32_t)i;
    }
    __syncthreads();
    for (int k = 0; k < w; ++k) base += wave[k];
    base += earlier;
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const bool in = first + 64 * k < a.n;
        const uint32_t d = (key[k] >> shift) % RADIX;
        const uint64_t same = same_digit(d, in);
        const uint32_t below = __popcll(same & ((1ull << lane) - 1));
        uint32_t before = 0;
        if (in) before = c[w][d];
        rank[k] = before + below;
        __builtin_amdgcn_wave_barrier();
        if (in && below == 0) c[w][d] = before + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    for (int k = 0; k < 4; ++k) {
        const uint32_t n = c[k][threadIdx.x];
        c[k][threadIdx.x] = base;
        base += n;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k)
        if (first + 64 * k < a.n) {
            const uint32_t to = c[w][(key[k] >> shift) % RADIX] + rank[k];
            a.key[(pass + 1) & 1][to] = key[k];
            a.pos[(pass + 1) & 1][to] = pos[k];
        }
}

// The whole sort in one launch, for as many positions as a workgroup holds: a position and its token are one word, positions below,
// R of them to a thread, and change places through LDS.  The other workgroups clear the gradient meanwhile.
constexpr int WIDE = 1024, MOST_AT_ONCE = 4 * WIDE;
template <int R> __global__ __launch_bounds__(WIDE) void k_sort_whole(EmbedArgs a, int bits, int passes)
{
    __shared__ uint32_t words[WIDE * R], c[WIDE / 64][RADIX], wave[RADIX / 64];
    const int tid = threadIdx.x, lane = tid % 64, w = tid / 64, first = w * 64 * R + lane;
    if (blockIdx.x > 0) {
        const int64_t all = (int64_t)a.V * a.D / 4;
        for (int64_t k = (int64_t)(blockIdx.x - 1) * WIDE + tid; k < all; k += (int64_t)(gridDim.x - 1) * WIDE) *(f4 *)(a.grad + 4 * k) = (f4)0.0f;
        return;
    }
    uint32_t word[R], rank[R];
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int i = first + 64 * k;
        word[k] = i < a.n ? key_of(a, i) << bits | (uint32_t)i : ~0u;  // places without a position stay the last
    }
    for (int shift = bits; passes > 0; --passes, shift += 8) {
        for (int k = tid; k < (WIDE / 64) * RADIX; k += WIDE) c[k / RADIX][k % RADIX] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < R; ++k) {
            const uint32_t d = (word[k] >> shift) % RADIX;
            const uint64_t same = same_digit(d, true);
            const uint32_t below = __popcll(same & ((1ull << lane) - 1)), before = c[w][d];
            rank[k] = before + below;
            __builtin_amdgcn_wave_barrier();
            if (below == 0) c[w][d] = before + (uint32_t)__popcll(same);
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t held[WIDE / 64], base = 0;
        if (tid < RADIX) {
            uint32_t sum = 0, all;
#pragma unroll
            for (int k = 0; k < WIDE / 64; ++k) {
                held[k] = sum;
                sum += c[k][tid];
            }
            base = before_lane(sum, all);
            if (lane == 0) wave[w] = all;
        }
        __syncthreads();
        if (tid < RADIX) {
            for (int k = 0; k < w; ++k) base += wave[k];
#pragma unroll
            for (int k = 0; k < WIDE / 64; ++k) c[k][tid] = base + held[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < R; ++k) words[c[w][(word[k] >> shift) % RADIX] + rank[k]] = word[k];
        __syncthreads();
#pragma unroll
        for (int k = 0; k < R; ++k) word[k] = words[first + 64 * k];
    }
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int i = first + 64 * k;
        if (i < a.n) a.key[0][i] = word[k] >> bits, a.pos[0][i] = word[k] & ((1u << bits) - 1);
    }
}

// One wave adds up one chunk of the sorted positions over 64 lanes of columns (80 us for 400 000 rows of 1 KB, 5.1 TB/s).  Keys and places are a lane's each, read once and
// handed round by lane, so that branches on them are the wave's and the rows of several positions are on their way at once.
// PAST: rows are read past the caches.
template <class T, bool PAST> __global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs a, const uint32_t *key, const uint32_t *pos)
{
    constexpr int E = PER16<T>, AHEAD = 8;
    typedef T X __attribute__((ext_vector_type(E)));
    const int slices = (a.D + 64 * E - 1) / (64 * E), lane = threadIdx.x % 64;
    const int id = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + threadIdx.x / 64), chunk = id / slices;
    const int col = (id % slices * 64 + lane) * E, first = chunk * a.chunk;
    if (chunk >= a.chunks) return;
    const int all = first + a.chunk < a.n ? a.chunk : a.n - first;
    const uint32_t mine = lane < all ? key[first + lane] : ~0u, at = lane < all ? pos[first + lane] : 0;
    // positions without a token are the last, and their rows are not read
    const int n = __popcll(__ballot(mine < (uint32_t)a.V));
    if (n == 0) return;
    const uint32_t last = first + n < a.n ? key[first + n] : ~0u;  // the key behind them
    uint32_t run = first > 0 ? key[first - 1] : ~0u;
    const bool here = col < a.D;
    const T *g = (const T *)a.g + (here ? col : 0);
    float s[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0.0f;
    bool entered = run == (uint32_t)__builtin_amdgcn_readlane((int)mine, 0);
    X next[AHEAD];
    auto fetch = [&](int i0) {
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k < n ? i0 + k : n - 1;
            const X *row = (const X *)(g + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)at, i) * a.D);
            next[k] = PAST ? __builtin_nontemporal_load(row) : *row;
        }
    };
    fetch(0);
    for (int i0 = 0; i0 < n; i0 += AHEAD) {
        X r[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) r[k] = next[k];
        if (i0 + AHEAD < n) fetch(i0 + AHEAD);
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k;
            if (i >= n) break;
            const uint32_t v = (uint32_t)__builtin_amdgcn_readlane((int)mine, i);
#pragma unroll
            for (int e = 0; e < E; ++e) s[e] += (float)r[k][e];
            const bool ends = (i + 1 < n ? (uint32_t)__builtin_amdgcn_readlane((int)mine, i + 1) : last) != v;
            if (ends || i + 1 == n) {
                float *to = entered ? a.part + ((int64_t)chunk * 2) * a.D + col
                                    : ends ? a.grad + (int64_t)v * a.D + col : a.part + ((int64_t)chunk * 2 + 1) * a.D + col;
                const float f = entered || !ends ? 1.0f : a.scale;
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] *= f;
                if (here) {
#pragma unroll
                    for (int q = 0; q < E; q += 4) *(f4 *)(to + q) = (f4){s[q], s[q + 1], s[q + 2], s[q + 3]};
                }
#pragma unroll
                for (int e = 0; e < E; ++e) s[e] = 0.0f;
                entered = false;
            }
        }
    }
}

// Tokens that no chunk held whole: the chunk that such a token's positions end in adds up its parts, in chunk order.
__global__ __launch_bounds__(256) void k_embed_join(EmbedArgs a, const uint32_t *key)
{
    const int lane = threadIdx.x % 64, chunk = blockIdx.x * 4 + threadIdx.x / 64, first = chunk * a.chunk;
    if (chunk < 1 || chunk >= a.chunks) return;
    const uint32_t v = key[first];
    const int end = first + a.chunk < a.n ? first + a.chunk : a.n;
    if (v >= (uint32_t)a.V || key[first - 1] != v) return;
    if (key[end - 1] == v && end < a.n && key[end] == v) return;  // goes on in the next chunk
    // the token's first position, 64 probes at a time: lo is at or before it, hi behind the last that may be
    int lo = 0, hi = first;
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, at = lo + lane * step;
        const int less = __popcll(__ballot(at < hi && key[at] < v));  // the first `less` probes lie before it
        if (less == 0) {
            hi = lo;
        } else {
            const int up = lo + less * step;
            lo += (less - 1) * step + 1;
            hi = up < hi ? up : hi;
        }
    }
    const int c0 = lo / a.chunk;
    const int col = (int)blockIdx.y * 256 + 4 * lane;
    if (col < a.D) {
        const float *part = a.part + col;
        typedef double d4 __attribute__((ext_vector_type(4)));
        d4 sum = __builtin_convertvector(*(const f4 *)(part + ((int64_t)c0 * 2 + 1) * a.D), d4);
        int c = c0 + 1;
        for (; c + 16 <= chunk + 1; c += 16) {
            f4 p[16];
#pragma unroll
            for (int q = 0; q < 16; ++q) p[q] = *(const f4 *)(part + (int64_t)(c + q) * 2 * a.D);
#pragma unroll
            for (int q = 0; q < 16; ++q) sum += __builtin_convertvector(p[q], d4);
        }
        for (; c <= chunk; ++c) sum += __builtin_convertvector(*(const f4 *)(part + (int64_t)c * 2 * a.D), d4);
        *(f4 *)(a.grad + (int64_t)v * a.D + col) = __builtin_convertvector(sum * (double)a.scale, f4);
    }
}

struct EmbedPlan {
    int n, tiles, chunk, chunks, passes, bits;  // bits: of a position, where one workgroup sorts all (0: it does not)
    bool large;
    size_t key[2], pos[2], count, digit, part, total;
};

int embed_plan(int B, int T, int V, int D, EmbedPlan *p)
{
    if (B < 1 || T < 1 || V < 1 || D < 1) return SEMICRF_EINVAL;
    if (D % 8 || (double)B * T > 1e9 || V > (1 << 24) || (double)V * D > 1e11) return SEMICRF_EUNSUPPORTED;
    p->n = B * T;
    // Tiles of 2048 positions, or of 512 where few would leave most of the chip idle (64 x 256 tokens: 9 us a pass, 16 with 2048);
    // chunks of 64, or of 16 for the same reason.
    p->large = p->n > 131072;
    p->tiles = (p->n + (p->large ? 2047 : 511)) / (p->large ? 2048 : 512);
    p->chunk = p->n > 262144 ? 64 : 16;
    p->chunks = (p->n + p->chunk - 1) / p->chunk;
    p->passes = 0;
    for (int64_t left = V; left > 0; left >>= 8) ++p->passes;
    // Up to 4096 positions are sorted in one launch by one workgroup, if a position and its token go into 32 bits: 1000 positions of
    // 300 tokens, 512 columns, take 15 us instead of 22, 4000 take 19 instead of 22.  16384 would take 36 instead of 18: one
    // workgroup's ranks take 16 us a pass.
    int bits = 0;
    while (p->n > 1 << bits) ++bits;
    if (bits == 0) bits = 1;
    p->bits = p->n <= MOST_AT_ONCE && (int64_t)V << bits < (int64_t)1 << 32 ? bits : 0;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    for (int k = 0; k < 2; ++k) p->key[k] = take((size_t)p->n * 4), p->pos[k] = take((size_t)p->n * 4);
    p->count = take((size_t)RADIX * p->tiles * 4);
    p->digit = take((size_t)RADIX * 4);
    p->part = take((size_t)p->chunks * 2 * D * 4);
    p->total = at;
    return SEMICRF_OK;
}

template <class T> void embed_sum(const EmbedArgs &a, const uint32_t *key, const uint32_t *pos, hipStream_t st)
{
    const int64_t waves = (int64_t)a.chunks * ((a.D + 64 * PER16<T> - 1) / (64 * PER16<T>));
    // Rows that the last-level cache (256 MB) hardly holds are read past it: 400 000 rows of 1 KB, forwards and gradient 203 us instead
    // of 232; 16 384 rows 46 us, and 48 past it.
    const bool past = (double)a.n * a.D * sizeof(T) > 128e6;
    const dim3 g((unsigned)((waves + 3) / 4)), t(256);
    if (past) hipLaunchKernelGGL((k_embed_sum<T, true>), g, t, 0, st, a, key, pos);
    else hipLaunchKernelGGL((k_embed_sum<T, false>), g, t, 0, st, a, key, pos);
}

}  // namespace semicrf_enc

using namespace semicrf_enc;

extern "C" {

int semicrf_embed_fwd(const int32_t *tokens, const int32_t *lengths, const void *table, float scale, int B, int T, int V,
                      int D, unsigned flags, void *out, void *stream)
{
    EmbedPlan p = {};
    if (int rc = embed_plan(B, T, V, D, &p)) return rc;
    const int type = act_type(flags);
    if (type < 0 || !tokens || !rows_ok(table, D, D, type) || !rows_ok(out, D, D, type)) return SEMICRF_EINVAL;
    EmbedArgs a = {};
    a.tokens = tokens; a.lengths = lengths; a.table = table; a.scale = scale;
    a.B = B; a.T = T; a.V = V; a.D = D; a.out = out; a.n = p.n;
    while (a.lanes < 8 && (16 / act_bytes(type)) << a.lanes < D) ++a.lanes;
    const int rows = ROWS * (256 >> a.lanes);
    if ((double)B * ((T + rows - 1) / rows) > 2e9) return SEMICRF_EUNSUPPORTED;
    const dim3 g((unsigned)B * ((T + rows - 1) / rows)), t(256);
    const hipStream_t st = (hipStream_t)stream;
    if (type == ACT_BF16) hipLaunchKernelGGL((k_embed_fwd<__bf16>), g, t, 0, st, a);
    else if (type == ACT_F16) hipLaunchKernelGGL((k_embed_fwd<_Float16>), g, t, 0, st, a);
    else hipLaunchKernelGGL((k_embed_fwd<float>), g, t, 0, st, a);
    return launched();
}

int semicrf_embed_bwd_workspace_bytes(int B, int T, int V, int D, size_t *bytes)
{
    if (!bytes) return SEMICRF_EINVAL;
    EmbedPlan p = {};
    const int rc = embed_plan(B, T, V, D, &p);
    if (rc == SEMICRF_OK) *bytes = p.total;
    return rc;
}

int semicrf_embed_bwd(const int32_t *tokens, const int32_t *lengths, const void *grad_out, float scale, int B, int T, int V,
                      int D, unsigned flags, void *workspace, size_t workspace_bytes, float *grad_table, void *stream)
{
    EmbedPlan p = {};
    if (int rc = embed_plan(B, T, V, D, &p)) return rc;
    const int type = act_type(flags);
    if ((double)p.chunks * (D / 256 + 1) > 2e9 || D > 65535 * 256) return SEMICRF_EUNSUPPORTED;
    if (type < 0 || !tokens || !rows_ok(grad_out, D, D, type) || !grad_table || ((uintptr_t)grad_table & 15))
        return SEMICRF_EINVAL;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < p.total) return SEMICRF_EWORKSPACE;
    EmbedArgs a = {};
    a.tokens = tokens; a.lengths = lengths; a.g = grad_out; a.scale = scale;
    a.B = B; a.T = T; a.V = V; a.D = D; a.grad = grad_table;
    a.n = p.n; a.tiles = p.tiles; a.chunk = p.chunk; a.chunks = p.chunks;
    char *w = (char *)workspace;
    for (int k = 0; k < 2; ++k) a.key[k] = (uint32_t *)(w + p.key[k]), a.pos[k] = (uint32_t *)(w + p.pos[k]);
    a.count = (uint32_t *)(w + p.count);
    a.digit = (uint32_t *)(w + p.digit);
    a.fills = 2 * p.passes;
    a.part = (float *)(w + p.part);
    const hipStream_t st = (hipStream_t)stream;
    if (p.bits) {
        const dim3 g(256), t(WIDE);
        if (p.n <= WIDE) hipLaunchKernelGGL((k_sort_whole<1>), g, t, 0, st, a, p.bits, p.passes);
        else hipLaunchKernelGGL((k_sort_whole<4>), g, t, 0, st, a, p.bits, p.passes);
    } else {
        for (int pass = 0; pass < p.passes; ++pass) {
            if (p.large) hipLaunchKernelGGL((k_sort_count<8>), dim3(p.tiles + CLEAR), dim3(256), 0, st, a, 8 * pass);
            else hipLaunchKernelGGL((k_sort_count<2>), dim3(p.tiles + CLEAR), dim3(256), 0, st, a, 8 * pass);
            if (p.tiles > FEW_TILES) hipLaunchKernelGGL(k_sort_offsets, dim3(RADIX), dim3(64), 0, st, a);
            if (p.large) hipLaunchKernelGGL((k_sort_scatter<8>), dim3(p.tiles + CLEAR), dim3(256), 0, st, a, 8 * pass);
            else hipLaunchKernelGGL((k_sort_scatter<2>), dim3(p.tiles + CLEAR), dim3(256), 0, st, a, 8 * pass);
        }
    }
    const int last = p.bits ? 0 : p.passes & 1;
    const uint32_t *key = a.key[last], *pos = a.pos[last];
    if (type == ACT_BF16) embed_sum<__bf16>(a, key, pos, st);
    else if (type == ACT_F16) embed_sum<_Float16>(a, key, pos, st);
    else embed_sum<float>(a, key, pos, st);
    hipLaunchKernelGGL(k_embed_join, dim3((p.chunks + 3) / 4, (D + 255) / 256), dim3(256), 0, st, a, key);
    return launched();
}

}  // extern "C"
