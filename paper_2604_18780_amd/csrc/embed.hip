// Token embedding with scaling, and the gradient of its table.
//
//   out[b,t,:] = scale * table[token[b,t],:]           grad_table[v,:] = scale * sum over positions that hold v of g[b,t,:]
//
// The gradient has no atomics: positions are sorted by token (stable radix sort, 8 bits a pass), and rows are added up in that
// order, in 32 bits.  Texts are skewed, so the sorted positions are cut into chunks of equal length instead of one piece of work
// for each token: a chunk writes the tokens that lie in it whole, and leaves a partial row where one enters from the chunk
// before or goes on in the next; those are joined in chunk order.  Bound by g read once and the table written once.
#include "encoder.h"

namespace semicrf_enc {

constexpr int TILE = 2048;     // positions a workgroup sorts at once
constexpr int RADIX = 256;

struct EmbedArgs {
    const int32_t *tokens, *lengths;
    const void *table, *g;
    float scale;
    int B, T, V, D;
    void *out;
    float *grad;
    int n, tiles, chunk, chunks;
    uint32_t *key[2], *pos[2], *count, *start;
    float *part;  // [chunks][2][D]
};

template <class T> __global__ __launch_bounds__(256) void k_embed_fwd(EmbedArgs a)
{
    constexpr int E = PER16<T>;
    const int per = a.D / E;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (int64_t)a.n * per) return;
    const int64_t row = at / per;
    const int col = (int)(at % per) * E, b = (int)(row / a.T), t = (int)(row % a.T);
    const int32_t v = a.tokens[row];
    float o[E];
    if (t < length_of(a.lengths, b, a.T) && v >= 0 && v < a.V) {
        load_n<T, E>((const T *)a.table + (int64_t)v * a.D + col, o);
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] *= a.scale;
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] = 0.0f;
    }
    store_n<T, E>((T *)a.out + row * a.D + col, o);
}

// The key of position i: its token, or V where it holds none (sorted to the end, never added).
__device__ __forceinline__ uint32_t key_of(const EmbedArgs &a, int i)
{
    const int b = i / a.T, t = i % a.T;
    const int32_t v = a.tokens[i];
    return t < length_of(a.lengths, b, a.T) && v >= 0 && v < a.V ? (uint32_t)v : (uint32_t)a.V;
}

// How often each digit occurs in each tile: count[digit][tile].
__global__ __launch_bounds__(256) void k_sort_count(EmbedArgs a, int shift)
{
    __shared__ uint32_t c[RADIX];
    c[threadIdx.x] = 0;
    __syncthreads();
    const int first = blockIdx.x * TILE;
    for (int k = threadIdx.x; k < TILE && first + k < a.n; k += 256) {
        const uint32_t key = shift ? a.key[(shift / 8) & 1][first + k] : key_of(a, first + k);
        atomicAdd(&c[(key >> shift) % RADIX], 1u);
    }
    __syncthreads();
    a.count[threadIdx.x * a.tiles + blockIdx.x] = c[threadIdx.x];
}

// Exclusive prefix sum over the counts, digits outside, tiles inside.  One workgroup.
__global__ __launch_bounds__(1024) void k_sort_offsets(EmbedArgs a)
{
    __shared__ uint32_t wave[16];
    const int n = RADIX * a.tiles, per = (n + 1023) / 1024, first = threadIdx.x * per;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    uint32_t sum = 0;
    for (int k = 0; k < per; ++k)
        if (first + k < n) sum += a.count[first + k];
    uint32_t run = sum;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(run, d);
        if (lane >= d) run += o;
    }
    if (lane == 63) wave[w] = run;
    __syncthreads();
    uint32_t base = run - sum;
    for (int k = 0; k < w; ++k) base += wave[k];
    for (int k = 0; k < per; ++k)
        if (first + k < n) {
            const uint32_t c = a.count[first + k];
            a.count[first + k] = base;
            base += c;
        }
}

// Puts a tile's positions in their places.  A wave takes 64 positions at a time, in order; its place among equal digits is
// what earlier waves, earlier rounds and lower lanes hold, so equal keys keep their order.
__global__ __launch_bounds__(256) void k_sort_scatter(EmbedArgs a, int shift)
{
    constexpr int ROUNDS = TILE / 256;
    __shared__ uint32_t c[4][RADIX];
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64, pass = shift / 8;
    for (int k = 0; k < 4; ++k) c[k][threadIdx.x] = 0;
    __syncthreads();
    const int first = blockIdx.x * TILE + w * (TILE / 4);
    uint32_t key[ROUNDS], rank[ROUNDS];
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int i = first + 64 * k + lane;
        const bool in = i < a.n;
        key[k] = !in ? 0 : pass ? a.key[pass & 1][i] : key_of(a, i);
        const uint32_t d = (key[k] >> shift) % RADIX;
        uint64_t same = __ballot(in);
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t set = __ballot((d >> bit) & 1);
            same &= (d >> bit) & 1 ? set : ~set;
        }
        const uint32_t below = __popcll(same & ((1ull << lane) - 1));
        uint32_t before = 0;
        if (in) before = c[w][d];
        rank[k] = before + below;
        __builtin_amdgcn_wave_barrier();
        if (in && below == 0) c[w][d] = before + (uint32_t)__popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    {
        uint32_t base = a.count[threadIdx.x * a.tiles + blockIdx.x];
        for (int k = 0; k < 4; ++k) {
            const uint32_t n = c[k][threadIdx.x];
            c[k][threadIdx.x] = base;
            base += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ROUNDS; ++k) {
        const int i = first + 64 * k + lane;
        if (i < a.n) {
            const uint32_t to = c[w][(key[k] >> shift) % RADIX] + rank[k];
            a.key[(pass + 1) & 1][to] = key[k];
            a.pos[(pass + 1) & 1][to] = pass ? a.pos[pass & 1][i] : (uint32_t)i;
        }
    }
}

// First sorted place of each token, by bisection; place V is where the positions without a token begin.
__global__ __launch_bounds__(256) void k_embed_starts(EmbedArgs a, const uint32_t *key)
{
    const int v = blockIdx.x * 256 + threadIdx.x;
    if (v > a.V) return;
    int lo = 0, hi = a.n;
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (key[mid] < (uint32_t)v) lo = mid + 1;
        else hi = mid;
    }
    a.start[v] = lo;
}

// One wave adds up one chunk of the sorted positions over 64 lanes of columns.
template <class T> __global__ __launch_bounds__(256) void k_embed_sum(EmbedArgs a, const uint32_t *key, const uint32_t *pos)
{
    constexpr int E = PER16<T>;
    const int slices = (a.D + 64 * E - 1) / (64 * E);
    const int id = blockIdx.x * 4 + threadIdx.x / 64, chunk = id / slices;
    const int col = (id % slices * 64 + threadIdx.x % 64) * E;
    const int end = (int)a.start[a.V];
    const int first = chunk * a.chunk;
    if (chunk >= a.chunks || first >= end || col >= a.D) return;
    const int last = first + a.chunk < end ? first + a.chunk : end;
    const T *g = (const T *)a.g + col;
    float s[E];
#pragma unroll
    for (int e = 0; e < E; ++e) s[e] = 0.0f;
    bool entered = first > 0 && key[first - 1] == key[first];
    for (int i = first; i < last; ++i) {
        const uint32_t v = key[i];
        float r[E];
        load_n<T, E>(g + (int64_t)pos[i] * a.D, r);
#pragma unroll
        for (int e = 0; e < E; ++e) s[e] += r[e];
        const bool ends = i + 1 == end || key[i + 1] != v;
        if (ends || i + 1 == last) {
            float *to = entered ? a.part + ((int64_t)chunk * 2) * a.D + col
                                : ends ? a.grad + (int64_t)v * a.D + col : a.part + ((int64_t)chunk * 2 + 1) * a.D + col;
            const float f = entered || !ends ? 1.0f : a.scale;
#pragma unroll
            for (int e = 0; e < E; ++e) to[e] = f * s[e], s[e] = 0.0f;
            entered = false;
        }
    }
}

// Tokens that no chunk held whole: zeros where there are none, else the parts in chunk order.  256 threads to a token and 256
// columns.
__global__ __launch_bounds__(256) void k_embed_join(EmbedArgs a)
{
    const int slices = (a.D + 255) / 256, v = blockIdx.x / slices, col = blockIdx.x % slices * 256 + threadIdx.x;
    if (col >= a.D) return;
    const int s = (int)a.start[v], e = (int)a.start[v + 1];
    float *to = a.grad + (int64_t)v * a.D + col;
    if (s == e) {
        *to = 0.0f;
        return;
    }
    const int c0 = s / a.chunk, c1 = (e - 1) / a.chunk;
    if (c0 == c1) return;
    const float *part = a.part + col;
    double sum = part[((int64_t)c0 * 2 + 1) * a.D];
    for (int c = c0 + 1; c <= c1; ++c) sum += part[(int64_t)c * 2 * a.D];
    *to = (float)(a.scale * sum);
}

struct EmbedPlan {
    int n, tiles, chunk, chunks, passes;
    size_t key[2], pos[2], count, start, part, total;
};

int embed_plan(int B, int T, int V, int D, EmbedPlan *p)
{
    if (B < 1 || T < 1 || V < 1 || D < 1) return SEMICRF_EINVAL;
    if (D % 8 || (double)B * T > 1e9 || V > (1 << 24) || (double)V * D > 1e11) return SEMICRF_EUNSUPPORTED;
    p->n = B * T;
    p->tiles = (p->n + TILE - 1) / TILE;
    p->chunk = p->n > 262144 ? 64 : 16;
    p->chunks = (p->n + p->chunk - 1) / p->chunk;
    p->passes = 0;
    for (int64_t left = V; left > 0; left >>= 8) ++p->passes;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t o = at;
        at += align256(bytes);
        return o;
    };
    for (int k = 0; k < 2; ++k) p->key[k] = take((size_t)p->n * 4), p->pos[k] = take((size_t)p->n * 4);
    p->count = take((size_t)RADIX * p->tiles * 4);
    p->start = take(((size_t)V + 1) * 4);
    p->part = take((size_t)p->chunks * 2 * D * 4);
    p->total = at;
    return SEMICRF_OK;
}

template <class T> void embed_sum(const EmbedArgs &a, const uint32_t *key, const uint32_t *pos, hipStream_t st)
{
    const int64_t waves = (int64_t)a.chunks * ((a.D + 64 * PER16<T> - 1) / (64 * PER16<T>));
    hipLaunchKernelGGL((k_embed_sum<T>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, st, a, key, pos);
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
    const int64_t items = (int64_t)p.n * (D / (16 / act_bytes(type)));
    if (items > (int64_t)0x7fffffff * 256) return SEMICRF_EUNSUPPORTED;
    const dim3 g((unsigned)((items + 255) / 256)), t(256);
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
    a.start = (uint32_t *)(w + p.start);
    a.part = (float *)(w + p.part);
    const hipStream_t st = (hipStream_t)stream;
    for (int pass = 0; pass < p.passes; ++pass) {
        hipLaunchKernelGGL(k_sort_count, dim3(p.tiles), dim3(256), 0, st, a, 8 * pass);
        hipLaunchKernelGGL(k_sort_offsets, dim3(1), dim3(1024), 0, st, a);
        hipLaunchKernelGGL(k_sort_scatter, dim3(p.tiles), dim3(256), 0, st, a, 8 * pass);
    }
    const uint32_t *key = a.key[p.passes & 1], *pos = a.pos[p.passes & 1];
    hipLaunchKernelGGL(k_embed_starts, dim3((V + 256) / 256), dim3(256), 0, st, a, key);
    if (type == ACT_BF16) embed_sum<__bf16>(a, key, pos, st);
    else if (type == ACT_F16) embed_sum<_Float16>(a, key, pos, st);
    else embed_sum<float>(a, key, pos, st);
    hipLaunchKernelGGL(k_embed_join, dim3((unsigned)((int64_t)V * ((D + 255) / 256))), dim3(256), 0, st, a);
    return launched();
}

}  // extern "C"
