// embedding.hip - the embedding of a language model beside its compressed gradient: lookup of rows by token, and the
// table's gradient, summed by token in a fixed order.
//
// Both are bound by memory.  The lookup is one gather.  The gradient is a sum over the tokens that name a row; adding row by
// row with atomics would give sums that depend on scheduling (and a queue at the row of a frequent token), so the tokens are
// sorted first, with their positions, by a stable radix sort: equal tokens then stand together in the order of their
// positions, a wavefront adds up the rows of its share of the sorted tokens in registers, and every row of the table is
// written by one wavefront.

#include <hip/hip_runtime.h>

#include <cstdint>

#include "elements.h"
#include "gravac.h"

namespace {

using namespace elements;

__device__ __forceinline__ int64_t token_at(const void* tokens, bool wide, int64_t i)
{
    return wide ? ((const int64_t*)tokens)[i] : (int64_t)((const int32_t*)tokens)[i];
}

// ---------------------------------------------------------------------------------------------------------------------
// lookup
// ---------------------------------------------------------------------------------------------------------------------

constexpr int64_t LOOKUP_GRID = 1 << 22;   // workgroups along the tokens at most (the global size has 32 bits)

struct LookupParams {
    const void* table;
    const void* tokens;
    void* out;
    int64_t vocab, table_stride, n, out_stride;
    int32_t dim;
    int32_t wide;    // tokens of 8 bytes
    int32_t lanes;   // lanes that share a row: a power of two up to 64
    float scale;
};

// out[t] = scale * table[tokens[t]]: the product in binary32, then one rounding to the output's type.  A group of `lanes`
// lanes takes K accesses of a row each, all in flight together; blockIdx.y walks along a row.
template <typename A, typename B, int K>
__global__ __launch_bounds__(256) void lookup_kernel(LookupParams p)
{
    constexpr int N = 16 / (A::SIZE > B::SIZE ? A::SIZE : B::SIZE);
    const int lane = threadIdx.x & (p.lanes - 1), groups = 256 / p.lanes;
    for (int64_t t = (int64_t)blockIdx.x * groups + threadIdx.x / p.lanes; t < p.n; t += (int64_t)gridDim.x * groups) {
        const int64_t token = token_at(p.tokens, p.wide, t);
        const bool inside = token >= 0 && token < p.vocab;
        const typename A::word* row = (const typename A::word*)p.table + (inside ? token : 0) * p.table_stride;
        typename B::word* to = (typename B::word*)p.out + t * p.out_stride;
        const int c0 = ((int)blockIdx.y * K * p.lanes + lane) * N;
        float x[K][N];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = c0 + k * p.lanes * N;
#pragma unroll
            for (int i = 0; i < N; ++i) x[k][i] = 0.0f;
            if (inside && c < p.dim) load_part<A, N>(row + c, p.dim - c, x[k]);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = c0 + k * p.lanes * N;
            if (c >= p.dim) continue;
            if (inside) {
#pragma unroll
                for (int i = 0; i < N; ++i) x[k][i] *= p.scale;
            }
            store_part<B, N>(to + c, p.dim - c, x[k]);
        }
    }
}

template <typename A, typename B>
void launch_lookup(LookupParams& p, hipStream_t stream)
{
    constexpr int N = 16 / (A::SIZE > B::SIZE ? A::SIZE : B::SIZE);
    const int64_t chunks = ((int64_t)p.dim + N - 1) / N;
    p.lanes = 4;
    while (p.lanes < 64 && p.lanes < chunks) p.lanes *= 2;
    const int64_t groups = 256 / p.lanes, rows = (p.n + groups - 1) / groups;
    const int64_t x = rows < LOOKUP_GRID ? rows : LOOKUP_GRID;
    // four accesses per lane once there are wavefronts enough to fill the card without them
    const int k = p.n * chunks >= (1 << 19) && chunks > p.lanes ? 4 : 1;
    const dim3 grid((uint32_t)x, (uint32_t)((chunks + (int64_t)p.lanes * k - 1) / ((int64_t)p.lanes * k)));
    if (k == 4) hipLaunchKernelGGL((lookup_kernel<A, B, 4>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((lookup_kernel<A, B, 1>), grid, dim3(256), 0, stream, p);
}

template <typename A>
void launch_lookup(LookupParams& p, int out_type, hipStream_t stream)
{
    if (out_type == GRAVAC_FLOAT32) launch_lookup<A, F32>(p, stream);
    else if (out_type == GRAVAC_BFLOAT16) launch_lookup<A, BF16>(p, stream);
    else launch_lookup<A, F16>(p, stream);
}

// ---------------------------------------------------------------------------------------------------------------------
// gradient: sort
// ---------------------------------------------------------------------------------------------------------------------

constexpr int SORT_T = 1024;                     // threads of a sorting workgroup
constexpr int SORT_W = SORT_T / 64;
constexpr int SORT_ROUNDS = 4;                   // tokens per thread in a tile
constexpr int SORT_TILE = SORT_T * SORT_ROUNDS;  // tokens of a tile
constexpr int MAX_BITS = 9;                      // bits of a digit at most: two passes for a vocabulary up to 2^18 - 1
constexpr int MIN_BITS = 4;
constexpr int BINS = 1 << MAX_BITS;
constexpr int SORT_GRID = 128;                   // sorting workgroups at most: each adds up all workgroups' counts
constexpr int FILL_GRID = 2048;                  // workgroups at most that clear the table beside the sort
constexpr int FEW = 128;                         // calls of at most this many tokens are not sorted

struct GradParams {
    const void* grad;
    const void* tokens;
    float* table;
    int64_t n, grad_stride, table_stride;
    int64_t vocab, padding;
    int32_t dim, wide;
    int32_t accumulate;
    float scale;
    uint2* pairs[2];       // (token or vocab, position): sorted, between two passes
    uint32_t* counts;      // [SORT_GRID][BINS]
    uint32_t* joins;       // [0]: number of shares whose last run goes on behind them, then their numbers
    float* head;           // [share][part_stride]: sums of a share's first run that began before it
    float* tail;           // ... of its last run that goes on behind it
    int64_t part_stride;
    int64_t per_wg;        // tokens per sorting workgroup
    int32_t sort_wgs, bits, share_log;
    uint32_t n_shares;
};

// The token at position i as a sort key: `vocab` for one that takes no part.
__device__ __forceinline__ uint32_t key_at(const GradParams& p, int64_t i)
{
    const int64_t t = token_at(p.tokens, p.wide, i);
    return t < 0 || t >= p.vocab || t == p.padding ? (uint32_t)p.vocab : (uint32_t)t;
}

// Clears the table: workgroup `wg` of `wgs`, T threads each.
template <int T>
__device__ void fill_table(const GradParams& p, int64_t wg, int64_t wgs)
{
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (p.table_stride == p.dim) {
        const int64_t n = p.vocab * p.dim;
        for (int64_t i = (wg * T + threadIdx.x) * 4; i < n; i += wgs * T * 4)
            store_part<F32, 4>((uint32_t*)p.table + i, n - i < 4 ? (int)(n - i) : 4, zero);
    } else {
        for (int64_t r = wg; r < p.vocab; r += wgs)
            for (int c = (int)threadIdx.x * 4; c < p.dim; c += T * 4)
                store_part<F32, 4>((uint32_t*)p.table + r * p.table_stride + c, p.dim - c, zero);
    }
}

// LDS of a sorting workgroup.
struct SortLds {
    uint32_t cnt[SORT_W][BINS];   // a wavefront's tokens per digit, then where its first one goes
    uint32_t base[BINS];          // where the workgroup's next token of a digit goes
    uint32_t wave[SORT_W];
};

// The exclusive sum of x over the workgroup's threads (all of them call it).
__device__ uint32_t exclusive_sum(uint32_t x, uint32_t* wave_sums)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t s = x;
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t o = __shfl_up(s, d, 64);
        if (lane >= d) s += o;
    }
    __syncthreads();
    if (lane == 63) wave_sums[w] = s;
    __syncthreads();
    for (int i = 0; i < w; ++i) s += wave_sums[i];
    return s - x;
}

// Places of a tile's tokens in the order of one digit, earlier tokens first.  A wavefront's tokens are consecutive, round by
// round; the lanes of a round that hold the same digit find each other with one ballot per bit.  On return at[r] is the
// place of the token of round r, and base has moved on by the tile's counts.
__device__ void place_tile(SortLds& s, int bits, const uint32_t (&digit)[SORT_ROUNDS], const bool (&have)[SORT_ROUNDS],
                           uint32_t (&at)[SORT_ROUNDS])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << bits;
    for (int i = threadIdx.x; i < SORT_W * bins; i += SORT_T) s.cnt[i >> bits][i & (bins - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SORT_ROUNDS; ++r) {
        uint64_t same = __ballot(have[r]);
        for (int b = 0; b < bits; ++b) {
            const bool one = (digit[r] >> b) & 1;
            const uint64_t ones = __ballot(one);
            same &= one ? ones : ~ones;
        }
        const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1));
        uint32_t old = 0;
        if (have[r]) old = s.cnt[w][digit[r]];
        at[r] = old + before;
        // a wavefront's LDS accesses are done in order: every lane has read before the first of a digit writes
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (have[r] && before == 0) s.cnt[w][digit[r]] = old + (uint32_t)__popcll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += SORT_T) {
        uint32_t sum = s.base[d];
#pragma unroll
        for (int i = 0; i < SORT_W; ++i) {
            const uint32_t c = s.cnt[i][d];
            s.cnt[i][d] = sum;
            sum += c;
        }
        s.base[d] = sum;
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < SORT_ROUNDS; ++r)
        if (have[r]) at[r] += s.cnt[w][digit[r]];
    __syncthreads();
}

// A call of at most SORT_TILE tokens: workgroup 0 sorts them in LDS, the others clear the table meanwhile.
__global__ __launch_bounds__(SORT_T) void sort_few_kernel(GradParams p, int passes)
{
    __shared__ SortLds s;
    __shared__ uint2 buf[SORT_TILE];
    if (blockIdx.x != 0) {
        fill_table<SORT_T>(p, (int64_t)blockIdx.x - 1, (int64_t)gridDim.x - 1);
        return;
    }
    if (threadIdx.x == 0) p.joins[0] = 0;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << p.bits;
    uint2 x[SORT_ROUNDS];
    bool have[SORT_ROUNDS];
    uint32_t digit[SORT_ROUNDS], at[SORT_ROUNDS];
#pragma unroll
    for (int r = 0; r < SORT_ROUNDS; ++r) {
        const uint32_t i = (uint32_t)((w * SORT_ROUNDS + r) * 64 + lane);
        have[r] = i < p.n;
        x[r] = have[r] ? make_uint2(key_at(p, i), i) : make_uint2(0, 0);
    }
    for (int q = 0; q < passes; ++q) {
        // the workgroup's counts per digit give the bases
        for (int i = threadIdx.x; i < bins; i += SORT_T) s.base[i] = 0;
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            digit[r] = (x[r].x >> (q * p.bits)) & (bins - 1);
            if (have[r]) atomicAdd(&s.base[digit[r]], 1u);
        }
        __syncthreads();
        const uint32_t c = (int)threadIdx.x < bins ? s.base[threadIdx.x] : 0;
        const uint32_t first = exclusive_sum(c, s.wave);
        if ((int)threadIdx.x < bins) s.base[threadIdx.x] = first;
        __syncthreads();
        place_tile(s, p.bits, digit, have, at);
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (have[r]) buf[at[r]] = x[r];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const int i = (w * SORT_ROUNDS + r) * 64 + lane;
            if (have[r]) x[r] = buf[i];
        }
        __syncthreads();
    }
#pragma unroll
    for (int r = 0; r < SORT_ROUNDS; ++r) {
        const int i = (w * SORT_ROUNDS + r) * 64 + lane;
        if (have[r]) p.pairs[0][i] = x[r];
    }
}

// Larger calls, one pass: how often each digit occurs among a workgroup's tokens.  Before the first pass (from < 0) the
// tokens come from the caller, and the workgroups behind the sorting ones clear the table.
__global__ __launch_bounds__(SORT_T) void count_kernel(GradParams p, int from, int shift)
{
    __shared__ uint32_t cnt[BINS];
    if ((int)blockIdx.x >= p.sort_wgs) {
        fill_table<SORT_T>(p, (int64_t)blockIdx.x - p.sort_wgs, (int64_t)gridDim.x - p.sort_wgs);
        return;
    }
    if (from < 0 && blockIdx.x == 0 && threadIdx.x == 0) p.joins[0] = 0;
    const int bins = 1 << p.bits;
    for (int i = threadIdx.x; i < bins; i += SORT_T) cnt[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.per_wg, end = begin + p.per_wg < p.n ? begin + p.per_wg : p.n;
    for (int64_t i = begin + threadIdx.x; i < end; i += SORT_T) {
        const uint32_t key = from < 0 ? key_at(p, i) : p.pairs[from][i].x;
        atomicAdd(&cnt[(key >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += SORT_T) p.counts[(int64_t)blockIdx.x * BINS + i] = cnt[i];
}

// ... and the tokens moved to their places: behind all smaller digits, and behind the same digit of earlier workgroups.
__global__ __launch_bounds__(SORT_T) void scatter_kernel(GradParams p, int from, int to, int shift)
{
    __shared__ SortLds s;
    __shared__ uint32_t part[2][SORT_T];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << p.bits;
    const int team = (int)threadIdx.x >> p.bits, teams = SORT_T >> p.bits, bin = threadIdx.x & (bins - 1);
    uint32_t before = 0, all = 0;
#pragma unroll 8
    for (int g = team; g < p.sort_wgs; g += teams) {
        const uint32_t c = p.counts[(int64_t)g * BINS + bin];
        all += c;
        if (g < (int)blockIdx.x) before += c;
    }
    part[0][threadIdx.x] = before;
    part[1][threadIdx.x] = all;
    __syncthreads();
    before = all = 0;
    if ((int)threadIdx.x < bins)
        for (int i = 0; i < teams; ++i) {
            before += part[0][(i << p.bits) + bin];
            all += part[1][(i << p.bits) + bin];
        }
    const uint32_t first = exclusive_sum(all, s.wave);
    if ((int)threadIdx.x < bins) s.base[threadIdx.x] = first + before;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.per_wg, end = begin + p.per_wg < p.n ? begin + p.per_wg : p.n;
    for (int64_t t0 = begin; t0 < end; t0 += SORT_TILE) {
        uint2 x[SORT_ROUNDS];
        bool have[SORT_ROUNDS];
        uint32_t digit[SORT_ROUNDS], at[SORT_ROUNDS];
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r) {
            const int64_t i = t0 + (w * SORT_ROUNDS + r) * 64 + lane;
            have[r] = i < end;
            x[r] = make_uint2(0, 0);
            if (have[r]) x[r] = from < 0 ? make_uint2(key_at(p, i), (uint32_t)i) : p.pairs[from][i];
            digit[r] = (x[r].x >> shift) & (bins - 1);
        }
        place_tile(s, p.bits, digit, have, at);
#pragma unroll
        for (int r = 0; r < SORT_ROUNDS; ++r)
            if (have[r]) p.pairs[to][at[r]] = x[r];
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// gradient: sums
// ---------------------------------------------------------------------------------------------------------------------

// A row's sum, scaled, into the table: written, or added to what is there.
template <int N>
__device__ __forceinline__ void put_row(const GradParams& p, uint32_t row, int c, const float (&sum)[N])
{
    uint32_t* to = (uint32_t*)p.table + (int64_t)row * p.table_stride + c;
    float x[N];
    if (p.accumulate) {
        load_part<F32, N>(to, p.dim - c, x);
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = x[i] + p.scale * sum[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = p.scale * sum[i];
    }
    store_part<F32, N>(to, p.dim - c, x);
}

// A share of the sorted tokens (1 << share_log of them, at most 64: a lane holds one each) and 64 * N columns per wavefront.
// Runs of one token that lie inside the share are written to the table; the sum of one that reaches over the share's begin or
// end goes to the workspace, for join_kernel.
template <typename E>
__global__ __launch_bounds__(64) void sum_kernel(GradParams p, int sorted)
{
    constexpr int N = 16 / E::SIZE, U = 4;
    const int lane = threadIdx.x;
    const uint32_t share = blockIdx.x;
    const int64_t i0 = (int64_t)share << p.share_log;
    const uint32_t size = 1u << p.share_log, none = (uint32_t)p.vocab;
    const uint2* pairs = p.pairs[sorted];
    uint2 mine = make_uint2(none, 0);
    if (lane < (int)size && i0 + lane < p.n) mine = pairs[i0 + lane];
    const uint32_t previous = i0 > 0 ? pairs[i0 - 1].x : none;
    const uint32_t next = i0 + size < p.n ? pairs[i0 + size].x : none;
    const int have = __popcll(__ballot(mine.x != none));
    if (have == 0) return;
    const int c = ((int)blockIdx.y * 64 + lane) * N;
    const bool active = c < p.dim;
    const typename E::word* grad = (const typename E::word*)p.grad + c;
    uint32_t row = __builtin_amdgcn_readlane(mine.x, 0);
    bool first = true;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;

    auto flush = [&](bool last) {
        if (first && previous == row) {
            if (active) store_part<F32, N>((uint32_t*)p.head + (int64_t)share * p.part_stride + c, p.dim - c, sum);
        } else if (last && next == row) {
            if (active) store_part<F32, N>((uint32_t*)p.tail + (int64_t)share * p.part_stride + c, p.dim - c, sum);
            if (blockIdx.y == 0 && lane == 0) p.joins[1 + atomicAdd(&p.joins[0], 1u)] = share;
        } else if (active) {
            put_row<N>(p, row, c, sum);
        }
    };
    for (int j0 = 0; j0 < have; j0 += U) {
        float x[U][N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u < have ? j0 + u : have - 1;
            const uint32_t pos = __builtin_amdgcn_readlane(mine.y, j);
            if (active) load_part<E, N>(grad + (int64_t)pos * p.grad_stride, p.dim - c, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j0 + u >= have) break;
            const uint32_t r = __builtin_amdgcn_readlane(mine.x, j0 + u);
            if (r != row) {
                flush(false);
                row = r;
                first = false;
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = 0.0f;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += x[u][i];
        }
    }
    flush(true);
}

// The runs that reach over shares: the tail of the share where one begins and the heads of the shares behind it, added up by
// eight wavefronts, each every eighth share in order, and these sums in order.
constexpr int JOIN_W = 8;
constexpr int JOIN_GRID = 1024;

__global__ __launch_bounds__(64 * JOIN_W) void join_kernel(GradParams p, int sorted)
{
    constexpr int N = 4, U = 4;
    __shared__ float lds[JOIN_W][64][N];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const uint32_t slabs = ((uint32_t)p.dim + 64 * N - 1) / (64 * N);
    const uint64_t items = (uint64_t)p.joins[0] * slabs;
    const uint2* pairs = p.pairs[sorted];
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t share = p.joins[1 + item / slabs];
        const int c = (int)((uint32_t)(item % slabs) * 64 + lane) * N;
        const bool active = c < p.dim;
        const uint32_t row = pairs[(((int64_t)share + 1) << p.share_log) - 1].x;
        // the shares behind it that begin with the same token: [share + 1, end), found by looking at 64 of them at a time
        uint32_t lo = share + 1, hi = p.n_shares;   // share `lo` begins with it, share `hi` (if there is one) does not
        while (hi - lo > 1) {
            const uint32_t step = (hi - lo + 63) / 64;
            const uint32_t at = lo + (uint32_t)lane * step;
            const bool same = at < hi && pairs[(int64_t)at << p.share_log].x == row;
            const uint32_t k = (uint32_t)__popcll(__ballot(same));   // lanes 0 .. k - 1, lane 0 among them
            lo += (k - 1) * step;
            if (lo + step < hi) hi = lo + step;
        }
        const uint32_t end = lo + 1;
        float sum[N] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (uint32_t g0 = share + 1 + w; g0 < end; g0 += JOIN_W * U) {
            float x[U][N];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t g = g0 + u * JOIN_W;
                if (active && g < end) load_part<F32, N>((const uint32_t*)p.head + (int64_t)g * p.part_stride + c, p.dim - c, x[u]);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (g0 + u * JOIN_W < end) {
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += x[u][i];
                }
        }
#pragma unroll
        for (int i = 0; i < N; ++i) lds[w][lane][i] = sum[i];
        __syncthreads();
        if (w == 0 && active) {
            load_part<F32, N>((const uint32_t*)p.tail + (int64_t)share * p.part_stride + c, p.dim - c, sum);
#pragma unroll
            for (int g = 0; g < JOIN_W; ++g)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += lds[g][lane][i];
            put_row<N>(p, row, c, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// gradient: few tokens
// ---------------------------------------------------------------------------------------------------------------------

// At most FEW tokens, one launch: a wavefront per token (and 64 * N columns) looks at all of them; the first of its kind
// adds up the rows of all of its kind, in order.  The wavefronts behind those clear the rows that no token names.
template <typename E>
__global__ __launch_bounds__(64) void sum_few_kernel(GradParams p)
{
    constexpr int N = 16 / E::SIZE, U = 4;
    static_assert(FEW == 128, "two tokens per lane");
    const int lane = threadIdx.x;
    const uint32_t none = (uint32_t)p.vocab;
    const uint32_t k0 = lane < p.n ? key_at(p, lane) : none, k1 = lane + 64 < p.n ? key_at(p, lane + 64) : none;
    if (blockIdx.x >= p.n) {
        const int64_t wgs = (int64_t)gridDim.x - p.n;
        const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int64_t r = ((int64_t)blockIdx.x - p.n) * gridDim.y + blockIdx.y; r < p.vocab; r += wgs * gridDim.y) {
            if (__ballot(k0 == (uint32_t)r || k1 == (uint32_t)r)) continue;
            for (int c = lane * 4; c < p.dim; c += 256)
                store_part<F32, 4>((uint32_t*)p.table + r * p.table_stride + c, p.dim - c, zero);
        }
        return;
    }
    const int t = (int)blockIdx.x;
    const uint32_t row = __builtin_amdgcn_readlane(t < 64 ? k0 : k1, t & 63);
    uint64_t m0 = __ballot(k0 == row), m1 = __ballot(k1 == row);
    const int leader = m0 ? __ffsll((unsigned long long)m0) - 1 : 64 + __ffsll((unsigned long long)m1) - 1;
    if (row == none || leader != t) return;
    const int c = ((int)blockIdx.y * 64 + lane) * N;
    if (c >= p.dim) return;
    const typename E::word* grad = (const typename E::word*)p.grad + c;
    float sum[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    while (m0 | m1) {
        float x[U][N];
        bool have[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            have[u] = (m0 | m1) != 0;
            int j = 0;
            if (m0) { j = __ffsll((unsigned long long)m0) - 1; m0 &= m0 - 1; }
            else if (m1) { j = 64 + __ffsll((unsigned long long)m1) - 1; m1 &= m1 - 1; }
            if (have[u]) load_part<E, N>(grad + (int64_t)j * p.grad_stride, p.dim - c, x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (have[u]) {
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += x[u][i];
            }
    }
    put_row<N>(p, row, c, sum);
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------

constexpr int64_t MAX_N = 2147483647LL, MAX_TOKENS = GRAVAC_EMBEDDING_MAX_TOKENS;

int share_log_of(int64_t n, int64_t dim)
{
    // tokens per share: the fewer, the more wavefronts; up to 32 once that leaves 8192 of them
    const int64_t slabs = (dim + 511) / 512;
    int log = 2;
    while (log < 5 && (n >> (log + 1)) * slabs >= 8192) ++log;
    return log;
}

struct GradLayout {
    size_t pairs[2], counts, joins, head, tail, total;
    int64_t part_stride;
    uint32_t n_shares;
    int share_log;
};

GradLayout grad_layout(int64_t n, int64_t dim)
{
    GradLayout L;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~(size_t)255;
        return here;
    };
    L.share_log = share_log_of(n, dim);
    L.n_shares = (uint32_t)((n + (1 << L.share_log) - 1) >> L.share_log);
    L.part_stride = (dim + 3) & ~(int64_t)3;
    L.pairs[0] = take(sizeof(uint2) * (size_t)n);
    L.pairs[1] = take(sizeof(uint2) * (size_t)n);
    L.counts = take(sizeof(uint32_t) * SORT_GRID * BINS);
    L.joins = take(sizeof(uint32_t) * ((size_t)L.n_shares + 1));
    L.head = take(sizeof(float) * (size_t)L.n_shares * (size_t)L.part_stride);
    L.tail = take(sizeof(float) * (size_t)L.n_shares * (size_t)L.part_stride);
    L.total = at;
    return L;
}

template <typename E>
void launch_gradient(GradParams& p, const GradLayout& L, hipStream_t stream)
{
    const uint32_t slabs = (uint32_t)((p.dim + 64 * (16 / E::SIZE) - 1) / (64 * (16 / E::SIZE)));
    if (p.n <= FEW) {
        int64_t fill = 0;
        if (!p.accumulate) {
            fill = (p.vocab + slabs - 1) / slabs;
            if (fill > FILL_GRID) fill = FILL_GRID;
        }
        if (p.n + fill > 0)
            hipLaunchKernelGGL(sum_few_kernel<E>, dim3((uint32_t)(p.n + fill), slabs), dim3(64), 0, stream, p);
        return;
    }
    int bits = 1;
    while (bits < 32 && (p.vocab >> bits) != 0) ++bits;
    const int passes = (bits + MAX_BITS - 1) / MAX_BITS;
    p.bits = (bits + passes - 1) / passes;
    if (p.bits < MIN_BITS) p.bits = MIN_BITS;
    int64_t fill = 0;
    if (!p.accumulate) {
        fill = (p.vocab * p.dim + 4 * SORT_T - 1) / (4 * SORT_T);
        if (fill > FILL_GRID) fill = FILL_GRID;
    }
    int sorted = 0;
    if (p.n <= SORT_TILE) {
        hipLaunchKernelGGL(sort_few_kernel, dim3(1 + (uint32_t)fill), dim3(SORT_T), 0, stream, p, passes);
    } else {
        const int64_t tiles = (p.n + SORT_TILE - 1) / SORT_TILE;
        p.per_wg = (tiles + SORT_GRID - 1) / SORT_GRID * SORT_TILE;
        p.sort_wgs = (int32_t)((p.n + p.per_wg - 1) / p.per_wg);
        int from = -1;
        for (int q = 0; q < passes; ++q) {
            const int to = q & 1;
            hipLaunchKernelGGL(count_kernel, dim3((uint32_t)p.sort_wgs + (q == 0 ? (uint32_t)fill : 0u)), dim3(SORT_T), 0,
                               stream, p, from, q * p.bits);
            hipLaunchKernelGGL(scatter_kernel, dim3((uint32_t)p.sort_wgs), dim3(SORT_T), 0, stream, p, from, to, q * p.bits);
            from = to;
        }
        sorted = from;
    }
    hipLaunchKernelGGL(sum_kernel<E>, dim3(L.n_shares, slabs), dim3(64), 0, stream, p, sorted);
    hipLaunchKernelGGL(join_kernel, dim3(JOIN_GRID), dim3(64 * JOIN_W), 0, stream, p, sorted);
}

bool misaligned(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

}  // namespace

extern "C" {

int gravac_embedding_lookup(const void* table, int table_type, int64_t vocab, int64_t dim, int64_t table_stride,
                            const void* tokens, int token_bytes, int64_t n_tokens, float scale, void* out, int out_type,
                            int64_t out_stride, void* stream_v)
{
    if (!known(table_type) || !known(out_type) || (token_bytes != 4 && token_bytes != 8)) return GRAVAC_ERR_INVALID_ARG;
    if (vocab < 1 || vocab > MAX_N || dim < 1 || dim > GRAVAC_EMBEDDING_MAX_DIM || n_tokens < 0 || n_tokens > MAX_TOKENS)
        return GRAVAC_ERR_INVALID_ARG;
    if (table_stride < dim || out_stride < dim || table_stride > MAX_N || out_stride > MAX_N) return GRAVAC_ERR_INVALID_ARG;
    if (!table || misaligned(table, size_of(table_type))) return GRAVAC_ERR_INVALID_ARG;
    if (n_tokens == 0) return GRAVAC_OK;
    if (!tokens || !out || misaligned(tokens, token_bytes) || misaligned(out, size_of(out_type))) return GRAVAC_ERR_INVALID_ARG;
    (void)hipGetLastError();
    LookupParams p;
    p.table = table; p.tokens = tokens; p.out = out;
    p.vocab = vocab; p.table_stride = table_stride; p.n = n_tokens; p.out_stride = out_stride;
    p.dim = (int32_t)dim; p.wide = token_bytes == 8; p.lanes = 0; p.scale = scale;
    hipStream_t stream = (hipStream_t)stream_v;
    if (table_type == GRAVAC_FLOAT32) launch_lookup<F32>(p, out_type, stream);
    else if (table_type == GRAVAC_BFLOAT16) launch_lookup<BF16>(p, out_type, stream);
    else launch_lookup<F16>(p, out_type, stream);
    return hipGetLastError() == hipSuccess ? GRAVAC_OK : GRAVAC_ERR_HIP;
}

int gravac_embedding_gradient_workspace_bytes(int64_t n_tokens, int64_t vocab, int64_t dim, size_t* bytes_out)
{
    if (!bytes_out || n_tokens < 0 || n_tokens > MAX_TOKENS || vocab < 1 || vocab > MAX_N || dim < 1 || dim > GRAVAC_EMBEDDING_MAX_DIM)
        return GRAVAC_ERR_INVALID_ARG;
    *bytes_out = grad_layout(n_tokens, dim).total;
    return GRAVAC_OK;
}

int gravac_embedding_gradient(const void* grad_out, int grad_type, int64_t n_tokens, int64_t dim, int64_t grad_stride,
                              const void* tokens, int token_bytes, int64_t padding_token, float scale, float* table_grad,
                              int64_t vocab, int64_t table_stride, void* workspace, size_t workspace_bytes, unsigned flags,
                              void* stream_v)
{
    if (!known(grad_type) || (token_bytes != 4 && token_bytes != 8) || (flags & ~GRAVAC_FLAG_ACCUMULATE)) return GRAVAC_ERR_INVALID_ARG;
    if (vocab < 1 || vocab > MAX_N || dim < 1 || dim > GRAVAC_EMBEDDING_MAX_DIM || n_tokens < 0 || n_tokens > MAX_TOKENS)
        return GRAVAC_ERR_INVALID_ARG;
    if (table_stride < dim || grad_stride < dim || table_stride > MAX_N || grad_stride > MAX_N) return GRAVAC_ERR_INVALID_ARG;
    if (!table_grad || misaligned(table_grad, 4)) return GRAVAC_ERR_INVALID_ARG;
    if (n_tokens > 0 && (!grad_out || !tokens || misaligned(grad_out, size_of(grad_type)) || misaligned(tokens, token_bytes)))
        return GRAVAC_ERR_INVALID_ARG;
    const GradLayout L = grad_layout(n_tokens, dim);
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < L.total) return GRAVAC_ERR_WORKSPACE;
    (void)hipGetLastError();
    char* ws = (char*)workspace;
    GradParams p;
    p.grad = grad_out; p.tokens = tokens; p.table = table_grad;
    p.n = n_tokens; p.grad_stride = grad_stride; p.table_stride = table_stride;
    p.vocab = vocab; p.padding = padding_token;
    p.dim = (int32_t)dim; p.wide = token_bytes == 8;
    p.accumulate = (flags & GRAVAC_FLAG_ACCUMULATE) ? 1 : 0;
    p.scale = scale;
    p.pairs[0] = (uint2*)(ws + L.pairs[0]); p.pairs[1] = (uint2*)(ws + L.pairs[1]);
    p.counts = (uint32_t*)(ws + L.counts); p.joins = (uint32_t*)(ws + L.joins);
    p.head = (float*)(ws + L.head); p.tail = (float*)(ws + L.tail);
    p.part_stride = L.part_stride; p.share_log = L.share_log; p.n_shares = L.n_shares;
    p.per_wg = 0; p.sort_wgs = 0; p.bits = 0;
    hipStream_t stream = (hipStream_t)stream_v;
    if (grad_type == GRAVAC_FLOAT32) launch_gradient<F32>(p, L, stream);
    else if (grad_type == GRAVAC_BFLOAT16) launch_gradient<BF16>(p, L, stream);
    else launch_gradient<F16>(p, L, stream);
    return hipGetLastError() == hipSuccess ? GRAVAC_OK : GRAVAC_ERR_HIP;
}

}  // extern "C"
