// embedding.hip - the embedding of a language model beside its compressed gradient: lookup of rows by token, and the
// table's gradient, summed by token in a fixed order.
//
// Both are bound by memory.  The lookup is one gather.  The gradient is a sum over the tokens that name a row; adding row by
// row with atomics would give sums that depend on scheduling (and a queue at the row of a frequent token), so the tokens are
// sorted first, with their positions, by a stable radix sort: equal tokens then stand together in the order of their
// positions, a wavefront adds up the rows of its share of the sorted tokens in registers, and every row of the table is
// written by one wavefront.
//
// Measured: the lookup of 65,539 rows of 8 KiB 136 us (5.1 TB/s; a copy of 2 GiB runs at 4.9); the gradient of 131,072
// tokens on as many rows of 4096 720 us (4.5 TB/s), of 700 tokens on 33,278 rows of 650 16 to 18 us (4.9 to 5.5 TB/s, nearly all of
// it zeros).  Calls of a few tokens are bound by the launch, 7 us with the call itself.

#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

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
    int32_t stream;  // see STREAM_BYTES
    float scale;
};

// out[t] = scale * table[tokens[t]]: the product in binary32, then one rounding to the output's type.  A group of `lanes`
// lanes takes K accesses of a row each, all in flight together; blockIdx.y walks along a row.  A token outside the table reads
// row 0 and drops it.
template <typename A, typename B, int N, int K>
__global__ __launch_bounds__(256) void lookup_kernel(LookupParams p)
{
    const int lane = threadIdx.x & (p.lanes - 1), groups = 256 / p.lanes;
    for (int64_t t = (int64_t)blockIdx.x * groups + threadIdx.x / p.lanes; t < p.n; t += (int64_t)gridDim.x * groups) {
        const int64_t token = token_at(p.tokens, p.wide, t);
        const bool inside = token >= 0 && token < p.vocab;
        const typename A::word* row = (const typename A::word*)p.table + (inside ? token : 0) * p.table_stride;
        typename B::word* to = (typename B::word*)p.out + t * p.out_stride;
        const int c0 = ((int)blockIdx.y * K * p.lanes + lane) * N;
        Pack<A, N> v[K];
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] = fetch<A, N>(row + Columns<N>(c0 + k * p.lanes * N, p.dim).at);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const Columns<N> c(c0 + k * p.lanes * N, p.dim);
            float x[N];
            unpack<A, N>(v[k], x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = inside ? x[i] * p.scale : 0.0f;
            if (c.skip >= N) continue;
            if (p.stream && c.skip == 0) store_streaming<B, N>(to + c.at, x);
            else store_behind<B, N>(to + c.at, c.skip, x);
        }
    }
}

template <typename A, typename B>
void launch_lookup(LookupParams& p, hipStream_t stream)
{
    constexpr int WIDE = 16 / (A::SIZE > B::SIZE ? A::SIZE : B::SIZE);
    const bool narrow = p.dim < WIDE;
    const int64_t n = narrow ? 1 : WIDE, chunks = ((int64_t)p.dim + n - 1) / n;
    p.lanes = 4;
    while (p.lanes < 64 && p.lanes < chunks) p.lanes *= 2;
    const int64_t groups = 256 / p.lanes, rows = (p.n + groups - 1) / groups;
    const int64_t x = rows < LOOKUP_GRID ? rows : LOOKUP_GRID;
    // four accesses per lane once there are wavefronts enough to fill the card without them
    const int k = p.n * chunks >= (1 << 19) && chunks > p.lanes ? 4 : 1;
    const dim3 grid((uint32_t)x, (uint32_t)((chunks + (int64_t)p.lanes * k - 1) / ((int64_t)p.lanes * k)));
    if (narrow) hipLaunchKernelGGL((lookup_kernel<A, B, 1, 1>), grid, dim3(256), 0, stream, p);
    else if (k == 4) hipLaunchKernelGGL((lookup_kernel<A, B, WIDE, 4>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((lookup_kernel<A, B, WIDE, 1>), grid, dim3(256), 0, stream, p);
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
constexpr int SORT_ROUNDS = 4;                   // tokens per thread in a tile at most
constexpr int SORT_TILE = SORT_T * SORT_ROUNDS;  // tokens of a tile at most
constexpr int MAX_BITS = 9;                      // bits of a digit at most: two passes for a vocabulary up to 2^18 - 1
constexpr int MIN_BITS = 4;
constexpr int BINS = 1 << MAX_BITS;
constexpr int SORT_GRID = 128;                   // sorting workgroups at most: each adds up all workgroups' counts
constexpr int FEW = 1024;                        // calls of at most this many tokens are not sorted
constexpr int FEW_T = 256, FEW_W = FEW_T / 64;
constexpr uint32_t FILL_GRID = 1 << 23;          // ... of its workgroups that clear rows at most (the global size has 32 bits)

struct GradParams {
    const void* grad;
    const void* tokens;
    float* table;
    int64_t n, grad_stride, table_stride;
    int64_t vocab, padding;
    int32_t dim, wide;
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
    int32_t fill_rows;     // rows of the table that a workgroup looks after, of those that no token names
    uint32_t fill_wgs;     // such workgroups
    uint32_t fills;        // ... along the grid
    int32_t stream;        // see STREAM_BYTES
};

// The token at position i as a sort key: `vocab` for one that takes no part.
__device__ __forceinline__ uint32_t key_at(const GradParams& p, int64_t i)
{
    const int64_t t = token_at(p.tokens, p.wide, i);
    return t < 0 || t >= p.vocab || t == p.padding ? (uint32_t)p.vocab : (uint32_t)t;
}

// A workgroup clears the rows that no token names of a block of fill_rows (at most 64, about FILL_ELEMENTS elements): all of
// its threads write consecutive places, and workgroups that run together neighbouring blocks.  (A wavefront per row, the
// rows of a workgroup far apart or not, wrote 2 to 4.7 TB/s, this 5.8.)  absent: a bit per row of the block, which begins inside
// the table.
constexpr int64_t FILL_ELEMENTS = 16384;

__device__ void clear_rows(const GradParams& p, int64_t row0, uint64_t absent)
{
    const float zero[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    const int threads = (int)blockDim.x;
    if (p.table_stride != p.dim || p.fill_rows == 1 || p.dim < 4) {
        for (; absent; absent &= absent - 1) {
            uint32_t* to = (uint32_t*)p.table + (row0 + __ffsll((unsigned long long)absent) - 1) * p.table_stride;
            for (int c = (int)threadIdx.x * 4; c < p.dim; c += threads * 4) store_part<F32, 4>(to + c, p.dim - c, zero);
        }
        return;
    }
    uint32_t* to = (uint32_t*)p.table + row0 * p.dim;
    const uint32_t n = (uint32_t)(p.vocab - row0 < p.fill_rows ? p.vocab - row0 : p.fill_rows) * (uint32_t)p.dim;
    // x / dim as the upper half of a product: exact as long as x dim < 2^32, and x <= 4 FILL_ELEMENTS, dim <= 2 FILL_ELEMENTS
    const uint32_t inverse = (uint32_t)(((1ull << 32) + p.dim - 1) / (uint32_t)p.dim);
    auto clear = [&](uint32_t e) { return (absent >> __umulhi(e, inverse)) & 1; };
    for (uint32_t e = threadIdx.x * 4; e < n; e += threads * 4) {
        if (e + 3 < n && clear(e) && clear(e + 3)) {   // (two rows at most)
            if (p.stream) store_streaming<F32, 4>(to + e, zero);
            else store<F32, 4>(to + e, zero);
        } else {
            for (uint32_t i = e; i < e + 4 && i < n; ++i)
                if (clear(i)) to[i] = 0;
        }
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
template <int ROUNDS>
__device__ void place_tile(SortLds& s, int bits, const uint32_t (&digit)[ROUNDS], const bool (&have)[ROUNDS], uint32_t (&at)[ROUNDS])
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << bits;
    for (int i = threadIdx.x; i < SORT_W * bins; i += SORT_T) s.cnt[i >> bits][i & (bins - 1)] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
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
    for (int r = 0; r < ROUNDS; ++r)
        if (have[r]) at[r] += s.cnt[w][digit[r]];
    __syncthreads();
}

// A call of at most SORT_TILE tokens: one workgroup sorts them in LDS.
__global__ __launch_bounds__(SORT_T) void sort_few_kernel(GradParams p, int passes)
{
    __shared__ SortLds s;
    __shared__ uint2 buf[SORT_TILE];
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

__device__ __forceinline__ uint32_t key_of(const GradParams& p, int from, int64_t i)   // from < 0: the caller's tokens
{
    return from < 0 ? key_at(p, i) : p.pairs[from][i].x;
}

// Larger calls, one pass: how often each digit occurs among a workgroup's tokens.
__global__ __launch_bounds__(SORT_T) void count_kernel(GradParams p, int from, int shift)
{
    __shared__ uint32_t cnt[BINS];
    const int bins = 1 << p.bits;
    for (int i = threadIdx.x; i < bins; i += SORT_T) cnt[i] = 0;
    __syncthreads();
    const int64_t begin = blockIdx.x * p.per_wg, end = begin + p.per_wg < p.n ? begin + p.per_wg : p.n;
    for (int64_t i = begin + threadIdx.x; i < end; i += SORT_T) atomicAdd(&cnt[(key_of(p, from, i) >> shift) & (bins - 1)], 1u);
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += SORT_T) p.counts[(int64_t)blockIdx.x * BINS + i] = cnt[i];
}

// ... and the tokens moved to their places: behind all smaller digits, and behind the same digit of earlier workgroups.
// (Workgroups that count all tokens themselves spare a launch per pass and took as long: 16,381 tokens in tiles of four tokens per
// thread 15.3 us instead of 8.1 and 3 to 5 for the counts.  With tiles of one the two kernels take 6.0 and 4.6.)
template <int ROUNDS>
__global__ __launch_bounds__(SORT_T) void scatter_kernel(GradParams p, int from, int to, int shift)
{
    __shared__ SortLds s;
    __shared__ uint32_t part[2][SORT_T];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << p.bits;
    const int team = (int)threadIdx.x >> p.bits, teams = SORT_T >> p.bits, bin = threadIdx.x & (bins - 1);
    const int64_t begin = blockIdx.x * p.per_wg, end = begin + p.per_wg < p.n ? begin + p.per_wg : p.n;
    uint32_t before = 0, all = 0;
    if (blockIdx.x == 0 && threadIdx.x == 0) p.joins[0] = 0;
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
    for (int64_t t0 = begin; t0 < end; t0 += SORT_T * ROUNDS) {
        uint2 x[ROUNDS];
        bool have[ROUNDS];
        uint32_t digit[ROUNDS], at[ROUNDS];
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r) {
            const int64_t i = t0 + (w * ROUNDS + r) * 64 + lane;
            have[r] = i < end;
            x[r] = make_uint2(0, 0);
            if (have[r]) x[r] = from < 0 ? make_uint2(key_at(p, i), (uint32_t)i) : p.pairs[from][i];
            digit[r] = (x[r].x >> shift) & (bins - 1);
        }
        place_tile(s, p.bits, digit, have, at);
#pragma unroll
        for (int r = 0; r < ROUNDS; ++r)
            if (have[r]) p.pairs[to][at[r]] = x[r];
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// gradient: sums
// ---------------------------------------------------------------------------------------------------------------------

// Columns of a row's sum, scaled, into the table: written, or added to what is there (`old`).
template <bool ADD, int N>
__device__ __forceinline__ void put_row(const GradParams& p, uint32_t row, const Columns<N>& c, const float (&sum)[N], const float (&old)[N])
{
    if (c.skip >= N) return;
    float x[N];
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = ADD ? old[i] + p.scale * sum[i] : p.scale * sum[i];
    uint32_t* to = (uint32_t*)p.table + (int64_t)row * p.table_stride + c.at;
    if (!ADD && p.stream && c.skip == 0) store_streaming<F32, N>(to, x);
    else store_behind<F32, N>(to, c.skip, x);
}

template <bool ADD, int N>
__device__ __forceinline__ void get_row(const GradParams& p, uint32_t row, const Columns<N>& c, float (&old)[N])
{
    if (ADD) load<F32, N>((const uint32_t*)p.table + (int64_t)row * p.table_stride + c.at, old);
}

// A share of the sorted tokens (1 << share_log of them, at most 64: a lane holds one each) per workgroup, 64 * N columns per
// wavefront: a workgroup reads and writes whole rows, up to SUM_W wavefronts of them at a time.
// The sum of a run of one token is written to the table by the wavefront of the share where it begins, which follows it into
// the next share; only a run that covers a whole share is left in parts in the workspace, for join_kernel.  (All runs that
// cross a share's end left to it: 131,072 tokens of a text give 2500 of them, and 146 us instead of 24.)
// The first wavefronts clear the rows that no token names: a lane looks for one row among the sorted tokens, so that no row is
// written twice (131,072 tokens on as many rows of 4096: 1079 us with all rows cleared beside the sort, 758 so; 719 since the loads of
// a round are under way together).
constexpr int SUM_W = 8;

// The place of the first sorted token that is not below `row`, by a wavefront that looks at 64 of them at a time.
__device__ __forceinline__ uint32_t first_at_least(const uint2* pairs, uint32_t n, uint32_t row)
{
    const uint32_t lane = threadIdx.x & 63;
    uint32_t lo = 0, hi = n;   // it lies in [lo, hi]
    while (lo < hi) {
        const uint32_t step = (hi - lo + 63) / 64, at = lo + lane * step;
        const uint32_t below = (uint32_t)__popcll(__ballot(at < hi && pairs[at].x < row));   // lanes 0 .. below - 1
        if (below == 0) break;
        hi = lo + below * step < hi ? lo + below * step : hi;
        lo += (below - 1) * step + 1;
    }
    return lo;
}

template <typename E, bool ADD, int N>
__global__ __launch_bounds__(64 * SUM_W) void sum_kernel(GradParams p, int sorted)
{
    constexpr int U = 4;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = (int)blockDim.x >> 6;
    const uint2* pairs = p.pairs[sorted];
    if (blockIdx.x < p.fills) {
        const int64_t id = (int64_t)blockIdx.x * gridDim.y + blockIdx.y, r = id * p.fill_rows + lane;
        if (id >= p.fill_wgs) return;   // (the grid holds whole groups of gridDim.y: the last may go on behind the table)
        const uint32_t row = (uint32_t)r;
        bool named = lane >= p.fill_rows || r >= p.vocab;
        uint32_t lo = first_at_least(pairs, (uint32_t)p.n, (uint32_t)(id * p.fill_rows));
        uint32_t hi = first_at_least(pairs, (uint32_t)p.n, (uint32_t)(id * p.fill_rows) + p.fill_rows);
        if (!named) {
            const uint32_t behind = hi;
            while (lo < hi) {
                const uint32_t mid = lo + (hi - lo) / 2;
                if (pairs[mid].x < row) lo = mid + 1;
                else hi = mid;
            }
            named = lo < behind && pairs[lo].x == row;
        }
        clear_rows(p, id * p.fill_rows, ~__ballot(named));
        return;
    }
    const uint32_t share = blockIdx.x - p.fills;
    const int64_t i0 = (int64_t)share << p.share_log;
    const int size = 1 << p.share_log;
    const uint32_t none = (uint32_t)p.vocab;
    uint2 mine = make_uint2(none, 0), behind = make_uint2(none, 0);
    if (lane < size && i0 + lane < p.n) mine = pairs[i0 + lane];
    if (lane < size && i0 + size + lane < p.n) behind = pairs[i0 + size + lane];
    const uint32_t previous = i0 > 0 ? pairs[i0 - 1].x : none, before = i0 > 0 ? pairs[i0 - size].x : none;
    const int have = __popcll(__ballot(mine.x != none));
    if (have == 0) return;
    uint32_t row = __builtin_amdgcn_readlane(mine.x, 0);
    const uint32_t last = __builtin_amdgcn_readlane(mine.x, have - 1);
    const int head = __popcll(__ballot(mine.x == row));        // tokens of the first run that lie in this share
    const int follow = have == size ? __popcll(__ballot(behind.x == last)) : 0;   // tokens of the last run in the next
    int begin = 0, end = have;
    bool to_head = false, to_tail = false;                      // the first run's or the last run's sum is a part
    if (row == previous) {
        if (head == size || before == row) to_head = true;      // the run covers this share or the one before
        else begin = head;                                      // ... it is the share's before
    }
    if (!(to_head && head == size) && follow > 0) {
        // (a run that fills this share and begins with it is in parts too)
        if (follow == size || (row == last && head == size)) to_tail = true;
        else end = have + follow;
    }
    if (begin == end) return;
    const int c0 = ((int)blockIdx.y * waves + w) * 64 * N;
    if (c0 >= p.dim) return;
    const Columns<N> c(c0 + lane * N, p.dim);
    const typename E::word* grad = (const typename E::word*)p.grad + c.at;
    if (to_tail && blockIdx.y == 0 && threadIdx.x == 0) p.joins[1 + atomicAdd(&p.joins[0], 1u)] = share;
    row = __builtin_amdgcn_readlane(mine.x, begin < have ? begin : 0);
    float sum[N], kept[N];   // kept: what the table holds in the row of the last token so far
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;

    auto flush = [&](bool ends) {
        if (to_head) {
            if (c.skip < N) store_behind<F32, N>((uint32_t*)p.head + (int64_t)share * p.part_stride + c.at, c.skip, sum);
            to_head = false;
        } else if (ends && to_tail) {
            if (c.skip < N) store_behind<F32, N>((uint32_t*)p.tail + (int64_t)share * p.part_stride + c.at, c.skip, sum);
        } else {
            put_row<ADD, N>(p, row, c, sum, kept);
        }
    };
    auto token_of = [&](int j) { return (uint32_t)(j < have ? __builtin_amdgcn_readlane(mine.x, j) : __builtin_amdgcn_readlane(behind.x, (j - have) & 63)); };
    auto place_of = [&](int j) { return (uint32_t)(j < have ? __builtin_amdgcn_readlane(mine.y, j) : __builtin_amdgcn_readlane(behind.y, (j - have) & 63)); };
    for (int j0 = begin; j0 < end; j0 += U) {
        Pack<E, N> v[U];
        float old[U][N];   // of the rows whose last token this is; all loads of a round are under way together
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = fetch<E, N>(grad + (int64_t)place_of(j0 + u < end ? j0 + u : end - 1) * p.grad_stride);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u < end ? j0 + u : end - 1;
            if (ADD && (j + 1 == end || token_of(j + 1) != token_of(j))) get_row<ADD, N>(p, token_of(j), c, old[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (j0 + u >= end) break;
            const uint32_t r = token_of(j0 + u);
            if (r != row) {
                flush(false);
                row = r;
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] = 0.0f;
            }
            float x[N];
            unpack<E, N>(v[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] += x[i];
            if (ADD) {
#pragma unroll
                for (int i = 0; i < N; ++i) kept[i] = old[u][i];
            }
        }
    }
    flush(true);
}

// The runs that cover a share and more: the tail of the share where one begins and the heads of the shares behind it, added up by
// eight wavefronts, each every eighth share in order, and these sums in order.  Eight loads are under way together, but two at the end:
// most runs are short (131,072 tokens of 4096: 24 us, 33 with eights alone; one of 440,000 tokens: 233 us, 283 with fours alone).
constexpr int JOIN_W = 8;
constexpr int JOIN_GRID = 1024;

template <bool ADD>
__global__ __launch_bounds__(64 * JOIN_W) void join_kernel(GradParams p, int sorted)
{
    constexpr int N = 4, U = 8;
    __shared__ float lds[JOIN_W][64][N];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t slabs = ((uint32_t)p.dim + 64 * N - 1) / (64 * N);
    const uint64_t items = (uint64_t)p.joins[0] * slabs;
    const uint2* pairs = p.pairs[sorted];
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t share = p.joins[1 + item / slabs];
        // (a part's stride is whole lanes' columns: what lies behind its row is read and dropped)
        const int c0 = (int)((uint32_t)(item % slabs) * 64 + lane) * N;
        const Columns<N> c(c0, (int)p.part_stride);
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
        uint32_t g = share + 1 + w;
        auto add = [&](auto count) {   // of this wavefront's next shares, loads together (behind the last one: of it again)
            constexpr int M = decltype(count)::value;
            float x[M][N];
#pragma unroll
            for (int u = 0; u < M; ++u)
                load<F32, N>((const uint32_t*)p.head + (int64_t)(g + u * JOIN_W < end ? g + u * JOIN_W : end - 1) * p.part_stride + c.at, x[u]);
#pragma unroll
            for (int u = 0; u < M; ++u)
                if (g + u * JOIN_W < end) {
#pragma unroll
                    for (int i = 0; i < N; ++i) sum[i] += x[u][i];
                }
            g += M * JOIN_W;
        };
        while (g + (U - 1) * JOIN_W < end) add(std::integral_constant<int, U>());
        while (g < end) add(std::integral_constant<int, 2>());
#pragma unroll
        for (int i = 0; i < N; ++i) lds[w][lane][i] = sum[i];
        __syncthreads();
        if (w == 0 && c0 < p.dim) {
            load<F32, N>((const uint32_t*)p.tail + (int64_t)share * p.part_stride + c.at, sum);
#pragma unroll
            for (int g = 0; g < JOIN_W; ++g)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += lds[g][lane][i];
            uint32_t* to = (uint32_t*)p.table + (int64_t)row * p.table_stride + c0;
            float old[N];
            if (ADD) load_part<F32, N>(to, p.dim - c0, old);
#pragma unroll
            for (int i = 0; i < N; ++i) sum[i] = ADD ? old[i] + p.scale * sum[i] : p.scale * sum[i];
            store_part<F32, N>(to, p.dim - c0, sum);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// gradient: few tokens
// ---------------------------------------------------------------------------------------------------------------------

// At most FEW tokens, one launch: a workgroup per token (and 64 * N columns) looks at all of them; the first of its kind adds
// up the rows of all of its kind, its wavefronts in turn, and their sums in order.  The first workgroups clear the rows
// that no token names.  (700 tokens of 33,278 rows of 650: 16 to 18 us, 32 with a sort beside the clearing and two more
// launches.)
template <typename E, bool ADD, int N>
__global__ __launch_bounds__(FEW_T) void sum_few_kernel(GradParams p)
{
    constexpr int U = 4;
    __shared__ uint32_t keys[FEW];
    __shared__ float lds[FEW_W][64][N + 1];
    __shared__ uint32_t named[64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t none = (uint32_t)p.vocab;
    if (blockIdx.x < p.fills) {
        for (uint32_t id = blockIdx.x * gridDim.y + blockIdx.y; id < p.fill_wgs; id += p.fills * gridDim.y) {
            __syncthreads();
            if (threadIdx.x < 64) named[threadIdx.x] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < p.n; i += FEW_T) {
                const uint32_t k = key_at(p, i);
                if (k != none && k / p.fill_rows == id) named[k % p.fill_rows] = 1;
            }
            __syncthreads();
            const int64_t row0 = (int64_t)id * p.fill_rows;
            clear_rows(p, row0, __ballot(lane < p.fill_rows && row0 + lane < p.vocab && !named[lane]));
        }
        return;
    }
    const int groups = (int)((p.n + 63) / 64), t = (int)(blockIdx.x - p.fills);
    for (int i = threadIdx.x; i < groups * 64; i += FEW_T) keys[i] = i < p.n ? key_at(p, i) : none;
    __syncthreads();
    const uint32_t row = keys[t];
    if (row == none) return;
    uint64_t seen = 0;   // of its kind, before it
    for (int g = 0; g <= t / 64; ++g) {
        const uint64_t before = t >= g * 64 + 64 ? ~0ull : (1ull << (t - g * 64)) - 1;
        seen |= __ballot(keys[g * 64 + lane] == row) & before;
    }
    if (seen) return;
    const Columns<N> c(((int)blockIdx.y * 64 + lane) * N, p.dim);
    const typename E::word* grad = (const typename E::word*)p.grad + c.at;
    float sum[N], old[N];
#pragma unroll
    for (int i = 0; i < N; ++i) sum[i] = 0.0f;
    if (w == 0) get_row<ADD, N>(p, row, c, old);
    int at = 0, count = 0;   // how many of its kind have been seen, and how many of them wait to be added
    int wait[U] = {t, t, t, t};
    auto add = [&]() {
        Pack<E, N> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = fetch<E, N>(grad + (int64_t)wait[u] * p.grad_stride);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < count) {
                float x[N];
                unpack<E, N>(v[u], x);
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += x[i];
            }
        count = 0;
    };
    for (int g = t / 64; g < groups; ++g) {
        uint64_t m = __ballot(keys[g * 64 + lane] == row);
        for (; m; m &= m - 1, ++at) {
            if (at % FEW_W != w) continue;
            const int j = g * 64 + __ffsll((unsigned long long)m) - 1;
#pragma unroll
            for (int u = 0; u < U; ++u) wait[u] = u == count ? j : wait[u];
            if (++count == U) add();
        }
    }
    if (count > 0) add();
    if (at > 1) {   // the same for all wavefronts
#pragma unroll
        for (int i = 0; i < N; ++i) lds[w][lane][i] = sum[i];
        __syncthreads();
        if (w == 0)
#pragma unroll
            for (int v = 1; v < FEW_W; ++v)
#pragma unroll
                for (int i = 0; i < N; ++i) sum[i] += lds[v][lane][i];
    }
    if (w == 0) put_row<ADD, N>(p, row, c, sum, old);
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------

constexpr int64_t MAX_N = 2147483647LL, MAX_TOKENS = GRAVAC_EMBEDDING_MAX_TOKENS;

int share_log_of(int64_t n, int64_t dim)
{
    // tokens per share: the fewer, the more wavefronts; the more, the fewer runs to join; up to 32 that leave 4096 of them
    const int64_t slabs = (dim + 511) / 512;
    int log = 2;
    while (log < 5 && (n >> (log + 1)) * slabs >= 4096) ++log;
    return (n >> log) > (1 << 24) ? 6 : log;   // (a lane holds a token; the grid has 32 bits)
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

// N: columns of a lane (one for rows of less than 16 bytes, so that a row holds a lane's)
template <typename E, bool ADD, int N>
void launch_gradient(GradParams& p, const GradLayout& L, hipStream_t stream)
{
    const uint32_t slabs = (uint32_t)((p.dim + 64 * N - 1) / (64 * N));
    const uint32_t waves = p.n <= FEW ? FEW_W : slabs < SUM_W ? slabs : SUM_W;
    const uint32_t columns = p.n <= FEW ? slabs : (slabs + waves - 1) / waves;   // workgroups side by side
    if (!ADD) {
        const int64_t rows = (p.n <= FEW ? 1 : 4) * FILL_ELEMENTS / p.dim;   // (four times as many to a search)
        p.fill_rows = (int32_t)(rows < 1 ? 1 : rows > 64 ? 64 : rows);
        p.fill_wgs = (uint32_t)((p.vocab + p.fill_rows - 1) / p.fill_rows);
        p.fills = (p.fill_wgs + columns - 1) / columns;
        if (p.n <= FEW && p.fills > FILL_GRID) p.fills = FILL_GRID;
    }
    if (p.n <= FEW) {
        if (p.n + p.fills > 0)
            hipLaunchKernelGGL((sum_few_kernel<E, ADD, N>), dim3((uint32_t)p.n + p.fills, slabs), dim3(FEW_T), 0, stream, p);
        return;
    }
    int bits = 1;
    while (bits < 32 && (p.vocab >> bits) != 0) ++bits;
    const int passes = (bits + MAX_BITS - 1) / MAX_BITS;
    p.bits = (bits + passes - 1) / passes;
    if (p.bits < MIN_BITS) p.bits = MIN_BITS;
    int sorted = 0;
    if (p.n <= SORT_TILE) {
        hipLaunchKernelGGL(sort_few_kernel, dim3(1), dim3(SORT_T), 0, stream, p, passes);
    } else {
        // tiles of one token per thread until a workgroup has several of them: more workgroups, each sooner done (against four
        // tokens per thread the call takes 6 us less with 5000 tokens, 7 with 16,384, 7 with 131,072, 3 with 262,144, 5 with
        // 600,000, and 6 us more with 1,048,576)
        const bool one = p.n <= 4 * SORT_GRID * SORT_T;
        const int64_t tile = one ? SORT_T : SORT_TILE, tiles = (p.n + tile - 1) / tile;
        p.per_wg = (tiles + SORT_GRID - 1) / SORT_GRID * tile;
        p.sort_wgs = (int32_t)((p.n + p.per_wg - 1) / p.per_wg);
        const dim3 grid((uint32_t)p.sort_wgs);
        int from = -1;
        for (int q = 0; q < passes; ++q) {
            const int to = q & 1;
            hipLaunchKernelGGL(count_kernel, grid, dim3(SORT_T), 0, stream, p, from, q * p.bits);
            if (one) hipLaunchKernelGGL(scatter_kernel<1>, grid, dim3(SORT_T), 0, stream, p, from, to, q * p.bits);
            else hipLaunchKernelGGL(scatter_kernel<SORT_ROUNDS>, grid, dim3(SORT_T), 0, stream, p, from, to, q * p.bits);
            from = to;
        }
        sorted = from;
    }
    hipLaunchKernelGGL((sum_kernel<E, ADD, N>), dim3(L.n_shares + p.fills, columns), dim3(64 * waves), 0, stream, p, sorted);
    hipLaunchKernelGGL(join_kernel<ADD>, dim3(JOIN_GRID), dim3(64 * JOIN_W), 0, stream, p, sorted);
}

template <typename E>
void launch_gradient(GradParams& p, const GradLayout& L, bool add, hipStream_t stream)
{
    constexpr int WIDE = 16 / E::SIZE;
    if (p.dim < WIDE) add ? launch_gradient<E, true, 1>(p, L, stream) : launch_gradient<E, false, 1>(p, L, stream);
    else add ? launch_gradient<E, true, WIDE>(p, L, stream) : launch_gradient<E, false, WIDE>(p, L, stream);
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
    const Rows written = rows_at(out, n_tokens, dim, out_stride, size_of(out_type));
    if (share(written, rows_at(table, vocab, dim, table_stride, size_of(table_type))) || share(written, bytes_at(tokens, n_tokens * token_bytes)))
        return GRAVAC_ERR_INVALID_ARG;
    (void)hipGetLastError();
    LookupParams p;
    p.table = table; p.tokens = tokens; p.out = out;
    p.vocab = vocab; p.table_stride = table_stride; p.n = n_tokens; p.out_stride = out_stride;
    p.dim = (int32_t)dim; p.wide = token_bytes == 8; p.lanes = 0; p.scale = scale;
    p.stream = n_tokens * dim * size_of(out_type) > STREAM_BYTES;
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
    const Rows written = rows_at(table_grad, vocab, dim, table_stride, 4), scratch = bytes_at(workspace, (int64_t)L.total);
    const Rows read[2] = {rows_at(grad_out, n_tokens, dim, grad_stride, size_of(grad_type)), bytes_at(tokens, n_tokens * token_bytes)};
    if (share(written, scratch) || share(written, read[0]) || share(written, read[1]) || share(scratch, read[0]) || share(scratch, read[1]))
        return GRAVAC_ERR_INVALID_ARG;
    (void)hipGetLastError();
    char* ws = (char*)workspace;
    GradParams p;
    p.grad = grad_out; p.tokens = tokens; p.table = table_grad;
    p.n = n_tokens; p.grad_stride = grad_stride; p.table_stride = table_stride;
    p.vocab = vocab; p.padding = padding_token;
    p.dim = (int32_t)dim; p.wide = token_bytes == 8;
    const bool add = (flags & GRAVAC_FLAG_ACCUMULATE) != 0;
    p.scale = scale;
    p.pairs[0] = (uint2*)(ws + L.pairs[0]); p.pairs[1] = (uint2*)(ws + L.pairs[1]);
    p.counts = (uint32_t*)(ws + L.counts); p.joins = (uint32_t*)(ws + L.joins);
    p.head = (float*)(ws + L.head); p.tail = (float*)(ws + L.tail);
    p.part_stride = L.part_stride; p.share_log = L.share_log; p.n_shares = L.n_shares;
    p.per_wg = 0; p.sort_wgs = 0; p.bits = 0; p.fill_rows = 0; p.fill_wgs = 0; p.fills = 0;
    p.stream = !add && 4 * vocab * dim > STREAM_BYTES;
    hipStream_t stream = (hipStream_t)stream_v;
    if (grad_type == GRAVAC_FLOAT32) launch_gradient<F32>(p, L, add, stream);
    else if (grad_type == GRAVAC_BFLOAT16) launch_gradient<BF16>(p, L, add, stream);
    else launch_gradient<F16>(p, L, add, stream);
    return hipGetLastError() == hipSuccess ? GRAVAC_OK : GRAVAC_ERR_HIP;
}

}  // extern "C"
