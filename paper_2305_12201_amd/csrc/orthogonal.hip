// orthogonal.hip - the nearest orthogonal factor of matrices by Newton-Schulz products, and the update of parameters along
// it (the step of Alg. 1 with a momentum whose singular values have been made equal, in place of plain SGD).
//
// A matrix U is taken in its wide form X (m x n, m <= n), divided by its Frobenius norm, and goes through
//     A = X X^T,   P = b A + c A A,   X <- a X + P X
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.  All three products are of
// matrix-core kind and bound the call; A and P are symmetric, so half of their tiles are computed and written twice.
//
// Numbers.  Operands are binary16, sums binary32.  A matrix is cut into two binary16 parts, x = hi + lo, 22 bits, and a product
// is hi hi + hi lo + lo hi: as exact as products in binary32 (the dropped lo lo is 2^-22 of the product), at three matrix
// instructions in place of the sixteen times slower binary32 ones.  That holds for 16-bit matrices and parameters too, whose
// steps are as exact: with hi alone, 11 bits, a bfloat16 result is off by 6e-4 before its own rounding and one entry in
// five is not the nearest one, for a third of the matrix instructions.  Three things keep the operands' rounding from growing
// with the steps, which multiply a small singular value by a each: the term a X is taken in binary32 from hi + lo;
// the diagonals of A and P, far larger than the rest, are kept in binary32 outside the products,
//     A = D + E:  A A = E E + (d_i + d_j) e_ij + [i = j] d_i^2,      P = D' + Q:  X <- (a + d'_i) x_i + Q X;
// and X is stored times 2^14, E and Q times 2^12, so that the largest entries possible, which the host bounds, lie just below 65504.
// Of an entry of X below 2^-17 (one of E or Q below 2^-15) the lower part is a subnormal number of binary16: it is off by 2^-39 (2^-37)
// at most, no longer by 2^-22 of itself, and the steps that raise it raise that too.  (Powers of two that follow the matrix's size,
// with typical entries near 1, leave less: a 16 x 64 matrix with one row 10^5 times the others was off by 5.2e-4 after 10 steps
// and is by 1.0e-6.)
//
// Memory.  Every product is of the form C = L R^T with rows of L and R contiguous along the sum: X is kept as X and as X^T,
// both written by the product that makes them.  Rows and columns are padded with zeros to whole tiles, so the products have
// no edges; their sums end with the matrix (four 2600 x 650 in float32 took 511 us with sums over the padding, and 473).
//
// Measured, five steps, three products each: 4096 x 4096 in bfloat16 3.7 to 4.0 ms (1020 to 1110 TFLOP/s of matrix instructions; the
// clock gives way to power there: 1.7 GHz), the 16 matrices of the VGG16 shape in float32 21.8 to 22.4 ms (1100 to 1130), the 105 of
// ResNet101 1.74 to 1.87 ms, where X, of 178 MB, passes memory four times a step, 512 x 128 in bfloat16 93 us, 15 products one after
// the other at 4.6 to 6.5 us.

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstring>

#include "elements.h"
#include "gravac.h"

namespace {

using namespace elements;

typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef _Float16 half4 __attribute__((ext_vector_type(4)));
typedef float float16v __attribute__((ext_vector_type(16)));

constexpr int SLAB = 64;           // bytes of an operand's row that are fetched at a time: 16 elements as hi and lo
constexpr int PART_SLABS = 128;    // slabs of a sum that are added one after the other (tiles of 64 and 128)
constexpr int64_t LONG_SIDE = 32768;   // no tiles of 256 for longer sums
constexpr int BLOCK = 128;         // rows whose slabs stand together in memory
constexpr int MAX_MAT = GRAVAC_MAX_MATRICES;
constexpr int MAX_PARTS = 1024;    // partial sums of a matrix's norm at most
constexpr int PART = 16384;        // bytes of one in the matrix's type, at least
constexpr int PER_INIT = 48;       // matrices of one launch of the table kernel (its argument holds them)
constexpr int CUT = 64;            // side of a tile of the kernel that cuts a matrix into operands

constexpr int LOW = 16;            // from a hi to its lo

struct MatIn {   // what the host says of a matrix
    int64_t offset, stride, base;     // base: its part of the workspace
    int32_t rows, cols;
    uint32_t tile[3];                 // its first tile in the tables of the three products
    uint32_t cut, part, parts;        // its first tile of the cutting kernel, its first partial sum, their number
    float scale;
    int32_t pad;
};

struct Mat {     // ... and what the kernels read
    int64_t offset, stride;
    int32_t rows, cols, m, n, mp, np, tall;
    uint32_t cut, part, parts;
    float scale;
    int32_t pad;
    int64_t x, xt0, xt1, e, q, da, dq;   // byte offsets in the workspace
};

struct Tile { uint32_t mat; uint16_t i, j; };
constexpr uint32_t NO_MAT = 0xFFFFFFFFu;

// Workgroups go to the eight dies, each with an L2 of its own, in turn.  A product's tiles are listed matrix by matrix, and
// each die gets one stretch of the list, of about an eighth of the work: its tiles share their operands' rows.  A table has
// room for the longest stretch on every die.
constexpr int DIES = 8;
struct Stretches { uint32_t begin[DIES + 1], longest; };

__host__ __device__ inline int64_t padded(int64_t x, int tile) { return (x + tile - 1) / tile * tile; }
__host__ __device__ inline int64_t aligned(int64_t x) { return (x + 255) & ~(int64_t)255; }

// What operands are stored multiplied by: entries of X are at most 3.9, those of A at most 3.9^2 and those of P at most 15 (the host
// has checked the coefficients).
constexpr float SX = 16384.0f, SA = 4096.0f, SQ = 4096.0f;

// Lays out a matrix's part of the workspace; returns its size.
__host__ __device__ inline int64_t lay_out(Mat& d, int64_t rows, int64_t cols, int64_t base, int tile)
{
    d.rows = (int32_t)rows; d.cols = (int32_t)cols;
    d.tall = rows > cols;
    d.m = (int32_t)(d.tall ? cols : rows); d.n = (int32_t)(d.tall ? rows : cols);
    d.mp = (int32_t)padded(d.m, tile); d.np = (int32_t)padded(d.n, tile);
    // (the rows of an operand stand in blocks)
    const int64_t el = 4, mb = padded(d.mp, BLOCK), nb = padded(d.np, BLOCK);
    const int64_t xb = aligned(el * mb * d.np), tb = aligned(el * nb * d.mp), ab = aligned(el * mb * d.mp);
    int64_t at = base;
    d.x = at; at += xb;
    d.xt0 = at; at += tb;
    d.xt1 = at; at += tb;
    d.e = at; at += ab;
    d.q = at; at += ab;
    d.da = at; at += aligned(4 * (int64_t)d.mp);
    d.dq = at; at += aligned(4 * (int64_t)d.mp);
    return at - base;
}

struct Call {
    char* ws;
    Mat* mats;
    Tile* tiles[3];
    double* parts;       // partial sums of the norms
    uint32_t* cut_of;    // matrix of a tile of the cutting kernel
    uint32_t* part_of;   // matrix of a partial sum
    const void* in;      // gravac_orthogonalize
    const float* grad;   // gravac_orthogonal_update
    float* momentum;
    void* out;
    float beta, keep, alpha;
    int32_t nesterov;
    double eps;
    float a, b, c;
    int32_t flip;        // which X^T buffer is read
};

// ---------------------------------------------------------------------------------------------------------------------
// tables, norms, operands
// ---------------------------------------------------------------------------------------------------------------------

struct InitArgs {
    int32_t n, first, tile, side[3];
    Stretches list[3];
    MatIn mat[PER_INIT];
};
static_assert(sizeof(InitArgs) + sizeof(Call) <= 4096 - 64, "kernel arguments");

__device__ inline uint32_t slot_of(const Stretches& s, uint32_t at)
{
    int die = 0;
    while (die + 1 < DIES && at >= s.begin[die + 1]) ++die;
    return (at - s.begin[die]) * DIES + die;
}

// A matrix's tiles are listed in bands of BAND rows, column by column, so that those next to each other in the list lie in
// a block about as high as it is wide.
constexpr uint32_t BAND = 8;

__device__ inline uint32_t place_in_triangle(uint32_t r, uint32_t c, uint32_t n)   // c <= r < n
{
    const uint32_t k = r / BAND * BAND, h = n - k < BAND ? n - k : BAND, before = k * (k + 1) / 2;
    if (c <= k) return before + c * h + (r - k);
    const uint32_t q = c - k;   // columns behind the band's first row: h, h - 1, ... tiles each
    return before + k * h + q * h - q * (q - 1) / 2 + (r - c);
}
__device__ inline uint32_t place_in_square(uint32_t r, uint32_t c, uint32_t rows, uint32_t cols)
{
    const uint32_t k = r / BAND * BAND, h = rows - k < BAND ? rows - k : BAND;
    return k * cols + c * h + (r - k);
}

// One workgroup per matrix: its entry, and its lines in the tables of tiles and partial sums.
__global__ __launch_bounds__(256) void table_kernel(Call p, InitArgs a)
{
    const MatIn& g = a.mat[blockIdx.x];
    const uint32_t id = (uint32_t)(a.first + blockIdx.x);
    Mat d;
    lay_out(d, g.rows, g.cols, g.base, a.tile);
    d.offset = g.offset; d.stride = g.stride;
    d.cut = g.cut; d.part = g.part; d.parts = g.parts; d.scale = g.scale;
    if (threadIdx.x == 0) p.mats[id] = d;
    for (int k = 0; k < 3; ++k) {
        const uint32_t tm = (uint32_t)(d.mp / a.side[k]), tn = k < 2 ? tm : (uint32_t)(d.np / a.side[k]);
        for (uint32_t i = threadIdx.x; i < tn * tm; i += 256) {
            const uint32_t r = i / tm, c = i % tm;
            if (k < 2 && c > r) continue;
            const uint32_t at = k < 2 ? place_in_triangle(r, c, tm) : place_in_square(r, c, tn, tm);
            p.tiles[k][slot_of(a.list[k], g.tile[k] + at)] = {id, (uint16_t)r, (uint16_t)c};
        }
    }
    const uint32_t cuts = (uint32_t)(d.mp / CUT) * (uint32_t)(d.np / CUT);
    for (uint32_t i = threadIdx.x; i < cuts; i += 256) p.cut_of[g.cut + i] = id;
    for (uint32_t i = threadIdx.x; i < g.parts; i += 256) p.part_of[g.part + i] = id;
    if (id == 0)   // the slots behind the shorter stretches
        for (int k = 0; k < 3; ++k)
            for (int die = 0; die < DIES; ++die)
                for (uint32_t i = a.list[k].begin[die + 1] - a.list[k].begin[die] + threadIdx.x; i < a.list[k].longest; i += 256)
                    p.tiles[k][i * DIES + die] = {NO_MAT, 0, 0};
}

// The sum over the workgroup's 256 threads, the same for all of them.
__device__ double sum_256(double x, double* lds)
{
    for (int d = 32; d > 0; d /= 2) x += __shfl_xor(x, d, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = x;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Up to four consecutive entries of what is orthogonalised (n of them; the rest is 0).  UPDATE: the momentum, or the gradient
// and the momentum.
template <typename E, bool UPDATE>
__device__ __forceinline__ void entries(const Call& p, int64_t at, int n, float (&x)[4])
{
    if (!UPDATE) {
        load_part<E, 4>((const typename E::word*)p.in + at, n, x);
        return;
    }
    load_part<F32, 4>((const uint32_t*)p.momentum + at, n, x);
    if (p.nesterov) {
        float g[4];
        load_part<F32, 4>((const uint32_t*)p.grad + at, n, g);
#pragma unroll
        for (int q = 0; q < 4; ++q) x[q] = g[q] + p.beta * x[q];
    }
}

// Squares of a share of a matrix's entries, in binary64: no entry is too large or too small for them.  UPDATE: the momentum
// moves on first.
template <typename E, bool UPDATE>
__global__ __launch_bounds__(256) void norm_kernel(Call p)
{
    __shared__ double lds[4];
    const Mat& d = p.mats[p.part_of[blockIdx.x]];
    const uint32_t part = blockIdx.x - d.part;
    // rows that lie one behind the other are one long row
    const bool whole = d.stride == d.cols;
    const int64_t length = whole ? (int64_t)d.rows * d.cols : d.cols, pieces = (length + 3) / 4;   // of four entries, per row
    const int64_t n = whole ? pieces : pieces * d.rows;
    const int64_t share = (n + d.parts - 1) / d.parts, begin = part * share, end = begin + share < n ? begin + share : n;
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
        const int64_t row = whole ? 0 : i / pieces, c = (i - row * pieces) * 4, at = d.offset + row * d.stride + c;
        const int have = length - c < 4 ? (int)(length - c) : 4;
        float x[4];
        if (UPDATE) {
            float g[4];
            load_part<F32, 4>((const uint32_t*)p.momentum + at, have, x);
            load_part<F32, 4>((const uint32_t*)p.grad + at, have, g);
#pragma unroll
            for (int q = 0; q < 4; ++q) x[q] = p.beta * x[q] + g[q];
            store_part<F32, 4>((uint32_t*)p.momentum + at, have, x);
            if (p.nesterov)
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = g[q] + p.beta * x[q];
        } else {
            load_part<E, 4>((const typename E::word*)p.in + at, have, x);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) sum += (double)x[q] * (double)x[q];
    }
    sum = sum_256(sum, lds);
    if (threadIdx.x == 0) p.parts[blockIdx.x] = sum;
}

__device__ __forceinline__ void cut_in_two(float x, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)x;
    lo = (_Float16)(x - (float)hi);
}

// Where element k of a row of an operand lies, in binary16 elements: the slabs of 128 rows stand one behind the other, so
// what a product fetches at a time is contiguous.  A row of a slab is 16 hi and their 16 lo.  `width`: elements of a row.
__device__ __forceinline__ int64_t place(int row, int width, int k)
{
    return ((int64_t)(row >> 7) * (width >> 4) + (k >> 4)) * (BLOCK * 32) + (row & (BLOCK - 1)) * 32 + (k & 15);
}

// X and X^T as operands, from the matrix over its norm; zeros in the padding.
template <typename E, bool UPDATE>
__global__ __launch_bounds__(256) void cut_kernel(Call p)
{
    __shared__ double lds[4];
    __shared__ float buf[CUT][CUT + 1];
    const uint32_t id = p.cut_of[blockIdx.x];
    const Mat& d = p.mats[id];
    double square = 0.0;
    for (uint32_t i = threadIdx.x; i < d.parts; i += 256) square += p.parts[d.part + i];
    square = sum_256(square, lds);
    // (zeros stay zeros whatever eps is; the inverse of one below 10^-304 is infinite)
    const double inv = square > 0.0 ? (double)SX / (sqrt(square) + p.eps) : square;
    const uint32_t local = blockIdx.x - d.cut;
    const int across = d.np / CUT;
    const int i0 = (int)(local / across) * CUT, j0 = (int)(local % across) * CUT;   // in X
    const int r0 = d.tall ? j0 : i0, c0 = d.tall ? i0 : j0;                         // in the matrix
#pragma unroll
    for (int k = 0; k < CUT * CUT / 1024; ++k) {
        const int e = k * 1024 + (int)threadIdx.x * 4, r = e / CUT, c = e % CUT;
        float x[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r0 + r < d.rows && c0 + c < d.cols)
            entries<E, UPDATE>(p, d.offset + (int64_t)(r0 + r) * d.stride + c0 + c, d.cols - c0 - c, x);
#pragma unroll
        for (int q = 0; q < 4; ++q) buf[r][c + q] = (float)((double)x[q] * inv);
    }
    __syncthreads();
    _Float16 *x = (_Float16*)(p.ws + d.x), *xt = (_Float16*)(p.ws + d.xt0);
    for (int e = threadIdx.x; e < 2 * CUT * CUT / 8; e += 256) {
        const bool second = e >= CUT * CUT / 8;                    // X^T
        const int row = (e & (CUT * CUT / 8 - 1)) / (CUT / 8), k = (e % (CUT / 8)) * 8;
        half8 h, l;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const bool swap = (d.tall != 0) != second;
            const float v = swap ? buf[k + q][row] : buf[row][k + q];
            _Float16 hi, low;
            cut_in_two(v, hi, low);
            h[q] = hi; l[q] = low;
        }
        const int64_t at = second ? place(j0 + row, d.mp, i0 + k) : place(i0 + row, d.np, j0 + k);
        *(half8*)((second ? xt : x) + at) = h;
        *(half8*)((second ? xt : x) + at + LOW) = l;
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------------------------------------

// A value that is the same in all lanes, in scalar registers.
template <typename S>
__device__ __forceinline__ S uniform(S x)
{
    static_assert(sizeof(S) % 4 == 0, "whole words");
    uint32_t words[sizeof(S) / 4];
    __builtin_memcpy(words, &x, sizeof(S));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(S) / 4); ++i) words[i] = (uint32_t)__builtin_amdgcn_readfirstlane((int)words[i]);
    __builtin_memcpy(&x, words, sizeof(S));
    return x;
}

enum Product { GRAM, POLY, NEXT, LAST };   // A; P; X of the next step; X of the last one, into the caller's buffers

// Sixteen rows of a slab from global memory into LDS without a register in between, 16 bytes per lane; AT is added to both
// addresses.  The LDS address is the wavefront's.  The compiler does not count these loads (arrived() does).  M0 is among the
// registers that it keeps for itself, so it takes no clobber of it: it writes M0 right before those of its own instructions that
// read it, of which there are none here (the kernels' assembly names M0 in this statement alone).
template <int AT>
__device__ __forceinline__ void fetch_16(const char* base, uint32_t offset, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" :: "s"(lds), "v"(offset), "s"(base), "n"(AT) : "memory");
}

// Waits until at most N of the wavefront's loads are under way, then for the workgroup's other wavefronts.
template <int N>
__device__ __forceinline__ void arrived()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" :: "n"(N) : "memory");
}

__device__ __forceinline__ void cut_8(const float (&v)[8], half8& h, half8& l)
{
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        _Float16 hi, lo;
        cut_in_two(v[q], hi, lo);
        h[q] = hi; l[q] = lo;
    }
}

// Entry number `at` of eight, if there is one, made zero: the diagonal's of a block on it.
__device__ __forceinline__ float take_diagonal(float (&v)[8], bool on_diagonal, int at)
{
    float x = 0.0f;
    if (on_diagonal) {   // the same for the wavefront
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            x = q == at ? v[q] : x;
            v[q] = q == at ? 0.0f : v[q];
        }
    }
    return x;
}

// C = L R^T on tiles of 64 F x 64 F (F = 1, 2, 4), four wavefronts of 32 F x 32 F.  A slab of an operand is 64 F rows of SLAB
// bytes in LDS; the 16-byte chunks of a row are stored in an order turned by the row, so that the lanes that read one chunk of eight
// consecutive rows touch all banks.  While a slab is multiplied from registers, the next is read from LDS into others and
// those behind it are on their way from memory, BUFFERS - 2 of them.
template <Product PRODUCT, typename E, bool UPDATE, int F, int BUFFERS>
__global__ __launch_bounds__(256, F == 4 || (F == 2 && BUFFERS > 4) ? 1 : 2) void product_kernel(Call p)
{
    constexpr int T = 64 * F, LOADS = 2 * F;              // a wavefront's loads per slab
    constexpr int SIDE = F == 1 ? 32 : 64;                // the epilogue goes through LDS in blocks of SIDE x SIDE
    constexpr int SLABS_BYTES = BUFFERS * 2 * T * SLAB, EPILOGUE_BYTES = 4 * SIDE * SIDE * 4;
    __shared__ __attribute__((aligned(1024))) char lds[SLABS_BYTES > EPILOGUE_BYTES ? SLABS_BYTES : EPILOGUE_BYTES];
    const Tile t = uniform(p.tiles[PRODUCT == GRAM ? 0 : PRODUCT == POLY ? 1 : 2][blockIdx.x]);
    if (t.mat == NO_MAT) return;
    const Mat d = uniform(p.mats[t.mat]);
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mp = d.mp, width = PRODUCT == GRAM ? d.np : mp;   // elements of an operand's row
    const int64_t left = PRODUCT == GRAM ? d.x : PRODUCT == POLY ? d.e : p.flip ? d.xt1 : d.xt0;
    const int64_t right = PRODUCT == GRAM ? d.x : PRODUCT == POLY ? d.e : d.q;
    // slabs of a sum, an even number of them (rows hold whole ones: sides are padded to 64 or more); the padding behind is left out
    const int slabs = (int)padded(PRODUCT == GRAM ? d.n : d.m, 32) / 16;

    // a wavefront fetches 16 F rows of each operand, sixteen with one instruction: lane l fetches for row l / 4 the chunk
    // whose place is l % 4
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
    const uint32_t fetch_at = (uint32_t)((lane >> 2) * SLAB + ((lane & 3) ^ ((lane >> 4) & 3)) * 16);
    const char* from_left = uniform(p.ws + left + 2 * place(t.i * T + w * 16 * F, width, 0));
    const char* from_right = uniform(p.ws + right + 2 * place(t.j * T + w * 16 * F, width, 0));
    const uint32_t fetch_to = lds0 + (uint32_t)(w * 16 * F) * SLAB;
    // load number `q` of a slab's 2 F (behind the last slab: of that one again, so that as many are always under way)
    auto fetch = [&](int slab, int q) {
        const int64_t at = (int64_t)(slab < slabs ? slab : slabs - 1) * (BLOCK * SLAB);
        const uint32_t to = fetch_to + (uint32_t)((slab & (BUFFERS - 1)) * 2 * T * SLAB);
        constexpr int ROWS = 16 * SLAB;
        if (q == 0) fetch_16<0>(from_left + at, fetch_at, to);
        if (F > 1 && q == 1) fetch_16<ROWS>(from_left + at, fetch_at, to);
        if (F == 4 && q == 2) fetch_16<2 * ROWS>(from_left + at, fetch_at, to);
        if (F == 4 && q == 3) fetch_16<3 * ROWS>(from_left + at, fetch_at, to);
        if (q == F) fetch_16<0>(from_right + at, fetch_at, to + T * SLAB);
        if (F > 1 && q == F + 1) fetch_16<ROWS>(from_right + at, fetch_at, to + T * SLAB);
        if (F == 4 && q == F + 2) fetch_16<2 * ROWS>(from_right + at, fetch_at, to + T * SLAB);
        if (F == 4 && q == F + 3) fetch_16<3 * ROWS>(from_right + at, fetch_at, to + T * SLAB);
    };
    const int wi = (w >> 1) * 32 * F, wj = (w & 1) * 32 * F;
    const int frag_row = lane & 31, frag_half = lane >> 5;
    // a slab's fragments: hi and lo of 32 rows by 16 elements each
    half8 l[2][2][F], r[2][2][F];
    const int chunk0 = (frag_half ^ ((frag_row >> 2) & 3)) * 16, chunk1 = chunk0 ^ 32;
    // fragment number `q` of a slab's 4 F, in the order of their use
    auto read = [&](int slab, int set, int q) {
        const char* at = lds + (slab & (BUFFERS - 1)) * 2 * T * SLAB + frag_row * SLAB;
        const int h = q / (2 * F), i = q % F, o = q / F % 2;
        const int part = o ? 1 - h : h;      // the first product takes hi of the left and lo of the right
        const char* from = at + (part ? chunk1 : chunk0) + (o ? T + wj + i * 32 : wi + i * 32) * SLAB;
        if (o) r[set][part][i] = *(const half8*)from;
        else l[set][part][i] = *(const half8*)from;
    };
    float16v acc[F][F];
#pragma unroll
    for (int i = 0; i < F; ++i)
#pragma unroll
        for (int j = 0; j < F; ++j)
#pragma unroll
            for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.0f;

    static_assert((BUFFERS & (BUFFERS - 1)) == 0 && BUFFERS >= 4, "slabs in turn");
    for (int s = 0; s < BUFFERS - 1; ++s)
#pragma unroll
        for (int q = 0; q < 2 * F; ++q) fetch(s, q);
    arrived<(BUFFERS - 2) * LOADS>();
#pragma unroll
    for (int q = 0; q < 4 * F; ++q) read(0, 0, q);
    // The matrix instructions of a slab, with what brings in the others between them: a wavefront is alone on its SIMD, so
    // what stands between two blocks of matrix instructions would leave the matrix core idle (in one block each, it was
    // busy 61 % of the time).
    constexpr int PRODUCTS = 3, INSTS = PRODUCTS * F * F, ITEMS = 6 * F;
    // A long sum is added up in parts: added one after the other, 70,001 elements of float32 are off by 16 times what the
    // plain evaluation's nested sums are.  There are no registers for that with tiles of 256, which sums beyond LONG_SIDE do not get:
    // 32,768 elements added one after the other are off by twice to three times what nested sums are, random ones and ones of one
    // sign (1024 x 20,011 2.0e-6 and 3.6e-6, a nested evaluation in binary32 1.4e-6 and 1.6e-6).
    constexpr bool PARTS = F <= 2;
    float16v sums[PARTS ? F : 1][PARTS ? F : 1];
    auto add_up = [&](bool first) {
#pragma unroll
        for (int i = 0; i < (PARTS ? F : 0); ++i)
#pragma unroll
            for (int j = 0; j < F; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) {
                    sums[i][j][q] = first ? acc[i][j][q] : sums[i][j][q] + acc[i][j][q];
                    acc[i][j][q] = 0.0f;
                }
    };
    for (int s0 = 0; s0 < slabs; s0 += 2) {
        if (PARTS && s0 % PART_SLABS == 0 && s0 > 0) add_up(s0 == PART_SLABS);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int s = s0 + u;
            // slab s + 1 has arrived, those behind it may be on their way, and every wavefront is done with slab s - 1
            arrived<(BUFFERS - 3) * LOADS>();
#pragma unroll
            for (int m = 0; m < INSTS; ++m) {
#pragma unroll
                for (int q = m * ITEMS / INSTS; q < (m + 1) * ITEMS / INSTS; ++q) {
                    if (q % 3 == 0) fetch(s + BUFFERS - 1, q / 3);
                    else read(s + 1, 1 - u, q - q / 3 - 1);
                }
                const int k = m / (F * F), i = m / F % F, j = m % F;
                const int a = k == 1 ? 1 : 0, b = k == 0 ? 1 : 0;
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[u][a][i], r[u][b][j], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
    if (PARTS && slabs > PART_SLABS) {
        add_up(false);
#pragma unroll
        for (int i = 0; i < (PARTS ? F : 0); ++i)
#pragma unroll
            for (int j = 0; j < F; ++j) acc[i][j] = sums[i][j];
    }
    arrived<0>();   // nothing more comes, and the LDS of the slabs is free

    // A wavefront puts 64 x 64 of its sums at a time into LDS and reads them back eight along the left index at a time, for
    // the rest of the arithmetic with 16-byte accesses; what it writes along the right index goes through LDS once more.
    // Column j of the block holds its 16 groups of four rows in an order turned by j + 2 (j / 8): four rows of a column as
    // the matrix instructions leave them, eight rows of a column and eight columns of a row all touch the banks evenly.
    // (Four bytes at a time in rows of 65 the epilogue of X took 3.4 us for a 128 x 512 matrix of operands in one part, so 2.7.)
    float* block = (float*)lds + w * SIDE * SIDE;
    auto spot = [](int i, int j) { return j * SIDE + (((i >> 2) + j + 2 * (j >> 3)) & (SIDE / 4 - 1)) * 4 + (i & 3); };
    constexpr int BLOCKS = 32 * F / SIDE, EIGHTS = SIDE / 8, COLUMNS = 64 / EIGHTS;   // lanes: eights of a column, columns
    char* ws = p.ws;
#pragma unroll
    for (int bi = 0; bi < BLOCKS; ++bi)
#pragma unroll
        for (int bj = 0; bj < BLOCKS; ++bj) {
            const int i0 = t.i * T + wi + bi * SIDE, j0 = t.j * T + wj + bj * SIDE;
            // A symmetric matrix takes its upper half from the lower one, in units of 32 whatever the tiles are (the parts of a
            // product are added in another order on the other side): so the result depends on the tiles only where sums are folded,
            // beyond PART_SLABS slabs, and the tile is 256, which the other matrices of the call decide too.
            constexpr bool SYMMETRIC = PRODUCT == GRAM || PRODUCT == POLY;
            if (SYMMETRIC && i0 < j0) continue;
            const int part = (lane % EIGHTS) * 8, column = lane / EIGHTS, i = i0 + part;
            // what the sums meet in memory, all of it under way before the first is used
            constexpr int ROWS = SIDE / COLUMNS;
            half8 mh[ROWS], ml[ROWS];
            float mj[ROWS], mi[8];
            if (PRODUCT == POLY) {
                const _Float16* e = (const _Float16*)(ws + d.e);
                const float* da = (const float*)(ws + d.da);
#pragma unroll
                for (int q = 0; q < 8; ++q) mi[q] = da[i + q];
#pragma unroll
                for (int it = 0; it < ROWS; ++it) {
                    const int j = j0 + it * COLUMNS + column;
                    const int64_t at = place(j, mp, i);
                    mj[it] = da[j];
                    mh[it] = *(const half8*)(e + at);
                    ml[it] = *(const half8*)(e + at + LOW);
                }
            } else if (PRODUCT == NEXT || PRODUCT == LAST) {
                // i: along n, j: along m
                const _Float16* x = (const _Float16*)(ws + d.x);
                const float* dq = (const float*)(ws + d.dq);
#pragma unroll
                for (int it = 0; it < ROWS; ++it) {
                    const int j = j0 + it * COLUMNS + column;
                    const int64_t at = place(j, d.np, i);
                    mj[it] = p.a + dq[j];
                    mh[it] = *(const half8*)(x + at);
                    ml[it] = *(const half8*)(x + at + LOW);
                }
            }
            // acc[4 g + q] of lane l is row 8 g + 4 (l / 32) + q, column l % 32 of its 32 x 32
#pragma unroll
            for (int ti = 0; ti < SIDE / 32; ++ti)
#pragma unroll
                for (int tj = 0; tj < SIDE / 32; ++tj)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float16v& v = acc[bi * (SIDE / 32) + ti][bj * (SIDE / 32) + tj];
                        if (SYMMETRIC && SIDE > 32 && ti != tj && i0 == j0) {
                            if (ti < tj) continue;
#pragma unroll
                            for (int q = 0; q < 4; ++q) block[spot(tj * 32 + frag_row, ti * 32 + g * 8 + frag_half * 4 + q)] = v[g * 4 + q];
                        }
                        *(float4*)&block[spot(ti * 32 + g * 8 + frag_half * 4, tj * 32 + frag_row)] =
                            make_float4(v[g * 4], v[g * 4 + 1], v[g * 4 + 2], v[g * 4 + 3]);
                    }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            bool other;   // whether the other orientation is wanted
            if (SYMMETRIC) other = i0 != j0;
            else if (PRODUCT == NEXT) other = true;
            else other = d.tall;
#pragma unroll
            for (int it = 0; it < ROWS; ++it) {
                const int jj = it * COLUMNS + column, j = j0 + jj;
                float4* mine[2] = {(float4*)&block[spot(part, jj)], (float4*)&block[spot(part + 4, jj)]};
                const float4 low = *mine[0], high = *mine[1];
                float v[8] = {low.x, low.y, low.z, low.w, high.x, high.y, high.z, high.w};
                half8 h, l;
                if (PRODUCT == GRAM) {
                    constexpr float f = SA / (SX * SX);
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] *= f;
                    const float ajj = take_diagonal(v, i0 == j0, j - i);
                    if (i0 == j0 && (unsigned)(j - i) < 8) ((float*)(ws + d.da))[j] = ajj * (1.0f / SA);
                } else if (PRODUCT == POLY) {
                    constexpr float sa = 1.0f / SA;
                    const float dj = mj[it];
#pragma unroll
                    for (int q = 0; q < 8; ++q) {
                        const float eij = ((float)mh[it][q] + (float)ml[it][q]) * sa;
                        v[q] = (p.b * eij + p.c * (v[q] * (sa * sa) + (mi[q] + dj) * eij)) * SQ;
                    }
                    const float pjj = take_diagonal(v, i0 == j0, j - i);   // (e_jj = 0: c times the sum)
                    if (i0 == j0 && (unsigned)(j - i) < 8) ((float*)(ws + d.dq))[j] = p.b * dj + p.c * dj * dj + pjj * (1.0f / SQ);
                } else {
                    constexpr float sq = 1.0f / SQ;
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = mj[it] * ((float)mh[it][q] + (float)ml[it][q]) + v[q] * sq;
                }
                if (PRODUCT != LAST) {
                    cut_8(v, h, l);
                    const int64_t at = place(j, PRODUCT == NEXT ? d.np : mp, i);
                    _Float16* to = (_Float16*)(ws + (PRODUCT == GRAM ? d.e : PRODUCT == POLY ? d.q : d.x));
                    *(half8*)(to + at) = h;
                    *(half8*)(to + at + LOW) = l;
                } else {
                    constexpr float sx = 1.0f / SX;
                    const float step = p.alpha * d.scale;
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = UPDATE ? step * (v[q] * sx) : v[q] * sx;
                    if (!other && i < d.n && j < d.m) {
                        typename E::word* out = (typename E::word*)p.out + d.offset + (int64_t)j * d.stride + i;
                        if (UPDATE) {
                            float old[8];
                            load_part<E, 8>(out, d.n - i, old);
#pragma unroll
                            for (int q = 0; q < 8; ++q) v[q] = p.keep * old[q] + v[q];
                        }
                        store_part<E, 8>(out, d.n - i, v);
                    }
                }
                if (other) {
                    *mine[0] = make_float4(v[0], v[1], v[2], v[3]);
                    *mine[1] = make_float4(v[4], v[5], v[6], v[7]);
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (other) {
#pragma unroll
                for (int it = 0; it < ROWS; ++it) {
                    const int ii = it * COLUMNS + column, i = i0 + ii, j = j0 + part;
                    float v[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = block[spot(ii, part + q)];
                    if (PRODUCT == LAST) {
                        if (i < d.n && j < d.m) {
                            typename E::word* out = (typename E::word*)p.out + d.offset + (int64_t)i * d.stride + j;
                            if (UPDATE) {
                                float old[8];
                                load_part<E, 8>(out, d.m - j, old);
#pragma unroll
                                for (int q = 0; q < 8; ++q) v[q] = p.keep * old[q] + v[q];
                            }
                            store_part<E, 8>(out, d.m - j, v);
                        }
                    } else {
                        half8 h, l;
                        cut_8(v, h, l);
                        const int64_t at = place(i, mp, j);
                        _Float16* to = (_Float16*)(ws + (PRODUCT == GRAM ? d.e : PRODUCT == POLY ? d.q : p.flip ? d.xt0 : d.xt1));
                        *(half8*)(to + at) = h;
                        *(half8*)(to + at + LOW) = l;
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------

constexpr int64_t MAX_SIDE = 1 << 20, MAX_SMALL_SIDE = 32768, MAX_FLAT = 1LL << 40;
constexpr uint64_t MAX_TILES = (1u << 24) - 8;   // (256 threads each: the grid has 32 bits)

struct Layout {
    int tile;            // sides are padded to whole tiles of it: the largest of the three
    int side[3];         // of a tile of A, P and X
    Stretches list[3];   // of the products' tiles
    uint32_t first[3][MAX_MAT];   // a matrix's first tile in them
    uint64_t cuts, parts;
    int64_t mats, tile_at[3], part_sums, cut_of, part_of, data, total;
};

int parts_of(int64_t rows, int64_t cols, int type)
{
    const int64_t n = (rows * cols * size_of(type) + PART - 1) / PART;
    return (int)(n < MAX_PARTS ? n : MAX_PARTS);
}

int64_t small_side(const int64_t* matrix) { return std::min(matrix[1], matrix[2]); }
int64_t large_side(const int64_t* matrix) { return std::max(matrix[1], matrix[2]); }

// Side of the products' tiles.  Tiles of 256 need half the LDS traffic, but there are a quarter as many and more of them is
// padding: they pay where A has tiles for half of the compute units, from matrices of four or more a side that are most of the
// work.  Measured in us with tiles of 128 and of 256, five steps in float32: 2560 x 5120 1899 and 2796 (55 tiles of A), twelve
// 1024 x 1024 998 and 1205 (120), four 2048 x 2048 2311 and 2314 (144), 4096 x 4096 4196 and 4039 (136), twelve 1500 x 3000 4765 and
// 4639 (252), twenty-four 1024 x 4096 5874 and 5443 (240), three 4096 x 11008 26.2 and 23.7 ms (408).  It is blind to sides just
// beyond a multiple of 256, whose padding makes it lose: nine 1025 x 2100 1590 and 2114 (135).
int tile_of(const int64_t* matrices, int n_mat)
{
    double all = 0.0, large = 0.0, tiles = 0.0;
    for (int i = 0; i < n_mat; ++i) {
        const int64_t *matrix = matrices + 4 * i;
        const double m = (double)small_side(matrix), n = (double)large_side(matrix), side = std::ceil(m / 256);
        all += m * m * n;
        if (large_side(matrix) > LONG_SIDE) return 128;
        if (side < 4) continue;
        large += m * m * n;
        tiles += side * (side + 1) / 2;
    }
    return tiles >= 128 && large >= 0.75 * all ? 256 : 128;
}

// A product's tiles (0: A, 1: P, 2: X) if they have this side and sides are padded to `pad`.
uint64_t tiles_of(const int64_t* matrix, int k, int64_t side, int64_t pad)
{
    const uint64_t m = (uint64_t)(padded(small_side(matrix), (int)pad) / side), n = (uint64_t)(padded(large_side(matrix), (int)pad) / side);
    return k < 2 ? m * (m + 1) / 2 : m * n;
}

// Tiles of 64 where those of 128 would be few: they bring more compute units to work and their epilogues are short.  us for five
// steps in float32 with A, P and X in tiles of 128 / A in 64 / A and P / all: 512 x 512 233, 201, 163, 132; 1024 x 1024 341, 293,
// 236, 196; four 2600 x 650 (84 tiles of 128 of A and P, 504 of X) 587, 520, 493, 510; 1536 x 1536 (78, 144) 465, 443, 405, 433;
// 2048 x 2048 (136, 256) 712, 736, 754, 811; four 1024 x 1024 (144, 256) 450, 457, 460, 492.  P alone in 64: 465 -> 437 with 78 tiles,
// 782 -> 778 with 288 (eight 1024 x 1024), 1740 -> 1742 with 405 (the ResNet101 shape), 960 -> 1004 with 504 (twenty-four 768 x 768).
// Twelve 300 x 900 are 258 with X in 128 and 217 in 64 for the padding.
// P among tiles of 256 takes 128 where a last round of those would leave more units idle: VGG16 shape 22.5 -> 21.9 ms, sixteen
// 2048 x 2048 8.27 -> 8.06, nine 1025 x 2100 2.11 -> 1.96.  (0.93: where all units are busy either way,
// tiles of 128 are 3 to 10 % slower, as the figures above say.)
void choose_sides(const int64_t* matrices, int n_mat, Layout& L)
{
    const int tile = tile_of(matrices, n_mat);
    auto count = [&](int k, int side) {
        double n = 0.0;
        for (int i = 0; i < n_mat; ++i) n += (double)tiles_of(matrices + 4 * i, k, side, tile == 256 ? 256 : side);
        return n;
    };
    L.tile = tile;
    L.side[0] = L.side[1] = L.side[2] = tile;
    if (tile == 256) {
        auto busy = [](double tiles, double at_once) { return tiles / (at_once * std::ceil(tiles / at_once)); };
        if (0.93 * busy(count(1, 128), 512.0) > busy(count(1, 256), 256.0)) L.side[1] = 128;
        return;
    }
    const double square = count(0, 128), whole = count(2, 128);
    if (square <= 128) L.side[0] = 64;
    if (square <= 512) L.side[1] = 64;
    if (whole <= 128 || (L.side[0] == 64 && 4.0 * whole > 1.2 * count(2, 64))) L.side[2] = 64;
    L.tile = std::max(std::max(L.side[0], L.side[1]), L.side[2]);
}

// The list of a product's tiles (0: A, 1: P, 2: X) and its stretches; false if there are too many.  Long sums come first: their
// tiles take longest, and a die that has several lengths fills the gaps at the end with short ones.
bool list_tiles(const int64_t* matrices, int n_mat, int k, Layout& L)
{
    uint16_t order[MAX_MAT];
    for (int i = 0; i < n_mat; ++i) order[i] = (uint16_t)i;
    auto length = [&](int i) { return k == 0 ? large_side(matrices + 4 * i) : small_side(matrices + 4 * i); };
    std::sort(order, order + n_mat, [&](int a, int b) { return length(a) != length(b) ? length(a) > length(b) : a < b; });
    auto tiles = [&](int i) {
        return tiles_of(matrices + 4 * i, k, L.side[k], L.tile);
    };
    auto work = [&](int i) { return (double)(length(i) + 256); };   // of a tile: its sum, and its begin and end
    uint64_t count = 0;
    double all = 0.0;
    for (int q = 0; q < n_mat; ++q) {
        L.first[k][order[q]] = (uint32_t)count;
        count += tiles(order[q]);
        all += (double)tiles(order[q]) * work(order[q]);
        if (count > MAX_TILES) return false;
    }
    Stretches& s = L.list[k];
    s.begin[0] = 0;
    int die = 1;
    double done = 0.0;
    for (int q = 0; q < n_mat; ++q) {
        const double here = (double)tiles(order[q]) * work(order[q]);
        for (; die < DIES && done + here >= all * die / DIES; ++die)
            s.begin[die] = L.first[k][order[q]] + (uint32_t)std::min((double)tiles(order[q]), std::round((all * die / DIES - done) / work(order[q])));
        done += here;
    }
    for (; die <= DIES; ++die) s.begin[die] = (uint32_t)count;
    s.longest = 0;
    for (int d = 0; d < DIES; ++d) s.longest = std::max(s.longest, s.begin[d + 1] - s.begin[d]);
    return s.longest <= MAX_TILES / DIES;
}

// matrices: {offset, rows, cols, stride} each.
bool lay_out_all(const int64_t* matrices, int n_mat, int type, Layout& L)
{
    L.cuts = L.parts = 0;
    int64_t data = 0;
    for (int i = 0; i < n_mat; ++i) {
        const int64_t rows = matrices[4 * i + 1], cols = matrices[4 * i + 2], stride = matrices[4 * i + 3];
        if (rows < 1 || cols < 1 || rows > MAX_SIDE || cols > MAX_SIDE || stride < cols || stride > MAX_FLAT) return false;
        if (rows > MAX_SMALL_SIDE && cols > MAX_SMALL_SIDE) return false;
    }
    choose_sides(matrices, n_mat, L);
    for (int k = 0; k < 3; ++k)
        if (!list_tiles(matrices, n_mat, k, L)) return false;
    for (int i = 0; i < n_mat; ++i) {
        Mat d;
        data += lay_out(d, matrices[4 * i + 1], matrices[4 * i + 2], 0, L.tile);
        L.cuts += (uint64_t)(d.mp / CUT) * (uint64_t)(d.np / CUT);
        L.parts += parts_of(matrices[4 * i + 1], matrices[4 * i + 2], type);
        if (L.cuts > MAX_TILES) return false;
    }
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += aligned(bytes); return here; };
    L.mats = take(sizeof(Mat) * (int64_t)n_mat);
    for (int k = 0; k < 3; ++k) L.tile_at[k] = take(sizeof(Tile) * DIES * (int64_t)L.list[k].longest);
    L.part_sums = take(8 * (int64_t)L.parts);
    L.cut_of = take(4 * (int64_t)L.cuts);
    L.part_of = take(4 * (int64_t)L.parts);
    L.data = at;
    L.total = at + data;
    return true;
}

// Whether the matrices of a table lie inside [0, n) and no two of them share an element.
bool lie_apart(const int64_t* matrices, int n_mat, int64_t n)
{
    auto end = [&](int i) { return matrices[4 * i] + (matrices[4 * i + 1] - 1) * matrices[4 * i + 3] + matrices[4 * i + 2]; };
    uint16_t order[MAX_MAT];
    for (int i = 0; i < n_mat; ++i) {
        order[i] = (uint16_t)i;
        if (matrices[4 * i] < 0 || matrices[4 * i] > n || end(i) > n) return false;
    }
    std::sort(order, order + n_mat, [&](int a, int b) { return matrices[4 * a] < matrices[4 * b]; });
    for (int i = 0; i < n_mat; ++i)
        for (int k = i + 1; k < n_mat && matrices[4 * order[k]] < end(order[i]); ++k) {
            const int64_t *a = matrices + 4 * order[i], *b = matrices + 4 * order[k];
            if (share({a[0], a[1], a[2], a[3]}, {b[0], b[1], b[2], b[3]})) return false;
        }
    return true;
}

constexpr double MOST_X = 3.9, MOST_P = 15.0;   // times SX, its square times SA, and times SQ: below 65504

// Coefficients of a step, as numbers that binary16 operands can hold through all steps: with |s| <= u before a step, the
// largest |a s + b s^3 + c s^5| and the largest |b l + c l^2|, l = s^2, follow from the ends and the extrema.
bool bounded(const double* coefficients, int steps)
{
    double u = 1.0;
    for (int k = 0; k < steps; ++k) {
        const double a = coefficients[3 * k], b = coefficients[3 * k + 1], c = coefficients[3 * k + 2];
        if (!std::isfinite(a) || !std::isfinite(b) || !std::isfinite(c) || std::fabs(a) > 1e3 || std::fabs(b) > 1e3 || std::fabs(c) > 1e3)
            return false;
        auto f = [&](double l) { return std::sqrt(l) * std::fabs(a + l * (b + l * c)); };
        auto g = [&](double l) { return std::fabs(l * (b + l * c)); };
        const double top = u * u;
        double most = f(top), p = g(top);
        auto look = [&](double l, bool poly) {
            if (l > 0.0 && l < top) { if (poly) p = std::max(p, g(l)); else most = std::max(most, f(l)); }
        };
        // a + 3 b l + 5 c l^2 = 0; the sum that does not cancel gives one root, the product of both the other (also with c = 0)
        const double disc = 9.0 * b * b - 20.0 * a * c;
        if (disc >= 0.0) {
            const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(disc), b));
            if (c != 0.0) look(q / (5.0 * c), false);
            if (q != 0.0) look(a / q, false);
        }
        if (c != 0.0) look(-b / (2.0 * c), true);
        if (!(most <= MOST_X) || !(p <= MOST_P)) return false;
        u = most > 1e-3 ? most : 1e-3;
    }
    return true;
}

constexpr double QUINTIC[3] = {3.4445, -4.7750, 2.0315};

// Tiles of 128: two workgroups on a compute unit, one of which multiplies while the other starts or ends; A, whose sums are the
// longest, has fewer tiles and takes one with twice the slabs under way (ResNet101 shape: 140 -> 97 us).
template <Product PRODUCT, typename E, bool UPDATE>
void launch_product(const Call& p, const Layout& L, hipStream_t stream)
{
    constexpr int K = PRODUCT == GRAM ? 0 : PRODUCT == POLY ? 1 : 2;
    const dim3 grid(DIES * L.list[K].longest);
    if (L.side[K] == 256) hipLaunchKernelGGL((product_kernel<PRODUCT, E, UPDATE, 4, 4>), grid, dim3(256), 0, stream, p);
    else if (L.side[K] == 128) hipLaunchKernelGGL((product_kernel<PRODUCT, E, UPDATE, 2, PRODUCT == GRAM ? 8 : 4>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((product_kernel<PRODUCT, E, UPDATE, 1, 8>), grid, dim3(256), 0, stream, p);
}

template <typename E, bool UPDATE>
void launch_products(Call& p, const Layout& L, int steps, const double* coefficients, hipStream_t stream)
{
    for (int k = 0; k < steps; ++k) {
        const double* c = coefficients ? coefficients + 3 * k : QUINTIC;
        p.a = (float)c[0]; p.b = (float)c[1]; p.c = (float)c[2];
        p.flip = k & 1;
        launch_product<GRAM, F32, false>(p, L, stream);
        launch_product<POLY, F32, false>(p, L, stream);
        if (k + 1 < steps) launch_product<NEXT, F32, false>(p, L, stream);
        else launch_product<LAST, E, UPDATE>(p, L, stream);
    }
}

template <typename E, bool UPDATE>
int run(Call& p, const Layout& L, const int64_t* matrices, const float* scales, int n_mat, int type, int steps, const double* coefficients,
        hipStream_t stream)
{
    int64_t base = L.data;
    uint32_t cut = 0, part = 0;
    for (int first = 0; first < n_mat; first += PER_INIT) {
        InitArgs a;
        std::memset(&a, 0, sizeof(a));
        a.first = first; a.n = std::min(PER_INIT, n_mat - first); a.tile = L.tile;
        for (int s = 0; s < 3; ++s) a.side[s] = L.side[s];
        for (int s = 0; s < 3; ++s) a.list[s] = L.list[s];
        for (int k = 0; k < a.n; ++k) {
            const int i = first + k;
            MatIn& g = a.mat[k];
            g.offset = matrices[4 * i]; g.rows = (int32_t)matrices[4 * i + 1]; g.cols = (int32_t)matrices[4 * i + 2];
            g.stride = matrices[4 * i + 3];
            for (int s = 0; s < 3; ++s) g.tile[s] = L.first[s][i];
            Mat d;
            g.base = base; base += lay_out(d, g.rows, g.cols, base, L.tile);
            g.cut = cut; cut += (uint32_t)(d.mp / CUT) * (uint32_t)(d.np / CUT);
            g.part = part; g.parts = (uint32_t)parts_of(g.rows, g.cols, type); part += g.parts;
            g.scale = scales ? scales[i] : 1.0f;
        }
        hipLaunchKernelGGL(table_kernel, dim3((uint32_t)a.n), dim3(256), 0, stream, p, a);
    }
    hipLaunchKernelGGL((norm_kernel<E, UPDATE>), dim3((uint32_t)L.parts), dim3(256), 0, stream, p);
    hipLaunchKernelGGL((cut_kernel<E, UPDATE>), dim3((uint32_t)L.cuts), dim3(256), 0, stream, p);
    launch_products<E, UPDATE>(p, L, steps, coefficients, stream);
    return hipGetLastError() == hipSuccess ? GRAVAC_OK : GRAVAC_ERR_HIP;
}

// What both entry points check, and the parts of the call that are the same.
int begin(Call& p, Layout& L, const int64_t* matrices, int n_mat, int type, int64_t n, int steps, const double* coefficients,
          double eps, void* workspace, size_t workspace_bytes)
{
    if (!known(type) || !matrices || n_mat < 1 || n_mat > MAX_MAT || n < 1 || n > MAX_FLAT) return GRAVAC_ERR_INVALID_ARG;
    if (steps < 1 || steps > GRAVAC_MAX_STEPS || !(eps >= 0.0) || std::isinf(eps)) return GRAVAC_ERR_INVALID_ARG;
    if (coefficients && !bounded(coefficients, steps)) return GRAVAC_ERR_INVALID_ARG;
    if (!lay_out_all(matrices, n_mat, type, L) || !lie_apart(matrices, n_mat, n)) return GRAVAC_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < (size_t)L.total) return GRAVAC_ERR_WORKSPACE;
    std::memset(&p, 0, sizeof(p));
    p.ws = (char*)workspace;
    p.mats = (Mat*)(p.ws + L.mats);
    for (int k = 0; k < 3; ++k) p.tiles[k] = (Tile*)(p.ws + L.tile_at[k]);
    p.parts = (double*)(p.ws + L.part_sums);
    p.cut_of = (uint32_t*)(p.ws + L.cut_of);
    p.part_of = (uint32_t*)(p.ws + L.part_of);
    p.eps = eps;
    (void)hipGetLastError();
    return GRAVAC_OK;
}

bool misaligned(const void* p, int size) { return ((uintptr_t)p & (uintptr_t)(size - 1)) != 0; }

bool overlap(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) { return share(bytes_at(a, a_bytes), bytes_at(b, b_bytes)); }

}  // namespace

extern "C" {

int gravac_orthogonalize_workspace_bytes(const int64_t* matrices, int n_mat, int type, size_t* bytes_out)
{
    Layout L;
    if (!bytes_out || !known(type) || !matrices || n_mat < 1 || n_mat > MAX_MAT ||
        !lay_out_all(matrices, n_mat, type, L))
        return GRAVAC_ERR_INVALID_ARG;
    *bytes_out = (size_t)L.total;
    return GRAVAC_OK;
}

int gravac_orthogonalize(const void* in, void* out, int type, int64_t n, const int64_t* matrices, int n_mat, int steps,
                         const double* coefficients, double eps, void* workspace, size_t workspace_bytes, void* stream_v)
{
    if (!known(type) || !in || !out || misaligned(in, size_of(type)) || misaligned(out, size_of(type))) return GRAVAC_ERR_INVALID_ARG;
    Call p;
    Layout L;
    if (const int rc = begin(p, L, matrices, n_mat, type, n, steps, coefficients, eps, workspace, workspace_bytes)) return rc;
    const int64_t bytes = n * size_of(type);
    if ((in != out && overlap(in, bytes, out, bytes)) || overlap(workspace, L.total, in, bytes) || overlap(workspace, L.total, out, bytes))
        return GRAVAC_ERR_INVALID_ARG;
    p.in = in; p.out = out;
    hipStream_t stream = (hipStream_t)stream_v;
    if (type == GRAVAC_FLOAT32) return run<F32, false>(p, L, matrices, nullptr, n_mat, type, steps, coefficients, stream);
    if (type == GRAVAC_BFLOAT16) return run<BF16, false>(p, L, matrices, nullptr, n_mat, type, steps, coefficients, stream);
    return run<F16, false>(p, L, matrices, nullptr, n_mat, type, steps, coefficients, stream);
}

int gravac_orthogonal_update(const float* grad, float* momentum, void* params, int type, int64_t n, const int64_t* matrices,
                             int n_mat, float beta, float keep, float alpha, const float* scales, int steps,
                             const double* coefficients, double eps, void* workspace, size_t workspace_bytes, unsigned flags,
                             void* stream_v)
{
    if (!known(type) || !grad || !momentum || !params || misaligned(grad, 4) || misaligned(momentum, 4) ||
        misaligned(params, size_of(type)) || (flags & ~GRAVAC_FLAG_NESTEROV))
        return GRAVAC_ERR_INVALID_ARG;
    Call p;
    Layout L;
    if (const int rc = begin(p, L, matrices, n_mat, type, n, steps, coefficients, eps, workspace, workspace_bytes)) return rc;
    if (overlap(grad, 4 * n, momentum, 4 * n) || overlap(grad, 4 * n, params, n * size_of(type)) ||
        overlap(momentum, 4 * n, params, n * size_of(type)) || overlap(workspace, L.total, grad, 4 * n) ||
        overlap(workspace, L.total, momentum, 4 * n) || overlap(workspace, L.total, params, n * size_of(type)))
        return GRAVAC_ERR_INVALID_ARG;
    p.grad = grad; p.momentum = momentum; p.out = params;
    p.beta = beta; p.keep = keep; p.alpha = alpha;
    p.nesterov = (flags & GRAVAC_FLAG_NESTEROV) ? 1 : 0;
    hipStream_t stream = (hipStream_t)stream_v;
    if (type == GRAVAC_FLOAT32) return run<F32, true>(p, L, matrices, scales, n_mat, type, steps, coefficients, stream);
    if (type == GRAVAC_BFLOAT16) return run<BF16, true>(p, L, matrices, scales, n_mat, type, steps, coefficients, stream);
    return run<F16, true>(p, L, matrices, scales, n_mat, type, steps, coefficients, stream);
}

}  // extern "C"
