// orthogonal.hip - the nearest orthogonal factor of matrices by Newton-Schulz products, and the update of parameters along
// it (the step of Alg. 1 with a momentum whose singular values have been made equal, in place of plain SGD).
//
// A matrix U is taken in its wide form X (m x n, m <= n), divided by its Frobenius norm, and goes through
//     A = X X^T,   P = b A + c A A,   X <- a X + P X
// which maps every singular value s to a s + b s^3 + c s^5 and leaves the singular vectors.  All three products are of
// matrix-core kind and bound the call; A and P are symmetric, so half of their tiles are computed and written twice.
//
// Numbers.  Operands are binary16, sums binary32.  A matrix of float32 or float16 (or of parameters of that type) is cut into
// two binary16 parts, x = hi + lo, 22 bits, and a product is hi hi + hi lo + lo hi: as exact as products in binary32 (the
// dropped lo lo is 2^-22 of the product), at three matrix instructions in place of the sixteen times slower binary32 ones.
// For bfloat16 the products take hi alone, 11 bits, which costs less than the result's rounding to 8 bits.  Three things keep their rounding (2^-12 relative) from growing
// with the steps, which multiply a small singular value by a each: the term a X is taken in binary32 from hi + lo;
// the diagonals of A and P, far larger than the rest, are kept in binary32 outside the products,
//     A = D + E:  A A = E E + (d_i + d_j) e_ij + [i = j] d_i^2,      P = D' + Q:  X <- (a + d'_i) x_i + Q X;
// and every operand is scaled by a power of two so that typical entries lie near 1 and the largest one possible below 65504.
//
// Memory.  Every product is of the form C = L R^T with rows of L and R contiguous along the sum: X is kept as X and as X^T,
// both written by the product that makes them.  Rows and columns are padded with zeros to whole tiles, so the products have
// no edges.

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

constexpr int T = 128;             // rows and columns of a tile
constexpr int SLAB = 128;          // bytes of an operand's row that are in LDS at a time: 32 elements as hi and lo, or 64 hi
constexpr int MAX_MAT = GRAVAC_MAX_MATRICES;
constexpr int MAX_PARTS = 1024;    // partial sums of a matrix's norm at most
constexpr int PART = 16384;        // elements of one
constexpr int PER_INIT = 48;       // matrices of one launch of the table kernel (its argument holds them)
constexpr int CUT = 64;            // side of a tile of the kernel that cuts a matrix into operands

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
    float sx, sa, sq;                 // powers of two: X, E and Q are stored multiplied by them
    int64_t x, xt[2], lo, e, q, da, dq;   // byte offsets in the workspace
};

struct Tile { uint32_t mat; uint16_t i, j; };

__host__ __device__ inline int64_t padded(int64_t x) { return (x + T - 1) / T * T; }
__host__ __device__ inline int64_t aligned(int64_t x) { return (x + 255) & ~(int64_t)255; }

// 2^round(log2(x)) up to 2^most
__host__ __device__ inline float power_of_two(double x, int most)
{
    int e = 0;
    while (e < most && x > 1.41421356) { x *= 0.5; ++e; }
    return (float)(1u << e);
}

// Lays out a matrix's part of the workspace; returns its size.
__host__ __device__ inline int64_t lay_out(Mat& d, int64_t rows, int64_t cols, int64_t base, bool split)
{
    d.rows = (int32_t)rows; d.cols = (int32_t)cols;
    d.tall = rows > cols;
    d.m = (int32_t)(d.tall ? cols : rows); d.n = (int32_t)(d.tall ? rows : cols);
    d.mp = (int32_t)padded(d.m); d.np = (int32_t)padded(d.n);
    const int64_t el = split ? 4 : 2, xb = aligned(el * d.mp * d.np), ab = aligned(el * d.mp * d.mp);
    int64_t at = base;
    d.x = at; at += xb;
    d.xt[0] = at; at += xb;
    d.xt[1] = at; at += xb;
    d.lo = at; at += split ? 0 : xb;
    d.e = at; at += ab;
    d.q = at; at += ab;
    d.da = at; at += aligned(4 * (int64_t)d.mp);
    d.dq = at; at += aligned(4 * (int64_t)d.mp);
    // entries of X are at most 3.9, those of A at most 3.9^2 and those of P at most 15 (the host has checked the coefficients)
    d.sx = power_of_two(sqrt((double)d.m * (double)d.n), 14);
    d.sa = power_of_two((double)d.m, 12);
    d.sq = power_of_two((double)d.m, 12);
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
    int32_t n, first, split;
    MatIn mat[PER_INIT];
};
static_assert(sizeof(InitArgs) + sizeof(Call) <= 4096 - 64, "kernel arguments");

// One workgroup per matrix: its entry, and its lines in the tables of tiles and partial sums.
__global__ __launch_bounds__(256) void table_kernel(Call p, InitArgs a)
{
    const MatIn& g = a.mat[blockIdx.x];
    const uint32_t id = (uint32_t)(a.first + blockIdx.x);
    Mat d;
    lay_out(d, g.rows, g.cols, g.base, a.split != 0);
    d.offset = g.offset; d.stride = g.stride;
    d.cut = g.cut; d.part = g.part; d.parts = g.parts; d.scale = g.scale;
    if (threadIdx.x == 0) p.mats[id] = d;
    const uint32_t tm = (uint32_t)d.mp / T, tn = (uint32_t)d.np / T;
    for (uint32_t i = threadIdx.x; i < tm * tm; i += 256) {
        const uint32_t r = i / tm, c = i % tm;
        if (c > r) continue;
        const Tile t = {id, (uint16_t)r, (uint16_t)c};
        p.tiles[0][g.tile[0] + r * (r + 1) / 2 + c] = t;
        p.tiles[1][g.tile[1] + r * (r + 1) / 2 + c] = t;
    }
    for (uint32_t i = threadIdx.x; i < tn * tm; i += 256)
        p.tiles[2][g.tile[2] + i] = {id, (uint16_t)(i / tm), (uint16_t)(i % tm)};
    const uint32_t cuts = (uint32_t)(d.mp / CUT) * (uint32_t)(d.np / CUT);
    for (uint32_t i = threadIdx.x; i < cuts; i += 256) p.cut_of[g.cut + i] = id;
    for (uint32_t i = threadIdx.x; i < g.parts; i += 256) p.part_of[g.part + i] = id;
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

// The matrix's entry that is orthogonalised.  UPDATE: along the momentum (or along the gradient and the momentum).
template <typename E, bool UPDATE>
__device__ __forceinline__ float entry(const Call& p, int64_t at)
{
    if (!UPDATE) return to_float<E>(((const typename E::word*)p.in)[at]);
    const float m = p.momentum[at];
    return p.nesterov ? p.grad[at] + p.beta * m : m;
}

// Squares of a share of a matrix's entries, in binary64: no entry is too large or too small for them.  UPDATE: the momentum
// moves on first.
template <typename E, bool UPDATE>
__global__ __launch_bounds__(256) void norm_kernel(Call p)
{
    __shared__ double lds[4];
    const Mat& d = p.mats[p.part_of[blockIdx.x]];
    const uint32_t part = blockIdx.x - d.part;
    const int64_t n = (int64_t)d.rows * d.cols;
    const int64_t share = (n + d.parts - 1) / d.parts, begin = part * share, end = begin + share < n ? begin + share : n;
    double sum = 0.0;
    for (int64_t i = begin + threadIdx.x; i < end; i += 256) {
        int64_t at = i;
        if (d.stride != d.cols) at = i / d.cols * d.stride + i % d.cols;
        at += d.offset;
        if (UPDATE) p.momentum[at] = p.beta * p.momentum[at] + p.grad[at];
        const double x = (double)entry<E, UPDATE>(p, at);
        sum += x * x;
    }
    sum = sum_256(sum, lds);
    if (threadIdx.x == 0) p.parts[blockIdx.x] = sum;
}

__device__ __forceinline__ void cut_in_two(float x, _Float16& hi, _Float16& lo)
{
    hi = (_Float16)x;
    lo = (_Float16)(x - (float)hi);
}

// Where element k of a row lies: in two parts, 32 hi and their 32 lo in turn.
template <bool SPLIT>
__device__ __forceinline__ int64_t place(int64_t row, int64_t width, int64_t k)
{
    return SPLIT ? row * width * 2 + (k >> 5) * 64 + (k & 31) : row * width + k;
}

// X and X^T as operands, from the matrix over its norm; zeros in the padding.
template <typename E, bool UPDATE, bool SPLIT>
__global__ __launch_bounds__(256) void cut_kernel(Call p)
{
    __shared__ double lds[4];
    __shared__ float buf[CUT][CUT + 1];
    const uint32_t id = p.cut_of[blockIdx.x];
    const Mat& d = p.mats[id];
    double square = 0.0;
    for (uint32_t i = threadIdx.x; i < d.parts; i += 256) square += p.parts[d.part + i];
    square = sum_256(square, lds);
    const double norm = sqrt(square) + p.eps;
    const double inv = norm > 0.0 ? (double)d.sx / norm : (norm == 0.0 ? 0.0 : norm);
    const uint32_t local = blockIdx.x - d.cut;
    const int across = d.np / CUT;
    const int i0 = (int)(local / across) * CUT, j0 = (int)(local % across) * CUT;   // in X
    const int r0 = d.tall ? j0 : i0, c0 = d.tall ? i0 : j0;                         // in the matrix
    for (int e = threadIdx.x; e < CUT * CUT; e += 256) {
        const int r = e / CUT, c = e % CUT;
        float x = 0.0f;
        if (r0 + r < d.rows && c0 + c < d.cols)
            x = (float)((double)entry<E, UPDATE>(p, d.offset + (int64_t)(r0 + r) * d.stride + c0 + c) * inv);
        buf[r][c] = x;
    }
    __syncthreads();
    _Float16 *x = (_Float16*)(p.ws + d.x), *xt = (_Float16*)(p.ws + d.xt[0]), *lo = (_Float16*)(p.ws + d.lo);
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
        const int64_t at = second ? place<SPLIT>(j0 + row, d.mp, i0 + k) : place<SPLIT>(i0 + row, d.np, j0 + k);
        *(half8*)((second ? xt : x) + at) = h;
        if (SPLIT) *(half8*)((second ? xt : x) + at + 32) = l;
        else if (second) *(half8*)(lo + at) = l;
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------------------------------------------------

enum Product { GRAM, POLY, NEXT, LAST };   // A; P; X of the next step; X of the last one, into the caller's buffers

// C = L R^T on tiles of 128 x 128, four wavefronts of 64 x 64.  An operand's tile is 128 rows of SLAB bytes in LDS, fetched
// there without passing through registers; the 16-byte chunks of a row are stored in an order turned by the row, so that
// the lanes that read one chunk of eight consecutive rows touch all banks.
template <Product PRODUCT, bool SPLIT, typename E, bool UPDATE>
__global__ __launch_bounds__(256, 2) void product_kernel(Call p)
{
    __shared__ __attribute__((aligned(16))) char lds[2][2][T * SLAB];
    const Tile t = p.tiles[PRODUCT == GRAM ? 0 : PRODUCT == POLY ? 1 : 2][blockIdx.x];
    const Mat& d = p.mats[t.mat];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int mp = d.mp, width = PRODUCT == GRAM ? d.np : mp;   // length of the sums
    const int64_t left = PRODUCT == GRAM ? d.x : PRODUCT == POLY ? d.e : d.xt[p.flip];
    const int64_t right = PRODUCT == GRAM ? d.x : PRODUCT == POLY ? d.e : d.q;
    const int64_t row_bytes = (int64_t)width * (SPLIT ? 4 : 2);
    const int slabs = (int)(row_bytes / SLAB);

    // a wavefront fetches 32 rows of each operand, eight with one instruction: lane l fetches for row l / 8 the chunk whose
    // place is l % 8
    const int fetch_row = lane >> 3, fetch_chunk = (lane & 7) ^ (fetch_row & 7);
    const char* from[2];
    from[0] = p.ws + left + (int64_t)(t.i * T + w * 32 + fetch_row) * row_bytes + fetch_chunk * 16;
    from[1] = p.ws + right + (int64_t)(t.j * T + w * 32 + fetch_row) * row_bytes + fetch_chunk * 16;
    auto fetch = [&](int slab, int buffer) {
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void*)(from[o] + (int64_t)slab * SLAB + q * 8 * row_bytes),
                    (__attribute__((address_space(3))) void*)(&lds[buffer][o][(w * 32 + q * 8) * SLAB]), 16, 0, 0);
    };
    const int wi = (w >> 1) * 64, wj = (w & 1) * 64;
    const int frag_row = lane & 31, frag_half = lane >> 5;
    auto fragment = [&](int buffer, int o, int row0, int chunk) {
        const int row = row0 + frag_row;
        return *(const half8*)&lds[buffer][o][row * SLAB + ((chunk + frag_half) ^ (row & 7)) * 16];
    };
    float16v acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;

    fetch(0, 0);
    for (int s = 0; s < slabs; ++s) {
        __syncthreads();   // this slab has arrived, and every wavefront is done with the one before
        half8 l[2][4], r[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                l[i][k] = fragment(s & 1, 0, wi + i * 32, k * 2);
                r[i][k] = fragment(s & 1, 1, wj + i * 32, k * 2);
            }
        if (s + 1 < slabs) fetch(s + 1, (s + 1) & 1);
        if (SPLIT) {
            // chunks 0 - 3 are hi, 4 - 7 lo: two steps of 16
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][k], r[j][k + 2], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][k + 2], r[j][k], acc[i][j], 0, 0, 0);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][k], r[j][k], acc[i][j], 0, 0, 0);
                    }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[i][k], r[j][k], acc[i][j], 0, 0, 0);
        }
    }

    // acc[i][j][4 g + q] of lane l is row 8 g + 4 (l / 32) + q, column l % 32 of its 32 x 32
    const float* da = (const float*)(p.ws + d.da);
    const float* dq = (const float*)(p.ws + d.dq);
#pragma unroll
    for (int ti = 0; ti < 2; ++ti)
#pragma unroll
        for (int tj = 0; tj < 2; ++tj)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int row = t.i * T + wi + ti * 32 + g * 8 + frag_half * 4;   // and the three behind it
                const int col = t.j * T + wj + tj * 32 + frag_row;
                float v[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] = acc[ti][tj][g * 4 + q];
                if (PRODUCT == GRAM || PRODUCT == POLY) {
                    // symmetric: (row, col) is written at (col, row), and at (row, col) too if that is another tile
                    _Float16* to = (_Float16*)(p.ws + (PRODUCT == GRAM ? d.e : d.q));
                    const int64_t at = place<SPLIT>(col, mp, row);
                    if (PRODUCT == GRAM) {
                        const float f = d.sa / (d.sx * d.sx);
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            v[q] *= f;
                            if (row + q == col) {
                                ((float*)(p.ws + d.da))[col] = v[q] / d.sa;
                                v[q] = 0.0f;
                            }
                        }
                    } else {
                        const _Float16* e = (const _Float16*)(p.ws + d.e);
                        const half4 eh = *(const half4*)(e + at);
                        half4 el = {0, 0, 0, 0};
                        if (SPLIT) el = *(const half4*)(e + at + 32);
                        const float dj = da[col], sa = 1.0f / d.sa;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float di = da[row + q], eij = ((float)eh[q] + (float)el[q]) * sa;
                            float aa = v[q] * (sa * sa) + (di + dj) * eij;
                            if (row + q == col) {
                                aa += di * di;
                                ((float*)(p.ws + d.dq))[col] = p.b * di + p.c * aa;
                                v[q] = 0.0f;
                            } else {
                                v[q] = (p.b * eij + p.c * aa) * d.sq;
                            }
                        }
                    }
                    half4 h, l;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        _Float16 hi, lo;
                        cut_in_two(v[q], hi, lo);
                        h[q] = hi; l[q] = lo;
                    }
                    *(half4*)(to + at) = h;
                    if (SPLIT) *(half4*)(to + at + 32) = l;
                    if (t.i != t.j) {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int64_t other = place<SPLIT>(row + q, mp, col);
                            to[other] = h[q];
                            if (SPLIT) to[other + 32] = l[q];
                        }
                    }
                } else {
                    // row: along n, col: along m
                    const _Float16* xt = (const _Float16*)(p.ws + d.xt[p.flip]);
                    const float f = p.a + dq[col], sq = 1.0f / d.sq;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int64_t at = place<SPLIT>(row + q, mp, col);
                        const float lo = (float)(SPLIT ? xt[at + 32] : ((const _Float16*)(p.ws + d.lo))[at]);
                        v[q] = f * ((float)xt[at] + lo) + v[q] * sq;
                    }
                    if (PRODUCT == NEXT) {
                        _Float16* x = (_Float16*)(p.ws + d.x);
                        _Float16* next = (_Float16*)(p.ws + d.xt[1 - p.flip]);
                        half4 h, l;
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            _Float16 hi, lo;
                            cut_in_two(v[q], hi, lo);
                            h[q] = hi; l[q] = lo;
                            const int64_t at = place<SPLIT>(row + q, mp, col);
                            next[at] = hi;
                            if (SPLIT) next[at + 32] = lo;
                            else ((_Float16*)(p.ws + d.lo))[at] = lo;
                        }
                        const int64_t at = place<SPLIT>(col, d.np, row);
                        *(half4*)(x + at) = h;
                        if (SPLIT) *(half4*)(x + at + 32) = l;
                    } else if (col < d.m) {
                        const float sx = 1.0f / d.sx, step = p.alpha * d.scale;
                        typename E::word* out = (typename E::word*)p.out + d.offset;
                        const int64_t along = d.tall ? d.stride : 1;
                        int64_t at = d.tall ? (int64_t)row * d.stride + col : (int64_t)col * d.stride + row;
#pragma unroll
                        for (int q = 0; q < 4; ++q, at += along) {
                            if (row + q >= d.n) break;
                            float o = v[q] * sx;
                            if (UPDATE) {
                                o = step * o;
                                o = p.keep * to_float<E>(out[at]) + o;
                            }
                            out[at] = from_float<E>(o);
                        }
                    }
                }
            }
}

// ---------------------------------------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------------------------------------

constexpr int64_t MAX_SIDE = 1 << 20, MAX_SMALL_SIDE = 32768, MAX_FLAT = 1LL << 40;
constexpr uint64_t MAX_TILES = 1u << 24;

struct Layout {
    uint64_t tiles[3], cuts, parts;
    int64_t mats, tile_at[3], part_sums, cut_of, part_of, data, total;
};

int parts_of(int64_t rows, int64_t cols)
{
    const int64_t n = (rows * cols + PART - 1) / PART;
    return (int)(n < MAX_PARTS ? n : MAX_PARTS);
}

// matrices: {offset, rows, cols, stride} each.
bool lay_out_all(const int64_t* matrices, int n_mat, bool split, Layout& L)
{
    std::memset(&L, 0, sizeof(L));
    int64_t data = 0;
    for (int i = 0; i < n_mat; ++i) {
        const int64_t rows = matrices[4 * i + 1], cols = matrices[4 * i + 2], stride = matrices[4 * i + 3];
        if (rows < 1 || cols < 1 || rows > MAX_SIDE || cols > MAX_SIDE || stride < cols || stride > MAX_FLAT) return false;
        if (rows > MAX_SMALL_SIDE && cols > MAX_SMALL_SIDE) return false;
        Mat d;
        data += lay_out(d, rows, cols, 0, split);
        const uint64_t tm = d.mp / T, tn = d.np / T;
        L.tiles[0] += tm * (tm + 1) / 2; L.tiles[1] += tm * (tm + 1) / 2; L.tiles[2] += tm * tn;
        L.cuts += (uint64_t)(d.mp / CUT) * (uint64_t)(d.np / CUT);
        L.parts += parts_of(rows, cols);
        if (L.tiles[0] > MAX_TILES || L.tiles[2] > MAX_TILES || L.cuts > MAX_TILES) return false;
    }
    int64_t at = 0;
    auto take = [&](int64_t bytes) { const int64_t here = at; at += aligned(bytes); return here; };
    L.mats = take(sizeof(Mat) * (int64_t)n_mat);
    for (int k = 0; k < 3; ++k) L.tile_at[k] = take(sizeof(Tile) * (int64_t)L.tiles[k]);
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
    bool ascending = true;
    for (int i = 0; i < n_mat; ++i) {
        if (matrices[4 * i] < 0 || matrices[4 * i] > n || end(i) > n) return false;
        if (i > 0 && matrices[4 * i] < end(i - 1)) ascending = false;
    }
    if (ascending) return true;
    for (int i = 0; i < n_mat; ++i)
        for (int k = 0; k < i; ++k) {
            const int64_t *a = matrices + 4 * i, *b = matrices + 4 * k;
            if (a[0] >= end(k) || b[0] >= end(i)) continue;
            // spans that overlap: only columns of one larger matrix lie apart (equal strides, and no columns in common)
            if (a[3] != b[3]) return false;
            const int64_t s = a[3], d = ((b[0] - a[0]) % s + s) % s;   // b's first column, counted from a's
            if (d < a[2] || d + b[2] > s) return false;
        }
    return true;
}

constexpr double MOST_X = 3.9, MOST_P = 15.0;   // times the scales in lay_out: below 65504

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
        if (c != 0.0) {
            const double disc = 9.0 * b * b - 20.0 * a * c;
            if (disc >= 0.0) {
                look((-3.0 * b + std::sqrt(disc)) / (10.0 * c), false);
                look((-3.0 * b - std::sqrt(disc)) / (10.0 * c), false);
            }
            look(-b / (2.0 * c), true);
        } else if (b != 0.0) {
            look(-a / (3.0 * b), false);
        }
        if (!(most <= MOST_X) || !(p <= MOST_P)) return false;
        u = most > 1e-3 ? most : 1e-3;
    }
    return true;
}

constexpr double QUINTIC[3] = {3.4445, -4.7750, 2.0315};

template <typename E, bool UPDATE, bool SPLIT>
int run(Call& p, const Layout& L, const int64_t* matrices, const float* scales, int n_mat, int steps, const double* coefficients,
        hipStream_t stream)
{
    // long sums first: their tiles take longest, and short ones fill the gaps at the end
    uint16_t by_m[MAX_MAT], by_n[MAX_MAT];
    for (int i = 0; i < n_mat; ++i) by_m[i] = by_n[i] = (uint16_t)i;
    auto small = [&](int i) { return std::min(matrices[4 * i + 1], matrices[4 * i + 2]); };
    auto large = [&](int i) { return std::max(matrices[4 * i + 1], matrices[4 * i + 2]); };
    std::sort(by_m, by_m + n_mat, [&](int a, int b) { return small(a) != small(b) ? small(a) > small(b) : a < b; });
    std::sort(by_n, by_n + n_mat, [&](int a, int b) { return large(a) != large(b) ? large(a) > large(b) : a < b; });
    uint32_t tile[3][MAX_MAT], at[3] = {0, 0, 0};
    for (int q = 0; q < n_mat; ++q) {
        const uint32_t n0 = (uint32_t)(padded(small(by_n[q])) / T);
        tile[0][by_n[q]] = at[0]; at[0] += n0 * (n0 + 1) / 2;
        const uint32_t m0 = (uint32_t)(padded(small(by_m[q])) / T), m1 = (uint32_t)(padded(large(by_m[q])) / T);
        tile[1][by_m[q]] = at[1]; at[1] += m0 * (m0 + 1) / 2;
        tile[2][by_m[q]] = at[2]; at[2] += m0 * m1;
    }
    int64_t base = L.data;
    uint32_t cut = 0, part = 0;
    for (int first = 0; first < n_mat; first += PER_INIT) {
        InitArgs a;
        std::memset(&a, 0, sizeof(a));
        a.first = first; a.n = std::min(PER_INIT, n_mat - first); a.split = SPLIT;
        for (int k = 0; k < a.n; ++k) {
            const int i = first + k;
            MatIn& g = a.mat[k];
            g.offset = matrices[4 * i]; g.rows = (int32_t)matrices[4 * i + 1]; g.cols = (int32_t)matrices[4 * i + 2];
            g.stride = matrices[4 * i + 3];
            for (int s = 0; s < 3; ++s) g.tile[s] = tile[s][i];
            Mat d;
            g.base = base; base += lay_out(d, g.rows, g.cols, base, SPLIT);
            g.cut = cut; cut += (uint32_t)(d.mp / CUT) * (uint32_t)(d.np / CUT);
            g.part = part; g.parts = (uint32_t)parts_of(g.rows, g.cols); part += g.parts;
            g.scale = scales ? scales[i] : 1.0f;
        }
        hipLaunchKernelGGL(table_kernel, dim3((uint32_t)a.n), dim3(256), 0, stream, p, a);
    }
    hipLaunchKernelGGL((norm_kernel<E, UPDATE>), dim3((uint32_t)L.parts), dim3(256), 0, stream, p);
    hipLaunchKernelGGL((cut_kernel<E, UPDATE, SPLIT>), dim3((uint32_t)L.cuts), dim3(256), 0, stream, p);
    for (int k = 0; k < steps; ++k) {
        const double* c = coefficients ? coefficients + 3 * k : QUINTIC;
        p.a = (float)c[0]; p.b = (float)c[1]; p.c = (float)c[2];
        p.flip = k & 1;
        hipLaunchKernelGGL((product_kernel<GRAM, SPLIT, F32, false>), dim3((uint32_t)L.tiles[0]), dim3(256), 0, stream, p);
        hipLaunchKernelGGL((product_kernel<POLY, SPLIT, F32, false>), dim3((uint32_t)L.tiles[1]), dim3(256), 0, stream, p);
        if (k + 1 < steps)
            hipLaunchKernelGGL((product_kernel<NEXT, SPLIT, F32, false>), dim3((uint32_t)L.tiles[2]), dim3(256), 0, stream, p);
        else
            hipLaunchKernelGGL((product_kernel<LAST, SPLIT, E, UPDATE>), dim3((uint32_t)L.tiles[2]), dim3(256), 0, stream, p);
    }
    return hipGetLastError() == hipSuccess ? GRAVAC_OK : GRAVAC_ERR_HIP;
}

bool in_two_parts(int type) { return type != GRAVAC_BFLOAT16; }

// What both entry points check, and the parts of the call that are the same.
int begin(Call& p, Layout& L, const int64_t* matrices, int n_mat, int type, int64_t n, int steps, const double* coefficients,
          double eps, void* workspace, size_t workspace_bytes)
{
    if (!known(type) || !matrices || n_mat < 1 || n_mat > MAX_MAT || n < 1 || n > MAX_FLAT) return GRAVAC_ERR_INVALID_ARG;
    if (steps < 1 || steps > GRAVAC_MAX_STEPS || !(eps >= 0.0) || std::isinf(eps)) return GRAVAC_ERR_INVALID_ARG;
    if (coefficients && !bounded(coefficients, steps)) return GRAVAC_ERR_INVALID_ARG;
    if (!lay_out_all(matrices, n_mat, in_two_parts(type), L) || !lie_apart(matrices, n_mat, n)) return GRAVAC_ERR_INVALID_ARG;
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

}  // namespace

extern "C" {

int gravac_orthogonalize_workspace_bytes(const int64_t* matrices, int n_mat, int type, size_t* bytes_out)
{
    Layout L;
    if (!bytes_out || !known(type) || !matrices || n_mat < 1 || n_mat > MAX_MAT ||
        !lay_out_all(matrices, n_mat, in_two_parts(type), L))
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
    p.in = in; p.out = out;
    hipStream_t stream = (hipStream_t)stream_v;
    if (type == GRAVAC_FLOAT32) return run<F32, false, true>(p, L, matrices, nullptr, n_mat, steps, coefficients, stream);
    if (type == GRAVAC_BFLOAT16) return run<BF16, false, false>(p, L, matrices, nullptr, n_mat, steps, coefficients, stream);
    return run<F16, false, true>(p, L, matrices, nullptr, n_mat, steps, coefficients, stream);
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
    p.grad = grad; p.momentum = momentum; p.out = params;
    p.beta = beta; p.keep = keep; p.alpha = alpha;
    p.nesterov = (flags & GRAVAC_FLAG_NESTEROV) ? 1 : 0;
    hipStream_t stream = (hipStream_t)stream_v;
    if (type == GRAVAC_FLOAT32) return run<F32, true, true>(p, L, matrices, scales, n_mat, steps, coefficients, stream);
    if (type == GRAVAC_BFLOAT16) return run<BF16, true, false>(p, L, matrices, scales, n_mat, steps, coefficients, stream);
    return run<F16, true, true>(p, L, matrices, scales, n_mat, steps, coefficients, stream);
}

}  // extern "C"
