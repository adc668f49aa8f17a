// Updates with their singular values brought towards one: X <- a X + (b S + c S^2) X with S = X X^T, an odd polynomial of the
// matrix that leaves its singular vectors alone and takes every singular value x to a x + b x^3 + c x^5, applied a few times to
// every matrix of a stack over its Frobenius norm.  With K <= C, S = X X^T and X <- P X for P = a + b S + c S^2; else S = X^T X and
// X <- X P: no matrix is transposed, the operands lie along or across the contraction as it comes (tile_product.h).
//
// Between the launches X, S and P are kept as pairs of fp16 (22 bits), each scaled by a power of two that keeps its largest possible
// entry below 2^15: a singular value of X is bounded by what the polynomial makes of [0, 1] (polynomial_bound), an entry by the
// largest singular value.  What a pair drops is below 2^-38 of that bound, or 2^-23 of the entry.  The polynomial multiplies small
// singular values by a (3.4445) a step, errors with them: sixteen bits or less would show in a result of bf16.  Against 64 bits, by the matrix's norm,
// the results are as near as those of products in fp32 or nearer (2048 x 1024: 4.0e-6 and 4.1e-6, 512 x 512: 2.2e-6 and 3.2e-6, 256 x 64:
// 1.5e-6 and 1.4e-6), and so are single rows down to 1e-4 of the others; a row at 1e-8 of them is off by 5 % of itself, where fp32 has 1e-5.
// Three bf16 parts would keep it, at twice the matrix instructions.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "tile_product.h"

namespace cadmm {

namespace {

using namespace tile;

constexpr int kNormBlocks = 256;       // most workgroups that add up one matrix's norm

// The direction of the update: the gradient, or what the momentum makes of it.
template <class T>
struct Source {
    const T* G; float* M; float mu; int nesterov;
    __device__ __forceinline__ float direction(float g, float m) const { return nesterov ? g + mu * m : m; }
    __device__ __forceinline__ float again(int64_t e) const { return M ? direction((float)G[e], M[e]) : (float)G[e]; }
};

// The sum of the squares of elements first, first + step, .. below count, with the momentum brought forward: sixteen loads are on their way
// before the first is used.
template <class T>
__device__ __forceinline__ double squares(const Source<T>& src, int64_t base, int64_t first, int64_t step, int64_t count) {
    constexpr int AHEAD = 8;
    double sum = 0.0;
    for (int64_t f = first; f < count; f += AHEAD * step) {
        float g[AHEAD], m[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int64_t e = base + (f + u * step < count ? f + u * step : first);
            g[u] = (float)src.G[e];
            m[u] = src.M ? src.M[e] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (f + u * step >= count) continue;
            float d = g[u];
            if (src.M) {
                const float now = src.mu * m[u] + g[u];
                src.M[base + f + u * step] = now;
                d = src.direction(g[u], now);
            }
            sum += (double)d * (double)d;
        }
    }
    return sum;
}

// over a workgroup; everybody gets it
template <int THREADS>
__device__ __forceinline__ double block_sum(double sum, double* shared) {
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.0;
    for (int i = 0; i < THREADS / 64; ++i) sum += shared[i];
    return sum;
}
// What the direction is multiplied by, from its sum of squares: nothing where there is no direction (it is zero), and an entry
// that is not finite leaves nothing finite.
__device__ __forceinline__ double normaliser(double sum, float eps, float scale) {
    const double norm = sqrt(sum) + (double)eps;
    return norm == 0.0 ? 0.0 : norm < HUGE_VAL ? (double)scale / norm : __builtin_nan("");
}

template <class T>
__global__ __launch_bounds__(256) void orthogonal_norm_kernel(Source<T> src, int64_t count, double* __restrict__ norms) {
    __shared__ double shared[4];
    const double sum = block_sum<256>(squares(src, blockIdx.y * count, (int64_t)blockIdx.x * 256 + threadIdx.x, (int64_t)gridDim.x * 256, count), shared);
    if (threadIdx.x == 0) norms[blockIdx.y * kNormBlocks + blockIdx.x] = sum;
}

__device__ __forceinline__ void split_pair(float x, _Float16& h, _Float16& l) {
    h = (_Float16)x;
    l = (_Float16)(x - (float)h);
}
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
// Where element e of a row of pairs is: eight high parts, then their eight low ones.
__device__ __forceinline__ int64_t pair_at(int64_t e) { return 2 * e - (e & 7); }
__device__ __forceinline__ void put_pair(_Float16* to, float4 v) {
    f16x4 h, l;
    _Float16 a, b;
    split_pair(v.x, a, b); h.x = a; l.x = b;
    split_pair(v.y, a, b); h.y = a; l.y = b;
    split_pair(v.z, a, b); h.z = a; l.z = b;
    split_pair(v.w, a, b); h.w = a; l.w = b;
    *reinterpret_cast<f16x4*>(to) = h;
    *reinterpret_cast<f16x4*>(to + 8) = l;
}

// Matrices of `each` fp16 numbers, rows of `ld` pairs of which `width` are used: whole chunks, zeros past the last column.
struct Stack {
    _Float16* p; int64_t each; int ld, width;
    __device__ __forceinline__ _Float16* matrix(int64_t b) const { return p + b * each; }
    __device__ __forceinline__ int64_t at(int row, int col) const { return (int64_t)row * 2 * ld + pair_at(col); }
    __device__ __forceinline__ View<Pair> view(int64_t b, int row, int col, int rows, int64_t depth) const { return {matrix(b) + at(row, col), 2 * ld, rows, depth}; }
};

// X = direction / (norm + eps), scaled, as pairs; what is past a row's end is zero.
template <class T>
__global__ __launch_bounds__(256) void orthogonal_begin_kernel(Source<T> src, const double* __restrict__ norms, int n_norms, int K, int C,
                                                               float eps, float scale, Stack X) {
    __shared__ double shared[4];
    const int64_t b = blockIdx.y;
    const double inv = normaliser(block_sum<256>((int)threadIdx.x < n_norms ? norms[b * kNormBlocks + threadIdx.x] : 0.0, shared), eps, scale);
    const int quads = X.width / 4;
    const int64_t most = (int64_t)K * quads;
    for (int64_t q0 = (int64_t)blockIdx.x * 1024 + threadIdx.x; q0 < most; q0 += (int64_t)gridDim.x * 1024) {
        float v[4][4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t q = q0 + 256 * u < most ? q0 + 256 * u : q0;
            const int64_t row = q / quads;
            const int c = (int)(q - row * quads) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = src.again(b * K * C + row * C + (c + e < C ? c + e : C - 1));
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t q = q0 + 256 * u;
            if (q >= most) continue;
            const int64_t row = q / quads;
            const int c = (int)(q - row * quads) * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) v[u][e] = c + e < C ? (float)((double)v[u][e] * inv) : 0.f;
            put_pair(X.matrix(b) + X.at((int)row, c), make_float4(v[u][0], v[u][1], v[u][2], v[u][3]));
        }
    }
}

// Workgroup -> (matrix, tile row, tile column); tiles of a matrix one after the other on one XCD (see the products over groups).
__device__ __forceinline__ void place(int tile_rows, int tile_cols, int64_t& b, int& ti, int& tj) {
    unsigned at = blockIdx.x;
    const unsigned each = gridDim.x / 8, whole = each * 8;
    if (at < whole) at = (at & 7u) * each + (at >> 3);
    const unsigned tiles = (unsigned)tile_rows * tile_cols;
    b = at / tiles;
    ti = (int)(at % tiles) / tile_cols;
    tj = (int)(at % tiles) % tile_cols;
}

// out = alpha X^T X or X X^T (LIE: kAlong forms X X^T), or with `from` = X symmetric: alpha X X + beta X + gamma 1.  The result is symmetric:
// tiles below the diagonal are left out, and those above it are stored to both their places.
template <class P, Lie LIE>
__global__ __launch_bounds__(P::THREADS, P::THREADS == 256 ? 2 : 1) void orthogonal_square_kernel(Stack x, int r, int64_t depth, Stack out, float alpha, float beta, float gamma,
                                                                          int with_linear, int tile_rows, int tile_cols) {
    __shared__ __align__(16) unsigned short S[P::kLds];
    int64_t b;
    int ti, tj;
    place(tile_rows, tile_cols, b, ti, tj);
    static_assert(P::BM == P::BN, "");
    const int i0 = ti * P::BM, c0 = tj * P::BN;
    if (ti > tj) return;
    floatx16 acc[P::TM][P::TN];
    if (LIE == kAlong) P::run(acc, x.view(b, i0, 0, r - i0, depth), x.view(b, c0, 0, r - c0, depth), S);
    else P::run(acc, x.view(b, 0, i0, x.width - i0, depth), x.view(b, 0, c0, x.width - c0, depth), S);
    _Float16* to = out.matrix(b);
    const _Float16* lin = x.matrix(b);
    auto own = [&](int row, int col, float4 v) {
        const int i = i0 + row, j = c0 + col;
        if (i >= r || j >= out.width) return v;
        float w[4] = {alpha * v.x, alpha * v.y, alpha * v.z, alpha * v.w};
        if (with_linear) {
            const f16x4 h = *reinterpret_cast<const f16x4*>(lin + x.at(i, j)), l = *reinterpret_cast<const f16x4*>(lin + x.at(i, j) + 8);
            const float s[4] = {(float)h.x + (float)l.x, (float)h.y + (float)l.y, (float)h.z + (float)l.z, (float)h.w + (float)l.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = w[e] + beta * s[e] + (j + e == i ? gamma : 0.f);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = j + e < r ? w[e] : 0.f;             // (columns r .. width hold zeros)
        const float4 q = make_float4(w[0], w[1], w[2], w[3]);
        put_pair(to + out.at(i, j), q);
        return q;
    };
    auto mirror = [&](int col, int row, float4 v) {                          // (above the diagonal every row is one of the r)
        if (ti < tj && c0 + col < r) put_pair(to + out.at(c0 + col, i0 + row), v);
    };
    P::template drain<true>(acc, S, own, mirror);
}

// X <- P X (YL: X lies across the contraction) or X P (P is symmetric and lies along it), alpha times; the last time to `out` or off W.
template <class O> struct Target { O* out; float* W; float keep, rate; };
template <class P, Lie YL, class O>
__global__ __launch_bounds__(P::THREADS, P::THREADS == 256 ? 2 : 1) void orthogonal_apply_kernel(Stack left, Stack right, int K, int C, int r, Stack next, Target<O> last, float alpha,
                                                                         int tile_rows, int tile_cols) {
    __shared__ __align__(16) unsigned short S[P::kLds];
    int64_t b;
    int ti, tj;
    place(tile_rows, tile_cols, b, ti, tj);
    const int i0 = ti * P::BM, c0 = tj * P::BN;
    floatx16 acc[P::TM][P::TN];
    P::run(acc, left.view(b, i0, 0, K - i0, r), YL == kAcross ? right.view(b, 0, c0, right.width - c0, r) : right.view(b, c0, 0, C - c0, r), S);
    if (next.p) {
        _Float16* to = next.matrix(b);
        P::drain(acc, S, [&](int row, int col, float4 v) {
            const int i = i0 + row, j = c0 + col;
            if (i >= K || j >= next.width) return;
            put_pair(to + next.at(i, j),
                     make_float4(j < C ? alpha * v.x : 0.f, j + 1 < C ? alpha * v.y : 0.f, j + 2 < C ? alpha * v.z : 0.f, j + 3 < C ? alpha * v.w : 0.f));
        });
    } else if (last.W) {
        float* W = last.W + b * K * C;
        P::drain(acc, S, [&](int row, int col, float4 v) {
            const int i = i0 + row, j = c0 + col;
            if (i >= K) return;
            const float w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e < C) W[(int64_t)i * C + j + e] = last.keep * W[(int64_t)i * C + j + e] - last.rate * (alpha * w[e]);
        });
    } else {
        O* to = last.out + b * K * C;
        const bool whole = C % 4 == 0 && (reinterpret_cast<uintptr_t>(to) & (4 * sizeof(O) - 1)) == 0;
        P::drain(acc, S, [&](int row, int col, float4 v) {
            const int i = i0 + row, j = c0 + col;
            if (i < K && j < C) put(to + (int64_t)i * C, j, C, make_float4(alpha * v.x, alpha * v.y, alpha * v.z, alpha * v.w), whole);
        });
    }
}

// Matrices with at most 32 RT (64 or 128) rows on the smaller side.  A workgroup of sixteen wavefronts holds X, that is a slab of up to
// 16384 / RT / 32 of its columns, and S, then P, in LDS; with one slab the whole polynomial is one launch (256 x 64 fp32: 37 us, and 95
// with its fifteen products as launches of their own): 4.9 us a step, and 13 for the norm, X and the result.  A step moves 0.77 MB through the compute
// unit's LDS, 2.6 us at 128 bytes a clock; the rest are the latencies of its six stages, each of which waits for all of the one before, and
// of which S^2 keeps four wavefronts busy.  With more slabs, a launch per step: every workgroup adds up the slabs' parts of S, forms P itself, applies
// it to its slab and leaves its part of the next S (8 x 128 x 2048: 21 us a step, where one slab of 128 x 128 takes 7.6; the rest is a second launch
// that adds the parts up, and 42 MB of X and S to memory and back).  X lies as its smaller side's rows, whichever way the matrix lies.
constexpr int kMostSteps = 64;
struct Schedule { float s[kMostSteps], p2[kMostSteps], p1[kMostSteps], p0[kMostSteps], x[kMostSteps]; };      // factors of S, S^2, S, 1 and of X' a step
constexpr int kBlockX = 65536, kBlockS = 65536;          // bytes of LDS
constexpr int kMostSlabs = 16, kFewParts = 4;            // of one matrix; of which a workgroup adds up the parts of S itself

// A wavefront's operands from rows of PIECES pieces of 16 bytes in LDS (a chunk's eight high parts, its eight low ones); the pieces of a row are
// permuted by its number so that both the sixteen rows that are read along it at once and the four that are read across hit different
// banks.
template <int PIECES>
struct Rows {
    __device__ __forceinline__ static int swizzle(int row) { return (row & 1) | (row & 2) << 2 | (row & 12) >> 1; }
    __device__ __forceinline__ static int at(int row, int col) { return (row * PIECES + ((col >> 3 << 1) ^ swizzle(row))) * 16 + (col & 7) * 2; }       // high part; the low one: ^ 16
    __device__ __forceinline__ static uintx4 along(const char* S, int b, int s, int p) {
        const int lane = threadIdx.x & 63, row = 32 * b + (lane & 31), piece = (2 * s + (lane >> 5)) * 2 + p;
        return *reinterpret_cast<const uintx4*>(S + (row * PIECES + (piece ^ swizzle(row))) * 16);
    }
    __device__ __forceinline__ static uintx4 across(const char* S, int b, int s, int p) {
        typedef __attribute__((address_space(3))) shortx4* Lds;
        const int lane = threadIdx.x & 63, k = 16 * s + 8 * (lane >> 5) + ((lane & 15) >> 2), col = 32 * b + (lane & 16) + 4 * (lane & 3);
        const int piece = (col >> 3 << 1) + p, half = (col & 4) * 2;
        const shortx4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(S + (k * PIECES + (piece ^ swizzle(k))) * 16 + half));
        const shortx4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(S + ((k + 4) * PIECES + (piece ^ swizzle(k + 4))) * 16 + half));
        uintx4 q;
        __builtin_memcpy(&q, &u, 8);
        __builtin_memcpy(reinterpret_cast<char*>(&q) + 8, &v, 8);
        return q;
    }
    __device__ __forceinline__ static void put(char* S, int row, int col, float4 v) {
        f16x4 h, l;
        _Float16 a, b;
        split_pair(v.x, a, b); h.x = a; l.x = b;
        split_pair(v.y, a, b); h.y = a; l.y = b;
        split_pair(v.z, a, b); h.z = a; l.z = b;
        split_pair(v.w, a, b); h.w = a; l.w = b;
        *reinterpret_cast<f16x4*>(S + at(row, col)) = h;
        *reinterpret_cast<f16x4*>(S + (at(row, col) ^ 16)) = l;
    }
    // rows 32 bi .., columns 32 bj .. from a wavefront's accumulator (a row per lane, four columns in a row)
    __device__ __forceinline__ static void put_tile(char* S, int bi, int bj, const floatx16& c) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int r = 0; r < 16; r += 4)
            put(S, 32 * bi + (lane & 31), 32 * bj + 2 * r + 4 * (lane >> 5), make_float4(c[r], c[r + 1], c[r + 2], c[r + 3]));
    }
};
__device__ __forceinline__ floatx16 multiply_pairs(const uintx4 (&y)[2], const uintx4 (&x)[2], floatx16 c) {
    c = multiply<Pair>(y[0], x[1], c);
    c = multiply<Pair>(y[1], x[0], c);
    return multiply<Pair>(y[0], x[0], c);
}

// f for the steps that begin below `most`, `each` apart (what lies behind is zeros); two at a time: a launch fetches this code anew.
template <class F>
__device__ __forceinline__ void over_steps(int most, int each, F f) {
#pragma unroll 2
    for (int s = 0; s * each < most; ++s) f(s);
}

// `one`: the whole polynomial (one slab); else step `step` of it, 0: only X and the first S.
template <class T, int RT>
__global__ __launch_bounds__(1024) void orthogonal_block_kernel(Source<T> src, const double* __restrict__ norms, int n_norms, int K, int C, float eps,
                                                                float scale, int slabs, int one, int step, int steps, Schedule sch,
                                                                char* __restrict__ images, const float* __restrict__ parts_in, int n_parts,
                                                                float* __restrict__ parts_out,
                                                                T* out, float* W, float keep, float rate) {       // (out may be src.G)
    constexpr int R = 32 * RT, WIDTH = kBlockX / 4 / R, CT = WIDTH / 32;         // rows, columns of the slab, tiles of 32 columns
    constexpr int GROUPS = 16 / (RT * RT);                                   // wavefronts that share a tile of S
    using XRows = Rows<WIDTH / 4>;
    using SRows = Rows<R / 4>;
    using Out = Tile<RT, 16 / RT, 1, 1>;
    static_assert(CT * RT == 16 && Out::kSlabs * 2 <= kBlockX + kBlockS, "");
    __shared__ __align__(256) char lds[kBlockX + kBlockS];
    __shared__ double shared[16];
    char* X = lds;
    char* S = lds + kBlockX;                                                 // R * R * 4 bytes, behind it what is added up
    float* sums = reinterpret_cast<float*>(S + R * R * 4);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t b = blockIdx.x / slabs;
    const int slab = (int)(blockIdx.x % slabs);
    const bool tall = K > C;
    const int r = tall ? C : K, w = tall ? K : C, w0 = slab * WIDTH, ws = w - w0 < WIDTH ? w - w0 : WIDTH;
    const int64_t base = b * K * C;

    if (one || step == 0) {
        const double sum = one ? squares(src, base, tid, 1024, (int64_t)K * C) : tid < n_norms ? norms[b * kNormBlocks + tid] : 0.0;
        const double inv = normaliser(block_sum<1024>(sum, shared), eps, scale);      // (its barriers: M is what every thread has made it)
        auto element = [&](int i, int j) {                                   // row i of the smaller side, column w0 + j
            const bool in = i < r && j < ws;
            const int64_t e = in ? tall ? (int64_t)(w0 + j) * C + i : (int64_t)i * C + w0 + j : 0;
            const float d = src.again(base + e);
            return in ? (float)((double)d * inv) : 0.f;
        };
        if (tall) {
            // neighbouring threads take neighbouring elements in memory
#pragma unroll 2
            for (int f = tid; f < R * WIDTH; f += 1024) {
                const int i = f % R, j = f / R;
                _Float16* at = reinterpret_cast<_Float16*>(X + XRows::at(i, j));
                _Float16* low = reinterpret_cast<_Float16*>(X + (XRows::at(i, j) ^ 16));
                split_pair(element(i, j), *at, *low);
            }
        } else {
#pragma unroll 1
            for (int f = tid; f < R * WIDTH / 4; f += 1024) {
                const int i = f / (WIDTH / 4), j = f % (WIDTH / 4) * 4;
                XRows::put(X, i, j, make_float4(element(i, j), element(i, j + 1), element(i, j + 2), element(i, j + 3)));
            }
        }
    } else {
        const uintx4* from = reinterpret_cast<const uintx4*>(images + (int64_t)blockIdx.x * kBlockX);
#pragma unroll
        for (int f = 0; f < kBlockX / 16384; ++f) reinterpret_cast<uintx4*>(X)[tid + 1024 * f] = from[tid + 1024 * f];
    }

    const int tile = wave % (RT * RT), group = wave / (RT * RT), ti = tile / RT, tj = tile % RT;       // of S
    const int xi = wave / CT, xj = wave % CT;                                                 // of X
    const bool holds = 32 * ti < r && 32 * tj < r;                             // (all else is zeros)
    floatx16 acc;
    // (parts: four numbers of a lane next to those of the other lanes, four such of a tile)
    auto load_sum = [&](const float* from) {
        floatx16 v;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 f = *reinterpret_cast<const float4*>(from + ((tile * 4 + q) * 64 + lane) * 4);
            v[4 * q] = f.x; v[4 * q + 1] = f.y; v[4 * q + 2] = f.z; v[4 * q + 3] = f.w;
        }
        return v;
    };
    auto store_sum = [&](float* to, const floatx16& v) {
#pragma unroll
        for (int q = 0; q < 4; ++q) *reinterpret_cast<float4*>(to + ((tile * 4 + q) * 64 + lane) * 4) = make_float4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
    };
    auto own_square = [&] {                                                    // this group's part of the slab's part of S
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.f;
        over_steps(holds ? ws - 16 * group : 0, 16 * GROUPS, [&](int t) {
            const int s = t * GROUPS + group;
            const uintx4 x[2] = {XRows::along(X, ti, s, 0), XRows::along(X, ti, s, 1)}, y[2] = {XRows::along(X, tj, s, 0), XRows::along(X, tj, s, 1)};
            acc = multiply_pairs(y, x, acc);
        });
    };
    auto join_groups = [&] {                                                   // to group 0
        if constexpr (GROUPS > 1) {
            if (group > 0) store_sum(sums + (group - 1) * R * R, acc);
            __syncthreads();
            if (group == 0)
#pragma unroll
                for (int g = 1; g < GROUPS; ++g) acc += load_sum(sums + (g - 1) * R * R);
        }
    };
    auto leave_part = [&] {
        own_square();
        join_groups();
        if (group == 0) store_sum(parts_out + (int64_t)blockIdx.x * R * R, acc);
    };

    if (!one && step == 0) leave_part();
    for (int k = one ? 0 : step > 0 ? step - 1 : 0; k < (one ? steps : step); ++k) {
        if (one) own_square();
        else {
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] = 0.f;
#pragma unroll 2
            for (int t = group; t < n_parts; t += GROUPS) acc += load_sum(parts_in + (b * n_parts + t) * R * R);
            __syncthreads();                                                 // (X is there)
        }
        join_groups();
        floatx16 square;
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[e] *= sch.s[k];
            SRows::put_tile(S, ti, tj, acc);
        }
        __syncthreads();
        if (group == 0) {
#pragma unroll
            for (int e = 0; e < 16; ++e) square[e] = 0.f;
            over_steps(holds ? r : 0, 16, [&](int s) {
                const uintx4 x[2] = {SRows::along(S, ti, s, 0), SRows::along(S, ti, s, 1)}, y[2] = {SRows::along(S, tj, s, 0), SRows::along(S, tj, s, 1)};
                square = multiply_pairs(y, x, square);
            });
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int col = 32 * tj + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3);
                square[e] = sch.p2[k] * square[e] + sch.p1[k] * acc[e] + (col == 32 * ti + (lane & 31) ? sch.p0[k] : 0.f);
            }
        }
        __syncthreads();
        if (group == 0) SRows::put_tile(S, ti, tj, square);
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.f;
        over_steps(32 * xi < r && 32 * xj < ws ? r : 0, 16, [&](int s) {
            const uintx4 x[2] = {SRows::along(S, xi, s, 0), SRows::along(S, xi, s, 1)}, y[2] = {XRows::across(X, xj, s, 0), XRows::across(X, xj, s, 1)};
            acc = multiply_pairs(y, x, acc);
        });
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] *= sch.x[k];
        __syncthreads();                                                     // (nobody reads the old X any more)
        if (k + 1 < steps && 32 * xj < ws) XRows::put_tile(X, xi, xj, acc);
    }
    if (!one && step < steps) {
        if (step > 0) leave_part();
        else __syncthreads();
        uintx4* to = reinterpret_cast<uintx4*>(images + (int64_t)blockIdx.x * kBlockX);
#pragma unroll
        for (int f = 0; f < kBlockX / 16384; ++f) to[tid + 1024 * f] = reinterpret_cast<const uintx4*>(X)[tid + 1024 * f];
        return;
    }
    floatx16 last[1][1] = {{acc}};
    auto store = [&](int row, int col, float4 v) {                             // four elements of a row of the matrix
        if (row >= K || col >= C) return;
        const float q[4] = {v.x, v.y, v.z, v.w};
        const int64_t at = base + (int64_t)row * C + col;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (col + e >= C) continue;
            if (W) W[at + e] = keep * W[at + e] - rate * q[e];
            else out[at + e] = (T)q[e];
        }
    };
    if (tall) Out::template drain<true>(last, reinterpret_cast<unsigned short*>(lds), [](int, int, float4 v) { return v; },
                                        [&](int col, int row, float4 v) { if (col < ws) store(w0 + col, row, v); });
    else Out::drain(last, reinterpret_cast<unsigned short*>(lds), [&](int row, int col, float4 v) { store(row, w0 + col, v); });
}

// The slabs' parts of S, added up: with many slabs, every workgroup of the next step would read all of them.
__global__ __launch_bounds__(256) void orthogonal_parts_kernel(const float* __restrict__ parts, int slabs, int size, float* __restrict__ sums) {
    const int e = (blockIdx.x * 256 + threadIdx.x) * 4;
    const float* from = parts + (int64_t)blockIdx.y * slabs * size + e;
    float4 v[kMostSlabs];
#pragma unroll
    for (int t = 0; t < kMostSlabs; ++t) v[t] = *reinterpret_cast<const float4*>(from + (int64_t)(t < slabs ? t : 0) * size);
    float4 s = v[0];
#pragma unroll
    for (int t = 1; t < kMostSlabs; ++t)
        if (t < slabs) { s.x += v[t].x; s.y += v[t].y; s.z += v[t].z; s.w += v[t].w; }
    *reinterpret_cast<float4*>(sums + (int64_t)blockIdx.y * size + e) = s;
}

template <Lie X, Lie Y> using Large = Direct<Pair, X, Y, 2, 4, 4, 2, 2>;         // 256 x 256
template <Lie X, Lie Y> using Middle = Direct<Pair, X, Y, 2, 2, 2, 2, 2>;        // 128 x 128
template <Lie X, Lie Y> using Small = Direct<Pair, X, Y, 2, 2, 1, 1, 2, 2>;      // 64 x 64, two workgroups a compute unit
template <Lie X, Lie Y> using Lone = Direct<Pair, X, Y, 2, 2, 1, 1, 2, 4>;       // 64 x 64, one
enum Size { kLarge, kMiddle, kSmall, kLone };
constexpr int kSizeRows[] = {256, 128, 64, 64}, kSizeCols[] = {256, 128, 64, 64};
template <Size SIZE, Lie X, Lie Y>
using Sized = std::conditional_t<SIZE == kLarge, Large<X, Y>, std::conditional_t<SIZE == kMiddle, Middle<X, Y>,
              std::conditional_t<SIZE == kSmall, Small<X, Y>, Lone<X, Y>>>>;

int64_t over(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }
// Pairs from one row to the next: whole chunks, and an odd number of 256-byte pieces, so that the rows of a tile spread over the L2's
// channels (256 bytes each, 16 of them).
int64_t row_pairs(int64_t n) { return n <= 64 ? round8(n) : (over(n, 64) | 1) * 64; }
constexpr int64_t kCus = 256;
// The largest tiles that give every compute unit one; of a symmetric result about half of them are formed, and large ones pay from
// four a compute unit on (32 x 1024 x 1024 in 320 tiles of 256 x 256: 320 and 182 us, in 1152 of 128 x 128: 296 and 169).  Up to one small tile a
// compute unit, sixteen wavefronts share its contraction, else eight (767 x 1000: 194 us a call for 216 with eight everywhere; 7 x 512 x 512: 193
// for 260 with sixteen everywhere).
Size size_of(int64_t batch, int64_t rows, int64_t cols, bool symmetric) {
    auto tiles = [&](Size s) { return batch * over(rows, kSizeRows[s]) * over(cols, kSizeCols[s]); };
    if (tiles(kLarge) >= (symmetric ? 8 : 1) * kCus) return kLarge;
    if (tiles(kMiddle) >= (symmetric ? 2 : 1) * kCus) return kMiddle;
    return tiles(kSmall) > kCus ? kSmall : kLone;
}
template <class F>
void with_size(Size s, F f) {
    if (s == kLarge) f(std::integral_constant<Size, kLarge>());
    else if (s == kMiddle) f(std::integral_constant<Size, kMiddle>());
    else if (s == kSmall) f(std::integral_constant<Size, kSmall>());
    else f(std::integral_constant<Size, kLone>());
}

// The power of two that brings `most` to 2^13 .. 2^14 (of what is far below one, less near).
int scale_for(double most) { return most > 0.0 ? std::min(13 - std::ilogb(most), 24) : 24; }

}  // namespace

double polynomial_bound(double a, double b, double c, double s) {
    auto f = [&](double x) { return std::fabs(x * (a + x * x * (b + c * x * x))); };
    double most = f(s);
    auto see = [&](double x2) {                        // where the derivative a + 3 b x^2 + 5 c x^4 is zero
        if (x2 > 0.0 && x2 < s * s) most = std::max(most, f(std::sqrt(x2)));
    };
    // its roots in x^2 are q / (5 c) and a / q: the sum in q has terms of one sign, so that neither root is lost to cancellation however small
    // c is next to b (with c = 0 the first is no number or none in the range, with b = 0 too both are; q = 0: a or c is zero then, x^2 = 0)
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
        const double q = -0.5 * (3.0 * b + std::copysign(std::sqrt(d), b));
        see(q / (5.0 * c));
        see(a / q);
    }
    return std::isfinite(most) && std::isfinite(f(s)) ? most : HUGE_VAL;
}

const char* orthogonal_fault(int batch, int K, int C) {
    if (K > 32768 || C > 32768) return "matrices of more than 32768 rows or columns";
    if (batch > 65535) return "more than 65535 matrices";
    if (over(K, 64) * over(C, 64) * batch >= 1 << 22)                    // (2^32 threads a launch)
        return "more result tiles than one launch holds";
    return "";
}

namespace {
// Rows of 32 on the smaller side that a workgroup holds in LDS, and slabs of columns; 0: it does not.
struct Blocks { int rt, slabs; };
Blocks blocks_of(int K, int C) {
    const int r = std::min(K, C), w = std::max(K, C), rt = r <= 64 ? 2 : 4;
    const int64_t slabs = over(w, kBlockX / 4 / 32 / rt);
    return r <= 128 && slabs <= kMostSlabs ? Blocks{rt, (int)slabs} : Blocks{0, 0};
}
struct Layout { int64_t x, s, parts, bytes; };         // elements of X and of S, floats of the slabs' parts of S, and bytes of everything
Layout layout(int64_t batch, int K, int C) {
    const int64_t r = std::min(K, C);
    const Blocks bl = blocks_of(K, C);
    Layout l{0, 0, 0, 8 * kNormBlocks * batch + 5 * 256};
    if (bl.rt) {
        l.parts = batch * bl.slabs * (32 * bl.rt) * (32 * bl.rt);
        if (bl.slabs > 1) l.bytes += batch * bl.slabs * kBlockX + 3 * 4 * l.parts;
    } else {
        l.x = batch * K * row_pairs(C);
        l.s = batch * r * row_pairs(r);
        l.bytes += 4 * (2 * l.x + 2 * l.s);
    }
    return l;
}

// Powers of two that X, S and P carry, step by step.
struct Scales { int x, s, p, next; };
struct Bounds {
    double a, b, c, bound = 1.0;
    Scales step() {
        const double s2 = bound * bound, vertex = c != 0.0 ? -b / (2.0 * c) : -1.0;
        auto p = [&](double x) { return std::fabs(a + x * (b + c * x)); };
        double most = std::max(p(0.0), p(s2));
        if (vertex > 0.0 && vertex < s2) most = std::max(most, p(vertex));
        Scales e{scale_for(bound), scale_for(s2), scale_for(most), 0};
        bound = polynomial_bound(a, b, c, bound);
        e.next = scale_for(bound);
        return e;
    }
};

template <class T, int RT>
void launch_blocks(hipStream_t s, const Orthogonal& a, const Source<T>& src, int slabs, double* norms, int n_norms, char* images, float* parts, int64_t part_floats) {
    Schedule sch;
    Bounds bounds{a.a, a.b, a.c};
    for (int k = 0; k < a.steps; ++k) {
        const Scales e = bounds.step();
        sch.s[k] = std::ldexp(1.f, e.s - 2 * e.x);
        sch.p2[k] = (float)std::ldexp((double)a.c, e.p - 2 * e.s);
        sch.p1[k] = (float)std::ldexp((double)a.b, e.p - e.s);
        sch.p0[k] = (float)std::ldexp((double)a.a, e.p);
        sch.x[k] = std::ldexp(1.f, (k + 1 == a.steps ? 0 : e.next) - e.p - e.x);
    }
    const float scale = std::ldexp(1.f, scale_for(1.0));
    const int size = 1024 * RT * RT;
    const bool summed = slabs > kFewParts;
    float* sums = parts + 2 * part_floats;
    for (int step = slabs > 1 ? 0 : a.steps; step <= a.steps; ++step) {
        const float* in = parts + (step + 1) % 2 * part_floats;
        if (summed && step > 0) orthogonal_parts_kernel<<<dim3(size / 1024, a.batch), dim3(256), 0, s>>>(in, slabs, size, sums);
        orthogonal_block_kernel<T, RT><<<dim3((unsigned)(a.batch * slabs)), dim3(1024), 0, s>>>(
            src, norms, n_norms, a.K, a.C, a.eps, scale, slabs, slabs == 1, step, a.steps, sch, images, summed ? sums : in, summed ? 1 : slabs,
            parts + step % 2 * part_floats, (T*)a.out, a.W, a.keep, a.rate);
    }
}
}  // namespace

size_t orthogonal_scratch(int batch, int K, int C) { return layout(batch, K, C).bytes; }

void launch_orthogonalise(hipStream_t s, int type, const Orthogonal& a) {
    const int r = std::min(a.K, a.C), w = std::max(a.K, a.C), ld = (int)row_pairs(a.C), lds = (int)row_pairs(r);
    const bool wide = a.K <= a.C;
    const Layout l = layout(a.batch, a.K, a.C);
    const Blocks bl = blocks_of(a.K, a.C);
    char* at = (char*)a.scratch;
    auto take = [&](int64_t bytes) { char* p = at; at += over(bytes, 256) * 256; return p; };
    double* norms = (double*)take(8 * kNormBlocks * (int64_t)a.batch);
    const int64_t count = (int64_t)a.K * a.C;
    const int nb = (int)std::min<int64_t>(over(count, 2048), kNormBlocks);
    auto typed = [&](auto f) {
        if (type == kBf16) f((__bf16*)nullptr);
        else if (type == kF16) f((_Float16*)nullptr);
        else f((float*)nullptr);
    };
    typed([&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Source<T> src{(const T*)a.G, a.M, a.mu, a.nesterov};
        if (bl.slabs != 1) orthogonal_norm_kernel<T><<<dim3(nb, a.batch), dim3(256), 0, s>>>(src, count, norms);
        if (!bl.rt) return;
        char* images = take(bl.slabs > 1 ? (int64_t)a.batch * bl.slabs * kBlockX : 0);
        float* parts = (float*)take(bl.slabs > 1 ? 3 * 4 * l.parts : 0);
        if (bl.rt == 2) launch_blocks<T, 2>(s, a, src, bl.slabs, norms, nb, images, parts, l.parts);
        else launch_blocks<T, 4>(s, a, src, bl.slabs, norms, nb, images, parts, l.parts);
    });
    if (bl.rt) return;

    Stack X{(_Float16*)take(4 * l.x), (int64_t)2 * a.K * ld, ld, (int)round8(a.C)}, Y{(_Float16*)take(4 * l.x), (int64_t)2 * a.K * ld, ld, (int)round8(a.C)};
    Stack S{(_Float16*)take(4 * l.s), (int64_t)2 * r * lds, lds, (int)round8(r)}, Q{(_Float16*)take(4 * l.s), (int64_t)2 * r * lds, lds, (int)round8(r)};
    typed([&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        orthogonal_begin_kernel<T><<<dim3((unsigned)std::min<int64_t>(over(a.K * (round8(a.C) / 4), 1024), 1024), a.batch), dim3(256), 0, s>>>(
            Source<T>{(const T*)a.G, a.M, a.mu, a.nesterov}, norms, nb, a.K, a.C, a.eps, std::ldexp(1.f, scale_for(1.0)), X);
    });

    const Size square = size_of(a.batch, r, r, true), apply = size_of(a.batch, a.K, a.C, false);
    Bounds bounds{a.a, a.b, a.c};
    for (int k = 0; k < a.steps; ++k) {
        const auto [ex, es, ep, en] = bounds.step();
        const bool last = k + 1 == a.steps;
        with_size(square, [&](auto size) {
            const int tr = (int)over(r, kSizeRows[size]), tc = (int)over(r, kSizeCols[size]);
            const dim3 grid((unsigned)((int64_t)tr * tc * a.batch));
            using Along = Sized<decltype(size)::value, kAlong, kAlong>;
            using Across = Sized<decltype(size)::value, kAcross, kAcross>;
            const float one = std::ldexp(1.f, es - 2 * ex);
            if (wide) orthogonal_square_kernel<Along, kAlong><<<grid, dim3(Along::THREADS), 0, s>>>(X, r, w, S, one, 0.f, 0.f, 0, tr, tc);
            else orthogonal_square_kernel<Across, kAcross><<<grid, dim3(Across::THREADS), 0, s>>>(X, r, w, S, one, 0.f, 0.f, 0, tr, tc);
            orthogonal_square_kernel<Along, kAlong><<<grid, dim3(Along::THREADS), 0, s>>>(
                S, r, r, Q, (float)std::ldexp((double)a.c, ep - 2 * es), (float)std::ldexp((double)a.b, ep - es), (float)std::ldexp((double)a.a, ep), 1, tr, tc);
        });
        with_size(apply, [&](auto size) {
            const int tr = (int)over(a.K, kSizeRows[size]), tc = (int)over(a.C, kSizeCols[size]);
            const dim3 grid((unsigned)((int64_t)tr * tc * a.batch));
            const float alpha = std::ldexp(1.f, (last ? 0 : en) - ep - ex);
            const Stack next = last ? Stack{nullptr, 0, 0, 0} : Y;
            auto go = [&](auto* o) {
                using O = std::remove_pointer_t<decltype(o)>;
                const Target<O> target{(O*)a.out, a.W, a.keep, a.rate};
                using Wide = Sized<decltype(size)::value, kAlong, kAcross>;
                using Tall = Sized<decltype(size)::value, kAlong, kAlong>;
                if (wide) orthogonal_apply_kernel<Wide, kAcross, O><<<grid, dim3(Wide::THREADS), 0, s>>>(Q, X, a.K, a.C, r, next, target, alpha, tr, tc);
                else orthogonal_apply_kernel<Tall, kAlong, O><<<grid, dim3(Tall::THREADS), 0, s>>>(X, Q, a.K, a.C, r, next, target, alpha, tr, tc);
            };
            if (!last || a.W || type == kF32) go((float*)nullptr);
            else if (type == kBf16) go((__bf16*)nullptr);
            else go((_Float16*)nullptr);
        });
        std::swap(X, Y);
    }
}

}  // namespace cadmm
