// Updates with their singular values brought towards one: X <- a X + (b S + c S^2) X with S = X X^T, an odd polynomial of the
// matrix that leaves its singular vectors alone and takes every singular value x to a x + b x^3 + c x^5, applied a few times to
// every matrix of a stack over its Frobenius norm.  With K <= C, S = X X^T and X <- P X for P = a + b S + c S^2; else S = X^T X and
// X <- X P: no matrix is transposed, the operands lie along or across the contraction as it comes (tile_product.h).
//
// Between the launches X, S and P are kept as pairs of fp16 (22 bits), each scaled by a power of two that keeps its largest possible
// entry below 2^15: a singular value of X is bounded by what the polynomial makes of [0, 1] (polynomial_bound), an entry by the
// largest singular value.  What a pair drops is below 2^-38 of that bound, or 2^-23 of the entry.  The polynomial multiplies small
// singular values by a (3.4445) a step, errors with them: sixteen bits or less would show in a result of bf16.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"
#include "tile_product.h"

namespace cadmm {

namespace {

using namespace tile;

constexpr int kNormBlocks = 64;        // most workgroups that add up one matrix's norm

// The direction of the update: the gradient, or what the momentum makes of it.
template <class T>
struct Source {
    const T* G; float* M; float mu; int nesterov;
    __device__ __forceinline__ float first(int64_t e) const {             // with the momentum brought forward
        const float g = (float)G[e];
        if (!M) return g;
        const float m = mu * M[e] + g;
        M[e] = m;
        return nesterov ? g + mu * m : m;
    }
    __device__ __forceinline__ float again(int64_t e) const {
        if (!M) return (float)G[e];
        const float m = M[e];
        return nesterov ? (float)G[e] + mu * m : m;
    }
};

template <class T>
__global__ __launch_bounds__(256) void orthogonal_norm_kernel(Source<T> src, int64_t count, double* __restrict__ norms) {
    const int64_t base = blockIdx.y * count;
    __shared__ double sums[4];
    double sum = 0.0;
    for (int64_t f = (int64_t)blockIdx.x * 256 + threadIdx.x; f < count; f += (int64_t)gridDim.x * 256) {
        const double d = src.first(base + f);
        sum += d * d;
    }
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) norms[blockIdx.y * kNormBlocks + blockIdx.x] = (sums[0] + sums[1]) + (sums[2] + sums[3]);
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
    const int64_t b = blockIdx.y;
    double sum = 0.0;
    for (int i = 0; i < n_norms; ++i) sum += norms[b * kNormBlocks + i];
    const double norm = sqrt(sum) + (double)eps;
    // (no direction: zero; an entry that is not finite: nothing is)
    const double inv = norm == 0.0 ? 0.0 : norm < HUGE_VAL ? (double)scale / norm : __builtin_nan("");
    const int quads = X.width / 4;
    for (int64_t q = (int64_t)blockIdx.x * 256 + threadIdx.x; q < (int64_t)K * quads; q += (int64_t)gridDim.x * 256) {
        const int64_t row = q / quads;
        const int c = (int)(q % quads) * 4;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = c + e < C ? (float)((double)src.again(b * K * C + row * C + c + e) * inv) : 0.f;
        put_pair(X.matrix(b) + X.at((int)row, c), make_float4(v[0], v[1], v[2], v[3]));
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
// tiles below the diagonal are left out, and of the others every entry on or above it is stored to both its places.
template <class P, Lie LIE>
__global__ __launch_bounds__(P::THREADS, P::THREADS == 256 ? 2 : 1) void orthogonal_square_kernel(Stack x, int r, int64_t depth, Stack out, float alpha, float beta, float gamma,
                                                                          int with_linear, int tile_rows, int tile_cols) {
    __shared__ __align__(16) unsigned short S[P::kLds];
    int64_t b;
    int ti, tj;
    place(tile_rows, tile_cols, b, ti, tj);
    const int i0 = ti * P::BM, c0 = tj * P::BN;
    if (i0 >= c0 + P::BN) return;
    floatx16 acc[P::TM][P::TN];
    if (LIE == kAlong) P::run(acc, x.view(b, i0, 0, r - i0, depth), x.view(b, c0, 0, r - c0, depth), S);
    else P::run(acc, x.view(b, 0, i0, x.width - i0, depth), x.view(b, 0, c0, x.width - c0, depth), S);
    _Float16* to = out.matrix(b);
    const _Float16* lin = x.matrix(b);
    const bool crossing = c0 < i0 + P::BM;                 // the tile holds entries below the diagonal
    auto own = [&](int row, int col, float4 v) {
        const int i = i0 + row, j = c0 + col;
        float w[4] = {alpha * v.x, alpha * v.y, alpha * v.z, alpha * v.w};
        if (i >= r || j >= out.width) return v;
        if (with_linear) {
            const f16x4 h = *reinterpret_cast<const f16x4*>(lin + x.at(i, j)), l = *reinterpret_cast<const f16x4*>(lin + x.at(i, j) + 8);
            const float s[4] = {(float)h.x + (float)l.x, (float)h.y + (float)l.y, (float)h.z + (float)l.z, (float)h.w + (float)l.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = w[e] + beta * s[e] + (j + e == i ? gamma : 0.f);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = j + e < r ? w[e] : 0.f;
        const float4 q = make_float4(w[0], w[1], w[2], w[3]);
        _Float16* at = to + out.at(i, j);
        if (!crossing || j >= i) put_pair(at, q);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (j + e >= i) split_pair(w[e], at[e], at[e + 8]);
        }
        return q;
    };
    // ( columns r .. width hold zeros, which the own side of the last tile column leaves)
    auto mirror = [&](int col, int row, float4 v) {
        const int i = i0 + row, j = c0 + col;
        if (j >= r || i >= r) return;
        const float w[4] = {v.x, v.y, v.z, v.w};
        _Float16* at = to + out.at(j, i);
        if (i + 3 < j) put_pair(at, v);
        else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (i + e < j) split_pair(w[e], at[e], at[e + 8]);
        }
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

template <Lie X, Lie Y> using Large = Direct<Pair, X, Y, 2, 4, 4, 2, 2>;         // 256 x 256
template <Lie X, Lie Y> using Middle = Direct<Pair, X, Y, 2, 2, 2, 2, 2>;        // 128 x 128
template <Lie X, Lie Y> using Small = Direct<Pair, X, Y, 2, 2, 1, 1, 4>;         // 64 x 64
enum Size { kLarge, kMiddle, kSmall };
constexpr int kSizeRows[] = {256, 128, 64}, kSizeCols[] = {256, 128, 64};
template <Size SIZE, Lie X, Lie Y>
using Sized = std::conditional_t<SIZE == kLarge, Large<X, Y>, std::conditional_t<SIZE == kMiddle, Middle<X, Y>, Small<X, Y>>>;

int64_t over(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t round8(int64_t n) { return (n + 7) / 8 * 8; }
// Pairs from one row to the next: whole chunks, and an odd number of 256-byte pieces, so that the rows of a tile spread over the L2's
// channels (256 bytes each, 16 of them).
int64_t row_pairs(int64_t n) { return n <= 64 ? round8(n) : (over(n, 64) | 1) * 64; }
constexpr int64_t kCus = 256;
// The largest tiles that give every compute unit one; half: of a symmetric result only that much is formed.
Size size_of(int64_t batch, int64_t rows, int64_t cols, bool half) {
    for (Size s : {kLarge, kMiddle})
        if (batch * over(rows, kSizeRows[s]) * over(cols, kSizeCols[s]) >= (half ? 2 : 1) * kCus) return s;
    return kSmall;
}
template <class F>
void with_size(Size s, F f) {
    if (s == kLarge) f(std::integral_constant<Size, kLarge>());
    else if (s == kMiddle) f(std::integral_constant<Size, kMiddle>());
    else f(std::integral_constant<Size, kSmall>());
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
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (c != 0.0 && d >= 0.0) {
        see((-3.0 * b + std::sqrt(d)) / (10.0 * c));
        see((-3.0 * b - std::sqrt(d)) / (10.0 * c));
    } else if (c == 0.0 && b != 0.0) {
        see(-a / (3.0 * b));
    }
    return std::isfinite(most) && std::isfinite(f(s)) ? most : HUGE_VAL;
}

const char* orthogonal_fault(int batch, int K, int C) {
    if (K > 32768 || C > 32768) return "matrices of more than 32768 rows or columns";
    if (batch > 65535) return "more than 65535 matrices";
    if (over(K, 64) * over(C, 64) * batch > 0x7fffffff || over(std::min(K, C), 64) * over(std::min(K, C), 64) * batch > 0x7fffffff)
        return "more result tiles than one launch holds";
    return "";
}

namespace {
struct Layout { int64_t x, s, bytes; };               // elements of X and of S, and bytes of everything
Layout layout(int64_t batch, int64_t K, int64_t C) {
    const int64_t r = std::min(K, C);
    Layout l;
    l.x = batch * K * row_pairs(C);
    l.s = batch * r * row_pairs(r);
    l.bytes = 8 * kNormBlocks * batch + 2 * (2 * 2 * l.x + 2 * 2 * l.s) + 5 * 256;
    return l;
}
}  // namespace

size_t orthogonal_scratch(int batch, int K, int C) { return layout(batch, K, C).bytes; }

void launch_orthogonalise(hipStream_t s, int type, const Orthogonal& a) {
    const int r = std::min(a.K, a.C), w = std::max(a.K, a.C), ld = (int)row_pairs(a.C), lds = (int)row_pairs(r);
    const bool wide = a.K <= a.C;
    const Layout l = layout(a.batch, a.K, a.C);
    char* at = (char*)a.scratch;
    auto take = [&](int64_t bytes) { char* p = at; at += over(bytes, 256) * 256; return p; };
    double* norms = (double*)take(8 * kNormBlocks * (int64_t)a.batch);
    Stack X{(_Float16*)take(4 * l.x), (int64_t)2 * a.K * ld, ld, (int)round8(a.C)}, Y{(_Float16*)take(4 * l.x), (int64_t)2 * a.K * ld, ld, (int)round8(a.C)};
    Stack S{(_Float16*)take(4 * l.s), (int64_t)2 * r * lds, lds, (int)round8(r)}, Q{(_Float16*)take(4 * l.s), (int64_t)2 * r * lds, lds, (int)round8(r)};

    double bound = 1.0;
    int ex = scale_for(bound);
    const int64_t count = (int64_t)a.K * a.C;
    auto begin = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const Source<T> src{(const T*)a.G, a.M, a.mu, a.nesterov};
        const int nb = (int)std::min<int64_t>(over(count, 1024), kNormBlocks);
        orthogonal_norm_kernel<T><<<dim3(nb, a.batch), dim3(256), 0, s>>>(src, count, norms);
        orthogonal_begin_kernel<T><<<dim3((unsigned)std::min<int64_t>(over(a.K * (round8(a.C) / 4), 256), 1024), a.batch), dim3(256), 0, s>>>(
            src, norms, nb, a.K, a.C, a.eps, std::ldexp(1.f, ex), X);
    };
    if (type == kBf16) begin((__bf16*)nullptr);
    else if (type == kF16) begin((_Float16*)nullptr);
    else begin((float*)nullptr);

    const Size square = size_of(a.batch, r, r, true), apply = size_of(a.batch, a.K, a.C, false);
    for (int k = 0; k < a.steps; ++k) {
        const double s2 = bound * bound, vertex = a.c != 0.f ? -(double)a.b / (2.0 * a.c) : -1.0;
        auto p = [&](double x) { return std::fabs(a.a + x * (a.b + (double)a.c * x)); };
        double most = std::max(p(0.0), p(s2));
        if (vertex > 0.0 && vertex < s2) most = std::max(most, p(vertex));
        const int es = scale_for(s2), ep = scale_for(most);
        bound = polynomial_bound(a.a, a.b, a.c, bound);
        const int en = scale_for(bound);
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
        ex = en;
    }
}

}  // namespace cadmm
