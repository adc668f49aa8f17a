// Updates with their singular values brought towards one: X <- a X + (b S + c S^2) X with S = X X^T, an odd polynomial of the
// matrix that leaves its singular vectors alone and takes every singular value x to a x + b x^3 + c x^5, applied a few times to
// every matrix of a stack over its Frobenius norm.  S is formed on the smaller side: r = min(K, C) rows of s = max(K, C).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "kernels.h"

namespace cadmm {

namespace {

constexpr int ST = 64, SK = 16;

// One workgroup a matrix: the direction D (G itself, or what the momentum makes of it) and its norm, then X = D / (norm + eps), tall
// matrices transposed.
template <class T>
__global__ __launch_bounds__(256) void orthogonal_begin_kernel(const T* __restrict__ G, float* __restrict__ M, float mu, int nesterov, int K,
                                                               int C, float eps, float* __restrict__ X) {
    const int64_t count = (int64_t)K * C, base = blockIdx.x * count;
    __shared__ double sums[256];
    double sum = 0.0;
    for (int64_t f = threadIdx.x; f < count; f += 256) {
        float d = (float)G[base + f];
        if (M) {
            const float m = mu * M[base + f] + d;
            M[base + f] = m;
            d = nesterov ? d + mu * m : m;
        }
        X[base + (K > C ? f % C * K + f / C : f)] = d;
        sum += (double)d * (double)d;
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    for (int o = 128; o > 0; o >>= 1) {
        if ((int)threadIdx.x < o) sums[threadIdx.x] += sums[threadIdx.x + o];
        __syncthreads();
    }
    const double norm = sqrt(sums[0]) + (double)eps, inv = norm > 0.0 ? 1.0 / norm : norm == 0.0 ? 0.0 : norm;
    for (int64_t f = threadIdx.x; f < count; f += 256) X[base + f] = (float)((double)X[base + f] * inv);
}

// out = alpha D + beta L R for every matrix of the stack (D may be null); L m x k, R k x p, or with RT its transpose p x k.
template <bool RT>
__global__ __launch_bounds__(256) void orthogonal_product_kernel(const float* __restrict__ L, const float* __restrict__ R, const float* __restrict__ D,
                                                                 float* __restrict__ out, int m, int k, int p, float alpha, float beta) {
    const int64_t b = blockIdx.z;
    const int i0 = blockIdx.y * ST, j0 = blockIdx.x * ST;
    L += b * m * k; R += b * k * p; out += b * m * p;
    __shared__ float Ls[SK][ST + 4], Rs[SK][ST + 4];
    const int tid = threadIdx.x, ti = tid >> 4, tj = tid & 15;
    float acc[4][4] = {}, sum[4][4] = {};
    // (sums of 128 products are added up: a single chain of thousands would cost three bits)
    auto gather = [&] {
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) { sum[i][j] += acc[i][j]; acc[i][j] = 0.f; }
    };
    for (int k0 = 0; k0 < k; k0 += SK) {
        if (k0 % 128 == 0) gather();
        __syncthreads();
        for (int f = tid; f < SK * ST; f += 256) {
            const int i = f / SK, kk = f % SK;
            const int row = i0 + i, col = j0 + i, at = k0 + kk;
            Ls[kk][i] = row < m && at < k ? L[(int64_t)row * k + at] : 0.f;
            Rs[kk][i] = col < p && at < k ? RT ? R[(int64_t)col * k + at] : R[(int64_t)at * p + col] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < SK; ++kk)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += Ls[kk][ti * 4 + i] * Rs[kk][tj * 4 + j];
    }
    gather();
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int row = i0 + ti * 4 + i, col = j0 + tj * 4 + j;
            if (row >= m || col >= p) continue;
            const int64_t o = (int64_t)row * p + col;
            out[o] = D ? alpha * D[b * m * p + o] + beta * sum[i][j] : beta * sum[i][j];
        }
}

template <class T>
__global__ __launch_bounds__(256) void orthogonal_end_kernel(const float* __restrict__ X, int K, int C, T* __restrict__ out, float* __restrict__ W,
                                                             float keep, float rate) {
    const int64_t count = (int64_t)K * C, base = blockIdx.y * count;
    for (int64_t f = blockIdx.x * 256 + threadIdx.x; f < count; f += (int64_t)gridDim.x * 256) {
        const float x = X[base + (K > C ? f % C * K + f / C : f)];
        if (W) W[base + f] = keep * W[base + f] - rate * x;
        else out[base + f] = (T)x;
    }
}

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
    return "";
}

size_t orthogonal_scratch(int batch, int K, int C) {
    const size_t r = std::min(K, C), s = std::max(K, C);
    return (size_t)batch * (2 * r * s + 2 * r * r) * sizeof(float);
}

void launch_orthogonalise(hipStream_t s, int type, const Orthogonal& a) {
    const int r = std::min(a.K, a.C), w = std::max(a.K, a.C);
    float* X = (float*)a.scratch;
    float* Y = X + (size_t)a.batch * r * w;
    float* S = Y + (size_t)a.batch * r * w;
    float* P = S + (size_t)a.batch * r * r;
    auto begin = [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        orthogonal_begin_kernel<T><<<dim3(a.batch), dim3(256), 0, s>>>((const T*)a.G, a.M, a.mu, a.nesterov, a.K, a.C, a.eps, X);
    };
    if (type == kBf16) begin((__bf16*)nullptr);
    else if (type == kF16) begin((_Float16*)nullptr);
    else begin((float*)nullptr);
    const unsigned tr = (r + ST - 1) / ST, tw = (w + ST - 1) / ST;
    for (int k = 0; k < a.steps; ++k) {
        orthogonal_product_kernel<true><<<dim3(tr, tr, a.batch), dim3(256), 0, s>>>(X, X, nullptr, S, r, w, r, 0.f, 1.f);
        orthogonal_product_kernel<true><<<dim3(tr, tr, a.batch), dim3(256), 0, s>>>(S, S, S, P, r, r, r, a.b, a.c);
        orthogonal_product_kernel<false><<<dim3(tw, tr, a.batch), dim3(256), 0, s>>>(P, X, X, Y, r, r, w, a.a, 1.f);
        std::swap(X, Y);
    }
    const dim3 grid((unsigned)std::min<int64_t>(((int64_t)a.K * a.C + 255) / 256, 1024), a.batch);
    if (type == kBf16) orthogonal_end_kernel<__bf16><<<grid, dim3(256), 0, s>>>(X, a.K, a.C, (__bf16*)a.out, a.W, a.keep, a.rate);
    else if (type == kF16) orthogonal_end_kernel<_Float16><<<grid, dim3(256), 0, s>>>(X, a.K, a.C, (_Float16*)a.out, a.W, a.keep, a.rate);
    else orthogonal_end_kernel<float><<<grid, dim3(256), 0, s>>>(X, a.K, a.C, (float*)a.out, a.W, a.keep, a.rate);
}

}  // namespace cadmm
