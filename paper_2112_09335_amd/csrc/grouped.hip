// Dense products over rows that are sorted into groups, each group with a matrix of its own (weights per community):
//   transform: out[r] = A[r] B_g      for the rows r of group g      (B_g K x C, or stored C x K and transposed)
//   wgrad    : out_g  = A_g^T G_g     the sum over the rows of group g
// Group g owns the rows [ptr[g], ptr[g+1]); the bounds are read on the device.  Whatever they hold, no row outside [0, n) is
// touched: every bound is clamped to that range first.
#include <type_traits>

#include "kernels.h"

namespace cadmm {

namespace {

template <class T> __device__ __forceinline__ float value(T x) { return (float)x; }

__device__ __forceinline__ int64_t bound_of(const int64_t* __restrict__ ptr, int g, int64_t n) {
    const int64_t p = ptr[g];
    return p < 0 ? 0 : p > n ? n : p;
}

// Rows go to workgroups in slots of BM: group g's rows [ptr[g] + i BM, ..) have slot ptr[g] / BM + g + i.  A group of len rows gets
// at least ceil(len / BM) slots this way and at most two more than it fills, slots of different groups are apart, and the
// group of a slot is found by a search in the bounds alone, without a prefix sum over the groups' tile counts.
template <int BM>
__device__ __forceinline__ int64_t first_slot(const int64_t* __restrict__ ptr, int g, int64_t n) { return bound_of(ptr, g, n) / BM + g; }
// The last group whose first slot is not behind `slot`; 64 bounds are looked at in one step.
template <int BM>
__device__ __forceinline__ int group_of_slot(const int64_t* __restrict__ ptr, int groups, int64_t n, int64_t slot) {
    const int lane = threadIdx.x & 63;
    int at = 0, left = groups;                         // the answer is in [at, at + left)
    while (left > 1) {
        const int stride = (left + 63) / 64;
        const int g = lane * stride;
        const bool in = g < left && first_slot<BM>(ptr, at + g, n) <= slot;
        const int found = __popcll(__ballot(in));      // (the bounds do not descend: the lanes that are in come first)
        const int skip = (found > 0 ? found - 1 : 0) * stride;
        at += skip;
        left = left - skip < stride ? left - skip : stride;
    }
    return at;
}

constexpr int ST = 64, SK = 16;        // results of a workgroup in each direction, and of the contraction per step

// 64 x 64 results on the vector ALU in fp32: X(i, k) at X + i xi + k xk, Y(k, j) at Y + k yk + j yj.
template <class T>
__device__ __forceinline__ void simple_tile(float (&acc)[4][4], const T* __restrict__ X, int64_t xi, int64_t xk, const T* __restrict__ Y,
                                            int64_t yk, int64_t yj, int64_t rows, int64_t cols, int64_t depth) {
    __shared__ float Xs[SK][ST + 4], Ys[SK][ST + 4];
    const int tid = threadIdx.x, ti = tid >> 4, tj = tid & 15;
    for (int64_t k0 = 0; k0 < depth; k0 += SK) {
        __syncthreads();
        for (int f = tid; f < SK * ST; f += 256) {
            const int i = f / SK, k = f % SK;
            Xs[k][i] = i < rows && k0 + k < depth ? value(X[i * xi + (k0 + k) * xk]) : 0.f;
            Ys[k][i] = i < cols && k0 + k < depth ? value(Y[(k0 + k) * yk + i * yj]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < SK; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[i][j] += Xs[k][ti * 4 + i] * Ys[k][tj * 4 + j];
    }
}
template <class O>
__device__ __forceinline__ void simple_store(const float (&acc)[4][4], O* __restrict__ out, int64_t ld, int64_t rows, int64_t cols) {
    const int ti = threadIdx.x >> 4, tj = threadIdx.x & 15;
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j)
            if (ti * 4 + i < rows && tj * 4 + j < cols) out[(ti * 4 + i) * ld + tj * 4 + j] = (O)acc[i][j];
}

template <class T>
__global__ __launch_bounds__(256) void grouped_nn_kernel(const T* __restrict__ A, int64_t n, int64_t lda, int K, const T* __restrict__ B,
                                                         int C, int transposed, int groups, const int64_t* __restrict__ ptr,
                                                         T* __restrict__ out, int64_t ldo, int col_tiles) {
    const int64_t slot = blockIdx.x / col_tiles;
    const int c0 = (int)(blockIdx.x % col_tiles) * ST;
    const int g = group_of_slot<ST>(ptr, groups, n, slot);
    const int64_t skip = slot - first_slot<ST>(ptr, g, n);
    const int64_t r0 = bound_of(ptr, g, n) + skip * ST, end = bound_of(ptr, g + 1, n);
    if (skip < 0 || r0 >= end) return;
    float acc[4][4] = {};
    const T* Bg = B + (int64_t)g * K * C + (transposed ? (int64_t)c0 * K : c0);
    simple_tile(acc, A + r0 * lda, lda, 1, Bg, transposed ? 1 : C, transposed ? K : 1, end - r0, C - c0, K);
    simple_store(acc, out + r0 * ldo + c0, ldo, end - r0, C - c0);
}

template <class T, class O>
__global__ __launch_bounds__(256) void grouped_tn_kernel(const T* __restrict__ A, int64_t n, int64_t lda, int K, const T* __restrict__ G,
                                                         int64_t ldg, int C, const int64_t* __restrict__ ptr, O* __restrict__ out,
                                                         int col_tiles, int tiles) {
    const int g = (int)(blockIdx.x / tiles), t = (int)(blockIdx.x % tiles);
    const int i0 = t / col_tiles * ST, c0 = t % col_tiles * ST;
    const int64_t lo = bound_of(ptr, g, n), hi = bound_of(ptr, g + 1, n);
    float acc[4][4] = {};
    simple_tile(acc, A + lo * lda + i0, 1, lda, G + lo * ldg + c0, ldg, 1, K - i0, C - c0, hi - lo);
    simple_store(acc, out + ((int64_t)g * K + i0) * C + c0, C, K - i0, C - c0);
}

template <class F>
void with_type(int type, F f) {
    if (type == kBf16) f((__bf16*)nullptr);
    else if (type == kF16) f((_Float16*)nullptr);
    else f((float*)nullptr);
}

}  // namespace

int64_t grouped_nn_blocks(int64_t n, int C, int groups) { return (n / ST + groups) * ((C + ST - 1) / ST); }
int64_t grouped_tn_blocks(int64_t, int K, int C, int groups) { return (int64_t)groups * ((K + ST - 1) / ST) * ((C + ST - 1) / ST); }
size_t grouped_tn_scratch(int64_t, int, int, int) { return 0; }

void launch_grouped_nn(hipStream_t s, int type, const GroupedNN& a) {
    const int col_tiles = (a.C + ST - 1) / ST;
    if (a.n == 0) return;
    with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        grouped_nn_kernel<T><<<dim3((unsigned)grouped_nn_blocks(a.n, a.C, a.groups)), dim3(256), 0, s>>>(
            (const T*)a.A, a.n, a.lda, a.K, (const T*)a.B, a.C, a.transposed, a.groups, a.ptr, (T*)a.out, a.ldo, col_tiles);
    });
}

void launch_grouped_tn(hipStream_t s, int type, int out_type, const GroupedTN& a) {
    const int col_tiles = (a.C + ST - 1) / ST, tiles = col_tiles * ((a.K + ST - 1) / ST);
    with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        const dim3 grid((unsigned)grouped_tn_blocks(a.n, a.K, a.C, a.groups));
        if (out_type == kF32)
            grouped_tn_kernel<T, float><<<grid, dim3(256), 0, s>>>((const T*)a.A, a.n, a.lda, a.K, (const T*)a.G, a.ldg, a.C, a.ptr,
                                                                   (float*)a.out, col_tiles, tiles);
        else
            grouped_tn_kernel<T, T><<<grid, dim3(256), 0, s>>>((const T*)a.A, a.n, a.lda, a.K, (const T*)a.G, a.ldg, a.C, a.ptr, (T*)a.out,
                                                               col_tiles, tiles);
    });
}

}  // namespace cadmm
