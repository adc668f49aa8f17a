// Dense products over rows that are sorted into groups, each group with a matrix of its own (weights per community):
//   transform: out[r] = A[r] B_g      for the rows r of group g      (B_g K x C, or stored C x K and transposed)
//   wgrad    : out_g  = A_g^T G_g     the sum over the rows of group g
// Group g owns the rows [ptr[g], ptr[g+1]); the bounds are read on the device.  Whatever they hold, no row outside [0, n) is
// touched: every bound is clamped to that range first.
#include <algorithm>
#include <type_traits>

#include "kernels.h"
#include "tile_product.h"

namespace cadmm {

namespace {

using namespace tile;

__device__ __forceinline__ int64_t bound_of(const int64_t* __restrict__ ptr, int g, int64_t n) {
    const int64_t p = ptr[g];
    return p < 0 ? 0 : p > n ? n : p;
}

// Rows go to workgroups in slots of `rows`: group g's rows [ptr[g] + i rows, ..) have slot ptr[g] / rows + g + i.  A group of len rows
// gets at least ceil(len / rows) slots this way and at most two more than it fills, one at least, slots of different groups are apart,
// and the group of a slot is found by a search in the bounds alone, without a prefix sum over the groups' tile counts.
__device__ __forceinline__ int64_t first_slot(const int64_t* __restrict__ ptr, int g, int64_t n, int64_t rows) {
    return bound_of(ptr, g, n) / rows + g;
}
// The last group whose first slot is not behind `slot`; 64 bounds are looked at in one step.
__device__ __forceinline__ int group_of_slot(const int64_t* __restrict__ ptr, int groups, int64_t n, int64_t rows, int64_t slot) {
    const int lane = threadIdx.x & 63;
    int at = 0, left = groups;                         // the answer is in [at, at + left)
    while (left > 1) {
        const int stride = (left + 63) / 64;
        const int g = lane * stride;
        const bool in = g < left && first_slot(ptr, at + g, n, rows) <= slot;
        const int found = __popcll(__ballot(in));      // (the bounds do not descend: the lanes that are in come first)
        const int skip = (found > 0 ? found - 1 : 0) * stride;
        at += skip;
        left = left - skip < stride ? left - skip : stride;
    }
    return __builtin_amdgcn_readfirstlane(at);
}

// Workgroup -> (slot, tile).  Consecutive workgroups go round-robin to the eight XCDs, each with an L2 of its own.  In slices, every
// XCD walks one contiguous part of the list, tiles of a slot one after the other and slots of a group too, so that what they share comes
// from its L2.  With few rows a group the slots that hold rows are not spread evenly over the list, and plain order is kept.
__device__ __forceinline__ void place(unsigned tiles, bool slices, int64_t& slot, int& t) {
    unsigned b = blockIdx.x;
    if (slices) {
        const unsigned nb = gridDim.x, each = nb / 8, whole = each * 8;
        if (b < whole) b = (b & 7u) * each + (b >> 3);
    }
    slot = b / tiles;
    t = (int)(b % tiles);
}

template <class P, class T, Lie YL>
__global__ __launch_bounds__(P::THREADS, P::THREADS <= 256 ? 2 : 1) void grouped_nn_kernel(
    const T* __restrict__ A, int64_t n, int64_t lda, int K, const T* __restrict__ B, int C, int groups, const int64_t* __restrict__ ptr,
    T* __restrict__ out, int64_t ldo, int col_tiles, int slices, int whole_out) {
    __shared__ __align__(16) unsigned short S[P::kLds];
    int64_t slot;
    int tile;
    place(col_tiles, slices, slot, tile);
    const int g = group_of_slot(ptr, groups, n, P::BM, slot);
    const int64_t skip = slot - first_slot(ptr, g, n, P::BM);
    const int64_t r0 = bound_of(ptr, g, n) + skip * P::BM, end = bound_of(ptr, g + 1, n);
    if (skip < 0 || r0 >= end) return;
    const int c0 = tile * P::BN, rows = end - r0 < P::BM ? (int)(end - r0) : P::BM;
    const T* Bg = B + (int64_t)g * K * C;
    floatx16 acc[P::TM][P::TN];
    const View<T> x{A + r0 * lda, lda, rows, K};
    const View<T> y = YL == kAlong ? View<T>{Bg + (int64_t)c0 * K, K, C - c0, K} : View<T>{Bg + c0, C, C - c0, K};
    P::run(acc, x, y, S);
    P::drain(acc, S, [&](int row, int col, float4 v) {
        if (row < rows && c0 + col < C) put(out + (r0 + row) * ldo, c0 + col, C, v, whole_out);
    });
}

// Rows of a group beyond `most` go to further workgroups of their own, whose sums are added by grouped_tn_reduce_kernel: the i-th such
// part of group g is number 2 (ptr[g] / most + i) (+ 1 unless it is the group's last) of `partial`.  (Groups in parts have more than
// `most` rows: no two parts that begin in the same stretch of `most` rows are both last or both not.)
__device__ __forceinline__ int64_t part_place(int64_t lo, int64_t hi, int64_t most, int64_t i) {
    return 2 * (lo / most + i) + (lo + (i + 1) * most < hi ? 1 : 0);
}

template <class P, class T, class O>
__global__ __launch_bounds__(P::THREADS, P::THREADS <= 256 ? 2 : 1) void grouped_tn_kernel(
    const T* __restrict__ A, int64_t n, int64_t lda, int K, const T* __restrict__ G, int64_t ldg, int C, int groups,
    const int64_t* __restrict__ ptr, O* __restrict__ out, float* __restrict__ partial, int64_t most, int64_t part_size, int col_tiles, int tiles,
    int slices, int whole_out) {
    __shared__ __align__(16) unsigned short S[P::kLds];
    int64_t slot;
    int tile;
    place(tiles, slices, slot, tile);
    const int g = group_of_slot(ptr, groups, n, most, slot);
    const int64_t lo = bound_of(ptr, g, n), end = bound_of(ptr, g + 1, n), hi = end > lo ? end : lo;
    const int64_t i = slot - first_slot(ptr, g, n, most), r0 = lo + i * most;
    if (i < 0 || (i > 0 && r0 >= hi)) return;
    const int i0 = tile / col_tiles * P::BM, c0 = tile % col_tiles * P::BN;
    floatx16 acc[P::TM][P::TN];
    const int64_t depth = hi - r0 < most ? hi - r0 : most;
    P::run(acc, View<T>{A + r0 * lda + i0, lda, K - i0, depth}, View<T>{G + r0 * ldg + c0, ldg, C - c0, depth}, S);
    if (hi - lo > most) {
        float* to = partial + part_place(lo, hi, most, i) * part_size;
        P::drain(acc, S, [&](int row, int col, float4 v) {
            if (i0 + row < K && c0 + col < C) put(to + (int64_t)(i0 + row) * C, c0 + col, C, v, whole_out);
        });
    } else {
        O* to = out + (int64_t)g * K * C;
        P::drain(acc, S, [&](int row, int col, float4 v) {
            if (i0 + row < K && c0 + col < C) put<true>(to + (int64_t)(i0 + row) * C, c0 + col, C, v, whole_out);
        });
    }
}

template <class O>
__global__ __launch_bounds__(256) void grouped_tn_reduce_kernel(const float* __restrict__ partial, int64_t n, const int64_t* __restrict__ ptr, int64_t most,
                                                                int64_t part_size, int64_t count, O* __restrict__ out) {
    const int g = blockIdx.y;
    const int64_t lo = bound_of(ptr, g, n), hi = bound_of(ptr, g + 1, n);
    if (hi - lo <= most) return;
    const int64_t parts = (hi - lo + most - 1) / most;
    for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < count; e += (int64_t)gridDim.x * 1024) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int64_t i = 0; i < parts; ++i) {
            const float4 v = *reinterpret_cast<const float4*>(partial + part_place(lo, hi, most, i) * part_size + e);      // (parts are padded to fours)
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        const float w[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (e + k < count) out[(int64_t)g * count + e + k] = (O)w[k];
    }
}

template <class F>
void with_type(int type, F f) {
    if (type == kBf16) f((__bf16*)nullptr);
    else if (type == kF16) f((_Float16*)nullptr);
    else f((float*)nullptr);
}

// Tiles: wavefronts, 32 x 32 accumulators of one; then, through registers, contraction per step, steps ahead, LDS buffers, or, straight to
// LDS, stages, sets of wavefronts and contraction per step.
//   kLarge  operands are read from LDS once for 128 x 256 results (two workgroups a compute unit) or 256 x 256.  16-bit transform, K = 512,
//           500000 rows: 128 x 256 391 us, 256 x 256 407, 128 x 128 431 (a library product of one matrix: 389); fp32, through registers,
//           is faster in 128 x 128 at every size tried (200000 x 256 x 256 170 us for 179, 20000 x 1024 x 1024 228 for 281) and has no larger
//           ones.  16-bit wgrad: 256 x 256 202 us, 128 x 256 214 (16384 x 2048 x 1024, 64 ragged groups).
//   kMiddle 128 x 128;  kSmall 64 x 64, where larger ones would not give every compute unit one
//   kFew    32 x 64, for groups of a few rows: reading the weights is all there is to it, from many places and far ahead.
//   kLone.. the same tiles, with more sets of wavefronts to share the contraction, where that leaves no compute unit a second workgroup
//           anyway.  fp32: one row of 512 x 512 15.7 -> 9.3 us, 16 rows through 16 x 2048 x 1024 57 -> 37, but 64 rows through 64 of them
//           103 -> 125; 300 x 1000 x 1000 in 4 groups 26.9 -> 24.5, but 100000 x 64 x 64 16.5 -> 28.
template <class T> constexpr int kStep = 128 / sizeof(T);
enum Size { kLarge, kMiddle, kSmall, kFew, kLoneSmall, kLoneFew };
template <class T, Lie X, Lie Y, Mode M, bool STRAIGHT = sizeof(T) == 2 && M == kWhole>
struct Sizes {
    using Large = Product<T, X, Y, M, 2, 2, 2, 4, kStep<T> / 2, 1, 1>;
    using Middle = Product<T, X, Y, M, 2, 2, 2, 2, kStep<T>, 1, 1>;
    using Small = Product<T, X, Y, M, 2, 2, 1, 1, kStep<T>, 2, 2>;
    using Few = Product<T, X, Y, M, 1, 2, 1, 1, kStep<T>, 4, 2>;
    using LoneSmall = Product<T, X, Y, M, 2, 2, 1, 1, kStep<T>, 1, 2, 2>;
    using LoneFew = Product<T, X, Y, M, 1, 2, 1, 1, kStep<T>, 2, 2, 4>;
};
template <class T, Lie X, Lie Y, Mode M>
struct Sizes<T, X, Y, M, true> {
    using Large = std::conditional_t<X == kAlong, Direct<T, X, Y, 2, 2, 2, 4, 3, 1, 32>, Direct<T, X, Y, 2, 4, 4, 2, 2>>;
    using Middle = Direct<T, X, Y, 2, 2, 2, 2, 2>;
    using Small = Direct<T, X, Y, 2, 2, 1, 1, 4>;
    using Few = Direct<T, X, Y, 1, 2, 1, 1, 3, 4>;             // (64 rows through 64 x 2048 x 1024: 64 us, with two sets 72)
    using LoneSmall = Direct<T, X, Y, 2, 2, 1, 1, 2, 4>;
    using LoneFew = Few;
};
template <Size SIZE, class S>
auto sized() {
    if constexpr (SIZE == kLarge) return (typename S::Large*)nullptr;
    else if constexpr (SIZE == kMiddle) return (typename S::Middle*)nullptr;
    else if constexpr (SIZE == kSmall) return (typename S::Small*)nullptr;
    else if constexpr (SIZE == kFew) return (typename S::Few*)nullptr;
    else if constexpr (SIZE == kLoneSmall) return (typename S::LoneSmall*)nullptr;
    else return (typename S::LoneFew*)nullptr;
}
template <Size SIZE, class T, Lie X, Lie Y, Mode M>
using Sized = std::remove_pointer_t<decltype(sized<SIZE, Sizes<T, X, Y, M>>())>;
constexpr int kSizeCols[] = {256, 128, 64, 64, 64, 64}, kNnRows[] = {128, 128, 64, 32, 64, 32};
int tn_rows(Size s, bool straight) { return s == kLarge ? straight ? 256 : 128 : kNnRows[s]; }
constexpr int64_t kCus = 256;

int64_t over(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The largest tiles that give every compute unit a workgroup.
Size nn_size(int64_t n, int C, int groups, bool straight) {
    const int64_t hit = std::min<int64_t>(n, groups), rows = over(n, hit);            // rows of a group that has any, if they share alike
    for (Size s : {kLarge, kMiddle, kSmall}) {
        if (s == kLarge && !straight) continue;
        const bool fits = C > kSizeCols[s] / 2 && rows > kNnRows[s] / 2;
        if (fits && (n / kNnRows[s] + hit / 2) * over(C, kSizeCols[s]) >= kCus) return s;
    }
    const Size s = rows > 32 ? kSmall : kFew;
    const int64_t tiles = (n / kNnRows[s] + hit) * over(C, kSizeCols[s]);
    return s == kSmall ? tiles <= kCus ? kLoneSmall : s : tiles <= 2 * kCus ? kLoneFew : s;
}

struct TnPlan { Size size; int64_t most, parts; };
TnPlan tn_plan(int64_t n, int K, int C, int groups, bool straight) {
    for (Size s : {kLarge, kMiddle, kSmall}) {
        const int rows = tn_rows(s, straight);
        if (s != kSmall && (K <= rows / 2 || C <= kSizeCols[s] / 2)) continue;
        const int64_t tiles = over(K, rows) * over(C, kSizeCols[s]);
        TnPlan p{s, n > 0 ? n : 1, 0};
        // too few tiles for two workgroups a compute unit: the rows are shared out too, 256 of them at least; large tiles only where 512 are
        // left to each (20000 x 512 x 512 fp32 in 8 groups: 128 x 256 104 us, 128 x 128 88; 200000 x 256 x 256: 169 and 207)
        const int64_t share = over(n * tiles, 2 * kCus);
        if (s == kLarge && share < 512) continue;
        if (tiles * groups < 2 * kCus * 2) p.most = std::max<int64_t>(256, over(share, 64) * 64);
        p.parts = p.most < n ? 2 * (n / p.most + 1) : 0;
        if (s == kSmall && (n / p.most + groups) * tiles <= kCus) p.size = kLoneSmall;
        return p;
    }
    return {};
}
int64_t part_floats(int K, int C) { return over((int64_t)K * C, 4) * 4; }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

template <class T, Lie YL, Mode MODE>
void nn_launch(hipStream_t s, const GroupedNN& a, Size size, bool whole_out) {
    auto go = [&](auto sized) {
        using P = Sized<decltype(sized)::value, T, kAlong, YL, MODE>;
        const int col_tiles = (int)over(a.C, P::BN);
        const int64_t blocks = (a.n / P::BM + a.groups) * col_tiles;
        grouped_nn_kernel<P, T, YL><<<dim3((unsigned)blocks), dim3(P::THREADS), 0, s>>>(
            (const T*)a.A, a.n, a.lda, a.K, (const T*)a.B, a.C, a.groups, a.ptr, (T*)a.out, a.ldo, col_tiles, a.n / P::BM >= a.groups, whole_out);
    };
    if (size == kLarge) {
        if constexpr (sizeof(T) == 2 && MODE == kWhole) go(std::integral_constant<Size, kLarge>());
    } else if (size == kMiddle) go(std::integral_constant<Size, kMiddle>());
    else if (size == kSmall) go(std::integral_constant<Size, kSmall>());
    else if (size == kFew) go(std::integral_constant<Size, kFew>());
    else if (size == kLoneSmall) go(std::integral_constant<Size, kLoneSmall>());
    else go(std::integral_constant<Size, kLoneFew>());
}

template <class T, Mode MODE, class O>
void tn_launch(hipStream_t s, const GroupedTN& a, const TnPlan& plan) {
    float* partial = (float*)a.scratch;
    const int64_t count = (int64_t)a.K * a.C;
    auto go = [&](auto sized) {
        using P = Sized<decltype(sized)::value, T, kAcross, kAcross, MODE>;
        const int col_tiles = (int)over(a.C, P::BN), tiles = col_tiles * (int)over(a.K, P::BM);
        const int64_t blocks = (a.n / plan.most + a.groups) * tiles;
        grouped_tn_kernel<P, T, O><<<dim3((unsigned)blocks), dim3(P::THREADS), 0, s>>>(
            (const T*)a.A, a.n, a.lda, a.K, (const T*)a.G, a.ldg, a.C, a.groups, a.ptr, (O*)a.out, partial, plan.most, part_floats(a.K, a.C), col_tiles,
            tiles, a.n / plan.most >= a.groups, a.C % 4 == 0 && ((uintptr_t)a.out & (4 * sizeof(O) - 1)) == 0);
    };
    if (plan.size == kLarge) go(std::integral_constant<Size, kLarge>());
    else if (plan.size == kMiddle) go(std::integral_constant<Size, kMiddle>());
    else if (plan.size == kSmall) go(std::integral_constant<Size, kSmall>());
    else go(std::integral_constant<Size, kLoneSmall>());
    if (plan.parts > 0) {
        const unsigned bx = (unsigned)std::min<int64_t>(over(count, 1024), std::max<int64_t>(1, 8 * kCus / a.groups));
        for (int g0 = 0; g0 < a.groups; g0 += 65535)       // (a grid's second dimension)
            grouped_tn_reduce_kernel<O><<<dim3(bx, (unsigned)std::min(a.groups - g0, 65535)), dim3(256), 0, s>>>(
                partial, a.n, a.ptr + g0, plan.most, part_floats(a.K, a.C), count, (O*)a.out + (int64_t)g0 * count);
    }
}

}  // namespace

// (whole chunks can go straight to LDS, or not: the most workgroups of either, and the scratch that serves both)
int64_t grouped_nn_blocks(int64_t n, int C, int groups) {
    int64_t most = 0;
    for (bool straight : {false, true}) {
        if (n == 0) continue;
        const Size s = nn_size(n, C, groups, straight);
        most = std::max(most, (n / kNnRows[s] + groups) * over(C, kSizeCols[s]));
    }
    return most;
}
int64_t grouped_tn_blocks(int64_t n, int K, int C, int groups) {
    int64_t most = 0;
    for (bool straight : {false, true}) {
        const TnPlan p = tn_plan(n, K, C, groups, straight);
        most = std::max(most, (n / p.most + groups) * over(K, tn_rows(p.size, straight)) * over(C, kSizeCols[p.size]));
    }
    return most;
}
size_t grouped_tn_scratch(int64_t n, int K, int C, int groups) {
    return sizeof(float) * std::max(tn_plan(n, K, C, groups, false).parts, tn_plan(n, K, C, groups, true).parts) * part_floats(K, C);
}

void launch_grouped_nn(hipStream_t s, int type, const GroupedNN& a) {
    if (a.n == 0) return;
    with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int64_t Q = 16 / sizeof(T);
        const bool whole = a.K % 8 == 0 && a.lda % Q == 0 && aligned16(a.A) && aligned16(a.B) && a.lda * (int64_t)sizeof(T) <= kMostRow && (a.transposed || a.C % 8 == 0);
        const bool whole_out = a.C % 4 == 0 && a.ldo % 4 == 0 && ((uintptr_t)a.out & (4 * sizeof(T) - 1)) == 0;
        const Size size = nn_size(a.n, a.C, a.groups, whole && sizeof(T) == 2);
        if (a.transposed) {
            if (whole) nn_launch<T, kAlong, kWhole>(s, a, size, whole_out);
            else nn_launch<T, kAlong, kAny>(s, a, size, whole_out);
        } else {
            if (whole) nn_launch<T, kAcross, kWhole>(s, a, size, whole_out);
            else nn_launch<T, kAcross, kAny>(s, a, size, whole_out);
        }
    });
}

void launch_grouped_tn(hipStream_t s, int type, int out_type, const GroupedTN& a) {
    with_type(type, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        constexpr int64_t Q = 16 / sizeof(T);
        const bool whole = a.K % 8 == 0 && a.C % 8 == 0 && a.lda % Q == 0 && a.ldg % Q == 0 && aligned16(a.A) && aligned16(a.G) &&
                           std::max(a.lda, a.ldg) * (int64_t)sizeof(T) <= kMostRow;
        const TnPlan plan = tn_plan(a.n, a.K, a.C, a.groups, whole && sizeof(T) == 2);
        auto go = [&](auto* o) {
            using O = std::remove_pointer_t<decltype(o)>;
            if (whole) tn_launch<T, kWhole, O>(s, a, plan);
            else tn_launch<T, kAny, O>(s, a, plan);
        };
        if (out_type == kF32) go((float*)nullptr);
        else go((T*)nullptr);
    });
}

}  // namespace cadmm
