// Tiles of matrix products on the 16-bit matrix cores (v_mfma_f32_32x32x16_bf16 / _f16), shared by the products over groups of rows
// and by the orthogonalised updates.  A workgroup forms BM x BN results acc(i, j) = sum_k X(i, k) Y(j, k).
//
// Operands.  Either may lie with its contraction along the rows in memory (an element's k is its column: kAlong) or across
// them (an element's k is its row: kAcross), and is one of
//   bf16 / fp16   as they are, one product per pair of elements;
//   Pair          two planes of fp16 whose sum is the value, 22 bits of significand: three products (the fourth is below 2^-22);
//   float         split on the way into three bf16 parts, exactly (8 + 8 + 8 bits): six products (the other three are below 2^-24).
//
// Way of the data: 16-byte chunks of eight k (kAlong) or eight i (kAcross) from memory into registers, PF steps of BK ahead; from
// there, split where need be, into one of two LDS buffers; from there into the matrix cores' operand layout, eight k of one
// row per lane.  One barrier per step.
//   kAlong tiles are kept in that layout, 64 lanes x 16 bytes for every 32 rows and 16 k, with the rows permuted by the chunk's number
//   so that the chunks of one row, which neighbouring lanes store, fall into different banks.
//   kAcross tiles are kept as rows of k; ds_read_b64_tr_b16 turns 4 k x 16 i over 16 lanes into four k of one i per lane.  The four rows
//   it reads at once are kept apart by a permutation of their 64-byte pieces.
// Results come out as the transposed product's, so that a lane holds four neighbouring columns of one row.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace cadmm {
namespace tile {

typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef unsigned uintx4 __attribute__((ext_vector_type(4)));

struct Pair {};                         // an operand of two fp16 planes
enum Lie { kAlong, kAcross };
// kWhole: chunks are there or not at all, and 16-byte aligned.  kAny: rows of any length at any element.
enum Mode { kWhole, kAny };

// X(i, k), i < rows, k < depth; `plane`: elements from the high to the low plane of a Pair.
template <class T> struct View {
    using Element = T;
    const T* p; int64_t ld; int rows; int64_t depth; int64_t plane;
};
template <> struct View<Pair> {
    using Element = _Float16;
    const _Float16* p; int64_t ld; int rows; int64_t depth; int64_t plane;
};

template <class T> inline constexpr int kParts = 1;
template <> inline constexpr int kParts<Pair> = 2;
template <> inline constexpr int kParts<float> = 3;

// a chunk of eight elements as loaded
template <class T> struct Chunk { uintx4 v[1]; };
template <> struct Chunk<Pair> { uintx4 v[2]; };
template <> struct Chunk<float> { uintx4 v[2]; };

typedef unsigned uintx4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned uintx4a2 __attribute__((ext_vector_type(4), aligned(2)));
template <int BYTES>
__device__ __forceinline__ uintx4 load16(const void* p) {              // 16 bytes at any multiple of BYTES
    if constexpr (BYTES == 16) return *reinterpret_cast<const uintx4*>(p);
    else if constexpr (BYTES == 4) return *reinterpret_cast<const uintx4a4*>(p);
    else return *reinterpret_cast<const uintx4a2*>(p);
}

// Loading and putting the chunk right are two steps, so that nothing waits for a load before the chunk is stored to LDS; and no
// load is under a condition that differs between lanes.  `row`: its row in memory, of which `width` elements exist; c: the first of the
// chunk's eight columns.  What lies past the row's end becomes zero.
template <class T, Mode MODE>
__device__ __forceinline__ void fetch(Chunk<T>& q, const typename View<T>::Element* row, int64_t plane, int c, int width) {
    using E = typename View<T>::Element;
    if constexpr (MODE == kWhole) {
        const E* at = row + (c < width ? c : 0);
        if constexpr (sizeof(E) == 4) { q.v[0] = load16<16>(at); q.v[1] = load16<16>(at + 4); }
        else {
            q.v[0] = load16<16>(at);
            if constexpr (kParts<T> == 2) q.v[1] = load16<16>(at + plane);
        }
    } else if (width >= 8) {                                            // (uniform) the last chunk is moved back to end with the row
        const E* at = row + (c + 8 <= width ? c : width - 8);
        q.v[0] = load16<sizeof(E)>(at);
        if constexpr (sizeof(E) == 4) q.v[1] = load16<sizeof(E)>(at + 4);
    } else {
        E v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row[c + e < width ? c + e : width - 1];
        __builtin_memcpy(&q, v, 8 * sizeof(E));
    }
}
template <class T, Mode MODE>
__device__ __forceinline__ void settle(Chunk<T>& q, int c, int width, bool in) {
    using E = typename View<T>::Element;
    constexpr int N = sizeof(Chunk<T>) / 4;
    unsigned w[N];
    __builtin_memcpy(w, &q, sizeof(q));
    if constexpr (MODE == kWhole) {
        const bool there = in && c < width;
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = there ? w[e] : 0u;
    } else {
        const int off = !in ? 8 : width < 8 || c + 8 <= width ? 0 : c + 8 - width;       // elements of the chunk that come before column c
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int s = 4; s > 0; s >>= 1)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = (off & s) ? (e + s < 8 ? w[e + s] : 0u) : w[e];
        } else {
            if (off & 4) { w[0] = w[2]; w[1] = w[3]; w[2] = w[3] = 0u; }
            if (off & 2) { w[0] = w[1]; w[1] = w[2]; w[2] = w[3]; w[3] = 0u; }
            if (off & 1) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = w[e] >> 16 | (e < 3 ? w[e + 1] << 16 : 0u);
            }
        }
        const int left = off >= 8 ? 0 : width < 8 ? width - c : 8;          // of a short row: the elements that exist
#pragma unroll
        for (int e = 0; e < N; ++e) {
            if constexpr (sizeof(E) == 4) w[e] = e < left ? w[e] : 0u;
            else w[e] = 2 * e + 1 < left ? w[e] : 2 * e < left ? w[e] & 0xffffu : 0u;
        }
    }
    __builtin_memcpy(&q, w, sizeof(q));
}

// two fp32 numbers -> their three bf16 parts, each pair packed into one dword (low half = first number)
__device__ __forceinline__ void three_parts(float x0, float x1, unsigned& h, unsigned& m, unsigned& l) {
    const unsigned u0 = __float_as_uint(x0), u1 = __float_as_uint(x1);
    h = __builtin_amdgcn_perm(u1, u0, 0x07060302u);                     // upper halves of u1 and u0
    const float r0 = x0 - __uint_as_float(u0 & 0xFFFF0000u), r1 = x1 - __uint_as_float(u1 & 0xFFFF0000u);          // exact
    const unsigned v0 = __float_as_uint(r0), v1 = __float_as_uint(r1);
    m = __builtin_amdgcn_perm(v1, v0, 0x07060302u);
    const float s0 = r0 - __uint_as_float(v0 & 0xFFFF0000u), s1 = r1 - __uint_as_float(v1 & 0xFFFF0000u);          // exact, 8 bits at most
    l = __builtin_amdgcn_perm(__float_as_uint(s1), __float_as_uint(s0), 0x07060302u);
}

__device__ __forceinline__ int along_swizzle(int chunk) { return (chunk & 3) << 2 | (chunk >> 2) << 1; }
template <int ROWS>
__device__ __forceinline__ int across_swizzle(int k) { return ROWS >= 128 ? (k & 3) << 2 : ROWS == 64 ? (k & 2) << 1 : 0; }

// One operand's tile: ROWS rows (i) by BK of the contraction, carried by THREADS threads.
template <class T, Lie LIE, Mode MODE, int ROWS, int BK, int THREADS, int PF>
struct Operand {
    using E = typename View<T>::Element;
    static constexpr int kParts_ = kParts<T>;
    static constexpr int kPlane = ROWS * BK;                            // 16-bit elements of a part
    static constexpr int kSize = kParts_ * kPlane;                      // of a buffer
    static constexpr int kPerRow = (LIE == kAlong ? BK : ROWS) / 8;       // chunks per row in memory
    static constexpr int kChunks = ROWS * BK / 8;
    static constexpr int kEach = (kChunks + THREADS - 1) / THREADS;
    static constexpr bool kIdle = kChunks % THREADS != 0;                 // some threads carry none at the last round
    Chunk<T> q[PF][kEach];
    const E* at[kEach];                                                  // start of the row (kAlong), or of the row of the step (kAcross)

    __device__ __forceinline__ static int row_of(int u) { return (threadIdx.x + u * THREADS) / kPerRow; }
    __device__ __forceinline__ static int chunk_of(int u) { return (threadIdx.x + u * THREADS) % kPerRow; }
    __device__ __forceinline__ static bool carries(int u) { return !kIdle || (int)threadIdx.x + u * THREADS < kChunks; }

    __device__ __forceinline__ void begin(const View<T>& x) {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int r = row_of(u);
            if constexpr (LIE == kAlong) at[u] = x.p + (int64_t)(r < x.rows ? r : x.rows - 1) * x.ld;    // rows past the end: any (their results are not stored)
            else at[u] = x.p + (int64_t)r * x.ld;
        }
    }
    // the step that begins at k0 < depth, into slot s
    __device__ __forceinline__ void load(const View<T>& x, int64_t k0, int s) {
        const int64_t rest = x.depth - k0;
        const int left = (int)(rest < BK ? rest : BK);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            if constexpr (LIE == kAlong) {
                const int c = 8 * chunk_of(u);
                if (MODE == kWhole) fetch<T, MODE>(q[s][u], at[u] + (c < left ? k0 : 0), x.plane, c < left ? c : 0, BK);
                else fetch<T, MODE>(q[s][u], at[u], x.plane, (int)k0 + c, (int)x.depth);
            } else {
                const bool in = row_of(u) < left;
                const E* row = in ? at[u] : x.p;                         // (row 0 of the view is there)
                fetch<T, MODE>(q[s][u], row, x.plane, 8 * chunk_of(u), x.rows);
                at[u] += BK * x.ld;
            }
        }
    }
    // slot s, which holds the step that begins at k0, to LDS
    __device__ __forceinline__ void store(const View<T>& x, int64_t k0, int s, unsigned short* S) {
        const int64_t rest = x.depth - k0;
        const int left = (int)(rest < BK ? rest : BK);
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const int r = row_of(u), ch = chunk_of(u);
            Chunk<T> v = q[s][u];
            int o;
            if constexpr (LIE == kAlong) {
                if (MODE == kWhole) settle<T, MODE>(v, 8 * ch, left, true);
                else settle<T, MODE>(v, (int)k0 + 8 * ch, (int)x.depth, 8 * ch < left);
                o = ((r >> 5) * (BK / 16) + (ch >> 1)) * 64 + (ch & 1) * 32 + ((r & 31) ^ along_swizzle(ch));
            } else {
                settle<T, MODE>(v, 8 * ch, x.rows, r < left && 8 * ch < x.rows);
                o = r * (ROWS / 8) + (ch ^ across_swizzle<ROWS>(r));
            }
            if (!carries(u)) continue;
            uintx4* to = reinterpret_cast<uintx4*>(S) + o;
            if constexpr (kParts_ == 3) {
                unsigned w[8], h[4], m[4], l[4];
                __builtin_memcpy(w, &v, sizeof(w));
#pragma unroll
                for (int e = 0; e < 4; ++e) three_parts(__uint_as_float(w[2 * e]), __uint_as_float(w[2 * e + 1]), h[e], m[e], l[e]);
                to[0] = uintx4{h[0], h[1], h[2], h[3]};
                to[kPlane / 8] = uintx4{m[0], m[1], m[2], m[3]};
                to[2 * (kPlane / 8)] = uintx4{l[0], l[1], l[2], l[3]};
            } else {
                to[0] = v.v[0];
                if constexpr (kParts_ == 2) to[kPlane / 8] = v.v[1];
            }
        }
    }
    // rows 32 b .. 32 b + 31, k 16 s .. 16 s + 15, part p, as the matrix cores take them
    __device__ __forceinline__ static uintx4 operand(const unsigned short* S, int b, int s, int p) {
        const int lane = threadIdx.x & 63;
        S += p * kPlane;
        if constexpr (LIE == kAlong) {
            const int h = lane >> 5;
            return *(reinterpret_cast<const uintx4*>(S) + (b * (BK / 16) + s) * 64 + h * 32 + ((lane & 31) ^ along_swizzle(2 * s + h)));
        } else {
            const int k = 16 * s + 8 * (lane >> 5) + ((lane & 15) >> 2);
            const int col = 32 * b + (lane & 16) + 4 * (lane & 3);
            const unsigned short* from = S + k * ROWS + (((col >> 3) ^ across_swizzle<ROWS>(k)) << 3) + (col & 7);
            typedef __attribute__((address_space(3))) shortx4* Lds;
            const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)from);
            const shortx4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from + 4 * ROWS));
            uintx4 v;
            __builtin_memcpy(&v, &a, 8);
            __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &c, 8);
            return v;
        }
    }
};

template <class T>
__device__ __forceinline__ floatx16 multiply(uintx4 a, uintx4 b, floatx16 c) {
    if constexpr (__is_same(T, Pair) || __is_same(T, _Float16))
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// WM x WN wavefronts, TM x TN accumulators of 32 x 32 each.
template <class T, Lie XL, Lie YL, Mode MODE, int WM_, int WN_, int TM_, int TN_, int BK_, int PF_>
struct Product {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, BK = BK_, PF = PF_;
    static constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, THREADS = 64 * WM * WN;
    using X = Operand<T, XL, MODE, BM, BK, THREADS, PF>;
    using Y = Operand<T, YL, MODE, BN, BK, THREADS, PF>;
    static constexpr int P = kParts<T>;
    static constexpr int kBuffer = X::kSize + Y::kSize;
    // results on their way out: 32 rows by up to 64 columns of a wavefront, at a time
    static constexpr int kSlabCols = TN >= 2 ? 64 : 32, kSlabLd = kSlabCols + 4;
    static constexpr int kSlabs = WM * WN * 32 * kSlabLd * 2;            // in 16-bit elements
    static constexpr int kLds = 2 * kBuffer > kSlabs ? 2 * kBuffer : kSlabs;

    __device__ __forceinline__ static void step(floatx16 (&acc)[TM][TN], const unsigned short* S) {
        const int wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int s = 0; s < BK / 16; ++s) {
            uintx4 a[P][TM];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < TM; ++i) a[p][i] = X::operand(S, wm * TM + i, s, p);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                uintx4 b[P];
#pragma unroll
                for (int p = 0; p < P; ++p) b[p] = Y::operand(S + X::kSize, wn * TN + j, s, p);
#pragma unroll
                for (int i = 0; i < TM; ++i) {                            // smallest terms first
                    floatx16 c = acc[i][j];
                    if constexpr (P == 3) {
                        c = multiply<T>(b[0], a[2][i], c);
                        c = multiply<T>(b[2], a[0][i], c);
                        c = multiply<T>(b[1], a[1][i], c);
                    }
                    if constexpr (P >= 2) {
                        c = multiply<T>(b[0], a[1][i], c);
                        c = multiply<T>(b[1], a[0][i], c);
                    }
                    acc[i][j] = multiply<T>(b[0], a[0][i], c);
                }
            }
        }
    }

    __device__ __forceinline__ static void run(floatx16 (&acc)[TM][TN], const View<T>& x, const View<T>& y, unsigned short* S) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        const int64_t depth = x.depth;
        if (depth <= 0) return;
        X X_;
        Y Y_;
        X_.begin(x);
        Y_.begin(y);
#pragma unroll
        for (int s = 0; s < PF; ++s)
            if (s * BK < depth) { X_.load(x, s * BK, s); Y_.load(y, s * BK, s); }
        X_.store(x, 0, 0, S);
        Y_.store(y, 0, 0, S + X::kSize);
        __syncthreads();
        int buffer = 0;
        for (int64_t k0 = 0; k0 < depth; k0 += PF * BK) {
#pragma unroll
            for (int u = 0; u < PF; ++u) {
                const int64_t k = k0 + u * BK;
                if (k >= depth) break;                                   // (uniform)
                if (k + PF * BK < depth) { X_.load(x, k + PF * BK, u); Y_.load(y, k + PF * BK, u); }
                step(acc, S + buffer * kBuffer);
                buffer ^= 1;
                if (k + BK < depth) {
                    X_.store(x, k + BK, (u + 1) % PF, S + buffer * kBuffer);
                    Y_.store(y, k + BK, (u + 1) % PF, S + buffer * kBuffer + X::kSize);
                }
                __syncthreads();
            }
        }
    }

    // f(row, column, four results) for every quad of the tile, 16 (TN >= 2) or 8 neighbouring lanes along a row.  Every wavefront passes
    // its results through LDS of its own.  MIRROR: what f returns goes on to m(column, row, four results of neighbouring rows).
    template <bool MIRROR, class F, class M>
    __device__ __forceinline__ static void drain(floatx16 (&acc)[TM][TN], unsigned short* S, F f, M m) {
        constexpr int J = kSlabCols / 32, Q = kSlabCols / 4;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
        float* C = reinterpret_cast<float*>(S) + wave * 32 * kSlabLd;
        auto settled = [] {                                             // a wavefront's LDS accesses are done in their order
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j0 = 0; j0 < TN; j0 += J) {
                const int r0 = (wm * TM + i) * 32, c0 = (wn * TN + j0) * 32;
                settled();
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *reinterpret_cast<float4*>(C + (lane & 31) * kSlabLd + 32 * j + 2 * r + 4 * (lane >> 5)) =
                            make_float4(acc[i][j0 + j][r], acc[i][j0 + j][r + 1], acc[i][j0 + j][r + 2], acc[i][j0 + j][r + 3]);
                settled();
#pragma unroll
                for (int u = 0; u < 32 * Q / 64; ++u) {
                    const int row = (lane + 64 * u) / Q, col = (lane + 64 * u) % Q * 4;
                    float4* at = reinterpret_cast<float4*>(C + row * kSlabLd + col);
                    if constexpr (MIRROR) *at = f(r0 + row, c0 + col, *at);
                    else f(r0 + row, c0 + col, *at);
                }
                if constexpr (MIRROR) {
                    settled();
#pragma unroll
                    for (int u = 0; u < 32 * Q / 64; ++u) {
                        const int row = lane % 8 * 4, col = lane / 8 + 8 * u;
                        const float* at = C + row * kSlabLd + col;
                        m(c0 + col, r0 + row, make_float4(at[0], at[kSlabLd], at[2 * kSlabLd], at[3 * kSlabLd]));
                    }
                }
            }
    }
    template <class F>
    __device__ __forceinline__ static void drain(floatx16 (&acc)[TM][TN], unsigned short* S, F f) { drain<false>(acc, S, f, [](int, int, float4) {}); }
};

// One quad of a row of `width` results at column c (c < width), the row at `to`; whole: width and the row's place are multiples of four
// elements.
template <class O>
__device__ __forceinline__ void put(O* to, int c, int width, float4 v, bool whole) {
    typedef O ox4 __attribute__((ext_vector_type(4)));
    const ox4 q = {(O)v.x, (O)v.y, (O)v.z, (O)v.w};
    if (whole) *reinterpret_cast<ox4*>(to + c) = q;
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < width) to[c + e] = q[e];
    }
}

}  // namespace tile
}  // namespace cadmm
