// Tiles of matrix products on the 16-bit matrix cores (v_mfma_f32_32x32x16_bf16 / _f16), shared by the products over groups of rows
// and by the orthogonalised updates.  A workgroup forms BM x BN results acc(i, j) = sum_k X(i, k) Y(j, k).
//
// Operands.  Either may lie with its contraction along the rows in memory (an element's k is its column: kAlong) or across
// them (an element's k is its row: kAcross), and is one of
//   bf16 / fp16   as they are, one product per pair of elements;
//   Pair          two fp16 whose sum is the value, 22 bits of significand: three products (the fourth is below 2^-22); eight high
//                 parts are followed by their eight low ones in memory (straight to LDS only: Direct, below);
//   float         split on the way into three bf16 parts, exactly (8 + 8 + 8 bits): six products (the other three are below 2^-24 together).
//
// Way of the data: chunks of eight k (kAlong) or eight i (kAcross) from memory into registers, PF steps of BK ahead; from there,
// split where need be, to LDS; from there into the matrix cores' operand layout, eight k of one row per lane.  With two LDS
// buffers there is one barrier per step; with one there are two, and as much more of the contraction per step.  A step takes whole
// lines (128 bytes) of rows that lie along the contraction: what is left of a line is gone from the L1 by the next step (with
// 32 bytes a step, products of Pairs ran at 36 % of the matrix cores' cycles, whatever was loaded ahead).
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

struct Pair {};                         // an operand of two fp16 parts
enum Lie { kAlong, kAcross };
// kWhole: chunks are there or not at all, 16-byte aligned, and kMostRow bytes at most from one row to the next, so that a place in a
// tile is a base and 32 bits.  kAny: rows of any length and distance, at any element.
enum Mode { kWhole, kAny };
constexpr int64_t kMostRow = (int64_t)1 << 22;

// X(i, k), i < rows, k < depth; ld: elements from one row in memory to the next (of a Pair: fp16 numbers, two an element).
template <class T> struct View {
    using Element = T;
    const T* p; int64_t ld; int rows; int64_t depth;
};
template <> struct View<Pair> {
    using Element = _Float16;
    const _Float16* p; int64_t ld; int rows; int64_t depth;
};

template <class T> inline constexpr int kParts = 1;
template <> inline constexpr int kParts<Pair> = 2;
template <> inline constexpr int kParts<float> = 3;

// a chunk of eight elements as loaded
template <class T> struct Chunk { uintx4 v[1]; };
template <> struct Chunk<float> { uintx4 v[2]; };

typedef unsigned uintx4a4 __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned uintx4a2 __attribute__((ext_vector_type(4), aligned(2)));
template <int BYTES>
__device__ __forceinline__ uintx4 load16(const void* p) {              // 16 bytes at any multiple of BYTES
    if constexpr (BYTES == 4) return *reinterpret_cast<const uintx4a4*>(p);
    else return *reinterpret_cast<const uintx4a2*>(p);
}

// Loading and putting the chunk right are two steps, so that nothing waits for a load before the chunk is stored to LDS; and no
// load is under a condition that differs between lanes.  A chunk of whole ones:
template <class T>
__device__ __forceinline__ void fetch_whole(Chunk<T>& q, const char* at) {
    q.v[0] = *reinterpret_cast<const uintx4*>(at);
    if constexpr (sizeof(q) == 32) q.v[1] = *reinterpret_cast<const uintx4*>(at + 16);
}
// and any: `row`: its row in memory, of which `width` elements exist; c: the first of the chunk's eight columns.  What lies past the
// row's end becomes zero in settle.
template <class T>
__device__ __forceinline__ void fetch_any(Chunk<T>& q, const T* row, int c, int width) {
    if (width >= 8) {                                                   // (uniform) the last chunk is moved back to end with the row
        const T* at = row + (c + 8 <= width ? c : width - 8);
        q.v[0] = load16<sizeof(T)>(at);
        if constexpr (sizeof(T) == 4) q.v[1] = load16<sizeof(T)>(at + 4);
    } else {
        T v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row[c + e < width ? c + e : width - 1];
        __builtin_memcpy(&q, v, 8 * sizeof(T));
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

// Two fp32 numbers -> their three bf16 parts, each pair packed into one dword (low half = first number).  The first two are the nearest
// bf16 numbers, so that a part is at most 2^-8 of what it is the rest of; the last is what is left, 8 bits at most.  (Truncated, parts are up to 2^-7 of it
// and of one sign: the products that are left out would add up to 2^-21, always towards zero.)  Numbers that would round to infinity
// get the largest bf16 number.
__device__ __forceinline__ void three_parts(float x0, float x1, unsigned& h, unsigned& m, unsigned& l) {
    typedef float floatx2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    auto nearest = [](float a, float b) { return __builtin_bit_cast(unsigned, __builtin_convertvector((floatx2{a, b}), bf16x2)); };
    const float most = __uint_as_float(0x7F7F0000u);
    h = nearest(__builtin_amdgcn_fmed3f(x0, -most, most), __builtin_amdgcn_fmed3f(x1, -most, most));
    const float r0 = x0 - __uint_as_float(h << 16), r1 = x1 - __uint_as_float(h & 0xFFFF0000u);              // exact
    m = nearest(r0, r1);
    const float s0 = r0 - __uint_as_float(m << 16), s1 = r1 - __uint_as_float(m & 0xFFFF0000u);              // exact
    l = __builtin_amdgcn_perm(__float_as_uint(s1), __float_as_uint(s0), 0x07060302u);
}

__device__ __forceinline__ int along_swizzle(int chunk) { return (chunk & 3) << 2 | (chunk >> 2) << 1; }
template <int ROWS>
__device__ __forceinline__ int across_swizzle(int k) { return ROWS >= 128 ? (k & 3) << 2 : ROWS == 64 ? (k & 2) << 1 : 0; }

// One operand's tile: ROWS rows (i) by BK of the contraction, carried by THREADS threads (of a set of wavefronts).
template <class T, Lie LIE, Mode MODE, int ROWS, int BK, int THREADS, int PF, int WK>
struct Operand {
    using E = typename View<T>::Element;
    static constexpr int kParts_ = kParts<T>;
    static constexpr int kPlane = ROWS * BK;                            // 16-bit elements of a part
    static constexpr int kSize = kParts_ * kPlane;                      // of a buffer
    static constexpr int kPerRow = (LIE == kAlong ? BK : ROWS) / 8;       // chunks per row in memory
    static constexpr int kChunks = ROWS * BK / 8;
    static constexpr int kEach = (kChunks + THREADS - 1) / THREADS;
    static constexpr bool kIdle = kChunks % THREADS != 0;                 // some threads carry none at the last round
    static constexpr int kChunkBytes = sizeof(Chunk<T>);
    Chunk<T> q[PF][kEach];
    unsigned place[kEach];                                               // kWhole: bytes from the tile's (kAlong) or the step's (kAcross) first
    const E* at[kEach];                                                  // kAny: start of the row (kAlong), or of the row of the step (kAcross)

    __device__ __forceinline__ static int thread() { return threadIdx.x % THREADS; }
    __device__ __forceinline__ static int row_of(int u) { return (thread() + u * THREADS) / kPerRow; }
    __device__ __forceinline__ static int chunk_of(int u) { return (thread() + u * THREADS) % kPerRow; }
    __device__ __forceinline__ static bool carries(int u) { return !kIdle || thread() + u * THREADS < kChunks; }

    __device__ __forceinline__ void begin(const View<T>& x, int64_t from) {     // from: where the set's first step begins
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            int r = row_of(u);
            if (LIE == kAlong && r >= x.rows) r = x.rows - 1;               // rows past the end: any (their results are not stored)
            if constexpr (MODE == kWhole) place[u] = (unsigned)r * (unsigned)(x.ld * sizeof(E)) + chunk_of(u) * kChunkBytes;
            else at[u] = x.p + ((LIE == kAcross ? from : 0) + r) * x.ld;
        }
    }
    // the step that begins at k0, into slot s
    __device__ __forceinline__ void load(const View<T>& x, int64_t k0, int s) {
        const int64_t rest = x.depth - k0;
        const int left = (int)(rest < BK ? rest : BK);
        const int64_t ahead = left > 0 ? k0 : 0;                           // (a step past the end loads the first one's data)
        if constexpr (MODE == kWhole) {
            const char* base = reinterpret_cast<const char*>(x.p) + (LIE == kAlong ? ahead / 8 * kChunkBytes : ahead * x.ld * (int64_t)sizeof(E));
            const int here = left > 0 ? left : (int)(x.depth < BK ? x.depth : BK);
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const int c = 8 * chunk_of(u);
                const bool in = LIE == kAlong ? c < here : row_of(u) < here && c < x.rows;
                fetch_whole<T>(q[s][u], base + (in ? place[u] : 0u));       // (one that does not exist: the first one)
            }
        } else {
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                if constexpr (LIE == kAlong) fetch_any<T>(q[s][u], at[u], (int)k0 + 8 * chunk_of(u), (int)x.depth);
                else {
                    fetch_any<T>(q[s][u], row_of(u) < left ? at[u] : x.p, 8 * chunk_of(u), x.rows);          // (row 0 of the view is there)
                    at[u] += WK * BK * x.ld;
                }
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

// What tiles of WM x WN wavefronts, TM x TN accumulators of 32 x 32 each, have in common.
// WK: as many sets of WM x WN wavefronts share the steps of the contraction; the first set gets the results.
template <int WM_, int WN_, int TM_, int TN_, int WK_ = 1>
struct Tile {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, WK = WK_;
    static constexpr int BM = 32 * TM * WM, BN = 32 * TN * WN, THREADS = 64 * WM * WN * WK;
    // results on their way out: 32 rows by up to 64 columns of a wavefront, at a time
    static constexpr int kSlabCols = TN >= 2 ? 64 : 32, kSlabLd = kSlabCols + 4;
    static constexpr int kSlabs = WM * WN * 32 * kSlabLd * 2;            // in 16-bit elements

    __device__ __forceinline__ static void clear(floatx16 (&acc)[TM][TN]) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
    }

    // The sets' sums, to the first set; the LDS is free before, and behind the slabs not after.
    static constexpr int kSums = kSlabs + (WK - 1) * BM * BN * 2;          // in 16-bit elements
    __device__ __forceinline__ static void join(floatx16 (&acc)[TM][TN], unsigned short* lds) {
        if constexpr (WK > 1) {
            const int set = (threadIdx.x >> 6) / (WM * WN);
            float4* sums = reinterpret_cast<float4*>(lds + kSlabs) + threadIdx.x % (64 * WM * WN);
            constexpr int EACH = 64 * WM * WN;                                // (of a set's lanes, a quad of results next to the other lanes')
            if (set > 0)
#pragma unroll
                for (int q = 0; q < TM * TN * 4; ++q) {
                    const floatx16& v = acc[q / 4 / TN][q / 4 % TN];
                    sums[((set - 1) * TM * TN * 4 + q) * EACH] = make_float4(v[q % 4 * 4], v[q % 4 * 4 + 1], v[q % 4 * 4 + 2], v[q % 4 * 4 + 3]);
                }
            __syncthreads();
            if (set == 0)
#pragma unroll
                for (int t = 0; t < WK - 1; ++t)
#pragma unroll
                    for (int q = 0; q < TM * TN * 4; ++q) {
                        const float4 u = sums[(t * TM * TN * 4 + q) * EACH];
                        floatx16& v = acc[q / 4 / TN][q / 4 % TN];
                        v[q % 4 * 4] += u.x; v[q % 4 * 4 + 1] += u.y; v[q % 4 * 4 + 2] += u.z; v[q % 4 * 4 + 3] += u.w;
                    }
        }
    }

    // f(row, column, four results) for every quad of the tile, 16 (TN >= 2) or 8 neighbouring lanes along a row.  Every wavefront passes
    // its results through LDS of its own.  MIRROR: what f returns goes on to m(column, row, four results of neighbouring rows).
    template <bool MIRROR, class F, class M>
    __device__ __forceinline__ static void drain(floatx16 (&acc)[TM][TN], unsigned short* S, F f, M m) {
        constexpr int J = kSlabCols / 32, Q = kSlabCols / 4;
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wm = wave / WN, wn = wave % WN;
        if (wave >= WM * WN) return;
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
                // (rolled up: this code runs once a workgroup, and is fetched for it)
#pragma unroll 2
                for (int u = 0; u < 32 * Q / 64; ++u) {
                    const int row = (lane + 64 * u) / Q, col = (lane + 64 * u) % Q * 4;
                    float4* at = reinterpret_cast<float4*>(C + row * kSlabLd + col);
                    if constexpr (MIRROR) *at = f(r0 + row, c0 + col, *at);
                    else f(r0 + row, c0 + col, *at);
                }
                if constexpr (MIRROR) {
                    settled();
#pragma unroll 1
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

// Tiles whose operands go through registers: fp32, bf16 or fp16, any rows.
template <class T, Lie XL, Lie YL, Mode MODE, int WM_, int WN_, int TM_, int TN_, int BK_, int PF_, int BUFFERS_, int WK_ = 1>
struct Product : Tile<WM_, WN_, TM_, TN_, WK_> {
    using Base = Tile<WM_, WN_, TM_, TN_, WK_>;
    using Base::WM; using Base::WN; using Base::TM; using Base::TN; using Base::WK; using Base::BM; using Base::BN; using Base::THREADS; using Base::kSlabs;
    static_assert(kParts<T> != 2, "Pairs go straight to LDS");
    static constexpr int BK = BK_, PF = PF_, BUFFERS = BUFFERS_;
    using X = Operand<T, XL, MODE, BM, BK, 64 * WM * WN, PF, WK>;
    using Y = Operand<T, YL, MODE, BN, BK, 64 * WM * WN, PF, WK>;
    static constexpr int P = kParts<T>;
    static constexpr int kBuffer = X::kSize + Y::kSize;
    static constexpr int kLds = WK * BUFFERS * kBuffer > Base::kSums ? WK * BUFFERS * kBuffer : Base::kSums;

    __device__ __forceinline__ static void step(floatx16 (&acc)[TM][TN], const unsigned short* S) {
        const int wave = (threadIdx.x >> 6) % (WM * WN), wm = wave / WN, wn = wave % WN;
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
                auto add = [&](int p, int q) {                             // (neighbouring instructions have different accumulators)
#pragma unroll
                    for (int i = 0; i < TM; ++i) acc[i][j] = multiply<T>(b[p], a[q][i], acc[i][j]);
                };
                // smallest terms first
                if constexpr (P == 3) { add(0, 2); add(2, 0); add(1, 1); add(0, 1); add(1, 0); }
                add(0, 0);
            }
        }
    }

    __device__ __forceinline__ static void run(floatx16 (&acc)[TM][TN], const View<T>& x, const View<T>& y, unsigned short* S) {
        Base::clear(acc);
        const int64_t depth = x.depth;
        if (depth <= 0) return;
        const int set = WK > 1 ? __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / (WM * WN)) : 0;
        const int64_t from = set * BK;
        S += set * BUFFERS * kBuffer;
        X X_;
        Y Y_;
        X_.begin(x, from);
        Y_.begin(y, from);
#pragma unroll
        for (int s = 0; s < PF; ++s) { X_.load(x, from + s * WK * BK, s); Y_.load(y, from + s * WK * BK, s); }
        // (steps past the end load what is there and store zeros: a load or store that some steps leave out would make every wait
        // for loads one for all of them, whatever is ahead)
        int buffer = 0;
        if constexpr (BUFFERS == 2) {
            X_.store(x, from, 0, S);
            Y_.store(y, from, 0, S + X::kSize);
            __syncthreads();
        }
        for (int64_t k0 = 0; k0 < depth; k0 += PF * WK * BK) {
#pragma unroll
            for (int u = 0; u < PF; ++u) {
                const int64_t k = k0 + u * WK * BK;
                if (u > 0 && k >= depth) break;                          // (uniform, for all sets)
                if constexpr (BUFFERS == 1) {
                    X_.store(x, from + k, u, S);
                    Y_.store(y, from + k, u, S + X::kSize);
                    __syncthreads();
                }
                X_.load(x, from + k + PF * WK * BK, u);
                Y_.load(y, from + k + PF * WK * BK, u);
                step(acc, S + buffer * kBuffer);
                if constexpr (BUFFERS == 2) {
                    buffer ^= 1;
                    X_.store(x, from + k + WK * BK, (u + 1) % PF, S + buffer * kBuffer);
                    Y_.store(y, from + k + WK * BK, (u + 1) % PF, S + buffer * kBuffer + X::kSize);
                }
                __syncthreads();
            }
        }
        Base::join(acc, S - set * BUFFERS * kBuffer);
    }
};

// Tiles whose operands go from memory straight to LDS, STAGES - 1 steps ahead: bf16, fp16 and Pairs whose chunks are whole.  An LDS tile
// is made of pieces of 16 bytes, of a chunk of 16-bit numbers or of a chunk's high or low parts, as they come in memory: rows of 128 or 64 bytes
// (kAlong), or BK rows of the tile's width (kAcross); an instruction of a wavefront fills 64 pieces in a row, and which piece of memory a
// lane brings is chosen so that the 32 lanes that read at a time find theirs in different banks.  One barrier per step; the first
// operands of a step are read under the last matrix instructions of the one before.  32 x 2048 x 1024 x 1024 Pairs: 868 -> 997 TFLOP/s
// of matrix instructions over the way through registers, bf16 853 -> 1126 (a library product of 4096^3: 1130).
static __device__ const uintx4 zero_piece = {0u, 0u, 0u, 0u};

template <class T, Lie LIE, int ROWS, int BK, int WAVES>
struct DirectOperand {
    using E = typename View<T>::Element;
    static constexpr int kParts_ = kParts<T>, kBytes = 2 * kParts_;           // of an element
    static constexpr int kPerRow = (LIE == kAlong ? BK : ROWS) * kBytes / 16;   // pieces of a row in memory
    static constexpr int kSize = ROWS * BK * kBytes;                          // bytes of a stage
    static constexpr int kEach = kSize / 1024 / WAVES;                        // instructions of a wavefront per stage
    static_assert(kEach * 1024 * WAVES == kSize && (LIE == kAcross || kPerRow == 8 || kPerRow == 4), "");
    unsigned from[kEach];
    __device__ __forceinline__ static int swizzle(int row) {
        if constexpr (LIE == kAlong) return kPerRow == 8 ? row >> 1 & 7 : row >> 2 & 3;
        else if constexpr (kParts_ == 2) return kPerRow >= 16 ? (row & 1) | (row & 2) << 2 : 0;
        else return kPerRow >= 16 ? (row & 3) << 2 : kPerRow == 8 ? (row & 2) << 1 : 0;
    }
    __device__ __forceinline__ static int wave() { return (threadIdx.x >> 6) % WAVES; }
    __device__ __forceinline__ static int piece_index(int u) { return ((u * WAVES + wave()) << 6) + (int)(threadIdx.x & 63); }
    __device__ __forceinline__ static int row_of(int u) { return piece_index(u) / kPerRow; }
    __device__ __forceinline__ static int piece_of(int u) { return piece_index(u) % kPerRow ^ swizzle(row_of(u)); }
    __device__ __forceinline__ static int element_of(int u) { return piece_of(u) / kParts_ * 8; }      // the first of the piece's chunk

    __device__ __forceinline__ void begin(const View<T>& x) {
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            int r = row_of(u), piece = piece_of(u);
            if (LIE == kAlong && r >= x.rows) r = x.rows - 1;                  // rows past the end: any (their results are not stored)
            if (LIE == kAcross && element_of(u) >= x.rows) piece = 0;          // (likewise)
            from[u] = (unsigned)r * (unsigned)(x.ld * sizeof(E)) + piece * 16;
        }
    }
    __device__ __forceinline__ void load(const View<T>& x, int64_t k0, char* S) const {
        typedef const __attribute__((address_space(1))) void* Global;
        typedef __attribute__((address_space(3))) void* Local;
        const char* base = reinterpret_cast<const char*>(x.p) + (LIE == kAlong ? k0 * kBytes : k0 * x.ld * (int64_t)sizeof(E));
        S += __builtin_amdgcn_readfirstlane(wave()) * 1024;
        const int64_t left = x.depth - k0;
        if (kEach > 2 && left >= BK) {                                         // (uniform; small tiles: less code rather than fewer instructions)
#pragma unroll
            for (int u = 0; u < kEach; ++u) __builtin_amdgcn_global_load_lds((Global)(base + from[u]), (Local)(S + u * WAVES * 1024), 16, 0, 0);
        } else {                                                              // what lies past the end of the contraction is zero
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const bool in = (LIE == kAlong ? element_of(u) : row_of(u)) < left;
                const char* at = in ? base + from[u] : reinterpret_cast<const char*>(&zero_piece);
                __builtin_amdgcn_global_load_lds((Global)at, (Local)(S + u * WAVES * 1024), 16, 0, 0);
            }
        }
    }
    // rows 32 b .. 32 b + 31, k 16 s .. 16 s + 15, part p, as the matrix cores take them
    __device__ __forceinline__ static uintx4 operand(const char* S, int b, int s, int p) {
        const int lane = threadIdx.x & 63;
        if constexpr (LIE == kAlong) {
            const int row = 32 * b + (lane & 31), piece = (2 * s + (lane >> 5)) * kParts_ + p;
            return *reinterpret_cast<const uintx4*>(S + (row * kPerRow + (piece ^ swizzle(row))) * 16);
        } else {
            const int k = 16 * s + 8 * (lane >> 5) + ((lane & 15) >> 2), col = 32 * b + (lane & 16) + 4 * (lane & 3);
            const char* from = S + (k * kPerRow + (((col >> 3) * kParts_ + p) ^ swizzle(k))) * 16 + (col & 4) * 2;
            typedef __attribute__((address_space(3))) shortx4* Lds;
            const shortx4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)from);
            const shortx4 c = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from + 4 * kPerRow * 16));        // (k + 4: the same permutation)
            uintx4 v;
            __builtin_memcpy(&v, &a, 8);
            __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &c, 8);
            return v;
        }
    }
};

template <class T, Lie XL, Lie YL, int WM_, int WN_, int TM_, int TN_, int STAGES_, int WK_ = 1, int BK_ = 64 / kParts<T>>
struct Direct : Tile<WM_, WN_, TM_, TN_, WK_> {
    using Base = Tile<WM_, WN_, TM_, TN_, WK_>;
    using Base::WM; using Base::WN; using Base::TM; using Base::TN; using Base::WK; using Base::BM; using Base::BN; using Base::THREADS; using Base::kSlabs;
    static constexpr int P = kParts<T>, BK = BK_, SUBS = BK / 16, STAGES = STAGES_;
    using X = DirectOperand<T, XL, BM, BK, WM * WN>;
    using Y = DirectOperand<T, YL, BN, BK, WM * WN>;
    static constexpr int kStage = X::kSize + Y::kSize;
    static constexpr int kSet = STAGES * kStage;                              // bytes of a set of wavefronts
    static constexpr int kLds = WK * kSet / 2 > Base::kSums ? WK * kSet / 2 : Base::kSums;     // in 16-bit elements
    static constexpr int kAhead = (STAGES - 2) * (X::kEach + Y::kEach);      // loads that may be on their way when the next step begins

    struct Operands { uintx4 a[P][TM], b[P][TN]; };
    __device__ __forceinline__ static void read(Operands& f, const char* S, int s) {
        const int wave = (threadIdx.x >> 6) % (WM * WN), wm = wave / WN, wn = wave % WN;
#pragma unroll
        for (int p = P - 1; p >= 0; --p) {                                   // in the order of their use
#pragma unroll
            for (int j = 0; j < TN; ++j) f.b[P - 1 - p][j] = Y::operand(S + X::kSize, wn * TN + j, s, P - 1 - p);
#pragma unroll
            for (int i = 0; i < TM; ++i) f.a[p][i] = X::operand(S, wm * TM + i, s, p);
        }
    }
    __device__ __forceinline__ static void add(floatx16 (&acc)[TM][TN], const Operands& f) {
        auto product = [&](int p, int q) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int i = 0; i < TM; ++i) acc[i][j] = multiply<T>(f.b[p][j], f.a[q][i], acc[i][j]);
        };
        if constexpr (P == 2) { product(0, 1); product(1, 0); }               // smallest terms first
        product(0, 0);
    }
    // This wavefront's loads but for AHEAD, and its LDS reads, are done; then everybody's.  (The fences keep the compiler from moving
    // accesses across; of a workgroup's scope, they would wait for all loads.)
    template <int AHEAD>
    __device__ __forceinline__ static void meet() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_s_waitcnt((AHEAD & 15) | 7 << 4 | (AHEAD >> 4) << 14);     // vmcnt(AHEAD) lgkmcnt(0)
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    }

    __device__ __forceinline__ static void run(floatx16 (&acc)[TM][TN], const View<T>& x, const View<T>& y, unsigned short* lds) {
        Base::clear(acc);
        const int64_t depth = x.depth;
        if (depth <= 0) return;
        const int set = WK > 1 ? __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) / (WM * WN)) : 0;
        char* S = reinterpret_cast<char*>(lds) + set * kSet;
        X X_;
        Y Y_;
        X_.begin(x);
        Y_.begin(y);
        const int64_t from = set * BK;
#pragma unroll 1
        for (int t = 0; t < STAGES - 1; ++t) {
            X_.load(x, from + t * WK * BK, S + t * kStage);
            Y_.load(y, from + t * WK * BK, S + t * kStage + X::kSize);
        }
        meet<kAhead>();
        Operands f[2];
        read(f[0], S, 0);
        int now = 0, next = STAGES - 1;                                       // stages of this step and of the one loaded
        for (int64_t k0 = 0; k0 < depth; k0 += WK * BK) {
            // into the stage of the step before, which nobody reads any more
            X_.load(x, from + k0 + (STAGES - 1) * WK * BK, S + next * kStage);
            Y_.load(y, from + k0 + (STAGES - 1) * WK * BK, S + next * kStage + X::kSize);
#pragma unroll
            for (int s = 0; s + 1 < SUBS; ++s) {
                read(f[(s + 1) & 1], S + now * kStage, s + 1);
                add(acc, f[s & 1]);
            }
            meet<kAhead>();
            next = now;
            now = now + 1 < STAGES ? now + 1 : 0;
            read(f[0], S + now * kStage, 0);                                  // (after the last step: zeros)
            add(acc, f[(SUBS - 1) & 1]);
        }
        meet<0>();                                                            // the LDS is free
        Base::join(acc, lds);
    }
};

// One quad of a row of `width` results at column c (c < width), the row at `to`; whole: width and the row's place are multiples of four
// elements.  STREAM: past the caches' order of use, as all weight gradients over groups that are not summed in parts are stored.  With plain
// stores for it: results of up to 17 MB take the same 15 us; 67 MB 24.5 us for 26.0 (4096 x 1024 x 1024 bf16 to fp32, 16 groups), 134 MB 54.5 for
// 64.3 (16384 rows, 32 groups), 537 MB 164 for 173 (16384 x 2048 x 1024, 64 even groups).  A call behind it that reads the result finds less of it
// in the caches: with an optimiser step the two take 403 us for 398, 783 for 777 (the first two above), 1347 for 1367 (268 MB); what loses most is
// a result that is nearly the whole work and is read in one pass (200 rows in 64 groups of 1024 x 1024, 268 MB: 155 for 133).
template <bool STREAM = false, class O>
__device__ __forceinline__ void put(O* to, int c, int width, float4 v, bool whole) {
    typedef O ox4 __attribute__((ext_vector_type(4)));
    const ox4 q = {(O)v.x, (O)v.y, (O)v.z, (O)v.w};
    if (whole && STREAM) __builtin_nontemporal_store(q, reinterpret_cast<ox4*>(to + c));
    else if (whole) *reinterpret_cast<ox4*>(to + c) = q;
    else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < width) to[c + e] = q[e];
    }
}

}  // namespace tile
}  // namespace cadmm
