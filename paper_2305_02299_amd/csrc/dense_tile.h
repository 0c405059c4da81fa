// Dense products on the matrix cores whose operands lie either way in memory (device side): what the forward and backward passes of the
// structured-only layer and of the gated block share.
//
// A product is C[m][n] = sum_k A(m, k) B(n, k) over a BM x BN tile per workgroup, K walked in stages of 128 bytes of K a line.  An operand's
// lines either run along K (a row of x against a row of W: forward) or across it (row k of W holds the k-th value of every column: the gradient of x
// takes W this way, the gradient of W both operands).  The matrix units want eight consecutive k of one row in a lane's register pair.  Lines along K give
// them with one 16-byte read of the LDS; for lines across K in bf16 the LDS hands four lines' values of a column to a lane (ds_read_b64_tr_b16: of 16 lanes,
// lane i reads 8 bytes, columns 4 (i % 4) .. + 3 of line i / 4, and gets the values of column i in lines 0 .. 3), in fp32 a lane reads its four k as words.
//
// LDS layouts of a stage of R tile rows (R * 128 bytes): along K, row r at r * 128, its 16-byte piece q in slot q ^ ((r >> 1) & 7); across K, line k at
// k * R * sizeof(T), its piece q in slot q ^ across_swizzle(k): the lines that one read touches lie in different banks.
// MFMA operands: bf16 32x32x16, lane l holds row l % 32, k = 8 (l / 32) .. + 7 of a 32-byte step; fp32 32x32x2, lane l row l % 32, k = 4 (l / 32) + j in
// the j-th of four.  Result: register e of lane l is row 8 (e / 4) + 4 (l / 32) + e % 4, column l % 32.
#pragma once
#include "mma_tile.h"
#include <initializer_list>
#include <type_traits>

namespace srigl {

typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

template <typename T> struct DenseFrag;
template <> struct DenseFrag<uint16_t> { using type = bf16x8_t; };
template <> struct DenseFrag<float> { using type = f32x4_t; };
__device__ __forceinline__ void dense_mma(f32x16_t& acc, const bf16x8_t& a, const bf16x8_t& b) { acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0); }
__device__ __forceinline__ void dense_mma(f32x16_t& acc, const f32x4_t& a, const f32x4_t& b) {
#pragma unroll
    for (int j = 0; j < 4; ++j) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[j], b[j], acc, 0, 0, 0);
}

constexpr int kLineBytes = 128;                                              // of K a stage
template <typename T> constexpr int kStageK = kLineBytes / (int)sizeof(T);   // its elements
template <typename T> constexpr int kPiece = 16 / (int)sizeof(T);            // elements of a 16-byte piece

// From one matrix to another, in bytes
inline long long bytes_between(const void* a, const void* b) { return (long long)(reinterpret_cast<intptr_t>(b) - reinterpret_cast<intptr_t>(a)); }
// Whether 16-byte loads can take an operand whose rows are `pitch` apart, and a lane's 32 bits the offsets of `lines` of them
template <typename T> inline bool direct_rows(const T* base, long long pitch, int lines) {
    return (reinterpret_cast<uintptr_t>(base) & 15) == 0 && pitch * (long long)sizeof(T) % 16 == 0 && lines * pitch * (long long)sizeof(T) < (1ll << 31);
}

// Loads and stores of V consecutive elements from any element's address
template <typename T, int V> struct AnyPlace { typedef T type __attribute__((ext_vector_type(V), aligned(sizeof(T)))); };

// ---- operands ----
// line(l, first, valid): where elements first .. of line l begin, *valid how many of them there are (<= 0: none).
// For loads that go straight into the LDS, of operands whose lines begin at and are multiples of 16 bytes: stage(h, l) is the scalar address that lane_offset(l, first) bytes are
// added to (l: any line of the 1 KB that the wavefront's load fills, whose lines are of one matrix), with lines and columns past the last one at the last one.
// inside(h): every piece of stage h can be read as 16 bytes (lines along K: all of its K is there; across K: a piece may reach into the line behind, whose values
// go to columns that nobody stores, so all but the matrix's last line).
// Stages by number: whole() of them have all of their K, the i-th of these being stage index(i); of tails() others, stage tail(t), a part lies behind the end of K.
// Along K: line = tile row, elements = k.
template <typename T> struct RowsOf {
    static constexpr bool kAlong = true;
    const T* base;      // of the tile's first row
    long long pitch;
    int last, K;        // last row that there is, counted from the tile's first
    __device__ void move(int first) { base += (size_t)first * pitch; last -= first; }
    __device__ const T* line(int l, int first, int* valid) const { *valid = K - first; return base + (size_t)min(l, last) * pitch + first; }
    __device__ const unsigned char* stage(int h, int) const { return reinterpret_cast<const unsigned char*>(base) + (size_t)h * kLineBytes; }
    __device__ uint32_t lane_offset(int l, int first) const { return ((uint32_t)min(l, last) * (uint32_t)pitch + first) * (uint32_t)sizeof(T); }
    __device__ bool inside(int h) const { return (h + 1) * kStageK<T> <= K; }
    bool direct(int lines) const { return direct_rows(base, pitch, lines) && K % kPiece<T> == 0; }
    __device__ int whole() const { return K / kStageK<T>; }
    __device__ int index(int i) const { return i; }
    __device__ int tails() const { return K % kStageK<T> ? 1 : 0; }
    __device__ int tail(int) const { return K / kStageK<T>; }
};
// The weight rows of two matrices that a gated block multiplies with, next to each other in each wavefront's part of the tile: HALF rows of the first,
// the same HALF rows of the second.
template <typename T, int HALF> struct PairedRows {
    static constexpr bool kAlong = true;
    const T* base;
    long long to_second;   // bytes (a choice between two pointers of a struct went through scratch memory)
    long long pitch;
    int last, K;
    __device__ void move(int first) { base += (size_t)first * pitch; last -= first; }
    __device__ const unsigned char* of(bool second) const { return reinterpret_cast<const unsigned char*>(base) + (second ? to_second : 0); }
    __device__ const T* line(int l, int first, int* valid) const {
        const int part = l / HALF, r = (part >> 1) * HALF + l % HALF;
        *valid = K - first;
        return reinterpret_cast<const T*>(of(part & 1)) + (size_t)min(r, last) * pitch + first;
    }
    __device__ const unsigned char* stage(int h, int l) const { return of(l / HALF & 1) + (size_t)h * kLineBytes; }
    __device__ uint32_t lane_offset(int l, int first) const {
        return ((uint32_t)min((l / HALF >> 1) * HALF + l % HALF, last) * (uint32_t)pitch + first) * (uint32_t)sizeof(T);
    }
    __device__ bool inside(int h) const { return (h + 1) * kStageK<T> <= K; }
    bool direct(int lines) const { return direct_rows(base, pitch, lines) && to_second % 16 == 0 && K % kPiece<T> == 0; }
    __device__ int whole() const { return K / kStageK<T>; }
    __device__ int index(int i) const { return i; }
    __device__ int tails() const { return K % kStageK<T> ? 1 : 0; }
    __device__ int tail(int) const { return K / kStageK<T>; }
};
// Across K: line = k, elements = tile columns.
template <typename T> struct ColsOf {
    static constexpr bool kAlong = false;
    const T* base;      // of the tile's first column, line 0
    long long pitch;
    int cols, K;        // columns from there on
    __device__ void move(int first) { base += first; cols -= first; }
    __device__ const T* line(int l, int first, int* valid) const { *valid = l < K ? cols - first : 0; return base + (size_t)l * pitch + first; }
    __device__ const unsigned char* stage(int h, int) const { return reinterpret_cast<const unsigned char*>(base + (size_t)h * kStageK<T> * pitch); }
    __device__ uint32_t lane_offset(int l, int first) const { return ((uint32_t)l * (uint32_t)pitch + min(first, cols - kPiece<T>)) * (uint32_t)sizeof(T); }
    __device__ bool inside(int h) const { return (h + 1) * kStageK<T> < K && pitch >= kPiece<T>; }
    bool direct(int) const { return direct_rows(base, pitch, kStageK<T>) && cols % kPiece<T> == 0; }
    __device__ int whole() const { return K / kStageK<T>; }
    __device__ int index(int i) const { return i; }
    __device__ int tails() const { return K % kStageK<T> ? 1 : 0; }
    __device__ int tail(int) const { return K / kStageK<T>; }
};
// Lines 0 .. n - 1 of one matrix, then, from line `padded` on, those of a second.
template <typename T> struct PairedCols {
    static constexpr bool kAlong = false;
    const T* base;
    long long to_second;   // bytes
    long long pitch;
    int cols, n, padded;
    __device__ void move(int first) { base += first; cols -= first; }
    __device__ const T* of(bool second) const { return reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(base) + (second ? to_second : 0)); }
    __device__ const T* line(int l, int first, int* valid) const {
        const bool behind = l >= padded;
        const int r = behind ? l - padded : l;
        *valid = r < n ? cols - first : 0;
        return of(behind) + (size_t)r * pitch + first;
    }
    __device__ const unsigned char* stage(int h, int) const {   // (`padded` is a whole number of stages)
        const int in_first = padded / kStageK<T>;
        return reinterpret_cast<const unsigned char*>(of(h >= in_first) + (size_t)(h >= in_first ? h - in_first : h) * kStageK<T> * pitch);
    }
    __device__ uint32_t lane_offset(int l, int first) const { return ((uint32_t)l * (uint32_t)pitch + min(first, cols - kPiece<T>)) * (uint32_t)sizeof(T); }
    // (in_first * kStageK may reach a whole stage behind n: that one is left out)
    __device__ int whole() const { return 2 * (n / kStageK<T>); }
    __device__ int index(int i) const { const int w = n / kStageK<T>; return i < w ? i : i - w + padded / kStageK<T>; }
    __device__ int tails() const { return n % kStageK<T> ? 2 : 0; }
    __device__ int tail(int t) const { return n / kStageK<T> + t * (padded / kStageK<T>); }
    __device__ bool inside(int h) const {
        const int behind = padded / kStageK<T>;
        return ((h < behind ? h : h - behind) + 1) * kStageK<T> < n && pitch >= kPiece<T>;
    }
    bool direct(int) const { return direct_rows(base, pitch, kStageK<T>) && to_second % 16 == 0 && cols % kPiece<T> == 0; }
};

// 16 bytes from there, zeros behind the valid elements
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* p, int valid) {
    if (valid >= kPiece<T>) {
        typename AnyPlace<T, kPiece<T>>::type v = *reinterpret_cast<const typename AnyPlace<T, kPiece<T>>::type*>(p);
        return __builtin_bit_cast(uint4, v);
    }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < kPiece<T>; ++e)
        if (e < valid) {
            if constexpr (sizeof(T) == 4) w[e] = __float_as_uint(p[e]);
            else w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
        }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Slot of piece q of line k, lines across K of R columns.  bf16: a read takes four lines (k % 4 = 0 .. 3) and 64 bytes of each: the 64-byte quarters of
// 256 bytes are exchanged by the line; of 128-byte lines two share 256 bytes.  fp32: lines k and k + 8, 128 bytes of each.
template <typename T, int R>
__device__ __forceinline__ int across_swizzle(int k) {
    if constexpr (sizeof(T) == 4) return ((k >> 3) & 1) << 3;
    else return R >= 128 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
}

// (restrict: without it the compiler holds the read back until every load on its way into the LDS has landed, the stages ahead included; the waits for this stage are the loop's own)
__device__ __forceinline__ s16x4_t read_across(const unsigned char* __restrict__ at) {
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)at);
}

// Reads a lane's fragments of the TB 32-row blocks from block `first` on, in a stage of R rows.
template <typename T, bool ALONG, int R, int TB>
struct FragReader {
    using F = typename DenseFrag<T>::type;
    static constexpr int PITCH = R * (int)sizeof(T), KSTEPS = kLineBytes / 32;
    uint32_t at[ALONG ? KSTEPS : TB];   // a lane's byte offset by step (blocks are 32 * 128 bytes apart), or by block (steps are whole lines apart)
    __device__ __forceinline__ void init(int first, int lane) {
        const int half = lane >> 5, r = lane & 31;
        if constexpr (ALONG) {
#pragma unroll
            for (int kk = 0; kk < KSTEPS; ++kk) at[kk] = (first * 32 + r) * kLineBytes + (((2 * kk + half) ^ ((r >> 1) & 7)) << 4);
        } else {
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                if constexpr (sizeof(T) == 4) {
                    const int c = (first + b) * 32 + r;
                    at[b] = 4 * half * PITCH + (c >> 2 << 4 | (c & 3) << 2);   // (steps of 8 lines by turns: the swizzle flips bit 7)
                } else {
                    const int i = lane & 15, c = (first + b) * 32 + (lane & 16) + 4 * (i & 3);
                    at[b] = (8 * half + (i >> 2)) * PITCH + ((((c >> 3) ^ across_swizzle<T, R>(i >> 2)) << 4) | ((c & 4) << 1));
                }
            }
        }
    }
    __device__ __forceinline__ F read(const unsigned char* stage, int b, int kk) const {
        if constexpr (ALONG) {
            return *reinterpret_cast<const F*>(stage + at[kk] + b * 32 * kLineBytes);
        } else if constexpr (sizeof(T) == 4) {
            F f;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = *reinterpret_cast<const float*>(stage + (at[b] ^ (kk & 1 ? 128u : 0u)) + (8 * kk + j) * PITCH);
            return f;
        } else {
            union { s16x4_t part[2]; F f; } u;
#pragma unroll
            for (int s = 0; s < 2; ++s)
                u.part[s] = read_across(stage + at[b] + (16 * kk + 4 * s) * PITCH);
            return u.f;
        }
    }
};

// ---- fp32 on the bf16 units ----
// An fp32 value is exactly the sum of three bf16 values, each what the ones before leave, the first two rounded to nearest: the second is at most 2^-8 of the value's power of two, the third 2^-17, in seven
// bits.  Of the nine products of two values the six that reach 2^-17 of the first go through the bf16 units into the same fp32 sums; what is left out is at most 2^-24 of the product, half a step of fp32,
// and of either sign.  (Cut off in place of rounded, the parts are up to 2^-7 and 2^-15, all of the value's sign: up to 2^-21 of a product was left out, always towards zero.  Rounding costs what a
// conversion takes more than a byte permutation, in a longer chain: 768 -> 3072 at 512 rows 27.6 us, now 29.8, its gradients 51.0 and 52.9, 4096 -> 4096 at 2048 rows 336 and 337; the second part cut off, 2^-23,
// 29.1, 52.4 and 335.)  A product by itself came out within 2.2 half steps, the units' own rounding among them.  Six instructions of 32 clocks do what the fp32 ones do in 512 (2.7 times as fast), and sixteen
// products meet in one rounding where the fp32 instructions round every two; the lanes split the values on their way from the LDS, 5.5 instructions a value, between the multiplications.  (The units take bf16
// denormals as they are, down to 2^-133: a value below 2^-110 loses its last bits, as far as its products matter beside others'.)  Infinities, NaN and values that round beyond bf16's range come out as NaN, and so
// does a sum that leaves the range on its way: a tile with a sum that is not finite is computed again by the fp32 instructions.
template <bool ALONG, int R, int TB>
struct SplitReader {
    static constexpr int PITCH = R * 4;
    uint32_t at[ALONG ? 4 : TB];
    __device__ __forceinline__ void init(int first, int lane) {
        const int half = lane >> 5, r = lane & 31;
        if constexpr (ALONG) {
#pragma unroll
            for (int q = 0; q < 4; ++q) at[q] = (first * 32 + r) * kLineBytes + (((4 * (q >> 1) + 2 * half + (q & 1)) ^ ((r >> 1) & 7)) << 4);
        } else {
#pragma unroll
            for (int b = 0; b < TB; ++b) {
                const int c = (first + b) * 32 + r;
                at[b] = 8 * half * PITCH + ((((c >> 2) ^ across_swizzle<float, R>(8 * half)) << 4) | ((c & 3) << 2));
            }
        }
    }
    __device__ __forceinline__ void read(const unsigned char* stage, int b, int kk, f32x4_t (&v)[2]) const {
#pragma unroll
        for (int p = 0; p < 2; ++p)
            if constexpr (ALONG) v[p] = *reinterpret_cast<const f32x4_t*>(stage + at[2 * kk + p] + b * 32 * kLineBytes);
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) v[p][j] = *reinterpret_cast<const float*>(stage + at[b] + (16 * kk + 4 * p + j) * PITCH);
    }
};
struct SplitFrag { uint32_t part[3][4]; };
// values 2 i and 2 i + 1 of a fragment
__device__ __forceinline__ void split_pair(SplitFrag& f, const f32x4_t (&v)[2], int i) {
    float x = v[i >> 1][2 * (i & 1)], y = v[i >> 1][2 * (i & 1) + 1];
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        const uint32_t both = __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{x, y}, bf16x2_t));   // to nearest
        f.part[p][i] = both;
        x -= __uint_as_float(both << 16);
        y -= __uint_as_float(both & 0xffff0000u);
    }
    f.part[2][i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);   // the upper halves of both: there is nothing in the lower ones
}
__device__ __forceinline__ bf16x8_t split_part(const SplitFrag& f, int p) { return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(f.part[p])); }

// The products in the order of their size, as parts of both values
constexpr int kSplitA[6] = {2, 0, 1, 1, 0, 0}, kSplitB[6] = {0, 2, 1, 0, 1, 0};

// ---- the product of a tile, staged through registers: any address, any size ----
template <typename T, int R, int NT, class Op>
struct RegStage {
    static constexpr int PASSES = R * kLineBytes / 16 / NT, PER_LINE = Op::kAlong ? 8 : R / kPiece<T>;
    static_assert(R * kLineBytes % (16 * NT) == 0, "pieces to a thread");
    uint4 held[PASSES];
    __device__ __forceinline__ void load(const Op& op, int h) {
        int valid;
        if (op.inside(h)) {   // (one branch for all pieces: with one a piece each waited for the one before, 3 us a stage)
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int u = p * NT + threadIdx.x, l = u / PER_LINE, first = u % PER_LINE * kPiece<T>;
                if constexpr (Op::kAlong) held[p] = load_piece(op.line(l, h * kStageK<T> + first, &valid), kPiece<T>);
                else held[p] = load_piece(op.line(h * kStageK<T> + l, min(first, op.cols - 1), &valid), kPiece<T>);
            }
        } else {
#pragma unroll
            for (int p = 0; p < PASSES; ++p) {
                const int u = p * NT + threadIdx.x, l = u / PER_LINE, first = u % PER_LINE * kPiece<T>;
                const T* const at = Op::kAlong ? op.line(l, h * kStageK<T> + first, &valid) : op.line(h * kStageK<T> + l, first, &valid);
                held[p] = load_piece(at, valid);
            }
        }
    }
    __device__ void store(unsigned char* stage) const {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            const int u = p * NT + threadIdx.x, l = u / PER_LINE, q = u % PER_LINE;
            const int slot = Op::kAlong ? q ^ ((l >> 1) & 7) : q ^ across_swizzle<T, R>(l);
            *reinterpret_cast<uint4*>(stage + l * PER_LINE * 16 + slot * 16) = held[p];
        }
    }
};

// Stages h0 .. h1 - 1, whatever part of them there is.  SPLIT: fp32 on the bf16 units.
template <typename T, bool SPLIT, int BM, int BN, int WGM, int WGN, class OA, class OB>
__device__ __forceinline__ void product_of_tile(unsigned char* smem, const OA& oa, const OB& ob, int h0, int h1, f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32]) {
    constexpr int NT = WGM * WGN * 64, TM = BM / WGM / 32, TN = BN / WGN / 32, KSTEPS = kLineBytes / 32;
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv / WGN, wn = wv % WGN;
    unsigned char *const sa = smem, *const sb = smem + BM * kLineBytes;
    if (h0 >= h1) return;
    typename std::conditional<SPLIT, SplitReader<OA::kAlong, BM, TM>, FragReader<T, OA::kAlong, BM, TM>>::type fa;
    typename std::conditional<SPLIT, SplitReader<OB::kAlong, BN, TN>, FragReader<T, OB::kAlong, BN, TN>>::type fb;
    fa.init(wm * TM, lane);
    fb.init(wn * TN, lane);
    RegStage<T, BM, NT, OA> ra;
    RegStage<T, BN, NT, OB> rb;
    ra.load(oa, h0);
    rb.load(ob, h0);
    for (int h = h0; h < h1; ++h) {
        __syncthreads();   // the stage before has been read
        ra.store(sa);
        rb.store(sb);
        __syncthreads();
        if (h + 1 < h1) {
            ra.load(oa, h + 1);
            rb.load(ob, h + 1);
        }
        if constexpr (SPLIT) {
#pragma unroll
            for (int kk = 0; kk < KSTEPS / 2; ++kk) {
                f32x4_t raw[TM + TN][2];
                SplitFrag f[TM + TN];
#pragma unroll
                for (int i = 0; i < TM; ++i) fa.read(sa, i, kk, raw[i]);
#pragma unroll
                for (int j = 0; j < TN; ++j) fb.read(sb, j, kk, raw[TM + j]);
#pragma unroll
                for (int i = 0; i < 4 * (TM + TN); ++i) split_pair(f[i >> 2], raw[i >> 2], i & 3);
#pragma unroll
                for (int m = 0; m < 6 * TM * TN; ++m) {
                    const int q = m % (TM * TN), p = m / (TM * TN);
                    acc[q / TN][q % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(split_part(f[q / TN], kSplitA[p]), split_part(f[TM + q % TN], kSplitB[p]), acc[q / TN][q % TN], 0, 0, 0);
                }
            }
            continue;
        } else {
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) {
            typename DenseFrag<T>::type a[TM], b[TN];
#pragma unroll
            for (int i = 0; i < TM; ++i) a[i] = fa.read(sa, i, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) b[j] = fb.read(sb, j, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) dense_mma(acc[i][j], a[i], b[j]);
        }
        }
    }
    __syncthreads();
}

// ---- the product of a tile, staged by loads straight into the LDS (operands that are direct()): a ring of NS stages.
// Schedule of a stage (KSTEPS MFMA steps): the fragments of the next step are requested between the multiplications of a step.  Before the last step the wavefront waits until its own
// loads of the next stage have landed and its reads of this one have returned, and meets the others at the barrier: the next stage is then complete and this one's slot free.  Behind it the first
// fragments of the next stage are requested and, between the multiplications of this step and the next one, the pieces of stage h + NS.  A stage index past the last one requests the last one again, into a
// slot nobody reads: the number of loads in flight at each wait is fixed. ----
template <typename T, int R, int FIRST, int NWAVES, class Op>
struct DirectStage {
    static constexpr int PASSES = R * kLineBytes / 1024 / NWAVES, PER_LINE = Op::kAlong ? 8 : R / kPiece<T>;
    static_assert(R * kLineBytes % (1024 * NWAVES) == 0, "1 KB to a wavefront's load");
    uint32_t at[PASSES];
    __device__ __forceinline__ static void place(int p, int wv, int lane, int* l, int* first) {
        const int u = (p * NWAVES + wv) * 64 + lane;
        *l = u / PER_LINE;
        *first = ((u % PER_LINE) ^ (Op::kAlong ? (*l >> 1) & 7 : across_swizzle<T, R>(*l))) * kPiece<T>;
    }
    __device__ __forceinline__ void init(const Op& op, int wv, int lane) {
#pragma unroll
        for (int p = 0; p < PASSES; ++p) {
            int l, first;
            place(p, wv, lane, &l, &first);
            at[p] = op.lane_offset(l, first);
        }
    }
    __device__ __forceinline__ void issue(const Op& op, int p, int h, unsigned char* stage, int wv) const {
        uint32_t off = at[p];
        asm("" : "+v"(off));   // (a lane offset from a scalar base: seen to be 32 bits only next to the load)
        const unsigned char* g = op.stage(h, (p * NWAVES + wv) * 64 / PER_LINE) + off;
        __builtin_amdgcn_global_load_lds((gptr_t)g, (lptr_t)(stage + FIRST + 1024 * (p * NWAVES + wv)), 16, 0, 0);
    }
};

// Whole stages h0 .. h1 - 1, by their number; meanwhile(): done while the first ones are on their way.  (The part of a stage behind the end of K in the loop, its pieces from zeros by lane: 20 % longer in 128 x 128 tiles.)
template <typename T, int BM, int BN, int WGM, int WGN, int NS, class OA, class OB, class Meanwhile>
__device__ __forceinline__ void direct_product_of_tile(unsigned char* smem, const OA& oa, const OB& ob, int h0, int h1, f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32], Meanwhile meanwhile) {
    constexpr int NWAVES = WGM * WGN, TM = BM / WGM / 32, TN = BN / WGN / 32, KSTEPS = kLineBytes / 32, STAGE = (BM + BN) * kLineBytes;
    using SA = DirectStage<T, BM, 0, NWAVES, OA>;
    using SB = DirectStage<T, BN, BM * kLineBytes, NWAVES, OB>;
    constexpr int PASSES = SA::PASSES + SB::PASSES;
    static_assert(NS >= 2 && (NS - 1) * PASSES <= 63, "vmcnt range");
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv / WGN, wn = wv % WGN, n_st = h1 - h0;
    if (n_st <= 0) return meanwhile();
    SA la;
    SB lb;
    la.init(oa, wv, lane);
    lb.init(ob, wv, lane);
    auto issue_piece = [&](int p, int h_unclamped, int slot) {
        const int h = ob.index(h0 + min(h_unclamped, n_st - 1));
        if (p < SA::PASSES) la.issue(oa, p, h, smem + slot, wv);
        else lb.issue(ob, p - SA::PASSES, h, smem + slot, wv);
    };
    constexpr int EARLY = TM * TN == 1 ? PASSES : PASSES / 2;   // pieces requested right behind the barrier, the others a step later
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int p = 0; p < (s < NS - 1 ? PASSES : EARLY); ++p) issue_piece(p, s, s * STAGE);
    meanwhile();

    FragReader<T, OA::kAlong, BM, TM> fa;
    FragReader<T, OB::kAlong, BN, TN> fb;
    fa.init(wm * TM, lane);
    fb.init(wn * TN, lane);
    typename DenseFrag<T>::type a[2][TM], b[2][TN];
    // fragment f of a step, in the order the products take them: a[0], the b's, the other a's
    auto read_frag = [&](int f, int slot, int kk, int set) {
        if (f >= 1 && f <= TN) b[set][f - 1] = fb.read(smem + slot + BM * kLineBytes, f - 1, kk);
        else a[set][f ? f - TN : 0] = fa.read(smem + slot, f ? f - TN : 0, kk);
    };
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * PASSES + EARLY));
    __syncthreads();
#pragma unroll
    for (int f = 0; f < TM + TN; ++f) read_frag(f, 0, 0, 0);
    // (opaque: a value that is a load here and in the loop is loaded where it is used, behind everything that was to hide it)
#pragma unroll
    for (int i = 0; i < TM; ++i) asm volatile("" : "+v"(a[0][i]));
#pragma unroll
    for (int j = 0; j < TN; ++j) asm volatile("" : "+v"(b[0][j]));
    int slot = 0, before = (NS - 1) * STAGE;   // of stage h and of the one before it
    for (int h = 0; h < n_st; ++h) {
        const int after = slot == (NS - 1) * STAGE ? 0 : slot + STAGE;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) {
            constexpr int N_MMA = TM * TN, N_FRAG = TM + TN, N_READ = N_MMA > N_FRAG ? N_FRAG : (N_MMA + 1) / 2;
            const bool last = kk + 1 == KSTEPS;
            if (last) {
                __builtin_amdgcn_s_waitcnt(kLgkm0);
                __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * PASSES));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int m = 0; m < N_MMA; ++m) {
#pragma unroll
                for (int f = m * N_FRAG / N_READ; f < (m + 1) * N_FRAG / N_READ && f < N_FRAG; ++f)
                    read_frag(f, last ? after : slot, last ? 0 : kk + 1, (kk + 1) & 1);
                if (N_MMA > 1) dense_mma(acc[m / TN][m % TN], a[kk & 1][m / TN], b[kk & 1][m % TN]);
                if (last) {
#pragma unroll
                    for (int p = m * EARLY / N_MMA; p < (m + 1) * EARLY / N_MMA; ++p) issue_piece(p, h + NS, slot);
                }
                if (kk == 0) {
#pragma unroll
                    for (int p = EARLY + m * (PASSES - EARLY) / N_MMA; p < EARLY + (m + 1) * (PASSES - EARLY) / N_MMA; ++p) issue_piece(p, h + NS - 1, before);
                }
                if (N_MMA == 1) dense_mma(acc[0][0], a[kk & 1][0], b[kk & 1][0]);   // (it waits for the one before: requests first)
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        before = slot;
        slot = after;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));   // the stages requested again may still be landing in the ring
    __syncthreads();
}

// Whole stages h0 .. h1 - 1 of an fp32 product by direct loads, as in direct_product_of_tile: two steps of 16 k a stage
template <int BM, int BN, int WGM, int WGN, int NS, class OA, class OB, class Meanwhile>
__device__ __forceinline__ void split_product_of_tile(unsigned char* smem, const OA& oa, const OB& ob, int h0, int h1, f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32], Meanwhile meanwhile) {
    constexpr int NWAVES = WGM * WGN, TM = BM / WGM / 32, TN = BN / WGN / 32, KSTEPS = 2, STAGE = (BM + BN) * kLineBytes;
    using SA = DirectStage<float, BM, 0, NWAVES, OA>;
    using SB = DirectStage<float, BN, BM * kLineBytes, NWAVES, OB>;
    constexpr int PASSES = SA::PASSES + SB::PASSES, EARLY = PASSES / 2;
    constexpr int N_FRAG = TM + TN, N_BLOCK = TM * TN, N_MMA = 6 * N_BLOCK, N_PAIR = 4 * N_FRAG, WAIT = N_MMA / 4 + 1;   // the cutting begins behind so many multiplications
    static_assert(NS >= 2 && (NS - 1) * PASSES <= 63, "vmcnt range");
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv / WGN, wn = wv % WGN, n_st = h1 - h0;
    if (n_st <= 0) return meanwhile();
    SA la;
    SB lb;
    la.init(oa, wv, lane);
    lb.init(ob, wv, lane);
    auto issue_piece = [&](int p, int h_unclamped, int slot) {
        const int h = ob.index(h0 + min(h_unclamped, n_st - 1));
        if (p < SA::PASSES) la.issue(oa, p, h, smem + slot, wv);
        else lb.issue(ob, p - SA::PASSES, h, smem + slot, wv);
    };
#pragma unroll
    for (int s = 0; s < NS; ++s)
#pragma unroll
        for (int p = 0; p < (s < NS - 1 ? PASSES : EARLY); ++p) issue_piece(p, s, s * STAGE);
    meanwhile();
    SplitReader<OA::kAlong, BM, TM> fa;
    SplitReader<OB::kAlong, BN, TN> fb;
    fa.init(wm * TM, lane);
    fb.init(wn * TN, lane);
    f32x4_t raw[N_FRAG][2];
    SplitFrag frag[2][N_FRAG];   // the TM of A, then the TN of B
    auto read_raw = [&](int f, int slot, int kk) {
        if (f < TM) fa.read(smem + slot, f, kk, raw[f]);
        else fb.read(smem + slot + BM * kLineBytes, f - TM, kk, raw[f]);
    };
    __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * PASSES + EARLY));
    __syncthreads();
#pragma unroll
    for (int f = 0; f < N_FRAG; ++f) read_raw(f, 0, 0);
#pragma unroll
    for (int i = 0; i < N_PAIR; ++i) split_pair(frag[0][i >> 2], raw[i >> 2], i & 3);
    int slot = 0, before = (NS - 1) * STAGE;   // of stage h and of the one before it
    for (int h = 0; h < n_st; ++h) {
        const int after = slot == (NS - 1) * STAGE ? 0 : slot + STAGE;
#pragma unroll
        for (int kk = 0; kk < KSTEPS; ++kk) {
            const bool last = kk + 1 == KSTEPS;
            if (last) {   // this stage has been read; the next one must have landed
                __builtin_amdgcn_s_waitcnt(kLgkm0);
                __builtin_amdgcn_s_waitcnt(vmcnt_imm((NS - 2) * PASSES));
                asm volatile("" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
            }
#pragma unroll
            for (int m = 0; m < N_MMA; ++m) {
#pragma unroll
                for (int f = m * N_FRAG / 2; f < (m + 1) * N_FRAG / 2 && f < N_FRAG; ++f) read_raw(f, last ? after : slot, last ? 0 : 1);
                const int b = m % N_BLOCK, p = m / N_BLOCK;
                acc[b / TN][b % TN] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(split_part(frag[kk][b / TN], kSplitA[p]), split_part(frag[kk][TM + b % TN], kSplitB[p]), acc[b / TN][b % TN], 0, 0, 0);
                if (last) {
#pragma unroll
                    for (int q = m * EARLY / N_MMA; q < (m + 1) * EARLY / N_MMA; ++q) issue_piece(q, h + NS, slot);
                } else {
#pragma unroll
                    for (int q = EARLY + m * (PASSES - EARLY) / N_MMA; q < EARLY + (m + 1) * (PASSES - EARLY) / N_MMA; ++q) issue_piece(q, h + NS - 1, before);
                }
                if (m >= WAIT) {
#pragma unroll
                    for (int i = (m - WAIT) * N_PAIR / (N_MMA - WAIT); i < (m + 1 - WAIT) * N_PAIR / (N_MMA - WAIT); ++i) split_pair(frag[kk ^ 1][i >> 2], raw[i >> 2], i & 3);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        before = slot;
        slot = after;
    }
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));   // the stages requested again may still be landing in the ring
    __syncthreads();
}

// ---- a tile's sums as rows: 32 rows of every wavefront row at a time pass through the LDS.  out.start(c, valid): the thread's V columns from c on, the same for all of
// its rows, of which `valid` exist; out.row(m, valid, v): their sums in row m. ----
template <int BM, int BN, int WGM>
constexpr size_t rows_lds() { return (size_t)32 * WGM * (BN + 4) * 4; }

template <int WGN, int TM, int TN>
__device__ __forceinline__ void strip_to_lds(float* tile, int pitch, const f32x16_t (&acc)[TM][TN], int i) {
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wv / WGN, wn = wv % WGN;
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e)
            tile[(wm * 32 + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3)) * pitch + (wn * TN + j) * 32 + (lane & 31)] = acc[i][j][e];
}

template <int BM, int BN, int WGM, int WGN, int V, class Out>
__device__ __forceinline__ void tile_as_rows(unsigned char* smem, const f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32], int m0, int n0, int M, int N, Out& out) {
    constexpr int NT = WGM * WGN * 64, PITCH = BN + 4, GROUPS = BN / V, STEP = NT / GROUPS;
    static_assert(NT % GROUPS == 0 && V % 4 == 0, "a thread keeps its columns");
    float* const tile = reinterpret_cast<float*>(smem);
    const int tid = threadIdx.x, c = (tid % GROUPS) * V, valid = N - n0 - c;
    if (valid > 0) out.template start<V>(n0 + c, valid);
#pragma unroll
    for (int i = 0; i < BM / WGM / 32; ++i) {
        if (i > 0) __syncthreads();
        strip_to_lds<WGN>(tile, PITCH, acc, i);
        __syncthreads();
        for (int r = tid / GROUPS; r < 32 * WGM; r += STEP) {
            const int m = m0 + (r >> 5) * (BM / WGM) + i * 32 + (r & 31);
            if (m >= M || valid <= 0) continue;
            float v[V];
#pragma unroll
            for (int q = 0; q < V; q += 4) *reinterpret_cast<f32x4_t*>(v + q) = *reinterpret_cast<const f32x4_t*>(tile + r * PITCH + c + q);
            out.template row<V>(m, n0 + c, valid, v);
        }
    }
}

// The same for the two products of a gated block (PairedRows): BN / 2 columns of each; out.row(m, c, valid, first's sums, second's sums).
template <int BM, int BN, int WGM, int WGN, int V, class Out>
__device__ __forceinline__ void pair_as_rows(unsigned char* smem, const f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32], int m0, int n0, int M, int N, Out& out) {
    constexpr int NT = WGM * WGN * 64, PITCH = BN + 4, GROUPS = BN / 2 / V, STEP = NT / GROUPS, HALF = BN / WGN / 2;
    static_assert(NT % GROUPS == 0 && V % 4 == 0 && HALF % 32 == 0, "a thread keeps its columns");
    float* const tile = reinterpret_cast<float*>(smem);
    const int tid = threadIdx.x, c = (tid % GROUPS) * V, valid = N - n0 - c, at = c / HALF * 2 * HALF + c % HALF;
    if (valid > 0) out.template start<V>(n0 + c, valid);
#pragma unroll
    for (int i = 0; i < BM / WGM / 32; ++i) {
        if (i > 0) __syncthreads();
        strip_to_lds<WGN>(tile, PITCH, acc, i);
        __syncthreads();
        for (int r = tid / GROUPS; r < 32 * WGM; r += STEP) {
            const int m = m0 + (r >> 5) * (BM / WGM) + i * 32 + (r & 31);
            if (m >= M || valid <= 0) continue;
            float v[V], w[V];
#pragma unroll
            for (int q = 0; q < V; q += 4) {
                *reinterpret_cast<f32x4_t*>(v + q) = *reinterpret_cast<const f32x4_t*>(tile + r * PITCH + at + q);
                *reinterpret_cast<f32x4_t*>(w + q) = *reinterpret_cast<const f32x4_t*>(tile + r * PITCH + at + HALF + q);
            }
            out.template row<V>(m, n0 + c, valid, v, w);
        }
    }
}

// The same where the tile's neurons have places of their own in the result's rows (a list of columns, ablated ones between them): the columns from behind the tile before to this one's
// last neuron are one range, which passes through the LDS in windows of EL::COLS at its final columns.  out.listed(m, c, first, valid, v, gaps, flat): V columns from c on, of
// which [first, valid) are this tile's; columns with their bit in gaps are ablated and are `flat`.  out.stored(m, s, valid, v): sums (with bias) of neurons s .. in their own
// order, where out.wants_stored().
template <int BN, int V, class Out>
__device__ __forceinline__ TileColumns listed_columns(int n0, const Out& out) {
    TileColumns cols = tile_columns(n0, BN, out.active, out.n_active, out.d_out, 0);
    cols.base = cols.lo / V * V;   // (16-byte stores begin at whole pieces of the row)
    return cols;
}
// (tables: of the first window, filled)
template <int BM, int BN, int WGM, int WGN, int V, class Out>
__device__ __forceinline__ void listed_as_rows(unsigned char* smem, unsigned char* tables, const f32x16_t (&acc)[BM / WGM / 32][BN / WGN / 32], int m0, int n0, int M, Out& out) {
    using EL = EpiLayout<BN, WGM>;
    constexpr int NT = WGM * WGN * 64, TM = BM / WGM / 32, TN = BN / WGN / 32, PITCH = EL::PITCH;
    static_assert(NT >= EL::COLS / V && EL::COLS >= BN, "columns to the threads");
    float* const tile = reinterpret_cast<float*>(smem);
    const int* const place = reinterpret_cast<const int*>(tables);
    const int* const table = place + BN;
    float* const tbias = reinterpret_cast<float*>(tables + (size_t)(BN + EL::COLS) * 4);
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wv / WGN, wn = wv % WGN;
    const TileColumns cols = listed_columns<BN, V>(n0, out);
    if (out.wants_stored()) {
        const int c = (tid % (BN / V)) * V, valid = cols.stored - c;
        if (valid > 0) out.template start<V>(n0 + c, valid);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            strip_to_lds<WGN>(tile, PITCH, acc, i);
            __syncthreads();
            for (int r = tid / (BN / V); r < 32 * WGM; r += NT / (BN / V)) {
                const int m = m0 + (r >> 5) * (BM / WGM) + i * 32 + (r & 31);
                if (m >= M || valid <= 0) continue;
                float v[V];
#pragma unroll
                for (int q = 0; q < V; q += 4) *reinterpret_cast<f32x4_t*>(v + q) = *reinterpret_cast<const f32x4_t*>(tile + r * PITCH + c + q);
                out.template stored<V>(m, n0 + c, valid, v);
            }
            __syncthreads();
        }
    }
    for (int cc = cols.base; cc <= cols.hi; cc += EL::COLS) {
        const int wc = min(EL::COLS, cols.hi - cc + 1), head = max(cols.lo - cc, 0);
        if (cc != cols.base) {
            __syncthreads();   // the window before is done with the tables
            fill_table<BN, WGM, NT>(tables, cc, cols, n0, out.active, out.bias);
        }
        __syncthreads();
        int at[TN];   // this lane's columns in the window
        float add[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int q = place[(wn * TN + j) * 32 + (lane & 31)];
            at[j] = q < 0 ? -1 : q - (cc - cols.base);
            if (at[j] >= wc) at[j] = -1;
            add[j] = tbias[max(at[j], 0)];
        }
        // As many threads to a row as the window has columns for, those behind the last whole row of threads idle: a thread keeps its V columns, and none works on columns behind the range, which is 1.25 tile widths
        // with a fifth ablated and the window two (bf16 4096 -> 16384 at 2048 rows with GELU, a fifth ablated, 272 -> 253 us; 104 -> 3001, half ablated, 500 rows in 128 x 128 tiles 37 -> 25).
        const int groups = (wc + V - 1) / V, step = NT / groups, k0 = (tid % groups) * V, first = max(head - k0, 0), valid = tid < step * groups ? min(V, wc - k0) : 0;
        int gaps = 0;
        float flat[V];
#pragma unroll
        for (int q = 0; q < V; ++q) {
            const int k = min(max(k0 + q, head), wc - 1);
            if (table[k] < 0) gaps |= 1 << q;
            flat[q] = tbias[k];
        }
        out.template gap_values<V>(gaps, flat);
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            if (i > 0 || cc != cols.base) __syncthreads();   // the rows before have been read
#pragma unroll
            for (int j = 0; j < TN; ++j)
                if (at[j] >= 0) {
                    float* const t = tile + (wm * 32 + 4 * (lane >> 5)) * PITCH + at[j];
#pragma unroll
                    for (int e = 0; e < 16; ++e) t[(8 * (e >> 2) + (e & 3)) * PITCH] = acc[i][j][e] + add[j];
                }
            __syncthreads();
            for (int r = tid / groups; r < 32 * WGM; r += step) {
                const int m = m0 + (r >> 5) * (BM / WGM) + i * 32 + (r & 31);
                if (m >= M || valid <= first) continue;
                float v[V];
#pragma unroll
                for (int q = 0; q < V; q += 4) *reinterpret_cast<f32x4_t*>(v + q) = *reinterpret_cast<const f32x4_t*>(tile + r * PITCH + k0 + q);
                out.template listed<V>(m, cc + k0, first, valid, v, gaps, flat);
            }
        }
    }
}

// ---- values in and out ----
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return bf16_bits_to_float(v); }
// (bf16: to nearest, ties to even)
template <typename T> __device__ __forceinline__ T from_float(float v) {
    if constexpr (sizeof(T) == 4) return v;
    else return __builtin_bit_cast(uint16_t, (__bf16)v);
}
// ONCE: not read again soon and in whole pieces at 16-byte addresses: past the caches (gradients of a gated block, bf16 4096 x 16384 at 2048 rows, 1002 -> 983 us; pieces that begin anywhere 41 -> 42)
template <typename T, int V, bool ONCE = false>
__device__ __forceinline__ void store_values(T* p, const float (&v)[V], int valid, int first = 0) {
    if (valid >= V && first <= 0) {
        typename AnyPlace<T, V>::type w;
#pragma unroll
        for (int q = 0; q < V; ++q) w[q] = from_float<T>(v[q]);
        if (ONCE && (reinterpret_cast<uintptr_t>(p) & 15) == 0) __builtin_nontemporal_store(w, reinterpret_cast<typename AnyPlace<T, V>::type*>(p));
        else *reinterpret_cast<typename AnyPlace<T, V>::type*>(p) = w;
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q)
            if (q >= first && q < valid) p[q] = from_float<T>(v[q]);
    }
}
template <typename T, int V>
__device__ __forceinline__ void load_values(const T* p, float (&v)[V], int valid, int first = 0) {
    if (valid >= V && first <= 0) {
        const typename AnyPlace<T, V>::type w = *reinterpret_cast<const typename AnyPlace<T, V>::type*>(p);
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = to_float((T)w[q]);
    } else {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = q >= first && q < valid ? to_float(p[q]) : 0.0f;
    }
}

// The activations of these products and their slopes, for millions of values behind a product: one hardware exponential (of two) and one reciprocal each.
// GELU: Phi(-|v|) = erfc(|v| / sqrt 2) / 2 by Abramowitz and Stegun 7.1.26, a polynomial of degree 5 in t = 1 / (1 + p |v| / sqrt 2) times exp(-v^2 / 2), which is the density's exponential
// too; |error of erf| <= 1.5e-7, a step or two of fp32 beside 1.  (With erff the epilogue of 2048 x 13108 values was 40 us of vector instructions.)
// SiLU: the exponential is off by |v| 2^-24 of itself, the reciprocal by a step.  NaN stays NaN in all of them (ReLU's slope there is 0).
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896340736f); }
__device__ __forceinline__ float logistic(float v) { return __builtin_amdgcn_rcpf(1.0f + exp_of(-v)); }
// Phi(-|v|), and exp(-v^2 / 2)  (1 / sqrt 2, 1 / 2 and the exponential's log2 e are in the constants)
__device__ __forceinline__ float normal_tail(float v, float* e) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.23164189f, fabsf(v), 1.0f));
    *e = __builtin_amdgcn_exp2f(-0.72134752044448170368f * v * v);
    return *e * t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f);
}
__device__ __forceinline__ float act_value(float v, int act) {
    if (act == SRIGL_ACT_SILU) return v * logistic(v);
    if (act == SRIGL_ACT_RELU) return v < 0.0f ? 0.0f : v;
    if (act == SRIGL_ACT_GELU) {
        float e;
        const float q = normal_tail(v, &e);
        return v * (v < 0.0f ? q : 1.0f - q);
    }
    return v;
}
__device__ __forceinline__ float act_slope(float v, int act) {
    if (act == SRIGL_ACT_RELU) return v > 0.0f ? 1.0f : 0.0f;
    if (act == SRIGL_ACT_GELU) {
        float e;
        const float q = normal_tail(v, &e);
        return (v < 0.0f ? q : 1.0f - q) + v * e * 0.39894228040143267794f;
    }
    if (act == SRIGL_ACT_SILU) {
        const float p = logistic(v);
        return p * (1.0f + v * (1.0f - p));
    }
    return 1.0f;
}

// The same of V values, the choice made once for all: with a branch a value their chains of instructions followed each other (bf16 4096 -> 16384 at 2048 rows, in
// the epilogue: gated with SiLU 505 us, now 460, a layer with GELU 298 and 278)
template <int V>
__device__ __forceinline__ void act_values(float (&v)[V], int act) {
    const auto each = [&](int kind) {
#pragma unroll
        for (int q = 0; q < V; ++q) v[q] = act_value(v[q], kind);
    };
    if (act == SRIGL_ACT_GELU) each(SRIGL_ACT_GELU);
    else if (act == SRIGL_ACT_SILU) each(SRIGL_ACT_SILU);
    else if (act == SRIGL_ACT_RELU) each(SRIGL_ACT_RELU);
}
template <int V>
__device__ __forceinline__ void act_slopes(const float (&v)[V], float (&slope)[V], int act) {
    const auto each = [&](int kind) {
#pragma unroll
        for (int q = 0; q < V; ++q) slope[q] = act_slope(v[q], kind);
    };
    if (act == SRIGL_ACT_GELU) each(SRIGL_ACT_GELU);
    else if (act == SRIGL_ACT_SILU) each(SRIGL_ACT_SILU);
    else if (act == SRIGL_ACT_RELU) each(SRIGL_ACT_RELU);
    else each(SRIGL_ACT_NONE);
}

// ---- kernel and launch ----
// A dimension of a grid ends below 2^32 threads: more workgroups of so many threads than that stand in `times` layers of x each (whole eights, so that a workgroup's die is the one that tile_of_workgroup
// expects; those behind the last one find nothing to do).
struct GridLayers { unsigned x, times; };
inline GridLayers grid_layers(long long groups, int threads) {
    const long long most = ((1ll << 32) - 1) / threads / kXcds * kXcds, times = std::max(1ll, (groups + most - 1) / most), x = (groups + times - 1) / times;
    return {(unsigned)(times == 1 ? x : (x + kXcds - 1) / kXcds * kXcds), (unsigned)times};
}
constexpr long long kMostGroups = 0x7fffff00ll;   // numbers of workgroups are ints

// Sums of a part of K, [parts][M][N] (of a pair: [parts][M][2 N], the second's behind the first's)
struct PartOut {
    static constexpr bool kListed = false;
    float* part;
    int N;
    long long pitch;
    template <int V> __device__ void start(int, int) {}
    template <int V> __device__ void row(int m, int c, int valid, const float (&v)[V]) { store_values<float, V>(part + (size_t)m * pitch + c, v, valid); }
    template <int V> __device__ void row(int m, int c, int valid, const float (&v)[V], const float (&w)[V]) {
        store_values<float, V>(part + (size_t)m * pitch + c, v, valid);
        store_values<float, V>(part + (size_t)m * pitch + N + c, w, valid);
    }
};
// Whether some sum of the tile is not finite, for all wavefronts alike
template <int NWAVES, int TM, int TN>
__device__ __forceinline__ bool not_finite(unsigned char* smem, const f32x16_t (&acc)[TM][TN]) {
    bool odd = false;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) odd |= !(fabsf(acc[i][j][e]) <= 3.4028234e38f);
    int* const flags = reinterpret_cast<int*>(smem);
    const int any = __any(odd);
    if ((threadIdx.x & 63) == 0) flags[threadIdx.x >> 6] = any;
    __syncthreads();
    odd = false;
    for (int w = 0; w < NWAVES; ++w) odd |= flags[w] != 0;
    __syncthreads();
    return odd;
}

// One product: M x N results (PAIR: of both matrices) of `stages` stages of K, in `parts` parts whose sums go to `part` and are joined by a second launch.
template <class OA, class OB, class Out>
struct DenseProduct {
    OA oa;
    OB ob;
    Out out;
    int M, N, stages, parts;
    float* part;
};

template <int BM, int BN, int WGM, int NS, bool LISTED>
constexpr size_t dense_lds() {
    const size_t ring = (size_t)(NS > 0 ? NS : 1) * (BM + BN) * kLineBytes, rows = LISTED ? EpiLayout<BN, WGM>::TILE_BYTES : rows_lds<BM, BN, WGM>();
    return (ring > rows ? ring : rows) + (LISTED ? EpiLayout<BN, WGM>::TABLE_BYTES : 0);
}
// Tile `id` (of tile_of_workgroup's order) and part `part_no` of a product.  NS: stages of the ring of direct loads, 0: staged through registers.
template <typename T, int BM, int BN, int WGM, int WGN, int NS, bool PAIR, class OA, class OB, class Out>
__device__ __forceinline__ void dense_tile(unsigned char* smem, int id, int part_no, DenseProduct<OA, OB, Out>& p) {
    constexpr int COLS = PAIR ? BN / 2 : BN, V = kPiece<T>;
    int tile_m, tile_n;
    if (!tile_of_workgroup(id, (p.M + BM - 1) / BM, (p.N + COLS - 1) / COLS, &tile_m, &tile_n)) return;
    const int m0 = tile_m * BM, n0 = tile_n * COLS, parts = p.parts;
    p.oa.move(m0);
    p.ob.move(n0);
    const int stages = NS > 0 ? p.ob.whole() : p.stages;
    const int h0 = parts == 1 ? 0 : (int)((long long)part_no * stages / parts), h1 = parts == 1 ? stages : (int)((long long)(part_no + 1) * stages / parts);
    f32x16_t acc[BM / WGM / 32][BN / WGN / 32];
    const auto clear = [&] {
#pragma unroll
        for (int i = 0; i < BM / WGM / 32; ++i)
#pragma unroll
            for (int j = 0; j < BN / WGN / 32; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    };
    clear();
    constexpr bool SPLIT = sizeof(T) == 4;
    // (a list's tables stand behind everything else in the LDS, filled while the first stages come: two waits for memory that a small product would end with)
    unsigned char* const tables = smem + dense_lds<BM, BN, WGM, NS, Out::kListed>() - (Out::kListed ? EpiLayout<BN, WGM>::TABLE_BYTES : 0);
    const auto meanwhile = [&] {
        if constexpr (Out::kListed)
            if (p.out.active && parts == 1) {
                const TileColumns cols = listed_columns<BN, V>(n0, p.out);
                fill_table<BN, WGM, WGM * WGN * 64>(tables, cols.base, cols, n0, p.out.active, p.out.bias);
            }
    };
    if constexpr (NS == 0) {
        meanwhile();
        product_of_tile<T, SPLIT, BM, BN, WGM, WGN>(smem, p.oa, p.ob, h0, h1, acc);
    } else if constexpr (SPLIT) {
        split_product_of_tile<BM, BN, WGM, WGN, NS>(smem, p.oa, p.ob, h0, h1, acc, meanwhile);
    } else {
        direct_product_of_tile<T, BM, BN, WGM, WGN, NS>(smem, p.oa, p.ob, h0, h1, acc, meanwhile);
    }
    if constexpr (SPLIT)
        if (not_finite<WGM * WGN>(smem, acc)) {
            clear();
            for (int h = h0; h < h1; ++h) {
                const int stage = NS > 0 ? p.ob.index(h) : h;
                product_of_tile<T, false, BM, BN, WGM, WGN>(smem, p.oa, p.ob, stage, stage + 1, acc);
            }
        }
    if (NS > 0 && part_no == parts - 1)
        for (int t = 0; t < p.ob.tails(); ++t) product_of_tile<T, false, BM, BN, WGM, WGN>(smem, p.oa, p.ob, p.ob.tail(t), p.ob.tail(t) + 1, acc);
    if (parts > 1) {
        const long long pitch = PAIR ? 2ll * p.N : p.N;
        PartOut to{p.part + (size_t)part_no * p.M * pitch, p.N, pitch};
        if constexpr (PAIR) pair_as_rows<BM, BN, WGM, WGN, 4>(smem, acc, m0, n0, p.M, p.N, to);
        else tile_as_rows<BM, BN, WGM, WGN, 4>(smem, acc, m0, n0, p.M, p.N, to);
        return;
    }
    if constexpr (Out::kListed)
        if (p.out.active) {
            listed_as_rows<BM, BN, WGM, WGN, V>(smem, tables, acc, m0, n0, p.M, p.out);
            return;
        }
    if constexpr (PAIR) pair_as_rows<BM, BN, WGM, WGN, V>(smem, acc, m0, n0, p.M, p.N, p.out);
    else tile_as_rows<BM, BN, WGM, WGN, V>(smem, acc, m0, n0, p.M, p.N, p.out);
}

template <typename T, int BM, int BN, int WGM, int WGN, int NS, bool PAIR, class P>
__global__ __launch_bounds__(WGM * WGN * 64) void k_dense(P p) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    int id = blockIdx.x;
    if (blockIdx.z) id += (int)(blockIdx.z * gridDim.x);
    dense_tile<T, BM, BN, WGM, WGN, NS, PAIR>(smem, id, blockIdx.y, p);
}

// Two products that do not wait for each other in one launch (the gradients of x and of W): what one leaves idle the other takes, and a small pass is a launch shorter.  The first one's workgroups come
// first, then the second one's; both are whole multiples of 8 a part, so that a workgroup's die is the one that tile_of_workgroup expects.
// Behind both come the workgroups of something else that waits for neither: more(smem, its workgroup).
template <typename T, int BM, int BN, int WGM, int WGN, int NS, class P, class Q, class More>
__global__ __launch_bounds__(WGM * WGN * 64) void k_dense_two(P p, Q q, int p_wg, int q_wg, More more) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    int id = blockIdx.x;
    if (id >= p_wg * p.parts + q_wg * q.parts) {
        more(smem, id - (p_wg * p.parts + q_wg * q.parts));
        return;
    }
    if (id < p_wg * p.parts) {
        dense_tile<T, BM, BN, WGM, WGN, NS, false>(smem, id % p_wg, id / p_wg, p);
    } else {
        id -= p_wg * p.parts;
        dense_tile<T, BM, BN, WGM, WGN, NS, false>(smem, id % q_wg, id / q_wg, q);
    }
}

// ---- ablated columns where the stored neurons' are written one by one (few rows of x, and the join of parts) ----
// the place lo .. hi in the ascending list in front of which all entries are < c, by a whole wavefront: a trip to memory for each 6 bits of hi - lo
__device__ __forceinline__ int wave_place_of(const int32_t* active, int lo, int hi, int c) {
    const int lane = threadIdx.x & 63;
    while (lo < hi) {
        const int step = (hi - lo + 63) >> 6, at = lo + (lane + 1) * step - 1;
        lo += __popcll(__ballot(at < hi && active[min(at, hi - 1)] < c)) * step;
        hi = min(hi, lo + step - 1);
    }
    return lo;
}
// They have workgroups of their own, NT columns and kAblatedRows rows each, in front of the others in the same launch: a thread its column, whatever run of neighbours it stands in.  (The thread of the neuron
// behind a run wrote it, an element after the other, 0.13 to 0.3 us each, since the residual may be y: 4096 -> 16384 bf16 at one row, half of the neurons ablated at one end, 1140 us and at random 16.7, now 16.8 and 17.0;
// in the kernel trace, at random, 3072 -> 768 with 538 stored at 16 rows 7.2 and now 6.7, 768 -> 768 with a fifth ablated at 64 11.6 and 7.1, the join of 2048 -> 1024 at 40 5.8 and 4.7; with short lines the search is what is
// waited for: 128 -> 12000 at 8 rows 4.2 and 4.6.)
constexpr int kAblatedRows = 16;
template <int NT, class Out> inline long long ablated_groups(int B, const Out& out) {
    if constexpr (Out::kListed)
        if (out.active) return ((out.d_out + (long long)NT - 1) / NT) * ((B + kAblatedRows - 1ll) / kAblatedRows);
    return 0;
}
template <int NT, class Out>
__device__ __forceinline__ void write_ablated(int group, int B, const Out& out) {
    __shared__ int stored[NT];
    const int tid = threadIdx.x, slices = (int)((out.d_out + (long long)NT - 1) / NT), c0 = group % slices * NT, c = c0 + tid;
    const int m0 = group / slices * kAblatedRows, m1 = min(m0 + kAblatedRows, B);
    const bool there = c < out.d_out;
    const float flat = out.ablated_value(there ? c : 0);
    stored[tid] = 0;
    // The slice's neurons begin at their column's number in the list less the ablated columns in front, some of all that there are: where these are few, everything from the first possible place on is read
    // (one trip; 1001 -> 777 with a tenth ablated at 37 rows, the join of parts 5.0 us with a search, 4.4 without).
    const int n = out.n_active, gone = out.d_out - n;
    int lo = max(c0 - gone, 0), hi = min(c0, n);
    if (hi - lo > 3 * NT) hi = lo = wave_place_of(out.active, lo, hi, c0);
    int entry[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int k = lo + i * NT + tid;
        entry[i] = k < min(hi + NT, n) ? out.active[k] : -1;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (entry[i] >= c0 && entry[i] - c0 < NT) stored[entry[i] - c0] = 1;
    __syncthreads();
    if (there && !stored[tid]) out.template ablated_rows<kAblatedRows>(c, m0, m1, flat);
}

// ---- joining the parts' sums: a thread takes V columns of a row; eight parts' values are requested together, so that it waits for memory once or twice ----
template <int V, bool PAIR, class P>
__device__ __forceinline__ void dense_join(long long item, P& p) {
    constexpr int TOGETHER = 8;
    const int groups = (p.N + V - 1) / V, m = (int)(item / groups), c = (int)(item - (long long)m * groups) * V, valid = p.N - c;
    if (m >= p.M) return;
    p.out.template start<V>(c, valid);
    const long long pitch = PAIR ? 2ll * p.N : p.N;
    float v[V] = {}, w[V] = {};
    for (int z0 = 0; z0 < p.parts; z0 += TOGETHER) {
        float t[TOGETHER][V] = {}, u[TOGETHER][V] = {};
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k) {
            const float* const at = p.part + ((size_t)min(z0 + k, p.parts - 1) * p.M + m) * pitch + c;
            load_values<float, V>(at, t[k], valid);
            if constexpr (PAIR) load_values<float, V>(at + p.N, u[k], valid);
        }
#pragma unroll
        for (int k = 0; k < TOGETHER; ++k)
            if (z0 + k < p.parts)
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    v[q] += t[k][q];
                    if constexpr (PAIR) w[q] += u[k][q];
                }
    }
    if constexpr (PAIR) p.out.template row<V>(m, c, valid, v, w);
    else p.out.template row<V>(m, c, valid, v);
}
template <bool PAIR, class P>
__global__ __launch_bounds__(256) void k_dense_join(P p) { dense_join<4, PAIR>((long long)blockIdx.x * 256 + threadIdx.x, p); }
// with a list a neuron to a thread, behind the ablated columns' workgroups
template <class P>
__global__ __launch_bounds__(256) void k_dense_join_listed(P p, int ablated) {
    int id = blockIdx.x;
    if (blockIdx.y) id += (int)(blockIdx.y * gridDim.x);
    if (id < ablated) write_ablated<256>(id, p.M, p.out);
    else dense_join<1, false>((long long)(id - ablated) * 256 + threadIdx.x, p);
}
template <class P, class Q>
__global__ __launch_bounds__(256) void k_dense_join_two(P p, Q q, unsigned p_groups) {
    if (blockIdx.x < p_groups) dense_join<4, false>((long long)blockIdx.x * 256 + threadIdx.x, p);
    else dense_join<4, false>((long long)(blockIdx.x - p_groups) * 256 + threadIdx.x, q);
}
// workgroups of a join
template <class P> inline long long join_groups(const P& p, int V) { return p.parts > 1 ? ((long long)p.M * ((p.N + V - 1ll) / V) + 255) / 256 : 0; }

// workgroups of a part
template <int BM, int COLS, class P> inline long long dense_groups(const P& p) {
    return (((p.M + BM - 1ll) / BM) * ((p.N + COLS - 1ll) / COLS) + kXcds - 1) / kXcds * kXcds;
}

template <typename T, int BM, int BN, int WGM, int WGN, int NS, bool PAIR, class OA, class OB, class Out>
static srigl_status launch_tiles(const DenseProduct<OA, OB, Out>& p, hipStream_t st) {
    using P = DenseProduct<OA, OB, Out>;
    constexpr size_t lds = dense_lds<BM, BN, WGM, NS, Out::kListed>();
    static_assert(lds <= kLdsMax, "LDS");
    auto kern = k_dense<T, BM, BN, WGM, WGN, NS, PAIR, P>;
    static LdsLimit limit;
    if (limit.ensure(kern, lds) != SRIGL_OK) return SRIGL_ERR_HIP;
    const long long n_wg = dense_groups<BM, PAIR ? BN / 2 : BN>(p);
    if (n_wg > kMostGroups || p.parts < 1 || p.parts > 65535) return SRIGL_ERR_UNSUPPORTED;
    const GridLayers grid = grid_layers(n_wg, WGM * WGN * 64);
    hipLaunchKernelGGL(kern, dim3(grid.x, (unsigned)p.parts, grid.times), dim3(WGM * WGN * 64), lds, st, p);
    if (p.parts > 1) {
        if constexpr (Out::kListed)
            if (p.out.active) {
                const long long ablated = ablated_groups<256>(p.M, p.out), all = ablated + join_groups(p, 1);
                if (all > kMostGroups) return SRIGL_ERR_UNSUPPORTED;
                const GridLayers layers = grid_layers(all, 256);
                hipLaunchKernelGGL((k_dense_join_listed<P>), dim3(layers.x, layers.times), dim3(256), 0, st, p, (int)ablated);
                return hip_ok(hipGetLastError());
            }
        hipLaunchKernelGGL((k_dense_join<PAIR, P>), dim3((unsigned)join_groups(p, 4)), dim3(256), 0, st, p);
    }
    return hip_ok(hipGetLastError());
}
template <typename T, int BM, int BN, int WGM, int WGN, int NS, class P, class Q, class More>
static srigl_status launch_tiles_two(const P& p, const Q& q, const More& more, hipStream_t st) {
    constexpr size_t lds = dense_lds<BM, BN, WGM, NS, false>();
    auto kern = k_dense_two<T, BM, BN, WGM, WGN, NS, P, Q, More>;
    static LdsLimit limit;
    if (limit.ensure(kern, lds) != SRIGL_OK) return SRIGL_ERR_HIP;
    const long long p_wg = dense_groups<BM, BN>(p), q_wg = dense_groups<BM, BN>(q), all = p_wg * p.parts + q_wg * q.parts + more.groups();
    if (all * WGM * WGN * 64 >= 1ll << 32) return SRIGL_ERR_UNSUPPORTED;   // (pairs of products beyond a quarter of a millisecond don't come here)
    hipLaunchKernelGGL(kern, dim3((unsigned)all), dim3(WGM * WGN * 64), lds, st, p, q, (int)p_wg, (int)q_wg, more);
    const long long pj = join_groups(p, 4), qj = join_groups(q, 4);
    if (pj + qj > 0) hipLaunchKernelGGL((k_dense_join_two<P, Q>), dim3((unsigned)(pj + qj)), dim3(256), 0, st, p, q, (unsigned)pj);
    return hip_ok(hipGetLastError());
}

// Tile and parts of K of a product (of a pair: N neurons, two sums each)
struct DensePlan { int tile, parts; };
enum { kTileS = 0, kTileM = 1, kTileH = 2, kTileL = 3, kTileS2 = 4, kTileM2 = 5 };   // 64 x 64 (of a pair 64 x 128), 128 x 128, 256 x 128 (direct loads) and 256 x 256 (and bf16)
// S2, M2: S and M with two stages of the ring in place of four, so that five and two workgroups share a compute unit: one stores while another loads, for short K and large results
enum DenseKind { kDenseForward = 0, kDensePair = 1, kDenseGradX = 2, kDenseGradW = 3 };   // a layer's forward product, a gated block's, gradients of x and of W
// direct: rows are multiples of 16 bytes (a choice by sizes, so that the workspace does not depend on addresses)
DensePlan plan_dense(DenseKind kind, int M, int N, int stages, bool f32, bool direct);
// Both gradients' products (of x: B x d_in over K; of W: rows x d_in over B): tile and parts of each; together: one launch in tiles of one shape
struct DensePlans { DensePlan dx, dW; bool together; };
DensePlans plan_gradients(int B, int d_in, int K_stages, int rows, int B_stages, bool f32, bool direct);
// bytes of the parts' sums
inline size_t part_bytes(DensePlan p, int M, int N, bool pair) { return p.parts > 1 ? (size_t)p.parts * M * N * (pair ? 2 : 1) * sizeof(float) : 0; }

template <typename T, bool PAIR, class OA, class OB, class Out>
static srigl_status launch_dense(const DenseProduct<OA, OB, Out>& p, int tile, hipStream_t st) {
    if (p.M <= 0 || p.N <= 0) return SRIGL_OK;
    constexpr int SN = PAIR ? 128 : 64;
    if (!(p.oa.direct(256) && p.ob.direct(256))) {
        if (tile == kTileS) return launch_tiles<T, 64, SN, 2, 2, 0, PAIR>(p, st);
        return launch_tiles<T, 128, 128, 2, 2, 0, PAIR>(p, st);
    }
    if constexpr (sizeof(T) == 2)
        if (tile == kTileL) return launch_tiles<T, 256, 256, 2, 4, 2, PAIR>(p, st);
    if (tile == kTileH || tile == kTileL) return launch_tiles<T, 256, 128, 4, 2, 3, PAIR>(p, st);
    // 128 x 128 by eight wavefronts where both operands' lines run along K, in bf16 (four of 64 x 64 leave each SIMD one, which waits at every barrier: 512 rows, 768 -> 3072, 15.2 us, now 11.5); the
    // transposing reads of half as wide wavefronts are 1.5 times as many (gradient of W, 2048 rows, 4096 -> 4096, 83.5 us against 77.8), and so is the cutting of fp32 (forward, 409 and 364)
    constexpr bool EIGHT = sizeof(T) == 2 && OA::kAlong && OB::kAlong;
    if (tile == kTileM) return launch_tiles<T, 128, 128, EIGHT && PAIR ? 4 : 2, EIGHT && !PAIR ? 4 : 2, 4, PAIR>(p, st);
    if (tile == kTileM2) return launch_tiles<T, 128, 128, EIGHT && PAIR ? 4 : 2, EIGHT && !PAIR ? 4 : 2, 2, PAIR>(p, st);
    if (tile == kTileS2) return launch_tiles<T, 64, SN, 2, 2, 2, PAIR>(p, st);
    return launch_tiles<T, 64, SN, 2, 2, 4, PAIR>(p, st);
}
// Both products in tiles of one shape, side by side
template <typename T, class P, class Q, class More>
static srigl_status launch_dense_two(const P& p, const Q& q, const More& more, int tile, hipStream_t st) {
    if (!(p.oa.direct(256) && p.ob.direct(256) && q.oa.direct(256) && q.ob.direct(256))) {
        if (tile == kTileS) return launch_tiles_two<T, 64, 64, 2, 2, 0>(p, q, more, st);
        return launch_tiles_two<T, 128, 128, 2, 2, 0>(p, q, more, st);
    }
    if constexpr (sizeof(T) == 2)
        if (tile == kTileL) return launch_tiles_two<T, 256, 256, 2, 4, 2>(p, q, more, st);
    if (tile == kTileH || tile == kTileL) return launch_tiles_two<T, 256, 128, 4, 2, 3>(p, q, more, st);
    if (tile == kTileM) return launch_tiles_two<T, 128, 128, 2, 2, 4>(p, q, more, st);
    if (tile == kTileM2) return launch_tiles_two<T, 128, 128, 2, 2, 2>(p, q, more, st);
    if (tile == kTileS2) return launch_tiles_two<T, 64, 64, 2, 2, 2>(p, q, more, st);
    return launch_tiles_two<T, 64, 64, 2, 2, 4>(p, q, more, st);
}
// ---- few rows of x ----
// Products with at most 64 rows of x are bound by reading the weights.  A workgroup takes 16 neurons (of a pair: of both matrices) and all of K, its wavefronts 128 bytes of the lines in turn, straight
// from memory into the matrix units' registers: v_mfma_f32_16x16x32_bf16 with lane l holding row l % 16, k = 8 (l / 16) .. + 7 (fp32: 16x16x4, k = 4 (l / 16) + j in the j-th of four),
// neurons against 16 rows of x, so that a batch of one costs what 16 do.  The wavefronts' sums meet in the LDS: no second launch.
typedef float f32x4_acc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void few_mma(f32x4_acc_t& acc, const uint4& a, const uint4& b, uint16_t) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), acc, 0, 0, 0);
}
__device__ __forceinline__ void few_mma(f32x4_acc_t& acc, const uint4& a, const uint4& b, float) {
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), acc, 0, 0, 0);
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), acc, 0, 0, 0);
}

// NB: blocks of 16 rows of x; UNITS of 128 bytes of a line requested together
template <typename T, int NB, int NW, bool PAIR, int UNITS, class Out>
__global__ __launch_bounds__(NW * 64) void k_dense_few(const T* __restrict__ x, int B, int K, const T* __restrict__ W, long long to_second, int n, int rows, int ablated, Out out) {
    constexpr int MATS = PAIR ? 2 : 1, STEP = 64 / (int)sizeof(T), UNIT = 2 * STEP, P = kPiece<T>;
    __shared__ float sums[NW][MATS][16][17];   // [neuron][row of x], of 16 rows of x at a time
    const int lane = threadIdx.x & 63, wv = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int id = blockIdx.x;
    if (blockIdx.y) id += (int)(blockIdx.y * gridDim.x);
    if constexpr (Out::kListed)
        if (id < ablated) return write_ablated<NW * 64>(id, B, out);
    if (id - ablated > (n - 1) / rows) return;   // (layers of a grid may end behind the last one)
    const int s0 = (id - ablated) * rows;
    const T *w[MATS], *xr[NB];
    const int off = (lane >> 4) * P;
    w[0] = W + (size_t)min(s0 + min(lane & 15, rows - 1), n - 1) * K + off;
    if constexpr (PAIR) w[1] = reinterpret_cast<const T*>(reinterpret_cast<const unsigned char*>(w[0]) + to_second);
#pragma unroll
    for (int b = 0; b < NB; ++b) xr[b] = x + (size_t)min(b * 16 + (lane & 15), B - 1) * K + off;
    f32x4_acc_t acc[MATS][NB] = {};
    const int units = K / UNIT;
    auto compute = [&](int first, int count, auto load) {
        uint4 wp[MATS][UNITS][2], xp[NB][UNITS][2];
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u < count)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int k = (first + u * NW) * UNIT + h * STEP;
#pragma unroll
                    for (int i = 0; i < MATS; ++i) wp[i][u][h] = load(w[i], k);
#pragma unroll
                    for (int b = 0; b < NB; ++b) xp[b][u][h] = load(xr[b], k);
                }
#pragma unroll
        for (int u = 0; u < UNITS; ++u)
            if (u < count)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int i = 0; i < MATS; ++i)
#pragma unroll
                        for (int b = 0; b < NB; ++b) few_mma(acc[i][b], wp[i][u][h], xp[b][u][h], T{});
    };
    const auto whole_piece = [&](const T* p, int k) { return load_piece(p + k, P); };
    for (int u = wv; u < units; u += NW * UNITS) compute(u, (units - u + NW - 1) / NW, whole_piece);
    if (K % UNIT && wv == units % NW) compute(units, 1, [&](const T* p, int k) { return load_piece(p + k, K - k - off); });
    const int s = threadIdx.x & 15, r = threadIdx.x >> 4;   // 256 threads write
    if (s < rows && s0 + s < n) out.template start<1>(s0 + s, 1);
#pragma unroll
    for (int b = 0; b < NB; ++b) {
        if (b > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < MATS; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[wv][i][4 * (lane >> 4) + e][lane & 15] = acc[i][b][e];
        __syncthreads();
        const int m = 16 * b + r;
        if (r >= 16 || s >= rows || s0 + s >= n || m >= B) continue;
        float v[1] = {}, u[1] = {};
#pragma unroll
        for (int k = 0; k < NW; ++k) {
            v[0] += sums[k][0][s][r];
            if constexpr (PAIR) u[0] += sums[k][1][s][r];
        }
        if constexpr (PAIR) out.template row<1>(m, s0 + s, 1, v, u);
        else out.template row<1>(m, s0 + s, 1, v);
    }
}

// Whether the products of B rows of x with lines of K elements run here: up to 16 rows always, more while x, which every workgroup reads again, is short (`units` of 128 bytes a line).  us, weights out of
// HBM, here against tiles: bf16 4096 -> 16384 at 1 row 24.8 and 34.4, at 16 31.9 and 32.6, at 32 45.8 and 32.5; 1024 -> 1024 at 32 4.6 and 7.3, at 64 7.1 and 8.0; gated 4096 -> 4096 at 32 17.5 and
// 19.3, at 64 26.5 and 21.4; fp32 3072 -> 768 at 16 11.2 and 12.4, at 32 16.9 and 12.7; 1001 -> 777 (pieces that begin anywhere) at 32 7.5 and 8.2, at 64 12.1 and 9.0.
inline bool few_rows(int B, int K, bool f32, bool pair) {
    const long long units = (long long)K * (f32 ? 4 : 2) / 128;
    return B <= 16 || (B <= 32 && units <= (pair ? 64 : 48)) || (B <= 64 && units <= (pair ? 24 : 16) && K % (f32 ? 4 : 8) == 0);
}
template <typename T, bool PAIR, class Out>
static srigl_status launch_few(const T* x, int B, int K, const T* W, long long to_second, int n, const Out& out, hipStream_t st) {
    // Few neurons: four of them to a workgroup (the others' places in the matrix units repeat the last one), since a compute unit alone brings in little: bf16 3072 -> 768 at one row 4.6 us against 5.8 with
    // 16, 1024 -> 1024 2.7 and 3.0, but 768 -> 3072 3.9 and 3.2.
    const int rows = n >= 2048 ? 16 : 4;
    const bool wide = (long long)K * (int)sizeof(T) >= 20 * 128;   // eight wavefronts to a line, else four (bf16 4096 -> 16384 at one row 24.8 us, 27.3 with four)
    const long long ablated = wide ? ablated_groups<512>(B, out) : ablated_groups<256>(B, out), all = ablated + (n + (long long)rows - 1) / rows;
    if (all > kMostGroups) return SRIGL_ERR_UNSUPPORTED;
    const GridLayers layers = grid_layers(all, wide ? 512 : 256);
    const dim3 grid(layers.x, layers.times);
#define SRIGL_FEW(NB, UNITS) \
    do { \
        if (wide) hipLaunchKernelGGL((k_dense_few<T, NB, 8, PAIR, UNITS, Out>), grid, dim3(512), 0, st, x, B, K, W, to_second, n, rows, (int)ablated, out); \
        else hipLaunchKernelGGL((k_dense_few<T, NB, 4, PAIR, UNITS, Out>), grid, dim3(256), 0, st, x, B, K, W, to_second, n, rows, (int)ablated, out); \
    } while (0)
    if (B <= 16) SRIGL_FEW(1, 4);
    else if (B <= 32) SRIGL_FEW(2, PAIR ? 2 : 3);
    else SRIGL_FEW(4, 2);
#undef SRIGL_FEW
    return hip_ok(hipGetLastError());
}
template <typename T> inline int stages_of(long long K) { return (int)((K + kStageK<T> - 1) / kStageK<T>); }

constexpr int kMaxSide = 1 << 30;   // rows and columns of a product
inline bool known_dtype(srigl_dtype t) { return t == SRIGL_F32 || t == SRIGL_BF16; }
inline bool known_act(srigl_activation a) { return a == SRIGL_ACT_NONE || a == SRIGL_ACT_RELU || a == SRIGL_ACT_GELU || a == SRIGL_ACT_SILU; }
inline size_t dtype_bytes(srigl_dtype t) { return t == SRIGL_F32 ? 4 : 2; }
inline bool scratch_fits(const void* ws, size_t bytes, size_t need) { return need == 0 || (ws != nullptr && bytes >= need); }
// whether some of the pointers do not stand at an element
inline bool astray(size_t elem, std::initializer_list<const void*> ps) {
    uintptr_t bits = 0;
    for (const void* p : ps) bits |= reinterpret_cast<uintptr_t>(p);
    return (bits & (elem - 1)) != 0;
}

}  // namespace srigl
