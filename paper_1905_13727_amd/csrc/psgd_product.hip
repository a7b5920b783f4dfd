// Products of the linear layer on the matrix cores: C[i][j] = sum_l A(i, l) B(j, l).  x W^T has both operands along the
// contraction, dz W the second across it, dz^T x both.
//
// A workgroup owns a tile of BM x BN outputs and goes along the contraction in steps of 128 bytes a row (64 bf16, 32 fp32; with 64
// bytes, half of a cache line a request, the large tile reached 1050 TFLOP/s instead of 1420), two steps in LDS at a time:
// while one is read and multiplied, the next is loaded straight into LDS, sixteen bytes a lane.
// Such a load writes 64 consecutive chunks of sixteen bytes, so which chunk of the operand lies where is decided by
// which one a lane asks for; the places are permuted so that the reads of a wave meet no bank twice:
//   along    chunk c of row r lies at place c ^ (r & 7) of its eight;
//   across   row l of the contraction holds its chunks in the order c ^ f(l), f such that the four rows of a transposing read
//            (ds_read_b64_tr_b16: four rows of the contraction, sixteen of the output) lie in different banks.
// No conflict is counted along the contraction, nor across it in bf16 tiles of 128 and 256.  Across it two cases do meet banks twice: a bf16 tile of 64
// has eight chunks a row, too few for all of f (both operands across, 2048 cubed: 4.3e6 of 8.7e6 active LDS cycles), and fp32 rows are not permuted
// (1.7e7 of 4.2e7, of 8.1e7 that the units were busy, and the product takes 1 % longer than the one along / along, whose conflicts are 6.6e4).
// Operands that cannot be loaded that way go through registers instead: fp32 ones (their matrix instructions leave time enough,
// and a row may then begin at any element), bf16 ones whose rows do not begin on multiples of sixteen bytes, and fp32 weights
// rounded to bf16 on the way.
// The sums go through LDS once more, 32 rows a wave at a time: a lane then holds eight consecutive columns of a row, one
// store of sixteen bytes (bf16) and one call of the generator.
//
// The matrix instructions bound it: bf16, with bias, 4096 x 8192 x 2048 110 us and 4096 x 8192 x 4096 201 us, 1370 TFLOP/s; 8192 x 50304 x
// 2048 1365 us, 1240; across 4096 x 8192 x 2048, both gradients together, 217 us, 1270; fp32 4096 x 8192 x 2048 1020 us, 135.  On the
// largest tile they are busy four fifths of the time (SQ_VALU_MFMA_BUSY_CYCLES over SQ_BUSY_CU_CYCLES); most of the rest is waits at the step's
// barrier.  Matrix instructions of 32 x 32 x 16 in place of 16 x 16 x 32 lose (4096 x 8192 x 4096 204 -> 223 us), so do four waves of 128 x 128
// each (their sums and operands do not fit the registers) and workgroups that go on to a next tile (110 -> 113).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "psgd_epilogue.h"

namespace psgd {

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// ---- one operand of a tile ------------------------------------------------------------------------------------------

enum Source { kStraight, kBf16, kFp32 };   // straight to LDS; through registers, from bf16 or fp32 in memory

// ROWS: outputs of the tile in this operand's dimension; Z: bytes an element in LDS; THREADS of the workgroup
template <int ROWS, int Z, bool ALONG, Source SRC, int THREADS>
struct Operand {
    static_assert(Z == 2 || SRC == kFp32, "fp32 products read fp32");
    static constexpr int kElems = 16 / Z;                 // a chunk in LDS
    static constexpr int kSrc = SRC == kFp32 ? 4 : 2;     // bytes an element in memory
    static constexpr int kStep = 128 / Z;                 // contraction of a step
    static constexpr int kRowChunks = ROWS / kElems;      // across: chunks of a row of the contraction
    static constexpr int kBytes = ROWS * 128;
    static constexpr int kLoads = kBytes / 16 / THREADS;
    static constexpr int kWords = Z == 2 && SRC == kFp32 ? 2 : 1;   // registers of four words a chunk
    static_assert(kBytes % (16 * THREADS) == 0, "whole loads");

    static __device__ __forceinline__ int key(int l) { return Z == 2 ? ((l & 3) << 1) | (kRowChunks > 8 ? l & 8 : 0) : 0; }   // across
    // the row (along) or row of the contraction (across) and the chunk of it that this lane's i-th load brings
    static __device__ __forceinline__ void place(int i, int& line, int& chunk) {
        const int q = i * THREADS + threadIdx.x;
        if constexpr (ALONG) {
            line = q >> 3;
            chunk = (q & 7) ^ (line & 7);
        } else {
            line = q / kRowChunks;
            chunk = (q % kRowChunks) ^ key(line);
        }
    }
    // byte offsets of this lane's chunks from the operand's base for the first step.  Outputs past the end are clamped to the last
    // ones: what they give is not stored.
    static __device__ __forceinline__ void sources(unsigned (&off)[kLoads], int64_t ld, int64_t extent) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int line, c;
            place(i, line, c);
            if constexpr (ALONG) {
                const int row = line < extent ? line : (int)extent - 1;
                off[i] = (unsigned)((row * (int)ld + c * kElems) * kSrc);
            } else {
                const int many = (int)(extent < ROWS ? extent : ROWS), last = (many + kElems - 1) / kElems - 1;
                const int e = SRC == kBf16 ? (c * kElems < many - 8 ? c * kElems : many - 8) : (c < last ? c : last) * kElems;
                off[i] = (unsigned)((line * (int)ld + e) * kSrc);
            }
        }
    }
    // straight to LDS
    static __device__ __forceinline__ void load(const char* base, const unsigned (&off)[kLoads], lds_char* to) {
        const buf_rsrc r = make_rsrc(base, 0x7fffffff);
        lds_char* at = to + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave) * (kWave * 16);
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void*)(at + i * THREADS * 16), 16, (int)off[i], 0, 0, 0);
    }
    // To registers, and by store() to LDS.  `left`: elements of the contraction to go, those past the end are zero; `extent`: outputs
    // from the tile's first on, those past the end are never stored, but memory may end there.
    // bf16: a chunk that the row's end cuts (or that lies behind it) is read as the row's last eight elements and shifted into place by
    // store(), so that no lane reads past the end and none reads element by element; `tiny` (a row of fewer than eight): it does.
    // WHOLE: nothing of the step is cut off, and no row is tiny.
    template <bool WHOLE>
    static __device__ __forceinline__ void load(const char* base, const unsigned (&off)[kLoads], int64_t ld, int64_t extent, int64_t left,
                                                bool tiny, v4u (&held)[kLoads * kWords]) {
        if constexpr (SRC == kFp32) {   // what lies behind the end reads as zero
            const int64_t room = (ALONG ? (extent - 1) * ld + left : (left - 1) * ld + extent) * 4;
            const buf_rsrc r = make_rsrc(base, room < 0x7fffffff ? room : 0x7fffffff);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int line, c;
                place(i, line, c);
                const int at = !WHOLE && !ALONG && line >= left ? (int)kOutOfRange : (int)off[i];
#pragma unroll
                for (int h = 0; h < kWords; ++h) held[i * kWords + h] = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16 * h, 0, 0);
            }
        } else if (!WHOLE && tiny) {
            const int many = (int)(ALONG ? left : extent < ROWS ? extent : ROWS);
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int line, c;
                place(i, line, c);
                const int count = !ALONG && line >= left ? 0 : many - c * kElems;
                const int row = ALONG && line >= extent ? (int)extent - 1 : line;
                v4u t = v4u{0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e < count) t[e >> 1] |= (unsigned)reinterpret_cast<const bf16_t*>(base)[row * (int)ld + c * kElems + e] << (16 * (e & 1));
                held[i] = t;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kLoads; ++i) {
                int at = (int)off[i];
                if (!WHOLE && left < kStep) {
                    int line, c;
                    place(i, line, c);
                    if constexpr (ALONG) at += c * kElems < (int)left - 8 ? 0 : ((int)left - 8 - c * kElems) * 2;
                    else at -= line < left ? 0 : (line - (int)left + 1) * (int)ld * 2;
                }
                held[i] = *reinterpret_cast<const v4u_any*>(base + at);
            }
        }
    }
    template <bool WHOLE>
    static __device__ __forceinline__ void store(const v4u (&held)[kLoads * kWords], int64_t extent, int64_t left, bool tiny, lds_char* to) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            v4u t[kWords];
#pragma unroll
            for (int h = 0; h < kWords; ++h) t[h] = held[i * kWords + h];
            if constexpr (SRC == kFp32) {
                if (!WHOLE && ALONG && left < kStep) {
                    int line, c;
                    place(i, line, c);
#pragma unroll
                    for (int h = 0; h < kWords; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (c * kElems + 4 * h + e >= left) t[h][e] = 0;
                }
            } else if ((WHOLE || !tiny) && ((!ALONG && extent < ROWS) || (!WHOLE && left < kStep))) {
                int line, c;
                place(i, line, c);
                const int many = (int)(ALONG ? left : extent < ROWS ? extent : ROWS);
                int count = many - c * kElems;
                count = (!ALONG && line >= left) || count < 0 ? 0 : count > 8 ? 8 : count;
                const int words = (8 - count) >> 1;   // the last `count` of eight elements become the first
                v4u u = t[0];
                u = words & 2 ? v4u{u[2], u[3], 0, 0} : u;
                u = words & 1 ? v4u{u[1], u[2], u[3], 0} : u;
                if (count & 1) u = v4u{u[0] >> 16 | u[1] << 16, u[1] >> 16 | u[2] << 16, u[2] >> 16 | u[3] << 16, u[3] >> 16};
                t[0] = count == 0 ? v4u{0, 0, 0, 0} : u;
            }
            if constexpr (kWords == 2) {   // rounded to nearest even
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const v4f x = __builtin_bit_cast(v4f, t[h]);
                    t[0][2 * h] = pack_bf16x2(x.x, x.y);
                    t[0][2 * h + 1] = pack_bf16x2(x.z, x.w);
                }
            }
            *reinterpret_cast<__attribute__((address_space(3))) v4u*>(to + (i * THREADS + threadIdx.x) * 16) = t[0];
        }
    }
    // the last step, cut short: chunks past the end of the contraction, `left` elements on, are zero
    static __device__ __forceinline__ void load_cut(const char* base, const unsigned (&off)[kLoads], lds_char* to, int left) {
        const buf_rsrc r = make_rsrc(base, 0x7fffffff);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            int line, c;
            place(i, line, c);
            v4u t = v4u{0, 0, 0, 0};
            if ((ALONG ? c * kElems : line) < left) t = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off[i], 0, 0);
            *reinterpret_cast<__attribute__((address_space(3))) v4u*>(to + (i * THREADS + threadIdx.x) * 16) = t;
        }
    }
    static __device__ __forceinline__ int64_t step_bytes(int64_t ld) { return (ALONG ? 1 : ld) * kStep * kSrc; }

    // Fragment f of half h of a step: lane i of lane group g holds output first + 16 f + i.  bf16: elements 8 g .. 8 g + 7 of the
    // half's 32; fp32: 4 g .. 4 g + 3 of its 16
    static __device__ __forceinline__ auto frag(const lds_char* s, int first, int f, int h) {
        const int lane = threadIdx.x & 63, i = lane & 15, g = lane >> 4;
        if constexpr (ALONG) {
            typedef typename std::conditional<Z == 2, v8bf, v4f>::type Frag;
            const int row = first + 16 * f + i;
            return *reinterpret_cast<const __attribute__((address_space(3))) Frag*>(s + row * 128 + (((4 * h + g) ^ (row & 7)) << 4));
        } else if constexpr (Z == 2) {
            // the four rows l .. l + 3 of a lane group's eight, sixteen outputs each: lane i asks for row i / 4, outputs 4 (i % 4)
            // (first is a multiple of all the fragments' outputs, so that the fragment's number can go in by exclusive or)
            const int l = 32 * h + 8 * g + (i >> 2), m = first + 4 * (i & 3);
            const lds_char* p = s + l * (ROWS * Z) + ((((m * Z) >> 4) ^ key(l) ^ (2 * f)) << 4) + ((m * Z) & 15);
            typedef __attribute__((address_space(3))) v4s* lds_v4s;
            const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)p);
            const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s)(p + 4 * (ROWS * Z)));   // key(l + 4) = key(l)
            return __builtin_bit_cast(v8bf, (v8s)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            v4f t;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                t[e] = *reinterpret_cast<const __attribute__((address_space(3))) float*>(s + (16 * h + 4 * g + e) * (ROWS * Z) + (first + 16 * f + i) * 4);
            return t;
        }
    }
};

// ---- tiles ----------------------------------------------------------------------------------------------------------

// s_waitcnt: no load (to LDS too) in flight and every LDS access done
constexpr int kLandedAndRead = 0x0070;

// Orders a wave's LDS accesses before this point ahead of those behind it, where lanes read what other lanes wrote.  The hardware keeps a wave's
// LDS accesses in order, so this is no instruction; it keeps the compiler from moving one past another that it can tell apart lane by lane.
__device__ __forceinline__ void lanes_meet() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// The workgroups that run at the same time on one die (own L2) get neighbouring tiles: numbers are dealt to the eight dies in
// ranges, and a range goes along the rows of C in bands of eight tiles (four are as fast, sixteen take 2 to 7 % more).
__device__ __forceinline__ void tile_of(int number, int count, int tiles_m, int tiles_n, int& tm, int& tn) {
    const int each = count / 8, more = count % 8, die = number % 8;
    int t = die * each + (die < more ? die : more) + number / 8;
    constexpr int kBand = 8;
    const int wide = kBand * tiles_n;
    const int band = t / wide, first = band * kBand, high = tiles_m - first < kBand ? tiles_m - first : kBand;
    t -= band * wide;
    tn = t / high;
    tm = first + t - tn * high;
}

struct ProductArgs {
    const char *a, *b;
    int64_t a_ld, b_ld;
    void* c;
    int64_t c_ld, M, N, K;
    int tiles_m, tiles_n, steps_each, splits;
    float* partial;          // [split][M][N], with several splits of the contraction
    Epilogue ep;
};

template <bool BF, bool AA, bool BA, Source AS, Source BS, int WM, int WN, int MF, int NF>
struct Shape {   // WM x WN waves, each MF x NF fragments of 16 x 16
    static constexpr int BM = WM * MF * 16, BN = WN * NF * 16, T = WM * WN * kWave;
    static constexpr int Z = BF ? 2 : 4;
    typedef Operand<BM, Z, AA, AS, T> A;
    typedef Operand<BN, Z, BA, BS, T> B;
    typedef typename std::conditional<BF, v8bf, v4f>::type Frag;
    static constexpr int kStepBytes = A::kBytes + B::kBytes;
    static constexpr int kSums = 2 * kStepBytes;   // the steps' place, and the sums' behind them
    static constexpr int kLds = kSums + BN * 4 + 16;   // then the tile's bias in fp32 and the generator's words
    static constexpr int kPartBytes = 32 * NF * 64;   // 32 rows of a wave's sums
    static_assert(kSums >= WM * WN * kPartBytes && MF % 2 == 0 && (NF == 4 || NF == 2), "32 rows of sums a wave");
};

// The order of a stretch of instructions: its loads from memory one by one and then its LDS reads two by two, spread evenly between the products
template <int FETCHES, int READS, int PRODUCTS>
__device__ __forceinline__ void deal_out() {
    constexpr int kProduct = 8, kFetch = 0x20, kRead = 0x100, kGroups = FETCHES + READS / 2;   // the builtin's names for them
    static_assert(READS % 2 == 0, "two by two");
    auto deal = [](auto at, auto self) __attribute__((always_inline)) {
        constexpr int i = decltype(at)::value, some = (i + 1) * PRODUCTS / kGroups - i * PRODUCTS / kGroups;
        if constexpr (i < kGroups) {
            __builtin_amdgcn_sched_group_barrier(i < FETCHES ? kFetch : kRead, i < FETCHES ? 1 : 2, 0);
            if constexpr (some > 0) __builtin_amdgcn_sched_group_barrier(kProduct, some, 0);
            self(std::integral_constant<int, i + 1>(), self);
        }
    };
    deal(std::integral_constant<int, 0>(), deal);
}

// Tile and split number `block` of tiles_m * tiles_n * splits
template <bool BF, bool AA, bool BA, Source AS, Source BS, int WM, int WN, int MF, int NF>
__device__ __forceinline__ void product_tile(const ProductArgs& p, unsigned block, char* lds_raw) {
    const char *const a = p.a, *const b = p.b;
    const int64_t a_ld = p.a_ld, b_ld = p.b_ld, M = p.M, N = p.N, K = p.K;
    const int tiles_m = p.tiles_m, tiles_n = p.tiles_n;
    void* const c = p.c;
    int64_t c_ld = p.c_ld;
    float* const partial = p.partial;
    const Epilogue& ep = p.ep;
    typedef Shape<BF, AA, BA, AS, BS, WM, WN, MF, NF> S;
    typedef typename S::A A;
    typedef typename S::B B;
    typedef typename S::Frag Frag;
    lds_char* const lds = (lds_char*)lds_raw;
    int tm, tn;
    const int tiles = tiles_m * tiles_n;
    const int64_t split = block / (unsigned)tiles;
    tile_of((int)(block - (unsigned)split * tiles), tiles, tiles_m, tiles_n, tm, tn);
    const int64_t i0 = (int64_t)tm * S::BM, j0 = (int64_t)tn * S::BN;
    const int64_t all = (K + A::kStep - 1) / A::kStep, s0 = split * p.steps_each;
    const int steps = (int)(s0 + p.steps_each < all ? p.steps_each : all - s0);
    const int cut = s0 + steps == all ? (int)(K % A::kStep) : 0;   // what the last step holds, if it is cut short
    const int whole = steps - (cut ? 1 : 0);

    unsigned a_off[A::kLoads], b_off[B::kLoads];
    A::sources(a_off, a_ld, M - i0);
    B::sources(b_off, b_ld, N - j0);
    const char* ap = a + (AA ? i0 * a_ld : i0) * A::kSrc + s0 * A::step_bytes(a_ld);
    const char* bp = b + (BA ? j0 * b_ld : j0) * B::kSrc + s0 * B::step_bytes(b_ld);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), wm = wave / WN, wn = wave % WN;

    v4f acc[MF][NF];
#pragma unroll
    for (int m = 0; m < MF; ++m)
#pragma unroll
        for (int n = 0; n < NF; ++n) acc[m][n] = v4f{0.f, 0.f, 0.f, 0.f};

    // Step s: straight to LDS at once, through registers by settle() one barrier later.  `left` of the contraction from step s on,
    // for the loads through registers.
    v4u a_held[A::kLoads * A::kWords], b_held[B::kLoads * B::kWords];
    auto fetch = [&](auto all, int s, int buf) __attribute__((always_inline)) {
        constexpr bool W = decltype(all)::value;
        lds_char* to = lds + buf * S::kStepBytes;
        const int64_t left = K - (s0 + s) * A::kStep;
        if constexpr (AS == kStraight) {
            if (W || s < whole) A::load(ap, a_off, to);
            else A::load_cut(ap, a_off, to, cut);
        } else {
            A::template load<W>(ap, a_off, a_ld, M - i0, left, (AA ? K : M) < 8, a_held);
        }
        if constexpr (BS == kStraight) {
            if (W || s < whole) B::load(bp, b_off, to + A::kBytes);
            else B::load_cut(bp, b_off, to + A::kBytes, cut);
        } else {
            B::template load<W>(bp, b_off, b_ld, N - j0, left, (BA ? K : N) < 8, b_held);
        }
        ap += A::step_bytes(a_ld);
        bp += B::step_bytes(b_ld);
    };
    auto settle = [&](auto all, int s, int buf) __attribute__((always_inline)) {
        constexpr bool W = decltype(all)::value;
        lds_char* to = lds + buf * S::kStepBytes;
        const int64_t left = K - (s0 + s) * A::kStep;
        if constexpr (AS != kStraight) A::template store<W>(a_held, M - i0, left, (AA ? K : M) < 8, to);
        if constexpr (BS != kStraight) B::template store<W>(b_held, N - j0, left, (BA ? K : N) < 8, to + A::kBytes);
        __builtin_amdgcn_s_waitcnt(kLandedAndRead);
    };
    auto read = [&](int buf, int h, Frag (&x)[MF], Frag (&y)[NF]) __attribute__((always_inline)) {
        const lds_char *as = lds + buf * S::kStepBytes, *bs = as + A::kBytes;
#pragma unroll
        for (int n = 0; n < NF; ++n) y[n] = B::frag(bs, wn * NF * 16, n, h);
#pragma unroll
        for (int m = 0; m < MF; ++m) x[m] = A::frag(as, wm * MF * 16, m, h);
    };
    auto multiply = [&](const Frag (&x)[MF], const Frag (&y)[NF]) __attribute__((always_inline)) {
        if constexpr (BF) {
#pragma unroll
            for (int m = 0; m < MF; ++m)
#pragma unroll
                for (int n = 0; n < NF; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y[n], x[m], acc[m][n], 0, 0, 0);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int m = 0; m < MF; ++m)
#pragma unroll
                    for (int n = 0; n < NF; ++n) acc[m][n] = __builtin_amdgcn_mfma_f32_16x16x4f32(y[n][e], x[m][e], acc[m][n], 0, 0, 0);
        }
    };
    // The fragments of one half step are read while the other half's are multiplied, across the steps too: the barrier that
    // hands a buffer over stands in the middle of a step, where a half's products are ready to issue on both sides of it.
    // The bias and the generator's words are asked for ahead of the first step and wait in LDS: read behind the last one, they would make the
    // epilogue wait for memory, and each of its rows for the stores of the rows before.
    __attribute__((address_space(3))) float* const bias_at = (__attribute__((address_space(3))) float*)(lds + S::kSums);
    __attribute__((address_space(3))) v4u* const draw_at = (__attribute__((address_space(3))) v4u*)(bias_at + S::BN);
    float bias_one = 0.f;
    v4u draw_words{0, 0, 0, 0};
    if (!partial) {
        if ((int)threadIdx.x < S::BN && ep.bias && j0 + threadIdx.x < N) bias_one = ld_any(ep.bias, j0 + threadIdx.x, ep.bias_bf);
        if (threadIdx.x == 0 && ep.drop.below) draw_words = words_ahead(ep.drop.rng, ep.drop.offset);
    }
    auto ends_ahead = [&]() __attribute__((always_inline)) {
        if ((int)threadIdx.x < S::BN) bias_at[threadIdx.x] = bias_one;
        if (threadIdx.x == 0) *draw_at = draw_words;
    };
    if (steps > 0) {
        Frag x0[MF], y0[NF], x1[MF], y1[NF];
        const std::true_type all;
        const std::false_type some;
        fetch(some, 0, 0);
        ends_ahead();
        settle(some, 0, 0);
        __syncthreads();
        if (steps > 1) fetch(some, 1, 1);
        read(0, 0, x0, y0);
        int buf = 0, s = 0;
        // Steps with two whole ones behind them have no branches, so that their loads and reads of LDS can stand between the products: a wave goes
        // on multiplying while it asks for what comes next.  4096 x 8192 x 4096 along / along 228 us with the branches, 216 without, 202 dealt
        // out in the order above; 8192 x 2048 x 4096 across / across, with twice the reads, 129, 113 and 116, so there the order is left to the
        // compiler, as it is where loads go through registers.
        constexpr bool kDeal = BF && AA && BA && AS == kStraight && BS == kStraight;
        const int64_t least = std::min(AA ? K : M, BA ? K : N);
        const int full = AS == kStraight || !BF || least >= 8 ? whole : 0;
        for (; s + 2 < full; ++s, buf ^= 1) {
            read(buf, 1, x1, y1);
            multiply(x0, y0);
            if constexpr (kDeal) deal_out<0, MF + NF, MF * NF>();
            __builtin_amdgcn_sched_barrier(0);
            settle(all, s + 1, buf ^ 1);
            __syncthreads();
            fetch(all, s + 2, buf);
            read(buf ^ 1, 0, x0, y0);
            multiply(x1, y1);
            if constexpr (kDeal) deal_out<A::kLoads + B::kLoads, MF + NF, MF * NF>();
            __builtin_amdgcn_sched_barrier(0);
        }
        for (; s < steps; ++s, buf ^= 1) {
            read(buf, 1, x1, y1);
            __builtin_amdgcn_sched_barrier(0);
            multiply(x0, y0);
            __builtin_amdgcn_sched_barrier(0);
            if (s + 1 < steps) {
                settle(some, s + 1, buf ^ 1);   // step s + 1 has landed, this step's fragments are in registers
                __syncthreads();
                if (s + 2 < steps) fetch(some, s + 2, buf);
                read(buf ^ 1, 0, x0, y0);
            }
            __builtin_amdgcn_sched_barrier(0);
            multiply(x1, y1);
        }
    } else {
        ends_ahead();
    }

    // 32 rows of a wave's sums at a time: row r holds its quads in the order q ^ (r & (4 NF - 1))
    __syncthreads();
    constexpr int kQuads = 4 * NF, kAcross = 2 * NF, kRowsAtOnce = 64 / kAcross;   // quads of a row, lanes along one, rows of all lanes
    const int lane = threadIdx.x & 63, g = lane >> 4, lr = lane / kAcross, lc = lane % kAcross;
    lds_char* const mine = lds + wave * S::kPartBytes;
    const int64_t j = j0 + wn * NF * 16 + 8 * lc;
    Draw d{};
    float bias[8] = {};
    if (!partial) {
        const v4u words = *draw_at;
        d = make_draw(words);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const v4f t = *reinterpret_cast<const __attribute__((address_space(3))) v4f*>(bias_at + wn * NF * 16 + 8 * lc + 4 * h);
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[4 * h + e] = t[e];
        }
    }
    auto pick_up = [&](int r, float (&sum)[8]) __attribute__((always_inline)) {   // eight columns of row r
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const v4f t = *reinterpret_cast<const __attribute__((address_space(3))) v4f*>(mine + (r * kQuads + ((2 * lc + h) ^ (r & (kQuads - 1)))) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[4 * h + e] = t[e];
        }
    };
    const int count = N - j < 8 ? (int)(N - j) : 8;
    const int64_t first = i0 + wm * MF * 16 + lr;
    const int rows = (int)(M - first < MF * 16 ? M - first : MF * 16);   // this lane's rows of the wave's, from `first` on
    int64_t c_at = first * c_ld + j, pre_at = first * ep.pre_ld + j, residual_at = first * ep.residual_ld + j, i = first;
    if (partial) c_at = (split * M + first) * N + j, c_ld = N;
    // A tile that lies inside C and has neither dropout nor a residual to go through: no choice is left to a row, and a row's place is the
    // lane's fixed offset behind an address that is the same for all.  4096 x 8192 x 2048 bf16 116 us without this, 111 with it.
    constexpr int kOut = BF ? 2 : 4;
    const bool plain = !partial && !ep.drop.below && !ep.residual && M - i0 >= S::BM && N - j0 >= S::BN;
    const int64_t row = i0 + wm * MF * 16, col = j0 + wn * NF * 16;
    char* at = static_cast<char*>(c) + (row * c_ld + col) * kOut;
    char* pre = ep.pre ? static_cast<char*>(ep.pre) + (row * ep.pre_ld + col) * kOut : nullptr;
    const unsigned c_lane = (unsigned)(lr * (int)c_ld + 8 * lc) * kOut, pre_lane = (unsigned)(lr * (int)ep.pre_ld + 8 * lc) * kOut;
#pragma unroll 1
    for (int part = 0; part < MF / 2; ++part) {
        lanes_meet();   // the part before has been picked up
#pragma unroll
        for (int q = 0; q < MF / 2; ++q)
            if (q == part)
#pragma unroll
                for (int m = 0; m < 2; ++m)
#pragma unroll
                    for (int n = 0; n < NF; ++n) {
                        const int r = 16 * m + (lane & 15);
                        *reinterpret_cast<__attribute__((address_space(3))) v4f*>(mine + (r * kQuads + ((4 * n + g) ^ (r & (kQuads - 1)))) * 16) = acc[2 * q + m][n];
                    }
        lanes_meet();   // this part's sums are there, those of other lanes too
        if (plain) {
            auto finish = [&](auto kind) __attribute__((always_inline)) {
#pragma unroll
                for (int r0 = 0; r0 < 32; r0 += kRowsAtOnce) {
                    float sum[8];
                    pick_up(r0 + lr, sum);
                    finish_oct<BF, decltype(kind)::value>(ep.scale, bias, at + c_lane, pre ? pre + pre_lane : nullptr, sum);
                    at += kRowsAtOnce * c_ld * kOut;
                    if (pre) pre += kRowsAtOnce * ep.pre_ld * kOut;
                }
            };
            switch (ep.act) {
                case PSGD_ACT_RELU: finish(std::integral_constant<int, PSGD_ACT_RELU>()); break;
                case PSGD_ACT_GELU: finish(std::integral_constant<int, PSGD_ACT_GELU>()); break;
                case PSGD_ACT_GELU_TANH: finish(std::integral_constant<int, PSGD_ACT_GELU_TANH>()); break;
                case PSGD_ACT_SILU: finish(std::integral_constant<int, PSGD_ACT_SILU>()); break;
                default: finish(std::integral_constant<int, PSGD_ACT_IDENTITY>()); break;
            }
            continue;
        }
#pragma unroll 2
        for (int r0 = 0; r0 < 32; r0 += kRowsAtOnce) {
            if (32 * part + r0 < rows && count > 0) {
                float sum[8];
                RawOct residual;
                if (!partial) residual = residual_ahead<BF>(ep, residual_at, count);
                pick_up(r0 + lr, sum);
                if (partial) st_oct<false>(partial, c_at, count, sum);
                else finish_oct<BF>(ep, d, c, c_at, pre_at, i, j, count, sum, bias, residual);
            }
            i += kRowsAtOnce;
            c_at += kRowsAtOnce * c_ld;
            pre_at += kRowsAtOnce * ep.pre_ld;
            residual_at += kRowsAtOnce * ep.residual_ld;
        }
    }
}

template <bool BF, bool AA, bool BA, Source AS, Source BS, int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(WM* WN* kWave, 2) void k_product(ProductArgs p) {
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    product_tile<BF, AA, BA, AS, BS, WM, WN, MF, NF>(p, blockIdx.x, lds_raw);
}

// A product p and, in front of it in the same launch, the rows q beyond its last full tile in tiles of 64 rows, divided along the contraction so that
// each unit has one more short tile.  bf16, in two launches and so: 4099 x 8192 x 2048 124 and 115 us, 4099 x 2048 x 2048 40.3 and 37.7; with a long
// contraction it gains nothing, 4099 x 2048 x 8192 131 and 132, with dropout and residual 139 and 139 (188 as one product).
template <bool BA, int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(WM* WN* kWave, 2) void k_product_and_rest(ProductArgs p, ProductArgs q, unsigned first) {
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    if (blockIdx.x < first) product_tile<true, true, BA, kStraight, kStraight, WM, WN, 2, 2>(q, blockIdx.x, lds_raw);
    else product_tile<true, true, BA, kStraight, kStraight, WM, WN, MF, NF>(p, blockIdx.x - first, lds_raw);
}

// The columns' sums over one block of rows and 256 columns; 256 lanes, each eight columns of every eighth row
template <bool BF>
__device__ __forceinline__ void sum_block(const ColumnSums& s, unsigned block, char* lds_raw) {
    float(*part)[264] = reinterpret_cast<float(*)[264]>(lds_raw);
    const int lane_c = threadIdx.x & 31, lane_t = threadIdx.x >> 5;
    const int64_t wide = (s.n + 255) / 256, bt = block / wide, bc = block - bt * wide, c0 = bc * 256 + 8 * lane_c;
    const int64_t t0 = bt * kSumRows + lane_t;
    const int count = s.n - c0 < 8 ? (int)(s.n - c0) : 8;
    float v[8] = {};
    if (count > 0)
#pragma unroll
        for (int r = 0; r < kSumRows; r += 8)
            if (t0 + r < s.T) {
                float x[8];
                ld_oct<BF>(s.dy, (t0 + r) * s.dy_ld + c0, count, x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += x[e];
            }
#pragma unroll
    for (int e = 0; e < 8; ++e) part[lane_t][8 * lane_c + e] = v[e];
    __syncthreads();
    const int64_t col = bc * 256 + threadIdx.x;
    if (col >= s.n) return;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += part[i][threadIdx.x];
    s.sums[bt * s.n + col] = sum;
}

template <bool BF>
__global__ __launch_bounds__(256) void k_sum_blocks(ColumnSums s) {
    __shared__ __attribute__((aligned(16))) char lds_raw[8 * 264 * 4];
    sum_block<BF>(s, blockIdx.x, lds_raw);
}

// The input gradient (`first` workgroups) and the weight gradient (up to `second`) of a layer in one launch, and behind them the columns'
// sums: none waits for another, and small ones fill the chip together
template <bool BF, Source AS, Source BS, Source BS2, int WM, int WN, int MF, int NF>
__global__ __launch_bounds__(WM* WN* kWave, 2) void k_product_two(ProductArgs p, ProductArgs q, ColumnSums sums, unsigned first,
                                                                  unsigned second) {
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    static_assert(WM * WN * kWave == 256 && Shape<BF, true, false, AS, BS, WM, WN, MF, NF>::kLds >= 8 * 264 * 4, "sum_block");
    if (blockIdx.x < first) product_tile<BF, true, false, AS, BS, WM, WN, MF, NF>(p, blockIdx.x, lds_raw);
    else if (blockIdx.x < second) product_tile<BF, false, false, AS, BS2, WM, WN, MF, NF>(q, blockIdx.x - first, lds_raw);
    else sum_block<BF>(sums, blockIdx.x - second, lds_raw);
}

// The same in the largest tiles, for large products: `first` workgroups of the one whose tiles take longer, so that the other one's fill
// the units that they leave
__global__ __launch_bounds__(512, 2) void k_product_two_large(ProductArgs p, ProductArgs q, unsigned first, int p_first) {
    extern __shared__ __attribute__((aligned(16))) char lds_raw[];
    const bool head = blockIdx.x < first;
    const unsigned block = head ? blockIdx.x : blockIdx.x - first;
    if (head == (p_first != 0)) product_tile<true, true, false, kStraight, kStraight, 2, 4, 8, 4>(p, block, lds_raw);
    else product_tile<true, false, false, kStraight, kStraight, 2, 4, 8, 4>(q, block, lds_raw);
}

// The sum over the splits, in order, and the epilogue.  One lane: eight columns.  Latency bounds it where it is used, 4 to 6 us a launch, of
// which 0.5 are memory's for 19 x 2048 outputs of 16 splits; workgroups of one wave put that on as many units as there are.
template <bool BF>
__device__ __forceinline__ void join_octs(const ProductArgs& p, unsigned block) {
    const unsigned per_row = (unsigned)((p.N + 7) / 8), at = block * kWave + threadIdx.x;   // the sums of all splits are below 2^24
    const DrawWords words = p.ep.drop.below ? words_ahead(p.ep.drop.rng, p.ep.drop.offset) : DrawWords{0, 0, 0, 0};
    const unsigned row = at / per_row;
    if (row >= p.M) return;
    const int64_t i = row, j = 8 * (int64_t)(at - row * per_row);
    const int count = p.N - j < 8 ? (int)(p.N - j) : 8;
    float v[8] = {}, bias[8];
    const RawOct raw = bias_ahead(p.ep, j, p.N), residual = residual_ahead<BF>(p.ep, i * p.ep.residual_ld + j, count);
    for (int s = 0; s < p.splits; s += 8) {   // eight splits' loads in flight, added in order
        float x[8][8];
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (s + q < p.splits) ld_oct<false>(p.partial, ((s + q) * p.M + i) * p.N + j, count, x[q]);
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (s + q < p.splits)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] += x[q][e];
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) bias[e] = widened(raw, e, p.ep.bias_bf);
    finish_oct<BF>(p.ep, make_draw(words), p.c, i * p.c_ld + j, i * p.ep.pre_ld + j, i, j, count, v, bias, residual);
}

// Sixteen columns of the blocks' column sums: four lanes a column take every fourth block, eight in flight, and are added in order
template <bool BF>
__device__ __forceinline__ void column_sums(const ColumnSums& s, int64_t block) {
    __shared__ float part[4][16];
    const int lc = threadIdx.x & 15, lg = threadIdx.x >> 4;
    const int64_t col = block * 16 + lc, blocks = (s.T + kSumRows - 1) / kSumRows;
    float v = 0.f;
    if (col < s.n)
        for (int64_t i = lg; i < blocks; i += 32) {
            float x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) x[q] = i + 4 * q < blocks ? s.sums[(i + 4 * q) * s.n + col] : 0.f;
#pragma unroll
            for (int q = 0; q < 8; ++q) v += x[q];
        }
    part[lg][lc] = v;
    __syncthreads();
    if (lg || col >= s.n) return;
    v = ((part[0][lc] + part[1][lc]) + (part[2][lc] + part[3][lc])) * s.scale;
    if (s.accumulate) v += ld_any(s.db, col, BF);
    st_any(s.db, col, v, BF);
}

// What is left to add up behind the products of one call: the splits of up to two, and the bias gradient
template <bool BF>
__global__ __launch_bounds__(kWave) void k_join(ProductArgs p, int64_t p_blocks, ProductArgs q, int64_t q_blocks, ColumnSums s) {
    if (blockIdx.x < p_blocks) join_octs<BF>(p, blockIdx.x);
    else if (blockIdx.x < p_blocks + q_blocks) join_octs<BF>(q, blockIdx.x - p_blocks);
    else column_sums<BF>(s, blockIdx.x - p_blocks - q_blocks);
}

namespace {

ProductArgs args_of(const ProductCall& p, const Choice& ch) {
    return ProductArgs{static_cast<const char*>(p.a), static_cast<const char*>(p.b), p.a_ld, p.b_ld, p.c, p.c_ld, p.M, p.N, p.K, (int)ch.tiles_m,
                       (int)ch.tiles_n, (int)ch.steps_each, (int)ch.splits, ch.splits > 1 ? p.partial : nullptr, epilogue_of(p.ep)};
}

// More than 64 KB of LDS has to be asked for
template <typename Kernel>
hipError_t with_lds(Kernel k, int bytes) {
    return bytes > 65536 ? hipFuncSetAttribute(reinterpret_cast<const void*>(k), hipFuncAttributeMaxDynamicSharedMemorySize, bytes) : hipSuccess;
}

template <bool BF, bool AA, bool BA, Source AS, Source BS, int WM, int WN, int MF, int NF>
hipError_t start(const ProductArgs& p, hipStream_t stream) {
    typedef Shape<BF, AA, BA, AS, BS, WM, WN, MF, NF> S;
    auto k = k_product<BF, AA, BA, AS, BS, WM, WN, MF, NF>;
    const hipError_t e = with_lds(k, S::kLds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(k, dim3((unsigned)(p.tiles_m * p.tiles_n * p.splits)), dim3(S::T), S::kLds, stream, p);
    return hipGetLastError();
}

template <bool BF, Source AS, Source BS>
hipError_t start_by_shape(const ProductCall& p, const Choice& ch) {
    const ProductArgs d = args_of(p, ch);
    auto by_side = [&](auto aa, auto ba) {
        constexpr bool A = decltype(aa)::value, B = decltype(ba)::value;
        if constexpr (BF && AS == kStraight)
            if (ch.kind == 0) return start<BF, A, B, AS, BS, 2, 4, 8, 4>(d, p.stream);
        return ch.kind == 1 ? start<BF, A, B, AS, BS, 2, 2, 4, 4>(d, p.stream) : start<BF, A, B, AS, BS, 2, 2, 2, 2>(d, p.stream);
    };
    if (p.a_along) return p.b_along ? by_side(std::true_type(), std::true_type()) : by_side(std::true_type(), std::false_type());
    if constexpr (BF && BS == kFp32) return hipErrorInvalidValue;   // the weight gradient reads no weights
    else return by_side(std::false_type(), std::false_type());
}

// Workgroups of the columns' sums that are still to be computed
int64_t sum_blocks(const ColumnSums* s) { return s && s->dy ? (s->n + 255) / 256 * ((s->T + kSumRows - 1) / kSumRows) : 0; }

template <bool BF, Source AS, Source BS, Source BS2>
hipError_t start_two(const ProductArgs& p, const ProductArgs& q, const ColumnSums* sums, int kind, hipStream_t stream) {
    auto go = [&](auto k, auto shape) {
        typedef decltype(shape) S;
        const unsigned first = (unsigned)(p.tiles_m * p.tiles_n * p.splits), second = first + (unsigned)(q.tiles_m * q.tiles_n * q.splits);
        const hipError_t e = with_lds(k, S::kLds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(k, dim3(second + (unsigned)sum_blocks(sums)), dim3(S::T), S::kLds, stream, p, q, sums ? *sums : ColumnSums{}, first, second);
        return hipGetLastError();
    };
    return kind == 1 ? go(k_product_two<BF, AS, BS, BS2, 2, 2, 4, 4>, Shape<BF, true, false, AS, BS, 2, 2, 4, 4>())
                     : go(k_product_two<BF, AS, BS, BS2, 2, 2, 2, 2>, Shape<BF, true, false, AS, BS, 2, 2, 2, 2>());
}

Way way_of(const ProductCall& p) { return way_by(p.bf16, p.a_ready, p.b_ready && !p.b_fp32, p.a_along && p.b_along); }
int64_t join_blocks(const ProductArgs& p) { return p.partial ? (p.M * ((p.N + 7) / 8) + kWave - 1) / kWave : 0; }

psgd_status join(bool bf16, const ProductArgs& p, const ProductArgs& q, const ColumnSums* sums, hipStream_t stream, std::string* what) {
    const int64_t pb = join_blocks(p), qb = join_blocks(q), sb = sums ? (sums->n + 15) / 16 : 0;
    if (pb + qb + sb == 0) return PSGD_OK;
    auto k = bf16 ? k_join<true> : k_join<false>;
    hipLaunchKernelGGL(k, dim3((unsigned)(pb + qb + sb)), dim3(kWave), 0, stream, p, pb, q, qb, sums ? *sums : ColumnSums{});
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PSGD_OK;
    *what = std::string("launch k_join: ") + hipGetErrorString(e);
    return PSGD_EHIP;
}

// The columns' sums in a launch of their own, if they are still to be computed
psgd_status sum_blocks_alone(bool bf16, const ColumnSums* sums, hipStream_t stream, std::string* what) {
    const int64_t blocks = sum_blocks(sums);
    if (!blocks) return PSGD_OK;
    auto k = bf16 ? k_sum_blocks<true> : k_sum_blocks<false>;
    hipLaunchKernelGGL(k, dim3((unsigned)blocks), dim3(256), 0, stream, *sums);
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return PSGD_OK;
    *what = std::string("launch k_sum_blocks: ") + hipGetErrorString(e);
    return PSGD_EHIP;
}

psgd_status product_failed(hipError_t e, std::string* what) {
    if (e == hipSuccess) return PSGD_OK;
    *what = std::string("launch k_product: ") + hipGetErrorString(e);
    return PSGD_EHIP;
}

}  // namespace

int64_t product_partial_bytes(bool bf16, int64_t M, int64_t N, int64_t K) {
    const int64_t splits = std::min<int64_t>(kMostSplits, (K + (bf16 ? 63 : 31)) / (bf16 ? 64 : 32) / kLeastSteps);
    return splits > 1 ? std::min(splits * M * N * 4, kMostPartial) : 0;
}

namespace {

// The rows q beyond the last full tile of p, in one launch with it
psgd_status launch_with_rest(const ProductCall& p, const ProductCall& q, const ProductRoute& route, std::string* what) {
    typedef Shape<true, true, true, kStraight, kStraight, 2, 4, 8, 4> Large;
    typedef Shape<true, true, true, kStraight, kStraight, 2, 2, 4, 4> Small;
    const ProductArgs a = args_of(p, route.main), b = args_of(q, route.rest);
    const unsigned first = (unsigned)(b.tiles_m * b.tiles_n * b.splits), all = first + (unsigned)(a.tiles_m * a.tiles_n);
    auto go = [&](auto k, int lds, int threads) {
        const hipError_t e = with_lds(k, lds);
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL(k, dim3(all), dim3(threads), lds, p.stream, a, b, first);
        return hipGetLastError();
    };
    const hipError_t e = route.main.kind == 0 ? go(p.b_along ? k_product_and_rest<true, 2, 4, 8, 4> : k_product_and_rest<false, 2, 4, 8, 4>, Large::kLds, Large::T)
                                              : go(p.b_along ? k_product_and_rest<true, 2, 2, 4, 4> : k_product_and_rest<false, 2, 2, 4, 4>, Small::kLds, Small::T);
    const psgd_status st = product_failed(e, what);
    return st != PSGD_OK ? st : join(true, b, ProductArgs{}, nullptr, p.stream, what);
}

}  // namespace

psgd_status launch_product(const ProductCall& p, std::string* what) {
    const Way way = way_of(p);
    const ProductRoute route = product_route(way, p.a_along, p.M, p.N, p.K);
    const Choice& ch = route.whole;
    if (route.over) {
        const bool rows = route.rows;
        const int64_t z = p.bf16 ? 2 : 4, zb = p.bf16 && !p.b_fp32 ? 2 : 4, zp = p.ep.bias_bf ? 2 : 4;
        ProductCall main = p, q = p;
        (rows ? main.M : main.N) -= route.over;
        const int64_t row = rows ? main.M : 0, col = rows ? 0 : main.N;
        (rows ? q.M : q.N) = route.over;
        auto moved = [&](const void* at, int64_t ld, int64_t size) { return at ? static_cast<const char*>(at) + (row * ld + col) * size : nullptr; };
        q.a = static_cast<const char*>(p.a) + (p.a_along ? row * p.a_ld : row) * z;
        q.b = static_cast<const char*>(p.b) + (p.b_along ? col * p.b_ld : col) * zb;
        q.c = const_cast<char*>(moved(p.c, p.c_ld, z));
        q.ep.pre = const_cast<char*>(moved(p.ep.pre, p.ep.pre_ld, z));
        q.ep.residual = moved(p.ep.residual, p.ep.residual_ld, z);
        if (p.ep.bias) q.ep.bias = static_cast<const char*>(p.ep.bias) + col * zp;
        q.ep.row0 = p.ep.row0 + row;
        q.ep.col0 = p.ep.col0 + col;
        if (route.one_launch) return launch_with_rest(main, q, route, what);
        const psgd_status st = launch_product(main, what);
        if (st != PSGD_OK) return st;
        return launch_product(q, what);
    }
    const psgd_status st = product_failed(!p.bf16 ? start_by_shape<false, kFp32, kFp32>(p, ch) : way >= kStraightAcross ? start_by_shape<true, kStraight, kStraight>(p, ch)
                                          : p.b_fp32 ? start_by_shape<true, kBf16, kFp32>(p, ch) : start_by_shape<true, kBf16, kBf16>(p, ch), what);
    return st != PSGD_OK ? st : join(p.bf16, args_of(p, ch), ProductArgs{}, nullptr, p.stream, what);
}

psgd_status launch_backward_products(bool bf16, const ProductCall* x, const ProductCall* w, const ColumnSums* sums, hipStream_t stream,
                                     std::string* what) {
    if (x && w) {
        const Extent ex{way_of(*x), x->M, x->N, x->K}, ew{way_of(*w), w->M, w->N, w->K};
        const BackwardRoute route = backward_route(ex, ew, sum_blocks(sums));
        const ProductArgs p = args_of(*x, route.x), q = args_of(*w, route.w);
        if (route.kind == BackwardRoute::kLarge) {
            if (const psgd_status st = sum_blocks_alone(bf16, sums, stream, what); st != PSGD_OK) return st;
            typedef Shape<true, true, false, kStraight, kStraight, 2, 4, 8, 4> S;
            const int64_t px = p.tiles_m * p.tiles_n, pw = q.tiles_m * q.tiles_n;
            hipError_t e = with_lds(k_product_two_large, S::kLds);
            if (e == hipSuccess) {
                hipLaunchKernelGGL(k_product_two_large, dim3((unsigned)(px + pw)), dim3(S::T), S::kLds, stream, p, q, (unsigned)(route.x_first ? px : pw), (int)route.x_first);
                e = hipGetLastError();
            }
            const psgd_status st = product_failed(e, what);
            return st != PSGD_OK || !sums ? st : join(bf16, ProductArgs{}, ProductArgs{}, sums, stream, what);
        }
        if (route.kind == BackwardRoute::kTogether) {
            const int kind = route.x.kind;
            const hipError_t e = !bf16 ? start_two<false, kFp32, kFp32, kFp32>(p, q, sums, kind, stream)
                                 : ex.way >= kStraightAcross && ew.way >= kStraightAcross ? start_two<true, kStraight, kStraight, kStraight>(p, q, sums, kind, stream)
                                 : x->b_fp32 ? start_two<true, kBf16, kFp32, kBf16>(p, q, sums, kind, stream)
                                             : start_two<true, kBf16, kBf16, kBf16>(p, q, sums, kind, stream);
            const psgd_status st = product_failed(e, what);
            return st != PSGD_OK ? st : join(bf16, p, q, sums, stream, what);
        }
    }
    if (const psgd_status st = sum_blocks_alone(bf16, sums, stream, what); st != PSGD_OK) return st;
    for (const ProductCall* p : {x, w})
        if (p) {
            const psgd_status st = launch_product(*p, what);
            if (st != PSGD_OK) return st;
        }
    return sums ? join(bf16, ProductArgs{}, ProductArgs{}, sums, stream, what) : PSGD_OK;
}

}  // namespace psgd
