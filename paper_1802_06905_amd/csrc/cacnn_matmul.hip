// Matrix products of the feed-forward operators for gfx950: Out[m][n] = sum over k of Q(m, k) P(n, k), in bf16, fp32 and 8-bit floats with a
// scale for each block of 128, as they are or two at a time with the activation and the product of the gated projection behind them.
//
// Out's rows m are tokens (or, for a weight's gradient, the weight's rows), its columns n channels or features.  An MFMA takes 32 columns
// as its first operand and 32 rows as its second, so a lane ends up with one row m and runs of four adjacent columns, which
// leave in one store each, and the scale of a row in 8 bits is one number per lane.
//
// A workgroup owns BM x BN of Out and walks the contraction in slabs of 128 bytes a row (bf16 on 256 x 256: 64), two or four of them in LDS or on their way.
//   contraction contiguous ([row][k]): LDS keeps rows of a slab's length; the 16-byte chunk c of row r lies at c ^ ((r >> 1) & 7) (64 bytes: c ^ ((r >> 2) & 3)), so
//     that the lanes of an LDS access, adjacent rows at the same chunk, spread over all banks (two, or four, rows are as wide as these).  A lane's chunk holds the 8 (bf16), 4 (fp32) or 16 (8 bits)
//     contraction indices that it feeds to the matrix instructions; which index goes to which half of a wave does not matter, because
//     both operands use the same assignment.
//   contraction strided ([k][row]): LDS keeps the rows of k as they lie in memory, in blocks of 64 bytes (bf16, read by the
//     transposing loads) or 128 (fp32, read word by word) that change places with k, for the same reason.
// Counted on tiles of 256 x 256, bf16 (4096, 4096, 4096), gated and both gradients, and 8 bits (8192, 8192, 4096), and on fp32's of 128 x 128: bank conflicts
// are 1 or 2 % of LDS's busy cycles, which are 21 to 25 % of all (fp32 7 to 11 %).
//
// What bounds large products is the chip's power and what is left between the matrix instructions: those calls keep the matrix pipes busy for 59 % (gated), 53 % (its
// gradients) and 56 % (8 bits) of the cycles at 1.83 to 1.96 GHz, fp32 for 76 to 79 %; an earlier state of the bf16 kernel took 985 us for (8192, 4096, 8192) with
// random data and 786 with zeros.  Measured (in brackets a library product of 8192 x 8192 x 8192 in the same process, its right operand transposed, as here):
//     8 bits (8192, 8192, 4096)                       273 us one after another with other calls between, 252 alone, 2010 to 2180 TFLOP/s (3270)
//     bf16 gated (8192, 4096, 8192), three results    1004 and 975 us, 1095 to 1130 TFLOP/s (1620);  its gradients, 8 T C F, 2050 us, 1070 TFLOP/s
//     fp32 gated (1028, 6976, 3712)                   863 us, 123 TFLOP/s (154)
// Few rows are bound by the weights' way: one token bf16 (4096, 2 x 8192) 31 us with weights from memory, 4.3 TB/s, 24 where the last call's are still in the last-level
// cache; in 8 bits (4096, 8192) 10.3 and 7.5, 3.3 and 4.5 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cacnn_feed.h"
#include "cacnn_gate.h"
#include "cacnn_internal.h"
#include "cacnn_lds_load.h"

namespace cacnn {

typedef float mf32x4 __attribute__((ext_vector_type(4)));
typedef float mf32x16 __attribute__((ext_vector_type(16)));
typedef int mi32x8 __attribute__((ext_vector_type(8)));
typedef unsigned int mu32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int mu32x4 __attribute__((ext_vector_type(4)));
typedef short ms16x4 __attribute__((ext_vector_type(4)));
// (a lambda that is called twice may stay a function, with everything it refers to in memory)
#define MAT_INLINE __attribute__((always_inline))
typedef __bf16 mbf16x8 __attribute__((ext_vector_type(8)));
#define MAT_LDS(T) __attribute__((address_space(3))) T
#define MAT_CONST(T) __attribute__((address_space(4))) const T
// 16 and 8 bytes at any address: the memory takes them in one access, over two lines where they lie so
struct __attribute__((packed, aligned(1))) MatBytes16 {
    mu32x4 v;
};
struct __attribute__((packed, aligned(1))) MatBytes8 {
    mu32x2 v;
};

// Where the strided operand's block b of contraction index k lies: b ^ strided_turn.  The lanes of one access have k = 8 g + (0..3) (bf16, blocks of
// 64 bytes) or 4 g + e (fp32, blocks of 128), g = 0 and 1.
template <int ESZ, int ROWS>
__device__ __forceinline__ int strided_turn(int k) {
    constexpr int BLOCKS = ROWS / 32;
    if constexpr (ESZ == 4) return BLOCKS > 1 ? (k >> 2) & 1 : 0;
    else return BLOCKS >= 8 ? (k & 3) | ((k >> 3) & 1) << 2 : BLOCKS == 4 ? k & 3 : BLOCKS == 2 ? (k >> 1) & 1 : 0;
}

// What a lane's i-th 16 bytes of a slab are: the slab's 16-byte pieces in the order in which they lie in LDS, dealt to the lanes
// of a wave, 1024 bytes at a time, in turns to the waves.
// SLAB: bytes of a row and slab, 64 or 128.
__device__ __forceinline__ int chunk_turn(int slab, int row) { return slab == 128 ? (row >> 1) & 7 : (row >> 2) & 3; }
template <int ESZ, bool STRIDED, int ROWS, int WAVES, int SLAB>
struct SlabMap {
    static constexpr int N = ROWS * SLAB / 1024 / WAVES, KR = SLAB / ESZ, LANES = ROWS * ESZ / 16;   // pieces a lane; indices a slab; lanes a strided row
    static constexpr int CHUNKS = SLAB / 16;
    static_assert(N >= 1 && N * WAVES * 1024 == ROWS * SLAB, "a slab is whole wave loads");
    // contiguous: row and byte of the slab's row
    static __device__ __forceinline__ int row(int i, int wave, int lane) { return (i * WAVES + wave) * (64 / CHUNKS) + lane / CHUNKS; }
    static __device__ __forceinline__ int byte(int i, int wave, int lane) { return (lane % CHUNKS ^ chunk_turn(SLAB, row(i, wave, lane))) * 16; }
    // strided: contraction index within the slab, and byte of that row
    static __device__ __forceinline__ int index(int i, int wave, int lane) { return (i * WAVES + wave) * (64 / LANES) + lane / LANES; }
    static __device__ __forceinline__ int column(int i, int wave, int lane) {
        constexpr int PIECES = ESZ == 4 ? 8 : 4;                                  // of 16 bytes in a block
        const int at = lane % LANES, k = index(i, wave, lane);
        return (at / PIECES ^ strided_turn<ESZ, ROWS>(k)) * (PIECES * 16) + at % PIECES * 16;
    }
};

// 16 bytes moved down by `bytes` (0 to 16), zeros behind them
__device__ __forceinline__ mu32x4 moved_down(mu32x4 v, int bytes) {
    if (bytes & 4) v = mu32x4{v[1], v[2], v[3], 0};
    if (bytes & 8) v = mu32x4{v[2], v[3], 0, 0};
    if (bytes & 16) v = mu32x4{0, 0, 0, 0};
    const int b = bytes & 3;
    return mu32x4{__builtin_amdgcn_alignbyte(v[1], v[0], b), __builtin_amdgcn_alignbyte(v[2], v[1], b), __builtin_amdgcn_alignbyte(v[3], v[2], b),
                  __builtin_amdgcn_alignbyte(0, v[3], b)};
}

// Brings slabs to LDS through registers, from any address, 16 bytes a load, where rows have 16 bytes or more.  Every load is made, and within the array: a
// piece that the end of a row cuts is loaded as the row's last 16 bytes and moved down when it has come, all the way where it lies behind the last
// contraction index; rows and columns behind the last stand for it again (what comes of them is not stored).  (With a question before each load
// the compiler waits for all that are on their way before it uses one, and with the cut pieces read element by element the tiles at the edge took as
// long as all others together.)
// SETS of registers: slabs on their way at a time; which set a slab has is known where it is loaded and put.
template <int ESZ, bool STRIDED, int ROWS, int WAVES, int SLAB, int SETS>
struct RegisterLoader {
    using Map = SlabMap<ESZ, STRIDED, ROWS, WAVES, SLAB>;
    const char* base;
    int64_t ld, k;
    int rows, wave, lane;
    bool cut[SETS];                // the slab's pieces have to be moved
    int off[Map::N];               // (strided, in a tile of few columns: the row's last 16 bytes begin before it)
    int down[SETS][Map::N], edge[Map::N];    // bytes to move the slab's pieces by, and (strided) those at the last column
    mu32x4 r[SETS][Map::N];

    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave_, int lane_) {
        ld = o.ld, k = o.k, wave = wave_, lane = lane_;
        rows = (int)max((int64_t)0, min((int64_t)ROWS, o.rows - row0));
        move(o, row0);
#pragma unroll
        for (int i = 0; i < Map::N; ++i) {
            edge[i] = 0;
            if constexpr (STRIDED) {
                const int col = Map::column(i, wave, lane), last = rows ? rows * ESZ - 16 : 0;
                edge[i] = min(max(col - last, 0), 16);
                off[i] = Map::index(i, wave, lane) * (int)ld + min(col, last);
            } else {
                off[i] = min(Map::row(i, wave, lane), max(rows - 1, 0)) * (int)ld;
            }
        }
    }
    // (a tile behind the last row or column: the first ones')
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) { base = o.base + (rows ? (STRIDED ? row0 * ESZ : row0 * ld) : 0); }
    // slab s of the operand (none if !any: zeros)
    __device__ __forceinline__ void load(int64_t s, bool any, int set) {
        any = any && rows > 0;
        s = any ? s : 0;                                                          // (a load from there for nothing)
        cut[set] = !any || (STRIDED ? rows < ROWS || (s + 1) * Map::KR > k : (s + 1) * SLAB > k * ESZ);
        const char* const from = base + (STRIDED ? s * Map::KR * ld : 0);
        const int left = (int)min(k - s * Map::KR, (int64_t)Map::KR);             // strided: indices from the slab's first to the operand's last
        const int end = (int)(k * ESZ);
#pragma unroll
        for (int i = 0; i < Map::N; ++i) {
            if constexpr (STRIDED) {
                const int behind = max(Map::index(i, wave, lane) - left + 1, 0);
                down[set][i] = any && !behind ? edge[i] : 16;
                r[set][i] = ((const MatBytes16*)(from + (off[i] - behind * (int)ld)))->v;
            } else {
                const int at = (int)s * SLAB + Map::byte(i, wave, lane), to = min(at, end - 16);
                down[set][i] = any ? min(at - to, 16) : 16;
                r[set][i] = ((const MatBytes16*)(from + (off[i] + to)))->v;
            }
        }
    }
    __device__ __forceinline__ void put(char* slab, int set) {
        if (cut[set])
#pragma unroll
            for (int i = 0; i < Map::N; ++i) r[set][i] = moved_down(r[set][i], down[set][i]);
#pragma unroll
        for (int i = 0; i < Map::N; ++i) *(mu32x4*)(slab + (i * WAVES + wave) * 1024 + lane * 16) = r[set][i];
    }
};

// Brings slabs straight to LDS: rows and their parts are whole 16 bytes at multiples of 16 (or zeros follow them there).  Offsets beyond the operand are
// turned into ones beyond the descriptor's bytes, which are at most 2^30: the load puts zeros there.
constexpr uint32_t kOutside = 0x40000000u;
__device__ __forceinline__ i32x4 bytes_from(const char* p, int64_t bytes) {
    const uint64_t a = (uint64_t)p;
    i32x4 d;
    d[0] = __builtin_amdgcn_readfirstlane((int)(uint32_t)a);
    d[1] = __builtin_amdgcn_readfirstlane((int)(uint32_t)(a >> 32) & 0xffff);
    d[2] = __builtin_amdgcn_readfirstlane((int)bytes);
    d[3] = 0x00020000;
    return d;
}
template <int ESZ, bool STRIDED, int ROWS, int WAVES, int SLAB>
struct DirectLoader {
    using Map = SlabMap<ESZ, STRIDED, ROWS, WAVES, SLAB>;
    const char* base;
    int64_t ld, k;
    int bytes;                     // contiguous: of a row; strided: of a row of the tile; whole pieces of 16
    int wave, lane;
    i32x4 d;
    uint32_t off[Map::N], at;

    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave_, int lane_) {
        wave = wave_, lane = lane_, ld = o.ld, k = o.k;
        const int rows = (int)max((int64_t)0, min((int64_t)ROWS, o.rows - row0));
        base = o.base + (STRIDED ? row0 * ESZ : row0 * ld);
        if constexpr (STRIDED) {
            bytes = (rows * ESZ + 15) & ~15;
#pragma unroll
            for (int i = 0; i < Map::N; ++i) {
                const int col = Map::column(i, wave, lane);
                off[i] = col < bytes ? (uint32_t)Map::index(i, wave, lane) * (uint32_t)ld + col : kOutside;
            }
        } else {
            bytes = (int)((k * ESZ + 15) & ~15);
            d = bytes_from(base, rows ? (int64_t)(rows - 1) * ld + bytes : 0);
#pragma unroll
            for (int i = 0; i < Map::N; ++i) {
                const int row = Map::row(i, wave, lane);
                off[i] = row < rows ? (uint32_t)row * (uint32_t)ld + Map::byte(i, wave, lane) : kOutside;
            }
        }
    }
    // another array of the same shape
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) {
        base = o.base + (STRIDED ? row0 * ESZ : row0 * ld);
        if constexpr (!STRIDED) d = bytes_from(base, (uint32_t)d[2]);
    }
    // Slab s (none if !any: zeros) is the one that issue() brings, a load at a time
    __device__ __forceinline__ void prepare(int s, bool any) {
        if constexpr (STRIDED) {
            const int64_t from = (int64_t)s * Map::KR;
            const int64_t left = any ? min(k - from, (int64_t)Map::KR) : 0;
            d = bytes_from(base + from * ld, left > 0 ? (left - 1) * ld + bytes : 0);
        } else {
            at = any ? (uint32_t)(s * SLAB) : kOutside;
        }
    }
    __device__ __forceinline__ void issue(int i, uint32_t slab) {
        uint32_t more = 0;
        if constexpr (!STRIDED) more = at + Map::byte(i, wave, lane) < (uint32_t)bytes ? at : kOutside;
        load_to_lds_unseen(d, off[i] + more, slab + (i * WAVES + wave) * 1024);
    }
};
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(MAT_LDS(const char)*)p; }
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// One operand's way to LDS
template <int ESZ, bool STRIDED, int ROWS, int WAVES, int SLAB, bool DIRECT, int SETS>
struct Loader {
    static constexpr int LOADS = SlabMap<ESZ, STRIDED, ROWS, WAVES, SLAB>::N;
    DirectLoader<ESZ, STRIDED, ROWS, WAVES, SLAB> l;
    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave, int lane) { l.init(o, row0, wave, lane); }
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) { l.move(o, row0); }
    // slab s is brought by the LOADS calls of issue() that follow, or by put() after the loads that prepare() made have come
    __device__ __forceinline__ void prepare(int s, bool any, int) { l.prepare(s, any); }
    __device__ __forceinline__ void issue(int i, uint32_t slab) { l.issue(i, slab); }
    __device__ __forceinline__ void put(char*, int) {}
};
template <int ESZ, bool STRIDED, int ROWS, int WAVES, int SLAB, int SETS>
struct Loader<ESZ, STRIDED, ROWS, WAVES, SLAB, false, SETS> {
    static constexpr int LOADS = 0;
    RegisterLoader<ESZ, STRIDED, ROWS, WAVES, SLAB, SETS> l;
    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave, int lane) { l.init(o, row0, wave, lane); }
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) { l.move(o, row0); }
    __device__ __forceinline__ void prepare(int s, bool any, int set) { l.load(s, any, set); }
    __device__ __forceinline__ void issue(int, uint32_t) {}
    __device__ __forceinline__ void put(char* slab, int set) { l.put(slab, set); }
};

// A block of 32 rows (or columns) of step `st` of a slab, as the matrix instructions take it: 16 bytes a lane
template <int ESZ, bool STRIDED, int ROWS, int SLAB>
__device__ __forceinline__ mu32x4 read_block(const char* slab, int block, int st, int lane) {
    const int j = lane & 31, g = lane >> 5;
    if constexpr (!STRIDED) {
        return *(const mu32x4*)(slab + (block * 32 + j) * SLAB + (((2 * st + g) ^ chunk_turn(SLAB, j)) * 16));
    } else if constexpr (ESZ == 4) {
        mu32x4 v;
        const int k = 8 * st + 4 * g;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = *(const uint32_t*)(slab + (k + e) * ROWS * 4 + (block ^ strided_turn<4, ROWS>(k)) * 128 + j * 4);
        return v;
    } else {
        // the transposing read: four rows (contraction indices) of 16 columns to a lane per column
        const int i16 = lane & 15, half = (lane >> 4) & 1, k = 16 * st + 8 * g + (i16 >> 2);
        const char* const p = slab + k * ROWS * 2 + (block ^ strided_turn<2, ROWS>(k)) * 64 + half * 32 + (i16 & 3) * 8;
        const ms16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MAT_LDS(ms16x4)*)p);
        const ms16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((MAT_LDS(ms16x4)*)(p + 4 * ROWS * 2));
        return __builtin_bit_cast(mu32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    }
}

template <int DT>
__device__ __forceinline__ void multiply(mf32x16& acc, mu32x4 p, mu32x4 q) {
    if constexpr (DT == FEED_F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(p[e]), __uint_as_float(q[e]), acc, 0, 0, 0);
    } else {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(mbf16x8, p), __builtin_bit_cast(mbf16x8, q), acc, 0, 0, 0);
    }
}
// Eight of the sixteen 8-bit floats of a chunk as bf16, exactly
__device__ __forceinline__ mu32x4 half_as_bf16(mu32x4 v, int half) {
    mu32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = v[half * 2 + i / 2];
        r[i] = __builtin_bit_cast(uint32_t, i & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false));
    }
    return r;
}
// Two chunks of either operand, 64 contraction indices of 8 bits (the instruction without scales)
__device__ __forceinline__ mf32x16 multiply_e4m3(const mf32x16& c, const mu32x4 (&p)[2], const mu32x4 (&q)[2]) {
    mi32x8 a, b;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = (int)p[i / 4][i % 4], b[i] = (int)q[i / 4][i % 4];
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, 0, 0, 0, 0);
}

__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    return (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)lo) | (uint32_t)__builtin_bit_cast(uint16_t, (__bf16)hi) << 16;
}

// E adjacent columns from n on of row m, those below `cols`: 16 or 8 bytes.  STREAM: past the L2, for lines that a wave writes whole
template <int DT, int E, bool STREAM = false>
__device__ __forceinline__ void store_run(const FeedOut& o, int64_t m, int64_t n, int64_t cols, const float (&v)[E]) {
    constexpr bool WORDS = DT == FEED_F32 || DT == FEED_E4M3_EXACT;
    static_assert(E == 4 || (E == 8 && !WORDS), "what one store takes");
    char* const p = o.base + m * o.ld + n * (WORDS ? 4 : 2);
    if (n + E <= cols) {
        if constexpr (!WORDS && E == 4) {
            ((MatBytes8*)p)->v = mu32x2{two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
        } else {
            mu32x4 x;
            if constexpr (WORDS) x = __builtin_bit_cast(mu32x4, mf32x4{v[0], v[1], v[2], v[3]});
            else x = mu32x4{two_bf16(v[0], v[1]), two_bf16(v[2], v[3]), two_bf16(v[4], v[5]), two_bf16(v[6], v[7])};
            if constexpr (STREAM) __builtin_nontemporal_store(x, (mu32x4*)p);
            else ((MatBytes16*)p)->v = x;
        }
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (n + e < cols) {
                if constexpr (WORDS) ((float*)p)[e] = v[e];
                else ((uint16_t*)p)[e] = __builtin_bit_cast(uint16_t, (__bf16)v[e]);
            }
    }
}

// What becomes of E adjacent columns of a row, given their sums (gated: v of gate, u of up)
template <int DT, bool GATED, bool STREAM, int E>
__device__ __forceinline__ void finish_run(const FeedArgs& a, int product, int64_t m, int64_t n, const float (&v)[E], const float (&u)[E]) {
    if (m >= a.M) return;
    if constexpr (!GATED) {
        store_run<DT, E, STREAM>(a.out[product], m, n, a.N, v);
    } else if (feed_size(DT) > 1 && a.grad_out) {
        if (n >= a.grad_cols) return;
        float d[E];
        const char* const p = a.grad_out + m * a.grad_out_ld + n * feed_size(DT);
        if (n + E <= a.N) {
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                if constexpr (DT == FEED_F32) {
                    const mf32x4 w = __builtin_bit_cast(mf32x4, ((const MatBytes16*)(p + e * 4))->v);
#pragma unroll
                    for (int x = 0; x < 4; ++x) d[e + x] = w[x];
                } else {
                    const mu32x2 w = ((const MatBytes8*)(p + e * 2))->v;
#pragma unroll
                    for (int x = 0; x < 4; ++x) d[e + x] = __uint_as_float(x & 1 ? w[x / 2] & 0xffff0000u : w[x / 2] << 16);
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                d[e] = n + e >= a.N ? 0.f : DT == FEED_F32 ? ((const float*)p)[e] : __uint_as_float((uint32_t)((const uint16_t*)p)[e] << 16);
        }
        float dg[E], du[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            dg[e] = du[e] = 0.f;
            if (n + e < a.N) gate_grad(a.activation, v[e], u[e], d[e], dg[e], du[e]);
        }
        store_run<DT>(a.out[0], m, n, a.grad_cols, dg);
        store_run<DT>(a.out[1], m, n, a.grad_cols, du);
    } else {
        float h[E];
#pragma unroll
        for (int e = 0; e < E; ++e) h[e] = gate_value(a.activation, v[e]) * u[e];
        store_run<DT>(a.out[0], m, n, a.N, h);
        if (a.gate_out.base) {
            store_run<DT>(a.gate_out, m, n, a.N, v);
            store_run<DT>(a.up_out, m, n, a.N, u);
        }
    }
}

// Tile number -> product and place.  Consecutive workgroups go to different XCDs: each XCD gets one run of the tiles, and walks it in groups of
// eight rows of tiles, so that the 32 tiles it works on at a time share eight rows' and four columns' operands in its L2.
struct TilePlace {
    int product, m, n;
};
__device__ __forceinline__ TilePlace tile_place(const FeedArgs& a, int wg) {
    const int each = a.n_tiles / 8, rest = a.n_tiles % 8, x = wg % 8;
    int t = x * each + min(x, rest) + wg / 8;
    const int of_product = a.tiles_m * a.tiles_n;
    TilePlace p;
    p.product = t / of_product;
    t -= p.product * of_product;
    const int group = t / (8 * a.tiles_n), first = group * 8, high = min(8, a.tiles_m - first), in = t - group * 8 * a.tiles_n;
    p.m = first + in % high;
    p.n = in / high;
    return p;
}

// QB x PB blocks of 32 x 32 to a wave, WM x WN waves.  GATED: half of a wave's columns are of the gate, the others the same ones of up.
// Of STAGES slabs one is multiplied, the others are in LDS or on their way.
template <int DT, int FORM, int QB, int PB, int WM, int WN, int SLAB, int STAGES>
struct BlockShape {
    static constexpr int ESZ = feed_size(DT), WAVES = WM * WN, BM = WM * QB * 32, BN = WN * PB * 32;
    static constexpr bool GATED = FORM == FEED_GATED, Q_STRIDED = FORM == FEED_BOTH, P_STRIDED = FORM >= FEED_RIGHT;
    static constexpr int COLS = GATED ? BN / 2 : BN;                    // of Out
    static constexpr int P_PARTS = GATED ? 2 : 1, P_ROWS = BN / P_PARTS;
    static constexpr int Q_BYTES = BM * SLAB, P_BYTES = BN * SLAB, SCALES = ESZ == 1 ? BM * 4 : 0;
    static constexpr int STAGE = Q_BYTES + P_BYTES + SCALES, LDS = STAGES * STAGE;
    static_assert(ESZ > 1 || SLAB == kScaleBlock, "a slab in 8 bits has one scale");
};

// QD, PD: whether the operands go straight to LDS.
template <int DT, int FORM, int QB, int PB, int WM, int WN, int SLAB, int STAGES, bool QD, bool PD>
__global__ void __launch_bounds__(WM* WN * 64, WM* WN == 4 ? 2 : 1) matmul_block_kernel(const FeedArgs a) {
    using S = BlockShape<DT, FORM, QB, PB, WM, WN, SLAB, STAGES>;
    constexpr int ESZ = S::ESZ, WAVES = S::WAVES, KE = SLAB / ESZ;
    static_assert(STAGES == 2 || (QD && PD), "operands that come through registers are one slab ahead");
    extern __shared__ __align__(16) char s_mem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM, j = lane & 31, g = lane >> 5;
    const TilePlace at = tile_place(a, blockIdx.x);
    const int64_t m0 = (int64_t)at.m * S::BM, n0 = (int64_t)at.n * S::COLS;

    // (both through registers: two slabs on their way.  With one, a slab took as long as its loads: bf16 gated (777, 1001, 1515) 25.5 us)
    constexpr int SETS = !QD && !PD && ESZ > 1 ? 2 : 1;
    using QLoader = Loader<ESZ, S::Q_STRIDED, S::BM, WAVES, SLAB, QD, SETS>;
    using PLoader = Loader<ESZ, S::P_STRIDED, S::P_ROWS, WAVES, SLAB, PD, SETS>;
    constexpr int LOADS = QLoader::LOADS + S::P_PARTS * PLoader::LOADS + (ESZ == 1 ? 1 : 0);    // of a wave and slab
    QLoader q;
    PLoader p0, p1;                                            // (p1: of up, where there is one)
    q.init(a.q[at.product], m0, wave, lane);
    p0.init(a.p[0], n0, wave, lane);
    if constexpr (S::GATED) p1.init(a.p[1], n0, wave, lane);
    const int per_segment = (int)((a.q[0].k + KE - 1) / KE), slabs = max(1, per_segment * a.segments);
    // 8 bits: the scales of a slab's rows, a word each, 64 rows a wave (rows behind the last: zeros; more waves bring the same again, so that
    // every wave has as many loads on their way)
    const int scale_wave = wave % (S::BM / 64);
    const i32x4 scales = ESZ == 1 ? bytes_from((const char*)(a.q_scale + m0 * a.scale_cols), min((int64_t)S::BM, a.M - m0) * a.scale_cols * 4) : i32x4{0, 0, 0, 0};
    const uint32_t scale_off = (uint32_t)(scale_wave * 64 + lane) * a.scale_cols * 4;
    // Slab s is the one that load_some() brings (behind the last: zeros, so that the loads on their way can be counted)
    const uint32_t lds = lds_address(s_mem);
    uint32_t coming = lds;
    int coming_slab = 0;
    auto prepare = [&](int s, int at_stage, int set) MAT_INLINE {
        coming = lds + at_stage * S::STAGE;
        coming_slab = s;
        if constexpr (FORM == FEED_RIGHT)
            if (s >= per_segment && a.segments > 1) {
                coming_slab = s - per_segment;
                q.move(a.q[1], m0);
                p0.move(a.p[1], n0);
            }
        const bool any = s < slabs && coming_slab < per_segment;
        q.prepare(coming_slab, any, set);
        p0.prepare(coming_slab, any, set);
        if constexpr (S::GATED) p1.prepare(coming_slab, any, set);
    };
    auto load_some = [&](int from, int to) MAT_INLINE {
#pragma unroll
        for (int l = from; l < to; ++l) {
            if constexpr (QD)
                if (l < QLoader::LOADS) q.issue(l, coming);
            if constexpr (PD) {
                const int i = l - QLoader::LOADS;
                if (i >= 0 && i < PLoader::LOADS) p0.issue(i, coming + S::Q_BYTES);
                if constexpr (S::GATED)
                    if (i >= PLoader::LOADS && i < 2 * PLoader::LOADS) p1.issue(i - PLoader::LOADS, coming + S::Q_BYTES + S::P_ROWS * SLAB);
            }
            if constexpr (ESZ == 1)
                if (l == LOADS - 1)
                    load_word_to_lds_unseen(scales, scale_off + coming_slab * 4, coming + S::Q_BYTES + S::P_BYTES + scale_wave * 256);
        }
    };
    auto put = [&](int at_stage, int set) MAT_INLINE {
        char* const stage = s_mem + at_stage * S::STAGE;
        q.put(stage, set);
        p0.put(stage + S::Q_BYTES, set);
        if constexpr (S::GATED) p1.put(stage + S::Q_BYTES + S::P_ROWS * SLAB, set);
    };
    // a wave's i-th block of columns: part of p, block within it
    auto part_of = [&](int i) { return S::GATED ? i / (PB / 2) : 0; };
    auto block_of = [&](int i) { return S::GATED ? wn * (PB / 2) + i % (PB / 2) : wn * PB + i; };
    int stage = 0;                                             // of the slab that is multiplied
    auto q_slab = [&](int at_stage) -> const char* { return s_mem + at_stage * S::STAGE; };
    auto p_slab = [&](int at_stage, int i) -> const char* { return s_mem + at_stage * S::STAGE + S::Q_BYTES + part_of(i) * S::P_ROWS * SLAB; };
    // This wave has read what it needs of slab s - 1, and slab s is there for all; the stage of slab s - 1 takes the next one
    auto next = [&](int s, int set) MAT_INLINE {
        const int free = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        if constexpr (LOADS > 0) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((STAGES - 2) * LOADS) : "memory");
        put(stage, set);
        lds_done();
        __builtin_amdgcn_s_barrier();
        prepare(s + (SETS > 1 ? SETS : STAGES - 1), free, set);
        asm volatile("" ::: "memory");
    };
    // Between two calls of next() the wave multiplies several times, and behind each brings a part of the next slab: all at once, the loads keep it
    // from issuing products for as long as those of all waves take to be accepted (bf16, 256 x 256: 1012 -> 977 us for 1.1 TFLOP).  With two stages there is one slab only between a load
    // and its wait: early, in one go with four waves, in two with eight (128 x 128 tiles 3 to 20 % slower if spread).
    auto phase_of = [](int phase, int phases) {
        const int n = STAGES > 2 ? phases : WAVES > 4 ? 2 : 1;
        return min(LOADS, (LOADS + n - 1) / n * phase);
    };

    mf32x16 acc[PB][QB];
#pragma unroll
    for (int i = 0; i < PB; ++i)
#pragma unroll
        for (int h = 0; h < QB; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][h][v] = 0.f;

#pragma unroll
    for (int s = 0; s < (SETS > 1 ? SETS : STAGES - 1); ++s) {
        prepare(s, s, SETS > 1 ? s : 0);
        load_some(0, LOADS);
    }
    stage = STAGES - 1;
    next(0, 0);
    if constexpr (DT == FEED_E4M3) load_some(0, phase_of(1, QB));
    if constexpr (DT == FEED_E4M3_EXACT) load_some(0, LOADS);
    if constexpr (ESZ > 1) {
        // The operands of a step are read under the products of the step before, across slabs too
        mu32x4 pv[2][PB], qv[2][QB];
        auto read = [&](int st, int set) MAT_INLINE {
#pragma unroll
            for (int i = 0; i < PB; ++i) pv[set][i] = read_block<ESZ, S::P_STRIDED, S::P_ROWS, SLAB>(p_slab(stage, i), block_of(i), st, lane);
#pragma unroll
            for (int h = 0; h < QB; ++h) qv[set][h] = read_block<ESZ, S::Q_STRIDED, S::BM, SLAB>(q_slab(stage), wm * QB + h, st, lane);
            __builtin_amdgcn_sched_barrier(0);
        };
        constexpr int STEPS = SLAB / 32;
        auto products = [&](int set, int phase) MAT_INLINE {
#pragma unroll
            for (int i = 0; i < PB; ++i) {
#pragma unroll
                for (int h = 0; h < QB; ++h) multiply<DT>(acc[i][h], pv[set][i], qv[set][h]);
                __builtin_amdgcn_sched_barrier(0);
                load_some(phase_of(phase * PB + i, PB * STEPS), phase_of(phase * PB + i + 1, PB * STEPS));
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        read(0, 0);
        // (the first slab's phases but the last, which is the first one's behind next())
        load_some(0, phase_of(PB, PB * STEPS));
        for (int from = 0; from < slabs; from += SETS)
#pragma unroll
            for (int set = 0; set < SETS; ++set) {
                const int s = from + set;
                if (set > 0 && s >= slabs) break;
#pragma unroll
                for (int st = 0; st < STEPS; ++st) {
                    if (st + 1 < STEPS) {
                        read(st + 1, (st + 1) & 1);
                    } else if (s + 1 < slabs) {
                        next(s + 1, (set + 1) % SETS);
                        read(0, 0);
                    }
                    products(st & 1, (st + 1) % STEPS);
                }
            }
    } else {
        for (int s = 0; s < slabs; ++s) {
            // a slab is one block of the scales: its sum of products first, then the product of the two scales times it
            float sp[PB], sq[QB];
#pragma unroll
            for (int i = 0; i < PB; ++i) {
                const int64_t col = min(n0 + block_of(i) * 32, a.N - 1);
                sp[i] = ((MAT_CONST(float)*)(uintptr_t)a.p_scale[part_of(i)])[col / kScaleBlock * a.scale_cols + s];
            }
#pragma unroll
            for (int h = 0; h < QB; ++h) sq[h] = *(const float*)(q_slab(stage) + S::Q_BYTES + S::P_BYTES + ((wm * QB + h) * 32 + j) * 4);
            auto add = [&](int i, int h, const mf32x16& c) MAT_INLINE {
                const float f = sp[i] * sq[h];
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][h][v] = __builtin_fmaf(c[v], f, acc[i][h][v]);
                // (here and now: the compiler puts all of them off to the end of the slab, with a register for every product until then)
                asm volatile("" : "+v"(acc[i][h]));
            };
            if constexpr (DT == FEED_E4M3) {
                // (one address for each of the four chunks and operand, the blocks at constant distances: more and the sums spill)
                const uint32_t qa = lds_address(q_slab(stage)) + (wm * QB * 32 + j) * SLAB, pa = lds_address(q_slab(stage)) + S::Q_BYTES + (block_of(0) * 32 + j) * SLAB;
                uint32_t chunk[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) chunk[x] = ((2 * x + g) ^ chunk_turn(SLAB, j)) * 16;
                auto chunk_at = [](uint32_t at, int more) { return *(MAT_LDS(const mu32x4)*)((MAT_LDS(const char)*)(uintptr_t)at + more); };
                mu32x4 pv[PB][2][2], qv[2][2];
                auto read_q = [&](int h) MAT_INLINE {
#pragma unroll
                    for (int x = 0; x < 4; ++x) qv[x / 2][x % 2] = chunk_at(qa + chunk[x], h * 32 * SLAB);
                };
#pragma unroll
                for (int i = 0; i < PB; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        pv[i][x / 2][x % 2] = chunk_at(pa + chunk[x], (part_of(i) * S::P_ROWS + (block_of(i) - block_of(0)) * 32) * SLAB);
                read_q(0);
#pragma unroll
                for (int h = 0; h < QB; ++h) {
                    if (h + 1 == QB && s + 1 < slabs) next(s + 1, 0);
                    mf32x16 c[PB];
#pragma unroll
                    for (int i = 0; i < PB; ++i) {
#pragma unroll
                        for (int v = 0; v < 16; ++v) c[i][v] = 0.f;
                        c[i] = multiply_e4m3(multiply_e4m3(c[i], pv[i][0], qv[0]), pv[i][1], qv[1]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (h + 1 < QB) read_q(h + 1);
                    load_some(phase_of((h + 1) % QB, QB), phase_of((h + 1) % QB + 1, QB));
#pragma unroll
                    for (int i = 0; i < PB; ++i) add(i, h, c[i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            } else {
                mf32x16 c[PB][QB];
#pragma unroll
                for (int i = 0; i < PB; ++i)
#pragma unroll
                    for (int h = 0; h < QB; ++h)
#pragma unroll
                        for (int v = 0; v < 16; ++v) c[i][h][v] = 0.f;
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    mu32x4 pv[PB], qv[QB];
#pragma unroll
                    for (int i = 0; i < PB; ++i) pv[i] = read_block<1, false, S::P_ROWS, SLAB>(p_slab(stage, i), block_of(i), x, lane);
#pragma unroll
                    for (int h = 0; h < QB; ++h) qv[h] = read_block<1, false, S::BM, SLAB>(q_slab(stage), wm * QB + h, x, lane);
#pragma unroll
                    for (int half = 0; half < 2; ++half)
#pragma unroll
                        for (int i = 0; i < PB; ++i)
#pragma unroll
                            for (int h = 0; h < QB; ++h) multiply<FEED_BF16>(c[i][h], half_as_bf16(pv[i], half), half_as_bf16(qv[h], half));
                }
#pragma unroll
                for (int i = 0; i < PB; ++i)
#pragma unroll
                    for (int h = 0; h < QB; ++h) add(i, h, c[i][h]);
                if (s + 1 < slabs) {
                    next(s + 1, 0);
                    load_some(0, LOADS);
                }
            }
        }
    }

    // Out: a wave turns the sums of 32 rows round in its part of LDS, so that a lane has 16 bytes of a row, and several lanes the row's columns of the
    // wave: stored from where the matrix instructions leave them, 16 bytes of a row at a time, results make four times as many pieces of lines.  (bf16 gated
    // (8192, 4096, 8192) with gate and up kept, 400 MB of results: 1160 us that way.)
    loads_done();                                              // (also those of zeros: their LDS is given up)
    __syncthreads();
    constexpr int RUN = DT == FEED_F32 || DT == FEED_E4M3_EXACT ? 4 : 8, COLS = (S::GATED ? PB / 2 : PB) * 32, PITCH = PB * 128 + 16, LANES = COLS / RUN;
    static_assert(WAVES * 32 * PITCH <= S::LDS, "a block's rows for each wave");
    char* const turn = s_mem + wave * (32 * PITCH);
#pragma unroll
    for (int h = 0; h < QB; ++h) {
#pragma unroll
        for (int i = 0; i < PB; ++i)
#pragma unroll
            for (int v = 0; v < 16; v += 4)
                *(mf32x4*)(turn + j * PITCH + (i * 32 + v * 2 + g * 4) * 4) = mf32x4{acc[i][h][v], acc[i][h][v + 1], acc[i][h][v + 2], acc[i][h][v + 3]};
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
        auto rows = [&](auto stream) MAT_INLINE {
#pragma unroll 1
            for (int row = lane / LANES; row < 32; row += 64 / LANES) {
                const int col = lane % LANES * RUN;
                float v[RUN], u[RUN];
#pragma unroll
                for (int e = 0; e < RUN; ++e) {
                    v[e] = *(const float*)(turn + row * PITCH + (col + e) * 4);
                    u[e] = S::GATED ? *(const float*)(turn + row * PITCH + (COLS + col + e) * 4) : 0.f;
                }
                finish_run<DT, S::GATED, decltype(stream)::value>(a, at.product, m0 + (wm * QB + h) * 32 + row, n0 + block_of(0) * 32 + col, v, u);
            }
        };
        // (whole lines past the L2: the 8-bit product of (8192, 8192, 4096) 281 -> 271 us; with fp32 results (8192, 2048, 8192) 274 -> 268, (1024, 4096, 4096) 48.7 -> 47.4,
        // (8192, 512, 8192) 96 either way.  A gated wave's are half lines: 1015 -> 1042; the gradients in bf16, four times the arithmetic to a line, gain nothing: 2024 -> 2038)
        constexpr bool STREAMS = ESZ == 1 && !S::GATED;
        if (STREAMS && a.out[at.product].lines) rows(std::integral_constant<bool, STREAMS>{});
        else rows(std::false_type{});
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
    }
}

// Few rows: the weights set the pace, and there are more compute units than tiles of the kernel above.  A workgroup owns QB x PB blocks of 32 x 32 of Out and
// its four waves divide the contraction, every fourth slab each; a wave brings its slabs to LDS and multiplies them alone, so that nothing waits at a
// barrier, and the four sums are added at the end, in the order of the waves.  DEPTH slabs of a wave are in LDS or on their way.
template <int DT, int FORM, int QB, int PB>
struct WaveShape {
    static constexpr int ESZ = feed_size(DT), BM = QB * 32;
    static constexpr bool GATED = FORM == FEED_GATED, Q_STRIDED = FORM == FEED_BOTH, P_STRIDED = FORM >= FEED_RIGHT;
    static constexpr int P_PARTS = GATED ? 2 : 1, P_ROWS = PB * 32 / P_PARTS, COLS = P_ROWS;
    static constexpr int SLAB = 128, Q_BYTES = BM * SLAB, P_BYTES = PB * 32 * SLAB, STAGE = Q_BYTES + P_BYTES + (ESZ == 1 ? 256 : 0);
    static constexpr int LOADS = (QB + PB) * 4 + (ESZ == 1 ? 1 : 0);            // of a slab
    static constexpr int FIT = 160 * 1024 / (4 * STAGE), DEPTH = FIT < 4 ? FIT : 4, LDS = 4 * DEPTH * STAGE;
    static_assert(DEPTH >= 2 && (DEPTH - 1) * LOADS < 64 && LDS >= 4 * QB * PB * 4096, "a wave's slabs, and the sums at the end");
};

template <int DT, int FORM, int QB, int PB, bool QD, bool PD>
__global__ void __launch_bounds__(256) matmul_waves_kernel(const FeedArgs a) {
    using S = WaveShape<DT, FORM, QB, PB>;
    constexpr int ESZ = S::ESZ, SLAB = S::SLAB, KE = SLAB / ESZ, DEPTH = QD && PD ? S::DEPTH : 2;
    extern __shared__ __align__(16) char s_mem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int j = lane & 31, g = lane >> 5;
    const TilePlace at = tile_place(a, blockIdx.x);
    const int64_t m0 = (int64_t)at.m * S::BM, n0 = (int64_t)at.n * S::COLS;
    char* const mine = s_mem + wave * (S::DEPTH * S::STAGE);

    constexpr int SETS = !QD && !PD && ESZ > 1 ? 2 : 1;        // (as above)
    Loader<ESZ, S::Q_STRIDED, S::BM, 1, SLAB, QD, SETS> q;
    Loader<ESZ, S::P_STRIDED, S::P_ROWS, 1, SLAB, PD, SETS> p[S::P_PARTS];
    q.init(a.q[at.product], m0, 0, lane);
#pragma unroll
    for (int h = 0; h < S::P_PARTS; ++h) p[h].init(a.p[h], n0, 0, lane);
    const int per_segment = (int)((a.q[0].k + KE - 1) / KE), slabs = per_segment * a.segments, turns = (slabs + 3) / 4;
    const i32x4 scales = ESZ == 1 ? bytes_from((const char*)(a.q_scale + m0 * a.scale_cols), min((int64_t)S::BM, a.M - m0) * a.scale_cols * 4) : i32x4{0, 0, 0, 0};
    const uint32_t scale_off = (uint32_t)lane * a.scale_cols * 4;
    int segment = 0;
    // the wave's slab of turn `i` into stage `stage`; none behind the last: zeros, so that the loads on their way can be counted
    auto begin = [&](int i, int stage, int set) MAT_INLINE {
        const int s = i * 4 + wave;
        const uint32_t to = lds_address(mine) + stage * S::STAGE;
        int x = s;
        if constexpr (FORM == FEED_RIGHT)
            if (s >= per_segment) {
                x = s - per_segment;
                if (segment == 0 && a.segments > 1) {
                    segment = 1;
                    q.move(a.q[1], m0);
                    p[0].move(a.p[1], n0);
                }
            }
        q.prepare(x, s < slabs, set);
#pragma unroll
        for (int l = 0; l < S::BM / 8; ++l) q.issue(l, to);
#pragma unroll
        for (int h = 0; h < S::P_PARTS; ++h) {
            p[h].prepare(x, s < slabs, set);
#pragma unroll
            for (int l = 0; l < S::P_ROWS / 8; ++l) p[h].issue(l, to + S::Q_BYTES + h * S::P_ROWS * SLAB);
        }
        if constexpr (ESZ == 1) load_word_to_lds_unseen(scales, scale_off + x * 4, to + S::Q_BYTES + S::P_BYTES);
    };
    auto put = [&](int stage, int set) MAT_INLINE {
        char* const to = mine + stage * S::STAGE;
        q.put(to, set);
#pragma unroll
        for (int h = 0; h < S::P_PARTS; ++h) p[h].put(to + S::Q_BYTES + h * S::P_ROWS * SLAB, set);
    };
    auto part_of = [&](int i) { return S::GATED ? i / (PB / 2) : 0; };
    auto block_of = [&](int i) { return S::GATED ? i % (PB / 2) : i; };

    mf32x16 acc[PB][QB];
#pragma unroll
    for (int i = 0; i < PB; ++i)
#pragma unroll
        for (int h = 0; h < QB; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][h][v] = 0.f;
    auto compute = [&](int s, int stage) MAT_INLINE {
        const char* const qs = mine + stage * S::STAGE;
        const char* const ps = qs + S::Q_BYTES;
        mu32x4 pv[4][PB], qv[4][QB];
#pragma unroll
        for (int st = 0; st < 4; ++st) {
#pragma unroll
            for (int i = 0; i < PB; ++i) pv[st][i] = read_block<ESZ, S::P_STRIDED, S::P_ROWS, SLAB>(ps + part_of(i) * S::P_ROWS * SLAB, block_of(i), st, lane);
#pragma unroll
            for (int h = 0; h < QB; ++h) qv[st][h] = read_block<ESZ, S::Q_STRIDED, S::BM, SLAB>(qs, h, st, lane);
        }
        if constexpr (ESZ > 1) {
#pragma unroll
            for (int st = 0; st < 4; ++st)
#pragma unroll
                for (int i = 0; i < PB; ++i)
#pragma unroll
                    for (int h = 0; h < QB; ++h) multiply<DT>(acc[i][h], pv[st][i], qv[st][h]);
        } else {
            float sq[QB];
#pragma unroll
            for (int h = 0; h < QB; ++h) sq[h] = *(const float*)(ps + S::P_BYTES + (h * 32 + j) * 4);
#pragma unroll
            for (int i = 0; i < PB; ++i) {
                const int64_t col = min(n0 + block_of(i) * 32, a.N - 1);
                const float sp = ((MAT_CONST(float)*)(uintptr_t)a.p_scale[part_of(i)])[col / kScaleBlock * a.scale_cols + s];
#pragma unroll
                for (int h = 0; h < QB; ++h) {
                    mf32x16 c;
#pragma unroll
                    for (int v = 0; v < 16; ++v) c[v] = 0.f;
                    if constexpr (DT == FEED_E4M3) {
#pragma unroll
                        for (int x = 0; x < 2; ++x)
                            c = multiply_e4m3(c, {pv[2 * x][i], pv[2 * x + 1][i]}, {qv[2 * x][h], qv[2 * x + 1][h]});
                    } else {
#pragma unroll
                        for (int x = 0; x < 8; ++x) multiply<FEED_BF16>(c, half_as_bf16(pv[x / 2][i], x % 2), half_as_bf16(qv[x / 2][h], x % 2));
                    }
                    const float f = sp * sq[h];
#pragma unroll
                    for (int v = 0; v < 16; ++v) acc[i][h][v] = __builtin_fmaf(c[v], f, acc[i][h][v]);
                }
            }
        }
    };

    if constexpr (QD && PD) {
#pragma unroll
        for (int i = 0; i < DEPTH - 1; ++i) begin(i, i, 0);
        int stage = 0, free = DEPTH - 1;
        for (int i = 0; i < turns; ++i) {
            lds_done();                                    // what was read of the stage that is filled now
            begin(i + DEPTH - 1, free, 0);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"((DEPTH - 1) * S::LOADS) : "memory");
            if (i * 4 + wave < slabs) compute(i * 4 + wave, stage);
            free = stage;
            stage = stage + 1 == DEPTH ? 0 : stage + 1;
        }
    } else if constexpr (SETS == 2) {
        begin(0, 0, 0);
        begin(1, 1, 1);
        put(0, 0);
        begin(2, 0, 0);
        for (int from = 0; from < turns; from += 2)
#pragma unroll
            for (int set = 0; set < 2; ++set) {
                const int i = from + set;
                if (set > 0 && i >= turns) break;
                if (i * 4 + wave < slabs) compute(i * 4 + wave, set);
                put(1 - set, 1 - set);
                begin(i + 3, 1 - set, 1 - set);
            }
    } else {
        begin(0, 0, 0);
        loads_done();
        put(0, 0);
        for (int i = 0; i < turns; ++i) {
            lds_done();
            begin(i + 1, (i + 1) & 1, 0);
            asm volatile("" ::: "memory");
            if (i * 4 + wave < slabs) compute(i * 4 + wave, i & 1);
            loads_done();
            put((i + 1) & 1, 0);
        }
    }
    loads_done();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PB; ++i)
#pragma unroll
        for (int h = 0; h < QB; ++h)
#pragma unroll
            for (int v = 0; v < 4; ++v)
                *(mf32x4*)(s_mem + ((((wave * PB + i) * QB + h) * 4 + v) * 64 + lane) * 16) =
                    mf32x4{acc[i][h][v * 4], acc[i][h][v * 4 + 1], acc[i][h][v * 4 + 2], acc[i][h][v * 4 + 3]};
    __syncthreads();
    // wave w finishes the w-th four of every eight columns
    auto sum = [&](int i, int h, float (&t)[4]) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const mf32x4 x = *(const mf32x4*)(s_mem + ((((w * PB + i) * QB + h) * 4 + wave) * 64 + lane) * 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = w == 0 ? x[e] : t[e] + x[e];
        }
    };
#pragma unroll
    for (int h = 0; h < QB; ++h)
#pragma unroll
        for (int i = 0; i < (S::GATED ? PB / 2 : PB); ++i) {
            float v[4], u[4];
            sum(i, h, v);
            sum(S::GATED ? i + PB / 2 : i, h, u);
            finish_run<DT, S::GATED, false>(a, at.product, m0 + h * 32 + j, n0 + block_of(i) * 32 + wave * 8 + g * 4, v, u);
        }
}

// Contractions of less than 16 bytes: four columns of a row a thread, element by element
template <int DT, bool GATED>
__global__ void __launch_bounds__(256) matmul_short_kernel(const FeedArgs a) {
    auto element = [](const char* p, int64_t i) -> float {
        if constexpr (DT == FEED_F32) return ((const float*)p)[i];
        else if constexpr (DT == FEED_BF16) return __uint_as_float((uint32_t)((const uint16_t*)p)[i] << 16);
        else return __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)p)[i], 0);
    };
    const int64_t fours = (a.N + 3) / 4;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < a.M * fours; t += (int64_t)gridDim.x * 256) {
        const int64_t m = t / fours, n = t % fours * 4;
        float sum[2][4];
#pragma unroll
        for (int h = 0; h < (GATED ? 2 : 1); ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                float x = 0.f;
                if (n + e < a.N)
                    for (int64_t i = 0; i < a.q[0].k; ++i)
                        x = __builtin_fmaf(element(a.q[0].base + m * a.q[0].ld, i), element(a.p[h].base + (n + e) * a.p[h].ld, i), x);
                if (feed_size(DT) == 1 && n + e < a.N) x *= a.q_scale[m] * a.p_scale[h][(n + e) / kScaleBlock];
                sum[h][e] = x;
            }
        finish_run<DT, GATED, false>(a, 0, m, n, sum[0], sum[GATED ? 1 : 0]);
    }
}

// One launch of a kernel whose workgroups own S::BM x S::COLS of Out
template <class S>
static int launch_tiles(void (*kernel)(const FeedArgs), OncePerDevice& once, FeedArgs a, int threads, void* stream) {
    if constexpr (S::LDS > 64 * 1024) {
        int device = -1;
        if (hipGetDevice(&device) != hipSuccess || !once(device, [&] {
                return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024) == hipSuccess;
            })) {
            (void)hipGetLastError();
            return 1;
        }
    }
    a.tiles_m = (int32_t)((a.M + S::BM - 1) / S::BM);
    // (a gradient's columns go on to the end of its rows in the workspace)
    a.tiles_n = (int32_t)(((S::GATED && a.grad_out ? a.grad_cols : a.N) + S::COLS - 1) / S::COLS);
    a.n_tiles = a.tiles_m * a.tiles_n * a.products;
    hipLaunchKernelGGL(kernel, dim3(a.n_tiles), dim3(threads), S::LDS, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}
// Whether kernel KERNEL's workgroups are what its choice takes them for
template <int KERNEL, int DT, int FORM, class S>
constexpr bool as_chosen(int threads) {
    return matmul_tile(KERNEL, FORM, DT).rows == S::BM && matmul_tile(KERNEL, FORM, DT).cols == S::COLS && matmul_tile(KERNEL, FORM, DT).threads == threads;
}
template <int KERNEL, int DT, int FORM, int QB, int PB, int WM, int WN, int SLAB, int STAGES, bool QD, bool PD>
static int launch_block(const FeedArgs& a, void* stream) {
    static_assert(as_chosen<KERNEL, DT, FORM, BlockShape<DT, FORM, QB, PB, WM, WN, SLAB, STAGES>>(WM * WN * 64), "the tile in cacnn_feed.h");
    static OncePerDevice once;
    return launch_tiles<BlockShape<DT, FORM, QB, PB, WM, WN, SLAB, STAGES>>(matmul_block_kernel<DT, FORM, QB, PB, WM, WN, SLAB, STAGES, QD, PD>, once, a,
                                                                            WM * WN * 64, stream);
}
template <int KERNEL, int DT, int FORM, int QB, int PB, bool QD, bool PD>
static int launch_waves(const FeedArgs& a, void* stream) {
    static_assert(as_chosen<KERNEL, DT, FORM, WaveShape<DT, FORM, QB, PB>>(256), "the tile in cacnn_feed.h");
    static OncePerDevice once;
    return launch_tiles<WaveShape<DT, FORM, QB, PB>>(matmul_waves_kernel<DT, FORM, QB, PB, QD, PD>, once, a, 256, stream);
}

// Whether an operand can go straight to LDS
static bool direct(const FeedOperand& o, int size, bool strided) {
    return reinterpret_cast<uintptr_t>(o.base) % 16 == 0 && o.ld % 16 == 0 && (o.padded || (strided ? o.rows : o.k) * size % 16 == 0);
}
template <int DT, int FORM, bool QD, bool PD>
static int launch_shape(const FeedArgs& a, void* stream) {
    constexpr bool DIRECT = QD && PD;
    constexpr int HALF = FORM == FEED_GATED ? 2 : 1;
    const int kernel = matmul_kernel(a, FORM, DT, DIRECT);
    if (kernel == MATMUL_WAVES_32) return launch_waves<MATMUL_WAVES_32, DT, FORM, 1, HALF, QD, PD>(a, stream);
    if (kernel == MATMUL_WAVES_64_32) return launch_waves<MATMUL_WAVES_64_32, DT, FORM, 2, HALF, QD, PD>(a, stream);
    if constexpr (FORM != FEED_GATED)
        if (kernel == MATMUL_WAVES_64) return launch_waves<MATMUL_WAVES_64, DT, FORM, 2, 2, QD, PD>(a, stream);
    // (two waves to a SIMD where one workgroup has the compute unit: bf16 gated (777, 1008, 1515) 15.3 -> 14.0 us, (512, 2048, 2048) 24.4 -> 23.0; the 8-bit
    // instructions then have a block of rows each for the columns' operands read from LDS, (1024, 4096, 4096) 32 -> 39)
    if constexpr (DIRECT && feed_size(DT) > 1)
        if (kernel == MATMUL_128_DEEP) return launch_block<MATMUL_128_DEEP, DT, FORM, 1, 2, 4, 2, 128, 4, QD, PD>(a, stream);
    if constexpr (DIRECT && feed_size(DT) == 1)
        if (kernel == MATMUL_128_DEEP) return launch_block<MATMUL_128_DEEP, DT, FORM, 2, 2, 2, 2, 128, 4, QD, PD>(a, stream);
    if constexpr (DIRECT && DT == FEED_BF16)
        if (kernel == MATMUL_256) return launch_block<MATMUL_256, DT, FORM, 4, 2, 2, 4, 64, 4, QD, PD>(a, stream);
    if constexpr (DIRECT && DT == FEED_E4M3)
        if (kernel == MATMUL_256) return launch_block<MATMUL_256, DT, FORM, 4, 2, 2, 4, 128, 2, QD, PD>(a, stream);
    if constexpr (DT == FEED_F32)
        if (kernel == MATMUL_64_128) return launch_block<MATMUL_64_128, DT, FORM, 1, 2, 2, 2, 128, 2, QD, PD>(a, stream);
    return launch_block<MATMUL_128, DT, FORM, 2, 2, 2, 2, 128, 2, QD, PD>(a, stream);
}
template <int DT, int FORM>
static int launch_form(const FeedArgs& a, void* stream) {
    constexpr bool Q_STRIDED = FORM == FEED_BOTH, P_STRIDED = FORM >= FEED_RIGHT;
    const int size = feed_size(DT);
    constexpr bool TWO = FORM == FEED_GATED || FORM == FEED_RIGHT;
    if constexpr (FORM == FEED_GATED || FORM == FEED_PLAIN)
        if (a.q[0].k * size < 16 && !a.q[0].padded) {
            const int64_t grid = (a.M * ((a.N + 3) / 4) + 255) / 256;
            hipLaunchKernelGGL((matmul_short_kernel<DT, FORM == FEED_GATED>), dim3((uint32_t)(grid < (1 << 22) ? grid : 1 << 22)), dim3(256), 0, (hipStream_t)stream, a);
            return hipGetLastError() == hipSuccess ? 0 : 1;
        }
    const bool q = direct(a.q[0], size, Q_STRIDED), p = direct(a.p[0], size, P_STRIDED) && (!TWO || direct(a.p[1], size, P_STRIDED));
    if constexpr (FORM >= FEED_RIGHT) return p ? launch_shape<DT, FORM, true, true>(a, stream) : launch_shape<DT, FORM, true, false>(a, stream);
    else return q && p ? launch_shape<DT, FORM, true, true>(a, stream) : launch_shape<DT, FORM, false, false>(a, stream);
}
template <int DT>
static int launch_type(const FeedArgs& a, int form, void* stream) {
    if constexpr (feed_size(DT) == 1) {
        return form == FEED_GATED ? launch_form<DT, FEED_GATED>(a, stream) : launch_form<DT, FEED_PLAIN>(a, stream);
    } else {
        if (form == FEED_GATED) return launch_form<DT, FEED_GATED>(a, stream);
        if (form == FEED_RIGHT) return launch_form<DT, FEED_RIGHT>(a, stream);
        return launch_form<DT, FEED_BOTH>(a, stream);
    }
}

int launch_matmul(const FeedArgs& a, int form, int dtype, void* stream) {
    if (dtype == FEED_F32) return launch_type<FEED_F32>(a, form, stream);
    if (dtype == FEED_BF16) return launch_type<FEED_BF16>(a, form, stream);
    if (a.out[0].size == 2) return launch_type<FEED_E4M3>(a, form, stream);
    return launch_type<FEED_E4M3_EXACT>(a, form, stream);
}

}  // namespace cacnn
