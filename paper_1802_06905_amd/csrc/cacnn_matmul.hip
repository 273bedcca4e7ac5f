// Matrix products of the feed-forward operators for gfx950: Out[m][n] = sum over k of Q(m, k) P(n, k), in bf16, fp32 and 8-bit floats with a
// scale for each block of 128, as they are or two at a time with the activation and the product of the gated projection behind them.
//
// Out's rows m are tokens (or, for a weight's gradient, the weight's rows), its columns n channels or features.  An MFMA takes 32 columns
// as its first operand and 32 rows as its second, so a lane ends up with one row m and runs of four adjacent columns, which
// leave in one store each, and the scale of a row in 8 bits is one number per lane.
//
// A workgroup owns BM x BN of Out and walks the contraction in slabs of 128 bytes a row, which are staged in LDS, two at a time.
//   contraction contiguous ([row][k]): LDS keeps rows of 128 bytes; the 16-byte chunk c of row r lies at c ^ (r & 7), so that the eight lanes of
//     an LDS access, eight rows at the same chunk, meet all banks once.  A lane's chunk holds the 8 (bf16), 4 (fp32) or 16 (8 bits)
//     contraction indices that it feeds to the matrix instructions; which index goes to which half of a wave does not matter, because
//     both operands use the same assignment.
//   contraction strided ([k][row]): LDS keeps the rows of k as they lie in memory, in blocks of 64 bytes (bf16, read by the
//     transposing loads) or 128 (fp32, read word by word) that change places with k, for the same reason.
#include <hip/hip_runtime.h>
#include <stdint.h>

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
typedef __bf16 mbf16x8 __attribute__((ext_vector_type(8)));
#define MAT_LDS(T) __attribute__((address_space(3))) T
#define MAT_CONST(T) __attribute__((address_space(4))) const T
// 16 bytes at any address
struct __attribute__((packed, aligned(1))) MatBytes16 {
    mu32x4 v;
};

constexpr int kSlab = 128;   // bytes of a row and slab

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
template <int ESZ, bool STRIDED, int ROWS, int WAVES>
struct SlabMap {
    static constexpr int N = ROWS * kSlab / 1024 / WAVES, KR = kSlab / ESZ, LANES = ROWS * ESZ / 16;   // pieces a lane; indices a slab; lanes a strided row
    static_assert(N >= 1 && N * WAVES * 1024 == ROWS * kSlab, "a slab is whole wave loads");
    // contiguous: row and byte of the slab's row
    static __device__ __forceinline__ int row(int i, int wave, int lane) { return (i * WAVES + wave) * 8 + (lane >> 3); }
    static __device__ __forceinline__ int byte(int lane) { return ((lane & 7) ^ (lane >> 3)) * 16; }
    // strided: contraction index within the slab, and byte of that row
    static __device__ __forceinline__ int index(int i, int wave, int lane) { return (i * WAVES + wave) * (64 / LANES) + lane / LANES; }
    static __device__ __forceinline__ int column(int i, int wave, int lane) {
        constexpr int PIECES = ESZ == 4 ? 8 : 4;                                  // of 16 bytes in a block
        const int at = lane % LANES, k = index(i, wave, lane);
        return (at / PIECES ^ strided_turn<ESZ, ROWS>(k)) * (PIECES * 16) + at % PIECES * 16;
    }
};

// Brings slabs to LDS through registers, from any address and of any size: whole 16 bytes where the array has them, else element by element
// with zeros behind its end.
template <int ESZ, bool STRIDED, int ROWS, int WAVES>
struct RegisterLoader {
    using Map = SlabMap<ESZ, STRIDED, ROWS, WAVES>;
    const char* base;
    int64_t ld, k, k0;
    int rows, wave, lane;
    mu32x4 r[Map::N];

    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave_, int lane_) {
        ld = o.ld, k = o.k, wave = wave_, lane = lane_;
        base = o.base + (STRIDED ? row0 * ESZ : row0 * ld);
        rows = (int)max((int64_t)0, min((int64_t)ROWS, o.rows - row0));
    }
    // slab s of the operand (none if !any: zeros)
    __device__ __forceinline__ void load(int64_t s, bool any) {
#pragma unroll
        for (int i = 0; i < Map::N; ++i) {
            const char* p;
            int64_t left;                                                         // bytes from p on that belong to the operand
            if constexpr (STRIDED) {
                const int64_t at = s * Map::KR + Map::index(i, wave, lane);
                const int col = Map::column(i, wave, lane);
                p = base + at * ld + col;
                left = any && at < k ? (int64_t)rows * ESZ - col : 0;
            } else {
                const int row = Map::row(i, wave, lane);
                const int64_t at = s * kSlab + Map::byte(lane);
                p = base + row * ld + at;
                left = any && row < rows ? k * ESZ - at : 0;
            }
            mu32x4 v = {0, 0, 0, 0};
            if (left >= 16) {
                v = ((const MatBytes16*)p)->v;
            } else if (left > 0) {
#pragma unroll
                for (int e = 0; e < 16 / ESZ; ++e)
                    if (e * ESZ < left) {
                        uint32_t x;
                        if constexpr (ESZ == 4) x = *(const uint32_t*)(p + e * 4);
                        else if constexpr (ESZ == 2) x = *(const uint16_t*)(p + e * 2);
                        else x = *(const uint8_t*)(p + e);
                        v[e * ESZ / 4] |= x << (e * ESZ % 4 * 8);
                    }
            }
            r[i] = v;
        }
    }
    __device__ __forceinline__ void put(char* slab) {
#pragma unroll
        for (int i = 0; i < Map::N; ++i) *(mu32x4*)(slab + (i * WAVES + wave) * 1024 + lane * 16) = r[i];
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
template <int ESZ, bool STRIDED, int ROWS, int WAVES>
struct DirectLoader {
    using Map = SlabMap<ESZ, STRIDED, ROWS, WAVES>;
    const char* base;
    int64_t ld, k;
    int bytes;                     // contiguous: of a row; strided: of a row of the tile; whole pieces of 16
    int byte, wave;
    i32x4 d;
    uint32_t off[Map::N];

    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave_, int lane) {
        wave = wave_, ld = o.ld, k = o.k;
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
            byte = Map::byte(lane);
            d = bytes_from(base, rows ? (int64_t)(rows - 1) * ld + bytes : 0);
#pragma unroll
            for (int i = 0; i < Map::N; ++i) {
                const int row = Map::row(i, wave, lane);
                off[i] = row < rows ? (uint32_t)row * (uint32_t)ld + byte : kOutside;
            }
        }
    }
    // another array of the same shape
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) {
        base = o.base + (STRIDED ? row0 * ESZ : row0 * ld);
        if constexpr (!STRIDED) d = bytes_from(base, (uint32_t)d[2]);
    }
    // slab s (none if !any: zeros) to LDS bytes `slab`
    __device__ __forceinline__ void issue(int s, bool any, uint32_t slab) {
        uint32_t more = 0;
        if constexpr (STRIDED) {
            const int64_t at = (int64_t)s * Map::KR;
            const int64_t left = any ? min(k - at, (int64_t)Map::KR) : 0;
            d = bytes_from(base + at * ld, left > 0 ? (left - 1) * ld + bytes : 0);
        } else {
            more = any && s * kSlab + byte < bytes ? s * kSlab : kOutside;
        }
#pragma unroll
        for (int i = 0; i < Map::N; ++i) load_to_lds_unseen(d, off[i] + more, slab + (i * WAVES + wave) * 1024);
    }
};
__device__ __forceinline__ uint32_t lds_address(const char* p) { return (uint32_t)(uintptr_t)(MAT_LDS(const char)*)p; }
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void lds_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// One operand's way to LDS
template <int ESZ, bool STRIDED, int ROWS, int WAVES, bool DIRECT>
struct Loader {
    static constexpr bool direct = DIRECT;
    DirectLoader<ESZ, STRIDED, ROWS, WAVES> l;
    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave, int lane) { l.init(o, row0, wave, lane); }
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) { l.move(o, row0); }
    // begins to bring slab s, to `slab`: now, or with put() after the loads have come
    __device__ __forceinline__ void begin(int s, bool any, char* slab) { l.issue(s, any, lds_address(slab)); }
    __device__ __forceinline__ void put(char*) {}
};
template <int ESZ, bool STRIDED, int ROWS, int WAVES>
struct Loader<ESZ, STRIDED, ROWS, WAVES, false> {
    static constexpr bool direct = false;
    RegisterLoader<ESZ, STRIDED, ROWS, WAVES> l;
    __device__ __forceinline__ void init(const FeedOperand& o, int64_t row0, int wave, int lane) { l.init(o, row0, wave, lane); }
    __device__ __forceinline__ void move(const FeedOperand& o, int64_t row0) { l.base = o.base + (STRIDED ? row0 * ESZ : row0 * l.ld); }
    __device__ __forceinline__ void begin(int s, bool any, char*) { l.load(s, any); }
    __device__ __forceinline__ void put(char* slab) { l.put(slab); }
};

// A block of 32 rows (or columns) of step `st` of a slab, as the matrix instructions take it: 16 bytes a lane
template <int ESZ, bool STRIDED, int ROWS>
__device__ __forceinline__ mu32x4 read_block(const char* slab, int block, int st, int lane) {
    const int j = lane & 31, g = lane >> 5;
    if constexpr (!STRIDED) {
        return *(const mu32x4*)(slab + (block * 32 + j) * kSlab + (((2 * st + g) ^ (j & 7)) * 16));
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

// Columns n .. n + 3 of row m, those below `cols`
template <int DT>
__device__ __forceinline__ void store_four(const FeedOut& o, int64_t m, int64_t n, int64_t cols, mf32x4 v) {
    constexpr bool words = DT == FEED_F32 || DT == FEED_E4M3_EXACT;
    char* const p = o.base + m * o.ld + n * (words ? 4 : 2);
    const mu32x2 packed = {two_bf16(v[0], v[1]), two_bf16(v[2], v[3])};
    if (o.wide && n + 4 <= cols) {
        if (words) *(mf32x4*)p = v;
        else *(mu32x2*)p = packed;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < cols) {
                if (words) ((float*)p)[e] = v[e];
                else ((uint16_t*)p)[e] = (uint16_t)(packed[e / 2] >> (e % 2 * 16));
            }
    }
}

// What is done with four adjacent columns of a row: sums of the plain products, or of gate and up
template <int DT, bool GATED>
__device__ __forceinline__ void finish_four(const FeedArgs& a, int product, int64_t m, int64_t n, mf32x4 v, mf32x4 u) {
    if (m >= a.M) return;
    if constexpr (!GATED) {
        store_four<DT>(a.out[product], m, n, a.N, v);
    } else if (feed_size(DT) > 1 && a.grad_out) {
        if (n >= a.grad_cols) return;
        mf32x4 d = {0.f, 0.f, 0.f, 0.f};
        const char* const p = a.grad_out + m * a.grad_out_ld + n * feed_size(DT);
        if (a.grad_out_wide && n + 4 <= a.N) {
            if constexpr (DT == FEED_F32) {
                d = *(const mf32x4*)p;
            } else {
                const mu32x2 w = *(const mu32x2*)p;
                d = mf32x4{__uint_as_float(w[0] << 16), __uint_as_float(w[0] & 0xffff0000u), __uint_as_float(w[1] << 16), __uint_as_float(w[1] & 0xffff0000u)};
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n + e < a.N) d[e] = DT == FEED_F32 ? ((const float*)p)[e] : __uint_as_float((uint32_t)((const uint16_t*)p)[e] << 16);
        }
        mf32x4 dg, du;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float g = 0.f, h = 0.f;
            if (n + e < a.N) gate_grad(a.activation, v[e], u[e], d[e], g, h);
            dg[e] = g, du[e] = h;
        }
        store_four<DT>(a.out[0], m, n, a.grad_cols, dg);
        store_four<DT>(a.out[1], m, n, a.grad_cols, du);
    } else {
        mf32x4 h;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = gate_value(a.activation, v[e]) * u[e];
        store_four<DT>(a.out[0], m, n, a.N, h);
        if (a.gate_out.base) store_four<DT>(a.gate_out, m, n, a.N, v);
        if (a.up_out.base) store_four<DT>(a.up_out, m, n, a.N, u);
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
template <int DT, int FORM, int QB, int PB, int WM, int WN>
struct BlockShape {
    static constexpr int ESZ = feed_size(DT), WAVES = WM * WN, BM = WM * QB * 32, BN = WN * PB * 32;
    static constexpr bool GATED = FORM == FEED_GATED, Q_STRIDED = FORM == FEED_BOTH, P_STRIDED = FORM >= FEED_RIGHT;
    static constexpr int COLS = GATED ? BN / 2 : BN;                    // of Out
    static constexpr int P_PARTS = GATED ? 2 : 1, P_ROWS = BN / P_PARTS;
    static constexpr int Q_BYTES = BM * kSlab, P_BYTES = BN * kSlab, SCALES = ESZ == 1 ? BM * 4 : 0;
    static constexpr int STAGE = Q_BYTES + P_BYTES + SCALES, LDS = 2 * STAGE;
};

// QD, PD: whether the operands go straight to LDS.
template <int DT, int FORM, int QB, int PB, int WM, int WN, bool QD, bool PD>
__global__ void __launch_bounds__(WM* WN * 64, WM* WN == 4 ? 2 : 1) matmul_block_kernel(const FeedArgs a) {
    using S = BlockShape<DT, FORM, QB, PB, WM, WN>;
    constexpr int ESZ = S::ESZ, WAVES = S::WAVES, KE = kSlab / ESZ;
    extern __shared__ __align__(16) char s_mem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM, j = lane & 31, g = lane >> 5;
    const TilePlace at = tile_place(a, blockIdx.x);
    const int64_t m0 = (int64_t)at.m * S::BM, n0 = (int64_t)at.n * S::COLS;

    Loader<ESZ, S::Q_STRIDED, S::BM, WAVES, QD> q;
    Loader<ESZ, S::P_STRIDED, S::P_ROWS, WAVES, PD> p[S::P_PARTS];
    q.init(a.q[at.product], m0, wave, lane);
#pragma unroll
    for (int h = 0; h < S::P_PARTS; ++h) p[h].init(a.p[h], n0, wave, lane);
    const int per_segment = (int)((a.q[0].k + KE - 1) / KE), slabs = max(1, per_segment * a.segments);
    // 8 bits: the scales of a slab's rows, a word each, brought by as many waves as they fill (rows behind the last: zeros)
    const bool brings_scales = ESZ == 1 && wave * 64 < S::BM;
    const i32x4 scales = ESZ == 1 ? bytes_from((const char*)(a.q_scale + m0 * a.scale_cols), min((int64_t)S::BM, a.M - m0) * a.scale_cols * 4) : i32x4{0, 0, 0, 0};
    const uint32_t scale_off = (uint32_t)threadIdx.x * a.scale_cols * 4;
    // Slab s on its way to its half of LDS, and there
    auto begin = [&](int s) {
        char* const stage = s_mem + (s & 1) * S::STAGE;
        int i = s;
        if constexpr (FORM == FEED_RIGHT)
            if (s >= per_segment && a.segments > 1) {
                i = s - per_segment;
                q.move(a.q[1], m0);
                p[0].move(a.p[1], n0);
            }
        const bool any = i < per_segment;
        q.begin(i, any, stage);
#pragma unroll
        for (int h = 0; h < S::P_PARTS; ++h) p[h].begin(i, any, stage + S::Q_BYTES + h * S::P_ROWS * kSlab);
        if constexpr (ESZ == 1)
            if (brings_scales) load_word_to_lds_unseen(scales, scale_off + i * 4, lds_address(stage + S::Q_BYTES + S::P_BYTES + wave * 256));
    };
    auto put = [&](int s) {
        char* const stage = s_mem + (s & 1) * S::STAGE;
        q.put(stage);
#pragma unroll
        for (int h = 0; h < S::P_PARTS; ++h) p[h].put(stage + S::Q_BYTES + h * S::P_ROWS * kSlab);
    };
    // a wave's i-th block of columns: part of p, block within it
    auto part_of = [&](int i) { return S::GATED ? i / (PB / 2) : 0; };
    auto block_of = [&](int i) { return S::GATED ? wn * (PB / 2) + i % (PB / 2) : wn * PB + i; };
    auto q_slab = [&](int s) -> const char* { return s_mem + (s & 1) * S::STAGE; };
    auto p_slab = [&](int s, int i) -> const char* { return s_mem + (s & 1) * S::STAGE + S::Q_BYTES + part_of(i) * S::P_ROWS * kSlab; };
    // This wave has read what it needs of slab s - 1, and slab s is there for all; the buffer of slab s - 1 takes slab s + 1
    auto next = [&](int s) {
        loads_done();
        put(s);
        lds_done();
        __builtin_amdgcn_s_barrier();
        if (s + 1 < slabs) begin(s + 1);
        asm volatile("" ::: "memory");
    };

    mf32x16 acc[PB][QB];
#pragma unroll
    for (int i = 0; i < PB; ++i)
#pragma unroll
        for (int h = 0; h < QB; ++h)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][h][v] = 0.f;

    begin(0);
    next(0);
    if constexpr (ESZ > 1) {
        // The operands of a step are read under the products of the step before, across slabs too
        mu32x4 pv[2][PB], qv[2][QB];
        auto read = [&](int s, int st, int set) {
#pragma unroll
            for (int i = 0; i < PB; ++i) pv[set][i] = read_block<ESZ, S::P_STRIDED, S::P_ROWS>(p_slab(s, i), block_of(i), st, lane);
#pragma unroll
            for (int h = 0; h < QB; ++h) qv[set][h] = read_block<ESZ, S::Q_STRIDED, S::BM>(q_slab(s), wm * QB + h, st, lane);
            __builtin_amdgcn_sched_barrier(0);
        };
        auto products = [&](int set) {
#pragma unroll
            for (int i = 0; i < PB; ++i)
#pragma unroll
                for (int h = 0; h < QB; ++h) multiply<DT>(acc[i][h], pv[set][i], qv[set][h]);
            __builtin_amdgcn_sched_barrier(0);
        };
        read(0, 0, 0);
        for (int s = 0; s < slabs; ++s) {
            read(s, 1, 1);
            products(0);
            read(s, 2, 0);
            products(1);
            read(s, 3, 1);
            products(0);
            if (s + 1 < slabs) {
                next(s + 1);
                read(s + 1, 0, 0);
            }
            products(1);
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
            for (int h = 0; h < QB; ++h) sq[h] = *(const float*)(q_slab(s) + S::Q_BYTES + S::P_BYTES + ((wm * QB + h) * 32 + j) * 4);
            auto add = [&](int i, int h, const mf32x16& c) {
                const float f = sp[i] * sq[h];
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][h][v] = __builtin_fmaf(c[v], f, acc[i][h][v]);
                // (here and now: the compiler puts all of them off to the end of the slab, with a register for every product until then)
                asm volatile("" : "+v"(acc[i][h]));
            };
            if constexpr (DT == FEED_E4M3) {
                // (one address for each of the four chunks and operand, the blocks at constant distances: more and the sums spill)
                const uint32_t qa = lds_address(q_slab(s)) + (wm * QB * 32 + j) * kSlab, pa = lds_address(q_slab(s)) + S::Q_BYTES + (block_of(0) * 32 + j) * kSlab;
                uint32_t chunk[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) chunk[x] = ((2 * x + g) ^ (j & 7)) * 16;
                auto chunk_at = [](uint32_t at, int more) { return *(MAT_LDS(const mu32x4)*)((MAT_LDS(const char)*)(uintptr_t)at + more); };
                mu32x4 pv[PB][2][2], qv[2][2];
                auto read_q = [&](int h) {
#pragma unroll
                    for (int x = 0; x < 4; ++x) qv[x / 2][x % 2] = chunk_at(qa + chunk[x], h * 32 * kSlab);
                };
#pragma unroll
                for (int i = 0; i < PB; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        pv[i][x / 2][x % 2] = chunk_at(pa + chunk[x], (part_of(i) * S::P_ROWS + (block_of(i) - block_of(0)) * 32) * kSlab);
                read_q(0);
#pragma unroll
                for (int h = 0; h < QB; ++h) {
                    if (h + 1 == QB && s + 1 < slabs) next(s + 1);
                    mf32x16 c[PB];
#pragma unroll
                    for (int i = 0; i < PB; ++i) {
#pragma unroll
                        for (int v = 0; v < 16; ++v) c[i][v] = 0.f;
                        c[i] = multiply_e4m3(multiply_e4m3(c[i], pv[i][0], qv[0]), pv[i][1], qv[1]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (h + 1 < QB) read_q(h + 1);
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
                    for (int i = 0; i < PB; ++i) pv[i] = read_block<1, false, S::P_ROWS>(p_slab(s, i), block_of(i), x, lane);
#pragma unroll
                    for (int h = 0; h < QB; ++h) qv[h] = read_block<1, false, S::BM>(q_slab(s), wm * QB + h, x, lane);
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
                if (s + 1 < slabs) next(s + 1);
            }
        }
    }

#pragma unroll
    for (int h = 0; h < QB; ++h) {
        const int64_t m = m0 + (wm * QB + h) * 32 + j;
#pragma unroll
        for (int i = 0; i < (S::GATED ? PB / 2 : PB); ++i)
#pragma unroll
            for (int v = 0; v < 16; v += 4) {
                const int64_t n = n0 + block_of(i) * 32 + v * 2 + g * 4;
                const mf32x16 &x = acc[i][h], &y = acc[S::GATED ? i + PB / 2 : i][h];
                finish_four<DT, S::GATED>(a, at.product, m, n, mf32x4{x[v], x[v + 1], x[v + 2], x[v + 3]}, mf32x4{y[v], y[v + 1], y[v + 2], y[v + 3]});
            }
    }
}

template <int DT, int FORM, int QB, int PB, int WM, int WN, bool QD, bool PD>
static int launch_block(FeedArgs a, void* stream) {
    using S = BlockShape<DT, FORM, QB, PB, WM, WN>;
    auto kernel = matmul_block_kernel<DT, FORM, QB, PB, WM, WN, QD, PD>;
    if constexpr (S::LDS > 64 * 1024) {
        static OncePerDevice once;
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
    hipLaunchKernelGGL(kernel, dim3(a.n_tiles), dim3(S::WAVES * 64), S::LDS, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

// Whether an operand can go straight to LDS
static bool direct(const FeedOperand& o, int size, bool strided) {
    return reinterpret_cast<uintptr_t>(o.base) % 16 == 0 && o.ld % 16 == 0 && (o.padded || (strided ? o.rows : o.k) * size % 16 == 0);
}
static int64_t tiles(const FeedArgs& a, int64_t rows, int64_t cols) { return (a.M + rows - 1) / rows * ((a.N + cols - 1) / cols) * a.products; }

template <int DT, int FORM, bool QD, bool PD>
static int launch_shape(const FeedArgs& a, void* stream) {
    constexpr bool LARGE = QD && PD && (DT == FEED_BF16 || DT == FEED_E4M3);
    if constexpr (LARGE)
        if (tiles(a, 256, FORM == FEED_GATED ? 128 : 256) >= 192) return launch_block<DT, FORM, 4, 2, 2, 4, QD, PD>(a, stream);
    return launch_block<DT, FORM, 2, 2, 2, 2, QD, PD>(a, stream);
}
template <int DT, int FORM>
static int launch_form(const FeedArgs& a, void* stream) {
    constexpr bool Q_STRIDED = FORM == FEED_BOTH, P_STRIDED = FORM >= FEED_RIGHT;
    const int size = feed_size(DT);
    const bool q = direct(a.q[0], size, Q_STRIDED), p = direct(a.p[0], size, P_STRIDED) && (FORM != FEED_GATED && FORM != FEED_RIGHT || direct(a.p[1], size, P_STRIDED));
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
