// The feed-forward operators' elementwise kernels for gfx950: quantisation to 8-bit floats with a scale for each block of 128, and the
// gradients of the gated projection's two products.  Every input is read once and every result written once: bound by memory.
// Measured on the device: an fp32 weight of 8192 x 4096 in blocks of 128 x 128 28 us, 6.0 TB/s of 168 MB; one token of 4096 bf16 2.5 us, the least a launch
// takes; gradients of gate and up, 8192 x 8192 bf16, 112 us, 6.0 TB/s of 671 MB.  A call of 8192 tokens, bf16: of 4096 channels 20.8 us, 4.8 TB/s of 102 MB; of 512, 10.0, and
// of 128, 9.4: a workgroup to a token, of which 64 and 16 of 256 threads have something to do.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cacnn_feed.h"
#include "cacnn_gate.h"

namespace cacnn {

typedef unsigned int eu32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int eu32x4 __attribute__((ext_vector_type(4)));
// 16 and 8 bytes at any address: the memory takes them in one access, over two lines where they lie so
struct __attribute__((packed, aligned(1))) FeedBytes16 {
    eu32x4 v;
};
struct __attribute__((packed, aligned(1))) FeedBytes8 {
    eu32x2 v;
};

// ---- quantisation
// A block's scale is the smallest power of two, from 2^-126 on, by which its largest finite magnitude a is at most 448, the largest number
// in 8 bits (four of exponent, three of fraction): a power of two, so that dividing by it is exact and the rounding to 8 bits, half a step or 2^-4 of
// the value, is the only one.  a = 1.f x 2^n: 448 = 1.75 x 2^8, so the power is n - 8, and one more where 1.f > 1.75.
__device__ __forceinline__ int scale_power(uint32_t largest_bits) {
    const int e = (int)(largest_bits >> 23) - 127 - 8 + ((largest_bits & 0x7fffffu) > 0x600000u);
    return largest_bits ? max(e, -126) : 0;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ uint32_t finite_magnitude(float x) {
    const uint32_t b = __float_as_uint(x) & 0x7fffffffu;
    return b < 0x7f800000u ? b : 0u;
}

// Eight adjacent elements of a row
template <int DT>
struct Eight {
    uint32_t w[DT == FEED_F32 ? 8 : 4];
    __device__ __forceinline__ float at(int i) const {
        if constexpr (DT == FEED_F32) return __uint_as_float(w[i]);
        else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
    // the first n of them, zeros behind
    __device__ __forceinline__ void load(const char* p, int n) {
        if (n >= 8) {
#pragma unroll
            for (int i = 0; i < (DT == FEED_F32 ? 2 : 1); ++i) {
                const eu32x4 v = ((const FeedBytes16*)p)[i].v;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[i * 4 + e] = v[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t x = 0;
                if (i < n) x = DT == FEED_F32 ? ((const uint32_t*)p)[i] : ((const uint16_t*)p)[i];
                if constexpr (DT == FEED_F32) w[i] = x;
                else w[i / 2] = i & 1 ? w[i / 2] | x << 16 : x;
            }
        }
    }
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t a = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, finite_magnitude(at(i)));
        return a;
    }
    // in 8 bits, times 2^-e; infinities and NaN as NaN
    __device__ __forceinline__ eu32x2 quantized(int e) const {
        const float f = power_of_two(-e);
        eu32x2 q;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            int v = 0;
            v = __builtin_amdgcn_cvt_pk_fp8_f32(at(i * 4) * f, at(i * 4 + 1) * f, v, false);
            v = __builtin_amdgcn_cvt_pk_fp8_f32(at(i * 4 + 2) * f, at(i * 4 + 3) * f, v, true);
#pragma unroll
            for (int b = 0; b < 4; ++b)
                if ((__float_as_uint(at(i * 4 + b)) & 0x7f800000u) == 0x7f800000u) v |= 0x7f << (b * 8);
            q[i] = (uint32_t)v;
        }
        return q;
    }
};

__device__ __forceinline__ void store_eight(uint8_t* p, int n, eu32x2 q) {
    if (n >= 8) {
        ((FeedBytes8*)p)->v = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (uint8_t)(q[i / 4] >> (i % 4 * 8));
    }
}

// Blocks of 1 x 128: 16 lanes a block, 16 adjacent blocks of a row to a workgroup
template <int DT>
__global__ void __launch_bounds__(256) quantize_rows_kernel(const QuantizeArgs a) {
    const int col = (blockIdx.x * 16 + (threadIdx.x >> 4)) * kScaleBlock + (threadIdx.x & 15) * 8;
    const int n = (int)min((int64_t)8, a.C - col);
    for (int64_t t = blockIdx.y; t < a.T; t += gridDim.y) {
        Eight<DT> x;
        x.load(a.x + t * a.ld_x + (int64_t)col * feed_size(DT), n);
        uint32_t largest = x.largest();
#pragma unroll
        for (int d = 1; d < 16; d *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, d));
        const int e = scale_power(largest);
        if (n > 0) store_eight(a.q + t * a.ld_q + col, n, x.quantized(e));
        if ((threadIdx.x & 15) == 0 && n > 0) a.scale[t * a.blocks + col / kScaleBlock] = power_of_two(e);
    }
}

// Blocks of 128 x 128: a workgroup each, eight rows of eight elements to a thread
template <int DT>
__global__ void __launch_bounds__(256) quantize_blocks_kernel(const QuantizeArgs a) {
    __shared__ uint32_t s_largest[4];
    const int col = blockIdx.x * kScaleBlock + (threadIdx.x & 15) * 8, row = threadIdx.x >> 4;
    const int n = (int)min((int64_t)8, a.C - col);
    const int64_t row_blocks = (a.T + kScaleBlock - 1) / kScaleBlock;
    for (int64_t b = blockIdx.y; b < row_blocks; b += gridDim.y) {
        const int64_t t0 = b * kScaleBlock + row;
        Eight<DT> x[8];
        uint32_t largest = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i].load(a.x + (t0 + i * 16) * a.ld_x + (int64_t)col * feed_size(DT), t0 + i * 16 < a.T ? n : 0);
            largest = max(largest, x[i].largest());
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) largest = max(largest, (uint32_t)__shfl_xor((int)largest, d));
        if ((threadIdx.x & 63) == 0) s_largest[threadIdx.x >> 6] = largest;
        __syncthreads();
        const int e = scale_power(max(max(s_largest[0], s_largest[1]), max(s_largest[2], s_largest[3])));
        __syncthreads();
        if (threadIdx.x == 0) a.scale[b * a.blocks + blockIdx.x] = power_of_two(e);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (t0 + i * 16 < a.T && n > 0) store_eight(a.q + (t0 + i * 16) * a.ld_q + col, n, x[i].quantized(e));
    }
}

template <int DT>
static void launch_quantize_as(const QuantizeArgs& a, int block_rows, hipStream_t stream) {
    const int64_t rows = block_rows == 1 ? a.T : (a.T + kScaleBlock - 1) / kScaleBlock;
    const uint32_t y = (uint32_t)(rows < 65535 ? rows : 65535);
    if (block_rows == 1) hipLaunchKernelGGL(quantize_rows_kernel<DT>, dim3((a.blocks + 15) / 16, y), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL(quantize_blocks_kernel<DT>, dim3(a.blocks, y), dim3(256), 0, stream, a);
}

int launch_quantize(const QuantizeArgs& a, int dtype, int block_rows, void* stream) {
    if (dtype == FEED_F32) launch_quantize_as<FEED_F32>(a, block_rows, (hipStream_t)stream);
    else launch_quantize_as<FEED_BF16>(a, block_rows, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

// ---- gradients of gate and up from the values that the forward pass kept, eight columns a thread; columns from F to `cols`, the end of a row in the
// workspace, are written with zeros.  Rounded to the arrays' type, as operands of the matrix instructions: bf16 gradients are then 2.3e-3 of their norm off, where
// operands in fp32, at a tenth of the products' rate, would leave the 1.7e-3 of their own rounding
template <int DT>
__device__ __forceinline__ void gate_grad_piece(const GateArgs& a, int64_t t, int64_t col) {
    const int n = (int)max((int64_t)0, min((int64_t)8, a.F - col));
    Eight<DT> g, u, d;
    g.load(a.gate + t * a.ld_pre + col * feed_size(DT), n);
    u.load(a.up + t * a.ld_pre + col * feed_size(DT), n);
    d.load(a.grad_out + t * a.ld_out + col * feed_size(DT), n);
    uint32_t wg[8], wu[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float x = 0.f, y = 0.f;
        if (i < n) gate_grad(a.activation, g.at(i), u.at(i), d.at(i), x, y);
        if constexpr (DT == FEED_F32) {
            wg[i] = __float_as_uint(x), wu[i] = __float_as_uint(y);
        } else {
            const uint32_t bx = __builtin_bit_cast(uint16_t, (__bf16)x), by = __builtin_bit_cast(uint16_t, (__bf16)y);
            wg[i / 2] = i & 1 ? wg[i / 2] | bx << 16 : bx;
            wu[i / 2] = i & 1 ? wu[i / 2] | by << 16 : by;
        }
    }
    char* const pg = a.grad_gate + t * a.ld + col * feed_size(DT);
    char* const pu = a.grad_up + t * a.ld + col * feed_size(DT);
#pragma unroll
    for (int i = 0; i < (DT == FEED_F32 ? 2 : 1); ++i) {
        ((eu32x4*)pg)[i] = eu32x4{wg[i * 4], wg[i * 4 + 1], wg[i * 4 + 2], wg[i * 4 + 3]};
        ((eu32x4*)pu)[i] = eu32x4{wu[i * 4], wu[i * 4 + 1], wu[i * 4 + 2], wu[i * 4 + 3]};
    }
}

template <int DT>
__global__ void __launch_bounds__(256) gate_grad_kernel(const GateArgs a) {
    const uint32_t pieces = (uint32_t)(a.cols / 8);
    // (the 64-bit division is uniform; a thread's own is of 32 bits)
    for (uint64_t first = (uint64_t)blockIdx.x * 256; first < (uint64_t)a.T * pieces; first += (uint64_t)gridDim.x * 256) {
        const uint64_t row0 = first / pieces;
        const uint32_t in = (uint32_t)(first - row0 * pieces) + threadIdx.x;
        const int64_t t = (int64_t)(row0 + in / pieces);
        if (t < a.T) gate_grad_piece<DT>(a, t, (int64_t)(in % pieces) * 8);
    }
}

// The workgroups of `pieces` threads: those of a launch have to be below 2^32 threads, the others are walked
static uint32_t workgroups(int64_t pieces) { return (uint32_t)((pieces + 255) / 256 < (1 << 22) ? (pieces + 255) / 256 : 1 << 22); }

int launch_gate_grad(const GateArgs& a, int dtype, void* stream) {
    const dim3 grid(workgroups(a.T * (a.cols / 8)));
    if (dtype == FEED_F32) hipLaunchKernelGGL(gate_grad_kernel<FEED_F32>, grid, dim3(256), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(gate_grad_kernel<FEED_BF16>, grid, dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

// ---- arrays whose rows 16-byte loads cannot start with, to rows where they can: a piece of 16 bytes a thread
__device__ __forceinline__ void pad_piece(const PadArgs& a, int64_t row, int64_t at) {
    char* const to = a.to + row * a.ld + at;
    int i = 0;
    while (i < 3 && row >= a.rows[i]) row -= a.rows[i++];
    if (i == 3) return;                                      // (threads behind the last row)
    const char* const from = (i == 0 ? a.from[0] : i == 1 ? a.from[1] : a.from[2]) + row * (i == 0 ? a.ld_from[0] : i == 1 ? a.ld_from[1] : a.ld_from[2]) + at;
    eu32x4 v = {0, 0, 0, 0};
    if (at + 16 <= a.bytes) {
        v = ((const FeedBytes16*)from)->v;
    } else {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (a.size == 4) {
                if (at + w * 4 < a.bytes) v[w] = *(const uint32_t*)(from + w * 4);
            } else {
                if (at + w * 4 < a.bytes) v[w] = *(const uint16_t*)(from + w * 4);
                if (at + w * 4 + 2 < a.bytes) v[w] |= (uint32_t)*(const uint16_t*)(from + w * 4 + 2) << 16;
            }
        }
    }
    *(eu32x4*)to = v;
}
__global__ void __launch_bounds__(256) pad_kernel(const PadArgs a) {
    const uint32_t pieces = (uint32_t)(a.ld / 16);
    const uint64_t all = (uint64_t)(a.rows[0] + a.rows[1] + a.rows[2]) * pieces;
    for (uint64_t first = (uint64_t)blockIdx.x * 256; first < all; first += (uint64_t)gridDim.x * 256) {
        const uint64_t row0 = first / pieces;
        const uint32_t in = (uint32_t)(first - row0 * pieces) + threadIdx.x;
        pad_piece(a, (int64_t)(row0 + in / pieces), (int64_t)(in % pieces) * 16);
    }
}

int launch_pad(const PadArgs& a, void* stream) {
    const int64_t pieces = (a.rows[0] + a.rows[1] + a.rows[2]) * (a.ld / 16);
    if (pieces > 0) hipLaunchKernelGGL(pad_kernel, dim3(workgroups(pieces)), dim3(256), 0, (hipStream_t)stream, a);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

__global__ void __launch_bounds__(256) zeros_kernel(const FeedOut o, int64_t rows, int64_t cols) {
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < rows * cols; t += (int64_t)gridDim.x * 256) {
        char* const p = o.base + t / cols * o.ld + t % cols * o.size;
        if (o.size == 4) *(uint32_t*)p = 0;
        else *(uint16_t*)p = 0;
    }
}
int launch_zeros(const FeedOut& o, int64_t rows, int64_t cols, void* stream) {
    hipLaunchKernelGGL(zeros_kernel, dim3(workgroups(rows * cols)), dim3(256), 0, (hipStream_t)stream, o, rows, cols);
    return hipGetLastError() == hipSuccess ? 0 : 1;
}

}  // namespace cacnn
