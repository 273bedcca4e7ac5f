// Feed-forward operators, host side: checks of the arguments and what is launched.  See include/cacnn.h.
#include <stdint.h>

#include <algorithm>
#include <climits>
#include <cmath>

#include "../../include/cacnn.h"
#include "cacnn_feed.h"
#include "cacnn_internal.h"

using namespace cacnn;

namespace {

// Row lengths and strides: 32-bit offsets within the 256 rows of a tile, in units of a byte, stay below 2^30
constexpr int64_t kMostColumns = 1 << 20, kMostRows = INT32_MAX;
// and the threads of a launch below 2^32 on the 128 x 128 tiles, 256 for each 128 x 64 of a gated projection's result (other kernels are not chosen where
// they would need more)
bool tiles_in_range(int64_t rows, int64_t cols) { return (rows + 127) / 128 * ((cols + 63) / 64) < (1 << 24); }

bool columns(int64_t n) { return n >= 1 && n <= kMostColumns; }
bool rows(int64_t n) { return n >= 0 && n <= kMostRows; }
// a row stride, 0 for dense rows
bool stride(int64_t* ld, int64_t cols) {
    if (*ld == 0) *ld = cols;
    return *ld >= cols && *ld <= kMostColumns;
}
bool multiple(const void* p, size_t of) { return reinterpret_cast<uintptr_t>(p) % of == 0; }
bool element_type(int dtype) { return dtype == CACNN_F32 || dtype == CACNN_BF16_F32ACC; }

FeedOperand operand(const void* p, int64_t ld, int size, int64_t rows, int64_t k, bool padded = false) {
    return {static_cast<const char*>(p), ld * size, k, rows, padded};
}
FeedOut output(void* p, int64_t ld, int size) { return {static_cast<char*>(p), ld * size, size, multiple(p, 128) && ld * size % 128 == 0}; }

int64_t padded(int64_t n) { return (n + 63) / 64 * 64; }      // columns of a row in the workspace

// The workspace of the backward pass: the gradients of gate and up, and, where rows of C elements are no multiple of 16 bytes, X and both weights with rows
// that are: the products read them two and three times each, and faster straight to LDS.  Not for few rows, where the copies would be most of the traffic, unless C is
// too short for a 16-byte load.  us in all, without copies and with them, gate and up kept | computed again:
//     T                      64                       128                      256                      2048
//     bf16 (T, 4095, 4095)   69 : 75 | 85 : 85        77 : 82 | 101 : 95       101 : 94 | 152 : 121     414 : 320 | 597 : 428
//     bf16 (T, 1001, 1515)   25.5 : 26.6 | 32 : 31    27.2 : 27.2 | 34 : 32    31 : 30 | 42 : 36        97 : 66 | 123 : 81
//     fp32 (T, 2047, 4095)   112 : 114 | 135 : 135    133 : 130 | 174 : 168    199 : 198 | 284 : 273    1224 : 1108 | 1725 : 1584
// (Rows of a wider array and arrays that start elsewhere are not copied: the workspace's size does not depend on where they lie.)
struct Workspace {
    int64_t ld_f, ld_c;            // elements of a row; ld_c 0: no copies
    int64_t grad, x, w;            // bytes of grad_gate (and of grad_up), of the copies of X and of a weight
    Workspace(const cacnn_gated_problem& p, int size)
        : ld_f(padded(p.F)), ld_c(p.T > 0 && (p.C * size < 16 || (p.C * size % 16 && p.T >= 128)) ? padded(p.C) : 0), grad(p.T * ld_f * size), x(p.T * ld_c * size), w(p.F * ld_c * size) {}
    int64_t bytes() const { return 2 * grad + x + 2 * w; }
};

bool valid_gated(cacnn_gated_problem* p) {
    return rows(p->T) && columns(p->C) && columns(p->F) && stride(&p->ld_x, p->C) && stride(&p->ld_w, p->C) && stride(&p->ld_out, p->F) &&
           stride(&p->ld_pre, p->F) && stride(&p->ld_grad_x, p->C) && stride(&p->ld_grad_w, p->C) && tiles_in_range(p->T, padded(p->F)) &&
           tiles_in_range(p->T, p->C) && tiles_in_range(2 * p->F, p->C);
}
bool activation(int64_t a) { return a == CACNN_GATE_SILU || a == CACNN_GATE_GELU || a == CACNN_GATE_GELU_TANH; }

int launched(int rc) { return rc == 0 ? CACNN_OK : CACNN_ERR_LAUNCH; }

}  // namespace

// The kernel with the least estimated time.  A workgroup has a compute unit to itself (two of the 128 x 128 tiles with two stages share one), a launch runs in
// rounds of 256, and a round takes 3 us and what a slab of 128 bytes of the contraction (the dividing waves: four slabs, one each) was measured to take, in us, on
// shapes of 64 to 8192 rows; operands that come through registers take the dividing waves 1.7 times as long:
//                                            bf16, 8 bits   fp32 (bound by its matrix instructions)
//     32 x 32 divided (gated: 32 x 2 x 32)   0.75 (1.15)     0.8 (1.15)
//     64 x 32 divided (gated: 64 x 2 x 32)   1.15 (1.25)     1.4 (2.15)
//     64 x 64 divided                        1.45            2.4
//     128 x 128, four stages                 0.85            2.0
//     128 x 128, two of two stages           1.6             3.8
//     256 x 256                              2.0             -
//     64 x 128, three of two stages          -               1.0 for each tile of a compute unit, 1.3 for one
// Examples, us, the chosen kernel first: 8 bits (64, 8192, 4096) 12 on 32 x 32, 16 on 64 x 32; (256, 4096, 4096) 14 on 64 x 64, 19 on 64 x 32; (1024, 4096, 4096)
// 30 on 128 x 128 with four stages, 35 with two, 47 on 64 x 64; (2048, 4096, 4096) 42 with two stages, 54 with four, 53 on 256 x 256; bf16 gated (8192, 4096, 8192)
// 952 on 256 x 256, 1139 on 128 x 128 with two stages; fp32 gated (1028, 6976, 3712) 863 on 64 x 128, 971 on 64 x 32, 1262 on 128 x 128, (6261, 2494, 912) through
// registers 516, 630 and 627.
int cacnn::matmul_kernel(const FeedArgs& a, int form, int dtype, bool direct) {
    const bool f32 = dtype == FEED_F32, gated = form == FEED_GATED;
    const double slabs = (double)a.q[0].k * feed_size(dtype) / 128 * a.segments, ahead = direct ? 1.0 : 1.7;
    auto tiles = [&](const MatmulTile& t, int64_t cols) { return (a.M + t.rows - 1) / t.rows * ((cols + t.cols - 1) / t.cols) * a.products; };
    // (the 128 x 128 tiles take whatever the entry points let through)
    int best = MATMUL_128;
    double least = INFINITY;
    auto candidate = [&](int kernel, double us) {
        const MatmulTile t = matmul_tile(kernel, form, dtype);
        // the runtime launches less than 2^32 threads
        if (us < least && tiles(t, gated && a.grad_out ? a.grad_cols : a.N) * t.threads < (1ll << 32)) least = us, best = kernel;
    };
    auto rounds = [&](int kernel, int waves, double slab_us, int64_t at_once = 256) {
        candidate(kernel, (double)((tiles(matmul_tile(kernel, form, dtype), a.N) + at_once - 1) / at_once) * (3.0 + std::ceil(slabs / waves) * slab_us));
    };
    rounds(MATMUL_WAVES_32, 4, ahead * (gated ? 1.15 : f32 ? 0.8 : 0.75));
    rounds(MATMUL_WAVES_64_32, 4, ahead * (gated ? (f32 ? 2.15 : 1.25) : f32 ? 1.4 : 1.15));
    if (!gated) rounds(MATMUL_WAVES_64, 4, ahead * (f32 ? 2.4 : 1.45));
    if (direct) rounds(MATMUL_128_DEEP, 1, f32 ? 2.0 : 0.85);
    rounds(MATMUL_128, 1, f32 ? 3.8 : 1.6, 512);
    // (what a compute unit's tiles take is what their matrix instructions take, however many share it, and for one tile the time from load to LDS)
    if (f32)
        candidate(MATMUL_64_128, 3.0 + std::ceil(slabs) * std::max(direct ? 1.3 : 1.9, (double)((tiles(matmul_tile(MATMUL_64_128, form, dtype), a.N) + 255) / 256)));
    if (direct && (dtype == FEED_BF16 || dtype == FEED_E4M3)) rounds(MATMUL_256, 1, 2.0);
    return best;
}

extern "C" {

// The kernel (its number in cacnn_feed.h) of a product with M x N results and a contraction of k elements: form and dtype as there
int cacnn_internal_matmul_kernel(int form, int dtype, int direct, int64_t M, int64_t N, int64_t k) {
    FeedArgs a = {};
    a.M = M, a.N = N, a.q[0].k = k;
    a.segments = form == FEED_RIGHT ? 2 : 1, a.products = form == FEED_BOTH ? 2 : 1;
    return matmul_kernel(a, form, dtype, direct != 0);
}

int cacnn_quantize(const cacnn_quantize_problem* problem, int dtype, const void* x, void* q, float* scale, void* hip_stream) {
    if (!problem || (problem->T != 0 && (!x || !q || !scale))) return CACNN_ERR_NULL;
    cacnn_quantize_problem p = *problem;
    if (!element_type(dtype) || (p.block_rows != 1 && p.block_rows != kScaleBlock)) return CACNN_ERR_UNSUPPORTED;
    if (!rows(p.T) || !columns(p.C) || !stride(&p.ld_x, p.C) || !stride(&p.ld_q, p.C)) return CACNN_ERR_INVALID_ARG;
    const int size = feed_size(dtype);
    if (!multiple(x, size) || !multiple(scale, 4)) return CACNN_ERR_INVALID_ARG;
    if (!device_present()) return CACNN_ERR_NO_DEVICE;
    if (p.T == 0) return CACNN_OK;
    QuantizeArgs a = {};
    a.x = static_cast<const char*>(x), a.ld_x = p.ld_x * size;
    a.q = static_cast<uint8_t*>(q), a.ld_q = p.ld_q, a.scale = scale;
    a.T = p.T, a.C = p.C;
    a.blocks = (int32_t)((p.C + kScaleBlock - 1) / kScaleBlock);
    return launched(launch_quantize(a, dtype, (int)p.block_rows, hip_stream));
}

int cacnn_matmul_scaled(const cacnn_matmul_problem* problem, const void* x, const float* x_scale, const void* w, const float* w_scale, int out_dtype,
                        void* out, void* hip_stream) {
    if (!problem || !w || !w_scale || (problem->T != 0 && (!x || !x_scale || !out))) return CACNN_ERR_NULL;
    if (!element_type(out_dtype)) return CACNN_ERR_UNSUPPORTED;
    cacnn_matmul_problem p = *problem;
    if (!rows(p.T) || !columns(p.C) || !columns(p.K) || !stride(&p.ld_x, p.C) || !stride(&p.ld_w, p.C) || !stride(&p.ld_out, p.K) ||
        !tiles_in_range(p.T, p.K))
        return CACNN_ERR_INVALID_ARG;
    const int size = feed_size(out_dtype);
    if (!multiple(x_scale, 4) || !multiple(w_scale, 4) || !multiple(out, size)) return CACNN_ERR_INVALID_ARG;
    if (!device_present()) return CACNN_ERR_NO_DEVICE;
    if (p.T == 0) return CACNN_OK;
    FeedArgs a = {};
    a.segments = a.products = 1;
    a.q[0] = operand(x, p.ld_x, 1, p.T, p.C);
    a.p[0] = operand(w, p.ld_w, 1, p.K, p.C);
    a.out[0] = output(out, p.ld_out, size);
    a.M = p.T, a.N = p.K;
    a.q_scale = x_scale, a.p_scale[0] = w_scale;
    a.scale_cols = (int32_t)((p.C + kScaleBlock - 1) / kScaleBlock);
    return launched(launch_matmul(a, FEED_PLAIN, FEED_E4M3, hip_stream));
}

int cacnn_gated_forward(const cacnn_gated_problem* problem, int dtype, const void* x, const void* w_gate, const void* w_up, void* out, void* gate,
                        void* up, void* hip_stream) {
    if (!problem || !w_gate || !w_up || (problem->T != 0 && (!x || !out))) return CACNN_ERR_NULL;
    cacnn_gated_problem p = *problem;
    if (!element_type(dtype) || !activation(p.activation)) return CACNN_ERR_UNSUPPORTED;
    if (!valid_gated(&p) || (p.T != 0 && !gate != !up)) return CACNN_ERR_INVALID_ARG;
    const int size = feed_size(dtype);
    if (!multiple(x, size) || !multiple(w_gate, size) || !multiple(w_up, size) || !multiple(out, size) || !multiple(gate, size) || !multiple(up, size))
        return CACNN_ERR_INVALID_ARG;
    if (!device_present()) return CACNN_ERR_NO_DEVICE;
    if (p.T == 0) return CACNN_OK;
    FeedArgs a = {};
    a.segments = a.products = 1;
    a.q[0] = operand(x, p.ld_x, size, p.T, p.C);
    a.p[0] = operand(w_gate, p.ld_w, size, p.F, p.C);
    a.p[1] = operand(w_up, p.ld_w, size, p.F, p.C);
    a.out[0] = output(out, p.ld_out, size);
    if (gate) a.gate_out = output(gate, p.ld_pre, size), a.up_out = output(up, p.ld_pre, size);
    a.M = p.T, a.N = p.F;
    a.activation = (int32_t)p.activation;
    return launched(launch_matmul(a, FEED_GATED, dtype, hip_stream));
}

int cacnn_gated_forward_scaled(const cacnn_gated_problem* problem, const void* x, const float* x_scale, const void* w_gate, const float* w_gate_scale,
                               const void* w_up, const float* w_up_scale, int out_dtype, void* out, void* hip_stream) {
    if (!problem || !w_gate || !w_gate_scale || !w_up || !w_up_scale || (problem->T != 0 && (!x || !x_scale || !out))) return CACNN_ERR_NULL;
    cacnn_gated_problem p = *problem;
    if (!element_type(out_dtype) || !activation(p.activation)) return CACNN_ERR_UNSUPPORTED;
    if (!valid_gated(&p)) return CACNN_ERR_INVALID_ARG;
    const int size = feed_size(out_dtype);
    if (!multiple(x_scale, 4) || !multiple(w_gate_scale, 4) || !multiple(w_up_scale, 4) || !multiple(out, size)) return CACNN_ERR_INVALID_ARG;
    if (!device_present()) return CACNN_ERR_NO_DEVICE;
    if (p.T == 0) return CACNN_OK;
    FeedArgs a = {};
    a.segments = a.products = 1;
    a.q[0] = operand(x, p.ld_x, 1, p.T, p.C);
    a.p[0] = operand(w_gate, p.ld_w, 1, p.F, p.C);
    a.p[1] = operand(w_up, p.ld_w, 1, p.F, p.C);
    a.out[0] = output(out, p.ld_out, size);
    a.M = p.T, a.N = p.F;
    a.q_scale = x_scale, a.p_scale[0] = w_gate_scale, a.p_scale[1] = w_up_scale;
    a.scale_cols = (int32_t)((p.C + kScaleBlock - 1) / kScaleBlock);
    a.activation = (int32_t)p.activation;
    return launched(launch_matmul(a, FEED_GATED, FEED_E4M3, hip_stream));
}

int cacnn_gated_workspace(const cacnn_gated_problem* problem, int dtype, size_t* bytes) {
    if (!problem || !bytes) return CACNN_ERR_NULL;
    cacnn_gated_problem p = *problem;
    if (!element_type(dtype) || !activation(p.activation)) return CACNN_ERR_UNSUPPORTED;
    if (!valid_gated(&p)) return CACNN_ERR_INVALID_ARG;
    *bytes = (size_t)Workspace(p, feed_size(dtype)).bytes();
    return CACNN_OK;
}

int cacnn_gated_backward(const cacnn_gated_problem* problem, int dtype, const void* x, const void* w_gate, const void* w_up, const void* gate,
                         const void* up, const void* grad_out, void* grad_x, void* grad_w_gate, void* grad_w_up, void* workspace,
                         size_t workspace_bytes, void* hip_stream) {
    if (!problem || !w_gate || !w_up || (problem->T != 0 && (!x || !grad_out || !workspace))) return CACNN_ERR_NULL;
    cacnn_gated_problem p = *problem;
    if (!element_type(dtype) || !activation(p.activation)) return CACNN_ERR_UNSUPPORTED;
    if (!valid_gated(&p) || (p.T != 0 && !gate != !up) || !grad_w_gate != !grad_w_up || (p.T != 0 && !grad_x && !grad_w_gate))
        return CACNN_ERR_INVALID_ARG;
    const int size = feed_size(dtype);
    for (const void* q : {x, w_gate, w_up, gate, up, grad_out, (const void*)grad_x, (const void*)grad_w_gate, (const void*)grad_w_up})
        if (!multiple(q, size)) return CACNN_ERR_INVALID_ARG;
    const Workspace ws(p, size);
    if (!multiple(workspace, 16) || (int64_t)std::min(workspace_bytes, (size_t)INT64_MAX) < ws.bytes()) return CACNN_ERR_INVALID_ARG;
    if (!device_present()) return CACNN_ERR_NO_DEVICE;
    const int64_t ld = ws.ld_f;
    // the gradients of the two products, in the workspace with rows padded by zeros
    char* const grad_gate = static_cast<char*>(workspace);
    char* const grad_up = grad_gate + ws.grad;
    if (ws.ld_c && p.T != 0) {
        char* const copies = grad_up + ws.grad;
        PadArgs a = {};
        a.from[0] = static_cast<const char*>(x), a.from[1] = static_cast<const char*>(w_gate), a.from[2] = static_cast<const char*>(w_up);
        a.ld_from[0] = p.ld_x * size, a.ld_from[1] = a.ld_from[2] = p.ld_w * size;
        // (what is read: X where the products are computed again or a weight's gradient is wanted, the weights where X's is)
        a.rows[0] = !gate || grad_w_gate ? p.T : 0, a.rows[1] = a.rows[2] = !gate || grad_x ? p.F : 0;
        a.to = copies + (a.rows[0] ? 0 : ws.x), a.bytes = p.C * size, a.ld = ws.ld_c * size, a.size = size;
        if (launch_pad(a, hip_stream) != 0) return CACNN_ERR_LAUNCH;
        x = copies, w_gate = copies + ws.x, w_up = copies + ws.x + ws.w;
        p.ld_x = p.ld_w = ws.ld_c;
    }
    const bool copied = ws.ld_c != 0;
    if (p.T != 0) {
        if (gate) {
            GateArgs a = {};
            a.gate = static_cast<const char*>(gate), a.up = static_cast<const char*>(up), a.grad_out = static_cast<const char*>(grad_out);
            a.ld_pre = p.ld_pre * size, a.ld_out = p.ld_out * size;
            a.grad_gate = grad_gate, a.grad_up = grad_up, a.ld = ld * size;
            a.T = p.T, a.F = p.F, a.cols = ld;
            a.activation = (int32_t)p.activation;
            if (launch_gate_grad(a, dtype, hip_stream) != 0) return CACNN_ERR_LAUNCH;
        } else {
            FeedArgs a = {};
            a.segments = a.products = 1;
            a.q[0] = operand(x, p.ld_x, size, p.T, p.C, copied);
            a.p[0] = operand(w_gate, p.ld_w, size, p.F, p.C, copied);
            a.p[1] = operand(w_up, p.ld_w, size, p.F, p.C, copied);
            a.out[0] = output(grad_gate, ld, size), a.out[1] = output(grad_up, ld, size);
            a.M = p.T, a.N = p.F;
            a.activation = (int32_t)p.activation;
            a.grad_out = static_cast<const char*>(grad_out), a.grad_out_ld = p.ld_out * size;
            a.grad_cols = (int32_t)ld;
            if (launch_matmul(a, FEED_GATED, dtype, hip_stream) != 0) return CACNN_ERR_LAUNCH;
        }
    }
    if (grad_x && p.T != 0) {
        FeedArgs a = {};
        a.segments = 2, a.products = 1;
        a.q[0] = operand(grad_gate, ld, size, p.T, p.F, true), a.q[1] = operand(grad_up, ld, size, p.T, p.F, true);
        a.p[0] = operand(w_gate, p.ld_w, size, p.C, p.F, copied), a.p[1] = operand(w_up, p.ld_w, size, p.C, p.F, copied);
        a.out[0] = output(grad_x, p.ld_grad_x, size);
        a.M = p.T, a.N = p.C;
        if (launch_matmul(a, FEED_RIGHT, dtype, hip_stream) != 0) return CACNN_ERR_LAUNCH;
    }
    if (grad_w_gate && p.T == 0) {
        for (void* const w : {grad_w_gate, grad_w_up})
            if (launch_zeros(output(w, p.ld_grad_w, size), p.F, p.C, hip_stream) != 0) return CACNN_ERR_LAUNCH;
    } else if (grad_w_gate) {
        FeedArgs a = {};
        a.segments = 1, a.products = 2;
        a.q[0] = operand(grad_gate, ld, size, p.F, p.T, true), a.q[1] = operand(grad_up, ld, size, p.F, p.T, true);
        a.p[0] = operand(x, p.ld_x, size, p.C, p.T, copied);
        a.out[0] = output(grad_w_gate, p.ld_grad_w, size), a.out[1] = output(grad_w_up, p.ld_grad_w, size);
        a.M = p.F, a.N = p.C;
        if (launch_matmul(a, FEED_BOTH, dtype, hip_stream) != 0) return CACNN_ERR_LAUNCH;
    }
    return CACNN_OK;
}

}  // extern "C"
