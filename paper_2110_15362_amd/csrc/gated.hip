// The gated projections h = act(x Wg^T) * (x Wu^T) and their backward pass: see include/bittrain.h for the contract.
//
// Three products on the matrix cores, all with 32-bit sums:
//   forward    h   [rows, f]   both products of a tile of h in one workgroup, the activation and the product on its registers
//   grad_x     [rows, d]       dg Wg + du Wu: one sum over 2 f
//   grad_w     [2 f, d]        dg^T x and du^T x
// with dg and du computed once, into the workspace, by a pass over grad_h, gate and up.
#include <math.h>

#include "block.h"

namespace btb {
namespace {

typedef float acc4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
#define BT_LDS __attribute__((address_space(3)))

// ---- one step of a product -------------------------------------------------------------------------------------
//
// A fragment is 16 rows (or columns) by kKStep of the summed index, 16 bytes a lane: lane l holds row l % 16 and, of every kKStep, the
// kPer<T> summed indices from (l / 16) * kPer<T> on.  The result of P's fragment and Q's has row 4 * (l / 16) + r (from P) and column l % 16 (from
// Q) in element r of lane l: with P the operand along which the output is contiguous, a lane holds four neighbours of a row.

template <class T> constexpr int kKStep = 4 * kPer<T>;       // 32 or, in single precision, 16
constexpr int kKBytes = 128;                                 // of the summed index in a tile
template <class T> constexpr int kK = kKBytes / (int)sizeof(T);

template <class T> __device__ inline acc4 multiply(const raw16 p, const raw16 q, acc4 c) {
    if constexpr (std::is_same_v<T, bf16>) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, p), __builtin_bit_cast(bf16x8, q), c, 0, 0, 0);
    else if constexpr (std::is_same_v<T, f16>) return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, (uint32_t)p[j]), __builtin_bit_cast(float, (uint32_t)q[j]), c, 0, 0, 0);
        return c;
    }
}

// ---- tiles in LDS ----------------------------------------------------------------------------------------------
//
// An operand comes in one of two orders: with the summed index contiguous in memory (K rows: an LDS row is one row or column of the
// product, 128 bytes of the summed index) or with it across the rows (N rows: an LDS row is one summed index, the tile's rows or
// columns lie along it).  16-byte chunks of an LDS row are stored in an order that depends on the row, so that the lanes that read one
// fragment meet different banks.

enum Order { kAlong, kAcross };      // the summed index: along memory rows, across them

template <class T, Order O, int N> struct Tile {      // N rows or columns of the product
    static constexpr int ROWS = O == kAlong ? N : kK<T>;
    static constexpr int CHUNKS = (O == kAlong ? kKBytes : N * (int)sizeof(T)) / kVec;      // of a row
    static constexpr int BYTES = ROWS * CHUNKS * kVec;

    __device__ static int place(const int row, const int chunk) {
        int key;
        if constexpr (O == kAlong) key = row & 7;
        else if constexpr (sizeof(T) == 2) key = 2 * ((row & 3) | ((row >> 1) & 4));
        else key = 4 * ((row >> 2) & 3);
        return (row * CHUNKS + (chunk ^ key)) * kVec;
    }

    // The fragment of rows or columns [at, at + 16) and step `step` of the summed index.
    __device__ static raw16 fragment(const char *tile, const int at, const int step) {
        const int lane = threadIdx.x % kWave, group = lane / 16, t = lane % 16;
        if constexpr (O == kAlong) {
            return *(const raw16 *)(tile + place(at + t, step * 4 + group));
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 summed indices by 16 columns, 4 columns a lane, and get one column each
            raw16 v;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int k = step * 32 + group * 8 + half * 4 + t / 4, n = at + (t % 4) * 4;
                const char *const from = tile + place(k, n / 8) + (n % 8) * 2;
                const short4v got = __builtin_amdgcn_ds_read_tr16_b64_v4i16((BT_LDS short4v *)from);
                typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
                const uint2v bits = __builtin_bit_cast(uint2v, got);
                v[2 * half] = bits[0];
                v[2 * half + 1] = bits[1];
            }
            return v;
        } else {
            raw16 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int k = step * 16 + group * 4 + j, n = at + t;
                v[j] = *(const uint32_t *)(tile + place(k, n / 4) + (n % 4) * 4);
            }
            return v;
        }
    }
};

// An operand in memory: element (row, column) at p[row * pitch + column], `rows` by `cols`.
struct Operand {
    const void *p;
    uint64_t pitch;
    uint32_t rows, cols;
};

constexpr int kTileN = 128, kThreads = 256;      // of both operands of a product; threads of a workgroup: 2 by 2 waves of 64 by 64

// Chunks of a tile on their way from memory to LDS, in registers.
template <class T, Order O> struct Staged {
    typedef Tile<T, O, kTileN> L;
    static constexpr int PER = L::ROWS * L::CHUNKS / kThreads;
    raw16 v[PER];

    // `n`: the product's row or column that the tile begins at (of 64 of two operands in turn, where `other` is given), `k`: the summed index.
    __device__ void load(const Operand &a, const Operand &other, const bool two, const uint32_t n, const uint32_t k) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * kThreads + threadIdx.x, row = q / L::CHUNKS, col = (q % L::CHUNKS) * kPer<T>;
            if constexpr (O == kAlong) {
                // the forward pass: 32 rows of one weight and 32 of the other for each wave
                const Operand &from = two && (row & 32) ? other : a;
                const uint32_t r = n + (two ? (row / 64) * 32 + row % 32 : row);
                v[i] = raw16{0, 0, 0, 0};
                if (r < from.rows) v[i] = load_vec((const T *)from.p + r * from.pitch + k + col, (int64_t)from.cols - k - col);
            } else {
                v[i] = raw16{0, 0, 0, 0};
                if (k + row < a.rows) v[i] = load_vec((const T *)a.p + (k + row) * a.pitch + n + col, (int64_t)a.cols - n - col);
            }
        }
    }
    __device__ void store(char *tile) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * kThreads + threadIdx.x;
            *(raw16 *)(tile + L::place(q / L::CHUNKS, q % L::CHUNKS)) = v[i];
        }
    }
};

// 1 / (1 + exp(-g)).  Where the result is rounded to 16 bits, with the instructions for 2^x and 1 / x, whose last places are lost anyway.
template <class T> __device__ inline float sigmoid(const float g) {
    if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-g));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
}

// act(g) and its derivative, of SiLU and of the GELU, whose (1 + tanh(y)) / 2 is sigmoid(2 y).
constexpr float kGelu = 1.5957691216057308f, kGeluCube = 0.044715f;      // 2 sqrt(2 / pi)

template <class T> __device__ inline float activate(const int activation, const float g) {
    if (activation == BT_ACT_SILU) return g * sigmoid<T>(g);
    return g * sigmoid<T>(kGelu * (g + kGeluCube * g * g * g));
}

template <class T> __device__ inline void activate(const int activation, const float g, float *value, float *slope) {
    float s, inner = 1.0f;
    if (activation == BT_ACT_SILU) s = sigmoid<T>(g);
    else {
        s = sigmoid<T>(kGelu * (g + kGeluCube * g * g * g));
        inner = kGelu * (1.0f + 3.0f * kGeluCube * g * g);
    }
    *value = g * s;
    *slope = s * (1.0f + g * (1.0f - s) * inner);
}

template <class T> __device__ inline void store4(T *p, const int64_t left, const float (&x)[4]) {
    if (left >= 4) {
        if constexpr (sizeof(T) == 4) store_vec(p, 4, pack<T>(x));
        else {
            typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
            struct __attribute__((packed, aligned(2))) Half { uint2v v; };
            ((Half *)p)->v = uint2v{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) p[i] = narrow<T>(x[i]);
}

enum Product { kForward, kGradX, kGradW };

struct GatedJob {
    Operand p[2], q[2];              // (of the forward pass p: both weights; of the others p and q: the first and the second sum, or output)
    void *out[2];                    // h; grad_x; grad_w_gate and grad_w_up
    void *gate, *up;                 // what the forward pass keeps, or NULL
    uint64_t pitch;                  // of all outputs
    uint32_t m, n, k;                // rows and columns of the output (of each), and the summed index (of each sum)
    uint32_t tiles_n, tiles_m;       // of each output
    int activation;
};

template <class T, Product K> constexpr Order kOrderP = K == kForward ? kAlong : kAcross;
template <class T, Product K> constexpr Order kOrderQ = K == kGradW ? kAcross : kAlong;

template <class T, Product K> __global__ __launch_bounds__(kThreads) void gated_kernel(const GatedJob a) {
    typedef Tile<T, kOrderP<T, K>, kTileN> P;
    typedef Tile<T, kOrderQ<T, K>, kTileN> Q;
    __shared__ __align__(16) char tiles[P::BYTES + Q::BYTES];
    char *const tile_p = tiles, *const tile_q = tiles + P::BYTES;
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, wp = wave % 2, wq = wave / 2;
    constexpr int kCols = K == kForward ? kTileN / 2 : kTileN;      // columns of the output in a tile
    uint32_t tile = blockIdx.x;
    const int part = K == kGradW ? tile / (a.tiles_m * a.tiles_n) : 0;
    tile -= part * a.tiles_m * a.tiles_n;
    const uint32_t m = (tile / a.tiles_n) * kTileN, n = (tile % a.tiles_n) * kCols;
    acc4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = acc4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int sum = 0; sum < (K == kGradX ? 2 : 1); ++sum) {
        const Operand &op = a.p[K == kGradX ? sum : 0], &oq = a.q[K == kGradX ? sum : part];
        for (uint32_t k = 0; k < a.k; k += kK<T>) {
            Staged<T, kOrderP<T, K>> sp;
            Staged<T, kOrderQ<T, K>> sq;
            sp.load(op, a.p[1], K == kForward, n, k);
            sq.load(oq, oq, false, m, k);
            __syncthreads();
            sp.store(tile_p);
            sq.store(tile_q);
            __syncthreads();
#pragma unroll
            for (int step = 0; step < kK<T> / kKStep<T>; ++step) {
                raw16 p[4], q[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = P::fragment(tile_p, wp * 64 + i * 16, step);
#pragma unroll
                for (int i = 0; i < 4; ++i) q[i] = Q::fragment(tile_q, wq * 64 + i * 16, step);
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] = multiply<T>(p[i], q[j], acc[i][j]);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t row = m + wq * 64 + j * 16 + lane % 16;
        if (row >= a.m) continue;
        if constexpr (K == kForward) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t col = n + wp * 32 + i * 16 + lane / 16 * 4;
                const int64_t left = (int64_t)a.n - col;
                const uint64_t at = row * a.pitch + col;
                if (left <= 0) continue;
                float g[4], u[4], h[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    g[r] = acc[i][j][r];
                    u[r] = acc[i + 2][j][r];
                    if (a.activation == BT_ACT_RELU) {
                        const bool closed = g[r] <= 0.0f;
                        h[r] = closed ? 0.0f : g[r] * u[r];
                        g[r] = closed ? 0.0f : g[r];
                        u[r] = closed ? 0.0f : u[r];
                    } else h[r] = activate<T>(a.activation, g[r]) * u[r];
                }
                store4((T *)a.out[0] + at, left, h);
                if (a.gate) {
                    store4((T *)a.gate + at, left, g);
                    store4((T *)a.up + at, left, u);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t col = n + wp * 64 + i * 16 + lane / 16 * 4;
                const int64_t left = (int64_t)a.n - col;
                const float x[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (left > 0) store4((T *)a.out[part] + row * a.pitch + col, left, x);
            }
        }
    }
}

// dg = grad_h u act'(g) and du = grad_h act(g), rounded to the type: they are factors of the products, whose matrix instructions take them
// so, and an error of half a unit in the last place of each term averages out in the sums.  Rows of `pitch` elements, whole vectors.
template <class T> __global__ __launch_bounds__(256) void gated_slopes_kernel(const T *grad_h, const T *gate, const T *up, T *dg, T *du,
                                                                             const uint32_t f, const uint32_t pitch, const uint64_t vectors, const int activation) {
    const uint32_t a_row = pitch / kPer<T>;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / a_row;
        const uint32_t col = (uint32_t)(i - row * a_row) * kPer<T>;
        const uint64_t at = row * f + col;
        float h[kPer<T>], g[kPer<T>], u[kPer<T>];
        unpack<T>(load_vec(grad_h + at, (int64_t)f - col), h);
        unpack<T>(load_vec(gate + at, (int64_t)f - col), g);
        unpack<T>(load_vec(up + at, (int64_t)f - col), u);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) {
            if (activation == BT_ACT_RELU) {
                const bool closed = g[e] <= 0.0f;
                u[e] = closed ? 0.0f : h[e] * u[e];
                g[e] = closed ? 0.0f : h[e] * g[e];
            } else {
                float value, slope;
                activate<T>(activation, g[e], &value, &slope);
                u[e] *= h[e] * slope;
                g[e] = h[e] * value;
            }
        }
        store_vec(dg + i * kPer<T>, kPer<T>, pack<T>(u));
        store_vec(du + i * kPer<T>, kPer<T>, pack<T>(g));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

uint64_t padded(const uint64_t f, const int width) { return (f * width + kVec - 1) / kVec * kVec / width; }

bt_status check_sizes(const uint64_t rows, const uint64_t d, const uint64_t f, const bt_dtype dtype) {
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (rows > BT_MAX_ROWS || d > BT_MAX_FEATURES || f > BT_MAX_FEATURES) return BT_ERR_SIZE;
    return BT_OK;
}

bool known(const bt_activation a) { return a == BT_ACT_RELU || a == BT_ACT_SILU || a == BT_ACT_GELU_TANH; }

uint32_t ceil_div(const uint64_t a, const uint64_t b) { return (uint32_t)((a + b - 1) / b); }

template <class T, Product K> bt_status run_product(GatedJob &a, hipStream_t hs) {
    a.tiles_m = ceil_div(a.m, kTileN);
    a.tiles_n = ceil_div(a.n, K == kForward ? kTileN / 2 : kTileN);
    const uint64_t tiles = (uint64_t)a.tiles_m * a.tiles_n * (K == kGradW ? 2 : 1);
    if (tiles >= 1u << 24) return BT_ERR_SIZE;      // (a grid holds less than 2^32 threads)
    return launch(gated_kernel<T, K>, dim3((unsigned)tiles), kThreads, hs, a);
}

}  // namespace
}  // namespace btb

using namespace btb;

extern "C" {

size_t bt_gated_workspace_bytes(uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, int backward) {
    if (check_sizes(rows, d, f, dtype) != BT_OK || rows == 0 || f == 0) return 0;
    return backward ? (size_t)(2 * rows * padded(f, width_of(dtype)) * (uint64_t)width_of(dtype)) : 0;
}

bt_status bt_gated_forward(const void *d_x, const void *d_w_gate, const void *d_w_up,
                           uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation,
                           void *d_h, void *d_gate, void *d_up,
                           void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    const bt_status st = check_sizes(rows, d, f, dtype);
    if (st != BT_OK) return st;
    if (!known(activation) || (d_gate == nullptr) != (d_up == nullptr)) return BT_ERR_ARGUMENT;
    if (rows == 0 || f == 0) return BT_OK;
    if (d_h == nullptr || (d != 0 && (d_x == nullptr || d_w_gate == nullptr || d_w_up == nullptr))) return BT_ERR_NULL;
    const size_t need = bt_gated_workspace_bytes(rows, d, f, dtype, 0), w = (size_t)width_of(dtype);
    if (need != 0 && d_workspace == nullptr) return BT_ERR_NULL;
    if (misaligned(d_x, w) || misaligned(d_w_gate, w) || misaligned(d_w_up, w) || misaligned(d_h, w) || misaligned(d_gate, w) || misaligned(d_up, w) ||
        misaligned(d_workspace, 128))
        return BT_ERR_ALIGN;
    if (workspace_bytes < need) return BT_ERR_WORKSPACE;
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        GatedJob a = {};
        a.p[0] = {d_w_gate, d, (uint32_t)f, (uint32_t)d};
        a.p[1] = {d_w_up, d, (uint32_t)f, (uint32_t)d};
        a.q[0] = {d_x, d, (uint32_t)rows, (uint32_t)d};
        a.out[0] = d_h;
        a.gate = d_gate;
        a.up = d_up;
        a.pitch = f;
        a.m = (uint32_t)rows;
        a.n = (uint32_t)f;
        a.k = (uint32_t)d;
        a.activation = activation;
        return run_product<T, kForward>(a, (hipStream_t)stream);
    });
}

bt_status bt_gated_backward(const void *d_grad_h, const void *d_x, const void *d_w_gate, const void *d_w_up,
                            const void *d_gate, const void *d_up,
                            uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation,
                            void *d_grad_x, void *d_grad_w_gate, void *d_grad_w_up,
                            void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    const bt_status st = check_sizes(rows, d, f, dtype);
    if (st != BT_OK) return st;
    if (!known(activation) || (d_grad_w_gate == nullptr) != (d_grad_w_up == nullptr)) return BT_ERR_ARGUMENT;
    const size_t w = (size_t)width_of(dtype);
    for (const void *p : {d_grad_h, d_x, d_w_gate, d_w_up, d_gate, d_up, (const void *)d_grad_x, (const void *)d_grad_w_gate, (const void *)d_grad_w_up})
        if (misaligned(p, w)) return BT_ERR_ALIGN;
    if (misaligned(d_workspace, 128)) return BT_ERR_ALIGN;
    const hipStream_t hs = (hipStream_t)stream;
    if (d == 0 || (d_grad_x == nullptr && d_grad_w_gate == nullptr)) return BT_OK;
    const size_t need = bt_gated_workspace_bytes(rows, d, f, dtype, 1);
    if (rows != 0 && f != 0) {
        if (d_grad_h == nullptr || d_gate == nullptr || d_up == nullptr || d_workspace == nullptr ||
            (d_grad_x && (d_w_gate == nullptr || d_w_up == nullptr)) || (d_grad_w_gate && d_x == nullptr))
            return BT_ERR_NULL;
        if (workspace_bytes < need) return BT_ERR_WORKSPACE;
    }
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (rows == 0 || f == 0) {      // sums of nothing
            bt_status s = d_grad_x ? zeros<T>(d_grad_x, rows * d, hs) : BT_OK;
            if (s == BT_OK && d_grad_w_gate) s = zeros<T>(d_grad_w_gate, f * d, hs);
            if (s == BT_OK && d_grad_w_up) s = zeros<T>(d_grad_w_up, f * d, hs);
            return s;
        }
        const uint64_t pitch = padded(f, sizeof(T)), vectors = rows * pitch / kPer<T>;
        T *const dg = (T *)d_workspace, *const du = dg + rows * pitch;
        const uint64_t blocks = (vectors + 255) / 256;
        bt_status s = launch(gated_slopes_kernel<T>, dim3((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20)), 256, hs, (const T *)d_grad_h, (const T *)d_gate,
                             (const T *)d_up, dg, du, (uint32_t)f, (uint32_t)pitch, vectors, (int)activation);
        if (s == BT_OK && d_grad_x) {
            GatedJob a = {};
            a.p[0] = {d_w_gate, d, (uint32_t)f, (uint32_t)d};
            a.p[1] = {d_w_up, d, (uint32_t)f, (uint32_t)d};
            a.q[0] = {dg, pitch, (uint32_t)rows, (uint32_t)f};
            a.q[1] = {du, pitch, (uint32_t)rows, (uint32_t)f};
            a.out[0] = d_grad_x;
            a.pitch = d;
            a.m = (uint32_t)rows;
            a.n = (uint32_t)d;
            a.k = (uint32_t)f;
            s = run_product<T, kGradX>(a, hs);
        }
        if (s == BT_OK && d_grad_w_gate) {
            GatedJob a = {};
            a.p[0] = {d_x, d, (uint32_t)rows, (uint32_t)d};
            a.q[0] = {dg, pitch, (uint32_t)rows, (uint32_t)f};
            a.q[1] = {du, pitch, (uint32_t)rows, (uint32_t)f};
            a.out[0] = d_grad_w_gate;
            a.out[1] = d_grad_w_up;
            a.pitch = d;
            a.m = (uint32_t)f;
            a.n = (uint32_t)d;
            a.k = (uint32_t)rows;
            s = run_product<T, kGradW>(a, hs);
        }
        return s;
    });
}

}  // extern "C"
