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

// `x`, which the compiler takes for another one each time: what follows from it is worked out where it is needed, and holds no registers until then.
__device__ inline int fresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// ---- one step of a product -------------------------------------------------------------------------------------
//
// A fragment is 16 rows (or columns) by kKStep of the summed index, 16 bytes a lane: lane l holds row l % 16 and, of every kKStep, the
// kPer<T> summed indices from (l / 16) * kPer<T> on.  The result of P's fragment and Q's has row 4 * (l / 16) + r (from P) and column l % 16 (from
// Q) in element r of lane l: with P the operand along which the output is contiguous, a lane holds four neighbours of a row.

template <class T> constexpr int kKStep = 4 * kPer<T>;       // 32 or, in single precision, 16
constexpr int kKBytes = 64;                                  // of the summed index in a tile: one step
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
// product, 64 bytes of the summed index) or with it across the rows (N rows: an LDS row is one summed index, the tile's rows or
// columns lie along it).  16-byte chunks of an LDS row are stored in an order that depends on the row, so that the lanes that read one
// fragment meet different banks.

enum Order { kAlong, kAcross };      // the summed index: along memory rows, across them

template <class T, Order O, int N> struct Tile {      // N rows or columns of the product
    static constexpr int ROWS = O == kAlong ? N : kK<T>;
    static constexpr int CHUNKS = (O == kAlong ? kKBytes : N * (int)sizeof(T)) / kVec;      // of a row
    static constexpr int BYTES = ROWS * CHUNKS * kVec;

    // (Of the rows that one fragment has, those of a lane share the key.)
    __device__ static int place(const int row, const int chunk) {
        int key;
        if constexpr (O == kAlong) key = (row >> 1) & 2;
        else if constexpr (sizeof(T) == 2 && CHUNKS == 8) key = 2 * (((row >> 1) & 1) | ((row >> 2) & 2));
        else if constexpr (sizeof(T) == 2) key = 2 * ((row & 3) | ((row >> 1) & 4));
        else key = 4 * ((row >> 2) & 3);
        return (row * CHUNKS + (chunk ^ key)) * kVec;
    }
};

// A wave's fragments of a tile: F times 16 rows or columns from `first` on.  Where a lane reads depends on the fragment and the tile by constants
// alone, but for one address (summed index along) or one a fragment (across).
template <class T, Order O, int N, int F> struct Reader {
    typedef Tile<T, O, N> L;
    static constexpr int ROW = L::CHUNKS * kVec, READS = O == kAlong ? 1 : sizeof(T) == 2 ? 2 : 4;      // instructions a fragment
    uint32_t at[O == kAlong ? 1 : F];

    __device__ void start(const int first) {
        const int lane = threadIdx.x % kWave, group = lane / 16, t = lane % 16;
        if constexpr (O == kAlong) at[0] = L::place(first + t, group);
        else {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int n = first + i * 16;
                if constexpr (sizeof(T) == 2) at[i] = L::place(group * 8 + t / 4, (n + t % 4 * 4) / 8) + t % 2 * 8;
                else at[i] = L::place(group * 4, (n + t) / 4) + t % 4 * 4;
            }
        }
    }

    __device__ raw16 read(const char *tile, const int i) const {
        if constexpr (O == kAlong) {
            return *(const raw16 *)(tile + at[0] + i * 16 * ROW);
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 summed indices by 16 columns, 4 columns a lane, and get one column each
            typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
            const char *const from = tile + at[i];
            const uint2v low = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((BT_LDS short4v *)from));
            const uint2v high = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((BT_LDS short4v *)(from + 4 * ROW)));
            return raw16{low[0], low[1], high[0], high[1]};
        } else {
            raw16 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t *)(tile + at[i] + j * ROW);
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

// A workgroup: WP waves along P by two along Q, each of FP fragments of P by FQ of Q.
template <int WP_, int FP_, int FQ_, int PLACES_> struct Shape {
    static constexpr int WP = WP_, FP = FP_, FQ = FQ_, PLACES = PLACES_, WAVES = 2 * WP, THREADS = WAVES * kWave, NP = WP * FP * 16, NQ = 2 * FQ * 16;
};
typedef Shape<4, 4, 8, 4> Large;      // 256 by 256, 8 waves
typedef Shape<2, 4, 4, 4> Middle;     // 128 by 128, 4 waves
typedef Shape<2, 2, 2, 4> Small;      // 64 by 64, 4 waves

// The forward pass: which row of a weight, of the 8 F that a wave has of it, lies in row r of them in LDS, the wave having F fragments, F / 2 of each
// weight.  In this order a lane's results of all fragments are 2 F neighbours of h.
template <int F> __device__ inline int weight_row(const int r) { return r % 16 / 4 * (2 * F) + r / 16 * 4 + r % 4; }

// Chunks of a tile on their way from memory to LDS, in registers.  (F: of the forward pass, fragments of a wave.)
template <class T, Order O, int N, int F, int kThreads> struct Staged {
    typedef Tile<T, O, N> L;
    static constexpr int PER = L::ROWS * L::CHUNKS / kThreads;
    raw16 v[PER];

    // `n`: the product's row or column that the tile begins at, `k`: the summed index.  `two`: the forward pass, each wave's rows half of one
    // weight and half of the other.
    __device__ void load(const Operand &a, const Operand &other, const bool two, const uint32_t n, const uint32_t k) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * kThreads + fresh(threadIdx.x), row = q / L::CHUNKS, col = (q % L::CHUNKS) * kPer<T>;
            if constexpr (O == kAlong) {
                constexpr int kHalf = F * 8;      // rows of a wave that belong to one weight
                const Operand &from = two && (row / kHalf) % 2 ? other : a;
                const uint32_t r = n + (two ? row / (2 * kHalf) * kHalf + weight_row<F>(row % kHalf) : row);
                v[i] = raw16{0, 0, 0, 0};
                if (r < from.rows) v[i] = load_vec((const T *)from.p + r * from.pitch + k + col, (int)(from.cols - k) - col, (int)k + col);
            } else {
                v[i] = raw16{0, 0, 0, 0};
                if (k + row < a.rows) v[i] = load_vec((const T *)a.p + (k + row) * a.pitch + n + col, (int)(a.cols - n) - col, (int)n + col);
            }
        }
    }
    __device__ void store(char *tile) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * kThreads + fresh(threadIdx.x);
            *(raw16 *)(tile + L::place(q / L::CHUNKS, q % L::CHUNKS)) = v[i];
        }
    }
};

// The elements of a vector from `shift` on, zeros behind them.
template <class T> __device__ inline raw16 moved(const raw16 v, const int shift) {
    typedef uint64_t two __attribute__((ext_vector_type(2)));
    const two x = __builtin_bit_cast(two, v);
    const uint32_t bits = (uint32_t)shift * (8 * sizeof(T)), rest = bits % 64;
    const uint64_t low = bits < 64 ? x[0] : bits < 128 ? x[1] : 0, high = bits < 64 ? x[1] : 0;
    return __builtin_bit_cast(raw16, two{low >> rest | high << 1 << (63 - rest), high >> rest});
}

// Rows of an odd number of 16-bit elements begin off the 4-byte boundaries in turn, and a load off them takes the memory more than twice as long (bf16
// forward of [1, 3001] x 11003: 48 us; x 3002: 30).  With a tensor that begins on one, such a vector is read from the element before it, its last
// element by itself, and moved.  (`before`: the vector from there, `end`: the last element.)
template <class T> __device__ inline raw16 from_odd(const raw16 before, const uint32_t end, const bool odd) {
    const uint32_t by = odd ? 16 : 0;
    raw16 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_alignbit(i < 3 ? before[i < 3 ? i + 1 : 0] : end, before[i], by);
    return v;
}

template <class T> __device__ inline uint32_t bits_at(const T *p) {
    static_assert(sizeof(T) == 2);
    return *(const uint16_t *)p;
}

// A tile's chunks on their way to LDS like those above, but each by one load that no condition skips, so that the compiler knows how many are on their way
// behind it: what would end beyond its row is read from further in front and moved when it is stored, and rows beyond the last are the last again.
// Needs rows of a vector or more.
template <class T, Order O, int N, int F, int kThreads> struct Ring {
    typedef Tile<T, O, N> L;
    static constexpr int PER = L::ROWS * L::CHUNKS / kThreads, E = kPer<T>;
    uint64_t offset[O == kAlong ? PER : 1];      // of the lane's row
    int first;                                   // the lane's column, of N as it is read
    int shift;

    __device__ static int chunk(const int i) { return i * kThreads + fresh(threadIdx.x); }

    __device__ void start(const Operand &a, const bool two, const uint32_t n) {
        static_assert(kThreads % L::CHUNKS == 0, "a lane has the same column of all its rows");
        const int col = (int)(threadIdx.x % L::CHUNKS) * E;
        first = col;
        shift = 0;
        if constexpr (O == kAlong) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                constexpr int kHalf = F * 8;
                const int row = (i * kThreads + (int)threadIdx.x) / L::CHUNKS;
                const uint32_t r = n + (two ? row / (2 * kHalf) * kHalf + weight_row<F>(row % kHalf) : row);
                offset[i] = (r < a.rows ? r : a.rows - 1) * a.pitch;
            }
        } else {
            first = (int)n + col;
            const int over = first + E - (int)a.cols;
            if (over > 0) {
                shift = over < E ? over : E;
                first = (int)a.cols - E;
            }
        }
    }
    // Which weight a lane's chunk belongs to, of the forward pass.
    __device__ static bool second(const int i) { return (i * kThreads + (int)threadIdx.x) / L::CHUNKS / (F * 8) % 2 != 0; }

    __device__ void load(raw16 (&v)[PER], const Operand &a, const void *other, const bool two, const uint32_t k) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const T *p = (const T *)a.p;
            if (two && second(i)) p = (const T *)other;
            if constexpr (O == kAlong) {
                const uint32_t col = k + first, end = a.cols - E;
                p += offset[i] + (col < end ? col : end);
            } else {
                const uint32_t row = k + chunk(i) / L::CHUNKS;
                p += (row < a.rows ? row : a.rows - 1) * a.pitch + first;
            }
            v[i] = reinterpret_cast<const Unaligned<T> *>(p)->v;
        }
    }
    // (`k`: where the tile begins that is stored.)
    __device__ void store(char *tile, const raw16 (&v)[PER], const Operand &a, const uint32_t k) const {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = chunk(i);
            raw16 x = v[i];
            asm volatile("" : "+v"(x));      // (or the vectors of the steps behind are moved, and waited for, as soon as this one)
            if constexpr (O == kAlong) {
                if (k + kK<T> > a.cols) {
                    const int over = (int)(k + first) + E - (int)a.cols;
                    x = moved<T>(x, over < 0 ? 0 : over < E ? over : E);
                }
            } else {
                x = moved<T>(x, shift);
                if (k + kK<T> > a.rows && k + q / L::CHUNKS >= a.rows) x = raw16{0, 0, 0, 0};
            }
            *(raw16 *)(tile + L::place(q / L::CHUNKS, q % L::CHUNKS)) = x;
        }
    }
};

// 1 / (1 + exp(-g)).  Where the result is rounded to 16 bits, with the instructions for 2^x and 1 / x, whose last places are lost anyway.
template <class T> __device__ inline float sigmoid(const float g) {
    if constexpr (sizeof(T) == 4) return 1.0f / (1.0f + expf(-g));
    else return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.4426950408889634f * g));
}

// act(g) and its derivative, of SiLU and of the GELU, whose (1 + tanh(y)) / 2 is sigmoid(2 y).  Where the sigmoid is 0 or 1 it is the derivative, and 0 is act(g): the
// other factors, g^2 and g^3 among them, may be infinite there (and g, where it was rounded to 16 bits), and 0 times them is a NaN.
constexpr float kGelu = 1.5957691216057308f, kGeluCube = 0.044715f;      // 2 sqrt(2 / pi)

template <class T> __device__ inline float activate(const int activation, const float g) {
    const float s = sigmoid<T>(activation == BT_ACT_SILU ? g : kGelu * (g + kGeluCube * g * g * g));
    return s == 0.0f ? -0.0f : g * s;
}

template <class T> __device__ inline void activate(const int activation, const float g, float *value, float *slope) {
    float s, inner = 1.0f;
    if (activation == BT_ACT_SILU) s = sigmoid<T>(g);
    else {
        s = sigmoid<T>(kGelu * (g + kGeluCube * g * g * g));
        inner = kGelu * (1.0f + 3.0f * kGeluCube * g * g);
    }
    *value = s == 0.0f ? -0.0f : g * s;
    *slope = s == 0.0f || s == 1.0f ? s : s * (1.0f + g * (1.0f - s) * inner);
}

// The smallest number above 0 that T holds.
template <class T> constexpr float kLeast = 0x1p-149f;
template <> constexpr float kLeast<f16> = 0x1p-24f;
template <> constexpr float kLeast<bf16> = 0x1p-133f;

// h of both products; with ReLU what is kept of them where the gate is closed is 0 too.  An open gate that T would round to 0 is kept as the smallest number
// instead: the backward pass, which has the rounded one, is to find it open.
template <class T> __device__ inline float gated(const int activation, float &g, float &u) {
    if (activation != BT_ACT_RELU) return activate<T>(activation, g) * u;
    const bool closed = g <= 0.0f;
    const float h = closed ? 0.0f : g * u;
    g = closed ? 0.0f : g < kLeast<T> ? kLeast<T> : g;
    u = closed ? 0.0f : u;
    return h;
}

template <class T> __device__ inline void store4(T *p, const int left, const float (&x)[4]) {
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

// N neighbours, whole vectors where there are any.
template <class T, int N> __device__ inline void store_run(T *p, const int left, const float (&x)[N]) {
    constexpr int E = kPer<T> < N ? kPer<T> : N;
#pragma unroll
    for (int i = 0; i < N; i += E) {
        float y[E];
#pragma unroll
        for (int e = 0; e < E; ++e) y[e] = x[i + e];
        if constexpr (E == kPer<T>) {
            if (left > i) store_vec(p + i, left - i, pack<T>(y));
        } else if (left > i) store4(p + i, left - i, y);
    }
}

enum Product { kForward, kGradX, kGradW };

struct GatedJob {
    Operand p[2], q[2];              // (of the forward pass p: both weights; of the others p and q: the first and the second sum, or output)
    void *out[2];                    // h; grad_x; grad_w_gate and grad_w_up
    void *gate, *up;                 // what the forward pass keeps, or NULL
    uint64_t pitch;                  // of all outputs
    uint32_t m, n, k;                // rows and columns of the output (of each), and the summed index (of each sum)
    uint32_t tiles_n, tiles_m;       // of each output
    uint32_t splits;                 // parts of the summed index, each of other workgroups
    uint32_t groups;                 // tiles of all outputs and splits
    uint32_t first, end;             // those of them that the launch has
    float *parts;                    // their sums, [splits, 2 of the forward pass and the weights' gradients, m, n]; with one split NULL
    int activation;
};

template <class T, Product K> constexpr Order kOrderP = K == kForward ? kAlong : kAcross;
template <class T, Product K> constexpr Order kOrderQ = K == kGradW ? kAcross : kAlong;

// The tile of a number, of a workgroup as a rule.  Workgroups go to the eight XCDs in turn, each of which has an L2 of its own: an XCD's are neighbours, in bands
// of four rows of tiles, so that those that run at once share what they read.
struct Place {
    uint32_t m, n, part, split;
};

template <Product K> __device__ inline Place place_of(const GatedJob &a, const uint32_t number, const uint32_t tile_m, const uint32_t tile_n) {
    constexpr uint32_t kXcds = 8, kBand = 4;
    const uint32_t xcd = number % kXcds, more = a.groups % kXcds;
    uint32_t tile = xcd * (a.groups / kXcds) + (xcd < more ? xcd : more) + number / kXcds;
    const uint32_t a_split = a.tiles_m * a.tiles_n * (K == kGradW ? 2 : 1);
    Place at;
    at.split = tile / a_split;
    tile -= at.split * a_split;
    at.part = K == kGradW ? tile / (a.tiles_m * a.tiles_n) : 0;
    tile -= at.part * a.tiles_m * a.tiles_n;
    const uint32_t band = tile / (kBand * a.tiles_n), left = a.tiles_m - band * kBand, high = left < kBand ? left : kBand;
    tile -= band * kBand * a.tiles_n;
    at.m = (band * kBand + tile % high) * tile_m;
    at.n = tile / high * tile_n;
    return at;
}

// Results of two fragments, 32 columns of 16 rows: lane l has columns 4 (l / 16) to 4 (l / 16) + 3 of each, and gets columns 8 (l / 16) to 8 (l / 16) + 7 of
// both, so that four lanes write 64 bytes in a row.  `low`, `high`: of either fragment two results in a word.
__device__ inline raw16 eight_neighbours(uint32_t (&low)[2], uint32_t (&high)[2]) {
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const auto halves = __builtin_amdgcn_permlane32_swap(low[w], high[w], false, false);
        const auto quarters = __builtin_amdgcn_permlane16_swap(halves[0], halves[1], false, false);
        low[w] = quarters[0];
        high[w] = quarters[1];
    }
    return raw16{low[0], low[1], high[0], high[1]};
}

// Fragments of which a lane writes its results together, where that is done.
constexpr int kTogether = 2;

// Stores that a lane makes of each output (h, gate, up; a gradient; a split's sums), in the function below, of a tile that lies inside the output: at the least, since
// it also stores smaller pieces.  What a wait that counts them may rely on: one that counts on more than there are waits for nothing.
template <class T, Product K, int FP, int FQ> constexpr int kStoresAtLeast = K == kForward ? FQ : sizeof(T) == 2 ? FQ * (FP / kTogether) : FQ * FP;

// What becomes of a wave's sums: rows from m on, FQ fragments of 16; columns from n on, FP fragments, of the forward pass half of them columns
// of the gate's product and half the same columns of the other.
template <class T, Product K, int FP, int FQ> __device__ inline void finish(const GatedJob &a, const acc4 (&acc)[FP][FQ], const uint32_t m, const uint32_t n, const Place &of) {
    const int lane = fresh(threadIdx.x) % kWave;
    float *const parts = a.parts ? a.parts + ((uint64_t)of.split * (K == kGradX ? 1 : 2) + of.part) * a.m * a.n : nullptr;
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        const uint32_t row = m + j * 16 + lane % 16;
        if constexpr (K != kForward && sizeof(T) == 2) {
            // Where rows begin on 64-byte boundaries (us, weights' gradients with 8 or 64 bytes in a row: [40, 3008] x 11008 66 and 49, [96, 4096] x 16384 98 and 76;
            // but, where rows do not, [1, 4008] x 16008 71 and 84, [100, 4008] x 16008 109 and 103).  All lanes take part, those beyond the last row too.
            if (!parts && a.pitch % 32 == 0) {
                static_assert(kStoresAtLeast<T, K, FP, FQ> <= FQ * (FP / kTogether));
#pragma unroll
                for (int i = 0; i < FP; i += kTogether) {
                    uint32_t low[2] = {pack2<T>(acc[i][j][0], acc[i][j][1]), pack2<T>(acc[i][j][2], acc[i][j][3])};
                    uint32_t high[2] = {pack2<T>(acc[i + 1][j][0], acc[i + 1][j][1]), pack2<T>(acc[i + 1][j][2], acc[i + 1][j][3])};
                    const raw16 v = eight_neighbours(low, high);
                    const uint32_t col = n + i * 16 + lane / 16 * 8;
                    if (row < a.m) store_vec((T *)a.out[of.part] + row * a.pitch + col, (int)(a.n - col), v);
                }
                continue;
            }
        }
        if (row >= a.m) continue;
        if constexpr (K == kForward) {
            constexpr int N = 2 * FP;      // neighbours that the lane has
            static_assert(kStoresAtLeast<T, K, FP, FQ> <= FQ * ((N + kPer<T> - 1) / kPer<T>));
            const uint32_t col = n + lane / 16 * N;
            const int left = (int)(a.n - col);
            const uint64_t at = row * a.pitch + col;
            if (left <= 0) continue;
            float g[N], u[N], h[N];
#pragma unroll
            for (int i = 0; i < N; ++i) {
                g[i] = acc[i / 4][j][i % 4];
                u[i] = acc[i / 4 + FP / 2][j][i % 4];
            }
            if (parts) {
                store_run<float, N>(parts + at, left, g);
                store_run<float, N>(parts + (uint64_t)a.m * a.n + at, left, u);
                continue;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = gated<T>(a.activation, g[i], u[i]);
            store_run<T, N>((T *)a.out[0] + at, left, h);
            if (a.gate) {
                store_run<T, N>((T *)a.gate + at, left, g);
                store_run<T, N>((T *)a.up + at, left, u);
            }
        } else {
            static_assert(kStoresAtLeast<T, K, FP, FQ> <= FQ * FP);
#pragma unroll
            for (int i = 0; i < FP; ++i) {
                const uint32_t col = n + i * 16 + lane / 16 * 4;
                const int left = (int)(a.n - col);
                const float x[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (left <= 0) continue;
                if (parts) store4(parts + (uint64_t)row * a.n + col, left, x);
                else store4((T *)a.out[of.part] + row * a.pitch + col, left, x);
            }
        }
    }
}

// What the two kernels below share: their waves, tiles and steps.
template <class T, Product K, class S> struct Work {
    typedef Tile<T, kOrderP<T, K>, S::NP> P;
    typedef Tile<T, kOrderQ<T, K>, S::NQ> Q;
    typedef acc4 Sums[S::FP][S::FQ];
    static constexpr int COLS = K == kForward ? S::NP / 2 : S::NP;      // columns of the output in a tile
    static constexpr int SUMS = K == kGradX ? 2 : 1;

    Reader<T, kOrderP<T, K>, S::NP, S::FP> rp;
    Reader<T, kOrderQ<T, K>, S::NQ, S::FQ> rq;
    raw16 p[2][S::FP], q[S::FQ];      // fragments: of P of a tile and the next one, of Q the halves in turn

    __device__ Work() {
        const int wave = threadIdx.x / kWave;
        rp.start((wave / 2) * S::FP * 16);
        rq.start((wave % 2) * S::FQ * 16);
    }
    __device__ void read_p(const char *tile, const int parity) {
#pragma unroll
        for (int i = 0; i < S::FP; ++i) p[parity][i] = rp.read(tile, i);
    }
    __device__ void read_q(const char *tile, const int half) {
#pragma unroll
        for (int j = half * S::FQ / 2; j < (half + 1) * S::FQ / 2; ++j) q[j] = rq.read(tile, j);
    }
    __device__ void multiply(Sums &acc, const int parity, const int half) {
#pragma unroll
        for (int i = 0; i < S::FP; ++i)
#pragma unroll
            for (int j = half * S::FQ / 2; j < (half + 1) * S::FQ / 2; ++j) acc[i][j] = btb::multiply<T>(p[parity][i], q[j], acc[i][j]);
    }

    // The products of two tiles that lie in LDS, with nothing else on its way.
    __device__ void multiply_all(Sums &acc, const char *tile_p, const char *tile_q) {
        read_p(tile_p, 0);
        read_q(tile_q, 0);
        read_q(tile_q, 1);
        multiply(acc, 0, 0);
        multiply(acc, 0, 1);
    }

    // Tiles through registers.
    typedef Staged<T, kOrderP<T, K>, S::NP, S::FP, S::THREADS> ThroughP;
    typedef Staged<T, kOrderQ<T, K>, S::NQ, S::FQ, S::THREADS> ThroughQ;

    // The tiles that begin at k of the summed index, and their products.
    __device__ void staged(const GatedJob &a, const Operand &op, const Operand &oq, const Place &at, const uint32_t k, char *tile_p, char *tile_q, Sums &acc) {
        __syncthreads();
        {
            ThroughP sp;
            sp.load(op, a.p[1], K == kForward, at.n, k);
            sp.store(tile_p);
        }
        {
            ThroughQ sq;
            sq.load(oq, oq, false, at.m, k);
            sq.store(tile_q);
        }
        __syncthreads();
        multiply_all(acc, tile_p, tile_q);
    }

    __device__ static void end(const GatedJob &a, const Sums &acc, const Place &at) {
        const int wave = threadIdx.x / kWave;
        finish<T, K, S::FP, S::FQ>(a, acc, at.m + (wave % 2) * S::FQ * 16, at.n + (wave / 2) * (COLS / S::WP), at);
    }
};

// Of `count` tiles of the summed index, in order, the first of a split: one of an even number, since two share the memory's lines.
__device__ inline uint32_t split_start(const GatedJob &a, const uint32_t split, const uint32_t count) {
    return split == a.splits ? count : (uint32_t)((uint64_t)count * split / a.splits) & ~1u;
}

// Any alignment and any size: tiles go through registers, kDeep of them on their way while one is multiplied; a tile has one of two places in LDS,
// so that one barrier a tile is enough.  Rows of less than a vector, and the weights' gradients, which have few tiles to sum and many workgroups to
// wait beside each other: one tile at a time.  Bound by what loads off the boundaries cost (bf16, us: forward of [40, 3001] x 11003 56, of x 3008 on
// them 37; with one tile on its way 138; with eight as with four) and, in single precision, by the products (forward of [100, 4001] x 16001 327 us, 78
// TFLOP/s).
template <class T, Product K> __global__ __launch_bounds__(Small::THREADS, 2) void gated_any_kernel(const GatedJob a) {
    typedef Work<T, K, Small> W;
    typedef Ring<T, kOrderP<T, K>, Small::NP, Small::FP, Small::THREADS> RingP;
    typedef Ring<T, kOrderQ<T, K>, Small::NQ, Small::FQ, Small::THREADS> RingQ;
    constexpr int kDeep = 4;
    __shared__ __align__(16) char tiles[2][W::P::BYTES + W::Q::BYTES];
    const Place at = place_of<K>(a, a.first + blockIdx.x, Small::NQ, W::COLS);
    typename W::Sums acc = {};
    W w;
    const uint32_t a_sum = (a.k + kK<T> - 1) / kK<T>, last = split_start(a, at.split + 1, a_sum * W::SUMS);
    uint32_t t = split_start(a, at.split, a_sum * W::SUMS);
    const auto sum_of = [&](const uint32_t i) { return W::SUMS == 2 && i >= a_sum ? 1u : 0u; };
    const auto start_of = [&](const uint32_t i) { return (i - sum_of(i) * a_sum) * kK<T>; };
    if (K == kGradW || a.p[0].cols < kPer<T> || a.q[0].cols < kPer<T>) {
        for (; t < last; ++t) w.staged(a, a.p[sum_of(t)], a.q[sum_of(t) + at.part], at, start_of(t), tiles[0], tiles[0] + W::P::BYTES, acc);
        W::end(a, acc, at);
        return;
    }
    RingP rp;
    RingQ rq;
    rp.start(a.p[0], K == kForward, at.n);
    rq.start(a.q[0], false, at.m);
    raw16 p[kDeep][RingP::PER], q[kDeep][RingQ::PER];
    const auto load = [&](raw16 (&to_p)[RingP::PER], raw16 (&to_q)[RingQ::PER], const uint32_t i) {
        rp.load(to_p, a.p[sum_of(i)], a.p[1].p, K == kForward, start_of(i));
        rq.load(to_q, a.q[sum_of(i) + at.part], nullptr, false, start_of(i));
    };
    const auto step = [&](const raw16 (&from_p)[RingP::PER], const raw16 (&from_q)[RingQ::PER], const int place) {
        rp.store(tiles[place], from_p, a.p[0], start_of(t));
        rq.store(tiles[place] + W::P::BYTES, from_q, a.q[0], start_of(t));
        __syncthreads();
        ++t;
    };
    // (Of a short sum the last tile several times: a condition here would be one that the compiler's count of loads has to allow for in every turn.)
    if (t < last) {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) load(p[j], q[j], t + j < last ? t + j : last - 1);
    }
#pragma unroll 1
    while (t + kDeep < last) {
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            step(p[j], q[j], j % 2);
            const uint32_t next = t + kDeep - 1;
            load(p[j], q[j], next < last ? next : last - 1);
            w.multiply_all(acc, tiles[j % 2], tiles[j % 2] + W::P::BYTES);
        }
    }
#pragma unroll
    for (int j = 0; j < kDeep; ++j) {
        if (t >= last) break;
        step(p[j], q[j], j % 2);
        w.multiply_all(acc, tiles[j % 2], tiles[j % 2] + W::P::BYTES);
    }
    W::end(a, acc, at);
}

// An operand's tiles straight from memory to LDS, 1 KiB an instruction of a wave, an equal part of the tile a wave.  Needs rows of whole vectors on
// 16-byte boundaries.  What a tile has beyond the operand's rows (or, where the summed index lies across, columns) is read from inside of it: it
// belongs to rows or columns of the product that are not stored.
template <class T, Order O, int N, int WAVES, bool ROUND> struct Direct {
    typedef Tile<T, O, N> L;
    static constexpr int S = (int)sizeof(T), PER = N / 16 / WAVES;
    uint32_t offset[PER];        // of the lane's vector in each instruction's KiB, from the tile's first
    const char *base;
    uint64_t advance, round;     // bytes from one tile to the next; of all tiles
    uint32_t ahead;              // tiles before the first one is next

    // `n`: the product's row or column that the tile begins at.  F: of the forward pass, whose weights' rows are those of `n` on in another order.
    template <int F = 0> __device__ void start(const Operand &a, const uint32_t n) {
        const int lane = fresh(threadIdx.x) % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = (wave * PER + i) * kWave + lane, chunk = (L::place(q / L::CHUNKS, q % L::CHUNKS) / kVec) % L::CHUNKS;
            uint32_t row = q / L::CHUNKS, col = chunk * kPer<T>;
            if constexpr (F != 0) row = weight_row<F>(row % (8 * F));
            if (O == kAlong && n + row >= a.rows) row = 0;
            if (O == kAcross && n + col >= a.cols) col = 0;
            offset[i] = (uint32_t)(row * a.pitch + col) * S;
        }
        base = (const char *)a.p + (O == kAlong ? n * a.pitch : (uint64_t)n) * S;
        advance = (O == kAlong ? kK<T> : kK<T> * a.pitch) * S;
    }
    // The forward pass: rows of the two weights in turn, 8 F of each.  The loading wave's part of the tile is one such run.
    template <int F> __device__ void start_pair(const Operand &gate, const Operand &up, const uint32_t n) {
        static_assert(2 * PER == F, "a wave's part belongs to one weight");
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        const uint32_t first = n + wave / 2 * F * 8;         // row of the weight that the part begins with
        const Operand &a = wave % 2 ? up : gate;
        start<F>(a, first < a.rows ? first : 0);
    }
    // The next tile's descriptor.
    __device__ __amdgpu_buffer_rsrc_t next() {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, 0x7fffffff, 0x00020000);
        base += advance;
        if (ROUND && --ahead == 0) base -= round;
        return r;
    }
    __device__ void piece(const __amdgpu_buffer_rsrc_t r, char *tile, const int i) const {
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (BT_LDS void *)(tile + (wave * PER + i) * 1024), 16, (int)offset[i], 0, 0, 0);
    }
    __device__ void fetch(char *tile) {
        const __amdgpu_buffer_rsrc_t r = next();
#pragma unroll
        for (int i = 0; i < PER; ++i) piece(r, tile, i);
    }
    // The next tile and the one after it, piece by piece.
    __device__ void fetch(char *tile, char *after) {
        const __amdgpu_buffer_rsrc_t r = next(), s = next();
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            piece(r, tile, i);
            piece(s, after, i);
        }
    }
    // Begin at tile `at` of the `count` from `first` on; with ROUND the tiles before it come last.
    __device__ void rotate(const uint32_t first, const uint32_t at, const uint32_t count) {
        base += (uint64_t)(first + at) * advance;
        ahead = count - at;
        round = (uint64_t)count * advance;
    }
};

// Until all but the last `LEFT` of this wave's fetches have landed, then for the other waves: their fetches have landed too, and they have read
// what they need of the tiles before.
constexpr int kFetchesNever = 64;      // (all are known to have)

template <int LEFT> __device__ inline void wait_for_tiles() {
    static_assert(LEFT <= kFetchesNever);
    asm volatile("" ::: "memory");           // (the barrier itself keeps the compiler's loads and stores from nothing)
    if (LEFT < kFetchesNever) __builtin_amdgcn_s_waitcnt(0x0f70 | (LEFT & 15) | (LEFT >> 4 & 3) << 14);      // vmcnt
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Tiles of either operand in LDS, the next ones on their way while one is multiplied.  A tile's products are made in two halves (of Q's
// fragments).  While the first is made, the second's fragments are read and further tiles are asked for, while the second is made, the next
// tile's first fragments are read; behind the barrier between them a tile's place has been read by all.  The instructions of either kind
// are spread among the products: each waits for the unit that takes it, and a wave that waits for that multiplies nothing.
//
// With the summed index along the rows a tile has half of each 128-byte line that it touches, and a line asked for a tile later is fetched again from
// the L2 where that has other things to hold in between.  The forward pass in tiles of 64, whose weights nothing else reads, asks for two tiles at a time,
// in every second one, piece by piece, and has five places (f16 forward of [37, 4096] x 11003: 50 -> 46 us); larger tiles ask for one in each and have
// four: with two the bf16 forward pass of [16384, 2048] x 8192 took the same time, and grad_x has no registers for it.
//
// That holds for the forward pass and for single precision.  In 16 bits grad_x and the weights' gradients read fragments of the operands that lie across by the
// transposing reads, which the compiler takes for reads of what any fetch may write: it waits for all of a wave's fetches behind the barrier of each step, those that
// were asked for half a step ago too, and at a tile's start for the stores of the one before.  The waits below have to be right without that one: it says nothing of other
// waves' fetches.
template <int KIND, int COUNT, int PRODUCTS, int GROUPS, int G = 0> __device__ inline void spread_kind() {
    if constexpr (G < GROUPS) {
        constexpr int c = COUNT * (G + 1) / GROUPS - COUNT * G / GROUPS, m = PRODUCTS * (G + 1) / GROUPS - PRODUCTS * G / GROUPS;
        __builtin_amdgcn_sched_group_barrier(KIND, c, 0);
        if constexpr (m != 0) __builtin_amdgcn_sched_group_barrier(0x8, m, 0);
        spread_kind<KIND, COUNT, PRODUCTS, GROUPS, G + 1>();
    }
}

// The schedule of a half: `READS` reads of LDS, then `FETCHES` fetches (which the compiler takes for writes to what is read), among `PRODUCTS`
// products.
template <int READS, int FETCHES, int PRODUCTS> __device__ inline void spread() {
    constexpr int kFirst = PRODUCTS * READS / (READS + FETCHES), kSecond = PRODUCTS - kFirst;
    spread_kind<0x100, READS, kFirst, (READS < kFirst ? READS : kFirst)>();
    if constexpr (FETCHES != 0) spread_kind<0x10, FETCHES, kSecond, (FETCHES < kSecond ? FETCHES : kSecond)>();
}

template <int N, int I = 0, class Go> __device__ inline void turn(Go go) {
    if constexpr (I < N) {
        go(std::integral_constant<int, I>{});
        turn<N, I + 1>(go);
    }
}

// Bound by the matrix units (and, in the largest forward passes, by the power that they take: they are busy for 59 to 62 % of the cycles at 1.9 GHz), in 16 bits grad_x and
// the weights' gradients by them and the full wait in every step (61 and 66 %).  bf16, tiles of 256 by 256: forward of [16384, 1024] x 4096 232 us, 1185 TFLOP/s, of
// [16384, 2048] x 8192 with gate and up kept 977 us, 1125; grad_x of the latter 892 us, 1233, its weights' gradients 825 us, 1333 (on a
// slower card 241, 1061, 948 and 886); instructions for 32 by 32 results, which read half as many registers, 4 % slower;
// four waves of 128 by 128, 667; 256 by 128, two workgroups a compute unit, 8 % slower.  Single precision, tiles of 64 by 64: [1024, 2048] x 8192 537 to 554
// us each, 124 to 128 TFLOP/s.  Smaller sizes take smaller tiles, and parts of the sum each, so that there is work for all compute units: see plan_of.
template <class T, Product K, class S> __global__ __launch_bounds__(S::THREADS, S::FQ == 8 ? 2 : 1) void gated_kernel(const GatedJob a) {
    typedef Work<T, K, S> W;
    // Rows of a power of two of bytes all begin in the same channel of the memory, and workgroups in step would ask one after the other: each XCD
    // begins elsewhere in the summed index (us: forward [16384, 2048] x 8192 1045 -> 970, grad_x 915 -> 885), or with few rows each of 64
    // workgroups.  The weights' gradients sum over rows, and have no registers for it.
    constexpr bool kRound = K != kGradW;
    typedef Direct<T, kOrderP<T, K>, S::NP, S::WAVES, kRound> FetchP;
    typedef Direct<T, kOrderQ<T, K>, S::NQ, S::WAVES, kRound> FetchQ;
    constexpr bool kTwo = K == kForward && S::FQ == 2;
    constexpr int kPlaces = kTwo ? 5 : S::PLACES, kTurn = kPlaces % 2 == 0 ? kPlaces : 2 * kPlaces;
    constexpr int kAhead = kPlaces - 1, kLeft = kTwo ? 2 : kAhead - 1;      // from a tile to the furthest that it asks for; tiles that may be on their way behind the next
    constexpr int PB = W::P::BYTES, QB = W::Q::BYTES, kFetches = FetchP::PER + FetchQ::PER;      // kFetches: instructions of a tile
    constexpr int kReadsP = S::FP * Reader<T, kOrderP<T, K>, S::NP, S::FP>::READS, kReadsQ = S::FQ / 2 * Reader<T, kOrderQ<T, K>, S::NQ, S::FQ>::READS;
    constexpr int kProducts = S::FP * S::FQ / 2 * (sizeof(T) == 4 ? 4 : 1);
    __shared__ __align__(1024) char tiles[kPlaces * (PB + QB)];
    W w;
    FetchP dp;
    FetchQ dq;
    const uint32_t a_sum = a.k / kK<T>;      // whole tiles
    const uint32_t phases = a.tiles_m == 1 ? 64 : 8;
    const auto tile_p = [&](const int t) { return tiles + t % kPlaces * PB; };
    const auto tile_q = [&](const int t) { return tiles + kPlaces * PB + t % kPlaces * QB; };
    // The first tiles of a sum are asked for; returns how many there are.
    const auto begin = [&](const Place &at, const int sum) {
        const uint32_t from = split_start(a, at.split, a_sum * W::SUMS), to = split_start(a, at.split + 1, a_sum * W::SUMS);
        const uint32_t before = sum * a_sum, behind = before + a_sum, first = from > before ? from : before, last = to < behind ? to : behind;
        if (first >= last) return 0u;
        const uint32_t count = last - first, phase = kRound ? (uint32_t)((uint64_t)(blockIdx.x % phases) * count / phases) & ~1u : 0;
        if constexpr (K == kForward) dp.template start_pair<S::FP>(a.p[0], a.p[1], at.n);
        else dp.start(a.p[sum], at.n);
        dq.start(a.q[sum + at.part], at.m);
        dp.rotate(first - before, phase, count);
        dq.rotate(first - before, phase, count);
#pragma unroll
        for (int t = 0; t < kAhead; ++t)
            if ((uint32_t)t < count) {
                dp.fetch(tile_p(t));
                dq.fetch(tile_q(t));
            }
        return count;
    };
    // Workgroups of the largest tiles, one to a compute unit, take several: the next one's first tiles of the summed index are asked for before
    // the results of this one are worked out and stored.
    uint32_t number = a.first + blockIdx.x;
    Place at = place_of<K>(a, number, S::NQ, W::COLS);
    uint32_t count = begin(at, 0);
    bool stored = false;      // since the first tiles were asked for: by each lane, kStores of each output or more
    constexpr int kStores = kStoresAtLeast<T, K, S::FP, S::FQ>;
    for (;;) {
        typename W::Sums acc = {};
        // Tile i of a turn, which lies in place i % kPlaces, with `left` tiles from it to the end.
        const auto tile = [&](auto turn_number, const uint32_t left) {
            constexpr int i = decltype(turn_number)::value;
            constexpr bool kAsks = !kTwo || i % 2 == 1;
            w.read_q(tile_q(i), 1);
            if (kTwo && kAsks && left > 4) {
                dp.fetch(tile_p(i + 3), tile_p(i + 4));
                dq.fetch(tile_q(i + 3), tile_q(i + 4));
            } else if (kAsks && left > (kTwo ? 3 : kAhead)) {
                dp.fetch(tile_p(i + (kTwo ? 3 : kAhead)));
                dq.fetch(tile_q(i + (kTwo ? 3 : kAhead)));
            }
            w.multiply(acc, i & 1, 0);
            spread<kReadsQ, kAsks ? (kTwo ? 2 : 1) * kFetches : 0, kProducts>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): the last fragments of this tile are here
            // The next tile has come: what is asked for behind it may still be on its way.  (Of two that were asked for together the second came
            // with the first.)
            if (!kAsks) wait_for_tiles<kFetchesNever>();
            else if (left > kAhead) wait_for_tiles<kLeft * kFetches>();
            else wait_for_tiles<0>();
            w.read_p(tile_p(i + 1), (i + 1) & 1);      // (behind the last tile: what lies there, unused)
            w.read_q(tile_q(i + 1), 0);
            w.multiply(acc, i & 1, 1);
            spread<kReadsP + kReadsQ, 0, kProducts>();
            __builtin_amdgcn_sched_barrier(0);
        };
        bool through = false;      // registers
        for (int sum = 0; sum < W::SUMS; ++sum) {
            if (sum != 0) {
                __syncthreads();
                count = begin(at, sum);
            }
            if (count != 0) {
                // The first tile of every wave has to be in LDS.  Fetches and stores are counted together, in order: of those that may still be on their way,
                // the first tile's fetches are followed by those of kLeft tiles and by the stores.
                if (count < kAhead) wait_for_tiles<0>();
                else if (!stored || sum != 0) wait_for_tiles<kLeft * kFetches>();
                else if (K == kForward && a.gate && !a.parts) wait_for_tiles<kLeft * kFetches + (K == kForward ? 3 : 1) * kStores>();
                else wait_for_tiles<kLeft * kFetches + kStores>();
                w.read_p(tile_p(0), 0);
                w.read_q(tile_q(0), 0);
                __builtin_amdgcn_sched_barrier(0);
                uint32_t t = 0;
                for (; t + kTurn + kAhead <= count; t += kTurn) turn<kTurn>([&](auto i) { tile(i, kTurn + kAhead); });
                for (; t < count; t += kTurn)
                    turn<kTurn>([&](auto i) {
                        if (t + decltype(i)::value < count) tile(i, count - t - decltype(i)::value);
                    });
            }
            // The rest of the summed index, less than a tile, through registers: of the split that has the last whole tile, or the only one.
            const uint32_t behind = (sum + 1) * a_sum;
            if (a_sum * kK<T> < a.k && (a.splits == 1 || (split_start(a, at.split, a_sum * W::SUMS) < behind && behind <= split_start(a, at.split + 1, a_sum * W::SUMS)))) {
                w.staged(a, a.p[sum], a.q[sum + at.part], at, a_sum * kK<T>, tiles, tiles + PB, acc);
                through = true;
            }
        }
        const Place here = at;
        number += gridDim.x;
        const bool more = number < a.end;
        if (more) {
            if (through) __syncthreads();
            at = place_of<K>(a, number, S::NQ, W::COLS);
            count = begin(at, 0);
            asm volatile("" ::: "memory");      // (the stores stay behind the fetches: see the wait that counts both)
        }
        W::end(a, acc, here);
        if (!more) break;
        stored = sizeof(T) == 2 && here.m + S::NQ <= a.m && here.n + W::COLS <= a.n;
    }
}

// Few rows (tokens to answer with): the weights are read once and bound the time, so they go from memory to the registers that multiply them, as many
// vectors at once as those hold.  A workgroup has 16 columns of h, its waves take units of 128 bytes of the summed index in turn; their sums
// meet in LDS.  In a unit a lane holds 32 bytes in a row of each operand: which summed index belongs to which lane does not matter as long as both
// have the same; in single precision, whose products take longer, two vectors 64 bytes apart, so that an instruction asks for whole lines (20 rows of
// [11003, 3001]: 110 -> 84 us).  Any alignment; ODD: rows of an odd number of 16-bit elements, from a 4-byte boundary on.  (bf16, weights of [4096, 1024],
// 1 row: 4.7 us, 3.6 TB/s; of [16384, 4096], 52.8 us, 5.1 TB/s; of [11008, 4096], 16 rows: 42 us, 4.3 TB/s.  32 columns a workgroup, which read x half
// as often: 59 and 63.  From 33 rows on tiles in LDS are faster.)
constexpr int kTokenWaves = 8;
template <class T> constexpr int kUnit = 128 / (int)sizeof(T);

template <class T, int FQ, bool ODD> __global__ __launch_bounds__(kTokenWaves * kWave) void gated_tokens_kernel(const GatedJob a) {
    constexpr int kUnits = 4;      // on their way at once
    constexpr int kLane = sizeof(T) == 4 ? kPer<T> : 2 * kPer<T>, kNext = sizeof(T) == 4 ? 4 * kPer<T> : kPer<T>;      // from one lane's first vector to the next one's, to its second
    __shared__ float sums[kTokenWaves][2][FQ][kWave][4];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), group = lane / 16, t = lane % 16;
    const uint32_t n = blockIdx.x * 16;
    const T *p[2], *q[FQ];
    // (Rows that are not there are others again: their results are not stored.)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        p[i] = (const T *)a.p[i].p + (n + t < a.n ? n + t : a.n - 1) * a.p[i].pitch + group * kLane;
    }
#pragma unroll
    for (int j = 0; j < FQ; ++j) q[j] = (const T *)a.q[0].p + (uint64_t)((uint32_t)(j * 16 + t) < a.m ? j * 16 + t : a.m - 1) * a.q[0].pitch + group * kLane;
    bool odd_p[2], odd_q[FQ];      // where a lane's vectors are read from the element before (`k` is even)
#pragma unroll
    for (int i = 0; i < 2; ++i) odd_p[i] = ODD && ((uintptr_t)p[i] & 2) != 0;
#pragma unroll
    for (int j = 0; j < FQ; ++j) odd_q[j] = ODD && ((uintptr_t)q[j] & 2) != 0;
    acc4 acc[2][FQ] = {};
    // The workgroups begin in different places of the summed index, or all would ask the same channels of the memory at a time.
    const uint32_t whole = a.k / kUnit<T>, shift = whole == 0 ? 0 : blockIdx.x * kTokenWaves % whole;
    uint32_t unit = wave;
    const auto take = [&](auto many) {
        constexpr int N = decltype(many)::value;
        raw16 w[N][2][2], x[N][FQ][2];
        uint32_t w_end[N][2], x_end[N][FQ];
#pragma unroll
        for (int s = 0; s < N; ++s) {
            uint32_t at = unit + s * kTokenWaves + shift;
            if (at >= whole) at -= whole;
            const uint64_t k = (uint64_t)at * kUnit<T>;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < 2; ++i) w[s][i][h] = reinterpret_cast<const Unaligned<T> *>(p[i] + k + h * kNext - (odd_p[i] ? 1 : 0))->v;
#pragma unroll
                for (int j = 0; j < FQ; ++j) x[s][j][h] = reinterpret_cast<const Unaligned<T> *>(q[j] + k + h * kNext - (odd_q[j] ? 1 : 0))->v;
            }
            if constexpr (ODD) {
#pragma unroll
                for (int i = 0; i < 2; ++i) w_end[s][i] = bits_at(p[i] + k + (2 * kPer<T> - 1));
#pragma unroll
                for (int j = 0; j < FQ; ++j) x_end[s][j] = bits_at(q[j] + k + (2 * kPer<T> - 1));
            }
        }
        __builtin_amdgcn_sched_barrier(0);      // (all of them before the first product)
        const auto move = [&](raw16 (&v)[2], const uint32_t end, const bool odd) {
            v[0] = from_odd<T>(v[0], v[1][0], odd);
            v[1] = from_odd<T>(v[1], end, odd);
        };
#pragma unroll
        for (int s = 0; s < N; ++s) {
            if constexpr (ODD) {
#pragma unroll
                for (int i = 0; i < 2; ++i) move(w[s][i], w_end[s][i], odd_p[i]);
#pragma unroll
                for (int j = 0; j < FQ; ++j) move(x[s][j], x_end[s][j], odd_q[j]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < FQ; ++j) acc[i][j] = multiply<T>(w[s][i][h], x[s][j][h], acc[i][j]);
        }
        unit += N * kTokenWaves;
    };
    while (unit + (kUnits - 1) * kTokenWaves < whole) take(std::integral_constant<int, kUnits>{});
    while (unit < whole) take(std::integral_constant<int, 1>{});
    if (wave == 0 && whole * kUnit<T> < a.k) {      // the rest, less than a unit
        const uint32_t k = whole * kUnit<T>;
        const int left = (int)(a.k - k) - group * kLane;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            raw16 w[2], x[FQ];
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i] = load_vec(p[i] + k + h * kNext, left - h * kNext, (int)a.k - left + h * kNext);
#pragma unroll
            for (int j = 0; j < FQ; ++j) x[j] = load_vec(q[j] + k + h * kNext, left - h * kNext, (int)a.k - left + h * kNext);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < FQ; ++j) acc[i][j] = multiply<T>(w[i], x[j], acc[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < FQ; ++j) *(acc4 *)sums[wave][i][j][lane] = acc[i][j];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < FQ * 256; c += kTokenWaves * kWave) {
        const uint32_t col = c % 16, token = c / 16, from = col / 4 * 16 + token % 16, r = col % 4, j = token / 16;
        float g = 0.0f, u = 0.0f;
#pragma unroll
        for (int w = 0; w < kTokenWaves; ++w) {
            g += sums[w][0][j][from][r];
            u += sums[w][1][j][from][r];
        }
        if (token >= a.m || n + col >= a.n) continue;
        const uint64_t at = token * a.pitch + n + col;
        ((T *)a.out[0])[at] = narrow<T>(gated<T>(a.activation, g, u));
        if (a.gate) {
            ((T *)a.gate)[at] = narrow<T>(g);
            ((T *)a.up)[at] = narrow<T>(u);
        }
    }
}

// The splits' sums added up, in order, and what becomes of them.  `cells` elements of each output, which has no gaps.  Bound by memory, and where there
// is little by the launch (two splits of [37, 11003], forward: 4.7 us).
// Several splits are on their way at once (a power of two, as their number is); small sums go to workgroups of one wave, for there to be some on all compute
// units (16 splits of [64, 1001], grad_x: 7.6 us one split at a time with 256 threads, 4.0 now; 8 of [1024, 2048], bound by memory: 12.0 to 12.6 with 256 threads, 13.0 with
// 64).
template <class T, Product K> __global__ __launch_bounds__(256) void gated_join_kernel(const GatedJob a, const uint64_t cells) {
    constexpr int E = kPer<T>, kSums = K == kGradX ? 1 : 2;
    const uint64_t c = ((uint64_t)blockIdx.x * blockDim.x + threadIdx.x) * E;
    if (c >= cells) return;
    const int left = cells - c < 64 ? (int)(cells - c) : 64;
    float x[kSums][E] = {};
    const auto add = [&](auto at_once) {
        constexpr int N = decltype(at_once)::value;
        for (uint32_t split = 0; split < a.splits; split += N) {
            raw16 v[N][kSums][E / 4];
#pragma unroll
            for (int s = 0; s < N; ++s)
#pragma unroll
                for (int k = 0; k < kSums; ++k)
#pragma unroll
                    for (int e = 0; e < E; e += 4)
                        v[s][k][e / 4] = reinterpret_cast<const Unaligned<float> *>(a.parts + ((split + s) * kSums + k) * cells + c + e)->v;
#pragma unroll
            for (int s = 0; s < N; ++s)
#pragma unroll
                for (int k = 0; k < kSums; ++k)
#pragma unroll
                    for (int e = 0; e < E; ++e) x[k][e] += __builtin_bit_cast(float, (uint32_t)v[s][k][e / 4][e % 4]);
        }
    };
    if (left >= E) {
        if (a.splits >= 8) add(std::integral_constant<int, 8 / kSums>{});
        else if (a.splits >= 4) add(std::integral_constant<int, 4>{});
        else add(std::integral_constant<int, 2>{});
    } else for (uint32_t split = 0; split < a.splits; ++split)
#pragma unroll
        for (int k = 0; k < kSums; ++k)
#pragma unroll
            for (int e = 0; e < E; e += 4) {
                float y[4];
                unpack<float>(load_vec(a.parts + (split * kSums + k) * cells + c + e, left - e, (c != 0 ? 4 : 0) + e), y);
#pragma unroll
                for (int i = 0; i < 4; ++i) x[k][e + i] += y[i];
            }
    if constexpr (K == kForward) {
        float h[E];
#pragma unroll
        for (int e = 0; e < E; ++e) h[e] = gated<T>(a.activation, x[0][e], x[1][e]);
        store_vec((T *)a.out[0] + c, left, pack<T>(h));
        if (a.gate) {
            store_vec((T *)a.gate + c, left, pack<T>(x[0]));
            store_vec((T *)a.up + c, left, pack<T>(x[1]));
        }
    } else {
#pragma unroll
        for (int k = 0; k < kSums; ++k) store_vec((T *)a.out[k] + c, left, pack<T>(x[k]));
    }
}

// Rows of `cols` elements, one behind the other, to rows of `pitch`, zeros behind them: where rows are to begin on 16-byte boundaries.  Up to
// three matrices a launch, blockIdx.y.  Bound by memory (single precision, both weights of [2731, 1001] and x of [500, 1001]: 9.1 us, 5.2 TB/s).
struct PadJob {
    const void *from[3];
    void *to[3];
    uint32_t rows[3], cols, pitch;
};

template <class T> __global__ __launch_bounds__(256) void pad_kernel(const PadJob a) {
    const uint32_t a_row = a.pitch / kPer<T>;
    const uint64_t vectors = (uint64_t)a.rows[blockIdx.y] * a_row;
    const T *const from = (const T *)a.from[blockIdx.y];
    T *const to = (T *)a.to[blockIdx.y];
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / a_row;
        const uint32_t col = (uint32_t)(i - row * a_row) * kPer<T>;
        store_vec(to + i * kPer<T>, kPer<T>, load_vec(from + row * a.cols + col, (int)(a.cols - col), (int)col));
    }
}

// dg = grad_h u act'(g) and du = grad_h act(g), rounded to the type: they are factors of the products, whose matrix instructions take them so (in two
// parts each they would be twice the work).  With gate and up, rounded between the passes, that makes the gradients of bf16 [16384, 2048] x 8192 off by 0.0031 of them, in the mean of
// squares, and a form in 32 bits that is rounded at its end by 0.0017.  In f16 they also have its range: beyond 65504 an infinity, below 6e-5 fewer bits, as if they
// were the tensors that a step made of single operators has there.  Rows of `pitch` elements, whole vectors.  Bound by memory
// ([16384, 8192] in bf16: 258 us, 5.2 TB/s).
template <class T> __global__ __launch_bounds__(256) void gated_slopes_kernel(const T *grad_h, const T *gate, const T *up, T *dg, T *du,
                                                                             const uint32_t f, const uint32_t pitch, const uint64_t vectors, const int activation) {
    const uint32_t a_row = pitch / kPer<T>;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / a_row;
        const uint32_t col = (uint32_t)(i - row * a_row) * kPer<T>;
        const uint64_t at = row * f + col;
        float h[kPer<T>], g[kPer<T>], u[kPer<T>];
        unpack<T>(load_vec(grad_h + at, (int)(f - col), (int)col), h);
        unpack<T>(load_vec(gate + at, (int)(f - col), (int)col), g);
        unpack<T>(load_vec(up + at, (int)(f - col), (int)col), u);
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

// Elements of a row that is padded to whole tiles of the summed index.
uint64_t padded(const uint64_t cols, const int width) { return (cols * width + kKBytes - 1) / kKBytes * kKBytes / width; }

bt_status check_sizes(const uint64_t rows, const uint64_t d, const uint64_t f, const bt_dtype dtype) {
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (rows > BT_MAX_ROWS || d > BT_MAX_FEATURES || f > BT_MAX_FEATURES) return BT_ERR_SIZE;
    return BT_OK;
}

bool known(const bt_activation a) { return a == BT_ACT_RELU || a == BT_ACT_SILU || a == BT_ACT_GELU_TANH; }

uint64_t ceil_div(const uint64_t a, const uint64_t b) { return (a + b - 1) / b; }

// How a product of m by n with a summed index of k (of each of `sums` sums) is run, by its sizes alone.
enum Kind { kAnyKind, kSmall, kMiddle, kLarge };
struct Plan {
    Kind kind;
    uint32_t splits;
};

// By a model of the time, us, whose constants are measured: what a compute unit multiplies in tiles of either size (of 5.9 TFLOP/s in 16 bits, 0.6 in
// single precision), a tile's step when nothing else runs beside it, and for the splits a launch and their sums' way to memory and back.  Single precision has the
// smallest tiles alone: they reach 0.8 of that rate, and larger ones would only leave more of the last turn idle.
Plan plan_of(const Product product, const uint64_t m, const uint64_t n, const uint64_t k, const int width, const bool any) {
    struct Form {
        Kind kind;
        int rows, cols, together;      // rows and columns of a tile, workgroups that a compute unit holds
        double rate, alone;
    };
    const bool single = width == 4;
    static const Form forms[] = {{kSmall, 64, 64, 4, 0.33, 0.28}, {kMiddle, 128, 128, 2, 0.6, 0.38}, {kLarge, 256, 256, 1, 0.95, 0.75}};
    const double peak = single ? 0.6e6 : 5.9e6;                                  // operations a us of a compute unit
    const uint64_t steps = ceil_div(k * width, kKBytes) * (product == kGradX ? 2 : 1), outputs = product == kGradX ? 1 : 2;
    Plan best = {kSmall, 1};
    double least = 1e300;
    for (const Form &f : forms) {
        if (f.kind != kSmall && (any || single)) break;
        const uint64_t tiles = ceil_div(m, f.rows) * ceil_div(n, product == kForward ? f.cols / 2 : f.cols) * (product == kGradW ? 2 : 1);
        for (uint32_t splits = 1; splits <= 32 && (splits == 1 || (steps / splits >= 8 && tiles * splits <= 4096)); splits *= 2) {
            const double work = 2.0 * f.rows * f.cols * (kKBytes / width) * (double)steps / splits;      // of a workgroup
            const double a_unit = (double)ceil_div(tiles * splits, 256);
            const double rate = single ? 0.8 : f.rate;
            double time = a_unit * work / (peak * rate);
            const double alone = (double)steps / splits * (any ? 0.3 : f.alone) * (double)ceil_div((uint64_t)a_unit, f.together);
            if (time < alone) time = alone;
            if (splits > 1) time += (any ? 5.0 : 4.0) + (double)splits * m * n * outputs * 8.0 / 4e6;
            if (time < least) {
                least = time;
                best = {f.kind, splits};
            }
        }
    }
    if (any) best.kind = kAnyKind;
    return best;
}

// Rows of x up to which the forward pass reads the weights straight to registers.
constexpr uint64_t kTokens = 32;

// Rows from which on operands whose rows do not begin on 16-byte boundaries are copied to ones that do.  (A copy is read and written once, a weight's
// two elements for each that a product of few rows reads anyway.)
constexpr uint64_t kPadRows = 128;

// Of x alone, for the weights' gradients (bf16, us, copied or not: [40, 3001] x 11003 87 and 65, [100, 4001] x 16001 152 and 160).
constexpr uint64_t kPadRowsX = 96;

bool ragged(const uint64_t d, const int width) { return d * width % kVec != 0; }
bool pads(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows >= kPadRows; }
bool pads_x(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows >= kPadRowsX; }
bool any_way(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows < kPadRows; }

uint64_t whole(const uint64_t bytes) { return (bytes + 127) / 128 * 128; }

uint64_t parts_bytes(const Product product, const uint64_t m, const uint64_t n, const uint64_t k, const int width, const bool any) {
    const uint32_t splits = plan_of(product, m, n, k, width, any).splits;
    return splits == 1 ? 0 : whole(4 * m * n * splits * (product == kGradX ? 1 : 2));
}

// What is to be copied to rows of `pitch`, and where to.
template <class T> struct Pads {
    PadJob job = {};
    int count = 0;

    T *add(char **ws, const void *from, const uint64_t rows, const uint64_t pitch, const bool wanted = true) {
        T *const to = (T *)*ws;
        *ws += whole(rows * pitch * sizeof(T));
        if (wanted) {
            job.from[count] = from;
            job.to[count] = to;
            job.rows[count++] = (uint32_t)rows;
        }
        return to;
    }
    bt_status run(const uint64_t cols, const uint64_t pitch, hipStream_t hs) {
        job.cols = (uint32_t)cols;
        job.pitch = (uint32_t)pitch;
        uint64_t most = 1;
        for (int i = 0; i < count; ++i) most = job.rows[i] > most ? job.rows[i] : most;
        const uint64_t blocks = ceil_div(most * (pitch / kPer<T>), 256);
        return launch(pad_kernel<T>, dim3((unsigned)(blocks < 1u << 14 ? blocks : 1u << 14), (unsigned)count), 256, hs, job);
    }
};

// Rows of whole vectors on 16-byte boundaries, and a tile within 32 bits of offsets.
template <class T> bool direct(const Operand &a) {
    return !misaligned(a.p, kVec) && a.pitch % kPer<T> == 0 && a.pitch * sizeof(T) * 320 < 1u << 31;
}

// An odd number of (16-bit) elements from each row to the next, the first on a 4-byte boundary.
bool odd_rows(const Operand &a) { return a.pitch % 2 != 0 && !misaligned(a.p, 4); }

template <class T, Product K> bt_status run_product(GatedJob &a, const Plan &plan, float *parts, hipStream_t hs) {
    bool straight = direct<T>(a.p[0]) && direct<T>(a.q[0]);
    if (K != kGradW) straight = straight && direct<T>(a.p[1]);
    if (K != kForward) straight = straight && direct<T>(a.q[1]);
    a.splits = plan.splits;
    a.parts = plan.splits > 1 ? parts : nullptr;
    const auto go = [&](auto kernel, auto shape) {
        typedef decltype(shape) S;
        const uint64_t tiles_m = ceil_div(a.m, S::NQ), tiles_n = ceil_div(a.n, K == kForward ? S::NP / 2 : S::NP);
        const uint64_t groups = tiles_m * tiles_n * (K == kGradW ? 2 : 1) * a.splits;
        if (groups >= 1u << 31) return BT_ERR_SIZE;      // (outputs of terabytes)
        a.tiles_m = (uint32_t)tiles_m;
        a.tiles_n = (uint32_t)tiles_n;
        a.groups = (uint32_t)groups;
        constexpr bool kSeveral = S::THREADS == Large::THREADS;      // tiles to a workgroup, 256 of those at the most
        constexpr uint32_t kMost = kSeveral ? 1u << 31 : 1u << 22;   // of a launch: a grid holds less than 2^32 threads
        bt_status s = BT_OK;
        for (a.first = 0; a.first < a.groups && s == BT_OK; a.first = a.end) {
            a.end = a.groups - a.first < kMost ? a.groups : a.first + kMost;
            const uint32_t here = a.end - a.first;
            s = launch(kernel, dim3(kSeveral && here > 256 ? 256 : here), S::THREADS, hs, a);
        }
        return s;
    };
    bt_status st = BT_OK;
    if (!straight || plan.kind == kAnyKind) st = go(gated_any_kernel<T, K>, Small{});
    else if (sizeof(T) == 4 || plan.kind == kSmall) st = go(gated_kernel<T, K, Small>, Small{});
    else if constexpr (sizeof(T) == 2) st = plan.kind == kMiddle ? go(gated_kernel<T, K, Middle>, Middle{}) : go(gated_kernel<T, K, Large>, Large{});
    if (st != BT_OK || a.splits == 1) return st;
    const uint64_t cells = (uint64_t)a.m * a.n;
    const int threads = cells / kPer<T> < 256 * 512 ? kWave : 256;      // (two workgroups of 256 a compute unit or more)
    return launch(gated_join_kernel<T, K>, dim3((unsigned)ceil_div(cells, threads * kPer<T>)), threads, hs, a, cells);
}

}  // namespace
}  // namespace btb

using namespace btb;

extern "C" {

size_t bt_gated_workspace_bytes(uint64_t rows, uint64_t d, uint64_t f, bt_dtype dtype, int backward) {
    if (check_sizes(rows, d, f, dtype) != BT_OK || rows == 0 || f == 0) return 0;
    const int w = width_of(dtype);
    const bool copies = pads(rows, d, w), any = any_way(rows, d, w);
    const uint64_t pitch = padded(d, w);
    uint64_t bytes = copies || (backward && pads_x(rows, d, w)) ? whole(rows * pitch * w) : 0;
    if (copies) bytes += 2 * whole(f * pitch * w);
    if (!backward && rows <= kTokens) return 0;
    if (!backward) return (size_t)(bytes + parts_bytes(kForward, rows, f, copies ? pitch : d, w, any));
    bytes += 2 * whole(rows * padded(f, w) * w);
    const uint64_t x = parts_bytes(kGradX, rows, d, f, w, any), weights = parts_bytes(kGradW, f, d, rows, w, ragged(d, w) && !pads_x(rows, d, w));
    return (size_t)(bytes + (x > weights ? x : weights));
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
        const hipStream_t hs = (hipStream_t)stream;
        char *ws = (char *)d_workspace;
        const void *x = d_x, *w_gate = d_w_gate, *w_up = d_w_up;
        uint64_t pitch = d;
        bt_status s = BT_OK;
        if (pads(rows, d, sizeof(T))) {
            pitch = padded(d, sizeof(T));
            Pads<T> copies;
            x = copies.add(&ws, d_x, rows, pitch);
            w_gate = copies.add(&ws, d_w_gate, f, pitch);
            w_up = copies.add(&ws, d_w_up, f, pitch);
            s = copies.run(d, pitch, hs);
            if (s != BT_OK) return s;
        }
        GatedJob a = {};
        a.p[0] = {w_gate, pitch, (uint32_t)f, (uint32_t)pitch};
        a.p[1] = {w_up, pitch, (uint32_t)f, (uint32_t)pitch};
        a.q[0] = {x, pitch, (uint32_t)rows, (uint32_t)pitch};
        a.out[0] = d_h;
        a.gate = d_gate;
        a.up = d_up;
        a.pitch = f;
        a.m = (uint32_t)rows;
        a.n = (uint32_t)f;
        a.k = (uint32_t)pitch;
        a.activation = activation;
        if (rows <= kTokens) {
            const dim3 grid((unsigned)ceil_div(f, 16));
            const auto go = [&](auto kernel) { return launch(kernel, grid, kTokenWaves * kWave, hs, a); };
            if constexpr (sizeof(T) == 2)
                if (odd_rows(a.p[0]) && odd_rows(a.p[1]) && odd_rows(a.q[0])) return rows <= 16 ? go(gated_tokens_kernel<T, 1, true>) : go(gated_tokens_kernel<T, 2, true>);
            return rows <= 16 ? go(gated_tokens_kernel<T, 1, false>) : go(gated_tokens_kernel<T, 2, false>);
        }
        return run_product<T, kForward>(a, plan_of(kForward, rows, f, pitch, sizeof(T), any_way(rows, d, sizeof(T))), (float *)ws, hs);
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
    if (rows != 0 && f != 0) {
        if (d_grad_h == nullptr || d_gate == nullptr || d_up == nullptr || d_workspace == nullptr ||
            (d_grad_x && (d_w_gate == nullptr || d_w_up == nullptr)) || (d_grad_w_gate && d_x == nullptr))
            return BT_ERR_NULL;
        if (workspace_bytes < bt_gated_workspace_bytes(rows, d, f, dtype, 1)) return BT_ERR_WORKSPACE;
    }
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (rows == 0 || f == 0) {      // sums of nothing
            bt_status s = d_grad_x ? zeros<T>(d_grad_x, rows * d, hs) : BT_OK;
            if (s == BT_OK && d_grad_w_gate) s = zeros<T>(d_grad_w_gate, f * d, hs);
            if (s == BT_OK && d_grad_w_up) s = zeros<T>(d_grad_w_up, f * d, hs);
            return s;
        }
        char *ws = (char *)d_workspace;
        const auto take = [&](const uint64_t elements) {
            T *const p = (T *)ws;
            ws += whole(elements * sizeof(T));
            return p;
        };
        const uint64_t pitch_f = padded(f, sizeof(T)), vectors = rows * pitch_f / kPer<T>, blocks = ceil_div(vectors, 256);
        T *const dg = take(rows * pitch_f), *const du = take(rows * pitch_f);
        bt_status s = launch(gated_slopes_kernel<T>, dim3((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20)), 256, hs, (const T *)d_grad_h, (const T *)d_gate,
                             (const T *)d_up, dg, du, (uint32_t)f, (uint32_t)pitch_f, vectors, (int)activation);
        const bool copies = pads(rows, d, sizeof(T)), any = any_way(rows, d, sizeof(T));
        const void *x = d_x, *w_gate = d_w_gate, *w_up = d_w_up;
        const bool copies_x = pads_x(rows, d, sizeof(T));
        const uint64_t pitch = copies_x ? padded(d, sizeof(T)) : d;
        Pads<T> to;
        if (copies_x) x = to.add(&ws, d_x, rows, pitch, d_grad_w_gate != nullptr);
        if (copies) {
            w_gate = to.add(&ws, d_w_gate, f, pitch, d_grad_x != nullptr);
            w_up = to.add(&ws, d_w_up, f, pitch, d_grad_x != nullptr);
        }
        if (s == BT_OK && to.count != 0) s = to.run(d, pitch, hs);
        if (s == BT_OK && d_grad_x) {
            GatedJob a = {};
            a.p[0] = {w_gate, copies ? pitch : d, (uint32_t)f, (uint32_t)d};
            a.p[1] = {w_up, copies ? pitch : d, (uint32_t)f, (uint32_t)d};
            a.q[0] = {dg, pitch_f, (uint32_t)rows, (uint32_t)f};
            a.q[1] = {du, pitch_f, (uint32_t)rows, (uint32_t)f};
            a.out[0] = d_grad_x;
            a.pitch = d;
            a.m = (uint32_t)rows;
            a.n = (uint32_t)d;
            a.k = (uint32_t)f;
            s = run_product<T, kGradX>(a, plan_of(kGradX, rows, d, f, sizeof(T), any), (float *)ws, hs);
        }
        if (s == BT_OK && d_grad_w_gate) {
            GatedJob a = {};
            a.p[0] = {x, pitch, (uint32_t)rows, (uint32_t)d};
            a.q[0] = {dg, pitch_f, (uint32_t)rows, (uint32_t)f};
            a.q[1] = {du, pitch_f, (uint32_t)rows, (uint32_t)f};
            a.out[0] = d_grad_w_gate;
            a.out[1] = d_grad_w_up;
            a.pitch = d;
            a.m = (uint32_t)f;
            a.n = (uint32_t)d;
            a.k = (uint32_t)rows;
            s = run_product<T, kGradW>(a, plan_of(kGradW, f, d, rows, sizeof(T), ragged(d, sizeof(T)) && !copies_x), (float *)ws, hs);
        }
        return s;
    });
}

}  // extern "C"
