// What the products on the matrix cores share (gated.hip, experts.hip): steps, tiles in LDS, ways from memory to LDS, schedules, activations, copies.
#ifndef BT_PRODUCT_H
#define BT_PRODUCT_H

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
constexpr int kKBytes = 64;                                  // of the summed index in a step, and in a tile where it is not said otherwise (KB)
template <class T, int KB = kKBytes> constexpr int kK = KB / (int)sizeof(T);

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

template <class T, Order O, int N, int KB = kKBytes> struct Tile {      // N rows or columns of the product
    static constexpr int ROWS = O == kAlong ? N : kK<T, KB>;
    static constexpr int CHUNKS = (O == kAlong ? KB : N * (int)sizeof(T)) / kVec;      // of a row
    static constexpr int BYTES = ROWS * CHUNKS * kVec;

    // (Of the rows that one fragment has, those of a lane share the key.)
    __host__ __device__ static constexpr int place(const int row, const int chunk) {
        int key = 0;
        if constexpr (O == kAlong) key = (row >> 1) & (KB == kKBytes ? 2 : 7);
        else if constexpr (sizeof(T) == 2 && CHUNKS == 8) key = 2 * (((row >> 1) & 1) | ((row >> 2) & 2));
        else if constexpr (sizeof(T) == 2) key = 2 * ((row & 3) | ((row >> 1) & 4));
        else key = 4 * ((row >> 2) & 3);
        return (row * CHUNKS + (chunk ^ key)) * kVec;
    }
};

// The transposing read.  __restrict, which says that no fetch writes what is read while it is: without it the compiler takes the read for one of what any fetch on its way may write, and waits for all of them in every
// step.  That the tile has landed is for the waits in the kernels to see to, which count fetches.
__device__ __attribute__((always_inline)) inline short4v transposed(BT_LDS short4v *__restrict from) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(from); }

// A wave's fragments of a tile: F times 16 rows or columns from `first` on.  Where a lane reads depends on the fragment and the tile by constants
// alone, but for one address (summed index along) or one a fragment (across).
template <class T, Order O, int N, int F, int KB = kKBytes> struct Reader {
    typedef Tile<T, O, N, KB> L;
    static constexpr int STEPS = KB / kKBytes, ROW = L::CHUNKS * kVec, READS = O == kAlong ? 1 : sizeof(T) == 2 ? 2 : 4;      // instructions a fragment
    uint32_t at[O == kAlong ? STEPS : F];

    __device__ void start(const int first) {
        const int lane = threadIdx.x % kWave, group = lane / 16, t = lane % 16;
        if constexpr (O == kAlong) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) at[s] = L::place(first + t, s * 4 + group);
        } else {
#pragma unroll
            for (int i = 0; i < F; ++i) {
                const int n = first + i * 16;
                if constexpr (sizeof(T) == 2) at[i] = L::place(group * 8 + t / 4, (n + t % 4 * 4) / 8) + t % 2 * 8;
                else at[i] = L::place(group * 4, (n + t) / 4) + t % 4 * 4;
            }
        }
    }

    // The operand's tiles begin `bytes` into the LDS, as the compiler is not to know: it would add the constants of beyond 64 KiB up to a register for each read.
    __device__ void move(const uint32_t bytes) {
#pragma unroll
        for (uint32_t &a : at) a = fresh(a + bytes);
    }

    // Fragment i of a step of the tile.
    __device__ raw16 read(const char *tile, const int i, const int step = 0) const {
        if constexpr (O == kAlong) {
            return *(const raw16 *)(tile + at[step] + i * 16 * ROW);
        } else if constexpr (sizeof(T) == 2) {
            // 16 lanes read 4 summed indices by 16 columns, 4 columns a lane, and get one column each
            typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
            const char *const from = tile + at[i] + step * kK<T> * ROW;
            const uint2v low = __builtin_bit_cast(uint2v, transposed((BT_LDS short4v *)from));
            const uint2v high = __builtin_bit_cast(uint2v, transposed((BT_LDS short4v *)(from + 4 * ROW)));
            return raw16{low[0], low[1], high[0], high[1]};
        } else {
            raw16 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = *(const uint32_t *)(tile + at[i] + (step * kK<T> + j) * ROW);
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

// A kind of product: whether P has rows of two weights in turn, how the summed index lies in either operand, and how many sums are added up.
template <bool PAIR_, Order P_, Order Q_, int SUMS_> struct Form {
    static constexpr bool PAIR = PAIR_;
    static constexpr Order P = P_, Q = Q_;
    static constexpr int SUMS = SUMS_;
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

// The row of an operand in memory: here its own number.
struct InOrder {
    __device__ uint32_t operator()(const uint32_t row) const { return row; }
};

// Chunks of a tile on their way from memory to LDS, in registers.  (F: of the forward pass, fragments of a wave.)
template <class T, Order O, int N, int F, int kThreads, int KB = kKBytes> struct Staged {
    typedef Tile<T, O, N, KB> L;
    static constexpr int PER = L::ROWS * L::CHUNKS / kThreads;
    raw16 v[PER];

    // `n`: the product's row or column that the tile begins at, `k`: the summed index.  `two`: the forward pass, each wave's rows half of one
    // weight and half of the other.
    template <class Map> __device__ void load(const Operand &a, const Operand &other, const bool two, const uint32_t n, const uint32_t k, const Map &rows) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = i * kThreads + fresh(threadIdx.x), row = q / L::CHUNKS, col = (q % L::CHUNKS) * kPer<T>;
            if constexpr (O == kAlong) {
                constexpr int kHalf = F * 8;      // rows of a wave that belong to one weight
                const Operand &from = two && (row / kHalf) % 2 ? other : a;
                const uint32_t r = n + (two ? row / (2 * kHalf) * kHalf + weight_row<F>(row % kHalf) : row);
                v[i] = raw16{0, 0, 0, 0};
                if (r < from.rows) v[i] = load_vec((const T *)from.p + rows(r) * from.pitch + k + col, (int)(from.cols - k) - col, (int)k + col);
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

    template <class Map = InOrder> __device__ void start(const Operand &a, const bool two, const uint32_t n, const Map &rows = {}) {
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
                offset[i] = rows(r < a.rows ? r : a.rows - 1) * a.pitch;
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

// What the kernels of a product share: their waves, tiles and steps.
template <class T, class F, class S, int KB = kKBytes> struct Work {
    typedef Tile<T, F::P, S::NP, KB> P;
    typedef Tile<T, F::Q, S::NQ, KB> Q;
    typedef acc4 Sums[S::FP][S::FQ];
    static constexpr int COLS = F::PAIR ? S::NP / 2 : S::NP;      // columns of the output in a tile
    static constexpr int SUMS = F::SUMS;

    Reader<T, F::P, S::NP, S::FP, KB> rp;
    Reader<T, F::Q, S::NQ, S::FQ, KB> rq;
    raw16 p[2][S::FP], q[S::FQ];      // fragments: of P of a tile and the next one, of Q the halves in turn

    __device__ Work() {
        const int wave = threadIdx.x / kWave;
        rp.start((wave / 2) * S::FP * 16);
        rq.start((wave % 2) * S::FQ * 16);
    }
    __device__ void read_p(const char *tile, const int parity, const int step = 0) {
#pragma unroll
        for (int i = 0; i < S::FP; ++i) p[parity][i] = rp.read(tile, i, step);
    }
    __device__ void read_q(const char *tile, const int half, const int step = 0) {
#pragma unroll
        for (int j = half * S::FQ / 2; j < (half + 1) * S::FQ / 2; ++j) q[j] = rq.read(tile, j, step);
    }
    __device__ void multiply(Sums &acc, const int parity, const int half) {
#pragma unroll
        for (int i = 0; i < S::FP; ++i)
#pragma unroll
            for (int j = half * S::FQ / 2; j < (half + 1) * S::FQ / 2; ++j) acc[i][j] = btb::multiply<T>(p[parity][i], q[j], acc[i][j]);
    }

    // The products of two tiles that lie in LDS, with nothing else on its way.
    __device__ void multiply_all(Sums &acc, const char *tile_p, const char *tile_q) {
#pragma unroll
        for (int step = 0; step < KB / kKBytes; ++step) {
            read_p(tile_p, 0, step);
            read_q(tile_q, 0, step);
            read_q(tile_q, 1, step);
            multiply(acc, 0, 0);
            multiply(acc, 0, 1);
        }
    }

    // Tiles through registers.
    typedef Staged<T, F::P, S::NP, S::FP, S::THREADS, KB> ThroughP;
    typedef Staged<T, F::Q, S::NQ, S::FQ, S::THREADS, KB> ThroughQ;

    // The tiles that begin at column n and row m of the output and at k of the summed index, and their products.  (`other`: of a pair the second weight; `from_q`: as the reader, which
    // may have been moved, is to be given tile_q.)
    template <class MapP = InOrder, class MapQ = InOrder>
    __device__ void staged(const Operand &op, const Operand &other, const Operand &oq, const uint32_t n, const uint32_t m, const uint32_t k, char *tile_p, char *tile_q,
                           const char *from_q, Sums &acc, const MapP &rows_p = {}, const MapQ &rows_q = {}) {
        __syncthreads();
        {
            ThroughP sp;
            sp.load(op, other, F::PAIR, n, k, rows_p);
            sp.store(tile_p);
        }
        {
            ThroughQ sq;
            sq.load(oq, oq, false, m, k, rows_q);
            sq.store(tile_q);
        }
        __syncthreads();
        multiply_all(acc, tile_p, from_q);
    }
};

// An operand's tiles straight from memory to LDS, 1 KiB an instruction of a wave, an equal part of the tile a wave.  Needs rows of whole vectors on
// 16-byte boundaries.  What a tile has beyond the operand's rows (or, where the summed index lies across, columns) is read from inside of it: it
// belongs to rows or columns of the product that are not stored.
template <class T, Order O, int N, int WAVES, bool ROUND, int KB = kKBytes> struct Direct {
    typedef Tile<T, O, N, KB> L;
    static constexpr int S = (int)sizeof(T), PER = N * KB / 1024 / WAVES;
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
        advance = (O == kAlong ? kK<T, KB> : kK<T, KB> * a.pitch) * S;
    }
    // Rows that do not lie one behind the other: those of `map` from n on, of the a.rows that there are.
    template <class Map> __device__ void start_rows(const Operand &a, const uint32_t n, const Map &map) {
        static_assert(O == kAlong);
        const int lane = fresh(threadIdx.x) % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int q = (wave * PER + i) * kWave + lane, chunk = (L::place(q / L::CHUNKS, q % L::CHUNKS) / kVec) % L::CHUNKS;
            const uint32_t row = n + q / L::CHUNKS < a.rows ? n + q / L::CHUNKS : n;
            offset[i] = (uint32_t)(map(row) * a.pitch + chunk * kPer<T>) * S;
        }
        base = (const char *)a.p;
        advance = kK<T, KB> * S;
    }
    // The forward pass: rows of the two weights in turn, 8 F of each.  The loading wave's part of the tile is one such run.
    template <int F> __device__ void start_pair(const Operand &gate, const Operand &up, const uint32_t n) {
        static_assert(N / WAVES == 8 * F, "a wave's part belongs to one weight");
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
inline uint64_t padded(const uint64_t cols, const int width) { return (cols * width + kKBytes - 1) / kKBytes * kKBytes / width; }

bt_status check_sizes(const uint64_t rows, const uint64_t d, const uint64_t f, const bt_dtype dtype) {
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (rows > BT_MAX_ROWS || d > BT_MAX_FEATURES || f > BT_MAX_FEATURES) return BT_ERR_SIZE;
    return BT_OK;
}

bool known(const bt_activation a) { return a == BT_ACT_RELU || a == BT_ACT_SILU || a == BT_ACT_GELU_TANH; }

uint64_t ceil_div(const uint64_t a, const uint64_t b) { return (a + b - 1) / b; }

bool ragged(const uint64_t d, const int width) { return d * width % kVec != 0; }

uint64_t whole(const uint64_t bytes) { return (bytes + 127) / 128 * 128; }

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

}  // namespace
}  // namespace btb
#endif  // BT_PRODUCT_H
