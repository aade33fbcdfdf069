// The gated projections h = act(x Wg^T) * (x Wu^T) and their backward pass: see include/bittrain.h for the contract.
//
// Three products on the matrix cores, all with 32-bit sums:
//   forward    h   [rows, f]   both products of a tile of h in one workgroup, the activation and the product on its registers
//   grad_x     [rows, d]       dg Wg + du Wu: one sum over 2 f
//   grad_w     [2 f, d]        dg^T x and du^T x
// with dg and du computed once, into the workspace, by a pass over grad_h, gate and up.
#include <math.h>

#include "product.h"

namespace btb {
namespace {

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

template <Product K> using FormOf = Form<K == kForward, K == kForward ? kAlong : kAcross, K == kGradW ? kAcross : kAlong, K == kGradX ? 2 : 1>;

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

template <class T, Product K, class S, class Sums> __device__ inline void end(const GatedJob &a, const Sums &acc, const Place &at) {
    constexpr int kCols = Work<T, FormOf<K>, S>::COLS;
    const int wave = threadIdx.x / kWave;
    finish<T, K, S::FP, S::FQ>(a, acc, at.m + (wave % 2) * S::FQ * 16, at.n + (wave / 2) * (kCols / S::WP), at);
}

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
    typedef Work<T, FormOf<K>, Small> W;
    typedef Ring<T, FormOf<K>::P, Small::NP, Small::FP, Small::THREADS> RingP;
    typedef Ring<T, FormOf<K>::Q, Small::NQ, Small::FQ, Small::THREADS> RingQ;
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
        for (; t < last; ++t) w.staged(a.p[sum_of(t)], a.p[1], a.q[sum_of(t) + at.part], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, tiles[0] + W::P::BYTES, acc);
        end<T, K, Small>(a, acc, at);
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
    end<T, K, Small>(a, acc, at);
}

// Bound by the matrix units, by the power that they take (the clock falls to 1.9 GHz) and, the forward pass most, by the wait for the next tile.  bf16, tiles of 256 by 256: forward of [16384, 1024] x
// 4096 232 us, 1185 TFLOP/s, of [16384, 2048] x 8192 with gate and up kept 977 us, 1125 (on a slower card 241 and 1061); grad_x of the latter 763 us, 1441, its weights' gradients 715 us, 1538 (with a wait for all
// fetches in every step, see `transposed`, 859 and 804); instructions for 32 by 32 results, which read half as many registers, 4 % slower;
// four waves of 128 by 128, 667; 256 by 128, two workgroups a compute unit, 8 % slower.  Single precision, tiles of 64 by 64: [1024, 2048] x 8192 537 to 554
// us each, 124 to 128 TFLOP/s.  Smaller sizes take smaller tiles, and parts of the sum each, so that there is work for all compute units: see plan_of.
template <class T, Product K, class S> __global__ __launch_bounds__(S::THREADS, S::FQ == 8 ? 2 : 1) void gated_kernel(const GatedJob a) {
    typedef Work<T, FormOf<K>, S> W;
    // Rows of a power of two of bytes all begin in the same channel of the memory, and workgroups in step would ask one after the other: each XCD
    // begins elsewhere in the summed index (us: forward [16384, 2048] x 8192 1045 -> 970, grad_x 915 -> 885), or with few rows each of 64
    // workgroups.  The weights' gradients sum over rows, and have no registers for it.
    constexpr bool kRound = K != kGradW;
    typedef Direct<T, FormOf<K>::P, S::NP, S::WAVES, kRound> FetchP;
    typedef Direct<T, FormOf<K>::Q, S::NQ, S::WAVES, kRound> FetchQ;
    constexpr bool kTwo = K == kForward && S::FQ == 2;
    constexpr int kPlaces = kTwo ? 5 : S::PLACES, kTurn = kPlaces % 2 == 0 ? kPlaces : 2 * kPlaces;
    constexpr int kAhead = kPlaces - 1, kLeft = kTwo ? 2 : kAhead - 1;      // from a tile to the furthest that it asks for; tiles that may be on their way behind the next
    constexpr int PB = W::P::BYTES, QB = W::Q::BYTES, kFetches = FetchP::PER + FetchQ::PER;      // kFetches: instructions of a tile
    constexpr int kReadsP = S::FP * Reader<T, FormOf<K>::P, S::NP, S::FP>::READS, kReadsQ = S::FQ / 2 * Reader<T, FormOf<K>::Q, S::NQ, S::FQ>::READS;
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
                w.staged(a.p[sum], a.p[1], a.q[sum + at.part], at.n, at.m, a_sum * kK<T>, tiles, tiles + PB, tiles + PB, acc);
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
        end<T, K, S>(a, acc, here);
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

// ---- host ------------------------------------------------------------------------------------------------------

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

bool pads(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows >= kPadRows; }
bool pads_x(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows >= kPadRowsX; }
bool any_way(const uint64_t rows, const uint64_t d, const int width) { return ragged(d, width) && rows < kPadRows; }

uint64_t parts_bytes(const Product product, const uint64_t m, const uint64_t n, const uint64_t k, const int width, const bool any) {
    const uint32_t splits = plan_of(product, m, n, k, width, any).splits;
    return splits == 1 ? 0 : whole(4 * m * n * splits * (product == kGradX ? 1 : 2));
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
