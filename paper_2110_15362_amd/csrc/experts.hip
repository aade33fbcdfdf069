// The products of a sublayer of several experts, and their backward passes: see include/bittrain.h for the contract.
//
// As in gated.hip, but for each expert's rows with its own weights: how many rows each has is known on the device alone, so a grid is as large as it could have to be and
// every workgroup finds its expert and tile in the sums of the experts' tiles.  Behind the last expert comes a group of the rows of no expert, whose sum is empty.
#include <math.h>

#include "expert_rules.h"
#include "product.h"
#include "route.h"

namespace btb {
namespace {

static_assert(kStepBytes == kKBytes);

template <Kind K> using FormOf = Form<K == kPair, K <= kPlain ? kAlong : kAcross, K == kWeights ? kAcross : kAlong, K == kBackPair ? 2 : 1>;

struct ExpertJob {
    const void *p[2], *q[2];           // of the first expert, or the first row; p: weights (kWeights: x), q: x, gradients
    uint64_t pitch_p, pitch_q;         // elements from a row to the next
    uint64_t step;                     // elements from one expert's weights (kWeights: gradients) to the next one's
    void *out[2], *gate, *up;
    float *sums;                       // kBack: [rows, n] in single precision instead of out
    uint64_t pitch;                    // of the outputs
    const int32_t *offsets, *source;   // source: forward, x has a row a token; else NULL (the weights' gradients have a copy of x in the rows' order)
    uint32_t experts, rows, tokens;
    uint32_t m, n, k;                  // kWeights: m by n of each expert, k is not used; else n columns and k summed indices
    uint32_t tiles_m, tiles_n, outputs;  // kWeights: tiles of an output, outputs; else tiles_n alone
    uint32_t first;                    // tile that the launch begins with
    float *parts;                      // sums of the parts of tiles, see Round
    uint32_t most_splits;              // parts that a tile may be in
    uint32_t padded_q;                 // kBack: q's rows go on with zeros to the end of a tile, as those of kBackPair do
    int activation;
};

// An expert's rows [first, first + rows).
struct Group {
    uint32_t expert, first, rows;
};

__device__ inline uint32_t bound(const ExpertJob &a, const uint32_t e) {
    const int32_t o = a.offsets[e];
    return o < 0 ? 0 : (uint32_t)o < a.rows ? (uint32_t)o : a.rows;
}

// (By each lane for an expert of its own.)
__device__ inline uint32_t rows_of(const ExpertJob &a, const uint32_t e) {
    const uint32_t first = bound(a, e), end = e < a.experts ? bound(a, e + 1) : a.rows;
    return end > first ? end - first : 0;
}

// (By all lanes for one: the numbers go to scalar registers, and what is addressed with them too.)
__device__ inline Group group_of(const ExpertJob &a, const uint32_t e) {
    return {e, (uint32_t)__builtin_amdgcn_readfirstlane(bound(a, e)), (uint32_t)__builtin_amdgcn_readfirstlane(rows_of(a, e))};
}

// The row of x that a row takes.
struct Taken {
    const int32_t *source;      // of the group's first row; NULL: the rows themselves
    uint32_t tokens;
    __device__ uint32_t operator()(const uint32_t row) const {
        if (source == nullptr) return row;
        const uint32_t t = (uint32_t)source[row];
        return t < tokens ? t : 0;
    }
};

constexpr int kMostExperts = BT_MAX_EXPERTS;

// The experts' tiles of `a_tile` rows, added up: those of expert e are numbered from starts[e] on; starts[experts + 1] is how many there are.  For workgroups that take several tiles.
struct Tiles {
    uint32_t starts[kMostExperts + 2];

    // (A wave's work, and everybody's wait.)
    __device__ void find(const ExpertJob &a, const uint32_t a_tile) {
        if (threadIdx.x < kWave) {
            uint32_t sum = 0;
            for (uint32_t e0 = 0; e0 <= a.experts; e0 += kWave) {
                const uint32_t e = e0 + threadIdx.x, n = e <= a.experts ? (rows_of(a, e) + a_tile - 1) / a_tile : 0, x = before_and(n);
                if (e <= a.experts) starts[e] = sum + x - n;
                sum += __shfl(x, kWave - 1);
            }
            if (threadIdx.x == 0) starts[a.experts + 1] = sum;
        }
        __syncthreads();
    }
    // (The sum of the lanes up to this one.)
    __device__ static uint32_t before_and(uint32_t x) {
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const uint32_t y = __shfl_up(x, d);
            if ((int)(threadIdx.x % kWave) >= d) x += y;
        }
        return x;
    }
    __device__ uint32_t count(const ExpertJob &a) const { return __builtin_amdgcn_readfirstlane(starts[a.experts + 1]); }
    // The group that a tile belongs to, and the tiles before and of it.
    __device__ Group group(const ExpertJob &a, const uint32_t tile, uint32_t *start, uint32_t *tiles) const {
        uint32_t low = 0, high = a.experts + 1;      // starts[low] <= tile < starts[high]
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if ((uint32_t)__builtin_amdgcn_readfirstlane(starts[mid]) <= tile) low = mid;
            else high = mid;
        }
        *start = __builtin_amdgcn_readfirstlane(starts[low]);
        *tiles = __builtin_amdgcn_readfirstlane(starts[low + 1]) - *start;
        return group_of(a, __builtin_amdgcn_readfirstlane(low));
    }
};

// The same for workgroups of one tile: each wave for itself, without LDS and without a wait for the others, 64 experts at a time.
struct TilesOnce {
    uint32_t a_tile, sum;
    // of the last 64 experts that were looked at, the lane's one: from where it begins, rows and tiles up to it and of it
    uint32_t first, rows, upto, n;

    __device__ uint32_t look(const ExpertJob &a, const uint32_t e0) {
        const uint32_t e = e0 + threadIdx.x % kWave;
        first = e <= a.experts ? bound(a, e) : 0;
        const uint32_t end = e < a.experts ? bound(a, e + 1) : a.rows;
        rows = e <= a.experts && end > first ? end - first : 0;
        n = (rows + a_tile - 1) / a_tile;
        upto = Tiles::before_and(n);
        return __builtin_amdgcn_readlane(upto, kWave - 1);
    }
    __device__ void find(const ExpertJob &a, const uint32_t tile_rows) {
        a_tile = tile_rows;
        sum = 0;
        for (uint32_t e0 = 0; e0 <= a.experts; e0 += kWave) sum += look(a, e0);
    }
    __device__ uint32_t count(const ExpertJob &) const { return sum; }
    __device__ Group group(const ExpertJob &a, const uint32_t tile, uint32_t *start, uint32_t *tiles) {
        uint32_t before = 0;
        for (uint32_t e0 = 0;; e0 += kWave) {
            const uint32_t here = a.experts < kWave ? sum : look(a, e0);      // (of so few they have all been looked at)
            if (tile < before + here) {
                const int lane = __builtin_ctzll(__ballot(before + upto > tile));
                *tiles = __builtin_amdgcn_readlane(n, lane);
                *start = before + __builtin_amdgcn_readlane(upto, lane) - *tiles;
                return {e0 + lane, (uint32_t)__builtin_amdgcn_readlane(first, lane), (uint32_t)__builtin_amdgcn_readlane(rows, lane)};
            }
            before += here;
        }
    }
};

// Workgroups that run at once, of a shape.
template <class S> constexpr uint32_t kSlots = 256 * (S::THREADS == 512 ? 1 : S::FQ == 4 ? 2 : 4);

// Parts of a tile's summed index are other workgroups' work where the last tiles, kSlots of which run at once, would leave most compute units idle: the tiles from `full` on are in `splits` parts each, whose sums
// experts_join_kernel adds up.  How many there are follows from the tiles' number, and so from the experts' rows alone.
struct Round {
    uint32_t full, splits, tiles;

    __device__ void find(const uint32_t total, const uint32_t slots, const uint32_t most) {
        full = total / slots * slots;
        const uint32_t rest = total - full;
        splits = 1;
        while (splits < most && rest * splits * 2 <= slots) splits *= 2;
        tiles = full + rest * splits;
    }
};

struct Place {
    Group of;
    uint32_t m, n, part;
    uint32_t slot;      // of a part of a tile: which of the parts' sums are its, of a tile's parts in a row (else beyond them)
};

// Tiles that there are, and the tile of a number.  Workgroups go to the eight XCDs in turn, each of which has an L2 of its own.  Of the 256 tiles that run at once an XCD's are
// neighbours, in bands of four rows of tiles of one expert, so that they share what they read; all XCDs are at the same expert, whose weights then come from memory once, and (the weights' gradients)
// have sums of about the same length.  (256: one tile to a compute unit.)
template <Kind K, class Map> __device__ inline uint32_t tiles_of(const ExpertJob &a, const Map &tiles) {
    if constexpr (K == kWeights) return a.experts * a.outputs * a.tiles_m * a.tiles_n;
    else return tiles.count(a) * a.tiles_n;
}

template <Kind K, class Map> __device__ inline Place tile_of(const ExpertJob &a, Map &tiles, uint32_t tile, const uint32_t tile_m, const uint32_t tile_n) {
    constexpr uint32_t kBand = 4;
    Place at;
    at.slot = ~0u;
    uint32_t rows;
    if constexpr (K == kWeights) {
        const uint32_t a_part = a.tiles_m * a.tiles_n, e = tile / (a_part * a.outputs);
        at.of = group_of(a, e);
        tile -= e * a_part * a.outputs;
        at.part = tile / a_part;
        tile -= at.part * a_part;
        rows = a.tiles_m;
    } else {
        uint32_t start;
        at.of = tiles.group(a, tile / a.tiles_n, &start, &rows);
        at.part = 0;
        tile -= start * a.tiles_n;
    }
    const uint32_t band = tile / (kBand * a.tiles_n), left = rows - band * kBand, high = left < kBand ? left : kBand;
    tile -= band * kBand * a.tiles_n;
    at.m = (band * kBand + tile % high) * tile_m;
    at.n = tile / high * tile_n;
    if (K != kWeights && (at.m >= at.of.rows || at.n >= a.n)) {      // (offsets that do not ascend may add up to anything)
        at.of = {a.experts, 0, 0};
        at.m = at.n = 0;
    }
    return at;
}

template <Kind K, class Map> __device__ inline Place place_of(const ExpertJob &a, Map &tiles, const uint32_t number, const Round &r, const uint32_t tile_m, const uint32_t tile_n) {
    constexpr uint32_t kXcds = 8, kTogether = 256;
    const uint32_t first = number / kTogether * kTogether, here = r.tiles - first < kTogether ? r.tiles - first : kTogether, xcd = number % kXcds, more = here % kXcds;
    const uint32_t item = first + xcd * (here / kXcds) + (xcd < more ? xcd : more) + number % kTogether / kXcds, slot = item - r.full;
    const bool in_parts = item >= r.full;      // (or a whole one of the last)
    Place at = tile_of<K>(a, tiles, in_parts ? r.full + slot / r.splits : item, tile_m, tile_n);
    at.slot = in_parts && r.splits != 1 ? slot : ~0u;
    return at;
}

// The operands of a tile's product, of sum `sum`; rows and summed indices that it has.
template <class T, Kind K> __device__ inline Operand operand_p(const ExpertJob &a, const Group &g, const int sum) {
    if constexpr (K == kWeights) return {(const T *)a.p[0] + g.first * a.pitch_p, a.pitch_p, g.rows, a.n};
    else {
        const T *const w = (const T *)a.p[sum] + (g.expert < a.experts ? g.expert : 0) * a.step;
        if constexpr (K <= kPlain) return {w, a.pitch_p, a.n, a.k};
        else return {w, a.pitch_p, a.k, a.n};
    }
}
template <class T, Kind K> __device__ inline Operand operand_q(const ExpertJob &a, const Group &g, const int sum) {
    const uint64_t first = K <= kPlain && a.source ? 0 : g.first * a.pitch_q;
    return {(const T *)a.q[sum] + first, a.pitch_q, g.rows, K == kWeights ? a.m : a.k};
}
template <Kind K> __device__ inline uint32_t summed(const ExpertJob &a, const Group &g) { return K == kWeights ? g.rows : __builtin_amdgcn_readfirstlane(g.expert < a.experts ? a.k : 0); }
__device__ inline Taken taken(const ExpertJob &a, const Group &g) { return {a.source ? a.source + g.first : nullptr, a.tokens}; }

// Stores that a lane makes of each output in the function below, of a tile that lies inside it: at the least, which is what a wait that counts them may rely on (one that counts on more than there
// are lets a tile be read that has not landed).
template <class T, Kind K, int FP, int FQ> constexpr int kStoresAtLeast = K == kPair ? FQ : sizeof(T) == 2 ? FQ * (FP / kTogether) : FQ * FP;

// What becomes of a wave's sums: rows from m on, FQ fragments of 16; columns from n on, FP fragments, of a pair half of them columns of the gate's product and half the
// same columns of the other.
template <class T, Kind K, int FP, int FQ> __device__ inline void finish(const ExpertJob &a, const acc4 (&acc)[FP][FQ], const uint32_t m, const uint32_t n, const Place &of) {
    const int lane = fresh(threadIdx.x) % kWave;
    const uint32_t rows = K == kWeights ? a.m : of.of.rows;
    const uint64_t first = K == kWeights ? of.of.expert * a.step : of.of.first * a.pitch;      // element that the group's outputs begin with
    T *const out = (T *)a.out[K == kWeights ? of.part : 0] + first;
#pragma unroll
    for (int j = 0; j < FQ; ++j) {
        const uint32_t row = m + j * 16 + lane % 16;
        if constexpr (K != kPair && sizeof(T) == 2) {
            // Where rows begin on 64-byte boundaries four lanes write 64 bytes in a row.  All lanes take part, those beyond the last row too.
            if (!a.sums && a.pitch % 32 == 0) {
                static_assert(kStoresAtLeast<T, K, FP, FQ> <= FQ * (FP / kTogether));
#pragma unroll
                for (int i = 0; i < FP; i += kTogether) {
                    uint32_t low[2] = {pack2<T>(acc[i][j][0], acc[i][j][1]), pack2<T>(acc[i][j][2], acc[i][j][3])};
                    uint32_t high[2] = {pack2<T>(acc[i + 1][j][0], acc[i + 1][j][1]), pack2<T>(acc[i + 1][j][2], acc[i + 1][j][3])};
                    const raw16 v = eight_neighbours(low, high);
                    const uint32_t col = n + i * 16 + lane / 16 * 8;
                    if (row < rows) store_vec(out + row * a.pitch + col, (int)(a.n - col), v);
                }
                continue;
            }
        }
        if (row >= rows) continue;
        if constexpr (K == kPair) {
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
#pragma unroll
            for (int i = 0; i < N; ++i) h[i] = gated<T>(a.activation, g[i], u[i]);
            store_run<T, N>(out + at, left, h);
            if (a.gate) {
                store_run<T, N>((T *)a.gate + first + at, left, g);
                store_run<T, N>((T *)a.up + first + at, left, u);
            }
        } else {
            static_assert(kStoresAtLeast<T, K, FP, FQ> <= FQ * FP);
#pragma unroll
            for (int i = 0; i < FP; ++i) {
                const uint32_t col = n + i * 16 + lane / 16 * 4;
                const int left = (int)(a.n - col);
                const float x[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
                if (left <= 0) continue;
                if (a.sums) store4(a.sums + first + row * a.pitch + col, left, x);
                else store4(out + row * a.pitch + col, left, x);
            }
        }
    }
}

template <class T, Kind K, class S, class Sums> __device__ inline void end(const ExpertJob &a, const Sums &acc, const Place &at) {
    constexpr int kCols = Work<T, FormOf<K>, S>::COLS;
    const int wave = threadIdx.x / kWave;
    finish<T, K, S::FP, S::FQ>(a, acc, at.m + (wave % 2) * S::FQ * 16, at.n + (wave / 2) * (kCols / S::WP), at);
}

// Any alignment and any size: as gated_any_kernel.
template <class T, Kind K> __global__ __launch_bounds__(Small::THREADS, 2) void experts_any_kernel(const ExpertJob a) {
    typedef FormOf<K> F;
    typedef Work<T, F, Small> W;
    typedef Ring<T, F::P, Small::NP, Small::FP, Small::THREADS> RingP;
    typedef Ring<T, F::Q, Small::NQ, Small::FQ, Small::THREADS> RingQ;
    constexpr int kDeep = 4;
    __shared__ __align__(16) char tiles[2][W::P::BYTES + W::Q::BYTES];
    TilesOnce map;
    if constexpr (K != kWeights) map.find(a, Small::NQ);
    const uint32_t total = tiles_of<K>(a, map), number = a.first + blockIdx.x;
    if (number >= total) return;
    const Place at = place_of<K>(a, map, number, Round{total, 1, total}, Small::NQ, W::COLS);
    typename W::Sums acc = {};
    W w;
    const uint32_t k = summed<K>(a, at.of), a_sum = (k + kK<T> - 1) / kK<T>, last = a_sum * W::SUMS;
    uint32_t t = 0;
    const auto sum_of = [&](const uint32_t i) { return W::SUMS == 2 && i >= a_sum ? 1u : 0u; };
    const auto start_of = [&](const uint32_t i) { return (i - sum_of(i) * a_sum) * kK<T>; };
    const Taken rows = taken(a, at.of);
    Operand p[2], q[2];
    for (int s = 0; s < 2; ++s) {
        p[s] = operand_p<T, K>(a, at.of, K == kPair || s < W::SUMS ? s : 0);
        q[s] = operand_q<T, K>(a, at.of, K == kWeights ? at.part : s < W::SUMS ? s : 0);
    }
    if (K == kWeights || p[0].cols < kPer<T> || q[0].cols < kPer<T>) {
        for (; t < last; ++t) {
            const uint32_t s = sum_of(t);
            if constexpr (K == kWeights) w.staged(p[0], p[0], q[0], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, tiles[0] + W::P::BYTES, acc);
            else if constexpr (K <= kPlain) w.staged(p[s], p[1], q[s], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, tiles[0] + W::P::BYTES, acc, InOrder{}, rows);
            else w.staged(p[s], p[1], q[s], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, tiles[0] + W::P::BYTES, acc);
        }
        end<T, K, Small>(a, acc, at);
        return;
    }
    if (t < last) {
        RingP rp;
        RingQ rq;
        rp.start(p[0], K == kPair, at.n);
        if constexpr (K <= kPlain) rq.start(q[0], false, at.m, rows);
        else rq.start(q[0], false, at.m);
        raw16 vp[kDeep][RingP::PER], vq[kDeep][RingQ::PER];
        const auto load = [&](raw16 (&to_p)[RingP::PER], raw16 (&to_q)[RingQ::PER], const uint32_t i) {
            const uint32_t s = sum_of(i);
            rp.load(to_p, s ? p[1] : p[0], p[1].p, K == kPair, start_of(i));
            rq.load(to_q, s ? q[1] : q[0], nullptr, false, start_of(i));
        };
        const auto step = [&](const raw16 (&from_p)[RingP::PER], const raw16 (&from_q)[RingQ::PER], const int place) {
            rp.store(tiles[place], from_p, p[0], start_of(t));
            rq.store(tiles[place] + W::P::BYTES, from_q, q[0], start_of(t));
            __syncthreads();
            ++t;
        };
#pragma unroll
        for (int j = 0; j < kDeep; ++j) load(vp[j], vq[j], t + j < last ? t + j : last - 1);
#pragma unroll 1
        while (t + kDeep < last) {
#pragma unroll
            for (int j = 0; j < kDeep; ++j) {
                step(vp[j], vq[j], j % 2);
                const uint32_t next = t + kDeep - 1;
                load(vp[j], vq[j], next < last ? next : last - 1);
                w.multiply_all(acc, tiles[j % 2], tiles[j % 2] + W::P::BYTES);
            }
        }
#pragma unroll
        for (int j = 0; j < kDeep; ++j) {
            if (t >= last) break;
            step(vp[j], vq[j], j % 2);
            w.multiply_all(acc, tiles[j % 2], tiles[j % 2] + W::P::BYTES);
        }
    }
    end<T, K, Small>(a, acc, at);
}

// An operand's tiles straight from memory to LDS, as a ring: of one sum, begun anywhere, or of two, one behind the other, so that nothing is waited for between them.
// (As two sums in turn, each with its own first fetches, the kernel also had 161 registers too many.)  Where the summed index lies across, the last tile may be a part: what
// its descriptor has not got is zeros.
template <class T, Order O, int N, int WAVES, int KB> struct Looped : Direct<T, O, N, WAVES, false, KB> {
    typedef Direct<T, O, N, WAVES, false, KB> One;
    int64_t way, both;      // bytes from the end of the sum that is being fetched to the start of the next, and of both ways
    uint32_t each, last;    // tiles of a sum; bytes that its last one has
    // Across, of the largest tiles: instructions two apart are four rows apart, in the same order of the chunks, and share their offsets' registers.
    static constexpr bool kShared = O == kAcross && One::PER == 4 && sizeof(T) == 2 && N == 256;
    static_assert(!kShared || One::L::place(4, 1) - One::L::place(0, 1) == 4 * N * (int)sizeof(T));
    uint32_t four;          // rows, in bytes

    __device__ void fetch(char *tile) {
        // (By masks: with branches, or selects of 64 bits, these numbers go to vector registers, and a descriptor that lies there is read in a loop.)
        uint32_t there = 0x7fffffff;
        if constexpr (O == kAcross) there = __builtin_amdgcn_readfirstlane(there ^ ((there ^ last) & (uint32_t)((int32_t)(One::ahead - 2) >> 31)));
        const char *const start = One::base;
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)start, 0, there, 0x00020000);
        --One::ahead;
        const int32_t over = (int32_t)(One::ahead - 1) >> 31;      // all ones behind the last tile of a sum
        const int64_t mask = over;
        One::base += (int64_t)One::advance + (way & mask);
        way ^= (way ^ (both - way)) & mask;
        One::ahead += each & (uint32_t)over;
        if constexpr (kShared) {
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), behind = (int)there - (int)four;
            const __amdgpu_buffer_rsrc_t s = __builtin_amdgcn_make_buffer_rsrc((void *)(start + four), 0, behind > 0 ? behind : 0, 0x00020000);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i < 2 ? r : s, (BT_LDS void *)(tile + (wave * 4 + i) * 1024), 16, (int)One::offset[i % 2], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < One::PER; ++i) One::piece(r, tile, i);
        }
    }
    __device__ static int64_t scalar(const int64_t x) {
        return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x));
    }
    // `second`: bytes from the first sum's operand to the second's, 0 of one sum; `count`: tiles of a sum; begin at tile `at` of all; `k`: the summed index.
    __device__ void rotate(const int64_t second, const uint32_t at, const uint32_t count, const uint32_t k) {
        const int64_t length = (int64_t)(count * One::advance);
        const bool late = at >= count;
        const uint32_t row = (uint32_t)(One::advance / kK<T, KB>);
        each = __builtin_amdgcn_readfirstlane(count);
        last = __builtin_amdgcn_readfirstlane((k - (count - 1) * kK<T, KB>) * row);
        four = __builtin_amdgcn_readfirstlane(4 * row);
        both = scalar(-2 * length);
        way = scalar(late ? -second - length : second - length);
        One::base = (const char *)scalar((int64_t)(One::base + (late ? second : 0) + (late ? at - count : at) * One::advance));
        One::ahead = __builtin_amdgcn_readfirstlane(count - (late ? at - count : at));
    }
};

// Tiles of either operand in LDS, the next ones on their way while one is multiplied, in steps of 64 bytes of the summed index; workgroups of the largest tiles take several.  A step's products are made in two halves
// (of Q's fragments): while the first is made the second's fragments are read, while the second is made the next step's first ones.  Behind the barrier in a tile's last step, between its halves, the next tile has
// landed and all waves have read what they need of this one.  x's rows are fetched from where their tokens have them, or, for the weights' gradients, from a copy in the order of the experts.
//
// The forward pass, both of whose operands have the summed index along their rows, has tiles of whole 128-byte lines, two of them in LDS, and asks for a tile as soon as its place is free.  The others have four of 64
// bytes, and ask for one among the first products of a step.  (us, 32768 rows, eight weights of [2048, 4096] in bf16, both ways: forward 567 and 590, grad_x 545 and 521, the weights' gradients 430 and 405.)
template <Kind K> constexpr int kTileBytes = K <= kPlain ? 2 * kKBytes : kKBytes;
template <Kind K> constexpr int kPlaces = K <= kPlain ? 2 : 4;

template <class T, Kind K, class S> __global__ __launch_bounds__(S::THREADS, S::THREADS == 512 ? 2 : 1) void experts_kernel(const ExpertJob a) {
    constexpr int KB = kTileBytes<K>, PLACES = kPlaces<K>, STEPS = KB / kKBytes, kKs = kK<T, KB>;
    constexpr int kAhead = STEPS == 1 ? PLACES - 1 : PLACES;      // from a tile to the furthest that it asks for
    constexpr int kLeft = STEPS == 1 ? kAhead - 1 : PLACES - 2;   // tiles that may be on their way behind the next
    typedef FormOf<K> F;
    typedef Work<T, F, S, KB> W;
    // Each XCD begins elsewhere in the summed index, as the dense projections do; the weights' gradients sum over rows, of which each expert has other numbers.
    constexpr bool kRound = K != kWeights;
    typedef Looped<T, F::P, S::NP, S::WAVES, KB> FetchP;
    typedef Looped<T, F::Q, S::NQ, S::WAVES, KB> FetchQ;
    constexpr int PB = W::P::BYTES, QB = W::Q::BYTES, kFetches = FetchP::PER + FetchQ::PER;      // kFetches: instructions of a tile
    constexpr int kReadsP = S::FP * Reader<T, F::P, S::NP, S::FP>::READS, kReadsQ = S::FQ / 2 * Reader<T, F::Q, S::NQ, S::FQ>::READS;
    constexpr int kProducts = S::FP * S::FQ / 2 * (sizeof(T) == 4 ? 4 : 1);
    __shared__ __align__(1024) char tiles[PLACES * (PB + QB)];
    constexpr bool kSeveral = S::THREADS == Large::THREADS;      // tiles to a workgroup
    using Map = std::conditional_t<kSeveral && K != kWeights, Tiles, TilesOnce>;      // (the weights' gradients have all experts' tiles: nothing is looked up)
    __shared__ std::conditional_t<std::is_same_v<Map, Tiles>, Tiles, char> shared_map;
    TilesOnce own_map;
    Map &map = [&]() -> Map & {
        if constexpr (std::is_same_v<Map, Tiles>) return shared_map;
        else return own_map;
    }();
    if constexpr (K != kWeights) map.find(a, S::NQ);
    Round r;
    r.find(tiles_of<K>(a, map), kSlots<S>, a.most_splits);
    uint32_t number = a.first + blockIdx.x;
    if (number >= r.tiles) return;
    W w;
    FetchP dp;
    FetchQ dq;
    const auto tile_p = [&](const int t) { return tiles + t % PLACES * PB; };
    const auto tile_q = [&](const int t) { return tiles + PLACES * PB + t % PLACES * QB; };
    const auto read_q = [&](const int t, const int half, const int step) { w.read_q(tiles + t % PLACES * QB, half, step); };
    w.rq.move(PLACES * PB);
    // The rest of the summed index, less than a tile, goes through registers where it lies along an operand's rows (there the next row follows), unless zeros follow (the two-sum and the padded
    // gradients; the other operand, across, has zeros there too).
    const bool whole_only = K <= kPlain || (K == kBack && a.padded_q == 0);
    // A tile's first fetches are asked for; returns how many tiles of the summed index it has.
    const auto begin = [&](const Place &at) {
        const uint32_t k = summed<K>(a, at.of), each = __builtin_amdgcn_readfirstlane(whole_only ? k / kKs : (k + kKs - 1) / kKs);
        uint32_t count = each * F::SUMS, phase = kRound ? (uint32_t)((uint64_t)(blockIdx.x % 8) * count / 8) : 0;
        if (at.slot != ~0u) {
            const uint32_t split = at.slot % r.splits;
            phase = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)count * split / r.splits));
            count = __builtin_amdgcn_readfirstlane((uint32_t)((uint64_t)count * (split + 1) / r.splits)) - phase;
        }
        if (count == 0) return 0u;
        if constexpr (K == kPair) dp.template start_pair<S::FP>(operand_p<T, K>(a, at.of, 0), operand_p<T, K>(a, at.of, 1), at.n);
        else dp.start(operand_p<T, K>(a, at.of, 0), at.n);
        const Operand q = operand_q<T, K>(a, at.of, K == kWeights ? at.part : 0);
        if constexpr (K <= kPlain) {
            if (a.source) dq.start_rows(q, at.m, taken(a, at.of));
            else dq.start(q, at.m);
        } else dq.start(q, at.m);
        dp.rotate(F::SUMS == 2 ? (const char *)a.p[1] - (const char *)a.p[0] : 0, phase, each, k);
        dq.rotate(F::SUMS == 2 ? (const char *)a.q[1] - (const char *)a.q[0] : 0, phase, each, k);
#pragma unroll
        for (int t = 0; t < kAhead; ++t)
            if ((uint32_t)t < count) {
                dp.fetch(tile_p(t));
                dq.fetch(tile_q(t));
            }
        return count;
    };
    Place at = place_of<K>(a, map, number, r, S::NQ, W::COLS);
    uint32_t count = begin(at);
    number += gridDim.x;
    bool stored = false;      // since the first tiles were asked for: by each lane, kStores of each output or more
    constexpr int kStores = kStoresAtLeast<T, K, S::FP, S::FQ>;
    for (;;) {
        // The next tile's place is looked up while this one's first fetches are on their way.
        const bool more = kSeveral && number < r.tiles;
        Place next = at;
        if (more) next = place_of<K>(a, map, number, r, S::NQ, W::COLS);
        typename W::Sums acc = {};
        // Tile i of a turn, which lies in place i % PLACES, with `left` tiles from it to the end.
        const auto tile = [&](auto turn_number, const uint32_t left) {
            constexpr int i = decltype(turn_number)::value, kParity = STEPS == 1 ? i & 1 : 0;
            if constexpr (STEPS == 2) {
                read_q(i, 1, 0);
                w.multiply(acc, 0, 0);
                spread<kReadsQ, 0, kProducts>();
                __builtin_amdgcn_sched_barrier(0);
                w.read_p(tile_p(i), 1, 1);
                read_q(i, 0, 1);
                w.multiply(acc, 0, 1);
                spread<kReadsP + kReadsQ, 0, kProducts>();
                __builtin_amdgcn_sched_barrier(0);
            }
            constexpr int kLast = STEPS == 1 ? kParity : 1, kNext = STEPS == 1 ? 1 - kParity : 0;
            read_q(i, 1, STEPS - 1);
            if (STEPS == 1 && left > kAhead) {
                dp.fetch(tile_p(i + kAhead));
                dq.fetch(tile_q(i + kAhead));
            }
            w.multiply(acc, kLast, 0);
            spread<kReadsQ, STEPS == 1 ? kFetches : 0, kProducts>();
            __builtin_amdgcn_sched_barrier(0);
            __builtin_amdgcn_s_waitcnt(0xc07f);      // lgkmcnt(0): the last fragments of this tile are here
            // The next tile has come: what is asked for behind it may still be on its way.
            if (kLeft != 0 && left > kAhead) wait_for_tiles<kLeft * kFetches>();
            else wait_for_tiles<0>();
            w.read_p(tile_p(i + 1), kNext, 0);      // (behind the last tile: what lies there, unused)
            read_q(i + 1, 0, 0);
            if (STEPS == 2 && left > kAhead) {
                dp.fetch(tile_p(i));
                dq.fetch(tile_q(i));
            }
            w.multiply(acc, kLast, 1);
            spread<kReadsP + kReadsQ, STEPS == 2 ? kFetches : 0, kProducts>();
            __builtin_amdgcn_sched_barrier(0);
        };
        const uint32_t k = summed<K>(a, at.of), rest = whole_only ? k / kKs * kKs : k;
        if (count != 0) {
            // The first tile of every wave has to be in LDS.  Fetches and stores are counted together, in order: of those that may still be on their way, the first tile's fetches are
            // followed by those of the other places and by the stores.
            constexpr int kBehind = (kAhead - 1) * kFetches;
            if (count < kAhead) wait_for_tiles<0>();
            else if (!stored) wait_for_tiles<kBehind>();
            else if (K == kPair && a.gate) wait_for_tiles<kBehind + (K == kPair ? 3 : 1) * kStores>();
            else wait_for_tiles<kBehind + kStores>();
            w.read_p(tile_p(0), 0, 0);
            read_q(0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
            constexpr uint32_t kMany = PLACES + kAhead;
            uint32_t t = 0;
            for (; t + kMany <= count; t += PLACES) turn<PLACES>([&](auto i) { tile(i, kMany); });
            for (; t < count; t += PLACES)
                turn<PLACES>([&](auto i) {
                    if (t + decltype(i)::value < count) tile(i, count - t - decltype(i)::value);
                });
        }
        // The rest of the summed index, less than a tile, through registers.
        const bool in_parts = at.slot != ~0u;
        const bool through = (K <= kPlain || K == kBack) && rest < k && (!in_parts || at.slot % r.splits + 1 == r.splits);
        if (through) {
            const Operand p = operand_p<T, K>(a, at.of, 0), q = operand_q<T, K>(a, at.of, 0);
            if constexpr (K <= kPlain)
                w.staged(p, operand_p<T, K>(a, at.of, 1), q, at.n, at.m, rest, tiles, tiles + PLACES * PB, tiles, acc, InOrder{}, taken(a, at.of));
            else if constexpr (K == kBack) w.staged(p, p, q, at.n, at.m, rest, tiles, tiles + PLACES * PB, tiles, acc);
        }
        const Place here = at;
        if (more) {
            if (through) __syncthreads();
            at = next;
            number += gridDim.x;
            count = begin(at);
            asm volatile("" ::: "memory");      // (the stores stay behind the fetches: see the wait that counts both)
        }
        if (in_parts) {
            float *const to = a.parts + (uint64_t)here.slot * (S::NP * S::NQ) + threadIdx.x * 4;
#pragma unroll
            for (int i = 0; i < S::FP; ++i)
#pragma unroll
                for (int j = 0; j < S::FQ; ++j) *(acc4 *)(to + (i * S::FQ + j) * (S::THREADS * 4)) = acc[i][j];
        } else end<T, K, S>(a, acc, here);
        if (!more) break;
        stored = sizeof(T) == 2 && !in_parts && here.m + S::NQ <= (K == kWeights ? a.m : here.of.rows) && here.n + W::COLS <= a.n;
    }
}

// The parts of the last tiles added up, in order, and what becomes of the sums: kSlice of Q's fragments a workgroup, each lane those that it has in experts_kernel.  Bound by memory.
constexpr int kSlice = 2;

template <class T, Kind K, class S> __global__ __launch_bounds__(S::THREADS) void experts_join_kernel(const ExpertJob a) {
    constexpr int kCols = Work<T, FormOf<K>, S>::COLS, kSlices = S::FQ / kSlice;
    TilesOnce map;
    if constexpr (K != kWeights) map.find(a, S::NQ);
    Round r;
    r.find(tiles_of<K>(a, map), kSlots<S>, a.most_splits);
    const uint32_t tile = blockIdx.x / kSlices, slice = blockIdx.x % kSlices;
    if (r.splits == 1 || tile * r.splits >= r.tiles - r.full) return;
    acc4 acc[S::FP][kSlice] = {};
    const float *const from = a.parts + (uint64_t)tile * r.splits * (S::NP * S::NQ) + slice * kSlice * (S::THREADS * 4) + threadIdx.x * 4;
    for (uint32_t split = 0; split < r.splits; split += 2) {
        acc4 x[2][S::FP][kSlice];
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < S::FP; ++i)
#pragma unroll
                for (int j = 0; j < kSlice; ++j) x[h][i][j] = *(const acc4 *)(from + (uint64_t)(split + h) * (S::NP * S::NQ) + (i * S::FQ + j) * (S::THREADS * 4));
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < S::FP; ++i)
#pragma unroll
                for (int j = 0; j < kSlice; ++j) acc[i][j] += x[h][i][j];
    }
    // (As the place of a whole tile.)
    const Place at = tile_of<K>(a, map, r.full + tile, S::NQ, kCols);
    const int wave = threadIdx.x / kWave;
    finish<T, K, S::FP, kSlice>(a, acc, at.m + (wave % 2) * S::FQ * 16 + slice * kSlice * 16, at.n + (wave / 2) * (kCols / S::WP), at);
}

// Few rows an expert (tokens to answer with): as gated_tokens_kernel, for 16 columns and 16 rows of one expert.  The weights are read once for as many rows and bound
// the time.
constexpr int kTokenWaves = 8;
template <class T> constexpr int kUnit = 128 / (int)sizeof(T);

template <class T, Kind K, bool ODD> __global__ __launch_bounds__(kTokenWaves * kWave) void experts_tokens_kernel(const ExpertJob a) {
    constexpr int N = K == kPair ? 2 : 1;      // weights
    constexpr int kUnits = 4;      // on their way at once (of one weight and 16 rows eight: 21.4 us where four take 18.9, 16 rows at 16 experts, 4096 to 1024 features in bf16)
    constexpr int kLane = sizeof(T) == 4 ? kPer<T> : 2 * kPer<T>, kNext = sizeof(T) == 4 ? 4 * kPer<T> : kPer<T>;      // from one lane's first vector to the next one's, to its second
    __shared__ float sums[kTokenWaves][N][kWave][4];
    TilesOnce map;
    map.find(a, 16);
    const uint32_t tile = (a.first + blockIdx.x) / a.tiles_n, n = ((a.first + blockIdx.x) - tile * a.tiles_n) * 16;
    if (tile >= map.count(a)) return;
    uint32_t start, tiles;
    const Group g = map.group(a, tile, &start, &tiles);
    const uint32_t m = (tile - start) * 16;
    if (m >= g.rows) return;
    const Taken rows = taken(a, g);
    const Operand oq = operand_q<T, K>(a, g, 0);
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), group = lane / 16, t = lane % 16;
    const T *p[N];
    // (Rows that are not there are others again: their results are not stored.)
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Operand op = operand_p<T, K>(a, g, i);
        p[i] = (const T *)op.p + (n + t < a.n ? n + t : a.n - 1) * op.pitch + group * kLane;
    }
    const T *const q = (const T *)oq.p + rows(m + t < g.rows ? m + t : g.rows - 1) * oq.pitch + group * kLane;
    bool odd_p[N];      // where a lane's vectors are read from the element before (`k` is even)
#pragma unroll
    for (int i = 0; i < N; ++i) odd_p[i] = ODD && ((uintptr_t)p[i] & 2) != 0;
    const bool odd_q = ODD && ((uintptr_t)q & 2) != 0;
    acc4 acc[N] = {};
    // The workgroups begin in different places of the summed index, or all would ask the same channels of the memory at a time.
    const uint32_t k_end = summed<K>(a, g), whole = k_end / kUnit<T>, shift = whole == 0 ? 0 : blockIdx.x * kTokenWaves % whole;
    uint32_t unit = wave;
    const auto take = [&](auto many) {
        constexpr int M = decltype(many)::value;
        raw16 w[M][N][2], x[M][2];
        uint32_t w_end[M][N], x_end[M];
#pragma unroll
        for (int s = 0; s < M; ++s) {
            uint32_t at = unit + s * kTokenWaves + shift;
            if (at >= whole) at -= whole;
            const uint64_t k = (uint64_t)at * kUnit<T>;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int i = 0; i < N; ++i) w[s][i][h] = reinterpret_cast<const Unaligned<T> *>(p[i] + k + h * kNext - (odd_p[i] ? 1 : 0))->v;
                x[s][h] = reinterpret_cast<const Unaligned<T> *>(q + k + h * kNext - (odd_q ? 1 : 0))->v;
            }
            if constexpr (ODD) {
#pragma unroll
                for (int i = 0; i < N; ++i) w_end[s][i] = bits_at(p[i] + k + (2 * kPer<T> - 1));
                x_end[s] = bits_at(q + k + (2 * kPer<T> - 1));
            }
        }
        __builtin_amdgcn_sched_barrier(0);      // (all of them before the first product)
        const auto move = [&](raw16 (&v)[2], const uint32_t end, const bool odd) {
            v[0] = from_odd<T>(v[0], v[1][0], odd);
            v[1] = from_odd<T>(v[1], end, odd);
        };
#pragma unroll
        for (int s = 0; s < M; ++s) {
            if constexpr (ODD) {
#pragma unroll
                for (int i = 0; i < N; ++i) move(w[s][i], w_end[s][i], odd_p[i]);
                move(x[s], x_end[s], odd_q);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] = multiply<T>(w[s][i][h], x[s][h], acc[i]);
        }
        unit += M * kTokenWaves;
    };
    while (unit + (kUnits - 1) * kTokenWaves < whole) take(std::integral_constant<int, kUnits>{});
    while (unit < whole) take(std::integral_constant<int, 1>{});
    if (wave == 0 && whole * kUnit<T> < k_end) {      // the rest, less than a unit
        const uint32_t k = whole * kUnit<T>;
        const int left = (int)(k_end - k) - group * kLane;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            raw16 w[N];
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = load_vec(p[i] + k + h * kNext, left - h * kNext, (int)k_end - left + h * kNext);
            const raw16 x = load_vec(q + k + h * kNext, left - h * kNext, (int)k_end - left + h * kNext);
#pragma unroll
            for (int i = 0; i < N; ++i) acc[i] = multiply<T>(w[i], x, acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) *(acc4 *)sums[wave][i][lane] = acc[i];
    __syncthreads();
    for (uint32_t c = threadIdx.x; c < 256; c += kTokenWaves * kWave) {
        const uint32_t col = c % 16, token = c / 16, from = col / 4 * 16 + token, r = col % 4;
        float s[2] = {};
#pragma unroll
        for (int w = 0; w < kTokenWaves; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) s[i] += sums[w][i][from][r];
        if (m + token >= g.rows || n + col >= a.n) continue;
        const uint64_t at = (uint64_t)(g.first + m + token) * a.pitch + n + col;
        if constexpr (K == kPair) {
            ((T *)a.out[0])[at] = narrow<T>(gated<T>(a.activation, s[0], s[1]));
            if (a.gate) {
                ((T *)a.gate)[at] = narrow<T>(s[0]);
                ((T *)a.up)[at] = narrow<T>(s[1]);
            }
        } else ((T *)a.out[0])[at] = narrow<T>(s[0]);
    }
}

// Matrices to rows of `pitch`, zeros behind their `cols`: where rows are to begin on 16-byte boundaries, or to lie in another order.  One for each blockIdx.y.
struct CopyJob {
    const void *from[4];
    void *to[4];
    const int32_t *source[4];      // the row of `from` that a row takes; NULL: its own
    uint32_t rows[4], cols[4], pitch[4];
    uint32_t tokens;               // rows of `from` where there is a source
};

template <class T> __global__ __launch_bounds__(256) void copy_kernel(const CopyJob a) {
    const int y = blockIdx.y;
    const uint32_t cols = a.cols[y], a_row = a.pitch[y] / kPer<T>;
    const uint64_t vectors = (uint64_t)a.rows[y] * a_row;
    const Taken rows = {a.source[y], a.tokens};
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < vectors; i += (uint64_t)gridDim.x * 256) {
        const uint64_t row = i / a_row;
        const uint32_t col = (uint32_t)(i - row * a_row) * kPer<T>;
        store_vec((T *)a.to[y] + i * kPer<T>, kPer<T>, load_vec((const T *)a.from[y] + (uint64_t)rows((uint32_t)row) * cols + col, (int)(cols - col), (int)col));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

// Without `source` the plan's order is that of x.
struct Call {
    const bt_expert_plan &plan;
    bool ordered;
    hipStream_t hs;
    uint64_t rows() const { return plan.tokens * plan.chosen; }
    ExpertJob job() const {
        ExpertJob a = {};
        a.offsets = plan.d_offsets;
        a.experts = (uint32_t)plan.experts;
        a.rows = (uint32_t)rows();
        a.tokens = (uint32_t)plan.tokens;
        return a;
    }
};

// Elements of a row that goes on with zeros to the end of a tile.
uint64_t filled(const uint64_t cols, const int width) { return ceil_div(cols * width, 2 * kKBytes) * (2 * kKBytes) / width; }

// Rows of an expert, where all have the same.
uint64_t each(const bt_expert_plan &p) { return p.tokens * p.chosen / p.experts; }

// Rows of an expert from which on operands whose rows do not begin on 16-byte boundaries are copied to ones that do, as with the dense projections.
constexpr uint64_t kPadEach = 128;

bool pads(const bt_expert_plan &p, const uint64_t cols, const int width) { return ragged(cols, width) && each(p) >= kPadEach; }

// Rows of whole vectors on 16-byte boundaries, and a tile within 32 bits of offsets.
template <class T> bool direct(const void *p, const uint64_t pitch) { return !misaligned(p, kVec) && pitch % kPer<T> == 0 && pitch * sizeof(T) * 320 < 1u << 31; }

template <class T, Kind K> bt_status run_product(ExpertJob &a, hipStream_t hs) {
    const auto go = [&](auto kernel, const uint32_t rows, const uint32_t cols, const int threads, const uint32_t slots = 0) {
        const uint64_t tiles_n = ceil_div(a.n, cols);
        uint64_t tiles_m;
        if (K == kWeights) tiles_m = ceil_div(a.m, rows);
        else {      // each group's last tile may be a part
            tiles_m = a.rows / rows + a.experts + 1;
            if (tiles_m > a.rows) tiles_m = a.rows;
        }
        const uint64_t groups = tiles_m * tiles_n * (K == kWeights ? (uint64_t)a.experts * a.outputs : 1);
        if (groups >= 1u << 31) return BT_ERR_SIZE;
        a.tiles_m = (uint32_t)tiles_m;
        a.tiles_n = (uint32_t)tiles_n;
        a.first = 0;
        // (What is in parts are at most as many workgroups as run at once.)
        const uint64_t items = a.most_splits > 1 ? groups + slots : groups;
        // The largest tiles' workgroups, one to a compute unit, take several each.
        if (threads == Large::THREADS && rows == Large::NQ) return launch(kernel, dim3((unsigned)(items < 256 ? items : 256)), threads, hs, a);
        constexpr uint64_t kMost = 1u << 22;      // of a launch: a grid holds less than 2^32 threads
        bt_status s = BT_OK;
        for (uint64_t first = 0; first < items && s == BT_OK; first += kMost) {
            a.first = (uint32_t)first;
            s = launch(kernel, dim3((unsigned)(items - first < kMost ? items - first : kMost)), threads, hs, a);
        }
        return s;
    };
    a.most_splits = 1;
    const auto tiled = [&](auto kernel, auto join, auto shape) {
        typedef decltype(shape) S;
        const Parts parts = parts_of(K, S::THREADS == 512 ? kLarge : S::FQ == 4 ? kMiddle : kSmall, a.rows, a.experts, a.m, a.n, a.k, a.outputs, sizeof(T));
        a.most_splits = parts.most;
        const bt_status s = go(kernel, S::NQ, K == kPair ? S::NP / 2 : S::NP, S::THREADS, kSlots<S>);
        if (s != BT_OK || parts.most == 1) return s;
        return launch(join, dim3(kSlots<S> / 2 * (S::FQ / kSlice)), S::THREADS, hs, a);
    };
    if constexpr (K <= kPlain) {
        if (few_rows(K == kPair, a.rows, a.experts, a.n, a.k, sizeof(T))) {
            const auto tokens = [&](auto kernel) { return go(kernel, 16, 16, kTokenWaves * kWave); };
            if constexpr (sizeof(T) == 2)
                if (a.pitch_p % 2 != 0 && !misaligned(a.p[0], 4) && !misaligned(a.p[1], 4) && !misaligned(a.q[0], 4)) return tokens(experts_tokens_kernel<T, K, true>);
            return tokens(experts_tokens_kernel<T, K, false>);
        }
    }
    bool straight = direct<T>(a.p[0], a.pitch_p) && direct<T>(a.q[0], a.pitch_q);
    if (K == kPair || K == kBackPair) straight = straight && direct<T>(a.p[1], a.pitch_p);
    if (K == kBackPair || (K == kWeights && a.outputs == 2)) straight = straight && direct<T>(a.q[1], a.pitch_q);
    if constexpr (K <= kPlain)
        if (a.source) straight = straight && a.tokens * a.pitch_q * sizeof(T) < 1u << 31;
    if (!straight) return go(experts_any_kernel<T, K>, Small::NQ, K == kPair ? Small::NP / 2 : Small::NP, Small::THREADS);
    const Size size = size_of(K, a.rows, a.experts, a.m, a.n, a.k, a.outputs, sizeof(T));
    if constexpr (sizeof(T) == 2) {
        if (size == kLarge) return tiled(experts_kernel<T, K, Large>, experts_join_kernel<T, K, Large>, Large{});
        if (size == kMiddle) return tiled(experts_kernel<T, K, Middle>, experts_join_kernel<T, K, Middle>, Middle{});
    }
    return tiled(experts_kernel<T, K, Small>, experts_join_kernel<T, K, Small>, Small{});
}

// What is to be copied, and where to in the workspace.
template <class T> struct Copies {
    CopyJob job = {};
    int count = 0;

    T *add(char **ws, const void *from, const uint64_t rows, const uint64_t cols, const uint64_t pitch, const int32_t *source = nullptr, const bool wanted = true) {
        T *const to = (T *)*ws;
        *ws += whole(rows * pitch * sizeof(T));
        if (wanted) {
            job.from[count] = from;
            job.to[count] = to;
            job.source[count] = source;
            job.rows[count] = (uint32_t)rows;
            job.cols[count] = (uint32_t)cols;
            job.pitch[count++] = (uint32_t)pitch;
        }
        return to;
    }
    bt_status run(const Call &c) {
        if (count == 0) return BT_OK;
        job.tokens = (uint32_t)c.plan.tokens;
        uint64_t most = 1;
        for (int i = 0; i < count; ++i) {
            const uint64_t vectors = (uint64_t)job.rows[i] * (job.pitch[i] / kPer<T>);
            most = vectors > most ? vectors : most;
        }
        const uint64_t blocks = ceil_div(most, 256);
        return launch(copy_kernel<T>, dim3((unsigned)(blocks < 1u << 14 ? blocks : 1u << 14), (unsigned)count), 256, c.hs, job);
    }
};

// Bytes of the copies that the forward pass makes of x and `weights` weights (f rows of each), and the backward pass of x, where it is not in the order of the rows, and of the weights.
uint64_t copies_bytes(const bt_expert_plan &p, const uint64_t d, const uint64_t f, const int weights, const int width, const bool ordered, const bool back) {
    const uint64_t rows = p.tokens * p.chosen, pitch = filled(d, width);
    if (!pads(p, d, width)) return back && !ordered ? whole(rows * pitch * width) : 0;
    return whole((back || ordered ? rows : p.tokens) * pitch * width) + weights * whole(p.experts * f * pitch * width);
}

bt_status check(const bt_expert_plan *plan, const uint64_t d, const uint64_t f, const bt_dtype dtype) {
    const bt_status st = check_plan(plan);
    return st != BT_OK ? st : check_sizes(plan->tokens * plan->chosen, d, f, dtype);
}

bt_status check_tables(const bt_expert_plan &plan, const bool ordered, const bool back) {
    if (plan.d_offsets == nullptr || (!ordered && (plan.d_source == nullptr || (back && plan.d_slots == nullptr)))) return BT_ERR_NULL;
    return misaligned(plan.d_offsets, 4) || misaligned(plan.d_source, 4) || misaligned(plan.d_slots, 4) ? BT_ERR_ALIGN : BT_OK;
}

template <class... P> bool any_misaligned(const size_t a, P... p) { return (misaligned(p, a) || ...); }

// Bytes of the sums of parts of tiles, of the forward pass and of the larger of both backward products.
uint64_t parts_bytes(const bt_expert_plan &p, const Kind kind, const uint64_t m, const uint64_t n, const uint64_t k, const uint64_t outputs, const int width) {
    const uint64_t rows = p.tokens * p.chosen;
    if (kind <= kPlain && few_rows(kind == kPair, rows, p.experts, n, k, width)) return 0;
    return whole(parts_of(kind, size_of(kind, rows, p.experts, m, n, k, outputs, width), rows, p.experts, m, n, k, outputs, width).bytes);
}
uint64_t forward_parts(const bt_expert_plan &p, const uint64_t d, const uint64_t f, const bool pair, const int width) {
    return parts_bytes(p, pair ? kPair : kPlain, 0, f, pads(p, d, width) ? filled(d, width) : d, 0, width);
}
uint64_t backward_parts(const bt_expert_plan &p, const uint64_t d, const uint64_t f, const bool pair, const int width) {
    const uint64_t x = parts_bytes(p, pair ? kBackPair : kBack, 0, d, f, 0, width), weights = parts_bytes(p, kWeights, f, d, 0, pair ? 2 : 1, width);
    return x > weights ? x : weights;
}

// x and one weight (w_up NULL) or two of the forward pass, as they are or copied.
template <class T>
bt_status operands(const Call &c, ExpertJob &a, const void *x, const void *w_gate, const void *w_up, const uint64_t d, const uint64_t f, char *ws) {
    bt_status s = BT_OK;
    uint64_t pitch = d;
    if (pads(c.plan, d, sizeof(T))) {
        pitch = filled(d, sizeof(T));
        Copies<T> copies;
        x = copies.add(&ws, x, c.ordered ? c.rows() : c.plan.tokens, d, pitch);
        w_gate = copies.add(&ws, w_gate, c.plan.experts * f, d, pitch);
        if (w_up) w_up = copies.add(&ws, w_up, c.plan.experts * f, d, pitch);
        s = copies.run(c);
    }
    a.p[0] = w_gate;
    a.p[1] = w_up ? w_up : w_gate;
    a.q[0] = a.q[1] = x;
    a.pitch_p = a.pitch_q = pitch;
    a.step = f * pitch;
    a.k = (uint32_t)pitch;
    a.parts = (float *)ws;
    return s;
}

// The gradient of x, and those of the weights, of one product (du NULL) or of both projections, whose factors are dg and du: rows of `pitch_g`.
// `copies`: what else is to be copied before.
template <class T>
bt_status backward(const Call &c, Copies<T> &copies, const T *dg, const T *du, const uint64_t pitch_g, const void *x, const void *w_gate, const void *w_up, const uint64_t d, const uint64_t f,
                   void *grad_x, void *grad_w_gate, void *grad_w_up, char *ws) {
    const bool filled_too = pads(c.plan, d, sizeof(T));
    const uint64_t pitch = filled_too ? filled(d, sizeof(T)) : d, pitch_x = c.ordered ? pitch : filled(d, sizeof(T));
    if (!c.ordered || filled_too) x = copies.add(&ws, x, c.rows(), d, pitch_x, c.ordered ? nullptr : c.plan.d_source, grad_w_gate != nullptr);
    if (filled_too) {
        w_gate = copies.add(&ws, w_gate, c.plan.experts * f, d, pitch, nullptr, grad_x != nullptr);
        if (du) w_up = copies.add(&ws, w_up, c.plan.experts * f, d, pitch, nullptr, grad_x != nullptr);
    }
    float *const sums = (float *)ws, *const parts = (float *)(ws + (c.ordered ? 0 : whole(4 * c.rows() * d)));
    bt_status s = copies.run(c);
    if (s == BT_OK && grad_x) {
        ExpertJob a = c.job();
        a.parts = parts;
        a.p[0] = w_gate;
        a.p[1] = w_up;
        a.q[0] = dg;
        a.q[1] = du;
        a.pitch_p = pitch;
        a.pitch_q = pitch_g;
        a.step = f * pitch;
        a.pitch = d;
        a.n = (uint32_t)d;
        a.k = (uint32_t)f;
        a.padded_q = pitch_g == filled(f, sizeof(T));
        if (c.ordered) a.out[0] = grad_x;
        else a.sums = sums;
        s = du ? run_product<T, kBackPair>(a, c.hs) : run_product<T, kBack>(a, c.hs);
        if (s == BT_OK && !c.ordered) {
            const bt_dtype dtype = std::is_same_v<T, float> ? BT_F32 : std::is_same_v<T, f16> ? BT_F16 : BT_BF16;
            s = sum_rows(c.plan, a.sums, d, dtype, grad_x, c.hs);
        }
    }
    if (s == BT_OK && grad_w_gate) {
        ExpertJob a = c.job();
        a.parts = parts;
        a.p[0] = x;
        a.q[0] = dg;
        a.q[1] = du;
        a.pitch_p = pitch_x;
        a.pitch_q = pitch_g;
        a.step = f * d;
        a.out[0] = grad_w_gate;
        a.out[1] = grad_w_up;
        a.pitch = d;
        a.m = (uint32_t)f;
        a.n = (uint32_t)d;
        a.outputs = du ? 2 : 1;
        s = run_product<T, kWeights>(a, c.hs);
    }
    return s;
}

// Sums of nothing.
template <class T> bt_status nothing(const Call &c, const uint64_t d, const uint64_t f, void *grad_x, void *grad_w_gate, void *grad_w_up) {
    bt_status s = grad_x ? zeros<T>(grad_x, (c.ordered ? c.rows() : c.plan.tokens) * d, c.hs) : BT_OK;
    if (s == BT_OK && grad_w_gate) s = zeros<T>(grad_w_gate, c.plan.experts * f * d, c.hs);
    if (s == BT_OK && grad_w_up) s = zeros<T>(grad_w_up, c.plan.experts * f * d, c.hs);
    return s;
}

}  // namespace
}  // namespace btb

using namespace btb;

extern "C" {

size_t bt_expert_gated_workspace_bytes(const bt_expert_plan *plan, uint64_t d, uint64_t f, bt_dtype dtype, int ordered, int backward) {
    if (check(plan, d, f, dtype) != BT_OK || plan->tokens == 0 || f == 0) return 0;
    const uint64_t rows = plan->tokens * plan->chosen, w = (uint64_t)width_of(dtype), copies = copies_bytes(*plan, d, f, 2, (int)w, ordered != 0, backward != 0);
    if (!backward) return (size_t)(copies + forward_parts(*plan, d, f, true, (int)w));
    return (size_t)(copies + 2 * whole(rows * filled(f, (int)w) * w) + (ordered ? 0 : whole(4 * rows * d)) + backward_parts(*plan, d, f, true, (int)w));
}

bt_status bt_expert_gated_forward(const void *d_x, const void *d_w_gate, const void *d_w_up, const bt_expert_plan *plan,
                                  uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation, int ordered,
                                  void *d_h, void *d_gate, void *d_up, void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check(plan, d, f, dtype);
    if (st != BT_OK) return st;
    if (!known(activation) || (d_gate == nullptr) != (d_up == nullptr)) return BT_ERR_ARGUMENT;
    if (plan->tokens == 0 || f == 0) return BT_OK;
    if (d_h == nullptr || (d != 0 && (d_x == nullptr || d_w_gate == nullptr || d_w_up == nullptr))) return BT_ERR_NULL;
    st = check_tables(*plan, ordered != 0, false);
    if (st != BT_OK) return st;
    const size_t need = bt_expert_gated_workspace_bytes(plan, d, f, dtype, ordered, 0);
    if (need != 0 && d_workspace == nullptr) return BT_ERR_NULL;
    if (any_misaligned((size_t)width_of(dtype), d_x, d_w_gate, d_w_up, d_h, d_gate, d_up) || misaligned(d_workspace, 128)) return BT_ERR_ALIGN;
    if (workspace_bytes < need) return BT_ERR_WORKSPACE;
    const Call c = {*plan, ordered != 0, (hipStream_t)stream};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        ExpertJob a = c.job();
        const bt_status s = operands<T>(c, a, d_x, d_w_gate, d_w_up, d, f, (char *)d_workspace);
        if (s != BT_OK) return s;
        a.out[0] = d_h;
        a.gate = d_gate;
        a.up = d_up;
        a.pitch = f;
        a.source = c.ordered ? nullptr : plan->d_source;
        a.n = (uint32_t)f;
        a.activation = activation;
        return run_product<T, kPair>(a, c.hs);
    });
}

bt_status bt_expert_gated_backward(const void *d_grad_h, const void *d_x, const void *d_w_gate, const void *d_w_up,
                                   const void *d_gate, const void *d_up, const bt_expert_plan *plan,
                                   uint64_t d, uint64_t f, bt_dtype dtype, bt_activation activation, int ordered,
                                   void *d_grad_x, void *d_grad_w_gate, void *d_grad_w_up,
                                   void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check(plan, d, f, dtype);
    if (st != BT_OK) return st;
    if (!known(activation) || (d_grad_w_gate == nullptr) != (d_grad_w_up == nullptr)) return BT_ERR_ARGUMENT;
    if (any_misaligned((size_t)width_of(dtype), d_grad_h, d_x, d_w_gate, d_w_up, d_gate, d_up, d_grad_x, d_grad_w_gate, d_grad_w_up) || misaligned(d_workspace, 128))
        return BT_ERR_ALIGN;
    if (d == 0 || (d_grad_x == nullptr && d_grad_w_gate == nullptr)) return BT_OK;
    const uint64_t rows = plan->tokens * plan->chosen;
    const Call c = {*plan, ordered != 0, (hipStream_t)stream};
    if (rows != 0 && f != 0) {
        if (d_grad_h == nullptr || d_gate == nullptr || d_up == nullptr || d_workspace == nullptr ||
            (d_grad_x && (d_w_gate == nullptr || d_w_up == nullptr)) || (d_grad_w_gate && d_x == nullptr))
            return BT_ERR_NULL;
        st = check_tables(*plan, c.ordered, d_grad_x != nullptr);
        if (st != BT_OK) return st;
        if (workspace_bytes < bt_expert_gated_workspace_bytes(plan, d, f, dtype, ordered, 1)) return BT_ERR_WORKSPACE;
    }
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (rows == 0 || f == 0) return nothing<T>(c, d, f, d_grad_x, d_grad_w_gate, d_grad_w_up);
        char *ws = (char *)d_workspace;
        const uint64_t pitch = filled(f, sizeof(T)), vectors = rows * pitch / kPer<T>, blocks = ceil_div(vectors, 256);
        T *const dg = (T *)ws, *const du = (T *)(ws + whole(rows * pitch * sizeof(T)));
        ws += 2 * whole(rows * pitch * sizeof(T));
        const bt_status s = launch(gated_slopes_kernel<T>, dim3((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20)), 256, c.hs, (const T *)d_grad_h, (const T *)d_gate,
                                   (const T *)d_up, dg, du, (uint32_t)f, (uint32_t)pitch, vectors, (int)activation);
        if (s != BT_OK) return s;
        Copies<T> copies;
        return backward<T>(c, copies, dg, du, pitch, d_x, d_w_gate, d_w_up, d, f, d_grad_x, d_grad_w_gate, d_grad_w_up, ws);
    });
}

size_t bt_expert_linear_workspace_bytes(const bt_expert_plan *plan, uint64_t d_in, uint64_t d_out, bt_dtype dtype, int ordered, int backward) {
    if (check(plan, d_in, d_out, dtype) != BT_OK || plan->tokens == 0 || d_out == 0) return 0;
    const uint64_t rows = plan->tokens * plan->chosen, w = (uint64_t)width_of(dtype), copies = copies_bytes(*plan, d_in, d_out, 1, (int)w, ordered != 0, backward != 0);
    if (!backward) return (size_t)(copies + forward_parts(*plan, d_in, d_out, false, (int)w));
    return (size_t)(copies + backward_parts(*plan, d_in, d_out, false, (int)w) + (pads(*plan, d_out, (int)w) ? whole(rows * filled(d_out, (int)w) * w) : 0) + (ordered ? 0 : whole(4 * rows * d_in)));
}

bt_status bt_expert_linear_forward(const void *d_x, const void *d_w, const bt_expert_plan *plan, uint64_t d_in, uint64_t d_out, bt_dtype dtype, int ordered,
                                   void *d_y, void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check(plan, d_in, d_out, dtype);
    if (st != BT_OK) return st;
    if (plan->tokens == 0 || d_out == 0) return BT_OK;
    if (d_y == nullptr || (d_in != 0 && (d_x == nullptr || d_w == nullptr))) return BT_ERR_NULL;
    st = check_tables(*plan, ordered != 0, false);
    if (st != BT_OK) return st;
    const size_t need = bt_expert_linear_workspace_bytes(plan, d_in, d_out, dtype, ordered, 0);
    if (need != 0 && d_workspace == nullptr) return BT_ERR_NULL;
    if (any_misaligned((size_t)width_of(dtype), d_x, d_w, d_y) || misaligned(d_workspace, 128)) return BT_ERR_ALIGN;
    if (workspace_bytes < need) return BT_ERR_WORKSPACE;
    const Call c = {*plan, ordered != 0, (hipStream_t)stream};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        ExpertJob a = c.job();
        const bt_status s = operands<T>(c, a, d_x, d_w, nullptr, d_in, d_out, (char *)d_workspace);
        if (s != BT_OK) return s;
        a.out[0] = d_y;
        a.pitch = d_out;
        a.source = c.ordered ? nullptr : plan->d_source;
        a.n = (uint32_t)d_out;
        return run_product<T, kPlain>(a, c.hs);
    });
}

bt_status bt_expert_linear_backward(const void *d_grad_y, const void *d_x, const void *d_w, const bt_expert_plan *plan,
                                    uint64_t d_in, uint64_t d_out, bt_dtype dtype, int ordered, void *d_grad_x, void *d_grad_w,
                                    void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check(plan, d_in, d_out, dtype);
    if (st != BT_OK) return st;
    if (any_misaligned((size_t)width_of(dtype), d_grad_y, d_x, d_w, d_grad_x, d_grad_w) || misaligned(d_workspace, 128)) return BT_ERR_ALIGN;
    if (d_in == 0 || (d_grad_x == nullptr && d_grad_w == nullptr)) return BT_OK;
    const Call c = {*plan, ordered != 0, (hipStream_t)stream};
    const uint64_t rows = c.rows();
    if (rows != 0 && d_out != 0) {
        if (d_grad_y == nullptr || (d_grad_x && d_w == nullptr) || (d_grad_w && d_x == nullptr)) return BT_ERR_NULL;
        st = check_tables(*plan, c.ordered, d_grad_x != nullptr);
        if (st != BT_OK) return st;
        const size_t need = bt_expert_linear_workspace_bytes(plan, d_in, d_out, dtype, ordered, 1);
        if (need != 0 && d_workspace == nullptr) return BT_ERR_NULL;
        if (workspace_bytes < need) return BT_ERR_WORKSPACE;
    }
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        if (rows == 0 || d_out == 0) return nothing<T>(c, d_in, d_out, d_grad_x, d_grad_w, nullptr);
        char *ws = (char *)d_workspace;
        const T *grad_y = (const T *)d_grad_y;
        uint64_t pitch = d_out;
        Copies<T> copies;
        if (pads(*plan, d_out, sizeof(T))) {
            pitch = filled(d_out, sizeof(T));
            grad_y = copies.add(&ws, d_grad_y, rows, d_out, pitch);
        }
        return backward<T>(c, copies, grad_y, nullptr, pitch, d_x, d_w, nullptr, d_in, d_out, d_grad_x, d_grad_w, nullptr, ws);
    });
}

}  // extern "C"
