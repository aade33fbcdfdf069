// The products of a sublayer of several experts, and their backward passes: see include/bittrain.h for the contract.
//
// As in gated.hip, but for each expert's rows with its own weights: how many rows each has is known on the device alone, so a grid is as large as it could have to be and
// every workgroup finds its expert and tile in the sums of the experts' tiles.  Behind the last expert comes a group of the rows of no expert, whose sum is empty.
#include <math.h>

#include "product.h"
#include "route.h"

namespace btb {
namespace {

// Both gated projections; one product; its way back, and that of both projections (two sums); the weights' gradients.
enum Kind { kPair, kPlain, kBack, kBackPair, kWeights };

template <Kind K> using FormOf = Form<K == kPair, K <= kPlain ? kAlong : kAcross, K == kWeights ? kAcross : kAlong, K == kBackPair ? 2 : 1>;

struct ExpertJob {
    const void *p[2], *q[2];           // of the first expert, or the first row; p: weights (kWeights: x), q: x, gradients
    uint64_t pitch_p, pitch_q;         // elements from a row to the next
    uint64_t step;                     // elements from one expert's weights (kWeights: gradients) to the next one's
    void *out[2], *gate, *up;
    float *sums;                       // kBack: [rows, n] in single precision instead of out
    uint64_t pitch;                    // of the outputs
    const int32_t *offsets, *source;   // source: x has a row a token; else NULL
    uint32_t experts, rows, tokens;
    uint32_t m, n, k;                  // kWeights: m by n of each expert, k is not used; else n columns and k summed indices
    uint32_t tiles_m, tiles_n, parts;  // kWeights: tiles of an output, outputs; else tiles_n alone
    uint32_t first;                    // tile that the launch begins with
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

__device__ inline Group group_of(const ExpertJob &a, const uint32_t e) {
    const uint32_t first = bound(a, e), end = e < a.experts ? bound(a, e + 1) : a.rows;
    return {e, first, end > first ? end - first : 0};
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

// The experts' tiles of `a_tile` rows, added up: those of expert e are numbered from starts[e] on; starts[experts + 1] is how many there are.
struct Tiles {
    uint32_t starts[kMostExperts + 2];

    // (A wave's work, and everybody's wait.)
    __device__ void find(const ExpertJob &a, const uint32_t a_tile) {
        if (threadIdx.x < kWave) {
            uint32_t sum = 0;
            for (uint32_t e0 = 0; e0 <= a.experts; e0 += kWave) {
                const uint32_t e = e0 + threadIdx.x;
                uint32_t n = 0;
                if (e <= a.experts) n = (group_of(a, e).rows + a_tile - 1) / a_tile;
                uint32_t x = n;
#pragma unroll
                for (int d = 1; d < kWave; d *= 2) {
                    const uint32_t y = __shfl_up(x, d);
                    if ((int)threadIdx.x >= d) x += y;
                }
                if (e <= a.experts) starts[e] = sum + x - n;
                sum += __shfl(x, kWave - 1);
            }
            if (threadIdx.x == 0) starts[a.experts + 1] = sum;
        }
        __syncthreads();
    }
    __device__ uint32_t count(const ExpertJob &a) const { return __builtin_amdgcn_readfirstlane(starts[a.experts + 1]); }
    // The expert that a tile belongs to.
    __device__ uint32_t expert(const ExpertJob &a, const uint32_t tile) const {
        uint32_t low = 0, high = a.experts + 1;      // starts[low] <= tile < starts[high]
        while (high - low > 1) {
            const uint32_t mid = (low + high) / 2;
            if ((uint32_t)__builtin_amdgcn_readfirstlane(starts[mid]) <= tile) low = mid;
            else high = mid;
        }
        return low;
    }
};

struct Place {
    Group of;
    uint32_t m, n, part;
};

// Tiles that there are, and the tile of a number.  Workgroups go to the eight XCDs in turn, each of which has an L2 of its own: an XCD's are neighbours, in bands of four rows of
// tiles of one expert, so that those that run at once share what they read.
template <Kind K> __device__ inline uint32_t tiles_of(const ExpertJob &a, const Tiles &tiles) {
    if constexpr (K == kWeights) return a.experts * a.parts * a.tiles_m * a.tiles_n;
    else return tiles.count(a) * a.tiles_n;
}

template <Kind K> __device__ inline Place place_of(const ExpertJob &a, const Tiles &tiles, const uint32_t number, const uint32_t total, const uint32_t tile_m, const uint32_t tile_n) {
    constexpr uint32_t kXcds = 8, kBand = 4;
    const uint32_t xcd = number % kXcds, more = total % kXcds;
    uint32_t tile = xcd * (total / kXcds) + (xcd < more ? xcd : more) + number / kXcds, rows;
    Place at;
    if constexpr (K == kWeights) {
        const uint32_t a_part = a.tiles_m * a.tiles_n, e = tile / (a_part * a.parts);
        at.of = group_of(a, e);
        tile -= e * a_part * a.parts;
        at.part = tile / a_part;
        tile -= at.part * a_part;
        rows = a.tiles_m;
    } else {
        const uint32_t e = tiles.expert(a, tile / a.tiles_n);
        at.of = group_of(a, e);
        at.part = 0;
        const uint32_t start = __builtin_amdgcn_readfirstlane(tiles.starts[e]);
        rows = __builtin_amdgcn_readfirstlane(tiles.starts[e + 1]) - start;
        tile -= start * a.tiles_n;
    }
    const uint32_t band = tile / (kBand * a.tiles_n), left = rows - band * kBand, high = left < kBand ? left : kBand;
    tile -= band * kBand * a.tiles_n;
    at.m = (band * kBand + tile % high) * tile_m;
    at.n = tile / high * tile_n;
    return at;
}

// The operands of a tile's product, of sum `sum`; rows and summed indices that it has.
template <class T, Kind K> __device__ inline Operand operand_p(const ExpertJob &a, const Group &g, const int sum) {
    if constexpr (K == kWeights) return {(const T *)a.p[0] + (a.source ? 0 : g.first * a.pitch_p), a.pitch_p, g.rows, a.n};
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
template <Kind K> __device__ inline uint32_t summed(const ExpertJob &a, const Group &g) { return K == kWeights ? g.rows : g.expert < a.experts ? a.k : 0; }
__device__ inline Taken taken(const ExpertJob &a, const Group &g) { return {a.source ? a.source + g.first : nullptr, a.tokens}; }

// Stores that a lane makes of each output in the function below, of a tile that lies inside it: at the least.
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
    __shared__ Tiles map;
    if constexpr (K != kWeights) map.find(a, Small::NQ);
    const uint32_t total = tiles_of<K>(a, map), number = a.first + blockIdx.x;
    if (number >= total) return;
    const Place at = place_of<K>(a, map, number, total, Small::NQ, W::COLS);
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
            if constexpr (K == kWeights) w.staged(p[0], p[0], q[0], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, acc, rows);
            else if constexpr (K <= kPlain) w.staged(p[s], p[1], q[s], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, acc, InOrder{}, rows);
            else w.staged(p[s], p[1], q[s], at.n, at.m, start_of(t), tiles[0], tiles[0] + W::P::BYTES, acc);
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

template <class T, Kind K> bt_status run_product(ExpertJob &a, hipStream_t hs) {
    const auto go = [&](auto kernel, auto shape) {
        typedef decltype(shape) S;
        const uint64_t tiles_n = ceil_div(a.n, K == kPair ? S::NP / 2 : S::NP);
        uint64_t tiles_m;
        if (K == kWeights) tiles_m = ceil_div(a.m, S::NQ);
        else {      // each group's last tile may be a part
            tiles_m = a.rows / S::NQ + a.experts + 1;
            if (tiles_m > a.rows) tiles_m = a.rows;
        }
        const uint64_t groups = tiles_m * tiles_n * (K == kWeights ? (uint64_t)a.experts * a.parts : 1);
        if (groups >= 1u << 31) return BT_ERR_SIZE;
        a.tiles_m = (uint32_t)tiles_m;
        a.tiles_n = (uint32_t)tiles_n;
        constexpr uint64_t kMost = 1u << 22;      // of a launch: a grid holds less than 2^32 threads
        bt_status s = BT_OK;
        for (uint64_t first = 0; first < groups && s == BT_OK; first += kMost) {
            a.first = (uint32_t)first;
            s = launch(kernel, dim3((unsigned)(groups - first < kMost ? groups - first : kMost)), S::THREADS, hs, a);
        }
        return s;
    };
    return go(experts_any_kernel<T, K>, Small{});
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

// The gradient of x, and those of the weights, of one product (du NULL) or of both projections, whose factors are dg and du: rows of `pitch_g`.
template <class T>
bt_status backward(const Call &c, const T *dg, const T *du, const uint64_t pitch_g, const void *x, const void *w_gate, const void *w_up, const uint64_t d, const uint64_t f,
                   void *grad_x, void *grad_w_gate, void *grad_w_up, char *ws) {
    bt_status s = BT_OK;
    if (grad_x) {
        ExpertJob a = c.job();
        a.p[0] = w_gate;
        a.p[1] = w_up;
        a.q[0] = dg;
        a.q[1] = du;
        a.pitch_p = d;
        a.pitch_q = pitch_g;
        a.step = f * d;
        a.pitch = d;
        a.n = (uint32_t)d;
        a.k = (uint32_t)f;
        if (c.ordered) a.out[0] = grad_x;
        else a.sums = (float *)ws;
        s = du ? run_product<T, kBackPair>(a, c.hs) : run_product<T, kBack>(a, c.hs);
        if (s == BT_OK && !c.ordered) {
            const bt_dtype dtype = std::is_same_v<T, float> ? BT_F32 : std::is_same_v<T, f16> ? BT_F16 : BT_BF16;
            s = sum_rows(c.plan, a.sums, d, dtype, grad_x, c.hs);
        }
    }
    if (s == BT_OK && grad_w_gate) {
        ExpertJob a = c.job();
        a.p[0] = x;
        a.q[0] = dg;
        a.q[1] = du;
        a.pitch_p = d;
        a.pitch_q = pitch_g;
        a.step = f * d;
        a.out[0] = grad_w_gate;
        a.out[1] = grad_w_up;
        a.pitch = d;
        a.m = (uint32_t)f;
        a.n = (uint32_t)d;
        a.parts = du ? 2 : 1;
        a.source = c.ordered ? nullptr : c.plan.d_source;
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
    if (check(plan, d, f, dtype) != BT_OK || plan->tokens == 0 || f == 0 || !backward) return 0;
    const uint64_t rows = plan->tokens * plan->chosen, w = (uint64_t)width_of(dtype);
    return (size_t)(2 * whole(rows * padded(f, (int)w) * w) + (ordered ? 0 : whole(4 * rows * d)));
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
        a.p[0] = d_w_gate;
        a.p[1] = d_w_up;
        a.q[0] = a.q[1] = d_x;
        a.pitch_p = a.pitch_q = d;
        a.step = f * d;
        a.out[0] = d_h;
        a.gate = d_gate;
        a.up = d_up;
        a.pitch = f;
        a.source = c.ordered ? nullptr : plan->d_source;
        a.n = (uint32_t)f;
        a.k = (uint32_t)d;
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
        const uint64_t pitch = padded(f, sizeof(T)), vectors = rows * pitch / kPer<T>, blocks = ceil_div(vectors, 256);
        T *const dg = (T *)ws, *const du = (T *)(ws + whole(rows * pitch * sizeof(T)));
        ws += 2 * whole(rows * pitch * sizeof(T));
        const bt_status s = launch(gated_slopes_kernel<T>, dim3((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20)), 256, c.hs, (const T *)d_grad_h, (const T *)d_gate,
                                   (const T *)d_up, dg, du, (uint32_t)f, (uint32_t)pitch, vectors, (int)activation);
        if (s != BT_OK) return s;
        return backward<T>(c, dg, du, pitch, d_x, d_w_gate, d_w_up, d, f, d_grad_x, d_grad_w_gate, d_grad_w_up, ws);
    });
}

size_t bt_expert_linear_workspace_bytes(const bt_expert_plan *plan, uint64_t d_in, uint64_t d_out, bt_dtype dtype, int ordered, int backward) {
    if (check(plan, d_in, d_out, dtype) != BT_OK || plan->tokens == 0 || d_out == 0 || !backward || ordered) return 0;
    return (size_t)whole(4 * plan->tokens * plan->chosen * d_in);
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
        a.p[0] = a.p[1] = d_w;
        a.q[0] = a.q[1] = d_x;
        a.pitch_p = a.pitch_q = d_in;
        a.step = d_out * d_in;
        a.out[0] = d_y;
        a.pitch = d_out;
        a.source = c.ordered ? nullptr : plan->d_source;
        a.n = (uint32_t)d_out;
        a.k = (uint32_t)d_in;
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
        return backward<T>(c, (const T *)d_grad_y, nullptr, d_out, d_x, d_w, nullptr, d_in, d_out, d_grad_x, d_grad_w, nullptr, (char *)d_workspace);
    });
}

}  // extern "C"
