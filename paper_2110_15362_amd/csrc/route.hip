// Which experts a token goes to, the order of the rows that this makes, and a token's rows added up again: see include/bittrain.h for the contract.
//
// The order is a counting sort that keeps the tokens' order: each workgroup of choose_kernel counts its tokens' experts, and each of order_kernel adds up
// the counts of those before it.  No atomics across workgroups: equal inputs give equal tables.
#include <math.h>

#include "route.h"

namespace btb {
namespace {

constexpr int kMostExperts = BT_MAX_EXPERTS, kMostChosen = BT_MAX_CHOSEN;

// The largest (smallest) of the values that L neighbouring lanes hold, in all of them.
template <int L, class Op> __device__ inline uint32_t across(uint32_t x, Op op) {
    const auto step = [&](auto ctrl) { x = op(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, decltype(ctrl)::value, 0xf, 0xf, false)); };
    step(std::integral_constant<int, 0xb1>{});                               // quad_perm 1, 0, 3, 2
    step(std::integral_constant<int, 0x4e>{});                               // quad_perm 2, 3, 0, 1
    step(std::integral_constant<int, 0x141>{});                              // row_half_mirror
    if constexpr (L >= 16) step(std::integral_constant<int, 0x140>{});       // row_mirror
    if constexpr (L >= 32) {
        const auto halves = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        x = op((uint32_t)halves[0], (uint32_t)halves[1]);
    }
    if constexpr (L >= 64) {
        const auto halves = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        x = op((uint32_t)halves[0], (uint32_t)halves[1]);
    }
    return x;
}

template <int L> __device__ inline uint32_t largest(const uint32_t x) { return across<L>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int L> __device__ inline uint32_t smallest(const uint32_t x) { return across<L>(x, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }
template <int L> __device__ inline float total(const float x) {
    return __builtin_bit_cast(float, across<L>(__builtin_bit_cast(uint32_t, x), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
    }));
}

// A logit as a number without sign that is ordered as the logits are: 0 for -infinity, all ones for a NaN; both zeros are one.
__device__ inline uint32_t key_of(const float x) {
    if (x != x) return 0xffffffffu;
    const uint32_t bits = __builtin_bit_cast(uint32_t, x + 0.0f);
    if (bits == 0xff800000u) return 0;
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}
__device__ inline float value_of(const uint32_t key) {
    if (key == 0xffffffffu) return __builtin_bit_cast(float, 0x7fc00000u);
    return __builtin_bit_cast(float, key >> 31 ? key & 0x7fffffffu : ~key);
}

struct RouteJob {
    const void *logits;      // NULL: index is there already
    float *weights;
    int32_t *index, *slots, *source, *offsets;
    int32_t *counts;         // [workgroups, experts]
    uint32_t tokens, experts, chosen, normalise;
    uint32_t a_group, groups;      // tokens of a workgroup, workgroups
};

// A lane's R logits of one token, from `first` on: -infinity beyond the last.
template <class T, int R> __device__ inline void read_logits(const RouteJob &a, const uint32_t token, const uint32_t first, float (&x)[R]) {
    const T *const p = (const T *)a.logits + (uint64_t)token * a.experts;
    constexpr int E = kPer<T>;
#pragma unroll
    for (int r = 0; r < R; r += E) {
        const int left = (int)a.experts - (int)first - r;
        float y[E];
        unpack<T>(load_vec(p + first + r, left, left < 0 ? 0 : (int)first + r), y);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (r + e < R) x[r + e] = e < left ? y[e] : -INFINITY;
    }
}

// The experts and weights of the tokens [first, end), L lanes a token and R logits a lane; `count` of the workgroup's experts in LDS is raised.
// A pass finds the largest of what is left: each lane has its own largest at hand, two reductions across the lanes give the value and, of equal ones, the first
// place.
template <class T, int L, int R, int THREADS> __device__ inline void choose(const RouteJob &a, const uint32_t first, const uint32_t end, uint32_t *count) {
    constexpr int kHeld = (kMostChosen + L - 1) / L;      // choices that a lane keeps
    const uint32_t lane = threadIdx.x % L;
    for (uint32_t token0 = first; token0 < end; token0 += THREADS / L) {
        const uint32_t token = token0 + threadIdx.x / L;
        const bool real = token < end;
        float x[R];
        uint32_t key[R];
        read_logits<T, R>(a, real ? token : end - 1, lane * R, x);
#pragma unroll
        for (int r = 0; r < R; ++r) key[r] = key_of(x[r]);
        uint32_t best = 0, place = 0;
        const auto look = [&]() {
            best = key[0];
            place = 0;
#pragma unroll
            for (int r = 1; r < R; ++r)
                if (key[r] > best) {
                    best = key[r];
                    place = r;
                }
        };
        look();
        float held[kHeld], top = 0.0f, sum = 0.0f;
        int32_t expert[kHeld];
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            held[h] = 0.0f;
            expert[h] = -1;
        }
        for (uint32_t j = 0; j < a.chosen; ++j) {
            const uint32_t most = largest<L>(best);
            const uint32_t mine = best == most ? lane * R + place : 0xffffffffu, who = smallest<L>(mine);
            if (j == 0) top = value_of(most);
            float e = 0.0f;
            if (most != 0) {
                e = expf(value_of(most) - top);
                sum += e;
            }
#pragma unroll
            for (int h = 0; h < kHeld; ++h)
                if (j == h * L + lane) {
                    held[h] = e;
                    expert[h] = most != 0 ? (int32_t)who : -1;
                }
            if (mine == who && most != 0) {
#pragma unroll
                for (int r = 0; r < R; ++r)
                    if (r == (int)place) key[r] = 0;
                look();
            }
        }
        if (!a.normalise) {
            sum = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (key_of(x[r]) != 0) sum += expf(x[r] - top);
            sum = total<L>(sum);
        }
        if (!real) continue;
#pragma unroll
        for (int h = 0; h < kHeld; ++h) {
            const uint32_t j = h * L + lane;
            if (j >= a.chosen) continue;
            const uint64_t at = (uint64_t)token * a.chosen + j;
            a.index[at] = expert[h];
            a.weights[at] = expert[h] < 0 ? 0.0f : held[h] / sum;
            if (expert[h] >= 0) atomicAdd(&count[expert[h]], 1u);
        }
    }
}

template <int THREADS> __device__ inline void clear_counts(const RouteJob &a, uint32_t *count) {
    for (uint32_t e = threadIdx.x; e < a.experts; e += THREADS) count[e] = 0;
}

// Of the wave's 64 choices those with the lane's expert.
__device__ inline uint64_t alike(const int32_t expert, const uint32_t experts) {
    const bool there = expert >= 0;
    uint64_t same = __ballot(there);
    if (!there) same = ~same;
    for (uint32_t bit = 1; bit < experts; bit <<= 1) {
        const bool set = there && (expert & bit) != 0;
        const uint64_t those = __ballot(set);
        same &= set ? those : ~those;
    }
    return same;
}

__device__ inline int32_t expert_at(const RouteJob &a, const uint64_t at, const uint64_t end) {
    const int32_t e = at < end ? a.index[at] : -1;
    return (uint32_t)e < a.experts ? e : -1;
}

// The rows of the choices [begin, end): `base` has, of each expert, the row that its first choice among them goes to (WAVES x experts in LDS, the first wave's filled in).
// Each wave takes a part of them in order: it counts, hears of the waves before it, and counts again.
template <int WAVES> __device__ inline void place_choices(const RouteJob &a, const uint64_t begin, const uint64_t end, uint32_t *base) {
    const uint32_t lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, experts = a.experts;
    const uint64_t part = ((end - begin + WAVES - 1) / WAVES + kWave - 1) / kWave * kWave;
    const uint64_t from = begin + wave * part < end ? begin + wave * part : end, to = from + part < end ? from + part : end;
    uint32_t *const mine = base + (wave + 1) * experts;      // (raised by this wave alone; the last wave's is not looked at)
    for (uint32_t e = lane; e < experts; e += kWave) mine[e] = 0;
    for (uint64_t at = from; at < to; at += kWave) {
        const int32_t e = expert_at(a, at + lane, to);
        const uint64_t same = alike(e, experts);
        if (e >= 0 && (same & ((1ull << lane) - 1)) == 0) mine[e] += (uint32_t)__popcll(same);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < experts; e += WAVES * kWave)
        for (int w = 1; w < WAVES; ++w) base[w * experts + e] += base[(w - 1) * experts + e];
    __syncthreads();
    uint32_t *const next = base + wave * experts;
    const uint64_t rows = (uint64_t)a.tokens * a.chosen;
    for (uint64_t at = from; at < to; at += kWave) {
        const int32_t e = expert_at(a, at + lane, to);
        const uint64_t same = alike(e, experts), before = same & ((1ull << lane) - 1);
        int32_t row = -1;
        if (e >= 0) row = (int32_t)(next[e] + (uint32_t)__popcll(before));
        if (e >= 0 && before == 0) next[e] += (uint32_t)__popcll(same);      // (the wave's reads above come first: it runs in step)
        if (at + lane < to) a.slots[at + lane] = row;
        if (row >= 0 && (uint64_t)row < rows) a.source[row] = (int32_t)((at + lane) / a.chosen);
    }
}

// offsets and, in `base`, the first row of each expert, plus what `before` says of it, from the counts of all experts in `all` (LDS).  A wave's work.
__device__ inline uint32_t add_up(const RouteJob &a, const uint32_t *all, uint32_t *base, const bool write) {
    const uint32_t lane = threadIdx.x;
    uint32_t sum = 0;
    for (uint32_t e0 = 0; e0 < a.experts; e0 += kWave) {
        const uint32_t e = e0 + lane, n = e < a.experts ? all[e] : 0;
        uint32_t x = n;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const uint32_t y = __shfl_up(x, d);
            if ((int)lane >= d) x += y;
        }
        if (e < a.experts) {
            base[e] += sum + x - n;
            if (write) a.offsets[e] = (int32_t)(sum + x - n);
        }
        sum += __shfl(x, kWave - 1);
    }
    if (write && lane == 0) a.offsets[a.experts] = (int32_t)sum;
    return sum;
}

// A workgroup's tokens at once, or most of them.
constexpr int kChooseThreads = 1024;

template <class T, int L, int R> __global__ __launch_bounds__(kChooseThreads) void choose_kernel(const RouteJob a) {
    __shared__ uint32_t count[kMostExperts];
    clear_counts<kChooseThreads>(a, count);
    __syncthreads();
    const uint32_t first = blockIdx.x * a.a_group, end = a.tokens - first < a.a_group ? a.tokens : first + a.a_group;
    choose<T, L, R, kChooseThreads>(a, first, end, count);
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += kChooseThreads) a.counts[(uint64_t)blockIdx.x * a.experts + e] = (int32_t)count[e];
}

// The counts of an index that is there already.
__global__ __launch_bounds__(256) void count_kernel(const RouteJob a) {
    __shared__ uint32_t count[kMostExperts];
    clear_counts<256>(a, count);
    __syncthreads();
    const uint32_t first = blockIdx.x * a.a_group, end = a.tokens - first < a.a_group ? a.tokens : first + a.a_group;
    for (uint64_t at = (uint64_t)first * a.chosen + threadIdx.x; at < (uint64_t)end * a.chosen; at += 256) {
        const int32_t e = expert_at(a, at, (uint64_t)end * a.chosen);
        if (e >= 0) atomicAdd(&count[e], 1u);
    }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.experts; e += 256) a.counts[(uint64_t)blockIdx.x * a.experts + e] = (int32_t)count[e];
}

// Bound by the way to the counts of the groups, which every workgroup reads: threads that have no expert of their own take a part of the groups, 32 at once (us, 16384 tokens, 8 of 128 experts: 64 one
// count after the other by 256 threads).
constexpr int kOrderWaves = 8;

__global__ __launch_bounds__(kOrderWaves * kWave) void order_kernel(const RouteJob a) {
    constexpr uint32_t kThreads = kOrderWaves * kWave, kAtOnce = 32;
    __shared__ uint32_t base[(kOrderWaves + 1) * kMostExperts], all[kMostExperts], rows_there;
    clear_counts<kThreads>(a, base);
    clear_counts<kThreads>(a, all);
    __syncthreads();
    const uint32_t parts = a.experts >= kThreads ? 1 : kThreads / a.experts, a_part = (a.groups + parts - 1) / parts;
    for (uint32_t i = threadIdx.x; i < parts * a.experts; i += kThreads) {
        const uint32_t part = i / a.experts, e = i - part * a.experts, end = (part + 1) * a_part;
        const uint32_t from = part * a_part < a.groups ? part * a_part : a.groups, to = end < a.groups ? end : a.groups;
        uint32_t before = 0, sum = 0;
        for (uint32_t g0 = from; g0 < to; g0 += kAtOnce) {
            uint32_t n[kAtOnce];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) n[j] = (uint32_t)a.counts[(uint64_t)(g0 + j < to ? g0 + j : to - 1) * a.experts + e];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) {
                if (g0 + j >= to) n[j] = 0;
                if (g0 + j < blockIdx.x) before += n[j];
                sum += n[j];
            }
        }
        if (before) atomicAdd(&base[e], before);
        if (sum) atomicAdd(&all[e], sum);
    }
    __syncthreads();
    if (threadIdx.x < kWave) {
        const uint32_t sum = add_up(a, all, base, blockIdx.x == 0);
        if (threadIdx.x == 0) rows_there = sum;
    }
    __syncthreads();
    const uint32_t first = blockIdx.x * a.a_group, end = a.tokens - first < a.a_group ? a.tokens : first + a.a_group;
    place_choices<kOrderWaves>(a, (uint64_t)first * a.chosen, (uint64_t)end * a.chosen, base);
    for (uint64_t row = (uint64_t)rows_there + blockIdx.x * (kOrderWaves * kWave) + threadIdx.x; row < (uint64_t)a.tokens * a.chosen; row += (uint64_t)a.groups * kOrderWaves * kWave)
        a.source[row] = -1;
}

// Few tokens: everything in one workgroup.
constexpr int kOneThreads = 512;

template <class T, int L, int R> __global__ __launch_bounds__(kOneThreads) void route_one_kernel(const RouteJob a) {
    constexpr int kWaves = kOneThreads / kWave;
    __shared__ uint32_t base[(kWaves + 1) * kMostExperts], all[kMostExperts], rows_there;
    clear_counts<kOneThreads>(a, all);
    clear_counts<kOneThreads>(a, base);
    __syncthreads();
    const uint64_t choices = (uint64_t)a.tokens * a.chosen;
    if (a.logits) choose<T, L, R, kOneThreads>(a, 0, a.tokens, all);
    else
        for (uint64_t at = threadIdx.x; at < choices; at += kOneThreads) {
            const int32_t e = expert_at(a, at, choices);
            if (e >= 0) atomicAdd(&all[e], 1u);
        }
    __threadfence_block();      // (the index is read again by other waves of the workgroup)
    __syncthreads();
    if (threadIdx.x < kWave) {
        const uint32_t sum = add_up(a, all, base, true);
        if (threadIdx.x == 0) rows_there = sum;
    }
    __syncthreads();
    place_choices<kWaves>(a, 0, choices, base);
    for (uint64_t row = rows_there + threadIdx.x; row < choices; row += kOneThreads) a.source[row] = -1;
}

// The gradient of the logits.  L lanes a token and R logits a lane, as in choose.
struct RouteBackJob {
    RouteJob a;
    const float *grad_weights;
    void *grad_logits;
};

template <class T, int L, int R> __global__ __launch_bounds__(256) void route_back_kernel(const RouteBackJob b) {
    const RouteJob &a = b.a;
    const uint32_t lane = threadIdx.x % L, step = gridDim.x * (256 / L);
    for (uint32_t token = blockIdx.x * (256 / L) + threadIdx.x / L; token < a.tokens; token += step) {
        const uint64_t at = (uint64_t)token * a.chosen;
        float p[R], grad[R];
        if (!a.normalise) {
            read_logits<T, R>(a, token, lane * R, p);
            uint32_t most = 0;
#pragma unroll
            for (int r = 0; r < R; ++r) most = most > key_of(p[r]) ? most : key_of(p[r]);
            const float top = value_of(largest<L>(most));
            float sum = 0.0f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                p[r] = key_of(p[r]) == 0 ? 0.0f : expf(p[r] - top);
                sum += p[r];
            }
            sum = total<L>(sum);
#pragma unroll
            for (int r = 0; r < R; ++r) p[r] = p[r] == 0.0f ? 0.0f : p[r] / sum;
        }
        float mean = 0.0f;
        for (uint32_t j = 0; j < a.chosen; ++j)
            if ((uint32_t)a.index[at + j] < a.experts) mean += a.weights[at + j] * b.grad_weights[at + j];
#pragma unroll
        for (int r = 0; r < R; ++r) grad[r] = a.normalise || p[r] == 0.0f ? 0.0f : -p[r] * mean;
        for (uint32_t j = 0; j < a.chosen; ++j) {
            const uint32_t expert = (uint32_t)a.index[at + j], e = expert - lane * R;
            if (expert >= a.experts || e >= (uint32_t)R) continue;
            const float w = a.weights[at + j], g = b.grad_weights[at + j];
#pragma unroll
            for (int r = 0; r < R; ++r)
                if (e == (uint32_t)r) grad[r] = w * (g - mean);
        }
        T *const to = (T *)b.grad_logits + (uint64_t)token * a.experts + lane * R;
        constexpr int E = kPer<T> < R ? kPer<T> : R;
        static_assert(E == kPer<T>);
#pragma unroll
        for (int r = 0; r < R; r += E) {
            float y[E];
#pragma unroll
            for (int e = 0; e < E; ++e) y[e] = grad[r + e];
            store_vec(to + r, (int)a.experts - (int)(lane * R) - r, pack<T>(y));
        }
    }
}

// ---- a token's rows --------------------------------------------------------------------------------------------

struct CombineJob {
    const void *y;                 // [rows, cols]
    const int32_t *slots;
    const float *weights;          // or NULL
    void *out;
    uint64_t tokens, rows, cols;
    uint32_t chosen;
};

// Tin: the rows' type.  G threads a token (a wave, or all 256), a vector of the output's type each, K rows on their way at once.  Bound by memory.
// With few tokens the columns of one are those of several workgroups, blockIdx.y.
template <class Tin, class T, int G, int K> __global__ __launch_bounds__(256) void combine_kernel(const CombineJob a) {
    constexpr int E = kPer<T>, H = E / kPer<Tin>;      // columns of a thread, vectors that they are
    const uint32_t t = threadIdx.x % G;
    for (uint64_t token = (uint64_t)blockIdx.x * (256 / G) + threadIdx.x / G; token < a.tokens; token += (uint64_t)gridDim.x * (256 / G)) {
        const int32_t *const slots = a.slots + token * a.chosen;
        for (uint64_t col = ((uint64_t)blockIdx.y * G + t) * E; col < a.cols; col += (uint64_t)gridDim.y * G * E) {
            const int left = a.cols - col < E ? (int)(a.cols - col) : E, before = col == 0 ? 0 : E;
            float sum[E] = {};
            for (uint32_t j0 = 0; j0 < a.chosen; j0 += K) {
                raw16 v[K][H];
                float w[K];
                bool there[K];
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    const uint64_t slot = j0 + j < a.chosen ? (uint64_t)(int64_t)slots[j0 + j] : ~0ull;
                    there[j] = slot < a.rows;
                    w[j] = there[j] ? a.weights ? a.weights[token * a.chosen + j0 + j] : 1.0f : 0.0f;
                    const Tin *const p = (const Tin *)a.y + (there[j] ? slot : 0) * a.cols + col;
#pragma unroll
                    for (int h = 0; h < H; ++h) v[j][h] = load_vec(p + h * kPer<Tin>, there[j] ? left - h * kPer<Tin> : 0, left - h * kPer<Tin> > 0 ? before + h * kPer<Tin> : 0);
                }
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    if (!there[j]) continue;
#pragma unroll
                    for (int h = 0; h < H; ++h) {
                        float x[kPer<Tin>];
                        unpack<Tin>(v[j][h], x);
#pragma unroll
                        for (int e = 0; e < kPer<Tin>; ++e) sum[h * kPer<Tin> + e] += w[j] * x[e];
                    }
                }
            }
            store_vec((T *)a.out + token * a.cols + col, left, pack<T>(sum));
        }
    }
}

struct CombineBackJob {
    const void *grad_out, *y;
    const int32_t *slots, *last;       // last: offsets[experts]
    const float *weights;
    void *grad_y;
    float *grad_weights;
    uint64_t tokens, rows, cols;
    uint32_t chosen;
};

// G threads a token (a wave, or all 256), K of its rows at a time, or with few tokens in each of several workgroups, blockIdx.y.  The workgroups behind those of the tokens write zeros to the rows of no
// expert.
template <class T, int G, int K> __global__ __launch_bounds__(256) void combine_back_kernel(const CombineBackJob a, const uint32_t groups) {
    constexpr int E = kPer<T>;
    __shared__ float sums[256 / kWave][K];
    const uint32_t t = threadIdx.x % G;
    if (blockIdx.x >= groups) {
        if (!a.grad_y || blockIdx.y != 0) return;
        const int32_t last = *a.last;
        const uint64_t first = last < 0 ? 0 : (uint64_t)last;
        for (uint64_t row = first + (blockIdx.x - groups); row < a.rows; row += gridDim.x - groups)
            for (uint64_t col = (uint64_t)threadIdx.x * E; col < a.cols; col += 256 * E)
                store_vec((T *)a.grad_y + row * a.cols + col, a.cols - col < E ? (int)(a.cols - col) : E, raw16{0, 0, 0, 0});
        return;
    }
    for (uint64_t token0 = (uint64_t)blockIdx.x * (256 / G); token0 < a.tokens; token0 += (uint64_t)groups * (256 / G)) {
        const uint64_t token = token0 + threadIdx.x / G;
        const bool real = token < a.tokens;
        for (uint32_t j0 = blockIdx.y * K; j0 < a.chosen; j0 += gridDim.y * K) {
            uint64_t slot[K];
            float w[K], sum[K];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                slot[j] = real && j0 + j < a.chosen ? (uint64_t)(int64_t)a.slots[token * a.chosen + j0 + j] : ~0ull;
                w[j] = slot[j] < a.rows ? (a.weights ? a.weights[token * a.chosen + j0 + j] : 1.0f) : 0.0f;
                sum[j] = 0.0f;
            }
            for (uint64_t col = (uint64_t)t * E; col < a.cols && real; col += G * E) {
                const int left = a.cols - col < E ? (int)(a.cols - col) : E, before = col == 0 ? 0 : E;
                raw16 v[K];
                const raw16 of_out = load_vec((const T *)a.grad_out + token * a.cols + col, left, before);
                if (a.grad_weights) {
#pragma unroll
                    for (int j = 0; j < K; ++j)
                        if (slot[j] < a.rows) v[j] = load_vec((const T *)a.y + slot[j] * a.cols + col, left, before);
                }
                float g[E];
                unpack<T>(of_out, g);
#pragma unroll
                for (int j = 0; j < K; ++j) {
                    if (slot[j] >= a.rows) continue;
                    if (a.grad_weights) {
                        float x[E];
                        unpack<T>(v[j], x);
#pragma unroll
                        for (int e = 0; e < E; ++e) sum[j] += g[e] * x[e];
                    }
                    if (a.grad_y) {
                        float x[E];
#pragma unroll
                        for (int e = 0; e < E; ++e) x[e] = w[j] * g[e];
                        store_vec((T *)a.grad_y + slot[j] * a.cols + col, left, pack<T>(x));
                    }
                }
            }
            if (!a.grad_weights) continue;
#pragma unroll
            for (int j = 0; j < K; ++j) sum[j] = total<kWave>(sum[j]);
            if constexpr (G == kWave) {
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (real && t == (uint32_t)j && j0 + j < a.chosen) a.grad_weights[token * a.chosen + j0 + j] = slot[j] < a.rows ? sum[j] : 0.0f;
            } else {
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (threadIdx.x % kWave == 0) sums[threadIdx.x / kWave][j] = sum[j];
                __syncthreads();
#pragma unroll
                for (int j = 0; j < K; ++j)
                    if (t == (uint32_t)j && j0 + j < a.chosen) {
                        float s = 0.0f;
                        for (int wave = 0; wave < 256 / kWave; ++wave) s += sums[wave][j];
                        a.grad_weights[token * a.chosen + j0 + j] = slot[j] < a.rows ? s : 0.0f;
                    }
                __syncthreads();
            }
        }
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

// Lanes that a token's logits take.
constexpr uint32_t lanes_of(const uint64_t experts) { return experts <= 64 ? 8 : experts <= 128 ? 16 : experts <= 256 ? 32 : 64; }

struct Groups {
    uint32_t a_group, groups;
};

// The tokens that a workgroup takes at once, up to 64, and no more than 256 workgroups, each of which reads all counts (us, bt_route_forward, bfloat16, 8 of 1024 experts: 1024 tokens with
// 64 tokens a workgroup 57, with 16 26; 16384 tokens with at most 64, 128 and 256 workgroups 178, 102 and 71).
Groups groups_of(const uint64_t tokens, const uint64_t experts) {
    const uint64_t at_once = kChooseThreads / lanes_of(experts), least = at_once < 64 ? at_once : 64;
    const uint64_t a_group = tokens <= least * 256 ? least : (tokens + 255) / 256;
    return {(uint32_t)a_group, (uint32_t)((tokens + a_group - 1) / a_group)};
}

// One workgroup does it all: the order where it has few choices to place, the choice as well where it takes its tokens in at most two turns (us, bt_route_forward, one workgroup and two
// launches: 8 of 64 experts, 64 tokens 7.2 and 11.3; 1 of 128, 64 tokens 6.0 and 7.6, 2048 tokens 70 and 8.9; 1 of 1024, 2048 tokens 466 and 24.
// bt_route_order, 128 experts: 1024 choices 5.7 and 7.5, 2048 8.6 and 7.5).
constexpr uint64_t kOneChoices = 1024;
bool one_orders(const bt_expert_plan &p) { return p.tokens * p.chosen <= kOneChoices; }
bool one_chooses(const bt_expert_plan &p) { return one_orders(p) && p.tokens * lanes_of(p.experts) <= 2 * kOneThreads; }

RouteJob job_of(const bt_expert_plan &p, void *workspace) {
    RouteJob a = {};
    a.index = p.d_index;
    a.slots = p.d_slots;
    a.source = p.d_source;
    a.offsets = p.d_offsets;
    a.counts = (int32_t *)workspace;
    a.tokens = (uint32_t)p.tokens;
    a.experts = (uint32_t)p.experts;
    a.chosen = (uint32_t)p.chosen;
    const Groups g = groups_of(p.tokens, p.experts);
    a.a_group = g.a_group;
    a.groups = g.groups;
    return a;
}

// Lanes a token and logits a lane: whole vectors of either width.
template <class Go> bt_status with_lanes(const uint32_t experts, Go go) {
    using std::integral_constant;
    if (lanes_of(experts) == 8) return go(integral_constant<int, 8>{}, integral_constant<int, 8>{});
    if (lanes_of(experts) == 16) return go(integral_constant<int, 16>{}, integral_constant<int, 8>{});
    if (lanes_of(experts) == 32) return go(integral_constant<int, 32>{}, integral_constant<int, 8>{});
    if (experts <= 512) return go(integral_constant<int, 64>{}, integral_constant<int, 8>{});
    return go(integral_constant<int, 64>{}, integral_constant<int, 16>{});
}

bt_status check_tables(const bt_expert_plan &p, const void *ws, const size_t bytes) {
    const bool some = p.tokens != 0;
    if (p.d_offsets == nullptr || (some && (p.d_index == nullptr || p.d_slots == nullptr || p.d_source == nullptr))) return BT_ERR_NULL;
    const size_t need = bt_route_workspace_bytes(p.tokens, p.experts, p.chosen);
    if (need != 0 && ws == nullptr) return BT_ERR_NULL;
    if (misaligned(p.d_index, 4) || misaligned(p.d_slots, 4) || misaligned(p.d_source, 4) || misaligned(p.d_offsets, 4) || misaligned(ws, 128)) return BT_ERR_ALIGN;
    return bytes < need ? BT_ERR_WORKSPACE : BT_OK;
}

bt_status order(const RouteJob &a, hipStream_t hs) { return launch(order_kernel, dim3(a.groups), kOrderWaves * kWave, hs, a); }

// Into how many pieces a token's work goes, of those that it has, where `groups` workgroups take the tokens: while there are no more than the 1024 that keep the card busy (us, one token, bfloat16: forward, 2 rows of 16384
// columns 7.2 -> 2.9, 32 rows 58 -> 9.7, float32 8 rows 31 -> 4.1; backward 32 rows of 4096 24 -> 5.0).
unsigned pieces_of(const uint64_t groups, const uint64_t there) {
    const uint64_t wanted = 1024 / groups;
    return (unsigned)(wanted <= 1 ? 1 : wanted < there ? wanted : there);
}

template <class Tin, class T> bt_status combine(const bt_expert_plan &p, const void *y, const float *weights, const uint64_t cols, void *out, hipStream_t hs) {
    CombineJob a = {};
    a.y = y;
    a.slots = p.d_slots;
    a.weights = weights;
    a.out = out;
    a.tokens = p.tokens;
    a.rows = p.tokens * p.chosen;
    a.cols = cols;
    a.chosen = (uint32_t)p.chosen;
    const auto go = [&](auto kernel, const int a_group) {
        const uint64_t blocks = (a.tokens + a_group - 1) / a_group;
        const uint64_t a_piece = 256 / a_group * kPer<T>;
        return launch(kernel, dim3((unsigned)(blocks < 1u << 20 ? blocks : 1u << 20), pieces_of(blocks, (cols + a_piece - 1) / a_piece)), 256, hs, a);
    };
    const bool wide = cols > 64 * kPer<T> * 2;
    if (a.chosen <= 2) return wide ? go(combine_kernel<Tin, T, 256, 2>, 1) : go(combine_kernel<Tin, T, 64, 2>, 4);
    if (a.chosen <= 4) return wide ? go(combine_kernel<Tin, T, 256, 4>, 1) : go(combine_kernel<Tin, T, 64, 4>, 4);
    return wide ? go(combine_kernel<Tin, T, 256, 8>, 1) : go(combine_kernel<Tin, T, 64, 8>, 4);
}

}  // namespace

bt_status sum_rows(const bt_expert_plan &p, const float *y, const uint64_t cols, const bt_dtype dtype, void *out, hipStream_t hs) {
    return with_type(dtype, [&](auto type) { return combine<float, decltype(type)>(p, y, nullptr, cols, out, hs); });
}

bt_status check_plan(const bt_expert_plan *p) {
    if (p == nullptr) return BT_ERR_NULL;
    if (p->experts == 0 || p->experts > BT_MAX_EXPERTS || p->chosen == 0 || p->chosen > BT_MAX_CHOSEN || p->chosen > p->experts) return BT_ERR_SIZE;
    return p->tokens > BT_MAX_ROWS / p->chosen ? BT_ERR_SIZE : BT_OK;
}

}  // namespace btb

using namespace btb;

extern "C" {

size_t bt_route_workspace_bytes(uint64_t tokens, uint64_t experts, uint64_t chosen) {
    const bt_expert_plan p = {tokens, experts, chosen, nullptr, nullptr, nullptr, nullptr};
    if (check_plan(&p) != BT_OK || one_chooses(p)) return 0;
    return ((size_t)groups_of(tokens, experts).groups * experts * 4 + 127) / 128 * 128;
}

bt_status bt_route_forward(const void *d_logits, bt_dtype dtype, int normalise, const bt_expert_plan *plan, float *d_weights,
                           void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check_plan(plan);
    if (st != BT_OK) return st;
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (plan->tokens != 0 && (d_logits == nullptr || d_weights == nullptr)) return BT_ERR_NULL;
    if (misaligned(d_logits, (size_t)width_of(dtype)) || misaligned(d_weights, 4)) return BT_ERR_ALIGN;
    st = check_tables(*plan, d_workspace, workspace_bytes);
    if (st != BT_OK) return st;
    const hipStream_t hs = (hipStream_t)stream;
    RouteJob a = job_of(*plan, d_workspace);
    a.logits = plan->tokens != 0 ? d_logits : nullptr;
    a.weights = d_weights;
    a.normalise = normalise != 0;
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_lanes(a.experts, [&](auto lanes, auto each) {
            constexpr int L = decltype(lanes)::value, R = decltype(each)::value;
            if (one_chooses(*plan)) return launch(route_one_kernel<T, L, R>, dim3(1), kOneThreads, hs, a);
            const bt_status s = launch(choose_kernel<T, L, R>, dim3(a.groups), kChooseThreads, hs, a);
            return s == BT_OK ? order(a, hs) : s;
        });
    });
}

bt_status bt_route_order(const bt_expert_plan *plan, void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check_plan(plan);
    if (st != BT_OK) return st;
    st = check_tables(*plan, d_workspace, workspace_bytes);
    if (st != BT_OK) return st;
    const hipStream_t hs = (hipStream_t)stream;
    RouteJob a = job_of(*plan, d_workspace);
    const Groups g = groups_of(plan->tokens, 1);      // (counting takes no lanes of a token: no more groups than the workspace has room for)
    a.a_group = g.a_group;
    a.groups = g.groups;
    if (one_orders(*plan)) return launch(route_one_kernel<float, 8, 8>, dim3(1), kOneThreads, hs, a);
    st = launch(count_kernel, dim3(a.groups), 256, hs, a);
    return st == BT_OK ? order(a, hs) : st;
}

bt_status bt_route_backward(const float *d_grad_weights, const void *d_logits, bt_dtype dtype, int normalise, const bt_expert_plan *plan,
                            const float *d_weights, void *d_grad_logits, bt_stream stream) {
    const bt_status st = check_plan(plan);
    if (st != BT_OK) return st;
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (plan->tokens == 0) return BT_OK;
    if (d_grad_weights == nullptr || (d_logits == nullptr && !normalise) || plan->d_index == nullptr || d_weights == nullptr || d_grad_logits == nullptr) return BT_ERR_NULL;
    const size_t w = (size_t)width_of(dtype);
    if (misaligned(d_grad_weights, 4) || misaligned(d_logits, w) || misaligned(plan->d_index, 4) || misaligned(d_weights, 4) || misaligned(d_grad_logits, w)) return BT_ERR_ALIGN;
    RouteBackJob b = {job_of(*plan, nullptr), d_grad_weights, d_grad_logits};
    b.a.logits = d_logits;
    b.a.weights = const_cast<float *>(d_weights);      // (read alone)
    b.a.normalise = normalise != 0;
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_lanes(b.a.experts, [&](auto lanes, auto each) {
            constexpr int L = decltype(lanes)::value, R = decltype(each)::value;
            const uint64_t blocks = (plan->tokens + 256 / L - 1) / (256 / L);
            return launch(route_back_kernel<T, L, R>, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), 256, (hipStream_t)stream, b);
        });
    });
}

bt_status bt_combine_forward(const void *d_y, const bt_expert_plan *plan, const float *d_weights, uint64_t cols, bt_dtype dtype, void *d_out, bt_stream stream) {
    const bt_status st = check_plan(plan);
    if (st != BT_OK) return st;
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (cols > BT_MAX_FEATURES) return BT_ERR_SIZE;
    if (plan->tokens == 0 || cols == 0) return BT_OK;
    if (d_y == nullptr || plan->d_slots == nullptr || d_out == nullptr) return BT_ERR_NULL;
    const size_t w = (size_t)width_of(dtype);
    if (misaligned(d_y, w) || misaligned(plan->d_slots, 4) || misaligned(d_weights, 4) || misaligned(d_out, w)) return BT_ERR_ALIGN;
    return with_type(dtype, [&](auto type) { return combine<decltype(type), decltype(type)>(*plan, d_y, d_weights, cols, d_out, (hipStream_t)stream); });
}

bt_status bt_combine_backward(const void *d_grad_out, const void *d_y, const bt_expert_plan *plan, const float *d_weights, uint64_t cols, bt_dtype dtype,
                              void *d_grad_y, float *d_grad_weights, bt_stream stream) {
    const bt_status st = check_plan(plan);
    if (st != BT_OK) return st;
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    if (cols > BT_MAX_FEATURES) return BT_ERR_SIZE;
    if (plan->tokens == 0 || (d_grad_y == nullptr && d_grad_weights == nullptr) || (cols == 0 && d_grad_weights == nullptr)) return BT_OK;
    const size_t w = (size_t)width_of(dtype);
    if (plan->d_slots == nullptr || plan->d_offsets == nullptr || (cols != 0 && (d_grad_out == nullptr || (d_grad_weights && d_y == nullptr)))) return BT_ERR_NULL;
    if (misaligned(d_grad_out, w) || misaligned(d_y, w) || misaligned(plan->d_slots, 4) || misaligned(plan->d_offsets, 4) || misaligned(d_weights, 4) ||
        misaligned(d_grad_y, w) || misaligned(d_grad_weights, 4))
        return BT_ERR_ALIGN;
    CombineBackJob a = {};
    a.grad_out = d_grad_out;
    a.y = d_y;
    a.slots = plan->d_slots;
    a.last = plan->d_offsets + plan->experts;
    a.weights = d_weights;
    a.grad_y = d_grad_y;
    a.grad_weights = d_grad_weights;
    a.tokens = plan->tokens;
    a.rows = plan->tokens * plan->chosen;
    a.cols = cols;
    a.chosen = (uint32_t)plan->chosen;
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        const auto go = [&](auto kernel, const int a_group, const uint32_t at_once) {
            const uint64_t blocks = (a.tokens + a_group - 1) / a_group;
            const uint32_t groups = (uint32_t)(blocks < 1u << 20 ? blocks : 1u << 20), rest = groups < 256 ? groups : 256;
            return launch(kernel, dim3(groups + (d_grad_y ? rest : 0), pieces_of(groups, (a.chosen + at_once - 1) / at_once)), 256, (hipStream_t)stream, a, groups);
        };
        const bool wide = cols > 64 * kPer<T> * 2;
        if (a.chosen <= 2) return wide ? go(combine_back_kernel<T, 256, 2>, 1, 2) : go(combine_back_kernel<T, 64, 2>, 4, 2);
        return wide ? go(combine_back_kernel<T, 256, 4>, 1, 4) : go(combine_back_kernel<T, 64, 4>, 4, 4);
    });
}

}  // extern "C"
