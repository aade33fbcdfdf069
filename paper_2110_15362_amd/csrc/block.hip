// The norms, gate and residual sum between two blocks, and the clipping of gradients: see include/bittrain.h for the contract.
//
// Both are bound by memory: a handful of operations an element against 2 or 4 bytes of it.  What matters is that every tensor
// crosses the memory bus once, in 16-byte vectors, with enough of them on their way.
#include <math.h>

#include "block.h"

namespace btb {
namespace {

// ---- reductions ------------------------------------------------------------------------------------------------

// The sum over a wave, in every lane: the same order always.
template <class F> __device__ inline F wave_sum(F x) {
#pragma unroll
    for (int d = kWave / 2; d > 0; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// The sum over the NT threads that share a row, in each of them.  `room` has a slot for each wave of the workgroup; calls in turn take
// two rooms in turn, so that one barrier a call is enough.
template <int NT> __device__ inline float row_sum(float x, float *room) {
    x = wave_sum(x);
    if constexpr (NT > kWave) {
        if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = x;
        __syncthreads();
        x = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / kWave; ++w) x += room[w];
    }
    return x;
}

// ---- norms around a block ------------------------------------------------------------------------------------------
//
// A row stays in the registers of the threads that share it: NT threads hold V vectors each, vector i of thread t being number
// i * NT + t of the row, so that the root mean squares are known before anything is read twice.
//
// Forward, bytes read and written at the least: x, block, out and y (bf16 [16384, 4096]: 97.5 us, 5.5 TB/s; f32 [8192, 1024]: 27.6 us, 4.9 TB/s; one row
// of 4096: 3.4 us, the time of a launch and of one way to memory and back).

struct NormForward {
    const void *x, *block, *post_weight, *gate, *pre_weight;
    void *out, *y;
    float *stats;
    uint32_t rows, cols, rows_a_gate, first_row;
    float eps, scale, residual_scale;
};

template <int NT> constexpr int kRowsABlock = NT < 256 ? 256 / NT : 1;

template <class T, int NT, int V>
__global__ __launch_bounds__(NT < 256 ? 256 : NT) void norm_forward_kernel(const NormForward a) {
    constexpr int E = kPer<T>;
    static_assert(NT == kWave || NT >= 256, "a workgroup's barrier is one row's");
    __shared__ float room[2][NT > kWave ? NT / kWave : 1];
    const int t = threadIdx.x % NT;
    const uint32_t row = a.first_row + blockIdx.x * kRowsABlock<NT> + threadIdx.x / NT;
    if (row >= a.rows) return;
    const uint64_t at = (uint64_t)row * a.cols;
    const int cols = (int)a.cols;
    const float inverse = 1.0f / (float)a.cols;
    raw16 x[V], b[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (i * NT + t) * E;
        x[i] = load_vec((const T *)a.x + at + c, cols - c, c);
        if (a.block) b[i] = load_vec((const T *)a.block + at + c, cols - c, c);
    }
    float rb = 1.0f;
    if (a.post_weight) {
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float f[E];
            unpack<T>(b[i], f);
#pragma unroll
            for (int e = 0; e < E; ++e) sum = fmaf(f[e], f[e], sum);
        }
        rb = 1.0f / sqrtf(row_sum<NT>(sum, room[0]) * inverse + a.eps);
    }
    float out[V][E], sum = 0.0f;
    const uint64_t gate_at = a.gate ? (uint64_t)(row / a.rows_a_gate) * a.cols : 0;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (i * NT + t) * E;
        unpack<T>(x[i], out[i]);
        if (a.block) {
            float f[E], w[E];
            unpack<T>(b[i], f);
            if (a.post_weight) {
                unpack<T>(load_vec((const T *)a.post_weight + c, cols - c, c), w);
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] = f[e] * rb * w[e];
            }
            if (a.gate) {
                unpack<T>(load_vec((const T *)a.gate + gate_at + c, cols - c, c), w);
#pragma unroll
                for (int e = 0; e < E; ++e) f[e] *= w[e];
            }
#pragma unroll
            for (int e = 0; e < E; ++e) out[i][e] = fmaf(a.scale, f[e], a.residual_scale * out[i][e]);
            if (c < cols) store_vec((T *)a.out + at + c, cols - c, pack<T>(out[i]));
        }
#pragma unroll
        for (int e = 0; e < E; ++e) sum = fmaf(out[i][e], out[i][e], sum);
    }
    float ro = 1.0f;
    if (a.pre_weight) {
        ro = 1.0f / sqrtf(row_sum<NT>(sum, room[1]) * inverse + a.eps);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * NT + t) * E;
            if (c >= cols) continue;
            float w[E];
            unpack<T>(load_vec((const T *)a.pre_weight + c, cols - c, c), w);
#pragma unroll
            for (int e = 0; e < E; ++e) w[e] *= out[i][e] * ro;
            store_vec((T *)a.y + at + c, cols - c, pack<T>(w));
        }
    }
    if (a.stats && t == 0) {
        a.stats[row] = rb;
        a.stats[(uint64_t)a.rows + row] = ro;
    }
}

// The backward pass.  With v = out ro, z = block rb and the sums over a row as means:
//   total = grad_out + ro (grad_y wn - v mean(grad_y wn v))     grad_x = residual_scale total
//   dn = scale total gate     grad_block = rb (dn wp - z mean(dn wp z))
// and, summed over the rows that share them, grad_gate = scale total z wp, grad_post_weight = dn z, grad_pre_weight = grad_y v.
// A workgroup takes a run of rows, one after the other, and keeps its columns' sums in registers; its partial sums go to the workspace
// and are joined by norm_join_kernel.
// `out` is the tensor that the forward pass stored, rounded to the type, and ro that of the row before it was: half the bytes of a copy in 32 bits, for an error of half a
// unit in the last place of each v (bf16 [4095, 1999], all gradients: off by 0.0023, in the mean of squares, and with out in 32 bits by 0.0017).
struct NormBackward {
    const void *grad_out, *grad_y, *out, *block, *post_weight, *gate, *pre_weight;
    const float *stats;
    void *grad_x, *grad_block, *grad_post_weight, *grad_gate, *grad_pre_weight;
    float *part_post, *part_pre, *part_gate;      // [runs, cols], [runs, cols], [runs, 2, cols]
    uint32_t rows, cols, rows_a_gate, gate_rows, runs;
    float scale, residual_scale;
};

// `p`, which the compiler takes for another one each time: what is read there is read again, not held in registers.
template <class T> __device__ inline const T *again(const T *p) {
    asm volatile("" : "+s"(p));
    return p;
}

// Backward: x, block, grad_out and grad_y are read and two gradients written; the weights' are sums over the rows, which a workgroup makes in its registers
// over a run of rows and a second kernel over the runs, in order, so that no result depends on who came first.  (f32 [8192, 1024]: 37.6 us, 5.4 TB/s;
// bf16 [4096, 16384]: 230 us, 3.5 TB/s, where registers hold one row's vectors alone; bf16 [4095, 1999] with a gate a row, off all boundaries: 36.7 us, 3.6
// TB/s.)
__device__ __host__ inline uint32_t run_start(const uint32_t run, const uint32_t rows, const uint32_t runs) {
    return (uint32_t)((uint64_t)run * rows / runs);
}

template <class T, int NT, int V>
__global__ __launch_bounds__(NT, 4) void norm_backward_kernel(const NormBackward a) {
    constexpr int E = kPer<T>;
    // 16 columns a thread of a full workgroup: three sums of each are more than its registers hold beside the row, so two of them are kept in LDS
    // (128 of 160 KiB; 256 KiB of LDS traffic a row of 16384, a tenth of the time that the row takes from memory).
    constexpr bool kWide = V * E > 8;
    // Workgroups of up to 512 threads have registers for two rows and for what all rows share; of 1024, half as many a thread, for one row's
    // sums; where two of those are in LDS a row's vectors are read again (from the caches) rather than held.
    constexpr bool kAhead = NT <= 512;
    __shared__ float room[2][NT / kWave];
    __shared__ float kept[kWide ? 2 : 1][kWide ? V * E : 1][kWide ? NT : 1];
    const int t = threadIdx.x;
    const int cols = (int)a.cols;
    const float inverse = 1.0f / (float)a.cols;
    const uint32_t first = run_start(blockIdx.x, a.rows, a.runs), end = run_start(blockIdx.x + 1, a.rows, a.runs);
    float sum_post[kWide ? 1 : V][E], sum_pre[kWide ? 1 : V][E], sum_gate[V][E];
    const auto add_post = [&](const int i, const int e, const float p, const float q) {
        float &sum = kWide ? kept[0][kWide ? i * E + e : 0][kWide ? t : 0] : sum_post[kWide ? 0 : i][e];
        sum = fmaf(p, q, sum);
    };
    const auto add_pre = [&](const int i, const int e, const float p, const float q) {
        float &sum = kWide ? kept[kWide][kWide ? i * E + e : 0][kWide ? t : 0] : sum_pre[kWide ? 0 : i][e];
        sum = fmaf(p, q, sum);
    };
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) {
            sum_gate[i][e] = 0.0f;
            if constexpr (kWide) kept[0][i * E + e][t] = kept[1][i * E + e][t] = 0.0f;
            else sum_post[i][e] = sum_pre[i][e] = 0.0f;
        }
    // The gate row of the row at hand and where its rows begin and end.
    uint32_t group = 0, group_first = 0, group_end = ~0u;
    if (a.gate) {
        group = first / a.rows_a_gate;
        group_first = group * a.rows_a_gate;
        group_end = group_first + a.rows_a_gate;
    }
    // What follows from the thread's number is worked out again each time where it would take registers that hold the row.
    const auto number = [&] {
        int n = t;
        if (kWide || sizeof(T) == 2) asm volatile("" : "+v"(n));
        return n;
    };
    // A row's vectors: with kAhead the next row's are on their way while one is worked on.
    struct Row {
        raw16 gy[V], o[V], go[V], b[V];
        float rb, ro;
    };
    const auto load = [&](Row &r, const uint32_t row) {
        const uint64_t at = (uint64_t)row * a.cols;
        r.rb = a.block ? a.stats[row] : 1.0f;
        r.ro = a.grad_y ? a.stats[(uint64_t)a.rows + row] : 1.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * NT + number()) * E;
            if (a.grad_y) {
                r.gy[i] = load_vec((const T *)a.grad_y + at + c, cols - c, c);
                r.o[i] = load_vec((const T *)a.out + at + c, cols - c, c);
            }
            if (!kAhead) continue;
            if (a.grad_out) r.go[i] = load_vec((const T *)a.grad_out + at + c, cols - c, c);
            if (a.block) r.b[i] = load_vec((const T *)a.block + at + c, cols - c, c);
        }
    };
    // What all rows share, or a group's do.
    raw16 wn[V], wp[V], gate[V];
    const auto load_gate = [&] {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * NT + t) * E;
            if (kAhead && a.gate) gate[i] = load_vec((const T *)a.gate + (uint64_t)group * a.cols + c, cols - c, c);
        }
    };
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (i * NT + t) * E;
        if (kAhead && a.pre_weight) wn[i] = load_vec((const T *)a.pre_weight + c, cols - c, c);
        if (kAhead && a.post_weight) wp[i] = load_vec((const T *)a.post_weight + c, cols - c, c);
    }
    load_gate();
    Row next;
    if (kAhead) load(next, first);
    for (uint32_t row = first; row < end; ++row) {
        const uint64_t at = (uint64_t)row * a.cols;
        Row r;
        if constexpr (kAhead) {
            r = next;
            if (row + 1 < end) load(next, row + 1);
        } else load(r, row);
        float total[V][E], mean = 0.0f;
        if (a.grad_y) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * NT + number()) * E;
                float g[E], v[E], w[E];
                unpack<T>(r.gy[i], g);
                unpack<T>(r.o[i], v);
                unpack<T>(!kAhead ? load_vec(again((const T *)a.pre_weight) + c, cols - c, c) : wn[i], w);
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[e] *= r.ro;
                    add_pre(i, e, g[e], v[e]);
                    mean = fmaf(g[e] * w[e], v[e], mean);
                }
            }
            mean = row_sum<NT>(mean, room[0]) * inverse;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * NT + number()) * E;
                float g[E], v[E], w[E];
                unpack<T>(kWide ? load_vec((const T *)a.grad_y + at + c, cols - c, c) : r.gy[i], g);
                unpack<T>(kWide ? load_vec((const T *)a.out + at + c, cols - c, c) : r.o[i], v);
                unpack<T>(!kAhead ? load_vec(again((const T *)a.pre_weight) + c, cols - c, c) : wn[i], w);
#pragma unroll
                for (int e = 0; e < E; ++e) total[i][e] = r.ro * (g[e] * w[e] - v[e] * r.ro * mean);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) total[i][e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * NT + number()) * E;
            if (a.grad_out) {
                float g[E];
                unpack<T>(!kAhead ? load_vec((const T *)a.grad_out + at + c, cols - c, c) : r.go[i], g);
#pragma unroll
                for (int e = 0; e < E; ++e) total[i][e] += g[e];
            }
            if (a.grad_x && c < cols) {
                float g[E];
#pragma unroll
                for (int e = 0; e < E; ++e) g[e] = a.block ? a.residual_scale * total[i][e] : total[i][e];
                store_vec((T *)a.grad_x + at + c, cols - c, pack<T>(g));
            }
        }
        if (!a.block) {
            if constexpr (NT > kWave) __syncthreads();      // (one room only is used)
            continue;
        }
        if (row >= group_end) {
            ++group;
            group_first = group_end;
            group_end += a.rows_a_gate;
            load_gate();
        }
        const bool last_of_group = row + 1 == group_end || row + 1 == end;
        float kept_z[kWide ? 1 : V][E];
        mean = 0.0f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int c = (i * NT + number()) * E;
            float w[E];
            float (&z)[E] = kept_z[kWide ? 0 : i];
            unpack<T>(!kAhead ? load_vec((const T *)a.block + at + c, cols - c, c) : r.b[i], z);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                z[e] *= r.rb;
                w[e] = 1.0f;
                total[i][e] *= a.scale;
            }
            if (a.post_weight) unpack<T>(!kAhead ? load_vec(again((const T *)a.post_weight) + c, cols - c, c) : wp[i], w);
            if (a.gate) {
#pragma unroll
                for (int e = 0; e < E; ++e) sum_gate[i][e] = fmaf(total[i][e], z[e] * w[e], sum_gate[i][e]);
                float g[E];
                unpack<T>(!kAhead ? load_vec(again((const T *)a.gate) + (uint64_t)group * a.cols + c, cols - c, c) : gate[i], g);
#pragma unroll
                for (int e = 0; e < E; ++e) total[i][e] *= g[e];
                if (last_of_group && a.grad_gate && c < cols) {
                    // A group that lies in this run is done; the part of one that goes beyond it is kept for the join, apart from that of
                    // one that came from the run before.
                    if (group_first >= first && group_end <= end) store_vec((T *)a.grad_gate + (uint64_t)group * a.cols + c, cols - c, pack<T>(sum_gate[i]));
                    else {
                        float *const to = a.part_gate + ((uint64_t)blockIdx.x * 2 + (group_first >= first ? 1 : 0)) * a.cols + c;
#pragma unroll
                        for (int e = 0; e < E; ++e)
                            if (c + e < cols) to[e] = sum_gate[i][e];
                    }
                }
                if (last_of_group)
#pragma unroll
                    for (int e = 0; e < E; ++e) sum_gate[i][e] = 0.0f;
            }
            if (a.post_weight) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    add_post(i, e, total[i][e], z[e]);
                    total[i][e] *= w[e];
                    mean = fmaf(total[i][e], z[e], mean);
                }
            }
        }
        if (a.post_weight) {
            mean = row_sum<NT>(mean, room[1]) * inverse;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float (&z)[E] = kept_z[kWide ? 0 : i];
                if (kWide) {
                    const int c = (i * NT + number()) * E;
                    unpack<T>(load_vec((const T *)a.block + at + c, cols - c, c), z);
#pragma unroll
                    for (int e = 0; e < E; ++e) z[e] *= r.rb;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) total[i][e] = r.rb * (total[i][e] - z[e] * mean);
            }
        }
        if (a.grad_block)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int c = (i * NT + number()) * E;
                if (c < cols) store_vec((T *)a.grad_block + at + c, cols - c, pack<T>(total[i]));
            }
        // (Where a row uses both rooms, each is read before its threads come to the barrier of the other.)
        if constexpr (NT > kWave)
            if (!a.grad_y || !a.post_weight) __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = (i * NT + t) * E;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c + e < cols) {
                if (a.grad_post_weight) a.part_post[(uint64_t)blockIdx.x * a.cols + c + e] = kWide ? kept[0][kWide ? i * E + e : 0][kWide ? t : 0] : sum_post[kWide ? 0 : i][e];
                if (a.grad_pre_weight) a.part_pre[(uint64_t)blockIdx.x * a.cols + c + e] = kWide ? kept[kWide][kWide ? i * E + e : 0][kWide ? t : 0] : sum_pre[kWide ? 0 : i][e];
            }
    }
}

// The runs' partial sums, added up: blockIdx.y 0 for post_weight, 1 for pre_weight, from 2 on for the gate rows ("groups" of rows) that more
// than one run has a part of.  A workgroup has 32 columns, half a wave a run, 16 runs of each on their way at once: there are few workgroups, and what
// they have on its way bounds them ([1024 runs, 1024], two weights: 6.0 us; one run a wave at a time and 64 columns: 9.0).
constexpr int kJoinCols = 32, kJoinTeams = 32, kJoinAtOnce = 16;

template <class T> __global__ __launch_bounds__(kJoinCols * kJoinTeams) void norm_join_kernel(const NormBackward a) {
    __shared__ float part[kJoinTeams][kJoinCols];
    const int lane = threadIdx.x % kJoinCols, team = threadIdx.x / kJoinCols;
    const uint32_t c = blockIdx.x * kJoinCols + lane;
    uint32_t from = 0, to = a.runs;       // runs
    const float *parts = blockIdx.y == 0 ? a.part_post : a.part_pre;
    T *result = (T *)(blockIdx.y == 0 ? a.grad_post_weight : a.grad_pre_weight);
    uint64_t pitch = a.cols;
    if (blockIdx.y >= 2) {
        // The group, and the first run that begins behind its first row.  (A run begins at floor(run * rows / runs), at or behind row r from run
        // ceil(r * runs / rows) on.)  Up to `runs` groups are looked at one by one, of more only those that a run begins inside of.
        const auto run_from = [&](const uint32_t row) { return (uint32_t)(((uint64_t)row * a.runs + a.rows - 1) / a.rows); };
        uint32_t group = blockIdx.y - 2, run = blockIdx.y - 1;
        if (a.gate_rows <= a.runs) run = run_from(group * a.rows_a_gate + 1);
        else group = run_start(run, a.rows, a.runs) / a.rows_a_gate;
        const uint32_t first = group * a.rows_a_gate, end = first + a.rows_a_gate;
        if (run >= a.runs || run_start(run, a.rows, a.runs) >= end) return;                  // within one run, which has written it
        if (run_start(run, a.rows, a.runs) == first || run_start(run - 1, a.rows, a.runs) > first) return;      // another workgroup's
        from = run - 1;
        to = run_from(end);
        parts = a.part_gate;
        pitch = 2 * (uint64_t)a.cols;
        result = a.grad_gate ? (T *)a.grad_gate + (uint64_t)group * a.cols : nullptr;
    }
    if (result == nullptr) return;
    float sum = 0.0f;
    if (c < a.cols) {
        // (A gate row's part lies in the second place of the run that it begins in, in the first of the others.)
        uint32_t run = from + team;
        if (blockIdx.y >= 2 && team == 0) {
            sum = parts[run * pitch + a.cols + c];
            run += kJoinTeams;
        }
        for (; run + (kJoinAtOnce - 1) * kJoinTeams < to; run += kJoinAtOnce * kJoinTeams) {
            float x[kJoinAtOnce];
#pragma unroll
            for (int i = 0; i < kJoinAtOnce; ++i) x[i] = parts[(run + i * kJoinTeams) * pitch + c];
#pragma unroll
            for (int i = 0; i < kJoinAtOnce; ++i) sum += x[i];
        }
#pragma unroll 4
        for (; run < to; run += kJoinTeams) sum += parts[run * pitch + c];
    }
    part[team][lane] = sum;
    __syncthreads();
    if (team == 0 && c < a.cols) {
#pragma unroll
        for (int w = 1; w < kJoinTeams; ++w) sum += part[w][lane];
        result[c] = narrow<T>(sum);
    }
}

// ---- the norm of gradients and their clipping -----------------------------------------------------------------------
//
// Up to kTable tensors a launch, laid end to end in chunks of 32 KiB.  The workgroups of a launch take the chunks in turn and leave one
// partial sum each, in 64 bits: squares of any float fit them, so there is no range to mind.

constexpr int kTable = 168;
constexpr int kChunk = 32768;                  // bytes
constexpr int kClipThreads = 256;
constexpr int kClipVecs = kChunk / kVec / kClipThreads;
constexpr uint32_t kSums = 1024;               // workgroups of a launch that sums, and partial sums of it
constexpr uint32_t kScalers = 2048;            // workgroups of a launch that scales

struct ClipTable {
    const void *in[kTable];
    void *out[kTable];
    uint32_t start[kTable];                    // first chunk; of a tensor that is not there more than there are
    uint32_t last[kTable];                     // elements of the last chunk, and the type in the two highest bits
    uint32_t chunks;
};
static_assert(sizeof(ClipTable) + 5 * 8 <= 4096, "kernel arguments");

struct Piece {
    const void *in;
    void *out;
    uint64_t first;
    uint32_t left;                             // elements of the piece
    int dtype;
};

__device__ inline Piece piece_of(const ClipTable &a, const uint32_t chunk) {
    // the last tensor that starts at or before the chunk
    const int lane = threadIdx.x % kWave;
    int i = -1;
#pragma unroll
    for (int from = 0; from < kTable; from += kWave) i += __popcll(__ballot(from + lane < kTable && a.start[from + lane < kTable ? from + lane : 0] <= chunk));
    const int k = __builtin_amdgcn_readfirstlane(i);
    Piece p;
    p.dtype = a.last[k] >> 30;
    const uint32_t per = p.dtype == BT_F32 ? kChunk / 4 : kChunk / 2, end = k + 1 < kTable && a.start[k + 1] < a.chunks ? a.start[k + 1] : a.chunks;
    p.first = (uint64_t)(chunk - a.start[k]) * per;
    p.in = a.in[k];
    p.out = a.out[k];
    p.left = chunk + 1 == end ? a.last[k] & 0x3fffffffu : per;
    return p;
}

template <class T> __device__ inline void load_chunk(const Piece &p, raw16 (&v)[kClipVecs]) {
    const T *const in = (const T *)p.in + p.first;
    if (p.left == kChunk / sizeof(T)) {
#pragma unroll
        for (int i = 0; i < kClipVecs; ++i) v[i] = reinterpret_cast<const Unaligned<T> *>(in + (i * kClipThreads + threadIdx.x) * kPer<T>)->v;
        return;
    }
#pragma unroll
    for (int i = 0; i < kClipVecs; ++i) {
        const int c = (int)((i * kClipThreads + threadIdx.x) * kPer<T>);
        v[i] = load_vec(in + c, (int)p.left - c, p.first != 0 ? kPer<T> : c);
    }
}

__device__ inline void load_chunk(const Piece &p, raw16 (&v)[kClipVecs]) {
    if (p.dtype == BT_F32) load_chunk<float>(p, v);
    else load_chunk<bf16>(p, v);      // (bits)
}

template <class T> __device__ inline double sum_chunk(const raw16 (&v)[kClipVecs]) {
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < kClipVecs; ++i) {
        float x[kPer<T>];
        unpack<T>(v[i], x);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) sum = fma((double)x[e], (double)x[e], sum);
    }
    return sum;
}

template <class T> __device__ inline void scale_chunk(const Piece &p, const raw16 (&v)[kClipVecs], const float factor) {
    T *const out = (T *)p.out + p.first;
#pragma unroll
    for (int i = 0; i < kClipVecs; ++i) {
        const int c = (int)((i * kClipThreads + threadIdx.x) * kPer<T>);
        float x[kPer<T>];
        unpack<T>(v[i], x);
#pragma unroll
        for (int e = 0; e < kPer<T>; ++e) x[e] *= factor;
        if (c < (int)p.left) store_vec(out + c, (int)p.left - c, pack<T>(x));
    }
}

__device__ inline double block_sum(double x, double *room) {
    x = wave_sum(x);
    if (threadIdx.x % kWave == 0) room[threadIdx.x / kWave] = x;
    __syncthreads();
    x = 0.0;
#pragma unroll
    for (int w = 0; w < kClipThreads / kWave; ++w) x += room[w];
    return x;
}

// The norm is the square root of the sum of all squares, in 64 bits, in which no square of a 32-bit number overflows or vanishes.  Chunks of all gradients
// go to the workgroups in turn.  Both passes are bound by memory (1.2 G elements in bf16: 416 us, 5.8 TB/s, and 939 us, 5.1 TB/s; a ResNet-50's 161
// gradients in f32: 16 us and 32).
__global__ __launch_bounds__(kClipThreads) void square_sum_kernel(const ClipTable a, double *const sums) {
    __shared__ double room[kClipThreads / kWave];
    double sum = 0.0;
    for (uint32_t chunk = blockIdx.x; chunk < a.chunks; chunk += gridDim.x) {
        const Piece p = piece_of(a, chunk);
        raw16 v[kClipVecs];
        load_chunk(p, v);
        sum += p.dtype == BT_F32 ? sum_chunk<float>(v) : p.dtype == BT_F16 ? sum_chunk<f16>(v) : sum_chunk<bf16>(v);
    }
    sum = block_sum(sum, room);
    if (threadIdx.x == 0) sums[blockIdx.x] = sum;
}

// The sum of `count` partial sums, the same in every workgroup that asks.
__device__ inline double total_of(const double *sums, const uint32_t count, double *room) {
    double x = 0.0;
    for (uint32_t i = threadIdx.x; i < count; i += kClipThreads) x += sums[i];
    return block_sum(x, room);
}

// Partial sums of many launches to one, and the norm itself.
__global__ __launch_bounds__(kClipThreads) void total_kernel(const double *sums, const uint32_t count, double *total, float *norm) {
    __shared__ double room[kClipThreads / kWave];
    const double x = total_of(sums, count, room);
    if (threadIdx.x == 0) {
        *total = x;
        *norm = (float)sqrt(x);
    }
}

// (norm: NULL where another launch writes it.)
__global__ __launch_bounds__(kClipThreads) void scale_kernel(const ClipTable a, const double *sums, const uint32_t count, const double max_norm,
                                                             const double eps, float *norm) {
    __shared__ double room[kClipThreads / kWave];
    // From the last chunk to the first: the last ones read are those that the caches still hold.  The first one comes while the sums do.
    uint32_t i = blockIdx.x;
    Piece p = piece_of(a, a.chunks - 1 - i);
    raw16 v[kClipVecs];
    load_chunk(p, v);
    const double x = sqrt(total_of(sums, count, room));
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)x;
    double ratio = max_norm / (x + eps);
    if (ratio > 1.0 || max_norm == INFINITY || x + eps == 0.0) ratio = 1.0;      // (a NaN stays one, but for infinity / infinity and 0 / 0: nothing is clipped)
    const float factor = (float)ratio;
    for (;;) {
        if (factor != 1.0f || p.in != p.out) {      // (else it is there)
            if (p.dtype == BT_F32) scale_chunk<float>(p, v, factor);
            else if (p.dtype == BT_F16) scale_chunk<f16>(p, v, factor);
            else scale_chunk<bf16>(p, v, factor);
        }
        i += gridDim.x;
        if (i >= a.chunks) break;
        p = piece_of(a, a.chunks - 1 - i);
        load_chunk(p, v);
    }
}

// ---- host ------------------------------------------------------------------------------------------------------

// (Few rows leave most compute units idle: what counts is how soon one row is through, and more threads are through sooner.)
constexpr uint64_t kFewRows = 256;

template <class T, class Go> bt_status with_forward_shape(const uint64_t rows, const uint64_t vectors, Go go) {
    if (rows <= kFewRows && vectors > 256 && vectors <= 512) return go(norm_forward_kernel<T, 512, 1>, 512);
    if (rows <= kFewRows && vectors > 512 && vectors <= 1024) return go(norm_forward_kernel<T, 1024, 1>, 1024);
    if (vectors <= 64) return go(norm_forward_kernel<T, 64, 1>, 64);
    if (vectors <= 128) return go(norm_forward_kernel<T, 64, 2>, 64);
    if (vectors <= 256) return go(norm_forward_kernel<T, 256, 1>, 256);
    if (vectors <= 512) return go(norm_forward_kernel<T, 256, 2>, 256);
    if (vectors <= 1024) return go(norm_forward_kernel<T, 256, 4>, 256);
    if (vectors <= 2048) return go(norm_forward_kernel<T, 1024, 2>, 1024);
    if constexpr (sizeof(T) == 4) return go(norm_forward_kernel<T, 1024, 4>, 1024);
    else return BT_ERR_SIZE;
}

// Threads that share a row in the backward pass.
int backward_threads(const uint64_t vectors) {
    int nt = 64;
    while (nt < 1024 && (uint64_t)nt < vectors) nt *= 2;
    return nt;
}

// As many runs as the card holds workgroups, but of some rows each, up to four, where a run for each row would have its partial sums written and read for
// little else; and no fewer than there are compute units.  Two sums of each column go to memory for each run: their time grows with rows * cols / (rows a
// run), that of a run with its rows, so the rows that are best grow with the root of rows * cols.  (us, bf16, a run a row or as below: [1024, 2048] 31.0 and
// 19.8, [2048, 2048] 35.2 and 28.5, [4096, 1024] 36.0 and 29.2; with four rows each throughout [1000, 300] 15.4 and 19.7, [64, 8192] 22.0 and 30.7.)
uint32_t norm_runs(const uint64_t rows, const uint64_t cols, const int width) {
    constexpr uint64_t kUnits = 256;
    const int nt = backward_threads((cols * width + kVec - 1) / kVec);
    const uint64_t most = kUnits * (nt <= 128 ? 8 : 1024 / nt), cells = rows * cols;
    const uint64_t a_run = cells < 360000 ? 1 : cells < 1000000 ? 2 : cells < 1960000 ? 3 : 4;
    uint64_t runs = (rows + a_run - 1) / a_run;
    if (runs < kUnits) runs = rows < kUnits ? rows : kUnits;
    return (uint32_t)(runs < most ? runs : most);
}

template <class T, class Go> bt_status with_backward_shape(const uint64_t vectors, Go go) {
    if (vectors <= 64) return go(norm_backward_kernel<T, 64, 1>, 64);
    if (vectors <= 128) return go(norm_backward_kernel<T, 128, 1>, 128);
    if (vectors <= 256) return go(norm_backward_kernel<T, 256, 1>, 256);
    if (vectors <= 512) return go(norm_backward_kernel<T, 512, 1>, 512);
    if (vectors <= 1024) return go(norm_backward_kernel<T, 1024, 1>, 1024);
    if (vectors <= 2048) return go(norm_backward_kernel<T, 1024, 2>, 1024);
    if constexpr (sizeof(T) == 4) return go(norm_backward_kernel<T, 1024, 4>, 1024);
    else return BT_ERR_SIZE;
}

bool is_finite(const double x) { return x - x == 0.0; }

bt_status check_rows(const uint64_t rows, const uint64_t cols, const bt_dtype dtype) {
    if (width_of(dtype) == 0) return BT_ERR_DTYPE;
    return rows > BT_MAX_ROWS || cols > BT_MAX_NORM_COLS ? BT_ERR_SIZE : BT_OK;
}

template <class... P> bool any_misaligned(const size_t a, const P *...p) { return (misaligned(p, a) || ...); }

struct ClipPlan {
    ClipTable table;

    // Items from *next on that fit a launch; false: there are none left with elements.
    bool fill(const bt_clip_item *items, const size_t count, size_t *next) {
        int used = 0;
        uint64_t at = 0;
        while (*next < count && used < kTable) {
            const bt_clip_item &it = items[*next];
            const uint64_t chunks = (it.n * (uint64_t)width_of(it.dtype) + kChunk - 1) / kChunk;
            if (at + chunks > 0x7fffffffu) break;
            ++*next;
            if (it.n == 0) continue;
            table.in[used] = it.d_in;
            table.out[used] = it.d_out;
            const uint32_t per = kChunk / width_of(it.dtype);
            table.start[used] = (uint32_t)at;
            table.last[used] = (uint32_t)((it.n - 1) % per + 1) | (uint32_t)it.dtype << 30;
            at += chunks;
            ++used;
        }
        table.chunks = (uint32_t)at;
        for (int i = used; i < kTable; ++i) table.start[i] = 0xffffffffu;
        return used > 0;
    }
};

size_t clip_launches(const size_t count) { return count / (kTable / 2) + 1; }      // (the chunks of the largest tensors may cut one short)

bt_status check_clip(const bt_clip_item *items, const size_t count, const bool outs, const float *d_norm, const void *ws, const size_t bytes) {
    if (d_norm == nullptr || ws == nullptr || (items == nullptr && count != 0)) return BT_ERR_NULL;
    for (size_t i = 0; i < count; ++i) {
        const bt_clip_item &it = items[i];
        const int w = width_of(it.dtype);
        if (w == 0) return BT_ERR_DTYPE;
        if (it.n > BT_MAX_ELEMENTS) return BT_ERR_SIZE;
        if (it.n == 0) continue;
        if (it.d_in == nullptr || (outs && it.d_out == nullptr)) return BT_ERR_NULL;
        if (misaligned(it.d_in, w) || (outs && misaligned(it.d_out, w))) return BT_ERR_ALIGN;
    }
    if (misaligned(d_norm, 4) || misaligned(ws, 128)) return BT_ERR_ALIGN;
    return bytes < bt_clip_workspace_bytes(count) ? BT_ERR_WORKSPACE : BT_OK;
}

bt_status sum_squares(ClipPlan &plan, const bt_clip_item *items, const size_t count, double *sums, uint32_t *partials, uint32_t *launches, hipStream_t hs) {
    *partials = *launches = 0;
    for (size_t next = 0; plan.fill(items, count, &next);) {
        const uint32_t grid = plan.table.chunks < kSums ? plan.table.chunks : kSums;
        const bt_status st = launch(square_sum_kernel, dim3(grid), kClipThreads, hs, plan.table, sums + *partials);
        if (st != BT_OK) return st;
        *partials += grid;
        ++*launches;
    }
    return BT_OK;
}

}  // namespace
}  // namespace btb

using namespace btb;

extern "C" {

bt_status bt_residual_norm_forward(const void *d_x, const void *d_block, const void *d_post_weight, const void *d_gate,
                                   const void *d_pre_weight, uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype,
                                   double eps, double scale, double residual_scale,
                                   void *d_out, void *d_y, float *d_stats, bt_stream stream) {
    bt_status st = check_rows(rows, cols, dtype);
    if (st != BT_OK) return st;
    if (!(eps >= 0.0) || !is_finite(eps) || !is_finite(scale) || !is_finite(residual_scale)) return BT_ERR_ARGUMENT;
    if (rows == 0 || cols == 0) return BT_OK;
    if ((d_block == nullptr && (d_out || d_post_weight || d_gate)) || (d_pre_weight == nullptr) != (d_y == nullptr)) return BT_ERR_ARGUMENT;
    if (d_gate && (gate_rows == 0 || rows % gate_rows != 0)) return BT_ERR_ARGUMENT;
    if (d_x == nullptr || (d_block && d_out == nullptr)) return BT_ERR_NULL;
    if (any_misaligned((size_t)width_of(dtype), d_x, d_block, d_post_weight, d_gate, d_pre_weight, d_out, d_y) || misaligned(d_stats, 4)) return BT_ERR_ALIGN;
    NormForward a = {d_x, d_block, d_post_weight, d_gate, d_pre_weight, d_out, d_y, d_stats, (uint32_t)rows, (uint32_t)cols,
                           (uint32_t)(d_gate ? rows / gate_rows : 1), 0, (float)eps, (float)scale, (float)residual_scale};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        return with_forward_shape<T>(rows, (cols + kPer<T> - 1) / kPer<T>, [&](auto kernel, const int nt) {
            // (A grid holds less than 2^32 threads.)
            const uint64_t a_block = nt < 256 ? 256 / nt : 1, most = (uint64_t)1 << 21;
            bt_status s = BT_OK;
            for (uint64_t first = 0; first < rows && s == BT_OK; first += most * a_block) {
                const uint64_t blocks = (rows - first + a_block - 1) / a_block;
                a.first_row = (uint32_t)first;
                s = launch(kernel, dim3((unsigned)(blocks < most ? blocks : most)), nt < 256 ? 256 : nt, (hipStream_t)stream, a);
            }
            return s;
        });
    });
}

size_t bt_residual_norm_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype) {
    if (check_rows(rows, cols, dtype) != BT_OK || rows == 0 || cols == 0) return 0;
    const uint64_t runs = norm_runs(rows, cols, width_of(dtype));
    return (size_t)(4 * cols * runs * (gate_rows != 0 && gate_rows < rows ? 4 : 2));
}

bt_status bt_residual_norm_backward(const void *d_grad_out, const void *d_grad_y, const void *d_out, const void *d_block,
                                    const void *d_post_weight, const void *d_gate, const void *d_pre_weight, const float *d_stats,
                                    uint64_t rows, uint64_t cols, uint64_t gate_rows, bt_dtype dtype, double scale, double residual_scale,
                                    void *d_grad_x, void *d_grad_block, void *d_grad_post_weight, void *d_grad_gate, void *d_grad_pre_weight,
                                    void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check_rows(rows, cols, dtype);
    if (st != BT_OK) return st;
    if (!is_finite(scale) || !is_finite(residual_scale)) return BT_ERR_ARGUMENT;
    if (cols == 0) return BT_OK;
    const size_t w = (size_t)width_of(dtype);
    if (any_misaligned(w, d_grad_out, d_grad_y, d_out, d_block, d_post_weight, d_gate, d_pre_weight) ||
        any_misaligned(w, d_grad_x, d_grad_block, d_grad_post_weight, d_grad_gate, d_grad_pre_weight) || misaligned(d_stats, 4) ||
        misaligned(d_workspace, 128))
        return BT_ERR_ALIGN;
    if (rows == 0)      // sums of nothing
        return with_type(dtype, [&](auto type) {
            using T = decltype(type);
            bt_status s = d_grad_post_weight ? zeros<T>(d_grad_post_weight, cols, (hipStream_t)stream) : BT_OK;
            if (s == BT_OK && d_grad_pre_weight) s = zeros<T>(d_grad_pre_weight, cols, (hipStream_t)stream);
            if (s == BT_OK && d_grad_gate) s = zeros<T>(d_grad_gate, gate_rows * cols, (hipStream_t)stream);
            return s;
        });
    if ((d_block == nullptr && (d_post_weight || d_gate || d_grad_block)) || (d_grad_y == nullptr) != (d_pre_weight == nullptr) ||
        (d_grad_pre_weight && !d_pre_weight) || (d_grad_post_weight && !d_post_weight) || (d_grad_gate && !d_gate))
        return BT_ERR_ARGUMENT;
    if (d_gate && (gate_rows == 0 || rows % gate_rows != 0)) return BT_ERR_ARGUMENT;
    if ((d_grad_y && d_out == nullptr) || ((d_grad_y || d_block) && d_stats == nullptr)) return BT_ERR_NULL;
    const bool sums = d_grad_post_weight || d_grad_pre_weight || d_grad_gate;
    if (sums && d_workspace == nullptr) return BT_ERR_NULL;
    if (sums && workspace_bytes < bt_residual_norm_workspace_bytes(rows, cols, d_gate ? gate_rows : 0, dtype)) return BT_ERR_WORKSPACE;
    const uint32_t runs = norm_runs(rows, cols, width_of(dtype));
    float *const ws = (float *)d_workspace;
    const bool parts = d_gate && gate_rows < rows;
    NormBackward a = {d_grad_out, d_grad_y, d_out, d_block, d_post_weight, d_gate, d_pre_weight, d_stats,
                      d_grad_x, d_grad_block, d_grad_post_weight, d_grad_gate, d_grad_pre_weight,
                      ws, ws + (uint64_t)runs * cols, ws + 2 * (uint64_t)runs * cols,
                      (uint32_t)rows, (uint32_t)cols, (uint32_t)(d_gate ? rows / gate_rows : 1), (uint32_t)(d_gate ? gate_rows : 0), runs,
                      (float)scale, (float)residual_scale};
    return with_type(dtype, [&](auto type) {
        using T = decltype(type);
        const bt_status s = with_backward_shape<T>((cols + kPer<T> - 1) / kPer<T>, [&](auto kernel, const int nt) { return launch(kernel, dim3(runs), nt, (hipStream_t)stream, a); });
        if (s != BT_OK || !(d_grad_post_weight || d_grad_pre_weight || (parts && d_grad_gate))) return s;
        return launch(norm_join_kernel<T>, dim3((unsigned)((cols + kJoinCols - 1) / kJoinCols), 2 + (unsigned)(!parts || !d_grad_gate ? 0 : gate_rows <= runs ? gate_rows : runs - 1)), kJoinCols * kJoinTeams,
                      (hipStream_t)stream, a);
    });
}

size_t bt_clip_workspace_bytes(size_t count) { return 128 + clip_launches(count) * kSums * sizeof(double); }

bt_status bt_grad_norm(const bt_clip_item *items, size_t count, float *d_norm, void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    bt_status st = check_clip(items, count, false, d_norm, d_workspace, workspace_bytes);
    if (st != BT_OK) return st;
    ClipPlan plan;
    double *const total = (double *)d_workspace, *const sums = total + 16;
    uint32_t partials, launches;
    st = sum_squares(plan, items, count, sums, &partials, &launches, (hipStream_t)stream);
    return st != BT_OK ? st : launch(total_kernel, dim3(1), kClipThreads, (hipStream_t)stream, (const double *)sums, partials, total, d_norm);
}

bt_status bt_clip_grads(const bt_clip_item *items, size_t count, double max_norm, double eps, float *d_norm,
                        void *d_workspace, size_t workspace_bytes, bt_stream stream) {
    if (!(max_norm >= 0.0) || !(eps >= 0.0)) return BT_ERR_ARGUMENT;
    bt_status st = check_clip(items, count, true, d_norm, d_workspace, workspace_bytes);
    if (st != BT_OK) return st;
    ClipPlan plan;
    double *const total = (double *)d_workspace, *sums = total + 16;
    uint32_t partials, launches;
    st = sum_squares(plan, items, count, sums, &partials, &launches, (hipStream_t)stream);
    if (st != BT_OK) return st;
    float *norm = d_norm;
    if (launches != 1) {
        st = launch(total_kernel, dim3(1), kClipThreads, (hipStream_t)stream, (const double *)sums, partials, total, d_norm);
        if (st != BT_OK) return st;
        sums = total;
        partials = 1;
        norm = nullptr;
    }
    for (size_t next = 0; plan.fill(items, count, &next);) {
        const uint32_t grid = plan.table.chunks < kScalers ? plan.table.chunks : kScalers;
        st = launch(scale_kernel, dim3(grid), kClipThreads, (hipStream_t)stream, plan.table, (const double *)sums, partials, max_norm, eps, norm);
        if (st != BT_OK) return st;
    }
    return BT_OK;
}

}  // extern "C"
