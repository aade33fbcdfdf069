// Which kernel and which tiles an expert's product takes, by its sizes: plain C++ of the host.
#ifndef BT_EXPERT_RULES_H
#define BT_EXPERT_RULES_H

#include <stdint.h>

namespace btb {
namespace {

// Both gated projections; one product; its way back, and that of both projections (two sums); the weights' gradients.
enum Kind { kPair, kPlain, kBack, kBackPair, kWeights };

constexpr int kStepBytes = 64;      // of the summed index in a step

// Pieces of b that a takes.
inline uint64_t pieces(const uint64_t a, const uint64_t b) { return (a + b - 1) / b; }

// Whether the forward pass reads the weights straight to registers: with long sums few rows an expert, with short ones so few tiles that each has a compute unit (us, bf16, that way and in tiles: one product, 16 experts of
// [1024, 4096], 64 rows 30 and 36, 256 rows 37 and 37; 64 experts of [2048, 768], 64 rows 50 and 33; both projections, 8 experts of [11008, 4096], 16 rows 209 and 229, 32 rows 241 and 241).
inline bool few_rows(const bool pair, const uint64_t rows, const uint64_t experts, const uint64_t n, const uint64_t k, const int width) {
    if (k * width >= 8192) return rows <= experts * (pair ? 2 : 8);
    return rows <= experts * 8 && (rows < experts ? rows : experts) * pieces(n, pair ? 32 : 64) <= 256;
}

enum Size { kSmall, kMiddle, kLarge };

// Tiles of which size, by the model of the time that gated.hip's plan_of has: an expert's last tile is half empty as a rule.
inline Size size_of(const Kind kind, const uint64_t rows, const uint64_t experts, const uint64_t m, const uint64_t n, const uint64_t k, const uint64_t parts, const int width) {
    struct Form {
        Size size;
        int side, together;      // rows and columns of a tile, workgroups that a compute unit holds
        double rate, alone;
    };
    static const Form forms[] = {{kSmall, 64, 4, 0.33, 0.28}, {kMiddle, 128, 2, 0.6, 0.38}, {kLarge, 256, 1, 0.95, 0.75}};
    if (width == 4) return kSmall;
    const double steps = (double)((kind == kWeights ? rows / experts : k) * width) / kStepBytes * (kind == kBackPair ? 2 : 1);
    Size best = kSmall;
    double least = 1e300;
    for (const Form &f : forms) {
        const uint64_t tiles_m = kind == kWeights ? pieces(m, f.side) * experts * parts : rows / f.side + (rows / experts < (uint64_t)f.side / 2 ? experts : experts / 2);
        const uint64_t tiles = (tiles_m > 0 ? tiles_m : 1) * pieces(n, kind == kPair ? f.side / 2 : f.side), a_unit = pieces(tiles, 256);
        double time = (double)a_unit * 2.0 * f.side * f.side * (kStepBytes / width) * steps / (5.9e6 * f.rate);
        const double alone = steps * f.alone * (double)pieces(a_unit, f.together);
        if (time < alone) time = alone;
        if (time < least) {
            least = time;
            best = f.size;
        }
    }
    return best;
}

// Into how many parts the last tiles may go (a power of two), and the bytes that the parts' sums take: none where the time of a tile that parts would save, by the steps' time that size_of's model has and the number of
// tiles that experts with the same number of rows would have, is not well above that of the join, 5 to 15 us (bf16 [32768, 4096] x 8 weights of [4096, 2048] twice, grad_x: 1183 -> 1080 us; with parts
// everywhere bf16 [65536, 1024] x 32 weights of [2048, 1024] 333 -> 342).
struct Parts {
    uint32_t most;
    uint64_t bytes;
};
inline Parts parts_of(const Kind kind, const Size size, const uint64_t rows, const uint64_t experts, const uint64_t m, const uint64_t n, const uint64_t k, const uint64_t outputs, const int width) {
    const uint64_t side = size == kLarge ? 256 : size == kMiddle ? 128 : 64, slots = size == kLarge ? 256 : size == kMiddle ? 512 : 1024;
    const uint64_t steps = pieces((kind == kWeights ? rows / experts : k) * width, kStepBytes) * (kind == kBackPair ? 2 : 1);
    const uint64_t tiles_m = kind == kWeights ? pieces(m, side) * experts * outputs : rows / side + experts / 2 + 1, tiles = tiles_m * pieces(n, kind == kPair ? side / 2 : side);
    Parts p = {1, 0};
    const double step = size == kLarge ? 0.75 : size == kMiddle ? 0.38 : 0.28;      // us
    const uint64_t rest = tiles % slots;
    uint64_t splits = 1;
    while (splits < 16 && rest * splits * 2 <= slots && steps / (splits * 2) >= 16) splits *= 2;
    if ((double)steps * step * (1.0 - 1.0 / (double)splits) < 20.0) return p;
    while (p.most < 16 && steps / (p.most * 2) >= 16) p.most *= 2;
    p.bytes = slots * side * side * 4;
    return p;
}

}  // namespace
}  // namespace btb
#endif  // BT_EXPERT_RULES_H
