// a3 for a handful of tokens, bf16 operands: where a launch comes here (the kernel is in moe_ffn_thin.h).
#include <algorithm>
#include <cmath>

#include "moe_ffn_thin.h"

namespace moe {
// experts with rows, on average over routings that favour none, and the standard deviation
static double experts_with_rows(const moe_shape& s, double* deviation = nullptr) {
    const double E = s.E, none = std::pow(1.0 - s.k / E, s.T);                      // an expert, two experts without a row
    const double neither = s.E > 1 ? std::pow((E - s.k) * (E - s.k - 1.0) / (E * (E - 1.0)), s.T) : none;
    if (deviation) *deviation = std::sqrt(std::max(0.0, E * none * (1.0 - none) + E * (E - 1.0) * (neither - none * none)));
    return E * (1.0 - none);
}

// Where the launches of at most 16 tokens come here, by the blocks that moe_ffn_rows.h would keep busy.
// Gate/up: up to about one and a half blocks of 64 features per compute unit.  us, that kernel / this one: 1024 x 2816 (8 experts, 2
// per token) 1 token (88 blocks) 13 / 11, 16 tokens (348) 25 / 22; 2048 x 4096 1 token (128) 22 / 18, 4 tokens (350) 34 / 31, 16 tokens (506)
// 47 / 46; 64 experts of 2048 x 1024, 8 per token, 3 tokens (337) 40 / 36, 8 tokens (671) 61 / 63; Mixtral-8x7B shape 1 token (448) 76 / 79.
bool thin_takes_gate_up(const moe_shape& s) { return s.T <= 16 && experts_with_rows(s) * (s.F / 64) <= 440; }
// Down: with clearly fewer blocks of 128 columns than compute units, or with between one and one and a half per compute unit, which share
// out unevenly; here 384 blocks' worth of wavefronts, twelve per compute unit, are the most that run at once.  us for both
// launches, by experts with rows (blocks), that kernel / this one:
//   k of 14336 (4096 x 14336) 2 experts (64) 153 / 114, 4 (128) 233 / 214, 6 (192) 326 / 321, 8 (256) 416 / 416, 9 (288) 515 / 468, 12 (384) 625 / 615,
//   13 (416) 668 / 691; 10752 (6144 x 10752) 3 (144) 205 / 199, 4 (192) 254 / 253, 5 (240) 321 / 329, 6 (288) 405 / 374, 9 (432) 522 / 538;
//   8192 (5120 x 8192) 2 (80) 100 / 85, 3 (120) 133 / 126, 5 (200) 196 / 204, 7 (280) 299 / 282, 10 (400) 378 / 416; (3072 x 8192) 6 (144) 150 / 153, 8
//   (192) 186 / 199; 4096 (4096 x 4096) 5 (160) 91 / 89, 6 (192) 96 / 100;
//   2048 (2048 x 2048) 8 (128) 40 / 37, 11 (176) 50 / 50, 15 (240) 64 / 66, (4096 x 2048) 9 (288) 90 / 81, 13 (416) 108 / 109, 15 (480) 119 / 118.
// The routing is not known here.  The lower range goes by the average; the upper one by the average plus the deviation, or all experts, and where
// k is not long by the average less half the deviation (routings that fill one round or less lose as much there as the others gain; with a long
// k they lose little: 6144 x 16384, 8 experts, 4 tokens, 262 blocks on average, layer 522 / 502 over sixteen routings).
bool thin_takes_down(const moe_shape& s, int k) {
    if (s.T > 16) return false;
    const double per_expert = s.H / 128;
    double deviation;
    const double blocks = experts_with_rows(s, &deviation) * per_expert;
    if (k <= 2048) return blocks < 190 || (blocks > 256 && blocks < 500);
    const bool long_k = k > 10240;
    if (blocks < (long_k ? 190 : 130)) return true;
    return blocks - (long_k ? 0.0 : 0.5 * deviation * per_expert) > 256 && std::min(blocks + deviation * per_expert, s.E * per_expert) <= 384;
}

int launch_gate_up_thin_bf16(GemmParams& p, int F, int R, int n_exp, hipStream_t st) { return launch_thin<Bf16, 0, 2>(p, F, R, n_exp, st); }

int launch_down_thin_bf16(GemmParams& p, int H, int R, int n_exp, hipStream_t st) { return launch_thin<Bf16, 1, 1>(p, H, R, n_exp, st); }

}  // namespace moe
