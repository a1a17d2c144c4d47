// fp32 attention of packed prompts and of drafted tokens (see reform_prompt_attend and reform_tree_attend in
// reform.h), on v_mfma_f32_16x16x4f32: fp32 operands, products and sums.
//
// Blocks of rows as attend_seq_f32.h takes them.
//
// Bound: the fp32 matrix pipe (0.15 PFLOP/s, of which it reaches 0.35 to 0.57: 2048 rows, 32/8 heads of 128, 495 us; 4096, 32/8 of 64, 776; 8 x 1000, 32/8 of 128, 1232) and,
// at the sizes of checks, latency (three prompts of up to 301 rows, 4 heads of 64: 11 us).  32 rows to a workgroup, so that K and V are read half
// as often: the same time for large batches, twice as long for small ones (60 batches, 1.27).
#include "attend_seq_f32.h"
#include "prompt_share.h"

namespace reform {

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void prompt_attend_f32(PromptParams p)
{
    __shared__ F32Sums<DP> sh;
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<kF32Rows, kF32Keys>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<float>(p, blk, kvh, blk.rb * kF32Rows, r, k);
    f32_segment<DP, false>(r, k, p.D, p.scale, 0, blk.tiles, nullptr, nullptr, sh);
}

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void prompt_attend_f32_shared(PromptParams p)
{
    __shared__ F32Sums<DP> sh;
    prompt_walk<float, kF32Rows, kF32Keys>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        f32_segment<DP, false>(r, k, p.D, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * DP,
                               slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, sh);
    });
}

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void tree_attend_f32(TreeParams p)
{
    __shared__ F32Sums<DP> sh;
    tree_walk<float, kF32Rows, kF32Keys>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        f32_segment<DP, true>(r, k, p.D, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * DP,
                              slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, sh);
    });
}

namespace {

template <int DP>
hipError_t launch_prompt(const PromptParams &p, hipStream_t st)
{
    if (p.shares) {
        hipLaunchKernelGGL((prompt_attend_f32_shared<DP>), dim3(p.shares), dim3(kF32Waves * 64), 0, st, p);
        prompt_merge_launch<DP, kF32Rows, kF32Keys, false>(p, st);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((prompt_attend_f32<DP>), dim3(prompt_grid(p, kF32Rows)), dim3(kF32Waves * 64), 0, st, p);
    return hipGetLastError();
}

template <int DP>
hipError_t launch_tree(const TreeParams &p, hipStream_t st)
{
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    hipLaunchKernelGGL((tree_attend_f32<DP>), dim3(grid), dim3(kF32Waves * 64), 0, st, p);
    if (p.shares) tree_merge_launch<DP, kF32Rows, kF32Keys, false>(p, st);
    return hipGetLastError();
}

}  // namespace

// A step is eight tiles of 16 keys by the waves of a workgroup, some 0.03 us for each element of a row (3.7 us at 128, 1.9 at 64), whether the chip
// is full or not.  What sharing out saves is the longest block's chain, for some 8 us; but where a sequence's blocks are then at different keys, each
// brings them from memory (ten rows, 12/4 heads of 96 behind 16000 keys 430 -> 48 us; 282 rows, 12/4 of 256 behind 4 x 3000 221 -> 396).
// 80 batches of 1 to 50 sequences behind up to 16000 keys each: 0.62 of the time without sharing, at worst 1.26 (three rows behind 200, 8/4 of 256).
void prompt_plan_f32(PromptParams &p)
{
    const double step = 0.03 * (p.D <= 32 ? 32 : p.D <= 64 ? 64 : p.D <= 128 ? 128 : 256), keys = (double)p.n_k / p.n_seq;
    const double blocks = ((double)p.n_q * p.G / kF32Rows + p.n_seq) * p.Hkv, full = blocks * (keys / 128.0 + 1.0) * step / p.units;
    const double alone = keys / 128.0 * step, memory = blocks * keys * p.D * 8.0 / 3.5e6;
    if (alone < 8.0 || p.n_seq > 64 || blocks * ((double)p.n_k / kF32Keys + 16.0) >= 33554432.0) return;          // as in prompt_share_rows
    if (std::cbrt(full * full * full + alone * alone * alone) < 8.0 + (full > memory ? full : memory)) return;
    const int rows = p.n_q * p.G;
    p.block = kF32Rows;
    p.part_rows = rows < kF32Rows ? rows : kF32Rows;
    p.least = kF32Waves;
    p.shares = 2 * p.units > kTreeMaxShares ? kTreeMaxShares : 2 * p.units;
}

hipError_t prompt_attend_f32_launch(const PromptParams &p, hipStream_t st)
{
    if (p.D <= 32) return launch_prompt<32>(p, st);
    if (p.D <= 64) return launch_prompt<64>(p, st);
    if (p.D <= 128) return launch_prompt<128>(p, st);
    return launch_prompt<256>(p, st);
}

// Elements of a row of the pieces: heads are padded to the next form.
size_t tree_part_dim(bool bf16, int D) { return bf16 ? D : D <= 32 ? 32 : D <= 64 ? 64 : D <= 128 ? 128 : 256; }

// Fitted as in tree.hip, to 90 batches of 1 to 40 rows over 300 to 3000 keys in heads of 32 to 256: shares of a tile for each wave and more take
// 0.87 of the time that two tiles for each take, whole items of up to 1024 keys up to 4.8 times as much where heads are wide.  70 other batches of 1 to 64
// rows: 0.61 of all whole, at worst 1.21 times (37 rows of 8 x 4 caches of up to 432 keys, 128 wide, 21.7 us whole, 26.2).
void tree_plan_f32(TreeParams &p, int compute_units)
{
    const int whole = p.D <= 32 ? 1200 : p.D <= 64 ? 850 : p.D <= 128 ? 350 : 200;
    tree_plan(p, kF32Rows, kF32Keys, whole, kF32Waves, compute_units, 2 * compute_units);
}

hipError_t tree_attend_f32_launch(const TreeParams &p, hipStream_t st)
{
    if (p.D <= 32) return launch_tree<32>(p, st);
    if (p.D <= 64) return launch_tree<64>(p, st);
    if (p.D <= 128) return launch_tree<128>(p, st);
    return launch_tree<256>(p, st);
}

}  // namespace reform
