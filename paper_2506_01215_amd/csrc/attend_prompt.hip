// Causal attention over packed prompts, bf16 (see reform_prompt_attend in reform.h).
//
//   prompt_attend<D,NW,KG>   a workgroup takes a block of 32 NW rows of one KV head (counted over query rows and the heads
//                            of the group) over all keys that the block sees; KG groups of its waves divide the key tiles
//   prompt_attend_short<D,NB,NW>   blocks of 16 NB rows whose NW waves divide the keys (attend_seq.h)
//
//   prompt_attend_shared<D,NB,NW>, prompt_attend_rows_shared<D,NW,KG>   blocks of 16 NB and of 32 NW rows, their keys shared out over the chip: few
//                            rows behind many keys (prompt_share.h)
//
// Large blocks read K and V less often, small ones and divided keys fill the chip with few rows and make the longest
// block's chain of tiles shorter; prompt_plan.h says which when.
//
// Bound: the matrix pipe, and the power it draws (attend_bf16.hip): one prompt of 16384, 32/8 heads of 128, 1.8 ms, 1.2 PFLOP/s; ten of
// together 16384 425 us, 0.97 PFLOP/s, of which some 8 us a block are its beginning and end, half hidden by the other workgroup on its compute
// unit; small batches: the longest block's chain, and latency.  A grid that stays and takes block after block: ten prompts 421 -> 456 us, since the
// blocks of a compute unit's two workgroups are then dealt before it is known which is done first.
#include "attend_rows.h"
#include "prompt_blocks.h"
#include "prompt_plan.h"
#include "prompt_share.h"

namespace reform {

template <int D, int NW, int KG>
__global__ __launch_bounds__(NW * KG * 64, 2) void prompt_attend(PromptParams p)
{
    using S = RowsShape<D, NW, KG>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::ROWS, S::BN>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<u16>(p, blk, kvh, blk.rb * S::ROWS, r, k);
    rows_segment<D, NW, KG, false>(r, k, p.by_head, p.scale, 0, blk.tiles, nullptr, nullptr, lds);
}

template <int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attend_short(PromptParams p)
{
    using S = SeqShape<D, NB, NW>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::R, S::TK>(p, blockIdx.x / p.Hkv);
    if (blk.rb < 0) return;
    SeqRows r;
    SeqKeys k;
    prompt_block_operands<u16>(p, blk, kvh, blk.rb * S::R, r, k);
    seq_segment<D, NB, NW, false>(r, k, p.scale, 0, blk.tiles, nullptr, nullptr, smem);
}

template <int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void prompt_attend_shared(PromptParams p)
{
    using S = SeqShape<D, NB, NW>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    prompt_walk<u16, S::R, S::TK>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        seq_segment<D, NB, NW, false>(r, k, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                      slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, smem);
    });
}

template <int D, int NW, int KG>
__global__ __launch_bounds__(NW * KG * 64, 2) void prompt_attend_rows_shared(PromptParams p)
{
    using S = RowsShape<D, NW, KG>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    prompt_walk<u16, S::ROWS, S::BN>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        rows_segment<D, NW, KG, false>(r, k, false, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                       slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, lds);
    });
}

namespace {

template <int D, int NW, int KG>
hipError_t launch_long(PromptParams p, hipStream_t st)
{
    using S = RowsShape<D, NW, KG>;
    const hipError_t e = raise_lds<prompt_attend<D, NW, KG>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    p.by_head = NW % p.G == 0;
    hipLaunchKernelGGL((prompt_attend<D, NW, KG>), dim3(prompt_grid(p, S::ROWS)), dim3(NW * KG * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D, int NB, int NW>
hipError_t launch_short(const PromptParams &p, hipStream_t st)
{
    using S = SeqShape<D, NB, NW>;
    const hipError_t e = raise_lds<prompt_attend_short<D, NB, NW>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_attend_short<D, NB, NW>), dim3(prompt_grid(p, S::R)), dim3(NW * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D, int NB, int NW>
hipError_t launch_shared(const PromptParams &p, hipStream_t st)
{
    using S = SeqShape<D, NB, NW>;
    const hipError_t e = raise_lds<prompt_attend_shared<D, NB, NW>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_attend_shared<D, NB, NW>), dim3(p.shares), dim3(NW * 64), S::lds_bytes, st, p);
    prompt_merge_launch<D, S::R, S::TK, true>(p, st);
    return hipGetLastError();
}

template <int D, int NW, int KG>
hipError_t launch_rows_shared(const PromptParams &p, hipStream_t st)
{
    using S = RowsShape<D, NW, KG>;
    const hipError_t e = raise_lds<prompt_attend_rows_shared<D, NW, KG>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_attend_rows_shared<D, NW, KG>), dim3(p.shares), dim3(NW * KG * 64), S::lds_bytes, st, p);
    prompt_merge_launch<D, S::ROWS, S::BN, true>(p, st);
    return hipGetLastError();
}

template <int D>
hipError_t launch(const PromptParams &p, hipStream_t st)
{
    if (p.shares) {
        constexpr int NW = D == 64 ? 4 : 8;
        if (p.block == 64) return launch_rows_shared<D, 2, 2>(p, st);
        if (p.block == 128) return launch_rows_shared<D, 4, 1>(p, st);
        return p.block == 16 ? launch_shared<D, 1, NW>(p, st) : launch_shared<D, 2, NW>(p, st);
    }
    const PromptForm &f = prompt_forms(D)[prompt_choose(D, p.G, p.Hkv, p.n_seq, p.n_q, p.n_k, p.units)];
    if (f.rows == 32) return launch_short<D, 2, 4>(p, st);
    if (f.rows == 16) return launch_short<D, 1, 8>(p, st);
    if constexpr (D == 64) {
        if (f.rows == 256) return launch_long<D, 8, 1>(p, st);
    } else {
        if (f.groups == 2) return launch_long<D, 4, 2>(p, st);
    }
    return launch_long<D, 4, 1>(p, st);
}

}  // namespace

void prompt_plan_bf16(PromptParams &p)
{
    PromptShared f;
    p.block = prompt_share_rows(p.D, p.G, p.Hkv, p.n_seq, p.n_q, p.n_k, p.units, f);
    if (!p.block) return;
    const int rows = p.n_q * p.G;
    p.part_rows = rows < p.block ? rows : p.block;
    p.least = f.least / f.form.keys;
    p.shares = f.workgroups * p.units;
    if (p.shares > kTreeMaxShares) p.shares = kTreeMaxShares;
}

hipError_t prompt_attend_bf16(const PromptParams &p, hipStream_t st)
{
    return p.D == 64 ? launch<64>(p, st) : launch<128>(p, st);
}

}  // namespace reform
