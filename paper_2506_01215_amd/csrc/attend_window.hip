// Attention over packed prompts whose rows see a sliding window and a few first keys (see reform_window_attend in reform.h).
//
// The blocks of rows of attend_prompt.hip, each of which goes through two runs of keys, the first ones and those from
// the first key that its first row's window shows to the last that its last row sees, in tiles cut from both counted through (WindowKeys).  Only tiles at the
// ends of the runs are masked.
//
// The probabilities of P.V are rounded to bf16 once, as the packed prompts' are: outputs are off by 0.0020 to 0.0023 of their norm, where their
// own rounding alone makes 0.0016 to 0.0017.  What the rounding leaves would take a second product, half as much again of what bounds long prompts; the
// matrix pipe of single tokens waits for memory, and they take it.
//
//   window_attend<D,NW,KG>         blocks of 32 NW rows, all waves through the same tiles, KG groups of them (attend_rows.h)
//   window_attend_short<D,NB,NW>   blocks of 16 NB rows whose NW waves divide the tiles (attend_seq.h)
//   window_attend_f32<DP>          blocks of 16 rows, fp32 (attend_seq_f32.h)
#include "attend_rows.h"
#include "attend_seq_f32.h"
#include "prompt_blocks.h"
#include "window_plan.h"

namespace reform {

namespace {

// The block's operands; returns the number of its tiles.
template <class T, int ROWS, int TK>
__device__ __forceinline__ int window_operands(const WindowParams &p, const PromptBlock &blk, int kvh, SeqRows &r, WindowKeys &k)
{
    prompt_block_operands<T>(p, blk, kvh, blk.rb * ROWS, r, k);
    k.window = p.window;
    const int lo = max(k.shift + r.row0 / r.G - p.window + 1, 0);        // first key of the first row's window
    const int last = k.shift + (min(r.row0 + ROWS, r.rows) - 1) / r.G;   // last key that the block sees
    k.skip = max(lo - p.n_sink, 0);
    k.cut = k.skip ? p.n_sink : 0;
    k.stay = max(lo, p.n_sink);
    return last < 0 ? 0 : (last - k.skip) / TK + 1;
}

template <int D, int NW, int KG>
__global__ __launch_bounds__(NW * KG * 64, 2) void window_attend(WindowParams p)
{
    using S = RowsShape<D, NW, KG>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::ROWS, S::BN>(p, blockIdx.x / p.Hkv, p.sorted);
    if (blk.rb < 0) return;
    SeqRows r;
    WindowKeys k;
    const int tiles = window_operands<u16, S::ROWS, S::BN>(p, blk, kvh, r, k);
    rows_segment<D, NW, KG, false>(r, k, p.by_head, p.scale, 0, tiles, nullptr, nullptr, lds);
}

template <int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void window_attend_short(WindowParams p)
{
    using S = SeqShape<D, NB, NW>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<S::R, S::TK>(p, blockIdx.x / p.Hkv, p.sorted);
    if (blk.rb < 0) return;
    SeqRows r;
    WindowKeys k;
    const int tiles = window_operands<u16, S::R, S::TK>(p, blk, kvh, r, k);
    seq_segment<D, NB, NW, false>(r, k, p.scale, 0, tiles, nullptr, nullptr, smem);
}

template <int DP>
__global__ __launch_bounds__(kF32Waves * 64, 2) void window_attend_f32(WindowParams p)
{
    __shared__ F32Sums<DP> sh;
    const int kvh = blockIdx.x % p.Hkv;
    const PromptBlock blk = prompt_block<kF32Rows, kF32Keys>(p, blockIdx.x / p.Hkv, p.sorted);
    if (blk.rb < 0) return;
    SeqRows r;
    WindowKeys k;
    const int tiles = window_operands<float, kF32Rows, kF32Keys>(p, blk, kvh, r, k);
    f32_segment<DP, false>(r, k, p.D, p.scale, 0, tiles, nullptr, nullptr, sh);
}

template <int D, int NW, int KG>
hipError_t launch_long(WindowParams p, hipStream_t st)
{
    using S = RowsShape<D, NW, KG>;
    const hipError_t e = raise_lds<window_attend<D, NW, KG>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    p.by_head = NW % p.G == 0;
    hipLaunchKernelGGL((window_attend<D, NW, KG>), dim3(prompt_grid(p, S::ROWS)), dim3(NW * KG * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D, int NB, int NW>
hipError_t launch_short(const WindowParams &p, hipStream_t st)
{
    using S = SeqShape<D, NB, NW>;
    const hipError_t e = raise_lds<window_attend_short<D, NB, NW>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((window_attend_short<D, NB, NW>), dim3(prompt_grid(p, S::R)), dim3(NW * 64), S::lds_bytes, st, p);
    return hipGetLastError();
}

template <int D>
hipError_t launch_bf16(const WindowParams &p, hipStream_t st)
{
    const PromptForm &f = window_forms(D)[window_choose(D, p.G, p.Hkv, p.n_seq, p.n_q, p.n_k, p.window, p.n_sink, p.units)];
    if (f.rows == 32) return launch_short<D, 2, 4>(p, st);
    if (f.rows == 16) return launch_short<D, 1, 8>(p, st);
    if constexpr (D == 128) {
        if (f.groups == 2) return launch_long<D, 4, 2>(p, st);
    }
    return launch_long<D, 4, 1>(p, st);
}

template <int DP>
hipError_t launch_f32(const WindowParams &p, hipStream_t st)
{
    hipLaunchKernelGGL((window_attend_f32<DP>), dim3(prompt_grid(p, kF32Rows)), dim3(kF32Waves * 64), 0, st, p);
    return hipGetLastError();
}

}  // namespace

hipError_t window_attend_launch(const WindowParams &p, bool bf16, hipStream_t st)
{
    if (bf16) return p.D == 64 ? launch_bf16<64>(p, st) : launch_bf16<128>(p, st);
    if (p.D <= 32) return launch_f32<32>(p, st);
    if (p.D <= 64) return launch_f32<64>(p, st);
    if (p.D <= 128) return launch_f32<128>(p, st);
    return launch_f32<256>(p, st);
}

}  // namespace reform
