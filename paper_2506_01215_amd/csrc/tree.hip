// Drafted tokens over a batch of caches, bf16 (see reform_tree_attend in reform.h): one token per sequence, a
// chain or a tree of up to 64.
//
// Bound: reading K and V once (a row of 256 bytes meets 16 query rows per matrix instruction; 64 nodes of four
// heads are 256 rows, which reach 0.7 of the matrix pipe at the rate K and V arrive).  So the keys are shared
// out over the whole chip (tree_list.h), the rows of a group's heads and nodes are one block of up to 256 rows,
// and the waves of a workgroup divide the keys as far as the rows allow: up to 16 and 32 rows every wave has
// key tiles of its own, beyond that two, four or eight waves share each tile.
#include "attend_seq.h"
#include "tree_list.h"

namespace reform {

template <int D, int NB, int RG>
__global__ __launch_bounds__(kSeqWaves * 64, 2) void tree_attend(TreeParams p)
{
    using S = SeqShape<D, NB, RG>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    tree_walk<u16, S::R, S::TK>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        seq_segment<D, NB, RG, true>(r, k, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                     slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, smem);
    });
}

namespace {

template <int D, int NB, int RG>
hipError_t launch(const TreeParams &p, hipStream_t st)
{
    using S = SeqShape<D, NB, RG>;
    const hipError_t e = raise_lds<tree_attend<D, NB, RG>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    const unsigned grid = p.shares ? p.shares : (unsigned)p.n_seq * p.Hkv * p.row_blocks;
    hipLaunchKernelGGL((tree_attend<D, NB, RG>), dim3(grid), dim3(kSeqWaves * 64), S::lds_bytes, st, p);
    if (p.shares) tree_merge_launch<D, S::R, S::TK, true>(p, st);
    return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const TreeParams &p, hipStream_t st)
{
    const int rows = p.T * p.G;
    if (rows <= 16) return launch<D, 1, 1>(p, st);
    if (rows <= 32) return launch<D, 2, 1>(p, st);
    if (rows <= 64) return launch<D, 2, 2>(p, st);
    if (rows <= 128) return launch<D, 2, 4>(p, st);
    return launch<D, 2, 8>(p, st);
}

}  // namespace

void tree_plan_bf16(TreeParams &p, int compute_units)
{
    const int rows = p.T * p.G;
    const int R = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 128 ? 128 : 256;
    tree_plan(p, R, R == 256 ? 64 : 32, 8, compute_units);
}

hipError_t tree_attend_bf16(const TreeParams &p, hipStream_t st)
{
    return p.D == 64 ? launch_rows<64>(p, st) : launch_rows<128>(p, st);
}

}  // namespace reform
