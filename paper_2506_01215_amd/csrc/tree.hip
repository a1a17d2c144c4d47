// Drafted tokens over a batch of caches, bf16 (see reform_tree_attend in reform.h): one token per sequence, a
// chain or a tree of up to 64.
//
// Bound: reading K and V once, up to some 64 rows (a 16-row block of queries costs a compute unit a sixth of the time that its
// share of the memory bandwidth takes to bring the keys), then the matrix pipe as well.  So the keys are shared out over the
// whole chip (tree_list.h), and where the chip is busy the rows of a group's heads and nodes are one block of up to 256, for which K and V are
// read once; where it is not, smaller blocks (tree_rows).  In blocks of up to 32 rows every wave has key tiles of its own and no
// barrier (attend_seq.h); in larger ones the waves divide the rows and go through the tiles together (attend_rows.h).
// Measured, 32/8 heads of 128: one token for each of 32 sequences over 8192 rows (1.07 GB) 183 us, 5.9 TB/s; 24 nodes 206 us, 64 nodes
// 301 us.  8 waves at head_dim 128, 4 at 64 (two workgroups to a compute unit): 8 nodes, 24/8 of 64, 16 caches of up to 4096 rows
// 37.6 us with 8 waves, 31.6 with 4; one token, 32/8 of 128, 16 caches of up to 8000 rows 49.7 with 8, 50.2 with 4.
// 64 rows: two groups of two waves that divide the tiles, one such workgroup to a compute unit, so that there are half as many pieces to
// put together as with two workgroups of two waves (36 batches of 33 to 64 rows over 200 to 12500 keys, mean: 0.89 of the time; four groups at
// head_dim 64 0.92).  128 rows: two groups take as long as two workgroups (25 batches, 1.00).  192 rows: a wave of 32 and one of 16 to each SIMD (48
// nodes over 16640 rows, 32/8 of 128 32.1 -> 30.1 us against a block of 256; 32 caches of up to 4492 rows, 48 nodes, 32/8 of 64 81 -> 74).
#include "attend_rows.h"
#include "prompt_plan.h"
#include "tree_list.h"

namespace reform {

template <int D, int NB, int NW>
__global__ __launch_bounds__(NW * 64, 2) void tree_attend(TreeParams p)
{
    using S = SeqShape<D, NB, NW>;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    tree_walk<u16, S::R, S::TK>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        seq_segment<D, NB, NW, true>(r, k, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                     slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, smem);
    });
}

template <int D, int NW, int KG, bool THIN>
__global__ __launch_bounds__(NW * KG * 64, 2) void tree_attend_rows(TreeParams p)
{
    using S = RowsShape<D, NW, KG, THIN>;
    extern __shared__ __attribute__((aligned(16))) u16 lds[];
    tree_walk<u16, S::ROWS, S::BN>(p, [&](const SeqRows &r, const SeqKeys &k, int t0, int t1, long slot) {
        rows_segment<D, NW, KG, true, THIN>(r, k, false, p.scale, t0, t1, slot < 0 ? nullptr : p.part_o + (size_t)slot * p.part_rows * D,
                                  slot < 0 ? nullptr : p.part_ml + (size_t)slot * p.part_rows, lds);
    });
}

namespace {

// Rows of a block (shared_rows).  Fitted to 230 batches of 17 to 512 rows over 300 to 12000 keys, 1 to 64 sequences, in every form: the choice takes
// 1.3 % more time in the mean than the best form, at worst 1.34 times it; the smallest block that takes all rows 23 %.  146 other batches, with the form
// of 192 rows: 2.3 %, at worst 1.47 times (504 rows of 8 caches of up to 3682 keys, 128 wide, 14.8 us in blocks of 16, 21.8).
int tree_rows(const TreeParams &p, int compute_units)
{
    const int rows = p.T * p.G;
    const bool narrow = p.D == 64;
    const double keys = (double)p.max_len + p.T, items = (double)p.n_seq * p.Hkv;
    const int R = shared_rows(p.D, rows, keys, items, compute_units);
    if (R < 128) return R;
    if (rows <= 128) return 128;
    if (rows <= 192) return 192;
    const int by_128 = (rows + 127) / 128, by_192 = (rows + 191) / 192;
    if (by_128 % 2 == 0) return 256;                     // none is half empty
    // As few rows empty by 192, and K and V read less often: 371 rows of 32 x 4 caches of up to 1328 keys, 128 wide, 37.3 us against 41.3; but 64
    // wide 74.6 against 73.0 (280 of 64 x 4 of up to 2351), and where the chip is not busy 35.2 against 28.0 (304 of 32 x 2 of up to 1035).
    return !narrow && by_192 * 192 <= by_128 * 128 && by_192 * (keys + 400) * items / compute_units > 1500 ? 192 : 128;
}

// Keys of a tile.
int tree_keys(int rows) { return rows > 32 ? kRowsKeys : 32; }

template <int D, int NB, int NW>
hipError_t launch(const TreeParams &p, hipStream_t st)
{
    using S = SeqShape<D, NB, NW>;
    const hipError_t e = raise_lds<tree_attend<D, NB, NW>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    hipLaunchKernelGGL((tree_attend<D, NB, NW>), dim3(grid), dim3(NW * 64), S::lds_bytes, st, p);
    if (p.shares) tree_merge_launch<D, S::R, S::TK, true>(p, st);
    return hipGetLastError();
}

template <int D, int NW, int KG, bool THIN = false>
hipError_t launch_long(const TreeParams &p, hipStream_t st)
{
    using S = RowsShape<D, NW, KG, THIN>;
    const hipError_t e = raise_lds<tree_attend_rows<D, NW, KG, THIN>>(S::lds_bytes);
    if (e != hipSuccess) return e;
    const unsigned grid = (unsigned)(p.shares ? p.shares : p.n_seq * p.Hkv) * p.row_blocks;
    hipLaunchKernelGGL((tree_attend_rows<D, NW, KG, THIN>), dim3(grid), dim3(NW * KG * 64), S::lds_bytes, st, p);
    if (p.shares) tree_merge_launch<D, S::ROWS, S::BN, true>(p, st);
    return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const TreeParams &p, hipStream_t st)
{
    const int R = p.block;
    constexpr int NW = D == 64 ? 4 : 8;
    if (R == 16) return launch<D, 1, NW>(p, st);
    if (R == 32) return launch<D, 2, NW>(p, st);
    if (R == 64) return launch_long<D, 2, 2>(p, st);
    if (R == 128) return launch_long<D, 4, 1>(p, st);
    if (R == 192) return launch_long<D, 8, 1, true>(p, st);
    return launch_long<D, 8, 1>(p, st);
}

}  // namespace

void tree_plan_bf16(TreeParams &p, int compute_units)
{
    const int R = tree_rows(p, compute_units), keys = tree_keys(R);
    const bool narrow = p.D == 64;
    // Keys that one workgroup takes alone before sharing them out is faster, and that a share has at least: fitted to 360 batches of 1 to
    // 512 rows, 1 to 64 sequences of 300 to 8000 keys, each whole and shared out with 128 and 256 keys or more.  240 other ones of 300 to 25000 keys
    // against 1024 and 256 for all, means by rows: up to 16 0.96, 32 0.95, 64 0.90 (with the two groups), 128 0.97, 256 0.97, 512 0.98; at
    // worst 1.12 (77 rows of 4 x 8 caches of up to 990 keys 14.8 -> 16.3 us).  150 others of 1 to 512 rows over 300 to 8000 keys: 0.88 of all whole, 0.86 of all
    // shared out, at worst 1.21 times the better (224 rows of 32 x 8 caches of up to 2471 keys, 128 wide, 76.7 us whole, 93.1).
    const int whole = R == 16 ? (narrow ? 2000 : 1600) : R == 32 ? (narrow ? 2000 : 1300) : R == 64 ? (narrow ? 1600 : 1000) :
                      R == 128 ? (narrow ? 1000 : 700) : narrow ? 800 : 600;
    const int least = (R == 16 && narrow ? 256 : 128) / keys;
    tree_plan(p, R, keys, whole, least, compute_units, (R == 128 || (R <= 32 && narrow) ? 2 : 1) * compute_units);
}

hipError_t tree_attend_bf16(const TreeParams &p, hipStream_t st)
{
    return p.D == 64 ? launch_rows<64>(p, st) : launch_rows<128>(p, st);
}

}  // namespace reform
