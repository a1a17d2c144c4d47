// Building blocks of the bf16 attention kernels for gfx950: matrix instruction, transposing LDS read and the
// probabilities of a tile.
#pragma once
#include "common.h"

namespace reform {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// A row whose tile sum reaches this outgrew its reference maximum: the tile is formed anew with the true one.
constexpr float kBigSum = 65536.0f;

// ds_read_b64_tr_b16 (gfx950).  Within each group of 16 lanes, lane r supplies the address of four
// consecutive 16-bit elements B[r][0..3]; lane i of the group receives, as element j,
// B[4*j + i/4][i%4] (established by writing element indices into LDS and reading them back).  With
// lane r = 4*j + q pointing at V[key_j][d0 + 4*q .. +3], lane i therefore receives
// V[key_0..3][d0 + i]: four keys of one d column, half of an MFMA A operand of V^T.
__device__ __forceinline__ v2u lds_read_tr16(const u16 *p)
{
    typedef short v4s __attribute__((ext_vector_type(4)));
    const v4s r = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s *)p);
    return __builtin_bit_cast(v2u, r);
}

__device__ __forceinline__ f32x4 mfma16(v4u a, v4u b, f32x4 c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}

// p = exp2(s*c - mc) for the 16 logits a lane holds of one query and one 64-key tile (four 16-key
// blocks x 4 keys), packed to bf16 as the two B operands of P.V (key pairs 0 and 1); returns the
// lane's partial row sum.  Plain v_add_f32 on purpose: v_dot2c_f32_bf16 was measured NOT to
// co-execute with another wave's MFMAs on gfx950, while v_fma / v_add / v_exp / v_cvt_pk do.
__device__ __forceinline__ float softmax_row(const f32x4 (&s)[4], float c, float mc, v4u (&pb)[2])
{
    float rs = 0.f;
#pragma unroll
    for (int kp = 0; kp < 2; ++kp) {
        float pv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            pv[j] = __builtin_amdgcn_exp2f(fmaf(s[2 * kp + (j >> 2)][j & 3], c, -mc));
            rs += pv[j];
        }
        v4u w;
        w.x = pack_bf16x2(pv[0], pv[1]);
        w.y = pack_bf16x2(pv[2], pv[3]);
        w.z = pack_bf16x2(pv[4], pv[5]);
        w.w = pack_bf16x2(pv[6], pv[7]);
        pb[kp] = w;
    }
    return rs;
}

}  // namespace reform
