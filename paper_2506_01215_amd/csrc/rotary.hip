// Rotary positions: queries and keys of new tokens rotated to their positions, keys and values put
// into the rows of the caches that the attention calls read (see reform_rotary_embed in reform.h).
//
// A pair (x, x') of a token at position p is turned by the angle p f_c, the same for every head, so a
// thread owns one token and one unit of two 16-byte pieces (the low and the high half's with
// PAIRS_HALVES, two neighbours with PAIRS_ADJACENT), forms the unit's sines and cosines once, in
// registers, and walks over heads with them.
//
// Bound: HBM (every element is read and written once).
#include "rope_math.h"

namespace reform {

constexpr int kRotaryThreads = 256;

template <bool BF16, bool ADJACENT>
__global__ __launch_bounds__(kRotaryThreads) void rotary_embed(RotaryParams p, int heads_each)
{
    __shared__ double table[kRotaryMaxDim / 2];          // quarter turns per position of every pair
    constexpr int E = BF16 ? 8 : 4;                      // elements of a piece
    const int pieces = p.elts / E, rot_pieces = p.rot / E;
    // units: first those that rotate, then those that are copied, two pieces each (the last may have one)
    const int rot_units = ADJACENT ? (rot_pieces + 1) / 2 : rot_pieces / 2;
    const int units = rot_units + (pieces - rot_pieces + 1) / 2;
    for (int c = threadIdx.x; c < p.rot / 2; c += kRotaryThreads) {
        double f = exp2(p.neg2_log2_theta_over_rot * (double)c) * 0.63661977236758134 * p.scale;
        if (p.ramp) {
            const double x = p.ramp == 1 ? (double)c : f * p.turns;
            const double r = fmin(fmax((x - p.ramp_at) * p.ramp_inv, 0.0), 1.0);
            f *= 1.0 - r + r * p.ramp_low;
        }
        table[c] = p.inverse ? -f : f;
    }
    __syncthreads();
    const long gid = (long)blockIdx.x * kRotaryThreads + threadIdx.x;
    const int token = (int)(gid / units), unit = (int)(gid - (long)token * units);
    if (token >= p.n) return;
    const bool turns = unit < rot_units;
    int a, b;                                            // the unit's pieces; b < 0: it has one
    if (turns) {
        a = ADJACENT ? 2 * unit : unit;
        b = ADJACENT ? (2 * unit + 1 < rot_pieces ? 2 * unit + 1 : -1) : unit + rot_units;
    } else {
        a = rot_pieces + 2 * (unit - rot_units);
        b = a + 1 < pieces ? a + 1 : -1;
    }
    float sn[E], cs[E];
    if (turns) {
        const double at = (double)p.pos[token];
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = min(unit * E + i, p.rot / 2 - 1);
            sin_cos_quarter(at * table[c], sn[i], cs[i]);
            sn[i] *= p.magnitude;
            cs[i] *= p.magnitude;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) sn[i] = 0.f, cs[i] = 1.f;
    }
    const int s = p.n_slots ? p.slot[token] : 0;
    const bool stored = !p.n_slots || (unsigned)s < p.n_slots;
    const int first = blockIdx.y * heads_each, last = first + heads_each;
    int base = 0;
#pragma unroll
    for (int part = 0; part < 3; ++part) {
        const int h0 = max(first - base, 0), h1 = min(last - base, p.heads[part]);
        base += p.heads[part];
        if (h0 >= h1 || (part && !stored)) continue;
        const bool rotate = part < 2 && turns;
        if (!rotate && p.skip_rest[part]) continue;
        const char *src = (const char *)p.src[part] + (size_t)token * p.src_rs[part];
        char *dst = (char *)p.dst[part];
        if (part && p.n_slots) dst += (size_t)(s / p.block_len) * p.block_bytes + (size_t)(s % p.block_len) * p.dst_rs[part];
        else dst += (size_t)token * p.dst_rs[part];
#pragma unroll 4
        for (int h = h0; h < h1; ++h) {
            const char *from = src + (size_t)h * p.src_hs[part];
            char *to = dst + (size_t)h * p.dst_hs[part];
            v4u lo = *(const v4u *)(from + a * 16), hi = {0u, 0u, 0u, 0u};
            if (b >= 0) hi = *(const v4u *)(from + b * 16);
            if (rotate) {
                float x[2 * E];
                const uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if (BF16) {
                        x[2 * i] = __uint_as_float(w[i] << 16);
                        x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
                    } else {
                        x[i] = __uint_as_float(w[i]);
                    }
                }
                float y[2 * E];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const int u = ADJACENT ? 2 * i : i, v = ADJACENT ? 2 * i + 1 : i + E;
                    y[u] = x[u] * cs[i] - x[v] * sn[i];
                    y[v] = x[v] * cs[i] + x[u] * sn[i];
                }
                uint32_t o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = BF16 ? pack_bf16x2(y[BF16 ? 2 * i : i], y[BF16 ? 2 * i + 1 : i]) : __float_as_uint(y[i]);
                lo = (v4u){o[0], o[1], o[2], o[3]};
                hi = (v4u){o[4], o[5], o[6], o[7]};
            }
            *(v4u *)(to + a * 16) = lo;
            if (b >= 0) *(v4u *)(to + b * 16) = hi;
        }
    }
}

hipError_t rotary_embed_launch(const RotaryParams &p, bool bf16, bool adjacent, hipStream_t st)
{
    const int E = bf16 ? 8 : 4, pieces = p.elts / E, rot_pieces = p.rot / E;
    const int units = (adjacent ? (rot_pieces + 1) / 2 : rot_pieces / 2) + (pieces - rot_pieces + 1) / 2;
    const int heads = p.heads[0] + p.heads[1] + p.heads[2];
    if (p.n == 0 || heads == 0) return hipSuccess;
    const long groups = ((long)p.n * units + kRotaryThreads - 1) / kRotaryThreads;
    const int each = 8;
    const dim3 grid((unsigned)groups, (unsigned)((heads + each - 1) / each));
#define REFORM_ROTARY(B, A) hipLaunchKernelGGL((rotary_embed<B, A>), grid, dim3(kRotaryThreads), 0, st, p, each)
    if (bf16 && adjacent) REFORM_ROTARY(true, true);
    else if (bf16) REFORM_ROTARY(true, false);
    else if (adjacent) REFORM_ROTARY(false, true);
    else REFORM_ROTARY(false, false);
#undef REFORM_ROTARY
    return hipGetLastError();
}

}  // namespace reform
