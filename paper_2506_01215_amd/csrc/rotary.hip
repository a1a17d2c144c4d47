// Rotary positions: queries and keys of new tokens rotated to their positions, keys and values put
// into the rows of the caches that the attention calls read (see reform_rotary_embed in reform.h).
//
// A pair (x, x') of a token at position p is turned by the angle p f_c, the same for every head, so a
// thread owns one token and one unit of two 16-byte pieces (the low and the high half's with
// PAIRS_HALVES, two neighbours with PAIRS_ADJACENT), forms the unit's sines and cosines once, in
// registers, and walks over heads with them.
//
// Bound: HBM (every element is read and written once): 8192 tokens, 32/8 heads of 128 into a cache 44 us, 4.6 TB/s, a copy's rate.  Few tokens:
// latency, 4.3 us for 16.
#include "rope_math.h"

namespace reform {

constexpr int kRotaryThreads = 256;

// BATCH heads are loaded at once; the first of them while the frequencies and angles are formed.
template <bool BF16, bool ADJACENT, int BATCH>
__global__ __launch_bounds__(kRotaryThreads) void rotary_embed(RotaryParams p, int heads_each)
{
    __shared__ double table[kRotaryMaxDim / 2];          // quarter turns per position of every pair
    constexpr int E = BF16 ? 8 : 4;                      // elements of a piece
    const int pieces = p.elts / E, rot_pieces = p.rot / E;
    // units: first those that rotate, then those that are copied, two pieces each (the last may have one)
    const int rot_units = ADJACENT ? (rot_pieces + 1) / 2 : rot_pieces / 2;
    const int units = rot_units + (pieces - rot_pieces + 1) / 2;
    const unsigned gid = blockIdx.x * kRotaryThreads + threadIdx.x;      // tokens x units are below 2^31
    const unsigned row = gid / (unsigned)units;
    const bool live = row < (unsigned)p.n;
    const int token = live ? (int)row : 0, unit = (int)(gid - row * (unsigned)units);
    const bool turns = unit < rot_units;
    int a, b;                                            // the unit's pieces; b < 0: it has one
    if (turns) {
        a = ADJACENT ? 2 * unit : unit;
        b = ADJACENT ? (2 * unit + 1 < rot_pieces ? 2 * unit + 1 : -1) : unit + rot_units;
    } else {
        a = rot_pieces + 2 * (unit - rot_units);
        b = a + 1 < pieces ? a + 1 : -1;
    }
    const int first = blockIdx.y * heads_each, last = min(first + heads_each, p.heads[0] + p.heads[1] + p.heads[2]);
    // part (0 q, 1 k, 2 v) and head of the h-th of all heads; the same for the whole workgroup
    auto part_of = [&](int &h) {
        if (h < p.heads[0]) return 0;
        h -= p.heads[0];
        if (h < p.heads[1]) return 1;
        h -= p.heads[1];
        return 2;
    };
    v4u lo[BATCH], hi[BATCH];
    auto load = [&](int g) {
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            int h = min(g + i, last - 1);
            const int part = part_of(h);
            const char *from = (const char *)p.src[part] + (size_t)h * p.src_hs[part] + (size_t)token * p.src_rs[part];
            lo[i] = *(const v4u *)(from + a * 16);
            hi[i] = *(const v4u *)(from + (b < 0 ? a : b) * 16);
        }
    };
    if (live) load(first);
    const int s = p.n_slots && live ? p.slot[token] : 0, pos = live ? p.pos[token] : 0;
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
    if (!live) return;
    float sn[E], cs[E];
    if (turns) {
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const int c = min(unit * E + i, p.rot / 2 - 1);
            sin_cos_quarter((double)pos * table[c], sn[i], cs[i]);
            sn[i] *= p.magnitude;
            cs[i] *= p.magnitude;
        }
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) sn[i] = 0.f, cs[i] = 1.f;
    }
    const bool stored = !p.n_slots || (unsigned)s < p.n_slots;
    for (int g = first; g < last; g += BATCH) {
        if (g != first) load(g);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            if (g + i >= last) break;
            int h = g + i;
            const int part = part_of(h);
            const bool rotate = part < 2 && turns;
            if ((part && !stored) || (!rotate && p.skip_rest[part])) continue;
            if (rotate) {
                float x[2 * E], y[2 * E];
                const uint32_t w[8] = {lo[i].x, lo[i].y, lo[i].z, lo[i].w, hi[i].x, hi[i].y, hi[i].z, hi[i].w};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (BF16) {
                        x[2 * e] = __uint_as_float(w[e] << 16);
                        x[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    } else {
                        x[e] = __uint_as_float(w[e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const int u = ADJACENT ? 2 * e : e, v = ADJACENT ? 2 * e + 1 : e + E;
                    y[u] = x[u] * cs[e] - x[v] * sn[e];
                    y[v] = x[v] * cs[e] + x[u] * sn[e];
                }
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = BF16 ? pack_bf16x2(y[BF16 ? 2 * e : e], y[BF16 ? 2 * e + 1 : e]) : __float_as_uint(y[e]);
                lo[i] = (v4u){o[0], o[1], o[2], o[3]};
                hi[i] = (v4u){o[4], o[5], o[6], o[7]};
            }
            char *to = (char *)p.dst[part] + (size_t)h * p.dst_hs[part];
            if (part && p.n_slots) to += (size_t)(s / p.block_len) * p.block_bytes + (size_t)(s % p.block_len) * p.dst_rs[part];
            else to += (size_t)token * p.dst_rs[part];
            *(v4u *)(to + a * 16) = lo[i];
            if (b >= 0) *(v4u *)(to + b * 16) = hi[i];
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
    // Up to eight heads to a thread, which forms its sines and cosines once for them; fewer where the workgroups would not give
    // every compute unit a few (16 tokens, 32/8 heads of 128: eight heads to a thread 6.7 us, one 4.4).
    int each = 8;
    while (each > 1 && groups * ((heads + each - 1) / each) < 1024) each /= 2;
    const dim3 grid((unsigned)groups, (unsigned)((heads + each - 1) / each));
#define REFORM_ROTARY(B, A) \
    do { \
        if (each >= 4) hipLaunchKernelGGL((rotary_embed<B, A, 4>), grid, dim3(kRotaryThreads), 0, st, p, each); \
        else hipLaunchKernelGGL((rotary_embed<B, A, 1>), grid, dim3(kRotaryThreads), 0, st, p, each); \
    } while (0)
    if (bf16 && adjacent) REFORM_ROTARY(true, true);
    else if (bf16) REFORM_ROTARY(true, false);
    else if (adjacent) REFORM_ROTARY(false, true);
    else REFORM_ROTARY(false, false);
#undef REFORM_ROTARY
    return hipGetLastError();
}

}  // namespace reform
