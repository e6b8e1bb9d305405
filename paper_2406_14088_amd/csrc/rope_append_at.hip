// Rotary embedding and cache append of a span of new tokens at given positions and slots (rl_op_rope_append_at): part of a head
// or all of it, neighbouring or half-split pairs, the cache half or block-scaled, contiguous or paged.
#include "kernels.h"

// One thread per pair of elements; a head is hd / 2 consecutive lanes, so the maximum of a block-scaled row is a shuffle reduction.
__global__ __launch_bounds__(256) void rope_append_at_kernel(RopeAppendAtArgs a) {
    const int m = blockIdx.x, b = m / a.T, t = m % a.T;
    if (a.d_span && t >= a.d_span[b]) return;
    const long pos = (long)a.d_pos[b] + t, slot = (long)a.d_slot[b] + t;
    if (pos < 0 || pos >= a.tab_rows || slot < 0 || slot >= a.S) return;
    const int hd = a.hd, half = hd >> 1, rh = a.rot_dim >> 1;
    const int it = blockIdx.y * 256 + threadIdx.x;
    const int head = it / half, r = it % half;
    const int heads = a.Hq + 2 * a.Hkv;
    const bool valid = head < heads;
    const int kind = head < a.Hq ? 0 : (head < a.Hq + a.Hkv ? 1 : 2);
    const int kvh = kind == 0 ? 0 : (head - a.Hq) % a.Hkv;
    // pair r of a head: the first rot_dim / 2 pairs rotate, the others are neighbours behind them
    int ia = 2 * r, ib = 2 * r + 1;
    if (r < rh && a.rope_style == 1) { ia = r; ib = r + rh; }
    float x = 0.f, y = 0.f;
    if (valid) {
        const float *row = a.qkv + (size_t)m * heads * hd + (size_t)head * hd;
        for (int s = 0; s < a.nsplit; ++s) {
            x += row[s * a.split_stride + ia];
            y += row[s * a.split_stride + ib];
        }
        if (kind != 2 && r < rh) {
            const float *cs = a.rope_tab + (size_t)pos * a.rot_dim + 2 * r;
            const float xr = x * cs[0] - y * cs[1], yr = x * cs[1] + y * cs[0];
            x = xr; y = yr;
        }
        if (kind == 0) {
            const size_t o = ((size_t)m * a.Hq + head) * hd;
            if (a.q_f32) { a.q_f32[o + ia] = x; a.q_f32[o + ib] = y; }
            if (a.q_f16) {
                const f16_t hx = f32_to_f16(x), hy = f32_to_f16(y);
                a.q_f16[o + ia] = hx; a.q_f16[o + ib] = hy;
                if (a.q_f16_lo) { a.q_f16_lo[o + ia] = f32_to_f16(x - f16_to_f32(hx)); a.q_f16_lo[o + ib] = f32_to_f16(y - f16_to_f32(hy)); }
            }
        }
    }
    float am = kind != 0 ? fmaxf(fabsf(x), fabsf(y)) : 0.f;
    if (a.map.kscale)
        for (int o = 1; o < half; o <<= 1) am = fmaxf(am, __shfl_xor(am, o, 64));
    if (!valid || kind == 0) return;
    const size_t rowi = kv_row_index(a.map, b, kvh, a.Hkv, a.S, (int)slot);
    f16_t *dst = (kind == 1 ? a.kc : a.vc) + rowi * hd;
    if (a.map.kscale) {
        const float inv = kv_inv_of(am);
        dst[ia] = (f16_t)(kv_quant(x, inv) & 0xffff);
        dst[ib] = (f16_t)(kv_quant(y, inv) & 0xffff);
        if (r == 0) (kind == 1 ? a.map.kscale : a.map.vscale)[rowi] = kv_scale_of(am);
    } else {
        dst[ia] = f32_to_f16(x);
        dst[ib] = f32_to_f16(y);
    }
    if (kind == 1 && r == 0) {
        const size_t w = ((size_t)b * a.Hkv + kvh) * a.S + slot;
        if (a.weight) a.weight[w] = 0.f;
        if (a.row_pos) a.row_pos[w] = (int32_t)pos;
    }
}

void launch_rope_append_at(const RopeAppendAtArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    rope_append_at_kernel<<<dim3(a.B * a.T, ceil_div((a.Hq + 2 * a.Hkv) * (a.hd / 2), 256)), 256, 0, st>>>(a);
}
