// Rotary embedding and cache append of a span of new tokens at given positions and slots (rl_op_rope_append_at): part of a head
// or all of it, neighbouring or half-split pairs, the cache half or block-scaled, contiguous or paged.
//
// A stream: every value of the projection (nsplit fp32 partials) is read once, q and the cache rows are written once.  A thread takes 8
// elements of a head -- four pairs, or 8 neighbours of the part that does not rotate -- as two 16-byte loads per partial, issued before the
// positions are known, so that the chain of latencies is positions -> table -> stores.  8 or 16 consecutive lanes hold a head: the
// maximum of a block-scaled row is a reduction among them.
//
// Measured: 8 x 509 tokens, 32/8 heads of 128, paged, 40 us (185 MB, 4.6 TB/s; a copy of 4 GiB reaches 4.8); 32 x 5 tokens, 32 heads, four
// partials, 8.0 us (37 MB, 4.6 TB/s).  Block-scaled rows take as long (39.7 and 39.1 us, 11.3 and 11.2 with the host's call).
#include "kernels.h"

template <bool SCALED>
__global__ __launch_bounds__(256) void rope_append_at_kernel(RopeAppendAtArgs a) {
    const int m = blockIdx.x, b = m / a.T, t = m % a.T, hd = a.hd;
    const int lph = hd >> 3, sh = hd == 128 ? 4 : 3;  // threads of a head
    const int it = blockIdx.y * 256 + threadIdx.x, head = it >> sh, u = it & (lph - 1);
    const int heads = a.Hq + 2 * a.Hkv;
    const bool valid = head < heads;
    const int kind = head < a.Hq ? 0 : (head < a.Hq + a.Hkv ? 1 : 2);
    // first and second group of four elements: elements that pair up with each other in style 1, neighbours otherwise
    const int rh = a.rot_dim >> 1;
    const bool turns = kind != 2 && 8 * u < a.rot_dim, halves = a.rope_style == 1 && 8 * u < a.rot_dim;
    const int e0 = halves ? 4 * u : 8 * u, e1 = halves ? 4 * u + rh : 8 * u + 4;
    f32x4_t x = {0.f, 0.f, 0.f, 0.f}, y = {0.f, 0.f, 0.f, 0.f};
    if (valid) {
        const float *row = a.qkv + ((size_t)m * heads + head) * hd;
        x = *reinterpret_cast<const f32x4_t *>(row + e0);
        y = *reinterpret_cast<const f32x4_t *>(row + e1);
        for (int s = 1; s < a.nsplit; ++s) {
            x += *reinterpret_cast<const f32x4_t *>(row + s * a.split_stride + e0);
            y += *reinterpret_cast<const f32x4_t *>(row + s * a.split_stride + e1);
        }
    }
    if (a.d_span && t >= a.d_span[b]) return;
    const int64_t pos = (int64_t)a.d_pos[b] + t, slot = (int64_t)a.d_slot[b] + t;
    if (pos < 0 || pos >= a.tab_rows || slot < 0 || slot >= a.S) return;
    if (valid && turns) {
        const float *cs = a.rope_tab + (size_t)pos * a.rot_dim + 8 * u;  // (cos, sin) of pairs 4 u .. 4 u + 3
        const f32x4_t c0 = *reinterpret_cast<const f32x4_t *>(cs), c1 = *reinterpret_cast<const f32x4_t *>(cs + 4);
        const float co[4] = {c0.x, c0.z, c1.x, c1.z}, si[4] = {c0.y, c0.w, c1.y, c1.w};
        if (halves) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = x[i], q = y[i];
                x[i] = __builtin_fmaf(p, co[i], -(q * si[i]));  // the roundings of rope_append_kernel
                y[i] = __builtin_fmaf(q, co[i], p * si[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float p = x[2 * i], q = x[2 * i + 1], r = y[2 * i], s = y[2 * i + 1];
                x[2 * i] = __builtin_fmaf(p, co[i], -(q * si[i]));
                x[2 * i + 1] = __builtin_fmaf(q, co[i], p * si[i]);
                y[2 * i] = __builtin_fmaf(r, co[2 + i], -(s * si[2 + i]));
                y[2 * i + 1] = __builtin_fmaf(s, co[2 + i], r * si[2 + i]);
            }
        }
    }
    float am = 0.f;
    if (SCALED) {  // the largest magnitude by its bits: a NaN is above everything and gives a row whose scale is one
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t p = __float_as_uint(x[i]) & 0x7fffffffu, q = __float_as_uint(y[i]) & 0x7fffffffu, r = p > q ? p : q;
            top = r > top ? r : top;
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) {
            if (o == 8 && hd != 128) break;
            const uint32_t r = __shfl_xor(top, o, 64);
            top = r > top ? r : top;
        }
        am = __uint_as_float(top);
    }
    if (!valid) return;
    if (kind == 0) {
        const size_t o = ((size_t)m * a.Hq + head) * hd;
        if (a.q_f32) {
            *reinterpret_cast<f32x4_t *>(a.q_f32 + o + e0) = x;
            *reinterpret_cast<f32x4_t *>(a.q_f32 + o + e1) = y;
        }
        if (a.q_f16) {
            const u32x2_t hx = {pack_f16x2_nan(x.x, x.y), pack_f16x2_nan(x.z, x.w)}, hy = {pack_f16x2_nan(y.x, y.y), pack_f16x2_nan(y.z, y.w)};
            *reinterpret_cast<u32x2_t *>(a.q_f16 + o + e0) = hx;
            *reinterpret_cast<u32x2_t *>(a.q_f16 + o + e1) = hy;
            if (a.q_f16_lo) {
                *reinterpret_cast<u32x2_t *>(a.q_f16_lo + o + e0) = u32x2_t{pack_f16x2_lo_nan(x.x, x.y, hx.x), pack_f16x2_lo_nan(x.z, x.w, hx.y)};
                *reinterpret_cast<u32x2_t *>(a.q_f16_lo + o + e1) = u32x2_t{pack_f16x2_lo_nan(y.x, y.y, hy.x), pack_f16x2_lo_nan(y.z, y.w, hy.y)};
            }
        }
        return;
    }
    const int kvh = kind == 1 ? head - a.Hq : head - a.Hq - a.Hkv;
    const size_t rowi = kv_row_index(a.map, b, kvh, a.Hkv, a.S, (int)slot);
    f16_t *dst = (kind == 1 ? a.kc : a.vc) + rowi * hd;
    u32x2_t hx, hy;
    if (SCALED) {
        const float inv = am > 0x1p-100f ? kv_inv_of(am) : 0.f;  // a smaller row counts as zeros: its reciprocal may be infinite
        hx = u32x2_t{pack_i16x2(kv_quant(x.x, inv), kv_quant(x.y, inv)), pack_i16x2(kv_quant(x.z, inv), kv_quant(x.w, inv))};
        hy = u32x2_t{pack_i16x2(kv_quant(y.x, inv), kv_quant(y.y, inv)), pack_i16x2(kv_quant(y.z, inv), kv_quant(y.w, inv))};
        if (u == 0) (kind == 1 ? a.map.kscale : a.map.vscale)[rowi] = kv_scale_of(am);
    } else {
        hx = u32x2_t{pack_f16x2_nan(x.x, x.y), pack_f16x2_nan(x.z, x.w)};
        hy = u32x2_t{pack_f16x2_nan(y.x, y.y), pack_f16x2_nan(y.z, y.w)};
    }
    *reinterpret_cast<u32x2_t *>(dst + e0) = hx;
    *reinterpret_cast<u32x2_t *>(dst + e1) = hy;
    if (kind == 1 && u == 0) {
        const size_t w = ((size_t)b * a.Hkv + kvh) * a.S + slot;
        if (a.weight) a.weight[w] = 0.f;
        if (a.row_pos) a.row_pos[w] = (int32_t)pos;
    }
}

void launch_rope_append_at(const RopeAppendAtArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    const dim3 grid(a.B * a.T, ceil_div((a.Hq + 2 * a.Hkv) * (a.hd / 8), 256));
    if (a.map.kscale) rope_append_at_kernel<true><<<grid, 256, 0, st>>>(a);
    else rope_append_at_kernel<false><<<grid, 256, 0, st>>>(a);
}
