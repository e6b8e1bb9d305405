// Attention of a span of new tokens over a cache (rl_op_span_attention), with the attention weight of every cached row on request.
#include "kernels.h"

__device__ __forceinline__ float span_elem(const f16_t *row, int e, const float *scale, size_t rowi) {
    return scale ? (float)(int16_t)row[e] * scale[rowi] : f16_to_f32(row[e]);
}

// One wavefront per (sequence, token, query head): scores to the workspace, softmax, weighted sum.
__global__ __launch_bounds__(64) void span_attention_kernel(SpanArgs a) {
    const int u = blockIdx.x % a.Hq, t = blockIdx.x / a.Hq, b = blockIdx.y, lane = threadIdx.x, hd = a.hd;
    if (a.d_span && t >= a.d_span[b]) return;
    int n = a.d_len[b];
    n = n < 0 ? 0 : (n > a.S ? a.S : n);
    n = n + t + 1 < a.S ? n + t + 1 : a.S;
    const int kvh = u / (a.Hq / a.Hkv);
    const size_t m = (size_t)b * a.T + t;
    const float *q = a.q + (m * a.Hq + u) * hd;
    float *sc = a.ws + (m * a.Hq + u) * a.S;
    const float scale = rsqrtf((float)hd);
    float mx = -INFINITY;
    for (int j = lane; j < n; j += 64) {
        const size_t rowi = kv_row_index(a.map, b, kvh, a.Hkv, a.S, j);
        float s = 0.f;
        for (int e = 0; e < hd; ++e) s += q[e] * span_elem(a.kc + rowi * hd, e, a.map.kscale, rowi);
        s *= scale;
        sc[j] = s;
        mx = fmaxf(mx, s);
        if (s != s) mx = s;
    }
    mx = wave_max(mx);
    float den = 0.f;
    for (int j = lane; j < n; j += 64) { sc[j] = expf(sc[j] - mx); den += sc[j]; }
    den = wave_sum(den);
    __syncthreads();
    for (int j = lane; j < n; j += 64) sc[j] /= den;
    __syncthreads();
    for (int e = lane; e < hd; e += 64) {
        float o = 0.f;
        for (int j = 0; j < n; ++j) {
            const size_t rowi = kv_row_index(a.map, b, kvh, a.Hkv, a.S, j);
            o += sc[j] * span_elem(a.vc + rowi * hd, e, a.map.vscale, rowi);
        }
        const f16_t h = f32_to_f16(o);
        a.out[(m * a.Hq + u) * hd + e] = h;
        if (a.out_lo) a.out_lo[(m * a.Hq + u) * hd + e] = f32_to_f16(o - f16_to_f32(h));
    }
}

// One thread per cached row: the probabilities of all queries that see it, token after token.
__global__ __launch_bounds__(256) void span_weight_kernel(SpanArgs a) {
    const int j = blockIdx.x * 256 + threadIdx.x, kvh = blockIdx.y, b = blockIdx.z, g = a.Hq / a.Hkv;
    int n0 = a.d_len[b];
    n0 = n0 < 0 ? 0 : (n0 > a.S ? a.S : n0);
    int T = a.T;
    if (a.d_span) T = a.d_span[b] < T ? a.d_span[b] : T;
    if (j >= a.S || j >= n0 + T || T <= 0) return;
    float w = 0.f;
    for (int t = j < n0 ? 0 : j - n0; t < T; ++t)
        for (int u = kvh * g; u < (kvh + 1) * g; ++u) w += a.ws[(((size_t)b * a.T + t) * a.Hq + u) * a.S + j];
    a.weight[((size_t)b * a.Hkv + kvh) * a.S + j] += w;
}

int span_attention_splits(int B, int T, int Hq, int Hkv, int hd, int S) { return 1; }

size_t span_attention_ws_floats(int B, int T, int Hq, int Hkv, int hd, int S, int nsplit, bool weights) {
    return (size_t)B * T * Hq * S;
}

void launch_span_attention(const SpanArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    span_attention_kernel<<<dim3(a.T * a.Hq, a.B), 64, 0, st>>>(a);
    if (a.weight) span_weight_kernel<<<dim3(ceil_div(a.S, 256), a.Hkv, a.B), 256, 0, st>>>(a);
}
