// Verification of drafted tokens against the target's probabilities (rl_op_verify_drafts).
#include "kernels.h"

#define VD_THREADS 1024
#define VD_WAVES (VD_THREADS / RL_WAVE)

__device__ __forceinline__ double vd_wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// A logits row: its largest value and lowest index (ties), whether it can be used, and the sum of exp((x - max) * inv).
struct VdRow {
    double max, sum;
    int arg;
    bool ok;
};

__device__ VdRow vd_row(const float *row, int V, double inv, bool greedy, double *redd, int *redi) {
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    float m = -INFINITY;
    int arg = 0x7fffffff;
    int nan = 0;
    for (int i = tid; i < V; i += VD_THREADS) {
        const float x = row[i];
        nan |= x != x;
        if (x > m || (x == m && i < arg)) { m = x; arg = i; }
    }
    for (int o = 32; o > 0; o >>= 1) {
        const float om = __shfl_xor(m, o, 64);
        const int oa = __shfl_xor(arg, o, 64);
        nan |= __shfl_xor(nan, o, 64);
        if (om > m || (om == m && oa < arg)) { m = om; arg = oa; }
    }
    __syncthreads();
    if (lane == 0) { redd[wv] = m; redi[wv] = nan ? -1 : arg; }
    __syncthreads();
    VdRow r;
    r.max = -INFINITY; r.arg = 0x7fffffff; r.ok = true; r.sum = 0;
    for (int w = 0; w < VD_WAVES; ++w) {
        if (redi[w] < 0) r.ok = false;
        else if (redd[w] > r.max || (redd[w] == r.max && redi[w] < r.arg)) { r.max = redd[w]; r.arg = redi[w]; }
    }
    if (!greedy && !(fabs(r.max) < INFINITY)) r.ok = false;
    __syncthreads();
    double s = 0;
    if (r.ok && fabs(r.max) < INFINITY)
        for (int i = tid; i < V; i += VD_THREADS) s += exp(((double)row[i] - r.max) * inv);
    s = vd_wave_sum(s);
    if (lane == 0) redd[wv] = s;
    __syncthreads();
    for (int w = 0; w < VD_WAVES; ++w) r.sum += redd[w];
    __syncthreads();
    return r;
}

// One workgroup per sequence, row after row.
__global__ __launch_bounds__(VD_THREADS) void verify_drafts_kernel(VerifyArgs a) {
    __shared__ double redd[VD_WAVES], s_pre;
    __shared__ int redi[VD_WAVES], s_tok, s_owner;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    const bool greedy = !(a.temperature > 0);
    const double inv = greedy ? 1.0 : 1.0 / a.temperature;
    int n = a.T;
    if (a.d_span) n = a.d_span[b] < 0 ? 0 : (a.d_span[b] < n ? a.d_span[b] : n);
    int32_t *tokens = a.tokens + (size_t)b * (a.T + 1);
    float *logp = a.logp ? a.logp + (size_t)b * (a.T + 1) : nullptr;
    int i = 0;
    bool rejected = false, bad = false;
    VdRow p, q;
    const float *prow, *qrow = nullptr;
    int x = -1;
    for (;; ++i) {
        prow = a.target + ((size_t)b * (a.T + 1) + i) * a.ldt;
        p = vd_row(prow, a.V, inv, greedy, redd, redi);
        bad = !p.ok;
        if (bad || i == n) break;
        x = a.drafts[(size_t)b * a.T + i];
        const bool in = x >= 0 && x < a.V;
        bool ok;
        if (greedy) {
            ok = x == p.arg;
        } else {
            double qx = 1.0;
            if (a.draft) {
                qrow = a.draft + ((size_t)b * a.T + i) * a.ldd;
                q = vd_row(qrow, a.V, inv, false, redd, redi);
                if (!q.ok) { bad = true; break; }
                qx = in ? exp(((double)qrow[x] - q.max) * inv) / q.sum : 0.0;
            }
            ok = in && (double)a.u[(size_t)b * (a.T + 1) + i] * qx < exp(((double)prow[x] - p.max) * inv) / p.sum;
        }
        if (!ok) { rejected = true; break; }
        if (tid == 0) {
            tokens[i] = x;
            if (logp) logp[i] = (float)(((double)prow[x] - p.max) * inv - log(p.sum));
        }
    }
    int next = -1;
    if (!bad && greedy) next = p.arg;
    if (!bad && !greedy) {
        auto weight = [&](int v, bool residual) -> double {
            const double pv = exp(((double)prow[v] - p.max) * inv) / p.sum;
            if (!residual) return pv;
            const double qv = a.draft ? exp(((double)qrow[v] - q.max) * inv) / q.sum : (v == x ? 1.0 : 0.0);
            return pv > qv ? pv - qv : 0.0;
        };
        const int seg = (a.V + VD_THREADS - 1) / VD_THREADS;
        const int i0 = tid * seg < a.V ? tid * seg : a.V, i1 = i0 + seg < a.V ? i0 + seg : a.V;
        for (int pass = 0; pass < 2; ++pass) {
            const bool residual = rejected && pass == 0;
            double s = 0;
            for (int v = i0; v < i1; ++v) s += weight(v, residual);
            double incl = s;
            for (int o = 1; o < 64; o <<= 1) {
                const double up = __shfl_up(incl, o, 64);
                if (lane >= o) incl += up;
            }
            __syncthreads();
            if (lane == 63) redd[wv] = incl;
            if (tid == 0) { s_owner = VD_THREADS; s_tok = -1; s_pre = 0; }
            __syncthreads();
            double base = 0, total = 0;
            for (int w = 0; w < VD_WAVES; ++w) { if (w < wv) base += redd[w]; total += redd[w]; }
            if (residual && !(total > 0)) continue;
            const double target = (double)a.u[(size_t)b * (a.T + 1) + a.T] * total;
            if (s > 0 && base + incl > target) atomicMin(&s_owner, tid);
            __syncthreads();
            if (s_owner == VD_THREADS && s > 0) atomicMax(&s_tok, i1 - 1);  // rounding: the last segment with weight
            if (tid == s_owner) {
                double run = base + incl - s;
                int last = i0;
                for (int v = i0; v < i1; ++v) {
                    const double w = weight(v, residual);
                    if (w > 0) last = v;
                    run += w;
                    if (w > 0 && run > target) break;
                }
                s_tok = last;
            }
            __syncthreads();
            next = s_tok;
            break;
        }
    }
    if (tid == 0) {
        a.accepted[b] = i;
        tokens[i] = next;
        if (logp) logp[i] = next >= 0 ? (float)(((double)prow[next] - p.max) * inv - log(p.sum)) : 0.f;
        for (int k = i + 1; k <= a.T; ++k) { tokens[k] = -1; if (logp) logp[k] = 0.f; }
    }
}

size_t verify_drafts_ws_bytes(int B, int T, int V) { return 256; }

void launch_verify_drafts(const VerifyArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    verify_drafts_kernel<<<a.B, VD_THREADS, 0, st>>>(a);
}
