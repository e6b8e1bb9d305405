// Verification of drafted tokens against the target's probabilities (rl_op_verify_drafts).
//
// With x a logits row, m its largest value and z = sum_v exp((x_v - m) / temperature), p_v = exp((x_v - m) / temperature) / z.  Every row
// is read once (vd_rows_kernel: maximum, its index, sum, per chunk of the vocabulary); a sequence's first rejection then
// follows from one probability pair per drafted token, and the next token from the weights max(0, p - q) or p of one row by inversion.
//
// A draw may land next to a border of the cumulative distribution, and a vocabulary of V tokens has V of them: weights with a
// relative error e move a draw to a neighbour with a probability of the order of V * e, about one in a hundred for fp32 (1e-7) and
// V = 128256.  So weights and sums are fp64: 2^g by rounding g to an integer with an addition, a polynomial of degree 8 (relative error
// 1.1e-12 on [-1/2, 1/2]; interpolation at the Chebyshev nodes) and an addition to the exponent: 16 instructions per logit.  fp64
// multiply-adds run at the rate of unpacked fp32 ones here, so the rows stay a stream from HBM.
#include "kernels.h"

#define VD_THREADS 256
#define VD_PICK_THREADS 256

__device__ __forceinline__ double vd_wave_sum(double v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// exp(d / temperature) with c = log2(e) / temperature, for -1020 <= d c <= 1000.
__device__ __forceinline__ double vd_exp(double d, double c) {
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: adding it leaves the nearest integer in the low bits
    const double t = __builtin_fma(d, c, magic);
    const double f = __builtin_fma(d, c, -(t - magic));
    double p = 1.3255224878668817e-06;
    p = __builtin_fma(p, f, 1.5310079402249296e-05);
    p = __builtin_fma(p, f, 0.00015403455852453838);
    p = __builtin_fma(p, f, 0.0013333450568000645);
    p = __builtin_fma(p, f, 0.009618129159402558);
    p = __builtin_fma(p, f, 0.05550410941205933);
    p = __builtin_fma(p, f, 0.2402265069581299);
    p = __builtin_fma(p, f, 0.6931471805459335);
    p = __builtin_fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}
// exp((x - m) / temperature); 0 where it is below 2^-1020 (and for x = -inf), which no sum notices.
__device__ __forceinline__ double vd_weight(float x, double m, double c) {
    const double d = (double)x - m, least = -1020.0 / c;
    const double w = vd_exp(__builtin_fmax(d, least), c);
    return d >= least ? w : 0.0;
}

// Workspace: per (sequence, row, chunk) sum, maximum and index of the maximum (-1: the chunk holds a NaN); per sequence and target
// row its maximum and sum; per (sequence, chunk) the weight of the decisive row; per sequence what was decided.
struct VdDecision {
    int stop, bad, rejected, token;  // first token not accepted; row unusable; draft rejected; the drafted token there
};
struct VdWs {
    double *sum, *row_sum, *mass;
    float *max, *row_max;
    int32_t *arg;
    VdDecision *dec;
};
__host__ __device__ static inline size_t vd_ws(void *base, int B, int T, int chunks, VdWs *w) {
    const size_t rows = (size_t)B * (2 * T + 1), cells = rows * chunks, n8 = cells + rows + (size_t)B * chunks;
    double *d = reinterpret_cast<double *>(base);
    float *f = reinterpret_cast<float *>(d + n8);
    if (w) {
        w->sum = d; w->row_sum = d + cells; w->mass = d + cells + rows;
        w->max = f; w->row_max = f + cells; w->arg = reinterpret_cast<int32_t *>(f + cells + rows);
        w->dec = reinterpret_cast<VdDecision *>(f + 2 * cells + rows);
    }
    return n8 * 8 + (2 * cells + rows) * 4 + (size_t)B * sizeof(VdDecision);
}

__device__ __forceinline__ int vd_span(const VerifyArgs &a, int b) {
    int n = a.T;
    if (a.d_span) { const int s = a.d_span[b]; n = s < 0 ? 0 : (s < n ? s : n); }
    return n;
}
// Row r of a sequence: target rows 0 .. T, then draft rows.
__device__ __forceinline__ const float *vd_row(const VerifyArgs &a, int b, int r) {
    return r <= a.T ? a.target + ((size_t)b * (a.T + 1) + r) * a.ldt : a.draft + ((size_t)b * a.T + (r - a.T - 1)) * a.ldd;
}

// One wavefront per (row, chunk of 64 * EPT logits), four chunks of a row per workgroup: the logits stay in registers between the maximum and the weights, which refer to the
// chunk's own maximum.  SUMS, ARG: whether the sum and the index of the maximum are wanted (sampled: sums; greedy: the index, and sums for
// log-probabilities).
template <int EPT, bool SUMS, bool ARG>
__global__ __launch_bounds__(VD_THREADS, 8) void vd_rows_kernel(VerifyArgs a, int chunks, int rows, int groups) {
    const unsigned id = blockIdx.x / groups;
    const int chunk = (int)(blockIdx.x % groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = (int)(id % rows), b = (int)(id / rows);
    if (chunk >= chunks) return;
    const int n = vd_span(a, b);
    if (r <= a.T ? r > n : r - a.T - 1 >= n) return;  // not reached in any case
    const int first = chunk * (64 * EPT);
    const int left = a.V - first < 64 * EPT ? a.V - first : 64 * EPT;
    const float *row = vd_row(a, b, r) + first;
    float x[EPT];
    // element e of the lane: index 4 * (lane + 64 * (e / 4)) + e % 4, whole vectors where row and length allow them
    if ((reinterpret_cast<uintptr_t>(row) & 15) == 0) {
#pragma unroll
        for (int k = 0; k < EPT / 4; ++k) {
            const int i = 4 * (lane + 64 * k);
            f32x4_t v = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (i + 4 <= left) {
                v = __builtin_nontemporal_load(reinterpret_cast<const f32x4_t *>(row + i));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (i + e < left) v[e] = row[i + e];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * k + e] = v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < EPT; ++e) {
            const int i = 4 * (lane + 64 * (e / 4)) + e % 4;
            x[e] = i < left ? row[i] : -INFINITY;
        }
    }
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int e = 0; e < EPT; ++e) { nan |= x[e] != x[e]; m = fmaxf(m, x[e]); }
    m = wave_max(m);
    int arg = 0x7fffffff;
    if (ARG) {
#pragma unroll
        for (int e = EPT - 1; e >= 0; --e)
            if (x[e] == m) arg = 4 * (lane + 64 * (e / 4)) + e % 4;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const int other = __shfl_xor(arg, o, 64);
            arg = other < arg ? other : arg;
        }
    }
    double s = 0.0;
    if (SUMS) {
        const double md = m == -INFINITY ? 0.0 : (double)m, c = 1.4426950408889634074 / (a.temperature > 0 ? a.temperature : 1.0);
        const double least = -1020.0 / c;
        double s1 = 0.0;
#pragma unroll
        for (int e = 0; e < EPT; e += 2) {
            s += vd_exp(__builtin_fmax((double)x[e] - md, least), c);
            s1 += vd_exp(__builtin_fmax((double)x[e + 1] - md, least), c);
        }
        s = vd_wave_sum(s + s1);
    }
    nan = __any(nan);
    if (lane == 0) {
        VdWs w;
        vd_ws(a.ws, a.B, a.T, chunks, &w);
        const size_t cell = ((size_t)b * (2 * a.T + 1) + r) * chunks + chunk;
        w.max[cell] = m;
        w.arg[cell] = nan ? -1 : (arg < left ? arg + first : 0x7fffffff);
        w.sum[cell] = s;
    }
}

// What happens to sequence b, worked out by a whole workgroup (every thread returns it): rows joined from their chunks by 16 lanes
// each, then the first draft that is not accepted.  s_*: shared arrays of 2 T + 1 (T + 1 for s_arg) elements.
template <int THREADS>
__device__ VdDecision vd_decide(const VerifyArgs &a, const VdWs &w, int b, int chunks, bool sums, double *s_z, float *s_m, int *s_arg, int *s_stop) {
    const int n = vd_span(a, b), T = a.T, tid = threadIdx.x;
    const bool greedy = !(a.temperature > 0);
    const double c = 1.4426950408889634074 / (greedy ? 1.0 : a.temperature);
    const int rows = a.draft ? 2 * T + 1 : T + 1;
    if (tid == 0) *s_stop = n;
    // the first THREADS drafted tokens' logits travel while the rows are joined
    int x = -1;
    float xp = 0.f, xq = 0.f, u = 0.f;
    auto fetch = [&](int i) {
        x = a.drafts[(size_t)b * T + i];
        const bool in = x >= 0 && x < a.V;
        xp = in ? vd_row(a, b, i)[x] : -INFINITY;
        xq = in && a.draft ? vd_row(a, b, T + 1 + i)[x] : -INFINITY;
        u = greedy ? 0.f : a.u[(size_t)b * (T + 1) + i];
    };
    if (tid < n) fetch(tid);
    const int l = tid & 15;  // 16 lanes join the chunks of a row
    for (int r = tid >> 4; r < rows; r += THREADS / 16) {
        if (r <= T ? r > n : r - T - 1 >= n) continue;
        const size_t cell = ((size_t)b * (2 * T + 1) + r) * chunks;
        float m = -INFINITY;
        int arg = 0x7fffffff, bad = 0;
#pragma unroll 4
        for (int k = l; k < chunks; k += 16) {
            const float cm = w.max[cell + k];
            const int ca = w.arg[cell + k];
            bad |= ca < 0;
            if (cm > m || (cm == m && ca < arg)) { m = cm; arg = ca; }
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) {
            const float om = __shfl_xor(m, o, 64);
            const int oa = __shfl_xor(arg, o, 64);
            bad |= __shfl_xor(bad, o, 64);
            if (om > m || (om == m && oa < arg)) { m = om; arg = oa; }
        }
        const bool finite = fabsf(m) < INFINITY;
        double z = 0.0;
        if (sums && finite) {
#pragma unroll 4
            for (int k = l; k < chunks; k += 16) {
                const float cm = w.max[cell + k];
                z += cm == -INFINITY ? 0.0 : w.sum[cell + k] * vd_weight(cm, m, c);
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) z += __shfl_xor(z, o, 64);
        }
        if (l == 0) { s_m[r] = m; s_z[r] = z; s_arg[r] = bad || (!greedy && !finite) ? -1 : arg; }
    }
    __syncthreads();
    for (int i = tid; i < n; i += THREADS) {
        if (i != tid) fetch(i);
        bool go = s_arg[i] >= 0;
        if (greedy) {
            go = go && x == s_arg[i];
        } else if (go) {
            const bool in = x >= 0 && x < a.V;
            double q = 1.0;
            if (a.draft) {
                const int r = T + 1 + i;
                go = s_arg[r] >= 0;
                if (go) q = vd_weight(xq, s_m[r], c) / s_z[r];
            }
            go = go && in && (double)u * q < vd_weight(xp, s_m[i], c) / s_z[i];
        }
        if (!go) atomicMin(s_stop, i);
    }
    __syncthreads();
    VdDecision d;
    d.stop = *s_stop;
    d.bad = s_arg[d.stop] < 0 || (d.stop < n && a.draft && s_arg[T + 1 + d.stop] < 0);
    d.rejected = d.stop < n;
    d.token = d.rejected ? a.drafts[(size_t)b * T + d.stop] : -1;
    return d;
}

#define VD_MAX_ROWS (2 * 256 + 1)

// Weights max(0, p - q) of the rejected position, summed per chunk: a wavefront per chunk, four chunks per workgroup.  The decision is
// worked out in each workgroup (a launch of its own would cost more); the first of a sequence keeps it for the choice.
__global__ __launch_bounds__(VD_THREADS) void vd_residual_kernel(VerifyArgs a, int chunks, int chunk_len, int groups) {
    __shared__ double s_z[VD_MAX_ROWS];
    __shared__ float s_m[VD_MAX_ROWS];
    __shared__ int s_arg[VD_MAX_ROWS], s_stop;
    const int group = blockIdx.x % groups, b = blockIdx.x / groups, tid = threadIdx.x, lane = tid & 63, chunk = group * 4 + (tid >> 6);
    VdWs w;
    vd_ws(a.ws, a.B, a.T, chunks, &w);
    const VdDecision d = vd_decide<VD_THREADS>(a, w, b, chunks, true, s_z, s_m, s_arg, &s_stop);
    if (group == 0) {
        if (tid == 0) w.dec[b] = d;
        const int rows = 2 * a.T + 1;
        for (int r = tid; r < rows; r += VD_THREADS)
            if (r <= a.T ? r <= d.stop : r - a.T - 1 <= d.stop && d.rejected) {
                w.row_max[(size_t)b * rows + r] = s_m[r];
                w.row_sum[(size_t)b * rows + r] = s_z[r];
            }
    }
    if (d.bad || !d.rejected || chunk >= chunks) return;
    const int rp = d.stop, rq = a.T + 1 + d.stop;
    const double c = 1.4426950408889634074 / a.temperature, mp = s_m[rp], mq = s_m[rq], ip = 1.0 / s_z[rp], iq = 1.0 / s_z[rq];
    const float *prow = vd_row(a, b, rp), *qrow = vd_row(a, b, rq);
    const int first = chunk * chunk_len, last = first + chunk_len < a.V ? first + chunk_len : a.V;
    double s = 0.0;
    auto add = [&](float x, float y) {
        const double e = vd_weight(x, mp, c) * ip - vd_weight(y, mq, c) * iq;
        s += e > 0.0 ? e : 0.0;
    };
    const bool whole = ((reinterpret_cast<uintptr_t>(prow + first) | reinterpret_cast<uintptr_t>(qrow + first)) & 15) == 0;
    const int vectors = whole ? (last - first) / 4 : 0;
#pragma unroll 4
    for (int i = lane; i < vectors; i += 64) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(prow + first + 4 * i), y = *reinterpret_cast<const f32x4_t *>(qrow + first + 4 * i);
#pragma unroll
        for (int e = 0; e < 4; ++e) add(x[e], y[e]);
    }
#pragma unroll 4
    for (int v = first + 4 * vectors + lane; v < last; v += 64) add(prow[v], qrow[v]);
    s = vd_wave_sum(s);
    if (lane == 0) w.mass[(size_t)b * chunks + chunk] = s;
}

// The next token and the outputs: one workgroup per sequence.  DECIDE: no residual kernel ran (greedy, or drafts that were not
// sampled), so the decision is worked out here.
template <bool DECIDE, int PER>
__global__ __launch_bounds__(VD_PICK_THREADS) void vd_pick_kernel(VerifyArgs a, int chunks) {
    constexpr int WAVES = VD_PICK_THREADS / RL_WAVE, chunk_len = VD_PICK_THREADS * PER;
    __shared__ double s_z[VD_MAX_ROWS], s_red[WAVES], s_before, s_total, s_part;
    __shared__ float s_m[VD_MAX_ROWS];
    __shared__ int s_arg[VD_MAX_ROWS], s_stop, s_chunk, s_owner, s_next;
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, T = a.T, rows = 2 * T + 1;
    const bool greedy = !(a.temperature > 0), sums = !greedy || a.logp;
    const double c = 1.4426950408889634074 / (greedy ? 1.0 : a.temperature);
    VdWs w;
    vd_ws(a.ws, a.B, T, chunks, &w);
    VdDecision d;
    if (DECIDE) {
        d = vd_decide<VD_PICK_THREADS>(a, w, b, chunks, sums, s_z, s_m, s_arg, &s_stop);
    } else {
        d = w.dec[b];
        for (int r = tid; r < rows; r += VD_PICK_THREADS)
            if (r <= T ? r <= d.stop : r - T - 1 == d.stop && d.rejected) {
                s_m[r] = w.row_max[(size_t)b * rows + r];
                s_z[r] = w.row_sum[(size_t)b * rows + r];
            }
        __syncthreads();
    }
    const float *prow = vd_row(a, b, d.stop);
    int next = -1;
    if (!d.bad && greedy) {
        next = s_arg[d.stop];
    } else if (!d.bad) {
        const double mp = s_m[d.stop], ip = 1.0 / s_z[d.stop];
        const bool sampled = d.rejected && a.draft;
        const int rq = T + 1 + d.stop;
        const float *qrow = sampled ? vd_row(a, b, rq) : nullptr;
        const double mq = sampled ? (double)s_m[rq] : 0.0, iq = sampled ? 1.0 / s_z[rq] : 0.0;
        bool residual = d.rejected;
        auto weight_of = [&](int v, float xp, float xq) -> double {
            const double p = vd_weight(xp, mp, c) * ip;
            if (!residual) return p;
            if (!sampled) return v == d.token ? 0.0 : p;
            const double e = p - vd_weight(xq, mq, c) * iq;
            return e > 0.0 ? e : 0.0;
        };
        // a drafted token that was not sampled leaves its own chunk without its weight: that chunk is summed again
        const int own = residual && !sampled && d.token >= 0 && d.token < a.V ? d.token / chunk_len : -1;
        if (own >= 0) {
            const int last = (own + 1) * chunk_len < a.V ? (own + 1) * chunk_len : a.V;
            double s = 0.0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int v = own * chunk_len + tid + k * VD_PICK_THREADS;
                s += v < last ? weight_of(v, prow[v], 0.f) : 0.0;
            }
            s = vd_wave_sum(s);
            if (lane == 0) s_red[wv] = s;
            __syncthreads();
            if (tid == 0) {
                double t = 0.0;
                for (int k = 0; k < WAVES; ++k) t += s_red[k];
                s_part = t;
            }
            __syncthreads();
        }
        const size_t cell = ((size_t)b * rows + d.stop) * chunks;
        auto mass = [&](int k) -> double {
            if (residual && sampled) return w.mass[(size_t)b * chunks + k];
            if (residual && k == own) return s_part;
            const float cm = w.max[cell + k];
            return cm == -INFINITY ? 0.0 : w.sum[cell + k] * vd_weight(cm, mp, c) * ip;
        };
        // the chunk that the draw falls into: the first whose running sum exceeds it (the last with weight, should none by rounding)
        for (;;) {
            if (wv == 0) {
                double total = 0.0;
                for (int k0 = 0; k0 < chunks; k0 += 64) {
                    const double v = k0 + lane < chunks ? mass(k0 + lane) : 0.0;
                    total += vd_wave_sum(v);
                }
                if (lane == 0) s_total = total;
            }
            __syncthreads();
            if (!residual || s_total > 0.0) break;
            residual = false;  // p and q are the same: p itself
            __syncthreads();
        }
        const double target = (double)a.u[(size_t)b * (T + 1) + T] * s_total;
        if (wv == 0) {
            double before = 0.0, chosen_before = 0.0;
            int chosen = -1, lastk = 0;
            double last_before = 0.0;
            for (int k0 = 0; k0 < chunks && chosen < 0; k0 += 64) {
                const double v = k0 + lane < chunks ? mass(k0 + lane) : 0.0;
                double incl = v;
#pragma unroll
                for (int o = 1; o < 64; o <<= 1) {
                    const double up = __shfl_up(incl, o, 64);
                    if (lane >= o) incl += up;
                }
                const uint64_t over = __ballot(v > 0.0 && before + incl > target), some = __ballot(v > 0.0);
                if (some) {
                    const int l = 63 - __builtin_clzll(some);
                    lastk = k0 + l;
                    last_before = before + __shfl(incl - v, l, 64);
                }
                if (over) {
                    const int l = __builtin_ctzll(over);
                    chosen = k0 + l;
                    chosen_before = before + __shfl(incl - v, l, 64);
                }
                before += __shfl(incl, 63, 64);
            }
            if (lane == 0) {
                s_chunk = chosen >= 0 ? chosen : lastk;
                s_before = chosen >= 0 ? chosen_before : last_before;
                s_owner = VD_PICK_THREADS;
                s_next = -1;
            }
        }
        __syncthreads();
        // within the chunk: every thread owns consecutive tokens, their sums are scanned in order, the first thread whose running sum
        // exceeds the draw walks its own
        const int first = s_chunk * chunk_len, last = first + chunk_len < a.V ? first + chunk_len : a.V;
        const int i0 = first + tid * PER;
        float xp[PER], xq[PER];
        double e[PER], s = 0.0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int v = i0 + k < last ? i0 + k : last - 1;  // loads without conditions: all of them in flight
            xp[k] = prow[v];
            xq[k] = residual && sampled ? qrow[v] : 0.f;
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            e[k] = i0 + k < last ? weight_of(i0 + k, xp[k], xq[k]) : 0.0;
            s += e[k];
        }
        double incl = s;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const double up = __shfl_up(incl, o, 64);
            if (lane >= o) incl += up;
        }
        if (lane == 63) s_red[wv] = incl;
        __syncthreads();
        double before = s_before;
        for (int k = 0; k < wv; ++k) before += s_red[k];
        if (s > 0.0 && before + incl > target) atomicMin(&s_owner, tid);
        __syncthreads();
        if (tid == s_owner) {
            double run = before + incl - s;
            int pick = -1, last_pick = i0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                run += e[k];
                if (e[k] > 0.0) {
                    last_pick = i0 + k;
                    if (pick < 0 && run > target) pick = i0 + k;
                }
            }
            s_next = pick >= 0 ? pick : last_pick;
        } else if (s_owner == VD_PICK_THREADS && s > 0.0) {  // by rounding nobody's: the last token with weight
            int pick = i0;
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (e[k] > 0.0) pick = i0 + k;
            atomicMax(&s_next, pick);
        }
        __syncthreads();
        next = s_next;
    }
    int32_t *tokens = a.tokens + (size_t)b * (T + 1);
    float *logp = a.logp ? a.logp + (size_t)b * (T + 1) : nullptr;
    if (tid == 0) a.accepted[b] = d.stop;
    for (int i = tid; i <= T; i += VD_PICK_THREADS) {
        const int tok = i < d.stop ? a.drafts[(size_t)b * T + i] : (i == d.stop ? next : -1);
        tokens[i] = tok;
        if (logp) logp[i] = tok < 0 ? 0.f : (float)(((double)vd_row(a, b, i)[tok] - (double)s_m[i]) * (greedy ? 1.0 : 1.0 / a.temperature) - log(s_z[i]));
    }
}

// Logits per wavefront: 2048 where that still gives every compute unit a dozen wavefronts, else 512.
static int vd_chunk_len(int B, int T, int V) { return (int64_t)B * (T + 1) * ceil_div(V, 2048) >= 2048 ? 2048 : 512; }

size_t verify_drafts_ws_bytes(int B, int T, int V) { return vd_ws(nullptr, B, T, ceil_div(V, vd_chunk_len(B, T, V)), nullptr) + 8; }

template <int EPT>
static void vd_launch(const VerifyArgs &a, hipStream_t st) {
    constexpr int LEN = 64 * EPT, PER = LEN / VD_PICK_THREADS;
    const int chunks = ceil_div(a.V, LEN), rows = a.draft ? 2 * a.T + 1 : a.T + 1, groups = ceil_div(chunks, 4);
    const unsigned blocks = (unsigned)((int64_t)a.B * rows * groups);
    if (a.temperature > 0) vd_rows_kernel<EPT, true, false><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    else if (a.logp) vd_rows_kernel<EPT, true, true><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    else vd_rows_kernel<EPT, false, true><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    if (a.draft) {
        vd_residual_kernel<<<a.B * groups, VD_THREADS, 0, st>>>(a, chunks, LEN, groups);
        vd_pick_kernel<false, PER><<<a.B, VD_PICK_THREADS, 0, st>>>(a, chunks);
    } else {
        vd_pick_kernel<true, PER><<<a.B, VD_PICK_THREADS, 0, st>>>(a, chunks);
    }
}

void launch_verify_drafts(const VerifyArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    if (vd_chunk_len(a.B, a.T, a.V) == 2048) vd_launch<32>(a, st);
    else vd_launch<8>(a, st);
}
