// Verification of drafted tokens against the target's probabilities (rl_op_verify_drafts).
//
// With x a logits row, m its largest value and z = sum_v exp((x_v - m) / temperature), p_v = exp((x_v - m) / temperature) / z.  Every row
// is read once (vd_rows_kernel: maximum, its index, sum, per chunk of the vocabulary); a sequence's first rejection then
// follows from one probability pair per drafted token, and the next token from the weights max(0, p - q) or p of one row by inversion.
//
// A draw may land next to a border of the cumulative distribution, and a vocabulary of V tokens has V of them: weights with a
// relative error e move a draw to a neighbour with a probability of the order of V * e, about one in a hundred for fp32 (1e-7) and
// V = 128256.  So weights and sums are fp64: 2^g from a table of 128 powers in LDS and a polynomial of degree 3 for the rest
// (interpolation at the Chebyshev nodes, relative error 6e-13), 11 fp64 instructions per logit.  They take twice the time of fp32 ones and
// bound the reading of the rows (with a polynomial of degree 8 and no table, 15 of them): 4.9 TB/s, 6.3 TB/s for the maxima alone.
//
// Measured: 64 x 5 drafts, vocabulary 32000 (90 MB): 43 us, of it 22 for the rows, 5 for the decision, 7 for the weights of the rejected row
// and 9 for the token, the last three a chain of dependent loads each; 128 x up to 7 drafts, vocabulary 128256: 130 to 156 us with the lengths drawn, at 156
// rows 113, 10, 26, 10.  Drafts that were not sampled: 25 us for 64 x 5 of 32000, greedy 20.
#include "kernels.h"

#define VD_THREADS 256

// Over a wavefront: within rows of 16 lanes by DPP (lane ^ 1, lane ^ 2, mirrored half row, mirrored row), then across the four rows.
template <int CTRL>
__device__ __forceinline__ float vd_dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ double vd_dpp(double v) {
    return __hiloint2double(__builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xf, 0xf, true), __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ double vd_wave_sum(double v) {
    v += vd_dpp<0xb1>(v);
    v += vd_dpp<0x4e>(v);
    v += vd_dpp<0x141>(v);
    v += vd_dpp<0x140>(v);
    v += __shfl_xor(v, 16, 64);
    return v + __shfl_xor(v, 32, 64);
}
__device__ __forceinline__ float vd_wave_max(float v) {
    v = fmaxf(v, vd_dpp<0xb1>(v));
    v = fmaxf(v, vd_dpp<0x4e>(v));
    v = fmaxf(v, vd_dpp<0x141>(v));
    v = fmaxf(v, vd_dpp<0x140>(v));
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

static __device__ const double vd_pow2[128] = {  // 2^(k / 128)
    1.0, 1.0054299011128027, 1.0108892860517005, 1.016378314910953, 1.0218971486541166, 1.0274459491187637,
    1.0330248790212284, 1.0386341019613787, 1.0442737824274138, 1.0499440858006872, 1.0556451783605572, 1.061377227289262,
    1.0671404006768237, 1.0729348675259756, 1.0787607977571199, 1.0846183622133092, 1.0905077326652577, 1.0964290818163769,
    1.102382583307841, 1.1083684117236787, 1.1143867425958924, 1.1204377524096067, 1.1265216186082418, 1.1326385195987192,
    1.1387886347566916, 1.1449721444318042, 1.1511892299529827, 1.1574400736337511, 1.1637248587775775, 1.1700437696832502,
    1.1763969916502812, 1.182784710984341, 1.189207115002721, 1.1956643920398273, 1.202156731452703, 1.2086843236265816,
    1.215247359980469, 1.2218460329727576, 1.22848053610687, 1.2351510639369334, 1.241857812073484, 1.2486009771892048,
    1.255380757024691, 1.2621973503942507, 1.2690509571917332, 1.275941778396392, 1.2828700160787783, 1.2898358734066657,
    1.2968395546510096, 1.3038812651919358, 1.3109612115247644, 1.318079601266064, 1.3252366431597413, 1.3324325470831615,
    1.339667524053303, 1.3469417862329458, 1.3542555469368927, 1.3616090206382248, 1.3690024229745905, 1.3764359707545302,
    1.383909881963832, 1.3914243757719262, 1.3989796725383112, 1.4065759938190154, 1.4142135623730951, 1.4218926021691656,
    1.42961333839197, 1.4373759974489824, 1.4451808069770467, 1.4530279958490526, 1.460917794180647, 1.4688504333369818,
    1.4768261459394993, 1.4848451658727524, 1.4929077282912648, 1.5010140696264256, 1.5091644275934228, 1.5173590411982147,
    1.5255981507445384, 1.533881997840956, 1.5422108254079407, 1.550584877685, 1.559004400237837, 1.567469639965553,
    1.5759808451078865, 1.5845382652524937, 1.593142151342267, 1.6017927556826934, 1.6104903319492543, 1.6192351351948637,
    1.6280274218573478, 1.6368674497669644, 1.645755478153965, 1.6546917676561943, 1.6636765803267364, 1.6727101796415966,
    1.681792830507429, 1.6909247992693053, 1.7001063537185235, 1.709337763100463, 1.718619298122478, 1.7279512309618377,
    1.7373338352737062, 1.746767386199169, 1.7562521603732995, 1.7657884359332727, 1.7753764925265212, 1.785016611318935,
    1.7947090750031072, 1.804454167806624, 1.8142521755003989, 1.8241033854070534, 1.8340080864093424, 1.843966568958626,
    1.8539791250833855, 1.864046048397789, 1.8741676341103, 1.8843441790323345, 1.8945759815869656, 1.9048633418176741,
    1.9152065613971474, 1.925605943636125, 1.9360617934922943, 1.9465744175792332, 1.9571441241754002, 1.9677712232331759,
    1.978456026387951, 1.9891988469672663,
};

// The table in shared memory; every thread of the workgroup calls this, a barrier follows before its first use.
__device__ __forceinline__ void vd_table(double *pow2) {
    if (threadIdx.x < 128) pow2[threadIdx.x] = vd_pow2[threadIdx.x];
}
static constexpr double kVdLog2e = 1.4426950408889634074 * 128;  // exponents are counted in 128ths
static constexpr double kVdLeast = -1020.0 * 128;                // weights below 2^-1020 of the largest count as zero

// 2^(d c / 128) for kVdLeast <= d c <= 128000 (c = kVdLog2e / temperature: VerifyArgs::rate, from the host, since two fp64 divisions cost a
// wavefront as much as eight logits).
__device__ __forceinline__ double vd_exp(double d, double c, const double *pow2) {
    const double magic = 6755399441055744.0;  // 1.5 * 2^52: adding it leaves the nearest integer in the low bits
    const double t = __builtin_fma(d, c, magic);
    const double f = __builtin_fma(d, c, magic - t);
    const int n = __double2loint(t);
    const double p = pow2[n & 127];
    const double q = f * __builtin_fma(f, __builtin_fma(f, 2.6466428720412216e-08, 1.4662269105827228e-05), 0.0054152123481245725);
    const double s = __hiloint2double(__double2hiint(p) + ((n & ~127) << 13), __double2loint(p));
    return __builtin_fma(s, q, s);
}
// The weight of a logit x next to the largest one m; 0 for x = -inf.
__device__ __forceinline__ double vd_weight(float x, double m, const VerifyArgs &a, const double *pow2) {
    const double d = (double)x - m;
    const double w = vd_exp(__builtin_fmax(d, a.least), a.rate, pow2);
    return d >= a.least ? w : 0.0;
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

// One wavefront per (row, chunk of 64 * EPT logits), four chunks of a row per workgroup: the logits stay in registers between the maximum
// and the weights, which refer to the chunk's own maximum.  SUMS, ARG: whether the sum and the index of the maximum are wanted (sampled: sums; greedy: the index, and sums for
// log-probabilities).
template <int EPT, bool SUMS, bool ARG>
__global__ __launch_bounds__(VD_THREADS, 8) void vd_rows_kernel(VerifyArgs a, int chunks, int rows, int groups) {
    const unsigned id = blockIdx.x / groups;
    const int chunk = (int)(blockIdx.x % groups) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int r = (int)(id % rows), b = (int)(id / rows);
    __shared__ double pow2[128];
    const int n = vd_span(a, b);
    if (r <= a.T ? r > n : r - a.T - 1 >= n) return;  // not reached in any case
    const int first = chunk * (64 * EPT);
    const int left = a.V - first < 64 * EPT ? a.V - first : 64 * EPT;  // none for a wavefront behind the last chunk
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
    if (SUMS) {
        vd_table(pow2);
        __syncthreads();
    }
    if (chunk >= chunks) return;
    float m = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int e = 0; e < EPT; ++e) { nan |= x[e] != x[e]; m = fmaxf(m, x[e]); }
    m = vd_wave_max(m);
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
        const double md = m == -INFINITY ? 0.0 : (double)m;
        double s1 = 0.0;
#pragma unroll
        for (int e = 0; e < EPT; e += 2) {
            s += vd_exp(__builtin_fmax((double)x[e] - md, a.least), a.rate, pow2);
            s1 += vd_exp(__builtin_fmax((double)x[e + 1] - md, a.least), a.rate, pow2);
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
__device__ VdDecision vd_decide(const VerifyArgs &a, const VdWs &w, int b, int chunks, bool sums, const double *pow2, double *s_z, float *s_m, int *s_arg,
                                int *s_stop) {
    const int n = vd_span(a, b), T = a.T, tid = threadIdx.x;
    const bool greedy = !(a.temperature > 0);
    const int rows = a.draft ? 2 * T + 1 : T + 1;
    if (tid == 0) *s_stop = n;
    __syncthreads();  // the table as well
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
                z += cm == -INFINITY ? 0.0 : w.sum[cell + k] * vd_weight(cm, m, a, pow2);
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
                if (go) q = vd_weight(xq, s_m[r], a, pow2) / s_z[r];
            }
            go = go && in && (double)u * q < vd_weight(xp, s_m[i], a, pow2) / s_z[i];
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

// The decision of a sequence, and the maxima and sums that the choice needs, once per sequence.
__global__ __launch_bounds__(VD_THREADS) void vd_decide_kernel(VerifyArgs a, int chunks) {
    __shared__ double s_z[VD_MAX_ROWS], pow2[128];
    __shared__ float s_m[VD_MAX_ROWS];
    __shared__ int s_arg[VD_MAX_ROWS], s_stop;
    const int b = blockIdx.x, tid = threadIdx.x, rows = 2 * a.T + 1;
    VdWs w;
    vd_ws(a.ws, a.B, a.T, chunks, &w);
    vd_table(pow2);
    const VdDecision d = vd_decide<VD_THREADS>(a, w, b, chunks, true, pow2, s_z, s_m, s_arg, &s_stop);
    if (tid == 0) w.dec[b] = d;
    for (int r = tid; r < rows; r += VD_THREADS)
        if (r <= a.T ? r <= d.stop : r - a.T - 1 == d.stop && d.rejected) {
            w.row_max[(size_t)b * rows + r] = s_m[r];
            w.row_sum[(size_t)b * rows + r] = s_z[r];
        }
}

// Weights max(0, p - q) of the rejected position, summed per chunk: one workgroup per chunk, PER logits of either row a thread.
template <int PER>
__global__ __launch_bounds__(VD_THREADS) void vd_residual_kernel(VerifyArgs a, int chunks) {
    constexpr int chunk_len = VD_THREADS * PER;
    __shared__ double pow2[128], s_sum[4];
    const int chunk = blockIdx.x % chunks, b = blockIdx.x / chunks, tid = threadIdx.x;
    VdWs w;
    vd_ws(a.ws, a.B, a.T, chunks, &w);
    vd_table(pow2);
    const VdDecision d = w.dec[b];
    if (d.bad || !d.rejected) return;
    const int rp = d.stop, rq = a.T + 1 + d.stop;
    const float *prow = vd_row(a, b, rp), *qrow = vd_row(a, b, rq);
    const int first = chunk * chunk_len, last = first + chunk_len < a.V ? first + chunk_len : a.V;
    float x[PER], y[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int v = first + tid + k * VD_THREADS < last ? first + tid + k * VD_THREADS : last - 1;
        x[k] = prow[v];
        y[k] = qrow[v];
    }
    const size_t row0 = (size_t)b * (2 * a.T + 1);
    const double mp = w.row_max[row0 + rp], mq = w.row_max[row0 + rq], ip = 1.0 / w.row_sum[row0 + rp], iq = 1.0 / w.row_sum[row0 + rq];
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const double e = vd_weight(x[k], mp, a, pow2) * ip - vd_weight(y[k], mq, a, pow2) * iq;
        s += e > 0.0 && first + tid + k * VD_THREADS < last ? e : 0.0;
    }
    s = vd_wave_sum(s);
    if ((tid & 63) == 0) s_sum[tid >> 6] = s;
    __syncthreads();
    if (tid == 0) w.mass[(size_t)b * chunks + chunk] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// The next token and the outputs: one workgroup per sequence; its four wavefronts work out the chunk of the draw each for itself.
// DECIDE: greedy, or drafts that were not sampled: no kernel decided before.
template <bool DECIDE, int PER>
__global__ __launch_bounds__(VD_THREADS) void vd_pick_kernel(VerifyArgs a, int chunks) {
    constexpr int chunk_len = VD_THREADS * PER;
    __shared__ double s_z[VD_MAX_ROWS], pow2[128], s_own[4], s_red[4];
    __shared__ float s_m[VD_MAX_ROWS];
    __shared__ int s_arg[VD_MAX_ROWS], s_stop, s_first[4], s_last[4];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, T = a.T, rows = 2 * T + 1;
    const bool greedy = !(a.temperature > 0), sums = !greedy || a.logp;
    VdWs w;
    vd_ws(a.ws, a.B, T, chunks, &w);
    vd_table(pow2);
    // the accepted tokens are put out last, by the wavefronts behind the first: their loads travel with the others
    int at = tid - 64, tok = at >= 0 && at < T ? a.drafts[(size_t)b * T + at] : -1;
    const float u = greedy ? 0.f : a.u[(size_t)b * (T + 1) + T];
    VdDecision d;
    if (DECIDE) {
        d = vd_decide<VD_THREADS>(a, w, b, chunks, sums, pow2, s_z, s_m, s_arg, &s_stop);
    } else {
        d = w.dec[b];
        for (int r = tid; r < rows; r += VD_THREADS)
            if (r <= T ? r <= d.stop : r - T - 1 == d.stop && d.rejected) {
                s_m[r] = w.row_max[(size_t)b * rows + r];
                s_z[r] = w.row_sum[(size_t)b * rows + r];
            }
        __syncthreads();
    }
    int32_t *tokens = a.tokens + (size_t)b * (T + 1);
    float *logp = a.logp ? a.logp + (size_t)b * (T + 1) : nullptr;
    auto put = [&](int i, int tok, float x) {     // x: the token's logit
        tokens[i] = tok;
        if (logp) logp[i] = tok < 0 ? 0.f : (float)(((double)x - (double)s_m[i]) * (greedy ? 1.0 : 1.0 / a.temperature) - log(s_z[i]));
    };
    auto logit = [&](int i, int tok) { return logp && tok >= 0 ? vd_row(a, b, i)[tok] : 0.f; };
    if (at >= d.stop) tok = -1;
    const float x_tok = at >= 0 ? logit(at, tok) : 0.f;
    if (tid == 0) a.accepted[b] = d.stop;
    auto put_others = [&] {
        if (at >= 0 && at <= T && at != d.stop) put(at, tok, x_tok);
        for (int i = at + VD_THREADS - 64; at >= 0 && i <= T; i += VD_THREADS - 64) {
            const int t = i < d.stop ? a.drafts[(size_t)b * T + i] : -1;
            if (i != d.stop) put(i, t, logit(i, t));
        }
    };
    if (d.bad || greedy) {
        const int next = d.bad ? -1 : s_arg[d.stop];
        if (tid == 0) put(d.stop, next, logit(d.stop, next));
        put_others();
        return;
    }

    const float *prow = vd_row(a, b, d.stop);
    const double mp = s_m[d.stop], ip = 1.0 / s_z[d.stop];
    const bool sampled = d.rejected && a.draft;
    const int rq = T + 1 + d.stop;
    const float *qrow = sampled ? vd_row(a, b, rq) : prow;
    const double mq = sampled ? (double)s_m[rq] : 0.0, iq = sampled ? 1.0 / s_z[rq] : 0.0;
    bool residual = d.rejected;
    auto weight_of = [&](int v, float xp, float xq) -> double {
        const double p = vd_weight(xp, mp, a, pow2) * ip;
        if (!residual) return p;
        if (!sampled) return v == d.token ? 0.0 : p;
        const double e = p - vd_weight(xq, mq, a, pow2) * iq;
        return e > 0.0 ? e : 0.0;
    };
    // a drafted token that was not sampled leaves its own chunk without its weight: that chunk is summed again
    const int own = residual && !sampled && d.token >= 0 && d.token < a.V ? d.token / chunk_len : -1;
    double own_mass = 0.0;
    if (own >= 0) {
        const int first = own * chunk_len, last = first + chunk_len < a.V ? first + chunk_len : a.V;
        float x[PER];
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int v = first + tid + k * VD_THREADS;
            x[k] = prow[v < last ? v : last - 1];
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int v = first + tid + k * VD_THREADS;
            s += v < last ? weight_of(v, x[k], 0.f) : 0.0;
        }
        s = vd_wave_sum(s);
        if (lane == 0) s_own[wv] = s;
        __syncthreads();
        own_mass = s_own[0] + s_own[1] + s_own[2] + s_own[3];
    }
    const size_t cell = ((size_t)b * rows + d.stop) * chunks;
    auto mass = [&](int k) -> double {
        if (residual && sampled) return w.mass[(size_t)b * chunks + k];
        if (residual && k == own) return own_mass;
        const float cm = w.max[cell + k];
        return cm == -INFINITY ? 0.0 : w.sum[cell + k] * vd_weight(cm, mp, a, pow2) * ip;
    };
    double total, v0;                             // v0: of the first 64 chunks, kept
    for (;;) {
        v0 = lane < chunks ? mass(lane) : 0.0;
        total = vd_wave_sum(v0);
        for (int k0 = 64; k0 < chunks; k0 += 64) total += vd_wave_sum(k0 + lane < chunks ? mass(k0 + lane) : 0.0);
        if (!residual || total > 0.0) break;
        residual = false;  // p and q are the same: p itself
    }
    const double target = (double)u * total;
    // the chunk that the draw falls into: the first whose running sum exceeds it (the last with weight, should none by rounding)
    int chosen = 0;
    double before = 0.0;
    {
        double run = 0.0;
        for (int k0 = 0; k0 < chunks; k0 += 64) {
            const double v = k0 == 0 ? v0 : k0 + lane < chunks ? mass(k0 + lane) : 0.0;
            double incl = v;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const double up = __shfl_up(incl, o, 64);
                if (lane >= o) incl += up;
            }
            const uint64_t over = __ballot(v > 0.0 && run + incl > target), some = __ballot(v > 0.0);
            if (some) {
                const int l = over ? __builtin_ctzll(over) : 63 - __builtin_clzll(some);
                chosen = k0 + l;
                before = run + __shfl(incl - v, l, 64);
            }
            if (over) break;
            run += __shfl(incl, 63, 64);
        }
    }
    // within the chunk: every thread owns consecutive tokens, their sums are scanned in order, the first thread whose running sum
    // exceeds the draw walks its own
    const int first = chosen * chunk_len, last = first + chunk_len < a.V ? first + chunk_len : a.V, i0 = first + tid * PER;
    float xp[PER], xq[PER];
    double e[PER], s = 0.0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int v = i0 + k < last ? i0 + k : last - 1;  // loads without conditions: all of them in flight
        xp[k] = prow[v];
        xq[k] = qrow[v];
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
    for (int k = 0; k < wv; ++k) before += s_red[k];
    const uint64_t over = __ballot(s > 0.0 && before + incl > target), some = __ballot(s > 0.0);
    double run = before + incl - s;
    int pick = -1, last_pick = -1;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        run += e[k];
        if (e[k] > 0.0) {
            last_pick = i0 + k;
            if (pick < 0 && run > target) pick = i0 + k;
        }
    }
    if (pick < 0) pick = last_pick;
    // of the wavefront: the token of its first thread over the draw, and of its last thread with weight
    const int mine = over ? __builtin_amdgcn_readlane(pick, (int)__builtin_ctzll(over)) : -1;
    const int rest = some ? __builtin_amdgcn_readlane(last_pick, 63 - (int)__builtin_clzll(some)) : -1;
    if (lane == 0) { s_first[wv] = mine; s_last[wv] = rest; }
    __syncthreads();
    if (tid == 0) {
        int next = -1;
        for (int k = 3; k >= 0; --k)
            if (s_first[k] >= 0) next = s_first[k];
        for (int k = 3; k >= 0 && next < 0; --k) next = s_last[k];  // by rounding nobody's: the last token with weight
        put(d.stop, next, logit(d.stop, next));
    }
    put_others();
}

// Logits per wavefront: 512 where 2048 would leave a compute unit less than four wavefronts and a sequence has few chunks to join, else
// 2048.  With 512 and 2048: 1 x 3 drafts, vocabulary 1024: 17.1 and 19.3 us; 8 x 5, 32000: 23.6 and 24.3; 16 x 5, 32000: 27.4 and 26.5; 64 x 5, 32000:
// 50.8 and 43.2; and where a workgroup joins more than 512 chunks: 2 x 16, 32000: 30.8 and 26.8; 1 x 4, 128256: 31.6 and 22.9.
static int vd_chunk_len(int B, int T, int V) {
    return (int64_t)B * (T + 1) * ceil_div(V, 2048) < 1024 && (int64_t)(T + 1) * ceil_div(V, 512) <= 512 ? 512 : 2048;
}

size_t verify_drafts_ws_bytes(int B, int T, int V) { return vd_ws(nullptr, B, T, ceil_div(V, vd_chunk_len(B, T, V)), nullptr) + 8; }

// Chunks of 512 appear as a batch shrinks: for every number of tokens, the largest batch that takes them.
size_t verify_drafts_ws_bytes_up_to(int B, int T, int V) {
    size_t most = vd_ws(nullptr, B, T, ceil_div(V, 2048), nullptr) + 8;
    for (int t = 1; t <= T; ++t) {
        const int64_t per = (int64_t)(t + 1) * ceil_div(V, 2048);
        const int b = (int)(1023 / per < B ? 1023 / per : B);
        if (b < 1) break;
        const size_t n = verify_drafts_ws_bytes(b, t, V);
        most = n > most ? n : most;
    }
    return most;
}

bool verify_drafts_grid_fits(int B, int T, int V, bool draft) {
    const int chunks = ceil_div(V, vd_chunk_len(B, T, V));
    return grid_fits((int64_t)B * (draft ? 2 * T + 1 : T + 1) * ceil_div(chunks, 4), VD_THREADS) && grid_fits((int64_t)B * chunks, VD_THREADS);
}

template <int EPT>
static void vd_launch(const VerifyArgs &a, hipStream_t st) {
    constexpr int LEN = 64 * EPT, PER = LEN / VD_THREADS;
    const int chunks = ceil_div(a.V, LEN), rows = a.draft ? 2 * a.T + 1 : a.T + 1, groups = ceil_div(chunks, 4);
    const unsigned blocks = (unsigned)((int64_t)a.B * rows * groups);
    if (a.temperature > 0) vd_rows_kernel<EPT, true, false><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    else if (a.logp) vd_rows_kernel<EPT, true, true><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    else vd_rows_kernel<EPT, false, true><<<blocks, VD_THREADS, 0, st>>>(a, chunks, rows, groups);
    if (a.draft) {
        vd_decide_kernel<<<a.B, VD_THREADS, 0, st>>>(a, chunks);
        vd_residual_kernel<PER><<<a.B * chunks, VD_THREADS, 0, st>>>(a, chunks);
        vd_pick_kernel<false, PER><<<a.B, VD_THREADS, 0, st>>>(a, chunks);
    } else {
        vd_pick_kernel<true, PER><<<a.B, VD_THREADS, 0, st>>>(a, chunks);
    }
}

void launch_verify_drafts(const VerifyArgs &a0, hipStream_t st) {
    VerifyArgs a = a0;
    if (a.B <= 0) return;
    a.rate = kVdLog2e / (a.temperature > 0 ? a.temperature : 1.0);
    a.least = kVdLeast / a.rate;
    if (vd_chunk_len(a.B, a.T, a.V) == 2048) vd_launch<32>(a, st);
    else vd_launch<8>(a, st);
}
