// Eviction from a cache by accumulated attention weight (rl_op_evict_rows): which rows of a (sequence, kv head) slab stay, and the
// moves that bring them below slot `keep`.
#include "kernels.h"

#define EV_THREADS 1024
#define EV_WAVES (EV_THREADS / RL_WAVE)

// Order-preserving image of a weight: larger weight, larger number.  -0 counts as 0, NaN as minus infinity.
__device__ __forceinline__ uint32_t ev_key(float w) {
    w = w != w ? -INFINITY : w + 0.f;
    const uint32_t u = __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Workspace of a slab: int32 count, then pairs (free slot, row that moves there).
__device__ __forceinline__ int32_t *ev_list(const EvictArgs &a, int slab) { return a.moves + (size_t)slab * (2 + 2 * (size_t)a.max_moves); }

// Exclusive prefix sum over the workgroup's threads; *total receives the sum.
__device__ __forceinline__ int ev_scan(int v, int *red, int *total) {
    const int lane = threadIdx.x & 63, wv = threadIdx.x >> 6;
    int incl = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int up = __shfl_up(incl, o, 64);
        if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == 63) red[wv] = incl;
    __syncthreads();
    int base = 0, sum = 0;
    for (int w = 0; w < EV_WAVES; ++w) { if (w < wv) base += red[w]; sum += red[w]; }
    *total = sum;
    return base + incl - v;
}

// One workgroup per slab.  The keep-th largest key by four rounds of 256 bins; rows above it stay, of those equal to it the first
// in slot order.
__global__ __launch_bounds__(EV_THREADS) void evict_select_kernel(EvictArgs a) {
    __shared__ int bins[256], red[EV_WAVES];
    __shared__ int s_max;
    __shared__ uint32_t s_key;
    __shared__ int s_need;
    const int slab = blockIdx.x, b = slab / a.Hkv, tid = threadIdx.x;
    int n = a.d_len[b];
    n = n < 0 ? 0 : (n > a.S ? a.S : n);
    const float *w = a.weight + (size_t)slab * a.S;
    const int32_t *pos = a.pos ? a.pos + (size_t)slab * a.S : nullptr;
    float *wo = a.weight_out + (size_t)slab * a.S;
    int32_t *po = a.pos ? a.pos_out + (size_t)slab * a.S : nullptr;
    int32_t *list = ev_list(a, slab);
    const int stay = n < a.keep ? n : a.keep;
    if (n <= a.keep) {
        if (tid == 0) list[0] = 0;
        if (wo != w) for (int j = tid; j < stay; j += EV_THREADS) wo[j] = w[j];
        if (pos && po != pos) for (int j = tid; j < stay; j += EV_THREADS) po[j] = pos[j];
        return;
    }
    int newest = INT32_MIN;
    if (pos) {
        for (int j = tid; j < n; j += EV_THREADS) newest = newest > pos[j] ? newest : pos[j];
        if (tid == 0) s_max = INT32_MIN;
        __syncthreads();
        atomicMax(&s_max, newest);
        __syncthreads();
        newest = s_max;
    } else {
        newest = n - 1;
    }
    const int64_t cut = (int64_t)newest - a.recent;
    auto key_of = [&](int j) -> uint32_t { return (int64_t)(pos ? pos[j] : j) > cut ? 0xffffffffu : ev_key(w[j]); };
    uint32_t prefix = 0, mask = 0;
    int need = a.keep;
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) bins[tid] = 0;
        __syncthreads();
        for (int j = tid; j < n; j += EV_THREADS) {
            const uint32_t k = key_of(j);
            if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & 255], 1);
        }
        __syncthreads();
        if (tid == 0) {
            int left = need, v = 255;
            for (; v > 0 && bins[v] < left; --v) left -= bins[v];
            s_key = prefix | ((uint32_t)v << shift);
            s_need = left;
        }
        __syncthreads();
        prefix = s_key;
        need = s_need;
        mask |= 0xffu << shift;
        __syncthreads();
    }
    // two walks in slot order: free slots below keep, staying rows above
    int ties = 0, holes = 0, fillers = 0;
    for (int j0 = 0; j0 < n; j0 += EV_THREADS) {
        const int j = j0 + tid;
        const uint32_t k = j < n ? key_of(j) : 0u;
        const bool tie = j < n && k == prefix;
        int sum;
        const int rank = ties + ev_scan(tie, red, &sum);
        ties += sum;
        const bool stays = j < n && (k > prefix || (tie && rank < need));
        const bool hole = j < a.keep && j < n && !stays, filler = j >= a.keep && stays;
        const int hr = holes + ev_scan(hole, red, &sum);
        holes += sum;
        const int fr = fillers + ev_scan(filler, red, &sum);
        fillers += sum;
        if (hole) list[2 + 2 * hr] = j;
        if (filler) list[2 + 2 * fr + 1] = j;
    }
    if (tid == 0) list[0] = holes;
    __syncthreads();
    if (wo != w) for (int j = tid; j < stay; j += EV_THREADS) wo[j] = w[j];
    if (pos && po != pos) for (int j = tid; j < stay; j += EV_THREADS) po[j] = pos[j];
    __syncthreads();
    for (int i = tid; i < holes; i += EV_THREADS) {
        const int to = list[2 + 2 * i], of = list[2 + 2 * i + 1];
        wo[to] = w[of];
        if (pos) po[to] = pos[of];
    }
}

// One wavefront per (slab, group of moves): K row, V row and their scales.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int slab = blockIdx.x, b = slab / a.Hkv, kvh = slab % a.Hkv, lane = threadIdx.x & 63;
    const int32_t *list = ev_list(a, slab);
    const int count = list[0], piece = a.hd / 8;  // 16-byte pieces of a row
    if (a.d_len_out && kvh == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        int n = a.d_len[b];
        n = n < 0 ? 0 : (n > a.S ? a.S : n);
        a.d_len_out[b] = n < a.keep ? n : a.keep;
    }
    for (int i = blockIdx.y * 4 + (threadIdx.x >> 6); i < count; i += gridDim.y * 4) {
        const size_t to = kv_row_index(a.map, b, kvh, a.Hkv, a.S, list[2 + 2 * i]), of = kv_row_index(a.map, b, kvh, a.Hkv, a.S, list[2 + 2 * i + 1]);
        if (lane < 2 * piece) {
            f16_t *c = lane < piece ? a.kc : a.vc;
            const int e = (lane < piece ? lane : lane - piece) * 8;
            *reinterpret_cast<u32x4_t *>(c + to * a.hd + e) = *reinterpret_cast<const u32x4_t *>(c + of * a.hd + e);
        } else if (a.map.kscale && lane < 2 * piece + 2) {
            float *s = lane == 2 * piece ? a.map.kscale : a.map.vscale;
            s[to] = s[of];
        }
    }
}

size_t evict_rows_ws_bytes(int B, int Hkv, int S, int keep) {
    const int64_t moves = keep < S - keep ? keep : S - keep;
    return (size_t)B * Hkv * (2 + 2 * (size_t)(moves < 0 ? 0 : moves)) * sizeof(int32_t);
}

void launch_evict_rows(const EvictArgs &a0, hipStream_t st) {
    EvictArgs a = a0;
    if (a.B <= 0) return;
    a.max_moves = a.keep < a.S - a.keep ? a.keep : a.S - a.keep;
    evict_select_kernel<<<a.B * a.Hkv, EV_THREADS, 0, st>>>(a);
    int groups = ceil_div(a.max_moves, 16);
    if (groups < 1) groups = 1;
    if (groups > 64) groups = 64;
    evict_move_kernel<<<dim3(a.B * a.Hkv, groups), 256, 0, st>>>(a);
}
