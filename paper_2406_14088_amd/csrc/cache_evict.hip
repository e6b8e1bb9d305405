// Eviction from a cache by accumulated attention weight (rl_op_evict_rows): which rows of a (sequence, kv head) slab stay, and the
// moves that bring them below slot `keep`.
//
// One workgroup per slab holds the slab's weights in registers, as unsigned keys whose order is that of the rows (recent rows above every
// weight); a wavefront owns consecutive rows.  The keep-th largest key is found by counting keys in 256 bins of its interval and going on
// with the bin it falls into; the interval starts between the least and the largest key of the slab, so that the bins are used, and a round
// that splits off exactly `keep` rows is the last: two rounds as a rule, five at most, when ties at the threshold go to the lowest
// slots.  (15 pivots a round counted by ballots took three times as long: the instructions of 16 wavefronts, not latency.)
// Free slots below `keep` and staying rows above it are numbered by ballots and one sum over wavefronts; the j-th of the one takes the
// j-th of the other, so a step that appended a few rows moves at most as many, whatever the cache holds.  Sources lie above `keep`
// and targets below, so the moves need no order.  A slab's latency is what counts (three dependent loads, about twelve barriers)
// until many rows move.
//
// Measured: 48 x 8 slabs of 2112 rows of 128 halves down to 2048, 15 us (34 MB, of which the rows that move are 18); 8 x 32 slabs of 8000
// block-scaled rows in pages of 64 down to 1000, 77 us (262 MB read and written: the selection takes 20, the moves 4.6 TB/s).
#include "kernels.h"

// Order-preserving image of a weight: larger weight, larger number.  -0 counts as 0, NaN as minus infinity.
__device__ __forceinline__ uint32_t ev_key(float w) {
    w = w != w ? -INFINITY : w + 0.f;
    const uint32_t u = __float_as_uint(w);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
static constexpr uint32_t kEvRecent = 0xffffffffu;  // above the key of every weight; 0: no row (below every weight)

// Workspace of a slab (where another kernel moves the rows): int32 count, unused, then pairs (free slot, row that moves there).
__device__ __forceinline__ int32_t *ev_list(const EvictArgs &a, int slab) { return a.moves + (size_t)slab * (2 + 2 * (size_t)a.max_moves); }

__device__ __forceinline__ int ev_len(const EvictArgs &a, int b) {
    const int n = a.d_len[b];
    return n < 0 ? 0 : (n > a.S ? a.S : n);
}

// Rows of a slab, `part` of `parts` equal parts of its moves: K and V row and, block-scaled, their scales.  lanes_per_row = 2 * hd / 8.
template <typename PAIR>
__device__ __forceinline__ void ev_move(const EvictArgs &a, int b, int kvh, int count, int wave, int waves, PAIR pair) {
    const int lane = threadIdx.x & 63, piece = a.hd / 8, lpr = 2 * piece, rpw = 64 / lpr;  // 16-byte pieces of a row; lanes of a (K, V) pair; rows at once
    const int sub = lane / lpr, l = lane % lpr;
    f16_t *c = l < piece ? a.kc : a.vc;
    const int e = (l < piece ? l : l - piece) * 8;
    constexpr int U = 4;
    for (int i0 = (wave * U) * rpw; i0 < count; i0 += waves * U * rpw) {
        size_t to[U], of[U];
        u32x4_t x[U];
        bool on[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u * rpw + sub;
            on[u] = i < count;
            if (on[u]) {
                int t, f;
                pair(i, &t, &f);
                to[u] = kv_row_index(a.map, b, kvh, a.Hkv, a.S, t);
                of[u] = kv_row_index(a.map, b, kvh, a.Hkv, a.S, f);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on[u]) x[u] = *reinterpret_cast<const u32x4_t *>(c + of[u] * a.hd + e);
        if (a.map.kscale && (l == 0 || l == piece)) {
            float *s = l == 0 ? a.map.kscale : a.map.vscale, y[U];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (on[u]) y[u] = s[of[u]];
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (on[u]) s[to[u]] = y[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (on[u]) *reinterpret_cast<u32x4_t *>(c + to[u] * a.hd + e) = x[u];
    }
}

// Sum, least and largest over a wavefront.
__device__ __forceinline__ int ev_wave_sum(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
template <typename T>
__device__ __forceinline__ T ev_wave_max(T v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const T x = __shfl_xor(v, o, 64);
        v = x > v ? x : v;
    }
    return v;
}

// THREADS threads with REGS rows each in registers.  REGS == 0: slabs of any length, the keys are read again whenever they are needed.
template <int THREADS, int REGS>
__device__ __forceinline__ void ev_slab(const EvictArgs &a, int slab, int n, bool move, int *s_bin, int *s_misc, uint16_t *s_hole, uint16_t *s_fill) {
    constexpr int WAVES = THREADS / RL_WAVE, N = REGS ? REGS : 1;
    const int b = slab / a.Hkv, kvh = slab % a.Hkv, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const float *w = a.weight + (size_t)slab * a.S;
    const int32_t *pos = a.pos ? a.pos + (size_t)slab * a.S : nullptr;
    float *wo = a.weight_out + (size_t)slab * a.S;
    int32_t *po = a.pos ? a.pos_out + (size_t)slab * a.S : nullptr;
    const int steps = (n + THREADS - 1) / THREADS;   // of 64 rows per wavefront
    const int j0 = wave * steps * 64 + lane;         // this lane's rows: j0 + 64 k, k < steps
    auto for_rows = [&](auto f) {                    // f(k); unrolled where the rows are in registers
        if (REGS) {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k < steps) f(k);
        } else {
            for (int k = 0; k < steps; ++k) f(k);
        }
    };
    float wr[N];
    int32_t pr[N];
    uint32_t kr[N];

    // ---- rows into registers, the newest position
    if (REGS) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const int j = j0 + 64 * k;
            wr[k] = 0.f; pr[k] = INT32_MIN;
            if (k < steps && j < n) {
                wr[k] = w[j];
                if (pos) pr[k] = pos[j];
            }
        }
    }
    int newest = n - 1;
    if (pos) {
        newest = INT32_MIN;
        for_rows([&](int k) {
            const int j = j0 + 64 * k, p = REGS ? pr[REGS ? k : 0] : (j < n ? pos[j] : INT32_MIN);
            newest = p > newest ? p : newest;
        });
        newest = ev_wave_max(newest);
        if (lane == 0) s_misc[wave] = newest;
        __syncthreads();
        newest = ev_wave_max(s_misc[lane & (WAVES - 1)]);
    }
    const int64_t cut = (int64_t)newest - a.recent;
    auto make_key = [&](int j, float x, int32_t p) -> uint32_t { return j >= n ? 0u : ((int64_t)(pos ? p : j) > cut ? kEvRecent : ev_key(x)); };
    auto key = [&](int k) -> uint32_t {
        if (REGS) return kr[REGS ? k : 0];
        const int j = j0 + 64 * k;
        return j < n ? make_key(j, w[j], pos ? pos[j] : 0) : 0u;
    };
    if (REGS) {
#pragma unroll
        for (int k = 0; k < N; ++k) kr[k] = make_key(j0 + 64 * k, wr[k], pr[k]);
    }

    // ---- recent rows, least and largest key of the others
    int recent = 0;
    uint32_t kmax = 0u, kmin_inv = 0u;
    for_rows([&](int k) {
        const uint32_t x = key(k);
        recent += __popcll(__ballot(x == kEvRecent));
        const bool plain = x != 0u && x != kEvRecent;
        kmin_inv = plain && ~x > kmin_inv ? ~x : kmin_inv;
        kmax = plain && x > kmax ? x : kmax;
    });
    kmin_inv = ev_wave_max(kmin_inv);
    kmax = ev_wave_max(kmax);
    if (lane == 0) { s_misc[16 + wave] = recent; s_misc[32 + wave] = (int)kmin_inv; s_misc[48 + wave] = (int)kmax; }
    for (int i = tid; i < 256; i += THREADS) s_bin[i] = 0;
    __syncthreads();
    recent = __builtin_amdgcn_readfirstlane(ev_wave_sum(lane < WAVES ? s_misc[16 + lane] : 0));

    // ---- the keep-th largest key: rows above `lo` stay, of those equal to it the first `need` (need >= n: all of them)
    uint32_t lo = kEvRecent;
    int need = a.keep;
    if (recent < a.keep) {
        lo = ~(uint32_t)__builtin_amdgcn_readfirstlane(ev_wave_max((uint32_t)s_misc[32 + (lane & (WAVES - 1))]));
        uint32_t hi = __builtin_amdgcn_readfirstlane(ev_wave_max((uint32_t)s_misc[48 + (lane & (WAVES - 1))]));  // inclusive
        int above = recent;                          // rows > hi
        for (int round = 0;; ++round) {
            const int bits = 32 - __builtin_clz(hi - lo | 1u), shift = bits > 8 ? bits - 8 : 0;
            // three sets of bins: the next round's is cleared while the last round's may still be read
            int *bin = s_bin + round % 3 * 256, *next = s_bin + (round + 1) % 3 * 256;
            for_rows([&](int k) {
                const uint32_t x = key(k);
                if (x >= lo && x <= hi) atomicAdd(&bin[(x - lo) >> shift], 1);
            });
            for (int i = tid; i < 256; i += THREADS) next[i] = 0;
            __syncthreads();
            // lane l: bins 255 - 4 l downwards; the first whose rows, with all above it, are `keep` or more
            const int4 q = *reinterpret_cast<const int4 *>(bin + 252 - 4 * lane);
            const int own = q.x + q.y + q.z + q.w;
            int incl = own;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const int up = __shfl_up(incl, o, 64);
                if (lane >= o) incl += up;
            }
            const int l = __builtin_ctzll(__ballot(above + incl >= a.keep));  // there is one: all rows together are more than keep
            int before = above + incl - own, at = 255 - 4 * lane, in = q.w;
            if (before + in < a.keep) { before += in; --at; in = q.z; }
            if (at == 254 - 4 * lane && before + in < a.keep) { before += in; --at; in = q.y; }
            if (at == 253 - 4 * lane && before + in < a.keep) { before += in; --at; in = q.x; }
            before = __builtin_amdgcn_readlane(before, l);
            at = __builtin_amdgcn_readlane(at, l);
            in = __builtin_amdgcn_readlane(in, l);
            above = before;
            lo += (uint32_t)at << shift;
            const uint32_t top = lo + ((1u << shift) - 1u);
            hi = top < hi && top >= lo ? top : hi;
            if (before + in == a.keep) { need = n; break; }
            if (shift == 0) { need = a.keep - before; break; }
        }
    }

    // ---- number the free slots below keep and the staying rows above it, in slot order
    int ties = 0;
    if (need < n) {
        for_rows([&](int k) { ties += __popcll(__ballot(key(k) == lo)); });
        if (lane == 0) s_misc[wave] = ties;
        __syncthreads();
        ties = ev_wave_sum(lane < wave ? s_misc[lane & (WAVES - 1)] : 0);  // in the wavefronts before this one
    }
    int32_t *list = ev_list(a, slab);
    int holes = 0, fills = 0, tie = ties;
    auto stays_of = [&](int k, uint32_t x, int &rank) {  // rank: ties before the wavefront's row k, moved on
        if (need >= n) return x >= lo;
        const uint64_t m = __ballot(x == lo);
        const bool stays = x > lo || (x == lo && rank + __popcll(m & ((1ull << lane) - 1)) < need);
        rank += __popcll(m);
        return stays;
    };
    for_rows([&](int k) {
        const int j = j0 + 64 * k;
        const bool stays = stays_of(k, key(k), tie) && j < n;
        holes += __popcll(__ballot(j < a.keep && !stays));
        fills += __popcll(__ballot(j >= a.keep && stays));
        if (stays && j < a.keep) {
            if (wo != w) wo[j] = REGS ? wr[REGS ? k : 0] : w[j];
            if (pos && po != pos) po[j] = REGS ? pr[REGS ? k : 0] : pos[j];
        }
    });
    if (lane == 0) { s_misc[16 + wave] = holes; s_misc[32 + wave] = fills; }
    __syncthreads();
    const int h = lane < WAVES ? s_misc[16 + lane] : 0, f = lane < WAVES ? s_misc[32 + lane] : 0;
    const int count = ev_wave_sum(h);
    holes = ev_wave_sum(lane < wave ? h : 0);
    fills = ev_wave_sum(lane < wave ? f : 0);
    tie = ties;
    for_rows([&](int k) {
        const int j = j0 + 64 * k;
        const bool stays = stays_of(k, key(k), tie) && j < n, hole = j < a.keep && !stays, fill = j >= a.keep && stays;
        const uint64_t hm = __ballot(hole), fm = __ballot(fill), below = (1ull << lane) - 1;
        const int hr = holes + __popcll(hm & below), fr = fills + __popcll(fm & below);
        if (hole) { if (REGS) s_hole[hr] = (uint16_t)j; else list[2 + 2 * (size_t)hr] = j; }
        if (fill) { if (REGS) s_fill[fr] = (uint16_t)j; else list[2 + 2 * (size_t)fr + 1] = j; }
        holes += __popcll(hm);
        fills += __popcll(fm);
    });
    if (!REGS) __threadfence_block();
    __syncthreads();

    // ---- weights and positions of the rows that move, and the list for the kernel that moves them
    const volatile int32_t *vlist = list;
    for (int i = tid; i < count; i += THREADS) {
        const int to = REGS ? s_hole[i] : vlist[2 + 2 * (size_t)i], of = REGS ? s_fill[i] : vlist[2 + 2 * (size_t)i + 1];
        wo[to] = w[of];
        if (pos) po[to] = pos[of];
        if (REGS && !move) { list[2 + 2 * (size_t)i] = to; list[2 + 2 * (size_t)i + 1] = of; }
    }
    if (tid == 0 && !move) list[0] = count;
    if (REGS && move) ev_move(a, b, kvh, count, wave, WAVES, [&](int i, int *to, int *of) { *to = s_hole[i]; *of = s_fill[i]; });
}

// move: the workgroup moves its slab's rows itself and keeps no list (slabs of up to THREADS * REGS rows).
template <int THREADS, int REGS>
__global__ __launch_bounds__(THREADS) void evict_select_kernel(EvictArgs a, int move) {
    __shared__ __attribute__((aligned(16))) int s_bin[768];
    __shared__ int s_misc[64];
    __shared__ uint16_t s_hole[THREADS * REGS / 2], s_fill[THREADS * REGS / 2];  // there are as many free slots as rows for them
    const int slab = blockIdx.x, b = slab / a.Hkv, n = ev_len(a, b), tid = threadIdx.x;
    if (move && a.d_len_out && slab % a.Hkv == 0 && tid == 0) a.d_len_out[b] = n < a.keep ? n : a.keep;
    if (n <= a.keep) {
        const float *w = a.weight + (size_t)slab * a.S;
        float *wo = a.weight_out + (size_t)slab * a.S;
        if (tid == 0 && !move) ev_list(a, slab)[0] = 0;
        if (wo != w) for (int j = tid; j < n; j += THREADS) wo[j] = w[j];
        if (a.pos && a.pos_out != a.pos)
            for (int j = tid; j < n; j += THREADS) a.pos_out[(size_t)slab * a.S + j] = a.pos[(size_t)slab * a.S + j];
        return;
    }
    if (n <= THREADS * REGS) ev_slab<THREADS, REGS>(a, slab, n, move != 0, s_bin, s_misc, s_hole, s_fill);
    else ev_slab<THREADS, 0>(a, slab, n, false, s_bin, s_misc, s_hole, s_fill);
}

// Rows that the selection listed: workgroups of four wavefronts, gridDim.y of them per slab.
__global__ __launch_bounds__(256) void evict_move_kernel(EvictArgs a) {
    const int slab = blockIdx.x, b = slab / a.Hkv, kvh = slab % a.Hkv;
    const int32_t *list = ev_list(a, slab);
    if (a.d_len_out && kvh == 0 && blockIdx.y == 0 && threadIdx.x == 0) {
        const int n = ev_len(a, b);
        a.d_len_out[b] = n < a.keep ? n : a.keep;
    }
    ev_move(a, b, kvh, list[0], blockIdx.y * 4 + (threadIdx.x >> 6), gridDim.y * 4,
            [&](int i, int *to, int *of) { *to = list[2 + 2 * (size_t)i]; *of = list[2 + 2 * (size_t)i + 1]; });
}

size_t evict_rows_ws_bytes(int B, int Hkv, int S, int keep) {
    const int64_t moves = keep < S - keep ? keep : S - keep;
    return (size_t)B * Hkv * (2 + 2 * (size_t)(moves < 0 ? 0 : moves)) * sizeof(int32_t);
}

bool evict_rows_grid_fits(int B, int Hkv, int S) { return grid_fits((int64_t)B * Hkv, S <= 4096 ? 512 : 1024); }

void launch_evict_rows(const EvictArgs &a0, hipStream_t st) {
    EvictArgs a = a0;
    if (a.B <= 0) return;
    a.max_moves = a.keep < a.S - a.keep ? a.keep : a.S - a.keep;
    const int slabs = a.B * a.Hkv;
    // The selecting workgroups move the rows themselves where there are enough of them for the memory system, or few rows to move; in
    // place lengths need a second kernel (the workgroups of a sequence all read its length).  Moved by themselves and by a second
    // kernel: 4 slabs of 320 rows down to 256, 9.5 and 12.0 us; 384 of 2112 down to 2048, 15.7 and 19.2; 8000 down to 1000: 32 slabs 27.8 and 23.0, 64
    // slabs 33.2 and 29.2, 128 slabs 44.5 and 47.9, 256 slabs 66.8 and 75.4.
    const bool move = a.S <= 16384 && a.d_len_out != a.d_len && (slabs >= 128 || a.max_moves <= 128);
    // The smallest workgroup that holds a slab in registers, by capacity: 512 threads and 1024 take 17 and 26.7 us for 384 slabs of 2112 rows down to 2048, 87 and
    // 95 for 384 of 4096 down to 3000, 19.7 and 20.4 for 32 of 4000 down to 1000, 9.9 and 10.9 for 4 of 320.
    if (a.S <= 4096) evict_select_kernel<512, 8><<<slabs, 512, 0, st>>>(a, move);
    else evict_select_kernel<1024, 16><<<slabs, 1024, 0, st>>>(a, move);
    if (move) return;
    // A workgroup per 32 moves a slab may make, 64 at most.  With 8 (at most 256), 32 and 128 moves: 32 slabs of 4000 down to 1000, 19.6, 19.7 and 25.6 us; 384
    // of 2112 down to 2048, 21.9, 22 and 24.8; 256 of 8000 down to 1000, 95, 93 and 92; 8 of 30000 down to 4000, 86.5, 88.5 and 92.4 (at most 16: 101).
    int groups = ceil_div(a.max_moves, 32);
    groups = groups < 1 ? 1 : (groups > 64 ? 64 : groups);
    evict_move_kernel<<<dim3(slabs, groups), 256, 0, st>>>(a);
}
