// Attention of a span of new tokens over a cache (rl_op_span_attention), with the attention weight of every cached row on request.
//
// The T tokens of a sequence and the G = Hq / Hkv query heads of a kv head are R = T * G query rows that share every cache row: per tile
// of 32 cache rows two matrix products,
//     S^T[32 keys x 16 columns] = K[32 x hd] * Q^T[hd x 16],     O^T[hd x 16 columns] += V^T[hd x 32 keys] * P^T[32 x 16],
// where q and the probabilities enter the matrix cores as two half terms, and K and V as stored: about 22 significant bits for elements of the
// scaled q from 2^-3 on (smaller ones to 2^-25) and for probabilities as said below.  Up to 8
// query rows share the 16 columns with their low terms (columns c and c + 8: one product for both); with more a column is a row
// and the low terms take a second product, which leaves the softmax without idle lanes (32 query rows on one wavefront: 77 us as four
// tiles of 8, 71 as two of 16, at 3 x 8 tokens over 30011 rows, 32/8 heads).
// A workgroup takes 8, 16 or 32 query rows; more rows are further workgroups that find the cache rows in the L2 of their XCD.
// A block-scaled int16 n = 64 h + l is taken as h + l / 64: two exact halves by packed 16-bit instructions, five for two elements (h in
// [-512, 511] and l / 64 in [0, 1) come out of the mantissa of 1024 + x and 16 + x / 64); the factor 64 goes with the row scale.  S^T
// leaves a lane with 4 keys of a column per 16-key product, which is the layout that P^T needs: key 4 j + i of the first 16 keys is
// contraction index 8 j + i, of the second 8 j + 4 + i.
//
// One pass with a running maximum and sum per query row.  The maximum is raised (and the accumulators rescaled) only when a score
// exceeds it by more than 2^8, so that most tiles need no reduction across lanes.  A weight at the maximum enters the products as 2^7 (half rows:
// the maximum is taken 7 lower; block-scaled: with the reference of the row scales), the largest as 2^15: weights from 2^-10 of the maximum on keep
// about 22 bits, smaller ones are rounded to nearest on a grid of 2^-31, so that thousands of rows with little weight each do not lose any
// on average (at their own size, cut off, rows 2^-17 below the maximum lost 0.4 % of theirs).  Scores are kept in units of log 2 (q is scaled by
// log2(e) / sqrt(hd) before it is split).
//
// Memory: bound by reading K and V once.  Each wavefront copies V tiles from HBM into its own two-stage LDS ring (buffer loads with the
// LDS destination, 16 rows per buffer descriptor: pages hold a multiple of 16 rows; rows past the end arrive as zeros), so no barrier is
// needed in the loop.  16-byte pieces are stored XOR-permuted, so that the transposing reads are free of bank conflicts.  K goes straight
// into the registers that feed the products, which leaves LDS for two workgroups of four wavefronts per compute unit; with 32 query rows,
// whose registers allow no more than four wavefronts anyway, it goes through the ring as well: whole lines per instruction, and the
// next tile's copies start before the scores (3 x 8 tokens over 30011 rows: 57 us instead of 69, each at its best number of workgroups).
// W = 2 or 4 wavefronts share the rows of a sequence and join through LDS at the end; nsplit workgroups join in a second kernel.
// Weights need the scores again once maximum and sum are final.  A workgroup with up to 16 query rows that has seen all rows and queries
// of a kv head keeps them lane by lane, most of them in registers, and adds up the weights itself; else they go to the workspace and the
// second kernel does.  (The kernel of 16 query rows of 128 keeps 8 tiles at the price of up to 14 spilled registers over half rows, 3 over int16.)
//
// Measured, cold caches: 32 x 5 drafts over up to 1030 int16 rows, 32 heads of 128, 77 us (420 MB, 5.5 TB/s); 3 x 8 tokens over up to 30011
// rows in pages of 64, 32/8 heads, 61 us (308 MB, 5.0 TB/s); 48 tokens with weights over up to 2111 rows, 64/8 heads, 78 us (321 MB,
// 4.1 TB/s; 86 with all scores in the workspace, 67 without weights); 8 x 512 tokens of a prompt over up to 4096 rows, 32/8 heads, 657 us
// (int16: 1328), the cache read from L2 once per 32 query rows.  A kernel that only reads 300 MB takes 45 us.  A
// workgroup's first tile arrives 5 to 10 us after the launch (lengths, page numbers and rows depend on each other while every compute
// unit starts); the loop itself reads 7 TB/s.  Equal shares of all tiles for a fixed number of workgroups instead of whole items
// balance lengths but leave nothing to overlap a workgroup's start and end with: 95 us for the drafts, 83 with weights.
#include "kernels.h"

#include <type_traits>

#define SPAN_LDS(p) ((__attribute__((address_space(3))) void *)(p))
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));

static constexpr int kSpanTile = 32;        // cache rows per tile
static constexpr float kSpanSlack = 8.f;    // how far (in powers of two) a weight may exceed the running reference
static constexpr float kSpanLeast = 0x1p-100f;  // values of weights times row scales below it count as zero: far below any half, and a subnormal has no reciprocal
static constexpr float kSpanShift = 7.f, kSpanUnit = 128.f;  // the reference in the products: 2^7, as exponent and factor

__device__ __forceinline__ float span_ror8(float v) {  // lane l of a row of 16 receives lane (l + 8) % 16
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));
}
// Another lane of the row of 16: 0xb1: lane ^ 1, 0x4e: lane ^ 2, 0x141 / 0x140: mirrored half row / row.
template <int CTRL>
__device__ __forceinline__ float span_dpp(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float span_max_groups(float v) {  // over the four lane groups that hold one column
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}

// Eight int16 elements n = 64 h + l as h and l / 64.
__device__ __forceinline__ void span_split(u32x4_t n, f16x8_t *h, f16x8_t *l) {
    typedef uint16_t u16x8_t __attribute__((ext_vector_type(8)));
    const u16x8_t top = (__builtin_bit_cast(u16x8_t, n) >> (uint16_t)6) ^ (uint16_t)0x6600;  // 1024 + (h + 512) as a half
    const u32x4_t low = (n & 0x003f003fu) | 0x4c004c00u;                                    // 16 + l / 64
    *h = __builtin_bit_cast(f16x8_t, top) - (_Float16)1536.f;
    *l = __builtin_bit_cast(f16x8_t, low) - (_Float16)16.f;
}

// Query rows of a workgroup: the fewest that hold them all.  At 8 rows the kernels of 8 and of 16 take 78 and 80 us (32 x 5 over 1030 int16 rows),
// 67.5 and 67.5 (48 over 2111 rows, 64/8 heads), with weights 78 and 97; at 16 rows the kernels of 16 and of 32 take 39.5 and 40.5 us (32 x 4 over 2000,
// 32/8 heads), 71.5 and 73 (64 x 2, 64/8 heads), with weights 106 and 126.
__host__ __device__ static inline int span_rows(int T, int G) {
    const int64_t R = (int64_t)T * G;
    return R <= 8 ? 8 : R <= 16 ? 16 : 32;
}

// The workspace: statistics (max, sum) of every (query row, split), then partial outputs (nsplit > 1), then scores (weights) -- of every
// (sequence, kv head, workgroup's query rows, tile of cache rows) a block of [query rows][32], written as whole lines.
struct SpanWs {
    size_t stats, part, scores, total;  // offsets in floats
    size_t slab;                        // floats of scores per (sequence, kv head)
    int tiles;                          // blocks of a workgroup's query rows
};
__host__ __device__ static inline SpanWs span_ws(int B, int T, int Hq, int Hkv, int hd, int S, int nsplit, bool weights) {
    SpanWs w;
    const size_t rows = (size_t)B * T * Hq;
    const int G = Hq / Hkv, per = span_rows(T, G);
    w.tiles = (S + kSpanTile - 1) / kSpanTile;
    w.slab = (size_t)((T * (int64_t)G + per - 1) / per) * per * w.tiles * kSpanTile;
    w.stats = 0;
    w.part = nsplit > 1 || weights ? (rows * nsplit * 2 + 3) / 4 * 4 : 0;
    w.scores = w.part + (nsplit > 1 ? rows * nsplit * hd : 0);
    w.total = w.scores + (weights ? (size_t)B * Hkv * w.slab : 0);
    return w;
}

// What a sequence's span looks like: rows that were there, new tokens.
__device__ __forceinline__ void span_extent(const SpanArgs &a, int b, int *n0, int *tn) {
    int n = a.d_len[b], t = a.T;
    if (a.d_span) { const int s = a.d_span[b]; t = s < 0 ? 0 : (s < t ? s : t); }
    *n0 = n < 0 ? 0 : (n > a.S ? a.S : n);
    *tn = t;
}

// ONCE: no other workgroup reads these cache rows (one row tile), so their copies are non-temporal: they stream faster.
// RT: 0: 8 query rows with both terms in one tile; 1, 2: so many tiles of 16 rows.
// WT: 0: no weights.  1: the scores go to the workspace, the second kernel adds the weights up.  2: this workgroup sees all rows and
// queries of a kv head and adds them up itself, from scores that every lane kept: the first KEEP tiles' in registers, further ones in the
// workspace.
template <int HD, int RT, int W, bool I16, bool ONCE, int WT>
__global__ __launch_bounds__(64 * W, RT == 2 ? 1 : 2) void span_attention_kernel(SpanArgs a, int row_tiles, int items) {
    constexpr int RB = HD * 2;                    // bytes of a cache row
    constexpr int KS = HD / 32, OT = HD / 16;     // k-steps of a score, tiles of the output
    constexpr int TILEB = kSpanTile * RB;
    constexpr bool KL = RT == 2;                  // K through LDS as well
    constexpr bool EARLY = KL || !WT;
    constexpr float SHIFT = I16 ? 0.f : kSpanShift;  // half rows: weights are exp2(score - (maximum - SHIFT)) from the start, sums included
    constexpr int NV = RT ? 8 : 4, KEEP = WT == 2 ? (RT ? 8 : 16) : 0;  // scores of a lane per tile and column tile
    constexpr int SCALES = KL ? 2 * TILEB : TILEB, STAGE = SCALES + (I16 ? 512 : 0);  // a V tile, with KL a K tile, the row scales of K and V
    constexpr int LPR = RB / 16;                  // lanes per row of a copy instruction
    constexpr int NT = RT ? RT : 1, TR = RT ? 16 : 8, ROWS = TR * NT;  // column tiles, query rows of a tile and of this workgroup
    constexpr int OWN = 2 * STAGE > ROWS * (HD + 2) * 4 ? 2 * STAGE : (ROWS * (HD + 2) * 4 + 1023) / 1024 * 1024;  // LDS of a wavefront
    __shared__ __attribute__((aligned(1024))) unsigned char ring_all[W * OWN];
    __shared__ float s_rows[2][ROWS];             // of every query row: maximum, 1 / sum

    // Row tiles of one item run at the same time on the same XCD (workgroups that are congruent modulo 8 share one).
    const int bid = blockIdx.x, rem = bid % (8 * row_tiles);
    const int rt = rem / 8;
    int item = bid / (8 * row_tiles) * 8 + rem % 8;
    if (item >= items) return;
    const int split = item % a.nsplit; item /= a.nsplit;
    const int kvh = item % a.Hkv, b = item / a.Hkv;
    const int G = a.Hq / a.Hkv;
    int n0, tn;
    span_extent(a, b, &n0, &tn);
    n0 = __builtin_amdgcn_readfirstlane(n0);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int R = tn * G, r0 = rt * ROWS;
    if (r0 >= R) return;
    const int rlast = (R < r0 + ROWS ? R : r0 + ROWS) - 1;
    auto limit = [&](int rr) { const int n = n0 + rr / G + 1; return n < a.S ? n : a.S; };  // rows that query row rr sees
    const int nmax = limit(rlast), nmin = limit(r0);

    const int wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int c = lane & 15, j = lane >> 4;       // column / group of 4 keys
    unsigned char *ring = ring_all + wave * (OWN);
    // Rows of a split: the same for all sequences, from the longest of them, so that workgroups have equal work whatever the lengths
    // (a short sequence has no rows in its last splits).
    int longest = nmax;
    if (a.nsplit > 1) {
        for (int i = lane; i < a.B; i += 64) longest = a.d_len[i] > longest ? a.d_len[i] : longest;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) {
            const int x = __shfl_xor(longest, o, 64);
            longest = x > longest ? x : longest;
        }
        longest = __builtin_amdgcn_readfirstlane(longest < a.S - a.T ? longest + a.T : a.S);
    }
    const int parts = a.nsplit * W;
    const int chunk = ((longest + parts - 1) / parts + kSpanTile - 1) / kSpanTile * kSpanTile;  // of a wavefront
    const int64_t start = (int64_t)(split * W + wave) * chunk;
    const int j0 = __builtin_amdgcn_readfirstlane(start < nmax ? (int)start : nmax);
    const int j1 = __builtin_amdgcn_readfirstlane(nmax - j0 > chunk ? j0 + chunk : nmax);
    const int ntiles = (j1 - j0 + kSpanTile - 1) / kSpanTile;

    // ---- the query rows' loads are issued before the first tile's and converted behind them
    f32x4_t qraw[NT][2 * KS];
    int lim[NT];
    bool row_ok[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int rr = r0 + TR * nt + c % TR;
        row_ok[nt] = rr <= rlast;
        const int rc = row_ok[nt] ? rr : rlast;
        lim[nt] = limit(rc);
        const float *qp = a.q + (((size_t)b * a.T + rc / G) * a.Hq + kvh * G + rc % G) * HD + 8 * j;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            qraw[nt][2 * s] = *reinterpret_cast<const f32x4_t *>(qp + 32 * s);
            qraw[nt][2 * s + 1] = *reinterpret_cast<const f32x4_t *>(qp + 32 * s + 4);
        }
    }

    // ---- copies: instruction i of 16 rows moves rows (64 / LPR) i ..; this lane fills slot lane % LPR of row (64 / LPR) i + lane / LPR
    constexpr int CI = 16 * RB / 1024;
    auto vperm = [](int r) { return HD == 128 ? 2 * (r & 7) : 2 * ((r >> 1) & 3); };
    auto kperm = [](int r) { return HD == 128 ? r & 15 : (r >> 1) & 7; };
    uint32_t vsrc[CI], ksrc[KL ? CI : 1];
#pragma unroll
    for (int i = 0; i < CI; ++i) {
        const int r = (64 / LPR) * i + lane / LPR, slot = lane % LPR;
        vsrc[i] = (uint32_t)(r * RB + ((slot ^ vperm(r)) << 4));
        if (KL) ksrc[KL ? i : 0] = (uint32_t)(r * RB + ((slot ^ kperm(r)) << 4));
    }
    // Page numbers: 64 entries of the sequence's list in a register, one per lane (a load per tile would wait for the copies
    // in flight, which return in order).
    const int32_t *pages = a.map.table ? a.map.table + (size_t)b * a.map.table_stride : nullptr;
    const int last_page = pages && ntiles ? (j1 - 1) >> a.map.page_shift : 0;
    int page_base = 0, page_reg = 0;
    auto load_pages = [&](int from) {
        page_base = from;
        const int at = from + lane < last_page ? from + lane : last_page;
        page_reg = pages[at];
        asm volatile("" : "+v"(page_reg));        // waited for here, not at every use
    };
    if (pages && ntiles) load_pages(j0 >> a.map.page_shift);
    const size_t slab = ((size_t)b * a.Hkv + kvh) * a.S;
    auto row_of = [&](int row) -> size_t {        // row: the same in every lane, rows ascend from call to call
        if (!pages) return slab + row;
        const int at = row >> a.map.page_shift;
        if (at - page_base >= 64) load_pages(at);
        const int page = __builtin_amdgcn_readlane(page_reg, at - page_base);
        return (((size_t)page * a.Hkv + kvh) << a.map.page_shift) + (row & ((1 << a.map.page_shift) - 1));
    };
    u32x4_t kreg[KL ? 1 : 2][KL ? 1 : KS];                          // K operands of the next tile: row c of 16, elements 32 s + 8 j + 0..7
    size_t first[2];                              // of the tile that is being copied: where its two blocks of 16 rows are, how many exist
    int rows[2];
    auto piece = [&](const f16_t *base, int h) {
        const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)first[h]), hi = __builtin_amdgcn_readfirstlane((uint32_t)(first[h] >> 32));
        const size_t at = ((size_t)hi << 32 | lo) * HD;
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<f16_t *>(base + at), 0, rows[h] * RB, 0x00020000);
    };
    auto issue_v = [&](int tile, unsigned char *st) {  // V, row scales, and K where it goes through LDS
        if (tile >= ntiles) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row0 = j0 + tile * kSpanTile + 16 * h;
            rows[h] = j1 - row0;                  // at most 16 of them exist; without any every lane is out of range
            rows[h] = __builtin_amdgcn_readfirstlane(rows[h] < 0 ? 0 : (rows[h] > 16 ? 16 : rows[h]));
            first[h] = rows[h] ? row_of(row0) : first[0];
        }
#if defined(__HIP_DEVICE_COMPILE__)  // the host pass does not know these builtins
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __amdgpu_buffer_rsrc_t vr = piece(a.vc, h);
            if (KL) {
                __amdgpu_buffer_rsrc_t kr = piece(a.kc, h);
#pragma unroll
                for (int i = 0; i < CI; ++i)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, SPAN_LDS(st + TILEB + h * 16 * RB + i * 1024), 16, (int)ksrc[KL ? i : 0], 0, 0, ONCE ? 3 : 0);
            }
#pragma unroll
            for (int i = 0; i < CI; ++i)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, SPAN_LDS(st + h * 16 * RB + i * 1024), 16, (int)vsrc[i], 0, 0, ONCE ? 3 : 0);
        }
        if (I16) {  // row scales: lane l takes row l % 32 (the tile's first row where there is none: its weight is 0)
            const int r = lane & 15, h = (lane >> 4) & 1;
            const size_t at = h ? (r < rows[1] ? first[1] + r : first[0]) : (r < rows[0] ? first[0] + r : first[0]);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a.map.kscale + at), SPAN_LDS(st + SCALES), 4, 0, 0);
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(a.map.vscale + at), SPAN_LDS(st + SCALES + 256), 4, 0, 0);
        }
#else
        (void)st; (void)piece;
#endif
    };
    auto issue_k = [&](int tile) {                // K of the tile that issue_v took last
        if (KL || tile >= ntiles) return;
#if defined(__HIP_DEVICE_COMPILE__)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            __amdgpu_buffer_rsrc_t kr = piece(a.kc, h);
#pragma unroll
            for (int s = 0; s < KS; ++s) kreg[KL ? 0 : h][KL ? 0 : s] = __builtin_amdgcn_raw_buffer_load_b128(kr, c * RB + (4 * s + j) * 16, 0, ONCE ? 3 : 0);
        }
#endif
    };

    issue_v(0, ring);
    issue_k(0);
    __builtin_amdgcn_sched_barrier(0);

    // ---- Q^T operands: column c of tile nt = query row r0 + TR nt + c % TR; k-step s covers elements 32 s + 8 j + 0..7
    f16x8_t qf[NT][KS], ql[RT ? NT : 1][RT ? KS : 1];
    const float qscale = rsqrtf((float)HD) * 1.44269504f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = row_ok[nt] ? qraw[nt][2 * s + (e >> 2)][e & 3] * qscale : 0.f;
                const _Float16 hi = (_Float16)__builtin_amdgcn_fmed3f(v, -65504.f, 65504.f);  // saturating, like every half here
                // v * 0: the limits take a NaN for the lower one, an infinity for the upper; the low term is a NaN then
                const _Float16 lo = (_Float16)__builtin_fmaf(v, 0.f, __builtin_amdgcn_fmed3f(v - (float)hi, -65504.f, 65504.f));
                qf[nt][s][e] = RT || c < 8 ? hi : lo;
                if (RT) ql[RT ? nt : 0][RT ? s : 0][e] = lo;
            }

    int vaddr[OT], kaddr[KL ? KS : 1];
#pragma unroll
    for (int s = 0; s < KS; ++s)
        if (KL) kaddr[KL ? s : 0] = c * RB + (((4 * s + j) ^ kperm(c)) << 4);
    {
        const int r = 4 * j + (c >> 2);  // the row whose 4 elements this lane hands to the transposing read
#pragma unroll
        for (int t = 0; t < OT; ++t) vaddr[t] = r * RB + (((2 * t + ((c >> 1) & 1)) ^ vperm(r)) << 4) + 8 * (c & 1);
    }

    f32x4_t acc[NT][OT];
    float mrun[NT], den[NT], ref[NT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        mrun[nt] = -INFINITY; den[nt] = 0.f; ref[nt] = 0.f;
#pragma unroll
        for (int t = 0; t < OT; ++t) acc[nt][t] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const SpanWs w = span_ws(a.B, a.T, a.Hq, a.Hkv, HD, a.S, a.nsplit, WT);
    const size_t row_base = ((size_t)b * a.Hkv + kvh) * a.T * G;  // query rows in the workspace: [b][kv head][t * G + g]
    float *scores = a.ws + w.scores + ((size_t)b * a.Hkv + kvh) * w.slab + (size_t)rt * w.tiles * (ROWS * kSpanTile);

    float kept[KEEP ? KEEP : 1][NT][NV];          // scores of the first tiles
#pragma unroll
    for (int i = 0; i < KEEP; ++i)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int e = 0; e < NV; ++e) kept[i][nt][e] = 0.f;
    auto consume = [&](int tile, unsigned char *st, unsigned char *other) {
        const int key0 = j0 + tile * kSpanTile;
        // V into the stage consumed one step ago: before the scores (79 us against 81 at 32 x 5 tokens over 1030 int16 rows, 32 heads),
        // but with weights behind them (85.7 against 87.1 at 48 tokens over 2111 rows, 64/8 heads)
        if (EARLY) issue_v(tile + 1, other);
        __builtin_amdgcn_sched_barrier(0);
        f32x4_t sacc[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sacc[nt][0] = sacc[nt][1] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const u32x4_t kw = KL ? *reinterpret_cast<const u32x4_t *>(st + TILEB + h * 16 * RB + kaddr[KL ? s : 0]) : kreg[KL ? 0 : h][KL ? 0 : s];
                f16x8_t kh, kl;
                if (I16) span_split(kw, &kh, &kl);
                else kh = __builtin_bit_cast(f16x8_t, kw);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    sacc[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, qf[nt][s], sacc[nt][h], 0, 0, 0);
                    if (RT) sacc[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kh, ql[RT ? nt : 0][RT ? s : 0], sacc[nt][h], 0, 0, 0);
                    if (I16) sacc[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, qf[nt][s], sacc[nt][h], 0, 0, 0);
                    if (I16 && RT) sacc[nt][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kl, ql[RT ? nt : 0][RT ? s : 0], sacc[nt][h], 0, 0, 0);
                }
            }
        f32x4_t ksc[2], vsc[2];
        if (I16) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                ksc[h] = *reinterpret_cast<const f32x4_t *>(st + SCALES + 64 * h + 16 * j);
#pragma unroll
                for (int i = 0; i < 4; ++i) ksc[h][i] = __builtin_fmaf(ksc[h][i], 64.f, ksc[h][i] * 0.f);  // infinite: NaN, as inf - inf over the row's elements is
                vsc[h] = *reinterpret_cast<const f32x4_t *>(st + SCALES + 256 + 64 * h + 16 * j);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        if (!EARLY) issue_v(tile + 1, other);
        issue_k(tile + 1);                        // into the registers just used
        __builtin_amdgcn_sched_barrier(0);
        const bool tail = key0 + kSpanTile > nmin || key0 + kSpanTile > j1;  // some query row does not see all of these keys
        if (!I16 && tail) {
            // A value that is not finite must not reach the query rows that do not see its row (0 * inf is NaN): such elements are
            // added to the others by hand and cleared from the tile.
            bool bad = false;
#pragma unroll
            for (int i = 0; i < TILEB / 1024; ++i) {
                const u32x4_t x = *reinterpret_cast<const u32x4_t *>(st + i * 1024 + lane * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) bad |= (x[e] & 0x7c00u) == 0x7c00u || (x[e] & 0x7c000000u) == 0x7c000000u;
            }
            if (__any(bad)) {
                for (int k = 0; k < kSpanTile; ++k)
#pragma unroll
                    for (int t = 0; t < OT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int e = 16 * t + 4 * j + i, kr = k & 15;
                            f16_t *p = reinterpret_cast<f16_t *>(st + k * RB + (((e >> 3) ^ vperm(kr)) << 4) + (e & 7) * 2);
                            const f16_t v = *p;
                            if ((v & 0x7c00u) == 0x7c00u) {
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt)
                                    if ((RT || c < 8) && key0 + k < lim[nt]) acc[nt][t][i] += f16_to_f32(v);
                            }
                        }
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int i = 0; i < TILEB / 1024; ++i) {
                    u32x4_t *p = reinterpret_cast<u32x4_t *>(st + i * 1024 + lane * 16);
                    u32x4_t x = *p;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if ((x[e] & 0x7c00u) == 0x7c00u) x[e] &= 0xffff0000u;
                        if ((x[e] & 0x7c000000u) == 0x7c000000u) x[e] &= 0xffffu;
                    }
                    *p = x;
                }
                __builtin_amdgcn_wave_barrier();
            }
        }
        f16x8_t pf[NT], pl[RT ? NT : 1];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float x = sacc[nt][e >> 2][e & 3];
                if (!RT) x += span_ror8(x);       // high and low term of the query row
                if (I16) x *= ksc[e >> 2][e & 3];
                v[e] = x;
            }
            if (tail) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (key0 + 16 * (e >> 2) + 4 * j + (e & 3) >= (lim[nt] < j1 ? lim[nt] : j1)) v[e] = -INFINITY;
            }
            if (WT == 2) {
#pragma unroll
                for (int e = 0; e < NV; ++e) {
                    const float x = RT || c < 8 ? v[e] : v[4 + (e & 3)];
#pragma unroll
                    for (int i = 0; i < KEEP; ++i) kept[i][nt][e] = tile == i ? x : kept[i][nt][e];  // (a branch here becomes an index into scratch)
                }
            }
            if (WT && tile >= KEEP) {             // lanes of the low term take the second 16 keys
                float *sp = scores + (size_t)(key0 / kSpanTile) * (ROWS * kSpanTile) + (TR * nt + c % TR) * kSpanTile + 4 * j;
                if (RT) {
                    *reinterpret_cast<f32x4_t *>(sp) = f32x4_t{v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<f32x4_t *>(sp + 16) = f32x4_t{v[4], v[5], v[6], v[7]};
                } else {
                    *reinterpret_cast<f32x4_t *>(sp + (c < 8 ? 0 : 16)) = c < 8 ? f32x4_t{v[0], v[1], v[2], v[3]} : f32x4_t{v[4], v[5], v[6], v[7]};
                }
            }
            float tmax = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
            if (__any(tmax > mrun[nt] + kSpanSlack)) {
                const float mnew = fmaxf(mrun[nt], span_max_groups(tmax));
                const float alpha = mrun[nt] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mrun[nt] - mnew);
                mrun[nt] = mnew;
                den[nt] *= alpha;
                if (I16) ref[nt] *= alpha;        // the accumulators count in it
#pragma unroll
                for (int t = 0; t < OT && !I16; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[nt][t][i] *= alpha;
            }
            const float m = mrun[nt] == -INFINITY ? 0.f : mrun[nt] - SHIFT;  // nothing seen yet: all weights are 0
            float wmax = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = __builtin_amdgcn_exp2f(v[e] - m);
            // the tile's sum first: added one by one to a large sum, equal small weights are all rounded the same way
            den[nt] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            float inv = 1.f;
            if (I16) {
                // The row scale of V rides on the probability.  Scales are far below the normal range of a half, so the weights are
                // measured in a reference per query row that follows their largest, and falls as the maximum rises: rows that have lost
                // their weight must not set the grid for those that took it.
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = key0 + 16 * (e >> 2) + 4 * j + (e & 3);
                    v[e] = tail && key >= (lim[nt] < j1 ? lim[nt] : j1) ? 0.f : v[e] * vsc[e >> 2][e & 3];
                    wmax = fmaxf(wmax, v[e]);
                }
                if (__any(wmax > ref[nt] * 256.f)) {
                    const float rnew = fmaxf(ref[nt], span_max_groups(wmax));
                    const float beta = rnew > 0.f ? ref[nt] / rnew : 0.f;
                    ref[nt] = rnew;
#pragma unroll
                    for (int t = 0; t < OT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[nt][t][i] *= beta;
                }
                inv = ref[nt] > kSpanLeast ? kSpanUnit * __builtin_amdgcn_rcpf(ref[nt]) : 0.f;
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) {      // the high term cut off, the low term takes what is left, rounded to nearest
                const float x0 = I16 ? v[e] * inv : v[e], x1 = I16 ? v[e + 1] * inv : v[e + 1];
                const f16x2_t hi = __builtin_bit_cast(f16x2_t, __builtin_amdgcn_cvt_pkrtz(x0, x1));
                const f16x2_t lo = __builtin_convertvector(f32x2_t{x0 - (float)hi.x, x1 - (float)hi.y}, f16x2_t);
                pf[nt][e] = RT || c < 8 ? hi.x : lo.x;
                pf[nt][e + 1] = RT || c < 8 ? hi.y : lo.y;
                if (RT) { pl[RT ? nt : 0][e] = lo.x; pl[RT ? nt : 0][e + 1] = lo.y; }
            }
        }
        s16x4_t vt[OT][2];
#if defined(__HIP_DEVICE_COMPILE__)
        {
            // Transposing reads: lane group j of 16 lanes receives the 4 keys of its group, one element per lane.  In assembly because the
            // compiler takes the builtin for a reader of every copy in flight and waits for them.
            const uint32_t sa = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) unsigned char *)st;
#pragma unroll
            for (int t = 0; t < OT; t += 4)
                asm volatile("ds_read_b64_tr_b16 %0, %8\n\tds_read_b64_tr_b16 %1, %8 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %2, %9\n\tds_read_b64_tr_b16 %3, %9 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %4, %10\n\tds_read_b64_tr_b16 %5, %10 offset:%12\n\t"
                             "ds_read_b64_tr_b16 %6, %11\n\tds_read_b64_tr_b16 %7, %11 offset:%12\n\ts_waitcnt lgkmcnt(0)"
                             : "=&v"(vt[t][0]), "=&v"(vt[t][1]), "=&v"(vt[t + 1][0]), "=&v"(vt[t + 1][1]), "=&v"(vt[t + 2][0]), "=&v"(vt[t + 2][1]),
                               "=&v"(vt[t + 3][0]), "=&v"(vt[t + 3][1])
                             : "v"(sa + vaddr[t]), "v"(sa + vaddr[t + 1]), "v"(sa + vaddr[t + 2]), "v"(sa + vaddr[t + 3]), "n"(16 * RB)
                             : "memory");
        }
#endif
#pragma unroll
        for (int t = 0; t < OT; ++t) {
            const s16x8_t vw = __builtin_shufflevector(vt[t][0], vt[t][1], 0, 1, 2, 3, 4, 5, 6, 7);
            f16x8_t vh, vl;
            if (I16) span_split(__builtin_bit_cast(u32x4_t, vw), &vh, &vl);
            else vh = __builtin_bit_cast(f16x8_t, vw);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, pf[nt], acc[nt][t], 0, 0, 0);
                if (RT) acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh, pl[RT ? nt : 0], acc[nt][t], 0, 0, 0);
                if (I16) acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, pf[nt], acc[nt][t], 0, 0, 0);
                if (I16 && RT) acc[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl, pl[RT ? nt : 0], acc[nt][t], 0, 0, 0);
            }
        }
    };

    constexpr int STORES = RT ? 2 * NT : 1;       // of scores, issued behind the next tile's copies: they need not have arrived
    for (int tile = 0; tile < ntiles; ++tile) {
        unsigned char *st = ring + (tile & 1) * STAGE;
        __builtin_amdgcn_sched_barrier(0);
        // the tile has landed once nothing older than those stores is pending: vmcnt(0) or (STORES) only
        if (tile <= KEEP || !WT) __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));
        else __builtin_amdgcn_s_waitcnt(STORES | (7 << 4) | (15 << 8));
        __builtin_amdgcn_sched_barrier(0);
        consume(tile, st, ring + (~tile & 1) * STAGE);
    }
    __builtin_amdgcn_sched_barrier(0);

    // ---- join the wavefronts: the lane groups j hold disjoint keys (den), columns c and c + 8 the two terms of a query row (acc)
    // over the wavefront's ring (all copies have landed): [ROWS][HD] sums, [ROWS] maxima, [ROWS] denominators
    float *part = reinterpret_cast<float *>(ring);
    auto s_max = [&](int i, int r) -> float & { return reinterpret_cast<float *>(ring_all + i * (OWN))[ROWS * HD + r]; };
    auto s_den = [&](int i, int r) -> float & { return reinterpret_cast<float *>(ring_all + i * (OWN))[ROWS * (HD + 1) + r]; };
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        float d = den[nt];
        d += __shfl_xor(d, 16, 64);
        d += __shfl_xor(d, 32, 64);
        if (j == 0 && c < TR) { s_max(wave, TR * nt + c) = mrun[nt] - SHIFT; s_den(wave, TR * nt + c) = d; }
#pragma unroll
        for (int t = 0; t < OT; ++t) {
            f32x4_t o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o[i] = RT ? acc[nt][t][i] : acc[nt][t][i] + span_ror8(acc[nt][t][i]);
            if (I16) o = o * (ref[nt] * (64.f / kSpanUnit));
            if (c < TR) *reinterpret_cast<f32x4_t *>(part + (TR * nt + c) * HD + 16 * t + 4 * j) = o;
        }
    }
    __builtin_amdgcn_s_waitcnt(0 | (7 << 4) | (15 << 8));  // the score stores have arrived
    __syncthreads();
    constexpr int TPR = HD / 8;                     // threads per query row, 8 elements each
    for (int r = threadIdx.x / TPR; r < ROWS && r0 + r <= rlast; r += 64 * W / TPR) {
        const int e0 = (threadIdx.x % TPR) * 8;
        float m = s_max(0, r);
#pragma unroll
        for (int i = 1; i < W; ++i) m = fmaxf(m, s_max(i, r));
        float d = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < W; ++i) {
            const float f = s_max(i, r) == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s_max(i, r) - m);
            if (s_max(i, r) == -INFINITY && !(s_den(i, r) != s_den(i, r))) continue;  // a part without visible keys
            d += s_den(i, r) * f;
            const float *p = reinterpret_cast<const float *>(ring_all + i * (OWN)) + r * HD + e0;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += p[e] * f;
        }
        const int rr = r0 + r;
        const size_t row = row_base + rr;
        if (WT == 2) {
            if (e0 == 0) { s_rows[0][r] = m; s_rows[1][r] = 1.0f / d; }
        } else if (a.nsplit > 1 || WT) {
            if (e0 == 0) {
                a.ws[w.stats + (row * a.nsplit + split) * 2] = m;
                a.ws[w.stats + (row * a.nsplit + split) * 2 + 1] = d;
            }
        }
        if (a.nsplit > 1) {
            float *p = a.ws + w.part + (row * a.nsplit + split) * HD + e0;
            *reinterpret_cast<f32x4_t *>(p) = f32x4_t{o[0], o[1], o[2], o[3]};
            *reinterpret_cast<f32x4_t *>(p + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
        } else {
            const float inv = 1.0f / d;
            const size_t at = (((size_t)b * a.T + rr / G) * a.Hq + kvh * G + rr % G) * HD + e0;
            u32x4_t h, l;
#pragma unroll
            for (int e = 0; e < 4; ++e) h[e] = pack_f16x2_nan(o[2 * e] * inv, o[2 * e + 1] * inv);
            *reinterpret_cast<u32x4_t *>(a.out + at) = h;
            if (a.out_lo) {
#pragma unroll
                for (int e = 0; e < 4; ++e) l[e] = pack_f16x2_lo_nan(o[2 * e] * inv, o[2 * e + 1] * inv, h[e]);
                *reinterpret_cast<u32x4_t *>(a.out_lo + at) = l;
            }
        }
    }
    if (WT == 2) {
        __syncthreads();
        float *wt = a.weight + ((size_t)b * a.Hkv + kvh) * a.S;
        float m[NT], inv[NT];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) { m[nt] = s_rows[0][TR * nt + c % TR]; inv[nt] = s_rows[1][TR * nt + c % TR]; }
        // Sums over the query rows, which are lanes of a group of 8 or 16; 4 keys of a tile are put out by one lane of it (two with RT).
        const bool puts = RT ? c < 2 : c % 8 == 0;
        const int half = RT ? c & 1 : c >> 3;
        auto weigh = [&](int t0, auto score) {    // 8 tiles: what was there travels meanwhile
            float old[8][4];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = j0 + (t0 + u) * kSpanTile + 16 * half + 4 * j + e;
                    old[u][e] = puts && key < j1 ? wt[key] : 0.f;
                }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (t0 + u >= ntiles) break;
                const int key0 = j0 + (t0 + u) * kSpanTile + 4 * j;
                float sum[NV];
#pragma unroll
                for (int e = 0; e < NV; ++e) {
                    const int key = key0 + (RT ? 16 * (e >> 2) + (e & 3) : 16 * half + e);
                    sum[e] = 0.f;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) sum[e] += row_ok[nt] && key < lim[nt] ? __builtin_amdgcn_exp2f(score(u, nt, e) - m[nt]) * inv[nt] : 0.f;
                    sum[e] += span_dpp<0xb1>(sum[e]);       // lanes c ^ 1, c ^ 2, then the mirrored half row and row
                    sum[e] += span_dpp<0x4e>(sum[e]);
                    sum[e] += span_dpp<0x141>(sum[e]);
                    if (RT) sum[e] += span_dpp<0x140>(sum[e]);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = key0 + 16 * half + e;
                    if (puts && key < j1) wt[key] = old[u][e] + (RT && half ? sum[NV - 4 + e] : sum[e]);
                }
            }
        };
#pragma unroll
        for (int t0 = 0; t0 < KEEP; t0 += 8)
            if (t0 < ntiles) weigh(t0, [&](int u, int nt, int e) { return kept[t0 + u][nt][e]; });
        for (int t0 = KEEP; t0 < ntiles; t0 += 8) {
            float x[8][NT][NV];
#pragma unroll
            for (int u = 0; u < 8; ++u)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int q = 0; q < NV / 4; ++q) {
                        const float *sp = scores + (size_t)(j0 / kSpanTile + t0 + u) * (ROWS * kSpanTile) + (TR * nt + c % TR) * kSpanTile + 4 * j;
                        const f32x4_t y = t0 + u < ntiles ? *reinterpret_cast<const f32x4_t *>(sp + 16 * (RT ? q : half)) : f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[u][nt][4 * q + e] = y[e];
                    }
            weigh(t0, [&](int u, int nt, int e) { return x[u][nt][e]; });
        }
    }
}

// Second launch, where the rows of a sequence or its queries are on several workgroups: the first `merge_blocks` workgroups join the
// splits of 4 query rows each (a wavefront per row, a lane per split's statistics), the others add up the weights of 1024 cache rows of
// a (sequence, kv head) each: exp2(score - max) / sum over the query rows, in their order.
template <int HD>
__global__ __launch_bounds__(256) void span_join_kernel(SpanArgs a, int merge_blocks, int key_blocks) {
    __shared__ float s_m[256], s_inv[256];
    const SpanWs w = span_ws(a.B, a.T, a.Hq, a.Hkv, HD, a.S, a.nsplit, a.weight != nullptr);
    const int G = a.Hq / a.Hkv, per_wg = span_rows(a.T, G);
    if ((int)blockIdx.x < merge_blocks) {
        const size_t row = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
        const int lane = threadIdx.x & 63;
        if (row >= (size_t)a.B * a.T * a.Hq) return;
        const int rr = (int)(row % ((size_t)a.T * G));
        const int kvh = (int)(row / ((size_t)a.T * G) % a.Hkv), b = (int)(row / ((size_t)a.T * a.Hq));
        int n0, tn;
        span_extent(a, b, &n0, &tn);
        if (rr >= tn * G) return;
        const float *st = a.ws + w.stats + row * a.nsplit * 2;
        constexpr int PER = HD / 64;
        const float *p = a.ws + w.part + row * a.nsplit * HD + lane * PER;
        const float pm = lane < a.nsplit ? st[2 * lane] : -INFINITY, pd = lane < a.nsplit ? st[2 * lane + 1] : 0.f;
        float x[8][PER];                          // parts of 8 splits in flight
        auto fetch = [&](int s0) {
#pragma unroll
            for (int s = 0; s < 8; ++s)
#pragma unroll
                for (int e = 0; e < PER; ++e) x[s][e] = s0 + s < a.nsplit ? p[(s0 + s) * HD + e] : 0.f;
        };
        fetch(0);
        float m = pm;
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        const float f = pm == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(pm - m);
        float d = pd * f, o0 = 0.f, o1 = 0.f;     // (a split without visible rows has zeros throughout)
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) d += __shfl_xor(d, o, 64);
        for (int s0 = 0; s0 < a.nsplit; s0 += 8) {
            if (s0) fetch(s0);
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const float fs = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, f), (s0 + s) & 63));
                o0 += x[s][0] * fs;
                if (PER == 2) o1 += x[s][PER - 1] * fs;
            }
        }
        const float inv = 1.0f / d;
        const size_t at = (((size_t)b * a.T + rr / G) * a.Hq + kvh * G + rr % G) * HD + lane * PER;
        if (PER == 2) {
            const uint32_t h = pack_f16x2_nan(o0 * inv, o1 * inv);
            *reinterpret_cast<uint32_t *>(a.out + at) = h;
            if (a.out_lo) *reinterpret_cast<uint32_t *>(a.out_lo + at) = pack_f16x2_lo_nan(o0 * inv, o1 * inv, h);
        } else {
            const _Float16 h = f32_to_half_nan(o0 * inv);
            a.out[at] = __builtin_bit_cast(f16_t, h);
            if (a.out_lo) a.out_lo[at] = __builtin_bit_cast(f16_t, f32_to_half_nan(o0 * inv - (float)h));
        }
        return;
    }
    const int blk = blockIdx.x - merge_blocks;
    const int slab = blk / key_blocks, key = (blk % key_blocks) * 1024 + threadIdx.x * 4;
    const int b = slab / a.Hkv;
    int n0, tn;
    span_extent(a, b, &n0, &tn);
    const int n = n0 + tn < a.S ? n0 + tn : a.S;  // rows that the last token sees
    if (tn == 0 || (blk % key_blocks) * 1024 >= n) return;
    const size_t row0 = (size_t)slab * a.T * G;
    const float *sc = a.ws + w.scores + (size_t)slab * w.slab + (size_t)(key / kSpanTile) * (per_wg * kSpanTile) + key % kSpanTile;
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
    for (int rr0 = 0; rr0 < tn * G; rr0 += 256) {
        __syncthreads();
        const int mine = rr0 + threadIdx.x;
        if (mine < tn * G) {
            const float *st = a.ws + w.stats + (row0 + mine) * a.nsplit * 2;
            float m = -INFINITY, d = 0.f;
#pragma unroll 8
            for (int s = 0; s < a.nsplit; ++s) m = fmaxf(m, st[2 * s]);
#pragma unroll 8
            for (int s = 0; s < a.nsplit; ++s)
                if (st[2 * s] != -INFINITY || st[2 * s + 1] != st[2 * s + 1]) d += st[2 * s + 1] * __builtin_amdgcn_exp2f(st[2 * s] - m);
            s_m[threadIdx.x] = m;
            s_inv[threadIdx.x] = 1.0f / d;
        }
        __syncthreads();
        const int count = tn * G - rr0 < 256 ? tn * G - rr0 : 256;
        if (key < n)
#pragma unroll 4
            for (int r = 0; r < count; ++r) {
                int lim = n0 + (rr0 + r) / G + 1;
                lim = lim < a.S ? lim : a.S;
                const int rr = rr0 + r;
                const f32x4_t s = *reinterpret_cast<const f32x4_t *>(sc + (size_t)(rr / per_wg) * w.tiles * (per_wg * kSpanTile) + rr % per_wg * kSpanTile);
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (key + i < lim) sum[i] += __builtin_amdgcn_exp2f(s[i] - s_m[r]) * s_inv[r];
            }
    }
    float *wt = a.weight + (size_t)slab * a.S + key;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (key + i < n) wt[i] += sum[i];
}

static int64_t span_items(int B, int T, int Hq, int Hkv) {
    const int G = Hq / Hkv, rows = span_rows(T, G);
    return (int64_t)B * Hkv * ((T * (int64_t)G + rows - 1) / rows);
}

int span_attention_splits(int B, int T, int Hq, int Hkv, int hd, int S) {
    const int64_t items = span_items(B, T, Hq, Hkv);
    // One workgroup of four wavefronts per compute unit: 16 x 4 tokens over 2000 rows (32/8 heads, 128 items) take 26.6 us with 2 splits, 33.7
    // with 1, 33.9 with 3; 1 x 5 over 2000 int16 rows (32 heads) 16.0 with 8, 36.2 with 1, 17.4 with 16.  Short sequences stay whole: 4 tokens over
    // 260 rows (32 heads) take 8.2 us on one workgroup per head, 11.6 with 2 splits and the second launch.
    int64_t s = items > 0 ? 256 / items : 1;
    const int cap = S / 256;
    if (s > cap) s = cap;
    if (s > 64) s = 64;
    return s < 1 ? 1 : (int)s;
}

size_t span_attention_ws_floats(int B, int T, int Hq, int Hkv, int hd, int S, int nsplit, bool weights) {
    return span_ws(B, T, Hq, Hkv, hd, S, nsplit, weights).total;
}

// With nsplit given, need grows with B and T.  Chosen from the shape, splits appear as a batch shrinks: b sequences of t tokens in k workgroups
// per kv head take s <= 256 / (b Hkv k) of them, so b t Hq s = b Hkv k s (t G / k) is at most 256 rows of a workgroup, min(t G, 32).
size_t span_attention_ws_floats_up_to(int B, int T, int Hq, int Hkv, int hd, int S, int nsplit, bool weights) {
    const int most = nsplit || B == 0 ? 1 : span_attention_splits(1, 1, Hq, Hkv, hd, S);
    if (most <= 1) return span_ws(B, T, Hq, Hkv, hd, S, nsplit ? nsplit : 1, weights).total;
    const int64_t rows = (int64_t)B * T * Hq, tg = (int64_t)T * (Hq / Hkv);
    int64_t parts = 256 * (tg < 32 ? tg : 32);
    parts = parts < rows * most ? parts : rows * most;
    parts = parts > rows ? parts : rows;
    const SpanWs one = span_ws(B, T, Hq, Hkv, hd, S, 1, weights);
    return (size_t)(parts * 2 + 3) / 4 * 4 + (size_t)parts * hd + (one.total - one.scores);
}

// Wavefronts that share a sequence's rows: four where that does not make more workgroups than run at once, two per compute unit (one
// with 32 query rows), else two: 384 items (48 tokens over 2111 rows) 85.7 us with four, 88.7 with two; 4096 (128 x 5 tokens over 390 rows,
// 32 heads) 121.6 and 115.4; 512 of 32 query rows (64 x 8 tokens over 1000, 32/8 heads) 46.8 and 42.7.
static bool span_four_waves(int64_t workgroups, int T, int G) { return workgroups <= (span_rows(T, G) > 16 ? 256 : 512); }

static int span_join_merge_blocks(int B, int T, int Hq, int nsplit) { return nsplit > 1 ? (int)(((int64_t)B * T * Hq + 3) / 4) : 0; }
// Blocks of 1024 cache rows per (sequence, kv head) whose weights the second kernel adds up.
static int span_join_key_blocks(int T, int G, int S, int nsplit, bool weights) { return weights && (nsplit > 1 || span_rows(T, G) > 16) ? ceil_div(S, 1024) : 0; }

bool span_attention_grid_fits(int B, int T, int Hq, int Hkv, int S, int nsplit, bool weights) {
    const int64_t items = (int64_t)B * Hkv * nsplit, row_tiles = span_items(1, T, Hq, Hkv) / Hkv;
    const int64_t join = span_join_merge_blocks(B, T, Hq, nsplit) + (int64_t)B * Hkv * span_join_key_blocks(T, Hq / Hkv, S, nsplit, weights);
    return grid_fits(ceil_div64(items, 8) * 8 * row_tiles, span_four_waves(items * row_tiles, T, Hq / Hkv) ? 256 : 128) && grid_fits(join, 256);
}

template <int HD, int RT, bool I16, bool ONCE>
static void span_launch(const SpanArgs &a, int row_tiles, hipStream_t st) {
    const int items = a.B * a.Hkv * a.nsplit;
    const unsigned blocks = (unsigned)((int64_t)ceil_div(items, 8) * 8 * row_tiles);
    const bool four = span_four_waves((int64_t)items * row_tiles, a.T, a.Hq / a.Hkv);
    auto launch = [&](auto wt) {
        constexpr int WT = decltype(wt)::value;
        if (four) span_attention_kernel<HD, RT, 4, I16, ONCE, WT><<<blocks, 256, 0, st>>>(a, row_tiles, items);
        else span_attention_kernel<HD, RT, 2, I16, ONCE, WT><<<blocks, 128, 0, st>>>(a, row_tiles, items);
    };
    // Weights by the workgroup itself (WT 2) and by the second kernel (WT 1), 64/8 heads over up to 2111 rows: 48 x 1 tokens 78 us and 86, 48 x 2 (16
    // query rows) 99.5 and 105, 48 x 4 (32 query rows, whose lanes keep 16 scores a tile and add over 16 lanes) 133 and 117.
    if (!a.weight) launch(std::integral_constant<int, 0>());
    else if (RT < 2 && a.nsplit == 1) launch(std::integral_constant<int, RT < 2 ? 2 : 1>());
    else launch(std::integral_constant<int, 1>());
}
template <int HD, bool I16>
static void span_launch_tiles(const SpanArgs &a, hipStream_t st) {
    const int G = a.Hq / a.Hkv, rows = span_rows(a.T, G), row_tiles = (int)((a.T * (int64_t)G + rows - 1) / rows);
    if (rows == 8) span_launch<HD, 0, I16, true>(a, 1, st);
    else if (rows == 16) span_launch<HD, 1, I16, true>(a, 1, st);
    else if (row_tiles == 1) span_launch<HD, 2, I16, true>(a, 1, st);
    else span_launch<HD, 2, I16, false>(a, row_tiles, st);
}

void launch_span_attention(const SpanArgs &a, hipStream_t st) {
    if (a.B <= 0) return;
    if (a.hd == 128) a.map.kscale ? span_launch_tiles<128, true>(a, st) : span_launch_tiles<128, false>(a, st);
    else a.map.kscale ? span_launch_tiles<64, true>(a, st) : span_launch_tiles<64, false>(a, st);
    const int merge_blocks = span_join_merge_blocks(a.B, a.T, a.Hq, a.nsplit);
    const int key_blocks = span_join_key_blocks(a.T, a.Hq / a.Hkv, a.S, a.nsplit, a.weight != nullptr);
    const int64_t blocks = merge_blocks + (int64_t)a.B * a.Hkv * key_blocks;
    if (blocks > 0) (a.hd == 128 ? span_join_kernel<128> : span_join_kernel<64>)<<<(unsigned)blocks, 256, 0, st>>>(a, merge_blocks, key_blocks ? key_blocks : 1);
}
