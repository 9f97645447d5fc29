// kdn_weigh: the attention weight that the tokens of a paged pool receive from new tokens, accumulated per KV head.
#include "kdn_ops.cuh"
#include "kdn_tc.cuh"

#include <new>
#include <vector>

using namespace kdn;

namespace {

struct WeighRec {
    const int32_t *table;
    float *acc;
    long long acc_stride;
    long long q_pos;
    int n_tokens;                           // those that some row sees
    int row, rows;                          // first row in q; n_q * g rows a KV head
    unsigned unit;                          // first unit (see each kernel)
    int tiles;                              // tiles of tokens
    int segment;                            // number of the first segment (see below)
    long long score;                        // few rows, lse not given: where in scores the request's begin, [head][row][n_tokens]
};
static_assert(sizeof(WeighRec) == 64, "");

constexpr int kInline = 16;
struct WeighLaunch {
    const WeighRec *recs;                   // in the workspace, or nullptr: inl
    const __nv_bfloat16 *q;
    long long q_stride;
    float *lse;
    const __nv_bfloat16 *const *k_layers;
    float *scores;                          // in powers of two
    float2 *stats;                          // maximum and sum of powers of two of what one part of the tokens holds
    long long n_blocks;
    unsigned long long wait_limit_ns;
    int *status;
    float scale;                            // of scores in powers of two
    unsigned units;
    int n, layer, H, g, bs;
    WeighRec inl[kInline];
};
__device__ __forceinline__ const WeighRec *records(const WeighLaunch &L) { return L.recs ? L.recs : L.inl; }

// Units of a launch are numbered record by record; worker b of G (a CTA, or a warp where rows are few) takes units [bU/G, (b+1)U/G).  The units that share
// all but the tile are a segment, numbered in the same order.  A worker leaves what it found of segment s in place b + s: along the units one of the two
// grows wherever a place is left, so that no two fall together, however many segments a worker goes through.
__device__ __forceinline__ unsigned first_unit(unsigned b, unsigned units, unsigned ctas) { return (unsigned)((unsigned long long)units * b / ctas); }
__device__ __forceinline__ unsigned cta_of(unsigned u, unsigned units, unsigned ctas)
{
    return (unsigned)((((unsigned long long)u + 1) * ctas - 1) / units);
}
// The record that holds unit u (records with no units stand in front of the one that does).
__device__ __forceinline__ int record_of(const WeighRec *recs, int n, unsigned u)
{
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (recs[mid].unit <= u) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
// Row of a token's key in the layer's pool, head 0, or -1.
__device__ __forceinline__ long long key_row(const WeighLaunch &L, const WeighRec &r, int t)
{
    const int id = r.table[t / L.bs];
    if (id < 0 || id >= L.n_blocks) { atomicCAS(L.status, 0, kStatusRange); return -1; }
    return ((long long)id * L.bs + t % L.bs) * L.H;
}
__device__ __forceinline__ const __nv_bfloat16 *query_of(const WeighLaunch &L, const WeighRec &r, int h, int rho, int D)
{
    return L.q + (long long)(r.row + rho / L.g) * L.q_stride + (long long)(h * L.g + rho % L.g) * D;
}
__device__ __forceinline__ long long lse_at(const WeighLaunch &L, const WeighRec &r, int h, int rho)
{
    return (long long)(r.row + rho / L.g) * (L.H * L.g) + h * L.g + rho % L.g;
}

// ---------------------------------------------------------------------------------------- few rows a head --
//
// Up to 16 rows (a step of grouped heads): the bytes of K bound it, 2 a channel.  Tokens are the rows and query rows the columns of
// mma.m16n8k16; a lane loads its operands straight from the pool (64 contiguous bytes of eight keys an instruction; which channel stands where in the
// sum is free), so there is no shared memory in between and K is read once: where the lse is not given, the scores (4 bytes a row, against 2 D
// of a key) wait in the workspace for it.

// A call here and with the kernels for many rows, in microseconds at 8 heads of 128, lse to be found and (given):
//     rows    1 x 10272 tokens           16 x 4096                  1 x 65536
//     4       15 and 27 (9 and 12)       36 and 88 (32 and 41)      38 and 86 (30 and 39)
//     16      23 and 28 (13 and 12)      52 and 88 (37 and 41)      59 and 86 (35 and 39)
// A given lse at 4 rows of 16 x 4096 tokens reads 134 MB of keys at 4.3 TB/s.
constexpr int kFewRows = 16, kFewWarps = 8, kFewTokens = 32;     // tokens a warp's unit
// The warps of a launch that have units.  Whoever joins the parts of a segment takes every worker between its first and its last to have left one, so that
// there must be none without a unit.
__host__ __device__ __forceinline__ unsigned few_workers(unsigned ctas, unsigned units) { return ctas * kFewWarps < units ? ctas * kFewWarps : units; }

template <int D, int NB, bool GIVEN>
__global__ void __launch_bounds__(kFewWarps * 32, 2) kdn_weigh_few_kernel(const __grid_constant__ WeighLaunch L)
{
    constexpr int KS = D / 32;                                   // loads of 8 channels a lane
    release_dependents();
    dependency_wait();
    const WeighRec *recs = records(L);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
    const __nv_bfloat16 *pool = L.k_layers[L.layer];
    const unsigned workers = few_workers(gridDim.x, L.units), me = blockIdx.x * kFewWarps + (unsigned)warp;
    if (me >= workers) return;
    // units are (record, head, tile of 32 tokens), tiles fastest; a warp is the worker
    const unsigned u0 = first_unit(me, L.units, workers), u1 = first_unit(me + 1, L.units, workers);
    int ri = record_of(recs, L.n, u0);
    WeighRec r = recs[ri];
    int h = (int)((u0 - r.unit) / (unsigned)r.tiles), tile = (int)((u0 - r.unit) % (unsigned)r.tiles);
    bool fresh = true;
    uint4 q[NB][KS];                                             // channels 32 s + 8 c .. of query row 8 b + g
    float lse[NB][2], m[NB][2], l[NB][2];
    uint4 k[2][2][KS];                                           // the same channels of tokens 16 i + 8 e + g
    bool there[2][2];                                            // those tokens exist and can be found
    auto fetch = [&](int t0) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int t = t0 + 16 * i + 8 * e + g;
                const long long row = t < r.n_tokens ? key_row(L, r, t) : -1;
                there[i][e] = row >= 0;
                const uint4 *from = reinterpret_cast<const uint4 *>(pool + (row + h) * D) + c;
#pragma unroll
                for (int s = 0; s < KS; ++s) k[i][e][s] = row < 0 ? make_uint4(0u, 0u, 0u, 0u) : __ldcs(from + 4 * s);
            }
    };
    auto finish = [&]() {                                        // maxima and sums of this worker's part of (record, head)
        if (GIVEN) return;
        const unsigned slot = me + (unsigned)(r.segment + h);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float mm = m[b][j], ll = l[b][j];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    const float m2 = __shfl_xor_sync(0xffffffffu, mm, d), l2 = __shfl_xor_sync(0xffffffffu, ll, d);
                    const float top = fmaxf(mm, m2), base = top == -INFINITY ? 0.0f : top;
                    ll = ll * exp2_approx(mm - base) + l2 * exp2_approx(m2 - base);
                    mm = top;
                }
                if (g == 0) L.stats[(long long)slot * kFewRows + 8 * b + 2 * c + j] = make_float2(mm, ll);
            }
    };
    for (unsigned u = u0; u < u1; ++u) {
        if (fresh) {
            fresh = false;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int rho = 8 * b + g;
                const uint4 *from = reinterpret_cast<const uint4 *>(query_of(L, r, h, rho < r.rows ? rho : 0, D)) + c;
#pragma unroll
                for (int s = 0; s < KS; ++s) q[b][s] = rho < r.rows ? from[4 * s] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int row = 8 * b + 2 * c + j;
                    m[b][j] = -INFINITY;
                    l[b][j] = 0.0f;
                    if (GIVEN) {                                 // what is added to a score; -infinity: nothing is seen, or no such row
                        const float x = row < r.rows ? L.lse[lse_at(L, r, h, row)] : -INFINITY;
                        lse[b][j] = x == -INFINITY ? -INFINITY : -x * 1.4426950408889634f;
                    }
                }
            }
        }
        fetch(tile * kFewTokens);
        const int t0 = tile * kFewTokens;
        const bool all = t0 + kFewTokens <= r.n_tokens && (long long)t0 + kFewTokens - 1 <= r.q_pos;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float add[2] = { 0.0f, 0.0f };
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float x[4] = { 0.0f, 0.0f, 0.0f, 0.0f };
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    mma_16x8x16(x, k[i][0][s].x, k[i][1][s].x, k[i][0][s].y, k[i][1][s].y, q[b][s].x, q[b][s].y);
                    mma_16x8x16(x, k[i][0][s].z, k[i][1][s].z, k[i][0][s].w, k[i][1][s].w, q[b][s].z, q[b][s].w);
                }
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int t = t0 + 16 * i + 8 * e + g, row = 8 * b + 2 * c + j;
                        bool seen = there[i][e];
                        if (!all) seen = seen && row < r.rows && t <= r.q_pos + row / L.g;
                        if (GIVEN) {
                            const float y = exp2_approx(fmaf(x[2 * e + j], L.scale, lse[b][j]));
                            add[e] += seen && lse[b][j] != -INFINITY ? y : 0.0f;
                        } else {
                            const float y = seen && row < r.rows ? x[2 * e + j] * L.scale : -INFINITY;
                            if (row < r.rows && t < r.n_tokens) __stcs(L.scores + r.score + ((long long)h * r.rows + row) * r.n_tokens + t, y);
                            if (y > m[b][j]) { l[b][j] *= exp2_approx(m[b][j] - y); m[b][j] = y; }
                            if (y != -INFINITY) l[b][j] += exp2_approx(y - m[b][j]);
                        }
                    }
            }
            if (GIVEN) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    add[e] += __shfl_xor_sync(0xffffffffu, add[e], 1);
                    add[e] += __shfl_xor_sync(0xffffffffu, add[e], 2);
                    if (c == 0 && there[i][e]) r.acc[(long long)h * r.acc_stride + t0 + 16 * i + 8 * e + g] += add[e];
                }
            }
        }
        if (u + 1 < u1 && ++tile == r.tiles) {
            finish();
            tile = 0;
            fresh = true;
            if (++h == L.H) { h = 0; do r = recs[++ri]; while (r.tiles == 0); }
        }
    }
    finish();
}

// Few rows: the lse from the parts, by every CTA for itself (16 threads a row), and the weights from the scores that wait.
template <int ROWS> __global__ void __launch_bounds__(256) kdn_weigh_add_scores_kernel(const __grid_constant__ WeighLaunch L, unsigned workers)
{
    __shared__ float lse[kFewRows];
    release_dependents();
    dependency_wait();
    const WeighRec *recs = records(L);
    const int h = (int)blockIdx.y, row = (int)threadIdx.x / 16, part = (int)threadIdx.x % 16;
    for (int ri = (int)blockIdx.z; ri < L.n; ri += (int)gridDim.z) {
        const WeighRec r = recs[ri];
        if (blockIdx.x * 1024 >= (unsigned)r.n_tokens && blockIdx.x > 0) continue;
        // this thread's scores and weights are on their way while the sums are made
        const int first = (int)(blockIdx.x * 1024 + threadIdx.x);
        const float *scores = L.scores + r.score + (long long)h * r.rows * r.n_tokens;
        float ahead[ROWS][4], was[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool in = first + 256 * j < r.n_tokens;
            was[j] = in ? r.acc[(long long)h * r.acc_stride + first + 256 * j] : 0.0f;
#pragma unroll
            for (int i = 0; i < ROWS; ++i)
                ahead[i][j] = in && i < r.rows ? __ldcs(scores + (long long)i * r.n_tokens + first + 256 * j) : -INFINITY;
        }
        float m = -INFINITY, l = 0.0f;
        if (r.tiles > 0 && row < r.rows) {
            const unsigned s0 = r.unit + (unsigned)h * (unsigned)r.tiles, s1 = s0 + (unsigned)r.tiles;
            const unsigned c0 = cta_of(s0, L.units, workers), n = cta_of(s1 - 1, L.units, workers) - c0 + 1, at = c0 + (unsigned)(r.segment + h);
            constexpr unsigned kLoads = 8;                       // in flight: a long context of one request has 300 parts a head
            for (unsigned j0 = (unsigned)part; j0 < n; j0 += 16 * kLoads) {
                float2 ml[kLoads];
                float top = m;
#pragma unroll
                for (unsigned i = 0; i < kLoads; ++i) {
                    const unsigned j = j0 + 16 * i;
                    ml[i] = j < n ? L.stats[(long long)(at + j) * kFewRows + row] : make_float2(-INFINITY, 0.0f);
                }
#pragma unroll
                for (unsigned i = 0; i < kLoads; ++i) top = ml[i].y == 0.0f ? top : fmaxf(top, ml[i].x);
                const float base = top == -INFINITY ? 0.0f : top;
                l *= exp2_approx(m - base);
#pragma unroll
                for (unsigned i = 0; i < kLoads; ++i) l += ml[i].y == 0.0f ? 0.0f : ml[i].y * exp2_approx(ml[i].x - base);
                m = top;
            }
        }
        for (int d = 8; d; d >>= 1) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m, d), l2 = __shfl_xor_sync(0xffffffffu, l, d);
            const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
            l = l * exp2_approx(m - base) + l2 * exp2_approx(m2 - base);
            m = top;
        }
        __syncthreads();
        if (part == 0 && row < r.rows) {
            lse[row] = l == 0.0f ? -INFINITY : m + log2f(l);
            if (blockIdx.x == 0) L.lse[lse_at(L, r, h, row)] = lse[row] * 0.69314718055994531f;
        }
        __syncthreads();
        float add[4] = { 0.0f, 0.0f, 0.0f, 0.0f };
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const float base = i < r.rows ? lse[i] : 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) add[j] += ahead[i][j] == -INFINITY ? 0.0f : exp2_approx(ahead[i][j] - base);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (first + 256 * j < r.n_tokens && add[j] != 0.0f) r.acc[(long long)h * r.acc_stride + first + 256 * j] = was[j] + add[j];
    }
}

// --------------------------------------------------------------------------------------- many rows a head --
//
// Scores of 128 tokens by 128 rows come from the tensor core into tensor memory, K and Q in shared memory.  What bounds it is the exponentials: rows * tokens of
// them at 16 a clock and SM, against rows * tokens * D / 4096 clocks of the products.  Two passes, each laid out so that a thread sums what it holds and no
// thread needs another's: for the lse the rows are the lanes of tensor memory and the tokens its columns, for the weights the other way round.  K is
// read by both (the second time mostly from L2).  Measured, 8 heads of 128 with 4 query heads each: 64 tokens of eight requests over 8209 tokens with the lse
// given 73 us (0.47 PFLOP/s; its exponentials alone 30 us at 16 a clock); 32 tokens over 10272, lse to be found, 30 us: five tiles a CTA, so the chain from
// the launch to the first scores counts twice.  8 of 32 exponentials of a full block go over the multipliers (12: 77 us).
//
// Warps 0-3 copy keys and queries (asynchronous 16-byte copies, a fence to the tensor core's proxy), warp 4 issues the products, warps 5-8 and 9-12 take
// the tiles in turn, each with two buffers of 128 columns.

constexpr int kTile = 128, kStagesK = 4, kTcThreads = 13 * 32;
template <int D> constexpr int tc_smem() { return 1024 + (kStagesK + 2) * kTile * D * 2; }

struct TcShared {
    unsigned long long k_full[kStagesK], k_empty[kStagesK], q_full[2], q_empty[2], s_full[4], s_empty[4], drained;
    uint32_t tmem;
    volatile int abort_flag;
    uint32_t there[kStagesK][4];            // which of a tile's tokens can be found
    float lse[2][kTile];                    // weights: what is added to a row's scores
    int last[2][kTile];                     // last token that a row sees
    uint32_t odd[2][4];                     // weights: some row's lse is -infinity
};

// LSE: units are (record, head, block of 128 rows, tile of 128 tokens); else (record, head, tile), with the blocks of rows one after the other inside.
// Units that share all but the tile are a segment.  One or two blocks of queries stay in shared memory for a segment, more pass by for every unit.
template <int D, bool LSE>
__global__ void __launch_bounds__(kTcThreads, 1) kdn_weigh_many_kernel(const __grid_constant__ WeighLaunch L)
{
    constexpr int kBytes = kTile * D * 2;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(8) TcShared sh;
    unsigned char *smem = raw + (1024 - (smem_u32(raw) & 1023u)) % 1024;
    const uint32_t keys = smem_u32(smem), queries = keys + kStagesK * kBytes;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    release_dependents();
    if (threadIdx.x == 0) {
        // a stage of keys is left by the products and by the four warps that took the tile; a block of queries by the products and all eight
        for (int i = 0; i < kStagesK; ++i) { mbar_init(smem_u32(&sh.k_full[i]), 128u); mbar_init(smem_u32(&sh.k_empty[i]), 5u); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&sh.q_full[i]), 128u); mbar_init(smem_u32(&sh.q_empty[i]), 9u); }
        for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&sh.s_full[i]), 1u); mbar_init(smem_u32(&sh.s_empty[i]), 4u); }
        mbar_init(smem_u32(&sh.drained), 1u);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 4) tc_alloc(smem_u32(&sh.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    dependency_wait();
    const uint32_t tmem = sh.tmem;
    const WeighRec *recs = records(L);
    const unsigned u0 = first_unit(blockIdx.x, L.units, gridDim.x), u1 = first_unit(blockIdx.x + 1, L.units, gridDim.x);

    // every role goes through the units in the same way
    int ri = record_of(recs, L.n, u0);
    WeighRec r = recs[ri];
    int blocks = (r.rows + kTile - 1) / kTile, seg = (int)((u0 - r.unit) / (unsigned)r.tiles), tile = (int)((u0 - r.unit) % (unsigned)r.tiles);
    bool fresh = true;                                           // the unit is the first of its segment here
    auto advance = [&]() {
        fresh = false;
        if (++tile < r.tiles) return;
        tile = 0;
        fresh = true;
        if (++seg < L.H * (LSE ? blocks : 1)) return;
        seg = 0;
        do r = recs[++ri]; while (r.tiles == 0);
        blocks = (r.rows + kTile - 1) / kTile;
    };
    auto wait = [&](unsigned long long &bar, unsigned parity) { return warp_wait(smem_u32(&bar), parity, &sh.abort_flag, L.wait_limit_ns); };
    unsigned nk = 0, nq = 0, base_q = 0;                         // tiles and blocks so far, and the first block of this unit
    bool ok = true;

    if (warp < 4) {
        // ------------------------------------------------------------------------------------ copies
        constexpr int kRowLanes = D / 8, kRows = 32 / kRowLanes, kPasses = 32 / kRows;            // a warp brings 32 rows, kRows at a time
        const int chunk = lane % kRowLanes, sub = lane / kRowLanes;
        const __nv_bfloat16 *pool = L.k_layers[L.layer];
        const uint32_t half = (uint32_t)(chunk / 8) * (kTile * 128u);
        // the set of copies before the one that is issued stays in flight, for the barrier `before`
        uint32_t before = 0u;
        auto drain = [&]() {
            copies_wait_all();
            fence_async_smem();
            if (before) mbar_arrive(before);
            before = 0u;
        };
        auto push = [&](uint32_t bar) {
            asm volatile("cp.async.commit_group;" ::: "memory");
            if (before) {
                asm volatile("cp.async.wait_group 1;" ::: "memory");
                fence_async_smem();
                mbar_arrive(before);
            }
            before = bar;
        };
        // what is waited for may itself wait for copies that are still in flight here
        auto claim = [&](unsigned long long &bar, unsigned parity) {
            if (!__all_sync(0xffffffffu, mbar_test(smem_u32(&bar), parity))) drain();
            return wait(bar, parity);
        };
        for (unsigned u = u0; u < u1 && ok; ++u) {
            if (u != u0) advance();
            const int h = LSE ? seg / blocks : seg, todo = LSE ? 1 : blocks;
            const bool queries_too = fresh || todo > 2;
            for (int b = -1; b < todo && ok; ++b) {              // block 0, the keys, blocks 1 ..
                const int block = b < 0 ? 0 : b;
                if (b != 0) {
                    if (!queries_too) continue;
                    const int buf = (int)(nq & 1u);
                    if (!(ok = claim(sh.q_empty[buf], ((nq >> 1) & 1u) ^ 1u))) break;
                    const int rho0 = (LSE ? seg % blocks : block) * kTile;
                    // a lane finds a row, all copy it
                    const int row = 32 * warp + lane, rho = rho0 + row;
                    const __nv_bfloat16 *mine = rho < r.rows ? query_of(L, r, h, rho, D) : nullptr;
                    const float x = !LSE && rho < r.rows ? L.lse[lse_at(L, r, h, rho)] : -INFINITY;
#pragma unroll
                    for (int p = 0; p < kPasses; ++p) {
                        const int i = p * kRows + sub;
                        const uint64_t from = __shfl_sync(0xffffffffu, (unsigned long long)mine, i);
                        const uint32_t to = queries + buf * kBytes + half + swizzled((uint32_t)(32 * warp + i), (uint32_t)(chunk & 7));
                        if (from) copy_async<16>(to, reinterpret_cast<const __nv_bfloat16 *>(from) + chunk * 8);
                        else asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(to), "r"(0u) : "memory");
                    }
                    const long long last = r.q_pos + rho / L.g;
                    sh.lse[buf][row] = x == -INFINITY ? -INFINITY : -x * 1.4426950408889634f;
                    sh.last[buf][row] = last > 0x7fffffff ? 0x7fffffff : (int)last;
                    const unsigned odd = __ballot_sync(0xffffffffu, rho < r.rows && x == -INFINITY);
                    if (lane == 0) sh.odd[buf][warp] = odd;
                    push(smem_u32(&sh.q_full[buf]));
                    ++nq;
                } else {
                    // a lane looks a token up, before the stage is waited for
                    const int st = (int)(nk % kStagesK), t = tile * kTile + 32 * warp + lane;
                    const long long mine = t < r.n_tokens ? key_row(L, r, t) : -1;
                    const uint32_t there = __ballot_sync(0xffffffffu, mine >= 0);
                    if (!(ok = claim(sh.k_empty[st], ((nk / kStagesK) & 1u) ^ 1u))) break;
                    const __nv_bfloat16 *from = pool + (mine + h) * D;
                    const uint32_t to = keys + st * kBytes + half;
#pragma unroll
                    for (int p = 0; p < kPasses; ++p) {
                        const int row = p * kRows + sub;
                        const uint64_t at = __shfl_sync(0xffffffffu, (unsigned long long)from, row);
                        if (there >> row & 1u)
                            copy_async<16>(to + swizzled((uint32_t)(32 * warp + row), (uint32_t)(chunk & 7)), reinterpret_cast<const __nv_bfloat16 *>(at) + chunk * 8);
                    }
                    if (lane == 0) sh.there[st][warp] = there;
                    push(smem_u32(&sh.k_full[st]));
                    ++nk;
                }
            }
        }
        drain();
    } else if (warp == 4) {
        // ------------------------------------------------------------------------------------ products
        const uint32_t what = mma_descriptor(kBf16, kTile, kTile, false);
        const uint64_t k_desc = tile_descriptor(keys, 16, 1024), q_desc = tile_descriptor(queries, 16, 1024);
        unsigned turn[2] = { 0u, 0u };
        for (unsigned u = u0; u < u1 && ok; ++u, ++nk) {
            if (u != u0) advance();
            const int st = (int)(nk % kStagesK), set = (int)((u - u0) & 1u), todo = LSE ? 1 : blocks;
            const bool bring = fresh || todo > 2, leave = todo > 2 || tile + 1 == r.tiles || u + 1 == u1;
            if (bring) { base_q = nq; nq += (unsigned)todo; }
            for (int b = 0; b < todo; ++b) {
                const unsigned qi = base_q + (unsigned)b;
                const int buf = 2 * set + (int)(turn[set] & 1u);
                if (bring) ok = wait(sh.q_full[qi & 1u], (qi >> 1) & 1u);
                if (ok && b == 0) ok = wait(sh.k_full[st], (nk / kStagesK) & 1u);
                if (ok) ok = wait(sh.s_empty[buf], ((turn[set] >> 1) & 1u) ^ 1u);
                if (!ok) break;
                ++turn[set];
                tc_fence_after();
                if (one_lane()) {
                    const uint64_t k0 = k_desc + (uint64_t)(st * kBytes / 16), q0 = q_desc + (uint64_t)((qi & 1u) * kBytes / 16);
                    const uint64_t a0 = LSE ? q0 : k0, b0 = LSE ? k0 : q0;
#pragma unroll
                    for (int s = 0; s < D / 16; ++s)
                        tc_mma(tmem + buf * 128u, a0 + (s / 4) * (kTile * 128 / 16) + (s % 4) * 2, b0 + (s / 4) * (kTile * 128 / 16) + (s % 4) * 2, what, s > 0);
                    tc_commit(smem_u32(&sh.s_full[buf]));
                    if (b == todo - 1) tc_commit(smem_u32(&sh.k_empty[st]));
                    if (leave) tc_commit(smem_u32(&sh.q_empty[qi & 1u]));
                }
                __syncwarp();
            }
        }
        if (one_lane()) tc_commit(smem_u32(&sh.drained));
        __syncwarp();
        volatile int never = 0;                                  // products in flight end by themselves
        mbar_wait(smem_u32(&sh.drained), 0u, &never, 2000000000ull);
    } else {
        // -------------------------------------------------------------------------------- exponentials
        const int set = (warp - 5) / 4, quad = warp & 3, place = quad * 32 + lane;                // lanes of tensor memory go by the warp's number modulo 4
        unsigned turn = 0;
        float m = -INFINITY, l = 0.0f;
        for (unsigned u = u0; u < u1 && ok; ++u, ++nk) {
            if (u != u0) advance();
            const int h = LSE ? seg / blocks : seg, todo = LSE ? 1 : blocks, t0 = tile * kTile, st = (int)(nk % kStagesK);
            const bool over = tile + 1 == r.tiles || u + 1 == u1, leave = todo > 2 || over, mine = ((u - u0) & 1u) == (unsigned)set;
            if (fresh || todo > 2) { base_q = nq; nq += (unsigned)todo; }
            if (LSE && fresh) { m = -INFINITY; l = 0.0f; }
            float sum = 0.0f, was = 0.0f;
            uint32_t there = 0u;
            float *acc = LSE ? nullptr : r.acc + (long long)h * r.acc_stride + t0 + place;
            const bool inside = t0 + place < r.n_tokens;
            if (!LSE && mine && inside) was = *acc;
            for (int b = 0; b < todo && ok; ++b) {
                const unsigned qi = base_q + (unsigned)b;
                const int qb = (int)(qi & 1u);
                if (mine) {
                    const int buf = 2 * set + (int)(turn & 1u);
                    if (!(ok = wait(sh.s_full[buf], (turn >> 1) & 1u))) break;
                    ++turn;
                    tc_fence_after();
                    const uint32_t at = tmem + buf * 128u + ((uint32_t)(quad * 32) << 16);
                    if (LSE) {
                        const int last = sh.last[qb][place] - t0, tokens = r.n_tokens - t0;
                        const uint32_t th[4] = { sh.there[st][0], sh.there[st][1], sh.there[st][2], sh.there[st][3] };
                        const bool all = __all_sync(0xffffffffu, last >= kTile - 1 && (th[0] & th[1] & th[2] & th[3]) == 0xffffffffu);
                        auto some = [&](uint32_t (&x)[32], int c0) {
                            if (!all) {
                                const uint32_t found = th[c0 / 32];
#pragma unroll
                                for (int i = 0; i < 32; ++i)
                                    if (!(found >> i & 1u) || c0 + i > last) x[i] = 0xff800000u;
                            }
                            float t0 = -INFINITY, t1 = -INFINITY;
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                t0 = fmaxf(t0, __uint_as_float(x[i]));
                                t1 = fmaxf(t1, __uint_as_float(x[i + 1]));
                            }
                            const float top = fmaxf(t0, t1) * L.scale;
                            if (top > m + 8.0f) {                // the reference moves when it has to, and so seldom
                                l *= exp2_approx(m - top);
                                m = top;
                            }
                            float by = L.scale;
                            if (__any_sync(0xffffffffu, fabsf(top) > kHugeScore && top != -INFINITY) && fabsf(top) > kHugeScore) {
                                by = 1.0f;
#pragma unroll
                                for (int i = 0; i < 32; ++i) x[i] = __float_as_uint(__uint_as_float(x[i]) * L.scale);
                            }
                            const float base = m == -INFINITY ? 0.0f : -m;
                            const f32x2 scale2 = pack2(by, by), base2 = pack2(base, base);
                            f32x2 sum2 = pack2(0.0f, 0.0f);
#pragma unroll
                            for (int i = 0; i < 32; i += 2) {
                                float e0, e1;
                                unpack2(fma2(pack2(__uint_as_float(x[i]), __uint_as_float(x[i + 1])), scale2, base2), e0, e1);
                                sum2 = add2(sum2, pack2(exp2_approx(e0), exp2_approx(e1)));
                            }
                            float l0, l1;
                            unpack2(sum2, l0, l1);
                            l += l0 + l1;
                        };
                        // the next 32 columns are on their way while these are worked on (all that stand in tensor memory may be read)
                        uint32_t x[32], y[32];
                        tc_load32(x, at);
#pragma unroll 1
                        for (int c0 = 0; c0 < kTile && c0 < tokens; c0 += 64) {
                            tc_wait_loads();
                            tc_load32(y, at + c0 + 32u);
                            some(x, c0);
                            tc_wait_loads();
                            if (c0 + 64 < kTile) tc_load32(x, at + c0 + 64u);
                            if (c0 + 32 < tokens) some(y, c0 + 32);
                        }
                        tc_wait_loads();
                    } else {
                        if (b == 0) there = sh.there[st][quad];
                        const int rows = r.rows - b * kTile < kTile ? r.rows - b * kTile : kTile;
                        const bool all = rows == kTile && (long long)(t0 + kTile - 1) <= r.q_pos && !(sh.odd[qb][0] | sh.odd[qb][1] | sh.odd[qb][2] | sh.odd[qb][3]);
                        auto some = [&](const uint32_t (&x)[32], int c0) {
                            if (all) {
                                const float4 *ls = reinterpret_cast<const float4 *>(&sh.lse[qb][c0]);
                                const f32x2 scale2 = pack2(L.scale, L.scale);
                                f32x2 sum2 = pack2(0.0f, 0.0f);
#pragma unroll
                                for (int i = 0; i < 8; ++i) {
                                    const float4 v = ls[i];
                                    const f32x2 a = fma2(pack2(__uint_as_float(x[4 * i]), __uint_as_float(x[4 * i + 1])), scale2, pack2(v.x, v.y));
                                    const f32x2 b = fma2(pack2(__uint_as_float(x[4 * i + 2]), __uint_as_float(x[4 * i + 3])), scale2, pack2(v.z, v.w));
                                    if (i % 8 == 2 || i % 8 == 6) {        // 8 of 32 beside the special-function unit
                                        sum2 = fma2(half_exp2_pair(a), pack2(2.0f, 2.0f), sum2);
                                        sum2 = fma2(half_exp2_pair(b), pack2(2.0f, 2.0f), sum2);
                                    } else {
                                        float e0, e1, e2, e3;
                                        unpack2(a, e0, e1);
                                        unpack2(b, e2, e3);
                                        sum2 = add2(sum2, pack2(exp2_approx(e0), exp2_approx(e1)));
                                        sum2 = add2(sum2, pack2(exp2_approx(e2), exp2_approx(e3)));
                                    }
                                }
                                float s0, s1;
                                unpack2(sum2, s0, s1);
                                sum += s0 + s1;
                            } else {
                                float s0 = 0.0f;
#pragma unroll
                                for (int i = 0; i < 32; ++i) {
                                    const float v = sh.lse[qb][c0 + i], e = exp2_approx(fmaf(__uint_as_float(x[i]), L.scale, v));
                                    s0 += t0 + place <= sh.last[qb][c0 + i] && v != -INFINITY ? e : 0.0f;
                                }
                                sum += s0;
                            }
                        };
                        uint32_t x[32], y[32];
                        tc_load32(x, at);
#pragma unroll 1
                        for (int c0 = 0; c0 < rows; c0 += 64) {
                            tc_wait_loads();
                            tc_load32(y, at + c0 + 32u);
                            some(x, c0);
                            tc_wait_loads();
                            if (c0 + 64 < kTile) tc_load32(x, at + c0 + 64u);
                            if (c0 + 32 < rows) some(y, c0 + 32);
                        }
                        tc_wait_loads();
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        mbar_arrive(smem_u32(&sh.s_empty[buf]));
                        if (b == todo - 1) mbar_arrive(smem_u32(&sh.k_empty[st]));
                    }
                }
                if (leave) {
                    // (a warp that has not read the block leaves it no sooner than it is there: the buffer's turn before is over by then)
                    if (!mine && !(ok = wait(sh.q_full[qb], (qi >> 1) & 1u))) break;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&sh.q_empty[qb]));
                }
            }
            if (!LSE && ok && mine && inside && (there >> lane & 1u)) *acc = was + sum;
            if (LSE && ok && over) {
                const unsigned slot = (blockIdx.x + (unsigned)(r.segment + seg)) * 2u + (unsigned)set;
                L.stats[(long long)slot * kTile + place] = make_float2(m, l);
            }
        }
    }
    if (sh.abort_flag && lane == 0) atomicCAS(L.status, 0, kStatusTimeout);
    tc_fence_before();
    __syncthreads();
    if (warp == 4) tc_free(tmem, 512);
}

// The lse of each row from its parts' maxima and sums, a warp a row.
__global__ void __launch_bounds__(256) kdn_weigh_lse_kernel(const __grid_constant__ WeighLaunch L, unsigned ctas)
{
    release_dependents();
    dependency_wait();
    const WeighRec *recs = records(L);
    const int lane = threadIdx.x & 31;
    const int head = (int)blockIdx.y, h = head / L.g;
    for (int ri = (int)blockIdx.z; ri < L.n; ri += (int)gridDim.z) {
        const WeighRec r = recs[ri];
        for (int i = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)); i < r.rows / L.g; i += (int)gridDim.x * 8) {
            const int rho = i * L.g + head % L.g;
            float m = -INFINITY, l = 0.0f;
            if (r.tiles > 0) {
                const unsigned blocks = (unsigned)((r.rows + kTile - 1) / kTile);
                const unsigned seg = (unsigned)h * blocks + (unsigned)(rho / kTile), s0 = r.unit + seg * (unsigned)r.tiles, s1 = s0 + (unsigned)r.tiles;
                const unsigned c0 = cta_of(s0, L.units, ctas), n = (cta_of(s1 - 1, L.units, ctas) - c0 + 1) * 2u, first = (c0 + (unsigned)r.segment + seg) * 2u;
                for (unsigned j = (unsigned)lane; j < n; j += 32) {
                    const float2 ml = L.stats[(long long)(first + j) * kTile + rho % kTile];
                    if (ml.y == 0.0f) continue;
                    const float top = fmaxf(m, ml.x), base = top == -INFINITY ? 0.0f : top;
                    l = l * exp2_approx(m - base) + ml.y * exp2_approx(ml.x - base);
                    m = top;
                }
            }
            for (int d = 16; d; d >>= 1) {
                const float m2 = __shfl_xor_sync(0xffffffffu, m, d), l2 = __shfl_xor_sync(0xffffffffu, l, d);
                const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
                l = l * exp2_approx(m - base) + l2 * exp2_approx(m2 - base);
                m = top;
            }
            if (lane == 0) L.lse[lse_at(L, r, h, rho)] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
        }
    }
}

struct Layout {
    unsigned few_workers, many_ctas;
    size_t recs, lse, stats, scores, whole;
};

// From sizes alone, so that a workspace stays large enough while positions move.
Layout layout_of(const kdn_pool_desc &pool, const kdn_weigh_req *reqs, int n, int n_q_heads, bool given, int sm_count)
{
    Layout w{};
    const int H = pool.n_kv_heads, g = n_q_heads / H;
    size_t rows = 0, scores = 0, few_segments = 0, many_segments = 0;
    for (int i = 0; i < n; ++i) {
        const kdn_weigh_req &q = reqs[i];
        const size_t r = (size_t)q.n_q * (size_t)g;
        rows += (size_t)q.n_q;
        if (r <= (size_t)kFewRows) few_segments += r ? (size_t)H : 0;
        else many_segments += (size_t)H * ((r + kTile - 1) / kTile);
        if ((int64_t)q.n_q * g <= kFewRows) scores += align_up((size_t)H * (size_t)q.n_q * (size_t)g * (size_t)q.n_tokens, 4);
    }
    w.few_workers = 2u * (unsigned)sm_count * kFewWarps;
    w.many_ctas = (unsigned)sm_count;
    w.recs = n > kInline ? align_up(sizeof(WeighRec) * (size_t)n, 256) : 0;
    if (!given) {
        w.lse = align_up(rows * (size_t)n_q_heads * 4, 256);
        const size_t few = (w.few_workers + few_segments) * kFewRows, many = (w.many_ctas + many_segments) * 2 * kTile;
        w.stats = align_up((few > many ? few : many) * sizeof(float2), 256);
        w.scores = scores * 4;
    }
    w.whole = w.recs + w.lse + w.stats + w.scores;
    return w;
}

template <int D>
kdn_status launch_few(const Context &c, const WeighLaunch &L, int rows, bool given, unsigned ctas, cudaStream_t stream)
{
    if (rows <= 8)
        return given ? launch(c, kdn_weigh_few_kernel<D, 1, true>, dim3(ctas), kFewWarps * 32, 0, stream, L)
                     : launch(c, kdn_weigh_few_kernel<D, 1, false>, dim3(ctas), kFewWarps * 32, 0, stream, L);
    return given ? launch(c, kdn_weigh_few_kernel<D, 2, true>, dim3(ctas), kFewWarps * 32, 0, stream, L)
                 : launch(c, kdn_weigh_few_kernel<D, 2, false>, dim3(ctas), kFewWarps * 32, 0, stream, L);
}

template <int D, bool LSE>
kdn_status launch_many(const Context &c, const WeighLaunch &L, unsigned ctas, cudaStream_t stream)
{
    const kdn_status st = allow_smem<kdn_weigh_many_kernel<D, LSE>>(c, tc_smem<D>());
    return st != KDN_OK ? st : launch(c, kdn_weigh_many_kernel<D, LSE>, dim3(ctas), kTcThreads, (size_t)tc_smem<D>(), stream, L);
}

kdn_status check_reqs(const kdn_pool_desc *pool, const kdn_weigh_req *reqs, int n_reqs, int n_q_heads)
{
    kdn_status st = check_pool_shape(pool);
    if (st != KDN_OK) return st;
    if (n_reqs < 0 || (n_reqs > 0 && !reqs)) return KDN_E_INVAL;
    if (n_q_heads <= 0 || n_q_heads % pool->n_kv_heads) return KDN_E_INVAL;
    if (pool->head_dim != 64 && pool->head_dim != 128) return KDN_E_UNSUPPORTED;
    if (n_q_heads > 65535) return KDN_E_UNSUPPORTED;
    int64_t rows = 0;
    uint64_t units = 0;
    for (int i = 0; i < n_reqs; ++i) {
        const kdn_weigh_req &q = reqs[i];
        if (q.n_q < 0 || q.n_table_blocks < 0 || q.n_tokens < 0 || q.q_pos < 0 || q.q_pos >= (int64_t)1 << 40) return KDN_E_INVAL;
        if (q.n_tokens > (int64_t)q.n_table_blocks * pool->block_size) return KDN_E_RANGE;
        rows += q.n_q;
        if (rows * n_q_heads > 0x7fffffff || q.n_tokens > kMostTokens) return KDN_E_UNSUPPORTED;
        // what the kernels number their work by: at most (few rows) a tile of 32 tokens of a head, or (many) of 128 by 128 rows
        units += (((uint64_t)q.n_tokens + kFewTokens - 1) / kFewTokens) * (uint64_t)pool->n_kv_heads *
                 ((uint64_t)q.n_q * (unsigned)(n_q_heads / pool->n_kv_heads) / kTile + 1);
        if (units > 0x7fffffffull) return KDN_E_UNSUPPORTED;
        if (q.n_tokens == 0) continue;
        if (!q.block_table || !q.acc || q.acc_stride < q.n_tokens) return KDN_E_INVAL;
        if (!aligned(q.acc, 4) || !aligned(q.block_table, 4)) return KDN_E_ALIGN;
    }
    return KDN_OK;
}

}  // namespace

extern "C" {

kdn_status kdn_validate_weigh(const kdn_pool_desc *pool, int layer, const kdn_weigh_req *reqs, int n_reqs, const kdn_weigh_io *io)
{
    if (!io) return KDN_E_INVAL;
    const kdn_status st = check_reqs(pool, reqs, n_reqs, io->n_q_heads);
    if (st != KDN_OK) return st;
    if (layer < 0 || layer >= pool->n_layers) return KDN_E_INVAL;
    if (!usable_scale(io->scale)) return KDN_E_INVAL;
    int64_t rows = 0;
    for (int i = 0; i < n_reqs; ++i) rows += reqs[i].n_q;
    if (rows == 0) return KDN_OK;
    if (!io->q || io->q_stride < (int64_t)io->n_q_heads * pool->head_dim || (io->lse_given && !io->lse)) return KDN_E_INVAL;
    if (!aligned(io->q, 16) || io->q_stride % 8 || !aligned(io->lse, 4)) return KDN_E_ALIGN;
    return KDN_OK;
}

kdn_status kdn_weigh_workspace(kdn_ctx *ctx, int pool_id, const kdn_weigh_req *reqs, int n_reqs, int n_q_heads, int lse_given, size_t *bytes)
{
    Context c;
    PoolShape pool;
    if (!bytes || !context_of(ctx, &c) || !pool_of(ctx, pool_id, &pool)) return KDN_E_INVAL;
    *bytes = 0;
    const kdn_status st = check_reqs(&pool.desc, reqs, n_reqs, n_q_heads);
    if (st == KDN_OK) *bytes = layout_of(pool.desc, reqs, n_reqs, n_q_heads, lse_given != 0, c.sm_count).whole;
    return st;
}

kdn_status kdn_weigh(kdn_ctx *ctx, int pool_id, int layer, const kdn_weigh_req *reqs, int n_reqs, const kdn_weigh_io *io, void *cuda_stream)
{
    Context c;
    PoolShape pool;
    if (!context_of(ctx, &c) || !pool_of(ctx, pool_id, &pool)) return KDN_E_INVAL;
    kdn_status st = kdn_validate_weigh(&pool.desc, layer, reqs, n_reqs, io);
    if (st != KDN_OK) return st;
    const bool given = io->lse_given != 0;
    const Layout w = layout_of(pool.desc, reqs, n_reqs, io->n_q_heads, given, c.sm_count);
    if (w.whole && (!io->workspace || io->workspace_bytes < w.whole)) return KDN_E_INVAL;
    if (!aligned(io->workspace, 16)) return KDN_E_ALIGN;
    if (make_current(c.device) != KDN_OK) return KDN_E_CUDA;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    unsigned char *at = static_cast<unsigned char *>(io->workspace);
    WeighLaunch L{};
    L.q = static_cast<const __nv_bfloat16 *>(io->q);
    L.q_stride = io->q_stride;
    L.lse = io->lse ? io->lse : reinterpret_cast<float *>(at + w.recs);
    L.stats = reinterpret_cast<float2 *>(at + w.recs + w.lse);
    L.scores = reinterpret_cast<float *>(at + w.recs + w.lse + w.stats);
    L.k_layers = reinterpret_cast<const __nv_bfloat16 *const *>(pool.k_layers);
    L.n_blocks = pool.desc.n_blocks;
    L.wait_limit_ns = c.wait_limit_ns;
    L.status = c.status;
    L.scale = (float)(io->scale * kLog2e);
    L.layer = layer;
    L.H = pool.desc.n_kv_heads;
    L.g = io->n_q_heads / L.H;
    L.bs = pool.desc.block_size;
    const bool d64 = pool.desc.head_dim == 64;
    std::vector<WeighRec> recs;
    try { recs.reserve((size_t)n_reqs); } catch (const std::bad_alloc &) { return KDN_E_NOMEM; }
    long long score = 0;
    for (int many = 0; many < 2; ++many) {                 // requests of few rows a head, then those of many
        recs.clear();
        int row = 0, rows = 0, n_q = 0, tokens = 0, segment = 0;
        unsigned long long units = 0;
        for (int i = 0; i < n_reqs; row += reqs[i].n_q, ++i) {
            const kdn_weigh_req &q = reqs[i];
            if (q.n_q == 0 || ((int64_t)q.n_q * L.g > kFewRows) != (many != 0)) continue;
            const int64_t seen = q.q_pos + q.n_q < q.n_tokens ? q.q_pos + q.n_q : q.n_tokens;
            const int tiles = (int)((seen + (many ? kTile : kFewTokens) - 1) / (many ? kTile : kFewTokens));
            const int r = q.n_q * L.g;
            recs.push_back(WeighRec{ q.block_table, q.acc, q.acc_stride, q.q_pos, (int)seen, row, r, 0u, tiles, segment, score });
            segment += L.H * (many ? (r + kTile - 1) / kTile : 1);
            units += (unsigned long long)tiles * (unsigned)L.H;
            if (!many) score += (long long)align_up((size_t)L.H * (size_t)r * (size_t)q.n_tokens, 4);
            rows = r > rows ? r : rows;
            n_q = q.n_q > n_q ? q.n_q : n_q;
            tokens = (int)seen > tokens ? (int)seen : tokens;
        }
        const int n = (int)recs.size();
        if (n == 0) continue;
        const unsigned most = many ? w.many_ctas : w.few_workers / kFewWarps;
        // the records, with the units numbered for the kernel that is next
        auto send = [&](bool by_rows) -> kdn_status {
            unsigned u = 0;
            for (WeighRec &r : recs) {
                r.unit = u;
                u += (unsigned)r.tiles * (unsigned)L.H * (by_rows ? (unsigned)((r.rows + kTile - 1) / kTile) : 1u);
            }
            L.units = u;
            L.n = n;
            L.recs = nullptr;
            if (n <= kInline) {
                std::memcpy(L.inl, recs.data(), sizeof(WeighRec) * (size_t)n);
                return KDN_OK;
            }
            L.recs = reinterpret_cast<const WeighRec *>(at);
            return put_records(c, at, recs.data(), sizeof(WeighRec) * (size_t)n, stream);
        };
        const dim3 by_row((unsigned)((n_q + 7) / 8), (unsigned)io->n_q_heads, (unsigned)(n < 65535 ? n : 65535));
        if (many) {
            if (!given) {
                if ((st = send(true)) != KDN_OK) return st;
                const unsigned ctas = L.units < most ? L.units : most;
                if (ctas) st = d64 ? launch_many<64, true>(c, L, ctas, stream) : launch_many<128, true>(c, L, ctas, stream);
                if (st == KDN_OK) st = launch(c, kdn_weigh_lse_kernel, by_row, 256, 0, stream, L, ctas);
                if (st != KDN_OK) return st;
            }
            if (units == 0) continue;
            if ((st = send(false)) != KDN_OK) return st;
            const unsigned ctas = L.units < most ? L.units : most;
            st = d64 ? launch_many<64, false>(c, L, ctas, stream) : launch_many<128, false>(c, L, ctas, stream);
        } else {
            if ((st = send(false)) != KDN_OK) return st;
            const unsigned all = (L.units + kFewWarps - 1) / kFewWarps, ctas = all < most ? all : most;
            if (ctas) st = d64 ? launch_few<64>(c, L, rows, given, ctas, stream) : launch_few<128>(c, L, rows, given, ctas, stream);
            if (st == KDN_OK && !given) {
                const dim3 by_token((unsigned)(tokens ? (tokens + 1023) / 1024 : 1), (unsigned)L.H, by_row.z);
                st = launch(c, rows <= 8 ? kdn_weigh_add_scores_kernel<8> : kdn_weigh_add_scores_kernel<16>, by_token, 256, 0, stream, L, few_workers(ctas, L.units));
            }
        }
        if (st != KDN_OK) return st;
    }
    return KDN_OK;
}

}  // extern "C"
