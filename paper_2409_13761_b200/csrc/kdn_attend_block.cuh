// Attention of many new tokens over stored 4-bit chunks, on the tensor core.
//
// Mathematics as for a few (kdn_attend_step.cuh), other places for the scales.  Rows of queries are the lanes of tensor memory, 64 tokens of a tile its
// columns:  S = Q K^T with K = code * scale as the sum of two fp16 matrices (scale = a number of eight bits, whose products with a code are exact, and what
// that leaves, to 11 bits) and Q, turned and times a power of two, as the sum of two more (the second is nothing, and left out, where the queries are taken as they came);  P = exp(S) *
// value scale, bf16, one matrix for each group of 64 channels;  O += P C with C the value codes, exact in bf16.  The keys of a tile are held times a
// power of two that brings the largest of their scales to 2^11, or, where scales are more than 2^12 apart, each token's times one of its own, which its
// column of S is multiplied by before the softmax.  P is rounded once (2^-9 relative): tensor memory has no room for a second number, and fp16 not the
// range that scales need; the result is 1.4 to 1.5 times as far off (root mean square, against 64 bits) as its own rounding alone makes it.
//
// What bounds it: shared memory's 128 bytes a clock, at about four fifths.  A tile of 64 tokens by 256 rows takes some 4200 clocks (four requests of 512
// over 8192: 465 thousand for 111 tiles), of which the operands of the products take 1800 (queries as they came) or 2600 (turned: a third product), what the warps store and load themselves 1600 (operands, the values' scales, waits);
// the products alone would take 1500, the exponentials 1024 at 16 a clock, the instructions half of the issue slots.  Over ten documents, turned, it is 5500 (180 thousand
// for 33 tiles): the third product, and the pipeline runs dry where a part brings queries of its own, whatever it turns by.  Without any softmax or without any expanding of codes a
// call is up to 9 per cent faster, without both up to 13.  Measured, 8 heads of 128: 203 tokens over ten documents of 1024 125 us (0.26 PFLOP/s); four
// requests of 512 tokens over 8192, two heads of 8 query heads each, keys in channel groups: 296 us (0.47 PFLOP/s); the first with key scales over eight orders
// of magnitude 128 us.  A CTA takes 256 rows as two sets of 128, so that codes are expanded once for both.  A set's scores are made a
// tile ahead of its softmax, which turns them into P in place: 16 columns of S become the 8 of P that go with one group and the 8 that go with the
// other, just what one product of 16 tokens reads.  Warps 0-3 and 4-7 are the softmax of a set, a row a thread; warps 8-11 expand codes; warps 12
// and 13 issue the products of a set each (one for both was what everything waited for: 40 to 60 clocks a product).
#pragma once
#include "kdn_attend_step.cuh"
#include "kdn_tc.cuh"

#include <type_traits>

namespace kdn {

constexpr int kBlockRows = 256, kBlockTile = 64, kBlockThreads = 14 * 32;
template <int D> struct BlockShape {
    static constexpr int NG = D / 64;
    static constexpr int kQ = 128 * D * 2;                                // one half (leading, rest) of a set's queries
    static constexpr int kK = kBlockTile * D * 2;                         // one half of a tile's keys; also a tile's values
    static constexpr int kSmem = 1024 + 4 * kQ + 4 * kK + kK;             // queries of two sets, two tiles of keys, one of values
};

struct BlockShared {
    unsigned long long k_full[2], k_empty[2], v_full, v_empty, q_full[2], s_full[2][2], p_full[2][2], o_full[2], drained;
    uint32_t tmem;
    volatile int abort_flag;
    // Of the tiles under way, by tile number modulo 4.  key_power: what the tile's keys were divided by, or 0 where each token's were divided by a power
    // of its own (key_column).
    float value_scale[4][2][kBlockTile], key_power[4], key_column[4][kBlockTile];
    float2 table[8][64];                                                  // rotation of the part, for each softmax warp
    uint32_t channel[4][2][32];                                           // codes in channel groups: a warp's 64 channels' scales, leading and rest
};

// Units are (request, block of 256 rows, head, tile of 64 tokens), tiles fastest; those that share all but the tile are a segment.
struct BlockWalk {
    const ReqRec *reqs;
    const PartRec *parts;
    ReqRec r;
    int ri, seg, tile, pi, part_first, part_end;
    int head, row0, sets;                   // of the segment: KV head, first row, sets that have rows
    bool new_seg, new_part;
    __device__ __forceinline__ void enter_part(int i)
    {
        pi = i;
        part_first = parts[r.part + i].tile;
        part_end = i + 1 < r.n_parts ? parts[r.part + i + 1].tile : r.tiles;
        new_part = true;
    }
    __device__ __forceinline__ void enter_segment(int H)
    {
        head = seg % H;
        row0 = seg / H * kBlockRows;
        sets = r.rows - row0 > 128 ? 2 : 1;
        new_seg = true;
    }
    __device__ __forceinline__ void start(const AttendLaunch &L, unsigned u, int lane)
    {
        reqs = L.reqs ? L.reqs : L.inl_reqs;
        parts = L.reqs ? L.parts : L.inl_parts;
        ri = last_at_most(L.n_reqs, [&](int i) { return reqs[i].unit; }, u, lane);
        r = reqs[ri];
        seg = (int)((u - r.unit) / (unsigned)r.tiles);
        tile = (int)((u - r.unit) % (unsigned)r.tiles);
        enter_part(last_at_most(r.n_parts, [&](int i) { return (unsigned)parts[r.part + i].tile; }, (unsigned)tile, lane));
        enter_segment(L.H);
    }
    __device__ __forceinline__ void step(int H)
    {
        new_seg = new_part = false;
        if (++tile < r.tiles) {
            if (tile == part_end) enter_part(pi + 1);
            return;
        }
        tile = 0;
        if (++seg == H * ((r.rows + kBlockRows - 1) / kBlockRows)) { seg = 0; r = reqs[++ri]; }
        enter_part(0);
        enter_segment(H);
    }
};

// a = h + l: eight bits each
__device__ __forceinline__ void split_scale(float a, float &h, float &l)
{
    h = __uint_as_float((__float_as_uint(a) + 0x8000u) & 0xffff0000u);
    l = a - h;
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ void store16(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t from)
{
    uint4 x;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(from) : "memory");
    return x;
}
// 2^-e and 2^e for the exponent of a (0 and subnormal numbers, infinities and NaN: the nearest that both can hold)
__device__ __forceinline__ void powers_of(float a, float &down, float &up)
{
    int e = (int)(__float_as_uint(a) >> 23 & 255u);
    e = e < 2 ? 2 : e > 252 ? 252 : e;
    down = __uint_as_float((unsigned)(254 - e) << 23);
    up = __uint_as_float((unsigned)e << 23);
}
// Powers of two that bring a scale of exponent field e (at least kLeastKey counts) to 2^kKeyTop and over, and back: times a code of 8 it is below 2^15 in fp16, and 2^-12
// of it still has all the bits of an fp32 scale above fp16's smallest step, 2^-24.
constexpr int kKeyTop = 11, kKeySpread = 12, kLeastKey = 14;
__device__ __forceinline__ void key_powers(int e, float &down, float &up)
{
    e = e < kLeastKey ? kLeastKey : e > 254 ? 254 : e;
    down = __uint_as_float((unsigned)(254 + kKeyTop - e) << 23);
    up = __uint_as_float((unsigned)(e - kKeyTop) << 23);
}

template <int D>
__global__ void __launch_bounds__(kBlockThreads, 1) kdn_attend_block_kernel(const __grid_constant__ AttendLaunch L)
{
    using S = BlockShape<D>;
    constexpr int NG = S::NG;
    extern __shared__ unsigned char raw[];
    __shared__ __align__(16) BlockShared sh;
    unsigned char *smem = raw + (1024 - (smem_u32(raw) & 1023u)) % 1024;
    const uint32_t q_at = smem_u32(smem), k_at = q_at + 4 * S::kQ, v_at = k_at + 4 * S::kK;      // [set][half], [buffer][half]
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    release_dependents();
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.k_full[i]), 128u); mbar_init(smem_u32(&sh.k_empty[i]), 2u);
            mbar_init(smem_u32(&sh.q_full[i]), 128u); mbar_init(smem_u32(&sh.s_full[i][0]), 1u); mbar_init(smem_u32(&sh.s_full[i][1]), 1u);
            mbar_init(smem_u32(&sh.p_full[i][0]), 128u); mbar_init(smem_u32(&sh.p_full[i][1]), 128u); mbar_init(smem_u32(&sh.o_full[i]), 1u);
        }
        mbar_init(smem_u32(&sh.v_full), 128u);
        mbar_init(smem_u32(&sh.v_empty), 2u);
        mbar_init(smem_u32(&sh.drained), 2u);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 12) tc_alloc(smem_u32(&sh.tmem), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    // tensor memory of a set: twice 64 columns of S and then P, D of O
    const uint32_t tmem = sh.tmem;
    const unsigned u0 = first_unit(blockIdx.x, L.units, gridDim.x), u1 = first_unit(blockIdx.x + 1, L.units, gridDim.x);
    auto wait = [&](unsigned long long &bar, unsigned parity) { return warp_wait(smem_u32(&bar), parity, &sh.abort_flag, L.wait_limit_ns); };
    bool ok = true;
    BlockWalk w;
    if (L.reqs) dependency_wait();                               // records that are launch parameters can be read before
    w.start(L, u0, lane);
    if (!L.reqs) dependency_wait();

    if (warp < 8) {
        // ------------------------------------------------------------------------------------- softmax
        const int set = warp >> 2, place = (int)threadIdx.x & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t s_base = tmem + set * 256u + lanes, o_col = s_base + 128u;
        const uint32_t q_hi = q_at + set * 2 * S::kQ, q_lo = q_hi + S::kQ;
        unsigned turns = 0;                                      // tiles taken
        float m = -INFINITY, l = 0.0f, factor = 0.0f, up = 0.0f;
        int rho = 0, seen = 0, token = 0;                        // row, tokens of the part that some row sees, new token of the row
        long long ahead = 0;
        const __nv_bfloat16 *q = nullptr;
        for (unsigned u = u0; u < u1 && ok; ++u) {
            if (u != u0) w.step(L.H);
            if (set >= w.sets) continue;
            const int h = w.head;
            if (w.new_seg) {
                rho = w.row0 + set * 128 + place;
                token = rho / L.g;
                q = rho < w.r.rows ? L.q + (long long)(w.r.row + token) * L.q_stride + (long long)(h * L.g + rho % L.g) * D : nullptr;
                m = -INFINITY;
                l = 0.0f;
            }
            if (w.new_part) {
                const PartRec &p = w.parts[w.r.part + w.pi];
                ahead = p.ahead;
                seen = p.seen;
                // this row's queries, turned; within eight channels in the order in which words of codes come apart: 0 4 1 5 2 6 3 7
                const long long turn = p.turn;
                if (turn) {
                    __syncwarp();
                    for (int i = lane; i < D / 2; i += 32) sh.table[warp][i] = turn_of(L.turns[i], turn);
                    __syncwarp();
                }
                // The warp brings its rows, whole rows at a time, to where their second halves will stand; each thread then goes through its own.
                constexpr int kRowLanes = D / 8, kRowsAtOnce = 32 / kRowLanes;
                const uint32_t copy_to = q_lo + (uint32_t)(lane % kRowLanes / 8) * (128u * 128u);
#pragma unroll 4
                for (int i = lane / kRowLanes; i < 32; i += kRowsAtOnce) {
                    const uint64_t from = __shfl_sync(0xffffffffu, (unsigned long long)q, i);
                    const uint32_t to = copy_to + swizzled((uint32_t)((warp & 3) * 32 + i), (uint32_t)(lane & 7 & (kRowLanes - 1)));
                    if (from) copy_async<16>(to, reinterpret_cast<const __nv_bfloat16 *>(from) + lane % kRowLanes * 8);
                    else store16(to, 0u, 0u, 0u, 0u);
                }
                copies_wait_all();
                __syncwarp();
                auto at = [&](int i) { return D == 128 ? (uint32_t)(i / 8) * (128u * 128u) + swizzled((uint32_t)place, (uint32_t)(i % 8)) : swizzled((uint32_t)place, (uint32_t)i); };
                if (w.new_seg) {
                    float most = 0.0f;                           // a turned channel is at most 2^1/2 times this
#pragma unroll 4
                    for (int i = 0; i < D / 8; ++i) {
                        const uint4 x = load16(q_lo + at(i));
                        most = fmaxf(most, fmaxf(fmaxf(fabsf(bf16_lo(x.x)), fabsf(bf16_hi(x.x))), fmaxf(fabsf(bf16_lo(x.y)), fabsf(bf16_hi(x.y)))));
                        most = fmaxf(most, fmaxf(fmaxf(fabsf(bf16_lo(x.z)), fabsf(bf16_hi(x.z))), fmaxf(fabsf(bf16_lo(x.w)), fabsf(bf16_hi(x.w)))));
                    }
                    powers_of(most, up, factor);
                    factor *= L.scale;
                }
#pragma unroll 2
                for (int i = 0; i < D / 16; ++i) {               // channels 8 i .. and D/2 + 8 i ..
                    const uint32_t to_a = at(i), to_b = at(i + D / 16);
                    const uint4 x = load16(q_lo + to_a), y = load16(q_lo + to_b);
                    float a[8] = { bf16_lo(x.x), bf16_hi(x.x), bf16_lo(x.y), bf16_hi(x.y), bf16_lo(x.z), bf16_hi(x.z), bf16_lo(x.w), bf16_hi(x.w) };
                    float b[8] = { bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y), bf16_lo(y.z), bf16_hi(y.z), bf16_lo(y.w), bf16_hi(y.w) };
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        a[j] *= up;
                        b[j] *= up;
                        if (turn) {
                            const float2 cs = sh.table[warp][8 * i + j];
                            const float t = fmaf(a[j], cs.x, -b[j] * cs.y);
                            b[j] = fmaf(b[j], cs.x, a[j] * cs.y);
                            a[j] = t;
                        }
                    }
                    uint32_t ah[4], al[4], bh[4], bl[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        split_f16x2(a[j], a[j + 4], ah[j], al[j]);
                        split_f16x2(b[j], b[j + 4], bh[j], bl[j]);
                    }
                    store16(q_hi + to_a, ah[0], ah[1], ah[2], ah[3]);
                    store16(q_hi + to_b, bh[0], bh[1], bh[2], bh[3]);
                    if (turn) {
                        store16(q_lo + to_a, al[0], al[1], al[2], al[3]);
                        store16(q_lo + to_b, bl[0], bl[1], bl[2], bl[3]);
                    }
                }
                fence_async_smem();
                mbar_arrive(smem_u32(&sh.q_full[set]));
            }
            const int t0 = (w.tile - w.part_first) * kBlockTile;
            const long long see = ahead - t0 + token;
            const int n = seen - t0, limit = see >= n ? n : see < -1 ? 0 : (int)see + 1;       // columns in front of it are seen
            const bool all = __all_sync(0xffffffffu, limit >= kBlockTile);
            const unsigned ring = (u - u0) & 3u;
            if (!(ok = wait(sh.s_full[set][turns & 1u], (turns >> 1) & 1u))) break;
            tc_fence_after();
            // Two passes over the row's 64 scores, the second in a short loop that reads them again from tensor memory: code that stays in the
            // instruction cache and few registers are worth more than that read.
            const uint32_t s_col = s_base + (turns & 1u) * 64u;
            const float power = sh.key_power[ring];
            if (power == 0.0f) {                                 // a power of two for each token's scores
#pragma unroll 1
                for (int c0 = 0; c0 < kBlockTile; c0 += 16) {
                    uint32_t y[16];
                    tc_load16(y, s_col + c0);
                    tc_wait_loads();
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * sh.key_column[ring][c0 + i]);
                    tc_store16(s_col + c0, y);
                }
                tc_wait_stores();
            }
            float scale = power == 0.0f ? factor : factor * power;
            float top = -INFINITY;
            auto maxima = [&](auto whole) {
                uint32_t x[2][32];
                tc_load32(x[0], s_col);
                tc_load32(x[1], s_col + 32u);
                tc_wait_loads();
                if (!decltype(whole)::value) {
#pragma unroll
                    for (int i = 0; i < 64; ++i)
                        if (i >= limit) x[i / 32][i % 32] = 0xff800000u;
                }
                float a[4] = { -INFINITY, -INFINITY, -INFINITY, -INFINITY };
#pragma unroll
                for (int i = 0; i < 64; ++i) a[i % 4] = fmaxf(a[i % 4], __uint_as_float(x[i / 32][i % 32]));
                top = fmaxf(fmaxf(a[0], a[1]), fmaxf(a[2], a[3]));
            };
            if (all) maxima(std::true_type{});
            else maxima(std::false_type{});
            top *= scale;
            // huge scores are multiplied and rounded before the reference is taken off (a row of scores past fp32's range is NaN then)
            if (__any_sync(0xffffffffu, fabsf(top) > kHugeScore && top != -INFINITY)) {
                const float by = fabsf(top) > kHugeScore ? scale : 1.0f;
#pragma unroll 1
                for (int c0 = 0; c0 < kBlockTile; c0 += 16) {
                    uint32_t y[16];
                    tc_load16(y, s_col + c0);
                    tc_wait_loads();
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * by);
                    tc_store16(s_col + c0, y);
                }
                tc_wait_stores();
                if (by != 1.0f) scale = 1.0f;
            }
            // the reference follows the maximum when that is 2^8 above it
            const bool move = top > m + 8.0f;
            if (__any_sync(0xffffffffu, move)) {
                const float a = move ? exp2_approx(m - top) : 1.0f;
                if (move) m = top;
                l *= a;
                if (!w.new_seg && u != u0) {                     // there is something in O, once the tile before is in it
                    if (!(ok = wait(sh.o_full[set], (turns & 1u) ^ 1u))) break;
                    tc_fence_after();
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 16) {
                        uint32_t y[16];
                        tc_load16(y, o_col + c0);
                        tc_wait_loads();
#pragma unroll
                        for (int i = 0; i < 16; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * a);
                        tc_store16(o_col + c0, y);
                    }
                }
            }
            const float base = m == -INFINITY ? 0.0f : -m;
            const f32x2 scale2 = pack2(scale, scale), base2 = pack2(base, base);
            f32x2 sum = pack2(0.0f, 0.0f);
            auto weights = [&](auto whole) {
                auto sixteen = [&](const uint32_t (&x)[16], int c0) {
                    f32x2 e[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float e0, e1;
                        unpack2(fma2(pack2(__uint_as_float(x[2 * i]), __uint_as_float(x[2 * i + 1])), scale2, base2), e0, e1);
                        e0 = exp2_approx(e0);
                        e1 = exp2_approx(e1);
                        if (!decltype(whole)::value) {
                            if (c0 + 2 * i >= limit) e0 = 0.0f;
                            if (c0 + 2 * i + 1 >= limit) e1 = 0.0f;
                        }
                        e[i] = pack2(e0, e1);
                        sum = add2(sum, e[i]);
                    }
                    uint32_t z[8 * NG];
#pragma unroll
                    for (int G = 0; G < NG; ++G)
#pragma unroll
                        for (int i = 0; i < 8; i += 2) {
                            const float4 vs = *reinterpret_cast<const float4 *>(&sh.value_scale[ring][G][c0 + 2 * i]);
                            float p0, p1, p2, p3;
                            unpack2(mul2(e[i], pack2(vs.x, vs.y)), p0, p1);
                            unpack2(mul2(e[i + 1], pack2(vs.z, vs.w)), p2, p3);
                            if (!decltype(whole)::value) {       // what is not seen may hold anything
                                if (c0 + 2 * i >= limit) p0 = 0.0f;
                                if (c0 + 2 * i + 1 >= limit) p1 = 0.0f;
                                if (c0 + 2 * i + 2 >= limit) p2 = 0.0f;
                                if (c0 + 2 * i + 3 >= limit) p3 = 0.0f;
                            }
                            z[8 * G + i] = pack_bf16x2(p0, p1);
                            z[8 * G + i + 1] = pack_bf16x2(p2, p3);
                        }
                    if constexpr (NG == 2) tc_store16(s_col + c0, z);
                    else tc_store8(s_col + c0, z);
                };
                // the next sixteen are on their way while these are worked on
                uint32_t x[16], y[16];
                tc_load16(x, s_col);
#pragma unroll 1
                for (int c0 = 0; c0 < kBlockTile; c0 += 32) {
                    tc_wait_loads();
                    tc_load16(y, s_col + c0 + 16u);
                    sixteen(x, c0);
                    tc_wait_loads();
                    if (c0 + 32 < kBlockTile) tc_load16(x, s_col + c0 + 32u);
                    sixteen(y, c0 + 16);
                }
            };
            if (all) weights(std::true_type{});
            else weights(std::false_type{});
            {
                float l0, l1;
                unpack2(sum, l0, l1);
                l += l0 + l1;
            }
            tc_wait_stores();
            tc_fence_before();
            const bool over = w.tile + 1 == w.r.tiles || u + 1 == u1;
            // (what is waited for below must be the only turn of the barrier that can be pending)
            if (over && turns > 0 && !(ok = wait(sh.o_full[set], (turns & 1u) ^ 1u))) break;
            mbar_arrive(smem_u32(&sh.p_full[set][turns & 1u]));
            ++turns;
            if (over) {
                // the segment ends here
                if (!(ok = wait(sh.o_full[set], (turns & 1u) ^ 1u))) break;
                tc_fence_after();
                const unsigned s0 = w.r.unit + (unsigned)w.seg * (unsigned)w.r.tiles, s1 = s0 + (unsigned)w.r.tiles;
                const bool whole = s0 >= u0 && s1 <= u1, in = rho < w.r.rows;
                const long long at = (2ll * blockIdx.x + (s0 > u0 ? 1 : 0)) * kBlockRows + set * 128 + place;
                const long long qrow = w.r.row + token;
                const int head = h * L.g + rho % L.g;
                const float inv = !whole ? 1.0f : l == 0.0f ? 0.0f : 1.0f / l;
                // Through the place of the warp's queries, which nothing reads any more, 32 channels at a time (D / 32 pieces of 32 rows of 128 bytes), so that
                // whole rows are written
                const uint32_t piece = q_hi + (uint32_t)(warp & 3) * 4096u;
#pragma unroll 1
                for (int p = 0; p < D / 32; ++p) {
                    uint32_t y[32];
                    tc_load32(y, o_col + 32 * p);
                    tc_wait_loads();
                    if (whole) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) y[i] = __float_as_uint(__uint_as_float(y[i]) * inv);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {                // columns 0 .. 7 are channels 0 4 1 5 2 6 3 7
                        const int c0 = 8 * (i / 2) + i % 2;
                        store16(piece + 16384u * p + swizzled((uint32_t)lane, (uint32_t)i), y[c0], y[c0 + 2], y[c0 + 4], y[c0 + 6]);
                    }
                }
                __syncwarp();
                unsigned long long mine = 0;
                if (in) mine = whole ? (unsigned long long)(L.out + qrow * L.out_stride + (long long)head * D) : (unsigned long long)(L.part_o + at * D);
#pragma unroll 2
                for (int i = lane / 8; i < 32; i += 4) {
                    const unsigned long long to = __shfl_sync(0xffffffffu, mine, i);
                    if (to)
#pragma unroll
                        for (int p = 0; p < D / 32; ++p) {
                            const uint4 x = load16(piece + 16384u * p + swizzled((uint32_t)i, (uint32_t)(lane & 7)));
                            const int c0 = 32 * p + 4 * (lane & 7);
                            if (whole)
                                *reinterpret_cast<uint2 *>(reinterpret_cast<__nv_bfloat16 *>(to) + c0) =
                                    make_uint2(pack_bf16x2(__uint_as_float(x.x), __uint_as_float(x.y)), pack_bf16x2(__uint_as_float(x.z), __uint_as_float(x.w)));
                            else
                                *reinterpret_cast<uint4 *>(reinterpret_cast<float *>(to) + c0) = x;
                        }
                }
                __syncwarp();
                if (in && !whole) L.part_ml[at] = make_float2(m, l);
                if (in && whole && L.lse) L.lse[qrow * (L.H * L.g) + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
                tc_fence_before();
            }
        }
    } else if (warp < 12) {
        // ----------------------------------------------------------------------------- codes to operands
        // A thread takes a token and a group of 64 channels (head_dim 64: half a group).
        const int me = (int)threadIdx.x - 256, t = me & 63, side = me >> 6, G = D == 128 ? side : 0;
        constexpr int kWords = D / 16, kLoads = kWords / 4;      // words of codes a thread, loads of them
        uint32_t *const channel = &sh.channel[warp - 8][0][0];
        // Loads run ahead: of tile i + 1 between the expansion of tile i's keys and that of the values of the tile before.
        uint4 kc[kLoads], vc[kLoads], v_now[kLoads], v_before[kLoads];
        float ks = 0.0f, vs = 0.0f, near[2 * NG];                // scales of the token's codes; key scales of the tile of which the largest is wanted
        float cs[2] = { 0.0f, 0.0f };                            // codes in channel groups: two channels of the warp's
        bool group_keys = false;
        int n = 0;
        const uint4 *codes_at = nullptr, *values_at = nullptr;   // of this thread's token
        const float *key_at = nullptr, *value_at = nullptr, *near_at = nullptr;
        auto fetch = [&]() {
            if (w.new_part) {
                const PartRec p = w.parts[w.r.part + w.pi];
                const int h = w.head, t0 = (w.tile - w.part_first) * kBlockTile;
                const long long row_bytes = (long long)L.H * (D / 2), at = ((long long)(t0 + t) * L.H + h) * NG;
                n = p.seen - t0;
                group_keys = p.kc != 0;
                codes_at = reinterpret_cast<const uint4 *>(p.codes + (t0 + t) * row_bytes + h * (D / 2) + side * (kLoads * 16));
                values_at = reinterpret_cast<const uint4 *>(reinterpret_cast<const unsigned char *>(codes_at) + p.T * row_bytes);
                key_at = p.scales + at + G;
                value_at = key_at + (group_keys ? (long long)((p.T + 63) / 64) * L.H * D : (long long)p.T * L.H * NG);
                near_at = group_keys ? p.scales + ((long long)(t0 / 64) * L.H + h) * D + 2 * lane : p.scales + ((long long)(t0 + lane) * L.H + h) * NG;
            } else {
                const long long rows = (long long)kBlockTile * L.H;
                n -= kBlockTile;
                codes_at += rows * (D / 32);
                values_at += rows * (D / 32);
                key_at += rows * NG;
                value_at += rows * NG;
                near_at += group_keys ? (long long)L.H * D : rows * NG;
            }
            ks = vs = 0.0f;
#pragma unroll
            for (int i = 0; i < 2 * NG; ++i) near[i] = 0.0f;
#pragma unroll
            for (int i = 0; i < kLoads; ++i) kc[i] = vc[i] = make_uint4(0u, 0u, 0u, 0u);
            if (t < n) {
#pragma unroll
                for (int i = 0; i < kLoads; ++i) { kc[i] = codes_at[i]; vc[i] = values_at[i]; }
                if (!group_keys) ks = *key_at;
                vs = *value_at;
            }
            // every warp finds the largest for itself
            if (group_keys) {
                if (n > 0) {
#pragma unroll
                    for (int i = 0; i < NG; ++i) {
                        near[2 * i] = near_at[64 * i];
                        near[2 * i + 1] = near_at[64 * i + 1];
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < NG; ++j)
                        if (lane + 32 * i < n) near[i * NG + j] = near_at[(long long)32 * i * L.H * NG + j];
            }
        };
        auto words = [](const uint4 (&x)[kLoads], int i) { const uint4 &y = x[i / 4]; return i % 4 == 0 ? y.x : i % 4 == 1 ? y.y : i % 4 == 2 ? y.z : y.w; };
        fetch();
        unsigned i = 0;
        for (unsigned u = u0; u <= u1 && ok; ++u, ++i) {
            const int b = (int)(i & 1u);
            const unsigned ring = i & 3u;
            // keys of tile i, then values of the one before, whose place is left later
            if (u < u1) {
            float down, up, column = 0.0f;
            float hi = 0.0f, lo = 0.0f;
            if (NG == 2 && G) { cs[0] = near[2 * NG - 2]; cs[1] = near[2 * NG - 1]; }
            else { cs[0] = near[0]; cs[1] = near[1]; }
            // Exponents of the tile's scales.  Where they are few apart, all keys are divided by one power of two; else, and where some are infinite, each token's by its own.  Both
            // give a token's scores the same bits, so that no row's go by tokens that it does not see.
            int e_max = 0, e_min = 255;
#pragma unroll
            for (int j = 0; j < 2 * NG; ++j) {
                const int e = (int)(__float_as_uint(near[j]) >> 23 & 255u);
                e_max = max(e_max, e);
                if (e > 0) e_min = min(e_min, e);
            }
            e_max = __reduce_max_sync(0xffffffffu, e_max);
            e_min = __reduce_min_sync(0xffffffffu, e_min);
            key_powers(e_max, down, up);
            if (!group_keys && e_max > 0 && (e_max == 255 || e_max - e_min > kKeySpread)) {
                int e = 0;                                       // of this thread's token
#pragma unroll
                for (int j = 0; j < NG; ++j) e = max(e, (int)(__float_as_uint(t < 32 ? near[j] : near[NG + j]) >> 23 & 255u));
                key_powers(e, down, column);
                up = 0.0f;
            }
            const bool by_channel = group_keys;
            if (by_channel) {
                float h0, l0, h1, l1;
                split_scale(cs[0] * down, h0, l0);
                split_scale(cs[1] * down, h1, l1);
                __syncwarp();
                // channels 2 lane, 2 lane + 1 of a word's eight: pairs (j, j + 4) side by side
                __half *hs = reinterpret_cast<__half *>(channel), *ls = reinterpret_cast<__half *>(channel + 32);
                const int c0 = 2 * lane, p0 = (c0 & ~7) + (c0 & 3) * 2 + ((c0 >> 2) & 1), p1 = (c0 & ~7) + ((c0 + 1) & 3) * 2 + ((c0 >> 2) & 1);
                hs[p0] = __float2half_rn(h0); hs[p1] = __float2half_rn(h1);
                ls[p0] = __float2half_rn(l0); ls[p1] = __float2half_rn(l1);
                __syncwarp();
            } else {
                split_scale(ks * down, hi, lo);
            }
            if (!(ok = wait(sh.k_empty[b], ((i >> 1) & 1u) ^ 1u))) break;
            {
                const uint32_t h2 = pack_f16x2(hi, hi), l2 = pack_f16x2(lo, lo);
                const uint32_t to = k_at + b * 2 * S::kK + (D == 128 ? G * (kBlockTile * 128u) : 0u);
#pragma unroll
                for (int j = 0; j < kWords; ++j) {
                    uint32_t c[4], a[4], d[4];
                    code_pairs_f16(c, words(kc, j), L.bits);
                    uint4 ch = make_uint4(h2, h2, h2, h2), cl = make_uint4(l2, l2, l2, l2);
                    if (by_channel) {
                        const int word = D == 128 ? j : side * kWords + j;
                        ch = *reinterpret_cast<const uint4 *>(channel + 4 * word);
                        cl = *reinterpret_cast<const uint4 *>(channel + 32 + 4 * word);
                    }
                    a[0] = mul_f16x2(c[0], ch.x); a[1] = mul_f16x2(c[1], ch.y); a[2] = mul_f16x2(c[2], ch.z); a[3] = mul_f16x2(c[3], ch.w);
                    d[0] = mul_f16x2(c[0], cl.x); d[1] = mul_f16x2(c[1], cl.y); d[2] = mul_f16x2(c[2], cl.z); d[3] = mul_f16x2(c[3], cl.w);
                    const uint32_t at = to + swizzled((uint32_t)t, (uint32_t)(D == 128 ? j : side * kWords + j));
                    store16(at, a[0], a[1], a[2], a[3]);
                    store16(at + S::kK, d[0], d[1], d[2], d[3]);
                }
            }
            if (me == 0) sh.key_power[ring] = up;
            if (up == 0.0f && me < kBlockTile) sh.key_column[ring][t] = column;
            if (D == 128 || side == 0) sh.value_scale[ring][G][t] = vs;
            fence_async_smem();
            mbar_arrive(smem_u32(&sh.k_full[b]));
            }
#pragma unroll
            for (int j = 0; j < kLoads; ++j) { v_before[j] = v_now[j]; v_now[j] = vc[j]; }
            if (u + 1 < u1) {
                w.step(L.H);
                fetch();
            }
            if (i > 0) {
                if (!(ok = wait(sh.v_empty, i & 1u))) break;
                const uint32_t to = v_at + (D == 128 ? G * (kBlockTile * 128u) : 0u);
#pragma unroll
                for (int j = 0; j < kWords; ++j) {
                    const uint32_t x = words(v_before, j);
                    store16(to + swizzled((uint32_t)t, (uint32_t)(D == 128 ? j : side * kWords + j)), code_pair<0>(x, L.bits), code_pair<1>(x, L.bits),
                            code_pair<2>(x, L.bits), code_pair<3>(x, L.bits));
                }
                fence_async_smem();
                mbar_arrive(smem_u32(&sh.v_full));
            }
        }
    } else {
        // --------------------------------------------------------------------------------------- products
        const int set = warp - 12;
        const uint32_t qk = mma_descriptor(kF16, 128, kBlockTile, false), pv = mma_descriptor(kBf16, 128, 64, true);
        // Descriptors of the operands' first elements; what comes behind is a constant further on.
        const uint64_t q_desc = tile_descriptor(q_at, 16, 1024), k_desc = tile_descriptor(k_at, 16, 1024), v_desc = tile_descriptor(v_at, 8192, 1024);
        // S of a set: leading Q by both of K, and what is left of a turned Q by leading K
        auto scores = [&](int b, int column, bool turned) {
            const uint64_t q = q_desc + (uint64_t)(set * 2 * S::kQ / 16), k = k_desc + (uint64_t)(b * 2 * S::kK / 16);
            const uint32_t d = tmem + set * 256u + column * 64u;
#pragma unroll
            for (int s = 0; s < D / 16; ++s) {
                const uint64_t qs = q + (s / 4) * (128 * 128 / 16) + (s % 4) * 2, ks = k + (s / 4) * (kBlockTile * 128 / 16) + (s % 4) * 2;
                tc_mma(d, qs, ks, qk, s > 0);
                tc_mma(d, qs, ks + S::kK / 16, qk, true);
            }
            if (turned) {
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    tc_mma(d, q + S::kQ / 16 + (s / 4) * (128 * 128 / 16) + (s % 4) * 2, k + (s / 4) * (kBlockTile * 128 / 16) + (s % 4) * 2, qk, true);
            }
            tc_commit(smem_u32(&sh.s_full[set][column]));
        };
        auto output = [&](int b, bool first) {
            const uint32_t d = tmem + set * 256u + 128u, p = tmem + set * 256u + b * 64u;
#pragma unroll
            for (int G = 0; G < NG; ++G)
#pragma unroll
                for (int s = 0; s < kBlockTile / 16; ++s)
                    tc_mma_ts(d + 64u * G, p + 16u * s + 8u * G, v_desc + (G * (kBlockTile * 128) + s * 2048) / 16, pv, !first || s > 0);
            tc_commit(smem_u32(&sh.o_full[set]));
        };
        // Turn i: the scores of tile i, then the output of the tile before it; the other way round where the tile's queries are new, since those that
        // write them first finish the tile before.  A set without rows leaves the tiles as they come.
        const unsigned n = u1 - u0;
        unsigned made = 0, done = 0, queries = 0;                // scores, outputs, and parts whose queries were taken
        bool here_before = false, first_before = false, turned = false;
        for (unsigned i = 0; i <= n && ok; ++i) {
            const int b = (int)(i & 1u);
            const bool here = i < n && set < w.sets, first_now = i < n && (w.new_seg || i == 0), late = i < n && w.new_part && i > 0;
            if (i < n && w.new_part) turned = w.parts[w.r.part + w.pi].turn != 0;
            // scores go to the columns that held the P of two tiles ago; what has been issued of outputs is over, so no turn is mistaken for another
            if (here_before && done > 0) ok = wait(sh.o_full[set], (done - 1) & 1u);
#pragma unroll 1
            for (int half = 0; half < 2 && ok; ++half) {
                if ((half == 0) != late) {
                    if (i == n) continue;
                    ok = wait(sh.k_full[b], (i >> 1) & 1u);
                    if (ok && here && w.new_part) {
                        ok = wait(sh.q_full[set], queries & 1u);
                        ++queries;
                    }
                    if (!ok) break;
                    tc_fence_after();
                    if (one_lane()) {
                        if (here) {
                            scores(b, (int)(made & 1u), turned);
                            tc_commit(smem_u32(&sh.k_empty[b]));
                        } else {
                            mbar_arrive(smem_u32(&sh.k_empty[b]));
                        }
                    }
                    if (here) ++made;
                    __syncwarp();
                } else if (i > 0) {
                    ok = wait(sh.v_full, (i - 1) & 1u);
                    if (ok && here_before) ok = wait(sh.p_full[set][done & 1u], (done >> 1) & 1u);
                    if (!ok) break;
                    tc_fence_after();
                    if (one_lane()) {
                        if (here_before) {
                            output((int)(done & 1u), first_before);
                            tc_commit(smem_u32(&sh.v_empty));
                        } else {
                            mbar_arrive(smem_u32(&sh.v_empty));
                        }
                    }
                    if (here_before) ++done;
                    __syncwarp();
                }
            }
            here_before = here;
            first_before = first_now;
            if (i + 1 < n) w.step(L.H);
        }
        if (one_lane()) tc_commit(smem_u32(&sh.drained));
        __syncwarp();
        volatile int never = 0;                                  // products in flight end by themselves
        mbar_wait(smem_u32(&sh.drained), 0u, &never, 2000000000ull);
    }
    if (sh.abort_flag && lane == 0) atomicCAS(L.status, 0, kStatusTimeout);
    tc_fence_before();
    __syncthreads();
    if (warp == 12) tc_free(tmem, 512);
}

}  // namespace kdn
