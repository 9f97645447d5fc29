// Attention of a few new tokens over stored 4-bit chunks, and the joining of partial results.
//
// Mathematics.  With codes c, scales s and queries q turned against the part's shift (q.(R k) = (R^-1 q).k):
//     group-64 keys     score[t] = sum over groups of 64 channels G of s[t][G] * (q_G . c[t]_G)
//     keys in channel groups   score[t] = (q * s[group of t]) . c[t]
//     out = sum over t of (p[t] s_v[t][G]) c_v[t]_G,   p = 2^(score * scale * log2 e - m), one pass with the running maximum m
// so that the matrix instructions only ever see codes, which are exact in fp16 and bf16, and the scales meet 8 scores a token and not 128
// channels.  Roundings: a query that goes with group-64 keys is held as fp16 (exact as it came, times a power of two) and, where it was turned, as two fp16
// numbers (22 bits); so is one that is multiplied by the scales of channel groups; weights times value scale are held as two bf16 numbers (16 bits, and
// the range that a product with any scale needs).  One number for the weights would save a quarter to a third of the products and
// cost as much precision as the rounding of the result does.
//
// What bounds it: instructions and what one waits for another; no pipe is full (32 requests of 8192 tokens: 60 of 100 issue slots, the integer pipe
// 46, 16 warps an SM).  A token of one head is 144 bytes of K and V at head_dim 128; at 6.4 TB/s an SM may take 6 cycles for it, in
// which 256 codes have to become matrix operands.  Tokens are the 16 rows of mma.m16n8k16 and the (up to 8) query rows of a KV head its
// 8 columns, so that no operand is wasted on one-token steps of grouped heads, and codes go from shared memory to the operand registers by 0.5
// to 0.75 integer or half-precision instructions a code, with no shared memory in between: some 800 instructions for 32 tokens of a head.
// Measured, one layer of 8 heads of 128: a token over 131072 tokens 53 us (151 MB, 2.9 TB/s); 32 requests of a token over four documents of
// 2048, keys in channel groups, turned: 122 us (2.5 TB/s; 119 with queries held to 16 bits); a token over ten documents of 1024, turned: 20 us, about
// half of it this kernel (a launch, two dependent reads, a tile a CTA) and half the joining of 296 parts a head.
#pragma once
#include "kdn_ops.cuh"

namespace kdn {

// One part of one request: a layer of a chunk at its place in the request.
struct PartRec {
    const unsigned char *codes;             // keys' nibbles [T][H][D/2], the values' behind them
    const float *scales;                    // keys' scales of the layer, the values' behind them
    long long ahead;                        // q_pos - part_pos: new token i sees chunk tokens up to ahead + i
    long long turn;                         // positions by which the queries are rotated: base_pos - part_pos
    int T;
    int seen;                               // tokens that some row sees
    int tile;                               // first tile within the request
    int kc;                                 // keys in channel groups
};
static_assert(sizeof(PartRec) == 48, "");

struct ReqRec {
    int row, rows;                          // first row in q; n_q * g rows a KV head
    int part, n_parts;
    unsigned unit;                          // first unit
    int tiles;                              // tiles of a pass over the context (at least one)
};
static_assert(sizeof(ReqRec) == 24, "");

// Masks, mantissas and what comes off again arrive as launch parameters: as literals they do not fit one three-input logic instruction, and the
// integer pipe is what this kernel runs out of first.
struct Bits {
    uint32_t mask, bias;                    // 0x000f000f, 0x43084308: a nibble, its sign bit flipped, in the mantissa of 128 as bf16; 136 too much
    uint32_t bias_f16;                      // 0x64086408: the same in the mantissa of 1024 as fp16; 1032 too much
    uint32_t mask_up, bias_up;              // 0x00f000f0, 0x64806480: a nibble four bits further up, 16 times the code, 1024 + 128 too much
    uint32_t sixteenth, less;               // 1/16 and -72 as fp16
};
__device__ __forceinline__ uint32_t masked(uint32_t w, uint32_t mask, uint32_t bias)
{
    uint32_t x;
    asm("lop3.b32 %0, %1, %2, %3, 0x6a;" : "=r"(x) : "r"(w), "r"(mask), "r"(bias));                    // (w & mask) ^ bias
    return x;
}
// Nibbles J and J + 4 of the eight in w as two codes in bf16.
template <int J> __device__ __forceinline__ uint32_t code_pair(uint32_t w, const Bits &k)
{
    uint32_t x = masked(w >> (4 * J), k.mask, k.bias);
    asm("sub.rn.bf16x2 %0, %0, %1;" : "+r"(x) : "r"(k.bias));
    return x;
}
// All eight as fp16: pairs (0, 4), (1, 5), (2, 6), (3, 7).
__device__ __forceinline__ void code_pairs_f16(uint32_t (&x)[4], uint32_t w, const Bits &k)
{
    const uint32_t v = w >> 8;
    x[0] = masked(w, k.mask, k.bias_f16);
    x[1] = masked(w, k.mask_up, k.bias_up);
    x[2] = masked(v, k.mask, k.bias_f16);
    x[3] = masked(v, k.mask_up, k.bias_up);
    asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(x[0]) : "r"(k.bias_f16));
    asm("sub.rn.f16x2 %0, %0, %1;" : "+r"(x[2]) : "r"(k.bias_f16));
    asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(x[1]) : "r"(k.sixteenth), "r"(k.less));
    asm("fma.rn.f16x2 %0, %0, %1, %2;" : "+r"(x[3]) : "r"(k.sixteenth), "r"(k.less));
}

constexpr int kInlineParts = 16, kInlineReqs = 16;
struct AttendLaunch {
    const ReqRec *reqs;                     // in the workspace, or nullptr: inl_reqs, inl_parts
    const PartRec *parts;
    const __nv_bfloat16 *q;
    __nv_bfloat16 *out;
    float *lse;
    float *part_o;                          // [slot][heads of a unit][rows of a unit][D]
    float2 *part_ml;                        // [slot][heads of a unit][rows of a unit]
    int *status;
    long long q_stride, out_stride;
    unsigned long long wait_limit_ns;
    float scale;                            // of scores in powers of two
    int H, g, n_reqs;
    Bits bits;
    unsigned units;
    double turns[64];                       // theta^(-2i/D) / (2 pi): pair i turns by that part of a circle a position
    ReqRec inl_reqs[kInlineReqs];
    PartRec inl_parts[kInlineParts];
};

// The angle is reduced to a part of one turn in 64 bits; its sine and cosine are taken in 32.
__device__ __forceinline__ float2 turn_of(double turns, long long by)
{
    double x = turns * (double)by;
    x -= rint(x);
    float s, c;
    sincospif(2.0f * (float)x, &s, &c);
    return make_float2(c, s);
}

// Units are (request, block of 8 rows, block of HB heads, tile of tokens), tiles fastest, and CTA b of G takes units [bU/G, (b+1)U/G).  The units
// that share all but the tile form a segment; where its tiles fall into several CTAs each leaves a partial result in a slot (two to a
// CTA: only its first and its last segment can be shared) and kdn_attend_join_kernel joins them.
__host__ __device__ __forceinline__ unsigned first_unit(unsigned b, unsigned units, unsigned ctas) { return (unsigned)((unsigned long long)units * b / ctas); }
__host__ __device__ __forceinline__ unsigned cta_of(unsigned u, unsigned units, unsigned ctas)
{
    return (unsigned)((((unsigned long long)u + 1) * ctas - 1) / units);
}

// A warp takes one head and kWarpTokens tokens of a tile, through a pipeline of its own: it copies what it needs two tiles
// ahead (16-byte asynchronous copies, 64 contiguous bytes a token and head), so no warp waits for another but where warps that share
// a head join at the end of a segment.
template <int D, int HB> struct StepShape {
    static constexpr int kSub = 8 / HB;                                   // warps that share a head, each with its tokens of the tile
    static constexpr int kWarpTokens = 32;
    static constexpr int kTile = kSub * kWarpTokens;                      // 32, 64, 128, 256
    static constexpr int kGroups = D / 64;
    static constexpr int kCodes = kWarpTokens * D / 2;
    static constexpr int kKeyScales = D * 4 > kWarpTokens * kGroups * 4 ? D * 4 : kWarpTokens * kGroups * 4;
    static constexpr int kValueScales = kWarpTokens * kGroups * 4;
    static constexpr int kMeta = 64;
    static constexpr int kStage = 2 * kCodes + kKeyScales + kValueScales + kMeta;
    static constexpr int kTable = D / 2 * 8;
    static constexpr int kLow = D / 64 * 8 * 32 * 4;                      // second halves of the query operands
    // partial results of warps that share a head, 64 channels at a time, where the second halves lie otherwise
    static constexpr int kMerge = kSub > 1 && 8 * 8 * 64 * 4 > 8 * kLow ? 8 * 8 * 64 * 4 : 8 * kLow;
    static constexpr int kThreads = 256;
    static constexpr int kStages = 2;
    static constexpr int kCold = 128;
    static constexpr int kWarpBytes = kStages * kStage + kTable + kCold;
    static constexpr int kSmem = 8 * kWarpBytes + kMerge + 8 * 8 * 8;
    static_assert(kStage % 16 == 0 && kSmem <= 113 * 1024, "two CTAs an SM");
};

struct __align__(16) StepMeta {             // what is to be known of a tile when it is taken
    int flags;                              // 1: a new segment, 2: a new part or segment; with neither, only the first four are written
    int n;                                  // this warp's tokens in the tile
    int full;                               // kWarpTokens, and every one is seen by every row
    int ahead;                              // last token (of the warp's) that new token 0 sees, may be negative
    long long turn;
    int kc;
    int row, rows, row0;                    // request's first row in q, rows a head, first row of this block
    int head;
    int slot;                               // -1: the segment is whole here
};
static_assert(sizeof(StepMeta) <= 64, "");

struct StepCursor {                         // of the unit that is copied next: what only a new part or segment reads
    ReqRec r;
    int ri, pi, seg, tile;                  // request, part within it, segment within it, tile of the part's first copy
};

// The last i in [0, n) whose unit (or tile) is at most x; first(i) increases.  One lane an entry.
template <typename F> __device__ __forceinline__ int last_at_most(int n, F first, unsigned x, int lane)
{
    int found = 0;
    for (int i0 = 0; i0 < n; i0 += 32) {
        const unsigned in = __ballot_sync(0xffffffffu, i0 + lane < n && first(i0 + lane) <= x);
        if (!in) break;
        found = i0 + 31 - __clz(in);
        if (in != 0xffffffffu) break;
    }
    return found;
}

// Where 16-byte chunk i of token t's row lies in a warp's codes: the same chunk of eight neighbouring tokens, one matrix of a load, meets
// no bank twice.
template <int D> __device__ __forceinline__ int chunk_at(int t, int i)
{
    return t * (D / 2) + (D == 128 ? i ^ ((t >> 1) & 3) : i ^ ((t >> 2) & 1)) * 16;
}

// WHOLE: the pool has no heads but the HB of a unit, so that rows follow one another at a constant distance.
template <int D, int HB, bool ANY_KC, bool WHOLE>
__global__ void __launch_bounds__(256, 2) kdn_attend_step_kernel(const __grid_constant__ AttendLaunch L)
{
    using S = StepShape<D, HB>;
    constexpr int NG = S::kGroups, MT = S::kWarpTokens / 16, WT = S::kWarpTokens;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31;
    const int hi = warp % HB, sub = warp / HB;              // head of the unit, token slice of the tile
    const int g = lane >> 2, c = lane & 3;
    unsigned char *mine = smem + warp * S::kWarpBytes;
    float2 *table = reinterpret_cast<float2 *>(mine + S::kStages * S::kStage);
    float *merge_o = reinterpret_cast<float *>(smem + 8 * S::kWarpBytes);
    float2 *merge_ml = reinterpret_cast<float2 *>(smem + 8 * S::kWarpBytes + S::kMerge);
    uint4 *low_q = reinterpret_cast<uint4 *>(smem + 8 * S::kWarpBytes + warp * S::kLow) + lane;      // [2 G + w][32]
    release_dependents();
    if (L.reqs) dependency_wait();                          // records that are launch parameters can be read before
    const ReqRec *reqs = L.reqs ? L.reqs : L.inl_reqs;
    const PartRec *parts = L.reqs ? L.parts : L.inl_parts;
    const unsigned u0 = first_unit(blockIdx.x, L.units, gridDim.x), u1 = first_unit(blockIdx.x + 1, L.units, gridDim.x);
    const int hblocks = WHOLE ? 1 : L.H / HB;

    // The unit that is copied next: request, part, tile, and where this lane's copies of it come from.  A lane copies 16-byte chunk lane % kChunks
    // of every (32 / kChunks)th token and the scales of token `lane`.
    constexpr int kChunks = D / 32, kStep = 32 / kChunks;
    const int heads = WHOLE ? HB : L.H;
    const long long row_bytes = (long long)heads * (D / 2);
    const int my_chunk = chunk_at<D>(lane / kChunks, lane % kChunks);
    StepCursor &cur = *reinterpret_cast<StepCursor *>(mine + S::kStages * S::kStage + S::kTable);
    StepMeta &seg = *reinterpret_cast<StepMeta *>(mine + S::kStages * S::kStage + S::kTable + 64);    // the segment whose tiles are taken now
    unsigned next = u0;
    int flags = 3, tiles_left, part_left, left, t_next;     // tiles of the segment and of the part; tokens of the part; first token (codes in channel groups)
    int ahead;
    bool kc_next;
    const unsigned char *codes_at, *values_at;
    const float *ks_at, *vs_at;
    auto enter_part = [&](int ri, const ReqRec &r, int pi, int seg_i, int tile) {      // tile: of the request
        const PartRec p = parts[r.part + pi];
        const int t0 = (tile - p.tile) * S::kTile + sub * WT, head = seg_i % hblocks * HB + hi;
        part_left = (pi + 1 < r.n_parts ? parts[r.part + pi + 1].tile : r.tiles) - tile;
        left = p.seen - t0;
        t_next = t0;
        const long long see = p.ahead - t0;
        ahead = see > (1 << 30) ? 1 << 30 : see < -(1 << 30) ? -(1 << 30) : (int)see;
        kc_next = p.kc != 0;
        codes_at = p.codes + (long long)(t0 + lane / kChunks) * row_bytes + head * (D / 2) + lane % kChunks * 16;
        values_at = codes_at + (long long)p.T * row_bytes;
        const long long at = ((long long)(t0 + lane) * heads + head) * NG;
        vs_at = p.scales + at + (p.kc ? (long long)((p.T + 63) / 64) * heads * D : (long long)p.T * heads * NG);
        ks_at = p.kc ? p.scales + ((long long)(t0 / 64) * heads + head) * D + NG * lane : p.scales + at;
        __syncwarp();
        if (lane == 0) { cur.r = r; cur.ri = ri; cur.pi = pi; cur.seg = seg_i; cur.tile = tile; }
        __syncwarp();
    };
    {
        const int ri = last_at_most(L.n_reqs, [&](int i) { return reqs[i].unit; }, u0, lane);
        const ReqRec r = reqs[ri];
        const int tile = (int)((u0 - r.unit) % (unsigned)r.tiles);
        const int pi = last_at_most(r.n_parts, [&](int i) { return (unsigned)parts[r.part + i].tile; }, (unsigned)tile, lane);
        tiles_left = r.tiles - tile;
        enter_part(ri, r, pi, (int)((u0 - r.unit) / (unsigned)r.tiles), tile);
    }
    auto copy_next = [&](int st) {
        if (next < u1) {
            unsigned char *stage = mine + st * S::kStage;
            const uint32_t to = smem_u32(stage);
            auto tokens = [&](bool all) {
#pragma unroll
                for (int k = 0; k < WT / kStep; ++k)
                    if (all || lane / kChunks + kStep * k < left) {
                        copy_async<16>(to + my_chunk + kStep * k * (D / 2), codes_at + kStep * k * row_bytes);
                        copy_async<16>(to + S::kCodes + my_chunk + kStep * k * (D / 2), values_at + kStep * k * row_bytes);
                    }
                if (all || lane < left) {
                    if (!ANY_KC || !kc_next) copy_async<4 * NG>(to + 2 * S::kCodes + 4u * NG * lane, ks_at);
                    copy_async<4 * NG>(to + 2 * S::kCodes + S::kKeyScales + 4u * NG * lane, vs_at);
                }
            };
            if (left >= WT) tokens(true);
            else tokens(false);
            if (ANY_KC && kc_next && left > 0)
#pragma unroll
                for (int i = 0; i < D / (32 * NG); ++i)
                    copy_async<4 * NG>(to + 2 * S::kCodes + 4u * NG * (i * 32 + lane), ks_at + NG * i * 32);
            if (lane == 0) {
                StepMeta *meta = reinterpret_cast<StepMeta *>(stage + S::kStage - S::kMeta);
                const int n = left < WT ? left : WT;
                *reinterpret_cast<int4 *>(meta) = make_int4(flags, n, n == WT && ahead >= WT - 1, ahead);
                if (flags) {
                    const ReqRec r = cur.r;
                    const unsigned s0 = r.unit + (unsigned)cur.seg * (unsigned)r.tiles, s1 = s0 + (unsigned)r.tiles;
                    meta->turn = parts[r.part + cur.pi].turn;
                    meta->kc = kc_next;
                    meta->row = r.row;
                    meta->rows = r.rows;
                    meta->row0 = cur.seg / hblocks * 8;
                    meta->head = cur.seg % hblocks * HB + hi;
                    meta->slot = s0 >= u0 && s1 <= u1 ? -1 : (int)(2u * blockIdx.x + (s0 > u0 ? 1u : 0u));
                }
            }
            flags = 0;
            if (++next < u1) {
                --part_left;
                if (--tiles_left == 0) {
                    flags = 3;
                    ReqRec r = cur.r;
                    int seg_i = cur.seg + 1, ri = cur.ri;
                    if (next - r.unit == (unsigned)r.tiles * (unsigned)((r.rows + 7) / 8) * (unsigned)hblocks) { r = reqs[++ri]; seg_i = 0; }
                    tiles_left = r.tiles;
                    enter_part(ri, r, 0, seg_i, 0);
                } else if (part_left == 0) {
                    flags = 2;
                    const ReqRec r = cur.r;
                    const int pi = cur.pi + 1;
                    enter_part(cur.ri, r, pi, cur.seg, parts[r.part + pi].tile);
                } else {
                    left -= S::kTile;
                    ahead -= S::kTile;
                    codes_at += S::kTile * row_bytes;
                    values_at += S::kTile * row_bytes;
                    vs_at += (long long)S::kTile * heads * NG;
                    if (!ANY_KC || !kc_next) {
                        ks_at += (long long)S::kTile * heads * NG;
                    } else {                                // a row of scales for 64 tokens
                        t_next += S::kTile;
                        if (S::kTile >= 64 || t_next % 64 < S::kTile) ks_at += (long long)(S::kTile >= 64 ? S::kTile / 64 : 1) * heads * D;
                    }
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (!L.reqs) dependency_wait();
#pragma unroll 1
    for (int st = 0; st < S::kStages - 1; ++st) copy_next(st);

    // The queries, eight channels (of one word of codes) to four registers.  Codes in row groups: fp16 pairs (j, j + 4), all there is of a query
    // as it came, and in low_q what that leaves of one that was turned: 22 bits.  Codes in channel groups: fp32, four channels here and four
    // there, times the power of two that brings the largest scale to about 1 (it moves when that has moved by 2^7, but by no more than leaves the queries,
    // 2^8 at most, finite); before each use times the scales of 64 tokens and then as two fp16 numbers too.  A group whose scales are all zero moves nothing.
    uint32_t qa[8 * NG];
    float factor[2] = { 0.0f, 0.0f };
    int near = 127;                                         // codes in channel groups: the exponent that the largest scale has, or nearly
    float o[4 * NG][4], m[2], l[2];                         // columns are query rows 2c and 2c + 1
    bool have = false, kc = false, low = false;

    auto write_row = [&](int k, int d, float v0, float v1, float v2, float v3, float mm, float ll, bool first) {
        // four channels of query row k of this unit
        const int rho = seg.row0 + k;
        if (rho >= seg.rows) return;
        if (seg.slot >= 0) {
            const long long at = ((long long)seg.slot * HB + hi) * 8 + k;
            *reinterpret_cast<float4 *>(L.part_o + at * D + d) = make_float4(v0, v1, v2, v3);
            if (first) L.part_ml[at] = make_float2(mm, ll);
            return;
        }
        const long long qrow = seg.row + rho / L.g;
        const int qhead = seg.head * L.g + rho % L.g;
        const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;    // NaN stays NaN
        *reinterpret_cast<uint2 *>(L.out + qrow * L.out_stride + (long long)qhead * D + d) = make_uint2(pack_bf16x2(v0 * inv, v1 * inv), pack_bf16x2(v2 * inv, v3 * inv));
        if (first && L.lse) L.lse[qrow * (L.H * L.g) + qhead] = ll == 0.0f ? -INFINITY : (mm + log2f(ll)) * 0.69314718055994531f;
    };
    auto flush = [&]() {                                    // hands the finished segment over
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[j] += __shfl_xor_sync(0xffffffffu, l[j], d);
#pragma unroll
        for (int G = 0; G < NG; ++G) {
            if (S::kSub > 1) __syncthreads();               // the round before has been read
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float v0 = o[4 * G][2 * e + j], v1 = o[4 * G + 1][2 * e + j], v2 = o[4 * G + 2][2 * e + j], v3 = o[4 * G + 3][2 * e + j];
                    if (S::kSub == 1) {
                        write_row(2 * c + j, 64 * G + 32 * e + 4 * g, v0, v1, v2, v3, m[j], l[j], G == 0 && e == 0 && g == 0);
                    } else {
                        *reinterpret_cast<float4 *>(merge_o + (warp * 8 + 2 * c + j) * 64 + 32 * e + 4 * g) = make_float4(v0, v1, v2, v3);
                        if (g == 0 && e == 0) merge_ml[warp * 8 + 2 * c + j] = make_float2(m[j], l[j]);
                    }
                }
            if (S::kSub > 1) {
                __syncthreads();
#pragma unroll 1
                for (int i = sub * 32 + lane; i < 8 * 16; i += S::kSub * 32) {
                    const int k = i / 16, d = i % 16 * 4;
                    float mm = -INFINITY, ll = 0.0f;
                    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    for (int w = 0; w < S::kSub; ++w) mm = fmaxf(mm, merge_ml[(w * HB + hi) * 8 + k].x);
                    for (int w = 0; w < S::kSub; ++w) {
                        const float2 ml = merge_ml[(w * HB + hi) * 8 + k];
                        if (ml.y == 0.0f) continue;         // saw nothing
                        const float a = exp2_approx(ml.x - mm);
                        const float4 x = *reinterpret_cast<const float4 *>(merge_o + ((w * HB + hi) * 8 + k) * 64 + d);
                        ll = fmaf(ml.y, a, ll);
                        v.x = fmaf(x.x, a, v.x); v.y = fmaf(x.y, a, v.y); v.z = fmaf(x.z, a, v.z); v.w = fmaf(x.w, a, v.w);
                    }
                    write_row(k, 64 * G + d, v.x, v.y, v.z, v.w, mm, ll, G == 0 && d == 0);
                }
            }
        }
        if (S::kSub > 1) __syncthreads();                   // the queries of the next segment go where this was
    };

    // the row this lane names in a load: tokens 0 .. 15 twice, chunk 0 and then chunk 1 of a group
    const int k_at = chunk_at<D>(lane & 15, lane >> 4);
    int st = 0;
#pragma unroll 1
    for (unsigned u = u0; u < u1; ++u) {
        copy_next(st == 0 ? S::kStages - 1 : st - 1);       // into the stage that the tile before this one has left
        __syncwarp();
        const unsigned char *stage = mine + st * S::kStage;
        const uint32_t at = smem_u32(stage);
        const float *ks = reinterpret_cast<const float *>(stage + 2 * S::kCodes);
        const float *vs = reinterpret_cast<const float *>(stage + 2 * S::kCodes + S::kKeyScales);
        const StepMeta &meta = *reinterpret_cast<const StepMeta *>(stage + S::kStage - S::kMeta);
        const int4 now = *reinterpret_cast<const int4 *>(&meta);
        const int fl = now.x, n = now.y, full_tile = now.z;
        if (fl & 1) {
            if (have) flush();
            have = true;
            __syncwarp();
            if (lane < (int)(sizeof(StepMeta) / 4)) reinterpret_cast<int *>(&seg)[lane] = reinterpret_cast<const int *>(&meta)[lane];
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 4 * NG; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.0f;
            m[0] = m[1] = -INFINITY;
            l[0] = l[1] = 0.0f;
        }
        if (fl & 2) {
            // this lane's channels 32 w + 8 c .. + 7 of query row g, turned: what it will hold of every token's codes
            const long long turn = meta.turn;
            kc = ANY_KC && meta.kc;
            near = 127;
            low = kc || turn != 0;
            if (turn) {
                for (int i = lane; i < D / 2; i += 32) table[i] = turn_of(L.turns[i], turn);
                __syncwarp();
            }
            const int rho = seg.row0 + g;
            const bool in = rho < seg.rows;
            const __nv_bfloat16 *q = L.q + (long long)(seg.row + (in ? rho / L.g : 0)) * L.q_stride + (long long)(seg.head * L.g + (in ? rho % L.g : 0)) * D;
            float f[2 * NG][8];
#pragma unroll
            for (int w = 0; w < 2 * NG; ++w) {
                const int d0 = 32 * w + 8 * c;
                const int other = d0 < D / 2 ? d0 + D / 2 : d0 - D / 2;
                uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x;
                if (in) {
                    x = *reinterpret_cast<const uint4 *>(q + d0);
                    if (turn) y = *reinterpret_cast<const uint4 *>(q + other);
                }
                f[w][0] = bf16_lo(x.x); f[w][1] = bf16_hi(x.x); f[w][2] = bf16_lo(x.y); f[w][3] = bf16_hi(x.y);
                f[w][4] = bf16_lo(x.z); f[w][5] = bf16_hi(x.z); f[w][6] = bf16_lo(x.w); f[w][7] = bf16_hi(x.w);
                if (turn) {
                    const float h[8] = { bf16_lo(y.x), bf16_hi(y.x), bf16_lo(y.y), bf16_hi(y.y), bf16_lo(y.z), bf16_hi(y.z), bf16_lo(y.w), bf16_hi(y.w) };
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float2 cs = table[d0 % (D / 2) + i];
                        f[w][i] = fmaf(f[w][i], cs.x, h[i] * (d0 < D / 2 ? -cs.y : cs.y));
                    }
                }
            }
            // the row times a power of two that brings its largest channel to 128 .. 256
            float top = 0.0f;
#pragma unroll
            for (int w = 0; w < 2 * NG; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[w][i]));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            int e = (int)(__float_as_uint(top) >> 23);
            e = e < 8 ? 8 : e > 253 ? 253 : e;
            const float up = __uint_as_float((unsigned)(254 + 7 - e) << 23), down = __uint_as_float((unsigned)(e - 7) << 23);
#pragma unroll
            for (int j = 0; j < 2; ++j) factor[j] = __shfl_sync(0xffffffffu, down, (2 * c + j) * 4) * L.scale;
#pragma unroll
            for (int w = 0; w < 2 * NG; ++w)
#pragma unroll
                for (int i = 0; i < 8; ++i) f[w][i] *= up;
#pragma unroll
            for (int w = 0; w < 2 * NG; ++w) {
                uint32_t b[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (kc) { qa[4 * w + i] = __float_as_uint(f[w][i]); b[i] = __float_as_uint(f[w][i + 4]); }
                    else split_f16x2(f[w][i], f[w][i + 4], qa[4 * w + i], b[i]);
                }
                if (low) low_q[w * 32] = make_uint4(b[0], b[1], b[2], b[3]);
            }
        }
        // (what is above needs none of what is copied)
        asm volatile("cp.async.wait_group %0;" ::"n"(S::kStages - 1) : "memory");
        __syncwarp();
        if (n > 0) {
            // scores of 16 MT tokens (rows g, g + 8 of each 16) by 8 query rows (columns 2c, 2c + 1)
            float x[MT][4];
            // a load brings this lane the words (chunk 2 G, tokens g), (2 G, 8 + g), (2 G + 1, g), (2 G + 1, 8 + g) of 16 tokens' rows
            if (ANY_KC && kc) {
                float acc[MT][4];
#pragma unroll
                for (int t = 0; t < MT; ++t) acc[t][0] = acc[t][1] = acc[t][2] = acc[t][3] = 0.0f;
                float largest;
                if (D == 128) {
                    const float4 y = *reinterpret_cast<const float4 *>(ks + 4 * lane);
                    largest = fmaxf(fmaxf(fabsf(y.x), fabsf(y.y)), fmaxf(fabsf(y.z), fabsf(y.w)));
                } else {
                    const float2 y = *reinterpret_cast<const float2 *>(ks + 2 * lane);
                    largest = fmaxf(fabsf(y.x), fabsf(y.y));
                }
                const int e0 = (int)__reduce_max_sync(0xffffffffu, __float_as_uint(largest) >> 23), e = min(max(e0, 8), 253);
                if (e0 != 0 && (e > near + 6 || e < near - 6)) {         // (a product is 2^15 at most, and what is lost of it 2^-25)
                    const int half = (near - e) / 2, rest = near - e - half;
                    const float u0 = __uint_as_float((unsigned)(127 + half) << 23), u1 = __uint_as_float((unsigned)(127 + rest) << 23);
                    auto moved = [&](uint32_t y) { return __float_as_uint(__uint_as_float(y) * u0 * u1); };
#pragma unroll
                    for (int i = 0; i < 8 * NG; ++i) qa[i] = moved(qa[i]);
#pragma unroll 1
                    for (int w = 0; w < 2 * NG; ++w) {
                        const uint4 y = low_q[w * 32];
                        low_q[w * 32] = make_uint4(moved(y.x), moved(y.y), moved(y.z), moved(y.w));
                    }
                    near = e;
                }
#pragma unroll
                for (int G = 0; G < NG; ++G) {
                    uint32_t wd[MT][4];
#pragma unroll
                    for (int t = 0; t < MT; ++t) load_matrices<false>(wd[t], at + (k_at ^ (32 * G)) + 16 * t * (D / 2));
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        uint32_t bh[4], bl[4];              // four pairs of channels (j, j + 4)
                        const uint4 b = low_q[(2 * G + w) * 32];
                        const uint32_t qb[4] = { b.x, b.y, b.z, b.w };
                        const float2 *sc = reinterpret_cast<const float2 *>(ks + 64 * G + 32 * w + 8 * c);
                        const float2 s0 = sc[0], s1 = sc[1], s2 = sc[2], s3 = sc[3];
                        const float sa[4] = { s0.x, s0.y, s1.x, s1.y }, sb[4] = { s2.x, s2.y, s3.x, s3.y };
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            split_f16x2(__uint_as_float(qa[8 * G + 4 * w + i]) * sa[i], __uint_as_float(qb[i]) * sb[i], bh[i], bl[i]);
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            uint32_t a[4], e[4];
                            code_pairs_f16(a, wd[t][2 * w], L.bits);
                            code_pairs_f16(e, wd[t][2 * w + 1], L.bits);
                            mma_16x8x16_f16(acc[t], a[0], e[0], a[1], e[1], bh[0], bh[1]);
                            mma_16x8x16_f16(acc[t], a[2], e[2], a[3], e[3], bh[2], bh[3]);
                            mma_16x8x16_f16(acc[t], a[0], e[0], a[1], e[1], bl[0], bl[1]);
                            mma_16x8x16_f16(acc[t], a[2], e[2], a[3], e[3], bl[2], bl[3]);
                        }
                    }
                }
                const float back = __uint_as_float((unsigned)near << 23);            // made anew for each tile: the factors keep their bits
                const float by[2] = { factor[0] * back, factor[1] * back };
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][i] = acc[t][i] * by[i % 2];
            } else {
                float acc[MT][NG][4];
                auto products = [&](bool lower) {
#pragma unroll
                    for (int G = 0; G < NG; ++G) {
                        uint4 b[2];
                        if (lower) { b[0] = low_q[2 * G * 32]; b[1] = low_q[(2 * G + 1) * 32]; }
#pragma unroll
                        for (int t = 0; t < MT; ++t) {
                            uint32_t wd[4];
                            load_matrices<false>(wd, at + (k_at ^ (32 * G)) + 16 * t * (D / 2));
                            float (&d)[4] = acc[t][G];
                            d[0] = d[1] = d[2] = d[3] = 0.0f;
#pragma unroll
                            for (int w = 0; w < 2; ++w) {
                                uint32_t a[4], e[4];
                                code_pairs_f16(a, wd[2 * w], L.bits);
                                code_pairs_f16(e, wd[2 * w + 1], L.bits);
                                const uint32_t *qh = qa + 8 * G + 4 * w;
                                mma_16x8x16_f16(d, a[0], e[0], a[1], e[1], qh[0], qh[1]);
                                mma_16x8x16_f16(d, a[2], e[2], a[3], e[3], qh[2], qh[3]);
                                if (lower) {
                                    mma_16x8x16_f16(d, a[0], e[0], a[1], e[1], b[w].x, b[w].y);
                                    mma_16x8x16_f16(d, a[2], e[2], a[3], e[3], b[w].z, b[w].w);
                                }
                            }
                        }
                    }
                };
                if (low) products(true);
                else products(false);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float s0, s1 = 0.0f;
                        if (NG == 2) {
                            const float2 y = *reinterpret_cast<const float2 *>(ks + (16 * t + 8 * e + g) * 2);
                            s0 = y.x;
                            s1 = y.y;
                        } else {
                            s0 = ks[16 * t + 8 * e + g];
                        }
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float v = acc[t][0][2 * e + j] * s0;
                            if (NG == 2) v = fmaf(acc[t][NG - 1][2 * e + j], s1, v);
                            x[t][2 * e + j] = v * factor[j];
                        }
                    }
            }
            int last0 = 0, last1 = 0;                           // last tokens that the two rows see
            if (!full_tile) {
                last0 = min(n - 1, now.w + (seg.row0 + 2 * c) / L.g);
                last1 = min(n - 1, now.w + (seg.row0 + 2 * c + 1) / L.g);
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int tok = 16 * t + 8 * e + g;
                        if (tok > last0) x[t][2 * e] = -INFINITY;
                        if (tok > last1) x[t][2 * e + 1] = -INFINITY;
                    }
            }
            // m follows the maximum only when that is 2^8 above it: weights stay below 2^8, and sums are seldom rescaled.  Each row for itself, so that
            // no row's rounding goes by what another one sees.
            float top[2], base[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                top[j] = m[j];
#pragma unroll
                for (int t = 0; t < MT; ++t) top[j] = fmaxf(top[j], fmaxf(x[t][j], x[t][2 + j]));
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) top[j] = fmaxf(top[j], __shfl_xor_sync(0xffffffffu, top[j], d));
            }
            if (__any_sync(0xffffffffu, top[0] > m[0] + 8.0f || top[1] > m[1] + 8.0f)) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const bool move = top[j] > m[j] + 8.0f;
                    const float a = move ? exp2_approx(m[j] - top[j]) : 1.0f;
                    if (move) m[j] = top[j];
                    l[j] *= a;
#pragma unroll
                    for (int i = 0; i < 4 * NG; ++i) { o[i][j] *= a; o[i][2 + j] *= a; }
                }
            }
            base[0] = m[0] == -INFINITY ? 0.0f : m[0];
            base[1] = m[1] == -INFINITY ? 0.0f : m[1];
#pragma unroll
            for (int t = 0; t < MT; ++t)
#pragma unroll
                for (int e = 0; e < 2; ++e)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        x[t][2 * e + j] = exp2_approx(x[t][2 * e + j] - base[j]);
                        l[j] += x[t][2 * e + j];
                    }
            // values: channels are the rows of the product, tokens are summed
            uint32_t pw[MT][NG][2], pl[MT][NG][2];
            auto weights = [&](bool all) {
#pragma unroll
                for (int t = 0; t < MT; ++t)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float s[2];
                        if (NG == 2) {
                            const float2 y = *reinterpret_cast<const float2 *>(vs + (16 * t + 8 * e + g) * 2);
                            s[0] = y.x;
                            s[1] = y.y;
                        } else {
                            s[0] = vs[16 * t + 8 * e + g];
                        }
#pragma unroll
                        for (int G = 0; G < NG; ++G) {
                            float p0 = x[t][2 * e] * s[G], p1 = x[t][2 * e + 1] * s[G];
                            if (!all) {                     // what is not seen may hold anything
                                if (16 * t + 8 * e + g > last0) p0 = 0.0f;
                                if (16 * t + 8 * e + g > last1) p1 = 0.0f;
                            }
                            split_bf16x2(p0, p1, pw[t][G][e], pl[t][G][e]);
                        }
                    }
            };
            if (full_tile) weights(true);
            else weights(false);
#pragma unroll
            for (int t = 0; t < MT; ++t) {
                // a load brings this lane, of tokens 2c and 2c + 1 side by side, channels 64 G + 4 g .. + 3 and 64 G + 32 + 4 g .. + 3, and the same
                // of tokens 8 + 2c and 9 + 2c
#pragma unroll
                for (int G = 0; G < NG; ++G) {
                    uint32_t v[4];
                    load_matrices<true>(v, at + S::kCodes + (k_at ^ (32 * G)) + 16 * t * (D / 2));
                    const uint32_t b0 = transpose_8x8(pw[t][G][0]), b1 = transpose_8x8(pw[t][G][1]);
                    const uint32_t l0 = transpose_8x8(pl[t][G][0]), l1 = transpose_8x8(pl[t][G][1]);
                    auto four = [&](float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
                        mma_16x8x16(d, a0, a1, a2, a3, b0, b1);
                        mma_16x8x16(d, a0, a1, a2, a3, l0, l1);
                    };
                    four(o[4 * G], code_pair<0>(v[0], L.bits), code_pair<0>(v[2], L.bits), code_pair<0>(v[1], L.bits), code_pair<0>(v[3], L.bits));
                    four(o[4 * G + 1], code_pair<1>(v[0], L.bits), code_pair<1>(v[2], L.bits), code_pair<1>(v[1], L.bits), code_pair<1>(v[3], L.bits));
                    four(o[4 * G + 2], code_pair<2>(v[0], L.bits), code_pair<2>(v[2], L.bits), code_pair<2>(v[1], L.bits), code_pair<2>(v[3], L.bits));
                    four(o[4 * G + 3], code_pair<3>(v[0], L.bits), code_pair<3>(v[2], L.bits), code_pair<3>(v[1], L.bits), code_pair<3>(v[3], L.bits));
                }
            }
        }
        __syncwarp();
        st = st + 1 == S::kStages ? 0 : st + 1;
    }
    if (have) flush();
}

// Joins the partial results of segments whose tiles fell into several CTAs: a CTA per row of q and query head.  First the slots' maxima and sums,
// a thread each, then the channels, four to a lane, the warps taking slots in turn.
constexpr int kJoinWarps = 32, kJoinSlots = 640;
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) kdn_attend_join_kernel(const __grid_constant__ AttendLaunch L, int HB, int R, unsigned ctas)
{
    constexpr int LD = D / 4, PER = kJoinWarps * 32 / LD;    // lanes a slot, slots at a time
    __shared__ float weight[kJoinSlots], ms[kJoinWarps], ls[kJoinWarps];
    __shared__ float4 os[PER][LD];
    release_dependents();
    dependency_wait();
    const ReqRec *reqs = L.reqs ? L.reqs : L.inl_reqs;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, head = (int)blockIdx.y;
    for (int ri = (int)blockIdx.z; ri < L.n_reqs; ri += (int)gridDim.z) {
        const ReqRec r = reqs[ri];
        for (int i = (int)blockIdx.x; i < r.rows / L.g; i += (int)gridDim.x) {
            const int kv = head / L.g, rho = i * L.g + head % L.g;
            const unsigned seg = (unsigned)(rho / R) * (unsigned)(L.H / HB) + (unsigned)(kv / HB);
            const unsigned s0 = r.unit + seg * (unsigned)r.tiles, s1 = s0 + (unsigned)r.tiles;
            const unsigned c0 = cta_of(s0, L.units, ctas), c1 = cta_of(s1 - 1, L.units, ctas), n = c1 - c0 + 1;
            if (n == 1) continue;
            const bool second = first_unit(c0, L.units, ctas) < s0;
            // row of slot j of this segment
            auto at = [&](unsigned j) { return ((2ll * (c0 + j) + (j == 0 && second ? 1 : 0)) * HB + kv % HB) * R + rho % R; };
            float m = -INFINITY, l = 0.0f;
            for (unsigned j = threadIdx.x; j < n; j += kJoinWarps * 32) {
                const float2 ml = L.part_ml[at(j)];
                if (ml.y != 0.0f) m = fmaxf(m, ml.x);       // else it saw nothing
            }
            for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            if (lane == 0) ms[warp] = m;
            __syncthreads();
            for (int w = 0; w < kJoinWarps; ++w) m = fmaxf(m, ms[w]);
            for (unsigned j = threadIdx.x; j < n; j += kJoinWarps * 32) {
                const float2 ml = L.part_ml[at(j)];
                const float a = ml.y == 0.0f ? 0.0f : exp2_approx(ml.x - m);
                weight[j] = a;
                l = fmaf(ml.y, a, l);
            }
            for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            if (lane == 0) ls[warp] = l;
            __syncthreads();
            float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            const int d4 = (int)threadIdx.x % LD;
#pragma unroll 5
            for (unsigned j = threadIdx.x / LD; j < n; j += PER) {   // (what saw nothing left zeros)
                const float4 x = __ldcg(reinterpret_cast<const float4 *>(L.part_o + at(j) * D + d4 * 4));
                const float a = weight[j];
                v.x = fmaf(x.x, a, v.x); v.y = fmaf(x.y, a, v.y); v.z = fmaf(x.z, a, v.z); v.w = fmaf(x.w, a, v.w);
            }
            os[threadIdx.x / LD][d4] = v;
            __syncthreads();
            if (threadIdx.x < D) {
                float ll = 0.0f, o = 0.0f;
                for (int w = 0; w < kJoinWarps; ++w) ll += ls[w];
                for (int w = 0; w < PER; ++w) o += reinterpret_cast<const float *>(os[w])[threadIdx.x];
                const long long row = r.row + i;
                L.out[row * L.out_stride + (long long)head * D + threadIdx.x] = __float2bfloat16(ll == 0.0f ? 0.0f : o / ll);
                if (L.lse && threadIdx.x == 0) L.lse[row * (L.H * L.g) + head] = ll == 0.0f ? -INFINITY : (m + log2f(ll)) * 0.69314718055994531f;
            }
            __syncthreads();
        }
    }
}

// The same where a segment has no more parts than a warp has lanes (many rows, short contexts a CTA): a warp a row.  A call with either, in
// microseconds: 57.6 and 79.9 with the other (32 requests of 4096 tokens, 8 heads, a token each: 9 or 10 parts), 58 and 223 (one request of 2048, 203 tokens: 5 or 6).
constexpr int kJoinFew = 32;
template <int D>
__global__ void __launch_bounds__(256) kdn_attend_join_few_kernel(const __grid_constant__ AttendLaunch L, int HB, int R, unsigned ctas)
{
    constexpr int E = D / 32;
    release_dependents();
    dependency_wait();
    const ReqRec *reqs = L.reqs ? L.reqs : L.inl_reqs;
    const int warp = (int)threadIdx.x >> 5, lane = (int)threadIdx.x & 31, heads = L.H * L.g;
    for (int ri = (int)blockIdx.y; ri < L.n_reqs; ri += (int)gridDim.y) {
        const ReqRec r = reqs[ri];
        const long long rows = (long long)(r.rows / L.g) * heads;
        for (long long x = (long long)blockIdx.x * 8 + warp; x < rows; x += (long long)gridDim.x * 8) {
            const int i = (int)(x / heads), head = (int)(x % heads);
            const int kv = head / L.g, rho = i * L.g + head % L.g;
            const unsigned seg = (unsigned)(rho / R) * (unsigned)(L.H / HB) + (unsigned)(kv / HB);
            const unsigned s0 = r.unit + seg * (unsigned)r.tiles, s1 = s0 + (unsigned)r.tiles;
            const unsigned c0 = cta_of(s0, L.units, ctas), c1 = cta_of(s1 - 1, L.units, ctas), n = c1 - c0 + 1;
            if (n == 1) continue;
            const bool second = first_unit(c0, L.units, ctas) < s0;
            auto at = [&](unsigned j) { return ((2ll * (c0 + j) + (j == 0 && second ? 1 : 0)) * HB + kv % HB) * R + rho % R; };
            float2 ml = make_float2(-INFINITY, 0.0f);
            if ((unsigned)lane < n) ml = L.part_ml[at((unsigned)lane)];
            if (ml.y == 0.0f) ml.x = -INFINITY;              // saw nothing
            float m = ml.x;
            for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
            const float mine = ml.y == 0.0f ? 0.0f : exp2_approx(ml.x - m);
            float l = ml.y * mine;
            for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(0xffffffffu, l, d);
            float o[E] = {};
#pragma unroll 4
            for (unsigned j = 0; j < n; ++j) {               // (what saw nothing left zeros)
                const float a = __shfl_sync(0xffffffffu, mine, (int)j);
                const float *from = L.part_o + at(j) * D + E * lane;
                float x[E];
                if (E == 4) {
                    const float4 y = __ldcg(reinterpret_cast<const float4 *>(from));
                    x[0] = y.x; x[1 % E] = y.y; x[2 % E] = y.z; x[3 % E] = y.w;
                } else {
                    const float2 y = __ldcg(reinterpret_cast<const float2 *>(from));
                    x[0] = y.x; x[1] = y.y;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) o[e] = fmaf(x[e], a, o[e]);
            }
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
            const long long row = r.row + i;
            uint32_t *to = reinterpret_cast<uint32_t *>(L.out + row * L.out_stride + (long long)head * D + E * lane);
#pragma unroll
            for (int e = 0; e < E / 2; ++e) to[e] = pack_bf16x2(o[2 * e] * inv, o[2 * e + 1] * inv);
            if (L.lse && lane == 0) L.lse[row * heads + head] = l == 0.0f ? -INFINITY : (m + log2f(l)) * 0.69314718055994531f;
        }
    }
}

}  // namespace kdn
