// kdn_attend: attention of new tokens over stored chunks that stay in 4 bits.
#include "kdn_ops.cuh"
#include "kdn_attend_step.cuh"
#include "kdn_attend_block.cuh"

#include <cmath>
#include <new>
#include <vector>

using namespace kdn;

namespace {

// Requests of up to this many rows a KV head go to the kernel that is bound by the bytes of the chunks and takes eight rows a pass; the others to the
// one that is bound by the scores and takes 256.  Both, in microseconds (one request of 4096 tokens, one of 65536, eight of 8192, eight of 8192 with keys in
// channel groups; all of 8 heads of 128, turned):
//     rows    eight a pass             256 a pass
//     16       17   54   58   66       29  135  134  134
//     32       24   98   95  111       30  136  136  136
//     40       31  122  115  134       30  137  136  136
//     48       32  141  134  157       30  136  136  136
//     64       38  185  173  203       31  136  137  136
constexpr int kStepRows = 40;

// As many heads a unit as the pool has, up to eight: warps that share no head have nothing to add up.  With eight, four and two heads a unit of eight heads of 128, in microseconds:
// a token over ten documents of 1024 20.1, 18.9 and 18.8; over 65536 tokens 37.5, 36.6 and 37.4; over 4096 15.6, 15.8 and 20.2; 32 requests of 8192 with keys
// in channel groups 122.4, 127.8 and 128.8; eight of 8192 with 16 rows 52.0, 54.9 and 55.7, with 8 rows 45.3, 39.2 and 38.0.
int heads_of_unit(int H) { return H % 8 == 0 ? 8 : H % 4 == 0 ? 4 : H % 2 == 0 ? 2 : 1; }

// How the requests of one of the two kernels are cut.
struct Cut {
    int HB, R, tile;                        // heads and rows of a unit, tokens
    unsigned long long units;
    unsigned ctas;                          // most that are launched
};
struct Plan {
    Cut step, block;
    size_t reqs, parts, ml, o, whole;
};

// From sizes alone, so that a workspace stays large enough while positions move.  false: too many units.
bool plan_of(const kdn_pool_desc &pool, const kdn_attend_req *reqs, int n, int g, int sm_count, Plan *out)
{
    Plan w{};
    const int H = pool.n_kv_heads;
    w.step = Cut{ heads_of_unit(H), 8, 256 / heads_of_unit(H), 0, 2u * (unsigned)sm_count };
    w.block = Cut{ 1, kBlockRows, kBlockTile, 0, (unsigned)sm_count };
    size_t parts = 0;
    for (int i = 0; i < n; ++i) {
        if (reqs[i].n_q == 0) continue;
        const unsigned long long rows = (unsigned long long)reqs[i].n_q * (unsigned)g;
        Cut &c = rows <= (unsigned)kStepRows ? w.step : w.block;
        unsigned long long tiles = 0;
        for (int j = 0; j < reqs[i].n_parts; ++j) {
            const int T = reqs[i].parts[j].n_tokens;
            tiles += ((unsigned)T + (unsigned)c.tile - 1) / (unsigned)c.tile;
            parts += T > 0;
        }
        parts += 1;
        c.units += (tiles ? tiles : 1) * ((rows + (unsigned)c.R - 1) / (unsigned)c.R) * (unsigned)(H / c.HB);
        if (c.units > 0x7fffffffull) return false;
    }
    if (n > kInlineReqs || parts > (size_t)kInlineParts) {
        w.reqs = align_up(sizeof(ReqRec) * (size_t)n, 256);
        w.parts = align_up(sizeof(PartRec) * parts, 256);
    }
    size_t rows = 0;                                       // of partial results: two slots a CTA
    for (Cut *c : { &w.step, &w.block }) {
        if (c->units < c->ctas) c->ctas = (unsigned)c->units;
        const size_t r = 2 * (size_t)c->ctas * (size_t)(c->HB * c->R);
        rows = r > rows ? r : rows;
    }
    w.ml = align_up(rows * sizeof(float2), 256);
    w.o = rows * (size_t)pool.head_dim * 4;
    w.whole = w.reqs + w.parts + w.ml + w.o;
    *out = w;
    return true;
}

template <int D, int HB, bool ANY_KC, bool WHOLE>
kdn_status launch_step_form(const Context &c, const AttendLaunch &L, unsigned ctas, cudaStream_t stream)
{
    using S = StepShape<D, HB>;
    const kdn_status st = allow_smem<kdn_attend_step_kernel<D, HB, ANY_KC, WHOLE>>(c, S::kSmem);
    return st != KDN_OK ? st : launch(c, kdn_attend_step_kernel<D, HB, ANY_KC, WHOLE>, dim3(ctas), S::kThreads, (size_t)S::kSmem, stream, L);
}

template <int D, int HB>
kdn_status launch_step(const Context &c, const AttendLaunch &L, bool any_kc, unsigned ctas, cudaStream_t stream)
{
    const bool whole = L.H == HB;
    if (any_kc) return whole ? launch_step_form<D, HB, true, true>(c, L, ctas, stream) : launch_step_form<D, HB, true, false>(c, L, ctas, stream);
    return whole ? launch_step_form<D, HB, false, true>(c, L, ctas, stream) : launch_step_form<D, HB, false, false>(c, L, ctas, stream);
}

template <int D>
kdn_status launch_block(const Context &c, const AttendLaunch &L, unsigned ctas, cudaStream_t stream)
{
    const kdn_status st = allow_smem<kdn_attend_block_kernel<D>>(c, BlockShape<D>::kSmem);
    return st != KDN_OK ? st : launch(c, kdn_attend_block_kernel<D>, dim3(ctas), kBlockThreads, (size_t)BlockShape<D>::kSmem, stream, L);
}

constexpr int64_t kMostPos = (int64_t)1 << 40;

kdn_status check_reqs(const kdn_pool_desc *pool, const kdn_attend_req *reqs, int n_reqs, int n_q_heads, bool *moved)
{
    kdn_status st = check_pool_shape(pool);
    if (st != KDN_OK) return st;
    if (n_reqs < 0 || (n_reqs > 0 && !reqs)) return KDN_E_INVAL;
    if (n_q_heads <= 0 || n_q_heads % pool->n_kv_heads) return KDN_E_INVAL;
    if (pool->head_dim != 64 && pool->head_dim != 128) return KDN_E_UNSUPPORTED;
    if (n_q_heads > 65535) return KDN_E_UNSUPPORTED;
    int64_t rows = 0, all_parts = 0;
    *moved = false;
    for (int i = 0; i < n_reqs; ++i) {
        const kdn_attend_req &r = reqs[i];
        if (r.n_q < 0 || r.n_parts < 0 || r.q_pos < 0 || r.q_pos >= kMostPos) return KDN_E_INVAL;
        if (r.n_parts > 0 && (!r.parts || !r.part_pos)) return KDN_E_INVAL;
        rows += r.n_q;
        all_parts += r.n_parts;
        if (rows * n_q_heads > 0x7fffffff || all_parts > 0x7fffffff) return KDN_E_UNSUPPORTED;
        for (int j = 0; j < r.n_parts; ++j) {
            const kdn_chunk &k = r.parts[j];
            st = check_stored_chunk(pool, &k);
            if (st != KDN_OK) return st;
            if (k.codec != KDN_CODEC_INT4_G64 && k.codec != KDN_CODEC_INT4_KC64) return KDN_E_UNSUPPORTED;
            if (k.mem != KDN_MEM_DEVICE) return KDN_E_UNSUPPORTED;
            if (k.n_tokens > kMostTokens) return KDN_E_UNSUPPORTED;
            if (r.part_pos[j] < 0 || r.part_pos[j] >= kMostPos || k.base_pos < 0 || k.base_pos >= kMostPos) return KDN_E_INVAL;
            if (k.n_tokens > 0 && r.part_pos[j] != k.base_pos) *moved = true;
        }
    }
    return KDN_OK;
}

}  // namespace

extern "C" {

kdn_status kdn_validate_attend(const kdn_pool_desc *pool, int layer, const kdn_attend_req *reqs, int n_reqs, const kdn_attend_io *io)
{
    if (!io) return KDN_E_INVAL;
    bool moved;
    const kdn_status st = check_reqs(pool, reqs, n_reqs, io->n_q_heads, &moved);
    if (st != KDN_OK) return st;
    if (layer < 0 || layer >= pool->n_layers) return KDN_E_INVAL;
    if (!usable_scale(io->scale)) return KDN_E_INVAL;
    if (io->rope_style != 0) return KDN_E_UNSUPPORTED;
    if (moved && (!(io->rope_theta > 0.0) || io->rope_theta > 1e300)) return KDN_E_INVAL;
    int64_t rows = 0;
    for (int i = 0; i < n_reqs; ++i) rows += reqs[i].n_q;
    if (rows == 0) return KDN_OK;
    const int64_t width = (int64_t)io->n_q_heads * pool->head_dim;
    if (!io->q || !io->out || io->q_stride < width || io->out_stride < width) return KDN_E_INVAL;
    if (!aligned(io->q, 16) || !aligned(io->out, 16) || io->q_stride % 8 || io->out_stride % 8 || !aligned(io->lse, 4)) return KDN_E_ALIGN;
    return KDN_OK;
}

kdn_status kdn_attend_workspace(kdn_ctx *ctx, int pool_id, const kdn_attend_req *reqs, int n_reqs, int n_q_heads, size_t *bytes)
{
    Context c;
    PoolShape pool;
    if (!bytes || !context_of(ctx, &c) || !pool_of(ctx, pool_id, &pool)) return KDN_E_INVAL;
    *bytes = 0;
    bool moved;
    const kdn_status st = check_reqs(&pool.desc, reqs, n_reqs, n_q_heads, &moved);
    if (st != KDN_OK) return st;
    Plan w;
    if (!plan_of(pool.desc, reqs, n_reqs, n_q_heads / pool.desc.n_kv_heads, c.sm_count, &w)) return KDN_E_UNSUPPORTED;
    *bytes = w.whole;
    return KDN_OK;
}

kdn_status kdn_attend(kdn_ctx *ctx, int pool_id, int layer, const kdn_attend_req *reqs, int n_reqs, const kdn_attend_io *io, void *cuda_stream)
{
    Context c;
    PoolShape pool;
    if (!context_of(ctx, &c) || !pool_of(ctx, pool_id, &pool)) return KDN_E_INVAL;
    kdn_status st = kdn_validate_attend(&pool.desc, layer, reqs, n_reqs, io);
    if (st != KDN_OK) return st;
    Plan w;
    const int H = pool.desc.n_kv_heads, D = pool.desc.head_dim, g = io->n_q_heads / H;
    if (!plan_of(pool.desc, reqs, n_reqs, g, c.sm_count, &w)) return KDN_E_UNSUPPORTED;
    if (w.whole && (!io->workspace || io->workspace_bytes < w.whole)) return KDN_E_INVAL;
    if (!aligned(io->workspace, 16)) return KDN_E_ALIGN;
    if (make_current(c.device) != KDN_OK) return KDN_E_CUDA;
    cudaStream_t stream = (cudaStream_t)cuda_stream;
    const size_t row_elems = (size_t)H * D;
    unsigned char *at = static_cast<unsigned char *>(io->workspace);
    AttendLaunch L{};
    L.q = static_cast<const __nv_bfloat16 *>(io->q);
    L.out = static_cast<__nv_bfloat16 *>(io->out);
    L.lse = io->lse;
    L.part_ml = reinterpret_cast<float2 *>(at + w.reqs + w.parts);
    L.part_o = reinterpret_cast<float *>(at + w.reqs + w.parts + w.ml);
    L.status = c.status;
    L.q_stride = io->q_stride;
    L.out_stride = io->out_stride;
    L.wait_limit_ns = c.wait_limit_ns;
    L.scale = (float)(io->scale * kLog2e);
    L.H = H;
    L.g = g;
    L.bits = Bits{ 0x000f000fu, 0x43084308u, 0x64086408u, 0x00f000f0u, 0x64806480u, 0x2c002c00u, 0xd480d480u };
    std::vector<ReqRec> rr;
    std::vector<PartRec> pp;
    bool angles = false;
    for (const bool block : { false, true }) {
        const Cut &cut = block ? w.block : w.step;
        if (cut.units == 0) continue;
        int row = 0, n_q = 0;
        unsigned units = 0;
        bool kc = false, turned = false;
        rr.clear();
        pp.clear();
        try {
            for (int i = 0; i < n_reqs; row += reqs[i].n_q, ++i) {
                const kdn_attend_req &r = reqs[i];
                if (r.n_q == 0 || ((int64_t)r.n_q * g > kStepRows) != block) continue;
                const int first = (int)pp.size();
                int tiles = 0;
                for (int j = 0; j < r.n_parts; ++j) {
                    const kdn_chunk &k = r.parts[j];
                    const int64_t ahead = r.q_pos - r.part_pos[j], seen = ahead + r.n_q < k.n_tokens ? ahead + r.n_q : k.n_tokens;
                    if (seen <= 0) continue;
                    const size_t T = (size_t)k.n_tokens, plane = T * row_elems / 2, by_row = T * row_elems / 64;
                    const int by_channel = k.codec == KDN_CODEC_INT4_KC64;
                    const size_t per_layer = by_row + (by_channel ? (T + 63) / 64 * row_elems : by_row);
                    const unsigned char *base = static_cast<const unsigned char *>(k.data);
                    pp.push_back(PartRec{ base + 2 * (size_t)layer * plane,
                                          reinterpret_cast<const float *>(base + 2 * (size_t)pool.desc.n_layers * plane) + (size_t)layer * per_layer,
                                          ahead, k.base_pos - r.part_pos[j], k.n_tokens, (int)seen, tiles, by_channel });
                    tiles += (int)((seen + cut.tile - 1) / cut.tile);
                    kc = kc || by_channel;
                    turned = turned || k.base_pos != r.part_pos[j];
                }
                if (tiles == 0) {                          // sees nothing: a unit of no tokens writes its rows
                    pp.push_back(PartRec{});
                    tiles = 1;
                }
                rr.push_back(ReqRec{ row, r.n_q * g, first, (int)pp.size() - first, units, tiles });
                units += (unsigned)tiles * (((unsigned)r.n_q * (unsigned)g + (unsigned)cut.R - 1) / (unsigned)cut.R) * (unsigned)(H / cut.HB);
                n_q = r.n_q > n_q ? r.n_q : n_q;
            }
        } catch (const std::bad_alloc &) { return KDN_E_NOMEM; }
        const int n = (int)rr.size();
        L.n_reqs = n;
        L.units = units;
        if (turned && !angles) {
            // (products in 64-bit mantissas: 64 of them are still off by less than a step of a double)
            const long double ratio = powl((long double)io->rope_theta, -2.0L / D);
            long double x = 1.0L / (2.0L * 3.14159265358979323846264338L);
            for (int i = 0; i < D / 2; ++i, x *= ratio) L.turns[i] = (double)x;
            angles = true;
        }
        if (w.reqs) {
            st = put_records(c, at, rr.data(), sizeof(ReqRec) * rr.size(), stream);
            if (st == KDN_OK) st = put_records(c, at + w.reqs, pp.data(), sizeof(PartRec) * pp.size(), stream);
            if (st != KDN_OK) return st;
            L.reqs = reinterpret_cast<const ReqRec *>(at);
            L.parts = reinterpret_cast<const PartRec *>(at + w.reqs);
        } else {
            std::memcpy(L.inl_reqs, rr.data(), sizeof(ReqRec) * rr.size());
            std::memcpy(L.inl_parts, pp.data(), sizeof(PartRec) * pp.size());
        }
        const unsigned ctas = units < cut.ctas ? units : cut.ctas;
        if (block) {
            st = D == 64 ? launch_block<64>(c, L, ctas, stream) : launch_block<128>(c, L, ctas, stream);
        } else {
            switch (cut.HB * 1000 + D) {
            case 8128: st = launch_step<128, 8>(c, L, kc, ctas, stream); break;
            case 4128: st = launch_step<128, 4>(c, L, kc, ctas, stream); break;
            case 2128: st = launch_step<128, 2>(c, L, kc, ctas, stream); break;
            case 1128: st = launch_step<128, 1>(c, L, kc, ctas, stream); break;
            case 8064: st = launch_step<64, 8>(c, L, kc, ctas, stream); break;
            case 4064: st = launch_step<64, 4>(c, L, kc, ctas, stream); break;
            case 2064: st = launch_step<64, 2>(c, L, kc, ctas, stream); break;
            default: st = launch_step<64, 1>(c, L, kc, ctas, stream); break;
            }
        }
        if (st != KDN_OK) return st;
        unsigned most = 1;                                 // CTAs that a segment's tiles fall into
        for (int i = 0; i < n; ++i) {
            const unsigned end = i + 1 < n ? rr[(size_t)i + 1].unit : units;
            for (unsigned s = rr[(size_t)i].unit; s < end; s += (unsigned)rr[(size_t)i].tiles) {
                const unsigned c0 = cta_of(s, units, ctas), c1 = cta_of(s + (unsigned)rr[(size_t)i].tiles - 1, units, ctas);
                most = c1 - c0 + 1 > most ? c1 - c0 + 1 : most;
            }
        }
        if (most == 1) continue;
        const unsigned zn = (unsigned)(n < 65535 ? n : 65535);
        if (most <= (unsigned)kJoinFew) {
            const unsigned long long warps = (unsigned long long)n_q * (unsigned)io->n_q_heads;
            const dim3 grid((unsigned)(warps / 8 < 65535 ? (warps + 7) / 8 : 65535), zn);
            st = D == 64 ? launch(c, kdn_attend_join_few_kernel<64>, grid, 256, 0, stream, L, cut.HB, cut.R, ctas)
                         : launch(c, kdn_attend_join_few_kernel<128>, grid, 256, 0, stream, L, cut.HB, cut.R, ctas);
        } else {
            const dim3 grid((unsigned)(n_q < 65535 ? n_q : 65535), (unsigned)io->n_q_heads, zn);
            st = D == 64 ? launch(c, kdn_attend_join_kernel<64>, grid, kJoinWarps * 32, 0, stream, L, cut.HB, cut.R, ctas)
                         : launch(c, kdn_attend_join_kernel<128>, grid, kJoinWarps * 32, 0, stream, L, cut.HB, cut.R, ctas);
        }
        if (st != KDN_OK) return st;
    }
    return KDN_OK;
}

}  // extern "C"
