// Attention of drafted tokens over a paged cache: the entry point, and the kernels for bf16 (attend_core.h).
#include "attend_core.h"

void launch_attend_bf16(const attend_args& a, hipStream_t stream) { launch_attend_type<true>(a, stream); }

extern "C" swarm_status swarm_tree_attend(swarm_ctx* ctx, const swarm_cache* cache, int32_t layer, const void* q, const void* k_new,
                                          const void* v_new, int32_t B, int32_t T, int32_t G, const int32_t* n_new, const uint32_t* mask,
                                          const int32_t* sel, int32_t n_sel, int32_t unit, float scale, void* out, float* lse) {
    SWARM_ENTER(ctx);
    swarm_status st = swarm_check_cache(ctx, "tree_attend", cache);
    if (st != SWARM_OK) return st;
    if (!q || !out) SWARM_REJECT(ctx, "tree_attend: NULL q or out");
    if ((k_new == nullptr) != (v_new == nullptr)) SWARM_REJECT(ctx, "tree_attend: k_new and v_new go together");
    if (layer < 0 || layer >= cache->L) SWARM_REJECT(ctx, "tree_attend: layer=%d outside [0,L=%d)", layer, cache->L);
    if (B < 1 || B > cache->rows) SWARM_REJECT(ctx, "tree_attend: B=%d outside [1,rows=%d]", B, cache->rows);
    if (T < 1 || T > 256) SWARM_REJECT(ctx, "tree_attend: T=%d outside [1,256]", T);
    if (G < 1 || G > 1024) SWARM_REJECT(ctx, "tree_attend: G=%d outside [1,1024]", G);
    const int64_t rows = (int64_t)B * T * cache->H * G;
    if (rows > ((int64_t)1 << 30)) SWARM_REJECT(ctx, "tree_attend: B*T*H*G above 2^30");
    if ((int64_t)cache->P * cache->H * cache->page * (cache->d / 8) > UINT32_MAX || (int64_t)B * T * cache->H * (cache->d / 8) > UINT32_MAX)
        SWARM_REJECT(ctx, "tree_attend: a layer of the pool, or k_new, of 64 GiB or more");
    if (sel && (n_sel < 1 || n_sel > (1 << 30) / (unit == SWARM_SEL_PAGES ? cache->page : 1)))
        SWARM_REJECT(ctx, "tree_attend: n_sel=%d below 1, or above 2^30 tokens", n_sel);
    if (sel && unit != SWARM_SEL_PAGES && unit != SWARM_SEL_TOKENS) SWARM_REJECT(ctx, "tree_attend: unknown unit %d", unit);
    const float scale_log2 = scale * 1.44269504088896341f;
    if (!(fabsf(scale_log2) < INFINITY)) SWARM_REJECT(ctx, "tree_attend: scale / ln 2 must be finite");
    if (swarm_misaligned(q, 16) || swarm_misaligned(out, 16) || swarm_misaligned(k_new, 16) || swarm_misaligned(v_new, 16) || swarm_misaligned(lse, 4) ||
        swarm_misaligned(n_new, 4) || swarm_misaligned(mask, 4) || swarm_misaligned(sel, 4))
        SWARM_REJECT(ctx, "tree_attend: q, k_new, v_new and out must be 16-byte aligned, the others 4-byte");
    const size_t row = 2 * (size_t)cache->d, pool = row * cache->L * cache->P * cache->H * cache->page, news = row * B * T * cache->H;
    const size_t bits = 4 * (size_t)B * T * ((T + 31) / 32), picks = sel ? 4 * (size_t)B * cache->H * n_sel : 0;
    const swarm_range outs[] = {{out, row * rows}, {lse, 4 * (size_t)rows}};
    const swarm_range ins[] = {{q, row * rows},        {k_new, news},        {v_new, news},     {cache->k, pool}, {cache->v, pool},
                               {cache->table, 4 * (size_t)cache->rows * cache->cap}, {cache->len, 4 * (size_t)cache->rows}, {n_new, 4 * (size_t)B},
                               {mask, bits},           {sel, picks}};
    if (swarm_overlap(outs, 2, ins, 10)) SWARM_REJECT(ctx, "tree_attend: out or lse overlaps an input, or the other");

    attend_args a{};
    // Up to 32 rows (16 of heads wider than 128, which take more registers) go to the kernel whose waves have keys of their own, more to the one whose waves
    // share them: as few tiles of up to 256 (128) rows as they need, and in each the smallest of that kernel's forms.
    const int M = T * G, DP = attend_width(cache->d), most = DP > 128 ? 128 : 256;
    a.tiles = (M + most - 1) / most;
    const int each = (M + a.tiles - 1) / a.tiles;
    a.rows = each <= 16 ? 16 : each <= 32 ? 32 : each <= 64 ? 64 : each <= 96 && DP > 128 ? 96 : each <= 128 ? 128 : each <= 192 ? 192 : 256;
    // as many parts as workgroups are resident at once, and no more than there can be units
    const int64_t slots = !sel ? (int64_t)cache->cap * cache->page : unit == SWARM_SEL_PAGES ? (int64_t)n_sel * cache->page : n_sel;
    const int64_t units = (int64_t)B * cache->H * ((slots + ATTEND_UNIT - 1) / ATTEND_UNIT);
    if (units > INT32_MAX - 65536) SWARM_REJECT(ctx, "tree_attend: contexts of up to %lld times 128 keys, above 2^31", (long long)units);
    const int resident = 256 * ((DP <= 128 ? a.rows <= 128 : a.rows > 16 && a.rows <= 64) ? 2 : 1), want = a.tiles < resident ? resident / a.tiles : 1;
    a.parts = (int)(units < want ? units : want);
    // Scratch for what the parts leave, a slot for each pair and one more for each part.  The parts' share is taken as its bound over all launches
    // (512 workgroups of up to 128 rows, 256 of up to 256, or one part), which grows with the rows, so that smaller calls never need more.
    const size_t rows_all = (size_t)a.tiles * a.rows, share = 512 * rows_all < 65536 ? 512 * rows_all : rows_all > 65536 ? rows_all : 65536;
    const size_t heads = (4 * ((size_t)B + 1) + 15) / 16 * 16, left = (size_t)B * cache->H * rows_all + share;
    st = swarm_scratch(ctx, &ctx->attend, &ctx->attend_bytes, heads + left * (DP + 2) * 4);
    if (st != SWARM_OK) return st;
    a.starts = static_cast<int32_t*>(ctx->attend);
    a.part_o = reinterpret_cast<float*>(static_cast<char*>(ctx->attend) + heads);
    a.part_ml = a.part_o + left * DP;
    while ((1 << a.page_log2) < cache->page) ++a.page_log2;
    a.per_g = (uint32_t)(((uint64_t)1 << 32) / G + (((uint64_t)1 << 32) % G != 0));
    const int64_t base = (int64_t)layer * cache->P * cache->H * cache->page * cache->d;
    a.k = static_cast<const uint16_t*>(cache->k) + base;
    a.v = static_cast<const uint16_t*>(cache->v) + base;
    a.q = static_cast<const uint16_t*>(q);
    a.k_new = static_cast<const uint16_t*>(k_new);
    a.v_new = static_cast<const uint16_t*>(v_new);
    a.table = cache->table;
    a.len = cache->len;
    a.n_new = n_new;
    a.sel = sel;
    a.mask = mask;
    a.out = static_cast<uint16_t*>(out);
    a.lse = lse;
    a.flags = ctx->dev_flags;
    a.P = cache->P, a.H = cache->H, a.d = cache->d, a.cap = cache->cap;
    a.B = B, a.T = T, a.G = G, a.n_sel = n_sel, a.unit = unit;
    a.scale_log2 = scale_log2;
    cache->dtype == SWARM_BF16 ? launch_attend_bf16(a, ctx->stream) : launch_attend_fp16(a, ctx->stream);
    return swarm_check_launch(ctx, "attend");
}
