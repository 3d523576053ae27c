// Attention of drafted tokens over a paged cache.
//
// One wave takes one query row (stream, drafted token, query head) and walks the keys that it sees 64 at a time, a key per lane, with
// the running maximum and sum of a softmax; the values are then added up with a channel group per lane.
#include <math.h>

#include "common.h"

namespace {

struct attend_args {
    const uint16_t *k, *v, *q, *k_new, *v_new;   // k, v: the layer's part of the pool
    const int32_t *table, *len, *n_new, *sel;
    const uint32_t* mask;
    uint16_t* out;
    float* lse;
    uint32_t* flags;
    int P, H, page, d, cap, B, T, G, n_sel, unit;
    float scale;
};

template <bool BF16>
__device__ __forceinline__ float widen(uint16_t x) {
    if (BF16) return __uint_as_float((uint32_t)x << 16);
    return (float)__builtin_bit_cast(_Float16, x);
}
template <bool BF16>
__device__ __forceinline__ uint16_t narrow(float x) {
    if (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    return __builtin_bit_cast(uint16_t, (_Float16)x);
}

template <bool BF16>
__global__ __launch_bounds__(64) void attend_row_kernel(attend_args a) {
    __shared__ float w[64];
    __shared__ const uint16_t* rows[64];
    const int HG = a.H * a.G, lane = threadIdx.x;
    const int64_t row = blockIdx.x;
    const int hq = (int)(row % HG), i = (int)(row / HG % a.T), b = (int)(row / HG / a.T), h = hq / a.G;
    int drafted = a.n_new ? a.n_new[b] : a.T, len = a.len[b];
    if (drafted < 0 || drafted > a.T || len < 0 || len > a.cap * a.page) {
        if (lane == 0) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        drafted = min(max(drafted, 0), a.T);
        len = min(max(len, 0), a.cap * a.page);
    }
    if (i >= drafted) return;
    const uint16_t* q = a.q + row * a.d;
    const int ctx = !a.sel ? len : a.unit == SWARM_SEL_PAGES ? a.n_sel * a.page : a.n_sel;
    const int keys = ctx + (a.k_new ? drafted : 0);
    const int32_t* sel = a.sel ? a.sel + ((int64_t)b * a.H + h) * a.n_sel : nullptr;
    float m = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};   // channels lane, lane + 64, ...
    for (int at = 0; at < keys; at += 64) {
        const int x = at + lane;
        const uint16_t *kr = nullptr, *vr = nullptr;
        if (x < ctx) {
            int pos = x;
            if (sel) {
                const int e = sel[a.unit == SWARM_SEL_PAGES ? x / a.page : x];
                const int limit = a.unit == SWARM_SEL_PAGES ? a.cap : a.cap * a.page;
                pos = a.unit == SWARM_SEL_PAGES ? e * a.page + x % a.page : e;
                if (e < 0 || e >= limit) {
                    if (e != -1) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
                    pos = len;
                }
            }
            if (pos < len) {
                const int id = a.table[(int64_t)b * a.cap + pos / a.page];
                if (id < 0 || id >= a.P) {
                    atomicOr(a.flags, SWARM_DEV_BAD_PAGE);
                } else {
                    const int64_t at_row = (((int64_t)id * a.H + h) * a.page + pos % a.page) * a.d;
                    kr = a.k + at_row;
                    vr = a.v + at_row;
                }
            }
        } else if (x < keys) {
            const int j = x - ctx;
            const bool sees = a.mask ? a.mask[((int64_t)b * a.T + i) * ((a.T + 31) / 32) + j / 32] >> (j % 32) & 1u : j <= i;
            if (sees) {
                const int64_t at_row = (((int64_t)b * a.T + j) * a.H + h) * a.d;
                kr = a.k_new + at_row;
                vr = a.v_new + at_row;
            }
        }
        float s = -INFINITY;
        if (kr) {
            s = 0.f;
            for (int c = 0; c < a.d; ++c) s += widen<BF16>(q[c]) * widen<BF16>(kr[c]);
            s *= a.scale;
        }
        float top = s;
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
        const float next = fmaxf(m, top), base = next == -INFINITY ? 0.f : next;
        const float p = kr ? expf(s - base) : 0.f, old = expf(m - base);
        float part = p;
        for (int o = 32; o; o >>= 1) part += __shfl_xor(part, o);
        sum = sum * old + part;
        m = next;
        __syncthreads();
        w[lane] = p;
        rows[lane] = vr;
        __syncthreads();
        for (int c = 0; c < 4; ++c) acc[c] *= old;
        for (int j = 0; j < 64; ++j) {
            if (w[j] == 0.f) continue;
            for (int c = 0; c < 4; ++c)
                if (lane + 64 * c < a.d) acc[c] += w[j] * widen<BF16>(rows[j][lane + 64 * c]);
        }
    }
    for (int c = 0; c < 4; ++c)
        if (lane + 64 * c < a.d) a.out[row * a.d + lane + 64 * c] = narrow<BF16>(sum == 0.f ? 0.f : acc[c] / sum);
    if (a.lse && lane == 0) a.lse[row] = sum == 0.f ? -INFINITY : m + logf(sum);
}

}  // namespace

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
    if (G < 1 || (int64_t)T * G > (1 << 20)) SWARM_REJECT(ctx, "tree_attend: G=%d below 1 or T*G above 2^20", G);
    const int64_t rows = (int64_t)B * T * cache->H * G;
    if (rows > ((int64_t)1 << 30)) SWARM_REJECT(ctx, "tree_attend: B*T*H*G above 2^30");
    if (sel && (n_sel < 1 || n_sel > (1 << 30) / (unit == SWARM_SEL_PAGES ? cache->page : 1)))
        SWARM_REJECT(ctx, "tree_attend: n_sel=%d below 1, or above 2^30 tokens", n_sel);
    if (sel && unit != SWARM_SEL_PAGES && unit != SWARM_SEL_TOKENS) SWARM_REJECT(ctx, "tree_attend: unknown unit %d", unit);
    if (!(fabsf(scale) < INFINITY)) SWARM_REJECT(ctx, "tree_attend: scale must be finite");
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
    a.P = cache->P, a.H = cache->H, a.page = cache->page, a.d = cache->d, a.cap = cache->cap;
    a.B = B, a.T = T, a.G = G, a.n_sel = n_sel, a.unit = unit;
    a.scale = scale;
    if (cache->dtype == SWARM_BF16) hipLaunchKernelGGL(attend_row_kernel<true>, dim3((unsigned)rows), dim3(64), 0, ctx->stream, a);
    else hipLaunchKernelGGL(attend_row_kernel<false>, dim3((unsigned)rows), dim3(64), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "attend_row_kernel");
}
