// Beam search's selection over beams and vocabulary.
#include <math.h>

#include "common.h"

namespace {

struct beam_args {
    const void* logits;
    int64_t stride;
    const float* scores;
    const uint8_t* finished;
    const int32_t *hist, *step;
    float* out_score;
    int32_t *out_parent, *out_token, *hist_out;
    uint32_t* flags;
    // candidates of each beam in their order: [B*K][k] scores, logits and tokens (-1: no candidate)
    double* score;
    float* logit;
    int32_t* token;
    int eos, K, V, k, hist_cap, dtype;
};

__device__ __forceinline__ float load_logit(const beam_args& a, int64_t at) {
    float x;
    if (a.dtype == SWARM_FP32) x = static_cast<const float*>(a.logits)[at];
    else if (a.dtype == SWARM_BF16) x = __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.logits)[at] << 16);
    else x = (float)static_cast<const _Float16*>(a.logits)[at];
    return x != x ? -INFINITY : x;
}

// Workgroup r: beam r's normaliser and its k best tokens, one round each.
__global__ __launch_bounds__(256) void beam_row_kernel(beam_args a) {
    __shared__ float best[256];
    __shared__ int where[256];
    __shared__ double sums[256];
    const int64_t r = blockIdx.x, row = r * a.stride;
    const int t = threadIdx.x;
    if (a.finished && a.finished[r]) {
        for (int i = t; i < a.k; i += 256) a.token[r * a.k + i] = i == 0 ? a.eos : -1;
        if (t == 0) a.score[r * a.k] = a.scores[r] != a.scores[r] ? -INFINITY : a.scores[r], a.logit[r * a.k] = 0.f;
        return;
    }
    float after = INFINITY;
    int last = -1;
    double norm = 0.0;
    for (int i = 0; i < a.k; ++i) {
        float x = -INFINITY;
        int at = -1;
        for (int j = t; j < a.V; j += 256) {
            const float y = load_logit(a, row + j);
            const bool later = i == 0 || y < after || (y == after && j > last);
            if (later && (at < 0 || y > x)) x = y, at = j;
        }
        best[t] = x;
        where[t] = at;
        __syncthreads();
        for (int o = 128; o; o >>= 1) {
            if (t < o) {
                const float y = best[t + o];
                const int j = where[t + o];
                if (j >= 0 && (where[t] < 0 || y > best[t] || (y == best[t] && j < where[t]))) best[t] = y, where[t] = j;
            }
            __syncthreads();
        }
        after = best[0];
        last = where[0];
        __syncthreads();
        if (i == 0) {
            double s = 0.0;
            for (int j = t; j < a.V; j += 256) s += exp((double)load_logit(a, row + j) - after);
            sums[t] = s;
            __syncthreads();
            for (int o = 128; o; o >>= 1) {
                if (t < o) sums[t] += sums[t + o];
                __syncthreads();
            }
            norm = after + log(sums[0]);
        }
        if (t == 0) {
            const double s = a.scores[r] + ((double)after - norm);
            a.token[r * a.k + i] = last;
            a.logit[r * a.k + i] = after;
            a.score[r * a.k + i] = s != s ? -INFINITY : s;
        }
        if (last < 0) {
            for (int j = i + t; j < a.k; j += 256) a.token[r * a.k + j] = -1;
            break;
        }
    }
}

// Workgroup b: the k best of its beams' candidates, which each stand in their order, and the histories.
__global__ __launch_bounds__(64) void beam_join_kernel(beam_args a) {
    __shared__ int head[64];
    const int64_t b = blockIdx.x;
    const int t = threadIdx.x;
    int step = a.step ? a.step[0] : 0;
    if (a.step && (step < 0 || step >= a.hist_cap)) {
        if (t == 0) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
        step = step < 0 ? 0 : a.hist_cap;
    }
    if (t < a.K) head[t] = 0;
    __syncthreads();
    for (int i = 0; i < a.k; ++i) {
        int beam = -1;
        double top = 0.0;
        for (int j = 0; j < a.K; ++j) {
            const int64_t at = (b * a.K + j) * a.k + head[j];
            if (head[j] >= a.k || a.token[at] < 0) continue;
            if (beam < 0 || a.score[at] > top) beam = j, top = a.score[at];
        }
        const int token = beam < 0 ? -1 : a.token[(b * a.K + beam) * a.k + head[beam]];
        const int64_t out = b * a.k + i, parent = beam < 0 ? -1 : b * a.K + beam;
        __syncthreads();
        if (t == 0) {
            a.out_score[out] = beam < 0 ? -INFINITY : (float)top;
            a.out_parent[out] = (int)parent;
            a.out_token[out] = token;
            if (beam >= 0) ++head[beam];
        }
        if (a.hist && parent >= 0) {
            for (int j = t; j < step; j += 64) a.hist_out[out * a.hist_cap + j] = a.hist[parent * a.hist_cap + j];
            if (t == 0 && a.step[0] == step) a.hist_out[out * a.hist_cap + step] = token;
        }
        __syncthreads();
    }
}

}  // namespace

extern "C" swarm_status swarm_beam_select(swarm_ctx* ctx, const void* logits, int32_t dtype, int64_t stride, const float* scores,
                                          const uint8_t* finished, int32_t eos, int32_t B, int32_t K, int32_t V, int32_t k,
                                          float* out_score, int32_t* out_parent, int32_t* out_token, const int32_t* hist,
                                          const int32_t* step, int32_t hist_cap, int32_t* hist_out) {
    SWARM_ENTER(ctx);
    if (!logits || !scores || !out_score || !out_parent || !out_token) SWARM_REJECT(ctx, "beam_select: NULL required pointer");
    if (dtype != SWARM_BF16 && dtype != SWARM_FP16 && dtype != SWARM_FP32) SWARM_REJECT(ctx, "beam_select: unknown type %d", dtype);
    if (B < 1 || K < 1 || K > 64 || V < 1 || V > (1 << 24) || k < 1 || k > 128 || (int64_t)B * K > (1 << 20))
        SWARM_REJECT(ctx, "beam_select: B=%d K=%d V=%d k=%d out of range", B, K, V, k);
    if (stride < V || stride > ((int64_t)1 << 40)) SWARM_REJECT(ctx, "beam_select: stride=%lld below V=%d", (long long)stride, V);
    if (finished && (eos < 0 || eos >= V)) SWARM_REJECT(ctx, "beam_select: eos=%d outside [0,V=%d)", eos, V);
    if ((hist == nullptr) != (hist_out == nullptr) || (hist == nullptr) != (step == nullptr)) SWARM_REJECT(ctx, "beam_select: hist, step and hist_out go together");
    if (hist && (hist_cap < 1 || hist_cap > (1 << 28))) SWARM_REJECT(ctx, "beam_select: hist_cap=%d outside [1,2^28]", hist_cap);
    const uintptr_t size = dtype == SWARM_FP32 ? 4 : 2;
    if (swarm_misaligned(logits, size) || swarm_misaligned(scores, 4) || swarm_misaligned(out_score, 4) || swarm_misaligned(out_parent, 4) ||
        swarm_misaligned(out_token, 4) || swarm_misaligned(hist, 4) || swarm_misaligned(step, 4) || swarm_misaligned(hist_out, 4))
        SWARM_REJECT(ctx, "beam_select: misaligned pointer");
    const size_t rows = (size_t)B * K, found = (size_t)B * k;
    const swarm_range ins[] = {{logits, size * ((rows - 1) * (size_t)stride + V)}, {scores, 4 * rows}, {finished, rows}, {hist, 4 * rows * hist_cap}, {step, 4}};
    const swarm_range outs[] = {{out_score, 4 * found}, {out_parent, 4 * found}, {out_token, 4 * found}, {hist_out, 4 * found * hist_cap}};
    if (swarm_overlap(outs, 4, ins, 5)) SWARM_REJECT(ctx, "beam_select: an output overlaps an input, or another output");

    const swarm_status st = swarm_scratch(ctx, &ctx->beams, &ctx->beams_bytes, rows * k * 16);
    if (st != SWARM_OK) return st;
    beam_args a{};
    a.logits = logits, a.stride = stride, a.scores = scores, a.finished = finished;
    a.hist = hist, a.step = step, a.hist_out = hist_out;
    a.out_score = out_score, a.out_parent = out_parent, a.out_token = out_token;
    a.flags = ctx->dev_flags;
    a.score = static_cast<double*>(ctx->beams);
    a.logit = reinterpret_cast<float*>(a.score + rows * k);
    a.token = reinterpret_cast<int32_t*>(a.logit + rows * k);
    a.eos = eos, a.K = K, a.V = V, a.k = k, a.hist_cap = hist_cap, a.dtype = dtype;
    hipLaunchKernelGGL(beam_row_kernel, dim3((unsigned)rows), dim3(256), 0, ctx->stream, a);
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)B), dim3(64), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "beam_select");
}
