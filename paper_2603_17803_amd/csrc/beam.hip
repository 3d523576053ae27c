// Beam search's selection over beams and vocabulary.
//
// One pass over the logits.  A beam's best k tokens and its normaliser ln sum exp x come from one read: a workgroup takes a slice of a
// row in chunks of 4096 logits, holds a lower bound of the slice's k-th best logit, and puts the few that exceed it into a list in LDS, which is
// cut down to its k best whenever it has grown.  The first bound is the k-th largest of the first chunk's maxima of 64 groups of threads (of 256 threads for
// k above 32).  A logit costs its exponential, one comparison and one addition.  What bounds it is memory for fp32 (512 rows of 128000, k = 1: 52 us
// with the second kernel, 5.0 TB/s), and with 16-bit logits the candidates: without the few that each chunk adds after the first, and the waits of
// the other waves for the one that adds them, k = 16 takes 42 us in place of 54; the exponentials cost one.
//
// A second kernel, a workgroup for each group of beams, merges the sorted lists and moves the histories.
#include <math.h>

#include <type_traits>

#include "common.h"
#include "wave_ops.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef unsigned long long u64;

constexpr int CHUNK = 4096, EACH = 16;           // logits of a workgroup's step, and of a thread's
constexpr int TRIM = 512;                        // candidates from which a list is cut down, at most
constexpr int MOST_LISTS = 64 * 64, STAGED = 4096;   // lists of a group; candidates of a group that its merge holds in LDS

struct beam_args {
    const void* logits;
    int64_t stride;
    const float* scores;
    const uint8_t* finished;
    const int32_t *hist, *step;
    float* out_score;
    int32_t *out_parent, *out_token, *hist_out;
    uint32_t* flags;
    // of each slice of each beam: reference and sum of exponentials, candidates in their order (logit, token), how many
    double* sums;                                // [rows][J]
    double* refs;                                // [rows][J], in units of ln 2
    int32_t* found;                              // [rows][J]
    u64* lists;                                  // [rows][J][k]
    int eos, K, V, k, hist_cap, J, per, trim, halving;    // per: vectors of 16 bytes of a slice; trim: candidates from which a list is cut down
};

// Logits in their order as unsigned integers; 0 is below all of them.
__device__ __forceinline__ uint32_t ordered(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);               // -0 is 0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(u64 key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u);
}
// A candidate: the better logit is the larger number, and of equal ones the lower token.
__device__ __forceinline__ u64 candidate(float x, int token) { return (u64)ordered(x) << 32 | (uint32_t)~token; }
__device__ __forceinline__ int token_of(u64 key) { return (int)~(uint32_t)key; }

// The next float below a number above -inf.
__device__ __forceinline__ float below(float x) {
    const uint32_t u = __float_as_uint(x + 0.f);
    return __uint_as_float(u == 0 ? 0x80000001u : u >> 31 ? u + 1 : u - 1);
}

template <int TYPE>
__device__ __forceinline__ float widen(uint32_t bits) {
    float x;
    if (TYPE == SWARM_FP32) x = __uint_as_float(bits);
    else if (TYPE == SWARM_BF16) x = __uint_as_float(bits << 16);
    else x = (float)__builtin_bit_cast(_Float16, (uint16_t)bits);
    return x;
}

// How many of n keys in LDS are above `key`; n is rounded up to a multiple of 2 by zeros.
__device__ __forceinline__ int above(const u64* keys, int n, u64 key) {
    int c = 0;
#pragma unroll 8
    for (int i = 0; i < n; i += 2) {
        const ulonglong2 x = *reinterpret_cast<const ulonglong2*>(keys + i);
        c += x.x > key;
        c += x.y > key;
    }
    return c;
}

// Cuts a list in LDS of n different keys down to its k best (at most 128), in order, by a workgroup of 256; `best` has room for 258.
// Returns how many are left.
__device__ int trim(u64* list, int n, int k, u64* best, int* count) {
    const int t = threadIdx.x;
    if (n > 256) {
        // only keys from the k-th of the threads' maxima on can be among the k best
        u64 mine = 0;
        for (int i = t; i < n; i += 256) mine = list[i] > mine ? list[i] : mine;
        best[t] = mine;
        if (t == 0) *count = 0;
        __syncthreads();
        const int rank = above(best, 256, mine);
        __syncthreads();
        if (rank == k - 1) best[256] = mine;
        __syncthreads();
        const u64 bound = best[256];
        // in place: what a thread reads before the barrier is written behind it
        for (int base = 0; base < n; base += 256) {
            const u64 x = base + t < n ? list[base + t] : 0;
            __syncthreads();
            if (x >= bound) list[atomicAdd(count, 1)] = x;
        }
        __syncthreads();
        n = *count;
        __syncthreads();
    }
    if (t == 0) list[n] = 0;
    __syncthreads();
    const int left = n < k ? n : k;
    for (int i = t; i < n; i += 256) {
        const u64 x = list[i];
        const int rank = above(list, n, x);
        if (rank < k) best[rank] = x;
    }
    __syncthreads();
    if (t < left) list[t] = best[t];
    if (t == 0) *count = left;
    __syncthreads();
    return left;
}

// Workgroup (beam, slice).
template <int TYPE>
__global__ __launch_bounds__(256) void beam_slice_kernel(beam_args a) {
    constexpr int E = TYPE == SWARM_FP32 ? 4 : 8, VECS = EACH / E, STEP = CHUNK / E;   // logits of a vector; vectors of a thread's step and of a chunk
    typedef typename std::conditional<TYPE == SWARM_FP32, uint32_t, uint16_t>::type word;
    __shared__ __align__(16) u64 list[TRIM + CHUNK + 2], best[258];
    __shared__ int count;
    __shared__ double sum[4];
    __shared__ float ref[4], low[4];
    const int64_t r = blockIdx.x / a.J;
    const int j = blockIdx.x % a.J, t = threadIdx.x, lane = t % 64;
    const int64_t at = r * a.J + j;
    if (a.finished && a.finished[r]) {
        if (t == 0) a.found[at] = j == 0 ? -1 : 0;                      // its one candidate is the second kernel's
        return;
    }
    const word* row = static_cast<const word*>(a.logits) + r * a.stride;
    const int skew = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(word));      // the row's first logit in its vector
    const word* base = row - skew;
    const int from = j * a.per, upto = min(from + a.per, (skew + a.V + E - 1) / E);
    // whether all vectors of a chunk are the slice's, and whole in the row
    auto whole = [&](int chunk) { return chunk + STEP <= upto && chunk * (int64_t)E >= skew && (chunk + STEP) * (int64_t)E <= skew + (int64_t)a.V; };
    auto load = [&](v4i (&v)[VECS], int chunk) {
        if (chunk >= upto) return;
        if (whole(chunk)) {
            const v4i* p = reinterpret_cast<const v4i*>(base) + chunk + t;
#pragma unroll
            for (int i = 0; i < VECS; ++i) v[i] = __builtin_nontemporal_load(p + i * 256);
            return;
        }
        // the row's own logits alone of the vectors that it begins and ends in
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            const int64_t e = (int64_t)(chunk + i * 256 + t) * E;
            uint32_t w[4] = {0, 0, 0, 0};
            if (chunk + i * 256 + t < upto) {
                if (e >= skew && e + E <= skew + a.V) {
                    const v4i x = *reinterpret_cast<const v4i*>(base + e);
                    for (int q = 0; q < 4; ++q) w[q] = (uint32_t)x[q];
                } else {
#pragma unroll
                    for (int x = 0; x < E; ++x)
                        if (e + x >= skew && e + x < skew + a.V) w[x * sizeof(word) / 4] |= (uint32_t)base[e + x] << (x * sizeof(word) % 4 * 8);
                }
            }
            v[i] = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
        }
    };
    auto raw = [&](const v4i (&v)[VECS], int i, int e) {
        const uint32_t w = (uint32_t)v[i][e * (int)sizeof(word) / 4];
        if (TYPE == SWARM_BF16 && e & 1) return __uint_as_float(w & 0xffff0000u);
        return widen<TYPE>(TYPE == SWARM_FP32 ? w : e & 1 ? w >> 16 : w & 0xffffu);
    };
    auto token = [&](int chunk, int i, int e) { return (chunk + i * 256 + t) * E + e - skew; };
    auto there = [&](int chunk, int i, int e) {
        const int tok = token(chunk, i, e);
        return chunk + i * 256 + t < upto && tok >= 0 && tok < a.V;
    };

    v4i even[VECS], odd[VECS];                   // the chunks of even and odd number: one on its way while the other is worked on
    load(even, from);
    load(odd, from + STEP);
    // The first bound: the k-th largest of the maxima of 64 groups of four threads, or for many candidates of 256 threads.  At least k logits of the
    // first chunk are not below it; 16 of 64 maxima leave hardly more of them than 16 of 256 do.
    float mine = -INFINITY;
#pragma unroll
    for (int i = 0; i < VECS; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) mine = fmaxf(mine, there(from, i, e) ? raw(even, i, e) : -INFINITY);
    const int groups = a.k <= 32 ? 64 : 256;
    if (groups == 64) {
        mine = fmaxf(mine, waveops::dpp_f<0xB1>(mine));        // quad_perm [1,0,3,2]
        mine = fmaxf(mine, waveops::dpp_f<0x4E>(mine));        // quad_perm [2,3,0,1]
    }
    const int group = groups == 64 ? t / 4 : t;
    const u64 key = candidate(mine, group);                     // of equal maxima one is the larger
    best[group] = key;
    if (t == 0) count = 0;
    __syncthreads();
    if (t < groups) {
        const u64 own = best[t];
        const int rank = above(best, groups, own);
        if (rank == a.k - 1) best[256] = own;
        if (rank == 0) best[257] = own;
    }
    __syncthreads();
    const float bound = logit_of(best[256]), high = logit_of(best[257]);
    // Logits have to be above `floor`: in the first chunk not below the bound (where that is -inf, all are taken), later above it, as equal ones lose to
    // the lower tokens.
    bool every = bound == -INFINITY;
    float floor = every ? -INFINITY : below(bound);
    // Exponentials refer to the first chunk's largest logit, as 2^(x log2 e - at); a thread that meets a logit more than 8 octaves above it, candidate or
    // not, refers to that one from then on, so that no exponential overflows or has an argument that rounds far off.  Where the first chunk has no finite
    // logit, a thread's first one is its reference.  `at` is rounded, and stands for the logit at / log2 e exactly.  log2 e is taken in two parts, as what fp32 leaves out of it (2^-26 of
    // it) grows with the logits and not with their differences: logits of 300 would be off by 4e-6 all the same way.
    constexpr float LOG2E = 1.44269504088896341f, LOG2E_REST = (float)(1.4426950408889634074 - (double)LOG2E);
    constexpr float ABOVE = 5.5f;                // just below 8 octaves
    float at2 = high == -INFINITY ? -3.4e38f : high * LOG2E;
    float edge = high + ABOVE;                   // from which logit on the reference is raised; -inf: there is none yet
    float gate = fminf(floor, edge);
    double total = 0.0;
    auto weight = [&](float x, float to) { return __builtin_amdgcn_exp2f(__builtin_fmaf(x, LOG2E_REST, __builtin_fmaf(x, LOG2E, -to))); };
    auto take = [&](const v4i (&v)[VECS], int chunk) {
        if (chunk > from) {
            __syncthreads();
            const int n = count;
            __syncthreads();
            every = false;
            floor = fmaxf(floor, bound);
            if (n >= a.trim) {
                trim(list, n, a.k, best, &count);
                floor = logit_of(list[a.k - 1]);
            }
            gate = fminf(floor, edge);
        }
        const bool plain = whole(chunk);
#pragma unroll
        for (int i = 0; i < VECS; ++i) {
            float part = 0.f, top = -INFINITY, x[E];
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = raw(v, i, e);
            if (!plain) {
#pragma unroll
                for (int e = 0; e < E; ++e) x[e] = there(chunk, i, e) ? x[e] : -INFINITY;
            }
#pragma unroll
            for (int e = 0; e < E; e += 2) top = fmaxf(fmaxf(top, x[e]), x[e + 1]);
            if (top > gate || every) {
                if (top > edge) {
                    total *= exp2((double)at2 - (double)(top * LOG2E));
                    at2 = top * LOG2E;
                    edge = top + ABOVE;
                    gate = fminf(floor, edge);
                }
                uint32_t m = 0;
#pragma unroll
                for (int e = 0; e < E; ++e) m |= x[e] > floor || (every && there(chunk, i, e)) ? 1u << e : 0u;
                while (m) {
                    const int e = __ffs((int)m) - 1;
                    m &= m - 1;
                    float y = x[0];
#pragma unroll
                    for (int q = 1; q < E; ++q) y = e == q ? x[q] : y;
                    list[atomicAdd(&count, 1)] = candidate(fmaxf(y, -INFINITY), token(chunk, i, e));
                }
            }
#pragma unroll
            for (int e = 0; e < E; ++e) part += weight(x[e], at2);
            total += part;
        }
    };
    for (int chunk = from; chunk < upto; chunk += 2 * STEP) {
        take(even, chunk);
        load(even, chunk + 2 * STEP);
        if (chunk + STEP >= upto) break;
        take(odd, chunk + STEP);
        load(odd, chunk + 3 * STEP);
    }
    __syncthreads();
    const int pushed = count;
    __syncthreads();
    const int n = trim(list, pushed, a.k, best, &count);
    for (int i = t; i < n; i += 256) a.lists[at * a.k + i] = list[i];
    double big;
    const bool met = edge > -INFINITY;           // a finite logit, or one in the workgroup's first chunk
    if (__syncthreads_or(!(total < INFINITY) || (met && !(fabsf(at2) < 1e5f)))) {
        // A logit that is no number or infinite, or logits so large that 2^(x log2 e - at) says nothing: the sum again, in 64 bits, referred to the
        // best candidate.  (A candidate of +inf leaves no number, as the definition does.)
        const double best_logit = n ? logit_of(list[0]) : -INFINITY;
        total = 0.0;
        for (int chunk = from; chunk < upto; chunk += STEP) {
            load(even, chunk);
#pragma unroll
            for (int i = 0; i < VECS; ++i)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    const float x = there(chunk, i, e) ? fmaxf(raw(even, i, e), -INFINITY) : -INFINITY;
                    if (x > -INFINITY) total += exp((double)x - best_logit);
                }
        }
        big = best_logit * 1.4426950408889634074;
    } else {
        // The threads' sums at one reference.  Added in 64 bits, they are off by the rounding of the largest exponentials above all: those of the list
        // are taken again in 64 bits in place of the 32 (unless references differ, where 1e-7 is what the logarithm is good to).
        float high2 = at2, small = met ? at2 : 3.4e38f;
        for (int o = 32; o; o >>= 1) high2 = fmaxf(high2, __shfl_xor(high2, o)), small = fminf(small, __shfl_xor(small, o));
        if (lane == 0) ref[t / 64] = high2, low[t / 64] = small;
        __syncthreads();
        high2 = fmaxf(fmaxf(ref[0], ref[1]), fmaxf(ref[2], ref[3]));
        small = fminf(fminf(low[0], low[1]), fminf(low[2], low[3]));
        if (at2 != high2) total *= exp2((double)at2 - (double)high2);
        if (small == high2 && t < n) {
            const float x = logit_of(list[t]);
            if (x > -INFINITY) total += exp2((double)x * 1.4426950408889634074 - (double)high2) - weight(x, high2);
        }
        big = high2;
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    if (lane == 0) sum[t / 64] = total;
    __syncthreads();
    if (t == 0) {
        const double all = sum[0] + sum[1] + sum[2] + sum[3];
        a.sums[at] = all;
        a.refs[at] = all == 0.0 ? (double)-INFINITY : big;      // a slice without a finite logit refers to nothing
        a.found[at] = n;
    }
}

__device__ __forceinline__ u64 ordered(double x) {
    const u64 u = (u64)__double_as_longlong(x + 0.0);
    return u >> 63 ? ~u : u | (u64)1 << 63;
}
__device__ __forceinline__ double score_of(u64 key) { return __longlong_as_double((long long)(key >> 63 ? key & ~((u64)1 << 63) : ~key)); }

// Workgroup b.  Few lists are merged by all threads at once; otherwise its first wave merges: a lane has every 64th of the K * J lists and the best candidate among them, and each round takes
// the best lane's.  Then all move the histories.
__global__ __launch_bounds__(1024) void beam_join_kernel(beam_args a) {
    __shared__ double norm[64];                  // ln sum exp of each beam's logits; of a finished one nothing
    __shared__ float base[64];
    __shared__ uint8_t head[MOST_LISTS], length[MOST_LISTS], beams[MOST_LISTS];   // where each list stands, its candidates (255: the one of a finished beam), its beam
    __shared__ u64 staged[STAGED], scored[STAGED];   // candidates, and their scores
    __shared__ int parent[128], token[128], places[STAGED];
    __shared__ float best[128];
    const int64_t b = blockIdx.x;
    const int t = threadIdx.x, lists = a.K * a.J, n_staged = lists * a.k <= STAGED ? lists * a.k : 0;
    for (int i = t; i < lists; i += 1024) head[i] = 0, length[i] = (uint8_t)a.found[b * lists + i], beams[i] = (uint8_t)(i / a.J);
    for (int i = t; i < n_staged; i += 1024) staged[i] = a.lists[b * lists * a.k + i];
    int step = a.hist ? a.step[0] : 0;
    {
        // 16 lanes a beam, four of its up to 64 slices each
        const int beam = t / 16, lane = t % 16;
        const int64_t at = (b * a.K + beam) * a.J;
        double ref[4], sum[4], big = -INFINITY, z = 0.0;
        const bool live = beam < a.K && a.found[at] >= 0;
        for (int i = 0; i < 4; ++i) {
            const bool there = live && lane + 16 * i < a.J;
            ref[i] = there ? a.refs[at + lane + 16 * i] : -INFINITY;
            sum[i] = there ? a.sums[at + lane + 16 * i] : 0.0;
            big = fmax(big, ref[i]);
        }
        for (int o = 8; o; o >>= 1) big = fmax(big, __shfl_xor(big, o, 16));
        for (int i = 0; i < 4; ++i)
            if (lane + 16 * i < a.J) z += sum[i] * exp2(ref[i] - big);
        for (int o = 8; o; o >>= 1) z += __shfl_xor(z, o, 16);
        if (beam < a.K && lane == 0) {
            base[beam] = a.scores[b * a.K + beam];
            norm[beam] = big * 0.69314718055994530942 + log(z);
        }
    }
    __syncthreads();
    auto score_of_key = [&](int beam, u64 c, bool finished) {
        double x = base[beam];
        if (!finished) x += (double)logit_of(c) - norm[beam];
        return ordered(x != x ? (double)-INFINITY : x);
    };
    for (int i = t; i < n_staged; i += 1024) {
        const int list = i / a.k;
        const bool finished = length[list] == 255;
        if (finished && i == list * a.k) staged[i] = candidate(0.f, a.eos);
        if (i - list * a.k < (finished ? 1 : length[list])) scored[i] = score_of_key(beams[list], staged[i], finished);
    }
    const bool searched = n_staged && a.k >= 4 && lists <= 16;
    if (searched) {
        for (int i = t; i < n_staged; i += 1024) places[i] = i % a.k;
        if (t < a.k) parent[t] = -1, token[t] = -1, best[t] = -INFINITY;
    }
    __syncthreads();
    if (searched) {
        // A candidate's place is how many stand above it: in each list the first few, found by halving.  The lists are divided over as many threads
        // as there are for a candidate.  Its work grows with the square of the lists, that of the rounds below with k.  The whole call, 64 groups, 32000
        // bf16 logits, k = 4, 16, 32, 64: 16 lists 30.0, 36.4, 45.2, 64.3 us by rounds and 29.6, 35.1, 42.9, 61.1 so; 18 lists 41.0, 50.1, 60.1, 82.0 and 40.8,
        // 50.4, 66.1, 92.4; 24 lists 44.9, 54.0, 63.8, 86.9 and 45.3, 58.1, 74.8, 110.
        const int shares = max(1, 1024 / n_staged);
        for (int x = t; x < n_staged * shares; x += 1024) {
            const int share = x / n_staged, i = x - share * n_staged, list = i / a.k, beam = beams[list];
            if (i - list * a.k >= (length[list] == 255 ? 1 : length[list])) continue;
            const u64 score = scored[i], key = staged[i];
            int above = 0;
            for (int l = share; l < lists; l += shares) {
                const int n = l == list ? 0 : length[l] == 255 ? 1 : length[l], other = beams[l], from = l * a.k;
                int first = 0;
                for (int step = a.halving; step; step >>= 1) {
                    const int at = first + step - 1;
                    if (at < n) {
                        const u64 s = scored[from + at];
                        first += s > score || (s == score && (other < beam || (other == beam && staged[from + at] > key))) ? step : 0;
                    }
                }
                above += first;
            }
            if (above) atomicAdd(&places[i], above);
        }
        __syncthreads();
        for (int i = t; i < n_staged; i += 1024) {
            const int list = i / a.k, place = places[i];
            if (i - list * a.k < (length[list] == 255 ? 1 : length[list]) && place < a.k) {
                parent[place] = (int)(b * a.K) + beams[list];
                token[place] = token_of(staged[i]);
                best[place] = (float)score_of(scored[i]);
            }
        }
    } else if (t < 64) {
        // The lane's best candidate (score 0: none), its beam and its list; where it has one list alone, the candidate behind it too.
        u64 score = 0, key = 0, behind = 0, behind_score = 0;
        int owner = 0, mine = t, at = 0, n = 0;
        const bool single = lists <= 64;
        auto key_of = [&](int list, int place) { return n_staged ? staged[list * a.k + place] : a.lists[(b * lists + list) * a.k + place]; };
        auto score_at = [&](int list, int place, int beam, u64 c) { return n_staged ? scored[list * a.k + place] : score_of_key(beam, c, false); };
        auto refresh = [&]() {
            score = 0;
            for (int i = t; i < lists; i += 64) {
                const int beam = beams[i], count = length[i], place = head[i];
                const bool finished = count == 255;
                if (place >= (finished ? 1 : count)) continue;
                const u64 c = finished ? candidate(0.f, a.eos) : key_of(i, place), s = finished ? score_of_key(beam, c, true) : score_at(i, place, beam, c);
                // lists come in the order of beams, a beam's in the order of its slices
                if (s > score || (s == score && beam == owner && c > key)) score = s, key = c, mine = i, owner = beam;
            }
        };
        refresh();
        if (single && t < lists) {
            n = length[t] == 255 ? 1 : length[t];
            if (n > 1) behind = key_of(t, 1), behind_score = score_at(t, 1, owner, behind);
        }
        for (int i = 0; i < a.k; ++i) {
            // the largest score, then the lowest beam, the largest logit, the lowest token
            const uint32_t hi = waveops::wave_min_u32(~(uint32_t)(score >> 32));
            bool in = ~(uint32_t)(score >> 32) == hi;
            u64 who = __ballot(in);
            if (who & (who - 1)) {
                const uint32_t lo = waveops::wave_min_u32(in ? ~(uint32_t)score : ~0u);
                in = in && ~(uint32_t)score == lo;
                who = __ballot(in);
            }
            if (hi == ~0u) {
                if (t == 0) parent[i] = -1, token[i] = -1, best[i] = -INFINITY;
                continue;
            }
            if (who & (who - 1)) {
                const uint32_t beam = waveops::wave_min_u32(in ? (uint32_t)owner : ~0u);
                in = in && (uint32_t)owner == beam;
                const uint32_t x = waveops::wave_min_u32(in ? ~(uint32_t)(key >> 32) : ~0u);
                in = in && ~(uint32_t)(key >> 32) == x;
                const uint32_t y = waveops::wave_min_u32(in ? ~(uint32_t)key : ~0u);
                in = in && ~(uint32_t)key == y;
                who = __ballot(in);
            }
            if (t == __ffsll((long long)who) - 1) {
                parent[i] = (int)(b * a.K) + owner;
                token[i] = token_of(key);
                best[i] = (float)score_of(score);
                if (single) {
                    ++at;
                    key = behind;
                    score = at < n ? behind_score : 0;
                    if (at + 1 < n) behind = key_of(t, at + 1), behind_score = score_at(t, at + 1, owner, behind);
                } else {
                    ++head[mine];
                    refresh();
                }
            }
        }
    }
    __syncthreads();
    for (int i = t; i < a.k; i += 1024) a.out_parent[b * a.k + i] = parent[i], a.out_token[b * a.k + i] = token[i], a.out_score[b * a.k + i] = best[i];
    if (!a.hist) return;
    const bool fits = step >= 0 && step < a.hist_cap;
    if (!fits) {
        if (t == 0) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
        step = step < 0 ? 0 : a.hist_cap;
    }
    // a wave a history, several loads on their way at a time; in 16 bytes where histories and rows allow it
    const bool wide = ((reinterpret_cast<uintptr_t>(a.hist) | reinterpret_cast<uintptr_t>(a.hist_out)) & 15) == 0 && a.hist_cap % 4 == 0;
    const int lane = t % 64;
    for (int i = t / 64; i < a.k; i += 16) {
        if (parent[i] < 0) continue;
        const int32_t* from = a.hist + (int64_t)parent[i] * a.hist_cap;
        int32_t* to = a.hist_out + (b * a.k + i) * a.hist_cap;
        int x = 0;
        if (wide) {
            for (; x + 4 <= step; x += 4096) {
                v4i v[16];
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    if (x + q * 256 + lane * 4 + 4 <= step) v[q] = *reinterpret_cast<const v4i*>(from + x + q * 256 + lane * 4);
#pragma unroll
                for (int q = 0; q < 16; ++q)
                    if (x + q * 256 + lane * 4 + 4 <= step) *reinterpret_cast<v4i*>(to + x + q * 256 + lane * 4) = v[q];
            }
            x = step / 4 * 4;
        }
        for (; x < step; x += 1024) {
            int v[16];
#pragma unroll
            for (int q = 0; q < 16; ++q)
                if (x + q * 64 + lane < step) v[q] = from[x + q * 64 + lane];
#pragma unroll
            for (int q = 0; q < 16; ++q)
                if (x + q * 64 + lane < step) to[x + q * 64 + lane] = v[q];
        }
        if (fits && lane == 0) to[step] = token[i];
    }
}

template <int TYPE>
void launch_beams(const beam_args& a, int64_t rows, hipStream_t stream) {
    hipLaunchKernelGGL(beam_slice_kernel<TYPE>, dim3((unsigned)(rows * a.J)), dim3(256), 0, stream, a);
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

    // Slices of a row: enough workgroups for four on each compute unit, of at least one chunk each, at most 64.
    const int each = dtype == SWARM_FP32 ? 4 : 8;
    const int64_t vectors = ((int64_t)V + each - 1) / each + 1, most = (vectors * each + CHUNK - 1) / CHUNK;
    int64_t J = (1024 + (int64_t)rows - 1) / (int64_t)rows;
    J = J < most ? J : most;
    J = J < 64 ? J : 64;
    const size_t slices = rows + 1024;           // rows * J is below, and this grows with the rows: smaller calls never need more
    const swarm_status st = swarm_scratch(ctx, &ctx->beams, &ctx->beams_bytes, slices * (8 + 8 + 4 + 8 * (size_t)k));
    if (st != SWARM_OK) return st;
    beam_args a{};
    a.logits = logits, a.stride = stride, a.scores = scores, a.finished = finished;
    a.hist = hist, a.step = step, a.hist_out = hist_out;
    a.out_score = out_score, a.out_parent = out_parent, a.out_token = out_token;
    a.flags = ctx->dev_flags;
    a.sums = static_cast<double*>(ctx->beams);
    a.lists = reinterpret_cast<u64*>(a.sums + slices);
    a.refs = reinterpret_cast<double*>(a.lists + slices * k);
    a.found = reinterpret_cast<int32_t*>(a.refs + slices);
    a.eos = eos, a.K = K, a.V = V, a.k = k, a.hist_cap = hist_cap, a.J = (int)J, a.per = (int)((vectors + J - 1) / J);
    // Cutting a list costs barriers and gives a higher bound: 512 rows of 128001 bf16 logits, k = 16 (32): at 48 (96) candidates 54 us (66), at 64 (128) 55 (69).
    for (a.halving = 1; a.halving * 2 <= k;) a.halving *= 2;
    a.trim = 3 * k < 48 ? 48 : 3 * k;            // below 512
    if (dtype == SWARM_FP32) launch_beams<SWARM_FP32>(a, (int64_t)rows, ctx->stream);
    else if (dtype == SWARM_BF16) launch_beams<SWARM_BF16>(a, (int64_t)rows, ctx->stream);
    else launch_beams<SWARM_FP16>(a, (int64_t)rows, ctx->stream);
    hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)B), dim3(1024), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "beam_select");
}
