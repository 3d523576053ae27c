// Attention of drafted tokens over a paged cache.
//
// The T*G query rows that a KV head's group has (drafted token i, query head g: row i*G + g) share every key and value, so a
// workgroup takes up to 64 of them and streams the keys past: per 16 rows, S^T = K Q^T on the 16x16x32 matrix instruction (keys are
// the rows of its result, query rows its columns), the softmax's running maximum and sum a lane per query row, O^T += V^T P^T on the
// same instruction.  A lane's eight weights of 32 keys are, as they come out of the first product, one operand of the
// second; V^T's operand is read out of LDS by the transposing read.  K goes straight from memory into registers.
//
// Two kernels.  The first takes the contexts: the 128-key units of all (stream, head) pairs stand in one line, which is cut into equal parts, one
// for each workgroup, whatever the streams' lengths are.  The four waves of a workgroup each take 32 keys of a unit, all rows, and meet only
// where a pair ends: no barrier in the loop.  What a part finds for a pair stays in scratch (fp32, unnormalised).  The second takes
// 16 rows of a pair, works the drafted tokens in under their masks, joins the parts, divides and rounds once.
#include <math.h>

#include "common.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int UNIT = 128;                        // keys of a unit, 32 for each wave
constexpr int LISTED = 2048;                     // keys whose rows are looked up at a time

struct attend_args {
    const uint16_t *k, *v, *q, *k_new, *v_new;   // k, v: the layer's part of the pool
    const int32_t *table, *len, *n_new, *sel;
    const uint32_t* mask;
    uint16_t* out;
    float* lse;
    int32_t* starts;                             // [B + 1]: where each stream's units start in the line, and their number
    float* part_o;                               // [slots][rows of a tile][DP]: sums of weighted values
    float* part_ml;                              // [slots][rows of a tile][2]: maximum (in units of ln 2) and sum of weights
    uint32_t* flags;
    int P, H, page_log2, d, cap, B, T, G, n_sel, unit;
    int parts, tiles, rows;                      // parts of the line; tiles of a pair's rows, rows of a tile
    uint32_t per_g;                              // ceil(2^32 / G)
    float scale_log2;
};

template <bool BF16>
__device__ __forceinline__ v4f mfma(v4i x, v4i y, v4f c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, x), __builtin_bit_cast(bf8, y), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(hf8, x), __builtin_bit_cast(hf8, y), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ uint32_t bits_of(float x) {
    if constexpr (BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
}
template <bool BF16>
__device__ __forceinline__ float value_of(uint32_t x) {
    if constexpr (BF16) return __uint_as_float(x << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
}
template <bool BF16>
__device__ __forceinline__ int pack(float lo, float hi) { return (int)(bits_of<BF16>(lo) | bits_of<BF16>(hi) << 16); }

// Maximum and sum over the four lanes (l, l + 16, l + 32, l + 48) that share a query row.
__device__ __forceinline__ float rows_max(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float rows_sum(float x) {
    auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The same value in all lanes, said so: it stays in scalar registers and its branches are branches.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// What a stream brings: the tokens it holds, slots of its selection (or tokens), drafted tokens, units of a (head, tile).
struct stream {
    int len, slots, drafted, units;
};
__device__ __forceinline__ stream stream_of(const attend_args& a, int b, bool tell) {
    stream s;
    const int most = a.cap << a.page_log2;
    s.len = a.len[b];
    s.drafted = a.n_new ? a.n_new[b] : a.T;
    if (s.len < 0 || s.len > most || s.drafted < 0 || s.drafted > a.T) {
        if (tell) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        s.len = min(max(s.len, 0), most);
        s.drafted = min(max(s.drafted, 0), a.T);
    }
    s.slots = !a.sel ? s.len : a.unit == SWARM_SEL_PAGES ? a.n_sel << a.page_log2 : a.n_sel;
    s.units = s.drafted > 0 ? (s.slots + UNIT - 1) / UNIT : 0;
    return s;
}
__device__ __forceinline__ int token_of(const attend_args& a, int row) { return a.G == 1 ? row : (int)__umulhi((uint32_t)row, a.per_g); }

// Sum over the lower threads of a workgroup, and over all of them.
__device__ __forceinline__ int block_before(int v, int* waves, int* total) {
    int x = v;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = x;
    __syncthreads();
    int below = 0, sum = 0;
    for (int i = 0; i < (int)blockDim.x / 64; ++i) {
        below += i < w ? waves[i] : 0;
        sum += waves[i];
    }
    *total = sum;
    return below + x - v;
}
// Units of a part: part p takes units p * quota to (p + 1) * quota of the line, and unit g stands in part g / quota.
__device__ __forceinline__ int quota_of(const attend_args& a, int units) { return max(1, (units + a.parts - 1) / a.parts); }

// What a wave carries of NR * 16 query rows: lane l has row l % 16 of each 16, and of the sums of values the channels
// 16 c + 4 (l / 16) + 0..3.  KT keys are taken at a time.
//   TERMS: how many terms of the cache's type a weight enters its product with v as.  Two are a weight to 2^-16 and more,
//   and cost half as many products again.
template <bool BF16, int DP, int NR, int KT, int TERMS, bool FULL>
struct flash {
    static constexpr int KS = DP / 32, CT = DP / 16;
    static constexpr int VLD = DP + 16;          // LDS row of V in elements: 32 bytes behind each, so that 16 rows' reads meet no bank twice
    v4i qf[NR][KS], pf[NR][TERMS][KT / 32];
    v4f o[NR][CT], sc[NR][KT / 16];
    float m[NR], l[NR];

    __device__ __forceinline__ void start(const attend_args& a, int b, int h, int row0, int drafted) {
        const int col = threadIdx.x % 16, quad = threadIdx.x % 64 / 16;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const int r = row0 + n * 16 + col, i = token_of(a, r);
            const uint16_t* q = a.q + ((((int64_t)b * a.T + i) * a.H + h) * a.G + (r - i * a.G)) * a.d;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                const int c = k * 4 + quad;
                qf[n][k] = i < drafted && (FULL || c < a.d / 8) ? *reinterpret_cast<const v4i*>(q + c * 8) : v4i{0, 0, 0, 0};
            }
            m[n] = -INFINITY;
            l[n] = 0.f;
#pragma unroll
            for (int c = 0; c < CT; ++c) o[n][c] = v4f{0.f, 0.f, 0.f, 0.f};
        }
    }
    // q . k of KT keys whose rows stand in LDS.
    template <int KLD>
    __device__ __forceinline__ void scores(const uint16_t* ks) {
        const int col = threadIdx.x % 16, quad = threadIdx.x % 64 / 16;
#pragma unroll
        for (int k = 0; k < KT / 16; ++k) {
#pragma unroll
            for (int n = 0; n < NR; ++n) sc[n][k] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KS; ++c) {
                const v4i kf = *reinterpret_cast<const v4i*>(ks + (k * 16 + col) * KLD + c * 32 + quad * 8);
#pragma unroll
                for (int n = 0; n < NR; ++n) sc[n][k] = mfma<BF16>(kf, qf[n][c], sc[n][k]);
            }
        }
    }
    // V^T of 16 channels and 32 keys, as the operand of the second product: elements 0..3 and 4..7 of lane l are keys 4 (l / 16) + 0..3 and
    // 16 more.
    static __device__ __forceinline__ v4i get_v(const uint16_t* vs, int c) {
        const int col = threadIdx.x % 16, quad = threadIdx.x % 64 / 16;
        const uint16_t* from = vs + (quad * 4 + col / 4) * VLD + col % 4 * 4 + c * 16;
        const v2i x = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(from)));
        const v2i y = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(from + 16 * VLD)));
        return v4i{x[0], x[1], y[0], y[1]};
    }
    // The weights of KT keys; sees[j]: which of the keys 32 j to 32 j + 31 the lane's rows see.  The maximum that weights refer to is raised only
    // when one of the 16 rows has outgrown it by 2^8: a row's weights stay below that, which no sum here minds, and most
    // tiles rescale nothing.
    __device__ __forceinline__ void weigh(float scale_log2, const uint32_t* sees, bool all) {
        const int quad = threadIdx.x % 64 / 16;
        float mx[NR];
        bool grown = false;
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int e = 0; e < KT / 4; ++e) sc[n][e / 4][e % 4] *= scale_log2;
        if (!all) {
#pragma unroll
            for (int e = 0; e < KT / 4; ++e) {
                const bool seen = sees[e / 8] >> quad * 4 & 1u << (e / 4 % 2 * 16 + e % 4);
#pragma unroll
                for (int n = 0; n < NR; ++n) sc[n][e / 4][e % 4] = seen ? sc[n][e / 4][e % 4] : -INFINITY;
            }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            mx[n] = -INFINITY;
#pragma unroll
            for (int e = 0; e < KT / 16; ++e) mx[n] = fmaxf(fmaxf(fmaxf(mx[n], sc[n][e][0]), fmaxf(sc[n][e][1], sc[n][e][2])), sc[n][e][3]);
            mx[n] = rows_max(mx[n]);
            grown |= mx[n] > m[n] + 8.f;
        }
        if (__any(grown)) {
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const float next = fmaxf(m[n], mx[n]);
                rescale(n, m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - next));
                m[n] = next;
            }
        }
#pragma unroll
        for (int n = 0; n < NR; ++n) {
            const float base = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
            for (int j = 0; j < KT / 32; ++j) {
                float p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(sc[n][j * 2 + e / 4][e % 4] - base);
                    l[n] += p[e];
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pf[n][0][j][e] = pack<BF16>(p[2 * e], p[2 * e + 1]);
                    if constexpr (TERMS == 2)
                        pf[n][1][j][e] = pack<BF16>(p[2 * e] - value_of<BF16>((uint32_t)pf[n][0][j][e] & 0xffffu), p[2 * e + 1] - value_of<BF16>((uint32_t)pf[n][0][j][e] >> 16));
                }
            }
        }
    }
    __device__ __forceinline__ void rescale(int n, float f) {
        l[n] *= f;
#pragma unroll
        for (int c = 0; c < CT; ++c) o[n][c] *= f;
    }
    __device__ __forceinline__ void add(const uint16_t* vs) {
#pragma unroll
        for (int j = 0; j < KT / 32; ++j)
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const v4i vf = get_v(vs + j * 32 * VLD, c);
#pragma unroll
                for (int n = 0; n < NR; ++n)
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) o[n][c] = mfma<BF16>(vf, pf[n][k][j], o[n][c]);
            }
    }
};

// The same with the wave's own keys: K and V through registers into the wave's LDS, one after the other in the same place.  Whole rows
// come from memory at a time (as the operand of the first product K would come in 64 bytes of 16 rows).
template <bool BF16, int DP, int NR, int TERMS, bool FULL>
struct own_keys : flash<BF16, DP, NR, 32, TERMS, FULL> {
    typedef flash<BF16, DP, NR, 32, TERMS, FULL> base;
    static constexpr int VI = DP / 16, LPR = DP / 8, RPI = 64 / LPR;   // pieces of a lane, lanes on a row, rows at a time
    static constexpr int KLD = DP + 8, VLD = base::VLD;                // LDS rows in elements: 16 rows' pieces of 16 bytes meet no bank twice
    v4i kr[VI], vr[VI];
    // Pieces behind the head dimension read another one; on K's side they then count as 0.
    static __device__ __forceinline__ void load(v4i (&r)[VI], const v4i* from, const uint32_t* rows, int d) {
        const int lane = threadIdx.x % 64;
        from += FULL ? lane % LPR : min(lane % LPR, d / 8 - 1);
#pragma unroll
        for (int j = 0; j < VI; ++j) r[j] = __builtin_nontemporal_load(from + rows[j * RPI + lane / LPR]);
    }
    __device__ __forceinline__ void put_k(uint16_t* lds, int d) {
        const int lane = threadIdx.x % 64;
        uint16_t* to = lds + (lane / LPR) * KLD + lane % LPR * 8;
#pragma unroll
        for (int j = 0; j < VI; ++j) {
            if (!FULL) kr[j] &= (lane % LPR - d / 8) >> 31;
            *reinterpret_cast<v4i*>(to + j * RPI * KLD) = kr[j];
        }
    }
    // Rows of keys that are not there become 0.
    __device__ __forceinline__ void put_v(uint16_t* lds, uint32_t there) {
        const int lane = threadIdx.x % 64;
        if (there != ~0u) {
            const uint32_t held = there >> (lane / LPR);
#pragma unroll
            for (int j = 0; j < VI; ++j)
                if (!(held & 1u << (j * RPI))) vr[j] = v4i{0, 0, 0, 0};
        }
        uint16_t* to = lds + (lane / LPR) * VLD + lane % LPR * 8;
#pragma unroll
        for (int j = 0; j < VI; ++j) *reinterpret_cast<v4i*>(to + j * RPI * VLD) = vr[j];
    }
};

// Joins what the four waves of a workgroup carry of 16 rows, through LDS (16 rows of OLD floats for each wave): calls
// put(row, channel, sums of four channels, maximum, sum of weights) for each row and each four channels.
template <int DP, typename F, typename PUT>
__device__ __forceinline__ void join_waves(F& f, int n, float* os, float (*top)[16], float (*sum)[16], PUT&& put) {
    constexpr int OLD = DP + 4;
    const int t = threadIdx.x, col = t % 16, quad = t % 64 / 16, wave = t / 64;
    __syncthreads();
    const float l = rows_sum(f.l[n]);
    if (quad == 0) top[wave][col] = f.m[n], sum[wave][col] = l;
#pragma unroll
    for (int c = 0; c < DP / 16; ++c) *reinterpret_cast<v4f*>(os + (wave * 16 + col) * OLD + c * 16 + quad * 4) = f.o[n][c];
    __syncthreads();
    for (int x = t; x < 16 * (DP / 4); x += 256) {
        const int r = x / (DP / 4), c = x % (DP / 4) * 4;
        const float big = fmaxf(fmaxf(top[0][r], top[1][r]), fmaxf(top[2][r], top[3][r]));
        v4f y = {0.f, 0.f, 0.f, 0.f};
        float z = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float g = top[w][r] == -INFINITY ? 0.f * sum[w][r] : __builtin_amdgcn_exp2f(top[w][r] - big);   // a sum that is no number stays
            z += g * sum[w][r];
            if (g > 0.f || g != g) y += g * *reinterpret_cast<const v4f*>(os + (w * 16 + r) * OLD + c);
        }
        put(r, c, y, big, z);
    }
}

// Where a workgroup's part of the line starts and ends, and the stream and the unit within it that it starts at.  Thread 0 of workgroup 0 and
// its fellows leave the streams' places for the second kernel.
__device__ __forceinline__ bool place_part(const attend_args& a, int part, int* waves, int* where, int* at, int* end) {
    const int t = threadIdx.x, threads = blockDim.x;
    int quota = 0;
    for (int pass = a.B <= threads; pass < 2; ++pass) {
        int before = 0, all;
        for (int base = 0; base < a.B; base += threads) {
            const int i = base + t, n = i < a.B ? a.H * stream_of(a, i, blockIdx.x == 0).units : 0;
            const int start = before + block_before(n, waves, &all);
            before += all;
            if (pass == 0 || a.B <= threads) {
                const int units = uniform(before);
                quota = quota_of(a, units);
                *at = part * quota;
                *end = min(*at + quota, units);
            }
            if (pass) {
                if (start <= *at && *at < start + n) where[0] = i, where[1] = *at - start;
                if (blockIdx.x == 0 && i < a.B) a.starts[i] = start;
            }
        }
        if (blockIdx.x == 0 && t == 0) a.starts[a.B] = before;
    }
    __syncthreads();
    return *at < *end && part < a.parts;
}

// Looks up where the rows of keys from * UNIT .. (from + n) * UNIT of a pair start in its layer's pool, in pieces of 16 bytes, and which
// keys are there; one that is not reads row 0 and weighs nothing.
__device__ __forceinline__ void list_keys(const attend_args& a, const stream& s, int b, int h, int from, int n, uint32_t* listed, uint32_t* held) {
    const int lane = threadIdx.x % 64, inside = (1 << a.page_log2) - 1;
    __syncthreads();
    for (int x = threadIdx.x; x < n * UNIT; x += blockDim.x) {
        uint32_t row = 0;
        bool there = false;
        int pos = from * UNIT + x;
        if (pos < s.slots) {
            if (a.sel) {
                const bool by_page = a.unit == SWARM_SEL_PAGES;
                const int e = a.sel[((int64_t)b * a.H + h) * a.n_sel + (by_page ? pos >> a.page_log2 : pos)];
                pos = by_page ? e << a.page_log2 | (pos & inside) : e;
                if (e < 0 || e >= (by_page ? a.cap : a.cap << a.page_log2)) {
                    if (e != -1) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
                    pos = s.len;
                }
            }
            if (pos < s.len) {
                const int id = a.table[(int64_t)b * a.cap + (pos >> a.page_log2)];
                if (id < 0 || id >= a.P) atomicOr(a.flags, SWARM_DEV_BAD_PAGE);
                else there = true, row = (((uint32_t)id * a.H + h) << a.page_log2) + (pos & inside);
            }
        }
        listed[x] = row * (uint32_t)(a.d / 8);
        const uint64_t which = __ballot(there);
        if (lane % 32 == 0) held[x / 32] = (uint32_t)(which >> lane);
    }
    __syncthreads();
}

// Workgroup (part, tile of up to 32 rows): the part's keys, pair by pair, each wave 32 keys of a unit and all rows.
template <bool BF16, int DP, int NR, bool FULL>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attend_context_kernel(attend_args a) {
    constexpr int ROWS = 16 * NR;
    typedef own_keys<BF16, DP, NR, 2, FULL> state;
    __shared__ __align__(16) unsigned char pool[4 * 32 * state::VLD * 2];
    __shared__ uint32_t listed[LISTED], held[LISTED / 32];
    __shared__ float top[4][16], sum[4][16];
    __shared__ int waves[4], where[2];
    static_assert(4 * 16 * (DP + 4) * 4 <= sizeof(pool), "the waves' parts of the result fit their rows of V");

    const int wave = uniform(threadIdx.x / 64);
    // workgroups of the same part and different tiles read the same keys: 8 apart, they run behind the same L2
    const int tile = (int)(blockIdx.x / 8) % a.tiles, part = (int)(blockIdx.x / 8) / a.tiles * 8 + (int)(blockIdx.x % 8);
    int at, end;
    if (!place_part(a, part, waves, where, &at, &end)) return;
    int b = uniform(where[0]);
    const int offset = uniform(where[1]);
    stream s = stream_of(a, b, false);
    int h = offset / s.units, first = offset % s.units;
    uint16_t* vs = reinterpret_cast<uint16_t*>(pool) + wave * 32 * state::VLD;
    const uint32_t* mine = listed + wave * 32;
    const v4i *kp = reinterpret_cast<const v4i*>(a.k), *vp = reinterpret_cast<const v4i*>(a.v);
    state f;

    for (;;) {
        const int last = min(s.units, first + (end - at));
        const int rows = min(s.drafted * a.G - tile * ROWS, ROWS);   // query rows here
        if (rows > 0) {
            f.start(a, b, h, tile * ROWS, s.drafted);
            for (int u0 = first; u0 < last; u0 += LISTED / UNIT) {
                const int n = min(last - u0, LISTED / UNIT);
                list_keys(a, s, b, h, u0, n, listed, held);
                // K and V of the next tile are on their way while one is worked on: into registers as soon as LDS has taken the last one's
                f.load(f.kr, kp, mine, a.d);
                __builtin_amdgcn_sched_barrier(0);   // K's loads stay older than V's, as in the loop: whoever waits for K then need not wait for V
                f.load(f.vr, vp, mine, a.d);
                for (int u = 0; u < n; ++u) {
                    const uint32_t there = (uint32_t)uniform((int)held[u * 4 + wave]);
                    const int next = min(u + 1, n - 1) * UNIT;
                    f.put_k(vs, a.d);
                    f.load(f.kr, kp, mine + next, a.d);
                    f.template scores<state::KLD>(vs);
                    f.put_v(vs, there);
                    f.load(f.vr, vp, mine + next, a.d);
                    f.weigh(a.scale_log2, &there, there == ~0u);
                    f.add(vs);
                }
            }
            // along the line a step goes to the next pair or to the next part: their sum names what a part found for a pair
            const int64_t slot = (((int64_t)b * a.H + h + part) * a.tiles + tile) * ROWS;
#pragma unroll
            for (int r = 0; r < NR; ++r)
                join_waves<DP>(f, r, reinterpret_cast<float*>(pool), top, sum, [&](int row, int c, v4f y, float big, float z) {
                    if (r * 16 + row >= rows) return;
                    *reinterpret_cast<v4f*>(a.part_o + (slot + r * 16 + row) * DP + c) = y;
                    if (c == 0) a.part_ml[(slot + r * 16 + row) * 2] = big, a.part_ml[(slot + r * 16 + row) * 2 + 1] = z;
                });
        }
        at += last - first;
        if (at >= end) break;
        first = 0;
        if (++h == a.H) {
            h = 0;
            do s = stream_of(a, ++b, false);
            while (s.units == 0);
        }
    }
}

// The same for many rows: W waves of 32 rows each share tiles of KT keys in LDS, K and V, two of them: while one is worked on,
// the next comes into registers, and from there into the other's place.
template <bool BF16, int DP, int W, bool FULL>
__global__ __launch_bounds__(64 * W, DP == 256 ? 1 : 2) void attend_wide_kernel(attend_args a) {
    constexpr int ROWS = 32 * W, KT = DP == 256 || W == 2 ? 32 : 64, THREADS = 64 * W;
    typedef flash<BF16, DP, 2, KT, 2, FULL> state;
    constexpr int KLD = DP + 8, VLD = state::VLD;     // LDS rows: 16 rows' pieces of 16 bytes meet no bank twice
    constexpr int LPR = DP / 8, PIECES = KT * LPR, MINE = (PIECES + THREADS - 1) / THREADS;
    __shared__ __align__(16) uint16_t ks[2][KT * KLD], vs[2][KT * VLD];
    __shared__ uint32_t listed[LISTED], held[LISTED / 32];
    __shared__ int waves[W], where[2];

    const int t = threadIdx.x, lane = t % 64, col = lane % 16, quad = lane / 16, wave = uniform(t / 64);
    const int tile = (int)(blockIdx.x / 8) % a.tiles, part = (int)(blockIdx.x / 8) / a.tiles * 8 + (int)(blockIdx.x % 8);
    int at, end;
    if (!place_part(a, part, waves, where, &at, &end)) return;
    int b = uniform(where[0]);
    const int offset = uniform(where[1]);
    stream s = stream_of(a, b, false);
    int h = offset / s.units, first = offset % s.units;
    const v4i *kp = reinterpret_cast<const v4i*>(a.k), *vp = reinterpret_cast<const v4i*>(a.v);
    state f;
    v4i kr[MINE], vr[MINE];

    for (;;) {
        const int last = min(s.units, first + (end - at));
        const int rows = min(s.drafted * a.G - tile * ROWS, ROWS);   // query rows here
        if (rows > 0) {
            f.start(a, b, h, tile * ROWS + wave * 32, s.drafted);
            for (int u0 = first; u0 < last; u0 += LISTED / UNIT) {
                const int n = min(last - u0, LISTED / UNIT) * (UNIT / KT);
                list_keys(a, s, b, h, u0, n / (UNIT / KT), listed, held);
                auto load = [&](int u) {
#pragma unroll
                    for (int j = 0; j < MINE; ++j) {
                        const int x = min(t + j * THREADS, PIECES - 1), piece = x % LPR;
                        const uint32_t row = listed[u * KT + x / LPR] + (FULL ? piece : min(piece, a.d / 8 - 1));
                        kr[j] = kp[row];
                        vr[j] = vp[row];
                    }
                };
                // pieces behind the head dimension count as 0 on K's side; rows of keys that are not there do on V's
                auto put = [&](int u) {
#pragma unroll
                    for (int j = 0; j < MINE; ++j) {
                        const int x = t + j * THREADS, key = x / LPR, piece = x % LPR;
                        if (PIECES % THREADS == 0 || x < PIECES) {
                            const bool there = held[u * (KT / 32) + key / 32] >> (key % 32) & 1u;
                            *reinterpret_cast<v4i*>(&ks[u & 1][key * KLD + piece * 8]) = FULL || piece < a.d / 8 ? kr[j] : v4i{0, 0, 0, 0};
                            *reinterpret_cast<v4i*>(&vs[u & 1][key * VLD + piece * 8]) = there ? vr[j] : v4i{0, 0, 0, 0};
                        }
                    }
                };
                load(0);
                put(0);
                __syncthreads();
                for (int u = 0; u < n; ++u) {
                    load(min(u + 1, n - 1));
                    uint32_t there[KT / 32], every = ~0u;
#pragma unroll
                    for (int j = 0; j < KT / 32; ++j) {
                        there[j] = (uint32_t)uniform((int)held[u * (KT / 32) + j]);
                        every &= there[j];
                    }
                    f.template scores<KLD>(ks[u & 1]);
                    f.weigh(a.scale_log2, there, every == ~0u);
                    f.add(vs[u & 1]);
                    if (u + 1 < n) put(u + 1);
                    __syncthreads();
                }
            }
            const int64_t slot = (((int64_t)b * a.H + h + part) * a.tiles + tile) * ROWS;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = wave * 32 + r * 16 + col;
                const float l = rows_sum(f.l[r]);
                if (row < rows) {
#pragma unroll
                    for (int c = 0; c < state::CT; ++c) *reinterpret_cast<v4f*>(a.part_o + (slot + row) * DP + c * 16 + quad * 4) = f.o[r][c];
                    if (quad == 0) a.part_ml[(slot + row) * 2] = f.m[r], a.part_ml[(slot + row) * 2 + 1] = l;
                }
            }
        }
        at += last - first;
        if (at >= end) break;
        first = 0;
        if (++h == a.H) {
            h = 0;
            do s = stream_of(a, ++b, false);
            while (s.units == 0);
        }
    }
}

// Workgroup (pair, 16 rows): the drafted tokens, the parts of the context, the end.
template <bool BF16, int DP, bool FULL>
__global__ __launch_bounds__(256, DP == 256 ? 1 : 2) void attend_finish_kernel(attend_args a) {
    typedef own_keys<BF16, DP, 1, 2, FULL> state;
    constexpr uint32_t EXP = BF16 ? 0x7f80u : 0x7c00u;
    __shared__ __align__(16) unsigned char pool[4 * 32 * state::VLD * 2];
    __shared__ uint32_t listed[256];
    __shared__ float top[4][16], sum[4][16];
    const int t = threadIdx.x, lane = t % 64, wave = uniform(t / 64), col = lane % 16, quad = lane / 16;
    const int row0 = blockIdx.y * 16, h = blockIdx.x % a.H, b = blockIdx.x / a.H;
    const stream s = stream_of(a, b, blockIdx.y == 0 && h == 0);
    const int rows = min(s.drafted * a.G - row0, 16);
    if (rows <= 0) return;
    uint16_t* vs = reinterpret_cast<uint16_t*>(pool) + wave * 32 * state::VLD;
    state f;
    f.start(a, b, h, row0, s.drafted);
    if (a.k_new) {
        const v4i *kp = reinterpret_cast<const v4i*>(a.k_new), *vp = reinterpret_cast<const v4i*>(a.v_new);
        listed[t] = (((uint32_t)b * a.T + min(t, s.drafted - 1)) * a.H + h) * (uint32_t)(a.d / 8);
        __syncthreads();
        const int token = token_of(a, row0 + col);
        for (int j0 = wave * 32; j0 < s.drafted; j0 += UNIT) {
            const uint32_t there = s.drafted - j0 >= 32 ? ~0u : (1u << (s.drafted - j0)) - 1u;
            f.load(f.kr, kp, listed + j0, a.d);
            f.load(f.vr, vp, listed + j0, a.d);
            f.put_k(vs, a.d);
            f.template scores<state::KLD>(vs);
            // Not every row sees these: values that are not numbers stand apart.
            bool odd = false;
#pragma unroll
            for (int j = 0; j < state::VI; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t x = (uint32_t)f.vr[j][e];
                    if ((x & EXP) == EXP) x &= 0xffff0000u, odd = true;
                    if ((x & EXP << 16) == EXP << 16) x &= 0xffffu, odd = true;
                    f.vr[j][e] = (int)x;
                }
            f.put_v(vs, there);
            uint32_t word = 0;
            if (token < s.drafted) {
                if (a.mask) word = a.mask[((int64_t)b * a.T + token) * ((a.T + 31) / 32) + j0 / 32];
                else word = token - j0 >= 31 ? ~0u : token < j0 ? 0u : (2u << (token - j0)) - 1u;
            }
            const uint32_t sees = word & there;
            f.weigh(a.scale_log2, &sees, false);
            f.add(vs);
            if (__any(odd)) {
                // One drafted token at a time: its values that are not numbers alone in LDS, and only the rows that weigh it take the
                // product.
#pragma unroll 1
                for (int j = 0; j < 32; ++j) {
                    if (!(there >> j & 1u)) continue;
                    f.load(f.vr, vp, listed + j0, a.d);
#pragma unroll
                    for (int i = 0; i < state::VI; ++i)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint32_t y = (uint32_t)f.vr[i][e];
                            f.vr[i][e] = (int)(((y & EXP) == EXP ? y & 0xffffu : 0u) | ((y & EXP << 16) == EXP << 16 ? y & 0xffff0000u : 0u));
                        }
                    f.put_v(vs, 1u << j);
                    v4i alone = {0, 0, 0, 0};
                    uint32_t any = 0;
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (e / 4 * 16 + quad * 4 + e % 4 == j) {
                            any = (uint32_t)f.pf[0][0][0][e / 2] & (e % 2 ? 0xffff0000u : 0xffffu);
                            alone[e / 2] = (int)any;
                        }
                    const bool takes = rows_max(any ? 1.f : 0.f) > 0.f;
#pragma unroll
                    for (int c = 0; c < state::CT; ++c) {
                        const v4f x = mfma<BF16>(f.get_v(vs, c), alone, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                        for (int r = 0; r < 4; ++r) f.o[0][c][r] += takes ? x[r] : 0.f;
                    }
                }
            }
        }
    }
    if (s.units > 0) {
        const int units = a.starts[a.B], g = a.starts[b] + h * s.units, quota = quota_of(a, units);
        const int p0 = g / quota, p1 = (g + s.units - 1) / quota;
        // this row in the tiles of the first kernel
        const int tile = row0 / a.rows, in = row0 % a.rows + min(col, rows - 1);
        auto slot = [&](int p) { return (((int64_t)b * a.H + h + p) * a.tiles + tile) * a.rows + in; };
        // Every other part's maximum first, then their sums, several parts on their way at a time.  A part without keys left zeros.
        float big = f.m[0];
#pragma unroll 4
        for (int p = p0 + wave; p <= p1; p += 4) big = fmaxf(big, a.part_ml[slot(p) * 2]);
        if (f.m[0] != -INFINITY) f.rescale(0, __builtin_amdgcn_exp2f(f.m[0] - big));
        f.m[0] = big;
#pragma unroll 4
        for (int p = p0 + wave; p <= p1; p += 4) {
            const int64_t at = slot(p);
            const float m = a.part_ml[at * 2], z = a.part_ml[at * 2 + 1];
            const float* part = a.part_o + at * DP + quad * 4;
            v4f x[state::CT];
#pragma unroll
            for (int c = 0; c < state::CT; ++c) x[c] = *reinterpret_cast<const v4f*>(part + c * 16);
            const float w = m == -INFINITY ? 0.f * z : __builtin_amdgcn_exp2f(m - big);
            if (quad == 0) f.l[0] += w * z;
#pragma unroll
            for (int c = 0; c < state::CT; ++c) f.o[0][c] += w * x[c];
        }
    }
    join_waves<DP>(f, 0, reinterpret_cast<float*>(pool), top, sum, [&](int row, int c, v4f y, float m, float z) {
        if (row >= rows) return;
        const int i = token_of(a, row0 + row);
        const int64_t to = (((int64_t)b * a.T + i) * a.H + h) * a.G + (row0 + row - i * a.G);
        const bool some = z > 0.f || z != z;
        const float g = some ? 1.f / z : 0.f;
        if (FULL || c < a.d) *reinterpret_cast<v2i*>(a.out + to * a.d + c) = v2i{pack<BF16>(y[0] * g, y[1] * g), pack<BF16>(y[2] * g, y[3] * g)};
        if (c == 0 && a.lse) a.lse[to] = some ? (m + log2f(z)) * 0.693147180559945309f : -INFINITY;
    });
}

template <bool BF16, int DP, bool FULL>
void launch_attend(const attend_args& a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.parts + 7) / 8 * 8 * a.tiles)), block(256);
    if (a.rows == 16) hipLaunchKernelGGL((attend_context_kernel<BF16, DP, 1, FULL>), grid, block, 0, stream, a);
    else if (a.rows == 32) hipLaunchKernelGGL((attend_context_kernel<BF16, DP, 2, FULL>), grid, block, 0, stream, a);
    else if (a.rows == 64) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 2, FULL>), grid, dim3(128), 0, stream, a);
    else if (a.rows == 128) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 4, FULL>), grid, block, 0, stream, a);
    else if (a.rows == 192) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 6, FULL>), grid, dim3(384), 0, stream, a);
    else hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 8, FULL>), grid, dim3(512), 0, stream, a);
    hipLaunchKernelGGL((attend_finish_kernel<BF16, DP, FULL>), dim3((unsigned)(a.B * a.H), (unsigned)((a.T * a.G + 15) / 16)), block, 0, stream, a);
}

template <bool BF16>
void launch_attend(const attend_args& a, hipStream_t stream) {
    if (a.d <= 64) a.d == 64 ? launch_attend<BF16, 64, true>(a, stream) : launch_attend<BF16, 64, false>(a, stream);
    else if (a.d <= 128) a.d == 128 ? launch_attend<BF16, 128, true>(a, stream) : launch_attend<BF16, 128, false>(a, stream);
    else a.d == 256 ? launch_attend<BF16, 256, true>(a, stream) : launch_attend<BF16, 256, false>(a, stream);
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
    if (G < 1 || G > 1024) SWARM_REJECT(ctx, "tree_attend: G=%d outside [1,1024]", G);
    const int64_t rows = (int64_t)B * T * cache->H * G;
    if (rows > ((int64_t)1 << 30)) SWARM_REJECT(ctx, "tree_attend: B*T*H*G above 2^30");
    if ((int64_t)cache->P * cache->H * cache->page * (cache->d / 8) > UINT32_MAX || (int64_t)B * T * cache->H * (cache->d / 8) > UINT32_MAX)
        SWARM_REJECT(ctx, "tree_attend: a layer of the pool, or k_new, of 64 GiB or more");
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
    // Up to 32 rows go to the kernel whose waves have keys of their own, more to the one whose waves share them, 32 rows a wave: as few tiles
    // of rows as 8 waves allow, and in each as few waves as the rows need.
    const int M = T * G, DP = cache->d <= 64 ? 64 : cache->d <= 128 ? 128 : 256;
    if (M <= 32) {
        a.tiles = 1;
        a.rows = (M + 15) / 16 * 16;
    } else {
        a.tiles = (M + 255) / 256;
        a.rows = (M + 64 * a.tiles - 1) / (64 * a.tiles) * 64;
    }
    // as many parts as workgroups are resident at once, and no more than there can be units
    const int64_t slots = !sel ? (int64_t)cache->cap * cache->page : unit == SWARM_SEL_PAGES ? (int64_t)n_sel * cache->page : n_sel;
    const int64_t units = (int64_t)B * cache->H * ((slots + UNIT - 1) / UNIT);
    if (units > INT32_MAX - 65536) SWARM_REJECT(ctx, "tree_attend: contexts of up to %lld times 128 keys, above 2^31", (long long)units);
    const int resident = 256 * (DP > 128 ? 1 : a.rows <= 128 ? 2 : 1), want = a.tiles < resident ? resident / a.tiles : 1;
    a.parts = (int)(units < want ? units : want);
    const size_t heads = (4 * ((size_t)B + 1) + 15) / 16 * 16, left = ((size_t)B * cache->H + a.parts) * a.tiles * a.rows;
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
    a.scale_log2 = scale * 1.44269504088896341f;
    cache->dtype == SWARM_BF16 ? launch_attend<true>(a, ctx->stream) : launch_attend<false>(a, ctx->stream);
    return swarm_check_launch(ctx, "attend");
}
