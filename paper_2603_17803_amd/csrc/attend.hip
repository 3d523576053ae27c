// Attention of drafted tokens over a paged cache.
//
// The T*G query rows that a KV head's group has (drafted token i, query head g: row i*G + g) share every key and value, so a
// workgroup takes up to 64 of them and streams the keys past: per 16 rows, S^T = K Q^T on the 16x16x32 matrix instruction (keys are
// the rows of its result, query rows its columns), the softmax's running maximum and sum a lane per query row, O^T += V^T P^T on the
// same instruction.  A lane's eight weights of 32 keys are, as they come out of the first product, one operand of the
// second; V^T's operand is read out of LDS by the transposing read.  K goes straight from memory into registers.
//
// The four waves of a workgroup each take 32 of the 128 keys of a unit, all rows, and meet only at a segment's end: no barrier in the
// loop.  The units of all (stream, head) pairs stand in one line, which is cut into equal parts, one for each workgroup, whatever
// the streams' lengths are; a pair that a cut goes through leaves partial results (fp32, unnormalised) that a second kernel joins.
#include <math.h>

#include "common.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));

constexpr int UNIT = 128;                        // keys of a unit, 32 for each wave
constexpr int LISTED = 2048;                     // keys whose rows are looked up at a time
constexpr uint32_t NO_ROW = 0xffffffffu;

struct attend_args {
    const uint16_t *k, *v, *q, *k_new, *v_new;   // k, v: the layer's part of the pool
    const int32_t *table, *len, *n_new, *sel;
    const uint32_t* mask;
    uint16_t* out;
    float* lse;
    float* part_o;                               // [slots][rows][DP], then [slots][rows] maxima and sums
    float* part_ml;
    uint32_t* flags;
    int P, H, page, d, cap, B, T, G, n_sel, unit;
    int parts, tiles;                            // parts of the line of units; tiles of rows of a (stream, head)
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

// What a stream brings: tokens of its context (slots of its selection), drafted tokens, units of one (head, tile).
struct stream {
    int len, slots, drafted, context_units, units;
};
__device__ __forceinline__ stream stream_of(const attend_args& a, int b, bool tell) {
    stream s;
    const int64_t most = (int64_t)a.cap * a.page;
    s.len = a.len[b];
    s.drafted = a.n_new ? a.n_new[b] : a.T;
    if (s.len < 0 || s.len > most || s.drafted < 0 || s.drafted > a.T) {
        if (tell) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        s.len = s.len < 0 ? 0 : s.len > most ? (int)most : s.len;
        s.drafted = min(max(s.drafted, 0), a.T);
    }
    s.slots = !a.sel ? s.len : a.unit == SWARM_SEL_PAGES ? a.n_sel * a.page : a.n_sel;
    s.context_units = (s.slots + UNIT - 1) / UNIT;
    const int all = s.context_units + (a.k_new ? (s.drafted + UNIT - 1) / UNIT : 0);
    s.units = all < 1 ? 1 : all;                 // a row that sees nothing is written too
    return s;
}

// Sums over a workgroup of four waves.
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* waves) {
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % 64 == 0) waves[threadIdx.x / 64] = v;
    __syncthreads();
    return waves[0] + waves[1] + waves[2] + waves[3];
}
__device__ __forceinline__ int64_t block_before(int64_t v, int64_t* waves, int64_t* total) {
    int64_t x = v;
    const int lane = threadIdx.x % 64, w = threadIdx.x / 64;
    for (int o = 1; o < 64; o <<= 1) {
        const int64_t y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) waves[w] = x;
    __syncthreads();
    int64_t below = 0;
    for (int i = 0; i < w; ++i) below += waves[i];
    *total = waves[0] + waves[1] + waves[2] + waves[3];
    return below + x - v;
}

// All units of the call, for each tile of rows.
__device__ int64_t all_units(const attend_args& a, int64_t* waves, bool tell) {
    int64_t mine = 0;
    for (int b = threadIdx.x; b < a.B; b += 256) mine += (int64_t)a.H * stream_of(a, b, tell).units;
    return block_sum(mine, waves);
}
// Where part p of n starts in a line of `units`, and the part that holds unit g: the last one that starts at or before it.
__device__ __forceinline__ int64_t part_start(int64_t units, int p, int n) { return units * p / n; }
__device__ __forceinline__ int part_of(int64_t units, int64_t g, int n) { return (int)(((g + 1) * n + units - 1) / units) - 1; }

// Four channels of a finished row: the sum over its keys divided by that of their weights, and its lse.  A row without keys is 0.
template <bool BF16>
__device__ __forceinline__ void put_row(const attend_args& a, int b, int h, int row, int c, v4f y, float m, float z) {
    const int64_t to = (((int64_t)b * a.T + row / a.G) * a.H + h) * a.G + row % a.G;
    const bool some = z > 0.f || z != z;
    const float f = some ? 1.f / z : 0.f;
    if (c < a.d) *reinterpret_cast<v2i*>(a.out + to * a.d + c) = v2i{pack<BF16>(y[0] * f, y[1] * f), pack<BF16>(y[2] * f, y[3] * f)};
    if (c == 0 && a.lse) a.lse[to] = some ? (m + log2f(z)) * 0.693147180559945309f : -INFINITY;
}

template <bool BF16, int DP, int NR>
__global__ __launch_bounds__(256, DP == 256 ? 1 : NR == 1 ? 3 : NR == 2 ? 2 : 1) void attend_kernel(attend_args a) {
    constexpr int KS = DP / 32, CT = DP / 16, VI = DP / 16, ROWS = 16 * NR;
    constexpr int VLD = DP + 16;                 // LDS row of V in elements: 32 bytes behind each, so that 16 rows' reads meet no bank twice
    constexpr int OLD = DP + 4;                  // row of a wave's part of the result in floats
    constexpr int LPR = DP / 8, RPI = 64 / LPR;  // lanes on a row of V, rows that a wave moves at a time
    constexpr int TERMS = 2;
    constexpr uint32_t EXP = BF16 ? 0x7f80u : 0x7c00u;
    __shared__ __align__(16) unsigned char pool[4 * 32 * VLD * 2];
    __shared__ uint32_t listed[LISTED];
    __shared__ float top[4][ROWS], sum[4][ROWS];
    __shared__ int64_t waves[4], where[2];
    static_assert(16 * OLD * 4 <= 32 * VLD * 2, "a wave's part of the result fits its rows of V");

    const int t = threadIdx.x, lane = t % 64, wave = t / 64, col = lane % 16, quad = lane / 16;
    const int tile = (int)(blockIdx.x / 8) % a.tiles, part = (int)(blockIdx.x / 8) / a.tiles * 8 + (int)(blockIdx.x % 8);
    if (part >= a.parts) return;
    const int64_t units = all_units(a, waves, blockIdx.x == 0);
    int64_t at = part_start(units, part, a.parts);
    const int64_t end = part_start(units, part + 1, a.parts);
    if (at >= end) return;
    {
        int64_t before = 0, all;
        for (int base = 0; base < a.B; base += 256) {
            const int b = base + t;
            const int64_t n = b < a.B ? (int64_t)a.H * stream_of(a, b, false).units : 0;
            const int64_t start = before + block_before(n, waves, &all);
            if (start <= at && at < start + n) where[0] = b, where[1] = at - start;
            before += all;
            if (before > at) break;
        }
        __syncthreads();
    }
    int b = (int)where[0];
    stream s = stream_of(a, b, false);
    int h = (int)(where[1] / s.units), first = (int)(where[1] % s.units);
    const int chunks = a.d / 8;
    uint16_t* vs = reinterpret_cast<uint16_t*>(pool) + wave * 32 * VLD;
    uint16_t* vput = vs + (lane / LPR) * VLD + lane % LPR * 8;
    typedef __attribute__((address_space(3))) v4s lds_v4s;
    const uint16_t* vget = vs + (quad * 4 + col / 4) * VLD + col % 4 * 4;
    // where a lane's pieces stand in a row; pieces behind the head dimension read another and count as 0
    int kat[KS];
#pragma unroll
    for (int c = 0; c < KS; ++c) kat[c] = min(c * 4 + quad, chunks - 1) * 8;
    const int vat = min(lane % LPR, chunks - 1) * 8;

    for (;;) {
        const int last = (int)min((int64_t)s.units, first + (end - at));
        const int rows = min(s.drafted * a.G - tile * ROWS, ROWS);   // query rows here
        if (rows > 0) {
            v4i qf[NR][KS];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                const int r = tile * ROWS + n * 16 + col, i = r / a.G;
                const uint16_t* q = a.q + ((((int64_t)b * a.T + i) * a.H + h) * a.G + r % a.G) * a.d;
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                    const int c = k * 4 + quad;
                    qf[n][k] = i < s.drafted && c < chunks ? *reinterpret_cast<const v4i*>(q + c * 8) : v4i{0, 0, 0, 0};
                }
            }
            float m[NR], l[NR];
            v4f o[NR][CT];
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                m[n] = -INFINITY;
                l[n] = 0.f;
#pragma unroll
                for (int c = 0; c < CT; ++c) o[n][c] = v4f{0.f, 0.f, 0.f, 0.f};
            }

            // Pieces of the line of keys whose rows are looked up together: some of the context, then the drafted tokens.
            for (int u0 = first; u0 < last;) {
                const bool drafts = u0 >= s.context_units;
                const int u1 = drafts ? last : min(min(u0 + LISTED / UNIT, s.context_units), last);
                const uint16_t *kbase = drafts ? a.k_new : a.k, *vbase = drafts ? a.v_new : a.v;
                const int j0 = (u0 - s.context_units) * UNIT;     // the first drafted token of the piece
                __syncthreads();
                for (int x = t; x < (u1 - u0) * UNIT; x += 256) {
                    uint32_t row = NO_ROW;
                    if (drafts) {
                        if (a.k_new && j0 + x < s.drafted) row = ((uint32_t)b * a.T + j0 + x) * a.H + h;
                    } else if (u0 * UNIT + x < s.slots) {
                        int pos = u0 * UNIT + x;
                        if (a.sel) {
                            const bool by_page = a.unit == SWARM_SEL_PAGES;
                            const int e = a.sel[((int64_t)b * a.H + h) * a.n_sel + (by_page ? pos / a.page : pos)];
                            if (e < 0 || e >= (by_page ? a.cap : a.cap * a.page)) {
                                if (e != -1) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
                                pos = s.len;
                            } else {
                                pos = by_page ? e * a.page + (pos & (a.page - 1)) : e;
                            }
                        }
                        if (pos < s.len) {
                            const int id = a.table[(int64_t)b * a.cap + pos / a.page];
                            if (id < 0 || id >= a.P) atomicOr(a.flags, SWARM_DEV_BAD_PAGE);
                            else row = ((uint32_t)id * a.H + h) * a.page + (pos & (a.page - 1));
                        }
                    }
                    listed[x] = row;
                }
                __syncthreads();

                v4i kf[2][KS], vr[VI];
                uint32_t valid = 0;              // keys of the tile that are there; the others are read as row 0
                const uint32_t* mine = listed + wave * 32;
                auto load_k = [&](int u) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        uint32_t row = mine[(u - u0) * UNIT + k * 16 + col];
                        row = row == NO_ROW ? 0 : row;
                        const uint16_t* p = kbase + (uint64_t)row * a.d;
#pragma unroll
                        for (int c = 0; c < KS; ++c) kf[k][c] = *reinterpret_cast<const v4i*>(p + kat[c]);
                    }
                };
                auto load_v = [&](int u) {
                    valid = (uint32_t)__ballot(mine[(u - u0) * UNIT + lane % 32] != NO_ROW);
#pragma unroll
                    for (int j = 0; j < VI; ++j) {
                        uint32_t row = mine[(u - u0) * UNIT + j * RPI + lane / LPR];
                        row = row == NO_ROW ? 0 : row;
                        vr[j] = *reinterpret_cast<const v4i*>(vbase + (uint64_t)row * a.d + vat);
                    }
                };
                // a piece without any key (a row that sees nothing, bad pages) reads nothing: its bases may be NULL
                bool some = false;
                for (int x = lane; x < (u1 - u0) * UNIT; x += 64) some |= listed[x] != NO_ROW;
                if (__any(some)) {
                    load_v(u0);
                    load_k(u0);
                    for (int u = u0; u < u1; ++u) {
                        const uint32_t there = valid;
                        if (there != ~0u) {
#pragma unroll
                            for (int j = 0; j < VI; ++j)
                                if (!(there >> (j * RPI + lane / LPR) & 1u)) vr[j] = v4i{0, 0, 0, 0};
                        }
                        bool odd = false;        // drafted tokens' values that are not numbers: not every row sees them
                        if (drafts) {
#pragma unroll
                            for (int j = 0; j < VI; ++j)
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    uint32_t x = (uint32_t)vr[j][e];
                                    if ((x & EXP) == EXP) x &= 0xffff0000u, odd = true;
                                    if ((x & EXP << 16) == EXP << 16) x &= 0xffffu, odd = true;
                                    vr[j][e] = (int)x;
                                }
                            odd = __any(odd);
                        }
#pragma unroll
                        for (int j = 0; j < VI; ++j) *reinterpret_cast<v4i*>(vput + j * RPI * VLD) = vr[j];
                        if (u + 1 < u1) load_v(u + 1);

                        if (chunks < DP / 8) {
#pragma unroll
                            for (int c = 0; c < KS; ++c)
                                if (c * 4 + quad >= chunks) kf[0][c] = kf[1][c] = v4i{0, 0, 0, 0};
                        }
                        v4f sc[NR][2];
#pragma unroll
                        for (int k = 0; k < 2; ++k)
#pragma unroll
                            for (int n = 0; n < NR; ++n) {
                                sc[n][k] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                                for (int c = 0; c < KS; ++c) sc[n][k] = mfma<BF16>(kf[k][c], qf[n][c], sc[n][k]);
                            }
                        if (u + 1 < u1) load_k(u + 1);

                        v4i pf[NR][TERMS];
#pragma unroll
                        for (int n = 0; n < NR; ++n) {
                            float p[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) p[e] = sc[n][e / 4][e % 4] * a.scale_log2;
                            uint32_t sees = there;
                            if (drafts) {
                                const int i = (tile * ROWS + n * 16 + col) / a.G, j = (u - s.context_units) * UNIT + wave * 32;
                                uint32_t word = 0;
                                if (i < s.drafted && there) {
                                    if (a.mask) word = a.mask[((int64_t)b * a.T + i) * ((a.T + 31) / 32) + j / 32];
                                    else word = i - j >= 31 ? ~0u : i < j ? 0u : (2u << (i - j)) - 1u;
                                }
                                sees &= word;
                            }
                            if (drafts || there != ~0u) {
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (!(sees >> (e / 4 * 16 + quad * 4 + e % 4) & 1u)) p[e] = -INFINITY;
                            }
                            const float mx = rows_max(fmaxf(fmaxf(fmaxf(p[0], p[1]), fmaxf(p[2], p[3])), fmaxf(fmaxf(p[4], p[5]), fmaxf(p[6], p[7]))));
                            if (__any(mx > m[n])) {
                                const float next = fmaxf(m[n], mx), old = m[n] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[n] - next);
                                m[n] = next;
                                l[n] *= old;
#pragma unroll
                                for (int c = 0; c < CT; ++c) o[n][c] *= old;
                            }
                            const float base = m[n] == -INFINITY ? 0.f : m[n];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                p[e] = __builtin_amdgcn_exp2f(p[e] - base);
                                l[n] += p[e];
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                pf[n][0][e] = pack<BF16>(p[2 * e], p[2 * e + 1]);
                                if (TERMS == 2)
                                    pf[n][TERMS - 1][e] = pack<BF16>(p[2 * e] - value_of<BF16>((uint32_t)pf[n][0][e] & 0xffffu), p[2 * e + 1] - value_of<BF16>((uint32_t)pf[n][0][e] >> 16));
                            }
                        }
                        auto v_of = [&](int c) {
                            v4i vf;
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const v2i x = __builtin_bit_cast(v2i, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s*)(vget + k * 16 * VLD + c * 16)));
                                vf[2 * k] = x[0];
                                vf[2 * k + 1] = x[1];
                            }
                            return vf;
                        };
#pragma unroll
                        for (int c = 0; c < CT; ++c) {
                            const v4i vf = v_of(c);
#pragma unroll
                            for (int n = 0; n < NR; ++n)
#pragma unroll
                                for (int k = 0; k < TERMS; ++k) o[n][c] = mfma<BF16>(vf, pf[n][k], o[n][c]);
                        }
                        if (odd) {
                            // One drafted token at a time: its values that are not numbers alone in LDS, and only the rows that weigh
                            // it take the product.
                            for (int j = 0; j < 32; ++j) {
                                if (!(there >> j & 1u)) continue;
                                const uint32_t row = mine[(u - u0) * UNIT + j];
#pragma unroll
                                for (int i = 0; i < VI; ++i) {
                                    v4i x = {0, 0, 0, 0};
                                    if (i * RPI + lane / LPR == j) {
                                        x = *reinterpret_cast<const v4i*>(vbase + (uint64_t)row * a.d + vat);
#pragma unroll
                                        for (int e = 0; e < 4; ++e) {
                                            const uint32_t y = (uint32_t)x[e];
                                            x[e] = (int)(((y & EXP) == EXP ? y & 0xffffu : 0u) | ((y & EXP << 16) == EXP << 16 ? y & 0xffff0000u : 0u));
                                        }
                                    }
                                    *reinterpret_cast<v4i*>(vput + i * RPI * VLD) = x;
                                }
#pragma unroll
                                for (int n = 0; n < NR; ++n) {
                                    v4i alone = {0, 0, 0, 0};
                                    uint32_t any = 0;
#pragma unroll
                                    for (int e = 0; e < 8; ++e)
                                        if (e / 4 * 16 + quad * 4 + e % 4 == j) {
                                            const uint32_t w = (uint32_t)pf[n][0][e / 2] & (e % 2 ? 0xffff0000u : 0xffffu);
                                            alone[e / 2] = (int)w;
                                            any = w;
                                        }
                                    const bool takes = rows_max(any ? 1.f : 0.f) > 0.f;
#pragma unroll
                                    for (int c = 0; c < CT; ++c) {
                                        const v4f x = mfma<BF16>(v_of(c), alone, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                                        for (int r = 0; r < 4; ++r) o[n][c][r] += takes ? x[r] : 0.f;
                                    }
                                }
                            }
                        }
                    }
                }
                u0 = u1;
            }

            // the four waves' parts, 16 rows at a time
            const bool whole = first == 0 && last == s.units;
            const int64_t slot = ((int64_t)part * 2 + (first > 0 ? 0 : 1)) * a.tiles + tile;
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                l[n] = rows_sum(l[n]);
                if (quad == 0) top[wave][n * 16 + col] = m[n], sum[wave][n * 16 + col] = l[n];
            }
            float* os = reinterpret_cast<float*>(pool) + wave * (32 * VLD / 2);
#pragma unroll
            for (int n = 0; n < NR; ++n) {
                if (n) __syncthreads();
#pragma unroll
                for (int c = 0; c < CT; ++c) *reinterpret_cast<v4f*>(os + col * OLD + c * 16 + quad * 4) = o[n][c];
                __syncthreads();
                for (int x = t; x < 16 * (DP / 4); x += 256) {
                    const int r16 = x / (DP / 4), c = x % (DP / 4) * 4, r = n * 16 + r16;
                    if (r >= rows) continue;
                    const float big = fmaxf(fmaxf(top[0][r], top[1][r]), fmaxf(top[2][r], top[3][r]));
                    v4f y = {0.f, 0.f, 0.f, 0.f};
                    float z = 0.f;
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const float f = top[w][r] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top[w][r] - big);
                        z += f * sum[w][r];
                        const v4f ow = *reinterpret_cast<const v4f*>(reinterpret_cast<float*>(pool) + w * (32 * VLD / 2) + r16 * OLD + c);
                        if (f > 0.f) y += f * ow;
                    }
                    if (whole) {
                        put_row<BF16>(a, b, h, tile * ROWS + r, c, y, big, z);
                    } else {
                        *reinterpret_cast<v4f*>(a.part_o + (slot * ROWS + r) * DP + c) = y;
                        if (c == 0) a.part_ml[(slot * ROWS + r) * 2] = big, a.part_ml[(slot * ROWS + r) * 2 + 1] = z;
                    }
                }
            }
            __syncthreads();
        }
        at += last - first;
        if (at >= end) break;
        first = 0;
        if (++h == a.H) {
            h = 0;
            s = stream_of(a, ++b, false);
        }
    }
}

// Workgroup (stream, head, tile): joins what the parts left of it.
template <bool BF16, int DP>
__global__ __launch_bounds__(256) void attend_join_kernel(attend_args a, int ROWS) {
    __shared__ int64_t waves[4];
    const int t = threadIdx.x;
    const int tile = blockIdx.x % a.tiles, h = blockIdx.x / a.tiles % a.H, b = blockIdx.x / a.tiles / a.H;
    const int64_t units = all_units(a, waves, false);
    int64_t mine = 0;
    for (int i = t; i < b; i += 256) mine += (int64_t)a.H * stream_of(a, i, false).units;
    const stream s = stream_of(a, b, false);
    const int64_t g = block_sum(mine, waves) + (int64_t)h * s.units;
    const int p0 = part_of(units, g, a.parts), p1 = part_of(units, g + s.units - 1, a.parts);
    if (p0 == p1) return;
    const int rows = min(s.drafted * a.G - tile * ROWS, ROWS);
    for (int x = t; x < rows * (DP / 4); x += 256) {
        const int r = x / (DP / 4), c = x % (DP / 4) * 4;
        // the first part's piece is the last one of that part, the others' pieces their first ones; parts without a unit left none
        float big = -INFINITY;
        for (int p = p0; p <= p1; ++p) {
            if (part_start(units, p, a.parts) == part_start(units, p + 1, a.parts)) continue;
            const int64_t slot = ((int64_t)p * 2 + (p == p0)) * a.tiles + tile;
            big = fmaxf(big, a.part_ml[(slot * ROWS + r) * 2]);
        }
        v4f y = {0.f, 0.f, 0.f, 0.f};
        float z = 0.f;
        for (int p = p0; p <= p1; ++p) {
            if (part_start(units, p, a.parts) == part_start(units, p + 1, a.parts)) continue;
            const int64_t slot = ((int64_t)p * 2 + (p == p0)) * a.tiles + tile;
            const float m = a.part_ml[(slot * ROWS + r) * 2], f = m == -INFINITY ? 0.f : exp2f(m - big);
            z += f * a.part_ml[(slot * ROWS + r) * 2 + 1];
            if (f > 0.f) y += f * *reinterpret_cast<const v4f*>(a.part_o + (slot * ROWS + r) * DP + c);
        }
        put_row<BF16>(a, b, h, tile * ROWS + r, c, y, big, z);
    }
}

template <bool BF16, int DP>
void launch_attend(const attend_args& a, int groups, hipStream_t stream) {
    const unsigned grid = (unsigned)((a.parts + 7) / 8 * 8 * a.tiles);
    if (groups == 1) hipLaunchKernelGGL((attend_kernel<BF16, DP, 1>), dim3(grid), dim3(256), 0, stream, a);
    else if (groups == 2) hipLaunchKernelGGL((attend_kernel<BF16, DP, 2>), dim3(grid), dim3(256), 0, stream, a);
    else if constexpr (DP > 128) return;          // wider heads come in tiles of 32 rows
    else if (groups == 3) hipLaunchKernelGGL((attend_kernel<BF16, DP, 3>), dim3(grid), dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((attend_kernel<BF16, DP, 4>), dim3(grid), dim3(256), 0, stream, a);
    if (a.parts > 1) hipLaunchKernelGGL((attend_join_kernel<BF16, DP>), dim3((unsigned)(a.B * a.H * a.tiles)), dim3(256), 0, stream, a, groups * 16);
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

    // Row tiles of at most 64 rows, as even as multiples of 16 allow: a tile of n x 16 rows pays for all of them.
    attend_args a{};
    const int M = T * G, DP = cache->d <= 64 ? 64 : cache->d <= 128 ? 128 : 256;
    const int most = DP > 128 ? 32 : 64;
    a.tiles = (M + most - 1) / most;
    const int groups = (M + 16 * a.tiles - 1) / (16 * a.tiles);
    // As many parts as workgroups are resident at once, and no more than there can be units.
    const int64_t slots = !sel ? (int64_t)cache->cap * cache->page : unit == SWARM_SEL_PAGES ? (int64_t)n_sel * cache->page : n_sel;
    const int64_t units = (int64_t)B * cache->H * ((slots + UNIT - 1) / UNIT + (T + UNIT - 1) / UNIT);
    const int resident = 256 * (DP > 128 ? 1 : groups == 1 ? 3 : groups == 2 ? 2 : 1);
    const int64_t want = a.tiles < resident ? resident / a.tiles : 1;
    a.parts = (int)(units < want ? units : want);
    if (a.parts > 1) {
        const size_t rows_left = (size_t)a.parts * 2 * a.tiles * groups * 16;
        st = swarm_scratch(ctx, &ctx->attend, &ctx->attend_bytes, rows_left * (DP + 2) * 4);
        if (st != SWARM_OK) return st;
        a.part_o = static_cast<float*>(ctx->attend);
        a.part_ml = a.part_o + rows_left * DP;
    }
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
    a.scale_log2 = scale * 1.44269504088896341f;
    const bool bf = cache->dtype == SWARM_BF16;
    if (DP == 64) bf ? launch_attend<true, 64>(a, groups, ctx->stream) : launch_attend<false, 64>(a, groups, ctx->stream);
    else if (DP == 128) bf ? launch_attend<true, 128>(a, groups, ctx->stream) : launch_attend<false, 128>(a, groups, ctx->stream);
    else bf ? launch_attend<true, 256>(a, groups, ctx->stream) : launch_attend<false, 256>(a, groups, ctx->stream);
    return swarm_check_launch(ctx, "attend_kernel");
}
