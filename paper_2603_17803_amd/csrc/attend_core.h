// Attention of drafted tokens over a paged cache.
//
// The T*G query rows that a KV head's group has (drafted token i, query head g: row i*G + g) share every key and value, so a
// workgroup takes up to 256 of them and streams the keys past: per 16 rows, S^T = K Q^T on the 16x16x32 matrix instruction (keys are
// the rows of its result, query rows its columns), the softmax's running maximum and sum a lane per query row, O^T += V^T P^T on the
// same instruction.  A lane's eight weights of 32 keys are, as they come out of the first product, one operand of the
// second; V^T's operand is read out of LDS by the transposing read.
//
// Two launches.  The first takes the contexts: the 128-key units of all (stream, head) pairs stand in one line, which is cut into equal parts, one
// for each workgroup, whatever the streams' lengths are.  What a part finds for a pair stays in scratch (fp32, unnormalised).  Up to 32 rows (16 of heads
// wider than 128) memory bounds it, and each of four waves takes 32 keys of a unit and all rows, with no barrier in the loop; above, waves have rows of their
// own and share the keys in LDS.  The second launch takes 16 rows of a pair, joins the parts, works the drafted tokens in under their masks,
// divides and rounds once.
#include <math.h>

#include "common.h"

struct attend_args {
    const uint16_t *k, *v, *q, *k_new, *v_new;   // k, v: the layer's part of the pool
    const int32_t *table, *len, *n_new, *sel;
    const uint32_t* mask;
    uint16_t* out;
    float* lse;
    int32_t* starts;                             // [B + 1]: where each stream's units start in the line, and their number
    float* part_o;                               // [slots][rows of a tile][DP]: sums of weighted values
    float* part_ml;                              // [slots][rows of a tile][2]: what weights refer to (in units of ln 2) and their sum
    uint32_t* flags;
    int P, H, page_log2, d, cap, B, T, G, n_sel, unit;
    int parts, tiles, rows;                      // parts of the line; tiles of a pair's rows, rows of a tile
    uint32_t per_g;                              // ceil(2^32 / G)
    float scale_log2;
};

// Head dimension that the kernels work with: the next of five.
inline int attend_width(int d) { return d <= 64 ? 64 : d <= 96 ? 96 : d <= 128 ? 128 : d <= 192 ? 192 : 256; }
constexpr int ATTEND_UNIT = 128;                 // keys of a unit of the line

void launch_attend_bf16(const attend_args& a, hipStream_t stream);
void launch_attend_fp16(const attend_args& a, hipStream_t stream);

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef _Float16 hf8 __attribute__((ext_vector_type(8)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s lds_v4s;

constexpr int UNIT = ATTEND_UNIT;                // 32 keys for each wave
constexpr int LISTED = 2048;                     // keys whose rows are looked up at a time

template <bool BF16>
__device__ __forceinline__ v4f mfma(v4i x, v4i y, v4f c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, x), __builtin_bit_cast(bf8, y), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(hf8, x), __builtin_bit_cast(hf8, y), c, 0, 0, 0);
}
template <bool BF16>
__device__ __forceinline__ float value_of(uint32_t x) {
    if constexpr (BF16) return __uint_as_float(x << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
}
// Two numbers cut to the type.
template <bool BF16>
__device__ __forceinline__ uint32_t cut_pair(float lo, float hi) {
    if constexpr (BF16) return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(lo, hi));
}
// Two numbers rounded to it, in one instruction.  (Rounded one by one: 192 rows of 96 73 us, so: 70.)
template <bool BF16>
__device__ __forceinline__ int pack(float lo, float hi) {
    typedef float v2f __attribute__((ext_vector_type(2)));
    typedef __bf16 v2b __attribute__((ext_vector_type(2)));
    typedef _Float16 v2h __attribute__((ext_vector_type(2)));
    if constexpr (BF16) return __builtin_bit_cast(int, __builtin_convertvector((v2f{lo, hi}), v2b));
    else return __builtin_bit_cast(int, __builtin_convertvector((v2f{lo, hi}), v2h));
}

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

// Between lanes of a wave that hand one another values through LDS: what was written before is written, and what was read is read.  The wave's LDS accesses
// run in order, so it costs nothing; it holds the compiler to that order.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

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
//   TERMS: how many terms of the cache's type a weight enters its product with v as.  Two are a weight to 2^-15 and more, and cost half as
//   many products again.  The first is cut, not rounded, and the second is what is left and 2^-23 of the weight (in fp16, which has no such small numbers,
//   its smallest number where nothing is left): neither is negative, and the second is not 0 where the first is not, so that a value that is
//   infinite stays so.
//   CS: into how many shares the channels of the result are cut, of which it has one: CT tiles of 16 channels.
template <bool BF16, int DP, int NR, int KT, int TERMS, bool FULL, int CS = 1>
struct flash {
    static constexpr int KS = DP / 32, CT = DP / 16 / CS;
    static constexpr int VLD = DP + 16;          // LDS row of V in elements: 32 bytes behind each, so that 16 rows' reads meet no bank twice
    // A row's weights are 2^(s - m).  m is raised to the row's maximum less LIFT when that has outgrown it by LAG more, so the largest weight is 2^LIFT to
    // 2^(LIFT + LAG).  fp16 holds no number from 2^16 on and none below 2^-24, and bits fewer than all below 2^-14: its weights stand as high as they may,
    // so that one is lost only below 2^-35 of the largest.  (At a maximum of 1 to 2^8, 131071 keys 25 octaves below one brought nothing.)
    static constexpr float LAG = BF16 ? 8.f : 4.f, LIFT = BF16 ? 0.f : 11.f;
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
    // What the first term leaves of a weight.  The middle one of three numbers is what is left or fp16's smallest number, where the weight is not below
    // that, and the weight itself where it is.
    static __device__ __forceinline__ float left(float p, float cut) {
        if constexpr (BF16) return __builtin_fmaf(p, 1.f + 0x1p-23f, -cut);
        else return __builtin_amdgcn_fmed3f(p - cut, 0x1p-24f, p);
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
    // The weights of KT keys; sees[j]: which of the keys 32 j to 32 j + 31 the lane's rows see.  What weights refer to is raised only
    // when one of the 16 rows has outgrown it: no sum here minds the larger weights, and most tiles rescale nothing.
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
            mx[n] = rows_max(mx[n]) - LIFT;
            grown |= mx[n] > m[n] + LAG;
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
                    if constexpr (TERMS == 1) {
                        pf[n][0][j][e] = pack<BF16>(p[2 * e], p[2 * e + 1]);
                    } else {
                        const uint32_t cut = cut_pair<BF16>(p[2 * e], p[2 * e + 1]);
                        pf[n][0][j][e] = (int)cut;
                        pf[n][1][j][e] = pack<BF16>(left(p[2 * e], value_of<BF16>(cut & 0xffffu)), left(p[2 * e + 1], value_of<BF16>(cut >> 16)));
                    }
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
template <bool BF16, int DP, int NR, int TERMS, bool FULL, int CS = 1>
struct own_keys : flash<BF16, DP, NR, 32, TERMS, FULL, CS> {
    typedef flash<BF16, DP, NR, 32, TERMS, FULL, CS> base;
    static constexpr int LPR = DP <= 64 ? 8 : DP <= 128 ? 16 : 32, RPI = 64 / LPR, VI = 32 / RPI;   // lanes on a row, rows at a time, pieces of a lane
    static constexpr int KLD = DP + 8, VLD = base::VLD;                // LDS rows in elements: 16 rows' pieces of 16 bytes meet no bank twice
    v4i kr[VI], vr[VI];
    // row(key): where the row of one of the 32 keys starts, in pieces.  Pieces behind the head dimension read another one; on K's
    // side they then count as 0.
    template <typename ROW>
    static __device__ __forceinline__ void load(v4i (&r)[VI], const v4i* from, int d, ROW&& row) {
        const int lane = threadIdx.x % 64;
        from += FULL && LPR == DP / 8 ? lane % LPR : min(lane % LPR, d / 8 - 1);
#pragma unroll
        for (int j = 0; j < VI; ++j) r[j] = __builtin_nontemporal_load(from + row(j * RPI + lane / LPR));
    }
    __device__ __forceinline__ void put_k(uint16_t* lds, int d) {
        const int lane = threadIdx.x % 64;
        uint16_t* to = lds + (lane / LPR) * KLD + lane % LPR * 8;
        if (LPR == DP / 8 || lane % LPR < DP / 8) {
#pragma unroll
            for (int j = 0; j < VI; ++j) {
                if (!FULL) kr[j] &= (lane % LPR - d / 8) >> 31;
                *reinterpret_cast<v4i*>(to + j * RPI * KLD) = kr[j];
            }
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
        if (LPR == DP / 8 || lane % LPR < DP / 8) {
#pragma unroll
            for (int j = 0; j < VI; ++j) *reinterpret_cast<v4i*>(to + j * RPI * VLD) = vr[j];
        }
    }
};

// Joins what the W waves of a workgroup carry of 16 rows, through LDS (16 rows of OLD floats for each wave): calls
// put(row, channel, sums of four channels, what weights refer to, sum of weights) for each row and each four channels.
template <int W, typename F, typename PUT>
__device__ __forceinline__ void join_waves(F& f, int n, float* os, float (*top)[16], float (*sum)[16], PUT&& put) {
    constexpr int CT = F::CT, OLD = CT * 16 + 4;
    const int t = threadIdx.x, col = t % 16, quad = t % 64 / 16, wave = t / 64;
    __syncthreads();
    const float l = rows_sum(f.l[n]);
    if (quad == 0) top[wave][col] = f.m[n], sum[wave][col] = l;
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<v4f*>(os + (wave * 16 + col) * OLD + c * 16 + quad * 4) = f.o[n][c];
    __syncthreads();
    for (int x = t; x < 16 * (CT * 4); x += 64 * W) {
        const int r = x / (CT * 4), c = x % (CT * 4) * 4;
        float big = top[0][r];
#pragma unroll
        for (int w = 1; w < W; ++w) big = fmaxf(big, top[w][r]);
        v4f y = {0.f, 0.f, 0.f, 0.f};
        float z = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const float g = top[w][r] == -INFINITY ? 0.f * sum[w][r] : __builtin_amdgcn_exp2f(top[w][r] - big);   // a sum that is no number stays
            z += g * sum[w][r];
            y += g * *reinterpret_cast<const v4f*>(os + (w * 16 + r) * OLD + c);      // so does an infinite value, as none, where g is 0
        }
        put(r, c, y, big, z);
    }
}

// Where a workgroup's part of the line starts and ends, and the stream and the unit within its pairs that it starts at; false if the
// part is empty.  Workgroup 0 leaves the streams' places for the second kernel.
__device__ __forceinline__ bool place_part(const attend_args& a, int part, int* waves, int* where, int* at, int* end, int* b, int* offset, stream* s) {
    const int t = threadIdx.x, threads = blockDim.x;
    if (a.B <= 64) {
        // every wave by itself
        const int lane = t % 64;
        stream mine = {0, 0, 0, 0};
        if (lane < a.B) mine = stream_of(a, lane, blockIdx.x == 0 && t < 64);
        const int n = a.H * mine.units;
        int upto = n;
        for (int o = 1; o < 64; o <<= 1) {
            const int y = __shfl_up(upto, o);
            upto += lane >= o ? y : 0;
        }
        const int units = __builtin_amdgcn_readlane(upto, 63), quota = quota_of(a, units);
        if (blockIdx.x == 0) {
            if (t < a.B) a.starts[t] = upto - n;
            if (t == 0) a.starts[a.B] = units;
        }
        *at = part * quota;
        *end = min(*at + quota, units);
        if (*at >= *end || part >= a.parts) return false;
        *b = __popcll(__ballot(upto <= *at));          // streams that end before it
        *offset = *at - (__builtin_amdgcn_readlane(upto, *b) - __builtin_amdgcn_readlane(n, *b));
        s->len = __builtin_amdgcn_readlane(mine.len, *b);
        s->slots = __builtin_amdgcn_readlane(mine.slots, *b);
        s->drafted = __builtin_amdgcn_readlane(mine.drafted, *b);
        s->units = __builtin_amdgcn_readlane(mine.units, *b);
        return true;
    }
    int quota = 0;
    for (int pass = a.B <= threads; pass < 2; ++pass) {
        int before = 0, all;
        for (int base = 0; base < a.B; base += threads) {
            const int i = base + t;
            stream mine = {0, 0, 0, 0};
            if (i < a.B) mine = stream_of(a, i, blockIdx.x == 0);
            const int n = a.H * mine.units;
            const int start = before + block_before(n, waves, &all);
            before += all;
            if (pass == 0 || a.B <= threads) {
                const int units = uniform(before);
                quota = quota_of(a, units);
                *at = part * quota;
                *end = min(*at + quota, units);
            }
            if (pass) {
                if (start <= *at && *at < start + n) where[0] = i, where[1] = *at - start, where[2] = mine.len, where[3] = mine.slots, where[4] = mine.drafted, where[5] = mine.units;
                if (blockIdx.x == 0 && i < a.B) a.starts[i] = start;
            }
        }
        if (blockIdx.x == 0 && t == 0) a.starts[a.B] = before;
    }
    __syncthreads();
    if (*at >= *end || part >= a.parts) return false;
    *b = uniform(where[0]);
    *offset = uniform(where[1]);
    *s = {uniform(where[2]), uniform(where[3]), uniform(where[4]), uniform(where[5])};
    return true;
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

// Workgroup (part, tile of up to 32 rows): the part's keys, pair by pair, each wave 32 keys of a unit and all rows.  K and V go through
// registers into LDS, a tile ahead, by loads that leave no trace in the caches.  (64 streams of 517 to 8100 tokens, 8 heads of 128: 1.13 GB in 188 us, 6.0
// TB/s, of the 6.95 that a plain read reaches; with cached loads 8 us more, with three workgroups on a compute unit in place of two 40.)
template <bool BF16, int DP, int NR, bool FULL>
__global__ __launch_bounds__(256, DP > 128 ? 1 : 2) void attend_context_kernel(attend_args a) {
    constexpr int ROWS = 16 * NR;   // two terms of a weight: what bounds this one is memory
    typedef own_keys<BF16, DP, NR, 2, FULL> state;
    __shared__ __align__(16) unsigned char pool[4 * 32 * state::VLD * 2];
    __shared__ uint32_t listed[LISTED], held[LISTED / 32];
    __shared__ float top[4][16], sum[4][16];
    __shared__ int waves[4], where[6];
    static_assert(4 * 16 * (DP + 4) * 4 <= sizeof(pool), "the waves' parts of the result fit their rows of V");

    const int wave = uniform(threadIdx.x / 64);
    // workgroups of the same part and different tiles read the same keys: 8 apart, they run behind the same L2
    const int tile = (int)(blockIdx.x / 8) % a.tiles, part = (int)(blockIdx.x / 8) / a.tiles * 8 + (int)(blockIdx.x % 8);
    int at, end, b, offset;
    stream s;
    if (!place_part(a, part, waves, where, &at, &end, &b, &offset, &s)) return;
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
                auto row = [&](int key) { return mine[key]; };
                f.load(f.kr, kp, a.d, row);
                __builtin_amdgcn_sched_barrier(0);   // K's loads stay older than V's, as in the loop: whoever waits for K then need not wait for V
                f.load(f.vr, vp, a.d, row);
                for (int u = 0; u < n; ++u) {
                    const uint32_t there = (uint32_t)uniform((int)held[u * 4 + wave]);
                    const uint32_t* ahead = mine + min(u + 1, n - 1) * UNIT;
                    auto next = [&](int key) { return ahead[key]; };
                    f.put_k(vs, a.d);
                    wave_fence();
                    f.load(f.kr, kp, a.d, next);
                    f.template scores<state::KLD>(vs);
                    wave_fence();
                    f.put_v(vs, there);
                    wave_fence();
                    f.load(f.vr, vp, a.d, next);
                    f.weigh(a.scale_log2, &there, there == ~0u);
                    f.add(vs);
                    wave_fence();
                }
            }
            // along the line a step goes to the next pair or to the next part: their sum names what a part found for a pair
            const int64_t slot = (((int64_t)b * a.H + h + part) * a.tiles + tile) * ROWS;
#pragma unroll
            for (int r = 0; r < NR; ++r)
                join_waves<4>(f, r, reinterpret_cast<float*>(pool), top, sum, [&](int row, int c, v4f y, float big, float z) {
                    if (r * 16 + row >= rows || (!FULL && c >= a.d)) return;
                    *reinterpret_cast<v4f*>(a.part_o + (slot + r * 16 + row) * DP + c) = y;
                    if (c == 0) a.part_ml[(slot + r * 16 + row) * 2] = big, a.part_ml[(slot + r * 16 + row) * 2 + 1] = z;
                });
        }
        at += last - first;
        if (at >= end) break;
        first = 0;
        if (++h == a.H) {
            h = 0;
            do {
                if (++b >= a.B) return;
                s = stream_of(a, b, false);
            } while (s.units == 0);
        }
    }
}

// The same for many rows: W waves of NR * 16 share tiles of KT keys in LDS, K and V, two of them: while one is worked on, the next comes into
// registers, and from there into the other's place.  The vector units bound it (the exponentials and their sums, and the matrix cores' work on top), so a
// weight enters its product with v as one term of the cache's type: off by half a step at most, as the result is by its own rounding.  (Two terms: 131000
// tokens x 256 rows x 8 heads 243 us, one: 186.)
// Which form takes how many rows is measured.  Heads of 128 / 64, 96 pairs of 700 to 6000 tokens: 64 rows by four waves of 16 51 / 32 us, by two of 32
// 61 / 42; 96 rows by four of 32 66 / 43, by six of 16 78 / 44; 128 rows by four of 32 71 / 46, by eight of 16 81 / 48; 192 rows by twelve of 16 77 / 50,
// by six of 32 81 / 54.  8 pairs of 131000 tokens, heads of 128: 256 rows by eight of 32 215, by sixteen of 16 235.
template <bool BF16, int DP, int W, int NR, bool FULL>
__global__ __launch_bounds__(64 * W, DP > 128 ? (W == 4 ? 2 : 1) : W * (16 * NR * W <= 128 ? 2 : 1) / 4) void attend_wide_kernel(attend_args a) {
    constexpr int ROWS = 16 * NR * W, KT = DP > 128 ? 32 : 64, THREADS = 64 * W;
    typedef flash<BF16, DP, NR, KT, 1, FULL> state;
    constexpr int KLD = DP + 8, VLD = state::VLD;     // LDS rows: 16 rows' pieces of 16 bytes meet no bank twice
    constexpr int LPR = DP / 8, PIECES = KT * LPR, MINE = (PIECES + THREADS - 1) / THREADS;
    __shared__ __align__(16) uint16_t ks[2][KT * KLD], vs[2][KT * VLD];
    __shared__ uint32_t listed[LISTED], held[LISTED / 32];
    __shared__ int waves[W], where[6];

    const int t = threadIdx.x, lane = t % 64, col = lane % 16, quad = lane / 16, wave = uniform(t / 64);
    const int tile = (int)(blockIdx.x / 8) % a.tiles, part = (int)(blockIdx.x / 8) / a.tiles * 8 + (int)(blockIdx.x % 8);
    int at, end, b, offset;
    stream s;
    if (!place_part(a, part, waves, where, &at, &end, &b, &offset, &s)) return;
    int h = offset / s.units, first = offset % s.units;
    const v4i *kp = reinterpret_cast<const v4i*>(a.k), *vp = reinterpret_cast<const v4i*>(a.v);
    state f;
    v4i kr[MINE], vr[MINE];

    for (;;) {
        const int last = min(s.units, first + (end - at));
        const int rows = min(s.drafted * a.G - tile * ROWS, ROWS);   // query rows here
        if (rows > 0) {
            f.start(a, b, h, tile * ROWS + wave * NR * 16, s.drafted);
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
            for (int r = 0; r < NR; ++r) {
                const int row = (wave * NR + r) * 16 + col;
                const float l = rows_sum(f.l[r]);
                if (row < rows) {
#pragma unroll
                    for (int c = 0; c < state::CT; ++c)
                        if (FULL || c * 16 < a.d) *reinterpret_cast<v4f*>(a.part_o + (slot + row) * DP + c * 16 + quad * 4) = f.o[r][c];
                    if (quad == 0) a.part_ml[(slot + row) * 2] = f.m[r], a.part_ml[(slot + row) * 2 + 1] = l;
                }
            }
        }
        at += last - first;
        if (at >= end) break;
        first = 0;
        if (++h == a.H) {
            h = 0;
            do {
                if (++b >= a.B) return;
                s = stream_of(a, b, false);
            } while (s.units == 0);
        }
    }
}

// Workgroup (pair, 16 rows): the parts of the context, the drafted tokens, the end.  W waves share the parts and the drafted tokens: one
// where a pair has few parts, as many rows fill the device then, or eight (four for wide heads, for their registers) where it has many.  Latency bounds it:
// three trips to memory, the drafted tokens' products, the join.  Where that are few workgroups, two share the channels, each with all scores; with more they only
// do the scores twice.  Which form is measured, 8 heads of 128 x 4 query heads, the whole call by one wave / eight / eight in two shares, us:
//   workgroups  parts of a pair  (streams x tokens, context)
//   32          64               1 x 16, 8000     42.5 / 32.1 / 26.0
//   128         8                4 x 16, 1000     18.0 / 17.8 / 16.8
//   128         32               1 x 64, 8000     45.5 / 40.3 / 38.4
//   256         8                8 x 16, 8000     59.4 / 58.9 / 62.9
//   256         16               2 x 64, 8000     48.9 / 47.1 / 51.8
//   512         8                4 x 64, 8000     64.5 / 69.1 / 76.6
//   128         4                16 x 1, 8000     93.6 / 93.4 / 93.1
//   512         4                16 x 16, 8000    119 / 123 / 129
//   8           8                1 x 1, 1000      14.1 / 13.2 / 13.7
template <bool BF16, int DP, int W, int CS, bool FULL>
__global__ __launch_bounds__(64 * W, DP > 128 ? 1 : 2) void attend_finish_kernel(attend_args a) {
    typedef own_keys<BF16, DP, 1, 2, FULL, CS> state;
    constexpr uint32_t EXP = BF16 ? 0x7f80u : 0x7c00u;
    __shared__ __align__(16) unsigned char pool[W * 32 * state::VLD * 2];
    __shared__ float top[W][16], sum[W][16];
    const int t = threadIdx.x, lane = t % 64, wave = uniform(t / 64), col = lane % 16, quad = lane / 16;
    const int row0 = blockIdx.y * 16, h = blockIdx.x % a.H, b = blockIdx.x / a.H, c0 = CS > 1 ? blockIdx.z * state::CT * 16 : 0;   // the share's first channel
    const int units = a.starts[a.B], start = a.starts[b];
    const stream s = stream_of(a, b, blockIdx.y == 0 && h == 0 && c0 == 0);
    const int rows = min(s.drafted * a.G - row0, 16);
    if (rows <= 0) return;
    uint16_t* vs = reinterpret_cast<uint16_t*>(pool) + wave * 32 * state::VLD;
    const v4i *kp = reinterpret_cast<const v4i*>(a.k_new), *vp = reinterpret_cast<const v4i*>(a.v_new);
    int j0 = a.k_new ? wave * 32 : s.drafted;         // this wave's drafted tokens: j0 and the 31 behind it, then 32 W further on
    auto row = [&](int key) { return (((uint32_t)b * a.T + min(j0 + key, s.drafted - 1)) * a.H + h) * (uint32_t)(a.d / 8); };
    state f;
    f.start(a, b, h, row0, s.drafted);
    if (j0 < s.drafted) {
        f.load(f.kr, kp, a.d, row);                   // they come while the parts are joined
        f.load(f.vr, vp, a.d, row);
    }
    if (s.units > 0) {
        const int g = start + h * s.units, quota = quota_of(a, units), p0 = g / quota, p1 = min((g + s.units - 1) / quota, a.parts - 1);
        // this row in the tiles of the first kernel
        const int tile = row0 / a.rows, in = row0 % a.rows + min(col, rows - 1);
        auto slot = [&](int p) { return (((int64_t)b * a.H + h + p) * a.tiles + tile) * a.rows + in; };
        // Each wave every W-th part, two on their way at a time.  A part without keys left zeros.
        typedef float v2f __attribute__((ext_vector_type(2)));
        v4f x[2][state::CT];
        v2f ml[2];
        auto get = [&](int i, int p) {
            const int64_t at = slot(p);
            ml[i] = *reinterpret_cast<const v2f*>(a.part_ml + at * 2);
#pragma unroll
            for (int c = 0; c < state::CT; ++c) x[i][c] = FULL || c0 + c * 16 < a.d ? *reinterpret_cast<const v4f*>(a.part_o + at * DP + c0 + c * 16 + quad * 4) : v4f{0.f, 0.f, 0.f, 0.f};
        };
        auto join = [&](int i) {
            const float m = ml[i][0], z = ml[i][1], next = fmaxf(f.m[0], m);
            const float w = m == -INFINITY ? 0.f * z : __builtin_amdgcn_exp2f(m - next);   // a sum that is no number stays
            f.rescale(0, f.m[0] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(f.m[0] - next));
            f.m[0] = next;
            if (quad == 0) f.l[0] += w * z;
#pragma unroll
            for (int c = 0; c < state::CT; ++c) f.o[0][c] += w * x[i][c];
        };
        if (p0 + wave <= p1) get(0, p0 + wave);
        for (int p = p0 + wave; p <= p1; p += 2 * W) {
            if (p + W <= p1) get(1, p + W);
            join(0);
            if (p + W > p1) break;
            if (p + 2 * W <= p1) get(0, p + 2 * W);
            join(1);
        }
    }
    const int token = token_of(a, row0 + col);
    while (j0 < s.drafted) {
        const uint32_t there = s.drafted - j0 >= 32 ? ~0u : (1u << (s.drafted - j0)) - 1u;
        uint32_t word = 0;
        if (token < s.drafted) {
            if (a.mask) word = a.mask[((int64_t)b * a.T + token) * ((a.T + 31) / 32) + j0 / 32];
            else word = token - j0 >= 31 ? ~0u : token < j0 ? 0u : (2u << (token - j0)) - 1u;
        }
        // Not every row sees these: values that are not numbers stand apart.
        typedef uint16_t v2h __attribute__((ext_vector_type(2)));
        v2h largest = {0, 0};
#pragma unroll
        for (int j = 0; j < state::VI; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) largest = __builtin_elementwise_max(largest, __builtin_bit_cast(v2h, f.vr[j][e] & 0x7fff7fff));
        const bool odd = __any(largest[0] >= EXP || largest[1] >= EXP);
        if (odd) {
#pragma unroll
            for (int j = 0; j < state::VI; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = (uint32_t)f.vr[j][e];
                    f.vr[j][e] = (int)(x & ((x & EXP) == EXP ? 0xffff0000u : ~0u) & ((x & EXP << 16) == EXP << 16 ? 0xffffu : ~0u));
                }
        }
        f.put_k(vs, a.d);
        wave_fence();
        f.template scores<state::KLD>(vs);
        wave_fence();
        f.put_v(vs, there);
        wave_fence();
        const uint32_t sees = word & there;
        f.weigh(a.scale_log2, &sees, false);
        f.add(vs + c0);
        wave_fence();
        if (odd) {
            // One drafted token at a time: its values that are not numbers alone in LDS, and only the rows that see it take the product.
#pragma unroll 1
            for (int j = 0; j < 32; ++j) {
                if (!(there >> j & 1u)) continue;
                f.load(f.vr, vp, a.d, row);
#pragma unroll
                for (int i = 0; i < state::VI; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint32_t y = (uint32_t)f.vr[i][e];
                        f.vr[i][e] = (int)(((y & EXP) == EXP ? y & 0xffffu : 0u) | ((y & EXP << 16) == EXP << 16 ? y & 0xffff0000u : 0u));
                    }
                f.put_v(vs, 1u << j);
                wave_fence();
                v4i alone = {0, 0, 0, 0};
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (e / 4 * 16 + quad * 4 + e % 4 == j) alone[e / 2] = (int)((uint32_t)f.pf[0][0][0][e / 2] & (e % 2 ? 0xffff0000u : 0xffffu));
                const bool takes = sees >> j & 1u;
#pragma unroll
                for (int c = 0; c < state::CT; ++c) {
                    const v4f x = mfma<BF16>(f.get_v(vs + c0, c), alone, v4f{0.f, 0.f, 0.f, 0.f});
#pragma unroll
                    for (int r = 0; r < 4; ++r) f.o[0][c][r] += takes ? x[r] : 0.f;
                }
                wave_fence();
            }
        }
        j0 += 32 * W;
        if (j0 < s.drafted) {
            f.load(f.kr, kp, a.d, row);
            f.load(f.vr, vp, a.d, row);
        }
    }
    auto put = [&](int row, int c, v4f y, float m, float z) {
        if (row >= rows) return;
        const int i = token_of(a, row0 + row);
        const int64_t to = (((int64_t)b * a.T + i) * a.H + h) * a.G + (row0 + row - i * a.G);
        const bool some = z > 0.f || z != z;
        const float g = some ? 1.f / z : 0.f;
        if (!some) y = v4f{0.f, 0.f, 0.f, 0.f};       // scores of -inf alone, whatever the values were
        if (FULL || c0 + c < a.d) *reinterpret_cast<v2i*>(a.out + to * a.d + c0 + c) = v2i{pack<BF16>(y[0] * g, y[1] * g), pack<BF16>(y[2] * g, y[3] * g)};
        if (c0 + c == 0 && a.lse) a.lse[to] = some ? (m + log2f(z)) * 0.693147180559945309f : -INFINITY;
    };
    if constexpr (W == 1) {
        const float z = rows_sum(f.l[0]);
#pragma unroll
        for (int c = 0; c < state::CT; ++c) put(col, c * 16 + quad * 4, f.o[0][c], f.m[0], z);
    } else {
        join_waves<W>(f, 0, reinterpret_cast<float*>(pool), top, sum, put);
    }
}

template <bool BF16, int DP, bool FULL>
void launch_attend(const attend_args& a, hipStream_t stream) {
    const dim3 grid((unsigned)((a.parts + 7) / 8 * 8 * a.tiles)), block(256);
    if (a.rows == 16) hipLaunchKernelGGL((attend_context_kernel<BF16, DP, 1, FULL>), grid, block, 0, stream, a);
    else if constexpr (DP <= 128) {
        if (a.rows == 32) hipLaunchKernelGGL((attend_context_kernel<BF16, DP, 2, FULL>), grid, block, 0, stream, a);
        else if (a.rows == 64) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 4, 1, FULL>), grid, block, 0, stream, a);
        else if (a.rows == 128) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 4, 2, FULL>), grid, block, 0, stream, a);
        else if (a.rows == 192) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 12, 1, FULL>), grid, dim3(768), 0, stream, a);
        else hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 8, 2, FULL>), grid, dim3(512), 0, stream, a);
    } else {
        if (a.rows == 32) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 2, 1, FULL>), grid, dim3(128), 0, stream, a);
        else if (a.rows == 64) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 4, 1, FULL>), grid, block, 0, stream, a);
        else if (a.rows == 96) hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 6, 1, FULL>), grid, dim3(384), 0, stream, a);
        else hipLaunchKernelGGL((attend_wide_kernel<BF16, DP, 8, 1, FULL>), grid, dim3(512), 0, stream, a);
    }
    constexpr int MANY = DP > 128 ? 4 : 8;      // eight waves would leave wide heads too few registers
    const unsigned pairs = (unsigned)(a.B * a.H), rows = (unsigned)((a.T * a.G + 15) / 16);
    const int64_t groups = (int64_t)pairs * rows, each = (a.parts + (int64_t)pairs - 1) / pairs;   // parts of a pair
    if (a.T <= 64 && (each <= 4 || (each <= 8 && groups >= 512))) hipLaunchKernelGGL((attend_finish_kernel<BF16, DP, 1, 1, FULL>), dim3(pairs, rows), dim3(64), 0, stream, a);
    else if (groups > 128) hipLaunchKernelGGL((attend_finish_kernel<BF16, DP, MANY, 1, FULL>), dim3(pairs, rows), dim3(64 * MANY), 0, stream, a);
    else hipLaunchKernelGGL((attend_finish_kernel<BF16, DP, MANY, 2, FULL>), dim3(pairs, rows, 2), dim3(64 * MANY), 0, stream, a);
}

template <bool BF16, int DP>
void launch_width(const attend_args& a, hipStream_t stream) {
    a.d == DP ? launch_attend<BF16, DP, true>(a, stream) : launch_attend<BF16, DP, false>(a, stream);
}

template <bool BF16>
void launch_attend_type(const attend_args& a, hipStream_t stream) {
    const int DP = attend_width(a.d);
    if (DP == 64) launch_width<BF16, 64>(a, stream);
    else if (DP == 96) launch_width<BF16, 96>(a, stream);
    else if (DP == 128) launch_width<BF16, 128>(a, stream);
    else if (DP == 192) launch_width<BF16, 192>(a, stream);
    else launch_width<BF16, 256>(a, stream);
}

}  // namespace
