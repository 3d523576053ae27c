// Pages of a cache: forking rows (sharing, copying, freeing, reserving), appending tokens, compacting the pool.
#include "common.h"
#include "wave_ops.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));

// Sum over the lower threads of a workgroup of up to 16 waves, and over all of them; `waves` has room for one value per wave.
__device__ __forceinline__ int block_excl_scan(int v, int* waves, int* total) {
    uint32_t all;
    const int mine = (int)waveops::wave_excl_scan((uint32_t)v, &all), w = threadIdx.x / 64, n = blockDim.x / 64;
    __syncthreads();
    if (threadIdx.x % 64 == 0) waves[w] = (int)all;
    __syncthreads();
    int below = 0, sum = 0;
    for (int i = 0; i < n; ++i) {
        below += i < w ? waves[i] : 0;
        sum += waves[i];
    }
    *total = sum;
    return below + mine;
}

// ---- fork ---------------------------------------------------------------------------------------------------------------

struct fork_args {
    v4i *k, *v;                                  // the pool in pieces of 16 bytes
    const int32_t *table, *len, *refs, *parent, *room;
    int32_t *table_out, *len_out, *refs_out;
    int32_t *fresh, *start, *lens, *free_ids, *state;   // new pages of each row, where they start in free_ids, its length; state[0]: how many are free
    int32_t* copies;                             // [rows][3]: page that a row copies from and to (-1: none), tokens of it
    uint32_t* flags;
    int L, P, H, page, chunks, rows, cap;        // chunks of 16 bytes in a token of one head
};

__global__ void copy_words_kernel(const int32_t* src, int32_t* dst, int n) {
    for (int64_t i = blockIdx.x * (int64_t)blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) dst[i] = src[i];
}

// Leading slots of a row that hold pages of the pool, by a workgroup of 256.
__device__ int held_pages(const int32_t* row, int cap, int P, int* shared) {
    if (threadIdx.x == 0) *shared = cap;
    __syncthreads();
    for (int j = threadIdx.x; j < cap; j += blockDim.x)
        if (row[j] < 0 || row[j] >= P) {
            atomicMin(shared, j);
            break;
        }
    __syncthreads();
    const int held = *shared;
    __syncthreads();
    return held;
}

// What a row holds, cut to what its pages can hold.
__device__ int row_length(const fork_args& a, int row, int held) {
    const int64_t most = (int64_t)held * a.page;
    const int len = a.len[row];
    if (len < 0 || len > most) {
        if (threadIdx.x == 0) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        return len < 0 ? 0 : (int)most;
    }
    return len;
}

__device__ __forceinline__ int parent_of(const fork_args& a, int r) {
    const int p = a.parent[r];
    return p < -1 || p >= a.rows ? r : p;
}

__device__ int pages_needed(const fork_args& a, int len, int r) {
    const int64_t room = a.room ? max(a.room[r], 0) : 0, need = (len + room + a.page - 1) / a.page;
    return need > a.cap ? a.cap : (int)need;
}

// Workgroup r: counts what becomes of the pages of old row r, and lays new row r out up to its new pages.
__global__ __launch_bounds__(256) void fork_plan_kernel(fork_args a) {
    __shared__ int tmp, children, eldest, lead;
    const int r = blockIdx.x, t = threadIdx.x, p = parent_of(a, r);
    if (t == 0) children = 0, eldest = a.rows, lead = a.rows;
    __syncthreads();
    for (int c = t; c < a.rows; c += 256) {
        const int q = parent_of(a, c);
        if (q == r) atomicAdd(&children, 1), atomicMin(&eldest, c);
        if (q == p) atomicMin(&lead, c);
    }
    if (t == 0 && a.parent[r] != p) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
    __syncthreads();
    {
        const int32_t* old = a.table + (int64_t)r * a.cap;
        const int held = held_pages(old, a.cap, a.P, &tmp), len = row_length(a, r, held), full = len / a.page;
        const int kept = children ? min(held, pages_needed(a, len, eldest)) : 0;
        for (int j = t; j < a.cap; j += 256) {
            const int id = old[j];
            if (id < 0 || id >= a.P) {
                if (id != -1) atomicOr(a.flags, SWARM_DEV_BAD_PAGE);
                continue;
            }
            const int now = j < full ? children : j < kept ? 1 : 0;
            if (now != 1) atomicAdd(a.refs_out + id, now - 1);
        }
    }
    int32_t* out = a.table_out + (int64_t)r * a.cap;
    int kept = 0, need = 0, len = 0;
    if (p >= 0) {
        const int held = held_pages(a.table + (int64_t)p * a.cap, a.cap, a.P, &tmp);
        len = row_length(a, p, held);
        need = pages_needed(a, len, r);
        kept = lead == r ? min(held, need) : len / a.page;
        if (t == 0 && a.room && (int64_t)len + max(a.room[r], 0) > (int64_t)a.cap * a.page) atomicOr(a.flags, SWARM_DEV_NO_PAGE);
    }
    for (int j = t; j < a.cap; j += 256) out[j] = j < kept ? a.table[(int64_t)p * a.cap + j] : -1;
    if (t == 0) a.fresh[r] = need - kept, a.lens[r] = len;
}

// One workgroup: where each row's new pages start, and the lowest free ids for all of them.
__global__ __launch_bounds__(1024) void fork_scan_kernel(fork_args a) {
    __shared__ int waves[16];
    const int t = threadIdx.x;
    int want = 0, found = 0, sum;
    for (int base = 0; base < a.rows; base += 1024) {
        const int before = block_excl_scan(base + t < a.rows ? a.fresh[base + t] : 0, waves, &sum);
        if (base + t < a.rows) a.start[base + t] = want + before;
        want += sum;
    }
    for (int base = 0; base < a.P && found < want; base += 4096) {
        int n[4], mine = 0;
        for (int i = 0; i < 4; ++i) {
            const int id = base + 4 * t + i;
            n[i] = id < a.P && a.refs_out[id] == 0;
            mine += n[i];
        }
        int at = found + block_excl_scan(mine, waves, &sum);
        for (int i = 0; i < 4; ++i) {
            if (n[i] && at < want) a.free_ids[at] = base + 4 * t + i;
            at += n[i];
        }
        found += sum;
    }
    if (t == 0) a.state[0] = min(found, want);
}

// Workgroup r: row r's new pages, where there are any, its length and what it copies.
__global__ __launch_bounds__(256) void fork_fill_kernel(fork_args a) {
    const int r = blockIdx.x, t = threadIdx.x, p = parent_of(a, r);
    const int n = a.fresh[r], start = a.start[r], have = a.state[0], len = a.lens[r];
    const int kept = p < 0 ? 0 : pages_needed(a, len, r) - n, full = len / a.page, tail = len % a.page;
    int32_t* out = a.table_out + (int64_t)r * a.cap;
    for (int j = t; j < n; j += 256) {
        if (start + j < have) {
            const int id = a.free_ids[start + j];
            out[kept + j] = id;
            a.refs_out[id] = 1;
        } else {
            atomicOr(a.flags, SWARM_DEV_NO_PAGE);
        }
    }
    if (t == 0) {
        const bool copies = p >= 0 && tail > 0 && kept <= full, there = n > 0 && start < have;
        a.len_out[r] = copies && !there ? full * a.page : len;
        a.copies[3 * r] = copies && there ? a.table[(int64_t)p * a.cap + full] : -1;
        a.copies[3 * r + 1] = copies && there ? a.free_ids[start] : -1;
        a.copies[3 * r + 2] = tail;
    }
}

// The same in one workgroup, for tables of up to 4096 slots (16 waves' rows in pieces of 64, four a wave, so 64 rows at most) and pools that LDS holds: what bounds
// a small fork is launches and the trips to memory between them.  A wave has every 16th row, and holds its rows' slots in registers.  (4 rows of 64 slots:
// 7 us here, 20 by the four kernels; 256 rows of 128 slots, with more turns a wave: 100 here, 22 there.)
constexpr int ONE_SLOTS = 4, ONE_ROWS = 16 * ONE_SLOTS, ONE_PAGES = 8192;
__global__ __launch_bounds__(1024) void fork_one_kernel(fork_args a) {
    __shared__ int refs[ONE_PAGES], ids[ONE_PAGES];
    __shared__ int held[ONE_ROWS], kids[ONE_ROWS], eldest[ONE_ROWS], lens[ONE_ROWS], rooms[ONE_ROWS], parents[ONE_ROWS];
    __shared__ int old_kept[ONE_ROWS], old_full[ONE_ROWS], new_kept[ONE_ROWS], new_need[ONE_ROWS], start[ONE_ROWS], waves[16];
    const int t = threadIdx.x, lane = t % 64, wave = __builtin_amdgcn_readfirstlane(t / 64), pieces = (a.cap + 63) / 64;
    int slot[ONE_SLOTS];
    {
        int r = wave, c = 0;
#pragma unroll
        for (int q = 0; q < ONE_SLOTS; ++q) {
            slot[q] = r < a.rows && c * 64 + lane < a.cap ? a.table[(int64_t)r * a.cap + c * 64 + lane] : -1;
            if (++c == pieces) c = 0, r += 16;
        }
    }
    const int mine = t < a.rows ? parent_of(a, t) : -1, room = t < a.rows && a.room ? max(a.room[t], 0) : 0, had = t < a.rows ? a.len[t] : 0;
    if (t < a.rows && a.parent[t] != mine) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
    for (int i = t; i < a.P; i += 1024) refs[i] = a.refs[i];
    if (t < a.rows) {
        held[t] = a.cap;
        parents[t] = mine;
        rooms[t] = room;
        kids[t] = 0;
        eldest[t] = a.rows;
    }
    __syncthreads();
    if (mine >= 0) atomicAdd(&kids[mine], 1), atomicMin(&eldest[mine], t);
    {
        int r = wave, c = 0;
#pragma unroll
        for (int q = 0; q < ONE_SLOTS; ++q) {
            if (r < a.rows && c * 64 + lane < a.cap && (slot[q] < 0 || slot[q] >= a.P)) {
                if (slot[q] != -1) atomicOr(a.flags, SWARM_DEV_BAD_PAGE);
                atomicMin(&held[r], c * 64 + lane);
            }
            if (++c == pieces) c = 0, r += 16;
        }
    }
    __syncthreads();
    auto need_of = [&](int len, int more) {
        const int64_t n = ((int64_t)len + more + a.page - 1) / a.page;
        return n > a.cap ? a.cap : (int)n;
    };
    if (t < a.rows) {
        const int64_t most = (int64_t)held[t] * a.page;
        if (had < 0 || had > most) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        lens[t] = had < 0 ? 0 : had > most ? (int)most : had;
    }
    __syncthreads();
    // as a new row: pages that it needs and keeps; as an old one: full ones, which all its children share, and those that the eldest keeps
    const int len = mine >= 0 ? lens[mine] : 0, need = mine >= 0 ? need_of(len, room) : 0;
    const int kept = mine < 0 ? 0 : eldest[mine] == t ? min(held[mine], need) : len / a.page;
    if (mine >= 0 && (int64_t)len + room > (int64_t)a.cap * a.page) atomicOr(a.flags, SWARM_DEV_NO_PAGE);
    if (t < a.rows) {
        new_kept[t] = kept;
        new_need[t] = need;
        old_full[t] = lens[t] / a.page;
        old_kept[t] = kids[t] ? min(held[t], need_of(lens[t], rooms[eldest[t]])) : 0;
    }
    int want;
    const int before = block_excl_scan(t < a.rows ? need - kept : 0, waves, &want);
    if (t < a.rows) start[t] = before;
    __syncthreads();
    {
        int r = wave, c = 0;
#pragma unroll
        for (int q = 0; q < ONE_SLOTS; ++q) {
            const int j = c * 64 + lane;
            if (r < a.rows && j < a.cap && slot[q] >= 0 && slot[q] < a.P) {
                const int now = j < old_full[r] ? kids[r] : j < old_kept[r] ? 1 : 0;
                if (now != 1) atomicAdd(&refs[slot[q]], now - 1);
            }
            // in its place what the new row takes over
            const int p = r < a.rows ? parents[r] : -1;
            slot[q] = p >= 0 && j < new_kept[r] ? a.table[(int64_t)p * a.cap + j] : -1;
            if (++c == pieces) c = 0, r += 16;
        }
    }
    const int tail_page = mine >= 0 && len / a.page < a.cap ? a.table[(int64_t)mine * a.cap + len / a.page] : -1;
    __syncthreads();
    int found = 0;
    for (int at = 0; at < a.P && found < want; at += 1024) {
        int n;
        const bool is_free = at + t < a.P && refs[at + t] == 0;
        const int place = found + block_excl_scan(is_free, waves, &n);
        if (is_free && place < want) ids[place] = at + t;
        found += n;
    }
    const int have = min(found, want);
    __syncthreads();
    {
        int r = wave, c = 0;
#pragma unroll
        for (int q = 0; q < ONE_SLOTS; ++q) {
            const int j = c * 64 + lane;
            if (r < a.rows && j < a.cap) {
                const int keep = new_kept[r];
                if (j >= keep && j < new_need[r]) {
                    if (start[r] + j - keep < have) {
                        slot[q] = ids[start[r] + j - keep];
                        refs[slot[q]] = 1;
                    } else {
                        atomicOr(a.flags, SWARM_DEV_NO_PAGE);
                    }
                }
                a.table_out[(int64_t)r * a.cap + j] = slot[q];
            }
            if (++c == pieces) c = 0, r += 16;
        }
    }
    if (t < a.rows) {
        const int full = len / a.page, tail = len % a.page;
        const bool copies = mine >= 0 && tail > 0 && kept <= full, there = need > kept && start[t] < have;
        a.len_out[t] = copies && !there ? full * a.page : len;
        a.copies[3 * t] = copies && there ? tail_page : -1;
        a.copies[3 * t + 1] = copies && there ? ids[start[t]] : -1;
        a.copies[3 * t + 2] = tail;
    }
    __syncthreads();
    for (int i = t; i < a.P; i += 1024) a.refs_out[i] = refs[i];
}

// Workgroups (r, y): the tokens that row r copies, layers and heads divided over y.
__global__ __launch_bounds__(256) void fork_copy_kernel(fork_args a) {
    const int r = blockIdx.x, src = a.copies[3 * r], dst = a.copies[3 * r + 1], piece = a.copies[3 * r + 2] * a.chunks;
    if (src < 0) return;
    for (int64_t part = blockIdx.y; part < (int64_t)a.L * a.H * 2; part += gridDim.y) {
        v4i* pool = part & 1 ? a.v : a.k;
        const int64_t l = part / 2 / a.H, h = part / 2 % a.H;
        const int64_t from = ((l * a.P + src) * a.H + h) * a.page * a.chunks, to = ((l * a.P + dst) * a.H + h) * a.page * a.chunks;
        for (int i = threadIdx.x; i < piece; i += 256) pool[to + i] = pool[from + i];
    }
}

// ---- append -------------------------------------------------------------------------------------------------------------

struct append_args {
    v4i *k, *v;
    const v4i *k_new, *v_new;
    const int32_t *table, *len, *path, *n;
    int32_t* len_out;
    uint32_t* flags;
    int L, P, H, page, chunks, rows, cap, B, T, n_max;
};

// Workgroups (b, y): what row b takes, the (layer, token) pairs divided over y.
__global__ __launch_bounds__(256) void append_kernel(append_args a) {
    __shared__ int stop;
    const int b = blockIdx.x, t = threadIdx.x;
    const int64_t most = (int64_t)a.cap * a.page;
    int len = a.len[b];
    if (b >= a.B) {
        if (blockIdx.y == 0 && t == 0) a.len_out[b] = len;
        return;
    }
    int n = a.n ? a.n[b] : a.n_max;
    if (len < 0 || len > most || n < 0 || n > a.n_max) {
        if (t == 0) atomicOr(a.flags, SWARM_DEV_BAD_LEN);
        len = len < 0 ? 0 : len > most ? (int)most : len;
        n = min(max(n, 0), a.n_max);
    }
    const int32_t* row = a.table + (int64_t)b * a.cap;
    // the first slot without a page ends what the row can take
    const int first = len / a.page;
    const int64_t last = ((int64_t)len + n + a.page - 1) / a.page;
    if (t == 0) stop = (int)(last < a.cap ? last : a.cap);
    __syncthreads();
    for (int j = first + t; j < last && j < a.cap; j += 256)
        if (row[j] < 0 || row[j] >= a.P) {
            atomicMin(&stop, j);
            break;
        }
    __syncthreads();
    const int64_t room = max((int64_t)stop * a.page - len, (int64_t)0);
    if (n > room) {
        if (t == 0) atomicOr(a.flags, SWARM_DEV_NO_PAGE);
        n = (int)room;
    }
    if (blockIdx.y == 0 && t == 0) a.len_out[b] = len + n;
    const int piece = a.H * a.chunks;
    for (int64_t part = blockIdx.y; part < (int64_t)a.L * n; part += gridDim.y) {
        const int64_t l = part / n;
        const int i = (int)(part % n), pos = len + i, src = a.path ? a.path[(int64_t)b * a.n_max + i] : i;
        if (src < 0 || src >= a.T) {
            if (t == 0) atomicOr(a.flags, SWARM_DEV_BAD_ENTRY);
            continue;
        }
        const int64_t from = ((l * a.B + b) * a.T + src) * piece;
        const int64_t to = ((l * a.P + row[pos / a.page]) * a.H * a.page + pos % a.page) * a.chunks;
        for (int x = t; x < 2 * piece; x += 256) {
            const int y = x < piece ? x : x - piece, h = y / a.chunks, c = y % a.chunks;
            const int64_t at = to + (int64_t)h * a.page * a.chunks + c;
            if (x < piece) a.k[at] = a.k_new[from + y];
            else a.v[at] = a.v_new[from + y];
        }
    }
}

// ---- compact ------------------------------------------------------------------------------------------------------------

struct compact_args {
    v4i *k, *v;
    const int32_t *table, *refs;
    int32_t *table_out, *refs_out, *live;
    int32_t *below, *src, *dst, *state;          // pages in use below each id; those in use by that number; the free ids; state[0]: how many move
    int L, P, H, page, chunks, rows, cap;
};

// One workgroup.  With n pages in use and m of them at n or higher, the r-th that moves is src[n - m + r], and goes to dst[r].
__global__ __launch_bounds__(1024) void compact_scan_kernel(compact_args a) {
    __shared__ int waves[16];
    const int t = threadIdx.x;
    int live = 0, used = 0, sum;
    for (int i = t; i < a.P; i += 1024) live += a.refs[i] > 0;
    block_excl_scan(live, waves, &sum);
    live = sum;
    if (t == 0) a.live[0] = live, a.state[0] = 0;
    __syncthreads();
    for (int base = 0; base < a.P; base += 4096) {
        int u[4], mine = 0;
        for (int i = 0; i < 4; ++i) {
            const int id = base + 4 * t + i;
            u[i] = id < a.P && a.refs[id] > 0;
            mine += u[i];
        }
        int before = used + block_excl_scan(mine, waves, &sum);
        for (int i = 0; i < 4; ++i) {
            const int id = base + 4 * t + i;
            if (id < a.P) {
                a.below[id] = before;
                if (u[i]) a.src[before] = id;
                else a.dst[id - before] = id;
                if (id == live) a.state[0] = live - before;
            }
            before += u[i];
        }
        used += sum;
    }
}

__global__ __launch_bounds__(256) void compact_move_kernel(compact_args a) {
    const int n = a.live[0], m = a.state[0];
    const int64_t piece = (int64_t)a.H * a.page * a.chunks, step = (int64_t)gridDim.x * 256, me = blockIdx.x * (int64_t)256 + threadIdx.x;
    for (int64_t i = me; i < a.P; i += step) {
        const int r = a.refs[i];
        a.refs_out[i] = i >= n ? 0 : r > 0 ? r : a.refs[a.src[n - m + (i - a.below[i])]];
    }
    for (int64_t i = me; i < (int64_t)a.rows * a.cap; i += step) {
        const int id = a.table[i];
        a.table_out[i] = id >= n && id < a.P && a.refs[id] > 0 ? a.dst[a.below[id] - (n - m)] : id;
    }
    for (int64_t part = blockIdx.x; part < (int64_t)m * a.L * 2; part += gridDim.x) {
        v4i* pool = part & 1 ? a.v : a.k;
        const int64_t l = part / 2 % a.L;
        const int64_t r = part / 2 / a.L;
        const v4i* from = pool + (l * a.P + a.src[n - m + r]) * piece;
        v4i* to = pool + (l * a.P + a.dst[r]) * piece;
        for (int64_t i = threadIdx.x; i < piece; i += 256) to[i] = from[i];
    }
}

}  // namespace

swarm_status swarm_check_cache(swarm_ctx* ctx, const char* fn, const swarm_cache* c) {
    if (!c || !c->k || !c->v || !c->table || !c->len) SWARM_REJECT(ctx, "%s: NULL cache, k, v, table or len", fn);
    if (c->dtype != SWARM_BF16 && c->dtype != SWARM_FP16) SWARM_REJECT(ctx, "%s: cache type %d is neither bf16 nor fp16", fn, c->dtype);
    if (c->L < 1 || c->P < 1 || c->H < 1 || c->rows < 1 || c->cap < 1)
        SWARM_REJECT(ctx, "%s: L=%d P=%d H=%d rows=%d cap=%d must all be >= 1", fn, c->L, c->P, c->H, c->rows, c->cap);
    if (c->page < 1 || c->page > 256 || (c->page & (c->page - 1))) SWARM_REJECT(ctx, "%s: page=%d must be a power of two in [1,256]", fn, c->page);
    if (c->d < 8 || c->d % 8 != 0 || c->d > 256) SWARM_REJECT(ctx, "%s: d=%d must be a multiple of 8 in [8,256]", fn, c->d);
    if (c->L > 65535 || c->H > 65535 || c->rows > 65535 || c->P > (1 << 26)) SWARM_REJECT(ctx, "%s: L, H or rows above 65535, or P above 2^26", fn);
    if ((int64_t)c->cap * c->page > (1 << 30) || (int64_t)c->rows * c->cap > (1 << 28))
        SWARM_REJECT(ctx, "%s: cap*page above 2^30 or rows*cap above 2^28", fn);
    if ((int64_t)c->H * c->page * c->d > (1 << 28)) SWARM_REJECT(ctx, "%s: H*page*d above 2^28", fn);
    if (swarm_misaligned(c->k, 16) || swarm_misaligned(c->v, 16)) SWARM_REJECT(ctx, "%s: k and v must be 16-byte aligned", fn);
    if (swarm_misaligned(c->table, 4) || swarm_misaligned(c->len, 4) || swarm_misaligned(c->refs, 4))
        SWARM_REJECT(ctx, "%s: table, len and refs must be 4-byte aligned", fn);
    return SWARM_OK;
}

bool swarm_overlap(const swarm_range* outs, int n_outs, const swarm_range* ins, int n_ins) {
    const auto meet = [](const swarm_range& x, const swarm_range& y) {
        if (!x.at || !y.at || !x.bytes || !y.bytes) return false;
        const uintptr_t a = reinterpret_cast<uintptr_t>(x.at), b = reinterpret_cast<uintptr_t>(y.at);
        return a < b + y.bytes && b < a + x.bytes;
    };
    for (int i = 0; i < n_outs; ++i) {
        for (int j = 0; j < n_ins; ++j)
            if (meet(outs[i], ins[j])) return true;
        for (int j = 0; j < i; ++j)
            if (meet(outs[i], outs[j])) return true;
    }
    return false;
}

// What a caller's own graph refers to is kept when later calls outgrow it.
swarm_status swarm_scratch(swarm_ctx* ctx, void** buf, size_t* have, size_t bytes) {
    if (swarm_capturing(ctx)) {
        if (*have < bytes) SWARM_REJECT(ctx, "scratch must grow to %zu bytes while the stream is captured; run the call once first", bytes);
        ctx->recorded = true;
        return SWARM_OK;
    }
    return swarm_grow(ctx, buf, have, bytes);
}

static void cache_ranges(const swarm_cache* c, swarm_range out[5]) {
    const size_t pool = 2 * (size_t)c->d * c->L * c->P * c->H * c->page;
    out[0] = {c->k, pool};
    out[1] = {c->v, pool};
    out[2] = {c->table, 4 * (size_t)c->rows * c->cap};
    out[3] = {c->len, 4 * (size_t)c->rows};
    out[4] = {c->refs, 4 * (size_t)c->P};
}

extern "C" {

swarm_status swarm_cache_fork(swarm_ctx* ctx, const swarm_cache* c, const int32_t* parent, const int32_t* room, int32_t* table_out,
                              int32_t* len_out, int32_t* refs_out) {
    SWARM_ENTER(ctx);
    swarm_status st = swarm_check_cache(ctx, "cache_fork", c);
    if (st != SWARM_OK) return st;
    if (!c->refs || !parent || !table_out || !len_out || !refs_out) SWARM_REJECT(ctx, "cache_fork: NULL refs, parent or output");
    if (c->rows > 16384) SWARM_REJECT(ctx, "cache_fork: rows=%d above 16384", c->rows);
    if (swarm_misaligned(parent, 4) || swarm_misaligned(room, 4) || swarm_misaligned(table_out, 4) || swarm_misaligned(len_out, 4) || swarm_misaligned(refs_out, 4))
        SWARM_REJECT(ctx, "cache_fork: integer arrays must be 4-byte aligned");
    swarm_range ins[7] = {};
    cache_ranges(c, ins);
    ins[5] = {parent, 4 * (size_t)c->rows};
    ins[6] = {room, 4 * (size_t)c->rows};
    const swarm_range outs[] = {{table_out, ins[2].bytes}, {len_out, ins[3].bytes}, {refs_out, ins[4].bytes}};
    if (swarm_overlap(outs, 3, ins, 7)) SWARM_REJECT(ctx, "cache_fork: an output overlaps an input, or another output");

    // new pages of each row, their starts, lengths and copies, the ids for all new pages (no more than there are pages), one count
    st = swarm_scratch(ctx, &ctx->pages, &ctx->pages_bytes, 4 * (6 * (size_t)c->rows + c->P + 4));
    if (st != SWARM_OK) return st;
    fork_args a{};
    a.k = static_cast<v4i*>(c->k);
    a.v = static_cast<v4i*>(c->v);
    a.table = c->table, a.len = c->len, a.refs = c->refs, a.parent = parent, a.room = room;
    a.table_out = table_out, a.len_out = len_out, a.refs_out = refs_out;
    a.state = static_cast<int32_t*>(ctx->pages);
    a.fresh = a.state + 4;
    a.start = a.fresh + c->rows;
    a.lens = a.start + c->rows;
    a.copies = a.lens + c->rows;
    a.free_ids = a.copies + 3 * (size_t)c->rows;
    a.flags = ctx->dev_flags;
    a.L = c->L, a.P = c->P, a.H = c->H, a.page = c->page, a.chunks = c->d / 8, a.rows = c->rows, a.cap = c->cap;
    const int turns = (c->rows + 15) / 16 * ((c->cap + 63) / 64);       // slots of a lane where one workgroup has all rows
    if (c->P <= ONE_PAGES && turns <= ONE_SLOTS) {
        hipLaunchKernelGGL(fork_one_kernel, dim3(1), dim3(1024), 0, ctx->stream, a);
    } else {
        hipLaunchKernelGGL(copy_words_kernel, dim3((unsigned)((c->P + 255) / 256 < 1024 ? (c->P + 255) / 256 : 1024)), dim3(256), 0, ctx->stream, c->refs, refs_out, c->P);
        hipLaunchKernelGGL(fork_plan_kernel, dim3((unsigned)c->rows), dim3(256), 0, ctx->stream, a);
        hipLaunchKernelGGL(fork_scan_kernel, dim3(1), dim3(1024), 0, ctx->stream, a);
        hipLaunchKernelGGL(fork_fill_kernel, dim3((unsigned)c->rows), dim3(256), 0, ctx->stream, a);
    }
    const int64_t parts = (int64_t)2 * c->L * c->H;
    hipLaunchKernelGGL(fork_copy_kernel, dim3((unsigned)c->rows, (unsigned)(parts < 64 ? parts : 64)), dim3(256), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "cache_fork");
}

swarm_status swarm_cache_append(swarm_ctx* ctx, const swarm_cache* c, const void* k_new, const void* v_new, int32_t B, int32_t T,
                                const int32_t* path, int32_t n_max, const int32_t* n, int32_t* len_out) {
    SWARM_ENTER(ctx);
    const swarm_status st = swarm_check_cache(ctx, "cache_append", c);
    if (st != SWARM_OK) return st;
    if (!k_new || !v_new || !len_out) SWARM_REJECT(ctx, "cache_append: NULL k_new, v_new or len_out");
    if (B < 1 || B > c->rows) SWARM_REJECT(ctx, "cache_append: B=%d outside [1,rows=%d]", B, c->rows);
    if (T < 1 || T > (1 << 20)) SWARM_REJECT(ctx, "cache_append: T=%d outside [1,2^20]", T);
    if (!path) n_max = T;
    if (n_max < 1 || n_max > (1 << 20)) SWARM_REJECT(ctx, "cache_append: n_max=%d outside [1,2^20]", n_max);
    if (swarm_misaligned(k_new, 16) || swarm_misaligned(v_new, 16)) SWARM_REJECT(ctx, "cache_append: k_new and v_new must be 16-byte aligned");
    if (swarm_misaligned(path, 4) || swarm_misaligned(n, 4) || swarm_misaligned(len_out, 4)) SWARM_REJECT(ctx, "cache_append: integer arrays must be 4-byte aligned");
    swarm_range ins[7] = {};
    cache_ranges(c, ins);
    const size_t news = 2 * (size_t)c->d * c->H * c->L * B * T;
    const swarm_range given[] = {{k_new, news}, {v_new, news}, {path, 4 * (size_t)B * n_max}, {n, 4 * (size_t)B}};
    const swarm_range outs[] = {{len_out, 4 * (size_t)c->rows}, ins[0], ins[1]};
    if (swarm_overlap(outs, 3, given, 4) || swarm_overlap(outs, 1, ins, 5)) SWARM_REJECT(ctx, "cache_append: len_out or the pool overlaps an input");

    append_args a{};
    a.k = static_cast<v4i*>(c->k);
    a.v = static_cast<v4i*>(c->v);
    a.k_new = static_cast<const v4i*>(k_new);
    a.v_new = static_cast<const v4i*>(v_new);
    a.table = c->table, a.len = c->len, a.path = path, a.n = n, a.len_out = len_out;
    a.flags = ctx->dev_flags;
    a.L = c->L, a.P = c->P, a.H = c->H, a.page = c->page, a.chunks = c->d / 8, a.rows = c->rows, a.cap = c->cap;
    a.B = B, a.T = T, a.n_max = n_max;
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)c->rows, 64), dim3(256), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "append_kernel");
}

swarm_status swarm_cache_compact(swarm_ctx* ctx, const swarm_cache* c, int32_t* table_out, int32_t* refs_out, int32_t* live) {
    SWARM_ENTER(ctx);
    swarm_status st = swarm_check_cache(ctx, "cache_compact", c);
    if (st != SWARM_OK) return st;
    if (!c->refs || !table_out || !refs_out || !live) SWARM_REJECT(ctx, "cache_compact: NULL refs or output");
    if (swarm_misaligned(table_out, 4) || swarm_misaligned(refs_out, 4) || swarm_misaligned(live, 4))
        SWARM_REJECT(ctx, "cache_compact: integer arrays must be 4-byte aligned");
    swarm_range ins[5] = {};
    cache_ranges(c, ins);
    const swarm_range outs[] = {{table_out, ins[2].bytes}, {refs_out, ins[4].bytes}, {live, 4}};
    if (swarm_overlap(outs, 3, ins, 5)) SWARM_REJECT(ctx, "cache_compact: an output overlaps an input, or another output");
    st = swarm_scratch(ctx, &ctx->pages, &ctx->pages_bytes, 4 * (3 * (size_t)c->P + 4));
    if (st != SWARM_OK) return st;
    compact_args a{};
    a.k = static_cast<v4i*>(c->k);
    a.v = static_cast<v4i*>(c->v);
    a.table = c->table, a.refs = c->refs;
    a.table_out = table_out, a.refs_out = refs_out, a.live = live;
    a.state = static_cast<int32_t*>(ctx->pages);
    a.below = a.state + 4;
    a.src = a.below + c->P;
    a.dst = a.src + c->P;
    a.L = c->L, a.P = c->P, a.H = c->H, a.page = c->page, a.chunks = c->d / 8, a.rows = c->rows, a.cap = c->cap;
    hipLaunchKernelGGL(compact_scan_kernel, dim3(1), dim3(1024), 0, ctx->stream, a);
    hipLaunchKernelGGL(compact_move_kernel, dim3(2048), dim3(256), 0, ctx->stream, a);
    return swarm_check_launch(ctx, "cache_compact");
}

}  // extern "C"
