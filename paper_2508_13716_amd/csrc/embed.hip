// Rows of a learnt table, out[i] = scale * table[ids[i]], and their gradient, dtable[v] = scale * sum over i with ids[i] = v of dY[i].
//
// Both move memory and compute next to nothing.  The gradient's sums have to be the same every time, so no float is added atomically:
// positions are sorted by id (a stable radix sort of our own), and teams of lanes, 16 bytes of a row each, walk tiles of the sorted list
// and sum runs of equal ids in registers.  A run inside a tile goes straight to the table; one that crosses tiles leaves a part per tile,
// added in their order by a team, a wave or a workgroup.  Rows that no id names are zeroed first; that is shared out over the sort's launches,
// which wait for memory more than they use it.
// us: 300001 bf16 rows of 256 into 500009 fp32 ones (0.67 GB) 212, of them 118 for six launches that sort and zero 512 MB (the zeros shared out
// over four of them; over all six 123: the moves have room for three workgroups a compute unit), 82 for the sums (rows of 512 bytes
// from everywhere), 17 for the joins; 64 rows of 1024 looked up 3.2.
#include "rows.h"
#include "grid.h"

#include <algorithm>
#include <type_traits>

namespace capgnn {

// ------------------------------------------------------------------ lookup
struct EmbedArgs {
    int64_t n, V;
    int F, lanes;
    const int64_t *ids;
    const char *table;
    int64_t ldt, ldo;           // in bytes
    float scale;
    char *out;
    int out_bf16;
};

template <bool BF16, int V> __global__ __launch_bounds__(256) void embed_kernel(EmbedArgs a) {
    const int lane = threadIdx.x & (a.lanes - 1), teams = 256 / a.lanes;
    for (int64_t row = int64_t(blockIdx.x) * teams + threadIdx.x / a.lanes; row < a.n; row += int64_t(gridDim.x) * teams) {
        const int64_t id = a.ids[row];
        const bool inside = id >= 0 && id < a.V;
        const char *src = a.table + (inside ? id : 0) * a.ldt;
        char *dst = a.out + row * a.ldo;
        for (int j = lane * V; j < a.F; j += a.lanes * V) {
            const int from = min(j, a.F - V);           // (the last vector of a row may repeat elements of the one before)
            float v[V];
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] = 0.f;
            if (inside) {
                ld_row<BF16, V>(src, from, v);
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] *= a.scale;
            }
            st_row_of<V>(a.out_bf16, dst, from, v);
        }
    }
}

// ------------------------------------------------------------------ zeros, in `parts` shares
struct Fill {
    float *p;
    int64_t rows, ld;           // p null: nothing to do
    int F, part, parts;
};
// by `groups` workgroups of which the caller is number `group`
__device__ __forceinline__ void fill_share(const Fill &f, int64_t group, int64_t groups) {
    const int64_t threads = groups * blockDim.x, t = group * blockDim.x + threadIdx.x;
    const float zero[4] = {0.f, 0.f, 0.f, 0.f};
    if (f.ld == f.F || f.rows == 1) {
        const int64_t all = f.rows * f.F, first = all / f.parts * f.part, end = f.part + 1 == f.parts ? all : all / f.parts * (f.part + 1);
        char *p = reinterpret_cast<char *>(f.p + first);
        int64_t i = t * 4;
        for (; i + 4 <= end - first; i += threads * 4) st_vector<false, 4>(p + i * 4, 0, zero);
        for (; i < end - first; i = (i & ~int64_t(3)) + threads * 4)
            for (int64_t k = i; k < end - first; ++k) f.p[first + k] = 0.f;
        return;
    }
    const int64_t first = f.rows / f.parts * f.part, end = f.part + 1 == f.parts ? f.rows : f.rows / f.parts * (f.part + 1);
    int lanes = 1;
    while (lanes < 64 && lanes * 4 < f.F) lanes *= 2;
    const int lane = threadIdx.x & (lanes - 1);
    for (int64_t row = first + t / lanes; row < end; row += threads / lanes) {
        char *p = reinterpret_cast<char *>(f.p + row * f.ld);
        if (f.F < 4) {
            if (lane == 0)
                for (int k = 0; k < f.F; ++k) f.p[row * f.ld + k] = 0.f;
        } else {
            for (int j = lane * 4; j < f.F; j += lanes * 4) st_vector<false, 4>(p, min(j, f.F - 4), zero);
        }
    }
}

// ------------------------------------------------------------------ positions by id
// Keys are ids in 32 bits, V for an id outside the table (the last ones then, and no run of theirs is summed).  A pass sorts by `bits` bits of
// the key from `shift` on, keeping the order of equal digits: counts of every digit per tile, their prefix along the tiles (a wave per
// digit), and the move.
constexpr int SORT_THREADS = 256, SORT_WAVES = SORT_THREADS / 64, SORT_ITEMS = 4, SORT_TILE = SORT_THREADS * SORT_ITEMS;
constexpr int SORT_BITS = 11;               // of a digit, at most
constexpr int SMALL_THREADS = 1024, SMALL_WAVES = SMALL_THREADS / 64, SMALL_ITEMS = 8, SMALL_TILE = SMALL_THREADS * SMALL_ITEMS, SMALL_BITS = 8, SMALL_COUNT = 128;

struct SortPass {
    int64_t n;
    const int64_t *ids;         // first pass: the ids themselves, else null
    uint32_t V;
    const uint32_t *key, *pos;
    uint32_t *key_out, *pos_out;
    uint32_t *count;            // [digits][tiles]
    uint32_t *total;            // [digits]
    int shift, bits;
    unsigned tiles;
    Fill fill;
};

__device__ __forceinline__ uint32_t sort_key(const SortPass &s, int64_t i) {
    if (!s.ids) return s.key[i];
    const int64_t id = s.ids[i];
    return id >= 0 && id < s.V ? static_cast<uint32_t>(id) : s.V;
}

__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortPass s) {
    __shared__ uint32_t count[1 << SORT_BITS];
    if (blockIdx.x >= s.tiles) return fill_share(s.fill, blockIdx.x - s.tiles, gridDim.x - s.tiles);
    const int digits = 1 << s.bits;
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) count[d] = 0;
    __syncthreads();
    const int64_t first = int64_t(blockIdx.x) * SORT_TILE;
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const int64_t k = first + i * SORT_THREADS + threadIdx.x;
        if (k < s.n) atomicAdd(&count[(sort_key(s, k) >> s.shift) & (digits - 1)], 1u);     // (integers: any order gives the same)
    }
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += SORT_THREADS) s.count[int64_t(d) * s.tiles + blockIdx.x] = count[d];
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {          // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        const uint32_t u = static_cast<uint32_t>(__shfl_up(static_cast<int>(v), o));
        if (lane >= o) v += u;
    }
    return v;
}

__global__ __launch_bounds__(SORT_THREADS) void sort_prefix_kernel(SortPass s) {
    const unsigned groups = ((1u << s.bits) + SORT_WAVES - 1) / SORT_WAVES;
    if (blockIdx.x >= groups) return fill_share(s.fill, blockIdx.x - groups, gridDim.x - groups);
    const unsigned d = blockIdx.x * SORT_WAVES + threadIdx.x / 64;
    if (d >= 1u << s.bits) return;
    uint32_t *c = s.count + int64_t(d) * s.tiles;
    uint32_t before = 0;
    for (unsigned t0 = 0; t0 < s.tiles; t0 += 64) {
        const unsigned t = t0 + (threadIdx.x & 63);
        const uint32_t v = t < s.tiles ? c[t] : 0u, upto = wave_scan(v);
        if (t < s.tiles) c[t] = before + upto - v;
        before += static_cast<uint32_t>(__shfl(static_cast<int>(upto), 63));
    }
    if ((threadIdx.x & 63) == 0) s.total[d] = before;
}

// For a wave's 64 items: how many of the lanes before this one have its digit, and how many lanes have it
__device__ __forceinline__ void same_digit(uint32_t digit, bool on, int bits, int *before, int *all) {
    uint64_t mask = __ballot(on);
    for (int b = 0; b < bits; ++b) {
        const uint64_t m = __ballot((digit >> b) & 1u);
        mask &= (digit >> b) & 1u ? m : ~m;
    }
    const uint64_t lower = (uint64_t(1) << (threadIdx.x & 63)) - 1;
    *before = __popcll(mask & lower);
    *all = __popcll(mask);
}

// Ranks of a wave's items among its own of the same digit; count[digit] (the wave's, zero before) is their number afterwards.
template <int ITEMS>
__device__ __forceinline__ void rank_items(const uint32_t (&key)[ITEMS], const bool (&on)[ITEMS], int shift, int bits, volatile uint32_t *count,
                                           uint32_t (&rank)[ITEMS]) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
        const uint32_t digit = (key[i] >> shift) & ((1u << bits) - 1);
        int before, all;
        same_digit(digit, on[i], bits, &before, &all);
        rank[i] = 0;
        if (on[i]) {
            const uint32_t base = count[digit];
            rank[i] = base + before;
            __builtin_amdgcn_wave_barrier();
            if (before == 0) count[digit] = base + all;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// exclusive prefix over the digits, in place, by a workgroup of W waves; sum[] is scratch of W entries
template <int W> __device__ __forceinline__ void digit_scan(uint32_t *v, int digits, uint32_t *sum) {
    constexpr int T = W * 64;
    const int each = (digits + T - 1) / T, first = threadIdx.x * each;
    uint32_t mine = 0;
    for (int k = 0; k < each; ++k) mine += first + k < digits ? v[first + k] : 0u;
    const uint32_t upto = wave_scan(mine);
    if ((threadIdx.x & 63) == 63) sum[threadIdx.x / 64] = upto;
    __syncthreads();
    uint32_t at = upto - mine;
    for (int w = 0; w < static_cast<int>(threadIdx.x / 64); ++w) at += sum[w];
    for (int k = 0; k < each; ++k)
        if (first + k < digits) {
            const uint32_t x = v[first + k];
            v[first + k] = at;
            at += x;
        }
    __syncthreads();
}

__global__ __launch_bounds__(SORT_THREADS) void sort_move_kernel(SortPass s) {
    __shared__ uint32_t count[SORT_WAVES][1 << SORT_BITS], start[1 << SORT_BITS], sum[SORT_WAVES];
    const int digits = 1 << s.bits, wave = threadIdx.x / 64;
    // a wave has SORT_ITEMS * 64 neighbouring items, 64 at a time; all that is read is asked for first
    const int64_t first = int64_t(blockIdx.x) * SORT_TILE + wave * (SORT_ITEMS * 64) + (threadIdx.x & 63);
    uint32_t key[SORT_ITEMS], pos[SORT_ITEMS], rank[SORT_ITEMS];
    bool on[SORT_ITEMS];
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i) {
        const int64_t k = first + i * 64;
        on[i] = k < s.n;
        key[i] = on[i] ? sort_key(s, k) : 0u;
        pos[i] = on[i] ? (s.ids ? static_cast<uint32_t>(k) : s.pos[k]) : 0u;
    }
    constexpr int EACH = (1 << SORT_BITS) / SORT_THREADS;
    uint32_t before[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int d = i * SORT_THREADS + threadIdx.x;
        before[i] = 0;
        if (d < digits) {
            before[i] = s.count[int64_t(d) * s.tiles + blockIdx.x];
            start[d] = s.total[d];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) count[w][d] = 0;
        }
    }
    __syncthreads();
    digit_scan<SORT_WAVES>(start, digits, sum);
    rank_items(key, on, s.shift, s.bits, count[wave], rank);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int d = i * SORT_THREADS + threadIdx.x;
        if (d < digits) {
            uint32_t at = start[d] + before[i];
#pragma unroll
            for (int w = 0; w < SORT_WAVES; ++w) {
                const uint32_t c = count[w][d];
                count[w][d] = at;
                at += c;
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < SORT_ITEMS; ++i)
        if (on[i]) {
            const uint32_t to = count[wave][(key[i] >> s.shift) & (digits - 1)] + rank[i];
            s.key_out[to] = key[i];
            s.pos_out[to] = pos[i];
        }
}

// Up to SMALL_TILE ids: every pass in one workgroup, through LDS.  (The other workgroups zero the table.)
__global__ __launch_bounds__(SMALL_THREADS) void sort_small_kernel(SortPass s) {
    __shared__ uint32_t count[SMALL_WAVES][1 << SMALL_BITS], start[1 << SMALL_BITS], sum[SMALL_WAVES], keys[SMALL_TILE], poss[SMALL_TILE];
    if (blockIdx.x >= 1) return fill_share(s.fill, blockIdx.x - 1, gridDim.x - 1);
    const int n = static_cast<int>(s.n), wave = threadIdx.x / 64, digits = 1 << SMALL_BITS;
    if (n <= SMALL_COUNT) {             // a key's place is the number of keys before it
        const int t = threadIdx.x;
        const uint32_t mine = t < n ? sort_key(s, t) : ~0u;
        if (t < SMALL_COUNT) keys[t] = mine;
        __syncthreads();
        if (t >= n) return;
        int to = 0;
        for (int j = 0; j < n; j += 8) {
            uint32_t k[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) k[e] = keys[j + e];
#pragma unroll
            for (int e = 0; e < 8; ++e) to += k[e] < mine || (k[e] == mine && j + e < t);
        }
        s.key_out[to] = mine;
        s.pos_out[to] = t;
        return;
    }
    const int first = wave * (SMALL_ITEMS * 64) + (threadIdx.x & 63);
    uint32_t key[SMALL_ITEMS], pos[SMALL_ITEMS], rank[SMALL_ITEMS];
    bool on[SMALL_ITEMS];
#pragma unroll
    for (int i = 0; i < SMALL_ITEMS; ++i) {
        const int k = first + i * 64;
        on[i] = k < n;
        key[i] = on[i] ? sort_key(s, k) : 0u;
        pos[i] = static_cast<uint32_t>(k);
    }
    for (int shift = 0; shift < s.bits; shift += SMALL_BITS) {
        for (int d = threadIdx.x; d < SMALL_WAVES * digits; d += SMALL_THREADS) (&count[0][0])[d] = 0;
        __syncthreads();
        rank_items(key, on, shift, SMALL_BITS, count[wave], rank);
        __syncthreads();
        if (threadIdx.x < digits) {
            uint32_t at = 0;
            for (int w = 0; w < SMALL_WAVES; ++w) {
                const uint32_t c = count[w][threadIdx.x];
                count[w][threadIdx.x] = at;
                at += c;
            }
            start[threadIdx.x] = at;
        }
        __syncthreads();
        digit_scan<SMALL_WAVES>(start, digits, sum);
#pragma unroll
        for (int i = 0; i < SMALL_ITEMS; ++i)
            if (on[i]) {
                const uint32_t d = (key[i] >> shift) & (digits - 1), to = start[d] + count[wave][d] + rank[i];
                keys[to] = key[i];
                poss[to] = pos[i];
            }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SMALL_ITEMS; ++i)
            if (on[i]) {
                key[i] = keys[first + i * 64];
                pos[i] = poss[first + i * 64];
            }
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < SMALL_ITEMS; ++i)
        if (on[i]) {
            s.key_out[first + i * 64] = key[i];
            s.pos_out[first + i * 64] = pos[i];
        }
}

// ------------------------------------------------------------------ sums of runs
struct RunArgs {
    int64_t n;
    uint32_t V;
    int F, lanes, R;            // a tile has R sorted entries
    int64_t tiles;
    const uint32_t *key, *pos;
    const char *dY;
    int64_t lddy;               // in bytes
    float scale;
    float *dtable;
    int64_t lddt;
    int accumulate;
    float *part;                // [tiles][2][vectors * V]: the run that comes in from the tile before, and the one that goes on into the next
    int64_t part_ld;
};

template <int V> __device__ __forceinline__ void put_row(const RunArgs &a, uint32_t id, int from, int skip, const float (&acc)[V]) {
    float *out = a.dtable + int64_t(id) * a.lddt + from;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = acc[e] * a.scale;
    if (skip == 0) {
        if (a.accumulate) {
            float old[V];
            ld_row<false, V>(reinterpret_cast<const char *>(out), 0, old);
#pragma unroll
            for (int e = 0; e < V; ++e) v[e] += old[e];
        }
        st_row<false, V>(reinterpret_cast<char *>(out), 0, v);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (e >= skip) out[e] = a.accumulate ? out[e] + v[e] : v[e];
    }
}

constexpr int RUN_AHEAD = 8;        // rows of a batch: one is on its way while another is added

// A team's next entries are in its lanes, one each, and handed round from there, so that a row's address waits for nothing but its entry's load
// a whole stretch before.
template <bool BF16, int V> __global__ __launch_bounds__(256) void run_sums_kernel(RunArgs a) {
    const int lane = threadIdx.x & (a.lanes - 1), teams = 256 / a.lanes;
    const int64_t tile = int64_t(blockIdx.x) * teams + threadIdx.x / a.lanes;
    const int vec = blockIdx.y * a.lanes + lane, j = vec * V;
    const bool live = tile < a.tiles && j < a.F;
    const int from = min(j, a.F - V), skip = j - from;
    const int64_t p0 = min(tile, a.tiles - 1) * a.R, p1 = min(p0 + a.R, a.n);
    const int count = static_cast<int>(p1 - p0);
    // (loaded without conditions, so that they are under way together)
    uint32_t cur = a.key[p0];
    const uint32_t last = a.key[max(p0 - 1, int64_t(0))], after = a.key[min(p1, a.n - 1)];
    bool head = p0 > 0 && last == cur;
    const uint32_t next = p1 < a.n ? after : ~0u;
    float *part = a.part + tile * 2 * a.part_ld + vec * V;
    float acc[V];
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e] = 0.f;
    uint32_t keys[2][RUN_AHEAD];
    RawRow<BF16, V> rows[2][RUN_AHEAD];
    // entries of a team that its lanes hold: [held, held + lanes)
    int held = 0;
    uint32_t key_here = 0, pos_here = 0;
    auto hold = [&](int from_entry) __attribute__((always_inline)) {
        held = from_entry;
        const int64_t p = p0 + min(from_entry + lane, count - 1);
        key_here = a.key[p];
        pos_here = a.pos[p];
    };
    auto fetch = [&](int set, int entry) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < RUN_AHEAD; ++i) {
            const int at = min(entry + i, count - 1);
            if (at >= held + a.lanes) hold(at);
            const int source = (threadIdx.x & 63 & ~(a.lanes - 1)) + at - held;
            keys[set][i] = static_cast<uint32_t>(__shfl(static_cast<int>(key_here), source));
            const uint32_t pos = static_cast<uint32_t>(__shfl(static_cast<int>(pos_here), source));
            rows[set][i].load(a.dY + int64_t(pos) * a.lddy, from);
        }
    };
    auto add = [&](int set, int entry) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < RUN_AHEAD; ++i) {
            if (entry + i < count) {
                if (keys[set][i] != cur) {
                    if (live) {
                        if (head) st_row<false, V>(reinterpret_cast<char *>(part), 0, acc);
                        else if (cur < a.V) put_row<V>(a, cur, from, skip, acc);
                    }
                    head = false;
                    cur = keys[set][i];
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += rows[set][i].get(e);
            }
        }
    };
    // (all lanes of a wave walk as many batches: what is behind a tile's end repeats its last entry and is not added)
    hold(0);
    fetch(0, 0);
    for (int p = 0; p < a.R; p += 2 * RUN_AHEAD) {
        if (p + RUN_AHEAD < a.R) fetch(1, p + RUN_AHEAD);
        add(0, p);
        if (p + 2 * RUN_AHEAD < a.R) fetch(0, p + 2 * RUN_AHEAD);
        if (p + RUN_AHEAD < a.R) add(1, p + RUN_AHEAD);
    }
    if (!live || cur >= a.V) return;            // (ids outside the table are the last ones)
    if (head) st_row<false, V>(reinterpret_cast<char *>(part), 0, acc);
    else if (cur == next) st_row<false, V>(reinterpret_cast<char *>(part + a.part_ld), 0, acc);
    else put_row<V>(a, cur, from, skip, acc);
}

// The runs that cross tiles: where one begins, its parts are added, by the tile's team if they are few, by a wave if its teams have a few batches
// each of them, else by the whole workgroup, every team those of a stretch of tiles.  (us of the whole gradient, without the waves / with them:
// 117176 rows of 2 into 1660 57 / 38, 60000 of 8 into 1000 66 / 33, 500000 of 8 into 5000 100 / 73, 300001 of 256 into 500009 no other.)
constexpr int JOIN_THREADS = 1024, JOIN_FEW = 8, JOIN_STEPS = 4;

template <int V> __global__ __launch_bounds__(JOIN_THREADS) void run_join_kernel(RunArgs a) {
    __shared__ float sums[JOIN_THREADS * V];
    __shared__ int run_end, many[JOIN_THREADS], n_many;
    __shared__ uint32_t many_id[JOIN_THREADS];
    const int lane = threadIdx.x & (a.lanes - 1), teams = JOIN_THREADS / a.lanes, team = threadIdx.x / a.lanes;
    const int vec = blockIdx.y * a.lanes + lane, j = vec * V, from = min(j, a.F - V);
    const bool live = j < a.F;
    auto part = [&](int64_t tile, int which) { return reinterpret_cast<const char *>(a.part + (tile * 2 + which) * a.part_ld + vec * V); };
    if (threadIdx.x == 0) n_many = 0;
    __syncthreads();
    {
        const int64_t tile = int64_t(blockIdx.x) * teams + team, p0 = tile * a.R, p1 = p0 + a.R, last = a.n - 1;
        // (everything that may be asked is asked for together: a step that waits for memory costs two microseconds here)
        const uint32_t id = a.key[min(p1, last)], id_end = a.key[min(p1 - 1, last)], id_begin = a.key[min(p0, last)];
        const uint32_t id_last = a.key[min(max(p0 - 1, int64_t(0)), last)];
        uint32_t begins[JOIN_FEW];
#pragma unroll
        for (int i = 0; i < JOIN_FEW; ++i) begins[i] = a.key[min(tile + 2 + i, a.tiles - 1) * a.R];
        // (ids beyond the table are no run; one that came in from the tile before begins elsewhere)
        if (p1 < a.n && id < a.V && id_end == id && !(id_begin == id && p0 > 0 && id_last == id)) {
            int m = 1;
#pragma unroll
            for (int i = 0; i < JOIN_FEW; ++i)
                if (m == i + 1 && tile + 2 + i < a.tiles && begins[i] == id) ++m;
            if (m <= JOIN_FEW) {
                if (live) {
                    float acc[V], v[4][V];
                    ld_row<false, V>(part(tile, 1), 0, acc);
                    for (int t = 1; t <= m; t += 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) ld_row<false, V>(part(tile + min(t + i, m), 0), 0, v[i]);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (t + i <= m) {
#pragma unroll
                                for (int e = 0; e < V; ++e) acc[e] += v[i][e];
                            }
                    }
                    put_row<V>(a, id, from, j - from, acc);
                }
            } else if (lane == 0) {
                const int k = atomicAdd(&n_many, 1);        // (each is added by itself: their order changes nothing)
                many[k] = team;
                many_id[k] = id;
            }
        }
    }
    __syncthreads();
    constexpr int PROBES = 4;           // of a thread at a time
    using Few = std::integral_constant<int, V == 1 ? 16 : 8>;           // parts of a team on their way at a time
    using Many = std::integral_constant<int, V == 8 ? 8 : 16>;
    // what a team adds up of a run's parts: of tiles [first, end), behind what acc has
    auto add_parts = [&](auto ahead, int64_t first, int64_t end, float (&acc)[V]) __attribute__((always_inline)) {
        constexpr int AHEAD = ahead.value;
        for (int64_t t = first; t < end; t += AHEAD) {
            float v[AHEAD][V];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) ld_row<false, V>(part(min(t + i, end - 1), 0), 0, v[i]);
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (t + i < end) {
#pragma unroll
                    for (int e = 0; e < V; ++e) acc[e] += v[i][e];
                }
        }
    };
    {
        // (of narrow rows many such runs begin in one workgroup)
        const int wave = threadIdx.x / 64, own = 64 / a.lanes, mine = (threadIdx.x & 63) / a.lanes;
        const int64_t most = int64_t(own) * Few::value * JOIN_STEPS;
        for (int k = wave; own > 1 && k < n_many; k += JOIN_THREADS / 64) {
            const int64_t tile = int64_t(blockIdx.x) * teams + many[k];
            const uint32_t id = many_id[k];
            int64_t m = JOIN_FEW;
            for (bool more = true; more && m <= most;) {
                const int64_t t = tile + 1 + m + (threadIdx.x & 63);
                uint32_t probe[PROBES];
#pragma unroll
                for (int i = 0; i < PROBES; ++i) probe[i] = a.key[min(t + i * 64, a.tiles - 1) * a.R];
#pragma unroll
                for (int i = 0; i < PROBES; ++i)
                    if (more) {
                        const uint64_t out = __ballot(t + i * 64 >= a.tiles || probe[i] != id);
                        m += out ? __ffsll(static_cast<unsigned long long>(out)) - 1 : 64;
                        more = out == 0;
                    }
            }
            if (m > most) continue;
            const int64_t each = (m + own - 1) / own;
            float acc[V];
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = 0.f;
            if (live) {
                if (mine == 0) ld_row<false, V>(part(tile, 1), 0, acc);
                add_parts(Few(), tile + 1 + min(each * mine, m), tile + 1 + min(each * (mine + 1), m), acc);
            }
            for (int half = own / 2; half; half /= 2) {
#pragma unroll
                for (int e = 0; e < V; ++e) acc[e] += __shfl_down(acc[e], half * a.lanes);
            }
            if (mine == 0 && live) put_row<V>(a, id, from, j - from, acc);
            if ((threadIdx.x & 63) == 0) many[k] = -1;
        }
    }
    __syncthreads();
    for (int k = 0; k < n_many; ++k) {
        if (many[k] < 0) continue;
        const int64_t tile = int64_t(blockIdx.x) * teams + many[k];
        const uint32_t id = many_id[k];
        int64_t m = JOIN_FEW;               // tiles tile + 1 .. tile + m begin with this id (by the order every one between does)
        for (bool more = true; more;) {
            if (threadIdx.x == 0) run_end = PROBES * JOIN_THREADS;
            __syncthreads();
            uint32_t probe[PROBES];
            const int64_t t = tile + 1 + m + threadIdx.x;
#pragma unroll
            for (int i = 0; i < PROBES; ++i) probe[i] = a.key[min(t + i * JOIN_THREADS, a.tiles - 1) * a.R];
#pragma unroll
            for (int i = 0; i < PROBES; ++i) {
                const uint64_t out = __ballot(t + i * JOIN_THREADS >= a.tiles || probe[i] != id);
                if (out && (threadIdx.x & 63) == 0) atomicMin(&run_end, static_cast<int>(threadIdx.x) + i * JOIN_THREADS + __ffsll(static_cast<unsigned long long>(out)) - 1);
            }
            __syncthreads();
            m += run_end;
            more = run_end == PROBES * JOIN_THREADS;
            __syncthreads();
        }
        const int64_t each = (m + teams - 1) / teams, first = tile + 1 + min(each * team, m), end = tile + 1 + min(each * (team + 1), m);
        float acc[V];
#pragma unroll
        for (int e = 0; e < V; ++e) acc[e] = 0.f;
        if (live) {
            if (team == 0) ld_row<false, V>(part(tile, 1), 0, acc);
            add_parts(Many(), first, end, acc);
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sums[e * JOIN_THREADS + threadIdx.x] = acc[e];
        __syncthreads();
        // the teams' sums, half of them to the other half, in a fixed order
        for (int half = teams / 2; half; half /= 2) {
            if (team < half) {
#pragma unroll
                for (int e = 0; e < V; ++e) sums[e * JOIN_THREADS + threadIdx.x] += sums[e * JOIN_THREADS + threadIdx.x + half * a.lanes];
            }
            __syncthreads();
        }
        if (team == 0 && live) {
#pragma unroll
            for (int e = 0; e < V; ++e) acc[e] = sums[e * JOIN_THREADS + threadIdx.x];
            put_row<V>(a, id, from, j - from, acc);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ tables of a few rows
// A table that fits LDS many times over needs no sorting: a team of lanes has a copy of its own there and adds the rows of dY to it, one
// after the other, each lane its columns; a workgroup's copies are added at its end, and the workgroups' sums by a second launch, in
// their order.  (612000 rows of 100 floats into 47: 102 us by sorting, of which the sums alone take 57; here 64, 3.9 TB/s, and 5 for the
// join; with one batch of rows on its way instead of two 80.)  What nothing was added to is -0,
// which changes no sum and is none: a -0 of dY is added as 0.
struct TableArgs {
    int64_t n;
    int V, F, lanes, chunk;     // a workgroup takes `chunk` vectors of a row (at most 64)
    const int64_t *ids;
    const char *dY;
    int64_t lddy;               // in bytes
    int64_t rows;               // of a workgroup
    float *part;                // [workgroups][V][F]
};

constexpr int TABLE_THREADS = 256, TABLE_AHEAD = 16;         // rows of a team on their way

template <bool BF16, int V> __global__ __launch_bounds__(TABLE_THREADS, 1) void table_sums_kernel(TableArgs a) {
    extern __shared__ float tables[];
    const int lane = threadIdx.x & (a.lanes - 1), teams = TABLE_THREADS / a.lanes, team = threadIdx.x / a.lanes;
    const int vec = blockIdx.y * a.chunk + lane, j = vec * V;
    const bool live = lane < a.chunk && j < a.F;
    const int from = min(j, a.F - V), size = a.V * a.chunk * V;         // of a copy
    for (int i = threadIdx.x; i < teams * size; i += TABLE_THREADS) tables[i] = -0.f;
    __syncthreads();
    float *mine = tables + team * size + lane * V;
    const int64_t first = blockIdx.x * a.rows, end = min(first + a.rows, a.n);
    if (live && first + team < end) {
        int64_t id[2][TABLE_AHEAD];
        RawRow<BF16, V> row[2][TABLE_AHEAD];
        const int64_t step = int64_t(teams) * TABLE_AHEAD;
        auto fetch = [&](int set, int64_t i) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < TABLE_AHEAD; ++u) {
                const int64_t r = min(i + int64_t(u) * teams, end - 1);
                id[set][u] = a.ids[r];
                row[set][u].load(a.dY + r * a.lddy, from);
            }
        };
        auto add = [&](int set, int64_t i) __attribute__((always_inline)) {
#pragma unroll
            for (int u = 0; u < TABLE_AHEAD; ++u) {
                if (i + int64_t(u) * teams < end && id[set][u] >= 0 && id[set][u] < a.V) {
                    float *t = mine + static_cast<int>(id[set][u]) * a.chunk * V;
                    float v[V];
#pragma unroll
                    for (int e = 0; e < V; ++e) v[e] = t[e];
#pragma unroll
                    for (int e = 0; e < V; ++e) t[e] = v[e] + (row[set][u].get(e) + 0.f);        // (no -0: that is the mark)
                }
            }
        };
        int64_t i = first + team;
        fetch(0, i);
        for (; i < end; i += 2 * step) {
            if (i + step < end) fetch(1, i + step);
            add(0, i);
            if (i + 2 * step < end) fetch(0, i + 2 * step);
            if (i + step < end) add(1, i + step);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < size; i += TABLE_THREADS) {
        float sum = tables[i];
        for (int q = 1; q < teams; ++q) sum += tables[q * size + i];
        // entry i: element e of vector k of row r; a row's last vector has its elements from the row's end backwards
        const int r = i / (a.chunk * V), k = i / V % a.chunk, e = i % V, at = (blockIdx.y * a.chunk + k) * V;
        if (at < a.F && e >= at - min(at, a.F - V)) a.part[(int64_t(blockIdx.x) * a.V + r) * a.F + min(at, a.F - V) + e] = sum;
    }
}

// dtable (+)= scale * the workgroups' sums: 16 columns a workgroup, 16 threads each with every 16th part, then their sums in order
__global__ __launch_bounds__(256) void table_join_kernel(const float *part, int parts, int64_t size, int F, float scale, float *dtable, int64_t lddt,
                                                         int accumulate) {
    __shared__ float s[16][17];
    const int c = threadIdx.x & 15, q = threadIdx.x / 16;
    const int64_t j = int64_t(blockIdx.x) * 16 + c;
    float v = -0.f;
    if (j < size) {
#pragma unroll 8
        for (int p = q; p < parts; p += 16) v += part[p * size + j];
    }
    s[q][c] = v;
    __syncthreads();
    if (q == 0 && j < size) {
        for (int i = 1; i < 16; ++i) v += s[i][c];
        float *out = dtable + j / F * lddt + j % F;
        const bool added = __float_as_uint(v) != 0x80000000u;       // (nothing stays nothing at a scale that is infinite or NaN, too)
        if (!accumulate) *out = added ? v * scale + 0.f : 0.f;
        else if (added) *out += v * scale;
    }
}

__global__ __launch_bounds__(256) void fill_kernel(Fill f) { fill_share(f, blockIdx.x, gridDim.x); }

// ------------------------------------------------------------------ host side
constexpr int EMBED_WIDEST = 1 << 22;       // (teams side by side along a row are a launch's second dimension)
struct EmbedShape {
    int V, lanes, chunks;       // elements and lanes of a team, teams side by side along a row
};
static EmbedShape embed_shape(int F, bool bf16) {
    const int V = F < (bf16 ? ROW_V<true> : ROW_V<false>) ? 1 : bf16 ? ROW_V<true> : ROW_V<false>;
    const int vectors = (F + V - 1) / V, lanes = std::min(64, pow2_at_least(vectors));
    return {V, lanes, (vectors + lanes - 1) / lanes};
}

// entries of a tile: enough tiles for 16 waves on every compute unit, 8 to 128 entries (and at most 2^22 tiles)
static int run_tile(int64_t n, const EmbedShape &s) {
    const int64_t teams = std::max<int64_t>(int64_t(NUM_CU) * 16 * (64 / s.lanes) / s.chunks, 1);
    const int64_t R = std::min<int64_t>(std::max<int64_t>((n + teams - 1) / teams, 8), 128);
    return static_cast<int>(std::max<int64_t>(R, (n >> 22) + 1));
}

// A table in LDS: workgroups and LDS of each; 0 workgroups where sorting is the shorter way.  What it costs at any n grows with the copies of
// all teams, which are cleared and added up; bf16 rows in several stretches read twice as many places of LDS per byte.  (us, LDS / sorted: 100000
// fp32 rows of 250 into 35 47 / 60, 3000 into 35 25 / 21, into 18 17 / 23, 200 rows of 64 into 40 20 / 16, into 20 12 / 14; bf16 rows of 1000
// into 4: 9000 25 / 36, 30000 45 / 52, 300000 277 / 227; 100000 fp32 rows of 250 into 70, two teams of 64 lanes a workgroup, 89 / 56.)
struct TableShape {
    int groups, chunk;
    int64_t rows;
    size_t lds;
};
static TableShape table_shape(int64_t n, int64_t V, const EmbedShape &s, int F) {
    TableShape t{};
    const int64_t vectors = (F + s.V - 1) / s.V, teams = TABLE_THREADS / s.lanes;
    t.chunk = static_cast<int>(std::min<int64_t>(vectors, s.lanes));
    t.lds = size_t(V) * t.chunk * s.V * sizeof(float) * teams;
    if (t.lds > size_t(n <= SMALL_TILE ? 80 : 156) * 1024 || (s.V == 8 && s.chunks > 1 && n > 32768)) return {};
    if (V * F > int64_t(1) << 27) return {};        // (the join's grid: fewer than 2^32 threads)
    const int64_t room = std::min<int64_t>(160 * 1024 / t.lds, 8), most = std::max<int64_t>(NUM_CU * room / s.chunks, 1);
    t.rows = std::max<int64_t>((n + most - 1) / most, teams * TABLE_AHEAD);
    t.groups = static_cast<int>((n + t.rows - 1) / t.rows);
    return t;
}

struct EmbedWork {              // offsets into the workspace
    size_t key[2], pos[2], count, total, part, bytes;
    int passes, bits;
    unsigned tiles;
};
static EmbedWork embed_work(int64_t n, int64_t V, int F) {
    EmbedWork w{};
    int bits = 1;
    while ((int64_t(1) << bits) <= V) ++bits;       // keys go up to V itself
    w.passes = (bits + SORT_BITS - 1) / SORT_BITS;
    w.bits = n <= SMALL_TILE ? bits : (bits + w.passes - 1) / w.passes;
    w.tiles = static_cast<unsigned>((n + SORT_TILE - 1) / SORT_TILE);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes, 256);
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        w.key[i] = take(n * sizeof(uint32_t));
        w.pos[i] = take(n * sizeof(uint32_t));
    }
    w.count = take((size_t(1) << SORT_BITS) * w.tiles * sizeof(uint32_t));
    w.total = take((size_t(1) << SORT_BITS) * sizeof(uint32_t));
    size_t part = 0;
    for (bool bf16 : {false, true}) {
        const EmbedShape s = embed_shape(F, bf16);
        const int R = run_tile(n, s);
        part = std::max(part, size_t((n + R - 1) / R) * 2 * ((F + s.V - 1) / s.V * s.V) * sizeof(float));
    }
    w.part = take(part);
    w.bytes = at;
    for (bool bf16 : {false, true}) {
        const EmbedShape s = embed_shape(F, bf16);
        w.bytes = std::max(w.bytes, align_up(sizeof(float) * table_shape(n, V, s, F).groups * V * F, 256));
    }
    return w;
}

}  // namespace capgnn

using namespace capgnn;

extern "C" int capgnn_embed(int64_t n, const int64_t *ids, int64_t V, int F, const void *table, int64_t ldt, int dtype, float scale, void *out,
                            int64_t ldo, int out_dtype, void *stream) {
    if (!is_float_type(dtype) || !is_float_type(out_dtype)) CG_FAIL(CAPGNN_EINVAL, "embed: unknown dtype or out_dtype");
    if (n < 0 || V <= 0 || V >= int64_t(1) << 31 || F <= 0) CG_FAIL(CAPGNN_EINVAL, "embed: bad sizes");
    if (F > EMBED_WIDEST) CG_FAIL(CAPGNN_EUNSUPPORTED, "embed: rows of %d elements, at most %d are supported", F, EMBED_WIDEST);
    if (n == 0) return CAPGNN_OK;
    if (!ids || !table || !out) CG_FAIL(CAPGNN_EINVAL, "embed: NULL operand");
    if (ldt < F || ldo < F) CG_FAIL(CAPGNN_EINVAL, "embed: leading dimension smaller than the row");
    if (!row_aligned(table, dtype) || !row_aligned(out, out_dtype) || reinterpret_cast<uintptr_t>(ids) & 7u)
        CG_FAIL(CAPGNN_EINVAL, "embed: an operand is not aligned to its elements");
    if (out == table) CG_FAIL(CAPGNN_EINVAL, "embed: out must not be the table");
    const EmbedShape s = embed_shape(F, dtype == CAPGNN_BF16);
    const EmbedArgs a{n, V, F, s.lanes, ids, static_cast<const char *>(table), ldt * elem_bytes(dtype), ldo * elem_bytes(out_dtype), scale,
                      static_cast<char *>(out), out_dtype == CAPGNN_BF16};
    const int teams = 256 / s.lanes;
    const unsigned grid = stride_grid((n + teams - 1) / teams, 256);
    hipStream_t st = static_cast<hipStream_t>(stream);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, st, a); };
    if (dtype == CAPGNN_BF16) s.V == 1 ? go(embed_kernel<true, 1>) : go(embed_kernel<true, 8>);
    else s.V == 1 ? go(embed_kernel<false, 1>) : go(embed_kernel<false, 4>);
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" size_t capgnn_embed_bwd_workspace_bytes(int64_t n, int64_t V, int F) {
    if (n <= 0 || n >= int64_t(1) << 31 || V <= 0 || V >= int64_t(1) << 31 || F <= 0 || F > EMBED_WIDEST) return 0;
    return embed_work(n, V, F).bytes;
}

extern "C" int capgnn_embed_bwd(int64_t n, const int64_t *ids, int64_t V, int F, const void *dY, int64_t lddy, int dy_dtype, float scale,
                                float *dtable, int64_t lddt, int accumulate, void *ws, size_t ws_bytes, void *stream) {
    if (!is_float_type(dy_dtype)) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: unknown dy_dtype");
    if (n < 0 || n >= int64_t(1) << 31 || V <= 0 || V >= int64_t(1) << 31 || F <= 0) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: bad sizes");
    if (F > EMBED_WIDEST) CG_FAIL(CAPGNN_EUNSUPPORTED, "embed_bwd: rows of %d elements, at most %d are supported", F, EMBED_WIDEST);
    if (!dtable || (n > 0 && (!ids || !dY))) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: NULL operand");
    if (lddt < F || (n > 0 && lddy < F)) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: leading dimension smaller than the row");
    if ((n > 0 && (!row_aligned(dY, dy_dtype) || reinterpret_cast<uintptr_t>(ids) & 7u)) || !row_aligned(dtable, CAPGNN_F32))
        CG_FAIL(CAPGNN_EINVAL, "embed_bwd: an operand is not aligned to its elements");
    if (dY == dtable) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: dtable must not be dY");
    hipStream_t st = static_cast<hipStream_t>(stream);
    Fill fill{accumulate ? nullptr : dtable, V, lddt, F, 0, 1};
    const int64_t fill_jobs = (V * int64_t(F) + 4095) / 4096;       // 16 floats a thread
    if (n == 0) {
        if (!fill.p) return CAPGNN_OK;
        hipLaunchKernelGGL(fill_kernel, dim3(stride_grid(fill_jobs, 256)), dim3(256), 0, st, fill);
        CG_HIP(hipGetLastError());
        return CAPGNN_OK;
    }
    const EmbedWork w = embed_work(n, V, F);
    if (!ws || ws_bytes < w.bytes) CG_FAIL(CAPGNN_ENOMEM, "embed_bwd: workspace of %zu bytes needed, %zu given", w.bytes, ws ? ws_bytes : size_t(0));
    if (reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "embed_bwd: workspace must be 256-byte aligned");
    const bool bf16 = dy_dtype == CAPGNN_BF16;
    const EmbedShape e = embed_shape(F, bf16);
    if (const TableShape t = table_shape(n, V, e, F); t.groups) {
        const TableArgs a{n, static_cast<int>(V), F, e.lanes, t.chunk, ids, static_cast<const char *>(dY), lddy * elem_bytes(dy_dtype), t.rows,
                          static_cast<float *>(ws)};
        const dim3 grid(t.groups, e.chunks);
        auto go = [&](auto kernel) {
            if (t.lds > 64 * 1024) CG_HIP(hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(t.lds)));
            hipLaunchKernelGGL(kernel, grid, dim3(TABLE_THREADS), t.lds, st, a);
            CG_HIP(hipGetLastError());
            return static_cast<int>(CAPGNN_OK);
        };
        if (bf16) CG_TRY(e.V == 1 ? go(table_sums_kernel<true, 1>) : go(table_sums_kernel<true, 8>));
        else CG_TRY(e.V == 1 ? go(table_sums_kernel<false, 1>) : go(table_sums_kernel<false, 4>));
        const int64_t size = V * int64_t(F);
        hipLaunchKernelGGL(table_join_kernel, dim3(static_cast<unsigned>((size + 15) / 16)), dim3(256), 0, st, a.part, t.groups, size, F, scale, dtable, lddt, accumulate != 0);
        CG_HIP(hipGetLastError());
        return CAPGNN_OK;
    }
    char *base = static_cast<char *>(ws);
    auto at = [&](size_t off) { return reinterpret_cast<uint32_t *>(base + off); };
    const bool small = n <= SMALL_TILE;
    SortPass s{};
    s.n = n;
    s.V = static_cast<uint32_t>(V);
    s.tiles = w.tiles;
    s.count = at(w.count);
    s.total = at(w.total);
    s.fill = fill;
    s.fill.parts = small ? 1 : 2 * w.passes;
    auto fill_groups = [&](int threads) {           // workgroups that a launch has for its share of the zeros
        return s.fill.p ? static_cast<unsigned>(std::min<int64_t>(std::max<int64_t>(fill_jobs * 256 / threads / s.fill.parts, 1), 4096)) : 0u;
    };
    int now = 0;
    if (small) {
        s.ids = ids;
        s.bits = w.bits;
        s.key_out = at(w.key[0]);
        s.pos_out = at(w.pos[0]);
        hipLaunchKernelGGL(sort_small_kernel, dim3(1 + fill_groups(SMALL_THREADS)), dim3(SMALL_THREADS), 0, st, s);
    } else {
        for (int p = 0; p < w.passes; ++p) {
            s.ids = p == 0 ? ids : nullptr;
            s.key = at(w.key[now]);
            s.pos = at(w.pos[now]);
            now ^= p > 0;
            s.key_out = at(w.key[now]);
            s.pos_out = at(w.pos[now]);
            s.shift = p * w.bits;
            s.bits = w.bits;
            const unsigned more = fill_groups(SORT_THREADS);
            hipLaunchKernelGGL(sort_count_kernel, dim3(s.tiles + more), dim3(SORT_THREADS), 0, st, s);
            ++s.fill.part;
            hipLaunchKernelGGL(sort_prefix_kernel, dim3(((1u << s.bits) + SORT_WAVES - 1) / SORT_WAVES + more), dim3(SORT_THREADS), 0, st, s);
            ++s.fill.part;
            hipLaunchKernelGGL(sort_move_kernel, dim3(s.tiles), dim3(SORT_THREADS), 0, st, s);
        }
    }
    CG_HIP(hipGetLastError());
    const int R = run_tile(n, e);
    const RunArgs a{n, s.V, F, e.lanes, R, (n + R - 1) / R, at(w.key[now]), at(w.pos[now]), static_cast<const char *>(dY),
                    lddy * elem_bytes(dy_dtype), scale, dtable, lddt, accumulate != 0, reinterpret_cast<float *>(base + w.part),
                    (F + e.V - 1) / e.V * e.V};
    const int teams = 256 / e.lanes;
    const dim3 sums(static_cast<unsigned>((a.tiles + teams - 1) / teams), e.chunks);
    const dim3 join(static_cast<unsigned>((a.tiles * e.lanes + JOIN_THREADS - 1) / JOIN_THREADS), e.chunks);
    if (bf16) {
        if (e.V == 1) hipLaunchKernelGGL((run_sums_kernel<true, 1>), sums, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((run_sums_kernel<true, 8>), sums, dim3(256), 0, st, a);
    } else {
        if (e.V == 1) hipLaunchKernelGGL((run_sums_kernel<false, 1>), sums, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((run_sums_kernel<false, 4>), sums, dim3(256), 0, st, a);
    }
    if (a.tiles > 1) {
        if (e.V == 1) hipLaunchKernelGGL(run_join_kernel<1>, join, dim3(JOIN_THREADS), 0, st, a);
        else if (e.V == 4) hipLaunchKernelGGL(run_join_kernel<4>, join, dim3(JOIN_THREADS), 0, st, a);
        else hipLaunchKernelGGL(run_join_kernel<8>, join, dim3(JOIN_THREADS), 0, st, a);
    }
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}
