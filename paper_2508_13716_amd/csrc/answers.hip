// What a classifier answers with: log-probabilities of given classes, entropy, the most likely classes; and their gradient.
#include "grid.h"
#include "softrow.h"

#include <algorithm>
#include <type_traits>

namespace capgnn {

struct AnswerArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const int32_t *ids; int64_t ldi; int m;
    float *logp; int64_t ldp;
    float *entropy, *stats;
    int k;
    int32_t *top_ids; float *top_logp; int64_t ldt;
};

__device__ __forceinline__ void masked_out_row(const AnswerArgs &a, int64_t row, int threads) {
    for (int i = threadIdx.x; i < a.m; i += threads) a.logp[row * a.ldp + i] = 0.f;
    for (int i = threadIdx.x; i < a.k; i += threads) {
        if (a.top_ids) a.top_ids[row * a.ldt + i] = -1;
        if (a.top_logp) a.top_logp[row * a.ldt + i] = 0.f;
    }
    if (threadIdx.x == 0) {
        if (a.entropy) a.entropy[row] = 0.f;
        if (a.stats) a.stats[2 * row] = a.stats[2 * row + 1] = 0.f;
    }
}

// What a row's sums come to.
struct RowEnd {
    float m0, ln_s, inv_T;
    bool empty;
    __device__ RowEnd(float m, float s, float inv_t) : m0(safe_max(m)), ln_s(s == 0.f ? -INFINITY : logf(s)), inv_T(inv_t), empty(s == 0.f) {}
    __device__ float logp(float z) const { return empty ? -INFINITY : (z - m0) * inv_T - ln_s; }
    // sum of p u, u = log2 of the exponentials: entropy = ln s - ln 2 * (sum of e u) / s
    __device__ float entropy(float s, float e1) const { return empty ? 0.f : ln_s - e1 / s * 0.69314718f; }
};

// ------------------------------------------------------------------ the k largest of a stream of logits
// Every wave walks its share of a row and keeps the keys (logit, class) that may still be among the k largest in LDS, together with a
// threshold: of at least k logits of the row it is known that they are no smaller.  The first tile's thread maxima give one for the whole
// workgroup: the k-th largest of them is exceeded by hardly more than k logits of the tile (64 largest of 16384: 73 on average).  What
// passes the threshold is appended; a wave's list that is half full is ranked, each key by counting the larger ones, and cut to k.
// Keys are distinct, so the order of appending does not show.  A wave alone has 64 maxima, of which the 64th largest is passed by 260 of 4096
// logits and sometimes twice as many: for k > 32 it takes the k-th largest of its 512 vectors' maxima.  A tile that passes more than
// the list holds is tried again with those, then with its exact k-th largest key (equal logits): slower, never wrong.  The waves meet
// at the first threshold and at the end of the row only (a list for the workgroup, with an atomic counter and a barrier per tile:
// 4096 x 131072 bf16, k = 64, 471 us).
template <int THREADS> struct TopLds {
    static constexpr int WAVES = THREADS / 64, CAP = THREADS == 64 ? 512 : 256;
    unsigned long long key[WAVES][CAP], best[WAVES][CAPGNN_TOP_MAX];
    int32_t noted[WAVES][CAP];      // classes whose keys are not formed yet stand here, in their keys' places
    uint32_t maxima[THREADS];
    int kept[WAVES];
    uint32_t bound;
};

// the float just below every logit of order o and more; NaN (no logit is <= it) where there is none
__device__ __forceinline__ float just_below(uint32_t o) {
    uint32_t b = o - 1u;
    if (b == 0x7fffffffu) b = 0x7ffffffeu;      // below both zeros
    return o <= 0x007fffffu ? __uint_as_float(0x7fc00000u) : order_logit(b);
}

// how many of n keys (n even, 16 bytes aligned) are larger
__device__ __forceinline__ int larger_keys(const unsigned long long *key, int n, unsigned long long own) {
    const ulonglong2 *q = reinterpret_cast<const ulonglong2 *>(key);
    int larger = 0;
#pragma unroll 4
    for (int j = 0; j < n / 2; ++j) {
        const ulonglong2 v = q[j];
        larger += (v.x > own) + (v.y > own);
    }
    return larger;
}

template <int THREADS> struct Top {
    static constexpr int CAP = TopLds<THREADS>::CAP, WAVES = THREADS / 64;
    TopLds<THREADS> &l;
    int k, kept = 0, formed = 0;                        // classes in the wave's list, of which so many have their keys
    int again = -1;                                     // the first tile that has not been worked on
    float below = __uint_as_float(0x7fc00000u);         // a logit is a candidate unless it is <= this

    __device__ Top(TopLds<THREADS> &lds, int k_) : l(lds), k(k_) {}
    static __device__ __forceinline__ int wave() { return THREADS == 64 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
    static __device__ __forceinline__ int lane() { return threadIdx.x & 63; }

    __device__ void raise(uint32_t order, bool inclusive) {
        const float f = inclusive ? just_below(order) : order_logit(order);
        if (f == f && !(f <= below)) below = f;         // (from NaN to anything, to NaN never)
    }

    // The k-th largest of N threads' maxima (k <= N), or hardly less: the last bits of the order are the thread's number, so that no two are
    // equal and one comparison each ranks them.  N = THREADS: of the workgroup; 64: of the wave.
    template <int N> __device__ uint32_t kth_maximum(float tmax) {
        const int t = N == 64 ? lane() : threadIdx.x;
        uint32_t *maxima = N == 64 ? l.maxima + wave() * 64 : l.maxima;
        const uint32_t mine = (logit_order(tmax) & ~(N - 1u)) | t;
        maxima[t] = mine;
        N == 64 ? wave_sync() : __syncthreads();
        int larger = 0;
        const uint4 *q = reinterpret_cast<const uint4 *>(maxima);
#pragma unroll 4
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = q[i];
            larger += v.x > mine;
            larger += v.y > mine;
            larger += v.z > mine;
            larger += v.w > mine;
        }
        if constexpr (N == 64) {
            const unsigned long long at = __ballot(larger == k - 1);
            return __shfl(mine, __ffsll(at) - 1) & ~(N - 1u);
        } else {
            if (larger == k - 1) l.bound = mine & ~(N - 1u);
            __syncthreads();
            return l.bound;                             // (written once a row: a barrier lies before the next time)
        }
    }

    // Only classes are noted during the scan, one read of their logits (out of the caches) forms the keys of many.
    template <bool BF16> __device__ void form(const char *z) {
        wave_sync();
#pragma unroll 1
        for (int i = formed + lane(); i < kept; i += 64) {
            const int j = l.noted[wave()][i];
            l.key[wave()][i] = logit_key(ld_logit<BF16>(z, j), j);
        }
        formed = kept;
    }

    // The same of the maxima of the wave's NV vectors of every lane, bit by bit: seldom more than a few logits behind the exact k-th largest.
    template <int NV> __device__ uint32_t kth_vector(const float (&vmax)[NV]) {
        uint32_t o[NV], T = 0;
#pragma unroll
        for (int i = 0; i < NV; ++i) o[i] = logit_order(vmax[i]);
#pragma unroll 1
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t t = T | 1u << bit;
            int c = 0;
#pragma unroll
            for (int i = 0; i < NV; ++i) c += __popcll(__ballot(o[i] >= t));
            if (c >= k) T = t;
        }
        return T;
    }

    // cuts the wave's list to its k largest, in descending order
    template <bool BF16> __device__ void cut(const char *z) {
        form<BF16>(z);
        unsigned long long *key = l.key[wave()], *best = l.best[wave()];
        const int n = kept;
        if (lane() == 0 && (n & 1)) key[n] = 0;
        wave_sync();
#pragma unroll 1
        for (int i = lane(); i < n; i += 64) {
            const unsigned long long own = key[i];
            const int at = larger_keys(key, n + 1 & ~1, own);
            if (at < k) best[at] = own;
        }
        wave_sync();
        kept = formed = n < k ? n : k;
        if (lane() < kept) key[lane()] = best[lane()];
        if (kept == k) raise(static_cast<uint32_t>(best[k - 1] >> 32), false);
        wave_sync();
    }

    // one class of every lane that has one; false if the list does not hold them
    __device__ bool append(bool has, int j) {
        const unsigned long long lanes = __ballot(has);
        const int count = __popcll(lanes);
        if (kept + count > CAP) return false;
        const int at = kept + __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(lanes >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(lanes), 0));
        if (has) l.noted[wave()][at] = j;
        kept += count;
        return true;
    }

    // the tile of NV vectors a thread, as the row's scan has read them; classes [from, end) are in the tile
    template <bool BF16, int NV>
    __device__ void tile(raw16 (&r)[NV], const float (&vmax)[NV], float tmax, const char *z, int from, int end, bool first) {
        typedef Raw<BF16> R;
        constexpr int V = R::V, HALF = NV * V / 2;
        static_assert(HALF <= 32 && NV % 2 == 0, "a thread's logits of a tile are two words of bits");
        if (first && end - from > THREADS / 64 * CAP / 2) raise(THREADS == 64 && k > 32 ? kth_vector<NV>(vmax) : kth_maximum<THREADS>(tmax), true);
        if (again >= 0) return;
        const int before = kept;
#pragma unroll 1
        for (int attempt = 0; attempt < 2; ++attempt) {
            const int tid = thread_anew();
            uint32_t passed[2] = {0, 0};        // bit i * V + e of a half: class from + (i * THREADS + tid) * V + e
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (!__any(!(vmax[i] <= below))) continue;
                forget(r[i]);
                uint32_t p = 0;
#pragma unroll
                for (int e = 0; e < V; ++e) p |= !(R::get(r[i], e) <= below) ? 1u << e : 0u;
                const int own = from + (i * THREADS + tid) * V;
                if (__any(own + V > end)) p = own >= end ? 0u : own + V > end ? p >> (own + V - end) : p;    // (the row's last vectors start earlier)
                passed[2 * i / NV] |= p << i % (NV / 2) * V;
            }
            bool fits = true;
#pragma unroll
            for (int h = 0; h < 2; ++h)
                while (fits && __any(passed[h] != 0)) {
                    const bool has = passed[h] != 0;
                    const int b = __ffs(passed[h]) - 1;
                    passed[h] &= passed[h] - 1;
                    fits = append(has, from + ((h * (NV / 2) + b / V) * THREADS + tid) * V + b % V);
                }
            if (fits) {
                if (kept > CAP / 2) cut<BF16>(z);
                return;
            }
            kept = before;
            if (attempt == 0) raise(kth_vector<NV>(vmax), true);
        }
        again = from;
    }

    // The tiles from `again` on, out of memory (kept out of the scan, whose registers it would take): those with more candidates than the list
    // holds by the exact k-th largest key of the wave's share (4096 x 131072 equal logits, k = 64: 2.0 ms; random ones 0.31).
    template <bool BF16, int NV> __device__ void rest(const char *z, int row_end) {
        constexpr int V = Raw<BF16>::V, TILE = THREADS * NV * V;
#pragma unroll 1
        for (int from = again; from < row_end; from += TILE) {
            const int end = row_end - from < TILE ? row_end : from + TILE, mine = from + wave() * 64 * V;
            auto each = [&](auto f) {
#pragma unroll 1
                for (int q = lane(); q < NV * 64 * V; q += 64) {        // (whole waves)
                    const int j = mine + q / (64 * V) * (THREADS * V) + q % (64 * V);
                    f(j < end ? ld_logit<BF16>(z, j) : 0.f, j, j < end);
                }
            };
            auto count = [&](auto in) {             // (eight loads in flight)
                int c = 0;
#pragma unroll 1
                for (int q = lane(); q < NV * 64 * V; q += 8 * 64) {
                    float x[8];
                    int j[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        j[u] = mine + (q + u * 64) / (64 * V) * (THREADS * V) + (q + u * 64) % (64 * V);
                        x[u] = j[u] < end ? ld_logit<BF16>(z, j[u]) : 0.f;
                    }
#pragma unroll
                    for (int u = 0; u < 8; ++u) c += j[u] < end && in(x[u], j[u]);
                }
                return wave_all(c, OpSum());
            };
            const float limit = below;
            const int all = count([&](float x, int) { return !(x <= limit); }), want = all < k ? all : k;
            uint32_t T = 0;
            int equal = all;                // how many of order T are wanted
            if (kept + all > CAP) {
                // the k-th largest of the lanes' maxima, if fewer than k are above it (many equal logits); else bit by bit
                float most[1] = {-INFINITY};
                each([&](float x, int, bool there) { if (there) most[0] = max_of(most[0], x); });
                T = kth_vector<1>(most);
                int above = count([&](float x, int) { return logit_order(x) > T; });
                if (above >= want) {
                    T = 0;
                    for (int bit = 31; bit >= 0; --bit) {
                        const uint32_t t = T | 1u << bit;
                        if (count([&](float x, int) { return logit_order(x) >= t; }) >= want) T = t;
                    }
                    above = count([&](float x, int) { return logit_order(x) > T; });
                }
                equal = want - above;
            }
            // classes come in ascending order: the first ones of order T are taken
            each([&](float x, int j, bool there) {
                const uint32_t o = logit_order(x);
                const unsigned long long same = __ballot(there && !(x <= limit) && o == T);
                const int before = __builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(same >> 32), __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(same), 0));
                append(there && !(x <= limit) && (o > T || (o == T && before < equal)), j);      // k at most, or all, which the list holds
                equal -= __popcll(same);
            });
            if (kept > CAP / 2 || kept + all > CAP) cut<BF16>(z);
        }
    }

    // The row's k largest in descending order, in l.best[0]; how many there are.  Barriers before and after.
    template <bool BF16, int NV> __device__ int finish(const char *z, int row_end) {
        if (again >= 0) rest<BF16, NV>(z, row_end);
        if constexpr (WAVES == 1) {
            cut<BF16>(z);
            return kept;
        } else {
            form<BF16>(z);
            if (lane() == 0) {
                l.kept[wave()] = kept;
                if (kept & 1) l.key[wave()][kept] = 0;
            }
            __syncthreads();
            int total = 0, n[WAVES];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { n[w] = l.kept[w]; total += n[w]; }
#pragma unroll 1
            for (int i = lane(); i < kept; i += 64) {
                const unsigned long long own = l.key[wave()][i];
                int at = 0;
#pragma unroll 1
                for (int w = 0; w < WAVES; ++w) at += larger_keys(l.key[w], l.kept[w] + 1 & ~1, own);
                if (at < k) l.best[0][at] = own;
            }
            __syncthreads();
            return total < k ? total : k;
        }
    }
};

// One workgroup (or wave) per row, or per part of a row (parts > 1): running maximum and sums in every thread, one pass over the logits, eight
// 16-byte loads a thread in flight, which read -> sums -> threshold out of registers; sixteen waves on a compute unit cover one another's waits.
// Bound by HBM: 4096 x 131072 bf16 without top classes 5.3 TB/s (200 us), with 8 of them 217, with 64 312 us, where the instructions of the
// threshold and the ranking show (VALU issue about 60 % of the time).
constexpr int ANSWER_VECTORS = 8;       // 16-byte loads that a thread has in flight

struct AnswerParts {
    int parts;                      // of a row
    int64_t chunk;                  // classes of one
    float4 *sums;                   // [n][parts]: maximum, sum, sum of e u
    unsigned long long *keys;       // [n][parts][k], 0 = none
};

template <bool BF16, int THREADS, bool ENT>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4))) void answers_rows_kernel(AnswerArgs a, AnswerParts w) {
    typedef Raw<BF16> R;
    constexpr int NV = ANSWER_VECTORS, TILE = THREADS * NV * R::V;
    __shared__ __align__(16) TopLds<THREADS> lds;
    __shared__ float red[THREADS / 64];
    for (int64_t job = blockIdx.x; job < a.n * w.parts; job += gridDim.x) {
        const int64_t row = w.parts > 1 ? job / w.parts : job;
        const int part = w.parts > 1 ? static_cast<int>(job % w.parts) : 0;
        if (a.mask && !a.mask[row]) {
            if (part == 0) masked_out_row(a, row, THREADS);
            continue;
        }
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        const int lo = static_cast<int>(part * w.chunk);
        const int hi = static_cast<int>(lo + w.chunk < a.C ? lo + w.chunk : a.C);
        Top<THREADS> top(lds, a.k);
        float m = -INFINITY, s = 0.f, e1 = 0.f;
        for (int t0 = lo; t0 < hi; t0 += TILE) {
            raw16 r[NV];
            float vmax[NV], tmax = -INFINITY;
            const int tid = thread_anew();
            int start;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (t0 + (i + 1) * THREADS * R::V <= hi) r[i] = R::load(z, t0 + (i * THREADS + tid) * R::V);
                else if (t0 + i * THREADS * R::V < hi) r[i] = R::load_until(z, t0 + (i * THREADS + tid) * R::V, hi, &start);
                else r[i] = raw16{R::BARRED, R::BARRED, R::BARRED, R::BARRED};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                vmax[i] = R::get(r[i], 0);
                if (t0 + i * THREADS * R::V >= hi) continue;          // (the same for all threads)
#pragma unroll
                for (int e = 1; e < R::V; ++e) vmax[i] = max_of(vmax[i], R::get(r[i], e));
                tmax = max_of(tmax, vmax[i]);
            }
            const float m_new = max_of(m, tmax), ref = safe_max(m_new);
            const float du = (m - ref) * a.t.L, f = exp2_raw(du);
            if constexpr (ENT) e1 = f * fmaf(s, fmaxf(du, -160.f), e1);
            s *= f;
            m = m_new;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (t0 + i * THREADS * R::V >= hi) continue;
                forget(r[i]);
#pragma unroll
                for (int e = 0; e < R::V; ++e) {
                    const float u = (R::get(r[i], e) - ref) * a.t.L, x = exp2_raw(u);
                    s += x;
                    if constexpr (ENT) e1 = fmaf(x, fmaxf(u, -160.f), e1);
                }
            }
            if (a.k) top.template tile<BF16>(r, vmax, tmax, z, t0, hi - t0 < TILE ? hi : t0 + TILE, t0 == lo);
        }
        // a thread's sums, taken from its own maximum to the row's
        const float M = group_all<THREADS>(m, red, OpMax()), ref = safe_max(M);
        const float du = (m - ref) * a.t.L, f = exp2_raw(du);
        if constexpr (ENT) e1 = group_all<THREADS>(f * fmaf(s, fmaxf(du, -160.f), e1), red, OpSum());
        s = group_all<THREADS>(s * f, red, OpSum());
        const int found = a.k ? top.template finish<BF16, NV>(z, hi) : 0;
        if (w.parts > 1) {
            if (threadIdx.x == 0) w.sums[job] = make_float4(M, s, e1, 0.f);
            for (int i = threadIdx.x; i < a.k; i += THREADS) w.keys[job * a.k + i] = i < found ? lds.best[0][i] : 0;
        } else {
            const RowEnd end(M, s, a.t.inv_T);
            if (threadIdx.x == 0) {
                if (a.entropy) a.entropy[row] = end.entropy(s, e1);
                if (a.stats) { a.stats[2 * row] = M; a.stats[2 * row + 1] = end.ln_s; }
            }
            for (int i = threadIdx.x; i < a.m; i += THREADS) {
                const int c = a.ids[row * a.ldi + i];
                a.logp[row * a.ldp + i] = c >= 0 && c < a.C ? end.logp(ld_logit<BF16>(z, c)) : 0.f;
            }
            for (int i = threadIdx.x; i < a.k; i += THREADS) {
                const unsigned long long key = lds.best[0][i];
                if (a.top_ids) a.top_ids[row * a.ldt + i] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(key));
                if (a.top_logp) a.top_logp[row * a.ldt + i] = end.logp(order_logit(static_cast<uint32_t>(key >> 32)));
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ few classes (NARROW_C) and at most NARROW_TOP top ones
// Pass 1 keeps the k largest logits of a lane sorted, one median of three per place and logit (lanes of a row merge theirs); pass 2 forms the
// sums, and a class that reaches the k-th largest finds its place among them as the number of those that are larger.  Rows with equal
// logits among the k largest, or with NaN, are gone over once more by one lane, class by class.  The places of the wave's rows are
// written out together.  612000 x 47, k = 5: 53 us, 2.8 TB/s, bound by instruction issue and LDS latency in about equal parts; without top
// classes 28 us, 4.1 TB/s.  (Ranking the classes found against one another, out of LDS: 131 us.)
// 100000 rows, this kernel with k = 8 against a wave a row with 9, us: 20 f32 12 / 139, 47 f32 15 / 149, bf16 22 / 178, 100 f32 25 / 218, 256 f32
// 44 / 582, bf16 93 / 617.
constexpr int NARROW_TOP = 8;
template <bool BF16, bool ENT, bool TOP>
__global__ __launch_bounds__(64 * NARROW_WAVES) __attribute__((amdgpu_waves_per_eu(4))) void answers_narrow_kernel(AnswerArgs a, NarrowShape s) {
    extern __shared__ __align__(16) char lds_all[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const size_t per_wave = s.lds_wave + 64 * (sizeof(float2) + NARROW_TOP);
    float *tile = reinterpret_cast<float *>(lds_all + wave * per_wave);
    float2 *ends = reinterpret_cast<float2 *>(lds_all + wave * per_wave + s.lds_wave);        // of every row: maximum, ln of the sum
    uint8_t *places = reinterpret_cast<uint8_t *>(ends + 64);
    const int G = 1 << s.lg, sub = lane & (G - 1), C = s.C, mine = lane >> s.lg;
    const float *z = tile + mine * s.pitch;
    uint8_t *place = places + mine * NARROW_TOP;
    const int64_t step = static_cast<int64_t>(gridDim.x) * NARROW_WAVES * s.rows;
    int64_t row0 = (static_cast<int64_t>(blockIdx.x) * NARROW_WAVES + wave) * s.rows;
    const int magic = a.k ? (65536 + a.k - 1) / a.k : 0;
    narrow_ends(s, tile, lane);
    NarrowLoad<BF16> next;
    if (row0 < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0);
    for (; row0 < a.n; row0 += step) {
        next.put(s, tile);
        wave_sync();
        if (row0 + step < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0 + step);
        const int64_t row = row0 + mine;
        const bool in = row < a.n, on = in && (!a.mask || a.mask[row]);
        const int given = a.m && on && sub < a.m ? a.ids[row * a.ldi + sub] : -1;
        float v[NARROW_TOP], m = -INFINITY;
        if constexpr (TOP) {
#pragma unroll
            for (int i = 0; i < NARROW_TOP; ++i) v[i] = -INFINITY;
            auto insert = [&](float x) {
#pragma unroll
                for (int i = NARROW_TOP - 1; i > 0; --i) v[i] = __builtin_amdgcn_fmed3f(v[i - 1], v[i], x);
                v[0] = max_of(v[0], x);
            };
            for (int b = 0; b < s.each; b += NARROW_BATCH) {
                float x[NARROW_BATCH];
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[sub + (b + i) * G];
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) insert(x[i]);
            }
            for (int off = 1; off < G; off <<= 1) {
                float o[NARROW_TOP];
#pragma unroll
                for (int i = 0; i < NARROW_TOP; ++i) o[i] = __shfl_xor(v[i], off);
#pragma unroll
                for (int i = 0; i < NARROW_TOP; ++i) insert(o[i]);
            }
            m = v[0];
        } else {
            for (int b = 0; b < s.each; b += NARROW_BATCH)
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) m = max_of(m, z[sub + (b + i) * G]);
            for (int off = 1; off < G; off <<= 1) m = max_of(m, __shfl_xor(m, off));
        }
        float kth = 0.f;
        bool twice = false;                 // two of the k largest, or one and the next, are equal
        if constexpr (TOP) {
#pragma unroll
            for (int i = 0; i < NARROW_TOP; ++i) {
                if (i == a.k - 1) kth = v[i];
                if (i > 0) twice = twice || (i < a.k && v[i] == v[i - 1]);
            }
#pragma unroll
            for (int i = 0; i < NARROW_TOP; ++i) if (i >= a.k) v[i] = -INFINITY;      // (no place of the k)
        }
        const float ref = safe_max(m);
        float sum = 0.f, e1 = 0.f;
        uint32_t hits = 0;                  // the lane's classes that reach the k-th largest, a bit each
        for (int b = 0; b < s.each; b += NARROW_BATCH) {
            float x[NARROW_BATCH];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[sub + (b + i) * G];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) {
                const float u = (x[i] - ref) * a.t.L, e = exp2_raw(u);
                sum += e;
                if constexpr (ENT) e1 = fmaf(e, fmaxf(u, -160.f), e1);
                if constexpr (TOP) hits |= x[i] >= kth ? 1u << (b + i) : 0u;
            }
        }
        int reached = 0;
        if constexpr (TOP) {
            const int own = (C - sub + G - 1) >> s.lg;          // (behind the row's end: -inf, which a k-th largest may be as well)
            hits &= own < 32 ? (1u << own) - 1u : ~0u;
            reached = __popc(hits);
            while (__any(hits != 0)) {
                const int i = __ffs(hits) - 1;
                const float x = z[i < 0 ? sub : sub + i * G];
                int larger = 0;
#pragma unroll
                for (int q = 0; q < NARROW_TOP; ++q) larger += v[q] > x;
                if (hits) place[larger & (NARROW_TOP - 1)] = static_cast<uint8_t>(sub + i * G);         // (8 only next to a NaN)
                hits &= hits - 1;
            }
        }
        for (int off = 1; off < G; off <<= 1) {
            sum += __shfl_xor(sum, off);
            if constexpr (ENT) e1 += __shfl_xor(e1, off);
            if constexpr (TOP) reached += __shfl_xor(reached, off);
        }
        const RowEnd end(m, sum, a.t.inv_T);
        if (in && sub == 0) {
            if (a.entropy) a.entropy[row] = on ? end.entropy(sum, e1) : 0.f;
            if (a.stats) { a.stats[2 * row] = on ? m : 0.f; a.stats[2 * row + 1] = on ? end.ln_s : 0.f; }
        }
        if (in && sub < a.m) a.logp[row * a.ldp + sub] = given >= 0 && given < C ? end.logp(z[given]) : 0.f;
        if (in)
            for (int i = sub + G; i < a.m; i += G) {
                const int c = on ? a.ids[row * a.ldi + i] : -1;
                a.logp[row * a.ldp + i] = c >= 0 && c < C ? end.logp(z[c]) : 0.f;
            }
        if constexpr (TOP) {
            const bool nan = !(sum == sum), again = on && (twice || reached != a.k || nan);
            if (sub == 0) ends[mine] = make_float2(on ? end.m0 : -INFINITY, end.ln_s);        // (-inf: a row that is masked out)
            if (__any(again)) {
                wave_sync();
                if (again && sub == 0) {
                    unsigned long long last = ~0ull;
                    if (nan) {
                        for (int i = 0; i < a.k; ++i) {
                            unsigned long long best = 0;
                            for (int j = 0; j < C; ++j) {
                                const unsigned long long key = logit_key(z[j], j);
                                if (key < last && key > best) best = key;
                            }
                            last = best;
                            place[i] = static_cast<uint8_t>(0xffffffffu - static_cast<uint32_t>(best));
                        }
                    } else {
                        uint32_t taken = 0;         // equal logits: the first of their places that is open
                        for (int b = 0; b < C; b += NARROW_BATCH) {
                            float x[NARROW_BATCH];
#pragma unroll
                            for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[b + i < s.pitch ? b + i : s.pitch - 1];
#pragma unroll
                            for (int i = 0; i < NARROW_BATCH; ++i)
                                if (x[i] >= kth && b + i < C) {
                                    int larger = 0;
#pragma unroll
                                    for (int q = 0; q < NARROW_TOP; ++q) larger += v[q] > x[i];
                                    const uint32_t open = ~taken & (~0u << larger) & ((1u << a.k) - 1u);
                                    if (open) place[__ffs(open) - 1] = static_cast<uint8_t>(b + i);
                                    taken |= open & (0u - open);
                                }
                        }
                    }
                }
            }
            wave_sync();
            for (int i = lane; i < s.rows * a.k; i += 64) {
                const int r = i * magic >> 16, p = i - r * a.k;
                if (row0 + r >= a.n) break;
                const float2 e = ends[r];
                const bool there = e.x != -INFINITY;
                const int c = places[r * NARROW_TOP + p];
                if (a.top_ids) a.top_ids[(row0 + r) * a.ldt + p] = there ? c : -1;
                if (a.top_logp)
                    a.top_logp[(row0 + r) * a.ldt + p] = !there ? 0.f : e.y == -INFINITY ? -INFINITY : (tile[r * s.pitch + c] - e.x) * a.t.inv_T - e.y;
            }
        }
        wave_sync();
    }
}

// The parts of a row put together: sums from the parts' maxima to the row's, and the k largest of the parts' k largest.  One row of 40000
// classes, k = 20: 15 us in two launches, both latency (one workgroup a row: 60 us and more of one compute unit's loads).
constexpr int ANSWER_PARTS = 64;
template <bool BF16>
__global__ __launch_bounds__(256) void answers_join_kernel(AnswerArgs a, AnswerParts w) {
    constexpr int OWN = ANSWER_PARTS * CAPGNN_TOP_MAX / 256;
    __shared__ __align__(16) unsigned long long key[ANSWER_PARTS * CAPGNN_TOP_MAX / 4], maxima[256], best_of[CAPGNN_TOP_MAX];
    __shared__ unsigned long long shared_bound;
    __shared__ int kept;
    __shared__ float red[4];
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        if (a.mask && !a.mask[row]) continue;
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        const int i = threadIdx.x;
        unsigned long long own[OWN], best = 0;
#pragma unroll
        for (int o = 0; o < OWN; ++o) {
            own[o] = i + o * 256 < w.parts * a.k ? w.keys[row * w.parts * a.k + i + o * 256] : 0;
            best = own[o] > best ? own[o] : best;
        }
        const float4 p = i < w.parts ? w.sums[row * w.parts + i] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        const float M = group_all<256>(p.x, red, OpMax());
        const float du = (p.x - safe_max(M)) * a.t.L, f = exp2_raw(du);
        const float s = group_all<256>(p.y * f, red, OpSum());
        const float e1 = group_all<256>(f * fmaf(p.y, fmaxf(du, -160.f), p.z), red, OpSum());
        const RowEnd end(M, s, a.t.inv_T);
        if (i == 0) {
            if (a.entropy) a.entropy[row] = end.entropy(s, e1);
            if (a.stats) { a.stats[2 * row] = M; a.stats[2 * row + 1] = end.ln_s; }
        }
        if (i < a.m) {
            const int c = a.ids[row * a.ldi + i];
            a.logp[row * a.ldp + i] = c >= 0 && c < a.C ? end.logp(ld_logit<BF16>(z, c)) : 0.f;
        }
        if (a.k) {
            // keys at least as large as the k-th largest of the threads' maxima: k threads have them, OWN at most each
            maxima[i] = best;
            if (i == 0) { shared_bound = 1; kept = 0; }
            __syncthreads();
            if (w.parts * a.k > 256 && best && larger_keys(maxima, 256, best) == a.k - 1) shared_bound = best;
            __syncthreads();
            const unsigned long long bound = shared_bound;
#pragma unroll
            for (int o = 0; o < OWN; ++o)
                if (own[o] >= bound) key[atomicAdd(&kept, 1)] = own[o];
            __syncthreads();
            const int n = kept;
            if (i == 0 && (n & 1)) key[n] = 0;
            __syncthreads();
            for (int q = i; q < n; q += 256) {
                const unsigned long long mine = key[q];
                const int at = larger_keys(key, n + 1 & ~1, mine);
                if (at < a.k) best_of[at] = mine;
            }
            __syncthreads();
            if (i < a.k) {
                const unsigned long long k1 = best_of[i];
                if (a.top_ids) a.top_ids[row * a.ldt + i] = static_cast<int32_t>(0xffffffffu - static_cast<uint32_t>(k1));
                if (a.top_logp) a.top_logp[row * a.ldt + i] = end.logp(order_logit(static_cast<uint32_t>(k1 >> 32)));
            }
            __syncthreads();
        }
    }
}

// Few long rows are cut into parts, about a thousand workgroups in all and ANSWER_PART_LEAST classes or more each; one workgroup a row is
// as fast where the second launch costs what the parts save.  Parts against whole rows, us, k = 20: 1 x 24000 f32 15.7 / 14.5, 1 x 40000
// f32 15.5 / 19.7, bf16 15.1 / 16.0, 1 x 150000 f32 18.5 / 57.9, 128 x 40000 f32 20.9 / 20.9, 128 x 65536 f32 21.8 / 34.2, 200 x 40000
// f32 21.8 / 21.3, 200 x 65536 bf16 23.0 / 22.0, 300 x 9000 f32 19.0 / 12.4, 300 x 50000 f32 28.2 / 28.4.
constexpr int ANSWER_PART_LEAST = 2048, ANSWER_WORKGROUPS = 1024, ANSWER_WAVE_C = 16384;
constexpr int ANSWER_LONG = 32768, ANSWER_FEW = 256;
static int answer_parts(int64_t n, int C, int64_t *chunk) {
    if (C < ANSWER_LONG || C / ANSWER_FEW < n) { *chunk = C; return 1; }
    int64_t parts = std::min<int64_t>(std::min<int64_t>(ANSWER_PARTS, ANSWER_WORKGROUPS / std::max<int64_t>(n, 1)), (C + ANSWER_PART_LEAST - 1) / ANSWER_PART_LEAST);
    if (parts <= 1) { *chunk = C; return 1; }
    *chunk = (C + parts - 1) / parts;
    *chunk = (*chunk + 511) / 512 * 512;
    return static_cast<int>((C + *chunk - 1) / *chunk);
}

struct AnswerGradArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const float *stats, *entropy;
    const int32_t *ids; int64_t ldi; int m;
    const float *dlogp; int64_t lddp;
    const float *dentropy;
    char *dZ; int64_t lddz;
};

// What a row's logits are turned into their gradients with: dz = (-p (G + h (ln p + H)) + g) / T, g for the given classes.
struct GradRow {
    float m0, ln_s, inv_s, G, h, H;
    bool none;                      // masked out, or no class allowed

    // (nothing is read under a condition on what was read before: one wait for all of it)
    __device__ __forceinline__ void read(const AnswerGradArgs &a, int64_t row) {
        const bool on = !a.mask || a.mask[row];
        const float top = a.stats[2 * row], ln = a.stats[2 * row + 1], dh = a.dentropy ? a.dentropy[row] : 0.f, e = a.dentropy ? a.entropy[row] : 0.f;
        none = !on || ln == -INFINITY;
        ln_s = none ? 0.f : ln;
        m0 = none ? 0.f : top;
        h = none ? 0.f : dh;
        H = none ? 0.f : e;
        inv_s = expf(-ln_s);
    }
    template <bool ENT, bool EXACT = true> __device__ __forceinline__ float base(float z, const TempScale &t) const {
        const float d = difference(z, m0, t), p = exp_scaled<EXACT>(d, t) * inv_s;
        return -p * (ENT ? fmaf(h, fmaf(d, t.inv_T, H - ln_s), G) : G);
    }
};

// Workgroups of THREADS take CHUNK classes of a row each; the sums of the row come with the call.  The given classes' own terms follow
// the rest of the chunk, behind a barrier, from the thread that holds the first mention of the class.  Bound by HBM: 4096 x 65536 bf16
// 188 us, 5.7 TB/s read and written.
constexpr int GRAD_VECTORS = 4;
template <bool BF16, bool DBF16, int THREADS, bool ENT>
__global__ __launch_bounds__(THREADS) void answers_grad_rows_kernel(AnswerGradArgs a, int chunks) {
    typedef Raw<BF16> R;
    constexpr int V = R::V, CHUNK = THREADS * GRAD_VECTORS * V, MOST = CAPGNN_GIVEN_MAX / THREADS;
    __shared__ int32_t id[CAPGNN_GIVEN_MAX];
    __shared__ float g[CAPGNN_GIVEN_MAX];
    __shared__ float red[THREADS / 64];
    for (int64_t job = blockIdx.x; job < a.n * chunks; job += gridDim.x) {
        const int64_t row = chunks > 1 ? job / chunks : job;
        const int lo = chunks > 1 ? static_cast<int>(job % chunks) * CHUNK : 0, hi = a.C - lo < CHUNK ? a.C : lo + CHUNK;
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        char *dz = a.dZ + row * a.lddz * (DBF16 ? 2 : 4);
        GradRow w;
        w.read(a, row);
        raw16 r[GRAD_VECTORS];
        int from = 0;
        if (!a.mask || a.mask[row])         // (before what the row's sums say)
#pragma unroll
            for (int i = 0; i < GRAD_VECTORS; ++i)
                if (lo + i * THREADS * V < hi) r[i] = R::load_until(z, lo + (i * THREADS + static_cast<int>(threadIdx.x)) * V, hi, &from);
        int mine[MOST];
        float zc[MOST], G = 0.f;
#pragma unroll
        for (int o = 0; o < MOST; ++o) {
            const int i = threadIdx.x + o * THREADS;
            mine[o] = -1;
            if (o * THREADS >= a.m) break;
            if (i < a.m) {
                const int c = w.none ? -1 : a.ids[row * a.ldi + i];
                const float read = a.dlogp[row * a.lddp + i];
                const bool ok = c >= 0 && c < a.C;
                const float gi = ok ? read : 0.f;
                id[i] = ok ? c : -1;
                g[i] = gi;
                G += gi;
                if (c >= lo && c < hi) {
                    mine[o] = c;
                    zc[o] = ld_logit<BF16>(z, c);
                }
            }
        }
        w.G = a.m ? group_all<THREADS>(G, red, OpSum()) : 0.f;
#pragma unroll
        for (int i = 0; i < GRAD_VECTORS; ++i) {
            const int j = lo + (i * THREADS + static_cast<int>(threadIdx.x)) * V;
            if (lo + i * THREADS * V >= hi) break;
            if (j >= hi) continue;
            float o[V];
            const int shift = j + V <= hi ? 0 : j + V - hi;         // a row's last vector starts earlier than j by that
#pragma unroll
            for (int e = 0; e < V; ++e) o[e] = w.none ? 0.f : w.base<ENT, !DBF16>(R::get(r[i], e), a.t) * a.t.inv_T;
            if (shift == 0) st_vector<DBF16>(dz, j, o);
            else
#pragma unroll
                for (int e = 0; e < V; ++e) if (e >= shift) st_grad<DBF16>(dz, hi - V + e, o[e]);
        }
        if (a.m) {
            __syncthreads();
#pragma unroll
            for (int o = 0; o < MOST; ++o) {
                if (o * THREADS >= a.m) break;
                const int at = threadIdx.x + o * THREADS, c = mine[o];
                if (c < 0) continue;
                bool first = true;
                float sum = 0.f;
                for (int i = 0; i < a.m; ++i)
                    if (id[i] == c) {
                        first = first && i >= at;
                        sum += g[i];
                    }
                if (first) st_grad<DBF16>(dz, c, (w.base<ENT>(zc[o], a.t) + sum) * a.t.inv_T);
            }
            __syncthreads();
        }
    }
}

// Few classes: the rows' gradients take their logits' places in LDS and leave in whole vectors.  60000 x 41: 9 us, one or two
// rounds of rows a wave, each a chain of the row's statistics, ids and logits.
template <bool BF16, bool DBF16, bool ENT>
__global__ __launch_bounds__(64 * NARROW_WAVES) void answers_grad_narrow_kernel(AnswerGradArgs a, NarrowShape s) {
    extern __shared__ __align__(16) char lds_all[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float *tile = reinterpret_cast<float *>(lds_all + wave * s.lds_wave);
    const int G = 1 << s.lg, sub = lane & (G - 1), C = s.C;
    float *z = tile + (lane >> s.lg) * s.pitch;
    const int64_t step = static_cast<int64_t>(gridDim.x) * NARROW_WAVES * s.rows;
    int64_t row0 = (static_cast<int64_t>(blockIdx.x) * NARROW_WAVES + wave) * s.rows;
    NarrowLoad<BF16> next;
    if (row0 < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0);
    for (; row0 < a.n; row0 += step) {
        const int64_t row = row0 + (lane >> s.lg) < a.n ? row0 + (lane >> s.lg) : a.n - 1;
        GradRow w;
        w.read(a, row);
        int c0 = a.m ? a.ids[row * a.ldi] : -1;                 // the first class given (often the only one), and its gradient
        const float g0 = a.m ? a.dlogp[row * a.lddp] : 0.f;
        if (c0 >= C || w.none) c0 = -1;
        w.G = c0 >= 0 ? g0 : 0.f;
        for (int i = 1; i < a.m; ++i) {
            const int c = a.ids[row * a.ldi + i];
            const float g = a.dlogp[row * a.lddp + i];
            if (c >= 0 && c < C) w.G += g;
        }
        next.put(s, tile);
        wave_sync();
        if (row0 + step < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0 + step);
        for (int b = 0; b < s.each; b += NARROW_BATCH) {
            float x[NARROW_BATCH];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[sub + (b + i) * G];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) {
                const float g = w.none ? 0.f : w.base<ENT, !DBF16>(x[i], a.t) * a.t.inv_T;
                if (sub + (b + i) * G < C) z[sub + (b + i) * G] = g;
            }
        }
        wave_sync();
        if (sub == 0 && !w.none) {          // one lane a row: the same class may be given again
            if (c0 >= 0) z[c0] = fmaf(g0, a.t.inv_T, z[c0]);
            for (int i = 1; i < a.m; ++i) {
                const int c = a.ids[row * a.ldi + i];
                if (c >= 0 && c < C) z[c] = fmaf(a.dlogp[row * a.lddp + i], a.t.inv_T, z[c]);
            }
        }
        wave_sync();
        narrow_store<BF16, DBF16>(s, tile, a.dZ, a.lddz, a.n, row0, false);
        wave_sync();
    }
}

}  // namespace capgnn

using namespace capgnn;

extern "C" size_t capgnn_logprobs_workspace_bytes(int64_t n, int C, int k) {
    if (n <= 0 || C <= 0 || k < 0) return 0;
    int64_t chunk;
    const int parts = answer_parts(n, C, &chunk);
    if (parts == 1) return 0;
    return align_up(sizeof(float4) * n * parts, 256) + align_up(sizeof(unsigned long long) * n * parts * k, 256);
}

extern "C" int capgnn_logprobs(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, float temperature, const uint8_t *mask,
                               const int32_t *ids, int64_t ldi, int m, float *logp, int64_t ldp, float *entropy, float *stats,
                               int k, int32_t *top_ids, float *top_logp, int64_t ldt, void *ws, size_t ws_bytes, void *stream) {
    if (z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) CG_FAIL(CAPGNN_EINVAL, "logprobs: unknown z_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "logprobs: bad sizes");
    if (C > CLASSES_MOST) CG_FAIL(CAPGNN_EUNSUPPORTED, "logprobs: more than 2^30 classes");
    if (m < 0 || m > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "logprobs: m = %d, 0 to %d classes can be given per row", m, CAPGNN_GIVEN_MAX);
    if (k < 0 || k > CAPGNN_TOP_MAX || k > C) CG_FAIL(CAPGNN_EINVAL, "logprobs: k = %d, 0 to min(C, %d) expected", k, CAPGNN_TOP_MAX);
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "logprobs: the temperature must lie between 2^-64 and 2^64");
    if (n == 0) return CAPGNN_OK;
    if (!Z || (m > 0 && (!ids || !logp)) || (k > 0 && !top_ids && !top_logp)) CG_FAIL(CAPGNN_EINVAL, "logprobs: NULL operand");
    if (ldz < C || (m > 0 && (ldi < m || ldp < m)) || (k > 0 && ldt < k)) CG_FAIL(CAPGNN_EINVAL, "logprobs: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs: Z is not aligned to its elements");
    const size_t need = capgnn_logprobs_workspace_bytes(n, C, k);
    if (need && (!ws || ws_bytes < need)) CG_FAIL(CAPGNN_ENOMEM, "logprobs: workspace of %zu bytes needed, %zu given", need, ws ? ws_bytes : size_t(0));
    if (need && reinterpret_cast<uintptr_t>(ws) & 255u) CG_FAIL(CAPGNN_EINVAL, "logprobs: workspace must be 256-byte aligned");
    hipStream_t st = static_cast<hipStream_t>(stream);
    AnswerArgs a{n, C, static_cast<const char *>(Z), ldz, temp_scale(temperature), mask, ids, ldi, m, logp, ldp, entropy, stats, k, top_ids,
                 top_logp, ldt};
    const bool bf16 = z_dtype == CAPGNN_BF16;
    if (C <= NARROW_C && k <= NARROW_TOP) {
        const NarrowShape s = narrow_shape(C, z_dtype);
        const size_t lds = NARROW_WAVES * (s.lds_wave + 64 * (sizeof(float2) + NARROW_TOP));
        auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(narrow_grid(s, n, lds)), dim3(64 * NARROW_WAVES), lds, st, a, s); };
        if (bf16) {
            if (entropy) k ? go(answers_narrow_kernel<true, true, true>) : go(answers_narrow_kernel<true, true, false>);
            else k ? go(answers_narrow_kernel<true, false, true>) : go(answers_narrow_kernel<true, false, false>);
        } else {
            if (entropy) k ? go(answers_narrow_kernel<false, true, true>) : go(answers_narrow_kernel<false, true, false>);
            else k ? go(answers_narrow_kernel<false, false, true>) : go(answers_narrow_kernel<false, false, false>);
        }
        CG_HIP(hipGetLastError());
        return CAPGNN_OK;
    }
    AnswerParts w{};
    w.parts = answer_parts(n, C, &w.chunk);
    w.sums = static_cast<float4 *>(ws);
    w.keys = reinterpret_cast<unsigned long long *>(static_cast<char *>(ws) + align_up(sizeof(float4) * n * w.parts, 256));
    // A wave alone walks rows of one tile and, where there are enough rows for two waves on every SIMD, rows up to ANSWER_WAVE_C classes, half
    // as many for long lists (no meeting of waves: 3001 x 10007 bf16, k = 10, 40 us by workgroups of four waves, 23 by waves; 8000 x 5000
    // fp32 82 and 36; but 600 x 10007 fp32 15 and 19, and from 33000 classes on no difference; k = 64: 8000 x 5000 fp32 95 and 72, 2500 x
    // 16384 bf16 41 and 70).
    const bool wave = w.chunk <= 64 * ANSWER_VECTORS * (bf16 ? 8 : 4) || (n >= 2048 && C <= (k > 32 ? ANSWER_WAVE_C / 2 : ANSWER_WAVE_C));
    auto go = [&](auto kernel, int threads) { hipLaunchKernelGGL(kernel, dim3(stride_grid(n * w.parts, threads)), dim3(threads), 0, st, a, w); };
    if (bf16) {
        if (wave) entropy ? go(answers_rows_kernel<true, 64, true>, 64) : go(answers_rows_kernel<true, 64, false>, 64);
        else entropy ? go(answers_rows_kernel<true, 256, true>, 256) : go(answers_rows_kernel<true, 256, false>, 256);
    } else {
        if (wave) entropy ? go(answers_rows_kernel<false, 64, true>, 64) : go(answers_rows_kernel<false, 64, false>, 64);
        else entropy ? go(answers_rows_kernel<false, 256, true>, 256) : go(answers_rows_kernel<false, 256, false>, 256);
    }
    if (w.parts > 1) {
        const unsigned rows = static_cast<unsigned>(n);
        if (bf16) hipLaunchKernelGGL(answers_join_kernel<true>, dim3(rows), dim3(256), 0, st, a, w);
        else hipLaunchKernelGGL(answers_join_kernel<false>, dim3(rows), dim3(256), 0, st, a, w);
    }
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}

extern "C" int capgnn_logprobs_bwd(int64_t n, int C, const void *Z, int64_t ldz, int z_dtype, float temperature, const uint8_t *mask,
                                   const float *stats, const float *entropy, const int32_t *ids, int64_t ldi, int m, const float *dlogp,
                                   int64_t lddp, const float *dentropy, void *dZ, int64_t lddz, int dz_dtype, void *stream) {
    if ((z_dtype != CAPGNN_F32 && z_dtype != CAPGNN_BF16) || (dz_dtype != CAPGNN_F32 && dz_dtype != CAPGNN_BF16))
        CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: unknown z_dtype or dz_dtype");
    if (n < 0 || C <= 0) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: bad sizes");
    if (C > CLASSES_MOST) CG_FAIL(CAPGNN_EUNSUPPORTED, "logprobs_bwd: more than 2^30 classes");
    if (m < 0 || m > CAPGNN_GIVEN_MAX) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: m = %d, 0 to %d classes can be given per row", m, CAPGNN_GIVEN_MAX);
    if (!good_temperature(temperature)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: the temperature must lie between 2^-64 and 2^64");
    if (n == 0) return CAPGNN_OK;
    if (!Z || !stats || !dZ || (m > 0 && (!ids || !dlogp)) || (dentropy && !entropy)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: NULL operand");
    if (ldz < C || lddz < C || (m > 0 && (ldi < m || lddp < m))) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: leading dimension smaller than the row");
    if (!element_aligned(Z, z_dtype) || !element_aligned(dZ, dz_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: Z or dZ is not aligned to its elements");
    if (dZ == Z && (lddz != ldz || dz_dtype != z_dtype)) CG_FAIL(CAPGNN_EINVAL, "logprobs_bwd: dZ may be Z only with the same type and pitch");
    hipStream_t st = static_cast<hipStream_t>(stream);
    AnswerGradArgs a{n, C, static_cast<const char *>(Z), ldz, temp_scale(temperature), mask, stats, entropy, ids, ldi, m, dlogp, lddp,
                     dentropy, static_cast<char *>(dZ), lddz};
    const bool zb = z_dtype == CAPGNN_BF16, db = dz_dtype == CAPGNN_BF16, ent = dentropy != nullptr;
    auto types = [&](auto f) {          // f(type of Z, type of dZ, with entropy), as compile-time truth values
        using Y = std::true_type;
        using N = std::false_type;
        if (zb) {
            if (db) ent ? f(Y(), Y(), Y()) : f(Y(), Y(), N());
            else ent ? f(Y(), N(), Y()) : f(Y(), N(), N());
        } else {
            if (db) ent ? f(N(), Y(), Y()) : f(N(), Y(), N());
            else ent ? f(N(), N(), Y()) : f(N(), N(), N());
        }
    };
    if (C <= NARROW_C) {
        const NarrowShape s = narrow_shape(C, z_dtype);
        const size_t lds = NARROW_WAVES * s.lds_wave;
        types([&](auto z, auto d, auto e) {
            hipLaunchKernelGGL((answers_grad_narrow_kernel<z.value, d.value, e.value>), dim3(narrow_grid(s, n, lds)), dim3(64 * NARROW_WAVES), lds, st, a, s);
        });
    } else {
        // One wave a row where it holds the row, 256 threads on longer ones: 50000 rows of 600 f32 49 us against 87 with 256 threads, 1000
        // f32 87 / 116, 2000 bf16 84 / 114.
        const int V = zb ? 8 : 4, threads = C <= 64 * GRAD_VECTORS * V ? 64 : 256;
        const int chunks = (C + threads * GRAD_VECTORS * V - 1) / (threads * GRAD_VECTORS * V);
        const unsigned grid = stride_grid(n * chunks, threads);
        types([&](auto z, auto d, auto e) {
            if (threads == 64) hipLaunchKernelGGL((answers_grad_rows_kernel<z.value, d.value, 64, e.value>), dim3(grid), dim3(64), 0, st, a, chunks);
            else hipLaunchKernelGGL((answers_grad_rows_kernel<z.value, d.value, 256, e.value>), dim3(grid), dim3(256), 0, st, a, chunks);
        });
    }
    CG_HIP(hipGetLastError());
    return CAPGNN_OK;
}
