// Distillation from a teacher's top logits: the divergence of a row's softmax from the teacher's classes, and its gradient.  The kernels, as
// templates; distill.hip has them without the teacher's remaining probability, distill_rest.hip with it.
#pragma once

#include "softrow.h"

#include <algorithm>

namespace capgnn {

struct DistillArgs {
    int64_t n;
    int C;
    const char *Z; int64_t ldz;
    TempScale t;
    const uint8_t *mask;
    const int32_t *t_ids; const float *t_val; int64_t ldt; int k, rest;
    float weight;
    float norm_val; const double *counts; int n_counts;       // the normaliser, or the parts (64 at most) of the number of masked rows
    double *part;                   // [gridDim.x]
    float *row_loss;
    char *dZ; int64_t lddz; int accumulate;
};

// by every wave for itself
__device__ __forceinline__ float distill_norm(const DistillArgs &a) {
    if (!a.counts) return a.norm_val;
    const int lane = threadIdx.x & 63;
    const double c = wave_all(lane < a.n_counts ? a.counts[lane] : 0.0, OpSum());
    return c > 0.0 ? static_cast<float>(c) : 1.f;
}

constexpr float REST_LEAST = 9.5367431640625e-7f;       // 2^-20
// Next to no other class a remainder makes the divergence infinite, so it has to be one: z / T and ln sum exp(z / T) as floats, up to some 500 each,
// leave the sum of q off by 2^-14.
constexpr float REST_LEAST_ALONE = 1.220703125e-4f;     // 2^-13

// Exponential and logarithm in doubles, of a few numbers a row, to some 1e-14 (what they give is stored as a float): the series of exp on
// |r| <= ln 2 / 2 and of 2 atanh((m - 1) / (m + 1)) on 1/sqrt 2 <= m <= sqrt 2.  READ: their coefficients are read where they are used.  (As constants
// of the program they are kept in registers across the loop over the rows, next to the logits, up to 53 of them in scratch memory.  Read and
// held, us: workgroups of 512 threads, 8192 x 64000 bf16 410 and 444, 2048 x 131072 fp32 with rest 582 and 622; of fewer, 2999 x 10007 fp32
// with rest 72.4 and 71.3, 20000 x 1000 bf16 40.5 and 39.1, with rest 52.5 and 47.8; few classes, 612000 x 47 118.9 and 116.7, with rest 136 and 156.)
struct Terms { double c[12]; };
constexpr Terms EXP_TERMS = {{1.0 / 39916800, 1.0 / 3628800, 1.0 / 362880, 1.0 / 40320, 1.0 / 5040, 1.0 / 720, 1.0 / 120, 1.0 / 24, 1.0 / 6, 0.5,
                              1.4426950408889634074, 0.69314718055994530942}};
constexpr Terms LOG_TERMS = {{1.0 / 17, 1.0 / 15, 1.0 / 13, 1.0 / 11, 1.0 / 9, 1.0 / 7, 1.0 / 5, 1.0 / 3, 1.0, 0.69314718055994530942}};
static __constant__ Terms exp_terms = EXP_TERMS, log_terms = LOG_TERMS;
__device__ __forceinline__ const double *terms_anew(const Terms &t) {
    const double *p = t.c;
    asm volatile("" : "+s"(p));
    return p;
}
// x from -inf (0) to what a double holds; NaN stays
template <bool READ> __device__ __forceinline__ double exp_wide(double x) {
    constexpr Terms held = EXP_TERMS;
    const double *c = READ ? terms_anew(exp_terms) : held.c;
    x = x < -800.0 ? -800.0 : x > 800.0 ? 800.0 : x;
    const double n = rint(x * c[10]), r = fma(-n, c[11], x);
    double e = c[0];
#pragma unroll
    for (int i = 1; i < 10; ++i) e = fma(e, r, c[i]);
    e = fma(e, r, 1.0);
    return ldexp(fma(e, r, 1.0), static_cast<int>(n));
}
__device__ __forceinline__ double inverse(double x) {
    double y = __builtin_amdgcn_rcp(x);
    y = fma(y, fma(-x, y, 1.0), y);
    return fma(y, fma(-x, y, 1.0), y);
}
// x > 0 and finite; NaN stays
template <bool READ> __device__ __forceinline__ double log_wide(double x) {
    constexpr Terms held = LOG_TERMS;
    const double *c = READ ? terms_anew(log_terms) : held.c;
    int n;
    double m = frexp(x, &n);
    if (m < 0.70710678118654752) { m += m; --n; }
    const double t = (m - 1.0) * inverse(m + 1.0), t2 = t * t;
    double l = c[0];
#pragma unroll
    for (int i = 1; i < 9; ++i) l = fma(l, t2, c[i]);
    return fma(static_cast<double>(n), c[9], 2.0 * t * l);
}

// (z - m0) / T in doubles.  1 / T is taken from L as the float exponentials have it, so that its rounding means another temperature, not another
// distribution.
__device__ __forceinline__ double student_scale(const TempScale &t) { return t.L * 0.6931471805599453094; }
__device__ __forceinline__ double scaled(float z, float m0, const TempScale &t) { return (static_cast<double>(z) - m0) * student_scale(t); }

// 1 / T as exp_difference has it, for the teacher's values
__device__ __forceinline__ double teacher_scale(const TempScale &t) { return (static_cast<double>(t.L) + t.L_lo) * 0.6931471805599453094; }

// ------------------------------------------------------------------ the teacher of a row, in LDS; the first wave of a workgroup works on it
struct Teacher {
    static constexpr int OWN = CAPGNN_GIVEN_MAX / 64;       // entries of a lane: l, l + 64, ...
    alignas(16) int32_t id[CAPGNN_GIVEN_MAX];   // class of every entry, -1: none
    int32_t c[CAPGNN_GIVEN_MAX];    // the same at a class's first mention, else -1
    float v[CAPGNN_GIVEN_MAX];      // value of the entry
    float w[CAPGNN_GIVEN_MAX];      // probability of the entry
    float q[CAPGNN_GIVEN_MAX];      // of the class in all
    float z[CAPGNN_GIVEN_MAX];      // the row's logit of the class
    float old[CAPGNN_GIVEN_MAX];    // what its gradient is added to
    int entries;                    // that count
    float mass;                     // Q + r
    double r;                       // what the teacher leaves
    float top;                      // rest: largest of z, and the sum of the listed classes' exponentials from there
    double sum;                     // else: the same of v
};

// A bit for every listed class: set by the first wave between two barriers.  The bits of a thread's classes of a tile lie together, one read of
// LDS a tile.  Tiles beyond those there is room for share the bits of earlier ones.
constexpr int SEEN_BYTES = 32768;
template <bool BF16, int THREADS, int NV> struct Seen {
    static constexpr int V = Raw<BF16>::V, STEP = THREADS * V, TILE = NV * STEP, W = NV * V <= 32 ? 1 : NV * V <= 64 ? 2 : 4;
    static constexpr int MOST = SEEN_BYTES / (THREADS * W * 4);             // tiles
    typedef uint32_t Words __attribute__((ext_vector_type(W)));
    Words *own;             // [tiles][THREADS]
    int tiles;
    bool shared;            // the row (or part) has more tiles
    static int tiles_for(int classes) { return std::min((classes + TILE - 1) / TILE, MOST); }
    __device__ __forceinline__ Words *at(int tile) const { return own + (tile < tiles ? tile : tile % tiles) * THREADS; }
    __device__ __forceinline__ void clear() const {
        for (int t = 0; t < tiles; ++t) own[t * THREADS + threadIdx.x] = 0u;
    }
    __device__ __forceinline__ void set(int c) const {                      // c: from the row's (or part's) first class on
        const int tile = c / TILE, in = c % TILE, bit = in / STEP * V + in % V;
        atomicOr(reinterpret_cast<uint32_t *>(at(tile) + in % STEP / V) + bit / 32, 1u << bit % 32);
    }
    static __device__ __forceinline__ uint32_t vector(Words w, int i) {     // the i-th of the thread's vectors
        return w[i * V / 32] >> (i * V % 32) & ((1u << V) - 1u);
    }
};

// What the teacher leaves (rest) is the small difference of numbers near 1: its exponentials and their sum are doubles.  listed: where another
// launch has left the logits of the entries' classes, or null.
template <bool BF16, bool READ>
__device__ __forceinline__ void read_teacher(const DistillArgs &a, int64_t row, const char *z, const float *listed, Teacher &t) {
    const int lane = threadIdx.x;
    float top = -INFINITY, top_z = -INFINITY, v[Teacher::OWN], z_of[Teacher::OWN];
    int entries = 0;
#pragma unroll
    for (int o = 0; o < Teacher::OWN; ++o) {
        if (o * 64 >= a.k) break;
        const int i = lane + o * 64;
        v[o] = z_of[o] = -INFINITY;
        bool here = false;
        if (i < a.k) {
            int c = a.t_ids[row * a.ldt + i];
            v[o] = a.t_val[row * a.ldt + i];
            if (c < 0 || c >= a.C || v[o] == -INFINITY) { c = -1; v[o] = -INFINITY; }
            t.id[i] = c;
            t.v[i] = v[o];
            if (c >= 0) {
                t.z[i] = z_of[o] = listed ? listed[i] : ld_logit<BF16>(z, c);
                top_z = max_of(top_z, z_of[o]);
                top = max_of(top, v[o]);
                here = true;
            }
        }
        entries += __popcll(__ballot(here));
    }
    if (a.rest) top_z = wave_all(top_z, OpMax());
    else top = safe_max(wave_all(top, OpMax()));
    const float ref_z = safe_max(top_z);
    double Q = 0.0, listed_sum = 0.0, w[Teacher::OWN];
#pragma unroll
    for (int o = 0; o < Teacher::OWN; ++o) {
        if (o * 64 >= a.k) break;
        w[o] = a.rest ? exp_wide<READ>(v[o]) : static_cast<double>(exp_difference(v[o], top, a.t));      // (none: 0)
        Q += w[o];
        if (a.rest) listed_sum += exp_wide<READ>(scaled(z_of[o], ref_z, a.t));
    }
    Q = wave_all(Q, OpSum());
    const double one = a.rest ? 1.0 : 1.0 / Q;
#pragma unroll
    for (int o = 0; o < Teacher::OWN; ++o) {
        if (o * 64 >= a.k) break;
        if (lane + o * 64 < a.k) t.w[lane + o * 64] = static_cast<float>(w[o] * one);
    }
    wave_sync();
    // a class listed again: its first mention takes the sum (ids four at a time; the sums only where there are some)
#pragma unroll 1
    for (int i = lane; i < (a.k + 63 & ~63); i += 64) {
        const int c = i < a.k ? t.id[i] : -1;
        int same = 0, before = 0;
        for (int b = 0; b < a.k; b += 4) {
            const int4 v = *reinterpret_cast<const int4 *>(&t.id[b]);
            const int there[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const bool hit = there[u] == c && b + u < a.k;
                same += hit;
                before += hit && b + u < i;
            }
        }
        float sum = i < a.k ? t.w[i] : 0.f;
        if (__any(c >= 0 && same > 1)) {
            sum = 0.f;
            for (int b = 0; b < a.k; ++b) sum += t.id[b] == c ? t.w[b] : 0.f;
        }
        if (i < a.k) {
            t.q[i] = sum;
            t.c[i] = c >= 0 && before == 0 ? c : -1;
            if (a.rest && c >= 0 && before > 0) listed_sum -= exp_wide<READ>(scaled(t.z[i], ref_z, a.t));        // (the very number that was added)
        }
    }
    double r = a.rest ? 1.0 - Q : 0.0;
    if (r < REST_LEAST) r = 0.0;
    if (a.rest) listed_sum = wave_all(listed_sum, OpSum());
    if (lane == 0) {
        t.top = a.rest ? top_z : top;
        t.sum = a.rest ? listed_sum : Q;
        t.entries = entries;
        t.r = r;
        t.mass = static_cast<float>(a.rest ? Q + r : 1.0 + 0.0 * Q);       // (a NaN among the values reaches every class)
    }
    wave_sync();
}

// Bars the logits of a vector whose bits are set in `out`.
template <bool BF16> __device__ __forceinline__ void bar(raw16 &r, uint32_t out) {
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if constexpr (BF16) {
            const uint32_t m = (out >> (2 * w) & 1u ? 0xffffu : 0u) | (out >> (2 * w + 1) & 1u ? 0xffff0000u : 0u);
            r[w] = (r[w] & ~m) | (Raw<true>::BARRED & m);
        } else {
            r[w] = out >> w & 1u ? Raw<false>::BARRED : r[w];
        }
    }
}

// Maximum and sum of a thread's logits of one tile, added to what it has (m, s).  REST: of the classes that are not listed; the listed ones are
// barred in r.  The others have a maximum of their own: what the row gives to them may be far below the rounding of a sum that holds the listed
// ones, and (from a distance of 88 T on) below the least float as well.
template <bool BF16, int THREADS, int NV, bool REST>
__device__ __forceinline__ void scan_tile(raw16 (&r)[NV], int t0, int hi, int tile, const DistillArgs &a, const Teacher &l,
                                          const Seen<BF16, THREADS, NV> &seen, float &m, float &s) {
    typedef Raw<BF16> R;
    typedef Seen<BF16, THREADS, NV> S;
    const int tid = thread_anew();
    hi = uniform_anew(hi);
    float tmax = -INFINITY;
    typename S::Words listed = 0u;
    if constexpr (REST) listed = seen.at(tile)[tid];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (t0 + i * THREADS * R::V >= hi) continue;
        if constexpr (REST) {
            uint32_t out = S::vector(listed, i);
            if (__any(out != 0)) {
                const int j = t0 + (i * THREADS + tid) * R::V, from = j + R::V <= hi ? j : hi - R::V;
                if (seen.shared && out) {                  // some other class may have set the bit
                    uint32_t sure = 0;
                    for (int b = 0; b < a.k; ++b) {
                        const int d = l.id[b] - j;
                        if (d >= 0 && d < R::V) sure |= 1u << d;
                    }
                    out &= sure;
                }
                bar<BF16>(r[i], out << (j < hi ? j - from : 0));
            }
        }
#pragma unroll
        for (int e = 0; e < R::V; ++e) tmax = max_of(tmax, R::get(r[i], e));
    }
    const float m_new = max_of(m, tmax), ref = safe_max(m_new);
    s *= exp2_raw((m - ref) * a.t.L);
    m = m_new;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (t0 + i * THREADS * R::V >= hi) continue;
        forget(r[i]);
#pragma unroll
        for (int e = 0; e < R::V; ++e) s += exp2_raw((R::get(r[i], e) - ref) * a.t.L);
    }
}

// SHORT: the row may be shorter than a vector.  Vectors behind the row's end are barred, not left as they were: registers without a value in some
// of the rows are taken for carried on from row to row, next to their new values.
template <bool BF16, int THREADS, int NV, bool SHORT = THREADS == 64>
__device__ __forceinline__ void read_tile(raw16 (&r)[NV], const char *z, int t0, int hi) {
    typedef Raw<BF16> R;
    const int tid = thread_anew();
    hi = uniform_anew(hi);
    int from;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (t0 + i * THREADS * R::V >= hi) {
            r[i] = raw16{R::BARRED, R::BARRED, R::BARRED, R::BARRED};
            continue;
        }
        const int j = t0 + (i * THREADS + tid) * R::V;
        if (t0 + (i + 1) * THREADS * R::V <= hi) r[i] = R::load(z, j);
        else r[i] = R::template load_until<SHORT>(z, j, hi, &from);
    }
}

// dz = exp((z - m0) / T) * factor for the tile's classes, added to dz's contents when add.  (REST: m0 is the others' maximum, and what comes out for a
// listed class, which may lie above it, is replaced.)
template <bool BF16, bool DBF16, int THREADS, int NV>
__device__ __forceinline__ void grad_tile(raw16 (&r)[NV], char *dz, int t0, int hi, const TempScale &t, float m0, float factor, int add) {
    typedef Raw<BF16> R;
    constexpr int V = R::V;
    const int tid = thread_anew();
    hi = uniform_anew(hi);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        if (t0 + i * THREADS * V >= hi) continue;
        const int j = t0 + (i * THREADS + tid) * V;
        forget(r[i]);
        float o[V];
#pragma unroll
        for (int e = 0; e < V; ++e) o[e] = exp_scaled<!DBF16>(difference(R::get(r[i], e), m0, t), t) * factor;
        if (t0 + (i + 1) * THREADS * V <= hi || j + V <= hi) {
            if (add) {
                float old[V];
                ld_vector<DBF16>(dz, j, old);
#pragma unroll
                for (int e = 0; e < V; ++e) o[e] += old[e];
            }
            st_vector<DBF16>(dz, j, o);
        } else if (j < hi) {
            const int shift = j + V - hi;           // a row's last vector starts earlier than j by that
#pragma unroll
            for (int e = 0; e < V; ++e)
                if (e >= shift) st_grad<DBF16>(dz, hi - V + e, add ? o[e] + ld_logit<DBF16>(dz, hi - V + e) : o[e]);
        }
    }
}

// A row that adds nothing: zeros, unless they were to be added.
template <bool BF16, bool DBF16, int THREADS>
__device__ __forceinline__ void no_gradient(const DistillArgs &a, char *dz, int lo, int hi) {
    constexpr int V = Raw<BF16>::V;
    if (a.accumulate) return;
    const float zero[V] = {};
    int j = lo + static_cast<int>(threadIdx.x) * V;
    for (; j + V <= hi; j += THREADS * V) st_vector<DBF16>(dz, j, zero);
    for (; j < hi; ++j) st_grad<DBF16>(dz, j, 0.f);
}

// What the row gives to the classes that are not listed: P = exp((m - m0) / T) s / S, from their own maximum and sum (m, s), next to the listed
// classes' (top, sum); m0: the larger maximum.  P may leave float's (and double's) range; its logarithm and the others' shares of it do not.
template <bool READ> struct RestSums {
    double S, own;          // over all classes, from m0; 0 for an empty row; the others' part of it
    float m0;
    __device__ __forceinline__ RestSums(float m, float s, float top, double sum, const TempScale &t) {
        const double e = m == top ? 1.0 : exp_wide<READ>(-fabs(scaled(m, top, t)));
        m0 = safe_max(max_of(m, top));
        own = m < top ? s * e : s;
        S = own + (m < top ? sum : sum * e);
    }
    // dz of a class that is not listed is this by exp((z - m) / T): (P mass - r) / s; 0 where all of them are barred
    __device__ __forceinline__ float factor(float s, double r, float mass, float scale) const {
        return s == 0.f ? 0.f * mass : static_cast<float>((own * mass - r * S) * inverse(S * s)) * scale;
    }
};

// what a teacher leaves counts as, next to others of sum s (0: none, or all barred)
__device__ __forceinline__ double rest_left(double r, float s) { return s == 0.f && r < REST_LEAST_ALONE ? 0.0 : r; }

// r (ln r - ln P), from the logarithm of r S / s
__device__ __forceinline__ double rest_others(float s, double r, double ln, double far) {
    if (s == 0.f) return rest_left(r, s) > 0.0 ? INFINITY : 0.0;
    return r > 0.0 ? r * (ln - far) : 0.0;
}

// The divergence of one row, sum q (ln q - ln p) over the listed classes, ln p = (z - m0) / T - ln S, and with REST r (ln r - ln P): in the first
// wave (every lane); s is the row's sum, or (REST) that of the others, S over all.  It is the small difference of its terms where the student is
// close to the teacher.  So they are doubles, ln q comes from the teacher's value (from q only where a class is listed again), and q's
// rounding counts with ln q - ln p.  With REST the others' sum counts with P - r; without, the roundings of S stay, some 1e-7.
template <bool REST, bool READ>
__device__ __forceinline__ double divergence(const DistillArgs &a, const Teacher &t, float m, float m0, float s, double S) {
    // both logarithms at once, one in the even lanes, one in the odd ones: of S and r S / s, or of S / Z with Z the sum of the teacher's exponentials
    const double ln = log_wide<READ>(!REST ? s * inverse(t.sum) : threadIdx.x & 1 ? t.r * S * inverse(s) : S), ln_S = REST ? __shfl(ln, 0) : ln;
    double kl = 0.0;
#pragma unroll 1
    for (int i = threadIdx.x; i < a.k; i += 64) {
        const float q = t.q[i];
        if (t.c[i] < 0 || q == 0.f) continue;
        double ln_q = REST ? static_cast<double>(t.v[i]) : (static_cast<double>(t.v[i]) - t.top) * teacher_scale(a.t);     // (without REST: and ln Z)
        if (q != t.w[i]) ln_q = log_wide<READ>(REST ? q : q * t.sum);
        kl += q * (ln_q + ln_S - scaled(t.z[i], m0, a.t));
    }
    if (REST && threadIdx.x == 1) kl += rest_others(s, t.r, ln, scaled(m, m0, a.t));
    return wave_all(kl, OpSum());
}

struct DistillParts {
    int parts, chunk;       // of a row; classes of one
    float2 *sums;           // [n][parts]: maximum, sum (rest: of the classes not listed)
    float *listed;          // [n][GIVEN_MAX]: logits of the entries' classes (dZ may be Z: another part may have replaced them)
    int seen;               // tiles with bits of their own (Seen)
};

// How much of the work on a row (or a part of it) a launch does
enum DistillStage : int {
    ROW_HELD,       // all of it, the row's logits in registers from the sums to the gradient
    ROW_READ_TWICE, // all of it, longer rows: all but the last tile read again for the gradient (out of the caches where the rows under way fit)
    PART_SUMS,      // maximum and sum of a part
    PART_GRADIENT   // the parts' sums put together, gradient of a part
};

// One workgroup per row (or part): the first wave reads the teacher while all of them have the row's logits on their way; maximum and sums from
// registers, one meeting, then the gradient from the same registers; the listed classes' own terms follow behind a barrier.  Bound by
// HBM: 8192 x 64000 bf16 406 us (5.2 TB/s read and written).  Rows longer than the registers hold come out of the Infinity Cache a second
// time, all but the last tile: 2048 x 131072 fp32 580 us for 2.1 GB (a second pass over everything: 650).  Rows of some ten thousand
// classes are held up by the teacher's chain of dependent reads, four workgroups a compute unit: 2999 x 10007 fp32, k = 32, rest, 70 us.
// At most 128 registers, for sixteen waves per compute unit: without that bound the compiler takes twice as many and has half the waves.  With
// 12 and 16 vectors a thread up to 21 registers go to scratch memory (80 bytes a thread).
template <bool BF16, bool DBF16, int THREADS, int NV, bool REST, DistillStage STAGE>
__global__ __launch_bounds__(THREADS) __attribute__((amdgpu_waves_per_eu(4))) void distill_rows_kernel(DistillArgs a, DistillParts w) {
    typedef Raw<BF16> R;
    constexpr int TILE = THREADS * NV * R::V;
    constexpr bool READ = THREADS == 512;
    constexpr bool PARTS = STAGE == PART_SUMS || STAGE == PART_GRADIENT;
    extern __shared__ __align__(16) uint32_t seen_bits[];
    __shared__ Teacher t;
    __shared__ float2 red[THREADS / 64];
    typedef Seen<BF16, THREADS, NV> S;
    const S seen{reinterpret_cast<typename S::Words *>(seen_bits), w.seen, (PARTS ? w.chunk : a.C) > w.seen * S::TILE};
    const bool first_wave = threadIdx.x < 64;
    const float norm = distill_norm(a);
    const float scale = a.weight / norm * a.t.inv_T;
    double loss = 0.0;
    for (int64_t job = blockIdx.x; job < a.n * (PARTS ? w.parts : 1); job += gridDim.x) {
        const int64_t row = PARTS ? job / w.parts : job;
        const int part = PARTS ? static_cast<int>(job % w.parts) : 0;
        const int lo = PARTS ? part * w.chunk : 0, hi = PARTS && a.C - lo > w.chunk ? lo + w.chunk : a.C;
        const char *z = a.Z + row * a.ldz * (BF16 ? 2 : 4);
        char *dz = a.dZ ? a.dZ + row * a.lddz * (DBF16 ? 2 : 4) : nullptr;
        if (a.mask && !a.mask[row]) {
            if (STAGE != PART_SUMS) {
                if (a.row_loss && part == 0 && threadIdx.x == 0) a.row_loss[row] = 0.f;
                if (dz) no_gradient<BF16, DBF16, THREADS>(a, dz, lo, hi);
            }
            continue;
        }
        raw16 r[NV];
        read_tile<BF16, THREADS, NV>(r, z, lo, STAGE != PART_GRADIENT || dz ? hi : lo);
        if constexpr (REST && STAGE != PART_GRADIENT) {
            seen.clear();
            __syncthreads();
        }
        if (first_wave) {
            float *left = STAGE == PART_SUMS || STAGE == PART_GRADIENT ? w.listed + row * CAPGNN_GIVEN_MAX : nullptr;
            if (STAGE != PART_SUMS || REST || part == 0) read_teacher<BF16, READ>(a, row, z, STAGE == PART_GRADIENT ? left : nullptr, t);
            if constexpr (STAGE == PART_SUMS)
                if (part == 0)
                    for (int i = threadIdx.x; i < a.k; i += 64) left[i] = t.z[i];
            if constexpr (REST && STAGE != PART_GRADIENT)
                for (int i = threadIdx.x; i < a.k; i += 64)
                    if (t.c[i] >= lo && t.c[i] < hi) seen.set(t.c[i] - lo);
        }
        if constexpr (REST && STAGE != PART_GRADIENT) __syncthreads();
        float m = -INFINITY, s = 0.f;
        if constexpr (STAGE == PART_GRADIENT) {
            for (int p = threadIdx.x & 63; p < w.parts; p += 64) {          // every wave for itself
                const float2 v = w.sums[row * w.parts + p];
                const float both = max_of(m, v.x), ref = safe_max(both);
                s = s * exp2_raw((m - ref) * a.t.L) + v.y * exp2_raw((v.x - ref) * a.t.L);
                m = both;
            }
            group_softmax<64>(m, s, a.t, red);
        } else {
            scan_tile<BF16, THREADS, NV, REST>(r, lo, hi, 0, a, t, seen, m, s);
            if constexpr (STAGE != ROW_HELD)
#pragma unroll 1
                for (int t0 = lo + TILE, tile = 1; t0 < hi; t0 += TILE, ++tile) {
                    read_tile<BF16, THREADS, NV>(r, z, t0, hi);
                    scan_tile<BF16, THREADS, NV, REST>(r, t0, hi, tile, a, t, seen, m, s);
                }
            group_softmax<THREADS>(m, s, a.t, red);
        }
        if constexpr (STAGE == PART_SUMS) {
            if (threadIdx.x == 0) w.sums[job] = make_float2(m, s);
            __syncthreads();
            continue;
        }
        __syncthreads();
        const float ref = safe_max(m);          // REST: of the others
        const RestSums<READ> rest(m, s, REST ? t.top : m, REST ? t.sum : 0.0, a.t);
        const float m0 = REST ? rest.m0 : ref, S = REST ? static_cast<float>(rest.S) : s;
        if (t.entries == 0 || S == 0.f) {
            if (a.row_loss && part == 0 && threadIdx.x == 0) a.row_loss[row] = 0.f;
            if (dz) no_gradient<BF16, DBF16, THREADS>(a, dz, lo, hi);
            __syncthreads();
            continue;
        }
        if (first_wave && part == 0) {
            const double kl = divergence<REST, READ>(a, t, m, m0, s, rest.S);
            loss += kl;
            if (a.row_loss && threadIdx.x == 0) a.row_loss[row] = static_cast<float>(kl);
        }
        if (dz) {
            const float inv_s = 1.f / S, mass = (REST ? t.mass - static_cast<float>(t.r - rest_left(t.r, s)) : t.mass) * scale;
            const float away = REST ? rest.factor(s, t.r, t.mass, scale) : mass * inv_s;
            if (a.accumulate) {         // what the listed classes hold, before anything is written
                if (first_wave)
                    for (int i = threadIdx.x; i < a.k; i += 64)
                        if (t.c[i] >= lo && t.c[i] < hi) t.old[i] = ld_logit<DBF16>(dz, t.c[i]);
                __syncthreads();
            }
            // a longer row: its last tile is still there, the others come again, the latest first
            int t0 = STAGE == ROW_READ_TWICE ? lo + (hi - lo - 1) / TILE * TILE : lo;
            grad_tile<BF16, DBF16, THREADS, NV>(r, dz, t0, hi, a.t, ref, away, a.accumulate);
            if constexpr (STAGE == ROW_READ_TWICE) {
#pragma unroll 1
                for (t0 -= TILE; t0 >= lo; t0 -= TILE) {
                    read_tile<BF16, THREADS, NV>(r, z, t0, hi);
                    grad_tile<BF16, DBF16, THREADS, NV>(r, dz, t0, hi, a.t, ref, away, a.accumulate);
                }
            } else if constexpr (STAGE == PART_GRADIENT) {
#pragma unroll 1
                for (t0 += TILE; t0 < hi; t0 += TILE) {
                    read_tile<BF16, THREADS, NV>(r, z, t0, hi);
                    grad_tile<BF16, DBF16, THREADS, NV>(r, dz, t0, hi, a.t, ref, away, a.accumulate);
                }
            }
            __syncthreads();
            if (first_wave)
                for (int i = threadIdx.x; i < a.k; i += 64) {
                    const int c = t.c[i];
                    if (c < lo || c >= hi) continue;
                    const float g = fmaf(exp_scaled(difference(t.z[i], m0, a.t), a.t) * inv_s, mass, -t.q[i] * scale);
                    st_grad<DBF16>(dz, c, a.accumulate ? t.old[i] + g : g);
                }
        }
        __syncthreads();
    }
    if constexpr (STAGE != PART_SUMS)
        if (threadIdx.x == 0) a.part[blockIdx.x] = loss;
}

// ------------------------------------------------------------------ few classes
// As answers_grad_narrow_kernel, the teacher's entries beside the rows in LDS, shared by the lanes of a row; each entry looks for other
// mentions of its class.  rest: the listed classes' logits are taken out of the row before its maximum.
// 612000 x 47, k = 8: 109 us, 2 TB/s, bound by instruction issue (59 us of it) and LDS latency (with rest, and
// 16 registers in scratch memory, the call takes 135 us against 116).  (Entries read where they are used, by one lane
// a row: 278 us; the teacher's probabilities by class in a second set of rows, which leaves LDS for ten waves per compute unit: 170 us.)
// Every entry is compared with all of its row's, so long lists go to a wave a row.  100000 rows, few-class kernel against a wave a row, us: 30 f32
// k = 16 87 / 138 (k = 17 by a wave 143), 64 f32 k = 24 90 / 144, 100 f32 k = 32 113 / 153, k = 40 196 / 162, k = 64 448 / 190, 256 f32 k = 40 168 /
// 169, k = 64 298 / 194; with rest 100 f32 k = 40 217 / 222, 256 f32 k = 48 217 / 260, k = 64 326 / 277; bf16 256 k = 40 142 / 175, k = 64 274 / 213.
constexpr int NARROW_ENTRIES = 16;      // of a lane
constexpr int NARROW_LIST = 40;         // of a row
// (an odd number of words between rows: their lanes hit different banks)
static inline size_t distill_narrow_lds(const NarrowShape &s, int k) { return s.lds_wave + static_cast<size_t>(s.rows) * (k | 1) * 3 * sizeof(float); }

template <bool BF16, bool DBF16, bool REST>
__global__ __launch_bounds__(64 * NARROW_WAVES) __attribute__((amdgpu_waves_per_eu(4))) void distill_narrow_kernel(DistillArgs a, NarrowShape s) {
    constexpr bool READ = REST;
    extern __shared__ __align__(16) uint32_t seen_bits[];
    __shared__ double red[NARROW_WAVES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), k = a.k, kp = k | 1, all_items = s.rows * k;
    float *tile = reinterpret_cast<float *>(reinterpret_cast<char *>(seen_bits) + wave * (s.lds_wave + s.rows * kp * 3 * sizeof(float)));
    float *tile_w = tile + s.rows * s.pitch, *tile_q = tile_w + s.rows * kp;
    int32_t *tile_id = reinterpret_cast<int32_t *>(tile_q + s.rows * kp);
    const int G = 1 << s.lg, sub = lane & (G - 1), C = s.C, mine = lane >> s.lg;
    float *z = tile + mine * s.pitch, *w = tile_w + mine * kp, *q = tile_q + mine * kp;
    int32_t *id = tile_id + mine * kp;
    const float norm = distill_norm(a);
    const float scale = a.weight / norm * a.t.inv_T;
    const int magic = ((1 << 20) + k - 1) / k; // item / k = item * magic >> 20 for item < 1024, k <= 128
    const int64_t step = static_cast<int64_t>(gridDim.x) * NARROW_WAVES * s.rows;
    int64_t row0 = (static_cast<int64_t>(blockIdx.x) * NARROW_WAVES + wave) * s.rows;
    double loss = 0.0;
    narrow_ends(s, tile, lane);
    NarrowLoad<BF16> next;
    if (row0 < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0);
    for (; row0 < a.n; row0 += step) {
        const int64_t row = row0 + mine;
        const bool in = row < a.n, on = in && (!a.mask || a.mask[row]);
        {
            int32_t c[NARROW_ENTRIES];
            float v[NARROW_ENTRIES];
            const int items = uniform_anew(all_items), anew = thread_anew() & 63, last = static_cast<int>(a.n - row0 < s.rows ? a.n - row0 : s.rows) - 1;
            const int32_t *t_ids = a.t_ids + row0 * a.ldt;
            const float *t_val = a.t_val + row0 * a.ldt;
            const bool near = a.ldt < 1 << 22;
            const uint32_t ldt = static_cast<uint32_t>(a.ldt);
#pragma unroll
            for (int i = 0; i < NARROW_ENTRIES; ++i) {
                const int item = i * 64 + anew;
                c[i] = -1;                                  // (as the vectors of read_tile)
                v[i] = 0.f;
                if (i * 64 >= items) continue;              // (the same for all lanes)
                int r = item * magic >> 20;
                const int e = item - __mul24(r, k);
                r = r < last ? r : last;                    // (rows and entries beyond the last ones again those)
                if (near) {
                    const uint32_t at = __umul24(r, ldt) + e;
                    c[i] = t_ids[at];
                    v[i] = t_val[at];
                } else {
                    c[i] = t_ids[r * a.ldt + e];
                    v[i] = t_val[r * a.ldt + e];
                }
            }
            next.put(s, tile);
#pragma unroll
            for (int i = 0; i < NARROW_ENTRIES; ++i) {
                const int item = i * 64 + anew;
                if (i * 64 >= items) continue;
                if (item < items) {
                    const int at = item + (kp - k) * (item * magic >> 20);
                    tile_id[at] = c[i] >= 0 && c[i] < C && v[i] != -INFINITY ? c[i] : -1;
                    tile_w[at] = v[i];
                }
            }
        }
        wave_sync();
        if (row0 + step < a.n) next.fetch(s, a.Z, a.ldz, a.n, row0 + step);
        // REST: the largest logit of the listed classes and, once these are barred, of the others; else the row's and the teacher's
        auto largest = [&] {
            float m = -INFINITY;
            for (int b = 0; b < s.each; b += NARROW_BATCH)
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) m = max_of(m, z[sub + (b + i) * G]);
            return m;
        };
        float m = REST ? -INFINITY : largest(), top = -INFINITY;
        int entries = 0;
        for (int i = sub; i < k; i += G)
            if (id[i] >= 0) {
                top = max_of(top, REST ? z[id[i]] : w[i]);
                ++entries;
            }
        for (int off = 1; off < G; off <<= 1) {
            if constexpr (!REST) m = max_of(m, __shfl_xor(m, off));
            top = max_of(top, __shfl_xor(top, off));
            entries += __shfl_xor(entries, off);
        }
        // w: the entry's probability (without REST not divided by its sum Q yet), and the lane's part of sum q ln q from the very numbers
        double Q = 0.0, kl = 0.0;
        for (int i = sub; i < k; i += G)
            if (id[i] >= 0) {
                const float v = w[i];
                const double p = REST ? exp(static_cast<double>(v)) : static_cast<double>(exp_difference(v, top, a.t));     // (exp: coefficients read for every entry take longer)
                const float held = static_cast<float>(p);
                Q += p;
                w[i] = held;
                if (held != 0.f) kl += held * (REST ? static_cast<double>(v) : static_cast<double>(v) - top);
            }
        if constexpr (!REST) kl *= teacher_scale(a.t);
        for (int off = 1; off < G; off <<= 1) Q += __shfl_xor(Q, off);
        wave_sync();
        for (int i = sub; i < k; i += G) {          // q: of the class in all, at its first mention; -1 elsewhere
            const int c = id[i];
            float p = 0.f;
            bool first = c >= 0;
#pragma unroll 4
            for (int b = 0; b < k; ++b) {
                const bool hit = id[b] == c;
                first = first && !(hit && b < i);
                p += hit ? w[b] : 0.f;
            }
            q[i] = first ? p : -1.f;
            if (c >= 0 && p != w[i]) {              // a class listed again: q ln q of the sum for that of its parts (a part that is the sum stays)
                if (w[i] != 0.f) kl -= w[i] * log_wide<READ>(w[i]);
                if (first) {
                    bool there = false;
                    for (int b = 0; b < k; ++b) there = there || (id[b] == c && w[b] == p);
                    if (!there) kl += p * log_wide<READ>(p);
                }
            }
        }
        wave_sync();
        for (int i = sub; i < k; i += G) {          // w: the class's logit from here on
            if (q[i] == -1.f) continue;
            w[i] = z[id[i]];
            if constexpr (REST) z[id[i]] = -INFINITY;
        }
        wave_sync();
        if constexpr (REST) {
            m = largest();
            for (int off = 1; off < G; off <<= 1) m = max_of(m, __shfl_xor(m, off));
        }
        const float ref = safe_max(m), ref_z = safe_max(top);       // REST: of the others (as in scan_tile), of the listed classes
        float m0 = ref;
        double listed = 0.0;
        float others = 0.f;
        if constexpr (REST)
            for (int i = sub; i < k; i += G)
                if (q[i] != -1.f) listed += exp(scaled(w[i], ref_z, a.t));
        for (int b = 0; b < s.each; b += NARROW_BATCH) {
            float x[NARROW_BATCH];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[sub + (b + i) * G];
#pragma unroll
            for (int i = 0; i < NARROW_BATCH; ++i) others += exp2_raw((x[i] - ref) * a.t.L);
        }
        for (int off = 1; off < G; off <<= 1) {
            others += __shfl_xor(others, off);
            if constexpr (REST) listed += __shfl_xor(listed, off);
        }
        float S = others, mass, away;
        double ln_S = 0.0, tail = 0.0;
        const float one = REST ? 1.f : static_cast<float>(inverse(Q));
        if constexpr (REST) {
            double r = 1.0 - Q;
            if (r < REST_LEAST) r = 0.0;
            mass = static_cast<float>(Q + rest_left(r, others));
            const RestSums<READ> rest(m, others, top, listed, a.t);
            m0 = rest.m0;
            S = static_cast<float>(rest.S);
            away = rest.factor(others, r, mass, scale);
            mass *= scale;
            ln_S = log_wide<READ>(rest.S);
            tail = rest_others(others, r, log_wide<READ>(r * rest.S * inverse(others)), scaled(m, m0, a.t));
        } else {
            ln_S = log_wide<READ>(S * inverse(Q));
            mass = (1.f + 0.f * one) * scale;         // (a NaN among the teacher's values reaches every class)
        }
        const bool live = on && entries > 0 && S != 0.f;
        const float inv_s = 1.f / S;
        if constexpr (!REST) away = mass * inv_s;
        if (a.dZ) {
            const float none = a.accumulate ? -0.f : 0.f;       // (adding -0 leaves everything as it is)
            for (int b = 0; b < s.each; b += NARROW_BATCH) {
                float x[NARROW_BATCH];
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) x[i] = z[sub + (b + i) * G];
#pragma unroll
                for (int i = 0; i < NARROW_BATCH; ++i) {
                    const float g = exp_scaled<!DBF16>(difference(x[i], ref, a.t), a.t) * away;
                    if (sub + (b + i) * G < C) z[sub + (b + i) * G] = live ? g : none;
                }
            }
        }
        wave_sync();
        if (live) {
            // as in divergence; kl has sum q ln q
            double d = 0.0, all = 0.0;
            for (int i = sub; i < k; i += G) {
                const float p = q[i];
                if (p == -1.f) continue;
                if (p != 0.f) d += p * (static_cast<double>(w[i]) - m0);
                if constexpr (REST) all += p;
                z[id[i]] = fmaf(exp_scaled(difference(w[i], m0, a.t), a.t) * inv_s, mass, -p * (scale * one));
            }
            d *= student_scale(a.t);
            if constexpr (REST) kl += all * ln_S - d + (sub == 0 ? tail : 0.0);
            else kl = (kl - d) * inverse(Q) + (sub == 0 ? ln_S : 0.0);
        } else {
            kl = 0.0;
        }
        for (int off = 1; off < G; off <<= 1) kl += __shfl_xor(kl, off);
        if (sub == 0) {
            loss += kl;
            if (in && a.row_loss) a.row_loss[row] = static_cast<float>(kl);
        }
        wave_sync();
        if (a.dZ) narrow_store<BF16, DBF16>(s, tile, a.dZ, a.lddz, a.n, row0, a.accumulate);
        wave_sync();
    }
    loss = wave_all(loss, OpSum());
    if (lane == 0) red[wave] = loss;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int o = 1; o < NARROW_WAVES; ++o) loss += red[o];
        a.part[blockIdx.x] = loss;
    }
}

constexpr int DISTILL_GROUPS = 8192;        // workgroups that leave a sum of the loss, at most

template <bool BF16, bool DBF16, bool REST>
void launch_distill(const DistillArgs &a, DistillParts w, int *groups, hipStream_t st) {
    constexpr int V = Raw<BF16>::V;
    const NarrowShape s = narrow_shape(a.C < NARROW_C ? a.C : NARROW_C, BF16 ? CAPGNN_BF16 : CAPGNN_F32);
    if (a.C <= NARROW_C && a.k <= NARROW_LIST && a.k <= NARROW_ENTRIES << s.lg) {
        const size_t lds = NARROW_WAVES * distill_narrow_lds(s, a.k);
        *groups = static_cast<int>(narrow_grid(s, a.n, lds));
        hipLaunchKernelGGL((distill_narrow_kernel<BF16, DBF16, REST>), dim3(*groups), dim3(64 * NARROW_WAVES), lds, st, a, s);
        return;
    }
    *groups = static_cast<int>(std::min<int64_t>(a.n * w.parts, DISTILL_GROUPS));
    // The fewest threads that hold a row (more rows on a compute unit, whose chains overlap: 2999 x 10007 fp32 with 512 threads 102 us, with 256
    // 72; 12 vectors a thread rather than 16 there, which spills: 63.6 and 62.1 us).
    auto go = [&](auto kernel, auto seen) {
        typedef decltype(seen) S;
        constexpr int threads = S::STEP / V;
        w.seen = S::tiles_for(w.parts > 1 ? w.chunk : a.C);
        hipLaunchKernelGGL(kernel, dim3(*groups), dim3(threads), REST ? w.seen * threads * sizeof(typename S::Words) : 0, st, a, w);
    };
    if (w.parts > 1) {
        go(distill_rows_kernel<BF16, DBF16, 256, 8, REST, PART_SUMS>, Seen<BF16, 256, 8>());
        go(distill_rows_kernel<BF16, DBF16, 256, 8, REST, PART_GRADIENT>, Seen<BF16, 256, 8>());
    } else if (a.C <= 64 * 8 * V) {
        go(distill_rows_kernel<BF16, DBF16, 64, 8, REST, ROW_HELD>, Seen<BF16, 64, 8>());
    } else if (a.C <= 256 * 8 * V) {
        go(distill_rows_kernel<BF16, DBF16, 256, 8, REST, ROW_HELD>, Seen<BF16, 256, 8>());
    } else if (a.C <= 256 * 12 * V) {
        go(distill_rows_kernel<BF16, DBF16, 256, 12, REST, ROW_HELD>, Seen<BF16, 256, 12>());
    } else if (a.C <= 512 * 16 * V) {
        go(distill_rows_kernel<BF16, DBF16, 512, 16, REST, ROW_HELD>, Seen<BF16, 512, 16>());
    } else {
        go(distill_rows_kernel<BF16, DBF16, 512, 12, REST, ROW_READ_TWICE>, Seen<BF16, 512, 12>());
    }
}

// by the types of Z and dZ
typedef void (*DistillLaunch)(const DistillArgs &, DistillParts, int *, hipStream_t);
template <bool REST> DistillLaunch distill_launch_of(bool z_bf16, bool dz_bf16) {
    return z_bf16 ? (dz_bf16 ? launch_distill<true, true, REST> : launch_distill<true, false, REST>)
                  : (dz_bf16 ? launch_distill<false, true, REST> : launch_distill<false, false, REST>);
}
DistillLaunch distill_launch_rest(bool z_bf16, bool dz_bf16);       // distill_rest.hip

}  // namespace capgnn
