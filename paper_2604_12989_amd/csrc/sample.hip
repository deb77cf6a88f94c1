// Sampling with temperature, top-k, top-p and min-p from given uniforms: one token a row, and the verifier's walk over
// them (paper Section 4.4, second paragraph: verification follows the target's own decoding rule).
//
// A row, M its largest logit:  w_v = exp(-(M - x_v) / tau), 0 where (M - x_v) / tau > 40 ln 2.  In the order of falling
// logits (equal ones by id) a token stays if its rank is below top_k, if the w of what is in front of it (among those)
// is below top_p times their sum, and if w_v >= min_p.  The token is the first that stays, in the order of ids, whose
// running sum of w exceeds u times the sum of all that stay: no order has to be found to draw it.
//
// Weights are fp64 (a float's neighbours differ by 2^-24 of a logit, and a sum of 150 000 weights is compared with
// borders that lie 1e-6 of it apart: fp32 weights select another token in one of a few thousand flat rows).
//
//   scan   bound by HBM: one workgroup per (row, segment), the segment in registers.  It leaves the best element, the sum
//          of its weights (where the row's sum is asked for) relative to its own best, and a list of its largest
//          elements with the bound that they reach.
//   pick   one workgroup per row.  Without filters: the segment where the running sum passes u S, then the token in it,
//          from one more read of the segment.  With filters: what stays is nearly always among the listed elements
//          above the largest of the segments' bounds (about 1200 of a row): their ranks and the weights in front of them
//          from buckets.  Otherwise (flat rows, ties in thousands) the row is read again, three or four times: thresholds
//          by buckets over the logits, the sums of chunks, the token.
// Sums that are taken with atomics are integers (weights in units of 2^-52 of the largest, or as fine as 62 bits allow):
// their order does not matter.
#include <algorithm>

#include "common.hpp"

namespace ddt {

constexpr int kScanThreads = 256;
constexpr int kPickThreads = 512;
constexpr int kCandidates = 2048;   // listed elements that one row's pick holds
constexpr int kCandBuckets = 1024;
constexpr int kHistBuckets = 2048;
constexpr int kChunk = 1024;        // elements per partial sum of a row that is read again
constexpr int kMaxChunks = 4096;
constexpr int kSampleMaxV = kChunk * kMaxChunks;
constexpr int kMaxSegs = 1024;
constexpr double kCut = -40.0;      // log2 of the smallest weight

struct SampleOpts {
    float tau[DDTREE_MAX_BATCH], top_p[DDTREE_MAX_BATCH], min_p[DDTREE_MAX_BATCH];
    int32_t top_k[DDTREE_MAX_BATCH];
};

struct SegStat {
    ArgPart best;
    double sum;      // of the weights relative to the segment's best
    float low;       // the smallest element with a weight
    uint32_t bound;  // key: every element that reaches it is listed (0: every finite one)
    int32_t listed;  // more than the list holds: it is not complete
    uint32_t pad;
};
static_assert(sizeof(SegStat) == 32, "one line of two 16-byte stores");

struct SamplePlan {
    int segs, seg_len, vecs, hot_rank, hot_cap;
    size_t stat_off, hot_off, part_off, bytes;
};

// Segments of 6140 elements, 24 a thread with room for a row that starts inside a 16-byte group; of 2044 where those make
// fewer than two workgroups a compute unit.  The lists together hold about 1600 of a row's largest, enough for the usual top-k.
static SamplePlan sample_plan(int batch, int T, int V)
{
    SamplePlan p{};
    const long long rows = (long long)batch * T;
    p.vecs = rows * ((V + 6139) / 6140) < 512 && V <= 2044ll * kMaxSegs ? 2 : 6;
    p.seg_len = p.vecs * 1024 - 4;
    p.segs = (V + p.seg_len - 1) / p.seg_len;
    p.hot_rank = std::min(200, std::max(16, 1600 / p.segs));
    p.hot_cap = 64;
    while (p.hot_cap < 2 * p.hot_rank) p.hot_cap *= 2;
    const size_t per = (size_t)rows * p.segs;
    p.stat_off = 0;
    p.hot_off = align_up(per * sizeof(SegStat), 256);
    p.part_off = p.hot_off + align_up(per * p.hot_cap * 8, 256);
    p.bytes = p.part_off + align_up((size_t)rows * 8, 256);
    return p;
}

// A bound on sample_plan(...).bytes over every call of at most this many rows and elements.
size_t sample_scratch_upper(int batch, int T, int V)
{
    const size_t rows = (size_t)batch * T;
    size_t most = 0;
    if (V > kSampleMaxV) V = kSampleMaxV;
    // (a segment's list is at most four times what 1600 divided by the segments asks for, or 64; short segments only below 512
    // workgroups of long ones)
    const size_t long_segs = rows * ((V + 6139) / 6140), short_segs = std::min<size_t>(rows * ((V + 2043) / 2044), 512 * 4 + rows);
    const size_t segs = std::max(long_segs, short_segs);
    most = segs * (sizeof(SegStat) + 64 * 8) + rows * (size_t)(4 * 1600) * 8 + rows * 8 + 1024;
    return align_up(most, 256);
}

// 2^t for t <= 0: 2^f, f within half of 0, from its interpolation at ten Chebyshev nodes (6e-16 off); 1 at 0 exactly.
__device__ __forceinline__ double exp2_of(double t)
{
    t = fmax(t, -64.0);
    const double n = __builtin_rint(t), f = t - n;
    double p = 0x1.e5e9f548e5725p-28;
    p = fma(p, f, 0x1.b6571de2f2351p-24);
    p = fma(p, f, 0x1.62bfe46117445p-20);
    p = fma(p, f, 0x1.ffcb76789860fp-17);
    p = fma(p, f, 0x1.4309130378460p-13);
    p = fma(p, f, 0x1.5d87fe908f88ap-10);
    p = fma(p, f, 0x1.3b2ab6fba385fp-7);
    p = fma(p, f, 0x1.c6b08d7044119p-5);
    p = fma(p, f, 0x1.ebfbdff82c590p-3);
    p = fma(p, f, 0x1.62e42fefa39f7p-1);
    p = fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

// What counts as a logit: NaN as -inf (never selected), +inf as the largest finite number.
__device__ __forceinline__ float clean(float x)
{
    const uint32_t b = __float_as_uint(x);
    if ((b & 0x7FFFFFFFu) > 0x7F800000u) return -INFINITY;
    return b == 0x7F800000u ? 3.4028235e38f : x;
}
constexpr uint32_t kKeyOfNone = 0x007FFFFFu;  // float_key(-inf)

// Elements 4 v - a .. of `n` at p; a: elements that p is behind a 16-byte boundary.
__device__ __forceinline__ float4 load_group(const float *p, int v, int a, int n)
{
    const int e = 4 * v - a;
    float4 x;
    if (e >= 0 && e + 3 < n) {
        x = *reinterpret_cast<const float4 *>(p + e);
    } else {
        x.x = e >= 0 && e < n ? p[e] : -INFINITY;
        x.y = e + 1 >= 0 && e + 1 < n ? p[e + 1] : -INFINITY;
        x.z = e + 2 >= 0 && e + 2 < n ? p[e + 2] : -INFINITY;
        x.w = e + 3 >= 0 && e + 3 < n ? p[e + 3] : -INFINITY;
    }
    x.x = clean(x.x), x.y = clean(x.y), x.z = clean(x.z), x.w = clean(x.w);
    return x;
}
__device__ __forceinline__ int behind_boundary(const float *p) { return (int)((reinterpret_cast<uintptr_t>(p) >> 2) & 3); }

template <int VECS>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(
    const float *__restrict__ logits, int T, int V, int seg_len, int segs, int hot_rank, int hot_cap,
    const int32_t *__restrict__ n_nodes, SegStat *__restrict__ stat, ArgPart *__restrict__ hot, SampleOpts opt)
{
    __shared__ ArgPart s_best[kScanThreads / 64];
    __shared__ double s_sum[kScanThreads / 64];
    __shared__ float s_low[kScanThreads / 64];
    __shared__ float s_max[kScanThreads];
    __shared__ int s_alive[kScanThreads / 64], s_listed;
    __shared__ uint32_t s_bound;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int seg = blockIdx.x, i = blockIdx.y, seq = blockIdx.z;
    if (n_nodes && i > n_nodes[seq]) return;  // padding row
    const size_t row = (size_t)seq * T + i;
    const int start = seg * seg_len, n = min(seg_len, V - start);
    const float *const p = logits + row * (size_t)V + start;
    const int a = behind_boundary(p);
    float x[VECS][4];
#pragma unroll
    for (int j = 0; j < VECS; ++j) {
        const float4 v = load_group(p, j * kScanThreads + tid, a, n);
        x[j][0] = v.x, x[j][1] = v.y, x[j][2] = v.z, x[j][3] = v.w;
    }
    const float tau = opt.tau[seq];
    const bool filtered = opt.top_k[seq] > 0 || opt.top_p[seq] < 1.0f || opt.min_p[seq] > 0.0f;
    // the sum of the row: where nothing is filtered, and where top-p goes by it
    const bool want_sum = tau > 0.0f && opt.top_k[seq] == 0 && (opt.top_p[seq] < 1.0f || !filtered);
    if (tid == 0) s_listed = 0;

    float bv = -INFINITY;
    int bi = 0x7FFFFFFF, alive = 0;
#pragma unroll
    for (int j = 0; j < VECS; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool more = x[j][e] > bv;
            bv = more ? x[j][e] : bv;
            bi = more ? 4 * (j * kScanThreads + tid) - a + e : bi;
            alive += x[j][e] > -INFINITY ? 1 : 0;
        }
    const ArgPart mine = wave_arg_max(bv > -INFINITY ? arg_part(bv, start + bi) : kNoPart);
    if (lane == 63) s_best[wave] = mine;
    s_max[tid] = bv;
    alive = wave_scan_inclusive_i32(alive);
    if (lane == 63) s_alive[wave] = alive;
    __syncthreads();
    ArgPart best = s_best[0];
    int n_alive = s_alive[0];
#pragma unroll
    for (int w = 1; w < kScanThreads / 64; ++w) best = s_best[w] > best ? s_best[w] : best, n_alive += s_alive[w];

    if (want_sum && best != kNoPart) {
        const double m = (double)key_float((uint32_t)(best >> 32)), c = 1.4426950408889634 / (double)tau;
        double sum = 0.0;
        float low = INFINITY;
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const double t = ((double)x[j][e] - m) * c;
                const bool counts = t >= kCut;
                sum += counts ? exp2_of(t) : 0.0;
                low = counts ? fminf(low, x[j][e]) : low;
            }
        sum = wave_sum_f64_lane63(sum);
        low = -wave_max_f32(-low);
        if (lane == 63) s_sum[wave] = sum, s_low[wave] = low;
    }
    if (filtered && tau > 0.0f && wave == 0) {
        // A bound that about hot_rank of the thread maxima reach, by bisection over their keys
        uint32_t k[4], lo = kKeyOfNone + 1u;
        if (n_alive > hot_cap) {
#pragma unroll
            for (int u = 0; u < 4; ++u) k[u] = float_key(s_max[u * 64 + lane]);
            auto reach = [&](uint32_t b) {
                int c = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) c += __popcll(__builtin_amdgcn_ballot_w64(k[u] >= b));
                return c;
            };
            uint32_t hi = (uint32_t)(best >> 32) + 1u;
            if (reach(lo) > hot_rank) {
                while (hi - lo > 1u) {
                    const uint32_t mid = lo + (hi - lo) / 2u;
                    const int c = reach(mid);
                    if (c >= hot_rank) lo = mid;
                    else hi = mid;
                    if (c >= hot_rank && c <= hot_rank + hot_rank / 8) break;
                }
            }
        } else {
            lo = 0u;
        }
        if (lane == 0) s_bound = lo;
    }
    __syncthreads();
    if (filtered && tau > 0.0f) {
        const uint32_t bound = s_bound;
        const uint32_t at_least = max(bound, kKeyOfNone + 1u);
        ArgPart *const list = hot + (row * segs + seg) * (size_t)hot_cap;
        if (float_key(bv) >= at_least) {
#pragma unroll
            for (int j = 0; j < VECS; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (float_key(x[j][e]) >= at_least) {
                        const int at = atomicAdd(&s_listed, 1);
                        if (at < hot_cap) list[at] = arg_part(x[j][e], start + 4 * (j * kScanThreads + tid) - a + e);
                    }
        }
        __syncthreads();
    }
    if (tid == 0) {
        SegStat s{};
        s.best = best;
        s.low = INFINITY;
        if (want_sum && best != kNoPart) {
            s.sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
            s.low = fminf(fminf(s_low[0], s_low[1]), fminf(s_low[2], s_low[3]));
        }
        s.bound = filtered && tau > 0.0f ? s_bound : 0u;
        s.listed = s_listed;
        stat[row * segs + seg] = s;
    }
}

// ---- pick: what a workgroup shares ----
struct PickShared {
    union {
        struct {
            uint32_t key[kCandidates], id[kCandidates];
            ArgPart w[kCandidates];
            uint16_t order[kCandidates];
            ArgPart mass[kCandBuckets];
            uint32_t count[kCandBuckets], cursor[kCandBuckets];
        } c;
        struct {
            ArgPart mass[kHistBuckets];
            uint32_t count[kHistBuckets];
            ArgPart list[kCandidates], w[kCandidates];
        } h;
        double chunk[kMaxChunks + kPickThreads];
        double seg[kMaxSegs];
    };
    double wave_d[kPickThreads / 64];
    ArgPart wave_u[kPickThreads / 64];
    ArgPart found, base;
    double found_d;
    int n, last, token;
};

template <class X>
__device__ __forceinline__ X shfl_up(X v, int d)
{
    static_assert(sizeof(X) == 8, "64 bits");
    const ArgPart u = __builtin_bit_cast(ArgPart, v);
    const uint32_t lo = __shfl_up((uint32_t)u, d, 64), hi = __shfl_up((uint32_t)(u >> 32), d, 64);
    return __builtin_bit_cast(X, (ArgPart)hi << 32 | lo);
}
// Sum over the threads in front of this one, and over all (both in one fixed order).
template <class X>
__device__ __forceinline__ X block_scan(X v, X *waves, X &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    X s = v;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const X o = shfl_up(s, d);
        s = lane >= d ? s + o : s;
    }
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    X before = X(0);
    total = X(0);
#pragma unroll
    for (int w = 0; w < kPickThreads / 64; ++w) {
        before = w < wave ? before + waves[w] : before;
        total += waves[w];
    }
    // (the inclusive sum less the own value, taken from the neighbour so that nothing is subtracted)
    const X up = shfl_up(s, 1);
    return before + (lane > 0 ? up : X(0));
}

// A row, and what stays of it as far as that is known.
struct PickRow {
    const float *x;
    int V, a;
    double M, c;       // largest logit, log2(e) / tau
    ArgPart floor;     // composites below it do not stay
    double min_w;      // nor do weights below this one
    __device__ __forceinline__ double log_weight(float v) const { return ((double)v - M) * c; }
    // weight of element id if it stays, else 0
    __device__ __forceinline__ double weight(float v, int id) const
    {
        const double t = log_weight(v);
        if (!(t >= kCut) || arg_part(v, id) < floor) return 0.0;
        const double w = exp2_of(t);
        return w >= min_w ? w : 0.0;
    }
    template <class F>
    __device__ __forceinline__ void each(F &&f) const
    {
        const int groups = (V + a + 3) >> 2;
        for (int g = threadIdx.x; g < groups; g += 2 * kPickThreads) {
            const float4 p = load_group(x, g, a, V), q = load_group(x, g + kPickThreads, a, V);
            const float e[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (e[u] > -INFINITY) f(e[u], 4 * (g + (u >> 2) * kPickThreads) - a + (u & 3));
        }
    }
};

// The element of [start, start + n) where the running sum, `base` in front of it, exceeds `target` (the last one with a
// weight, should rounding leave none).  c0, c1: the running sum in front of it and behind it.
__device__ int pick_locate(const PickRow &r, int start, int n, double base, double target, PickShared &sh, double &c0, double &c1)
{
    const int per = (n + kPickThreads - 1) / kPickThreads, from = start + (int)threadIdx.x * per, to = min(from + per, start + n);
    double mine = 0.0, total;
    int last = -1;
    for (int e = from; e < to; ++e) {
        const double w = r.weight(clean(r.x[e]), e);
        if (w > 0.0) last = e;
        mine += w;
    }
    if (threadIdx.x == 0) sh.last = -1, sh.token = -1;
    const double before = base + block_scan(mine, sh.wave_d, total);
    if (last >= 0) atomicMax(&sh.last, last);
    if (last >= 0 && before <= target && target < before + mine) atomicMax(&sh.token, (int)threadIdx.x);
    __syncthreads();
    // (should rounding leave no such thread: the one that holds the last element)
    const int who = sh.token >= 0 ? sh.token : sh.last >= 0 ? (sh.last - start) / per : -1;
    __syncthreads();
    if (who == (int)threadIdx.x) {
        double c = before, w = 0.0;
        int token = last;
        for (int e = from; e < to; ++e) {
            w = r.weight(clean(r.x[e]), e);
            if (w > 0.0 && (target < c + w || e == last)) {
                token = e;
                break;
            }
            c += w;
        }
        sh.token = token;
        sh.wave_d[0] = c, sh.wave_d[1] = c + w;
    }
    __syncthreads();
    c0 = sh.wave_d[0], c1 = sh.wave_d[1];
    const int token = who >= 0 ? sh.token : -1;
    __syncthreads();
    return token;
}

// The composite of the last element, in falling order, with less than `limit` in front of it: elements counted, or their
// weights summed (in units of 1 / unit).  Elements below r.floor do not take part; r.floor if all stay.
template <bool MASS>
__device__ ArgPart pick_threshold(const PickRow &r, double limit, double unit, PickShared &sh)
{
    auto value = [&](double w) -> ArgPart { return MASS ? (ArgPart)(w * unit + 0.5) : 1ull; };
    auto bucket_of = [&](double t) { return min(kHistBuckets - 1, (int)(t * (kHistBuckets / kCut))); };
    const double bound = MASS ? limit * unit : limit;
    int bucket = -1, shift = 64;
    ArgPart prefix = 0ull, base = 0ull;
    for (;;) {
        // the elements left: of one bucket of the first round, and with one prefix of the composite after that
        auto left = [&](float v, int id, double t) {
            if (!(t >= kCut) || arg_part(v, id) < r.floor) return false;
            if (bucket >= 0 && bucket_of(t) != bucket) return false;
            return shift == 64 || (arg_part(v, id) >> shift) == prefix;
        };
        const int next = shift == 64 ? (bucket < 0 ? 64 : 53) : max(shift - 11, 0);
        const int width = shift - next;
        for (int b = threadIdx.x; b < kHistBuckets; b += kPickThreads) sh.h.mass[b] = 0ull, sh.h.count[b] = 0u;
        __syncthreads();
        r.each([&](float v, int id) {
            const double t = r.log_weight(v);
            if (!left(v, id, t)) return;
            const int b = bucket < 0 ? bucket_of(t) : kHistBuckets - 1 - (int)((arg_part(v, id) >> next) & ((1ull << width) - 1ull));
            atomicAdd(&sh.h.count[b], 1u);
            if (MASS) atomicAdd(&sh.h.mass[b], value(exp2_of(t)));
        });
        __syncthreads();
        constexpr int kPer = kHistBuckets / kPickThreads;
        ArgPart v[kPer], mine = 0ull, total;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int b = (int)threadIdx.x * kPer + u;
            v[u] = MASS ? sh.h.mass[b] : (ArgPart)sh.h.count[b];
            mine += v[u];
        }
        ArgPart before = base + block_scan(mine, sh.wave_u, total);
        if ((double)(base + total) < bound || total == 0ull) {
            // (all of them stay.  Of a narrowed set only by the rounding of the weights' sum: the set's end is then the border)
            if (bucket < 0) return r.floor;
        }
        if (threadIdx.x == 0) sh.n = -1;
        __syncthreads();
        // the last bucket that holds elements and has less than the bound in front of it
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if (sh.h.count[(int)threadIdx.x * kPer + u] > 0u && (double)before < bound) atomicMax(&sh.n, (int)threadIdx.x * kPer + u);
            before += v[u];
        }
        __syncthreads();
        const int at = sh.n;
        if (at < 0) return r.floor;
        before -= mine;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if ((int)threadIdx.x * kPer + u == at) sh.base = before;
            before += v[u];
        }
        const uint32_t members = sh.h.count[at];
        __syncthreads();
        base = sh.base;
        if (bucket < 0) {
            bucket = at;
        } else {
            prefix = (shift == 64 ? 0ull : prefix << width) | (ArgPart)(kHistBuckets - 1 - at);
            shift = next;
        }
        if (members <= (uint32_t)kCandidates || shift == 0) {
            // few enough to be compared with one another
            if (threadIdx.x == 0) sh.n = 0, sh.found = ~0ull;
            __syncthreads();
            r.each([&](float v, int id) {
                const double t = r.log_weight(v);
                if (!left(v, id, t)) return;
                const int k = atomicAdd(&sh.n, 1);
                if (k < kCandidates) sh.h.list[k] = arg_part(v, id), sh.h.w[k] = value(MASS ? exp2_of(t) : 1.0);
            });
            __syncthreads();
            const int n = min(sh.n, kCandidates);
            for (int k = threadIdx.x; k < n; k += kPickThreads) {
                const ArgPart me = sh.h.list[k];
                ArgPart front = base;
                for (int o = 0; o < n; ++o) front += sh.h.list[o] > me ? sh.h.w[o] : 0ull;
                if ((double)front < bound) atomicMin(&sh.found, me);
            }
            __syncthreads();
            const ArgPart found = sh.found;
            __syncthreads();
            return found == ~0ull ? r.floor : found;
        }
    }
}

// The row read again: thresholds, sums of chunks, token.
__device__ int pick_again(PickRow r, int top_k, float top_p, float min_p, float u, PickShared &sh)
{
    double total;
    r.floor = 0ull, r.min_w = 0.0;
    __syncthreads();
    if (top_k > 0) r.floor = pick_threshold<false>(r, (double)top_k, 1.0, sh);
    if (top_p < 1.0f) {
        double mine = 0.0;
        r.each([&](float v, int id) { mine += r.weight(v, id); });
        (void)block_scan(mine, sh.wave_d, total);
        // as fine as sums below 2^62 allow
        const double unit = __builtin_amdgcn_ldexp(1.0, 61 - __builtin_amdgcn_frexp_exp(total));
        r.floor = pick_threshold<true>(r, (double)top_p * total, unit, sh);
    }
    r.min_w = (double)min_p;
    const int chunks = (r.V + kChunk - 1) / kChunk, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int k = wave; k < chunks; k += kPickThreads / 64) {
        const int start = k * kChunk, n = min(kChunk, r.V - start), a = behind_boundary(r.x + start);
        double sum = 0.0;
#pragma unroll
        for (int g = 0; g < kChunk / 256 + 1; ++g) {  // (one group more where the chunk starts inside one)
            if (4 * (g * 64) - a >= n) break;
            const float4 p = load_group(r.x + start, g * 64 + lane, a, n);
            const int id = start + 4 * (g * 64 + lane) - a;
            sum += (r.weight(p.x, id) + r.weight(p.y, id + 1)) + (r.weight(p.z, id + 2) + r.weight(p.w, id + 3));
        }
        sum = wave_sum_f64_lane63(sum);
        if (lane == 63) sh.chunk[k] = sum;
    }
    __syncthreads();
    const int per = (chunks + kPickThreads - 1) / kPickThreads, from = (int)threadIdx.x * per, to = min(from + per, chunks);
    double mine = 0.0;
    for (int k = from; k < to; ++k) mine += sh.chunk[k];
    double before = block_scan(mine, sh.wave_d, total);
    const double target = (double)u * total;
    if (threadIdx.x == 0) sh.n = -1;
    __syncthreads();
    // the last chunk with a weight that has at most the target in front of it
    for (int k = from; k < to; ++k) {
        if (sh.chunk[k] > 0.0 && before <= target) atomicMax(&sh.n, k);
        const double b = before;
        before += sh.chunk[k];
        sh.chunk[k] = b;  // from now on: the sum in front of it
    }
    __syncthreads();
    const int k = sh.n;
    if (k < 0) return -1;
    const double base = sh.chunk[k];
    __syncthreads();
    double c0, c1;
    return pick_locate(r, k * kChunk, min(kChunk, r.V - k * kChunk), base, target, sh, c0, c1);
}

__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(
    const float *__restrict__ logits, int T, int V, int seg_len, int segs, int hot_cap,
    const int32_t *__restrict__ n_nodes, const float *__restrict__ uniforms, const SegStat *__restrict__ stat_all,
    const ArgPart *__restrict__ hot_all, ArgPart *__restrict__ part, int32_t *__restrict__ tokens, SampleOpts opt)
{
    __shared__ PickShared sh;
    const int tid = threadIdx.x, i = blockIdx.x, seq = blockIdx.y;
    if (n_nodes && i > n_nodes[seq]) return;  // padding row
    const size_t row = (size_t)seq * T + i;
    const SegStat *const stat = stat_all + row * segs;
    const ArgPart *const hot = hot_all + row * segs * (size_t)hot_cap;
    const float tau = opt.tau[seq], top_p = opt.top_p[seq], min_p = opt.min_p[seq];
    const int top_k = opt.top_k[seq];
    // u from [0, 1): what is below, or no number, counts as 0, what is above as the largest float below 1
    float u = uniforms[row];
    const uint32_t ub = __float_as_uint(u);
    u = ub > 0x7F800000u ? 0.0f : ub >= 0x3F800000u ? 0x1.fffffep-1f : u;

    // the row's best, and the largest of the bounds (a list that is not complete: no bound holds)
    ArgPart best = kNoPart;
    uint32_t bound = 0u;
    for (int s = tid; s < segs; s += kPickThreads) {
        const ArgPart b = stat[s].best;
        best = b > best ? b : best;
        bound = max(bound, stat[s].listed > hot_cap ? ~0u : stat[s].bound);
    }
    best = wave_arg_max(best);
    bound = ~wave_min_u32(~bound);
    if ((tid & 63) == 63) sh.wave_u[tid >> 6] = best, sh.wave_d[tid >> 6] = (double)bound;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPickThreads / 64; ++w) {
        best = sh.wave_u[w] > best ? sh.wave_u[w] : best;
        bound = max(bound, (uint32_t)sh.wave_d[w]);
    }
    __syncthreads();

    auto done = [&](int token) {
        if (tid == 0) {
            if (tokens) tokens[row] = token;
            else part[row] = 1ull << 32 | (uint32_t)~token;
        }
    };
    if (best == kNoPart) return done(-1);
    if (!(tau > 0.0f)) return done(arg_token(best));

    PickRow r;
    r.x = logits + row * (size_t)V;
    r.V = V;
    r.a = behind_boundary(r.x);
    r.M = (double)key_float((uint32_t)(best >> 32));
    r.c = 1.4426950408889634 / (double)tau;
    r.floor = 0ull;
    r.min_w = 0.0;
    const bool filtered = top_k > 0 || top_p < 1.0f || min_p > 0.0f;
    const bool has_sum = top_k == 0 && (top_p < 1.0f || !filtered);

    // The row's sum.  A segment has also counted elements that are too small beside the row's best but not beside its own:
    // `slack` bounds what they add (each is below 2^-40, if there are any).  A decision that this could change is left to
    // the row read again.
    double Z = 0.0, slack = 0.0;
    if (has_sum) {
        const int per = (segs + kPickThreads - 1) / kPickThreads, from = tid * per, to = min(from + per, segs);
        double mine = 0.0;
        bool doubt = false;
        for (int s = from; s < to; ++s) {
            double w = 0.0;
            if (stat[s].best != kNoPart) {
                const double t = r.log_weight(key_float((uint32_t)(stat[s].best >> 32)));
                if (t >= kCut) {
                    w = exp2_of(t) * stat[s].sum;
                    doubt = doubt || !(r.log_weight(stat[s].low) >= kCut);
                }
            }
            sh.seg[s] = w;
            mine += w;
        }
        const double before = block_scan(mine, sh.wave_d, Z);
        if (__syncthreads_or(doubt ? 1 : 0)) slack = (double)V * 0x1p-40;
        if (!filtered) {
            const double target = (double)u * Z;
            if (tid == 0) sh.n = -1;
            __syncthreads();
            double b = before;
            for (int s = from; s < to; ++s) {
                if (sh.seg[s] > 0.0 && b <= target) atomicMax(&sh.n, s);
                const double w = sh.seg[s];
                sh.seg[s] = b;
                b += w;
            }
            __syncthreads();
            const int s = sh.n;
            const double base = sh.seg[s];
            __syncthreads();
            double c0, c1;
            int token = pick_locate(r, s * seg_len, min(seg_len, V - s * seg_len), base, target, sh, c0, c1);
            if (slack > 0.0 && !(c0 <= (double)u * (Z - slack) && target < c1 - slack)) token = pick_again(r, 0, 1.0f, 0.0f, u, sh);
            return done(token);
        }
        __syncthreads();
    }

    // ---- the listed elements that reach the bound ----
    auto &c = sh.c;
    const uint32_t at_least = max(bound, kKeyOfNone + 1u);
    if (tid == 0) sh.n = 0;
    for (int b = tid; b < kCandBuckets; b += kPickThreads) c.mass[b] = 0ull, c.count[b] = 0u;
    __syncthreads();
    if (bound != ~0u) {
        for (int k = tid; k < segs * hot_cap; k += kPickThreads) {
            const int s = k / hot_cap, e = k - s * hot_cap;
            if (e < stat[s].listed) {
                const ArgPart h = hot[k];
                if ((uint32_t)(h >> 32) >= at_least) {
                    const int at = atomicAdd(&sh.n, 1);
                    if (at < kCandidates) c.key[at] = (uint32_t)(h >> 32), c.id[at] = (uint32_t)arg_token(h);
                }
            }
        }
    }
    __syncthreads();
    const int n = sh.n;
    bool again = bound == ~0u || n > kCandidates;
    // (below the bound nothing has a weight: the list is all there is)
    const double t_bound = bound == 0u ? -1e30 : again ? 0.0 : r.log_weight(key_float(bound));
    const bool all = bound == 0u || t_bound < kCut;
    if (!again) {
        // buckets in falling order: equal steps between the best and the least listed (for elements without a weight, the last)
        const double span = fmax(all ? kCut : t_bound, kCut);
        const double step = span < 0.0 ? (double)(kCandBuckets - 1) / span : 0.0;
        auto bucket = [&](uint32_t key) { return min(kCandBuckets - 1, max(0, (int)(fmax(r.log_weight(key_float(key)), 2.0 * kCut) * step))); };
        for (int k = tid; k < n; k += kPickThreads) {
            const double t = r.log_weight(key_float(c.key[k]));
            const ArgPart w = t >= kCut ? (ArgPart)(exp2_of(t) * 0x1p52 + 0.5) : 0ull;
            c.w[k] = w;
            const int b = bucket(c.key[k]);
            atomicAdd(&c.mass[b], w);
            atomicAdd(&c.count[b], 1u);
        }
        __syncthreads();
        constexpr int kPer = kCandBuckets / kPickThreads;
        ArgPart m[kPer], q[kPer], m_mine = 0ull, q_mine = 0ull, m_all, q_all;
#pragma unroll
        for (int v = 0; v < kPer; ++v) {
            m[v] = c.mass[tid * kPer + v], q[v] = c.count[tid * kPer + v];
            m_mine += m[v], q_mine += q[v];
        }
        ArgPart m_front = block_scan(m_mine, sh.wave_u, m_all), q_front = block_scan(q_mine, sh.wave_u, q_all);
#pragma unroll
        for (int v = 0; v < kPer; ++v) {
            c.mass[tid * kPer + v] = m_front, c.cursor[tid * kPer + v] = (uint32_t)q_front;
            m_front += m[v], q_front += q[v];
        }
        __syncthreads();
        for (int k = tid; k < n; k += kPickThreads) c.order[atomicAdd(&c.cursor[bucket(c.key[k])], 1u)] = (uint16_t)k;
        __syncthreads();
        // rank and weight in front of each, of at most kCandidates / kPickThreads elements a thread
        constexpr int kEach = kCandidates / kPickThreads;
        int rank[kEach];
        ArgPart front[kEach];
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            const int k = tid + v * kPickThreads;
            rank[v] = 0, front[v] = 0ull;
            if (k >= n) continue;
            const int b = bucket(c.key[k]), end = (int)c.cursor[b], begin = end - (int)c.count[b];
            ArgPart f = c.mass[b];
            int before = begin;
            for (int o = begin; o < end; ++o) {
                const int j = c.order[o];
                const bool larger = c.key[j] > c.key[k] || (c.key[j] == c.key[k] && c.id[j] < c.id[k]);
                f += larger ? c.w[j] : 0ull;
                before += larger ? 1 : 0;
            }
            rank[v] = before, front[v] = f;
        }
        // what top-k keeps, and its weight
        if (top_k > 0) {
            ArgPart kept = 0ull, sum;
#pragma unroll
            for (int v = 0; v < kEach; ++v)
                if (tid + v * kPickThreads < n && rank[v] < top_k) kept += c.w[tid + v * kPickThreads];
            (void)block_scan(kept, sh.wave_u, sum);
            Z = (double)sum * 0x1p-52;
        }
        const double limit = (double)top_p * Z * 0x1p52, doubt = slack * 0x1p52;
        // Everything that stays is listed if top-k, top-p or min-p ends above the bound, or nothing below it has a weight.
        // (The limit of top-p behind a top-k that the list does not hold is not known.)
        const bool k_ends = all || (top_k > 0 && n >= top_k);
        const bool ends = k_ends || ((top_k == 0 || top_p >= 1.0f) && ((top_p < 1.0f && (double)m_all >= limit) ||
                                                                      (min_p > 0.0f && exp2_of(t_bound) < (double)min_p)));
        bool unsure = false;
        ArgPart stays[kEach], kept = 0ull, S;
#pragma unroll
        for (int v = 0; v < kEach; ++v) {
            const int k = tid + v * kPickThreads;
            stays[v] = 0ull;
            if (k >= n) continue;
            const double f = (double)front[v];
            unsure = unsure || (top_p < 1.0f && slack > 0.0 && f > limit - doubt && f < limit);
            const double t = r.log_weight(key_float(c.key[k]));
            if ((top_k == 0 || rank[v] < top_k) && (top_p >= 1.0f || f < limit) && t >= kCut &&
                (min_p == 0.0f || exp2_of(t) >= (double)min_p))
                stays[v] = c.w[k];
            kept += stays[v];
        }
        if (__syncthreads_or((unsure || !ends) ? 1 : 0)) {
            again = true;
        } else {
            // in the order of ids: buckets of ids, then the elements of the bucket where the running sum passes u S
            (void)block_scan(kept, sh.wave_u, S);
            const double target = (double)u * (double)S;
            const int id_shift = max(0, 32 - __builtin_clz((unsigned)max(V - 1, 1)) - 10);
            for (int b = tid; b < kCandBuckets; b += kPickThreads) c.mass[b] = 0ull;
            if (tid == 0) sh.n = -1, sh.token = -1, sh.last = 0;
            __syncthreads();
#pragma unroll
            for (int v = 0; v < kEach; ++v)
                if (stays[v] != 0ull) atomicAdd(&c.mass[c.id[tid + v * kPickThreads] >> id_shift], stays[v]);
            __syncthreads();
            m_mine = 0ull;
#pragma unroll
            for (int v = 0; v < kPer; ++v) m[v] = c.mass[tid * kPer + v], m_mine += m[v];
            m_front = block_scan(m_mine, sh.wave_u, m_all);
#pragma unroll
            for (int v = 0; v < kPer; ++v) {
                c.mass[tid * kPer + v] = m_front;
                if (m[v] > 0ull && (double)m_front <= target) atomicMax(&sh.n, tid * kPer + v);
                m_front += m[v];
            }
            __syncthreads();
            const int at = sh.n;
            // (the bucket's elements: at most all)
#pragma unroll
            for (int v = 0; v < kEach; ++v) {
                const int k = tid + v * kPickThreads;
                if (stays[v] != 0ull && (int)(c.id[k] >> id_shift) == at) {
                    const int o = atomicAdd(&sh.last, 1);
                    c.order[o] = (uint16_t)k;
                }
            }
            __syncthreads();
            const int in = sh.last;
            const ArgPart base = c.mass[at];
            // the last of them, by id, with at most the target in front of it
            for (int o = tid; o < in; o += kPickThreads) {
                const int k = c.order[o];
                ArgPart f = base;
                for (int j = 0; j < in; ++j) f += c.id[c.order[j]] < c.id[k] ? c.w[c.order[j]] : 0ull;
                if ((double)f <= target) atomicMax(&sh.token, (int)c.id[k]);
            }
            __syncthreads();
            return done(sh.token);
        }
    }
    if (again) done(pick_again(r, top_k, top_p, min_p, u, sh));
}

// Segments tile a row, a thread's registers hold them wherever the row starts, and the scratch of a shape covers
// every smaller one.  0, or 10031 and up.
int sample_selftest_host()
{
    for (int V : {1, 2, 63, 1024, 2044, 2045, 6140, 6141, 32003, 50021, 151936, 262144, 1000003, 2093057, kSampleMaxV})
        for (int T : {1, 2, 17, 65, 257, 513, 1025})
            for (int batch : {1, 2, 5, 16, 64}) {
                const SamplePlan p = sample_plan(batch, T, V);
                if ((long long)(p.segs - 1) * p.seg_len >= V || (long long)p.segs * p.seg_len < V || p.segs > kMaxSegs) return 10031;
                if (p.seg_len + 3 > p.vecs * kScanThreads * 4 || (p.vecs != 2 && p.vecs != 6)) return 10032;
                if (p.hot_cap < p.hot_rank || p.hot_rank > kScanThreads) return 10033;
                const size_t per = (size_t)batch * T * p.segs;
                if (p.hot_off < per * sizeof(SegStat) || p.part_off < p.hot_off + per * p.hot_cap * 8 || p.bytes < p.part_off + (size_t)batch * T * 8 ||
                    ((p.hot_off | p.part_off) & 255u))
                    return 10034;
                const size_t have = sample_scratch_upper(batch, T, V);
                for (int b = 1; b <= batch; b += 1 + b / 2)
                    for (int t = 1; t <= T; t += 1 + t / 3)
                        for (int v = 1; v <= V; v += 1 + v / 2)
                            if (sample_plan(b, t, v).bytes > have) return 10035;
            }
    return 0;
}

}  // namespace ddt

// Options of the sequences: in range, or false.
static bool sample_opts(ddt::SampleOpts &o, int batch, const float *temperature, const int32_t *top_k, const float *top_p, const float *min_p)
{
    if (!temperature) return false;
    for (int s = 0; s < batch; ++s) {
        o.tau[s] = temperature[s];
        o.top_k[s] = top_k ? top_k[s] : 0;
        o.top_p[s] = top_p ? top_p[s] : 1.0f;
        o.min_p[s] = min_p ? min_p[s] : 0.0f;
        // (compared by their bits: the compiler takes a comparison to have no NaN in it)
        auto at_most = [](float x, float most) {
            uint32_t b, m;
            __builtin_memcpy(&b, &x, 4);
            __builtin_memcpy(&m, &most, 4);
            return b <= m || b == 0x80000000u;  // (not negative, but for -0)
        };
        if (!at_most(o.tau[s], 1e30f) || !at_most(o.top_p[s], 1.0f) || o.top_p[s] == 0.0f || !at_most(o.min_p[s], 1.0f) || o.top_k[s] < 0)
            return false;
    }
    return true;
}

static int sample_rows(const float *logits, int batch, int T, int V, const int32_t *n_nodes, const float *temperature,
                       const int32_t *top_k, const float *top_p, const float *min_p, const float *uniforms, int32_t *tokens,
                       ddt::ArgPart **part, void *workspace, size_t workspace_bytes, hipStream_t st)
{
    using namespace ddt;
    if (!logits || !uniforms || batch < 1 || batch > DDTREE_MAX_BATCH || T < 1 || T > DDTREE_MAX_N + 1 || V < 1 || V > kSampleMaxV)
        return DDTREE_ERR_ARG;
    if ((reinterpret_cast<uintptr_t>(logits) & 3u) || (reinterpret_cast<uintptr_t>(uniforms) & 3u)) return DDTREE_ERR_ARG;
    SampleOpts opt;
    if (!sample_opts(opt, batch, temperature, top_k, top_p, min_p)) return DDTREE_ERR_ARG;
    const SamplePlan p = sample_plan(batch, T, V);
    if (!ws_ok(workspace, workspace_bytes, p.bytes)) return DDTREE_ERR_WORKSPACE;
    char *const ws = static_cast<char *>(workspace);
    SegStat *const stat = reinterpret_cast<SegStat *>(ws + p.stat_off);
    ArgPart *const hot = reinterpret_cast<ArgPart *>(ws + p.hot_off);
    *part = reinterpret_cast<ArgPart *>(ws + p.part_off);
    auto *scan = p.vecs == 2 ? sample_scan_kernel<2> : sample_scan_kernel<6>;
    DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_SCAN, st, scan, dim3(p.segs, T, batch), dim3(kScanThreads), 0, st, logits, T, V, p.seg_len, p.segs,
               p.hot_rank, p.hot_cap, n_nodes, stat, hot, opt);
    DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_PICK, st, sample_pick_kernel, dim3(T, batch), dim3(kPickThreads), 0, st, logits, T, V, p.seg_len, p.segs,
               p.hot_cap, n_nodes, uniforms, stat, hot, *part, tokens, opt);
    return launch_status();
}

extern "C" int ddtree_sample(const float *logits, int batch, int T, int V, const float *temperature, const int32_t *top_k,
                             const float *top_p, const float *min_p, const float *uniforms, int32_t *tokens, void *workspace,
                             size_t workspace_bytes, void *stream)
{
    if (!tokens || (reinterpret_cast<uintptr_t>(tokens) & 3u)) return DDTREE_ERR_ARG;
    ddt::ArgPart *part;
    return sample_rows(logits, batch, T, V, nullptr, temperature, top_k, top_p, min_p, uniforms, tokens, &part, workspace,
                       workspace_bytes, ddt::as_stream(stream));
}

extern "C" int ddtree_accept_filtered(const float *target_logits, int batch, int T, int V, const int32_t *tokens,
                                      const int32_t *parent, const int32_t *depth, const int32_t *n_nodes,
                                      const float *temperature, const int32_t *top_k, const float *top_p,
                                      const float *min_p, const float *uniforms, int32_t *path, int32_t *n_accepted,
                                      int32_t *bonus_token, int32_t *posterior, int B, void *workspace,
                                      size_t workspace_bytes, void *stream)
{
    using namespace ddt;
    if (!tokens || !parent || !depth || !n_nodes || !path || !n_accepted || !bonus_token || T < 2 || B < 1 || B > DDTREE_MAX_B)
        return DDTREE_ERR_ARG;
    ArgPart *part = nullptr;
    const int rc = sample_rows(target_logits, batch, T, V, n_nodes, temperature, top_k, top_p, min_p, uniforms, nullptr, &part,
                               workspace, workspace_bytes, as_stream(stream));
    if (rc != DDTREE_OK) return rc;
    accept_walk_launch(part, batch, T, 1, B, tokens, parent, depth, n_nodes, path, n_accepted, bonus_token, posterior, as_stream(stream));
    return launch_status();
}
