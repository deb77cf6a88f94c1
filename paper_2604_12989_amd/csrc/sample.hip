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
//          from one more read of the segment.  With filters: what stays is mostly among the listed elements above the
//          largest of the segments' bounds (about 1200 of a row): their ranks and the weights in front of them from
//          buckets.  A row of which that does not hold (thousands of tokens stay) is put on a list.
//   steps, gather, again   what is on the list.  Many workgroups a row: each leaves, for 8192 elements, the weight (and the number) in
//          front of each of 256 steps of the logit; they add these up and gather the elements of the one step where the
//          border lies; then one puts those in order and draws the token.  (In one launch, the last workgroup of a row going
//          on by itself, the fences between the XCDs' caches took 20 times as long as the work.)
// Measured (begin to end of each launch), 257 rows of 151936, top-k 50: scan 28 to 30 us (5.2 to 5.5 TB/s), pick 11, the empty list 4.  256 flat
// rows, N(0, 1/4), top-p 0.95: scan 65 (some 25 fp64 operations an element), pick 25, steps 73, gather 85, again 25 (of 257, one row without a
// place, 309); one flat row: 6, 18, 6, 8, 20.  Rows whose border lies in a step with more than kStepList
// elements are left to one workgroup each: equal logits, but also flat rows by min-p or a large top-k, where the steps are as
// wide as the 40 powers of two that weights span make them (again: 16 rows N(0, 4) at temperature 2 by min-p 0.02: 95 us; 16 rows
// N(0, 1/4) by top-k 20000: 242; 16 rows of equal logits by top-p: 1.7 ms).
// Sums that are taken with atomics are integers (weights in units of 2^-52 of the largest, or as fine as 63 bits allow):
// their order does not matter.
#include <algorithm>

#include "common.hpp"

namespace ddt {

constexpr int kScanThreads = 256;
constexpr int kPickThreads = 256;
constexpr int kStepThreads = 512;
constexpr int kAgainThreads = 512;
constexpr int kStepGrid = 1024, kAgainGrid = 256;  // workgroups that look for rows on the list
constexpr int kPart = 8192;         // elements of a row that a workgroup takes at a time there
constexpr int kSteps = 256;         // steps of the logit
constexpr int kStepList = 4096;     // elements of one step that are put in order
constexpr int kSlots = 256;         // rows on the list that many workgroups take
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
    double sum;      // of the weights relative to the segment's best; where the row's sum is not asked for, a bound on it
    float low;       // the smallest element with a weight
    uint32_t bound;  // key: every element that reaches it is listed (0: every finite one)
    int32_t listed;  // more than the list holds: it is not complete
    uint32_t pad;
};
static_assert(sizeof(SegStat) == 32, "one line of two 16-byte stores");

struct SamplePlan {
    int segs, seg_len, vecs, hot, hot_cap;  // elements that a list is to hold, and room for
    int parts, slots;  // of a row on the list; rows that the steps' sums have room for
    size_t stat_off, hot_off, part_off, hard_off, step_off, few_off, bytes;
};

// A row on the list, and what is known of it.
struct HardRow {
    double unit, best;  // units of its integer weights, its largest logit
    double scale;       // steps of the logit for a log-weight
    int32_t row;
    int32_t border, listed;  // the step whose elements were gathered (-1: none yet), their number
    int32_t pad;
};
// In front of each step of the logit, over kPart elements: their weights and their number.
struct StepSum {
    ArgPart mass, count;
};

// How many of its largest elements a segment lists, and the room for them (the number that reach the bound varies).  The
// lists together hold about 1400 of a row's largest, enough for the usual top-k.
static int list_size(int segs) { return std::min(200, std::max(16, 1400 / segs)); }
static int list_room(int segs)
{
    int room = 64;
    while (5 * room < 8 * list_size(segs)) room *= 2;
    return room;
}
static void sample_layout(SamplePlan &p, long long rows, int V)
{
    p.hot = list_size(p.segs);
    p.hot_cap = list_room(p.segs);
    p.parts = (V + kPart - 1) / kPart;
    p.slots = (int)std::min<long long>(rows, kSlots);
    const size_t per = (size_t)rows * p.segs;
    p.stat_off = 0;
    p.hot_off = align_up(per * sizeof(SegStat), 256);
    p.part_off = p.hot_off + align_up(per * p.hot_cap * 8, 256);
    p.hard_off = p.part_off + align_up((size_t)rows * 8, 256);
    p.step_off = p.hard_off + align_up(256 + (size_t)rows * sizeof(HardRow), 256);
    p.few_off = p.step_off + align_up((size_t)p.slots * p.parts * ((kSteps + 1) * sizeof(StepSum)), 256);
    p.bytes = p.few_off + align_up((size_t)p.slots * kStepList * 8, 256);
}

// Segments of 6144 elements, 24 a thread; of 2048 where those make fewer than two workgroups a compute unit.
static SamplePlan sample_plan(int batch, int T, int V)
{
    SamplePlan p{};
    const long long rows = (long long)batch * T;
    p.vecs = rows * ((V + 6143) / 6144) < 512 && V <= 2048ll * kMaxSegs ? 2 : 6;
    p.seg_len = p.vecs * 1024;
    p.segs = (V + p.seg_len - 1) / p.seg_len;
    sample_layout(p, rows, V);
    return p;
}

// A bound on sample_plan(...).bytes over every call of at most this many rows and elements: the largest layout for any
// number of segments, the short ones with no more rows than leave them short.
size_t sample_scratch_upper(int batch, int T, int V)
{
    const long long rows = (long long)batch * T;
    size_t most = 0;
    if (V > kSampleMaxV) V = kSampleMaxV;
    for (int vecs : {2, 6})
        for (int segs = 1; segs <= kMaxSegs && (segs - 1) * (vecs * 1024ll) < V; ++segs) {
            const long long longs = ((segs - 1) * 2048ll + 1 + 6143) / 6144;  // at least, with `segs` short ones
            SamplePlan p{};
            p.segs = segs;
            sample_layout(p, vecs == 6 ? rows : std::min(rows, std::max(1ll, 511 / longs)), V);
            most = std::max(most, p.bytes);
        }
    return most;
}

// 2^t for t <= 0: 2^f, f within half of 0, from its interpolation at ten Chebyshev nodes (6e-16 off); 1 at 0 exactly.
__device__ __forceinline__ double exp2_of(double t)
{
    // (rounded by the addition of 1.5 2^52, whose low word is then the integer: the conversions and v_ldexp_f64 take four times
    // an addition's time)
    t = fmax(t, -64.0);
    const double shifted = t + 0x1.8p52, f = t - (shifted - 0x1.8p52);
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
    return __hiloint2double(__double2hiint(p) + (__double2loint(shifted) << 20), __double2loint(p));
}

// What counts as a logit: NaN as -inf (never selected), +inf as the largest finite number.
__device__ __forceinline__ float clean(float x)
{
    // (The median of three is the smaller of the other two where one is no number; in the compiler's own terms there are none.  A
    // signalling NaN would be made a quiet one inside it, by its first minimum, and be left out of the second, with the largest
    // finite number as the result: the maximum of x with itself makes it quiet before.)
    float y;
    asm("v_max_f32 %0, %1, %1\n\tv_med3_f32 %0, %0, %2, %3" : "=&v"(y) : "v"(x), "v"(-INFINITY), "v"(3.4028235e38f));
    return y;
}
constexpr uint32_t kKeyOfNone = 0x007FFFFFu;  // float_key(-inf)

// A run of elements as the 16-byte groups inside it and up to six elements at its edges: thread e < head has element e, thread 4 + e
// element head + 4 groups + e.  (Groups are loaded at clamped places and masked afterwards: under a branch each load would
// be waited for before the next one, 44 us for a scan that takes 30.)
struct Run {
    const float *p;
    int n, head, groups;
    __device__ __forceinline__ Run(const float *from, int len) : p(from), n(len)
    {
        head = min(n, (int)((4 - ((reinterpret_cast<uintptr_t>(p) >> 2) & 3)) & 3));
        groups = (n - head) >> 2;
    }
    __device__ __forceinline__ int id(int g) const { return head + 4 * g; }
    __device__ __forceinline__ float4 load(int g) const  // (groups > 0)
    {
        return reinterpret_cast<const float4 *>(p + head)[min(g, groups - 1)];
    }
    __device__ __forceinline__ void four(int g, const float4 &x, float (&e)[4]) const
    {
        const bool in = g < groups;
        e[0] = in ? clean(x.x) : -INFINITY, e[1] = in ? clean(x.y) : -INFINITY;
        e[2] = in ? clean(x.z) : -INFINITY, e[3] = in ? clean(x.w) : -INFINITY;
    }
    __device__ __forceinline__ int edge_id() const
    {
        const int t = threadIdx.x;
        return t < 4 ? (t < head ? t : -1) : t < 8 && head + 4 * groups + (t - 4) < n ? head + 4 * groups + (t - 4) : -1;
    }
};

// Sum over the wave; valid in lane 63 only.
__device__ __forceinline__ float wave_sum_f32_lane63(float v)
{
    v += dpp_f<0xB1>(0.0f, v);
    v += dpp_f<0x4E>(0.0f, v);
    v += dpp_f<0x141>(0.0f, v);
    v += dpp_f<0x140>(0.0f, v);
    v += dpp_f<0x142, 0xA>(0.0f, v);
    return v + dpp_f<0x143, 0xC>(0.0f, v);
}

template <int VECS>
__global__ __launch_bounds__(kScanThreads) void sample_scan_kernel(
    const float *__restrict__ logits, int T, int V, int seg_len, int segs, int hot_size, int hot_cap,
    const int32_t *__restrict__ n_nodes, SegStat *__restrict__ stat, ArgPart *__restrict__ hot, uint32_t *__restrict__ n_hard,
    SampleOpts opt)
{
    __shared__ ArgPart s_best[kScanThreads / 64];
    __shared__ double s_sum[kScanThreads / 64];
    __shared__ float s_low[kScanThreads / 64];
    __shared__ float s_max[kScanThreads];
    __shared__ int s_alive[kScanThreads / 64], s_listed;
    __shared__ uint32_t s_bound;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int seg = blockIdx.x, i = blockIdx.y, seq = blockIdx.z;
    if (tid == 0 && (seg | i | seq) == 0) *n_hard = 0u;
    if (n_nodes && i > n_nodes[seq]) return;  // padding row
    const size_t row = (size_t)seq * T + i;
    const int start = seg * seg_len, n = min(seg_len, V - start);
    const float *const p = logits + row * (size_t)V + start;
    const Run run(p, n);
    float4 raw[VECS];
    if (run.groups > 0)
#pragma unroll
        for (int j = 0; j < VECS; ++j) raw[j] = run.load(j * kScanThreads + tid);
    const int edge = run.edge_id();
    const float at_edge = edge >= 0 ? clean(p[edge]) : -INFINITY;
    float x[VECS][4];
#pragma unroll
    for (int j = 0; j < VECS; ++j) run.four(j * kScanThreads + tid, raw[j], x[j]);
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
            bi = more ? run.id(j * kScanThreads + tid) + e : bi;
            alive += x[j][e] > -INFINITY ? 1 : 0;
        }
    ArgPart mine = bv > -INFINITY ? arg_part(bv, start + bi) : kNoPart;
    if (at_edge > -INFINITY) {
        const ArgPart o = arg_part(at_edge, start + edge);
        mine = o > mine ? o : mine;
        bv = fmaxf(bv, at_edge);
        ++alive;
    }
    mine = wave_arg_max(mine);
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
        auto add = [&](float v) {
            const double t = ((double)v - m) * c;
            const bool counts = t >= kCut;
            sum += counts ? exp2_of(t) : 0.0;
            low = counts ? fminf(low, v) : low;
        };
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) add(x[j][e]);
        if (wave == 0) add(at_edge);
        sum = wave_sum_f64_lane63(sum);
        low = -wave_max_f32(-low);
        if (lane == 63) s_sum[wave] = sum, s_low[wave] = low;
    }
    if (filtered && !want_sum && tau > 0.0f && wave == 1) {
        // (no four threads' elements weigh more than the largest of them each: at most 16 VECS + 4 times the sum, mostly a few times.
        // Beside the bisection, by a wave that waits for it)
        const float m = key_float((uint32_t)(best >> 32)), c = fminf(1.44269504f * __builtin_amdgcn_rcpf(tau), 3.4028235e38f);
        const float top = fmaxf(fmaxf(s_max[lane], s_max[64 + lane]), fmaxf(s_max[128 + lane], s_max[192 + lane]));
        const float sum = wave_sum_f32_lane63(__builtin_amdgcn_exp2f(fmaxf((top - m) * c, -64.0f)));
        if (lane == 63) s_sum[0] = (double)(sum * (16 * VECS + 4)), s_sum[1] = s_sum[2] = s_sum[3] = 0.0;
    }
    if (filtered && tau > 0.0f && wave == 0) {
        // A bound that about `size` elements reach, by bisection over the keys of the thread maxima: as many as
        // 256 (1 - e^(-size / 256)) of these reach a bound that `size` elements at random places do.  Of top-k's tokens a
        // segment has its share and some more; too few listed (rows that are not at random) go on the list of rows.
        uint32_t k[4], lo = kKeyOfNone + 1u;
        if (n_alive > hot_cap) {
            const int top_k = opt.top_k[seq];
            const int size = top_k > 0 ? min(hot_size, 3 * top_k / segs + 16) : hot_size;
            const int rank = max(1, (int)(256.0f - 256.0f * __builtin_amdgcn_exp2f((float)size * (-1.44269504f / 256.0f))));
#pragma unroll
            for (int u = 0; u < 4; ++u) k[u] = float_key(s_max[u * 64 + lane]);
            auto reach = [&](uint32_t b) {
                int c = 0;
#pragma unroll
                for (int u = 0; u < 4; ++u) c += __popcll(__builtin_amdgcn_ballot_w64(k[u] >= b));
                return c;
            };
            lo = max(lo, wave_min_u32(min(min(k[0], k[1]), min(k[2], k[3]))));
            uint32_t hi = (uint32_t)(best >> 32) + 1u;
            if (reach(lo) > rank) {
                while (hi - lo > 1u) {
                    const uint32_t mid = lo + (hi - lo) / 2u;
                    const int c = reach(mid);
                    if (c >= rank) lo = mid;
                    else hi = mid;
                    if (c >= rank && c <= rank + rank / 8) break;
                }
            }
        } else {
            lo = 0u;
        }
        if (lane == 0) s_bound = lo;
    }
    __syncthreads();
    if (filtered && tau > 0.0f) {
        const float least = key_float(max(s_bound, kKeyOfNone + 1u));
        ArgPart *const list = hot + (row * segs + seg) * (size_t)hot_cap;
        // (the wave's share of the list is taken at once: an LDS atomic for each element costs the scan 8 us)
        int listed = 0;
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) listed += __popcll(__builtin_amdgcn_ballot_w64(x[j][e] >= least));
        int at = 0;
        if (lane == 0 && listed > 0) at = atomicAdd(&s_listed, listed);
        at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
        for (int j = 0; j < VECS; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const unsigned long long who = __builtin_amdgcn_ballot_w64(x[j][e] >= least);
                if (who == 0ull) continue;
                const int mine = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
                if (x[j][e] >= least && mine < hot_cap) list[mine] = arg_part(x[j][e], start + run.id(j * kScanThreads + tid) + e);
                at += __popcll(who);
            }
        if (at_edge >= least) {
            const int mine = atomicAdd(&s_listed, 1);
            if (mine < hot_cap) list[mine] = arg_part(at_edge, start + edge);
        }
        __syncthreads();
    }
    if (tid == 0) {
        SegStat s{};
        s.best = best;
        s.low = INFINITY;
        if (tau > 0.0f && best != kNoPart) s.sum = (s_sum[0] + s_sum[1]) + (s_sum[2] + s_sum[3]);
        if (want_sum && best != kNoPart) {
            s.low = fminf(fminf(s_low[0], s_low[1]), fminf(s_low[2], s_low[3]));
        }
        s.bound = filtered && tau > 0.0f ? s_bound : 0u;
        s.listed = s_listed;
        stat[row * segs + seg] = s;
    }
}

// ---- what pick and again share ----
template <int CTRL, int ROW_MASK, class X>
__device__ __forceinline__ X dpp64_or_zero(X v)
{
    static_assert(sizeof(X) == 8, "64 bits");
    const ArgPart u = __builtin_bit_cast(ArgPart, v);
    return __builtin_bit_cast(X, (ArgPart)(uint32_t)dpp_or_zero<CTRL, ROW_MASK>((int)(u >> 32)) << 32 |
                                     (uint32_t)dpp_or_zero<CTRL, ROW_MASK>((int)(uint32_t)u));
}
// Inclusive sum over the wave's lanes (see wave_scan_inclusive_i32).
template <class X>
__device__ __forceinline__ X wave_scan64(X v)
{
    v += dpp64_or_zero<0x111, 0xF>(v);
    v += dpp64_or_zero<0x112, 0xF>(v);
    v += dpp64_or_zero<0x114, 0xF>(v);
    v += dpp64_or_zero<0x118, 0xF>(v);
    v += dpp64_or_zero<0x142, 0xA>(v);
    v += dpp64_or_zero<0x143, 0xC>(v);
    return v;
}
// Sum over the threads in front of this one, and over all (both in one fixed order).  waves: one entry a wave.
template <int NT, class X>
__device__ __forceinline__ X block_scan(X v, X *waves, X &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const X s = wave_scan64(v);
    // (the neighbour's: the inclusive sum less the own value, without a subtraction)
    X up = dpp64_or_zero<0x138, 0xF>(s);  // wave_shr:1
    __syncthreads();
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    X before = X(0);
    total = X(0);
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) {
        before = w < wave ? before + waves[w] : before;
        total += waves[w];
    }
    return before + up;
}

// The largest of the values of the lanes where `on`, which rise with the lane: one lane's atomic.  (64 lanes' atomics on one
// address take the wave through a loop of 64 rounds: a search over 8192 elements 25 us, with this 3.)
__device__ __forceinline__ void wave_last(int *out, bool on, int value)
{
    const unsigned long long who = __builtin_amdgcn_ballot_w64(on);
    if (who != 0ull && (int)(threadIdx.x & 63) == 63 - __builtin_clzll(who)) atomicMax(out, value);
}

// A row, and what stays of it as far as that is known.
struct PickRow {
    const float *x;
    int V;
    double M, c;       // largest logit, log2(e) / tau
    ArgPart floor;     // composites below it do not stay
    double unit;       // units of integer weights
    double scale;      // steps of the logit for a log-weight
    // step of an element with log-weight t, in falling order
    __device__ __forceinline__ int step_of(double t) const { return min(kSteps - 1, (int)(t * scale)); }
    __device__ __forceinline__ double log_weight(float v) const { return ((double)v - M) * c; }
    __device__ __forceinline__ double weight(float v) const
    {
        const double t = log_weight(v);
        return t >= kCut ? exp2_of(t) : 0.0;
    }
    __device__ __forceinline__ ArgPart in_units(double w) const { return (ArgPart)(w * unit + 0.5); }
    // f(value, id) for every finite element
    template <int NT, class F>
    __device__ __forceinline__ void each(F &&f) const
    {
        constexpr int kAhead = 8;
        const Run run(x, V);
        for (int g = threadIdx.x; g < run.groups; g += kAhead * NT) {
            float4 p[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) p[u] = run.load(g + u * NT);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                float e[4];
                run.four(g + u * NT, p[u], e);
#pragma unroll 1
                for (int v = 0; v < 4; ++v) {
                    const float y = v == 0 ? e[0] : v == 1 ? e[1] : v == 2 ? e[2] : e[3];
                    if (y > -INFINITY) f(y, run.id(g + u * NT) + v);
                }
            }
        }
        const int edge = run.edge_id();
        const float v = edge >= 0 ? clean(x[edge]) : -INFINITY;
        if (v > -INFINITY) f(v, edge);
    }
    // The composites of the elements from lo to hi (lo > -inf) into a list with room for `room`; their number, also where that is
    // more, through n (0 before).  A wave takes its place in the list once for 2048 elements.
    template <int NT>
    __device__ __forceinline__ void collect(float lo, float hi, ArgPart *list, int room, int *n) const
    {
        collect_of<NT, 8>(Run(x, V), 0, lo, hi, list, room, n);
    }
    // The same of a run of the row, `start` elements into it.
    template <int NT, int kAhead>
    __device__ __forceinline__ void collect_of(const Run &run, int start, float lo, float hi, ArgPart *list, int room, int *n) const
    {
        const int lane = threadIdx.x & 63;
        for (int g0 = (int)threadIdx.x - lane; g0 < run.groups; g0 += kAhead * NT) {  // (uniform over a wave)
            float4 p[kAhead];
            float e[kAhead][4];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) p[u] = run.load(g0 + lane + u * NT);
            int hits = 0;
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                run.four(g0 + lane + u * NT, p[u], e[u]);
#pragma unroll
                for (int v = 0; v < 4; ++v) hits += __popcll(__builtin_amdgcn_ballot_w64(e[u][v] >= lo && e[u][v] <= hi));
            }
            if (hits == 0) continue;
            int at = 0;
            if (lane == 0) at = atomicAdd(n, hits);
            at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const bool hit = e[u][v] >= lo && e[u][v] <= hi;
                    const unsigned long long who = __builtin_amdgcn_ballot_w64(hit);
                    if (who == 0ull) continue;
                    const int mine = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
                    if (hit && mine < room) list[mine] = arg_part(e[u][v], start + run.id(g0 + lane + u * NT) + v);
                    at += __popcll(who);
                }
        }
        const int edge = run.edge_id();
        const float v = edge >= 0 ? clean(run.p[edge]) : -INFINITY;
        if (v >= lo && v <= hi) {
            const int mine = atomicAdd(n, 1);
            if (mine < room) list[mine] = arg_part(v, start + edge);
        }
    }
    // A logit whose log-weight is at least t, and whose neighbours' are not far below: what `each` is to look at
    __device__ __forceinline__ float about(double t, double side) const
    {
        const double v = M + t / c;
        return (float)fmax(-3.4028234e38, fmin(3.4028234e38, v + side * (1e-5 * (fabs(v) + fabs(M)) + 1e-30)));
    }
    // ends of a step, a little outside
    __device__ __forceinline__ float lo_of(int step) const { return about(step == kSteps - 1 ? kCut : (step + 1) / scale, -1.0); }
    __device__ __forceinline__ float hi_of(int step) const { return about(step / scale, 1.0); }
};
__device__ __forceinline__ PickRow pick_row(const float *logits, size_t row, int V, double M, float tau)
{
    PickRow r;
    r.x = logits + row * (size_t)V;
    r.V = V;
    r.M = M;
    r.c = 1.4426950408889634 / (double)tau;
    r.floor = 0ull;
    r.unit = 0.0;
    r.scale = kSteps / kCut;
    return r;
}
// Elements [from, to) of a row, at most 4 G of them, -inf behind them.  (From any place: loads of 16 bytes on 4-byte boundaries, all
// requested before any is looked at; the last ones of the row one by one.)
template <int G>
__device__ __forceinline__ void load_run(const float *x, int V, int from, int to, float (&e)[4 * G])
{
    typedef float four __attribute__((ext_vector_type(4), aligned(4)));
    four f[G];
    if (V >= 4)
#pragma unroll
        for (int g = 0; g < G; ++g) f[g] = *reinterpret_cast<const four *>(x + max(0, min(from + 4 * g, V - 4)));
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int v = 0; v < 4; ++v) e[4 * g + v] = from + 4 * g + v < to ? clean(f[g][v]) : -INFINITY;
    if (to > V - 4 && from < to) {  // (at most a few threads)
#pragma unroll
        for (int k = 0; k < 4 * G; ++k)
            if ((from + (k & ~3) > V - 4) && from + k < to) e[k] = clean(x[from + k]);
    }
}
// u from [0, 1): what is below, or no number, counts as 0, what is above as the largest float below 1
__device__ __forceinline__ float clean_uniform(float u)
{
    const uint32_t b = __float_as_uint(u);
    return b > 0x7F800000u ? 0.0f : b >= 0x3F800000u ? 0x1.fffffep-1f : u;
}
// Units of the integer weights of a row whose sum is at most `most` (at least 1): as fine as sums below 2^63 allow.  (A bound 100 times
// the sum leaves a weight off by 2^-56 of it.  By the number of elements alone it was 2^-45 where one token has most of the weight, and with
// equal others, all rounded alike, borders were off by 1e-9 of the sum.)
__device__ __forceinline__ double unit_of(double most) { return __builtin_amdgcn_ldexp(1.0, 63 - __builtin_amdgcn_frexp_exp(most)); }
__device__ __forceinline__ void put_token(int token, size_t row, ArgPart *part, int32_t *tokens)
{
    if (threadIdx.x != 0) return;
    if (tokens) tokens[row] = token;
    else part[row] = 1ull << 32 | (uint32_t)~token;
}

struct LocateShared {
    double wave_d[kPickThreads / 64];
    int last, token;
};
// The element of [start, start + n) where the running sum, `base` in front of it, exceeds `target` (the last one with a
// weight, should rounding leave none).  c0, c1: the running sum in front of it and behind it.
__device__ int pick_locate(const PickRow &r, int start, int n, double base, double target, LocateShared &sh, double &c0, double &c1)
{
    constexpr int NT = kPickThreads;
    // (a multiple of four elements a thread: as many loads of 16 bytes where the row allows)
    const int per = ((n + NT - 1) / NT + 3) / 4 * 4, from = start + (int)threadIdx.x * per, to = min(from + per, start + n);
    double mine = 0.0, total;
    int last = -1;
    constexpr int G = 6;  // groups of a thread
    static_assert(4 * G * NT >= 6144, "a segment fits");
    float x[4 * G];
    load_run<G>(r.x, r.V, from, to, x);
#pragma unroll
    for (int k = 0; k < 4 * G; ++k) {
        const double w = x[k] > -INFINITY ? r.weight(x[k]) : 0.0;
        if (w > 0.0) last = from + k;
        mine += w;
    }
    if (threadIdx.x == 0) sh.last = -1, sh.token = -1;
    const double before = base + block_scan<NT>(mine, sh.wave_d, total);
    wave_last(&sh.last, last >= 0, last);
    wave_last(&sh.token, last >= 0 && before <= target && target < before + mine, (int)threadIdx.x);
    __syncthreads();
    // (should rounding leave no such thread: the one that holds the last element)
    const int who = sh.token >= 0 ? sh.token : sh.last >= 0 ? (sh.last - start) / per : -1;
    __syncthreads();
    if (who == (int)threadIdx.x) {
        double c = before, w = 0.0;
        int token = last;
        for (int e = from; e < to; ++e) {
            w = r.weight(clean(r.x[e]));
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

struct PickShared {
    union {
        struct {
            uint32_t key[kCandidates], id[kCandidates];
            ArgPart w[kCandidates];
            uint16_t order[kCandidates];
            ArgPart mass[kCandBuckets];
            uint32_t count[kCandBuckets], cursor[kCandBuckets];
        } c;
        double seg[kMaxSegs];
    };
    int32_t listed[kMaxSegs];
    ArgPart wave_u[kPickThreads / 64];
    LocateShared locate;
    int n, last, token;
};

__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(
    const float *__restrict__ logits, int T, int V, int seg_len, int segs, int hot_cap,
    const int32_t *__restrict__ n_nodes, const float *__restrict__ uniforms, const SegStat *__restrict__ stat_all,
    const ArgPart *__restrict__ hot_all, ArgPart *__restrict__ part, int32_t *__restrict__ tokens, uint32_t *__restrict__ n_hard,
    HardRow *__restrict__ hard, SampleOpts opt)
{
    __shared__ PickShared sh;
    const int tid = threadIdx.x, i = blockIdx.x, seq = blockIdx.y;
    if (n_nodes && i > n_nodes[seq]) return;  // padding row
    const size_t row = (size_t)seq * T + i;
    const SegStat *const stat = stat_all + row * segs;
    const ArgPart *const hot = hot_all + row * segs * (size_t)hot_cap;
    const float tau = opt.tau[seq], top_p = opt.top_p[seq], min_p = opt.min_p[seq];
    const int top_k = opt.top_k[seq];
    const bool filtered = top_k > 0 || top_p < 1.0f || min_p > 0.0f;
    const float u = clean_uniform(uniforms[row]);
    // the lists are requested before anything is known of them (what is past a list's end is not looked at)
    constexpr int kAhead = 8;
    const int slots = filtered && tau > 0.0f ? segs * hot_cap / 2 : 0;  // pairs
    ulonglong2 ahead[kAhead];
#pragma unroll
    for (int v = 0; v < kAhead; ++v)
        if (slots > 0) ahead[v] = reinterpret_cast<const ulonglong2 *>(hot)[min(tid + v * kPickThreads, slots - 1)];

    // the row's best, and the largest of the bounds (a list that is not complete: no bound holds)
    ArgPart best = kNoPart;
    uint32_t bound = 0u;
    for (int s = tid; s < segs; s += kPickThreads) {
        const ArgPart b = stat[s].best;
        const int listed = stat[s].listed;
        best = b > best ? b : best;
        bound = max(bound, listed > hot_cap ? ~0u : stat[s].bound);
        sh.listed[s] = listed;
    }
    best = wave_arg_max(best);
    bound = ~wave_min_u32(~bound);
    if ((tid & 63) == 63) sh.wave_u[tid >> 6] = best, sh.locate.wave_d[tid >> 6] = (double)bound;
    __syncthreads();
    best = kNoPart;
#pragma unroll
    for (int w = 0; w < kPickThreads / 64; ++w) {
        best = sh.wave_u[w] > best ? sh.wave_u[w] : best;
        bound = max(bound, (uint32_t)sh.locate.wave_d[w]);
    }
    __syncthreads();
    if (best == kNoPart) return put_token(-1, row, part, tokens);
    if (!(tau > 0.0f)) return put_token(arg_token(best), row, part, tokens);

    const PickRow r = pick_row(logits, row, V, (double)key_float((uint32_t)(best >> 32)), tau);
    const bool has_sum = top_k == 0 && (top_p < 1.0f || !filtered);
    double Z = 0.0;
    auto put_on_list = [&](double sum) {
        if (tid >= 64) return;
        // the sum, or a bound on it from those of the segments: the units go by it
        double most = Z;
        if (!has_sum) {
            most = 0.0;
            for (int s = tid; s < segs; s += 64) {
                const ArgPart b = stat[s].best;
                most += b != kNoPart ? exp2_of(r.log_weight(key_float((uint32_t)(b >> 32)))) * stat[s].sum : 0.0;
            }
            most = wave_sum_f64_lane63(most);
        }
        if (tid != 63) return;
        // Where the sum is known and top-p is the first filter, its border lies above log-weights of which all V elements would
        // not make up half of what it leaves out: the steps go that far only
        double deep = -kCut;
        if (sum > 0.0 && top_p < 1.0f) deep = fmin(deep, fmax(1.0, log2((double)V / ((1.0 - (double)top_p) * sum)) + 2.0));
        hard[atomicAdd(n_hard, 1u)] = HardRow{unit_of(most), r.M, -kSteps / deep, (int32_t)row, -1, 0, 0};
    };

    // The row's sum.  A segment has also counted elements that are too small beside the row's best but not beside its own:
    // `slack` bounds what they add (each is below 2^-40, if there are any).  Where this could change a decision, the row goes
    // on the list.
    double slack = 0.0;
    if (has_sum) {
        const int per = (segs + kPickThreads - 1) / kPickThreads, from = tid * per, to = min(from + per, segs);
        double mine = 0.0;
        bool doubt = false;
        for (int s = from; s < to; ++s) {
            double w = 0.0;
            const ArgPart b = stat[s].best;
            if (b != kNoPart) {
                const double t = r.log_weight(key_float((uint32_t)(b >> 32)));
                if (t >= kCut) {
                    w = exp2_of(t) * stat[s].sum;
                    doubt = doubt || !(r.log_weight(stat[s].low) >= kCut);
                }
            }
            if (!filtered) sh.seg[s] = w;
            mine += w;
        }
        const double before = block_scan<kPickThreads>(mine, sh.locate.wave_d, Z);
        if (__syncthreads_or(doubt ? 1 : 0)) slack = (double)V * 0x1p-40;
        if (!filtered) {
            const double target = (double)u * Z;
            if (tid == 0) sh.n = -1;
            __syncthreads();
            double b = before;
            int last = -1;
            for (int s = from; s < to; ++s) {
                const double w = sh.seg[s];
                if (w > 0.0 && b <= target) last = s;
                sh.seg[s] = b;
                b += w;
            }
            wave_last(&sh.n, last >= 0, last);
            __syncthreads();
            const int s = sh.n;
            const double base = sh.seg[s];
            double c0, c1;
            const int token = pick_locate(r, s * seg_len, min(seg_len, V - s * seg_len), base, target, sh.locate, c0, c1);
            if (slack > 0.0 && !(c0 <= (double)u * (Z - slack) && target < c1 - slack)) return put_on_list(0.0);
            return put_token(token, row, part, tokens);
        }
    }

    // ---- the listed elements that reach the bound ----
    auto &c = sh.c;
    const uint32_t at_least = max(bound, kKeyOfNone + 1u);
    if (tid == 0) sh.n = 0;
    for (int b = tid; b < kCandBuckets; b += kPickThreads) c.mass[b] = 0ull, c.count[b] = 0u;
    __syncthreads();
    if (bound != ~0u) {
        auto look = [&](int pair, const ulonglong2 &h, bool &x, bool &y) {
            const int s = 2 * pair / hot_cap, left = sh.listed[s] - (2 * pair - s * hot_cap);
            x = left > 0 && (uint32_t)(h.x >> 32) >= at_least;
            y = left > 1 && (uint32_t)(h.y >> 32) >= at_least;
        };
        // (a wave takes its places at once)
        const int lane = tid & 63;
        auto place = [&](int at, unsigned long long who, bool on, ArgPart h) {
            const int mine = at + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(who >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)who, 0u));
            if (on && mine < kCandidates) c.key[mine] = (uint32_t)(h >> 32), c.id[mine] = (uint32_t)arg_token(h);
        };
        for (int k0 = 0; k0 < slots; k0 += kAhead * kPickThreads) {
            if (k0 > 0) {
#pragma unroll
                for (int v = 0; v < kAhead; ++v)
                    ahead[v] = reinterpret_cast<const ulonglong2 *>(hot)[min(k0 + tid + v * kPickThreads, slots - 1)];
            }
            bool x[kAhead], y[kAhead];
            int hits = 0;
#pragma unroll
            for (int v = 0; v < kAhead; ++v) {
                const int pair = k0 + tid + v * kPickThreads;
                look(min(pair, slots - 1), ahead[v], x[v], y[v]);
                x[v] = x[v] && pair < slots, y[v] = y[v] && pair < slots;
                hits += __popcll(__builtin_amdgcn_ballot_w64(x[v])) + __popcll(__builtin_amdgcn_ballot_w64(y[v]));
            }
            int at = 0;
            if (lane == 0 && hits > 0) at = atomicAdd(&sh.n, hits);
            at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
            for (int v = 0; v < kAhead; ++v) {
                const unsigned long long wx = __builtin_amdgcn_ballot_w64(x[v]), wy = __builtin_amdgcn_ballot_w64(y[v]);
                if (wx != 0ull) place(at, wx, x[v], ahead[v].x);
                at += __popcll(wx);
                if (wy != 0ull) place(at, wy, y[v], ahead[v].y);
                at += __popcll(wy);
            }
        }
    }
    __syncthreads();
    const int n = sh.n;
    if (bound == ~0u || n > kCandidates) return put_on_list(slack > 0.0 ? 0.0 : Z);
    // (below the bound nothing has a weight: the list is all there is)
    const double t_bound = bound == 0u ? -1e30 : r.log_weight(key_float(bound));
    const bool all = bound == 0u || t_bound < kCut;
    // buckets in falling order: equal steps between the best and the least listed (for elements without a weight, the last)
    const double span = fmax(all ? kCut : t_bound, kCut);
    const double step = span < 0.0 ? (double)(kCandBuckets - 1) / span : 0.0;
    auto bucket_of = [&](double t) { return min(kCandBuckets - 1, max(0, (int)(fmax(t, 2.0 * kCut) * step))); };
    constexpr int kEach = kCandidates / kPickThreads;
    uint16_t bucket[kEach];
    bool counts[kEach];  // has a weight, and not below min-p
#pragma unroll
    for (int v = 0; v < kEach; ++v) {
        const int k = tid + v * kPickThreads;
        bucket[v] = 0, counts[v] = false;
        if (k >= n) continue;
        const double t = r.log_weight(key_float(c.key[k])), weight = exp2_of(t);
        const ArgPart w = t >= kCut ? (ArgPart)(weight * 0x1p52 + 0.5) : 0ull;
        counts[v] = t >= kCut && weight >= (double)min_p;
        c.w[k] = w;
        bucket[v] = (uint16_t)bucket_of(t);
        atomicAdd(&c.mass[bucket[v]], w);
        atomicAdd(&c.count[bucket[v]], 1u);
    }
    __syncthreads();
    constexpr int kPer = kCandBuckets / kPickThreads;
    ArgPart m[kPer], q[kPer], m_mine = 0ull, q_mine = 0ull, m_all, q_all;
#pragma unroll
    for (int v = 0; v < kPer; ++v) {
        m[v] = c.mass[tid * kPer + v], q[v] = c.count[tid * kPer + v];
        m_mine += m[v], q_mine += q[v];
    }
    ArgPart m_front = block_scan<kPickThreads>(m_mine, sh.wave_u, m_all), q_front = block_scan<kPickThreads>(q_mine, sh.wave_u, q_all);
#pragma unroll
    for (int v = 0; v < kPer; ++v) {
        c.mass[tid * kPer + v] = m_front, c.cursor[tid * kPer + v] = (uint32_t)q_front;
        m_front += m[v], q_front += q[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kEach; ++v)
        if (tid + v * kPickThreads < n) c.order[atomicAdd(&c.cursor[bucket[v]], 1u)] = (uint16_t)(tid + v * kPickThreads);
    __syncthreads();
    // rank and weight in front of each; where its bucket lies behind the end of top-k or top-p, or the element has no weight, it
    // does not matter which (a row's list is mostly made of those: 50 of 1200 stay at top-k 50)
    const double p_ends = top_k == 0 && top_p < 1.0f ? (double)top_p * Z * 0x1p52 : 0x1p64;
    int rank[kEach];
    ArgPart front[kEach], kept = 0ull, sum;
#pragma unroll
    for (int v = 0; v < kEach; ++v) {
        const int k = tid + v * kPickThreads;
        rank[v] = 0, front[v] = 0ull;
        if (k >= n) continue;
        const int b = bucket[v], end = (int)c.cursor[b], begin = end - (int)c.count[b];
        const uint32_t key = c.key[k], id = c.id[k];
        ArgPart f = c.mass[b];
        int before = begin;
        if ((top_k == 0 || begin < top_k) && (double)f < p_ends && (counts[v] || (top_k > 0 && top_p < 1.0f)))
        for (int o = begin; o < end; ++o) {
            const int j = c.order[o];
            const bool larger = c.key[j] > key || (c.key[j] == key && c.id[j] < id);
            f += larger ? c.w[j] : 0ull;
            before += larger ? 1 : 0;
        }
        rank[v] = before, front[v] = f;
        if (before < top_k) kept += c.w[k];  // (weights below min-p among them)
    }
    // what top-k keeps: its weight is what top-p goes by
    if (top_k > 0) {
        (void)block_scan<kPickThreads>(kept, sh.wave_u, sum);
        Z = (double)sum * 0x1p-52;
    }
    const double limit = (double)top_p * Z * 0x1p52, uncertain = slack * 0x1p52;
    // Everything that stays is listed if top-k, top-p or min-p ends above the bound, or nothing below it has a weight.
    // (The limit of top-p behind a top-k that the list does not hold is not known.)
    const bool k_ends = all || (top_k > 0 && n >= top_k);
    const bool ends = k_ends || ((top_k == 0 || top_p >= 1.0f) && ((top_p < 1.0f && (double)m_all >= limit) ||
                                                                  (min_p > 0.0f && exp2_of(t_bound) < (double)min_p)));
    bool unsure = !ends;
    ArgPart stays[kEach], S;
    kept = 0ull;
#pragma unroll
    for (int v = 0; v < kEach; ++v) {
        const int k = tid + v * kPickThreads;
        stays[v] = 0ull;
        if (k >= n) continue;
        const double f = (double)front[v];
        unsure = unsure || (top_p < 1.0f && slack > 0.0 && f > limit - uncertain && f < limit);
        if ((top_k == 0 || rank[v] < top_k) && (top_p >= 1.0f || f < limit) && counts[v]) stays[v] = c.w[k];
        kept += stays[v];
    }
    if (__syncthreads_or(unsure ? 1 : 0)) return put_on_list(has_sum && slack == 0.0 ? Z : 0.0);
    // in the order of ids: buckets of ids, then the elements of the bucket where the running sum passes u S
    const int id_shift = max(0, 32 - __builtin_clz((unsigned)max(V - 1, 1)) - 10);
    for (int b = tid; b < kCandBuckets; b += kPickThreads) c.mass[b] = 0ull;
    if (tid == 0) sh.n = -1, sh.token = -1, sh.last = 0;
    (void)block_scan<kPickThreads>(kept, sh.wave_u, S);  // (with barriers inside)
    const double target = (double)u * (double)S;
#pragma unroll
    for (int v = 0; v < kEach; ++v)
        if (stays[v] != 0ull) atomicAdd(&c.mass[c.id[tid + v * kPickThreads] >> id_shift], stays[v]);
    __syncthreads();
    m_mine = 0ull;
#pragma unroll
    for (int v = 0; v < kPer; ++v) m[v] = c.mass[tid * kPer + v], m_mine += m[v];
    m_front = block_scan<kPickThreads>(m_mine, sh.wave_u, m_all);
    int last = -1;
#pragma unroll
    for (int v = 0; v < kPer; ++v) {
        c.mass[tid * kPer + v] = m_front;
        if (m[v] > 0ull && (double)m_front <= target) last = tid * kPer + v;
        m_front += m[v];
    }
    wave_last(&sh.n, last >= 0, last);
    __syncthreads();
    const int at = sh.n;
    // (the bucket's elements: at most all)
#pragma unroll
    for (int v = 0; v < kEach; ++v) {
        const int k = tid + v * kPickThreads;
        if (stays[v] != 0ull && (int)(c.id[k] >> id_shift) == at) c.order[atomicAdd(&sh.last, 1)] = (uint16_t)k;
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
    put_token(sh.token, row, part, tokens);
}

// ---- rows on the list ----
struct AgainShared {
    union {
        struct {
            ArgPart mass[kHistBuckets];
            uint32_t count[kHistBuckets];
            ArgPart list[kCandidates];
        } h;
        struct {
            ArgPart mass[kSteps], count[kSteps];  // in front of a step
            ArgPart sub[kSteps], list[kStepList], few[kStepList];
            ArgPart part[kSampleMaxV / kPart];
        } s;
        ArgPart chunk[kMaxChunks];
    };
    ArgPart wave_u[kAgainThreads / 64];
    ArgPart found, base;
    int n, token;
};

// n composites in falling order, padded with zeros to a power of two (the list's size is one).  A sorting
// network: 66 steps of 60 cycles for 2048.  (Each compared with all others: 110 us for 1300.)
__device__ void sort_falling(ArgPart *list, int n)
{
    constexpr int NT = kAgainThreads;
    int size = 2;
    while (size < n) size *= 2;
    for (int k = n + (int)threadIdx.x; k < size; k += NT) list[k] = 0ull;
    __syncthreads();
    for (int run = 2; run <= size; run *= 2)
        for (int d = run / 2; d >= 1; d /= 2) {
            for (int k = threadIdx.x; k < size / 2; k += NT) {
                const int i = 2 * k - (k & (d - 1)), j = i + d;  // (bit d of i is clear)
                const ArgPart a = list[i], b = list[j];
                if ((a < b) == ((i & run) == 0)) list[i] = b, list[j] = a;
            }
            __syncthreads();
        }
}
// Of n composites (sorted here) the last one, in falling order, with less than `bound` in front of it, `front` included; value(k):
// what the k-th of the order adds.  ~0 if there is none.
template <int N, class F>
__device__ ArgPart last_in_order(ArgPart *list, int n, ArgPart front, double bound, F &&value, ArgPart *waves, ArgPart &found)
{
    constexpr int NT = kAgainThreads, kEach = N / NT;  // n <= N
    sort_falling(list, n);
    ArgPart v[kEach], mine = 0ull, all, last = 0ull;
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int k = (int)threadIdx.x * kEach + e;
        v[e] = k < n && list[k] != 0ull ? value(list[k]) : 0ull;
        mine += v[e];
    }
    if (threadIdx.x == 0) found = ~0ull;
    ArgPart before = front + block_scan<NT>(mine, waves, all);  // (with barriers inside)
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int k = (int)threadIdx.x * kEach + e;
        if (k < n && list[k] != 0ull && (double)before < bound) last = list[k];
        before += v[e];
    }
    // (falling order: the least of the threads' last ones; a wave's is that of its last lane that has any)
    const unsigned long long who = __builtin_amdgcn_ballot_w64(last != 0ull);
    if (who != 0ull && (int)(threadIdx.x & 63) == 63 - __builtin_clzll(who)) atomicMin(&found, last);
    __syncthreads();
    const ArgPart r = found;
    __syncthreads();
    return r;
}

// The composite of the last element, in falling order, with less than `bound` in front of it: elements counted, or (MASS) their weights
// in units summed and `bound` a share of the sum of all.  Elements below r.floor do not take part; r.floor if all stay.  However many
// elements lie together: equal logits are told apart by their ids.
template <bool MASS>
__device__ ArgPart pick_threshold(const PickRow &r, double bound, AgainShared &sh)
{
    constexpr int NT = kAgainThreads;
    auto value = [&](double w) -> ArgPart { return MASS ? r.in_units(w) : 1ull; };
    auto bucket_of = [&](double t) { return min(kHistBuckets - 1, (int)(t * (kHistBuckets / kCut))); };
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
        for (int b = threadIdx.x; b < kHistBuckets; b += NT) sh.h.mass[b] = 0ull, sh.h.count[b] = 0u;
        __syncthreads();
        r.each<NT>([&](float v, int id) {
            const double t = r.log_weight(v);
            if (!left(v, id, t)) return;
            const int b = bucket < 0 ? bucket_of(t) : kHistBuckets - 1 - (int)((arg_part(v, id) >> next) & ((1ull << width) - 1ull));
            atomicAdd(&sh.h.count[b], 1u);
            if (MASS) atomicAdd(&sh.h.mass[b], value(exp2_of(t)));
        });
        __syncthreads();
        constexpr int kPer = kHistBuckets / NT;
        ArgPart v[kPer], mine = 0ull, total;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            const int b = (int)threadIdx.x * kPer + u;
            v[u] = MASS ? sh.h.mass[b] : (ArgPart)sh.h.count[b];
            mine += v[u];
        }
        ArgPart before = base + block_scan<NT>(mine, sh.wave_u, total);
        if (MASS && bucket < 0) bound *= (double)total;
        if (bucket < 0 && (double)total < bound) return r.floor;  // all of them stay
        if (threadIdx.x == 0) sh.n = -1;
        __syncthreads();
        // the last bucket that holds elements and has less than the bound in front of it
        const ArgPart first = before;
        int last = -1;
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
            if (sh.h.count[(int)threadIdx.x * kPer + u] > 0u && (double)before < bound) last = (int)threadIdx.x * kPer + u;
            before += v[u];
        }
        wave_last(&sh.n, last >= 0, last);
        __syncthreads();
        const int at = sh.n;
        if (at < 0) return r.floor;
        before = first;
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
            if (threadIdx.x == 0) sh.n = 0;
            __syncthreads();
            r.each<NT>([&](float v, int id) {
                if (!left(v, id, r.log_weight(v))) return;
                const int k = atomicAdd(&sh.n, 1);
                if (k < kCandidates) sh.h.list[k] = arg_part(v, id);
            });
            __syncthreads();
            const int n = min(sh.n, kCandidates);
            __syncthreads();
            const ArgPart found = last_in_order<kCandidates>(sh.h.list, n, base, bound, [&](ArgPart c) {
                return MASS ? value(exp2_of(r.log_weight(key_float((uint32_t)(c >> 32))))) : 1ull; }, sh.wave_u, sh.found);
            return found == ~0ull ? r.floor : found;
        }
    }
}

__device__ __forceinline__ int step_of_min_p(const PickRow &r, float min_p)
{
    return min_p > 0.0f ? r.step_of(fmax(log2((double)min_p), kCut)) : kSteps;
}
// The last element of [start, end) that stays with at most `target` in front of it (`base` in front of `start`); PER a thread.
template <int PER, class F>
__device__ __forceinline__ int last_to_target(const PickRow &r, int start, int end, ArgPart base, double target, F &&stays, AgainShared &sh)
{
    constexpr int NT = kAgainThreads;
    const int id0 = start + (int)threadIdx.x * PER;
    ArgPart w[PER], mine = 0ull, total;
    float x[PER];
    load_run<PER / 4>(r.x, r.V, id0, min(id0 + PER, end), x);
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        w[e] = x[e] > -INFINITY ? stays(x[e], id0 + e) : 0ull;
        mine += w[e];
    }
    ArgPart before = base + block_scan<NT>(mine, sh.wave_u, total);
    if (threadIdx.x == 0) sh.token = -1;
    __syncthreads();
    int last = -1;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        if (w[e] > 0ull && (double)before <= target) last = id0 + e;
        before += w[e];
    }
    wave_last(&sh.token, last >= 0, last);
    __syncthreads();
    return sh.token;
}

// A row by one workgroup: thresholds, sums of chunks, token.  For rows whose border lies in a step with thousands of elements, and those past
// `slots`.  The same integers are summed and compared as by the way with steps, so that a row's token does not depend on which of the
// two it is given.  (With fp64 sums here 344 of 600 equal rows drew another token than the other 256, their uniform on a border.)
__device__ __attribute__((noinline)) int pick_alone(PickRow r, int top_k, float top_p, float min_p, float u, AgainShared &sh)
{
    constexpr int NT = kAgainThreads;
    ArgPart total;
    r.floor = 0ull;
    __syncthreads();
    if (top_k > 0) r.floor = pick_threshold<false>(r, (double)top_k, sh);
    if (top_p < 1.0f) r.floor = pick_threshold<true>(r, (double)top_p, sh);
    // (from the step where min-p ends on weights are looked at, behind it none stays; the last one has no end)
    const int min_step = step_of_min_p(r, min_p);
    const double from_step = min_step < kSteps ? min_step : 1e30, past_step = min_step < kSteps - 1 ? min_step + 1 : 1e30;
    auto stays = [&](float v, int id) -> ArgPart {
        const double t = r.log_weight(v), step = t * r.scale;
        if (!(t >= kCut) || step >= past_step || arg_part(v, id) < r.floor) return 0ull;
        const double weight = exp2_of(t);
        return step >= from_step && weight < (double)min_p ? 0ull : r.in_units(weight);
    };
    const int chunks = (r.V + kChunk - 1) / kChunk, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int k = wave; k < chunks; k += NT / 64) {
        const int start = k * kChunk, from = start + lane * (kChunk / 64);
        ArgPart sum = 0ull;
        float x[kChunk / 64];
        load_run<kChunk / 256>(r.x, r.V, from, min(from + kChunk / 64, r.V), x);
#pragma unroll
        for (int e = 0; e < kChunk / 64; ++e) sum += x[e] > -INFINITY ? stays(x[e], from + e) : 0ull;
        sum = wave_scan64(sum);
        if (lane == 63) sh.chunk[k] = sum;
    }
    __syncthreads();
    const int per = (chunks + NT - 1) / NT, from = (int)threadIdx.x * per, to = min(from + per, chunks);
    ArgPart mine = 0ull;
    for (int k = from; k < to; ++k) mine += sh.chunk[k];
    ArgPart before = block_scan<NT>(mine, sh.wave_u, total);
    const double target = (double)u * (double)total;
    if (threadIdx.x == 0) sh.n = -1;
    __syncthreads();
    // the last chunk with a weight that has at most the target in front of it
    int last = -1;
    for (int k = from; k < to; ++k) {
        const ArgPart w = sh.chunk[k];
        if (w > 0ull && (double)before <= target) last = k;
        sh.chunk[k] = before;  // from now on: the sum in front of it
        before += w;
    }
    wave_last(&sh.n, last >= 0, last);
    __syncthreads();
    const int k = sh.n;
    if (k < 0) return -1;
    return last_to_target<4>(r, k * kChunk, min((k + 1) * kChunk, r.V), sh.chunk[k], target, stays, sh);
}

// Weight and count of the thread's step over a row, from its parts' sums (threads past the steps: nothing).
__device__ __forceinline__ void step_totals(const StepSum *steps, int parts, ArgPart &mass, ArgPart &count)
{
    mass = count = 0ull;
    if (threadIdx.x >= kSteps) return;
    for (int p = 0; p < parts; p += 8) {
        StepSum q[16];
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            const StepSum *const at = steps + (size_t)min(p + v, parts - 1) * (kSteps + 1) + threadIdx.x;
            q[2 * v] = at[0], q[2 * v + 1] = at[1];
        }
#pragma unroll
        for (int v = 0; v < 8; ++v) {
            mass += p + v < parts ? q[2 * v + 1].mass - q[2 * v].mass : 0ull;
            count += p + v < parts ? q[2 * v + 1].count - q[2 * v].count : 0ull;
        }
    }
}

// The border from the steps' sums, then the token.  `few`: the elements of step `ready`, gathered by others.  False: too many elements
// in the border's step.
__device__ bool pick_by_steps(const PickRow &r, const StepSum *steps, int parts, int top_k, float top_p, float min_p,
                              float u, int ready, int listed, const ArgPart *few, AgainShared &sh, int &token)
{
    constexpr int NT = kAgainThreads;
    static_assert(NT >= kSteps, "a thread a step");
    auto &s = sh.s;
    const int tid = threadIdx.x;
    // weight and count of each step over the row, then in front of it
    ArgPart mass, count, mass_all, count_all;
    step_totals(steps, parts, mass, count);
    const ArgPart mass_front = block_scan<NT>(mass, sh.wave_u, mass_all), count_front = block_scan<NT>(count, sh.wave_u, count_all);
    if (tid < kSteps) s.mass[tid] = mass_front, s.count[tid] = count_front;
    // Elements of steps in front of `border` stay, those behind it do not; of it those from `floor` on with a weight of min_p.
    int border = kSteps, n = 0;
    ArgPart floor = 0ull;
    auto last_below = [&](ArgPart front, bool holds, double limit) {  // the last step that holds elements with less than the limit in front
        if (tid == 0) sh.n = -1;
        __syncthreads();
        wave_last(&sh.n, tid < kSteps && holds && (double)front < limit, tid);
        __syncthreads();
        const int at = sh.n;
        __syncthreads();
        return at;
    };
    auto gather = [&](int step) {  // the step's elements that take part, into s.list, anything else there as 0; false: too many
        if (step == ready) {
            n = listed;
            if (n > kStepList) return false;
            for (int k = tid; k < n; k += NT) s.list[k] = few[k];
            __syncthreads();
        } else {
            if (tid == 0) sh.n = 0;
            __syncthreads();
            r.collect<NT>(r.lo_of(step), r.hi_of(step), s.list, kStepList, &sh.n);
            __syncthreads();
            n = sh.n;
            __syncthreads();
            if (n > kStepList) return false;
        }
        for (int k = tid; k < n; k += NT) {
            const double t = r.log_weight(key_float((uint32_t)(s.list[k] >> 32)));
            if (!(t >= kCut) || r.step_of(t) != step || s.list[k] < floor) s.list[k] = 0ull;
        }
        __syncthreads();
        return true;
    };
    auto weight_of = [&](ArgPart c) { return r.in_units(exp2_of(r.log_weight(key_float((uint32_t)(c >> 32))))); };
    // Of the gathered step the composite of the last element with less than `limit` in front of it: once more by steps, 256 of
    // the step, and the elements of one of those against one another.
    auto sub_step = [&](ArgPart c) {
        const double t = r.log_weight(key_float((uint32_t)(c >> 32))) * r.scale;
        return max(0, min(kSteps - 1, (int)((t - (double)border) * kSteps)));
    };
    auto last_in_step = [&](bool by_mass, ArgPart front, double limit) {
        if (tid < kSteps) s.sub[tid] = 0ull;
        if (tid == 0) sh.n = 0, sh.found = ~0ull;
        __syncthreads();
        for (int k = tid; k < n; k += NT)
            if (s.list[k] != 0ull) atomicAdd(&s.sub[sub_step(s.list[k])], by_mass ? weight_of(s.list[k]) : 1ull);
        __syncthreads();
        ArgPart all;
        const ArgPart own = tid < kSteps ? s.sub[tid] : 0ull, before = front + block_scan<NT>(own, sh.wave_u, all);
        const int at = last_below(before, own > 0ull, limit);
        if (tid == at) sh.base = before;
        if (tid == 0) sh.n = 0;
        __syncthreads();
        for (int k = tid; k < n; k += NT)
            if (s.list[k] != 0ull && sub_step(s.list[k]) == at) s.few[atomicAdd(&sh.n, 1)] = s.list[k];
        __syncthreads();
        const int m = sh.n;
        const ArgPart base = sh.base;
        for (int k = tid; k < m; k += NT) {
            ArgPart f = base;
            for (int o = 0; o < m; ++o) f += s.few[o] > s.few[k] ? (by_mass ? weight_of(s.few[o]) : 1ull) : 0ull;
            if ((double)f < limit) atomicMin(&sh.found, s.few[k]);
        }
        __syncthreads();
        const ArgPart found = sh.found;
        __syncthreads();
        return found;
    };
    // weight of the gathered elements from the floor on
    auto weight_from_floor = [&]() {
        ArgPart mine = 0ull, all;
        for (int k = tid; k < n; k += NT) mine += s.list[k] != 0ull && s.list[k] >= floor ? weight_of(s.list[k]) : 0ull;
        (void)block_scan<NT>(mine, sh.wave_u, all);
        return all;
    };
    // The step where min-p ends is known ahead; what ends behind it needs no closer look.
    const int min_step = step_of_min_p(r, min_p);
    ArgPart kept = mass_all;  // weight of what top-k keeps
    if (top_k > 0 && count_all > (ArgPart)top_k) {
        const int at = last_below(count_front, count > 0ull, (double)top_k);
        if (at <= min_step || top_p < 1.0f) {
            border = at;
            if (!gather(border)) return false;
            floor = last_in_step(false, s.count[border], (double)top_k);
            if (floor == ~0ull) return false;
            kept = s.mass[border] + weight_from_floor();
        }
    }
    if (top_p < 1.0f) {
        const double limit = (double)top_p * (double)kept;
        const int at = last_below(mass_front, mass > 0ull, limit);
        if (at <= border && at <= min_step) {
            if (at < border) {
                border = at;
                floor = 0ull;
                if (!gather(border)) return false;
            }
            const ArgPart found = last_in_step(true, s.mass[border], limit);
            if (found != ~0ull && found > floor) floor = found;
        }
    }
    if (min_step < border) {
        border = min_step;
        floor = 0ull;
        if (!gather(border)) return false;
    }
    auto stays = [&](float v, int id) -> ArgPart {
        const double t = r.log_weight(v);
        if (!(t >= kCut)) return 0ull;
        const int step = r.step_of(t);
        if (step > border || (step == border && arg_part(v, id) < floor)) return 0ull;
        const double weight = exp2_of(t);
        return step == min_step && weight < (double)min_p ? 0ull : r.in_units(weight);
    };
    // ---- weights of the parts: steps in front of the border, and the border's elements ----
    for (int p = tid; p < parts; p += NT) s.part[p] = steps[(size_t)p * (kSteps + 1) + border].mass;
    __syncthreads();
    if (border < kSteps)
        for (int k = tid; k < n; k += NT) {
            if (s.list[k] == 0ull) continue;
            const int id = arg_token(s.list[k]);
            const ArgPart w = stays(key_float((uint32_t)(s.list[k] >> 32)), id);
            if (w != 0ull) atomicAdd(&s.part[id / kPart], w);
        }
    __syncthreads();
    const int per = (parts + NT - 1) / NT, from = tid * per, to = min(from + per, parts);
    ArgPart mine = 0ull, S;
    for (int p = from; p < to; ++p) mine += s.part[p];
    ArgPart before = block_scan<NT>(mine, sh.wave_u, S);
    const double target = (double)u * (double)S;
    if (tid == 0) sh.n = -1;
    __syncthreads();
    // the last part with a weight that has at most the target in front of it, then the last such element
    int last = -1;
    for (int p = from; p < to; ++p) {
        const ArgPart w = s.part[p];
        if (w > 0ull && (double)before <= target) last = p;
        s.part[p] = before;
        before += w;
    }
    wave_last(&sh.n, last >= 0, last);
    __syncthreads();
    const int p = sh.n;
    if (p < 0) return false;
    token = last_to_target<kPart / NT>(r, p * kPart, min((p + 1) * kPart, r.V), s.part[p], target, stays, sh);
    return true;
}

// The rows on the list, kPart elements at a time: what lies in front of each step.
__global__ __launch_bounds__(kStepThreads) void sample_steps_kernel(
    const float *__restrict__ logits, int T, int V, int parts, int slots, const uint32_t *__restrict__ n_hard,
    const HardRow *__restrict__ hard, StepSum *__restrict__ steps, SampleOpts opt)
{
    constexpr int NT = kStepThreads;
    __shared__ ArgPart s_mass[kSteps], s_waves[NT / 64];
    __shared__ uint32_t s_count[kSteps];
    const int tid = threadIdx.x;
    const int items = min((int)*n_hard, slots) * parts;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int h = item / parts, p = item - h * parts;
        const HardRow row = hard[h];
        const int seq = row.row / T;
        const bool by_count = opt.top_k[seq] > 0;
        PickRow r = pick_row(logits, (size_t)row.row, V, row.best, opt.tau[seq]);
        r.unit = row.unit, r.scale = row.scale;
        const int start = p * kPart;
        const Run run(r.x + start, min(kPart, V - start));
        constexpr int G = kPart / (4 * NT);
        float4 x[G];
        if (run.groups > 0)
#pragma unroll
            for (int g = 0; g < G; ++g) x[g] = run.load(g * NT + tid);
        const int edge = run.edge_id();
        const float at_edge = edge >= 0 ? clean(run.p[edge]) : -INFINITY;
        __syncthreads();  // (the shared memory of the item before)
        if (tid < kSteps) s_mass[tid] = 0ull, s_count[tid] = 0u;
        __syncthreads();
        auto add = [&](float v) {
            const double t = v > -INFINITY ? r.log_weight(v) : 2.0 * kCut;
            if (!(t >= kCut)) return;
            const int step = r.step_of(t);
            atomicAdd(&s_mass[step], r.in_units(exp2_of(t)));
            if (by_count) atomicAdd(&s_count[step], 1u);
        };
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float e[4];
            run.four(g * NT + tid, x[g], e);
#pragma unroll
            for (int v = 0; v < 4; ++v) add(e[v]);
        }
        if (tid < 64) add(at_edge);
        __syncthreads();
        ArgPart mass_all, count_all;
        const ArgPart mass = block_scan<NT>(tid < kSteps ? s_mass[tid] : 0ull, s_waves, mass_all);
        const ArgPart count = block_scan<NT>(tid < kSteps ? (ArgPart)s_count[tid] : 0ull, s_waves, count_all);
        StepSum *const out = steps + ((size_t)h * parts + p) * (kSteps + 1);
        if (tid <= kSteps) out[tid] = tid < kSteps ? StepSum{mass, count} : StepSum{mass_all, count_all};
    }
}

// The elements of the step where a row's border lies, by the workgroups that took its parts: one alone reads a row of 151936 at
// what its outstanding loads allow, 26 us.  (Top-p behind a top-k: its border is known only when the first one is, and left.)
__global__ __launch_bounds__(kStepThreads) void sample_gather_kernel(
    const float *__restrict__ logits, int T, int V, int parts, int slots, const uint32_t *__restrict__ n_hard,
    HardRow *hard, const StepSum *__restrict__ steps, ArgPart *__restrict__ few, SampleOpts opt)
{
    constexpr int NT = kStepThreads;
    __shared__ ArgPart s_waves[NT / 64], s_list[kStepList];
    __shared__ int s_border[2], s_n, s_at;
    const int tid = threadIdx.x;
    const int items = min((int)*n_hard, slots) * parts;
    for (int item = blockIdx.x; item < items; item += gridDim.x) {
        const int h = item / parts, p = item - h * parts;
        const int row = hard[h].row, seq = row / T, top_k = opt.top_k[seq];
        const float top_p = opt.top_p[seq], min_p = opt.min_p[seq];
        if (top_k > 0 && top_p < 1.0f) continue;
        PickRow r = pick_row(logits, (size_t)row, V, hard[h].best, opt.tau[seq]);
        r.scale = hard[h].scale;
        ArgPart mass, count, mass_all, count_all;
        step_totals(steps + (size_t)h * parts * (kSteps + 1), parts, mass, count);
        __syncthreads();  // (the shared memory of the item before)
        if (tid == 0) s_border[0] = s_border[1] = -1, s_n = 0;
        const ArgPart mass_front = block_scan<NT>(mass, s_waves, mass_all), count_front = block_scan<NT>(count, s_waves, count_all);
        wave_last(&s_border[0], tid < kSteps && count > 0ull && count_front < (ArgPart)top_k, tid);
        wave_last(&s_border[1], tid < kSteps && mass > 0ull && (double)mass_front < (double)top_p * (double)mass_all, tid);
        __syncthreads();
        int border = step_of_min_p(r, min_p);
        if (top_k > 0 && count_all > (ArgPart)top_k) border = min(border, s_border[0]);
        if (top_p < 1.0f) border = min(border, s_border[1]);
        if (border < 0 || border >= kSteps) continue;
        const int start = p * kPart;
        r.collect_of<NT, kPart / (4 * NT)>(Run(r.x + start, min(kPart, V - start)), start, r.lo_of(border), r.hi_of(border), s_list, kStepList, &s_n);
        __syncthreads();
        if (tid == 0) {
            s_at = atomicAdd(&hard[h].listed, s_n);
            if (p == 0) hard[h].border = border;
        }
        __syncthreads();
        const int at = s_at, n = min(s_n, kStepList - at);
        for (int k = tid; k < n; k += NT) few[(size_t)h * kStepList + at + k] = s_list[k];
    }
}

// Then a workgroup a row.  Rows past `slots` (the room for the steps' sums) and those with thousands of elements in one
// step are read as often as it takes.
__global__ __launch_bounds__(kAgainThreads) void sample_again_kernel(
    const float *__restrict__ logits, int T, int V, int parts, int slots, const float *__restrict__ uniforms, const uint32_t *__restrict__ n_hard,
    const HardRow *__restrict__ hard, const StepSum *__restrict__ steps, const ArgPart *__restrict__ few,
    ArgPart *__restrict__ part, int32_t *__restrict__ tokens, SampleOpts opt)
{
    __shared__ AgainShared sh;
    const int n = (int)*n_hard;
    for (int h = blockIdx.x; h < n; h += gridDim.x) {
        const HardRow row = hard[h];
        const int seq = row.row / T, top_k = opt.top_k[seq];
        const float top_p = opt.top_p[seq], min_p = opt.min_p[seq], u = clean_uniform(uniforms[row.row]);
        PickRow r = pick_row(logits, (size_t)row.row, V, row.best, opt.tau[seq]);
        r.unit = row.unit, r.scale = row.scale;
        int token = -1;
        __syncthreads();  // (the shared memory of the row before)
        if (h >= slots ||
            !pick_by_steps(r, steps + (size_t)h * parts * (kSteps + 1), parts, top_k, top_p, min_p, u, row.border,
                           row.listed, few + (size_t)h * kStepList, sh, token))
            token = pick_alone(r, top_k, top_p, min_p, u, sh);
        put_token(token, (size_t)row.row, part, tokens);
    }
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
                if (p.seg_len > p.vecs * kScanThreads * 4 || (p.vecs != 2 && p.vecs != 6)) return 10032;
                if (p.hot_cap < p.hot || p.hot > kScanThreads) return 10033;
                const size_t per = (size_t)batch * T * p.segs;
                if (p.hot_off < per * sizeof(SegStat) || p.part_off < p.hot_off + per * p.hot_cap * 8 || p.hard_off < p.part_off + (size_t)batch * T * 8 ||
                    p.step_off < p.hard_off + 256 + (size_t)batch * T * sizeof(HardRow) ||
                    p.few_off < p.step_off + (size_t)p.slots * p.parts * (kSteps + 1) * sizeof(StepSum) ||
                    p.bytes < p.few_off + (size_t)p.slots * kStepList * 8 || (p.few_off & 255u) ||
                    (long long)p.parts * kPart < V || ((p.hot_off | p.part_off | p.hard_off | p.step_off) & 255u))
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
        o.top_k[s] = top_k ? std::min(top_k[s], (int32_t)ddt::kSampleMaxV) : 0;  // (no row is longer; the kernels multiply it)
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
    uint32_t *const n_hard = reinterpret_cast<uint32_t *>(ws + p.hard_off);
    HardRow *const hard = reinterpret_cast<HardRow *>(ws + p.hard_off + 256);
    StepSum *const steps = reinterpret_cast<StepSum *>(ws + p.step_off);
    ArgPart *const few = reinterpret_cast<ArgPart *>(ws + p.few_off);
    auto *scan = p.vecs == 2 ? sample_scan_kernel<2> : sample_scan_kernel<6>;
    DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_SCAN, st, scan, dim3(p.segs, T, batch), dim3(kScanThreads), 0, st, logits, T, V, p.seg_len, p.segs,
               p.hot, p.hot_cap, n_nodes, stat, hot, n_hard, opt);
    DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_PICK, st, sample_pick_kernel, dim3(T, batch), dim3(kPickThreads), 0, st, logits, T, V, p.seg_len, p.segs,
               p.hot_cap, n_nodes, uniforms, stat, hot, *part, tokens, n_hard, hard, opt);
    // (A row goes on the list by what its logits are: these look whether there are any.)
    // The launches for their steps are made where some sequence's rows are often on it: top-p or min-p alone, or a top-k above 700.  Other rows
    // that get there are read as often as it takes, by a workgroup each.  These are rows of a top-k beyond what their lists hold above the
    // largest of the bounds (elements of rows at random: some 200 for V = 2000, 500 to 900 with 75 segments of 2048, 950 to 1250 with 25 of 6144), and
    // rows with many of the likely ids in one segment.  Without the launches 257 rows of 151936 by top-k 50 take 48 us instead
    // of 51; but where 16 rows by top-k 701 take 28 us from the list on, by top-k 700 it is 185, and 257 rows by top-k 50 whose first
    // 6144 logits are higher by 2 take 190.
    bool shared = false;
    for (int s = 0; s < batch; ++s)
        shared = shared || (opt.tau[s] > 0.0f && (opt.top_k[s] > 700 || (opt.top_k[s] == 0 && (opt.top_p[s] < 1.0f || opt.min_p[s] > 0.0f))));
    const int rows = batch * T, slots = shared ? p.slots : 0, most = (int)std::min<long long>(kStepGrid, (long long)p.slots * p.parts);
    if (shared) {
        DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_STEPS, st, sample_steps_kernel, dim3(most), dim3(kStepThreads), 0, st, logits, T, V, p.parts,
                   slots, n_hard, hard, steps, opt);
        DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_GATHER, st, sample_gather_kernel, dim3(most), dim3(kStepThreads), 0, st, logits, T, V, p.parts,
                   slots, n_hard, hard, steps, few, opt);
    }
    DDT_LAUNCH(DDTREE_KERNEL_SAMPLE_AGAIN, st, sample_again_kernel, dim3(std::min(rows, kAgainGrid)), dim3(kAgainThreads), 0, st, logits, T, V,
               p.parts, slots, uniforms, n_hard, hard, steps, few, *part, tokens, opt);
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
