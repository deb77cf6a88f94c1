// A KV cache in 4 bits: quantised as it is written (prompts, and the accepted path that closes a round, paper
// Section 4.4, last sentence), and read back.
//
// The head dim is cut into blocks of 32.  A block is stored as a power of two 2^e and 32 codes of 4 bits, sign and
// one of 0, 0.5, 1, 1.5, 2, 3, 4, 6:
//   e     exponent of the block's largest magnitude, rounded to two significant bits (ties to even), less 2, so that
//         the largest magnitude lies in [3.5, 7) 2^e and rounds to 4 or 6: no element is off by more than half a
//         step of the grid.  From -124 to 125, so that every value is a normal, finite number in bf16 too (magnitudes
//         from 7 2^125 on, those within an eighth of the largest of the type, are stored as 6 2^125).
//   code  x / 2^e rounded to the nearest (ties to even): the conversion instructions of gfx950 do that, and exactly so
//         the way back (checked for every scale from 2^-127 to 2^127 and every code, on values on and beside each border)
// Arrays are head-major, codes [Hkv, rows, D/2] and scales [Hkv, rows, D/32]: what a workgroup of the attention reads is
// one run of bytes (4 KB for 64 keys of 128), where token-major rows would be half a cache line each.
//
// Bound by the memory system (43960 tokens of 8 heads of 128, bf16, written 57 us, 4.0 TB/s, read back 35 us, 6.5): 4 lanes hold a block, 8 elements (16 bytes of bf16) each; a wave reads runs of D elements
// of successive tokens of one head and writes one run of codes.
#include "attn_common.hpp"

namespace ddt {

constexpr int kQ4Threads = 256;
constexpr int kQ4Units = 4;  // groups of 8 elements per thread, their loads in flight together

// A group's row, and its place in the row (shift: log2 of the groups of a row, -1 where that is no whole number).
__device__ __forceinline__ uint32_t q4_row(uint32_t i, int per_row, int shift)
{
    return shift >= 0 ? i >> shift : i / (uint32_t)per_row;
}

struct Q4Rows {
    int32_t src[DDTREE_MAX_BATCH];   // first row of each sequence, in the row tensor or the cache
    int32_t dst[DDTREE_MAX_BATCH];
    int32_t rows[DDTREE_MAX_BATCH];
};

// Eight elements as fp32.
__device__ __forceinline__ void q4_load8(const float *p, float (&x)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}
__device__ __forceinline__ void q4_load8(const uint16_t *p, float (&x)[8])
{
    const uint4 a = *reinterpret_cast<const uint4 *>(p);
    const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// The codes of eight elements and their block's scale byte; the four lanes of a block are neighbours.  Magnitudes
// are compared as integers, where an infinity or a NaN is the largest: such a block gets the byte 255, which reads
// back as NaN.
__device__ __forceinline__ uint32_t q4_encode8(const float (&x)[8], uint32_t &scale_byte)
{
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7FFFFFFFu);
    top = max(top, dpp_u<0xB1>(top));
    top = max(top, dpp_u<0x4E>(top));
    const bool finite = top < 0x7F800000u;
    // (an addition of a quarter of the leading bit's weight carries into the exponent from 1.75 on)
    const int e = min(max((int)((top + 0x00200000u) >> 23) - 127 - 2, -124), 125);
    scale_byte = finite ? (uint32_t)(e + 127) : 255u;
    const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    uint32_t c = 0u;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
    return finite ? c : 0u;
}

// One workgroup: kQ4Units * 256 groups of eight elements of one (sequence, head), of K or of V.  PATH: row j of a
// sequence is the tree row path[j], for j up to n_accepted; otherwise rows are consecutive.
template <class In, bool PATH>
__global__ __launch_bounds__(kQ4Threads) void q4_write_kernel(
    const In *__restrict__ k, const In *__restrict__ v, uint32_t *__restrict__ k_codes, uint8_t *__restrict__ k_scales,
    uint32_t *__restrict__ v_codes, uint8_t *__restrict__ v_scales, int cache_rows, int Hkv, int per_row, int shift,
    const int32_t *__restrict__ path, const int32_t *__restrict__ n_accepted, int T, int B, Q4Rows args)
{
    const int seq = blockIdx.z, hk = (int)blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const In *const in = is_v ? v : k;
    uint32_t *const codes = is_v ? v_codes : k_codes;
    uint8_t *const scales = is_v ? v_scales : k_scales;
    int rows = args.rows[seq];
    if constexpr (PATH) rows = min(n_accepted[seq], B) + 1;
    const uint32_t n = (uint32_t)max(rows, 0) * per_row;  // groups of eight (the host has seen to it that 31 bits hold them)
    const uint32_t first = blockIdx.x * (kQ4Units * kQ4Threads) + threadIdx.x;
    if (first - threadIdx.x >= n) return;
    float x[kQ4Units][8];
    size_t at[kQ4Units];
    bool on[kQ4Units];
#pragma unroll
    for (int u = 0; u < kQ4Units; ++u) {
        const uint32_t i = first + u * kQ4Threads;
        on[u] = i < n;
        const int row = on[u] ? (int)q4_row(i, per_row, shift) : 0, c = on[u] ? (int)i - row * per_row : 0;
        int src = args.src[seq] + row;
        if constexpr (PATH) {
            const int node = path[(size_t)seq * (B + 1) + row];
            on[u] = on[u] && node >= 0 && node < T;  // (the lanes of a block agree)
            src = seq * T + (on[u] ? node : 0);
        }
        at[u] = ((size_t)hk * cache_rows + args.dst[seq] + row) * per_row + c;
        if (on[u]) {
            q4_load8(in + ((size_t)src * Hkv + hk) * ((size_t)per_row * 8) + c * 8, x[u]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[u][e] = 0.0f;
        }
    }
#pragma unroll
    for (int u = 0; u < kQ4Units; ++u) {
        uint32_t scale_byte;
        const uint32_t c = q4_encode8(x[u], scale_byte);
        if (on[u]) {
            codes[at[u]] = c;
            if ((threadIdx.x & 3) == 0) scales[at[u] >> 2] = (uint8_t)scale_byte;
        }
    }
}

__device__ __forceinline__ void q4_store8(float *p, const uint32_t (&w)[4])
{
    reinterpret_cast<uint4 *>(p)[0] = make_uint4(w[0] << 16, w[0] & 0xFFFF0000u, w[1] << 16, w[1] & 0xFFFF0000u);
    reinterpret_cast<uint4 *>(p)[1] = make_uint4(w[2] << 16, w[2] & 0xFFFF0000u, w[3] << 16, w[3] & 0xFFFF0000u);
}
__device__ __forceinline__ void q4_store8(uint16_t *p, const uint32_t (&w)[4])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}

// The way back, laid out alike.  The values are exact in bf16 (two significant bits), so fp32 rows are made of them.
template <class Out>
__global__ __launch_bounds__(kQ4Threads) void q4_read_kernel(
    const uint32_t *__restrict__ k_codes, const uint8_t *__restrict__ k_scales, const uint32_t *__restrict__ v_codes,
    const uint8_t *__restrict__ v_scales, int cache_rows, int Hkv, int per_row, int shift, Out *__restrict__ k,
    Out *__restrict__ v, Q4Rows args)
{
    const int seq = blockIdx.z, hk = (int)blockIdx.y >> 1;
    const bool is_v = blockIdx.y & 1;
    const uint32_t *const codes = is_v ? v_codes : k_codes;
    const uint8_t *const scales = is_v ? v_scales : k_scales;
    Out *const out = is_v ? v : k;
    const uint32_t n = (uint32_t)args.rows[seq] * per_row;
    const uint32_t first = blockIdx.x * (kQ4Units * kQ4Threads) + threadIdx.x;
    const size_t base = ((size_t)hk * cache_rows + args.src[seq]) * per_row;
    uint32_t c[kQ4Units], b[kQ4Units];
#pragma unroll
    for (int u = 0; u < kQ4Units; ++u) {
        const uint32_t i = first + u * kQ4Threads;
        c[u] = i < n ? codes[base + i] : 0u;
        b[u] = i < n ? scales[(base + i) >> 2] : 0u;
    }
#pragma unroll
    for (int u = 0; u < kQ4Units; ++u) {
        const uint32_t i = first + u * kQ4Threads;
        if (i >= n) break;
        uint32_t w[4];
        q4_decode8(c[u], __uint_as_float(b[u] << 23), w);
        const uint32_t row = q4_row(i, per_row, shift);
        q4_store8(out + (((size_t)args.dst[seq] + row) * Hkv + hk) * ((size_t)per_row * 8) + (i - row * per_row) * 8, w);
    }
}

// What every call on a 4-bit cache wants of it.
bool q4_cache_ok(const void *k_codes, const void *k_scales, const void *v_codes, const void *v_scales, int cache_rows,
                 int Hkv, int D)
{
    if (!k_codes || !k_scales || !v_codes || !v_scales || cache_rows < 1 || Hkv < 1 || Hkv > 32767 || D < 32 || D > 256 ||
        D % 32 != 0)
        return false;
    for (const void *t : {k_codes, v_codes})
        if (reinterpret_cast<uintptr_t>(t) & 15u) return false;
    // (the scales of a row of 128 are read as one word)
    for (const void *t : {k_scales, v_scales})
        if (reinterpret_cast<uintptr_t>(t) & 3u) return false;
    return true;
}

}  // namespace ddt

namespace {

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Whether two sequences would write a row both: its codes could be one's and its scales the other's.
bool q4_shared_rows(const int32_t *first, const int32_t *rows, int batch)
{
    for (int s = 1; s < batch; ++s)
        for (int t = 0; t < s; ++t)
            if (rows[s] > 0 && rows[t] > 0 && (long long)first[s] < (long long)first[t] + rows[t] &&
                (long long)first[t] < (long long)first[s] + rows[s])
                return true;
    return false;
}

// Sequence s has rows offset[s] .. offset[s + 1] of the row tensor and as many from cache_row[s] on of the cache.
// Returns the most rows of a sequence, or -1; the groups of eight elements of a sequence and head are counted in 31 bits.
int q4_ranges(const int32_t *offset, const int32_t *cache_row, int batch, int cache_rows, int D, int32_t *row0, int32_t *cache0, int32_t *rows)
{
    int most = 0;
    if (offset[0] < 0) return -1;
    for (int s = 0; s < batch; ++s) {
        if (offset[s + 1] < offset[s]) return -1;
        const int n = offset[s + 1] - offset[s];
        if (cache_row[s] < 0 || (long long)cache_row[s] + n > cache_rows || (long long)n * (D / 8) > 0x7FFFF000ll)
            return -1;
        row0[s] = offset[s];
        cache0[s] = cache_row[s];
        rows[s] = n;
        most = n > most ? n : most;
    }
    return most;
}

dim3 q4_grid(int most_rows, int per_row, int Hkv, int batch)
{
    const long long groups = (long long)most_rows * per_row, per_wg = ddt::kQ4Units * ddt::kQ4Threads;
    return dim3((unsigned)((groups + per_wg - 1) / per_wg), (unsigned)(2 * Hkv), (unsigned)batch);
}

int q4_shift(int D) { return D == 32 ? 2 : D == 64 ? 3 : D == 128 ? 4 : D == 256 ? 5 : -1; }

}  // namespace

extern "C" int ddtree_q4_store(const void *k, const void *v, const int32_t *src_offset, const int32_t *dst_row,
                               int batch, int Hkv, int D, int dtype, void *k_codes, void *k_scales, void *v_codes,
                               void *v_scales, int cache_rows, void *stream)
{
    using namespace ddt;
    if (!src_offset || !dst_row || batch < 1 || batch > DDTREE_MAX_BATCH) return DDTREE_ERR_ARG;
    if (!q4_cache_ok(k_codes, k_scales, v_codes, v_scales, cache_rows, Hkv, D)) return DDTREE_ERR_ARG;
    if (dtype != DDTREE_DTYPE_BF16 && dtype != DDTREE_DTYPE_FP32) return DDTREE_ERR_ARG;
    Q4Rows args{};
    const int most = q4_ranges(src_offset, dst_row, batch, cache_rows, D, args.src, args.dst, args.rows);
    if (most < 0 || q4_shared_rows(args.dst, args.rows, batch)) return DDTREE_ERR_ARG;
    if (most == 0) return DDTREE_OK;  // (a tensor without rows may have no address)
    if (!k || !v || !aligned16(k) || !aligned16(v)) return DDTREE_ERR_ARG;
    const dim3 grid = q4_grid(most, D / 8, Hkv, batch);
    uint32_t *const kc = static_cast<uint32_t *>(k_codes), *const vc = static_cast<uint32_t *>(v_codes);
    uint8_t *const ks = static_cast<uint8_t *>(k_scales), *const vs = static_cast<uint8_t *>(v_scales);
    if (dtype == DDTREE_DTYPE_BF16)
        DDT_LAUNCH(DDTREE_KERNEL_Q4_WRITE, as_stream(stream), (q4_write_kernel<uint16_t, false>), grid, dim3(kQ4Threads), 0,
                   as_stream(stream), static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v), kc, ks, vc, vs,
                   cache_rows, Hkv, D / 8, q4_shift(D), nullptr, nullptr, 0, 0, args);
    else
        DDT_LAUNCH(DDTREE_KERNEL_Q4_WRITE, as_stream(stream), (q4_write_kernel<float, false>), grid, dim3(kQ4Threads), 0,
                   as_stream(stream), static_cast<const float *>(k), static_cast<const float *>(v), kc, ks, vc, vs,
                   cache_rows, Hkv, D / 8, q4_shift(D), nullptr, nullptr, 0, 0, args);
    return launch_status();
}

extern "C" int ddtree_q4_append(const void *k_tree, const void *v_tree, const int32_t *path, const int32_t *n_accepted,
                                const int32_t *dst_row, int batch, int T, int B, int Hkv, int D, int dtype, void *k_codes,
                                void *k_scales, void *v_codes, void *v_scales, int cache_rows, void *stream)
{
    using namespace ddt;
    if (!k_tree || !v_tree || !path || !n_accepted || !dst_row || batch < 1 || batch > DDTREE_MAX_BATCH || T < 1 ||
        T > DDTREE_MAX_N + 1 || B < 1 || B > DDTREE_MAX_B || !aligned16(k_tree) || !aligned16(v_tree))
        return DDTREE_ERR_ARG;
    if (!q4_cache_ok(k_codes, k_scales, v_codes, v_scales, cache_rows, Hkv, D)) return DDTREE_ERR_ARG;
    if (dtype != DDTREE_DTYPE_BF16 && dtype != DDTREE_DTYPE_FP32) return DDTREE_ERR_ARG;
    Q4Rows args{};
    for (int s = 0; s < batch; ++s) {
        if (dst_row[s] < 0 || (long long)dst_row[s] + B + 1 > cache_rows) return DDTREE_ERR_ARG;
        args.dst[s] = dst_row[s];
        args.rows[s] = B + 1;  // (at most: the kernel goes by n_accepted)
    }
    if (q4_shared_rows(args.dst, args.rows, batch)) return DDTREE_ERR_ARG;
    const dim3 grid = q4_grid(B + 1, D / 8, Hkv, batch);
    uint32_t *const kc = static_cast<uint32_t *>(k_codes), *const vc = static_cast<uint32_t *>(v_codes);
    uint8_t *const ks = static_cast<uint8_t *>(k_scales), *const vs = static_cast<uint8_t *>(v_scales);
    if (dtype == DDTREE_DTYPE_BF16)
        DDT_LAUNCH(DDTREE_KERNEL_Q4_WRITE, as_stream(stream), (q4_write_kernel<uint16_t, true>), grid, dim3(kQ4Threads), 0,
                   as_stream(stream), static_cast<const uint16_t *>(k_tree), static_cast<const uint16_t *>(v_tree), kc, ks,
                   vc, vs, cache_rows, Hkv, D / 8, q4_shift(D), path, n_accepted, T, B, args);
    else
        DDT_LAUNCH(DDTREE_KERNEL_Q4_WRITE, as_stream(stream), (q4_write_kernel<float, true>), grid, dim3(kQ4Threads), 0,
                   as_stream(stream), static_cast<const float *>(k_tree), static_cast<const float *>(v_tree), kc, ks, vc,
                   vs, cache_rows, Hkv, D / 8, q4_shift(D), path, n_accepted, T, B, args);
    return launch_status();
}

extern "C" int ddtree_q4_load(const void *k_codes, const void *k_scales, const void *v_codes, const void *v_scales,
                              int cache_rows, const int32_t *src_row, const int32_t *dst_offset, int batch, int Hkv,
                              int D, int dtype, void *k, void *v, void *stream)
{
    using namespace ddt;
    if (!src_row || !dst_offset || batch < 1 || batch > DDTREE_MAX_BATCH) return DDTREE_ERR_ARG;
    if (!q4_cache_ok(k_codes, k_scales, v_codes, v_scales, cache_rows, Hkv, D)) return DDTREE_ERR_ARG;
    if (dtype != DDTREE_DTYPE_BF16 && dtype != DDTREE_DTYPE_FP32) return DDTREE_ERR_ARG;
    Q4Rows args{};
    const int most = q4_ranges(dst_offset, src_row, batch, cache_rows, D, args.dst, args.src, args.rows);
    if (most < 0) return DDTREE_ERR_ARG;
    if (most == 0) return DDTREE_OK;  // (a tensor without rows may have no address)
    if (!k || !v || !aligned16(k) || !aligned16(v)) return DDTREE_ERR_ARG;
    const dim3 grid = q4_grid(most, D / 8, Hkv, batch);
    const uint32_t *const kc = static_cast<const uint32_t *>(k_codes), *const vc = static_cast<const uint32_t *>(v_codes);
    const uint8_t *const ks = static_cast<const uint8_t *>(k_scales), *const vs = static_cast<const uint8_t *>(v_scales);
    if (dtype == DDTREE_DTYPE_BF16)
        DDT_LAUNCH(DDTREE_KERNEL_Q4_READ, as_stream(stream), q4_read_kernel<uint16_t>, grid, dim3(kQ4Threads), 0,
                   as_stream(stream), kc, ks, vc, vs, cache_rows, Hkv, D / 8, q4_shift(D), static_cast<uint16_t *>(k),
                   static_cast<uint16_t *>(v), args);
    else
        DDT_LAUNCH(DDTREE_KERNEL_Q4_READ, as_stream(stream), q4_read_kernel<float>, grid, dim3(kQ4Threads), 0,
                   as_stream(stream), kc, ks, vc, vs, cache_rows, Hkv, D / 8, q4_shift(D), static_cast<float *>(k),
                   static_cast<float *>(v), args);
    return launch_status();
}
