// fp4.hip -- a block cache held in 4 bits: writes and reads.
//
// 32 neighbouring values of a head (the last of D may be fewer) share a power of two, of which each is a multiple by 0, 0.5, 1,
// 1.5, 2, 3, 4 or 6 and a sign.  With a the largest of them in magnitude and e the least whole number with a <= 7 2^e,
// a value is off by at most half the distance of its neighbours on that grid, or by a - 6 2^e <= 2^e.  Everything is exact but the one rounding to
// that grid, so what the cache holds follows from the values alone.
#include <hip/hip_runtime.h>

#include "rk_internal.h"

namespace rk {

// The bytes of the powers that a type's caches use: with them all values are the type's own, none of them subnormal in bf16
// (8 bits of exponent hold 2^-126 and more), none of them past its range.
template <bool Half>
constexpr int32_t kLeastPower = Half ? 127 - 23 : 127 - 125;
template <bool Half>
constexpr int32_t kMostPower = Half ? 127 + 13 : 127 + 125;

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

// The codes of eight values, the first's in the lowest bits.
template <bool Half>
__device__ __forceinline__ uint32_t fp4_codes(u32x4 x, float scale)
{
    const uint32_t a = x.x, b = x.y, c = x.z, d = x.w;       // (a bit_cast takes no vector's element)
    uint32_t codes = 0;
    if constexpr (Half) {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, a), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, b), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, c), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(codes, __builtin_bit_cast(f16x2, d), scale, 3);
    } else {
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, a), scale, 0);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, b), scale, 1);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, c), scale, 2);
        codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, d), scale, 3);
    }
    return codes;
}

constexpr int kAtOnce = 4;                           // places that a thread loads for together
// x / d of 32-bit numbers: m = 2^32 / d rounded up is exact for x * d < 2^32.
struct Divisor {
    uint32_t d, m;
};
inline Divisor divisor_of(uint32_t d) { return Divisor{d, (uint32_t)(((1ull << 32) + d - 1) / d)}; }
__device__ __forceinline__ uint32_t divided(uint32_t x, Divisor d) { return d.d == 1 ? x : __umulhi(x, d.m); }

// Four lanes a group of 32 values, 8 each: whole rows are read and written.  blockIdx.y: keys or values.  A workgroup takes stretches of
// tokens, a thread kAtOnce places of them.  Memory bounds it: 16,384 tokens of 8 heads of 128 (67 MB read, 18 MB written) 17.8 us, 4.8 TB/s.
// (One place a thread at a time: 51 us with the reading of the same tokens, now 41.)
template <bool Half>
__global__ __launch_bounds__(256) void write_fp4_kernel(int64_t T, int32_t stretch, Divisor per, Divisor pieces, int32_t D,
                                                        const uint16_t* __restrict__ k, int64_t k_token, int64_t k_head,
                                                        const uint16_t* __restrict__ v, int64_t v_token, int64_t v_head, rk_fp4_cache kc,
                                                        rk_fp4_cache vc, int32_t n_blocks, const int64_t* __restrict__ slots,
                                                        int32_t* status)
{
    const bool values = blockIdx.y != 0;
    const uint16_t* __restrict__ src = values ? v : k;
    const rk_fp4_cache c = values ? vc : kc;
    const int64_t s_token = values ? v_token : k_token, s_head = values ? v_head : k_head;
    for (int64_t t0 = (int64_t)blockIdx.x * stretch; t0 < T; t0 += (int64_t)gridDim.x * stretch) {
        const uint32_t tokens = (uint32_t)(T - t0 < stretch ? T - t0 : stretch), n = tokens * per.d;      // (a multiple of 4)
        for (uint32_t x0 = threadIdx.x; x0 < (n + 255) / 256 * 256; x0 += 256 * kAtOnce) {
            u32x4 val[kAtOnce];
            int64_t slot[kAtOnce];
            uint32_t h[kAtOnce], piece[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t at = x0 + 256 * u, x = at < n ? at : n - 4 + (at & 3);      // (four lanes stay together)
                const uint32_t tok = divided(x, per), r = x - tok * per.d;
                h[u] = divided(r, pieces);
                piece[u] = r - h[u] * pieces.d;
                const int64_t t = t0 + tok;
                slot[u] = at < n ? slots[t] : -1;
                val[u] = u32x4{0u, 0u, 0u, 0u};
                if (8 * piece[u] < (uint32_t)D) val[u] = *reinterpret_cast<const u32x4*>(src + t * s_token + h[u] * s_head + 8 * piece[u]);
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                // the largest magnitude, by its bits
                u16x2 most = {0, 0};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, val[u][i] & 0x7fff7fffu));
                uint32_t top = most.x > most.y ? most.x : most.y;
#pragma unroll
                for (int d = 1; d < 4; d <<= 1) {
                    const uint32_t other = __shfl_xor(top, d);
                    top = top > other ? top : other;
                }
                const bool finite = top < (Half ? 0x7c00u : 0x7f80u);
                const uint32_t bits =
                    __float_as_uint(Half ? (float)__builtin_bit_cast(_Float16, (uint16_t)top) : __uint_as_float(top << 16));
                int32_t power = (int32_t)((bits + 0x1fffffu) >> 23) - 2;     // 1.75 2^n or less: 2^(n-2), else 2^(n-1)
                power = power < kLeastPower<Half> ? kLeastPower<Half> : power > kMostPower<Half> ? kMostPower<Half> : power;
                const uint32_t codes = fp4_codes<Half>(val[u], __uint_as_float((uint32_t)power << 23));
                const int64_t block = slot[u] / RK_BLOCK_TOKENS, tok = slot[u] % RK_BLOCK_TOKENS;
                if (slot[u] < 0) continue;
                if (block >= n_blocks) {
                    if (h[u] == 0 && piece[u] == 0) atomicOr(status, RK_DEV_BAD_BLOCK);
                    continue;
                }
                *reinterpret_cast<uint32_t*>((uint8_t*)c.codes + block * c.cs.block + tok * c.cs.token + h[u] * c.cs.head + 4 * piece[u]) =
                    finite ? codes : 0u;
                if (piece[u] % 4 == 0)
                    ((uint8_t*)c.scales)[block * c.ss.block + tok * c.ss.token + h[u] * c.ss.head + piece[u] / 4] =
                        finite ? (uint8_t)power : 255;
            }
        }
    }
}

// The reverse, a thread 8 values of a place.  The outputs are whole lines that this kernel does not read again, and pass the caches by.
// Memory bounds it: 65,536 tokens of 8 heads of 128 (71 MB read, 268 MB written) 78 us, 4.3 TB/s; 93
// with one place a thread at a time and ordinary stores.
template <bool Half>
__global__ __launch_bounds__(256) void read_fp4_kernel(int64_t T, int32_t stretch, Divisor per, Divisor D8, uint16_t* __restrict__ k,
                                                       int64_t k_token, int64_t k_head, uint16_t* __restrict__ v,
                                                       int64_t v_token, int64_t v_head, rk_fp4_cache kc, rk_fp4_cache vc,
                                                       int32_t n_blocks, const int64_t* __restrict__ slots, int32_t* status)
{
    const bool values = blockIdx.y != 0;
    uint16_t* __restrict__ dst = values ? v : k;
    const rk_fp4_cache c = values ? vc : kc;
    const int64_t d_token = values ? v_token : k_token, d_head = values ? v_head : k_head;
    for (int64_t t0 = (int64_t)blockIdx.x * stretch; t0 < T; t0 += (int64_t)gridDim.x * stretch) {
        const uint32_t tokens = (uint32_t)(T - t0 < stretch ? T - t0 : stretch), n = tokens * per.d;
        for (uint32_t x0 = threadIdx.x; x0 < n; x0 += 256 * kAtOnce) {
            int64_t slot[kAtOnce];
            uint32_t h[kAtOnce], piece[kAtOnce], codes[kAtOnce], power[kAtOnce];
            int64_t t[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t x = x0 + 256 * u < n ? x0 + 256 * u : n - 1, tok = divided(x, per), r = x - tok * per.d;
                h[u] = divided(r, D8);
                piece[u] = r - h[u] * D8.d;
                t[u] = t0 + tok;
                slot[u] = slots[t[u]];
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int64_t block = slot[u] / RK_BLOCK_TOKENS, tok = slot[u] % RK_BLOCK_TOKENS;
                const bool there = slot[u] >= 0 && block < n_blocks;
                if (slot[u] >= 0 && block >= n_blocks && h[u] == 0 && piece[u] == 0) atomicOr(status, RK_DEV_BAD_BLOCK);
                codes[u] = power[u] = 0;
                if (there) {
                    codes[u] = *reinterpret_cast<const uint32_t*>((const uint8_t*)c.codes + block * c.cs.block + tok * c.cs.token +
                                                                  h[u] * c.cs.head + 4 * piece[u]);
                    power[u] = ((const uint8_t*)c.scales)[block * c.ss.block + tok * c.ss.token + h[u] * c.ss.head + piece[u] / 4];
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                if (x0 + 256 * u >= n) break;
                const u32x4 val = codes[u] | power[u] ? fp4_values<Half>(codes[u], __uint_as_float(power[u] << 23)) : u32x4{0u, 0u, 0u, 0u};
                u32x4* to = reinterpret_cast<u32x4*>(dst + t[u] * d_token + h[u] * d_head + 8 * piece[u]);
                __builtin_nontemporal_store(val, to);
            }
        }
    }
}

// Tokens of a stretch, `per` threads each, so that a workgroup has work for `at_once` places a thread; stretches of T tokens, or as many
// workgroups as take them in turn.
static int32_t stretch_of(int32_t per, int32_t at_once) { return per >= 256 * at_once ? 1 : (256 * at_once + per - 1) / per; }
static unsigned stretches(int64_t T, int32_t stretch)
{
    const int64_t n = (T + stretch - 1) / stretch;
    return (unsigned)(n < (1 << 20) ? n : 1 << 20);
}

// What the two entry points refuse alike: `k` and `v` are the tokens' rows, [T, Hkv, D].
static int tokens_arguments(const char* name, int64_t T, int32_t Hkv, int32_t D, int32_t dtype, const void* k, int64_t k_token,
                            int64_t k_head, const void* v, int64_t v_token, int64_t v_head, const rk_fp4_cache* kc,
                            const rk_fp4_cache* vc, int32_t n_blocks, const int64_t* slots)
{
    if (T < 0 || n_blocks < 0) return fail(RK_EINVAL, "%s: a negative size", name);
    if (Hkv < 1 || Hkv > 1024) return fail(RK_EUNSUPPORTED, "%s: Hkv outside 1..1024", name);
    if (D < 8 || D > 256 || D % 8) return fail(RK_EUNSUPPORTED, "%s: D is no multiple of 8 in 8..256", name);
    if (dtype != RK_BF16 && dtype != RK_F16) return fail(RK_EUNSUPPORTED, "%s: dtype %d", name, dtype);
    if (!kc || !vc) return fail(RK_EINVAL, "%s: NULL cache", name);
    for (int64_t x : {k_token, k_head, v_token, v_head})
        if (x < 0 || x % 8) return fail(RK_EINVAL, "%s: a stride is negative or no multiple of 8", name);
    for (const rk_fp4_cache& c : {*kc, *vc})
        if (!fp4_strides(c)) return fail(RK_EINVAL, "%s: a stride is negative, or one of codes no multiple of 16", name);
    if (T == 0) return RK_OK;
    if (!k || !v || !slots || (n_blocks > 0 && (!kc->codes || !kc->scales || !vc->codes || !vc->scales)))
        return fail(RK_EINVAL, "%s: NULL array", name);
    if (((uintptr_t)k | (uintptr_t)v | (uintptr_t)kc->codes | (uintptr_t)vc->codes) % 16)
        return fail(RK_EINVAL, "%s: an array is not aligned to 16 bytes", name);
    return RK_OK;
}

}  // namespace rk

using namespace rk;

extern "C" {

int rk_kv_write_fp4(int64_t T, int32_t Hkv, int32_t D, int32_t dtype, const void* k, int64_t k_token, int64_t k_head, const void* v,
                    int64_t v_token, int64_t v_head, const rk_fp4_cache* k_cache, const rk_fp4_cache* v_cache, int32_t n_blocks,
                    const int64_t* slots, void* stream)
{
    const char* name = "rk_kv_write_fp4";
    if (int rc = tokens_arguments(name, T, Hkv, D, dtype, k, k_token, k_head, v, v_token, v_head, k_cache, v_cache, n_blocks, slots))
        return rc;
    const int32_t shares = (D + 31) / 32;
    for (const rk_fp4_cache& c : {*k_cache, *v_cache})
        if (!rows_apart({{n_blocks, c.cs.block}, {RK_BLOCK_TOKENS, c.cs.token}, {Hkv, c.cs.head}}, 16 * shares) ||
            !rows_apart({{n_blocks, c.ss.block}, {RK_BLOCK_TOKENS, c.ss.token}, {Hkv, c.ss.head}}, shares))
            return fail(RK_EINVAL, "%s: a cache's strides lay heads, tokens or blocks over each other", name);
    if (T == 0) return RK_OK;
    int32_t* st = status_word();
    if (!st) return fail(RK_EHIP, "%s: no status word", name);
    const int32_t per = Hkv * shares * 4, stretch = stretch_of(per, kAtOnce);
    hipLaunchKernelGGL(dtype == RK_F16 ? write_fp4_kernel<true> : write_fp4_kernel<false>, dim3(stretches(T, stretch), 2), dim3(256), 0,
                       (hipStream_t)stream, T, stretch, divisor_of((uint32_t)per), divisor_of((uint32_t)shares * 4), D, (const uint16_t*)k,
                       k_token, k_head, (const uint16_t*)v, v_token, v_head, *k_cache, *v_cache, n_blocks, slots, st);
    return hip_check(hipGetLastError(), "rk_kv_write_fp4 launch");
}

int rk_kv_read_fp4(int64_t T, int32_t Hkv, int32_t D, int32_t dtype, const rk_fp4_cache* k_cache, const rk_fp4_cache* v_cache,
                   int32_t n_blocks, const int64_t* slots, void* k, int64_t k_token, int64_t k_head, void* v, int64_t v_token,
                   int64_t v_head, void* stream)
{
    const char* name = "rk_kv_read_fp4";
    if (int rc = tokens_arguments(name, T, Hkv, D, dtype, k, k_token, k_head, v, v_token, v_head, k_cache, v_cache, n_blocks, slots))
        return rc;
    if (!rows_apart({{T, k_token}, {Hkv, k_head}}, D) || !rows_apart({{T, v_token}, {Hkv, v_head}}, D))
        return fail(RK_EINVAL, "%s: an output's strides lay heads or tokens over each other", name);
    if (T == 0) return RK_OK;
    int32_t* st = status_word();
    if (!st) return fail(RK_EHIP, "%s: no status word", name);
    const int32_t per = Hkv * (D / 8), stretch = stretch_of(per, kAtOnce);
    hipLaunchKernelGGL(dtype == RK_F16 ? read_fp4_kernel<true> : read_fp4_kernel<false>,
                       dim3(stretches(T, stretch), 2), dim3(256), 0, (hipStream_t)stream, T, stretch,
                       divisor_of((uint32_t)per), divisor_of((uint32_t)D / 8), (uint16_t*)k, k_token, k_head, (uint16_t*)v, v_token,
                       v_head, *k_cache, *v_cache, n_blocks, slots, st);
    return hip_check(hipGetLastError(), "rk_kv_read_fp4 launch");
}

}  // extern "C"
