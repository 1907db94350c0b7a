// attend.hip -- attention of a step's new tokens over the block cache.
#include <hip/hip_runtime.h>

#include <math.h>

#include "rk_internal.h"

namespace rk {

struct AttendArgs {
    rk_attention a;
    int32_t* status;
};

template <bool Half>
__device__ __forceinline__ float to_float(uint16_t x)
{
    if constexpr (Half) return (float)__builtin_bit_cast(_Float16, x);
    else return __uint_as_float((uint32_t)x << 16);
}

// fp32 to 16 bits, to nearest even.
template <bool Half>
__device__ __forceinline__ uint16_t from_float(float x)
{
    if constexpr (Half) return __builtin_bit_cast(uint16_t, (_Float16)x);
    else return __builtin_bit_cast(uint16_t, (__bf16)x);
}

// A workgroup of one wavefront per (token, query head): a lane per four-element
// piece of the head, one key after another.
template <bool Half>
__global__ __launch_bounds__(64) void attend_plain_kernel(AttendArgs p)
{
    const rk_attention& a = p.a;
    const int lane = threadIdx.x;
    const int32_t h = (int32_t)blockIdx.y, hk = h / (a.Hq / a.Hkv);
    const int64_t t = blockIdx.x;
    int32_t i = -1;
    for (int32_t x = lane; x < a.B; x += 64) {
        const int64_t x0 = a.q_off[x], x1 = a.q_off[x + 1];
        if (x0 < 0 || x1 < x0 || x1 > a.T) atomicOr(p.status, RK_DEV_BAD_OFFSETS);
        else if (x0 <= t && t < x1) i = x;
    }
    if (a.group_off && t == 0 && h == 0)
        for (int32_t x = lane; x < a.B; x += 64)
            if (a.group_off[x] < 0 || a.group_off[x] > a.group_off[x + 1] || (x == 0 && a.group_off[x] != 0) ||
                (x == a.B - 1 && a.group_off[x + 1] != a.B))
                atomicOr(p.status, RK_DEV_BAD_OFFSETS);
    const uint64_t m = __ballot(i >= 0);
    if (m == 0ull) return;
    i = __builtin_amdgcn_readlane(i, __ffsll((unsigned long long)m) - 1);
    const int64_t q0 = a.q_off[i], q1 = a.q_off[i + 1];
    const int32_t kv = a.kv_len[i];
    const bool large = kv > (int64_t)a.table_stride * RK_BLOCK_TOKENS;
    if (q1 - q0 > kv || large) {
        if (lane == 0) atomicOr(p.status, large ? RK_DEV_TOO_LARGE : RK_DEV_BAD_OFFSETS);
        return;
    }
    const int32_t pos = kv - (int32_t)(q1 - q0) + (int32_t)(t - q0);
    const uint16_t* q = (const uint16_t*)a.q + t * a.q_token + h * a.q_head;
    float qf[4] = {}, o[4] = {}, mx = -INFINITY, l = 0.0f;
    for (int c = 0; c < 4; ++c)
        if (4 * lane + c < a.D) qf[c] = to_float<Half>(q[4 * lane + c]);
    for (int32_t j = 0; j <= pos; ++j) {
        const int32_t b = a.tables[(int64_t)i * a.table_stride + j / RK_BLOCK_TOKENS];
        if (b < 0 || b >= a.n_blocks) {
            if (lane == 0) atomicOr(p.status, RK_DEV_BAD_BLOCK);
            continue;
        }
        const uint16_t* k = (const uint16_t*)a.k_cache + b * a.ks.block + (j % RK_BLOCK_TOKENS) * a.ks.token + hk * a.ks.head;
        const uint16_t* v = (const uint16_t*)a.v_cache + b * a.vs.block + (j % RK_BLOCK_TOKENS) * a.vs.token + hk * a.vs.head;
        float s = 0.0f;
        for (int c = 0; c < 4; ++c)
            if (4 * lane + c < a.D) s += qf[c] * to_float<Half>(k[4 * lane + c]);
        for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
        s *= a.scale;
        const float nm = fmaxf(mx, s), w = expf(s - nm), keep = expf(mx - nm);
        l = l * keep + w;
        for (int c = 0; c < 4; ++c)
            if (4 * lane + c < a.D) o[c] = o[c] * keep + w * to_float<Half>(v[4 * lane + c]);
        mx = nm;
    }
    uint16_t* out = (uint16_t*)a.out + t * a.out_token + h * a.out_head;
    for (int c = 0; c < 4; ++c)
        if (4 * lane + c < a.D) out[4 * lane + c] = from_float<Half>(l > 0.0f ? o[c] / l : 0.0f);
    if (a.lse && lane == 0) a.lse[t * a.Hq + h] = l > 0.0f ? mx + logf(l) : -INFINITY;
}

}  // namespace rk

using namespace rk;

static const char* attention_sizes(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D, int* rc)
{
    *rc = RK_EINVAL;
    if (T < 0 || B < 0) return "a negative size";
    if (Hq < 1 || Hkv < 1 || Hq % Hkv) return "Hq is no multiple of Hkv";
    *rc = RK_EUNSUPPORTED;
    if (B > RK_MAX_BATCH) return "B > RK_MAX_BATCH";
    if (Hq / Hkv > 128) return "more than 128 query heads per key head";
    if (Hkv > 1024) return "Hkv > 1024";
    if (D < 8 || D > 256 || D % 8) return "D is no multiple of 8 in 8..256";
    if (T > 0x7fffffff / Hq) return "T * Hq >= 2^31";
    *rc = RK_OK;
    return nullptr;
}

extern "C" {

size_t rk_prefix_attention_workspace_size(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    int rc;
    if (attention_sizes(T, B, Hq, Hkv, D, &rc)) return 0;
    return 256;
}

int rk_prefix_attention(const rk_attention* a, void* workspace, size_t ws_bytes, void* stream)
{
    if (!a) return fail(RK_EINVAL, "rk_prefix_attention: NULL arguments");
    int rc;
    if (const char* what = attention_sizes(a->T, a->B, a->Hq, a->Hkv, a->D, &rc))
        return fail(rc, "rk_prefix_attention: %s", what);
    if (a->dtype != RK_BF16 && a->dtype != RK_F16) return fail(RK_EUNSUPPORTED, "rk_prefix_attention: dtype %d", a->dtype);
    if (a->n_blocks < 0 || a->table_stride < 0) return fail(RK_EINVAL, "rk_prefix_attention: a negative size");
    if (!(fabsf(a->scale) <= 3.0e38f)) return fail(RK_EINVAL, "rk_prefix_attention: scale is not finite");
    const int64_t strides[] = {a->q_token, a->q_head, a->out_token, a->out_head, a->ks.block, a->ks.token, a->ks.head,
                               a->vs.block, a->vs.token, a->vs.head};
    for (int64_t x : strides)
        if (x < 0 || x % 8) return fail(RK_EINVAL, "rk_prefix_attention: a stride is negative or no multiple of 8");
    if (a->ks.token < a->D || a->vs.token < a->D || a->ks.token >= 1 << 26 || a->vs.token >= 1 << 26)
        return fail(RK_EINVAL, "rk_prefix_attention: a cache's token stride is below D or past 2^26");
    if (!a->group_off != !a->shared)
        return fail(RK_EINVAL, "rk_prefix_attention: group_off without shared, or the reverse");
    if (a->B == 0 || a->T == 0) return RK_OK;
    if (!a->q || !a->out || !a->kv_len || !a->q_off || (a->table_stride > 0 && !a->tables) ||
        (a->n_blocks > 0 && (!a->k_cache || !a->v_cache)))
        return fail(RK_EINVAL, "rk_prefix_attention: NULL array");
    if (((uintptr_t)a->q | (uintptr_t)a->out | (uintptr_t)a->k_cache | (uintptr_t)a->v_cache) % 16)
        return fail(RK_EINVAL, "rk_prefix_attention: an array is not aligned to 16 bytes");
    const size_t need = rk_prefix_attention_workspace_size(a->T, a->B, a->Hq, a->Hkv, a->D);
    if (!workspace || ws_bytes < need)
        return fail(RK_ENOMEM, "rk_prefix_attention: workspace of %zu bytes, %zu needed", workspace ? ws_bytes : (size_t)0, need);
    if ((uintptr_t)workspace % 256) return fail(RK_EINVAL, "rk_prefix_attention: workspace is not aligned to 256 bytes");
    AttendArgs p;
    p.a = *a;
    p.status = status_word();
    if (!p.status) return fail(RK_EHIP, "rk_prefix_attention: no status word");
    const dim3 grid((unsigned)a->T, (unsigned)a->Hq);
    if (a->dtype == RK_F16) hipLaunchKernelGGL(attend_plain_kernel<true>, grid, dim3(64), 0, (hipStream_t)stream, p);
    else hipLaunchKernelGGL(attend_plain_kernel<false>, grid, dim3(64), 0, (hipStream_t)stream, p);
    return hip_check(hipGetLastError(), "rk_prefix_attention launch");
}

}  // extern "C"
