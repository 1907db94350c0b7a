// attend.hip -- rk_prefix_attention: the entry points, and the kernels of 16-bit caches.
#include "attend.h"

using namespace rk;

extern "C" {

size_t rk_prefix_attention_workspace_size(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    int rc;
    if (attention_sizes(T, B, Hq, Hkv, D, &rc)) return 0;
    return attend_layout(T, B, Hq, Hkv, D).bytes;
}

int rk_prefix_attention(const rk_attention* a, void* workspace, size_t ws_bytes, void* stream)
{
    const char* name = "rk_prefix_attention";
    if (!a) return fail(RK_EINVAL, "%s: NULL arguments", name);
    if (int rc = attention_arguments(*a, name)) return rc;
    for (int64_t x : {a->ks.block, a->ks.token, a->ks.head, a->vs.block, a->vs.token, a->vs.head})
        if (x < 0 || x % 8) return fail(RK_EINVAL, "%s: a stride is negative or no multiple of 8", name);
    if (a->ks.token < a->D || a->vs.token < a->D || a->ks.token >= 1 << 26 || a->vs.token >= 1 << 26)
        return fail(RK_EINVAL, "%s: a cache's token stride is below D or past 2^26", name);
    if (a->B == 0 || a->T == 0) return RK_OK;
    if (!attention_arrays(*a) || (a->n_blocks > 0 && (!a->k_cache || !a->v_cache))) return fail(RK_EINVAL, "%s: NULL array", name);
    if (((uintptr_t)a->q | (uintptr_t)a->out | (uintptr_t)a->k_cache | (uintptr_t)a->v_cache) % 16)
        return fail(RK_EINVAL, "%s: an array is not aligned to 16 bytes", name);
    return attention_call<false>(*a, nullptr, nullptr, workspace, ws_bytes, stream, name);
}

}  // extern "C"
