// attend_fp4.hip -- rk_prefix_attention_fp4: the entry points, and the kernels of caches held in 4 bits.
#include "attend.h"

using namespace rk;

extern "C" {

size_t rk_prefix_attention_fp4_workspace_size(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    int rc;
    if (attention_sizes(T, B, Hq, Hkv, D, &rc)) return 0;
    return attend_layout(T, B, Hq, Hkv, D).bytes;
}

int rk_prefix_attention_fp4(const rk_attention_fp4* a4, void* workspace, size_t ws_bytes, void* stream)
{
    const char* name = "rk_prefix_attention_fp4";
    if (!a4) return fail(RK_EINVAL, "%s: NULL arguments", name);
    const rk_attention& a = a4->a;
    if (int rc = attention_arguments(a, name)) return rc;
    const int32_t shares = (a.D + 31) / 32;
    for (const rk_fp4_cache& c : {a4->k, a4->v}) {
        if (!fp4_strides(c)) return fail(RK_EINVAL, "%s: a stride is negative, or one of codes no multiple of 16", name);
        if (c.cs.token < 16 * shares || c.ss.token < shares || c.cs.token >= 1 << 26 || c.ss.token >= 1 << 26)
            return fail(RK_EINVAL, "%s: a cache's token stride is below a row or past 2^26", name);
    }
    if (a.B == 0 || a.T == 0) return RK_OK;
    if (!attention_arrays(a) || (a.n_blocks > 0 && (!a4->k.codes || !a4->k.scales || !a4->v.codes || !a4->v.scales)))
        return fail(RK_EINVAL, "%s: NULL array", name);
    if (((uintptr_t)a.q | (uintptr_t)a.out | (uintptr_t)a4->k.codes | (uintptr_t)a4->v.codes) % 16)
        return fail(RK_EINVAL, "%s: an array is not aligned to 16 bytes", name);
    return attention_call<true>(a, &a4->k, &a4->v, workspace, ws_bytes, stream, name);
}

}  // extern "C"
