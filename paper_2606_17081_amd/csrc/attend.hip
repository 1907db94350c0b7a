// attend.hip -- attention of a step's new tokens over the block cache.
//
// out_t = sum_j w_j v_j / sum_j w_j, w_j = exp(scale q_t . k_j), in one pass over the keys: with m at least near the largest
// score so far, o = sum 2^(s_j - m) v_j and l = sum 2^(s_j - m) (scores in units of log2) are rescaled when m moves, and
// any split of the keys is joined by the same rule, o = sum_p 2^(m_p - m) o_p.  Both products run on matrix
// instructions; m, l, o and the scores are fp32.  The w_j of a step are rounded to the cache's 16 bits, the only operands that the
// instructions take: half a step of that type each, relative, so as much of the mean of |v| in a result (l sums them unrounded).
// fp16's range is narrow, so there m follows each step's own scores, down as well as up (`strays`): a key of far
// larger weight takes no bits from those after it.
//
// What bounds it: few rows (a decoding batch) the reading of keys and values, 4 D bytes a key and head for 4 D
// operations a row; from some hundred rows a key head on (a prompt, or a group on its prefix) the matrix instructions.  So there are tiles of two
// shapes, wide and narrow, and solo ones for what is short.  Kernels in a trace, the same inputs over and over: 128 requests on
// one prefix of 8,192 tokens (64 / 8 heads of 128) 66 + 10 us; prompts of 2,500-6,000 tokens 1.15-1.26 ms, 860-940 TFLOP/s;
// 5 requests of 60,000-131,072 tokens 193-199 us, 5.1 TB/s.
#include <hip/hip_runtime.h>

#include <math.h>

#include "rk_internal.h"

namespace rk {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kWaves = 4;
constexpr int32_t kLaunch = 1024;                    // requests of a launch: what is known of each is kept in LDS
constexpr int kWideRows = 128, kWideKeys = 64;       // a wide step: 32 rows a wavefront, 64 keys
constexpr int kNarrowRows = 32, kNarrowKeys = 128;   // a narrow step: 32 keys a wavefront
constexpr int kSoloKeys = 32, kSoloMost = 512;       // a narrow tile of so few keys is one wavefront's: 32 a step

// Kinds of tiles, each on a line of its own.
enum Kind { kWide, kNarrow, kSolo };
// What a step of a tile costs, and its beginning and end, relative to each other (a solo tile's to a wavefront, the others' to a
// workgroup): a wide or narrow step takes about 2 us, what comes before a wide tile's first and after its last 12 (a prologue without
// products, and results out).  Measured: ends of 4 for narrow and solo ones, 128 requests on one prefix 82 -> 87 us, of 8,
// groups of 200 62 -> 70; of 10 or 16 for wide ones, 0-5% more.  A piece of a line has at least kLeast, a step or more, so that a tile's
// parts follow each other without a gap.
constexpr uint32_t kStepCost[3] = {2, 2, 2}, kEndsCost[3] = {12, 6, 6};
constexpr uint32_t kLeast = 4;
static_assert(kLeast >= kStepCost[kWide] && kLeast >= kStepCost[kNarrow], "a step begins in every piece of a tile");
constexpr int kKeysOf[3] = {kWideKeys, kNarrowKeys, kSoloKeys};
constexpr int kJoinCost = 2;                         // of a request whose prefix and own keys are joined
constexpr float kLn2 = 0.69314718055994530942f, kLog2e = 1.44269504088896340736f;

// A tile that more than one workgroup worked on, as the workgroup that began it noted it; n = 0: none.
struct __align__(16) Split {
    int32_t n, wg, token, tokens, head, pad[3];
};

// A row of tables that shares its prefix: its parts, as the workgroup that began its tile noted them.
struct __align__(16) Parts {
    int32_t n, wg, row, pad;                 // n = 0: one part, in the shared rows' own place
};

// A request whose group attends to its prefix together: its first token, tokens (0: there is no such thing) and
// those of such requests before it.
struct __align__(16) Shared {
    int32_t q0, tokens, base, pad;
};

struct AttendArgs {
    rk_attention a;
    int32_t* status;
    int32_t b0, n;                           // the launch's requests: n from b0 on
    int32_t G, wide_tokens;                  // query heads of a key head, tokens of a wide tile
    uint32_t g_inverse;                      // 2^16 / G, rounded up
    int32_t solo_most;                       // most keys of a solo tile
    Split* split;                            // [grid]
    Shared* shared;                          // [n]: the requests' tokens that share a prefix
    Parts* parts;                            // [2][Hkv][shared tokens]
    // Rows of [DP] values, and their [2] statistics: first [2 grid][kWideRows], the first and last tile of each workgroup,
    // then [2][Hkv][shared rows], the whole tiles of rows that share a prefix.
    float *part, *part_ml;
    int32_t shared_rows, shared_tokens;      // of a head
};

// The first row of the whole tiles of a kind (prefixes: 0, requests' own keys: 1) and key head.
__device__ __forceinline__ int64_t whole_row(const AttendArgs& p, uint32_t grid, int kind, int32_t head)
{
    return 2 * (int64_t)grid * kWideRows + ((int64_t)kind * p.a.Hkv + head) * p.shared_rows;
}

template <bool Half>
__device__ __forceinline__ uint32_t pack16(float x, float y)
{
    if constexpr (Half) {
        return (uint32_t)__builtin_bit_cast(uint16_t, (_Float16)x) |
               ((uint32_t)__builtin_bit_cast(uint16_t, (_Float16)y) << 16);
    } else {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        bf2 v = {(__bf16)x, (__bf16)y};
        return __builtin_bit_cast(uint32_t, v);
    }
}

template <bool Half>
__device__ __forceinline__ float unpack16(uint32_t x)      // the low half
{
    if constexpr (Half) return (float)__builtin_bit_cast(_Float16, (uint16_t)x);
    else return __uint_as_float(x << 16);
}

template <bool Half>
__device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
{
    if constexpr (Half)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

template <bool Half>
__device__ __forceinline__ f32x4 mfma16(u32x4 a, u32x4 b, f32x4 c)
{
    if constexpr (Half)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
}

// 16-bit values of an exponent of all ones: infinities and NaN
template <bool Half>
constexpr uint32_t kExponent = Half ? 0x7c007c00u : 0x7f807f80u;

// x with a half of all-ones exponent replaced by 0
template <bool Half>
__device__ __forceinline__ uint32_t finite_or_zero(uint32_t x)
{
    const uint32_t e = kExponent<Half>;
    if ((x & e & 0xffffu) == (e & 0xffffu)) x &= 0xffff0000u;
    if ((x & e & 0xffff0000u) == (e & 0xffff0000u)) x &= 0xffffu;
    return x;
}

template <bool Half>
__device__ __forceinline__ bool not_finite(uint32_t x)
{
    const uint32_t e = kExponent<Half>;
    return (x & e & 0xffffu) == (e & 0xffffu) || (x & e & 0xffff0000u) == (e & 0xffff0000u);
}

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// The larger, half by half, of x and v's values without their signs: not finite if one of them is not.
__device__ __forceinline__ u16x2 without_sign(u16x2 x, u32x4 v)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x = __builtin_elementwise_max(x, __builtin_bit_cast(u16x2, v[i] & 0x7fff7fffu));
    return x;
}

// The 16-bit value x if it is not finite and its row sees it, else 0.
template <bool Half>
__device__ __forceinline__ float only_odd(bool sees, uint32_t x)
{
    return sees && not_finite<Half>(x) ? unpack16<Half>(x) : 0.0f;
}

typedef __attribute__((address_space(3))) uint8_t lds_u8;

__device__ __forceinline__ u32x4 lds_read16(uint32_t at)
{
    return *reinterpret_cast<__attribute__((address_space(3))) const u32x4*>((lds_u8*)(uintptr_t)at);
}
__device__ __forceinline__ u32x2 lds_read8(uint32_t at)
{
    return *reinterpret_cast<__attribute__((address_space(3))) const u32x2*>((lds_u8*)(uintptr_t)at);
}
__device__ __forceinline__ void lds_write16(uint32_t at, u32x4 x)
{
    *reinterpret_cast<__attribute__((address_space(3))) u32x4*>((lds_u8*)(uintptr_t)at) = x;
}
__device__ __forceinline__ void lds_write8(uint32_t at, u32x2 x)
{
    *reinterpret_cast<__attribute__((address_space(3))) u32x2*>((lds_u8*)(uintptr_t)at) = x;
}
// Four rows of 16 values, transposed: the 16 lanes of a group each name 8 bytes (lane j: row j / 4, values
// 4 (j % 4) ..), lane j gets value j of the four rows.
__device__ __forceinline__ u32x2 lds_read_columns(uint32_t at)
{
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                         (__attribute__((address_space(3))) s16x4*)(lds_u8*)(uintptr_t)at));
}

// x, in a way that what is computed from it stays where it is used: hoisted out of the loop over tiles, the
// addresses of all three kinds of tile would be held (and spilled) at once.
__device__ __forceinline__ int32_t afresh(int32_t x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// The larger number; NaN gives way to a number (and shows in the weights).
__device__ __forceinline__ float larger(float x, float y) { return fmaxf(x, y); }

// x, the same in all lanes, as the compiler then knows.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint64_t uniform(uint64_t x)
{
    return ((uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int32_t)(x >> 32)) << 32) |
           (uint32_t)__builtin_amdgcn_readfirstlane((int32_t)x);
}

// The workgroup's inclusive sums; tmp: 4 * kWaves words, the wavefronts' sums afterwards.
__device__ __forceinline__ void incl_sums(uint64_t (&x)[3], uint32_t& z, uint64_t* tmp)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        uint64_t ox[3];
        for (int k = 0; k < 3; ++k) ox[k] = __shfl_up(x[k], d);
        const uint32_t oz = __shfl_up(z, d);
        if (lane >= d) {
            for (int k = 0; k < 3; ++k) x[k] += ox[k];
            z += oz;
        }
    }
    if (lane == 63) {
        for (int k = 0; k < 3; ++k) tmp[kWaves * k + wave] = x[k];
        tmp[3 * kWaves + wave] = z;
    }
    __syncthreads();
    for (int w = 0; w < wave; ++w) {
        for (int k = 0; k < 3; ++k) x[k] += tmp[kWaves * k + w];
        z += (uint32_t)tmp[3 * kWaves + w];
    }
}

// a / b of numbers below 2^51 (a line has at most 2^31 / 64 tiles of 2^24 steps): the quotient in 64-bit floating point, correctly
// rounded, reaches the next whole number only if it is that, since what it lacks otherwise, 1 / b or more, is more than its rounding.
// (Integer division, long code with a branch for large numbers, takes 0.5 us more a call.)
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) { return (uint64_t)((double)a / (double)b); }
__device__ __forceinline__ uint64_t quotient_up(uint64_t a, uint64_t b) { return quotient(a + b - 1, b); }

// One tile's work, or a part of it: rows of the tokens [token, token + tokens) on key head `head`, steps [s0, s1).
struct Tile {
    const __attribute__((address_space(4))) int32_t* row;        // the block table's row
    int32_t block0;                          // first block of the segment
    int32_t keys_end;                        // first position that no row sees
    int32_t token, tokens, pos;              // of the first row's token
    int32_t head;
    int32_t s0, s1;
    bool mask;                               // rows see up to their own position (else up to keys_end)
    float *part, *part_ml;                   // where the result goes; NULL: to out and lse
};

template <int DP, bool Half>
struct Attend {
    static constexpr int kHead = DP;
    static constexpr int NC = DP / 8;                 // 16-byte pieces of a row
    static constexpr int NI = NC / 4;                 // loads of 64 pieces that bring a block
    static constexpr uint32_t kRow = DP * 2;          // bytes of a row in LDS
    static constexpr uint32_t kTileBytes = 512 * DP;  // LDS for keys and values

    // Row r of a block keeps its piece x at place x ^ turn(r), so that what a wavefront reads together lies in all of the
    // 256 bytes of banks: one piece of 16 rows (keys), two or four neighbouring ones of 8 or 4 rows (values).  The
    // rows' lengths turn rows of 128 or 384 bytes by half of that already.
    static constexpr int kTurn = NC % 16 == 0 ? 16 : 8;
    static __device__ __forceinline__ uint32_t turn(uint32_t r)
    {
        const uint32_t t = (r >> 1 & 1) << 2 | (r >> 2 & 1) << 1 | (r >> 3 & 1);
        return kTurn == 16 ? (r & 1) << 3 | t : t;
    }

    const AttendArgs& p;
    const uint32_t tile;                              // LDS address of the keys and values
    float* const join;                                // LDS: 2 * kWaves * kNarrowRows
    const int wave;
    const int32_t G;                                  // query heads of a key head
    const uint32_t g_inverse;                         // (exact quotients of a tile's rows: fewer than 2^7)
    const float c;                                    // |scale| log2(e)
    const uint32_t last_piece;                        // of a row: the bytes before it
    // the pieces of a block that the lane loads: whole rows a load, or not
    static constexpr bool kEven = 64 % NC == 0;
    uint32_t k_at[kEven ? 2 : NI], v_at[kEven ? 2 : NI];

    __device__ __forceinline__ Attend(const AttendArgs& args, uint32_t lds, float* j, float scale)
        : p(args), tile(lds), join(j), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)), G(args.G),
          g_inverse(args.g_inverse), c(scale),
          last_piece(2 * args.a.D - 16)
    {
        const int lane = threadIdx.x & 63;
        if constexpr (kEven) {
            const uint32_t r = lane / NC;
            k_at[0] = r * (uint32_t)p.a.ks.token * 2;
            v_at[0] = r * (uint32_t)p.a.vs.token * 2;
            k_at[1] = v_at[1] = 16 * ((uint32_t)(lane % NC) ^ turn(r));
        } else {
#pragma unroll
            for (int i = 0; i < NI; ++i) {
                const uint32_t x = 64 * i + lane, r = x / NC, piece = 16 * ((x % NC) ^ turn(r));
                k_at[i] = place(r * (uint32_t)p.a.ks.token * 2, piece);
                v_at[i] = place(r * (uint32_t)p.a.vs.token * 2, piece);
            }
        }
    }

    // The byte offset of a row's piece, or, of a piece behind D (of rows that D does not fill), one past any block's end, whose load
    // brings zeros: the query's are 0 there, and a product with anything that is not finite would not be.
    __device__ __forceinline__ uint32_t place(uint32_t row, uint32_t piece) const
    {
        return piece <= last_piece ? row + piece : 0x80000000u;
    }

    // The byte offset in a block of the piece that the lane loads i-th.
    __device__ __forceinline__ uint32_t offset(const uint32_t* at, int i, int64_t token) const
    {
        if constexpr (!kEven) {
            return at[i];
        } else {
            const uint32_t piece = at[1] ^ (16 * turn((uint32_t)i * (64 / NC)));
            return place(at[0] + (uint32_t)(i * (64 / NC)) * (uint32_t)token * 2, piece);
        }
    }

    // The block's `rows` first rows from base to LDS, zeros after them.  Straight to LDS, in flight until a wait for
    // vector memory; written as asm with no register result so that the compiler does not place that wait before
    // every LDS read.  The compiler sees no need of wait states inside it, so they stand there: one between the write of m0 and the
    // load that takes its place in LDS from it, and before the block's first load five after an instruction of the vector unit that may
    // have written the descriptor's registers (a readfirstlane, a spilled register's return).  (Five before every load: pieces
    // of prompts with D = 192 110 -> 114 us.)
    __device__ __forceinline__ void load_block(const uint16_t* base, int64_t stride, int32_t rows, const uint32_t* at,
                                               uint32_t lds) const
    {
        const uint64_t b = (uint64_t)base;
        u32x4 rsrc;
        rsrc.x = (uint32_t)b;
        rsrc.y = (uint32_t)(b >> 32) & 0xffffu;
        rsrc.z = rows > 0 ? (uint32_t)((rows - 1) * (int32_t)stride * 2 + p.a.D * 2) : 0u;
        rsrc.w = 0x00027000u;
        rsrc.x = __builtin_amdgcn_readfirstlane(rsrc.x);
        rsrc.y = __builtin_amdgcn_readfirstlane(rsrc.y);
        rsrc.z = __builtin_amdgcn_readfirstlane(rsrc.z);
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const uint32_t to = __builtin_amdgcn_readfirstlane(lds + 1024u * i);
            if (i == 0)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 3\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to),
                             "v"(offset(at, i, stride)), "s"(rsrc)
                             : "m0", "memory");
            else
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to),
                             "v"(offset(at, i, stride)), "s"(rsrc)
                             : "m0", "memory");
        }
    }

    // Block number `b`'s block of the segment's sequence, keys to k_lds, values to v_lds (either may be left out).
    // (read by scalar loads, whose wait is not the one of the keys and values under way)
    __device__ __forceinline__ int32_t block_id(const Tile& t, int32_t b) const
    {
        const int32_t last = (t.keys_end - 1) / RK_BLOCK_TOKENS;
        return t.row[b < last ? b : last];
    }
    __device__ __forceinline__ int32_t rows_of(const Tile& t, int32_t b, int32_t id) const
    {
        const int32_t n = t.keys_end - b * RK_BLOCK_TOKENS;
        return (uint32_t)id < (uint32_t)p.a.n_blocks ? (n < RK_BLOCK_TOKENS ? n : RK_BLOCK_TOKENS) : 0;
    }
    __device__ __forceinline__ void load_keys(const Tile& t, int32_t b, int32_t id, uint32_t lds) const
    {
        const int32_t rows = rows_of(t, b, id);
        load_block((const uint16_t*)p.a.k_cache + (rows > 0 ? (int64_t)id * p.a.ks.block : 0) + t.head * p.a.ks.head,
                   p.a.ks.token, rows, k_at, lds);
    }
    __device__ __forceinline__ void load_values(const Tile& t, int32_t b, int32_t id, uint32_t lds) const
    {
        const int32_t rows = rows_of(t, b, id);
        load_block((const uint16_t*)p.a.v_cache + (rows > 0 ? (int64_t)id * p.a.vs.block : 0) + t.head * p.a.vs.head,
                   p.a.vs.token, rows, v_at, lds);
    }
    // a block whose number is outside the cache
    __device__ __forceinline__ bool bad_block(int32_t id) const { return (uint32_t)id >= (uint32_t)p.a.n_blocks; }
    __device__ __forceinline__ void report_bad() const
    {
        if ((threadIdx.x & 63) == 0) atomicOr(p.status, RK_DEV_BAD_BLOCK);
    }

    __device__ __forceinline__ int32_t token_of(int32_t r) const { return (int32_t)((uint32_t)r * g_inverse >> 16); }

    // piece x of the row's query, its sign turned with the scale's
    __device__ __forceinline__ u32x4 query(const Tile& t, int32_t r, int32_t piece) const
    {
        u32x4 q = {0u, 0u, 0u, 0u};
        const int32_t tok = token_of(r);
        if (tok < t.tokens && 8 * piece < p.a.D) {
            q = *reinterpret_cast<const u32x4*>((const uint16_t*)p.a.q + (t.token + (int64_t)tok) * p.a.q_token +
                                                (t.head * G + r - tok * G) * p.a.q_head + 8 * piece);
            if (p.a.scale < 0.0f) q ^= 0x80008000u;
        }
        return q;
    }

    // Whether a step whose largest score is `top` asks for another divisor than 2^m of its weights.  bf16 has fp32's range: the divisor
    // follows only when the scores have left it behind by 2^8, so that results are seldom rescaled.  fp16 weights lose bits
    // below 2^-14, so there a step's largest is to lie in 2^-8..2^15: what a key below 2^-14 loses is 2^-25, 2^-17 of that
    // largest at most, and the 64 of a step 2^-11, half a step of fp16, whatever other steps hold.  Scores that rise are given 2^7, so
    // that a row's largest weight has that at least and the 64 lose 2^-26 of it, below fp16's smallest number; scores that fall,
    // the middle.  (With a divisor that only rises, a key of value 0 took all from 131,071 others that it stood e^18 above, and with 2^7
    // for the largest of all, 10% at e^20.)  Scores that spread by e^3 move it seldom, by e^8 in every step: prompts of
    // 2,500-6,000 tokens 1,114 -> 1,153 and 1,115 -> 1,226 us.
    static __device__ __forceinline__ bool strays(float top, float m)
    {
        if constexpr (Half) return !(fabsf(top - m - 3.5f) <= 11.5f);
        else return top > m + 8.0f;
    }
    // The new m, where the row's weights so far are `sum` in the old one's units.  Sums are kept below 2^48 or so: a key whose weight is
    // still too small there has no part in a 16-bit result.
    static __device__ __forceinline__ float divisor(float top, float m, float sum)
    {
        if constexpr (Half) {
            if (!(top > -INFINITY && strays(top, m))) return m;
            return top > m ? top - 7.0f : larger(top - 3.5f, m + __builtin_log2f(sum) - 48.0f);
        } else {
            return larger(m, top);
        }
    }

    __device__ __forceinline__ uint16_t* out_row(const Tile& t, int32_t r) const
    {
        const int32_t tok = token_of(r);
        return (uint16_t*)p.a.out + (t.token + (int64_t)tok) * p.a.out_token + (t.head * G + r - tok * G) * p.a.out_head;
    }
    __device__ __forceinline__ void put_lse(const Tile& t, int32_t r, float m, float l) const
    {
        const int32_t tok = token_of(r);
        if (p.a.lse)
            p.a.lse[(t.token + (int64_t)tok) * p.a.Hq + t.head * G + r - tok * G] =
                l == 0.0f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
    }

    // ---------------------------------------------------------------- up to 128 rows, 32 a wavefront
    //
    // Scores are computed transposed, keys x rows: a lane then holds 32 of the 64 scores of one row (lane
    // % 32) in registers, in the order in which the product with the values takes them: the row of
    // the value that lane half h multiplies with its j-th weight is the key whose score it holds.
    //
    // Bound by nothing alone: at D = 128 the two wavefronts of a SIMD have 2,048 cycles of matrix instructions a step, their CU's eight
    // 2,048 of LDS reads (32 KB each at 128 B a cycle), and 1,600 of vector instructions, two thirds of them for exponentials and
    // sums; on whole prompts the matrix units are busy for 43-52% of the cycles.  Rows of 64 a wavefront would halve the LDS
    // reads, but need 300 registers of the 256 that two wavefronts a SIMD have; one a SIMD (as for D > 128) reaches
    // half the rate: pieces of prompts with D = 192, 107 us for 52 GFLOP.  Conflicts of LDS banks are rare.
    // One prompt of 8,192 tokens, 64 / 8 heads of 128: 1.12 ms, 975 TFLOP/s.
    __device__ void wide(const Tile& t)
    {
        constexpr int KS = DP / 16, DT = DP / 32;
        const int lane = afresh(threadIdx.x & 63);
        const int hi = lane >> 5, r = 32 * wave + (lane & 31);
        int32_t last = t.keys_end - 1;               // the last position that the row sees
        if (t.mask) {
            const int32_t pos = t.pos + token_of(r);
            last = pos < last ? pos : last;
        }
        const int32_t all_see = t.mask ? (t.pos < t.keys_end - 1 ? t.pos : t.keys_end - 1) : t.keys_end - 1;
        f32x16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = f32x16{};
        float m = -INFINITY, l = 0.0f;               // m: log2 of the weights' common divisor
        // LDS addresses in a stage, less what the unrolled loops add
        uint32_t k_read[kTurn / 2], v_read[kTurn / 4];
        {
            const uint32_t row = lane & 31, vr = 4 * hi + ((lane & 15) >> 2), vp = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
            for (int x = 0; x < kTurn / 2; ++x) k_read[x] = row * kRow + (((2 * x + hi) ^ turn(row & 15)) << 4);
#pragma unroll
            for (int x = 0; x < kTurn / 4; ++x) v_read[x] = vr * kRow + (((4 * x + vp) ^ turn(vr)) << 4) + 8 * (lane & 1);
        }
        constexpr uint32_t kKeys = kWideKeys * kRow;   // bytes of a step's keys; two of them, then two steps' values
        // Keys come two steps ahead, values one: while a step's weights are computed, the products of the next step's
        // scores run beside them (whole prompts 1,440 -> 1,360 us).  Pieces are read from LDS kAhead products before the one that
        // takes them: 3 are as good, 6 spill registers (whole prompts 1,230 -> 1,500 us).
        constexpr int kAhead = 4, kPairs = 16;       // (a lane has 32 scores of a step: kPairs pairs)
        struct Step {
            int32_t own;                             // this wavefront's block
            uint32_t bad;                            // of the four blocks, those outside the cache
        };
        auto look = [&](int32_t x) {
            const int32_t b = t.block0 + 4 * x;
            const int32_t b0 = block_id(t, b), b1 = block_id(t, b + 1), b2 = block_id(t, b + 2), b3 = block_id(t, b + 3);
            Step e;
            e.own = uniform(wave < 2 ? (wave == 0 ? b0 : b1) : (wave == 2 ? b2 : b3));
            e.bad = (bad_block(b0) ? 1u : 0u) | (bad_block(b1) ? 2u : 0u) | (bad_block(b2) ? 4u : 0u) | (bad_block(b3) ? 8u : 0u);
            return e;
        };
        auto keys_at = [&](int32_t x) { return tile + ((x - t.s0) & 1) * kKeys; };
        auto values_at = [&](int32_t x) { return tile + 2 * kKeys + ((x - t.s0) & 1) * kKeys; };
        auto issue_keys = [&](int32_t x, const Step& e) {
            load_keys(t, t.block0 + 4 * x + wave, e.own, keys_at(x) + wave * (RK_BLOCK_TOKENS * kRow));
        };
        auto issue_values = [&](int32_t x, const Step& e) {
            load_values(t, t.block0 + 4 * x + wave, e.own, values_at(x) + wave * (RK_BLOCK_TOKENS * kRow));
        };
        // the x-th product's piece of the keys, or values, in a stage; what differs by constants is added by the reads
        struct Keys {
            uint32_t at[kTurn / 2];
        };
        struct Values {
            uint32_t at[kTurn / 4], at8[kTurn / 4];  // (of rows 8 further, less those rows)
        };
        auto keys_in = [&](uint32_t at) {
            Keys k;
#pragma unroll
            for (int x = 0; x < kTurn / 2; ++x) k.at[x] = at + k_read[x];
            return k;
        };
        auto values_in = [&](uint32_t at) {
            Values v;
#pragma unroll
            for (int x = 0; x < kTurn / 4; ++x) {
                v.at[x] = at + v_read[x];
                v.at8[x] = v.at[x] ^ 16 * turn(8);
            }
            return v;
        };
        auto key_piece = [&](const Keys& k, int x) {
            const int kt = x & 1, ks = x >> 1;
            return lds_read16(k.at[ks % (kTurn / 2)] + (uint32_t)(kt * 32 * kRow + ks / (kTurn / 2) * (16 * kTurn)));
        };
        auto value_piece = [&](const Values& v, int x) {
            constexpr int n = kTurn / 4;
            const int d = x % DT, kk = x / DT;
            const uint32_t y = (uint32_t)(d / n * (16 * kTurn) + 16 * kk * kRow);
            const u32x2 lo = lds_read_columns(v.at[d % n] + y), up = lds_read_columns(v.at8[d % n] + y + 8 * kRow);
            return u32x4{lo.x, lo.y, up.x, up.y};
        };
        u32x4 q[KS];
        auto scores = [&](uint32_t stage, f32x16* sc) {
            const Keys at = keys_in(stage);
            u32x4 k[kAhead];
            sc[0] = sc[1] = f32x16{};
#pragma unroll
            for (int x = 0; x < kAhead; ++x) k[x] = key_piece(at, x);
#pragma unroll
            for (int x = 0; x < 2 * KS; ++x) {
                sc[x & 1] = mfma32<Half>(k[x % kAhead], q[x >> 1], sc[x & 1]);
                if (x + kAhead < 2 * KS) k[x % kAhead] = key_piece(at, x + kAhead);
            }
        };
        auto highest = [&](const f32x16* sc) {
            float top = sc[0][0];
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = larger(top, sc[kt][i]);
            return top;
        };
        auto follow = [&](float top) {
            if (__any(strays(top * c, m))) {
                top = larger(top, __shfl_xor(top, 32)) * c;
                const float nm = divisor(top, m, Half ? l + __shfl_xor(l, 32) : 0.0f);
                const float keep = nm == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - nm);
                m = nm;
                l *= keep;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= keep;
            }
            return m == -INFINITY ? 0.0f : -m;
        };
        auto exponent = [&](const f32x16* sc, int x, int e, float base) {
            return __builtin_fmaf(sc[x >> 3][2 * (x & 7) + e], c, base);
        };
        auto weight = [&](u32x4* w, int x, float a, float b) {
            l += a + b;
            w[x >> 2][x & 3] = pack16<Half>(a, b);
        };
        // A step whose keys every row sees: sc its scores, top their largest; the next step's into nx.
        auto open_step = [&](int32_t x, const f32x16* sc, f32x16* nx, float& top) {
            const float base = follow(top);
            const Keys ka = keys_in(keys_at(x + 1));
            constexpr int n = 2 * KS;
            u32x4 k[kAhead], w[4];
            nx[0] = nx[1] = f32x16{};
#pragma unroll
            for (int u = 0; u < kAhead; ++u) k[u] = key_piece(ka, u);
            float fa = exponent(sc, 0, 0, base), fb = exponent(sc, 0, 1, base), ea = 0.0f, eb = 0.0f;
#pragma unroll
            for (int u = 0; u < n; ++u) {
                __builtin_amdgcn_sched_barrier(0);
                nx[u & 1] = mfma32<Half>(k[u % kAhead], q[u >> 1], nx[u & 1]);
                if (u + kAhead < n) k[u % kAhead] = key_piece(ka, u + kAhead);
#pragma unroll
                for (int y = u * kPairs / n; y < (u + 1) * kPairs / n; ++y) {
                    const float na = __builtin_amdgcn_exp2f(fa), nb = __builtin_amdgcn_exp2f(fb);
                    if (y + 1 < kPairs) {
                        fa = exponent(sc, y + 1, 0, base);
                        fb = exponent(sc, y + 1, 1, base);
                    }
                    if (y > 0) weight(w, y - 1, ea, eb);
                    ea = na;
                    eb = nb;
                }
            }
            // (a wavefront in this product goes first: the other on its SIMD has its weights to compute meanwhile;
            // whole prompts 1,251 -> 1,214 us)
            __builtin_amdgcn_s_setprio(1);
            const Values va = values_in(values_at(x));
            u32x4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = value_piece(va, u);
            weight(w, kPairs - 1, ea, eb);
            top = nx[0][0];
#pragma unroll
            for (int u = 0; u < 4 * DT; ++u) {
                __builtin_amdgcn_sched_barrier(0);
                o[u % DT] = mfma32<Half>(v[u % kAhead], w[u / DT], o[u % DT]);
                if (u + kAhead < 4 * DT) v[u % kAhead] = value_piece(va, u + kAhead);
#pragma unroll
                for (int y = u * 32 / (4 * DT); y < (u + 1) * 32 / (4 * DT); ++y) top = larger(top, nx[y >> 4][y & 15]);
            }
            __builtin_amdgcn_s_setprio(0);
        };
        int32_t s = t.s0;
        Step now, next, then;
        // Step s + 1's keys and step s's values are there, and everyone has read what came before; the loads of those
        // after them begin.
        auto arrive = [&]() {
            __builtin_amdgcn_s_waitcnt(0);
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
            if (s + 1 < t.s1) {
                issue_values(s + 1, next);
                if (s + 2 < t.s1) issue_keys(s + 2, then);
            }
        };
        auto advance = [&]() {
            ++s;
            now = next;
            next = then;
            then = look(s + 2);
        };
        now = look(s);
        next = look(s + 1);
        then = look(s + 2);
        __syncthreads();                             // the LDS is the last tile's until here
        issue_keys(s, now);
        issue_values(s, now);
        if (s + 1 < t.s1) issue_keys(s + 1, next);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = query(t, r, 2 * ks + hi);
        __builtin_amdgcn_s_waitcnt(0);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        f32x16 sa[2], sb[2];
        scores(keys_at(s), sa);
        // the steps whose keys every row sees, if their blocks are good, but the last
        const int32_t open = (all_see + 1 - t.block0 * RK_BLOCK_TOKENS) / kWideKeys, s_open = open < t.s1 - 1 ? open : t.s1 - 1;
        float top = highest(sa);
        while (s + 1 < s_open && !(now.bad | next.bad)) {
            arrive();
            open_step(s, sa, sb, top);
            advance();
            arrive();
            open_step(s, sb, sa, top);
            advance();
        }
        for (;;) {
            arrive();
            const int32_t key0 = (t.block0 + 4 * s) * RK_BLOCK_TOKENS;
            const bool masked = key0 + kWideKeys - 1 > all_see;
            if (masked || now.bad) {
                if (now.bad) report_bad();
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int x = 32 * kt + 8 * (i >> 2) + 4 * hi + (i & 3);
                        if (key0 + x > last || ((now.bad >> (x >> 4)) & 1)) sa[kt][i] = -INFINITY;
                    }
            }
            const float base = follow(highest(sa));
            u32x4 w[4];
#pragma unroll
            for (int x = 0; x < kPairs; ++x)
                weight(w, x, __builtin_amdgcn_exp2f(exponent(sa, x, 0, base)), __builtin_amdgcn_exp2f(exponent(sa, x, 1, base)));
            const uint32_t va = values_at(s);
            if (masked && t.mask) {
                // A value that is not finite must not meet the weight of 0 of a row that does not see it: such values
                // are added to the rows that do, and are 0 in the product.  (All wavefronts decide alike.)
                u16x2 most = {0, 0};
#pragma unroll 4
                for (int x = lane; x < kWideKeys * NC; x += 64) most = without_sign(most, lds_read16(va + 16 * x));
                if (__any(not_finite<Half>(__builtin_bit_cast(uint32_t, most)))) {
#pragma unroll 1
                    for (int x = 0; x < kWideKeys; ++x) {
                        const bool sees = key0 + x <= last;
#pragma unroll
                        for (int d = 0; d < DT; ++d)
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                __builtin_amdgcn_sched_barrier(0);
                                const uint32_t piece = (uint32_t)(4 * d + g) ^ turn(x & 15);
                                const u32x2 v = lds_read8(va + x * kRow + (piece << 4) + 8 * hi);
                                o[d][4 * g] += only_odd<Half>(sees, v.x & 0xffffu);
                                o[d][4 * g + 1] += only_odd<Half>(sees, v.x >> 16);
                                o[d][4 * g + 2] += only_odd<Half>(sees, v.y & 0xffffu);
                                o[d][4 * g + 3] += only_odd<Half>(sees, v.y >> 16);
                            }
                    }
                    __builtin_amdgcn_s_waitcnt(0xc07f);              // (lgkmcnt 0: loads to LDS stay under way)
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    for (int x = 64 * wave + lane; x < kWideKeys * NC; x += kThreads) {
                        const u32x4 v = lds_read16(va + 16 * x);
                        lds_write16(va + 16 * x, u32x4{finite_or_zero<Half>(v.x), finite_or_zero<Half>(v.y),
                                                       finite_or_zero<Half>(v.z), finite_or_zero<Half>(v.w)});
                    }
                    __builtin_amdgcn_s_waitcnt(0xc07f);
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                }
            }
            const Values vs = values_in(va);
            u32x4 v[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) v[u] = value_piece(vs, u);
#pragma unroll
            for (int u = 0; u < 4 * DT; ++u) {
                __builtin_amdgcn_sched_barrier(0);
                o[u % DT] = mfma32<Half>(v[u % kAhead], w[u / DT], o[u % DT]);
                if (u + kAhead < 4 * DT) v[u % kAhead] = value_piece(vs, u + kAhead);
            }
            if (s + 1 >= t.s1) break;
            scores(keys_at(s + 1), sa);
            advance();
        }
        l += __shfl_xor(l, 32);
        // Out through LDS, so that whole rows are written: a lane's own pieces of a row are 8 or 16 bytes each, of 32 rows at a
        // time.  The keys' stages are free: everyone has read the last keys.
        const uint32_t mine = tile + wave * (32 * kRow);
        const int32_t rows = t.tokens * G - 32 * wave;
        const int late = afresh(lane);
        auto written = [&](auto&& put) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int i = 0; i < NC / 2; ++i) {
                const int x = 64 * i + late, row = x / NC, piece = x % NC;
                const u32x4 v = lds_read16(mine + row * kRow + ((piece ^ turn(row & 15)) << 4));
                if (row < rows) put(row, piece, v);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        };
        const uint32_t row_at = mine + (late & 31) * kRow, turned = turn(late & 15);
        if (t.part) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int d = 0; d < DT / 2; ++d)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x16& y = o[half * (DT / 2) + d];
                        lds_write16(row_at + (((8 * d + 2 * g + hi) ^ turned) << 4),
                                    __builtin_bit_cast(u32x4, f32x4{y[4 * g], y[4 * g + 1], y[4 * g + 2], y[4 * g + 3]}));
                    }
                float* to = t.part + (int64_t)(32 * wave) * DP + half * (DP / 2);
                written([&](int row, int piece, u32x4 v) { *reinterpret_cast<u32x4*>(to + row * DP + 4 * piece) = v; });
            }
            if (hi == 0 && (lane & 31) < rows) {
                t.part_ml[2 * r] = m;
                t.part_ml[2 * r + 1] = l;
            }
        } else {
            const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    lds_write8(row_at + (((4 * d + g) ^ turned) << 4) + 8 * hi,
                               u32x2{pack16<Half>(o[d][4 * g] * inv, o[d][4 * g + 1] * inv),
                                     pack16<Half>(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv)});
            written([&](int row, int piece, u32x4 v) {
                if (8 * piece < p.a.D) *reinterpret_cast<u32x4*>(out_row(t, 32 * wave + row) + 8 * piece) = v;
            });
            if (hi == 0 && (lane & 31) < rows) put_lse(t, r, m, l);
        }
    }

    // ---------------------------------------------------------------- up to 16 NQ rows, 32 keys a wavefront
    //
    // What bounds few rows is the reading of keys and values, so each wavefront takes keys of its own, with no
    // barrier: while it computes on the keys of a step its values are still under way, and the next step's keys
    // follow as soon as this step's are in registers.  The wavefronts' results are joined through LDS; of few keys a
    // wavefront does a tile alone.  Measured: 5 requests of 60,000-131,072 tokens, 16 / 4 heads of 128, 198 us for 1.01 GB, 5.1 TB/s; 128 of
    // 2,048 tokens, 8 key heads, 215 us, 5.0 TB/s; one of 8,192 tokens 21 us, of 100 tokens 12 us, both waits one after the
    // other (lengths, block numbers, keys, join).  (Kernels in a trace.)
    template <int NQ, bool Solo>
    __device__ void narrow(const Tile& t)
    {
        constexpr int KS = DP / 32, DT = DP / 16;
        const int lane = afresh(threadIdx.x & 63);
        const int g = lane >> 4, col = lane & 15;
        u32x4 q[NQ][KS];
        int32_t last[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int32_t r = 16 * n + col;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[n][ks] = query(t, r, 4 * ks + g);
            last[n] = t.keys_end - 1;
            if (t.mask) {
                const int32_t pos = t.pos + token_of(r);
                last[n] = pos < last[n] ? pos : last[n];
            }
        }
        const int32_t all_see = t.mask ? (t.pos < t.keys_end - 1 ? t.pos : t.keys_end - 1) : t.keys_end - 1;
        f32x4 o[NQ][DT];
        float m[NQ], l[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
#pragma unroll
            for (int d = 0; d < DT; ++d) o[n][d] = f32x4{};
            m[n] = -INFINITY;
            l[n] = 0.0f;
        }
        uint32_t k_read[kTurn / 4], v_read[kTurn / 2];
#pragma unroll
        for (int x = 0; x < kTurn / 4; ++x) k_read[x] = col * kRow + (((4 * x + g) ^ turn(col)) << 4);
        {
            const uint32_t vr = 4 * g + (col >> 2);
#pragma unroll
            for (int x = 0; x < kTurn / 2; ++x)
                v_read[x] = vr * kRow + (((2 * x + ((lane & 3) >> 1)) ^ turn(vr)) << 4) + 8 * (lane & 1);
        }
        const uint32_t keys = tile + wave * (64 * kRow), vals = keys + 32 * kRow;
        // this wavefront's steps: 32 keys at 128 s + 32 wave, or all of them
        constexpr int kKeys = Solo ? kSoloKeys : kNarrowKeys, kBlocks = kKeys / RK_BLOCK_TOKENS;
        const int32_t first_block = t.block0 + (Solo ? 0 : 2 * wave);
        int32_t s1 = (t.keys_end - first_block * RK_BLOCK_TOKENS + kKeys - 1) / kKeys;
        s1 = s1 < t.s1 ? s1 : t.s1;
        int32_t s = t.s0, id[2], later[2];
        auto ids = [&](int32_t* to, int32_t x) {
#pragma unroll
            for (int b = 0; b < 2; ++b) to[b] = block_id(t, first_block + kBlocks * x + b);
        };
        uint32_t bad = 0, next_bad = 0;
        auto issue_keys = [&](int32_t x) {
            next_bad = 0;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                load_keys(t, first_block + kBlocks * x + b, id[b], keys + b * (RK_BLOCK_TOKENS * kRow));
                next_bad |= (bad_block(id[b]) ? 1u : 0u) << b;
            }
        };
        auto issue_values = [&](int32_t x) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
                load_values(t, first_block + kBlocks * x + b, id[b], vals + b * (RK_BLOCK_TOKENS * kRow));
        };
        auto scores = [&](f32x4 (*sc)[2]) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) sc[n][kt] = f32x4{};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const u32x4 k = lds_read16(keys + k_read[ks % (kTurn / 4)] +
                                               (uint32_t)(kt * 16 * kRow + ks / (kTurn / 4) * (16 * kTurn)));
#pragma unroll
                    for (int n = 0; n < NQ; ++n) sc[n][kt] = mfma16<Half>(k, q[n][ks], sc[n][kt]);
                }
            }
        };
        auto weights = [&](f32x4 (*sc)[2], u32x4* w) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float top = sc[n][0][0];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) top = larger(top, sc[n][kt][i]);
                if (__any(strays(top * c, m[n]))) {
                    top = larger(top, __shfl_xor(top, 16));
                    top = larger(top, __shfl_xor(top, 32)) * c;
                    float sum = 0.0f;
                    if constexpr (Half) {
                        sum = l[n] + __shfl_xor(l[n], 16);
                        sum += __shfl_xor(sum, 32);
                    }
                    const float nm = divisor(top, m[n], sum);
                    const float keep = nm == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m[n] - nm);
                    m[n] = nm;
                    l[n] *= keep;
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[n][d] *= keep;
                }
                const float base = m[n] == -INFINITY ? 0.0f : -m[n];
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kt][i], c, base));
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kt][i + 1], c, base));
                        l[n] += x + y;
                        w[n][2 * kt + (i >> 1)] = pack16<Half>(x, y);
                    }
            }
        };
        auto values = [&](int d) {
            const uint32_t x = vals + v_read[d % (kTurn / 2)] + (uint32_t)(d / (kTurn / 2) * (16 * kTurn));
            const u32x2 lo = lds_read_columns(x), up = lds_read_columns(x + 16 * kRow);
            return u32x4{lo.x, lo.y, up.x, up.y};
        };
        // (vector memory operations end in the order of their issue: the step's keys are there when only its values'
        // loads are under way, its values when only the next keys' are)
        auto wait_keys = [&]() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory"); };
        auto keys_read = [&]() {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the keys are in registers
            bad = next_bad;
            if (s + 1 < s1) {
                id[0] = later[0];
                id[1] = later[1];
                issue_keys(s + 1);
                ids(later, s + 2);
            }
        };
        auto wait_values = [&]() {
            if (s + 1 < s1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * NI) : "memory");
            else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        };
        auto values_read = [&]() {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the values are in registers
            if (s + 1 < s1) issue_values(s + 1);
        };
        if constexpr (Solo) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the LDS is the last tile's until here
        else __syncthreads();
        if (s < s1) {
            ids(id, s);
            issue_keys(s);
            issue_values(s);
            ids(later, s + 1);
        }
        const int32_t seen = all_see + 1 - first_block * RK_BLOCK_TOKENS - 32;       // the last step's first key that all see
        const int32_t open = seen < 0 ? 0 : seen / kKeys + 1, s_open = open < s1 ? open : s1;
        for (; s < s_open && !next_bad; ++s) {
            f32x4 sc[NQ][2];
            u32x4 w[NQ];
            wait_keys();
            scores(sc);
            keys_read();
            weights(sc, w);
            wait_values();
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x4 v = values(d);
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][d] = mfma16<Half>(v, w[n], o[n][d]);
            }
            values_read();
        }
        for (; s < s1; ++s) {
            const int32_t key0 = (first_block + kBlocks * s) * RK_BLOCK_TOKENS;
            const bool masked = key0 + 31 > all_see;
            f32x4 sc[NQ][2];
            u32x4 w[NQ];
            wait_keys();
            scores(sc);
            keys_read();
            if (bad) report_bad();
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + 16 * kt + 4 * g + i > last[n] || ((bad >> kt) & 1)) sc[n][kt][i] = -INFINITY;
            weights(sc, w);
            wait_values();
            if (masked && t.mask && t.tokens > 1) {                      // (as for wide tiles, of values of the wavefront's own)
                u16x2 most = {0, 0};
#pragma unroll 4
                for (int x = lane; x < 32 * NC; x += 64) most = without_sign(most, lds_read16(vals + 16 * x));
                if (__any(not_finite<Half>(__builtin_bit_cast(uint32_t, most)))) {
#pragma unroll 1
                    for (int x = 0; x < 32; ++x)
#pragma unroll
                        for (int d = 0; d < DT; ++d) {
                            __builtin_amdgcn_sched_barrier(0);
                            const uint32_t piece = (uint32_t)(2 * d + (g >> 1)) ^ turn(x & 15);
                            const u32x2 v = lds_read8(vals + x * kRow + (piece << 4) + 8 * (g & 1));
#pragma unroll
                            for (int n = 0; n < NQ; ++n) {
                                const bool sees = key0 + x <= last[n];
                                o[n][d][0] += only_odd<Half>(sees, v.x & 0xffffu);
                                o[n][d][1] += only_odd<Half>(sees, v.x >> 16);
                                o[n][d][2] += only_odd<Half>(sees, v.y & 0xffffu);
                                o[n][d][3] += only_odd<Half>(sees, v.y >> 16);
                            }
                        }
                    for (int x = lane; x < 32 * NC; x += 64) {
                        const u32x4 v = lds_read16(vals + 16 * x);
                        lds_write16(vals + 16 * x, u32x4{finite_or_zero<Half>(v.x), finite_or_zero<Half>(v.y),
                                                         finite_or_zero<Half>(v.z), finite_or_zero<Half>(v.w)});
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            }
#pragma unroll
            for (int d = 0; d < DT; ++d) {
                const u32x4 v = values(d);
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][d] = mfma16<Half>(v, w[n], o[n][d]);
            }
            values_read();
        }
        constexpr int kRows = 16 * NQ;
        if constexpr (Solo) {
            // out through LDS, as of wide tiles; all of it is free
            const int32_t rows = t.tokens * G;
            const int late = afresh(lane);
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                l[n] += __shfl_xor(l[n], 16);
                l[n] += __shfl_xor(l[n], 32);
            }
            auto written = [&](auto&& put) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
                for (int i = 0; i < kRows * NC / 64; ++i) {
                    const int x = 64 * i + late, row = x / NC, piece = x % NC;
                    const u32x4 v = lds_read16(keys + row * kRow + ((piece ^ turn(row & 15)) << 4));
                    if (row < rows) put(row, piece, v);
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            };
            const uint32_t row_at = keys + (late & 15) * kRow, turned = turn(late & 15);
            if (t.part) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
#pragma unroll
                    for (int n = 0; n < NQ; ++n)
#pragma unroll
                        for (int d = 0; d < DT / 2; ++d)
                            lds_write16(row_at + 16 * n * kRow + (((4 * d + g) ^ turned) << 4),
                                        __builtin_bit_cast(u32x4, o[n][half * (DT / 2) + d]));
                    float* to = t.part + half * (DP / 2);
                    written([&](int row, int piece, u32x4 v) { *reinterpret_cast<u32x4*>(to + row * DP + 4 * piece) = v; });
                }
            } else {
#pragma unroll
                for (int n = 0; n < NQ; ++n) {
                    const float inv = l[n] == 0.0f ? 0.0f : 1.0f / l[n];
#pragma unroll
                    for (int d = 0; d < DT; ++d) {
                        const f32x4 y = o[n][d] * inv;
                        lds_write8(row_at + 16 * n * kRow + (((2 * d + (g >> 1)) ^ turned) << 4) + 8 * (g & 1),
                                   u32x2{pack16<Half>(y.x, y.y), pack16<Half>(y.z, y.w)});
                    }
                }
                written([&](int row, int piece, u32x4 v) {
                    if (8 * piece < p.a.D) *reinterpret_cast<u32x4*>(out_row(t, row) + 8 * piece) = v;
                });
            }
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                const int32_t r = 16 * n + col;
                if (g != 0 || r >= rows) continue;
                if (t.part) {
                    t.part_ml[2 * r] = m[n];
                    t.part_ml[2 * r + 1] = l[n];
                } else {
                    put_lse(t, r, m[n], l[n]);
                }
            }
            return;
        }
        // the four wavefronts' results: rows of DP floats in LDS, wavefront after wavefront
        __syncthreads();
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            l[n] += __shfl_xor(l[n], 16);
            l[n] += __shfl_xor(l[n], 32);
            if (g == 0) {
                join[2 * (wave * kRows + 16 * n + col)] = m[n];
                join[2 * (wave * kRows + 16 * n + col) + 1] = l[n];
            }
#pragma unroll
            for (int d = 0; d < DT; ++d)
                *reinterpret_cast<__attribute__((address_space(3))) f32x4*>(
                    (lds_u8*)(uintptr_t)(tile + 4 * ((wave * kRows + 16 * n + col) * DP + 16 * d + 4 * g))) = o[n][d];
        }
        __syncthreads();
        const int32_t rows = t.tokens * G;
        for (int x = 64 * wave + lane; x < kRows * (DP / 8); x += kThreads) {
            const int r = x / (DP / 8), piece = x % (DP / 8);
            if (r >= rows) continue;
            float mm[kWaves], nm = -INFINITY, total = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) nm = larger(nm, mm[w] = join[2 * (w * kRows + r)]);
            f32x4 a = {}, b = {};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = mm[w] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(mm[w] - nm);
                total += f * join[2 * (w * kRows + r) + 1];
                const uint32_t at = tile + 4 * ((w * kRows + r) * DP + 8 * piece);
                if (f != 0.0f) {
                    a += f * *reinterpret_cast<__attribute__((address_space(3))) f32x4*>((lds_u8*)(uintptr_t)at);
                    b += f * *reinterpret_cast<__attribute__((address_space(3))) f32x4*>((lds_u8*)(uintptr_t)(at + 16));
                }
            }
            if (t.part) {
                *reinterpret_cast<f32x4*>(t.part + (int64_t)r * DP + 8 * piece) = a;
                *reinterpret_cast<f32x4*>(t.part + (int64_t)r * DP + 8 * piece + 4) = b;
                if (piece == 0) {
                    t.part_ml[2 * r] = nm;
                    t.part_ml[2 * r + 1] = total;
                }
            } else {
                const float inv = total == 0.0f ? 0.0f : 1.0f / total;
                if (8 * piece < p.a.D)
                    *reinterpret_cast<u32x4*>(out_row(t, r) + 8 * piece) =
                        u32x4{pack16<Half>(a.x * inv, a.y * inv), pack16<Half>(a.z * inv, a.w * inv),
                              pack16<Half>(b.x * inv, b.y * inv), pack16<Half>(b.z * inv, b.w * inv)};
                if (piece == 0) put_lse(t, r, nm, total);
            }
        }
    }
};

// What a workgroup keeps of each request, in LDS.
struct Request {
    int32_t kv, q0, tokens;                  // tokens = 0: nothing to do
    int32_t shared;                          // blocks of the prefix that its group attends to together; 0: none
    int32_t end;                             // of the first that shares: the group's end; else 0
    int32_t base;                            // shared tokens before its own
};

// A segment's extent along the line of work: the tokens of one request over its own keys, or those of a group over
// its prefix, for one key head.  Wide segments of a request run over tiles whose keys grow with the position,
// paired first with last so that every pair takes the same.
struct Segment {
    int32_t tokens, rows, tiles, per;        // tokens in all, rows in all, tiles, tokens of a tile
    int32_t steps0;                          // steps of a tile (of the first, where they grow)
    int kind;
    bool grows;
    uint64_t pair, cost;                     // cost of a pair (or tile), and in all
};

__device__ __forceinline__ int32_t steps_for(int64_t keys, int kind)
{
    const int32_t per = kind == kWide ? kKeysOf[kWide] : kind == kNarrow ? kKeysOf[kNarrow] : kKeysOf[kSolo];
    return keys > 0 ? (int32_t)((keys + per - 1) / per) : 1;
}

// A tile's extent along the line (its steps, one after the other, then its ends' cost), and the steps of it that begin in its first
// `length`.  A solo tile is not cut: it belongs where it starts.
__device__ __forceinline__ uint64_t extent(int32_t steps, int kind)
{
    return kind == kWide ? kEndsCost[kWide] + (uint64_t)steps * kStepCost[kWide]
         : kind == kNarrow ? kEndsCost[kNarrow] + (uint64_t)steps * kStepCost[kNarrow]
                           : kEndsCost[kSolo] + (uint64_t)steps * kStepCost[kSolo];
}
template <int K>
__device__ __forceinline__ int32_t steps_before(uint64_t length, int32_t steps)
{
    if (K == kSolo) return length == 0 ? 0 : steps;
    const uint64_t n = quotient_up(length, kStepCost[K]);
    return n < (uint64_t)steps ? (int32_t)n : steps;
}

__device__ __forceinline__ Segment own_segment(const Request& r, const AttendArgs& p)
{
    Segment s{};
    s.tokens = r.tokens;
    s.rows = r.tokens * p.G;
    const int64_t own = (int64_t)r.kv - (int64_t)r.shared * RK_BLOCK_TOKENS;
    s.kind = s.rows > kNarrowRows ? kWide : own > p.solo_most ? kNarrow : kSolo;
    s.per = s.kind == kWide ? p.wide_tokens : s.tokens;
    if (s.tokens == 0) return s;
    s.tiles = (s.tokens + s.per - 1) / s.per;
    if (s.tiles == 1) {
        s.steps0 = steps_for(own, s.kind);
        s.pair = s.cost = extent(s.steps0, s.kind);
    } else {
        s.grows = true;
        s.steps0 = steps_for(own - s.tokens + s.per, kWide);
        const int32_t last = steps_for(own - s.tokens + (int64_t)s.tiles * s.per, kWide);
        s.pair = extent(s.steps0, kWide) + extent(last, kWide) + 2 * kStepCost[kWide];
        s.cost = s.pair * ((s.tiles + 1) / 2);
    }
    return s;
}

__device__ __forceinline__ Segment prefix_segment(int32_t tokens, int32_t blocks, const AttendArgs& p)
{
    Segment s{};
    s.tokens = tokens;
    s.rows = tokens * p.G;
    s.kind = s.rows > kNarrowRows ? kWide : blocks * RK_BLOCK_TOKENS > p.solo_most ? kNarrow : kSolo;
    s.per = s.kind == kWide ? p.wide_tokens : s.tokens;
    s.tiles = (s.tokens + s.per - 1) / s.per;
    s.steps0 = steps_for((int64_t)blocks * RK_BLOCK_TOKENS, s.kind);
    s.pair = extent(s.steps0, s.kind);
    s.cost = s.pair * s.tiles;
    return s;
}

// A workgroup's piece [from, to) of the line of tiles of kind K (of solo tiles: a wavefront's), from place `off` of
// request i's part on; wg: the workgroup's place among all.
template <int K, class A>
__device__ __forceinline__ void walk(A& work, const Request* req, int32_t i, uint64_t off, uint64_t from, uint64_t to,
                                     uint64_t each, int32_t wg)
{
    const AttendArgs& p = work.p;
    const rk_attention& a = p.a;
    const int32_t G = work.G, B = p.n;
    const int32_t tid = K == kSolo ? threadIdx.x & 63 : threadIdx.x, crew = K == kSolo ? 64 : kThreads;
    constexpr int DP = A::kHead;
    uint64_t x = from;
    while (x < to && i < B) {
        Request r = req[i];
        r.kv = uniform(r.kv);
        r.q0 = uniform(r.q0);
        r.tokens = uniform(r.tokens);
        r.shared = uniform(r.shared);
        r.end = uniform(r.end);
        r.base = uniform(r.base);
        Segment sg;
        bool prefix = false;
        uint64_t before = 0;
        if (r.end) {
            sg = prefix_segment(uniform(req[r.end - 1].q0 + req[r.end - 1].tokens) - r.q0, r.shared, p);
            before = sg.kind == K ? sg.cost * (uint64_t)a.Hkv : 0;
            prefix = off < before;
        }
        if (!prefix) {
            sg = own_segment(r, p);
            const uint64_t own = sg.kind == K ? sg.cost * (uint64_t)a.Hkv : 0;
            off -= before;
            if (off >= own) {                // on to the next request
                off -= own;
                ++i;
                continue;
            }
        }
        const int32_t head = (int32_t)quotient(off, sg.cost);
        uint64_t in = off - (uint64_t)head * sg.cost;              // place in the head's part
        int32_t j = (int32_t)quotient(in, sg.pair);
        in -= (uint64_t)j * sg.pair;
        int32_t steps = sg.steps0;
        uint64_t left = sg.pair;             // cost from the tile's start to the next tile's
        bool nothing = false;
        if (K == kWide && sg.grows) {
            auto steps_of = [&](int32_t k) {
                const int64_t seen = (int64_t)(k + 1) * sg.per < sg.tokens ? (int64_t)(k + 1) * sg.per : sg.tokens;
                return steps_for((int64_t)r.kv - (int64_t)r.shared * RK_BLOCK_TOKENS - sg.tokens + seen, kWide);
            };
            const int32_t k = sg.tiles - 1 - j;
            const uint64_t first = extent(steps_of(j), kWide);
            steps = steps_of(j);
            left = first;
            if (in >= first) {               // the pair's other tile
                in -= first;
                left = sg.pair - first;
                nothing = k == j;
                j = k;
                steps = steps_of(k);
            }
        }
        // the steps of the tile that begin in [from, to)
        const int32_t s0 = steps_before<K>(in, steps), s1 = steps_before<K>(to - x + in, steps);
        if (!nothing && s0 < s1) {
            Tile t;
            t.token = r.q0 + j * sg.per;
            t.tokens = sg.tokens - j * sg.per < sg.per ? sg.tokens - j * sg.per : sg.per;
            t.head = head;
            t.s0 = s0;
            t.s1 = s1;
            t.mask = !prefix;
            t.row = (const __attribute__((address_space(4))) int32_t*)(a.tables + (int64_t)(p.b0 + i) * a.table_stride);
            if (prefix) {
                t.block0 = 0;
                t.keys_end = r.shared * RK_BLOCK_TOKENS;
                t.pos = 0;
            } else {
                t.block0 = r.shared;
                t.pos = r.kv - r.tokens + j * sg.per;
                t.keys_end = t.pos + t.tokens;
            }
            const bool whole = s0 == 0 && s1 == steps, joined = r.shared != 0;
            t.part = t.part_ml = nullptr;
            const int kind = prefix ? 0 : 1;
            if (!whole) {
                const int64_t slot = 2 * (int64_t)wg + (s0 == 0 ? 1 : 0);
                t.part = p.part + slot * kWideRows * DP;
                t.part_ml = p.part_ml + slot * kWideRows * 2;
            } else if (joined) {
                const int64_t row = whole_row(p, gridDim.x, kind, head) + (int64_t)(r.base + j * sg.per) * G;
                t.part = p.part + row * DP;
                t.part_ml = p.part_ml + row * 2;
            }
            if (s0 == 0 && (joined || !whole)) {
                // workgroups that the tile's steps fall to, up to the one in whose piece the last begins
                const uint64_t of_mine = x - in - from + (uint64_t)(steps - 1) * kStepCost[K];
                const int32_t n = (int32_t)quotient(of_mine, each) + 1;
                if (joined) {
                    for (int32_t k = tid; k < t.tokens; k += crew)
                        p.parts[((int64_t)kind * a.Hkv + head) * p.shared_tokens + r.base + j * sg.per + k] =
                            Parts{whole ? 0 : n, wg, k * G, 0};
                } else if (tid == 0) {
                    p.split[blockIdx.x] = Split{n, wg, t.token, t.tokens, head, {0, 0, 0}};
                }
            }
            if constexpr (K == kWide) work.wide(t);
            else if (sg.rows <= 16) work.template narrow<1, K == kSolo>(t);
            else work.template narrow<2, K == kSolo>(t);
        }
        x += left - in;
        off += left - in + (prefix ? 0 : before);
    }
}

// Of `of` places, n spread evenly: whether place `at` is one of them.  at: its number among these, or among the others.
__device__ __forceinline__ bool spread(uint32_t& at, uint32_t n, uint32_t of)
{
    if (of == 0) return false;
    const uint32_t before = at * n / of;
    const bool in = (at + 1) * n / of > before;
    at = in ? before : at - before;
    return in;
}

// One launch over a line of work: request after request (a group's prefix before its first member's own keys), key head
// after key head, tile after tile, step after step.  The line is cut into equal pieces, a workgroup each, whatever the
// lengths are; a tile that is cut is joined by the next kernel.  Every workgroup works out the line for itself, from lengths
// that only the device knows: 4-6 us, as long as another launch that told them would take.  Each kind has a line of its own, so
// that a workgroup keeps to one kind's code; workgroups of different kinds lie side by side on a CU, where one waits for memory while the other
// computes (128 requests on one prefix 86 -> 83 us, groups of 200 64 -> 62 us against kind after kind).
template <int DP, bool Half>
__global__ __launch_bounds__(kThreads, DP <= 128 ? 2 : 1) void attend_kernel(AttendArgs p)
{
    extern __shared__ __align__(1024) uint8_t lds[];
    __shared__ float s_join[2 * kWaves * kNarrowRows];
    __shared__ uint64_t s_tmp[4 * kWaves], s_off[kWaves];
    __shared__ int32_t s_i[kWaves], s_bad;
    using A = Attend<DP, Half>;
    const rk_attention& a = p.a;
    const int tid = threadIdx.x;
    const int32_t B = p.n, G = p.G;
    Request* req = reinterpret_cast<Request*>(lds + A::kTileBytes);
    int32_t* goff = reinterpret_cast<int32_t*>(lds);                 // until the keys and values come
    const bool tell = blockIdx.x == 0;
    if (tid == 0) {
        s_bad = 0;
        for (int w = 0; w < kWaves; ++w) {
            s_i[w] = B;
            s_off[w] = 0;
        }
    }
    __syncthreads();
    // (loads of all of a thread's requests, or groups, together: one after the other, 533 requests take 2 us more)
    constexpr int kMost = kLaunch / kThreads;
    {
        int64_t q0[kMost], q1[kMost];
        int32_t kv[kMost];
#pragma unroll
        for (int u = 0; u < kMost; ++u) {
            const int32_t i = p.b0 + (tid + u * kThreads < B ? tid + u * kThreads : B - 1);
            q0[u] = a.q_off[i];
            q1[u] = a.q_off[i + 1];
            kv[u] = a.kv_len[i];
        }
#pragma unroll
        for (int u = 0; u < kMost; ++u) {
            const int32_t i = tid + u * kThreads;
            if (i >= B) break;
            Request r{};
            const bool large = (int64_t)kv[u] > (int64_t)a.table_stride * RK_BLOCK_TOKENS;
            if (q1[u] < q0[u]) s_bad = 1;    // then requests may claim the same tokens, and what groups share have no room
            if (q0[u] < 0 || q1[u] < q0[u] || q1[u] > a.T || q1[u] - q0[u] > kv[u] || large) {
                if (tell) atomicOr(p.status, large ? RK_DEV_TOO_LARGE : RK_DEV_BAD_OFFSETS);
                r.tokens = -1;
            } else {
                r.kv = kv[u];
                r.q0 = (int32_t)q0[u];
                r.tokens = (int32_t)(q1[u] - q0[u]);
            }
            req[i] = r;
        }
    }
    if (a.group_off)
        for (int32_t g0 = tid; g0 < a.B; g0 += kMost * kThreads) {
            int64_t x[kMost], y[kMost];
#pragma unroll
            for (int u = 0; u < kMost; ++u) {
                const int32_t g = g0 + u * kThreads < a.B ? g0 + u * kThreads : a.B - 1;
                x[u] = a.group_off[g];
                y[u] = a.group_off[g + 1];
            }
#pragma unroll
            for (int u = 0; u < kMost; ++u) {
                const int32_t g = g0 + u * kThreads;
                if (g >= a.B) break;
                if (x[u] > y[u] || x[u] < 0 || y[u] > a.B || (g == 0 && x[u] != 0) || (g == a.B - 1 && y[u] != a.B)) s_bad = 1;
                goff[g] = (int32_t)x[u];
                if (g == a.B - 1) goff[a.B] = (int32_t)y[u];
            }
        }
    __syncthreads();
    const bool groups = a.group_off && !s_bad;
    if (tell && tid == 0 && s_bad) atomicOr(p.status, RK_DEV_BAD_OFFSETS);
    if (groups) {
        // A group attends to its prefix together where every member sees all of it; if only the first
        // does not (it brings the prefix), the others do.  (Members in another launch are a group of their own.)
        struct Members {
            int32_t lent, first, end;
            bool whole;                      // the group's first request is among them
        };
        Members of[kMost];
        int32_t group[kMost] = {}, most[kMost], sh[kMost];
        for (int32_t step = 1 << (31 - __clz(a.B)); step > 0; step >>= 1)        // the last group that does not begin behind the request
#pragma unroll
            for (int u = 0; u < kMost; ++u) {
                const int32_t g = group[u] + step < a.B ? group[u] + step : a.B;
                if (goff[g] <= p.b0 + tid + u * kThreads && g < a.B) group[u] = g;
            }
#pragma unroll
        for (int u = 0; u < kMost; ++u) {
            const int32_t f = goff[group[u]];
            Members& m = of[u];
            m.whole = f >= p.b0;
            m.first = m.whole ? f - p.b0 : 0;
            m.end = goff[group[u] + 1] - p.b0 < B ? goff[group[u] + 1] - p.b0 : B;
            most[u] = a.kv_len[f < a.B ? f : a.B - 1];
            sh[u] = a.shared[group[u]];
        }
#pragma unroll
        for (int u = 0; u < kMost; ++u) {
            const int32_t i = tid + u * kThreads;
            Members& m = of[u];
            most[u] /= RK_BLOCK_TOKENS;
            m.lent = i < B && m.end - m.first >= 2 ? (sh[u] < most[u] ? sh[u] : most[u]) : 0;
            if (m.lent <= 0) continue;
            const int32_t tokens = req[i].tokens;
            if (tokens < 0 || (tokens > 0 && req[i].kv - tokens < m.lent * RK_BLOCK_TOKENS - 1))
                atomicOr(&req[m.first].base, i == m.first && m.whole ? 1 : 2);       // (base is not needed yet)
            // one without new tokens may be shorter than the prefix, but not the one whose row is read for all
            else if (i - m.first < 2 && req[i].kv < m.lent * RK_BLOCK_TOKENS)
                atomicOr(&req[m.first].base, i == m.first ? 4 : 8);
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kMost; ++u) {
            const int32_t i = tid + u * kThreads;
            const Members& m = of[u];
            if (i >= B || m.lent <= 0) continue;
            const int32_t broken = req[m.first].base, f = m.first + (broken & 1);
            if (m.end - f < 2 || (broken & 2) || (broken & (broken & 1 ? 8 : 4)) || i < f) continue;
            // Together where that costs less along the line than each member's own steps over the prefix, a join a member
            // counted; and only if most members have fewer rows than a wide tile (what the workspace holds).  Calls one after the
            // other on the same inputs: 128 requests on 8,192 tokens 80 us together, 507 us each for itself; 200 of 24 groups 62 and 129;
            // pieces of prompts in 3 groups, of 350 tokens each, 117 and 116 (there the matrix instructions bound both); 533 requests that
            // share 5 blocks stay apart, for 141 us, 134 when no groups are named.
            const int64_t n = m.end - f, tokens = req[m.end - 1].q0 + req[m.end - 1].tokens - req[f].q0, rows = tokens * G;
            if (rows == 0 || rows >= kWideRows * n) continue;
            const Segment sg = prefix_segment((int32_t)tokens, m.lent, p);
            const int64_t apart = n * m.lent * (rows > kNarrowRows * n ? 2 : 1), costs = sg.kind == kSolo ? 1 : 4;    // in quarters
            if ((int64_t)sg.cost * costs + 4 * kJoinCost * n >= apart) continue;
            req[i].shared = m.lent;
            if (i == f) req[i].end = m.end;
        }
        __syncthreads();
    }
    // the line of work: per thread's requests, then over the threads; each kind of tiles on its own
    const int32_t per = (B + kThreads - 1) / kThreads;
    const int32_t i0 = tid * per, i1 = i0 + per < B ? i0 + per : B;
    struct Cost {
        uint64_t of[3];
    };
    auto cost_of = [&](int32_t i, Cost& x) {
        auto add = [&](const Segment& sg) {
#pragma unroll
            for (int k = 0; k < 3; ++k) x.of[k] += sg.kind == k ? sg.cost * (uint64_t)a.Hkv : 0;
        };
        add(own_segment(req[i], p));
        if (req[i].end) {
            const Request& l = req[req[i].end - 1];
            add(prefix_segment(l.q0 + l.tokens - req[i].q0, req[i].shared, p));
        }
    };
    uint32_t together = 0;
    for (int32_t i = i0; i < i1; ++i) {
        if (req[i].tokens < 0) req[i].tokens = 0;
        if (req[i].shared) together += req[i].tokens;
    }
    __syncthreads();
    Cost mine{};
    for (int32_t i = i0; i < i1; ++i) cost_of(i, mine);
    Cost upto = mine, all{};
    uint32_t tokens_upto = together;
    incl_sums(upto.of, tokens_upto, s_tmp);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        for (int w = 0; w < kWaves; ++w) all.of[k] += s_tmp[kWaves * k + w];
        all.of[k] = uniform(all.of[k]);
    }
    // pieces for at most gridDim.x workgroups (each kind's last may be short)
    uint64_t each = quotient_up(all.of[kWide] + all.of[kNarrow] + (all.of[kSolo] + kWaves - 1) / kWaves, gridDim.x - 3);
    if (each < kLeast) each = kLeast;
    const uint32_t n_wide = (uint32_t)quotient_up(all.of[kWide], each), n_narrow = (uint32_t)quotient_up(all.of[kNarrow], each);
    const uint32_t n_solo = (uint32_t)((quotient_up(all.of[kSolo], each) + kWaves - 1) / kWaves);
    const uint32_t active = n_wide + n_narrow + n_solo;
    // workgroups go to the 8 XCDs in turn: each XCD takes a stretch of each kind's line, the kinds mixed
    const uint32_t stretch = (active + 7) / 8, place = (blockIdx.x & 7u) * stretch + (blockIdx.x >> 3);
    const bool idle = (blockIdx.x >> 3) >= stretch || place >= active;
    uint32_t at = place;                     // the number among its kind's
    const int kind = spread(at, n_wide, active) ? kWide : spread(at, n_narrow, n_narrow + n_solo) ? kNarrow : kSolo;
    const uint32_t wg = at + (kind == kWide ? 0 : kind == kNarrow ? n_wide : n_wide + n_narrow);
    const uint64_t end = kind == kWide ? all.of[kWide] : kind == kNarrow ? all.of[kNarrow] : all.of[kSolo];
    // the workgroup's piece, or its wavefronts' of solo tiles
    const uint64_t first = (kind == kSolo ? (uint64_t)kWaves * at : at) * each;
    {
        uint32_t tok = tokens_upto - together;
        const uint64_t top = kind == kWide ? upto.of[kWide] : kind == kNarrow ? upto.of[kNarrow] : upto.of[kSolo];
        uint64_t x = top - (kind == kWide ? mine.of[kWide] : kind == kNarrow ? mine.of[kNarrow] : mine.of[kSolo]);
        const int pieces = kind == kSolo ? kWaves : 1;
        const bool here = !idle && first + (pieces - 1) * each >= x && first < top;
        for (int32_t i = i0; i < i1; ++i) {
            req[i].base = (int32_t)tok;
            if (req[i].shared) tok += req[i].tokens;
            if (tell) p.shared[i] = Shared{req[i].q0, req[i].shared ? req[i].tokens : 0, req[i].base, 0};
            if (!here) continue;
            Cost k = mine;
            if (per > 1) {
                k = Cost{};
                cost_of(i, k);
            }
            const uint64_t w = kind == kWide ? k.of[kWide] : kind == kNarrow ? k.of[kNarrow] : k.of[kSolo];
            for (int q = 0; q < pieces; ++q) {
                const uint64_t from = first + q * each;
                if (from >= x && from < x + w) {
                    s_i[q] = i;
                    s_off[q] = from - x;
                }
            }
            x += w;
        }
    }
    __syncthreads();
    if (tid == 0) p.split[blockIdx.x].n = 0;
    if (idle) return;
    float c = fabsf(a.scale) * kLog2e;
    if (c < 1e-30f) c = 1e-30f;              // scores of 0, and -infinity stays what it is
    A work(p, (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)lds, s_join, c);
    const int piece = kind == kSolo ? work.wave : 0;
    const int32_t i = uniform(s_i[piece]);
    const uint64_t off = uniform(s_off[piece]), from = first + piece * each, to = from + each < end ? from + each : end;
    if (kind == kWide) walk<kWide>(work, req, i, off, from, to, each, (int32_t)wg);
    else if (kind == kNarrow) walk<kNarrow>(work, req, i, off, from, to, each, (int32_t)wg);
    else walk<kSolo>(work, req, i, off, from, to, each, (int32_t)wg);
}

// The parts of rows that more than one workgroup worked on, joined: a wavefront a row, DP / 64 neighbouring values a
// lane.  The parts' weights come first, a lane each; then their values, several loads under way at a time.  Waiting for
// loads is all that bounds it (4 us with nothing to join, 8-10 us for decoding batches), but of the rows of whole prompts'
// 500 cut tiles (30 us for 100 MB).
template <int DP, bool Half>
__global__ __launch_bounds__(kThreads) void join_kernel(AttendArgs p, int32_t grid, int32_t chunks, int32_t shared_chunks)
{
    const rk_attention& a = p.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t G = p.G;
    constexpr int N = DP / 64;
    // n parts at the rows row_of(k), to the output's row of the token and query head
    auto join = [&](int32_t n, auto&& row_of, int64_t token, int32_t h) {
        float o[N] = {}, m = -INFINITY, l = 0.0f;
        for (int32_t k0 = 0; k0 < n; k0 += 64) {
            const int32_t k = k0 + lane;
            float pm = -INFINITY, pl = 0.0f;
            if (k < n) {
                const int64_t row = row_of(k);
                pm = p.part_ml[2 * row];
                pl = p.part_ml[2 * row + 1];
            }
            float top = pm;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) top = larger(top, __shfl_xor(top, d));
            const float nm = larger(m, top);
            if (nm == -INFINITY) {           // no key seen, or scores that are no numbers: l tells
#pragma unroll
                for (int d = 32; d > 0; d >>= 1) pl += __shfl_xor(pl, d);
                l += pl;
                continue;
            }
            const float old = __builtin_amdgcn_exp2f(m - nm), w = __builtin_amdgcn_exp2f(pm - nm);
            float sum = w * pl;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
            l = l * old + sum;
            m = nm;
#pragma unroll
            for (int x = 0; x < N; ++x) o[x] = old == 0.0f ? 0.0f : o[x] * old;
            const int32_t here = n - k0 < 64 ? n - k0 : 64;
            constexpr int kAtOnce = 8;
            for (int32_t q = 0; q < here; q += kAtOnce) {
                float v[kAtOnce][N];
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const int64_t row = row_of(k0 + (q + u < here ? q + u : here - 1));
#pragma unroll
                    for (int x = 0; x < N; ++x) v[u][x] = p.part[row * DP + N * lane + x];
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    const float f = q + u < here ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), q + u)) : 0.0f;
                    if (f != 0.0f)           // (a weight of 0 takes nothing of a part, whatever that holds)
#pragma unroll
                        for (int x = 0; x < N; ++x) o[x] += f * v[u][x];
                }
            }
        }
        const float inv = l == 0.0f ? 0.0f : 1.0f / l;
        uint16_t* to = (uint16_t*)a.out + token * a.out_token + h * a.out_head + N * lane;
#pragma unroll
        for (int x = 0; x < N; x += N % 2 ? 1 : 2) {
            if (N * lane + x >= a.D) break;
            if constexpr (N % 2 == 0) *reinterpret_cast<uint32_t*>(to + x) = pack16<Half>(o[x] * inv, o[x + 1] * inv);
            else to[x] = (uint16_t)pack16<Half>(o[x] * inv, 0.0f);
        }
        if (lane == 0 && a.lse) a.lse[token * a.Hq + h] = l == 0.0f ? -INFINITY : (m + __builtin_log2f(l)) * kLn2;
    };
    // the k-th part of a cut tile's row r that workgroup wg began: its last, then the first of those after it
    auto cut = [&](int32_t wg, int32_t r, int32_t k) { return (2 * (int64_t)(wg + k) + (k == 0 ? 1 : 0)) * kWideRows + r; };
    const int32_t of_shared = a.group_off ? p.n * a.Hkv * shared_chunks : 0;
    if ((int32_t)blockIdx.x >= of_shared) {
        const int32_t b = (int32_t)blockIdx.x - of_shared;
        const Split t = p.split[b / chunks];
        const int32_t rows = t.tokens * G;
        if (t.n == 0) return;
        for (int32_t r = b % chunks * kWaves + wave; r < rows; r += chunks * kWaves)
            join(t.n, [&](int32_t k) { return cut(t.wg, r, k); }, t.token + (int64_t)(r / G), t.head * G + r % G);
        return;
    }
    const int32_t u = (int32_t)blockIdx.x / shared_chunks, head = u % a.Hkv;
    const Shared t = p.shared[u / a.Hkv];
    const int32_t rows = t.tokens * G;
    for (int32_t r = (int32_t)blockIdx.x % shared_chunks * kWaves + wave; r < rows; r += shared_chunks * kWaves) {
        const int32_t tok = r / G, h = r % G;
        Parts x[2];
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            x[kind] = p.parts[((int64_t)kind * a.Hkv + head) * p.shared_tokens + t.base + tok];
        const int32_t n0 = uniform(x[0].n), n1 = uniform(x[1].n), first = n0 > 0 ? n0 : 1;
        const int32_t wg0 = uniform(x[0].wg), wg1 = uniform(x[1].wg), r0 = uniform(x[0].row) + h, r1 = uniform(x[1].row) + h;
        join(first + (n1 > 0 ? n1 : 1), [&](int32_t k) {
            const bool own = k >= first;
            if ((own ? n1 : n0) == 0) return whole_row(p, grid, own ? 1 : 0, head) + (int64_t)t.base * G + r;
            return own ? cut(wg1, r1, k - first) : cut(wg0, r0, k);
        }, t.q0 + (int64_t)tok, head * G + h);
    }
}

// ---------------------------------------------------------------- host

inline int head_size(int32_t D) { return D <= 64 ? 64 : D <= 128 ? 128 : D <= 192 ? 192 : 256; }

inline int32_t launch_size(int32_t B) { return B < kLaunch ? B : kLaunch; }

inline size_t lds_bytes(int dp, int32_t n) { return (size_t)512 * dp + sizeof(Request) * (size_t)n; }

// Workgroups that the device holds at once.
inline int32_t grid_for(int dp, int32_t n)
{
    const int32_t cus = compute_units();
    const int fit = dp <= 128 && lds_bytes(dp, n) + 4096 <= (160u << 10) / 2 ? 2 : 1;
    return ((cus > 0 ? cus : 256) * fit + 7) / 8 * 8;
}

struct AttendLayout {
    size_t split, shared, parts, part, part_ml, bytes;
    int32_t grid, shared_rows, shared_tokens;
};

inline AttendLayout attend_layout(int64_t T, int32_t B, int32_t Hq, int32_t Hkv, int32_t D)
{
    AttendLayout L;
    const int dp = head_size(D);
    const int32_t G = Hq / Hkv, n = launch_size(B);
    L.grid = grid_for(dp, n);
    // rows of groups that attend together: fewer than a wide tile's for each member
    const int64_t most = (int64_t)kWideRows * n / G, tokens = T < most ? T : most;
    L.shared_tokens = (int32_t)tokens;
    L.shared_rows = (int32_t)(tokens * G);
    size_t o = 0;
    auto take = [&](size_t n) {
        const size_t at = o;
        o = align_up(o + n, 256);
        return at;
    };
    L.split = take(sizeof(Split) * (size_t)L.grid);
    L.shared = take(sizeof(Shared) * (size_t)n);
    L.parts = take(sizeof(Parts) * 2 * (size_t)Hkv * L.shared_tokens);
    const size_t all_rows = 2 * (size_t)L.grid * kWideRows + 2 * (size_t)Hkv * L.shared_rows;
    L.part_ml = take(4 * 2 * all_rows);
    L.part = take(4 * (size_t)dp * all_rows);
    L.bytes = o;
    return L;
}

template <int DP, bool Half>
static int launch(AttendArgs& p, int32_t grid, hipStream_t s)
{
    const int64_t rows = p.a.T * p.G;
    const int32_t chunks = rows <= 4 ? 1 : rows <= 32 ? 4 : 8;
    const int32_t shared_chunks = (p.G + kWaves - 1) / kWaves;       // a row a wavefront, of one new token
    for (p.b0 = 0; p.b0 < p.a.B; p.b0 += p.n) {
        p.n = launch_size(p.a.B - p.b0);
        // With few tiles, one wavefront with all of a tile's keys would be what the others wait for (16 requests of 300 tokens
        // on 2 key heads 25 us, 21 by workgroups; 64 of 128 on 8 22 us, 27 by workgroups).
        p.solo_most = (int64_t)p.n * p.a.Hkv > grid / 2 ? kSoloMost : 0;
        hipLaunchKernelGGL((attend_kernel<DP, Half>), dim3((unsigned)grid), dim3(kThreads), lds_bytes(DP, p.n), s, p);
        int rc = hip_check(hipGetLastError(), "rk_prefix_attention launch");
        if (rc) return rc;
        const int64_t blocks = (int64_t)grid * chunks + (p.a.group_off ? (int64_t)p.n * p.a.Hkv * shared_chunks : 0);
        hipLaunchKernelGGL((join_kernel<DP, Half>), dim3((unsigned)blocks), dim3(kThreads), 0, s, p, grid, chunks,
                           shared_chunks);
        rc = hip_check(hipGetLastError(), "rk_prefix_attention join launch");
        if (rc) return rc;
    }
    return RK_OK;
}

template <bool Half>
static int launch_of(AttendArgs& p, int32_t grid, hipStream_t s)
{
    switch (head_size(p.a.D)) {
    case 64: return launch<64, Half>(p, grid, s);
    case 128: return launch<128, Half>(p, grid, s);
    case 192: return launch<192, Half>(p, grid, s);
    default: return launch<256, Half>(p, grid, s);
    }
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
    return attend_layout(T, B, Hq, Hkv, D).bytes;
}

int rk_prefix_attention(const rk_attention* a, void* workspace, size_t ws_bytes, void* stream)
{
    if (!a) return fail(RK_EINVAL, "rk_prefix_attention: NULL arguments");
    int rc;
    if (const char* what = attention_sizes(a->T, a->B, a->Hq, a->Hkv, a->D, &rc))
        return fail(rc, "rk_prefix_attention: %s", what);
    if (a->dtype != RK_BF16 && a->dtype != RK_F16) return fail(RK_EUNSUPPORTED, "rk_prefix_attention: dtype %d", a->dtype);
    if (a->n_blocks < 0 || a->table_stride < 0) return fail(RK_EINVAL, "rk_prefix_attention: a negative size");
    if (a->table_stride > 1 << 26) return fail(RK_EUNSUPPORTED, "rk_prefix_attention: table_stride > 2^26 blocks");
    if (!(fabsf(a->scale) <= 1e18f)) return fail(RK_EINVAL, "rk_prefix_attention: scale outside -1e18..1e18");
    const int64_t strides[] = {a->q_token, a->q_head, a->out_token, a->out_head, a->ks.block, a->ks.token, a->ks.head,
                               a->vs.block, a->vs.token, a->vs.head};
    for (int64_t x : strides)
        if (x < 0 || x % 8) return fail(RK_EINVAL, "rk_prefix_attention: a stride is negative or no multiple of 8");
    if (!rows_apart({{a->T, a->out_token}, {a->Hq, a->out_head}}, a->D))
        return fail(RK_EINVAL, "rk_prefix_attention: out's strides lay heads or tokens over each other");
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
    const AttendLayout L = attend_layout(a->group_off ? a->T : 0, a->B, a->Hq, a->Hkv, a->D);       // (no groups: no rows of such)
    if (!workspace || ws_bytes < L.bytes)
        return fail(RK_ENOMEM, "rk_prefix_attention: workspace of %zu bytes, %zu needed", workspace ? ws_bytes : (size_t)0, L.bytes);
    if ((uintptr_t)workspace % 256) return fail(RK_EINVAL, "rk_prefix_attention: workspace is not aligned to 256 bytes");
    uint8_t* ws = (uint8_t*)workspace;
    AttendArgs p;
    p.a = *a;
    p.status = status_word();
    if (!p.status) return fail(RK_EHIP, "rk_prefix_attention: no status word");
    p.split = (Split*)(ws + L.split);
    p.shared = (Shared*)(ws + L.shared);
    p.parts = (Parts*)(ws + L.parts);
    p.part = (float*)(ws + L.part);
    p.part_ml = (float*)(ws + L.part_ml);
    p.G = a->Hq / a->Hkv;
    p.wide_tokens = kWideRows / p.G;
    p.g_inverse = (uint32_t)((65535 + p.G) / p.G);
    p.shared_rows = L.shared_rows;
    p.shared_tokens = L.shared_tokens;
    return a->dtype == RK_F16 ? launch_of<true>(p, L.grid, (hipStream_t)stream) : launch_of<false>(p, L.grid, (hipStream_t)stream);
}

}  // extern "C"
