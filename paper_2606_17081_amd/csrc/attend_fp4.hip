// attend_fp4.hip -- rk_prefix_attention_fp4: the entry points, and the kernels of caches held in 4 bits.
//
// The mathematics, the tiles and the line of work are attend.h's.  A key or value is 17/64 of its 16-bit bytes; the codes come to
// registers, and the unit that converts two of them in an instruction gives 16-bit values that are exact, so that both products are
// those of a 16-bit cache that holds the same, and differ from 64 bits by the weights' rounding alone.
//
// What bounds it: few rows the reading, 17 D / 16 bytes a key and head; from some hundred rows a key head on the matrix instructions.
// Kernels in a trace, the same inputs over and over: 96 requests of 500-12,000 tokens (64 / 8 heads of 128) 98 + 5 us, 3.9 TB/s, of
// which 20-25 us are the beginning (lengths, pieces, block numbers, queries) and the ends of pieces (longer and shorter batches
// differ by 5.7 TB/s); 5 requests of 60,000-200,000 tokens (16 / 4 heads) 88 + 6 us, 4.3 TB/s; 128 requests on one prefix of 8,192
// tokens 67 + 10 us, as over 16 bits; whole prompts of 2,500-6,000 tokens 1.10-1.22 ms, 890-980 TFLOP/s.
#include "attend.h"

namespace rk {

struct AttendFp4Args : AttendArgs {
    rk_fp4_cache kc, vc;
};

// Tiles over a cache in 4 bits.
template <int DP, bool Half>
struct AttendFp4 : AttendBase<DP, Half> {
    typedef AttendFp4Args Args;
    using Base = AttendBase<DP, Half>;
    using Base::NC, Base::kRow, Base::kTurn, Base::turn, Base::p, Base::tile, Base::join, Base::wave, Base::G, Base::c;
    using Base::block_id, Base::report_bad, Base::token_of, Base::query_of, Base::strays, Base::divisor;
    // Keys of a wavefront in a narrow step: a key is a quarter of the bytes of a 16-bit one, and as many should be under way.
    static constexpr int kNarrowKeys = DP <= 128 ? 64 : 32;
    // As of 16-bit caches, though a narrow step has a quarter of the bytes and twice the keys.  (96 requests of 500-12,000 tokens 113 us; ends of 2, 3, 4
    // or 10 for narrow tiles 115-120, a wide step of 1: 119.  A shared prompt 74 us, with ends of 2 or 3 82-84.)
    static constexpr uint32_t kStepCost[3] = {2, 2, 2}, kEndsCost[3] = {12, 6, 6};
    static_assert(kLeast >= kStepCost[kWide] && kLeast >= kStepCost[kNarrow], "a step begins in every piece of a tile");

    using Base::Base;

    // The kernel's arguments, to be read where they are used: what is read through `p` is read at the kernel's beginning and kept in
    // scalar registers through all tiles, more than there are.  (The address is the kernel's own: in a function that it calls the compiler
    // has none, and takes 0.  So all that asks for it is inlined.)
    typedef const __attribute__((address_space(4))) AttendFp4Args Held;
    static __device__ __forceinline__ Held& args()
    {
        Held* a = (Held*)__builtin_amdgcn_kernarg_segment_ptr();
        asm volatile("" : "+s"(a));
        return *a;
    }
    typedef const __attribute__((address_space(4))) rk_fp4_cache Cache;

    // A lane loads a quarter of a row of a block: in each round a share (32 values of one power of two), in the last, of a DP that is
    // no multiple of 128, half a share.
    static constexpr int kShares = DP / 32, kRounds = (kShares + 3) / 4, kPieces = DP / 32;   // (kPieces: of 8 values, a lane's)
    static constexpr bool kHalfRound = kShares % 4 != 0;
    static constexpr uint32_t kNowhere = 0x80000000u;        // past any block's end: what is loaded there is 0

    // Which of a row's pieces of 8 values quarter j has as its ks-th.
    static __device__ __forceinline__ int piece_of(int ks, int j)
    {
        if (kHalfRound && ks / 4 == kRounds - 1) return 4 * (ks / 4 * 4 + j / 2) + 2 * (j & 1) + ks % 4;
        return 4 * (ks / 4 * 4 + j) + ks % 4;
    }

    // Byte offsets in a block of what a lane loads of it, quarter j of row r: codes and powers of two.
    struct Places {
        uint32_t codes[kRounds], powers[kRounds];
    };
    static __device__ __forceinline__ Places places(const Cache& cache, int32_t D, uint32_t r, uint32_t j)
    {
        Places at;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            const bool half = kHalfRound && i == kRounds - 1;
            const uint32_t share = 4 * i + (half ? j / 2 : j);
            const bool there = 32 * share < (uint32_t)D;
            at.codes[i] = there ? r * (uint32_t)cache.cs.token + 16 * share + (half ? 8 * (j & 1) : 0) : kNowhere;
            at.powers[i] = there ? r * (uint32_t)cache.ss.token + share : kNowhere;
        }
        return at;
    }

    struct Codes {
        u32x4 w[kRounds];
        uint32_t power[kRounds];
        // the lane's ks-th piece in 16 bits, which hold the values exactly
        __device__ __forceinline__ u32x4 values(int ks) const
        {
            return fp4_values<Half>(w[ks / 4][ks % 4], __uint_as_float(power[ks / 4] << 23));
        }
    };
    // 0 for a key's codes behind D, beside values of the same power of two before it: the type may not hold what they stand for, and the
    // query's zeros do not make 0 of an infinity.  (Values there are in products of their own, which go nowhere.)  A D that its class
    // takes ends in a row's last round, and behind a lane's first piece there if rounds are whole.
    static __device__ __forceinline__ void end_at(Codes& x, int32_t D, uint32_t j)
    {
        constexpr int r = kRounds - 1;
#pragma unroll
        for (int e = kHalfRound ? 0 : 1; e < (kHalfRound ? 2 : 4); ++e) x.w[r][e] = 8 * piece_of(4 * r + e, j) < D ? x.w[r][e] : 0u;
    }
    // A key head's keys or values: where they begin, and how many bytes a block of them spans (0: there is none).
    struct Side {
        const uint8_t *codes, *powers;
        uint32_t code_block, power_block;    // bytes from block to block (below 2^32)
        int32_t code_bytes, power_bytes;
    };
    static __device__ __forceinline__ Side side(const Cache& c, Held& a, int32_t head)
    {
        const int32_t shares = (a.a.D + 31) / 32, last = RK_BLOCK_TOKENS - 1;
        const bool some = a.a.n_blocks > 0;
        return Side{(const uint8_t*)c.codes + head * c.cs.head, (const uint8_t*)c.scales + head * c.ss.head, (uint32_t)c.cs.block,
                    (uint32_t)c.ss.block, some ? last * (int32_t)c.cs.token + 16 * shares : 0, some ? last * (int32_t)c.ss.token + shares : 0};
    }
    // The lane's part of block `id` of the cache.  All of the block is loaded: a key behind a sequence's end gets no weight, and
    // of values there only what is no number could show.
    template <int Aux>
    static __device__ __forceinline__ Codes codes_of(const Side& from, int32_t id, const Places& at)
    {
        const Memory codes = memory(from.codes + (uint64_t)(uint32_t)id * from.code_block, from.code_bytes);
        const Memory powers = memory(from.powers + (uint64_t)(uint32_t)id * from.power_block, from.power_bytes);
        Codes x;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) {
            if (kHalfRound && i == kRounds - 1) {
                const u32x2 w = load8<Aux>(codes, at.codes[i]);
                x.w[i] = u32x4{w.x, w.y, 0u, 0u};
            } else {
                x.w[i] = load16<Aux>(codes, at.codes[i]);
            }
            x.power[i] = load1<Aux>(powers, at.powers[i]);
        }
        return x;
    }
    // A use of x's powers beside their loads, on a path that is hardly taken.  Without it they leave the loads in 16 bits and are extended
    // to 32 as soon as there is time, long before they are used, which waits for the memory.
    static __device__ __forceinline__ void keep_wide(const Codes& x)
    {
#pragma unroll
        for (int i = 0; i < kRounds; ++i) asm volatile("" ::"v"(x.power[i]));
    }
    // The least power in the place of those of rows (lane % 16) that block number b of the tile's sequence does not have: what weights of
    // 0 are multiplied with is a number then.
    static __device__ __forceinline__ void only_rows(Codes& x, const Tile& t, int32_t b, bool bad, uint32_t lane)
    {
        const bool there = !bad && (int32_t)(lane & 15) < t.keys_end - b * RK_BLOCK_TOKENS;
#pragma unroll
        for (int i = 0; i < kRounds; ++i) x.power[i] = there ? x.power[i] : 0u;
    }
    // The ks-th piece of a lane's quarter (lane / 16) of row lane % 16, and all of them, as 16-bit values to a block's place in LDS.
    // (Eight lanes' 16 bytes are written at once, to 128 bytes of banks, of which rows 2 r and 2 r + 1 want the same: 8 cycles beside the 8
    // that a write takes.  A row by four lanes beside each other takes 26 more.  Without the 8, by odd rows' pieces in another order,
    // all cases are within 2% of these; with loads in another order of rows, prompts 5% slower.)
    __device__ __forceinline__ void place_piece(const Codes& x, int ks, uint32_t lds, uint32_t lane) const
    {
        const uint32_t r = lane & 15;
        lds_write16(lds + r * kRow + (((uint32_t)piece_of(ks, lane >> 4) ^ turn(r)) << 4), x.values(ks));
    }
    __device__ __forceinline__ void place_values(const Codes& x, uint32_t lds, uint32_t lane) const
    {
#pragma unroll
        for (int ks = 0; ks < kPieces; ++ks) place_piece(x, ks, lds, lane);
    }

    // The numbers of the blocks that a tile's steps load, N of each step, 64 of them in the lanes of each of M registers.
    // (Scalar loads of each step's would be waited for with the LDS operations beside them, the memory's whole time in every
    // step.  So would loads in the midst of a tile, so there are M registers to choose from: decoding batches read all at a tile's beginning.)
    template <int N, int M>
    struct Numbers {
        static constexpr int kSteps = 64 / N;
        const __attribute__((address_space(4))) int32_t* row;
        int32_t from, per, last, n_blocks;   // step x loads the entries from + per x .. + N - 1, of which `last` is the last there is
        int32_t base, held[M];               // the steps' from `base` on; of a block outside the cache, kBad
        bool odd;                            // there is one among them
        static constexpr int32_t kBad = (int32_t)0x80000000u;
        __device__ __forceinline__ Numbers(const Tile& t, int32_t from_, int32_t per_, int32_t n, int32_t step, uint32_t lane)
            : row(t.row), from(from_), per(per_), last((t.keys_end - 1) / RK_BLOCK_TOKENS), n_blocks(n)
        {
            load(step, lane);
        }
        __device__ __forceinline__ void load(int32_t step, uint32_t lane)
        {
            base = step;
            odd = false;
#pragma unroll
            for (int k = 0; k < M; ++k) {
                const int32_t b = from + per * (step + kSteps * k + (int32_t)(lane / N)) + (int32_t)(lane % N);
                held[k] = row[b < last ? b : last];
            }
#pragma unroll
            for (int k = 0; k < M; ++k) {
                const bool outside = (uint32_t)held[k] >= (uint32_t)n_blocks;
                odd |= __any(outside);
                held[k] = outside ? kBad : held[k];
            }
        }
        // Step x's (x grows): the numbers, 0 of a block outside the cache; a bit of each such.
        __device__ __forceinline__ uint32_t of(int32_t x, int32_t (&id)[N], uint32_t lane)
        {
            if (x - base >= M * kSteps) load(x, lane);
            const int32_t y = x - base, k = y / kSteps, place = (y % kSteps) * N;
            int32_t here = held[0];
#pragma unroll
            for (int j = 1; j < M; ++j) here = k >= j ? held[j] : here;
            uint32_t bad = 0;
#pragma unroll
            for (int b = 0; b < N; ++b) id[b] = __builtin_amdgcn_readlane(here, place + b);
            if (odd) {
#pragma unroll
                for (int b = 0; b < N; ++b) {
                    bad |= ((uint32_t)id[b] >> 31) << b;
                    id[b] &= ~kBad;
                }
            }
            return bad;
        }
    };

    // ---------------------------------------------------------------- up to 128 rows, 32 a wavefront
    //
    // As over 16-bit caches: scores are computed transposed, keys x rows, and the weights lie in registers in the order in which the
    // product with the values takes them.  All that differs is how keys and values come to LDS: by registers, a wavefront a block of
    // each step, converted once for the four of them.  Matrix instructions bound it (D = 128: 32 products of 32 cycles
    // a step and wavefront; 32 conversions and 32 exponentials a lane lie beside them).
    __device__ __forceinline__ void wide(const Tile& t)
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
        // scores run beside them.  Pieces are read from LDS kAhead products before the one that takes them.  (Both as over 16 bits, where they
        // were measured: 1,440 -> 1,360 us of whole prompts, and with 6 ahead, which spills, 1,230 -> 1,500.)
        constexpr int kAhead = 4, kPairs = 16;       // (a lane has 32 scores of a step: kPairs pairs)
        Held& a = args();
        const int32_t n_blocks = a.a.n_blocks, D = a.a.D;
        const Side k_side = side(a.kc, a, t.head), v_side = side(a.vc, a, t.head);
        const Places k_at = places(a.kc, a.a.D, lane & 15, lane >> 4), v_at = places(a.vc, a.a.D, lane & 15, lane >> 4);
        struct Step {
            int32_t own;                             // this wavefront's block
            uint32_t bad;                            // of the four blocks, those outside the cache
        };
        Numbers<4, 2> numbers(t, t.block0, 4, n_blocks, t.s0, lane);
        auto look = [&](int32_t x) {
            int32_t id[4];
            const uint32_t bad = numbers.of(x, id, lane);
            return Step{wave < 2 ? (wave == 0 ? id[0] : id[1]) : (wave == 2 ? id[2] : id[3]), bad};
        };
        auto keys_at = [&](int32_t x) { return tile + ((x - t.s0) & 1) * kKeys; };
        auto values_at = [&](int32_t x) { return tile + 2 * kKeys + ((x - t.s0) & 1) * kKeys; };
        // Of a cache in 4 bits the codes of keys three steps ahead and of values two are under way to registers; they are
        // converted into the stages of keys two steps ahead and values one beside the second product, which leaves the vector units idle.
        Codes k_raw, v_raw;
        auto issue_keys = [&](int32_t x, const Step& e) {
            k_raw = codes_of<0>(k_side, e.own, k_at);
            if (numbers.odd) keep_wide(k_raw);
        };
        auto issue_values = [&](int32_t x, const Step& e) {
            v_raw = codes_of<0>(v_side, e.own, v_at);
            if (numbers.odd) keep_wide(v_raw);
        };
        auto put_keys = [&](int32_t x) {
            end_at(k_raw, D, lane >> 4);
            place_values(k_raw, keys_at(x) + wave * (RK_BLOCK_TOKENS * kRow), lane);
        };
        auto true_values = [&](int32_t x, const Step& e) { only_rows(v_raw, t, t.block0 + 4 * x + wave, e.bad >> wave & 1, lane); };
        auto put_values = [&](int32_t x, const Step& e) {
            true_values(x, e);
            place_values(v_raw, values_at(x) + wave * (RK_BLOCK_TOKENS * kRow), lane);
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
        // A step whose keys every row sees: sc its scores, top their largest; the next step's into nx; e1, e2, e3: the blocks of the
        // steps after it.
        auto open_step = [&](int32_t x, const f32x16* sc, f32x16* nx, float& top, const Step& e1, const Step& e2, const Step& e3) {
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
            // whole prompts over 16 bits 1,251 -> 1,214 us)
            __builtin_amdgcn_s_setprio(1);
            const Values va = values_in(values_at(x));
            true_values(x + 1, e1);
            end_at(k_raw, D, lane >> 4);
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
                if (u % 2 == 0 && u / 2 < kPieces) place_piece(v_raw, u / 2, values_at(x + 1) + wave * (RK_BLOCK_TOKENS * kRow), lane);
                if (u % 2 == 0 && u / 2 >= kPieces) place_piece(k_raw, u / 2 - kPieces, keys_at(x + 2) + wave * (RK_BLOCK_TOKENS * kRow), lane);
            }
            __builtin_amdgcn_s_setprio(0);
            issue_values(x + 2, e2);         // (past the tile's end they bring zeros, to a stage that is not read again)
            issue_keys(x + 3, e3);
        };
        int32_t s = t.s0;
        uint32_t any_bad = 0;
        Step now, next, then, far;
        // Step s + 1's keys and step s's values are there, and everyone has read what came before.
        auto arrive = [&]() {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        auto advance = [&]() {
            ++s;
            now = next;
            next = then;
            then = far;
            far = look(s + 3);
        };
        now = look(s);
        next = look(s + 1);
        then = look(s + 2);
        far = look(s + 3);
        __syncthreads();                             // the LDS is the last tile's until here
        issue_keys(s, now);
        issue_values(s, now);
        put_keys(s);
        issue_keys(s + 1, next);
        put_values(s, now);
        issue_values(s + 1, next);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) q[ks] = query_of(a.a, t, r, 2 * ks + hi);
        put_keys(s + 1);
        issue_keys(s + 2, then);
        arrive();
        f32x16 sa[2], sb[2];
        scores(keys_at(s), sa);
        // the steps whose keys every row sees, if their blocks are good, but the last
        const int32_t open = (all_see + 1 - t.block0 * RK_BLOCK_TOKENS) / kWideKeys, s_open = open < t.s1 - 1 ? open : t.s1 - 1;
        float top = highest(sa);
        while (s + 1 < s_open && !(now.bad | next.bad)) {
            arrive();
            open_step(s, sa, sb, top, next, then, far);
            advance();
            arrive();
            open_step(s, sb, sa, top, next, then, far);
            advance();
        }
        for (;;) {
            arrive();
            const int32_t key0 = (t.block0 + 4 * s) * RK_BLOCK_TOKENS;
            const bool masked = key0 + kWideKeys - 1 > all_see;
            if (masked || now.bad) {
                any_bad |= now.bad;
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
            put_values(s + 1, next);         // (not in the last step: then others write their results there)
            put_keys(s + 2);
            issue_values(s + 2, then);
            issue_keys(s + 3, far);
            scores(keys_at(s + 1), sa);
            advance();
        }
        this->template wide_out<DT>(t, o, m, l, r, lane);
        if (any_bad) report_bad();
    }

    // ---------------------------------------------------------------- up to 16 NQ rows, kNarrowKeys keys a wavefront
    //
    // What bounds few rows is the reading of keys and values: each wavefront takes keys of its own, with no barrier.  The codes of
    // kSets steps are under way to registers, keys in the order in which the product takes them, so that they are converted
    // there; values pass LDS once they are 16 bits, since the second product takes them by columns.
    template <int NQ, bool Solo>
    __device__ __forceinline__ void narrow(const Tile& t)
    {
        // Where a head's rows of a block lie side by side, what is read is read once, by whole lines, and need not stay in caches.  Calls on
        // inputs that change, 64 requests of 5,504 tokens on 8 heads: 101 us so, 110 without the hint; rows of all heads of a token
        // side by side, which share lines with other tiles': 167 us with it, 138 without.  Solo tiles are few keys of small caches.
        Held& a = args();
        const int32_t row = (a.a.D + 31) / 32 * 16;
        if (!Solo && a.kc.cs.token == row && a.vc.cs.token == row) narrow_of<NQ, Solo, 2>(t);
        else narrow_of<NQ, Solo, 0>(t);
    }
    // kStream: how loads treat the caches (2: as of a stream).
    template <int NQ, bool Solo, int kStream>
    __device__ __forceinline__ void narrow_of(const Tile& t)
    {
        constexpr int KS = DP / 32, DT = DP / 16, NB = kNarrowKeys / RK_BLOCK_TOKENS;     // blocks of a step
        constexpr int kSets = NQ == 1 || DP < 128 ? 2 : 1;      // steps whose codes are under way or in registers
        const int lane = afresh(threadIdx.x & 63);
        const int g = lane >> 4, col = lane & 15;
        Held& a = args();
        u32x4 q[NQ][KS];
        int32_t last[NQ];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            const int32_t r = 16 * n + col;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) q[n][ks] = query_of(a.a, t, r, piece_of(ks, g));
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
        const int32_t n_blocks = a.a.n_blocks, D = a.a.D;
        Side k_side = side(a.kc, a, t.head), v_side = side(a.vc, a, t.head);
        const int32_t k_bytes = k_side.code_bytes, k_powers = k_side.power_bytes, v_bytes = v_side.code_bytes, v_powers = v_side.power_bytes;
        const Places k_at = places(a.kc, a.a.D, col, g), v_at = places(a.vc, a.a.D, col, g);
        uint32_t v_read[kTurn / 2];
        {
            const uint32_t vr = 4 * g + (col >> 2);
#pragma unroll
            for (int x = 0; x < kTurn / 2; ++x)
                v_read[x] = vr * kRow + (((2 * x + ((lane & 3) >> 1)) ^ turn(vr)) << 4) + 8 * (lane & 1);
        }
        const uint32_t vals = tile + wave * (64 * kRow);
        // this wavefront's steps: of each 4 NB blocks (of a workgroup's tile) NB from NB wave on, or all of them
        constexpr int kKeys = Solo ? kNarrowKeys : kWaves * kNarrowKeys, kBlocks = kKeys / RK_BLOCK_TOKENS;
        const int32_t first_block = t.block0 + (Solo ? 0 : NB * wave);
        int32_t s1 = (t.keys_end - first_block * RK_BLOCK_TOKENS + kKeys - 1) / kKeys;
        s1 = s1 < t.s1 ? s1 : t.s1;
        int32_t s = t.s0, id[NB];
        Numbers<NB, 4> numbers(t, first_block, kBlocks, n_blocks, s, lane);
        uint32_t bad = 0, any_bad = 0, next_bad[kSets] = {};
        Codes k_raw[kSets][NB], v_raw[kSets][NB];
        // (Loads are made in any case, of nothing behind the last step: of loads that may or may not have been made, all later ones are
        // waited for with the earlier.)
        auto for_step = [&](int32_t x) {
            const bool some = x < s1;
            k_side.code_bytes = some ? k_bytes : 0;
            k_side.power_bytes = some ? k_powers : 0;
            v_side.code_bytes = some ? v_bytes : 0;
            v_side.power_bytes = some ? v_powers : 0;
        };
        auto issue_keys = [&](auto u, int32_t x) {
            next_bad[u] = numbers.of(x, id, lane);
            for_step(x);
#pragma unroll
            for (int b = 0; b < NB; ++b) k_raw[u][b] = codes_of<kStream>(k_side, id[b], k_at);
            __builtin_amdgcn_sched_barrier(0);
            if (numbers.odd) {
#pragma unroll
                for (int b = 0; b < NB; ++b) keep_wide(k_raw[u][b]);
            }
        };
        auto issue_values = [&](auto u) {
#pragma unroll
            for (int b = 0; b < NB; ++b) v_raw[u][b] = codes_of<kStream>(v_side, id[b], v_at);
            __builtin_amdgcn_sched_barrier(0);
            if (numbers.odd) {
#pragma unroll
                for (int b = 0; b < NB; ++b) keep_wide(v_raw[u][b]);
            }
        };
        auto scores = [&](auto u, f32x4 (*sc)[NB]) {
            if (D % 32 != 0) {
#pragma unroll
                for (int b = 0; b < NB; ++b) end_at(k_raw[u][b], D, g);
            }
#pragma unroll
            for (int kt = 0; kt < NB; ++kt) {
#pragma unroll
                for (int n = 0; n < NQ; ++n) sc[n][kt] = f32x4{};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const u32x4 k = k_raw[u][kt].values(ks);
#pragma unroll
                    for (int n = 0; n < NQ; ++n) sc[n][kt] = mfma16<Half>(k, q[n][ks], sc[n][kt]);
                }
            }
        };
        auto weights = [&](f32x4 (*sc)[NB], u32x4 (*w)[NB / 2]) {
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float top = sc[n][0][0];
#pragma unroll
                for (int kt = 0; kt < NB; ++kt)
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
                for (int kt = 0; kt < NB; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; i += 2) {
                        const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kt][i], c, base));
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[n][kt][i + 1], c, base));
                        l[n] += x + y;
                        w[n][kt / 2][2 * (kt % 2) + (i >> 1)] = pack16<Half>(x, y);
                    }
            }
        };
        auto values = [&](int d, int c) {
            const uint32_t x = vals + c * (32 * kRow) + v_read[d % (kTurn / 2)] + (uint32_t)(d / (kTurn / 2) * (16 * kTurn));
            const u32x2 lo = lds_read_columns(x), up = lds_read_columns(x + 16 * kRow);
            return u32x4{lo.x, lo.y, up.x, up.y};
        };
        // The second product; values are read from LDS kAhead products before the one that takes them.
        auto product = [&](const u32x4 (*w)[NB / 2]) {
            constexpr int N = DT * (NB / 2), kAhead = 4;
            u32x4 v[kAhead];
#pragma unroll
            for (int x = 0; x < kAhead; ++x) v[x] = values(x % DT, x / DT);
#pragma unroll
            for (int x = 0; x < N; ++x) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int n = 0; n < NQ; ++n) o[n][x % DT] = mfma16<Half>(v[x % kAhead], w[n][x / DT], o[n][x % DT]);
                if (x + kAhead < N) v[x % kAhead] = values((x + kAhead) % DT, (x + kAhead) / DT);
            }
        };
        auto keys_read = [&](auto u) {
            bad = next_bad[u];
            issue_keys(u, s + kSets);
        };
        auto put_values = [&](auto u, bool some_behind) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (some_behind) only_rows(v_raw[u][b], t, first_block + kBlocks * s + b, bad >> b & 1, lane);
                place_values(v_raw[u][b], vals + b * (RK_BLOCK_TOKENS * kRow), lane);
            }
            issue_values(u);
        };
        constexpr std::integral_constant<int, 0> first{};
        constexpr std::integral_constant<int, kSets - 1> second{};
        if constexpr (Solo) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the LDS is the last tile's until here
        else __syncthreads();
        if (s < s1) {
            issue_keys(first, s);
            issue_values(first);
            if (kSets > 1) {
                issue_keys(second, s + 1);
                issue_values(second);
            }
        }
        const int32_t seen = all_see + 1 - first_block * RK_BLOCK_TOKENS - kNarrowKeys;       // the last step's first key that all see
        const int32_t open = seen < 0 ? 0 : seen / kKeys + 1, s_open = open < s1 ? open : s1;
        auto open_step = [&](auto u) {           // a step whose keys every row sees
            f32x4 sc[NQ][NB];
            u32x4 w[NQ][NB / 2];
            scores(u, sc);
            keys_read(u);
            weights(sc, w);
            put_values(u, false);
            product(w);
        };
        auto any_step = [&](auto u) {
            const int32_t key0 = (first_block + kBlocks * s) * RK_BLOCK_TOKENS;
            const bool masked = key0 + kNarrowKeys - 1 > all_see;
            f32x4 sc[NQ][NB];
            u32x4 w[NQ][NB / 2];
            scores(u, sc);
            keys_read(u);
            any_bad |= bad;
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int kt = 0; kt < NB; ++kt)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (key0 + 16 * kt + 4 * g + i > last[n] || ((bad >> kt) & 1)) sc[n][kt][i] = -INFINITY;
            weights(sc, w);
            put_values(u, true);
            if (masked && t.mask && t.tokens > 1) {                      // (as for wide tiles, of values of the wavefront's own)
                u16x2 most = {0, 0};
#pragma unroll 4
                for (int x = lane; x < kNarrowKeys * NC; x += 64) most = without_sign(most, lds_read16(vals + 16 * x));
                if (__any(not_finite<Half>(__builtin_bit_cast(uint32_t, most)))) {
#pragma unroll 1
                    for (int x = 0; x < kNarrowKeys; ++x)
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
                    for (int x = lane; x < kNarrowKeys * NC; x += 64) {
                        const u32x4 v = lds_read16(vals + 16 * x);
                        lds_write16(vals + 16 * x, u32x4{finite_or_zero<Half>(v.x), finite_or_zero<Half>(v.y),
                                                         finite_or_zero<Half>(v.z), finite_or_zero<Half>(v.w)});
                    }
                    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                }
            }
            product(w);
        };
        if constexpr (kSets == 1) {
            for (; s < s_open && !next_bad[0]; ++s) open_step(first);
            for (; s < s1; ++s) any_step(first);
        } else {
            while (s + 1 < s_open && !(next_bad[0] | next_bad[1])) {
                open_step(first);
                ++s;
                open_step(second);
                ++s;
            }
            while (s < s1) {
                any_step(first);
                if (++s == s1) break;
                any_step(second);
                ++s;
            }
        }
        this->template narrow_out<NQ, Solo, DT>(t, o, m, l, vals, lane);
        if (any_bad) report_bad();
    }
};

}  // namespace rk

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
        if (a.n_blocks > 1 && (c.cs.block >> 32 || c.ss.block >> 32)) return fail(RK_EUNSUPPORTED, "%s: a block stride past 2^32 bytes", name);
    }
    if (a.B == 0 || a.T == 0) return RK_OK;
    if (!attention_arrays(a) || (a.n_blocks > 0 && (!a4->k.codes || !a4->k.scales || !a4->v.codes || !a4->v.scales)))
        return fail(RK_EINVAL, "%s: NULL array", name);
    if (((uintptr_t)a.q | (uintptr_t)a.out | (uintptr_t)a4->k.codes | (uintptr_t)a4->v.codes) % 16)
        return fail(RK_EINVAL, "%s: an array is not aligned to 16 bytes", name);
    AttendFp4Args p{};
    p.kc = a4->k;
    p.vc = a4->v;
    return attention_call<AttendFp4>(a, p, workspace, ws_bytes, stream, name);
}

}  // extern "C"
