// attend.hip -- rk_prefix_attention: the entry points, and the kernels of 16-bit caches.
#include "attend.h"

namespace rk {

// Tiles over a 16-bit cache.
template <int DP, bool Half>
struct Attend : AttendBase<DP, Half> {
    typedef AttendArgs Args;
    using Base = AttendBase<DP, Half>;
    using Base::NC, Base::NI, Base::kRow, Base::kTurn, Base::turn, Base::p, Base::tile, Base::join, Base::wave, Base::G, Base::c;
    using Base::block_id, Base::rows_of, Base::bad_block, Base::report_bad, Base::token_of, Base::query_of, Base::strays, Base::divisor,
        Base::out_row, Base::put_lse;
    static constexpr int kNarrowKeys = 32;            // of a wavefront in a narrow step
    // A wide or narrow step takes about 2 us, what comes before a wide tile's first and after its last 12 (a prologue without
    // products, and results out).  Measured: ends of 4 for narrow and solo ones, 128 requests on one prefix 82 -> 87 us, of 8,
    // groups of 200 62 -> 70; of 10 or 16 for wide ones, 0-5% more.
    static constexpr uint32_t kStepCost[3] = {2, 2, 2}, kEndsCost[3] = {12, 6, 6};
    static_assert(kLeast >= kStepCost[kWide] && kLeast >= kStepCost[kNarrow], "a step begins in every piece of a tile");

    const uint32_t last_piece;                        // of a row: the bytes before it
    // the pieces of a block that the lane loads: whole rows a load, or not
    static constexpr bool kEven = 64 % NC == 0;
    uint32_t k_at[kEven ? 2 : NI], v_at[kEven ? 2 : NI];

    __device__ __forceinline__ Attend(const AttendArgs& args, uint32_t lds, float* j, float scale)
        : Base(args, lds, j, scale), last_piece(2 * args.a.D - 16)
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
        {
            // As query_of gives them, but the tile's first row in the place of those that are not there, whose results nobody reads: where D
            // fills its rows nothing waits for these loads here.  (600 prompts of 300 tokens 1,003 us, 1,050 with query_of.)
            const bool there = token_of(r) < t.tokens;
            const int32_t tok = there ? token_of(r) : 0, head = there ? r - tok * G : 0;
            const uint16_t* row = (const uint16_t*)p.a.q + (t.token + (int64_t)tok) * p.a.q_token + (t.head * G + head) * p.a.q_head;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int32_t at = 8 * (2 * ks + hi);
                q[ks] = *reinterpret_cast<const u32x4*>(row + (at < p.a.D ? at : 0));
            }
            if (p.a.scale < 0.0f || p.a.D < DP) {
                const uint32_t sign = p.a.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) q[ks] = (q[ks] ^ sign) & (8 * (2 * ks + hi) < p.a.D ? 0xffffffffu : 0u);
            }
        }
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
        this->template wide_out<DT>(t, o, m, l, r, lane);
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
            for (int ks = 0; ks < KS; ++ks) q[n][ks] = query_of(p.a, t, r, 4 * ks + g);
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
        constexpr int kKeys = Solo ? kNarrowKeys : kWaves * kNarrowKeys, kBlocks = kKeys / RK_BLOCK_TOKENS;
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
        this->template narrow_out<NQ, Solo, DT>(t, o, m, l, keys, lane);
    }
};

}  // namespace rk

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
    AttendArgs p{};
    return attention_call<Attend>(*a, p, workspace, ws_bytes, stream, name);
}

}  // extern "C"
