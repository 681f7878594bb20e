// Differential attention: out = norm(o_1 - lambda o_2), o_m = softmax(scale q_m K_m^T) V.
//
// A KV head of the pools is [K_1 | K_2], two maps' keys of d channels each, beside V of 2d.  With the query of map m in its half of
// a row of 2d channels and zeros in the other, scale q_m K_m^T is an ordinary score of that head.  So plans, their tasks and partial
// rows are the ordinary ones, with two query heads for every head of the result, and K_1, K_2 and V are read once for both
// maps.  The zeros themselves are nowhere: times an infinite key of the other map they would be NaN.
//  * The stream path runs tasks of at most sixteen rows, and with 64 channels those of up to 32 in plans without packs.  A tile's
//    sixteen rows, of either map in turn, are multiplied with both halves of the keys, a product each, and a row takes that of its
//    own map.  It takes the matrix instructions of an ordinary row (twice what two tiles of 64 channels, a map each, would need).
//  * Larger tasks run in the path below, where a wave's rows are all of one map and only that map's half of the keys is multiplied.
//  * A reduction folds both rows of a head, subtracts and normalises; where every request has a single partial result the attention
//    kernel does that itself (store_finished_pairs).
#include "kernels.hpp"

namespace codec {
namespace {

// ---- tasks of more than sixteen rows ---------------------------------------------------------------------
//
// A wave owns 32 rows of one map, pairs 32 g .. 32 g + 31 of the task (pair p is the task's rows 2p and 2p + 1), and runs 32 x 32 x 16
// tiles: d / 16 k-steps of scores S^T = K_m Q_m^T and 2 * D / 32 matrix instructions of O^T += V^T P^T in a block of 32 tokens, where
// rows of either map in turn would take 2 * d / 16 k-steps.  Blocks are copied HBM -> LDS asynchronously into a ring of all of the CU's LDS, K is
// read by 16 bytes a lane and V by transposing reads (swizzles below).
//
// A step is NB blocks between two barriers, the row groups' waves taking turns with them (SHARE); S slots hold blocks, so that
// S - NB of them are on their way when a step starts.  In a wave the scores of a block and the accumulation of its block before are one
// stream of matrix instructions, between which stand the exponentials of the block before, the reads of V and the copies.  ns a
// block, K and V out of L2, all CUs busy (with the accumulation, the scores, the reads and the exponentials one after the other):
// 256 channels, 32 pairs 514 (763), 64 pairs 830 (1125); 128 channels 32, 64, 128 pairs 286 (379), 443 (518), 771 (973); 64 channels
// 170 (229), 284 (372), 512 (619).  Out of HBM tasks of up to 64 pairs run at what HBM gives, 6.5 to 6.8 TB/s.
template <int D, int GROUPS>
struct PairPath {
    static constexpr int kWaves = kernel_waves(kFormWide, D), kUnits = 2 * GROUPS;
    static constexpr int kRowBytes = D * 2, kHalf = 32 * kRowBytes, kBlock = 2 * kHalf;      // K (or V) of a block; both
    static constexpr int kLds = 163840, kSlots = kLds / kBlock;                                 // 20, 10, 5
    // 256 channels: 32 pairs are two units for four waves; more are four
    static constexpr int kBlocks = D == 256 ? (GROUPS == 1 ? 2 : 1) : 256 / D;
    static constexpr int kShare = kWaves / kUnits < kBlocks ? kWaves / kUnits : kBlocks;
    static constexpr int kMine = kBlocks * 4 / kWaves;      // blocks of a step of which a wave copies eight tokens
    static constexpr int kStride = kWaves / 4;              // from one of them to the next
    static constexpr int kPieces = 8 * kRowBytes / 1024;    // 1 KB copies of eight tokens of one pool
    static constexpr int kCopies = kMine * 2 * kPieces;     // copies of a wave in a step
    static constexpr int kAhead = kSlots - kBlocks;         // blocks requested when a step starts
    static constexpr int kOutstanding = (kSlots - 2 * kBlocks) * kCopies / kBlocks;         // copies that a step need not wait for
    static_assert(kUnits * kShare <= kWaves && kBlocks % kShare == 0 && kOutstanding < 64, "waves for all row groups and shares");
    static_assert(kAhead % kBlocks == 0 || kStride == 1, "a step's copies are requested together");
};

constexpr int kTurnMinLen = 2048;       // tokens of a slice; see token_block

// A wave-uniform address, in scalar registers also where the compiler has lost track of that.
__device__ __forceinline__ const char *uniform_pointer(const char *p)
{
    const uint64_t x = uint64_t(uintptr_t(p));
    return reinterpret_cast<const char *>(uintptr_t(uint64_t(uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x >> 32)))) << 32 |
                                                     uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(x)))));
}

// dma16 (kernels.hip) from a base that is in scalar registers already.
template <bool ONCE>
__device__ __forceinline__ void copy_1k(uint32_t lds_addr, uint32_t voff, const char *base)
{
    uint32_t m0_saved;
    if constexpr (ONCE)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3 nt\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_saved) : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, %3\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_saved) : "s"(lds_addr), "v"(voff), "s"(base) : "memory");
}

template <int DT, int D, int GROUPS, bool ONCE>
__device__ __forceinline__ void run_pairs_of(const PairParams &P, const DevTask &t, int head, char *lds, RowStore how)
{
    using T = PairPath<D, GROUPS>;
    constexpr int RB = T::kRowBytes, KS = D / 32, CT = D / 32, NB = T::kBlocks, S = T::kSlots, SHARE = T::kShare;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = opaque_lane();
    const int l32 = lane & 31, kg = lane >> 5, l16 = lane & 15, grp = lane >> 4;
    const int pairs = t.n_req * P.group / 2;
    const int unit = wave % T::kUnits, phase = wave / T::kUnits;
    const int map = unit & 1, pair0 = (unit >> 1) * 32;
    const bool live = pair0 < pairs && phase < SHARE;       // else: the wave only helps moving blocks
    const SliceCtx c = make_ctx(P, t, head);
    const int nblk = (t.kv_len + 31) >> 5, nstep = (nblk + NB - 1) / NB;

    // Copies, TPC tokens each.  A K row keeps its 16-byte column g in slot g ^ fk(token) and a V row in slot g ^ fv(token): eight lanes of
    // a K read, on eight tokens, then meet eight different columns of the 256 bytes of banks, and the four tokens of 64 bytes that 32
    // lanes of a transposing V read take lie in its four quarters (64 channels: a row is half of the banks).
    constexpr int LPR = RB / 16, TPC = 64 / LPR, MINE = T::kMine;
    auto fk = [](int token) { return D == 64 ? (token >> 1) & 7 : token & 15; };
    auto fv = [](int token) { return D == 64 ? ((token >> 1) & 1) << 2 : (token & 3) << 2; };
    const int my_block = wave >> 2, my_token = (wave & 3) * 8;
    const uint32_t lds_base = uint32_t(uintptr_t(lds));
    uint32_t voff_k[T::kPieces], voff_v[T::kPieces];
#pragma unroll
    for (int i = 0; i < T::kPieces; ++i) {
        const int in_copy = lane / LPR, token = my_token + i * TPC + in_copy;
        voff_k[i] = uint32_t(i * TPC + in_copy) * c.token_bytes + uint32_t(((lane % LPR) ^ fk(token)) << 4);
        voff_v[i] = uint32_t(i * TPC + in_copy) * c.token_bytes + uint32_t(((lane % LPR) ^ fv(token)) << 4);
    }
    // Tasks that read a slice beside one another (the packs of a node's rows) would ask L2 for the same lines at the same time.  With 256
    // channels, where a block has only up to 64 pairs of work, each takes every eight blocks from another one on: 564 -> 440 ns a block for a
    // root alone.  32/8 heads of two maps of 128 channels, requests on a root of 32768 tokens, us: 16 requests 100 -> 91, 32 174 -> 149,
    // 64 318 -> 245, 128 601 -> 459; a forest whose other tasks set the time 449 -> 459.  Slices of 1024 tokens lose 5 %, and up to
    // 128 channels there is nothing to gain (0.97 to 1.05).
    constexpr bool TURN = D == 256 && !ONCE;
    int turn = 0;
    if constexpr (TURN) {
        const uint32_t nth = uint32_t(t.q_off) / uint32_t(t.n_req);     // of the packs, for all but the last
        if (!(t.flags & kTaskReadOnce) && t.kv_len >= kTurnMinLen) turn = int((nth & 1) << 2 | (nth & 2) | (nth >> 2 & 1));
    }
    auto token_block = [&](int block) {                     // eight whole blocks, none of them the last
        return TURN && (block | 7) < nblk - 1 ? (block & ~7) | ((block + turn) & 7) : block;
    };
    // eight tokens past the end of the slice are redirected to its first ones (masked later): no address leaves the slice's
    // pages, and every step has the same number of copies
    auto first_token = [&](int block) {
        const int tok0 = token_block(block) * 32 + my_token;
        return tok0 >= c.kv_len ? 0 : tok0;
    };
    auto block_of = [&](int first, int u) { return first + my_block + u * T::kStride; };     // that the wave copies, of NB from `first` on
    auto page_issue = [&](int block) { return uniform_load(c.pages, first_token(block) >> c.page_shift); };
    auto slot_of = [&](int block) { return lds_base + uint32_t(block % S) * T::kBlock; };
    // copies of the wave's blocks of a step, each K first
    const char *k_head = uniform_pointer(c.k_head), *v_head = uniform_pointer(c.v_head);
    struct Copies {
        uint32_t at[MINE];
        const char *k[MINE], *v[MINE];
    };
    auto copies_of = [&](int first, const int (&pg)[MINE]) __attribute__((always_inline)) {        // pg: their page_issue
        Copies x;
#pragma unroll
        for (int u = 0; u < MINE; ++u) {
            const int block = block_of(first, u);
            const int64_t off = page_offset(c, pg[u], first_token(block) & c.page_mask);
            x.at[u] = slot_of(block) + uint32_t(my_token) * RB;
            x.k[u] = k_head + off;
            x.v[u] = v_head + off;
        }
        return x;
    };
    auto copy = [&](const Copies &x, int n) __attribute__((always_inline)) {
        const int u = n / (2 * T::kPieces), i = n % (2 * T::kPieces), piece = i % T::kPieces;
        if (i < T::kPieces) copy_1k<ONCE>(x.at[u] + piece * 1024, voff_k[piece], x.k[u]);
        else                copy_1k<ONCE>(x.at[u] + T::kHalf + piece * 1024, voff_v[piece], x.v[u]);
    };
    auto request_block = [&](const Copies &x, int u) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < 2 * T::kPieces; ++n) copy(x, u * 2 * T::kPieces + n);
    };
    auto request = [&](int first, const int (&pg)[MINE]) __attribute__((always_inline)) {
        const Copies x = copies_of(first, pg);
#pragma unroll
        for (int u = 0; u < MINE; ++u) request_block(x, u);
    };

    // Operand reads, as in the dense path.  K, k-step ks: lane (l32, kg) reads 16-byte column map * D / 16 + 2 * ks + kg of token l32.  V,
    // channel tile ct, k-step tt, h: lane (k, q) of lane group (kg, ch) addresses token 16 * tt + 8 * h + 4 * kg + k, channels
    // 32 * ct + 16 * ch + 4 * q .. +3, and receives channel 32 * ct + l32 of tokens 16 * tt + 8 * h + 4 * kg .. +3.
    const uint32_t k_lane = uint32_t(l32 * RB + ((kg ^ fk(l32)) << 4)) ^ uint32_t(map * (D / 16) << 4);
    const int vtok = 4 * kg + (l16 >> 2), vq = l16 & 3;
    const uint32_t v_lane = uint32_t(T::kHalf + vtok * RB + (((2 * (grp & 1) + (vq >> 1)) ^ fv(vtok)) << 4) + 8 * (vq & 1));
    typedef const u32x4 __attribute__((address_space(3))) *lds_u32x4_ptr;
    typedef __attribute__((ext_vector_type(4))) short s16x4;
    typedef s16x4 __attribute__((address_space(3))) *lds_s16x4_ptr;

    u32x4 qb[KS];           // row l32 (of pair pair0 + l32), channels 16 * ks + 8 * kg .. +7 of the map
    f32x16 o[CT];           // O^T: row l32, channel 32 * ct + 8 * (r / 4) + 4 * kg + r % 4
    u32x4 kr[KS], p[2];
    u32x4 vr[CT][2];
    f32x16 sc[2];           // scores of the wave's even and odd blocks: row l32, token 8 * (r / 4) + 4 * kg + r % 4
    float m = kNoReference, l2[2] = {0.f, 0.f};
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[ct][r] = 0.f;

    auto reference = [&](const f32x16 &s) __attribute__((always_inline)) {
        float lm = s[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) lm = fmaxf(lm, s[r]);
        lm *= P.scale_log2e;
        if (__any(lm > m + kLag)) {                         // see raise_reference
            const float m_new = fmaxf(m, fmaxf(lm, __shfl_xor(lm, 32))), alpha = fast_exp2(m - m_new);
            l2[0] *= alpha;
            l2[1] *= alpha;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[ct][r] *= alpha;
            m = m_new;
        }
    };
    // Weights are rounded to 16 bits, which the matrix instructions take (fp16 by 2^-11 of themselves, bf16 by 2^-8), as in every path of ordinary
    // attention.  The row sum adds the rounded ones: a result is off by the roundings' share of the values' distances from it, not of
    // the values.  What is subtracted later are two such results, in 32 bits.
    auto exponential_pair = [&](const f32x16 &s, int tt, int d) __attribute__((always_inline)) {
        p[tt][d] = pack2<DT>(fast_exp2(__builtin_fmaf(s[8 * tt + 2 * d], P.scale_log2e, -m)),
                             fast_exp2(__builtin_fmaf(s[8 * tt + 2 * d + 1], P.scale_log2e, -m)));
        l2[tt] = add_pair<DT>(p[tt][d], l2[tt]);
    };
    // n of `of` steps through four pairs of exponentials
    auto exponentials = [&](const f32x16 &s, int tt, int n, int of) __attribute__((always_inline)) {
#pragma unroll
        for (int d = n * 4 / of; d < (n + 1) * 4 / of; ++d) exponential_pair(s, tt, d);
    };
    auto load_value = [&](uint32_t at, int ct, int tt) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t from = ((at + v_lane) ^ uint32_t(ct << 6)) + (16 * tt + 8 * h) * RB;
            const uint2 w = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_s16x4_ptr>(uintptr_t(from))));
            vr[ct][tt][2 * h] = w.x;
            vr[ct][tt][2 * h + 1] = w.y;
        }
    };
    // The wave's next block, whose scores go to set X; the other set's are those of the block before, whose V is in registers (FIRST:
    // there is none).  COPY: the copies x of a step are issued, too, one by one between the matrix instructions: all at once they keep the wave,
    // and those of the other SIMDs, until the last of them has been taken (a CU takes 64 bytes a cycle).
    auto compute = [&](int block, auto set, auto first, auto copying, const Copies &x) __attribute__((always_inline)) {
        constexpr int X = decltype(set)::value, kAll = KS + 2 * CT;
        constexpr bool COPY = decltype(copying)::value;
        const uint32_t at = slot_of(block);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) kr[ks] = *reinterpret_cast<lds_u32x4_ptr>(uintptr_t((at + k_lane) ^ uint32_t(ks << 5)));
        __builtin_amdgcn_sched_barrier(0);
        f32x16 &acc = sc[X];
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[r] = 0.f;
        if constexpr (decltype(first)::value) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) acc = mfma32<DT>(kr[ks], qb[ks], acc);
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                load_value(at, ct, 0);
                load_value(at, ct, 1);
            }
        } else {
            auto behind = [&](int i) __attribute__((always_inline)) {      // matrix instruction i of kAll
                if constexpr (COPY) {
#pragma unroll
                    for (int n = i * T::kCopies / kAll; n < (i + 1) * T::kCopies / kAll; ++n) copy(x, n);
                }
                __builtin_amdgcn_sched_barrier(0);
            };
            const f32x16 &s = sc[1 - X];
            reference(s);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                acc = mfma32<DT>(kr[ks], qb[ks], acc);
                exponentials(s, 0, ks, KS);
                behind(ks);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                o[ct] = mfma32<DT>(vr[ct][0], p[0], o[ct]);
                exponentials(s, 1, ct, CT);
                behind(KS + ct);
            }
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) {
                o[ct] = mfma32<DT>(vr[ct][1], p[1], o[ct]);
                load_value(at, ct, 0);
                if (ct > 0) load_value(at, ct - 1, 1);
                behind(KS + CT + ct);
            }
            load_value(at, CT - 1, 1);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // the last of the wave's blocks, in set X
    auto complete = [&](int block, auto x) __attribute__((always_inline)) {
        constexpr int X = decltype(x)::value;
        f32x16 &s = sc[X];
        const int valid = c.kv_len - block * 32;
        if (valid < 32) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = 8 * (r >> 2) + 4 * kg + (r & 3) >= valid ? -INFINITY : s[r];
        }
        reference(s);
        exponentials(s, 0, 0, 1);
        exponentials(s, 1, 0, 1);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int ct = 0; ct < CT; ++ct) o[ct] = mfma32<DT>(vr[ct][tt], p[tt], o[ct]);
    };

    // V rows of the last block past the end of the slice count as zero: each wave clears the ones that it copied
    auto clear_tail = [&]() __attribute__((always_inline)) {
        const int valid = c.kv_len - (nblk - 1) * 32;
        if ((nblk - 1) % T::kStride != my_block) return;
        const uint32_t at = slot_of(nblk - 1) + T::kHalf + uint32_t(my_token) * RB + uint32_t(lane) * 16;
#pragma unroll
        for (int n = 0; n < T::kPieces; ++n)
            if (my_token + n * TPC + lane / LPR >= valid)
                *reinterpret_cast<u32x4 __attribute__((address_space(3))) *>(uintptr_t(at + n * 1024)) = u32x4{0u, 0u, 0u, 0u};
    };

    // Start: the rows' requests and the page ids, read together; then the first step's copies and the query rows.  Waiting for the
    // rows (the compiler waits for every load in flight) waits for that step too, so the others are requested behind it.
    constexpr int kRounds = (T::kAhead + NB - 1) / NB;      // of requests ahead of the first step
    int pg[kRounds][MINE], pg_next[MINE];
#pragma unroll
    for (int i = 0; i < kRounds; ++i)
#pragma unroll
        for (int u = 0; u < MINE; ++u) pg[i][u] = page_issue(block_of(i * NB, u));
#pragma unroll
    for (int u = 0; u < MINE; ++u) pg_next[u] = page_issue(block_of(T::kAhead, u));
    const bool row_live = pair0 + l32 < pairs;
    {
        const int row = row_live ? 2 * (pair0 + l32) + map : map, qi = row / P.group, hj = row - qi * P.group;
        int req = t.single_req >= 0 ? t.single_req : P.node_q[t.q_off + qi];
        pin(req);
        const char *qp = static_cast<const char *>(P.q) + (int64_t(req) * P.h_q + int64_t(head) * P.group + hj) * D + kg * 16;
        request(0, pg[0]);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            qb[ks] = ld16(qp + ks * 32);
            if (!row_live) qb[ks] = u32x4{0u, 0u, 0u, 0u};
        }
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) pin(qb[ks]);
    }
#pragma unroll
    for (int i = 1; i < kRounds; ++i)
        if (i * NB < nblk) {
            const Copies x = copies_of(i * NB, pg[i]);
#pragma unroll
            for (int u = 0; u < MINE; ++u)
                if (i * NB + u * T::kStride < T::kAhead) request_block(x, u);
        }
    auto meet = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(0xC07F);     // V of the step before is in registers
        __syncthreads();                        // everyone's part has landed; step j - 1 has been read by all
    };
    // the blocks of step j have landed once at most the copies requested after them are outstanding
    auto enter_step = [&](int j) __attribute__((always_inline)) {
        if (NB * j + T::kAhead <= nblk) __builtin_amdgcn_s_waitcnt(vmcnt_imm(T::kOutstanding));
        else                            __builtin_amdgcn_s_waitcnt(0x0F70);
        if (j == nstep - 1 && (c.kv_len & 31)) clear_tail();
        meet();
    };
    auto pages_of = [&](int first) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < MINE; ++u) pg_next[u] = page_issue(block_of(first, u));
    };
    if (live) {
        int last = -1;                          // the wave's last block so far
        using yes = std::true_type;
        using no = std::false_type;
        // FULL: all blocks of step j and of the copies behind it exist
        auto step = [&](int j, auto set, auto first, auto full) __attribute__((always_inline)) {
            constexpr int X = decltype(set)::value;
            constexpr bool FIRST = decltype(first)::value, FULL = decltype(full)::value;
            const int next = NB * j + T::kAhead;
            Copies x{};
            if constexpr (FULL) {
                __builtin_amdgcn_s_waitcnt(vmcnt_imm(T::kOutstanding));
                x = copies_of(next, pg_next);
                meet();
                pages_of(next + NB);
            } else {
                enter_step(j);
                if (next < nblk) {
                    request(next, pg_next);
                    pages_of(next + NB);
                }
            }
            auto own = [&](auto n) __attribute__((always_inline)) {
                constexpr int U = decltype(n)::value;
                if constexpr (U < NB / SHARE) {
                    const int block = NB * j + phase + U * SHARE;
                    if (!FULL && block >= nblk) return;
                    compute(block, std::integral_constant<int, (X + U) % 2>{}, std::integral_constant<bool, FIRST && U == 0>{},
                            std::integral_constant<bool, FULL && U == 0>{}, x);
                    last = block;
                }
            };
            static_assert(NB / SHARE <= 4, "blocks of a step");
            own(std::integral_constant<int, 0>{});
            own(std::integral_constant<int, 1>{});
            own(std::integral_constant<int, 2>{});
            own(std::integral_constant<int, 3>{});
        };
        constexpr bool kEven = NB / SHARE % 2 == 0;             // a step leaves the sets as they were
        using zero = std::integral_constant<int, 0>;
        using other = std::integral_constant<int, kEven ? 0 : 1>;
        step(0, zero{}, yes{}, no{});
        int j = 1;
#pragma unroll 1
        for (; NB * (j + 1) + T::kAhead < nblk; j += 2) {
            step(j, other{}, no{}, yes{});
            step(j + 1, zero{}, no{}, yes{});
        }
#pragma unroll 1
        for (; j < nstep; j += 2) {
            step(j, other{}, no{}, no{});
            if (j + 1 < nstep) step(j + 1, zero{}, no{}, no{});
        }
        if (last >= 0) {
            const bool odd = (kEven ? (last % NB) / SHARE : last / NB) & 1;
            if (odd) complete(last, std::integral_constant<int, 1>{});
            else     complete(last, std::integral_constant<int, 0>{});
        }
    } else {
#pragma unroll 1
        for (int j = 0; j < nstep; ++j) {
            enter_step(j);
            const int next = NB * j + T::kAhead;
            if (next < nblk) {
                request(next, pg_next);
                pages_of(next + NB);
            }
        }
    }
    float l = l2[0] + l2[1];
    l += __shfl_xor(l, 32);
    __syncthreads();                        // every block has been read: the ring is free

    // the waves of a row group hand their states over pairwise: phases [h, 2h) to phases [0, h)
    constexpr int kState = (16 * CT + 2) * 64;              // floats
    static_assert(GROUPS * SHARE * kState * 4 <= T::kLds || SHARE == 1, "hand-over areas fit");
    if constexpr (SHARE > 1) {
#pragma unroll 1
        for (int h = SHARE / 2; h >= 1; h >>= 1) {
            float *x = reinterpret_cast<float *>(lds) + (phase % h * 2 * GROUPS + unit) * kState + lane;
            if (phase >= h && phase < 2 * h) {
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[(ct * 16 + r) * 64] = o[ct][r];
                x[16 * CT * 64] = m;
                x[(16 * CT + 1) * 64] = l;
            }
            __syncthreads();
            if (phase < h) {
                const float m2 = x[16 * CT * 64], mm = fmaxf(m, m2), a = weight(m, mm), b = weight(m2, mm);
                l = l * a + x[(16 * CT + 1) * 64] * b;
                m = mm;
#pragma unroll
                for (int ct = 0; ct < CT; ++ct)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[ct][r] = o[ct][r] * a + x[(ct * 16 + r) * 64] * b;
            }
            __syncthreads();
        }
    }

    // Partial rows go out through LDS, up to 128 channels of the wave's rows at a time, so that a store instruction covers
    // consecutive memory of a few rows (see dense32_wave).
    if (live && phase == 0) {
        const bool tiled = (t.flags & kTaskTiles) != 0;
        const int tile_rows = (t.flags >> kTaskTileShift) & 255, stride = ~t.single_req;
        const int last_tile = tiled ? (2 * pairs - 1) / tile_rows : 0, last_back = t.flags >> kTaskLastShift;
        auto place = [&](int row) {                         // of a row of the task among the partial rows
            if (!tiled) return int64_t(row);
            const int tile = row / tile_rows;
            return int64_t(tile) * stride + (row - tile * tile_rows) - (tile == last_tile ? last_back : 0);
        };
        float *po = P.part_o + (int64_t(head) * P.part_rows + t.part_row_base) * D;
        float *pml = P.part_ml + (int64_t(head) * P.part_rows + t.part_row_base) * 2;
        if (tiled && how == kRowsThrough && int64_t(last_tile + 1) * stride * (D * 4) >= int64_t(1) << 31) how = kRowsPlain;   // see run_tile_of
        constexpr int kWidth = D < 128 ? D : 128, kPitch = kWidth * 4 + 16, kLanes = kWidth / 4, kRows = 64 / kLanes;
        static_assert(T::kUnits * 32 * kPitch <= T::kLds, "staging areas fit");
        typedef f32x4 __attribute__((address_space(3))) *lds_f32x4_ptr;
        const uint32_t area = lds_base + uint32_t(unit) * 32 * kPitch, put = area + uint32_t(l32) * kPitch + uint32_t(kg) * 16;
        const uint32_t get = area + uint32_t(lane / kLanes) * kPitch + uint32_t(lane % kLanes) * 16;
        auto store = [&](auto h) __attribute__((always_inline)) {
            constexpr RowStore HOW = decltype(h)::value;
            if (row_live && kg == 0) st8_partial<HOW>(pml + place(2 * (pair0 + l32) + map) * 2, m, l);
#pragma unroll
            for (int u = 0; u < D / kWidth; ++u) {
#pragma unroll
                for (int ct = 0; ct < kWidth / 32; ++ct)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const f32x16 &x = o[u * (kWidth / 32) + ct];
                        *reinterpret_cast<lds_f32x4_ptr>(uintptr_t(put + ct * 128 + q * 32)) = f32x4{x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]};
                    }
                __builtin_amdgcn_wave_barrier();            // LDS serves a wave's accesses in order: no wait needed
#pragma unroll
                for (int j = 0; j < 32 / kRows; ++j) {
                    const int pair = pair0 + j * kRows + lane / kLanes;
                    const f32x4 x = *reinterpret_cast<lds_f32x4_ptr>(uintptr_t(get + j * kRows * kPitch));
                    if (pair < pairs) {
                        const int64_t off = place(2 * pair + map) * D + u * kWidth + (lane % kLanes) * 4;
                        if constexpr (HOW == kRowsThrough) st16_rows<HOW>(rows_at(po, -1), int(off) * 4, x);
                        else                               st16_partial<HOW>(po + off, x);
                    }
                }
                __builtin_amdgcn_wave_barrier();
            }
        };
        if (how == kRowsThrough) store(std::integral_constant<RowStore, kRowsThrough>{});
        else                     store(std::integral_constant<RowStore, kRowsPlain>{});
    }
    __syncthreads();                        // the staging areas are free for the next task
}

// Row groups of 32 pairs: one, two or four, times two maps, over the waves.  Slices that one task alone reads are read with the
// streaming hint, but not under more than 64 pairs.  32 nodes of 4096 tokens and eight KV heads, us with / without it: 256 channels
// 173 / 195 (16 pairs), 179 / 202 (32), 187 / 214 (64); 128 channels 89 / 101, 91 / 104, 98 / 113, but 198 / 147 (128 pairs).
template <int DT, int D>
__device__ __forceinline__ void run_pairs(const PairParams &P, const DevTask &t, int head, char *lds, RowStore how)
{
    const int pairs = t.n_req * P.group / 2;
    auto run = [&](auto groups) __attribute__((always_inline)) {
        constexpr int GROUPS = decltype(groups)::value;
        if (t.flags & kTaskReadOnce) run_pairs_of<DT, D, GROUPS, true>(P, t, head, lds, how);
        else                         run_pairs_of<DT, D, GROUPS, false>(P, t, head, lds, how);
    };
    if (pairs <= 32)                    run(std::integral_constant<int, 1>{});
    else if (D == 256 || pairs <= 64)   run(std::integral_constant<int, 2>{});
    else if constexpr (D != 256)        run_pairs_of<DT, D, 4, false>(P, t, head, lds, how);
}

// The kernel of differential attention: pac_kernel's task loop (there is more about it), for two launches or finished rows.
template <int DT, int FORM, int D>
__global__ void __launch_bounds__(kernel_waves(FORM, D) * 64, D > 128 ? 1 : 2) pair_kernel(const PairParams P)
{
    constexpr bool WIDE = FORM == kFormWide, FINISH = FORM == kFormFinish;
    constexpr int W = kernel_waves(FORM, D), kMerge = merge_bytes(W, stream_tiles(D), D);
    char *lds;
    if constexpr (WIDE) {
        static_assert(kMerge + W * solo_stage_bytes(D) <= PairPath<D, 1>::kLds, "staging areas fit the ring");
        lds = dyn_lds;
    } else {
        __shared__ __attribute__((aligned(16))) char static_lds[kMerge + W * solo_stage_bytes(D)];
        lds = static_lds;
    }
    const int head = blockIdx.x % P.h_kv, slot = blockIdx.x / P.h_kv;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    char *stage = lds + kMerge + wave * solo_stage_bytes(D);
    const RowStore early = int64_t(P.part_rows) * P.h_kv * (D * 4) > kEarlyThroughBytes ? kRowsThrough : kRowsPlain;
    const RowStore late = last_rows_through(P.h_kv) ? kRowsThrough : kRowsPlain;
    // Stream tasks that alone read their slice go round the KV heads where pac_kernel's do ([token][head] pools): 300 contexts of up to
    // 2000 tokens, eight heads of 64 channels 143 -> 113 us, 200 of up to 4000 of 128 channels 306 -> 285.  A choice at run
    // time: a kernel for each takes long to build.
    auto head_of = [&](const DevTask &t, int i) __attribute__((always_inline)) {
        if constexpr (FINISH || D <= 128) {
            if ((t.flags & kTaskReadOnce) && (FINISH || P.turns)) return int(uint32_t(head + i) % uint32_t(P.h_kv));
        }
        return head;
    };
    auto run_tasks = [&](const DevTask *recs, int i, int end, bool marked, bool more) __attribute__((always_inline)) {
#pragma unroll 1
        while (i < end) {
            const DevTask t = recs[i];
            const int n = marked ? t.solo_run : end - i;
            if (n >= 2) {                       // short tasks, a wave each
                int *next = reinterpret_cast<int *>(lds);
                if (threadIdx.x == 0) *next = W;
                __syncthreads();
                int k = wave;
#pragma unroll 1
                while (k < n) {
                    const DevTask mine = recs[i + k];
                    const int own = head_of(mine, i + k);
                    if (mine.flags & kTaskReadOnce) run_stream<DT, true, 1, 1, D, FINISH>(P, mine, own, lds, 0, stage);
                    else                            run_stream<DT, false, 1, 1, D, FINISH>(P, mine, own, lds, 0, stage);
                    k = 0;
                    if ((threadIdx.x & 63) == 0) k = atomicAdd(next, 1);
                    k = __builtin_amdgcn_readfirstlane(k);
                }
                __syncthreads();
                i += n;
                continue;
            }
            const int rows = t.n_req * P.group;
            if (rows <= 16) {
                const int own = head_of(t, i);
                if (t.flags & kTaskReadOnce) run_stream<DT, true, 1, W, D, FINISH>(P, t, own, lds, wave);
                else                         run_stream<DT, false, 1, W, D, FINISH>(P, t, own, lds, wave);
            } else if constexpr (WIDE) {
                run_pairs<DT, D>(P, t, head, lds, i + 1 < end || more ? early : late);
            } else if constexpr (stream_tiles(D) == 2 && !FINISH) {
                const int own = head_of(t, i);
                if (t.flags & kTaskReadOnce) run_stream<DT, true, 2, W, D>(P, t, own, lds, wave);
                else                         run_stream<DT, false, 2, W, D>(P, t, own, lds, wave);
            }
            ++i;
        }
    };
    const bool queued = P.queue_off != nullptr, fetching = queued && P.num_entries > P.num_slots;
    const DevTask *recs = queued ? P.queue_recs : P.slot_recs;
    const int32_t *off = queued ? P.queue_off : P.slot_off;
    const int limit = queued ? P.num_entries : slot + 1;
    int32_t *taken = P.counters + 2 * head, *finished = taken + 1;
    int *word = reinterpret_cast<int *>(lds);
    int e = slot;
#pragma unroll 1
    while (e < limit) {
        run_tasks(recs, off[e], off[e + 1], !queued, fetching);
        if (!fetching) break;
        if (threadIdx.x == 0) *word = P.num_slots + atomicAdd(taken, 1);
        __syncthreads();
        e = __builtin_amdgcn_readfirstlane(*word);
        __syncthreads();
    }
    if (fetching && threadIdx.x == 0 && atomicAdd(finished, 1) == P.num_slots - 1) {
        atomicExch(taken, 0);
        atomicExch(finished, 0);
    }
}

// ---- both rows of a head ----------------------------------------------------------------------------------

// The two rows of a head in a wave: row `row` (the map) in 32 lanes, whose channels are 128 * (c / 4) + 4 * lane + c % 4 (64
// channels: 2 * lane + c).
template <int D>
struct PairRows {
    static constexpr int CPL = D / 32, PIECE = CPL < 4 ? CPL : 4;
    int lane, row;
    int64_t first;                              // row of the head's partials behind an entry of the list

    __device__ __forceinline__ PairRows(const MergeParams &P, int head, int hj)
    {
        lane = threadIdx.x & 31;
        row = (threadIdx.x >> 5) & 1;
        first = int64_t(head) * P.part_rows + hj + row;
    }
    __device__ __forceinline__ void load(const MergeParams &P, int entry, float2 &ml, float (&o)[CPL]) const
    {
        const int64_t prow = first + entry;
        ml = *reinterpret_cast<const float2 *>(P.part_ml + prow * 2);
        const float *src = P.part_o + prow * D + lane * PIECE;
#pragma unroll
        for (int u = 0; u < CPL / PIECE; ++u) {
            if constexpr (PIECE == 2) {
                const float2 x = *reinterpret_cast<const float2 *>(src);
                o[0] = x.x;
                o[1] = x.y;
            } else {
                const f32x4 x = *reinterpret_cast<const f32x4 *>(src + u * 128);
#pragma unroll
                for (int c = 0; c < 4; ++c) o[u * 4 + c] = x[c];
            }
        }
    }
};

// Weight of channel `channel` of the norm
__device__ __forceinline__ float norm_weight(const DifferentialParams &P, int channel)
{
    if (P.weight_dtype == CODEC_DTYPE_FP32) return static_cast<const float *>(P.weight)[channel];
    const uint16_t bits = static_cast<const uint16_t *>(P.weight)[channel];
    return P.weight_dtype == CODEC_DTYPE_FP16 ? float(__builtin_bit_cast(_Float16, bits)) : __uint_as_float(uint32_t(bits) << 16);
}

// The finished rows of a stream task: the rows of a head are neighbouring lanes.  Each stores half of the channels.
template <int DT, int D>
__device__ __forceinline__ void store_finished_pairs(const PairParams &P, const DevTask &t, int head, int rows, int l16, int grp,
                                                     const RowState<1, D> &st)
{
    const DifferentialParams &F = P.finish;
    const bool live = l16 < rows;
    const int qi = live ? l16 / P.group : 0, hj = live ? l16 - qi * P.group : l16 & 1;
    const int r = t.single_req >= 0 ? t.single_req : P.node_q[t.q_off + qi], h = (head * P.group + hj) >> 1;
    const float inv = 1.f / st.l[0], lambda = F.lambda[r * F.lambda_request_stride + h * F.lambda_head_stride];
    const bool second = hj & 1, whole = D >= 128 || grp * 32 < D;       // whole: channels that the head has
    float x[channel_tiles(D)][4], squares = 0.f;
#pragma unroll
    for (int dt = 0; dt < channel_tiles(D); ++dt)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float mine = st.o[0][dt][e] * inv, other = __shfl_xor(mine, 1);
            x[dt][e] = __builtin_fmaf(-lambda, second ? mine : other, second ? other : mine);
            squares = __builtin_fmaf(x[dt][e], x[dt][e], squares);
        }
    float factor = F.gain;
    if (F.norm) {
        squares = whole ? squares : 0.f;
        squares += __shfl_xor(squares, 16);
        squares += __shfl_xor(squares, 32);
        factor = F.gain / __builtin_sqrtf(squares * (1.f / D) + F.eps);
    }
    if (!live || !whole) return;
    char *out = static_cast<char *>(F.merge.out) + ((int64_t(r) * (P.h_q / 2) + h) * D + grp * 32) * 2;
#pragma unroll
    for (int u = 0; u < BlockRegs<D>::VU; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            u32x4 y;
            float w[8];
#pragma unroll
            for (int c = 0; c < 8; ++c) w[c] = x[8 * u + c][e] * factor;
            if (F.weight) {
#pragma unroll
                for (int c = 0; c < 8; ++c) w[c] *= norm_weight(F, 128 * u + 32 * grp + 8 * e + c);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) y[c] = pack2<DT>(w[2 * c], w[2 * c + 1]);
            if (second == (e >= 2)) *reinterpret_cast<u32x4 *>(out + u * 256 + e * 16) = y;
        }
}

// Both rows of a head, unnormalised, to its result.
template <int DT, int D>
__device__ __forceinline__ void finish_pair(const DifferentialParams &P, const PairRows<D> &at, int r, int h, float l, float (&o)[PairRows<D>::CPL])
{
    constexpr int CPL = PairRows<D>::CPL, PIECE = PairRows<D>::PIECE;
    const float inv = 1.f / l, lambda = P.lambda[r * P.lambda_request_stride + h * P.lambda_head_stride];
    float x[CPL], squares = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c) {
        const float mine = o[c] * inv, other = __shfl_xor(mine, 32);
        x[c] = __builtin_fmaf(-lambda, at.row ? mine : other, at.row ? other : mine);
        squares = __builtin_fmaf(x[c], x[c], squares);
    }
    float factor = P.gain;
    if (P.norm) {
#pragma unroll
        for (int d = 1; d < 32; d *= 2) squares += __shfl_xor(squares, d);
        factor = P.gain / __builtin_sqrtf(squares * (1.f / D) + P.eps);
    }
    if (at.row) return;
    char *out = static_cast<char *>(P.merge.out) + ((int64_t(r) * (P.merge.h_q / 2) + h) * D + at.lane * PIECE) * 2;
#pragma unroll
    for (int u = 0; u < CPL / PIECE; ++u) {
        float y[PIECE];
#pragma unroll
        for (int c = 0; c < PIECE; ++c) {
            y[c] = x[u * PIECE + c] * factor;
            if (P.weight) y[c] *= norm_weight(P, u * 128 + at.lane * PIECE + c);
        }
#pragma unroll
        for (int c = 0; c < PIECE; c += 2) *reinterpret_cast<unsigned int *>(out + u * 256 + c * 2) = pack2<DT>(y[c], y[c + 1]);
    }
}

// The reduction (Alg. 3) of both rows of a head and what becomes of them.  W = 1: a wave a head, two in a workgroup; W > 1: a list
// shared by W waves, whose sums meet in LDS.  Grid as in merge_kernel: blockIdx.x is the KV head.  Bound by the partial rows' reads in flight: 12.6 MB
// of them (32 requests of 32 heads, twelve rows a list) 4.9 us, out of the caches they were left in.
template <int DT, int D, int W>
__global__ void __launch_bounds__((W == 1 ? kMergeWaves : W) * 64) differential_reduction_kernel(const DifferentialParams P)
{
    constexpr int CPL = PairRows<D>::CPL;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave_lane = threadIdx.x & 63;
    const int heads = P.merge.group / 2;
    int unit = blockIdx.z * gridDim.y + blockIdx.y;
    if constexpr (W == 1) unit = unit * kMergeWaves + wave;
    if (unit >= P.merge.num_requests * heads) return;
    const int r = unit / heads, member = unit - r * heads;
    const PairRows<D> at(P.merge, blockIdx.x, 2 * member);
    const int32_t *line = W == 1 ? P.merge.req_inline + int64_t(r) * (kInlineParts + 1) : P.merge.req_line + int64_t(r) * split_line_words(W);
    constexpr int kInLine = W == 1 ? kInlineParts : split_rows(W);
    const int total = line[0];
    const int32_t *list = total <= kInLine ? line + 1 : P.merge.req_part + P.merge.req_part_off[r];

    float M = -INFINITY, L = 0.f, acc[CPL];
#pragma unroll
    for (int c = 0; c < CPL; ++c) acc[c] = 0.f;
#pragma unroll 1
    for (int base = (W == 1 ? 0 : wave) * kFoldChunk; base < total; base += W * kFoldChunk) {
        const int cnt = total - base < kFoldChunk ? total - base : kFoldChunk;
        int rows[kFoldChunk];
#pragma unroll
        for (int j = 0; j < kFoldChunk; ++j) rows[j] = list[base + (j < cnt ? j : 0)];
        Chunk<kFoldChunk, CPL> x;
        x.load(P.merge, at, rows, cnt);
        const float mm = x.top(M, cnt);
        float l, sum[CPL];
        x.sum_up(cnt, mm, l, sum);
        add_chunk(M, L, acc, mm, l, sum);
        M = mm;
    }
    if constexpr (W > 1) {
        __shared__ float sums[W - 1][CPL + 2][64];
        if (wave > 0) {
            float (*put)[64] = sums[wave - 1];
            put[CPL][wave_lane] = L;
            put[CPL + 1][wave_lane] = M;
#pragma unroll
            for (int c = 0; c < CPL; ++c) put[c][wave_lane] = acc[c];
        }
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 0; w < W - 1; ++w) {
            const float m = sums[w][CPL + 1][wave_lane], mm = fmaxf(M, m), theirs = weight(m, mm);
            float sum[CPL];
#pragma unroll
            for (int c = 0; c < CPL; ++c) sum[c] = sums[w][c][wave_lane] * theirs;
            add_chunk(M, L, acc, mm, sums[w][CPL][wave_lane] * theirs, sum);
            M = mm;
        }
    }
    finish_pair<DT, D>(P, at, r, blockIdx.x * heads + member, L, acc);
}

template <int DT, int D>
int launch_differential_of(const DifferentialParams &p, hipStream_t s)
{
    const int64_t units = int64_t(p.merge.num_requests) * (p.merge.group / 2);
    constexpr int64_t kMaxY = 32768;
    auto launch = [&](auto kernel, int units_of, int waves) {
        const int64_t groups = (units + units_of - 1) / units_of, y = groups < kMaxY ? groups : kMaxY;
        const dim3 grid(unsigned(p.merge.h_q / p.merge.group), unsigned(y), unsigned((groups + y - 1) / y)), block(waves * 64);
        hipLaunchKernelGGL(kernel, grid, block, 0, s, p);
    };
    if (p.merge.split_waves == 8)      launch(differential_reduction_kernel<DT, D, 8>, 1, 8);
    else if (p.merge.split_waves == 4) launch(differential_reduction_kernel<DT, D, 4>, 1, 4);
    else                               launch(differential_reduction_kernel<DT, D, 1>, kMergeWaves, kMergeWaves);
    return int(hipGetLastError());
}

}  // namespace

// See prepare_kernels
int prepare_pair_kernels()
{
    auto wide = [](auto dt, auto d) {
        constexpr int DT = decltype(dt)::value, D = decltype(d)::value;
        return int(hipFuncSetAttribute(reinterpret_cast<const void *>(pair_kernel<DT, kFormWide, D>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, PairPath<D, 1>::kLds));
    };
    int e = 0;
    auto all = [&](auto dt) {
        for (int one : {wide(dt, std::integral_constant<int, 64>{}), wide(dt, std::integral_constant<int, 128>{}), wide(dt, std::integral_constant<int, 256>{})})
            e = e ? e : one;
    };
    all(std::integral_constant<int, CODEC_DTYPE_FP16>{});
    all(std::integral_constant<int, CODEC_DTYPE_BF16>{});
    return e;
}

int launch_pairs(const PairParams &p, int dtype, int head_dim, int num_slots, int max_rows_in_plan, bool tiles, void *stream)
{
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return int(hipErrorInvalidValue);
    const bool wide = head_dim == kHeadDim ? max_rows_in_plan > 16 : tiles;         // see launch_pac
    if (!wide && max_rows_in_plan > 16 * stream_tiles(head_dim)) return int(hipErrorInvalidValue);
    if (!p.part_o && (wide || max_rows_in_plan > 16)) return int(hipErrorInvalidValue);
    const dim3 grid(unsigned(num_slots) * unsigned(p.h_kv));
    hipStream_t s = static_cast<hipStream_t>(stream);
    auto launch = [&](auto dt, auto d) {
        constexpr int DT = decltype(dt)::value, D = decltype(d)::value;
        const dim3 block((wide ? kernel_waves(kFormWide, D) : kNarrowWaves) * 64);
        constexpr size_t kLds = PairPath<D, 1>::kLds;
        if (!p.part_o) hipLaunchKernelGGL((pair_kernel<DT, kFormFinish, D>), grid, block, 0, s, p);
        else if (wide) hipLaunchKernelGGL((pair_kernel<DT, kFormWide, D>), grid, block, kLds, s, p);
        else           hipLaunchKernelGGL((pair_kernel<DT, kFormNarrow, D>), grid, block, 0, s, p);
    };
    auto launch_dim = [&](auto dt) {
        if (head_dim == 64)       launch(dt, std::integral_constant<int, 64>{});
        else if (head_dim == 128) launch(dt, std::integral_constant<int, 128>{});
        else                      launch(dt, std::integral_constant<int, 256>{});
    };
    if (dtype == CODEC_DTYPE_FP16) launch_dim(std::integral_constant<int, CODEC_DTYPE_FP16>{});
    else                           launch_dim(std::integral_constant<int, CODEC_DTYPE_BF16>{});
    return int(hipGetLastError());
}

int launch_differential(const DifferentialParams &p, int dtype, int head_dim, void *stream)
{
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool half = dtype == CODEC_DTYPE_FP16;
    if (head_dim == 64)  return half ? launch_differential_of<CODEC_DTYPE_FP16, 64>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 64>(p, s);
    if (head_dim == 128) return half ? launch_differential_of<CODEC_DTYPE_FP16, 128>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 128>(p, s);
    if (head_dim == 256) return half ? launch_differential_of<CODEC_DTYPE_FP16, 256>(p, s) : launch_differential_of<CODEC_DTYPE_BF16, 256>(p, s);
    return int(hipErrorInvalidValue);
}

}  // namespace codec
