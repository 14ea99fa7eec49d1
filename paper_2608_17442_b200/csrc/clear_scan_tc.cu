// The sweep of the cleartext recurrence on the fifth-generation tensor cores (tcgen05), for bfloat16 and rows that allow 16-byte accesses: the
// deployed layer's.  The mathematics is that of clear_scan.cuh, with chunks of 128 tokens.
//
// Of its operands one pair is broad (a group's rows of N columns) and one narrow (a head's 64 channels); the state H [N][64] is always
// broad^T (faded narrow).  Per chunk four products, accumulators in tensor memory:
//   S  = q k^T                        128 x 128, both operands as they were loaded
//   H  = broad^T (faded narrow)       128 x 64, the faded values in three planes (they enter the state)
//   O1 = q state                      128 x 64 (MODE_OUT) or 128 x 128 (MODE_GRAD), the state in two planes or three
//   O2 = (decayed S) v                the same, the decayed scores in two planes or three, as left operand from tensor memory
// out = decay since the chunk's start * O1 + O2.  A tile of 128 tokens x 64 columns in shared memory (a panel, 16 KB, 128-byte swizzle) is the
// K-major operand of one product and the MN-major operand of another, so nothing is stored twice or transposed.
//
// Sixteen warps compute (a thread owns a row and a quarter of the columns), one issues the products, one sums up the log decays of the next chunks,
// two copy the next chunk's operands.  Shared memory leaves the L1 so little that a spilled register is read back from L2: with the copies
// in the computing warps, whose 96 registers their addresses overflowed, a chunk took 10 500 cycles.
// The products of a chunk run while the threads are at something else: O1 while the faded values are formed, H while the scores are decayed,
// O2 while the state is updated; the next chunk's S while the outputs are written.  Reading operands from shared memory (128 bytes a cycle) is
// what a product of these widths takes, so the planes of one right operand are multiplied side by side where tensor memory has room
// (H 1150 -> 640 cycles a chunk, O1 770 -> 510) and the sums over planes are left to the threads.
//
// Decays of pairs in different blocks of 32 tokens are products of two factors not above one (from the earlier token to its block's end,
// from there to the later one): one exponential per row and block; only the blocks on the diagonal take one per pair.
#define FESC_DBG_FILE 21   // file id in the sites a debug build reports
#include "clear_scan.cuh"

#define TC_Q 128
#define PANEL 16384u
#define TC_BACK_UNROLL 2        // products in a row in the backward pass: 8 x 2048 tokens 431 us, 2048 101 (8: 427 and 104); in the scan all of them (299 us; 4: 314)
#define TC_WARPS 16             // that compute; one more issues, one more sums decays, two copy
#define TC_THREADS (32 * (TC_WARPS + 4))

template <int MODE>
struct TcLayout {
    static constexpr bool GRAD = MODE == MODE_GRAD, OUT = MODE == MODE_OUT;
    static constexpr int NO = GRAD ? 3 : 2;                        // planes of scores and states
    // panels in shared memory; k and v have two sets (without outputs the faded values, too: they are formed while the product before runs)
    static constexpr int q = 0, QP = OUT ? 2 : GRAD ? 1 : 0;
    static constexpr int broad = QP, narrow = broad + 4, w = narrow + 2, W_SETS = MODE ? 1 : 2, st = w + 3 * W_SETS, panels = st + (MODE ? NO : 0);
    // Columns of tensor memory, of which a CTA takes all 512: they begin at 0.  The first two planes of 16 decayed scores lie over the 16 scores, so a warp overwrites what it
    // has read itself; a third plane has columns of its own.
    static constexpr uint32_t DV = GRAD ? 128 : 64, O1_PARTS = OUT ? 2 : 1, H_PARTS = GRAD ? 1 : 3;      // accumulators side by side, one per plane
    static constexpr uint32_t S = 0, P3 = 128, O1 = GRAD ? 192 : 128, O2 = O1 + O1_PARTS * DV, H = MODE ? O2 + DV : 0, columns = 512;
    static constexpr uint32_t H_SET = MODE ? 0 : 64 * H_PARTS;      // from one set's H to the other's
    static_assert(H + H_SET + 64 * H_PARTS <= columns, "accumulators fit");
    static constexpr size_t bytes = (size_t)panels * PANEL + 1024;  // panels start on 1024 bytes
};

static __device__ uint32_t g_clear_status[2];   // not 0: a bounded wait gave up; products were still under way at a kernel's end

// what the decays' warp leaves for a chunk
struct alignas(16) TcDecays {      // read four words at a time
    float2 cum[TC_Q];        // log2 of the decay up to a token, as two floats
    float tail[TC_Q];        // decay from a token to the end of its block of 32
    float grow[TC_Q];        // from the chunk's start to a token
    float fade[TC_Q];        // from a token to the chunk's end
    float2 ref[4];           // cum at the blocks' ends
    float keep;              // over the chunk
};

// off by two units at most, and the rounding of x: what a 16-bit output or a sum over a chunk takes once; the chunk's decay goes by exp2_near
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ bool poll(uint32_t bar, uint32_t parity) {
#pragma unroll 1
    for (uint32_t it = 0; it < (1u << 18); it++) {      // about a second; a chunk takes microseconds
        if (mbar_try_wait(bar, parity)) return true;
        if (it > 64) __nanosleep(64);
    }
    return false;
}
// The longer part of a wait, out of line: the kernel has some thirty of them, and its instructions have to stay in the cache of one SM.
static __device__ __noinline__ void wait_on(uint32_t bar, uint32_t parity, volatile uint32_t* dead) {
    if (*dead || poll(bar, parity)) return;
    *dead = 1, g_clear_status[0] = 1;
}
// The last wait, for the products under way, before tensor memory is given back: also after another one gave up.
static __device__ __noinline__ void drain(uint32_t bar) {
    if (!poll(bar, 0)) g_clear_status[1] = 1;
}
// bytes of (row, 16-byte chunk c of eight) in a panel
__device__ __forceinline__ uint32_t panel_at(uint32_t row, uint32_t c) { return row * 128 + ((c ^ (row & 7)) << 4); }

// K-major: rows of 128 bytes, groups of 8 rows 1024 bytes apart; MN-major: the same words with K down the rows, blocks of 64 columns a panel apart
#define TC_DESC_HI ((1024u >> 4) | (1u << 14) | (2u << 29))
__device__ __forceinline__ uint32_t tc_desc(uint32_t addr) { return (addr >> 4) | ((PANEL >> 4) << 16); }
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\tmov.b64 a, {%1, %5};\n\tmov.b64 b, {%2, %5};\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(TC_DESC_HI)
                 : "memory");
}
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 b;\n\tmov.b64 b, {%2, %5};\n\tsetp.ne.u32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n\t}" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"((uint32_t)add), "r"(TC_DESC_HI)
                 : "memory");
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t (&r)[16], uint32_t addr) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(addr)
                 : "memory");
}
__device__ __forceinline__ void tc_st8(uint32_t addr, const uint32_t (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]),
                 "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void bar_sync(uint32_t id, uint32_t threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
// v as a sum of NM pairs of bfloat16 numbers
template <int NM>
__device__ __forceinline__ void split2(f2 v, uint32_t (&p)[NM]) {
#pragma unroll
    for (int i = 0; i < NM; i++) {
        p[i] = pack_bf16(v.x, v.y);
        if (i + 1 < NM) {
            v = fma2(both(p[i]), {-1.f, -1.f}, v);
        }
    }
}
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// 32 bytes at a 32-byte boundary
__device__ __forceinline__ void st32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}

struct TcShared {
    TcDecays decays[2];
    alignas(8) u64 bars[16];        // see below
    uint32_t tmem_base;
    volatile uint32_t dead;         // a wait gave up: the rest of the chunks goes through without waiting, with nothing of worth in it
    float words[2][TC_WARPS];
};

// UNROLL: products of a loop that are issued in a row (8: all)
template <int MODE, int UNROLL>
__device__ __forceinline__ void tc_sweep(const ScanArgs& a, uint32_t block, TcShared& sh) {
    using Lay = TcLayout<MODE>;
    constexpr int NO = Lay::NO, NS = 3;
    extern __shared__ __align__(1024) uint8_t tc_smem[];
    auto& decays = sh.decays;
    auto& bars = sh.bars;
    auto& tmem_base = sh.tmem_base;
    auto& dead = sh.dead;
    auto& words = sh.words;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t vheads = a.H * a.tiles, vh = block % vheads, seg = block / vheads % a.segments, b = block / vheads / a.segments;
    const uint32_t head = vh / a.tiles, tile = vh % a.tiles, group = head / (a.H / a.G);
    const int length = a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L;
    const int seg_tokens = (int)a.seg_chunks * SCAN_Q, t_lo = (int)seg * seg_tokens, t_hi = min(length, t_lo + seg_tokens);
    const int pw = min(SCAN_TILE, (int)a.P - (int)tile * SCAN_TILE);
    const bool is_last = a.backwards ? seg == 0 : (t_hi == length && (t_lo < length || seg == 0));
    const size_t state_at = (size_t)head * a.P * a.N + (size_t)tile * SCAN_TILE * a.N, states = (size_t)a.H * a.P * a.N;
    const size_t slot = (size_t)b * a.segments + seg;
    if (MODE != MODE_STATE && t_lo >= length && !is_last) {
        if (MODE == MODE_GRAD && a.ends && tid == 0) {
            a.ends[slot * vheads + vh] = 0.f;
            if (a.diag) a.diag[slot * vheads + vh] = 0.f;
        }
        return;
    }
    const ScanOperand& ob = MODE == MODE_GRAD ? a.v : a.k;      // broad
    const ScanOperand& on = MODE == MODE_GRAD ? a.k : a.v;      // narrow
    const int qw = a.q.tiled ? pw : (int)a.N, vw = MODE == MODE_GRAD ? (int)a.N : pw;
    typedef __nv_bfloat16 T;
#ifdef FESC_DEBUG_BOUNDS
    if (t_lo < t_hi) {
        const long long n = t_hi - t_lo - 1;
        bool ok = DBG_REGION(scan_row<T>(ob, b, t_lo, head, group, tile), (n * ob.st + a.N) * sizeof(T)) &&
                  DBG_REGION(scan_row<T>(on, b, t_lo, head, group, tile), (n * on.st + pw) * sizeof(T)) &&
                  DBG_REGION(a.g + b * a.gb + t_lo * a.gt + head * a.gh, (n * a.gt + 1) * sizeof(float));
        if (MODE) ok = ok && DBG_REGION(scan_row<T>(a.q, b, t_lo, head, group, tile), (n * a.q.st + qw) * sizeof(T));
        if (MODE == MODE_OUT) ok = ok && DBG_REGION((T*)a.out + b * a.ob + t_lo * a.ot + head * a.oh + tile * SCAN_TILE, (n * a.ot + vw) * sizeof(T));
        if (MODE == MODE_GRAD)
            ok = ok && DBG_REGION(a.part + (((size_t)b * vheads + vh) * a.segments + seg) * (a.seg_chunks / 2) * (TC_Q * 128),
                                  (size_t)((n + TC_Q) / TC_Q) * TC_Q * 128 * sizeof(float));
        if (!ok) return;
    }
    if ((MODE && a.init && !DBG_REGION(a.init + (a.segments > 1 ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (a.last && !DBG_REGION(a.last + (MODE == MODE_STATE ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (MODE == MODE_GRAD && a.meet && !DBG_REGION(a.meet + (a.segments > 1 && !a.backwards ? slot : b) * states + state_at, (size_t)pw * a.N * 4)))
        return;
#endif
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(tc_smem) + 1023) & ~1023u, bar = (uint32_t)__cvta_generic_to_shared(bars);
    uint8_t* const panels = tc_smem + (base - (uint32_t)__cvta_generic_to_shared(tc_smem));
    // Per chunk: q copied; decayed scores written; products S, O1, O2 done.  Of the two sets of chunks: faded values and state written, H done, decays
    // filled, k and v copied, all used (and O1 and O2 read).  No one may get to what completes a barrier's next phase before everyone who waits for
    // this one has: two phases on, a barrier looks as it did before.  Where those who complete it run up to two chunks ahead, each set has a
    // barrier of its own.
    const uint32_t b_q = bar, b_p = bar + 8, b_s = bar + 16, b_o1 = bar + 24, b_o = bar + 32, drained = bar + 40;
    const uint32_t b_wv = bar + 48, b_h = bar + 64, b_g = bar + 80, b_kv = bar + 96, b_used = bar + 112;
    if (warp == TC_WARPS) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_base)), "n"(Lay::columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        mbar_init(b_q, 2), mbar_init(b_p, TC_WARPS), mbar_init(b_s, 1), mbar_init(b_o1, 1), mbar_init(b_o, 1), mbar_init(drained, 1);
        for (uint32_t i = 0; i < 16; i += 8)
            mbar_init(b_wv + i, TC_WARPS), mbar_init(b_h + i, 1), mbar_init(b_g + i, 1), mbar_init(b_kv + i, 2), mbar_init(b_used + i, TC_WARPS);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    auto left = [&](int c) { return min(TC_Q, t_hi - t_lo - c * TC_Q); };      // tokens of a chunk
    const int chunks = t_hi > t_lo ? (t_hi - t_lo + TC_Q - 1) / TC_Q : 0, dir = a.backwards ? -1 : 1;
    const int t_first = a.backwards ? t_hi - 1 : t_lo;
    auto wait = [&](uint32_t which, uint32_t parity) {
        if (!mbar_try_wait(which, parity & 1)) wait_on(which, parity & 1, &dead);
    };

    if (warp == TC_WARPS) {
        // issues the products
        constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);        // bfloat16 x bfloat16 -> float32, 128 rows
        constexpr uint32_t I_S = IDESC | (16u << 17), I_H = IDESC | (1u << 15) | (1u << 16) | ((8u * Lay::H_PARTS) << 17);
        constexpr uint32_t I_O1 = IDESC | (16u << 17) | (Lay::GRAD ? 0 : 1u << 16), I_O2 = IDESC | (1u << 16) | ((Lay::DV / 8) << 17);
        constexpr uint32_t STEP = PANEL >> 4, QK = Lay::OUT ? 8 : 4;                        // steps of 16 along q's columns
        // One thread issues, and what it computes per product counts: with everything unrolled and the operands' set known when compiled the scan of
        // 65536 tokens takes 300 us, in loops 343.  But a chunk's work has to stay in instruction caches that neighbouring SMs share: where they
        // run different sweeps (the backward pass), unrolled code took turns of up to twice the time, and loops are used (529 -> 475 us).
        auto product = [&](uint32_t d, uint32_t left, uint32_t left_step, uint32_t right, uint32_t right_step, uint32_t idesc, uint32_t n, bool add, auto from_tmem) {
#pragma unroll UNROLL
            for (uint32_t k = 0; k < n; k++, left += left_step, right += right_step, add = true) {
                if constexpr (decltype(from_tmem)::value) tc_mma_ts(d, left, right, idesc, add);
                else tc_mma_ss(d, left, right, idesc, add);
            }
        };
        constexpr std::false_type SHARED{};
        constexpr std::true_type TENSOR{};
        auto chunk = [&](int c, uint32_t set) {
            const uint32_t d0 = tc_desc(base), pq = d0 + Lay::q * STEP, pw_ = d0 + (Lay::w + (Lay::W_SETS == 2 ? 3 * set : 0)) * STEP, ps = d0 + Lay::st * STEP, pb = d0 + (Lay::broad + 2 * set) * STEP,
                           pn = d0 + (Lay::narrow + set) * STEP;
            if (MODE) {
                wait(b_kv + 8 * set, c >> 1);
                wait(b_q, c);
                if (c) wait(b_o, c - 1);                             // the scores' planes lie over the scores
                tc_after();
#pragma unroll
                for (uint32_t j = 0; j < QK / 4; j++)
                    if (!j || a.N > 64) product(Lay::S, pq + j * STEP, 2, (Lay::OUT ? pb : pn) + j * STEP, 2, I_S, 4, j, SHARED);
                tc_commit(b_s);
            }
            wait(b_wv + 8 * set, c >> 1);
            tc_after();
#pragma unroll
            for (uint32_t p = 0; p < (Lay::H_PARTS == 1 ? NS : 1); p++)
                product(Lay::H + Lay::H_SET * set, pb, 128, pw_ + p * STEP, 128, I_H, 8, p, SHARED);
            tc_commit(b_h + 8 * set);
            if (MODE) {
                if (c) wait(b_used + 8 * (set ^ 1), (c - 1) >> 1);
                tc_after();
                if (Lay::OUT) {
#pragma unroll
                    for (uint32_t j = 0; j < 2; j++)
                        if (!j || a.N > 64) product(Lay::O1, pq + j * STEP, 2, ps + 512 * j, 128, I_O1, 4, j, SHARED);
                } else {
#pragma unroll
                    for (uint32_t p = 0; p < NO; p++) product(Lay::O1, pq, 2, ps + p * STEP, 2, I_O1, 4, p, SHARED);
                }
                tc_commit(b_o1);
                wait(b_p, c);
                tc_after();
#pragma unroll
                for (uint32_t p = 0; p < NO; p++)
                    product(Lay::O2, p < 2 ? Lay::S + 8 * p : Lay::P3, p < 2 ? 16 : 8, Lay::GRAD ? pb : pn, 128, I_O2, 8, p, TENSOR);
                tc_commit(b_o);
            }
        };
        if (lane == 0) {
            if constexpr (UNROLL > 4) {
                for (int c = 0; c < chunks; c += 2) {
                    chunk(c, 0);
                    if (c + 1 < chunks) chunk(c + 1, 1);
                }
            } else {
                for (int c = 0; c < chunks; c++) chunk(c, c & 1);
            }
            tc_commit(drained);
            drain(drained);
        }
        __syncwarp();
    } else if (warp == TC_WARPS + 1) {
        // log decays of a chunk, four tokens a lane
        const float* g = a.g + b * a.gb + head * a.gh;
        double through = 0.0;
        float gv[4];
        auto read = [&](int c) {
            const int valid = min(TC_Q, t_hi - t_lo - c * TC_Q), t0 = a.backwards ? t_hi - 1 - c * TC_Q : t_lo + c * TC_Q;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int pos = 4 * lane + i, t = t0 + dir * pos + (a.backwards ? 1 : 0);
                gv[i] = pos < valid && t < length ? g[t * a.gt] : 0.f;
            }
        };
        if (chunks) read(0);
        for (int c = 0; c < chunks; c++) {
            double sum[4];
#pragma unroll
            for (int i = 0; i < 4; i++) sum[i] = (double)(gv[i] < SCAN_DROP ? SCAN_DROP : gv[i]) * 1.4426950408889634 + (i ? sum[i - 1] : 0.0);
            if (c + 1 < chunks) read(c + 1);
            double run = sum[3];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double w = __shfl_up_sync(~0u, run, o);
                if (lane >= o) run += w;
            }
            const double before = run - sum[3], total = __shfl_sync(~0u, run, 31), end = __shfl_sync(~0u, run, lane | 7);
            if (c >= 2) wait(b_used + 8 * (c & 1), (c >> 1) - 1);
            TcDecays& d = decays[c & 1];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const double v = before + sum[i];
                const float hi = (float)v;
                d.cum[4 * lane + i] = make_float2(hi, (float)(v - hi));
                d.grow[4 * lane + i] = ex2((float)v), d.fade[4 * lane + i] = ex2((float)(total - v)), d.tail[4 * lane + i] = ex2((float)(end - v));
            }
            if ((lane & 7) == 7) d.ref[lane >> 3] = make_float2((float)end, (float)(end - (float)end));
            if (lane == 0) d.keep = exp2_near(total);
            through += total;
            __syncwarp();
            if (lane == 0) mbar_arrive(b_g + 8 * (c & 1));
        }
        if (MODE == MODE_STATE && lane == 0 && tile == 0) a.decay[slot * a.H + head] = exp2_near(through);
    } else if (warp > TC_WARPS + 1) {
        // Copies.  A thread has one 16-byte chunk of every eighth row: its place in a panel moves by 1024 bytes from row to row.
        const uint32_t me = tid - 32 * (TC_WARPS + 2), r0 = me >> 3, col = (me & 7) * 8, to = base + panel_at(r0, me & 7);
        const T *pb = nullptr, *pn = nullptr, *pq = nullptr;
        if (chunks) {
            pb = scan_row<T>(ob, b, t_first + dir * (int)r0, head, group, tile) + col, pn = scan_row<T>(on, b, t_first + dir * (int)r0, head, group, tile) + col;
            if (MODE) pq = scan_row<T>(a.q, b, t_first + dir * (int)r0, head, group, tile) + col;
        }
        // Panels first .. first + n - 1 of a chunk.  What does not exist is not read: zero bytes are copied from the start of an operand, which lies on
        // 16 bytes, as the source of a copy of 16 has to however few of them are read (g may lie on four).
        const T* const none = (const T*)ob.p;
        auto copy = [&](uint32_t first, int n, const T* src, long long step, int width, int valid) {
#pragma unroll 1
            for (int j = 0; j < n; j++, src += 64, width -= 64) {
                const int bytes = min(max(width - (int)col, 0), 8) * 2;
                const uint32_t dst = to + (first + j) * PANEL;
                const T* p = bytes ? src : none;
                const long long by = bytes ? step : 0;
                if (valid == TC_Q) {
#pragma unroll 8
                    for (uint32_t i = 0; i < TC_Q / 8; i++, p += by) cp_async16_part(dst + 1024 * i, p, bytes);
                } else {
#pragma unroll 1
                    for (uint32_t i = 0; i < TC_Q / 8; i++, p += by) {
                        const int some = (int)(r0 + 8 * i) < valid ? bytes : 0;
                        cp_async16_part(dst + 1024 * i, some ? p : none, some);
                    }
                }
            }
        };
        const int wide_panels = a.N > 64 ? 2 : 1;        // the second panel of narrower rows is zero from the first chunk of its set on
        auto landed = [&](uint32_t which) {
            cp_async_wait();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(which);
        };
        const long long sb = 8 * dir * ob.st, sn = 8 * dir * on.st, sq = 8 * dir * a.q.st;
        for (int c = 0; c < chunks; c++) {
            const uint32_t set = c & 1;
            if (c >= 2) wait(b_used + 8 * set, (c >> 1) - 1);
            copy(Lay::broad + 2 * set, c < 2 ? 2 : wide_panels, pb, sb, (int)a.N, left(c));
            copy(Lay::narrow + set, 1, pn, sn, pw, left(c));
            landed(b_kv + 8 * set);
            if (MODE) {
                if (c) wait(b_o1, c - 1);
                copy(Lay::q, Lay::OUT ? wide_panels : 1, pq, sq, qw, left(c));
                landed(b_q);
            }
            pb += sb * (TC_Q / 8), pn += sn * (TC_Q / 8), pq += sq * (TC_Q / 8);
        }
    } else {
        const uint32_t quarter = warp & 3, part = warp >> 2, row = 32 * quarter + lane;     // row: token of the chunk, or column of the state
        const uint32_t lanes = quarter << 21, at0 = panel_at(row, 2 * part), at1 = panel_at(row, 2 * part + 1);   // this thread's 16 of 64 columns
        f2 st[8];                                                                            // state[channel 16 part + i][column row]
        const float* init = MODE && a.init ? a.init + (a.segments > 1 ? slot : b) * states + state_at : nullptr;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int p = 16 * part + i;
            const float v = init && p < pw && row < a.N ? init[(size_t)p * a.N + row] : 0.f;
            if (i & 1) st[i / 2].y = v;
            else st[i / 2].x = v;
        }
        auto put = [&](int first, const uint32_t (&pl)[8][3], int planes) {
#pragma unroll
            for (int p = 0; p < planes; p++) {
                *reinterpret_cast<uint4*>(panels + (first + p) * PANEL + at0) = make_uint4(pl[0][p], pl[1][p], pl[2][p], pl[3][p]);
                *reinterpret_cast<uint4*>(panels + (first + p) * PANEL + at1) = make_uint4(pl[4][p], pl[5][p], pl[6][p], pl[7][p]);
            }
        };
        auto put_state = [&]() {
            uint32_t pl[8][3];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                uint32_t s[NO];
                split2<NO>(st[e], s);
#pragma unroll
                for (int p = 0; p < NO; p++) pl[e][p] = s[p];
            }
            put(Lay::st, pl, NO);
        };
        auto arrive = [&](uint32_t which) {
            __syncwarp();
            if (lane == 0) mbar_arrive(which);
        };
        float diag = 0.f;
        const float skip = Lay::OUT && a.skip ? a.skip[head] : 0.f;
        // what the products of chunk c need from here: the state before it, and its faded values
        auto provide = [&](int c) {
            if (MODE) put_state();
            wait(b_kv + 8 * (c & 1), c >> 1);
            wait(b_g + 8 * (c & 1), c >> 1);
            const float f = decays[c & 1].fade[row];
            const uint8_t* src = panels + (Lay::narrow + (c & 1)) * PANEL;
            const uint4 v0 = *reinterpret_cast<const uint4*>(src + at0), v1 = *reinterpret_cast<const uint4*>(src + at1);
            const uint32_t u[8] = {v0.x, v0.y, v0.z, v0.w, v1.x, v1.y, v1.z, v1.w};
            uint32_t pl[8][3];
#pragma unroll
            for (int e = 0; e < 8; e++) split2<NS>(mul2(both(u[e]), {f, f}), pl[e]);
            put(Lay::w + (Lay::W_SETS == 2 ? 3 * (c & 1) : 0), pl, NS);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_before();
            arrive(b_wv + 8 * (c & 1));
        };
        if (chunks) provide(0);
        for (int c = 0; c < chunks; c++) {
            const int set = c & 1;
            const TcDecays& d = decays[set];
            if (MODE) {
                // decayed scores of this row and the columns 32 part .. 32 part + 31
                wait(b_s, c);
                tc_after();
                const float2 ci = d.cum[row];
                // whole loops per case: a branch inside would keep the columns from overlapping
                auto read = [&](f2 (&x)[8], int h) {
                    uint32_t u[16];
                    tc_ld16(u, lanes + Lay::S + 32 * part + 16 * h);
                    tc_wait_ld();
#pragma unroll
                    for (int e = 0; e < 8; e++) x[e] = {__uint_as_float(u[2 * e]), __uint_as_float(u[2 * e + 1])};
                };
                auto write = [&](const uint32_t (&pl)[8][NO], int h) {
#pragma unroll
                    for (int p = 0; p < NO; p++) {
                        uint32_t q[8];
#pragma unroll
                        for (int e = 0; e < 8; e++) q[e] = pl[e][p];
                        tc_st8(lanes + (p < 2 ? Lay::S + 32 * part + 16 * h + 8 * p : Lay::P3 + 16 * part + 8 * h), q);
                    }
                };
                if (part < quarter) {
                    const float r = ex2((ci.x - d.ref[part].x) + (ci.y - d.ref[part].y));
#pragma unroll 1
                    for (int h = 0; h < 2; h++) {
                        f2 x[8];
                        uint32_t pl[8][NO];
                        read(x, h);
#pragma unroll
                        for (int e = 0; e < 8; e += 2) {
                            const float4 tl = *reinterpret_cast<const float4*>(&d.tail[32 * part + 16 * h + 2 * e]);
                            split2<NO>(mul2(x[e], mul2({r, r}, {tl.x, tl.y})), pl[e]);
                            split2<NO>(mul2(x[e + 1], mul2({r, r}, {tl.z, tl.w})), pl[e + 1]);
                        }
                        write(pl, h);
                    }
                } else if (part == quarter) {
#pragma unroll 1
                    for (int h = 0; h < 2; h++) {
                        f2 x[8];
                        uint32_t pl[8][NO];
                        read(x, h);
#pragma unroll
                        for (int e = 0; e < 8; e++) {
                            const int j = 16 * h + 2 * e;
                            const float4 cj = *reinterpret_cast<const float4*>(&d.cum[32 * part + j]);
                            const f2 d0 = fma2({cj.x, cj.y}, {-1.f, -1.f}, {ci.x, ci.y}), d1 = fma2({cj.z, cj.w}, {-1.f, -1.f}, {ci.x, ci.y});
                            if (Lay::GRAD) diag += (lane == j ? x[e].x : 0.f) + (lane == j + 1 ? x[e].y : 0.f);
                            f2 v = mul2(x[e], {ex2(d0.x + d0.y), ex2(d1.x + d1.y)});
                            v.x = j <= lane ? v.x : 0.f, v.y = j + 1 <= lane ? v.y : 0.f;
                            split2<NO>(v, pl[e]);
                        }
                        write(pl, h);
                    }
                } else {
                    const uint32_t pl[8][NO] = {};
#pragma unroll 1
                    for (int h = 0; h < 2; h++) write(pl, h);
                }
                tc_wait_st();
                tc_before();
                arrive(b_p);
            }
            if (!MODE && c + 1 < chunks) provide(c + 1);      // into the other set, while this chunk's product runs
            wait(b_h + 8 * set, c >> 1);
            tc_after();
            {
                const float keep = d.keep;
                uint32_t x[Lay::H_PARTS][16];
#pragma unroll
                for (int p = 0; p < (int)Lay::H_PARTS; p++) tc_ld16(x[p], lanes + Lay::H + Lay::H_SET * set + 64 * p + 16 * part);
                tc_wait_ld();
                if (keep == 0.f) {         // also an infinite state is dropped
#pragma unroll
                    for (int e = 0; e < 8; e++) st[e] = {0.f, 0.f};
                }
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    auto pair = [&](int p) { return f2{__uint_as_float(x[p][2 * e]), __uint_as_float(x[p][2 * e + 1])}; };
                    f2 v = pair((int)Lay::H_PARTS - 1);
#pragma unroll
                    for (int p = (int)Lay::H_PARTS - 2; p >= 0; p--) v = add2(v, pair(p));
                    st[e] = fma2(st[e], {keep, keep}, v);
                }
            }
            if (MODE && c + 1 < chunks) {
                wait(b_o1, c);                 // the state's panels are free
                provide(c + 1);                // before the outputs: O2 is under way
            }
            if (!MODE) {
                arrive(b_used + 8 * set);
                continue;
            }

            const float grow = d.grow[row];
            const bool live = (int)row < left(c);
            const long long t = t_first + (long long)dir * (c * TC_Q + (int)row);
            if (Lay::OUT) {
                uint32_t skipped[8] = {};
                if (a.skip) {
                    const uint8_t* src = panels + (Lay::narrow + set) * PANEL;
                    const uint4 v0 = *reinterpret_cast<const uint4*>(src + at0), v1 = *reinterpret_cast<const uint4*>(src + at1);
                    skipped[0] = v0.x, skipped[1] = v0.y, skipped[2] = v0.z, skipped[3] = v0.w, skipped[4] = v1.x, skipped[5] = v1.y, skipped[6] = v1.z, skipped[7] = v1.w;
                }
                wait(b_o, c);
                tc_after();
                uint32_t x[16], x1[16], y[16];
                tc_ld16(x, lanes + Lay::O1 + 16 * part);
                tc_ld16(x1, lanes + Lay::O1 + 64 + 16 * part);
                tc_ld16(y, lanes + Lay::O2 + 16 * part);
                tc_wait_ld();
                tc_before();
                arrive(b_used + 8 * set);
                if (grow == 0.f) {
#pragma unroll
                    for (int e = 0; e < 16; e++) x[e] = x1[e] = 0;
                }
                T* out = (T*)a.out + b * a.ob + t * a.ot + head * a.oh + tile * SCAN_TILE + 16 * part;
                const int count = live ? vw - 16 * (int)part : 0;
                uint32_t o[8];
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const f2 s = add2({__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])}, {__uint_as_float(x1[2 * e]), __uint_as_float(x1[2 * e + 1])});
                    const f2 v = fma2({skip, skip}, both(skipped[e]), fma2({grow, grow}, s, {__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])}));
                    o[e] = pack_bf16(v.x, v.y);
                }
                if (a.out_wide > 1 && count >= 16) {
                    st32(out, o);
                } else if (a.out_wide && !(count & 7)) {
                    if (count >= 8) *reinterpret_cast<uint4*>(out) = make_uint4(o[0], o[1], o[2], o[3]);
                    if (count >= 16) *reinterpret_cast<uint4*>(out + 8) = make_uint4(o[4], o[5], o[6], o[7]);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; e++)
                        if (e < count) reinterpret_cast<uint16_t*>(out)[e] = (uint16_t)(o[e / 2] >> (e & 1 ? 16 : 0));
                }
            } else {
                // A warp's 32 rows x 32 columns lie together, a thread's eight columns after another's (the sums read them the same way): as rows of
                // a matrix they would be 32 pieces of 32 bytes per store, and a chunk's stores took 4000 cycles.
                float* to_part = a.part + ((((size_t)b * vheads + vh) * a.segments + seg) * (a.seg_chunks / 2) + c) * (TC_Q * 128) + (quarter * 4 + part) * 1024 + lane * 8;
                wait(b_o, c);
                tc_after();
#pragma unroll 1
                for (int k = 0; k < 2; k++) {
                    uint32_t x[16], y[16];
                    tc_ld16(x, lanes + Lay::O1 + 32 * part + 16 * k);
                    tc_ld16(y, lanes + Lay::O2 + 32 * part + 16 * k);
                    tc_wait_ld();
                    if (k == 1) {
                        tc_before();
                        arrive(b_used + 8 * set);
                    }
                    if (grow == 0.f) {
#pragma unroll
                        for (int e = 0; e < 16; e++) x[e] = 0;
                    }
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        const f2 v = fma2({grow, grow}, {__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])}, {__uint_as_float(y[2 * e]), __uint_as_float(y[2 * e + 1])});
                        x[2 * e] = __float_as_uint(v.x), x[2 * e + 1] = __float_as_uint(v.y);
                    }
                    if (live) st32(to_part + 512 * k, x), st32(to_part + 512 * k + 256, x + 8);
                }
            }
        }
        if (a.last && (MODE == MODE_STATE || is_last)) {
            float* last = a.last + (MODE == MODE_STATE ? slot : b) * states + state_at;
            const float f = MODE && a.backwards && length > 0 ? expf(a.g[b * a.gb + head * a.gh]) : 1.f;
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int p = 16 * part + i;
                if (p < pw && row < a.N) last[(size_t)p * a.N + row] = decayed(f, i & 1 ? st[i / 2].y : st[i / 2].x);
            }
        }
        if (Lay::GRAD && a.ends) {
            float sum = 0.f;
            const float* meet = a.meet && (!a.backwards || seg == 0) ? a.meet + (a.segments > 1 && !a.backwards ? slot : b) * states + state_at : nullptr;
            if (meet) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int p = 16 * part + i;
                    if (p < pw && row < a.N) sum += (i & 1 ? st[i / 2].y : st[i / 2].x) * meet[(size_t)p * a.N + row];
                }
                const int next = a.backwards ? 0 : t_hi;
                if (next < length) sum = decayed(expf(a.g[b * a.gb + next * a.gt + head * a.gh]), sum);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o), diag += __shfl_xor_sync(~0u, diag, o);
            if (lane == 0) words[0][warp] = sum, words[1][warp] = diag;
            bar_sync(1, 32 * TC_WARPS);
            if (tid == 0) {
                float s0 = 0.f, s1 = 0.f;
                for (int w = 0; w < TC_WARPS; w++) s0 += words[0][w], s1 += words[1][w];
                a.ends[slot * vheads + vh] = s0;
                if (a.diag) a.diag[slot * vheads + vh] = s1;
            }
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == TC_WARPS) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "n"(Lay::columns));
}

// The sweeps of one call in one grid: those of the backward pass are independent, and a wave of CTAs that is not full is left once and not three
// times (16384 tokens of 24 heads: 576 CTAs in 3.9 waves instead of three times 1.3).  Neighbouring blocks work on the same rows.
__global__ void __launch_bounds__(TC_THREADS, 1) k_clear_scan_tc_state(const __grid_constant__ ScanSet s) {
    __shared__ TcShared sh;
    pdl_begin();
    tc_sweep<MODE_STATE, 8>(s.a[blockIdx.x % s.count], blockIdx.x / s.count, sh);
}
__global__ void __launch_bounds__(TC_THREADS, 1) k_clear_scan_tc(const __grid_constant__ ScanSet s) {
    __shared__ TcShared sh;
    pdl_begin();
    tc_sweep<MODE_OUT, 8>(s.a[0], blockIdx.x, sh);
}
__global__ void __launch_bounds__(TC_THREADS, 1) k_clear_scan_tc_backward(const __grid_constant__ ScanSet s) {
    __shared__ TcShared sh;
    pdl_begin();
    // one sweep after the other, the shortest at the end: neighbouring SMs mostly run the same instructions
    const uint32_t each = gridDim.x / 3, which = blockIdx.x / each, block = blockIdx.x % each;
    if (which < 2) tc_sweep<MODE_GRAD, TC_BACK_UNROLL>(s.a[which], block, sh);
    else tc_sweep<MODE_OUT, TC_BACK_UNROLL>(s.a[2], block, sh);
}

// Sums of the tcgen05 sweeps' dB and dC over the heads of a group, and what each head's rows give with the rows of C and B (for the gradient of the
// log decays).  A block has 32 positions of a chunk, a warp eight columns of them, a thread one position; heads one after the other, eight on their
// way at a time.  Bound by memory: 403 MB of 16384 tokens and 24 heads in 70 us.
#define SUM_HEADS 16
#define SUM_AHEAD 8
__global__ void __launch_bounds__(512) k_clear_scan_tc_sums(const TcSums a) {
    __shared__ float dots[SUM_HEADS][16][33];
    pdl_begin();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31, which = blockIdx.x & 1, quarter = (blockIdx.x >> 1) & 3;
    const uint32_t per_seg = a.seg_chunks / 2, chunk = (blockIdx.x >> 3) % per_seg, seg = (blockIdx.x >> 3) / per_seg, grp = blockIdx.y, b = blockIdx.z;
    const int length = a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L;
    const int t_lo = (int)(seg * a.seg_chunks) * SCAN_Q, t_hi = min(length, t_lo + (int)a.seg_chunks * SCAN_Q), at = (int)(chunk * TC_Q + quarter * 32);
    if (t_lo + at >= t_hi) return;                                  // none of these positions exists
    const int pos = at + (int)lane, t = which ? t_hi - 1 - pos : t_lo + pos;          // 0: dC, forwards; 1: dB, backwards
    const bool live = t_lo + pos < t_hi;
    const uint32_t vheads = a.H * a.tiles, per = vheads / a.G, n = 8 * warp;
    const size_t step = (size_t)a.segments * per_seg * (TC_Q * 128);
    const float* src = (which ? a.part_b : a.part_c) + ((size_t)b * vheads + grp * per) * step + ((size_t)seg * per_seg + chunk) * (TC_Q * 128) +
                       (quarter * 4 + (warp >> 2)) * 1024 + (warp & 3) * 256 + lane * 8;
    const ScanOperand& o = which ? a.uB : a.uC;
    __nv_bfloat16* dst = which ? a.dB + b * a.Bb + t * a.Bt + grp * a.Bg : a.dC + b * a.Cb + t * a.Ct + grp * a.Cg;
    if (!DBG_REGION(src - lane * 8, ((per - 1) * step + 256) * sizeof(float)) || (live && !DBG_REGION(dst, a.N * sizeof(__nv_bfloat16)))) return;
    const bool there = live && n < a.N;
    const uint4 v = there ? *reinterpret_cast<const uint4*>((const __nv_bfloat16*)o.p + b * o.sb + t * o.st + grp * o.sh + n) : make_uint4(0, 0, 0, 0);
    const f2 u[4] = {both(v.x), both(v.y), both(v.z), both(v.w)};
    f2 sum[4] = {};
    float* out = which ? a.col : a.row;
    for (uint32_t h0 = 0; h0 < per; h0 += SUM_HEADS) {
        const uint32_t heads = min(per - h0, (uint32_t)SUM_HEADS);
        for (uint32_t h1 = 0; h1 < heads; h1 += SUM_AHEAD) {
            float4 x[SUM_AHEAD][2];
#pragma unroll
            for (uint32_t h = 0; h < SUM_AHEAD; h++)
                if (there && h1 + h < heads) {
                    const float4* p = reinterpret_cast<const float4*>(src + (h0 + h1 + h) * step);
                    x[h][0] = p[0], x[h][1] = p[1];
                }
#pragma unroll
            for (uint32_t h = 0; h < SUM_AHEAD; h++)
                if (h1 + h < heads) {
                    f2 dot = {0.f, 0.f};
                    if (there) {
#pragma unroll
                        for (int k = 0; k < 2; k++) {
                            const f2 p = {x[h][k].x, x[h][k].y}, q = {x[h][k].z, x[h][k].w};
                            sum[2 * k] = add2(sum[2 * k], p), sum[2 * k + 1] = add2(sum[2 * k + 1], q);
                            dot = fma2(u[2 * k + 1], q, fma2(u[2 * k], p, dot));
                        }
                    }
                    dots[h1 + h][warp][lane] = dot.x + dot.y;
                }
        }
        __syncthreads();
        for (uint32_t i = warp; i < heads; i += 16)
            if (live) {
                float s = 0.f;
#pragma unroll
                for (int w = 0; w < 16; w++) s += dots[i][w][lane];
                out[((size_t)b * vheads + grp * per + h0 + i) * a.L + t] = s;
            }
        __syncthreads();
    }
    if (!there) return;
    const uint32_t r[4] = {pack_bf16(sum[0].x, sum[0].y), pack_bf16(sum[1].x, sum[1].y), pack_bf16(sum[2].x, sum[2].y), pack_bf16(sum[3].x, sum[3].y)};
    if (a.wide && n + 8 <= a.N) {
        *reinterpret_cast<uint4*>(dst + n) = make_uint4(r[0], r[1], r[2], r[3]);
    } else {
#pragma unroll
        for (uint32_t e = 0; e < 8; e++)
            if (n + e < a.N) reinterpret_cast<uint16_t*>(dst)[n + e] = (uint16_t)(r[e / 2] >> (e & 1 ? 16 : 0));
    }
}
cudaError_t scan_tc_sums(const TcSums& a, uint32_t batch, cudaStream_t st) {
    return launch(k_clear_scan_tc_sums, dim3(8 * a.segments * (a.seg_chunks / 2), a.G, batch), dim3(512), 0, st, a);
}

cudaError_t scan_tc_launch(const ScanSet& s, int mode, cudaStream_t st) {
    auto go = [&](auto kernel, size_t smem) {
        cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        const ScanArgs& a = s.a[0];
        return e != cudaSuccess ? e : launch(kernel, dim3(s.count * a.b * a.segments * a.H * a.tiles), dim3(TC_THREADS), smem, st, s);
    };
    return mode == MODE_STATE ? go(k_clear_scan_tc_state, TcLayout<MODE_STATE>::bytes)
         : mode == MODE_OUT   ? go(k_clear_scan_tc, TcLayout<MODE_OUT>::bytes)
                              : go(k_clear_scan_tc_backward, std::max(TcLayout<MODE_GRAD>::bytes, TcLayout<MODE_OUT>::bytes));
}

// Copies operands whose rows do not allow 16-byte accesses into rows that do, with zeros behind their columns: at the price of one pass over them the
// sweeps run on tcgen05 (2048 tokens of 24 heads and 127 columns 98 -> 40 us).  A warp takes a token, blockIdx.z an operand.
__global__ void __launch_bounds__(256) k_clear_scan_pack(const TcPack a) {
    pdl_begin();
    const auto& o = a.o[blockIdx.z];
    const uint32_t lane = threadIdx.x & 31, b = blockIdx.y;
    const long long t = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int length = a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L;
    if (t >= length) return;
    const uint32_t pieces = (o.width + 7) / 8;
    const uint16_t* src = (const uint16_t*)o.src + b * o.sb + t * o.st;
    uint4* dst = (uint4*)o.dst + ((size_t)b * a.L + t) * o.heads * pieces;
    if (!DBG_REGION(src, ((o.heads - 1) * o.sh + o.width) * 2) || !DBG_REGION(dst, (size_t)o.heads * pieces * 16)) return;
    for (uint32_t i = lane; i < o.heads * pieces; i += 32) {
        const uint32_t h = i / pieces, c = i % pieces * 8;
        const uint16_t* p = src + h * o.sh + c;
        uint32_t v[4];
#pragma unroll
        for (uint32_t e = 0; e < 4; e++) v[e] = (c + 2 * e < o.width ? (uint32_t)p[2 * e] : 0u) | (c + 2 * e + 1 < o.width ? (uint32_t)p[2 * e + 1] << 16 : 0u);
        dst[i] = make_uint4(v[0], v[1], v[2], v[3]);
    }
}
cudaError_t scan_tc_pack(const TcPack& a, uint32_t batch, cudaStream_t st) {
    return a.L ? launch(k_clear_scan_pack, dim3((a.L + 7) / 8, batch, a.count), dim3(256), 0, st, a) : cudaSuccess;
}

// One warp waits on a barrier that nothing completes, as a sweep does under way and as it does at its end; the waits run out, the kernel records
// both and returns.
__global__ void k_clear_wait_limit() {
    __shared__ __align__(8) u64 bar;
    __shared__ volatile uint32_t dead;
    pdl_begin();
    const uint32_t at = (uint32_t)__cvta_generic_to_shared(&bar);
    if (threadIdx.x == 0) {
        mbar_init(at, 1);
        dead = 0;
        wait_on(at, 0, &dead);
        drain(at);
    }
}
extern "C" int fesc_clear_selftest_wait_limit(void* stream) {
    CLEAR_CUDA(launch(k_clear_wait_limit, dim3(1), dim3(32), 0, (cudaStream_t)stream));
    return FESC_OK;
}

extern "C" int fesc_clear_sync(void* stream) {
    CLEAR_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
    CLEAR_CUDA(cudaGetLastError());
    uint32_t status[2] = {};
    CLEAR_CUDA(cudaMemcpyFromSymbol(status, g_clear_status, sizeof(status)));
    if (!status[0] && !status[1]) return FESC_OK;
    const uint32_t none[2] = {};
    CLEAR_CUDA(cudaMemcpyToSymbol(g_clear_status, none, sizeof(none)));
    return clear_fail(FESC_ETIMEOUT, status[1] ? "a bounded wait on the tensor cores gave up, with products still under way at a kernel's end"
                                               : "a bounded wait on the tensor cores gave up");
}
