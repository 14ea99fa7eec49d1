// The sweep of the cleartext recurrence on the fifth-generation tensor cores (tcgen05), for bfloat16 and states of 65 to 128 columns: the
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
// Eight warps compute (a thread owns a row and half of the columns), one issues the products, one sums up the log decays of the next chunk.  The
// products of a chunk run while the threads are at something else: S and O1 while the faded values are formed, H while the scores are
// decayed, O2 while the state is updated; the next chunk's S while the outputs are written.
//
// Decays of pairs in different blocks of 32 tokens are products of two factors not above one (from the earlier token to its block's end,
// from there to the later one): one exponential per row and block; only the blocks on the diagonal take one per pair.
#define FESC_DBG_FILE 21   // file id in the sites a debug build reports
#include "clear_scan.cuh"

#define TC_Q 128
#define PANEL 16384u
#define TC_THREADS 320          // 8 computing warps, one that issues, one for the decays

template <int MODE>
struct TcLayout {
    static constexpr int NO = MODE == MODE_GRAD ? 3 : 2;            // planes of scores and states
    // panels in shared memory; k and v have two sets
    static constexpr int q = 0, QP = MODE == MODE_STATE ? 0 : MODE == MODE_OUT ? 2 : 1;
    static constexpr int broad = QP, narrow = broad + (MODE == MODE_STATE ? 2 : 4), w = narrow + (MODE == MODE_STATE ? 1 : 2), st = w + 3;
    static constexpr int panels = st + (MODE == MODE_STATE ? 0 : NO);
    // columns of tensor memory.  MODE_GRAD needs all 512: there the planes of the scores lie over the scores themselves
    static constexpr uint32_t DV = MODE == MODE_GRAD ? 128 : 64;
    static constexpr uint32_t S = MODE == MODE_GRAD ? 64 : 0, P = MODE == MODE_GRAD ? 0 : 128, O1 = MODE == MODE_GRAD ? 192 : 256, O2 = O1 + DV,
                              H = MODE == MODE_STATE ? 0 : O2 + DV, columns = MODE == MODE_STATE ? 64 : 512;
    static constexpr size_t bytes = (size_t)panels * PANEL + 1024;  // panels start on 1024 bytes
};

static __device__ uint32_t g_clear_status;      // not 0: a bounded wait gave up

// what the decays' warp leaves for a chunk
struct alignas(16) TcDecays {      // read four words at a time
    float2 cum[TC_Q];        // log2 of the decay up to a token, as two floats
    float tail[TC_Q];        // decay from a token to the end of its block of 32
    float grow[TC_Q];        // from the chunk's start to a token
    float fade[TC_Q];        // from a token to the chunk's end
    float2 ref[4];           // cum at the blocks' ends
    float keep;              // over the chunk
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
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
__device__ __forceinline__ void tc_ld32(uint32_t (&r)[32], uint32_t addr) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, "
        "%24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
          "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]),
          "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(addr), "r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
                 "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void bar_sync(uint32_t id, uint32_t threads) { asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory"); }
__device__ __forceinline__ void cp_async16_part(uint32_t dst, const void* src, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
// 32 bytes at a 32-byte boundary
__device__ __forceinline__ void st32(void* p, const uint32_t* v) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]),
                 "r"(v[7])
                 : "memory");
}

template <int MODE>
__global__ void __launch_bounds__(TC_THREADS, 1) k_clear_scan_tc(const ScanArgs a) {
    using Lay = TcLayout<MODE>;
    constexpr int NO = Lay::NO, NS = 3;
    extern __shared__ __align__(1024) uint8_t tc_smem[];
    __shared__ TcDecays decays[2];
    __shared__ __align__(8) u64 bars[12];
    __shared__ uint32_t tmem_base;
    __shared__ volatile uint32_t dead;          // a wait gave up: the rest of the chunks goes through without waiting, with nothing of worth in it
    __shared__ float words[2][8];
    pdl_begin();
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t vheads = a.H * a.tiles, vh = blockIdx.x % vheads, seg = blockIdx.x / vheads % a.segments, b = blockIdx.x / vheads / a.segments;
    const uint32_t head = vh / a.tiles, tile = vh % a.tiles, group = head / (a.H / a.G);
    const int length = a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L;
    const int seg_tokens = (int)a.seg_chunks * SCAN_Q, t_lo = (int)seg * seg_tokens, t_hi = min(length, t_lo + seg_tokens);
    const int pw = min(SCAN_TILE, (int)a.P - (int)tile * SCAN_TILE);
    const bool is_last = a.backwards ? seg == 0 : (t_hi == length && (t_lo < length || seg == 0));
    const size_t state_at = (size_t)head * a.P * a.N + (size_t)tile * SCAN_TILE * a.N, states = (size_t)a.H * a.P * a.N;
    const size_t slot = (size_t)b * a.segments + seg;
    if (MODE != MODE_STATE && t_lo >= length && !is_last) {
        if (MODE == MODE_GRAD && a.ends && tid == 0) a.ends[slot * vheads + vh] = 0.f, a.diag[slot * vheads + vh] = 0.f;
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
            ok = ok && DBG_REGION(scan_row<T>(a.u, b, t_lo, head, group, tile), (n * a.u.st + a.N) * sizeof(T)) &&
                 DBG_REGION(a.part + (((size_t)b * vheads + vh) * a.L + t_lo) * 128, (n + 1) * 128 * sizeof(float)) &&
                 DBG_REGION(a.dots + ((size_t)b * vheads + vh) * 2 * a.L, 2 * (size_t)a.L * sizeof(float));
        if (!ok) return;
    }
    if ((MODE && a.init && !DBG_REGION(a.init + (a.segments > 1 ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (a.last && !DBG_REGION(a.last + (MODE == MODE_STATE ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (MODE == MODE_GRAD && a.meet && !DBG_REGION(a.meet + (a.segments > 1 ? slot : b) * states + state_at, (size_t)pw * a.N * 4)))
        return;
#endif
    const uint32_t base = ((uint32_t)__cvta_generic_to_shared(tc_smem) + 1023) & ~1023u, bar = (uint32_t)__cvta_generic_to_shared(bars);
    uint8_t* const panels = tc_smem + (base - (uint32_t)__cvta_generic_to_shared(tc_smem));
    const uint32_t b_load = bar, b_wv = bar + 8, b_p = bar + 16, b_epi = bar + 24, b_so = bar + 32, b_h = bar + 40, b_o = bar + 48, drained = bar + 56;
    // of the two sets of decays: filled, and used; a set has barriers of its own because the warp that fills them runs up to two chunks ahead
    const uint32_t b_g = bar + 64, b_used = bar + 80;
    if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"((uint32_t)__cvta_generic_to_shared(&tmem_base)), "n"(Lay::columns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        mbar_init(b_load, 8), mbar_init(b_wv, 8), mbar_init(b_p, 8), mbar_init(b_epi, 8);
        for (uint32_t i = 0; i < 2; i++) mbar_init(b_g + 8 * i, 1), mbar_init(b_used + 8 * i, 8);
        mbar_init(b_so, 1), mbar_init(b_h, 1), mbar_init(b_o, 1), mbar_init(drained, 1);
        dead = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = tmem_base;
    const int chunks = t_hi > t_lo ? (t_hi - t_lo + TC_Q - 1) / TC_Q : 0, dir = a.backwards ? -1 : 1;
    auto wait = [&](uint32_t which, uint32_t parity) {
        if (!dead && mbar_wait_bounded(which, parity & 1)) dead = 1, g_clear_status = 1;
    };

    if (warp == 8) {
        // issues the products
        constexpr uint32_t IDESC = (1u << 4) | (1u << 7) | (1u << 10) | (8u << 24);        // bfloat16 x bfloat16 -> float32, 128 rows
        constexpr uint32_t I_S = IDESC | (16u << 17), I_H = IDESC | (1u << 15) | (1u << 16) | (8u << 17);
        constexpr uint32_t I_O1 = IDESC | (MODE == MODE_GRAD ? 16u << 17 : (8u << 17) | (1u << 16)), I_O2 = IDESC | (1u << 16) | ((Lay::DV / 8) << 17);
        if (lane == 0) {
            const uint32_t pq = tc_desc(base + Lay::q * PANEL), pw_ = tc_desc(base + Lay::w * PANEL), ps = tc_desc(base + Lay::st * PANEL);
            constexpr uint32_t STEP = PANEL >> 4;
            for (int c = 0; c < chunks; c++) {
                const uint32_t set = MODE == MODE_STATE ? 0 : c & 1;
                const uint32_t pb = tc_desc(base + (Lay::broad + 2 * set) * PANEL), pn = tc_desc(base + (Lay::narrow + set) * PANEL);
                if (MODE) {
                    wait(b_load, c);
                    if (MODE == MODE_GRAD && c) wait(b_o, c - 1);        // the scores' planes lie over the scores
                    tc_after();
                    if (!dead) {
#pragma unroll
                        for (uint32_t k = 0; k < (MODE == MODE_OUT ? 8 : 4); k++) {
                            const uint32_t at = (k >> 2) * STEP + (k & 3) * 2;
                            tc_mma_ss(tmem + Lay::S, pq + at, (MODE == MODE_OUT ? pb : pn) + at, I_S, k);
                        }
                    }
                    if (c) wait(b_epi, c - 1);
                    tc_after();
                    if (!dead) {
#pragma unroll
                        for (uint32_t p = 0; p < NO; p++)
#pragma unroll
                            for (uint32_t k = 0; k < (MODE == MODE_OUT ? 8 : 4); k++) {
                                const uint32_t at = (k >> 2) * STEP + (k & 3) * 2;
                                tc_mma_ss(tmem + Lay::O1, pq + at, ps + p * STEP + (MODE == MODE_OUT ? k * 128 : (k & 3) * 2), I_O1, p || k);
                            }
                        tc_commit(b_so);
                    }
                }
                wait(b_wv, c);
                tc_after();
                if (!dead) {
#pragma unroll
                    for (uint32_t p = 0; p < NS; p++)
#pragma unroll
                        for (uint32_t k = 0; k < 8; k++) tc_mma_ss(tmem + Lay::H, pb + k * 128, pw_ + p * STEP + k * 128, I_H, p || k);
                    tc_commit(b_h);
                }
                if (MODE) {
                    wait(b_p, c);
                    tc_after();
                    if (!dead) {
#pragma unroll
                        for (uint32_t p = 0; p < NO; p++)
#pragma unroll
                            for (uint32_t k = 0; k < 8; k++)
                                tc_mma_ts(tmem + Lay::O2, tmem + Lay::P + 64 * p + 8 * k, (MODE == MODE_GRAD ? pb : pn) + k * 128, I_O2, p || k);
                        tc_commit(b_o);
                    }
                }
            }
            tc_commit(drained);
            mbar_wait_bounded(drained, 0);
        }
        __syncwarp();
    } else if (warp == 9) {
        // log decays of a chunk, four tokens a lane
        const float* g = a.g + b * a.gb + head * a.gh;
        double through = 0.0;
        for (int c = 0; c < chunks; c++) {
            const int valid = min(TC_Q, t_hi - t_lo - c * TC_Q), t0 = a.backwards ? t_hi - 1 - c * TC_Q : t_lo + c * TC_Q;
            float gv[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int pos = 4 * lane + i, t = t0 + dir * pos + (a.backwards ? 1 : 0);
                gv[i] = pos < valid && t < length ? g[t * a.gt] : 0.f;
            }
            double sum[4];
#pragma unroll
            for (int i = 0; i < 4; i++) sum[i] = (double)(gv[i] < SCAN_DROP ? SCAN_DROP : gv[i]) * 1.4426950408889634 + (i ? sum[i - 1] : 0.0);
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
            if (lane == 0) d.keep = ex2((float)total);
            through += total;
            __syncwarp();
            if (lane == 0) mbar_arrive(b_g + 8 * (c & 1));
        }
        if (MODE == MODE_STATE && lane == 0 && tile == 0) a.decay[slot * a.H + head] = (float)exp2(through);
    } else {
        const uint32_t quarter = warp & 3, half = warp >> 2, row = 32 * quarter + lane;     // row: token of the chunk, or column of the state
        const uint32_t lanes = tmem + (quarter << 21);
        float st[32];                                                                        // state[channel 32 half + i][column row]
        const float* init = MODE && a.init ? a.init + (a.segments > 1 ? slot : b) * states + state_at : nullptr;
#pragma unroll
        for (int i = 0; i < 32; i++) {
            const int p = 32 * half + i;
            st[i] = init && p < pw && row < a.N ? init[(size_t)p * a.N + row] : 0.f;
        }
        auto put_state = [&]() {
#pragma unroll
            for (int k = 0; k < 4; k++) {
                uint32_t pl[4][NO];
#pragma unroll
                for (int e = 0; e < 4; e++) split<NO>(st[8 * k + 2 * e], st[8 * k + 2 * e + 1], pl[e]);
#pragma unroll
                for (int p = 0; p < NO; p++)
                    *reinterpret_cast<uint4*>(panels + (Lay::st + p) * PANEL + panel_at(row, 4 * half + k)) = make_uint4(pl[0][p], pl[1][p], pl[2][p], pl[3][p]);
            }
        };
        // `n` panels of an operand's rows for chunk c: a thread copies chunks of 16 bytes, eight threads a row of 128
        auto fetch = [&](const ScanOperand& o, int width, int first, int n, int c) {
            const int valid = min(TC_Q, t_hi - t_lo - c * TC_Q), t0 = a.backwards ? t_hi - 1 - c * TC_Q : t_lo + c * TC_Q;
            const T* src = scan_row<T>(o, b, t0, head, group, tile);
            const long long step = dir * o.st;
#pragma unroll
            for (int i = 0; i < n * 4; i++) {
                const int r = (int)(tid >> 3) + 32 * (i & 3), col = (int)(tid & 7) * 8 + 64 * (i >> 2), left = r < valid ? min(width - col, 8) : 0;
                cp_async16_part(base + (first + (i >> 2)) * PANEL + panel_at(r, tid & 7), left > 0 ? src + r * step + col : src, left > 0 ? left * 2 : 0);
            }
        };
        auto arrive = [&](uint32_t which) {
            __syncwarp();
            if (lane == 0) mbar_arrive(which);
        };
        float diag = 0.f;
        if (chunks) {
            if (MODE) fetch(a.q, qw, Lay::q, Lay::QP, 0);
            fetch(ob, (int)a.N, Lay::broad, 2, 0);
            fetch(on, pw, Lay::narrow, 1, 0);
            if (MODE) {
                put_state();
                if (MODE == MODE_OUT) {
                    // blocks above the diagonal are zero for good
                    uint32_t zero[16] = {};
                    for (uint32_t J = quarter + 1; J < 4; J++)
                        if ((J & 1) == half)
                            for (int p = 0; p < NO; p++) tc_st16(lanes + Lay::P + 64 * p + 16 * J, zero);
                    tc_wait_st();
                }
            }
            cp_async_wait();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_before();
            if (MODE) arrive(b_load);
        }
        for (int c = 0; c < chunks; c++) {
            const int valid = min(TC_Q, t_hi - t_lo - c * TC_Q), t0 = a.backwards ? t_hi - 1 - c * TC_Q : t_lo + c * TC_Q;
            const int set = MODE == MODE_STATE ? 0 : c & 1, nset = MODE == MODE_STATE ? 0 : set ^ 1;
            const TcDecays& d = decays[c & 1];
            bar_sync(1, 256);                    // everyone's copies have landed, everyone is done with the chunk before
            if (MODE && c + 1 < chunks) {
                fetch(ob, (int)a.N, Lay::broad + 2 * nset, 2, c + 1);
                fetch(on, pw, Lay::narrow + nset, 1, c + 1);
            }
            wait(b_g + 8 * (c & 1), c >> 1);
            {
                const float f = d.fade[row];
                const uint8_t* src = panels + (Lay::narrow + set) * PANEL;
#pragma unroll
                for (int k = 0; k < 4; k++) {
                    const uint4 v = *reinterpret_cast<const uint4*>(src + panel_at(row, 4 * half + k));
                    const uint32_t u[4] = {v.x, v.y, v.z, v.w};
                    uint32_t pl[4][NS];
#pragma unroll
                    for (int e = 0; e < 4; e++) split<NS>(__uint_as_float(u[e] << 16) * f, __uint_as_float(u[e] & 0xFFFF0000u) * f, pl[e]);
#pragma unroll
                    for (int p = 0; p < NS; p++)
                        *reinterpret_cast<uint4*>(panels + (Lay::w + p) * PANEL + panel_at(row, 4 * half + k)) = make_uint4(pl[0][p], pl[1][p], pl[2][p], pl[3][p]);
                }
            }
            const float keep = d.keep;
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            arrive(b_wv);
            if (MODE) {
                wait(b_so, c);
                tc_after();
                // decayed scores of this row, blocks half and half + 2 of 32 columns
                const float2 ci = d.cum[row];
                uint32_t x[2][32];
#pragma unroll
                for (int B = 0; B < 2; B++)
                    if (2 * B + half <= quarter) tc_ld32(x[B], lanes + Lay::S + 32 * (2 * B + half));
                tc_wait_ld();
                if (MODE == MODE_GRAD) {
                    tc_before();
                    bar_sync(2 + quarter, 64);      // the other warp of these rows has its scores too
                    tc_after();
                }
#pragma unroll
                for (int B = 0; B < 2; B++) {
                    const uint32_t J = 2 * B + half;
                    uint32_t pl[NO][16];
                    if (J > quarter) {
                        if (MODE == MODE_OUT) continue;
#pragma unroll
                        for (int p = 0; p < NO; p++)
#pragma unroll
                            for (int e = 0; e < 16; e++) pl[p][e] = 0;
                    } else if (J < quarter) {
                        const float2 ref = d.ref[J];
                        const float r = ex2((ci.x - ref.x) + (ci.y - ref.y));
#pragma unroll
                        for (int e = 0; e < 16; e++) {
                            const float2 t = *reinterpret_cast<const float2*>(&d.tail[32 * J + 2 * e]);
                            uint32_t q[NO];
                            split<NO>(__uint_as_float(x[B][2 * e]) * (r * t.x), __uint_as_float(x[B][2 * e + 1]) * (r * t.y), q);
#pragma unroll
                            for (int p = 0; p < NO; p++) pl[p][e] = q[p];
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 16; e++) {
                            const float4 cj = *reinterpret_cast<const float4*>(&d.cum[32 * J + 2 * e]);
                            const float s0 = __uint_as_float(x[B][2 * e]), s1 = __uint_as_float(x[B][2 * e + 1]);
                            const float g0 = ex2((ci.x - cj.x) + (ci.y - cj.y)), g1 = ex2((ci.x - cj.z) + (ci.y - cj.w));
                            if (MODE == MODE_GRAD) diag += (lane == 2 * e ? s0 : 0.f) + (lane == 2 * e + 1 ? s1 : 0.f);
                            uint32_t q[NO];
                            split<NO>(2 * e <= lane ? s0 * g0 : 0.f, 2 * e + 1 <= lane ? s1 * g1 : 0.f, q);
#pragma unroll
                            for (int p = 0; p < NO; p++) pl[p][e] = q[p];
                        }
                    }
#pragma unroll
                    for (int p = 0; p < NO; p++) tc_st16(lanes + Lay::P + 64 * p + 16 * J, pl[p]);
                }
                tc_wait_st();
                tc_before();
                arrive(b_p);
                if (c + 1 < chunks) fetch(a.q, qw, Lay::q, Lay::QP, c + 1);
            }
            wait(b_h, c);
            tc_after();
            {
                uint32_t x[32];
                tc_ld32(x, lanes + Lay::H + 32 * half);
                tc_wait_ld();
#pragma unroll
                for (int i = 0; i < 32; i++) st[i] = fmaf(st[i], keep, __uint_as_float(x[i]));
            }
            if (MODE == MODE_STATE) {
                if (c + 1 < chunks) {
                    fetch(ob, (int)a.N, Lay::broad, 2, c + 1);
                    fetch(on, pw, Lay::narrow, 1, c + 1);
                    cp_async_wait();
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                }
                tc_before();
                arrive(b_used + 8 * (c & 1));
                continue;
            }
            if (c + 1 < chunks) put_state();
            cp_async_wait();
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            tc_before();
            if (c + 1 < chunks) arrive(b_load);

            const float grow = d.grow[row];
            arrive(b_used + 8 * (c & 1));
            const bool live = (int)row < valid;
            const long long t = t0 + (long long)dir * (int)row;
            if (MODE == MODE_OUT) {
                uint32_t skipped[4][4] = {};
                const float skip = a.skip ? a.skip[head] : 0.f;
                if (a.skip) {
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        const uint4 v = *reinterpret_cast<const uint4*>(panels + (Lay::narrow + set) * PANEL + panel_at(row, 4 * half + k));
                        skipped[k][0] = v.x, skipped[k][1] = v.y, skipped[k][2] = v.z, skipped[k][3] = v.w;
                    }
                }
                wait(b_o, c);
                tc_after();
                uint32_t x[32], y[32];
                tc_ld32(x, lanes + Lay::O1 + 32 * half);
                tc_ld32(y, lanes + Lay::O2 + 32 * half);
                tc_wait_ld();
                tc_before();
                arrive(b_epi);
                T* out = (T*)a.out + b * a.ob + t * a.ot + head * a.oh + tile * SCAN_TILE + 32 * half;
                const int count = live ? vw - 32 * (int)half : 0;
                uint32_t o[16];
#pragma unroll
                for (int e = 0; e < 16; e++) {
                    const uint32_t s = skipped[e >> 2][e & 3];
                    const float o0 = fmaf(grow, __uint_as_float(x[2 * e]), __uint_as_float(y[2 * e])) + skip * __uint_as_float(s << 16);
                    const float o1 = fmaf(grow, __uint_as_float(x[2 * e + 1]), __uint_as_float(y[2 * e + 1])) + skip * __uint_as_float(s & 0xFFFF0000u);
                    o[e] = pack_bf16(o0, o1);
                }
                if (a.out_wide > 1 && count >= 32) {
                    st32(out, o), st32(out + 16, o + 8);
                } else if (a.out_wide) {
#pragma unroll
                    for (int k = 0; k < 4; k++) {
                        if (count >= 8 * k + 8) {
                            *reinterpret_cast<uint4*>(out + 8 * k) = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                            continue;
                        }
#pragma unroll
                        for (int e = 0; e < 8; e++)
                            if (8 * k + e < count) reinterpret_cast<uint16_t*>(out)[8 * k + e] = (uint16_t)(o[4 * k + e / 2] >> (e & 1 ? 16 : 0));
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 32; e++)
                        if (e < count) reinterpret_cast<uint16_t*>(out)[e] = (uint16_t)(o[e / 2] >> (e & 1 ? 16 : 0));
                }
            } else {
                // u's half row is on its way while the products finish
                uint32_t u[32];
                const T* pu = scan_row<T>(a.u, b, t0 + dir * min((int)row, valid - 1), head, group, tile) + 64 * half;
#pragma unroll
                for (int k = 0; k < 8; k++) {
                    const int count = (int)a.N - 64 * (int)half - 8 * k;
                    uint4 v = make_uint4(0, 0, 0, 0);
                    if (a.u.wide && count >= 8) v = *reinterpret_cast<const uint4*>(pu + 8 * k);
                    else {
                        uint32_t h[4];
#pragma unroll
                        for (int e = 0; e < 4; e++)
                            h[e] = (2 * e < count ? (uint32_t)reinterpret_cast<const uint16_t*>(pu)[8 * k + 2 * e] : 0u) |
                                   (2 * e + 1 < count ? (uint32_t)reinterpret_cast<const uint16_t*>(pu)[8 * k + 2 * e + 1] << 16 : 0u);
                        v = make_uint4(h[0], h[1], h[2], h[3]);
                    }
                    u[4 * k] = v.x, u[4 * k + 1] = v.y, u[4 * k + 2] = v.z, u[4 * k + 3] = v.w;
                }
                wait(b_o, c);
                tc_after();
                float dot = 0.f;
                float* part = a.part + (((size_t)b * vheads + vh) * a.L + t) * 128 + 64 * half;
#pragma unroll
                for (int k = 0; k < 2; k++) {
                    uint32_t x[32], y[32];
                    tc_ld32(x, lanes + Lay::O1 + 64 * half + 32 * k);
                    tc_ld32(y, lanes + Lay::O2 + 64 * half + 32 * k);
                    tc_wait_ld();
                    if (k == 1) {
                        tc_before();
                        arrive(b_epi);
                    }
#pragma unroll
                    for (int e = 0; e < 32; e++) {
                        const float v = fmaf(grow, __uint_as_float(x[e]), __uint_as_float(y[e]));
                        const uint32_t w = u[16 * k + e / 2];
                        dot = fmaf(v, __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16), dot);
                        x[e] = __float_as_uint(v);
                    }
                    if (live)
#pragma unroll
                        for (int e = 0; e < 4; e++) st32(part + 32 * k + 8 * e, x + 8 * e);
                }
                if (live) a.dots[(((size_t)b * vheads + vh) * 2 + half) * a.L + t] = dot;
            }
        }
        if (a.last && (MODE == MODE_STATE || is_last)) {
            float* last = a.last + (MODE == MODE_STATE ? slot : b) * states + state_at;
            const float f = MODE && a.backwards && length > 0 ? expf(a.g[b * a.gb + head * a.gh]) : 1.f;
#pragma unroll
            for (int i = 0; i < 32; i++) {
                const int p = 32 * half + i;
                if (p < pw && row < a.N) last[(size_t)p * a.N + row] = st[i] * f;
            }
        }
        if (MODE == MODE_GRAD && a.ends) {
            float sum = 0.f;
            const float* meet = a.meet ? a.meet + (a.segments > 1 ? slot : b) * states + state_at : nullptr;
            if (meet) {
#pragma unroll
                for (int i = 0; i < 32; i++) {
                    const int p = 32 * half + i;
                    if (p < pw && row < a.N) sum += st[i] * meet[(size_t)p * a.N + row];
                }
                if (t_hi < length) sum *= expf(a.g[b * a.gb + t_hi * a.gt + head * a.gh]);
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o), diag += __shfl_xor_sync(~0u, diag, o);
            if (lane == 0) words[0][warp] = sum, words[1][warp] = diag;
            bar_sync(1, 256);
            if (tid == 0) {
                float s0 = 0.f, s1 = 0.f;
                for (int w = 0; w < 8; w++) s0 += words[0][w], s1 += words[1][w];
                a.ends[slot * vheads + vh] = s0, a.diag[slot * vheads + vh] = s1;
            }
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Lay::columns));
}

cudaError_t scan_tc_launch(const ScanArgs& a, int mode, cudaStream_t st) {
    auto go = [&](auto kernel, size_t smem) {
        cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        return e != cudaSuccess ? e : launch(kernel, dim3(a.b * a.segments * a.H * a.tiles), dim3(TC_THREADS), smem, st, a);
    };
    return mode == MODE_STATE ? go(k_clear_scan_tc<MODE_STATE>, TcLayout<MODE_STATE>::bytes)
         : mode == MODE_OUT   ? go(k_clear_scan_tc<MODE_OUT>, TcLayout<MODE_OUT>::bytes)
                              : go(k_clear_scan_tc<MODE_GRAD>, TcLayout<MODE_GRAD>::bytes);
}

extern "C" int fesc_clear_sync(void* stream) {
    CLEAR_CUDA(cudaStreamSynchronize((cudaStream_t)stream));
    CLEAR_CUDA(cudaGetLastError());
    uint32_t status = 0;
    CLEAR_CUDA(cudaMemcpyFromSymbol(&status, g_clear_status, sizeof(status)));
    if (!status) return FESC_OK;
    status = 0;
    CLEAR_CUDA(cudaMemcpyToSymbol(g_clear_status, &status, sizeof(status)));
    return clear_fail(FESC_ETIMEOUT, "a bounded wait on the tensor cores gave up");
}
