// The sweep behind the cleartext gated linear recurrence: over the tokens of a sequence, forwards or backwards in time,
//   out_i = sum_{j<=i} G_ij (q_i . k_j) v_j + G_i state q_i,   G_ij = exp(sum of the log decays after j up to i),
//   state <- G_last state + sum_j G_last,j v_j k_j^T.
// The scan is the sweep with (q, k, v) = (C, B, x); of its backward pass dx is the sweep backwards with (B, C, dy), dB the one with
// (x, dy, C) and dC the sweep forwards with (dy, x, B).  Heads of more than 64 channels are cut into tiles of 64, which act as heads of their own.
//
// Tokens go in chunks of 64.  Within a chunk the sum is two matrix products with the decays between them (64 x 64 scores); the state carries
// everything before it.  The state of a head tile (64 channels x up to 128) stays in the warps' registers in the accumulator layout of
// mma.m16n8k16, which is also the layout of a left operand: the products are formed transposed (out^T = state q^T + v^T S^T) so that the state
// multiplies q without going through memory.
// A long sequence is cut into segments when there are too few heads to fill the SMs: the sweep in MODE_STATE gives what every segment adds to
// its state, k_clear_combine chains the segments, and every segment then runs with the state before it.
// Measured (24 heads, 128 columns, 2048 tokens): float16 95 us, float32 113; 8 x 1024 tokens of 12 heads in float32 192.  A chunk is loads, scores,
// products, outputs one after the other, with three to six matrix instructions per product of float32 planes; what bounds it are those chains.
//
// Operands are sums of bfloat16 numbers ("planes"): bfloat16 inputs one, float16 two (exact), float32 three (24 bits).  What the kernel
// computes itself (decayed scores, weighted values, states) is cut into two planes (17 bits) where only outputs of 16 bits depend on it, and
// into three (25 bits) where a float32 result does: states and the gradient of the log decays.  One plane would take
// the error of 16-bit results to 1.4 times theirs (another rounding as large as the one at the end) and that of states to 2^-9.  Products of two parts
// that are both small are left out: what they would add is below 2^-26 of the whole, in 16-bit outputs below 2^-17.  All sums are in float32.
// The tensor cores cut what does not fit into such a sum, always towards zero.  Outputs are sums of a chunk's tokens, where that stays near 2^-20 (float32
// results of 4096 tokens: 5e-7 to 1e-6); a state lives on, so what 16 tokens add to it is summed apart and added with rounding.  Summed in the state itself, a
// state of 4096 tokens that forgets little was off by 2e-5 (now 4e-7), for 3 to 8 % of the time.
//
// Log decays are summed in float64 per chunk and kept as two floats: with |g| up to 300 a token (below that a decay is zero: also -inf), one
// float would leave 2^-10 of an exponent behind a strong decay.
#pragma once
#include "clear.cuh"

#define SCAN_Q 64            // tokens of a chunk
#define SCAN_TILE 64         // channels of a head tile
#define SCAN_MAX_STATE 128   // columns of a state
#define SCAN_DROP (-300.f)   // log decays below this drop the state
#define SCAN_PAD 8           // bfloat16 numbers behind a row in shared memory: eight rows start in different banks
enum { MODE_STATE = 0, MODE_OUT = 1, MODE_GRAD = 2 };

struct ScanOperand {
    const void* p;
    long long sb, st, sh;    // strides of batch, token and head (or group), in elements
    uint32_t tiled;          // 1: a head's channels (64 of P from the tile), 0: a group's columns (N)
    uint32_t align;          // bytes that rows are aligned to: 16, 8, 4 or less
};
struct ScanArgs {
    ScanOperand q, k, v, u;          // u (MODE_GRAD): the row that the output's row is multiplied with, for the gradient of the log decays
    const float* g;
    long long gb, gt, gh;
    const int* lengths;              // tokens of every sequence, nullptr: L
    const float* skip;               // MODE_OUT: out += skip[head] v
    void* out;                       // MODE_OUT
    long long ob, ot, oh;
    uint32_t out_wide;               // 16-byte accesses are possible (2: 32-byte ones)
    const float* init;               // state before the sweep (or before every segment): [b][H][P][N] (segments: [b][segment][H][P][N])
    float* last;                     // state behind the sweep (MODE_STATE: what a segment adds), or nullptr
    float* decay;                    // MODE_STATE: [b][segment][H], the decay over the segment
    float* part;                     // MODE_GRAD: [b][head tile][L][NP], NP = 64 or 128
    float* dots;                     // MODE_GRAD: [b][head tile][L], u . out
    const float* meet;               // MODE_GRAD forwards: states of the sweep backwards, as `init`; their product with this one's at the segments' ends
    float* ends;                     //   [b][segment][head tile]; backwards: of h0 (meet) with the gradient before the first token, segment 0
    float* diag;                     //   sum over a segment's tokens of q . k, [b][segment][head tile]; segments are added up in 64 bits
    uint32_t b, L, H, P, G, N, tiles, segments, seg_chunks, backwards;
};

// The sweeps of a launch: MODE_STATE one or two, MODE_OUT one, MODE_GRAD three (dC, dB, and dx as MODE_OUT).  Heads, tokens and segments are the same.
struct ScanSet {
    ScanArgs a[3];
    uint32_t count;
};

// an operand's row: token t of sequence b for head h, tile s
template <class T>
__device__ __forceinline__ const T* scan_row(const ScanOperand& o, uint32_t b, long long t, uint32_t head, uint32_t group, uint32_t tile) {
    return (const T*)o.p + b * o.sb + t * o.st + (o.tiled ? head * o.sh + tile * SCAN_TILE : group * o.sh);
}

// 2^v to 0.6 units in the last place: the series of exp around the nearest whole exponent, (v - n) ln 2 within 0.35, so that its ninth term is below 2^-27.
// A decay that is multiplied into the state chunk after chunk takes this: the two units of exp2f lean to one side for decays that are alike, and add up.
__device__ __forceinline__ float exp2_near(double v) {
    if (!(fabs(v) < 126.0)) return exp2f((float)v);       // also NaN
    const float n = rintf((float)v), x = (float)((v - n) * 0.6931471805599453);
    float p = 1.f;
#pragma unroll
    for (int k = 8; k >= 2; k--) p = fmaf(p * x, 1.f / k, 1.f);
    return fmaf(x, p, 1.f) * __int_as_float(((int)n + 127) << 23);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
// two numbers as sums of NM bfloat16 numbers each, largest first
template <int NM>
__device__ __forceinline__ void split(float a, float b, uint32_t (&p)[NM]) {
#pragma unroll
    for (int i = 0; i < NM; i++) {
        p[i] = pack_bf16(a, b);
        if (i + 1 < NM) a -= __uint_as_float(p[i] << 16), b -= __uint_as_float(p[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// a piece of `SIZE` bytes of every row's end to end copy, `bytes` of them from memory and zeros behind
template <int SIZE>
__device__ __forceinline__ void cp_async_part(uint32_t dst, const void* src, uint32_t bytes) {
    if constexpr (SIZE == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(dst), "l"(src), "r"(bytes), "n"(SIZE) : "memory");
}
template <int SIZE, int D, int THREADS, class T>
__device__ __forceinline__ void copy_tile(uint32_t base, const T* src, long long step, int rows, int width) {
    constexpr int E = SIZE / 2;       // numbers in a piece
#pragma unroll 4
    for (int i = threadIdx.x; i < SCAN_Q * D / E; i += THREADS) {
        const int r = i / (D / E), c = i % (D / E) * E, bytes = r < rows ? min(max(width - c, 0), E) * 2 : 0;
        cp_async_part<SIZE>(base + (r * (D + SCAN_PAD) + c) * 2, bytes ? src + r * step + c : src, bytes);
    }
}

// SCAN_Q rows of up to D columns into shared memory, plane by plane; zeros beyond `rows` and `width`.  step: elements from one row to the next.
// align: bytes that rows are aligned to.  bfloat16 rows are copied asynchronously in the largest pieces that allows; what has to be cut into planes
// passes through registers, several loads at a time.
template <class T, int D, int THREADS>
__device__ __forceinline__ void load_tile(__nv_bfloat16* dst, const T* src, long long step, int rows, int width, uint32_t align) {
    constexpr int NI = ClearType<T>::planes, STR = D + SCAN_PAD, AHEAD = SCAN_Q * D / 8 / THREADS;      // all of a thread's pieces at once
    if (align < (NI == 1 ? 4 : 16)) {
        // element by element, neighbouring threads neighbouring columns, 16 loads at a time
#pragma unroll 1
        for (int i0 = threadIdx.x; i0 < SCAN_Q * D; i0 += THREADS * 16) {
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; k++) {
                const int i = i0 + k * THREADS, r = i / D, c = i % D;
                v[k] = r < rows && c < width ? ClearType<T>::to(src[r * step + c]) : 0.f;
            }
#pragma unroll
            for (int k = 0; k < 16; k++) {
                const int i = i0 + k * THREADS, r = i / D, c = i % D;
                uint32_t pl[NI];
                split<NI>(v[k], 0.f, pl);
#pragma unroll
                for (int j = 0; j < NI; j++) reinterpret_cast<uint16_t*>(dst)[j * SCAN_Q * STR + r * STR + c] = (uint16_t)pl[j];
            }
        }
        return;
    }
    if constexpr (NI == 1) {
        const uint32_t base = (uint32_t)__cvta_generic_to_shared(dst);
        if (align >= 16) copy_tile<16, D, THREADS>(base, src, step, rows, width);
        else if (align >= 8) copy_tile<8, D, THREADS>(base, src, step, rows, width);
        else copy_tile<4, D, THREADS>(base, src, step, rows, width);
    } else {
#pragma unroll 1
        for (int i0 = threadIdx.x; i0 < SCAN_Q * D / 8; i0 += THREADS * AHEAD) {
            float v[AHEAD][8];
#pragma unroll
            for (int k = 0; k < AHEAD; k++) {
                const int i = i0 + k * THREADS, r = i / (D / 8), c = i % (D / 8) * 8, count = r < rows ? width - c : 0;
                clear_load8(src + r * step + c, count >= 8 ? 8 : 0, count >= 8, v[k]);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; k++) {
                const int i = i0 + k * THREADS, r = i / (D / 8), c = i % (D / 8) * 8;
                uint32_t pl[4][NI];
#pragma unroll
                for (int e = 0; e < 4; e++) split<NI>(v[k][2 * e], v[k][2 * e + 1], pl[e]);
#pragma unroll
                for (int j = 0; j < NI; j++)
                    *reinterpret_cast<uint4*>(dst + j * SCAN_Q * STR + r * STR + c) = make_uint4(pl[0][j], pl[1][j], pl[2][j], pl[3][j]);
            }
        }
        if (width & 7) {         // the columns behind the last eight, over the zeros
            __syncthreads();
#pragma unroll 1
            for (int i = threadIdx.x; i < rows * 8; i += THREADS) {
                const int r = i >> 3, c = (width & ~7) + (i & 7);
                if (c >= width) continue;
                uint32_t pl[NI];
                split<NI>(ClearType<T>::to(src[r * step + c]), 0.f, pl);
#pragma unroll
                for (int j = 0; j < NI; j++) reinterpret_cast<uint16_t*>(dst)[j * SCAN_Q * STR + r * STR + c] = (uint16_t)pl[j];
            }
        }
    }
}

// A CTA has four warps for four slices of v's columns, and as many again where two share a slice, one for each half of k's columns: with operands of
// several planes one CTA or two fill an SM's shared memory, and four warps each wait for their own products (8 x 1024 tokens of 12 heads in
// float32 284 us against 210).  With one plane three CTAs fit, and what two warps of a slice both have to do costs more (66 against 89).
template <class T>
struct ScanWarps {
    static constexpr int halves = ClearType<T>::planes == 1 ? 1 : 2, threads = 128 * halves;
};
template <class T, int DK, int DV, int MODE>
struct ScanShared {
    static constexpr int NI = ClearType<T>::planes;
    static constexpr int NO = MODE == MODE_GRAD || NI == 3 ? 3 : 2;   // planes of what only the outputs depend on
    static constexpr int K_STR = DK + SCAN_PAD, V_STR = DV + SCAN_PAD, S_STR = SCAN_Q + SCAN_PAD;
    static constexpr int k = 0, v = k + NI * SCAN_Q * K_STR, q = v + NI * SCAN_Q * V_STR, s = q + (MODE ? NI * SCAN_Q * K_STR : 0);
    static constexpr int words = s + (MODE ? NO * SCAN_Q * S_STR : 0);                        // in bfloat16 numbers
    static constexpr int O_STR = DV + 4;                                                       // floats; the outputs' rows lie over q and the scores
    static_assert(!MODE || (words - q) * 2 >= SCAN_Q * O_STR * 4, "outputs fit over q and the scores");
    static constexpr int H_STR = (MODE == MODE_GRAD ? DV : DK) + 4;                           // floats; states pass through all of it, 64 rows
    static constexpr size_t bytes = std::max((size_t)words * 2, (size_t)SCAN_TILE * H_STR * 4);
};

template <class T, int DK, int DV, int MODE>
__device__ __forceinline__ void sweep(const ScanArgs& a, uint32_t block) {
    using S = ScanShared<T, DK, DV, MODE>;
    constexpr int NI = S::NI, NO = S::NO, NS = 3, MT = DV / 64, HALVES = ScanWarps<T>::halves, THREADS = ScanWarps<T>::threads, KH = DK / HALVES, KT = KH / 8;
    extern __shared__ __align__(128) __nv_bfloat16 sm[];
    __shared__ __align__(16) float2 cum[SCAN_Q];               // log2 of the decay up to a token of the chunk, as a sum of two floats
    __shared__ __align__(16) float grow[SCAN_Q], fade[SCAN_Q]; // decay from the chunk's start to a token; from a token to the chunk's end
    __shared__ float words[2][THREADS / 32];
    // a warp's slice of the columns of v, and its half of those of k (or all of them); the halves of a slice's outputs are added up at the end
    const uint32_t tid = threadIdx.x, warp = tid >> 5, slice = warp & 3, half = HALVES == 1 ? 0 : warp >> 2, lane = tid & 31, g8 = lane >> 2, q4 = lane & 3;
    // heads vary fastest: neighbours in the grid share the rows of their group
    const uint32_t vheads = a.H * a.tiles, vh = block % vheads, seg = block / vheads % a.segments, b = block / vheads / a.segments;
    const uint32_t head = vh / a.tiles, tile = vh % a.tiles, group = head / (a.H / a.G);
    const int length = a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L;
    const int seg_tokens = (int)a.seg_chunks * SCAN_Q, t_lo = (int)seg * seg_tokens, t_hi = min(length, t_lo + seg_tokens);
    const int pw = min(SCAN_TILE, (int)a.P - (int)tile * SCAN_TILE);   // channels of this tile
    const bool is_last = a.backwards ? seg == 0 : (t_hi == length && (t_lo < length || seg == 0));
    const size_t state_at = (size_t)head * a.P * a.N + (size_t)tile * SCAN_TILE * a.N, states = (size_t)a.H * a.P * a.N;
    const size_t slot = (size_t)b * a.segments + seg;
    if (MODE != MODE_STATE && t_lo >= length && !is_last) {
        // nothing of the sequence lies here; what later kernels read is zero
        if (MODE == MODE_GRAD && a.ends && tid == 0) {
            a.ends[slot * vheads + vh] = 0.f;
            if (a.diag) a.diag[slot * vheads + vh] = 0.f;
        }
        return;
    }
    const int kw = a.k.tiled ? pw : (int)a.N, vw = a.v.tiled ? pw : (int)a.N;
#ifdef FESC_DEBUG_BOUNDS
    if (t_lo < t_hi) {
        const long long n = t_hi - t_lo - 1;
        bool ok = DBG_REGION(scan_row<T>(a.k, b, t_lo, head, group, tile), (n * a.k.st + kw) * sizeof(T)) &&
                  DBG_REGION(scan_row<T>(a.v, b, t_lo, head, group, tile), (n * a.v.st + vw) * sizeof(T)) &&
                  DBG_REGION(a.g + b * a.gb + t_lo * a.gt + head * a.gh, (n * a.gt + 1) * sizeof(float));
        if (MODE) ok = ok && DBG_REGION(scan_row<T>(a.q, b, t_lo, head, group, tile), (n * a.q.st + kw) * sizeof(T));
        if (MODE == MODE_OUT) ok = ok && DBG_REGION((T*)a.out + b * a.ob + t_lo * a.ot + head * a.oh + tile * SCAN_TILE, (n * a.ot + vw) * sizeof(T));
        if (MODE == MODE_GRAD)
            ok = ok && DBG_REGION(scan_row<T>(a.u, b, t_lo, head, group, tile), (n * a.u.st + vw) * sizeof(T)) &&
                 DBG_REGION(a.part + (((size_t)b * vheads + vh) * a.L + t_lo) * DV, (n + 1) * DV * sizeof(float)) &&
                 DBG_REGION(a.dots + ((size_t)b * vheads + vh) * a.L + t_lo, (n + 1) * sizeof(float));
        if (!ok) return;
    }
    if ((MODE && a.init && !DBG_REGION(a.init + (a.segments > 1 ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (a.last && !DBG_REGION(a.last + (MODE == MODE_STATE ? slot : b) * states + state_at, (size_t)pw * a.N * 4)) ||
        (MODE == MODE_GRAD && a.meet && !DBG_REGION(a.meet + (a.segments > 1 && !a.backwards ? slot : b) * states + state_at, (size_t)pw * a.N * 4)))
        return;
#endif
    __nv_bfloat16 *sk = sm + S::k, *sv = sm + S::v, *sq = sm + S::q, *ss = sm + S::s;
    const uint32_t ak = (uint32_t)__cvta_generic_to_shared(sk), av = (uint32_t)__cvta_generic_to_shared(sv);
    const uint32_t aq = (uint32_t)__cvta_generic_to_shared(sq), as = (uint32_t)__cvta_generic_to_shared(ss);
    // the rows and columns that this lane addresses in a 16 x 16 block: left operands and transposed right ones (blocks of 8 x 8 down, then
    // right), right operands (right, then down)
    const int row_l = lane & 15, col_l = lane >> 4 << 3, row_r = (lane & 7) | (lane >> 4 << 3), col_r = lane & 8;
    const int row_t = (lane & 7) | (lane >> 4 << 3), col_t = lane & 8;   // transposed left operands

    // this warp's part of the state: rows (of v) slice * DV/4 + 16 m + g8 (+ 8), columns (of k) half * KH + 8 n + 2 q4 (+ 1)
    float st[MT][KT][4];
    float* sh = reinterpret_cast<float*>(sm);
    // states go between global memory and the registers by way of shared memory: [channel][column] as in global memory
    auto state_word = [&](int m, int n, int e) -> float& {
        const int rv = slice * (DV / 4) + 16 * m + g8 + (e & 2 ? 8 : 0), ck = half * KH + 8 * n + 2 * q4 + (e & 1);
        return MODE == MODE_GRAD ? sh[ck * S::H_STR + rv] : sh[rv * S::H_STR + ck];
    };
    auto fetch_state = [&](const float* src) {      // zeros beyond the tile and its columns, and without a source
        constexpr int NC = MODE == MODE_GRAD ? DV : DK;
#pragma unroll 4
        for (int i = tid; i < SCAN_TILE * NC; i += THREADS) {
            const int p = i / NC, c = i % NC;
            sh[p * S::H_STR + c] = src && p < pw && c < (int)a.N ? src[p * (int)a.N + c] : 0.f;
        }
    };
    const float* init = MODE && a.init ? a.init + (a.segments > 1 ? slot : b) * states + state_at : nullptr;
    if (init) fetch_state(init);
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; m++)
#pragma unroll
        for (int n = 0; n < KT; n++)
#pragma unroll
            for (int e = 0; e < 4; e++) st[m][n][e] = init ? state_word(m, n, e) : 0.f;
    __syncthreads();

    const int chunks = t_hi > t_lo ? (t_hi - t_lo + SCAN_Q - 1) / SCAN_Q : 0;
    float diag = 0.f;
    double through = 0.0;                        // log2 of the decay over the segment (thread 0)
    // warp 0: log decays of two positions a lane, read a chunk ahead.  The decay that applies on the way to a position is its own token's forwards, the
    // token's behind it backwards (none at the end).
    float gv[2] = {};
    auto read_decays = [&](int c) {
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const int pos = c * SCAN_Q + 2 * lane + i, t = a.backwards ? t_hi - pos : t_lo + pos;
            gv[i] = t_lo + pos < t_hi && t < length ? a.g[b * a.gb + t * a.gt + head * a.gh] : 0.f;
        }
    };
    if (warp == 0 && chunks) read_decays(0);
    for (int c = 0; c < chunks; c++) {
        // token of position i of the chunk: t0 + dir * i
        const int valid = min(SCAN_Q, t_hi - t_lo - c * SCAN_Q), dir = a.backwards ? -1 : 1, t0 = a.backwards ? t_hi - 1 - c * SCAN_Q : t_lo + c * SCAN_Q;
        load_tile<T, DK, THREADS>(sk, scan_row<T>(a.k, b, t0, head, group, tile), dir * a.k.st, valid, kw, a.k.align);
        load_tile<T, DV, THREADS>(sv, scan_row<T>(a.v, b, t0, head, group, tile), dir * a.v.st, valid, vw, a.v.align);
        if (MODE) load_tile<T, DK, THREADS>(sq, scan_row<T>(a.q, b, t0, head, group, tile), dir * a.q.st, valid, kw, a.q.align);
        if (warp == 0) {
            double sum[2];
#pragma unroll
            for (int i = 0; i < 2; i++) sum[i] = (double)(gv[i] < SCAN_DROP ? SCAN_DROP : gv[i]) * 1.4426950408889634 + (i ? sum[0] : 0.0);
            if (c + 1 < chunks) read_decays(c + 1);
            double run = sum[1];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double w = __shfl_up_sync(~0u, run, o);
                if (lane >= o) run += w;
            }
            const double before = run - sum[1], total = __shfl_sync(~0u, run, 31);
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const double v = before + sum[i];
                const float hi = (float)v;
                cum[2 * lane + i] = make_float2(hi, (float)(v - hi));
                grow[2 * lane + i] = exp2f(hi) * exp2f((float)(v - hi));
                const double f = total - v;
                fade[2 * lane + i] = exp2f((float)f);
            }
            if (lane == 31) grow[SCAN_Q - 1] = exp2_near(total);
            through += total;
        }
        cp_async_wait();
        __syncthreads();

        if (MODE) {
            // scores of 16 rows i per warp, columns j <= i: S_ij = G_ij (q_i . k_j), cut into planes
            const int i0 = 16 * slice + g8, ks = (kw + 15) / 16;
            const float2 ci[2] = {cum[i0], cum[i0 + 8]};
#pragma unroll 1
            for (int j = half; j <= (int)slice; j += HALVES) {
                // products that depend on one another wait: each plane of k has sums of its own, with one plane every other step
                float ds[NI == 1 ? 2 : NI][2][4] = {};
#pragma unroll 2
                for (int kk = 0; kk < ks; kk++) {
                    uint32_t qf[NI][4], kf[NI][4];
#pragma unroll
                    for (int p = 0; p < NI; p++) {
                        ldsm4(qf[p], aq + (p * SCAN_Q * S::K_STR + (16 * slice + row_l) * S::K_STR + 16 * kk + col_l) * 2);
                        ldsm4(kf[p], ak + (p * SCAN_Q * S::K_STR + (16 * j + row_r) * S::K_STR + 16 * kk + col_r) * 2);
                    }
                    if constexpr (NI == 1) {
                        if (kk & 1) mma(ds[1][0], qf[0], kf[0][0], kf[0][1]), mma(ds[1][1], qf[0], kf[0][2], kf[0][3]);
                        else mma(ds[0][0], qf[0], kf[0][0], kf[0][1]), mma(ds[0][1], qf[0], kf[0][2], kf[0][3]);
                    } else {
#pragma unroll
                        for (int pq = 0; pq < NI; pq++)
#pragma unroll
                            for (int pk = 0; pk < NI; pk++)
                                if (pk + pq < 3) mma(ds[pk][0], qf[pq], kf[pk][0], kf[pk][1]), mma(ds[pk][1], qf[pq], kf[pk][2], kf[pk][3]);
                    }
                }
                float d[2][4];
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) d[n][e] = NI == 3 ? ds[0][n][e] + (ds[1][n][e] + ds[NI == 3 ? 2 : 1][n][e]) : ds[0][n][e] + ds[1][n][e];
#pragma unroll
                for (int n = 0; n < 2; n++) {
                    const int jc = 16 * j + 8 * n + 2 * q4;
                    const float2 c0 = cum[jc], c1 = cum[jc + 1];
#pragma unroll
                    for (int h = 0; h < 2; h++) {
                        const int i = i0 + 8 * h;
                        if (MODE == MODE_GRAD) diag += (i == jc ? d[n][2 * h] : 0.f) + (i == jc + 1 ? d[n][2 * h + 1] : 0.f);
                        const float e0 = exp2f((ci[h].x - c0.x) + (ci[h].y - c0.y)), e1 = exp2f((ci[h].x - c1.x) + (ci[h].y - c1.y));
                        uint32_t pl[NO];
                        split<NO>(jc <= i ? d[n][2 * h] * e0 : 0.f, jc + 1 <= i ? d[n][2 * h + 1] * e1 : 0.f, pl);
#pragma unroll
                        for (int p = 0; p < NO; p++) *reinterpret_cast<uint32_t*>(ss + p * SCAN_Q * S::S_STR + i * S::S_STR + jc) = pl[p];
                    }
                }
            }
            __syncthreads();
        }

        // out^T = state q^T, columns times the decay since the chunk's start, + v^T S^T
        float acc[MODE ? MT : 1][MODE ? 8 : 1][4];
        if (MODE) {
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int n = 0; n < 8; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) acc[m][n][e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KH / 16; kk++) {
                if ((int)half * KH + 16 * kk >= kw) break;         // columns that do not exist
                uint32_t sf[MT][NO][4];
#pragma unroll
                for (int m = 0; m < MT; m++)
#pragma unroll
                    for (int r = 0; r < 4; r++) {
                        uint32_t pl[NO];
                        const float(&x)[4] = st[m][2 * kk + (r >> 1)];
                        split<NO>(x[2 * (r & 1)], x[2 * (r & 1) + 1], pl);
#pragma unroll
                        for (int p = 0; p < NO; p++) sf[m][p][r] = pl[p];
                    }
#pragma unroll
                for (int pq = 0; pq < NI; pq++) {
                    uint32_t qf[4][4];
#pragma unroll
                    for (int n = 0; n < 4; n++)
                        ldsm4(qf[n], aq + (pq * SCAN_Q * S::K_STR + (16 * n + row_r) * S::K_STR + half * KH + 16 * kk + col_r) * 2);
#pragma unroll
                    for (int p = 0; p < NO; p++)
                        if (p + pq < NO || NI == 1)
#pragma unroll
                            for (int n = 0; n < 4; n++)
#pragma unroll
                                for (int m = 0; m < MT; m++) mma(acc[m][2 * n], sf[m][p], qf[n][0], qf[n][1]), mma(acc[m][2 * n + 1], sf[m][p], qf[n][2], qf[n][3]);
                }
            }
#pragma unroll
            for (int n = 0; n < 8; n++) {
                const float2 e = *reinterpret_cast<const float2*>(grow + 8 * n + 2 * q4);
#pragma unroll
                for (int m = 0; m < MT; m++)
#pragma unroll
                    for (int i = 0; i < 4; i++) acc[m][n][i] = decayed(i & 1 ? e.y : e.x, acc[m][n][i]);
            }
        }
        // state <- G_last state + (fade v)^T k
        {
            const float keep = grow[SCAN_Q - 1];
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int n = 0; n < KT; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) st[m][n][e] = decayed(keep, st[m][n][e]);
        }
#pragma unroll 1
        for (int kk = 0; kk < SCAN_Q / 16; kk++) {
            uint32_t vf[MT][NI][4], wf[MT][NS][4];
#pragma unroll
            for (int m = 0; m < MT; m++) {
#pragma unroll
                for (int p = 0; p < NI; p++)
                    ldsm4t(vf[m][p], av + (p * SCAN_Q * S::V_STR + (16 * kk + row_t) * S::V_STR + slice * (DV / 4) + 16 * m + col_t) * 2);
                // rows of the block are positions 16 kk + 2 q4 (+ 1), + 8 for the right half
#pragma unroll
                for (int r = 0; r < 4; r++) {
                    float x = 0.f, y = 0.f;
#pragma unroll
                    for (int p = NI - 1; p >= 0; p--) x += __uint_as_float(vf[m][p][r] << 16), y += __uint_as_float(vf[m][p][r] & 0xFFFF0000u);
                    const float2 f = *reinterpret_cast<const float2*>(fade + 16 * kk + 2 * q4 + (r & 2 ? 8 : 0));
                    uint32_t pl[NS];
                    split<NS>(x * f.x, y * f.y, pl);
#pragma unroll
                    for (int p = 0; p < NS; p++) wf[m][p][r] = pl[p];
                }
            }
            if (MODE && (HALVES == 1 || (kk & 1) == (int)half)) {
#pragma unroll
                for (int p = 0; p < NO; p++) {
                    uint32_t sf[4][4];
#pragma unroll
                    for (int n = 0; n < 4; n++)
                        if (n >= kk) ldsm4(sf[n], as + (p * SCAN_Q * S::S_STR + (16 * n + row_r) * S::S_STR + 16 * kk + col_r) * 2);      // positions i before all of these j have none
#pragma unroll
                    for (int pv = 0; pv < NI; pv++)
                        if (p + pv < NO || NI == 1)
#pragma unroll
                            for (int n = 0; n < 4; n++)
                                if (n >= kk)
#pragma unroll
                                    for (int m = 0; m < MT; m++) mma(acc[m][2 * n], vf[m][pv], sf[n][0], sf[n][1]), mma(acc[m][2 * n + 1], vf[m][pv], sf[n][2], sf[n][3]);
                }
            }
            // sums of their own that are then added to the state (see above), two pieces of 16 columns under way
#pragma unroll
            for (int n0 = 0; n0 < KH / 16; n0 += 2) {
                if ((int)half * KH + 16 * n0 >= kw) continue;
                float d[2][MT][2][4] = {};
#pragma unroll
                for (int pk = 0; pk < NI; pk++) {
                    uint32_t kf[2][4];
#pragma unroll
                    for (int n = 0; n < 2; n++)
                        ldsm4t(kf[n], ak + (pk * SCAN_Q * S::K_STR + (16 * kk + row_l) * S::K_STR + half * KH + 16 * (n0 + n) + col_l) * 2);
#pragma unroll
                    for (int p = 0; p < NS; p++)
                        if (p + pk < NS)
#pragma unroll
                            for (int n = 0; n < 2; n++)
#pragma unroll
                                for (int m = 0; m < MT; m++) mma(d[n][m][0], wf[m][p], kf[n][0], kf[n][1]), mma(d[n][m][1], wf[m][p], kf[n][2], kf[n][3]);
                }
#pragma unroll
                for (int n = 0; n < 2; n++)
#pragma unroll
                    for (int m = 0; m < MT; m++)
#pragma unroll
                        for (int e = 0; e < 4; e++) st[m][2 * (n0 + n)][e] += d[n][m][0][e], st[m][2 * (n0 + n) + 1][e] += d[n][m][1][e];
            }
        }

        if (MODE) {
            // out through shared memory (over q and the scores) for whole rows
            __syncthreads();
            float* so = reinterpret_cast<float*>(sq);
#pragma unroll
            for (int h = 0; h < HALVES; h++) {
                if ((int)half == h)
#pragma unroll
                    for (int m = 0; m < MT; m++)
#pragma unroll
                        for (int n = 0; n < 8; n++)
#pragma unroll
                            for (int e = 0; e < 4; e++) {
                                float& o = so[(8 * n + 2 * q4 + (e & 1)) * S::O_STR + slice * (DV / 4) + 16 * m + g8 + (e & 2 ? 8 : 0)];
                                o = h ? o + acc[m][n][e] : acc[m][n][e];
                            }
                __syncthreads();
            }
            if (MODE == MODE_OUT) {
                T* out = (T*)a.out + b * a.ob + head * a.oh + tile * SCAN_TILE;
                const float skip = a.skip ? a.skip[head] : 0.f;
#pragma unroll 2
                for (int i = tid; i < SCAN_Q * DV / 8; i += THREADS) {
                    const int r = i / (DV / 8), cc = i % (DV / 8) * 8;
                    float v[8];
#pragma unroll
                    for (int e = 0; e < 8; e++) v[e] = so[r * S::O_STR + cc + e];
                    if (a.skip) {
#pragma unroll
                        for (int p = NI - 1; p >= 0; p--)
#pragma unroll
                            for (int e = 0; e < 8; e++) v[e] += skip * __bfloat162float(sv[p * SCAN_Q * S::V_STR + r * S::V_STR + cc + e]);
                    }
                    if (r < valid) clear_store8(out + (long long)(t0 + dir * r) * a.ot + cc, vw - cc, a.out_wide, v);
                }
            } else {
                constexpr int E = DV / 32;
                float* part = a.part + ((size_t)b * vheads + vh) * a.L * DV;
                float* dots = a.dots + ((size_t)b * vheads + vh) * a.L;
                for (int r = warp; r < valid; r += THREADS / 32) {
                    const int t = t0 + dir * r;
                    const T* u = scan_row<T>(a.u, b, t, head, group, tile) + lane * E;
                    float v[E], dot = 0.f;
#pragma unroll
                    for (int e = 0; e < E; e++) {
                        v[e] = so[r * S::O_STR + lane * E + e];
                        if ((int)lane * E + e < vw) dot += v[e] * ClearType<T>::to(u[e]);
                    }
                    if constexpr (E == 4) *reinterpret_cast<float4*>(part + (size_t)t * DV + lane * E) = make_float4(v[0], v[1], v[2], v[3]);
                    else *reinterpret_cast<float2*>(part + (size_t)t * DV + lane * E) = make_float2(v[0], v[1]);
#pragma unroll
                    for (int o = 16; o; o >>= 1) dot += __shfl_xor_sync(~0u, dot, o);
                    if (lane == 0) dots[t] = dot;
                }
            }
        }
        __syncthreads();
    }

    // the state behind the sweep (shared memory is free: every chunk ends with a barrier)
    if (a.last && (MODE == MODE_STATE || is_last)) {
        float* last = a.last + (MODE == MODE_STATE ? slot : b) * states + state_at;
        // backwards the state belongs to the first token: the gradient of the state before it is one decay further
        const float f = MODE && a.backwards && length > 0 ? expf(a.g[b * a.gb + head * a.gh]) : 1.f;
#pragma unroll
        for (int m = 0; m < MT; m++)
#pragma unroll
            for (int n = 0; n < KT; n++)
#pragma unroll
                for (int e = 0; e < 4; e++) state_word(m, n, e) = decayed(f, st[m][n][e]);
        __syncthreads();
#pragma unroll 4
        for (int i = tid; i < pw * (int)a.N; i += THREADS) last[i] = sh[i / a.N * S::H_STR + i % a.N];
        __syncthreads();
    }
    if (MODE == MODE_STATE && tid == 0 && tile == 0) a.decay[slot * a.H + head] = exp2_near(through);
    if (MODE == MODE_GRAD && a.ends) {
        // <state, gradient of the state> at the segment's end, one decay on from what the sweep backwards starts this segment with
        float sum = 0.f;
        if (a.meet && (!a.backwards || seg == 0)) {
            fetch_state(a.meet + (a.segments > 1 && !a.backwards ? slot : b) * states + state_at);
            __syncthreads();
#pragma unroll
            for (int m = 0; m < MT; m++)
#pragma unroll
                for (int n = 0; n < KT; n++)
#pragma unroll
                    for (int e = 0; e < 4; e++) sum += st[m][n][e] * state_word(m, n, e);
            const int next = a.backwards ? 0 : t_hi;
            if (next < length) sum = decayed(expf(a.g[b * a.gb + next * a.gt + head * a.gh]), sum);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o), diag += __shfl_xor_sync(~0u, diag, o);
        if (lane == 0) words[0][warp] = sum, words[1][warp] = diag;
        __syncthreads();
        if (tid == 0) {
            float s0 = 0.f, s1 = 0.f;
            for (int w = 0; w < THREADS / 32; w++) s0 += words[0][w], s1 += words[1][w];
            a.ends[slot * vheads + vh] = s0;
            if (a.diag) a.diag[slot * vheads + vh] = s1;
        }
    }
}

// one grid for the sweeps of a call: those of the backward pass are independent
#define SCAN_CTAS(T, NP) (ClearType<T>::planes == 1 ? (NP == 64 ? 3 : 2) : ClearType<T>::planes == 3 && NP == 128 ? 1 : 2)      // of an SM
template <class T, int NP>
__global__ void __launch_bounds__(ScanWarps<T>::threads, SCAN_CTAS(T, NP)) k_clear_scan_state(const __grid_constant__ ScanSet s) {
    pdl_begin();
    sweep<T, NP, 64, MODE_STATE>(s.a[blockIdx.x % s.count], blockIdx.x / s.count);
}
template <class T, int NP>
__global__ void __launch_bounds__(ScanWarps<T>::threads, SCAN_CTAS(T, NP)) k_clear_scan(const __grid_constant__ ScanSet s) {
    pdl_begin();
    sweep<T, NP, 64, MODE_OUT>(s.a[0], blockIdx.x);
}
template <class T, int NP>
__global__ void __launch_bounds__(ScanWarps<T>::threads, NP == 128 ? 1 : SCAN_CTAS(T, NP)) k_clear_scan_backward(const __grid_constant__ ScanSet s) {
    pdl_begin();
    const uint32_t which = blockIdx.x % 3, block = blockIdx.x / 3;
    if (which < 2) sweep<T, 64, NP, MODE_GRAD>(s.a[which], block);
    else sweep<T, NP, 64, MODE_OUT>(s.a[2], block);
}

// one type's kernels, by mode and by whether states have more than 64 columns
template <class T>
cudaError_t scan_launch(const ScanSet& s, int mode, cudaStream_t st) {
    auto go = [&](auto kernel, size_t smem) {
        cudaError_t e = cudaFuncSetAttribute((const void*)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        const ScanArgs& a = s.a[0];
        return e != cudaSuccess ? e : launch(kernel, dim3(s.count * a.b * a.segments * a.H * a.tiles), dim3(ScanWarps<T>::threads), smem, st, s);
    };
    auto pick = [&](auto np) {
        constexpr int NP = decltype(np)::value;
        constexpr size_t out = ScanShared<T, NP, 64, MODE_OUT>::bytes, grad = ScanShared<T, 64, NP, MODE_GRAD>::bytes;
        return mode == MODE_STATE ? go(k_clear_scan_state<T, NP>, ScanShared<T, NP, 64, MODE_STATE>::bytes)
             : mode == MODE_OUT   ? go(k_clear_scan<T, NP>, out)
                                  : go(k_clear_scan_backward<T, NP>, out > grad ? out : grad);
    };
    return s.a[0].N > 64 ? pick(std::integral_constant<int, 128>()) : pick(std::integral_constant<int, 64>());
}
extern template cudaError_t scan_launch<__nv_bfloat16>(const ScanSet&, int, cudaStream_t);
extern template cudaError_t scan_launch<__half>(const ScanSet&, int, cudaStream_t);
extern template cudaError_t scan_launch<float>(const ScanSet&, int, cudaStream_t);
// The same on tcgen05: bfloat16, operands with 16-byte rows (clear_scan_tc.cu; states of 8 columns take as long as states of 64 there, and still less than
// on mma.sync).  Operands whose strides or widths are not of 16 bytes are copied into such rows first.  Those whose strides are but whose address is not
// (the workspace is sized without addresses) take mma.sync, element by element: 2048 tokens of 24 heads 221 us, where 28 are possible.
// part is [b][head tile][segment][chunk of 128][16384] in an order of its own there, and dots is left to the kernel that sums it up over heads.
cudaError_t scan_tc_launch(const ScanSet& s, int mode, cudaStream_t st);
struct TcSums {
    const float *part_b, *part_c;
    ScanOperand uB, uC;
    __nv_bfloat16 *dB, *dC;
    float *row, *col;
    const int* lengths;
    long long Bb, Bt, Bg, Cb, Ct, Cg;
    uint32_t L, H, G, N, tiles, segments, seg_chunks;
    uint32_t wide;              // rows of dB and dC allow 16-byte accesses
};
cudaError_t scan_tc_sums(const TcSums& a, uint32_t batch, cudaStream_t st);
struct TcPack {
    struct {
        const void* src;
        void* dst;               // [b][L][heads][width in pieces of 8]
        long long sb, st, sh;
        uint32_t heads, width;
    } o[4];
    const int* lengths;
    uint32_t L, count;
};
cudaError_t scan_tc_pack(const TcPack& a, uint32_t batch, cudaStream_t st);
