// Cleartext gated linear recurrence, the operator that fesc_scan_contract evaluates on ciphertexts (Sec. 5.4, Eqs. fesc_recurrence /
// fesc_contract):  h_t = exp(g_t) h_{t-1} + x_t B_t^T,  y_t = h_t C_t + D x_t; its backward pass, and one token of it.
// clear_scan.cuh holds the sweep; here are the kernels around it and the entry points.
//
// The gradient of the log decays comes from what the sweeps give: with row_t = C_t . dC_t and col_t = B_t . dB_t of one head,
//   dg_t = <h_t, dh_t>' summed back from the segment's end:  R_t = R_{t+1} + row_t - col_t,  R behind a segment = <h, dh> there,
// so no state has to be kept per token.  Rounding adds up over a segment only, whose ends are computed from the states themselves.
#define FESC_DBG_FILE 20   // file id in the sites a debug build reports
#include "clear_scan.cuh"

static thread_local std::string clear_error;
int clear_fail(int code, const char* what) {
    try {
        clear_error = what;
    } catch (...) {      // no memory for the text: the code stands
    }
    return code;
}
extern "C" const char* fesc_clear_last_error(void) { return clear_error.c_str(); }

// Chains the segments: slot s gets the state before segment s (in the sweep's direction) and what the segment adds goes into the chain.  blockIdx.z:
// forwards, backwards.
struct Chain {
    float* states;
    const float *decay, *init;
};
__global__ void __launch_bounds__(256) k_clear_combine(const Chain forwards, const Chain back, uint32_t segments, uint32_t per_head, size_t per_b) {
    pdl_begin();
    const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 4;
    const uint32_t b = blockIdx.y;
    const bool backwards = blockIdx.z;
    float* const states = backwards ? back.states : forwards.states;
    const float *const decay = backwards ? back.decay : forwards.decay, *const init = backwards ? back.init : forwards.init;
    if (i >= per_b) return;
    float* s = states + (size_t)b * segments * per_b + i;
    const uint32_t H = (uint32_t)(per_b / per_head), n = (uint32_t)(per_b - i < 4 ? per_b - i : 4);
    if (!DBG_REGION(decay + (size_t)b * segments * H, (size_t)segments * H * sizeof(float)) ||
        !DBG_REGION(s, ((segments - 1) * per_b + n) * sizeof(float)) || (init && !DBG_REGION(init + b * per_b + i, n * sizeof(float))))
        return;
    const bool wide = per_b % 4 == 0 && per_head % 4 == 0 && ((size_t)init & 15) == 0;
    const uint32_t h0 = (uint32_t)i / per_head;      // H * P * N is below 2^32 (checked)
    float run[4] = {};
    for (uint32_t e = 0; e < n && init; e++) run[e] = init[b * per_b + i + e];
    if (wide) {
        // the loads of eight segments before the first of their stores: one trip to memory for all
        for (uint32_t c = 0; c < segments; c += 8) {
            float4 add[8];
            float f[8];
#pragma unroll
            for (uint32_t k = 0; k < 8; k++)
                if (c + k < segments) {
                    const uint32_t at = backwards ? segments - 1 - c - k : c + k;
                    add[k] = *reinterpret_cast<const float4*>(s + (size_t)at * per_b), f[k] = decay[((size_t)b * segments + at) * H + h0];
                }
#pragma unroll
            for (uint32_t k = 0; k < 8; k++)
                if (c + k < segments) {
                    const uint32_t at = backwards ? segments - 1 - c - k : c + k;
                    *reinterpret_cast<float4*>(s + (size_t)at * per_b) = make_float4(run[0], run[1], run[2], run[3]);
                    run[0] = decayed(f[k], run[0]) + add[k].x, run[1] = decayed(f[k], run[1]) + add[k].y, run[2] = decayed(f[k], run[2]) + add[k].z,
                    run[3] = decayed(f[k], run[3]) + add[k].w;
                }
        }
        return;
    }
    for (uint32_t c = 0; c < segments; c++) {
        const uint32_t at = backwards ? segments - 1 - c : c;
        float* p = s + (size_t)at * per_b;
        for (uint32_t e = 0; e < n; e++) {
            const float add = p[e];
            p[e] = run[e];
            run[e] = decayed(decay[((size_t)b * segments + at) * H + ((uint32_t)i + e) / per_head], run[e]) + add;
        }
    }
}

struct FinishArgs {
    const float *part_b, *part_c, *row, *col, *ends, *starts, *diag, *g;
    void *dB, *dC;
    float *dg, *dskip;
    const int* lengths;
    long long Bb, Bt, Bg, Cb, Ct, Cg, gb, gt, gh, ib, it, ih;
    uint32_t b, L, H, G, N, tiles, segments, seg_chunks;
    uint32_t log_quads;                                  // columns of part_b and part_c: 4 << log_quads
    uint32_t sum_each, sum_blocks, dg_blocks;            // blocks: of a sequence's group in one sum, of both sums, of dg
};
// What is left of the backward pass, by block: sums of dB and dC over the heads of a group; the gradient of the log decays, a block per
// sequence, head and segment; that of the skip.
template <class T, int THREADS>
__global__ void __launch_bounds__(THREADS) k_clear_scan_finish(const FinishArgs a) {
    constexpr uint32_t WARPS = THREADS / 32;
    __shared__ double words[2][WARPS];
    pdl_begin();
    const uint32_t vheads = a.H * a.tiles, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto tokens = [&](uint32_t b) { return a.lengths ? min(max(a.lengths[b], 0), (int)a.L) : (int)a.L; };
    if (blockIdx.x < a.sum_blocks) {
        const uint32_t piece = blockIdx.x / a.sum_each, c_sum = piece & 1, grp = (piece >> 1) % a.G, b = (piece >> 1) / a.G;
        const size_t i = (size_t)(blockIdx.x % a.sum_each) * 256 + tid, t = i >> a.log_quads;
        const uint32_t n = 4 * ((uint32_t)i & ((1u << a.log_quads) - 1)), per = vheads / a.G, NP = 4u << a.log_quads;
        if (t >= (size_t)tokens(b) || n >= a.N) return;
        const size_t step = (size_t)a.L * NP;
        const float* src = (c_sum ? a.part_c : a.part_b) + (((size_t)b * vheads + grp * per) * a.L + t) * NP + n;
        T* dst = c_sum ? (T*)a.dC + b * a.Cb + (long long)t * a.Ct + grp * a.Cg + n : (T*)a.dB + b * a.Bb + (long long)t * a.Bt + grp * a.Bg + n;
        if (!DBG_REGION(src, ((per - 1) * step + 4) * sizeof(float)) || !DBG_REGION(dst, min(4u, a.N - n) * sizeof(T))) return;
        float s[4] = {};
#pragma unroll 8
        for (uint32_t h = 0; h < per; h++) {
            const float4 v = *reinterpret_cast<const float4*>(src + h * step);
            s[0] += v.x, s[1] += v.y, s[2] += v.z, s[3] += v.w;
        }
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (n + e < a.N) dst[e] = ClearType<T>::from(s[e]);
        return;
    }
    const uint32_t blk = blockIdx.x - a.sum_blocks;
    if (blk < a.dg_blocks) {
        // R_t = R_{t+1} + row_t - col_t from the segment's end, where R is known; it is known at the segment's beginning, too, and what the sum
        // misses it by is spread over the tokens: the products' rounding leans to one side and adds up with the tokens (1024 of them took the error
        // from 1e-6 to 2e-6).  A token a thread; the next ones' words are read while these are summed
        const uint32_t head = blk % a.H, seg = blk / a.H % a.segments, b = blk / a.H / a.segments;
        const int length = tokens(b), lo = (int)(seg * a.seg_chunks) * SCAN_Q, hi = min(length, lo + (int)a.seg_chunks * SCAN_Q);
        if (lo >= hi) return;
        const float* row = a.row + ((size_t)b * a.H + head) * a.tiles * a.L;
        const float* col = a.col + ((size_t)b * a.H + head) * a.tiles * a.L;
        float* dg = a.dg + b * a.gb + head * a.gh;
        const float* g = a.g + b * a.ib + head * a.ih;
        if (!DBG_REGION(dg + lo * a.gt, ((long long)(hi - 1 - lo) * a.gt + 1) * sizeof(float))) return;
        double run = 0.0;
        for (uint32_t s = 0; s < a.tiles; s++) run += a.ends[((size_t)b * a.segments + seg) * vheads + head * a.tiles + s];
        double low = 0.0, total = 0.0, slope = 0.0;
        const float* begin = seg ? a.ends + ((size_t)b * a.segments + seg - 1) * vheads : a.starts ? a.starts + (size_t)b * a.segments * vheads : nullptr;
        for (uint32_t s = 0; begin && s < a.tiles; s++) low += begin[head * a.tiles + s];
        bool dropped = false;
        for (int t = hi - 1 - (int)tid; t >= lo; t -= THREADS) {
            for (uint32_t s = 0; s < a.tiles; s++) total += (double)row[(size_t)s * a.L + t] - (double)col[(size_t)s * a.L + t];
            dropped = dropped || g[t * a.it] < SCAN_DROP;
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(~0u, total, o);
        if (lane == 0) words[0][warp] = total;
        if (!__syncthreads_or(dropped)) {        // a dropped state is a beginning of its own
            total = 0.0;
            for (uint32_t w = 0; w < WARPS; w++) total += words[0][w];
            slope = (run + total - low) / (double)(hi - lo);
            if (!(fabs(slope) < 1e300)) slope = 0.0;      // an infinity or NaN stays with the tokens that it reaches
        }
        __syncthreads();
        double next = 0.0;
        bool next_drop = false;
        auto read = [&](int t) {
            next = 0.0, next_drop = false;
            if (t < lo) return;
            for (uint32_t s = 0; s < a.tiles; s++) next += (double)row[(size_t)s * a.L + t] - (double)col[(size_t)s * a.L + t];
            next_drop = g[t * a.it] < SCAN_DROP;
        };
        read(hi - 1 - (int)tid);
        uint32_t turn = 0;
        for (int top = hi - 1; top >= lo; top -= THREADS, turn ^= 1) {
            const int t = top - (int)tid;
            double v = next;
            const bool drop = next_drop;
            read(t - THREADS);
            // a dropped state has the gradient zero, from which the sum goes on: what a token adds up goes back to the nearest drop at or behind it
            if (__syncthreads_or(drop)) {
                // seldom: token by token
                __shared__ double all[THREADS];
                __shared__ bool drops[THREADS];
                all[tid] = v, drops[tid] = drop;
                __syncthreads();
                if (tid == 0)
                    for (int k = 0; k < THREADS && top - k >= lo; k++) {
                        run = drops[k] ? 0.0 : run + all[k];
                        dg[(long long)(top - k) * a.gt] = (float)run;
                    }
                if (tid == 0) words[0][0] = run;
                __syncthreads();
                run = words[0][0];
                __syncthreads();
                continue;
            }
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double u = __shfl_up_sync(~0u, v, o);
                if ((int)lane >= o) v += u;
            }
            if (lane == 31) words[turn][warp] = v;
            __syncthreads();
            double sums = lane < WARPS ? words[turn][lane] : 0.0;
#pragma unroll
            for (int o = 1; o < (int)WARPS; o <<= 1) {
                const double u = __shfl_up_sync(~0u, sums, o);
                if ((int)lane >= o) sums += u;
            }
            const double before = __shfl_sync(~0u, sums, warp ? warp - 1 : 0);
            if (t >= lo) dg[t * a.gt] = (float)(run + (warp ? before : 0.0) + v - slope * (double)(hi - t));
            run += __shfl_sync(~0u, sums, WARPS - 1);
        }
        return;
    }
    // the skip: a warp per head
    const uint32_t head = (blk - a.dg_blocks) * WARPS + warp;
    if (!a.dskip || head >= a.H) return;
    double s = 0.0;
    const size_t all = (size_t)a.b * a.segments * a.tiles;
    for (size_t i = lane; i < all; i += 32) s += a.diag[i / a.tiles * vheads + head * a.tiles + i % a.tiles];
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    if (lane == 0 && DBG_REGION(a.dskip + head, sizeof(float))) a.dskip[head] = (float)s;
}

// One token.  A warp takes ROWS rows of the state, a lane up to four of its columns; read and written once, past what the caches hold on to: bound
// by that (192 sequences of 24 heads: 303 MB in 51 us; with four rows on their way 60).
struct StepArgs {
    const void *x, *B, *C;
    const float *g, *skip, *state;
    float* out;
    void* y;
    long long xb, xh, Bb, Bg, Cb, Cg, gb, gh, yb, yh;
    uint32_t H, P, N, G;
};
template <class T, bool WIDE, int ROWS>
__global__ void __launch_bounds__(256) k_clear_scan_step(const StepArgs a) {
    pdl_begin();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, head = blockIdx.x % a.H, b = blockIdx.x / a.H, group = head / (a.H / a.G);
    const T* B = (const T*)a.B + b * a.Bb + group * a.Bg;
    const T* C = (const T*)a.C + b * a.Cb + group * a.Cg;
    const T* x = (const T*)a.x + b * a.xb + head * a.xh;
    T* y = (T*)a.y + b * a.yb + head * a.yh;
    const size_t at = ((size_t)b * a.H + head) * a.P * a.N;
    if (!DBG_REGION(B, a.N * sizeof(T)) || !DBG_REGION(C, a.N * sizeof(T)) || !DBG_REGION(x, a.P * sizeof(T)) || !DBG_REGION(y, a.P * sizeof(T)) ||
        !DBG_REGION(a.state + at, (size_t)a.P * a.N * 4) || !DBG_REGION(a.out + at, (size_t)a.P * a.N * 4) || !DBG_REGION(a.g + b * a.gb + head * a.gh, 4))
        return;
    const float keep = expf(a.g[b * a.gb + head * a.gh]), skip = a.skip ? a.skip[head] : 0.f;
    float vB[4], vC[4];
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const uint32_t n = WIDE ? lane * 4 + e : lane + 32 * e;
        vB[e] = n < a.N ? ClearType<T>::to(B[n]) : 0.f, vC[e] = n < a.N ? ClearType<T>::to(C[n]) : 0.f;
    }
    const uint32_t first = (blockIdx.y * 8 + warp) * ROWS;
    float h[ROWS][4], xv[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; r++) {       // all of a warp's rows on their way before the first is used
        const uint32_t p = first + r;
        const float* s = a.state + at + (size_t)p * a.N;
        const bool live = p < a.P;
        xv[r] = live ? ClearType<T>::to(x[p]) : 0.f;
        if (WIDE) {
            const float4 v = live && lane * 4 < a.N ? __ldcs(reinterpret_cast<const float4*>(s + lane * 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
            h[r][0] = v.x, h[r][1] = v.y, h[r][2] = v.z, h[r][3] = v.w;
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++) h[r][e] = live && lane + 32 * e < a.N ? s[lane + 32 * e] : 0.f;
        }
    }
#pragma unroll
    for (int r = 0; r < ROWS; r++) {
        const uint32_t p = first + r;
        if (p >= a.P) break;
        float* o = a.out + at + (size_t)p * a.N;
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            h[r][e] = decayed(keep, h[r][e]) + xv[r] * vB[e];
            sum += h[r][e] * vC[e];        // B and C are zero beyond the columns
        }
        if (WIDE) {
            if (lane * 4 < a.N) __stcs(reinterpret_cast<float4*>(o + lane * 4), make_float4(h[r][0], h[r][1], h[r][2], h[r][3]));
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (lane + 32 * e < a.N) o[lane + 32 * e] = h[r][e];
        }
#pragma unroll
        for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(~0u, sum, w);
        if (lane == 0) y[p] = ClearType<T>::from(sum + skip * xv[r]);
    }
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------
struct ScanShape {
    uint32_t tiles, vheads, segments, seg_chunks, np;
    bool tc;                   // the sweeps run on tcgen05 (if the operands' addresses allow)
    bool pack;                 // their operands are copied into rows of 16 bytes first
    size_t x_pack, b_pack;     // floats of a copy of x or dy, and of B or C
    size_t states, state_floats, decay_floats, part_floats, dot_floats, end_floats;
};

// The shape of a call's sweeps, the backward pass's three at once.  Segments: what takes least time by a model in pieces of 128 tokens.  A CTA takes
// as long as its pieces and START of them besides (pieces are slower on mma.sync); a grid as many rounds of that as its CTAs fill the places where they run; with more than
// one segment a pass over the keys and values, at a third (mma.sync: half) of the time a piece, and the chaining come first.  (2048 tokens of 24 heads on tcgen05: forwards 6
// segments, 30 us, with one 65; backwards 2, 95 us, with 6 128.)
static ScanShape scan_shape(const fesc_clear_scan_desc* d, bool backward) {
    ScanShape s;
    s.tc = d->type == FESC_BF16;
    auto odd = [](const int64_t(&st)[3]) { return (st[0] | st[1] | st[2]) % 8 != 0; };
    s.pack = s.tc && (d->N % 8 || d->P % 8 || odd(d->x) || odd(d->B) || odd(d->C) || (backward && odd(d->y)));
    s.tiles = (d->P + SCAN_TILE - 1) / SCAN_TILE, s.vheads = d->H * s.tiles, s.np = s.tc || d->N > 64 ? 128 : 64;
    const uint64_t pieces = ((uint64_t)d->L + 127) / 128, ctas = (uint64_t)d->batch * s.vheads, sweeps = backward ? 3 : 1;
    const double START = s.tc ? 2.0 : 0.5, CHAIN = s.tc ? 1.5 : 0.5, STATE = s.tc ? 0.35 : 0.5;
    // CTAs on an SM, by registers and shared memory: of the state pass, of the sweeps (as their launch bounds have it)
    const bool broad = d->N > 64;
    const uint64_t of_state = 148 * (s.tc || (broad && d->type == FESC_F32) ? 1 : 2), places = broad && backward ? 148 : of_state;
    uint64_t each = pieces ? pieces : 1, last = 0;
    double least = 1e300;
    for (uint64_t want = 1; want <= pieces && want <= 1024; want++) {
        const uint64_t of = (pieces + want - 1) / want, segments = (pieces + of - 1) / of;
        if (segments == last) continue;
        last = segments;
        auto rounds = [&](uint64_t n, uint64_t at_once) { return (double)((n * ctas * segments + at_once - 1) / at_once); };
        double time = rounds(sweeps, places) * (START + of);
        if (segments > 1) time += rounds(backward ? 2 : 1, of_state) * (START + STATE * of) + CHAIN;
        if (time < least) each = of, least = time;
        if (ctas * segments > 8 * places) break;          // more only adds rounds
    }
    s.seg_chunks = (uint32_t)(each * (128 / SCAN_Q));
    s.segments = pieces ? (uint32_t)((pieces + each - 1) / each) : 1;
    s.states = (size_t)d->H * d->P * d->N;
    auto whole = [](size_t floats) { return (floats + 63) / 64 * 64; };      // parts of the workspace start on 256 bytes
    s.state_floats = s.segments > 1 ? whole((size_t)d->batch * s.segments * s.states) : 0;
    s.decay_floats = s.segments > 1 ? whole((size_t)d->batch * s.segments * d->H) : 0;
    // rows of a sequence, or whole chunks
    s.part_floats = whole((size_t)d->batch * s.vheads * s.np * (s.tc ? (size_t)s.segments * s.seg_chunks * SCAN_Q : d->L));
    s.dot_floats = whole((size_t)d->batch * s.vheads * d->L);
    s.end_floats = whole((size_t)d->batch * s.segments * s.vheads);
    s.x_pack = s.pack ? whole((size_t)d->batch * d->L * d->H * ((d->P + 7) / 8 * 4)) : 0;
    s.b_pack = s.pack ? whole((size_t)d->batch * d->L * d->G * ((d->N + 7) / 8 * 4)) : 0;
    return s;
}

static const char* scan_check(const fesc_clear_scan_desc* d) {
    if (d->type > FESC_F32) return "clear_scan: unknown type";
    if (!d->H || !d->P || !d->N || !d->G || d->H % d->G) return "clear_scan: an empty dimension, or groups that do not divide the heads";
    if (d->N > SCAN_MAX_STATE) return "clear_scan: states of more than 128 columns";
    if (d->G > 65535) return "clear_scan: more than 65535 groups";
    if (d->P > 4096 || d->L >= (1u << 30)) return "clear_scan: more than 4096 channels of a head or 2^30 tokens";
    const ScanShape s = scan_shape(d, false), back = scan_shape(d, true);
    const uint64_t segments = std::max(s.segments, back.segments);
    if (3 * (uint64_t)d->batch * segments * s.vheads >= (1ull << 31) || d->batch > 65535 ||
        (uint64_t)d->batch * d->G * ((uint64_t)d->L / 8 + 1) * 2 + (uint64_t)d->batch * d->H * segments >= (1ull << 31) - d->H || (uint64_t)d->H * d->P * d->N >= (1ull << 31))
        return "clear_scan: too many sequences, heads or tokens for one call";
    return nullptr;
}

// Strides of a buffer with rows of `inner` elements: none is negative; elements of a written buffer are distinct.
static bool scan_strides(const int64_t (&s)[3], uint64_t b, uint64_t t, uint64_t h, uint64_t inner, bool written) {
    uint64_t count[3] = {b, t, h};
    for (int i = 0; i < 3; i++)
        if (s[i] < 0 || s[i] > (int64_t)1 << 40) return false;
    if (!written) return true;
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; i++)
        for (int j = i + 1; j < 3; j++)
            if (s[order[j]] < s[order[i]]) std::swap(order[i], order[j]);
    uint64_t span = inner;
    for (int i = 0; i < 3; i++) {
        const int k = order[i];
        if (count[k] <= 1) continue;
        if ((uint64_t)s[k] < span) return false;
        span += (uint64_t)s[k] * (count[k] - 1);
    }
    return true;
}
static ScanOperand operand(const void* p, const int64_t (&s)[3], bool tiled, uint32_t bytes) {
    ScanOperand o = {p, s[0], s[1], s[2], tiled, bytes};
    for (uint32_t to = 16; to > bytes; to /= 2)
        if ((size_t)p % to == 0 && s[0] * bytes % to == 0 && s[1] * bytes % to == 0 && s[2] * bytes % to == 0) {
            o.align = to;
            break;
        }
    return o;
}
static uint32_t out_width(const void* p, const int64_t (&s)[3], uint32_t bytes) {
    auto fits = [&](int64_t to) { return (int64_t)((size_t)p % to) == 0 && s[0] * bytes % to == 0 && s[1] * bytes % to == 0 && s[2] * bytes % to == 0; };
    return fits(32) ? 2 : fits(16) ? 1 : 0;
}
static ScanArgs scan_args(const fesc_clear_scan_desc* d, const ScanShape& s, const float* g, const int* lengths) {
    ScanArgs a = {};
    a.g = g, a.gb = d->g[0], a.gt = d->g[1], a.gh = d->g[2], a.lengths = lengths;
    a.b = d->batch, a.L = d->L, a.H = d->H, a.P = d->P, a.G = d->G, a.N = d->N;
    a.tiles = s.tiles, a.segments = s.segments, a.seg_chunks = s.seg_chunks;
    return a;
}
static cudaError_t scan_go(const fesc_clear_scan_desc* d, bool tc, const ScanSet& a, int mode, cudaStream_t st) {
    return tc                    ? scan_tc_launch(a, mode, st)
         : d->type == FESC_BF16 ? scan_launch<__nv_bfloat16>(a, mode, st)
         : d->type == FESC_F16  ? scan_launch<__half>(a, mode, st)
                                : scan_launch<float>(a, mode, st);
}
static cudaError_t combine(const fesc_clear_scan_desc* d, const ScanShape& s, const Chain& forwards, const Chain& back, cudaStream_t st) {
    return launch(k_clear_combine, dim3((uint32_t)((s.states + 1023) / 1024), d->batch, back.states ? 2 : 1), dim3(256), 0, st, forwards, back, s.segments, d->P * d->N,
                  s.states);
}

// Copies of operands in rows of whole 16-byte pieces, at `w` and on; the operands then are the copies.
struct Packed {
    ScanOperand* o;
    uint32_t heads, width;
    size_t floats;
};
static cudaError_t pack(const fesc_clear_scan_desc* d, std::initializer_list<Packed> list, float* w, const int* lengths, cudaStream_t st) {
    TcPack a = {};
    a.lengths = lengths, a.L = d->L;
    for (const Packed& p : list) {
        auto& o = a.o[a.count++];
        const long long row = (p.width + 7) / 8 * 8;
        o.src = p.o->p, o.dst = w, o.sb = p.o->sb, o.st = p.o->st, o.sh = p.o->sh, o.heads = p.heads, o.width = p.width;
        *p.o = {w, (long long)d->L * p.heads * row, p.heads * row, row, p.o->tiled, 16};
        w += p.floats;
    }
    return scan_tc_pack(a, d->batch, st);
}

extern "C" size_t fesc_clear_scan_work(const fesc_clear_scan_desc* desc) {
    if (!desc || scan_check(desc)) return 0;
    const ScanShape s = scan_shape(desc, false);
    return (s.state_floats + s.decay_floats + s.x_pack + 2 * s.b_pack) * sizeof(float);
}
extern "C" size_t fesc_clear_scan_backward_work(const fesc_clear_scan_desc* desc) {
    if (!desc || scan_check(desc)) return 0;
    const ScanShape s = scan_shape(desc, true);
    return (2 * (s.state_floats + s.decay_floats + s.part_floats + s.dot_floats + s.x_pack + s.b_pack) + 3 * s.end_floats) * sizeof(float);
}

extern "C" int fesc_clear_scan(const fesc_clear_scan_desc* desc, const void* d_x, const float* d_g, const void* d_B, const void* d_C, const float* d_skip,
                               const float* d_h0, const int32_t* d_lengths, void* d_y, float* d_h_out, void* d_work, size_t work_bytes, void* stream) {
    if (!desc) return clear_fail(FESC_EINVAL, "clear_scan: no descriptor");
    if (const char* what = scan_check(desc)) return clear_fail(FESC_EINVAL, what);
    const fesc_clear_scan_desc& d = *desc;
    if (d.batch == 0) return FESC_OK;
    if (!scan_strides(d.x, d.batch, d.L, d.H, d.P, false) || !scan_strides(d.g, d.batch, d.L, d.H, 1, false) || !scan_strides(d.B, d.batch, d.L, d.G, d.N, false) ||
        !scan_strides(d.C, d.batch, d.L, d.G, d.N, false) || !scan_strides(d.y, d.batch, d.L, d.H, d.P, true))
        return clear_fail(FESC_EINVAL, "clear_scan: a stride is negative or beyond 2^40, or elements of y overlap");
    if (d.L && (!d_x || !d_g || !d_B || !d_C || !d_y)) return clear_fail(FESC_EINVAL, "clear_scan: x, g, B, C and y have to be given");
    if (same_buffer({d_y, d_h_out}, {d_x, d_g, d_B, d_C, d_skip, d_h0, d_lengths})) return clear_fail(FESC_EINVAL, "clear_scan: an output is an input or the other output");
    const ScanShape s = scan_shape(desc, false);
    const size_t need = fesc_clear_scan_work(desc);
    if (need && (!d_work || ((size_t)d_work & 255) || work_bytes < need))
        return clear_fail(FESC_EINVAL, "clear_scan: the workspace is too small or not aligned to 256 bytes");
    cudaStream_t st = (cudaStream_t)stream;
    const uint32_t bytes = clear_type_bytes(d.type);
    ScanArgs a = scan_args(desc, s, d_g, d_lengths);
    a.q = operand(d_C, d.C, false, bytes), a.k = operand(d_B, d.B, false, bytes), a.v = operand(d_x, d.x, true, bytes);
    if (s.pack)
        CLEAR_CUDA(pack(desc, {{&a.v, d.H, d.P, s.x_pack}, {&a.k, d.G, d.N, s.b_pack}, {&a.q, d.G, d.N, s.b_pack}}, (float*)d_work + s.state_floats + s.decay_floats,
                        d_lengths, st));
    const bool tc = s.tc && a.q.align == 16 && a.k.align == 16 && a.v.align == 16;
    a.init = d_h0;
    if (s.segments > 1) {
        float* states = (float*)d_work;
        float* decay = states + s.state_floats;
        a.last = states, a.decay = decay;
        CLEAR_CUDA(scan_go(desc, tc, {{a}, 1}, MODE_STATE, st));
        CLEAR_CUDA(combine(desc, s, {states, decay, d_h0}, {}, st));
        a.init = states;
    }
    a.last = d_h_out, a.skip = d_skip, a.out = d_y, a.ob = d.y[0], a.ot = d.y[1], a.oh = d.y[2];
    a.out_wide = out_width(d_y, d.y, bytes);
    CLEAR_CUDA(scan_go(desc, tc, {{a}, 1}, MODE_OUT, st));
    return FESC_OK;
}

extern "C" int fesc_clear_scan_backward(const fesc_clear_scan_desc* desc, const void* d_x, const float* d_g, const void* d_B, const void* d_C, const float* d_skip,
                                        const float* d_h0, const int32_t* d_lengths, const void* d_dy, const float* d_dh_out, void* d_dx, float* d_dg, void* d_dB,
                                        void* d_dC, float* d_dskip, float* d_dh0, void* d_work, size_t work_bytes, void* stream) {
    if (!desc) return clear_fail(FESC_EINVAL, "clear_scan_backward: no descriptor");
    if (const char* what = scan_check(desc)) return clear_fail(FESC_EINVAL, what);
    const fesc_clear_scan_desc& d = *desc;
    cudaStream_t st = (cudaStream_t)stream;
    if (d.batch == 0) {
        if (d_dskip) CLEAR_CUDA(cudaMemsetAsync(d_dskip, 0, d.H * sizeof(float), st));
        return FESC_OK;
    }
    if (!scan_strides(d.x, d.batch, d.L, d.H, d.P, false) || !scan_strides(d.g, d.batch, d.L, d.H, 1, false) || !scan_strides(d.B, d.batch, d.L, d.G, d.N, false) ||
        !scan_strides(d.C, d.batch, d.L, d.G, d.N, false) || !scan_strides(d.y, d.batch, d.L, d.H, d.P, false) ||
        !scan_strides(d.dx, d.batch, d.L, d.H, d.P, true) || !scan_strides(d.dg, d.batch, d.L, d.H, 1, true) || !scan_strides(d.dB, d.batch, d.L, d.G, d.N, true) ||
        !scan_strides(d.dC, d.batch, d.L, d.G, d.N, true))
        return clear_fail(FESC_EINVAL, "clear_scan_backward: a stride is negative or beyond 2^40, or elements of an output overlap");
    if (d.L && (!d_x || !d_g || !d_B || !d_C || !d_dy || !d_dx || !d_dg || !d_dB || !d_dC))
        return clear_fail(FESC_EINVAL, "clear_scan_backward: x, g, B, C, dy, dx, dg, dB and dC have to be given");
    if (same_buffer({d_dx, d_dg, d_dB, d_dC, d_dskip, d_dh0}, {d_x, d_g, d_B, d_C, d_skip, d_h0, d_lengths, d_dy, d_dh_out}))
        return clear_fail(FESC_EINVAL, "clear_scan_backward: an output is an input, or two outputs are the same");
    const ScanShape s = scan_shape(desc, true);
    const size_t need = fesc_clear_scan_backward_work(desc);
    if (!d_work || ((size_t)d_work & 255) || work_bytes < need)
        return clear_fail(FESC_EINVAL, "clear_scan_backward: the workspace is too small or not aligned to 256 bytes");
    float* w = (float*)d_work;
    auto take = [&](size_t floats) { float* p = w; w += floats; return p; };
    float *before = take(s.state_floats), *behind = take(s.state_floats), *decay = take(s.decay_floats), *decay_back = take(s.decay_floats);
    float *part_b = take(s.part_floats), *part_c = take(s.part_floats), *row = take(s.dot_floats), *col = take(s.dot_floats);
    float *ends = take(s.end_floats), *diag = take(s.end_floats), *starts = take(s.end_floats);
    const uint32_t bytes = clear_type_bytes(d.type);
    ScanOperand x = operand(d_x, d.x, true, bytes), B = operand(d_B, d.B, false, bytes), C = operand(d_C, d.C, false, bytes), dy = operand(d_dy, d.y, true, bytes);
    if (s.pack)
        CLEAR_CUDA(pack(desc, {{&x, d.H, d.P, s.x_pack}, {&dy, d.H, d.P, s.x_pack}, {&B, d.G, d.N, s.b_pack}, {&C, d.G, d.N, s.b_pack}}, w, d_lengths, st));
    const bool tc = s.tc && x.align == 16 && B.align == 16 && C.align == 16 && dy.align == 16;
    const ScanArgs base = scan_args(desc, s, d_g, d_lengths);
    const float *h = d_h0, *dh = d_dh_out;
    if (s.segments > 1) {
        ScanSet states = {{base, base}, 2};
        states.a[0].k = B, states.a[0].v = x, states.a[0].last = before, states.a[0].decay = decay;
        states.a[1].k = C, states.a[1].v = dy, states.a[1].last = behind, states.a[1].decay = decay_back, states.a[1].backwards = 1;
        CLEAR_CUDA(scan_go(desc, tc, states, MODE_STATE, st));
        CLEAR_CUDA(combine(desc, s, {before, decay, d_h0}, {behind, decay_back, d_dh_out}, st));
        h = before, dh = behind;
    }
    ScanSet set = {{base, base, base}, 3};
    ScanArgs &c = set.a[0], &b = set.a[1], &o = set.a[2];
    c.q = dy, c.k = x, c.v = B, c.u = C, c.init = h, c.meet = dh, c.part = part_c, c.dots = row, c.ends = ends, c.diag = diag;      // dC
    b.q = x, b.k = dy, b.v = C, b.u = B, b.init = dh, b.part = part_b, b.dots = col, b.backwards = 1;                               // dB
    if (d_h0) b.meet = d_h0, b.ends = starts;
    // dx, and the gradient of the state before the first token
    o.q = B, o.k = C, o.v = dy, o.init = dh, o.last = d_dh0, o.skip = d_skip, o.out = d_dx, o.ob = d.dx[0], o.ot = d.dx[1], o.oh = d.dx[2];
    o.out_wide = out_width(d_dx, d.dx, bytes), o.backwards = 1;
    CLEAR_CUDA(scan_go(desc, tc, set, MODE_GRAD, st));
    FinishArgs f = {};
    f.part_b = part_b, f.part_c = part_c, f.row = row, f.col = col, f.ends = ends, f.starts = d_h0 ? starts : nullptr, f.diag = diag;
    f.dB = d_dB, f.dC = d_dC, f.dg = d_dg, f.dskip = d_dskip, f.lengths = d_lengths, f.g = d_g, f.ib = d.g[0], f.it = d.g[1], f.ih = d.g[2];
    f.Bb = d.dB[0], f.Bt = d.dB[1], f.Bg = d.dB[2], f.Cb = d.dC[0], f.Ct = d.dC[1], f.Cg = d.dC[2], f.gb = d.dg[0], f.gt = d.dg[1], f.gh = d.dg[2];
    f.b = d.batch, f.L = d.L, f.H = d.H, f.G = d.G, f.N = d.N, f.tiles = s.tiles, f.segments = s.segments, f.seg_chunks = s.seg_chunks;
    f.log_quads = d.N > 64 ? 5 : 4, f.dg_blocks = d.batch * d.H * s.segments;
    if (tc) {        // sums of their own; the decays after them
        TcSums t = {part_b, part_c, B, C, (__nv_bfloat16*)d_dB, (__nv_bfloat16*)d_dC, row, col, d_lengths, f.Bb, f.Bt, f.Bg, f.Cb, f.Ct, f.Cg,
                    d.L, d.H, d.G, d.N, s.tiles, s.segments, s.seg_chunks, out_width(d_dB, d.dB, bytes) && out_width(d_dC, d.dC, bytes)};
        CLEAR_CUDA(scan_tc_sums(t, d.batch, st));
    } else {
        f.sum_each = (uint32_t)((((size_t)d.L << f.log_quads) + 255) / 256), f.sum_blocks = 2 * d.batch * d.G * f.sum_each;
    }
    auto finish = [&](auto kernel, uint32_t threads) {
        return launch(kernel, dim3(f.sum_blocks + f.dg_blocks + (d.H + threads / 32 - 1) / (threads / 32)), dim3(threads), 0, st, f);
    };
    if (tc) CLEAR_CUDA(finish(k_clear_scan_finish<__nv_bfloat16, 1024>, 1024));
    else if (d.type == FESC_BF16) CLEAR_CUDA(finish(k_clear_scan_finish<__nv_bfloat16, 256>, 256));
    else if (d.type == FESC_F16) CLEAR_CUDA(finish(k_clear_scan_finish<__half, 256>, 256));
    else CLEAR_CUDA(finish(k_clear_scan_finish<float, 256>, 256));
    return FESC_OK;
}

extern "C" int fesc_clear_scan_step(const fesc_clear_scan_desc* desc, const void* d_x, const float* d_g, const void* d_B, const void* d_C, const float* d_skip,
                                    const float* d_state, float* d_state_out, void* d_y, void* stream) {
    if (!desc) return clear_fail(FESC_EINVAL, "clear_scan_step: no descriptor");
    fesc_clear_scan_desc d = *desc;
    d.L = 1;
    if (const char* what = scan_check(&d)) return clear_fail(FESC_EINVAL, what);
    if (d.batch == 0) return FESC_OK;
    if (!d_x || !d_g || !d_B || !d_C || !d_state || !d_state_out || !d_y) return clear_fail(FESC_EINVAL, "clear_scan_step: x, g, B, C, the states and y have to be given");
    if (!scan_strides(d.x, d.batch, 1, d.H, d.P, false) || !scan_strides(d.g, d.batch, 1, d.H, 1, false) || !scan_strides(d.B, d.batch, 1, d.G, d.N, false) ||
        !scan_strides(d.C, d.batch, 1, d.G, d.N, false) || !scan_strides(d.y, d.batch, 1, d.H, d.P, true))
        return clear_fail(FESC_EINVAL, "clear_scan_step: a stride is negative or beyond 2^40, or elements of y overlap");
    if (same_buffer({d_y, d_state_out}, {d_x, d_g, d_B, d_C, d_skip}) || d_y == d_state)
        return clear_fail(FESC_EINVAL, "clear_scan_step: y is an input or a state, or the new state an input other than the old");
    if ((uint64_t)d.batch * d.H >= (1ull << 31)) return clear_fail(FESC_EINVAL, "clear_scan_step: too many sequences and heads for one call");
    StepArgs a = {d_x, d_B, d_C, d_g, d_skip, d_state, d_state_out, d_y, d.x[0], d.x[2], d.B[0], d.B[2], d.C[0], d.C[2], d.g[0], d.g[2], d.y[0], d.y[2],
                  d.H, d.P, d.N, d.G};
    const bool wide = d.N % 4 == 0 && ((size_t)d_state & 15) == 0 && ((size_t)d_state_out & 15) == 0;
    // eight rows per warp share B and C; where that leaves SMs without a CTA, one (a token of 24 heads: 192 CTAs instead of 24)
    const bool many = (uint64_t)d.batch * d.H * ((d.P + 63) / 64) >= 4 * 148;
    const dim3 grid(d.batch * d.H, many ? (d.P + 63) / 64 : (d.P + 7) / 8);
    auto pick = [&](auto t) {
        using T = decltype(t);
        return wide ? many ? k_clear_scan_step<T, true, 8> : k_clear_scan_step<T, true, 1> : many ? k_clear_scan_step<T, false, 8> : k_clear_scan_step<T, false, 1>;
    };
    auto kernel = d.type == FESC_BF16 ? pick(__nv_bfloat16()) : d.type == FESC_F16 ? pick(__half()) : pick(float());
    CLEAR_CUDA(launch(kernel, grid, dim3(256), 0, (cudaStream_t)stream, a));
    return FESC_OK;
}
