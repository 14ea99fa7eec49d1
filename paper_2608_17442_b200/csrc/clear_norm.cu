// Cleartext RMS norm with the gate before it and the residual around it, forward and backward:
//   v = y * silu(z),  h = r + s * v,  n = gamma * h / sqrt(mean h^2 + eps)      (mean over a group of channels)
// the products that the encrypted path forms in fesc_norm_square and fesc_norm_scale, with the gate and residual of the block.
//
// One pass: a group of a row is read once into registers, its sums go through shuffles (and shared memory between warps), and what depends on
// them is written from the registers.  Bound by memory.  A thread holds up to NV x 8 neighbours; a CTA deals out as many rows as it has
// teams of threads.
// The gradients of gamma and s are sums over rows: a CTA adds up its own rows in a fixed order, a second kernel adds up the CTAs, so the
// results do not depend on the order in which CTAs run.
#define FESC_DBG_FILE 16   // file id in the sites a debug build reports
#include "clear.cuh"

#define NORM_THREADS 256
#define NORM_MAX_WIDTH 8192     // channels of a group: 512 threads x 16 registers

struct NormArgs {
    const void *y, *gate, *residual, *dn, *dh;
    void *n, *h, *dy, *dgate, *dresidual;
    const float *gamma, *scale;
    float* part;                 // backward: [CTA][gamma, scale][d]
    long long sy, sgate, sresidual, sdn, sdh, sn, sh, sdy, sdgate, sdresidual;
    uint32_t rows, d, width;     // width: channels of a group
    float eps;
    uint32_t wide;               // every buffer allows 16-byte accesses
};

// The sums of a and b over a team of TPR threads, in the same order for every thread.  `turn` alternates between calls: the words of a turn are
// written again only after the barrier of the next.
template <int TPR, int TEAMS>
__device__ __forceinline__ void team_sum(float& a, float& b, float2 (*words)[TEAMS][TPR / 32], uint32_t turn) {
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(~0u, a, o), b += __shfl_xor_sync(~0u, b, o);
    if constexpr (TPR > 32) {
        const uint32_t team = threadIdx.x / TPR, warp = threadIdx.x % TPR / 32;
        float2(&w)[TPR / 32] = words[turn & 1][team];
        if (threadIdx.x % 32 == 0) w[warp] = make_float2(a, b);
        __syncthreads();
        a = b = 0.f;
#pragma unroll
        for (int i = 0; i < TPR / 32; i++) a += w[i].x, b += w[i].y;
    }
}

__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + expf(-z)); }

template <class T, int TPR, int NV>
__global__ void __launch_bounds__(TPR > NORM_THREADS ? TPR : NORM_THREADS) k_clear_norm(const NormArgs a) {
    constexpr int TEAMS = TPR > NORM_THREADS ? 1 : NORM_THREADS / TPR;
    __shared__ float2 words[2][TEAMS][TPR / 32];
    pdl_begin();
    const uint32_t row = blockIdx.x * TEAMS + threadIdx.x / TPR, lane = threadIdx.x % TPR, first = blockIdx.y * a.width;
    const T* y = (const T*)a.y + (long long)row * a.sy + first;
    const T* z = a.gate ? (const T*)a.gate + (long long)row * a.sgate + first : nullptr;
    const T* r = a.residual ? (const T*)a.residual + (long long)row * a.sresidual + first : nullptr;
    T* n = (T*)a.n + (long long)row * a.sn + first;
    T* ho = a.h ? (T*)a.h + (long long)row * a.sh + first : nullptr;
    const size_t bytes = a.width * sizeof(T);
    bool live = row < a.rows;
    if (live) live = DBG_REGION(y, bytes) && (!z || DBG_REGION(z, bytes)) && (!r || DBG_REGION(r, bytes)) && DBG_REGION(n, bytes) &&
                     (!ho || DBG_REGION(ho, bytes)) && DBG_REGION(a.gamma, a.d * sizeof(float)) && (!a.scale || DBG_REGION(a.scale, a.d * sizeof(float)));
    float h[NV][8], sum = 0.f, unused = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = (i * TPR + lane) * 8, count = live ? (int)a.width - c : 0;
        clear_load8(y + c, count, a.wide, h[i]);
        if (z) {
            float g[8];
            clear_load8(z + c, count, a.wide, g);
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= g[e] * sigmoid(g[e]);
        }
        if (a.scale) {
            float s[8];
            clear_load8(a.scale + first + c, count, a.wide, s);
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] *= s[e];
        }
        if (r) {
            float v[8];
            clear_load8(r + c, count, a.wide, v);
#pragma unroll
            for (int e = 0; e < 8; e++) h[i][e] += v[e];
        }
        if (ho) clear_store8(ho + c, count, a.wide, h[i]);
#pragma unroll
        for (int e = 0; e < 8; e++) sum += e < count ? h[i][e] * h[i][e] : 0.f;
    }
    team_sum<TPR, TEAMS>(sum, unused, words, 0);
    const float rho = rsqrtf(sum / (float)a.width + a.eps);
#pragma unroll
    for (int i = 0; i < NV; i++) {
        const int c = (i * TPR + lane) * 8, count = live ? (int)a.width - c : 0;
        float g[8];
        clear_load8(a.gamma + first + c, count, a.wide, g);
#pragma unroll
        for (int e = 0; e < 8; e++) g[e] *= h[i][e] * rho;
        clear_store8(n + c, count, a.wide, g);
    }
}

// dh_tot = dh + rho w - h rho^3 mean(w h),  w = gamma dn;  dr = dh_tot;  ds = sum_rows dh_tot v;  dv = s dh_tot;
// dy = dv silu(z);  dz = dv y sigma (1 + z (1 - sigma));  dgamma = sum_rows dn h rho
template <class T, int TPR, int NV>
__global__ void __launch_bounds__(TPR > NORM_THREADS ? TPR : NORM_THREADS) k_clear_norm_backward(const NormArgs a) {
    constexpr int TEAMS = TPR > NORM_THREADS ? 1 : NORM_THREADS / TPR;
    __shared__ float2 words[2][TEAMS][TPR / 32];
    __shared__ float cols[TEAMS > 1 ? TEAMS : 1][TEAMS > 1 ? TPR * 8 : 1];
    pdl_begin();
    const uint32_t team = threadIdx.x / TPR, lane = threadIdx.x % TPR, first = blockIdx.y * a.width;
    const size_t bytes = a.width * sizeof(T);
    float dgamma[NV][8] = {}, dscale[NV][8] = {};
    uint32_t turn = 0;
    // the same number of turns for every team: barriers inside
    for (uint32_t base = blockIdx.x * TEAMS; base < a.rows; base += gridDim.x * TEAMS, turn++) {
        const uint32_t row = base + team;
        const T* y = (const T*)a.y + (long long)row * a.sy + first;
        const T* z = a.gate ? (const T*)a.gate + (long long)row * a.sgate + first : nullptr;
        const T* r = a.residual ? (const T*)a.residual + (long long)row * a.sresidual + first : nullptr;
        const T* dn = (const T*)a.dn + (long long)row * a.sdn + first;
        const T* dh = a.dh ? (const T*)a.dh + (long long)row * a.sdh + first : nullptr;
        T* dy = (T*)a.dy + (long long)row * a.sdy + first;
        T* dz = a.dgate ? (T*)a.dgate + (long long)row * a.sdgate + first : nullptr;
        T* dr = a.dresidual ? (T*)a.dresidual + (long long)row * a.sdresidual + first : nullptr;
        bool live = row < a.rows;
        if (live) live = DBG_REGION(y, bytes) && (!z || DBG_REGION(z, bytes)) && (!r || DBG_REGION(r, bytes)) && DBG_REGION(dn, bytes) &&
                         (!dh || DBG_REGION(dh, bytes)) && DBG_REGION(dy, bytes) && (!dz || DBG_REGION(dz, bytes)) && (!dr || DBG_REGION(dr, bytes));
        float yv[NV][8], zv[NV][8], h[NV][8], w[NV][8], sum = 0.f, dot = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (i * TPR + lane) * 8, count = live ? (int)a.width - c : 0;
            clear_load8(y + c, count, a.wide, yv[i]);
            clear_load8(dn + c, count, a.wide, w[i]);
            if (z) clear_load8(z + c, count, a.wide, zv[i]);
            if (r) clear_load8(r + c, count, a.wide, h[i]);
        }
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (i * TPR + lane) * 8, count = live ? (int)a.width - c : 0;
            float s[8], g[8];
            if (a.scale) clear_load8(a.scale + first + c, count, a.wide, s);
            clear_load8(a.gamma + first + c, count, a.wide, g);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                float v = yv[i][e];
                if (z) v *= zv[i][e] * sigmoid(zv[i][e]);
                if (a.scale) v *= s[e];
                h[i][e] = r ? h[i][e] + v : v;
                if (e < count) sum += h[i][e] * h[i][e], dot += g[e] * w[i][e] * h[i][e];
            }
        }
        team_sum<TPR, TEAMS>(sum, dot, words, turn);
        const float rho = rsqrtf(sum / (float)a.width + a.eps), k = rho * rho * rho * (dot / (float)a.width);
#pragma unroll
        for (int i = 0; i < NV; i++) {
            const int c = (i * TPR + lane) * 8, count = live ? (int)a.width - c : 0;
            float s[8], g[8], d[8];
            if (a.scale) clear_load8(a.scale + first + c, count, a.wide, s);
            clear_load8(a.gamma + first + c, count, a.wide, g);
            if (dh) clear_load8(dh + c, count, a.wide, d);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float t = rho * g[e] * w[i][e] - k * h[i][e];
                d[e] = dh ? d[e] + t : t;
                if (e < count) dgamma[i][e] += w[i][e] * h[i][e] * rho;
            }
            if (dr) clear_store8(dr + c, count, a.wide, d);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float sig = z ? sigmoid(zv[i][e]) : 1.f, gate = z ? zv[i][e] * sig : 1.f, yy = yv[i][e];
                if (a.scale && e < count) dscale[i][e] += d[e] * yy * gate;
                if (a.scale) d[e] *= s[e];
                yv[i][e] = d[e] * gate;
                if (z) zv[i][e] = d[e] * yy * sig * (1.f + zv[i][e] * (1.f - sig));
            }
            clear_store8(dy + c, count, a.wide, yv[i]);
            if (dz) clear_store8(dz + c, count, a.wide, zv[i]);
        }
    }
    // the teams' sums, team by team
    float* part = a.part + (size_t)blockIdx.x * 2 * a.d + first;
    if (!DBG_REGION(part, (a.d + a.width) * sizeof(float))) return;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        if (q && !a.scale) break;
#pragma unroll
        for (int i = 0; i < NV; i++) {
            float(&v)[8] = q ? dscale[i] : dgamma[i];
            const int c = (i * TPR + lane) * 8;
            if constexpr (TEAMS > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < 8; e++) cols[team][lane * 8 + e] = v[e];
                __syncthreads();
                for (uint32_t j = threadIdx.x; j < TPR * 8; j += NORM_THREADS) {
                    float t = 0.f;
                    for (int m = 0; m < TEAMS; m++) t += cols[m][j];
                    if (i * TPR * 8 + j < a.width) part[(size_t)q * a.d + i * TPR * 8 + j] = t;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (c + e < (int)a.width) part[(size_t)q * a.d + c + e] = v[e];
            }
        }
    }
}

// out[c] = the CTAs' sums of channel c: 8 threads take every eighth CTA each, then add up
__global__ void __launch_bounds__(256) k_clear_norm_columns(const float* part, float* dgamma, float* dscale, uint32_t ctas, uint32_t d) {
    __shared__ float words[8][33];
    pdl_begin();
    const uint32_t x = threadIdx.x & 31, s = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float* out = blockIdx.y ? dscale : dgamma;
    if (!DBG_REGION(part, (size_t)ctas * 2 * d * sizeof(float)) || !DBG_REGION(out, d * sizeof(float))) return;
    double t = 0.0;
    if (c < d)
        for (uint32_t i = s; i < ctas; i += 8) t += part[((size_t)i * 2 + blockIdx.y) * d + c];
    words[s][x] = (float)t;
    __syncthreads();
    if (s == 0 && c < d) {
        double v = 0.0;
        for (int i = 0; i < 8; i++) v += words[i][x];
        out[c] = (float)v;
    }
}

// ---------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------
// threads of a row and vectors of a thread: as few threads as keep at most `most` vectors each
struct NormShape {
    uint32_t tpr, nv;
};
static NormShape norm_shape(uint32_t width, uint32_t small, uint32_t middle, uint32_t most) {
    const uint32_t tpr = width <= small * 8 * most ? small : width <= middle * 8 * most ? middle : 512;
    return {tpr, (width + tpr * 8 - 1) / (tpr * 8)};
}

static int norm_check(const fesc_clear_norm_desc* desc, const char** what) {
    *what = nullptr;
    if (desc->type > FESC_F32) *what = "clear_norm: unknown type";
    else if (!desc->d || !desc->groups || desc->d % desc->groups) *what = "clear_norm: groups have to divide the channels";
    else if (desc->d / desc->groups > NORM_MAX_WIDTH) *what = "clear_norm: a group has more than 8192 channels";
    else if (desc->groups > 65535) *what = "clear_norm: more than 65535 groups";
    else if (desc->rows > 0x7fffff00u) *what = "clear_norm: too many rows";
    else if (!(desc->eps > 0.f)) *what = "clear_norm: eps has to be positive (a row of zeros has no norm)";
    return *what ? FESC_EINVAL : FESC_OK;
}

// a buffer of rows: its stride holds a row, and 16-byte accesses are possible
static bool norm_stride(const fesc_clear_norm_desc* desc, const void* p, int64_t stride, bool written) {
    if (!p) return true;
    return stride >= 0 && (written ? stride >= (int64_t)desc->d || desc->rows <= 1 : true);
}
static bool norm_wide(const fesc_clear_norm_desc* desc, const void* p, int64_t stride, uint32_t bytes) {
    return !p || (((size_t)p & 15) == 0 && (stride * bytes) % 16 == 0);
}

template <class T>
static void (*norm_kernel(NormShape s))(NormArgs) {
#define NORM_PICK(t, v) \
    if (s.tpr == t && s.nv == v) return k_clear_norm<T, t, v>;
    NORM_PICK(32, 1) NORM_PICK(32, 2) NORM_PICK(32, 3) NORM_PICK(32, 4) NORM_PICK(64, 3) NORM_PICK(64, 4) NORM_PICK(512, 1) NORM_PICK(512, 2)
#undef NORM_PICK
    return nullptr;
}
template <class T>
static void (*norm_backward_kernel(NormShape s))(NormArgs) {
#define NORM_PICK(t, v) \
    if (s.tpr == t && s.nv == v) return k_clear_norm_backward<T, t, v>;
    NORM_PICK(32, 1) NORM_PICK(32, 2) NORM_PICK(128, 1) NORM_PICK(128, 2) NORM_PICK(512, 1) NORM_PICK(512, 2)
#undef NORM_PICK
    return nullptr;
}
template <class F>
static auto by_type(uint32_t type, F f) {
    return type == FESC_BF16 ? f(__nv_bfloat16()) : type == FESC_F16 ? f(__half()) : f(float());
}

// CTAs of the backward pass per group of channels: rows are dealt out to at most this many, whose column sums are added up afterwards
static uint32_t norm_ctas(const fesc_clear_norm_desc* desc, const NormShape& s) {
    const uint32_t teams = s.tpr > NORM_THREADS ? 1 : NORM_THREADS / s.tpr, all = (desc->rows + teams - 1) / teams;
    const uint32_t most = 4 * 148;
    return all < most ? all : most;
}

extern "C" int fesc_clear_norm(const fesc_clear_norm_desc* desc, const void* d_y, const float* d_gamma, const void* d_gate, const void* d_residual,
                               const float* d_scale, void* d_n, void* d_h, void* stream) {
    const char* what;
    if (!desc) return clear_fail(FESC_EINVAL, "clear_norm: no descriptor");
    if (norm_check(desc, &what) != FESC_OK) return clear_fail(FESC_EINVAL, what);
    if (desc->rows == 0) return FESC_OK;
    if (!d_y || !d_gamma || !d_n) return clear_fail(FESC_EINVAL, "clear_norm: y, gamma and n have to be given");
    if (d_scale && !d_residual) return clear_fail(FESC_EINVAL, "clear_norm: a scale belongs to a residual");
    if (!norm_stride(desc, d_y, desc->y_stride, false) || !norm_stride(desc, d_gate, desc->gate_stride, false) ||
        !norm_stride(desc, d_residual, desc->residual_stride, false) || !norm_stride(desc, d_n, desc->n_stride, true) ||
        !norm_stride(desc, d_h, desc->h_stride, true))
        return clear_fail(FESC_EINVAL, "clear_norm: a row stride is negative, or rows of an output overlap");
    if (d_n == d_y || d_n == d_gate || d_n == d_residual || d_n == d_h || same_buffer(d_h, d_y) || same_buffer(d_h, d_gate) || same_buffer(d_h, d_residual))
        return clear_fail(FESC_EINVAL, "clear_norm: an output is an input or another output");
    const uint32_t bytes = clear_type_bytes(desc->type), width = desc->d / desc->groups;
    NormArgs a = {};
    a.y = d_y, a.gate = d_gate, a.residual = d_residual, a.n = d_n, a.h = d_h, a.gamma = d_gamma, a.scale = d_scale;
    a.sy = desc->y_stride, a.sgate = desc->gate_stride, a.sresidual = desc->residual_stride, a.sn = desc->n_stride, a.sh = desc->h_stride;
    a.rows = (uint32_t)desc->rows, a.d = desc->d, a.width = width, a.eps = desc->eps;
    a.wide = width * bytes % 16 == 0 && width % 4 == 0 && norm_wide(desc, d_y, a.sy, bytes) && norm_wide(desc, d_gate, a.sgate, bytes) &&
             norm_wide(desc, d_residual, a.sresidual, bytes) && norm_wide(desc, d_n, a.sn, bytes) && norm_wide(desc, d_h, a.sh, bytes) &&
             norm_wide(desc, d_gamma, 0, 4) && norm_wide(desc, d_scale, 0, 4);
    const NormShape s = norm_shape(width, 32, 64, 4);
    const uint32_t teams = s.tpr > NORM_THREADS ? 1 : NORM_THREADS / s.tpr;
    auto kernel = by_type(desc->type, [&](auto t) { return norm_kernel<decltype(t)>(s); });
    if (!kernel) return clear_fail(FESC_EINVAL, "clear_norm: no kernel for this width");
    CLEAR_CUDA(launch(kernel, dim3((a.rows + teams - 1) / teams, desc->groups), dim3(s.tpr > NORM_THREADS ? s.tpr : NORM_THREADS), 0, (cudaStream_t)stream, a));
    return FESC_OK;
}

extern "C" size_t fesc_clear_norm_backward_work(const fesc_clear_norm_desc* desc) {
    const char* what;
    if (!desc || norm_check(desc, &what) != FESC_OK) return 0;
    return (size_t)norm_ctas(desc, norm_shape(desc->d / desc->groups, 32, 128, 2)) * 2 * desc->d * sizeof(float);
}

extern "C" int fesc_clear_norm_backward(const fesc_clear_norm_desc* desc, const void* d_y, const float* d_gamma, const void* d_gate,
                                        const void* d_residual, const float* d_scale, const void* d_dn, const void* d_dh, void* d_dy, float* d_dgamma,
                                        void* d_dgate, void* d_dresidual, float* d_dscale, void* d_work, size_t work_bytes, void* stream) {
    const char* what;
    if (!desc) return clear_fail(FESC_EINVAL, "clear_norm_backward: no descriptor");
    if (norm_check(desc, &what) != FESC_OK) return clear_fail(FESC_EINVAL, what);
    cudaStream_t st = (cudaStream_t)stream;
    if (desc->rows == 0 && d_dgamma) {     // sums over no rows
        CLEAR_CUDA(cudaMemsetAsync(d_dgamma, 0, desc->d * sizeof(float), st));
        if (d_dscale) CLEAR_CUDA(cudaMemsetAsync(d_dscale, 0, desc->d * sizeof(float), st));
        return FESC_OK;
    }
    if (!d_y || !d_gamma || !d_dn || !d_dy || !d_dgamma) return clear_fail(FESC_EINVAL, "clear_norm_backward: y, gamma, dn, dy and dgamma have to be given");
    if (d_scale && !d_residual) return clear_fail(FESC_EINVAL, "clear_norm_backward: a scale belongs to a residual");
    if (!d_gate != !d_dgate || !d_residual != !d_dresidual || !d_scale != !d_dscale)
        return clear_fail(FESC_EINVAL, "clear_norm_backward: gate, residual and scale are given together with their gradients");
    if (!norm_stride(desc, d_y, desc->y_stride, false) || !norm_stride(desc, d_gate, desc->gate_stride, false) ||
        !norm_stride(desc, d_residual, desc->residual_stride, false) || !norm_stride(desc, d_dn, desc->dn_stride, false) ||
        !norm_stride(desc, d_dh, desc->dh_stride, false) || !norm_stride(desc, d_dy, desc->dy_stride, true) ||
        !norm_stride(desc, d_dgate, desc->dgate_stride, true) || !norm_stride(desc, d_dresidual, desc->dresidual_stride, true))
        return clear_fail(FESC_EINVAL, "clear_norm_backward: a row stride is negative, or rows of an output overlap");
    const void* outs[5] = {d_dy, d_dgate, d_dresidual, d_dgamma, d_dscale};
    const void* ins[7] = {d_y, d_gate, d_residual, d_dn, d_dh, d_gamma, d_scale};
    for (int i = 0; i < 5; i++) {
        for (int j = 0; j < 7; j++)
            if (same_buffer(outs[i], ins[j])) return clear_fail(FESC_EINVAL, "clear_norm_backward: an output is an input");
        for (int j = 0; j < i; j++)
            if (same_buffer(outs[i], outs[j])) return clear_fail(FESC_EINVAL, "clear_norm_backward: two outputs are the same");
    }
    const size_t need = fesc_clear_norm_backward_work(desc);
    if (!d_work || ((size_t)d_work & 15) || work_bytes < need) return clear_fail(FESC_EINVAL, "clear_norm_backward: the workspace is too small or not aligned to 16 bytes");
    const uint32_t bytes = clear_type_bytes(desc->type), width = desc->d / desc->groups;
    NormArgs a = {};
    a.y = d_y, a.gate = d_gate, a.residual = d_residual, a.dn = d_dn, a.dh = d_dh, a.dy = d_dy, a.dgate = d_dgate, a.dresidual = d_dresidual;
    a.gamma = d_gamma, a.scale = d_scale, a.part = (float*)d_work;
    a.sy = desc->y_stride, a.sgate = desc->gate_stride, a.sresidual = desc->residual_stride, a.sdn = desc->dn_stride, a.sdh = desc->dh_stride;
    a.sdy = desc->dy_stride, a.sdgate = desc->dgate_stride, a.sdresidual = desc->dresidual_stride;
    a.rows = (uint32_t)desc->rows, a.d = desc->d, a.width = width, a.eps = desc->eps;
    a.wide = width * bytes % 16 == 0 && width % 4 == 0 && norm_wide(desc, d_y, a.sy, bytes) && norm_wide(desc, d_gate, a.sgate, bytes) &&
             norm_wide(desc, d_residual, a.sresidual, bytes) && norm_wide(desc, d_dn, a.sdn, bytes) && norm_wide(desc, d_dh, a.sdh, bytes) &&
             norm_wide(desc, d_dy, a.sdy, bytes) && norm_wide(desc, d_dgate, a.sdgate, bytes) && norm_wide(desc, d_dresidual, a.sdresidual, bytes) &&
             norm_wide(desc, d_gamma, 0, 4) && norm_wide(desc, d_scale, 0, 4);
    const NormShape s = norm_shape(width, 32, 128, 2);
    const uint32_t ctas = norm_ctas(desc, s);
    auto kernel = by_type(desc->type, [&](auto t) { return norm_backward_kernel<decltype(t)>(s); });
    if (!kernel) return clear_fail(FESC_EINVAL, "clear_norm_backward: no kernel for this width");
    CLEAR_CUDA(launch(kernel, dim3(ctas, desc->groups), dim3(s.tpr > NORM_THREADS ? s.tpr : NORM_THREADS), 0, st, a));
    CLEAR_CUDA(launch(k_clear_norm_columns, dim3((desc->d + 31) / 32, d_dscale ? 2 : 1), dim3(256), 0, st, (const float*)a.part, d_dgamma, d_dscale, ctas, desc->d));
    return FESC_OK;
}
