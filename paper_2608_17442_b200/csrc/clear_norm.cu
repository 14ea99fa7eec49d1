// Cleartext RMS norm with the gate before it and the residual around it, forward and backward:
//   v = y * silu(z),  h = r + s * v,  n = gamma * h / sqrt(mean h^2 + eps)      (mean over a group of channels)
// the products that the encrypted path forms in fesc_norm_square and fesc_norm_scale, with the gate and residual of the block.
//
// One pass: a thread holds eight neighbours of a row, as many warps as a group of channels needs form a team (3 for 768 channels, 6 for
// 1536), sums go through shuffles and one exchange in shared memory, and what depends on them is written from the registers.  Bound by memory.
// The gradients of gamma and s are sums over rows: a CTA adds up its own rows in a fixed order, a second kernel adds up the CTAs, so the
// results do not depend on the order in which CTAs run.  There the next row's loads are under way while a row is computed.
#define FESC_DBG_FILE 16   // file id in the sites a debug build reports
#include "clear.cuh"

#define NORM_WARPS 8            // of a CTA, unless a team is larger
#define NORM_MAX_WIDTH 8192     // channels of a group: 32 warps of 256

struct NormArgs {
    const void *y, *gate, *residual, *dn, *dh;
    void *n, *h, *dy, *dgate, *dresidual;
    const float *gamma, *scale;
    float* part;                 // backward: [CTA][gamma, scale][d]
    long long sy, sgate, sresidual, sdn, sdh, sn, sh, sdy, sdgate, sdresidual;
    uint32_t rows, d, width;     // width: channels of a group
    float eps;
    uint32_t wide;               // every buffer allows 16-byte accesses
    uint32_t team_warps;
};

// The sums of a and b over a team of warps, in the same order for every thread.  The words of a turn are written again two turns later, behind the
// barrier of the next.
__device__ __forceinline__ void team_sum(float& a, float& b, float2* words, uint32_t team_warps) {
#pragma unroll
    for (int o = 16; o; o >>= 1) a += __shfl_xor_sync(~0u, a, o), b += __shfl_xor_sync(~0u, b, o);
    if (team_warps == 1) return;
    const uint32_t warp = threadIdx.x >> 5, first = warp / team_warps * team_warps;
    if ((threadIdx.x & 31) == 0) words[warp] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
    for (uint32_t i = 0; i < team_warps; i++) {
        const float2 w = words[first + i];
        a += w.x, b += w.y;
    }
}

// By the approximate exponential and reciprocal (2 units each; the exponent's rounding adds 2^-24 |z|): with the exact ones the backward pass of the
// gate issues for as long as it moves bytes.
__device__ __forceinline__ float sigmoid(float z) {
    float e, s;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return s;
}

// Eight neighbours of a row as they are in memory: what a thread keeps between its two looks at them (half the registers of float32 for 16-bit types)
template <class T>
struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p, int count, bool wide) {
        if (wide && count >= 8) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) w[i] = reinterpret_cast<const uint4*>(p)[i];
        } else {
            T v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = i < count ? p[i] : ClearType<T>::from(0.f);
            memcpy(w, v, sizeof(v));
        }
    }
    __device__ __forceinline__ float operator[](int i) const {      // i known when compiled
        const uint32_t u[4] = {w[0].x, w[0].y, w[0].z, w[0].w};
        if constexpr (sizeof(T) == 4) {
            const uint32_t x[4] = {w[sizeof(T) / 2 - 1].x, w[sizeof(T) / 2 - 1].y, w[sizeof(T) / 2 - 1].z, w[sizeof(T) / 2 - 1].w};
            return __uint_as_float(i < 4 ? u[i & 3] : x[i & 3]);
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            return __uint_as_float(i & 1 ? u[i >> 1] & 0xFFFF0000u : u[i >> 1] << 16);
        } else {
            const __half2 h = *reinterpret_cast<const __half2*>(&u[i >> 1]);
            return i & 1 ? __high2float(h) : __low2float(h);
        }
    }
};

template <class T, bool GATE, bool RESIDUAL, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : 4) k_clear_norm(const NormArgs a) {
    __shared__ float2 words[2][32];
    pdl_begin();
    const uint32_t teams = (blockDim.x >> 5) / a.team_warps, team = (threadIdx.x >> 5) / a.team_warps, first = blockIdx.y * a.width;
    const int c = (int)(threadIdx.x - team * a.team_warps * 32) * 8, width = (int)a.width - c;
    const T *py = (const T*)a.y + first + c, *pz = (const T*)a.gate + first + c, *pr = (const T*)a.residual + first + c;
    float g[8], s[8];
    const bool ok = DBG_REGION(a.gamma, a.d * sizeof(float)) && (!a.scale || DBG_REGION(a.scale, a.d * sizeof(float)));
    Eight<T> y, z, r, ny, nz, nr;
    auto fetch = [&](uint32_t row) {
        int count = row < a.rows && width > 0 ? width : 0;
        const size_t bytes = (size_t)min(count, 8) * sizeof(T);
        if (count && !(DBG_REGION(py + row * a.sy, bytes) && (!GATE || DBG_REGION(pz + row * a.sgate, bytes)) && (!RESIDUAL || DBG_REGION(pr + row * a.sresidual, bytes))))
            count = 0;
        ny.load(py + row * a.sy, count, a.wide);
        if (GATE) nz.load(pz + row * a.sgate, count, a.wide);
        if (RESIDUAL) nr.load(pr + row * a.sresidual, count, a.wide);
    };
    fetch(blockIdx.x * teams + team);
    clear_load8(a.gamma + first + c, ok ? width : 0, a.wide, g);
    if (RESIDUAL && a.scale) clear_load8(a.scale + first + c, ok ? width : 0, a.wide, s);
    uint32_t turn = 0;
    // the same number of turns for every team: barriers inside
    for (uint32_t base = blockIdx.x * teams; base < a.rows; base += gridDim.x * teams, turn ^= 1) {
        const uint32_t row = base + team;
        y = ny, z = nz, r = nr;
        fetch(row + gridDim.x * teams);
        float h[8], sum = 0.f, unused = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            float v = y[e];
            if (GATE) v *= z[e] * sigmoid(z[e]);
            if (RESIDUAL) v = r[e] + (a.scale ? s[e] * v : v);
            h[e] = v, sum += v * v;      // zeros behind the row's end
        }
        T* n = (T*)a.n + (long long)row * a.sn + first + c;
        T* ho = a.h ? (T*)a.h + (long long)row * a.sh + first + c : nullptr;
        int count = row < a.rows ? width : 0;
        const size_t bytes = (size_t)min(max(count, 0), 8) * sizeof(T);
        if (count > 0 && !(DBG_REGION(n, bytes) && (!ho || DBG_REGION(ho, bytes)))) count = 0;
        if (ho) clear_store8(ho, count, a.wide, h);
        team_sum(sum, unused, words[turn], a.team_warps);
        const float rho = rsqrtf(sum / (float)a.width + a.eps);
#pragma unroll
        for (int e = 0; e < 8; e++) h[e] *= g[e] * rho;
        clear_store8(n, count, a.wide, h);
    }
}

// dh_tot = dh + rho w - h rho^3 mean(w h),  w = gamma dn;  dr = dh_tot;  ds = sum_rows dh_tot v;  dv = s dh_tot;
// dy = dv silu(z);  dz = dv y sigma (1 + z (1 - sigma));  dgamma = sum_rows dn h rho
template <class T, bool GATE, bool RESIDUAL, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : RESIDUAL ? 2 : 3) k_clear_norm_backward(const NormArgs a) {
    __shared__ float2 words[2][32];
    __shared__ float cols[NORM_WARPS * 256];
    pdl_begin();
    const uint32_t teams = (blockDim.x >> 5) / a.team_warps, team = (threadIdx.x >> 5) / a.team_warps, first = blockIdx.y * a.width;
    const int c = (int)(threadIdx.x - team * a.team_warps * 32) * 8, width = (int)a.width - c;
    const T *py = (const T*)a.y + first + c, *pz = (const T*)a.gate + first + c, *pr = (const T*)a.residual + first + c, *pn = (const T*)a.dn + first + c,
            *ph = (const T*)a.dh + first + c;
    const bool dh = RESIDUAL && a.dh;
    float g[8], s[8], dgamma[8] = {}, dscale[8] = {};
    const bool ok = DBG_REGION(a.gamma, a.d * sizeof(float)) && (!a.scale || DBG_REGION(a.scale, a.d * sizeof(float)));
    clear_load8(a.gamma + first + c, ok ? width : 0, a.wide, g);
    if (RESIDUAL && a.scale) clear_load8(a.scale + first + c, ok ? width : 0, a.wide, s);
    Eight<T> y, z, r, w, hh, ny, nz, nr, nw, nh;
    auto fetch = [&](uint32_t row, Eight<T>& vy, Eight<T>& vz, Eight<T>& vr, Eight<T>& vw, Eight<T>& vh) {
        int count = row < a.rows && width > 0 ? width : 0;
        const size_t bytes = (size_t)min(count, 8) * sizeof(T);
        if (count && !(DBG_REGION(py + row * a.sy, bytes) && DBG_REGION(pn + row * a.sdn, bytes) && (!GATE || DBG_REGION(pz + row * a.sgate, bytes)) &&
                       (!RESIDUAL || DBG_REGION(pr + row * a.sresidual, bytes)) && (!dh || DBG_REGION(ph + row * a.sdh, bytes))))
            count = 0;
        vy.load(py + row * a.sy, count, a.wide), vw.load(pn + row * a.sdn, count, a.wide);
        if (GATE) vz.load(pz + row * a.sgate, count, a.wide);
        if (RESIDUAL) vr.load(pr + row * a.sresidual, count, a.wide);
        if (dh) vh.load(ph + row * a.sdh, count, a.wide);
    };
    fetch(blockIdx.x * teams + team, ny, nz, nr, nw, nh);
    uint32_t turn = 0;
    // the same number of turns for every team: barriers inside
    for (uint32_t base = blockIdx.x * teams; base < a.rows; base += gridDim.x * teams, turn ^= 1) {
        const uint32_t row = base + team;
        y = ny, z = nz, r = nr, w = nw, hh = nh;
        fetch(row + gridDim.x * teams, ny, nz, nr, nw, nh);
        float h[8], sig[8], sum = 0.f, dot = 0.f;
#pragma unroll
        for (int e = 0; e < 8; e++) {
            sig[e] = GATE ? sigmoid(z[e]) : 1.f;
            float v = y[e];
            if (GATE) v *= z[e] * sig[e];
            if (RESIDUAL) v = r[e] + (a.scale ? s[e] * v : v);
            h[e] = v;
            sum += v * v, dot += g[e] * w[e] * v;
        }
        team_sum(sum, dot, words[turn], a.team_warps);
        const float rho = rsqrtf(sum / (float)a.width + a.eps), k = rho * rho * rho * (dot / (float)a.width);
        int count = row < a.rows ? width : 0;
        T* dy = (T*)a.dy + (long long)row * a.sdy + first + c;
        T* dz = GATE ? (T*)a.dgate + (long long)row * a.sdgate + first + c : nullptr;
        T* dr = RESIDUAL ? (T*)a.dresidual + (long long)row * a.sdresidual + first + c : nullptr;
        const size_t bytes = (size_t)min(max(count, 0), 8) * sizeof(T);
        if (count > 0 && !(DBG_REGION(dy, bytes) && (!GATE || DBG_REGION(dz, bytes)) && (!RESIDUAL || DBG_REGION(dr, bytes)))) count = 0;
        float d[8];
#pragma unroll
        for (int e = 0; e < 8; e++) {
            d[e] = rho * g[e] * w[e] - k * h[e];
            if (dh) d[e] += hh[e];
            dgamma[e] += w[e] * h[e] * rho;
        }
        if (RESIDUAL) {
            clear_store8(dr, count, a.wide, d);
            if (a.scale) {
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    dscale[e] += d[e] * (GATE ? y[e] * z[e] * sig[e] : y[e]);
                    d[e] *= s[e];
                }
            }
        }
        if (GATE) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[e] = d[e] * y[e] * sig[e] * (1.f + z[e] * (1.f - sig[e]));
                d[e] *= z[e] * sig[e];
            }
            clear_store8(dz, count, a.wide, v);
        }
        clear_store8(dy, count, a.wide, d);
    }
    // the teams' sums, team by team
    float* part = a.part + (size_t)blockIdx.x * 2 * a.d + first;
    if (!DBG_REGION(part, (a.d + a.width) * sizeof(float))) return;
    auto leave = [&](const float(&v)[8], float* out) {
        if (teams == 1) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (e < width) out[c + e] = v[e];
            return;
        }
        const uint32_t span = a.team_warps * 256;       // a CTA of several teams has at most NORM_WARPS warps
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; e++) cols[team * span + c + e] = v[e];
        __syncthreads();
        for (uint32_t j = threadIdx.x; j < a.width; j += blockDim.x) {
            float t = 0.f;
            for (uint32_t m = 0; m < teams; m++) t += cols[m * span + j];
            out[j] = t;
        }
    };
    leave(dgamma, part);
    if (RESIDUAL && a.scale) leave(dscale, part + a.d);
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
// warps of a group of channels, and teams of them in a CTA
struct NormShape {
    uint32_t warps, teams;
};
static NormShape norm_shape(const fesc_clear_norm_desc* desc) {
    const uint32_t warps = (desc->d / desc->groups + 255) / 256;
    return {warps, warps < NORM_WARPS ? NORM_WARPS / warps : 1};
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

template <class T, int THREADS>
static void (*norm_kernel(bool gate, bool residual))(NormArgs) {
    return gate ? residual ? k_clear_norm<T, true, true, THREADS> : k_clear_norm<T, true, false, THREADS>
                : residual ? k_clear_norm<T, false, true, THREADS> : k_clear_norm<T, false, false, THREADS>;
}
// CTAs of more than 256 threads (rows of more than 2048 channels) have 64 registers a thread and keep some of a row's words in local memory
template <class T, int THREADS>
static void (*norm_backward_kernel(bool gate, bool residual))(NormArgs) {
    return gate ? residual ? k_clear_norm_backward<T, true, true, THREADS> : k_clear_norm_backward<T, true, false, THREADS>
                : residual ? k_clear_norm_backward<T, false, true, THREADS> : k_clear_norm_backward<T, false, false, THREADS>;
}
template <class F>
static auto by_type(uint32_t type, F f) {
    return type == FESC_BF16 ? f(__nv_bfloat16()) : type == FESC_F16 ? f(__half()) : f(float());
}

// CTAs per group of channels, to which rows are dealt out: as many as are resident (a thread has up to 64 registers forwards, 80 backwards, 128
// backwards with a residual).
// Backwards their column sums are added up afterwards.
static uint32_t norm_ctas(const fesc_clear_norm_desc* desc, const NormShape& s, bool backward, bool residual) {
    const uint64_t all = (desc->rows + s.teams - 1) / s.teams;
    const uint32_t threads = s.warps * s.teams * 32, resident = threads > 256 ? (threads > 512 ? 1 : 2) : 65536 / (threads * (!backward ? 64 : residual ? 128 : 80));
    return all < 148 * resident ? (uint32_t)all : 148 * resident;
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
    const NormShape s = norm_shape(desc);
    a.team_warps = s.warps;
    auto kernel = by_type(desc->type, [&](auto t) { 
        return s.warps > NORM_WARPS ? norm_kernel<decltype(t), 1024>(d_gate, d_residual) : norm_kernel<decltype(t), 256>(d_gate, d_residual);
    });
    CLEAR_CUDA(launch(kernel, dim3(norm_ctas(desc, s, false, d_residual), desc->groups), dim3(s.teams * s.warps * 32), 0, (cudaStream_t)stream, a));
    return FESC_OK;
}

extern "C" size_t fesc_clear_norm_backward_work(const fesc_clear_norm_desc* desc) {
    const char* what;
    if (!desc || norm_check(desc, &what) != FESC_OK) return 0;
    return (size_t)norm_ctas(desc, norm_shape(desc), true, false) * 2 * desc->d * sizeof(float);
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
    const NormShape s = norm_shape(desc);
    a.team_warps = s.warps;
    const uint32_t ctas = norm_ctas(desc, s, true, d_residual);
    auto kernel = by_type(desc->type, [&](auto t) { 
        return s.warps > NORM_WARPS ? norm_backward_kernel<decltype(t), 1024>(d_gate, d_residual) : norm_backward_kernel<decltype(t), 256>(d_gate, d_residual);
    });
    CLEAR_CUDA(launch(kernel, dim3(ctas, desc->groups), dim3(s.teams * s.warps * 32), 0, st, a));
    CLEAR_CUDA(launch(k_clear_norm_columns, dim3((desc->d + 31) / 32, d_dscale ? 2 : 1), dim3(256), 0, st, (const float*)a.part, d_dgamma, d_dscale, ctas, desc->d));
    return FESC_OK;
}
