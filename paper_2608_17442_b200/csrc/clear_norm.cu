// Cleartext RMS norm with the gate before it and the residual around it, forward and backward:
//   v = y * silu(z),  h = r + s * v,  n = gamma * h / sqrt(mean h^2 + eps)      (mean over a group of channels)
// the products that the encrypted path forms in fesc_norm_square and fesc_norm_scale, with the gate and residual of the block.
//
// One pass: a thread holds eight channels of a row (neighbours where 16-byte accesses are possible, every 32nd otherwise), as many warps as a
// group of channels needs form a team (3 for 768 channels, 6 for 1536), sums go through shuffles and one exchange in shared memory, and what
// depends on them is written from the registers.  Rows are dealt out to the CTAs that are resident, and the next row's loads are under way while a
// row is computed.  Bound by memory forwards (32768 x 768 with residual: 201 MB in 35 us, 0.89 of the copy rate).  The gate's backward pass (16384 x 1536:
// 252 MB in 61 us) fills neither memory (44 %) nor issue (64 %): 22 warps an SM wait for exponentials, reciprocals and shuffles, for one
// another at the row's exchange, and for the instruction before.
// The gradients of gamma and s are sums over rows: a thread adds up its own rows in float32, a CTA its teams, in a fixed order, a second kernel the CTAs in
// float64, so the results do not depend on the order in which CTAs run.
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

// For 16-bit rows by the approximate exponential (2 units; its argument's rounding adds 2^-24 |z|): with the exact one the backward pass of the gate
// issues for as long as it moves bytes.  Float32 rows would lose up to six bits by that (z = -80).  The reciprocal is off by one unit.
template <class T>
__device__ __forceinline__ float sigmoid(float z) {
    float e, s;
    if constexpr (sizeof(T) == 4) e = expf(-z);
    else asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(z * -1.4426950408889634f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(s) : "f"(1.f + e));
    return s;
}

// Eight channels of a row as they are in memory: what a thread keeps between its two looks at them (half the registers of float32 for 16-bit types).
// `left`: channels from the thread's first one to the group's end.
template <class T>
struct Eight {
    uint4 w[sizeof(T) / 2];
    __device__ __forceinline__ void load(const T* p, int left, bool wide) {
        if (wide) {
#pragma unroll
            for (int i = 0; i < (int)sizeof(T) / 2; i++) w[i] = left > 0 ? reinterpret_cast<const uint4*>(p)[i] : make_uint4(0, 0, 0, 0);
        } else {
            T v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = 32 * i < left ? p[32 * i] : ClearType<T>::from(0.f);
            memcpy(w, v, sizeof(v));
        }
    }
    __device__ __forceinline__ f2 operator[](int i) const {      // two of them, i known when compiled
        const uint4& v = w[sizeof(T) == 4 ? i >> 1 : 0];
        const uint32_t u[4] = {v.x, v.y, v.z, v.w};
        if constexpr (sizeof(T) == 4) {
            return {__uint_as_float(u[2 * (i & 1)]), __uint_as_float(u[2 * (i & 1) + 1])};
        } else if constexpr (std::is_same_v<T, __nv_bfloat16>) {
            return both(u[i]);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
            return {f.x, f.y};
        }
    }
};
template <class T>
__device__ __forceinline__ void store8(T* p, int left, bool wide, const f2 (&v)[4]) {
    if (wide) {
        const float x[8] = {v[0].x, v[0].y, v[1].x, v[1].y, v[2].x, v[2].y, v[3].x, v[3].y};
        if (left > 0) clear_store8(p, 8, true, x);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (32 * i < left) p[32 * i] = ClearType<T>::from(i & 1 ? v[i / 2].y : v[i / 2].x);
    }
}
__device__ __forceinline__ f2 twice(float v) { return {v, v}; }

// the channels of a thread: the first one, and how many there are from there to the group's end
__device__ __forceinline__ int first_channel(uint32_t thread, bool wide) { return wide ? thread * 8 : thread / 32 * 256 + thread % 32; }
// its bytes of a row, for the debug build
template <class T>
__device__ __forceinline__ size_t span8(int left, bool wide) {
    return left <= 0 ? 0 : wide ? 8 * sizeof(T) : (size_t)(min((left - 1) / 32, 7) * 32 + 1) * sizeof(T);
}

// CTAs of 256 threads on an SM.  Forwards a thread has 64 registers, for float32 rows with gate and residual 80 (16384 x 1536: 60 us, with 64 and what then
// goes to local memory 85); backwards 80, with a residual, or for float32 rows with a gate, 128 (93 us, with 80 108).
#define NORM_CTAS(BYTES, GATE, RESIDUAL) ((BYTES) == 4 && (GATE) && (RESIDUAL) ? 3 : 4)
#define NORM_BACK_CTAS(BYTES, GATE, RESIDUAL) ((RESIDUAL) || ((BYTES) == 4 && (GATE)) ? 2 : 3)
template <class T, bool GATE, bool RESIDUAL, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : NORM_CTAS(sizeof(T), GATE, RESIDUAL)) k_clear_norm(const NormArgs a) {
    __shared__ float2 words[2][32];
    pdl_begin();
    const uint32_t teams = (blockDim.x >> 5) / a.team_warps, team = (threadIdx.x >> 5) / a.team_warps, first = blockIdx.y * a.width;
    const int c = first_channel(threadIdx.x - team * a.team_warps * 32, a.wide), width = (int)a.width - c;
    const T *py = (const T*)a.y + first + c, *pz = (const T*)a.gate + first + c, *pr = (const T*)a.residual + first + c;
    const bool ok = DBG_REGION(a.gamma, a.d * sizeof(float)) && (!a.scale || DBG_REGION(a.scale, a.d * sizeof(float)));
    Eight<T> y, z, r, ny, nz, nr;
    Eight<float> g, s;
    auto fetch = [&](uint32_t row) {
        int left = row < a.rows ? width : 0;
        const size_t bytes = span8<T>(left, a.wide);
        if (left > 0 && !(DBG_REGION(py + row * a.sy, bytes) && (!GATE || DBG_REGION(pz + row * a.sgate, bytes)) && (!RESIDUAL || DBG_REGION(pr + row * a.sresidual, bytes))))
            left = 0;
        ny.load(py + row * a.sy, left, a.wide);
        if (GATE) nz.load(pz + row * a.sgate, left, a.wide);
        if (RESIDUAL) nr.load(pr + row * a.sresidual, left, a.wide);
    };
    fetch(blockIdx.x * teams + team);
    g.load(a.gamma + first + c, ok ? width : 0, a.wide);
    if (RESIDUAL && a.scale) s.load(a.scale + first + c, ok ? width : 0, a.wide);
    uint32_t turn = 0;
    // the same number of turns for every team: barriers inside
    for (uint32_t base = blockIdx.x * teams; base < a.rows; base += gridDim.x * teams, turn ^= 1) {
        const uint32_t row = base + team;
        y = ny, z = nz, r = nr;
        fetch(row + gridDim.x * teams);
        f2 h[4], sums = {0.f, 0.f};
        float unused = 0.f;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            f2 v = y[e];
            if (GATE) v = mul2(v, mul2(z[e], {sigmoid<T>(z[e].x), sigmoid<T>(z[e].y)}));
            if (RESIDUAL) v = a.scale ? fma2(s[e], v, r[e]) : add2(v, r[e]);
            h[e] = v, sums = fma2(v, v, sums);      // zeros behind the row's end
        }
        T* n = (T*)a.n + (long long)row * a.sn + first + c;
        T* ho = a.h ? (T*)a.h + (long long)row * a.sh + first + c : nullptr;
        int left = row < a.rows ? width : 0;
        const size_t bytes = span8<T>(left, a.wide);
        if (left > 0 && !(DBG_REGION(n, bytes) && (!ho || DBG_REGION(ho, bytes)))) left = 0;
        if (ho) store8(ho, left, a.wide, h);
        float sum = sums.x + sums.y;
        team_sum(sum, unused, words[turn], a.team_warps);
        const float rho = rsqrtf(sum / (float)a.width + a.eps);
#pragma unroll
        for (int e = 0; e < 4; e++) h[e] = mul2(h[e], mul2(g[e], twice(rho)));
        store8(n, left, a.wide, h);
    }
}

// dh_tot = dh + rho w - h rho^3 mean(w h),  w = gamma dn;  dr = dh_tot;  ds = sum_rows dh_tot v;  dv = s dh_tot;
// dy = dv silu(z);  dz = dv y sigma (1 + z (1 - sigma)) = dv y (sigma + silu(z) (1 - sigma));  dgamma = sum_rows dn h rho
// RESIDUAL: a residual, dh, or both
template <class T, bool GATE, bool RESIDUAL, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS > 256 ? 1 : NORM_BACK_CTAS(sizeof(T), GATE, RESIDUAL)) k_clear_norm_backward(const NormArgs a) {
    __shared__ float2 words[2][32];
    __shared__ float cols[NORM_WARPS * 256];
    pdl_begin();
    const uint32_t teams = (blockDim.x >> 5) / a.team_warps, team = (threadIdx.x >> 5) / a.team_warps, first = blockIdx.y * a.width;
    const int c = first_channel(threadIdx.x - team * a.team_warps * 32, a.wide), width = (int)a.width - c;
    const T *py = (const T*)a.y + first + c, *pz = (const T*)a.gate + first + c, *pr = (const T*)a.residual + first + c, *pn = (const T*)a.dn + first + c,
            *ph = (const T*)a.dh + first + c;
    const bool dh = RESIDUAL && a.dh;
    f2 dgamma[4] = {}, dscale[4] = {};
    const bool ok = DBG_REGION(a.gamma, a.d * sizeof(float)) && (!a.scale || DBG_REGION(a.scale, a.d * sizeof(float)));
    Eight<T> y, z, r, w, hh, ny, nz, nr, nw, nh;
    Eight<float> g, s;
    auto fetch = [&](uint32_t row) {
        int left = row < a.rows ? width : 0;
        const size_t bytes = span8<T>(left, a.wide);
        if (left > 0 && !(DBG_REGION(py + row * a.sy, bytes) && DBG_REGION(pn + row * a.sdn, bytes) && (!GATE || DBG_REGION(pz + row * a.sgate, bytes)) &&
                          (!RESIDUAL || !a.residual || DBG_REGION(pr + row * a.sresidual, bytes)) && (!dh || DBG_REGION(ph + row * a.sdh, bytes))))
            left = 0;
        ny.load(py + row * a.sy, left, a.wide), nw.load(pn + row * a.sdn, left, a.wide);
        if (GATE) nz.load(pz + row * a.sgate, left, a.wide);
        if (RESIDUAL) nr.load(pr + row * a.sresidual, a.residual ? left : 0, a.wide);
        if (dh) nh.load(ph + row * a.sdh, left, a.wide);
    };
    fetch(blockIdx.x * teams + team);
    g.load(a.gamma + first + c, ok ? width : 0, a.wide);
    if (RESIDUAL && a.scale) s.load(a.scale + first + c, ok ? width : 0, a.wide);
    uint32_t turn = 0;
    // the same number of turns for every team: barriers inside
    for (uint32_t base = blockIdx.x * teams; base < a.rows; base += gridDim.x * teams, turn ^= 1) {
        const uint32_t row = base + team;
        y = ny, z = nz, r = nr, w = nw, hh = nh;
        fetch(row + gridDim.x * teams);
        f2 h[4], sig[4], sums = {0.f, 0.f}, dots = {0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 4; e++) {
            f2 v = y[e];
            if (GATE) sig[e] = {sigmoid<T>(z[e].x), sigmoid<T>(z[e].y)}, v = mul2(v, mul2(z[e], sig[e]));
            if (RESIDUAL) v = a.scale ? fma2(s[e], v, r[e]) : add2(v, r[e]);
            h[e] = v;
            sums = fma2(v, v, sums), dots = fma2(mul2(g[e], w[e]), v, dots);
        }
        float sum = sums.x + sums.y, dot = dots.x + dots.y;
        team_sum(sum, dot, words[turn], a.team_warps);
        const float rho = rsqrtf(sum / (float)a.width + a.eps), k = rho * (rho * (rho * (dot / (float)a.width)));      // rho cubed alone may overflow
        int left = row < a.rows ? width : 0;
        T* dy = (T*)a.dy + (long long)row * a.sdy + first + c;
        T* dz = GATE ? (T*)a.dgate + (long long)row * a.sdgate + first + c : nullptr;
        T* dr = RESIDUAL && a.dresidual ? (T*)a.dresidual + (long long)row * a.sdresidual + first + c : nullptr;
        const size_t bytes = span8<T>(left, a.wide);
        if (left > 0 && !(DBG_REGION(dy, bytes) && (!GATE || DBG_REGION(dz, bytes)) && (!dr || DBG_REGION(dr, bytes)))) left = 0;
        f2 d[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const f2 wr = mul2(w[e], twice(rho));
            d[e] = fma2(h[e], twice(-k), mul2(g[e], wr));
            if (dh) d[e] = add2(d[e], hh[e]);
            dgamma[e] = fma2(wr, h[e], dgamma[e]);
        }
        if (RESIDUAL && dr) store8(dr, left, a.wide, d);
        f2 o[4];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const f2 silu = GATE ? mul2(z[e], sig[e]) : f2{1.f, 1.f};
            if (RESIDUAL && a.scale) {
                dscale[e] = fma2(d[e], GATE ? mul2(y[e], silu) : y[e], dscale[e]);
                d[e] = mul2(d[e], s[e]);
            }
            if (GATE) o[e] = mul2(mul2(d[e], y[e]), fma2(silu, fma2(sig[e], twice(-1.f), twice(1.f)), sig[e])), d[e] = mul2(d[e], silu);
        }
        if (GATE) store8(dz, left, a.wide, o);
        store8(dy, left, a.wide, d);
    }
    // the teams' sums, team by team
    float* part = a.part + (size_t)blockIdx.x * 2 * a.d + first;
    if (!DBG_REGION(part, (a.d + a.width) * sizeof(float))) return;
    auto leave = [&](const f2 (&v)[4], float* out) {
        const int step = a.wide ? 1 : 32;
        if (teams == 1) {
#pragma unroll
            for (int e = 0; e < 8; e++)
                if (e * step < width) out[c + e * step] = e & 1 ? v[e / 2].y : v[e / 2].x;
            return;
        }
        const uint32_t span = a.team_warps * 256;       // a CTA of several teams has at most NORM_WARPS warps
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; e++) cols[team * span + c + e * step] = e & 1 ? v[e / 2].y : v[e / 2].x;
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

// out[c] = the CTAs' sums of channel c: 32 threads take every 32nd CTA each, then add up in a tree (8 threads with 74 loads each took longer than
// the pass over the rows)
__global__ void __launch_bounds__(1024) k_clear_norm_columns(const float* part, float* dgamma, float* dscale, uint32_t ctas, uint32_t d) {
    __shared__ double words[32][33];
    pdl_begin();
    const uint32_t x = threadIdx.x & 31, s = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float* out = blockIdx.y ? dscale : dgamma;
    if (!DBG_REGION(part, (size_t)ctas * 2 * d * sizeof(float)) || !DBG_REGION(out, d * sizeof(float))) return;
    double t = 0.0;
    if (c < d) {
#pragma unroll 4
        for (uint32_t i = s; i < ctas; i += 32) t += part[((size_t)i * 2 + blockIdx.y) * d + c];
    }
    words[s][x] = t;
    __syncthreads();
    double v = words[x][s];      // warp s adds up column s
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    if (x == 0 && blockIdx.x * 32 + s < d) out[blockIdx.x * 32 + s] = (float)v;
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
// Some of a row's words go to local memory: in CTAs of more than 256 threads (rows of more than 2048 channels, 64 registers a thread), in 16-bit rows with a
// gate (40 bytes at 80 registers) and in float32 rows with gate and residual (96 bytes at 128).
template <class T, int THREADS>
static void (*norm_backward_kernel(bool gate, bool residual))(NormArgs) {
    return gate ? residual ? k_clear_norm_backward<T, true, true, THREADS> : k_clear_norm_backward<T, true, false, THREADS>
                : residual ? k_clear_norm_backward<T, false, true, THREADS> : k_clear_norm_backward<T, false, false, THREADS>;
}
template <class F>
static auto by_type(uint32_t type, F f) {
    return type == FESC_BF16 ? f(__nv_bfloat16()) : type == FESC_F16 ? f(__half()) : f(float());
}

// CTAs per group of channels, to which rows are dealt out: as many as are resident, by the registers of a thread.  Backwards their column sums are added up afterwards.
static uint32_t norm_ctas(const fesc_clear_norm_desc* desc, const NormShape& s, uint32_t registers) {
    const uint64_t all = (desc->rows + s.teams - 1) / s.teams;
    const uint32_t threads = s.warps * s.teams * 32, resident = threads > 256 ? (threads > 512 ? 1 : 2) : 65536 / (threads * registers);
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
    if (same_buffer({d_n, d_h}, {d_y, d_gate, d_residual, d_gamma, d_scale}))
        return clear_fail(FESC_EINVAL, "clear_norm: an output is an input or another output");
    const uint32_t bytes = clear_type_bytes(desc->type), width = desc->d / desc->groups;
    NormArgs a = {};
    a.y = d_y, a.gate = d_gate, a.residual = d_residual, a.n = d_n, a.h = d_h, a.gamma = d_gamma, a.scale = d_scale;
    a.sy = desc->y_stride, a.sgate = desc->gate_stride, a.sresidual = desc->residual_stride, a.sn = desc->n_stride, a.sh = desc->h_stride;
    a.rows = (uint32_t)desc->rows, a.d = desc->d, a.width = width, a.eps = desc->eps;
    a.wide = width % 8 == 0 && norm_wide(desc, d_y, a.sy, bytes) && norm_wide(desc, d_gate, a.sgate, bytes) &&
             norm_wide(desc, d_residual, a.sresidual, bytes) && norm_wide(desc, d_n, a.sn, bytes) && norm_wide(desc, d_h, a.sh, bytes) &&
             norm_wide(desc, d_gamma, 0, 4) && norm_wide(desc, d_scale, 0, 4);
    const NormShape s = norm_shape(desc);
    a.team_warps = s.warps;
    auto kernel = by_type(desc->type, [&](auto t) {
        return s.warps > NORM_WARPS ? norm_kernel<decltype(t), 1024>(d_gate, d_residual) : norm_kernel<decltype(t), 256>(d_gate, d_residual);
    });
    CLEAR_CUDA(launch(kernel, dim3(norm_ctas(desc, s, NORM_CTAS(bytes, d_gate, d_residual) == 3 ? 80 : 64), desc->groups), dim3(s.teams * s.warps * 32), 0, (cudaStream_t)stream, a));
    return FESC_OK;
}

extern "C" size_t fesc_clear_norm_backward_work(const fesc_clear_norm_desc* desc) {
    const char* what;
    if (!desc || norm_check(desc, &what) != FESC_OK) return 0;
    return (size_t)norm_ctas(desc, norm_shape(desc), 80) * 2 * desc->d * sizeof(float);
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
    if (same_buffer({d_dy, d_dgate, d_dresidual, d_dgamma, d_dscale}, {d_y, d_gate, d_residual, d_dn, d_dh, d_gamma, d_scale}))
        return clear_fail(FESC_EINVAL, "clear_norm_backward: an output is an input, or two outputs are the same");
    const size_t need = fesc_clear_norm_backward_work(desc);
    if (!d_work || ((size_t)d_work & 15) || work_bytes < need) return clear_fail(FESC_EINVAL, "clear_norm_backward: the workspace is too small or not aligned to 16 bytes");
    const uint32_t bytes = clear_type_bytes(desc->type), width = desc->d / desc->groups;
    NormArgs a = {};
    a.y = d_y, a.gate = d_gate, a.residual = d_residual, a.dn = d_dn, a.dh = d_dh, a.dy = d_dy, a.dgate = d_dgate, a.dresidual = d_dresidual;
    a.gamma = d_gamma, a.scale = d_scale, a.part = (float*)d_work;
    a.sy = desc->y_stride, a.sgate = desc->gate_stride, a.sresidual = desc->residual_stride, a.sdn = desc->dn_stride, a.sdh = desc->dh_stride;
    a.sdy = desc->dy_stride, a.sdgate = desc->dgate_stride, a.sdresidual = desc->dresidual_stride;
    a.rows = (uint32_t)desc->rows, a.d = desc->d, a.width = width, a.eps = desc->eps;
    a.wide = width % 8 == 0 && norm_wide(desc, d_y, a.sy, bytes) && norm_wide(desc, d_gate, a.sgate, bytes) &&
             norm_wide(desc, d_residual, a.sresidual, bytes) && norm_wide(desc, d_dn, a.sdn, bytes) && norm_wide(desc, d_dh, a.sdh, bytes) &&
             norm_wide(desc, d_dy, a.sdy, bytes) && norm_wide(desc, d_dgate, a.sdgate, bytes) && norm_wide(desc, d_dresidual, a.sdresidual, bytes) &&
             norm_wide(desc, d_gamma, 0, 4) && norm_wide(desc, d_scale, 0, 4);
    const NormShape s = norm_shape(desc);
    a.team_warps = s.warps;
    const bool both = d_residual || d_dh;
    const uint32_t ctas = norm_ctas(desc, s, NORM_BACK_CTAS(bytes, d_gate, both) == 2 ? 128 : 80);
    auto kernel = by_type(desc->type, [&](auto t) {
        return s.warps > NORM_WARPS ? norm_backward_kernel<decltype(t), 1024>(d_gate, both) : norm_backward_kernel<decltype(t), 256>(d_gate, both);
    });
    CLEAR_CUDA(launch(kernel, dim3(ctas, desc->groups), dim3(s.teams * s.warps * 32), 0, st, a));
    CLEAR_CUDA(launch(k_clear_norm_columns, dim3((desc->d + 31) / 32, d_dscale ? 2 : 1), dim3(1024), 0, st, (const float*)a.part, d_dgamma, d_dscale, ctas, desc->d));
    return FESC_OK;
}
