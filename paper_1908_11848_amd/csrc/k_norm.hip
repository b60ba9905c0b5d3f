// Layer norm over the channels of a row, forward and backward, fp32 or bf16.
//
// Both are bound by memory: forward reads and writes a row once (2 x C elements), backward reads x and dy (and the shortcut's gradient) and writes dx. So
// a row stays in registers between its sums and its result: mean, then the squares of the deviations from it (two passes over
// registers, one over memory), everything in fp32.  WAVES wavefronts share a row, a lane holds E elements of it in vectors of 16 bytes.
// Measured: forward 16384 x 1024 fp32 20.8 us in the kernel (6.4 TB/s: part of it comes out of the last cache), 25.5 a call; backward 65536 x 2048 bf16 with a shortcut 192 us and 5.5 for the sums, 201 a
// call (5.4 TB/s; a copy of 1 GB runs at 5.0 to 5.1).  Rows of more than 8192 channels backward run at half that: no registers are left to fetch ahead.
//
// The weights' gradients are sums over rows.  A workgroup takes every G-th group of rows, and as a lane's channels stay the same, adds
// its share up in registers; G records of 2 C sums go to scratch memory and are added up by a second kernel in the order of their number.  No atomics: the
// order is that of the sizes alone.
#include "rows.hpp"
#include "../../include/dssp_kernels.h"

namespace {

constexpr int MAX_C = DSSPK_LAYERNORM_MAX_C;

// Sums of N numbers over the WAVES wavefronts of a row.  lds: N WAVES floats of the row's own, other ones in the call before and the one behind: one barrier a call is
// enough then, whoever writes a place again has passed the barrier behind its readers.
template <int WAVES, int N> __device__ __forceinline__ void row_sums(float (&v)[N], float* lds) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = rows::wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        const int wave = (threadIdx.x >> 6) % WAVES;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) lds[N * wave + i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = lds[i];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += lds[N * w + i];
    }
}

// WAVES wavefronts a row, ROWS rows a workgroup
template <class T, int E, int WAVES, int ROWS>
__global__ __launch_bounds__(64 * WAVES * ROWS) void layernorm_fwd_kernel(const T* x, const float* __restrict__ gamma, const float* __restrict__ beta, T* y,
                                                                          float* __restrict__ stats, long ldx, long ldy, long M, int C, float eps, bool past) {
    constexpr int VEC = rows::VEC<T>, NV = E / VEC, LANES = 64 * WAVES;
    __shared__ float lds[2][ROWS][WAVES];
    const int lane = threadIdx.x % LANES, part = threadIdx.x / LANES;
    const bool there = (long)blockIdx.x * ROWS + part < M;
    const long row = there ? (long)blockIdx.x * ROWS + part : M - 1;        // behind the last row: the last row again, for the barriers
    float v[E], g[E], b[E];
#pragma unroll
    for (int i = 0; i < NV; ++i) rows::load(x + row * ldx + (i * LANES + lane) * VEC, C - (i * LANES + lane) * VEC, v + i * VEC);
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        const int at = (i / VEC * LANES + lane) * VEC + i % VEC;
        rows::load(gamma + at, C - at, g + i);
        rows::load(beta + at, C - at, b + i);
    }
    const float inv = 1.f / C;
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < E; ++i) s[0] += v[i];
    row_sums<WAVES>(s, lds[0][part]);
    const float mean = s[0] * inv;
    s[0] = 0.f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        v[i] = (i / VEC * LANES + lane) * VEC + i % VEC < C ? v[i] - mean : 0.f;
        s[0] = fmaf(v[i], v[i], s[0]);
    }
    row_sums<WAVES>(s, lds[1][part]);
    const float invstd = 1.f / sqrtf(s[0] * inv + eps);
    if (!there) return;
    if (stats && lane == 0) *reinterpret_cast<float2*>(stats + 2 * row) = make_float2(mean, invstd);
#pragma unroll
    for (int i = 0; i < E; ++i) v[i] = fmaf(v[i] * invstd, g[i], b[i]);
#pragma unroll
    for (int i = 0; i < NV; ++i) rows::store(y + row * ldy + (i * LANES + lane) * VEC, C - (i * LANES + lane) * VEC, v + i * VEC, past);
}

// While a row is worked on, the next one of the workgroup is on its way from memory (not where registers are short: 16 wavefronts of 16 elements).
template <class T, int E, int WAVES, int ROWS>
__global__ __launch_bounds__(64 * WAVES * ROWS) void layernorm_bwd_kernel(const T* __restrict__ x, const float* __restrict__ gamma, const float* __restrict__ stats,
                                                                          const T* dy, const T* add, T* dx, float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                                          long ldx, long lddy, long ldadd, long lddx, long M, int C, bool past) {
    constexpr int VEC = rows::VEC<T>, NV = E / VEC, LANES = 64 * WAVES;
    constexpr bool AHEAD = E <= 8;
    __shared__ float lds[2][ROWS][2 * WAVES];
    extern __shared__ float sums[];     // ROWS > 1: 2 C
    const int lane = threadIdx.x % LANES, part = threadIdx.x / LANES;
    auto column = [&](int i) { return (i / VEC * LANES + lane) * VEC + i % VEC; };      // of element i
    float g[E], dg[E], db[E];
#pragma unroll
    for (int i = 0; i < E; i += 4) rows::load(gamma + column(i), C - column(i), g + i);
#pragma unroll
    for (int i = 0; i < E; ++i) dg[i] = db[i] = 0.f;
    const float inv = 1.f / C;
    struct Row { uint4 x[NV], d[NV], a[NV]; float2 s; };
    auto fetch = [&](long row) {
        Row r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int at = column(i * VEC);
            r.x[i] = rows::fetch(x + row * ldx + at, C - at);
            r.d[i] = rows::fetch(dy + row * lddy + at, C - at);
            if (add) r.a[i] = rows::fetch(add + row * ldadd + at, C - at);
        }
        r.s = make_float2(stats[2 * row], stats[2 * row + 1]);
        return r;
    };
    const long step = (long)gridDim.x * ROWS;
    long row = (long)blockIdx.x * ROWS + part;
    Row next;
    if (AHEAD) next = fetch(min(row, M - 1));
    int turn = 0;
    for (long first = (long)blockIdx.x * ROWS; first < M; first += step, row += step, turn ^= 1) {     // as often for every wavefront
        const Row now = AHEAD ? next : fetch(min(row, M - 1));
        const bool there = row < M;
        if (AHEAD && first + step < M) next = fetch(min(row + step, M - 1));
        float xh[E], d[E], s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            rows::convert<T>(now.x[i], xh + i * VEC);
            rows::convert<T>(now.d[i], d + i * VEC);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
            const bool in = column(i) < C;
            xh[i] = in ? (xh[i] - now.s.x) * now.s.y : 0.f;
            if (there) {
                dg[i] = fmaf(d[i], xh[i], dg[i]);
                db[i] += d[i];
            }
            d[i] = in ? d[i] * g[i] : 0.f;
            s[0] += d[i];
            s[1] = fmaf(d[i], xh[i], s[1]);
        }
        row_sums<WAVES>(s, lds[turn][part]);
        if (!there) continue;
        s[0] *= inv;
        s[1] *= inv;
#pragma unroll
        for (int i = 0; i < E; ++i) d[i] = now.s.y * (d[i] - s[0] - xh[i] * s[1]);
        if (add) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float a[VEC];
                rows::convert<T>(now.a[i], a);
#pragma unroll
                for (int e = 0; e < VEC; ++e) d[i * VEC + e] += a[e];
            }
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) rows::store(dx + row * lddx + column(i * VEC), C - column(i * VEC), d + i * VEC, past);
    }
    // the rows of the workgroup, one after the other
    if constexpr (ROWS > 1) {
        for (int r = 1; r < ROWS; ++r) {
            if (part == r)
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (column(i) < C) {
                        sums[column(i)] = dg[i];
                        sums[C + column(i)] = db[i];
                    }
            __syncthreads();
            if (part == 0)
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (column(i) < C) {
                        dg[i] += sums[column(i)];
                        db[i] += sums[C + column(i)];
                    }
            __syncthreads();
        }
        if (part) return;
    }
    float* og = dgamma + (long)blockIdx.x * 2 * C;
    float* ob = dbeta + (long)blockIdx.x * 2 * C;
#pragma unroll
    for (int i = 0; i < E; i += 4) {
        rows::store(og + column(i), C - column(i), dg + i);
        rows::store(ob + column(i), C - column(i), db + i);
    }
}

// G records of dgamma[C], dbeta[C] -> their sums, in the order of a fixed tree: 32 columns and 32 groups of records a workgroup.  In fp64: 64 additions one after the other
// in fp32 would cost more bits than all rows before them (42115 x 48: 2.0e-7 of the sums' norm).
__global__ __launch_bounds__(1024) void layernorm_sums_kernel(const float* __restrict__ records, float* __restrict__ dgamma, float* __restrict__ dbeta, int G, int C) {
    __shared__ double part[32][33];
    const int col = threadIdx.x & 31, group = threadIdx.x >> 5, at = blockIdx.x * 32 + col;
    double s = 0.;
    if (at < 2 * C)
#pragma unroll 8
        for (int r = group; r < G; r += 32) s += records[(long)r * 2 * C + at];
    part[group][col] = s;
    __syncthreads();
    if (group == 0 && at < 2 * C) {
        double t = 0.;
#pragma unroll
        for (int i = 0; i < 32; ++i) t += part[i][col];
        if (at < C) dgamma[at] = (float)t;
        else dbeta[at - C] = (float)t;
    }
}

__global__ void layernorm_zero_kernel(float* dgamma, float* dbeta, int C) {
    const int at = blockIdx.x * 256 + threadIdx.x;
    if (at < C) dgamma[at] = dbeta[at] = 0.f;
}

// Workgroups of the backward pass, each with a record of the columns' sums: four on a compute unit.
constexpr int RECORDS = 1024;
int rows_together(int C) { return C <= 512 ? 4 : C <= 1024 ? 2 : 1; }       // of a workgroup, backward
int records_of(int64_t M, int C) {
    const int64_t groups = (M + rows_together(C) - 1) / rows_together(C);
    return (int)(groups < RECORDS ? groups : RECORDS);
}

template <class T, int E, int WAVES, int ROWS>
void launch_fwd(hipStream_t s, const void* x, const float* gamma, const float* beta, void* y, float* stats, long ldx, long ldy, long M, int C, float eps) {
    const long most = most_blocks(64 * WAVES * ROWS) * ROWS;        // rows of a launch
    for (long at = 0; at < M; at += most) {
        const long n = M - at < most ? M - at : most;
        hipLaunchKernelGGL((layernorm_fwd_kernel<T, E, WAVES, ROWS>), dim3(ceil_div(n, ROWS)), dim3(64 * WAVES * ROWS), 0, s, (const T*)x + at * ldx, gamma, beta,
                           (T*)y + at * ldy, stats ? stats + 2 * at : nullptr, ldx, ldy, n, C, eps, rows::past_the_caches(M * C * (int64_t)sizeof(T)));
    }
}
template <class T, int E, int WAVES, int ROWS>
void launch_bwd(hipStream_t s, int G, const void* x, const float* gamma, const float* stats, const void* dy, const void* add, void* dx, float* dgamma,
                float* dbeta, long ldx, long lddy, long ldadd, long lddx, long M, int C) {
    hipLaunchKernelGGL((layernorm_bwd_kernel<T, E, WAVES, ROWS>), dim3(G), dim3(64 * WAVES * ROWS), ROWS > 1 ? 8 * C : 0, s, (const T*)x, gamma, stats,
                       (const T*)dy, (const T*)add, (T*)dx, dgamma, dbeta, ldx, lddy, ldadd, lddx, M, C, rows::past_the_caches(M * C * (int64_t)sizeof(T)));
}

// Elements a lane holds, wavefronts a row, rows a workgroup.
#define FORWARD(...)                                                     \
    if (C <= 512) launch_fwd<T, 8, 1, 4>(__VA_ARGS__);                   \
    else if (C <= 1024) launch_fwd<T, 16, 1, 4>(__VA_ARGS__);            \
    else if (C <= 2048) launch_fwd<T, 16, 2, 2>(__VA_ARGS__);            \
    else if (C <= 4096) launch_fwd<T, 16, 4, 1>(__VA_ARGS__);            \
    else if (C <= 8192) launch_fwd<T, 16, 8, 1>(__VA_ARGS__);            \
    else launch_fwd<T, 16, 16, 1>(__VA_ARGS__);
#define BACKWARD(...)                                                    \
    if (C <= 512) launch_bwd<T, 8, 1, 4>(__VA_ARGS__);                   \
    else if (C <= 1024) launch_bwd<T, 8, 2, 2>(__VA_ARGS__);             \
    else if (C <= 2048) launch_bwd<T, 8, 4, 1>(__VA_ARGS__);             \
    else if (C <= 4096) launch_bwd<T, 8, 8, 1>(__VA_ARGS__);             \
    else if (C <= 8192) launch_bwd<T, 8, 16, 1>(__VA_ARGS__);            \
    else launch_bwd<T, 16, 16, 1>(__VA_ARGS__);

bool bad(int type, int64_t M, int C) { return (type != DSSPK_F32 && type != DSSPK_BF16) || M < 0 || M > (1L << 30) || C < 1 || C > MAX_C; }

}  // namespace

extern "C" int dsspk_layernorm_fwd(void* stream, int type, const void* x, int64_t ldx, const float* gamma, const float* beta, void* y, int64_t ldy, float* stats,
                                   int64_t M, int C, float eps) {
    if (bad(type, M, C) || !x || !gamma || !beta || !y || ldx < C || ldy < C || (x == y && ldx != ldy) || !(eps >= 0.f) || ((uintptr_t)stats & 7)) return -1;
    if (M == 0) return 0;
    const hipStream_t s = (hipStream_t)stream;
    if (type == DSSPK_F32) { using T = float; FORWARD(s, x, gamma, beta, y, stats, ldx, ldy, M, C, eps) }
    else { using T = rows::bf16; FORWARD(s, x, gamma, beta, y, stats, ldx, ldy, M, C, eps) }
    return DSSPK_LAUNCH_RC();
}

extern "C" size_t dsspk_layernorm_bwd_scratch_floats(int64_t M, int C) {
    if (bad(DSSPK_F32, M, C)) return 0;
    const int G = records_of(M, C);
    return G > 1 ? (size_t)G * 2 * C : 0;
}

extern "C" int dsspk_layernorm_bwd(void* stream, int type, const void* x, int64_t ldx, const float* gamma, const float* stats, const void* dy, int64_t lddy,
                                   const void* add, int64_t ldadd, void* dx, int64_t lddx, float* dgamma, float* dbeta, float* scratch, int64_t M, int C) {
    if (bad(type, M, C) || !x || !gamma || !stats || !dy || !dx || !dgamma || !dbeta || ldx < C || lddy < C || lddx < C || (add && ldadd < C)) return -1;
    if (dx == x || (dx == dy && lddx != lddy) || (add && dx == add && lddx != ldadd)) return -1;
    const hipStream_t s = (hipStream_t)stream;
    if (M == 0) {
        hipLaunchKernelGGL(layernorm_zero_kernel, dim3(ceil_div(C, 256)), dim3(256), 0, s, dgamma, dbeta, C);
        return DSSPK_LAUNCH_RC();
    }
    const int G = records_of(M, C);
    if (G > 1 && (!scratch || ((uintptr_t)scratch & 15))) return -1;
    float *og = G > 1 ? scratch : dgamma, *ob = G > 1 ? scratch + C : dbeta;
    if (type == DSSPK_F32) { using T = float; BACKWARD(s, G, x, gamma, stats, dy, add, dx, og, ob, ldx, lddy, ldadd, lddx, M, C) }
    else { using T = rows::bf16; BACKWARD(s, G, x, gamma, stats, dy, add, dx, og, ob, ldx, lddy, ldadd, lddx, M, C) }
    if (const int rc = DSSPK_LAUNCH_RC()) return rc;
    if (G > 1) hipLaunchKernelGGL(layernorm_sums_kernel, dim3(ceil_div(2L * C, 32)), dim3(1024), 0, s, scratch, dgamma, dbeta, G, C);
    return DSSPK_LAUNCH_RC();
}
