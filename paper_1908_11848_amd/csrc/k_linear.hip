// The product of a layer with its epilogue, y = act(x W + b) + r, and its gradients dx = (dz W^T) act'(pre), dW = x^T dz, db = column sums of dz.
//
// All three products are tile_product.hpp's, with the operands as they are in memory: x and dz have the reduction index contiguous in the first two and the
// other index in the third, W the other way round.  fp32 operands are first written as three bf16 terms, and bf16 ones whose rows
// are not aligned to 16 bytes are copied (pack_kernel; rows padded with zeros to a multiple of 32 and 8).
// Where the tiles of a result are fewer than the chip takes at once, the reduction index is split over workgroups: partial sums in fp32, added up
// in order by a second kernel, which then does the epilogue.
//
// Measured (us): 16384 x 1024 -> 4096 bf16 with GELU and its input saved 157, a library product alone 124, the rest 268 MB of results, since all workgroups come to their epilogue together; its like
// backward, through the activation, 339 in all (134 MB read on top), of which dw in four parts is 132 + 15 and db 14; fp32, 4096 rows, 1024 and 2048 channels 201: dx and dw 94 to 98 each under the
// profiler, joining dw 7, terms 23, db 12.
#include <type_traits>

#include "activation.hpp"
#include "rows.hpp"
#include "tile_product.hpp"

namespace {

using rows::bf16;

// ---------------------------------------------------------------- operands

struct Pack {
    const void* from;
    char* to;
    long ld, rows;
    int cols, padded;       // columns, rounded up to 8 (bf16) or 32 (fp32)
    long first_block;
};
struct Packs { Pack p[3]; int count; long base; };      // base: blocks of the launches before

constexpr int PACK_THREADS = 256;
// a lane writes 8 elements of each plane
template <class T> __global__ __launch_bounds__(PACK_THREADS) void pack_kernel(Packs packs) {
    int j = 0;
    for (int i = 1; i < packs.count; ++i)
        if (packs.base + blockIdx.x >= packs.p[i].first_block) j = i;
    const Pack& p = packs.p[j];
    const long at = (packs.base + blockIdx.x - p.first_block) * PACK_THREADS + threadIdx.x;
    const int chunks = p.padded / 8;
    const long row = at / chunks;
    const int col = (int)(at - row * chunks) * 8;
    if (row >= p.rows) return;
    const T* from = (const T*)p.from + row * p.ld + col;
    float v[8];
    rows::load8(from, p.cols - col, v);
    if constexpr (sizeof(T) == 2) {
        rows::store((bf16*)(p.to + row * 2L * p.padded + 2L * col), 8, v);
    } else {
        uint2 lo[split::PLANES], hi[split::PLANES];
        split::split4(split::scaled(make_float4(v[0], v[1], v[2], v[3])), lo);
        split::split4(split::scaled(make_float4(v[4], v[5], v[6], v[7])), hi);
#pragma unroll
        for (int q = 0; q < split::PLANES; ++q)
            *reinterpret_cast<uint4*>(p.to + prod::terms_at(prod::terms_pitch(p.padded), row, col) + q * prod::TERM) = make_uint4(lo[q].x, lo[q].y, hi[q].x, hi[q].y);
    }
}

// ---------------------------------------------------------------- epilogues

struct Epilogue {
    const float* bias;
    const void* side;       // forward: the residual, added; backward: pre, the result is multiplied by act'(pre)
    void* out;
    void* z;
    long lds, ldo, ldz;
    int act;
    bool past;              // results go past the caches
};

// v: eight columns of a row, n of them in the result.  SLOPE: a gradient; T: type of side and z, O: of out.
template <bool SLOPE, class T, class O, int ACT>
__device__ __forceinline__ void finish(const Epilogue& e, long row, int col, int n, const float (&bias)[8], const rows::Raw8<T>& side, float (&v)[8]) {
    constexpr bool FINE = sizeof(T) == 4;
    float u[8];
    if constexpr (SLOPE) {
        if (ACT != DSSPK_ACT_NONE) {
            rows::convert8(side, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= act::slope<FINE>(ACT, u[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += bias[i];
        if (e.z) rows::store8((T*)e.z + row * e.ldz + col, n, v, e.past);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = act::value<FINE>(ACT, v[i]);
        if (e.side) {
            rows::convert8(side, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += u[i];
        }
    }
    rows::store8((O*)e.out + row * e.ldo + col, n, v, e.past);
}

// ---------------------------------------------------------------- products

struct Plain {              // an operand in fp32, for sums outside the range of the bf16 terms: element (i, k) at p[i s + k ks]
    const float* p;
    long s, ks;
};
struct Job {
    prod::Operand a, b;
    Plain fa, fb;
    int rows, cols, K;
    int tiles_i, tiles_j, parts, steps;     // steps: reduction tiles a part
    float* partial;                 // [parts][rows][cols], or null
    Epilogue e;
};

// A 16 x 16 tile whose sums are infinite or NaN, computed again on the fp32 matrix cores from the operands themselves.
// a, b: this lane's row and column, elements as, bs apart.
__device__ __noinline__ floatx4 again(const float* pa, const float* pb, long as, long bs, int k0, int k1) {
    const int q = (threadIdx.x & 63) >> 4;
    floatx4 s{0.f, 0.f, 0.f, 0.f};
    for (int k = k0; k < k1; k += 4) {
        const bool in = k + q < k1;
        const float a = in ? pa[(k + q) * as] : 0.f, b = in ? pb[(k + q) * bs] : 0.f;
        s = __builtin_amdgcn_mfma_f32_16x16x4f32(b, a, s, 0, 0, 0);
    }
    return s;
}

template <class S, bool A_KO, bool B_KO, bool SLOPE, class T, class O>
__global__ __launch_bounds__(S::THREADS) void product_kernel(Job j) {
    using Out = prod::Out<S>;
    __shared__ __attribute__((aligned(128))) char lds[S::LDS + (A_KO ? 0 : 16 * S::THREADS)];
    const prod::Place at = prod::place(blockIdx.x, j.tiles_i, j.tiles_j, j.parts);
    const int steps = (j.K + S::BK - 1) / S::BK, t0 = min(at.part * j.steps, steps), t1 = min(t0 + j.steps, steps);
    floatx4 sum[S::WM][S::WN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15;
    const int row0 = at.i * S::BM + wave / S::GN * 16 * S::WM, col0 = at.j * S::BN + wave % S::GN * 16 * S::WN;
    // What the epilogue will read is called into the caches during the last tiles, 64 x 16 bytes a tile and wavefront, by loads into a corner of LDS that nobody reads:
    // read only when the products are done, by everybody at once, it took as long as half of them.
    constexpr int SIDE_LANES = 16 * S::WN * (int)sizeof(T) / 16, SIDE_ROWS = 64 / SIDE_LANES;
    const bool has_side = j.e.side && !j.partial;
    const prod::intx4 side_buffer = prod::describe((const char*)((uintptr_t)((const char*)j.e.side + (row0 * j.e.lds + col0) * sizeof(T)) & ~(uintptr_t)15), has_side ? ((long)(j.rows - 1 - row0) * j.e.lds + j.cols - col0) * (long)sizeof(T) : 0);
    const unsigned side_at = (unsigned)((lane / SIDE_LANES * j.e.lds) * sizeof(T)) + 16u * (lane % SIDE_LANES);
    const unsigned side_to = prod::lds_address(lds) + S::LDS + wave * 1024;
    auto call = [&](int n) {
        prod::fetch16(side_buffer, n >= 0 && n < 16 * S::WM / SIDE_ROWS ? side_at + (unsigned)(n * SIDE_ROWS * j.e.lds * sizeof(T)) : split::OUTSIDE, side_to);
    };
    if constexpr (A_KO) prod::tile<S, A_KO, B_KO>(j.a, j.b, at.i * S::BM, at.j * S::BN, t0, t1, lds, sum);          // dw: its epilogue reads nothing
    else prod::tile<S, A_KO, B_KO>(j.a, j.b, at.i * S::BM, at.j * S::BN, t0, t1, lds, sum, prod::Something<decltype(call)>{call});
    char* region = lds + wave * Out::REGION;
    bool spoiled = false;
    if constexpr (S::PLANES == 3) {
        float bad = 0.f;
#pragma unroll
        for (int m = 0; m < S::WM; ++m)
#pragma unroll
            for (int n = 0; n < S::WN; ++n) {
                bad = split::spoil(sum[m][n], bad);
                sum[m][n] *= split::UNSCALE;
            }
        spoiled = split::spoiled(bad);
    }
    // Eight columns a lane, the same ones in all its rows.  What a row takes from memory is fetched for the whole round, before the sums go through LDS: one after the
    // other, these loads took twice as long as the products (232 us of the gradient of 16384 x 4096 x 1024).
    constexpr int LANES = Out::COLS / 8, STEP = 64 / LANES, ROUNDS = Out::ROWS / STEP;
    const int in = lane % LANES * 8, col = col0 + in, left = j.cols - col;
    float bias[8] = {};
    if (!SLOPE && j.e.bias && !j.partial && left > 0) rows::load8(j.e.bias + col, left, bias);
    auto round = [&](auto number) {
        constexpr int pass = decltype(number)::value;
        const int first = row0 + pass * Out::ROWS;
        rows::Raw8<T> side[ROUNDS];
        if (j.e.side && !j.partial)
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                const long row = first + i * STEP + lane / LANES;
                if (row < j.rows && left > 0) side[i] = rows::fetch8((const T*)j.e.side + row * j.e.lds + col, left);
            }
#pragma unroll
        for (int m = 0; m < Out::TILES; ++m)
#pragma unroll
            for (int n = 0; n < S::WN; ++n) Out::put(region, m, n, lane, sum[pass * Out::TILES + m][n]);
        if (S::PLANES == 3 && spoiled)
            for (int m = 0; m < Out::TILES; ++m)
                for (int n = 0; n < S::WN; ++n)
                    Out::put(region, m, n, lane, again(j.fa.p + min(first + 16 * m + l16, j.rows - 1) * j.fa.s, j.fb.p + min(col0 + 16 * n + l16, j.cols - 1) * j.fb.s,
                                                       j.fa.ks, j.fb.ks, t0 * S::BK, min(t1 * S::BK, j.K)));
        __builtin_amdgcn_wave_barrier();        // a wavefront's own region: its LDS accesses are in order
        if (j.partial) {
            for (int i = 0; i < ROUNDS; ++i) {
                const int r = i * STEP + lane / LANES;
                float v[8];
                Out::get(region, r, in, v);
                if (first + r < j.rows && left > 0) rows::store8(j.partial + ((long)at.part * j.rows + first + r) * j.cols + col, left, v);
            }
        } else {
            act::with(j.e.act, [&](auto which) {
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i) {
                    const int r = i * STEP + lane / LANES;
                    float v[8];
                    Out::get(region, r, in, v);
                    if (first + r < j.rows && left > 0) finish<SLOPE, T, O, decltype(which)::value>(j.e, first + r, col, left, bias, side[i], v);
                }
            });
        }
        __builtin_amdgcn_wave_barrier();
    };
    round(prod::Set<0>{});
    static_assert(Out::PASSES <= 2, "");
    if constexpr (Out::PASSES > 1) round(prod::Set<1>{});
}

// the partial sums of eight columns, in the order of the parts, and the epilogue
template <bool SLOPE, class T, class O> __global__ __launch_bounds__(256) void join_kernel(const float* __restrict__ partial, int parts, long rows, int cols, Epilogue e) {
    const int eights = (cols + 7) / 8;
    const long at = (long)blockIdx.x * 256 + threadIdx.x, row = at / eights;
    const int col = (int)(at - row * eights) * 8;
    if (row >= rows) return;
    float s[8] = {};
    const float* p = partial + row * cols + col;
    for (int i = 0; i < parts; ++i, p += rows * cols) {
        float v[8];
        rows::load8(p, cols - col, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += v[k];
    }
    const int n = cols - col;
    float bias[8] = {};
    rows::Raw8<T> side = {};
    if (!SLOPE && e.bias) rows::load8(e.bias + col, n, bias);
    if (e.side) side = rows::fetch8((const T*)e.side + row * e.lds + col, n);
    act::with(e.act, [&](auto which) { finish<SLOPE, T, O, decltype(which)::value>(e, row, col, n, bias, side, s); });
}

// Few rows (a token or a handful of them): bound by the weights' bytes, and by the time until the first of them are there.  No tiles: the wavefronts of a workgroup
// share the reduction index of LANES * 8 columns, each lane with eight columns of every row it meets, in fp32 from either type; x in LDS as fp32.  One launch, no partial sums in
// memory: 1024 -> 4096 channels of one token in bf16 7.2 + 3.6 us as tiles and their sums.
// Up to 8 rows; of fp32, whose tiles need the weights as terms first, 16 (1024 -> 4096, 9 rows: 12.6 us, 28 as tiles).  Weights of more than 32 million numbers in
// bf16 are better streamed by tiles (8192 -> 8192, one row: 41 us so, 34 as tiles; 1024 -> 16384: 9.4 and 14.2).
inline bool few(int type, int64_t M, int64_t N, int64_t K) { return type == DSSPK_F32 ? M <= 16 : M <= 8 && N * K <= 1L << 25; }
constexpr int few_threads(int M) { return M > 8 ? 512 : 1024; }
// Sums of N numbers over lanes S, S / 2 .. STOP apart.  Of two lanes each takes over half of what both have, as long as there are two sums left: N exchanges and
// not N log.  first: number of acc[0] among the N.
template <int N, int S, int STOP, int ALL> __device__ __forceinline__ void fold(float (&acc)[ALL], int lane, int& first) {
    if constexpr (S >= STOP && N > 1) {
        constexpr int H = N / 2;
        const bool upper = lane & S;
        first += upper ? H : 0;
#pragma unroll
        for (int i = 0; i < H; ++i) {
            const float give = upper ? acc[i] : acc[H + i], keep = upper ? acc[H + i] : acc[i];
            acc[i] = keep + __shfl_xor(give, S);
        }
        fold<H, S / 2, STOP>(acc, lane, first);
    } else if constexpr (S >= STOP) {
        acc[0] += __shfl_xor(acc[0], S);
        fold<1, S / 2, STOP>(acc, lane, first);
    }
}

template <class T, int M, int LANES>
__global__ __launch_bounds__(few_threads(M)) void few_rows_kernel(const T* __restrict__ x, const T* __restrict__ w, long ldx, int rows, int N, int K, Epilogue e) {
    constexpr int FEW_THREADS = few_threads(M), FEW_K = 16384 / M, WAVES = FEW_THREADS / 64, DEEP = 64 / LANES * WAVES, COLS = 8 * LANES;
    __shared__ float xs[M][FEW_K];
    __shared__ float part[WAVES][M][COLS];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, cl = lane % LANES, deep = wave * (64 / LANES) + lane / LANES;
    const int col0 = xcd_tile(blockIdx.x, gridDim.x) * COLS, col = col0 + 8 * cl, left = N - col;
    float acc[8 * M] = {};
    for (int k0 = 0; k0 < K; k0 += FEW_K) {
        const int ks = min(FEW_K, K - k0);
        if (k0) __syncthreads();
        for (int k = tid; k < ks; k += FEW_THREADS)
#pragma unroll
            for (int m = 0; m < M; ++m) xs[m][k] = m < rows ? (float)x[m * ldx + k0 + k] : 0.f;
        __syncthreads();
        if (left <= 0) continue;
        const T* at = w + (long)k0 * N + col;
#pragma unroll(M <= 2 ? 8 : 4)
        for (int k = deep; k < ks; k += DEEP) {
            float v[8];
            rows::convert8(rows::fetch8(at + (long)k * N, left), v);
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[8 * m + i] = fmaf(xs[m][k], v[i], acc[8 * m + i]);
        }
    }
    int first = 0;
    fold<8 * M, 32, LANES>(acc, lane, first);
    constexpr int HALVINGS = LANES == 8 ? 3 : LANES == 4 ? 4 : LANES == 2 ? 5 : 6, LEFT = 8 * M >> HALVINGS > 0 ? 8 * M >> HALVINGS : 1;
#pragma unroll
    for (int i = 0; i < LEFT; ++i) part[wave][(first + i) / 8][8 * cl + (first + i) % 8] = acc[i];      // (lanes with the same sum write the same)
    __syncthreads();
    const int row = tid / LANES;
    if (tid >= M * LANES || row >= rows || left <= 0) return;
    float v[8] = {}, bias[8] = {};
#pragma unroll 4
    for (int u = 0; u < WAVES; ++u)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += part[u][row][8 * cl + i];
    rows::Raw8<T> side = {};
    if (e.bias) rows::load8(e.bias + col, left, bias);
    if (e.side) side = rows::fetch8((const T*)e.side + row * e.lds + col, left);
    act::with(e.act, [&](auto which) { finish<false, T, T, decltype(which)::value>(e, row, col, left, bias, side, v); });
}

// Column sums: of slabs of rows, then of the slabs, in an order that the sizes alone decide.  A lane has eight columns, a workgroup 32 lanes of them and eight rows at a time.
constexpr int SLABS = 256;
template <class T> __global__ __launch_bounds__(256) void colsum_kernel(const T* __restrict__ x, long ld, float* __restrict__ out, long M, int N, int slabs) {
    __shared__ float part[8][32][9];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5, col = (blockIdx.x * 32 + lane) * 8, left = N - col;
    const long per = (M + slabs - 1) / slabs, r0 = blockIdx.y * per, r1 = min(r0 + per, M);
    float s[8] = {};
    if (left > 0)
#pragma unroll 4
        for (long r = r0 + group; r < r1; r += 8) {
            float v[8];
            rows::convert8(rows::fetch8(x + r * ld + col, left), v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += v[i];
        }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[group][lane][i] = s[i];
    __syncthreads();
    // one column a thread
    const int l = threadIdx.x >> 3, i = threadIdx.x & 7, c = (blockIdx.x * 32 + l) * 8 + i;
    if (c >= N) return;
    float t = 0.f;
#pragma unroll
    for (int g = 0; g < 8; ++g) t += part[g][l][i];
    out[(long)blockIdx.y * N + c] = t;
}
int slabs_of(int64_t M, int N) {            // some 1024 workgroups, 16 rows a slab at least
    const int64_t most = 1024 / ceil_div(N, 256), rows = M / 16;
    const int64_t n = most < rows ? most : rows;
    return n < 2 ? 1 : n > SLABS ? SLABS : (int)n;
}

__global__ __launch_bounds__(256) void zero_kernel(float* p, long n) {
    for (long at = (long)blockIdx.x * 256 + threadIdx.x; at < n; at += (long)gridDim.x * 256) p[at] = 0.f;
}

__global__ __launch_bounds__(256) void to_bf16_kernel(bf16* __restrict__ dst, const float* __restrict__ src, long n) {
    const long at = ((long)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    float v[8];
    const int left = (int)min(n - at, 8L);
    rows::load(src + at, left, v);
    rows::load(src + at + (left > 4 ? 4 : 0), left - 4, v + 4);
    rows::store(dst + at, left, v);
}

// ---------------------------------------------------------------- host

constexpr int64_t MAX_ROWS = 1L << 30;
constexpr int MAX_COLS = 1 << 20;
inline size_t round256(size_t v) { return (v + 255) & ~(size_t)255; }
inline int64_t padded(int type, int64_t cols) { return type == DSSPK_F32 ? (cols + 31) & ~31L : (cols + 7) & ~7L; }
inline size_t pack_bytes(int type, int64_t rows, int64_t cols) { return round256((type == DSSPK_F32 ? 6 : 2) * (size_t)(rows * padded(type, cols))); }

// Which tile, and in how many parts the reduction: whatever comes out fastest by these figures (us; measured on products of 4096 x 4096 x 4096 and 4096 x 1024 x 16384,
// all operand orders alike within 5 %): a step of BK indices with one workgroup on a compute unit and with all it holds, what a tile costs besides its steps, and partial
// sums that are written and read at 4 TB/s behind another launch.
struct Choice { int tile, parts; };
struct Cost { int bm, bn, bk, threads, fit; float alone, full, more; };
constexpr int TILES = 3;
constexpr Cost COSTS[2][TILES] = {{{128, 64, 32, 256, 2, 0.75f, 1.27f, 3.f}, {128, 128, 32, 512, 1, 0.88f, 1.11f, 3.f}, {64, 64, 32, 256, 1, 0.46f, 0.48f, 3.f}},      // fp32
                                  {{128, 128, 64, 256, 2, 0.68f, 0.99f, 3.f}, {256, 256, 64, 512, 1, 1.40f, 1.56f, 4.f}}};                                          // bf16 (none)
inline int64_t tiles_of(const Cost& c, int64_t rows, int64_t cols) { return ((rows + c.bm - 1) / c.bm) * ((cols + c.bn - 1) / c.bn); }
// whether there is a tile for a result of that size: one launch has all of its tiles
inline bool launchable(int type, int64_t rows, int64_t cols) {
    for (const Cost& c : COSTS[type == DSSPK_BF16])
        if (c.bm && tiles_of(c, rows, cols) <= most_blocks(c.threads)) return true;
    return false;
}
constexpr int CUS = 256, MAX_PARTS = 64;
Choice choose(int type, int64_t rows, int64_t cols, int64_t K) {
    Choice best = {0, 1};
    float least = 1e30f;
    for (int tile = 0; tile < TILES; ++tile) {
        const Cost& c = COSTS[type == DSSPK_BF16][tile];
        if (!c.bm) continue;
        const int64_t tiles = tiles_of(c, rows, cols), steps = (K + c.bk - 1) / c.bk;
        if (tiles > most_blocks(c.threads)) continue;
        // (what is split has few tiles: so many that their parts or their join would not fit a launch are never worth it)
        for (int parts = 1; parts <= MAX_PARTS && (parts == 1 || (steps / parts >= 4 && tiles * parts <= 1 << 20)); ++parts) {
            const int64_t n = tiles * parts, each = (steps + parts - 1) / parts, slots = (int64_t)CUS * c.fit;
            const int64_t full = n / slots, rest = n - full * slots;
            float t = full * (each * c.full + c.more);
            if (rest) t += each * (rest > CUS ? c.full : c.alone) + c.more;
            if (parts > 1) t += 4.f + 8.f * parts * rows * cols / 4e6f;
            if (t < least) {
                least = t;
                best = {tile, parts};
            }
        }
    }
    return best;
}
size_t partial_bytes(int type, int64_t rows, int64_t cols, int64_t K) {
    const int parts = choose(type, rows, cols, K).parts;
    return parts > 1 ? round256(4 * (size_t)(parts * rows * cols)) : 0;
}

inline size_t slab_bytes(int64_t M, int N) { return round256(4 * (size_t)slabs_of(M, N) * N); }

struct Matrix {             // an operand as given: rows x cols elements, ld
    const void* p;
    int64_t ld, rows;
    int cols;
};
struct Source {             // as the product takes it
    const char* p;
    long pitch;
    int64_t rows, cols;     // cols padded
    const float* f;
    int64_t ld;
};

inline bool direct(int type, const Matrix& m) { return type == DSSPK_BF16 && ((uintptr_t)m.p & 15) == 0 && m.ld % 8 == 0 && m.cols % 8 == 0; }

// packs the operands that need it, one launch
int pack(hipStream_t s, int type, int n, const Matrix* m, Source* out, char*& ws) {
    Packs packs = {};
    long blocks = 0;
    for (int i = 0; i < n; ++i) {
        out[i] = {(const char*)m[i].p, 2 * m[i].ld, m[i].rows, m[i].cols, (const float*)m[i].p, m[i].ld};
        if (direct(type, m[i])) continue;
        const int64_t cols = padded(type, m[i].cols);
        Pack& p = packs.p[packs.count++];
        p = {m[i].p, ws, m[i].ld, m[i].rows, m[i].cols, (int)cols, blocks};
        blocks += (m[i].rows * (cols / 8) + PACK_THREADS - 1) / PACK_THREADS;
        out[i].p = ws;
        out[i].pitch = type == DSSPK_F32 ? prod::terms_pitch(cols) : 2 * cols;
        out[i].cols = cols;
        ws += pack_bytes(type, m[i].rows, m[i].cols);
    }
    if (!packs.count) return 0;
    for (const long most = most_blocks(PACK_THREADS); packs.base < blocks; packs.base += most) {
        const dim3 grid(blocks - packs.base < most ? blocks - packs.base : most);
        if (type == DSSPK_F32) hipLaunchKernelGGL((pack_kernel<float>), grid, dim3(PACK_THREADS), 0, s, packs);
        else hipLaunchKernelGGL((pack_kernel<bf16>), grid, dim3(PACK_THREADS), 0, s, packs);
    }
    return DSSPK_LAUNCH_RC();
}

template <class S, bool A_KO, bool B_KO, bool SLOPE, class T, class O>
int launch(hipStream_t s, Job j, int parts, float* partial) {
    j.tiles_i = ceil_div(j.rows, S::BM);
    j.tiles_j = ceil_div(j.cols, S::BN);
    const int steps = ceil_div(j.K, S::BK);
    j.parts = parts;
    j.steps = ceil_div(steps, parts);
    j.partial = parts > 1 ? partial : nullptr;
    hipLaunchKernelGGL((product_kernel<S, A_KO, B_KO, SLOPE, T, O>), dim3(j.tiles_i * j.tiles_j * parts), dim3(S::THREADS), 0, s, j);
    if (parts > 1)
        hipLaunchKernelGGL((join_kernel<SLOPE, T, O>), dim3(ceil_div((long)j.rows * ((j.cols + 7) / 8), 256)), dim3(256), 0, s, j.partial, parts, (long)j.rows, j.cols, j.e);
    return DSSPK_LAUNCH_RC();
}

// C[rows][cols] = sum over K; KO: the operand's own rows are the reduction index
template <bool A_KO, bool B_KO>
int product(hipStream_t s, int type, const Source& a, const Source& b, int64_t rows, int cols, int64_t K, const Epilogue& e, char* partial) {
    auto operand = [](const Source& o, bool ko) {
        return ko ? prod::Operand{o.p, o.pitch, (int)o.cols, (int)o.rows} : prod::Operand{o.p, o.pitch, (int)o.rows, (int)o.cols};
    };
    auto plain = [](const Source& o, bool ko) { return ko ? Plain{o.f, 1, (long)o.ld} : Plain{o.f, (long)o.ld, 1}; };
    Job j = {};
    j.a = operand(a, A_KO);
    j.b = operand(b, B_KO);
    j.fa = plain(a, A_KO);
    j.fb = plain(b, B_KO);
    j.rows = (int)rows;
    j.cols = cols;
    j.K = (int)K;
    j.e = e;
    constexpr bool SLOPE = !(B_KO && !A_KO);            // both gradients; the forward product alone has KC rows and KO columns
    using O = std::conditional_t<A_KO, float, bf16>;    // dw is fp32
    const Choice c = choose(type, rows, cols, K);
    float* p = (float*)partial;
    if (type == DSSPK_F32) return c.tile == 2 ? launch<prod::Shape<3, 64, 64, 32, 2, 2, 4>, A_KO, B_KO, SLOPE, float, float>(s, j, c.parts, p)
                                : c.tile == 1 ? launch<prod::Shape<3, 128, 128, 32, 2, 4>, A_KO, B_KO, SLOPE, float, float>(s, j, c.parts, p)
                                              : launch<prod::Shape<3, 128, 64, 32, 2, 2>, A_KO, B_KO, SLOPE, float, float>(s, j, c.parts, p);
    return c.tile ? launch<prod::Shape<1, 256, 256, 64, 2, 4>, A_KO, B_KO, SLOPE, bf16, O>(s, j, c.parts, p)
                  : launch<prod::Shape<1, 128, 128, 64, 2, 2>, A_KO, B_KO, SLOPE, bf16, O>(s, j, c.parts, p);
}

// 8 to 64 columns a workgroup, as many as leave most compute units one
template <class T, int M> int few_rows(hipStream_t s, const void* x, int64_t ldx, const void* w, int rows, int N, int K, const Epilogue& e) {
    auto launch = [&](auto lanes) {
        constexpr int LANES = decltype(lanes)::value;
        hipLaunchKernelGGL((few_rows_kernel<T, M, LANES>), dim3(ceil_div(N, 8 * LANES)), dim3(few_threads(M)), 0, s, (const T*)x, (const T*)w, (long)ldx, rows, N, K, e);
    };
    constexpr int MOST = CUS * 3 / 4;
    if (N >= 64 * MOST) launch(prod::Set<8>{});
    else if (N >= 32 * MOST) launch(prod::Set<4>{});
    else if (N >= 16 * MOST) launch(prod::Set<2>{});
    else launch(prod::Set<1>{});
    return DSSPK_LAUNCH_RC();
}
template <class T> int few_rows(hipStream_t s, const void* x, int64_t ldx, const void* w, int rows, int N, int K, const Epilogue& e) {
    return rows <= 1 ? few_rows<T, 1>(s, x, ldx, w, rows, N, K, e) : rows <= 2 ? few_rows<T, 2>(s, x, ldx, w, rows, N, K, e)
         : rows <= 4 ? few_rows<T, 4>(s, x, ldx, w, rows, N, K, e) : few_rows<T, 8>(s, x, ldx, w, rows, N, K, e);
}

bool bad(int type, int64_t M, int N, int K) {
    return (type != DSSPK_F32 && type != DSSPK_BF16) || M < 0 || M > MAX_ROWS || N < 1 || K < 1 || N > MAX_COLS || K > MAX_COLS;
}
// a tile's rows times the pitch have to fit 31 bits
inline bool wide(int64_t ld) { return ld > 1L << 21; }

}  // namespace

extern "C" size_t dsspk_linear_fwd_workspace_bytes(int type, int64_t M, int N, int K) {
    if (bad(type, M, N, K)) return 0;
    if (few(type, M, N, K)) return 256;
    return pack_bytes(type, M, K) + pack_bytes(type, K, N) + partial_bytes(type, M, N, K) + 256;
}

extern "C" int dsspk_linear_fwd(void* stream, int type, const void* x, int64_t ldx, const void* w, const float* bias, int act, const void* residual, int64_t ldr,
                                void* y, int64_t ldy, void* z, int64_t ldz, int64_t M, int N, int K, void* workspace, size_t workspace_bytes) {
    if (bad(type, M, N, K) || !x || !w || !y || ldx < K || ldy < N || (residual && ldr < N) || (z && ldz < N) || act < DSSPK_ACT_NONE || act > DSSPK_ACT_SILU) return -1;
    if (y == x || z == x || y == w || (z && z == y) || (residual == y && ldr != ldy) || (z && z == residual)) return -1;
    if (wide(ldx) || (residual && wide(ldr)) || !launchable(type, M, N)) return -1;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < dsspk_linear_fwd_workspace_bytes(type, M, N, K)) return -1;
    if (M == 0) return 0;
    const hipStream_t s = (hipStream_t)stream;
    Epilogue e = {};
    e.bias = bias;
    e.side = residual;
    e.out = y;
    e.z = z;
    e.lds = ldr;
    e.ldo = ldy;
    e.ldz = ldz;
    e.act = act;
    e.past = rows::past_the_caches(M * N * (type == DSSPK_F32 ? 4 : 2));
    if (few(type, M, N, K))
        return type == DSSPK_BF16 ? few_rows<bf16>(s, x, ldx, w, (int)M, N, K, e)
             : M > 8 ? few_rows<float, 16>(s, x, ldx, w, (int)M, N, K, e) : few_rows<float>(s, x, ldx, w, (int)M, N, K, e);
    char* ws = (char*)workspace;
    const Matrix m[2] = {{x, ldx, M, K}, {w, N, K, N}};
    Source o[2];
    if (const int rc = pack(s, type, 2, m, o, ws)) return rc;
    return product<false, true>(s, type, o[0], o[1], M, N, K, e, ws);
}

extern "C" size_t dsspk_linear_bwd_workspace_bytes(int type, int64_t M, int N, int K) {
    if (bad(type, M, N, K)) return 0;
    const size_t dx = partial_bytes(type, M, K, N), dw = M ? partial_bytes(type, K, N, M) : 0;
    return pack_bytes(type, M, K) + pack_bytes(type, K, N) + pack_bytes(type, M, N) + (dx > dw ? dx : dw) + slab_bytes(M, N) + 256;
}

extern "C" int dsspk_linear_bwd(void* stream, int type, const void* x, int64_t ldx, const void* w, const void* dz, int64_t lddz, void* dx, int64_t lddx,
                                const void* pre, int64_t ldpre, int act, float* dw, float* db, int64_t M, int N, int K, void* workspace, size_t workspace_bytes) {
    if (bad(type, M, N, K) || !dz || lddz < N || (dw && (!x || ldx < K)) || (dx && (!w || lddx < K)) || (pre && (!dx || ldpre < K))) return -1;
    if (act < DSSPK_ACT_NONE || act > DSSPK_ACT_SILU || (!dx && !dw && !db)) return -1;
    if ((dx && (dx == dz || dx == x || dx == w || dx == pre)) || wide(lddz) || (dw && wide(ldx)) || (pre && wide(ldpre)) || (dx && !launchable(type, M, K)) || (dw && !launchable(type, K, N))) return -1;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < dsspk_linear_bwd_workspace_bytes(type, M, N, K)) return -1;
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;
    float* slabs = (float*)ws;
    ws += slab_bytes(M, N);
    if (db) {
        const int n = slabs_of(M, N);
        const dim3 grid(ceil_div(N, 256), n);
        float* to = n > 1 ? slabs : db;
        if (type == DSSPK_F32) hipLaunchKernelGGL((colsum_kernel<float>), grid, dim3(256), 0, s, (const float*)dz, lddz, to, M, N, n);
        else hipLaunchKernelGGL((colsum_kernel<bf16>), grid, dim3(256), 0, s, (const bf16*)dz, lddz, to, M, N, n);
        if (n > 1) hipLaunchKernelGGL((colsum_kernel<float>), dim3(ceil_div(N, 256), 1), dim3(256), 0, s, slabs, (long)N, db, (long)n, N, 1);
        if (const int rc = DSSPK_LAUNCH_RC()) return rc;
    }
    if (M == 0 && dw) {
        const long n = (long)K * N, blocks = (n + 255) / 256, most = most_blocks(256);
        hipLaunchKernelGGL(zero_kernel, dim3(blocks < most ? blocks : most), dim3(256), 0, s, dw, n);
        return DSSPK_LAUNCH_RC();
    }
    if (M == 0 || (!dx && !dw)) return 0;
    const Matrix m[3] = {{dz, lddz, M, N}, {dx ? w : x, dx ? N : ldx, dx ? K : M, dx ? N : K}, {x, ldx, M, K}};
    Source o[3];
    const int both = dx && dw;
    if (const int rc = pack(s, type, 2 + both, m, o, ws)) return rc;
    const Source &odz = o[0], &ow = o[1], &ox = o[both ? 2 : 1];
    if (dx) {
        Epilogue e = {};
        e.side = act != DSSPK_ACT_NONE ? pre : nullptr;
        e.out = dx;
        e.lds = ldpre;
        e.ldo = lddx;
        e.past = rows::past_the_caches(M * K * (type == DSSPK_F32 ? 4 : 2));
        e.act = e.side ? act : DSSPK_ACT_NONE;
        if (const int rc = product<false, false>(s, type, odz, ow, M, K, N, e, ws)) return rc;
    }
    if (dw) {
        Epilogue e = {};
        e.out = dw;
        e.ldo = N;
        return product<true, true>(s, type, ox, odz, K, N, M, e, ws);
    }
    return 0;
}

extern "C" int dsspk_linear_form(int type, int64_t rows, int64_t cols, int64_t K, int* tile_rows, int* tile_cols, int* parts) {
    if ((type != DSSPK_F32 && type != DSSPK_BF16) || rows < 1 || cols < 1 || K < 1 || rows > MAX_ROWS || cols > MAX_ROWS || K > MAX_ROWS || !tile_rows || !tile_cols || !parts) return -1;
    if (!launchable(type, rows, cols)) return -1;
    const Choice c = choose(type, rows, cols, K);
    *tile_rows = COSTS[type == DSSPK_BF16][c.tile].bm;
    *tile_cols = COSTS[type == DSSPK_BF16][c.tile].bn;
    *parts = c.parts;
    return 0;
}

extern "C" int dsspk_to_bf16(void* stream, void* dst, const float* src, int64_t n) {
    if (!dst || (!src && n) || n < 0 || (const void*)dst == (const void*)src || n > (1L << 40)) return -1;
    if (n == 0) return 0;
    const int64_t most = most_blocks(256) * 2048;        // of a launch
    for (int64_t at = 0; at < n; at += most) {
        const int64_t m = n - at < most ? n - at : most;
        hipLaunchKernelGGL(to_bf16_kernel, dim3(ceil_div(m, 2048)), dim3(256), 0, (hipStream_t)stream, (bf16*)dst + at, src + at, (long)m);
    }
    return DSSPK_LAUNCH_RC();
}
