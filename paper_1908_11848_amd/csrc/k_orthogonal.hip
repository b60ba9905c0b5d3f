// Server step 2 with an orthogonalised update: momentum, then for every matrix of the flat vector the Newton-Schulz products that drive its singular values
// towards one, then the step.
//
//   X = u / (|u| + eps);  A = X X^T,  B = a I + b A + c A A,  X <- B X  (X: the shorter side first, n x m)
//
// All matrices of a call go through every launch together (a workgroup finds its matrix by its number), as three bf16 terms a number in the workspace: the
// products are tile_product.hpp's, and every epilogue writes the terms that the next product reads, so that no operand is split twice.  A and B
// are symmetric: their tiles on and below the diagonal are computed, and written a second time with rows and columns exchanged.
// Work per matrix and step: n^2 m + n^3 + 2 n^2 m multiplications and additions, six times that in bf16.
//
// Matrices with a short side of at most DSSPK_ORTHOGONAL_SMALL go through a step in one launch: a workgroup holds a stretch of X in LDS, works out B for itself from the
// partial sums of A that all stretches left behind, multiplies, and leaves its own share of the next A.
//
// Measured (us a call, 5 steps): four matrices of 1024 x 4096 and four of 4096 x 1024 3340 to 3400 (a step: A 199 + 16, B 62 + 23, X 361; X at 1.14 PFLOP/s in bf16), ResNet-110's 109 filters 101 (a
// launch a step: 15.5), AlexNet-style 395: 3136 x 384 and 384 x 192 in launches of 11 to 14 that few compute units have a part in.
#include "rows.hpp"
#include "tile_product.hpp"
#include "../../include/dssp_kernels.h"

namespace {

constexpr float QA = 3.4445f, QB = -4.7750f, QC = 2.0315f;
constexpr int GROUP = 128;          // matrices of a launch (3.6 KB of arguments): two a lane when a workgroup looks for its own
constexpr int CHUNK = 4096;         // entries a workgroup takes of a matrix's momentum,
constexpr int GAP_CHUNK = 512;      // and of what lies between matrices, which is little (4096: 16 us for three dozen vectors)
using Shape = prod::Shape<3, 128, 128, 32, 2, 4>;
using Out = prod::Out<Shape>;
using Half = prod::Shape<3, 128, 64, 32, 2, 2>;      // two of these on a compute unit

struct Matrix {
    int64_t offset, ws;             // in the flat vector (elements), in the workspace (bytes)
    int rows, cols;
};
struct Group {
    int count;
    int first[GROUP];               // workgroup with which a matrix begins
    Matrix m[GROUP];
};

__host__ __device__ inline long align256(long v) { return (v + 255) & ~255L; }

// A matrix's part of the workspace: sums of squares of its chunks, u, two X, A, B.
struct Room {
    long n, m, np, mp, chunks;      // short and long side, rounded up to 32
    long u, x0, x1, a, b, end;
    __host__ __device__ Room(int rows, int cols) {
        n = rows < cols ? rows : cols;
        m = rows < cols ? cols : rows;
        np = (n + 31) & ~31L;
        mp = (m + 31) & ~31L;
        chunks = ((long)rows * cols + CHUNK - 1) / CHUNK;
        u = align256(8 * chunks);
        x0 = u + align256(4 * (long)rows * cols);
        x1 = x0 + align256(6 * n * mp);
        a = x1 + align256(6 * n * mp);
        b = a + align256(6 * n * np);
        end = b + align256(6 * n * np);
    }
    __device__ __forceinline__ long x(int which) const { return which ? x1 : x0; }
};

// which of the stretches of workgroups that begin at first[0 .. count - 1] this one is in
__device__ __forceinline__ int stretch_with(const int* first, int count, int block) {
    static_assert(GROUP == 128, "");
    const int lane = threadIdx.x & 63;
    const uint64_t lo = __ballot(lane < count && block >= first[lane]), hi = __ballot(64 + lane < count && block >= first[64 + lane]);
    return __builtin_amdgcn_readfirstlane(__popcll(lo) + __popcll(hi) - 1);
}
// The matrix of this workgroup, and the workgroup's number within it.  Neighbours go to one XCD: the tiles of a product read the same rows, which then come over
// the fabric once and not eight times (four matrices of 1024 x 4096 and four of 4096 x 1024: 4.2 ms a call without that).
template <bool TOGETHER = true> __device__ __forceinline__ int find(const Group& g, int& block) {
    const int mine = TOGETHER ? xcd_tile(blockIdx.x, gridDim.x) : blockIdx.x, at = stretch_with(g.first, g.count, mine);
    block = mine - g.first[at];
    return at;
}

// ---------------------------------------------------------------- momentum

struct Gaps {                       // stretches of the vector between matrices
    int count;
    int first[GROUP];
    int64_t from[GROUP], to[GROUP];
};

__device__ __forceinline__ float momentum_of(float m, float g, float mu) { return fmaf(mu, m, g); }

template <bool NESTEROV>
__global__ __launch_bounds__(256) void momentum_gaps_kernel(Gaps gaps, const float* w, float* w_out, const float* m, float* m_out, const float* __restrict__ g,
                                                            float mu, float scale) {
    const int at = stretch_with(gaps.first, gaps.count, blockIdx.x);
    const int64_t from = gaps.from[at] + (int64_t)(blockIdx.x - gaps.first[at]) * GAP_CHUNK, to = min(from + GAP_CHUNK, gaps.to[at]);
    for (int64_t i = from + threadIdx.x; i < to; i += 256) {
        const float gi = g[i], mi = momentum_of(m[i], gi, mu), u = NESTEROV ? fmaf(mu, mi, gi) : mi;
        m_out[i] = mi;
        w_out[i] = fmaf(-scale, u, w[i]);
    }
}

// u of the matrices, and the sum of squares of every chunk (squares and sums in fp64: they neither overflow nor vanish)
template <bool NESTEROV>
__global__ __launch_bounds__(256) void momentum_kernel(Group grp, char* ws, const float* m, float* m_out, const float* __restrict__ g, float mu) {
    __shared__ double part[4];
    int block;
    const Matrix mat = grp.m[find(grp, block)];
    const Room room(mat.rows, mat.cols);
    const long n = (long)mat.rows * mat.cols, from = (long)block * CHUNK, to = min(from + CHUNK, n);
    float* u = (float*)(ws + mat.ws + room.u);
    double s = 0.;
    for (long i = from + threadIdx.x; i < to; i += 256) {
        const float gi = g[mat.offset + i], mi = momentum_of(m[mat.offset + i], gi, mu), ui = NESTEROV ? fmaf(mu, mi, gi) : mi;
        m_out[mat.offset + i] = mi;
        u[i] = ui;
        s += (double)ui * ui;
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) ((double*)(ws + mat.ws))[block] = (part[0] + part[1]) + (part[2] + part[3]);
}

// ---------------------------------------------------------------- terms

// eight entries of a row, the first of them at `to`
__device__ __forceinline__ void write_terms(char* to, const float (&v)[8]) {
    uint2 lo[split::PLANES], hi[split::PLANES];
    split::split4(make_float4(v[0], v[1], v[2], v[3]), lo);
    split::split4(make_float4(v[4], v[5], v[6], v[7]), hi);
#pragma unroll
    for (int p = 0; p < split::PLANES; ++p) *reinterpret_cast<uint4*>(to + p * prod::TERM) = make_uint4(lo[p].x, lo[p].y, hi[p].x, hi[p].y);
}
__device__ __forceinline__ void write_term(char* to, float v) {
    float nothing = 0.f;
#pragma unroll
    for (int p = 0; p < split::PLANES; ++p) *reinterpret_cast<unsigned short*>(to + p * prod::TERM) = (unsigned short)split::take(v, nothing);
}
struct Terms { rows::Raw8<rows::bf16> v[split::PLANES]; };
__device__ __forceinline__ Terms fetch_terms(const char* from) {
    Terms t;
#pragma unroll
    for (int p = 0; p < split::PLANES; ++p) t.v[p] = rows::fetch8((const rows::bf16*)(from + p * prod::TERM), 8);
    return t;
}
__device__ __forceinline__ void add_up(const Terms& t, float (&v)[8]) {
    float u[8];
    rows::convert8(t.v[2], v);
#pragma unroll
    for (int p = 1; p >= 0; --p) {              // the small ones first: their sum is exact
        rows::convert8(t.v[p], u);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += u[i];
    }
}

// What u is divided by, |u| + eps, and is multiplied by first: a norm may be too large for fp32 where no entry is, and both are taken 2^-32 times then.
struct Norm {
    float by, norm;
    __device__ __forceinline__ Norm() = default;
    __device__ __forceinline__ Norm(double squares, float eps) {
        const double d = sqrt(squares) + (double)eps;
        by = d > 0x1p126 ? 0x1p-32f : 1.f;
        norm = (float)(d * (double)by);
    }
    __device__ __forceinline__ float operator()(float u) const { return u * by / norm; }
};

// X = u / (|u| + eps) as terms, the shorter side first; 64 x 64 entries a workgroup
__global__ __launch_bounds__(256) void normalise_kernel(Group grp, char* ws, float eps) {
    __shared__ float tile[64][65];
    __shared__ double part[4];
    int block;
    const Matrix mat = grp.m[find(grp, block)];
    const Room room(mat.rows, mat.cols);
    char* base = ws + mat.ws;
    double s = 0.;
    for (long i = threadIdx.x; i < room.chunks; i += 256) s += ((const double*)base)[i];
#pragma unroll
    for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    const int across = (mat.cols + 63) / 64, r0 = block / across * 64, c0 = block % across * 64;
    const float* u = (const float*)(base + room.u);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int r = wave; r < 64; r += 4) tile[r][lane] = r0 + r < mat.rows && c0 + lane < mat.cols ? u[(long)(r0 + r) * mat.cols + c0 + lane] : 0.f;
    __syncthreads();
    const Norm norm((part[0] + part[1]) + (part[2] + part[3]), eps);
    const bool turned = mat.rows > mat.cols;
    const int i0 = turned ? c0 : r0, j0 = turned ? r0 : c0;         // of X
    for (int t = threadIdx.x; t < 64 * 8; t += 256) {
        const int i = t >> 3, j = (t & 7) * 8;
        if (i0 + i >= room.n || j0 + j >= room.mp) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = norm(turned ? tile[j + e][i] : tile[i][j + e]);
        write_terms(base + room.x0 + prod::terms_at(prod::terms_pitch(room.mp), i0 + i, j0 + j), v);
    }
}

// ---------------------------------------------------------------- products

// tiles of a symmetric result that reach the diagonal or lie below it, row of tiles by row of tiles
__host__ __device__ inline int tiles_of_row(int i, int tiles_j) {
    const int t = ((i + 1) * Shape::BM + Shape::BN - 1) / Shape::BN;
    return t < tiles_j ? t : tiles_j;
}
__host__ inline int64_t lower_tiles(int n) {
    int64_t t = 0;
    for (int i = 0; i < ceil_div(n, Shape::BM); ++i) t += tiles_of_row(i, ceil_div(n, Shape::BN));
    return t;
}

// A = X X^T (POLY false) or B = a I + b A + c A A (A is symmetric: A A^T).
//
// Tiles are few and their reductions long and of any length, so the steps of all tiles of all matrices, one after the other, are cut into equal shares, one a
// workgroup: a share begins and ends inside a tile.  What a workgroup has of a tile that it shares goes to the workspace, and join_kernel adds that up in order.
struct Shares { int steps, groups; };       // steps of a workgroup, workgroups
struct Tile { int at, steps, i0, j0; };     // its first step, how many
template <bool POLY> __host__ __device__ inline int steps_of(const Room& room) { return (int)((POLY ? room.np : room.mp) / Shape::BK); }
// the tile of matrix `mat` that step `at` (counted from the matrix's first) belongs to
template <bool POLY> __device__ __forceinline__ Tile tile_at(const Room& room, int at) {
    const int steps = steps_of<POLY>(room), tiles_j = ((int)room.n + Shape::BN - 1) / Shape::BN;
    int block = at / steps, ti = 0;
    const int first = block * steps;
    while (block >= tiles_of_row(ti, tiles_j)) block -= tiles_of_row(ti++, tiles_j);
    return {first, steps, ti * Shape::BM, block * Shape::BN};
}
constexpr int WAVE_FLOATS = 16 * Shape::WM * 16 * Shape::WN, TILE_FLOATS = Shape::BM * Shape::BN;

template <bool POLY>
__device__ __forceinline__ void symmetric_finish(const Room& room, char* base, const floatx4 (&sum)[Shape::WM][Shape::WN], int row0, int col0, int lane, char* region) {
    const int n = (int)room.n;
    const long pitch = prod::terms_pitch(room.np);
    char* to = base + (POLY ? room.b : room.a);
    // rows as they are, up to the diagonal, and columns as rows, from behind the diagonal to the end of the padding
    constexpr int ROUNDS = Out::ROWS * Out::COLS / 8 / 64;
    auto direct = [&](int i, int& r, int& c) {
        const int t = 64 * i + lane;
        r = t / (Out::COLS / 8);
        c = t % (Out::COLS / 8) * 8;
        return row0 + r < n && col0 + c <= row0 + r;
    };
    auto mirror = [&](int i, int& r, int& c) {
        const int t = 64 * i + lane;
        c = t / (Out::ROWS / 8);
        r = t % (Out::ROWS / 8) * 8;
        return col0 + c < n && row0 + r < room.np && row0 + r + 7 > col0 + c;
    };
#pragma unroll
    for (int m = 0; m < Shape::WM; ++m)
#pragma unroll
        for (int k = 0; k < Shape::WN; ++k) Out::put(region, m, k, lane, sum[m][k]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        int r, c;
        float v[8], x[8];
        if (direct(i, r, c)) {
            const int row = row0 + r, col = col0 + c;
            Out::get(region, r, c, v);
            if constexpr (POLY) {
                add_up(fetch_terms(base + room.a + prod::terms_at(pitch, row, col)), x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(QB, x[e], fmaf(QC, v[e], col + e == row ? QA : 0.f));
            }
            char* at = to + prod::terms_at(pitch, row, col);
            if (col + 7 <= row) write_terms(at, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (col + e <= row) write_term(at + 2 * e, v[e]);
        }
    }
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        int r, c;
        float v[8], x[8];
        if (mirror(i, r, c)) {
            const int row = row0 + r, col = col0 + c;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = *reinterpret_cast<const float*>(region + Out::at(r + e, c / 4) + 4 * (c & 3));
            if constexpr (POLY) {
                add_up(fetch_terms(base + room.a + prod::terms_at(pitch, col, row)), x);
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = fmaf(QB, x[e], QC * v[e]);
            }
            char* at = to + prod::terms_at(pitch, col, row);
            if (row > col) write_terms(at, v);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (row + e > col) write_term(at + 2 * e, v[e]);
        }
    }
}

template <bool POLY> __global__ __launch_bounds__(Shape::THREADS) void symmetric_kernel(Group grp, char* ws, float* partial, Shares shares, int total, int from) {
    __shared__ __attribute__((aligned(128))) char lds[Shape::LDS];
    static_assert(Out::PASSES == 1, "");
    const int me = xcd_tile(blockIdx.x, gridDim.x), begin = me * shares.steps, end = min(begin + shares.steps, total);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    char* region = lds + wave * Out::REGION;
    for (int at = begin; at < end;) {
        const int which = stretch_with(grp.first, grp.count, at);
        const Matrix mat = grp.m[which];
        const Room room(mat.rows, mat.cols);
        char* base = ws + mat.ws;
        const Tile tile = tile_at<POLY>(room, at - grp.first[which]);
        const int t0 = at - grp.first[which] - tile.at, t1 = min(tile.steps, t0 + end - at);
        const prod::Operand o = POLY ? prod::Operand{base + room.a, prod::terms_pitch(room.np), (int)room.n, (int)room.np}
                                     : prod::Operand{base + room.x(from), prod::terms_pitch(room.mp), (int)room.n, (int)room.mp};
        floatx4 sum[Shape::WM][Shape::WN];
        prod::tile<Shape, false, false>(o, o, tile.i0, tile.j0, t0, t1, lds, sum);
        if (t1 - t0 == tile.steps) {
            symmetric_finish<POLY>(room, base, sum, tile.i0 + wave / Shape::GN * 16 * Shape::WM, tile.j0 + wave % Shape::GN * 16 * Shape::WN, lane, region);
        } else {
            float* p = partial + (2L * me + (at > begin)) * TILE_FLOATS + wave * WAVE_FLOATS;
#pragma unroll
            for (int m = 0; m < Shape::WM; ++m)
#pragma unroll
                for (int k = 0; k < Shape::WN; ++k) *reinterpret_cast<floatx4*>(p + ((m * Shape::WN + k) * 64 + lane) * 4) = sum[m][k];
        }
        at += t1 - t0;
        __syncthreads();                // the regions are free
    }
}

// the tiles that several workgroups share: a wavefront's part a workgroup.  first: tiles in front of each matrix.
template <bool POLY> __global__ __launch_bounds__(64) void join_kernel(Group grp, char* ws, const float* partial, Shares shares) {
    __shared__ __attribute__((aligned(128))) char region[Out::REGION];
    constexpr int WAVES = Shape::GM * Shape::GN;
    const int number = blockIdx.x / WAVES, wave = blockIdx.x % WAVES, which = stretch_with(grp.first, grp.count, number), lane = threadIdx.x;
    const Matrix mat = grp.m[which];
    const Room room(mat.rows, mat.cols);
    int before = 0;                     // steps of the matrices in front
    for (int i = 0; i < which; ++i) before += (grp.first[i + 1] - grp.first[i]) * steps_of<POLY>(Room(grp.m[i].rows, grp.m[i].cols));
    const int steps = steps_of<POLY>(room);
    const Tile tile = tile_at<POLY>(room, (number - grp.first[which]) * steps);
    const int at = before + tile.at, w0 = at / shares.steps, w1 = (at + steps - 1) / shares.steps;
    if (w0 == w1) return;               // had it to itself
    floatx4 sum[Shape::WM][Shape::WN];
#pragma unroll
    for (int m = 0; m < Shape::WM; ++m)
#pragma unroll
        for (int k = 0; k < Shape::WN; ++k) sum[m][k] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int w = w0; w <= w1; ++w) {
        const float* p = partial + (2L * w + (w * shares.steps < at)) * TILE_FLOATS + wave * WAVE_FLOATS;
#pragma unroll
        for (int m = 0; m < Shape::WM; ++m)
#pragma unroll
            for (int k = 0; k < Shape::WN; ++k) sum[m][k] += *reinterpret_cast<const floatx4*>(p + ((m * Shape::WN + k) * 64 + lane) * 4);
    }
    symmetric_finish<POLY>(room, ws + mat.ws, sum, tile.i0 + wave / Shape::GN * 16 * Shape::WM, tile.j0 + wave % Shape::GN * 16 * Shape::WN, lane, region);
}

// X' = B X; the last one goes into the weights
template <class S, bool LAST>
__global__ __launch_bounds__(S::THREADS) void update_kernel(Group grp, char* ws, int from, const float* w, float* w_out, float scale) {
    using Out = prod::Out<S>;
    __shared__ __attribute__((aligned(128))) char lds[S::LDS];
    int block;
    const Matrix mat = grp.m[find(grp, block)];
    const Room room(mat.rows, mat.cols);
    char* base = ws + mat.ws;
    const int n = (int)room.n, mp = (int)room.mp, tiles_i = (n + S::BM - 1) / S::BM;
    const int i0 = block % tiles_i * S::BM, j0 = block / tiles_i * S::BN;
    const long pitch = prod::terms_pitch(mp);
    const char* x = base + room.x(from);
    const prod::Operand ob{base + room.b, prod::terms_pitch(room.np), n, (int)room.np}, ox{x, pitch, mp, n};
    floatx4 sum[S::WM][S::WN];
    prod::tile<S, false, true>(ob, ox, i0, j0, 0, (n + S::BK - 1) / S::BK, lds, sum);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row0 = i0 + wave / S::GN * 16 * S::WM, col0 = j0 + wave % S::GN * 16 * S::WN;
    char* region = lds + wave * Out::REGION;
    const bool turned = mat.rows > mat.cols;
    const float step = scale * sqrtf(fmaxf(1.f, (float)mat.cols / (float)mat.rows));
    constexpr int ROUNDS = Out::ROWS * Out::COLS / 8 / 64;
    auto mine = [&](int i, int& r, int& c) {
        const int t = 64 * i + lane;
        r = t / (Out::COLS / 8);
        c = t % (Out::COLS / 8) * 8;
        return row0 + r < n && col0 + c < mp;
    };
#pragma unroll
    for (int m = 0; m < S::WM; ++m)
#pragma unroll
        for (int k = 0; k < S::WN; ++k) Out::put(region, m, k, lane, sum[m][k]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int i = 0; i < ROUNDS; ++i) {
        int r, c;
        if (!mine(i, r, c)) continue;
        const int row = row0 + r, col = col0 + c;
        float v[8];
        Out::get(region, r, c, v);
        if constexpr (!LAST) {
            write_terms(base + room.x(from ^ 1) + prod::terms_at(pitch, row, col), v);
        } else if (!turned) {
            const long at = mat.offset + (long)row * mat.cols + col;
            float now[8];
            rows::load8(w + at, mat.cols - col, now);
#pragma unroll
            for (int e = 0; e < 8; ++e) now[e] = fmaf(-step, v[e], now[e]);
            rows::store8(w_out + at, mat.cols - col, now);
        } else {        // back into the region, to be read by columns
            *reinterpret_cast<float4*>(region + Out::at(r, c / 4)) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4*>(region + Out::at(r, c / 4 + 1)) = make_float4(v[4], v[5], v[6], v[7]);
        }
    }
    if (LAST && turned) {
        __builtin_amdgcn_wave_barrier();
        for (int t = lane; t < Out::ROWS * Out::COLS / 8; t += 64) {
            const int c = t / (Out::ROWS / 8), r = t % (Out::ROWS / 8) * 8, row = row0 + r, col = col0 + c;
            if (col >= mat.rows || row >= n) continue;
            const long at = mat.offset + (long)col * mat.cols + row;
            float now[8];
            rows::load8(w + at, n - row, now);
#pragma unroll
            for (int e = 0; e < 8; ++e) now[e] = fmaf(-step, *reinterpret_cast<const float*>(region + Out::at(r + e, c / 4) + 4 * (c & 3)), now[e]);
            rows::store8(w_out + at, n - row, now);
        }
    }
}

// ---------------------------------------------------------------- matrices with a short side of at most 64

// X is m x n here (long side first), n padded to 32 NB; a workgroup takes a stretch of the long side, LINES lines of it at a time.  In the workspace X is what such
// lines are in LDS, so that they come back by themselves, without a register or a conversion.
constexpr int LINES = 128, SMALL_THREADS = 512, WAVES = SMALL_THREADS / 64;
// Stretches: at most 32, since every workgroup reads the sums of all.
__host__ __device__ inline long stretch_of(long m) {
    const long s = (m + 31) / 32;
    return s <= LINES ? LINES : (s + LINES - 1) / LINES * LINES;
}
struct SmallRoom {
    long n, m, stretch, stretches, chunks;
    int nb;
    long u, x, sums0, sums1, end;
    __host__ __device__ SmallRoom(int rows, int cols) {
        n = rows < cols ? rows : cols;
        m = rows < cols ? cols : rows;
        nb = n <= 32 ? 1 : 2;
        stretch = stretch_of(m);
        stretches = (m + stretch - 1) / stretch;
        chunks = ((long)rows * cols + CHUNK - 1) / CHUNK;
        u = align256(8 * chunks);
        x = u + align256(4 * (long)rows * cols);
        sums0 = x + align256(stretches * stretch * prod::TERMS * nb);
        sums1 = sums0 + align256(4 * stretches * 1024 * nb * nb);
        end = sums1 + align256(4 * stretches * 1024 * nb * nb);
    }
};
inline bool is_small(int rows, int cols) { return (rows < cols ? rows : cols) <= DSSPK_ORTHOGONAL_SMALL; }
inline long room_of(int rows, int cols) { return is_small(rows, cols) ? SmallRoom(rows, cols).end : Room(rows, cols).end; }

// Lines of 32 NB numbers in LDS as terms; the 16-byte chunks of a line are exchanged so that eight lines' same chunk is in different banks.
template <int NB> struct Lines {
    static constexpr int PITCH = prod::TERMS * NB;
    static __device__ __forceinline__ int at(int line, int chunk) { return line * PITCH + 16 * (chunk ^ (NB == 2 ? line & 7 : (line >> 1) & 3)); }
    // four numbers of a line, the first of them number 4 g
    static __device__ __forceinline__ void put(char* lds, int line, int g, const float4& v) {
        uint2 t[split::PLANES];
        split::split4(v, t);
#pragma unroll
        for (int p = 0; p < split::PLANES; ++p) *reinterpret_cast<uint2*>(lds + at(line, g / 8 * 12 + 4 * p + g % 8 / 2) + 8 * (g & 1)) = t[p];
    }
    // operand of 16 lines for the numbers 32 b .. of each
    static __device__ __forceinline__ void along(const char* lds, int line, int b, int lane, uint4 (&f)[split::PLANES]) {
#pragma unroll
        for (int p = 0; p < split::PLANES; ++p) f[p] = *reinterpret_cast<const uint4*>(lds + at(line + (lane & 15), 12 * b + 4 * p + (lane >> 4)));
    }
    // operand of the numbers 16 i .. of 32 lines, the lines being the reduction index
    static __device__ __forceinline__ void across(const char* lds, int line, int i, int lane, uint4 (&f)[split::PLANES]) {
        const int l16 = lane & 15, row = line + 8 * (lane >> 4) + (l16 >> 2), chunk = i / 2 * 12 + 2 * (i & 1) + ((l16 & 3) >> 1);
#pragma unroll
        for (int p = 0; p < split::PLANES; ++p) {
            const uint2 lo = split::read_tr(lds + at(row, chunk + 4 * p) + 8 * (l16 & 1)), hi = split::read_tr(lds + at(row + 4, chunk + 4 * p) + 8 * (l16 & 1));
            f[p] = make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
    }
};
// the six products of terms of N tiles, one after the other over all tiles: a result is not waited for
template <int N, class A, class B> __device__ __forceinline__ void six(A a, B b, floatx4 (&sum)[N]) {
    constexpr int PA[6] = {0, 2, 1, 0, 1, 0}, PB[6] = {2, 0, 1, 1, 0, 0};
#pragma unroll
    for (int p = 0; p < 6; ++p)
#pragma unroll
        for (int t = 0; t < N; ++t) sum[t] = split::mfma(a(t)[PA[p]], b(t)[PB[p]], sum[t]);
}

// FIRST: X = u / (|u| + eps).  Otherwise X <- B X.  LAST: into the weights; otherwise X and this stretch's share of X^T X are left behind.
enum { FIRST = 0, BETWEEN = 1, LAST = 2 };
template <int NB, int KIND>
__device__ __forceinline__ void small_step(const Matrix& mat, const SmallRoom& room, char* base, int which, int turn, const float* w, float* w_out, float scale, float eps,
                                           char* lds) {
    using L = Lines<NB>;
    constexpr int T = 2 * NB;                       // 16-wide tiles of the short side
    constexpr int SQUARES = T * T >= WAVES ? T * T / WAVES : 1, WORKERS = T * T / SQUARES;      // tiles of A a wavefront, wavefronts that have some
    constexpr int FLOATS = LINES * 8 * NB / SMALL_THREADS;                  // groups of four a lane takes of the lines
    constexpr int COPIES = LINES * L::PITCH / 16 / SMALL_THREADS;           // the same as terms, 16 bytes each
    static_assert(LINES * L::PITCH % (16 * SMALL_THREADS) == 0, "");
    typedef uint4 Terms3[split::PLANES];
    char *xs = lds, *as = lds + LINES * L::PITCH;   // lines of X; lines of A, then of B
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, q = lane >> 4;
    const bool turned = mat.rows > mat.cols;        // the long side is the matrix's rows
    const float *sums_in = (const float*)(base + (turn ? room.sums1 : room.sums0));
    float* sums_out = (float*)(base + (turn ? room.sums0 : room.sums1));
    char* x = base + room.x;                        // line l at x + l L::PITCH
    const int n = (int)room.n;
    const long begin = which * room.stretch, end = min(begin + room.stretch, room.m);
    // tile t of this wavefront's share of A: rows 16 i + 4 q .., column 16 j + l16, one j for all
    const int j = wave % T;
    auto row_tile = [&](int t) { return wave / T * SQUARES + t; };
    Norm norm;
    float4 mine[FLOATS];
    auto fetch = [&](long l0) {
        if constexpr (KIND == FIRST) {
            const int lines = (int)min(end - l0, (long)LINES);
            const float* u = (const float*)(base + room.u);
#pragma unroll
            for (int k = 0; k < FLOATS; ++k) {
                const int t = tid + k * SMALL_THREADS, line = turned ? t / (8 * NB) : t % LINES, g = turned ? t % (8 * NB) : t / LINES;    // neighbours in a row go to neighbouring lanes
                float e[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = 4 * g + i;
                    e[i] = line < lines && c < n ? (turned ? u[(l0 + line) * n + c] : u[c * room.m + l0 + line]) : 0.f;
                }
                mine[k] = make_float4(e[0], e[1], e[2], e[3]);
            }
        } else {
            const prod::intx4 lines = prod::describe(x + l0 * L::PITCH, (long)LINES * L::PITCH);
            const unsigned to = prod::lds_address(xs) + wave * 1024;
#pragma unroll
            for (int k = 0; k < COPIES; ++k) prod::fetch16(lines, (k * SMALL_THREADS + tid) * 16u, to + k * SMALL_THREADS * 16);
        }
    };
    auto put = [&]() {
#pragma unroll
        for (int k = 0; k < FLOATS; ++k) {
            const int t = tid + k * SMALL_THREADS, line = turned ? t / (8 * NB) : t % LINES, g = turned ? t % (8 * NB) : t / LINES;
            L::put(xs, line, g, make_float4(norm(mine[k].x), norm(mine[k].y), norm(mine[k].z), norm(mine[k].w)));
        }
    };
    fetch(begin);
    if constexpr (KIND == FIRST) {
        double* part = (double*)as;
        double s = 0.;
        for (long i = tid; i < room.chunks; i += SMALL_THREADS) s += ((const double*)base)[i];
#pragma unroll
        for (int k = 32; k; k >>= 1) s += __shfl_xor(s, k);
        if (lane == 0) part[wave] = s;
        __syncthreads();
        s = 0.;
        for (int i = 0; i < WAVES; ++i) s += part[i];
        norm = Norm(s, eps);
        put();
    } else {
        // A from all stretches, in their order; B = a I + b A + c A A
        floatx4 A[SQUARES], B[SQUARES];
#pragma unroll
        for (int t = 0; t < SQUARES; ++t) A[t] = B[t] = floatx4{0.f, 0.f, 0.f, 0.f};
        if (wave < WORKERS) {
            const float* from = sums_in + (wave * SQUARES * 64 + lane) * 4;
#pragma unroll 8
            for (int c = 0; c < room.stretches; ++c)
#pragma unroll
                for (int t = 0; t < SQUARES; ++t) A[t] += *reinterpret_cast<const floatx4*>(from + (long)c * 1024 * NB * NB + 256 * t);
        }
        if (wave < WORKERS)
#pragma unroll
            for (int t = 0; t < SQUARES; ++t) L::put(as, 16 * j + l16, 4 * row_tile(t) + q, make_float4(A[t][0], A[t][1], A[t][2], A[t][3]));
        __syncthreads();
        if (wave < WORKERS)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                Terms3 fa[SQUARES], fb;
                L::along(as, 16 * j, b, lane, fb);
#pragma unroll
                for (int t = 0; t < SQUARES; ++t) L::along(as, 16 * row_tile(t), b, lane, fa[t]);
                six([&](int t) -> const Terms3& { return fa[t]; }, [&](int) -> const Terms3& { return fb; }, B);
            }
        __syncthreads();
        if (wave < WORKERS)
#pragma unroll
            for (int t = 0; t < SQUARES; ++t) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = fmaf(QB, A[t][e], fmaf(QC, B[t][e], row_tile(t) == j && 4 * q + e == l16 ? QA : 0.f));
                L::put(as, 16 * j + l16, 4 * row_tile(t) + q, make_float4(v[0], v[1], v[2], v[3]));
            }
    }
    floatx4 next[SQUARES];
#pragma unroll
    for (int t = 0; t < SQUARES; ++t) next[t] = floatx4{0.f, 0.f, 0.f, 0.f};
    const float step = scale * sqrtf(fmaxf(1.f, (float)mat.cols / (float)mat.rows));
    for (long l0 = begin; l0 < end; l0 += LINES) {
        const int lines = (int)min(end - l0, (long)LINES);
        if (l0 > begin) {
            __syncthreads();                        // the lines before have been read
            fetch(l0);
            if constexpr (KIND == FIRST) put();
        }
        prod::arrived();                            // the lines are there, by fetches or by put()
        if constexpr (KIND != FIRST) {
            // a wavefront's own 16 lines: rows of a result tile are the short side, columns the lines
            static_assert(LINES == 16 * WAVES, "");
            const int line = 16 * wave + l16;
            floatx4 sum[T];
#pragma unroll
            for (int i = 0; i < T; ++i) sum[i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                Terms3 fx, fb[T];
                L::along(xs, 16 * wave, b, lane, fx);
#pragma unroll
                for (int i = 0; i < T; ++i) L::along(as, 16 * i, b, lane, fb[i]);
                six([&](int i) -> const Terms3& { return fb[i]; }, [&](int) -> const Terms3& { return fx; }, sum);
            }
#pragma unroll
            for (int i = 0; i < T; ++i) {
                if constexpr (KIND == LAST) {
                    if (line < lines) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int c = 16 * i + 4 * q + k;
                            const long at = mat.offset + (turned ? (l0 + line) * n + c : c * room.m + l0 + line);
                            if (c < n) w_out[at] = fmaf(-step, sum[i][k], w[at]);
                        }
                    }
                } else {
                    L::put(xs, line, 4 * i + q, make_float4(sum[i][0], sum[i][1], sum[i][2], sum[i][3]));
                }
            }
            if constexpr (KIND != LAST) __syncthreads();
        }
        if constexpr (KIND != LAST) {
#pragma unroll
            for (int k = 0; k < COPIES; ++k) {
                const int at = (k * SMALL_THREADS + tid) * 16;
                *reinterpret_cast<uint4*>(x + l0 * L::PITCH + at) = *reinterpret_cast<const uint4*>(xs + at);
            }
            if (wave < WORKERS)
#pragma unroll
                for (int b = 0; b < LINES / 32; ++b) {
                    Terms3 fa[SQUARES], fb;
                    L::across(xs, 32 * b, j, lane, fb);
#pragma unroll
                    for (int t = 0; t < SQUARES; ++t) L::across(xs, 32 * b, row_tile(t), lane, fa[t]);
                    six([&](int t) -> const Terms3& { return fa[t]; }, [&](int) -> const Terms3& { return fb; }, next);
                }
        }
    }
    if constexpr (KIND != LAST)
        if (wave < WORKERS)
#pragma unroll
            for (int t = 0; t < SQUARES; ++t) *reinterpret_cast<floatx4*>(sums_out + (long)which * 1024 * NB * NB + ((wave * SQUARES + t) * 64 + lane) * 4) = next[t];
}

template <int KIND>
__global__ __launch_bounds__(SMALL_THREADS, 4) void small_kernel(Group grp, char* ws, int turn, const float* w, float* w_out, float scale, float eps) {
    __shared__ __attribute__((aligned(128))) char lds[(LINES + 64) * Lines<2>::PITCH];
    int which;
    const Matrix mat = grp.m[find<false>(grp, which)];      // (neighbours share little here, and the larger matrices would be one XCD's)
    const SmallRoom room(mat.rows, mat.cols);
    if (room.nb == 1) small_step<1, KIND>(mat, room, ws + mat.ws, which, turn, w, w_out, scale, eps, lds);
    else small_step<2, KIND>(mat, room, ws + mat.ws, which, turn, w, w_out, scale, eps, lds);
}

// ---------------------------------------------------------------- host

constexpr int64_t MAX_ENTRIES = 1LL << 38;
bool bad(const dsspk_matrix* m, int count) {
    if (count < 0 || (count && !m)) return true;
    int64_t steps = 0;
    for (int i = 0; i < count; ++i) {
        if (m[i].offset > MAX_ENTRIES) return true;          // (behind which an offset's sums might not fit 64 bits)
        if (m[i].rows < 1 || m[i].cols < 1 || m[i].rows > 1 << 20 || m[i].cols > 1 << 20 || (int64_t)m[i].rows * m[i].cols > 1LL << 31 || m[i].offset < 0) return true;
        if ((m[i].rows < m[i].cols ? m[i].rows : m[i].cols) > 1 << 14) return true;
        const Room r(m[i].rows, m[i].cols);
        steps += lower_tiles((int)r.n) * (r.mp / Shape::BK);
        if (i && m[i].offset < m[i - 1].offset + (int64_t)m[i - 1].rows * m[i - 1].cols) return true;
    }
    return steps > 1LL << 30;           // numbered by 32 bits
}

// the workgroups of a launch over the matrices of a group, `of` each
template <class F> int deal(Group& g, F of) {
    int blocks = 0;
    for (int i = 0; i < g.count; ++i) {
        g.first[i] = blocks;
        blocks += of(g.m[i]);
    }
    return blocks;
}

constexpr int CUS = 256;
template <bool V> struct Set { static constexpr bool value = V; };
template <bool POLY> int steps_of_group(Group& g) {
    return deal(g, [](const Matrix& x) { const Room r(x.rows, x.cols); return (int)(lower_tiles((int)r.n) * steps_of<POLY>(r)); });
}
// The shares of a group's symmetric products (g.first: steps, as steps_of_group leaves it): a workgroup on every compute unit, but of eight steps (10 us) at least once half of
// them have one, and never of less than four: joining costs as much then.  Short reductions are not cut at all where that works out without remainders.  Us a call, cut and
// uncut: 16 matrices of 256 x 1024 346 and 320, 100 of 192 x 384 690 and 561, four of 320 x 320 287 and 255, one of 448 x 448 285 and 298, three 315 and 308.  But with twelve or
// sixteen steps, and so few tiles that shares of four steps, which end where tiles do, leave compute units idle, they are: one matrix of 512 x 512 271 and 325, three 301 and
// 333 (four: 358 and 329), four of 384 x 384 273 and 282 (eight: 303 and 275), AlexNet-style 395 and 415.
template <bool POLY> Shares shares_of(const Group& g, int total, bool& whole) {
    int most = 0;
    for (int i = 0; i < g.count; ++i) {
        const int steps = steps_of<POLY>(Room(g.m[i].rows, g.m[i].cols));
        most = most > steps ? most : steps;
    }
    whole = most <= 16 && !((most == 12 || most == 16) && total < 2 * CUS);
    for (int i = 0; i < g.count && whole; ++i) whole = g.first[i] % most == 0 && most % steps_of<POLY>(Room(g.m[i].rows, g.m[i].cols)) == 0;
    Shares s;
    s.steps = ceil_div(total, CUS);
    if (s.steps < 8) s.steps = total / (CUS / 2) < 4 ? 4 : total / (CUS / 2) < 8 ? total / (CUS / 2) : 8;
    if (whole) s.steps = most;
    s.groups = ceil_div(total, s.steps);
    return s;
}
constexpr size_t PARTIAL_BYTES = 2 * (size_t)CUS * TILE_FLOATS * 4;

}  // namespace

extern "C" size_t dsspk_orthogonal_workspace_bytes(const dsspk_matrix* matrices, int count) {
    if (bad(matrices, count)) return 0;
    size_t bytes = 256;
    bool large = false;
    for (int i = 0; i < count; ++i) {
        bytes += (size_t)room_of(matrices[i].rows, matrices[i].cols);
        large = large || !is_small(matrices[i].rows, matrices[i].cols);
    }
    return bytes + (large ? PARTIAL_BYTES : 0);
}

extern "C" int dsspk_orthogonal_apply(void* stream, const float* w, float* w_out, const float* m, float* m_out, const float* g, int64_t n, const dsspk_matrix* matrices,
                                      int count, float scale, float rest_scale, float momentum, int nesterov, int steps, float eps, void* workspace,
                                      size_t workspace_bytes) {
    if (bad(matrices, count) || !w || !w_out || !m || !m_out || !g || n < 0 || n > MAX_ENTRIES || steps < 1 || steps > 64 || !(eps > 0.f)) return -1;
    if (count && matrices[count - 1].offset + (int64_t)matrices[count - 1].rows * matrices[count - 1].cols > n) return -1;
    if (w_out == g || m_out == g || w_out == m || m_out == w || w_out == m_out) return -1;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < dsspk_orthogonal_workspace_bytes(matrices, count)) return -1;
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;
    float* partial = (float*)workspace;
    // what lies between the matrices
    Gaps gaps = {};
    int blocks = 0;
    int64_t at = 0;
    auto flush = [&]() {
        if (gaps.count) {
            if (nesterov) hipLaunchKernelGGL(momentum_gaps_kernel<true>, dim3(blocks), dim3(256), 0, s, gaps, w, w_out, m, m_out, g, momentum, rest_scale);
            else hipLaunchKernelGGL(momentum_gaps_kernel<false>, dim3(blocks), dim3(256), 0, s, gaps, w, w_out, m, m_out, g, momentum, rest_scale);
        }
        gaps.count = blocks = 0;
    };
    for (int i = 0; i <= count; ++i) {
        const int64_t to = i < count ? matrices[i].offset : n;
        const int64_t most = most_blocks(256);          // of a launch; a longer gap takes several
        while (to > at) {
            if (gaps.count == GROUP || blocks == most) flush();
            const int64_t room = (most - blocks) * GAP_CHUNK, end = to - at < room ? to : at + room;
            gaps.first[gaps.count] = blocks;
            gaps.from[gaps.count] = at;
            gaps.to[gaps.count++] = end;
            blocks += ceil_div(end - at, GAP_CHUNK);
            at = end;
        }
        if (i < count) at = to + (int64_t)matrices[i].rows * matrices[i].cols;
    }
    flush();
    auto momentum_of_group = [&](Group& grp, auto chunks) {
        const int b = deal(grp, chunks);
        if (nesterov) hipLaunchKernelGGL(momentum_kernel<true>, dim3(b), dim3(256), 0, s, grp, ws, m, m_out, g, momentum);
        else hipLaunchKernelGGL(momentum_kernel<false>, dim3(b), dim3(256), 0, s, grp, ws, m, m_out, g, momentum);
    };
    auto chunks = [](const Matrix& x) { return (int)(((long)x.rows * x.cols + CHUNK - 1) / CHUNK); };
    auto small = [&](Group& grp) {
        momentum_of_group(grp, chunks);
        const int b = deal(grp, [](const Matrix& x) { return (int)SmallRoom(x.rows, x.cols).stretches; });
        hipLaunchKernelGGL(small_kernel<FIRST>, dim3(b), dim3(SMALL_THREADS), 0, s, grp, ws, 0, w, w_out, scale, eps);
        for (int k = 0; k < steps; ++k)
            if (k + 1 < steps) hipLaunchKernelGGL(small_kernel<BETWEEN>, dim3(b), dim3(SMALL_THREADS), 0, s, grp, ws, ~k & 1, w, w_out, scale, eps);
            else hipLaunchKernelGGL(small_kernel<LAST>, dim3(b), dim3(SMALL_THREADS), 0, s, grp, ws, ~k & 1, w, w_out, scale, eps);
    };
    auto symmetric = [&](Group& grp, auto poly, int from) {
        constexpr bool POLY = decltype(poly)::value;
        const int total = steps_of_group<POLY>(grp);
        bool whole = false;
        const Shares shares = shares_of<POLY>(grp, total, whole);
        hipLaunchKernelGGL(symmetric_kernel<POLY>, dim3(shares.groups), dim3(Shape::THREADS), 0, s, grp, ws, partial, shares, total, from);
        if (whole) return;
        const int tiles = deal(grp, [](const Matrix& x) { return (int)lower_tiles((int)Room(x.rows, x.cols).n); });
        hipLaunchKernelGGL(join_kernel<POLY>, dim3(8 * tiles), dim3(64), 0, s, grp, ws, partial, shares);
    };
    auto large = [&](Group& grp) {
        momentum_of_group(grp, chunks);
        int b = deal(grp, [](const Matrix& x) { return ceil_div(x.rows, 64) * ceil_div(x.cols, 64); });
        hipLaunchKernelGGL(normalise_kernel, dim3(b), dim3(256), 0, s, grp, ws, eps);
        for (int k = 0; k < steps; ++k) {
            symmetric(grp, Set<false>{}, k & 1);
            symmetric(grp, Set<true>{}, k & 1);
            const bool last = k + 1 == steps;
            auto update = [&](auto shape) {
                using S = decltype(shape);
                b = deal(grp, [](const Matrix& x) { const Room r(x.rows, x.cols); return ceil_div(r.n, S::BM) * ceil_div(r.m, S::BN); });
                if (last) hipLaunchKernelGGL((update_kernel<S, true>), dim3(b), dim3(S::THREADS), 0, s, grp, ws, k & 1, w, w_out, scale);
                else hipLaunchKernelGGL((update_kernel<S, false>), dim3(b), dim3(S::THREADS), 0, s, grp, ws, k & 1, w, w_out, scale);
            };
            // Rounds of workgroups times us of a step: 1.11 with one square tile on a compute unit, 0.80 and 1.27 with one and two halves.  One matrix of 2048 x 2048: 2110 us a
            // call with squares, 2172 with halves; four of 768 x 1500 and the reverse: 692 and 631.
            b = deal(grp, [](const Matrix& x) { const Room r(x.rows, x.cols); return ceil_div(r.n, Shape::BM) * ceil_div(r.m, Shape::BN); });
            const int halves = 2 * b, rest = halves % (2 * CUS);
            const float squares = 1.11f * ceil_div(b, CUS), half = 1.27f * (halves / (2 * CUS)) + (rest > CUS ? 1.27f : rest ? 0.80f : 0.f);
            if (half < squares) update(Half{});
            else update(Shape{});
        }
    };
    // small and large matrices through launches of their own, a group at a time
    Group groups[2] = {};
    bool any_large = false;
    for (int i = 0; i < count; ++i) any_large = any_large || !is_small(matrices[i].rows, matrices[i].cols);
    int64_t room_at = any_large ? PARTIAL_BYTES : 0;
    for (int i = 0; i <= count; ++i) {
        for (int kind = 0; kind < 2; ++kind) {
            Group& grp = groups[kind];
            if (grp.count == GROUP || (i == count && grp.count)) {
                if (kind) small(grp);
                else large(grp);
                grp.count = 0;
            }
        }
        if (i == count) break;
        const dsspk_matrix& x = matrices[i];
        Group& grp = groups[is_small(x.rows, x.cols)];
        grp.m[grp.count++] = {x.offset, room_at, x.rows, x.cols};
        room_at += room_of(x.rows, x.cols);
    }
    return DSSPK_LAUNCH_RC();
}
