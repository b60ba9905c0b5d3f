// Products of large matrices on the bf16 matrix cores (internal): one output tile by one workgroup.
//
//   C[i][j] = sum_k a(i, k) b(j, k)
//
// Operands are bf16 in memory, PLANES of them.  One plane: the operand is bf16.  Three planes: the operand is fp32, written as three bf16
// terms (split.hpp: of 2^24 x, six of the nine products, the small ones in an accumulator of their own).
// An operand is stored either with the reduction index contiguous (KC: element (i, k) at p + i pitch + 2 k) or with the other index
// contiguous (KO: at p + k pitch + 2 i); both reach LDS as they are in memory.  KC tiles are read with 16-byte reads, KO tiles with
// the transposing 8-byte ones.  The three terms of 32 neighbours in a row lie one behind the other, 64 bytes each: a tile then has 192 contiguous bytes or more in
// every row (with each plane a matrix of its own, 64 for a KC tile, half a cache line, products of two KC operands took 13 % longer).
//
// Tiles go from memory to LDS without passing through registers (buffer loads with an LDS destination, 16 bytes a lane): lane l's 16 bytes land at
// the wavefront's base + 16 l, so the order inside a tile is made by choosing which 16 bytes a lane fetches.  Chunks of 16 bytes are swapped within a row
// by an exclusive or with a function of the row, such that the lanes that LDS serves together read different banks.  Rows beyond the
// operand's end are outside the buffer and arrive as zero; so do columns, whose offset is moved outside.
//
// Two tiles in LDS, or more where a workgroup has a compute unit to itself and little to do on it: while the matrix cores work on one, the next ones arrive; one
// barrier a tile.
//
// The matrix-core tile is transposed: its rows are C's columns, so that a lane holds four consecutive columns of one row of C.
//
// Measured, whole calls of a forward product: bf16 4096 x 4096 x 4096 117 to 127 us, 8192 cubed 751 to 804 us, 1.37 to 1.46 PFLOP/s (the library 795 to 890); three planes, 4096 x 4096 x 4096 633
// to 639 us, 217 TFLOP/s of fp32, 1.3 PFLOP/s in bf16 (the library's fp32 125 to 133 TFLOP/s).  Bound by the matrix cores and their clock under load: busy 55 to 70 % of the cycles in the
// kernels of three planes, but 25 with the 64 x 64 tile; of one plane 57 in a split product, 32 and 42 where an epilogue follows.  LDS is active in 15 to 27 % of them, with conflicts in 0 to 3 % of
// those, 9 where the last step of an update turns its results round in LDS and 33 with the 64 x 64 tile of three planes, whose KO rows have 24 chunks; why was not followed up.
#pragma once
#include "split.hpp"

namespace prod {

struct Operand {
    const char* p;          // 16-byte aligned
    long pitch;             // bytes from row to row, a multiple of 16
    int ext, K;             // i < ext, k < K; the contiguous one is a multiple of 8, with three planes of 32 (padded with zeros)
};
// where the terms of element (row, col) of such a matrix begin, and how far apart they are
constexpr int TERM = 64, TERMS = 192;
__host__ __device__ inline long terms_pitch(long cols) { return cols / 32 * TERMS; }
__device__ __forceinline__ long terms_at(long pitch, long row, long col) { return row * pitch + (col >> 5) * TERMS + 2 * (col & 31); }

template <int PLANES_, int BM_, int BN_, int BK_, int GM_, int GN_, int STAGES_ = 2> struct Shape {
    static constexpr int STAGES = STAGES_;      // tiles in LDS
    static constexpr int PLANES = PLANES_, BM = BM_, BN = BN_, BK = BK_;
    static constexpr int GM = GM_, GN = GN_, THREADS = 64 * GM * GN;        // wavefronts along i and j
    static constexpr int WM = BM / GM / 16, WN = BN / GN / 16;              // 16 x 16 tiles of a wavefront
    static constexpr int A_BYTES = PLANES * BM * BK * 2, B_BYTES = PLANES * BN * BK * 2;
    static constexpr int STAGE = A_BYTES + B_BYTES, LDS = STAGES * STAGE;
};

typedef int intx4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned lds_address(const char* p) { return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)p; }

// 16 bytes a lane from buffer + offset to LDS at `to` + 16 lane; counted by vmcnt, zero where offset + 16 passes the buffer's end
__device__ __forceinline__ void fetch16(const intx4& buffer, unsigned offset, unsigned to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(__builtin_amdgcn_readfirstlane(to)), "v"(offset), "s"(buffer) : "m0", "memory");
}

__device__ __forceinline__ intx4 describe(const char* p, long bytes) {
    const uint64_t a = (uint64_t)(uintptr_t)p;
    intx4 d;
    d[0] = __builtin_amdgcn_readfirstlane((int)(unsigned)a);
    d[1] = __builtin_amdgcn_readfirstlane((int)(unsigned)(a >> 32));
    d[2] = __builtin_amdgcn_readfirstlane((int)(bytes < 0 ? 0 : bytes > 0x7fffffffL ? 0x7fffffffL : bytes));
    d[3] = 0x00027000;      // untyped 32-bit data, no swizzle
    return d;
}

// One operand's part of a stage: I x BK (KC) or BK x I (KO), staged by THREADS lanes, read as 16-row fragments of 32 k.
template <int PLANES, int I, int BK, int THREADS, bool KO> struct Tile {
    static_assert(PLANES == 1 || BK == 32, "");
    static constexpr int CHUNKS = PLANES * (KO ? I / 8 : BK / 8);       // 16-byte chunks of a row
    static constexpr int ROWS = KO ? BK : I, PITCH = 16 * CHUNKS;
    static constexpr int LOADS = ROWS * CHUNKS / THREADS;
    static_assert(ROWS * CHUNKS % THREADS == 0, "");

    // KC: eight lanes read one chunk of eight consecutive rows.  KO: sixteen lanes read 32 bytes of four consecutive rows.
    static __device__ __forceinline__ int turned(int row) {
        if constexpr (KO) return (2 * (row & 3)) | (CHUNKS % 16 == 0 ? 8 * ((row >> 3) & 1) : 0);
        else return BK == 64 ? row & 7 : (row >> 1) & 3;
    }
    // Load u covers THREADS chunks of the tile, row by row.  Where that is a number of rows after which the exchange of chunks repeats, a lane's place in the
    // first KINDS loads says it all.
    static constexpr bool WHOLE = THREADS % CHUNKS == 0 && THREADS / CHUNKS % 8 == 0;
    static constexpr int STEP = WHOLE ? THREADS / CHUNKS : 0, KINDS = !WHOLE ? LOADS : STEP % 16 == 0 ? 1 : LOADS < 2 ? LOADS : 2;
    static_assert(LOADS % KINDS == 0, "");
    int row[KINDS], chunk[KINDS];
    __device__ __forceinline__ void start(int tid) {
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const int slot = i * THREADS + tid;
            row[i] = slot / CHUNKS;
            chunk[i] = slot % CHUNKS ^ turned(row[i]);
        }
    }
    // The loads of a tile: a buffer that begins at its corner and moves along the reduction index, offsets that stay.  Rows (KC) or columns (KO) beyond the operand's end
    // are outside from the start, reduction indices from `limit` on as the buffer comes to them.
    struct Source {
        uint64_t p;
        int bytes;
        long step;              // bytes from tile to tile
        int left;               // reduction indices up to the limit
        unsigned at[KINDS], hop;
        int k[KINDS];
        __device__ __forceinline__ void advance() {
            p += step;
            left -= BK;
        }
        __device__ __forceinline__ intx4 buffer() const {
            intx4 d;
            d[0] = (int)(unsigned)p;
            d[1] = (int)(unsigned)(p >> 32);
            d[2] = bytes;
            d[3] = 0x00027000;  // untyped 32-bit data, no swizzle
            return d;
        }
    };
    __device__ __forceinline__ Source source(const Operand& o, int i0, int k0, int limit) const {
        const long row0 = KO ? k0 : i0, col0 = KO ? i0 : k0, cols = KO ? o.ext : o.K;
        const long skip = PLANES == 3 ? col0 / 32 * TERMS : 2 * col0, width = PLANES == 3 ? cols / 32 * TERMS : 2 * cols;       // of a row, in bytes
        const long bytes = KO ? BK * o.pitch : (o.ext - row0 - 1) * o.pitch + width;
        const uint64_t p = (uint64_t)(uintptr_t)o.p + row0 * o.pitch + skip;
        Source s;
        s.p = ((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(p >> 32)) << 32) | (unsigned)__builtin_amdgcn_readfirstlane((int)p);
        s.bytes = __builtin_amdgcn_readfirstlane((int)(bytes < 0 ? 0 : bytes > 0x7fffffffL ? 0x7fffffffL : bytes));
        s.step = KO ? BK * o.pitch : PLANES == 3 ? BK / 32 * TERMS : 2 * BK;
        s.left = __builtin_amdgcn_readfirstlane(min(limit, o.K) - k0);
        s.hop = (unsigned)(STEP * o.pitch);
#pragma unroll
        for (int i = 0; i < KINDS; ++i) {
            const unsigned offset = (unsigned)((row[i] - i * STEP) * o.pitch) + 16u * chunk[i];
            s.at[i] = KO && 16 * chunk[i] >= width - skip ? split::OUTSIDE : offset;
            s.k[i] = KO ? row[i] - i * STEP : PLANES == 3 ? 0 : 8 * chunk[i];
        }
        return s;
    }
    __device__ __forceinline__ void fetch(const Source& s, const intx4& buffer, int u, unsigned to) const {
        const bool here = s.k[u % KINDS] < s.left - (KO ? u * STEP : 0);
        fetch16(buffer, here ? s.at[u % KINDS] + u * s.hop : split::OUTSIDE, to + u * THREADS * 16);
    }
    // term p of fragment i (16 rows of the wavefront's part, which begins at row `first`, a multiple of 32) for indices 32 kk ..
    static __device__ __forceinline__ uint4 read(const char* tile, int p, int first, int i, int kk, int lane) {
        const int l16 = lane & 15, q = lane >> 4;
        if constexpr (!KO) {
            return *reinterpret_cast<const uint4*>(tile + (first + 16 * i + l16) * PITCH + 16 * ((4 * kk + q) ^ turned(l16)) + TERM * p);
        } else {
            const int row = 8 * q + (l16 >> 2), c = PLANES * (first / 8 + i / 2 * 4) + 4 * p + 2 * (i & 1) + ((l16 & 3) >> 1);
            const char* at = tile + (32 * kk + row) * PITCH + 16 * (c ^ turned(row)) + 8 * (l16 & 1);
            const uint2 lo = split::read_tr(at), hi = split::read_tr(at + 4 * PITCH);
            return make_uint4(lo.x, lo.y, hi.x, hi.y);
        }
    }
};

// all but this wavefront's newest FLYING fetches have arrived, its LDS reads are done, and so it is for everybody
template <int FLYING = 0> __device__ __forceinline__ void arrived() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(FLYING) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A wavefront's registers: fragments of the present 32 indices and, while the matrix cores work on those, of the next.
//
// Everything that is not a product - LDS reads of the next fragments, fetches of the tile after next - is spread over the products by hand and held there by
// scheduling barriers: left to itself the compiler reads a fragment just in front of its use, and the matrix cores wait for LDS most of the time.
//   one plane:    BK / 32 phases of WM WN products.  During phase kk the fragments of phase kk + 1 are read; the last one begins with the barrier behind which the
//                 next tile is there and this one has been read by everybody, reads the next tile's first fragments and sends for the tile after it.
//   three planes: BK = 32; six phases, the products of terms.  A term's registers are free behind its last product, and take the next tile's;
//                 the leading terms, which the last product needs, have a second set.
template <class S, bool A_KO, bool B_KO> struct Wave {
    static constexpr int P = S::PLANES, KK = S::BK / 32, WM = S::WM, WN = S::WN, NM = WM * WN;
    static_assert(P == 1 ? KK == 2 : KK == 1, "");
    using TA = Tile<P, S::BM, S::BK, S::THREADS, A_KO>;
    using TB = Tile<P, S::BN, S::BK, S::THREADS, B_KO>;
    static constexpr int FETCHES = TA::LOADS + TB::LOADS;
    TA ta;
    TB tb;
    const Operand &a, &b;
    int i0, j0, row, col, lane;
    unsigned base;
    const char* lds;

    __device__ __forceinline__ Wave(const Operand& a_, const Operand& b_, int i0_, int j0_, const char* lds_) : a(a_), b(b_), i0(i0_), j0(j0_), lds(lds_) {
        const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        lane = tid & 63;
        row = wave / S::GN * 16 * WM;
        col = wave % S::GN * 16 * WN;
        ta.start(tid);
        tb.start(tid);
        base = __builtin_amdgcn_readfirstlane(lds_address(lds) + (unsigned)(wave * 64 * 16));
    }
    typename TA::Source sa;
    typename TB::Source sb;
    __device__ __forceinline__ void start(int t0, int t1) {
        sa = ta.source(a, i0, t0 * S::BK, t1 * S::BK);
        sb = tb.source(b, j0, t0 * S::BK, t1 * S::BK);
    }
    // fetch f of the tile that is next, to place `buf`; behind the last of them, advance()
    __device__ __forceinline__ void fetch(int buf, int f) const {
        if (f < TA::LOADS) ta.fetch(sa, sa.buffer(), f, base + buf * S::STAGE);
        else tb.fetch(sb, sb.buffer(), f - TA::LOADS, base + buf * S::STAGE + S::A_BYTES);
    }
    __device__ __forceinline__ void advance() {
        sa.advance();
        sb.advance();
    }
    __device__ __forceinline__ uint4 read_a(int buf, int p, int m, int kk) const { return TA::read(lds + buf * S::STAGE, p, row, m, kk, lane); }
    __device__ __forceinline__ uint4 read_b(int buf, int p, int n, int kk) const { return TB::read(lds + buf * S::STAGE + S::A_BYTES, p, col, n, kk, lane); }
};

template <int N> struct Set { static constexpr int value = N; };

// work j of NS that are spread over the first three quarters of NM products: how many of them come before product i
constexpr int before(int i, int NS, int NM) {
    const int over = NM * 3 / 4 > 0 ? NM * 3 / 4 : 1;
    return i >= over ? NS : i * NS / over;
}
template <int NM, int NS, class Product, class Side> __device__ __forceinline__ void interleave(Product product, Side side) {
#pragma unroll
    for (int i = 0; i < NM; ++i) {
#pragma unroll
        for (int j = before(i, NS, NM); j < before(i + 1, NS, NM); ++j) side(j);
        product(i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// The tile at (i0, j0), reduction tiles t0 .. t1 - 1 of BK indices.  sum[m][n][v]: row i0 + wavefront's row + 16 m + lane % 16, column j0 + wavefront's column +
// 16 n + 4 (lane / 16) + v; with three planes 2^48 times the product if the planes are those of 2^24 x.  All lanes of the workgroup take part; lds: S::LDS bytes,
// free again on return.  ahead(n), n tiles before the end: one fetch of something else (Ahead::FETCHES).
struct Nothing {
    static constexpr int FETCHES = 0;
    __device__ __forceinline__ void operator()(int) const {}
};
template <class F> struct Something {
    static constexpr int FETCHES = 1;
    F f;
    __device__ __forceinline__ void operator()(int n) const { f(n); }
};
template <class S, bool A_KO, bool B_KO, class Ahead = Nothing>
__device__ __forceinline__ void tile(const Operand& a, const Operand& b, int i0, int j0, int t0, int t1, char* lds, floatx4 (&sum)[S::WM][S::WN], const Ahead& ahead = {}) {
    using W = Wave<S, A_KO, B_KO>;
    constexpr int P = S::PLANES, WM = S::WM, WN = S::WN, NM = W::NM;
#pragma unroll
    for (int m = 0; m < WM; ++m)
#pragma unroll
        for (int n = 0; n < WN; ++n) sum[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};
    if (t0 >= t1) return;
    W w(a, b, i0, j0, lds);
    w.start(t0, t1);
    // Tiles behind the last one are fetched as well, from outside the buffers (zeros, no memory traffic): a loop without branches, around which the compiler would
    // move accumulators.
    auto fetch_all = [&](int buf) {
#pragma unroll
        for (int f = 0; f < W::FETCHES; ++f) w.fetch(buf, f);
        w.advance();
    };
    constexpr int AHEAD = Ahead::FETCHES, STAGES = S::STAGES, EACH = W::FETCHES + AHEAD;       // fetches a tile, those of ahead() the newest
    static_assert(AHEAD <= 1 && (STAGES - 1) * EACH < 64, "");
    constexpr int FLYING = AHEAD + (STAGES - 2) * EACH;         // of later tiles, when the next one has to be there
    fetch_all(0);
#pragma unroll
    for (int i = 1; i < STAGES; ++i) {
        fetch_all(i);
        ahead(t1 - t0 + STAGES - 1 - i);
    }
    arrived<(STAGES - 1) * EACH>();
    int buf = 0;
    if constexpr (P == 1) {
        constexpr int KK = W::KK, READS = WM + WN;
        static_assert(KK % 2 == 0, "the next tile's first fragments go into set 0");
        uint4 fa[2][WM], fb[2][WN];
        auto read = [&](int set, int j, int buf, int kk) {
            if (j < WN) fb[set][j] = w.read_b(buf, 0, j, kk);
            else fa[set][j - WN] = w.read_a(buf, 0, j - WN, kk);
        };
#pragma unroll
        for (int j = 0; j < READS; ++j) read(0, j, 0, 0);
        for (int t = t0; t < t1; ++t) {
            const int next = buf + 1 == STAGES ? 0 : buf + 1;
#pragma unroll
            for (int kk = 0; kk < KK - 1; ++kk)
                interleave<NM, READS>([&](int i) { sum[i / WN][i % WN] = split::mfma(fb[kk & 1][i % WN], fa[kk & 1][i / WN], sum[i / WN][i % WN]); },
                                      [&](int j) { read((kk + 1) & 1, j, buf, kk + 1); });
            arrived<FLYING>();
            interleave<NM, READS + W::FETCHES + Ahead::FETCHES>([&](int i) { sum[i / WN][i % WN] = split::mfma(fb[1][i % WN], fa[1][i / WN], sum[i / WN][i % WN]); },
                                                   [&](int j) {
                                                       if (j < READS) read(0, j, next, 0);
                                                       else if (j < READS + W::FETCHES) w.fetch(buf, j - READS);
                                                       else ahead(t1 - 1 - t);
                                                   });
            w.advance();
            buf = next;
        }
    }
    if constexpr (P == 3) {
        floatx4 small[WM][WN];
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int n = 0; n < WN; ++n) small[m][n] = floatx4{0.f, 0.f, 0.f, 0.f};
        uint4 a0[2][WM], b0[2][WN], a1[WM], b1[WN], a2[WM], b2[WN];
#pragma unroll
        for (int n = 0; n < WN; ++n) { b2[n] = w.read_b(0, 2, n, 0); b0[0][n] = w.read_b(0, 0, n, 0); b1[n] = w.read_b(0, 1, n, 0); }
#pragma unroll
        for (int m = 0; m < WM; ++m) { a0[0][m] = w.read_a(0, 0, m, 0); a2[m] = w.read_a(0, 2, m, 0); a1[m] = w.read_a(0, 1, m, 0); }
        // tile t, whose leading terms are in set X; the tile that takes its place in LDS is sent for
        auto step = [&](auto set, int t) {
            constexpr int X = decltype(set)::value, Y = X ^ 1;
            const int here = STAGES == 2 ? X : buf, next = STAGES == 2 ? Y : buf + 1 == STAGES ? 0 : buf + 1;
            auto product = [&](const uint4 (&fa)[WM], const uint4 (&fb)[WN], floatx4 (&to)[WM][WN]) {
                return [&](int i) { to[i / WN][i % WN] = split::mfma(fb[i % WN], fa[i / WN], to[i / WN][i % WN]); };
            };
            arrived<FLYING>();
            interleave<NM, W::FETCHES + Ahead::FETCHES>(product(a0[X], b2, small), [&](int j) {
                if (j < W::FETCHES) w.fetch(here, j);
                else ahead(t1 - 1 - t);
            });
            w.advance();
            interleave<NM, WN>(product(a2, b0[X], small), [&](int j) { b2[j] = w.read_b(next, 2, j, 0); });
            interleave<NM, WM>(product(a1, b1, small), [&](int j) { a2[j] = w.read_a(next, 2, j, 0); });
            interleave<NM, WM + WN>(product(a0[X], b1, small), [&](int j) {
                if (j < WN) b0[Y][j] = w.read_b(next, 0, j, 0);
                else a0[Y][j - WN] = w.read_a(next, 0, j - WN, 0);
            });
            interleave<NM, WN>(product(a1, b0[X], small), [&](int j) { b1[j] = w.read_b(next, 1, j, 0); });
            interleave<NM, WM>(product(a0[X], b0[X], sum), [&](int j) { a1[j] = w.read_a(next, 1, j, 0); });
            buf = next;
        };
        for (int t = t0; t < t1; t += 2) {      // an odd number of tiles: one of zeros behind them
            step(Set<0>{}, t);
            step(Set<1>{}, t + 1);
        }
#pragma unroll
        for (int m = 0; m < WM; ++m)
#pragma unroll
            for (int n = 0; n < WN; ++n) sum[m][n] += small[m][n];
    }
    arrived();
}

// The way of a wavefront's sums out: through LDS, so that eight lanes hold a row of 64 columns, eight consecutive ones each.  Every wavefront has a region of its own,
// taken in PASSES rounds of ROWS rows; 16-byte chunks of a row are exchanged so that neither writing (16 rows, one chunk) nor reading meets a bank twice.
template <class S> struct Out {
    static constexpr int COLS = 16 * S::WN, REGION = S::LDS / (S::GM * S::GN);
    static constexpr int FIT = REGION / (4 * COLS) / 16, TILES = FIT >= S::WM ? S::WM : FIT >= 4 ? 4 : FIT >= 2 ? 2 : 1, ROWS = 16 * TILES, PASSES = S::WM / TILES;
    static_assert(S::WM % TILES == 0 && COLS % 32 == 0, "");
    static __device__ __forceinline__ int at(int row, int chunk) { return 4 * COLS * row + 16 * (chunk ^ (row & 7)); }
    // row 16 m + lane % 16, columns 16 n + 4 (lane / 16) ..
    static __device__ __forceinline__ void put(char* region, int m, int n, int lane, const floatx4& v) {
        *reinterpret_cast<floatx4*>(region + at(16 * m + (lane & 15), 4 * n + (lane >> 4))) = v;
    }
    static __device__ __forceinline__ void get(const char* region, int row, int col, float (&v)[8]) {
        const floatx4 lo = *reinterpret_cast<const floatx4*>(region + at(row, col / 4)), hi = *reinterpret_cast<const floatx4*>(region + at(row, col / 4 + 1));
#pragma unroll
        for (int i = 0; i < 4; ++i) { v[i] = lo[i]; v[4 + i] = hi[i]; }
    }
};

// Order of the tiles: consecutive ones to one XCD, and of those, eight rows of tiles side by side, so that what an L2 holds serves eight tiles either way; the parts
// of a reduction one after the other, so that an XCD reads as little as possible of what others read too.
struct Place { int i, j, part; };
__device__ __forceinline__ Place place(int block, int tiles_i, int tiles_j, int parts) {
    constexpr int BAND = 8;
    const int all = tiles_i * tiles_j, u = xcd_tile(block, all * parts), part = u / all, t = u - part * all;
    const int band = t / (BAND * tiles_j), in = t - band * BAND * tiles_j, height = min(BAND, tiles_i - band * BAND);
    return {band * BAND + in % height, in / height, part};
}

}  // namespace prod
