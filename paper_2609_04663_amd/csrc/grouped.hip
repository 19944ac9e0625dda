// Which kernels run a grouped product, and what prepares their operands: 16-bit
// matrices copied to 16-byte alignment, and an expert's rows in pieces.
#include "api_state.h"
#include "emu_internal.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int BK = 64;                               // k-block of the kernels of grouped16.h
constexpr int64_t OFFSETS = (int64_t)1 << 32;        // what a copy's 32-bit offset spans
constexpr int64_t MOST_COPIED = (int64_t)1 << 31;    // bytes of workspace for copies

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

// A matrix (or one for each expert) of 16-bit entries as the copy has it: rows x ld,
// ld a multiple of 8, zeros around the entries that exist.
struct Realigned {
    const void *src;
    int64_t lds, stride, src_rows;
    int cols;
    const int *map;                 // row r is row map[r] of the source (zeros if it has none); or null
    int mats;
    const int *offsets;             // matrix e is copied if expert e has rows; or null
    int64_t R;                      // of offsets
    int64_t rows, ld;
    int64_t bytes() const { return mats * rows * ld * 2; }
};

// 16 bytes a thread: unaligned loads, aligned stores.  Bound by bytes.
__global__ __launch_bounds__(256) void realign_kernel(Realigned m, uint16_t *__restrict__ dst) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x, per_row = (unsigned)(m.ld / 8);
    const int64_t row = i / per_row;
    const int c = i % per_row * 8;
    if (row >= m.rows) return;
    for (int e = blockIdx.y; e < m.mats; e += gridDim.y) {
        if (m.offsets) {
            int64_t lo, hi;
            expert_rows(m.offsets, m.mats, m.R, e, lo, hi);
            if (lo == hi) continue;
        }
        const int64_t at = m.map ? m.map[row] : row;
        vec<uint16_t, 8> v = {};
        if (at >= 0 && at < m.src_rows) {
            const uint16_t *const p = static_cast<const uint16_t *>(m.src) + e * m.stride + at * m.lds + c;
            if (c + 8 <= m.cols) {
                v = *reinterpret_cast<const vec<uint16_t, 8> *>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) v[j] = c + j < m.cols ? p[j] : 0;
            }
        }
        typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
        *reinterpret_cast<u16x8 *>(dst + (e * m.rows + row) * m.ld + c) = v;
    }
}
hipError_t realign(const Realigned &m, char *dst, hipStream_t s) {
    const dim3 grid((unsigned)((m.rows * m.ld / 8 + 255) / 256), m.mats < 32768 ? m.mats : 32768);
    realign_kernel<<<grid, 256, 0, s>>>(m, reinterpret_cast<uint16_t *>(dst));
    return hipGetLastError();
}
// us that a copy takes: a launch, and read and written bytes at 4 TB/s
double copy_time(const Realigned &m) { return 6 + m.bytes() * 2 / 4e6; }

// dW[e] = the sum of the pieces' matrices, in order.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float *__restrict__ part, int64_t ld, int M, int N,
                                                   int pieces, T *__restrict__ dW, int64_t ldw, int64_t sw) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / N, n = i % N;
    if (m >= M) return;
    const float *const p = part + blockIdx.y * (int64_t)pieces * M * ld + m * ld + n;
    float v = p[0];
    for (int k = 1; k < pieces; ++k) v += p[k * M * ld];
    dW[blockIdx.y * sw + m * ldw + n] = (T)v;
}

}  // namespace

// The kernels of grouped16.h: whole 16-byte chunks and k-blocks, and offsets of 32 bits.
// padded: the rows of W are readable up to a multiple of 8 entries.
static bool direct_gemm(const GroupedGemm &g, bool padded = false) {
    return g.dtype != EMU_F32 && g.K >= 2 * BK && g.K % BK == 0 && aligned16(g.X) && aligned16(g.W) &&
           g.ldx % 8 == 0 && g.ldw % 8 == 0 && g.sw % 8 == 0 && (g.transb || padded || g.N % 8 == 0) && g.E > 0 &&
           (g.rows ? g.xrows : 256) * g.ldx * 2 < OFFSETS && 256 * g.ldw * 2 < OFFSETS &&
           (!g.rows || g.xrows > 0);
}
// Rows per expert up to which the kernel for few rows is the faster one.  Measured, us,
// that kernel and the other one, 64 experts of 2048 x 2048:
//   16 bits, copied straight to LDS   8 rows 112 and 124, 16 rows 119 and 94
//   float32                          32 rows 306 and 615 ('T' 303 to 343 and 433),
//                                    64 rows 600 and 623 ('T' 757 and 436)
//   16 bits, 2041 x 2041 'N'         30 rows 230 and 326, 50 rows 438 and 326
//                        'T'          8 rows 191 and 161
// A rule on the average: where the rows lie is known on the device only.  All rows at
// one of the 64 experts, whose matrix is then read again for each block: float32, 32
// rows on average, 227 and 259 ('T' 257 and 171), 16 bits, 8 rows, 45 and 18.
static int64_t few_rows(const GroupedGemm &g, bool direct) {
    return g.dtype == EMU_F32 || (!direct && !g.transb) ? FEW_ROWS : 8;
}

// Whether the direct kernels' tiles of 256 x 256 take less time than those of
// 128 x 128, `large` and `small` of them: rounds of one of the large ones or two of
// the small ones on a CU, the latter `two` of a round of the former long, or `one`
// where half the places stay empty.  Measured at 8192 x 8192 x 8192, in rounds: the
// product 0.58, the matrices' gradient 0.76; at 512 x 512 x 4096 (alone on a CU) 0.36.
// 4096 x 4096 x 4096: 124 and 139 us (the gradient 116 and 155); 4096 x 4352 x 4096:
// 188 and 156; 8 experts of 1024 x 1024 and 1000 rows, the gradient: 31 and 23.
static double rounds_of_large(int64_t large) {
    const int64_t cus = device_cu_count();
    return (double)((large + cus - 1) / cus);
}
static double rounds_of_small(int64_t small, double two, double one) {
    const int64_t cus = device_cu_count(), rest = small % (2 * cus);
    return small / (2 * cus) * two + (rest > cus ? two : (rest > 0 ? one : 0));
}

static hipError_t run_direct(const GroupedGemm &g, hipStream_t s) {
    auto tiles = [&](int64_t t) {               // an expert's last block is half full on average
        const int64_t blocks = (g.R + g.E * t / 2) / t, least = g.R < g.E ? g.R : g.E;
        return (blocks > least ? blocks : least) * ((g.N + t - 1) / t);
    };
    const int tile = rounds_of_large(tiles(256)) <= rounds_of_small(tiles(128), 0.58, 0.36) ? 256 : 128;
    return g.dtype == EMU_BF16 ? launch_gemm16_bf16(g, tile, s) : launch_gemm16_f16(g, tile, s);
}

// A 16-bit product on copies of the operands that the direct kernels cannot take, if
// that is faster than the kernels of grouped_staged.h: *done, or else nothing was
// launched.
// Those reach 550 TFLOP/s ('N' 330, whose matrix they transpose by narrow loads).  8
// experts of 2041 x 2041 with 1000 rows in bfloat16 'N': staged 237 us, on copies 109;
// 64 with 300 rows: 1270 and 462; 8191 x 8191 x 8191 'T': 1341 and 977, the gradient
// of its matrix 7358 and 1040.
static int realigned_gemm(const GroupedGemm &g, hipStream_t s, bool *done) {
    *done = false;
    if (g.dtype == EMU_F32 || g.K == 0 || g.E == 0) return EMU_OK;
    const int64_t K = g.K <= BK ? 2 * BK : up(g.K, BK), xr = g.rows && g.xrows <= g.R ? g.xrows : g.R;
    const bool pad = K != g.K, x = pad || !aligned16(g.X) || g.ldx % 8;
    const bool w = pad || !aligned16(g.W) || g.ldw % 8 || g.sw % 8 || (!g.transb && g.N % 8);
    const int *const map = xr < g.xrows ? g.rows : nullptr;     // through it into the copy
    const Realigned cx = {g.X, g.ldx, 0, g.rows ? g.xrows : g.R, g.K, map, 1, nullptr, 0, xr, K};
    const int mats = g.sw == 0 ? 1 : g.E;                       // one matrix for all experts
    const int *const offsets = g.sw == 0 ? nullptr : g.offsets;
    const Realigned cw = g.transb ? Realigned{g.W, g.ldw, g.sw, g.N, g.K, nullptr, mats, offsets, g.R, g.N, K}
                                  : Realigned{g.W, g.ldw, g.sw, g.K, g.N, nullptr, mats, offsets, g.R, K, up(g.N, 8)};
    const int64_t xb = x ? up(cx.bytes(), 256) : 0, wb = w ? cw.bytes() : 0;
    const double work = 2.0 * g.R * g.N * g.K / 1e6;            // operations per us at 1 TFLOP/s
    const double copied = work / 1000 + (x ? copy_time(cx) : 0) + (w ? copy_time(cw) : 0);
    if (copied >= work / (g.transb ? 550 : 330) || xb + wb > MOST_COPIED) return EMU_OK;
    GroupedGemm d = g;
    d.K = (int)K;
    if (x) {
        d.ldx = K;
        d.xrows = xr;
        if (map) d.rows = nullptr;
    }
    if (w) {
        d.ldw = cw.ld;
        d.sw = g.sw == 0 ? 0 : cw.rows * cw.ld;
    }
    if (x) d.X = nullptr;
    if (w) d.W = nullptr;
    if (!direct_gemm(d, w)) return EMU_OK;                      // offsets
    char *at = nullptr;
    if (int rc = api_try_workspace(xb + wb, &at)) return rc;
    if (!at) return EMU_OK;
    if (x) d.X = at;
    if (w) d.W = at + xb;
    *done = true;
    hipError_t e = x ? realign(cx, at, s) : hipSuccess;
    if (e == hipSuccess && w) e = realign(cw, at + xb, s);
    if (e == hipSuccess) e = run_direct(d, s);
    return api_done(e, "grouped_gemm");
}

int launch_grouped_gemm(const GroupedGemm &g, hipStream_t s) {
    const bool direct = direct_gemm(g), few = g.R <= few_rows(g, direct) * g.E;
    if (!few && !direct) {
        bool done;
        if (int rc = realigned_gemm(g, s, &done)) return rc;
        if (done) return EMU_OK;
    }
    hipError_t e;
    if (few) e = launch_few(g, s);
    else if (direct) e = run_direct(g, s);
    else if (g.dtype == EMU_F32) e = launch_staged_gemm_f32(g, s);
    else e = g.dtype == EMU_BF16 ? launch_staged_gemm_bf16(g, s) : launch_staged_gemm_f16(g, s);
    return api_done(e, "grouped_gemm");
}

// Pieces of an expert's rows where the matrices have too few tiles to fill the chip:
// each at least 128 rows long on average.  4 experts of 86 x 338 and 800 rows in
// float32: 48 us in one piece, 22 in two; 8 of 256 x 256 and 1000 rows 58 and 25.
static int pieces_of(const GroupedWgrad &g) {
    const int64_t tiles = (int64_t)g.E * ((g.M + 127) / 128) * ((g.N + 127) / 128);
    int n = 1;
    while (n < 16 && tiles * n * 2 <= device_cu_count() && g.R >= (int64_t)g.E * 256 * n) n *= 2;
    return n;
}

// How the direct kernels would compute a gradient: with tiles of 256 or 128, and
// copies of the operands that they cannot take as they are.  Row numbers of the
// k-block ahead arrive in time for the large tiles only (16 experts of 1280 x 1280 and
// 1000 rows: large 72 us, small 85, gathered 227): for the small ones the rows are
// copied into order.
struct DirectWgrad {
    int tile, pieces;
    bool p, q;                      // is copied
    Realigned cp, cq;
    double time;                    // us
    int64_t pb() const { return p ? up(cp.bytes(), 256) : 0; }
    int64_t qb() const { return q ? up(cq.bytes(), 256) : 0; }
};
static DirectWgrad direct_wgrad(const GroupedWgrad &g, int tile) {
    DirectWgrad w = {};
    w.tile = tile;
    w.pieces = tile == 128 ? pieces_of(g) : 1;
    const bool order = tile == 128;
    auto needs = [&](const void *X, int64_t ld, int n, const int *rows) {
        return !aligned16(X) || ld % 8 || n % 8 || ld * 2 >= OFFSETS || (rows && order);
    };
    auto copy = [&](const void *X, int64_t ld, int n, const int *rows, int64_t entries) {
        const bool through = rows && (order || entries > g.R);  // the fewer rows
        return Realigned{X, ld, 0, rows ? entries : g.R, n, through ? rows : nullptr, 1, nullptr, 0,
                         rows && !through ? entries : g.R, up(n, 8)};
    };
    w.p = needs(g.P, g.ldp, g.M, g.prow);
    w.q = needs(g.Q, g.ldq, g.N, g.qrow);
    w.cp = copy(g.P, g.ldp, g.M, g.prow, g.prows);
    w.cq = copy(g.Q, g.ldq, g.N, g.qrow, g.qrows);
    const int64_t tiles = (int64_t)g.E * ((g.M + tile - 1) / tile) * ((g.N + tile - 1) / tile);
    // a round of large tiles: 65536 sums of an expert's rows on every CU
    const double rounds = tile == 256 ? rounds_of_large(tiles) : rounds_of_small(tiles, 0.76, 0.45) / w.pieces;
    w.time = rounds * ((double)g.R / g.E * 0.028) + (w.p ? copy_time(w.cp) : 0) + (w.q ? copy_time(w.cq) : 0);
    return w;
}

int launch_grouped_wgrad(const GroupedWgrad &g, hipStream_t s) {
    GroupedWgrad d = g;
    const bool f32 = g.dtype == EMU_F32;
    bool direct = !f32 && g.R > 0 && (!g.prow || g.prows > 0) && (!g.qrow || g.qrows > 0);
    DirectWgrad w = {};
    if (direct) {
        const DirectWgrad large = direct_wgrad(g, 256), small = direct_wgrad(g, 128);
        w = large.time <= small.time ? large : small;
        // rounds of 128 x 128 tiles at 130 TFLOP/s
        const int64_t tiles = (int64_t)g.E * ((g.M + 127) / 128) * ((g.N + 127) / 128);
        const double staged = rounds_of_large(tiles) * ((double)g.R / g.E * 0.065);
        if ((w.p || w.q) && (w.time >= staged || w.pb() + w.qb() > MOST_COPIED)) w = large;
        if ((w.p || w.q) && (w.time >= staged || w.pb() + w.qb() > MOST_COPIED)) direct = false;
    }
    d.pieces = direct ? w.pieces : (f32 ? pieces_of(g) : 1);
    int64_t pb = direct ? w.pb() : 0, qb = direct ? w.qb() : 0;
    const int64_t ld = up(g.N, 4), sums = d.pieces > 1 ? 4 * (int64_t)d.pieces * g.E * g.M * ld : 0;
    char *at = nullptr;
    if (pb + qb + sums > 0)
        if (int rc = api_try_workspace(pb + qb + sums, &at)) return rc;
    if (pb + qb + sums > 0 && !at) {    // the operands as they are, every expert in one piece
        if (direct) w = direct_wgrad(g, 256);
        direct = direct && !w.p && !w.q;
        pb = qb = 0;
        d.pieces = 1;
    }
    hipError_t e = hipSuccess;
    if (pb > 0) {
        e = realign(w.cp, at, s);
        d.P = at;
        d.ldp = w.cp.ld;
        d.prows = w.cp.rows;
        if (w.cp.map) d.prow = nullptr;
    }
    if (e == hipSuccess && qb > 0) {
        e = realign(w.cq, at + pb, s);
        d.Q = at + pb;
        d.ldq = w.cq.ld;
        d.qrows = w.cq.rows;
        if (w.cq.map) d.qrow = nullptr;
    }
    if (e != hipSuccess) return api_done(e, "grouped_wgrad");
    if (d.pieces > 1) {
        d.dW = at + pb + qb;
        d.ldw = ld;
        d.sw = g.M * ld;
    }
    if (direct) e = g.dtype == EMU_BF16 ? launch_wgrad16_bf16(d, w.tile, s) : launch_wgrad16_f16(d, w.tile, s);
    else if (f32) e = launch_staged_wgrad_f32(d, s);
    else e = g.dtype == EMU_BF16 ? launch_staged_wgrad_bf16(d, s) : launch_staged_wgrad_f16(d, s);
    if (e != hipSuccess || d.pieces == 1) return api_done(e, "grouped_wgrad");
    with_type(g.dtype, [&](auto z) {
        using T = decltype(z);
        const dim3 grid((unsigned)(((int64_t)g.M * g.N + 255) / 256), g.E);
        join_kernel<T><<<grid, 256, 0, s>>>(reinterpret_cast<const float *>(d.dW), ld, g.M, g.N, d.pieces,
                                            static_cast<T *>(g.dW), g.ldw, g.sw);
    });
    return api_done(hipGetLastError(), "grouped_wgrad");
}

}  // namespace emu
