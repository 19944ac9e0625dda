// Which kernel runs a product of 8-bit integers, and copies of operands whose rows are not
// multiples of 16 bytes.
#include <cstdlib>
#include "api_state.h"
#include "emu_internal.h"
#include "moe.h"
#include "moe_common.h"

namespace emu {
namespace {

constexpr int64_t OFFSETS = (int64_t)1 << 32;        // what a copy's 32-bit offset spans
constexpr int64_t MOST_COPIED = (int64_t)1 << 33;    // bytes of workspace for copies

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
int64_t up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

// A matrix (or one for each expert) of 8-bit integers as the copy has it: rows x ld, ld a
// multiple of 16, zeros behind the entries that exist.
struct Copied {
    const int8_t *src;
    int64_t lds, stride, src_rows;
    int cols;
    const int *map;                 // row r is row map[r] of the source (zeros if it has none); or null
    int mats;
    const int *offsets;             // matrix e is copied if expert e has rows; or null
    int64_t R;                      // of offsets
    int64_t rows, ld;
    int64_t bytes() const { return mats * rows * ld; }
};

// 16 bytes a thread: unaligned loads, aligned stores.  Bound by bytes.
__global__ __launch_bounds__(256) void q8_copy_kernel(Copied m, int8_t *__restrict__ dst) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int per_row = (int)(m.ld / 16);
    const int64_t row = i / per_row;
    const int c = (int)(i % per_row) * 16;
    if (row >= m.rows) return;
    typedef int i32x4 __attribute__((ext_vector_type(4)));
    typedef int __attribute__((ext_vector_type(4), aligned(1))) unaligned;
    for (int e = blockIdx.y; e < m.mats; e += gridDim.y) {
        if (m.offsets) {
            int64_t lo, hi;
            expert_rows(m.offsets, m.mats, m.R, e, lo, hi);
            if (lo == hi) continue;
        }
        const int64_t at = m.map ? m.map[row] : row;
        i32x4 v = {};
        if (at >= 0 && at < m.src_rows) {
            const int8_t *const p = m.src + e * m.stride + at * m.lds + c;
            if (c + 16 <= m.cols) {
                v = *reinterpret_cast<const unaligned *>(p);
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    if (c + j < m.cols) v[j / 4] |= (int)(uint8_t)p[j] << (8 * (j % 4));
            }
        }
        *reinterpret_cast<i32x4 *>(dst + (e * m.rows + row) * m.ld + c) = v;
    }
}
hipError_t copy(const Copied &m, char *dst, hipStream_t s) {
    const dim3 grid((unsigned)((m.rows * m.ld / 16 + 255) / 256), m.mats < 32768 ? m.mats : 32768);
    q8_copy_kernel<<<grid, 256, 0, s>>>(m, reinterpret_cast<int8_t *>(dst));
    return hipGetLastError();
}

// The kernel of q8_tiles.h: rows of whole 16-byte chunks, and offsets of 32 bits.
bool fits_tiles(const Q8Gemm &g) {
    return g.K > 0 && g.K % 16 == 0 && g.E > 0 && aligned16(g.X) && aligned16(g.W) && g.ldx % 16 == 0 &&
           g.ldw % 16 == 0 && g.sw % 16 == 0 && (g.rows ? g.xrows : 256) * g.ldx < OFFSETS && 256 * g.ldw < OFFSETS &&
           (!g.rows || g.xrows > 0);
}

hipError_t run_tiles_kernel(const Q8Gemm &g, hipStream_t s) {
    const int64_t cus = device_cu_count();
    auto tiles = [&](int64_t t) {               // an expert's last block is half full on average
        const int64_t blocks = (g.R + g.E * t / 2) / t, least = g.R < g.E ? g.R : g.E;
        return (blocks > least ? blocks : least) * ((g.N + t - 1) / t);
    };
    const int64_t small = tiles(128), rest = small % (2 * cus);
    const double large = (double)((tiles(256) + cus - 1) / cus);
    Q8Tiles how = large <= small / (2 * cus) * 0.58 + (rest > cus ? 0.58 : (rest > 0 ? 0.36 : 0)) ? Q8Tiles::LARGE : Q8Tiles::SMALL;
    if (const char *e = getenv("Q8HOW")) how = (Q8Tiles)atoi(e);
    if (g.dtype == EMU_F32) return launch_q8_tiles_f32(g, how, s);
    return g.dtype == EMU_BF16 ? launch_q8_tiles_bf16(g, how, s) : launch_q8_tiles_f16(g, how, s);
}

}  // namespace

int launch_q8_gemm(const Q8Gemm &g, hipStream_t s) {
    const bool few = g.R <= 16 * (int64_t)g.E || g.K == 0 || g.E == 0 || (g.rows && g.xrows == 0);
    if (few) return api_done(launch_q8_few(g, s), "q8_gemm");
    if (fits_tiles(g)) return api_done(run_tiles_kernel(g, s), "q8_gemm");
    // the rows of X through their numbers into the copy, where those are fewer
    const int *const map = g.rows && g.xrows > g.R ? g.rows : nullptr;
    const int64_t K = up(g.K, 16), xr = g.rows && !map ? g.xrows : g.R;
    const bool pad = K != g.K, x = pad || !aligned16(g.X) || g.ldx % 16 || (map && g.xrows * g.ldx >= OFFSETS);
    const bool w = pad || !aligned16(g.W) || g.ldw % 16 || g.sw % 16;
    const int mats = g.sw == 0 ? 1 : g.E;                       // one matrix for all experts
    const Copied cx = {g.X, g.ldx, 0, g.xrows, g.K, map, 1, nullptr, 0, xr, K};
    const Copied cw = {g.W, g.ldw, g.sw, g.N, g.K, nullptr, mats, g.sw == 0 ? nullptr : g.offsets, g.R, g.N, K};
    const int64_t xb = x ? up(cx.bytes(), 256) : 0, wb = w ? cw.bytes() : 0;
    Q8Gemm d = g;
    d.K = (int)K;
    if (x) {
        d.X = nullptr;
        d.ldx = K;
        if (map) d.rows = nullptr;
    }
    if (w) {
        d.W = nullptr;
        d.ldw = K;
        d.sw = g.sw == 0 ? 0 : cw.rows * K;
    }
    char *at = nullptr;
    if (fits_tiles(d) && xb + wb <= MOST_COPIED)
        if (int rc = api_try_workspace(xb + wb, &at)) return rc;
    if (!at) return api_done(launch_q8_few(g, s), "q8_gemm");
    if (x) d.X = reinterpret_cast<int8_t *>(at);
    if (w) d.W = reinterpret_cast<int8_t *>(at + xb);
    hipError_t e = x ? copy(cx, at, s) : hipSuccess;
    if (e == hipSuccess && w) e = copy(cw, at + xb, s);
    if (e == hipSuccess) e = run_tiles_kernel(d, s);
    return api_done(e, "q8_gemm");
}

}  // namespace emu
