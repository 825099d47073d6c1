// Uniform 4-bit quantisation with a scale and a zero point per group of 32, 64 or 128 columns, the form that SKIM (arXiv 2412.04180)
// compares its codebooks with, into the stored form of skim_grouped.cuh, and back.
//
//   low = min(0, min x), high = max(0, max x) of the group;  s = binary16((high - low) / 15);  z = clamp(rint(-low / s), 0, 15)
//   q = clamp(rint(x / s) + z, 0, 15);  the value a code stands for is (q - z) s.
//
// Rounding to whole numbers is decided as by exact quotients: x / s in binary32 with correct rounding never lands on a border k + 1/2 that the exact quotient
// misses (k + 1/2 has 5 bits, s 11, x 24, so x - (k + 1/2) s is zero or at least 2^-23 of x, more than the half unit that the rounding can move).  The
// kernel multiplies by 1 / s instead and divides only where the quotient comes within 2^-15 of a border, or of the limits of the codes.
//
// Both kernels stream: weights (and importances) in, half a byte a weight out, or the other way round.  A thread has one row's four runs of eight
// columns of a record, so the group's extremes are two shuffles within a quad, its 16 bytes of codes leave in one store, and a row's error
// stays in a register until the row ends.  4096 x 11008, groups of 128: quantised with importances in 62 us (294 MB, 4.7 TB/s; 16 warps an SM of 117 registers do not cover
// the loads), without 42, with an installed scale vector 83 and 62; back in 19 us (114 MB, 6.0 TB/s).  Rows that do not lie at whole 16-byte pieces are moved element by element, lanes
// 16 bytes apart, so every instruction touches all the sectors of its span: 4096 x 11007 118 us, without importances 72, back 184.
#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int QT = 256, QW = QT / 32;    // a block has 8 rows, its warps every eighth record

struct QuantArgs {
    const uint16_t *W;
    const float *g;          // importance or nullptr
    const float *r;          // reciprocal of the installed scale vector or nullptr
    int64_t rows, cols, ld;
    int ct, record;
    int vec, gvec;           // 16-byte loads of weights, of importances
    unsigned char *tiles;
    float *err;              // nullptr: the importances are looked over all the same
    unsigned long long *status;
};

// Least and greatest of the eight values of four words and of `low`, `high`; NaN where there is one.
__device__ __forceinline__ void extremes(const uint32_t raw[4], __half2 &low, __half2 &high)
{
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        low = __hmin2_nan(low, bits_half2(raw[u]));
        high = __hmax2_nan(high, bits_half2(raw[u]));
    }
}

template <int PER, bool SCALED, bool ERR>
__global__ void __launch_bounds__(QT, 2) skim_grouped_quantize_kernel(QuantArgs a)
{
    __shared__ float sums[QW][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, p = lane & 3;
    const int64_t row = (int64_t)blockIdx.x * 8 + (lane >> 2);
    const bool live = row < a.rows;
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    const uint16_t *Wr = a.W + row * a.ld;
    const float *Gr = ERR && a.g ? a.g + row * a.ld : nullptr;
    unsigned char *tile = a.tiles + (row / SKIM_RECORD_ROWS) * a.ct * (int64_t)a.record;
    const int in_tile = (int)(row % SKIM_RECORD_ROWS);
    float err = 0.0f;
    bool bad = false, bad_g = false;
    for (int c = warp; c < a.ct; c += QW) {
        const int64_t first = (int64_t)c * SKIM_RECORD_COLS + 8 * p;
        uint32_t raw[4][4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t j = first + 32 * t;
            uint4 v = make_uint4(0u, 0u, 0u, 0u);
            if (live && j < a.cols) {
                if (a.vec && j + 8 <= a.cols) {
                    v = __ldcs(reinterpret_cast<const uint4 *>(Wr + j));
                } else {
                    uint32_t h[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) h[e] = j + e < a.cols ? (uint32_t)Wr[j + e] : 0u;
                    v = make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
                }
            }
            raw[t][0] = v.x; raw[t][1] = v.y; raw[t][2] = v.z; raw[t][3] = v.w;
        }
        float g[4][8];
        if (ERR) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int64_t j = first + 32 * t;
                if (Gr && a.gvec && live && j + 8 <= a.cols) {
                    const float4 u = __ldcs(reinterpret_cast<const float4 *>(Gr + j)), v = __ldcs(reinterpret_cast<const float4 *>(Gr + j + 4));
                    g[t][0] = u.x; g[t][1] = u.y; g[t][2] = u.z; g[t][3] = u.w; g[t][4] = v.x; g[t][5] = v.y; g[t][6] = v.z; g[t][7] = v.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) g[t][e] = Gr && live && j + e < a.cols ? Gr[j + e] : 1.0f;
                }
            }
        }
        // the clustered value of element e of run t
        auto value = [&](int t, int e) {
            const float w = __half2float(__ushort_as_half((unsigned short)(raw[t][e / 2] >> (16 * (e & 1)))));
            if (!SCALED) return w;
            const int64_t j = first + 32 * t + e;
            return __fmul_rn(w, j < a.cols ? a.r[j] : 0.0f);
        };
        float low[PER], high[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            __half2 lo = bits_half2(0u), hi = bits_half2(0u);
#pragma unroll
            for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t) extremes(raw[t], lo, hi);
            const float l = __low2float(lo), m = __high2float(lo), n = __low2float(hi), o = __high2float(hi);
            bad |= !(l >= -65504.0f && m >= -65504.0f && n <= 65504.0f && o <= 65504.0f);
            low[k] = fminf(l, m);
            high[k] = fmaxf(n, o);
            if (SCALED) {
                low[k] = high[k] = 0.0f;
#pragma unroll
                for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = value(t, e);
                        low[k] = fminf(low[k], x);
                        high[k] = fmaxf(high[k], x);
                    }
            }
        }
        uint32_t meta[PER], word[4];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
#pragma unroll
            for (int off = 1; off < 4; off <<= 1) {
                low[k] = fminf(low[k], __shfl_xor_sync(0xffffffffu, low[k], off));
                high[k] = fmaxf(high[k], __shfl_xor_sync(0xffffffffu, high[k], off));
            }
            const __half h = __float2half_rn(__fdiv_rn(__fsub_rn(high[k], low[k]), 15.0f));
            const float s = __half2float(h);
            const bool some = s > 0.0f;
            bad |= !(s <= 65504.0f);                         // scaled values may leave the range
            const float by = some ? __frcp_rn(s) : 0.0f;     // no scale: every quotient, code and zero point is 0
            const float z = some ? fminf(rintf(__fdiv_rn(-low[k], s)), 15.0f) : 0.0f;
            const float least = -z, most = some ? 15.0f - z : 0.0f, as_code = z + 8388608.0f, border = s * (0.5f - 0x1p-15f);
            meta[k] = (uint32_t)__half_as_ushort(h) | (uint32_t)(int)z << 16;
#pragma unroll
            for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t) {
                // code - z is the quotient's whole number (by way of 1.5 * 2^23) within its limits, which keeps what is left of x at hand: that is the
                // error, and says whether the quotient came near a border
                uint32_t codes = 0x05000000u;                // less what the eight binary32 images add
                float left[8], far = 0.0f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = value(t, e), q = fminf(fmaxf(__fadd_rn(__fmaf_rn(x, by, 12582912.0f), -12582912.0f), least), most);
                    left[e] = __fmaf_rn(-q, s, x);
                    far = fmaxf(far, fabsf(left[e]));
                    codes += __float_as_uint(q + as_code) << (4 * nibble_of(e));
                }
                if (far > border && some) {
                    codes = 0x05000000u;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = value(t, e), q = fminf(fmaxf(rintf(__fdiv_rn(x, s)), least), most);
                        left[e] = __fmaf_rn(-q, s, x);
                        codes += __float_as_uint(q + as_code) << (4 * nibble_of(e));
                    }
                }
                word[t] = codes;
                if (ERR) {
                    if (Gr) {
                        uint32_t top = 0u;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            top = max(top, __float_as_uint(g[t][e]));
                            err = fmaf(left[e] * left[e], g[t][e], err);
                        }
                        if (top >= 0x7f800000u) {            // infinite, NaN or negative, or a negative zero among the others
#pragma unroll
                            for (int e = 0; e < 8; ++e) bad_g |= !(g[t][e] >= 0.0f && g[t][e] <= 3.402823466e38f);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) err = fmaf(left[e], left[e], err);
                    }
                }
            }
        }
        // columns and rows beyond the matrix came in as zeros; a ragged group's codes there are its zero point
        unsigned char *rec = tile + (int64_t)c * a.record;
        if ((int64_t)(c + 1) * SKIM_RECORD_COLS > a.cols) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (first + 32 * t + e >= a.cols) word[t] &= ~(15u << (4 * nibble_of(e)));
        }
        *reinterpret_cast<uint4 *>(rec + in_tile * 64 + p * 16) = make_uint4(word[0], word[1], word[2], word[3]);
        uint32_t mine = meta[0];
#pragma unroll
        for (int k = 1; k < PER; ++k)
            if (p == k) mine = meta[k];
        if (p < PER) reinterpret_cast<uint32_t *>(rec + SKIM_RECORD_CODES)[in_tile * PER + p] = mine;
    }
    if (live && bad) atomicOr(a.status, (unsigned long long)SKIM_STATUS_BAD_WEIGHT);
    if (ERR) {
        if (live && bad_g) atomicOr(a.status, (unsigned long long)SKIM_STATUS_BAD_IMPORTANCE);
        err += __shfl_xor_sync(0xffffffffu, err, 1);
        err += __shfl_xor_sync(0xffffffffu, err, 2);
        if (p == 0) sums[warp][lane >> 2] = err;
        __syncthreads();
        if (a.err && threadIdx.x < 8 && (int64_t)blockIdx.x * 8 + threadIdx.x < a.rows) {
            float v = sums[0][threadIdx.x];
#pragma unroll
            for (int w = 1; w < QW; ++w) v += sums[w][threadIdx.x];
            a.err[(int64_t)blockIdx.x * 8 + threadIdx.x] = v;
        }
    }
}

// ---------------------------------------------------------------- back to binary16

constexpr int DT = 256, DW = DT / 32, AHEAD = 4;      // a warp has 8 rows of four records

struct BackArgs {
    const unsigned char *tiles;
    int64_t rows, cols, ld;
    int ct, record, spans;   // spans of AHEAD records in a row of records
    int vec;
    uint16_t *out;
};

// (q - z) s in binary16 arithmetic is the exact product rounded once.
template <int PER>
__global__ void __launch_bounds__(DT) skim_grouped_dequantize_kernel(BackArgs a)
{
    const int lane = threadIdx.x & 31, p = lane & 3;
    const int64_t unit = (int64_t)blockIdx.x * DW + (threadIdx.x >> 5);
    const int64_t half = unit / a.spans, row = half * 8 + (lane >> 2);
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    if (row >= a.rows) return;
    const int c0 = (int)(unit % a.spans) * AHEAD;
    const unsigned char *rec = a.tiles + ((row / SKIM_RECORD_ROWS) * a.ct + c0) * (int64_t)a.record;
    const int in_tile = (int)(row % SKIM_RECORD_ROWS);
    uint4 w[AHEAD];
    uint32_t meta[AHEAD][PER];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
        if (c0 + u < a.ct) {
            w[u] = __ldg(reinterpret_cast<const uint4 *>(rec + (int64_t)u * a.record + in_tile * 64 + p * 16));
#pragma unroll
            for (int k = 0; k < PER; ++k) meta[u][k] = __ldg(reinterpret_cast<const uint32_t *>(rec + (int64_t)u * a.record + SKIM_RECORD_CODES) + in_tile * PER + k);
        }
    uint16_t *dst = a.out + row * a.ld;
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) {
        if (c0 + u >= a.ct) break;
        const uint32_t word[4] = {w[u].x, w[u].y, w[u].z, w[u].w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t m = meta[u][t * PER / 4];
            const Zero<false> z(m);
            const __half2 s = bits_half2(__byte_perm(m, 0u, 0x1010));
            uint32_t v[4];
            expand(word[t], z, v);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = half2_bits(__hmul2(bits_half2(v[i]), s));
            const int64_t j = (int64_t)(c0 + u) * SKIM_RECORD_COLS + 32 * t + 8 * p;
            if (a.vec && j + 8 <= a.cols) {
                *reinterpret_cast<uint4 *>(dst + j) = make_uint4(v[0], v[1], v[2], v[3]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (j + e < a.cols) dst[j + e] = (uint16_t)(v[e / 2] >> (16 * (e & 1)));
            }
        }
    }
}

// ---------------------------------------------------------------- token rows at any address, copied to whole 16-byte pieces

// A block has a token; a thread moves words of the copy, so a warp's loads lie side by side.
template <typename E>
__global__ void __launch_bounds__(256) skim_align_rows_kernel(const E *x, int64_t ldx, int cols, uint32_t *out, int words)
{
    constexpr int N = 4 / sizeof(E);
    const int64_t token = blockIdx.x;
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    const E *row = x + token * ldx;
    for (int w = threadIdx.x; w < words; w += 256) {
        uint32_t v = 0u;
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (w * N + e < cols) v |= (uint32_t)row[w * N + e] << (8 * sizeof(E) * e);
        out[token * words + w] = v;
    }
}

}  // namespace

int skim_launch_grouped_quantize(skim_ctx *ctx, const uint16_t *W, const float *importance, const float *rscale, int64_t rows, int64_t cols, int64_t ld, int group,
                                 unsigned char *tiles, float *err)
{
    if (rows == 0) return SKIM_OK;
    QuantArgs a;
    a.W = W; a.g = importance; a.r = rscale; a.rows = rows; a.cols = cols; a.ld = ld;
    a.ct = (int)skim_record_tiles(cols, SKIM_RECORD_COLS);
    a.record = skim_record_bytes(group);
    a.vec = (reinterpret_cast<uintptr_t>(W) & 15u) == 0 && ld % 8 == 0;
    a.gvec = (reinterpret_cast<uintptr_t>(importance) & 15u) == 0 && ld % 4 == 0;
    a.tiles = tiles; a.err = err;
    a.status = (unsigned long long *)ctx->ws;
    const dim3 grid((unsigned)(skim_record_tiles(rows, SKIM_RECORD_ROWS) * 2));     // whole records: rows beyond the last are zeros
    const int per = SKIM_RECORD_COLS / group;
    const bool with_err = err || importance;
#define SKIM_QUANT(P)                                                                                                                                  \
    return rscale ? (with_err ? skim_launch_dependent(ctx, skim_grouped_quantize_kernel<P, true, true>, grid, QT, 0, a)                                      \
                         : skim_launch_dependent(ctx, skim_grouped_quantize_kernel<P, true, false>, grid, QT, 0, a))                                    \
                  : (with_err ? skim_launch_dependent(ctx, skim_grouped_quantize_kernel<P, false, true>, grid, QT, 0, a)                                     \
                         : skim_launch_dependent(ctx, skim_grouped_quantize_kernel<P, false, false>, grid, QT, 0, a))
    if (per == 1) { SKIM_QUANT(1); }
    if (per == 2) { SKIM_QUANT(2); }
    SKIM_QUANT(4);
#undef SKIM_QUANT
}

int skim_launch_grouped_dequantize(skim_ctx *ctx, const unsigned char *tiles, int64_t rows, int64_t cols, int group, uint16_t *out, int64_t ld_out)
{
    if (rows == 0) return SKIM_OK;
    BackArgs a;
    a.tiles = tiles; a.rows = rows; a.cols = cols; a.ld = ld_out;
    a.ct = (int)skim_record_tiles(cols, SKIM_RECORD_COLS);
    a.record = skim_record_bytes(group);
    a.spans = (a.ct + AHEAD - 1) / AHEAD;
    a.vec = (reinterpret_cast<uintptr_t>(out) & 15u) == 0 && ld_out % 8 == 0;
    a.out = out;
    const int64_t units = skim_record_tiles(rows, 8) * a.spans, blocks = (units + DW - 1) / DW;
    if (blocks > 0x7fffffff) return SKIM_ERR_SHAPE;
    const dim3 grid((unsigned)blocks);
    switch (SKIM_RECORD_COLS / group) {
    case 1: return skim_launch_dependent(ctx, skim_grouped_dequantize_kernel<1>, grid, DT, 0, a);
    case 2: return skim_launch_dependent(ctx, skim_grouped_dequantize_kernel<2>, grid, DT, 0, a);
    default: return skim_launch_dependent(ctx, skim_grouped_dequantize_kernel<4>, grid, DT, 0, a);
    }
}

// Elements between rows of the copy.
int64_t skim_aligned_stride(int64_t cols, int x_type)
{
    const int64_t piece = x_type == SKIM_TYPE_I8 ? 16 : 8;
    return (cols + piece - 1) / piece * piece;
}
int skim_launch_align_rows(skim_ctx *ctx, const SkimGroupedProduct &p, void *scratch)
{
    const int bytes = p.x_type == SKIM_TYPE_I8 ? 1 : 2, words = (int)(skim_aligned_stride(p.cols, p.x_type) * bytes / 4);
    const dim3 grid((unsigned)p.tokens);
    if (bytes == 1) return skim_launch_dependent(ctx, skim_align_rows_kernel<uint8_t>, grid, 256, 0, static_cast<const uint8_t *>(p.x), p.ldx, (int)p.cols, static_cast<uint32_t *>(scratch), words);
    return skim_launch_dependent(ctx, skim_align_rows_kernel<uint16_t>, grid, 256, 0, static_cast<const uint16_t *>(p.x), p.ldx, (int)p.cols, static_cast<uint32_t *>(scratch), words);
}
