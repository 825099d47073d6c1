// The residual's addition and the root-mean-square norm of token rows, in one pass, with rows of 16 or 8 bits as the result:
//
//   h = x + residual (binary32);  sum_out = h rounded to the rows' type;  rstd = 1 / sqrt(mean(h^2) + eps);  p = h * weight (binary32)
//   16 bits:  out = p * rstd, rounded once.
//   8 bits:   a = max |p|;  out = rint(127 p / a), scale = a * rstd / 127: rstd does not enter the codes, so the sum of squares and the maximum are found
//             together, by one exchange between the warps.
//
// A bfloat16 row's squares may leave the binary32 range where the norm does not (above, or below 2^-90 under an eps that would show it).  A warp whose sums come near that
// takes them again of h 2^-96, or h 2^96, while the row is still in its registers; they count where the row's sum is out of range.
//
// 2048 x 8192 bf16: 25.4 us (134 MB, 5.3 TB/s), to 8 bits 37 to 42 (117 MB, 18 us: not bound by them; codes near a border divide in binary64); 2048 x 8191, no
// whole pieces and so element by element, 115 and 82 us.
// A row is a block's; its values stay in registers between the sum and the result, so that each is read once and written once.  Bound by those bytes where rows
// are many, by the chain load - exchange - store where they are few.  Rows too long for the registers are read again.
#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int MAX_T = 1024;
constexpr float MOST = 3.402823466e38f, MOST_OF_THREAD = 0x1p108f;       // the greatest finite number; sums of MAX_T threads' stay below it

template <bool BF16>
__device__ __forceinline__ float value_of(uint32_t h)
{
    return BF16 ? __uint_as_float(h << 16) : __half2float(__ushort_as_half((unsigned short)h));
}
template <bool BF16>
__device__ __forceinline__ uint32_t bits_of(float v)
{
    return BF16 ? (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(v)) : (uint32_t)__half_as_ushort(__float2half_rn(v));
}

// Eight neighbours as they lie in memory, from column j on; columns beyond the row are zeros.
template <bool VEC>
__device__ __forceinline__ uint4 load8(const uint16_t *row, int64_t j, int64_t cols)
{
    if constexpr (VEC) {
        return *reinterpret_cast<const uint4 *>(row + j);
    } else {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = j + e < cols ? (uint32_t)row[j + e] : 0u;
        return make_uint4(h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16);
    }
}
template <bool BF16>
__device__ __forceinline__ void values8(uint4 u, float v[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = value_of<BF16>((w[e / 2] >> (16 * (e & 1))) & 0xffffu);
}
template <bool BF16, bool VEC>
__device__ __forceinline__ void store8(uint16_t *row, int64_t j, int64_t cols, const float v[8])
{
    if (VEC) {
        uint32_t w[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = bits_of<BF16>(v[2 * u]) | bits_of<BF16>(v[2 * u + 1]) << 16;
        *reinterpret_cast<uint4 *>(row + j) = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (j + e < cols) row[j + e] = (uint16_t)bits_of<BF16>(v[e]);
    }
}

// The greater one, NaN where either is: a maximum that drops NaN would hide it under a finite scale.
__device__ __forceinline__ float greatest(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}

// rint(127 p / a), decided as by the exact quotient: the product with 127 / a is off by less than 2^-14, and within 5e-5 of a border the quotient is
// taken in binary64, where 127 p is exact and the rounding cannot reach a border that the exact quotient does not lie on.
__device__ __forceinline__ int code_of(float p, float a, float by)
{
    const float t = p * by;
    float r = rintf(t);
    if (!(fabsf(t - r) <= 0.49995f)) r = a > 0.0f ? (float)rint(127.0 * (double)p / (double)a) : 0.0f;      // (also where 127 / a overflows)
    return r == r ? (int)fminf(fmaxf(r, -127.0f), 127.0f) : 0;
}

// NV pieces of eight columns a thread, in registers; NV = 0: as many as the row takes, read again for the result.  A block goes from row to row, the next row's
// values on their way while the warps exchange this one's sums (2048 x 8192: a block for every row 29.3 us).
template <bool BF16, bool VEC, int NV>
__global__ void __launch_bounds__(NV == 4 ? 512 : MAX_T) skim_add_rmsnorm_kernel(SkimNorm n)
{
    __shared__ float sums[2][32], tops[2][32];
    __shared__ float again[BF16 ? 2 : 1][32];                // sums of squares of a warp that may be out of range, of h 2^96 or h 2^-96
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    const uint16_t *wr = static_cast<const uint16_t *>(n.weight);
    const int64_t step = (int64_t)blockDim.x * 8;
    auto x_of = [&](int64_t row) { return static_cast<const uint16_t *>(n.x) + row * n.ldx; };
    auto r_of = [&](int64_t row) { return static_cast<const uint16_t *>(n.residual) + row * n.ldr; };
    auto sum8 = [&](uint4 x, uint4 r, float h[8]) {
        values8<BF16>(x, h);
        if (n.residual) {
            float v[8];
            values8<BF16>(r, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += v[e];
        }
    };
    auto weighted8 = [&](int64_t j, const float h[8], float p[8]) {
        if (wr) values8<BF16>(load8<VEC>(wr, j, n.cols), p);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = wr ? h[e] * p[e] : h[e];
    };
    auto take8 = [&](const float h[8], const float p[8], float &sq, float &top) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            sq = fmaf(h[e], h[e], sq);
            top = greatest(top, fabsf(p[e]));
        }
    };
    auto again8 = [&](uint4 x, uint4 r, float by, float sq) {
        // (whole pieces as if unknown: kept from the first sum the values would cost every row registers; others are not packed on the way)
        if (VEC) asm volatile("" : "+r"(x.x), "+r"(x.y), "+r"(x.z), "+r"(x.w));
        float h[8];
        sum8(x, r, h);
#pragma unroll
        for (int e = 0; e < 8; ++e) sq = fmaf(h[e] * by, h[e] * by, sq);
        return sq;
    };
    const float least = BF16 && n.eps < 0x1p-70f ? 0x1p-90f : 0.0f;
    constexpr int M = NV ? NV : 1;
    uint4 xs[M], rs[M];
    auto ask = [&](int64_t row) {
        if constexpr (NV != 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int64_t j = v * step + tid * 8;
                if (j >= n.cols) break;
                xs[v] = load8<VEC>(x_of(row), j, n.cols);
                if (n.residual) rs[v] = load8<VEC>(r_of(row), j, n.cols);
            }
        }
    };
    int turn = 0;
    ask(blockIdx.x);
    for (int64_t row = blockIdx.x; row < n.rows; row += gridDim.x, turn ^= 1) {
        uint16_t *sr = n.sum_out ? static_cast<uint16_t *>(n.sum_out) + row * n.lds : nullptr;
        float sq = 0.0f, top = 0.0f;
        float p[M][8];
        if constexpr (NV != 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int64_t j = v * step + tid * 8;
                if (j >= n.cols) break;
                float h[8];
                sum8(xs[v], rs[v], h);
                weighted8(j, h, p[v]);
                if (sr) store8<BF16, VEC>(sr, j, n.cols, h);
                take8(h, p[v], sq, top);
            }
        } else {
            for (int64_t j = tid * 8; j < n.cols; j += step) {
                float h[8];
                sum8(load8<VEC>(x_of(row), j, n.cols), n.residual ? load8<VEC>(r_of(row), j, n.cols) : make_uint4(0u, 0u, 0u, 0u), h);
                weighted8(j, h, p[0]);
                take8(h, p[0], sq, top);
            }
        }
        if constexpr (BF16) {
            // in range for all threads: so is any sum of them; below it for all: the warp's may be
            if (__any_sync(0xffffffffu, !(sq >= least && sq <= MOST_OF_THREAD))) {
                const float by = __any_sync(0xffffffffu, sq > MOST_OF_THREAD) ? 0x1p-96f : 0x1p96f;
                float d = 0.0f;
                if constexpr (NV != 0) {
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        if (v * step + tid * 8 >= n.cols) break;
                        d = again8(xs[v], rs[v], by, d);
                    }
                } else {
                    for (int64_t j = tid * 8; j < n.cols; j += step) d = again8(load8<VEC>(x_of(row), j, n.cols), n.residual ? load8<VEC>(r_of(row), j, n.cols) : make_uint4(0u, 0u, 0u, 0u), by, d);
                }
#pragma unroll
                for (int off = 16; off; off >>= 1) d += __shfl_xor_sync(0xffffffffu, d, off);
                if (lane == 0) again[turn][warp] = d;
            }
        }
        if (NV != 0 && row + gridDim.x < n.rows) ask(row + gridDim.x);
#pragma unroll
        for (int off = 16; off; off >>= 1) {
            sq += __shfl_xor_sync(0xffffffffu, sq, off);
            top = greatest(top, __shfl_xor_sync(0xffffffffu, top, off));
        }
        if (lane == 0) {
            sums[turn][warp] = sq;
            tops[turn][warp] = top;
        }
        __syncthreads();                                     // (the next row's sums go to the other places: one barrier a row)
        sq = lane < warps ? sums[turn][lane] : 0.0f;
        top = lane < warps ? tops[turn][lane] : 0.0f;
#pragma unroll
        for (int off = 16; off; off >>= 1) {
            sq += __shfl_xor_sync(0xffffffffu, sq, off);
            top = greatest(top, __shfl_xor_sync(0xffffffffu, top, off));
        }
        float eps = n.eps, root = 1.0f, lift = 1.0f;         // rstd = root / sqrt(mean + eps), and p takes lift before it: 1 / sqrt may be beyond the range where the result is not
        if constexpr (BF16) {
            if (sq < least || sq > MOST) {                   // the same for the whole block.  (One by one: with shuffles here p was spilled)
                const bool small = sq < least;
                const float by = small ? 0x1p96f : 0x1p-96f;
                sq = 0.0f;
#pragma unroll 1
                for (int w = 0; w < warps; ++w) {
                    const float of = sums[turn][w];
                    sq += of >= least && of <= MOST ? of * by * by : small == (of < least) ? again[turn][w] : 0.0f;
                }
                eps = eps * by * by;
                root = by;
                if (small && sq / (float)n.cols + eps < 0x1p-8f) {
                    lift = 0x1p64f;
                    root = 0x1p32f;
                    if (NV != 0 && n.out_type != SKIM_TYPE_I8) {         // (8 bits: the codes are of p as it is)
#pragma unroll
                        for (int v = 0; v < NV; ++v)
#pragma unroll
                            for (int e = 0; e < 8; ++e) p[v][e] *= 0x1p64f;
                    }
                }
            }
        }
        const float rstd = 1.0f / sqrtf(sq / (float)n.cols + eps) * root;
        if (n.out_scale && tid == 0) n.out_scale[row] = top * rstd / 127.0f * lift;
        const float by = top > 0.0f ? 127.0f / top : 0.0f;
        auto result8 = [&](int64_t j, float v[8]) {
            if (n.out_type == SKIM_TYPE_I8) {
                int8_t *o = static_cast<int8_t *>(n.out) + row * n.ldo;
                uint32_t w[2] = {0u, 0u};
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(code_of(v[e], top, by) & 255) << (8 * (e & 3));
                if (VEC) {
                    *reinterpret_cast<uint2 *>(o + j) = make_uint2(w[0], w[1]);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (j + e < n.cols) o[j + e] = (int8_t)(w[e / 4] >> (8 * (e & 3)));
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (BF16 && NV == 0 ? v[e] * lift : v[e]) * rstd;
                store8<BF16, VEC>(static_cast<uint16_t *>(n.out) + row * n.ldo, j, n.cols, v);
            }
        };
        if constexpr (NV != 0) {
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const int64_t j = v * step + tid * 8;
                if (j < n.cols) result8(j, p[v]);
            }
        } else {
            for (int64_t j = tid * 8; j < n.cols; j += step) {
                float h[8];
                sum8(load8<VEC>(x_of(row), j, n.cols), n.residual ? load8<VEC>(r_of(row), j, n.cols) : make_uint4(0u, 0u, 0u, 0u), h);
                weighted8(j, h, p[0]);
                if (sr) store8<BF16, VEC>(sr, j, n.cols, h);
                result8(j, p[0]);
            }
        }
    }
}

template <bool BF16, bool VEC>
int launch(skim_ctx *ctx, const SkimNorm &n)
{
    // a warp for every 256 columns; from 2048 columns on more pieces a thread where rows are many.  Many rows are dealt to as many blocks as the SMs hold.
    // (bfloat16 rows that are no whole pieces: four a thread 140 us, two 116, 2048 x 8191.)
    constexpr int MOST_PIECES = BF16 && !VEC ? 2 : 4;
    const int64_t pieces = (n.cols + 7) / 8;
    int nv = 1;
    while (nv < MOST_PIECES && (pieces > (int64_t)nv * MAX_T || (n.rows > ctx->sm_count && pieces >= (int64_t)nv * 256))) nv *= 2;
    if (pieces > (nv == 4 ? 4 * 512 : nv * MAX_T)) nv = 0;
    const int64_t threads = nv ? (pieces + nv - 1) / nv : MAX_T;
    const unsigned block = (unsigned)((threads + 31) / 32 * 32);
    const int64_t held = (int64_t)ctx->sm_count * (block <= 64 ? 16 : nv == 4 ? (512 / block > 0 ? 512 / block : 1) : 1024 / block);
    const dim3 grid((unsigned)(nv && n.rows > held ? held : n.rows));
    switch (nv) {
    case 1: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 1>, grid, block, 0, n);
    case 2: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 2>, grid, block, 0, n);
    case 4: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, MOST_PIECES>, grid, block, 0, n);
    default: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 0>, grid, block, 0, n);
    }
}

}  // namespace

int skim_launch_add_rmsnorm(skim_ctx *ctx, const SkimNorm &n)
{
    if (n.rows == 0) return SKIM_OK;
    auto whole = [](const void *p, int64_t ld, unsigned bytes) { return !p || (reinterpret_cast<uintptr_t>(p) % bytes == 0 && ld % 8 == 0); };
    const bool vec = n.cols % 8 == 0 && whole(n.x, n.ldx, 16) && whole(n.residual, n.ldr, 16) && whole(n.weight, 0, 16) && whole(n.sum_out, n.lds, 16) &&
                     whole(n.out, n.ldo, n.out_type == SKIM_TYPE_I8 ? 8 : 16);
    if (n.type == SKIM_TYPE_BF16) return vec ? launch<true, true>(ctx, n) : launch<true, false>(ctx, n);
    return vec ? launch<false, true>(ctx, n) : launch<false, false>(ctx, n);
}
