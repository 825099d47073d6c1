// The residual's addition and the root-mean-square norm of token rows, in one pass, with rows of 16 or 8 bits as the result:
//
//   h = x + residual (binary32);  sum_out = h rounded to the rows' type;  rstd = 1 / sqrt(mean(h^2) + eps);  p = h * weight (binary32)
//   16 bits:  out = p * rstd, rounded once.
//   8 bits:   a = max |p|;  out = rint(127 p / a), scale = a * rstd / 127: rstd does not enter the codes, so the sum of squares and the maximum are found
//             together, by one exchange between the warps.
//
// A row is a block's; its values stay in registers between the sum and the result, so that each is read once and written once.  Bound by those bytes where rows
// are many, by the chain load - exchange - store where they are few.  Rows too long for the registers are read again.
#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int MAX_T = 1024;

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

// Eight values from column j on; columns beyond the row are zeros.
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const uint16_t *row, int64_t j, int64_t cols, float v[8])
{
    if (VEC) {
        const uint4 u = *reinterpret_cast<const uint4 *>(row + j);
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = value_of<BF16>((w[e / 2] >> (16 * (e & 1))) & 0xffffu);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = j + e < cols ? value_of<BF16>(row[j + e]) : 0.0f;
    }
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

// rint(127 p / a), decided as by the exact quotient: the product with 127 / a is off by less than 2^-14, and within 5e-5 of a border the quotient is
// taken in binary64, where 127 p is exact and the rounding cannot reach a border that the exact quotient does not lie on.
__device__ __forceinline__ int code_of(float p, float a, float by)
{
    const float t = p * by;
    float r = rintf(t);
    if (!(fabsf(t - r) <= 0.49995f)) r = a > 0.0f ? (float)rint(127.0 * (double)p / (double)a) : 0.0f;      // (also where 127 / a overflows)
    return r == r ? (int)fminf(fmaxf(r, -127.0f), 127.0f) : 0;
}

// NV pieces of eight columns a thread, in registers; NV = 0: as many as the row takes, read again for the result.
template <bool BF16, bool VEC, int NV>
__global__ void __launch_bounds__(MAX_T) skim_add_rmsnorm_kernel(SkimNorm n)
{
    __shared__ float sums[32], tops[32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, warps = blockDim.x >> 5;
    const int64_t row = blockIdx.x;
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    const uint16_t *xr = static_cast<const uint16_t *>(n.x) + row * n.ldx;
    const uint16_t *rr = n.residual ? static_cast<const uint16_t *>(n.residual) + row * n.ldr : nullptr;
    const uint16_t *wr = static_cast<const uint16_t *>(n.weight);
    uint16_t *sr = n.sum_out ? static_cast<uint16_t *>(n.sum_out) + row * n.lds : nullptr;
    const int64_t step = (int64_t)blockDim.x * 8;
    auto sum8 = [&](int64_t j, float h[8]) {
        load8<BF16, VEC>(xr, j, n.cols, h);
        if (rr) {
            float r[8];
            load8<BF16, VEC>(rr, j, n.cols, r);
#pragma unroll
            for (int e = 0; e < 8; ++e) h[e] += r[e];
        }
    };
    auto weighted8 = [&](int64_t j, const float h[8], float p[8]) {
        if (wr) load8<BF16, VEC>(wr, j, n.cols, p);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] = wr ? h[e] * p[e] : h[e];
    };
    float sq = 0.0f, top = 0.0f;
    float p[NV ? NV : 1][8];
    if (NV) {
        float h[NV ? NV : 1][8];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t j = v * step + tid * 8;
            if (j < n.cols) sum8(j, h[v]);
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t j = v * step + tid * 8;
            if (j >= n.cols) break;
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(h[v][e], h[v][e], sq);
            weighted8(j, h[v], p[v]);
            if (sr) store8<BF16, VEC>(sr, j, n.cols, h[v]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(p[v][e]));
        }
    } else {
        for (int64_t j = tid * 8; j < n.cols; j += step) {
            float h[8];
            sum8(j, h);
#pragma unroll
            for (int e = 0; e < 8; ++e) sq = fmaf(h[e], h[e], sq);
            weighted8(j, h, p[0]);
#pragma unroll
            for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(p[0][e]));
        }
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        sq += __shfl_xor_sync(0xffffffffu, sq, off);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    }
    if (lane == 0) {
        sums[warp] = sq;
        tops[warp] = top;
    }
    __syncthreads();
    sq = lane < warps ? sums[lane] : 0.0f;
    top = lane < warps ? tops[lane] : 0.0f;
#pragma unroll
    for (int off = 16; off; off >>= 1) {
        sq += __shfl_xor_sync(0xffffffffu, sq, off);
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    }
    const float rstd = 1.0f / sqrtf(sq / (float)n.cols + n.eps);
    const float by = top > 0.0f ? 127.0f / top : 0.0f;
    if (n.out_scale && tid == 0) n.out_scale[row] = top * rstd / 127.0f;
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
            for (int e = 0; e < 8; ++e) v[e] *= rstd;
            store8<BF16, VEC>(static_cast<uint16_t *>(n.out) + row * n.ldo, j, n.cols, v);
        }
    };
    if (NV) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int64_t j = v * step + tid * 8;
            if (j < n.cols) result8(j, p[v]);
        }
    } else {
        for (int64_t j = tid * 8; j < n.cols; j += step) {
            float h[8];
            sum8(j, h);
            weighted8(j, h, p[0]);
            if (sr) store8<BF16, VEC>(sr, j, n.cols, h);
            result8(j, p[0]);
        }
    }
}

template <bool BF16, bool VEC>
int launch(skim_ctx *ctx, const SkimNorm &n)
{
    // a warp for every 256 columns; from 2048 columns on more pieces a thread where rows are many
    const int64_t pieces = (n.cols + 7) / 8;
    int nv = 1;
    while (nv < 4 && (pieces > (int64_t)nv * MAX_T || (n.rows > ctx->sm_count && pieces >= (int64_t)nv * 512))) nv *= 2;
    if (pieces > (int64_t)nv * MAX_T) nv = 0;
    const int64_t threads = nv ? (pieces + nv - 1) / nv : MAX_T;
    const unsigned block = (unsigned)((threads + 31) / 32 * 32);
    const dim3 grid((unsigned)n.rows);
    switch (nv) {
    case 1: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 1>, grid, block, 0, n);
    case 2: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 2>, grid, block, 0, n);
    case 4: return skim_launch_dependent(ctx, skim_add_rmsnorm_kernel<BF16, VEC, 4>, grid, block, 0, n);
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
