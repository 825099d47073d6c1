// The stored form of a matrix quantised with group scales, and what its kernels share.
//
// Records of 16 rows x 128 columns lie one row of records after another.  A record holds 1024 bytes of codes -- 16 words for each of its
// rows, word 4 p + t with columns 32 t + 8 p .. 32 t + 8 p + 7 of the record -- and behind them a word for every row and group, the scale's
// bits with the zero point above them.  So a lane's 16 bytes are four runs of eight columns that lie in the four quarters of the record: the
// quad of lanes that shares a row in a tensor instruction has one group, whatever its size, in front of it at a time; and all that a warp needs
// of 16 rows is one contiguous piece, which a bulk copy brings.
#pragma once

#include <cuda_bf16.h>

#include "skim_internal.cuh"

#define SKIM_RECORD_ROWS 16
#define SKIM_RECORD_COLS 128
#define SKIM_RECORD_CODES 1024

__host__ __device__ static inline int64_t skim_record_tiles(int64_t n, int64_t of) { return (n + of - 1) / of; }
__host__ __device__ static inline int skim_record_bytes(int group) { return SKIM_RECORD_CODES + SKIM_RECORD_ROWS * (SKIM_RECORD_COLS / group) * 4; }

namespace skimg {

// Column e of a word's eight lies in nibble 4 (e & 1) + e / 2: nibbles i and i + 4, which one mask takes out together, are neighbours.
__host__ __device__ __forceinline__ int nibble_of(int e) { return 4 * (e & 1) + e / 2; }

__device__ __forceinline__ uint32_t half2_bits(__half2 v) { return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ __half2 bits_half2(uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); }
__device__ __forceinline__ uint32_t bf162_bits(__nv_bfloat162 v) { return *reinterpret_cast<const uint32_t *>(&v); }
__device__ __forceinline__ __nv_bfloat162 bits_bf162(uint32_t v) { return *reinterpret_cast<const __nv_bfloat162 *>(&v); }

// A group's zero point, ready to be taken off the codes of a word.
template <bool BF16>
struct Zero;
template <>
struct Zero<false> {
    __half2 near, far;           // 1024 + z, -(64 + z)
    __device__ __forceinline__ explicit Zero(uint32_t meta)
    {
        near = bits_half2(__byte_perm(meta, 0x64u, 0x4242));
        far = __hsub2(bits_half2(0x63806380u), near);                    // 960 - (1024 + z)
    }
};
template <>
struct Zero<true> {
    __nv_bfloat162 near;         // 128 + z
    __device__ __forceinline__ explicit Zero(uint32_t meta) { near = bits_bf162(__byte_perm(meta, 0x43u, 0x4242)); }
};
__device__ __forceinline__ float meta_scale(uint32_t meta) { return __half2float(__ushort_as_half((unsigned short)(meta & 0xffffu))); }

// (a & mask) | with, one operation
__device__ __forceinline__ uint32_t and_or(uint32_t a, uint32_t mask, uint32_t with)
{
    uint32_t r;
    asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(r) : "r"(a), "r"(mask), "r"(with));
    return r;
}

// code - z of a word's eight columns, as pairs of neighbours.  A nibble ORed into the low bits of 1024 (the bfloat16 128) is that number plus the code,
// exactly; the second nibble of a byte comes out sixteenfold and is scaled back in the subtraction.  All results are whole and exact.
__device__ __forceinline__ void expand(uint32_t w, const Zero<false> &z, uint32_t out[4])
{
    const __half2 sixteenth = bits_half2(0x2c002c00u);
    out[0] = half2_bits(__hsub2(bits_half2(and_or(w, 0x000f000fu, 0x64006400u)), z.near));
    out[1] = half2_bits(__hfma2(bits_half2(and_or(w, 0x00f000f0u, 0x64006400u)), sixteenth, z.far));
    w >>= 8;
    out[2] = half2_bits(__hsub2(bits_half2(and_or(w, 0x000f000fu, 0x64006400u)), z.near));
    out[3] = half2_bits(__hfma2(bits_half2(and_or(w, 0x00f000f0u, 0x64006400u)), sixteenth, z.far));
}
__device__ __forceinline__ void expand(uint32_t w, const Zero<true> &z, uint32_t out[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) out[i] = bf162_bits(__hsub2(bits_bf162(and_or(w >> (4 * i), 0x000f000fu, 0x43004300u)), z.near));
}

// The same as signed bytes, four columns a word.
__device__ __forceinline__ void expand_bytes(uint32_t w, uint32_t meta, uint32_t out[2])
{
    const uint32_t z = __byte_perm(meta, 0u, 0x2222);
    const uint32_t a = (and_or(w, 0x0f0f0f0fu, 0x80808080u) - z) ^ 0x80808080u, b = (and_or(w >> 4, 0x0f0f0f0fu, 0x80808080u) - z) ^ 0x80808080u;      // columns 0 4 1 5, 2 6 3 7
    out[0] = __byte_perm(a, b, 0x6420);
    out[1] = __byte_perm(a, b, 0x7531);
}
// A whole number below 2^22 in magnitude, by way of 1.5 * 2^23: exact, and without the conversion unit.
__device__ __forceinline__ float whole_to_float(int v) { return __int_as_float(v + 0x4b400000) - 12582912.0f; }

enum { ACT_SILU = SKIM_ACT_SILU, ACT_GELU = SKIM_ACT_GELU };
// 0.5 (1 + tanh(u)) = 1 / (1 + exp(-2u)): either activation is g / (1 + exp(-v)).
__device__ __forceinline__ float activation(int act, float g)
{
    const float v = act == ACT_SILU ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
    return __fdividef(g, 1.0f + expf(-v));
}
__device__ __forceinline__ void store_as(void *out, int type, int64_t at, float v)
{
    if (type == SKIM_TYPE_F32) reinterpret_cast<float *>(out)[at] = v;
    else if (type == SKIM_TYPE_F16) reinterpret_cast<__half *>(out)[at] = __float2half_rn(v);
    else reinterpret_cast<__nv_bfloat16 *>(out)[at] = __float2bfloat16_rn(v);
}

// Barriers in shared memory and bulk copies into it.
__device__ __forceinline__ uint32_t smem_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void barrier_init(uint64_t *bar, uint32_t count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_address(bar)), "r"(count)); }
__device__ __forceinline__ void barrier_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void barrier_expect(uint64_t *bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_address(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t *bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_address(bar)) : "memory"); }
__device__ __forceinline__ bool barrier_try(uint64_t *bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(smem_address(bar)), "r"(parity)
                 : "memory");
    return ok != 0;
}
constexpr long long WAIT_CYCLES = 400000000ll;       // about 0.2 s; a launch takes milliseconds at most
__device__ __forceinline__ bool barrier_wait(uint64_t *bar, uint32_t parity, long long limit = WAIT_CYCLES)
{
    if (barrier_try(bar, parity)) return true;
    const long long t0 = clock64();
    while (!barrier_try(bar, parity))
        if (clock64() - t0 > limit) return false;
    return true;
}
// Source, destination and size are multiples of 16 bytes.
__device__ __forceinline__ void bulk_copy(void *dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(smem_address(dst)), "l"(src), "r"(bytes),
                 "r"(smem_address(bar))
                 : "memory");
}
// Between a thread's last read of a place in shared memory and what lets a bulk copy overwrite it.
__device__ __forceinline__ void read_before_copy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void cluster_barrier()
{
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_rank_of_block()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float load_from_rank(const float *p, uint32_t rank)
{
    uint32_t at;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_address(p)), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

}  // namespace skimg

// One product of token rows with one or two stored matrices.
struct SkimGroupedProduct {
    const unsigned char *tiles[2];   // the matrix; gated: gate and up
    int gated, act;
    int64_t rows, cols;
    int group;
    const void *x;
    int x_type;
    int64_t ldx;
    const float *x_scale;            // [tokens] or nullptr (1)
    int64_t tokens;
    void *out;
    int out_type;
    int64_t ldo;
    unsigned long long *status;
};
bool skim_grouped_gemm_takes(const skim_ctx *ctx, const SkimGroupedProduct &p);
int skim_launch_grouped_gemm(skim_ctx *ctx, const SkimGroupedProduct &p);
int64_t skim_aligned_stride(int64_t cols, int x_type);
int skim_launch_align_rows(skim_ctx *ctx, const SkimGroupedProduct &p, void *scratch);
int skim_launch_grouped_small(skim_ctx *ctx, const SkimGroupedProduct &p);
int skim_launch_grouped_quantize(skim_ctx *ctx, const uint16_t *W, const float *importance, const float *rscale, int64_t rows, int64_t cols, int64_t ld, int group,
                                 unsigned char *tiles, float *err);
int skim_launch_grouped_dequantize(skim_ctx *ctx, const unsigned char *tiles, int64_t rows, int64_t cols, int group, uint16_t *out, int64_t ld_out);
struct SkimNorm {
    const void *x, *residual, *weight;
    int type;
    int64_t rows, cols, ldx, ldr, lds, ldo;
    float eps;
    void *sum_out, *out;
    int out_type;
    float *out_scale;
};
int skim_launch_add_rmsnorm(skim_ctx *ctx, const SkimNorm &n);
