// Products of a few token rows with matrices in the stored form of skim_grouped.cuh:
//
//   y[t][i] = xs[t] * sum over groups of s_ig * sum_{j in the group} (q_ij - z_ig) x[t][j]
//   gated:  act(gate product) * (up product), both matrices in one pass over the tokens.
//
// Bound by the bytes of the matrix: at the copy bandwidth 46 weights a clock and SM, while a warp needs about 1.6 operations a weight and lane for them.
// A block has 16 rows of one (or two) matrices; its warps take the records of that row one by one, each through a ring of its own that bulk
// copies fill ahead, so no warp waits for another before the end.  A record goes through the tensor cores as m16n8k16: the codes, less their
// zero point, are exact binary16 (bfloat16) numbers, the products are exact and are added in binary32; after every group the sum is taken
// times the group's scale into the binary32 total.  Eight tokens are the narrow side of the instruction, so one to eight cost the
// same.  Eight-bit activations become exact binary16 numbers.  The warps' totals, and those of a cluster that shares
// the columns where rows are few, are added in a fixed order.
#include <type_traits>

#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int T = 256, NW = T / 32;
constexpr int DEPTH = 4;                 // records (per matrix) that a warp has in flight
constexpr int MAX_SPLIT = 8;

struct SmallArgs {
    SkimGroupedProduct p;
    int ct, record;
    int64_t rt;              // rows of records
    int split;               // blocks of a cluster: they share the columns
    int vec;                 // whole pieces of eight columns can be loaded at once
};

__device__ __forceinline__ void mma(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __half)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma(float c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1, __nv_bfloat16)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int XT>
struct Pieces {              // a lane's columns of one record: four runs of eight, as they lie in memory
    uint32_t w[4][XT == SKIM_TYPE_I8 ? 2 : 4];
};

// Columns beyond the matrix, and tokens beyond the last, are zeros.
template <int XT>
__device__ __forceinline__ void load_pieces(Pieces<XT> &o, const void *row, bool live, int64_t first, int64_t cols, int vec)
{
    constexpr int N = XT == SKIM_TYPE_I8 ? 2 : 4;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t j = first + 32 * t;
#pragma unroll
        for (int u = 0; u < N; ++u) o.w[t][u] = 0u;
        if (!live || j >= cols) continue;
        if (vec) {
            if (N == 2) {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(static_cast<const int8_t *>(row) + j));
                o.w[t][0] = v.x; o.w[t][1] = v.y;
            } else {
                const uint4 v = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint16_t *>(row) + j));
                o.w[t][0] = v.x; o.w[t][1] = v.y; o.w[t][N == 2 ? 0 : 2] = v.z; o.w[t][N == 2 ? 0 : 3] = v.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (j + e >= cols) break;
                if (N == 2) o.w[t][e / 4] |= (uint32_t)(uint8_t)static_cast<const int8_t *>(row)[j + e] << (8 * (e & 3));
                else o.w[t][e / 2] |= (uint32_t)static_cast<const uint16_t *>(row)[j + e] << (16 * (e & 1));
            }
        }
    }
}

template <int XT, int PER, int NREC, int NT>
__global__ void __launch_bounds__(T) skim_grouped_small_kernel(SmallArgs a)
{
    constexpr bool BF16 = XT == SKIM_TYPE_BF16;
    constexpr int RECORD = SKIM_RECORD_CODES + 64 * PER, STAGE = NREC * RECORD;
    constexpr int SUMS = NREC * NT * 128;                    // totals of a block
    static_assert(NW * SUMS * 4 <= NW * DEPTH * STAGE, "the ring holds the warps' totals at the end");
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) uint64_t full[NW][DEPTH];
    __shared__ float part[SUMS];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int rank = (int)(blockIdx.x % a.split);
    const int64_t block = blockIdx.x / a.split;
    const int c0 = (int)((int64_t)a.ct * rank / a.split), c1 = (int)((int64_t)a.ct * (rank + 1) / a.split);
    const int mine = c0 + warp < c1 ? (c1 - c0 - warp + NW - 1) / NW : 0;
    const int64_t row_bytes = (int64_t)a.ct * RECORD;
    const unsigned char *src[NREC];
    int here = 0;                                            // matrices (or rows of records) of the block
#pragma unroll
    for (int r = 0; r < NREC; ++r) {
        const int64_t tile = a.p.gated ? block : block * NREC + r;
        src[r] = a.p.tiles[a.p.gated ? r : 0] + tile * row_bytes + (int64_t)(c0 + warp) * RECORD;
        if (tile < a.rt) here = r + 1;
    }
    unsigned char *my_ring = ring + warp * DEPTH * STAGE;
    if (lane == 0) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) barrier_init(&full[warp][d], 1);
        barrier_init_fence();
    }
    __syncwarp();
    auto ask = [&](int i) {
        unsigned char *dst = my_ring + (i % DEPTH) * STAGE;
        barrier_expect(&full[warp][i % DEPTH], (uint32_t)(here * RECORD));
#pragma unroll
        for (int r = 0; r < NREC; ++r)
            if (r < here) bulk_copy(dst + r * RECORD, src[r] + (int64_t)i * NW * RECORD, RECORD, &full[warp][i % DEPTH]);
    };
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    if (lane == 0)
        for (int i = 0; i < DEPTH && i < mine; ++i) ask(i);

    const int64_t t0 = (int64_t)blockIdx.y * (8 * NT);
    const void *xr[NT];
    bool live[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int64_t t = t0 + 8 * n + g;
        live[n] = t < a.p.tokens;
        xr[n] = static_cast<const unsigned char *>(a.p.x) + (live[n] ? t : 0) * a.p.ldx * (XT == SKIM_TYPE_I8 ? 1 : 2);
    }
    Pieces<XT> next[NT];
    auto ask_x = [&](int i) {
#pragma unroll
        for (int n = 0; n < NT; ++n) load_pieces<XT>(next[n], xr[n], live[n], (int64_t)(c0 + warp + i * NW) * SKIM_RECORD_COLS + 8 * q, a.p.cols, a.vec);
    };
    if (mine > 0) ask_x(0);
    float total[NREC][NT][4] = {};
    int done = 0;
    for (; done < mine; ++done) {
        Pieces<XT> now[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) now[n] = next[n];
        if (done + 1 < mine) ask_x(done + 1);
        if (!barrier_wait(&full[warp][done % DEPTH], (uint32_t)(done / DEPTH) & 1u)) break;
        const unsigned char *stage = my_ring + (done % DEPTH) * STAGE;
#pragma unroll
        for (int r = 0; r < NREC; ++r) {
            if (r >= here) break;
            const unsigned char *rec = stage + r * RECORD;
            const uint4 ca = *reinterpret_cast<const uint4 *>(rec + lane * 16), cb = *reinterpret_cast<const uint4 *>(rec + 512 + lane * 16);
            const uint32_t wa[4] = {ca.x, ca.y, ca.z, ca.w}, wb[4] = {cb.x, cb.y, cb.z, cb.w};
            const uint32_t *meta = reinterpret_cast<const uint32_t *>(rec + SKIM_RECORD_CODES);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const uint32_t ma = meta[g * PER + k], mb = meta[(g + 8) * PER + k];
                const Zero<BF16> za(ma), zb(mb);
                float acc[NT][4] = {};
#pragma unroll
                for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t) {
                    uint32_t ea[4], eb[4];
                    expand(wa[t], za, ea);
                    expand(wb[t], zb, eb);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        uint32_t x[4];
                        if (XT == SKIM_TYPE_I8) bytes_to_halves(make_uint2(now[n].w[t][0], now[n].w[t][1]), x);
                        else
#pragma unroll
                            for (int u = 0; u < 4; ++u) x[u] = now[n].w[t][XT == SKIM_TYPE_I8 ? 0 : u];
                        using M = typename std::conditional<BF16, __nv_bfloat16, __half>::type;
                        mma(acc[n], ea[0], eb[0], ea[1], eb[1], x[0], x[1], M());
                        mma(acc[n], ea[2], eb[2], ea[3], eb[3], x[2], x[3], M());
                    }
                }
                const float sa = meta_scale(ma), sb = meta_scale(mb);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    total[r][n][0] = fmaf(sa, acc[n][0], total[r][n][0]);
                    total[r][n][1] = fmaf(sa, acc[n][1], total[r][n][1]);
                    total[r][n][2] = fmaf(sb, acc[n][2], total[r][n][2]);
                    total[r][n][3] = fmaf(sb, acc[n][3], total[r][n][3]);
                }
            }
        }
        __syncwarp();
        if (lane == 0 && done + DEPTH < mine) ask(done + DEPTH);
    }
    if (done < mine) {                                       // a copy did not come: those on their way land before the block ends
        if (lane == 0) {
            atomicOr(a.p.status, (unsigned long long)SKIM_STATUS_TIMEOUT);
            for (int i = done; i < done + DEPTH && i < mine; ++i) barrier_wait(&full[warp][i % DEPTH], (uint32_t)(i / DEPTH) & 1u);
        }
    }

    // totals: of the warps, then of the cluster's blocks, each in order
    __syncthreads();
    float *all = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int r = 0; r < NREC; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) *reinterpret_cast<float4 *>(all + warp * SUMS + (r * NT + n) * 128 + lane * 4) = make_float4(total[r][n][0], total[r][n][1], total[r][n][2], total[r][n][3]);
    __syncthreads();
    for (int e = threadIdx.x; e < SUMS; e += T) {
        float v = all[e];
#pragma unroll
        for (int w = 1; w < NW; ++w) v += all[w * SUMS + e];
        part[e] = v;
    }
    if (a.split > 1) cluster_barrier();
    else __syncthreads();
    if (rank == 0) {
        constexpr int OUTS = NT * 128;
        for (int e = threadIdx.x; e < (a.p.gated ? OUTS : SUMS); e += T) {
            const int i = e & 15, t = (e >> 4) & 7, n = (e >> 7) % NT, r = e / OUTS;
            const int at = n * 128 + ((i & 7) * 4 + (t >> 1)) * 4 + (i >> 3) * 2 + (t & 1);
            const int64_t token = t0 + 8 * n + t;
            const int64_t row = (a.p.gated ? block : block * NREC + r) * SKIM_RECORD_ROWS + i;
            if (token >= a.p.tokens || row >= a.p.rows) continue;
            float v = part[r * OUTS + at], up = a.p.gated ? part[(NREC - 1) * OUTS + at] : 0.0f;
            for (int s = 1; s < a.split; ++s) {
                v += load_from_rank(part + r * OUTS + at, s);
                if (a.p.gated) up += load_from_rank(part + (NREC - 1) * OUTS + at, s);
            }
            if (a.p.x_scale) {
                const float xs = a.p.x_scale[token];
                v *= xs;
                up *= xs;
            }
            store_as(a.p.out, a.p.out_type, token * a.p.ldo + row, a.p.gated ? activation(a.p.act, v) * up : v);
        }
    }
    if (a.split > 1) cluster_barrier();                      // the other blocks' totals are read before they end
}

template <int XT, int PER, int NREC, int NT>
int launch(skim_ctx *ctx, const SmallArgs &a, int64_t blocks)
{
    constexpr size_t smem = (size_t)NW * DEPTH * NREC * (SKIM_RECORD_CODES + 64 * PER);
    auto kernel = skim_grouped_small_kernel<XT, PER, NREC, NT>;
    if (smem > 40 * 1024) SKIM_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks * a.split), (unsigned)((a.p.tokens + 8 * NT - 1) / (8 * NT)));
    cfg.blockDim = dim3(T);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)a.split;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = a.split > 1 ? 2 : 1;
    SKIM_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, a));
    ctx->launches += 1;
    return SKIM_OK;
}

template <int XT, int PER>
int launch_of(skim_ctx *ctx, const SmallArgs &a, int64_t blocks)
{
    if (a.p.gated) return a.p.tokens <= 8 ? launch<XT, PER, 2, 1>(ctx, a, blocks) : launch<XT, PER, 2, 2>(ctx, a, blocks);
    return a.p.tokens <= 8 ? launch<XT, PER, 1, 1>(ctx, a, blocks) : launch<XT, PER, 2, 2>(ctx, a, blocks);
}
template <int XT>
int launch_by_group(skim_ctx *ctx, const SmallArgs &a, int64_t blocks)
{
    switch (a.p.group) {
    case 128: return launch_of<XT, 1>(ctx, a, blocks);
    case 64: return launch_of<XT, 2>(ctx, a, blocks);
    default: return launch_of<XT, 4>(ctx, a, blocks);
    }
}

}  // namespace

int skim_launch_grouped_small(skim_ctx *ctx, const SkimGroupedProduct &p)
{
    if (p.rows == 0 || p.tokens == 0) return SKIM_OK;
    SmallArgs a;
    a.p = p;
    a.ct = (int)skim_record_tiles(p.cols, SKIM_RECORD_COLS);
    a.record = skim_record_bytes(p.group);
    a.rt = skim_record_tiles(p.rows, SKIM_RECORD_ROWS);
    const int bytes = p.x_type == SKIM_TYPE_I8 ? 1 : 2;
    a.vec = (reinterpret_cast<uintptr_t>(p.x) % (8 * bytes)) == 0 && p.ldx % 8 == 0 && p.cols % 8 == 0;
    const int nrec = p.gated || p.tokens > 8 ? 2 : 1;
    const int64_t blocks = p.gated ? a.rt : skim_record_tiles(a.rt, nrec);
    // few rows: the blocks of a cluster share the columns, as long as every warp has a record
    a.split = 1;
    while (a.split < MAX_SPLIT && blocks * a.split * 2 <= 2 * (int64_t)ctx->sm_count && a.ct >= a.split * 2 * NW) a.split *= 2;
    if (blocks * a.split > 0x7fffffff) return SKIM_ERR_SHAPE;
    switch (p.x_type) {
    case SKIM_TYPE_F16: return launch_by_group<SKIM_TYPE_F16>(ctx, a, blocks);
    case SKIM_TYPE_BF16: return launch_by_group<SKIM_TYPE_BF16>(ctx, a, blocks);
    default: return launch_by_group<SKIM_TYPE_I8>(ctx, a, blocks);
    }
}
