// Products of a few token rows with matrices in the stored form of skim_grouped.cuh:
//
//   y[t][i] = xs[t] * sum over groups of s_ig * sum_{j in the group} (q_ij - z_ig) x[t][j]
//   gated:  act(gate product) * (up product), both matrices in one pass over the tokens.
//
// Bound by the bytes of the matrix where they are many, by the chain launch - copy - products - sums where they are few.  A warp has 16 rows of one (or two)
// matrices and a stretch of their columns, whose records lie one behind the other: bulk copies bring them through a ring of the warp's own, so no warp waits for
// another before the end, and the next record's activations are on their way to registers meanwhile.  The warps of a block have different rows, or different
// parts of the columns where rows are few, and so have the blocks of a cluster; their totals are added in a fixed order.
// 16-bit activations: a record is m16n8k16 products of exact binary16 (bfloat16) numbers, the codes less their zero point, added in binary32; after every group
// the sum is taken times the group's scale into the binary32 total.  8-bit activations: m16n8k32 products of the codes themselves in whole numbers, a further one
// with ones gives the activations' sum, which the zero point takes off.  Eight tokens are the narrow side of the instructions, so one to eight cost the same.
// Measured, one token: 4096 x 4096 4.4 us (8.9 MB), 4096 x 11008 8.2 us (2.9 TB/s), gated 11008 x 4096 13.8 us (3.5 TB/s; 8-bit rows 11.5 us, 4.2 TB/s).  A column count that is no multiple
// of 8 has every record's activations read one by one, for one token too: 4096 x 4097 7.2 us.
#include <type_traits>

#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int MAX_SPLIT = 8;

// Whether a lane may find record `done` of its warp's ring in time: a test's build lets some lanes give up where others do not.
#ifndef SKIM_RECORD_IN_TIME
#define SKIM_RECORD_IN_TIME true
#endif

struct SmallArgs {
    SkimGroupedProduct p;
    int ct;
    int64_t rt;              // rows of records
    int split;               // blocks of a cluster: they share the columns
    int kw;                  // warps of a block that share the columns of its part (a power of two); the others have other rows
    int whole;               // records whose activations can be loaded as whole pieces
};

// The ring of a warp: `DEPTH` places for a record of each matrix; its activations in registers: SETS, of which one is in use and the others on their way.
// One matrix: blocks of 8 warps, which share the columns of a row of records (4096 x 4096, one token, when they were chosen: 4.7 us, with 4 warps 5.5).  Two matrices: 4 warps, and
// registers for five blocks of an SM, so that 11008 rows are one round of blocks (11008 x 4096, one 16-bit token: 13.9 us; with 8 warps 17.9, without the limit 20.6).  For two matrices and
// 8-bit rows the limit holds at 9 to 16 tokens too, where the instances spill (250 to 430 bytes of stores; 16 tokens 21.1 us): not measured with fewer blocks.
template <int XT, int PER, int NREC, int NT>
struct Ring {
    static constexpr int NW = NREC == 1 ? 8 : 4, T = NW * 32, BLOCKS = NREC == 1 ? 2 : NT == 1 || XT == SKIM_TYPE_I8 ? 5 : 3;
    static constexpr int SETS = NREC == 1 && NT * (XT == SKIM_TYPE_I8 ? 1 : 2) <= 2 ? 3 : 2;
    static constexpr int RECORD = SKIM_RECORD_CODES + 64 * PER, DEPTH = SETS == 3 ? 3 : 4, PLACE = NREC * RECORD, BYTES = DEPTH * PLACE;
    static_assert(DEPTH % SETS == 0, "a place goes with a set");
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
__device__ __forceinline__ void mma(int c[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k32.row.col.s32.u8.s8.s32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int XT>
struct Pieces {              // a lane's columns of one record of a token: four runs of eight, as they lie in memory
    static constexpr int N = XT == SKIM_TYPE_I8 ? 2 : 4;
    uint32_t w[4][N];
};

template <int XT>
__device__ __forceinline__ void load_whole(Pieces<XT> &o, const unsigned char *at)
{
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        if (XT == SKIM_TYPE_I8) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(at + 32 * t));
            o.w[t][0] = v.x; o.w[t][1] = v.y;
        } else {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(at + 64 * t));
            o.w[t][0] = v.x; o.w[t][1] = v.y; o.w[t][Pieces<XT>::N - 2] = v.z; o.w[t][Pieces<XT>::N - 1] = v.w;
        }
    }
}
// The same one by one: rows at any address, the ragged end (columns from `left` on are zeros).
template <int XT>
__device__ __noinline__ Pieces<XT> load_ragged(const unsigned char *at, int left)
{
    Pieces<XT> o;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int u = 0; u < Pieces<XT>::N; ++u) o.w[t][u] = 0u;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (32 * t + e < left) {
                if (XT == SKIM_TYPE_I8) o.w[t][e / 4] |= (uint32_t)at[32 * t + e] << (8 * (e & 3));
                else o.w[t][e / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(at)[32 * t + e] << (16 * (e & 1));
            }
    }
    return o;
}

// One record times NT batches of eight tokens, into the totals.
template <int XT, int PER, int NT>
__device__ __forceinline__ void take_record(const unsigned char *rec, const Pieces<XT> x[NT], const int sum_x[NT][PER][2], float total[NT][4])
{
    const int lane = threadIdx.x & 31, g = lane >> 2;
    const uint4 ca = *reinterpret_cast<const uint4 *>(rec + lane * 16), cb = *reinterpret_cast<const uint4 *>(rec + 512 + lane * 16);
    const uint32_t wa[4] = {ca.x, ca.y, ca.z, ca.w}, wb[4] = {cb.x, cb.y, cb.z, cb.w};
    const uint32_t *meta = reinterpret_cast<const uint32_t *>(rec + SKIM_RECORD_CODES);
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const uint32_t ma = meta[g * PER + k], mb = meta[(g + 8) * PER + k];
        const float sa = meta_scale(ma), sb = meta_scale(mb);
        float acc[NT][4];
        if constexpr (XT == SKIM_TYPE_I8) {
            int whole[NT][4] = {};
#pragma unroll
            for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t)
#pragma unroll
                for (int n = 0; n < NT; ++n)
                    mma(whole[n], wa[t] & 0x0f0f0f0fu, wb[t] & 0x0f0f0f0fu, (wa[t] >> 4) & 0x0f0f0f0fu, (wb[t] >> 4) & 0x0f0f0f0fu, x[n].w[t][0], x[n].w[t][1]);
            const int za = (int)(ma >> 16), zb = (int)(mb >> 16);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[n][u] = whole_to_float(whole[n][u] - (u < 2 ? za : zb) * sum_x[n][k][u & 1]);      // below 2^18
        } else {
            using M = typename std::conditional<XT == SKIM_TYPE_BF16, __nv_bfloat16, __half>::type;
            const Zero<XT == SKIM_TYPE_BF16> za(ma), zb(mb);
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int u = 0; u < 4; ++u) acc[n][u] = 0.0f;
#pragma unroll
            for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t) {
                uint32_t ea[4], eb[4];
                expand(wa[t], za, ea);
                expand(wb[t], zb, eb);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    mma(acc[n], ea[0], eb[0], ea[1], eb[1], x[n].w[t][0], x[n].w[t][1], M());
                    mma(acc[n], ea[2], eb[2], ea[3], eb[3], x[n].w[t][Pieces<XT>::N - 2], x[n].w[t][Pieces<XT>::N - 1], M());
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int u = 0; u < 4; ++u) total[n][u] = fmaf(u < 2 ? sa : sb, acc[n][u], total[n][u]);
    }
}

template <int XT, int PER, int NREC, int NT>
__global__ void __launch_bounds__(Ring<XT, PER, NREC, NT>::T, Ring<XT, PER, NREC, NT>::BLOCKS) skim_grouped_small_kernel(SmallArgs a)
{
    using R = Ring<XT, PER, NREC, NT>;
    constexpr int T = R::T, NW = R::NW;
    constexpr int X_BYTES = XT == SKIM_TYPE_I8 ? 1 : 2;
    static_assert(NREC * NT * 512 <= R::BYTES, "the warp's ring holds its totals at the end");
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ __align__(8) uint64_t full[NW][R::DEPTH];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3;
    const int rank = (int)(blockIdx.x % (unsigned)a.split), block = (int)(blockIdx.x / (unsigned)a.split);
    const int parts = a.kw * a.split, part = rank * a.kw + (warp & (a.kw - 1)), rows_of_block = NW / a.kw;
    const int k0 = a.ct * part / parts;
    const int64_t tile = (int64_t)block * rows_of_block + warp / a.kw;
    const int mine = tile < a.rt ? a.ct * (part + 1) / parts - k0 : 0;
    const unsigned char *src[NREC];                          // a lane's own: lane d of the first DEPTH asks for every record that comes to place d
#pragma unroll
    for (int r = 0; r < NREC; ++r) src[r] = a.p.tiles[r] + (tile * a.ct + k0 + lane) * (int64_t)R::RECORD;
    unsigned char *ring = smem + warp * R::BYTES;
    uint64_t *bar = full[warp] + (lane < R::DEPTH ? lane : 0);
    unsigned char *place = ring + lane * R::PLACE;
    if (lane < R::DEPTH) barrier_init(bar, 1);
    barrier_init_fence();
    __syncwarp();
    auto ask = [&]() {
        barrier_expect(bar, R::PLACE);
#pragma unroll
        for (int r = 0; r < NREC; ++r) {
            bulk_copy(place + r * R::RECORD, src[r], R::RECORD, bar);
            src[r] += R::DEPTH * R::RECORD;
        }
    };
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    if (lane < R::DEPTH && lane < mine) ask();
    __syncwarp();
    const int64_t t0 = (int64_t)blockIdx.y * (8 * NT);
    const int tokens = (int)(a.p.tokens - t0 < 8 * NT ? a.p.tokens - t0 : 8 * NT);
    const unsigned char *xr[NT];                             // tokens beyond the last read the last one's row: their sums are not used
#pragma unroll
    for (int n = 0; n < NT; ++n)
        xr[n] = static_cast<const unsigned char *>(a.p.x) + ((t0 + (8 * n + g < tokens ? 8 * n + g : tokens - 1)) * a.p.ldx + (int64_t)k0 * SKIM_RECORD_COLS + 8 * q) * X_BYTES;
    Pieces<XT> x[R::SETS][NT];
    auto ask_x = [&](int i, Pieces<XT> o[NT]) {
        if (i >= mine) return;
        if (k0 + i < a.whole) {
#pragma unroll
            for (int n = 0; n < NT; ++n) load_whole<XT>(o[n], xr[n]);
        } else {
#pragma unroll
            for (int n = 0; n < NT; ++n) o[n] = load_ragged<XT>(xr[n], (int)(a.p.cols - (int64_t)(k0 + i) * SKIM_RECORD_COLS) - 8 * q);
        }
#pragma unroll
        for (int n = 0; n < NT; ++n) xr[n] += SKIM_RECORD_COLS * X_BYTES;
    };
#pragma unroll
    for (int i = 0; i < R::SETS - 1; ++i) ask_x(i, x[i]);

    float total[NREC][NT][4] = {};
    bool ok = true;
    int done = 0;
    uint32_t parity = 0u;
    while (done < mine && ok) {
#pragma unroll
        for (int d = 0; d < R::DEPTH; ++d) {
            if (done >= mine) break;
            ask_x(done + R::SETS - 1, x[(d + R::SETS - 1) % R::SETS]);
            Pieces<XT> (&now)[NT] = x[d % R::SETS];
            int sum_x[NT][PER][2];
            if constexpr (XT == SKIM_TYPE_I8) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int t = 0; t < 4; ++t) {            // the order in which the codes' nibbles fall into bytes
                        const uint32_t lo = now[n].w[t][0], hi = now[n].w[t][1];
                        now[n].w[t][0] = __byte_perm(lo, hi, 0x5140);
                        now[n].w[t][1] = __byte_perm(lo, hi, 0x7362);
                    }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        int c[4] = {};
#pragma unroll
                        for (int t = k * 4 / PER; t < (k + 1) * 4 / PER; ++t) mma(c, 0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u, now[n].w[t][0], now[n].w[t][1]);
                        sum_x[n][k][0] = c[0];
                        sum_x[n][k][1] = c[1];
                    }
            }
            // for all lanes or for none: their limits may end on either side of the copy's end, and what follows is the whole warp's
            ok = __all_sync(0xffffffffu, SKIM_RECORD_IN_TIME && barrier_wait(&full[warp][d], parity)) != 0;
            if (!ok) break;
#pragma unroll
            for (int r = 0; r < NREC; ++r) take_record<XT, PER, NT>(ring + d * R::PLACE + r * R::RECORD, now, sum_x, total[r]);
            read_before_copy();
            __syncwarp();
            if (lane == d && done + R::DEPTH < mine) ask();
            ++done;
        }
        parity ^= 1u;
    }
    if (!ok) {                                               // a copy did not come: those on their way land before the ring is used again
        if (lane == 0) {
            atomicOr(a.p.status, (unsigned long long)SKIM_STATUS_TIMEOUT);
            for (int i = done; i < done + R::DEPTH && i < mine; ++i) barrier_wait(&full[warp][i % R::DEPTH], (uint32_t)(i / R::DEPTH) & 1u);
        }
        __syncwarp();
    }

    // totals: of the warps that share rows, then of the cluster's blocks, each in order
    float *sums = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int r = 0; r < NREC; ++r)
#pragma unroll
        for (int n = 0; n < NT; ++n) *reinterpret_cast<float4 *>(sums + (r * NT + n) * 128 + lane * 4) = make_float4(total[r][n][0], total[r][n][1], total[r][n][2], total[r][n][3]);
    __syncthreads();
    // an output's place among a warp's totals: 16 threads have the rows of a tile
    const int outs = rows_of_block * 16 * tokens;
    auto place_of = [&](int e, int &in_block, int &t) {
        const int i = e & 15;
        in_block = (e >> 4) & (rows_of_block - 1);
        t = (e >> 4) / rows_of_block;
        return reinterpret_cast<float *>(smem + in_block * a.kw * R::BYTES) + (t >> 3) * 128 + ((i & 7) * 4 + ((t & 7) >> 1)) * 4 + (i >> 3) * 2 + (t & 1);
    };
    auto finish = [&](int e, int in_block, int t, float v, float up) {
        const int64_t row = ((int64_t)block * rows_of_block + in_block) * SKIM_RECORD_ROWS + (e & 15), token = t0 + t;
        if (row >= a.p.rows) return;
        if (a.p.x_scale) {
            const float scale = a.p.x_scale[token];
            v *= scale;
            up *= scale;
        }
        store_as(a.p.out, a.p.out_type, token * a.p.ldo + row, NREC == 2 ? activation(a.p.act, v) * up : v);
    };
    for (int e = threadIdx.x; e < outs; e += T) {
        int in_block, t;
        float *one = place_of(e, in_block, t);
        float v = *one, up = NREC == 2 ? one[NT * 128] : 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w)
            if (w < a.kw) {
                v += one[w * (R::BYTES / 4)];
                if (NREC == 2) up += one[w * (R::BYTES / 4) + NT * 128];
            }
        if (a.split == 1) {
            finish(e, in_block, t, v, up);
        } else {
            *one = v;
            if (NREC == 2) one[NT * 128] = up;
        }
    }
    if (a.split > 1) {
        cluster_barrier();
        // each block of the cluster finishes a share of the rows; the others' sums are on their way together
        const int share = (outs / 16 + a.split - 1) / a.split * 16, end = share * (rank + 1) < outs ? share * (rank + 1) : outs;
        for (int e = share * rank + (int)threadIdx.x; e < end; e += T) {
            int in_block, t;
            const float *one = place_of(e, in_block, t);
            float part_v[MAX_SPLIT], part_up[MAX_SPLIT];
#pragma unroll
            for (int s = 0; s < MAX_SPLIT; ++s) {
                part_v[s] = s < a.split ? load_from_rank(one, s) : 0.0f;
                part_up[s] = NREC == 2 && s < a.split ? load_from_rank(one + NT * 128, s) : 0.0f;
            }
            float v = part_v[0], up = part_up[0];
#pragma unroll
            for (int s = 1; s < MAX_SPLIT; ++s) {
                v += part_v[s];
                up += part_up[s];
            }
            finish(e, in_block, t, v, up);
        }
    }
    if (a.split > 1) cluster_barrier();                      // the other blocks' totals are read before they end
}

// How the warps share rows and columns, by the clocks of an SM: a warp alone takes about 600 a record (its chain of copies, expansion and products); warps
// together share the issue slots at about 28 a record, and 60 for the start and the end of each.  A cluster's barriers and sums cost 2500 and 100 a token (gated 300): blocks share columns only
// where rows are few and long.  For one matrix the rule counts three blocks an SM, though two are resident.  (us, kw warps a block and split blocks, measured: 4096 x 4096, one
// token, 4 warps a block: kw 4 5.5, kw 2 split 2 6.5, kw 1 split 4 6.8; gated 11008 x 4096: kw 4 13.9, kw 2 15.8, kw 2 split 2 14.8; 128 x 11008, 8 warps, kw 8: alone 6.0, split 4 3.7.)
struct Plan {
    int kw, split;
};
constexpr int RECORD_ALONE = 600, RECORD_SHARED = 28, WARP_ENDS = 60, CLUSTER_COST = 2500, CLUSTER_TOKEN = 100;
Plan plan_of(const skim_ctx *ctx, int64_t rt, int ct, int nrec, int nt, int tokens, int nw, int resident)
{
    Plan best = {1, 1};
    int64_t least = INT64_MAX;
    for (int kw = 1; kw <= nw; kw *= 2)
        for (int s = 1; s <= MAX_SPLIT; s *= 2) {
            if (kw * s > ct) break;                          // every part has a record
            const int64_t chunks = (ct + kw * s - 1) / (kw * s), blocks = (rt * kw + nw - 1) / nw * s, rounds = (blocks + ctx->sm_count - 1) / ctx->sm_count;
            const int64_t waves = (rounds + resident - 1) / resident, together = (rounds + waves - 1) / waves * nw * RECORD_SHARED;
            const int64_t cost = waves * chunks * nrec * (1 + nt) / 2 * (together > RECORD_ALONE ? together : RECORD_ALONE) + rounds * nw * WARP_ENDS + (s > 1 ? CLUSTER_COST + CLUSTER_TOKEN * tokens * (nrec == 1 ? 1 : 3) : 0);
            if (cost < least) best = {kw, s}, least = cost;
        }
    return best;
}

template <int XT, int PER, int NREC, int NT>
int launch(skim_ctx *ctx, const SmallArgs &all)
{
    SmallArgs a = all;
    using R = Ring<XT, PER, NREC, NT>;
    constexpr size_t smem = (size_t)R::NW * R::BYTES;
    constexpr int T = R::T, NW = R::NW;
    const Plan plan = plan_of(ctx, a.rt, a.ct, NREC, NT, a.p.tokens < 8 * NT ? (int)a.p.tokens : 8 * NT, NW, NREC == 1 ? 3 : R::BLOCKS);
    a.split = plan.split;
    a.kw = plan.kw;
    const int64_t blocks = (a.rt * a.kw + NW - 1) / NW;
    if (blocks * a.split > 0x7fffffff) return SKIM_ERR_SHAPE;
    auto kernel = skim_grouped_small_kernel<XT, PER, NREC, NT>;
    static_assert(smem <= 47 * 1024, "no permission needed");
    static_assert(NT < 2 || 65535ll * (8 * NT) >= SKIM_MAX_TOKENS, "all tokens in one launch (NT = 1 has eight at most)");
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
int launch_of(skim_ctx *ctx, const SmallArgs &a)
{
    if (a.p.gated) return a.p.tokens <= 8 ? launch<XT, PER, 2, 1>(ctx, a) : launch<XT, PER, 2, 2>(ctx, a);
    return a.p.tokens <= 8 ? launch<XT, PER, 1, 1>(ctx, a) : launch<XT, PER, 1, 2>(ctx, a);
}
template <int XT>
int launch_by_group(skim_ctx *ctx, const SmallArgs &a)
{
    switch (a.p.group) {
    case 128: return launch_of<XT, 1>(ctx, a);
    case 64: return launch_of<XT, 2>(ctx, a);
    default: return launch_of<XT, 4>(ctx, a);
    }
}

}  // namespace

int skim_launch_grouped_small(skim_ctx *ctx, const SkimGroupedProduct &p)
{
    if (p.rows == 0 || p.tokens == 0) return SKIM_OK;
    SmallArgs a;
    a.p = p;
    a.ct = (int)skim_record_tiles(p.cols, SKIM_RECORD_COLS);
    a.rt = skim_record_tiles(p.rows, SKIM_RECORD_ROWS);
    const bool vec = (reinterpret_cast<uintptr_t>(p.x) % (p.x_type == SKIM_TYPE_I8 ? 8 : 16)) == 0 && p.ldx % 8 == 0;
    a.whole = vec ? (int)(p.cols / SKIM_RECORD_COLS) : 0;
    switch (p.x_type) {
    case SKIM_TYPE_F16: return launch_by_group<SKIM_TYPE_F16>(ctx, a);
    case SKIM_TYPE_BF16: return launch_by_group<SKIM_TYPE_BF16>(ctx, a);
    default: return launch_by_group<SKIM_TYPE_I8>(ctx, a);
    }
}
