// Products of many token rows with matrices in the stored form of skim_grouped.cuh, on the fifth-generation tensor cores:
//
//   y[t][i] = sum over groups of s_ig * sum_{j in the group} (q_ij - z_ig) x[t][j],   gated: act(gate product) * (up product)
//
// Bound by the tensor pipe and by the round of signals about it.  A pair of CTAs has a tile of 256 weight rows, 128 each (gated: 64 of the gate and the same 64 of
// the up matrix), times up to 192 tokens.  The weights are operand A, and never touch shared memory as numbers: four warps expand a record's codes, less
// their zero points, in registers and store them to tensor memory (exact binary16 or bfloat16 numbers), from where tcgen05.mma reads them.  The tokens are operand
// B, brought by TMA, half of them by each CTA: a tile of its own for every CTA would ask the L2 for twice the bytes.  The values are not rounded to 16 bits: an
// accumulator holds one group's sum, in binary32, and eight warps take it times the group's scale into binary32 totals in their registers,
// while the tensor cores are at the next one.
// Where tiles are few the pairs of a cluster share the columns and add their totals, in a fixed order, through shared memory.
// Measured: 1024 bf16 tokens 11008 x 4096 85 us (1.08 PFLOP/s, 65 % of the measured peak), gated 300 tokens 22016 x 8192 207 us (1.05 PFLOP/s).  A step of 768 clocks of products takes
// 1230: the warp that issues them waits about 480 for an accumulator, of which there are two, and one goes 1480 clocks from the issue to the warps that read it and 400 more until it
// is free.  The last round of tiles is not full either (258 tiles on 74 pairs), nor the last tile of the tokens.  Groups of 64: 125 us, of 32: 215 us, a round for each of them.  8-bit rows: 109, 173
// and 301 us, gated 258: their products take half the clocks, but the round is the same and whole sums are converted on top, so the narrower rows are the slower ones here.
#include <cuda.h>
#include <cudaTypedefs.h>

#include "skim_grouped.cuh"

namespace {

using namespace skimg;

constexpr int CM = 128, BM = 2 * CM;             // weight rows of a CTA, of a pair
constexpr int BK = SKIM_RECORD_COLS;             // columns of a step: one record
constexpr int RECS = CM / SKIM_RECORD_ROWS;      // records of a CTA's rows in a step
constexpr int EXPAND_WARPS = 4;                  // for a step; two such groups take the steps in turn
constexpr int FIRST_SUM = 2 * EXPAND_WARPS, SUM_WARPS = 8, THREADS = (FIRST_SUM + SUM_WARPS + 4) * 32;
constexpr int WARP_TMA = FIRST_SUM + SUM_WARPS, WARP_MMA = WARP_TMA + 1, WARP_CODES = WARP_TMA + 2;
constexpr int MAX_SPLIT = 4;

// What tensor memory and shared memory hold.  A group's sum goes a round of product, signal, readback and signal; issuing a group's products and signals
// takes one warp some 700 clocks however long they are.  So with groups of 128 the accumulators are wide (192 tokens: 768 clocks of products) and two; with
// smaller groups, where the round counts, narrower and three.
template <int XT, int PER, bool GATED>
struct Shape {
    static constexpr bool I8 = XT == SKIM_TYPE_I8;
    static constexpr int K = I8 ? 32 : 16;                               // columns of an instruction
    static constexpr int N = PER == 1 ? 192 : 128, D_PLACES = PER == 1 ? 2 : 3;      // tokens of an accumulator, at most; accumulators
    static constexpr int A_PLACES = 2, A_COLS = I8 ? BK / 4 : BK / 2, A_COL = D_PLACES * N, TMEM_COLS = 512;
    static_assert(A_COL + A_PLACES * A_COLS <= TMEM_COLS, "tensor memory");
    static constexpr int BOX = N / 2 * 128, BOXES = I8 ? 1 : 2;          // this CTA's tokens, 128 bytes (64 or 128 columns) of each; boxes of a step
    static constexpr int B_PLACES = PER == 1 && GATED ? 4 : 5, B_BYTES = BOXES * BOX;
    static constexpr int RECORD = SKIM_RECORD_CODES + 64 * PER, C_PLACES = 6, C_BYTES = RECS * RECORD;
    static constexpr int CODES_AT = B_PLACES * B_BYTES, SWAP_AT = CODES_AT + C_PLACES * C_BYTES, SYNC_AT = SWAP_AT + (GATED ? CM * N / 2 * 4 : 0), SYNC_BYTES = 512;
    static constexpr size_t SMEM = 1024 + SYNC_AT + SYNC_BYTES;
    static_assert(SMEM <= 227 * 1024 && N * CM * 4 <= SYNC_AT, "shared memory; the totals of a split tile fit");
};

struct GemmArgs {
    SkimGroupedProduct p;
    int ct;
    int64_t rt;              // rows of records
    int mt, nt;              // tiles along weight rows, along tokens
    int n;                   // tokens of a tile (a multiple of 32, which products with operand A in tensor memory ask for)
    int split;               // pairs of a cluster: they share the columns
};

struct Sync {
    uint64_t b_full[5], b_empty[5];      // a step's tokens; b_empty: its products are done, which frees its operand A too
    uint64_t a_full[2];
    uint64_t c_full[6], c_empty[6];      // records
    uint64_t d_full[3], d_empty[3];      // accumulators
    uint32_t tmem;
    int abort;               // a wait ran out
};
static_assert(sizeof(Sync) <= 512, "the barriers' part of the shared memory");

__device__ __forceinline__ uint32_t address_in(const void *p, uint32_t rank)
{
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_address(p)), "r"(rank));
    return r;
}
// What is handed over lies in tensor memory and is ordered by tcgen05's fences: no release beyond the block, whose fence would cost hundreds of clocks a time.
__device__ __forceinline__ void arrive_at(uint32_t addr) { asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory"); }
// (Inline like all that these roles run: a function of its own might use registers that a warp has given up.)
// The end of a phase, or (false) the limit of the wait, or another role's.
__device__ __forceinline__ bool wait_longer(uint64_t *bar, uint32_t parity, Sync &sy)
{
    const long long t0 = clock64();
    while (!barrier_try(bar, parity)) {
        if (*(volatile int *)&sy.abort) return false;
        if (clock64() - t0 > WAIT_CYCLES) {
            *(volatile int *)&sy.abort = 1;
            return false;
        }
    }
    return true;
}
__device__ __forceinline__ bool wait_for(uint64_t *bar, uint32_t parity, Sync &sy) { return barrier_try(bar, parity) || wait_longer(bar, parity, sy); }
// By a whole warp, whose lanes go on together.  The roles whose loops count every clock go on after a wait that ran out, through what is left of their loops, in which no
// wait lasts any more; those that ask for copies stop.
__device__ __forceinline__ void warp_wait(uint64_t *bar, uint32_t parity, Sync &sy)
{
    wait_for(bar, parity, sy);
    __syncwarp();
}
__device__ __forceinline__ bool warp_wait_or_stop(uint64_t *bar, uint32_t parity, Sync &sy) { return __all_sync(0xffffffffu, wait_for(bar, parity, sy)) != 0; }
// 64 columns of some token rows into this CTA's shared memory; the bytes are counted at `bar`, in the pair's first CTA.
__device__ __forceinline__ void tma_tokens(void *dst, const CUtensorMap *map, uint32_t bar, int col, int token)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_address(dst)),
                 "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(col), "r"(token)
                 : "memory");
}
// Operand B in shared memory: rows of 64 16-bit numbers = 128 bytes, 128-byte swizzle, groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t operand_b(uint32_t addr)
{
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// A and B K-major, 256 rows, n columns.  kind::f16: binary32 accumulators, A and B both binary16 or both bfloat16; kind::i8: whole 32-bit accumulators, A and B signed bytes.
__device__ __forceinline__ uint32_t instruction_of(int xt, int n) { return (xt == SKIM_TYPE_I8 ? 2u << 4 : 1u << 4) | (xt == SKIM_TYPE_F16 ? 0u : (1u << 7) | (1u << 10)) | (uint32_t)(n >> 3) << 17 | (uint32_t)(BM >> 4) << 24; }
template <bool I8>
__device__ __forceinline__ void multiply(uint32_t d, uint32_t a, uint64_t b, uint32_t instruction, uint32_t accumulate)
{
    if constexpr (I8)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::i8 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(instruction),
                     "r"(accumulate)
                     : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a), "l"(b), "r"(instruction),
                     "r"(accumulate)
                     : "memory");
}
// Arrives at this offset in both CTAs of the pair once the products issued so far are done.
__device__ __forceinline__ void commit_to(uint64_t *bar, uint16_t both)
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_address(bar)), "h"(both) : "memory");
}
__device__ __forceinline__ bool elect_lane()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void wait_stores() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// 32 consecutive 32-bit columns of this thread's lane of tensor memory; wait_loads() before the values are used, which it names, so that no use moves in front of it.
__device__ __forceinline__ void tmem_load32(uint32_t at, uint32_t *v)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
                 : "r"(at));
}
__device__ __forceinline__ void tmem_store32(uint32_t at, const uint32_t *v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]), "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31])
                 : "memory");
}
__device__ __forceinline__ void wait_loads(uint32_t *v)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31])::"memory");
}
template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// A block is launched with 96 registers a thread; of the five warpgroups two take 72, two 152, one 32.
__device__ __forceinline__ void sums_barrier() { asm volatile("bar.sync 1, %0;" ::"n"(SUM_WARPS * 32) : "memory"); }
__device__ __forceinline__ void store_one(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_one(__half *p, float v) { *p = __float2half_rn(v); }
__device__ __forceinline__ void store_one(__nv_bfloat16 *p, float v) { *p = __float2bfloat16_rn(v); }
// The first n tokens of a row: few instructions for each, since they are many.
template <int N, typename Out>
__device__ __forceinline__ void store_totals(Out *p, int64_t stride, int n, const float *total)
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        if (i < n) store_one(p, total[i]);
        p += stride;
    }
}

// Row of the matrix, and the matrix, that row r of this CTA's tile m is.
template <bool GATED>
__device__ __forceinline__ int64_t row_of(int m, uint32_t mine, int r) { return GATED ? (int64_t)m * CM + mine * (CM / 2) + (r & (CM / 2 - 1)) : (int64_t)m * BM + mine * CM + r; }
template <bool GATED>
__device__ __forceinline__ int matrix_of(int r) { return GATED && r >= CM / 2 ? 1 : 0; }

template <int XT, int PER, bool GATED>
__global__ void __launch_bounds__(THREADS, 1) skim_grouped_gemm_kernel(const __grid_constant__ CUtensorMap tokens_map, GemmArgs a)
{
    using S = Shape<XT, PER, GATED>;
    constexpr int STEPS = BK / S::K / PER;                     // instructions of a group
    extern __shared__ unsigned char raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023), *code_ring = ring + S::CODES_AT;
    Sync &sy = *reinterpret_cast<Sync *>(ring + S::SYNC_AT);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank_of_block(), leader = rank & ~1u, mine = rank & 1u;
    const int part = (int)(rank >> 1), clusters = (int)gridDim.x / (2 * a.split), first = (int)blockIdx.x / (2 * a.split);
    const int k0 = a.ct * part / a.split, k1 = a.ct * (part + 1) / a.split, tiles = a.mt * a.nt;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::B_PLACES; ++s) { barrier_init(&sy.b_full[s], 1); barrier_init(&sy.b_empty[s], 1); }
        for (int s = 0; s < S::A_PLACES; ++s) barrier_init(&sy.a_full[s], 2 * EXPAND_WARPS);
        for (int s = 0; s < S::C_PLACES; ++s) { barrier_init(&sy.c_full[s], 1); barrier_init(&sy.c_empty[s], EXPAND_WARPS); }
        for (int s = 0; s < S::D_PLACES; ++s) { barrier_init(&sy.d_full[s], 1); barrier_init(&sy.d_empty[s], 2 * SUM_WARPS); }
        sy.abort = 0;
        barrier_init_fence();
    }
    if (warp == WARP_MMA) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&sy.tmem)), "r"(S::TMEM_COLS));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    }
    fence_before();
    __syncthreads();
    cluster_barrier();
    fence_after();
    skim_wait_for_previous_kernel();
    skim_let_next_kernel_start();
    const uint32_t tmem = 0u;                                // all columns are this block's, so they begin at 0: a constant keeps the operands warp-uniform
    if (sy.tmem != 0u) *(volatile int *)&sy.abort = 1;

    if (warp < FIRST_SUM) {
        // ---------------------------------------------------------------- codes to operand A; a thread has a row, its warps every other step and place
        fewer_registers<72>();
        static_assert(S::A_PLACES == 2 && S::C_PLACES % 2 == 0, "a place is always the same warps'");
        const int turn = warp / EXPAND_WARPS, in = (warp & 3) * 32 + lane;
        const uint32_t to = tmem + ((uint32_t)((warp & 3) * 32) << 16) + S::A_COL + turn * S::A_COLS;
        const uint32_t full_at = address_in(&sy.a_full[turn], leader);
        const int steps = (first < tiles ? (tiles - first + clusters - 1) / clusters : 0) * (k1 - k0);
        int from = turn, freed = turn;                       // places of the records' ring and, of the step two before, the tokens'
        uint32_t phase_c = 0, phase_b = 0;
        for (int step = turn; step < steps; step += 2) {
            warp_wait(&sy.c_full[from], phase_c, sy);
            const unsigned char *r = code_ring + from * S::C_BYTES + in / SKIM_RECORD_ROWS * S::RECORD;
            uint4 codes[4];
            uint32_t meta[PER];
#pragma unroll
            for (int p = 0; p < 4; ++p) codes[p] = *reinterpret_cast<const uint4 *>(r + (in % SKIM_RECORD_ROWS) * 64 + p * 16);
#pragma unroll
            for (int k = 0; k < PER; ++k) meta[k] = reinterpret_cast<const uint32_t *>(r + SKIM_RECORD_CODES)[in % SKIM_RECORD_ROWS * PER + k];
#pragma unroll
            for (int h = 0; h < S::A_COLS / 32; ++h) {
                constexpr int RUNS = S::I8 ? 4 : 2;          // of 32 columns, in 32 words
                uint32_t out[32];
#pragma unroll
                for (int t2 = 0; t2 < RUNS; ++t2) {
                    const int tt = RUNS * h + t2;
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        const uint32_t w = tt == 0 ? codes[p].x : tt == 1 ? codes[p].y : tt == 2 ? codes[p].z : codes[p].w;
                        if constexpr (S::I8) expand_bytes(w, meta[tt * PER / 4], out + 8 * t2 + 2 * p);
                        else expand(w, Zero<XT == SKIM_TYPE_BF16>(meta[tt * PER / 4]), out + 16 * t2 + 4 * p);
                    }
                }
                if (h == 0 && step >= 2) {                   // the place is free when the step that had it is done
                    warp_wait(&sy.b_empty[freed], phase_b, sy);
                    if ((freed += 2) >= S::B_PLACES) { freed -= S::B_PLACES; phase_b ^= 1u; }
                    fence_after();
                }
                tmem_store32(to + 32 * h, out);
            }
            wait_stores();
            fence_before();
            read_before_copy();                              // (given back before the values' last use, a place was overwritten before it was read)
            __syncwarp();
            if (lane == 0) {
                arrive_at(full_at);
                barrier_arrive(&sy.c_empty[from]);
            }
            if ((from += 2) >= S::C_PLACES) { from -= S::C_PLACES; phase_c ^= 1u; }
        }
    } else if (warp < FIRST_SUM + SUM_WARPS) {
        // ---------------------------------------------------------------- groups' sums times their scales; a thread has a row and half of the tokens
        more_registers<152>();
        constexpr int H = S::N / 2;
        const int quarter = warp & 3, half = (warp - FIRST_SUM) >> 2, r = quarter * 32 + lane, h = a.n / 2;
        int place = 0;
        uint32_t phase = 0;
        const uint32_t from = tmem + ((uint32_t)(quarter * 32) << 16) + half * h;
        const unsigned char *matrix = a.p.tiles[matrix_of<GATED>(r)];
        const uint32_t empty_at = address_in(&sy.d_empty[0], leader);
        for (int t = first; t < tiles; t += clusters) {
            const int64_t row = row_of<GATED>(t / a.nt, mine, r), rec = row / SKIM_RECORD_ROWS;
            const bool live = rec < a.rt;
            const unsigned char *at = matrix + (live ? (rec * a.ct + k0) * S::RECORD + SKIM_RECORD_CODES + (row % SKIM_RECORD_ROWS) * (4 * PER) : 0);
            uint32_t meta[PER];
            float total[H];
#pragma unroll
            for (int i = 0; i < H; ++i) total[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < PER; ++k) meta[k] = __ldg(reinterpret_cast<const uint32_t *>(at) + k);
            for (int c = k0; c < k1; ++c) {
                float scale[PER];
#pragma unroll
                for (int k = 0; k < PER; ++k) scale[k] = meta_scale(meta[k]);
                if (c + 1 < k1) {
                    if (live) at += S::RECORD;
#pragma unroll
                    for (int k = 0; k < PER; ++k) meta[k] = __ldg(reinterpret_cast<const uint32_t *>(at) + k);
                }
#pragma unroll
                for (int k = 0; k < PER; ++k) {
                    warp_wait(&sy.d_full[place], phase, sy);
                    fence_after();
                    const float s = scale[k];
#pragma unroll
                    for (int i = 0; i < H; i += 32) {
                        if (i >= h) break;                   // (h is a multiple of 16: the last read may take 16 columns of the other half along, unused)
                        uint32_t v[32];
                        tmem_load32(from + place * S::N + i, v);
                        wait_loads(v);
                        if (i + 32 >= H || i + 32 >= h) {
                            fence_before();
                            __syncwarp();
                            if (lane == 0) arrive_at(empty_at + place * 8);
                        }
#pragma unroll
                        for (int u = 0; u < 32; ++u) total[i + u] = fmaf(s, S::I8 ? whole_to_float((int)v[u]) : __uint_as_float(v[u]), total[i + u]);
                    }
                    if (++place == S::D_PLACES) { place = 0; phase ^= 1u; }
                }
            }
            const int64_t t0 = (int64_t)(t % a.nt) * a.n + half * h;
            const int left = (int)(a.p.tokens - t0 < h ? a.p.tokens - t0 : h);             // this thread's tokens (none: below 1)
            if (a.p.x_scale) {
#pragma unroll
                for (int i = 0; i < H; ++i)
                    if (i < left) total[i] *= __ldg(a.p.x_scale + t0 + i);
            }
            if (a.split > 1) {
                // the pairs of the cluster have one tile; the rings are no longer used: totals go there, [token][row]
                float *all = reinterpret_cast<float *>(ring) + half * h * CM + r;
#pragma unroll
                for (int i = 0; i < H; ++i)
                    if (i < h) all[i * CM] = total[i];
            } else if (GATED) {
                // Gate and up meet in shared memory, in two turns; the gate's threads finish one half of a turn's tokens, the up's the other.  (A loop: unrolled, with
                // its registers, this code did not fit the instruction cache and took 27 000 clocks a tile.)
                constexpr int TURN = H / 2;
                float *swap = reinterpret_cast<float *>(ring + S::SWAP_AT) + half * TURN * CM;
                const int up = matrix_of<GATED>(r), g = r & (CM / 2 - 1);
#pragma unroll
                for (int turn = 0; turn < 2; ++turn) {
#pragma unroll
                    for (int i = 0; i < TURN; ++i) swap[i * CM + r] = total[turn * TURN + i];
                    sums_barrier();
                    if (row < a.p.rows)
#pragma unroll 4
                        for (int i = up * (TURN / 2); i < (up + 1) * (TURN / 2) && turn * TURN + i < left; ++i)
                            store_as(a.p.out, a.p.out_type, (t0 + turn * TURN + i) * a.p.ldo + row, activation(a.p.act, swap[i * CM + g]) * swap[i * CM + CM / 2 + g]);
                    sums_barrier();
                }
            } else if (row < a.p.rows) {
                if (a.p.out_type == SKIM_TYPE_F32) store_totals<H>(static_cast<float *>(a.p.out) + t0 * a.p.ldo + row, a.p.ldo, left, total);
                else if (a.p.out_type == SKIM_TYPE_F16) store_totals<H>(static_cast<__half *>(a.p.out) + t0 * a.p.ldo + row, a.p.ldo, left, total);
                else store_totals<H>(static_cast<__nv_bfloat16 *>(a.p.out) + t0 * a.p.ldo + row, a.p.ldo, left, total);
            }
        }
    } else {
        fewer_registers<32>();
        bool ok = true;
        if (warp == WARP_TMA && lane == 0) {
            // ------------------------------------------------------------ tokens
            const uint32_t bytes = S::BOXES * (a.n / 2) * 128;
            int place = 0, issued = 0;
            uint32_t phase = 0;
            for (int t = first; t < tiles && ok; t += clusters) {
                const int t0 = (t % a.nt) * a.n + (int)mine * (a.n / 2);
                for (int c = k0; c < k1; ++c) {
                    if (!(ok = wait_for(&sy.b_empty[place], phase ^ 1u, sy))) break;
                    unsigned char *to = ring + (size_t)place * S::B_BYTES;
                    if (mine == 0) barrier_expect(&sy.b_full[place], 2 * bytes);
                    const uint32_t bar = address_in(&sy.b_full[place], leader);
                    for (int h = 0; h < S::BOXES; ++h) tma_tokens(to + h * S::BOX, &tokens_map, bar, c * BK + h * 64, t0);
                    ++issued;
                    if (++place == S::B_PLACES) { place = 0; phase ^= 1u; }
                }
            }
            if (!ok && mine == 0)                              // copies on their way land before the block ends
                for (int i = issued > S::B_PLACES ? issued - S::B_PLACES : 0; i < issued; ++i) barrier_wait(&sy.b_full[i % S::B_PLACES], (uint32_t)(i / S::B_PLACES) & 1u, WAIT_CYCLES / 16);
        } else if (warp == WARP_CODES) {
            // ------------------------------------------------------------ records: a lane has one of eight
            int place = 0, issued = 0;
            uint32_t phase = 0;
            const int r = (lane & (RECS - 1)) * SKIM_RECORD_ROWS;
            for (int t = first; t < tiles && ok; t += clusters) {
                const int64_t rec = row_of<GATED>(t / a.nt, mine, r) / SKIM_RECORD_ROWS;
                const bool live = lane < RECS && rec < a.rt;
                const uint32_t bytes = __popc(__ballot_sync(0xffffffffu, live)) * S::RECORD;
                const unsigned char *src = a.p.tiles[matrix_of<GATED>(r)] + (rec * a.ct + k0) * S::RECORD;
                for (int c = k0; c < k1; ++c, src += S::RECORD) {
                    if (!(ok = warp_wait_or_stop(&sy.c_empty[place], phase ^ 1u, sy))) break;
                    if (lane == 0) barrier_expect(&sy.c_full[place], bytes);
                    __syncwarp();
                    if (live) bulk_copy(code_ring + place * S::C_BYTES + lane * S::RECORD, src, S::RECORD, &sy.c_full[place]);
                    ++issued;
                    if (++place == S::C_PLACES) { place = 0; phase ^= 1u; }
                }
            }
            if (!ok)
                for (int i = issued > S::C_PLACES ? issued - S::C_PLACES : 0; i < issued; ++i) barrier_wait(&sy.c_full[i % S::C_PLACES], (uint32_t)(i / S::C_PLACES) & 1u, WAIT_CYCLES / 16);
        } else if (warp == WARP_MMA && mine == 0) {
            // ------------------------------------------------------------ products, for both CTAs.  The whole warp goes through the loops, so that operands are
            // warp-uniform values, and one lane issues
            const uint32_t instruction = instruction_of(XT, a.n);
            const uint16_t both = (uint16_t)(3u << leader);
            int pa = 0, pb = 0, pd = 0;
            uint32_t phase_a = 0, phase_b = 0, phase_d = 1;
            for (int t = first; t < tiles; t += clusters)
                for (int c = k0; c < k1; ++c) {
                    warp_wait(&sy.b_full[pb], phase_b, sy);
                    warp_wait(&sy.a_full[pa], phase_a, sy);
                    const uint64_t b = operand_b(smem_address(ring + (size_t)pb * S::B_BYTES));
                    const uint32_t a_at = tmem + S::A_COL + pa * S::A_COLS;
#pragma unroll
                    for (int k = 0; k < PER; ++k) {
                        warp_wait(&sy.d_empty[pd], phase_d, sy);
                        fence_after();
                        if (elect_lane()) {
#pragma unroll
                            for (int u = 0; u < STEPS; ++u) {
                                const int step = k * STEPS + u;
                                multiply<S::I8>(tmem + pd * S::N, a_at + step * 8, b + (((step >> 2) * S::BOX + (step & 3) * 32) >> 4), instruction, u > 0);
                            }
                            commit_to(&sy.d_full[pd], both);
                            if (k == PER - 1) commit_to(&sy.b_empty[pb], both);
                        }
                        __syncwarp();
                        if (++pd == S::D_PLACES) { pd = 0; phase_d ^= 1u; }
                    }
                    if (++pa == S::A_PLACES) { pa = 0; phase_a ^= 1u; }
                    if (++pb == S::B_PLACES) { pb = 0; phase_b ^= 1u; }
                }
        }
    }
    // what follows is every warp's, and compiled for the registers of the launch (a warpgroup's warps meet before they change their registers again)
    __syncthreads();
    if (warp >= FIRST_SUM && warp < FIRST_SUM + SUM_WARPS) fewer_registers<96>();
    else more_registers<96>();
    __syncthreads();
    if (sy.abort) {
        for (int i = 0; i < 1000; ++i) __nanosleep(1000);      // copies and products in flight end before the block does
        if (threadIdx.x == 0) atomicOr(a.p.status, (unsigned long long)SKIM_STATUS_TIMEOUT);
    }
    fence_before();
    cluster_barrier();
    if (a.split > 1) {
        // every pair's totals lie in shared memory; they are added in order of rank.  A pair finishes the tokens i with i % split == its number
        constexpr int ROWS = GATED ? CM / 2 : CM;
        const int r = (int)threadIdx.x % ROWS, slice = (int)threadIdx.x / ROWS;
        const int64_t row = row_of<GATED>(first / a.nt, mine, r), t0 = (int64_t)(first % a.nt) * a.n;
        const float *all = reinterpret_cast<const float *>(ring) + r;
        auto sum_of = [&](int i, int j) {
            float s = 0.0f;
            for (int p = 0; p < a.split; ++p) s += load_from_rank(all + i * CM + j * ROWS, 2 * p + mine);
            return s;
        };
        if (row < a.p.rows)
            for (int i = part + a.split * slice; i < a.n && t0 + i < a.p.tokens; i += a.split * (THREADS / ROWS))
                store_as(a.p.out, a.p.out_type, (t0 + i) * a.p.ldo + row, GATED ? activation(a.p.act, sum_of(i, 0)) * sum_of(i, 1) : sum_of(i, 0));
        cluster_barrier();                                     // read before the others end
    }
    if (warp == WARP_MMA) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(sy.tmem), "r"(S::TMEM_COLS));
    }
}

int encode_tokens(CUtensorMap *map, const SkimGroupedProduct &p, int box_rows)
{
    void *fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres) != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn) return SKIM_ERR_CUDA;
    const int bytes = p.x_type == SKIM_TYPE_I8 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)p.cols, (cuuint64_t)p.tokens}, strides[1] = {(cuuint64_t)p.ldx * bytes};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / bytes), (cuuint32_t)box_rows}, steps[2] = {1, 1};
    const CUresult r = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(fn)(
        map, p.x_type == SKIM_TYPE_I8 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : p.x_type == SKIM_TYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2,
        const_cast<void *>(p.x), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? SKIM_OK : SKIM_ERR_CUDA;
}

template <int XT, int PER, bool GATED>
int launch(skim_ctx *ctx, const CUtensorMap &map, const GemmArgs &a)
{
    auto kernel = skim_grouped_gemm_kernel<XT, PER, GATED>;
    constexpr size_t SMEM = Shape<XT, PER, GATED>::SMEM;
    SKIM_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SMEM));
    const int pairs = ctx->sm_count / 2, tiles = a.mt * a.nt;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(2 * (a.split > 1 ? tiles * a.split : tiles < pairs ? tiles : pairs)));
    cfg.blockDim = dim3(THREADS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = ctx->stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)(2 * a.split);
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    SKIM_CUDA_OK(cudaLaunchKernelEx(&cfg, kernel, map, a));
    ctx->launches += 1;
    return SKIM_OK;
}
template <int XT, bool GATED>
int launch_by_group(skim_ctx *ctx, const CUtensorMap &map, const GemmArgs &a)
{
    switch (a.p.group) {
    case 128: return launch<XT, 1, GATED>(ctx, map, a);
    case 64: return launch<XT, 2, GATED>(ctx, map, a);
    default: return launch<XT, 4, GATED>(ctx, map, a);
    }
}
template <int XT>
int launch_by_matrices(skim_ctx *ctx, const CUtensorMap &map, const GemmArgs &a)
{
    return a.p.gated ? launch_by_group<XT, true>(ctx, map, a) : launch_by_group<XT, false>(ctx, map, a);
}

// Tiles, and the time that they take, in clocks: a round of tiles takes 4 a token and column step of a group of 128 (or the 740 of the warp that issues the products), more in
// smaller groups, 5000 for its end, and a launch with its start 9000.  Pairs that share columns cost 5000 more, and four of them only as many clusters as the chip's
// parts hold at once (16 of them, on 4096 x 4096: 25 us, pairs of two 17).
int64_t plan_of(const skim_ctx *ctx, const SkimGroupedProduct &p, GemmArgs &a)
{
    a.p = p;
    a.ct = (int)skim_record_tiles(p.cols, SKIM_RECORD_COLS);
    a.rt = skim_record_tiles(p.rows, SKIM_RECORD_ROWS);
    a.mt = (int)skim_record_tiles(p.rows, p.gated ? CM : BM);
    const int per = SKIM_RECORD_COLS / p.group, most = per == 1 ? Shape<0, 1, false>::N : Shape<0, 2, false>::N;
    const int64_t pairs = ctx->sm_count / 2, fewest = skim_record_tiles(p.tokens, most);
    int64_t least = INT64_MAX;
    for (int64_t nt = fewest; nt <= fewest + 2; ++nt) {
        const int n = (int)skim_record_tiles(skim_record_tiles(p.tokens, nt), 32) * 32;
        const int64_t tiles = a.mt * nt;
        if (tiles > 0x1fffffff) break;
        int split = 1;
        while (split < MAX_SPLIT && tiles * split * 2 <= pairs && a.ct >= split * 4 && (split == 1 || tiles <= 8)) split *= 2;
        const int step = per == 1 ? (n < 160 ? 740 : 4 * n + 100) : per == 2 ? 1100 : 2000;
        const int64_t cost = 9000 + (tiles * split + pairs - 1) / pairs * ((int64_t)((a.ct + split - 1) / split) * step + 5000) + (split > 1 ? 5000 : 0);
        if (cost < least) least = cost, a.nt = (int)nt, a.n = n, a.split = split;
    }
    return least;
}

}  // namespace

// Whether the tensor-memory kernel takes the call: tokens enough, rows that TMA can read, and less time than passes of 16 tokens through the other kernel, which take about
// 4000 clocks and 1.5 a record each (us, this kernel and the other: 11008 x 4096, 64 tokens 22 and 47; 4096 x 4096, 32 tokens 17 and 12; 1024 x 1024, 128 tokens 11 and 6).
bool skim_grouped_gemm_takes(const skim_ctx *ctx, const SkimGroupedProduct &p)
{
    const int bytes = p.x_type == SKIM_TYPE_I8 ? 1 : 2;
    if (p.tokens <= 16 || (reinterpret_cast<uintptr_t>(p.x) & 15u) || (p.ldx * bytes) % 16 || p.rows > 0x3fffffff) return false;
    GemmArgs a;
    const int64_t cost = plan_of(ctx, p, a);
    if (cost == INT64_MAX) return false;
    const int64_t passes = (p.tokens + 15) / 16;
    return cost < 4000 + passes * (a.rt * a.ct) * (p.gated ? 6 : 3) / 2;
}

int skim_launch_grouped_gemm(skim_ctx *ctx, const SkimGroupedProduct &p)
{
    GemmArgs a;
    if (plan_of(ctx, p, a) == INT64_MAX) return SKIM_ERR_SHAPE;
    CUtensorMap map;
    const int rc = encode_tokens(&map, p, a.n / 2);
    if (rc) return rc;
    switch (p.x_type) {
    case SKIM_TYPE_F16: return launch_by_matrices<SKIM_TYPE_F16>(ctx, map, a);
    case SKIM_TYPE_BF16: return launch_by_matrices<SKIM_TYPE_BF16>(ctx, map, a);
    default: return launch_by_matrices<SKIM_TYPE_I8>(ctx, map, a);
    }
}
