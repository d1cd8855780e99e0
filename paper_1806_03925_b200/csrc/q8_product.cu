// Products of e4m3 rows with e4m3 weights, an fp32 scale for every 128 columns of a row and every 128 x 128 weights
// (gear_q8_matmul), on the 5th-generation tensor cores:
//
//     out[m][j] = sum_kb a_scale[m][kb] b_scale[j / 128][kb] (sum over k of block kb of a[m][k] b[j][k])
//
// The scales change with every block of 128 along K, so a block's products are a tile of their own: tcgen05.mma leaves them in one
// of a ring of accumulators in tensor memory, and the epilogue warps add them, times the two scales, to sums in registers while the
// tensor cores fill the next accumulator.  A warp's columns lie in one block of weights and a lane holds one row, so a lane has one
// factor per block of K; two columns are multiplied and added per instruction (fma.rn.f32x2).
//
// Bound by the chain of a tile's two accumulators where tiles are 256 wide (products issued to accumulator complete 1050 cycles, read and
// added 640, handed back 250: 970 per block of K with 512 of products in it): 131072 x 2048 x 1024 in 274 us, 2000 TFLOP/s, in a graph
// (in a run of calls, under the power cap, 321 us); by memory where the output is narrow (262144 x 1536 x 64 in fp32: 75 us, 0.98 of the copy rate).
//
// One persistent kernel, a CTA per SM: warps 0 and 3 stream the operands in by TMA (boxes of 128 bytes along K, which are one block),
// warps 1 and 2 issue the products (M 128, N BN, K 32: four per block), warps 4 to 11 add up and store.  Two warps share a quarter of the
// tensor-memory lanes and split the columns.  Every wait is bounded: on a timeout the kernel says so in the status words, leaves
// its loops, waits (bounded again) for the copies and products under way, frees its tensor memory and returns.  No cluster
// launch and no multicast.
#include <type_traits>

#include "internal.h"
#include "q8.cuh"
#include "tc_ptx.cuh"

namespace gear {

constexpr int QP_EW = 8;                                     // epilogue warps
constexpr int QP_THREADS = 128 + 32 * QP_EW;                 // a warpgroup of producers and issuers; the epilogue's two
constexpr int QP_OUT_BLOCK = 32 * 128;                       // a warp's results on their way out: 32 rows of 128 bytes

template <int BN> struct QpCfg {
    static constexpr int A_BYTES = TC_BM * Q8_BLOCK, B_BYTES = BN * Q8_BLOCK, STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int STAGES = BN == 256 ? 4 : 6;
    static constexpr int OUT_BLOCKS = BN == 64 ? 2 : 1;      // a warp's blocks on their way out
    static constexpr int ACCS = BN == 256 ? 2 : 4;           // accumulators: all of the tensor memory, or half of it
    static constexpr int TMEM_COLS = BN * ACCS;
    static constexpr bool SPLIT = BN == 256;                 // registers are handed from the first warpgroup to the others
    static constexpr int SMEM = STAGES * STAGE_BYTES + QP_EW * OUT_BLOCKS * QP_OUT_BLOCK + 1024 /*alignment slack*/ + 256 /*barriers*/;
    // A barrier's phases are told apart by their parity, which takes one thread that waits for every one of them: a stage and an
    // accumulator belong to the same producer and the same issuer (of the two that take blocks in turn) every time.
    static_assert(STAGES % 2 == 0 && ACCS % 2 == 0, "stages and accumulators come round to the same producer and issuer");
    static_assert(SMEM <= 227 * 1024 && SMEM > 116 * 1024, "one CTA per SM: two would both ask for tensor memory");
};

struct QpArgs {
    const float* a_scale; const float* b_scale;
    int64_t n; const int64_t* d_n;
    int N, K, n_tiles;
    void* out; int64_t ld_out; int unit;                     // rows of out start on boundaries of this many bytes: 16 (map_out is set), 4 or 2
    int32_t* status;
};

// Registers of a CTA with 128 columns a warp: launched with 168 a thread (384 x 168 = 64512), the epilogue's two warpgroups take 232,
// the first one keeps 40 (256 x 232 + 128 x 40 = 64512).
constexpr int QP_REGS_FEW = 40, QP_REGS_MANY = 232;

// mbar_wait that looks more often whether another wait has given up: a block whose epilogue has left ends soon.
__device__ __forceinline__ bool qp_wait(uint32_t bar, uint32_t parity, int32_t* err, int code) {
    for (uint32_t i = 0; i < TC_SPIN_LIMIT; ++i) {
        if (mbar_try(bar, parity)) return true;
        if (i > 64) __nanosleep(32);
        if ((i & 63u) == 63u && *reinterpret_cast<volatile int32_t*>(err) != 0) return false;
    }
    atomicCAS(err, 0, code);
    return false;
}
// One lane waits for its warp.
__device__ __forceinline__ bool qp_warp_wait(uint32_t bar, uint32_t parity, int32_t* err, int lane) {
    bool ok = true;
    if (lane == 0) ok = qp_wait(bar, parity, err, 4);
    return __all_sync(0xffffffffu, ok);
}
// All threads of the block meet, each from its own role's code; whether any of them brings a true.
__device__ __forceinline__ bool qp_any(bool mine) {
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(any) : "r"((uint32_t)mine), "n"(QP_THREADS) : "memory");
    return any != 0;
}

__device__ __forceinline__ uint64_t pair64(uint32_t lo, uint32_t hi) { return (uint64_t)lo | (uint64_t)hi << 32; }
__device__ __forceinline__ void fma_pair(uint64_t& acc, uint64_t v, uint64_t s) { asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(v), "l"(s)); }

// A warp's 32 rows x 128 bytes from shared memory (16-byte pieces XOR-swizzled by the row) to the output, where the copy engine cannot
// take them.  out: the block's first row and column; rows, cols: how much of it there is to write; unit: 16 where rows start on 16-byte
// boundaries (eight lanes write a row), else 4 or 2: a row is written by all lanes, a word each, whole lines at a time (16 bytes a lane in
// single values: 97839 x 400 x 306 in bf16 took 197 us).
template <typename T>
__device__ __forceinline__ void qp_store_block(uint32_t block, T* out, int64_t ld, int rows, int cols, int unit, int lane) {
    constexpr int PER = 16 / (int)sizeof(T), IN_WORD = 4 / (int)sizeof(T);
    if (unit == 16) {
        const int piece = lane & 7, row0 = lane >> 3, col = piece * PER;
        uint4 v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = i * 4 + row0;
            asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                         : "r"(block + (uint32_t)row * 128u + (((uint32_t)(piece ^ (row & 7))) << 4)) : "memory");
        }
        T* dst = out + row0 * ld + col;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (i * 4 + row0 >= rows) continue;
            T* d = dst + (int64_t)(4 * i) * ld;
            if (col + PER <= cols) *reinterpret_cast<uint4*>(d) = v[i];
            else {
                const T* e = reinterpret_cast<const T*>(&v[i]);
#pragma unroll
                for (int j = 0; j < PER; ++j) if (col + j < cols) d[j] = e[j];
            }
        }
        return;
    }
    const int col = lane * IN_WORD;
    for (int r0 = 0; r0 < rows; r0 += 8) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = r0 + i;
            asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[i]) : "r"(block + (uint32_t)row * 128u + (((uint32_t)((lane >> 2) ^ (row & 7))) << 4) + (uint32_t)(lane & 3) * 4u) : "memory");
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + i >= rows || col >= cols) continue;
            T* d = out + (int64_t)(r0 + i) * ld + col;
            if (sizeof(T) == 4 || (unit == 4 && col + 1 < cols)) *reinterpret_cast<uint32_t*>(d) = w[i];
            else {
                reinterpret_cast<uint16_t*>(d)[0] = (uint16_t)w[i];
                if (col + 1 < cols) reinterpret_cast<uint16_t*>(d)[1] = (uint16_t)(w[i] >> 16);
            }
        }
    }
}

// A place in a ring of N and the parity of its current round.
template <int N> struct Ring {
    int at = 0;
    uint32_t round = 0;
    __device__ __forceinline__ void next() { if (++at == N) { at = 0; round ^= 1u; } }
};
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

template <int BN, typename T>
__global__ void __launch_bounds__(QP_THREADS, 1)
q8_product_kernel(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out, const QpArgs g) {
    using Cfg = QpCfg<BN>;
    constexpr int STAGES = Cfg::STAGES, ACCS = Cfg::ACCS, COLS = BN / 2;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t tiles = (raw + 1023u) & ~1023u;
    const uint32_t out_blocks = tiles + STAGES * Cfg::STAGE_BYTES;
    const uint32_t bars = out_blocks + QP_EW * Cfg::OUT_BLOCKS * QP_OUT_BLOCK;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto acc_full = [&](int a) { return bars + 8u * (2 * STAGES + a); };
    auto acc_empty = [&](int a) { return bars + 8u * (2 * STAGES + ACCS + a); };
    const uint32_t tmem_word = bars + 8u * (2 * STAGES + 2 * ACCS);
    volatile uint32_t* tmem_word_ptr = reinterpret_cast<volatile uint32_t*>(smem_raw + (tmem_word - raw));
    int32_t* err = g.status + 1;

    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < ACCS; ++a) { mbar_init(acc_full(a), 1); mbar_init(acc_empty(a), QP_EW); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_a) : "memory");
        asm volatile("prefetch.tensormap [%0];" :: "l"(&map_b) : "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(tmem_word), "r"((uint32_t)Cfg::TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = __shfl_sync(0xffffffffu, *tmem_word_ptr, 0);
    wait_for_predecessor();

    int64_t live = g.n;
    if (g.d_n) { const int64_t d = *g.d_n; live = d < live ? (d < 0 ? 0 : d) : live; }
    const int kbs = (g.K + Q8_BLOCK - 1) / Q8_BLOCK;
    const uint32_t total = (uint32_t)((live + TC_BM - 1) / TC_BM) * (uint32_t)g.n_tiles, n_tiles = (uint32_t)g.n_tiles;

    if (warp < 4) {
        if (Cfg::SPLIT) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(QP_REGS_FEW));
        uint32_t it = 0;                                                              // producers: blocks walked past
        uint32_t last_full = 0, last_empty = 0, full_round = 0, empty_round = 0;      // issuers: the barriers of the last block issued
        bool ok = true;
        // ---------------- TMA producers: two warps, every second block of K each (one alone took 690 cycles from block to block); the
        // whole warp walks the loop, so that what it counts stays in uniform registers, and one lane issues
        if (warp == 0 || warp == 3) {
            Ring<STAGES> ring;
            const uint32_t odd = (uint32_t)(warp == 3);
            for (uint32_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
                const int mt = (int)(t / n_tiles), nt = (int)(t - (uint32_t)mt * n_tiles);      // the column tiles of a row tile side by side
                for (int kb = 0; kb < kbs; ++kb, ++it, ring.next()) {
                    if ((it & 1u) != odd) continue;
                    ok = __all_sync(0xffffffffu, qp_wait(empty_bar(ring.at), ring.round ^ 1u, err, 1));
                    if (!ok) break;
                    const uint32_t a_dst = tiles + ring.at * Cfg::STAGE_BYTES, b_dst = a_dst + Cfg::A_BYTES, bar = full_bar(ring.at);
                    if (elect_one()) {
                        mbar_expect_tx(bar, Cfg::STAGE_BYTES);
                        tma_load_2d(a_dst, &map_a, bar, kb * Q8_BLOCK, mt * TC_BM);
                        tma_load_2d(b_dst, &map_b, bar, kb * Q8_BLOCK, nt * BN);
                    }
                    __syncwarp();
                }
            }
        }
        // ---------------- MMA issuers: two warps, every second block of K each (blocks have accumulators of their own, so the order
        // between the two does not matter).  To wait for two barriers and to issue takes 700 cycles from block to block, the
        // products of 256 columns 512.  The whole warp walks the loop, so that what it counts stays in uniform registers; one lane issues.
        if (warp == 1 || warp == 2) {
            constexpr uint32_t idesc = instr_desc_e4m3(BN);
            const uint64_t a_desc = smem_desc(tiles, 16, 1024), b_desc = smem_desc(tiles + Cfg::A_BYTES, 16, 1024);
            Ring<STAGES> ring;
            Ring<ACCS> acc;
            uint32_t mine = (uint32_t)warp & 1u;
            for (uint32_t t = blockIdx.x; t < total && ok; t += gridDim.x) {
                for (int kb = 0; kb < kbs; ++kb, ring.next(), acc.next(), mine ^= 1u) {
                    if (!mine) continue;
                    ok = qp_wait(full_bar(ring.at), ring.round, err, 3) && qp_wait(acc_empty(acc.at), acc.round ^ 1u, err, 2);
                    if (!__all_sync(0xffffffffu, ok)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t step = (uint64_t)(uint32_t)(ring.at * (Cfg::STAGE_BYTES >> 4));      // (addresses in a descriptor are in 16 bytes)
                    const uint32_t d = tmem_base + (uint32_t)(acc.at * BN);
                    if (elect_one()) {
#pragma unroll
                        for (int k = 0; k < Q8_BLOCK / 32; ++k) tc_mma_f8(d, a_desc + step + 2 * k, b_desc + step + 2 * k, idesc, k > 0 ? 1u : 0u);
                        tc_commit(acc_full(acc.at));
                        tc_commit(empty_bar(ring.at));
                    }
                    last_full = acc_full(acc.at); full_round = acc.round; last_empty = empty_bar(ring.at); empty_round = ring.round;
                    __syncwarp();
                }
            }
        }
        // If any wait of the block gave up, in whatever role and however late, copies and products may be under way that nobody has waited
        // for: they land and end before the CTA gives its shared memory, its barriers and its tensor memory back.
        if (qp_any(!ok)) {
            if ((warp == 0 || warp == 3) && lane == 0) {
                const uint32_t first = it > (uint32_t)STAGES ? it - STAGES : 0u, odd = (uint32_t)(warp == 3);
                for (uint32_t j = first; j < it; ++j)
                    for (uint32_t spin = 0; (j & 1u) == odd && spin < (1u << 16) && !mbar_try(full_bar(j % STAGES), (j / STAGES) & 1u); ++spin)
                        __nanosleep(64);
            }
            if (last_full != 0)
                for (uint32_t spin = 0; spin < (1u << 16) && !(mbar_try(last_full, full_round) && mbar_try(last_empty, empty_round)); ++spin)
                    __nanosleep(64);
        }
    } else {
        if (Cfg::SPLIT) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(QP_REGS_MANY));
        // ---------------- epilogue warps
        const int quarter = warp & 3, part = (warp - 4) >> 2;
        const uint32_t block = out_blocks + (uint32_t)(warp - 4) * Cfg::OUT_BLOCKS * QP_OUT_BLOCK;
        const uint32_t t_lane = tmem_base + ((uint32_t)(quarter * 32) << 16) + (uint32_t)(part * COLS);
        // an accumulator is read in pieces of 32 columns, the next one on its way while one is added up: also across accumulators
        constexpr int WIDE = 32, PIECES = COLS / WIDE;
        Ring<ACCS> ring;
        uint32_t sent = 0;                                    // groups of copies (or empty ones) the warp has committed, over all of its tiles
        // (a status that an earlier call has left says that this call's results are void: none are written)
        const uint32_t start = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile int32_t*>(err) == 0 ? blockIdx.x : total, 0);
        bool ok = true;
        for (uint32_t t = start; t < total && ok; t += gridDim.x) {
            const uint32_t mt = t / n_tiles;
            const int nt = (int)(t - mt * n_tiles);
            const int64_t m0 = (int64_t)mt * TC_BM + quarter * 32, m = m0 + lane;
            const int n0 = nt * BN + part * COLS;
            const float* sa = m < live ? g.a_scale + m * kbs : nullptr;
            const float* sb = n0 < g.N ? g.b_scale + (int64_t)(n0 / Q8_BLOCK) * kbs : nullptr;
            uint64_t acc[COLS / 2];
#pragma unroll
            for (int i = 0; i < COLS / 2; ++i) acc[i] = 0ull;
            // (the two factors are multiplied where they are used: a product right behind the loads would wait for them)
            float sa_next = sa && sb ? __ldg(sa) : 0.f, sb_next = sa && sb ? __ldg(sb) : 0.f;
            uint32_t r[2][WIDE];
            ok = qp_warp_wait(acc_full(ring.at), ring.round, err, lane);
            tc_fence_after();
            if (ok) tc_ld32(t_lane + (uint32_t)(ring.at * BN), r[0]);
            // one block of K, whose first piece is in (or on its way to) r[FIRST]; the next block's goes to r[(FIRST + PIECES) & 1]
            auto block_of_k = [&](auto first, int kb) {
                constexpr int FIRST = decltype(first)::value;
                const uint32_t s32 = __float_as_uint(sa_next * sb_next);
                const uint64_t s2 = pair64(s32, s32);
                const bool more = kb + 1 < kbs;
                if (more && sa && sb) { sa_next = __ldg(sa + kb + 1); sb_next = __ldg(sb + kb + 1); }
                const int a = ring.at;
                ring.next();
#pragma unroll
                for (int c = 0; c < PIECES; ++c) {
                    uint32_t (&now)[WIDE] = r[(FIRST + c) & 1];
                    uint32_t (&then)[WIDE] = r[(FIRST + c + 1) & 1];
                    tc_wait_ld(now);
                    if (c + 1 < PIECES) tc_ld32(t_lane + (uint32_t)(a * BN + (c + 1) * WIDE), then);
                    else {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive_relaxed(acc_empty(a));      // all of it has been read
                        if (more) {
                            ok = qp_warp_wait(acc_full(ring.at), ring.round, err, lane);
                            tc_fence_after();
                            tc_ld32(t_lane + (uint32_t)(ring.at * BN), then);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < WIDE / 2; ++i) fma_pair(acc[c * (WIDE / 2) + i], pair64(now[2 * i], now[2 * i + 1]), s2);
                }
            };
            for (int kb = 0; kb < kbs && ok; kb += 2) {
                block_of_k(std::integral_constant<int, 0>{}, kb);
                if (kb + 1 < kbs && ok) block_of_k(std::integral_constant<int, PIECES & 1>{}, kb + 1);
            }
            tc_wait_ld(r[0]); tc_wait_ld(r[1]);               // (nothing is on its way, unless a wait gave up)
            if (!ok) break;
            // a lane's row leaves in pieces of 128 bytes through the warp's block
            T* out = static_cast<T*>(g.out);
            constexpr int PIECE = 128 / (int)sizeof(T);
            static_assert(COLS >= PIECE || sizeof(T) == 2, "a piece is whole or half full");
#pragma unroll
            for (int c = 0; c < (COLS + PIECE - 1) / PIECE; ++c) {
                if (n0 + c * PIECE >= g.N) break;             // (uniform over the warp)
                // the blocks in turn, across tiles: all groups but the last OUT_BLOCKS - 1 have been read, so this block's previous contents have
                const uint32_t box = block + (sent % Cfg::OUT_BLOCKS) * QP_OUT_BLOCK;
                ++sent;
                if (lane == 0) tma_store_wait_read<Cfg::OUT_BLOCKS - 1>();
                __syncwarp();
                const uint32_t row = box + (uint32_t)lane * 128u;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    uint32_t w[4] = {0u, 0u, 0u, 0u};
                    if (sizeof(T) == 4) {
                        const int i = c * (PIECE / 2) + 2 * j;
                        w[0] = (uint32_t)acc[i]; w[1] = (uint32_t)(acc[i] >> 32); w[2] = (uint32_t)acc[i + 1]; w[3] = (uint32_t)(acc[i + 1] >> 32);
                    } else {
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int i = c * (PIECE / 2) + 4 * j + q;
                            if (i >= COLS / 2) continue;      // (32 columns: half a piece)
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float((uint32_t)acc[i]), __uint_as_float((uint32_t)(acc[i] >> 32)));
                            w[q] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                    sts_u4(row + ((((uint32_t)j) ^ (uint32_t)(lane & 7)) << 4), make_uint4(w[0], w[1], w[2], w[3]));
                }
                const int rows = (int)min((int64_t)32, live - m0), cols = min(g.N, n0 + COLS) - (n0 + c * PIECE);     // (of half a piece: the other half is another warp's)
                if (g.unit == 16 && COLS >= PIECE && rows > 0 && (rows == 32 || live == g.n)) {
                    // the copy engine takes it from here and drops what lies past the edges
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) tma_store_2d(&map_out, box, n0 + c * PIECE, (int)m0);
                } else {
                    __syncwarp();
                    if (rows > 0) qp_store_block<T>(box, out + m0 * g.ld_out + n0 + c * PIECE, g.ld_out, rows, cols, g.unit, lane);
                    __syncwarp();
                    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");      // (an empty group, in the place of a copy's)
                }
            }
        }
        if (lane == 0) tma_store_wait_all();
        qp_any(!ok || start >= total);
    }

    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem_base), "r"((uint32_t)Cfg::TMEM_COLS) : "memory");
        if (lane == 0 && *reinterpret_cast<volatile int32_t*>(err) != 0) atomicOr(g.status, GEAR_DEV_TIMEOUT);
    }
}

// ---------------------------------------------------------------- few rows
// Up to QF_ROWS rows at a time: the weights are read once and what there is to compute is little, so a warp has a column of the
// output and reads its weights 16 bytes a lane (eight lanes per block of 128).  e4m3 values and their products are exact in fp32.
constexpr int QF_ROWS = 8;

__device__ __forceinline__ void e4m3_to_f32(const uint4& v, float (&f)[16]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[i >> 1] >> (16 * (i & 1))), __NV_E4M3);
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&h));
        f[2 * i] = p.x; f[2 * i + 1] = p.y;
    }
}
// 16 bytes of a row from byte k on, with zeros from K on.  The word is read whole: it begins in the row, is aligned, and so lies in the row's
// allocation (bytes one by one at the end of the last row: 8 rows of 1535 x 200 3.9 -> 4.9 us, and 3.4 -> 4.2 for 1536 x 64, which has no such end).
__device__ __forceinline__ uint4 load_bytes(const uint8_t* row, int k, int K) {
    uint4 v = __ldg(reinterpret_cast<const uint4*>(row + k));
    if (k + 16 > K) {
        uint32_t* w = reinterpret_cast<uint32_t*>(&v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int left = K - k - 4 * i;                   // bytes of this word that count
            if (left < 4) w[i] = left <= 0 ? 0u : w[i] & ((1u << (8 * left)) - 1u);
        }
    }
    return v;
}

template <int R, typename T>
__global__ void __launch_bounds__(128)
q8_few_rows_kernel(const Q8Args g) {
    wait_for_predecessor();
    int64_t live = g.n;
    if (g.d_n) { const int64_t d = *g.d_n; live = d < live ? (d < 0 ? 0 : d) : live; }
    const int lane = threadIdx.x & 31, j = blockIdx.x * 4 + (threadIdx.x >> 5);
    const int64_t m0 = (int64_t)blockIdx.y * R;
    if (j >= g.N || m0 >= live) return;
    const int rows = (int)min((int64_t)R, live - m0), kbs = (g.K + Q8_BLOCK - 1) / Q8_BLOCK;
    const uint8_t* b = g.b + (int64_t)j * g.ldb;
    const float* sb = g.b_scale + (int64_t)(j / Q8_BLOCK) * kbs;
    float acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0.f;
    for (int k = lane * 16; k < g.K; k += 512) {
        const int kb = k / Q8_BLOCK;
        const uint4 bv = load_bytes(b, k, g.K);
        const float s = __ldg(sb + kb);
        uint4 av[R];
        float sa[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t m = m0 + (r < rows ? r : 0);
            av[r] = load_bytes(g.a + m * g.lda, k, g.K);
            sa[r] = __ldg(g.a_scale + m * kbs + kb);
        }
        float w[16];
        e4m3_to_f32(bv, w);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[16], p = 0.f;
            e4m3_to_f32(av[r], x);
#pragma unroll
            for (int i = 0; i < 16; ++i) p = fmaf(x[i], w[i], p);
            acc[r] = fmaf(p, sa[r] * s, acc[r]);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float v = warp_sum(acc[r]);
        if (lane == 0 && r < rows) static_cast<T*>(g.out)[(m0 + r) * g.ld_out + j] = (T)v;
    }
}

// ---------------------------------------------------------------- host side
template <int BN, typename T> static cudaError_t qp_go(const Q8Args& q, cudaStream_t st) {
    using Cfg = QpCfg<BN>;
    constexpr auto kernel = q8_product_kernel<BN, T>;
    if (const cudaError_t e = allow_smem<kernel>(Cfg::SMEM)) return e;
    CUtensorMap ma, mb;
    if (!encode_map(&ma, TmaSpec{q.a, q.n, q.K, q.lda, 0, 1, TC_BM, Q8_BLOCK, 2, 128}) || !encode_map(&mb, TmaSpec{q.b, q.N, q.K, q.ldb, 0, 1, BN, Q8_BLOCK, 2, 128}))
        return cudaErrorInvalidValue;
    QpArgs g = {};
    g.a_scale = q.a_scale; g.b_scale = q.b_scale; g.n = q.n; g.d_n = q.d_n; g.N = q.N; g.K = q.K;
    g.n_tiles = (int)ceil_div(q.N, BN);
    g.out = q.out; g.ld_out = q.ld_out; g.status = q.status;
    const uintptr_t starts = reinterpret_cast<uintptr_t>(q.out) | (uintptr_t)(q.ld_out * (int64_t)sizeof(T));
    g.unit = starts % 16 == 0 ? 16 : starts % 4 == 0 ? 4 : 2;
    CUtensorMap mo = ma;
    if (g.unit == 16 && !encode_map(&mo, TmaSpec{q.out, q.n, q.N, q.ld_out, 0, 1, 32, 128 / (int)sizeof(T), sizeof(T) == 4, 128})) return cudaErrorInvalidValue;
    const int64_t tiles = ceil_div(q.n, TC_BM) * g.n_tiles;
    if (tiles > INT32_MAX) return cudaErrorInvalidValue;     // (an output of 2^31 tiles fits no memory)
    const int grid = tiles < sm_count() ? (int)tiles : sm_count();
    return launch_now(kernel, dim3(grid), dim3(QP_THREADS), (size_t)Cfg::SMEM, st, ma, mb, mo, g);
}
template <int R, typename T> static cudaError_t qf_go(const Q8Args& q, cudaStream_t st) {
    return launch_now(q8_few_rows_kernel<R, T>, dim3((unsigned)ceil_div(q.N, 4), (unsigned)ceil_div(q.n, R)), dim3(128), 0, st, q);
}

template <typename T> static cudaError_t qp_launch(const Q8Args& q, cudaStream_t st) {
    // A warp for every column and R rows, while that makes few blocks for every SM: 1536 x 256, 16 rows 3.5 us (tiles 6.1), 32 rows 4.4 (6.3), 64
    // rows 6.4 (6.4); 2048 x 1024, 8 rows 5.2 (7.0), 16 rows 7.8 (7.1).
    const int rows = q.n <= 1 ? 1 : q.n <= 2 ? 2 : q.n <= 4 ? 4 : QF_ROWS;
    if (ceil_div(q.N, 4) * ceil_div(q.n, rows) * rows <= 16 * (int64_t)sm_count())
        return rows == 1 ? qf_go<1, T>(q, st) : rows == 2 ? qf_go<2, T>(q, st) : rows == 4 ? qf_go<4, T>(q, st) : qf_go<QF_ROWS, T>(q, st);
    // The width of the tiles by what the busiest SM then has to do: its tiles, each some time per block of K and some for its start and its
    // results (in 10 ns, from launches of 512 to 131072 rows, K 80 to 2048, N 64 to 1024).
    const int64_t m_tiles = ceil_div(q.n, TC_BM), kbs = ceil_div(q.K, Q8_BLOCK);
    auto cost = [&](int bn, int64_t block, int64_t rest) { return ceil_div(m_tiles * ceil_div(q.N, bn), sm_count()) * (kbs * block + rest); };
    const int64_t c64 = cost(64, 36, 80), c128 = cost(128, 39, 100), c256 = cost(256, 55, 200);
    if (c64 <= c128 && c64 <= c256) return qp_go<64, T>(q, st);
    return c128 <= c256 ? qp_go<128, T>(q, st) : qp_go<256, T>(q, st);
}

cudaError_t launch_q8_product(const Q8Args& q, cudaStream_t st) {
    if (q.n <= 0) return cudaSuccess;
    return q.out_dtype == GEAR_BF16 ? qp_launch<__nv_bfloat16>(q, st) : qp_launch<float>(q, st);
}

}  // namespace gear
