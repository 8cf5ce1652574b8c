// Weight gradient of a layer from its input's 8-bit checkpoint:  dW[k][n] (+)= sum_r f(x[r][k]) dY[r][n],  f = identity or ReLU, on the
// 5th-generation tensor cores (small ones: k_wgrad_few).
//
// A kept value is an e4m3 number times a power of two: exact in bf16.  dY is one bf16 term, or two (fp16) or three (fp32) that sum to it, in planes
// that a first kernel writes.  So every product is exact in the MMA and the sums are the only rounding.  Both operands have the contraction index r
// as their slow index ("MN-major").
//
// A CTA, or a pair of CTAs whose tensor cores work as one, owns tiles of dW (128 x BN, or 256 x BN with a half of either operand in each CTA) and walks
// over rows in chunks of 64:
//   warp 0       TMA: the 64 x 128 codes and the planes of dY (64 x 64 boxes, 128-byte swizzle) into a ring of stages
//   then         three warpgroups (two with more than one plane) turn codes into bf16 in the swizzled layout, a chunk each in turn (a thread makes 16
//                bytes of 8 codes of a row; block scales are fetched ahead)
//   warp 1       (of a pair: the first CTA's) tcgen05.mma into one of two accumulators in tensor memory; commits free the stage
//   and two      add a finished accumulator to sums in registers; behind a tile's last chunk store them
// The tensor core's fp32 accumulation rounds toward zero, which biases long sums (about 5e-8 of the sum an MMA): an accumulator takes at most 32
// MMAs (512 rows of one bf16 term) and the groups are added with round-to-nearest.
// The chunks of all tiles, one tile after the other, are dealt out in equal runs, so that every SM has the same work; a tile that several runs share is
// summed from partial tiles, in their order, by a last kernel.
// What bounds it: shared memory.  A chunk of a lone CTA's 128 x 256 tile moves 112 KB there in the 512 cycles of its MMAs, a pair's 80 KB (dY's half is
// fetched and read once by each).  524288 x 1024 x 1024 bf16: 976 us in a burst, 1.13 PFLOP/s, and 1143 sustained
// (cuBLAS, the bf16 product alone: 816 and 980).  The tensor pipe is active 54 % of the time: codes come late, too.
#include <algorithm>
#include <cstring>
#include <type_traits>

#include "ckpt.cuh"
#include "tc_common.cuh"
#include "token_rows.cuh"

namespace anakin {
namespace ckpt {
namespace {

template <int BN_, int P_, bool PAIR>
struct Cfg {
    static constexpr int BN = BN_, P = P_, KC = 64, CONVERT = P == 1 ? 3 : 2, THREADS = 128 * (3 + CONVERT);  // CONVERT: converting warpgroups
    static constexpr int NB = PAIR ? BN / 2 : BN;  // columns of dY that a CTA holds
    static constexpr int BOX = 64 * 64 * 2;
    static constexpr int A_BYTES = 2 * BOX, B_PLANE = (NB / 64) * BOX, CODES = KC * 128;
    static constexpr int STAGE = A_BYTES + P * B_PLANE + CODES;
    static constexpr int FIT = (232448 - 1024 - 512) / STAGE;
    static constexpr int STAGES = FIT >= 6 ? 6 : FIT;
    static constexpr int GROUP = P == 1 ? 8 : P == 2 ? 4 : 2;  // chunks an accumulator takes: 32, 32 and 24 MMAs
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + 1024 + 512;
};

struct Maps {
    CUtensorMap codes, b[3];
};
struct Args {
    int R, K, N, blocks;
    int tiles_m, chunks;           // tiles along k; chunks of a tile
    long long run, total;          // chunks of a run, of all tiles
    int per_tile, tiles;           // per_tile > 0: so many runs to each tile, all tiles' first ones first; 0: runs go on from one tile to the next
    const uint8_t* scales;
    float* out;                    // dW, or partial tiles: that of a tile's i-th run at i * part_stride
    long long ld, part_stride;
    int add, relu;                 // add: to what dW holds
    int32_t* status;
};

// A run: tile after tile, chunk after chunk; groups of chunks end with a tile, with the run, and after GROUP chunks.
template <int GROUP>
struct Walk {
    int left, tile, chunk, in_group;
    __device__ __forceinline__ Walk(const Args& a, long long begin, long long end) : left((int)(end - begin)), tile((int)(begin / a.chunks)), chunk((int)(begin % a.chunks)), in_group(0) {}
    __device__ __forceinline__ bool tile_ends(const Args& a) const { return chunk == a.chunks - 1 || left == 1; }
    __device__ __forceinline__ bool group_ends(const Args& a) const { return in_group == GROUP - 1 || tile_ends(a); }
    __device__ __forceinline__ void next(const Args& a) {
        in_group = group_ends(a) ? 0 : in_group + 1;
        --left;
        if (++chunk == a.chunks) { chunk = 0; ++tile; }
    }
    // To the last chunk of the group.
    __device__ __forceinline__ void to_group_end(const Args& a) {
        const int more = min(min(GROUP - 1 - in_group, a.chunks - 1 - chunk), left - 1);
        chunk += more;
        in_group += more;
        left -= more;
    }
};

// v[J0 .. J0 + 31] of 32 lanes turned over: lane l's j-th becomes lane j's l-th.
template <int J0, int COLS>
__device__ __forceinline__ void transpose32(float (&v)[COLS], int lane) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) {
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            if (j & s) continue;
            const bool up = lane & s;
            const float x = __shfl_xor_sync(0xFFFFFFFFu, up ? v[J0 + j] : v[J0 + (j | s)], s);
            if (up) v[J0 + j] = x;
            else v[J0 + (j | s)] = x;
        }
    }
}

template <int BN, int P, bool PAIR>
__global__ void __launch_bounds__((Cfg<BN, P, PAIR>::THREADS), 1) k_ckpt_wgrad(const __grid_constant__ Maps maps, Args a) {
    using C = Cfg<BN, P, PAIR>;
    // A barrier of codes is waited on by one warpgroup, every time it is used: one that skipped a phase could take an older one for its own.  So there is one
    // for each stage and warpgroup.
    constexpr int RAWS = C::STAGES * C::CONVERT;
    constexpr int STAGES = C::STAGES, GROUP = C::GROUP, NCTA = PAIR ? 2 : 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* base = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    // raw: this CTA's codes (alone: and dY) have arrived; of a pair's first CTA: rawb: both halves of dY; full: operand A is written, in both
    uint64_t* raw = (uint64_t*)(base + STAGES * C::STAGE);
    uint64_t* rawb = raw + RAWS;
    uint64_t* full = rawb + STAGES;
    uint64_t* empty = full + STAGES;
    uint64_t* accfull = empty + STAGES;
    uint64_t* accempty = accfull + 2;
    uint32_t* tmem_slot = (uint32_t*)(accempty + 2);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const int rank = PAIR ? (int)tc::cluster_ctarank() : 0;
    const long long run = blockIdx.x / NCTA;
    const long long begin = a.per_tile > 0 ? run % a.tiles * a.chunks + run / a.tiles * a.run : run * a.run;
    const long long end = min(begin + a.run, a.per_tile > 0 ? (run % a.tiles + 1) * a.chunks : a.total);
    auto row0 = [&](int tile) { return (tile % a.tiles_m) * (128 * NCTA) + rank * 128; };  // this CTA's first row of dW
    auto col0 = [&](int tile) { return (tile / a.tiles_m) * BN; };

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            tc::mbar_init(&rawb[s], 1);
            tc::mbar_init(&full[s], 128 * NCTA);
            tc::mbar_init(&empty[s], 1);
        }
        for (int s = 0; s < RAWS; ++s) tc::mbar_init(&raw[s], 1);
        for (int q = 0; q < 2; ++q) { tc::mbar_init(&accfull[q], 1); tc::mbar_init(&accempty[q], 256 * NCTA); }
        tc::mbar_fence_init();
        tc::prefetch_map(&maps.codes);
        tc::prefetch_map(&maps.b[0]);
    }
    if (wid == 2) {
        if (PAIR) tc::tmem_alloc_pair(tmem_slot, 2 * BN);
        else tc::tmem_alloc(tmem_slot, 2 * BN);
    }
    tc::tc_fence_before();
    __syncthreads();
    if (PAIR) tc::cluster_sync_all();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();
    bool ok = true;
    // barriers that the pair's first CTA waits on, arrived at from both
    auto arrive_first = [&](uint64_t* bar) {
        if (PAIR) tc::mbar_arrive_remote_cta_release(tc::mapa(tc::smem_u32(bar), 0));
        else tc::mbar_arrive(bar);
    };
    auto wait_both = [&](uint64_t* bar, uint32_t parity) { return PAIR ? tc::mbar_wait_cluster(bar, parity) : tc::mbar_wait(bar, parity); };
    auto commit = [&](uint64_t* bar) {
        if (PAIR) tc::umma_commit_pair(bar, 3);
        else tc::umma_commit(bar);
    };

    if (wid < 4) {
        tc::regs_dec<32>();
        if (wid == 0 && lane == 0) {
            Walk<GROUP> w(a, begin, end);
            for (int u = 0; w.left > 0; ++u, w.next(a)) {
                const int s = u % STAGES, r0 = w.chunk * C::KC;
                if (u >= STAGES) ok = tc::mbar_wait_long(&empty[s], ((u / STAGES) - 1) & 1);
                if (!ok) break;
                unsigned char* st = base + s * C::STAGE;
                uint64_t* codes = &raw[u % RAWS];
                tc::mbar_expect_tx(codes, C::CODES + (PAIR ? 0 : P * C::B_PLANE));
                if (PAIR && rank == 0) tc::mbar_expect_tx(&rawb[s], 2 * P * C::B_PLANE);
                tc::tma_load_2d(st + C::A_BYTES + P * C::B_PLANE, &maps.codes, codes, row0(w.tile), r0);
                const int n0 = col0(w.tile) + rank * C::NB;
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int bx = 0; bx < C::NB / 64; ++bx) {
                        unsigned char* dst = st + C::A_BYTES + p * C::B_PLANE + bx * C::BOX;
                        if (PAIR) tc::tma_load_2d_pair(dst, &maps.b[p], tc::mapa(tc::smem_u32(&rawb[s]), 0), n0 + 64 * bx, r0);
                        else tc::tma_load_2d(dst, &maps.b[p], codes, n0 + 64 * bx, r0);
                    }
            }
            if (!ok && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
        } else if (wid == 1 && rank == 0) {
            const uint32_t idesc = tc::umma_idesc<1>(128 * NCTA, BN, true, true);
            int grp = 0;
            Walk<GROUP> w(a, begin, end);
            for (int u = 0; w.left > 0; ++u) {
                const int s = u % STAGES;
                const uint32_t acc = tmem + (uint32_t)((grp & 1) * BN);
                const bool first = w.in_group == 0, last = w.group_ends(a);
                if (first && grp >= 2) ok = wait_both(&accempty[grp & 1], ((grp >> 1) - 1) & 1);
                ok = tc::warp_all(ok && (PAIR ? tc::mbar_wait(&rawb[s], (u / STAGES) & 1) : tc::mbar_wait(&raw[u % RAWS], (u / RAWS) & 1)) && wait_both(&full[s], (u / STAGES) & 1));
                if (!ok) break;
                tc::tc_fence_after();
                unsigned char* sa = base + s * C::STAGE;
                unsigned char* sb = sa + C::A_BYTES;
                if (tc::elect_one()) {
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)  // (the small terms first)
#pragma unroll
                        for (int k16 = 0; k16 < C::KC / 16; ++k16) {
                            const uint64_t ad = tc::umma_desc(sa + k16 * 2048, C::BOX, 1024), bd = tc::umma_desc(sb + p * C::B_PLANE + k16 * 2048, C::BOX, 1024);
                            const uint32_t more = (!first || k16 > 0 || p < P - 1) ? 1u : 0u;
                            if (PAIR) tc::umma_pair(acc, ad, bd, idesc, more);
                            else tc::umma(acc, ad, bd, idesc, more);
                        }
                    commit(&empty[s]);
                    if (last) commit(&accfull[grp & 1]);
                }
                __syncwarp();
                if (last) ++grp;
                w.next(a);
            }
            if (!ok && lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
        }
    } else if (wid < 4 + 4 * C::CONVERT) {
        tc::regs_dec<C::CONVERT == 3 ? 40 : 64>();  // (launched with 80 or 96 a thread: 32 + 3 40 + 2 160 <= 6 80, 32 + 2 64 + 2 160 = 5 96)
        constexpr int WGS = C::CONVERT;
        const int wg = (wid >> 2) - 1;
        // A thread has a row's 64 columns of one half of the tile: two scales, eight times 8 codes -> 16 bytes.  It takes them in the order j ^ g(row), g and
        // row ^ g(row) both permutations of 0 .. 7 (twice and three times the row in GF(8); the second half's complemented): then neither the loads
        // nor the swizzled stores of a warp meet in a bank.
        const int row = (tid & 127) >> 1, half = tid & 1, r7 = row & 7, g = (((r7 << 1) ^ (r7 & 4 ? 11 : 0)) & 7) ^ (half ? 7 : 0);
        const uint32_t src0 = (uint32_t)(C::A_BYTES + P * C::B_PLANE + row * 128 + half * 64 + g * 8), dst0 = (uint32_t)(half * C::BOX + row * 128 + ((g ^ r7) << 4));
        const uint32_t relu = a.relu ? 0xFFFFFFFFu : 0u;
        uint32_t sc0, sc1;  // of the first four in that order, and of the others
        // This warpgroup's next chunk: its tile (and the block of columns in it that this thread begins with), its number in it, how many are left.
        Walk<GROUP> w(a, begin, end);
        int tile = w.tile, chunk = w.chunk, left = w.left, blk = 0;
        auto skip = [&](int on) {
            left -= on;
            for (chunk += on; chunk >= a.chunks; chunk -= a.chunks) blk = (row0(++tile) >> 5) + 2 * half;
        };
        blk = (row0(tile) >> 5) + 2 * half;
        skip(wg);
        auto fetch = [&]() {
            const int r = chunk * C::KC + row, b0 = blk + (g >> 2), b1 = b0 ^ 1;  // (blk is even)
            const uint8_t* p = a.scales + (size_t)r * a.blocks;
            const bool in = left > 0 && r < a.R;
            sc0 = in && b0 < a.blocks ? (uint32_t)p[b0] : 0u;
            sc1 = in && b1 < a.blocks ? (uint32_t)p[b1] : 0u;
        };
        auto convert = [&](int u, int s) {
            // (a stage's last MMAs have finished before its codes were asked for: operand A may be written again)
            ok = tc::mbar_wait_long(&raw[u % RAWS], (u / RAWS) & 1);
            if (!ok) return;
            unsigned char* st = base + s * C::STAGE;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint2 q = *reinterpret_cast<const uint2*>(st + (src0 ^ (uint32_t)(j * 8)));
                q = make_uint2(relu_codes(q.x, relu), relu_codes(q.y, relu));
                float v[8];
                decode8(q, j < 4 ? sc0 : sc1, v);
                *reinterpret_cast<uint4*>(st + (dst0 ^ (uint32_t)(j * 16))) = tok::pack16(v, (const __nv_bfloat16*)nullptr);
            }
            tc::fence_proxy_async();
            arrive_first(&full[s]);
            skip(WGS);
            fetch();
        };
        fetch();
        for (int u = wg, s = wg % STAGES; left > 0 && ok; u += WGS) {
            convert(u, s);
            s += WGS;
            if (s >= STAGES) s -= STAGES;
        }
        if (!ok && lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
    } else {
        tc::regs_inc<160>();
        constexpr int COLS = BN / 2;
        const int q = wid & 3, half = (wid >> 2) - 1 - C::CONVERT;
        float sum[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) sum[j] = 0.f;
        int grp = 0;
        for (Walk<GROUP> f(a, begin, end); f.left > 0; f.next(a)) {
            f.to_group_end(a);
            ok = tc::warp_all(ok && tc::mbar_wait_long(&accfull[grp & 1], (grp >> 1) & 1));
            if (ok) {
                tc::tc_fence_after();
                const uint32_t acc = tmem + (uint32_t)((grp & 1) * BN + half * COLS) + ((uint32_t)(32 * q) << 16);
#pragma unroll
                for (int j0 = 0; j0 < COLS; j0 += 16) {
                    uint32_t r[16];
                    tc::tmem_ld16_nowait(acc + (uint32_t)j0, r);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[j0 + j] += __uint_as_float(r[j]);
                }
                tc::tc_fence_before();
                arrive_first(&accempty[grp & 1]);
            }
            ++grp;
            if (f.tile_ends(a)) {
                const int m = row0(f.tile) + 32 * q + lane, nb = col0(f.tile) + half * COLS;
                // which of the tile's runs this is
                const long long part = a.per_tile > 0 ? run / a.tiles : run - (long long)f.tile * a.chunks / a.run;
                if (!ok) {  // the caller sees it in the result, too
#pragma unroll
                    for (int j = 0; j < COLS; ++j) sum[j] = NAN;
                }
                // (a warp stores 32 neighbours of a row at a time; rows of dW may start anywhere)
                float* row = a.out + (size_t)part * a.part_stride + (long long)(m - lane) * a.ld;
                auto store = [&](auto first) {
                    constexpr int J0 = decltype(first)::value;
                    transpose32<J0>(sum, lane);
                    const int n = nb + J0 + lane, rows = n < a.N ? min(a.K - (m - lane), 32) : 0;
                    if (a.add) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (j < rows) sum[J0 + j] += row[j * a.ld + n];
                    }
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (j < rows) row[j * a.ld + n] = sum[J0 + j];
                };
                store(std::integral_constant<int, 0>{});
                if constexpr (COLS > 32) store(std::integral_constant<int, 32>{});
                if constexpr (COLS > 64) {
                    store(std::integral_constant<int, 64>{});
                    store(std::integral_constant<int, 96>{});
                }
#pragma unroll
                for (int j = 0; j < COLS; ++j) sum[j] = 0.f;
            }
        }
        if (!ok && lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
    }
    tc::tc_fence_before();
    __syncthreads();
    if (PAIR) tc::cluster_sync_all();
    if (wid == 2) {
        if (PAIR) tc::tmem_dealloc_pair(tmem, 2 * BN);
        else tc::tmem_dealloc(tmem, 2 * BN);
    }
}

// Partial tiles summed in a fixed order.  WARPS = 1: a warp takes four segments of 32 neighbours of a row, a few parts each;
// 8: a block takes one segment, every warp each 8th part of it, so that many parts of a small dW are all in flight.
struct Parts {
    const float* at;
    long long stride;
    FastDiv run;
    int per_tile, chunks, tiles_m, log_k, log_n, pitch;  // (as in Args; a tile is 2^log_k x 2^log_n)
    __device__ __forceinline__ int count(int k, int n) const {
        if (per_tile > 0 || chunks == 0) return per_tile;
        const uint32_t t = (uint32_t)((n >> log_n) * tiles_m + (k >> log_k)) * (uint32_t)chunks;
        return (int)(run.div(t + chunks - 1) - run.div(t)) + 1;
    }
};
template <int WARPS>
__global__ void __launch_bounds__(256) k_wgrad_sum(Parts p, FastDiv per_row, uint32_t segments, int N, float* dw, long long ld, int add) {
    pdl_wait();
    constexpr int U = WARPS == 1 ? 4 : 1;
    __shared__ float sums[8][33];
    const int lane = threadIdx.x & 31, wid = threadIdx.x >> 5;
    const uint32_t first = WARPS == 1 ? (blockIdx.x * 8 + wid) * U : blockIdx.x, step = gridDim.x * (WARPS == 1 ? 8 * U : 1);
    for (uint32_t i0 = first; i0 < segments; i0 += step) {
        float v[U], old[U];
        const float* src[U];
        float* dst[U];
        int parts[U], most = 0;
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const uint32_t i = min(i0 + q, segments - 1), k = per_row.div(i);
            const int n = (int)(i - k * per_row.d) * 32 + lane;
            parts[q] = i0 + q < segments && n < N ? p.count((int)k, n) : 0;
            src[q] = p.at + (size_t)k * p.pitch + n;
            dst[q] = i0 + q < segments && n < N ? dw + k * ld + n : nullptr;
            old[q] = add && dst[q] && wid % WARPS == 0 ? *dst[q] : 0.f;
            v[q] = 0.f;
            most = max(most, parts[q]);
        }
        if constexpr (WARPS == 1) {
            for (int s = 0; s < most; ++s) {
#pragma unroll
                for (int q = 0; q < U; ++q)
                    if (s < parts[q]) v[q] += src[q][(size_t)s * p.stride];
            }
        } else {
#pragma unroll 8
            for (int s = wid; s < most; s += 8) v[0] += src[0][(size_t)s * p.stride];
            sums[wid][lane] = v[0];
            __syncthreads();
            v[0] = 0.f;
            if (wid == 0) {
#pragma unroll
                for (int w = 0; w < 8; ++w) v[0] += sums[w][lane];
            }
            __syncthreads();
            if (wid != 0) continue;
        }
#pragma unroll
        for (int q = 0; q < U; ++q)
            if (dst[q]) *dst[q] = add ? old[q] + v[q] : v[q];
    }
}

// dY as P bf16 planes [rows][pitch] that sum to it (fp32: 24 bits in three; fp16: 11 bits in two; bf16 whose rows TMA cannot address: one).  A thread
// takes 8 neighbouring elements: as 16-byte words where rows start on such boundaries (VEC), else as 4-byte words, those of 16-bit types that start
// in the middle of one shifted into place (5003 x 4099 bf16: 15 us, by 2-byte loads 19.5).
template <class T, int P, bool VEC>
__global__ void __launch_bounds__(256) k_split_planes(const T* dy, long long ld, FastDiv per_row, uint32_t pieces, int N, int pitch, __nv_bfloat16* planes,
                                                      long long plane) {
    pdl_wait();
    constexpr int E = 8, U = VEC ? 1 : 2;  // U: pieces of a thread in flight
    for (uint32_t i0 = blockIdx.x * 256 * U + threadIdx.x; i0 < pieces; i0 += gridDim.x * 256 * U) {
        float v[U][E];
        __nv_bfloat16* out[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const uint32_t i = min(i0 + 256 * q, pieces - 1);
            const uint32_t r = per_row.div(i);
            const int j = (int)(i - r * per_row.d) * E;
            const T* src = dy + (long long)r * ld + j;
            const int odd = sizeof(T) == 2 ? (int)((uintptr_t)src >> 1 & 1) : 0;  // from the middle of a word on
            out[q] = planes + (long long)r * pitch + j;
            if (j >= odd && j + E + odd <= N) {  // (whole words lie within the row)
                constexpr int W = E * (int)sizeof(T) / 4;
                uint32_t w[W + 1];
                if constexpr (VEC) {
#pragma unroll
                    for (int k = 0; k < W; k += 4) *reinterpret_cast<uint4*>(w + k) = reinterpret_cast<const uint4*>(src)[k / 4];
                } else {
                    const uint32_t* at = reinterpret_cast<const uint32_t*>(src - odd);
#pragma unroll
                    for (int k = 0; k < W; ++k) w[k] = at[k];
                    if (odd) {
                        w[W] = at[W];
#pragma unroll
                        for (int k = 0; k < W; ++k) w[k] = __funnelshift_r(w[k], w[k + 1], 16);
                    }
                }
                constexpr int V = 16 / sizeof(T);
#pragma unroll
                for (int k = 0; k < E; k += V) {
                    float f[V];
                    const int k4 = k * (int)sizeof(T) / 4;
                    tok::unpack16(make_uint4(w[k4], w[k4 + 1], w[k4 + 2], w[k4 + 3]), f, (const T*)nullptr);
#pragma unroll
                    for (int u = 0; u < V; ++u) v[q][k + u] = f[u];
                }
            } else {
#pragma unroll
                for (int k = 0; k < E; ++k) v[q][k] = j + k < N ? tok::to_f(src[k]) : 0.f;
            }
        }
#pragma unroll
        for (int q = 0; q < U; ++q) {
            if (i0 + 256 * q >= pieces) continue;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                uint32_t w[E / 2];
#pragma unroll
                for (int k = 0; k < E; k += 2) {
                    // (cut, not rounded: never past bf16's largest, and 8 bits a term are all 24)
                    const uint32_t a = v[q][k] == v[q][k] ? __float_as_uint(v[q][k]) & 0xFFFF0000u : 0x7FC00000u;
                    const uint32_t b = v[q][k + 1] == v[q][k + 1] ? __float_as_uint(v[q][k + 1]) & 0xFFFF0000u : 0x7FC00000u;
                    w[k / 2] = a >> 16 | b;
                    // (an infinity stays one: its rest would be NaN)
                    v[q][k] = fabsf(v[q][k]) < INFINITY ? v[q][k] - __uint_as_float(a) : 0.f;
                    v[q][k + 1] = fabsf(v[q][k + 1]) < INFINITY ? v[q][k + 1] - __uint_as_float(b) : 0.f;
                }
                *reinterpret_cast<uint4*>(out[q] + p * plane) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    }
}

// Up to 32 rows: what there is to do is to write dW, and setting tensor cores up costs more than the products (4 x 1024 x 32768 bf16: 27 us, by tensor
// cores 82; 32 rows 77; 32 x 1024 x 1024 7.7 and 11.8; with 48 rows tensor cores are ahead where tiles are many).  A CTA takes 64 rows of dW x 128
// columns, a warp 8 rows, a lane 4 columns of them 32 apart.  Sums in the order of the rows, fp32, one rounding a product.
// More rows while dW is small, too: 16 of them to a CTA (blockIdx.y), partial sums as from the tensor cores' runs (1024 x 64 x 64 fp32: 5.9 us, with 32
// rows 9.0, by tensor cores 9.9; 640 x 256 x 256 bf16 11.9, 13.2 and 14.7).
constexpr int kFewRows = 32, kSplitRows = 16, kFewK = 64, kFewN = 128;
template <class T, int ROWS>
__global__ void __launch_bounds__(256) k_wgrad_few(const uint8_t* codes, const uint8_t* scales, const T* dy, long long lddy, int R, int K, int N, int blocks, uint32_t tiles_n,
                                                   int relu, float* dw, long long lddw, long long part_stride, int add) {
    PDL_START();
    codes += (size_t)blockIdx.y * ROWS * blocks * 32;
    scales += (size_t)blockIdx.y * ROWS * blocks;
    dy += (long long)blockIdx.y * ROWS * lddy;
    dw += blockIdx.y * part_stride;
    R = min(R - (int)blockIdx.y * ROWS, ROWS);
    __shared__ __align__(16) float xs[ROWS][kFewK];
    __shared__ float ys[ROWS][kFewN];
    const int tid = threadIdx.x, lane = tid & 31, wid = tid >> 5;
    const uint32_t on = relu ? 0xFFFFFFFFu : 0u;
    const int k0 = (int)(blockIdx.x / tiles_n) * kFewK, n0 = (int)(blockIdx.x % tiles_n) * kFewN;
    float v[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) v[i][j] = 0.f;
    const int xr = tid >> 3, xk = k0 + (tid & 7) * 8;
    if (xr < R && xk < blocks * 32) {
        uint2 q = *reinterpret_cast<const uint2*>(codes + (size_t)xr * blocks * 32 + xk);
        q = make_uint2(relu_codes(q.x, on), relu_codes(q.y, on));
        float f[8];
        decode8(q, scales[(size_t)xr * blocks + xk / 32], f);
        float4* to = reinterpret_cast<float4*>(&xs[xr][xk - k0]);
        to[0] = make_float4(f[0], f[1], f[2], f[3]);
        to[1] = make_float4(f[4], f[5], f[6], f[7]);
    }
    const int c = tid & 127;
#pragma unroll
    for (int i = 0; i < ROWS / 2; ++i) {
        const int r = 2 * i + (tid >> 7);
        if (r < R) ys[r][c] = n0 + c < N ? tok::to_f(dy[(long long)r * lddy + n0 + c]) : 0.f;
    }
    __syncthreads();
#pragma unroll 4
    for (int r = 0; r < R; ++r) {
        const float4 a = *reinterpret_cast<const float4*>(&xs[r][8 * wid]), b = *reinterpret_cast<const float4*>(&xs[r][8 * wid + 4]);
        const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float y = ys[r][32 * j + lane];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i][j] = fmaf(x[i], y, v[i][j]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = k0 + 8 * wid + i;
        float* row = dw + (long long)k * lddw + n0 + lane;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (k < K && n0 + 32 * j + lane < N) row[32 * j] = add ? row[32 * j] + v[i][j] : v[i][j];
    }
}
// CTAs that share the rows, 0 for work of the tensor cores: one for 32 rows at most, more while all tiles are at work at once.
int few_splits(long long R, long long K, long long N) {
    const long long splits = (R + kSplitRows - 1) / kSplitRows, tiles = ((K + kFewK - 1) / kFewK) * ((N + kFewN - 1) / kFewN);
    return R <= kFewRows ? 1 : splits <= 128 && tiles * splits <= 148 * 4 ? (int)splits : 0;
}
int partial_width(long long N) { return (int)((N + 31) / 32 * 32); }
template <class T>
cudaError_t launch_few(const uint8_t* codes, const uint8_t* scales, const void* dy, long long lddy, int splits, int R, int K, int N, int relu, float* dw, long long lddw,
                       long long part_stride, int add, cudaStream_t s) {
    const uint32_t tiles_n = (uint32_t)((N + kFewN - 1) / kFewN), tiles = tiles_n * (uint32_t)((K + kFewK - 1) / kFewK);
    const dim3 grid(tiles, splits), block(256);
    return splits == 1 ? launch<k_wgrad_few<T, kFewRows>>(grid, block, 0, s, codes, scales, static_cast<const T*>(dy), lddy, R, K, N, (K + 31) / 32, tiles_n, relu, dw, lddw, part_stride, add)
                       : launch<k_wgrad_few<T, kSplitRows>>(grid, block, 0, s, codes, scales, static_cast<const T*>(dy), lddy, R, K, N, (K + 31) / 32, tiles_n, relu, dw, lddw, part_stride, add);
}
// (parts: the most that any element has)
cudaError_t launch_sum(const Parts& p, int parts, int K, int N, float* dw, long long lddw, int add, cudaStream_t s) {
    const uint32_t per_row = (uint32_t)(p.pitch / 32), segments = (uint32_t)K * per_row;
    // (a dW of few segments leaves most of the GPU's warps free for the parts)
    return parts > 4 && segments < 148 * 32 ? launch<k_wgrad_sum<8>>(dim3(segments), dim3(256), 0, s, p, FastDiv(per_row), segments, N, dw, lddw, add)
                                            : launch<k_wgrad_sum<1>>(dim3(std::min((segments + 31) / 32, 148u * 16)), dim3(256), 0, s, p, FastDiv(per_row), segments, N, dw, lddw, add);
}

struct Plan {
    int P, BN, pitch, width, runs, per_tile, tiles_m, tiles, chunks, parts;  // parts: the most runs that share a tile; width: floats of a partial row
    long long run, total;
    bool direct, pair, straight;  // TMA reads the caller's dY; pairs of CTAs; the tiles are stored into dW
    size_t plane_bytes, part_off, bytes;
};

Plan make_plan(int dtype, long long R, long long K, long long N, const void* dy, long long lddy) {
    Plan p = {};
    p.P = dtype == ANAKIN_DTYPE_F32 ? 3 : dtype == ANAKIN_DTYPE_F16 ? 2 : 1;
    p.pair = K > 128 && N > 64;  // (a pair's second CTA has the second 128 rows of dW)
    p.BN = N <= 64 ? 64 : N <= 128 || (p.P > 1 && !p.pair) ? 128 : 256;
    p.direct = dtype == ANAKIN_DTYPE_BF16 && ((uintptr_t)dy & 15) == 0 && lddy % 8 == 0;
    p.pitch = (int)((N + 7) / 8 * 8);
    p.plane_bytes = ((size_t)R * p.pitch * 2 + 255) / 256 * 256;
    const int tk = p.pair ? 256 : 128, most = p.pair ? 74 : 148;
    p.tiles_m = (int)((K + tk - 1) / tk);
    const long long tiles = p.tiles_m * ((N + p.BN - 1) / p.BN);
    p.tiles = (int)tiles;  // (at most 2^15 times 2^16)
    p.chunks = (int)((R + 63) / 64);
    p.total = tiles * p.chunks;
    // Either every tile gets the same number of runs: then all tiles' runs of the same rows are at work at one time and what they read comes from L2.
    // Or runs of the same length go on from tile to tile and every SM is busy; then, where codes and dY are more than L2 holds, each tile reads its
    // own from memory.  A run has four chunks at least; a chunk takes some 0.47 us (one term; 0.3 a term with more), a MB of partial sums written
    // and read 0.5 us, a kernel or another wave of runs 2.
    p.width = partial_width(N);
    if (p.chunks == 0) return p;
    const double us = p.P == 1 ? 0.47 : 0.3 * p.P, part_us = 2e-6 * (double)K * (double)N;
    const double tiles_n = (double)((N + p.BN - 1) / p.BN), code_mb = 1e-6 * R * K, dy_mb = 2e-6 * R * N * p.P;
    const long long most_each = std::max(1ll, std::min((p.chunks + 3ll) / 4, 3ll * most / tiles));
    long long even = p.chunks;
    double t_even = 1e30;
    for (long long e = 1; e <= most_each; ++e) {
        const long long len = (p.chunks + e - 1) / e, waves = (tiles * ((p.chunks + len - 1) / len) + most - 1) / most;
        const double w = (double)waves * (us * (double)len + 2.0) + (e > 1 ? 2.0 + part_us * (double)(e + 1) : 0.0);
        if (w < t_even) {
            t_even = w;
            even = len;
        }
    }
    const long long each = (p.chunks + even - 1) / even;
    long long flow = (p.total + most - 1) / most;
    if (flow < 4) flow = 4;
    const double read = (code_mb + dy_mb > 100.0 ? code_mb * tiles_n + dy_mb * p.tiles_m : code_mb + dy_mb) / 5.5;
    const double t_flow = std::max(us * (double)flow, read) + 4.0 + part_us * 3.0;
    if (t_even <= t_flow || p.total >= (1ll << 31)) {  // (k_wgrad_sum counts the chunks of flowing runs in 32 bits)
        p.per_tile = (int)each;
        p.run = even;
        p.parts = p.per_tile;
        p.runs = tiles * each < (1ll << 30) && p.total < (1ll << 40) ? (int)(tiles * each) : 0;
    } else {
        p.run = flow;
        p.parts = (int)((p.chunks + p.run - 2) / p.run) + 1;
        p.runs = (int)((p.total + p.run - 1) / p.run);
    }
    p.part_off = p.direct ? 0 : (size_t)p.P * p.plane_bytes;
    p.straight = p.parts == 1;
    p.bytes = p.part_off + (p.straight ? 0 : (size_t)p.parts * K * p.width * 4);
    return p;
}

// Tensor maps of matrices whose rows lie pitch_bytes apart (a multiple of 16): bf16 in 64 x 64 boxes with the 128-byte swizzle, or bytes in boxes of
// 128 columns x 64 rows.  Columns from `cols` on read as zeros, whatever lies there.
bool encode_map(CUtensorMap* map, bool bytes, const void* base, uint64_t rows, uint64_t cols, uint64_t pitch_bytes) {
    using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = []() -> Encode {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess) return nullptr;
        return reinterpret_cast<Encode>(p);
    }();
    const cuuint64_t dims[2] = {cols, rows}, strides[1] = {pitch_bytes};
    const cuuint32_t box[2] = {bytes ? 128u : 64u, 64}, steps[2] = {1, 1};
    return encode && encode(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims, strides, box, steps,
                            CU_TENSOR_MAP_INTERLEAVE_NONE, bytes ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
                            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int BN, int P, bool PAIR>
cudaError_t launch_wgrad(const Maps& maps, const Args& a, const Plan& p, cudaStream_t s) {
    return launch_cluster<k_ckpt_wgrad<BN, P, PAIR>>(dim3(p.runs * (PAIR ? 2 : 1)), dim3(Cfg<BN, P, PAIR>::THREADS), Cfg<BN, P, PAIR>::SMEM, s, PAIR ? 2 : 1, maps, a);
}
template <int P>
cudaError_t launch_wgrad_p(const Maps& maps, const Args& a, const Plan& p, cudaStream_t s) {
    if (p.pair) return p.BN == 128 ? launch_wgrad<128, P, true>(maps, a, p, s) : launch_wgrad<256, P, true>(maps, a, p, s);
    if constexpr (P == 1) {
        if (p.BN == 256) return launch_wgrad<256, P, false>(maps, a, p, s);
    }
    return p.BN == 64 ? launch_wgrad<64, P, false>(maps, a, p, s) : launch_wgrad<128, P, false>(maps, a, p, s);
}

template <class T, int P>
cudaError_t launch_split(const void* dy, long long ld, int R, int N, int pitch, void* ws, size_t plane_bytes, cudaStream_t s) {
    const bool vec = ((uintptr_t)dy & 15) == 0 && ld * sizeof(T) % 16 == 0;
    const int per_row = pitch / 8;
    const long long most = ((1ll << 31) - 1) / per_row;  // rows of a launch: fewer than 2^31 pieces
    for (long long r0 = 0; r0 < R; r0 += most) {
        const uint32_t pieces = (uint32_t)(std::min(most, R - r0) * per_row), ctas = (pieces + 255) / 256;
        const T* from = static_cast<const T*>(dy) + r0 * ld;
        __nv_bfloat16* planes = static_cast<__nv_bfloat16*>(ws) + r0 * pitch;
        const dim3 grid(std::min(ctas, 148u * 32));
        const cudaError_t e = vec ? launch<k_split_planes<T, P, true>>(grid, dim3(256), 0, s, from, ld, FastDiv((uint32_t)per_row), pieces, N, pitch, planes, (long long)(plane_bytes / 2))
                                  : launch<k_split_planes<T, P, false>>(grid, dim3(256), 0, s, from, ld, FastDiv((uint32_t)per_row), pieces, N, pitch, planes, (long long)(plane_bytes / 2));
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

int check_sizes(int dtype, int64_t rows, int64_t cols, int64_t n) {
    if (dtype < ANAKIN_DTYPE_F32 || dtype > ANAKIN_DTYPE_F16 || rows < 0 || rows >= (int64_t(1) << 31) - 64 || cols < 1 || n < 1) return ANAKIN_E_INVALID_ARG;
    if (cols > (int64_t(1) << 22) || n > (int64_t(1) << 22)) return ANAKIN_E_INVALID_ARG;  // (tiles of n: a grid's second dimension)
    return ANAKIN_OK;
}

}  // namespace
}  // namespace ckpt
}  // namespace anakin

using namespace anakin;
using namespace anakin::ckpt;

extern "C" {

int anakin_ckpt_weight_grad_workspace_bytes(int dtype, int64_t rows, int64_t cols, int64_t n, int dy_aligned, size_t* bytes) {
    if (!bytes) return ANAKIN_E_INVALID_ARG;
    const int rc = check_sizes(dtype, rows, cols, n);
    if (rc != ANAKIN_OK) return rc;
    const int splits = rows > 0 ? few_splits(rows, cols, n) : 0;
    *bytes = splits > 0 ? 256 + (splits > 1 ? sizeof(float) * splits * (size_t)cols * partial_width(n) : 0) : make_plan(dtype, rows, cols, n, reinterpret_cast<const void*>((uintptr_t)(dy_aligned ? 16 : 1)), 8).bytes + 256;
    return ANAKIN_OK;
}

int anakin_ckpt_weight_grad(int dtype, int act, int64_t rows, int64_t cols, int64_t n, const uint8_t* codes, const uint8_t* scales,
                            const void* dy, int64_t lddy, float* dw, int64_t lddw, int accumulate, void* dev_workspace, size_t bytes,
                            int32_t* dev_status, void* cuda_stream) {
    int rc = check_sizes(dtype, rows, cols, n);
    if (rc == ANAKIN_OK) rc = ckpt::check(dtype, act, rows, cols, codes, scales);
    if (rc != ANAKIN_OK) return rc;
    const int es = dtype == ANAKIN_DTYPE_F32 ? 4 : 2;
    if (!dw || ((uintptr_t)dw & 3) || lddw < n || (rows > 0 && (!dy || lddy < n || ((uintptr_t)dy & (es - 1))))) return ANAKIN_E_INVALID_ARG;
    if (lddy >= (int64_t(1) << 31) || lddw >= (int64_t(1) << 40)) return ANAKIN_E_INVALID_ARG;
    if (act != ANAKIN_ACT_IDENTITY && act != ANAKIN_ACT_RELU) return ANAKIN_E_UNSUPPORTED_CFG;
    if (!dev_workspace || ((uintptr_t)dev_workspace & 255)) return ANAKIN_E_INVALID_ARG;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const int K = (int)cols, N = (int)n, R = (int)rows;
    if (const int splits = rows > 0 ? few_splits(rows, cols, n) : 0) {
        if ((cols + kFewK - 1) / kFewK * ((n + kFewN - 1) / kFewN) >= (int64_t(1) << 31)) return ANAKIN_E_UNSUPPORTED_CFG;
        const int relu = act == ANAKIN_ACT_RELU, width = partial_width(n), direct = splits == 1;
        const long long stride = (long long)cols * width;
        if (!direct && bytes < sizeof(float) * splits * (size_t)stride) return ANAKIN_E_WORKSPACE_TOO_SMALL;
        float* part = static_cast<float*>(dev_workspace);
        auto run = [&](auto type) {
            return launch_few<decltype(type)>(codes, scales, dy, lddy, splits, R, K, N, relu, direct ? dw : part, direct ? lddw : width, stride, direct && accumulate, s);
        };
        cudaError_t e = dtype == ANAKIN_DTYPE_F32 ? run(float{}) : dtype == ANAKIN_DTYPE_F16 ? run(__half{}) : run(__nv_bfloat16{});
        if (e == cudaSuccess && !direct) e = launch_sum(Parts{part, stride, FastDiv(1), splits, 1, 1, 0, 0, width}, splits, K, N, dw, lddw, accumulate, s);
        return e == cudaSuccess ? ANAKIN_OK : tok::fail();
    }
    const Plan p = make_plan(dtype, rows, cols, n, dy, lddy);
    if ((rows > 0 && p.runs < 1) || (long long)cols * (p.width / 32) >= (1ll << 31)) return ANAKIN_E_UNSUPPORTED_CFG;  // (months of work; dW of 275 GB)
    if (bytes < p.bytes) return ANAKIN_E_WORKSPACE_TOO_SMALL;
    float* part = reinterpret_cast<float*>(static_cast<unsigned char*>(dev_workspace) + p.part_off);
    if (rows > 0) {
        Maps maps;
        memset(&maps, 0, sizeof(maps));
        Args a = {};
        a.blocks = (K + 31) / 32;
        if (!encode_map(&maps.codes, true, codes, (uint64_t)R, (uint64_t)a.blocks * 32, (uint64_t)a.blocks * 32)) return tok::fail();
        if (!p.direct) {
            const cudaError_t e = dtype == ANAKIN_DTYPE_F32 ? launch_split<float, 3>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s)
                                  : dtype == ANAKIN_DTYPE_F16 ? launch_split<__half, 2>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s)
                                                              : launch_split<__nv_bfloat16, 1>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s);
            if (e != cudaSuccess) return tok::fail();
        }
        for (int i = 0; i < p.P; ++i) {
            const void* b = p.direct ? dy : static_cast<const unsigned char*>(dev_workspace) + i * p.plane_bytes;
            if (!encode_map(&maps.b[i], false, b, (uint64_t)R, (uint64_t)N, (uint64_t)(p.direct ? lddy : p.pitch) * 2)) return tok::fail();
        }
        a.R = R;
        a.K = K;
        a.N = N;
        a.tiles_m = p.tiles_m;
        a.chunks = p.chunks;
        a.run = p.run;
        a.total = p.total;
        a.per_tile = p.per_tile;
        a.tiles = p.tiles;
        a.scales = scales;
        a.out = p.straight ? dw : part;
        a.ld = p.straight ? lddw : p.width;
        a.part_stride = (long long)K * p.width;
        a.add = p.straight && accumulate;
        a.relu = act == ANAKIN_ACT_RELU;
        a.status = dev_status;
        const cudaError_t e = p.P == 1 ? launch_wgrad_p<1>(maps, a, p, s) : p.P == 2 ? launch_wgrad_p<2>(maps, a, p, s) : launch_wgrad_p<3>(maps, a, p, s);
        if (e != cudaSuccess) return tok::fail();
    }
    if (!p.straight) {
        const Parts parts = {part, (long long)K * p.width, FastDiv((uint32_t)std::max(1ll, p.run)), p.per_tile, p.chunks, p.tiles_m, p.pair ? 8 : 7,
                             p.BN == 256 ? 8 : p.BN == 128 ? 7 : 6, p.width};
        const cudaError_t e = launch_sum(parts, p.parts, K, N, dw, (long long)lddw, accumulate, s);
        if (e != cudaSuccess) return tok::fail();
    }
    return ANAKIN_OK;
}

}  // extern "C"
