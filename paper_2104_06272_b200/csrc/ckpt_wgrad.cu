// Weight gradient of a layer from its input's 8-bit checkpoint:  dW[k][n] (+)= sum_r f(x[r][k]) dY[r][n],  f = identity or ReLU, on the
// 5th-generation tensor cores.
//
// A kept value is an e4m3 number times a power of two: exact in bf16.  dY is one bf16 term, or two (fp16) or three (fp32) that sum to it, in planes
// that a first kernel writes.  So every product is exact in the MMA and the sums are the only rounding.  Both operands have the contraction index r
// as their slow index ("MN-major").
//
// One CTA owns a 128 x BN tile of dW and a range of rows, in chunks of 64 rows:
//   warp 0       TMA: the 64 x 128 codes and the 64 x BN planes of dY (64 x 64 boxes, 128-byte swizzle) into a ring of stages
//   warps 4-7    codes -> bf16 in the swizzled layout (a thread turns 8 codes of a row into 16 bytes; block scales are fetched a chunk ahead)
//   warp 1       tcgen05.mma into one of two accumulators in tensor memory; commits free the stage
//   warps 8-15   add a finished accumulator to sums in registers; at the end store the tile, or the partial tile of a split
// The tensor core's fp32 accumulation rounds toward zero, which biases long sums (about 5e-8 of the sum an MMA): an accumulator takes at most 32
// MMAs (512 rows of one bf16 term) and the groups are added with round-to-nearest.
#include <cstring>

#include "ckpt.cuh"
#include "tc_common.cuh"
#include "token_rows.cuh"

namespace anakin {
namespace ckpt {
namespace {

template <int BN_, int P_>
struct Cfg {
    static constexpr int BN = BN_, P = P_, BM = 128, KC = 64;
    static constexpr int BOX = 64 * 64 * 2;
    static constexpr int A_BYTES = (BM / 64) * BOX, B_PLANE = (BN / 64) * BOX, CODES = KC * BM;
    static constexpr int STAGE = A_BYTES + P * B_PLANE + CODES;
    static constexpr int FIT = (232448 - 1024 - 256) / STAGE;
    static constexpr int STAGES = FIT >= 4 ? 4 : FIT;
    static constexpr int GROUP = P == 1 ? 8 : P == 2 ? 4 : 2;  // chunks an accumulator takes: 32, 32 and 24 MMAs
    static constexpr size_t SMEM = (size_t)STAGES * STAGE + 1024 + 256;
};

struct Maps {
    CUtensorMap codes, b[3];
};
struct Args {
    int R, K, N, blocks;
    int chunks_per_split;
    const uint8_t* scales;
    float* out;  // dW, or the partial tiles [split][K][N]
    long long ld, split_stride;
    int relu, add;
    bool vec;  // rows of `out` start on 16-byte boundaries
    int32_t* status;
};

template <int BN, int P>
__global__ void __launch_bounds__(512, 1) k_ckpt_wgrad(const __grid_constant__ Maps maps, Args a) {
    using C = Cfg<BN, P>;
    constexpr int STAGES = C::STAGES, GROUP = C::GROUP;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* base = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* raw = (uint64_t*)(base + STAGES * C::STAGE);  // TMA done
    uint64_t* full = raw + STAGES;                          // operand A written
    uint64_t* empty = full + STAGES;
    uint64_t* accfull = empty + STAGES;
    uint64_t* accempty = accfull + 2;
    uint32_t* tmem_slot = (uint32_t*)(accempty + 2);
    const int tid = threadIdx.x, wid = tid >> 5, lane = tid & 31;
    const int m0 = blockIdx.x * C::BM, n0 = blockIdx.y * BN;
    const int total = (a.R + C::KC - 1) / C::KC;
    const int c0 = min((int)blockIdx.z * a.chunks_per_split, total), nchunks = min(a.chunks_per_split, total - c0);
    const int ngroups = (nchunks + GROUP - 1) / GROUP;

    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) { tc::mbar_init(&raw[s], 1); tc::mbar_init(&full[s], 128); tc::mbar_init(&empty[s], 1); }
        for (int q = 0; q < 2; ++q) { tc::mbar_init(&accfull[q], 1); tc::mbar_init(&accempty[q], 256); }
        tc::mbar_fence_init();
        tc::prefetch_map(&maps.codes);
        tc::prefetch_map(&maps.b[0]);
    }
    if (wid == 2) tc::tmem_alloc(tmem_slot, 2 * BN);
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();
    bool ok = true;

    if (wid < 4) {
        tc::regs_dec<48>();
        if (wid == 0 && lane == 0) {
            for (int c = 0; c < nchunks; ++c) {
                const int s = c % STAGES, r0 = (c0 + c) * C::KC;
                if (c >= STAGES) ok = tc::mbar_wait(&empty[s], ((c / STAGES) - 1) & 1);
                if (!ok) break;
                unsigned char* st = base + s * C::STAGE;
                tc::mbar_expect_tx(&raw[s], P * C::B_PLANE + C::CODES);
                tc::tma_load_2d(st + C::A_BYTES + P * C::B_PLANE, &maps.codes, &raw[s], m0, r0);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int bx = 0; bx < BN / 64; ++bx)
                        tc::tma_load_2d(st + C::A_BYTES + p * C::B_PLANE + bx * C::BOX, &maps.b[p], &raw[s], n0 + 64 * bx, r0);
            }
            if (!ok && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
        } else if (wid == 1) {
            const uint32_t idesc = tc::umma_idesc<1>(C::BM, BN, true, true);
            for (int c = 0; c < nchunks; ++c) {
                const int s = c % STAGES, grp = c / GROUP, cg = c - grp * GROUP;
                const uint32_t acc = tmem + (uint32_t)((grp & 1) * BN);
                if (cg == 0 && grp >= 2) ok = tc::mbar_wait(&accempty[grp & 1], ((grp >> 1) - 1) & 1);
                ok = tc::warp_all(ok && tc::mbar_wait(&raw[s], (c / STAGES) & 1) && tc::mbar_wait(&full[s], (c / STAGES) & 1));
                if (!ok) break;
                tc::tc_fence_after();
                unsigned char* sa = base + s * C::STAGE;
                unsigned char* sb = sa + C::A_BYTES;
                if (tc::elect_one()) {
#pragma unroll
                    for (int p = P - 1; p >= 0; --p)  // (the small terms first)
#pragma unroll
                        for (int k16 = 0; k16 < C::KC / 16; ++k16)
                            tc::umma(acc, tc::umma_desc(sa + k16 * 2048, C::BOX, 1024), tc::umma_desc(sb + p * C::B_PLANE + k16 * 2048, C::BOX, 1024), idesc,
                                     (cg > 0 || k16 > 0 || p < P - 1) ? 1u : 0u);
                    tc::umma_commit(&empty[s]);
                    if (cg == GROUP - 1 || c == nchunks - 1) tc::umma_commit(&accfull[grp & 1]);
                }
                __syncwarp();
            }
            if (!ok && lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
        }
    } else if (wid < 8) {
        tc::regs_dec<96>();
        const int t = tid - 128, ch = t & 15, rr = t >> 4;  // 8 columns from 8 ch on, of rows rr, rr + 8, ...
        const int blk = (m0 >> 5) + (ch >> 2);
        const bool col = blk < a.blocks;
        const uint32_t dst0 = (uint32_t)((ch >> 3) * C::BOX + rr * 128 + (((ch & 7) ^ (rr & 7)) << 4));  // (rr + 8 i) & 7 = rr & 7
        uint32_t sc[8];
        auto fetch = [&](int c) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int r = (c0 + c) * C::KC + rr + 8 * i;
                sc[i] = col && c < nchunks && r < a.R ? (uint32_t)a.scales[(size_t)r * a.blocks + blk] : 0u;
            }
        };
        fetch(0);
        for (int c = 0; c < nchunks; ++c) {
            const int s = c % STAGES;
            // (a stage's last MMAs have finished before its codes were asked for: operand A may be written again)
            ok = tc::mbar_wait(&raw[s], (c / STAGES) & 1);
            if (!ok) break;
            unsigned char* st = base + s * C::STAGE;
            const unsigned char* src = st + C::A_BYTES + P * C::B_PLANE + rr * 128 + ch * 8;
            uint32_t now[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) now[i] = sc[i];
            fetch(c + 1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float v[8];
                decode8(*reinterpret_cast<const uint2*>(src + i * 1024), now[i], v);
                if (a.relu) {
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = v[k] < 0.f ? 0.f : v[k];
                }
                *reinterpret_cast<uint4*>(st + dst0 + i * 1024) = tok::pack16(v, (const __nv_bfloat16*)nullptr);
            }
            tc::fence_proxy_async();
            tc::mbar_arrive(&full[s]);
        }
        if (!ok && lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
    } else {
        tc::regs_inc<184>();
        constexpr int COLS = BN / 2;
        const int q = wid & 3, half = (wid - 8) >> 2;
        float sum[COLS];
#pragma unroll
        for (int j = 0; j < COLS; ++j) sum[j] = 0.f;
        for (int grp = 0; grp < ngroups; ++grp) {
            ok = tc::warp_all(tc::mbar_wait(&accfull[grp & 1], (grp >> 1) & 1));
            if (!ok) break;
            tc::tc_fence_after();
            const uint32_t acc = tmem + (uint32_t)((grp & 1) * BN + half * COLS) + ((uint32_t)(32 * q) << 16);
#pragma unroll
            for (int j0 = 0; j0 < COLS; j0 += 32) {
                uint32_t r[32];
                tc::tmem_ld32(acc + (uint32_t)j0, r);
#pragma unroll
                for (int j = 0; j < 32; ++j) sum[j0 + j] += __uint_as_float(r[j]);
            }
            tc::tc_fence_before();
            if (grp + 2 < ngroups) tc::mbar_arrive(&accempty[grp & 1]);
        }
        if (!ok) {  // the caller sees it in the result, too
            if (lane == 0 && a.status) atomicOr(a.status, DEV_E_WAIT_TIMEOUT);
#pragma unroll
            for (int j = 0; j < COLS; ++j) sum[j] = NAN;
        }
        const int m = m0 + 32 * q + lane, nb = n0 + half * COLS;
        if (m < a.K) {
            float* dst = a.out + (size_t)blockIdx.z * a.split_stride + (size_t)m * a.ld + nb;
#pragma unroll
            for (int j = 0; j < COLS; j += 4) {
                if (a.vec && nb + j + 4 <= a.N) {
                    float4 v = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
                    float4* p = reinterpret_cast<float4*>(dst + j);
                    if (a.add) { const float4 o = *p; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
                    *p = v;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (nb + j + i < a.N) dst[j + i] = a.add ? dst[j + i] + sum[j + i] : sum[j + i];
                }
            }
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (wid == 2) tc::tmem_dealloc(tmem, 2 * BN);
}

// Partial tiles summed in the order of the splits.
__global__ void __launch_bounds__(256) k_wgrad_sum(const float* part, int splits, long long stride, int K, int N, float* dw, long long ld, int add) {
    pdl_wait();
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)K * N; i += (long long)gridDim.x * 256) {
        const long long k = i / N, n = i - k * N;
        float v = 0.f;
        for (int s = 0; s < splits; ++s) v += part[(size_t)s * stride + i];
        float* p = dw + k * ld + n;
        *p = add ? *p + v : v;
    }
}

// dY as P bf16 planes [rows][pitch] that sum to it (fp32: 24 bits in three; fp16: 11 bits in two; bf16 whose rows TMA cannot address: one).
template <class T, int P>
__global__ void __launch_bounds__(256) k_split_planes(const T* dy, long long ld, int R, int N, int pitch, __nv_bfloat16* planes, long long plane) {
    pdl_wait();
    const int per_row = pitch / 8;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < (long long)R * per_row; i += (long long)gridDim.x * 256) {
        const long long r = i / per_row;
        const int j = (int)(i - r * per_row) * 8;
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = j + k < N ? tok::to_f(dy[r * ld + j + k]) : 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) h[k] = __bfloat162float(__float2bfloat16_rz(v[k]));  // (cut, not rounded: never past bf16's largest, and 8 bits a term are all 24)
            *reinterpret_cast<uint4*>(planes + p * plane + r * pitch + j) = tok::pack16(h, (const __nv_bfloat16*)nullptr);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = fabsf(h[k]) < INFINITY ? v[k] - h[k] : 0.f;  // (an infinity stays one: its rest would be NaN)
        }
    }
}

struct Plan {
    int P, BN, pitch, splits, chunks_per_split;
    bool direct;  // TMA reads the caller's dY
    size_t plane_bytes, part_off, bytes;
};

Plan make_plan(int dtype, long long R, long long K, long long N, const void* dy, long long lddy) {
    Plan p;
    p.P = dtype == ANAKIN_DTYPE_F32 ? 3 : dtype == ANAKIN_DTYPE_F16 ? 2 : 1;
    p.BN = N <= 64 ? 64 : N <= 128 || p.P > 1 ? 128 : 256;
    p.direct = dtype == ANAKIN_DTYPE_BF16 && ((uintptr_t)dy & 15) == 0 && lddy % 8 == 0;
    p.pitch = (int)((N + 7) / 8 * 8);
    p.plane_bytes = ((size_t)R * p.pitch * 2 + 255) / 256 * 256;
    const long long tiles = (K + 127) / 128 * ((N + p.BN - 1) / p.BN), chunks = (R + 63) / 64;
    // as many splits as one wave holds, of at least four chunks each
    long long splits = tiles < 148 ? 148 / tiles : 1;
    if (splits > (chunks + 3) / 4) splits = (chunks + 3) / 4;
    if (splits < 1) splits = 1;
    p.chunks_per_split = (int)((chunks + splits - 1) / splits);
    if (p.chunks_per_split < 1) p.chunks_per_split = 1;
    p.splits = (int)((chunks + p.chunks_per_split - 1) / p.chunks_per_split);
    p.part_off = p.direct ? 0 : (size_t)p.P * p.plane_bytes;
    p.bytes = p.part_off + (p.splits > 1 ? (size_t)p.splits * K * N * 4 : 0);
    return p;
}

template <int BN, int P>
cudaError_t launch_wgrad(const Maps& maps, const Args& a, const Plan& p, cudaStream_t s) {
    const dim3 grid((a.K + 127) / 128, (a.N + BN - 1) / BN, p.splits);
    return launch<k_ckpt_wgrad<BN, P>>(grid, dim3(512), Cfg<BN, P>::SMEM, s, maps, a);
}

template <class T, int P>
cudaError_t launch_split(const void* dy, long long ld, int R, int N, int pitch, void* ws, size_t plane_bytes, cudaStream_t s) {
    const long long n = ((long long)R * (pitch / 8) + 255) / 256;
    return launch<k_split_planes<T, P>>(dim3((unsigned)(n < 148 * 32 ? n : 148 * 32)), dim3(256), 0, s, static_cast<const T*>(dy), ld, R, N, pitch,
                                        static_cast<__nv_bfloat16*>(ws), (long long)(plane_bytes / 2));
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

int anakin_ckpt_weight_grad_workspace_bytes(int dtype, int64_t rows, int64_t cols, int64_t n, size_t* bytes) {
    if (!bytes) return ANAKIN_E_INVALID_ARG;
    const int rc = check_sizes(dtype, rows, cols, n);
    if (rc != ANAKIN_OK) return rc;
    *bytes = make_plan(dtype, rows, cols, n, (const void*)1, 1).bytes + 256;  // (for any address and stride of dy)
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
    const Plan p = make_plan(dtype, rows, cols, n, dy, lddy);
    if (bytes < p.bytes) return ANAKIN_E_WORKSPACE_TOO_SMALL;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    const int K = (int)cols, N = (int)n, R = (int)rows;
    float* part = reinterpret_cast<float*>(static_cast<unsigned char*>(dev_workspace) + p.part_off);
    const bool split = p.splits > 1 || rows == 0;
    if (rows > 0) {
        Maps maps;
        memset(&maps, 0, sizeof(maps));
        Args a = {};
        a.blocks = (K + 31) / 32;
        if (!make_tensor_map_u8(&maps.codes, codes, (uint64_t)R, (uint64_t)a.blocks * 32, 64, 128)) return tok::fail();
        if (!p.direct) {
            const cudaError_t e = dtype == ANAKIN_DTYPE_F32 ? launch_split<float, 3>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s)
                                  : dtype == ANAKIN_DTYPE_F16 ? launch_split<__half, 2>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s)
                                                              : launch_split<__nv_bfloat16, 1>(dy, lddy, R, N, p.pitch, dev_workspace, p.plane_bytes, s);
            if (e != cudaSuccess) return tok::fail();
        }
        for (int i = 0; i < p.P; ++i) {
            const void* b = p.direct ? dy : static_cast<const unsigned char*>(dev_workspace) + i * p.plane_bytes;
            if (!make_tensor_map_pitched(&maps.b[i], b, (uint64_t)R, (uint64_t)N, (uint64_t)(p.direct ? lddy : p.pitch) * 2, 64, true)) return tok::fail();
        }
        a.R = R;
        a.K = K;
        a.N = N;
        a.chunks_per_split = p.chunks_per_split;
        a.scales = scales;
        a.out = split ? part : dw;
        a.ld = split ? N : lddw;
        a.split_stride = split ? (long long)K * N : 0;
        a.relu = act == ANAKIN_ACT_RELU;
        a.add = !split && accumulate;
        a.vec = ((uintptr_t)a.out & 15) == 0 && a.ld % 4 == 0 && (!split || a.split_stride % 4 == 0);
        a.status = dev_status;
        cudaError_t e;
        if (p.P == 1) e = p.BN == 64 ? launch_wgrad<64, 1>(maps, a, p, s) : p.BN == 128 ? launch_wgrad<128, 1>(maps, a, p, s) : launch_wgrad<256, 1>(maps, a, p, s);
        else if (p.P == 2) e = p.BN == 64 ? launch_wgrad<64, 2>(maps, a, p, s) : launch_wgrad<128, 2>(maps, a, p, s);
        else e = p.BN == 64 ? launch_wgrad<64, 3>(maps, a, p, s) : launch_wgrad<128, 3>(maps, a, p, s);
        if (e != cudaSuccess) return tok::fail();
    }
    if (split) {
        const long long ctas = ((long long)K * N + 255) / 256;
        if (launch<k_wgrad_sum>(dim3((unsigned)(ctas < 148 * 32 ? ctas : 148 * 32)), dim3(256), 0, s, (const float*)part, rows == 0 ? 0 : p.splits, (long long)K * N, K, N,
                                dw, (long long)lddw, accumulate) != cudaSuccess)
            return tok::fail();
    }
    return ANAKIN_OK;
}

}  // extern "C"
