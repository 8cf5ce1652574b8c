// What the kernels over token rows share: element types, the bookkeeping of rows (which of them count, which sequence they belong to) and the
// per-token terms of the clipped policy loss.
#pragma once
#include <cuda_fp16.h>

#include "common.cuh"

namespace anakin {
namespace tok {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 16-bit and 32-bit elements as floats and back (to nearest, ties to even).
template <class T> __device__ __forceinline__ float to_f(T v);
template <> __device__ __forceinline__ float to_f<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_f<__half>(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of elements as floats, and back.
template <class T> struct Vec { static constexpr int N = 16 / sizeof(T); };
__device__ __forceinline__ void unpack16(const uint4& u, float (&f)[4], const float*) {
    f[0] = __uint_as_float(u.x); f[1] = __uint_as_float(u.y); f[2] = __uint_as_float(u.z); f[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ void unpack16(const uint4& u, float (&f)[8], const __nv_bfloat16*) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u); }
}
__device__ __forceinline__ void unpack16(const uint4& u, float (&f)[8], const __half*) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 p = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
        f[2 * i] = p.x; f[2 * i + 1] = p.y;
    }
}
__device__ __forceinline__ uint4 pack16(const float (&f)[4], const float*) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
__device__ __forceinline__ uint4 pack16(const float (&f)[8], const __nv_bfloat16*) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack16(const float (&f)[8], const __half*) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 p = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&p);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// 2^x to about 2^-22 of itself; 2^-inf = 0, NaN stays.
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// An integer of 4 or 8 bytes.
__device__ __forceinline__ long long load_int(const void* p, size_t i, int bytes) {
    return bytes == 8 ? static_cast<const long long*>(p)[i] : (long long)static_cast<const int*>(p)[i];
}

// The rows of a call, as the kernels see them.
struct Rows {
    long long rows, vocab, ld;
    const void* logits;
    const void* tokens;
    const uint8_t* mask;
    const void* offsets;
    int sequences, token_bytes, offset_bytes;
    float scale;
};

// The sequence of row r: the last i with offsets[i] <= r; -1 before the first and `sequences` behind the last.  Any offsets give a
// number in that range.  `near`: the offsets as 32-bit numbers in shared memory.
__device__ __forceinline__ int sequence_of(const Rows& q, long long r, const int* near) {
    if (!q.offsets) return 0;
    int lo = 0, hi = q.sequences + 1;  // the number of offsets <= r lies in [lo, hi]
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (near[mid] <= r) lo = mid + 1;
        else hi = mid;
    }
    return lo - 1;
}
// Counted as far as its token and the mask say.
__device__ __forceinline__ bool row_counts(const Rows& q, long long r) {
    if (q.mask && !q.mask[r]) return false;
    return !q.tokens || load_int(q.tokens, r, q.token_bytes) >= 0;
}

// ---- the clipped policy loss of one token ----
struct Objective {
    float lo, hi, dual, kl_coef, entropy_coef, inv_divisor;
    int kl, mean;
};
struct PolicyTerms { float pg, kl, cut, old_minus_new, dlogp; };  // dlogp without the row's weight

// fmin and fmax would drop a NaN.
__device__ __forceinline__ float bounded(float d) { return d > 80.f ? 80.f : d < -80.f ? -80.f : d; }

__device__ __forceinline__ PolicyTerms policy_terms(const Objective& o, float l, float old, bool has_old, float A, float ref) {
    PolicyTerms t;
    const float d = has_old ? bounded(l - old) : 0.f;
    const float r = expf(d);
    const float rA = r * A, cA = (r < o.lo ? o.lo : r > o.hi ? o.hi : r) * A;
    bool cut = cA < rA;
    float pg = cut ? -cA : -rA;
    if (o.dual > 0.f && A < 0.f && pg > -o.dual * A) { pg = -o.dual * A; cut = true; }
    t.pg = pg;
    t.cut = cut ? 1.f : 0.f;
    t.dlogp = cut ? 0.f : -rA;
    t.old_minus_new = has_old ? old - l : 0.f;
    t.kl = 0.f;
    if (o.kl != ANAKIN_KL_NONE) {
        const float z = l - ref;
        if (o.kl == ANAKIN_KL_1) { t.kl = z; t.dlogp += o.kl_coef; }
        else if (o.kl == ANAKIN_KL_2) { t.kl = 0.5f * z * z; t.dlogp += o.kl_coef * z; }
        else {
            const float y = bounded(z), e = expm1f(-y);
            // exp(-y) - 1 + y loses y itself where y is small: there its series, whose next term is below 2^-24 of the sum
            t.kl = fabsf(y) < 0.25f ? y * y * (0.5f + y * (-1.f / 6 + y * (1.f / 24 + y * (-1.f / 120 + y * (1.f / 720 + y * (-1.f / 5040 + y * (1.f / 40320)))))))
                                    : e + y;
            t.dlogp -= o.kl_coef * e;
        }
    }
    return t;
}

// Counted rows in all and, for the mean over sequences, the sequences that have one; counts of each sequence follow in the workspace.
struct Counts {
    unsigned long long rows, sequences;
};
__device__ __forceinline__ float row_weight(const Objective& o, const Counts* c, const int* per_seq, int seq) {
    if (o.mean == ANAKIN_MEAN_FIXED) return o.inv_divisor;
    if (o.mean == ANAKIN_MEAN_TOKEN) return 1.f / (float)c->rows;
    return 1.f / ((float)per_seq[seq] * (float)c->sequences);
}

// Sums of v[0 .. N-1] over the block's threads in a fixed order, in the threads of the first warp; `red` holds N doubles for each warp.
template <int N> __device__ __forceinline__ void block_sums(double (&v)[N], double* red) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < N; ++k) red[(threadIdx.x >> 5) * N + k] = v[k];
    }
    __syncthreads();
    if (threadIdx.x < 32) {
        const int warps = (int)(blockDim.x >> 5);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (int)threadIdx.x < warps ? red[threadIdx.x * N + k] : 0.0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += __shfl_xor_sync(0xFFFFFFFFu, v[k], o);
    }
}

// Rows of partial statistics, one for each CTA of a kernel, summed in order by one CTA (see token_loss.cu).
cudaError_t launch_policy_stats(const double* part, int n, const Objective& o, float* stats, cudaStream_t s);

constexpr int kPolicyParts = 5;         // sums a CTA leaves: pg, kl, H, cut, old - l
constexpr int kMaxPartials = 148 * 16;  // CTAs that may leave some

// Layout of the workspace of the losses.
struct Workspace {
    Counts* counts;
    int* per_seq;   // [sequences] (of the preference loss: times its splits), right behind the counts
    double* part;   // [kMaxPartials][kPolicyParts]
    double* sums;   // [sequences times splits] of the preference loss
    float* coef;    // [sequences] of the preference loss
    int2* info;     // [rows] of the policy gradient: the row's sequence (-1: no part in the loss, -2: does not count at all) and its token
    size_t bytes;
};
Workspace carve(void* base, long long rows, long long sequences);

// What the means divide by (ANAKIN_MEAN_*) and, with rows_too, every row's sequence and token, into the workspace.
cudaError_t launch_counts(const Rows& q, int mean, bool rows_too, const Workspace& w, cudaStream_t s);

// Host: checks of what every call has in common; fills q.
int check_rows(const anakin_token_rows* rows, bool need_logits, bool need_tokens, bool need_offsets, Rows* q);
int check_policy(const anakin_policy_objective* p, Objective* o);
int fail();  // clears the CUDA error that the call is about to report

}  // namespace tok
}  // namespace anakin
