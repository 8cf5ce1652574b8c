// Softmax rows over a token vocabulary: log-probability and entropy of the taken token, the gradient of the logits, and both around the
// clipped policy loss in one kernel.
//
// With x the logits of a row, c = scale log2(e), m = max x, M = c m rounded, d_j = c x_j - M (one fused multiply-add):
//   s = sum 2^d,  t = sum 2^d d   in one pass, rescaled whenever m grows;   log p_j = ln2 d_j - ln s;   H = ln s - ln2 t / s
//   dx_j = scale ( g ([j = token] - p_j) - h p_j (log p_j + H) ) = 2^d_j ( a + b d_j ) + [j = token] scale g
// M's rounding is the same in every term and cancels while it is small: up to |M| = 2^22 it is 1/8 at most, and the largest term between 2^-1/8 and
// 2^1/8.  Beyond that (a part of a row where nothing but masks stands, a large scale) it would be an exponent of any size: there d_j = c (x_j - m).
// Terms that are -inf give 2^d = 0, and 0 times d is kept from being NaN by a lower bound on d, in those groups of logits only that hold such a
// term, or one far below the others.
//
// What bounds these kernels is memory or, in 16-bit types, the issue slots: an element costs an exponential and some 4 other instructions forward
// and 5 backward, with fused multiply-adds on two floats at a time and maxima on two 16-bit numbers at a time.
#include "tc_common.cuh"
#include "token_rows.cuh"

namespace anakin {
namespace tok {
namespace {

struct RowArgs {
    Rows q;
    float* logp;
    float* entropy;
    float* norm;  // [rows][2]: m, ln s
    // backward
    const float* norm_in;
    const float* entropy_in;
    const float* dlogp;
    const float* dentropy;
    void* dlogits;
    long long ld_out;
    // fused
    Objective o;
    const float* old_logp;
    const float* adv;
    const float* ref;
    const Counts* counts;
    const int* per_seq;
    const int2* info;  // [rows]: sequence and token (k_token_counts)
    double* part;
};

enum { FORWARD = 0, BACKWARD = 1, FUSED = 2 };

// Two floats in one instruction.
using F2 = float2;
__device__ __forceinline__ F2 f2(float x, float y) { return make_float2(x, y); }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { return __fadd2_rn(a, b); }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { return __fmul2_rn(a, b); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { return __ffma2_rn(a, b, c); }

// Largest and smallest of the elements of U 16-byte vectors (NaN is passed over).
template <class T, int U> __device__ __forceinline__ void extremes(const uint4 (&u)[U], float& top, float& low) {
    if constexpr (sizeof(T) == 4) {
        top = low = __uint_as_float(u[0].x);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float f[4];
            unpack16(u[i], f, (const float*)nullptr);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                top = fmaxf(top, f[k]);
                low = fminf(low, f[k]);
            }
        }
    } else {
        using P = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        auto as = [](const uint32_t& w) { return *reinterpret_cast<const P*>(&w); };
        P hi = as(u[0].x), lo = hi;
#pragma unroll
        for (int i = 0; i < U; ++i) {
            hi = __hmax2(__hmax2(__hmax2(hi, as(u[i].x)), __hmax2(as(u[i].y), as(u[i].z))), as(u[i].w));
            lo = __hmin2(__hmin2(__hmin2(lo, as(u[i].x)), __hmin2(as(u[i].y), as(u[i].z))), as(u[i].w));
        }
        top = fmaxf(to_f(hi.x), to_f(hi.y));
        low = fminf(to_f(lo.x), to_f(lo.y));
    }
}

// Exponents from -2^60 on may be multiplied by anything that a gradient has (scale is at most 2^40); where a group's smallest is below, all are bounded by
// -1000, whose exponential is 0, too.
__device__ __forceinline__ bool near(float low, float c) { return low * c > -1.1529215e18f; }
__device__ __forceinline__ F2 floored(F2 d) { return f2(fmaxf(d.x, -1000.f), fmaxf(d.y, -1000.f)); }  // (a NaN comes through its exponential)
// Terms are relative to M = c m rounded, not to m itself.
__device__ __forceinline__ bool usual(float M) { return fabsf(M) < 4194304.f; }

// The logarithm to base 2 of the factor from sums relative to m to sums relative to a larger maximum.
__device__ __forceinline__ float log_factor(float m, float to, float c) {
    const float M = __fmul_rn(m, c), T = __fmul_rn(to, c);
    if (usual(M)) return usual(T) ? M - T : -fmaf(to, c, -M);
    return usual(T) ? fmaf(m, c, -T) : (m - to) * c;
}

// Maximum, sum and weighted sum of a part of a row.
struct Soft {
    float m, s, t;
    __device__ __forceinline__ void rescale(float to, float c) {  // to >= m
        if (m < to) {
            if (s != 0.f) {  // (nothing but -inf so far: nothing to rescale)
                const float d = log_factor(m, to, c), f = ex2(d);
                t = f * (t + (f > 0.f ? s * d : 0.f));
                s *= f;
            }
            m = to;
        }
    }
};

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xFFFFFFFFu, v, o));
    return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
    return v;
}

// Of a group of L neighbouring lanes, in all of them: the maximum first, then sums on one scale.
template <int L> __device__ __forceinline__ void group_sum(Soft& v, float c) {
    float top = v.m;
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
    v.rescale(top, c);
    F2 st = f2(v.s, v.t);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) st = add2(st, f2(__shfl_xor_sync(0xFFFFFFFFu, st.x, o), __shfl_xor_sync(0xFFFFFFFFu, st.y, o)));
    v.s = st.x;
    v.t = st.y;
}

// The same for one thread, the sums two lanes each.
struct Acc {
    float m;
    F2 s, t;
    __device__ __forceinline__ void clear() {
        m = -INFINITY;
        s = t = f2(0.f, 0.f);
    }
    __device__ __forceinline__ Soft sums() const {
        return Soft{m, s.x + s.y, t.x + t.y};
    }
    template <bool BOUND> __device__ __forceinline__ void term(F2 d) {
        const F2 e = f2(ex2(d.x), ex2(d.y));
        s = add2(s, e);
        t = fma2(e, BOUND ? floored(d) : d, t);
    }
    template <int N> __device__ __forceinline__ void add(const float (&f)[N], float low, float c) {
        const float M = __fmul_rn(m, c);
        if (usual(M)) {
            const F2 cc = f2(c, c), off = f2(-M, -M);
            if (near(low, c)) {
#pragma unroll
                for (int k = 0; k < N; k += 2) term<false>(fma2(f2(f[k], f[k + 1]), cc, off));
            } else {
#pragma unroll
                for (int k = 0; k < N; k += 2) term<true>(fma2(f2(f[k], f[k + 1]), cc, off));
            }
        } else {
            const float at = m == -INFINITY ? 0.f : m;
            const F2 cc = f2(c, c), off = f2(-at, -at);
#pragma unroll
            for (int k = 0; k < N; k += 2) term<true>(mul2(add2(f2(f[k], f[k + 1]), off), cc));
        }
    }
    __device__ __forceinline__ void raise(float top, float c) {
        if (top > m) {
            Soft v = sums();
            v.rescale(top, c);
            m = top;
            s = f2(v.s, 0.f);
            t = f2(v.t, 0.f);
        }
    }
    template <class T, int U> __device__ __forceinline__ void add_vectors(const uint4 (&u)[U], float c) {
        float top, low;
        extremes<T>(u, top, low);
        raise(top, c);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            float f[Vec<T>::N];
            unpack16(u[i], f, (const T*)nullptr);
            add(f, low, c);
        }
    }
    template <int N> __device__ __forceinline__ void add_scalars(const float (&f)[N], float c) {
        float top = f[0], low = f[0];
#pragma unroll
        for (int k = 1; k < N; ++k) {
            top = fmaxf(top, f[k]);
            low = fminf(low, f[k]);
        }
        raise(top, c);
        add(f, low, c);
    }
};

// What the gradient of a row needs: 2^d ( a + b d ), d = c x - off or c (x - off), and `onehot` more at the token.
struct RowGrad {
    float off, a, b, onehot;
    int token, kind;  // kind: 0 usual, 1 = from differences (M beyond 2^22, or a short row), 2 = zeros, 3 = NaN
    __device__ __forceinline__ void set(float m, float ln_s, float g, float h, float H, float scale, float c, long long tok, long long V, bool as_differences = false) {
        const float ls2 = ln_s * kLog2e, inv = ex2(-ls2);
        const float a0 = -scale * (g + h * H), b0 = -scale * h * kLn2;  // p ( a0 + b0 log2 p ),  p = 2^d / s
        a = (a0 - b0 * ls2) * inv;
        b = b0 * inv;
        onehot = scale * g;
        const float M = __fmul_rn(m, c);
        const bool fused = usual(M) && !as_differences;
        off = fused ? M : m;
        token = (int)tok;
        kind = tok >= V ? 3 : ln_s == INFINITY ? 2 : fused ? 0 : 1;
    }
    template <int N> __device__ __forceinline__ void at(float (&f)[N], float low, float c) const {
        const F2 cc = f2(c, c), oo = f2(-off, -off), aa = f2(a, a), bb = f2(b, b);
        auto one = [&](int k, F2 d, bool bound) {
            const F2 e = f2(ex2(d.x), ex2(d.y));
            const F2 y = mul2(e, fma2(bb, bound ? floored(d) : d, aa));
            f[k] = y.x;
            f[k + 1] = y.y;
        };
        if (kind == 0 && near(low, c)) {
#pragma unroll
            for (int k = 0; k < N; k += 2) one(k, fma2(f2(f[k], f[k + 1]), cc, oo), false);
        } else if (kind == 0) {
#pragma unroll
            for (int k = 0; k < N; k += 2) one(k, fma2(f2(f[k], f[k + 1]), cc, oo), true);
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 2) one(k, mul2(add2(f2(f[k], f[k + 1]), oo), cc), true);
        }
    }
    // A vector's gradients; `j0` its first column.
    template <class T> __device__ __forceinline__ uint4 vector(const uint4& u, int j0, float low, float c) const {
        constexpr int N = Vec<T>::N;
        float f[N];
        if (kind <= 1) {
            unpack16(u, f, (const T*)nullptr);
            at(f, low, c);
            const unsigned j = (unsigned)(token - j0);
            if (j < N) {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (k == (int)j) f[k] += onehot;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) f[k] = kind == 2 ? 0.f : NAN;
        }
        return pack16(f, (const T*)nullptr);
    }
    // The same where the smallest element is not known yet.
    template <class T> __device__ __forceinline__ uint4 vector(const uint4& u, int j0, float c) const {
        float top, low;
        const uint4 v[1] = {u};
        extremes<T>(v, top, low);
        return vector<T>(u, j0, low, c);
    }
    __device__ __forceinline__ float scalar(float x, int j, float c) const {
        if (kind > 1) return kind == 2 ? 0.f : NAN;
        float f[2] = {x, x};
        at(f, x, c);
        return f[0] + (j == token ? onehot : 0.f);
    }
};

// By how much c is off scale log2(e), relative to it.
__device__ __forceinline__ float error_of(float c, float scale) { return (fmaf(-scale, kLog2e, c) - scale * 1.925963e-8f) / c; }  // (log2(e) is kLog2e + 1.9e-8)

// The token's difference to the maximum as it is, less ln of the sum.  That sum is of 2^(x c - M) = e^(scale (x - m)) 2^((m c - M) + error (x - m) c): what M's and
// c's roundings make of it is taken out to the first order (`mean`: of x c - M under the softmax), or it would be a bias of 1e-8 |l| in every row, which sums
// over thousands of tokens keep.  So would be that ex2's results are 5.0e-8 of themselves too small on the average, alike for all fractions (measured over 4
// million arguments; 1.4e-7 at most): all terms' but the largest one's, whose share of the sum s is 2^(m c - M) / s.  (Terms that are differences: M = m c.)
__device__ __forceinline__ float logp_of(float xt, float m, float ls, float mean, float s, float scale, float c) {
    const float M = __fmul_rn(m, c), more = usual(M) ? fmaf(m, c, -M) : 0.f, others = 1.f - ex2(more) / s;
    const float off = kLn2 * (more + error_of(c, scale) * mean) - 5e-8f * (others < 0.f ? 0.f : others);
    const float l = scale * (xt - m) - (ls - off);
    return l > 0.f ? 0.f : l;  // (the sum's roundings: up to 1e-7 where the token has all the probability; NaN stays)
}
// The entropy from ln s and the mean of d (log to base 2); a difference of two equal numbers where one token has all the probability.
__device__ __forceinline__ float entropy_of(float ls, float mean) {
    const float H = ls - kLn2 * mean;
    return H < 0.f ? 0.f : H;
}

// The elements of a row that lie before the first 16-byte boundary.
template <class T> __device__ __forceinline__ int head_of(const void* p, long long n) {
    const int h = (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T));
    return (long long)h < n ? h : (int)n;
}

constexpr int kShortRow = 128;  // rows of up to so many logits are taken more exactly (see k_token_rows)

template <class T> __device__ __forceinline__ void store_vector(T* out, const uint4& u, bool vec) {
    if (vec) {
        *reinterpret_cast<uint4*>(out) = u;
    } else {
        T e[Vec<T>::N];
        *reinterpret_cast<uint4*>(e) = u;
#pragma unroll
        for (int k = 0; k < Vec<T>::N; ++k) out[k] = e[k];
    }
}

// A group of G threads works on one row: G <= 32 lanes of a warp, or the whole block (of 256 threads, or 1024).  Rows are read straight into registers; where the gradient
// follows (FUSED, rows of up to 1 KB, and those that no cluster holds) the second reading comes from the caches where the row fits.  A thread alone takes a row element by element.
// Backward alone, few rows: gridDim.y blocks share a row.
constexpr int threads_of(int G) { return G > 256 ? G : 256; }
template <class T, int G, int MODE>
__global__ void __launch_bounds__(threads_of(G)) k_token_rows(RowArgs A) {
    pdl_wait();
    constexpr int WARPS = threads_of(G) / 32;
    __shared__ float4 red[2][WARPS];
    __shared__ double redd[WARPS * kPolicyParts];
    __shared__ float2 both;  // of the row that the block works on (it is written again behind the barrier of the next row's sums)
    constexpr int GROUPS = threads_of(G) / G, N = Vec<T>::N, U = 4;
    const Rows& q = A.q;
    const int lane = threadIdx.x % G, V = (int)q.vocab;
    const float c = q.scale * kLog2e;
    const bool as_differences = G == 1 || (G <= 8 && V <= kShortRow);
    double part[kPolicyParts] = {0.0, 0.0, 0.0, 0.0, 0.0};
    int flip = 0;
    // (whole groups of a warp go through the loop together: the shuffles take all lanes)
    for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < q.rows; r0 += (long long)gridDim.x * GROUPS) {
        // (the gradient starts with the last rows, which the forward pass has left in L2: both passes over 1024 x 32000 bf16 40.6 us, this way 39.0)
        const long long r = MODE == BACKWARD ? q.rows - 1 - r0 - threadIdx.x / G : r0 + threadIdx.x / G;
        const bool there = r >= 0 && r < q.rows;
        const T* x = static_cast<const T*>(q.logits) + (there ? r : 0) * q.ld;
        // (a row of no sequence has its log-probability, but no part in the loss)
        const int info = !there ? -2 : MODE == FUSED ? A.info[r].x : row_counts(q, r) ? 0 : -2;
        const bool counts = info > -2, in_loss = info >= 0;
        const long long token = counts ? load_int(q.tokens, r, q.token_bytes) : 0;
        const int head = G > 1 ? head_of<T>(x, V) : 0;
        const int nvec = G > 1 ? (V - head) / N : 0, tail = head + nvec * N;
        const uint4* xv = reinterpret_cast<const uint4*>(x + head);
        // the elements of a row's head and tail: how many, and the e-th
        const int extras = head + (V - tail);
        auto extra = [&](int e) { return e < head ? e : tail + (e - head); };
        RowGrad gr;
        if constexpr (MODE != BACKWARD) {
            Acc acc;
            acc.clear();
            if (counts && as_differences) {  // (only the maximum is needed here)
                for (int j = lane; j < V; j += G) acc.m = fmaxf(acc.m, to_f(x[j]));
            } else if (counts) {
                if constexpr (G > 1) {
                    int i = lane;
                    for (; i + (U - 1) * G < nvec; i += U * G) {
                        uint4 u[U];
#pragma unroll
                        for (int k = 0; k < U; ++k) u[k] = xv[i + k * G];
                        acc.template add_vectors<T>(u, c);
                    }
                    for (; i < nvec; i += G) {
                        const uint4 u[1] = {xv[i]};
                        acc.template add_vectors<T>(u, c);
                    }
                    for (int e = lane; e < extras; e += G) {
                        const float f[2] = {to_f(x[extra(e)]), -INFINITY};
                        acc.add_scalars(f, c);
                    }
                }
            }
            Soft v = acc.sums();
            float ls, H;
            bool none;
            if (as_differences) {
                // Beside the largest logit the others may be next to nothing: s - 1 is summed, and ln s is its log1p.
                float top = v.m, s = 0.f, t = 0.f, n = 0.f;
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1)
                    if (G <= 8) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, o));
                for (int j = lane; counts && j < V; j += G) {
                    const float f = to_f(x[j]), d = q.scale * (f - top), e = expf(d);
                    if (f == top) n += 1.f;
                    else {
                        s += e;
                        if (e != 0.f) t = fmaf(e, d, t);
                    }
                }
#pragma unroll
                for (int o = G / 2; o > 0; o >>= 1) {
                    s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
                    t += __shfl_xor_sync(0xFFFFFFFFu, t, o);
                    n += __shfl_xor_sync(0xFFFFFFFFu, n, o);
                }
                none = top == -INFINITY && s == s;
                if (top == INFINITY) s = NAN;
                ls = none ? INFINITY : n == 1.f ? log1pf(s) : logf(n + s);
                H = none ? 0.f : ls - t / (n + s);
                v.m = top;
            } else {
                group_sum<(G < 32 ? G : 32)>(v, c);
                if constexpr (G > 32) {
                    // (two sets: a warp may be a row ahead of one that still reads)
                    if ((threadIdx.x & 31) == 0) red[flip][threadIdx.x >> 5] = make_float4(v.m, v.s, v.t, 0.f);
                    __syncthreads();
                    const float4 p = red[flip][threadIdx.x % WARPS];
                    flip ^= 1;
                    v = Soft{p.x, p.y, p.z};
                    group_sum<WARPS>(v, c);
                }
                none = v.s == 0.f;  // a row of -inf alone
                ls = none ? INFINITY : logf(v.s);
                H = none ? 0.f : entropy_of(ls, v.t / v.s);
            }
            float g = 0.f, h = 0.f;
            if (lane == 0 && there) {
                const float l = !counts ? 0.f : token >= V ? NAN : none ? -INFINITY : as_differences ? q.scale * (to_f(x[token]) - v.m) - ls : logp_of(to_f(x[token]), v.m, ls, v.t / v.s, v.s, q.scale, c);
                if (A.logp) A.logp[r] = l;
                if (A.entropy) A.entropy[r] = counts ? H : 0.f;
                if (MODE == FORWARD && A.norm) {
                    A.norm[2 * r] = counts && !none ? v.m : 0.f;
                    A.norm[2 * r + 1] = counts ? ls : 0.f;
                }
                if (MODE == FUSED && in_loss) {
                    const PolicyTerms p = policy_terms(A.o, l, A.old_logp ? A.old_logp[r] : 0.f, A.old_logp != nullptr, A.adv[r], A.ref ? A.ref[r] : 0.f);
                    const float w = row_weight(A.o, A.counts, A.per_seq, info);
                    part[0] += (double)(w * p.pg); part[1] += (double)(w * p.kl); part[2] += (double)(w * H);
                    part[3] += (double)(w * p.cut); part[4] += (double)(w * p.old_minus_new);
                    g = w * p.dlogp;
                    h = -A.o.entropy_coef * w;
                }
            }
            if constexpr (MODE == FUSED) {
                if constexpr (G > 32) {  // (the token's logit has been read before anything is stored, in place, too)
                    if (lane == 0) both = make_float2(g, h);
                    __syncthreads();
                    g = both.x;
                    h = both.y;
                } else {
                    const int src = (threadIdx.x & 31) / G * G;
                    g = __shfl_sync(0xFFFFFFFFu, g, src);
                    h = __shfl_sync(0xFFFFFFFFu, h, src);
                }
                gr.set(v.m, ls, g, h, H, q.scale, c, token, V, as_differences);
            }
        } else if (counts) {
            gr.set(A.norm_in[2 * r], A.norm_in[2 * r + 1], A.dlogp[r], A.dentropy ? A.dentropy[r] : 0.f, A.dentropy ? A.entropy_in[r] : 0.f, q.scale, c, token, V, as_differences);
        }
        if (MODE != FORWARD && there) {
            if (!in_loss) gr.kind = 2;
            T* out = static_cast<T*>(A.dlogits) + r * A.ld_out;
            if constexpr (G == 1) {
                for (int j = 0; j < V; ++j) out[j] = from_f<T>(gr.scalar(to_f(x[j]), j, c));
            } else {
                const bool vec = ((uintptr_t)(out + head) & 15) == 0;
                const int step = G * gridDim.y;
                int i = lane + G * blockIdx.y;
                for (; i + step < nvec; i += 2 * step) {
                    const uint4 u0 = xv[i], u1 = xv[i + step];
                    store_vector(out + head + (size_t)i * N, gr.template vector<T>(u0, head + i * N, c), vec);
                    store_vector(out + head + (size_t)(i + step) * N, gr.template vector<T>(u1, head + (i + step) * N, c), vec);
                }
                if (i < nvec) store_vector(out + head + (size_t)i * N, gr.template vector<T>(xv[i], head + i * N, c), vec);
                for (int e = lane; blockIdx.y == 0 && e < extras; e += G) out[extra(e)] = from_f<T>(gr.scalar(to_f(x[extra(e)]), extra(e), c));
            }
        }
    }
    if (MODE == FUSED) {
        block_sums(part, redd);
        if (threadIdx.x == 0) {
#pragma unroll
            for (int k = 0; k < kPolicyParts; ++k) A.part[(size_t)blockIdx.x * kPolicyParts + k] = part[k];
        }
    }
}

// ---- rows that a block, or a cluster of blocks, holds on chip ----
__device__ __forceinline__ uint32_t smem_of(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16_async(uint32_t dst, const void* src) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory"); }
__device__ __forceinline__ uint4 lds16(uint32_t a) {
    uint4 u;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(u.x), "=r"(u.y), "=r"(u.z), "=r"(u.w) : "r"(a) : "memory");
    return u;
}

constexpr int kMaxCluster = 8;

struct WideArgs {
    RowArgs a;
    int C, slice;  // blocks of a cluster, 16-byte vectors of a block's part of a row
};

// All but the last n groups of this thread's copies have arrived (n > 3: waits for more than that).
__device__ __forceinline__ void copies_but(int n) {
    if (n <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (n == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (n == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

// A cluster of C blocks walks over rows; each block holds its part of two rows in shared memory.  THREADS threads work on the logits: of the next row
// they take maxima and sums, then of this row the gradient, and replace each vector by one of the row after the next as soon as it is used
// (cp.async).  A thread reads only what it fetched itself, so its own waits are all the synchronisation the data needs.
// One warp more joins the sums: every warp's go into the shared memory of all blocks of the cluster (st.async, counted on an mbarrier; a cluster
// barrier would also wait for the gradient's stores to memory), and while the others work on the next row it takes the token's terms of the
// loss and leaves the row's constants for them.
// The logits are read from memory once and their gradient written once.  8192 x 131072 bf16, a tenth without a token: 878 us, 4.6 TB/s (at the copy rate 621); issue slots and the
// exponentials' unit are two thirds used.
template <class T, int THREADS, int PER_SM, int MODE>
__global__ void __launch_bounds__(THREADS + 32, PER_SM) k_token_rows_wide(WideArgs W) {
    pdl_wait();
    extern __shared__ __align__(16) unsigned char held[];
    // U vectors of a thread are a group of copies.  Four sets of sums: a block may be up to three rows behind its neighbours (see below).
    constexpr int WARPS = THREADS / 32, N = Vec<T>::N, U = 4, SETS = 4;
    __shared__ float4 parts[SETS][kMaxCluster * WARPS];
    __shared__ RowGrad row_grad[2];
    __shared__ uint64_t arrived[SETS], ready[2], done[2];
    const RowArgs& A = W.a;
    const Rows& q = A.q;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, C = W.C, rank = blockIdx.x % C;
    const int clusters = gridDim.x / C, V = (int)q.vocab;
    const float c = q.scale * kLog2e;
    if (tid == 0) {
        for (int k = 0; k < SETS; ++k) tc::mbar_init(&arrived[k], 1);
        for (int k = 0; k < 2; ++k) {
            tc::mbar_init(&ready[k], 1);
            tc::mbar_init(&done[k], WARPS);
        }
        tc::mbar_fence_init();
    }
    tc::cluster_sync_all();

    // A row's sequence (-1: no part in the loss; -2: does not count) and its token, from 2^31 - 1 on cut off (no column is).
    auto info_of = [&](long long r) -> int2 {
        if (r >= q.rows) return make_int2(-2, 0);
        if (MODE == FUSED) return A.info[r];
        return row_counts(q, r) ? make_int2(0, (int)min(load_int(q.tokens, r, q.token_bytes), 0x7FFFFFFFll)) : make_int2(-2, 0);
    };
    const long long first = blockIdx.x / C;
    bool ok = true;  // no wait has given up; what follows one that has is NaN

    if (warp < WARPS) {
        const uint32_t mine = smem_of(held) + (uint32_t)tid * 16, other = (uint32_t)W.slice * 16;  // the second row's part
        // Where a row's vectors of this thread begin, how far they (0, THREADS, 2 THREADS, ...) go, and the elements before the row's first vector.
        struct Place {
            const uint4* p;
            int n, head;
        };
        const unsigned char* ahead = static_cast<const unsigned char*>(q.logits) + first * q.ld * (long long)sizeof(T);  // the next row to be placed
        const long long stride = (long long)clusters * q.ld * (long long)sizeof(T);
        const int begin = rank * W.slice + tid;
        auto place = [&]() -> Place {
            Place w;
            w.head = head_of<T>(ahead, V);
            w.n = min((V - w.head) / N - rank * W.slice, W.slice) - tid;
            w.p = reinterpret_cast<const uint4*>(ahead + w.head * (int)sizeof(T)) + begin;
            ahead += stride;
            return w;
        };
        auto fetch = [&](const Place& w, int of, uint32_t at, int from) {  // vectors from the from-th on, in groups of U
            const int n = of > -2 ? w.n : 0;
            for (int i = from; i < n; i += U * THREADS) {
#pragma unroll
                for (int k = 0; k < U; ++k)
                    if (i + k * THREADS < n) copy16_async(at + (uint32_t)(i + k * THREADS) * 16, w.p + i + k * THREADS);
                asm volatile("cp.async.commit_group;" ::: "memory");
            }
        };
        struct Row {
            float xe, low;  // the element outside the vectors that this thread has; its smallest logit
            int extra;      // its column, or -1
        };
        int sets = 0;  // rows whose sums have been sent
        // Maxima and sums of a row, to all blocks.
        auto sums = [&](const Place& w, int of, int token, uint32_t at) -> Row {
            Row row = {0.f, INFINITY, -1};
            const int n = w.n;
            if (rank == 0) {
                const int tail = w.head + (V - w.head) / N * N, e = tid < w.head ? tid : tail + tid - w.head;
                if (e < V) row.extra = e;
            }
            if (of <= -2) return row;
            if (row.extra >= 0) row.xe = to_f(*(reinterpret_cast<const T*>(w.p - begin) - w.head + row.extra));
            float top = -INFINITY;
            if (row.extra >= 0) top = row.low = row.xe;
            const int groups = (n + U * THREADS - 1) / (U * THREADS);  // (n <= 0: none)
            int i = 0;
            for (int k = 1; i + (U - 1) * THREADS < n; i += U * THREADS, ++k) {
                copies_but(groups - k);
                uint4 u[U];
#pragma unroll
                for (int v = 0; v < U; ++v) u[v] = lds16(at + (uint32_t)(i + v * THREADS) * 16);
                float hi, lo;
                extremes<T>(u, hi, lo);
                top = fmaxf(top, hi);
                row.low = fminf(row.low, lo);
            }
            copies_but(0);
            for (; i < n; i += THREADS) {
                const uint4 u[1] = {lds16(at + (uint32_t)i * 16)};
                float hi, lo;
                extremes<T>(u, hi, lo);
                top = fmaxf(top, hi);
                row.low = fminf(row.low, lo);
            }
            Acc acc;
            acc.clear();
            acc.m = warp_max(top);
            const float M = __fmul_rn(acc.m, c);
            if (usual(M) && near(row.low, c)) {
                const F2 cc = f2(c, c), off = f2(-M, -M);
#pragma unroll 4
                for (i = 0; i < n; i += THREADS) {
                    float f[N];
                    unpack16(lds16(at + (uint32_t)i * 16), f, (const T*)nullptr);
#pragma unroll
                    for (int k = 0; k < N; k += 2) acc.template term<false>(fma2(f2(f[k], f[k + 1]), cc, off));
                }
            } else {
                for (i = 0; i < n; i += THREADS) {
                    float f[N];
                    unpack16(lds16(at + (uint32_t)i * 16), f, (const T*)nullptr);
                    acc.add(f, row.low, c);
                }
            }
            if (row.extra >= 0) {
                const float f[2] = {row.xe, -INFINITY};
                acc.add(f, -INFINITY, c);
            }
            // the token's logit goes with its owner's sums (-inf from everybody else)
            const int rel = token - w.head, vec = (rel >> (sizeof(T) == 4 ? 2 : 3)) - begin;  // (rel < 0: vec < 0)
            float xt = -INFINITY;
            bool own = false;
            if (vec >= 0 && vec < n && vec % THREADS == 0 && token < V) {
                own = true;
                if constexpr (sizeof(T) == 4) {
                    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(xt) : "r"(at + (uint32_t)vec * 16 + (uint32_t)(rel % N) * 4) : "memory");
                } else {
                    uint16_t h;
                    asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at + (uint32_t)vec * 16 + (uint32_t)(rel % N) * 2) : "memory");
                    xt = to_f(*reinterpret_cast<const T*>(&h));
                }
            } else if (row.extra >= 0 && row.extra == token) {
                own = true;
                xt = row.xe;
            }
            const unsigned owner = __ballot_sync(0xFFFFFFFFu, own);
            if (owner) xt = __shfl_sync(0xFFFFFFFFu, xt, __ffs(owner) - 1);
            Soft v = acc.sums();
            F2 st = f2(v.s, v.t);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) st = add2(st, f2(__shfl_xor_sync(0xFFFFFFFFu, st.x, o), __shfl_xor_sync(0xFFFFFFFFu, st.y, o)));
            v.s = st.x;
            v.t = st.y;
            const int set = sets++ & (SETS - 1);
            if (lane < C) {  // lane k writes to block k of the cluster
                const uint32_t dst = tc::mapa(smem_of(&parts[set][rank * WARPS + warp]), (uint32_t)lane), bar = tc::mapa(smem_of(&arrived[set]), (uint32_t)lane);
                asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(dst), "f"(v.m), "f"(v.s), "f"(v.t),
                             "f"(xt), "r"(bar)
                             : "memory");
            }
            return row;
        };

        int2 info_next = info_of(first + clusters);
        const int2 info_first = info_of(first);
        Place now = place(), next = place();
        fetch(now, info_first.x, mine, 0);
        fetch(next, info_next.x, mine + other, 0);
        Row row = sums(now, info_first.x, info_first.y, mine);  // (waits for both rows)
        unsigned char* out_row = static_cast<unsigned char*>(A.dlogits) + first * A.ld_out * (long long)sizeof(T);
        int k = 0;
        for (long long r = first; r < q.rows; r += clusters, ++k) {
            const uint32_t here = mine + (k & 1 ? other : 0u), there = mine + (k & 1 ? 0u : other);
            const int2 info_third = info_of(r + 2ll * clusters);
            const Row row_next = sums(next, info_next.x, info_next.y, there);
            const Place third = place();
            const uint4* p3 = third.p;
            const int n3 = info_third.x > -2 ? third.n : 0;
            int i = 0;
            ok = ok && tc::mbar_wait(&ready[k & 1], (k >> 1) & 1);
            if (MODE == FUSED) {
                RowGrad g = row_grad[k & 1];
                if (!ok) g.kind = 3;
                const int n = now.n;
                T* out = reinterpret_cast<T*>(out_row);
                T* part_out = out + now.head + (size_t)begin * N;
                const int j0 = now.head + begin * N;
                const bool vec = ((uintptr_t)part_out & 15) == 0;
                const bool fast = g.kind == 0 && near(row.low, c) && vec;
                if (fast) {
                    const F2 cc = f2(c, c), oo = f2(-g.off, -g.off), aa = f2(g.a, g.a), bb = f2(g.b, g.b);
                    const int at = g.token - j0;  // the taken token, from this thread's first element on
                    auto one = [&](int iv) {
                        float f[N];
                        unpack16(lds16(here + (uint32_t)iv * 16), f, (const T*)nullptr);
#pragma unroll
                        for (int u = 0; u < N; u += 2) {
                            const F2 d = fma2(f2(f[u], f[u + 1]), cc, oo), e = f2(ex2(d.x), ex2(d.y)), y = mul2(e, fma2(bb, d, aa));
                            f[u] = y.x;
                            f[u + 1] = y.y;
                        }
                        if ((unsigned)(at - iv * N) < (unsigned)N) {
#pragma unroll
                            for (int u = 0; u < N; ++u)
                                if (u == at - iv * N) f[u] += g.onehot;
                        }
                        *reinterpret_cast<uint4*>(part_out + (size_t)iv * N) = pack16(f, (const T*)nullptr);
                        if (iv < n3) copy16_async(here + (uint32_t)iv * 16, p3 + iv);
                    };
                    for (; i + (U - 1) * THREADS < n; i += U * THREADS) {
#pragma unroll
                        for (int v = 0; v < U; ++v) one(i + v * THREADS);
                        asm volatile("cp.async.commit_group;" ::: "memory");
                    }
                    for (; i < n; i += THREADS) one(i);
                    asm volatile("cp.async.commit_group;" ::: "memory");  // (a group too many only makes sums() wait for more)
                }
                for (int j = fast ? n : 0; j < n; j += THREADS) store_vector(part_out + (size_t)j * N, g.template vector<T>(lds16(here + (uint32_t)j * 16), j0 + j * N, row.low, c), vec);
                if (row.extra >= 0) out[row.extra] = from_f<T>(g.scalar(row.xe, row.extra, c));
            }
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&done[k & 1]);
            fetch(third, info_third.x, here, i);
            now = next;
            next = third;
            row = row_next;
            info_next = info_third;
            out_row += (long long)clusters * A.ld_out * (long long)sizeof(T);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // ---- the joining warp
        struct Taken { float old, adv, ref; int in_seq; };
        auto taken_of = [&](long long r, int of) {  // of a row ahead: nothing on the way from the sums to the gradient waits for memory
            Taken m = {0.f, 0.f, 0.f, 1};
            if (MODE == FUSED && of >= 0) {
                if (A.old_logp) m.old = A.old_logp[r];
                m.adv = A.adv[r];
                if (A.ref) m.ref = A.ref[r];
                if (A.o.mean == ANAKIN_MEAN_SEQUENCE) m.in_seq = A.per_seq[of];
            }
            return m;
        };
        int2 info_now = info_of(first), info_next = info_of(first + clusters);
        int sets = 0, k = 0;
        Taken taken = taken_of(first, info_now.x);
        float weight = A.o.inv_divisor;  // of a row, but for the rows of its sequence
        if (MODE == FUSED && A.o.mean != ANAKIN_MEAN_FIXED) weight = (float)(A.o.mean == ANAKIN_MEAN_TOKEN ? A.counts->rows : A.counts->sequences);
        double stat = 0.0;  // of lane i: the i-th sum
        for (long long r = first; r < q.rows; r += clusters, ++k) {
            const int info = info_now.x, token = info_now.y;
            const int2 info_third = info_of(r + 2ll * clusters);
            const Taken taken_next = taken_of(r + clusters, info_next.x);
            float l = 0.f, H = 0.f, ls = 0.f, m = 0.f;
            RowGrad g = {0.f, 0.f, 0.f, 0.f, 0, 2};
            if (info > -2) {
                const int set = sets & (SETS - 1);
                if (lane == 0) tc::mbar_expect_tx(&arrived[set], (uint32_t)(C * WARPS * 16));
                ok = tc::warp_all(ok && tc::mbar_wait(&arrived[set], (sets / SETS) & 1));
                ++sets;
                const float4* from = parts[set];
                const int np = C * WARPS;
                float top = -INFINITY, xt = -INFINITY, s = 0.f, t = 0.f;
                for (int i = lane; i < np; i += 32) {
                    top = fmaxf(top, from[i].x);
                    xt = fmaxf(xt, from[i].w);  // (-inf but from the token's owner; a NaN there is one in the sums, too)
                }
                m = warp_max(top);
                xt = warp_max(xt);
                for (int i = lane; i < np; i += 32) {
                    const float4 p4 = from[i];
                    Soft p{p4.x, p4.y, p4.z};
                    p.rescale(m, c);
                    s += p.s;
                    t += p.t;
                }
                s = warp_sum(s);
                t = warp_sum(t);
                const bool none = s == 0.f;  // a row of -inf alone
                ls = none ? INFINITY : logf(s);
                H = none ? 0.f : entropy_of(ls, t / s);
                l = token >= V || !ok ? NAN : none ? -INFINITY : logp_of(xt, m, ls, t / s, s, q.scale, c);
                if (none) m = 0.f;
                if (MODE == FUSED && info >= 0) {
                    const PolicyTerms p = policy_terms(A.o, l, taken.old, A.old_logp != nullptr, taken.adv, taken.ref);
                    // (as row_weight() has it)
                    const float w = A.o.mean == ANAKIN_MEAN_FIXED ? weight : 1.f / ((float)taken.in_seq * weight);
                    g.set(m, ls, w * p.dlogp, -A.o.entropy_coef * w, H, q.scale, c, token, V);
                    if (!ok) g.kind = 3;
                    stat += (double)(w * (lane == 0 ? p.pg : lane == 1 ? p.kl : lane == 2 ? H : lane == 3 ? p.cut : p.old_minus_new));
                }
            }
            if (k >= 2) ok = tc::warp_all(ok && tc::mbar_wait(&done[k & 1], ((k >> 1) - 1) & 1));  // its last row's constants have been used
            if (lane == 0) {
                row_grad[k & 1] = g;
                tc::mbar_arrive(&ready[k & 1]);
            }
            if (rank == 0 && lane == 0) {
                if (A.logp) A.logp[r] = l;
                if (A.entropy) A.entropy[r] = H;
                if (MODE == FORWARD && A.norm) {
                    A.norm[2 * r] = m;
                    A.norm[2 * r + 1] = ls;
                }
            }
            info_now = info_next;
            info_next = info_third;
            taken = taken_next;
        }
        if (MODE == FUSED && rank == 0 && lane < kPolicyParts) A.part[(size_t)(blockIdx.x / C) * kPolicyParts + lane] = stat;
    }
    tc::cluster_sync_all();  // (no block leaves while another may still write to it: also where a wait gave up)
}
// How far apart blocks of a cluster can be.  A block sends its sums of row k + 4 after its gradient of row k + 2, for which it needed everybody's
// sums of row k + 2; a block sends those after its gradient of row k, for which its joining warp was done with the sums of row k.  So a set is written
// again only when it has been read.

// Shapes of the kernel above.
struct WidePlan {
    int threads, C, slice;  // threads = 0: not for this shape
};
WidePlan wide_plan(const Rows& q, size_t es) {
    const long long bytes = q.vocab * (long long)es, vecs = (bytes + 15) / 16;
    WidePlan p = {0, 1, (int)vecs};
    if (bytes <= 1024) return p;
    if (bytes <= 16384 && q.rows >= 148) {
        p.threads = bytes <= 6144 ? 64 : 128;
        return p;
    }
    // Two rows' parts a block: 54 KB each with two blocks an SM (three up to 35 KB: 16384 x 32000 bf16 471 us, with two 506), 110 KB with one.  Large
    // parts, as every row costs every thread some 250 instructions besides its vectors (8192 x 131072 bf16 in clusters of 5 878 us, of 8 some 950).
    auto blocks = [&](long long most) { return (int)((vecs * 16 + most - 1) / most); };
    const int b = blocks(54272), d = blocks(111616);
    p.threads = b <= kMaxCluster ? 256 : d <= kMaxCluster ? 512 : 0;
    p.C = b <= kMaxCluster ? b : d;
    // few rows: more blocks a row
    while (p.threads != 0 && p.C * 2 <= kMaxCluster && q.rows * p.C < 148 * 2 && vecs / p.C > 512) {
        p.C *= 2;
        p.threads = 256;
    }
    p.slice = (int)((vecs + p.C - 1) / p.C);
    return p;
}

// Clusters that the GPU runs at once, by the runtime's own count; a few shapes come up again and again in a program.
template <auto K> cudaError_t clusters_at_once(int C, int threads, size_t smem, int* n) {
    static std::atomic<uint64_t> slots[64];  // device, C and shared memory of the shape above bit 16; the count below
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t key = ((uint64_t)(dev + 1) << 32) | ((uint64_t)C << 24) | (uint64_t)smem;
    std::atomic<uint64_t>& slot = slots[(key * 0x9E3779B97F4A7C15ull) >> 58];
    const uint64_t seen = slot.load(std::memory_order_relaxed);
    if (seen >> 16 == key) {
        *n = (int)(seen & 0xFFFFu);
        return cudaSuccess;
    }
    if ((e = allow_shared<K>()) != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(148 * 8 / C * C);
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if ((e = cudaOccupancyMaxActiveClusters(n, K, &cfg)) != cudaSuccess) return e;
    if (*n > 0xFFFF) *n = 0xFFFF;
    slot.store((key << 16) | (uint64_t)*n, std::memory_order_relaxed);
    return cudaSuccess;
}
template <class T, int THREADS, int PER_SM, int MODE>
cudaError_t launch_wide(const WideArgs& W, int* parts, cudaStream_t s) {
    constexpr auto K = k_token_rows_wide<T, THREADS, PER_SM, MODE>;
    const size_t smem = (size_t)W.slice * 32;
    int most = 0;
    const cudaError_t e = clusters_at_once<K>(W.C, THREADS + 32, smem, &most);
    if (e != cudaSuccess) return e;
    if (most < 1) return cudaErrorNotSupported;
    if (most > kMaxPartials) most = kMaxPartials;
    const int clusters = (int)(W.a.q.rows < most ? W.a.q.rows : most);
    if (parts) *parts = clusters;
    return launch_cluster<K>(dim3(clusters * W.C), dim3(THREADS + 32), smem, s, W.C, W);
}

template <class T, int G, int MODE>
cudaError_t launch_rows(const RowArgs& A, int* parts, cudaStream_t s) {
    constexpr int GROUPS = threads_of(G) / G;
    const long long ctas = (A.q.rows + GROUPS - 1) / GROUPS;
    const int grid = (int)(ctas < kMaxPartials ? ctas : kMaxPartials);
    int share = 1;  // blocks of a row
    if (MODE == BACKWARD && G > 32) {
        const long long vecs = A.q.vocab / Vec<T>::N;
        while (share < 16 && grid * share < 148 * 4 && vecs > 512ll * share) share *= 2;
    }
    if (parts) *parts = grid;
    return launch<k_token_rows<T, G, MODE>>(dim3(grid, share), dim3(threads_of(G)), 0, s, A);
}

template <class T, int MODE>
cudaError_t launch_rows_t(const RowArgs& A, int* parts, cudaStream_t s) {
    if (A.q.vocab <= 8) return launch_rows<T, 1, MODE>(A, parts, s);
    const long long bytes = A.q.vocab * (long long)sizeof(T);
    if (bytes <= 1024) return launch_rows<T, 8, MODE>(A, parts, s);
    if constexpr (MODE != BACKWARD) {
        const WidePlan p = wide_plan(A.q, sizeof(T));
        if (p.threads != 0 && (MODE == FUSED || (p.threads >= 256 && A.q.rows < 592))) {
            const WideArgs W = {A, p.C, p.slice};
            if (p.threads == 256 && p.slice * 16 <= 35840) return launch_wide<T, 256, 3, MODE>(W, parts, s);
            if (p.threads == 256) return launch_wide<T, 256, 2, MODE>(W, parts, s);
            if (p.threads == 512) return launch_wide<T, 512, 1, MODE>(W, parts, s);
            if constexpr (MODE == FUSED) return p.threads == 64 ? launch_wide<T, 64, 8, MODE>(W, parts, s) : launch_wide<T, 128, 5, MODE>(W, parts, s);
        }
    }
    // a warp a row while that gives every SM its fill of rows, several times over where rows are long (forward: 32768 x 12000 bf16 153 us, by whole
    // blocks 291; backward by blocks 260, by warps 281)
    if constexpr (MODE == FUSED) {
        // rows that no cluster holds, above 872 KB (64 x 262144 fp32: 59 us by blocks of 1024 threads, by those of 256 159, by warps 1004)
        return launch_rows<T, 1024, MODE>(A, parts, s);
    } else {
        if (bytes <= 4096 || (bytes <= 16384 && A.q.rows >= 148 * 16) || (MODE == FORWARD && bytes <= 65536 && A.q.rows >= 148 * 192)) return launch_rows<T, 32, MODE>(A, parts, s);
        return launch_rows<T, 256, MODE>(A, parts, s);
    }
}

template <int MODE>
cudaError_t launch_rows_any(int dtype, const RowArgs& A, int* parts, cudaStream_t s) {
    if (dtype == ANAKIN_DTYPE_F32) return launch_rows_t<float, MODE>(A, parts, s);
    if (dtype == ANAKIN_DTYPE_BF16) return launch_rows_t<__nv_bfloat16, MODE>(A, parts, s);
    return launch_rows_t<__half, MODE>(A, parts, s);
}

}  // namespace
}  // namespace tok
}  // namespace anakin

using namespace anakin;
using namespace anakin::tok;

static bool bad_output(const anakin_token_rows* rows, const void* dlogits, int64_t ld_out) {
    return ld_out < rows->vocab || (rows->rows > 0 && (!dlogits || ((uintptr_t)dlogits & (rows->dtype == ANAKIN_DTYPE_F32 ? 3 : 1))));
}

extern "C" {

int anakin_token_logp(const anakin_token_rows* rows, float* logp, float* entropy, float* norm, void* cuda_stream) {
    RowArgs A = {};
    const int rc = check_rows(rows, true, true, false, &A.q);
    if (rc != ANAKIN_OK) return rc;
    if (A.q.rows == 0) return ANAKIN_OK;
    if (!logp) return ANAKIN_E_INVALID_ARG;
    A.logp = logp;
    A.entropy = entropy;
    A.norm = norm;
    return launch_rows_any<FORWARD>(rows->dtype, A, nullptr, (cudaStream_t)cuda_stream) == cudaSuccess ? ANAKIN_OK : fail();
}

int anakin_token_logp_backward(const anakin_token_rows* rows, const float* norm, const float* entropy, const float* dlogp,
                               const float* dentropy, void* dlogits, int64_t ld_out, void* cuda_stream) {
    RowArgs A = {};
    const int rc = check_rows(rows, true, true, false, &A.q);
    if (rc != ANAKIN_OK) return rc;
    if (bad_output(rows, dlogits, ld_out)) return ANAKIN_E_INVALID_ARG;
    if (A.q.rows == 0) return ANAKIN_OK;
    if (!norm || !dlogp || (dentropy && !entropy)) return ANAKIN_E_INVALID_ARG;
    A.norm_in = norm;
    A.entropy_in = entropy;
    A.dlogp = dlogp;
    A.dentropy = dentropy;
    A.dlogits = dlogits;
    A.ld_out = ld_out;
    return launch_rows_any<BACKWARD>(rows->dtype, A, nullptr, (cudaStream_t)cuda_stream) == cudaSuccess ? ANAKIN_OK : fail();
}

int anakin_token_policy_grad(const anakin_token_rows* rows, const anakin_policy_objective* objective, const float* old_logp, const float* adv,
                             const float* ref_logp, float* stats, float* logp, float* entropy, void* dlogits, int64_t ld_out,
                             void* dev_workspace, size_t bytes, void* cuda_stream) {
    RowArgs A = {};
    int rc = check_rows(rows, true, true, false, &A.q);
    if (rc == ANAKIN_OK) rc = check_policy(objective, &A.o);
    if (rc != ANAKIN_OK) return rc;
    const bool empty = A.q.rows == 0;
    if (!stats || bad_output(rows, dlogits, ld_out) || (!empty && (!adv || (A.o.kl != ANAKIN_KL_NONE && !ref_logp)))) return ANAKIN_E_INVALID_ARG;
    const Workspace w = carve(dev_workspace, A.q.rows, A.q.sequences);
    if (!dev_workspace || ((uintptr_t)dev_workspace & 255)) return ANAKIN_E_INVALID_ARG;
    if (bytes < w.bytes) return ANAKIN_E_WORKSPACE_TOO_SMALL;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    A.logp = logp;
    A.entropy = entropy;
    A.dlogits = dlogits;
    A.ld_out = ld_out;
    A.old_logp = old_logp;
    A.adv = adv;
    A.ref = A.o.kl != ANAKIN_KL_NONE ? ref_logp : nullptr;
    A.counts = w.counts;
    A.per_seq = w.per_seq;
    A.part = w.part;
    A.info = w.info;
    int grid = 0;
    if (!empty) {
        if (launch_counts(A.q, A.o.mean, true, w, s) != cudaSuccess) return fail();
        if (launch_rows_any<FUSED>(rows->dtype, A, &grid, s) != cudaSuccess) return fail();
    }
    return launch_policy_stats(w.part, grid, A.o, stats, s) == cudaSuccess ? ANAKIN_OK : fail();
}

}  // extern "C"
