// Softmax rows over a token vocabulary: log-probability and entropy of the taken token, the gradient of the logits, and both around the
// clipped policy loss in one kernel.
//
// With x the logits of a row, c = scale log2(e), m = max x, d_j = c (x_j - m):
//   s = sum 2^d,  t = sum 2^d d   in one pass, rescaled whenever m grows;   log p_j = ln2 d_j - ln s;   H = ln s - ln2 t / s
//   dx_j = scale ( g ([j = token] - p_j) - h p_j (log p_j + H) )
// The differences x_j - m are formed before they are scaled: then masks of the type's lowest value stay finite and large logits lose nothing.
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
    double* part;
};

enum { FORWARD = 0, BACKWARD = 1, FUSED = 2 };

// Running maximum, sum and weighted sum of a part of a row.
struct Soft {
    float m, s, t;
    __device__ __forceinline__ void clear() { m = -INFINITY; s = 0.f; t = 0.f; }
    __device__ __forceinline__ void rescale(float to, float c) {  // to >= m
        if (m < to) {
            if (s != 0.f) {  // (nothing but -inf so far: nothing to rescale)
                const float d = (m - to) * c, f = ex2(d);
                t = f * (t + (f > 0.f ? s * d : 0.f));
                s *= f;
            }
            m = to;
        }
    }
    template <int N> __device__ __forceinline__ void add(const float (&x)[N], float c) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < N; ++i) top = fmaxf(top, x[i]);
        rescale(top, c);
        const float at = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float d = (x[i] - at) * c, e = ex2(d);
            s += e;
            t = fmaf(e, fmaxf(d, -1e30f), t);  // (0 times -inf would be NaN; a NaN comes through s)
        }
    }
    __device__ __forceinline__ void add1(float x, float c) {
        const float v[1] = {x};
        add(v, c);
    }
    __device__ __forceinline__ void join(float m2, float s2, float t2, float c) {
        Soft b{m2, s2, t2};
        const float to = fmaxf(m, m2);
        rescale(to, c);
        b.rescale(to, c);
        s += b.s;
        t += b.t;
    }
};

// What the gradient needs of a row.
struct RowGrad {
    float m, ls2, g, h, a;  // ls2 = log2 s;  dx = p ( -(g + h ln2 (d2 + ...)) )  with scale in: see grad()
    // d2 = log2 p;  scale (-(g) - h (ln2 d2 + H)) p = p (a + b d2),  a = -scale (g + h H),  b = -scale h ln2
    float b, onehot;
    __device__ __forceinline__ void set(float m_, float ln_s, float g_, float h_, float H, float scale) {
        m = m_;
        ls2 = ln_s * kLog2e;
        g = g_;
        h = h_;
        a = -scale * (g_ + h_ * H);
        b = -scale * h_ * kLn2;
        onehot = scale * g_;
    }
    __device__ __forceinline__ float at(float x, float c) const {
        const float d2 = fmaf(x - m, c, -ls2);
        const float p = ex2(d2);
        return p * fmaf(b, fmaxf(d2, -1e30f), a);
    }
};

// A group of G threads of the CTA works on one row: G <= 32 lanes of a warp, or the whole CTA.
template <int G> __device__ __forceinline__ void group_join(Soft& v, float c, float* red) {
    constexpr int W = G < 32 ? G : 32;
#pragma unroll
    for (int o = W / 2; o > 0; o >>= 1) {
        const float m2 = __shfl_xor_sync(0xFFFFFFFFu, v.m, o), s2 = __shfl_xor_sync(0xFFFFFFFFu, v.s, o), t2 = __shfl_xor_sync(0xFFFFFFFFu, v.t, o);
        v.join(m2, s2, t2, c);
    }
    if constexpr (G > 32) {
        const int w = threadIdx.x >> 5;
        __syncthreads();
        if ((threadIdx.x & 31) == 0) { red[3 * w] = v.m; red[3 * w + 1] = v.s; red[3 * w + 2] = v.t; }
        __syncthreads();
        v = Soft{red[0], red[1], red[2]};
        for (int i = 1; i < G / 32; ++i) v.join(red[3 * i], red[3 * i + 1], red[3 * i + 2], c);
    }
}

// The elements of a row that lie before the first 16-byte boundary.
template <class T> __device__ __forceinline__ int head_of(const void* p, long long n) {
    const int h = (int)(((16 - ((uintptr_t)p & 15)) & 15) / sizeof(T));
    return (long long)h < n ? h : (int)n;
}

template <class T, int G, int MODE>
__global__ void __launch_bounds__(256) k_token_rows(RowArgs A) {
    pdl_wait();
    __shared__ float red[3 * 8];
    __shared__ double redd[8];
    __shared__ float bc[4];
    constexpr int GROUPS = 256 / G, N = Vec<T>::N;
    const Rows& q = A.q;
    const int lane = threadIdx.x % G, V = (int)q.vocab;
    const float c = q.scale * kLog2e;
    double part[kPolicyParts] = {0.0, 0.0, 0.0, 0.0, 0.0};
    // (whole groups of a warp go through the loop together: the shuffles take all lanes)
    for (long long r0 = (long long)blockIdx.x * GROUPS; r0 < q.rows; r0 += (long long)gridDim.x * GROUPS) {
        const long long r = r0 + threadIdx.x / G;
        const bool there = r < q.rows;
        const T* x = static_cast<const T*>(q.logits) + (there ? r : 0) * q.ld;
        bool counts = there && row_counts(q, r);
        const long long token = there && q.tokens ? load_int(q.tokens, r, q.token_bytes) : 0;
        int seq = 0;
        bool in_loss = counts;  // a row of no sequence has its log-probability, but no part in the loss
        if (MODE == FUSED && counts) {
            seq = sequence_of(q, r);
            in_loss = seq >= 0 && seq < q.sequences;
            counts = in_loss || A.logp || A.entropy;
        }
        const int head = G >= 32 ? head_of<T>(x, V) : V;  // narrow groups walk a row element by element
        const int nvec = G >= 32 ? (V - head) / N : 0, tail = head + nvec * N;
        RowGrad gr;
        if (MODE != BACKWARD) {
            Soft v;
            v.clear();
            if (counts) {
                for (int j = lane; j < head; j += G) v.add1(to_f(x[j]), c);
                if constexpr (G >= 32) {
                    const uint4* xv = reinterpret_cast<const uint4*>(x + head);
                    for (int i = lane; i < nvec; i += G) {
                        float f[N];
                        unpack16(xv[i], f, (const T*)nullptr);
                        v.add(f, c);
                    }
                    for (int j = tail + lane; j < V; j += G) v.add1(to_f(x[j]), c);
                }
            }
            group_join<G>(v, c, red);
            // a row of -inf alone: s = 0
            const float ls = v.s == 0.f ? INFINITY : logf(v.s), H = v.s == 0.f ? 0.f : ls - kLn2 * (v.t / v.s);
            if (lane == 0 && there) {
                float l = 0.f;
                if (counts) l = token >= V ? NAN : v.s == 0.f ? -INFINITY : q.scale * (to_f(x[token]) - v.m) - ls;
                if (A.logp) A.logp[r] = l;
                if (A.entropy) A.entropy[r] = counts ? H : 0.f;
                if (MODE == FORWARD && A.norm) {
                    A.norm[2 * r] = counts ? (v.s == 0.f ? 0.f : v.m) : 0.f;
                    A.norm[2 * r + 1] = counts ? ls : 0.f;
                }
                if (MODE == FUSED) {
                    float g = 0.f, h = 0.f;
                    if (in_loss) {
                        const PolicyTerms p = policy_terms(A.o, l, A.old_logp ? A.old_logp[r] : 0.f, A.old_logp != nullptr, A.adv[r], A.ref ? A.ref[r] : 0.f);
                        const float w = row_weight(A.o, A.counts, A.per_seq, seq);
                        part[0] += (double)(w * p.pg); part[1] += (double)(w * p.kl); part[2] += (double)(w * H);
                        part[3] += (double)(w * p.cut); part[4] += (double)(w * p.old_minus_new);
                        g = w * p.dlogp;
                        h = -A.o.entropy_coef * w;
                    }
                    gr.g = g;
                    gr.h = h;
                }
            }
            if (MODE == FUSED) {
                float g = gr.g, h = gr.h;
                if constexpr (G > 32) {
                    if (threadIdx.x == 0) { bc[0] = g; bc[1] = h; }
                    __syncthreads();
                    g = bc[0];
                    h = bc[1];
                } else {
                    const int src = (threadIdx.x & 31) / G * G;
                    g = __shfl_sync(0xFFFFFFFFu, g, src);
                    h = __shfl_sync(0xFFFFFFFFu, h, src);
                }
                gr.set(v.m, ls, g, h, H, q.scale);
            }
        } else if (counts) {
            gr.set(A.norm_in[2 * r], A.norm_in[2 * r + 1], A.dlogp[r], A.dentropy ? A.dentropy[r] : 0.f, A.dentropy ? A.entropy_in[r] : 0.f, q.scale);
        }
        if (MODE != FORWARD && there) {
            const bool zero = !in_loss || gr.ls2 == INFINITY;
            T* out = static_cast<T*>(A.dlogits) + r * A.ld_out;
            auto one = [&](int j) {
                float v = zero ? 0.f : gr.at(to_f(x[j]), c);
                if (!zero && j == token) v += gr.onehot;
                if (!zero && token >= V) v = NAN;
                out[j] = from_f<T>(v);
            };
            const bool vec = G >= 32 && ((uintptr_t)(out + head) & 15) == 0;
            if (!vec) {
                for (int j = lane; j < V; j += G) one(j);
            } else {
                for (int j = lane; j < head; j += G) one(j);
                const uint4* xv = reinterpret_cast<const uint4*>(x + head);
                uint4* ov = reinterpret_cast<uint4*>(out + head);
                const long long tv = token - head;
                for (int i = lane; i < nvec; i += G) {
                    float f[N];
                    if (zero) {
                        ov[i] = make_uint4(0u, 0u, 0u, 0u);
                        continue;
                    }
                    unpack16(xv[i], f, (const T*)nullptr);
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] = gr.at(f[k], c);
                    const long long k = tv - (long long)i * N;
#pragma unroll
                    for (int u = 0; u < N; ++u) {
                        if (u == k) f[u] += gr.onehot;
                        if (token >= V) f[u] = NAN;
                    }
                    ov[i] = pack16(f, (const T*)nullptr);
                }
                for (int j = tail + lane; j < V; j += G) one(j);
            }
        }
        if (G > 32 && MODE != BACKWARD) __syncthreads();  // red and bc are written again
    }
    if (MODE == FUSED) {
#pragma unroll
        for (int k = 0; k < kPolicyParts; ++k) {
            const double s = block_sum(part[k], redd);
            if (threadIdx.x == 0) A.part[(size_t)blockIdx.x * kPolicyParts + k] = s;
        }
    }
}

template <class T, int G, int MODE>
cudaError_t launch_rows(const RowArgs& A, int* grid_out, cudaStream_t s) {
    const long long ctas = (A.q.rows + 256 / G - 1) / (256 / G);
    const int grid = (int)(ctas < 148 * 16 ? ctas : 148 * 16);
    if (grid_out) *grid_out = grid;
    return launch<k_token_rows<T, G, MODE>>(dim3(grid), dim3(256), 0, s, A);
}

template <class T, int MODE>
cudaError_t launch_rows_t(const RowArgs& A, int* grid, cudaStream_t s) {
    if (A.q.vocab <= 8) return launch_rows<T, 1, MODE>(A, grid, s);
    if (A.q.vocab <= 128) return launch_rows<T, 8, MODE>(A, grid, s);
    if (A.q.vocab <= 2048) return launch_rows<T, 32, MODE>(A, grid, s);
    return launch_rows<T, 256, MODE>(A, grid, s);
}

template <int MODE>
cudaError_t launch_rows_any(int dtype, const RowArgs& A, int* grid, cudaStream_t s) {
    if (dtype == ANAKIN_DTYPE_F32) return launch_rows_t<float, MODE>(A, grid, s);
    if (dtype == ANAKIN_DTYPE_BF16) return launch_rows_t<__nv_bfloat16, MODE>(A, grid, s);
    return launch_rows_t<__half, MODE>(A, grid, s);
}

}  // namespace
}  // namespace tok
}  // namespace anakin

using namespace anakin;
using namespace anakin::tok;

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
    if (ld_out < rows->vocab) return ANAKIN_E_INVALID_ARG;
    if (A.q.rows == 0) return ANAKIN_OK;
    if (!norm || !dlogp || !dlogits || (dentropy && !entropy)) return ANAKIN_E_INVALID_ARG;
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
    if (!stats || ld_out < rows->vocab || (!empty && (!adv || !dlogits || (A.o.kl != ANAKIN_KL_NONE && !ref_logp)))) return ANAKIN_E_INVALID_ARG;
    const Workspace w = carve(dev_workspace, A.q.sequences);
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
    int grid = 0;
    if (!empty) {
        if (A.o.mean != ANAKIN_MEAN_FIXED && launch_counts(A.q, w.counts, A.o.mean == ANAKIN_MEAN_SEQUENCE ? w.per_seq : nullptr, s) != cudaSuccess) return fail();
        if (launch_rows_any<FUSED>(rows->dtype, A, &grid, s) != cudaSuccess) return fail();
    }
    return launch_policy_stats(w.part, grid, A.o, stats, s) == cudaSuccess ? ANAKIN_OK : fail();
}

}  // extern "C"
