// The losses over tokens from log-probabilities: the clipped policy loss with a KL term, and the preference loss over pairs of answers; and the
// counts of rows that their means divide by.  All of it is a few vectors of one number a token: the launches cost more than the
// bytes up to some hundred thousand tokens, so short batches are done by one CTA in one launch.
#include <algorithm>

#include "token_rows.cuh"

namespace anakin {
namespace tok {

int fail() {
    cudaGetLastError();
    return ANAKIN_E_CUDA;
}

int check_rows(const anakin_token_rows* p, bool need_logits, bool need_tokens, bool need_offsets, Rows* q) {
    if (!p || p->struct_size != sizeof(anakin_token_rows) || p->reserved != 0) return ANAKIN_E_INVALID_ARG;
    constexpr int64_t LIMIT = int64_t(1) << 31;
    if (p->rows < 0 || p->rows >= LIMIT || p->sequences < 0 || p->sequences >= LIMIT - 1) return ANAKIN_E_INVALID_ARG;
    if (p->tokens && p->token_bytes != 4 && p->token_bytes != 8) return ANAKIN_E_INVALID_ARG;
    if (p->offsets && p->offset_bytes != 4 && p->offset_bytes != 8) return ANAKIN_E_INVALID_ARG;
    if (p->tokens && ((uintptr_t)p->tokens & (p->token_bytes - 1))) return ANAKIN_E_INVALID_ARG;
    if (p->offsets && ((uintptr_t)p->offsets & (p->offset_bytes - 1))) return ANAKIN_E_INVALID_ARG;
    if (need_offsets && !p->offsets) return ANAKIN_E_INVALID_ARG;
    if (need_logits) {
        if (p->dtype < ANAKIN_DTYPE_F32 || p->dtype > ANAKIN_DTYPE_F16) return ANAKIN_E_INVALID_ARG;
        if (p->vocab < 1 || p->vocab >= LIMIT || p->ld < p->vocab || !(p->scale > 0.f) || !(p->scale <= 1.0995116e12f)) return ANAKIN_E_INVALID_ARG;
        if (p->rows > 0 && (!p->logits || ((uintptr_t)p->logits & (p->dtype == ANAKIN_DTYPE_F32 ? 3 : 1)))) return ANAKIN_E_INVALID_ARG;
    }
    if (need_tokens && p->rows > 0 && !p->tokens) return ANAKIN_E_INVALID_ARG;
    q->rows = p->rows; q->vocab = p->vocab; q->ld = p->ld;
    q->logits = p->logits; q->tokens = p->tokens; q->mask = p->mask; q->offsets = p->offsets;
    q->sequences = p->offsets ? (int)p->sequences : 1;
    q->token_bytes = p->token_bytes; q->offset_bytes = p->offset_bytes;
    q->scale = p->scale;
    return ANAKIN_OK;
}

int check_policy(const anakin_policy_objective* p, Objective* o) {
    if (!p || p->struct_size != sizeof(anakin_policy_objective)) return ANAKIN_E_INVALID_ARG;
    if (!(p->clip_low >= 0.f && p->clip_low <= 1.f) || !(p->clip_high >= 0.f) || !(p->dual_clip == 0.f || p->dual_clip >= 1.f)) return ANAKIN_E_INVALID_ARG;
    if (p->kl < ANAKIN_KL_NONE || p->kl > ANAKIN_KL_3 || p->mean < ANAKIN_MEAN_TOKEN || p->mean > ANAKIN_MEAN_FIXED) return ANAKIN_E_INVALID_ARG;
    if (p->mean == ANAKIN_MEAN_FIXED && !(p->divisor > 0.f)) return ANAKIN_E_INVALID_ARG;
    if (p->kl_coef != p->kl_coef || p->entropy_coef != p->entropy_coef) return ANAKIN_E_INVALID_ARG;
    o->lo = 1.f - p->clip_low;
    o->hi = 1.f + p->clip_high;
    o->dual = p->dual_clip;
    o->kl = p->kl;
    o->kl_coef = p->kl == ANAKIN_KL_NONE ? 0.f : p->kl_coef;
    o->entropy_coef = p->entropy_coef;
    o->mean = p->mean;
    o->inv_divisor = p->mean == ANAKIN_MEAN_FIXED ? 1.f / p->divisor : 0.f;
    return ANAKIN_OK;
}

// Blocks of a sequence in the preference loss: of few long sequences each is shared, some 1024 rows a block.
static int prefer_splits(long long rows, long long sequences) {
    const long long n = sequences > 0 ? rows / sequences / 1024 : 1;
    return (int)(n < 1 ? 1 : n < 64 ? n : 64);
}

Workspace carve(void* base, long long rows, long long sequences) {
    size_t off = 0;
    auto take = [&](size_t bytes) { void* p = static_cast<unsigned char*>(base) + off; off += (bytes + 255) / 256 * 256; return p; };
    Workspace w;
    const size_t parts = (size_t)sequences * prefer_splits(rows, sequences);
    w.counts = static_cast<Counts*>(take(sizeof(Counts) + sizeof(int) * parts));
    w.per_seq = reinterpret_cast<int*>(w.counts + 1);
    w.part = static_cast<double*>(take(sizeof(double) * kMaxPartials * kPolicyParts));
    w.sums = static_cast<double*>(take(sizeof(double) * parts));
    w.coef = static_cast<float*>(take(sizeof(float) * (size_t)sequences));
    w.info = static_cast<int2*>(take(sizeof(int2) * (size_t)rows));
    w.bytes = off;
    return w;
}

namespace {

constexpr int kSmallRows = 8192, kSmallSeqs = 4096;  // up to here one CTA does it all

// Adds a warp's 32 rows to the counts: lanes whose rows lie in one sequence add once.  Sums of integers: any order gives the same.
__device__ __forceinline__ void add_counts(bool counts, int seq, unsigned long long* rows, unsigned long long* seqs, int* per_seq) {
    const unsigned in = __ballot_sync(0xFFFFFFFFu, counts);
    if (!in) return;
    const int lane = threadIdx.x & 31;
    if (lane == __ffs(in) - 1) atomicAdd(rows, (unsigned long long)__popc(in));
    if (!per_seq || !counts) return;
    const unsigned same = __match_any_sync(in, seq);
    if (lane == __ffs(same) - 1 && atomicAdd(&per_seq[seq], __popc(same)) == 0) atomicAdd(seqs, 1ull);
}

// sequence_of(r) for a row that is known to lie in sequence `from` or behind it.
__device__ __forceinline__ int sequence_from(const Rows& q, int from, long long r) {
    if (from >= q.sequences || load_int(q.offsets, from + 1, q.offset_bytes) > r) return from;
    int lo = from + 2, hi = q.sequences + 1;
    while (lo < hi) {
        const int mid = lo + ((hi - lo) >> 1);  // (their sum may pass 2^31)
        if (load_int(q.offsets, mid, q.offset_bytes) <= r) lo = mid + 1;
        else hi = mid;
    }
    return lo - 1;
}
// sequence_of(r) by a whole warp, which probes 32 offsets at once: three loads one after the other for thousands of sequences.
__device__ __forceinline__ int warp_sequence_of(const Rows& q, long long r) {
    const int lane = threadIdx.x & 31;
    int lo = 0, hi = q.sequences + 1;  // the number of offsets <= r lies in [lo, hi]
    while (hi - lo > 32) {
        const int at = lo + (int)((long long)(hi - lo) * (lane + 1) / 33);
        const int n = __popc(__ballot_sync(0xFFFFFFFFu, load_int(q.offsets, at, q.offset_bytes) <= r));
        const int below = __shfl_sync(0xFFFFFFFFu, at, n > 0 ? n - 1 : 0), above = __shfl_sync(0xFFFFFFFFu, at, n < 32 ? n : 31);
        if (n > 0) lo = below + 1;
        if (n < 32) hi = above;
    }
    lo += __popc(__ballot_sync(0xFFFFFFFFu, lane < hi - lo && load_int(q.offsets, lo + lane, q.offset_bytes) <= r));
    return lo - 1;
}
// The sequences of the rows r0 + lane.
__device__ __forceinline__ int warp_sequences(const Rows& q, long long r0) {
    return q.offsets ? sequence_from(q, warp_sequence_of(q, r0), r0 + (threadIdx.x & 31)) : 0;
}

// (a kernel, as a copy engine's memset would wait for all before it and be waited for: 65536 rows 12.3 us with it, 8.4 so)
__global__ void __launch_bounds__(256) k_zero_counts(Counts* c, int* per_seq, int sequences) {
    PDL_START();
    const int i0 = blockIdx.x * 256 + threadIdx.x;
    if (i0 == 0) *c = Counts{0ull, 0ull};
    for (long long i = i0; i < sequences; i += (long long)gridDim.x * 256) per_seq[i] = 0;
}

constexpr int kCountSteps = 4;  // groups of 32 rows, one behind the other, that a warp counts at least before it adds to the sums in memory

__global__ void __launch_bounds__(256) k_token_counts(Rows q, Counts* c, int* per_seq, int2* info) {
    pdl_wait();  // (no early trigger: blocks of the next kernel placed around this one's would leave its clusters without room, a wave late)
    __shared__ unsigned total;
    if (threadIdx.x == 0) total = 0;
    __syncthreads();
    const int lane = threadIdx.x & 31;
    const long long groups = (q.rows + 31) / 32, warps = (long long)gridDim.x * 8, each = (groups + warps - 1) / warps;
    const long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * each, last = min(first + each, groups);
    int from = 0;  // the sequence of the last row looked at
    int held = -1, n = 0;  // rows of one sequence that are not yet added to its count
    unsigned rows = 0;
    auto add = [&]() {
        if (lane == 0 && n > 0 && atomicAdd(&per_seq[held], n) == 0) atomicAdd(&c->sequences, 1ull);
    };
    if (first < last && q.offsets) from = warp_sequence_of(q, first * 32);
    for (long long g = first; g < last; ++g) {
        const long long r = g * 32 + lane;
        bool counts = r < q.rows && row_counts(q, r);
        const int found = q.offsets ? sequence_from(q, from, min(r, q.rows - 1)) : 0;
        from = __shfl_sync(0xFFFFFFFFu, found, 31);
        const int seq = !counts ? -2 : found >= 0 && found < q.sequences ? found : -1;
        if (info && r < q.rows) info[r] = make_int2(seq, q.tokens && seq > -2 ? (int)min(load_int(q.tokens, r, q.token_bytes), 0x7FFFFFFFll) : 0);
        counts = seq >= 0;
        const unsigned in = __ballot_sync(0xFFFFFFFFu, counts);
        if (!in || !c) continue;
        rows += __popc(in);
        if (!per_seq) continue;
        const int one = __shfl_sync(0xFFFFFFFFu, seq, __ffs(in) - 1);
        if (__ballot_sync(0xFFFFFFFFu, seq == one) == in) {
            if (one != held) {
                add();
                held = one;
                n = 0;
            }
            n += __popc(in);
        } else if (counts) {
            const unsigned same = __match_any_sync(in, seq);
            if (lane == __ffs(same) - 1 && atomicAdd(&per_seq[seq], __popc(same)) == 0) atomicAdd(&c->sequences, 1ull);
        }
    }
    if (!c) return;
    if (per_seq) add();
    if (lane == 0) atomicAdd(&total, rows);
    __syncthreads();
    if (threadIdx.x == 0 && total > 0) atomicAdd(&c->rows, (unsigned long long)total);
}

__device__ __forceinline__ void write_stats(const Objective& o, const double (&v)[kPolicyParts], float* stats) {
    stats[0] = (float)(v[0] + (double)o.kl_coef * v[1] - (double)o.entropy_coef * v[2]);
#pragma unroll
    for (int k = 0; k < kPolicyParts; ++k) stats[1 + k] = (float)v[k];
}

__global__ void __launch_bounds__(256) k_policy_stats(const double* part, int n, Objective o, float* stats) {
    PDL_START();
    __shared__ double red[8 * kPolicyParts];
    double v[kPolicyParts] = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (int i = threadIdx.x; i < n; i += 256)
#pragma unroll
        for (int k = 0; k < kPolicyParts; ++k) v[k] += part[(size_t)i * kPolicyParts + k];
    block_sums(v, red);
    if (threadIdx.x == 0) write_stats(o, v, stats);
}

struct PolicyArgs2 {
    Rows q;
    Objective o;
    const float* logp;
    const float* old_logp;
    const float* adv;
    const float* ref;
    const float* entropy;
    float* stats;
    float* dlogp;
    float* dentropy;
    Counts* counts;
    int* per_seq;
    double* part;
};

// A row whose sequence is known (-1: no part in the loss).
__device__ __forceinline__ void policy_row(const PolicyArgs2& A, long long r, int seq, const Counts* c, const int* per_seq, double (&part)[kPolicyParts]) {
    float g = 0.f, h = 0.f;
    if (seq >= 0) {
        const PolicyTerms p = policy_terms(A.o, A.logp[r], A.old_logp ? A.old_logp[r] : 0.f, A.old_logp != nullptr, A.adv[r], A.ref ? A.ref[r] : 0.f);
        const float w = row_weight(A.o, c, per_seq, seq);
        const float H = A.entropy ? A.entropy[r] : 0.f;
        part[0] += (double)(w * p.pg); part[1] += (double)(w * p.kl); part[2] += (double)(w * H);
        part[3] += (double)(w * p.cut); part[4] += (double)(w * p.old_minus_new);
        g = w * p.dlogp;
        h = A.entropy ? -A.o.entropy_coef * w : 0.f;
    }
    A.dlogp[r] = g;
    if (A.dentropy) A.dentropy[r] = h;
}
__device__ __forceinline__ int loss_sequence(const Rows& q, long long r, const int* near) {
    if (!row_counts(q, r)) return -1;
    const int seq = sequence_of(q, r, near);
    return seq < q.sequences ? seq : -1;
}

__global__ void __launch_bounds__(256) k_policy_loss(PolicyArgs2 A) {
    PDL_START();
    __shared__ double red[8 * kPolicyParts];
    double part[kPolicyParts] = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (long long r0 = (long long)blockIdx.x * 256 + (threadIdx.x & ~31); r0 < A.q.rows; r0 += (long long)gridDim.x * 256) {
        const long long r = r0 + (threadIdx.x & 31);
        const int seq = warp_sequences(A.q, r0);
        if (r < A.q.rows) policy_row(A, r, seq < A.q.sequences && row_counts(A.q, r) ? seq : -1, A.counts, A.per_seq, part);
    }
    block_sums(part, red);
    if (threadIdx.x == 0) {
#pragma unroll
        for (int k = 0; k < kPolicyParts; ++k) A.part[(size_t)blockIdx.x * kPolicyParts + k] = part[k];
    }
}

// Offsets into shared memory as 32-bit numbers (rows are fewer than 2^31: what lies outside is as good at the border).
__device__ __forceinline__ const int* fetch_offsets(const Rows& q, int* to) {
    if (!q.offsets) return nullptr;
    for (int i = threadIdx.x; i <= q.sequences; i += blockDim.x) {
        const long long v = load_int(q.offsets, i, q.offset_bytes);
        to[i] = v < -1 ? -1 : v > q.rows ? (int)q.rows : (int)v;
    }
    return to;
}

// One CTA: counts, terms and statistics of up to kSmallRows rows and kSmallSeqs sequences; every row's sequence is looked for once.
__global__ void __launch_bounds__(1024) k_policy_loss_small(PolicyArgs2 A) {
    PDL_START();
    constexpr int EACH = kSmallRows / 1024;
    __shared__ double red[32 * kPolicyParts];
    __shared__ Counts c;
    __shared__ int per_seq[kSmallSeqs], offsets[kSmallSeqs + 1];
    const Rows& q = A.q;
    const bool by_seq = A.o.mean == ANAKIN_MEAN_SEQUENCE;
    if (threadIdx.x == 0) c = Counts{0ull, 0ull};
    if (by_seq) for (int i = threadIdx.x; i < q.sequences; i += 1024) per_seq[i] = 0;
    const int* near = fetch_offsets(q, offsets);
    __syncthreads();
    int seq[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = k * 1024 + threadIdx.x;
        seq[k] = -1;
        if (k * 1024 >= (int)q.rows) continue;  // (the block's threads leave together)
        if (r < (int)q.rows) seq[k] = loss_sequence(q, r, near);
        if (A.o.mean != ANAKIN_MEAN_FIXED) add_counts(seq[k] >= 0, seq[k], &c.rows, &c.sequences, by_seq ? per_seq : nullptr);
    }
    __syncthreads();
    double part[kPolicyParts] = {0.0, 0.0, 0.0, 0.0, 0.0};
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int r = k * 1024 + threadIdx.x;
        if (r < (int)q.rows) policy_row(A, r, seq[k], &c, per_seq, part);
    }
    block_sums(part, red);
    if (threadIdx.x == 0) write_stats(A.o, part, A.stats);
}

// ---- preference loss ----
struct PreferArgs {
    Rows q;
    int P, kind, mean;
    float beta, margin, smoothing;
    const float* logp;
    const float* ref;
    float* stats;
    float* zout;
    float* dlogp;
    int splits;    // blocks of a sequence
    int* per_seq;  // [2P][splits] counted rows
    double* sums;  // [2P][splits] sums of l - ref
    float* coef;   // [2P] gradient of every counted row of a sequence
};

// First and last row of a sequence, within bounds whatever the offsets are.
__device__ __forceinline__ void rows_of(const Rows& q, int seq, long long& lo, long long& hi) {
    lo = load_int(q.offsets, seq, q.offset_bytes);
    hi = load_int(q.offsets, seq + 1, q.offset_bytes);
    lo = lo < 0 ? 0 : lo;
    hi = hi > q.rows ? q.rows : hi;
}

__device__ __forceinline__ double softplus(double v) { return (v > 0.0 ? v : 0.0) + log1p(exp(-fabs(v))); }

// Loss of a pair and its derivative by z.
__device__ __forceinline__ void pair_terms(const PreferArgs& A, double z, double& loss, double& dz) {
    if (A.kind == ANAKIN_PREFER_SIGMOID) {
        const double e = (double)A.smoothing;
        loss = (1.0 - e) * softplus(-z) + e * softplus(z);
        dz = e - 1.0 / (1.0 + exp(z));  // (not sigmoid(z) - (1 - e), which loses the digits of a slope near 0)
    } else if (A.kind == ANAKIN_PREFER_HINGE) {
        loss = z < 1.0 ? 1.0 - z : z >= 1.0 ? 0.0 : z;
        dz = z >= 1.0 ? 0.0 : -1.0;
        if (z != z) dz = z;
    } else {
        const double b = (double)A.beta, h = (z - 0.5) / b;
        loss = h * h;
        dz = 2.0 * h / b;
    }
}

// Sums and counts of the sequences, `splits` blocks each; in 64 bits, as sums of many thousand terms are subtracted from one another.
__global__ void __launch_bounds__(256) k_prefer_sums(PreferArgs A) {
    PDL_START();
    __shared__ double red[8 * 2];
    for (long long i = blockIdx.x; i < 2ll * A.P * A.splits; i += gridDim.x) {
        const int seq = (int)(i / A.splits), split = (int)(i - (long long)seq * A.splits);
        long long lo, hi;
        rows_of(A.q, seq, lo, hi);
        double v[2] = {0.0, 0.0};
        for (long long r0 = lo + split * 1024 + threadIdx.x; r0 < hi; r0 += 1024ll * A.splits) {
            float l[4], ref[4];
            bool counts[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {  // (all on their way before the first is used)
                const long long r = r0 + 256 * k;
                const bool in = r < hi;
                l[k] = in ? A.logp[r] : 0.f;
                ref[k] = in && A.ref ? A.ref[r] : 0.f;
                counts[k] = in && row_counts(A.q, r);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (counts[k]) {
                    v[0] += (double)l[k] - (double)ref[k];
                    v[1] += 1.0;
                }
        }
        block_sums(v, red);
        if (threadIdx.x == 0) {
            A.sums[i] = v[0];
            A.per_seq[i] = (int)v[1];
        }
        __syncthreads();
    }
}

// A pair's part of the statistics (v[0 .. 4], and v[5] counts it), its z, and the gradients of its sequences' rows but for the number of pairs.
__device__ __forceinline__ void take_pair(const PreferArgs& A, int p, double (&v)[6], double& z, double& d0, double& d1) {
    double a[2];
    int n[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const size_t at = (size_t)(p + k * A.P) * A.splits;
        a[k] = 0.0;
        n[k] = 0;
        for (int s = 0; s < A.splits; ++s) {
            a[k] += A.sums[at + s];
            n[k] += A.per_seq[at + s];
        }
        if (A.mean && n[k] > 0) a[k] /= n[k];
    }
    z = d0 = d1 = 0.0;
    if (n[0] < 1 || n[1] < 1) return;
    const double b = (double)A.beta;
    z = b * (a[0] - a[1]) - (double)A.margin;
    double loss, dz;
    pair_terms(A, z, loss, dz);
    d0 = b * dz / (A.mean ? n[0] : 1);
    d1 = -b * dz / (A.mean ? n[1] : 1);
    v[0] += loss;
    v[1] += z > 0.0 ? 1.0 : 0.0;
    v[2] += b * a[0];
    v[3] += b * a[1];
    v[4] += z;
    v[5] += 1.0;
}
__device__ __forceinline__ void write_pair_stats(const PreferArgs& A, const double (&v)[6]) {
    for (int k = 0; k < ANAKIN_PREFERENCE_STATS; ++k) A.stats[k] = v[5] > 0.0 ? (float)(v[k] / v[5]) : 0.f;
}

// Margins, statistics, and the gradient that every counted row of a sequence gets; by one CTA.
__global__ void __launch_bounds__(1024) k_prefer_pairs(PreferArgs A) {
    PDL_START();
    __shared__ double red[32 * 6];
    __shared__ double pairs;
    double v[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0};
    for (int p = threadIdx.x; p < A.P; p += 1024) {
        double z, d0, d1;
        take_pair(A, p, v, z, d0, d1);
        A.zout[p] = (float)z;
        // (without the number of pairs, which is not known yet: in the place of the sums)
        A.sums[(size_t)p * A.splits] = d0;
        A.sums[(size_t)(p + A.P) * A.splits] = d1;
    }
    block_sums(v, red);
    if (threadIdx.x == 0) {
        write_pair_stats(A, v);
        pairs = v[5] > 0.0 ? v[5] : 1.0;
    }
    __syncthreads();
    for (int p = threadIdx.x; p < A.P; p += 1024) {
        A.coef[p] = (float)(A.sums[(size_t)p * A.splits] / pairs);
        A.coef[p + A.P] = (float)(A.sums[(size_t)(p + A.P) * A.splits] / pairs);
    }
}
// A row's sequence, -1 for none that counts.
__device__ __forceinline__ int prefer_sequence(const PreferArgs& A, long long r, const int* near) {
    if (!row_counts(A.q, r)) return -1;
    const int seq = sequence_of(A.q, r, near);
    return seq < 2 * A.P ? seq : -1;
}
__global__ void __launch_bounds__(256) k_prefer_rows(PreferArgs A) {
    PDL_START();
    for (long long r0 = (long long)blockIdx.x * 256 + (threadIdx.x & ~31); r0 < A.q.rows; r0 += (long long)gridDim.x * 256) {
        const long long r = r0 + (threadIdx.x & 31);
        const int seq = warp_sequences(A.q, r0);
        if (r < A.q.rows) A.dlogp[r] = seq >= 0 && seq < 2 * A.P && row_counts(A.q, r) ? A.coef[seq] : 0.f;
    }
}

// Both for up to kFewPairs pairs: every CTA takes all pairs for itself, one a thread, instead of waiting for a kernel of one CTA (256 pairs, 262144
// rows: 13.4 us with it, 11.0 without).
constexpr int kFewPairs = 1024;
__global__ void __launch_bounds__(1024) k_prefer_few(PreferArgs A) {
    if (A.P == 0) pdl_wait();  // (no sums before it)
    __shared__ double red[32 * 6];
    __shared__ double pairs;
    __shared__ float coef[2 * kFewPairs];
    __shared__ int offsets[2 * kFewPairs + 1];
    // While the sums are still on their way: the sequences of the thread's first rows.  (k_prefer_sums lets this kernel start once all before it is
    // complete, so offsets, mask and tokens are.)
    const int* near = fetch_offsets(A.q, offsets);
    __syncthreads();
    const long long r0 = (long long)blockIdx.x * 1024 + threadIdx.x, step = (long long)gridDim.x * 1024;
    int seq[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) seq[k] = r0 + k * step < A.q.rows ? prefer_sequence(A, r0 + k * step, near) : -1;
    PDL_START();
    double v[6] = {0.0, 0.0, 0.0, 0.0, 0.0, 0.0}, z = 0.0, d0 = 0.0, d1 = 0.0;
    const int p = threadIdx.x;
    if (p < A.P) take_pair(A, p, v, z, d0, d1);
    if (blockIdx.x == 0 && p < A.P) A.zout[p] = (float)z;
    block_sums(v, red);
    if (threadIdx.x == 0) {
        if (blockIdx.x == 0) write_pair_stats(A, v);
        pairs = v[5] > 0.0 ? v[5] : 1.0;
    }
    __syncthreads();
    if (p < A.P) {
        coef[p] = (float)(d0 / pairs);
        coef[p + A.P] = (float)(d1 / pairs);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k)
        if (r0 + k * step < A.q.rows) A.dlogp[r0 + k * step] = seq[k] >= 0 ? coef[seq[k]] : 0.f;
    for (long long r = r0 + 2 * step; r < A.q.rows; r += step) {
        const int of = prefer_sequence(A, r, near);
        A.dlogp[r] = of >= 0 ? coef[of] : 0.f;
    }
}

int grid_for(long long rows, int per_cta, int most) {
    const long long n = (rows + per_cta - 1) / per_cta;
    return (int)(n < 1 ? 1 : n < most ? n : most);
}

}  // namespace

cudaError_t launch_counts(const Rows& q, int mean, bool rows_too, const Workspace& w, cudaStream_t s) {
    const bool by_seq = mean == ANAKIN_MEAN_SEQUENCE;
    if (mean != ANAKIN_MEAN_FIXED) {
        const int seqs = by_seq ? q.sequences : 0;
        const cudaError_t e = launch<k_zero_counts>(dim3(grid_for(seqs, 1024, 148)), dim3(256), 0, s, w.counts, w.per_seq, seqs);
        if (e != cudaSuccess) return e;
    } else if (!rows_too) {
        return cudaSuccess;
    }
    return launch<k_token_counts>(dim3(grid_for(q.rows, 256 * kCountSteps, 148 * 8)), dim3(256), 0, s, q, mean != ANAKIN_MEAN_FIXED ? w.counts : nullptr,
                                  by_seq ? w.per_seq : nullptr, rows_too ? w.info : nullptr);
}

cudaError_t launch_policy_stats(const double* part, int n, const Objective& o, float* stats, cudaStream_t s) {
    return launch<k_policy_stats>(dim3(1), dim3(256), 0, s, part, n, o, stats);
}

}  // namespace tok
}  // namespace anakin

using namespace anakin;
using namespace anakin::tok;

extern "C" {

int anakin_token_workspace_bytes(int64_t rows, int64_t sequences, size_t* bytes) {
    if (!bytes || rows < 0 || sequences < 0 || rows >= (int64_t(1) << 31) || sequences >= (int64_t(1) << 31) - 1) return ANAKIN_E_INVALID_ARG;
    // (the one sequence of rows without offsets may be shared by more blocks than a few of them)
    *bytes = std::max(carve(nullptr, rows, 1).bytes, carve(nullptr, rows, sequences).bytes);
    return ANAKIN_OK;
}

int anakin_token_policy_loss(const anakin_token_rows* rows, const anakin_policy_objective* objective, const float* logp, const float* old_logp,
                             const float* adv, const float* ref_logp, const float* entropy, float* stats, float* dlogp, float* dentropy,
                             void* dev_workspace, size_t bytes, void* cuda_stream) {
    PolicyArgs2 A = {};
    int rc = check_rows(rows, false, false, false, &A.q);
    if (rc == ANAKIN_OK) rc = check_policy(objective, &A.o);
    if (rc != ANAKIN_OK) return rc;
    const bool empty = A.q.rows == 0;
    if (!stats || (!empty && (!logp || !adv || !dlogp || (A.o.kl != ANAKIN_KL_NONE && !ref_logp)))) return ANAKIN_E_INVALID_ARG;
    if (!dev_workspace || ((uintptr_t)dev_workspace & 255)) return ANAKIN_E_INVALID_ARG;
    const Workspace w = carve(dev_workspace, A.q.rows, A.q.sequences);
    if (bytes < w.bytes) return ANAKIN_E_WORKSPACE_TOO_SMALL;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    A.logp = logp;
    A.old_logp = old_logp;
    A.adv = adv;
    A.ref = A.o.kl != ANAKIN_KL_NONE ? ref_logp : nullptr;
    A.entropy = entropy;
    A.stats = stats;
    A.dlogp = dlogp;
    A.dentropy = dentropy;
    A.counts = w.counts;
    A.per_seq = w.per_seq;
    A.part = w.part;
    if (A.q.rows <= kSmallRows && A.q.sequences <= kSmallSeqs) {
        return launch<k_policy_loss_small>(dim3(1), dim3(1024), 0, s, A) == cudaSuccess ? ANAKIN_OK : fail();
    }
    if (launch_counts(A.q, A.o.mean, false, w, s) != cudaSuccess) return fail();
    const int grid = grid_for(A.q.rows, 256, kMaxPartials);
    if (launch<k_policy_loss>(dim3(grid), dim3(256), 0, s, A) != cudaSuccess) return fail();
    return launch_policy_stats(w.part, grid, A.o, stats, s) == cudaSuccess ? ANAKIN_OK : fail();
}

int anakin_token_preference_loss(const anakin_token_rows* rows, const anakin_preference_objective* objective, const float* logp,
                                 const float* ref_logp, float* stats, float* margin, float* dlogp, void* dev_workspace, size_t bytes,
                                 void* cuda_stream) {
    PreferArgs A = {};
    const int rc = check_rows(rows, false, false, true, &A.q);
    if (rc != ANAKIN_OK) return rc;
    const anakin_preference_objective* p = objective;
    if (!p || p->struct_size != sizeof(*p) || p->kind < ANAKIN_PREFER_SIGMOID || p->kind > ANAKIN_PREFER_SQUARED || !(p->beta > 0.f) ||
        !(p->beta < INFINITY) || p->margin != p->margin || !(p->smoothing >= 0.f && p->smoothing <= 0.5f) || (p->mean != 0 && p->mean != 1))
        return ANAKIN_E_INVALID_ARG;
    if (A.q.sequences % 2 != 0 || !stats || (A.q.sequences > 0 && !margin) || (A.q.rows > 0 && (!logp || !dlogp))) return ANAKIN_E_INVALID_ARG;
    if (!dev_workspace || ((uintptr_t)dev_workspace & 255)) return ANAKIN_E_INVALID_ARG;
    const Workspace w = carve(dev_workspace, A.q.rows, A.q.sequences);
    if (bytes < w.bytes) return ANAKIN_E_WORKSPACE_TOO_SMALL;
    cudaStream_t s = (cudaStream_t)cuda_stream;
    A.P = A.q.sequences / 2;
    A.kind = p->kind;
    A.mean = p->mean;
    A.beta = p->beta;
    A.margin = p->margin;
    A.smoothing = p->smoothing;
    A.logp = logp;
    A.ref = ref_logp;
    A.stats = stats;
    A.zout = margin;
    A.dlogp = dlogp;
    A.per_seq = w.per_seq;
    A.sums = w.sums;
    A.coef = w.coef;
    A.splits = prefer_splits(A.q.rows, A.q.sequences);
    if (A.P > 0 && launch<k_prefer_sums>(dim3(grid_for(2ll * A.P * A.splits, 1, 148 * 16)), dim3(256), 0, s, A) != cudaSuccess) return fail();
    if (A.P <= kFewPairs) {
        return launch<k_prefer_few>(dim3(grid_for(A.q.rows, 1024, 148)), dim3(1024), 0, s, A) == cudaSuccess ? ANAKIN_OK : fail();
    }
    if (launch<k_prefer_pairs>(dim3(1), dim3(1024), 0, s, A) != cudaSuccess) return fail();
    if (A.q.rows > 0 && launch<k_prefer_rows>(dim3(grid_for(A.q.rows, 256, 148 * 8)), dim3(256), 0, s, A) != cudaSuccess) return fail();
    return ANAKIN_OK;
}

}  // extern "C"
