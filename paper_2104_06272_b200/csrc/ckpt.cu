// Activation checkpoints in 8 bits: every row in blocks of 32 columns, a block as e4m3 numbers times a power of two.
//
// scale exponent E = the smallest with top 2^-E <= 448, top the block's largest finite |x|; code = round(x 2^-E) to e4m3, ties to even.  Scaling by
// a power of two is exact, so the code is the only rounding.  Everything here is bound by memory: a thread moves 8 columns of a row (one 16-byte
// load of 16-bit elements, 8 code bytes), four neighbours share a block, and a thread has two such pieces in flight.
#include <cuda_fp8.h>

#include "ckpt.cuh"
#include "token_rows.cuh"

namespace anakin {
namespace ckpt {
namespace {

using tok::from_f;
using tok::to_f;

struct Args {
    long long rows;  // of this launch
    int cols, blocks;
    FastDiv per_row;  // pieces of 8 columns in a row (4 a block)
    uint32_t pieces;  // rows * per_row < 2^31
    const void* x;    // forward: x; backward: dy
    long long ldx;
    void* y;          // forward: act(x) or null; unpack: x; backward: dx
    long long ldy;
    uint8_t* codes;
    uint8_t* scales;
    bool vec_x, vec_y;  // every row starts on a 16-byte boundary
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 ex2(float2 v) { return make_float2(tok::ex2(v.x), tok::ex2(v.y)); }
// FINE (fp32): what a product's rounding r takes from an exponent is put back, 2^(q + r) = 2^q (1 + r ln 2); r is below 2^-16.  16-bit types do not see it.
constexpr float kLog2eRest = 1.925963e-8f;  // log2(e) is kLog2e + this
__device__ __forceinline__ float2 put_back(float2 e, float2 r) { return __ffma2_rn(__fmul2_rn(e, both(tok::kLn2)), r, e); }

// 1 / (1 + exp(-x)): 0 for x below -126 ln2 (there x times it is below 2^-119), NaN stays, but not in FINE (x times it is one all the same).
template <bool FINE> __device__ __forceinline__ float2 sigmoid(float2 x) {
    float2 e;
    if (FINE) {  // (exp(88) has an fp32 number, and 1 / (1 + it) is given as 0)
        const float2 a = make_float2(fminf(fmaxf(-x.x, -200.f), 88.f), fminf(fmaxf(-x.y, -200.f), 88.f)), q = __fmul2_rn(a, both(tok::kLog2e));
        e = put_back(ex2(q), __ffma2_rn(a, both(kLog2eRest), __ffma2_rn(a, both(tok::kLog2e), make_float2(-q.x, -q.y))));
    } else {
        e = ex2(__fmul2_rn(x, both(-tok::kLog2e)));
    }
    return make_float2(__fdividef(1.f, 1.f + e.x), __fdividef(1.f, 1.f + e.y));
}
// The normal distribution function and its density (times sqrt(2 pi)) of two numbers.  Q(|x|) = exp(-x^2 / 2) times a polynomial in t = 1 / (1 + p |x|) without a
// constant term, fitted for this file (least squares, reweighted until the largest error is smallest, over 0 <= |x| <= 16): nine terms, off by 1.6e-8 of Q
// (evaluated in fp32 4e-7); for 16-bit types six, off by 7e-8 or, where Q is below 1e-3, 7e-5 of it.
template <bool FINE> __device__ __forceinline__ float2 normal(float2 x, float2& density) {
    constexpr float kFine[9] = {0.106401980f, 0.106038909f, 0.102237833f, 0.0648655083f, 0.126530668f, -0.0988459486f, 0.200554947f, -0.137941195f, 0.0301573012f};
    constexpr float kShort[6] = {0.117681872f, 0.106051226f, 0.164907422f, -0.0652277831f, 0.261766630f, -0.0851794475f};
    constexpr float kHalfLog2e = -0.5f * tok::kLog2e;
    float2 z = make_float2(fabsf(x.x), fabsf(x.y)), p;
    if (FINE) {  // (from 16 on the density is 0)
        z = make_float2(fminf(z.x, 16.f), fminf(z.y, 16.f));
        const float2 h = __fmul2_rn(z, z), l = __ffma2_rn(z, z, make_float2(-h.x, -h.y)), q = __fmul2_rn(h, both(kHalfLog2e));
        const float2 r = __ffma2_rn(h, both(kHalfLog2e), make_float2(-q.x, -q.y));
        density = put_back(ex2(q), __ffma2_rn(l, both(kHalfLog2e), __ffma2_rn(h, both(-0.5f * kLog2eRest), r)));
    } else {
        density = ex2(__fmul2_rn(__fmul2_rn(z, z), both(kHalfLog2e)));
    }
    const float2 u = __ffma2_rn(z, both(FINE ? 0.266672194f : 0.293045700f), both(1.f));
    const float2 t = make_float2(__fdividef(1.f, u.x), __fdividef(1.f, u.y));
    constexpr int N = FINE ? 9 : 6;
    p = both(FINE ? kFine[8] : kShort[5]);
#pragma unroll
    for (int k = N - 2; k >= 0; --k) p = __ffma2_rn(t, p, both(FINE ? kFine[k] : kShort[k < 6 ? k : 5]));
    const float2 q = __fmul2_rn(__fmul2_rn(density, t), p);
    return make_float2(x.x > 0.f ? 1.f - q.x : q.x, x.y > 0.f ? 1.f - q.y : q.y);
}
template <bool FINE, int ACT> __device__ __forceinline__ float2 act_of(float2 x) {
    if (ACT == ANAKIN_ACT_SILU || ACT == ANAKIN_ACT_GELU) {
        float2 d;
        const float2 y = __fmul2_rn(x, ACT == ANAKIN_ACT_SILU ? sigmoid<FINE>(x) : normal<FINE>(x, d));
        return make_float2(x.x == -INFINITY ? 0.f : y.x, x.y == -INFINITY ? 0.f : y.y);
    }
    auto one = [](float v) { return ACT == ANAKIN_ACT_RELU ? (v > 0.f ? v : v != v ? v : 0.f) : v; };
    return make_float2(one(x.x), one(x.y));
}
template <bool FINE, int ACT> __device__ __forceinline__ float2 slope_of(float2 x) {
    if (ACT == ANAKIN_ACT_SILU) {
        const float2 g = sigmoid<FINE>(x);
        return __ffma2_rn(__fmul2_rn(x, g), make_float2(1.f - g.x, 1.f - g.y), g);
    }
    if (ACT == ANAKIN_ACT_GELU) {
        float2 d;
        const float2 n = normal<FINE>(x, d);
        return __ffma2_rn(__fmul2_rn(x, both(0.39894228040143268f)), d, n);
    }
    auto one = [](float v) { return ACT == ANAKIN_ACT_RELU ? (v > 0.f ? 1.f : v != v ? v : 0.f) : 1.f; };
    return make_float2(one(x.x), one(x.y));
}

// The smallest E in [-117, 120] with top 2^-E <= 448 = 1.75 2^8, from the bits of top (finite, >= 0).
__device__ __forceinline__ int exponent_of(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = (int)(u >> 23) - 127;  // (zero and subnormals: -127, below every limit)
    const int E = e - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return E < kMinExp ? kMinExp : E;  // (never above 120: e <= 127)
}

// A piece as it lies in memory: 16 bytes of a 16-bit type, 32 of fp32.
template <class T> struct Raw { uint4 v[sizeof(T) / 2]; };
// Eight columns of a row from column j on; what lies behind the row reads as zeros.
template <class T> __device__ __forceinline__ Raw<T> load_piece(const void* base, long long ld, uint32_t r, uint32_t j, int cols, bool vec) {
    const T* row = static_cast<const T*>(base) + (long long)r * ld;
    Raw<T> x;
    if (vec && (int)j + 8 <= cols) {
        const uint4* p = reinterpret_cast<const uint4*>(row + j);
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) x.v[k] = p[k];
    } else {
        T e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = (int)j + i < cols ? row[j + i] : from_f<T>(0.f);
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) x.v[k] = reinterpret_cast<const uint4*>(e)[k];
    }
    return x;
}
// The pieces of a warp's 32 lanes (none with in = false), all lanes together.  Where rows do not start on 16-byte boundaries (STAGED) they go element by
// element, neighbouring lanes neighbouring elements, through 32 pieces of shared memory: a lane's own eight elements would touch sixteen
// sectors a store instruction, a part of each (200000 x 777 bf16 unpacked: 445 us, this way 128; loads gain nothing by it).
template <class T, bool STAGED>
__device__ __forceinline__ void store_pieces(void* base, long long ld, uint32_t r, uint32_t j, bool in, int cols, T* stage, const Raw<T>& x) {
    T* row = static_cast<T*>(base) + (long long)r * ld;
    if constexpr (!STAGED) {
        if (!in) return;
        if ((int)j + 8 <= cols) {
            uint4* p = reinterpret_cast<uint4*>(row + j);
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) p[k] = x.v[k];
        } else {
            T e[8];
#pragma unroll
            for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<uint4*>(e)[k] = x.v[k];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if ((int)j + i < cols) row[j + i] = e[i];
        }
    } else {
        const int lane = threadIdx.x & 31, width = in ? min(cols - (int)j, 8) : 0;
        T* to = row + j;
#pragma unroll
        for (int k = 0; k < (int)sizeof(T) / 2; ++k) reinterpret_cast<uint4*>(stage)[lane * (sizeof(T) / 2) + k] = x.v[k];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 8; ++i) {  // elements 32 i + lane of the 256: of piece 4 i + lane / 8
            const int src = 4 * i + (lane >> 3);
            T* p = reinterpret_cast<T*>(__shfl_sync(0xFFFFFFFFu, (unsigned long long)to, src));
            const int w = __shfl_sync(0xFFFFFFFFu, width, src);
            if ((lane & 7) < w) p[lane & 7] = stage[32 * i + lane];
        }
        __syncwarp();
    }
}
template <class T> __device__ __forceinline__ void floats_of(const Raw<T>& r, float (&f)[8]) {
    if constexpr (sizeof(T) == 4) {
        const uint32_t w[8] = {r.v[0].x, r.v[0].y, r.v[0].z, r.v[0].w, r.v[1].x, r.v[1].y, r.v[1].z, r.v[1].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
    } else {
        tok::unpack16(r.v[0], f, (const T*)nullptr);
    }
}
template <class T> __device__ __forceinline__ Raw<T> raw_of(const float (&f)[8]) {
    Raw<T> r;
    if constexpr (sizeof(T) == 4) {
        r.v[0] = make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
        r.v[1] = make_uint4(__float_as_uint(f[4]), __float_as_uint(f[5]), __float_as_uint(f[6]), __float_as_uint(f[7]));
    } else {
        r.v[0] = tok::pack16(f, (const T*)nullptr);
    }
    return r;
}
// The largest |x| of a piece, infinities included, NaN passed over; 16-bit types two at a time.
template <class T> __device__ __forceinline__ float largest(const Raw<T>& r) {
    if constexpr (sizeof(T) == 4) {
        float f[8], top = 0.f;
        floats_of(r, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]));
        return top;
    } else {
        using P = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        auto abs2 = [](uint32_t w) { w &= 0x7FFF7FFFu; return *reinterpret_cast<const P*>(&w); };
        const uint4& u = r.v[0];
        const P m = __hmax2(__hmax2(abs2(u.x), abs2(u.y)), __hmax2(abs2(u.z), abs2(u.w)));
        return fmaxf(fmaxf(to_f(m.x), to_f(m.y)), 0.f);
    }
}

template <class T, int ACT, bool STAGED>
__global__ void __launch_bounds__(256) k_ckpt_forward(Args a) {
    pdl_wait();
    constexpr int U = 2;
    __shared__ __align__(16) T stages[STAGED ? 8 : 1][256];
    T* stage = stages[STAGED ? threadIdx.x >> 5 : 0];
    // (a warp's lanes stay together: four of them share a block's largest value; `pieces` is a multiple of 4)
    for (uint32_t p0 = blockIdx.x * 256u * U + (threadIdx.x & ~31u); p0 < a.pieces; p0 += gridDim.x * 256u * U) {
        Raw<T> x[U];
        uint32_t r[U], j[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t p = p0 + 256u * u + (threadIdx.x & 31);
            in[u] = p < a.pieces;
            r[u] = a.per_row.div(in[u] ? p : 0u);
            j[u] = ((in[u] ? p : 0u) - r[u] * a.per_row.d) * 8;
            x[u] = load_piece<T>(a.x, a.ldx, r[u], j[u], a.cols, a.vec_x);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float top = largest(x[u]), f[8];
            floats_of(x[u], f);
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            const bool odd = __any_sync(0xFFFFFFFFu, !(top < 2.6584559e36f));  // 2^121: an infinity in the block, or values near fp32's largest
            if (odd) {  // the largest finite value
                top = 0.f;
#pragma unroll
                for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(f[i]) < INFINITY ? fabsf(f[i]) : 0.f);
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
                top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
            }
            const int E = exponent_of(top);
            const float down = __uint_as_float((uint32_t)(127 - E) << 23);  // 2^-E: E in [-117, 120]
            uint32_t w[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                uint32_t c[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float x0 = f[4 * h + 2 * i], x1 = f[4 * h + 2 * i + 1];
                    float2 v = __fmul2_rn(make_float2(x0, x1), make_float2(down, down));
                    if (odd && E == kMaxExp) {  // (256 times 2^120 would be past the largest fp32 number)
                        v.x = v.x > 240.f ? 240.f : v.x < -240.f ? -240.f : v.x;
                        v.y = v.y > 240.f ? 240.f : v.y < -240.f ? -240.f : v.y;
                    }
                    c[i] = __nv_cvt_float2_to_fp8x2(v, __NV_SATFINITE, __NV_E4M3);  // (NaN: 0x7F)
                    if (odd) {
                        if (!(fabsf(x0) < INFINITY)) c[i] = (c[i] & 0xFF00u) | 0x7Fu;
                        if (!(fabsf(x1) < INFINITY)) c[i] = (c[i] & 0x00FFu) | 0x7F00u;
                    }
                }
                w[h] = __byte_perm(c[0], c[1], 0x5410);
            }
            if (in[u]) {
                *reinterpret_cast<uint2*>(a.codes + (size_t)r[u] * a.blocks * 32 + j[u]) = make_uint2(w[0], w[1]);
                if ((threadIdx.x & 3) == 0) a.scales[(size_t)r[u] * a.blocks + j[u] / 32] = (uint8_t)(E + 127);
            }
            if (a.y) {
                if (ACT != ANAKIN_ACT_IDENTITY) {
                    float g[8];
#pragma unroll
                    for (int i = 0; i < 8; i += 2) {
                        const float2 v = act_of<sizeof(T) == 4, ACT>(make_float2(f[i], f[i + 1]));
                        g[i] = v.x;
                        g[i + 1] = v.y;
                    }
                    x[u] = raw_of<T>(g);
                }
                store_pieces<T, STAGED>(a.y, a.ldy, r[u], j[u], in[u], a.cols, stage, x[u]);
            }
        }
    }
}

template <class T> __device__ __forceinline__ float within(float v) { return v; }
template <> __device__ __forceinline__ float within<__half>(float v) { return v > 65504.f ? 65504.f : v < -65504.f ? -65504.f : v; }

// Unpack (BACK = false): y = the kept values; BACK: y = x act'(kept).  Four pieces of a thread in flight, with dy's 32 bytes of fp32 two.
template <class T, int ACT, bool BACK, bool STAGED>
__global__ void __launch_bounds__(256) k_ckpt_read(Args a) {
    pdl_wait();
    constexpr int U = BACK && sizeof(T) == 4 ? 2 : 4;
    __shared__ __align__(16) T stages[STAGED ? 8 : 1][256];
    T* stage = stages[STAGED ? threadIdx.x >> 5 : 0];
    for (uint32_t p0 = blockIdx.x * 256u * U + (threadIdx.x & ~31u); p0 < a.pieces; p0 += gridDim.x * 256u * U) {
        uint2 c[U];
        Raw<T> d[U];
        uint32_t r[U], j[U], s[U];
        bool in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t p = p0 + 256u * u + (threadIdx.x & 31);
            in[u] = p < a.pieces;
            r[u] = a.per_row.div(in[u] ? p : 0u);
            j[u] = ((in[u] ? p : 0u) - r[u] * a.per_row.d) * 8;
            c[u] = *reinterpret_cast<const uint2*>(a.codes + (size_t)r[u] * a.blocks * 32 + j[u]);
            s[u] = a.scales[(size_t)r[u] * a.blocks + j[u] / 32];
            if (BACK) d[u] = load_piece<T>(a.x, a.ldx, r[u], j[u], a.cols, a.vec_x);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float v[8], f[8];
            decode8(c[u], s[u], v);
            if (BACK) floats_of(d[u], f);
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                if (BACK) {
                    const float2 g = __fmul2_rn(make_float2(f[i], f[i + 1]), slope_of<sizeof(T) == 4, ACT>(make_float2(v[i], v[i + 1])));
                    v[i] = g.x;
                    v[i + 1] = g.y;
                } else {
                    v[i] = within<T>(v[i]);
                    v[i + 1] = within<T>(v[i + 1]);
                }
            }
            store_pieces<T, STAGED>(a.y, a.ldy, r[u], j[u], in[u], a.cols, stage, raw_of<T>(v));
        }
    }
}

enum { FORWARD = 0, UNPACK = 1, BACKWARD = 2 };

template <class T, int ACT, int MODE, bool STAGED>
cudaError_t launch_with(const Args& a, cudaStream_t s) {
    const uint32_t n = (a.pieces + 511) / 512;
    const dim3 grid(n < 148u * 32 ? n : 148u * 32);
    if constexpr (MODE == FORWARD) return launch<k_ckpt_forward<T, ACT, STAGED>>(grid, dim3(256), 0, s, a);
    else return launch<k_ckpt_read<T, ACT, MODE == BACKWARD, STAGED>>(grid, dim3(256), 0, s, a);
}
template <class T, int ACT, int MODE>
cudaError_t launch_one(const Args& a, cudaStream_t s) {
    return a.y && !a.vec_y ? launch_with<T, ACT, MODE, true>(a, s) : launch_with<T, ACT, MODE, false>(a, s);
}
template <class T, int MODE>
cudaError_t launch_act(int act, const Args& a, cudaStream_t s) {
    if constexpr (MODE == UNPACK) return launch_one<T, ANAKIN_ACT_IDENTITY, MODE>(a, s);
    else switch (act) {
        case ANAKIN_ACT_RELU: return launch_one<T, ANAKIN_ACT_RELU, MODE>(a, s);
        case ANAKIN_ACT_SILU: return launch_one<T, ANAKIN_ACT_SILU, MODE>(a, s);
        case ANAKIN_ACT_GELU: return launch_one<T, ANAKIN_ACT_GELU, MODE>(a, s);
        default: return launch_one<T, ANAKIN_ACT_IDENTITY, MODE>(a, s);
    }
}

// A launch covers fewer than 2^31 pieces; a larger matrix takes several, each a range of rows.
template <int MODE>
int run(int dtype, int act, long long rows, long long cols, const void* x, long long ldx, void* y, long long ldy, uint8_t* codes, uint8_t* scales,
        cudaStream_t s) {
    const size_t es = dtype == ANAKIN_DTYPE_F32 ? 4 : 2;
    Args a;
    a.cols = (int)cols;
    a.blocks = (int)((cols + 31) / 32);
    a.per_row = FastDiv((uint32_t)a.blocks * 4);
    a.vec_x = ((uintptr_t)x & 15) == 0 && ldx * es % 16 == 0;
    a.vec_y = ((uintptr_t)y & 15) == 0 && ldy * es % 16 == 0;
    // (the last CTA's pieces, and a step of the whole grid, stay below 2^32)
    const long long most = ((1ll << 31) - 1) / ((long long)a.blocks * 4);
    for (long long r0 = 0; r0 < rows; r0 += most) {
        const long long n = rows - r0 < most ? rows - r0 : most;
        a.rows = n;
        a.pieces = (uint32_t)(n * a.blocks * 4);
        a.x = static_cast<const unsigned char*>(x) + (x ? (size_t)r0 * ldx * es : 0);
        a.ldx = ldx;
        a.y = y ? static_cast<unsigned char*>(y) + (size_t)r0 * ldy * es : nullptr;
        a.ldy = ldy;
        a.codes = codes + (size_t)r0 * a.blocks * 32;
        a.scales = scales + (size_t)r0 * a.blocks;
        const cudaError_t e = dtype == ANAKIN_DTYPE_F32 ? launch_act<float, MODE>(act, a, s)
                              : dtype == ANAKIN_DTYPE_BF16 ? launch_act<__nv_bfloat16, MODE>(act, a, s) : launch_act<__half, MODE>(act, a, s);
        if (e != cudaSuccess) return tok::fail();
    }
    return ANAKIN_OK;
}

}  // namespace

int check(int dtype, int act, int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales) {
    if (dtype < ANAKIN_DTYPE_F32 || dtype > ANAKIN_DTYPE_F16 || act < ANAKIN_ACT_IDENTITY || act > ANAKIN_ACT_GELU) return ANAKIN_E_INVALID_ARG;
    if (rows < 0 || cols < 1 || rows >= (int64_t(1) << 31) || cols > (int64_t(1) << 28)) return ANAKIN_E_INVALID_ARG;
    if (rows > 0 && (!codes || !scales || ((uintptr_t)codes & 15))) return ANAKIN_E_INVALID_ARG;
    return ANAKIN_OK;
}

}  // namespace ckpt
}  // namespace anakin

using namespace anakin;

static bool bad_matrix(int dtype, int64_t rows, int64_t cols, const void* p, int64_t ld) {
    return rows > 0 && (!p || ((uintptr_t)p & (dtype == ANAKIN_DTYPE_F32 ? 3 : 1)) || ld < cols || ld >= (int64_t(1) << 40));
}

extern "C" {

int anakin_ckpt_bytes(int64_t rows, int64_t cols, size_t* code_bytes, size_t* scale_bytes) {
    if (!code_bytes || !scale_bytes || rows < 0 || cols < 1 || rows >= (int64_t(1) << 31) || cols > (int64_t(1) << 28)) return ANAKIN_E_INVALID_ARG;
    const size_t blocks = (size_t)((cols + 31) / 32);
    *code_bytes = (size_t)rows * blocks * 32;
    *scale_bytes = (size_t)rows * blocks;
    return ANAKIN_OK;
}

int anakin_ckpt_forward(int dtype, int act, int64_t rows, int64_t cols, const void* x, int64_t ldx, void* y, int64_t ldy, uint8_t* codes,
                        uint8_t* scales, void* cuda_stream) {
    const int rc = ckpt::check(dtype, act, rows, cols, codes, scales);
    if (rc != ANAKIN_OK) return rc;
    if (bad_matrix(dtype, rows, cols, x, ldx) || (y && bad_matrix(dtype, rows, cols, y, ldy))) return ANAKIN_E_INVALID_ARG;
    return ckpt::run<ckpt::FORWARD>(dtype, act, rows, cols, x, ldx, y, ldy, codes, scales, (cudaStream_t)cuda_stream);
}

int anakin_ckpt_unpack(int dtype, int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales, void* x, int64_t ldx, void* cuda_stream) {
    const int rc = ckpt::check(dtype, ANAKIN_ACT_IDENTITY, rows, cols, codes, scales);
    if (rc != ANAKIN_OK) return rc;
    if (bad_matrix(dtype, rows, cols, x, ldx)) return ANAKIN_E_INVALID_ARG;
    return ckpt::run<ckpt::UNPACK>(dtype, 0, rows, cols, nullptr, 0, x, ldx, const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), (cudaStream_t)cuda_stream);
}

int anakin_ckpt_backward(int dtype, int act, int64_t rows, int64_t cols, const uint8_t* codes, const uint8_t* scales, const void* dy,
                         int64_t lddy, void* dx, int64_t lddx, void* cuda_stream) {
    const int rc = ckpt::check(dtype, act, rows, cols, codes, scales);
    if (rc != ANAKIN_OK) return rc;
    if (bad_matrix(dtype, rows, cols, dy, lddy) || bad_matrix(dtype, rows, cols, dx, lddx)) return ANAKIN_E_INVALID_ARG;
    return ckpt::run<ckpt::BACKWARD>(dtype, act, rows, cols, dy, lddy, dx, lddx, const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), (cudaStream_t)cuda_stream);
}

}  // extern "C"
