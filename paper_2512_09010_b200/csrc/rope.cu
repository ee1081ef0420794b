// Rotary positions: the pairs (x_a, x_b) of a head's first `rotary` elements are turned by the token's position,
//
//   y_a = f (x_a cos t - x_b sin t),   y_b = f (x_a sin t + x_b cos t),   t = position * freq,
//
// the inverse turn by -t.  f R(-t) is the transpose of f R(t), so the gradient of x is the inverse turn of the gradient of y.
//
// Bound.  Every element is read and written once, with a sine and a cosine for a pair that all heads of a token share: HBM, once there
// are enough tokens.  16384 tokens of 40 heads of 128 (bf16, 336 MB): 57 us, 0.90 of the copy rate (two CTAs of an SM instead of three,
// with twice the tokens: 63); the smallest calls are a chain of latencies
// (launch, position, sine, row).
//
// Angles.  A position of a long context times a frequency near 1 has more turns than a float has bits for the rest: the turns,
// t / (2 pi), are formed in 64 bits, their whole part is dropped exactly, and what is left goes to sincospif in 32.  An
// angle is off by 2^-23 radians and 2^-52 of itself at most.
//
// Split.  A CTA takes a few tokens and forms their table of sines and cosines in shared memory; the first rows are on their way
// meanwhile.  A thread keeps its place in a token's row, W elements and their partners, and takes one token after the other, four
// at a time, so that places are found by a division once; the number of threads follows from the row, so that few are idle.

#include <cuda_bf16.h>

#include "luvc_internal.h"
#include "sm100_ptx.cuh"

namespace luvc {
namespace {

using namespace ptx;

constexpr int kRopeBatch = 4;               // tokens whose rows a thread has in flight
constexpr int kRopeTable = 2048;            // pairs of all tokens of a CTA (16 KB)

struct RopeArgs {
    const void* x;
    void* out;
    long long x_stride, out_stride, position_stride;
    const int32_t* positions;
    const float* freqs;
    const int32_t* axis;
    int axes, tokens, heads, D, half, per;  // half: pairs of a head; per: tokens of a CTA
    int cols, step;                         // places of a token's row a sweep takes, tokens side by side
    float factor, sign;                     // sign: of the sine
};

// W elements of type T as floats, and back.
template <typename T, int W> struct Piece;
template <int W> struct Piece<float, W> {
    float v[W];
    __device__ void load(const float* p) {
        if constexpr (W == 4) *reinterpret_cast<float4*>(v) = __ldcs(reinterpret_cast<const float4*>(p));
        else if constexpr (W == 2) *reinterpret_cast<float2*>(v) = __ldcs(reinterpret_cast<const float2*>(p));
        else v[0] = __ldcs(p);
    }
    __device__ float get(int i) const { return v[i]; }
    __device__ static void store(float* p, const float (&f)[W]) {
        if constexpr (W == 4) __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
        else if constexpr (W == 2) __stcs(reinterpret_cast<float2*>(p), make_float2(f[0], f[1]));
        else __stcs(p, f[0]);
    }
};
template <int W> struct Piece<__nv_bfloat16, W> {
    unsigned v[W > 1 ? W / 2 : 1];
    __device__ void load(const __nv_bfloat16* p) {
        if constexpr (W == 8) {
            const uint4 x = __ldcs(reinterpret_cast<const uint4*>(p));
            v[0] = x.x; v[1] = x.y; v[2] = x.z; v[3] = x.w;
        } else if constexpr (W == 4) {
            const uint2 x = __ldcs(reinterpret_cast<const uint2*>(p));
            v[0] = x.x; v[1] = x.y;
        } else if constexpr (W == 2) {
            v[0] = __ldcs(reinterpret_cast<const unsigned*>(p));
        } else {
            v[0] = __ldcs(reinterpret_cast<const unsigned short*>(p));
        }
    }
    __device__ float get(int i) const { return __uint_as_float(i & 1 ? v[i >> 1] & 0xffff0000u : v[i >> 1] << 16); }
    __device__ static void store(__nv_bfloat16* p, const float (&f)[W]) {
        if constexpr (W == 1) {
            *p = __float2bfloat16_rn(f[0]);
        } else {
            unsigned r[W / 2];
#pragma unroll
            for (int i = 0; i < W / 2; ++i) {
                const __nv_bfloat162 two = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                r[i] = *reinterpret_cast<const unsigned*>(&two);
            }
            if constexpr (W == 8) __stcs(reinterpret_cast<uint4*>(p), make_uint4(r[0], r[1], r[2], r[3]));
            else if constexpr (W == 4) __stcs(reinterpret_cast<uint2*>(p), make_uint2(r[0], r[1]));
            else __stcs(reinterpret_cast<unsigned*>(p), r[0]);
        }
    }
};

// INTER: pairs are neighbours, a piece holds W / 2 of them; else a piece of W elements has its partners `half` elements on.  Places past
// the pairs are copied.
template <typename T, int W, bool INTER>
__global__ void __launch_bounds__(384, 3) rope_kernel(const __grid_constant__ RopeArgs a) {
    // (cos, sin) times the factor, of each token's pairs: pair k of all pieces side by side, so that threads next to one another meet
    // no bank twice
    __shared__ float2 table[kRopeTable];
    constexpr int NP = INTER ? W / 2 : W;                   // pairs of a piece
    const int t0 = blockIdx.x * a.per, tokens = min(a.per, a.tokens - t0);
    const int turned = (INTER ? 2 * a.half : a.half) / W, places = turned + (a.D - 2 * a.half) / W, row = a.heads * places;
    const int mine = threadIdx.x / a.cols;
    const T* const x = static_cast<const T*>(a.x);
    T* const out = static_cast<T*>(a.out);
    pdl_trigger();
    pdl_wait();
    Piece<T, W> lo[kRopeBatch], hi[kRopeBatch];
    auto fetch = [&](long long at, bool pair, int t) {
#pragma unroll
        for (int b = 0; b < kRopeBatch; ++b)
            if (t + b * a.step < tokens) {
                const T* const p = x + (t0 + t + b * a.step) * a.x_stride + at;
                lo[b].load(p);
                if (!INTER && pair) hi[b].load(p + a.half);
            }
    };
    // the element of column `col` of a row, and which of the head's pieces that is (-1: copied)
    const int pieces = a.half / NP;
    auto place = [&](int col, int& piece) {
        const int h = col / places, i = col - h * places;
        piece = i < turned ? i : -1;
        return (long long)h * a.D + (i < turned ? i * W : 2 * a.half + (i - turned) * W);
    };
    const int col0 = threadIdx.x - mine * a.cols;
    int piece;
    long long at = place(col0, piece);
    if (mine < a.step) fetch(at, piece >= 0, mine);

    for (int e = threadIdx.x; e < tokens * a.half; e += blockDim.x) {
        const int t = e / a.half, i = e - t * a.half;
        const int which = a.axis ? min(max(a.axis[i], 0), a.axes - 1) : 0;
        const double turns = (double)a.positions[which * a.position_stride + t0 + t] * ((double)a.freqs[i] * 0.15915494309189533577);
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        table[t * a.half + i % NP * pieces + i / NP] = make_float2(c * a.factor, s * (a.factor * a.sign));
    }
    __syncthreads();
    if (mine >= a.step) return;
    for (int col = col0; col < row; col += a.cols) {
        if (col != col0) at = place(col, piece);
        if (piece < 0 && a.out == a.x) continue;
        for (int t = mine; t < tokens; t += kRopeBatch * a.step) {
            if (col != col0 || t != mine) fetch(at, piece >= 0, t);
#pragma unroll
            for (int b = 0; b < kRopeBatch; ++b) {
                const int j = t + b * a.step;
                if (j >= tokens) continue;
                T* const p = out + (t0 + j) * a.out_stride + at;
                const float2* const cs = table + j * a.half + piece;
                float f[W], g[W];
                if (piece < 0) {
#pragma unroll
                    for (int i = 0; i < W; ++i) f[i] = lo[b].get(i);
                } else if constexpr (INTER) {
#pragma unroll
                    for (int i = 0; i < W / 2; ++i) {
                        const float2 w = cs[i * pieces];
                        const float u = lo[b].get(2 * i), v = lo[b].get(2 * i + 1);
                        f[2 * i] = fmaf(u, w.x, -(v * w.y));
                        f[2 * i + 1] = fmaf(u, w.y, v * w.x);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const float2 w = cs[i * pieces];
                        const float u = lo[b].get(i), v = hi[b].get(i);
                        f[i] = fmaf(u, w.x, -(v * w.y));
                        g[i] = fmaf(u, w.y, v * w.x);
                    }
                    Piece<T, W>::store(p + a.half, g);
                }
                Piece<T, W>::store(p, f);
            }
        }
    }
}

template <typename T, int W, bool INTER>
int launch(RopeArgs& a, cudaStream_t stream) {
    const int sms = sm_count();
    if (!sms) return LUVC_ERR_CUDA;
    const long long row = (long long)a.heads * ((INTER ? 2 * a.half : a.half) / W + (a.D - 2 * a.half) / W);
    // threads: a row in equal sweeps of up to 384 places, or several tokens side by side where it is short
    const long long sweeps = (row + 383) / 384;
    a.cols = (int)((row + sweeps - 1) / sweeps);
    a.step = a.cols >= 256 ? 1 : 256 / a.cols;
    const int threads = (a.cols * a.step + 31) / 32 * 32;
    // tokens of a CTA: one round of loads each, fewer while that leaves SMs without work, as many as the table has room for
    const long long even = ((long long)a.tokens + 2 * sms - 1) / (2 * sms);
    const int most = kRopeTable / a.half, full = kRopeBatch * a.step;
    a.per = (int)(even < full ? even : full);
    if (a.per > most) a.per = most;
    return launch_overlapped(rope_kernel<T, W, INTER>, (unsigned)((a.tokens - 1) / a.per + 1), threads, 0, stream, a);
}

// The widest pieces that pairs, and what is behind them, divide into.
template <typename T, bool INTER>
int launch_width(RopeArgs& a, cudaStream_t stream) {
    const int n = INTER ? 2 * a.half : a.half;
    if constexpr (sizeof(T) == 2)
        if (n % 8 == 0) return launch<T, 8, INTER>(a, stream);
    if (n % 4 == 0) return launch<T, 4, INTER>(a, stream);
    if constexpr (INTER) return launch<T, 2, INTER>(a, stream);
    else return n % 2 == 0 ? launch<T, 2, INTER>(a, stream) : launch<T, 1, INTER>(a, stream);
}

}  // namespace

int rope(const RopeProblem& p) {
    RopeArgs a;
    a.x = p.x; a.out = p.out; a.x_stride = p.x_stride; a.out_stride = p.out_stride; a.position_stride = p.position_stride;
    a.positions = p.positions; a.freqs = p.freqs; a.axis = p.axis; a.axes = p.axes; a.tokens = p.tokens; a.heads = p.heads; a.D = p.D;
    a.half = p.rotary / 2; a.factor = p.factor; a.sign = p.inverse ? -1.f : 1.f;
    if (p.dtype == LUVC_F32)
        return p.interleaved ? launch_width<float, true>(a, p.stream) : launch_width<float, false>(a, p.stream);
    return p.interleaved ? launch_width<__nv_bfloat16, true>(a, p.stream) : launch_width<__nv_bfloat16, false>(a, p.stream);
}

}  // namespace luvc
