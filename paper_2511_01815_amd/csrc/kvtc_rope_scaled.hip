// Rotary positions of part of every head, with scaled frequencies, from one tensor into another or in place, for gfx950.
//
// Of a head's features the first n_rotated turn, in pairs (a, b), pair j of the token at position m by m theta_j, and are multiplied by g:
//     a' = g (a cos - b sin),  b' = g (a sin + b cos)      (undoing it: the opposite angle, and 1 / g);
// the others are copied.  The frequencies theta_j are the caller's form, worked out once (kvtc_rope_form_init).
//
// Angles, sines and cosines are double precision -- an angle reaches 10^6 radians -- and rounded to fp32, the rotation is one product and one fused product in fp32, rounded once more to bf16.
// A workgroup has some tokens: first it works out their sines and cosines, one to a thread, into the LDS, for all heads; then threads take units of two pieces, the a's and the b's of
// some neighbouring pairs, of up to 16 bytes each.  Large calls are bound by memory (20001 tokens of 12 heads of 64 in fp32, 123 MB: 30.5 us, 4.0 TB/s), small ones by the launch and the double precision
// (64 tokens of 40 heads: 4.2 us in the kernel).
#include <hip/hip_runtime.h>
#include <cmath>
#include <cstring>
#include "kvtc_cache.h"
#include "kvtc_dev.h"
#include "kvtc_sincos.h"

namespace kvtc {
kvtc_status set_error(kvtc_status st, const char* fmt, ...);

constexpr int kTurns = 2048;                               // sines and cosines of a workgroup, at most

struct RopeScaledArgs {
    const void* x;
    void* out;
    int64_t x_token, x_head, out_token, out_head;          // strides in elements
    const int32_t* positions;
    int64_t position0;
    int64_t n_tokens, blocks;                              // blocks: of tokens_each tokens
    int32_t n_heads, half, tokens_each, heads_each;        // of a workgroup
    int32_t turning, units;                                // units of a head that turn; and all, with those that are copied
    int32_t heads_first;                                   // a head's tokens lie nearer to each other than a token's heads
    float sine_factor, cosine_factor;
    double theta[128];
};

template <typename XT, int E> struct Piece;
template <int E> struct Piece<float, E> { typedef float type __attribute__((ext_vector_type(E))); };
template <> struct Piece<float, 1> { typedef float type; };
template <int E> struct Piece<uint16_t, E> { typedef uint16_t type __attribute__((ext_vector_type(E))); };
template <> struct Piece<uint16_t, 1> { typedef uint16_t type; };
template <int E, typename V> __device__ __forceinline__ auto& element(V& v, int i) {
    if constexpr (E == 1) return v;
    else return reinterpret_cast<std::remove_reference_t<decltype(v[0])>*>(&v)[i];
}

// E features to a piece; half layout: pieces of the a's and of the b's; interleaved: two neighbouring pieces.
template <typename XT, int E, bool INTERLEAVED>
__global__ void __launch_bounds__(256) rope_scaled_kernel(const RopeScaledArgs a) {
    union Held {
        XT e[E];
        typename Piece<XT, E>::type v;
    };
    __shared__ float2 turns[kTurns];                       // cosine, sine
    for (int64_t block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        const int64_t token0 = block * a.tokens_each;
        const int tokens = (int)min((int64_t)a.tokens_each, a.n_tokens - token0), head0 = (int)blockIdx.y * a.heads_each, heads = min(a.heads_each, a.n_heads - head0);
        const uint32_t n = (uint32_t)tokens * (uint32_t)heads * (uint32_t)a.units;
        for (int i = threadIdx.x; i < tokens * a.half; i += 256) {
            const int t = i / a.half, j = i - t * a.half;
            const double position = (double)(a.positions ? (int64_t)a.positions[token0 + t] : a.position0 + token0 + t), angle = position * a.theta[j];
            double s, c;
            if (fabs(angle) <= 0x1p31) sincos_reduced(angle, &s, &c);
            else sincos(angle, &s, &c);
            turns[i] = make_float2((float)(c * a.cosine_factor), (float)(s * a.sine_factor));
        }
        __syncthreads();
        const XT* x = static_cast<const XT*>(a.x) + token0 * a.x_token + (int64_t)head0 * a.x_head;
        XT* out = static_cast<XT*>(a.out) + token0 * a.out_token + (int64_t)head0 * a.out_head;
        for (uint32_t i = threadIdx.x; i < n; i += 256) {
            const uint32_t row = i / (uint32_t)a.units, u = i - row * (uint32_t)a.units;
            uint32_t t, h;
            if (a.heads_first) { h = row / (uint32_t)tokens; t = row - h * (uint32_t)tokens; }
            else { t = row / (uint32_t)heads; h = row - t * (uint32_t)heads; }
            const bool turn = u < (uint32_t)a.turning;
            const int first = turn && !INTERLEAVED ? (int)u * E : (int)u * 2 * E, second = first + (turn && !INTERLEAVED ? a.half : E);
            const XT* from = x + (int64_t)t * a.x_token + (int64_t)h * a.x_head;
            XT* to = out + (int64_t)t * a.out_token + (int64_t)h * a.out_head;
            Held p, q;
            p.v = *reinterpret_cast<const typename Piece<XT, E>::type*>(from + first);
            q.v = *reinterpret_cast<const typename Piece<XT, E>::type*>(from + second);
            if (turn) {
                const float2* cs = turns + t * a.half + u * E;
    #pragma unroll
                for (int k = 0; k < E; ++k) {
                    // pair k of the unit: (p[k], q[k]), or neighbours of the 2 E features
                    XT& ea = INTERLEAVED ? (2 * k < E ? p.e[2 * k % E] : q.e[2 * k % E]) : p.e[k];
                    XT& eb = INTERLEAVED ? (2 * k + 1 < E ? p.e[(2 * k + 1) % E] : q.e[(2 * k + 1) % E]) : q.e[k];
                    float va, vb;
                    if constexpr (sizeof(XT) == 2) { va = bf16_f32(ea); vb = bf16_f32(eb); }
                    else { va = ea; vb = eb; }
                    const float2 w = cs[k];
                    const float ra = __builtin_fmaf(va, w.x, -(vb * w.y)), rb = __builtin_fmaf(va, w.y, vb * w.x);
                    if constexpr (sizeof(XT) == 2) { ea = f32_bf16(ra); eb = f32_bf16(rb); }
                    else { ea = ra; eb = rb; }
                }
            }
            *reinterpret_cast<typename Piece<XT, E>::type*>(to + first) = p.v;
            *reinterpret_cast<typename Piece<XT, E>::type*>(to + second) = q.v;
        }
        __syncthreads();                                   // (the next block's turns take these's place)
    }
}

template <typename XT, int E>
static void launch_rope_pieces(const RopeScaledArgs& a, bool interleaved, dim3 grid, hipStream_t stream) {
    if (interleaved) hipLaunchKernelGGL((rope_scaled_kernel<XT, E, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((rope_scaled_kernel<XT, E, false>), grid, dim3(256), 0, stream, a);
}

static hipError_t launch_rope_scaled(RopeScaledArgs& a, kvtc_dtype dtype, int n_rotated, int copied, bool interleaved, hipStream_t stream) {
    // the largest pieces that sizes, strides and addresses allow
    const int size = dtype == KVTC_BF16 ? 2 : 4;
    int e = 16 / size;
    const uint64_t multiple = (uint64_t)a.x_token | (uint64_t)a.x_head | (uint64_t)a.out_token | (uint64_t)a.out_head | (reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.out)) / size;
    while (e > 1 && (n_rotated % (2 * e) != 0 || copied % (2 * e) != 0 || multiple % e != 0)) e /= 2;
    a.turning = n_rotated / (2 * e);
    a.units = a.turning + copied / (2 * e);
    // tokens of a workgroup: some units to a thread, and a workgroup to every compute unit before that
    const int64_t row = (int64_t)a.n_heads * a.units;
    int64_t each = (1024 + row - 1) / row, spread = (a.n_tokens * row + (int64_t)compute_units() * 256 - 1) / ((int64_t)compute_units() * 256) * 256 / row;
    if (each > spread) each = spread;
    if (each > kTurns / a.half) each = kTurns / a.half;
    a.tokens_each = (int)(each < 1 ? 1 : each);
    const int64_t blocks = a.blocks = (a.n_tokens + a.tokens_each - 1) / a.tokens_each, at_once = (int64_t)1 << 20;
    int64_t shares = 1;                                    // of a token's heads
    while (shares < a.n_heads && blocks * shares < compute_units() && row * a.tokens_each > 512 * shares) shares *= 2;
    a.heads_each = (int)((a.n_heads + shares - 1) / shares);
    const dim3 grid((uint32_t)(blocks < at_once ? blocks : at_once), (uint32_t)((a.n_heads + a.heads_each - 1) / a.heads_each));
    if (dtype == KVTC_BF16) {
        if (e == 8) launch_rope_pieces<uint16_t, 8>(a, interleaved, grid, stream);
        else if (e == 4) launch_rope_pieces<uint16_t, 4>(a, interleaved, grid, stream);
        else if (e == 2) launch_rope_pieces<uint16_t, 2>(a, interleaved, grid, stream);
        else launch_rope_pieces<uint16_t, 1>(a, interleaved, grid, stream);
    } else {
        if (e == 4) launch_rope_pieces<float, 4>(a, interleaved, grid, stream);
        else if (e == 2) launch_rope_pieces<float, 2>(a, interleaved, grid, stream);
        else launch_rope_pieces<float, 1>(a, interleaved, grid, stream);
    }
    return hipGetLastError();
}

}  // namespace kvtc

extern "C" {

kvtc_status kvtc_rope_form_init(kvtc_rope_form* out, int n_rotated, kvtc_rope_pairing pairing, double base, kvtc_rope_scaling scaling, double factor, double original, double low, double high,
                                double magnitude) {
    using namespace kvtc;
    if (!out) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: null form");
    if (n_rotated < 2 || n_rotated > 256 || n_rotated % 2 != 0) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: n_rotated=%d must be even, in 2..256", n_rotated);
    if (pairing != KVTC_ROPE_HALF && pairing != KVTC_ROPE_INTERLEAVED) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: unknown pairing %d", (int)pairing);
    if ((unsigned)scaling > KVTC_ROPE_SCALE_RAMP) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: unknown scaling %d", (int)scaling);
    auto positive = [](double v) { return std::isfinite(v) && v > 0.0; };
    if (!positive(base) || !positive(magnitude) || !std::isfinite((float)magnitude) || !std::isfinite((float)(1.0 / magnitude)) || (float)magnitude == 0.0f)
        return set_error(KVTC_E_ARG, "kvtc_rope_form_init: base and magnitude must be positive and finite, magnitude and its inverse in fp32");
    if (scaling != KVTC_ROPE_SCALE_NONE && !positive(factor)) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: factor must be positive and finite");
    if ((scaling == KVTC_ROPE_SCALE_BANDS || scaling == KVTC_ROPE_SCALE_RAMP) && (!positive(original) || !positive(low) || !positive(high) || !(low < high)))
        return set_error(KVTC_E_ARG, "kvtc_rope_form_init: need original > 0 and 0 < low < high");
    if (scaling == KVTC_ROPE_SCALE_RAMP && !(base > 1.0)) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: a ramp needs a base above 1");
    kvtc_rope_form f;
    memset(&f, 0, sizeof(f));
    f.n_rotated = n_rotated;
    f.pairing = pairing;
    f.magnitude = magnitude;
    const double n = n_rotated, pi2 = 6.283185307179586;
    if (scaling == KVTC_ROPE_SCALE_BASE && n_rotated > 2) base *= std::pow(factor, n / (n - 2.0));
    double first = 0.0, last = 0.0;                        // of the ramp
    if (scaling == KVTC_ROPE_SCALE_RAMP) {
        auto pair_of = [&](double turns) { return n * std::log(original / (turns * pi2)) / (2.0 * std::log(base)); };
        first = std::fmax(std::floor(pair_of(high)), 0.0);
        last = std::fmin(std::ceil(pair_of(low)), n - 1.0);
    }
    for (int j = 0; j < n_rotated / 2; ++j) {
        const double theta = std::pow(base, -2.0 * (double)j / n);
        double kept = 1.0;                                 // share of the frequency that is not divided
        if (scaling == KVTC_ROPE_SCALE_LINEAR) kept = 0.0;
        else if (scaling == KVTC_ROPE_SCALE_BANDS) kept = (original * theta / pi2 - low) / (high - low);
        else if (scaling == KVTC_ROPE_SCALE_RAMP) kept = 1.0 - ((double)j - first) / std::fmax(last - first, 0.001);
        kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
        f.theta[j] = kept == 1.0 ? theta : kept * theta + (1.0 - kept) * theta / factor;
        if (!std::isfinite(f.theta[j])) return set_error(KVTC_E_ARG, "kvtc_rope_form_init: frequency %d is not finite", j);
    }
    *out = f;
    return KVTC_OK;
}

kvtc_status kvtc_rope_scaled(const void* x_dev, void* out_dev, kvtc_dtype dtype, int64_t n_tokens, int n_heads, int d_head, int64_t token_stride, int64_t head_stride, int64_t out_token_stride,
                             int64_t out_head_stride, const int32_t* positions_dev, int64_t position0, const kvtc_rope_form* form, int inverse, kvtc_stream stream) {
    using namespace kvtc;
    if (n_tokens < 0 || n_tokens > 0x7fffffffLL) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: n_tokens=%lld", (long long)n_tokens);
    if (n_heads < 1 || n_heads > kCacheMaxHeads || d_head < 2 || (d_head & 1) || d_head > 256)
        return set_error(KVTC_E_ARG, "kvtc_rope_scaled: need n_heads in 1..%d and an even d_head in 2..256 (n_heads=%d d_head=%d)", kCacheMaxHeads, n_heads, d_head);
    if (dtype != KVTC_BF16 && dtype != KVTC_F32) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: unknown dtype %d", (int)dtype);
    if (!form) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: null form");
    if (form->n_rotated < 2 || form->n_rotated % 2 != 0 || form->n_rotated > d_head || (form->pairing != KVTC_ROPE_HALF && form->pairing != KVTC_ROPE_INTERLEAVED) ||
        !((float)form->magnitude > 0.0f) || !std::isfinite((float)form->magnitude))
        return set_error(KVTC_E_ARG, "kvtc_rope_scaled: a form of %d features for heads of %d, or one that kvtc_rope_form_init has not made", form->n_rotated, d_head);
    if (inverse != 0 && inverse != 1) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: inverse must be 0 or 1");
    if (n_tokens == 0) return KVTC_OK;
    if (!x_dev || !out_dev) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: null buffer");
    const int64_t far = (int64_t)1 << 40, strides[2][2] = {{token_stride, head_stride}, {out_token_stride, out_head_stride}};
    for (const auto& s : strides) {
        const int64_t t = s[0], h = s[1];
        const bool in_range = t >= 0 && t <= far && h >= 0 && h <= far;
        const bool tokens_major = in_range && (n_heads == 1 || h >= d_head) && (n_tokens == 1 || t >= (int64_t)(n_heads - 1) * h + d_head);
        const bool heads_major = in_range && (n_tokens == 1 || t >= d_head) && (n_heads == 1 || (__int128)h >= (__int128)(n_tokens - 1) * t + d_head);
        if (!tokens_major && !heads_major) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: strides (token %lld, head %lld) let elements overlap", (long long)t, (long long)h);
    }
    const uintptr_t size = dtype == KVTC_BF16 ? 2 : 4;
    if (reinterpret_cast<uintptr_t>(x_dev) % size != 0 || reinterpret_cast<uintptr_t>(out_dev) % size != 0 || (reinterpret_cast<uintptr_t>(positions_dev) & 3u))
        return set_error(KVTC_E_ARG, "kvtc_rope_scaled: misaligned buffer");
    const bool in_place = x_dev == out_dev;
    if (in_place && ((n_tokens > 1 && token_stride != out_token_stride) || (n_heads > 1 && head_stride != out_head_stride)))
        return set_error(KVTC_E_ARG, "kvtc_rope_scaled: in place, the strides have to be the same");
    const int64_t most = (int64_t)1 << 62;
    if (!positions_dev && (position0 > most || position0 < -most)) return set_error(KVTC_E_ARG, "kvtc_rope_scaled: position0=%lld", (long long)position0);
    RopeScaledArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x_dev;
    a.out = out_dev;
    a.x_token = token_stride;
    a.x_head = head_stride;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.positions = positions_dev;
    a.position0 = position0;
    a.n_tokens = n_tokens;
    a.n_heads = n_heads;
    a.half = form->n_rotated / 2;
    a.heads_first = n_heads > 1 && n_tokens > 1 && head_stride > token_stride;
    a.cosine_factor = inverse ? (float)(1.0 / form->magnitude) : (float)form->magnitude;
    a.sine_factor = inverse ? -a.cosine_factor : a.cosine_factor;
    memcpy(a.theta, form->theta, sizeof(a.theta));
    const hipError_t e = launch_rope_scaled(a, dtype, form->n_rotated, in_place ? 0 : d_head - form->n_rotated, form->pairing == KVTC_ROPE_INTERLEAVED, static_cast<hipStream_t>(stream));
    if (e != hipSuccess) return set_error(KVTC_E_HIP, "kvtc_rope_scaled: launch failed: %s", hipGetErrorString(e));
    return KVTC_OK;
}

}  // extern "C"
