// kvc_norm_rope on CDNA4 (gfx950): a layer's query, key and value projections become what the cache calls
// take, in one pass over memory: per-head root-mean-square norm, rotary embedding, rounding to fp16 and the
// layout by unit.
//
// y = x rsqrt(mean_j x_j^2 + eps) w, then pairs (j, j + 64) turned by pos base^(-2j/128). Sixteen lanes take
// one head: lane c holds elements 4c + [0, 4) and their partners 64 + 4c + [0, 4), so that a rotation pair
// sits in one lane, the mean is four row rotations, and a head's loads and stores are whole 128-byte lines.
// A wavefront takes four heads at a time and several turns of them for one token, whose sines and cosines
// (turns of the angle reduced in fp64, then fp32) it forms once. Statistics and rotation are fp32; the only
// rounding to fewer bits is the one to fp16 on the way out (the unrotated and the rotated key are both
// rounded from the fp32 norm, not one from the other).
//
// At two limits where there is much of it: 16384 tokens of 48 heads in bf16 68 us, 436 MB at 6.4 TB/s (a large copy reaches 5.2 to
// 5.4), with vector instructions 95 % of the time; in fp32, 638 MB, 119 us at 5.4 TB/s and vector instructions 51 %. One token
// 3.3 us, 488 tokens of 80 heads 8.3 us: latency, and less than a call's 13 us on the host.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "kvc_device.h"
#include "kvc_internal.h"

namespace kvc {
namespace {

constexpr int kNrD = KVC_HEAD_DIM;
constexpr int kNrThreads = 256;
constexpr int64_t kNrCached = 128ll << 20;
constexpr float kNrLeast = 0x1p-100f;  // squares that fp32 holds to fewer bits (below 2^-126) are nothing beside a mean of this

struct NrArgs {
    const void* x[3];        // q, k, v: token-major rows of heads (null: absent)
    int64_t stride[3];       // elements between tokens
    int heads[3];            // heads per token: kv_heads G, kv_heads, kv_heads (0: absent)
    const float* w[3];       // norm weights (null: no norm)
    uint16_t* out[3];        // q rotated, k unrotated, v (null: not wanted)
    uint16_t* k_rot;         // k rotated (null: not wanted)
    const int32_t* pos;
    float eps;
    int n_tok, G, kv_heads;
    int64_t tokens;          // n_seq n_tok
    int turns;               // turns of four heads per wavefront
    int waves;               // wavefronts per token
    int rotate;
    double freq[kNrD / 2];   // turns per position of each pair
};

// Four consecutive elements as fp32.
template <int DT>
__device__ __forceinline__ float4 load4(const void* p, int64_t at) {
    if constexpr (DT == KVC_F32) {
        return *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + at);
    } else {
        const uint2 v = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + at);
        if constexpr (DT == KVC_BF16)
            return float4{__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xffff0000u), __uint_as_float(v.y << 16),
                          __uint_as_float(v.y & 0xffff0000u)};
        else
            return float4{h2f((uint16_t)v.x), h2f((uint16_t)(v.x >> 16)), h2f((uint16_t)v.y), h2f((uint16_t)(v.y >> 16))};
    }
}

// (The encoder takes finite input: what is too large is the largest number, NaN is left for the caller to see.)
template <bool NT>
__device__ __forceinline__ void store4(uint16_t* p, float4 v) {
    const sat_h4 h = saturated_half(v.x, v.y, v.z, v.w);
    if constexpr (NT) __builtin_nontemporal_store(h, reinterpret_cast<sat_h4*>(p));
    else *reinterpret_cast<sat_h4*>(p) = h;
}

__device__ __forceinline__ float row_sum16(float v) {
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x128, 0xf, 0xf, true));
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x124, 0xf, 0xf, true));
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x122, 0xf, 0xf, true));
    v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), 0x121, 0xf, 0xf, true));
    return v;
}

__device__ __forceinline__ float row_max16(float v) {
    for (int o = 1; o < 16; o <<= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ __forceinline__ float max4(float4 a) { return fmaxf(fmaxf(fabsf(a.x), fabsf(a.y)), fmaxf(fabsf(a.z), fabsf(a.w))); }
__device__ __forceinline__ float4 ldexp4(float4 a, int e) { return float4{ldexpf(a.x, e), ldexpf(a.y, e), ldexpf(a.z, e), ldexpf(a.w, e)}; }
__device__ __forceinline__ float dot4(float4 a) { return fmaf(a.x, a.x, fmaf(a.y, a.y, fmaf(a.z, a.z, a.w * a.w))); }

template <int DT, bool NT>
__global__ __launch_bounds__(kNrThreads) void norm_rope_kernel(const NrArgs a) {
    const int64_t wave = (int64_t)blockIdx.x * (kNrThreads / 64) + (threadIdx.x >> 6);
    const int64_t tok = wave / a.waves;
    if (tok >= a.tokens) return;
    const int part = (int)(wave - tok * a.waves);
    const int lane = threadIdx.x & 63, c = lane & 15, grp = lane >> 4;
    const int64_t seq = tok / a.n_tok, n = tok - seq * a.n_tok;
    float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.rotate) {
        const double p = (double)a.pos[tok];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const double t = p * a.freq[4 * c + e];
            const float f = (float)(t - rint(t));
            sn[e] = __builtin_amdgcn_sinf(f);
            cs[e] = __builtin_amdgcn_cosf(f);
        }
    }
    const int total = a.heads[0] + a.heads[1] + a.heads[2];
    for (int it = 0; it < a.turns; ++it) {
        const int hh = (part * a.turns + it) * 4 + grp;
        if (hh >= total) break;
        const int kind = hh < a.heads[0] ? 0 : (hh < a.heads[0] + a.heads[1] ? 1 : 2);
        const int h = hh - (kind > 0 ? a.heads[0] : 0) - (kind > 1 ? a.heads[1] : 0);
        const void* src = kind == 0 ? a.x[0] : (kind == 1 ? a.x[1] : a.x[2]);
        const float* w = kind == 0 ? a.w[0] : (kind == 1 ? a.w[1] : nullptr);
        const int64_t at = tok * (kind == 0 ? a.stride[0] : (kind == 1 ? a.stride[1] : a.stride[2])) + (int64_t)h * kNrD + 4 * c;
        float4 x = load4<DT>(src, at), y = load4<DT>(src, at + 64);
        if (w) {
            float ms = fmaf(row_sum16(dot4(x) + dot4(y)), 1.f / kNrD, a.eps);
            if (!(ms >= kNrLeast && ms < INFINITY)) {  // squares past fp32 or below its precision: again, the largest element in [1, 2)
                const float big = row_max16(fmaxf(max4(x), max4(y)));
                if (big > 0.f && big < INFINITY) {
                    const int e = ilogbf(big);
                    x = ldexp4(x, -e);
                    y = ldexp4(y, -e);
                    ms = fmaf(row_sum16(dot4(x) + dot4(y)), 1.f / kNrD, ldexpf(a.eps, -2 * e));
                }
            }
            const float s = 1.f / sqrtf(ms);
            const float4 wx = *reinterpret_cast<const float4*>(w + 4 * c), wy = *reinterpret_cast<const float4*>(w + 64 + 4 * c);
            x = float4{x.x * s * wx.x, x.y * s * wx.y, x.z * s * wx.z, x.w * s * wx.w};
            y = float4{y.x * s * wy.x, y.y * s * wy.y, y.z * s * wy.z, y.w * s * wy.w};
        }
        // unit-major rows: q [unit][token][g], k and v [unit][token]
        const int unit = kind == 0 ? h / a.G : h, g = kind == 0 ? h - unit * a.G : 0;
        const int64_t row = ((seq * a.kv_heads + unit) * a.n_tok + n) * (kind == 0 ? a.G : 1) + g;
        uint16_t* plain = kind == 0 ? nullptr : (kind == 1 ? a.out[1] : a.out[2]);
        uint16_t* turned = kind == 0 ? a.out[0] : (kind == 1 ? a.k_rot : nullptr);
        if (plain) {
            store4<NT>(plain + row * kNrD + 4 * c, x);
            store4<NT>(plain + row * kNrD + 64 + 4 * c, y);
        }
        if (turned && !a.rotate) {  // (a pair's other element does not enter, not even times 0)
            store4<NT>(turned + row * kNrD + 4 * c, x);
            store4<NT>(turned + row * kNrD + 64 + 4 * c, y);
        } else if (turned) {
            store4<NT>(turned + row * kNrD + 4 * c, float4{x.x * cs[0] - y.x * sn[0], x.y * cs[1] - y.y * sn[1], x.z * cs[2] - y.z * sn[2],
                                                           x.w * cs[3] - y.w * sn[3]});
            store4<NT>(turned + row * kNrD + 64 + 4 * c, float4{x.x * sn[0] + y.x * cs[0], x.y * sn[1] + y.y * cs[1],
                                                                x.z * sn[2] + y.z * cs[2], x.w * sn[3] + y.w * cs[3]});
        }
    }
}

template <int DT>
void launch_norm_rope(const NrArgs& a, bool nt, int64_t blocks, hipStream_t st) {
    if (nt) hipLaunchKernelGGL((norm_rope_kernel<DT, true>), dim3((unsigned)blocks), dim3(kNrThreads), 0, st, a);
    else hipLaunchKernelGGL((norm_rope_kernel<DT, false>), dim3((unsigned)blocks), dim3(kNrThreads), 0, st, a);
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" int kvc_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                             int32_t dtype, int32_t n_seq, int32_t n_tok, int32_t kv_heads, int32_t G, const float* wq, const float* wk,
                             float eps, const int32_t* pos, float rope_base, uint16_t* q_out, uint16_t* k_out, uint16_t* k_rot,
                             uint16_t* v_out, void* stream) {
    clear_error();
    if (dtype != KVC_F16 && dtype != KVC_BF16 && dtype != KVC_F32) return set_error(KVC_EUNSUPPORTED, "kvc_norm_rope: dtype %d", dtype);
    if (n_seq < 0 || n_tok < 0) return set_error(KVC_EINVAL, "kvc_norm_rope: negative n_seq or n_tok");
    if (kv_heads < 1 || G < 1 || kv_heads > 65536 || G > 65536 || (int64_t)kv_heads * G > 65536)
        return set_error(KVC_EINVAL, "kvc_norm_rope: kv_heads = %d, G = %d (at least one, at most 65536 query heads)", kv_heads, G);
    if (!(eps >= 0.f) || !std::isfinite(eps)) return set_error(KVC_EINVAL, "kvc_norm_rope: eps must be finite and >= 0");
    if (rope_base != 0.f && (!(rope_base > 1.f) || !std::isfinite(rope_base)))
        return set_error(KVC_EINVAL, "kvc_norm_rope: rope_base must be 0 (no rotation) or finite and > 1");
    if ((int64_t)n_seq * n_tok == 0) return KVC_OK;
    if (!q != !q_out || !v != !v_out || !k != (!k_out && !k_rot))
        return set_error(KVC_EINVAL, "kvc_norm_rope: an input without its output, or an output without its input");
    if (!q && !k && !v) return set_error(KVC_EINVAL, "kvc_norm_rope: null pointer");
    if (rope_base != 0.f && !pos && (q || k_rot)) return set_error(KVC_EINVAL, "kvc_norm_rope: a rotation needs positions");
    const int size = dtype == KVC_F32 ? 4 : 2, Hq = kv_heads * G;
    const struct { const void* x; int64_t stride; int heads; } in[3] = {{q, q_stride, Hq}, {k, k_stride, kv_heads}, {v, v_stride, kv_heads}};
    for (const auto& i : in)
        if (i.x && ((reinterpret_cast<uintptr_t>(i.x) & 15) || (i.stride * size & 15) || i.stride < (int64_t)i.heads * kNrD))
            return set_error(KVC_EINVAL, "kvc_norm_rope: inputs must be 16-byte aligned, token strides multiples of 16 bytes and >= a token's heads");
    for (const void* p : {(const void*)q_out, (const void*)k_out, (const void*)k_rot, (const void*)v_out, (const void*)wq, (const void*)wk})
        if (reinterpret_cast<uintptr_t>(p) & 15) return set_error(KVC_EINVAL, "kvc_norm_rope: outputs and weights must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(pos) & 3) return set_error(KVC_EINVAL, "kvc_norm_rope: pos must be 4-byte aligned");
    NrArgs a;
    a.tokens = (int64_t)n_seq * n_tok;
    for (int i = 0; i < 3; ++i) {
        a.x[i] = in[i].x;
        a.stride[i] = in[i].stride;
        a.heads[i] = in[i].x ? in[i].heads : 0;
    }
    a.w[0] = wq; a.w[1] = wk; a.w[2] = nullptr;
    a.out[0] = q_out; a.out[1] = k_out; a.out[2] = v_out;
    a.k_rot = k_rot;
    a.pos = pos;
    a.eps = eps;
    a.n_tok = n_tok;
    a.G = G;
    a.kv_heads = kv_heads;
    a.rotate = rope_base != 0.f;
    for (int j = 0; j < kNrD / 2; ++j) a.freq[j] = 0.0;
    if (a.rotate) rope_frequencies(rope_base, a.freq);
    const int fours = (a.heads[0] + a.heads[1] + a.heads[2] + 3) / 4;
    // A wavefront takes as many turns of its token as leave every place of the device (32 wavefronts a CU) one.
    const int64_t places = 32ll * device_cus(), want = (a.tokens * fours + places - 1) / places;
    a.turns = want < 1 ? 1 : (want > fours ? fours : (int)want);
    a.waves = (fours + a.turns - 1) / a.turns;
    const int64_t blocks = (a.tokens * a.waves + kNrThreads / 64 - 1) / (kNrThreads / 64);
    if (blocks > INT32_MAX) return set_error(KVC_EUNSUPPORTED, "kvc_norm_rope: too many tokens");
    // Results too large to be found in a cache afterwards go past them: 235 MB 90 -> 69 us (with a reader behind, 128 and 131);
    // 59 MB 20 us either way, and its reader finds them (36 us together, 40 past the caches).
    const int64_t rows = (int64_t)a.heads[0] + (k_out ? kv_heads : 0) + (k_rot ? kv_heads : 0) + (v_out ? kv_heads : 0);
    const bool nt = a.tokens * rows * kNrD * 2 > kNrCached;
    const hipStream_t st = (hipStream_t)stream;
    if (dtype == KVC_F16) launch_norm_rope<KVC_F16>(a, nt, blocks, st);
    else if (dtype == KVC_BF16) launch_norm_rope<KVC_BF16>(a, nt, blocks, st);
    else launch_norm_rope<KVC_F32>(a, nt, blocks, st);
    return check_launch("kvc_norm_rope");
}
