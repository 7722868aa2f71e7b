// kvc_tree_attn on CDNA4 (gfx950): attention of a tree of drafted tokens over the packed cache and over the
// tree itself.
//
// Rows (drafted token n, head g) of a unit, up to 1024 of them, share its keys, so that unlike a single
// query's decode the products are dense: S^T = K Q^T and O^T = Z_V^T P^T with the rows as columns. Two kernels:
//  tree_partial_kernel  the cached tokens, split over row blocks and context chunks: partials (m, l, O in the
//                       rank space of the values) per row and chunk;
//  tree_finish_kernel   per sixteen rows: merges the chunks, applies P_V, adds the drafted tokens.
#define KVC_DECODE_PARTIALS_UNIT
#include "kvc_decode.hip"

#include "kvc_codes.h"

namespace kvc {
namespace {

constexpr int kTreeWaves = 4;
constexpr int kTreeThreads = 64 * kTreeWaves;
constexpr float kTreeShift = 10.f;  // softmax weights are 2^(s - m + 10): fp16 keeps 11 bits of them down to 2^-24 of the largest
constexpr float kTreeLazy = 5.f;    // the running maximum is raised when a tile beats it by more: weights stay below 2^15
constexpr int kTreeResync = 32;     // tiles between exact sines and cosines (in between they advance by a rotation)

struct TreeRope {
    double freq[kD / 2];  // turns per position of each pair
};

struct TreeWork {
    int M, rows_pb, nrb, n_chunks;  // rows, rows per block, row blocks, chunks per unit
    int max_seq, k_cap_tiles, v_cap_tiles;
};

// Token of a 16-token quarter in slot (s, e) of the operand that the unpacked value field fills (k_pairs: dword d
// holds positions d and d + 8), and so of row 4 grp + v of key block tb = 2 s + e / 4, v = e % 4.
__device__ __forceinline__ int tree_tok(int bv, int tb, int v) {
    const int j = 4 * (tb >> 1) + 2 * (tb & 1) + (v >> 1) + 8 * (v & 1);
    return bv == 8 ? j : (bv == 4 ? 8 * (j >> 3) + 4 * (j & 1) + ((j & 7) >> 1) : 4 * (j & 3) + (j >> 2));
}

// ---------------------------------------------------------------- codes of one lane

// The field of one token's coordinate group, 16 codes at slot x of every plane: the dwords that hold it.
constexpr int tree_k_words(int b) { return b == 8 ? 5 : (b & 4 ? 3 : 0) + (b & 2 ? 2 : 0) + (b & 1 ? 2 : 0); }
template <int B>
__device__ __forceinline__ void tree_k_load(const __amdgpu_buffer_rsrc_t rs, int tile_off, int r, uint32_t x, uint32_t (&w)[7]) {
    int o = 0;
#pragma unroll
    for (int k = 0; k < n_planes(B); ++k) {
        const int P = plane_w(B, k);
        const int at = tile_off + 8 * r * plane_off(B, k) + (int)((P * x) >> 5) * 4;
        if (P <= 2) {
            const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0);
            w[o] = v[0]; w[o + 1] = v[1];
            o += 2;
        } else if (P == 4) {
            const auto v = __builtin_amdgcn_raw_buffer_load_b96(rs, at, 0, 0);
            w[o] = v[0]; w[o + 1] = v[1]; w[o + 2] = v[2];
            o += 3;
        } else {
            const v4u v = __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0);
            w[o] = v[0]; w[o + 1] = v[1]; w[o + 2] = v[2]; w[o + 3] = v[3];
            w[o + 4] = __builtin_amdgcn_raw_buffer_load_b32(rs, at + 16, 0, 0);
            o += 5;
        }
    }
}
template <int B>
__device__ __forceinline__ void tree_k_frag(const uint32_t (&w)[7], uint32_t x, uint32_t e512, rc_h8 (&z)[2]) {
    Fld f[3] = {};
    int o = 0;
#pragma unroll
    for (int k = 0; k < n_planes(B); ++k) {
        const int P = plane_w(B, k);
        const uint32_t sh = P * x;  // funnel shifts by its low five bits
        if (P <= 2) {
            f[k].w0 = funnel(w[o + 1], w[o], sh);
            o += 2;
        } else if (P == 4) {
            f[k].w0 = funnel(w[o + 1], w[o], sh);
            f[k].w1 = funnel(w[o + 2], w[o + 1], sh);
            o += 3;
        } else {
            f[k].w0 = funnel(w[o + 1], w[o], sh);
            f[k].w1 = funnel(w[o + 2], w[o + 1], sh);
            f[k].w2 = funnel(w[o + 3], w[o + 2], sh);
            f[k].w3 = funnel(w[o + 4], w[o + 3], sh);
            o += 5;
        }
    }
    k_pairs<B>(f, false, e512, z);
}

// The value field of coordinate 16 n + c, quarter q: 2p bytes per plane.
template <int B>
__device__ __forceinline__ void tree_v_load(const __amdgpu_buffer_rsrc_t rs, int tile_off, int r, int n, int c, int q, uint32_t (&w)[4]) {
    int o = 0;
#pragma unroll
    for (int k = 0; k < n_planes(B); ++k) {
        const int P = plane_w(B, k);
        const int at = tile_off + 8 * r * plane_off(B, k) + v_field_off(P, r, n, c, q);
        if (P == 1) {
            w[o] = __builtin_amdgcn_raw_buffer_load_b16(rs, at, 0, 0);
            o += 1;
        } else if (P == 2) {
            w[o] = __builtin_amdgcn_raw_buffer_load_b32(rs, at, 0, 0);
            o += 1;
        } else if (P == 4) {
            const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, at, 0, 0);
            w[o] = v[0]; w[o + 1] = v[1];
            o += 2;
        } else {
            const v4u v = __builtin_amdgcn_raw_buffer_load_b128(rs, at, 0, 0);
            w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3];
        }
    }
}
template <int B>
__device__ __forceinline__ void tree_v_frag(const uint32_t (&w)[4], uint32_t e512, rc_h8 (&z)[2]) {
    Fld f[3] = {};
    int o = 0;
#pragma unroll
    for (int k = 0; k < n_planes(B); ++k) {
        const int P = plane_w(B, k);
        if (P <= 2) {
            f[k].w0 = w[o];
            o += 1;
        } else if (P == 4) {
            f[k].w0 = w[o]; f[k].w1 = w[o + 1];
            o += 2;
        } else {
            f[k] = Fld{w[0], w[1], w[2], w[3]};
        }
    }
    k_pairs<B>(f, false, e512, z);
}

// ---------------------------------------------------------------- cached tokens

constexpr int kTreeK = kBtBytes;                     // LDS: P_K^T, then the tile's keys, values, rotation of 64 positions
constexpr int kTreeV = kTreeK + kTile * kD * 2;
constexpr int kTreeAdv = kTreeV + kTile * kD * 2;
constexpr int kTreeSmem = kTreeAdv + (kD / 2) * 8;

// Block: rows [rows_pb rb, ..) of one unit over one of its chunks. Per 64-token tile the wavefronts rebuild and rotate
// sixteen keys each (K^T = P_K^T Z^T) and unpack the value codes, both to LDS as fp16 operands; then each takes its own
// 16 CB rows: S^T = K Q^T, the online softmax, O^T += Z_V^T P^T. Key row m of block tb is the token whose value sits in
// slot (tb, m % 4) of quarter m / 4, so that the lane that computes a weight is the lane whose operand needs it.
template <int CB, bool ROPE>
__global__ __launch_bounds__(kTreeThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void tree_partial_kernel(
    DevSide K, DevSide V, const uint16_t* __restrict__ q, const int32_t* __restrict__ seq_len, TreeWork wk, TreeRope rope,
    float* __restrict__ acc_out, float2* __restrict__ ml_out) {
    const int rb = blockIdx.x % wk.nrb, ch = blockIdx.x / wk.nrb % wk.n_chunks, u = blockIdx.x / wk.nrb / wk.n_chunks;
    const int tid = threadIdx.x, wv = uni(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;
    int T = uni(seq_len[u]);
    T = T < 0 ? 0 : (T > wk.max_seq ? wk.max_seq : T);
    const int tiles = (T + kTile - 1) / kTile, per = (tiles + wk.n_chunks - 1) / wk.n_chunks;
    const int tile0 = ch * per, tile1 = min(tiles, tile0 + per);
    const int row0 = rb * wk.rows_pb + 16 * CB * wv;  // the wavefront's rows
    const int64_t prow = ((int64_t)u * wk.n_chunks + ch) * wk.M;
    if (tile0 >= tile1) {
        if (grp == 0) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
                if (row0 + 16 * cb + col < wk.M) ml_out[prow + row0 + 16 * cb + col] = float2{-INFINITY, 0.f};
        }
        return;
    }
    const int rk = uni(K.r[u]), bk = uni(K.b[u]), rv = uni(V.r[u]), bv = uni(V.b[u]);
    uint8_t* sm = kvc_dsm;
    uint8_t* kt = sm + kTreeK;
    uint8_t* vt = sm + kTreeV;
    float2* adv = reinterpret_cast<float2*>(sm + kTreeAdv);
    stage_basis_t<KVC_SIDE_K>(sm, K.basis + K.basis_off[u], rk, tid, kTreeThreads);
    if (ROPE && tid < kD / 2) {
        const double t = (double)kTile * rope.freq[tid];
        float s, c;
        sincospif(2.f * (float)(t - rint(t)), &s, &c);
        adv[tid] = float2{c, s};
    }
    __syncthreads();

    const uint8_t* kstream = uni(K.codes + K.code_off[u]);
    const uint8_t* vstream = uni(V.codes + V.code_off[u]);
    const int ktb = 8 * rk * bk, vtb = 8 * rv * bv;
    const auto krs = __builtin_amdgcn_make_buffer_rsrc((void*)kstream, (short)0, wk.k_cap_tiles * ktb, kRsrcWord3);
    const auto vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vstream, (short)0, wk.v_cap_tiles * vtb, kRsrcWord3);
    const uint32_t e512 = exp512();
    const int g16 = rk >> 4, rho = rk & 15, nk = (rk + 63) >> 6, nvt = (rv + 15) >> 4;
    // the lane's key token in the tile, and the slots of its fields
    const int ktok = 16 * (col >> 2) + tree_tok(bv, wv, col & 3);
    uint32_t xk[2];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
        const int cg = 4 * ks + grp;  // a group past the rank reads group 0 (its operand rows of P_K^T are zero)
        xk[ks] = cg < g16 ? (uint32_t)(1024 * cg + 16 * ktok) : (cg == g16 && rho ? (uint32_t)(1024 * g16 + ktok * rho) : (uint32_t)(g16 ? 16 * ktok : rho * ktok));
    }
    // queries: columns of the operand, features in the order of the rebuilt keys
    rc_h8 qf[CB][4];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row0 + 16 * cb + col;
        const uint16_t* qr = q + ((int64_t)u * wk.M + (row < wk.M ? row : 0)) * kD + 4 * grp;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            uint2 a = *reinterpret_cast<const uint2*>(qr + 32 * ks), b = *reinterpret_cast<const uint2*>(qr + 32 * ks + 16);
            if (row >= wk.M) a = b = uint2{0u, 0u};
            qf[cb][ks] = __builtin_bit_cast(rc_h8, v4u{a.x, a.y, b.x, b.y});
        }
    }
    const float qs = K.delta[u] * 1.4426950408889634f * 0.08838834764831845f;  // step_K log2(e) / sqrt(128)
    const float lazy = kTreeLazy / qs;
    float m[CB];  // running maxima of the raw products
    rc_f4 O[8][CB], L[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        m[cb] = -INFINITY;
        L[cb] = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < 8; ++n) O[n][cb] = L[cb];
    }
    const _Float16 h1 = (_Float16)1.f;
    const rc_h8 ones = {h1, h1, h1, h1, h1, h1, h1, h1};
    float cs[ROPE ? 4 : 1][4], sn[ROPE ? 4 : 1][4];  // of the lane's pairs 16 rb + 4 grp + v at its token's position

    uint32_t kw[2][7], vw[2][4];
    auto load = [&](int tile) {
        KVC_SWITCH_B(bk, {
            tree_k_load<B_>(krs, tile * ktb, rk, xk[0], kw[0]);
            if (nk > 1) tree_k_load<B_>(krs, tile * ktb, rk, xk[1], kw[1]);
        });
        KVC_SWITCH_B(bv, {
            if (wv < nvt) tree_v_load<B_>(vrs, tile * vtb, rv, wv, col, grp, vw[0]);
            if (wv + 4 < nvt) tree_v_load<B_>(vrs, tile * vtb, rv, wv + 4, col, grp, vw[1]);
        });
    };
    load(tile0);
#pragma unroll 1
    for (int tile = tile0; tile < tile1; ++tile) {
        // ---- keys of the wavefront's sixteen tokens
        if constexpr (ROPE) {
            if ((tile - tile0) % kTreeResync == 0) {
                const double pos = (double)(tile * kTile + ktok);
#pragma unroll
                for (int b4 = 0; b4 < 4; ++b4)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const double t = pos * rope.freq[16 * b4 + 4 * grp + v];
                        sincospif(2.f * (float)(t - rint(t)), &sn[b4][v], &cs[b4][v]);
                    }
            } else {
#pragma unroll
                for (int b4 = 0; b4 < 4; ++b4)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float2 a = adv[16 * b4 + 4 * grp + v];
                        const float c = cs[b4][v], s = sn[b4][v];
                        cs[b4][v] = fmaf(c, a.x, -s * a.y);
                        sn[b4][v] = fmaf(s, a.x, c * a.y);
                    }
            }
        }
        rc_h8 z[4];
        KVC_SWITCH_B(bk, {
            rc_h8 zz[2];
            tree_k_frag<B_>(kw[0], xk[0], e512, zz);
            z[0] = zz[0];
            z[1] = zz[1];
            if (nk > 1) {
                tree_k_frag<B_>(kw[1], xk[1], e512, zz);
                z[2] = zz[0];
                z[3] = zz[1];
            }
        });
        rc_h8 vz[2][2];
        KVC_SWITCH_B(bv, {
            tree_v_frag<B_>(vw[0], e512, vz[0]);
            tree_v_frag<B_>(vw[1], e512, vz[1]);
        });
        if (tile + 1 < tile1) load(tile + 1);
        {
            const uint8_t* pt = sm + bt_lane(col, grp);
            rc_h8 lo[2], hi[2];  // rotated features below and above d / 2, matrix steps ks and ks + 2
#pragma unroll
            for (int b4 = 0; b4 < 4; ++b4) {
                rc_f4 a = rc_f4{0.f, 0.f, 0.f, 0.f}, b = a;
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    if (s < 2 || nk > 1) {
                        a = mfma_h(*reinterpret_cast<const rc_h8*>(pt + bt_block(b4, s)), z[s], a);
                        b = mfma_h(*reinterpret_cast<const rc_h8*>(pt + bt_block(b4 + 4, s)), z[s], b);
                    }
                }
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int e = 4 * (b4 & 1) + v;
                    if constexpr (ROPE) {
                        lo[b4 >> 1][e] = (_Float16)fmaf(a[v], cs[b4][v], -b[v] * sn[b4][v]);
                        hi[b4 >> 1][e] = (_Float16)fmaf(a[v], sn[b4][v], b[v] * cs[b4][v]);
                    } else {
                        lo[b4 >> 1][e] = (_Float16)a[v];
                        hi[b4 >> 1][e] = (_Float16)b[v];
                    }
                }
            }
            uint8_t* dst = kt + (64 * grp + 16 * wv + col) * 16;
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                *reinterpret_cast<rc_h8*>(dst + 4096 * ks) = lo[ks];
                *reinterpret_cast<rc_h8*>(dst + 4096 * (ks + 2)) = hi[ks];
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (wv + 4 * i < nvt) {
                    *reinterpret_cast<rc_h8*>(vt + (wv + 4 * i) * 2048 + lane * 16) = vz[i][0];
                    *reinterpret_cast<rc_h8*>(vt + (wv + 4 * i) * 2048 + 1024 + lane * 16) = vz[i][1];
                }
        }
        __syncthreads();
        // ---- scores of the wavefront's rows
        rc_f4 S[4][CB];
#pragma unroll
        for (int tb = 0; tb < 4; ++tb)
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) S[tb][cb] = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks)
#pragma unroll
            for (int tb = 0; tb < 4; ++tb) {
                const rc_h8 kf = *reinterpret_cast<const rc_h8*>(kt + (256 * ks + 64 * grp + 16 * tb + col) * 16);
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) S[tb][cb] = mfma_h(kf, qf[cb][ks], S[tb][cb]);
            }
        if ((tile + 1) * kTile > T) {  // the context's last tile
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (tile * kTile + 16 * grp + tree_tok(bv, tb, v) >= T)
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) S[tb][cb][v] = -INFINITY;
        }
        // ---- online softmax
        float top[CB];
        bool raise = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            top[cb] = S[0][cb][0];
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int v = 0; v < 4; ++v) top[cb] = fmaxf(top[cb], S[tb][cb][v]);
            raise = raise || top[cb] > m[cb] + lazy;
        }
        if (__any(raise)) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                float t = fmaxf(top[cb], __shfl_xor(top[cb], 16));
                t = fmaxf(t, __shfl_xor(t, 32));
                if (t > m[cb]) {
                    const float a = __builtin_amdgcn_exp2f((m[cb] - t) * qs);
                    m[cb] = t;
                    L[cb] *= a;
#pragma unroll
                    for (int n = 0; n < 8; ++n) O[n][cb] *= a;
                }
            }
        }
        rc_h8 P[2][CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const float off = fmaf(-m[cb], qs, kTreeShift);
#pragma unroll
            for (int tb = 0; tb < 4; ++tb)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    P[tb >> 1][cb][4 * (tb & 1) + v] = (_Float16)__builtin_amdgcn_exp2f(fmaf(S[tb][cb][v], qs, off));
        }
        // ---- values
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) L[cb] = mfma_h(ones, P[s][cb], L[cb]);
#pragma unroll
            for (int n = 0; n < 8; ++n)
                if (n < nvt) {
                    const rc_h8 vf = *reinterpret_cast<const rc_h8*>(vt + n * 2048 + s * 1024 + lane * 16);
#pragma unroll
                    for (int cb = 0; cb < CB; ++cb) O[n][cb] = mfma_h(vf, P[s][cb], O[n][cb]);
                }
        }
        __syncthreads();
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        const int row = row0 + 16 * cb + col;
        if (row >= wk.M) continue;
        if (grp == 0) ml_out[prow + row] = float2{fmaf(m[cb], qs, -kTreeShift), L[cb][0]};
#pragma unroll
        for (int n = 0; n < 8; ++n)
            if (n < nvt) *reinterpret_cast<rc_f4*>(acc_out + (prow + row) * kD + 16 * n + 4 * grp) = O[n][cb];
    }
}

// ---------------------------------------------------------------- drafted tokens, merge, output

constexpr int kFinRows = 16;
constexpr int kFinZ = kBtBytes;                              // LDS: P_V^T, then z [16][132] f32
constexpr int kFinZPitch = kD + 4;
constexpr int kFinX = kFinZ + kFinRows * kFinZPitch * 4;     // drafted values [64][136] fp16
constexpr int kFinXPitch = kD + 8;
constexpr int kFinP = kFinX + KVC_TREE_MAX_TOKENS * kFinXPitch * 2;  // weights [16][72] fp16
constexpr int kFinPPitch = KVC_TREE_MAX_TOKENS + 8;
constexpr int kFinRed = kFinP + kFinRows * kFinPPitch * 2;   // maxima and sums of the wavefronts [2][4][16], row maxima [16], 1 / sums [16]
constexpr int kFinSmem = kFinRed + (2 * 4 * 16 + 32) * 4;

// Block: sixteen rows of one unit. z = sum_c acc_c 2^(m_c - M) over the chunks, the drafted tokens' weights 2^(s - M),
// out = (step_V P_V^T z + sum_m p_m xv_m) / l.
__global__ __launch_bounds__(kTreeThreads) void tree_finish_kernel(DevSide V, const uint16_t* __restrict__ q, int G, int n_tok,
                                                                   const uint16_t* __restrict__ xk, int64_t xk_stride,
                                                                   const uint16_t* __restrict__ xv, int64_t xv_stride,
                                                                   const uint64_t* __restrict__ mask, TreeWork wk,
                                                                   const float* __restrict__ acc, const float2* __restrict__ ml,
                                                                   uint16_t* __restrict__ out) {
    const int nfb = (wk.M + kFinRows - 1) / kFinRows;
    const int u = blockIdx.x / nfb, row0 = blockIdx.x % nfb * kFinRows;
    const int tid = threadIdx.x, wv = uni(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;
    uint8_t* sm = kvc_dsm;
    float* zs = reinterpret_cast<float*>(sm + kFinZ);
    _Float16* xs = reinterpret_cast<_Float16*>(sm + kFinX);
    _Float16* ps = reinterpret_cast<_Float16*>(sm + kFinP);
    float* red = reinterpret_cast<float*>(sm + kFinRed);
    float* big = red + 2 * 4 * 16;
    float* inv = big + 16;
    const int rv = uni(V.r[u]);
    const int row = min(row0 + col, wk.M - 1);
    const uint64_t live = n_tok == 64 ? ~0ull : (1ull << n_tok) - 1ull;
    const uint64_t mine = mask[(int64_t)u * n_tok + row / G] & live;
    if (wk.n_chunks > 0) stage_basis_t<KVC_SIDE_K>(sm, V.basis + V.basis_off[u], rv, tid, kTreeThreads);
    // drafted tokens that some row of the unit names
    uint64_t named = lane < n_tok ? mask[(int64_t)u * n_tok + lane] & live : 0ull;
    for (int o = 1; o < 64; o <<= 1) named |= __shfl_xor(named, o);
    for (int e = tid; e < KVC_TREE_MAX_TOKENS * (kD / 8); e += kTreeThreads) {
        const int t = e >> 4, c8 = e & 15;
        uint4 v = {0u, 0u, 0u, 0u};
        if ((named >> t) & 1) v = *reinterpret_cast<const uint4*>(xv + (int64_t)u * xv_stride + (int64_t)t * kD + 8 * c8);
        *reinterpret_cast<uint4*>(xs + t * kFinXPitch + 8 * c8) = v;
    }
    // scores of the wavefront's sixteen drafted tokens (rows of the result) and the block's rows (columns)
    float s[4];
    {
        const int t = 16 * wv + col;
        const bool there = (named >> t) & 1;
        const uint16_t* kr = xk + (int64_t)u * xk_stride + (int64_t)t * kD + 8 * grp;
        const uint16_t* qr = q + ((int64_t)u * wk.M + row) * kD + 8 * grp;
        rc_f4 c = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            uint4 a = {0u, 0u, 0u, 0u};
            if (there) a = *reinterpret_cast<const uint4*>(kr + 32 * ks);
            c = mfma_h(__builtin_bit_cast(rc_h8, a), *reinterpret_cast<const rc_h8*>(qr + 32 * ks), c);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v)
            s[v] = (mine >> (16 * wv + 4 * grp + v)) & 1 ? c[v] * (1.4426950408889634f * 0.08838834764831845f) : -INFINITY;
    }
    float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    if (grp == 0) red[wv * 16 + col] = top;
    __syncthreads();
    // row r's sixteen threads: maxima and sums over the chunks
    const int mr = tid >> 4, mc = tid & 15;
    const int mrow = min(row0 + mr, wk.M - 1);
    float M = fmaxf(fmaxf(red[mr], red[16 + mr]), fmaxf(red[32 + mr], red[48 + mr]));
    for (int c = 0; c < wk.n_chunks; ++c) M = fmaxf(M, ml[((int64_t)u * wk.n_chunks + c) * wk.M + mrow].x);
    const float Mf = M == -INFINITY ? 0.f : M;
    float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, l = 0.f;
    for (int c = 0; c < wk.n_chunks; ++c) {
        const int64_t pr = ((int64_t)u * wk.n_chunks + c) * wk.M + mrow;
        const float2 v = ml[pr];
        if (v.x == -INFINITY) continue;  // an empty chunk has no accumulators
        const float w = __builtin_amdgcn_exp2f(v.x - Mf);
        l = fmaf(w, v.y, l);
        if (8 * mc < ((rv + 15) & ~15)) {
            const float4 a = *reinterpret_cast<const float4*>(acc + pr * kD + 8 * mc), b = *reinterpret_cast<const float4*>(acc + pr * kD + 8 * mc + 4);
            z[0] = fmaf(w, a.x, z[0]); z[1] = fmaf(w, a.y, z[1]); z[2] = fmaf(w, a.z, z[2]); z[3] = fmaf(w, a.w, z[3]);
            z[4] = fmaf(w, b.x, z[4]); z[5] = fmaf(w, b.y, z[5]); z[6] = fmaf(w, b.z, z[6]); z[7] = fmaf(w, b.w, z[7]);
        }
    }
    if (mc == 0) big[mr] = Mf;
    __syncthreads();
    {
        const float Mc = big[col];
        float p[4], sum = 0.f;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const _Float16 h = (_Float16)__builtin_amdgcn_exp2f(s[v] - Mc);
            ps[col * kFinPPitch + 16 * wv + 4 * grp + v] = h;
            p[v] = (float)h;
            sum += p[v];
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (grp == 0) red[64 + wv * 16 + col] = sum;
    }
    __syncthreads();
    {
        const float sum = l + ((red[64 + mr] + red[80 + mr]) + (red[96 + mr] + red[112 + mr]));
        const float i = sum > 0.f ? 1.f / sum : 0.f;
        if (mc == 0) inv[mr] = i;
#pragma unroll
        for (int e = 0; e < 8; ++e) zs[mr * kFinZPitch + 8 * mc + e] = z[e] * i;
    }
    __syncthreads();
    const float step = V.delta[u], rinv = inv[col];
    rc_f4 o[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int rb = 2 * wv + i;
        rc_f4 c = rc_f4{0.f, 0.f, 0.f, 0.f}, t = c;
        if (wk.n_chunks > 0) {
#pragma unroll
            for (int st = 0; st < 4; ++st) {
                rc_h8 hi, lo;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float x = zs[col * kFinZPitch + bt_coord<KVC_SIDE_K>(32 * st) + 16 * grp + (e >> 1) + 8 * (e & 1)];
                    const _Float16 h = (_Float16)x;
                    hi[e] = h;
                    lo[e] = (_Float16)(x - (float)h);
                }
                const rc_h8 p = *reinterpret_cast<const rc_h8*>(sm + bt_block(rb, st) + bt_lane(col, grp));
                c = mfma_h(p, hi, c);
                c = mfma_h(p, lo, c);
            }
        }
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            rc_h8 a, b;
#pragma unroll
            for (int e = 0; e < 8; ++e) a[e] = xs[(32 * st + 8 * grp + e) * kFinXPitch + 16 * rb + col];
            b = *reinterpret_cast<const rc_h8*>(ps + col * kFinPPitch + 32 * st + 8 * grp);
            t = mfma_h(a, b, t);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) o[i][v] = fmaf(c[v], step, t[v] * rinv);
    }
    if (row0 + col < wk.M) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            typedef _Float16 h4 __attribute__((ext_vector_type(4)));
            const h4 h = {(_Float16)o[i][0], (_Float16)o[i][1], (_Float16)o[i][2], (_Float16)o[i][3]};
            *reinterpret_cast<h4*>(out + ((int64_t)u * wk.M + row0 + col) * kD + 16 * (2 * wv + i) + 4 * grp) = h;
        }
    }
}

// ---------------------------------------------------------------- host side

constexpr int kTreeMaxChunks = 128;

struct TreeLayout {
    TreeWork wk;
    int cb;
    int64_t acc, ml, total;
};

TreeLayout tree_layout(const kvc_stream_desc* k, const kvc_stream_desc* v, int G, int n_tok, int max_seq) {
    TreeLayout t;
    const int U = k->n_units, tiles = (max_seq + kTile - 1) / kTile;
    t.wk.M = n_tok * G;
    t.cb = t.wk.M <= 64 ? 1 : 2;
    t.wk.rows_pb = 64 * t.cb;
    t.wk.nrb = (t.wk.M + t.wk.rows_pb - 1) / t.wk.rows_pb;
    t.wk.max_seq = max_seq;
    t.wk.k_cap_tiles = (k->capacity + kTile - 1) / kTile;
    t.wk.v_cap_tiles = (v->capacity + kTile - 1) / kTile;
    // Chunks per unit: the count that minimises rounds of resident blocks (two per CU) x (tiles + set-up, about
    // three tiles) and the merge, which reads every chunk of every row.
    const int64_t slots = 2ll * device_cus();
    t.wk.n_chunks = 0;
    double best = -1.0;
    for (int n = 1; n <= std::min(tiles, kTreeMaxChunks); ++n) {
        const int per = (tiles + n - 1) / n;
        const int64_t blocks = (int64_t)U * t.wk.nrb * n;
        const double cost = (double)((blocks + slots - 1) / slots) * (per + 3.0) + 0.1 * n;
        if (best < 0.0 || cost < best) { best = cost; t.wk.n_chunks = n; }
    }
    const int64_t rows = (int64_t)U * t.wk.n_chunks * t.wk.M;
    auto up = [](int64_t x) { return (x + 255) / 256 * 256; };
    t.acc = 0;
    t.ml = up(rows * kD * 4);
    t.total = std::max<int64_t>(t.ml + up(rows * 8), 256);
    return t;
}

int tree_check(const kvc_stream_desc* k, const kvc_stream_desc* v, int32_t G, int32_t n_tok, int32_t max_seq_len) {
    if (int e = validate_desc(k, "kvc_tree_attn(k)")) return e;
    if (int e = validate_desc(v, "kvc_tree_attn(v)")) return e;
    if (k->side != KVC_SIDE_K || v->side != KVC_SIDE_V) return set_error(KVC_EINVAL, "kvc_tree_attn: descriptor sides");
    if (k->n_units != v->n_units) return set_error(KVC_EINVAL, "kvc_tree_attn: K and V unit counts differ");
    if (G < 1 || G > KVC_TREE_MAX_GROUP) return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: G = %d (1..%d)", G, KVC_TREE_MAX_GROUP);
    if (n_tok < 1 || n_tok > KVC_TREE_MAX_TOKENS)
        return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: n_tok = %d (1..%d)", n_tok, KVC_TREE_MAX_TOKENS);
    if (max_seq_len < 0) return set_error(KVC_EINVAL, "kvc_tree_attn: negative max_seq_len");
    if (max_seq_len > k->capacity || max_seq_len > v->capacity)
        return set_error(KVC_ENOSPACE, "kvc_tree_attn: max_seq_len exceeds capacity");
    const int64_t kct = ((int64_t)k->capacity + kTile - 1) / kTile, vct = ((int64_t)v->capacity + kTile - 1) / kTile;
    for (int u = 0; u < k->n_units; ++u)  // byte offsets inside a stream are 32 bits
        if (kct * 8 * k->r_host[u] * k->b_host[u] > INT32_MAX || vct * 8 * v->r_host[u] * v->b_host[u] > INT32_MAX)
            return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: a unit's stream exceeds 2 GiB");
    return KVC_OK;
}

template <int CB, bool ROPE>
int launch_tree(dim3 grid, hipStream_t st, const DevSide& K, const DevSide& V, const uint16_t* q, const int32_t* seq_len, const TreeWork& wk,
                const TreeRope& rope, float* acc, float2* ml) {
    const hipError_t e = hipFuncSetAttribute((const void*)tree_partial_kernel<CB, ROPE>, hipFuncAttributeMaxDynamicSharedMemorySize, kTreeSmem);
    if (e != hipSuccess) return set_error(KVC_EDEVICE, "hipFuncSetAttribute: %s", hipGetErrorString(e));
    hipLaunchKernelGGL((tree_partial_kernel<CB, ROPE>), grid, dim3(kTreeThreads), kTreeSmem, st, K, V, q, seq_len, wk, rope, acc, ml);
    return check_launch("kvc_tree_attn");
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" size_t kvc_tree_attn_workspace(const kvc_stream_desc* k, const kvc_stream_desc* v, int32_t G, int32_t n_tok, int32_t max_seq_len) {
    clear_error();
    if (tree_check(k, v, G, n_tok, max_seq_len)) return 0;
    return (size_t)tree_layout(k, v, G, n_tok, max_seq_len).total;
}

extern "C" int kvc_tree_attn(const kvc_stream_desc* k, const kvc_stream_desc* v, const uint16_t* q, int32_t G, int32_t n_tok,
                             const uint16_t* xk, int64_t xk_unit_stride, const uint16_t* xv, int64_t xv_unit_stride, const uint64_t* mask,
                             const int32_t* seq_len, int32_t max_seq_len, float rope_base, uint16_t* out, void* ws, size_t ws_bytes,
                             void* stream) {
    clear_error();
    if (int e = tree_check(k, v, G, n_tok, max_seq_len)) return e;
    if (rope_base != 0.f && (!(rope_base > 1.f) || !std::isfinite(rope_base)))
        return set_error(KVC_EINVAL, "kvc_tree_attn: rope_base must be 0 (no rotation) or finite and > 1");
    if (k->n_units == 0) return KVC_OK;
    if (!q || !mask || !seq_len || !out) return set_error(KVC_EINVAL, "kvc_tree_attn: null pointer");
    if ((reinterpret_cast<uintptr_t>(q) & 15) || (reinterpret_cast<uintptr_t>(out) & 15) || (reinterpret_cast<uintptr_t>(mask) & 7) ||
        (reinterpret_cast<uintptr_t>(seq_len) & 3))
        return set_error(KVC_EINVAL, "kvc_tree_attn: q and out must be 16-byte aligned, mask 8-byte, seq_len 4-byte");
    for (const auto& xs : {std::make_pair(xk, xk_unit_stride), std::make_pair(xv, xv_unit_stride)})
        if (!xs.first || (reinterpret_cast<uintptr_t>(xs.first) & 15) || (xs.second & 7) || xs.second < (int64_t)n_tok * kD)
            return set_error(KVC_EINVAL, "kvc_tree_attn: xk, xv must be 16-byte aligned with stride a multiple of 8 and >= n_tok*d");
    if (!ws) return set_error(KVC_EINVAL, "kvc_tree_attn: null workspace");
    if (reinterpret_cast<uintptr_t>(ws) & 255) return set_error(KVC_EINVAL, "kvc_tree_attn: workspace not 256-byte aligned");
    const TreeLayout t = tree_layout(k, v, G, n_tok, max_seq_len);
    if ((int64_t)ws_bytes < t.total)
        return set_error(KVC_ENOSPACE, "kvc_tree_attn: workspace %zu < %lld bytes", ws_bytes, (long long)t.total);
    float* acc = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + t.acc);
    float2* ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(ws) + t.ml);
    const hipStream_t st = (hipStream_t)stream;
    const DevSide K = dev_side(k), V = dev_side(v);
    const int64_t blocks = (int64_t)k->n_units * t.wk.nrb * t.wk.n_chunks, fin = (int64_t)k->n_units * ((t.wk.M + kFinRows - 1) / kFinRows);
    if (blocks > INT32_MAX || fin > INT32_MAX) return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: too many units");
    if (blocks) {
        TreeRope rope;
        for (int j = 0; j < kD / 2; ++j)
            rope.freq[j] = rope_base != 0.f ? std::pow((double)rope_base, -2.0 * j / kD) / 6.283185307179586476925 : 0.0;
        const dim3 grid((unsigned)blocks);
        int e;
        if (rope_base != 0.f)
            e = t.cb == 1 ? launch_tree<1, true>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml) : launch_tree<2, true>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
        else
            e = t.cb == 1 ? launch_tree<1, false>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml) : launch_tree<2, false>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
        if (e) return e;
    }
    const hipError_t he = hipFuncSetAttribute((const void*)tree_finish_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kFinSmem);
    if (he != hipSuccess) return set_error(KVC_EDEVICE, "hipFuncSetAttribute: %s", hipGetErrorString(he));
    hipLaunchKernelGGL(tree_finish_kernel, dim3((unsigned)fin), dim3(kTreeThreads), kFinSmem, st, V, q, G, n_tok, xk, xk_unit_stride, xv,
                       xv_unit_stride, mask, t.wk, acc, ml, out);
    return check_launch("kvc_tree_attn");
}
