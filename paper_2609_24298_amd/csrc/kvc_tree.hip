// kvc_tree_attn on CDNA4 (gfx950): attention of a tree of drafted tokens over the packed cache and over the
// tree itself.
//
// Rows (drafted token n, head g) of a unit, up to 1024 of them, share its keys, so that unlike a single
// query's decode the products are dense: S^T = K Q^T and O^T = Z_V^T P^T with the rows as columns. Two kernels:
//  tree_partial_kernel  the cached tokens, all units' tiles cut into equal runs: per row and piece of a run (m, l, O in the
//                       rank space of the values);
//  tree_finish_kernel   per sixteen (or four) rows: merges the pieces, applies P_V, adds the drafted tokens.
//
// What bounds it (2 bits per dimension, 64 units of ragged lengths unless said, times of both kernels):
//  256 rows x 32k  313 us, 560 TFLOP/s of score and value products (of 39 GFLOP more the rebuilt keys): vector instructions 44 % of
//                  the time, matrix units 37 %, which two wavefronts a SIMD (256 registers each) overlap only in part; the rest is
//                  waits of a step for the one before.
//   64 rows x 128k, 8 units at 1/2 bit  108 us: the wavefronts that make the keys (rotation, splitting), the same for one row or
//                  64; vector instructions 44 %, LDS 45 %, matrix units 23 %.
//  128 rows x 16k  118 us: as these; vector instructions 44 %, LDS 44 %, matrix units 29 %. (128 registers: some sixty values that a
//                  piece sets up are spilled.)
//   52 rows x 16k, keys not rotated  69 us: the latency of a tile's steps; vector instructions 35 %, matrix units 20 %, LDS 25 %. 128
//                  rows 101 us (30, 27, 22 %), 256 rows 154 us (34, 37, 15 %).
//   20 rows x 300  17 us: two launches of 7 to 10 us, each a chain of four reads of memory.
// (The bytes, at most 110 MB a call, are never the bound.)
#define KVC_DECODE_PARTIALS_UNIT
#include "kvc_decode.hip"

#include <type_traits>

#include "kvc_codes.h"

namespace kvc {
namespace {

constexpr float kTreeShift = 10.f;  // softmax weights are 2^(s - m + 10): fp16 keeps 11 bits of them down to 2^-24 of the largest
constexpr float kTreeLazy = 5.f;    // the running maximum is raised when a tile beats it by more: weights stay below 2^15
// Tiles between exact sines and cosines (in between they advance by a rotation of 64 positions, 2^-23 off each time). The
// exact ones are the hardware's, of the angle in turns reduced in fp64: at most 2^-22.9 off over a whole turn (measured).
constexpr int kTreeResync = 32;

constexpr float kRawScale = 16777216.f;  // 2^24: a raw code in an fp16 operand is this times too small
constexpr float kTreeLoScale = 2048.f;  // of the low part of a key
constexpr int kTreeLoExp = 127 - 11;    // its scale as a matrix operand's exponent

typedef int v8i __attribute__((ext_vector_type(8)));

// K's low parts (bf8, scaled up) times the queries' leading bits (bf8).
__device__ __forceinline__ rc_f4 mfma_lo(v8i a, v8i b, rc_f4 c) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 1, 1, 0, kTreeLoExp, 0, 127);
}
// The upper byte of each of a lane's 32 fp16 features: four features of a sixteen per dword, as the keys' low parts lie.
__device__ __forceinline__ v8i lead_bits(const rc_h8 (&q)[4]) {
    v8i r;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        const v4u d = __builtin_bit_cast(v4u, q[ks]);
        r[2 * ks] = (int)perm(d[1], d[0], 0x07050301u);
        r[2 * ks + 1] = (int)perm(d[3], d[2], 0x07050301u);
    }
    return r;
}

// Two values rounded to fp16 by one instruction (left to itself the compiler forms the value a second time for each half).
__device__ __forceinline__ rc_h2 to_half2(float x, float y) {
    uint32_t r;
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
    return __builtin_bit_cast(rc_h2, r);
}

// x = x y + z where x stands (the compiler's own choice for a value carried round a loop costs a copy).
__device__ __forceinline__ void fma_in_place(float& x, float y, float z) { asm("v_fma_f32 %0, %0, %1, %2" : "+v"(x) : "v"(y), "v"(z)); }

// Four values, times 2^11, as bf8.
typedef short s2v __attribute__((ext_vector_type(2)));
__device__ __forceinline__ s2v bf8_pairs(const float (&x)[4]) {
    s2v r = __builtin_bit_cast(s2v, x[0]);  // (both halves are written: any register will do)
    r = __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, x[0], x[1], 1.f / kTreeLoScale, false);
    return __builtin_amdgcn_cvt_scalef32_pk_bf8_f32(r, x[2], x[3], 1.f / kTreeLoScale, true);
}

struct TreeRope {
    double freq[kD / 2];  // turns per position of each pair
};

struct TreeWork {
    int U, M, rows_pb, nrb;  // units, rows of one, rows per block, row blocks
    int n_blocks;            // blocks that share the tiles of all units (0: no cache at all)
    int max_seq, k_cap_tiles, v_cap_tiles;
};

// ---------------------------------------------------------------- division of the work

// The tiles of all units, one after another, are cut into equal runs, one for each block: lengths differ between sequences and
// are known on the device only. Beginning a unit costs a block as much as some tiles (its basis, queries and first codes
// are fetched), so each unit with any tiles begins with start_cost tiles that hold nothing. The piece of unit u in block
// b's run leaves its partials in slot b + u, which is unique.
__device__ __forceinline__ int unit_tokens(const int32_t* __restrict__ seq_len, int u, int max_seq) {
    const int T = seq_len[u];
    return T < 0 ? 0 : (T > max_seq ? max_seq : T);
}
__device__ __forceinline__ int unit_tiles(const int32_t* __restrict__ seq_len, int u, int max_seq) {
    return (unit_tokens(seq_len, u, max_seq) + kTile - 1) / kTile;
}
// 64 units x 4k x 32 rows 48.3 us without, 45.0 with, x 16k x 52 rows 114.7 and 109.3; 8 units x 128k, which divide evenly without,
// 135 and 139. Three or seven instead of five are no better (38.4 and 37.7 against 38.0, 95.1 and 96.5 against 94.6); with 256 rows
// x 4k 80.4 us with two, 78.6 with four.
__host__ __device__ constexpr int start_cost(int M) { return M <= 64 ? 5 : 4; }
__device__ __forceinline__ uint32_t unit_work(int tiles, int M) { return tiles ? (uint32_t)(tiles + start_cost(M)) : 0u; }
// (32 bits: the host refuses more tiles)
__device__ __forceinline__ uint32_t run_tiles(uint32_t total, int n_blocks) { return (total + (uint32_t)n_blocks - 1u) / (uint32_t)n_blocks; }

__device__ __forceinline__ uint32_t wave_total(uint32_t v) {
    for (int o = 1; o < 64; o <<= 1) v += __shfl_xor(v, o);
    return v;
}

// Token of a 16-token quarter in slot (s, e) of the operand that the unpacked value field fills (k_pairs: dword d
// holds positions d and d + 8), and so of row 4 grp + v of key block tb = 2 s + e / 4, v = e % 4.
__device__ __forceinline__ int tree_tok(int bv, int tb, int v) {
    const int j = 4 * (tb >> 1) + 2 * (tb & 1) + (v >> 1) + 8 * (v & 1);
    return bv == 8 ? j : (bv == 4 ? 8 * (j >> 3) + 4 * (j & 1) + ((j & 7) >> 1) : 4 * (j & 3) + (j >> 2));
}

// ---------------------------------------------------------------- codes of one lane

// A field of sixteen codes is read plane by plane, the planes that a width has chosen by uniform branches (a switch over
// the widths, compiled eight times, took some fifty registers of the loop around it). w: the 4-bit plane's dwords
// (or the 8-bit one's first) at 0, the 2-bit one's (or the 8-bit one's rest) at 3, the 1-bit one's at 5.
constexpr int kFieldWords = 7;

// Byte of the dword in which slot x of each plane begins: of the widest plane (4 or 8 bits), the 2-bit and the 1-bit one.
struct PlaneAt { int a4, a2, a1; };

// One token's coordinate group, sixteen codes from slot x on of every plane.
__device__ __forceinline__ PlaneAt tree_k_at(int b, int r, uint32_t x) {
    PlaneAt p;
    p.a4 = b == 8 ? (int)(8 * x >> 5) * 4 : (int)(4 * x >> 5) * 4;
    p.a2 = 8 * r * (b & 4) + (int)(2 * x >> 5) * 4;
    p.a1 = 8 * r * (b & 6) + (int)(x >> 5) * 4;
    return p;
}
__device__ __forceinline__ void tree_k_load(const __amdgpu_buffer_rsrc_t rs, int tile_off, int b, const PlaneAt& p, uint32_t (&w)[kFieldWords]) {
    if (b & 12) {
        const auto v = __builtin_amdgcn_raw_buffer_load_b96(rs, p.a4, tile_off, 0);
        w[0] = v[0]; w[1] = v[1]; w[2] = v[2];
    }
    if (b & 8) {
        const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, p.a4 + 12, tile_off, 0);
        w[3] = v[0]; w[4] = v[1];
    }
    if (b & 2) {
        const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, p.a2, tile_off, 0);
        w[3] = v[0]; w[4] = v[1];
    }
    if (b & 1) {
        const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, p.a1, tile_off, 0);
        w[5] = v[0]; w[6] = v[1];
    }
}

// Codes m and m + 8 of a field in the halves of c[m].
__device__ __forceinline__ void pairs4(uint32_t w0, uint32_t w1, uint32_t (&c)[8]) {
    const uint32_t y0 = perm(w1, w0, 0x05040100u), y1 = perm(w1, w0, 0x07060302u);
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        c[m] = (y0 >> (4 * m)) & 0x000f000fu;
        c[m + 4] = (y1 >> (4 * m)) & 0x000f000fu;
    }
}
__device__ __forceinline__ void pairs2(uint32_t w, int up, uint32_t (&c)[8]) {
#pragma unroll
    for (int m = 0; m < 8; ++m) c[m] = (c[m] << up) | ((w >> (2 * m)) & 0x00030003u);
}
__device__ __forceinline__ void pairs1(uint32_t w, int up, uint32_t (&c)[8]) {
    const uint32_t y = perm(0u, w, 0x0c010c00u);
#pragma unroll
    for (int m = 0; m < 8; ++m) c[m] = (c[m] << up) | ((y >> m) & 0x00010001u);
}
__device__ __forceinline__ void pairs8(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3, uint32_t (&c)[8]) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
        const uint32_t sel = 0x0c040c00u + 0x00010001u * (uint32_t)m;
        c[m] = perm(w2, w0, sel);
        c[m + 4] = perm(w3, w1, sel);
    }
}

// The raw codes of a key field as an operand: the integer c in a half is the fp16 number c 2^-24, which the matrix cores
// take exactly, so that neither an exponent nor the centring costs an instruction here (both are in the accumulator's
// start and in the scale of the rotation). Widths up to 4 have code of their own (two or four operations a dword), the
// rest one path for all.
template <int B>
__device__ __forceinline__ void tree_k_codes(const uint32_t (&w)[kFieldWords], uint32_t x, uint32_t (&c)[8]) {
    uint32_t n[8];
    if constexpr (B == 4) {
        plane_pairs<4, 0>(Fld{funnel(w[1], w[0], 4 * x), funnel(w[2], w[1], 4 * x), 0u, 0u}, false, c);
    } else if constexpr (B >= 2) {
        plane_pairs<2, B - 2>(Fld{funnel(w[4], w[3], 2 * x), 0u, 0u, 0u}, false, c);
        if constexpr (B == 3) {
            plane_pairs<1, 0>(Fld{funnel(w[6], w[5], x), 0u, 0u, 0u}, false, n);
#pragma unroll
            for (int m = 0; m < 8; ++m) c[m] |= n[m];
        }
    } else {
        plane_pairs<1, 0>(Fld{funnel(w[6], w[5], x), 0u, 0u, 0u}, false, c);
    }
}
__device__ __forceinline__ void tree_k_frag(const uint32_t (&w)[kFieldWords], int b, uint32_t x, rc_h8 (&z)[2]) {
    uint32_t c[8];
    if (b == 1) tree_k_codes<1>(w, x, c);
    else if (b == 2) tree_k_codes<2>(w, x, c);
    else if (b == 3) tree_k_codes<3>(w, x, c);
    else if (b == 4) tree_k_codes<4>(w, x, c);
    else {
#pragma unroll
        for (int m = 0; m < 8; ++m) c[m] = 0u;
        if (b & 8) {
            const uint32_t sh = 8 * x;  // funnel shifts by its low five bits
            pairs8(funnel(w[1], w[0], sh), funnel(w[2], w[1], sh), funnel(w[3], w[2], sh), funnel(w[4], w[3], sh), c);
        } else {
            pairs4(funnel(w[1], w[0], 4 * x), funnel(w[2], w[1], 4 * x), c);
        }
        if (b & 2) pairs2(funnel(w[4], w[3], 2 * x), 2, c);
        if (b & 1) pairs1(funnel(w[6], w[5], x), 1, c);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) z[h] = __builtin_bit_cast(rc_h8, v4u{c[4 * h], c[4 * h + 1], c[4 * h + 2], c[4 * h + 3]});
}

// The value field of coordinate 16 n + c, quarter q: 2p bytes per plane (words 0, 1 of the 4-bit plane or all four of the
// 8-bit one, 2 and 3 of the narrow ones).
__device__ __forceinline__ PlaneAt tree_v_at(int b, int r, int n, int c, int q) {
    PlaneAt p;
    p.a4 = b == 8 ? v_field_off(8, r, n, c, q) : v_field_off(4, r, n, c, q);
    p.a2 = 8 * r * (b & 4) + v_field_off(2, r, n, c, q);
    p.a1 = 8 * r * (b & 6) + v_field_off(1, r, n, c, q);
    return p;
}
__device__ __forceinline__ void tree_v_load(const __amdgpu_buffer_rsrc_t rs, int tile_off, int b, const PlaneAt& p, uint32_t (&w)[4]) {
    if (b & 8) {
        const v4u v = __builtin_amdgcn_raw_buffer_load_b128(rs, p.a4, tile_off, 0);
        w[0] = v[0]; w[1] = v[1]; w[2] = v[2]; w[3] = v[3];
    }
    if (b & 4) {
        const v2u v = __builtin_amdgcn_raw_buffer_load_b64(rs, p.a4, tile_off, 0);
        w[0] = v[0]; w[1] = v[1];
    }
    if (b & 2) w[2] = __builtin_amdgcn_raw_buffer_load_b32(rs, p.a2, tile_off, 0);
    if (b & 1) w[3] = __builtin_amdgcn_raw_buffer_load_b16(rs, p.a1, tile_off, 0);
}
// Centred value codes c - 2^(b-1) + 1/2 (exact: 512 + c under fp16's exponent of 512, then one addition). Not left raw like
// the keys': over a long context the centre's share of the sum would swamp what remains of it.
__device__ __forceinline__ void tree_v_frag(const uint32_t (&w)[4], int b, uint32_t e512, rc_h8 (&z)[2]) {
    if (b == 1) k_pairs<1>({Fld{w[3], 0u, 0u, 0u}, Fld{}, Fld{}}, false, e512, z);
    else if (b == 2) k_pairs<2>({Fld{w[2], 0u, 0u, 0u}, Fld{}, Fld{}}, false, e512, z);
    else if (b == 3) k_pairs<3>({Fld{w[2], 0u, 0u, 0u}, Fld{w[3], 0u, 0u, 0u}, Fld{}}, false, e512, z);
    else if (b == 4) k_pairs<4>({Fld{w[0], w[1], 0u, 0u}, Fld{}, Fld{}}, false, e512, z);
    else {
        uint32_t c[8];
        if (b & 8) pairs8(w[0], w[1], w[2], w[3], c);
        else pairs4(w[0], w[1], c);
        if (b & 2) pairs2(w[2], 2, c);
        if (b & 1) pairs1(w[3], 1, c);
        const _Float16 mid = (_Float16)(-512.f - ((float)(1 << (b - 1)) - 0.5f));
        const rc_h2 mid2 = rc_h2{mid, mid};
        uint32_t d[8];
#pragma unroll
        for (int m = 0; m < 8; ++m) d[m] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(rc_h2, (c[m] << 1) | e512) + mid2);
#pragma unroll
        for (int h = 0; h < 2; ++h) z[h] = __builtin_bit_cast(rc_h8, v4u{d[4 * h], d[4 * h + 1], d[4 * h + 2], d[4 * h + 3]});
    }
}

// Item of the staged basis for a thread: four threads read 64 consecutive bytes of a row.
__device__ __forceinline__ int basis_item(int t) { return ((t & 3) | (t >> 7 << 2)) * (kD / 4) + (t >> 2 & 31); }

// ---------------------------------------------------------------- cached tokens

constexpr int kTreeWaves = 8;
constexpr int kTreeThreads = 64 * kTreeWaves;
// LDS: P_K^T, the rotation of 64 positions, then two buffers of a tile's keys (fp16), their low parts (bf8) and values (fp16)
constexpr int kTreeAdv = kBtBytes, kTreeMid = kTreeAdv + (kD / 2) * 8;  // and the centre's share of a rebuilt key
constexpr int kTreePRow = kD + 8;  // plain keys: P_K at 0 instead, in rows of this many elements
constexpr int kTreeBuf = kD * kTreePRow * 2;
static_assert(kTreeMid + kD * 4 <= kTreeBuf);
constexpr int kBufLo = kTile * kD * 2, kTreeBufV = kBufLo + kTile * kD, kTreeBufBytes = kTreeBufV + kTile * kD * 2;
constexpr int kTreeLead = kTreeBuf + 2 * kTreeBufBytes;  // the queries' leading bits, [wavefront][cb][2][lane], or two tiles' key codes
// Plain keys and up to 64 rows: two blocks share a CU, each with half its registers and LDS. (The basis lies in the buffers, the
// projected queries' low parts behind them: [row block][4][lane].) Against one block, 32 rows x 16k x 64 units
// 70 -> 56 us, x 32k 120 -> 89.5, 52 rows x 16k 79 -> 69; 8 units, 64 rows x 128k at 1/2 bit 80 -> 63.
constexpr bool tree_pair(int cb, int rw, bool rope) { return !rope && cb == 1 && rw <= 4; }
constexpr int kPairLow = 2 * kTile * kD * 4;
// Rotated keys and up to 64 (128) rows: eight wavefronts make the tiles and four (eight) more attend, three (four) to a SIMD. Fewer
// registers each, and what one waits for the others fill. Against eight that do both, 64 units: 32 rows x 4k 43.6 -> 37.3 us, 52
// rows x 16k 121 -> 95, 100 rows x 16k 130 -> 114, x 4k 53.4 -> 51.0; 8 units, 64 rows x 128k at 1/2 bit 132 -> 107. (32
// rows a wavefront need more than 168 registers.)
constexpr bool tree_split(int cb, int rw, bool rope) { return rope && cb == 1 && rw >= 4; }
constexpr int tree_threads(int cb, int rw, bool rope) { return kTreeThreads + (tree_split(cb, rw, rope) ? 64 * rw : 0); }
constexpr int tree_waves_per_simd(int cb, int rw, bool rope) { return tree_pair(cb, rw, rope) ? 4 : (tree_split(cb, rw, rope) ? tree_threads(cb, rw, rope) / 256 : 2); }
constexpr int tree_smem(int cb, int rw, bool rope) {
    if (tree_pair(cb, rw, rope)) return kPairLow + rw * 4096;
    return kTreeLead + (cb == 2 ? kTreeWaves * cb * 2048 : 2 * kTile * kD * 2);
}

// Block: rows [rows_pb rb, ..) over one run of 64-token tiles, unit by unit. While tile t is attended, eight wavefronts (all, or
// those that only make) make tile t + 1: wavefront w rebuilds the keys of token block w / 2, feature pairs of half w % 2
// (K^T = P_K^T Z^T), rotates them, and unpacks the values of N-tile w, all to LDS in operand order. Wavefront (rw, tw) of RW x 8 / RW
// (or of RW that only attend) takes rows 16 CB rw .. and the tw-th part of the tile's tokens: S^T = K Q^T, the online softmax,
// O^T += Z_V^T P^T.
// Key row m of block tb is the token whose value sits in slot (tb, m % 4) of quarter m / 4, so that the lane that computes
// a weight is the lane whose operand needs it.
// A rotated key is fp16 and the rest of it bf8 at 2^11 times its size, met by the queries' leading bits (e5m2 is fp16's upper byte):
// logits keep about 14 bits of the key for a quarter more matrix work, where fp16 alone would put an error of 2^-12 of
// each coordinate into the weights. (The query is cut, not rounded, to its upper byte: up to 2^-2 of a rest's share is lost, and
// more below 2^-14, where an fp16 number has fewer leading bits. Measured, logits are a ninth as far off as with fp16 alone.)
// Keys that are not rotated are not rebuilt: q . k = (P_K q) . z up to the step, so a piece begins by projecting its queries (kept
// as the sum of two fp16, 2^-22 off; each query at a scale of its own, its largest element in [1, 2), since the second fp16 of
// a small one would be below that type's range), a wavefront makes tile t + 1 by unpacking half of a token block's codes, and
// the products are of codes and projections. Twice the matrix steps for the scores, but the making is a quarter: 52 rows x 16k
// x 64 units 95 us rebuilt and rotated, 69 so; 256 rows x 16k 179 and 154.
// NV: N-tiles of values, so that ranks up to 64 and 96 do no products for the rest.
template <int CB, int RW, bool ROPE, int NV>
__device__ __forceinline__ void tree_piece(const DevSide& K, const DevSide& V, const uint16_t* __restrict__ q, const TreeWork& wk,
                                           const TreeRope& rope, int u, int T, int tile0, int tile1, int rb, int64_t slot,
                                           float* __restrict__ acc_out, float2* __restrict__ ml_out) {
    constexpr bool kPair = tree_pair(CB, RW, ROPE), kSplit = tree_split(CB, RW, ROPE);
    constexpr bool kShare = ROPE && CB == 1;
    // kShare: the two wavefronts of a token block unpack half of its key codes each, a tile ahead, and meet in LDS behind the
    // buffers (64 rows x 128k 134 -> 126 us, 100 rows x 16k 140 -> 136; with 32 rows a wavefront LDS has no room).
    constexpr int kBuf = kPair ? 0 : kTreeBuf, kBufV = ROPE ? kTreeBufV : kTile * kD * 2, kBufBytes = ROPE ? kTreeBufBytes : kTile * kD * 4;
    constexpr int NW = kSplit ? RW : kTreeWaves, TW = NW / RW, TB = 4 / TW;  // token parts, and key blocks of one
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));  // opaque: a lane's addresses are formed again for every piece, not kept across all of them
    const int wv = uni(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;
    const bool maker = !kSplit || wv < kTreeWaves, attends = !kSplit || wv >= kTreeWaves;  // roles of the wavefront
    const int aw = kSplit ? max(wv - kTreeWaves, 0) : wv, rw = aw % RW, tw = aw / RW;
    const int row0 = rb * wk.rows_pb + 16 * CB * rw;  // the wavefront's rows
    const int64_t prow = slot * wk.M;
    const int rk = uni(K.r[u]), bk = uni(K.b[u]), rv = uni(V.r[u]), bv = uni(V.b[u]);
    uint8_t* sm = kvc_dsm;
    float2* adv = reinterpret_cast<float2*>(sm + kTreeAdv);
    float* mid = reinterpret_cast<float*>(sm + kTreeMid);
    const uint8_t* kstream = uni(K.codes + K.code_off[u]);
    const uint8_t* vstream = uni(V.codes + V.code_off[u]);
    const int ktb = 8 * rk * bk, vtb = 8 * rv * bv;
    const auto krs = __builtin_amdgcn_make_buffer_rsrc((void*)kstream, (short)0, wk.k_cap_tiles * ktb, kRsrcWord3);
    const auto vrs = __builtin_amdgcn_make_buffer_rsrc((void*)vstream, (short)0, wk.v_cap_tiles * vtb, kRsrcWord3);
    const uint32_t e512 = exp512();
    const int g16 = rk >> 4, rho = rk & 15, nk = (rk + 63) >> 6, nvt = (rv + 15) >> 4;
    const int fh = wv & 1, kb = wv >> 1;  // the feature half and token block that the wavefront rebuilds
    const int ktok = 16 * (col >> 2) + tree_tok(bv, kb, col & 3);
    constexpr int KU = ROPE && !kShare ? 2 : 1;  // 64-coordinate parts of the keys' codes that a wavefront unpacks: all, or part fh
    uint32_t xk[KU];
    PlaneAt ka[KU];
    uint32_t kw[KU][kFieldWords] = {}, vw[4] = {};
#pragma unroll
    for (int ks = 0; ks < KU; ++ks) {
        const int cg = 4 * (KU > 1 ? ks : fh) + grp;  // a group past the rank reads the first one (its columns of P_K^T are zero)
        xk[ks] = cg < g16 ? (uint32_t)(1024 * cg + 16 * ktok) : (cg == g16 && rho ? (uint32_t)(1024 * g16 + ktok * rho) : (uint32_t)(g16 ? 16 * ktok : rho * ktok));
        ka[ks] = tree_k_at(bk, rk, xk[ks]);
    }
    const PlaneAt va = tree_v_at(bv, rv, wv, col, grp);
    auto load_k = [&](int tile) {
        if constexpr (KU > 1) {
            tree_k_load(krs, tile * ktb, bk, ka[0], kw[0]);
            if (nk > 1) tree_k_load(krs, tile * ktb, bk, ka[KU - 1], kw[KU - 1]);
        } else if (fh < nk) {
            tree_k_load(krs, tile * ktb, bk, ka[0], kw[0]);
        }
    };
    auto load_v = [&](int tile) {
        if (wv < nvt) tree_v_load(vrs, tile * vtb, bv, va, vw);
    };
    // The basis and the queries are requested first, then the first tile's codes.
    constexpr int kBasisItems = kD * kD / 8 / kTreeThreads;
    static_assert(kBasisItems == 4 && kBtItems == kTreeThreads);
    const uint16_t* Pg = K.basis + K.basis_off[u];
    uint4 pr[kBasisItems];
    if constexpr (ROPE) {
        if (maker) basis_t_load<KVC_SIDE_K>(pr, Pg, rk, basis_item(tid));
    } else {
#pragma unroll
        for (int j = 0; j < kBasisItems; ++j) {
            const int e = tid + j * kTreeThreads;
            pr[j] = uint4{0u, 0u, 0u, 0u};
            if (e < rk * (kD / 8)) pr[j] = load_basis8(Pg + 8 * e);
        }
    }
    // Queries: columns of the operand. Rotated keys: features in the order of the rebuilt keys, and their leading bits.
    // Plain keys: the projections onto the basis, in the order of the unpacked codes, as the sum of two fp16 (2^-22 of them)
    constexpr int QW = ROPE || kPair ? 1 : 2;  // parts held in registers
    uint8_t* low = sm + kPairLow + rw * 4096 + lane * 16;
    uint8_t* lead = sm + kTreeLead + wv * CB * 2048 + lane * 16;
    rc_h8 qr[CB][4], qf[QW][CB][4];
    v8i q1 = {};
    float base[CB];  // the centre's share of a row's raw products, -(2^(b-1) - 1/2) sum_i q_i
    float qexp[CB];  // plain keys: the power of two that the row's projection is divided by
    if (attends)
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int row = row0 + 16 * cb + col;
            const uint16_t* qp = q + ((int64_t)u * wk.M + (row < wk.M ? row : 0)) * kD;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                uint4 x;
                if constexpr (ROPE) {
                    const uint2 a = *reinterpret_cast<const uint2*>(qp + 4 * grp + 32 * ks), b = *reinterpret_cast<const uint2*>(qp + 4 * grp + 32 * ks + 16);
                    x = uint4{a.x, a.y, b.x, b.y};
                } else {
                    x = *reinterpret_cast<const uint4*>(qp + 8 * grp + 32 * ks);
                }
                if (row >= wk.M) x = uint4{0u, 0u, 0u, 0u};
                qr[cb][ks] = __builtin_bit_cast(rc_h8, x);
            }
        }
    if (maker) {
        load_k(tile0);
        load_v(tile0);
    }
    if constexpr (ROPE) {
        if (maker) basis_t_store(sm, pr, basis_item(tid));
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) qf[0][cb][ks] = qr[cb][ks];
            const v8i r = lead_bits(qr[cb]);
            if constexpr (CB == 1) {
                q1 = r;
            } else {  // for this wavefront alone
                *reinterpret_cast<v4i*>(lead + cb * 2048) = v4i{r[0], r[1], r[2], r[3]};
                *reinterpret_cast<v4i*>(lead + cb * 2048 + 1024) = v4i{r[4], r[5], r[6], r[7]};
            }
            base[cb] = 0.f;
        }
        if (tid < kD / 2) {
            const double t = (double)kTile * rope.freq[tid];
            const float f = (float)(t - rint(t));
            adv[tid] = float2{__builtin_amdgcn_cosf(f), __builtin_amdgcn_sinf(f)};
        }
        __syncthreads();  // P_K^T
        // the centre's share of a key, -(2^(b-1) - 1/2) sum_i P_i: features 16 wv + 4 grp + v, in every column
        const _Float16 c = (_Float16)(0.5f - (float)(1 << (bk - 1)));
        const rc_h8 cc = {c, c, c, c, c, c, c, c};
        rc_f4 a = rc_f4{0.f, 0.f, 0.f, 0.f};
        if (maker)
#pragma unroll
            for (int s = 0; s < 4; ++s) a = mfma_h(*reinterpret_cast<const rc_h8*>(sm + bt_block(wv, s) + bt_lane(col, grp)), cc, a);
        if (maker && col == 0) *reinterpret_cast<rc_f4*>(mid + 16 * wv + 4 * grp) = a * (1.f / kRawScale);
        __syncthreads();
    } else {
        // Rows of P_K, eight features to a chunk; a row's chunks are turned by four for every sixteen rows, since a read takes
        // rows i, i + 1, i + 2, i + 3 and those 16, 32 and 48 further.
        uint16_t* Pl = reinterpret_cast<uint16_t*>(sm);
        auto chunk = [&](int i, int c8) { return Pl + i * kTreePRow + 8 * ((c8 + 4 * (i >> 4)) & 15); };
#pragma unroll
        for (int j = 0; j < kBasisItems; ++j) {
            const int e = tid + j * kTreeThreads;
            *reinterpret_cast<uint4*>(chunk(e >> 4, e & 15)) = pr[j];
        }
        __syncthreads();
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {  // of the row's largest element, its four lanes together
            typedef uint16_t us2 __attribute__((ext_vector_type(2)));
            us2 most = {0, 0};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int d = 0; d < 4; ++d)
                    most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, __builtin_bit_cast(v4u, qr[cb][ks])[d] & 0x7fff7fffu));
            int x = max((int)most[0], (int)most[1]);
            x = max(x, __shfl_xor(x, 16));
            x = max(x, __shfl_xor(x, 32));
            qexp[cb] = x ? __uint_as_float(__float_as_uint(h2f((uint16_t)x)) & 0x7f800000u) : 1.f;
        }
        // matrix step ks of the scores: coordinates 64 (ks / 2) + 16 grp + 4 (ks % 2) + v, and 8 further
        auto project = [&](int ks, int cb, rc_h8& hi, rc_h8& lo) {
            rc_f4 d[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int i = 64 * (ks >> 1) + 16 * (col >> 2) + 4 * (ks & 1) + (col & 3) + 8 * h;
                d[h] = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int fs = 0; fs < 4; ++fs) d[h] = mfma_h(*reinterpret_cast<const rc_h8*>(chunk(i, 4 * fs + grp)), qr[cb][fs], d[h]);
            }
            const float down = __uint_as_float(0x7f000000u - __float_as_uint(qexp[cb]));  // 1 / qexp
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = d[e & 1][e >> 1] * down;
                hi[e] = (_Float16)x;
                lo[e] = (_Float16)(x - (float)hi[e]);
            }
        };
        rc_h8 ql[CB][4];
        if constexpr (kPair) {  // the wavefronts of the same rows share the steps (TW is 2 or 4), by way of the second buffer
            uint8_t* high = sm + kPairLow - RW * 4096 + rw * 4096 + lane * 16;
#pragma unroll 1
            for (int ks = tw; ks < 2 * nk; ks += TW) {
                rc_h8 hi, lo;
                project(ks, 0, hi, lo);
                *reinterpret_cast<rc_h8*>(high + 1024 * ks) = hi;
                *reinterpret_cast<rc_h8*>(low + 1024 * ks) = lo;
            }
            __syncthreads();  // and P_K has been read: its place is the first tile's
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                qf[0][0][ks] = ql[0][ks] = rc_h8{};
                if (ks < 2 * nk) {
                    qf[0][0][ks] = *reinterpret_cast<const rc_h8*>(high + 1024 * ks);
                    ql[0][ks] = *reinterpret_cast<const rc_h8*>(low + 1024 * ks);
                }
            }
        } else {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) {
                    project(ks, cb, qf[0][cb][ks], ql[cb][ks]);
                    qf[QW - 1][cb][ks] = ql[cb][ks];
                }
        }
        const _Float16 c = (_Float16)(0.5f - (float)(1 << (bk - 1)));
        const rc_h8 cc = {c, c, c, c, c, c, c, c};
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            rc_f4 sum = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) {
                sum = mfma_h(cc, qf[0][cb][ks], sum);
                sum = mfma_h(cc, ql[cb][ks], sum);
            }
            base[cb] = sum[0] * (1.f / kRawScale);
        }
    }
    // step_K log2(e) / sqrt(128), and what scales a raw product of the row
    const float unit = K.delta[u] * 1.4426950408889634f * 0.08838834764831845f;
    float qs[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) qs[cb] = ROPE ? unit : unit * kRawScale * qexp[cb];
    // What a row's scores start from: the centre's share less the running maximum, so that the accumulators hold S - m. (Taken off
    // afterwards it would have to be exact in the sum with the weights' shift: past 2^24 its rounding alone passes their range.)
    float start[CB];
    bool fresh = true;  // no maximum yet
    rc_f4 O[NV][CB], L[CB];
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
        start[cb] = base[cb];
        L[cb] = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int n = 0; n < NV; ++n) O[n][cb] = L[cb];
    }
    uint32_t toks[TB];  // the tokens of key rows 4 grp + v of the wavefront's blocks, v by byte, less 16 grp
#pragma unroll
    for (int t = 0; t < TB; ++t) {
        toks[t] = 0;
#pragma unroll
        for (int v = 0; v < 4; ++v) toks[t] |= (uint32_t)tree_tok(bv, TB * tw + t, v) << (8 * v);
    }
    const _Float16 h1 = (_Float16)1.f;
    const rc_h8 ones = {h1, h1, h1, h1, h1, h1, h1, h1};
    float cs[2][4], sn[2][4];  // of the lane's pairs 32 fh + 16 i + 4 grp + v at its token's position, times kRawScale

    // the wavefront's part of a tile's key codes to LDS, a tile before they are needed
    auto unpack = [&](int tile) {
        if (fh < nk) {
            rc_h8 zz[2];
            tree_k_frag(kw[0], bk, xk[0], zz);
            uint8_t* dst = sm + kTreeLead + ((tile - tile0) & 1) * 16384 + 8192 * fh + 1024 * kb + lane * 16;
            *reinterpret_cast<rc_h8*>(dst) = zz[0];
            *reinterpret_cast<rc_h8*>(dst + 4096) = zz[1];
        }
        if (tile + 1 < tile1) load_k(tile + 1);
    };
    if constexpr (kShare) {
        if (maker) unpack(tile0);
        __syncthreads();
    }
    // keys and values of a tile to a buffer; the codes of the tile after it are requested
    auto make = [&](int tile, uint8_t* buf) {
        rc_h8 z[4], vz[2];
        if constexpr (ROPE) {
            if ((tile - tile0) % kTreeResync == 0) {
                const double pos = (double)(tile * kTile + ktok);
                int p0 = 32 * fh + 4 * grp;
                asm volatile("" : "+v"(p0));  // opaque: the frequencies are read again, not kept across tiles
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const double t = pos * rope.freq[p0 + 16 * i + v];
                        const float f = (float)(t - rint(t));
                        cs[i][v] = kRawScale * __builtin_amdgcn_cosf(f);
                        sn[i][v] = kRawScale * __builtin_amdgcn_sinf(f);
                    }
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float2 a = adv[32 * fh + 16 * i + 4 * grp + v];
                        const float sy = sn[i][v] * a.y, cy = cs[i][v] * a.y;
                        fma_in_place(cs[i][v], a.x, -sy);
                        fma_in_place(sn[i][v], a.x, cy);
                    }
            }
        }
        if constexpr (kShare) {
            const uint8_t* src = sm + kTreeLead + ((tile - tile0) & 1) * 16384 + 1024 * kb + lane * 16;
            z[0] = *reinterpret_cast<const rc_h8*>(src);
            z[1] = *reinterpret_cast<const rc_h8*>(src + 4096);
            if (nk > 1) {
                z[2] = *reinterpret_cast<const rc_h8*>(src + 8192);
                z[3] = *reinterpret_cast<const rc_h8*>(src + 12288);
            }
            if (tile + 1 < tile1) unpack(tile + 1);
        } else if constexpr (ROPE) {
            rc_h8 zz[2];
            tree_k_frag(kw[0], bk, xk[0], zz);
            z[0] = zz[0];
            z[1] = zz[1];
            if (nk > 1) {
                tree_k_frag(kw[KU - 1], bk, xk[KU - 1], zz);
                z[2] = zz[0];
                z[3] = zz[1];
            }
        } else if (fh < nk) {
            rc_h8 zz[2];
            tree_k_frag(kw[0], bk, xk[0], zz);
            uint8_t* dst = buf + 8192 * fh + (64 * grp + 16 * kb + col) * 16;
            *reinterpret_cast<rc_h8*>(dst) = zz[0];
            *reinterpret_cast<rc_h8*>(dst + 4096) = zz[1];
        }
        if (wv < nvt) {
            tree_v_frag(vw, bv, e512, vz);
            *reinterpret_cast<rc_h8*>(buf + kBufV + wv * 2048 + lane * 16) = vz[0];
            *reinterpret_cast<rc_h8*>(buf + kBufV + wv * 2048 + 1024 + lane * 16) = vz[1];
        }
        if (tile + 1 < tile1) {
            if constexpr (!kShare) load_k(tile + 1);
            load_v(tile + 1);
        }
        if constexpr (!ROPE) return;
        int po = bt_lane(col, grp) + bt_block(2 * fh, 0);
        asm volatile("" : "+v"(po));  // opaque: P_K^T is read again for every tile and takes no registers in between
        const uint8_t* pt = sm + po;
        rc_f4 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = *reinterpret_cast<const rc_f4*>(mid + 16 * (2 * fh + i) + 4 * grp);
            b[i] = *reinterpret_cast<const rc_f4*>(mid + 16 * (2 * fh + i + 4) + 4 * grp);
        }
        auto rebuild = [&](auto first) {  // matrix steps `first` and `first` + 1: eight operands in flight
            constexpr int s0 = decltype(first)::value;
            rc_h8 p[2][4];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) p[s][i] = *reinterpret_cast<const rc_h8*>(pt + bt_block(i + (i & 2), s0 + s));
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    a[i] = mfma_h(p[s][i], z[s0 + s], a[i]);
                    b[i] = mfma_h(p[s][i + 2], z[s0 + s], b[i]);
                }
        };
        rebuild(std::integral_constant<int, 0>());
        if (nk > 1) rebuild(std::integral_constant<int, 2>());
        rc_h8 hx, hy;
        float m1 = -1.f;
        asm volatile("" : "+s"(m1));  // opaque: x - hi stays one mixed-precision multiply-add that reads the half
        int lx[2] = {0, 0}, ly[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float x[4], y[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                x[v] = fmaf(a[i][v], cs[i][v], -b[i][v] * sn[i][v]);
                y[v] = fmaf(a[i][v], sn[i][v], b[i][v] * cs[i][v]);
            }
#pragma unroll
            for (int v = 0; v < 4; v += 2) {
                const rc_h2 h = to_half2(x[v], x[v + 1]), g = to_half2(y[v], y[v + 1]);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    hx[4 * i + v + e] = h[e];
                    hy[4 * i + v + e] = g[e];
                    x[v + e] = fmaf((float)h[e], m1, x[v + e]);
                    y[v + e] = fmaf((float)g[e], m1, y[v + e]);
                }
            }
            lx[i] = __builtin_bit_cast(int, bf8_pairs(x));
            ly[i] = __builtin_bit_cast(int, bf8_pairs(y));
        }
        uint8_t* dst = buf + (64 * grp + 16 * kb + col) * 16;
        *reinterpret_cast<rc_h8*>(dst + 4096 * fh) = hx;
        *reinterpret_cast<rc_h8*>(dst + 4096 * (fh + 2)) = hy;
        *reinterpret_cast<int2*>(dst + kBufLo + 8 * fh) = int2{lx[0], lx[1]};
        *reinterpret_cast<int2*>(dst + kBufLo + 4096 + 8 * fh) = int2{ly[0], ly[1]};
    };
    // the wavefront's rows against its tokens of a tile
    auto attend = [&](int tile, const uint8_t* buf) {
        const int tb0 = TB * tw;  // first key block of the wavefront's tokens
        // ---- scores: the low parts first. Operands are read kAhead products ahead; the order is fixed by hand (left to itself the
        // compiler saves registers and waits for each read).
        rc_f4 S[TB][CB];
        if constexpr (ROPE) {
            constexpr int kAhead = 4;
            const uint8_t* kr = buf + (64 * grp + 16 * tb0 + col) * 16;
            auto key = [&](int i) { return *reinterpret_cast<const rc_h8*>(kr + 4096 * (i / TB) + 256 * (i % TB)); };
            constexpr int kLo = kSplit && TB > 2 ? 2 : TB;  // low parts read ahead
            v4i l0[kLo], l1[kLo];
            rc_h8 kf[kAhead];
            auto low_part = [&](int t) {
                l0[t % kLo] = *reinterpret_cast<const v4i*>(kr + kBufLo + 256 * t);
                l1[t % kLo] = *reinterpret_cast<const v4i*>(kr + kBufLo + 4096 + 256 * t);
            };
#pragma unroll
            for (int t = 0; t < kLo; ++t) low_part(t);
            v8i q8[CB];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                if constexpr (CB == 1) {
                    q8[cb] = q1;
                } else {
                    const v4i a = *reinterpret_cast<const v4i*>(lead + cb * 2048), b = *reinterpret_cast<const v4i*>(lead + cb * 2048 + 1024);
                    q8[cb] = v8i{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
                }
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int t = 0; t < TB; ++t) {
                const v4i a = l0[t % kLo], b = l1[t % kLo];
                const v8i lo = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) S[t][cb] = mfma_lo(lo, q8[cb], rc_f4{start[cb], start[cb], start[cb], start[cb]});
                if (t + kLo < TB) low_part(t + kLo);
#pragma unroll
                for (int i = kAhead * t / TB; i < kAhead * (t + 1) / TB; ++i) kf[i] = key(i);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < 4 * TB; ++i) {
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) S[i % TB][cb] = mfma_h(kf[i % kAhead], qf[0][cb][i / TB], S[i % TB][cb]);
                if (i + kAhead < 4 * TB) kf[i % kAhead] = key(i + kAhead);
                __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const uint8_t* kr = buf + (64 * grp + 16 * tb0 + col) * 16;
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) S[t][cb] = rc_f4{start[cb], start[cb], start[cb], start[cb]};
            auto part = [&](auto first) {  // matrix steps `first` and `first` + 1
                constexpr int s0 = decltype(first)::value;
                rc_h8 kf[2 * TB], lw[2];
                if constexpr (kPair)
#pragma unroll
                    for (int i = 0; i < 2; ++i) lw[i] = *reinterpret_cast<const rc_h8*>(low + 1024 * (s0 + i));
#pragma unroll
                for (int i = 0; i < 2 * TB; ++i) kf[i] = *reinterpret_cast<const rc_h8*>(kr + 4096 * (s0 + i / TB) + 256 * (i % TB));
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int i = 0; i < 2 * TB; ++i)
#pragma unroll
                    for (int w = 0; w < 2; ++w)
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb)
                            S[i % TB][cb] = mfma_h(kf[i], kPair && w ? lw[i / TB] : qf[w && !kPair ? QW - 1 : 0][cb][s0 + i / TB], S[i % TB][cb]);
            };
            part(std::integral_constant<int, 0>());
            if (nk > 1) part(std::integral_constant<int, 2>());
        }
        if ((tile + 1) * kTile > T) {  // the context's last tile
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if (tile * kTile + 16 * grp + (int)(toks[t] >> (8 * v) & 255u) >= T)
#pragma unroll
                        for (int cb = 0; cb < CB; ++cb) S[t][cb][v] = -INFINITY;
        }
        // ---- online softmax
        constexpr int NS = TB > 1 ? TB / 2 : 1;  // halves of a tile: one or two
        const uint8_t* vr = buf + kBufV + (tb0 >> 1) * 1024 + lane * 16;
        constexpr int AV = tree_waves_per_simd(CB, RW, ROPE) == 4 && NV > 4 ? 4 : NV;  // operands read ahead
        auto value = [&](int k) { return *reinterpret_cast<const rc_h8*>(vr + k / NV * 1024 + k % NV * 2048); };  // of the first half, then of the second
        rc_h8 vf[AV];  // N-tiles past the rank make rows that are not stored
#pragma unroll
        for (int n = 0; n < AV; ++n) vf[n] = value(n);
        float top[CB];
        bool raise = false;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            top[cb] = S[0][cb][0];
#pragma unroll
            for (int t = 0; t < TB; ++t)
#pragma unroll
                for (int v = 0; v < 4; ++v) top[cb] = fmaxf(top[cb], S[t][cb][v]);
            raise = raise || top[cb] * qs[cb] > kTreeLazy;
        }
        if (__any(raise) || fresh) {
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) {
                float t = fmaxf(top[cb], __shfl_xor(top[cb], 16));
                t = fmaxf(t, __shfl_xor(t, 32));
                t = fresh ? (t == -INFINITY ? 0.f : t) : fmaxf(t, 0.f);  // (nothing seen: a part of a short last tile)
                const float al = fresh ? 1.f : __builtin_amdgcn_exp2f(-t * qs[cb]);
                start[cb] -= t;
                L[cb] *= al;
#pragma unroll
                for (int n = 0; n < NV; ++n) O[n][cb] *= al;
#pragma unroll
                for (int i = 0; i < TB; ++i) S[i][cb] -= t;
            }
            fresh = false;
        }
        // ---- weights and values: the second half's weights and operands while the first half multiplies
        auto weight = [&](int s, int cb, int e) { return __builtin_amdgcn_exp2f(fmaf(S[TB > 1 ? 2 * s + (e >> 2) : 0][cb][e & 3], qs[cb], kTreeShift)); };
        rc_h8 P[CB];
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            if constexpr (TB == 1) P[cb] = rc_h8{};
#pragma unroll
            for (int e = 0; e < (TB > 1 ? 8 : 4); ++e) P[cb][e] = (_Float16)weight(0, cb, e);
            if constexpr (TB == 1)
                if (tb0 & 1) P[cb] = __builtin_shufflevector(P[cb], P[cb], 4, 5, 6, 7, 0, 1, 2, 3);
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) L[cb] = mfma_h(ones, P[cb], L[cb]);
        if constexpr (NS == 1) {
#pragma unroll
            for (int n = 0; n < NV; ++n) {
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) O[n][cb] = mfma_h(vf[n % AV], P[cb], O[n][cb]);
                if (n + AV < NV) vf[n % AV] = value(n + AV);
            }
        } else {
            float w1[CB][8];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) O[n][cb] = mfma_h(vf[n % AV], P[cb], O[n][cb]);
                vf[n % AV] = value(n + AV);
#pragma unroll
                for (int i = 8 * CB * n / NV; i < 8 * CB * (n + 1) / NV; ++i) w1[i >> 3][i & 7] = weight(1, i >> 3, i & 7);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int cb = 0; cb < CB; ++cb)
#pragma unroll
                for (int e = 0; e < 8; ++e) P[cb][e] = (_Float16)w1[cb][e];
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) L[cb] = mfma_h(ones, P[cb], L[cb]);
#pragma unroll
            for (int n = 0; n < NV; ++n) {
#pragma unroll
                for (int cb = 0; cb < CB; ++cb) O[n][cb] = mfma_h(vf[(NV + n) % AV], P[cb], O[n][cb]);
                if (n + AV < NV) vf[(NV + n) % AV] = value(NV + n + AV);
            }
        }
    };
    auto buffer = [&](int tile) { return sm + kBuf + ((tile - tile0) & 1) * kBufBytes; };
    if constexpr (kSplit) {
        if (maker) {
#pragma unroll 1
            for (int tile = tile0; tile <= tile1; ++tile) {
                if (tile < tile1) make(tile, buffer(tile));
                __syncthreads();
            }
        } else {
#pragma unroll 1
            for (int tile = tile0; tile <= tile1; ++tile) {
                if (tile > tile0 && row0 < wk.M) attend(tile - 1, buffer(tile - 1));
                __syncthreads();
            }
        }
    } else {
        const bool late = wv >= kTreeWaves / 2;
#pragma unroll 1
        for (int tile = tile0 - 1; tile < tile1; ++tile) {
            // One wavefront of each SIMD makes the next tile and then attends to the current one, the other (late) the other way
            // round, so that the matrix and vector work of the two overlap: the late ones meet the barrier between the two. (256
            // rows x 32k x 64 units: all in one order 471 us, so 353, when the rest of the kernel was simpler.)
            if (tile + 1 < tile1) make(tile + 1, buffer(tile + 1));
            if (late) __syncthreads();
            const int at = late ? tile + 1 : tile;
            if (at >= tile0 && at < tile1 && row0 < wk.M) attend(at, buffer(at));
            if (!late) __syncthreads();
        }
    }
    float m[CB];  // maxima of the raw products; a row whose weights sum to nothing has seen no token
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) m[cb] = L[cb][0] == 0.f ? -INFINITY : base[cb] - start[cb];
    if constexpr (TW == 1) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
            const int row = row0 + 16 * cb + col;
            if (!attends || row >= wk.M) continue;
            if (grp == 0) ml_out[prow + row] = float2{fmaf(m[cb], qs[cb], -kTreeShift), L[cb][0]};
#pragma unroll
            for (int n = 0; n < NV; ++n)
                if (n < nvt) *reinterpret_cast<rc_f4*>(acc_out + (prow + row) * kD + 16 * n + 4 * grp) = O[n][cb];
        }
    } else {  // the token parts meet in LDS (the tiles' buffers)
        static_assert(CB == 1 && !kSplit, "token parts have sixteen rows a wavefront, of every wavefront");
        constexpr int kPitch = kD + 4;
        float* parts = reinterpret_cast<float*>(sm + kBuf);             // [TW][16 RW][kPitch]
        float* tops = parts + NW * 16 * kPitch;                     // [TW][16 RW]
        float* sums = tops + NW * 16;                               // [TW][16 RW]
        static_assert((NW * 16 * (kPitch + 2)) * 4 <= tree_smem(CB, RW, ROPE) - kBuf, "parts exceed the buffers");
        __syncthreads();  // the late wavefronts have read their last tile
        if (grp == 0) tops[16 * wv + col] = m[0];  // wavefronts are in the order (tw, rw)
        __syncthreads();
        float t = tops[16 * rw + col];
#pragma unroll
        for (int i = 1; i < TW; ++i) t = fmaxf(t, tops[16 * (RW * i + rw) + col]);
        const float al = m[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m[0] - t) * qs[0]);
        if (grp == 0) sums[16 * wv + col] = al * L[0][0];
#pragma unroll
        for (int n = 0; n < NV; ++n)
            if (n < nvt) *reinterpret_cast<rc_f4*>(parts + (16 * wv + col) * kPitch + 16 * n + 4 * grp) = O[n][0] * al;
        __syncthreads();
        if (tw == 0 && grp == 0 && row0 + col < wk.M) {
            float l = sums[16 * rw + col];
#pragma unroll
            for (int i = 1; i < TW; ++i) l += sums[16 * (RW * i + rw) + col];
            ml_out[prow + row0 + col] = float2{fmaf(t, qs[0], -kTreeShift), l};
        }
        for (int e = tid; e < 16 * RW * (kD / 4); e += kTreeThreads) {
            const int r = e / (kD / 4), c4 = e % (kD / 4) * 4;
            const int row = rb * wk.rows_pb + r;
            if (c4 >= 16 * nvt || row >= wk.M) continue;
            rc_f4 x = *reinterpret_cast<const rc_f4*>(parts + r * kPitch + c4);
#pragma unroll
            for (int i = 1; i < TW; ++i) x += *reinterpret_cast<const rc_f4*>(parts + (16 * RW * i + r) * kPitch + c4);
            *reinterpret_cast<rc_f4*>(acc_out + (prow + row) * kD + c4) = x;
        }
    }
}

template <int CB, int RW, bool ROPE>
__global__ __launch_bounds__(tree_threads(CB, RW, ROPE)) __attribute__((
    amdgpu_waves_per_eu(tree_waves_per_simd(CB, RW, ROPE), tree_waves_per_simd(CB, RW, ROPE)))) void tree_partial_kernel(
    DevSide K, DevSide V, const uint16_t* __restrict__ q, const int32_t* __restrict__ seq_len, TreeWork wk, TreeRope rope,
    float* __restrict__ acc_out, float2* __restrict__ ml_out) {
    constexpr int kThreads = tree_threads(CB, RW, ROPE), kWaves = kThreads / 64;
    const int rb = blockIdx.x % wk.nrb, b = blockIdx.x / wk.nrb;
    const int tid = threadIdx.x, lane = tid & 63, wv = uni(tid >> 6);
    // the block's run of tiles and where it begins: a thread counts the tiles of some consecutive units
    uint32_t* waves = reinterpret_cast<uint32_t*>(kvc_dsm);  // tiles of each wavefront's units, then the first unit and tile
    const int cu = (wk.U + kThreads - 1) / kThreads, u_lo = min(wk.U, tid * cu), u_hi = min(wk.U, u_lo + cu);
    uint32_t mine = 0;
    for (int i = u_lo; i < u_hi; ++i) mine += unit_work(unit_tiles(seq_len, i, wk.max_seq), wk.M);
    uint32_t upto = mine;  // within the wavefront
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 63) waves[wv] = upto;
    __syncthreads();
    uint32_t total = 0, before = upto - mine;
    for (int i = 0; i < kWaves; ++i) {
        if (i < wv) before += waves[i];
        total += waves[i];
    }
    const uint32_t per = run_tiles(total, wk.n_blocks);
    const uint32_t g = min(total, per * b), g1 = min(total, g + per);
    if (g >= g1) return;
    if (g >= before && g < before + mine) {
        int u = u_lo;
        uint32_t at = before;
        for (uint32_t n; at + (n = unit_work(unit_tiles(seq_len, u, wk.max_seq), wk.M)) <= g; ++u) at += n;
        waves[kWaves] = u;
        waves[kWaves + 1] = g - at;
    }
    __syncthreads();
    int u = uni((int)waves[kWaves]), x0 = uni((int)waves[kWaves + 1]);  // the run begins at x0 of unit u
    int left = uni((int)(g1 - g));
#pragma unroll 1
    for (; left > 0; ++u, x0 = 0) {
        const int T = uni(unit_tokens(seq_len, u, wk.max_seq)), tiles = (T + kTile - 1) / kTile;
        const int x1 = min((int)unit_work(tiles, wk.M), x0 + left);
        left -= x1 - x0;
        const int t0 = max(x0 - start_cost(wk.M), 0), t1 = x1 - start_cost(wk.M);
        if (t1 <= t0) continue;
        __syncthreads();  // LDS of the piece before, or of the count above, has been read
        const int rv = uni(V.r[u]);
        if (rv <= 64) tree_piece<CB, RW, ROPE, 4>(K, V, q, wk, rope, u, T, t0, t1, rb, (int64_t)b + u, acc_out, ml_out);
        else if (rv <= 96) tree_piece<CB, RW, ROPE, 6>(K, V, q, wk, rope, u, T, t0, t1, rb, (int64_t)b + u, acc_out, ml_out);
        else tree_piece<CB, RW, ROPE, 8>(K, V, q, wk, rope, u, T, t0, t1, rb, (int64_t)b + u, acc_out, ml_out);
    }
}

// ---------------------------------------------------------------- drafted tokens, merge, output

constexpr int kFinThreads = 256;
constexpr int kFinRows = 16;
constexpr int kFinZ = kBtBytes;                              // LDS: P_V^T, then z [16][132] f32
constexpr int kFinZPitch = kD + 4;
constexpr int kFinX = kFinZ + kFinRows * kFinZPitch * 4;     // drafted values [64][136] fp16
constexpr int kFinXPitch = kD + 8;
constexpr int kFinP = kFinX + KVC_TREE_MAX_TOKENS * kFinXPitch * 2;  // weights [16][72] fp16
constexpr int kFinPPitch = KVC_TREE_MAX_TOKENS + 8;
constexpr int kFinRed = kFinP + kFinRows * kFinPPitch * 2;   // maxima and sums of the wavefronts [2][4][16], drafts' maxima, both parts' factors [16]
constexpr int kFinCount = kFinRed + (2 * 4 * 16 + 48) * 4;    // [8] tiles
constexpr int kFinSmem = kFinCount + 8 * 4;
static_assert(kFinSmem <= 64 * 1024, "no attribute is set for it");

// Block: R rows of one unit (columns of the products past R repeat the last row). Cached tokens: z = sum_c acc_c 2^(m_c - M) over
// the unit's pieces, by its own sum l; drafted ones: weights p_m = 2^(s - D) of their own maximum D; out = a step_V P_V^T z / l +
// b sum_m p_m xv_m, with the parts' factors a and b in fp32, so that neither part's fp16 operands lose bits where the other
// takes nearly all of the weights. With few rows in all, blocks of four rows, whose threads also share the pieces. Bound by
// latency, a chain of four reads of memory (8 to 10 us up to 64 rows x 64 units), and at 256 rows by the pieces' 42 MB.
template <int R>
__global__ __launch_bounds__(kFinThreads) void tree_finish_kernel(DevSide V, const uint16_t* __restrict__ q, int G, int n_tok,
                                                                  const uint16_t* __restrict__ xk, int64_t xk_stride,
                                                                  const uint16_t* __restrict__ xv, int64_t xv_stride,
                                                                  const uint64_t* __restrict__ mask, const int32_t* __restrict__ seq_len,
                                                                  TreeWork wk, int groups, const float* __restrict__ acc,
                                                                  const float2* __restrict__ ml, uint16_t* __restrict__ out) {
    constexpr int CG = 16 / R;  // threads of a row: CG x 16, eight coordinates each, every CG-th piece
    const int nfb = (wk.M + groups * R - 1) / (groups * R);
    const int u = blockIdx.x / nfb, row_lo = blockIdx.x % nfb * groups * R, row_hi = min(wk.M, row_lo + groups * R);
    const int tid = threadIdx.x, wv = uni(tid >> 6), lane = tid & 63, col = lane & 15, grp = lane >> 4;
    uint8_t* sm = kvc_dsm;
    float* zs = reinterpret_cast<float*>(sm + kFinZ);
    _Float16* xs = reinterpret_cast<_Float16*>(sm + kFinX);
    _Float16* ps = reinterpret_cast<_Float16*>(sm + kFinP);
    float* red = reinterpret_cast<float*>(sm + kFinRed);
    float* big = red + 2 * 4 * 16;
    float* of_cache = big + 16;
    float* of_drafts = of_cache + 16;
    uint32_t* count = reinterpret_cast<uint32_t*>(sm + kFinCount);  // tiles of all units and of those before u, by wavefront
    const int rv = uni(V.r[u]);
    const uint64_t live = n_tok == 64 ? ~0ull : (1ull << n_tok) - 1ull;
    // Everything that the block reads is requested as early as its address is known.
    uint64_t named = lane < n_tok ? mask[(int64_t)u * n_tok + lane] & live : 0ull;
    int tiles = 0;
    if (wk.n_blocks > 0) {
        tiles = uni(unit_tiles(seq_len, u, wk.max_seq));
        uint32_t all = 0, before = 0;
        for (int i = tid; i < wk.U; i += kFinThreads) {
            const uint32_t n = unit_work(unit_tiles(seq_len, i, wk.max_seq), wk.M);
            all += n;
            if (i < u) before += n;
        }
        all = wave_total(all);
        before = wave_total(before);
        if (lane == 0) { count[wv] = all; count[4 + wv] = before; }
    }
    // drafted tokens that some row of the unit names
    for (int o = 1; o < 64; o <<= 1) named |= __shfl_xor(named, o);
    constexpr int kXv = KVC_TREE_MAX_TOKENS * (kD / 8) / kFinThreads;
    uint4 xr[kXv];
#pragma unroll
    for (int j = 0; j < kXv; ++j) {
        const int e = tid + j * kFinThreads, t = e >> 4, c8 = e & 15;
        xr[j] = uint4{0u, 0u, 0u, 0u};
        if ((named >> t) & 1) xr[j] = *reinterpret_cast<const uint4*>(xv + (int64_t)u * xv_stride + (int64_t)t * kD + 8 * c8);
    }
    uint4 kr[4];  // the wavefront's sixteen drafted tokens
    {
        const int t = 16 * wv + col;
        const bool there = (named >> t) & 1;
        const uint16_t* kp = xk + (int64_t)u * xk_stride + (int64_t)t * kD + 8 * grp;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            kr[ks] = uint4{0u, 0u, 0u, 0u};
            if (there) kr[ks] = *reinterpret_cast<const uint4*>(kp + 32 * ks);
        }
    }
    constexpr int kBt = kBtItems / kFinThreads;
    uint4 bt[kBt][4];
    if (tiles)
#pragma unroll
        for (int j = 0; j < kBt; ++j) basis_t_load<KVC_SIDE_K>(bt[j], V.basis + V.basis_off[u], rv, basis_item(tid + j * kFinThreads));
    uint4 qr[4];  // a group's rows
    uint64_t mine;
    auto rows = [&](int row0) {
        const int row = min(row0 + min(col, R - 1), wk.M - 1);
        const uint16_t* qp = q + ((int64_t)u * wk.M + row) * kD + 8 * grp;
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) qr[ks] = *reinterpret_cast<const uint4*>(qp + 32 * ks);
        mine = mask[(int64_t)u * n_tok + row / G] & live;
    };
    rows(row_lo);
    __syncthreads();
    int row0 = row_lo;
    do {
        // the threads of row mr merge its pieces, whose slots follow one another: maxima, sums, eight coordinates each
        const int mr = tid / (16 * CG), mi = tid % (16 * CG), mc = mi & 15, cg = mi >> 4;
        const int mrow = min(row0 + mr, wk.M - 1);
        float Mp = -INFINITY, l = 0.f;
        float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (tiles) {
            const uint32_t before = (count[4] + count[5]) + (count[6] + count[7]) + start_cost(wk.M);
            const uint32_t per = run_tiles((count[0] + count[1]) + (count[2] + count[3]), wk.n_blocks);
            const uint32_t b0 = before / per;
            const int64_t slot0 = (int64_t)b0 + u;
            const int n_pieces = (int)((before + (uint32_t)tiles - 1u) / per - b0) + 1;
            const float2* mlr = ml + slot0 * wk.M + mrow;
            const bool have = 8 * mc < ((rv + 15) & ~15);
            const float* ar = acc + (slot0 * wk.M + mrow) * kD + (have ? 8 * mc : 0);
            const int64_t stride = (int64_t)wk.M * kD;
            auto raise = [&](float m) {  // to the maximum m: returns what weights are relative to
                const float top = fmaxf(Mp, m), ref = top == -INFINITY ? 0.f : top, w = __builtin_amdgcn_exp2f(Mp - ref);
                Mp = top;
                l *= w;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] *= w;
                return ref;
            };
            constexpr int kAt = 4;  // pieces requested at once, with their maxima: no pass for the maxima first
            for (int c0 = cg; c0 < n_pieces; c0 += kAt * CG) {
                float2 v[kAt];
                float4 a[kAt], b[kAt];
#pragma unroll
                for (int j = 0; j < kAt; ++j) {
                    const int c = c0 + j * CG < n_pieces ? c0 + j * CG : c0;
                    v[j] = mlr[(int64_t)c * wk.M];
                    a[j] = *reinterpret_cast<const float4*>(ar + c * stride);
                    b[j] = *reinterpret_cast<const float4*>(ar + c * stride + 4);
                }
#pragma unroll
                for (int j = 1; j < kAt; ++j)
                    if (c0 + j * CG >= n_pieces) v[j].x = -INFINITY;
                const float ref = raise(fmaxf(fmaxf(v[0].x, v[1].x), fmaxf(v[2].x, v[3].x)));
#pragma unroll
                for (int j = 0; j < kAt; ++j) {
                    const float w = __builtin_amdgcn_exp2f(v[j].x - ref);
                    l = fmaf(w, v[j].y, l);
                    z[0] = fmaf(w, a[j].x, z[0]); z[1] = fmaf(w, a[j].y, z[1]); z[2] = fmaf(w, a[j].z, z[2]); z[3] = fmaf(w, a[j].w, z[3]);
                    z[4] = fmaf(w, b[j].x, z[4]); z[5] = fmaf(w, b[j].y, z[5]); z[6] = fmaf(w, b[j].z, z[6]); z[7] = fmaf(w, b[j].w, z[7]);
                }
            }
            if constexpr (CG > 1) {  // the row's other threads
                float m = Mp;
#pragma unroll
                for (int o = 16; o < 16 * CG; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
                raise(m);
#pragma unroll
                for (int o = 16; o < 16 * CG; o <<= 1) {
                    l += __shfl_xor(l, o);
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] += __shfl_xor(z[e], o);
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) z[e] = have ? z[e] : 0.f;
        }
        if (row0 == row_lo) {
            if (tiles)
#pragma unroll
                for (int j = 0; j < kBt; ++j) basis_t_store(sm, bt[j], basis_item(tid + j * kFinThreads));
#pragma unroll
            for (int j = 0; j < kXv; ++j) {
                const int e = tid + j * kFinThreads;
                *reinterpret_cast<uint4*>(xs + (e >> 4) * kFinXPitch + 8 * (e & 15)) = xr[j];
            }
        }
        // scores of the drafted tokens (rows of the result) and the block's rows (columns)
        float s[4];
        {
            rc_f4 c = rc_f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) c = mfma_h(__builtin_bit_cast(rc_h8, kr[ks]), __builtin_bit_cast(rc_h8, qr[ks]), c);
#pragma unroll
            for (int v = 0; v < 4; ++v)
                s[v] = (mine >> (16 * wv + 4 * grp + v)) & 1 ? c[v] * (1.4426950408889634f * 0.08838834764831845f) : -INFINITY;
        }
        if (R == kFinRows && row0 + R < row_hi) rows(row0 + R);
        float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (grp == 0) red[wv * 16 + col] = top;
        __syncthreads();
        const float D = fmaxf(fmaxf(red[mr], red[16 + mr]), fmaxf(red[32 + mr], red[48 + mr]));
        if (mi == 0) big[mr] = D == -INFINITY ? 0.f : D;
        __syncthreads();
        {
            const float Mc = big[min(col, R - 1)];
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const _Float16 h = (_Float16)__builtin_amdgcn_exp2f(s[v] - Mc);
                ps[col * kFinPPitch + 16 * wv + 4 * grp + v] = h;
                sum += (float)h;
            }
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (grp == 0) red[64 + wv * 16 + col] = sum;
        }
        __syncthreads();
        {
            const float M = fmaxf(D, Mp), ref = M == -INFINITY ? 0.f : M;
            const float wc = __builtin_amdgcn_exp2f(Mp - ref), wd = __builtin_amdgcn_exp2f(D - ref);
            const float sum = fmaf(wc, l, wd * ((red[64 + mr] + red[80 + mr]) + (red[96 + mr] + red[112 + mr])));
            const float i = sum > 0.f ? 1.f / sum : 0.f, il = l > 0.f ? 1.f / l : 0.f;
            if (mi == 0) {
                of_cache[mr] = wc * l * i;
                of_drafts[mr] = wd * i;
            }
            if (cg == 0)
#pragma unroll
                for (int e = 0; e < 8; ++e) zs[mr * kFinZPitch + 8 * mc + e] = z[e] * il;
        }
        __syncthreads();
        const int zc = min(col, R - 1);
        const float by_cache = V.delta[u] * of_cache[zc], by_drafts = of_drafts[zc];
        rc_f4 o[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rb = 2 * wv + i;
            rc_f4 c = rc_f4{0.f, 0.f, 0.f, 0.f}, t = c;
            if (tiles) {
#pragma unroll
                for (int st = 0; st < 4; ++st) {
                    rc_h8 hi, lo;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float x = zs[zc * kFinZPitch + bt_coord<KVC_SIDE_K>(32 * st) + 16 * grp + (e >> 1) + 8 * (e & 1)];
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
            for (int v = 0; v < 4; ++v) o[i][v] = fmaf(c[v], by_cache, t[v] * by_drafts);
        }
        if (col < R && row0 + col < wk.M) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                *reinterpret_cast<sat_h4*>(out + ((int64_t)u * wk.M + row0 + col) * kD + 16 * (2 * wv + i) + 4 * grp) =
                    saturated_half(o[i][0], o[i][1], o[i][2], o[i][3]);
            }
        }
        row0 += R;
    } while (R == kFinRows && row0 < row_hi);  // (smaller groups come one to a block)
}

// ---------------------------------------------------------------- host side

struct TreeLayout {
    TreeWork wk;
    int cb, rw;
    int64_t acc, ml;
};

int64_t round_up(int64_t x) { return (x + 255) / 256 * 256; }

TreeLayout tree_layout(const kvc_stream_desc* k, const kvc_stream_desc* v, int G, int n_tok, int max_seq, bool rope) {
    TreeLayout t;
    const int U = k->n_units, tiles = tile_count(max_seq);
    t.wk.M = n_tok * G;
    // Rows of a wavefront and wavefronts side by side in rows, the rest of the eight sharing a tile's tokens. Sixteen rows until
    // eight wavefronts have them, then 32, since making a tile's operands costs the same for any number of rows: 256 rows x 16k
    // x 64 units 179 us, in two blocks of 128 each making them 209; 128 rows 117 us, as 32 rows a wavefront, half of them idle,
    // 139 (keys not rotated: 154 and 179, 101 and 111). As few wavefronts in rows as hold them: 52 rows 95 us in four (that only
    // attend), 102 in eight; keys not rotated 69 and 81, and 32 rows 56 in two and 66 in four.
    t.cb = t.wk.M <= 128 ? 1 : 2;
    t.rw = t.wk.M > 64 ? 8 : (t.wk.M > 32 || rope ? 4 : 2);
    t.wk.rows_pb = 16 * t.cb * t.rw;
    t.wk.nrb = (t.wk.M + t.wk.rows_pb - 1) / t.wk.rows_pb;
    t.wk.max_seq = max_seq;
    t.wk.k_cap_tiles = tile_count(k->capacity);
    t.wk.v_cap_tiles = tile_count(v->capacity);
    // One block for every CU (LDS or registers let no second one in), or two, as long as there are tiles for them.
    t.wk.U = U;
    t.wk.n_blocks = (int)std::min<int64_t>(std::max(1, device_cus() * (tree_pair(t.cb, t.rw, rope) ? 2 : 1) / t.wk.nrb), (int64_t)U * (tiles ? tiles + start_cost(t.wk.M) : 0));
    const int64_t rows = t.wk.n_blocks ? ((int64_t)t.wk.n_blocks + U) * t.wk.M : 0;
    t.acc = 0;
    t.ml = round_up(rows * kD * 4);
    return t;
}

// What either form of the call needs, and every call of fewer rows, units or tokens, so that a server may take one workspace for
// its largest: blocks times rows falls where a CU's second block or a whole row block no longer fits (past 64 rows, 256, 512, 768),
// this bound of it does not. Rows of one block's pieces: 2 M for a CU up to 64 rows, then at least 128 and at most 256; a call of
// few tiles has as many blocks as those, each unit's start counted as the most tiles that it may be.
int64_t tree_need(const kvc_stream_desc* k, int G, int n_tok, int max_seq) {
    const int64_t M = n_tok * G, U = k->n_units, tiles = tile_count(max_seq);
    const int64_t a_cu = M <= 64 ? 2 * M : std::min<int64_t>(std::max<int64_t>(M, 128), 256);
    const int64_t rows = tiles ? std::min(std::max(device_cus() * a_cu, M), U * (tiles + start_cost(0)) * M) + U * M : 0;
    return std::max<int64_t>(round_up(rows * kD * 4) + round_up(rows * 8), 256);
}

template <int CB, int RW, bool ROPE>
int launch_tree_as(dim3 grid, hipStream_t st, const DevSide& K, const DevSide& V, const uint16_t* q, const int32_t* seq_len, const TreeWork& wk,
                   const TreeRope& rope, float* acc, float2* ml) {
    const hipError_t e = hipFuncSetAttribute((const void*)tree_partial_kernel<CB, RW, ROPE>, hipFuncAttributeMaxDynamicSharedMemorySize, tree_smem(CB, RW, ROPE));
    if (e != hipSuccess) return set_error(KVC_EDEVICE, "hipFuncSetAttribute: %s", hipGetErrorString(e));
    hipLaunchKernelGGL((tree_partial_kernel<CB, RW, ROPE>), grid, dim3(tree_threads(CB, RW, ROPE)), tree_smem(CB, RW, ROPE), st, K, V, q, seq_len, wk, rope, acc, ml);
    return check_launch("kvc_tree_attn");
}

template <bool ROPE>
int launch_tree(const TreeLayout& t, dim3 grid, hipStream_t st, const DevSide& K, const DevSide& V, const uint16_t* q, const int32_t* seq_len,
                const TreeRope& rope, float* acc, float2* ml) {
    if (t.cb == 2) return launch_tree_as<2, 8, ROPE>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
    if (t.rw == 8) return launch_tree_as<1, 8, ROPE>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
    if constexpr (!ROPE)
        if (t.rw == 2) return launch_tree_as<1, 2, ROPE>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
    return launch_tree_as<1, 4, ROPE>(grid, st, K, V, q, seq_len, t.wk, rope, acc, ml);
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
    if (max_seq_len > INT32_MAX - kTile + 1) return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: max_seq_len past 2^31 - 64");
    const int64_t kct = tile_count(k->capacity), vct = tile_count(v->capacity);
    if ((int64_t)k->n_units * (tile_count(max_seq_len) + start_cost(0)) > INT32_MAX / 2)  // counted in 32 bits
        return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: more than 2^30 tiles of 64 tokens");
    for (int u = 0; u < k->n_units; ++u)  // byte offsets inside a stream are 32 bits
        if (kct * 8 * k->r_host[u] * k->b_host[u] > INT32_MAX || vct * 8 * v->r_host[u] * v->b_host[u] > INT32_MAX)
            return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: a unit's stream exceeds 2 GiB");
    return KVC_OK;
}

}  // namespace
}  // namespace kvc

using namespace kvc;

extern "C" size_t kvc_tree_attn_workspace(const kvc_stream_desc* k, const kvc_stream_desc* v, int32_t G, int32_t n_tok, int32_t max_seq_len) {
    clear_error();
    if (tree_check(k, v, G, n_tok, max_seq_len)) return 0;
    return (size_t)tree_need(k, G, n_tok, max_seq_len);
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
    const TreeLayout t = tree_layout(k, v, G, n_tok, max_seq_len, rope_base != 0.f);
    if (const int64_t need = tree_need(k, G, n_tok, max_seq_len); (int64_t)ws_bytes < need)
        return set_error(KVC_ENOSPACE, "kvc_tree_attn: workspace %zu < %lld bytes", ws_bytes, (long long)need);
    float* acc = reinterpret_cast<float*>(reinterpret_cast<char*>(ws) + t.acc);
    float2* ml = reinterpret_cast<float2*>(reinterpret_cast<char*>(ws) + t.ml);
    const hipStream_t st = (hipStream_t)stream;
    const DevSide K = dev_side(k), V = dev_side(v);
    const int64_t blocks = (int64_t)t.wk.nrb * t.wk.n_blocks;
    // Rows of a finishing block: four while sixteen would leave half the CUs without one. 8 units: 32 rows x 4k 23.5 us, with
    // sixteen 26.2; 64 rows x 128k 127 and 130. 64 units, 32 rows x 4k, where it takes sixteen: 42.5, with four 42.6.
    const int R = (int64_t)k->n_units * ((t.wk.M + 15) / 16) < device_cus() / 2 ? 4 : 16;
    // A block takes as many groups of R rows, one after another, as it takes to have no second turn of blocks (two fit a CU):
    // 256 rows x 4k x 64 units (keys not rotated) 74.2 -> 70.3 us.
    const int64_t all_groups = (int64_t)k->n_units * ((t.wk.M + R - 1) / R), turn = 2 * (int64_t)device_cus();
    const int groups = (int)std::min<int64_t>((t.wk.M + R - 1) / R, (all_groups + turn - 1) / turn);
    const int64_t fin = (int64_t)k->n_units * ((t.wk.M + groups * R - 1) / (groups * R));
    if (blocks > INT32_MAX || fin > INT32_MAX) return set_error(KVC_EUNSUPPORTED, "kvc_tree_attn: too many units");
    if (blocks) {
        TreeRope rope;
        for (int j = 0; j < kD / 2; ++j) rope.freq[j] = 0.0;
        if (rope_base != 0.f) rope_frequencies(rope_base, rope.freq);
        const dim3 grid((unsigned)blocks);
        const int e = rope_base != 0.f ? launch_tree<true>(t, grid, st, K, V, q, seq_len, rope, acc, ml)
                                       : launch_tree<false>(t, grid, st, K, V, q, seq_len, rope, acc, ml);
        if (e) return e;
    }
    const dim3 grid((unsigned)fin), blk(kFinThreads);
    if (R == 4)
        hipLaunchKernelGGL(tree_finish_kernel<4>, grid, blk, kFinSmem, st, V, q, G, n_tok, xk, xk_unit_stride, xv, xv_unit_stride, mask, seq_len,
                           t.wk, groups, acc, ml, out);
    else
        hipLaunchKernelGGL(tree_finish_kernel<16>, grid, blk, kFinSmem, st, V, q, G, n_tok, xk, xk_unit_stride, xv, xv_unit_stride, mask, seq_len,
                           t.wk, groups, acc, ml, out);
    return check_launch("kvc_tree_attn");
}
