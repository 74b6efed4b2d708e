// Layers in fixed point on shares, f = tau fraction bits: matrix products with bias, activation and residual, and a mixture
// of experts for a few tokens.
//   product:     the parties' parts z_p of v = X W (three-term products added up, Sec. II-B), 64-bit words
//   completion:  y = floor((v + (b << f) + 2^(f-1)) / 2^f), with ReLU times its sign bit, plus a residual (k_finish)
// The completion opens v once, masked with the edaBit r of the element: party p sends z_p + alpha_p + r_p to both others, which
// replaces the reshare and the opening of its result.  With c = v + 2^(f-1) + O + r, 0 <= v + 2^(f-1) + O < 2^63,
//   y = (c >> f) - (r >> f) + 2^(64-f) [c_63 = 0 and r_63 = 1] - [c mod 2^f < r mod 2^f] - (O >> f)
// where r >> f and r_63 are dealer material and the last bit comes from a tree of ANDs.  With ReLU O = 2^(f+31): v + 2^(f-1) >= 0 iff bit
// f+31 of c - r is set, and the borrow into that bit is the root of the tree whose lower half is the borrow of the rounding; so one
// opening and one tree (over bits 0 .. f+31, shifted up to end at bit 63; its lower half is bits 0 .. f-1) serve both.
#pragma once
#include <type_traits>
#include "gt_kernels.hpp"

#define GT_FIN_EL 16                              // elements of a wavefront's tile
#define GT_FIN_WORDS(NS) (22 * GT_FIN_EL + (NS) * 3 * 24)

// The wavefront model with 16 lanes per party (lanes 48-63 repeat party 2's and neither store nor count): two dealer blocks per element and nine blocks
// per stream (three groups of 8 elements that a tile can touch, three keys) make up one pass of the block function, 59 of 64 lanes with three streams.
struct FWire : WWire {
    __device__ __forceinline__ void init(uint4 *region, u64 *s_cnt)
    {
        const u32 l = threadIdx.x & (GT_LANES - 1);
        real = l < 3 * GT_FIN_EL; t = l & 15; p = l < 16 ? 0 : (l < 32 ? 1 : 2); pn = p == 2 ? 0 : p + 1;
        m = 16 * (u32)p + t;
        nx = 16 * (u32)pn + t; pv = 16 * (p == 0 ? 2u : (u32)p - 1) + t;
        buf = region; cnt = s_cnt; nopen = 0; nresh = 0;
        if (l < 6) cnt[l] = 0;
        wave_sync();
    }
    // a word to both others; the sum of the three
    __device__ __forceinline__ u64 open_both(u64 v, u32 bits)
    {
        nopen += bits; nresh += bits;
        wave_sync();
        *(uint2 *)&buf[m] = make_uint2((u32)v, (u32)(v >> 32));
        wave_sync();
        const uint2 a = *(const uint2 *)&buf[nx], b = *(const uint2 *)&buf[pv];
        return v + ((u64)a.x | ((u64)a.y << 32)) + ((u64)b.x | ((u64)b.y << 32));
    }
};

// Material of a tile: rows of GT_FIN_EL words.  0-2 r, 3-5 bits of r shifted up by 32 - f, 6-8 and 9 the daBit (arithmetic, both Boolean
// ones), 10-12 r >> f, 13-15 r_63 << (64 - f), 16-18 the second daBit, 19-21 products of adjacent bits of the shifted r, then rows of 24 words,
// [stream][key], of the streams 0 (opening), 1 (tree), 3 (product with ReLU's bit).  A tile may start anywhere.
template <int NS>
struct FinTile {
    const u32 *keys;
    u64 *mat;
    u32 f, w;                                     // w: the lane's word in the streams' rows
    __device__ __forceinline__ void deal(u32 op, u64 e0)
    {
        const u32 l = threadIdx.x & (GT_LANES - 1), el = l & 15, q = l - 32, i = q / 9, j = (q % 9) / 3, g = q % 3;
        const bool dealer = l < 32;
        w = ((u32)e0 & 7) + el;
        wave_sync();
        Key kv;
        const u32 *from = keys + 8 * (dealer ? GT_KEY_DEALER : (int)j);
#pragma unroll
        for (int v = 0; v < 8; v++) kv.k[v] = from[v];
        u64 D[8];
        chacha8<PRF_PAIR>(kv, dealer ? e0 + el : (e0 >> 3) + g, op, l < 16 ? 0u : (dealer ? 5u : i + (i >> 1)), D);
        const u64 r = (u64)__shfl((unsigned long long)D[0], (int)el, GT_LANES);          // of the element's first block
        const u64 bits = dealer ? (l < 16 ? D[5] : D[6]) : 0, beta = bits & 1;
        const u32 b0 = (u32)(bits >> 1) & 1, b1 = (u32)(bits >> 2) & 1, bb = b0 | (b1 << 1) | ((((u32)beta ^ b0 ^ b1) & 1) << 2);
        const u32 other = (u32)__shfl((int)bb, (int)el + 16, GT_LANES);
        u64 *to = mat + el;
        if (l < 16) {
            to[0] = D[1]; to[16] = D[2]; to[32] = r - D[1] - D[2];
            to[48] = D[3] << (32 - f); to[64] = D[4] << (32 - f); to[80] = (r ^ D[3] ^ D[4]) << (32 - f);
            to[96] = D[6]; to[112] = D[7]; to[128] = beta - D[6] - D[7];
            to[144] = bb | (other << 3);
        } else if (dealer) {
            to[160] = D[0]; to[176] = D[1]; to[192] = (r >> f) - D[0] - D[1];
            to[208] = D[2] << (64 - f); to[224] = D[3] << (64 - f); to[240] = ((r >> 63) - D[2] - D[3]) << (64 - f);
            to[256] = D[4]; to[272] = D[5]; to[288] = beta - D[4] - D[5];
            const u64 EVEN = 0x5555555555555555ull, win = r << (32 - f), p0 = D[7] & EVEN, p1 = (D[7] >> 1) & EVEN;
            to[304] = p0; to[320] = p1; to[336] = (win & (win >> 1) & EVEN) ^ p0 ^ p1;
        } else if (q < 9 * NS) {
#pragma unroll
            for (int v = 0; v < 8; v++) mat[22 * GT_FIN_EL + q * 8 + v] = D[v];
        }
        wave_sync();
    }
    __device__ __forceinline__ Sh pair(const WWire &W, int row) const { return Sh{ mat[(row + W.p) * GT_FIN_EL + W.t], mat[(row + W.pn) * GT_FIN_EL + W.t] }; }
    __device__ __forceinline__ u64 za(const WWire &W, int i) const { const u64 *m = mat + 22 * GT_FIN_EL + i * 72 + w; return m[W.p * 24] - m[W.pn * 24]; }
    __device__ __forceinline__ u64 zb(const WWire &W, int i) const { const u64 *m = mat + 22 * GT_FIN_EL + i * 72 + w; return m[W.p * 24] ^ m[W.pn * 24]; }
};

// [c < r] of a public and a bitwise shared word on the low 63 bits (HALVES = 2) or 32, prefix pairs (G, E) as in ge_bit_masks: borrow and equality
// of a block.  Pairs of two adjacent bits are local with the dealer's products of adjacent bits; they fill a dword for both halves: block b of a half
// has G at bit 2b (low half) ... so that one AND on 32 bits serves G and E of all blocks of a level: a nibble holds G, E of the low
// half's and G, E of the high half's block.  X' = (E_hi, E_hi) (G_lo, E_lo) xor (G_hi, 0).  low: the low half's borrow.
template <int HALVES>
__device__ __forceinline__ Sh less_tree(FWire &W, u64 c, Sh rho, Sh pr, u64 A, bool act, Sh &low)
{
    const u32 EV = 0x55555555u;
    const u32 m0 = W.p == 0 ? ~0u : 0u, m2 = W.p == 2 ? ~0u : 0u;
    u32 Xo[2], Xn[2];                              // G at even bits, E at odd ones, by half
#pragma unroll
    for (int h = 0; h < HALVES; h++) {
        const u32 nc = ~(u32)(c >> (32 * h)), live = h == 1 ? 0x7fffffffu : ~0u;       // bit 63 does not count: (G, E) = (0, 1)
        const u32 nl = nc & EV, nh = ((nc >> 1) | (h == 1 ? 0x40000000u : 0u)) & EV;
        const u32 both = nl & nh;
#pragma unroll
        for (int w = 0; w < 2; w++) {
            const u32 r = (u32)((w ? rho.n : rho.o) >> (32 * h)) & live, q = (u32)((w ? pr.n : pr.o) >> (32 * h)) & (h == 1 ? 0x15555555u : EV);
            const u32 rh = (r >> 1) & EV;
            const u32 u = nh & r, v = nl & rh;
            const u32 G = (nh & rh) ^ (nl & (q ^ u)), E = q ^ u ^ v ^ (both & (w ? m2 : m0));
            (w ? Xn[h] : Xo[h]) = G | (E << 1);
        }
    }
    // level 1, from one or two dwords of 16 blocks into one: low half's results at bits 0, 1 of a nibble, high half's at 2, 3
    u32 xo, xn, nresh = 0;
    {
        u32 l[2], e[2], g[2];
#pragma unroll
        for (int w = 0; w < 2; w++) {
            const u32 a = w ? Xn[0] : Xo[0], b = HALVES == 2 ? (w ? Xn[1] : Xo[1]) : 0;
            l[w] = (a & 0x33333333u) | (HALVES == 2 ? (b << 2) & 0xccccccccu : 0);
            const u32 ee = ((a >> 3) & 0x11111111u) | (HALVES == 2 ? (b >> 1) & 0x44444444u : 0);
            e[w] = ee | (ee << 1);
            g[w] = ((a >> 2) & 0x11111111u) | (HALVES == 2 ? b & 0x44444444u : 0);
        }
        const u32 M = HALVES == 2 ? (u32)A : (u32)A & 0x33333333u;
        u32 snd[1] = { and3l(e[0], e[1], l[0], l[1]) ^ M }, rcv[1];
        W.template reshare<1>(snd, rcv);
        xo = snd[0] ^ g[0]; xn = rcv[0] ^ g[1];
        nresh += HALVES == 2 ? 32 : 16;
    }
    const u32 B = (u32)(A >> 32);
#pragma unroll
    for (int v = 2; v <= 4; v++) {
        const int s = 2 << (v - 1);                // the neighbouring block's distance
        const u32 EM = (HALVES == 2 ? 5u : 1u) * (v == 2 ? 0x01010101u : v == 3 ? 0x00010001u : 1u);
        const u32 ho = xo >> s, hn = xn >> s;
        const u32 eo = (ho >> 1) & EM, en = (hn >> 1) & EM;
        const u32 M = (B >> (v == 2 ? 0 : v == 3 ? 4 : 12)) & (EM * 3);
        u32 snd[1] = { and3l(eo | (eo << 1), en | (en << 1), xo, xn) ^ M }, rcv[1];
        W.template reshare<1>(snd, rcv);
        xo = snd[0] ^ (ho & EM); xn = rcv[0] ^ (hn & EM);
        nresh += (HALVES == 2 ? 64 : 32) >> v;
    }
    low = Sh{ xo & 1, xn & 1 };
    Sh all = { 0, 0 };
    if (HALVES == 2) {
        u32 snd[1] = { (and3l(xo >> 3, xn >> 3, xo, xn) ^ (B >> 28)) & 1 }, rcv[1];
        W.template reshare<1>(snd, rcv);
        all.o = snd[0] ^ ((xo >> 2) & 1); all.n = rcv[0] ^ ((xn >> 2) & 1);
        nresh += 1;
    }
    W.nresh += act ? nresh : 0u;
    return all;
}

// Completion of a tile's elements: z the party's part of v, material dealt for the operation; returns y, with ReLU s y and the gate s.
template <bool RELU, class TileT>
__device__ __forceinline__ Sh finish_el(FWire &W, const TileT &T, u32 f, u64 z, bool act, Sh &gate)
{
    const int p = W.p;
    const u64 off = RELU ? 1ull << (f + 31) : 1ull << 62;
    const u64 c = W.open_both(z + T.za(W, 0) + T.pair(W, 0).o, act ? 64u : 0u) + ((1ull << (f - 1)) + off);
    const u32 bits = (u32)T.mat[9 * GT_FIN_EL + W.t];
    const Sh rho = T.pair(W, 3), d = T.pair(W, 6), one = pub(p, 1);
    Sh low;
    const Sh all = less_tree<RELU ? 2 : 1>(W, c << (32 - f), rho, T.pair(W, 19), T.zb(W, 1), act, low);
    // the bits to arithmetic: one message
    u32 fo[1] = { ((u32)low.o ^ (bits >> p)) & 1 }, fr[1];
    u32 fn = ((u32)low.n ^ (bits >> W.pn)) & 1;
    if (RELU) {
        const u32 ct = (u32)(c >> (f + 31)) & 1;
        const u32 so = (u32)(rho.o >> 63) ^ (u32)all.o ^ (p == 0 ? ct : 0), sn = (u32)(rho.n >> 63) ^ (u32)all.n ^ (p == 2 ? ct : 0);
        fo[0] |= ((so ^ (bits >> (3 + p))) & 1) << 1;
        fn |= ((sn ^ (bits >> (3 + W.pn))) & 1) << 1;
    }
    W.template pass<1>(fo, fr, W.pv);
    W.nopen += act ? (RELU ? 2u : 1u) : 0u;
    const u32 ff = fo[0] ^ fn ^ fr[0];
    const Sh b = ff & 1 ? one - d : d;
    Sh y = pub(p, (c >> f) - (off >> f)) - T.pair(W, 10) - b;
    if (!(c >> 63)) y = y + T.pair(W, 13);
    if (RELU) {
        const Sh d2 = T.pair(W, 16);
        gate = ff & 2 ? one - d2 : d2;
        y = mult_sh(W, gate, y, T.za(W, 2), act);
    }
    return y;
}

// ---------------------------------------------------------------------------------
// Residues.  Products of many rows run as products of small residues: words are taken as the numbers that their eight signed bytes stand for, -128 R to 127 R with
// R = (256^8 - 1) / 255, their products added up exactly (RNS_TERMS terms at a time, two products of words each: |S| <= 2 * RNS_TERMS * (128 R)^2), from 18 coprime
// moduli whose product M is 2^140.4, and only then reduced modulo 2^64.  A modulus costs one int8 product per term, so a ring product costs 18 of them where signed limbs cost 36.
//   r_i = (sum of the products of residues, the right factor's times (M / m_i)^-1) mod m_i, balanced
//   S = sum_i r_i M / m_i - q M,  q = round(sum_i r_i / m_i)
// q is exact: |S / M| < 0.3682 and the fixed-point sum below is off by at most 18 * 128 / 2^15 = 0.0704 < 0.5 - 0.3682.
#define RNS_N 18
struct RnsTable {
    int m[RNS_N];                                 // moduli
    float inv[RNS_N];
    u32 left[RNS_N][2], right[RNS_N][2];          // balanced 256^s mod m_i, the right factor's times (M / m_i)^-1, four s a word
    int c13[RNS_N];                               // 2^13 mod m_i, balanced
    u32 join[8][5];                               // signed byte s of (M / m_i) mod 2^64, four i a word; byte 2 of the last one: of M
    u32 quot[5];                                  // round(2^14 / m_i)
};
constexpr u32 rns_byte(int v, int at) { return ((u32)v & 0xffu) << (8 * at); }
constexpr int rns_balanced(u64 v, int m) { const int r = (int)(v % (u64)m); return 2 * r > m - 1 + (m & 1) ? r - m : r; }
constexpr RnsTable rns_make()
{
    const int m[RNS_N] = { 256, 255, 253, 251, 247, 241, 239, 233, 229, 227, 223, 217, 211, 199, 197, 193, 191, 181 };
    RnsTable t{};
    u64 all = 1;
    for (int i = 0; i < RNS_N; i++) all *= (u64)m[i];
    for (int i = 0; i < RNS_N; i++) {
        t.m[i] = m[i]; t.inv[i] = 1.0f / (float)m[i];
        u64 rest = 1, word = 1, inverse = 0;      // M / m_i modulo m_i and modulo 2^64
        for (int j = 0; j < RNS_N; j++) if (j != i) { rest = rest * (u64)m[j] % (u64)m[i]; word *= (u64)m[j]; }
        for (int v = 1; v < m[i]; v++) if (rest * (u64)v % (u64)m[i] == 1) inverse = (u64)v;
        u64 power = 1;
        for (int b = 0; b < 8; b++) {
            t.left[i][b / 4] |= rns_byte(rns_balanced(power, m[i]), b % 4);
            t.right[i][b / 4] |= rns_byte(rns_balanced(power * inverse, m[i]), b % 4);
            power = power * 256 % (u64)m[i];
        }
        t.c13[i] = rns_balanced(8192, m[i]);
        const u64 y = (word + GT_BIAS) ^ GT_BIAS;
        for (int b = 0; b < 8; b++) t.join[b][i / 4] |= rns_byte((int)(y >> (8 * b)), i % 4);
        t.quot[i / 4] |= rns_byte((16384 + m[i] / 2) / m[i], i % 4);
    }
    const u64 y = (all + GT_BIAS) ^ GT_BIAS;
    for (int b = 0; b < 8; b++) t.join[b][4] |= rns_byte((int)(y >> (8 * b)), 2);
    return t;
}
constexpr RnsTable RNS = rns_make();
static __device__ const RnsTable d_rns = rns_make();             // for a modulus that is not known when the kernel is compiled
#define RNS_MAGIC 0x4b400000u                     // 1.5 * 2^23: this plus an integer is the float 1.5 * 2^23 plus it

// An integer t, |t| < 2^21.1, given as RNS_MAGIC + t, to the balanced residue, in the low byte: t - round(t / m) m.  The low 24 bits of the
// float RNS_MAGIC + q are 2^22 + q; the low byte knows neither the 2^22 nor the difference of -m and neg = 256 - m.
__device__ __forceinline__ u32 rns_reduce(u32 tm, u32 neg, float inv)
{
    const float magic = __uint_as_float(RNS_MAGIC);
    const float q = __builtin_fmaf(__uint_as_float(tm) - magic, inv, magic);
    return (__float_as_uint(q) & 0xffffffu) * (neg & 0xffu) + tm;
}
__device__ __forceinline__ u32 low_bytes(u32 a, u32 b, u32 c, u32 d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0c0c0400u), __builtin_amdgcn_perm(b, a, 0x0c0c0400u), 0x05040100u);
}
// four bytes of four words to four words of a byte of each
__device__ __forceinline__ void transpose4x4(u32 (&x)[4])
{
    const u32 a = __builtin_amdgcn_perm(x[1], x[0], 0x06020400u), b = __builtin_amdgcn_perm(x[1], x[0], 0x07030501u);
    const u32 c = __builtin_amdgcn_perm(x[3], x[2], 0x06020400u), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030501u);
    x[0] = __builtin_amdgcn_perm(c, a, 0x05040100u); x[1] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    x[2] = __builtin_amdgcn_perm(c, a, 0x07060302u); x[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}
// The first of a chain of dot products.  It saturates, which no sum here comes near: the form that does takes any register as its third operand, the
// other one overwrites it and costs a move.
__device__ __forceinline__ int dot_first(u64 a, int b, int c) { return __builtin_amdgcn_sdot4((int)(u32)a, b, c, true); }
// the word that 18 residues (bytes of five words, four a word, the last two bytes zero) stand for
__device__ __forceinline__ u64 rns_join(const u32 (&r)[5])
{
    int qs = dot_first(r[0], (int)RNS.quot[0], 1 << 13);
#pragma unroll
    for (int g = 1; g < 5; g++) qs = __builtin_amdgcn_sdot4((int)r[g], (int)RNS.quot[g], qs, false);
    const u32 last = r[4] | (((u32)-(qs >> 14) & 0xffu) << 16);
    int D[8];
#pragma unroll
    for (int b = 0; b < 8; b++) {
        int d = dot_first(last, (int)RNS.join[b][4], 0);
#pragma unroll
        for (int g = 0; g < 4; g++) d = __builtin_amdgcn_sdot4((int)r[g], (int)RNS.join[b][g], d, false);
        D[b] = d;
    }
    return (u64)(long long)(D[0] + D[1] * 256) + ((u64)(long long)(D[2] + D[3] * 256) << 16) + ((u64)(u32)(D[4] + D[5] * 256) << 32) +
           ((u64)(u32)(D[6] + D[7] * 256) << 48);
}

// Completion.  Z: the parties' parts, [3][n] words, left at zero for the next product; bias: ncol words or none.
// k_finish_pair: of the elements from `first` on the parts, or R: residues, planes [chunk][party][modulus] of `plane` bytes, chunks added up; per: see there.
enum { FIN_PARTS = 0, FIN_SCALE = 1, FIN_RES = 2 };   // parts in memory; z = row factor S[e / ncol] times x (experts' gates); residues
struct FinArgs { KCommon c; u64 *Z; P6 bias, res, y, gate, S, x; u64 n; u32 ncol, f; int has_bias, has_res, has_gate; const unsigned char *R; u64 first, plane; u32 nchunk, per, nbig; };
// a party's parts of eight adjacent elements (of the launch's, from i0, a multiple of 8) from their residues
template <class Args>
__device__ __forceinline__ void rns_words(const Args &a, int p, u64 i0, u64 (&zw)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) zw[i] = 0;
    for (u32 ch = 0; ch < a.nchunk; ch++) {
        const unsigned char *R = a.R + (u64)(ch * 3 + p) * RNS_N * a.plane + i0;
        u32 r[2][20];
#pragma unroll
        for (int i = 0; i < RNS_N; i++) { const uint2 v = *(const uint2 *)(R + (u64)i * a.plane); r[0][i] = v.x; r[1][i] = v.y; }
#pragma unroll
        for (int h = 0; h < 2; h++) {
            r[h][18] = 0; r[h][19] = 0;
            u32 q[5][4];
#pragma unroll
            for (int g = 0; g < 5; g++) {
#pragma unroll
                for (int i = 0; i < 4; i++) q[g][i] = r[h][4 * g + i];
                transpose4x4(q[g]);
            }
#pragma unroll
            for (int i = 0; i < 4; i++) { const u32 w[5] = { q[0][i], q[1][i], q[2][i], q[3][i], q[4][i] }; zw[4 * h + i] += rns_join(w); }
        }
    }
}
// The words of some chunks' residues, n elements of a block of `cols` columns, added to the parts: [3][parts] words, rows of `ld`, the block's first column at c0.  For products whose
// residues are not kept until the completion.  Bound: what it reads and writes, 54 + 48 bytes an element a chunk (2^27 elements: 4.4 ms, 3.1 TB/s).
struct JoinArgs { const unsigned char *R; u64 *Z; u64 plane, n, parts, ld, c0, cols; u32 nchunk; };
__global__ __launch_bounds__(256) void k_join(JoinArgs a)
{
    const int p = (int)blockIdx.y;
    const u64 i0 = ((u64)blockIdx.x * 256 + threadIdx.x) * 8;
    if (i0 >= a.n) return;
    u64 zw[8];
    rns_words(a, p, i0, zw);
    u64 row = i0 / a.cols, col = i0 - row * a.cols;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (i0 + i >= a.n) return;
        a.Z[(u64)p * a.parts + row * a.ld + a.c0 + col] += zw[i];
        if (++col == a.cols) { col = 0; row++; }
    }
}
template <int SRC, bool RELU>
__global__ __launch_bounds__(64) void k_finish(FinArgs a)
{
    __shared__ uint4 s_msg[GT_LANES];
    __shared__ u64 s_mat[GT_FIN_WORDS(RELU ? 3 : 2)];
    __shared__ u64 s_cnt[6];
    FWire W; W.init(s_msg, s_cnt);
    FinTile<RELU ? 3 : 2> T; T.keys = a.c.keys; T.mat = s_mat; T.f = a.f;
    const int p = W.p;
    const u32 f = a.f;
    const bool narrow = a.n <= 0xffffffffu;
    const u64 tiles = (a.n + GT_FIN_EL - 1) / GT_FIN_EL;
    for (u64 tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const u64 e0 = tile * GT_FIN_EL, e = e0 + W.t;
        const bool act = e < a.n;
        const u64 row = !act ? 0 : (narrow ? (u64)((u32)e / a.ncol) : e / a.ncol), col = act ? e - row * a.ncol : 0;
        u64 z = 0;
        if (act) {
            if (SRC == FIN_PARTS) { z = a.Z[(u64)p * a.n + e]; if (W.real) a.Z[(u64)p * a.n + e] = 0; }
            else z = prod3(ld(a.S, p, row), ld(a.x, p, e));
            if (a.has_bias) z += own_of(a.bias, p)[col] << f;
        }
        T.deal(a.c.op, e0);
        Sh gate, y = finish_el<RELU>(W, T, f, z, act, gate);
        if (RELU && a.has_gate && act && W.real) st(a.gate, p, e, gate);
        if (act && W.real) {
            if (a.has_res) y = y + ld(a.res, p, e);
            st(a.y, p, e, y);
        }
        W.drain();
    }
    W.flush(a.c.wire);
}

// ---------------------------------------------------------------------------------
// The completion of residues, and of many parts: tiles of 40, two per lane of a party (lanes 0-19 of its 21), so that two passes of the block function (80 dealer
// blocks and 45 blocks of three streams on 2 x 63 lanes) and a chain of messages serve 40 elements where k_finish spends a pass and a chain on 16.
// Bound: the vector units, 1,590 instructions a tile with ReLU, half of them the block function's (2048 x 4096: 0.60 ms); three wavefronts per SIMD.
// Residues: the first nbig wavefronts take `per` tiles (at most 4), whose residues a party's 20 lanes join together, eight adjacent elements each, the others one.
#define GT_FP_EL 40
#define GT_FP_ROW 40                              // words of a row of material; rows as in FinTile, streams' rows from 22 on
template <int NS>
struct FinPair {
    const u32 *keys;
    u64 *mat;
    u32 f;
    __device__ __forceinline__ void deal(const WWire &W, u32 op, u64 e0)
    {
        const u32 m = W.m;
        const bool dealer = m < GT_FP_EL;
        u64 r = 0;
        u32 bits = 0;
        wave_sync();
#pragma unroll
        for (int pass = 0; pass < 2; pass++) {
            const u32 q = m - GT_FP_EL + 23 * pass, i = q / 15, j = (q % 15) / 5, g = q % 5;
            Key kv;
            const u32 *from = keys + 8 * (dealer ? GT_KEY_DEALER : (int)j);
#pragma unroll
            for (int v = 0; v < 8; v++) kv.k[v] = from[v];
            u64 D[8];
            chacha8<PRF_PAIR>(kv, dealer ? e0 + m : (e0 >> 3) + g, op, dealer ? 5u * (u32)pass : i + (i >> 1), D);
            if (dealer) {
                u64 *to = mat + m;
                const u64 w = pass == 0 ? D[5] : D[6], beta = w & 1;
                const u32 b0 = (u32)(w >> 1) & 1, b1 = (u32)(w >> 2) & 1, bb = b0 | (b1 << 1) | ((((u32)beta ^ b0 ^ b1) & 1) << 2);
                if (pass == 0) {
                    r = D[0];
                    bits = bb;
                    to[0] = D[1]; to[GT_FP_ROW] = D[2]; to[2 * GT_FP_ROW] = r - D[1] - D[2];
                    to[3 * GT_FP_ROW] = D[3] << (32 - f); to[4 * GT_FP_ROW] = D[4] << (32 - f); to[5 * GT_FP_ROW] = (r ^ D[3] ^ D[4]) << (32 - f);
                    to[6 * GT_FP_ROW] = D[6]; to[7 * GT_FP_ROW] = D[7]; to[8 * GT_FP_ROW] = beta - D[6] - D[7];
                } else {
                    to[9 * GT_FP_ROW] = bits | (bb << 3);
                    to[10 * GT_FP_ROW] = D[0]; to[11 * GT_FP_ROW] = D[1]; to[12 * GT_FP_ROW] = (r >> f) - D[0] - D[1];
                    to[13 * GT_FP_ROW] = D[2] << (64 - f); to[14 * GT_FP_ROW] = D[3] << (64 - f); to[15 * GT_FP_ROW] = ((r >> 63) - D[2] - D[3]) << (64 - f);
                    if (NS == 3) { to[16 * GT_FP_ROW] = D[4]; to[17 * GT_FP_ROW] = D[5]; to[18 * GT_FP_ROW] = beta - D[4] - D[5]; }
                    const u64 EVEN = 0x5555555555555555ull, win = r << (32 - f), p0 = D[7] & EVEN, p1 = (D[7] >> 1) & EVEN;
                    to[19 * GT_FP_ROW] = p0; to[20 * GT_FP_ROW] = p1; to[21 * GT_FP_ROW] = (win & (win >> 1) & EVEN) ^ p0 ^ p1;
                }
            } else if (q < 15 * NS) {
#pragma unroll
                for (int v = 0; v < 8; v++) mat[(22 + q / 5) * GT_FP_ROW + g * 8 + v] = D[v];
            }
        }
        wave_sync();
    }
    __device__ __forceinline__ Sh pair(const WWire &W, int row, u32 e) const { return Sh{ mat[(row + W.p) * GT_FP_ROW + e], mat[(row + W.pn) * GT_FP_ROW + e] }; }
    __device__ __forceinline__ u64 za(const WWire &W, int i, u32 e) const { const Sh w = pair(W, 22 + 3 * i, e); return w.o - w.n; }
    __device__ __forceinline__ u64 zb(const WWire &W, int i, u32 e) const { const Sh w = pair(W, 22 + 3 * i, e); return w.o ^ w.n; }
};
// less_tree of two elements, a message for both; on: bits 0, 1: which of them exist
template <int HALVES>
__device__ __forceinline__ void less_pair(WWire &W, const u64 (&c)[2], const Sh (&rho)[2], const Sh (&pr)[2], const u64 (&A)[2], u32 live2, u32 (&lo)[2], u32 (&ln)[2],
                                          u32 (&ao)[2], u32 (&an)[2])
{
    const u32 EV = 0x55555555u;
    const u32 m0 = W.p == 0 ? ~0u : 0u, m2 = W.p == 2 ? ~0u : 0u;
    u32 x[2], y[2], g0[2], g1[2], snd[2], rcv[2], nresh = HALVES == 2 ? 32 : 16;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        u32 Xo[2], Xn[2];
#pragma unroll
        for (int h = 0; h < HALVES; h++) {
            const u32 nc = ~(u32)(c[q] >> (32 * h)), live = h == 1 ? 0x7fffffffu : ~0u;
            const u32 nl = nc & EV, nh = ((nc >> 1) | (h == 1 ? 0x40000000u : 0u)) & EV;
            const u32 both = nl & nh;
#pragma unroll
            for (int w = 0; w < 2; w++) {
                const u32 r = (u32)((w ? rho[q].n : rho[q].o) >> (32 * h)) & live, d = (u32)((w ? pr[q].n : pr[q].o) >> (32 * h)) & (h == 1 ? 0x15555555u : EV);
                const u32 rh = (r >> 1) & EV;
                const u32 u = nh & r, v = nl & rh;
                const u32 G = (nh & rh) ^ (nl & (d ^ u)), E = d ^ u ^ v ^ (both & (w ? m2 : m0));
                (w ? Xn[h] : Xo[h]) = G | (E << 1);
            }
        }
        u32 l[2], e[2], g[2];
#pragma unroll
        for (int w = 0; w < 2; w++) {
            const u32 a = w ? Xn[0] : Xo[0], b = HALVES == 2 ? (w ? Xn[1] : Xo[1]) : 0;
            l[w] = (a & 0x33333333u) | (HALVES == 2 ? (b << 2) & 0xccccccccu : 0);
            const u32 ee = ((a >> 3) & 0x11111111u) | (HALVES == 2 ? (b >> 1) & 0x44444444u : 0);
            e[w] = ee | (ee << 1);
            g[w] = ((a >> 2) & 0x11111111u) | (HALVES == 2 ? b & 0x44444444u : 0);
        }
        snd[q] = and3l(e[0], e[1], l[0], l[1]) ^ (HALVES == 2 ? (u32)A[q] : (u32)A[q] & 0x33333333u);
        g0[q] = g[0]; g1[q] = g[1];
    }
    W.reshare<2>(snd, rcv);
#pragma unroll
    for (int q = 0; q < 2; q++) { x[q] = snd[q] ^ g0[q]; y[q] = rcv[q] ^ g1[q]; }
#pragma unroll
    for (int v = 2; v <= 4; v++) {
        const int s = 2 << (v - 1);
        const u32 EM = (HALVES == 2 ? 5u : 1u) * (v == 2 ? 0x01010101u : v == 3 ? 0x00010001u : 1u);
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const u32 ho = x[q] >> s, hn = y[q] >> s, eo = (ho >> 1) & EM, en = (hn >> 1) & EM;
            const u32 M = ((u32)(A[q] >> 32) >> (v == 2 ? 0 : v == 3 ? 4 : 12)) & (EM * 3);
            snd[q] = and3l(eo | (eo << 1), en | (en << 1), x[q], y[q]) ^ M;
            g0[q] = ho & EM; g1[q] = hn & EM;
        }
        W.reshare<2>(snd, rcv);
#pragma unroll
        for (int q = 0; q < 2; q++) { x[q] = snd[q] ^ g0[q]; y[q] = rcv[q] ^ g1[q]; }
        nresh += (HALVES == 2 ? 64 : 32) >> v;
    }
#pragma unroll
    for (int q = 0; q < 2; q++) { lo[q] = x[q] & 1; ln[q] = y[q] & 1; ao[q] = 0; an[q] = 0; }
    if (HALVES == 2) {
#pragma unroll
        for (int q = 0; q < 2; q++) snd[q] = (and3l(x[q] >> 3, y[q] >> 3, x[q], y[q]) ^ ((u32)(A[q] >> 32) >> 28)) & 1;
        W.reshare<2>(snd, rcv);
#pragma unroll
        for (int q = 0; q < 2; q++) { ao[q] = snd[q] ^ ((x[q] >> 2) & 1); an[q] = rcv[q] ^ ((y[q] >> 2) & 1); }
        nresh += 1;
    }
    W.nresh += nresh * live2;
}

// One or two completions in a launch: workgroups below na are the first one's.
struct FinSet { FinArgs f[2]; u32 na; };
template <int SRC, bool RELU>
__global__ __launch_bounds__(64) void k_finish_pair(FinSet set)
{
    const bool second = blockIdx.x >= set.na;
    const FinArgs &a = set.f[second ? 1 : 0];
    const u32 block = second ? blockIdx.x - set.na : blockIdx.x;
    constexpr int NS = RELU ? 3 : 2;
    __shared__ uint4 s_msg[GT_LANES];
    __shared__ u64 s_mat[(22 + 3 * NS) * GT_FP_ROW];
    __shared__ u64 s_cnt[6];
    WWire W; W.init(s_msg, s_cnt);
    FinPair<NS> T; T.keys = a.c.keys; T.mat = s_mat; T.f = a.f;
    const int p = W.p;
    const u32 f = a.f, t = W.t < 20 ? W.t : 19;
    const bool mine = W.real && W.t < 20, narrow = a.first + a.n <= 0xffffffffu;
    const u64 off = RELU ? 1ull << (f + 31) : 1ull << 62;
    const Sh one = pub(p, 1);
    // the party's planes, chosen once
    u64 *const yo = own_of(a.y, p), *const yn = nxt_of(a.y, p), *const go = own_of(a.gate, p), *const gn = nxt_of(a.gate, p);
    const u64 *const ro = own_of(a.res, p), *const rn = nxt_of(a.res, p), *const bo = own_of(a.bias, p);
    const u32 per = SRC == FIN_RES && block < a.nbig ? a.per : 1, chunk = per * GT_FP_EL, t8 = t < 5 * per ? t : 5 * per - 1;
    {
        const u64 c0 = (block < a.nbig ? (u64)block * a.per : (u64)a.nbig * (a.per - 1) + block) * GT_FP_EL;
        u64 zw[8];
        if (SRC == FIN_RES) rns_words(a, p, c0 + 8 * t8, zw);
        for (u32 k0 = 0; k0 < chunk && c0 + k0 < a.n; k0 += GT_FP_EL) {
            const u64 e0 = a.first + c0 + k0;
            const u32 el[2] = { t, t + 20 };
            bool act[2];
            u64 z[2], e[2];
            Sh res[2];
#pragma unroll
            for (int q = 0; q < 2; q++) {
                act[q] = W.t < 20 && c0 + k0 + el[q] < a.n;
                e[q] = a.first + (c0 + k0 + el[q] < a.n ? c0 + k0 + el[q] : a.n - 1);         // (a last tile loads its last element where none exists)
            }
            if (SRC == FIN_PARTS) {
                u64 *from = a.Z + (u64)p * a.n;
#pragma unroll
                for (int q = 0; q < 2; q++) z[q] = from[e[q] - a.first];
#pragma unroll
                for (int q = 0; q < 2; q++) if (mine && act[q]) from[e[q] - a.first] = 0;
            } else
            // the tile's words from the five lanes that joined them, through the message region
            {
                u64 *words = (u64 *)s_msg + GT_FP_EL * p;
                const u32 from = 8 * t8 - k0;                        // (wraps for the lanes of tiles before)
                wave_sync();
                if (from < GT_FP_EL)
#pragma unroll
                    for (int i = 0; i < 8; i++) words[from + i] = zw[i];
                wave_sync();
                z[0] = words[t]; z[1] = words[t + 20];
            }
            const u32 na = (u32)act[0] + (u32)act[1];
            if (a.has_bias)
#pragma unroll
                for (int q = 0; q < 2; q++) z[q] += bo[narrow ? (u64)((u32)e[q] % a.ncol) : e[q] % a.ncol] << f;
            if (a.has_res)
#pragma unroll
                for (int q = 0; q < 2; q++) res[q] = Sh{ ro[e[q]], rn[e[q]] };
            T.deal(W, a.c.op, e0);
            u64 m[2], c[2];
            {
#pragma unroll
                for (int q = 0; q < 2; q++) m[q] = z[q] + T.za(W, 0, el[q]) + T.mat[p * GT_FP_ROW + el[q]];
                wave_sync();
                s_msg[W.m] = make_uint4((u32)m[0], (u32)(m[0] >> 32), (u32)m[1], (u32)(m[1] >> 32));
                wave_sync();
                const uint4 x = s_msg[W.nx], y = s_msg[W.pv];
                c[0] = m[0] + ((u64)x.x | ((u64)x.y << 32)) + ((u64)y.x | ((u64)y.y << 32)) + ((1ull << (f - 1)) + off);
                c[1] = m[1] + ((u64)x.z | ((u64)x.w << 32)) + ((u64)y.z | ((u64)y.w << 32)) + ((1ull << (f - 1)) + off);
                W.nopen += 64u * na; W.nresh += 64u * na;
            }
            const Sh rho[2] = { T.pair(W, 3, el[0]), T.pair(W, 3, el[1]) }, pr[2] = { T.pair(W, 19, el[0]), T.pair(W, 19, el[1]) };
            const u64 A[2] = { T.zb(W, 1, el[0]), T.zb(W, 1, el[1]) }, cw[2] = { c[0] << (32 - f), c[1] << (32 - f) };
            u32 lo[2], ln[2], ao[2], an[2];
            less_pair<RELU ? 2 : 1>(W, cw, rho, pr, A, na, lo, ln, ao, an);
            u32 fo[1] = { 0 }, fr[1], fn = 0;
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const u32 bits = (u32)T.mat[9 * GT_FP_ROW + el[q]];
                u32 o = (lo[q] ^ (bits >> p)) & 1, n = (ln[q] ^ (bits >> W.pn)) & 1;
                if (RELU) {
                    const u32 ct = (u32)(c[q] >> (f + 31)) & 1;
                    const u32 so = (u32)(rho[q].o >> 63) ^ ao[q] ^ (p == 0 ? ct : 0), sn = (u32)(rho[q].n >> 63) ^ an[q] ^ (p == 2 ? ct : 0);
                    o |= ((so ^ (bits >> (3 + p))) & 1) << 1;
                    n |= ((sn ^ (bits >> (3 + W.pn))) & 1) << 1;
                }
                fo[0] |= o << (2 * q); fn |= n << (2 * q);
            }
            W.pass<1>(fo, fr, W.pv);
            W.nopen += (RELU ? 2u : 1u) * na;
            const u32 ff = fo[0] ^ fn ^ fr[0];
            Sh y[2], gate[2];
#pragma unroll
            for (int q = 0; q < 2; q++) {
                const Sh d = T.pair(W, 6, el[q]), b = (ff >> (2 * q)) & 1 ? one - d : d;
                y[q] = pub(p, (c[q] >> f) - (off >> f)) - T.pair(W, 10, el[q]) - b;
                const Sh top = T.pair(W, 13, el[q]);
                const u64 wrap = 0 - (u64)!(c[q] >> 63);
                y[q].o += top.o & wrap; y[q].n += top.n & wrap;
                if (RELU) {
                    const Sh d2 = T.pair(W, 16, el[q]);
                    gate[q] = (ff >> (2 * q)) & 2 ? one - d2 : d2;
                    m[q] = prod3(gate[q], y[q]) + T.za(W, 2, el[q]);
                }
            }
            if (RELU) {
                u64 rcv[2];
                W.reshare64<2>(m, rcv);
                W.nresh += 64u * na;
#pragma unroll
                for (int q = 0; q < 2; q++) y[q] = Sh{ m[q], rcv[q] };
            }
            if (a.has_res)
#pragma unroll
                for (int q = 0; q < 2; q++) y[q] = y[q] + res[q];
            if (mine && act[0]) {
                yo[e[0]] = y[0].o; yn[e[0]] = y[0].n;
                if (RELU && a.has_gate) { go[e[0]] = gate[0].o; gn[e[0]] = gate[0].n; }
            }
            if (mine && act[1]) {
                yo[e[1]] = y[1].o; yn[e[1]] = y[1].n;
                if (RELU && a.has_gate) { go[e[1]] = gate[1].o; gn[e[1]] = gate[1].n; }
            }
            W.drain();
        }
    }
    W.flush(a.c.wire);
}

// ---------------------------------------------------------------------------------
// A matrix of shared words by component. MAT_ROWS: element (row, k) at c[j][row * ld + k], MAT_COLS: at c[j][row + k * ld]; or weights in tiles, MAT_W: rows are
// theirs, MAT_WT: rows are their columns.
// Weights lie in tiles of 64 rows x 16 columns in the order in which a wavefront of k_mm_few takes them, [block of 16 columns][64 rows]
// [component][8][64 lanes][2 words]: lane n % 16 + 16 (k % 64 / 16) has the 16 words of its column in pairs, so that a step of a wavefront is 24 KB on end (with
// rows of words, 128 bytes at a time, 2.8-3.4 TB/s).  A word is kept as its eight signed bytes d_s, sum of d_s 256^s.
#define GT_WTILE 1024
enum { MAT_ROWS = 0, MAT_COLS = 1, MAT_W = 2, MAT_WT = 3 };
struct MatView { const u64 *c[3]; u64 ld; u32 kind, nst; };
__device__ __forceinline__ u64 wtile_at(u64 k, u64 n, u32 nst)
{
    return ((n >> 4) * nst + (k >> 6)) * (3 * GT_WTILE) + ((k & 15) >> 1) * 128 + ((n & 15) + (k & 48)) * 2 + (k & 1);
}

// Parts of the product of a few rows with a weight matrix, on the matrix cores in signed 8-bit limbs (36 products of
// limbs per ring product, as in k_count).  A wavefront owns 16 columns, a workgroup 64 and `per` steps of 64 terms of the long axis;
// the splits' parts meet by atomic adds of 64-bit words (exact, order-free).  z_p = (x_p + x_{p+1}) w_p + x_p w_{p+1}: the sum is made of
// the few rows' words, so each component of the weights is read once and meets both factors.  Up to 8 rows both factors share a 16-row tile:
//   rows 0-7: x_j + x_{j+1} -> z_j     rows 8-15: x_{j-1} -> z_{j-1}      (times w_j)
// so that a term costs 36 instructions a component and not 72.  The weights stay words in memory, 24 bytes each (tiles, see MatView), and are
// turned into limbs in registers (byte permutes; a quarter of the time in which they arrive): one copy serves both passes, KC: k contiguous (the
// transposed product of the backward pass).
// Bound: the rate at which the weights arrive (1 x 1024 x 4096, 101 MB: 20 us, 5 TB/s; 8 x 32784 x 512, 403 MB: 86 us, 4.7 TB/s; 16 x 8208 x 2048, 403 MB: 103 us,
// 3.9 TB/s with the left factor's limbs made ahead, 117 with its conversion in three of the four wavefronts).
struct FewArgs { const u64 *x[3]; const u64 *w; unsigned char *left; u64 *Z; u64 ldx, M, N, K; u32 nst, per, nsplit, blocks; DivArgs div; };
#define GT_FEW_PAD 66                             // words between the rows of the staging area
// division of a tile of elements by a workgroup of four wavefronts, as k_div<4>, in LDS that the caller has
#define GT_DIV_BYTES (4 * GT_LANES * 16 + GT_DIV_STEPS * GT_EL_WORDS(3) * 8 + 4 * 6 * 8)
__device__ __forceinline__ void div_block(const DivArgs &a, u64 tile, unsigned char *lds)
{
    uint4 (*s_msg)[GT_LANES] = (uint4 (*)[GT_LANES])lds;
    u64 *s_mat = (u64 *)(lds + 4 * GT_LANES * 16);
    u64 (*s_cnt)[6] = (u64 (*)[6])(lds + 4 * GT_LANES * 16 + GT_DIV_STEPS * GT_EL_WORDS(3) * 8);
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x / GT_LANES);
    DWire W; W.init(s_msg[wave], s_cnt[wave]);
    ElTile<3> T; T.init(a.c.keys, W, s_mat);
    const u64 e0 = tile * GT_EL, e = e0 + W.t;
    const bool act = W.t < GT_EL && e < a.n;
    Sh r = { 0, 0 }, Q = { 0, 0 }, quo = { 0, 0 };
    if (act) { Q = ld(a.Q, W.p, e); r = ld(a.S, W.p, e); }
    div_steps_el<4>(W, T, s_mat, W.p, a.c.op, e0, el_live(e0, a.n), a.nsteps, Q, r, quo, act);
    if (act && W.real && wave == 0) st(a.quo, W.p, e, quo);
    W.flush(a.c.wire);
}
// a word at a wave-uniform address plus a lane's offset in bytes
template <class T> __device__ __forceinline__ T ld_at(const void *base, u32 off) { return *(const T *)((const char *)base + off); }
// The left factor's limbs, as k_mm_few wants them in LDS: [tile of 16 rows][step][x_j + x_{j+1}, x_j by component][limb][lane of the operand][16 bytes].
// A launch of its own where so many workgroups take the same rows that converting them in each costs more (16 rows, 8208 x 2048: 116 -> 102 us).
#define GT_FEW_LEFT (6 * 8 * 1024)
__global__ __launch_bounds__(192) void k_few_left(FewArgs a)
{
    __shared__ __align__(16) u64 s_stage[3][2 * 8 * GT_FEW_PAD];
    const u32 lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), xr = lane >> 3, xg = lane & 7;
    const u64 r0 = (u64)blockIdx.y * 16, k = (u64)blockIdx.x * 64 + lane, at = k < a.K ? k : a.K - 1;
    const u64 *xa = wave == 0 ? a.x[0] : wave == 1 ? a.x[1] : a.x[2], *xb = wave == 0 ? a.x[1] : wave == 1 ? a.x[2] : a.x[0];
    u64 *stage = s_stage[wave], va[16], vb[16];
    // (rows and terms that exist where these do not, as in k_mm_few)
#pragma unroll
    for (int r = 0; r < 16; r++) {
        const u64 row = (r0 + r < a.M ? r0 + r : r0) * a.ldx + at;
        va[r] = xa[row]; vb[r] = xb[row];
    }
    unsigned char *out = a.left + ((u64)blockIdx.y * gridDim.x + blockIdx.x) * GT_FEW_LEFT + 256 * (xg >> 1) + 8 * (xg & 1) + xr * 16;
#pragma unroll
    for (int q = 0; q < 2; q++) {
        wave_sync();
#pragma unroll
        for (int r = 0; r < 8; r++) {
            const u64 x = va[r + 8 * q], y = x + vb[r + 8 * q];
            stage[r * GT_FEW_PAD + lane] = (y + GT_BIAS) ^ GT_BIAS;
            stage[(8 + r) * GT_FEW_PAD + lane] = (x + GT_BIAS) ^ GT_BIAS;
        }
        wave_sync();
        u64 ys[8], yp[8];
        ld8_whole(stage + xr * GT_FEW_PAD + xg * 8, ys);
        ld8_whole(stage + (8 + xr) * GT_FEW_PAD + xg * 8, yp);
        transpose8x8(ys); transpose8x8(yp);
#pragma unroll
        for (int sl = 0; sl < 8; sl++) {
            *(u64 *)(out + wave * 8192 + q * 128 + sl * 1024) = ys[sl];
            *(u64 *)(out + (3 + wave) * 8192 + q * 128 + sl * 1024) = yp[sl];
        }
    }
}
// DIV: workgroups from `blocks` on divide (the gates of a mixture, which nothing waits for before the first product is done). LEFT: the left factor's limbs are there.
template <int ROWS, bool KC, bool DIV, bool LEFT>
__global__ __launch_bounds__(256, 1) void k_mm_few(FewArgs a)
{
    constexpr int SLOTS = ROWS == 8 ? 3 : 6, XP = ROWS / 8;           // tiles of the left factor: both factors in one, or three of each
    constexpr int ABYTES = SLOTS * 8 * 1024;                          // [tile][limb][lane of the operand][16 bytes], twice
    constexpr int BYTES = 2 * ABYTES + (LEFT ? 0 : 3 * 2 * 8 * GT_FEW_PAD * 8);
    __shared__ __align__(16) unsigned char s_lds[DIV && GT_DIV_BYTES > BYTES ? GT_DIV_BYTES : BYTES];
    unsigned char (*s_a)[ABYTES] = (unsigned char (*)[ABYTES])s_lds;
    if (DIV && blockIdx.x >= a.blocks) { if (blockIdx.y == 0) div_block(a.div, blockIdx.x - a.blocks, s_lds); return; }
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const u32 lr = lane & 15, kq = lane >> 4;
    const u32 split = blockIdx.x % a.nsplit;
    const u64 c0 = ((u64)(blockIdx.x / a.nsplit) * 4 + wave) * 16, r0 = (u64)blockIdx.y * ROWS;
    const u32 nsteps = (u32)((a.K + 63) / 64), s0 = split * a.per, s1 = s0 + a.per < nsteps ? s0 + a.per : nsteps;
    const bool cols = c0 < a.N;                                      // whole wavefront; it takes part in the barriers
    const u32 nrow = a.M - r0 < (u64)ROWS ? (u32)(a.M - r0) : ROWS, K = (u32)a.K, ldx = (u32)a.ldx;
    // The left factor: wavefront j < 3 makes x_j + x_{j+1} (tile j) and x_j (meets w_{j+1}).  A lane loads one term of every row (whole lines; with eight
    // terms of a row per lane the 64 lines of every load took longer than the weights), and takes eight of a row through LDS.
    const u64 *xa = (wave == 0 ? a.x[0] : wave == 1 ? a.x[1] : a.x[2]) + r0 * a.ldx, *xb = (wave == 0 ? a.x[1] : wave == 1 ? a.x[2] : a.x[0]) + r0 * a.ldx;
    u64 *stage = (u64 *)(s_lds + 2 * ABYTES) + (wave < 3 ? wave : 0) * (2 * 8 * GT_FEW_PAD);
    const bool converts = LEFT || wave < 3;
    u64 va[ROWS], vb[ROWS];
    v4i ready[ABYTES / 4096];
    auto fetch = [&](u32 s) {
        if (LEFT) {
            const unsigned char *from = a.left + ((u64)blockIdx.y * nsteps + s) * ABYTES;
#pragma unroll
            for (int q = 0; q < ABYTES / 4096; q++) ready[q] = ld_at<v4i>(from + q * 4096, tid * 16);
            return;
        }
        const u32 k = s * 64 + lane, at = (k < K ? k : K - 1) * 8;
#pragma unroll
        for (int r = 0; r < ROWS; r++) {                              // (words that exist where these do not: loads without branches)
            const u64 row = (u64)((u32)r < nrow ? r : 0) * ldx;
            va[r] = ld_at<u64>(xa + row, at); vb[r] = ld_at<u64>(xb + row, at);
        }
    };
    auto put = [&](u32 s, int buf) {
        if (LEFT) {
#pragma unroll
            for (int q = 0; q < ABYTES / 4096; q++) *(v4i *)(s_a[buf] + q * 4096 + tid * 16) = ready[q];
            return;
        }
        const u32 xr = lane >> 3, xg = lane & 7;
        // (rows that do not exist make sums that nobody stores; terms that do not exist meet weights that are zero)
#pragma unroll
        for (int q = 0; q < XP; q++) {
            wave_sync();
#pragma unroll
            for (int r = 0; r < 8; r++) {
                const u64 x = va[r + 8 * q], y = x + vb[r + 8 * q];
                stage[r * GT_FEW_PAD + lane] = (y + GT_BIAS) ^ GT_BIAS;
                stage[(8 + r) * GT_FEW_PAD + lane] = (x + GT_BIAS) ^ GT_BIAS;
            }
            wave_sync();
            u64 ys[8], yp[8];
            ld8_whole(stage + xr * GT_FEW_PAD + xg * 8, ys);
            ld8_whole(stage + (8 + xr) * GT_FEW_PAD + xg * 8, yp);
            transpose8x8(ys); transpose8x8(yp);
            const u32 r = xr + 8 * q;
            const u32 slot = ROWS == 8 ? (wave == 2 ? 0 : wave + 1) : 3 + wave, row = ROWS == 8 ? 8 + r : r;     // of the component
            unsigned char *to = s_a[buf] + 256 * (xg >> 1) + 8 * (xg & 1);
#pragma unroll
            for (int sl = 0; sl < 8; sl++) {
                *(u64 *)(to + wave * 8192 + r * 16 + sl * 1024) = ys[sl];
                *(u64 *)(to + slot * 8192 + row * 16 + sl * 1024) = yp[sl];
            }
        }
    };
    u64 raw[3][16];
    // transposed: column c0 + lr is row c0 + lr of the weights, the 16 terms from 16 kq on lie in one tile
    const u32 woff = KC ? (kq * a.nst * 3 * GT_WTILE + (lr >> 1) * 128 + (lr & 1)) * 8 : lane * 16;
    const u64 *w0 = a.w + (KC ? (c0 >> 6) * (3 * GT_WTILE) + (c0 & 48) * 2 : (c0 >> 4) * a.nst * (3 * GT_WTILE));
    auto load = [&](int j, u32 s) {
        const u64 *from = w0 + (u64)j * GT_WTILE + (KC ? (u64)s * 4 * a.nst : (u64)s) * (3 * GT_WTILE);
#pragma unroll
        for (int i = 0; i < 16; i += 2) {
            if (KC) { raw[j][i] = ld_at<u64>(from, woff + i * 16); raw[j][i + 1] = ld_at<u64>(from, woff + i * 16 + 16); }
            else { const ulonglong2 v = ld_at<ulonglong2>(from, woff + i * 512); raw[j][i] = v.x; raw[j][i + 1] = v.y; }
        }
    };
    v4i acc[3][8];
#pragma unroll
    for (int j = 0; j < 3; j++)
#pragma unroll
        for (int u = 0; u < 8; u++) acc[j][u] = v4i{ 0, 0, 0, 0 };
    v4i B[2][8];
    // limbs of a component's words: byte permutes, between the matrix instructions of the component before
    auto limbs = [&](int to, int j) {
        u64 y[8], z[8];
#pragma unroll
        for (int i = 0; i < 8; i++) { y[i] = raw[j][i]; z[i] = raw[j][8 + i]; }
        transpose8x8(y); transpose8x8(z);
#pragma unroll
        for (int i = 0; i < 8; i++) B[to][i] = v4i{ (int)(u32)y[i], (int)(u32)(y[i] >> 32), (int)(u32)z[i], (int)(u32)(z[i] >> 32) };
    };
    // par: parity of the step's first component (its limbs are in B[par])
    auto step = [&](auto PAR, u32 s, int buf, bool more) {
        // (the fences keep the loads of the next step where they are: the compiler moves them to the end of the step to save registers)
        constexpr int P0 = decltype(PAR)::value;
        if (more && converts) fetch(s + 1);
        __builtin_amdgcn_sched_barrier(0);
        if (cols) {
#pragma unroll
            for (int j = 0; j < 3; j++) {
                const int b = (P0 + j) & 1;
                if (more) load(j, s + 1);
                __builtin_amdgcn_sched_barrier(0);
                if (j < 2 || more) limbs(b ^ 1, (j + 1) % 3);
#pragma unroll
                for (int h = 0; h < (ROWS == 8 ? 1 : 2); h++) {
                    // the sums' tile with w_j gives z_j; x_{j-1} with w_j gives z_{j-1}
                    const int slot = h == 0 ? j : 3 + (j + 2) % 3, to = h == 0 ? j : (j + 2) % 3;
                    const unsigned char *A0 = s_a[buf] + slot * 8192 + lane * 16;
#pragma unroll
                    for (int sl = 0; sl < 8; sl++) {
                        const v4i A = *(const v4i *)(A0 + sl * 1024);
#pragma unroll
                        for (int t = 0; t < 8 - sl; t++) acc[to][sl + t] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, B[b][t], acc[to][sl + t], 0, 0, 0);
                    }
                }
                __builtin_amdgcn_sched_group_barrier(0x100, 3, 0);
#pragma unroll
                for (int q = 0; q < (ROWS == 8 ? 36 : 72); q++) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, ROWS == 8 ? 4 : 2, 0);
                    if (q % 4 == 0) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (more && converts) put(s + 1, buf ^ 1);
    };
    if (converts) fetch(s0);
    if (cols)
#pragma unroll
        for (int j = 0; j < 3; j++) load(j, s0);
    if (converts) put(s0, 0);
    __syncthreads();
    if (cols) limbs(0, 0);
    std::integral_constant<int, 0> even;
    std::integral_constant<int, 1> odd;
    u32 s = s0;
    for (; s + 2 < s1; s += 2) {
        step(even, s, 0, true);
        __syncthreads();
        step(odd, s + 1, 1, true);
        __syncthreads();
    }
    if (s + 1 < s1) {
        step(even, s, 0, true);
        __syncthreads();
        step(odd, s + 1, 1, false);
    } else step(even, s, 0, false);
    if (!cols) return;
#pragma unroll
    for (int v = 0; v < 4; v++) {
        u64 z[3];
#pragma unroll
        for (int j = 0; j < 3; j++) {
            z[j] = 0;
#pragma unroll
            for (int u = 0; u < 8; u++) z[j] += (u64)(long long)acc[j][u][v] << (8 * u);
        }
        if (ROWS == 8) {                                             // rows 8-15 of the next component's tile belong to this party
            u64 o[3];
#pragma unroll
            for (int j = 0; j < 3; j++) o[j] = (u64)__shfl_xor((unsigned long long)z[j], 32, GT_LANES);
#pragma unroll
            for (int j = 0; j < 3; j++) z[j] += o[(j + 1) % 3];
        }
        const u32 row = 4 * kq + v;
        const u64 c = c0 + lr;
        if (row < nrow && c < a.N)
#pragma unroll
            for (int j = 0; j < 3; j++) {
                u64 *to = &a.Z[((u64)j * a.M + r0 + row) * a.N + c];
                if (a.nsplit > 1) atomicAdd((unsigned long long *)to, (unsigned long long)z[j]); else *to = z[j];
            }
    }
}

// ---------------------------------------------------------------------------------
// Residues of a matrix of words (rows x K) as operands of v_mfma_i32_32x32x32_i8: [matrix][modulus][32 terms][32 rows][64 lanes][16 bytes],
// lane l of an operand holds row l % 32 and the 16 terms from 16 (l / 32) on.  Matrices: the sums of adjacent components (0-2) and the components
// (3-5), or the components alone (0-2).  Rows and terms beyond the matrix are zero.  A residue: two four-byte dot products of the word's
// signed bytes with the powers of 256, a rounded quotient in floating point.  RIGHT: times (M / m_i)^-1.
// A wavefront makes an operand of 32 x 32 words of one matrix for `per` moduli; a launch makes both factors' (blocks below na: the left one's).
// MAT_ROWS: the words go through LDS, so that loads are of whole rows.  Bound: what it writes, 18 bytes a word, and reads, for large matrices (both factors of
// 2048 x 1024 x 4096, 453 MB written and 151 MB read, 122 us, 5 TB/s), else the vector units' 110 instructions per operand and modulus (1000 x 294 x 257
// backward: 95 MB written, 32 us).
struct ResArgs { MatView x; unsigned char *out; u64 rows, K, k0; u32 nrb, nkb, per, mats; };
// an operand's words, a lane's 16 terms (MAT_ROWS: of rows 2 i + hi its term lr): component x0, or with x1 its sum with that one, as signed bytes
// (a sum's second words are loaded in a loop of their own: with a condition at each, every load is waited for)
template <int KIND>
__device__ __forceinline__ void residue_words(const ResArgs &a, const u64 *x0, const u64 *x1, bool sum, u32 rb, u32 kb, u32 lr, u32 hi, u64 (&x)[16])
{
    const u64 r0 = (u64)rb * 32, k0 = (u64)kb * 32, ld = a.x.ld;
    u64 t[16];
    auto both = [&](auto at) {
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = at(x0, i);
        if (sum) {
#pragma unroll
            for (int i = 0; i < 16; i++) t[i] = at(x1, i);
        } else {
#pragma unroll
            for (int i = 0; i < 16; i++) t[i] = 0;
        }
    };
    if (KIND == MAT_W || KIND == MAT_WT) {
        // zero where the padded matrix has none
        const bool in = r0 < (a.rows + 63) / 64 * 64 && k0 < (a.K + 63) / 64 * 64;
        const u64 n = KIND == MAT_W ? a.k0 + k0 + 16 * hi : r0 + lr, k = KIND == MAT_W ? r0 + lr : a.k0 + k0 + 16 * hi;
        const u64 first = in ? wtile_at(k, n, a.x.nst) : 0;
        // (MAT_W: the next column, MAT_WT: the next row)
        both([&](const u64 *c, int i) { return c[first + (KIND == MAT_W ? 2 * i : (i >> 1) * 128 + (i & 1))]; });
        if (sum)
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = ((((x[i] ^ GT_BIAS) - GT_BIAS) + ((t[i] ^ GT_BIAS) - GT_BIAS)) + GT_BIAS) ^ GT_BIAS;
        if (!in)
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = 0;
        return;
    }
    if (r0 + 32 <= a.rows && k0 + 32 <= a.K) {                        // a whole operand: uniform addresses and a lane's offset
        const u64 first = KIND == MAT_ROWS ? r0 * ld + a.k0 + k0 : r0 + (a.k0 + k0) * ld, step = KIND == MAT_ROWS ? 2 * ld : ld;
        const u32 off = (KIND == MAT_ROWS ? hi * (u32)ld + lr : hi * 16 * (u32)ld + lr) * 8;
        both([&](const u64 *c, int i) { return ld_at<u64>(c + first + i * step, off); });
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = (x[i] + t[i] + GT_BIAS) ^ GT_BIAS;
        return;
    }
    // (words that exist are loaded where these do not, and cleared)
    auto row = [&](int i) { return r0 + (KIND == MAT_ROWS ? 2 * i + hi : lr); };
    auto term = [&](int i) { return k0 + (KIND == MAT_ROWS ? lr : hi * 16 + i); };
    both([&](const u64 *c, int i) {
        const u64 r = row(i) < a.rows ? row(i) : a.rows - 1, k = a.k0 + (term(i) < a.K ? term(i) : a.K - 1);
        return c[KIND == MAT_ROWS ? r * ld + k : r + k * ld];
    });
#pragma unroll
    for (int i = 0; i < 16; i++) x[i] = ((x[i] + t[i] + GT_BIAS) ^ GT_BIAS) & (0 - (u64)(row(i) < a.rows && term(i) < a.K));
}
template <bool RIGHT, int KIND>
__device__ __forceinline__ void residue_block(const ResArgs &a, u32 block, u64 (*s_t)[32 * 33])
{
    constexpr bool KC = KIND == MAT_ROWS || KIND == MAT_W;
    const u32 lane = threadIdx.x & 63, lr = lane & 31, hi = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const u32 nfb = (u32)(((u64)a.nrb * a.nkb + 3) / 4), q = block / nfb % a.mats, range = block / nfb / a.mats;
    const u64 nfr = (u64)a.nrb * a.nkb, mat = nfr * 1024;
    const u32 fr = block % nfb * 4 + wave;
    if (fr >= nfr) return;
    // neighbours along the axis that is contiguous in memory
    const u32 rb = KC ? fr / a.nkb : fr % a.nrb, kb = KC ? fr % a.nkb : fr / a.nrb;
    const bool sum = a.mats == 6 && q < 3;
    const u64 *x0 = q % 3 == 0 ? a.x.c[0] : (q % 3 == 1 ? a.x.c[1] : a.x.c[2]), *x1 = q == 0 ? a.x.c[1] : (q == 1 ? a.x.c[2] : a.x.c[0]);
    u64 x[16];
    residue_words<KIND>(a, x0, x1, sum, rb, kb, lr, hi, x);
    if (KIND == MAT_ROWS) {
#pragma unroll
        for (int i = 0; i < 16; i++) s_t[wave][(2 * i + hi) * 33 + lr] = x[i];
        wave_sync();
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = s_t[wave][lr * 33 + hi * 16 + i];
    }
    unsigned char *out = a.out + (u64)q * RNS_N * mat + ((u64)kb * a.nrb + rb) * 1024 + lane * 16;
    const u32 i0 = range * a.per, i1 = i0 + a.per < RNS_N ? i0 + a.per : RNS_N;
    for (u32 i = i0; i < i1; i++) {
        const int cl = (int)(RIGHT ? d_rns.right[i][0] : d_rns.left[i][0]), ch = (int)(RIGHT ? d_rns.right[i][1] : d_rns.left[i][1]);
        const u32 neg = 256 - (u32)d_rns.m[i];
        const float inv = d_rns.inv[i];
        u32 b[16];
#pragma unroll
        for (int e = 0; e < 16; e++)
            b[e] = rns_reduce((u32)__builtin_amdgcn_sdot4((int)(u32)x[e], cl, dot_first(x[e] >> 32, ch, (int)RNS_MAGIC), false), neg, inv);
        uint4 v;
        v.x = low_bytes(b[0], b[1], b[2], b[3]); v.y = low_bytes(b[4], b[5], b[6], b[7]);
        v.z = low_bytes(b[8], b[9], b[10], b[11]); v.w = low_bytes(b[12], b[13], b[14], b[15]);
        *(uint4 *)(out + (u64)i * mat) = v;
    }
}

// the factors of one or two products: left, right, left, right; end: their workgroups, added up
struct ResSet { ResArgs r[4]; u32 end[4]; };
__global__ __launch_bounds__(256) void k_residues(ResSet set)
{
    __shared__ u64 s_t[4][32 * 33];
    const u32 b = blockIdx.x, i = (b >= set.end[0] ? 1u : 0u) + (b >= set.end[1] ? 1u : 0u) + (b >= set.end[2] ? 1u : 0u);
    const ResArgs &a = set.r[i];
    const u32 block = b - (i ? set.end[i - 1] : 0);
    if (!(i & 1)) { if (a.x.kind == MAT_ROWS) residue_block<false, MAT_ROWS>(a, block, s_t); else residue_block<false, MAT_COLS>(a, block, s_t); }
    else if (a.x.kind == MAT_COLS) residue_block<true, MAT_COLS>(a, block, s_t);
    else if (a.x.kind == MAT_W) residue_block<true, MAT_W>(a, block, s_t);
    else residue_block<true, MAT_WT>(a, block, s_t);
}

// The products of residues: for every party and modulus the sum of two products, party p's
//   (a_p + a_{p+1}) b_p + a_p b_{p+1}      or      a_p (b_p + b_{p+1}) + a_{p+1} b_p
// (sums in the left or the right factor), reduced to balanced residues, [party][modulus] planes of bytes, row-major M x N.
// A workgroup of 2 x 2 wavefronts owns 64 WM x 64 WN outputs, a wavefront 32 WM x 32 WN; a step of 64 terms of both operands goes through LDS,
// where an operand lies as it is loaded: no bank conflicts.  The right factor takes the role of rows, so
// that a lane holds four adjacent columns of a result.  Consecutive workgroups of an XCD take the tiles of one product.
// Bound: the matrix cores at the clock that the card's power leaves: 2048 x 1024 x 4096, 1.86e15 operations in 0.96 ms, 1.94 POP/s (a large int8 product
// of the vendor's library 2.4-2.5; these matrix instructions alone on random registers 3.3, with this LDS traffic and a barrier a step 2.5; zeros 4.5).
// With the words to LDS behind the matrix instructions and loads a step ahead 1.09 ms; 256 x 256 outputs by eight wavefronts 0.97.
struct RmmArgs { const unsigned char *A, *B; unsigned char *R; u64 amat, bmat, plane; u32 M, N, narb, nbrb, nstep, ntm, ntn, total; int asums; };   // amat, bmat: bytes of a modulus's matrix; narb: blocks of 32 rows
// One or two products in a launch: workgroups below na are the first one's.
struct RmmSet { RmmArgs m[2]; u32 na; };
template <int WM, int WN>
__global__ __launch_bounds__(256, WM == 4 ? 2 : WM == 2 ? 3 : 4) void k_rns_mm(RmmSet set)
{
    const bool second = blockIdx.x >= set.na;
    const RmmArgs &a = set.m[second ? 1 : 0];
    const u32 block = second ? blockIdx.x - set.na : blockIdx.x;
    constexpr int FA = 2 * WM, FB = 2 * WN, STEP = 2 * (FA + FB) * 1024;       // operands of 32 rows a workgroup, bytes of a step
    constexpr int LD = 64 * WN + 16, OUT = 64 * WM * LD;
    constexpr int LOADS = STEP / 4096;                                         // of 16 bytes a lane
    __shared__ __align__(16) unsigned char s_buf[2 * STEP > OUT ? 2 * STEP : OUT];
    const u32 tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave & 1, wn = wave >> 1;
    // blocks go to the XCDs in turn: XCD x takes the x-th eighth of the work
    const u32 per = (a.total + 7) / 8, id = (block & 7) * per + (block >> 3);
    if ((block >> 3) >= per || id >= a.total) return;
    const u32 tiles = a.ntm * a.ntn, batch = id / tiles, tile = id % tiles, p = batch / RNS_N, mi = batch % RNS_N;
    // groups of 8 row tiles, column tiles one after the other
    const u32 grp = tile / (8 * a.ntn), gm = a.ntm - grp * 8 < 8 ? a.ntm - grp * 8 : 8, in = tile - grp * 8 * a.ntn;
    const u32 tm = grp * 8 + in % gm, tn = in / gm, pn = p == 2 ? 0 : p + 1;
    const unsigned char *A0 = a.A + ((u64)p * RNS_N + mi) * a.amat, *A1 = a.A + ((u64)(a.asums ? 3 + p : pn) * RNS_N + mi) * a.amat;
    const unsigned char *B0 = a.B + ((u64)p * RNS_N + mi) * a.bmat, *B1 = a.B + ((u64)(a.asums ? pn : 3 + p) * RNS_N + mi) * a.bmat;
    const u32 half = a.nstep / 2;                                              // steps of a product
    // a wavefront's loads of a step: operands q * 4 + wave of [2 blocks of terms][FA] of the left factor, then of the right one
    const unsigned char *at[LOADS];
#pragma unroll
    for (int q = 0; q < LOADS; q++) {
        const u32 o = q * 4 + wave;
        const bool isA = o < 2 * FA;
        const u32 w = isA ? o : o - 2 * FA, kb = isA ? w / FA : w / FB, r = isA ? w % FA : w % FB;
        at[q] = isA ? A0 + ((u64)kb * a.narb + tm * FA + r) * 1024 : B0 + ((u64)kb * a.nbrb + tn * FB + r) * 1024;
    }
    const u64 nextA = (u64)a.narb * 2048, nextB = (u64)a.nbrb * 2048;          // to the next step, or to the second product
    const u64 jumpA = (u64)(A1 - A0) - (half - 1) * nextA, jumpB = (u64)(B1 - B0) - (half - 1) * nextB;
    v4i st[2][LOADS];
    auto fetch = [&](u32 s, int to) {
        const bool jump = s + 1 == half;
        const u64 da = jump ? jumpA : nextA, db = jump ? jumpB : nextB;
#pragma unroll
        for (int q = 0; q < LOADS; q++) {
            st[to][q] = *(const v4i *)(at[q] + lane * 16);
            at[q] += q * 4 + (int)wave < 2 * FA ? da : db;
        }
    };
    auto put = [&](int buf) {
#pragma unroll
        for (int q = 0; q < LOADS; q++) *(v4i *)(s_buf + buf * STEP + (q * 4 + wave) * 1024 + lane * 16) = st[buf][q];
    };
    v16i acc[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; i++)
#pragma unroll
        for (int j = 0; j < WN; j++)
#pragma unroll
            for (int v = 0; v < 16; v++) acc[i][j][v] = 0;
    // Step s, of parity par: its matrix instructions, between them the words of step s + 1 (loaded during step s - 2) go to LDS, whose half was last read
    // in step s - 1, and the loads of step s + 3 start.
    auto step = [&](u32 s, int par, auto NEXT, auto MORE) {
        const unsigned char *buf = s_buf + par * STEP + lane * 16;
        v4i x[2][WM], w[2][WN];
#pragma unroll
        for (int kb = 0; kb < 2; kb++) {
#pragma unroll
            for (int j = 0; j < WN; j++) w[kb][j] = *(const v4i *)(buf + (2 * FA + kb * FB + wn * WN + j) * 1024);
#pragma unroll
            for (int i = 0; i < WM; i++) x[kb][i] = *(const v4i *)(buf + (kb * FA + wm * WM + i) * 1024);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (decltype(NEXT)::value) put(par ^ 1);
        if (decltype(MORE)::value) fetch(s + 3, par ^ 1);
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
            for (int i = 0; i < WM; i++)
#pragma unroll
                for (int j = 0; j < WN; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[kb][j], x[kb][i], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int q = 0; q < 2 * WM * WN; q++) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (decltype(NEXT)::value && q < LOADS) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
            if (decltype(MORE)::value && q < LOADS) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        __syncthreads();
    };
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    fetch(0, 0);
    fetch(1, 1);
    put(0);
    u32 s = 0;                                                                 // (steps are even in number)
    if (a.nstep > 2) {
        fetch(2, 0);
        __syncthreads();
        for (; s + 4 < a.nstep; s += 2) { step(s, 0, yes, yes); step(s + 1, 1, yes, yes); }
        step(s, 0, yes, yes);
        step(s + 1, 1, yes, no);
        s += 2;
    } else __syncthreads();
    step(s, 0, yes, no);
    step(s + 1, 1, no, no);
    // |sum| <= 2^27: low 13 bits and the rest times 2^13 mod m, below 2^21.1, then the balanced residue; through LDS to rows
    const float inv = d_rns.inv[mi];
    const u32 neg = 256 - (u32)d_rns.m[mi];
    const int c13 = d_rns.c13[mi];
#pragma unroll
    for (int i = 0; i < WM; i++)
#pragma unroll
        for (int j = 0; j < WN; j++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                u32 b[4];
#pragma unroll
                for (int v = 0; v < 4; v++) {
                    const int z = acc[i][j][4 * g + v];
                    b[v] = rns_reduce((u32)((z >> 13) * c13) + (((u32)z & 8191u) | RNS_MAGIC), neg, inv);
                }
                *(u32 *)(s_buf + ((wm * WM + i) * 32 + (lane & 31)) * LD + (wn * WN + j) * 32 + 8 * g + 4 * (lane >> 5)) = low_bytes(b[0], b[1], b[2], b[3]);
            }
    __syncthreads();
    unsigned char *R = a.R + (u64)batch * a.plane;
    constexpr u32 SEG = 4 * WN;                                                // of 16 bytes a row
    for (u32 u = tid; u < 64 * WM * SEG; u += 256) {
        const u32 r = u / SEG, c = (u % SEG) * 16;
        const u32 row = tm * 64 * WM + r, col = tn * 64 * WN + c;
        if (row >= a.M || col >= a.N) continue;
        const uint4 v = *(const uint4 *)(s_buf + r * LD + c);
        unsigned char *to = R + (u64)row * a.N + col;
        if (col + 16 <= a.N) __builtin_memcpy(to, &v, 16);
        else {
#pragma unroll
            for (u32 i = 0; i < 15; i++)
                if (i < a.N - col) to[i] = (unsigned char)((i < 4 ? v.x : i < 8 ? v.y : i < 12 ? v.z : v.w) >> (8 * (i & 3)));
        }
    }
}

// Components (own planes) of a rows x cols matrix into the tiles of weights, rows from row0 on; padding stays at zero.  A thread takes a pair of rows, whose words
// are adjacent there, so that 16 columns are 256 bytes on end (1024 x 4096: 30 us; a word at a time 188).
struct PutArgs { P6 src; u64 *dst; u64 row0, rows, cols; u32 nst; };
__global__ __launch_bounds__(256) void k_put(PutArgs a)
{
    const u64 first = a.row0 / 2, n = ((a.row0 + a.rows + 1) / 2 - first) * a.cols;
    for (u64 e = (u64)blockIdx.x * blockDim.x + threadIdx.x; e < n; e += (u64)gridDim.x * blockDim.x) {
        const u64 pair = e / a.cols, c = e - pair * a.cols, k = 2 * (first + pair), to = wtile_at(k, c, a.nst);
        const bool low = k >= a.row0, high = k + 1 < a.row0 + a.rows;
        const u64 from = (k - a.row0) * a.cols + c;                   // (wraps where the pair's first row is the one before; not read then)
#pragma unroll
        for (int j = 0; j < 3; j++) {
            u64 *out = a.dst + (u64)j * GT_WTILE + to;
            const u64 x = low ? (a.src.o[j][from] + GT_BIAS) ^ GT_BIAS : 0, y = high ? (a.src.o[j][from + a.cols] + GT_BIAS) ^ GT_BIAS : 0;
            if (low && high) { ulonglong2 v; v.x = x; v.y = y; *(ulonglong2 *)out = v; }
            else if (low) out[0] = x;
            else out[1] = y;
        }
    }
}

// Column sums of a shared matrix (local): a workgroup per 16 columns and component, 64 rows at a time.  Bound: reading the matrix (2048 x 1024, 50 MB).
struct ColsumArgs { P6 x, out; u64 rows; u32 cols; };
__global__ __launch_bounds__(1024) void k_colsum(ColsumArgs a)
{
    __shared__ u64 s_sum[64][17];
    const u32 c = threadIdx.x & 15, g = threadIdx.x >> 4, pl = blockIdx.y;
    const u64 col = (u64)blockIdx.x * 16 + c;
    const u64 *x = pl == 0 ? a.x.o[0] : (pl == 1 ? a.x.o[1] : a.x.o[2]);
    u64 s = 0;
    if (col < a.cols) {
#pragma unroll 8
        for (u64 r = g; r < a.rows; r += 64) s += x[r * a.cols + col];
    }
    s_sum[g][c] = s;
    __syncthreads();
    if (g < 8) {
#pragma unroll
        for (u32 i = 1; i < 8; i++) s += s_sum[g + 8 * i][c];
        s_sum[g][c] = s;
    }
    __syncthreads();
    if (g == 0 && col < a.cols) {
#pragma unroll
        for (int i = 1; i < 8; i++) s += s_sum[i][c];
        // component pl: party pl's own, its predecessor's next one
        own_of(a.out, (int)pl)[col] = s; nxt_of(a.out, pl == 0 ? 2 : (int)pl - 1)[col] = s;
    }
}

// ---------------------------------------------------------------------------------
// Mixture of experts.  Operation ids from c.op on: scores, pairs, choice, chosen scores, tau + 1 of the division, inputs, hidden values, their scaling,
// weighted hidden values, result.
__device__ __forceinline__ void pair_of(u32 q, u32 E, u32 &a, u32 &b)
{
    a = 0;
    while (q >= E - 1 - a) { q -= E - 1 - a; a++; }
    b = a + 1 + q;
}
struct MoeArgs { KCommon c; u64 *Z; P6 s, bias, o, S, Q, g, x, xe, hg, he; u64 rows; u32 E, k, d, ff, f; int parts, has_bias; };
// The choice for a row, a workgroup: completion of the scores (parts: from the router's parts, which are left at zero, else they are there), all pairs
// [s_a >= s_b], a < b (a beats b: ties go to the lower index), ranks (how many others beat an expert: local sums of the bits), o_j[a] = [rank of a = j] and the
// same times 2^f behind the row's inputs, S_j = sum_a o_j[a] s_a, Q = 1 + sum_a s_a.  Bound: the chain of its rounds.
__global__ __launch_bounds__(256) void k_moe_choose(MoeArgs a)
{
    __shared__ uint4 s_msg[4][GT_LANES];
    __shared__ u64 s_mat[4][GT_FIN_WORDS(3)];
    __shared__ u64 s_cnt[4][6];
    __shared__ u64 s_s[6][GT_MAX_EXPERTS], s_rank[6][GT_MAX_EXPERTS], s_sum[3][GT_MAX_EXPERTS];      // 2 p: own, 2 p + 1: next
    const u32 tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), E = a.E, k = a.k;
    const u64 t = blockIdx.x;
    for (u32 i = tid; i < GT_MAX_EXPERTS; i += 256) {
#pragma unroll
        for (int q = 0; q < 6; q++) s_rank[q][i] = 0;
#pragma unroll
        for (int q = 0; q < 3; q++) s_sum[q][i] = 0;
    }
    {
        FWire W; W.init(s_msg[wave], s_cnt[wave]);
        FinTile<3> T; T.keys = a.c.keys; T.mat = s_mat[wave]; T.f = a.f;
        for (u32 i0 = wave * GT_FIN_EL; i0 < E; i0 += 4 * GT_FIN_EL) {
            const u32 i = i0 + W.t;
            const bool act = i < E;
            const u64 e = t * E + i;
            Sh y = { 0, 0 }, gate;
            if (a.parts) {
                u64 z = 0;
                if (act) {
                    u64 *from = &a.Z[(u64)W.p * a.rows * E + e];
                    z = *from;
                    if (a.has_bias) z += own_of(a.bias, W.p)[i] << a.f;
                    if (W.real) *from = 0;
                }
                T.deal(a.c.op, t * E + i0);
                y = finish_el<true>(W, T, a.f, z, act, gate);
            } else if (act) y = ld(a.s, W.p, e);
            if (act && W.real) { s_s[2 * W.p][i] = y.o; s_s[2 * W.p + 1][i] = y.n; }
        }
        W.flush(a.c.wire);
    }
    __syncthreads();
    DWire W; W.init(s_msg[wave], s_cnt[wave]);
    const int p = W.p;
    ElTile<2> T; T.init(a.c.keys, W, s_mat[wave]);
    const u32 P = E * (E - 1) / 2;
    for (u32 q0 = wave * GT_EL; q0 < P; q0 += 4 * GT_EL) {
        const u32 q = q0 + W.t;
        const bool act = W.t < GT_EL && q < P;
        u32 x = 0, y = 0;
        Sh v = { 0, 0 };
        if (act) {
            pair_of(q, E, x, y);
            v = Sh{ s_s[2 * p][x] - s_s[2 * p][y], s_s[2 * p + 1][x] - s_s[2 * p + 1][y] };
        }
        const u64 e0 = t * P + q0;
        const u32 st2[2] = { 1, 2 }, w = (u32)(e0 & 7) + W.t;
        T.deal(W, a.c.op + 1, e0, st2, el_live(q0, P));
        const Dealer D = T.dealer(W);
        const Sh b = b2a(W, p, ge_bit_masks(W, p, v, D, T.zb(W, 0, w), T.zb(W, 1, w), act), D, act), nb = pub(p, 1) - b;
        if (act && W.real) {
            atomicAdd((unsigned long long *)&s_rank[2 * p][y], (unsigned long long)b.o); atomicAdd((unsigned long long *)&s_rank[2 * p + 1][y], (unsigned long long)b.n);
            atomicAdd((unsigned long long *)&s_rank[2 * p][x], (unsigned long long)nb.o); atomicAdd((unsigned long long *)&s_rank[2 * p + 1][x], (unsigned long long)nb.n);
        }
    }
    __syncthreads();
    for (u32 q0 = wave * GT_EL; q0 < k * E; q0 += 4 * GT_EL) {
        const u32 q = q0 + W.t, x = q % E, j = q / E;
        const bool act = W.t < GT_EL && q < k * E;
        Sh v = { 0, 0 };
        if (act) v = Sh{ s_rank[2 * p][x], s_rank[2 * p + 1][x] } - pub(p, j);
        const u64 e0 = t * k * E + q0;
        T.deal_mask(W, a.c.op + 2, e0, 1, el_live(q0, k * E));
        const Dealer D = T.dealer(W);
        const Sh b = b2a(W, p, eq_bit_mask(W, p, v, D, T.zb(W, 0, (u32)(e0 & 7) + W.t), act), D, act);
        if (act && W.real) {
            st(a.o, p, e0 + W.t, b);
            st(a.xe, p, (t * k + j) * ((u64)E * (a.d + 1)) + (u64)E * a.d + x, scale(b, 1ull << a.f));
            atomicAdd((unsigned long long *)&s_sum[p][j], (unsigned long long)prod3(b, Sh{ s_s[2 * p][x], s_s[2 * p + 1][x] }));
        }
    }
    __syncthreads();
    for (u32 q0 = wave * GT_EL; q0 < k; q0 += 4 * GT_EL) {
        const u32 j = q0 + W.t;
        const bool act = W.t < GT_EL && j < k;
        const u64 e0 = t * k + q0;
        T.deal_mask(W, a.c.op + 3, e0, 0, 0);
        Sh Q = pub(p, 1), z;
        for (u32 x = 0; x < E; x++) Q = Q + Sh{ s_s[2 * p][x], s_s[2 * p + 1][x] };
        z.o = (act ? s_sum[p][j] : 0) + T.za(W, 0, (u32)(e0 & 7) + W.t);
        z.n = W.reshare1(z.o, act ? 64u : 0u);
        if (act && W.real) { st(a.S, p, e0 + W.t, z); st(a.Q, p, e0 + W.t, Q); }
    }
    W.flush(a.c.wire);
}
// xe[r][a * d + i] = o[r][a] x[r / k][i]
__global__ __launch_bounds__(64) void k_moe_spread(MoeArgs a)
{
    GT_EL_SHARED(1, PRF_PAIR)
    const u64 Ed = (u64)a.E * a.d, n = a.rows * a.k * Ed;
    GT_FOR_EL(n) {
        const u64 e0 = tile_ * GT_EL, e = e0 + W.t;
        const bool act = W.t < GT_EL && e < n;
        const u64 r = e / Ed, q = e - r * Ed;
        u64 s = 0;
        if (act) s = prod3(ld(a.o, p, r * a.E + q / a.d), ld(a.x, p, r / a.k * a.d + q % a.d));
        T.deal_mask(W, a.c.op, e0, 0, 0);
        Sh z;
        z.o = s + T.za(W, 0, (u32)(e0 & 7) + W.t);
        z.n = W.reshare1(z.o, act ? 64u : 0u);
        if (act && W.real) st(a.xe, p, r * (Ed + a.E) + q, z);
        W.drain();
    }
    W.flush(a.c.wire);
}
// The hidden values of 16 columns of a row, a workgroup: h_j = ReLU of the first product's parts (left at zero; operation op), hg_j = g_j h_j rounded (op + 1), a
// wavefront per choice j, then he[a * ff + i] = sum_j o_j[a] hg_j[i] (op + 2, one reshare each), a wavefront per seven experts; the row's last workgroup does
// sum_j o_j[a] g_j, behind them.
__global__ __launch_bounds__(256) void k_moe_hidden(MoeArgs a)
{
    __shared__ uint4 s_msg[4][GT_LANES];
    __shared__ u64 s_all[4][GT_FIN_WORDS(3)];
    __shared__ u64 s_cnt[4][6];
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    u64 *s_mat = s_all[wave];
    FWire W; W.init(s_msg[wave], s_cnt[wave]);
    const int p = W.p;
    const u32 k = a.k, E = a.E, ff = a.ff, ntile = (ff + GT_FIN_EL - 1) / GT_FIN_EL;
    const u64 t = blockIdx.x / (ntile + 1), n = a.rows * k * ff, len = (u64)E * (ff + 1);
    const u32 ft = blockIdx.x % (ntile + 1);
    const bool tail = ft == ntile;
    const u32 i0 = ft * GT_FIN_EL, i = i0 + W.t;
    const bool act = !tail && i < ff;
    if (!tail)
        for (u32 j = wave; j < k; j += 4) {
            const u64 r = t * k + j, e0 = r * ff + i0, e = e0 + W.t;
            u64 z = 0;
            Sh g = { 0, 0 }, gate, y;
            if (act) {
                u64 *from = &a.Z[(u64)p * n + e];
                z = *from;
                if (W.real) *from = 0;
                g = ld(a.g, p, r);
            }
            {
                FinTile<3> T; T.keys = a.c.keys; T.mat = s_mat; T.f = a.f;
                T.deal(a.c.op, e0);
                y = finish_el<true>(W, T, a.f, z, act, gate);
            }
            {
                FinTile<2> T; T.keys = a.c.keys; T.mat = s_mat; T.f = a.f;
                T.deal(a.c.op + 1, e0);
                y = finish_el<false>(W, T, a.f, prod3(g, y), act, gate);
            }
            if (act && W.real) st(a.hg, p, e, y);
        }
    __syncthreads();
    // words of the zero sharing: nine blocks for 16 adjacent outputs, seven such runs a pass
    const u32 runs = tail ? (E + 15) / 16 : E, run = lane / 9, key = (lane % 9) / 3, grp = lane % 3;
    const u32 per = runs <= 28 ? (runs + 3) / 4 : 7;                       // runs of a wavefront at a time
    for (u32 x0 = wave * per; x0 < runs; x0 += 4 * per) {
        const u32 x = x0 + run;
        const u64 first = t * len + (tail ? (u64)E * ff + x * 16 : (u64)x * ff + i0);
        wave_sync();
        if (run < per && x < runs) {
            Key kv;
#pragma unroll
            for (int v = 0; v < 8; v++) kv.k[v] = a.c.keys[8 * key + v];
            u64 D[8];
            chacha8<PRF_PAIR>(kv, (first >> 3) + grp, a.c.op + 2, 0, D);
#pragma unroll
            for (int v = 0; v < 8; v++) s_mat[lane * 8 + v] = D[v];
        }
        wave_sync();
        const u32 most = runs - x0 < per ? runs - x0 : per;
        for (u32 q = 0; q < most; q++) {
            const u32 y = x0 + q, ex = tail ? y * 16 + W.t : y;           // expert
            const u64 at = t * len + (tail ? (u64)E * ff + y * 16 : (u64)y * ff + i0) + W.t;
            const bool on = tail ? ex < E : act;
            u64 z = 0;
            if (on)
                for (u32 j = 0; j < k; j++) {
                    const u64 r = t * k + j;
                    z += prod3(ld(a.o, p, r * E + ex), tail ? ld(a.g, p, r) : ld(a.hg, p, r * ff + i));
                }
            const u64 *m = s_mat + q * 72 + ((at - W.t) & 7) + W.t;
            Sh v = { z + (m[p * 24] - m[W.pn * 24]), 0 };
            v.n = W.reshare1(v.o, on ? 64u : 0u);
            if (on && W.real) st(a.he, p, at, v);
        }
    }
    W.flush(a.c.wire);
}
// he[t][a * ff + i] = sum_j o_j[a] hg_j[i]; behind them sum_j o_j[a] g_j
__global__ __launch_bounds__(64) void k_moe_gather(MoeArgs a)
{
    GT_EL_SHARED(1, PRF_PAIR)
    const u64 Ef = (u64)a.E * a.ff, len = Ef + a.E, n = a.rows * len;
    GT_FOR_EL(n) {
        const u64 e0 = tile_ * GT_EL, e = e0 + W.t;
        const bool act = W.t < GT_EL && e < n;
        const u64 t = e / len, q = e - t * len, x = q >= Ef ? q - Ef : q / a.ff;
        u64 s = 0;
        if (act)
            for (u32 j = 0; j < a.k; j++) {
                const u64 r = t * a.k + j;
                s += prod3(ld(a.o, p, r * a.E + x), q >= Ef ? ld(a.g, p, r) : ld(a.hg, p, r * a.ff + q % a.ff));
            }
        T.deal_mask(W, a.c.op, e0, 0, 0);
        Sh z;
        z.o = s + T.za(W, 0, (u32)(e0 & 7) + W.t);
        z.n = W.reshare1(z.o, act ? 64u : 0u);
        if (act && W.real) st(a.he, p, e, z);
        W.drain();
    }
    W.flush(a.c.wire);
}
