// A block of a network in fixed point on shares: the gated layer and its gradients, and linear attention with a decay for each head.
#pragma once
#include "gt_layers.hpp"

// ---------------------------------------------------------------------------------
// Gated layer: g = (x Wg + bg) s, u = x Wu + bu, h = g u, s ReLU's bit (or 1), f = tau fraction bits.  Both projections are one product with the weights side by side,
// ffp (ff rounded up to 64) columns each; one kernel completes g (operation c.op), u (c.op + 1) and h (c.op + 2), so that neither projection is written and
// read again.  Elements are rows of ff8 (ff rounded up to 8), so that eight adjacent ones lie in a row.
// Z: the parts, [3][rows][2 ffp], left at zero, or R: residues, planes of rows x 2 ffp.  first: the pass's first row.
// Bound: the vector units, half of them on the block function (2048 x 1024 -> 2048 with ReLU, 1.3e7 completions: 0.79 ms with three wavefronts a SIMD, 0.85 with two).
// Three were measured with ReLU, where 2 vector registers are spilled; without it 22 are (92 bytes a lane), and the same rows take longer (0.75 ms, with ReLU 0.69 on that card).
struct GatedArgs {
    KCommon c;
    u64 *Z;
    const unsigned char *R;
    u64 plane, first, rows;
    u32 nchunk, ff, ff8, ffp, f, per, nbig;
    P6 bias, h, g, u, s;                          // bias: bg, behind it bu; s: with ReLU
    int has_bias, keep;
};
// row and column of an element of the pass
struct GatedAt { u64 row; u32 col; };
__device__ __forceinline__ GatedAt gated_at(u64 i, u32 ff8, bool narrow)
{
    const u64 row = narrow ? (u64)((u32)i / ff8) : i / ff8;
    return GatedAt{ row, (u32)(i - row * ff8) };
}
template <int SRC, bool RELU>
__global__ __launch_bounds__(64, 3) void k_gated(GatedArgs a)
{
    constexpr int NS = RELU ? 3 : 2;
    __shared__ uint4 s_msg[GT_LANES];
    __shared__ u64 s_mat[(22 + 3 * NS) * GT_FP_ROW];
    __shared__ u64 s_cnt[6];
    WWire W; W.init(s_msg, s_cnt);
    const int p = W.p;
    const u32 f = a.f, t = W.t < 20 ? W.t : 19, block = blockIdx.x;
    const u64 n = a.rows * a.ff8, ld = 2 * (u64)a.ffp;
    const bool mine = W.real && W.t < 20, narrow = n <= 0xffffffffu;
    const u32 per = SRC == FIN_RES && block < a.nbig ? a.per : 1, chunk = per * GT_FP_EL;
    const u64 c0 = (SRC == FIN_RES ? (block < a.nbig ? (u64)block * a.per : (u64)a.nbig * (a.per - 1) + block) : (u64)block) * GT_FP_EL;
    // residues: lane t of a party joins eight adjacent words, of g in the first 5 per lanes, of u in the next
    const u32 half = t >= 5 * per ? 1 : 0, grp = half ? t - 5 * per : t;
    u64 zw[8];
    if (SRC == FIN_RES) {
        const u64 i = c0 + 8 * (grp < 5 * per ? grp : 5 * per - 1);
        const GatedAt at = gated_at(i < n ? i : n - 8, a.ff8, narrow);
        rns_words(a, p, at.row * ld + half * a.ffp + at.col, zw);
    }
    for (u32 k0 = 0; k0 < chunk && c0 + k0 < n; k0 += GT_FP_EL) {
        const u32 el[2] = { t, t + 20 };
        bool act[2];
        u64 zg[2], zu[2], e[2], from[2];
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const u64 i = c0 + k0 + el[q];
            GatedAt at = gated_at(i < n ? i : n - 1, a.ff8, narrow);
            act[q] = W.t < 20 && i < n && at.col < a.ff;
            if (at.col >= a.ff) at.col = a.ff - 1;                   // (words that exist where these do not)
            e[q] = (a.first + at.row) * a.ff + at.col;
            from[q] = at.row * ld + at.col;
            if (a.has_bias) { const u64 *b = own_of(a.bias, p); zg[q] = b[at.col] << f; zu[q] = b[a.ff + at.col] << f; }
            else zg[q] = zu[q] = 0;
        }
        if (SRC == FIN_PARTS) {
            u64 *Z = a.Z + (u64)p * a.rows * ld;
#pragma unroll
            for (int q = 0; q < 2; q++) { zg[q] += Z[from[q]]; zu[q] += Z[from[q] + a.ffp]; }
#pragma unroll
            for (int q = 0; q < 2; q++) if (mine && act[q]) { Z[from[q]] = 0; Z[from[q] + a.ffp] = 0; }
        } else {
            // the tile's words from the lanes that joined them, through the message region
            u64 *words = (u64 *)s_msg + GT_FP_EL * p;
            const u32 at = 8 * grp - k0;                              // (wraps for the lanes of tiles before)
#pragma unroll
            for (u32 w = 0; w < 2; w++) {
                wave_sync();
                if (half == w && grp < 5 * per && at < GT_FP_EL)
#pragma unroll
                    for (int i = 0; i < 8; i++) words[at + i] = zw[i];
                wave_sync();
                (w ? zu : zg)[0] += words[t]; (w ? zu : zg)[1] += words[t + 20];
            }
        }
        const u32 na = (u32)act[0] + (u32)act[1];
        const u64 e0 = a.first * a.ff8 + c0 + k0;
        Sh g[2], u[2], h[2], s[2], none[2];
        {
            FinPair<NS> T; T.keys = a.c.keys; T.mat = s_mat; T.f = f;
            T.deal(W, a.c.op, e0);
            finish_two<RELU>(W, T, f, zg, el, na, g, s);
        }
        FinPair<2> T; T.keys = a.c.keys; T.mat = s_mat; T.f = f;
        T.deal(W, a.c.op + 1, e0);
        finish_two<false>(W, T, f, zu, el, na, u, none);
        const u64 zh[2] = { prod3(g[0], u[0]), prod3(g[1], u[1]) };
        T.deal(W, a.c.op + 2, e0);
        finish_two<false>(W, T, f, zh, el, na, h, none);
#pragma unroll
        for (int q = 0; q < 2; q++)
            if (mine && act[q]) {
                st(a.h, p, e[q], h[q]);
                if (a.keep) { st(a.g, p, e[q], g[q]); st(a.u, p, e[q], u[q]); }
                if (RELU && a.keep) st(a.s, p, e[q], s[q]);
            }
        W.drain();
    }
    W.flush(a.c.wire);
}

// The same for few elements, 16 a workgroup, from parts: the first wavefront completes g, the second u beside it, whose material for h is there when both are: one chain of
// messages after the other, but one PRF pass before them.  Bound: those chains (1 x 128: 6.9 us, as tiles of 40 12.6).
template <bool RELU>
__global__ __launch_bounds__(128) void k_gated_few(GatedArgs a)
{
    constexpr int NS = RELU ? 3 : 2;
    __shared__ uint4 s_msg[2][GT_LANES];
    __shared__ u64 s_mat[3][GT_FIN_WORDS(3)], s_cnt[2][6], s_g[6][GT_FIN_EL];
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    FWire W; W.init(s_msg[wave], s_cnt[wave]);
    const int p = W.p;
    const u64 n = a.rows * a.ff8, ld = 2 * (u64)a.ffp, e0 = (u64)blockIdx.x * GT_FIN_EL, i = e0 + W.t;
    GatedAt at = gated_at(i < n ? i : n - 1, a.ff8, n <= 0xffffffffu);
    const bool act = i < n && at.col < a.ff;
    if (at.col >= a.ff) at.col = a.ff - 1;
    const u64 e = (a.first + at.row) * a.ff + at.col, id = a.first * a.ff8 + e0;
    u64 *Z = a.Z + ((u64)p * a.rows + at.row) * ld + at.col + (wave ? a.ffp : 0);
    u64 z = *Z;
    if (act && W.real) *Z = 0;
    if (a.has_bias) z += own_of(a.bias, p)[(wave ? a.ff : 0) + at.col] << a.f;
    Sh y, s, h;
    if (wave == 0) {
        FinTile<NS> T; T.keys = a.c.keys; T.mat = s_mat[0]; T.f = a.f;
        T.deal(a.c.op, id);
        y = finish_el<RELU>(W, T, a.f, z, act, s);
        if (W.real) { s_g[2 * p][W.t] = y.o; s_g[2 * p + 1][W.t] = y.n; }
        if (act && W.real && a.keep) { st(a.g, p, e, y); if (RELU) st(a.s, p, e, s); }
    } else {
        FinTile<2> T; T.keys = a.c.keys; T.mat = s_mat[1]; T.f = a.f;
        T.deal(a.c.op + 1, id);
        y = finish_el<false>(W, T, a.f, z, act, s);
        if (act && W.real && a.keep) st(a.u, p, e, y);
        T.mat = s_mat[2];
        T.deal(a.c.op + 2, id);
    }
    __syncthreads();
    if (wave) {
        FinTile<2> T; T.keys = a.c.keys; T.mat = s_mat[2]; T.f = a.f; T.w = ((u32)id & 7) + (threadIdx.x & 15);
        h = finish_el<false>(W, T, a.f, prod3(Sh{ s_g[2 * p][W.t], s_g[2 * p + 1][W.t] }, y), act, s);
        if (act && W.real) st(a.h, p, e, h);
    }
    W.flush(a.c.wire);
}

// Gradients behind the product and the activation: dg = s (dh u) (operation c.op, the product with the bit under its stream 3), du = dh g (c.op + 1), the components
// side by side, rows of 2 ffp: operands of the products that follow (columns behind ff are not written; they meet weights that are zero).
// Bound: the vector units (2048 x 1024, 4.2e6 completions: 0.27 ms).
struct GatedBackArgs { KCommon c; P6 dh, g, u, s; u64 *dz[3]; u64 rows, first; u32 ff, ff8, ffp, f; };           // first: the launch's first element
template <bool RELU>
__global__ __launch_bounds__(64) void k_gated_back(GatedBackArgs a)
{
    constexpr int NS = RELU ? 3 : 2;
    __shared__ uint4 s_msg[GT_LANES];
    __shared__ u64 s_mat[(22 + 3 * NS) * GT_FP_ROW];
    __shared__ u64 s_cnt[6];
    WWire W; W.init(s_msg, s_cnt);
    const int p = W.p;
    const u32 f = a.f, t = W.t < 20 ? W.t : 19;
    const u64 n = a.rows * a.ff8, c0 = a.first + (u64)blockIdx.x * GT_FP_EL;
    const bool mine = W.real && W.t < 20, narrow = n <= 0xffffffffu;
    const u32 el[2] = { t, t + 20 };
    bool act[2];
    u64 zg[2], zu[2], to[2];
    Sh s[2], dg[2], du[2], none[2];
#pragma unroll
    for (int q = 0; q < 2; q++) {
        const u64 i = c0 + el[q];
        GatedAt at = gated_at(i < n ? i : n - 1, a.ff8, narrow);
        act[q] = W.t < 20 && i < n && at.col < a.ff;
        if (at.col >= a.ff) at.col = a.ff - 1;
        const u64 e = at.row * a.ff + at.col;
        to[q] = at.row * 2 * a.ffp + at.col;
        const Sh dh = ld(a.dh, p, e);
        zg[q] = prod3(dh, ld(a.u, p, e)); zu[q] = prod3(dh, ld(a.g, p, e));
        if (RELU) s[q] = ld(a.s, p, e);
    }
    const u32 na = (u32)act[0] + (u32)act[1];
    {
        FinPair<NS> T; T.keys = a.c.keys; T.mat = s_mat; T.f = f;
        T.deal(W, a.c.op, c0);
        finish_two<false>(W, T, f, zg, el, na, dg, none);
        if (RELU) {
            u64 m[2], rcv[2];
#pragma unroll
            for (int q = 0; q < 2; q++) m[q] = prod3(s[q], dg[q]) + T.za(W, 2, el[q]);
            W.reshare64<2>(m, rcv);
            W.nresh += 64u * na;
#pragma unroll
            for (int q = 0; q < 2; q++) dg[q] = Sh{ m[q], rcv[q] };
        }
    }
    FinPair<2> T; T.keys = a.c.keys; T.mat = s_mat; T.f = f;
    T.deal(W, a.c.op + 1, c0);
    finish_two<false>(W, T, f, zu, el, na, du, none);
    u64 *dz = p == 0 ? a.dz[0] : (p == 1 ? a.dz[1] : a.dz[2]);
#pragma unroll
    for (int q = 0; q < 2; q++) if (mine && act[q]) { dz[to[q]] = dg[q].o; dz[to[q] + a.ffp] = du[q].o; }
    W.flush(a.c.wire);
}

// The same for few elements, 16 a workgroup: the first wavefront completes dg, the second du.
template <bool RELU>
__global__ __launch_bounds__(128) void k_gated_back_few(GatedBackArgs a)
{
    __shared__ uint4 s_msg[2][GT_LANES];
    __shared__ u64 s_mat[2][GT_FIN_WORDS(3)], s_cnt[2][6];
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    FWire W; W.init(s_msg[wave], s_cnt[wave]);
    const int p = W.p;
    const u64 n = a.rows * a.ff8, e0 = (u64)blockIdx.x * GT_FIN_EL, i = e0 + W.t;
    GatedAt at = gated_at(i < n ? i : n - 1, a.ff8, n <= 0xffffffffu);
    const bool act = i < n && at.col < a.ff;
    if (at.col >= a.ff) at.col = a.ff - 1;
    const u64 e = at.row * a.ff + at.col;
    const u64 z = prod3(ld(a.dh, p, e), wave ? ld(a.g, p, e) : ld(a.u, p, e));
    Sh y, none;
    if (wave == 0) {
        Sh s = { 0, 0 };
        if (RELU) s = ld(a.s, p, e);
        FinTile<RELU ? 3 : 2> T; T.keys = a.c.keys; T.mat = s_mat[0]; T.f = a.f;
        T.deal(a.c.op, e0);
        y = finish_el<false>(W, T, a.f, z, act, none);
        if (RELU) y = mult_sh(W, s, y, T.za(W, 2), act);
    } else {
        FinTile<2> T; T.keys = a.c.keys; T.mat = s_mat[1]; T.f = a.f;
        T.deal(a.c.op + 1, e0);
        y = finish_el<false>(W, T, a.f, z, act, none);
    }
    u64 *dz = p == 0 ? a.dz[0] : (p == 1 ? a.dz[1] : a.dz[2]);
    if (act && W.real) dz[at.row * 2 * a.ffp + at.col + (wave ? a.ffp : 0)] = y.o;
    W.flush(a.c.wire);
}

// ---------------------------------------------------------------------------------
// Linear attention, 64 tokens (a chunk) at a time, s = f + 12, D[n] = decay^n with 12 fraction bits:
//   P_ij = floor((D[i-j] q_i k_j + 2^(s-1)) / 2^s), j <= i                       operation c.op,     element b * 2080 + i (i + 1) / 2 + j
//   S'   = floor((2^f D[c] S + sum_j D[c-1-j] k_j v_j + 2^(s-1)) / 2^s)            c.op + 1,           element b * pk + row * dv + column
//   o_i  = floor((2^12 sum_j P_ij v_j + D[i+1] q_i S + 2^(s-1)) / 2^s)             c.op + 2,           element (b * 64 + i) * dv8 + column
// for chunk b = (sequence * heads + head) * chunks + chunk, c tokens of it, S the state before it; pk, dv8: dk dv and dv rounded up to 8.
//   k_lin_parts    the parts of D q k^T and of (D k)^T v, every chunk by itself
//   k_lin_states   the states one after the other, an element's chain in one wavefront; beside them the scores' completion
//   k_lin_out      the parts of [2^12 P, D q] [v; S]
//   k_lin_finish   their completion
// Bound: the completions' vector instructions, 1,170 to 1,270 a tile of 40, 770 of them the block function's (16 heads, 4096 tokens, 64 x 128: states and scores 456 us,
// outputs 402), then the products (286 and 385 us).
// A pass takes chunks ch0 .. ch0 + nch - 1 of sequences' heads bh0 .. bh0 + nbh - 1; b' = (bh - bh0) * nch + chunk - ch0 counts in its workspace.
#define GT_LIN_CHUNK 64
#define GT_LIN_TRI 2080
#define GT_LIN_DECAY 12                           // fraction bits of a decay: with tau <= 20 a completion's shift stays within 32, one half of the tree of ANDs
struct LinArgs {
    KCommon c;
    const u64 *q[3], *k[3], *v[3];
    P6 in, out, o;                                // states before and after, outputs
    const u32 *D;                                 // [head][65]
    u64 ldq, ldk, ldv, T;
    u32 H, dk, dv, dv8, pk, f, has_in;
    u64 nc, bh0;                                  // chunks of a sequence
    u32 ch0, nch, nbh;
    u64 *Zs, *Zk, *Zo, *P, *S;                    // parts [3][b'][2080], [pk], [64 dv8]; scores [3][b'][2080], states before a chunk [3][b'][pk]
    u32 tiles, each, per;                         // k_lin_states: workgroups of chains; k_lin_states, k_lin_finish: tiles of 40 of a head's chunks in the pass; tiles of a wavefront
};

struct LinChunk { u64 t0; u32 bh, h, len; };     // first row of q, k, v; head; tokens
__device__ __forceinline__ LinChunk lin_chunk(const LinArgs &a, u32 bhl, u32 ch)
{
    LinChunk r;
    const u64 bh = a.bh0 + bhl, t = (u64)ch * GT_LIN_CHUNK;
    r.bh = (u32)bh; r.h = (u32)(bh % a.H);
    r.t0 = bh / a.H * a.T + t;
    r.len = a.T - t < GT_LIN_CHUNK ? (u32)(a.T - t) : GT_LIN_CHUNK;
    return r;
}
__device__ __forceinline__ const u64 *comp_of(const u64 *const (&x)[3], int j) { return j == 0 ? x[0] : (j == 1 ? x[1] : x[2]); }

// Limbs of a lane's 16 words, as operands of v_mfma_i32_16x16x64_i8.
__device__ __forceinline__ void lin_limbs(const u64 (&x)[16], v4i (&B)[8])
{
    u64 y[8], z[8];
#pragma unroll
    for (int i = 0; i < 8; i++) { y[i] = (x[i] + GT_BIAS) ^ GT_BIAS; z[i] = (x[8 + i] + GT_BIAS) ^ GT_BIAS; }
    transpose8x8(y); transpose8x8(z);
#pragma unroll
    for (int i = 0; i < 8; i++) B[i] = v4i{ (int)(u32)y[i], (int)(u32)(y[i] >> 32), (int)(u32)z[i], (int)(u32)(z[i] >> 32) };
}
// The word that sums of products of limbs stand for, sum of D_u 256^u: bytes with carries below 2^32, above it modulo 2^32.
__device__ __forceinline__ u64 lin_word(const v4i (&acc)[8], int v)
{
    const int t0 = acc[0][v], t1 = acc[1][v] + (t0 >> 8), t2 = acc[2][v] + (t1 >> 8), t3 = acc[3][v] + (t2 >> 8), t4 = acc[4][v] + (t3 >> 8);
    const u32 high = (u32)t4 + ((u32)acc[5][v] << 8) + ((u32)acc[6][v] << 16) + ((u32)acc[7][v] << 24);
    return (u64)low_bytes((u32)t0, (u32)t1, (u32)t2, (u32)t3) | ((u64)high << 32);
}

enum { LIN_SCORES = 0, LIN_KV = 1, LIN_OUT = 2 };
#define GT_LIN_LDS (2 * 2 * 8 * 1024 + 64 * 4)
// A party's parts of 32 rows x 64 columns of a chunk's product, on the matrix cores in signed 8-bit limbs (36 products of limbs a ring product):
// z_p = x_p (y_p + y_{p+1}) + x_{p+1} y_p, terms in steps of 64.  A wavefront owns 16 columns, whose words stay in registers and become limbs there; the rows' limbs go through LDS,
// [component p or p + 1][16 rows][limb][lane][16 bytes], a block of them made by each wavefront.  A block of 16 rows (or columns) whose terms are adjacent in memory is loaded
// a row at a time, whole lines, and turned in LDS, where its limbs go afterwards.
// Bound: instructions of the vector units around the matrix instructions, which a SIMD's two or three wavefronts overlap in part (outputs of 16 heads, 4096 tokens, 64 x 128: 1.0e8 and
// 1.4e7 of them, 47 and 27 % of 385 us).  k_lin_parts spills 12 vector registers (52 bytes a lane) at its three wavefronts a SIMD, k_lin_out none at its two.  Three parties a workgroup, six wavefronts: 414 and 691 us instead of 286 and 385, as one such workgroup fits a compute unit.
template <int JOB>
__device__ __forceinline__ void lin_tile(const LinArgs &a, u32 lb, u32 p, u32 r0, u32 c0, unsigned char *s_a)
{
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    u32 lane = threadIdx.x & 63, lr = lane & 15, kq = lane >> 4;
    const u32 bhl = lb / a.nch, nb = a.nbh * a.nch;
    const LinChunk ck = lin_chunk(a, bhl, a.ch0 + lb % a.nch);
    const u32 len = ck.len, dk = a.dk, dv = a.dv, M = JOB == LIN_KV ? dk : len, N = JOB == LIN_SCORES ? len : dv;
    if (r0 >= M || c0 >= N) return;
    const u32 *D = a.D + ck.h * (GT_LIN_CHUNK + 1);
    const u32 nstep = JOB == LIN_KV ? 1 : (dk + 63) / 64 + (JOB == LIN_OUT ? 1 : 0), pn = p == 2 ? 0 : p + 1, first = c0 + 16 * wave;
    const bool cols = first < N && (JOB != LIN_SCORES || first <= r0 + 31);
    const u64 hq = ck.t0 * a.ldq + (u64)ck.h * dk, hk = ck.t0 * a.ldk + (u64)ck.h * dk, hv = ck.t0 * a.ldv + (u64)ck.h * dv;
    u32 *s_D = (u32 *)(s_a + 2 * 2 * 8 * 1024);                           // powers by the tokens between, or of a token's age (the loop's first barrier is theirs)
    if (threadIdx.x < 64) s_D[threadIdx.x] = threadIdx.x < len ? D[JOB == LIN_KV ? len - 1 - threadIdx.x : threadIdx.x + (JOB == LIN_OUT ? 1 : 0)] : 0;
    // 16 rows of 64 words through 8 KB of LDS: row i's word at(i) by lane, blocks of two words exchanged by row against bank conflicts
    auto turn = [&](unsigned char *to, u64 (&x)[16]) {
        wave_sync();
#pragma unroll
        for (int i = 0; i < 16; i++) *(u64 *)(to + i * 512 + (((lane >> 1) ^ i) * 16) + (lane & 1) * 8) = x[i];
        wave_sync();
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const ulonglong2 v = *(const ulonglong2 *)(to + lr * 512 + (((kq * 8 + i) ^ lr) * 16));
            x[2 * i] = v.x; x[2 * i + 1] = v.y;
        }
        wave_sync();
    };
    // terms k0 + lane of rows f .. f + 15 of a matrix of `rows` rows of K terms (zero where there are none)
    auto by_rows = [&](const u64 *m, u64 ld, u32 f, u32 rows, u32 k0, u32 K, u64 (&x)[16]) {
        if (k0 + 64 <= K && f + 16 <= rows) {
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = ld_at<u64>(m + k0 + (u64)(f + i) * ld, lane * 8);
            return;
        }
        const u32 k = k0 + lane, at = (k < K ? k : K - 1) * 8;
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = ld_at<u64>(m + (u64)(f + i < rows ? f + i : rows - 1) * ld, at);
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = k < K && f + i < rows ? x[i] : 0;
    };
    // terms k0 + 16 kq .. of column c + lr (of `columns`) of a matrix whose rows are terms (a chunk's rows lie within 32-bit offsets)
    auto by_terms = [&](const u64 *m, u32 ld, u32 c, u32 columns, u32 k0, u32 K, u64 (&x)[16]) {
        if (k0 + 64 <= K && c + 16 <= columns) {                          // (uniform addresses)
            const u32 off = (16 * kq * ld + lr) * 8;
#pragma unroll
            for (int i = 0; i < 16; i++) x[i] = ld_at<u64>(m + c + (u64)(k0 + i) * ld, off);
            return;
        }
        const u32 k = k0 + 16 * kq, cc = c + lr < columns ? c + lr : columns - 1;
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = ld_at<u64>(m, ((k + i < K ? k + i : K - 1) * ld + cc) * 8);
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = k + i < K && c + lr < columns ? x[i] : 0;
    };
    u32 here = r0;
    v4i acc[2][8];
#pragma unroll
    for (int i = 0; i < 16; i++) acc[i >> 3][i & 7] = v4i{ 0, 0, 0, 0 };
#pragma unroll 1
    for (u32 step = 0; step < nstep; step++) {
        const bool scores = JOB == LIN_OUT && step == 0;                  // the step of the scores and values
        const u32 k0 = JOB == LIN_KV || scores ? 0 : 64 * (JOB == LIN_OUT ? step - 1 : step);
        // (a step works its addresses out again: kept over the steps they take the registers of the sums)
        asm volatile("" : "+v"(lane), "+s"(here));
        lr = lane & 15; kq = lane >> 4;
        u64 y[16], t[16];
        __syncthreads();
        auto right = [&]() {
            if (!cols) return;
#pragma unroll
            for (int w = 0; w < 2; w++) {
                const int j = (int)(w ? pn : p);
                if (JOB == LIN_SCORES) {
                    by_rows(comp_of(a.k, j) + hk, a.ldk, first, N, k0, dk, w ? t : y);
                    turn(s_a + wave * 8192, w ? t : y);
                } else {
                    const bool tokens = JOB == LIN_KV || scores;
                    by_terms(tokens ? comp_of(a.v, j) + hv : a.S + ((u64)j * nb + lb) * a.pk, tokens ? (u32)a.ldv : dv, first, N, k0, tokens ? len : dk, w ? t : y);
                }
            }
#pragma unroll
            for (int i = 0; i < 16; i++) t[i] += y[i];
        };
        if (JOB == LIN_SCORES) right();                                // (through the LDS that the rows' limbs go to)
        {
            const u32 j = wave >> 1 ? pn : p, row = here + (wave & 1) * 16;
            unsigned char *to = s_a + wave * 8192;
            u64 x[16];
            v4i L[8];
            if (JOB == LIN_KV) {
                by_terms(comp_of(a.k, (int)j) + hk, (u32)a.ldk, row, M, 0, len, x);
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    const uint4 w = *(const uint4 *)(s_D + 16 * kq + i);
                    x[i] *= w.x; x[i + 1] *= w.y; x[i + 2] *= w.z; x[i + 3] *= w.w;
                }
            } else if (scores) {
                const u64 *P = a.P + ((u64)j * nb + lb) * GT_LIN_TRI;
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const u32 r = row + i < M ? row + i : M - 1;
                    x[i] = ld_at<u64>(P + r * (r + 1) / 2, (lane <= r ? lane : r) * 8);
                }
#pragma unroll
                for (int i = 0; i < 16; i++) x[i] = row + i < M && lane <= row + i ? x[i] : 0;
                turn(to, x);
#pragma unroll
                for (int i = 0; i < 16; i++) x[i] <<= GT_LIN_DECAY;
            } else {
                by_rows(comp_of(a.q, (int)j) + hq, a.ldq, row, M, k0, dk, x);
                turn(to, x);
                if (JOB == LIN_OUT) {
                    const u32 w = s_D[row + lr];
#pragma unroll
                    for (int i = 0; i < 16; i++) x[i] *= w;
                }
            }
            lin_limbs(x, L);
#pragma unroll
            for (int sl = 0; sl < 8; sl++) *(v4i *)(to + sl * 1024 + lane * 16) = L[sl];
        }
        if (JOB != LIN_SCORES) right();
        __syncthreads();
        if (!cols) continue;
        v4i B[8];
#pragma unroll
        for (int w = 0; w < 2; w++) {
            lin_limbs(w ? y : t, B);
            const unsigned char *A0 = s_a + w * 16384 + lane * 16;
#pragma unroll
            for (int rt = 0; rt < 2; rt++)
#pragma unroll
                for (int sl = 0; sl < 8; sl++) {
                    const v4i A = *(const v4i *)(A0 + (rt * 8 + sl) * 1024);
#pragma unroll
                    for (int u = 0; u < 8 - sl; u++) acc[rt][sl + u] = __builtin_amdgcn_mfma_i32_16x16x64_i8(A, B[u], acc[rt][sl + u], 0, 0, 0);
                }
        }
    }
    if (!cols) return;
    // (at most 320 terms of two products: |sums| < 2^27)
    const u32 col = first + lr, ld = JOB == LIN_KV ? dv : a.dv8;
    const u64 at = (u64)p * nb + lb;
    u64 *const Z = JOB == LIN_SCORES ? a.Zs + at * GT_LIN_TRI : JOB == LIN_KV ? a.Zk + at * a.pk : a.Zo + at * GT_LIN_CHUNK * a.dv8;
#pragma unroll
    for (int rt = 0; rt < 2; rt++)
#pragma unroll
        for (int v = 0; v < 4; v++) {
            const u32 row = r0 + rt * 16 + 4 * kq + v;
            u64 z = lin_word(acc[rt], v);
            if (JOB == LIN_SCORES) z *= s_D[col <= row ? row - col : 0];
            if (row < M && col < N && (JOB != LIN_SCORES || col <= row))
                *(u64 *)((char *)Z + (JOB == LIN_SCORES ? row * (row + 1) / 2 + col : row * ld + col) * 8) = z;
        }
}
// Workgroups go to the XCDs in turn: XCD x takes the x-th eighth of the work, so that a chunk's words are in one L2 (16 heads, 4096 tokens, 64 x 128: 467 -> 414 us).
__device__ __forceinline__ u32 lin_block(u32 total)
{
    const u32 per = (total + 7) / 8, id = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    return (blockIdx.x >> 3) < per && id < total ? id : ~0u;
}
// a chunk's workgroups, for each party: two of its scores, then its products k^T v
__global__ __launch_bounds__(256, 3) void k_lin_parts(LinArgs a)
{
    __shared__ __align__(16) unsigned char s_a[GT_LIN_LDS];
    const u32 ct = (a.dv + 63) / 64, per = 3 * (2 + (a.dk + 31) / 32 * ct), id = lin_block(a.nbh * a.nch * per), lb = id / per, t = id % per / 3, p = id % 3;
    if (id == ~0u) return;
    if (t < 2) lin_tile<LIN_SCORES>(a, lb, p, 32 * t, 0, s_a);
    else lin_tile<LIN_KV>(a, lb, p, (t - 2) / ct * 32, (t - 2) % ct * 64, s_a);
}
__global__ __launch_bounds__(256, 2) void k_lin_out(LinArgs a)
{
    __shared__ __align__(16) unsigned char s_a[GT_LIN_LDS];
    const u32 ct = (a.dv + 63) / 64, per = 6 * ct, id = lin_block(a.nbh * a.nch * per), lb = id / per, t = id % per / 3, p = id % 3;
    if (id == ~0u) return;
    lin_tile<LIN_OUT>(a, lb, p, t / ct * 32, t % ct * 64, s_a);
}

// Completion of tiles of 40, a wavefront's `per` tiles one after the other.
struct LinTile {
    WWire W;
    FinPair<2> T;
    u32 t, s, el[2];
    bool mine;
    __device__ __forceinline__ LinTile(const LinArgs &a, uint4 *msg, u64 *mat, u64 *cnt)
    {
        W.init(msg, cnt);
        T.keys = a.c.keys; T.mat = mat; T.f = s = a.f + GT_LIN_DECAY;
        t = W.t < 20 ? W.t : 19; el[0] = t; el[1] = t + 20;
        mine = W.real && W.t < 20;
    }
    __device__ __forceinline__ void finish(u32 op, u64 e0, const u64 (&z)[2], u32 na, Sh (&y)[2])
    {
        Sh none[2];
        T.deal(W, op, e0);
        finish_two<false>(W, T, s, z, el, na, y, none);
    }
};
#define GT_LIN_SHARED __shared__ uint4 s_msg[GT_LANES]; __shared__ u64 s_mat[28 * GT_FP_ROW]; __shared__ u64 s_cnt[6]; LinTile L(a, s_msg, s_mat, s_cnt);

// Workgroups below `tiles`: 40 elements of a head's state, all chunks of the pass; the others: `per` tiles of 40 scores for each wavefront.
// PAIR: of a chain's two wavefronts one deals the material of the next chunk while the other completes this one; for chains that are too few to fill the SIMDs.
template <bool PAIR>
__global__ __launch_bounds__(PAIR ? 128 : 64) void k_lin_states(LinArgs a)
{
    constexpr int NW = PAIR ? 2 : 1;
    __shared__ uint4 s_msg[NW][GT_LANES];
    __shared__ u64 s_mat[NW][28 * GT_FP_ROW], s_cnt[NW][6];
    const u32 wave = PAIR ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
    LinTile L(a, s_msg[wave], s_mat[wave], s_cnt[wave]);
    const int p = L.W.p;
    const u32 nb = a.nbh * a.nch, row = GT_LIN_TRI / GT_FP_EL;
    bool act[2];
    u64 z[2];
    Sh y[2], none[2];
    if (blockIdx.x >= a.tiles) {
        for (u32 i = 0; i < a.per; i++) {
            const u32 b = ((blockIdx.x - a.tiles) * NW + wave) * a.per + i, bhl = b / a.each, tile = b % a.each, chl = tile / row, i0 = tile % row * GT_FP_EL;
            if (bhl >= a.nbh) break;
            const LinChunk ck = lin_chunk(a, bhl, a.ch0 + chl);
            const u32 n = ck.len * (ck.len + 1) / 2;
            const u64 at = ((u64)p * nb + bhl * a.nch + chl) * GT_LIN_TRI + i0;
#pragma unroll
            for (int q = 0; q < 2; q++) { act[q] = L.W.t < 20 && i0 + L.el[q] < n; z[q] = act[q] ? a.Zs[at + L.el[q]] : 0; }
            L.finish(a.c.op, ((u64)ck.bh * a.nc + a.ch0 + chl) * GT_LIN_TRI + i0, z, (u32)act[0] + (u32)act[1], y);
#pragma unroll
            for (int q = 0; q < 2; q++) if (L.mine && act[q]) a.P[at + L.el[q]] = y[q].o;
        }
        L.W.flush(a.c.wire);
        return;
    }
    const u32 dkv = a.dk * a.dv, per = (dkv + GT_FP_EL - 1) / GT_FP_EL, bhl = blockIdx.x / per, i0 = blockIdx.x % per * GT_FP_EL;
    const u64 bh = a.bh0 + bhl, e0 = (bh * a.nc + a.ch0) * a.pk + i0;
    const u32 *D = a.D + (u32)(bh % a.H) * (GT_LIN_CHUNK + 1);
    if (PAIR && wave) {
        for (u32 chl = 0; chl < a.nch; chl++) {
            L.T.mat = s_mat[chl & 1];
            L.T.deal(L.W, a.c.op + 1, e0 + (u64)chl * a.pk);
            __syncthreads();                                          // (dealt; and the chunk before is completed)
        }
        return;
    }
    u64 next[2];
#pragma unroll
    for (int q = 0; q < 2; q++) {
        act[q] = L.W.t < 20 && i0 + L.el[q] < dkv;
        y[q] = act[q] && a.has_in ? ld(a.in, p, bh * dkv + i0 + L.el[q]) : Sh{ 0, 0 };
        next[q] = act[q] ? a.Zk[((u64)p * nb + bhl * a.nch) * a.pk + i0 + L.el[q]] : 0;
    }
    for (u32 chl = 0; chl < a.nch; chl++) {
        const LinChunk ck = lin_chunk(a, bhl, a.ch0 + chl);
        const u64 at = ((u64)p * nb + bhl * a.nch + chl) * a.pk + i0;
#pragma unroll
        for (int q = 0; q < 2; q++) {
            z[q] = ((y[q].o * D[ck.len]) << a.f) + next[q];
            if (L.mine && act[q]) a.S[at + L.el[q]] = y[q].o;
            if (chl + 1 < a.nch) next[q] = act[q] ? a.Zk[at + a.pk + L.el[q]] : 0;
        }
        if (PAIR) { L.T.mat = s_mat[chl & 1]; __syncthreads(); }
        else L.T.deal(L.W, a.c.op + 1, e0 + (u64)chl * a.pk);
        finish_two<false>(L.W, L.T, L.s, z, L.el, (u32)act[0] + (u32)act[1], y, none);
    }
#pragma unroll
    for (int q = 0; q < 2; q++) if (L.mine && act[q]) st(a.out, p, bh * dkv + i0 + L.el[q], y[q]);
    L.W.flush(a.c.wire);
}

__global__ __launch_bounds__(64) void k_lin_finish(LinArgs a)
{
    GT_LIN_SHARED
    const int p = L.W.p;
    const u32 nb = a.nbh * a.nch, full = (GT_LIN_CHUNK * a.dv8 + GT_FP_EL - 1) / GT_FP_EL;
    for (u32 j = 0; j < a.per; j++) {
        const u32 id = blockIdx.x * a.per + j, bhl = id / a.each, tile = id % a.each, chl = tile / full, i0 = tile % full * GT_FP_EL;
        if (bhl >= a.nbh) break;
        const LinChunk ck = lin_chunk(a, bhl, a.ch0 + chl);
        const u64 from = ((u64)p * nb + bhl * a.nch + chl) * GT_LIN_CHUNK * a.dv8;
        bool act[2];
        u64 z[2], to[2];
        Sh y[2];
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const u32 i = i0 + L.el[q], row = i / a.dv8, col = i % a.dv8;
            act[q] = L.W.t < 20 && row < ck.len && col < a.dv;
            z[q] = act[q] ? a.Zo[from + i] : 0;
            to[q] = (ck.t0 + row) * ((u64)a.H * a.dv) + (u64)ck.h * a.dv + col;
        }
        L.finish(a.c.op + 2, ((u64)ck.bh * a.nc + a.ch0 + chl) * GT_LIN_CHUNK * a.dv8 + i0, z, (u32)act[0] + (u32)act[1], y);
#pragma unroll
        for (int q = 0; q < 2; q++) if (L.W.real && act[q]) st(a.o, p, to[q], y[q]);
    }
    L.W.flush(a.c.wire);
}

// A token of every sequence: its score, output and state in one launch, without a workspace.  Workgroups below nout: 40 outputs of a head, whose one score, q k, the first
// wavefront works out (each such workgroup for itself) while the second deals the outputs' material and the others make q S, a sixth of the state's rows each
// (states come from memory, where the token before has put them: in place, one sequence of 16 heads of 64 x 64, both launches 21 us, with two wavefronts for it 35); the other workgroups: `per` tiles of 40 words of a
// state for each wavefront.  Where the new states take the place of the old ones, two launches: outputs first (4 heads of 64 x 64: 9.1 us in one launch, in place 11.8 + 8.5;
// 16 heads 10.2, 11.9 + 9.3).
// Bound: many sequences: the completions' block function; few: the outputs' two chains of messages.
#define GT_LIN_TOKEN 8
__global__ __launch_bounds__(64 * GT_LIN_TOKEN, 4) void k_lin_token(LinArgs a, u32 nout)
{
    __shared__ uint4 s_msg[GT_LIN_TOKEN][GT_LANES];
    __shared__ u64 s_mat[GT_LIN_TOKEN][28 * GT_FP_ROW], s_cnt[GT_LIN_TOKEN][6];
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    LinTile L(a, s_msg[wave], s_mat[wave], s_cnt[wave]);
    const int p = L.W.p, pn = L.W.pn;
    const u32 dk = a.dk, dv = a.dv, dkv = dk * dv;
    const u64 *q0 = comp_of(a.q, p), *q1 = comp_of(a.q, pn), *k0 = comp_of(a.k, p), *k1 = comp_of(a.k, pn), *v0 = comp_of(a.v, p), *v1 = comp_of(a.v, pn);
    bool act[2];
    u64 z[2];
    Sh y[2];
    if (blockIdx.x < nout) {
        const u32 ct = (a.dv8 + GT_FP_EL - 1) / GT_FP_EL, bh = blockIdx.x / ct, tile = blockIdx.x % ct, h = bh % a.H, seq = bh / a.H;
        const u64 hq = seq * a.ldq + (u64)h * dk, hk = seq * a.ldk + (u64)h * dk, hv = seq * a.ldv + (u64)h * dv;
        const u64 w = a.D[h * (GT_LIN_CHUNK + 1) + 1];
        u32 col[2];
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const u32 c = tile * GT_FP_EL + L.el[i];
            act[i] = L.W.t < 20 && c < dv;
            col[i] = c < dv ? c : dv - 1;
        }
        const u64 eo = (u64)bh * GT_LIN_CHUNK * a.dv8 + tile * GT_FP_EL;
        if (wave == 1) {
            L.T.deal(L.W, a.c.op + 2, eo);
            __syncthreads();
            return;
        }
        if (wave) {
            u64 acc[2] = { 0, 0 };
            if (a.has_in) {
                const u64 *s0 = own_of(a.in, p) + (u64)bh * dkv, *s1 = own_of(a.in, pn) + (u64)bh * dkv;
                const u32 each = (dk + GT_LIN_TOKEN - 3) / (GT_LIN_TOKEN - 2), d0 = (wave - 2) * each, d1 = d0 + each < dk ? d0 + each : dk;
#pragma unroll 8
                for (u32 d = d0; d < d1; d++) {
                    const Sh x = { q0[hq + d], q1[hq + d] };
#pragma unroll
                    for (int i = 0; i < 2; i++) acc[i] += prod3(x, Sh{ s0[d * dv + col[i]], s1[d * dv + col[i]] });
                }
            }
#pragma unroll
            for (int i = 0; i < 2; i++) if (L.mine) s_mat[wave][GT_FP_EL * p + L.el[i]] = acc[i];
            __syncthreads();
            return;
        }
        const Sh v[2] = { { v0[hv + col[0]], v1[hv + col[0]] }, { v0[hv + col[1]], v1[hv + col[1]] } };
        u64 dot = 0;
        if (L.mine) for (u32 d = L.t; d < dk; d += 20) dot += prod3(Sh{ q0[hq + d], q1[hq + d] }, Sh{ k0[hk + d], k1[hk + d] });
        u64 *sum = (u64 *)s_msg[0];
        wave_sync();
        if (L.mine) sum[20 * p + L.t] = dot;
        wave_sync();
        z[0] = 0; z[1] = 0;
#pragma unroll
        for (int i = 0; i < 20; i++) z[0] += sum[20 * p + i];
        z[0] <<= GT_LIN_DECAY;
        L.finish(a.c.op, (u64)bh * GT_LIN_TRI, z, tile == 0 && L.W.t == 0 ? 1u : 0u, y);
        const int from = (int)L.W.lane_of(0);
        const Sh P = { (u64)__shfl((unsigned long long)y[0].o, from, GT_LANES), (u64)__shfl((unsigned long long)y[0].n, from, GT_LANES) };
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; i++) {
            u64 qs = 0;
#pragma unroll
            for (int j = 2; j < GT_LIN_TOKEN; j++) qs += s_mat[j][GT_FP_EL * p + L.el[i]];
            z[i] = (prod3(P, v[i]) << GT_LIN_DECAY) + qs * w;
        }
        L.T.mat = s_mat[1];
        Sh none[2];
        finish_two<false>(L.W, L.T, L.s, z, L.el, (u32)act[0] + (u32)act[1], y, none);
#pragma unroll
        for (int i = 0; i < 2; i++) if (L.mine && act[i]) st(a.o, p, (u64)bh * dv + col[i], y[i]);
        L.W.flush(a.c.wire);
        return;
    }
    const u32 tiles = (dkv + GT_FP_EL - 1) / GT_FP_EL;
    for (u32 j = 0; j < a.per; j++) {
        const u32 id = ((blockIdx.x - nout) * GT_LIN_TOKEN + wave) * a.per + j, bh = id / tiles, i0 = id % tiles * GT_FP_EL, h = bh % a.H, seq = bh / a.H;
        if (bh >= a.nbh) break;
        const u64 hk = seq * a.ldk + (u64)h * dk, hv = seq * a.ldv + (u64)h * dv, w = a.D[h * (GT_LIN_CHUNK + 1) + 1], at = (u64)bh * dkv + i0;
#pragma unroll
        for (int i = 0; i < 2; i++) {
            const u32 e = i0 + L.el[i] < dkv ? i0 + L.el[i] : dkv - 1, d = e / dv, c = e - d * dv;
            act[i] = L.W.t < 20 && i0 + L.el[i] < dkv;
            z[i] = prod3(Sh{ k0[hk + d], k1[hk + d] }, Sh{ v0[hv + c], v1[hv + c] }) << GT_LIN_DECAY;
            if (a.has_in) z[i] += (own_of(a.in, p)[(u64)bh * dkv + e] * w) << a.f;
        }
        L.finish(a.c.op + 1, (u64)bh * a.pk + i0, z, (u32)act[0] + (u32)act[1], y);
#pragma unroll
        for (int i = 0; i < 2; i++) if (L.mine && act[i]) st(a.out, p, at + L.el[i], y[i]);
    }
    L.W.flush(a.c.wire);
}

// Powers of the heads' decays, 12 fraction bits, rounded from 46: D[n] = round(E[n] / 2^34), E[0] = 2^46, E[n + 1] = round(E[n] w / 2^12).
struct DecayArgs { u32 w[GT_MAX_HEADS]; u32 *D; u32 heads; };
__global__ __launch_bounds__(GT_MAX_HEADS) void k_lin_decays(DecayArgs a)
{
    const u32 h = threadIdx.x;
    if (h >= a.heads) return;
    u64 E = 1ull << 46;
    for (u32 n = 0; n <= GT_LIN_CHUNK; n++) {
        a.D[h * (GT_LIN_CHUNK + 1) + n] = (u32)((E + (1ull << 33)) >> 34);
        E = (E * a.w[h] + (1u << (GT_LIN_DECAY - 1))) >> GT_LIN_DECAY;
    }
}
