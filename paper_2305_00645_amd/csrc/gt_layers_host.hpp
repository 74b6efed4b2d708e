// Host side of the layers: argument checks, the operation schedule, message accounting, launches (part of gtree.hip).
#pragma once

// Words of a weight matrix in tiles (see MatView), rows and columns padded to multiples of 64, zero there.
struct WMat {
    u64 *base = nullptr;
    u64 K = 0, N = 0;
    u32 nst = 0;                 // tiles of 64 rows
};
static int wmat_alloc(WMat &w, u64 K, u64 N, hipStream_t st)
{
    w.K = K; w.N = N; w.nst = (u32)((K + 63) / 64);
    const u64 words = (N + 63) / 64 * 4 * w.nst * 3 * GT_WTILE;
    if (hipMalloc(&w.base, words * 8) != hipSuccess) { w.base = nullptr; return GT_ENOMEM; }
    HIPCHK(hipMemsetAsync(w.base, 0, words * 8, st));
    return GT_OK;
}
static int wmat_put(gt_ctx *c, const WMat &w, const gt_shares *src, u64 row0, u64 rows, u64 col0, u64 cols)
{
    PutArgs a{};
    a.src = to_p6(src); a.dst = w.base; a.row0 = row0; a.rows = rows; a.col0 = col0; a.cols = cols; a.nst = w.nst;
    return launch(c, GT_KC_LOCAL, k_put, g1(((row0 + rows + 1) / 2 - row0 / 2) * cols), B256, a);
}
static int wmat_put(gt_ctx *c, const WMat &w, const gt_shares *src, u64 row0, u64 rows) { return wmat_put(c, w, src, row0, rows, 0, w.N); }
static MatView wmat(const WMat &w, u32 kind)
{ MatView v{}; for (int j = 0; j < 3; j++) v.c[j] = w.base + (u64)j * GT_WTILE; v.kind = kind; v.nst = w.nst; return v; }
static MatView view(P6 a, u64 ld, u32 kind) { MatView v{}; for (int j = 0; j < 3; j++) v.c[j] = a.o[j]; v.ld = ld; v.kind = kind; return v; }

struct gt_dense { u32 din, dout; bool has_b; WMat W; DSh b; };
struct gt_moe {
    u32 d, ff, E, k, max_rows;
    bool has_br;
    WMat Wr, W1, W2;             // biases of the experts' layers as further rows
    DSh br, s, o, S, Q, g, xe, h, hg, he;
};

static void acct_finished(gt_ctx *c, u64 n, bool relu)
{
    wire_add(c, +1, n, 64); wire_add(c, -1, n, 64);
    for (int v = 1; v <= 4; v++) wire_add(c, -1, n, (relu ? 64u : 32u) >> v);
    if (relu) wire_add(c, -1, n, 1);
    wire_add(c, +1, n, relu ? 2 : 1);
    if (relu) wire_add(c, -1, n, 64);
}
static void acct_finish(gt_ctx *c, u64 n, bool relu) { acct_finished(c, n, relu); c->acc.rounds += relu ? 8 : 6; }

struct FinOut { P6 y{}, gate{}, res{}, bias{}; bool has_res = false, has_gate = false, has_bias = false; };
static dim3 gF(u64 n) { return dim3((unsigned)std::min<u64>((n + GT_FIN_EL - 1) / GT_FIN_EL, 1u << 16)); }
static int do_finish(gt_ctx *c, int src, bool relu, u64 n, u32 ncol, const FinOut &o, P6 S = {}, P6 x = {})
{
    FinArgs a{};
    a.c = kc(c, c->op++); a.Z = c->dacc; a.n = n; a.ncol = ncol; a.f = c->tau; a.S = S; a.x = x;
    a.y = o.y; a.gate = o.gate; a.res = o.res; a.bias = o.bias; a.has_res = o.has_res; a.has_gate = o.has_gate; a.has_bias = o.has_bias;
    if (src == FIN_PARTS && fin_pairs(c->simds, n)) {
        FinSet set{};
        set.f[0] = a; set.na = (u32)((n + GT_FP_EL - 1) / GT_FP_EL);
        GTCHK(relu ? launch(c, GT_KC_FINISH, k_finish_pair<FIN_PARTS, true>, dim3(set.na), B64, set) : launch(c, GT_KC_FINISH, k_finish_pair<FIN_PARTS, false>, dim3(set.na), B64, set));
    } else if (n) GTCHK(src == FIN_SCALE ? launch(c, GT_KC_FINISH, k_finish<FIN_SCALE, false>, gF(n), B64, a)
                 : relu ? launch(c, GT_KC_FINISH, k_finish<FIN_PARTS, true>, gF(n), B64, a)
                 : launch(c, GT_KC_FINISH, k_finish<FIN_PARTS, false>, gF(n), B64, a));
    acct_finish(c, n, relu);
    return GT_OK;
}
// The context's workspace of residues.
static int grow_res(gt_ctx *c, size_t need)
{
    if (c->res_bytes >= need) return GT_OK;
    (void)hipStreamSynchronize(c->stream);
    workspace_drop(c, c->res);
    c->res = nullptr; c->res_bytes = 0;
    if (hipMalloc(&c->res, need) != hipSuccess) { c->res = nullptr; return GT_ENOMEM; }
    c->res_bytes = need;
    return GT_OK;
}
// What a call needs of the context's workspaces: words of parts, bytes of residues.  It is reserved before the call takes operation ids, counts or launches
// anything, so that one that does not get it (GT_ENOMEM) leaves no trace; nothing below grows a workspace by itself.
struct Need {
    u64 words = 0, res = 0;
    void also(const Need &o) { words = std::max(words, o.words); res = std::max(res, o.res); }
};
static int reserve(gt_ctx *c, const Need &n)
{
    GTCHK(workspace_room(c, c->dacc_words >= n.words && c->res_bytes >= n.res));
    GTCHK(grow_dacc(c, n.words));
    return grow_res(c, n.res);
}
static Need job_need(gt_ctx *c, u64 M, u64 N, u64 K)
{
    const RnsPlan p = rns_plan(M, N, K, c->rns_limit);
    Need n;
    n.res = rns_bytes(c->simds, M, N, K, p);
    if (!p.whole) n.words = 3 * std::min(M, p.rows) * N;
    return n;
}
static bool few_ahead(gt_ctx *c, const FewShape &s, u64 steps) { return s.rows == 16 && few_left(c->simds, s.ntile, s.ngrp, steps); }
static Need few_need(gt_ctx *c, u64 M, u64 N, u64 K)
{
    const FewShape s = few_shape(c->simds, M, N, K);
    const u64 steps = (K + 63) / 64;
    Need n;
    n.words = 3 * M * N;
    if (few_ahead(c, s, steps)) n.res = s.ntile * steps * GT_FEW_LEFT;
    return n;
}
// a product with weights by either (do_dense_w)
static bool takes_few(gt_ctx *c, u64 M, u64 N, u64 K, u64 ldx) { return M != 0 && few_rows(c->simds, M, N, K, ldx); }
static Need dense_need(gt_ctx *c, u64 M, u64 N, u64 K, u64 ldx) { return takes_few(c, M, N, K, ldx) ? few_need(c, M, N, K) : job_need(c, M, N, K); }
// a completion of residues, and its workgroups
static u32 fin_residues(gt_ctx *c, FinArgs &f, const unsigned char *R, u64 first, u64 n, u64 plane, u32 nchunk)
{
    f.R = R; f.first = first; f.n = n; f.plane = plane; f.nchunk = nchunk;
    const FinShape s = fin_shape(c->simds, n);
    f.per = s.per; f.nbig = s.nbig;
    return s.waves;
}
// arguments of a factor's conversion, and its workgroups
static ResArgs residues(gt_ctx *c, const MatView &x, unsigned char *out, u64 rows, u64 K, u64 k0, u32 nrb, u32 nkb, bool sums, u32 *blocks)
{
    ResArgs a{};
    a.x = x; a.out = out; a.rows = rows; a.K = K; a.k0 = k0; a.nrb = nrb; a.nkb = nkb; a.mats = sums ? 6 : 3;
    const u64 nfr = (u64)nrb * nkb;
    a.per = residue_range(c->simds, nfr * a.mats);
    *blocks = (u32)((nfr + 3) / 4) * a.mats * ((RNS_N + a.per - 1) / a.per);
    return a;
}
// A product of A (M x K, MAT_ROWS or MAT_COLS) and B (N x K, MAT_COLS or weights) by residues with its completion: what a pass over some rows and all of the long axis needs.
struct RnsJob {
    MatView A, B;
    u64 M, N, K;
    bool relu;
    FinArgs f;
    RmmShape s;
    RnsPlan plan;
    bool asums;
    u32 nchunk, narb, nbrb;
    u64 plane, abytes, bbytes, rbytes;
    unsigned char *at;
    RnsJob() {}
    RnsJob(gt_ctx *c, const MatView &A_, const MatView &B_, u64 M_, u64 N_, u64 K_, bool relu_, const FinOut &o) : A(A_), B(B_), M(M_), N(N_), K(K_), relu(relu_), f{}
    {
        f.ncol = (u32)N; f.f = c->tau;
        f.y = o.y; f.gate = o.gate; f.res = o.res; f.bias = o.bias; f.has_res = o.has_res; f.has_gate = o.has_gate; f.has_bias = o.has_bias;
        plan = rns_plan(M, N, K, c->rns_limit);
        shape(c);
    }
    // the operation id and the messages
    void take(gt_ctx *c) { f.c = kc(c, c->op++); acct_finish(c, M * N, relu); }
    // rows from r0 and columns from c0 (multiples of 128 and 256) on
    RnsJob part(gt_ctx *c, u64 r0, u64 rows, u64 c0, u64 cols) const
    {
        RnsJob j = *this;
        for (int p = 0; p < 3; p++) {
            j.A.c[p] += A.kind == MAT_ROWS ? r0 * A.ld : r0;
            j.B.c[p] += B.kind == MAT_COLS ? c0 : (B.kind == MAT_W ? c0 >> 6 : (c0 >> 4) * B.nst) * (3 * GT_WTILE);
        }
        j.M = rows; j.N = cols;
        if (rows != M || cols != N) j.shape(c);
        return j;
    }
    void shape(gt_ctx *c)
    {
        const RnsSizes z = rns_sizes(c->simds, M, N, K);
        s = z.s; asums = z.asums; narb = z.narb; nbrb = z.nbrb; plane = z.plane; abytes = z.abytes; bbytes = z.bbytes; rbytes = z.rbytes;
        nchunk = (u32)((K + RNS_TERMS - 1) / RNS_TERMS);
    }
    u64 bytes() const { return abytes + bbytes + plan.keep * rbytes; }
    u32 nkb(u32 ch) const { return (u32)((std::min<u64>(K - (u64)ch * RNS_TERMS, RNS_TERMS) + 63) / 64 * 2); }
    ResArgs left(gt_ctx *c, u32 ch, u32 *blocks) const
    { const u64 k0 = (u64)ch * RNS_TERMS; return residues(c, A, at, M, std::min<u64>(K - k0, RNS_TERMS), k0, narb, nkb(ch), asums, blocks); }
    ResArgs right(gt_ctx *c, u32 ch, u32 *blocks) const
    { const u64 k0 = (u64)ch * RNS_TERMS; return residues(c, B, at + abytes, N, std::min<u64>(K - k0, RNS_TERMS), k0, nbrb, nkb(ch), !asums, blocks); }
    RmmArgs product(u32 ch) const
    {
        RmmArgs a{};
        a.A = at; a.B = at + abytes; a.R = at + abytes + bbytes + ch % plan.keep * rbytes; a.amat = (u64)narb * nkb(ch) * 1024; a.bmat = (u64)nbrb * nkb(ch) * 1024;
        a.plane = plane; a.M = (u32)M; a.N = (u32)N; a.narb = narb; a.nbrb = nbrb; a.nstep = nkb(ch); a.ntm = (u32)s.ntm; a.ntn = (u32)s.ntn; a.asums = asums;
        a.total = (u32)(3 * RNS_N * s.ntm * s.ntn);
        return a;
    }
};
static u32 rmm_blocks(const RmmArgs &a) { return (a.total + 7) / 8 * 8; }
static int rmm_launch(gt_ctx *c, u32 wm, const RmmSet &m, u32 blocks)
{
    return wm == 4 ? launch(c, GT_KC_DENSE, k_rns_mm<4, 2>, dim3(blocks), B256, m) : wm == 2 ? launch(c, GT_KC_DENSE, k_rns_mm<2, 2>, dim3(blocks), B256, m)
           : launch(c, GT_KC_DENSE, k_rns_mm<1, 1>, dim3(blocks), B256, m);
}
// rows and columns in blocks, the long axis in chunks of RNS_TERMS (see rns_plan); its workspace is there.  done(r0, rows, whole, R, plane, nchunk) completes the product's
// rows from r0 on: from residues R of all chunks (none of a product without terms, whatever R is), or unless whole from the parts' words.
// left_there: the left factor's residues are, from the product before (of one pass, see RnsJobs).
template <class Done>
static int run_products(gt_ctx *c, const RnsJob &all, Done done, bool left_there = false)
{
    const RnsPlan &plan = all.plan;
    for (u64 r0 = 0; r0 < all.M; r0 += plan.rows) {
        const u64 rows = std::min<u64>(all.M - r0, plan.rows), n = rows * all.N;
        const unsigned char *R = nullptr;
        u64 plane = 0;
        u32 nchunk = 0;
        for (u64 c0 = 0; c0 < all.N; c0 += plan.cols) {
            RnsJob j = all.part(c, r0, rows, c0, std::min<u64>(all.N - c0, plan.cols));
            j.at = c->res;
            for (u32 ch = 0; ch < j.nchunk; ch++) {
                ResSet r{};
                u32 na, nb;
                r.r[0] = j.left(c, ch, &na); r.r[1] = j.right(c, ch, &nb);
                if (left_there) na = 0;
                r.end[0] = na;
                for (int e = 1; e < 6; e++) r.end[e] = na + nb;
                GTCHK(launch(c, GT_KC_DENSE, k_residues, dim3(na + nb), B256, r));
                RmmSet m{};
                m.m[0] = j.product(ch); m.na = rmm_blocks(m.m[0]);
                GTCHK(rmm_launch(c, j.s.wm, m, m.na));
                if (plan.whole || (ch % plan.keep != plan.keep - 1 && ch != j.nchunk - 1)) continue;
                JoinArgs a{};
                a.R = j.at + j.abytes + j.bbytes; a.Z = c->dacc; a.plane = j.plane; a.n = rows * j.N; a.parts = n; a.ld = all.N; a.c0 = c0; a.cols = j.N; a.nchunk = ch % plan.keep + 1;
                GTCHK(launch(c, GT_KC_DENSE, k_join, dim3((unsigned)((a.n + 2047) / 2048), 3), B256, a));
            }
            if (plan.whole) { R = j.at + j.abytes + j.bbytes; plane = j.plane; nchunk = j.nchunk; }
        }
        GTCHK(done(r0, rows, plan.whole, R, plane, nchunk));
    }
    return GT_OK;
}
static int run_taken(gt_ctx *c, const RnsJob &all, bool left_there = false)
{
    return run_products(c, all, [&](u64 r0, u64 rows, bool whole, const unsigned char *R, u64 plane, u32 nchunk) {
        const u64 n = rows * all.N;
        FinSet f{};
        f.f[0] = all.f;
        if (whole) {
            f.na = fin_residues(c, f.f[0], R, r0 * all.N, n, plane, nchunk);
            return all.relu ? launch(c, GT_KC_FINISH, k_finish_pair<FIN_RES, true>, dim3(f.na), B64, f) : launch(c, GT_KC_FINISH, k_finish_pair<FIN_RES, false>, dim3(f.na), B64, f);
        }
        f.f[0].Z = c->dacc; f.f[0].first = r0 * all.N; f.f[0].n = n;
        f.na = (u32)((n + GT_FP_EL - 1) / GT_FP_EL);
        return all.relu ? launch(c, GT_KC_FINISH, k_finish_pair<FIN_PARTS, true>, dim3(f.na), B64, f) : launch(c, GT_KC_FINISH, k_finish_pair<FIN_PARTS, false>, dim3(f.na), B64, f);
    }, left_there);
}
static int run_job(gt_ctx *c, RnsJob j)
{
    j.take(c);
    return run_taken(c, j);
}
// Up to three products that do not wait for each other, without activation: side by side in the same three launches where none fills the chip alone (267 x 22 -> 16:
// 12 launches of a backward pass, 66 us, where the host's calls count, to 9).  Where one has the same left factor as the one before (same_left, the same sizes too), its
// residues are made once.
struct RnsJobs {
    RnsJob j[3];
    bool same_left[3] = { false, false, false };
    int n = 0;
    void add(const RnsJob &x, bool same = false) { j[n] = x; same_left[n++] = same; }
    static bool once(const RnsJob &x) { return x.nchunk == 1 && x.M <= x.plan.rows && x.plan.whole; }
    bool joined(int from) const
    {
        for (int i = from; i < n; i++) if (!once(j[i]) || j[i].s.wm != j[from].s.wm || j[i].s.wm == 4) return false;
        return n - from > 1;
    }
    // end of the jobs that share their launches with `from`: all of the others or none.  (Two of three never would: the last two are of the same sizes.)
    int group(int from) const { return joined(from) ? n : from + 1; }
};
static Need jobs_need(gt_ctx *c, const RnsJobs &all)
{
    Need n;
    for (int from = 0, to; from < all.n; from = to) {
        to = all.group(from);
        Need g;
        if (to - from == 1) g = job_need(c, all.j[from].M, all.j[from].N, all.j[from].K);
        else for (int i = from; i < to; i++) g.res += all.j[i].bytes();
        n.also(g);
    }
    return n;
}
static int run_jobs(gt_ctx *c, RnsJobs all)
{
    for (int i = 0; i < all.n; i++) all.j[i].take(c);
    bool alone = false;                           // the job before had the workspace for itself
    for (int from = 0, to; from < all.n; from = to) {
        to = all.group(from);
        RnsJob *j = all.j;
        if (to - from == 1) {
            GTCHK(run_taken(c, j[from], alone && all.same_left[from] && RnsJobs::once(j[from]) && RnsJobs::once(j[from - 1])));
            alone = true;
            continue;
        }
        alone = false;
        ResSet r{};
        RmmSet m{};
        FinSet f{};
        u32 rblocks = 0, mblocks = 0, fblocks = 0;
        unsigned char *at = c->res;
        for (int i = from; i < to; i++) {
            const int k = i - from;
            const bool shared = k && all.same_left[i];
            j[i].at = at;
            at += j[i].bytes();
            u32 na, nb;
            r.r[2 * k] = j[i].left(c, 0, &na); r.r[2 * k + 1] = j[i].right(c, 0, &nb);
            r.end[2 * k] = rblocks += shared ? 0 : na;
            r.end[2 * k + 1] = rblocks += nb;
            m.m[k] = j[i].product(0);
            if (shared) m.m[k].A = m.m[k - 1].A;
            mblocks += rmm_blocks(m.m[k]);
            f.f[k] = j[i].f;
            fblocks += fin_residues(c, f.f[k], j[i].at + j[i].abytes + j[i].bbytes, 0, j[i].M * j[i].N, j[i].plane, 1);
            if (k == 0) { m.na = mblocks; f.na = fblocks; }
            if (k == 1) { m.nb = mblocks; f.nb = fblocks; }
        }
        for (int k = 2 * (to - from); k < 6; k++) r.end[k] = rblocks;
        GTCHK(launch(c, GT_KC_DENSE, k_residues, dim3(rblocks), B256, r));
        GTCHK(rmm_launch(c, j[from].s.wm, m, mblocks));
        GTCHK(launch(c, GT_KC_FINISH, k_finish_pair<FIN_RES, false>, dim3(fblocks), B64, f));
    }
    return GT_OK;
}
// Parts of the product of few rows x (M rows of K words) and weights, or, transposed, the weights' rows as columns, in the workspace of
// partial inner products; div: a division that may run beside it.
static int few_parts(gt_ctx *c, P6 x, u64 ldx, const WMat &W, bool transposed, u64 M, const DivArgs *div = nullptr)
{
    const u64 N = transposed ? W.K : W.N, K = transposed ? W.N : W.K;
    FewArgs a{};
    for (int j = 0; j < 3; j++) a.x[j] = x.o[j];
    a.w = W.base; a.Z = c->dacc; a.nst = W.nst; a.ldx = ldx; a.M = M; a.N = N; a.K = K;
    const FewShape s = few_shape(c->simds, M, N, K);
    a.per = s.per; a.nsplit = s.nsplit; a.blocks = (u32)(s.ngrp * s.nsplit);
    if (div) a.div = *div;
    const u64 steps = (K + 63) / 64;
    const bool left = few_ahead(c, s, steps);
    if (left) {
        a.left = c->res;
        GTCHK(launch(c, GT_KC_DENSE, k_few_left, dim3((unsigned)steps, (unsigned)s.ntile), dim3(192), a));
    }
    const dim3 g(a.blocks + (div ? gE(div->n).x : 0), (unsigned)s.ntile);
    const auto go = [&](auto LEFT) {
        constexpr bool L = decltype(LEFT)::value;
        return div ? launch(c, GT_KC_DENSE, k_mm_few<16, false, true, L>, g, B256, a) : transposed ? launch(c, GT_KC_DENSE, k_mm_few<16, true, false, L>, g, B256, a)
               : launch(c, GT_KC_DENSE, k_mm_few<16, false, false, L>, g, B256, a);
    };
    if (s.rows == 16) return left ? go(std::integral_constant<bool, true>()) : go(std::integral_constant<bool, false>());
    return div ? launch(c, GT_KC_DENSE, k_mm_few<8, false, true, false>, g, B256, a) : transposed ? launch(c, GT_KC_DENSE, k_mm_few<8, true, false, false>, g, B256, a)
           : launch(c, GT_KC_DENSE, k_mm_few<8, false, false, false>, g, B256, a);
}
// the product of x and weights, completed
static int do_dense_w(gt_ctx *c, P6 x, u64 ldx, const WMat &W, bool transposed, u64 M, bool relu, const FinOut &o)
{
    const u64 N = transposed ? W.K : W.N, K = transposed ? W.N : W.K;
    if (!takes_few(c, M, N, K, ldx)) return run_job(c, RnsJob(c, view(x, ldx, MAT_ROWS), wmat(W, transposed ? MAT_W : MAT_WT), M, N, K, relu, o));
    GTCHK(few_parts(c, x, ldx, W, transposed, M));
    return do_finish(c, FIN_PARTS, relu, M * N, (u32)N, o);
}

static bool dim_ok(u64 n) { return n >= 1 && n <= GT_MAX_DIM; }
static void dense_free(gt_dense *l)
{
    if (l->W.base) (void)hipFree(l->W.base);
    dsh_free(l->b);
    delete l;
}
extern "C" int gt_dense_set(gt_ctx *c, gt_dense *l, const gt_shares *W, const gt_shares *b)
{
    if (!c || !l || !shares_ok(W, (size_t)l->din * l->dout) || l->has_b != (b != nullptr) || (b && !shares_ok(b, l->dout))) return GT_EINVAL;
    Timed T(c);
    int rc = wmat_put(c, l->W, W, 0, l->din);
    if (rc == GT_OK && b) rc = copy6(c, l->b.v, 0, to_p6(b), 0, l->dout);
    return T.finish(rc);
}
extern "C" int gt_dense_create(gt_ctx *c, const gt_shares *W, const gt_shares *b, uint32_t din, uint32_t dout, gt_dense **out)
{
    if (!c || !out || !dim_ok(din) || !dim_ok(dout) || !shares_ok(W, (size_t)din * dout) || (b && !shares_ok(b, dout))) return GT_EINVAL;
    gt_dense *l = new (std::nothrow) gt_dense();
    if (!l) return GT_ENOMEM;
    l->din = din; l->dout = dout; l->has_b = b != nullptr;
    int rc = wmat_alloc(l->W, din, dout, c->stream);
    if (rc == GT_OK && b) rc = dsh_alloc(l->b, dout, c->stream);
    if (rc == GT_OK) rc = gt_dense_set(c, l, W, b);
    if (rc != GT_OK) { dense_free(l); return rc; }
    *out = l;
    return GT_OK;
}
extern "C" int gt_dense_destroy(gt_dense *l)
{
    if (!l) return GT_EINVAL;
    dense_free(l);
    return GT_OK;
}

extern "C" int gt_dense_forward(gt_ctx *c, const gt_dense *l, const gt_shares *x, size_t rows, int act, const gt_shares *res, const gt_shares *y,
                                const gt_shares *gate)
{
    if (!c || !l || rows > GT_MAX_DIM || (act != GT_ACT_NONE && act != GT_ACT_RELU)) return GT_EINVAL;
    const size_t n = rows * l->dout;
    if (!shares_ok(x, rows * l->din) || !shares_ok(y, n) || (res && !shares_ok(res, n)) || (gate && (act != GT_ACT_RELU || !shares_ok(gate, n)))) return GT_EINVAL;
    Timed T(c);
    GTCHK(reserve(c, dense_need(c, rows, l->dout, l->din, l->din)));
    FinOut o;
    o.y = to_p6(y);
    if (res) { o.has_res = true; o.res = to_p6(res); }
    if (gate) { o.has_gate = true; o.gate = to_p6(gate); }
    if (l->has_b) { o.has_bias = true; o.bias = l->b.v; }
    return T.finish(do_dense_w(c, to_p6(x), l->din, l->W, false, rows, act == GT_ACT_RELU, o));
}

static int ws_grow(gt_ctx *c, DSh &w, size_t n)
{
    const bool fits = w.base && w.n >= n;
    GTCHK(workspace_room(c, fits));
    if (fits) return GT_OK;
    (void)hipStreamSynchronize(c->stream);
    workspace_drop(c, w.base);
    w.base = nullptr; w.n = 0;
    return dsh_alloc(w, n, c->stream);
}
extern "C" int gt_dense_backward(gt_ctx *c, const gt_dense *l, const gt_shares *x, const gt_shares *gate, const gt_shares *dy, size_t rows,
                                 const gt_shares *dx, const gt_shares *dW, const gt_shares *db)
{
    if (!c || !l || rows > GT_MAX_DIM) return GT_EINVAL;
    const size_t n = rows * l->dout, nx = rows * l->din, nw = (size_t)l->din * l->dout;
    if (!shares_ok(dy, n) || (gate && !shares_ok(gate, n)) || (dW && !shares_ok(x, nx)) || (dx && !shares_ok(dx, nx)) || (dW && !shares_ok(dW, nw)) ||
        (db && !shares_ok(db, l->dout))) return GT_EINVAL;
    Timed T(c);
    if (gate) GTCHK(ws_grow(c, c->ws_dz, n));
    const P6 dz = gate ? c->ws_dz.v : to_p6(dy);
    FinOut ox, ow;
    if (dx) ox.y = to_p6(dx);
    if (dW) ow.y = to_p6(dW);
    const bool apart = dx && (rows == 0 || !dW || few_rows_apart(rows, l->din, l->dout)), both = dx && !apart;
    RnsJobs jobs;
    Need need;
    if (apart) need = dense_need(c, rows, l->din, l->dout, l->dout);
    if (both) jobs.add(RnsJob(c, view(dz, l->dout, MAT_ROWS), wmat(l->W, MAT_W), rows, l->din, l->dout, false, ox));
    if (dW) jobs.add(RnsJob(c, view(to_p6(x), l->din, MAT_COLS), view(dz, l->dout, MAT_COLS), l->din, l->dout, rows, false, ow));
    need.also(jobs_need(c, jobs));
    GTCHK(reserve(c, need));
    if (gate) {
        MultArgs m{}; m.x = once(to_p6(gate)); m.y = once(to_p6(dy)); m.z = dz; m.n = n;
        m.c = kc(c, c->op++);
        if (n) GTCHK(launch(c, GT_KC_MULT, k_mult, dim3(tiles8(n)), GT_BLOCK, m));
        acct_reshare(c, n, 1);
    }
    if (apart) GTCHK(do_dense_w(c, dz, l->dout, l->W, true, rows, false, ox));
    GTCHK(run_jobs(c, jobs));
    if (db) {
        ColsumArgs a{}; a.x = dz; a.out = to_p6(db); a.rows = rows; a.cols = l->dout; a.ld = l->dout; a.half = ~0u;
        GTCHK(launch(c, GT_KC_LOCAL, k_colsum, dim3((l->dout + 15) / 16, 3), dim3(1024), a));
    }
    return T.finish(GT_OK);
}

static void moe_free(gt_moe *m)
{
    for (WMat *w : { &m->Wr, &m->W1, &m->W2 }) if (w->base) (void)hipFree(w->base);
    DSh *all[] = { &m->br, &m->s, &m->o, &m->S, &m->Q, &m->g, &m->xe, &m->h, &m->hg, &m->he };
    for (DSh *s : all) dsh_free(*s);
    delete m;
}
static int moe_init(gt_ctx *c, gt_moe *m, const gt_shares *Wr, const gt_shares *br, const gt_shares *W1, const gt_shares *b1, const gt_shares *W2,
                    const gt_shares *b2)
{
    const u64 E = m->E, d = m->d, ff = m->ff, rows = m->max_rows, rk = rows * m->k;
    GTCHK(wmat_alloc(m->Wr, d, E, c->stream));
    GTCHK(wmat_alloc(m->W1, E * (d + 1), ff, c->stream));
    GTCHK(wmat_alloc(m->W2, E * (ff + 1), d, c->stream));
    GTCHK(wmat_put(c, m->Wr, Wr, 0, d));
    GTCHK(wmat_put(c, m->W1, W1, 0, E * d));
    GTCHK(wmat_put(c, m->W2, W2, 0, E * ff));
    if (b1) GTCHK(wmat_put(c, m->W1, b1, E * d, E));
    if (b2) GTCHK(wmat_put(c, m->W2, b2, E * ff, E));
    if (br) { GTCHK(dsh_alloc(m->br, E, c->stream)); GTCHK(copy6(c, m->br.v, 0, to_p6(br), 0, E)); }
    GTCHK(dsh_alloc(m->s, rows * E, c->stream)); GTCHK(dsh_alloc(m->o, rk * E, c->stream));
    for (DSh *s : { &m->S, &m->Q, &m->g }) GTCHK(dsh_alloc(*s, rk, c->stream));
    GTCHK(dsh_alloc(m->xe, rk * E * (d + 1), c->stream));
    GTCHK(dsh_alloc(m->h, rk * ff, c->stream)); GTCHK(dsh_alloc(m->hg, rk * ff, c->stream));
    return dsh_alloc(m->he, rows * E * (ff + 1), c->stream);
}
extern "C" int gt_moe_create(gt_ctx *c, const gt_shares *Wr, const gt_shares *br, const gt_shares *W1, const gt_shares *b1, const gt_shares *W2,
                             const gt_shares *b2, uint32_t d, uint32_t ff, uint32_t experts, uint32_t top, uint32_t max_rows, gt_moe **out)
{
    const size_t E = experts, w = (size_t)d * ff;
    if (!c || !out || !dim_ok(d) || !dim_ok(ff) || !dim_ok(max_rows) || E < 1 || E > GT_MAX_EXPERTS || top < 1 || top > E) return GT_EINVAL;
    if (!shares_ok(Wr, E * d) || (br && !shares_ok(br, E)) || !shares_ok(W1, E * w) || (b1 && !shares_ok(b1, E * ff)) || !shares_ok(W2, E * w) ||
        (b2 && !shares_ok(b2, E * d))) return GT_EINVAL;
    gt_moe *m = new (std::nothrow) gt_moe();
    if (!m) return GT_ENOMEM;
    m->d = d; m->ff = ff; m->E = experts; m->k = top; m->max_rows = max_rows; m->has_br = br != nullptr;
    const int rc = moe_init(c, m, Wr, br, W1, b1, W2, b2);
    if (rc != GT_OK) { (void)hipStreamSynchronize(c->stream); moe_free(m); return rc; }
    *out = m;
    return GT_OK;
}
extern "C" int gt_moe_destroy(gt_moe *m)
{
    if (!m) return GT_EINVAL;
    moe_free(m);
    return GT_OK;
}

extern "C" int gt_moe_forward(gt_ctx *c, gt_moe *m, const gt_shares *x, size_t rows, const gt_shares *res, const gt_shares *y)
{
    if (!c || !m || rows > m->max_rows) return GT_EINVAL;
    const u64 E = m->E, d = m->d, ff = m->ff, rk = rows * m->k, P = E * (E - 1) / 2;
    if (!shares_ok(x, rows * d) || !shares_ok(y, rows * d) || (res && !shares_ok(res, rows * d))) return GT_EINVAL;
    Timed T(c);
    const bool few = rk && few_rows(c->simds, rk, ff, E * (d + 1), E * (d + 1)) && few_rows(c->simds, rows, d, E * (ff + 1), E * (ff + 1));     // parts of the products by k_mm_few, else results
    Need need = few ? few_need(c, rows, E, d) : dense_need(c, rows, E, d, d);
    need.also(dense_need(c, rk, ff, E * (d + 1), E * (d + 1)));
    need.also(dense_need(c, rows, d, E * (ff + 1), E * (ff + 1)));
    GTCHK(reserve(c, need));
    MoeArgs a{};
    a.s = m->s.v; a.bias = m->br.v; a.o = m->o.v; a.S = m->S.v; a.Q = m->Q.v; a.g = m->g.v; a.x = to_p6(x); a.xe = m->xe.v; a.hg = m->hg.v; a.he = m->he.v;
    a.rows = rows; a.E = (u32)E; a.k = m->k; a.d = m->d; a.ff = m->ff; a.f = c->tau; a.parts = few; a.has_bias = m->has_br;
    FinOut o;
    o.y = m->s.v;
    if (m->has_br) { o.has_bias = true; o.bias = m->br.v; }
    a.c = kc(c, c->op);
    if (few) { GTCHK(few_parts(c, a.x, d, m->Wr, false, rows)); acct_finish(c, rows * E, true); c->op++; }
    else GTCHK(do_dense_w(c, a.x, d, m->Wr, false, rows, true, o));
    a.Z = c->dacc;
    if (rk) GTCHK(launch(c, GT_KC_SMALL, k_moe_choose, dim3((unsigned)rows), B256, a));
    acct_ge(c, rows * P); acct_b2a(c, rows * P);
    acct_eq(c, rk * E); acct_b2a(c, rk * E);
    acct_reshare(c, rk, 1);
    c->op += 3;
    DivArgs q{}; q.c = kc(c, c->op); q.S = m->S.v; q.Q = m->Q.v; q.quo = m->g.v; q.n = rk; q.nsteps = c->tau + 1;
    c->op += c->tau + 1;
    acct_div(c, rk);
    a.c = kc(c, c->op++);
    if (rk) GTCHK(launch(c, GT_KC_MULT, k_moe_spread, gE(rk * E * d), B64, a));
    acct_reshare(c, rk * E * d, 1);
    if (few) {
        GTCHK(few_parts(c, m->xe.v, E * (d + 1), m->W1, false, rk, &q));
        a.c = kc(c, c->op); a.Z = c->dacc;
        const u64 blocks = rows * ((ff + GT_FIN_EL - 1) / GT_FIN_EL + 1);
        GTCHK(launch(c, GT_KC_FINISH, k_moe_hidden, dim3((unsigned)blocks), B256, a));
        acct_finish(c, rk * ff, true); acct_finish(c, rk * ff, false);
        c->op += 3;
    } else {
        if (rk) GTCHK(few_elements(c, rk) ? launch(c, GT_KC_SMALL, k_div<4>, gE(rk), dim3(4 * GT_LANES), q) : launch(c, GT_KC_SMALL, k_div<1>, gE(rk), B64, q));
        FinOut oh;
        oh.y = m->h.v;
        GTCHK(do_dense_w(c, m->xe.v, E * (d + 1), m->W1, false, rk, true, oh));
        FinOut og;
        og.y = m->hg.v;
        GTCHK(do_finish(c, FIN_SCALE, false, rk * ff, m->ff, og, m->g.v, m->h.v));
        a.c = kc(c, c->op++);
        if (rk) GTCHK(launch(c, GT_KC_MULT, k_moe_gather, gE(rows * E * (ff + 1)), B64, a));
    }
    acct_reshare(c, rows * E * (ff + 1), 1);
    FinOut oy;
    oy.y = to_p6(y);
    if (res) { oy.has_res = true; oy.res = to_p6(res); }
    return T.finish(do_dense_w(c, m->he.v, E * (ff + 1), m->W2, false, rows, false, oy));
}
