// Host side of the gated layer and of linear attention: argument checks, the operation schedule, message accounting, launches (part of gtree.hip).
#pragma once

// Both projections' weights side by side, ffp columns each (whole blocks of 64, zero behind ff), and their biases bg, bu on end.
struct gt_gated { u32 din, ff, ffp; bool has_b; WMat W; DSh b; };

static int gated_put(gt_ctx *c, gt_gated *l, const gt_shares *Wg, const gt_shares *bg, const gt_shares *Wu, const gt_shares *bu)
{
    GTCHK(wmat_put(c, l->W, Wg, 0, l->din, 0, l->ff));
    GTCHK(wmat_put(c, l->W, Wu, 0, l->din, l->ffp, l->ff));
    if (!l->has_b) return GT_OK;
    Copies cp;
    cp.add(l->b.v, 0, to_p6(bg), 0, l->ff);
    cp.add(l->b.v, l->ff, to_p6(bu), 0, l->ff);
    return cp.run(c);
}
static bool gated_ok(const gt_shares *Wg, const gt_shares *bg, const gt_shares *Wu, const gt_shares *bu, size_t din, size_t ff)
{
    return shares_ok(Wg, din * ff) && shares_ok(Wu, din * ff) && (bg != nullptr) == (bu != nullptr) && (!bg || (shares_ok(bg, ff) && shares_ok(bu, ff)));
}
static void gated_free(gt_gated *l)
{
    if (l->W.base) (void)hipFree(l->W.base);
    dsh_free(l->b);
    delete l;
}
extern "C" int gt_gated_set(gt_ctx *c, gt_gated *l, const gt_shares *Wg, const gt_shares *bg, const gt_shares *Wu, const gt_shares *bu)
{
    if (!c || !l || !gated_ok(Wg, bg, Wu, bu, l->din, l->ff) || l->has_b != (bg != nullptr)) return GT_EINVAL;
    Timed T(c);
    return T.finish(gated_put(c, l, Wg, bg, Wu, bu));
}
extern "C" int gt_gated_create(gt_ctx *c, const gt_shares *Wg, const gt_shares *bg, const gt_shares *Wu, const gt_shares *bu, uint32_t din, uint32_t ff, gt_gated **out)
{
    if (!c || !out || !dim_ok(din) || !dim_ok(ff) || ff > GT_MAX_DIM / 2 || !gated_ok(Wg, bg, Wu, bu, din, ff)) return GT_EINVAL;
    gt_gated *l = new (std::nothrow) gt_gated();
    if (!l) return GT_ENOMEM;
    l->din = din; l->ff = ff; l->ffp = (ff + 63) / 64 * 64; l->has_b = bg != nullptr;
    int rc = wmat_alloc(l->W, din, 2 * (u64)l->ffp, c->stream);
    if (rc == GT_OK && bg) rc = dsh_alloc(l->b, 2 * (size_t)ff, c->stream);
    if (rc == GT_OK) rc = gt_gated_set(c, l, Wg, bg, Wu, bu);
    if (rc != GT_OK) { (void)hipStreamSynchronize(c->stream); gated_free(l); return rc; }
    *out = l;
    return GT_OK;
}
extern "C" int gt_gated_destroy(gt_gated *l)
{
    if (!l) return GT_EINVAL;
    gated_free(l);
    return GT_OK;
}

static int gated_finish(gt_ctx *c, GatedArgs a, bool relu, u64 first, u64 rows, bool whole, const unsigned char *R, u64 plane, u32 nchunk)
{
    a.first = first; a.rows = rows; a.R = R; a.plane = plane; a.nchunk = nchunk; a.Z = c->dacc;
    const u64 n = rows * a.ff8;
    if (!whole && gated_few(c->simds, n)) {
        const dim3 g((unsigned)((n + GT_FIN_EL - 1) / GT_FIN_EL));
        return relu ? launch(c, GT_KC_FINISH, k_gated_few<true>, g, dim3(128), a) : launch(c, GT_KC_FINISH, k_gated_few<false>, g, dim3(128), a);
    }
    if (!whole) {
        const dim3 g((unsigned)((n + GT_FP_EL - 1) / GT_FP_EL));
        return relu ? launch(c, GT_KC_FINISH, k_gated<FIN_PARTS, true>, g, B64, a) : launch(c, GT_KC_FINISH, k_gated<FIN_PARTS, false>, g, B64, a);
    }
    const FinShape s = gated_shape(c->simds, n);
    a.per = s.per; a.nbig = s.nbig;
    return relu ? launch(c, GT_KC_FINISH, k_gated<FIN_RES, true>, dim3(s.waves), B64, a) : launch(c, GT_KC_FINISH, k_gated<FIN_RES, false>, dim3(s.waves), B64, a);
}
extern "C" int gt_gated_forward(gt_ctx *c, const gt_gated *l, const gt_shares *x, size_t rows, int act, const gt_shares *h, const gt_shares *g, const gt_shares *u,
                                const gt_shares *gate)
{
    if (!c || !l || rows > GT_MAX_DIM || (act != GT_ACT_NONE && act != GT_ACT_RELU)) return GT_EINVAL;
    const bool relu = act == GT_ACT_RELU, keep = g != nullptr;
    const size_t n = rows * l->ff;
    if (!shares_ok(x, rows * l->din) || !shares_ok(h, n) || keep != (u != nullptr) || (keep && relu) != (gate != nullptr)) return GT_EINVAL;
    if (keep && (!shares_ok(g, n) || !shares_ok(u, n) || (gate && !shares_ok(gate, n)))) return GT_EINVAL;
    Timed T(c);
    const u64 N = 2 * (u64)l->ffp;
    GTCHK(reserve(c, dense_need(c, rows, N, l->din, l->din)));
    GatedArgs a{};
    a.c = kc(c, c->op); c->op += 3;
    a.ff = l->ff; a.ff8 = (l->ff + 7) / 8 * 8; a.ffp = l->ffp; a.f = c->tau;
    a.h = to_p6(h); a.keep = keep;
    if (keep) { a.g = to_p6(g); a.u = to_p6(u); }
    if (gate) a.s = to_p6(gate);
    if (l->has_b) { a.has_bias = 1; a.bias = l->b.v; }
    acct_finished(c, n, relu); acct_finished(c, n, false); acct_finished(c, n, false);
    c->acc.rounds += relu ? 14 : 12;
    if (!rows) return T.finish(GT_OK);
    if (takes_few(c, rows, N, l->din, l->din)) {
        GTCHK(few_parts(c, to_p6(x), l->din, l->W, false, rows));
        return T.finish(gated_finish(c, a, relu, 0, rows, false, nullptr, 0, 0));
    }
    const RnsJob j(c, view(to_p6(x), l->din, MAT_ROWS), wmat(l->W, MAT_WT), rows, N, l->din, false, FinOut());
    return T.finish(run_products(c, j, [&](u64 r0, u64 nr, bool whole, const unsigned char *R, u64 plane, u32 nchunk) { return gated_finish(c, a, relu, r0, nr, whole, R, plane, nchunk); }));
}

extern "C" int gt_gated_backward(gt_ctx *c, const gt_gated *l, const gt_shares *x, const gt_shares *g, const gt_shares *u, const gt_shares *gate, const gt_shares *dh,
                                 size_t rows, const gt_shares *dx, const gt_shares *dWg, const gt_shares *dWu, const gt_shares *dbg, const gt_shares *dbu)
{
    if (!c || !l || rows > GT_MAX_DIM || (dWg != nullptr) != (dWu != nullptr) || (dbg != nullptr) != (dbu != nullptr)) return GT_EINVAL;
    const size_t n = rows * l->ff, nx = rows * l->din, nw = (size_t)l->din * l->ff;
    if (!shares_ok(g, n) || !shares_ok(u, n) || !shares_ok(dh, n) || (gate && !shares_ok(gate, n)) || (dx && !shares_ok(dx, nx)) ||
        (dWg && (!shares_ok(x, nx) || !shares_ok(dWg, nw) || !shares_ok(dWu, nw))) || (dbg && (!shares_ok(dbg, l->ff) || !shares_ok(dbu, l->ff)))) return GT_EINVAL;
    Timed T(c);
    const u64 N = 2 * (u64)l->ffp;
    GTCHK(ws_grow(c, c->ws_dz, rows * N));
    const P6 dz = c->ws_dz.v;
    P6 half[2] = { dz, dz };
    for (int p = 0; p < 3; p++) half[1].o[p] += l->ffp;
    FinOut ox, og, ou;
    if (dx) ox.y = to_p6(dx);
    // dx joins the others' launches unless the conversion of its weights is much
    const bool apart = dx && (rows == 0 || !dWg || gated_apart(rows, l->din, N));
    RnsJobs jobs;
    Need need;
    if (apart) need = dense_need(c, rows, l->din, N, N);
    else if (dx) jobs.add(RnsJob(c, view(dz, N, MAT_ROWS), wmat(l->W, MAT_W), rows, l->din, N, false, ox));
    if (dWg) {
        og.y = to_p6(dWg); ou.y = to_p6(dWu);
        const MatView xt = view(to_p6(x), l->din, MAT_COLS);
        jobs.add(RnsJob(c, xt, view(half[0], N, MAT_COLS), l->din, l->ff, rows, false, og));
        jobs.add(RnsJob(c, xt, view(half[1], N, MAT_COLS), l->din, l->ff, rows, false, ou), true);
    }
    need.also(jobs_need(c, jobs));
    GTCHK(reserve(c, need));
    GatedBackArgs a{};
    a.c = kc(c, c->op); c->op += 2;
    a.dh = once(to_p6(dh)); a.g = once(to_p6(g)); a.u = once(to_p6(u));
    if (gate) a.s = once(to_p6(gate));
    for (int p = 0; p < 3; p++) a.dz[p] = dz.o[p];
    a.rows = rows; a.ff = l->ff; a.ff8 = (l->ff + 7) / 8 * 8; a.ffp = l->ffp; a.f = c->tau;
    const u64 elements = rows * a.ff8;
    const dim3 few((unsigned)((elements + GT_FIN_EL - 1) / GT_FIN_EL));
    if (rows && gated_few(c->simds, elements)) GTCHK(gate ? launch(c, GT_KC_FINISH, k_gated_back_few<true>, few, dim3(128), a) : launch(c, GT_KC_FINISH, k_gated_back_few<false>, few, dim3(128), a));
    else for (; a.first < elements; a.first += (u64)GT_FP_EL << 24) {
        const dim3 grid((unsigned)std::min<u64>((elements - a.first + GT_FP_EL - 1) / GT_FP_EL, 1u << 24));
        GTCHK(gate ? launch(c, GT_KC_FINISH, k_gated_back<true>, grid, B64, a) : launch(c, GT_KC_FINISH, k_gated_back<false>, grid, B64, a));
    }
    acct_finished(c, n, false); acct_finished(c, n, false);
    if (gate) wire_add(c, -1, n, 64);
    c->acc.rounds += gate ? 7 : 6;
    if (apart) GTCHK(do_dense_w(c, dz, N, l->W, true, rows, false, ox));
    GTCHK(run_jobs(c, jobs));
    if (dbg) {
        ColsumArgs s{}; s.x = dz; s.out = to_p6(dbg); s.out2 = to_p6(dbu); s.rows = rows; s.ld = N; s.apart = l->ffp; s.cols = l->ff; s.half = (l->ff + 15) / 16;
        GTCHK(launch(c, GT_KC_LOCAL, k_colsum, dim3(2 * s.half, 3), dim3(1024), s));
    }
    return T.finish(GT_OK);
}

// ---- linear attention --------------------------------------------------------------------
struct gt_linattn { u32 heads, dk, dv; u32 *D; };

extern "C" int gt_linattn_create(gt_ctx *c, const uint32_t *decay, uint32_t heads, uint32_t dk, uint32_t dv, gt_linattn **out)
{
    if (!c || !out || !decay || heads < 1 || heads > GT_MAX_HEADS || dk < 1 || dk > GT_MAX_HEAD_DIM || dv < 1 || dv > GT_MAX_HEAD_DIM) return GT_EINVAL;
    DecayArgs a{};
    for (u32 h = 0; h < heads; h++) {
        if (decay[h] > 1u << GT_LIN_DECAY) return GT_EINVAL;
        a.w[h] = decay[h];
    }
    gt_linattn *l = new (std::nothrow) gt_linattn();
    if (!l) return GT_ENOMEM;
    l->heads = heads; l->dk = dk; l->dv = dv;
    if (hipMalloc(&l->D, (size_t)heads * (GT_LIN_CHUNK + 1) * 4) != hipSuccess) { delete l; return GT_ENOMEM; }
    a.D = l->D; a.heads = heads;
    const int rc = launch(c, GT_KC_LOCAL, k_lin_decays, dim3(1), dim3(GT_MAX_HEADS), a);
    if (rc != GT_OK) { (void)hipFree(l->D); delete l; return rc; }
    *out = l;
    return GT_OK;
}
extern "C" int gt_linattn_destroy(gt_linattn *l)
{
    if (!l) return GT_EINVAL;
    (void)hipFree(l->D);
    delete l;
    return GT_OK;
}

// whether two sharings of n words have memory in common
static bool shares_meet(const gt_shares *a, const gt_shares *b, size_t n)
{
    const u64 *x[6], *y[6];
    for (int p = 0; p < 3; p++) { x[2 * p] = a->party[p].own; x[2 * p + 1] = a->party[p].next; y[2 * p] = b->party[p].own; y[2 * p + 1] = b->party[p].next; }
    for (int i = 0; i < 36; i++) if (x[i / 6] < y[i % 6] + n && y[i % 6] < x[i / 6] + n) return true;
    return false;
}
extern "C" int gt_linattn_forward(gt_ctx *c, const gt_linattn *l, const gt_shares *q, const gt_shares *k, const gt_shares *v, size_t ld, size_t seqs, size_t tokens,
                                  const gt_shares *in, const gt_shares *out, const gt_shares *o)
{
    if (!c || !l || seqs > GT_MAX_DIM || tokens > GT_MAX_DIM || seqs * tokens > GT_MAX_DIM || seqs * l->heads > GT_MAX_DIM) return GT_EINVAL;
    const size_t rows = seqs * tokens, wk = (size_t)l->heads * l->dk, wv = (size_t)l->heads * l->dv, dkv = (size_t)l->dk * l->dv, nS = seqs * l->heads * dkv;
    if (ld && (ld < wk || ld < wv || ld > 4 * (size_t)GT_MAX_DIM)) return GT_EINVAL;
    const size_t ldk = ld ? ld : wk, ldv = ld ? ld : wv;
    const size_t nk = rows ? (rows - 1) * ldk + wk : 0, nv = rows ? (rows - 1) * ldv + wv : 0;
    if (!shares_ok(q, nk) || !shares_ok(k, nk) || !shares_ok(v, nv) || (in && !shares_ok(in, nS)) || !shares_ok(out, nS) || !shares_ok(o, rows * wv)) return GT_EINVAL;
    Timed T(c);
    if (!rows) {                                  // the states stay as they are
        if (nS && in && !shares_meet(in, out, nS)) GTCHK(copy6(c, to_p6(out), 0, to_p6(in), 0, nS));
        if (nS && !in) for (int p = 0; p < 3; p++) {
            GTCHK(launch(c, GT_KC_LOCAL, k_fill_words, g1(nS), B256, out->party[p].own, (u64)nS, (u64)0));
            GTCHK(launch(c, GT_KC_LOCAL, k_fill_words, g1(nS), B256, out->party[p].next, (u64)nS, (u64)0));
        }
        c->op += 3;
        return T.finish(GT_OK);
    }
    LinArgs a{};
    for (int p = 0; p < 3; p++) { a.q[p] = q->party[p].own; a.k[p] = k->party[p].own; a.v[p] = v->party[p].own; }
    a.out = to_p6(out); a.o = to_p6(o);
    a.D = l->D; a.ldq = a.ldk = ldk; a.ldv = ldv; a.T = tokens; a.H = l->heads; a.dk = l->dk; a.dv = l->dv; a.dv8 = (l->dv + 7) / 8 * 8;
    a.pk = (u32)((dkv + 7) / 8 * 8); a.f = c->tau; a.nc = (tokens + GT_LIN_CHUNK - 1) / GT_LIN_CHUNK;
    const u64 nbh = seqs * l->heads;
    if (tokens == 1) {
        const u64 nout = nbh * ((a.dv8 + GT_FP_EL - 1) / GT_FP_EL), tiles = nbh * ((dkv + GT_FP_EL - 1) / GT_FP_EL);
        a.c = kc(c, c->op); c->op += 3;
        a.nbh = (u32)nbh; a.per = tiles_of_wave(c->simds, tiles);
        a.has_in = in != nullptr;
        if (in) a.in = to_p6(in);
        acct_finished(c, nbh, false); acct_finished(c, nS, false); acct_finished(c, wv * seqs, false);
        c->acc.rounds += 12;
        const u32 nstate = (u32)((tiles + GT_LIN_TOKEN * a.per - 1) / (GT_LIN_TOKEN * a.per));
        if (in && shares_meet(in, out, nS)) {
            GTCHK(launch(c, GT_KC_FINISH, k_lin_token, dim3((unsigned)nout), dim3(64 * GT_LIN_TOKEN), a, (u32)nout));
            return T.finish(launch(c, GT_KC_FINISH, k_lin_token, dim3(nstate), dim3(64 * GT_LIN_TOKEN), a, 0u));
        }
        return T.finish(launch(c, GT_KC_FINISH, k_lin_token, dim3((unsigned)nout + nstate), dim3(64 * GT_LIN_TOKEN), a, (u32)nout));
    }
    const u64 sizes[5] = { GT_LIN_TRI, a.pk, (u64)GT_LIN_CHUNK * a.dv8, GT_LIN_TRI, a.pk };
    const LinPass pass = lin_pass(nbh, a.nc, l->dk, l->dv, c->rns_limit);
    Need need;
    for (u64 w : sizes) need.res += 24 * w * pass.nbh * pass.nch;
    GTCHK(reserve(c, need));
    a.c = kc(c, c->op); c->op += 3;
    const u64 full = tokens / GT_LIN_CHUNK, rest = tokens % GT_LIN_CHUNK;
    acct_finished(c, nbh * (full * GT_LIN_TRI + rest * (rest + 1) / 2), false);
    for (u64 ch = 0; ch < a.nc; ch++) acct_finished(c, nS, false);
    acct_finished(c, rows * wv, false);
    c->acc.rounds += 6 * std::max<u64>(2, a.nc);
    const u32 per_o = (GT_LIN_CHUNK * a.dv8 + GT_FP_EL - 1) / GT_FP_EL, ct = (l->dv + 63) / 64;
    for (u64 bh0 = 0; bh0 < nbh; bh0 += pass.nbh)
        for (u64 ch0 = 0; ch0 < a.nc; ch0 += pass.nch) {
            a.bh0 = bh0; a.nbh = (u32)std::min<u64>(pass.nbh, nbh - bh0); a.ch0 = (u32)ch0; a.nch = (u32)std::min<u64>(pass.nch, a.nc - ch0);
            const u32 nb = a.nbh * a.nch, last = ch0 + a.nch == a.nc && rest ? (u32)rest : GT_LIN_CHUNK;
            u64 *at = (u64 *)c->res, **to[5] = { &a.Zs, &a.Zk, &a.Zo, &a.P, &a.S };
            for (int i = 0; i < 5; i++) { *to[i] = at; at += 3 * sizes[i] * nb; }
            const gt_shares *from = ch0 ? out : in;
            a.has_in = from != nullptr;
            if (from) a.in = to_p6(from);
            GTCHK(launch(c, GT_KC_DENSE, k_lin_parts, dim3((nb * 3 * (2 + (l->dk + 31) / 32 * ct) + 7) / 8 * 8), B256, a));
            a.tiles = a.nbh * (u32)((dkv + GT_FP_EL - 1) / GT_FP_EL);
            a.each = (a.nch - 1) * (GT_LIN_TRI / GT_FP_EL) + (last * (last + 1) / 2 + GT_FP_EL - 1) / GT_FP_EL;
            a.per = tiles_of_wave(c->simds, (u64)a.nbh * a.each);
            const u32 waves = (a.nbh * a.each + a.per - 1) / a.per;
            GTCHK(lin_pairs(c->simds, a.tiles) ? launch(c, GT_KC_FINISH, k_lin_states<true>, dim3(a.tiles + (waves + 1) / 2), dim3(128), a)
                  : launch(c, GT_KC_FINISH, k_lin_states<false>, dim3(a.tiles + waves), B64, a));
            GTCHK(launch(c, GT_KC_DENSE, k_lin_out, dim3((nb * 6 * ct + 7) / 8 * 8), B256, a));
            a.each = (a.nch - 1) * per_o + (last * a.dv8 + GT_FP_EL - 1) / GT_FP_EL;
            a.per = tiles_of_wave(c->simds, (u64)a.nbh * a.each);
            GTCHK(launch(c, GT_KC_FINISH, k_lin_finish, dim3((a.nbh * a.each + a.per - 1) / a.per), B64, a));
        }
    return T.finish(GT_OK);
}
