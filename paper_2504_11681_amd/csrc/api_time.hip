// C ABI of the operators along time (head norm with rotation, gated delta rule): argument checking.  See include/tfno.h.
#include "../../include/tfno.h"
#include "deltarule.h"
#include "headnorm.h"
#include "views.h"

using namespace tfno;

namespace {

tfno_status head_norm(const tfno_head_norm_desc *d, bool backward, const void *q, const void *k, const float *wq, const float *wk,
                      const float *cos, const float *sin, const int *positions, const void *q_out, const void *k_out, void *dq, void *dk,
                      float *dwq, float *dwk, void *stream)
{
    if (!d) return TFNO_ERR_NULL;
    if ((d->dtype != TFNO_F32 && d->dtype != TFNO_BF16) || d->B < 0 || d->T < 0 || d->Hq < 0 || d->Hk < 0 || (long long)d->Hq + d->Hk < 1 ||
        d->D < 1 || d->D > 512 || d->R < 0 || d->R > d->D || d->R % 2 || d->P < 0 || d->positions_batch < 0 || !(d->eps > 0.0f))
        return TFNO_ERR_SHAPE;
    if ((long double)d->B * d->T * ((long double)d->Hq + d->Hk) >= 2147483647.0L) return TFNO_ERR_SHAPE;
    if (d->R > 0 && !positions && d->P < d->T) return TFNO_ERR_SHAPE;
    const bool empty = d->B == 0 || d->T == 0;
    if (empty && !(backward && (dwq || dwk))) return TFNO_OK;
    if (!empty) {
        if ((d->Hq > 0 && (!q || !q_out || (backward && !dq))) || (d->Hk > 0 && (!k || !k_out || (backward && !dk)))) return TFNO_ERR_NULL;
        if (d->R > 0 && (!cos || !sin)) return TFNO_ERR_NULL;
    }
    const int elem = d->dtype == TFNO_BF16 ? 2 : 4;
    auto heads = [&](const void *p, int H, const tfno_strides &s) { return View{H > 0 && !empty ? p : nullptr, elem, d->B, d->T, H, d->D, strides(s)}; };
    const long long table = (long long)d->P * (d->R / 2);
    const View none = flat(nullptr, 0);
    const View vq = heads(q, d->Hq, d->q), vk = heads(k, d->Hk, d->k), vqo = heads(q_out, d->Hq, d->q_out), vko = heads(k_out, d->Hk, d->k_out);
    const View vwq = flat(wq, d->D), vwk = flat(wk, d->D), vc = flat(cos, table), vs = flat(sin, table);
    const View vp = positions ? View{positions, 4, d->B, 1, 1, d->T, Strides{d->positions_batch, 0, 0}} : none;
    HeadNormArgs a{};
    tfno_status st;
    if (!backward) {
        const View views[] = {vqo, vko, vq, vk, vwq, vwk, vc, vs, vp};
        const std::pair<int, int> in_place[] = {{0, 2}, {1, 3}};
        st = check_views(views, 2, in_place, 2);
    } else {
        const View vdq = heads(dq, d->Hq, d->dq), vdk = heads(dk, d->Hk, d->dk), vdwq = flat(dwq, d->D), vdwk = flat(dwk, d->D);
        const View views[] = {vdq, vdk, vdwq, vdwk, vq, vk, vqo, vko, vwq, vwk, vc, vs, vp};
        const std::pair<int, int> in_place[] = {{0, 4}, {0, 6}, {1, 5}, {1, 7}};
        st = check_views(views, 4, in_place, 4);
        void *ws = nullptr;
        if (st == TFNO_OK && (dwq || dwk)) st = workspace(head_norm_workspace_bytes(d->D), views, 13, &ws);
        a.partial = (float *)ws;
        a.sdq = vdq.s, a.sdk = vdk.s;
    }
    if (st != TFNO_OK) return st;
    a.q = q, a.k = k, a.wq = wq, a.wk = wk, a.cos = cos, a.sin = sin, a.positions = positions, a.positions_batch = d->positions_batch;
    a.sq = vq.s, a.sk = vk.s, a.sq_out = vqo.s, a.sk_out = vko.s;
    a.B = d->B, a.T = d->T, a.Hq = d->Hq, a.Hk = d->Hk, a.D = d->D, a.R = d->R, a.P = d->P, a.eps = d->eps;
    a.bf16 = d->dtype == TFNO_BF16, a.interleaved = d->interleaved != 0;
    if (!backward) {
        a.q_out = (void *)q_out, a.k_out = (void *)k_out;
        return status(head_norm_launch(a, (hipStream_t)stream));
    }
    a.dq_out = q_out, a.dk_out = k_out, a.dq = dq, a.dk = dk, a.dwq = dwq, a.dwk = dwk;
    return status(head_norm_backward_launch(a, (hipStream_t)stream));
}

// Sizes of the rule, its strides, and whether there are kernels for it.
tfno_status rule_sizes(const tfno_delta_rule_desc *d)
{
    if (!d) return TFNO_ERR_NULL;
    if ((d->dtype != TFNO_F32 && d->dtype != TFNO_BF16) || d->B < 0 || d->T < 0 || d->Hk < 1 || d->Hv < 1 || d->Hv % d->Hk || d->Dk < 1 || d->Dv < 1)
        return TFNO_ERR_SHAPE;
    if (d->Dk > 128 || d->Dv > 256) return TFNO_ERR_UNSUPPORTED;
    // workgroups of a launch stay below 2^31: a chunk of 32 tokens of a head, or up to 16 blocks of a head's columns
    if (((long double)d->T + 31) / 32 * d->B * d->Hv >= 134217728.0L || (long double)d->B * d->Hv >= 67108864.0L || d->T > (1 << 30)) return TFNO_ERR_SHAPE;
    return TFNO_OK;
}

// The kernels reach the tokens of a chunk of v, o and their gradients with 32-bit offsets.
bool tokens_near(const DeltaArgs &a, const Strides &s) { return a.T <= 1 || s.token < (1 << 24); }

DeltaArgs rule_args(const tfno_delta_rule_desc *d)
{
    DeltaArgs a{};
    a.sq = strides(d->q), a.sk = strides(d->k), a.sv = strides(d->v), a.so = strides(d->o), a.sg = strides(d->g), a.sbeta = strides(d->beta);
    a.sdo = a.so, a.sdq = strides(d->dq), a.sdk = strides(d->dk), a.sdv = strides(d->dv), a.sdg = strides(d->dg), a.sdbeta = strides(d->dbeta);
    a.B = d->B, a.T = d->T, a.Hk = d->Hk, a.Hv = d->Hv, a.Dk = d->Dk, a.Dv = d->Dv, a.scale = d->scale, a.bf16 = d->dtype == TFNO_BF16;
    if (a.T == 1) a.sv.token = a.so.token = a.sdo.token = a.sdv.token = 0;      // whatever it is, no second token is reached with it
    return a;
}

}  // namespace

extern "C" {

tfno_status tfno_head_norm_rope(const tfno_head_norm_desc *d, const void *q, const void *k, const float *wq, const float *wk, const float *cos,
                                const float *sin, const int *positions, void *q_out, void *k_out, void *stream)
{
    return head_norm(d, false, q, k, wq, wk, cos, sin, positions, q_out, k_out, nullptr, nullptr, nullptr, nullptr, stream);
}

tfno_status tfno_head_norm_rope_backward(const tfno_head_norm_desc *d, const void *q, const void *k, const float *wq, const float *wk,
                                         const float *cos, const float *sin, const int *positions, const void *dq_out, const void *dk_out,
                                         void *dq, void *dk, float *dwq, float *dwk, void *stream)
{
    return head_norm(d, true, q, k, wq, wk, cos, sin, positions, dq_out, dk_out, dq, dk, dwq, dwk, stream);
}

size_t tfno_head_norm_rope_workspace_bytes(int D) { return D >= 1 && D <= 512 ? head_norm_workspace_bytes(D) : 0; }

tfno_status tfno_gated_delta_rule(const tfno_delta_rule_desc *d, const void *q, const void *k, const void *v, const float *g, const float *beta,
                                  const int *lengths, const float *initial, void *o, float *final, void *tape, void *stream)
{
    tfno_status st = rule_sizes(d);
    if (st != TFNO_OK) return st;
    if (d->B == 0 || (d->T == 0 && !final)) return TFNO_OK;
    if (d->T > 0 && (!q || !k || !v || !beta || !o)) return TFNO_ERR_NULL;
    DeltaArgs a = rule_args(d);
    if (!tokens_near(a, a.sv) || !tokens_near(a, a.so)) return TFNO_ERR_UNSUPPORTED;
    if (!delta_launches(a, tape != nullptr)) return TFNO_ERR_SHAPE;
    const int elem = a.bf16 ? 2 : 4;
    const long long states = (long long)a.B * a.Hv * a.Dk * a.Dv;
    const bool t = a.T > 0;
    const View views[] = {
        {t ? o : nullptr, elem, a.B, a.T, a.Hv, a.Dv, a.so}, flat(final, states), flat(t ? tape : nullptr, t ? (long long)delta_tape_bytes(a) : 0, 1),
        {t ? q : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sq}, {t ? k : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sk},
        {t ? v : nullptr, elem, a.B, a.T, a.Hv, a.Dv, a.sv}, {t ? g : nullptr, 4, a.B, a.T, a.Hv, 1, a.sg},
        {t ? beta : nullptr, 4, a.B, a.T, a.Hv, 1, a.sbeta}, flat(initial, states), flat(lengths, a.B)};
    if ((st = check_views(views, 3, nullptr, 0)) != TFNO_OK) return st;
    if (!aligned(tape, 256)) return TFNO_ERR_ALIGN;
    if (!tape && t) {
        void *ws = nullptr;
        if ((st = workspace(delta_workspace_bytes(a, false), views, 10, &ws)) != TFNO_OK) return st;
        a.workspace = (unsigned char *)ws;
    }
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.lengths = lengths, a.initial = initial, a.o = o, a.final_state = final;
    a.tape = (unsigned char *)tape;
    return status(delta_forward_launch(a, (hipStream_t)stream));
}

tfno_status tfno_gated_delta_rule_backward(const tfno_delta_rule_desc *d, const void *q, const void *k, const void *v, const float *g,
                                           const float *beta, const int *lengths, const float *initial, const void *tape, const void *d_o,
                                           const float *d_final, void *dq, void *dk, void *dv, float *dg, float *dbeta, float *d_initial,
                                           void *stream)
{
    tfno_status st = rule_sizes(d);
    if (st != TFNO_OK) return st;
    if (d->B == 0 || (d->T == 0 && !d_initial)) return TFNO_OK;
    if (d->T > 0 && (!q || !k || !v || !beta || !tape || !d_o || !dq || !dk || !dv || !dbeta)) return TFNO_ERR_NULL;
    DeltaArgs a = rule_args(d);
    if (!tokens_near(a, a.sdo) || !tokens_near(a, a.sdv)) return TFNO_ERR_UNSUPPORTED;
    if (!delta_launches(a, true)) return TFNO_ERR_SHAPE;
    const int elem = a.bf16 ? 2 : 4;
    const long long states = (long long)a.B * a.Hv * a.Dk * a.Dv;
    const bool t = a.T > 0;
    const View views[] = {
        {t ? dq : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sdq}, {t ? dk : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sdk},
        {t ? dv : nullptr, elem, a.B, a.T, a.Hv, a.Dv, a.sdv}, {t ? dg : nullptr, 4, a.B, a.T, a.Hv, 1, a.sdg},
        {t ? dbeta : nullptr, 4, a.B, a.T, a.Hv, 1, a.sdbeta}, flat(d_initial, states),
        {t ? q : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sq}, {t ? k : nullptr, elem, a.B, a.T, a.Hk, a.Dk, a.sk},
        {t ? v : nullptr, elem, a.B, a.T, a.Hv, a.Dv, a.sv}, {t ? g : nullptr, 4, a.B, a.T, a.Hv, 1, a.sg},
        {t ? beta : nullptr, 4, a.B, a.T, a.Hv, 1, a.sbeta}, flat(initial, states), flat(lengths, a.B),
        {t ? d_o : nullptr, elem, a.B, a.T, a.Hv, a.Dv, a.so}, flat(d_final, states), flat(t ? tape : nullptr, t ? (long long)delta_tape_bytes(a) : 0, 1)};
    if ((st = check_views(views, 6, nullptr, 0)) != TFNO_OK) return st;
    if (!aligned(tape, 256)) return TFNO_ERR_ALIGN;
    if (t) {
        void *ws = nullptr;
        if ((st = workspace(delta_workspace_bytes(a, true), views, 16, &ws)) != TFNO_OK) return st;
        a.workspace = (unsigned char *)ws;
    }
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.lengths = lengths, a.initial = initial, a.tape = (unsigned char *)tape;
    a.d_o = d_o, a.d_final = d_final, a.dq = dq, a.dk = dk, a.dv = dv, a.dg = dg, a.dbeta = dbeta, a.d_initial = d_initial;
    return status(delta_backward_launch(a, (hipStream_t)stream));
}

size_t tfno_gated_delta_rule_tape_bytes(const tfno_delta_rule_desc *d)
{
    return rule_sizes(d) == TFNO_OK ? delta_tape_bytes(rule_args(d)) : 0;
}

size_t tfno_gated_delta_rule_workspace_bytes(const tfno_delta_rule_desc *d, int backward)
{
    return rule_sizes(d) == TFNO_OK ? delta_workspace_bytes(rule_args(d), backward != 0) : 0;
}

tfno_status tfno_gated_delta_rule_step(const tfno_delta_rule_desc *d, const void *q, const void *k, const void *v, const float *g,
                                       const float *beta, float *states, const int *slots, int pool, void *o, void *stream)
{
    tfno_status st = rule_sizes(d);
    if (st != TFNO_OK) return st;
    if (d->T != 1 || pool < 0 || (!slots && pool < d->B)) return TFNO_ERR_SHAPE;
    if (d->B == 0) return TFNO_OK;
    if (!q || !k || !v || !beta || !o || (!states && pool > 0)) return TFNO_ERR_NULL;
    DeltaStepArgs a{};
    a.sq = strides(d->q), a.sk = strides(d->k), a.sv = strides(d->v), a.so = strides(d->o), a.sg = strides(d->g), a.sbeta = strides(d->beta);
    a.B = d->B, a.Hk = d->Hk, a.Hv = d->Hv, a.Dk = d->Dk, a.Dv = d->Dv, a.pool = pool, a.scale = d->scale, a.bf16 = d->dtype == TFNO_BF16;
    if ((long double)a.B * a.Hv * 64 >= 2147483647.0L) return TFNO_ERR_SHAPE;
    const int elem = a.bf16 ? 2 : 4;
    const View views[] = {
        {o, elem, a.B, 1, a.Hv, a.Dv, a.so}, flat(states, (long long)pool * a.Hv * a.Dk * a.Dv),
        {q, elem, a.B, 1, a.Hk, a.Dk, a.sq}, {k, elem, a.B, 1, a.Hk, a.Dk, a.sk}, {v, elem, a.B, 1, a.Hv, a.Dv, a.sv},
        {g, 4, a.B, 1, a.Hv, 1, a.sg}, {beta, 4, a.B, 1, a.Hv, 1, a.sbeta}, flat(slots, a.B)};
    if ((st = check_views(views, 2, nullptr, 0)) != TFNO_OK) return st;
    a.q = q, a.k = k, a.v = v, a.g = g, a.beta = beta, a.slots = slots, a.state = states, a.o = o;
    return status(delta_step_launch(a, (hipStream_t)stream));
}

}  // extern "C"
