// C ABI of the operators of a block along time (gated recurrence, norms around a block, clipping of gradients): argument checking.  See include/tfno.h.
#include "../../include/tfno.h"
#include "blocknorm.h"
#include "gradclip.h"
#include "recurrence.h"
#include "views.h"

#include <cmath>
#include <vector>

using namespace tfno;

namespace {

bool type_ok(int dtype) { return dtype == TFNO_F32 || dtype == TFNO_BF16; }

// A tensor [B, T, C] of the call.
View tokens(const void *p, int elem, int B, int T, int C, const tfno_strides &s) { return View{B > 0 && T > 0 ? p : nullptr, elem, B, T, 1, C, Strides{s.batch, s.token, 0}}; }

tfno_status recurrence_sizes(const tfno_gated_recurrence_desc *d)
{
    if (!d) return TFNO_ERR_NULL;
    if (!type_ok(d->dtype) || d->B < 0 || d->T < 0 || d->C < 1 || d->T > (1 << 30)) return TFNO_ERR_SHAPE;
    if ((long double)d->B * std::max(1.0L, ((long double)d->T + 7) / 8) * d->C >= 1099511627776.0L || d->C > (1 << 28)) return TFNO_ERR_SHAPE;
    if ((long double)d->B * ((d->C + 31) / 32) >= 2147483648.0L) return TFNO_ERR_SHAPE;       // workgroups
    return TFNO_OK;
}

// The kernels reach the tokens of a wave with 32-bit offsets.
bool tokens_near(int T, std::initializer_list<const tfno_strides *> of)
{
    for (const tfno_strides *s : of)
        if (T > 1 && s->token >= (1 << 24)) return false;
    return true;
}

RecurrenceArgs recurrence_args(const tfno_gated_recurrence_desc *d, const void *x, const void *gate, const void *input_gate, const float *rate)
{
    RecurrenceArgs a{};
    a.x = x, a.gate = gate, a.input_gate = input_gate, a.rate = rate;
    a.sx = strides(d->x), a.sgate = strides(d->gate), a.sinput = strides(d->input_gate), a.sy = strides(d->y);
    a.sdx = strides(d->dx), a.sdgate = strides(d->dgate), a.sdinput = strides(d->dinput_gate);
    a.B = d->B, a.T = d->T, a.C = d->C, a.bf16 = d->dtype == TFNO_BF16, a.normalise = d->normalise != 0;
    return a;
}

tfno_status block_norm_sizes(const tfno_block_norm_desc *d)
{
    if (!d) return TFNO_ERR_NULL;
    if (!type_ok(d->dtype) || !type_ok(d->residual_dtype) || (d->dtype == TFNO_F32 && d->residual_dtype != TFNO_F32) || d->B < 0 || d->T < 0 || d->C < 1 ||
        d->gate_kind < TFNO_GATE_NONE || d->gate_kind > TFNO_GATE_CHANNEL || d->activation < TFNO_ACTIVATION_NONE || d->activation > TFNO_ACTIVATION_SIGMOID ||
        !(d->eps > 0.0f) || !std::isfinite(d->residual_scale) || (long double)d->B * d->T >= 2147483647.0L)
        return TFNO_ERR_SHAPE;
    return d->C > 8192 ? TFNO_ERR_UNSUPPORTED : TFNO_OK;
}

}  // namespace

extern "C" {

tfno_status tfno_gated_recurrence(const tfno_gated_recurrence_desc *d, const void *x, const void *gate, const void *input_gate, const float *rate,
                                  const int *lengths, const float *initial, void *y, float *final, void *tape, void *stream)
{
    tfno_status st = recurrence_sizes(d);
    if (st != TFNO_OK) return st;
    if (d->B == 0 || (d->T == 0 && !final)) return TFNO_OK;
    if (d->T > 0 && (!x || !gate || !y)) return TFNO_ERR_NULL;
    if (!tokens_near(d->T, {&d->x, &d->gate, &d->y}) || (input_gate && !tokens_near(d->T, {&d->input_gate}))) return TFNO_ERR_UNSUPPORTED;
    RecurrenceArgs a = recurrence_args(d, x, gate, input_gate, rate);
    const int elem = a.bf16 ? 2 : 4;
    const long long states = (long long)a.B * a.C;
    const View views[] = {tokens(y, elem, a.B, a.T, a.C, d->y), flat(final, states), flat(a.T > 0 ? tape : nullptr, (long long)recurrence_tape_bytes(a.B, a.T, a.C, a.bf16), 1),
                          tokens(x, elem, a.B, a.T, a.C, d->x), tokens(gate, elem, a.B, a.T, a.C, d->gate),
                          tokens(input_gate, elem, a.B, a.T, a.C, d->input_gate), flat(rate, a.C), flat(initial, states), flat(lengths, a.B)};
    if ((st = check_views(views, 3, nullptr, 0)) != TFNO_OK) return st;
    if (!aligned(tape, 256)) return TFNO_ERR_ALIGN;
    if (const size_t need = recurrence_workspace_bytes(a.B, a.T, a.C, a.bf16, false)) {
        void *ws = nullptr;
        if ((st = workspace(need, views, 9, &ws)) != TFNO_OK) return st;
        a.effects = (float *)ws;
    }
    a.lengths = lengths, a.initial = initial, a.y = y, a.final_state = final, a.tape = (float *)tape;
    return status(recurrence_launch(a, (hipStream_t)stream));
}

tfno_status tfno_gated_recurrence_backward(const tfno_gated_recurrence_desc *d, const void *x, const void *gate, const void *input_gate,
                                           const float *rate, const int *lengths, const void *tape, const void *d_y, const float *d_final,
                                           void *dx, void *dgate, void *dinput_gate, float *drate, float *d_initial, void *stream)
{
    tfno_status st = recurrence_sizes(d);
    if (st != TFNO_OK) return st;
    const bool empty = d->B == 0 || d->T == 0;
    if (empty && !drate && (d->B == 0 || !d_initial)) return TFNO_OK;
    if (!empty && (!x || !gate || !tape || !d_y || !dx || !dgate || (!input_gate) != (!dinput_gate) || (drate && !rate))) return TFNO_ERR_NULL;
    if (!tokens_near(d->T, {&d->x, &d->gate, &d->y, &d->dx, &d->dgate}) || (input_gate && !tokens_near(d->T, {&d->input_gate, &d->dinput_gate})))
        return TFNO_ERR_UNSUPPORTED;
    RecurrenceArgs a = recurrence_args(d, x, gate, input_gate, rate);
    const int elem = a.bf16 ? 2 : 4;
    const long long states = (long long)a.B * a.C;
    const View views[] = {tokens(dx, elem, a.B, a.T, a.C, d->dx), tokens(dgate, elem, a.B, a.T, a.C, d->dgate),
                          tokens(dinput_gate, elem, a.B, a.T, a.C, d->dinput_gate), flat(drate, a.C), flat(a.B > 0 ? d_initial : nullptr, states),
                          tokens(x, elem, a.B, a.T, a.C, d->x), tokens(gate, elem, a.B, a.T, a.C, d->gate),
                          tokens(input_gate, elem, a.B, a.T, a.C, d->input_gate), tokens(d_y, elem, a.B, a.T, a.C, d->y), flat(rate, a.C),
                          flat(a.B > 0 ? d_final : nullptr, states), flat(a.B > 0 ? lengths : nullptr, a.B),
                          flat(empty ? nullptr : tape, (long long)recurrence_tape_bytes(a.B, a.T, a.C, a.bf16), 1)};
    if ((st = check_views(views, 5, nullptr, 0)) != TFNO_OK) return st;
    if (!aligned(tape, 256)) return TFNO_ERR_ALIGN;
    if (const size_t need = recurrence_workspace_bytes(a.B, a.T, a.C, a.bf16, true)) {
        void *ws = nullptr;
        if ((st = workspace(need, views, 13, &ws)) != TFNO_OK) return st;
        a.effects = (float *)ws;
    }
    a.lengths = lengths, a.tape = (float *)tape, a.dy = d_y, a.d_final = d_final;
    a.dx = dx, a.dgate = dgate, a.dinput_gate = dinput_gate, a.drate = drate, a.d_initial = d_initial;
    return status(recurrence_backward_launch(a, (hipStream_t)stream));
}

size_t tfno_gated_recurrence_tape_bytes(const tfno_gated_recurrence_desc *d)
{
    return recurrence_sizes(d) == TFNO_OK ? recurrence_tape_bytes(d->B, d->T, d->C, d->dtype == TFNO_BF16) : 0;
}

size_t tfno_gated_recurrence_workspace_bytes(const tfno_gated_recurrence_desc *d, int backward)
{
    return recurrence_sizes(d) == TFNO_OK ? recurrence_workspace_bytes(d->B, d->T, d->C, d->dtype == TFNO_BF16, backward != 0) : 0;
}

tfno_status tfno_gated_recurrence_step(const tfno_gated_recurrence_desc *d, const void *x, const void *gate, const void *input_gate,
                                       const float *rate, float *states, const int *slots, int pool, void *y, void *stream)
{
    tfno_status st = recurrence_sizes(d);
    if (st != TFNO_OK) return st;
    if (d->T != 1 || pool < 0 || (!slots && pool < d->B)) return TFNO_ERR_SHAPE;
    if (d->B == 0) return TFNO_OK;
    if (!x || !gate || !y || (!states && pool > 0)) return TFNO_ERR_NULL;
    RecurrenceArgs a = recurrence_args(d, x, gate, input_gate, rate);
    a.sx.token = a.sgate.token = a.sinput.token = a.sy.token = 0;
    const int elem = a.bf16 ? 2 : 4;
    const auto one = [&](const void *p, const tfno_strides &s) { return tokens(p, elem, a.B, 1, a.C, tfno_strides{s.batch, 0, 0}); };
    const View views[] = {one(y, d->y), flat(states, (long long)pool * a.C), one(x, d->x), one(gate, d->gate), one(input_gate, d->input_gate), flat(rate, a.C), flat(slots, a.B)};
    if ((st = check_views(views, 2, nullptr, 0)) != TFNO_OK) return st;
    a.states = states, a.slots = slots, a.pool = pool, a.y = y;
    return status(recurrence_step_launch(a, (hipStream_t)stream));
}

static tfno_status block_norm(const tfno_block_norm_desc *d, bool backward, const void *y, const void *r, const void *gate, const float *w_after,
                              const float *w_before, const int *lengths, const void *r_out, const void *n_out, void *dy, void *dr, void *dgate,
                              float *dw_after, float *dw_before, void *stream)
{
    tfno_status st = block_norm_sizes(d);
    if (st != TFNO_OK) return st;
    const bool empty = d->B == 0 || d->T == 0, shared = d->gate_kind == TFNO_GATE_SEQUENCE || d->gate_kind == TFNO_GATE_CHANNEL;
    if (empty && !(backward && (dw_after || dw_before || (shared && dgate)))) return TFNO_OK;
    if (!empty && (!y || (!r_out && !n_out) || (backward && !dy))) return TFNO_ERR_NULL;
    if (!empty && (d->gate_kind != TFNO_GATE_NONE && !gate)) return TFNO_ERR_NULL;
    if (!empty && backward && ((dr && !r) || (dgate && d->gate_kind == TFNO_GATE_NONE))) return TFNO_ERR_NULL;
    if (dw_after && !d->norm_after) return TFNO_ERR_SHAPE;
    const int elem = d->dtype == TFNO_BF16 ? 2 : 4, res = d->residual_dtype == TFNO_BF16 ? 2 : 4;
    const int B = d->B, T = d->T, C = d->C;
    const auto of_gate = [&](const void *p, const tfno_strides &s) {
        if (d->gate_kind == TFNO_GATE_TOKEN) return tokens(p, elem, B, T, C, s);
        if (d->gate_kind == TFNO_GATE_SEQUENCE) return View{B > 0 ? p : nullptr, 4, B, 1, 1, C, Strides{s.batch, 0, 0}};
        return flat(d->gate_kind == TFNO_GATE_CHANNEL ? p : nullptr, C);
    };
    const View vy = tokens(y, elem, B, T, C, d->y), vr = tokens(r, res, B, T, C, d->r), vg = of_gate(gate, d->gate);
    const View vro = tokens(r_out, res, B, T, C, d->r_out), vno = tokens(n_out, elem, B, T, C, d->n_out);
    const View va = flat(w_after, C), vb = flat(w_before, C), vl = flat(B > 0 ? lengths : nullptr, B);
    BlockNormArgs a{};
    if (!backward) {
        const View views[] = {vro, vno, vy, vr, vg, va, vb, vl};
        const std::pair<int, int> in_place[] = {{0, 3}, {1, 2}};
        if ((st = check_views(views, 2, in_place, 2)) != TFNO_OK) return st;
    } else {
        const View vdy = tokens(dy, elem, B, T, C, d->dy), vdr = tokens(dr, res, B, T, C, d->dr), vdg = of_gate(dgate, d->dgate);
        const View views[] = {vdy, vdr, vdg, flat(dw_after, C), flat(dw_before, C), vy, vr, vg, va, vb, vl, vro, vno};
        const std::pair<int, int> in_place[] = {{0, 12}, {1, 11}};
        if ((st = check_views(views, 5, in_place, 2)) != TFNO_OK) return st;
        if (d->gate_kind == TFNO_GATE_SEQUENCE && dgate && B > 1 && d->dgate.batch != C) return TFNO_ERR_SHAPE;
        if (dw_after || dw_before || (shared && dgate)) {
            void *ws = nullptr;
            if ((st = workspace(block_norm_workspace_bytes(B, T, C, d->gate_kind), views, 13, &ws)) != TFNO_OK) return st;
            a.workspace = (float *)ws;
        }
        a.sdy = vdy.s, a.sdr = vdr.s, a.sdgate = Strides{C, 0, 0};
        if (d->gate_kind == TFNO_GATE_TOKEN) a.sdgate = vdg.s;
    }
    a.y = y, a.r = r, a.gate = gate, a.w_after = w_after, a.w_before = w_before, a.lengths = lengths;
    a.sy = vy.s, a.sr = vr.s, a.sgate = vg.s, a.sr_out = vro.s, a.sn_out = vno.s;
    a.B = B, a.T = T, a.C = C, a.gate_kind = d->gate_kind, a.activation = d->activation, a.residual_scale = d->residual_scale, a.eps = d->eps;
    a.bf16 = d->dtype == TFNO_BF16, a.residual_bf16 = d->residual_dtype == TFNO_BF16, a.norm_after = d->norm_after != 0;
    if (!backward) {
        a.r_out = (void *)r_out, a.n_out = (void *)n_out;
        return status(block_norm_launch(a, (hipStream_t)stream));
    }
    a.d_r_out = r_out, a.d_n_out = n_out, a.dy = dy, a.dr = dr, a.dgate = dgate, a.dw_after = dw_after, a.dw_before = dw_before;
    return status(block_norm_backward_launch(a, (hipStream_t)stream));
}

tfno_status tfno_block_norm(const tfno_block_norm_desc *d, const void *y, const void *r, const void *gate, const float *w_after,
                            const float *w_before, const int *lengths, void *r_out, void *n_out, void *stream)
{
    return block_norm(d, false, y, r, gate, w_after, w_before, lengths, r_out, n_out, nullptr, nullptr, nullptr, nullptr, nullptr, stream);
}

tfno_status tfno_block_norm_backward(const tfno_block_norm_desc *d, const void *y, const void *r, const void *gate, const float *w_after,
                                     const float *w_before, const int *lengths, const void *d_r_out, const void *d_n_out, void *dy,
                                     void *dr, void *dgate, float *dw_after, float *dw_before, void *stream)
{
    return block_norm(d, true, y, r, gate, w_after, w_before, lengths, d_r_out, d_n_out, dy, dr, dgate, dw_after, dw_before, stream);
}

size_t tfno_block_norm_workspace_bytes(const tfno_block_norm_desc *d)
{
    return block_norm_sizes(d) == TFNO_OK ? block_norm_workspace_bytes(d->B, d->T, d->C, d->gate_kind) : 0;
}

tfno_status tfno_clip_grad_norm(const tfno_tensor *tensors, int count, double limit, float *norm, void *stream)
{
    if (count < 0 || !(limit >= 0.0)) return TFNO_ERR_SHAPE;
    if (count > 0 && !tensors) return TFNO_ERR_NULL;
    const auto bytes = [](const tfno_tensor &t) { return t.elements * (t.dtype == TFNO_BF16 ? 2 : 4); };
    for (int i = 0; i < count; ++i) {
        const tfno_tensor &t = tensors[i];
        if (!type_ok(t.dtype) || t.elements < 0 || t.elements >= (1LL << 40)) return TFNO_ERR_SHAPE;
        if (t.elements > 0 && !t.data) return TFNO_ERR_NULL;
        if (!aligned(t.data, t.dtype == TFNO_BF16 ? 2 : 4)) return TFNO_ERR_ALIGN;
    }
    if (!aligned(norm, 4)) return TFNO_ERR_ALIGN;
    // everything that is written, and what the sums go through, in the order of its addresses
    const size_t need = clip_workspace_bytes(count);
    const RegisteredWorkspace w = registered_workspace();
    if (!w.ptr || w.bytes < need) return TFNO_ERR_WORKSPACE;
    try {
        std::vector<std::pair<uintptr_t, uintptr_t>> ranges;
        ranges.reserve(count + 2);
        for (int i = 0; i < count; ++i)
            if (tensors[i].elements > 0) ranges.emplace_back((uintptr_t)tensors[i].data, (uintptr_t)tensors[i].data + bytes(tensors[i]));
        if (norm) ranges.emplace_back((uintptr_t)norm, (uintptr_t)norm + 4);
        ranges.emplace_back((uintptr_t)w.ptr, (uintptr_t)w.ptr + w.bytes);
        std::sort(ranges.begin(), ranges.end());
        for (size_t i = 1; i < ranges.size(); ++i)
            if (ranges[i].first < ranges[i - 1].second) return TFNO_ERR_ALIAS;
    } catch (...) {     // no memory on the host
        return TFNO_ERR_HIP;
    }
    return status(clip_launch(tensors, count, limit, norm, (double *)w.ptr, (hipStream_t)stream));
}

size_t tfno_clip_grad_norm_workspace_bytes(int count) { return count >= 0 ? clip_workspace_bytes(count) : 0; }

}  // extern "C"
