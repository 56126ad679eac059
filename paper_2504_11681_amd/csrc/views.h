// What the entry points of the operators along time check of their tensors.
#pragma once
#include "../../include/tfno.h"
#include "elements.h"
#include "workspace.h"

#include <algorithm>
#include <utility>

namespace tfno {

// A tensor [B, T, H, D] of the call with its last axis contiguous.
struct View {
    const void *p;
    int elem;
    long long B, T, H, D;
    Strides s;
    bool there() const { return p && B > 0 && T > 0 && H > 0; }
    long long span() const { return (B - 1) * s.batch + (T - 1) * s.token + (H - 1) * s.head + D; }   // in elements
    uintptr_t low() const { return (uintptr_t)p; }
    uintptr_t high() const { return (uintptr_t)p + (uintptr_t)span() * elem; }
};

inline Strides strides(const tfno_strides &s) { return Strides{s.batch, s.token, s.head}; }
inline View flat(const void *p, long long elements, int elem = 4) { return View{p, elem, 1, 1, 1, elements, Strides{0, 0, 0}}; }

inline bool strides_ok(const View &v)
{
    const Strides &s = v.s;
    if (s.batch < 0 || s.token < 0 || s.head < 0) return false;
    return (long double)v.B * s.batch + (long double)v.T * s.token + (long double)v.H * s.head < 1099511627776.0L;   // 2^40 elements
}

// No element of an output may be written twice: each axis steps over all that the finer ones cover.
inline bool distinct(const View &v)
{
    std::pair<long long, long long> axes[3] = {{v.s.head, v.H}, {v.s.token, v.T}, {v.s.batch, v.B}};
    std::sort(axes, axes + 3);
    long long covered = v.D;
    for (const auto &a : axes) {
        if (a.second <= 1) continue;
        if (a.first < covered) return false;
        covered += (a.second - 1) * a.first;
    }
    return true;
}

// What a tensor covers of every period of a buffer, in bytes from its pointer on: axes that step over whole periods do not count.  More than a period where it is no slice.
inline long long in_period(const View &v, long long period)
{
    const std::pair<long long, long long> axes[3] = {{v.s.head, v.H}, {v.s.token, v.T}, {v.s.batch, v.B}};
    long long covered = v.D * v.elem;
    for (const auto &a : axes)
        if (a.second > 1 && a.first * v.elem % period != 0) covered += (a.second - 1) * a.first * v.elem;
    return covered;
}
// Whether two tensors may share memory.  Ranges that meet are no clash where some axis of one of them is the period of a common buffer, in which both are slices that lie
// apart: rows of tokens, of batch elements or of heads, in whatever order the axes lie.
inline bool clash(const View &a, const View &b)
{
    if (!a.there() || !b.there() || a.high() <= b.low() || b.high() <= a.low()) return false;
    for (const View *v : {&a, &b}) {
        const std::pair<long long, long long> axes[3] = {{v->s.head, v->H}, {v->s.token, v->T}, {v->s.batch, v->B}};
        for (const auto &axis : axes) {
            const long long period = axis.first * v->elem;
            if (axis.second <= 1 || period <= 0) continue;
            const long long na = in_period(a, period), nb = in_period(b, period);
            const long long off = ((long long)((uintptr_t)a.p - (uintptr_t)b.p) % period + period) % period;     // a's slice begins here in b's period
            if (off >= nb && off + na <= period) return false;
        }
    }
    return true;
}
inline bool same(const View &a, const View &b)
{
    return a.p == b.p && (a.B <= 1 || a.s.batch == b.s.batch) && (a.T <= 1 || a.s.token == b.s.token) && (a.H <= 1 || a.s.head == b.s.head);
}

inline bool aligned(const void *p, int bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

// The registered workspace for a call that needs `need` bytes and touches `views`.
inline tfno_status workspace(size_t need, const View *views, int count, void **out)
{
    const RegisteredWorkspace w = registered_workspace();
    if (!w.ptr || w.bytes < need) return TFNO_ERR_WORKSPACE;
    for (int i = 0; i < count; ++i)
        if (clash(flat(w.ptr, (long long)w.bytes, 1), views[i])) return TFNO_ERR_ALIAS;
    *out = w.ptr;
    return TFNO_OK;
}

inline tfno_status status(hipError_t e) { return e == hipSuccess ? TFNO_OK : TFNO_ERR_HIP; }

template <int N>
tfno_status check_views(const View (&v)[N], int outputs, const std::pair<int, int> *in_place, int in_place_count)
{
    // the first `outputs` of the views are written; pairs of in_place may be one tensor
    for (int i = 0; i < N; ++i) {
        if (!strides_ok(v[i])) return TFNO_ERR_SHAPE;
        if (!aligned(v[i].p, v[i].elem)) return TFNO_ERR_ALIGN;
    }
    for (int i = 0; i < outputs; ++i) {
        if (v[i].there() && !distinct(v[i])) return TFNO_ERR_ALIAS;
        for (int j = 0; j < N; ++j) {
            if (i == j || (j < outputs && j < i) || !clash(v[i], v[j])) continue;
            bool allowed = false;
            for (int k = 0; k < in_place_count; ++k)
                allowed = allowed || (in_place[k].first == i && in_place[k].second == j && same(v[i], v[j]));
            if (!allowed) return TFNO_ERR_ALIAS;
        }
    }
    return TFNO_OK;
}

}  // namespace tfno
