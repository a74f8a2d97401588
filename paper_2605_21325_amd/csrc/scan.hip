// The gated recurrence, channel by channel:
//     h_t = a_t h_(t-1) + b_t,   a = e^g (g a log-decay) or sigmoid(g),   b = x or (1 - a) x (mix)
// with the state before a sequence's first token and the one behind its last in fp32.  The gradient, against the time, with R the gradient of the state
// behind a token that comes from the tokens after it:
//     r_t = dh_t + R;   dx = r or r (1 - a);   dg = r (h_(t-1) - [mix] x) a [or a (1 - a)];   R <- a_t r_t
// and the initial state's gradient is the last R.  h is read as it was written.
#include "layer.hpp"
#include "elems.hpp"

namespace triinv {

namespace {

// e^x, off by an ulp or so for every x: 2^y with the rounding of y = x log2(e) put right.
__device__ __forceinline__ float exp_full(float x)
{
    constexpr float LOG2E = 1.44269502f, LOW = 1.925963e-8f, LN2 = 0.693147182f;  // log2(e) in two parts
    const float y = x * LOG2E, rest = fmaf(x, LOG2E, -y) + x * LOW, e = __builtin_amdgcn_exp2f(y);
    return fabsf(y) < 128.f ? fmaf(e, rest * LN2, e) : e;
}
// 1 - e^x.
__device__ __forceinline__ float one_less_exp(float x, float e)
{
    if (fabsf(x) > 0.35f) return 1.f - e;
    float p = 1.f / 40320;  // x + x^2 / 2! + ... + x^8 / 8!
    p = fmaf(p, x, 1.f / 5040), p = fmaf(p, x, 1.f / 720), p = fmaf(p, x, 1.f / 120), p = fmaf(p, x, 1.f / 24), p = fmaf(p, x, 1.f / 6), p = fmaf(p, x, 0.5f), p = fmaf(p, x, 1.f);
    return -p * x;
}

struct Gate {
    float a, rest;  // the decay and one less it, where that is asked for
};
template <bool LOGIT, bool REST> __device__ __forceinline__ Gate gate(float g)
{
    if constexpr (!LOGIT) {
        const float a = exp_full(g);
        return {a, REST ? one_less_exp(g, a) : 0.f};
    } else {  // both of 1 / (1 + e) and e / (1 + e), e = e^-|g|, to their last bits
        const float e = exp_full(-fabsf(g)), d = 1.f + e;
        float r = __builtin_amdgcn_rcpf(d);
        r = fmaf(fmaf(-d, r, 1.f), r, r);
        const float s = e * r;
        return g >= 0.f ? Gate{r, s} : Gate{s, r};
    }
}

// First token of sequence s and one behind its last.
struct Sequence {
    int64_t t0, t1;
};
__device__ __forceinline__ Sequence sequence(const ScanCall& a, int64_t s)
{
    return a.cu_seqlens ? Sequence{a.cu_seqlens[s], a.cu_seqlens[s + 1]} : Sequence{s * a.Tlen, (s + 1) * a.Tlen};
}

constexpr int THREADS = 64;

// A lane takes a channel of a sequence through all its tokens.
template <int DT, int GT, bool LOGIT, bool MIX> __global__ __launch_bounds__(THREADS) void k_scan(ScanCall a)
{
    const int groups = (a.D + THREADS - 1) / THREADS;
    const int64_t s = blockIdx.x / groups;
    const int c = (int)(blockIdx.x % groups) * THREADS + threadIdx.x;
    if (c >= a.D) return;
    const Sequence q = sequence(a, s);
    float h = a.state ? a.state[s * a.D + c] : 0.f;
    for (int64_t t = q.t0; t < q.t1; ++t) {
        Elems<DT, 1> x;
        Elems<GT, 1> g;
        x.load(a.x, t * a.x_stride + c), g.load(a.g, t * a.g_stride + c);
        const Gate f = gate<LOGIT, MIX>(g[0]);
        h = fmaf(f.a, h, MIX ? f.rest * x[0] : x[0]);
        const float o[1] = {h};
        store_rounded<DT, 1>(a.out, t * a.out_stride + c, o);
    }
    if (a.last) a.last[s * a.D + c] = h;
}

template <int DT, int GT, bool LOGIT, bool MIX> __global__ __launch_bounds__(THREADS) void k_scan_bwd(ScanCall a)
{
    const int groups = (a.D + THREADS - 1) / THREADS;
    const int64_t s = blockIdx.x / groups;
    const int c = (int)(blockIdx.x % groups) * THREADS + threadIdx.x;
    if (c >= a.D) return;
    const Sequence q = sequence(a, s);
    float R = a.dstate ? a.dstate[s * a.D + c] : 0.f;
    for (int64_t t = q.t1 - 1; t >= q.t0; --t) {
        Elems<DT, 1> x, h, dh;
        Elems<GT, 1> g;
        if (MIX) x.load(a.x, t * a.x_stride + c);
        g.load(a.g, t * a.g_stride + c), dh.load(a.dh, t * a.dh_stride + c);
        float before = 0.f;
        if (t > q.t0)
            h.load(a.h, (t - 1) * a.h_stride + c), before = h[0];
        else if (a.state)
            before = a.state[s * a.D + c];
        const Gate f = gate<LOGIT, MIX || LOGIT>(g[0]);
        const float r = dh[0] + R, dx[1] = {MIX ? r * f.rest : r}, dg[1] = {r * (MIX ? before - x[0] : before) * (LOGIT ? f.a * f.rest : f.a)};
        store_rounded<DT, 1>(a.out, t * a.out_stride + c, dx);
        store_rounded<GT, 1>(a.dg, t * a.dg_stride + c, dg);
        R = f.a * r;
    }
    if (a.last) a.last[s * a.D + c] = R;
}

// A lane a channel.
template <int DT, int GT, bool LOGIT, bool MIX> __global__ __launch_bounds__(THREADS) void k_scan_step(ScanStepCall a)
{
    const int groups = (a.D + THREADS - 1) / THREADS;
    const int64_t b = blockIdx.x / groups;
    const int c = (int)(blockIdx.x % groups) * THREADS + threadIdx.x;
    if (c >= a.D) return;
    const int64_t slot = a.slots ? a.slots[b] : b;
    float o[1] = {0.f};
    if (slot >= 0 && slot < a.n_slot) {
        Elems<DT, 1> x;
        Elems<GT, 1> g;
        x.load(a.x, b * a.x_stride + c), g.load(a.g, b * a.g_stride + c);
        const Gate f = gate<LOGIT, MIX>(g[0]);
        float* const h = a.state + slot * a.D + c;
        *h = o[0] = fmaf(f.a, *h, MIX ? f.rest * x[0] : x[0]);
    }
    store_rounded<DT, 1>(a.h, b * a.h_stride + c, o);
}

// f with the kinds of the call as its template's arguments.
template <int DT, int GT, class F> int kinds(bool logit, bool mix, F f)
{
    if (logit) return mix ? f.template go<DT, GT, true, true>() : f.template go<DT, GT, true, false>();
    return mix ? f.template go<DT, GT, false, true>() : f.template go<DT, GT, false, false>();
}
template <class F> int types(int dtype, int g_dtype, bool logit, bool mix, F f)
{
    if (dtype == OP_F32) return kinds<OP_F32, OP_F32>(logit, mix, f);
    if (dtype == OP_F16) return g_dtype == OP_F32 ? kinds<OP_F16, OP_F32>(logit, mix, f) : kinds<OP_F16, OP_F16>(logit, mix, f);
    return g_dtype == OP_F32 ? kinds<OP_BF16, OP_F32>(logit, mix, f) : kinds<OP_BF16, OP_BF16>(logit, mix, f);
}

struct Forward {
    const ScanCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        const dim3 grid((unsigned)((int64_t)a.n_seq * ((a.D + THREADS - 1) / THREADS)));
        return launch_kernel(false, k_scan<DT, GT, LOGIT, MIX>, grid, dim3(THREADS), 0, a.stream, a);
    }
};
struct Backward {
    const ScanCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        const dim3 grid((unsigned)((int64_t)a.n_seq * ((a.D + THREADS - 1) / THREADS)));
        return launch_kernel(false, k_scan_bwd<DT, GT, LOGIT, MIX>, grid, dim3(THREADS), 0, a.stream, a);
    }
};
struct Step {
    const ScanStepCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        const dim3 grid((unsigned)((int64_t)a.B * ((a.D + THREADS - 1) / THREADS)));
        return launch_kernel(false, k_scan_step<DT, GT, LOGIT, MIX>, grid, dim3(THREADS), 0, a.stream, a);
    }
};

}  // namespace

int64_t scan_workspace(int64_t, int, int) { return 0; }
int launch_scan(const ScanCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Forward{a}); }
int launch_scan_bwd(const ScanCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Backward{a}); }
int launch_scan_step(const ScanStepCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Step{a}); }

}  // namespace triinv
