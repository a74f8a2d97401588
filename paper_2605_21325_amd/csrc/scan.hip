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

// Decays and what they bring over some tokens, C <- A C + H, put together.
__device__ __forceinline__ float carry_through(float C, float A, float H) { return fmaf(A, C, H); }

// What a tile tells the tiles behind it travels as one 64-bit word a channel, A above H, that is whole or not there yet: all ones, which no value becomes.
constexpr uint64_t NOT_YET = ~0ull;
__device__ __forceinline__ uint64_t word(float A, float H)
{
    const uint32_t h = H == H ? __builtin_bit_cast(uint32_t, H) : 0x7fc00000u;  // (a NaN of the inputs may be all ones)
    return (uint64_t)__builtin_bit_cast(uint32_t, A) << 32 | h;
}
__device__ __forceinline__ float high(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)(w >> 32)); }
__device__ __forceinline__ float low(uint64_t w) { return __builtin_bit_cast(float, (uint32_t)w); }

constexpr int TILE = SCAN_TILE, TOK = 8, WAVES = TILE / TOK;  // tokens of a tile, of a wavefront
constexpr int EVERY = 16;          // of a sequence's tiles the last of so many publishes the state behind it
constexpr int TOGETHER = 8;        // words a lane waits for at once
constexpr int PATIENCE = 1 << 22;  // polls of about a microsecond; see k_scan

struct ScanPlan {
    int64_t n_tile;          // of all sequences
    int groups;              // of channels
    uint32_t* tickets;       // [groups], or null: every sequence fits a tile
    uint64_t *part, *whole;  // [n_tile][D], [n_tile / EVERY + 1][D]
};

__global__ __launch_bounds__(256) void k_scan_clear(uint64_t* words, int64_t n, uint32_t* tickets, int groups)
{
    const int64_t i = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * 256 + threadIdx.x;
    if (2 * i + 1 < n)
        reinterpret_cast<v4u*>(words)[i] = v4u{~0u, ~0u, ~0u, ~0u};
    else if (2 * i < n)
        words[2 * i] = NOT_YET;
    if (i < groups) tickets[i] = 0u;
}

// A tile's sequence, its place among the sequence's tiles and the sequence's tokens t0 to t1 - 1.
struct Place {
    int s;
    int64_t j, tiles, t0, t1;
};
__device__ __forceinline__ Place place_of(const ScanCall& a, int64_t tile)
{
    if (!a.cu_seqlens) {  // the first tiles of all sequences, the second ones, ...: a tile waits for one that was begun long before
        const int64_t j = tile / a.n_seq;
        const int s = (int)(tile - j * a.n_seq);
        return {s, j, (a.Tlen + TILE - 1) / TILE, s * a.Tlen, (s + 1) * a.Tlen};
    }
    int lo = 0, n = a.n_seq;  // cu_chunks[lo] <= tile < cu_chunks[lo + n]; of several with the same first tile the last
    while (n > 1) {
        const int step = (n + 63) / 64, at = (threadIdx.x & 63) * step;
        const int there = __popcll(__ballot(at < n && a.cu_chunks[lo + at] <= tile)), k = there > 0 ? there - 1 : 0;
        lo += k * step, n = n - k * step < step ? n - k * step : step;
    }
    // (whatever the arrays hold, tokens and tiles stay among those there are)
    const auto among = [](int64_t x, int64_t from, int64_t to) { return x < from ? from : x > to ? to : x; };
    const int64_t c0 = among(a.cu_chunks[lo], 0, tile), t0 = among(a.cu_seqlens[lo], 0, a.N);
    return {lo, tile - c0, a.cu_chunks[lo + 1] - c0, t0, among(a.cu_seqlens[lo + 1], t0, a.N)};
}

template <int VEC> __device__ __forceinline__ void load_state(const float* from, int64_t i, float (&x)[VEC])
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = from ? from[i + e] : 0.f;
}

// One tile of a sequence: WAVES wavefronts of TOK tokens each, one after the other in time (the gradient's runs from the last token to the first), VEC channels a lane.
//   1  a wavefront loads its tokens, all at once, and forms its decay and what it brings;
//   2  the tile's own, from those, is published (the first one's with the initial state in it); the state before the tile is put together from the tiles before it:
//      from the last that published the state behind it, EVERY tiles apart;
//   3  the wavefronts go through their tokens, in registers still, from the states before them.
// Tiles are given out by ticket, each sequence's in order of time for each group of channels: every tile that one waits for has been begun, and publishes its own
// before it waits itself, so that the first tile not yet done never waits for one that is not running: every wait ends.  (A wait of seconds is given up, with NaN for a state.)
// A channel's sums have an order that follows from its place in its sequence alone: the same bits alone, in a batch and packed, and of a prompt's beginning.
template <int DT, int GT, bool LOGIT, bool MIX, bool BACK, int VEC> __global__ __launch_bounds__(64 * WAVES) void k_scan(ScanCall a, ScanPlan p)
{
    constexpr int CH = 64 * VEC;
    constexpr bool REST = MIX || (BACK && LOGIT);
    __shared__ float own[WAVES][CH][2];
    __shared__ float before_tile[CH];
    __shared__ uint32_t ticket;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    if (block >= p.n_tile * p.groups) return;
    const int group = (int)(block % p.groups);
    int64_t turn = block / p.groups;
    if (p.tickets) {
        if (threadIdx.x == 0) ticket = atomicAdd(p.tickets + group, 1u);
        __syncthreads();
        turn = __builtin_amdgcn_readfirstlane((int)ticket);
    }
    const Place at = place_of(a, turn);
    const int64_t tile = a.cu_seqlens ? turn : at.s * at.tiles + at.j;  // its words' place
    const int c = group * CH + lane * VEC;
    const bool in = c < a.D;
    const int64_t i0 = at.j * TILE + wave * TOK, length = at.t1 - at.t0;  // the wavefront's first token in the sequence's order
    const int n = (int)(length - i0 < TOK ? length - i0 : TOK);           // (may be negative)
    const int64_t first = BACK ? at.t1 - 1 - i0 : at.t0 + i0;
    constexpr int WAY = BACK ? -1 : 1;

    Elems<DT, VEC> rx[TOK], rd[BACK ? TOK : 1], rh[BACK ? TOK : 1];
    Elems<GT, VEC> rg[TOK];
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        rx[i].clear(), rg[i].clear();
        if constexpr (BACK) rd[i].clear(), rh[i].clear();
        if (i >= n || !in) continue;
        const int64_t t = first + WAY * i;
        if constexpr (!BACK || MIX) rx[i].load(a.x, t * a.x_stride + c);
        rg[i].load(a.g, t * a.g_stride + c);
        if constexpr (BACK) {
            rd[i].load(a.dh, t * a.dh_stride + c);
            if (i0 + i + 1 < length) rh[i].load(a.h, (t - 1) * a.h_stride + c);
        }
    }
    const float* const init = BACK ? a.dstate : a.state;
    if (at.j == 0 && wave == 0 && in) {  // (read before anything is published: the final state may go to the same place)
        float h[VEC];
        load_state<VEC>(init, (int64_t)at.s * a.D + c, h);
#pragma unroll
        for (int e = 0; e < VEC; ++e) before_tile[lane * VEC + e] = h[e];
    }

    float da[TOK][VEC], db[TOK][VEC];  // decays; what a token brings (gradient: one less the decay)
    float A[VEC], C[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) A[e] = 1.f, C[e] = 0.f;
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        if (i >= n) continue;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const Gate f = gate<LOGIT, REST>(rg[i][e]);
            da[i][e] = f.a;
            if constexpr (BACK) {
                db[i][e] = f.rest;
                C[e] = f.a * (rd[i][e] + C[e]);
            } else {
                db[i][e] = MIX ? f.rest * rx[i][e] : rx[i][e];
                C[e] = fmaf(f.a, C[e], db[i][e]);
            }
            A[e] *= f.a;
        }
    }
#pragma unroll
    for (int e = 0; e < VEC; ++e) own[wave][lane * VEC + e][0] = A[e], own[wave][lane * VEC + e][1] = C[e];
    __syncthreads();

    const bool others = p.tickets && at.tiles > 1;
    if (others) {
        if (wave == WAVES - 1 && in && at.j + 1 < at.tiles) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                A[e] = own[0][lane * VEC + e][0], C[e] = own[0][lane * VEC + e][1];
                if (at.j == 0) C[e] = carry_through(before_tile[lane * VEC + e], A[e], C[e]);
#pragma unroll
                for (int w = 1; w < WAVES; ++w) A[e] *= own[w][lane * VEC + e][0], C[e] = carry_through(C[e], own[w][lane * VEC + e][0], own[w][lane * VEC + e][1]);
                __hip_atomic_store(p.part + tile * a.D + c + e, word(A[e], C[e]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
        }
        if (wave == 0 && in && at.j > 0) {
            const int64_t back = at.j < EVERY ? at.j : at.j % EVERY + 1;  // tiles to put together
            const uint64_t* from = at.j < EVERY ? p.part + (tile - back) * a.D + c : p.whole + (tile - back) / EVERY * a.D + c;
            const uint64_t* const rest = p.part + (tile - back) * a.D + c;
            float h[VEC];
            for (int64_t j = 0; j < back; j += TOGETHER) {
                uint64_t v[TOGETHER][VEC];
                for (int polls = 0;; ++polls) {
                    bool there = true;
#pragma unroll
                    for (int i = 0; i < TOGETHER; ++i)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            v[i][e] = word(1.f, 0.f);
                            if (j + i < back) v[i][e] = __hip_atomic_load((j + i ? rest + (j + i) * a.D : from) + e, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                            there = there && v[i][e] != NOT_YET;
                        }
                    if (__all(there) || polls == PATIENCE) break;
                    __builtin_amdgcn_s_sleep(1);
                }
#pragma unroll
                for (int i = 0; i < TOGETHER; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) h[e] = j + i ? carry_through(h[e], high(v[i][e]), low(v[i][e])) : low(v[i][e]);
            }
#pragma unroll
            for (int e = 0; e < VEC; ++e) before_tile[lane * VEC + e] = h[e];
        }
        __syncthreads();
        if (wave == WAVES - 1 && in && at.j % EVERY == EVERY - 1 && at.j + 1 < at.tiles) {
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                __hip_atomic_store(p.whole + tile / EVERY * a.D + c + e, word(0.f, carry_through(before_tile[lane * VEC + e], A[e], C[e])), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (!in) return;
    const auto put_last = [&](int64_t s, const float (&x)[VEC]) {
        if (!a.last) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e) a.last[s * a.D + c + e] = x[e];
    };
    if (n > 0) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            C[e] = before_tile[lane * VEC + e];
            for (int w = 0; w < wave; ++w) C[e] = carry_through(C[e], own[w][lane * VEC + e][0], own[w][lane * VEC + e][1]);
        }
    }
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
        if (i >= n) continue;
        const int64_t t = first + WAY * i;
        if constexpr (BACK) {
            float dx[VEC], dg[VEC], past[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) past[e] = rh[i][e];
            if (i0 + i + 1 == length) load_state<VEC>(a.state, (int64_t)at.s * a.D + c, past);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float r = rd[i][e] + C[e];
                dx[e] = MIX ? r * db[i][e] : r;
                dg[e] = r * (MIX ? past[e] - rx[i][e] : past[e]) * (LOGIT ? da[i][e] * db[i][e] : da[i][e]);
                C[e] = da[i][e] * r;
            }
            store_rounded<DT, VEC>(a.out, t * a.out_stride + c, dx);
            store_rounded<GT, VEC>(a.dg, t * a.dg_stride + c, dg);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) C[e] = fmaf(da[i][e], C[e], db[i][e]);
            store_rounded<DT, VEC>(a.out, t * a.out_stride + c, C);
        }
        if (i0 + i + 1 == length) put_last(at.s, C);
    }
    // Sequences without tokens have no tile: the first tile of the next sequence sees to them, the last tile of all to those at the end.
    if (a.cu_seqlens && wave == 0) {
        const auto put_empty = [&](int64_t s) {
            const bool empty = a.cu_seqlens[s] == a.cu_seqlens[s + 1];
            if (empty) {
                float h[VEC];
                load_state<VEC>(init, s * a.D + c, h);
                put_last(s, h);
            }
            return empty;
        };
        if (at.j == 0)
            for (int64_t s = at.s - 1; s >= 0 && put_empty(s); --s) {}
        if (at.j == 0 && turn + at.tiles == p.n_tile)
            for (int64_t s = at.s + 1; s < a.n_seq && put_empty(s); ++s) {}
    }
}

// Final states of sequences that have no tokens, all of them.
__global__ __launch_bounds__(256) void k_scan_nothing(const float* init, float* last, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) last[i] = init ? init[i] : 0.f;
}

// A lane a channel.
constexpr int THREADS = 64;
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

// Whether a sequence may have several tiles.
bool chained(int64_t N, int64_t Tlen, bool packed) { return (packed ? N : Tlen) > TILE; }
int64_t words(int64_t n_tile, int D) { return (n_tile + n_tile / EVERY + 1) * D; }
constexpr int64_t aligned16(int64_t n) { return (n + 15) / 16 * 16; }

template <bool BACK> struct Scan {
    const ScanCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX, int VEC> int with() const
    {
        ScanPlan p{a.n_tile, (a.D + 64 * VEC - 1) / (64 * VEC), nullptr, nullptr, nullptr};
        if (chained(a.N, a.Tlen, a.cu_seqlens != nullptr)) {
            const int64_t n = words(a.n_tile, a.D);
            p.part = reinterpret_cast<uint64_t*>(a.workspace), p.whole = p.part + p.n_tile * a.D;
            p.tickets = reinterpret_cast<uint32_t*>(a.workspace + aligned16(8 * n));
            const int64_t threads = (n + 1) / 2 > p.groups ? (n + 1) / 2 : p.groups;
            const int rc = launch_kernel(false, k_scan_clear, long_grid((threads + 255) / 256), dim3(256), 0, a.stream, p.part, n, p.tickets, p.groups);
            if (rc != LAUNCHED) return rc;
        }
        return launch_kernel(false, k_scan<DT, GT, LOGIT, MIX, BACK, VEC>, long_grid(p.n_tile * p.groups), dim3(64 * WAVES), 0, a.stream, a, p);
    }
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        // Two channels a lane where every row's begin allows it.
        const auto even = [](const void* p, int64_t stride, int dtype) { return !p || (stride % 2 == 0 && reinterpret_cast<uintptr_t>(p) % (dtype == OP_F32 ? 8 : 4) == 0); };
        if (a.D % 2 == 0 && even(a.x, a.x_stride, DT) && even(a.g, a.g_stride, GT) && even(a.h, a.h_stride, DT) && even(a.dh, a.dh_stride, DT) && even(a.out, a.out_stride, DT) &&
            even(a.dg, a.dg_stride, GT))
            return with<DT, GT, LOGIT, MIX, 2>();
        return with<DT, GT, LOGIT, MIX, 1>();
    }
};
int nothing(const ScanCall& a, const float* init)
{
    if (!a.last) return LAUNCHED;
    const int64_t n = (int64_t)a.n_seq * a.D, groups = (n + 255) / 256;
    return launch_kernel(false, k_scan_nothing, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, a.stream, init, a.last, n);
}
struct Step {
    const ScanStepCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        const dim3 grid((unsigned)((int64_t)a.B * ((a.D + THREADS - 1) / THREADS)));
        return launch_kernel(false, k_scan_step<DT, GT, LOGIT, MIX>, grid, dim3(THREADS), 0, a.stream, a);
    }
};

}  // namespace

int64_t scan_workspace(int64_t N, int64_t n_tile, int D) { return N > TILE ? aligned16(8 * words(n_tile, D)) + aligned16(4 * ((D + 63) / 64)) : 0; }
int launch_scan(const ScanCall& a) { return a.N == 0 ? nothing(a, a.state) : types(a.dtype, a.g_dtype, a.logit, a.mix, Scan<false>{a}); }
int launch_scan_bwd(const ScanCall& a) { return a.N == 0 ? nothing(a, a.dstate) : types(a.dtype, a.g_dtype, a.logit, a.mix, Scan<true>{a}); }
int launch_scan_step(const ScanStepCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Step{a}); }

}  // namespace triinv
