// The gated recurrence, channel by channel:
//     h_t = a_t h_(t-1) + b_t,   a = e^g (g a log-decay) or sigmoid(g),   b = x or (1 - a) x (mix)
// with the state before a sequence's first token and the one behind its last in fp32.  The gradient, against the time, with R the gradient of the state
// behind a token that comes from the tokens after it:
//     r_t = dh_t + R;   dx = r or r (1 - a);   dg = r (h_(t-1) - [mix] x) a [or a (1 - a)];   R <- a_t r_t
// and the initial state's gradient is the last R.  h is read as it was written.
#include <algorithm>
#include <cmath>
#include "layer.hpp"
#include "attn_ops.hpp"
#include "elems.hpp"

namespace triinv {

namespace {

// e^x, off by an ulp or two: 2^y with what the product y = x log2(e) lacks put right.  x in 16 bits: the factor is cut so that the product is exact.  BELOW: x <= 0.
template <int T, bool BELOW = false> __device__ __forceinline__ float exp_of(float x)
{
    if constexpr (T == OP_F32) {
        constexpr float LOG2E = 1.44269502f, LOW = 1.925963e-8f, LN2 = 0.693147182f;  // log2(e) in two parts
        const float y = x * LOG2E, rest = (fmaf(x, LOG2E, -y) + x * LOW) * LN2, e = __builtin_amdgcn_exp2f(y);
        // (where x is infinite the rest is none; where e is, what the rest takes away is not)
        return fmaf(BELOW ? e : fminf(e, 3.402823466e38f), __builtin_amdgcn_fmed3f(rest, -1.f, 1.f), e);
    } else {
        // 13 bits of it for the 11 of an fp16 number, 15 for the 8 of a bf16 number; what they leave of log2(e), times ln 2
        constexpr float CUT = T == OP_F16 ? 0x1.715p0f : 0x1.7154p0f, LEFT = T == OP_F16 ? 4.7194842e-5f : 4.8884952e-6f;
        const float e = __builtin_amdgcn_exp2f(x * CUT), r = BELOW ? __builtin_amdgcn_fmed3f(-x * LEFT, 0.f, 1.f) : __builtin_amdgcn_fmed3f(x * LEFT, -1.f, 1.f);  // (BELOW: one instruction less, its result clamped)
        const float t = T == OP_F16 ? fmaf((BELOW ? -0.5f : 0.5f) * r, r, r) : r;  // (of 88 LEFT the square is 150 halves of an ulp in fp16, 2 in bf16)
        return fmaf(BELOW ? -e : e, t, e);
    }
}
// 1 - e^x.
__device__ __forceinline__ float one_less_exp(float x, float e)
{
    float p = 1.f / 40320;  // x + x^2 / 2! + ... + x^8 / 8!
    p = fmaf(p, x, 1.f / 5040), p = fmaf(p, x, 1.f / 720), p = fmaf(p, x, 1.f / 120), p = fmaf(p, x, 1.f / 24), p = fmaf(p, x, 1.f / 6), p = fmaf(p, x, 0.5f), p = fmaf(p, x, 1.f);
    return fabsf(x) > 0.35f ? 1.f - e : -p * x;
}

struct Gate {
    float a, rest;  // the decay and one less it, where that is asked for
};
template <int T, bool LOGIT, bool REST> __device__ __forceinline__ Gate gate(float g)
{
    if constexpr (!LOGIT) {
        const float a = exp_of<T>(g);
        return {a, REST ? one_less_exp(g, a) : 0.f};
    } else {
        // s = e / (1 + e), e = e^-|g|, with all its bits, and 1 - s, which has one rounding: a decay near 1 is a factor of thousands of tokens (as 1 / (1 + e) from the
        // approximate reciprocal it left the state behind 6000 tokens 2e-6 off, so it is 4e-7).
        const float e = exp_of<T, true>(-fabsf(g)), d = 1.f + e;
        float r = __builtin_amdgcn_rcpf(d);
        if constexpr (T == OP_F32) r = fmaf(fmaf(-d, r, 1.f), r, r);
        const float s = e * r, most = 1.f - s;
        return g >= 0.f ? Gate{most, s} : Gate{s, most};
    }
}

// Tokens of a strip (lanes that take VEC channels each, CH together: 64, or where workgroups are many 128), strips of a workgroup, one after the other in time.
constexpr int MOST_STRIPS = 16, SHORT = 64;  // SHORT: tokens of the fewest strips
template <int DT, int GT, bool BACK> constexpr int TOKENS = !BACK && DT != OP_F32 && GT != OP_F32 ? 16 : 8;

// A byte for each strip of a tile, read together.
template <int STRIPS> union StripMarks {
    uint8_t of[STRIPS];
    uint32_t words[STRIPS / 4];
    __device__ __forceinline__ bool any() const
    {
        uint32_t x = 0u;
#pragma unroll
        for (int i = 0; i < STRIPS / 4; ++i) x |= words[i];
        return __builtin_amdgcn_readfirstlane(x) != 0u;
    }
};

struct ScanPlan {
    int n_seg, fine, groups;  // segments of a sequence; parts of a segment; groups of channels
    bool neighbours;    // on one XCD
    bool longest_first;  // packed sequences, one segment each
    v2f* part;          // [n_seq][n_seg fine][D]: a part's decay and what it brings; in the last one's place the initial state as it was (n_seg > 1)
};

// Sequence s: its tokens t0 to t0 + len - 1.
struct Sequence {
    int64_t t0, len;
};
__device__ __forceinline__ Sequence sequence(const ScanCall& a, int s)
{
    const auto among = [](int64_t x, int64_t from, int64_t to) { return x < from ? from : x > to ? to : x; };  // (whatever the array holds, tokens stay among those there are)
    const int64_t t0 = a.cu_seqlens ? among(a.cu_seqlens[s], 0, a.N) : s * a.Tlen, len = a.cu_seqlens ? among(a.cu_seqlens[s + 1], t0, a.N) - t0 : a.Tlen;
    return {t0, len};
}

// Whether a product of decays, none of them below 0, is in fp32's range.
__device__ __forceinline__ bool in_range(float a) { return a <= 3.402823466e38f; }

template <int VEC> __device__ __forceinline__ void load_state(const float* from, int64_t i, float (&x)[VEC])
{
#pragma unroll
    for (int e = 0; e < VEC; ++e) x[e] = from ? from[i + e] : 0.f;
}

// Rows of a tensor for a wavefront's tokens, as a buffer from the first of them (in memory) on: a lane's place in it is an offset of 32 bits, a token's row another one of all lanes
// (8 x 8192 tokens of 2048 channels took 198 us with a 64-bit product for each row and lane, 178 with a sum).  OUT in a lane's place: nothing is read or written.
constexpr uint32_t OUT = 0x80000000u;
template <int T, int TOK, bool BACK> struct RowsOf {
    static constexpr int SIZE = Elems<T, 1>::SIZE;
    __amdgpu_buffer_rsrc_t buffer;
    uint32_t lane, stride;
    __device__ __forceinline__ RowsOf(const void* p, int64_t first, int64_t s, uint32_t row, int c, bool in)
        : buffer(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(static_cast<const char*>(p)) + first * s * SIZE, 0, OUT, 0x00020000)), lane(in ? (row * (uint32_t)s + (uint32_t)c) * SIZE : OUT),
          stride((uint32_t)s * SIZE)
    {
    }
    __device__ __forceinline__ uint32_t row(int i) const { return (BACK ? TOK - 1 - i : i) * stride; }
    template <int VEC> __device__ __forceinline__ void load(Elems<T, VEC>& to, int i, bool there) const { to.load(buffer, there ? lane : OUT, row(i)); }
    template <int VEC> __device__ __forceinline__ void store(const float (&x)[VEC], int i, bool there) const
    {
        Elems<T, VEC> e;
        e.set(x);
        e.store(buffer, there ? lane : OUT, row(i));
    }
};
// Where a strip is: its wavefront's first token in the order of the run and first row in memory, its own first row behind that.
template <int TOK, int PER_WAVE, bool BACK> struct Strip {
    int64_t k0, first;
    uint32_t row;
    int left;   // tokens from its first one on, counted up to one more than it has (may be negative)
    bool full;  // the wavefront's tokens are all there, and others behind them
    __device__ __forceinline__ Strip(const Sequence& q, int64_t i0, int strip)
    {
        const int r = strip % PER_WAVE;
        k0 = i0 + __builtin_amdgcn_readfirstlane(strip - r) * TOK;
        first = BACK ? q.t0 + q.len - k0 - PER_WAVE * TOK : q.t0 + k0;
        row = (BACK ? PER_WAVE - 1 - r : r) * TOK;
        full = k0 + PER_WAVE * TOK < q.len;
        const int64_t n = q.len - k0 - r * TOK;
        left = n > TOK ? TOK + 1 : (int)n;
    }
};

// A strip's rows as they are in memory.
template <int DT, int GT, bool MIX, bool BACK, int VEC, int CH, bool ONLY> struct Raw {
    static constexpr int TOK = TOKENS<DT, GT, BACK>, PER_WAVE = 64 * VEC / CH;
    static constexpr bool X = BACK ? MIX && !ONLY : true, H = BACK && !ONLY;
    Elems<DT, VEC> x[X ? TOK : 1], d[BACK ? TOK : 1], h[H ? TOK : 1];
    Elems<GT, VEC> g[TOK];
    template <bool FULL> __device__ __forceinline__ void load(const ScanCall& a, const Strip<TOK, PER_WAVE, BACK>& at, int c, bool in)
    {
        const RowsOf<DT, TOK, BACK> of_x(a.x, at.first, a.x_stride, at.row, c, in), of_d(a.dh, at.first, a.dh_stride, at.row, c, in), of_h(a.h, at.first - 1, a.h_stride, at.row, c, in);
        const RowsOf<GT, TOK, BACK> of_g(a.g, at.first, a.g_stride, at.row, c, in);
#pragma unroll
        for (int i = 0; i < TOK; ++i) {
            const bool there = FULL || i < at.left;
            if constexpr (X) of_x.load(x[i], i, there);
            of_g.load(g[i], i, there);
            if constexpr (BACK) of_d.load(d[i], i, there);
            if constexpr (H) of_h.load(h[i], i, FULL || i + 1 < at.left);
        }
    }
    __device__ __forceinline__ void load(const ScanCall& a, const Sequence& q, int64_t i0, int strip, int c, bool in)
    {
        const Strip<TOK, PER_WAVE, BACK> at(q, i0, strip);
        if (at.full)
            load<true>(a, at, c, in);
        else
            load<false>(a, at, c, in);
    }
};

// A workgroup takes CH channels through a sequence, or through a segment of it, a tile of STRIPS times TOK tokens at a time (the gradient's runs from the last token to the first):
//   1  a strip forms the decay of its tokens and what they bring, from registers, and asks for its tokens of the next tile;
//   2  these go through LDS, and every strip puts together the state before its tokens from those before it;
//   3  from there it goes through its tokens, in registers still; where the last one ends the next tile begins.
// Where sequences and channels are too few for the card a sequence is cut into segments of whole tiles: a first launch (ONLY) writes what each segment but the last brings, in
// parts, so many that they fill the card too; the second begins a segment with the state that those before it leave.
//
// Log-decays may be above 0, and a product of decays may leave fp32's range where the states do not (they are zero or small, or a decay of 0 follows): infinite times nothing is not a
// number.  In a tile with such a strip the strips find the states before them one after the other, token by token; so does, from the sequence's first token on, a lane whose segment is
// behind such a part.  us, bf16 log-decays, half of the channels zeros and decays of 1 / e^20: 16 x 1500 tokens of 2048 channels 51 / 59, gradient 102 / 125, 512 x 16 of 1024
// 20 / 23; 4096 tokens of 2048 in segments 17 / 360.  Looking for them costs up to 3 in a hundred, and nothing with logits.
//
// Bound by memory: x, g (gradient: dh, h too) are read and h (dx, dg) written once.  8 x 8192 tokens of 2048 channels, bf16, logits and mix, 176 us, 4.6 TB/s: pieces of 128 bytes of a
// row, vector instructions in two fifths of the cycles; 16 x 1500, in pieces of 256, 58 us, 5.1 TB/s, its gradient 123, 4.8.  In LDS go a strip's two numbers a channel, nothing else.
// Tried: tiles in workgroups of their own that hand states on (8 x 8192 229 to 275 us, the waiting), 32 channels a workgroup (250), 32 strips (179), 8 (184), the next tile's tokens
// asked for before this one's decays (185).  4096 tokens of one sequence take 21 us, 9 of them the first launch; of 4 sequences' gradient 24 of 107.
template <int DT, int GT, bool LOGIT, bool MIX, bool BACK, int VEC, int CH, int STRIPS, bool ONLY> __global__ __launch_bounds__(STRIPS * CH / VEC) void k_scan(ScanCall a, ScanPlan p)
{
    constexpr bool REST = MIX || (BACK && LOGIT);
    constexpr int TOK = TOKENS<DT, GT, BACK>, TILE = TOK * STRIPS;
    constexpr int LANES = CH / VEC, PER_WAVE = 64 / LANES;  // of a strip; strips of a wavefront
    __shared__ float own[2][STRIPS][CH][2];  // of one tile and the next: one barrier a tile
    __shared__ float base[2][CH];
    constexpr bool STEEP = !LOGIT && !ONLY;  // whether products of decays may leave the range (the first launch hands them on as they are)
    __shared__ StripMarks<STRIPS> steep[2];  // (STEEP) of one tile and the next: which strips have one
    const int strip = threadIdx.x / LANES, i_c = threadIdx.x % LANES * VEC;
    int64_t block = (int64_t)blockIdx.y * gridDim.x + blockIdx.x;
    const int parts = p.n_seg * p.fine, units = ONLY ? parts : p.n_seg;  // of a sequence
    const int64_t blocks = (int64_t)a.n_seq * units * p.groups;
    if (block >= blocks) return;
    if (p.neighbours) {  // workgroups go to the eight XCDs in turn
        const int64_t x = block & 7, most = blocks & 7;
        block = x * (blocks >> 3) + (x < most ? x : most) + (block >> 3);
    }
    int unit = (int)(block / p.groups), group = (int)(block - (int64_t)unit * p.groups);
    if (!ONLY && p.longest_first) {
        const SeqUnit of = seq_unit(SeqMap{a.cu_seqlens, nullptr, 0, a.n_seq}, (unsigned)block, (unsigned)blocks, (unsigned)p.groups, true, reinterpret_cast<char*>(own));
        unit = of.seq, group = (int)of.unit;
    }
    const int s = unit / units, part = unit - s * units, seg = ONLY ? part / p.fine : part;
    const Sequence q = sequence(a, s);
    const int tiles = (int)((q.len + TILE - 1) / TILE), per = (tiles + p.n_seg - 1) / p.n_seg, end = seg * per + per < tiles ? seg * per + per : tiles;
    const int step = ONLY ? (per + p.fine - 1) / p.fine : per, j0 = ONLY ? seg * per + (part - seg * p.fine) * step : seg * per, j1 = j0 + step < end ? j0 + step : end;
    const bool in = group * CH + i_c < a.D;
    const int c = in ? group * CH + i_c : a.D - VEC;  // (lanes without a channel read another one's)
    const int64_t at_state = (int64_t)s * a.D + c;
    const float* const init = BACK ? a.dstate : a.state;
    float C[VEC];
    const auto initial = [&] {
#pragma unroll
        for (int e = 0; e < VEC; ++e) C[e] = p.part && !ONLY ? p.part[((int64_t)(s + 1) * parts - 1) * a.D + c + e][1] : init ? init[at_state + e] : 0.f;
    };
    const auto put_last = [&] {  // (of lanes with a channel)
        if (!a.last) return;
#pragma unroll
        for (int e = 0; e < VEC; ++e) a.last[at_state + e] = C[e];
    };
    if (ONLY && part == 0 && strip == 0) {
        initial();
#pragma unroll
        for (int e = 0; e < VEC; ++e)
            if (in) p.part[((int64_t)(s + 1) * parts - 1) * a.D + c + e] = v2f{0.f, C[e]};
    }
    if (ONLY && end < tiles && j0 >= j1 && strip == 0 && in) {  // a part of no tiles
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.part[((int64_t)s * parts + part) * a.D + c + e] = v2f{1.f, 0.f};
    }
    if (j0 >= j1 || (ONLY && end == tiles)) {  // nothing to do; a sequence without tokens keeps its state
        if (!ONLY && seg == 0 && q.len == 0 && strip == 0 && in) initial(), put_last();
        return;
    }
    Raw<DT, GT, MIX, BACK, VEC, CH, ONLY> next;
    next.load(a, q, (int64_t)j0 * TILE, strip, c, in);
    v2f all[VEC];  // ONLY: of the segment so far
    if (strip == 0) {  // (read before anything is written: the final state may go to the same place)
        if (part == 0) initial();
        if (!ONLY && seg > 0) {
            const v2f* const from = p.part + (int64_t)s * parts * a.D + c;
            bool finite = true;
#pragma unroll
            for (int e = 0; e < VEC; ++e) C[e] = from[e][1], finite &= in_range(from[e][0]);
#pragma unroll 4
            for (int k = 1; k < seg * p.fine; ++k)
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const v2f w = from[(int64_t)k * a.D + e];
                    C[e] = fmaf(w[0], C[e], w[1]), finite &= in_range(w[0]);
                }
            if (STEEP && CH == 64 && !finite) {  // from the sequence's first token on
                initial();
                constexpr int AT_ONCE = 4;
                for (int64_t i = 0; i < (int64_t)j0 * TILE; i += AT_ONCE) {
                    Elems<GT, VEC> g[AT_ONCE];
                    Elems<DT, VEC> b[AT_ONCE];
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u) {
                        const int64_t row = BACK ? q.t0 + q.len - 1 - i - u : q.t0 + i + u;
                        g[u].load(a.g, row * a.g_stride + c), b[u].load(BACK ? a.dh : a.x, row * (BACK ? a.dh_stride : a.x_stride) + c);
                    }
#pragma unroll
                    for (int u = 0; u < AT_ONCE; ++u)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) {
                            const Gate f = gate<GT, LOGIT, MIX && !BACK>(g[u][e]);
                            C[e] = BACK ? f.a * (b[u][e] + C[e]) : fmaf(f.a, C[e], MIX ? f.rest * b[u][e] : b[u][e]);
                        }
                }
            }
        }
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            all[e] = v2f{1.f, ONLY && part == 0 ? C[e] : 0.f};
            base[j0 & 1][i_c + e] = C[e];
        }
    }
    for (int j = j0; j < j1; ++j) {
        auto now = next;
        const int64_t i0 = (int64_t)j * TILE;
        const Strip<TOK, PER_WAVE, BACK> at(q, i0, strip);
        float da[TOK][VEC], db[TOK][VEC];  // decays; what a token brings (gradient: one less the decay)
        float A[VEC], H[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) A[e] = 1.f, H[e] = 0.f;
        const auto form = [&](int i) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const Gate f = gate<GT, LOGIT, REST>(now.g[i][e]);
                da[i][e] = f.a;
                if constexpr (BACK) {
                    db[i][e] = f.rest;
                    H[e] = f.a * (now.d[i][e] + H[e]);
                } else {
                    db[i][e] = MIX ? f.rest * now.x[i][e] : now.x[i][e];
                    H[e] = fmaf(f.a, H[e], db[i][e]);
                }
                A[e] *= f.a;
            }
        };
        if (at.full) {
#pragma unroll
            for (int i = 0; i < TOK; ++i) form(i);
        } else {
#pragma unroll
            for (int i = 0; i < TOK; ++i) {
                if (i < at.left) {
                    form(i);
                } else if constexpr (STEEP && !BACK) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) da[i][e] = 1.f, db[i][e] = 0.f;
                }
            }
        }
        if (j + 1 < j1) next.load(a, q, i0 + TILE, strip, c, in);
        float (*const mine)[CH][2] = own[j & 1];
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine[strip][i_c + e][0] = A[e], mine[strip][i_c + e][1] = H[e];
        if constexpr (STEEP) {
            bool good = true;
#pragma unroll
            for (int e = 0; e < VEC; ++e) good &= in_range(A[e]);
            steep[j & 1].of[strip] = __all(good) ? 0 : 1;
        }
        __syncthreads();
        if constexpr (ONLY) {
            if (strip == 0) {
#pragma unroll
                for (int w = 0; w < STRIPS; ++w)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) all[e] = v2f{all[e][0] * mine[w][i_c + e][0], fmaf(mine[w][i_c + e][0], all[e][1], mine[w][i_c + e][1])};
            }
            continue;
        }
        {
            const int first = strip / PER_WAVE * PER_WAVE;  // the wavefront's first strip
#pragma unroll
            for (int e = 0; e < VEC; ++e) C[e] = base[j & 1][i_c + e];
            const int before = __builtin_amdgcn_readfirstlane(first);
#pragma unroll 1
            for (int w = 0; w < before; w += 2) {  // two at a time are asked for together (four leave no room for a second workgroup: 64 sequences of 100 tokens 34 us, so 23)
                float d[2][VEC], b[2][VEC];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) d[i][e] = mine[w + i][i_c + e][0], b[i][e] = mine[w + i][i_c + e][1];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (w + i < before) {
#pragma unroll
                        for (int e = 0; e < VEC; ++e) C[e] = fmaf(d[i][e], C[e], b[i][e]);
                    }
            }
            if (PER_WAVE > 1 && strip != first) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) C[e] = fmaf(mine[first][i_c + e][0], C[e], mine[first][i_c + e][1]);
            }
        }
        if (STEEP && steep[j & 1].any()) {
#pragma unroll 1
            for (int turn = 0; turn < STRIPS; ++turn) {
                __syncthreads();
                if (strip != turn) continue;
                float S[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) S[e] = C[e] = base[j & 1][i_c + e];
#pragma unroll
                for (int i = 0; i < TOK; ++i) {
                    auto d = now.d[BACK ? i : 0];
                    if constexpr (BACK) {  // (widened here, not before the loop: registers)
#pragma unroll
                        for (uint32_t& w : d.w) asm volatile("" : "+v"(w));
                    }
                    if (!BACK || i < at.left) {  // (forward: what is not there is a decay of 1 that brings nothing)
#pragma unroll
                        for (int e = 0; e < VEC; ++e) S[e] = BACK ? da[i][e] * (d[e] + S[e]) : fmaf(da[i][e], S[e], db[i][e]);
                    }
                }
#pragma unroll
                for (int e = 0; e < VEC; ++e) base[j & 1][i_c + e] = S[e];
            }
        }
        const RowsOf<DT, TOK, BACK> out(a.out, at.first, a.out_stride, at.row, c, in);
        const RowsOf<GT, TOK, BACK> out_g(a.dg, at.first, a.dg_stride, at.row, c, in);
        const auto go = [&](int i, bool last) {
            if constexpr (BACK) {
                float dx[VEC], dg[VEC], past[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) past[e] = now.h[i][e];
                if (last) load_state<VEC>(a.state, at_state, past);
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float r = now.d[i][e] + C[e];
                    dx[e] = MIX ? r * db[i][e] : r;
                    dg[e] = r * (MIX ? past[e] - now.x[i][e] : past[e]) * (LOGIT ? da[i][e] * db[i][e] : da[i][e]);
                    C[e] = da[i][e] * r;
                }
                out.template store<VEC>(dx, i, true);
                out_g.template store<VEC>(dg, i, true);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) C[e] = fmaf(da[i][e], C[e], db[i][e]);
                out.template store<VEC>(C, i, true);
            }
            if (last && in) put_last();
        };
        if (at.full) {
#pragma unroll
            for (int i = 0; i < TOK; ++i) go(i, false);
        } else {
#pragma unroll
            for (int i = 0; i < TOK; ++i)
                if (i < at.left) go(i, i + 1 == at.left);
        }
        if (strip == STRIPS - 1) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) base[j + 1 & 1][i_c + e] = C[e];
        }
    }
    if (ONLY && strip == 0 && in) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) p.part[((int64_t)s * parts + part) * a.D + c + e] = all[e];
    }
}

// One token: VEC channels a lane.  Bound by memory: the state is read and written once, 8 bytes a channel.  256 sequences of 8192 channels 6 us, 4.9 TB/s with states that the caches
// hold in part; one of 2048 2 us, the launch.
constexpr int THREADS = 256;
template <int DT, int GT, bool LOGIT, bool MIX, int VEC> __global__ __launch_bounds__(THREADS) void k_scan_step(ScanStepCall a)
{
    const int groups = (a.D + THREADS * VEC - 1) / (THREADS * VEC);
    const unsigned block = blockIdx.y * gridDim.x + blockIdx.x;
    const int b = (int)(block / (unsigned)groups), c = ((int)(block - (unsigned)b * (unsigned)groups) * THREADS + (int)threadIdx.x) * VEC;
    if (b >= a.B || c >= a.D) return;
    Elems<DT, VEC> x;
    Elems<GT, VEC> g;
    x.load(a.x, b * a.x_stride + c), g.load(a.g, b * a.g_stride + c);
    const int64_t slot = a.slots ? a.slots[b] : b;
    float o[VEC] = {};
    if (slot >= 0 && slot < a.n_slot) {
        float* const at = a.state + slot * a.D + c;
        Elems<OP_F32, VEC> h;
        h.load(at, 0);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            const Gate f = gate<GT, LOGIT, MIX>(g[e]);
            o[e] = fmaf(f.a, h[e], MIX ? f.rest * x[e] : x[e]);
        }
        store_rounded<OP_F32, VEC>(at, 0, o);
    }
    store_rounded<DT, VEC>(a.h, b * a.h_stride + c, o);
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

// Segments of a sequence, by the tokens, sequences and channels of the call: so many that one to four rounds of the 256 compute units are full, whichever costs least, as parts of a
// walk with all compute units at work to its end: the walk (what part of a round stays empty costs about half of itself; segments take as long as the longest), the first launch's
// time, AGAIN of the whole's for all segments but one (it reads two thirds of the call's bytes, in the gradient one third, at a lower rate), LAUNCH for the launch and CHAIN for each tile, one after the other.  In us, 1 / 2 / 3 / 4 / 6 segments, sequences of 3000 tokens of 2048
// channels (32 workgroups each), bf16, logits and mix: 2 sequences 45 / 36 / 31 / 30 / 31, 3 48 / 41 / 45 / 49 / 47, 4 50 / 45 / 56 / 54 / 54, 5 53 / 72 / 62 / 69 / 65, 6 54 / 78 / 76 / 82 / 78;
// gradient 2 85 / 60 / 50 / 45 / 48, 3 88 / 66 / 75 / 66 / 70, 4 92 / 78 / 90 / 81 / 82, 5 101 / 120 / 101 / 111 / 106; fp32 log-decays 3 76 / 64 / 72 / 70 / 77, 5 88 / 113 / 103 / 114 / 115.
// One of 4096 tokens in 8 and 16 segments 23 / 21.  256 at most, for a segment reads what all before it bring: one of 262144 tokens of 64 channels in 128 / 256 / 1024 132 / 123 / 143.
// Sequences of fewer than three tiles are walked through as they are: 512 tokens (2 tiles) 11.7 in one, 13.5 in two.
int segments(int64_t N, int n_seq, int D, int tile, bool back)
{
    const double AGAIN = back ? 0.4 : 0.67, LAUNCH = (back ? 1.0e6 : 1.7e6) / ((double)N * D), CHAIN = back ? 0 : 0.29 * LAUNCH * tile / 256;
    const int64_t units = (int64_t)n_seq * ((D + 63) / 64), tiles = (N / n_seq + tile - 1) / tile;
    if (units >= 256 || tiles < 3) return 1;
    const auto cost = [&](int64_t n, int64_t per) {
        const double r = units * n / 256.0, walk = (1 + (std::ceil(r) - r) / (2 * r)) * (per * n) / tiles;
        return walk + CHAIN * per + (n > 1 ? AGAIN * (n - 1) / n + LAUNCH : 0);
    };
    int64_t best = 1;
    double least = cost(1, tiles);
    for (int rounds = 1; rounds <= 4; ++rounds) {
        const int64_t most = std::min<int64_t>({256 * rounds / units, tiles, 256}), per = (tiles + most - 1) / most, n = (tiles + per - 1) / per;
        const double c = cost(n, per);
        if (c < least) best = n, least = c;
    }
    return (int)best;
}

// Packed sequences that are cut have as many times the segments that they would have if all were as long as the mean one, for the longest to be shorter.  In us, once / twice / three times,
// lengths up to twice the mean, bf16, 1024 channels: 2 sequences of 1000 tokens 21 / 15 / 15, 8 of 1000 33 / 28 / 31, 3 of 5000 55 / 48 / 43, 5 of 5000 76 / 82 / 71, 8 of 5000 112 / 99 / 98;
// gradient 27 (3 of 1000) / 22 / 24, 48 (8 of 1000) / 40 / 40, 61 (2 of 5000) / 41 / 52, 130 (5) / 133 / 115, 185 (8) / 165 / 164; 30 of 7408 of 32 channels 42 / 46 / 50.
// 128 at most: 2 of 65536 of 128 channels in 64 / 128 / 256 / 512 72 / 52 / 62 / 88.
int packed_segments(int n) { return n > 1 ? std::min(2 * n, 128) : 1; }

// Parts of a segment: three workgroups a compute unit in the first launch.  (Gradient of 4 sequences of 4096 tokens of 2048 channels, two segments: 30 us of 128 were the first launch's
// when it had one part a segment, on half of the compute units.)
int parts_of(int64_t N, int n_seq, int D, int tile, int n_seg)
{
    const int64_t units = (int64_t)n_seq * ((D + 63) / 64) * (n_seg - 1), per = ((N / n_seq + tile - 1) / tile + n_seg - 1) / n_seg, n = 768 / units;
    return (int)(n < 1 ? 1 : n < per ? n : per);
}

// Whether a workgroup takes 128 channels in place of 64, 256 bytes of a 16-bit row: where such workgroups, one to a compute unit, leave few of these without work in the last
// round.  us with 64 / 128, bf16, logits and mix, sequences of 1500 tokens of 2048 channels: 12 (192 workgroups of 128) 58 / 48, 16 65 / 59, 20 (320) 94 / 98, 24 104 / 104, 32
// 138 / 126, 48 203 / 184; gradient 114 / 101, 133 / 122, 176 / 190, 198 / 200, 266 / 244, 396 / 362; packed sequences to 1399 tokens, 200 of 1000 channels 218 / 198, 64 of 2048
// 146 / 132.
bool wide(int n_seq, int D)
{
    const int64_t n = (int64_t)n_seq * ((D + 127) / 128), last = n % 256;
    return (D + 63) / 64 % 2 == 0 && n >= 192 && (last == 0 || last >= 128 || n > 1024);
}

template <bool BACK> struct Scan {
    const ScanCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX, int VEC, int CH, int STRIPS> int with(int n_seg) const
    {
        const int groups = (a.D + CH - 1) / CH;
        // Neighbouring groups of channels share cache lines where rows do not begin on one: these are put on one XCD.  48 packed sequences of 1100 tokens of 1000 channels,
        // fp16, 138 us as they come, 114 so; 16 of 2048 tokens of 4096 channels, where there is nothing to share, 194 and 223.
        const bool share = (a.x_stride * Elems<DT, 1>::SIZE | a.g_stride * Elems<GT, 1>::SIZE | a.out_stride * Elems<DT, 1>::SIZE) % 128 != 0;
        ScanPlan p{n_seg, n_seg > 1 ? parts_of(a.N, a.n_seq, a.D, TOKENS<DT, GT, BACK> * STRIPS, n_seg) : 1, groups, share, false, nullptr};
        // Packed sequences of different lengths begin with the longest, each on one XCD and the next on the next, where the chunk attention's do.  In us, order of the call / by length: 48
        // of 1000 channels to 2199 tokens 111 / 106, 24 of 2048 to 3000 126 / 115, 20 of 1024 to 4000 85 / 73; gradient of 20 of 2048 to 2000 141 / 130; equal lengths 104 / 104.
        p.longest_first = n_seg == 1 && by_length(SeqMap{a.cu_seqlens, nullptr, 0, a.n_seq}, (unsigned)std::min<int64_t>((int64_t)a.n_seq * p.groups, 1 << 20));
        p.neighbours = share && !p.longest_first;
        const dim3 grid = long_grid((int64_t)a.n_seq * n_seg * p.groups), block(STRIPS * CH / VEC);
        if constexpr (CH == 64) {
            if (n_seg > 1) {
                p.part = reinterpret_cast<v2f*>(a.workspace);
                const int rc = launch_kernel(false, k_scan<DT, GT, LOGIT, MIX, BACK, VEC, CH, STRIPS, true>, long_grid((int64_t)a.n_seq * n_seg * p.fine * p.groups), block, 0, a.stream, a, p);
                if (rc != LAUNCHED) return rc;
            }
        }
        return launch_kernel(false, k_scan<DT, GT, LOGIT, MIX, BACK, VEC, CH, STRIPS, false>, grid, block, 0, a.stream, a, p);
    }
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        const int n_mean = segments(a.N, a.n_seq, a.D, TOKENS<DT, GT, BACK> * MOST_STRIPS, BACK), n_seg = a.cu_seqlens ? packed_segments(n_mean) : n_mean;
        // Two channels a lane where every row's begin allows it.
        const auto even = [](const void* p, int64_t stride, int dtype) { return !p || (stride % 2 == 0 && reinterpret_cast<uintptr_t>(p) % (dtype == OP_F32 ? 8 : 4) == 0); };
        if (a.D % 2 == 0 && even(a.x, a.x_stride, DT) && even(a.g, a.g_stride, GT) && even(a.h, a.h_stride, DT) && even(a.dh, a.dh_stride, DT) && even(a.out, a.out_stride, DT) &&
            even(a.dg, a.dg_stride, GT)) {
            // Short sequences (packed: of half of SHORT in the mean) take as many strips as hold SHORT tokens: what counts is to begin and end workgroups.  In us, 16
            // strips / so: 512 of 1024 channels of 1 token 63 / 13, 16 66 / 22, 64 71 / 38, packed of 20 in the mean 77 / 32; gradient of 16 74 / 43, packed 81 / 51.  (Packed of 60 86 / 49
            // too, but one of 4000 among 63 of one token, 63 in the mean as well, 100 / 132.)
            if (a.N <= (int64_t)a.n_seq * (a.cu_seqlens ? SHORT / 2 : SHORT)) return with<DT, GT, LOGIT, MIX, 2, 128, SHORT / TOKENS<DT, GT, BACK>>(1);
            if constexpr (!BACK || DT != OP_F32)  // (whose 128 registers a lane do not hold a strip of it)
                if (n_seg == 1 && wide(a.n_seq, a.D)) return with<DT, GT, LOGIT, MIX, 2, 128, MOST_STRIPS>(1);
            return with<DT, GT, LOGIT, MIX, 2, 64, MOST_STRIPS>(n_seg);
        }
        return with<DT, GT, LOGIT, MIX, 1, 64, MOST_STRIPS>(n_seg);
    }
};
struct Step {
    const ScanStepCall& a;
    template <int DT, int GT, bool LOGIT, bool MIX, int VEC> int with() const
    {
        const dim3 grid = long_grid((int64_t)a.B * ((a.D + THREADS * VEC - 1) / (THREADS * VEC)));
        return launch_kernel(false, k_scan_step<DT, GT, LOGIT, MIX, VEC>, grid, dim3(THREADS), 0, a.stream, a);
    }
    template <int DT, int GT, bool LOGIT, bool MIX> int go() const
    {
        // Four channels a lane where every row's begin allows it: 256 sequences of 8192 channels, bf16, 9.0 us one by one, 6.4 so (eight 7.2); 16 of 4096 1.9 either way.
        const auto fours = [](const void* p, int64_t stride, int dtype) { return stride % 4 == 0 && reinterpret_cast<uintptr_t>(p) % (dtype == OP_F32 ? 16 : 8) == 0; };
        if (a.D % 4 == 0 && fours(a.x, a.x_stride, DT) && fours(a.g, a.g_stride, GT) && fours(a.h, a.h_stride, DT) && fours(a.state, a.D, OP_F32))
            return with<DT, GT, LOGIT, MIX, 4>();
        return with<DT, GT, LOGIT, MIX, 1>();
    }
};

}  // namespace

int64_t scan_workspace(int64_t N, int n_seq, int D)
{
    int64_t most = 0;  // (of either direction and every type)
    const auto count = [&](int tile, bool back) {
        const int n = segments(N, n_seq, D, tile, back);
        for (const int m : {n, packed_segments(n)}) {
            const int64_t parts = n > 1 ? (int64_t)m * parts_of(N, n_seq, D, tile, m) : 0;
            most = parts > most ? parts : most;
        }
    };
    count(TOKENS<OP_BF16, OP_BF16, false> * MOST_STRIPS, false), count(TOKENS<OP_F32, OP_F32, false> * MOST_STRIPS, false), count(TOKENS<OP_F32, OP_F32, true> * MOST_STRIPS, true);
    return 8 * n_seq * most * D;
}
int launch_scan(const ScanCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Scan<false>{a}); }
int launch_scan_bwd(const ScanCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Scan<true>{a}); }
int launch_scan_step(const ScanStepCall& a) { return types(a.dtype, a.g_dtype, a.logit, a.mix, Step{a}); }

}  // namespace triinv
