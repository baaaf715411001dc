// Gated linear recurrence h_t = a_t h_{t-1} + u_t over long sequences, forwards and backwards: the product
// with a lower triangle whose entries are products of T gates, evaluated as a scan.
//
// Mathematics.  A step is the affine map c -> a c + u of the state; steps compose to
//     (A2, H2) o (A1, H1) = (A2 A1, A2 H1 + H2),
// so a stretch of steps is summarised by two numbers a channel and stretches can be evaluated side by side.
// Backwards r_t = a_t (dy_t + r_{t+1}) is the same kind of map, run from the end, and has the same A.
//
// Split.  A tile is 128 steps x one 128-byte row of channels (64 bf16, 32 fp32).  Warp w of eight has
// steps 16 w .. 16 w + 15, a lane has its channels.  A warp composes its 16 steps, the eight maps meet in
// shared memory, and the gates and inputs, kept in registers, are swept a second time from the true state:
// the sequence is read once and written once.  CTAs are persistent, two on an SM.  Two more warps do what is
// not arithmetic on the sequence, so that its latency stays out of the way.  One deals the tiles, works out their
// addresses and the sequence boundaries in them, and has them copied into a ring in shared memory ahead of time (bulk
// tensor copies where the tensors' alignment allows; otherwise each warp copies its own steps, by cp.async or plain
// loads).  The other finds the state that enters each tile.
//
// Joining the tiles of a chain (one sequence instance, one row of channels).  The CTAs of a cluster, up to eight,
// take neighbouring tiles, a run.  Each sends its composed map to the CTAs behind it (st.async into their shared
// memory), and each folds what it got onto the state at the run's beginning.  That state comes from the last CTA of
// the run before, through a word in the workspace that is its own flag: the workspace is filled with ones, a
// bit pattern that no published value has, so a reader needs one round trip and no fence.  The fold is the
// same chain of operations whatever finishes first, so results do not depend on timing; the serial path along
// the sequence is one hop through L2 every 1024 steps.  Runs are dealt by a counter, chains first and then along
// the sequence.  A run only waits for runs dealt earlier, and a cluster works through its runs in the order dealt,
// so the earliest unfinished run never waits; each wait has a budget all the same.
//
// Packed sequences: a warp's 16 steps are common to its lanes, so a sequence boundary is a warp-uniform
// branch.  At a first step the state is replaced (not multiplied by zero: an infinity or NaN stays in its
// own sequence), and a map that contains a first step does not depend on what came before it.
//
// Measured: 8 x 2048 steps x 4096 bf16 channels, sigmoid gate: 75 us, 5.4 TB/s.  There and backwards the sweeps' instructions
// bound it (issue slots 50 to 55 % busy with 20 warps an SM; memory at 82 % of a copy's rate forwards).  With few
// chains it is the time of a tile: copy, sweep, join and second sweep follow one another, and two CTAs an SM are
// all there is to overlap them (1 x 65536 steps x 2048 bf16 channels: 254 us, 3.2 TB/s).  Forwards and backwards,
// 4 x 4096 steps x 2560 bf16 channels: 180 us.  8 x 2048 steps x 2048 fp32 channels: 68 us forwards, 94 backwards.  bf16 rows
// that split a word are taken element by element: 8 x 2048 steps x 4095 channels: 558 us forwards, 699 backwards.
#include <cuda_bf16.h>

#include "bf16_mma.cuh"
#include "common.cuh"
#include "waits.cuh"

namespace dastac {
namespace {

constexpr int kSteps = 16;                // steps a warp holds
constexpr int kWarps = 8;                 // warps of a tile
constexpr int kChunk = kSteps * kWarps;   // steps of a tile
constexpr int kWarpJoin = kWarps, kWarpDeal = kWarps + 1;
constexpr int kThreads = 32 * (kWarps + 2);
constexpr int kShortSteps = 16;           // up to so many steps a thread walks a whole sequence
static_assert(kChunk == DASTAC_LINREC_CHUNK, "the header states the distance of the kept states");

constexpr int32_t kErrLinrec = 0x4c52;    // "LR": a tile's wait for the tiles before it ran out
constexpr int32_t kErrLinrecCopy = 0x4c43;  // "LC": a wait for a copy or for a free stage did

constexpr int kRun = 8;                   // most tiles of a run
constexpr uint32_t kAbsent = 0xffffffffu; // a word of the workspace that nobody has written
constexpr uint32_t kReset = 0xfffffffeu;  // in place of a map's product: the state behind it is H whatever came before
constexpr int kNoTile = -1, kNoMore = -2; // orders of a tile behind the sequence's end, and of no run at all

struct Seq {
    char* data;
    int64_t batch_stride, step_stride;  // elements
};

enum { kG, kX, kH, kDy, kDg, kTensors };   // forward: kH out.  backward: kH = dx out, kDy in, kDg out

// Division of a number below 2^31 by a fixed one: (n + floor(n m / 2^32)) >> shift.
struct Divisor {
    uint32_t m, shift, d;
    explicit Divisor(uint32_t by = 1) : d(by) {
        shift = 0;
        while (((uint64_t)1 << shift) < by) ++shift;
        m = (uint32_t)(((((uint64_t)1 << shift) - by) << 32) / by + 1);
    }
    __device__ uint32_t of(uint32_t n) const { return (__umulhi(n, m) + n) >> shift; }
};

struct Params {
    Seq seq[kTensors];
    Divisor by_chains, by_groups;
    const float* h0;
    int64_t ld_h0;
    float* last;            // forward: h_last.  backward: dh0
    int64_t ld_last;
    const float* dlast;     // backward: dh_last
    int64_t ld_dlast;
    float* carries;
    const int64_t* offsets;
    int64_t sequences;
    int64_t batch, steps, channels;
    int32_t groups, chunks, runs; // rows of channels; tiles and runs along the sequence
    int64_t units;                // runs of all chains
    // workspace (runs > 1), filled with ones: the counter (of the last run dealt) and a word that is zero once
    // a wait has run out; a state a run
    unsigned long long* counter;
    uint32_t* abort;
    uint32_t* states;
    int32_t* err_word;
};

// ---- a lane's channels as one value --------------------------------------------------------------------
// One fp32 number, or two that the packed fp32 instructions take at once: the sweeps are bound by the number of
// instructions, and half of theirs are products and sums.
template <int N>
struct Pack;
template <>
struct Pack<1> {
    float v;
    __device__ Pack() {}
    __device__ explicit Pack(float x) : v(x) {}
    __device__ float operator[](int) const { return v; }
    __device__ void set(int, float x) { v = x; }
};
template <>
struct Pack<2> {
    unsigned long long v;
    __device__ Pack() {}
    __device__ explicit Pack(float x) : Pack(x, x) {}
    __device__ Pack(float x, float y) { asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y)); }
    __device__ float operator[](int j) const {
        float x, y;
        asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v));
        return j ? y : x;
    }
    __device__ void set(int j, float x) { *this = j ? Pack((*this)[0], x) : Pack(x, (*this)[1]); }
};
__device__ __forceinline__ Pack<1> operator*(Pack<1> a, Pack<1> b) { return Pack<1>(a.v * b.v); }
__device__ __forceinline__ Pack<1> operator+(Pack<1> a, Pack<1> b) { return Pack<1>(a.v + b.v); }
__device__ __forceinline__ Pack<1> fma(Pack<1> a, Pack<1> b, Pack<1> c) { return Pack<1>(fmaf(a.v, b.v, c.v)); }
__device__ __forceinline__ Pack<2> operator*(Pack<2> a, Pack<2> b) {
    Pack<2> r;
    asm("mul.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pack<2> operator+(Pack<2> a, Pack<2> b) {
    Pack<2> r;
    asm("add.rn.ftz.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pack<2> fma(Pack<2> a, Pack<2> b, Pack<2> c) {
    Pack<2> r;
    asm("fma.rn.ftz.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// The gate; for the sigmoid also its complement s(-g) = e s(g) with e = exp(-g), which keeps its relative
// precision where 1 - s(g) would not.  e stays finite (2^115 at most), NaN passes.
// The approximate exponential and reciprocal are good to 2^-22: packed fp32 sequences with logarithmic gates come out with
// 2.9e-7 of their size, 1.4e-7 with gates to the last bit.
template <int GATE, int N>
__device__ __forceinline__ Pack<N> exp_of(Pack<N> g) {
    Pack<N> t = g * Pack<N>(GATE == DASTAC_GATE_LOG ? 1.4426950408889634f : -1.4426950408889634f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float e = t[j];
        if (GATE == DASTAC_GATE_SIGMOID) asm("min.NaN.f32 %0, %1, %2;" : "=f"(e) : "f"(e), "f"(115.f));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(e));
        t.set(j, e);
    }
    return t;
}
template <int GATE, int N>
__device__ __forceinline__ void gate_of(Pack<N> g, Pack<N>& a, Pack<N>& shut) {
    if (GATE == DASTAC_GATE_VALUE) {
        a = g;
        return;
    }
    const Pack<N> t = exp_of<GATE, N>(g);
    if (GATE == DASTAC_GATE_LOG) {
        a = t;
        return;
    }
    const Pack<N> d = t + Pack<N>(1.f);
#pragma unroll
    for (int j = 0; j < N; ++j) {
        float r;
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(d[j]));
        a.set(j, r);
    }
    shut = t * a;
}

// The product of gates of a map, kept finite so that it leaves a state of zero at zero.
template <int N>
__device__ __forceinline__ Pack<N> finite(Pack<N> a) {
#pragma unroll
    for (int j = 0; j < N; ++j) a.set(j, fminf(fmaxf(a[j], -3.4028235e38f), 3.4028235e38f));
    return a;
}

// ---- a lane's channels -------------------------------------------------------------------------------
// A lane holds one 32-bit word a step: an fp32 channel, or two bf16 channels.  PAIR: the two are neighbours
// in one aligned word of memory.  Otherwise they are channels lane and lane + 32, taken one element at a time
// (odd pitches and bases).
enum Access { kTensor, kWord, kElement };   // whole tiles by tensor copies (16-byte alignment); words; elements
template <typename T, int ACCESS>
struct Lane {
    static constexpr bool PAIR = sizeof(T) == 2 && ACCESS != kElement;
    static constexpr int N = sizeof(T) == 2 ? 2 : 1;
    static constexpr int kChannels = 32 * N;
    static constexpr bool kWords = sizeof(T) == 4 || PAIR;
    static constexpr int kAccess = ACCESS;
    __device__ static int channel(int lane, int j) { return PAIR ? 2 * lane + j : lane + 32 * j; }
    // p points at the row's first channel of this tile; live: how many channels the tile has (0: no row)
    __device__ static bool has(int lane, int live) { return (PAIR ? 2 * lane : lane) < live; }
    __device__ static uint32_t load(const char* p, int lane, int live) {
        if (kWords) return has(lane, live) ? __ldg((const uint32_t*)p + lane) : 0u;
        uint32_t v = lane < live ? (uint32_t)__ldg((const uint16_t*)p + lane) : 0u;
        if (lane + 32 < live) v |= (uint32_t)__ldg((const uint16_t*)p + lane + 32) << 16;
        return v;
    }
    // The same for a warp's steps into words of shared memory that only this lane reads, asynchronously where memory has
    // whole words: `rows` of them from p on, `pitch` bytes apart; what does not exist becomes zero.
    __device__ static void fetch(uint32_t* words, const char* p, uint32_t pitch, int lane, int live, int rows) {
        if (kWords) {
            const bool on = has(lane, live) && rows > 0;
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(words + lane);
            if (on) p += 4 * lane;
            if (rows >= kSteps) {
                const int size = on ? 4 : 0;
#pragma unroll
                for (int i = 0; i < kSteps; ++i)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 128 * i), "l"(p + (uint64_t)pitch * (uint32_t)i), "r"(size)
                                 : "memory");
            } else {
#pragma unroll 1
                for (int i = 0; i < kSteps; ++i)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to + 128 * i),
                                 "l"(p + (uint64_t)pitch * (uint32_t)(i < rows ? i : 0)), "r"(on && i < rows ? 4 : 0)
                                 : "memory");
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) words[32 * i + lane] = i < rows ? load(p + (uint64_t)pitch * (uint32_t)i, lane, live) : 0u;
        }
    }
    __device__ static Pack<N> get(uint32_t w) {
        if constexpr (N == 1) return Pack<1>(__uint_as_float(w));
        else return Pack<2>(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
    }
    // p points at the lane's own (first) channel
    __device__ static constexpr int lane_bytes(int lane) { return lane * (sizeof(T) == 4 || PAIR ? 4 : 2); }
    __device__ static void store(char* p, int lane, int live, Pack<N> v) {
        if (sizeof(T) == 4) {
            if (lane < live) *(float*)p = v[0];
        } else if (PAIR) {
            if (2 * lane < live) *(__nv_bfloat162*)p = __floats2bfloat162_rn(v[0], v[N - 1]);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (lane + 32 * j < live) ((__nv_bfloat16*)p)[32 * j] = __float2bfloat16_rn(v[j]);
        }
    }
    // an fp32 row (a state), the tile's first channel at p; p may be NULL
    __device__ static Pack<N> load_state(const float* p, int lane, int live) {
        Pack<N> v(0.f);
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (p && channel(lane, j) < live) v.set(j, p[channel(lane, j)]);
        return v;
    }
    __device__ static void store_state(float* p, int lane, int live, Pack<N> v) {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (channel(lane, j) < live) p[channel(lane, j)] = v[j];
    }
};

// ---- sequence boundaries -----------------------------------------------------------------------------------
// How many of the offsets are <= t (a whole warp): each round narrows the search 32-fold.
__device__ __forceinline__ int64_t offsets_upto(const Params& p, int64_t t, int lane) {
    int64_t lo = 0, hi = p.sequences + 1;   // offsets[lo - 1] <= t < offsets[hi] as far as they exist
    while (hi - lo > 0) {
        const int64_t step = (hi - lo + 31) / 32, at = lo + lane * step;
        const int n = __popc(__ballot_sync(~0u, at < hi && __ldg(p.offsets + at) <= t));   // the first n lanes
        if (n == 0) break;   // t < offsets[lo]
        const int64_t last = lo + (n - 1) * step;
        hi = min(hi, last + step);
        lo = last + 1;
    }
    return lo;
}

// Rows of empty sequences (packed only): the state comes out as it went in.
template <int CH>
__device__ __forceinline__ void copy_empty(const Params& p, const float* in, int64_t ld_in, int64_t c0, int live, int warp, int lane) {
    if (!p.offsets || !p.last) return;
    for (int64_t q0 = 32 * warp; q0 < p.sequences; q0 += 32 * kWarps) {
        const int64_t q = q0 + lane;
        uint32_t empty = __ballot_sync(~0u, q < p.sequences && __ldg(p.offsets + q) >= __ldg(p.offsets + q + 1));
        while (empty) {
            const int i = __ffs(empty) - 1;
            empty &= empty - 1;
            for (int c = lane; c < live; c += 32)
                p.last[(q0 + i) * p.ld_last + c0 + c] = in ? in[(q0 + i) * ld_in + c0 + c] : 0.f;
        }
    }
}

// ---- the tiles of a CTA ----------------------------------------------------------------------------------
template <int N>
struct __align__(8 * N) Map {
    Pack<N> A, H;   // c -> A c + H
};

// A tile as the dealing warp hands it over.
struct Dealt {
    int32_t order, live;   // place along the scan, or kNoTile, kNoMore; channels
    int32_t rows, any;     // steps; whether a step begins or ends a sequence or lies outside all of them
    int32_t chunk;         // place along the sequence
    int32_t run;           // ... of the scan
    int64_t instance, c0, chain;
    int64_t offset[kTensors];     // elements to the tile's first step and channel
    uint32_t first[kChunk / 32], last[kChunk / 32], inside[kChunk / 32];   // a bit a step: begins / ends a sequence, belongs to one
    int32_t seq[kChunk];   // the sequence of a step (written where any is set)
};
// A warp's share of it.
struct Bounds {
    uint32_t first, last, inside;
    const int32_t* seq;
};
__device__ __forceinline__ Bounds bounds_of(const Dealt& d, int warp) {
    static_assert(kSteps == 16, "two warps share a word");
    const int w = warp >> 1, s = 16 * (warp & 1);
    return Bounds{d.first[w] >> s & 0xffffu, d.last[w] >> s & 0xffffu, d.inside[w] >> s & 0xffffu, d.seq + kSteps * warp};
}

template <int N, bool BACK, int R>
struct Shared {
    Map<N> mail[2][kRun - 1][32];              // the maps of the run's tiles before this one, of this run and the next
    static constexpr int kSets = BACK ? 1 : 2;  // forward: of this tile and the one before, so that one barrier a tile is enough
    Pack<N> A[kSets][kWarps][32], H[kSets][kWarps][32];   // the warps' maps
    Pack<N> states[BACK ? kWarps : 1][32];     // backward: the sums of the forward maps (the same products), which give the states
    int reset[kSets][kWarps], states_reset[kWarps];       // whether they contain a first step
    Pack<N> entering[2][32];                   // the state that enters the tile
    uint64_t full[R], empty[R], ready[2];      // a stage is filled (or its tile dealt) / free; entering is there
    uint64_t dealt[R + 2];                     // for the joining warp: an entry of the queue is there
    uint64_t mailed[2], credit[2];             // the maps are there; each CTA behind has read the ones before last
    uint64_t told[4], taken[4];                // a run has been dealt to this CTA; rank 0: all CTAs know
    uint32_t inbox[4];
    Dealt queue[R + 2];                        // tile n's entry is rewritten once every warp is past tile n
    __device__ Dealt& tile(int n) { return queue[n % (R + 2)]; }
    int abort;
};

// A bounded wait by a whole warp; false after an expiry here or elsewhere in the CTA.  The warp sleeps up to kNap ns
// between looks, so that it does not take issue slots from those that work.  CLUSTER: what the barrier announces was
// written by another CTA.
constexpr uint32_t kNap = 4000;
template <bool CLUSTER>
__device__ __forceinline__ bool look(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    if (CLUSTER)
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(kNap)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\t"
            "mbarrier.try_wait.parity.acquire.cta.shared::cta.b64 p, [%1], %2, %3;\n\t"
            "selp.u32 %0, 1, 0, p;\n\t}"
            : "=r"(ok)
            : "r"(bar), "r"(parity), "r"(kNap)
            : "memory");
    return ok != 0;
}
template <bool CLUSTER>
__device__ __noinline__ bool wait_long(uint32_t bar, uint32_t parity, volatile int* abort, int32_t* err_word) {
    const long long t0 = clock64();
    while (!look<CLUSTER>(bar, parity)) {
        if (*abort) return false;
        if (clock64() - t0 > kDefaultWaitBudget) {
            *abort = 1;
            if (err_word) atomicCAS(err_word, 0, kErrLinrecCopy);
            return false;
        }
    }
    return true;
}
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait_on(uint64_t* bar, uint32_t parity, int* abort, const Params& p) {
    const uint32_t at = smem_u32(bar);
    return __all_sync(~0u, look<CLUSTER>(at, parity) || wait_long<CLUSTER>(at, parity, abort, p.err_word));
}

// ---- joining the tiles of a chain --------------------------------------------------------------------
// A value as a published word: every NaN is the same one, none of the reserved patterns.
__device__ __forceinline__ uint32_t word_of(float v) { return v != v ? 0x7fffffffu : __float_as_uint(v); }

template <int N>
__device__ __forceinline__ void publish_state(const Params& p, int64_t run, Pack<N> h, int lane) {
#pragma unroll
    for (int j = 0; j < N; ++j)
        asm volatile("st.relaxed.gpu.global.u32 [%0], %1;" ::"l"(p.states + (run * N + j) * 32 + lane), "r"(word_of(h[j])) : "memory");
}
// Whether to go on waiting since t0; gives up when the budget runs out here or elsewhere, with the error word
// set: the results of the call are void then, but every tile goes on.
__device__ __forceinline__ bool keep_waiting(const Params& p, long long t0) {
    uint32_t alive;
    asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(alive) : "l"(p.abort) : "memory");
    if (alive == 0) return false;
    if (clock64() - t0 <= kDefaultWaitBudget) return true;
    atomicExch(p.abort, 0u);
    if (p.err_word) atomicCAS(p.err_word, 0, kErrLinrec);
    return false;
}
__device__ __forceinline__ uint32_t read_word(const uint32_t* w) {
    uint32_t v;
    asm volatile("ld.relaxed.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(w) : "memory");
    return v;
}

// Sends a map to the CTA of this rank: one copy of a lane's words that its `mailed` barrier counts.
template <int N>
__device__ __forceinline__ void send_map(uint32_t to, uint32_t bar, uint32_t rank, bool reset, const Map<N>& m) {
    const uint32_t at = map_to_cta(to, rank), remote = map_to_cta(bar, rank);
    if constexpr (N == 2)
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];" ::"r"(at),
                     "r"(reset ? kReset : word_of(m.A[0])), "r"(reset ? kReset : word_of(m.A[1])), "r"(word_of(m.H[0])), "r"(word_of(m.H[1])),
                     "r"(remote)
                     : "memory");
    else
        asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];" ::"r"(at),
                     "r"(reset ? kReset : word_of(m.A[0])), "r"(word_of(m.H[0])), "r"(remote)
                     : "memory");
}

// What enters a chain: the state given for the sequence (backwards the gradient of its last state).  Packed
// sequences take theirs in where they begin.
template <bool BACK>
__device__ __forceinline__ const float* end_state(const Params& p, const Dealt& t) {
    const float* from = BACK ? p.dlast : p.h0;
    return p.offsets || !from ? nullptr : from + t.instance * (BACK ? p.ld_dlast : p.ld_h0) + t.c0;
}

// The state that enters the tile (joining warp).
template <typename L, int N, bool BACK, int R>
__device__ __forceinline__ Pack<N> enter(const Params& p, Shared<N, BACK, R>& sm, const Dealt& t, int it, uint32_t rank, int lane) {
    const int side = it & 1;
    if (rank > 0 && lane == 0) mbar_arrive_expect_tx(smem_u32(&sm.mailed[side]), rank * 32 * (uint32_t)sizeof(Map<N>));
    Pack<N> state(0.f);
    if (t.run == 0) {
        // the tiles behind the first get the given state within its map, so that it has been read when the last tile
        // writes its own, maybe in the same place
        if (rank == 0) state = L::load_state(end_state<BACK>(p, t), lane, t.live);
    } else {
        const uint32_t* w = p.states + ((t.chain * p.runs + t.run - 1) * N) * 32 + lane;
        uint32_t v[N];
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = read_word(w + 32 * j);
        const long long t0 = clock64();
#pragma unroll
        for (int j = 0; j < N; ++j) {
            while (v[j] == kAbsent && keep_waiting(p, t0)) v[j] = read_word(w + 32 * j);
            state.set(j, __uint_as_float(v[j]));
        }
        __syncwarp();
    }
    if (rank > 0) {
        wait_on<true>(&sm.mailed[side], it >> 1 & 1, &sm.abort, p);
#pragma unroll 1
        for (uint32_t k = 0; k < rank; ++k) {
            const Map<N> m = sm.mail[side][k][lane];
            state = __float_as_uint(m.A[0]) == kReset ? m.H : fma(m.A, state, m.H);
        }
    }
    return state;
}

// The map of the warps from .. to (exclusive, direction dir), and whether it contains a first step (`any`: whether
// one of the tile's maps does).
template <int N>
__device__ __forceinline__ Map<N> compose(const Pack<N> (*A)[32], const Pack<N> (*H)[32], const int* reset, bool any, int from, int to, int dir,
                                          int lane, bool& has) {
    Map<N> m;
    m.A = Pack<N>(1.f);
    m.H = Pack<N>(0.f);
    has = false;
    if (!any) {
#pragma unroll 4
        for (int w = from; w != to; w += dir) {
            const Pack<N> a = A[w][lane];
            m.H = fma(a, m.H, H[w][lane]);
            m.A = m.A * a;
        }
    } else {
#pragma unroll 1
        for (int w = from; w != to; w += dir) {
            const Pack<N> a = A[w][lane], h = H[w][lane];
            const bool r = reset[w] != 0;
            has |= r;
            m.H = r ? h : fma(a, m.H, h);
            m.A = m.A * a;
        }
    }
    m.A = finite<N>(m.A);
    return m;
}

// The scan's last warp sends the tile's map to the CTAs behind it in its cluster; the last tile of a run publishes the
// state behind it.  before, reset: the map of the warps before this one; own, r: this warp's.
template <int N, bool BACK, int R>
__device__ __forceinline__ void publish(const Params& p, Shared<N, BACK, R>& sm, const Dealt& t, const Map<N>& before, bool reset, const Map<N>& own,
                                        bool r, int it, uint32_t rank, uint32_t ranks, int lane) {
    bool known = reset || r;
    const int side = it & 1;
    Map<N> all;
    all.A = finite<N>(before.A * own.A);
    all.H = r ? own.H : fma(own.A, before.H, own.H);
    if (!known && ((t.run == 0 && rank == 0) || (rank == ranks - 1 && t.run + 1 < p.runs))) {
        wait_on(&sm.ready[side], it >> 1 & 1, &sm.abort, p);
        all.H = fma(all.A, sm.entering[side][lane], all.H);
        known = true;
    }
    // All CTAs behind get it, those without a tile of this run too: a CTA gives its credit for a run once it has that run's
    // mail, so none can give it twice before another has given it once, and a full count is one credit from each.
    if (rank + 1 < ranks) {
        wait_on<true>(&sm.credit[side], (it >> 1 & 1) ^ 1, &sm.abort, p);
        for (uint32_t to = rank + 1; to < ranks; ++to)
            send_map<N>(smem_u32(&sm.mail[side][rank][lane]), smem_u32(&sm.mailed[side]), to, known, all);
    }
    if (rank == ranks - 1 && t.run + 1 < p.runs) publish_state<N>(p, t.chain * p.runs + t.run, all.H, lane);
}

// ---- the two other warps -------------------------------------------------------------------------------
// The n-th run of this cluster, and this CTA's tile of it.  All of it is latency of one warp between others that
// compute, so it is kept short: the next run is drawn ahead, lanes work out the tensors' offsets side by side, and what
// only tiles with a sequence boundary need is written for those alone.
template <typename L, bool BACK, int R>
__device__ __forceinline__ bool deal(const Params& p, Shared<L::N, BACK, R>& sm, int n, unsigned long long& drawn, uint32_t rank, uint32_t ranks,
                                     int lane) {
    constexpr int CH = L::kChannels;
    Dealt& d = sm.tile(n);
    uint32_t unit = blockIdx.x / ranks + (uint32_t)n * (gridDim.x / ranks);
    if (p.runs > 1) {
        if (rank == 0) {
            unit = (uint32_t)min((unsigned long long)p.units, __shfl_sync(~0u, drawn, 0));
            if (lane == 0) drawn = atomicAdd(p.counter, 1ull) + 1;   // looked at the next time
        }
        if (ranks > 1) {
            const int box = n & 3;
            const uint32_t turn = n >> 2 & 1;
            if (rank == 0) {   // tells the cluster, once all have read what lay in the box before
                if (!wait_on<true>(&sm.taken[box], turn ^ 1, &sm.abort, p)) return false;
                if (lane < ranks) {
                    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(map_to_cta(smem_u32(&sm.inbox[box]), lane)), "r"(unit) : "memory");
                    mbar_arrive_cluster(map_to_cta(smem_u32(&sm.told[box]), lane));
                }
                __syncwarp();
            }
            if (!wait_on<true>(&sm.told[box], turn, &sm.abort, p)) return false;
            unit = *(volatile uint32_t*)&sm.inbox[box];
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(map_to_cta(smem_u32(&sm.taken[box]), 0));
        }
    }
    if (unit >= (uint32_t)p.units) {
        if (lane == 0) d.order = kNoMore;
        __syncwarp();
        return true;
    }
    const uint32_t run = p.by_chains.of(unit), chain = unit - run * p.by_chains.d;
    const uint32_t instance = p.by_groups.of(chain), group = chain - instance * p.by_groups.d;
    const int order = (int)(run * ranks + rank);
    if (order >= p.chunks) {
        if (lane == 0) d.order = kNoTile;
        __syncwarp();
        return true;
    }
    const int64_t c0 = (int64_t)(group * CH);
    const int chunk = BACK ? p.chunks - 1 - order : order;
    const int64_t t0 = (int64_t)(chunk * kChunk);   // below 2^30
    const int rows = min(kChunk, (int)(p.steps - t0));
    if (lane < (BACK ? kTensors : kH + 1)) d.offset[lane] = instance * p.seq[lane].batch_stride + t0 * p.seq[lane].step_stride + c0;
    if (lane == 0) {
        d.order = order;
        d.live = (int32_t)min((int64_t)CH, p.channels - c0);
        d.rows = rows;
        d.chunk = chunk;
        d.run = (int32_t)run;
        d.instance = instance;
        d.c0 = c0;
        d.chain = chain;
    }
    if (!p.offsets) {
        // the states enter and leave through the chain's ends, so only steps behind the last one are special
        const bool any = rows < kChunk;
        if (any && lane < kChunk / 32) {
            const int left = rows - 32 * lane;   // steps in this word and behind
            d.first[lane] = d.last[lane] = 0u;
            d.inside[lane] = left >= 32 ? ~0u : left > 0 ? (1u << left) - 1 : 0u;
        }
        if (lane == 0) d.any = any;
    } else {
        // the offsets behind the tile's beginning, as distances from it, and the one before
        const int64_t base = offsets_upto(p, t0, lane);
        const int64_t ahead = base + lane <= p.sequences ? __ldg(p.offsets + base + lane) - t0 : (int64_t)1 << 30;
        const int32_t next = (int32_t)min(ahead, (int64_t)1 << 30);
        const bool at_start = base > 0 && __ldg(p.offsets + base - 1) == t0;
        const bool quiet = !at_start && base > 0 && base <= p.sequences && rows == kChunk && __shfl_sync(~0u, next, 0) > kChunk &&
                           t0 + kChunk < p.steps;   // one sequence goes right through
        if (quiet) {
            if (lane == 0) d.any = 0;
        } else {
            uint32_t any = 0;
#pragma unroll
            for (int k = 0; k < kChunk / 32; ++k) {
                const int32_t t = 32 * k + lane;
                int n = 0;   // how many of these 32 offsets are <= t
#pragma unroll
                for (int step = 16; step > 0; step >>= 1)
                    if (__shfl_sync(~0u, next, n + step - 1) <= t) n += step;
                const int32_t prev_off = __shfl_sync(~0u, next, max(n - 1, 0)), next_off = __shfl_sync(~0u, next, n);
                int64_t q = base + n - 1;
                bool first = n > 0 ? prev_off == t : at_start && t == 0, last = next_off == t + 1;
                if (n == 31 && next_off <= t) {   // more boundaries than a warp holds: by bisection
                    int64_t lo = base + 32, hi = p.sequences + 1;
                    while (lo < hi) {
                        const int64_t mid = (lo + hi) >> 1;
                        if (__ldg(p.offsets + mid) - t0 <= t) lo = mid + 1; else hi = mid;
                    }
                    q = lo - 1;
                    first = __ldg(p.offsets + q) - t0 == t;
                    last = q < p.sequences && __ldg(p.offsets + q + 1) - t0 == t + 1;
                }
                const bool inside = t < rows && q >= 0 && q < p.sequences;
                const uint32_t in = __ballot_sync(~0u, inside);
                const uint32_t begins = __ballot_sync(~0u, inside && first);
                const uint32_t ends = __ballot_sync(~0u, inside && (last || t0 + t == p.steps - 1));
                d.seq[t] = (int32_t)(inside ? q : 0);
                if (lane == 0) {
                    d.first[k] = begins;
                    d.last[k] = ends;
                    d.inside[k] = in;
                }
                any |= begins | ends | ~in;
            }
            if (lane == 0) d.any = any != 0;
        }
    }
    __syncwarp();
    return true;
}

struct Maps {
    CUtensorMap g, x, dy;
};

// Announces a tile, with the copies of its tensors into the stage where tensor copies make them.
template <typename L, bool BACK>
__device__ __forceinline__ void fill(const Maps& maps, const Dealt& d, uint32_t* stage, uint64_t* full, int lane) {
    if (lane == 0) {
        const uint32_t bar = smem_u32(full);
        if (L::kAccess != kTensor || d.order < 0) {
            mbar_arrive(bar);
        } else {
            mbar_arrive_expect_tx(bar, (BACK ? 3 : 2) * kChunk * 128);
            auto copy = [&](int k, const CUtensorMap* m) {
                asm volatile(
                    "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                        smem_u32(stage + k * kChunk * 32)),
                    "l"(m), "r"((int)d.c0), "r"(d.chunk * kChunk), "r"((int)d.instance), "r"(bar)
                    : "memory");
            };
            copy(0, &maps.g);
            copy(1, &maps.x);
            if (BACK) copy(2, &maps.dy);
        }
    }
    __syncwarp();
}
// ... and the copies of a warp's own steps where they do not.
template <typename L, typename T, bool BACK>
__device__ __forceinline__ void fetch_own(const Params& p, const Dealt& d, uint32_t* stage, int warp, int lane) {
    if (d.order >= 0) {
        const int rows = d.rows - warp * kSteps;
        auto copy = [&](int k, const Seq& s, int64_t offset) {
            const uint32_t pitch = (uint32_t)(s.step_stride * (int64_t)sizeof(T));
            L::fetch(stage + k * kChunk * 32 + warp * (kSteps * 32),
                     s.data + offset * (int64_t)sizeof(T) + (rows > 0 ? (uint64_t)pitch * (uint32_t)(warp * kSteps) : 0), pitch, lane, d.live, rows);
        };
        copy(0, p.seq[kG], d.offset[kG]);
        copy(1, p.seq[kX], d.offset[kX]);
        if (BACK) copy(2, p.seq[kDy], d.offset[kDy]);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
}

// Nobody waits for this CTA's tiles any more, and copies in flight land before shared memory is released.
__device__ __forceinline__ void give_up(const Params& p, int lane) {
    if (p.runs > 1 && lane == 0) atomicExch(p.abort, 0u);
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000) {
    }
}

// The dealing warp.
template <typename L, bool BACK, int R>
__device__ __forceinline__ void deal_tiles(const Params& p, const Maps& maps, Shared<L::N, BACK, R>& sm, uint32_t* ring, uint32_t rank,
                                           uint32_t ranks, int lane) {
    constexpr int kStage = (BACK ? 3 : 2) * kChunk * 32;
    constexpr bool kTensorCopies = L::kAccess == kTensor;
    Turn fills{0, 0}, freed{0, 0};
    unsigned long long drawn = 0;
    if (p.runs > 1 && rank == 0 && lane == 0) drawn = atomicAdd(p.counter, 1ull) + 1;
    for (int n = 0;; ++n) {
        bool ok = true;
        // an entry may be rewritten once all warps have begun the tile R + 1 places back
        if (!kTensorCopies && n > R) {
            ok = wait_on(&sm.empty[freed.s], freed.parity, &sm.abort, p);
            freed.next(R);
        }
        ok = ok && deal<L, BACK, R>(p, sm, n, drawn, rank, ranks, lane);
        if (ok && kTensorCopies && n >= R) {   // a stage is filled once all warps have left the tile R places back
            ok = wait_on(&sm.empty[freed.s], freed.parity, &sm.abort, p);
            freed.next(R);
        }
        if (!ok) {
            give_up(p, lane);
            break;
        }
        if (lane == 0) mbar_arrive(smem_u32(&sm.dealt[n % (R + 2)]));
        fill<L, BACK>(maps, sm.tile(n), ring + fills.s * kStage, &sm.full[fills.s], lane);
        fills.next(R);
        if (sm.tile(n).order == kNoMore) break;
    }
}

// The joining warp.
template <typename L, bool BACK, int R>
__device__ __forceinline__ void join_tiles(const Params& p, Shared<L::N, BACK, R>& sm, uint32_t rank, uint32_t ranks, int lane) {
    if (p.chunks == 1) return;
    const uint32_t left = (uint32_t)p.chunks - (uint32_t)(p.runs - 1) * ranks;   // tiles of a chain's last run: of the ranks below
    Turn dealt{0, 0}, freed{0, 0};
    for (int it = 0;; ++it) {
        if (!wait_on(&sm.dealt[dealt.s], dealt.parity, &sm.abort, p)) break;
        dealt.next(R + 2);
        const Dealt& t = sm.tile(it);
        if (t.order == kNoMore) break;
        Pack<L::N> state(0.f);
        if (t.order >= 0) {
            state = enter<L, L::N, BACK, R>(p, sm, t, it, rank, lane);
        } else {   // no use for the mail, but it keeps this CTA in step with those that have a tile
            if (lane == 0) mbar_arrive_expect_tx(smem_u32(&sm.mailed[it & 1]), left * 32 * (uint32_t)sizeof(Map<L::N>));
            wait_on<true>(&sm.mailed[it & 1], it >> 1 & 1, &sm.abort, p);
        }
        __syncwarp();
        if (lane < rank) mbar_arrive_cluster(map_to_cta(smem_u32(&sm.credit[it & 1]), lane));   // the mail has been read
        // every warp has read what was there two tiles ago once it has begun or left the tile before this one
        if (it > 0) {
            if (!wait_on(&sm.empty[freed.s], freed.parity, &sm.abort, p)) break;
            freed.next(R);
        }
        sm.entering[it & 1][lane] = state;
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.ready[it & 1]));
    }
}

template <int N, bool BACK, int R>
__device__ __forceinline__ void init_barriers(Shared<N, BACK, R>& sm, uint32_t rank, uint32_t ranks) {
    if (threadIdx.x == 0) {
        for (int s = 0; s < R; ++s) {
            mbar_init(smem_u32(&sm.full[s]), 1);
            mbar_init(smem_u32(&sm.empty[s]), kWarps);
        }
        for (int k = 0; k < R + 2; ++k) mbar_init(smem_u32(&sm.dealt[k]), 1);
        for (int k = 0; k < 2; ++k) {
            mbar_init(smem_u32(&sm.ready[k]), 1);
            mbar_init(smem_u32(&sm.mailed[k]), 1);
            mbar_init(smem_u32(&sm.credit[k]), rank + 1 < ranks ? ranks - 1 - rank : 1);
        }
        for (int k = 0; k < 4; ++k) {
            mbar_init(smem_u32(&sm.told[k]), 1);
            mbar_init(smem_u32(&sm.taken[k]), ranks);
        }
        sm.abort = 0;
        fence_barrier_init();
    }
    __syncthreads();
    cluster_sync_all();   // the other CTAs' barriers exist
}
// A barrier of the eight warps; true if `stop` is set for one of them (they leave the loop together, whatever they saw).
__device__ __forceinline__ bool sync_eight(bool stop) {
    uint32_t any;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, 1, %2, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(any)
        : "r"((uint32_t)stop), "n"(32 * kWarps)
        : "memory");
    return any != 0;
}

// ---- forward -----------------------------------------------------------------------------------------
constexpr int kForwardStages = 2, kBackwardStages = 2;
constexpr size_t ring_bytes(bool back) { return (size_t)kChunk * 128 * (back ? 3 * kBackwardStages : 2 * kForwardStages); }

// A warp's first sweep: gates and inputs of its steps, and their map.  PLAIN: no boundary, every step is in.
template <typename L, int GATE, bool PLAIN, int N>
__device__ __forceinline__ Map<N> sweep_in(const Params& p, const Dealt& t, const Bounds& b, const uint32_t* wg, const uint32_t* wx, int lane,
                                           Pack<N> (&a)[kSteps], Pack<N> (&u)[kSteps]) {
    Map<N> m;
    m.A = Pack<N>(1.f);
    m.H = Pack<N>(0.f);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        Pack<N> shut;
        gate_of<GATE, N>(L::get(wg[32 * i]), a[i], shut);
        u[i] = L::get(wx[32 * i]);
        if (GATE == DASTAC_GATE_SIGMOID) u[i] = u[i] * shut;
        if (PLAIN) {
            m.H = fma(a[i], m.H, u[i]);
        } else {
            if (!(b.inside >> i & 1)) {
                a[i] = Pack<N>(1.f);
                u[i] = Pack<N>(0.f);
            }
            if (b.first >> i & 1) {   // the state is replaced by u
                if (p.h0) u[i] = fma(a[i], L::load_state(p.h0 + b.seq[i] * p.ld_h0 + t.c0, lane, t.live), u[i]);
                m.H = u[i];
            } else {
                m.H = fma(a[i], m.H, u[i]);
            }
        }
        m.A = m.A * a[i];
    }
    m.A = finite<N>(m.A);
    return m;
}

template <typename T, int GATE, int ACCESS>
__global__ void __launch_bounds__(kThreads, 2) linrec_forward_kernel(const __grid_constant__ Params p, const __grid_constant__ Maps maps) {
    using L = Lane<T, ACCESS>;
    constexpr int N = L::N, CH = L::kChannels, R = kForwardStages, kStage = 2 * kChunk * 32;
    extern __shared__ __align__(128) uint32_t ring[];
    __shared__ Shared<N, false, R> sm;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    uint32_t ranks;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    init_barriers(sm, rank, ranks);
    if (warp >= kWarps) {
        if (warp == kWarpDeal) deal_tiles<L, false, R>(p, maps, sm, ring, rank, ranks, lane);
        else join_tiles<L, false, R>(p, sm, rank, ranks, lane);
        __syncwarp();
        cluster_sync_all();   // no CTA leaves while another may still send to it
        return;
    }
    Turn turn{0, 0};
    bool filled = true, ended = false;
    // where the warps copy their own steps: tile n into its stage, once it is dealt; nothing is dealt behind the end
    auto fetch_tile = [&](int n, int to) {
        if (!ended && filled) {
            filled = wait_on(&sm.full[to], (uint32_t)(n / R) & 1, &sm.abort, p);
            ended = filled && sm.tile(n).order == kNoMore;
            if (filled) fetch_own<L, T, false>(p, sm.tile(n), ring + to * kStage, warp, lane);
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if (ACCESS != kTensor)
#pragma unroll 1
        for (int n = 0; n < R; ++n) fetch_tile(n, n);
    for (int it = 0;; ++it) {
        if (ACCESS == kTensor) filled = wait_on(&sm.full[turn.s], turn.parity, &sm.abort, p);
        else asm volatile("cp.async.wait_group %0;" ::"n"(R - 1) : "memory");
        const Dealt& t = sm.tile(it);
        const bool stop = !filled || t.order == kNoMore;
        const int stage = turn.s;
        if (!stop && t.order == kNoTile) {
            // in step with the joining warp, whose barriers must not get two phases ahead of it
            wait_on(&sm.ready[it & 1], it >> 1 & 1, &sm.abort, p);
            if (lane == 0) mbar_arrive(smem_u32(&sm.empty[stage]));
            turn.next(R);
            if (ACCESS != kTensor) fetch_tile(it + R, stage);
            continue;
        }
        if (stop) {   // nothing is written: others may still be composing the maps of the last tile on this side
            sync_eight(true);
            break;
        }
        const int side = it & 1;
        const uint32_t side_turn = it >> 1 & 1;
        const bool any = t.any != 0;
        Bounds b{0, 0, 0xffffu, nullptr};
        if (any) b = bounds_of(t, warp);

        Pack<N> a[kSteps], u[kSteps];
        const uint32_t* wg = ring + stage * kStage + warp * (kSteps * 32) + lane;
        const Map<N> own = !any ? sweep_in<L, GATE, true, N>(p, t, b, wg, wg + kChunk * 32, lane, a, u)
                                : sweep_in<L, GATE, false, N>(p, t, b, wg, wg + kChunk * 32, lane, a, u);
        sm.A[side][warp][lane] = own.A;
        sm.H[side][warp][lane] = own.H;
        __syncwarp();   // every lane has read the stage
        if (lane == 0) {
            sm.reset[side][warp] = b.first != 0;
            mbar_arrive(smem_u32(&sm.empty[stage]));
        }
        // with one tile a sequence: read before the last warp writes the state behind it, maybe in the same place
        if (p.chunks == 1 && warp == 0) sm.entering[side][lane] = L::load_state(end_state<false>(p, t), lane, t.live);
        if (sync_eight(false)) break;

        bool reset;
        const Map<N> before = compose<N>(sm.A[side], sm.H[side], sm.reset[side], any, 0, warp, 1, lane, reset);
        if (p.chunks > 1 && warp == kWarps - 1) publish<N, false, R>(p, sm, t, before, reset, own, b.first != 0, it, rank, ranks, lane);
        if (ACCESS != kTensor) fetch_tile(it + R, stage);   // a warp's steps lie in registers by now
        if (p.chunks > 1) wait_on(&sm.ready[side], side_turn, &sm.abort, p);
        Pack<N> state = sm.entering[side][lane];
        const int live = t.live;
        if (warp == 0 && p.carries) L::store_state(p.carries + (t.instance * p.chunks + t.chunk) * p.channels + t.c0, lane, live, state);
        state = reset ? before.H : fma(before.A, state, before.H);

        const uint32_t pitch = (uint32_t)(p.seq[kH].step_stride * (int64_t)sizeof(T));
        char* const hp = p.seq[kH].data + t.offset[kH] * (int64_t)sizeof(T) + (uint64_t)pitch * (uint32_t)(warp * kSteps) + L::lane_bytes(lane);
        if (!any) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                state = fma(a[i], state, u[i]);
                L::store(hp + (uint64_t)pitch * (uint32_t)i, lane, live, state);
            }
        } else {
            if (t.order == 0) copy_empty<CH>(p, p.h0, p.ld_h0, t.c0, live, warp, lane);
            const int rows = t.rows - warp * kSteps;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                state = b.first >> i & 1 ? u[i] : fma(a[i], state, u[i]);
                if (i < rows) L::store(hp + (uint64_t)pitch * (uint32_t)i, lane, live, b.inside >> i & 1 ? state : Pack<N>(0.f));
                if ((b.last >> i & 1) && p.last) L::store_state(p.last + b.seq[i] * p.ld_last + t.c0, lane, live, state);
            }
        }
        if (warp == kWarps - 1 && !p.offsets && p.last && t.chunk == p.chunks - 1)
            L::store_state(p.last + t.instance * p.ld_last + t.c0, lane, live, state);
        turn.next(R);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    cluster_sync_all();   // no CTA leaves while another may still send to it
}

// ---- backward ----------------------------------------------------------------------------------------
// The same tiles from the end.  The states in front of the steps are recomputed in fp32 from the kept
// state at the tile's beginning (forward maps of the eight warps, no waiting), the r at its end comes from
// the tiles behind it, joined in the other direction.  g, x and dy stay in their stage until the last sweep: gates
// and states fill the registers, and unpacking a word again is cheaper than spilling it.
// 4 x 4096 steps x 2560 bf16 channels: 112 us, 3.8 TB/s, bound by the issue and the fetch of instructions.
template <typename T, int GATE, int ACCESS>
__global__ void __launch_bounds__(kThreads, 2) linrec_backward_kernel(const __grid_constant__ Params p, const __grid_constant__ Maps maps) {
    using L = Lane<T, ACCESS>;
    constexpr int N = L::N, CH = L::kChannels, R = kBackwardStages, kStage = 3 * kChunk * 32;
    extern __shared__ __align__(128) uint32_t ring[];
    __shared__ Shared<N, true, R> sm;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    uint32_t ranks;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    init_barriers(sm, rank, ranks);
    if (warp >= kWarps) {
        if (warp == kWarpDeal) deal_tiles<L, true, R>(p, maps, sm, ring, rank, ranks, lane);
        else join_tiles<L, true, R>(p, sm, rank, ranks, lane);
        __syncwarp();
        cluster_sync_all();   // no CTA leaves while another may still send to it
        return;
    }
    Turn turn{0, 0};
    bool filled = true, ended = false;
    // where the warps copy their own steps: tile n into its stage, once it is dealt; nothing is dealt behind the end
    auto fetch_tile = [&](int n, int to) {
        if (!ended && filled) {
            filled = wait_on(&sm.full[to], (uint32_t)(n / R) & 1, &sm.abort, p);
            ended = filled && sm.tile(n).order == kNoMore;
            if (filled) fetch_own<L, T, true>(p, sm.tile(n), ring + to * kStage, warp, lane);
        } else {
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    if (ACCESS != kTensor)
#pragma unroll 1
        for (int n = 0; n < R - 1; ++n) fetch_tile(n, n);
    for (int it = 0;; ++it) {
        if (ACCESS != kTensor) fetch_tile(it + R - 1, turn.s == 0 ? R - 1 : turn.s - 1);   // the stage of the tile before
        if (ACCESS == kTensor) filled = wait_on(&sm.full[turn.s], turn.parity, &sm.abort, p);
        else asm volatile("cp.async.wait_group %0;" ::"n"(R - 1) : "memory");
        const Dealt& t = sm.tile(it);
        const bool stop = !filled || t.order == kNoMore;
        const int stage = turn.s;
        if (!stop && t.order == kNoTile) {
            // in step with the joining warp, whose barriers must not get two phases ahead of it
            wait_on(&sm.ready[it & 1], it >> 1 & 1, &sm.abort, p);
            if (lane == 0) mbar_arrive(smem_u32(&sm.empty[stage]));
            turn.next(R);
            continue;
        }
        const int side = it & 1;
        const uint32_t side_turn = it >> 1 & 1;
        const bool any = !stop && t.any != 0;
        Bounds b{0, 0, 0xffffu, nullptr};
        if (any) b = bounds_of(t, warp);
        const int live = stop ? 0 : t.live;
        Pack<N> prev = L::load_state(stop ? nullptr : p.carries + (t.instance * p.chunks + t.chunk) * p.channels + t.c0, lane, live);

        const uint32_t *wg = ring + stage * kStage + warp * (kSteps * 32) + lane, *wx = wg + kChunk * 32, *wd = wx + kChunk * 32;
        Pack<N> a[kSteps], u[kSteps];
        Map<N> own = !any ? sweep_in<L, GATE, true, N>(p, t, b, wg, wx, lane, a, u) : sweep_in<L, GATE, false, N>(p, t, b, wg, wx, lane, a, u);
        sm.states[warp][lane] = own.H;
        // the map of r over the same steps: the same product
        own.H = Pack<N>(0.f);
        if (!any) {
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) own.H = a[i] * (L::get(wd[32 * i]) + own.H);
        } else {
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                if (b.last >> i & 1) own.H = L::load_state(p.dlast ? p.dlast + b.seq[i] * p.ld_dlast + t.c0 : nullptr, lane, live);
                if (b.inside >> i & 1) own.H = a[i] * (L::get(wd[32 * i]) + own.H);
            }
        }
        sm.A[0][warp][lane] = own.A;
        sm.H[0][warp][lane] = own.H;
        if (lane == 0) {
            sm.states_reset[warp] = b.first != 0;
            sm.reset[0][warp] = b.last != 0;
        }
        if (sync_eight(stop)) break;

        bool reset;
        Map<N> before = compose<N>(sm.A[0], sm.states, sm.states_reset, any, 0, warp, 1, lane, reset);
        prev = reset ? before.H : fma(before.A, prev, before.H);
        before = compose<N>(sm.A[0], sm.H[0], sm.reset[0], any, kWarps - 1, warp, -1, lane, reset);
        sync_eight(false);   // the maps have been read
        if (p.chunks > 1 && warp == 0) publish<N, true, R>(p, sm, t, before, reset, own, b.last != 0, it, rank, ranks, lane);

        // u becomes the state in front of the step
        if (!any) {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const Pack<N> next = fma(a[i], prev, u[i]);
                u[i] = prev;
                prev = next;
            }
        } else {
            if (t.order == 0) copy_empty<CH>(p, p.dlast, p.ld_dlast, t.c0, live, warp, lane);
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const bool first = b.first >> i & 1;
                const Pack<N> next = first ? u[i] : fma(a[i], prev, u[i]);
                if (first) prev = L::load_state(p.h0 ? p.h0 + b.seq[i] * p.ld_h0 + t.c0 : nullptr, lane, live);
                u[i] = prev;
                prev = next;
            }
        }
        Pack<N> r(0.f);
        if (p.chunks > 1) {
            wait_on(&sm.ready[side], side_turn, &sm.abort, p);
            r = sm.entering[side][lane];
        } else {
            r = L::load_state(end_state<true>(p, t), lane, live);
        }
        r = reset ? before.H : fma(before.A, r, before.H);

        const uint32_t gpitch = (uint32_t)(p.seq[kDg].step_stride * (int64_t)sizeof(T)), xpitch = (uint32_t)(p.seq[kH].step_stride * (int64_t)sizeof(T));
        char* const dgp = p.seq[kDg].data + t.offset[kDg] * (int64_t)sizeof(T) + (uint64_t)gpitch * (uint32_t)(warp * kSteps) + L::lane_bytes(lane);
        char* const dxp = p.seq[kH].data + t.offset[kH] * (int64_t)sizeof(T) + (uint64_t)xpitch * (uint32_t)(warp * kSteps) + L::lane_bytes(lane);
        // gradients of step i; r becomes the r in front of it
        auto step = [&](int i, Pack<N>& dg, Pack<N>& dx) {
            const Pack<N> d = L::get(wd[32 * i]) + r;
            r = a[i] * d;
            if (GATE == DASTAC_GATE_SIGMOID) {
                const Pack<N> shut = exp_of<GATE, N>(L::get(wg[32 * i])) * a[i];   // as in gate_of, its reciprocal is at hand
                dx = d * shut;
                dg = r * shut * fma(L::get(wx[32 * i]), Pack<N>(-1.f), u[i]);
            } else {
                dx = d;
                dg = (GATE == DASTAC_GATE_LOG ? r : d) * u[i];
            }
        };
        if (!any) {
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                Pack<N> dg, dx;
                step(i, dg, dx);
                L::store(dgp + (uint64_t)gpitch * (uint32_t)i, lane, live, dg);
                L::store(dxp + (uint64_t)xpitch * (uint32_t)i, lane, live, dx);
            }
        } else {
            const int rows = t.rows - warp * kSteps;
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                if (b.last >> i & 1) r = L::load_state(p.dlast ? p.dlast + b.seq[i] * p.ld_dlast + t.c0 : nullptr, lane, live);
                Pack<N> dg(0.f), dx(0.f);
                if (b.inside >> i & 1) step(i, dg, dx);
                if (i < rows) {
                    L::store(dgp + (uint64_t)gpitch * (uint32_t)i, lane, live, dg);
                    L::store(dxp + (uint64_t)xpitch * (uint32_t)i, lane, live, dx);
                }
                if ((b.first >> i & 1) && p.last) L::store_state(p.last + b.seq[i] * p.ld_last + t.c0, lane, live, r);
            }
        }
        if (warp == 0 && !p.offsets && p.last && t.chunk == 0) L::store_state(p.last + t.instance * p.ld_last + t.c0, lane, live, r);
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&sm.empty[stage]));
        turn.next(R);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    cluster_sync_all();   // no CTA leaves while another may still send to it
}

// ---- a few steps: decoding -----------------------------------------------------------------------------
// A thread walks its channels' whole sequence (not packed, at most kShortSteps steps): no tile, no joining.
// 32 x 1 step x 4096 bf16 channels: 2 us, the latency of a launch and of one load after another.
template <typename T, int GATE, int ACCESS>
__global__ void __launch_bounds__(128) linrec_short_kernel(const Params p) {
    using L = Lane<T, ACCESS>;
    constexpr int N = L::N, CH = L::kChannels;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t chain = (int64_t)blockIdx.x * 4 + warp, instance = chain / p.groups;
    if (instance >= p.batch) return;
    const int64_t c0 = (chain - instance * p.groups) * CH;
    const int live = (int)min((int64_t)CH, p.channels - c0);
    const char* gp = p.seq[kG].data + (instance * p.seq[kG].batch_stride + c0) * (int64_t)sizeof(T);
    const char* xp = p.seq[kX].data + (instance * p.seq[kX].batch_stride + c0) * (int64_t)sizeof(T);
    char* hp = p.seq[kH].data + (instance * p.seq[kH].batch_stride + c0) * (int64_t)sizeof(T);
    Pack<N> state = L::load_state(p.h0 ? p.h0 + instance * p.ld_h0 + c0 : nullptr, lane, live);
    if (p.carries) L::store_state(p.carries + instance * p.channels + c0, lane, live, state);
#pragma unroll 4
    for (int i = 0; i < (int)p.steps; ++i) {
        const uint32_t vg = L::load(gp + i * p.seq[kG].step_stride * (int64_t)sizeof(T), lane, live);
        const uint32_t vx = L::load(xp + i * p.seq[kX].step_stride * (int64_t)sizeof(T), lane, live);
        Pack<N> a, shut, u = L::get(vx);
        gate_of<GATE, N>(L::get(vg), a, shut);
        if (GATE == DASTAC_GATE_SIGMOID) u = u * shut;
        state = fma(a, state, u);
        L::store(hp + i * p.seq[kH].step_stride * (int64_t)sizeof(T) + L::lane_bytes(lane), lane, live, state);
    }
    if (p.last) L::store_state(p.last + instance * p.ld_last + c0, lane, live, state);
}

// ---- host ----------------------------------------------------------------------------------------------
constexpr int64_t kMaxExtent = (int64_t)1 << 30;

dastac_status check_shape(const dastac_linrec_shape* s) {
    if (!s || s->batch < 0 || s->steps < 0 || s->channels < 0) return DASTAC_ERR_INVALID_ARG;
    if (s->gate != DASTAC_GATE_VALUE && s->gate != DASTAC_GATE_LOG && s->gate != DASTAC_GATE_SIGMOID)
        return DASTAC_ERR_INVALID_ARG;
    if (s->dtype != DASTAC_F32 && s->dtype != DASTAC_BF16) return DASTAC_ERR_UNSUPPORTED_EXPR;
    if (s->offsets ? s->sequences < 0 : s->sequences != 0) return DASTAC_ERR_INVALID_ARG;
    if (s->offsets && s->batch != 1) return DASTAC_ERR_SHAPE;
    if (s->batch > kMaxExtent || s->steps > kMaxExtent || s->channels > kMaxExtent || s->sequences > kMaxExtent)
        return DASTAC_ERR_OVERFLOW;
    return DASTAC_OK;
}

int group_width(int dtype) { return dtype == DASTAC_BF16 ? 64 : 32; }

// CTAs of a cluster.  As few as keep the chains ahead of the machine: with as many chains as clusters the run before
// is done when a run is dealt and nothing waits, and small clusters move more freely (512 chains of 16 tiles:
// 75 us with one CTA, 113 us with eight).  With fewer chains the tiles of a chain must be joined quickly
// (32 chains of 512 tiles: 254 us with eight, 364 us with four, 954 us with one).  Of the sizes from there on the one that leaves the
// fewest tiles of a run behind the sequence's end.
int run_length(int64_t chunks, int64_t chains) {
    int64_t least = (2LL * sm_count() + chains - 1) / (chains > 0 ? chains : 1);
    if (least > kRun) least = kRun;
    if (least > chunks) least = chunks;
    int best = least < 1 ? 1 : (int)least;
    int64_t fewest = INT64_MAX;
    for (int c = best; c <= kRun && c <= 2 * least; ++c) {
        const int64_t waste = (chunks + c - 1) / c * c - chunks;
        if (waste < fewest && (c == best || waste * 16 < fewest * 16 - chunks)) {
            fewest = waste;
            best = c;
        }
    }
    return best;
}

struct Layout {
    int64_t chunks, groups, chains, runs;
    int ranks;
    size_t bytes;  // the counter is at 0, the states at 256
};
Layout layout_of(const dastac_linrec_shape* s) {
    Layout l;
    const int64_t ch = group_width(s->dtype);
    l.chunks = (s->steps + kChunk - 1) / kChunk;
    l.groups = (s->channels + ch - 1) / ch;
    l.chains = l.groups * s->batch;
    l.ranks = run_length(l.chunks, l.chains);
    l.runs = (l.chunks + l.ranks - 1) / l.ranks;
    // whether there is any depends on the sequence's length alone, not on how its tiles are laid out on this device
    l.bytes = l.chunks > 1 ? 256 + (l.runs > 1 ? (size_t)(l.runs * l.chains) * ch * 4 : 0) : 0;
    return l;
}

// Whether the number of tiles of a valid shape is a grid.
bool tiles_fit(const dastac_linrec_shape* s) {
    const int64_t ch = group_width(s->dtype);
    const int64_t a = (s->steps + kChunk - 1) / kChunk, b = (s->channels + ch - 1) / ch;
    return a * b <= 0x7fffffffLL && a * b * s->batch <= 0x7fffffffLL;
}

dastac_status take(const dastac_linrec_shape* s, const dastac_sequence* q, bool output, Seq& out) {
    if (!q || !q->data || q->batch_stride < 0 || q->step_stride < 0) return DASTAC_ERR_INVALID_ARG;
    if ((uintptr_t)q->data % elt_size(s->dtype)) return DASTAC_ERR_ALIGNMENT;
    if (s->steps > 1 && q->step_stride >= kMaxExtent) return DASTAC_ERR_OVERFLOW;   // a step is at most 2^32 bytes
    // an input may repeat rows (stride 0), an output's rows must be apart
    if (output && ((s->steps > 1 && q->step_stride < s->channels) || (s->batch > 1 && q->batch_stride < s->channels)))
        return DASTAC_ERR_SHAPE;
    out = Seq{(char*)q->data, q->batch_stride, q->step_stride};
    return DASTAC_OK;
}
bool paired(const Seq& q) {   // neighbouring bf16 channels as one aligned word
    return ((uintptr_t)q.data & 3) == 0 && (q.batch_stride & 1) == 0 && (q.step_stride & 1) == 0;
}
// Whether a tensor map can describe the tensor: 16-byte alignment throughout, no repeated rows.
bool tensor_ok(const Params& p, const Seq& q, int e) {
    const int64_t per16 = 16 / e;
    return ((uintptr_t)q.data & 15) == 0 && (p.steps == 1 || (q.step_stride > 0 && q.step_stride % per16 == 0)) &&
           (p.batch == 1 || (q.batch_stride > 0 && q.batch_stride % per16 == 0));
}
bool encode(CUtensorMap* m, const Params& p, const Seq& q, int e) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const cuuint64_t row = (cuuint64_t)round_up(p.channels * e, 16);
    const cuuint64_t dims[3] = {(cuuint64_t)p.channels, (cuuint64_t)p.steps, (cuuint64_t)p.batch};
    const cuuint64_t strides[2] = {p.steps == 1 ? row : (cuuint64_t)q.step_stride * e, p.batch == 1 ? row : (cuuint64_t)q.batch_stride * e};
    const cuuint32_t box[3] = {(cuuint32_t)(128 / e), (cuuint32_t)kChunk, 1}, estr[3] = {1, 1, 1};
    return enc(m, e == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, 3, q.data, dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool BACK, typename T, int GATE, int ACCESS>
dastac_status launch(const Params& p, int ranks, cudaStream_t st) {
    Maps maps{};
    if (ACCESS == kTensor && !(encode(&maps.g, p, p.seq[kG], sizeof(T)) && encode(&maps.x, p, p.seq[kX], sizeof(T)) && (!BACK || encode(&maps.dy, p, p.seq[kDy], sizeof(T)))))
        return DASTAC_ERR_CUDA;
    auto kernel = BACK ? linrec_backward_kernel<T, GATE, ACCESS> : linrec_forward_kernel<T, GATE, ACCESS>;
    constexpr size_t smem = ring_bytes(BACK);
    static bool attr[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return DASTAC_ERR_CUDA;
    if (!attr[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return DASTAC_ERR_CUDA;
        attr[dev] = true;
    }
    const int64_t most = 2LL * sm_count() / ranks;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.units < most ? p.units : most) * ranks), 1, 1);
    cfg.blockDim = dim3(kThreads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)ranks;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kernel, p, maps) != cudaSuccess) {
        cudaGetLastError();
        return DASTAC_ERR_CUDA;
    }
    return launch_status();
}
template <typename T, int GATE, int ACCESS>
dastac_status launch_short(const Params& p, cudaStream_t st) {
    linrec_short_kernel<T, GATE, ACCESS><<<(unsigned)((p.batch * p.groups + 3) / 4), 128, 0, st>>>(p);
    return launch_status();
}
template <bool BACK, typename T, int GATE>
dastac_status launch_access(const Params& p, int ranks, bool pair, bool tensor, cudaStream_t st) {
    const bool few = !BACK && p.steps <= kShortSteps && !p.offsets;
    if (!pair && sizeof(T) == 2) return few ? launch_short<T, GATE, kElement>(p, st) : launch<BACK, T, GATE, kElement>(p, ranks, st);
    if (few) return launch_short<T, GATE, kWord>(p, st);
    return tensor ? launch<BACK, T, GATE, kTensor>(p, ranks, st) : launch<BACK, T, GATE, kWord>(p, ranks, st);
}
template <bool BACK, typename T>
dastac_status launch_gate(const Params& p, int gate, int ranks, bool pair, bool tensor, cudaStream_t st) {
    switch (gate) {
        case DASTAC_GATE_VALUE: return launch_access<BACK, T, DASTAC_GATE_VALUE>(p, ranks, pair, tensor, st);
        case DASTAC_GATE_LOG: return launch_access<BACK, T, DASTAC_GATE_LOG>(p, ranks, pair, tensor, st);
        default: return launch_access<BACK, T, DASTAC_GATE_SIGMOID>(p, ranks, pair, tensor, st);
    }
}

template <bool BACK>
dastac_status run(const dastac_linrec_shape* s, Params& p, void* workspace, size_t workspace_bytes, int32_t* err_word, cudaStream_t st) {
    const Layout l = layout_of(s);
    if (l.bytes) {
        if (!workspace || workspace_bytes < l.bytes || ((uintptr_t)workspace & 255)) return DASTAC_ERR_WORKSPACE;
        char* w = (char*)workspace;
        p.counter = (unsigned long long*)w;
        p.abort = (uint32_t*)(w + 8);
        p.states = (uint32_t*)(w + 256);
        if (l.runs > 1 && cudaMemsetAsync(w, 0xff, l.bytes, st) != cudaSuccess) {
            cudaGetLastError();
            return DASTAC_ERR_CUDA;
        }
    }
    p.offsets = s->offsets;
    p.sequences = s->sequences;
    p.batch = s->batch;
    p.steps = s->steps;
    p.channels = s->channels;
    p.groups = (int32_t)l.groups;
    p.chunks = (int32_t)l.chunks;
    p.runs = (int32_t)l.runs;
    p.units = l.runs * l.chains;
    p.by_chains = Divisor((uint32_t)l.chains);
    p.by_groups = Divisor((uint32_t)l.groups);
    p.err_word = err_word ? err_word : device_error_word();
    const int e = elt_size(s->dtype);
    const bool pair = e == 4 || (s->channels % 2 == 0 && paired(p.seq[kG]) && paired(p.seq[kX]) && paired(p.seq[kH]) && (!BACK || (paired(p.seq[kDy]) && paired(p.seq[kDg]))));
    const bool tensor = tensor_ok(p, p.seq[kG], e) && tensor_ok(p, p.seq[kX], e) && (!BACK || tensor_ok(p, p.seq[kDy], e));
    return e == 4 ? launch_gate<BACK, float>(p, s->gate, l.ranks, pair, tensor, st) : launch_gate<BACK, __nv_bfloat16>(p, s->gate, l.ranks, pair, tensor, st);
}

// Sequences without a step: the states come out as they went in.
dastac_status no_steps(const dastac_linrec_shape* s, const float* in, int64_t ld_in, float* out, int64_t ld_out, cudaStream_t st) {
    const int64_t rows = s->offsets ? s->sequences : s->batch;
    if (!out || rows == 0 || s->channels == 0 || in == out) return DASTAC_OK;
    // a single row may have any pitch, which a copy of rows would refuse
    const size_t width = (size_t)s->channels * 4, from = rows > 1 ? (size_t)ld_in * 4 : width, to = rows > 1 ? (size_t)ld_out * 4 : width;
    const cudaError_t e = in ? cudaMemcpy2DAsync(out, to, in, from, width, (size_t)rows, cudaMemcpyDeviceToDevice, st)
                             : cudaMemset2DAsync(out, to, 0, width, (size_t)rows, st);
    if (e == cudaSuccess) return DASTAC_OK;
    cudaGetLastError();
    return DASTAC_ERR_CUDA;
}

bool state_ok(const dastac_linrec_shape* s, const float* v, int64_t ld) {
    const int64_t rows = s->offsets ? s->sequences : s->batch;
    return !v || rows <= 1 || ld >= s->channels;
}

}  // namespace
}  // namespace dastac

using namespace dastac;

extern "C" dastac_status dastac_linrec_workspace(const dastac_linrec_shape* shape, size_t* bytes) {
    const dastac_status st = check_shape(shape);
    if (st != DASTAC_OK) return st;
    if (!bytes) return DASTAC_ERR_INVALID_ARG;
    if (!tiles_fit(shape)) return DASTAC_ERR_OVERFLOW;
    *bytes = layout_of(shape).bytes;
    return DASTAC_OK;
}

extern "C" dastac_status dastac_linrec_forward(const dastac_linrec_shape* shape, const dastac_sequence* g,
                                               const dastac_sequence* x, const float* h0, int64_t ld_h0,
                                               const dastac_sequence* h, float* h_last, int64_t ld_last,
                                               float* carries, void* workspace, size_t workspace_bytes,
                                               int32_t* err_word, void* stream) {
    dastac_status st = check_shape(shape);
    if (st != DASTAC_OK) return st;
    if (!state_ok(shape, h0, ld_h0) || !state_ok(shape, h_last, ld_last)) return DASTAC_ERR_SHAPE;
    if (((uintptr_t)h0 | (uintptr_t)h_last | (uintptr_t)carries) & 3) return DASTAC_ERR_ALIGNMENT;
    if (!tiles_fit(shape)) return DASTAC_ERR_OVERFLOW;
    if (shape->batch == 0 || shape->channels == 0) return DASTAC_OK;
    cudaStream_t cs = (cudaStream_t)stream;
    if (shape->steps == 0) return no_steps(shape, h0, ld_h0, h_last, ld_last, cs);
    Params p{};
    if ((st = take(shape, g, false, p.seq[kG])) != DASTAC_OK || (st = take(shape, x, false, p.seq[kX])) != DASTAC_OK ||
        (st = take(shape, h, true, p.seq[kH])) != DASTAC_OK)
        return st;
    p.h0 = h0;
    p.ld_h0 = ld_h0;
    p.last = h_last;
    p.ld_last = ld_last;
    p.carries = carries;
    return run<false>(shape, p, workspace, workspace_bytes, err_word, cs);
}

extern "C" dastac_status dastac_linrec_backward(const dastac_linrec_shape* shape, const dastac_sequence* g,
                                                const dastac_sequence* x, const dastac_sequence* dy, const float* h0,
                                                int64_t ld_h0, const float* carries, const float* dh_last,
                                                int64_t ld_dlast, const dastac_sequence* dg, const dastac_sequence* dx,
                                                float* dh0, int64_t ld_dh0, void* workspace, size_t workspace_bytes,
                                                int32_t* err_word, void* stream) {
    dastac_status st = check_shape(shape);
    if (st != DASTAC_OK) return st;
    if (!state_ok(shape, h0, ld_h0) || !state_ok(shape, dh_last, ld_dlast) || !state_ok(shape, dh0, ld_dh0))
        return DASTAC_ERR_SHAPE;
    if (((uintptr_t)h0 | (uintptr_t)dh_last | (uintptr_t)dh0 | (uintptr_t)carries) & 3) return DASTAC_ERR_ALIGNMENT;
    if (!tiles_fit(shape)) return DASTAC_ERR_OVERFLOW;
    if (shape->batch == 0 || shape->channels == 0) return DASTAC_OK;
    cudaStream_t cs = (cudaStream_t)stream;
    if (shape->steps == 0) return no_steps(shape, dh_last, ld_dlast, dh0, ld_dh0, cs);
    Params p{};
    if ((st = take(shape, g, false, p.seq[kG])) != DASTAC_OK || (st = take(shape, x, false, p.seq[kX])) != DASTAC_OK ||
        (st = take(shape, dy, false, p.seq[kDy])) != DASTAC_OK || (st = take(shape, dg, true, p.seq[kDg])) != DASTAC_OK ||
        (st = take(shape, dx, true, p.seq[kH])) != DASTAC_OK)
        return st;
    if (!carries) return DASTAC_ERR_INVALID_ARG;
    p.h0 = h0;
    p.ld_h0 = ld_h0;
    p.last = dh0;
    p.ld_last = ld_dh0;
    p.dlast = dh_last;
    p.ld_dlast = ld_dlast;
    p.carries = const_cast<float*>(carries);
    return run<true>(shape, p, workspace, workspace_bytes, err_word, cs);
}
