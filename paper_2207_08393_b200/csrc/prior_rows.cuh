// Layer norm and the residual tail on rows: a row stays with a team of threads that passes over every array once.
//
// A team is 2 to 32 lanes of a warp, or a few warps; a thread has up to 32 features of its row, in pieces of 16 bytes.  Pieces begin
// at multiples of 16 bytes of the array, not of the row: where rows begin anywhere (EDGES), the rows of a block are those that
// begin at the same place inside a piece, so that a thread's features are the same ones in each of its rows.  In a VJP it
// keeps the sums of their weights' gradients in registers; the teams of a block add those sums up at its end, and
// weight_grads (prior_norm.cuh) adds up the blocks.
//
// Bound by memory, if the instructions are few: what a row costs each thread apart from its features (about a hundred: the
// sums across lanes, the ring, the statistics) is shared by 32 features, and the arithmetic is done two numbers at a time.
// 51200 rows of 1024 in bf16, forward and VJP: eight features a thread with loads into registers 216 us, fetched ahead 177, 32
// features a thread 142, two numbers at a time 94 (36 + 58; the bytes take 80 at copy rate).  A tail of 12801 rows of 1000 in fp16
// takes 26 + 38 us (its bytes 35).  Rows that begin anywhere cost more, as the pieces at their ends go element by element and are
// copied for both of their rows (400000 rows in bf16: 96 features 32 + 51 us, 100 features 51 + 95).
#pragma once
#include "prior_common.cuh"

#include <type_traits>

namespace gleam {
namespace prior {

using True = std::true_type;
using False = std::false_type;

constexpr int ROW_BLOCK = 256, ROW_BLOCK_MOST = 512;     // threads a block: of teams inside a warp, and at most (one long row)
// Features a thread: 32 in a team inside a warp, 16 where warps share a row.  There the latency of a row's steps counts, and twice
// the warps on an SM hide it (2049 rows of 4096 and 4099 in float32, forward and VJP: 13.1 + 25.2 and 19.6 + 31.6 us; with 32
// features a thread 12.9 + 28.9 and 27.2 + 55.2).
constexpr int row_features(int team) { return team ? 32 : 16; }
// Threads that the registers of an SM are shared by.  A VJP of long rows has 96 registers, so that two blocks of nine warps fit, which
// rows of 4096 features that begin anywhere need (VJP of the rows above with 128 registers, for two blocks of eight warps: 24.2 for
// 4096 features, 38.4 us for 4099).
constexpr int row_block(bool vjp, int team) { return team ? ROW_BLOCK : vjp ? 608 : ROW_BLOCK_MOST; }
template <class T, int TEAM> constexpr int ROW_ITEMS = row_features(TEAM) / VEC<T>;     // pieces a thread

__device__ __forceinline__ void team_barrier(int team, int threads) { asm volatile("bar.sync %0, %1;" ::"r"(team + 1), "r"(threads) : "memory"); }
__device__ __forceinline__ void copy16(uint32_t to, const void* from) { asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory"); }
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT> __device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }

// s / n for a whole n with inv = 1 / n: the product, corrected by its residual (exact where the quotient is representable).
__device__ __forceinline__ float quotient(float s, float n, float inv) {
    const float q = s * inv, r = fmaf(-q, n, s);
    return r == r ? fmaf(r, inv, q) : q;
}
// 1 / sqrt(x) with one Newton step on the approximation.
__device__ __forceinline__ float inverse_root(float x) {
    const float r = rsqrtf(x), e = fmaf(-x * r, r, 1.f);
    return e == e ? fmaf(0.5f * r, e, r) : r;
}

// Where a thread stands: its team (in the block and in the grid), its place in it, and its features.  Each warp of a team has
// neighbouring pieces, so that only the first and the last one meet the ends of the row; the others are `full` and check nothing.
template <class T, int TEAM, bool EDGES>
struct RowPlace {
    static constexpr int V = VEC<T>, ITEMS = ROW_ITEMS<T, TEAM>, STEP = TEAM ? TEAM : 32;
    int width, team, t, phase;           // threads of a team, team in the block, thread in the team, where its rows begin in a piece
    int first_piece, first;              // the thread's first piece and the feature that it begins with
    bool full;
    long long row, rows_apart, lead;     // lead: from the row of the warp's first team to this one's; its lanes, which shuffle, loop together
    __device__ __forceinline__ RowPlace(const Args& a, int warps, int teams) {
        width = TEAM ? TEAM : warps * 32;
        team = threadIdx.x / width;
        t = threadIdx.x - team * width;
        rows_apart = (long long)gridDim.x * teams;
        if (EDGES) row = blockIdx.x % V + (long long)V * ((long long)(blockIdx.x / V) * teams + team);
        else row = (long long)blockIdx.x * teams + team;
        lead = TEAM ? (EDGES ? V : 1) * ((threadIdx.x & 31) / TEAM) : 0;
        phase = EDGES ? (int)(row % V) * (int)(a.features % V) % V : 0;
        first_piece = TEAM ? t : (t >> 5) * (32 * ITEMS) + (t & 31);
        first = first_piece * V - phase;
        full = __all_sync(0xffffffffu, first >= 0 && feature(ITEMS - 1) + V <= (int)a.features && (!EDGES || a.aligned));
    }
    __device__ __forceinline__ int piece(int k) const { return first_piece + k * STEP; }
    __device__ __forceinline__ int feature(int k) const { return first + k * STEP * V; }
};

// Whether a piece with its first feature at c lies in a row of n, or some of it does.
template <class T, bool FULL, bool EDGES>
__device__ __forceinline__ bool whole(int c, int n) { return FULL || (EDGES ? c >= 0 && c + VEC<T> <= n : c < n); }
template <class T, bool FULL, bool EDGES>
__device__ __forceinline__ bool partly(int c, int n) { return !FULL && EDGES && c < n && c + VEC<T> > 0; }

template <class T, bool FULL, bool EDGES>
__device__ __forceinline__ void store_piece(T* at, int c, int n, bool packed, const Pack<T>& p) {
    if (whole<T, FULL, EDGES>(c, n) && (FULL || !EDGES || packed)) {
        store_pack(at, p);
    } else if (partly<T, FULL, EDGES>(c, n)) {
#pragma unroll
        for (int j = 0; j < VEC<T>; ++j)
            if ((unsigned)(c + j) < (unsigned)n) at[j] = p.e[j];
    }
}
// The numbers of a piece; those beyond the row become 0.
template <class T, bool FULL, bool EDGES>
__device__ __forceinline__ void only_inside(int c, int n, Two (&v)[VEC<T> / 2]) {
    if (whole<T, FULL, EDGES>(c, n)) return;
#pragma unroll
    for (int j = 0; j < VEC<T>; j += 2)
        v[j / 2] = Two(EDGES && (unsigned)(c + j) < (unsigned)n ? v[j / 2].lo() : 0.f, EDGES && (unsigned)(c + j + 1) < (unsigned)n ? v[j / 2].hi() : 0.f);
}
template <class T, bool FULL, bool EDGES>
__device__ __forceinline__ void take(const Pack<T>& p, int c, int n, Two (&v)[VEC<T> / 2]) {
    unpack(p, v);
    only_inside<T, FULL, EDGES>(c, n, v);
}

template <int TEAM>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = (TEAM && TEAM < 32 ? TEAM : 32) / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// A vector of the weights as the pieces hold it, in shared memory; the quarters of the pieces lie one behind another (no bank
// conflicts).  The threads of a block fill it together, eight loads each at a time (one at a time, filling took longer than the
// rows of a small call: 2049 rows of 4096, 15 us).
template <class T, int TEAM, bool EDGES>
struct Weights {
    static constexpr int V = VEC<T>;
    const ulonglong2* shared;
    int pieces;
    template <class Place>
    __device__ __forceinline__ Weights(const void* w, const Args& a, float missing, const Place& at, float* room)
        : shared(reinterpret_cast<const ulonglong2*>(room)), pieces(at.width * Place::ITEMS) {
        const int n = (int)a.features, threads = (int)blockDim.x;
        for (int i0 = threadIdx.x; i0 < pieces * V; i0 += 8 * threads) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int c = i0 + u * threads - at.phase;
                v[u] = (unsigned)c >= (unsigned)n ? 0.f : w ? weight_at<T>(w, a.weight_f32, c) : missing;
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int i = i0 + u * threads;
                if (i < pieces * V) room[((i % V) / 4 * pieces + i / V) * 4 + i % 4] = v[u];
            }
        }
    }
    __device__ __forceinline__ void get(int piece, Two (&v)[V / 2]) const {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
            const ulonglong2 f = shared[q * pieces + piece];
            v[2 * q].bits = f.x; v[2 * q + 1].bits = f.y;
        }
    }
};

// What the warps of a team exchange: four numbers each, in two sets that take turns, so that one barrier is enough.
struct Exchange {
    float4* at; int warps, warp, team, turn;
    __device__ __forceinline__ Exchange(float* shared, int warps_, int team_, int t) : warps(warps_), warp(t >> 5), team(team_), turn(0) {
        at = reinterpret_cast<float4*>(shared) + team_ * 2 * warps_;
    }
    __device__ __forceinline__ const float4* put(float4 v, int t) {
        float4* set = at + turn * warps;
        if ((t & 31) == 0) set[warp] = v;
        team_barrier(team, warps * 32);
        turn ^= 1;
        return set;
    }
};
constexpr int EXCHANGE_BYTES = 2 * ROW_BLOCK_MOST / 32 * sizeof(float4);

// A thread's pieces of the rows to come, in shared memory: copied there by the thread itself, STAGES - 1 rows ahead, and read
// by it alone, so that no barrier is needed.  (Rows of 1024 in bf16, forward and VJP, teams of four warps: 216 us with loads into
// registers, 177 with the ring.)
template <class T, int TEAM, int ARRAYS, int STAGES, bool EDGES>
struct Ring {
    static constexpr int ITEMS = ROW_ITEMS<T, TEAM>;
    Pack<T>* base;                       // the warps' shares lie one behind another, their threads' pieces a warp's width apart
    uint32_t address;
    __device__ __forceinline__ explicit Ring(void* shared) {
        base = static_cast<Pack<T>*>(shared) + (threadIdx.x >> 5) * (STAGES * ARRAYS * ITEMS * 32) + (threadIdx.x & 31);
        address = (uint32_t)__cvta_generic_to_shared(base);
    }
    static __device__ __forceinline__ int place(int stage, int array, int k) { return ((stage * ARRAYS + array) * ITEMS + k) * 32; }
    __device__ __forceinline__ Pack<T> get(int stage, int array, int k) const { return base[place(stage, array, k)]; }
    // The pieces of row r of an array.  A piece over the row's ends is copied whole, with its neighbours' elements, where the
    // array has them.
    template <bool FULL, class Place>
    __device__ __forceinline__ void fetch(int stage, int array, const void* from, long long pitch, long long r, const Place& at, const Args& a) {
        const int n = (int)a.features;
        const T* mine = static_cast<const T*>(from) + (r * pitch + at.first);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            const T* p = mine + k * Place::STEP * VEC<T>;
            if (whole<T, FULL, EDGES>(c, n) && (FULL || !EDGES || a.aligned)) {
                copy16(address + 16u * place(stage, array, k), p);
            } else if (whole<T, FULL, EDGES>(c, n) || partly<T, FULL, EDGES>(c, n)) {
                if (a.aligned && r * pitch + c >= 0 && r * pitch + c + VEC<T> <= (a.outer - 1) * pitch + n) {
                    copy16(address + 16u * place(stage, array, k), p);
                } else {
                    Pack<T> v;
#pragma unroll
                    for (int j = 0; j < VEC<T>; ++j) v.e[j] = (unsigned)(c + j) < (unsigned)n ? p[j] : from_float<T>(0.f);
                    base[place(stage, array, k)] = v;
                }
            }
        }
    }
};

// Blocks of row_block() threads on an SM (registers), and rows in the ring: four, or as many as the shared memory holds beside
// the weights; two where warps share a row, for two blocks.
constexpr int row_blocks(bool vjp, int team) { return team ? (vjp ? 1 : 3) : vjp ? 1 : 2; }
constexpr int row_stages(bool vjp, bool tail, int size, int team) {
    const int stage = ROW_BLOCK * row_features(team) * size * ((vjp ? 2 : 1) + tail), room = 192 * 1024 / row_blocks(vjp, team);
    return !team ? 2 : room / stage >= 4 ? 4 : room / stage >= 3 ? 3 : 2;
}

template <class T, int TEAM, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(row_block(false, TEAM), row_blocks(false, TEAM)) row_team_forward(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    constexpr int V = VEC<T>, ITEMS = ROW_ITEMS<T, TEAM>, STAGES = row_stages(false, TAIL, sizeof(T), TEAM), ARRAYS = TAIL ? 2 : 1;
    using Place = RowPlace<T, TEAM, EDGES>;
    const Place at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    float* room = shared + EXCHANGE_BYTES / 4;
    Ring<T, TEAM, ARRAYS, STAGES, EDGES> ring(room);
    room += ARRAYS * ITEMS * STAGES * 4 * blockDim.x;
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned;
    const float count = (float)n, inv_count = 1.f / count;
    auto fetch = [&](auto full, long long r, int stage) {
        constexpr bool FULL = decltype(full)::value;
        if (r < a.outer) {
            ring.template fetch<FULL>(stage, 0, a.x, a.px, r, at, a);
            if (TAIL) ring.template fetch<FULL>(stage, 1, a.res, a.pres, r, at, a);
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(False{}, at.row + i * at.rows_apart, i);
    const Weights<T, TEAM, EDGES> weight(a.weight, a, 1.f, at, room), bias(a.bias, a, 0.f, at, room + at.width * ITEMS * V);
    __syncthreads();
    float here = 0.f;                              // features of the row that this warp has
    if (!TEAM) {
        int mine = 0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) mine += max(0, min(at.feature(k) + V, n) - max(at.feature(k), 0));
        here = (float)__reduce_add_sync(0xffffffffu, mine);
    }
    const float inv_here = here > 0.f ? 1.f / here : 0.f;
    int stage = 0;
    auto one_row = [&](auto full, long long r) {
        constexpr bool FULL = decltype(full)::value;
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        fetch(full, r + (STAGES - 1) * at.rows_apart, stage == 0 ? STAGES - 1 : stage - 1);
        copies_wait<STAGES - 1>();
        Two v[ITEMS][V / 2];
        T* sum = TAIL ? static_cast<T*>(a.out2) + (r * a.pout2 + at.first) : nullptr;
        const uint64_t counter = TAIL ? mask.counter((uint64_t)((r * n - at.phase) >> 2) + (uint32_t)(at.first_piece * (V / 4))) : 0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            unpack(ring.get(stage, 0, k), v[k]);
            if (TAIL) {
                Two rs[V / 2];
                unpack(ring.get(stage, 1, k), rs);
                if (a.dropping) mask.apply<true, true>(counter + (uint32_t)(k * Place::STEP * (V / 4)), v[k], rs);
                else mask.apply<true, false>(0, v[k], rs);
                const Pack<T> stored = pack<T>(v[k]);
                unpack(stored, v[k]);
                if (live) store_piece<T, FULL, EDGES>(sum + k * Place::STEP * V, c, n, packed, stored);
            }
            only_inside<T, FULL, EDGES>(c, n, v[k]);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        Two pair(0.f);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V / 2; ++j) pair = pair + v[k][j];
        float s = lanes_sum<TEAM>(pair.sum());
        auto deviations = [&](float m) {
            Two q(0.f);
            const Two less(-m);
#pragma unroll
            for (int k = 0; k < ITEMS; ++k) {
                const int c = at.feature(k);
                Two d[V / 2];
#pragma unroll
                for (int j = 0; j < V / 2; ++j) d[j] = v[k][j] + less;
                only_inside<T, FULL, EDGES>(c, n, d);
#pragma unroll
                for (int j = 0; j < V / 2; ++j) q = fma2(d[j], d[j], q);
            }
            return lanes_sum<TEAM>(q.sum());
        };
        float mean, q;
        if (TEAM) {
            mean = quotient(s, count, inv_count);
            q = deviations(mean);
        } else {
            // every warp's mean m_w and squared deviations from it; the sum of (d + m_w - m)^2 is that of d^2 and n_w (m_w - m)^2
            const float mw = s * inv_here;
            const float4* set = exchange.put(make_float4(s, deviations(mw), mw, here), at.t);
            s = q = 0.f;
            for (int u = 0; u < warps; ++u) s += set[u].x;
            mean = quotient(s, count, inv_count);
            for (int u = 0; u < warps; ++u) { const float4 f = set[u]; const float d = f.z - mean; q += fmaf(f.w * d, d, f.y); }
        }
        const float rstd = inverse_root(q * inv_count + a.eps);
        if (!live) return;
        T* y = static_cast<T*>(a.out) + (r * a.pout + at.first);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            Two w[V / 2], b[V / 2];
            weight.get(at.piece(k), w);
            bias.get(at.piece(k), b);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) v[k][j] = fma2((v[k][j] + Two(-mean)) * Two(rstd), w[j], b[j]);
            store_piece<T, FULL, EDGES>(y + k * Place::STEP * V, at.feature(k), n, packed, pack<T>(v[k]));
        }
        if (at.t == 0) {
            if (a.mean) a.mean[r] = mean;
            if (a.rstd) a.rstd[r] = rstd;
        }
    };
    if (at.full) for (long long r = at.row; r - at.lead < a.outer; r += at.rows_apart) one_row(True{}, r);
    else for (long long r = at.row; r - at.lead < a.outer; r += at.rows_apart) one_row(False{}, r);
}

template <class T, int TEAM, bool EDGES, bool TAIL>
__global__ void __launch_bounds__(row_block(true, TEAM), row_blocks(true, TEAM)) row_team_vjp(const __grid_constant__ Args a, int warps, int teams) {
    grid_dependency_wait();
    extern __shared__ __align__(16) float shared[];
    constexpr int V = VEC<T>, ITEMS = ROW_ITEMS<T, TEAM>, STAGES = row_stages(true, TAIL, sizeof(T), TEAM), ARRAYS = TAIL ? 3 : 2;
    using Place = RowPlace<T, TEAM, EDGES>;
    const Place at(a, warps, teams);
    Exchange exchange(shared, warps, at.team, at.t);
    float* room = shared + EXCHANGE_BYTES / 4;
    Ring<T, TEAM, ARRAYS, STAGES, EDGES> ring(room);
    room += ARRAYS * ITEMS * STAGES * 4 * blockDim.x;
    const Mask mask(a);
    const int n = (int)a.features;
    const bool packed = a.aligned, added = TAIL && a.gsum;
    const float inv_count = 1.f / (float)n;
    auto fetch = [&](auto full, long long r, int stage) {
        constexpr bool FULL = decltype(full)::value;
        if (r < a.outer) {
            ring.template fetch<FULL>(stage, 0, a.x, a.px, r, at, a);
            ring.template fetch<FULL>(stage, 1, a.res, a.pres, r, at, a);
            if (added) ring.template fetch<FULL>(stage, 2, a.gsum, a.pgsum, r, at, a);
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) fetch(False{}, at.row + i * at.rows_apart, i);
    float mean_next = 0.f, rstd_next = 0.f;
    if (at.row < a.outer) { mean_next = a.mean[at.row]; rstd_next = a.rstd[at.row]; }
    const Weights<T, TEAM, EDGES> weight(a.weight, a, 1.f, at, room);
    __syncthreads();
    Two gw[ITEMS][V / 2], gb[ITEMS][V / 2];
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < V / 2; ++j) gw[k][j] = gb[k][j] = Two(0.f);
    int stage = 0;
    auto one_row = [&](auto full, long long r) {
        constexpr bool FULL = decltype(full)::value;
        const bool live = !TEAM || TEAM == 32 || r < a.outer;
        fetch(full, r + (STAGES - 1) * at.rows_apart, stage == 0 ? STAGES - 1 : stage - 1);
        const float mean = mean_next, rstd = rstd_next;
        if (r + at.rows_apart < a.outer) { mean_next = a.mean[r + at.rows_apart]; rstd_next = a.rstd[r + at.rows_apart]; }
        copies_wait<STAGES - 1>();
        const int used = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
        Two p1(0.f), p2(0.f);
        const Two less(-mean), root(rstd);
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            if (!live || !(whole<T, FULL, EDGES>(c, n) || partly<T, FULL, EDGES>(c, n))) continue;
            Two g[V / 2], v[V / 2], w[V / 2];
            take<T, FULL, EDGES>(ring.get(used, 0, k), c, n, g);
            take<T, FULL, EDGES>(ring.get(used, 1, k), c, n, v);
            weight.get(at.piece(k), w);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) {
                // beyond the row g is 0
                const Two h = (v[j] + less) * root, d = g[j] * w[j];
                gw[k][j] = fma2(g[j], h, gw[k][j]);
                gb[k][j] = gb[k][j] + g[j];
                p1 = p1 + d;
                p2 = fma2(d, h, p2);
            }
        }
        float s1 = lanes_sum<TEAM>(p1.sum()), s2 = lanes_sum<TEAM>(p2.sum());
        if (!TEAM) {
            const float4* set = exchange.put(make_float4(s1, s2, 0.f, 0.f), at.t);
            s1 = s2 = 0.f;
            for (int u = 0; u < warps; ++u) { s1 += set[u].x; s2 += set[u].y; }
        }
        if (!live) return;
        // rstd (g w - mean(g w) - h mean(g w h))
        const float c1 = -rstd * (s1 * inv_count), c2 = -rstd * (s2 * inv_count);
        T* out = static_cast<T*>(a.out) + (r * a.pout + at.first);
        T* out2 = TAIL ? static_cast<T*>(a.out2) + (r * a.pout2 + at.first) : nullptr;
        const uint64_t counter = TAIL ? mask.counter((uint64_t)((r * n - at.phase) >> 2) + (uint32_t)(at.first_piece * (V / 4))) : 0;
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int c = at.feature(k);
            Two g[V / 2], v[V / 2], w[V / 2];
            unpack(ring.get(used, 0, k), g);
            unpack(ring.get(used, 1, k), v);
            weight.get(at.piece(k), w);
#pragma unroll
            for (int j = 0; j < V / 2; ++j) v[j] = fma2((v[j] + less) * root, Two(c2), fma2(g[j] * w[j], root, Two(c1)));
            if (TAIL) {
                if (added) {
                    unpack(ring.get(used, 2, k), g);
#pragma unroll
                    for (int j = 0; j < V / 2; ++j) v[j] = v[j] + g[j];
                }
                store_piece<T, FULL, EDGES>(out2 + k * Place::STEP * V, c, n, packed, pack<T>(v));
                if (a.dropping) mask.apply<false, true>(counter + (uint32_t)(k * Place::STEP * (V / 4)), v, v);
            }
            store_piece<T, FULL, EDGES>(out + k * Place::STEP * V, c, n, packed, pack<T>(v));
        }
    };
    if (at.full) for (long long r = at.row; r - at.lead < a.outer; r += at.rows_apart) one_row(True{}, r);
    else for (long long r = at.row; r - at.lead < a.outer; r += at.rows_apart) one_row(False{}, r);
    if (!a.gw && !a.gb) return;
    auto half = [](Two v, int j) { return j % 2 ? v.hi() : v.lo(); };
    auto put = [&](int c, int which, float v) {
        if ((unsigned)c >= (unsigned)n) return;
        if (gridDim.x > 1) a.part[((long long)blockIdx.x * 2 + which) * n + c] = v;
        else if (which ? a.gb : a.gw) store_weight_grad<T>(which ? a.gb : a.gw, a.weight_f32, c, v);
    };
    if (teams == 1) {
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) { put(at.feature(k) + j, 0, half(gw[k][j / 2], j)); put(at.feature(k) + j, 1, half(gb[k][j / 2], j)); }
        return;
    }
    __syncthreads();
    float* total = shared;
    // the teams' features are the same ones: every team leaves its sums, then each thread adds up those of some features
    const int mine = 2 * ITEMS * V * at.width;
#pragma unroll
    for (int k = 0; k < ITEMS; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            total[at.team * mine + (2 * (k * V + j)) * at.width + at.t] = half(gw[k][j / 2], j);
            total[at.team * mine + (2 * (k * V + j) + 1) * at.width + at.t] = half(gb[k][j / 2], j);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < mine; i += blockDim.x) {
        float s = 0.f;
#pragma unroll 8
        for (int u = 0; u < teams; ++u) s += total[u * mine + i];
        const int slot = i / at.width, t = i - slot * at.width, which = slot & 1, k = (slot >> 1) / V, j = (slot >> 1) % V;
        const int piece = (TEAM ? t : (t >> 5) * (32 * ITEMS) + (t & 31)) + k * Place::STEP;
        put(piece * V - at.phase + j, which, s);
    }
}

}  // namespace prior
}  // namespace gleam
