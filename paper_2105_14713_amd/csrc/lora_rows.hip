// Low-rank adapters beside a pruned fully connected layer: the products of one
// batch's rows with both factors of their adapters.
//
//   u[i][j] = s_l sum_c x[i][c] W1[l][j][c],   l = ids[i]
//   y[i][o] = base[i][o] + sum_j u[i][j] W2[l][j][o]
//
// (forward: W1, W2 = A, B; backward, on dy: W1, W2 = B, A, u = g, y = dx).
//
// Memory bound: x, base and y move once, the factors once per tile of rows from
// L2; r multiplies and adds per element of x and y are few for the matrix
// cores.  So one kernel does both products, and u never leaves the workgroup
// but where the caller keeps it.
//
// A workgroup has up to TM = 16 * NT rows of one adapter:
//  1. narrow product: the waves split the m columns; 16 bytes of x and of W1 are
//     a lane's operand as they lie (both contract along contiguous memory), but
//     the matrix instructions want neighbouring lanes to hold different rows,
//     and such a load takes 62 cycles of the CU's address unit, one lane each
//     (measured: 16.3k cycles for 256 KB).  So four lanes load 64 bytes of one
//     row, and a 4 KB corner of LDS per wave hands them to the lanes that
//     multiply them.  The waves' sums meet in LDS, in wave order.
//  2. wide product: u is the left operand, in registers for the whole pass; a
//     wave takes 16 * V columns at a time: V rows of W2, 16 bytes a lane, turned
//     in registers (v_perm) into V operands of V consecutive contraction
//     entries, so that the result's lane holds V consecutive columns: base and y
//     move as 16 bytes a lane, 256 consecutive bytes a row.
//     A bf16 layer's u enters in three bf16 planes side by side along the
//     contraction, all of it: a bf16 y may be a small difference of base and
//     update, and two planes (2^-15 of u) then show in it.  Against two: 175.3
//     us for 172.8 on 16384 rows, 4096 -> 8192, r = 64; 38.9 for 38.8 on 8192
//     rows of 4096, r = 8; one row of 2048 5.05 for 4.85.
//
// Ranks are padded to 16 * RT: u is 0 there and W2's last row is read again.  A
// lane whose 16 bytes would pass the end of a row takes the row's last 16
// instead and uses (or stores) those that are its own, so no load is guarded;
// layers of fewer columns than that take lora_rows_small.
#include "lora.h"

namespace onexn {
namespace {

constexpr int kGatherRows = 4096, kGatherAdapters = 1024;   // what lora_rows_gather counts

// The adapters among a workgroup's rows, one after the other: lane i holds row
// i's; `rows` is a mask of those of adapter l (none: l < 0).
struct Adapters {
    int32_t mine, l;
    uint64_t left, rows;
    __device__ Adapters(int32_t mine_, int32_t count) : mine(mine_), left(~0ull >> (64 - count)) { next(); }
    __device__ void next() {
        if (!left) return;
        l = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        rows = __ballot(mine == l) & left;
        left &= ~rows;
    }
};

struct OneAdapter {
    int32_t l;
    uint64_t rows;
    static constexpr uint64_t left = 0;
    __device__ OneAdapter(int32_t l_, int32_t count) : l(l_), rows(~0ull >> (64 - count)) {}
    __device__ void next() {}
};

// A workgroup's rows: those at an index below `count` exist, the others' places
// hold one of them again.  at() is where a row of an array starts: a uniform
// address and 32 bits a lane for consecutive rows.
struct RunRows {      // consecutive
    typedef Adapters Which;
    int32_t first_row, count;
    __device__ int32_t row(int i) const { return first_row + min(i, count - 1); }
    template <typename E> __device__ E* at(E* p, int64_t stride, int i) const {
        return p + first_row * stride + uint32_t(min(i, count - 1) * int32_t(stride));
    }
};
struct ListRows {     // gathered, all of one adapter
    typedef OneAdapter Which;
    const int32_t* rows;
    int32_t count;
    __device__ int32_t row(int i) const { return rows[i]; }
    template <typename E> __device__ E* at(E* p, int64_t stride, int i) const { return p + rows[i] * stride; }
};
constexpr int64_t kRunStride = INT32_MAX / 64;   // row strides that RunRows takes (64 rows at most)

// V elements of a row of base or y as they lie.
template <typename TY, int V> struct RowPart {
    static constexpr int H = V * sizeof(TY) / 16, VY = 16 / sizeof(TY);
    u32x4 w[H];
    __device__ void load(const TY* p) {
#pragma unroll
        for (int h = 0; h < H; ++h) w[h] = load16(p + h * VY);
    }
    __device__ float at(int e) const {
        if constexpr (sizeof(TY) == 4) return __uint_as_float(w[e / 4][e % 4]);
        else return __uint_as_float(e % 2 ? w[0][e / 2] & 0xffff0000u : w[0][e / 2] << 16);
    }
};

// Stores elements `skip` .. V - 1 (0 for nearly all lanes, V for those past the row).
template <typename TY, int V>
__device__ __forceinline__ void store_row(TY* p, int32_t skip, const float (&v)[V]) {
    constexpr int VY = 16 / sizeof(TY);
    if (skip == 0) {
#pragma unroll
        for (int h = 0; h < V / VY; ++h) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                w[k] = sizeof(TY) == 4 ? __float_as_uint(v[h * VY + k % VY])
                                       : round_pair(v[h * VY + (2 * k) % VY], v[h * VY + (2 * k + 1) % VY]);
            __builtin_nontemporal_store(typename Bytes16<TY>::type(w),
                                        reinterpret_cast<typename Bytes16<TY>::type*>(p + h * VY));
        }
        return;
    }
#pragma unroll
    for (int e = 1; e < V; ++e)
        if (e >= skip) p[e] = from_f32<TY>(v[e]);
}

// The same value, which the compiler takes for another: what is computed from it
// is not computed, and held in registers, ahead of a loop.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// A barrier that orders LDS only: loads from memory stay on their way across it.
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The part of a pass's u that belongs to adapter l: its rows of sU.
template <typename T, int RT, int NT, int W, typename Rows>
__device__ __forceinline__ void narrow_product(const LoraRowsArgs& a, const Rows rows, const int32_t l,
                                               const int lane, float* sPart, u32x4* sTurn) {
    constexpr int V = Mat<T>::V, KB = 4 * V, PITCH = 16 * RT + 4, TM = 16 * NT;
    constexpr int GC = 4 * KB;                   // columns of four steps
    constexpr int U = RT + NT <= 3 ? 2 : 1;      // times four of them at once
    const int wave = threadIdx.x / 64, n16 = lane % 16, q = lane / 16;
    const T* const w1 = static_cast<const T*>(a.W1) + int64_t(l) * a.r * a.m;
    const T* const x = static_cast<const T*>(a.x);
    // Load j of four: row 4 * (lane / 4 % 4) + j, 16 bytes lane % 4 of segment lane / 16.
    const int row0 = lane / 4 % 4 * 4, piece = lane % 4;
    // Lanes read what others of their wave wrote.  The unit takes a wave's accesses
    // in the program's order, so nothing is waited for; and the compiler keeps that
    // order, as it cannot know that a lane's reads and writes lie apart.  (A wave
    // barrier holds loads from memory back too: fp32, 8192 rows of 2048, r = 16,
    // 42.5 us for 39.1.)
    u32x4* const turn = sTurn + wave * 256;
    const u32x4* const turned_at = turn + opaque(0);
    auto turned = [&](const u32x4 (&in)[4], u32x4 (&out)[4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) turn[piece * 64 + q * 16 + ((row0 + j) ^ piece)] = in[j];
#pragma unroll
        for (int s = 0; s < 4; ++s) out[s] = turned_at[s * 64 + q * 16 + (n16 ^ s)];
    };
    f32x4 acc[RT][NT] = {};
    auto products = [&](const u32x4 (&wv)[RT][4], const u32x4 (&xv)[NT][4]) {
        u32x4 xt[NT][4];
#pragma unroll
        for (int t = 0; t < NT; ++t) turned(xv[t], xt[t]);
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            u32x4 wt[4];
            turned(wv[i], wt);
#pragma unroll
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[i][t] = Mat<T>::mma(wt[s], xt[t][s], acc[i][t]);
        }
    };
    auto load = [&](int32_t col, u32x4 (&wv)[RT][4], u32x4 (&xv)[NT][4]) {
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                wv[t][j] = load16(w1 + uint32_t(min(t * 16 + row0 + j, a.r - 1) * a.m + col));
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) xv[t][j] = load16(rows.at(x, a.x_stride, t * 16 + row0 + j) + col);
    };
    const int32_t groups = (a.m + GC - 1) / GC, share = (groups + W - 1) / W;
    int32_t g = wave * share;
    const int32_t end = min(g + share, groups), whole = min(end, a.m / GC);
    for (; g + U <= whole; g += U) {
        u32x4 wv[U][RT][4], xv[U][NT][4];
#pragma unroll
        for (int k = 0; k < U; ++k) load((g + k) * GC + (q * 4 + piece) * V, wv[k], xv[k]);
#pragma unroll
        for (int k = 0; k < U; ++k) products(wv[k], xv[k]);
    }
    for (; g < end; ++g) {       // what is left, the last one perhaps cut short
        const int32_t own = g * GC + (q * 4 + piece) * V, col = min(own, a.m - V);
        u32x4 wv[RT][4], xv[NT][4];
        load(col, wv, xv);
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) wv[t][j] = without_first<T>(wv[t][j], own - col);
        products(wv, xv);
    }
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int t = 0; t < NT; ++t)
            *reinterpret_cast<f32x4*>(sPart + (wave * TM + t * 16 + n16) * PITCH + i * 16 + q * 4) = acc[i][t];
}

template <typename T, typename TY, int RT, int NT, int W, typename Rows>
__device__ __forceinline__ void rows_pass(const LoraRowsArgs& a, const Rows rows, const int32_t adapter,
                                          const int32_t chunk0, const int32_t chunk1) {
    constexpr int V = Mat<T>::V, KB = 4 * V, RP = 16 * RT, PITCH = RP + 4, TM = 16 * NT;
    constexpr int P = sizeof(T) == 4 ? 1 : kPlanes;                   // planes of u
    constexpr int KS = (P * RP + KB - 1) / KB;                        // steps of the wide product
    constexpr int SETS = RP < KB ? 1 : RP / KB;                       // different operands of W2 among them
    __shared__ float sPart[W * TM * PITCH], sU[TM * PITCH];
    __shared__ u32x4 sTurn[W * 256];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n16 = lane % 16, q = lane / 16;
    typedef typename Rows::Which Which;
    const Which first(adapter, rows.count);

    u32x4 w[V];
    RowPart<TY, V> part[NT][4];
    auto column_of = [&](int32_t ch) { return min((ch * 16 + opaque(n16)) * V, a.n - V); };
    auto load_w = [&](int32_t l, int32_t ch, int set) {
        const int q = opaque(lane / 16);
        const T* const w2 = static_cast<const T*>(a.W2) + int64_t(l) * a.r * a.n;
        const int32_t col = column_of(ch);
        const int j0 = (set * KB + q * V) % RP;
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = load16(w2 + uint32_t(min(j0 + e, a.r - 1) * a.n + col));
    };
    auto load_base = [&](int32_t ch) {
        const int q = opaque(lane / 16);
        const int32_t col = column_of(ch);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[t][i].load(rows.at(static_cast<const TY*>(a.base), a.base_stride, t * 16 + q * 4 + i) + col);
    };
    auto sum = [&](int32_t l, uint64_t mask) {
        const float scale = l >= 0 && a.scale ? a.scale[l] : 1.f;
        if (l >= 0) lds_barrier();
        for (int e = threadIdx.x; e < TM * RP; e += W * 64) {
            const int i = e / RP, j = e % RP;
            if (!(mask >> i & 1)) continue;
            float s = 0;
            if (l >= 0 && j < a.r) {
#pragma unroll
                for (int k = 0; k < W; ++k) s += sPart[(k * TM + i) * PITCH + j];
                s *= scale;
            }
            sU[i * PITCH + j] = s;
            if (a.u && blockIdx.y == 0 && j < a.r) a.u[int64_t(rows.row(i)) * a.r + j] = s;
        }
        lds_barrier();
    };
    int32_t ch = chunk0 + wave;
    Which at = first;
    for (;;) {
        if (at.l >= 0) narrow_product<T, RT, NT, W>(a, rows, at.l, opaque(lane), sPart, sTurn);
        if (!at.left) break;
        sum(at.l, at.rows);
        at.next();
    }
    // The first chunk's operands are on their way while the last sums meet.
    if (a.y && ch < chunk1) {
        if (first.l >= 0) load_w(first.l, ch, 0);
        if (a.base) load_base(ch);
    }
    sum(at.l, at.rows);
    if (!a.y) return;
    u32x4 uf[KS][NT];
#pragma unroll
    for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int slot = s * KB + q * V, plane = slot / RP;
            const float* src = sU + (t * 16 + n16) * PITCH + slot % RP;
            if constexpr (sizeof(T) == 4) {
                uf[s][t] = *reinterpret_cast<const u32x4*>(src);
            } else {
                float v[8];
                u32x4 p[P];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = src[e];
                cut_planes(v, p);
                uf[s][t] = plane == 0 ? p[0] : plane == 1 ? p[1] : plane < P ? p[P - 1] : u32x4{0, 0, 0, 0};
            }
        }
    const bool in_place = a.y == a.base && a.y_stride == a.base_stride;
    const float none = a.base ? -0.f : 0.f;      // what changes no base, -0 neither
    for (; ch < chunk1; ch += W) {
        const int32_t col = column_of(ch), skip = min((ch * 16 + n16) * V - col, V);
        at = first;
        for (;;) {
            const int32_t l = at.l, next_ch = at.left ? ch : ch + W;
            const uint64_t now = at.rows;
            const bool last = !at.left;
            if (last) at = first;
            else at.next();
            f32x4 acc[NT][V];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[t][i] = l >= 0 ? f32x4{0, 0, 0, 0} : f32x4{none, none, none, none};
            if (l >= 0) {
#pragma unroll
                for (int set = 0; set < SETS; ++set) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const u32x4 wc = Mat<T>::column(w, i);
#pragma unroll
                        for (int s = set; s < KS; s += SETS)
#pragma unroll
                            for (int t = 0; t < NT; ++t) acc[t][i] = Mat<T>::mma(uf[s][t], wc, acc[t][i]);
                    }
                    if (set + 1 < SETS) load_w(l, ch, set + 1);
                }
            }
            if (at.l >= 0 && next_ch < chunk1) load_w(at.l, next_ch, 0);
            if (l >= 0 || !in_place) {
                const int q = opaque(lane / 16);
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int k = t * 16 + q * 4 + i;
                        float v[V];
#pragma unroll
                        for (int e = 0; e < V; ++e) v[e] = a.base ? part[t][i].at(e) + acc[t][e][i] : acc[t][e][i];
                        if (now >> k & 1)
                            store_row<TY, V>(rows.at(static_cast<TY*>(a.y), a.y_stride, k) + col, skip, v);
                    }
            }
            if (last) break;
        }
        if (a.base && ch + W < chunk1) load_base(ch + W);
    }
}

// Column chunks (16 * V columns) of this workgroup's part of the wide product.
__device__ __forceinline__ void chunk_range(const LoraRowsArgs& a, int32_t per, int32_t& c0, int32_t& c1) {
    const int32_t chunks = (a.n + per - 1) / per;
    c0 = int32_t(int64_t(chunks) * blockIdx.y / gridDim.y);
    c1 = int32_t(int64_t(chunks) * (blockIdx.y + 1) / gridDim.y);
}

__device__ __forceinline__ int32_t adapter_of(const LoraRowsArgs& a, int32_t row) {
    const int32_t l = a.ids[row];
    return l >= 0 && l < a.L ? l : -1;
}

// TM consecutive rows.
template <typename T, typename TY, int RT, int NT, int W>
__global__ void __launch_bounds__(W * 64, NT == 1 && RT == 1 ? 4 : NT == 1 && RT == 2 ? 3 : 2) lora_rows_run(const LoraRowsArgs a) {
    constexpr int TM = 16 * NT;
    const int lane = threadIdx.x % 64;
    int32_t c0, c1;
    chunk_range(a, 16 * Mat<T>::V, c0, c1);
    const int32_t first_row = blockIdx.x * TM;
    const RunRows rows{first_row, min(TM, a.rows - first_row)};
    rows_pass<T, TY, RT, NT, W>(a, rows, adapter_of(a, rows.row(lane)), c0, c1);
}

// Rows in any order, not too many of them: each adapter's rows are cut into tiles
// of TM, and a workgroup finds the tile that has its number: up to 64 rows by
// going through the adapters among them, else by counting every adapter's rows.
// Where there are too many adapters to count, a workgroup looks at the row that
// has its number, and takes the tile that begins with it if one does.
template <typename T, typename TY, int RT, int NT, int W>
__global__ void __launch_bounds__(W * 64, RT <= 2 ? 3 : 2) lora_rows_gather(const LoraRowsArgs a) {
    constexpr int TM = 16 * NT, THREADS = W * 64, STEPS = kGatherRows / THREADS, PER = kGatherAdapters / THREADS;
    __shared__ int32_t sCount[kGatherAdapters], sWave[STEPS * W], sRows[TM], sPick[3], sMine;
    static_assert(STEPS * W == 64, "a lane for each 64 rows");
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int32_t me = blockIdx.x;
    int32_t l = -1, count = 0;                 // my tile's adapter (L: none) and rows
    if (a.rows <= 64) {                        // every wave by itself: a row a lane
        int32_t slot = -1;
        if (lane < a.rows) {
            slot = adapter_of(a, lane);
            slot = slot < 0 ? a.L : slot;
        }
        int32_t ahead = 0;
        for (uint64_t left = ~0ull >> (64 - a.rows); left;) {
            const int32_t now = __builtin_amdgcn_readlane(slot, __builtin_ctzll(left));
            const uint64_t match = __ballot(slot == now);
            const int32_t tiles = (__popcll(match) + TM - 1) / TM;
            left &= ~match;
            if (me < ahead + tiles) {
                const int32_t from = (me - ahead) * TM, at = __popcll(match & ((1ull << lane) - 1)) - from;
                l = now;
                count = min(int32_t(__popcll(match)) - from, TM);
                if (wave == 0 && slot == now && at >= 0 && at < TM) sRows[at] = lane;
                break;
            }
            ahead += tiles;
        }
        if (l < 0) return;
    } else {
        int32_t slot[STEPS];                   // each row's adapter; L: none; -1: no row
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int32_t i = s * THREADS + threadIdx.x;
            slot[s] = -1;
            if (i < a.rows) {
                slot[s] = adapter_of(a, i);
                slot[s] = slot[s] < 0 ? a.L : slot[s];
            }
        }
        int32_t from = 0;                      // rows of the adapter ahead of my tile
        if (a.L < kGatherAdapters) {
#pragma unroll
            for (int k = 0; k < PER; ++k) sCount[k * THREADS + threadIdx.x] = 0;
            if (threadIdx.x == 0) sPick[0] = -1;
            __syncthreads();
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if (s * THREADS >= a.rows) break;
                // (The wave's first adapter, often the only one, is counted at once.)
                const int32_t lead = __builtin_amdgcn_readfirstlane(slot[s]);
                const uint64_t same = __ballot(slot[s] == lead);
                if (lead >= 0 && lane == 0) atomicAdd(&sCount[lead], __popcll(same));
                if (slot[s] >= 0 && slot[s] != lead) atomicAdd(&sCount[slot[s]], 1);
            }
            __syncthreads();
            // Tiles ahead of each thread's PER adapters.
            int32_t tiles[PER], sum = 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                tiles[k] = (sCount[threadIdx.x * PER + k] + TM - 1) / TM;
                sum += tiles[k];
            }
            int32_t upto = sum;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int32_t v = __shfl_up(upto, d);
                if (lane >= d) upto += v;
            }
            if (lane == 63) sWave[wave] = upto;
            __syncthreads();
            int32_t ahead = upto - sum;
#pragma unroll
            for (int w = 0; w < W; ++w) ahead += w < wave ? sWave[w] : 0;
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (me >= ahead && me < ahead + tiles[k]) {
                    sPick[0] = threadIdx.x * PER + k;
                    sPick[1] = (me - ahead) * TM;
                    sPick[2] = sCount[threadIdx.x * PER + k];
                }
                ahead += tiles[k];
            }
            __syncthreads();
            l = __builtin_amdgcn_readfirstlane(sPick[0]);
            if (l < 0) return;
            from = sPick[1];
            count = sPick[2];
        } else {
            l = adapter_of(a, me);
            l = l < 0 ? a.L : l;
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const uint64_t match = __ballot(slot[s] == l);
            if (lane == 0) sWave[s * W + wave] = __popcll(match);
            if (lane == me % 64 && s * W + wave == me / 64) sMine = __popcll(match & ((1ull << lane) - 1));
        }
        __syncthreads();
        if (a.L >= kGatherAdapters) {
            count = sWave[lane];
            from = lane < me / 64 ? count : 0;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) {
                count += __shfl_xor(count, d);
                from += __shfl_xor(from, d);
            }
            from += sMine;
            if (from % TM != 0) return;
        }
        count = __builtin_amdgcn_readfirstlane(min(count - from, TM));
        int32_t rank = -from;                  // of the rows ahead, counted from the tile's first
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (s * THREADS >= a.rows) break;
            const uint64_t match = __ballot(slot[s] == l);
            int32_t at = rank;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const int32_t v = sWave[s * W + w];
                at += w < wave ? v : 0;
                rank += v;
            }
            at += __popcll(match & ((1ull << lane) - 1));
            if (slot[s] == l && at >= 0 && at < TM) sRows[at] = s * THREADS + threadIdx.x;
        }
    }
    __syncthreads();
    if (threadIdx.x >= count && threadIdx.x < TM) sRows[threadIdx.x] = sRows[0];
    __syncthreads();
    int32_t c0, c1;
    chunk_range(a, 16 * Mat<T>::V, c0, c1);
    const ListRows rows{sRows, count};
    rows_pass<T, TY, RT, NT, W>(a, rows, l < a.L ? l : -1, c0, c1);
}

// Any size: one row a workgroup, one product a wave, one column a thread.
template <typename T, typename TY>
__global__ void __launch_bounds__(kThreads) lora_rows_small(const LoraRowsArgs a) {
    __shared__ float u[kMaxRank];
    const int32_t wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    for (int32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int32_t l = adapter_of(a, row);
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        for (int32_t j = wave; j < a.r; j += kThreads / 64) {
            float s = 0;
            if (l >= 0) {
                const T* w = static_cast<const T*>(a.W1) + (int64_t(l) * a.r + j) * a.m;
                for (int32_t c = lane; c < a.m; c += 64) s = fmaf(to_f32(x[c]), to_f32(w[c]), s);
#pragma unroll
                for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
                if (a.scale) s *= a.scale[l];
            }
            if (lane == 0) {
                u[j] = s;
                if (a.u) a.u[int64_t(row) * a.r + j] = s;
            }
        }
        __syncthreads();
        for (int32_t o = threadIdx.x; a.y && o < a.n; o += kThreads) {
            float s = l < 0 && a.base ? -0.f : 0.f;     // (as in rows_pass)
            if (l >= 0) {
                const T* w = static_cast<const T*>(a.W2) + int64_t(l) * a.r * a.n + o;
                for (int32_t j = 0; j < a.r; ++j) s = fmaf(u[j], to_f32(w[int64_t(j) * a.n]), s);
            }
            if (a.base) s += to_f32(static_cast<const TY*>(a.base)[row * a.base_stride + o]);
            static_cast<TY*>(a.y)[row * a.y_stride + o] = from_f32<TY>(s);
        }
        __syncthreads();
    }
}

constexpr int kWaves = 8;

// Workgroups for all CUs where there are few tiles: the wide product's columns
// are split, down to two chunks each (powers of two share them evenly), and
// every part does the narrow product again.
dim3 rows_grid(const LoraRowsArgs& a, int32_t tiles, int32_t cols) {
    const int32_t chunks = a.y ? (a.n + cols - 1) / cols : 1;
    int32_t split = 1;
    while (2 * split * tiles <= 256 && 4 * split <= chunks + 1) split *= 2;
    return dim3(tiles, split);
}

template <typename T, typename TY, int RT, int NT, int W>
void launch_run(const LoraRowsArgs& a, hipStream_t s) {
    const dim3 grid = rows_grid(a, (a.rows + 16 * NT - 1) / (16 * NT), 16 * Mat<T>::V);
    hipLaunchKernelGGL((lora_rows_run<T, TY, RT, NT, W>), grid, dim3(W * 64), 0, s, a);
}

template <typename T, typename TY, int RT>
void launch(const LoraRowsArgs& a, hipStream_t s) {
    if (a.L > 1 && a.rows > 1 && a.rows <= kGatherRows) {
        // The most tiles there can be: L adapters and that of none have one more each.
        const int32_t parts = a.rows < a.L + 1 ? a.rows : a.L + 1;
        const int32_t tiles = a.rows > 64 && a.L >= kGatherAdapters ? a.rows : parts + (a.rows - parts) / 16;
        hipLaunchKernelGGL((lora_rows_gather<T, TY, RT, 1, kWaves>), rows_grid(a, tiles, 16 * Mat<T>::V),
                           dim3(kWaves * 64), 0, s, a);
        return;
    }
    // Tiles of 32 rows read the factors half as often, which counts from rank 33
    // on where there is a tile for every CU (16384 rows, 4096 -> 8192, r = 64: 175
    // us against 195; r = 16, 8192 rows: 44 against 43).  Above rank 64 one tile of 16
    // takes all 256 registers already.
    if constexpr (RT == 4)
        if (a.rows >= 8192) return launch_run<T, TY, RT, 2, kWaves>(a, s);
    // Narrow layers have no work for eight waves in either product, and where tiles
    // wait for a CU, workgroups of four come in sooner: from 4097 rows on four waves
    // are as fast or faster at every rank (64 to 512 columns; 8192 rows of 256, r =
    // 16: 5.6 us against 6.0, r = 128: 10.7 and 14.7; 20000 rows 7.8 and 10.8), up to
    // 4096 rows as fast or slower (r = 128: up to 4 %).  Wider: 8192 rows of 256 ->
    // 1024, 9.1 and 8.3.
    if (a.rows > 16 * 256 && a.m <= 4 * 16 * Mat<T>::V && a.n <= 4 * 16 * Mat<T>::V)
        return launch_run<T, TY, RT, 1, 4>(a, s);
    launch_run<T, TY, RT, 1, kWaves>(a, s);
}

template <typename T, typename TY>
void launch_rank(const LoraRowsArgs& a, hipStream_t s) {
    const int64_t far = a.x_stride > a.base_stride ? a.x_stride : a.base_stride;
    if (a.m < Mat<T>::V || a.n < Mat<T>::V || far > kRunStride || a.y_stride > kRunStride)
        hipLaunchKernelGGL((lora_rows_small<T, TY>), dim3(a.rows < (1 << 20) ? a.rows : 1 << 20), dim3(kThreads), 0, s, a);
    else if (a.r <= 16) launch<T, TY, 1>(a, s);
    else if (a.r <= 32) launch<T, TY, 2>(a, s);
    else if (a.r <= 64) launch<T, TY, 4>(a, s);
    else launch<T, TY, 8>(a, s);
}

}  // namespace

void launch_lora_rows(const LoraRowsArgs& a, onexn_dtype xdt, onexn_dtype ydt, hipStream_t s) {
    if (xdt == ONEXN_F32) launch_rank<float, float>(a, s);
    else if (ydt == ONEXN_F32) launch_rank<uint16_t, float>(a, s);
    else launch_rank<uint16_t, uint16_t>(a, s);
}

}  // namespace onexn
