// Gradients of the adapters' factors:
//
//   dW[l][j][c] = sum over the rows i of adapter l of u[i][j] v[i][c]
//
// (dA: u = g, v = x; dB: u, v = dy), both factors in one launch.
//
// Memory bound: v is read once, 16 bytes a lane; u comes from L2.  A workgroup
// has 16 * V columns, up to 64 ranks, one adapter and a range of rows.  It
// lists the adapter's rows of the range in LDS, 2048 rows at a time, and its
// waves take the list's blocks of 4 * V rows in turn: whole blocks whatever the
// order of the rows, and no row of another adapter is read.  A block's V rows
// a lane are turned in registers into operands that contract over rows, as the
// factors are in the wide product.  A bf16 layer's u enters as three bf16
// planes, which hold it exactly: the sums are as exact as in fp32.  The waves'
// sums meet in LDS, the ranges' in a second launch, both in a fixed order.
#include "lora.h"

namespace onexn {
namespace {

constexpr int kWaves = 8, kList = 2048, kMostRanks = 64;     // ranks of a workgroup at most

struct Job {
    const float* u;      // [rows][r]
    const void* v;       // [rows][C]
    float* out;          // [splits][L][r][C] (splits > 1: partial sums)
    int64_t v_stride;
    int32_t C, chunks;
};

struct GradArgs {
    Job job[2];
    const int32_t* ids;
    int32_t* present;    // [splits][L]: whether the range has rows of the adapter
    int32_t rows, r, L, range;
};

template <typename T, int RT>
__global__ void __launch_bounds__(kWaves * 64) lora_grad(const GradArgs a) {
    constexpr int V = Mat<T>::V, KB = 4 * V, COLS = 16 * V, P = sizeof(T) == 4 ? 1 : kPlanes;
    constexpr int THREADS = kWaves * 64, STEPS = kList / THREADS;
    __shared__ float sPart[kWaves * 16 * COLS];
    __shared__ int32_t sList[kList], sCount[STEPS * kWaves];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n16 = lane % 16, q = lane / 16;
    const bool second = int32_t(blockIdx.x) >= a.job[0].chunks;
    const Job& job = a.job[second];
    const int32_t chunk = blockIdx.x - (second ? a.job[0].chunks : 0);
    const int32_t groups = (a.r + 16 * RT - 1) / (16 * RT);     // of ranks
    const int32_t l = blockIdx.y / groups, j0 = blockIdx.y % groups * 16 * RT;
    const int32_t begin = blockIdx.z * a.range, end = min(begin + a.range, a.rows);
    // (A lane past the end of the row has the row's last columns.)
    const int32_t own = (chunk * 16 + n16) * V, col = min(own, job.C - V);
    const T* v = static_cast<const T*>(job.v) + col;
    f32x4 acc[RT][V] = {};
    int32_t found = 0;
    int32_t next[STEPS];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int32_t i = begin + s * THREADS + threadIdx.x;
        next[s] = i < end ? a.ids[i] : -1;
    }
    for (int32_t at = begin; at < end; at += kList) {
        uint64_t match[STEPS];
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            match[s] = __ballot(next[s] == l);
            if (lane == 0) sCount[s * kWaves + wave] = __popcll(match[s]);
        }
        __syncthreads();             // (and the blocks before have been read)
        int32_t count = 0;
#pragma unroll
        for (int k = 0; k < STEPS * kWaves; ++k) {
            if (k % kWaves == wave && (match[k / kWaves] >> lane & 1))
                sList[count + __popcll(match[k / kWaves] & ((1ull << lane) - 1))] =
                    at + (k / kWaves) * THREADS + threadIdx.x;
            count += sCount[k];
        }
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            const int32_t i = at + kList + s * THREADS + threadIdx.x;
            next[s] = i < end ? a.ids[i] : -1;
        }
        __syncthreads();
        found += count;
        for (int32_t b = wave * KB; b < count; b += kWaves * KB) {
            const int32_t e0 = b + q * V;
            int32_t row[V];
#pragma unroll
            for (int e = 0; e < V; ++e) row[e] = sList[min(e0 + e, count - 1)];
            u32x4 w[V];
            float uv[RT][V];
#pragma unroll
            for (int e = 0; e < V; ++e) w[e] = load16(v + row[e] * job.v_stride);
#pragma unroll
            for (int t = 0; t < RT; ++t)
#pragma unroll
                for (int e = 0; e < V; ++e)
                    uv[t][e] = job.u[int64_t(row[e]) * a.r + min(j0 + t * 16 + n16, a.r - 1)];
            if (b + KB > count) {    // the last block: zeros behind the list
#pragma unroll
                for (int e = 0; e < V; ++e)
                    if (e0 + e >= count) {
                        w[e] = u32x4{0, 0, 0, 0};
#pragma unroll
                        for (int t = 0; t < RT; ++t) uv[t][e] = 0.f;
                    }
            }
            u32x4 uf[RT][P];
#pragma unroll
            for (int t = 0; t < RT; ++t) {
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int e = 0; e < V; ++e) uf[t][0][e] = __float_as_uint(uv[t][e]);
                } else {
                    cut_planes(uv[t], uf[t]);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const u32x4 wc = Mat<T>::column(w, i);
#pragma unroll
                for (int t = 0; t < RT; ++t)
#pragma unroll
                    for (int p = 0; p < P; ++p) acc[t][i] = Mat<T>::mma(uf[t][p], wc, acc[t][i]);
            }
        }
    }
    if (gridDim.z > 1) {
        if (blockIdx.x == 0 && blockIdx.y % groups == 0 && threadIdx.x == 0)
            a.present[int64_t(blockIdx.z) * a.L + l] = found > 0;
        if (!found) return;
    }
    float* out = job.out + (int64_t(blockIdx.z) * a.L + l) * a.r * job.C;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float* const row = sPart + (wave * 16 + q * 4 + k) * COLS;
            if (col == own) {
#pragma unroll
                for (int h = 0; h < V; h += 4)
                    *reinterpret_cast<f32x4*>(row + n16 * V + h) =
                        f32x4{acc[t][h][k], acc[t][h + 1][k], acc[t][h + 2][k], acc[t][h + 3][k]};
            } else {
#pragma unroll
                for (int i = 1; i < V; ++i)
                    if (col + i >= own) row[col + i - chunk * COLS] = acc[t][i][k];
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * COLS; e += THREADS) {
            const int32_t j = j0 + t * 16 + e / COLS, c = chunk * COLS + e % COLS;
            if (j >= a.r || c >= job.C) continue;
            float s = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) s += sPart[w * 16 * COLS + e];
            out[int64_t(j) * job.C + c] = s;
        }
    }
}

// Fewer columns than a lane's 16 bytes hold (job[0] alone): one rank of one adapter
// and a range of rows a workgroup, a row a thread, up to V - 1 sums each, which
// meet in lane, wave and range order (8192 rows of two bf16 columns, rank 16: 11
// us; a thread a column that goes through all rows: 1.1 ms, and one fp32 sum of
// all of them).  Each factor goes by its own width: the other one, 4096 wide, takes
// 39 us with lora_grad.
template <typename T>
__global__ void __launch_bounds__(kWaves * 64) lora_grad_small(const GradArgs a) {
    constexpr int MOST = Mat<T>::V - 1;
    __shared__ float sPart[kWaves][MOST];
    __shared__ int32_t sFound[kWaves];
    const Job& job = a.job[0];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int32_t j = blockIdx.x, l = blockIdx.y;
    const int32_t begin = blockIdx.z * a.range, end = min(begin + a.range, a.rows);
    float s[MOST] = {};
    bool mine = false;
    for (int32_t i = begin + int32_t(threadIdx.x); i < end; i += kWaves * 64) {
        if (a.ids[i] != l) continue;
        mine = true;
        const float u = job.u[int64_t(i) * a.r + j];
        const T* const v = static_cast<const T*>(job.v) + i * job.v_stride;
#pragma unroll
        for (int c = 0; c < MOST; ++c)
            if (c < job.C) s[c] = fmaf(u, to_f32(v[c]), s[c]);
    }
    const uint64_t any = __ballot(mine);
#pragma unroll
    for (int c = 0; c < MOST; ++c) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) s[c] += __shfl_xor(s[c], d);
        if (lane == 0) sPart[wave][c] = s[c];
    }
    if (lane == 0) sFound[wave] = any != 0;
    __syncthreads();
    const int c = threadIdx.x;
    if (c < job.C) {
        float sum = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) sum += sPart[w][c];
        job.out[((int64_t(blockIdx.z) * a.L + l) * a.r + j) * job.C + c] = sum;
    }
    if (gridDim.z > 1 && j == 0 && threadIdx.x == 0) {
        int32_t found = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) found |= sFound[w];
        a.present[int64_t(blockIdx.z) * a.L + l] = found;
    }
}

struct JoinArgs {
    const float* part[2];
    float* dW[2];
    int64_t size[2];     // L * r * C
    int64_t adapter[2];  // r * C
    const int32_t* present;
    int32_t L, splits;
};

__global__ void __launch_bounds__(kThreads) lora_grad_join(const JoinArgs a) {
    int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x;
    const int64_t step = int64_t(gridDim.x) * kThreads, total = a.size[0] + a.size[1];
    for (; i < total; i += step) {
        const bool second = i >= a.size[0];
        const int64_t e = second ? i - a.size[0] : i;
        const float* part = second ? a.part[1] : a.part[0];
        const int64_t size = second ? a.size[1] : a.size[0];
        const int32_t l = a.L == 1 ? 0 : int32_t(e / (second ? a.adapter[1] : a.adapter[0]));
        // (Loads ahead of the flags: a part that was not written is read, and left out.)
        float s = 0;
#pragma unroll 4
        for (int32_t k = 0; k < a.splits; ++k) {
            const float v = part[k * size + e];
            s += a.present[int64_t(k) * a.L + l] ? v : 0.f;
        }
        (second ? a.dW[1] : a.dW[0])[e] = s;
    }
}

// Ranges of rows, a power of two of them, joined by a second launch (2.6 us of the
// host, 2 to 5 of the GPU).  They pay from some 1536 rows of one bf16 adapter at
// ranks up to 16 on, fewer where a row takes longer (higher ranks, fp32) and more
// where adapters share the rows; as many, of 128 rows at least, as give one
// workgroup a CU (three from 10000 rows on).  Not two for several adapters: half of the
// workgroups then have no rows, in blocks that put the others on the same CUs.
// Against the best of 1, 2, 4, 8 and 16 ranges of each of 2084 calls (some 300 layers of
// 2 to 8192 columns, r = 2 to 128, one to 16 adapters in runs of equal and of random
// lengths and in any order, 256 to 16384 rows, both types) this takes 2.5 % longer on
// average and 70 % at most; one range always 22 %, at most seven times as long.  Both
// sides (us): fp32, 16384 rows of 1023 and 2047, r = 24, four adapters of as many rows:
// one range 101, two 155, four 152, eight 113; one adapter, bf16, 4096 such rows: one 48,
// four 27, eight 25, sixteen 32.  A step (forward and backward) called from Python,
// bf16: 1024 rows of 1024, r = 32: one 26.6, four 28.8; 2048 rows: 31.3 and 29.0.
constexpr int kCUs = 256, kSplitRows = 1536, kLongRows = 10000, kRangeRows = 128, kMostRanges = 16;

int32_t splits_of(int32_t rows, int32_t m, int32_t n, int32_t r, int32_t L, onexn_dtype dt) {
    const int32_t cols = 16 * (dt == ONEXN_F32 ? Mat<float>::V : Mat<uint16_t>::V);
    // (A row's cost goes with the root of its ranks and bytes; so does what L adapters share.)
    const int64_t cost = (r <= 16 ? 1 : r <= 32 ? 2 : 4) * (dt == ONEXN_F32 ? 2 : 1);
    if (int64_t(rows) * rows * cost < int64_t(kSplitRows) * kSplitRows * L) return 1;
    const int64_t chunks = (int64_t(m) + cols - 1) / cols + (int64_t(n) + cols - 1) / cols;
    const int64_t groups = chunks * ((r + kMostRanks - 1) / kMostRanks) * L, most = kCUs * (rows >= kLongRows ? 3 : 1);
    int32_t s = 1;
    while (2 * s <= kMostRanges && rows >= 2 * s * kRangeRows && 2 * s * groups <= most) s *= 2;
    return s == 2 && L > 1 ? 4 : s;
}

size_t round16(size_t v) { return (v + 15) / 16 * 16; }

}  // namespace

size_t lora_grad_workspace(int32_t rows, int32_t m, int32_t n, int32_t r, int32_t L) {
    const size_t f32 = splits_of(rows, m, n, r, L, ONEXN_F32), bf16 = splits_of(rows, m, n, r, L, ONEXN_BF16);
    const size_t s = f32 > bf16 ? f32 : bf16;
    return s == 1 ? 0 : round16(s * L * r * (size_t(m) + n) * 4) + round16(s * L * 4);
}

template <typename T>
static void launch_grad(const GradArgs& a, dim3 grid, hipStream_t s) {
    const dim3 block(kWaves * 64);
    if (a.r <= 16) hipLaunchKernelGGL((lora_grad<T, 1>), grid, block, 0, s, a);
    else if (a.r <= 32) hipLaunchKernelGGL((lora_grad<T, 2>), grid, block, 0, s, a);
    else {
        grid.y *= (a.r + kMostRanks - 1) / kMostRanks;
        hipLaunchKernelGGL((lora_grad<T, 4>), grid, block, 0, s, a);
    }
}

void launch_lora_grad(const LoraGradArgs& g, onexn_dtype dt, hipStream_t s) {
    const int32_t cols = 16 * (dt == ONEXN_F32 ? Mat<float>::V : Mat<uint16_t>::V);
    const int32_t splits = splits_of(g.rows, g.m, g.n, g.r, g.L, dt);
    GradArgs a{};
    JoinArgs join{};
    float* part = static_cast<float*>(g.workspace);
    a.ids = g.ids;
    a.rows = g.rows;
    a.r = g.r;
    a.L = g.L;
    a.range = (g.rows + splits - 1) / splits;
    a.present = reinterpret_cast<int32_t*>(static_cast<char*>(g.workspace) +
                                           round16(size_t(splits) * g.L * g.r * (size_t(g.m) + g.n) * 4));
    join.present = a.present;
    join.L = g.L;
    join.splits = splits;
    int wide = 0, joined = 0;
    for (int k = 0; k < 2; ++k) {
        float* dW = k ? g.dB : g.dA;
        if (!dW) continue;
        const int32_t C = k ? g.n : g.m;
        const int64_t size = int64_t(g.L) * g.r * C;
        const Job job{k ? g.u : g.g, k ? g.dy : g.x, splits > 1 ? part : dW, k ? g.dy_stride : g.x_stride, C,
                      (C + cols - 1) / cols};
        if (C >= (dt == ONEXN_F32 ? Mat<float>::V : Mat<uint16_t>::V)) {
            a.job[wide++] = job;
        } else {                         // (a row holds less than a lane's 16 bytes)
            GradArgs narrow = a;
            narrow.job[0] = job;
            const dim3 grid(g.r, g.L, splits), block(kWaves * 64);
            if (dt == ONEXN_F32) hipLaunchKernelGGL(lora_grad_small<float>, grid, block, 0, s, narrow);
            else hipLaunchKernelGGL(lora_grad_small<uint16_t>, grid, block, 0, s, narrow);
        }
        join.part[joined] = part;
        join.dW[joined] = dW;
        join.size[joined] = size;
        join.adapter[joined] = int64_t(g.r) * C;
        part += size * splits;
        ++joined;
    }
    const dim3 grid(a.job[0].chunks + a.job[1].chunks, g.L, splits);
    if (wide && dt == ONEXN_F32) launch_grad<float>(a, grid, s);
    else if (wide) launch_grad<uint16_t>(a, grid, s);
    if (splits > 1) {
        const int64_t blocks = (join.size[0] + join.size[1] + kThreads - 1) / kThreads;
        hipLaunchKernelGGL(lora_grad_join, dim3(uint32_t(blocks < 4096 ? blocks : 4096)), dim3(kThreads), 0, s, join);
    }
}

}  // namespace onexn
