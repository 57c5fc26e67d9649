// Sampling from decoded slots (he_sample_slots): a token per row of logits with temperature, top-k, top-p and min-p, from a
// given uniform number.
//
// Row r of slots [n][N/2][2] is a column: the logits of one slot's real (or imaginary) part, N/2 * 16 bytes apart.  With the
// row's maximum m the tokens' weights are whole numbers, w_v = round(2^47 exp((l_v - m) / T)): sums of up to 2^15 of them are exact in 64
// bits, whatever the order, so that the histograms below may be filled by atomics and a row's answer never changes.  All three filters keep a prefix
// of the tokens in descending order of weight (ties: the lower index first), so they end in one cut (v, r): what is above v,
// and the first r tokens of weight v.
//
// A workgroup reads its rows once and holds the weights in registers, as many threads per row as that takes (a thread up to 32
// consecutive tokens).  A cut is found by histograms in the LDS (counts and sums): 8 bins per octave first, then 256 bins of the
// bin that holds the cut, until that has one element or one value.  The token is found by the running sum in the order
// of the indices.  Bound by the one reading of the logits where there are many rows.
#include <math.h>

#include <algorithm>

#include "he_internal.h"

namespace {

constexpr int ONE_BITS = 47;
constexpr u64 ONE = 1ull << ONE_BITS;
constexpr u32 BINS = 384;        // 8 per octave of weights 1 .. 2^47
constexpr u32 MAX_PER_ROW = 32;  // tokens of a thread
constexpr u32 MAX_ROWS = 16;     // rows of a workgroup

struct SampleArgs {
    const double* slots;
    const double *temperature, *top_p, *min_p, *uniform;
    const u32* top_k;
    int32_t* tokens;
    double* log_prob;
    size_t stride;   // doubles from a token to the next
    u32 n, rows, parts;
    u32 rows_log;    // rows of a workgroup: 2^rows_log
    u32 per;         // tokens of a thread
};

// A bin: weights base .. base + 2^bits - 1
struct Bin {
    u64 base, above_sum, sum;
    u32 bits, above_count, count;
};

template <u32 T>
struct Shared {
    static constexpr u32 WAVES = T / 64;
    u64 sums[2][WAVES][MAX_ROWS];
    u32 counts[2][WAVES][MAX_ROWS];
    Bin found[MAX_ROWS];
};

// A thread's place among the threads of its row; sums over the row in the order of the threads.
template <u32 T>
struct Row {
    Shared<T>& sh;
    u32 rows, lane, wave, row, rank, threads;
    u32 buf = 0;
    __device__ Row(Shared<T>& s, u32 rows_log)
        : sh(s), rows(1u << rows_log), lane(threadIdx.x % 64), wave(threadIdx.x / 64), row(threadIdx.x & (rows - 1)),
          rank((lane >> rows_log) + wave * (64u >> rows_log)), threads(T >> rows_log) {}

    // sums over the threads of the row before this one, and over all of them
    __device__ __forceinline__ void scan(u64 sum, u32 count, u64& before, u64& total, u32& count_before, u32& count_total) {
        u64 s = sum;
        u32 c = count;
        for (u32 d = rows; d < 64; d <<= 1) {
            const u64 s1 = __shfl_up(s, d);
            const u32 c1 = __shfl_up(c, d);
            if (lane >= d) s += s1, c += c1;
        }
        buf ^= 1;
        if (lane >= 64 - rows) sh.sums[buf][wave][row] = s, sh.counts[buf][wave][row] = c;
        __syncthreads();  // (two buffers in turn: whoever passes the next barrier has read this one)
        before = s - sum;
        count_before = c - count;
        total = 0;
        count_total = 0;
        for (u32 w = 0; w < T / 64; w++) {
            const u64 s1 = sh.sums[buf][w][row];
            const u32 c1 = sh.counts[buf][w][row];
            if (w < wave) before += s1, count_before += c1;
            total += s1;
            count_total += c1;
        }
    }

    __device__ __forceinline__ double max(double v) {
        for (u32 d = rows; d < 64; d <<= 1) v = fmax(v, __shfl_xor(v, d));
        buf ^= 1;
        if (lane < rows) sh.sums[buf][wave][row] = __builtin_bit_cast(u64, v);
        __syncthreads();
        for (u32 w = 0; w < T / 64; w++) v = fmax(v, __builtin_bit_cast(double, sh.sums[buf][w][row]));
        return v;
    }
};

// The cut of a row: tokens above `value`, and the first `ties` of those of that weight.
struct Cut {
    u64 value;
    u32 ties;
    u64 above_sum;
};

// For the rows with `active`: the cut at which the count (BY_SUM: the sum of the weights) in descending order reaches `target`,
// 1 <= target <= what the row has.
template <u32 T, int PER, bool BY_SUM>
__device__ __forceinline__ void find_cut(Row<T>& row, const u64 (&w)[PER], u64 target, bool active, u64* bin_sum, u32* bin_count, Cut& cut) {
    u64* sums = bin_sum + row.row;    // bin b of this row: [b * rows]
    u32* counts = bin_count + row.row;
    u64 base = 0;
    u32 bits = 64;                    // 64: the first level, bins of an eighth of an octave
    u64 above_sum = 0;
    u32 above_count = 0;
    while (__syncthreads_or(active)) {
        for (u32 b = threadIdx.x; b < BINS * row.rows; b += T) bin_sum[b] = 0, bin_count[b] = 0;
        __syncthreads();
        const u32 shift = bits == 64 ? 0 : bits > 8 ? bits - 8 : 0;
        if (active) {
#pragma unroll
            for (int i = 0; i < PER; i++) {
                u32 bin;
                bool in;
                if (bits == 64) {
                    const u32 e = 63 - __builtin_clzll(w[i] | 1);
                    bin = e * 8 + (u32)((e >= 3 ? w[i] >> (e - 3) : w[i] << (3 - e)) & 7);
                    in = w[i] != 0;
                } else {
                    bin = (u32)((w[i] - base) >> shift);
                    in = w[i] - base < (1ull << bits);  // (wraps below base)
                }
                if (in) {
                    atomicAdd((unsigned long long*)&sums[bin * row.rows], (unsigned long long)w[i]);
                    atomicAdd(&counts[bin * row.rows], 1u);
                }
                if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
        // a thread takes consecutive bins, the highest first
        const u32 each = (BINS + row.threads - 1) / row.threads, first = row.rank * each;
        u64 sum = 0, before, total;
        u32 count = 0, count_before, count_total;
        for (u32 k = first; k < min(first + each, BINS); k++) {
            sum += sums[(BINS - 1 - k) * row.rows];
            count += counts[(BINS - 1 - k) * row.rows];
        }
        row.scan(sum, count, before, total, count_before, count_total);
        before += above_sum;
        count_before += above_count;
        const u64 reached = BY_SUM ? before : count_before, after = reached + (BY_SUM ? sum : count);
        if (active && reached < target && target <= after) {
            for (u32 k = first; k < min(first + each, BINS); k++) {
                const u32 bin = BINS - 1 - k;
                const u64 s = sums[bin * row.rows];
                const u32 c = counts[bin * row.rows];
                if (target <= (BY_SUM ? before + s : (u64)count_before + c)) {
                    Bin f;
                    if (bits == 64) {
                        const u32 e = bin / 8;
                        f.bits = e >= 3 ? e - 3 : 0;
                        f.base = e >= 3 ? (u64)(8 + bin % 8) << (e - 3) : (8 + bin % 8) >> (3 - e);
                    } else {
                        f.bits = shift;
                        f.base = base + ((u64)bin << shift);
                    }
                    f.above_sum = before;
                    f.above_count = count_before;
                    f.sum = s;
                    f.count = c;
                    row.sh.found[row.row] = f;
                    break;
                }
                before += s;
                count_before += c;
            }
        }
        __syncthreads();
        if (active) {
            const Bin f = row.sh.found[row.row];
            base = f.base;
            bits = f.bits;
            above_sum = f.above_sum;
            above_count = f.above_count;
            if (f.count == 1 || bits == 0) {  // one token, or one weight
                cut.value = f.count == 1 ? f.sum : base;
                cut.ties = (u32)(BY_SUM ? (target - above_sum + cut.value - 1) / cut.value : target - above_count);
                cut.above_sum = above_sum;
                active = false;
            }
        }
    }
}

template <u32 T, int PER>
__global__ void __launch_bounds__(T, 4) sample_kernel(SampleArgs a) {
    __shared__ Shared<T> sh;
    extern __shared__ u64 bins[];  // [BINS][rows] sums, then counts
    Row<T> row(sh, a.rows_log);
    // Workgroups go to the eight XCDs round-robin; neighbouring rows, which may share cache lines, run on one of them.
    const u32 tiles = (a.rows + row.rows - 1) >> a.rows_log, per_xcd = (tiles + 7) / 8;
    const u32 tile = blockIdx.x % 8 * per_xcd + blockIdx.x / 8;
    if (tile >= tiles) return;
    const u32 r = (tile << a.rows_log) + row.row, at = min(r, a.rows - 1);
    const double* col = a.slots + (a.parts == 2 ? at : 2 * (size_t)at);
    const u32 token0 = row.rank * a.per;
    u64 w[PER];
    double top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        double x = -INFINITY;
        if ((u32)i < a.per && token0 + i < a.n) x = col[(token0 + i) * a.stride];
        w[i] = __builtin_bit_cast(u64, x);
    }
#pragma unroll
    for (int i = 0; i < PER; i++) top = fmax(top, __builtin_bit_cast(double, w[i]));  // (fmax: NaN never wins)
    top = row.max(top);
    const double t = a.temperature ? a.temperature[at] : 1.0;
    const bool greedy = !(t > 0), none = top == -INFINITY;
    const double inv = 1.0 / t;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const double x = __builtin_bit_cast(double, w[i]);
        // 2^5 has the weight as its mantissa's last 47 bits: one addition rounds it to a whole number
        const double e = greedy ? 0.0 : exp((x - top) * inv);
        w[i] = none ? 0 : x == top ? ONE : e > 0 ? __builtin_bit_cast(u64, e + 32.0) - __builtin_bit_cast(u64, 32.0) : 0;  // (NaN: 0)
        if (i % 2) __builtin_amdgcn_sched_barrier(0);  // (two at a time: the temporaries of all would not fit the registers)
    }
    u64 unused, total;
    u32 unused_count, count;
    Cut cut{0, 0, 0};
    u64* bin_sum = bins;
    u32* bin_count = reinterpret_cast<u32*>(bins + BINS * row.rows);
    if (a.top_k || a.top_p) {  // the sum of the weights, and how many are not zero
        u64 sum = 0;
        u32 some = 0;
#pragma unroll
        for (int i = 0; i < PER; i++) sum += w[i], some += w[i] != 0;
        row.scan(sum, some, unused, total, unused_count, count);
        if (a.top_k) {
            const u32 k = a.top_k[at];
            const bool active = k != 0 && k < count && !greedy && !none;
            find_cut<T, PER, false>(row, w, k, active, bin_sum, bin_count, cut);
            if (active) total = cut.above_sum + cut.ties * cut.value;
        }
        if (a.top_p) {
            const double p = a.top_p[at], need = ceil((double)total * p);
            const u64 target = need >= 1 ? min((u64)need, total) : 1;
            find_cut<T, PER, true>(row, w, target, p < 1 && !greedy && !none, bin_sum, bin_count, cut);
        }
    }
    if (a.min_p && !greedy) {
        const double least = ceil(a.min_p[at] * (double)ONE);
        const u64 value = least >= (double)ONE ? ONE : least >= 1 ? (u64)least : 0;  // (the largest weight always stays)
        if (value > cut.value) cut = Cut{value - 1, 0, 0};
    }
    // the kept weights in the order of the indices
    u64 sum = 0, before;
    u32 ties = 0, ties_before;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        sum += w[i] > cut.value ? w[i] : 0;
        ties += w[i] == cut.value;
    }
    row.scan(0, ties, unused, unused, ties_before, count);
    const u32 free = cut.ties > ties_before ? cut.ties - ties_before : 0;  // of this thread's ties the first so many are kept
    sum += min(ties, free) * cut.value;
    row.scan(sum, 0, before, total, unused_count, count);
    if (r >= a.rows) return;
    if (none) {
        if (row.rank == 0) {
            a.tokens[r] = -1;
            if (a.log_prob) a.log_prob[r] = -INFINITY;
        }
        return;
    }
    const double u = greedy ? 0.0 : a.uniform[r], place = floor((double)total * u);
    const u64 target = place >= 1 ? min(place < 0x1p63 ? (u64)place : total, total - 1) : 0;
    if (before <= target && target < before + sum) {
        u32 token = 0, left = free;
        u64 run = before;
        bool found = false;
#pragma unroll
        for (int i = 0; i < PER; i++) {
            const bool tie = w[i] == cut.value && left > 0;
            left -= tie;
            run += w[i] > cut.value || tie ? w[i] : 0;
            if (!found && run > target) token = token0 + i, found = true;
        }
        a.tokens[r] = (int32_t)token;
        if (a.log_prob) {
            const double x = col[token * a.stride];
            a.log_prob[r] = greedy ? 0.0 : (x == top ? 0.0 : (x - top) * inv) - log((double)total * 0x1p-47);
        }
    }
}

template <u32 T, int PER>
int launch(const SampleArgs& a, int device, hipStream_t s) {
    const u32 rows = 1u << a.rows_log, tiles = (a.rows + rows - 1) / rows;
    const size_t lds = a.top_k || a.top_p ? (size_t)BINS * rows * (sizeof(u64) + sizeof(u32)) : 0;
    static std::atomic<uint32_t> allowed{0};
    const int rc = allow_dynamic_lds((const void*)sample_kernel<T, PER>, (size_t)BINS * MAX_ROWS * (sizeof(u64) + sizeof(u32)), device, allowed);
    if (rc != HE_OK) return rc;
    hipLaunchKernelGGL((sample_kernel<T, PER>), dim3((tiles + 7) / 8 * 8), dim3(T), lds, s, a);
    HE_HIP(hipGetLastError());
    return HE_OK;
}

}  // namespace

int launch_sample(he_ctx* ctx, const double* slots, u32 n, u32 n_slots, u32 parts, const double* temperature, const u32* top_k, const double* top_p,
                  const double* min_p, const double* uniform, int32_t* tokens, double* log_prob, hipStream_t s) {
    SampleArgs a{slots, temperature, top_p, min_p, uniform, top_k, tokens, log_prob, (size_t)ctx->N, n, n_slots * parts, parts, 4, 0};
    const bool wide = n > 512 * MAX_PER_ROW;
    const u32 T = wide ? 1024 : 512;
    while (a.rows_log > 0 && ((T >> a.rows_log) * MAX_PER_ROW < n || (a.rows >> a.rows_log) < 256)) a.rows_log--;
    const u32 threads = T >> a.rows_log;
    a.per = (n + threads - 1) / threads;
    if (wide) return launch<1024, 32>(a, ctx->device, s);
    if (a.per <= 4) return launch<512, 4>(a, ctx->device, s);
    if (a.per <= 8) return launch<512, 8>(a, ctx->device, s);
    if (a.per <= 16) return launch<512, 16>(a, ctx->device, s);
    return launch<512, 32>(a, ctx->device, s);
}
