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
// consecutive tokens).  A cut is found from a histogram in the LDS (counts and sums, 8 bins per octave): the bin that holds it, then, if
// that has more than LIST weights, bins of a 64th of it; what is left is ranked by comparing all with all.  Rows of up to LIST tokens
// are ranked at once.  The token is found by the running sum in the order of the indices.
//
// What bounds it: long rows the loads, of which a workgroup of two rows takes 16 bytes of every line, and the vector ALU in turn (8192 tokens, 4096 rows as 2048
// slots, top-k and top-p: 207 us for 268 MB, 144 without filters); shorter ones the histogram's atomics and the meetings of the wavefronts (1000
// tokens, 4096 rows, all filters: 49 us, 22 without); few rows and short ones latency (5003 tokens, 37 rows, top-p and min-p: 28 us, 19 without; ten tokens, 2048
// rows: 6.3 us, with the exponentials of eight tokens per thread, which any n takes).
#include <math.h>

#include <algorithm>

#include "he_internal.h"

namespace {

constexpr int ONE_BITS = 47;
constexpr u64 ONE = 1ull << ONE_BITS;
constexpr u32 BINS = 384;        // 8 per octave of weights 1 .. 2^47
constexpr u32 SUB_BITS = 6, SUB_BINS = 1 << SUB_BITS;
constexpr u32 LIST = 128;        // weights that are ranked by comparing all with all
constexpr u32 MAX_ROWS = 8;      // rows of a workgroup

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

// A range of weights, base .. base + 2^bits - 1, and what lies above it.
struct Bin {
    u64 base, above_sum, sum;
    u32 bits, above_count, count;
};

// The cut of a row: tokens above `value`, and the first `ties` of those of that weight.
struct Cut {
    u64 value;
    u32 ties;
    u64 above_sum;
};

template <u32 T>
struct Shared {
    static constexpr u32 WAVES = T / 64;
    u64 sums[2][WAVES][MAX_ROWS];
    u32 counts[2][WAVES][MAX_ROWS];
    Bin found[MAX_ROWS];
    Cut cut[MAX_ROWS];
    u32 listed[MAX_ROWS];
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

// A workgroup's histograms and lists: entry b of a row at [b * rows + row].
struct Tables {
    u64 *sums, *sub_sums, *list;
    u32 *counts, *sub_counts;
    __device__ Tables(u64* lds, u32 rows) {
        sums = lds;
        list = sub_sums = sums + BINS * rows;  // (the list takes the place of the finer histogram)
        counts = reinterpret_cast<u32*>(sub_sums + LIST * rows);
        sub_counts = counts + BINS * rows;
    }
    static size_t bytes(u32 rows) { return (size_t)rows * ((BINS + LIST) * sizeof(u64) + (BINS + SUB_BINS) * sizeof(u32)); }
};
static_assert(SUB_BINS <= LIST, "");

__device__ __forceinline__ void count_into(u64* sum, u32* count, u64 w) {
    atomicAdd((unsigned long long*)sum, (unsigned long long)w);
    atomicAdd(count, 1u);
}

template <u32 T, int PER>
__device__ __forceinline__ void octave_histogram(Row<T>& row, const u64 (&w)[PER], const Tables& t) {
    for (u32 b = threadIdx.x; b < BINS * row.rows; b += T) t.sums[b] = 0, t.counts[b] = 0;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (w[i]) {
            const u32 e = 63 - __builtin_clzll(w[i]);
            const u32 bin = (e * 8 + (u32)((w[i] << (63 - e)) >> 60 & 7)) * row.rows + row.row;
            count_into(&t.sums[bin], &t.counts[bin], w[i]);
        }
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
}

// Of the bins (the highest first) the one in which the count, or the sum, reaches `target`, into row.sh.found.
template <bool BY_SUM, u32 T>
__device__ __forceinline__ void find_bin(Row<T>& row, const u64* sums, const u32* counts, u32 n_bins, u64 target, bool active, const Bin& within) {
    const u32 each = (n_bins + row.threads - 1) / row.threads, first = row.rank * each, last = min(first + each, n_bins);
    u64 sum = 0, before, total;
    u32 count = 0, count_before, count_total;
    for (u32 k = first; k < last; k++) {
        sum += sums[(n_bins - 1 - k) * row.rows + row.row];
        count += counts[(n_bins - 1 - k) * row.rows + row.row];
    }
    row.scan(sum, count, before, total, count_before, count_total);
    before += within.above_sum;
    count_before += within.above_count;
    const u64 reached = BY_SUM ? before : count_before;
    if (active && reached < target && target <= reached + (BY_SUM ? sum : count)) {
        for (u32 k = first; k < last; k++) {
            const u32 bin = n_bins - 1 - k;
            const u64 s = sums[bin * row.rows + row.row];
            const u32 c = counts[bin * row.rows + row.row];
            if (target <= (BY_SUM ? before + s : (u64)count_before + c)) {
                Bin f;
                if (n_bins == BINS) {
                    const u32 e = bin / 8;
                    f.bits = e >= 3 ? e - 3 : 0;
                    f.base = e >= 3 ? (u64)(8 + bin % 8) << (e - 3) : (8 + bin % 8) >> (3 - e);
                } else {
                    f.bits = within.bits > SUB_BITS ? within.bits - SUB_BITS : 0;
                    f.base = within.base + ((u64)bin << f.bits);
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
}

// For the rows with `active`: the cut at which the count (BY_SUM: the sum of the weights) in descending order reaches `target`,
// 1 <= target <= what the row has.
template <bool BY_SUM, u32 T, int PER>
__device__ __forceinline__ void find_cut(Row<T>& row, const u64 (&w)[PER], u32 n, u64 target, bool active, const Tables& t, Cut& cut) {
    if (!__syncthreads_or(active)) return;
    Bin in{1, 0, 0, 63, 0, n};  // all weights but zero
    if (n > LIST) {
        find_bin<BY_SUM>(row, t.sums, t.counts, BINS, target, active, in);
        if (active) in = row.sh.found[row.row];
        while (true) {
            const bool finer = active && in.count > LIST && in.bits > 0;
            if (!__syncthreads_or(finer)) break;
            for (u32 b = threadIdx.x; b < SUB_BINS * row.rows; b += T) t.sub_sums[b] = 0, t.sub_counts[b] = 0;
            __syncthreads();
            if (finer) {
                const u32 shift = in.bits > SUB_BITS ? in.bits - SUB_BITS : 0;
#pragma unroll
                for (int i = 0; i < PER; i++) {
                    if (w[i] - in.base < (1ull << in.bits)) {  // (wraps below base)
                        const u32 bin = (u32)((w[i] - in.base) >> shift) * row.rows + row.row;
                        count_into(&t.sub_sums[bin], &t.sub_counts[bin], w[i]);
                    }
                    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
            __syncthreads();
            find_bin<BY_SUM>(row, t.sub_sums, t.sub_counts, SUB_BINS, target, finer, in);
            if (finer) in = row.sh.found[row.row];
        }
    }
    // the weights of the range, compared with one another; where they are all the same there is nothing to compare
    const bool ranked = active && in.bits > 0;
    if (row.rank == 0) row.sh.listed[row.row] = 0;
    __syncthreads();
    if (ranked) {
#pragma unroll
        for (int i = 0; i < PER; i++) {
            if (w[i] - in.base < (1ull << in.bits)) t.list[atomicAdd(&row.sh.listed[row.row], 1u) * row.rows + row.row] = w[i];
            if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
        }
    }
    __syncthreads();
    if (ranked) {
        const u32 count = row.sh.listed[row.row];
        for (u32 i = row.rank; i < count; i += row.threads) {
            const u64 v = t.list[i * row.rows + row.row];
            u64 sum = in.above_sum;
            u32 above = in.above_count, same = 0;
            for (u32 k = 0; k < count; k++) {
                const u64 y = t.list[k * row.rows + row.row];
                sum += y > v ? y : 0;
                above += y > v;
                same += y == v;
            }
            const u64 reached = BY_SUM ? sum : above;
            if (reached < target && target <= reached + (BY_SUM ? same * v : same))
                row.sh.cut[row.row] = Cut{v, (u32)(BY_SUM ? (target - sum + v - 1) / v : target - above), sum};
        }
    }
    __syncthreads();
    if (active) {
        cut = ranked ? row.sh.cut[row.row]
                     : Cut{in.base, (u32)(BY_SUM ? (target - in.above_sum + in.base - 1) / in.base : target - in.above_count), in.above_sum};
    }
}

template <u32 T, int PER>
__global__ void __launch_bounds__(T, 4) sample_kernel(SampleArgs a) {
    __shared__ Shared<T> sh;
    extern __shared__ u64 lds[];
    Row<T> row(sh, a.rows_log);
    // Workgroups go to the eight XCDs round-robin; neighbouring rows, which may share cache lines, run on one of them.
    const u32 tiles = (a.rows + row.rows - 1) >> a.rows_log, per_xcd = (tiles + 7) / 8;
    const u32 tile = blockIdx.x % 8 * per_xcd + blockIdx.x / 8;
    if (tile >= tiles) return;
    const u32 r = (tile << a.rows_log) + row.row, at = min(r, a.rows - 1);
    const double* col = a.slots + (a.parts == 2 ? at : 2 * (size_t)at);
    const u32 token0 = row.rank * a.per;
    const int mine = (int)min(a.n, token0 + a.per) - (int)token0;  // this thread's tokens (none: not above zero)
    u64 w[PER];
    const double* first = col + min(token0, a.n - 1) * a.stride;
    const int last = max(mine - 1, 0);
#pragma unroll
    for (int i = 0; i < PER; i++) {  // (past the end the last one again)
        w[i] = __builtin_bit_cast(u64, first[(u32)min(i, last) * (u32)a.stride]);
        if (i % 8 == 7) __builtin_amdgcn_sched_barrier(0);
    }
    double top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        if (i >= mine) w[i] = __builtin_bit_cast(u64, (double)-INFINITY);
        top = fmax(top, __builtin_bit_cast(double, w[i]));  // (NaN never wins)
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    top = row.max(top);
    const double t = a.temperature ? a.temperature[at] : 1.0;
    const bool greedy = !(t > 0), none = top == -INFINITY;
    const double inv = 1.0 / t;
    u64 sum = 0, unused, total;
    u32 some = 0, unused_count, count;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        const double x = __builtin_bit_cast(double, w[i]);
        // 2^5 has the weight as its mantissa's last 47 bits: one addition rounds it to a whole number
        const double e = greedy ? 0.0 : exp((x - top) * inv);
        w[i] = none ? 0 : x == top ? ONE : e > 0 ? __builtin_bit_cast(u64, e + 32.0) - __builtin_bit_cast(u64, 32.0) : 0;  // (NaN: 0)
        sum += w[i];
        some += w[i] != 0;
        if (i % 2) __builtin_amdgcn_sched_barrier(0);  // (two at a time: the temporaries of all would not fit the registers)
    }
    Cut cut{0, 0, 0};
    if (a.top_k || a.top_p) {
        const Tables tables(lds, row.rows);
        row.scan(sum, some, unused, total, unused_count, count);
        if (a.n > LIST) octave_histogram(row, w, tables);
        if (a.top_k) {
            const u32 k = a.top_k[at];
            const bool active = k != 0 && k < count && !greedy && !none;
            find_cut<false>(row, w, a.n, k, active, tables, cut);
            if (active) total = cut.above_sum + cut.ties * cut.value;
        }
        if (a.top_p) {
            const double p = a.top_p[at], need = ceil((double)total * p);
            const u64 target = need >= 1 ? min((u64)need, total) : 1;
            find_cut<true>(row, w, a.n, target, p < 1 && !greedy && !none, tables, cut);
        }
    }
    if (a.min_p && !greedy) {
        const double least = ceil(a.min_p[at] * (double)ONE);
        const u64 value = least >= (double)ONE ? ONE : least >= 1 ? (u64)least : 0;  // (the largest weight always stays)
        if (value > cut.value) cut = Cut{value - 1, 0, 0};
    }
    // the kept weights in the order of the indices: those above the cut, and of those at it the first cut.ties
    u64 before;
    u32 ties = 0, ties_before;
    sum = 0;
#pragma unroll
    for (int i = 0; i < PER; i++) {
        sum += w[i] > cut.value ? w[i] : 0;
        ties += w[i] == cut.value;
    }
    row.scan(sum, ties, before, total, ties_before, count);
    before += min(ties_before, cut.ties) * cut.value;
    total += min(count, cut.ties) * cut.value;
    const u32 free = cut.ties > ties_before ? cut.ties - ties_before : 0;  // of this thread's ties the first so many are kept
    sum += min(ties, free) * cut.value;
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
        asm volatile("" : "+v"(cut.value));  // (the comparisons above are not kept for this)
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
    static std::atomic<uint32_t> allowed{0};
    const int rc = allow_dynamic_lds((const void*)sample_kernel<T, PER>, Tables::bytes(MAX_ROWS), device, allowed);
    if (rc != HE_OK) return rc;
    hipLaunchKernelGGL((sample_kernel<T, PER>), dim3((tiles + 7) / 8 * 8), dim3(T), a.top_k || a.top_p ? Tables::bytes(rows) : 0, s, a);
    HE_HIP(hipGetLastError());
    return HE_OK;
}

template <u32 T>
int launch_threads(const SampleArgs& a, int device, hipStream_t s) {  // (a.per is at most 32)
    return a.per <= 8 ? launch<T, 8>(a, device, s) : a.per <= 16 ? launch<T, 16>(a, device, s) : launch<T, 32>(a, device, s);
}

}  // namespace

int launch_sample(he_ctx* ctx, const double* slots, u32 n, u32 n_slots, u32 parts, const double* temperature, const u32* top_k, const double* top_p,
                  const double* min_p, const double* uniform, int32_t* tokens, double* log_prob, hipStream_t s) {
    SampleArgs a{slots, temperature, top_p, min_p, uniform, top_k, tokens, log_prob, (size_t)ctx->N, n, n_slots * parts, parts, 3, 0};
    // Eight rows, which are a cache line (real parts) or half of one, as far as the registers hold them and there are rows enough for every compute
    // unit.  A workgroup is no larger than it must be, so that one loads while another searches.  Its threads take 16 tokens each up to n = 2048 and 32
    // beyond, where fewer rows would leave too little of a line (4096 rows, top-k and top-p: n = 2048 74 us, 97 with 32; n = 2049 98, 109 with 16; n = 8192
    // 238, 286 with 16; from 1025 to 2048 tokens 16 were as fast or faster at every number of rows from 256 to 4096, by up to 43 %; between 2049 and 4096
    // anything from 24 % faster to 11 % slower).  Rows beyond 16384 tokens need 1024 threads, whose registers leave one workgroup to a compute unit and three of a
    // thread's weights in scratch memory (512 rows, top-k and top-p: n = 16384 87 us, n = 16385 160, n = 32768 205).
    // Where few rows leave compute units idle, a thread takes eight.
    const u32 most = n > 2048 ? 32 : 16, widest = n > 512 * 32 ? 1024 : 512;
    while (a.rows_log > 0 && ((widest >> a.rows_log) * most < n || (a.rows >> a.rows_log) < 256)) a.rows_log--;
    const bool few = (a.rows >> a.rows_log) < 256;
    u32 T = 256;
    while (T < (few ? 1024 : widest) && (T >> a.rows_log) * (few ? 8 : most) < n) T *= 2;
    const u32 threads = T >> a.rows_log;
    a.per = (n + threads - 1) / threads;
    return T == 256 ? launch_threads<256>(a, ctx->device, s) : T == 512 ? launch_threads<512>(a, ctx->device, s) : launch_threads<1024>(a, ctx->device, s);
}
