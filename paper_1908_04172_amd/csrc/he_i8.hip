// Matrix product of ciphertexts and 8-bit integer weights (he_ct_i8_mac): for every output o of a layer, modulo each limb's q,
//   out[o][c][n] = tok[n] * (s_o * sum_t w_t * x_t[c][n]) + [c = 0] b[o],
// w_t whole numbers in [-128, 127], s_o the channel's scale and tok the tokens' (one per slot, where given).
//
// A weight is one digit, so the eight bytes of a residue need not be spread over sums of their own as for plaintexts of full
// width (he_mac_digits.hip: 64 int8 products per term): with x = sum_d x_d 256^d,
//   sum_t w_t x_t = sum_d 256^d S_d,   S_d = sum_t w_t x_td,
// one int8 product per byte.  Bytes are unsigned and the matrix cores' operands signed: x_d - 128 is the byte with its top bit
// flipped, and what that leaves out, 128 sum_d 256^d sum_t w_t, is a constant of the output.
//
// v_mfma_i32_32x32x32_i8 takes 32 terms times 32 outputs times 32 slots of one digit.  A lane's share of the input operand is one byte of 16
// terms at one slot: it loads the bytes of each of the 16 residues and transposes them in registers (4 x 4 bytes: eight byte
// permutations).  The digits go in two halves, bytes 0 .. ND-1 and ND .. 2 ND-1 (ND = 2, 3 or 4 by the modulus), in one of two forms:
//  - groups of up to 32 outputs (convolutions, narrow layers), with v_mfma_i32_16x16x32_i8 in the same manner: a wavefront takes both halves of 32 slots
//    and runs through several groups, the inputs of the next block of terms in flight; wavefronts never meet;
//  - larger ones: a workgroup shares the operands of 64 slots among four wavefronts, one for each half and 32 outputs, which exchange half of
//    their results at the end.
// Residues in packed storage are taken two at a time as one of eight bytes (first form), or one half alone (second).
//
// The end of an output, two products by constants of the output and one reduction: I8Channel in he_arith.h.
//
// What bounds it: the first form the vector ALU, whose instructions are 30 % transposition and 70 % ends (a 16x16x8 map, 3x3x16, N = 2^13, L = 3,
// with tokens: 842 us for 2.4 GB; a 28x28 image, 5x5x5, L = 4: 206 us for 0.79 GB, 3.8 TB/s); long sums over few groups the inputs' way from memory (845 -> 100 at
// 2^13, L = 4: 122 us for 0.50 GB, 4.0 TB/s; with the rescale 173 us, he_ct_pt_mac 411); many outputs of short sums the ends (256 -> 1000 at 2^12, L = 2:
// 102 us), of long ones the products, transposition and LDS in turn (1024 -> 1024 packed: 117 us, 1.2 int8 POP/s).
// Groups of the second form hold 64 outputs and not 128, whose sums would leave one workgroup per compute unit, with its ends in the open: with 128, the ends as
// they then were, 256 -> 1000 took 1.41 times as long, 845 -> 100 1.13 times, 1024 -> 1024 packed 1.04 times.
#include <string.h>

#include <algorithm>
#include <type_traits>
#include <unordered_map>
#include <unordered_set>

#include "he_internal.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef u32 u32x2 __attribute__((ext_vector_type(2), aligned(8)));

constexpr u32 THREADS = 256;
// Groups that a workgroup of the first form runs through, at most (the 16x16x8 map 845 us, with runs of 8, 4, 2 and 1 829, 858, 908 and 1035), and
// the workgroups that a launch keeps (the 28x28 image 209 us; with 1024 of them 242, with 4096 208, with 8192 229).
constexpr u32 WHOLE_RUN = 16;
constexpr u64 MIN_WORKGROUPS = 2048;

// slots of a workgroup, in units of eight bytes: 32 per wavefront in the first form, 64 in all in the second
template <typename V>
__host__ __device__ constexpr u32 whole_slots() { return THREADS / 2 * 8 / sizeof(V); }
template <typename V>
__host__ __device__ constexpr u32 split_slots() { return 64 * 8 / sizeof(V); }

template <typename V>
struct I8Args {
    const I8Group* groups;
    const u32* lists;
    const v4i* table;
    const I8Channel* channels;  // [limb][n_out]
    const V* ct_in;
    const V* token;             // [limbs][N] or null
    const u64* bias;            // [n_out][limbs] or null
    V* out;
    u32 limbs, N, n_out;
    u32 first, n_groups;        // the class's groups
    u32 run, runs;              // groups of a workgroup, runs of groups
    u32 accumulate;
};

__device__ __forceinline__ I8Group load_group(const I8Group* p) {  // (read-only, the same for the whole workgroup: a scalar load)
    typedef u32 u32x8 __attribute__((ext_vector_type(8)));
    const u32x8 v = *(const __attribute__((address_space(4))) u32x8*)(p);
    return I8Group{v[0], v[1], v[2], v[3], v[4], {0, 0, 0}};
}

// four bytes of four terms -> the same byte of the four terms, for the first ND bytes, as signed digits
template <int ND>
__device__ __forceinline__ void transpose4(u32 a, u32 b, u32 c, u32 d, u32 (&out)[ND]) {
    const u32 lo0 = __builtin_amdgcn_perm(b, a, 0x05010400u), lo1 = __builtin_amdgcn_perm(d, c, 0x05010400u);
    out[0] = __builtin_amdgcn_perm(lo1, lo0, 0x05040100u) ^ 0x80808080u;
    out[1] = __builtin_amdgcn_perm(lo1, lo0, 0x07060302u) ^ 0x80808080u;
    if constexpr (ND > 2) {
        const u32 hi0 = __builtin_amdgcn_perm(b, a, 0x07030602u), hi1 = __builtin_amdgcn_perm(d, c, 0x07030602u);
        out[2] = __builtin_amdgcn_perm(hi1, hi0, 0x05040100u) ^ 0x80808080u;
        if constexpr (ND > 3) out[3] = __builtin_amdgcn_perm(hi1, hi0, 0x07060302u) ^ 0x80808080u;
    }
}

// Workgroup barrier that orders LDS traffic only.
__device__ __forceinline__ void lds_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// floor(w * 2^64 / q) for w < q: the quotient estimate from the upper word of the Barrett ratio and the product with the lower
// one is short by at most 2
__device__ __forceinline__ u64 shoup_companion(u64 w, const LimbConst& c) {
    u64 e = w * c.ratio_hi + mul_hi64(w, c.ratio_lo);
    u64 r = 0 - e * c.q;  // w * 2^64 - e * q, below 3q < 2^64
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const bool more = r >= c.q;
        e += more;
        r -= more ? c.q : 0;
    }
    return e;
}

// What the end of an output reads from the LDS.  Without tokens the bias is part of the addend.
struct Ends {
    I8Channel ch;
    u64 bias;
};
template <typename V>
__device__ __forceinline__ Ends ends_of(const I8Args<V>& a, u32 row, u32 output, u64 q) {
    Ends e{a.channels[(size_t)(row >> 1) * a.n_out + output], a.bias && !(row & 1) ? a.bias[(size_t)output * a.limbs + (row >> 1)] : 0};
    if (!a.token) e.ch.addend = add_mod(e.ch.addend, e.bias, q);
    return e;
}

// What the ends of all outputs of a row have in common, for two neighbouring units of eight bytes per lane.
// STREAM: the stores go past the caches (stores_stream); by a branch per output both kinds would be the plain one.
template <typename V, bool STREAM>
struct End {
    static constexpr int SLOTS = 16 / sizeof(V);
    I8Limb c;
    u64 tok[SLOTS], tok_shoup[SLOTS];  // the tokens of this lane's slots
    bool has_token, accumulate;
    int32_t b8, b16, b24;              // 2^8, 2^16, 2^24 as data (multiplied by a literal they become shifts and additions)

    // the sum of one half's digits, made positive
    __device__ __forceinline__ u64 half(int32_t s0, int32_t s1) const { return (u64)((int64_t)s1 * b8 + ((int64_t)(1ull << I8_OFFSET_BITS) + (int64_t)s0)); }
    __device__ __forceinline__ u64 half(int32_t s0, int32_t s1, int32_t s2) const { return (u64)((int64_t)s2 * b16 + (int64_t)half(s0, s1)); }
    __device__ __forceinline__ u64 half(int32_t s0, int32_t s1, int32_t s2, int32_t s3) const { return (u64)((int64_t)s3 * b24 + (int64_t)half(s0, s1, s2)); }

    // f with the parameters of store
    template <int ND, typename F>
    __device__ __forceinline__ void with_kind(F f) const {
        using yes = std::true_type;
        using no = std::false_type;
        if constexpr (ND == 4 && sizeof(V) == 8) {  // (q >= 2^60 has eight bytes)
            if (c.exact) return has_token ? f(yes{}, yes{}) : f(yes{}, no{});
        }
        has_token ? f(no{}, yes{}) : f(no{}, no{});
    }
    // An output, from the sums of its halves at the two units.  (What no output of a call differs in is a parameter: a branch around every product
    // keeps those of the two units apart, each a chain that waits for itself.)
    template <bool EXACT, bool TOKEN>
    __device__ __forceinline__ void store(V* p, const Ends& e, const u64 (&y0)[2], const u64 (&y1)[2]) const {
        typedef V piece __attribute__((ext_vector_type(SLOTS), aligned(8)));  // 16 bytes (see u64x2)
        piece v;
#pragma unroll
        for (int k = 0; k < 2; k++) {
            if constexpr (sizeof(V) == 8) {
                const u64 r = i8_combine<EXACT>(y0[k], y1[k], e.ch, c);
                v[k] = TOKEN ? i8_token(r, tok[k], tok_shoup[k], e.bias, c) : i8_reduce(r, c);
            } else {  // the halves are two slots
                v[2 * k] = i8_finish32(y0[k], e.ch, c);
                v[2 * k + 1] = i8_finish32(y1[k], e.ch, c);
                if constexpr (TOKEN) {
                    v[2 * k] = (u32)i8_token(v[2 * k], tok[2 * k], tok_shoup[2 * k], e.bias, c);
                    v[2 * k + 1] = (u32)i8_token(v[2 * k + 1], tok[2 * k + 1], tok_shoup[2 * k + 1], e.bias, c);
                }
            }
        }
        if (accumulate) {
            const piece old = *reinterpret_cast<const piece*>(p);
#pragma unroll
            for (int k = 0; k < SLOTS; k++) v[k] = (V)add_mod(v[k], old[k], c.q);
        }
        if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<piece*>(p));
        else *reinterpret_cast<piece*>(p) = v;
    }
};

template <typename V, bool STREAM>
__device__ __forceinline__ End<V, STREAM> end_of(const I8Args<V>& a, const LimbConst& lc, const I8Limb& limb, u32 row, u32 slot) {
    End<V, STREAM> e;
    e.c = limb;
    e.has_token = a.token != nullptr;
    e.accumulate = a.accumulate;
    e.b8 = 1 << 8;
    e.b16 = 1 << 16;
    e.b24 = 1 << 24;
    asm volatile("" : "+s"(e.b8), "+s"(e.b16), "+s"(e.b24));
#pragma unroll
    for (int k = 0; k < e.SLOTS; k++) {
        e.tok[k] = e.tok_shoup[k] = 0;
        if (e.has_token) {
            e.tok[k] = a.token[(size_t)(row >> 1) * a.N + slot + k];
            e.tok_shoup[k] = shoup_companion(e.tok[k], lc);
        }
    }
    return e;
}

// The half of the digits (bytes 0 .. ND - 1, or ND .. 2 ND - 1) of unit k of a lane's 16 bytes
template <int ND>
__device__ __forceinline__ u32 half_bytes(const u32x4& x, int k, int half) {
    return half == 0 ? x[2 * k] : ND == 4 ? x[2 * k + 1] : __builtin_amdgcn_alignbyte(x[2 * k + 1], x[2 * k], ND);
}

// ---------------------------------------------------------------------------------------------
// First form: up to 32 outputs, RT tiles of 16.  A lane loads 16 bytes (units 2 l and 2 l + 1 of the wavefront's 32, l = lane % 16) of the eight
// terms of its quarter of a block (lane / 16); unit 2 l + k is column l of column tile k.  Of a result tile a lane holds the rows 4 (lane / 16) ..: row
// 4 i + r is output 4 r + i of the tile, so that few outputs are spread over all lanes.

struct Cursor {
    u32 group, block, blocks;
    u32 list, table;
};
template <typename V>
__device__ __forceinline__ Cursor enter(const I8Args<V>& a, u32 group) {
    const I8Group g = load_group(a.groups + a.first + group);
    Cursor c;
    c.group = __builtin_amdgcn_readfirstlane(group);
    c.block = 0;
    c.blocks = __builtin_amdgcn_readfirstlane((g.n_terms + 31) / 32);  // (at least one)
    c.list = __builtin_amdgcn_readfirstlane(g.list);
    c.table = __builtin_amdgcn_readfirstlane(g.table);
    return c;
}
template <typename V>
__device__ __forceinline__ void step(Cursor& c, const I8Args<V>& a, u32 end) {  // after the last block of the run the cursor stays
    if (c.block + 1 < c.blocks) c.block++;
    else if (c.group + 1 < end) c = enter(a, c.group + 1);
}

template <typename V, int RT, bool STREAM, int ND>
__device__ __forceinline__ void whole_body(const I8Args<V>& a, const LimbConst& lc, const I8Limb& limb_const, u32 part, u32 row, u32 begin, u32 end, Ends* lds) {
    const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64, quarter = lane / 16, col = lane % 16;
    constexpr u32 PER = 8 / sizeof(V);                       // residues of a unit
    const u32 comp = row & 1, limb = row >> 1;
    const u32 slot = part * whole_slots<V>() + (wave * 32 + col * 2) * PER;
    const size_t at = ((size_t)comp * a.limbs + limb) * a.N + slot;
    const u32 ct_stride = 2 * a.limbs * a.N * sizeof(V);     // bytes
    const char* x_base = reinterpret_cast<const char*>(a.ct_in + at);
    const size_t out_stride = (size_t)2 * a.limbs * a.N;
    V* const dst0 = a.out + at;
    for (u32 i = threadIdx.x; i < (end - begin) * 16 * RT; i += THREADS) {
        const I8Group& g = a.groups[a.first + begin + i / (16 * RT)];
        if (i % (16 * RT) < g.count) lds[i] = ends_of(a, row, g.out0 + i % (16 * RT), lc.q);
    }
    const End<V, STREAM> fin = end_of<V, STREAM>(a, lc, limb_const, row, slot);
    __syncthreads();

    Cursor cur = enter(a, begin), nxt = cur;
    step(nxt, a, end);
    Cursor after = nxt;
    step(after, a, end);
    u32 idx[8];
    u32x4 x[8];
    u64 w[RT], w_next[RT];
    auto request_idx = [&](const Cursor& p) {
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(a.lists + (size_t)(p.list + p.block) * 32 + quarter * 8 + 4 * j);
#pragma unroll
            for (int k = 0; k < 4; k++) idx[4 * j + k] = v[k];
        }
    };
    auto request_x = [&] {
#pragma unroll
        for (int k = 0; k < 8; k++) x[k] = *reinterpret_cast<const u32x4*>(x_base + (u64)idx[k] * ct_stride);
    };
    auto request_w = [&](const Cursor& p, u64 (&to)[RT]) {
#pragma unroll
        for (int o = 0; o < RT; o++) to[o] = reinterpret_cast<const u64*>(a.table)[((size_t)p.table + p.block * RT + o) * 64 + lane];
    };
    request_idx(cur);
    request_w(cur, w);
    request_x();
    request_idx(nxt);
    v4i sums[RT][2][2 * ND];
    while (true) {
        const bool last = cur.block + 1 == cur.blocks;
        if (cur.block == 0) {
#pragma unroll
            for (int o = 0; o < RT; o++)
#pragma unroll
                for (int k = 0; k < 2; k++)
#pragma unroll
                    for (int d = 0; d < 2 * ND; d++) sums[o][k][d] = v4i{0, 0, 0, 0};
        }
        request_w(nxt, w_next);
        u64 in[2][2 * ND];
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int h = 0; h < 2; h++) {
                u32 t[2][ND];
#pragma unroll
                for (int j = 0; j < 2; j++)
                    transpose4<ND>(half_bytes<ND>(x[4 * j], k, h), half_bytes<ND>(x[4 * j + 1], k, h), half_bytes<ND>(x[4 * j + 2], k, h),
                                   half_bytes<ND>(x[4 * j + 3], k, h), t[j]);
#pragma unroll
                for (int d = 0; d < ND; d++) in[k][h * ND + d] = (u64)t[1][d] << 32 | t[0][d];
            }
        request_x();
        request_idx(after);
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int d = 0; d < 2 * ND; d++)
#pragma unroll
                for (int o = 0; o < RT; o++)
                    sums[o][k][d] = __builtin_amdgcn_mfma_i32_16x16x32_i8((long)w[o], (long)in[k][d], sums[o][k][d], 0, 0, 0);
#pragma unroll
        for (int o = 0; o < RT; o++) w[o] = w_next[o];
        if (last) {
            const I8Group g = load_group(a.groups + a.first + cur.group);
            const Ends* ends = lds + (cur.group - begin) * 16 * RT;
            V* const dst = dst0 + g.out0 * out_stride;
            fin.template with_kind<ND>([&](auto exact, auto token) {
#pragma unroll
                for (int i = 0; i < 4 * RT; i++) {
                    if (4 * (u32)i >= g.count) break;
                    const u32 mine = 4 * i + quarter;
                    if (mine < g.count) {
                        u64 y[2][2];
#pragma unroll
                        for (int h = 0; h < 2; h++)
#pragma unroll
                            for (int k = 0; k < 2; k++) {
                                const v4i (&t)[2 * ND] = sums[i / 4][k];
                                const int r = i % 4;
                                if constexpr (ND == 2) y[h][k] = fin.half(t[2 * h][r], t[2 * h + 1][r]);
                                else if constexpr (ND == 3) y[h][k] = fin.half(t[3 * h][r], t[3 * h + 1][r], t[3 * h + 2][r]);
                                else y[h][k] = fin.half(t[4 * h][r], t[4 * h + 1][r], t[4 * h + 2][r], t[4 * h + 3][r]);
                            }
                        fin.template store<decltype(exact)::value, decltype(token)::value>(dst + mine * out_stride, ends[mine], y[0], y[1]);
                    }
                    __builtin_amdgcn_sched_barrier(0);           // one output at a time: its temporaries are few
                }
            });
            if (cur.group + 1 >= end) break;
        }
        cur = nxt;
        nxt = after;
        step(after, a, end);
    }
}

// Workgroups go to the eight XCDs round-robin: the eight slices of a run of slots fastest, then the runs of groups, so that what reads one
// slice runs on one XCD, close in time, and finds its inputs in that L2.
struct Place {
    u32 part, run, row;
};
__device__ __forceinline__ Place place_of(u32 parts, u32 runs) {
    const u32 side = min(parts, 8u);  // (parts is a power of two)
    u32 b = blockIdx.x / side;
    const u32 run = b % runs;
    b /= runs;
    return Place{b % (parts / side) * side + blockIdx.x % side, run, b / (parts / side)};
}

template <typename V, int RT, bool STREAM>
__global__ void __launch_bounds__(THREADS, 2) i8_whole_kernel(LimbTable lt, I8Limbs lc, I8Args<V> a) {
    __shared__ Ends lds[WHOLE_RUN * 16 * RT];
    const Place at = place_of(a.N / whole_slots<V>(), a.runs);
    const u32 begin = at.run * a.run, end = min(begin + a.run, a.n_groups);
    const LimbConst& c = lt.c[at.row >> 1];
    const I8Limb& l = lc.c[at.row >> 1];
    if constexpr (sizeof(V) == 4) whole_body<V, RT, STREAM, 4>(a, c, l, at.part, at.row, begin, end, lds);
    else if (l.nd == 4) whole_body<V, RT, STREAM, 4>(a, c, l, at.part, at.row, begin, end, lds);
    else if (l.nd == 3) whole_body<V, RT, STREAM, 3>(a, c, l, at.part, at.row, begin, end, lds);
    else whole_body<V, RT, STREAM, 2>(a, c, l, at.part, at.row, begin, end, lds);
}

// ---------------------------------------------------------------------------------------------
// Second form: two tiles of 32 outputs.  A workgroup takes 64 units of eight bytes and 64 terms at a time: each wavefront loads 16 of the
// terms, 16 bytes of a row per lane, transposes them and writes the operands to the LDS; then it multiplies the digits of one half by
// one of the tiles.  Unit 2 l + k of the 64 is column l of column tile k, so that a lane ends up with two neighbouring units.

// Operands of 64 terms: [block of 32 terms][digit][column tile][lane], twice (one is filled while the other is multiplied).
constexpr u32 OPERAND_PIECES = 2 * 8 * 2 * 64;
constexpr u32 LIST_STEPS = 32;  // steps whose list is in the LDS

template <typename V, bool STREAM, int ND>
__device__ __forceinline__ void split_body(const I8Args<V>& a, const LimbConst& c, const I8Limb& limb_const, const I8Group& g, u32 part, u32 row, Ends* ends,
                                           v4i* lds, u32* ct_list) {
    const u32 lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32, col = lane % 32;
    constexpr u32 PER = 8 / sizeof(V);                       // residues of a unit
    const u32 comp = row & 1, limb = row >> 1;
    const u32 slot = part * split_slots<V>() + col * 2 * PER;  // this lane's first, of four or two
    const size_t at = ((size_t)comp * a.limbs + limb) * a.N + slot;
    const u32 ct_stride = 2 * a.limbs * a.N * sizeof(V);     // bytes
    const char* x_base = reinterpret_cast<const char*>(a.ct_in + at);
    const u32 upper = wave & 1, tile = wave / 2;           // what this wavefront multiplies
    const u32 load_block = wave / 2, load_half = wave & 1;   // what it loads: 16 terms of one of the two blocks, eight per lane
    const v4i* table = a.table + (size_t)g.table * 32 + tile * 64 + lane;
    if (threadIdx.x < g.count) ends[threadIdx.x] = ends_of(a, row, g.out0 + threadIdx.x, c.q);

    v16i sums[2][ND];
#pragma unroll
    for (int k = 0; k < 2; k++)
#pragma unroll
        for (int d = 0; d < ND; d++)
#pragma unroll
            for (int i = 0; i < 16; i++) sums[k][d][i] = 0;

    // Step s multiplies blocks 2 s and 2 s + 1 while the residues of step s + 1 become its operands; those of steps s + 2 and s + 3 are on
    // their way; past the end the last step's are requested again.  Loads complete in order: what is waited for sooner is requested first, and
    // the list lies in the LDS, LIST_STEPS steps of it at a time.
    u32 steps, step0;  // of this part of the list
    u32x4 x[2][8];
    v4i w[2][2];       // [step's parity][block]
    auto request_x = [&](u32 s, u32x4 (&to)[8]) {
        const u32x4* p = reinterpret_cast<const u32x4*>(ct_list + min(s, steps - 1) * 64 + load_block * 32 + load_half * 16 + half * 8);
        const u32x4 i0 = p[0], i1 = p[1];
#pragma unroll
        for (int k = 0; k < 8; k++) to[k] = *reinterpret_cast<const u32x4*>(x_base + (u64)(k < 4 ? i0[k] : i1[k - 4]) * ct_stride);
    };
    auto request_w = [&](u32 s, v4i (&to)[2]) {
#pragma unroll
        for (int b = 0; b < 2; b++) to[b] = table[((size_t)(step0 + min(s, steps - 1)) * 2 + b) * (2 * 64)];
    };
    // one half of the digits of column tile k: eight terms
    auto write_operand = [&](v4i* to, const u32x4 (&from)[8], int k, int h) {
        u32 t[2][ND];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            transpose4<ND>(half_bytes<ND>(from[4 * j], k, h), half_bytes<ND>(from[4 * j + 1], k, h), half_bytes<ND>(from[4 * j + 2], k, h),
                           half_bytes<ND>(from[4 * j + 3], k, h), t[j]);
        }
#pragma unroll
        for (int d = 0; d < ND; d++) {
            u32x2* p = reinterpret_cast<u32x2*>(to + ((load_block * 8 + h * ND + d) * 2 + k) * 64 + load_half * 32 + col) + half;
            *p = u32x2{t[0][d], t[1][d]};
        }
    };
    auto multiply = [&](auto of_parity, u32 s) {
        constexpr int P = decltype(of_parity)::value;
        const v4i* from = lds + P * OPERAND_PIECES + upper * (ND * 2 * 64) + lane;
        v4i* to = lds + (P ^ 1) * OPERAND_PIECES;
        lds_barrier();  // the operands of this step are in place, and nobody reads the others any more
        v4i in[ND];     // the next ND operands: of digit d, block q / 2 and column tile q % 2
#pragma unroll
        for (int d = 0; d < ND; d++) in[d] = from[(d * 2) * 64];
#pragma unroll
        for (int q = 0; q < 4; q++) {  // a fourth of the products, and of the next step's operands
#pragma unroll
            for (int d = 0; d < ND; d++) {
                sums[q % 2][d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[P][q / 2], in[d], sums[q % 2][d], 0, 0, 0);
                if (q < 3) in[d] = from[(((q + 1) / 2 * 8 + d) * 2 + (q + 1) % 2) * 64];
            }
            write_operand(to, x[P ^ 1], q % 2, q / 2);
            // a product, an operand of the next fourth and a share of the arithmetic in turn (in any other order six registers too many are alive)
#pragma unroll
            for (int d = 0; d < ND; d++) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x002, 7, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        request_w(s + 2, w[P]);
        request_x(s + 3, x[P ^ 1]);
        __builtin_amdgcn_sched_barrier(0);
    };
    const u32 all_steps = (g.n_terms + 63) / 64;
    for (step0 = 0; step0 < all_steps; step0 += LIST_STEPS) {
        steps = min(all_steps - step0, LIST_STEPS);
        for (u32 i = threadIdx.x; i < steps * 64; i += THREADS) ct_list[i] = a.lists[(size_t)g.list * 32 + step0 * 64 + i];
        lds_barrier();
        request_w(0, w[0]);
        request_w(1, w[1]);
        request_x(0, x[0]);
        request_x(1, x[1]);
#pragma unroll
        for (int q = 0; q < 4; q++) write_operand(lds, x[0], q % 2, q / 2);
        request_x(2, x[0]);
        u32 s = 0;
        for (; s + 1 < steps; s += 2) {
            multiply(std::integral_constant<int, 0>{}, s);
            multiply(std::integral_constant<int, 1>{}, s + 1);
        }
        if (s < steps) multiply(std::integral_constant<int, 0>{}, s);
        lds_barrier();  // (the operands and the list are not read any more)
    }

    const End<V, STREAM> fin = end_of<V, STREAM>(a, c, limb_const, row, slot);
    const size_t out_stride = (size_t)2 * a.limbs * a.N;
    V* const dst = a.out + g.out0 * out_stride + at;
    auto sum = [&](int k, int r) {
        const v16i (&t)[ND] = sums[k];
        if constexpr (ND == 2) return fin.half(t[0][r], t[1][r]);
        else if constexpr (ND == 3) return fin.half(t[0][r], t[1][r], t[2][r]);
        else return fin.half(t[0][r], t[1][r], t[2][r], t[3][r]);
    };
    // The wavefront of the lower digits finishes the first eight of a lane's outputs, the other one the last eight: they exchange the others' sums.
    auto finish = [&](auto of_upper, auto exact, auto token) {
        constexpr bool UPPER = decltype(of_upper)::value;
        constexpr int KEEP = UPPER ? 8 : 0, SEND = 8 - KEEP;
        u64* exchange = reinterpret_cast<u64*>(lds) + lane;  // [wavefront][output][column tile][lane]
#pragma unroll
        for (int i = 0; i < 16; i++) exchange[(wave * 16 + i) * 64] = sum(i % 2, SEND + i / 2);
        lds_barrier();  // (also for the ends)
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const u32 r = KEEP + i, mine = 32 * tile + 8 * (r / 4) + 4 * half + r % 4;
            if (mine < g.count) {
                u64 own_sum[2], other[2];
#pragma unroll
                for (int k = 0; k < 2; k++) own_sum[k] = sum(k, KEEP + i), other[k] = exchange[((wave ^ 1) * 16 + 2 * i + k) * 64];
                fin.template store<decltype(exact)::value, decltype(token)::value>(dst + mine * out_stride, ends[mine], UPPER ? other : own_sum, UPPER ? own_sum : other);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    fin.template with_kind<ND>([&](auto exact, auto token) {
        if (upper) finish(std::true_type{}, exact, token);
        else finish(std::false_type{}, exact, token);
    });
}

template <typename V, bool STREAM>
__global__ void __launch_bounds__(THREADS, 2) i8_split_kernel(LimbTable lt, I8Limbs lc, I8Args<V> a) {
    __shared__ Ends ends[64];
    __shared__ v4i lds[2 * OPERAND_PIECES];
    __shared__ __align__(16) u32 ct_list[LIST_STEPS * 64];
    const Place at = place_of(a.N / split_slots<V>(), a.runs);
    const I8Group g = load_group(a.groups + a.first + at.run);
    const LimbConst& c = lt.c[at.row >> 1];
    const I8Limb& l = lc.c[at.row >> 1];
    if constexpr (sizeof(V) == 4) split_body<V, STREAM, 4>(a, c, l, g, at.part, at.row, ends, lds, ct_list);
    else if (l.nd == 4) split_body<V, STREAM, 4>(a, c, l, g, at.part, at.row, ends, lds, ct_list);
    else if (l.nd == 3) split_body<V, STREAM, 3>(a, c, l, g, at.part, at.row, ends, lds, ct_list);
    else split_body<V, STREAM, 2>(a, c, l, g, at.part, at.row, ends, lds, ct_list);
}

u32 class_count(const he_i8_layer* l, u32 cls) { return l->class_begin[cls + 1] - l->class_begin[cls]; }

// How a class is launched: the groups that a workgroup takes, and the workgroups.
struct Launch {
    u32 run;
    u64 blocks;
};
template <typename V>
Launch class_launch(const he_ctx* ctx, const he_i8_layer* l, u32 limbs, u32 cls) {
    const u64 rows = 2 * limbs, count = class_count(l, cls);
    if (cls >= 2) return Launch{1, count * (ctx->N / split_slots<V>()) * rows};
    Launch k{WHOLE_RUN, 0};
    auto blocks = [&] { return (count + k.run - 1) / k.run * (ctx->N / whole_slots<V>()) * rows; };
    while (k.run > 1 && blocks() < MIN_WORKGROUPS) k.run /= 2;
    k.blocks = blocks();
    return k;
}

template <typename V, bool STREAM, int CLS>
int launch_class(he_ctx* ctx, I8Args<V> a, const he_i8_layer* l, hipStream_t s) {
    a.first = l->class_begin[CLS];
    a.n_groups = class_count(l, CLS);
    if (a.n_groups == 0) return HE_OK;
    const Launch k = class_launch<V>(ctx, l, a.limbs, CLS);
    const dim3 grid((u32)k.blocks), block(THREADS);
    a.run = k.run;
    a.runs = (a.n_groups + a.run - 1) / a.run;
    if constexpr (CLS < 2) hipLaunchKernelGGL((i8_whole_kernel<V, CLS + 1, STREAM>), grid, block, 0, s, ctx->limbs, l->limbs, a);
    else hipLaunchKernelGGL((i8_split_kernel<V, STREAM>), grid, block, 0, s, ctx->limbs, l->limbs, a);
    HE_HIP(hipGetLastError());
    return HE_OK;
}

template <typename V>
int launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const V* ct_in, const V* token, const u64* bias, V* out, u32 accumulate, hipStream_t s) {
    const I8Args<V> a{l->groups_dev, l->lists_dev, reinterpret_cast<const v4i*>(l->table_dev), sizeof(V) == 8 ? l->channels_dev : l->channels32_dev,
                      ct_in, token, bias, out, limbs, ctx->N, l->n_out, 0, 0, 0, 0, accumulate};
    auto all = [&](auto stream) {
        constexpr bool STREAM = decltype(stream)::value;
        int rc = launch_class<V, STREAM, 0>(ctx, a, l, s);
        if (rc == HE_OK) rc = launch_class<V, STREAM, 1>(ctx, a, l, s);
        return rc == HE_OK ? launch_class<V, STREAM, 2>(ctx, a, l, s) : rc;
    };
    return stores_stream(l->n_read, l->n_out, limbs, ctx->N, sizeof(V)) ? all(std::true_type{}) : all(std::false_type{});
}

u64 mul_mod_host(u64 a, u64 b, u64 q) { return (u64)((u128)a * b % q); }

// the terms of an output: where they start
struct Rows {
    const u32 *off, *ct, *pt;
    u32 terms(u32 o) const { return off[o + 1] - off[o]; }
    bool same_inputs(u32 a, u32 b) const {
        return terms(a) == terms(b) && (terms(a) == 0 || memcmp(ct + off[a], ct + off[b], (size_t)terms(a) * 4) == 0);
    }
};

}  // namespace

// every launch of a call must fit a grid, whose threads HIP counts in 32 bits
int check_i8_launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, bool packed) {
    for (u32 cls = 0; cls < I8_CLASSES; cls++)
        if ((packed ? class_launch<u32>(ctx, l, limbs, cls) : class_launch<u64>(ctx, l, limbs, cls)).blocks * THREADS > 0xFFFFFFFFull) return HE_ERR_RANGE;
    return HE_OK;
}

I8Form i8_form(const he_i8_layer* l, u32 limbs, u32 cls, bool packed) {
    const he_ctx* ctx = l->ctx;
    const Launch k = packed ? class_launch<u32>(ctx, l, limbs, cls) : class_launch<u64>(ctx, l, limbs, cls);
    return I8Form{class_count(l, cls), k.run,
                  stores_stream(l->n_read, l->n_out, limbs, ctx->N, packed ? sizeof(u32) : sizeof(u64))};
}

void fill_i8_limb(I8Limb& c, u64 q) {
    u32 bits = 0;
    while (q >> bits) bits++;
    c.q = q;
    c.two_q = 2 * q;
    c.nd = std::max<u32>(2, ((bits + 7) / 8 + 1) / 2);
    c.exact = q >= 1ull << 60;
    c.bits_shift = bits - 8;
    c.mult = (u32)(((u128)1 << (16 + c.bits_shift)) / q);
}

I8Channel i8_channel(const I8Limb& c, u64 s, int64_t weight_sum, bool packed) {
    const u64 q = c.q, shift = (u64)(((u128)1 << (8 * c.nd)) % q), offset = (1ull << I8_OFFSET_BITS) % q;
    u64 flipped = 0;  // what the digits' top bits stand for: all of them, or the four of packed storage
    for (u32 d = 0; d < (packed ? 4 : 2 * c.nd); d++) flipped |= 0x80ull << (8 * d);
    const u64 sum = (u64)(((__int128)weight_sum % (__int128)q + q) % q);
    const u64 offsets = packed ? offset : (u64)(((u128)offset + mul_mod_host(offset, shift, q)) % q);
    const u64 s1 = mul_mod_host(s, shift, q);
    return I8Channel{s, (u64)(((u128)s << 64) / q), s1, (u64)(((u128)s1 << 64) / q),
                     mul_mod_host(s, (mul_mod_host(flipped % q, sum, q) + q - offsets) % q, q)};
}

namespace {

// Outputs of one or several runs (outputs with the same inputs in the same order), as one group over the union of their inputs.
struct Merged {
    struct Run {
        u32 first, count;
        std::vector<u32> place;  // of the run's terms in the list; empty: their own order
    };
    std::vector<Run> runs;
    std::vector<u32> list;
    std::unordered_map<u32, std::vector<u32>> at;  // the places of a ciphertext
    u32 count = 0;

    // The places of a run's terms; ciphertexts that the list lacks (or has fewer times) are to be appended to it.
    std::vector<u32> places(const u32* ct, u32 terms, std::vector<u32>& added) const {
        std::vector<u32> place(terms);
        std::unordered_map<u32, u32> seen;
        for (u32 t = 0; t < terms; t++) {
            const u32 k = seen[ct[t]]++;
            const auto it = at.find(ct[t]);
            const u32 have = it == at.end() ? 0 : (u32)it->second.size();
            if (k < have) {
                place[t] = it->second[k];
                continue;
            }
            place[t] = (u32)(list.size() + added.size());
            added.push_back(ct[t]);
        }
        return place;
    }
    void add(u32 first, u32 n, std::vector<u32> place, const std::vector<u32>& added) {
        for (u32 ct : added) {
            at[ct].push_back((u32)list.size());
            list.push_back(ct);
        }
        runs.push_back(Run{first, n, std::move(place)});
        count += n;
    }
};

// The classes of groups: one or two tiles of 16 in the first form, two of 32 in the second.  (One tile is half the products: 845 -> 10 at N = 2^13, L = 4,
// 79.4 us, 80.4 with two.)
u32 class_of(u32 count) { return count > 32 ? 2 : count > 16 ? 1 : 0; }
u32 blocks_of(u32 count, u32 terms) { return count > 32 ? (terms + 63) / 64 * 2 : (terms + 31) / 32; }

// What a group costs, as far as it matters for what to merge: loads, transposition and products of a block of terms, the ends of four outputs, and its
// start.  Only the proportions count.  Layers of 256 such groups (N = 2^13, moduli of 60 and 50 bits, inputs from the caches) take 780 (up to 16 outputs) and
// 1000 cycles of a SIMD per block and 32 slots, 530 per four outputs and 450 to start.  What is decided by it hangs little on them: six
// convolutions with each constant halved or doubled, or the start four times as dear or free, took from 4 % less time to 4 % more; unmerged 11 to 40 % more, but for
// one whose windows are too many outputs to merge.
u32 group_cost(u32 count, u32 terms) { return blocks_of(count, terms) * (count > 16 ? 700 : 600) + (count + 3) / 4 * 400 + 250; }

struct LayerBuilder {
    const Rows rows;
    const int8_t* weights;
    I8Host& h;
    std::vector<I8Group> classes[I8_CLASSES];
    std::unordered_multimap<u64, I8Group> known;  // groups by a hash of their tables, which equal ones share

    u32 add_list(const std::vector<u32>& list, u32 blocks) {
        const u32 at = (u32)(h.lists.size() / 32);
        for (u32 t = 0; t < blocks * 32; t++) h.lists.push_back(list[std::min<size_t>(t, list.size() - 1)]);
        return at;
    }

    // count outputs from `first` on, whose terms lie at these places of the list (null: in order)
    void add_group(const Merged& m, u32 first, u32 count, u32 list) {
        const u32 terms = (u32)m.list.size(), cls = terms == 0 ? 2 : class_of(count), blocks = blocks_of(cls == 2 ? 64 : count, terms);
        I8Group g{first, count, terms, list, (u32)(h.table.size() / 512), {0, 0, 0}};
        // First form: [block][tile of 16 rows][lane][8], lane's row lane % 16 (output 4 (row % 4) + row / 4 of the tile), terms 8 (lane / 16) .. of the
        // block.  Second form: [block][tile of 32 rows][lane][16], row lane % 32, terms 16 (lane / 32) ..
        const u32 units = cls < 2 ? cls + 1 : 4;  // of 512 bytes, per block
        const size_t start = h.table.size(), bytes = (size_t)blocks * units * 512;
        h.table.resize(start + bytes, 0);
        int8_t* const table = h.table.data() + start;
        for (const Merged::Run& run : m.runs)
            for (u32 o = std::max(run.first, first); o < std::min(run.first + run.count, first + count); o++) {
                const u32 r = o - first, row = r % 4 * 4 + r % 16 / 4, n = rows.terms(o);
                for (u32 k = 0; k < n; k++) {
                    const size_t t = run.place.empty() ? k : run.place[k];
                    const size_t at = cls < 2 ? ((t / 32 * units + r / 16) * 64 + t % 32 / 8 * 16 + row) * 8 + t % 8
                                              : ((t / 32 * 2 + r / 32) * 64 + t % 32 / 16 * 32 + r % 32) * 16 + t % 16;
                    table[at] = weights[rows.pt[rows.off[o] + k]];
                }
            }
        u64 hash = 0xCBF29CE484222325ull ^ bytes;
        for (size_t i = 0; i < bytes; i += 8) {
            u64 v;
            memcpy(&v, table + i, 8);
            hash = (hash ^ v) * 0x100000001B3ull;
            hash ^= hash >> 29;
        }
        const auto range = known.equal_range(hash);
        bool found = false;
        for (auto it = range.first; it != range.second && !found; ++it) {
            const I8Group& k = it->second;
            const u32 k_cls = k.n_terms == 0 ? 2 : class_of(k.count);
            if (k_cls != cls || blocks_of(cls == 2 ? 64 : k.count, k.n_terms) != blocks ||
                (bytes && memcmp(h.table.data() + (size_t)k.table * 512, table, bytes) != 0))
                continue;
            g.table = k.table;
            found = true;
        }
        if (found) h.table.resize(start);
        else known.emplace(hash, g);
        classes[cls].push_back(g);
    }

    void flush(Merged& m) {
        if (m.count) add_group(m, m.runs[0].first, m.count, add_list(m.list, blocks_of(m.count, (u32)m.list.size())));
        m = Merged();
    }

    // A run of outputs that is a group or several by itself, all with the same list
    void add_run(u32 first, u32 end) {
        const u32 terms = rows.terms(first), tiles = (end - first + 31) / 32, cuts = (tiles + 1) / 2, each = (tiles + cuts - 1) / cuts * 32;
        Merged m;
        m.list.assign(rows.ct + rows.off[first], rows.ct + rows.off[first] + terms);
        m.runs.push_back(Merged::Run{first, end - first, {}});
        const u32 list = terms ? add_list(m.list, blocks_of(64, terms)) : 0;
        for (u32 o = first; o < end; o += std::min(each, end - o)) add_group(m, o, std::min(each, end - o), list);
    }

    // Neighbouring windows of a convolution share most of their inputs: as one group over the union of them (with zeros where a window lacks
    // one) they are loaded and transposed once, and the tiles of outputs are fuller.
    void build(u32 n_out) {
        Merged m;
        for (u32 o = 0, end; o < n_out; o = end) {
            end = o + 1;
            while (end < n_out && rows.same_inputs(o, end)) end++;
            const u32 n = end - o, terms = rows.terms(o);
            if (n > 64 || terms == 0) {
                flush(m);
                add_run(o, end);
                continue;
            }
            std::vector<u32> added, place = m.places(rows.ct + rows.off[o], terms, added);
            const u32 joint = (u32)(m.list.size() + added.size());
            if (m.count && (m.count + n > 32 || group_cost(m.count + n, joint) >= group_cost(m.count, (u32)m.list.size()) + group_cost(n, terms))) {
                flush(m);
                added.clear();
                place = m.places(rows.ct + rows.off[o], terms, added);
            }
            m.add(o, n, std::move(place), added);
        }
        flush(m);
    }
};

}  // namespace

// The host's part of a layer: groups, lists, table and constants (throws std::bad_alloc).
void build_i8_layer(const he_ctx* ctx, const u32* off, const u32* term_ct, const u32* term_pt, const int8_t* weights, const u64* scale,
                    he_i8_layer* l, I8Host& h) {
    const u32 n_out = l->n_out;
    LayerBuilder b{Rows{off, term_ct, term_pt}, weights, h, {}, {}};
    b.build(n_out);
    for (u32 cls = 0; cls < I8_CLASSES; cls++) {
        l->class_begin[cls] = (u32)h.groups.size();
        h.groups.insert(h.groups.end(), b.classes[cls].begin(), b.classes[cls].end());
    }
    l->class_begin[I8_CLASSES] = (u32)h.groups.size();
    l->n_read = (u32)std::unordered_set<u32>(term_ct, term_ct + off[n_out]).size();
    // Per limb and output: the scale and the constant that goes with it.
    std::vector<int64_t> weight_sum(n_out);
    for (u32 o = 0; o < n_out; o++)
        for (u32 t = off[o]; t < off[o + 1]; t++) weight_sum[o] += weights[term_pt[t]];
    h.channels.resize((size_t)ctx->L * n_out);
    h.channels32.resize((size_t)ctx->L * n_out);
    for (u32 i = 0; i < ctx->L; i++) {
        fill_i8_limb(l->limbs.c[i], ctx->q[i]);
        for (u32 o = 0; o < n_out; o++) {
            const u64 s = scale ? scale[(size_t)o * ctx->L + i] : 1;
            h.channels[(size_t)i * n_out + o] = i8_channel(l->limbs.c[i], s, weight_sum[o], false);
            h.channels32[(size_t)i * n_out + o] = i8_channel(l->limbs.c[i], s, weight_sum[o], true);
        }
    }
}

int launch_i8(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const u64* ct_in, const u64* token, const u64* bias, u64* out, u32 accumulate,
              hipStream_t s) {
    return launch<u64>(ctx, l, limbs, ct_in, token, bias, out, accumulate, s);
}

int launch_i8_32(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const u32* ct_in, const u32* token, const u64* bias, u32* out, u32 accumulate,
                 hipStream_t s) {
    return launch<u32>(ctx, l, limbs, ct_in, token, bias, out, accumulate, s);
}
