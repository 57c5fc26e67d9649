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
//  - groups of up to 32 outputs (convolutions, narrow layers): a wavefront takes both halves of 32 slots and runs through several
//    groups, the inputs of the next block of terms in flight; wavefronts never meet;
//  - larger ones: a wavefront takes one half, which leaves room for the sums of up to 128 outputs, so that the inputs are read
//    once for so many; the two wavefronts of a slot exchange half of their results at the end.
// Residues in packed storage are taken two at a time as one of eight bytes (first form), or one half alone (second).
//
// The end of an output: with y0, y1 the halves' sums, |y| < 2^55.1, each plus 2^56, r = y0 + (y1 256^ND mod q) is one Shoup product, and
// r s_o another, whose result is below 2q; what the offsets, the flipped bits and s_o leave to add is a constant of the output and limb.
#include <string.h>

#include <algorithm>
#include <type_traits>
#include <unordered_map>

#include "he_internal.h"

namespace {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef u32 u32x2 __attribute__((ext_vector_type(2), aligned(8)));

constexpr u32 THREADS = 256, WAVES = THREADS / 64;
constexpr int OFFSET_BITS = 56;      // what makes a half of a sum positive
constexpr u32 WHOLE_RUN = 16;        // groups that a workgroup of the first form runs through, at most
constexpr u64 MIN_WORKGROUPS = 2048; // ... while the launch keeps at least this many workgroups

// slots of a workgroup: 32 units of eight bytes per wavefront in the first form, 64 in all in the second
template <typename V>
__host__ __device__ constexpr u32 whole_slots() { return 32 * WAVES * 8 / sizeof(V); }
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

template <typename T>
__device__ __forceinline__ T uniform_load(const T* p) {  // read-only, workgroup-uniform data: a scalar load
    return *(const __attribute__((address_space(4))) T*)(p);
}
__device__ __forceinline__ I8Group load_group(const I8Group* p) {
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
    u64 s, s_shoup, addend, bias;
};
template <typename V>
__device__ __forceinline__ Ends ends_of(const I8Args<V>& a, const LimbConst& c, u32 row, u32 output) {
    const I8Channel ch = a.channels[(size_t)(row >> 1) * a.n_out + output];
    const u64 bias = a.bias && !(row & 1) ? a.bias[(size_t)output * a.limbs + (row >> 1)] : 0;
    return Ends{ch.s, ch.s_shoup, a.token ? ch.addend : add_mod(ch.addend, bias, c.q), bias};
}

// What the ends of all outputs of a row have in common.
template <typename V, int UNITS>
struct End {
    static constexpr int SLOTS = UNITS * 8 / sizeof(V);
    u64 q, two_q;
    I8Limb limb;
    u64 tok[SLOTS], tok_shoup[SLOTS];  // the tokens of this lane's slots
    bool has_token, accumulate;
    int32_t b8, b16, b24;     // 2^8, 2^16, 2^24 as data (multiplied by a literal they become shifts and additions)

    // the sum of one half's digits, made positive
    template <int ND>
    __device__ __forceinline__ u64 half(int32_t s0, int32_t s1, int32_t s2, int32_t s3) const {
        int64_t v = (int64_t)(1ull << OFFSET_BITS) + (int64_t)s0;
        v = (int64_t)s1 * b8 + v;
        if constexpr (ND > 2) v = (int64_t)s2 * b16 + v;
        if constexpr (ND > 3) v = (int64_t)s3 * b24 + v;
        return (u64)v;
    }
    // both halves -> what the channel's scale multiplies: a 64-bit value congruent to the sum, below 4q + 2^57 for q < 2^61, else 2q + 2^57
    __device__ __forceinline__ u64 join(u64 y0, u64 y1) const {
        return shoup_remainder_add(y1, limb.shift, limb.cheap ? shoup_quotient_cheap(y1, limb.shift_shoup) : shoup_quotient(y1, limb.shift_shoup), q, y0);
    }
    // the residue of an output
    __device__ __forceinline__ u64 finish(u64 r, const Ends& e, int k) const {
        u64 v = shoup_remainder_add(r, e.s, shoup_quotient(r, e.s_shoup), q, e.addend);  // below 3q
        if (has_token) {
            v = shoup_remainder_add(v, tok[k], shoup_quotient(v, tok_shoup[k]), q, e.bias);
        }
        v = v >= two_q ? v - two_q : v;
        return v >= q ? v - q : v;
    }
    // an output at UNITS neighbouring units, from the sums of their halves
    __device__ __forceinline__ void store(V* p, const Ends& e, const u64 (&y0)[UNITS], const u64 (&y1)[UNITS]) const {
        typedef V piece __attribute__((ext_vector_type(SLOTS), aligned(8)));
        piece v;
#pragma unroll
        for (int k = 0; k < UNITS; k++) {
            if constexpr (sizeof(V) == 8) v[k] = finish(join(y0[k], y1[k]), e, k);
            else v[2 * k] = (V)finish(y0[k], e, 2 * k), v[2 * k + 1] = (V)finish(y1[k], e, 2 * k + 1);
        }
        if (accumulate) {
            const piece old = *reinterpret_cast<const piece*>(p);
#pragma unroll
            for (int k = 0; k < SLOTS; k++) v[k] = (V)add_mod(v[k], old[k], q);
        }
        *reinterpret_cast<piece*>(p) = v;
    }
};

template <typename V, int UNITS>
__device__ __forceinline__ End<V, UNITS> end_of(const I8Args<V>& a, const LimbConst& c, const I8Limb& limb, u32 row, u32 slot) {
    End<V, UNITS> e;
    e.q = c.q;
    e.two_q = c.two_q;
    e.limb = limb;
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
            e.tok_shoup[k] = shoup_companion(e.tok[k], c);
        }
    }
    return e;
}

// ---------------------------------------------------------------------------------------------
// First form: up to 32 outputs.

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

template <typename V, int ND>
__device__ __forceinline__ void whole_body(const I8Args<V>& a, const LimbConst& c, const I8Limb& limb_const, u32 part, u32 row, u32 begin, u32 end, Ends* lds) {
    const u32 lane = threadIdx.x % 64, wave = threadIdx.x / 64, half = lane / 32;
    constexpr u32 PER = 8 / sizeof(V);                       // residues of a unit of eight bytes
    const u32 comp = row & 1, limb = row >> 1;
    const u32 slot = part * whole_slots<V>() + (wave * 32 + lane % 32) * PER;
    const size_t at = ((size_t)comp * a.limbs + limb) * a.N + slot;
    const u32 ct_stride = 2 * a.limbs * a.N * sizeof(V);     // bytes
    const char* x_base = reinterpret_cast<const char*>(a.ct_in + at);
    const size_t out_stride = (size_t)2 * a.limbs * a.N;
    V* const dst0 = a.out + at;
    for (u32 i = threadIdx.x; i < (end - begin) * 32; i += THREADS) {
        const I8Group& g = a.groups[a.first + begin + i / 32];
        if (i % 32 < g.count) lds[i] = ends_of(a, c, row, g.out0 + i % 32);
    }
    const End<V, 1> fin = end_of<V, 1>(a, c, limb_const, row, slot);
    __syncthreads();

    Cursor cur = enter(a, begin), nxt = cur;
    step(nxt, a, end);
    Cursor after = nxt;
    step(after, a, end);
    u32 idx[16];
    u32x2 x[16];
    v4i w, w_next;
    auto request_idx = [&](const Cursor& p, int j) {  // four terms
        const u32x4 v = *reinterpret_cast<const u32x4*>(a.lists + (size_t)(p.list + p.block) * 32 + half * 16 + 4 * j);
#pragma unroll
        for (int k = 0; k < 4; k++) idx[4 * j + k] = v[k];
    };
    auto request_x = [&](int j) {
#pragma unroll
        for (int k = 4 * j; k < 4 * j + 4; k++) x[k] = *reinterpret_cast<const u32x2*>(x_base + (u64)idx[k] * ct_stride);
    };
    auto request_w = [&](const Cursor& p) { return a.table[(size_t)(p.table + p.block) * 64 + lane]; };
    w = request_w(cur);
#pragma unroll
    for (int j = 0; j < 4; j++) request_idx(cur, j);
#pragma unroll
    for (int j = 0; j < 4; j++) request_x(j);
#pragma unroll
    for (int j = 0; j < 4; j++) request_idx(nxt, j);
    v16i sums[2 * ND];
    while (true) {
        const bool first = cur.block == 0, last = cur.block + 1 == cur.blocks;
        if (first) {
#pragma unroll
            for (int d = 0; d < 2 * ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i++) sums[d][i] = 0;
        }
        v4i in[2 * ND];
        w_next = request_w(nxt);
#pragma unroll
        for (int j = 0; j < 4; j++) {  // (four terms at a time, whose registers take those of the next block)
            u32 lo[ND], hi[ND];
            // the second half's bytes start at byte ND
            auto up = [&](int k) -> u32 { return ND == 4 ? x[k][1] : __builtin_amdgcn_alignbyte(x[k][1], x[k][0], ND); };
            transpose4<ND>(x[4 * j][0], x[4 * j + 1][0], x[4 * j + 2][0], x[4 * j + 3][0], lo);
            transpose4<ND>(up(4 * j), up(4 * j + 1), up(4 * j + 2), up(4 * j + 3), hi);
#pragma unroll
            for (int d = 0; d < ND; d++) in[d][j] = (int)lo[d], in[ND + d][j] = (int)hi[d];
            request_x(j);
            request_idx(after, j);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int d = 0; d < 2 * ND; d++) sums[d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w, in[d], sums[d], 0, 0, 0);
        w = w_next;
        if (last) {
            const I8Group g = load_group(a.groups + a.first + cur.group);
            const Ends* ends = lds + (cur.group - begin) * 32;
            V* const dst = dst0 + g.out0 * out_stride;
#pragma unroll
            for (int r = 0; r < 16; r++) {
                if (8 * (u32)(r / 4) >= g.count) break;      // (rows of both halves)
                const u32 o = 8 * (r / 4) + 4 * half + r % 4;
                if (o < g.count) {
                    const Ends e = ends[o];
                    auto sum = [&](int h) {
                        return fin.template half<ND>(sums[h * ND][r], sums[h * ND + 1][r], ND > 2 ? sums[h * ND + (ND > 2 ? 2 : 0)][r] : 0,
                                                     ND > 3 ? sums[h * ND + (ND > 3 ? 3 : 0)][r] : 0);
                    };
                    const u64 y0[1] = {sum(0)}, y1[1] = {sum(1)};
                    fin.store(dst + o * out_stride, e, y0, y1);
                }
                __builtin_amdgcn_sched_barrier(0);           // one output at a time: its temporaries are few
            }
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
    const u32 side = min(parts, 8u);  // (parts is a power of two, below eight for packed residues at N = 2^10)
    u32 b = blockIdx.x / side;
    const u32 run = b % runs;
    b /= runs;
    return Place{b % (parts / side) * side + blockIdx.x % side, run, b / (parts / side)};
}

template <typename V>
__global__ void __launch_bounds__(THREADS, 2) i8_whole_kernel(LimbTable lt, I8Limbs lc, I8Args<V> a) {
    __shared__ Ends lds[WHOLE_RUN * 32];
    const Place at = place_of(a.N / whole_slots<V>(), a.runs);
    const u32 begin = at.run * a.run, end = min(begin + a.run, a.n_groups);
    const LimbConst& c = lt.c[at.row >> 1];
    const I8Limb& l = lc.c[at.row >> 1];
    if constexpr (sizeof(V) == 4) whole_body<V, 4>(a, c, l, at.part, at.row, begin, end, lds);
    else if (l.nd == 4) whole_body<V, 4>(a, c, l, at.part, at.row, begin, end, lds);
    else if (l.nd == 3) whole_body<V, 3>(a, c, l, at.part, at.row, begin, end, lds);
    else whole_body<V, 2>(a, c, l, at.part, at.row, begin, end, lds);
}

// ---------------------------------------------------------------------------------------------
// Second form: 2 OT tiles of 32 outputs.  A workgroup takes 64 units of eight bytes and 64 terms at a time: each wavefront loads 16 of the
// terms, 16 bytes of a row per lane, transposes them and writes the operands to the LDS; then it multiplies the digits of its half by
// its OT tiles.  Unit 2 l + k of the 64 is column l of column tile k, so that a lane ends up with two neighbouring units.

// Operands of 64 terms: [block of 32 terms][digit][column tile][lane], twice (one is filled while the other is multiplied).
constexpr u32 OPERAND_PIECES = 2 * 8 * 2 * 64;

template <typename V, int OT, int ND>
__device__ __forceinline__ void split_body(const I8Args<V>& a, const LimbConst& c, const I8Limb& limb_const, const I8Group& g, u32 part, u32 row, Ends* ends,
                                           v4i* lds) {
    const u32 lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), half = lane / 32, col = lane % 32;
    constexpr u32 PER = 8 / sizeof(V);                       // residues of a unit
    const u32 comp = row & 1, limb = row >> 1;
    const u32 slot = part * split_slots<V>() + col * 2 * PER;  // this lane's first, of four or two
    const size_t at = ((size_t)comp * a.limbs + limb) * a.N + slot;
    const u32 ct_stride = 2 * a.limbs * a.N * sizeof(V);     // bytes
    const char* x_base = reinterpret_cast<const char*>(a.ct_in + at);
    const u32 blocks = (g.n_terms + 31) / 32;
    const u32 upper = wave & 1, tile0 = wave / 2 * OT;       // what this wavefront multiplies
    const u32 load_block = wave / 2, load_half = wave & 1;   // what it loads: 16 terms of one of the two blocks, eight per lane
    const u32* list = a.lists + (size_t)g.list * 32 + load_half * 16 + half * 8;
    const v4i* table = a.table + ((size_t)g.table + tile0) * 64 + lane;
    if (threadIdx.x < g.count) ends[threadIdx.x] = ends_of(a, c, row, g.out0 + threadIdx.x);

    v16i sums[OT][2][ND];
#pragma unroll
    for (int o = 0; o < OT; o++)
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int d = 0; d < ND; d++)
#pragma unroll
                for (int i = 0; i < 16; i++) sums[o][k][d][i] = 0;

    // Step s multiplies blocks 2 s and 2 s + 1 while the residues of step s + 1 become its operands; those of AHEAD steps more are
    // on their way (one where two workgroups share a compute unit); past the end the last block's are requested again.
    constexpr int AHEAD = OT == 1 ? 1 : 2;
    u32 idx[8];
    u32x4 x[AHEAD][8];
    v4i w[2][OT];
    auto request_idx = [&](u32 s) {
        const u32* p = list + (size_t)min(2 * s + load_block, blocks - 1) * 32;
#pragma unroll
        for (int j = 0; j < 2; j++) {
            const u32x4 v = *reinterpret_cast<const u32x4*>(p + 4 * j);
#pragma unroll
            for (int k = 0; k < 4; k++) idx[4 * j + k] = v[k];
        }
    };
    auto request_x = [&](u32x4 (&to)[8]) {
#pragma unroll
        for (int k = 0; k < 8; k++) to[k] = *reinterpret_cast<const u32x4*>(x_base + (u64)idx[k] * ct_stride);
    };
    auto request_w = [&](u32 block, v4i (&to)[OT]) {
#pragma unroll
        for (int o = 0; o < OT; o++) to[o] = table[((size_t)min(block, blocks - 1) * (2 * OT) + o) * 64];
    };
    // one half of the digits of column tile k: eight terms
    auto write_operand = [&](v4i* to, const u32x4 (&from)[8], int k, int h) {
        u32 t[2][ND];
#pragma unroll
        for (int j = 0; j < 2; j++) {
            auto bytes = [&](int i) -> u32 {  // the second half's start at byte ND
                const u32 lo = from[i][2 * k], hi = from[i][2 * k + 1];
                return h == 0 ? lo : ND == 4 ? hi : __builtin_amdgcn_alignbyte(hi, lo, ND);
            };
            transpose4<ND>(bytes(4 * j), bytes(4 * j + 1), bytes(4 * j + 2), bytes(4 * j + 3), t[j]);
        }
#pragma unroll
        for (int d = 0; d < ND; d++) {
            u32x2* p = reinterpret_cast<u32x2*>(to + ((load_block * 8 + h * ND + d) * 2 + k) * 64 + load_half * 32 + col) + half;
            *p = u32x2{t[0][d], t[1][d]};
        }
    };
    auto multiply = [&](auto of_parity, u32 s) {
        constexpr int P = decltype(of_parity)::value;
        const v4i* from = lds + P * OPERAND_PIECES + lane;
        v4i* to = lds + (P ^ 1) * OPERAND_PIECES;
        lds_barrier();  // the operands of this step are in place, and nobody reads the others any more
#pragma unroll
        for (int q = 0; q < 4; q++) {  // block q / 2, column tile q % 2; a fourth of the next step's operands
            if (q < 2 || 2 * s + 1 < blocks) {
#pragma unroll
                for (int d = 0; d < ND; d++) {
                    const v4i in = from[((q / 2 * 8 + upper * ND + d) * 2 + q % 2) * 64];
#pragma unroll
                    for (int o = 0; o < OT; o++)
                        sums[o][q % 2][d] = __builtin_amdgcn_mfma_i32_32x32x32_i8(w[q / 2][o], in, sums[o][q % 2][d], 0, 0, 0);
                }
            }
            if (q % 2) request_w(2 * s + 2 + q / 2, w[q / 2]);
            write_operand(to, x[(P ^ 1) % AHEAD], q % 2, q / 2);
            __builtin_amdgcn_sched_barrier(0);
        }
        request_x(x[(P ^ 1) % AHEAD]);
        request_idx(s + AHEAD + 2);
        __builtin_amdgcn_sched_barrier(0);
    };
    if (blocks) {
        const u32 steps = (blocks + 1) / 2;
        request_w(0, w[0]);
        request_w(1, w[1]);
        request_idx(0);
        request_x(x[0]);
        request_idx(1);
        if constexpr (AHEAD == 2) {
            request_x(x[1]);
            request_idx(2);
        }
#pragma unroll
        for (int q = 0; q < 4; q++) write_operand(lds, x[0], q % 2, q / 2);
        request_x(x[0]);
        request_idx(AHEAD + 1);
        u32 s = 0;
        for (; s + 1 < steps; s += 2) {
            multiply(std::integral_constant<int, 0>{}, s);
            multiply(std::integral_constant<int, 1>{}, s + 1);
        }
        if (s < steps) multiply(std::integral_constant<int, 0>{}, s);
        lds_barrier();  // (the operands are not read any more)
    }

    const End<V, 2> fin = end_of<V, 2>(a, c, limb_const, row, slot);
    const size_t out_stride = (size_t)2 * a.limbs * a.N;
    V* const dst = a.out + g.out0 * out_stride + at;
    auto sum = [&](int o, int k, int r) {
        const v16i (&t)[ND] = sums[o][k];
        return fin.template half<ND>(t[0][r], t[1][r], ND > 2 ? t[ND > 2 ? 2 : 0][r] : 0, ND > 3 ? t[ND > 3 ? 3 : 0][r] : 0);
    };
    // Of every tile the wavefront of the lower digits finishes the first eight of a lane's outputs, the other one the last eight: they exchange the
    // others' sums.
    auto finish = [&](auto of_upper) {
        constexpr bool UPPER = decltype(of_upper)::value;
        constexpr int KEEP = UPPER ? 8 : 0, SEND = 8 - KEEP;
        u64* exchange = reinterpret_cast<u64*>(lds) + lane;  // [tile parity][wavefront][output][column tile][lane]
#pragma unroll
        for (int o = 0; o < OT; o++) {
            u64* buf = exchange + (o & 1) * (WAVES * 16 * 64);
#pragma unroll
            for (int i = 0; i < 16; i++) buf[(wave * 16 + i) * 64] = sum(o, i % 2, SEND + i / 2);
            lds_barrier();  // (also for the ends)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const u32 r = KEEP + i, mine = 32 * (tile0 + o) + 8 * (r / 4) + 4 * half + r % 4;
                if (mine < g.count) {
                    const Ends e = ends[mine];
                    V* const p = dst + mine * out_stride;
                    u64 own_sum[2], other[2];
#pragma unroll
                    for (int k = 0; k < 2; k++) own_sum[k] = sum(o, k, KEEP + i), other[k] = buf[((wave ^ 1) * 16 + 2 * i + k) * 64];
                    fin.store(p, e, UPPER ? other : own_sum, UPPER ? own_sum : other);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    if (upper) finish(std::true_type{});
    else finish(std::false_type{});
}

template <typename V, int OT>
__global__ void __launch_bounds__(THREADS, OT == 1 ? 2 : 1) i8_split_kernel(LimbTable lt, I8Limbs lc, I8Args<V> a) {
    __shared__ Ends ends[64 * OT];
    __shared__ v4i lds[2 * OPERAND_PIECES];
    const Place at = place_of(a.N / split_slots<V>(), a.runs);
    const I8Group g = load_group(a.groups + a.first + at.run);
    const LimbConst& c = lt.c[at.row >> 1];
    const I8Limb& l = lc.c[at.row >> 1];
    if constexpr (sizeof(V) == 4) split_body<V, OT, 4>(a, c, l, g, at.part, at.row, ends, lds);
    else if (l.nd == 4) split_body<V, OT, 4>(a, c, l, g, at.part, at.row, ends, lds);
    else if (l.nd == 3) split_body<V, OT, 3>(a, c, l, g, at.part, at.row, ends, lds);
    else split_body<V, OT, 2>(a, c, l, g, at.part, at.row, ends, lds);
}

template <typename V>
u32 class_count(const he_i8_layer* l, u32 cls) { return l->class_begin[cls + 1] - l->class_begin[cls]; }

// workgroups of a class; *run: the groups that each of them takes
template <typename V>
u64 class_blocks(const he_ctx* ctx, const he_i8_layer* l, u32 limbs, u32 cls, u32* run) {
    const u64 rows = 2 * limbs, parts = ctx->N / (cls == 0 ? whole_slots<V>() : split_slots<V>()), count = class_count<V>(l, cls);
    *run = cls == 0 ? WHOLE_RUN : 1;
    while (*run > 1 && (count + *run - 1) / *run * parts * rows < MIN_WORKGROUPS) *run /= 2;
    return (count + *run - 1) / *run * parts * rows;
}

template <typename V, int CLS>
int launch_class(he_ctx* ctx, I8Args<V> a, const he_i8_layer* l, hipStream_t s) {
    a.first = l->class_begin[CLS];
    a.n_groups = class_count<V>(l, CLS);
    if (a.n_groups == 0) return HE_OK;
    const dim3 grid((u32)class_blocks<V>(ctx, l, a.limbs, CLS, &a.run)), block(THREADS);
    a.runs = (a.n_groups + a.run - 1) / a.run;
    if constexpr (CLS == 0) hipLaunchKernelGGL(i8_whole_kernel<V>, grid, block, 0, s, ctx->limbs, l->limbs, a);
    else hipLaunchKernelGGL((i8_split_kernel<V, CLS>), grid, block, 0, s, ctx->limbs, l->limbs, a);
    HE_HIP(hipGetLastError());
    return HE_OK;
}

template <typename V>
int launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, const V* ct_in, const V* token, const u64* bias, V* out, u32 accumulate, hipStream_t s) {
    const I8Args<V> a{l->groups_dev, l->lists_dev, reinterpret_cast<const v4i*>(l->table_dev), sizeof(V) == 8 ? l->channels_dev : l->channels32_dev,
                      ct_in, token, bias, out, limbs, ctx->N, l->n_out, 0, 0, 0, 0, accumulate};
    int rc;
    if ((rc = launch_class<V, 0>(ctx, a, l, s)) != HE_OK) return rc;
    if ((rc = launch_class<V, 1>(ctx, a, l, s)) != HE_OK) return rc;
    return launch_class<V, 2>(ctx, a, l, s);
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

// every launch of a call must fit a grid
int check_i8_launch(he_ctx* ctx, const he_i8_layer* l, u32 limbs, bool packed) {
    u32 run;
    for (u32 cls = 0; cls < I8_CLASSES; cls++)
        if ((packed ? class_blocks<u32>(ctx, l, limbs, cls, &run) : class_blocks<u64>(ctx, l, limbs, cls, &run)) > 0x7FFFFFFFull) return HE_ERR_RANGE;
    return HE_OK;
}

// The host's part of a layer: groups, lists, table and constants (throws std::bad_alloc).
void build_i8_layer(const he_ctx* ctx, const u32* off, const u32* term_ct, const u32* term_pt, const int8_t* weights, const u64* scale,
                    he_i8_layer* l, I8Host& h) {
    const Rows rows{off, term_ct, term_pt};
    const u32 n_out = l->n_out;
    // Runs of outputs that read the same inputs in the same order, cut into groups of up to 128 with the same number of tiles.
    std::vector<I8Group> classes[I8_CLASSES];
    std::unordered_multimap<u64, I8Group> known;  // groups by a hash of their weights, to share tables
    for (u32 o = 0; o < n_out;) {
        u32 end = o + 1;
        while (end < n_out && rows.same_inputs(o, end)) end++;
        const u32 terms = rows.terms(o), blocks = (terms + 31) / 32;
        const u32 tiles = (end - o + 31) / 32, cuts = (tiles + 3) / 4, each = (tiles + cuts - 1) / cuts * 32;
        const u32 list = (u32)(h.lists.size() / 32);
        for (u32 t = 0; t < blocks * 32; t++) h.lists.push_back(term_ct[off[o] + std::min(t, terms - 1)]);
        for (u32 count; o < end; o += count) {
            count = std::min(each, end - o);
            I8Group g{o, count, terms, list, 0, {0, 0, 0}};
            // (outputs without terms go to the second form, whose loop over the blocks may be empty)
            const u32 cls = count > 64 ? 2 : count > 32 || terms == 0 ? 1 : 0, per = 1u << cls;
            const size_t n = (size_t)g.count * terms;  // the plaintexts of a group's outputs follow one another
            u64 hash = 0xCBF29CE484222325ull ^ n;
            for (size_t i = 0; i < n; i++) hash = (hash ^ term_pt[off[o] + i]) * 0x100000001B3ull;
            bool found = false;
            const auto range = known.equal_range(hash);
            for (auto it = range.first; it != range.second && !found; ++it) {
                const I8Group& k = it->second;
                if (k.count != g.count || k.n_terms != terms || (n && memcmp(term_pt + off[k.out0], term_pt + off[o], n * 4) != 0)) continue;
                g.table = k.table;
                found = true;
            }
            if (!found) {
                // [block][tile][lane][16]: row lane % 32 of the tile, terms 16 * (lane / 32) .. of the block
                g.table = (u32)(h.table.size() / 1024);
                h.table.resize(h.table.size() + (size_t)blocks * per * 1024, 0);
                int8_t* t0 = h.table.data() + (size_t)g.table * 1024;
                for (u32 r = 0; r < g.count; r++)
                    for (u32 t = 0; t < terms; t++)
                        t0[(((size_t)t / 32 * per + r / 32) * 64 + t % 32 / 16 * 32 + r % 32) * 16 + t % 16] = weights[term_pt[off[o + r] + t]];
                known.emplace(hash, g);
            }
            classes[cls].push_back(g);
        }
    }
    for (u32 cls = 0; cls < I8_CLASSES; cls++) {
        l->class_begin[cls] = (u32)h.groups.size();
        h.groups.insert(h.groups.end(), classes[cls].begin(), classes[cls].end());
    }
    l->class_begin[I8_CLASSES] = (u32)h.groups.size();
    // Per limb and output: the scale and the constant that goes with it.
    std::vector<int64_t> weight_sum(n_out);
    for (u32 o = 0; o < n_out; o++)
        for (u32 t = off[o]; t < off[o + 1]; t++) weight_sum[o] += weights[term_pt[t]];
    h.channels.resize((size_t)ctx->L * n_out);
    h.channels32.resize((size_t)ctx->L * n_out);
    for (u32 i = 0; i < ctx->L; i++) {
        const u64 q = ctx->q[i];
        u32 bits = 0;
        while (q >> bits) bits++;
        const u32 nd = std::max<u32>(2, ((bits + 7) / 8 + 1) / 2);
        const u64 shift = (u64)(((u128)1 << (8 * nd)) % q), offset = (1ull << OFFSET_BITS) % q;
        l->limbs.c[i] = I8Limb{nd, q < (1ull << 61), shift, (u64)(((u128)shift << 64) / q)};
        u64 flipped = 0;  // what the digits' top bits stand for, all 2 nd of them
        for (u32 d = 0; d < 2 * nd; d++) flipped |= 0x80ull << (8 * d);
        const u64 both = (u64)(((u128)offset + mul_mod_host(offset, shift, q)) % q);
        for (u32 o = 0; o < n_out; o++) {
            const u64 s = scale ? scale[(size_t)o * ctx->L + i] : 1, s_shoup = (u64)(((u128)s << 64) / q);
            const u64 sum = (u64)(((__int128)weight_sum[o] % (__int128)q + q) % q);
            const size_t k = (size_t)i * n_out + o;
            h.channels[k] = I8Channel{s, s_shoup, mul_mod_host(s, (mul_mod_host(flipped % q, sum, q) + q - both) % q, q)};
            h.channels32[k] = I8Channel{s, s_shoup, mul_mod_host(s, (mul_mod_host(0x80808080u % q, sum, q) + q - offset) % q, q)};
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
