// Packed work of different lengths dealt out to workgroups: which sequence, and which piece of it, a workgroup's number means.
// Every wave finds out for itself, from the lengths on the device: 64 sequences at a time, one a lane.
#pragma once
#include <hip/hip_runtime.h>

namespace qattn {

// Sums of the lanes up to each lane (of 32 bits, saturated), by DPP moves: 4 within rows of 16, then the rows' last lanes to the rows behind.
// Six of the LDS permutations that shuffles are made of would take 0.3 us of a kernel's start.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t add_from(uint32_t v) {
    return __builtin_elementwise_add_sat(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v = add_from<0x111, 0xF>(v);      // row_shr:1
    v = add_from<0x112, 0xF>(v);      // row_shr:2
    v = add_from<0x114, 0xF>(v);      // row_shr:4
    v = add_from<0x118, 0xF>(v);      // row_shr:8
    v = add_from<0x142, 0xA>(v);      // row_bcast:15 into rows 1 and 3
    return add_from<0x143, 0xC>(v);   // row_bcast:31 into rows 2 and 3
}
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t max_from(uint32_t v) {
    return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_scan_max(uint32_t v) {       // the largest of the lanes up to each lane
    v = max_from<0x111, 0xF>(v);
    v = max_from<0x112, 0xF>(v);
    v = max_from<0x114, 0xF>(v);
    v = max_from<0x118, 0xF>(v);
    v = max_from<0x142, 0xA>(v);
    return max_from<0x143, 0xC>(v);
}
__device__ __forceinline__ uint32_t last_lane(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)v, 63); }

struct Piece {
    int seq, piece, size;             // size: what size(seq) is
};

// Sequence and piece of number `item`, where sequence b has size(b) of something, pieces(size) pieces of it: seq -1 if there is no such item.
template <class S, class F>
__device__ __forceinline__ Piece find_piece(int n_seqs, uint32_t item, S &&size, F &&pieces) {
    const int lane = threadIdx.x & 63;
    uint32_t before = 0;
    for (int b0 = 0; b0 < n_seqs; b0 += 64) {
        const int len = b0 + lane < n_seqs ? size(b0 + lane) : 0;
        const uint32_t n = b0 + lane < n_seqs ? pieces(len) : 0, upto = wave_scan(n);
        const unsigned long long past = __ballot(before + upto > item);
        if (past != 0) {
            const int l = __builtin_ctzll(past);
            return {b0 + l, (int)(item - before - (uint32_t)__builtin_amdgcn_readlane((int)(upto - n), l)), __builtin_amdgcn_readlane(len, l)};
        }
        before += last_lane(upto);
    }
    return {-1, 0, 0};
}

// Rows of a packed sequence: its queries and its keys.
struct Span {
    int q0, nq, k0, nk;
};
// Largest offsets of queries and keys so far.
struct Reached {
    uint32_t q = 0, k = 0;
};
// The sequences of a call, 64 at a time, one a lane, from their offsets cu[b], cu[b + 1].  Where these descend a sequence begins at the largest before, so
// sequences share no row whatever the offsets hold; that is looked for once, in front (in every look, 1000 sequences of 9 queries take 508 us instead of 291).
struct Sequences {
    const int32_t *cu_q, *cu_k;
    int n, n_q, n_k;
    bool ascend;
    uint32_t top;                     // the largest n + e of a shape {n, e}
    template <class F>
    __device__ __forceinline__ Sequences(const int32_t *cu_q_, const int32_t *cu_k_, int n_, int n_q_, int n_k_, F &&shape)
        : cu_q(cu_q_), cu_k(cu_k_), n(n_), n_q(n_q_), n_k(n_k_), ascend(true) {
        int sign = 0, most = 0;
        Reached r;
        const auto look = [&]() {
            for (int b0 = 0; b0 < n; b0 += 64) {
                const Span s = at(b0, r);
                const int2 f = shape(s);
                sign |= s.nq | s.nk;
                most = max(most, f.x + f.y);
            }
        };
        look();
        ascend = !__any(sign < 0);
        if (!ascend) {
            most = 0;
            look();
        }
        top = last_lane(wave_scan_max((uint32_t)most));
    }
    // Sequence b0 + lane, entries held to the range only; behind the last no rows.
    __device__ __forceinline__ Span as_they_are(int b0) const {
        const int b = b0 + (threadIdx.x & 63);
        if (b >= n) return {0, 0, 0, 0};
        const int q0 = min(max(cu_q[b], 0), n_q), q1 = min(max(cu_q[b + 1], 0), n_q), k0 = min(max(cu_k[b], 0), n_k), k1 = min(max(cu_k[b + 1], 0), n_k);
        return {q0, q1 - q0, k0, k1 - k0};
    }
    // The same behind those that have reached so far (for b0 = 0, 64, ... in turn).
    __device__ __forceinline__ Span at(int b0, Reached &reached) const {
        Span s = as_they_are(b0);
        if (ascend) return s;
        const auto behind = [](int &first, int &count, uint32_t &from) {
            const uint32_t lo = max(from, wave_scan_max((uint32_t)first)), hi = max(lo, (uint32_t)(first + count));
            from = last_lane(hi);
            first = (int)lo;
            count = (int)(hi - lo);
        };
        behind(s.q0, s.nq, reached.q);
        behind(s.k0, s.nk, reached.k);
        return s;
    }
};
struct Tile {
    int piece, part;                  // piece -1: there is no such number
    int work;                         // of the piece
    Span span;                        // of its sequence
};

// The same for pieces that are dealt out heaviest first and come in parts: a sequence has pieces 0 .. n - 1, the work of piece p is e + p, and a piece
// of work w has parts(w) parts, those of all works below w sum(w) (sum(w + 1) - sum(w) = parts(w) > 0).  Numbers go by falling work, then by sequence, then by
// part.  shape(span): {n, e}.
template <class F, class P, class U>
__device__ __forceinline__ Tile find_heaviest(const Sequences &seqs, uint32_t number, F &&shape, P &&parts, U &&sum) {
    const int lane = threadIdx.x & 63;
    Reached behind_first;
    const Span first = seqs.at(0, behind_first);                      // all there is to load where there are 64 sequences or fewer
    const auto others = [&](auto &&f) {
        Reached r = behind_first;
        for (int b0 = 64; b0 < seqs.n; b0 += 64) f(seqs.at(b0, r));
    };
    const int2 mine = shape(first);
    const uint32_t mine_all = sum((uint32_t)(mine.x + mine.y));
    // parts of the pieces with work w or more, of this lane's sequences
    const auto from = [&](int2 s, uint32_t all, int w) { return all - sum((uint32_t)min(max(w, s.y), s.x + s.y)); };
    const auto count = [&](int w) {
        uint32_t n = from(mine, mine_all, w);
        others([&](const Span &span) {
            const int2 s = shape(span);
            n += from(s, sum((uint32_t)(s.x + s.y)), w);
        });
        return last_lane(wave_scan(n));
    };
    uint32_t hi = seqs.top, lo = 0;                                   // count(hi) = 0 <= number
    if (count(0) <= number) return {-1, 0, 0, first};
    while (hi - lo > 1) {                                             // count(lo) > number >= count(hi)
        const uint32_t mid = lo + (hi - lo) / 2;
        (count((int)mid) > number ? lo : hi) = mid;
    }
    // the number-th part of a piece with work lo, in the order of the sequences
    const uint32_t number_there = number - count((int)hi), each = parts(lo);
    uint32_t left = number_there / each;
    const int part = (int)(number_there - left * each);
    Reached r = behind_first;
    for (int b0 = 0; b0 < seqs.n; b0 += 64) {
        const Span s = b0 == 0 ? first : seqs.at(b0, r);
        const int2 f = shape(s);
        const unsigned long long has = __ballot((int)lo >= f.y && (int)lo < f.x + f.y);
        const uint32_t n = __popcll(has);
        if (left >= n) {
            left -= n;
            continue;
        }
        const int l = __builtin_ctzll(__ballot(((has >> lane) & 1) != 0 && __popcll(has & ((1ull << lane) - 1)) == left));
        return {(int)lo - __builtin_amdgcn_readlane(f.y, l), part, (int)lo,
                {__builtin_amdgcn_readlane(s.q0, l), __builtin_amdgcn_readlane(s.nq, l), __builtin_amdgcn_readlane(s.k0, l), __builtin_amdgcn_readlane(s.nk, l)}};
    }
    return {-1, 0, 0, first};
}

}  // namespace qattn
