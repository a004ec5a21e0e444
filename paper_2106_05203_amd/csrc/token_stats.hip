// Entropy and the most likely tokens of rows of logits beside their log-probabilities, and the gradient (token_rows.h has the mathematics).
//
//   With z_v = x_v log2 e - M, s = sum 2^z_v and t = sum 2^z_v z_v:   entropy = ln 2 (log2 s - t / s)
//   d logp / d x_v = [v = label] - p_v,   d entropy / d x_v = -p_v (log p_v + entropy)
//
// A row is cut into tiles of 512 pieces of 16 bytes, a wavefront's registers full.  Each tile has an M of its own, a whole number next to its maximum: no z
// is above 1/2, so that t's terms have one sign but for the largest entries', nothing leaves fp32's range and no maximum has to be carried along.  A tile
// leaves its M, s and t, and the tiles are joined in an order that the row's length alone fixes.
//   The alternatives: a wavefront keeps the 64 best entries that it has met, one a lane, in order.  The pieces' maxima, which M needs anyway, tell which
// pieces have an entry above the k-th.  Those few go through LDS, an entry a lane; an entry that is better is inserted, or ordered and merged with others.
// Where more pieces qualify than there are alternatives (the first tiles of a row, rising rows), the bound is raised first: halving finds a value that
// some k pieces' maxima reach.
//
// Measured (a plain read of this card's memory: 7.1 TB/s).  8192 rows of 131072 bf16, one in eight ignored, without alternatives: 277 us, 6.8 TB/s; 4096
// rows with 20: 204 us, 5.3 TB/s, bound by the vector instructions of the sums (a product, an exponential, a maximum and two sums an entry) and by the
// selection's latency.  2001 rows of 32064 fp32 with 8: 46 us, 4.9 TB/s: one turn of the card's wavefronts, whose last tiles are waited for.  One row of
// 131072: 13 us, two launches' latency.
#include "token_rows.h"

namespace ef21 {
namespace {

constexpr int kThreads = 256, kWaves = kThreads / kWave;
// Pieces of a lane, of a tile.  With 4, and up to 6 wavefronts a SIMD, what a tile costs once weighs more: 4096 rows of 131072 bf16 with 20 alternatives 223
// us for 204, 2001 rows of 32064 fp32 with 8 48.5 for 45.7.  The next tile on its way in registers of its own costs more than it hides: 8 pieces 210 and
// 57, 8 with 3 wavefronts a SIMD 236 and 59, 4 with 5 227 and 49.
constexpr int kEach = 8, kTile = kEach * kWave;
// Of rows that have no more in all, where most of eight would be empty.  16384 rows of 300 to 1020 bf16 columns 13 us for 26, with 5 alternatives 26 for 44
// (behind, 1030 columns by eight: 27 and 45); of 300 to 508 fp32 columns 11 for 17 and 22 for 36 (600 columns by eight: 18 and 36).
constexpr int kEachShort = 2;
constexpr int kMostSlices = 256;

// Tiles of a row and how they are grouped: into at most 256 slices, each a wavefront's at a time.
struct Slices {
    int32_t count, tiles;                                          // slices, tiles of each
};
template <class T>
constexpr bool is_short(int64_t vocab) { return vocab / Piece<T>::N < kEachShort * kWave; }
template <class T>
__host__ __device__ __forceinline__ Slices slices_of(int32_t vocab) {
    if (is_short<T>(vocab)) return {1, 1};
    const int32_t tiles = vocab / (Piece<T>::N * kTile) + 1;       // whether a row of so many has one piece more or less
    const int32_t each = (tiles + kMostSlices - 1) / kMostSlices;
    return {(tiles + each - 1) / each, each};
}

// ---------------------------------------------------------------- order
// An order of entries: by value (-0 and 0 alike), then the lower token first.  A larger key comes first; 0 is no entry's.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t v) {
    const uint32_t bits = __float_as_uint(x + 0.f);
    const uint32_t order = bits ^ ((int32_t)bits < 0 ? 0xffffffffu : 0x80000000u);
    return (uint64_t)order << 32 | (0xffffffffu - v);
}
__device__ __forceinline__ float value_of(uint64_t key) {
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order ^ ((int32_t)order < 0 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ int32_t token_of(uint64_t key) { return (int32_t)(0xffffffffu - (uint32_t)key); }
// The next value above a key's.
__device__ __forceinline__ float value_above(uint64_t key) { return value_of(key + ((uint64_t)1 << 32)); }

__device__ __forceinline__ uint64_t read_lane(uint64_t key, int lane) {
    const uint32_t high = (uint32_t)__builtin_amdgcn_readlane((int)(key >> 32), lane), low = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)key, lane);
    return (uint64_t)high << 32 | low;
}

// The key of the lane whose number differs in the bits of MASK.
template <int CTRL>
__device__ __forceinline__ uint64_t dpp_key(uint64_t key) {
    const uint32_t high = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(key >> 32), CTRL, 0xf, 0xf, true);
    const uint32_t low = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)key, CTRL, 0xf, 0xf, true);
    return (uint64_t)high << 32 | low;
}
// Both lanes' words of lanes 16 or 32 apart, which of the two is whose left open.
template <int MASK>
__device__ __forceinline__ void swap_words(uint32_t word, uint32_t &a, uint32_t &b) {
    static_assert(MASK == 16 || MASK == 32, "");
    const auto r = MASK == 16 ? __builtin_amdgcn_permlane16_swap(word, word, false, false) : __builtin_amdgcn_permlane32_swap(word, word, false, false);
    a = r[0];
    b = r[1];
}
template <int MASK>
__device__ __forceinline__ void both_keys(uint64_t key, uint64_t &a, uint64_t &b) {
    uint32_t ah, bh, al, bl;
    swap_words<MASK>((uint32_t)(key >> 32), ah, bh);
    swap_words<MASK>((uint32_t)key, al, bl);
    a = (uint64_t)ah << 32 | al;
    b = (uint64_t)bh << 32 | bl;
}
template <int MASK>
__device__ __forceinline__ uint64_t other_key(uint64_t key) {
    if constexpr (MASK == 1) return dpp_key<0xB1>(key);                // quad_perm [1,0,3,2]
    else if constexpr (MASK == 2) return dpp_key<0x4E>(key);           // quad_perm [2,3,0,1]
    else if constexpr (MASK == 3) return dpp_key<0x1B>(key);           // quad_perm [3,2,1,0]
    else if constexpr (MASK == 4) return dpp_key<0x1B>(dpp_key<0x141>(key));
    else if constexpr (MASK == 7) return dpp_key<0x141>(key);          // row_half_mirror
    else if constexpr (MASK == 8) return dpp_key<0x128>(key);          // row_ror:8
    else if constexpr (MASK == 15) return dpp_key<0x140>(key);         // row_mirror
    else if constexpr (MASK == 31) return dpp_key<0x140>(other_key<16>(key));
    else if constexpr (MASK == 63) return other_key<31>(other_key<32>(key));
    else {                                                             // of the two the one that is not mine; mine if both are alike
        uint64_t a, b;
        both_keys<MASK>(key, a, b);
        return a == key ? b : a;
    }
}
// The larger of two lanes' keys goes to the lane with the smaller number.
template <int MASK>
__device__ __forceinline__ void exchange(uint64_t &key) {
    constexpr int kHighest = MASK >= 32 ? 32 : MASK >= 16 ? 16 : MASK >= 8 ? 8 : MASK >= 4 ? 4 : MASK >= 2 ? 2 : 1;
    const bool upper = (lane_id() & kHighest) != 0;
    if constexpr (MASK == 16 || MASK == 32) {
        uint64_t a, b;
        both_keys<MASK>(key, a, b);
        key = (a > b) != upper ? a : b;
    } else {
        const uint64_t other = other_key<MASK>(key);
        if ((key < other) != upper) key = other;
    }
}
// Of two halves in descending order, the second from its end, one in descending order; and 64 keys in any order.
__device__ __forceinline__ void order_halves(uint64_t &key) {
    exchange<32>(key);
    exchange<16>(key);
    exchange<8>(key);
    exchange<4>(key);
    exchange<2>(key);
    exchange<1>(key);
}
__device__ __forceinline__ void order_keys(uint64_t &key) {
    exchange<1>(key);
    exchange<3>(key);
    exchange<1>(key);
    exchange<7>(key);
    exchange<2>(key);
    exchange<1>(key);
    exchange<15>(key);
    exchange<4>(key);
    exchange<2>(key);
    exchange<1>(key);
    exchange<31>(key);
    exchange<8>(key);
    exchange<4>(key);
    exchange<2>(key);
    exchange<1>(key);
    exchange<63>(key);
    exchange<16>(key);
    exchange<8>(key);
    exchange<4>(key);
    exchange<2>(key);
    exchange<1>(key);
}

// An entry inserted takes some 20 instructions, 64 ordered and merged 350; but the bound then rises at once, and fewer entries are met.  4096 rows of 131072
// bf16 with 20 alternatives: 203 us so (keys of up to 3 lanes inserted 207, of 10 207), 205 where they wait across the tiles until there are 64; with 64
// alternatives 235 and 222.
constexpr uint32_t kFewKeys = 6;
constexpr int kFewBest = 32;

struct SelectShared {
    uint64_t wait[2 * kWave];
    uint32_t piece[kWave][4], token[kWave];                        // token: of a piece's first entry
};

// The best entries that a wavefront has met.  An entry can be among the k best if it is at least `bound` and its key above `limit`.
struct Selection {
    uint64_t mine = 0, limit = 0;                                  // the lane's entry, by rank; the k-th
    float bound = -INFINITY;
    int waiting = 0;

    // Other entries in descending order, zeros last.
    __device__ __forceinline__ void merge_ordered(uint64_t other, int k) {
        const uint64_t turned = other_key<63>(other);              // the 64 best of both: the better of the first and the last, of the second and ...
        if (turned > mine) mine = turned;
        order_halves(mine);
        limit = read_lane(mine, k - 1);
        if (limit != 0) bound = fmaxf(bound, value_of(limit));
    }
    // What an entry of a tile from token `first` on has to be: above the k-th if that is a token in front.  (Where most entries are masked, or many alike,
    // they are not looked at again in each tile.)
    __device__ __forceinline__ float bound_from(uint32_t first) const {
        return limit != 0 && (uint32_t)token_of(limit) < first ? fmaxf(bound, value_above(limit)) : bound;
    }
    // One entry, the same in all lanes, above limit.
    __device__ __forceinline__ void insert(uint64_t key, int k) {
        const uint64_t before = dpp_key<0x138>(mine);              // wave_shr:1, the lane in front's
        const bool behind = mine < key, first = behind && !(lane_id() > 0 && before < key);
        mine = first ? key : behind ? before : mine;
        limit = read_lane(mine, k - 1);
    }
    // `has` lanes' entries: one after the other where they are few, or else to wait until there are 64, or the tile is done.
    __device__ __forceinline__ void offer(bool has, float x, uint32_t v, int k, SelectShared &sh) {
        const uint64_t key = key_of(x, v);
        has = has && key > limit;
        uint64_t lanes = __ballot(has);
        if (k <= kFewBest && waiting == 0 && popc64(lanes) <= kFewKeys) {
            while (lanes != 0) {
                const uint64_t one = read_lane(key, __builtin_ctzll(lanes));
                if (one > limit) insert(one, k);
                lanes &= lanes - 1;
            }
            if (limit != 0) bound = fmaxf(bound, value_of(limit));
            return;
        }
        if (has) sh.wait[waiting + (int)lanes_below(lanes)] = key;
        waiting += (int)popc64(lanes);
        if (waiting >= kWave) take_waiting(kWave, k, sh);
    }
    __device__ __forceinline__ void take_waiting(int n, int k, SelectShared &sh) {
        uint64_t other = lane_id() < n ? sh.wait[lane_id()] : 0;
        order_keys(other);
        merge_ordered(other, k);
        waiting -= n;
        const uint64_t rest = sh.wait[kWave + lane_id()];
        sh.wait[lane_id()] = rest;
    }
    __device__ __forceinline__ void finish(int k, SelectShared &sh) {
        if (waiting > 0) take_waiting(waiting, k, sh);
    }
    // Another wavefront's list.
    __device__ __forceinline__ void join(uint64_t list, int k) {
        if (__ballot(list > limit) != 0) merge_ordered(list, k);
    }
};

// ---------------------------------------------------------------- sums of a tile
// M as RowStat holds it; s = 0: no entry above -inf.
struct Record {
    float m, s, t;
};

// M in base 2, exactly.
__device__ __forceinline__ double base_of(float m) { return fabsf(m) >= kMostM / 2.f ? (double)m * (double)kLog2E : 2.0 * (double)m; }

// r's sums beside an M of `base`, which is not below its own.
__device__ __forceinline__ void rebase(const Record &r, double base, float &s, float &t) {
    // (without entries its M is zero, and may be infinitely far above)
    const float d = fminf(fmaxf((float)(base_of(r.m) - base), -1000.f), 0.f), f = r.s == 0.f ? 0.f : __builtin_amdgcn_exp2f(d);
    s = f * r.s;
    t = f * fmaf(d, r.s, r.t);
}
__device__ __forceinline__ Record joined(const Record &a, const Record &b) {
    if (a.s == 0.f) return b;
    if (b.s == 0.f) return a;
    Record r{fmaxf(a.m, b.m), 0.f, 0.f};
    const double base = base_of(r.m);
    float sa, ta, sb, tb;
    rebase(a, base, sa, ta);
    rebase(b, base, sb, tb);
    r.s = sa + sb;
    r.t = ta + tb;
    return r;
}

// Maxima by the instruction itself: fmaxf quiets its operands first, which doubles what a tile's maxima cost.  A NaN may come out or not; its row's
// results are NaN by the sum.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float max2(float a, float b) {
    float r;
    asm("v_max_f32 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}
__device__ __forceinline__ float wave_max(float v) {
    v = max2(v, dpp_move<0xB1>(v));
    v = max2(v, dpp_move<0x4E>(v));
    v = max2(v, dpp_move<0x141>(v));
    v = max2(v, dpp_move<0x140>(v));
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
    r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = max2(__uint_as_float(r[0]), __uint_as_float(r[1]));
    return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v)));
}

// The largest entry of a piece.
template <class T>
__device__ __forceinline__ float piece_max(Raw r) {
    if constexpr (sizeof(T) == 4) {
        return max3(max2(__uint_as_float(r[0]), __uint_as_float(r[1])), __uint_as_float(r[2]), __uint_as_float(r[3]));
    } else if constexpr (std::is_same<T, __bf16>::value) {
        float f[8];
        unpack<T>(r, f);
        return max3(max3(max3(max2(f[0], f[1]), f[2], f[3]), f[4], f[5]), f[6], f[7]);
    } else {
        uint32_t a, b;
        asm("v_pk_max_f16 %0, %1, %2" : "=v"(a) : "v"(r[0]), "v"(r[1]));
        asm("v_pk_max_f16 %0, %1, %2" : "=v"(b) : "v"(r[2]), "v"(r[3]));
        asm("v_pk_max_f16 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
        typedef _Float16 H2 __attribute__((ext_vector_type(2)));
        const H2 most = __builtin_bit_cast(H2, a);
        return max2((float)most[0], (float)most[1]);
    }
}

// Entry number `entry` of a piece from the word that holds it.
template <class T>
__device__ __forceinline__ float entry_of(uint32_t word, int entry) {
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(word);
    } else {
        const uint16_t half = (uint16_t)(entry & 1 ? word >> 16 : word);
        return (float)__builtin_bit_cast(T, half);
    }
}

template <class T, int EACH>
struct TileOf {
    static constexpr int N = Piece<T>::N;
    Raw raw[EACH];
    float edge;                                                    // an entry of the head or tail: of the row's first tile alone
    bool edges;
    int32_t left;                                                  // pieces from the tile's first on; may be none: a row of edges

    __device__ __forceinline__ void load(const T *x, const Cut &c, int32_t tile) {
        const int32_t lane = lane_id();
        const int64_t base = (int64_t)tile * (EACH * kWave);
        const T *from = x + c.head + base * N;
        left = (int32_t)((int64_t)c.pieces - base);
        if (left >= EACH * kWave) {
#pragma unroll
            for (int u = 0; u < EACH; ++u) raw[u] = load_piece(from + (u * kWave + lane) * N);
        } else {
#pragma unroll
            for (int u = 0; u < EACH; ++u) {
                raw[u] = nothing<T>();
                if (u * kWave + lane < left) raw[u] = load_piece(from + (u * kWave + lane) * N);
            }
        }
        edges = tile == 0 && c.edges() > 0;
        edge = edges && lane < c.edges() ? (float)x[c.edge<T>(lane)] : -INFINITY;
    }

    // The pieces' largest entries, and the lane's.
    __device__ __forceinline__ float maxima(float (&most)[EACH]) const {
        float top = edge;
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            most[u] = piece_max<T>(raw[u]);
            top = max2(top, most[u]);
        }
        return top;
    }

    // An entry of -inf takes no part in t: 2^-200 is zero, and so is its product.  The pieces are unpacked anew: left to itself the compiler keeps what the
    // maxima have unpacked, in 64 registers.
    __device__ __forceinline__ void add(Record &r) {
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            asm("" : "+v"(raw[u]));
            float f[N];
            unpack<T>(raw[u], f);
#pragma unroll
            for (int i = 0; i < N; ++i) add_one(fmaf(f[i], kLog2E, -2.f * r.m), r);
        }
        if (edges) add_one(fmaf(edge, kLog2E, -2.f * r.m), r);
    }
    static __device__ __forceinline__ void add_one(float z, Record &r) {
        const float e = __builtin_amdgcn_exp2f(z);
        r.s += e;
        r.t = fmaf(e, max2(z, -200.f), r.t);
    }

    __device__ __forceinline__ Record sums(const T *x, const Cut &c, int32_t tile, float top) {
        Record r{0.f, 0.f, 0.f};
        if (fabsf(top) < kLargeTop || top == -INFINITY) {
            r.m = top == -INFINITY ? 0.f : 0.5f * __builtin_rintf(top * kLog2E);
            add(r);
        } else if (!(top < INFINITY)) {                            // +inf or NaN
            r.s = r.t = __int_as_float(0x7fc00000);
        } else {                                                   // large: again from memory, piece by piece
            r.m = top;
            const T *from = x + c.head + (int64_t)tile * (EACH * kWave) * N;
#pragma unroll 1
            for (int32_t i = lane_id(); i < min(left, EACH * kWave); i += kWave) {
                float f[N];
                unpack<T>(load_piece(from + i * N), f);
#pragma unroll
                for (int j = 0; j < N; ++j) add_one((f[j] - top) * kLog2E, r);
            }
            if (edges) add_one((edge - top) * kLog2E, r);
        }
        r.s = group_sum<64>(r.s);
        r.t = group_sum<64>(r.t);
        return r;
    }

    // most: the pieces' largest entries.  Pieces that have an entry to offer go to LDS, and from there entry by entry to the lanes.  (Read again from memory
    // instead, with the next tile's loads under way meanwhile: 512 rows of 131072, k = 20: 45 us for 40.)
    __device__ __forceinline__ void select(const Cut &c, int32_t tile, const float (&most)[EACH], float lane_most, float top, int k, Selection &best,
                                           SelectShared &sh) const {
        float bound = best.bound_from((uint32_t)c.head + (uint32_t)(tile * (EACH * kWave)) * N);
        const uint64_t some = __ballot(lane_most >= bound);
        if (some == 0) return;
        const auto reach = [&](float least) {
            int n = 0;
#pragma unroll
            for (int u = 0; u < EACH; ++u) n += (int)popc64(__ballot(most[u] >= least));
            return n;
        };
        const int enough = k + k / 4;
        if ((int)popc64(some) > k / 2 && reach(bound) > enough) {
            // More pieces reach the bound than there are alternatives: halve the way to the largest entry, or from 8 below it, until a few more do.
            // (Where k pieces' maxima reach a bound, k entries do; equal entries may end it early, and so may a way that cannot be halved.)
            float high = top, step = 8.f;
            for (int i = 0; i < 16; ++i) {
                const float middle = fmaxf(0.5f * bound + 0.5f * high, top - step);
                if (!(middle > bound && middle < high)) break;
                const int n = reach(middle);
                if (n >= k) {
                    bound = middle;
                    if (n <= enough) break;
                } else {
                    high = middle;
                    step *= 4.f;
                }
            }
            best.bound = fmaxf(best.bound, bound);
        }
        const int32_t first = tile * (EACH * kWave) + lane_id();
        uint32_t flags = (1u << EACH) - 1u;                        // which of the lanes' pieces are still to be looked at
        do {
            int staged = 0;
#pragma unroll
            for (int u = 0; u < EACH; ++u) {
                const bool has = most[u] >= bound && first + u * kWave < c.pieces;
                const uint64_t lanes = __ballot(has);
                const int n = (int)popc64(lanes);
                if ((flags >> u & 1u) == 0 || staged + n > kWave) continue;
                flags &= ~(1u << u);
                if (lanes == 0) continue;
                if (has) {
                    const int at = staged + (int)lanes_below(lanes);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sh.piece[at][i] = raw[u][i];
                    sh.token[at] = (uint32_t)c.head + (uint32_t)(first + u * kWave) * N;
                }
                staged += n;
            }
            for (int at = 0; at < staged; at += kWave / N) {
                const int from = at + lane_id() / N, entry = lane_id() % N;
                const bool in = from < staged;
                const float x = in ? entry_of<T>(sh.piece[from][entry * (int)sizeof(T) / 4], entry) : 0.f;
                best.offer(in && x >= bound, x, in ? sh.token[from] + entry : 0u, k, sh);
            }
        } while (flags != 0);
        if (edges) best.offer(lane_id() < c.edges() && edge >= best.bound, edge, (uint32_t)c.edge<T>(lane_id()), k, sh);
        if (k <= kFewBest) best.finish(k, sh);
    }
};

// A wavefront takes a slice: its sums, and its entries for the selection.
template <class T, int EACH, bool SELECT>
__device__ __forceinline__ Record take_slice(const T *x, const Cut &c, const Slices &cut, int32_t slice, int k, Selection &best, SelectShared &sh) {
    Record sum{0.f, 0.f, 0.f};
    for (int32_t i = 0; i < cut.tiles; ++i) {
        const int32_t tile = slice * cut.tiles + i;
        if (tile > 0 && (int64_t)tile * (EACH * kWave) >= c.pieces) break;  // a row that has one tile less than its length allows
        TileOf<T, EACH> t;
        t.load(x, c, tile);
        float most[EACH];
        const float top = t.maxima(most);
        const float highest = wave_max(top);
        const Record r = t.sums(x, c, tile, highest);
        sum = joined(sum, r);
        if constexpr (SELECT) t.select(c, tile, most, top, highest, k, best, sh);
    }
    return sum;
}

// ---------------------------------------------------------------- a row's results
struct RowOut {
    RowStat st;
    float entropy;
    bool wrong;
};

// By one wavefront, from the records of all slices in LDS or memory.
__device__ __forceinline__ RowOut row_out(const Record *records, int32_t count) {
    float top = -INFINITY;
    for (int32_t i = lane_id(); i < count; i += kWave) top = records[i].s != 0.f ? fmaxf(top, records[i].m) : top;
    top = group_max<64>(top);
    float s = 0.f, t = 0.f;
    if (top > -INFINITY) {
        const double base = base_of(top);
        for (int32_t i = lane_id(); i < count; i += kWave) {
            float more_s, more_t;
            rebase(records[i], base, more_s, more_t);
            s += more_s;
            t += more_t;
        }
        s = group_sum<64>(s);
        t = group_sum<64>(t);
    }
    RowOut r{{top, -INFINITY}, 0.f, !(s < INFINITY)};
    if (r.wrong) {
        r.st = {0.f, __int_as_float(0x7fc00000)};
        r.entropy = __int_as_float(0x7fc00000);
    } else if (s == 0.f) {
        r.st.m = 0.f;
    } else {
        const float l = log2f(s);
        r.entropy = 0.69314718055994530942f * fmaxf(l - t / s, 0.f);
        if (r.st.large()) r.st.l = l;
        else r.st = stat_of(2.f * top, s);
    }
    return r;
}

__device__ __forceinline__ void write_row(const StatArgs &p, int64_t r, const RowOut &out, float at_label, uint64_t key) {
    const float nan = __int_as_float(0x7fc00000);
    if (lane_id() == 0) {
        if (p.logp) p.logp[r] = out.wrong ? nan : out.st.log_prob(at_label);
        p.lse[r] = out.wrong ? nan : out.st.lse();
        p.entropy[r] = out.entropy;
        if (p.sums) {
            p.sums[2 * r] = out.st.m;
            p.sums[2 * r + 1] = out.st.l;
        }
    }
    if (lane_id() < p.k) {
        p.top_tokens[r * p.k + lane_id()] = out.wrong ? -1 : token_of(key);
        p.top_logp[r * p.k + lane_id()] = out.wrong ? nan : out.st.log_prob(value_of(key));
    }
}
__device__ __forceinline__ void write_ignored(const StatArgs &p, int64_t r) {
    if (lane_id() == 0) {
        if (p.logp) p.logp[r] = 0.f;
        p.lse[r] = p.entropy[r] = 0.f;
        if (p.sums) {
            p.sums[2 * r] = 0.f;
            p.sums[2 * r + 1] = -INFINITY;
        }
    }
    if (lane_id() < p.k) {
        p.top_tokens[r * p.k + lane_id()] = -1;
        p.top_logp[r * p.k + lane_id()] = 0.f;
    }
}

// Whether the row counts; its label's logit.
template <class T>
__device__ __forceinline__ bool row_counts(const LogitRows &in, int64_t r, float &at_label) {
    at_label = 0.f;
    if (!in.labels.ptr) return true;
    const int32_t label = label_of(in, r);
    if (label < 0) return false;
    at_label = (float)(static_cast<const T *>(in.x) + r * in.stride)[label];
    return true;
}

// ---------------------------------------------------------------- kernels
// Wavefronts that a SIMD's registers are shared out among: 128 registers hold a tile and the selection.  With 5 and 6 (the tile spills, or is loaded in
// parts) 8192 rows of 131072 with their gradient take 946 and 1009 us for 937, 4096 rows with 20 alternatives 215 and 262 for 215, and 2048 rows of 50000
// with 57 and 65 for 47.
constexpr int kToSimd = 4;

// A team of WAVES wavefronts per row, which take the slices in turn; the first joins what they found while the others begin the next row.  Teams of one
// share a workgroup of four.
template <class T, int EACH, int WAVES, bool SELECT>
__global__ __launch_bounds__(Team<WAVES>::kBlock, kToSimd) void stats_row_kernel(LogitRows in, StatArgs p) {
    typedef Team<WAVES> G;
    constexpr int kTurns = WAVES == 1 ? 1 : 2;
    __shared__ SelectShared select[G::kBlock / kWave];
    __shared__ Record shared_records[kTurns * G::kPerBlock][EACH == kEach ? kMostSlices : 1];
    __shared__ uint64_t lists[kTurns][WAVES][WAVES == 1 ? 1 : kWave];
    __shared__ RowOut shared_out[kTurns];                          // by the last wavefront where the others take some time to join their lists
    constexpr bool kApart = SELECT && WAVES > 4;
    const Slices cut = slices_of<T>((int32_t)in.vocab);
    SelectShared &sh = select[wave_id()];
    const int member = WAVES == 1 ? 0 : wave_id();
    int turn = 0;
    for (int64_t r = G::first(); r < in.rows; r += G::step()) {
        float at_label;
        if (!row_counts<T>(in, r, at_label)) {
            if (member == 0) write_ignored(p, r);
            continue;
        }
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        const Cut c = cut_row(x, (int32_t)in.vocab);
        Record *records = shared_records[WAVES == 1 ? G::which() : turn];
        Selection best;
        for (int32_t s = member; s < cut.count; s += WAVES) {
            const Record record = take_slice<T, EACH, SELECT>(x, c, cut, s, p.k, best, sh);
            if (lane_id() == 0) records[s] = record;
        }
        if (SELECT) best.finish(p.k, sh);
        if constexpr (WAVES > 1) {
            if (SELECT) lists[turn][member][lane_id()] = best.mine;
            __syncthreads();
        }
        constexpr int kLast = WAVES > 4 ? 2 : WAVES;               // lists that the first wavefront joins alone
        if constexpr (SELECT) {
            if (kApart && member == WAVES - 1) {
                const RowOut out = row_out(records, cut.count);
                if (lane_id() == 0) shared_out[turn] = out;
            }
            for (int half = WAVES / 2; half >= kLast; half /= 2) {
                if (member < half) {
                    best.join(lists[turn][member + half][lane_id()], p.k);
                    lists[turn][member][lane_id()] = best.mine;
                }
                __syncthreads();
            }
        }
        if (member == 0) {
            if (SELECT)
                for (int w = 1; w < kLast; ++w) best.join(lists[turn][w][lane_id()], p.k);
            if constexpr (kApart) write_row(p, r, shared_out[turn], at_label, best.mine);
            else write_row(p, r, row_out(records, cut.count), at_label, best.mine);
        }
        turn ^= 1;
    }
}

// Few rows: a workgroup per part of a row, and a second launch that joins the parts.
struct Parts {
    int32_t slices, count;                                         // slices of a part, parts of a row
    Record *records;                                               // [rows][slices of a row]
    uint64_t *lists;                                               // [rows][parts][k]
};

template <class T, bool SELECT>
__global__ __launch_bounds__(kThreads, kToSimd) void stats_part_kernel(LogitRows in, StatArgs p, Parts parts) {
    __shared__ SelectShared select[kWaves];
    __shared__ uint64_t lists[kWaves][kWave];
    const Slices cut = slices_of<T>((int32_t)in.vocab);
    SelectShared &sh = select[wave_id()];
    const int64_t r = blockIdx.x / (uint32_t)parts.count;
    const int32_t part = (int32_t)(blockIdx.x % (uint32_t)parts.count);
    if (in.labels.ptr && label_of(in, r) < 0) return;
    const T *x = static_cast<const T *>(in.x) + r * in.stride;
    const Cut c = cut_row(x, (int32_t)in.vocab);
    Selection best;
    const int32_t end = min((part + 1) * parts.slices, cut.count);
    for (int32_t s = part * parts.slices + wave_id(); s < end; s += kWaves) {
        const Record record = take_slice<T, kEach, SELECT>(x, c, cut, s, p.k, best, sh);
        if (lane_id() == 0) parts.records[r * cut.count + s] = record;
    }
    if constexpr (!SELECT) return;
    best.finish(p.k, sh);
    lists[wave_id()][lane_id()] = best.mine;
    __syncthreads();
    if (wave_id() != 0) return;
    for (int w = 1; w < kWaves; ++w) best.join(lists[w][lane_id()], p.k);
    if (lane_id() < p.k) parts.lists[(r * parts.count + part) * p.k + lane_id()] = best.mine;
}

// A workgroup per row: the last wavefront takes the sums while the others join the lists.
template <class T>
__global__ __launch_bounds__(kThreads) void stats_join_kernel(LogitRows in, StatArgs p, Parts parts) {
    constexpr int kJoining = kWaves - 1;
    __shared__ uint64_t lists[kJoining][kWave];
    __shared__ RowOut out;
    const int32_t slices = slices_of<T>((int32_t)in.vocab).count;
    const int64_t r = blockIdx.x;
    float at_label;
    if (!row_counts<T>(in, r, at_label)) {
        if (wave_id() == 0) write_ignored(p, r);
        return;
    }
    Selection best;
    if (wave_id() == kJoining) {
        const RowOut sums = row_out(parts.records + r * slices, slices);
        if (lane_id() == 0) out = sums;
    } else if (p.k > 0) {
        for (int32_t i = wave_id(); i < parts.count; i += kJoining)
            best.join(lane_id() < p.k ? parts.lists[(r * parts.count + i) * p.k + lane_id()] : 0, p.k);
        lists[wave_id()][lane_id()] = best.mine;
    }
    __syncthreads();
    if (wave_id() != 0) return;
    if (p.k > 0)
        for (int w = 1; w < kJoining; ++w) best.join(lists[w][lane_id()], p.k);
    write_row(p, r, out, at_label, best.mine);
}

// How a call is cut.  parts.count = 1: without a second launch, `waves` wavefronts to a row.
//   Wavefronts in all: four times the card's SIMDs, as many as are resident.  512 rows of 131072, k = 20: 40 us so, 49 with half as many, 46 with twice
// (each begins a selection of its own); 1024 rows: 66, 84 and 74.
//   A tile to a wavefront where there are enough of them, even if some have none: 64 rows of 20000 fp16 (five tiles), k = 5 11.0 us by eight, 12.7 by four,
// k = 40 11.8 and 16.1.
//   Beyond those rows an alternative's bound is worth most where one wavefront sees the whole row; sums alone gain from four that read neighbouring tiles of
// one row, if it is long: 8192 rows of 131072 937 us (with gradient) for 974, 16384 of 65536 332 for 345; but 50000 274 for 267, and 16000 99 for 91.
constexpr int64_t kWavesInAll = 4096;
inline int waves_of(int64_t rows, int32_t slices, bool select) {
    const int least = select || slices < 16 ? 1 : 4;
    int waves = 1;
    while (waves < 16 && (waves < least || rows * waves * 2 <= kWavesInAll) && waves < slices) waves *= 2;
    return waves;
}
// By parts where a workgroup of 16 wavefronts would take more than one turn and the rows leave the card empty: one row of 131072, k = 20: 13.8 us for 20.3.
// 16 rows of 32000, one turn: 11.9 us by a workgroup each, 13.6 by parts.
template <class T>
Parts parts_of(int64_t rows, int64_t vocab) {
    const Slices cut = slices_of<T>((int32_t)vocab);
    Parts parts{cut.count, 1, nullptr, nullptr};
    if (cut.count <= 16 || rows * 16 >= kWavesInAll) return parts;
    const int64_t most = 2048 / (rows > 0 ? rows : 1);             // parts of a row
    int64_t each = (cut.count + most - 1) / most;
    each = (each + kWaves - 1) / kWaves * kWaves;
    parts.slices = (int32_t)each;
    parts.count = (int32_t)((cut.count + each - 1) / each);
    return parts;
}
size_t up_to_256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---------------------------------------------------------------- gradient
// With y = log2 p:  a ([v = label] - p) - b p (y ln 2 + entropy) = [v = label] a - p (slope y + level).  Where p is zero y is -inf, or far below; from
// -200 on p is zero without it.
struct StatGrad {
    float m, l, slope, level, a;                                   // m: what z subtracts
    int32_t label;                                                 // none: no entry's number
    bool large;
    __device__ __forceinline__ StatGrad(const RowStat &st, float a_, float b, float h, int32_t label_)
        : m(st.large() ? st.m : 2.f * st.m), l(st.l), slope(b * 0.69314718055994530942f), level(fmaf(b, h, a_)), a(a_), label(label_), large(st.large()) {}
    template <bool LARGE>
    __device__ __forceinline__ float of(float x) const {
        const float y = fmaxf((LARGE ? (x - m) * kLog2E : fmaf(x, kLog2E, -m)) - l, -200.f);
        return -(__builtin_amdgcn_exp2f(y) * fmaf(slope, y, level));
    }
    // A piece in which the label is entry `at`, if at < N.
    template <int N>
    __device__ __forceinline__ void piece(uint32_t at, float (&f)[N]) const {
        if (large) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = of<true>(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] = of<false>(f[i]);
        }
        if (at < (uint32_t)N) {
#pragma unroll
            for (int i = 0; i < N; ++i) f[i] += (int)at == i ? a : 0.f;
        }
    }
    __device__ __forceinline__ float entry(int32_t v, float x) const {
        float f[1] = {x};
        piece((uint32_t)label - (uint32_t)v, f);
        return f[0];
    }
};

// Pieces first, first + step, ... (EACH of them) of a row and, where `edges`, an entry of its head or tail for each thread.
template <class T, bool ADD, int EACH>
struct GradPieces {
    static constexpr int N = Piece<T>::N;
    typedef uint32_t Loose __attribute__((ext_vector_type(4), aligned(2)));
    Raw x[EACH], old[EACH];
    __device__ __forceinline__ void load(const T *from, const T *to, const Cut &c, int32_t first, int32_t step) {
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int32_t i = first + u * step;
            if (i >= c.pieces) continue;
            x[u] = load_piece(from + c.head + i * N);
            if constexpr (ADD) old[u] = Raw(__builtin_nontemporal_load(reinterpret_cast<const Loose *>(to + c.head + i * N)));
        }
    }
    __device__ __forceinline__ void store(T *to, const Cut &c, int32_t first, int32_t step, const StatGrad &d) const {
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
            const int32_t i = first + u * step;
            if (i >= c.pieces) continue;
            const int32_t v = c.head + i * N;
            float f[N];
            unpack<T>(x[u], f);
            d.piece((uint32_t)d.label - (uint32_t)v, f);
            if constexpr (ADD) {
                float more[N];
                unpack<T>(old[u], more);
#pragma unroll
                for (int k = 0; k < N; ++k) f[k] += more[k];
            }
            store_piece(to + v, f);
        }
    }
};

// In place of a label where there are none: no entry's number, nor within a piece of one.
constexpr int32_t kNoLabel = -(1 << 30);

// What a row's gradient is of; false: a row of zeros, or one that is left as it is.
template <class T>
__device__ __forceinline__ bool row_grad(const LogitRows &in, const StatGradArgs &p, int64_t r, StatGrad &d) {
    const int32_t label = in.labels.ptr ? label_of(in, r) : kNoLabel;
    const RowStat st{p.sums[2 * r], p.sums[2 * r + 1]};
    d = StatGrad(st, p.grad_logp ? p.grad_logp[r] : 0.f, p.grad_entropy ? p.grad_entropy[r] : 0.f, p.entropy[r], label);
    return label != -1 && !st.empty();
}

// A wavefront per row of up to 512 pieces.
template <class T, bool ADD>
__global__ __launch_bounds__(kThreads) void stats_grad_short_kernel(LogitRows in, StatGradArgs p, LogitGrad out) {
    const int32_t vocab = (int32_t)in.vocab, lane = lane_id();
    for (int64_t r = (int64_t)blockIdx.x * kWaves + wave_id(); r < in.rows; r += (int64_t)gridDim.x * kWaves) {
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        StatGrad d(RowStat{0.f, 0.f}, 0.f, 0.f, 0.f, 0);
        if (!row_grad<T>(in, p, r, d)) {
            if constexpr (!ADD) zero_row<T, kWave>(g, vocab, lane);
            continue;
        }
        const Cut c = cut_row(x, vocab);
        for (int32_t i = lane; i - lane < c.pieces; i += 4 * kWave) {
            GradPieces<T, ADD, 4> t;
            t.load(x, g, c, i, kWave);
            t.store(g, c, i, kWave, d);
        }
        if (lane < c.edges()) {
            const int32_t v = c.edge<T>(lane);
            const float e = d.entry(v, (float)x[v]);
            g[v] = stored<T>(ADD ? (float)g[v] + e : e);
        }
    }
}

// Longer rows in the tiles of token_rows.h, bound by memory: 8192 rows of 131072 bf16, one in eight ignored, in 655 us: 6.15 TB/s, where a plain kernel
// that reads and writes neighbouring stretches reaches 6.4.
template <class T, bool ADD>
__global__ __launch_bounds__(kGradThreads) void stats_grad_kernel(LogitRows in, StatGradArgs p, LogitGrad out, int32_t tiles) {
    const int32_t vocab = (int32_t)in.vocab;
    for (int64_t w = blockIdx.x; w < in.rows * tiles; w += gridDim.x) {
        const int64_t r = w / tiles;
        const int32_t tile = (int32_t)(w % tiles), first = tile * kGradPieces + (int32_t)threadIdx.x;
        const T *x = static_cast<const T *>(in.x) + r * in.stride;
        T *g = static_cast<T *>(out.ptr) + r * out.stride;
        StatGrad d(RowStat{0.f, 0.f}, 0.f, 0.f, 0.f, 0);
        if (!row_grad<T>(in, p, r, d)) {
            if constexpr (!ADD) {
                GradTile<T> t;
                t.load(x, g, vocab, false, tile);
                t.zero(g);
            }
            continue;
        }
        const Cut c = cut_row(x, vocab);
        GradPieces<T, ADD, kGradFlight> t;
        t.load(x, g, c, first, kGradThreads);
        const bool edge = tile == 0 && (int32_t)threadIdx.x < c.edges();
        const int32_t v = edge ? c.edge<T>((int32_t)threadIdx.x) : 0;
        const float x_edge = edge ? (float)x[v] : 0.f;
        t.store(g, c, first, kGradThreads, d);
        if (edge) {
            const float e = d.entry(v, x_edge);
            g[v] = stored<T>(ADD ? (float)g[v] + e : e);
        }
    }
}

}  // namespace

size_t stats_workspace_bytes(int type, int64_t rows, int64_t vocab, int32_t k) {
    size_t bytes = 0;
    (void)with_type(type, [&](auto as) {
        typedef typename ValueOf<decltype(as)::value>::type T;
        const Parts parts = parts_of<T>(rows, vocab);
        if (parts.count > 1)
            bytes = up_to_256((size_t)rows * slices_of<T>((int32_t)vocab).count * sizeof(Record)) + (size_t)rows * parts.count * k * sizeof(uint64_t);
        return hipSuccess;
    });
    return bytes;
}

hipError_t launch_token_stats(const LogitRows &in, const StatArgs &p, void *workspace, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        const Slices cut = slices_of<T>((int32_t)in.vocab);
        Parts parts = parts_of<T>(in.rows, in.vocab);
        const auto launch = [&](auto select) {
            constexpr bool SELECT = decltype(select)::value;
            if (parts.count > 1) {
                parts.records = static_cast<Record *>(workspace);
                parts.lists = reinterpret_cast<uint64_t *>(static_cast<char *>(workspace) + up_to_256((size_t)in.rows * cut.count * sizeof(Record)));
                hipLaunchKernelGGL((stats_part_kernel<T, SELECT>), dim3((unsigned)(in.rows * parts.count)), dim3(kThreads), 0, stream, in, p, parts);
                if (hipError_t st = hipGetLastError()) return st;
                hipLaunchKernelGGL(stats_join_kernel<T>, dim3((unsigned)in.rows), dim3(kThreads), 0, stream, in, p, parts);
                return hipGetLastError();
            }
            const auto rows = [&](auto each, auto waves) {
                typedef Team<decltype(waves)::value> G;
                hipLaunchKernelGGL((stats_row_kernel<T, decltype(each)::value, decltype(waves)::value, SELECT>),
                                   dim3(grid_of(in.rows, G::kPerBlock, G::kBlock)), dim3(G::kBlock), 0, stream, in, p);
                return hipGetLastError();
            };
            const std::integral_constant<int, kEach> each;
            if (is_short<T>(in.vocab)) return rows(std::integral_constant<int, kEachShort>(), std::integral_constant<int, 1>());
            switch (waves_of(in.rows, cut.count, SELECT)) {
                case 1: return rows(each, std::integral_constant<int, 1>());
                case 2: return rows(each, std::integral_constant<int, 2>());
                case 4: return rows(each, std::integral_constant<int, 4>());
                case 8: return rows(each, std::integral_constant<int, 8>());
                default: return rows(each, std::integral_constant<int, 16>());
            }
        };
        return p.k > 0 ? launch(std::true_type()) : launch(std::false_type());
    });
}

hipError_t launch_token_stats_grad(const LogitRows &in, const StatGradArgs &p, const LogitGrad &out, hipStream_t stream) {
    if (in.rows == 0) return hipSuccess;
    return with_type(in.type, [&](auto type) {
        typedef typename ValueOf<decltype(type)::value>::type T;
        const auto launch = [&](auto add) {
            constexpr bool ADD = decltype(add)::value;
            if (in.vocab <= kTile * Piece<T>::N) {
                hipLaunchKernelGGL((stats_grad_short_kernel<T, ADD>), dim3(grid_of(in.rows, kWaves, kThreads)), dim3(kThreads), 0, stream, in, p, out);
            } else {
                const int32_t tiles = grad_tiles<T>(in.vocab);
                hipLaunchKernelGGL((stats_grad_kernel<T, ADD>), dim3(grid_of(in.rows * tiles, 1, kGradThreads)), dim3(kGradThreads), 0, stream, in, p, out, tiles);
            }
            return hipGetLastError();
        };
        return p.accumulate ? launch(std::true_type()) : launch(std::false_type());
    });
}

}  // namespace ef21
