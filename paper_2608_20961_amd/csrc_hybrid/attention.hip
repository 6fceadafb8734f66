// treewy_tree_attention: draft nodes over a paged cache, their ancestors and
// themselves.
//
// One pass over the keys with the running maximum and sum of a softmax.  The
// query rows that share a head's keys (N nodes x H_q / H_kv heads, of one
// sequence, or of the whole batch where the keys are shared) are cut into row
// tiles of WR x 32, the keys into tiles of KT.  A tile's keys and values are
// loaded into LDS asynchronously, one tile ahead, and every wave takes 32 rows
// (WR groups) and every WK-th block of 32 keys of it: scores transposed,
// S^T = K Q^T, so that a lane holds one row's scores, its maximum and sum need
// one exchange between two lanes, and the likelihoods are the second product's
// operand, O^T = V^T P^T, as they stand; V's transpose comes out of LDS by
// transposed reads.
//
// All tiles of a call form one list (first those of shared keys, then sequence
// by sequence), of which every workgroup takes an equal, consecutive part,
// however ragged the lengths.  A row tile ("unit") that one workgroup has
// whole is written at once; the parts of others go to the workspace and are
// joined by a second launch.  Which part a workgroup has follows from the
// lengths, which only the device knows, so that no call waits for them.
#include "hybrid_launch.h"
#include "launch.h"
#include "mfma16.h"
#include "rotate.h"

namespace treewy {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;

__device__ __attribute__((aligned(16))) const uint4 zero_row[64] = {};   // what masked rows load

__device__ __forceinline__ f32x16 mma_f32(float a, float b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0);
}

// Tile and wave shape of a kernel: T and head size, row groups, key groups, keys of a tile.
template <typename T_, int HD_, int WR_, int WK_, int KT_> struct Shape {
    using T = T_;
    static constexpr int HD = HD_, WR = WR_, WK = WK_, KT = KT_;
    static constexpr int RT = 32 * WR, NT = 64 * WR * WK, WAVES = WR * WK;
    static constexpr int E = 16 / (int)sizeof(T), GRAN = HD / E, STEPS = GRAN / 2, DT = HD / 32;
    static constexpr int TILE = KT * GRAN;               // granules of a tile's keys (and of its values)
    static constexpr int LOADS = TILE / 64;              // wave-wide loads of them
    static_assert(KT % (32 * WK) == 0 && LOADS % WAVES == 0, "every wave has as much");
    static_assert((WK - 1) * WR * 32 * HD * 4 <= 2 * TILE * 16, "key groups meet in one tile's LDS");
};

// Where granule g of row r stands in its LDS row: the sixteen lanes that a
// 16-byte read serves at once, and the four rows of a transposed read, meet
// different banks (see swz).  Rows of 128 bytes share a bank row by twos.
template <int GRAN> __device__ __forceinline__ int place(int r, int g) {
    if constexpr (GRAN >= 16) return g ^ swz(r);
    const int a = (r >> 1) & 7;
    return g ^ (((a & 1) << 2) | (a >> 1));
}

// Sizes that follow from the call's, the same for host and device.
struct Cut {
    int G, M;                                            // query heads of a key head, rows of a (sequence, head)
    int units, shared_units;                             // row tiles of a (sequence, head), of a head's shared keys
    int shared_tiles;                                    // key tiles of the shared keys
    int draft_tiles;                                     // summed over a (sequence, head)'s row tiles
    int groups;                                          // workgroups that share the list; 0: one per unit
    int64_t slots;
};

__host__ __device__ inline int draft_tiles_of(int unit, int RT, int KT, int G, int N) {
    const int last = (int)(((int64_t)(unit + 1) * RT - 1) / G);
    return ((last < N ? last : N - 1) + KT) / KT;        // nodes after a row tile's last are nobody's ancestors in it
}

struct Work {
    AttendArgs a;
    Cut c;
    float *part;                                         // [slots][RT/32][HD/32][16][64]
    float2 *ml;                                          // [slots][RT] running maximum (log2) and sum
};

// ---- the list of tiles -----------------------------------------------------------
__device__ __forceinline__ int cached(const AttendArgs &a, int b) {
    const int64_t room = min((int64_t)a.max_pages << a.log2_page, (int64_t)1 << 30);
    return (int)min((int64_t)max(a.len[b], 0), room);
}

struct List {
    int64_t total, shared;                               // tiles of all, of the shared keys
    int groups;                                          // workgroups that have some
    int longest;                                         // a sequence with the most cached tokens
};

template <int KT> __device__ __forceinline__ int64_t tiles_of(const Work &w, int len) {
    const int own = max(len - w.a.shared, 0);
    return (int64_t)w.a.H_kv * ((int64_t)w.c.units * ((own + KT - 1) / KT) + w.c.draft_tiles);
}

// One wave: the list's length, and how many tiles lie before sequence `until`.
template <int KT> __device__ __forceinline__ List measure(const Work &w, int until, int64_t &before) {
    const int lane = threadIdx.x & 63;
    int64_t all = 0, part = 0;
    int most = -1, who = 0;
    for (int b = lane; b < w.a.B; b += 64) {
        const int len = cached(w.a, b);
        const int64_t t = tiles_of<KT>(w, len);
        all += t;
        part += b < until ? t : 0;
        if (len > most) most = len, who = b;
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        all += __shfl_xor(all, d);
        part += __shfl_xor(part, d);
        const int m = __shfl_xor(most, d), o = __shfl_xor(who, d);
        if (m > most || (m == most && o < who)) most = m, who = o;
    }
    List l;
    l.shared = (int64_t)w.a.H_kv * w.c.shared_units * w.c.shared_tiles;
    l.total = l.shared + all;
    l.groups = (int)min((int64_t)w.c.groups, l.total);
    l.longest = who;
    before = l.shared + part;
    return l;
}

// One wave: the sequence that tile `at` (past the shared ones) belongs to, and its first tile.
template <int KT> __device__ __forceinline__ int locate(const Work &w, const List &l, int64_t at, int64_t &first) {
    const int lane = threadIdx.x & 63;
    int64_t base = l.shared;
    for (int b0 = 0; b0 < w.a.B; b0 += 64) {
        const int64_t t = b0 + lane < w.a.B ? tiles_of<KT>(w, cached(w.a, b0 + lane)) : 0;
        int64_t s = t;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t y = __shfl_up(s, d);
            if (lane >= d) s += y;
        }
        const uint64_t past = __ballot(base + s > at);
        if (past) {
            const int i = __builtin_ctzll(past);
            first = base + __shfl(s - t, i);
            return b0 + i;
        }
        base += __shfl(s, 63);
    }
    first = base;
    return w.a.B;
}

// Workgroup whose part holds tile x, and the first tile of workgroup g.
__device__ __forceinline__ int64_t first_of(int64_t total, int groups, int64_t g) { return total * g / groups; }
__device__ __forceinline__ int group_of(int64_t total, int groups, int64_t x) { return (int)(((x + 1) * groups - 1) / total); }

// Where group g puts its part of the unit with tiles [begin, end): a group has at most one part that does not begin its unit,
// and one that begins it and does not end it.
__device__ __forceinline__ int64_t slot_of(int groups, int64_t unit, bool begins, bool ends, int g) {
    return begins && ends ? 2 * (int64_t)groups + unit : 2 * (int64_t)g + (begins ? 1 : 0);
}

// ---- results -----------------------------------------------------------------
// A lane's column of O^T: values dt 32 + 8 j + 4 hg + 0 .. 3 of its row, j = 0 .. 3.
template <typename T> __device__ __forceinline__ void store_row(T *o, int dt, int hg, const f32x16 &x, float scale) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x4 y = f32x4{x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]} * scale;
        T *at = o + dt * 32 + 8 * j + 4 * hg;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2 *>(at) = f32_to_bf4(y);
        else *reinterpret_cast<f32x4 *>(at) = y;
    }
}

template <typename T> __device__ __forceinline__ T *out_row(const AttendArgs &a, int b, int head, int n) {
    return (T *)a.o + b * a.os.seq + head * a.os.head + n * a.os.token;
}

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// ---- the kernel ----------------------------------------------------------------
template <typename S> struct Lds {
    typedef uint4 Tile[2 * S::TILE];                     // keys, then values
    uint32_t sees[MAX_TREE][MAX_TREE / 32];              // ancestors and self, a bit each
    int16_t up[MAX_TREE];                                // the next pointer jump's target
    int16_t depth[MAX_TREE];                             // ancestors
    uint32_t odd[MAX_TREE / 32];                         // nodes whose values hold an infinity or NaN, a bit each
};

// Whether 16 bytes hold an infinity or NaN; and those as zeros.
template <typename T> __device__ __forceinline__ bool not_finite(uint4 x) {
    constexpr uint32_t E = 0x7f800000u;
    bool odd = false;
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) odd |= (w[i] & E) == E || (sizeof(T) == 2 && (w[i] << 16 & E) == E);
    return odd;
}
template <typename T> __device__ __forceinline__ uint4 finite(uint4 x) {
    float f[Granule<T>::N];
    Granule<T>::wide(x, f);
#pragma unroll
    for (int i = 0; i < Granule<T>::N; ++i) f[i] = fabsf(f[i]) < INFINITY ? f[i] : 0.0f;
    return Granule<T>::narrow(f);
}

// Ancestors of every node of sequence b by pointer jumping; a bad parent counts as -1.
template <typename S> __device__ void climb(Lds<S> &s, const AttendArgs &a, int b) {
    constexpr int W = MAX_TREE / 32, PER = (MAX_TREE + S::NT - 1) / S::NT;
    const int words = (a.N + 31) / 32;
    __syncthreads();
    for (int t = threadIdx.x; t < a.N; t += S::NT) {
        int p = a.parent[(int64_t)b * a.N + t];
        if (p < -1 || p >= t) {
            flag_error(a.err, b, TREEWY_FLAG_BAD_PARENT);
            p = -1;
        }
        for (int i = 0; i < words; ++i) s.sees[t][i] = i == t / 32 ? 1u << (t % 32) : 0u;
        s.up[t] = (int16_t)p;
    }
    for (bool more = true; more;) {
        __syncthreads();
        uint32_t add[PER][W];
        int next[PER];
        bool any = false;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int t = threadIdx.x + k * S::NT;
            next[k] = -1;
            const int p = t < a.N ? s.up[t] : -1;
#pragma unroll
            for (int i = 0; i < W; ++i) add[k][i] = p >= 0 && i < words ? s.sees[p][i] : 0u;
            if (p >= 0) next[k] = s.up[p];
            any |= next[k] >= 0;
        }
        more = __syncthreads_or(any);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int t = threadIdx.x + k * S::NT;
            if (t < a.N) {
#pragma unroll
                for (int i = 0; i < W; ++i)
                    if (i < words) s.sees[t][i] |= add[k][i];
                s.up[t] = (int16_t)next[k];
            }
        }
    }
    __syncthreads();
    for (int t = threadIdx.x; t < a.N; t += S::NT) {
        int n = -1;
        for (int i = 0; i < words; ++i) n += __popc(s.sees[t][i]);
        s.depth[t] = (int16_t)n;
    }
    __syncthreads();
}

// A unit: a row tile with the tiles of its keys.
struct Unit {
    bool shared;
    int b, h, rt;                                        // (b: whose page table is read)
    int old_tiles, tiles;                                // tiles of cached keys, of all
    int first_key, len;                                  // the cached keys [first_key, len)
};

// One lane's query row.
struct Row {
    bool live;
    int b, n, head, pos, limit;                          // cached keys below `limit` are seen
};

template <typename S> struct Part {
    const Work &w;
    const AttendArgs &a;
    Lds<S> &s;
    const Unit &u;
    const int lane, wave, hg, wr, wk;
    Row row;
    uint4 q[S::STEPS];
    f32x16 acc[S::DT];
    float m, l, c;

    using T = typename S::T;
    static constexpr int E = S::E, GRAN = S::GRAN, KT = S::KT;

    __device__ __forceinline__ Part(const Work &w, Lds<S> &s, const Unit &u)
        : w(w), a(w.a), s(s), u(u), lane(threadIdx.x & 63), wave(__builtin_amdgcn_readfirstlane(threadIdx.x >> 6)),
          hg(lane >> 5), wr(wave / S::WK), wk(wave % S::WK) {}

    __device__ __forceinline__ bool chain() const { return a.parent == nullptr; }
    __device__ __forceinline__ int position(int len, int before, int b) const {
        const int p = len + before;
        if (a.rot && p >= a.positions) {
            flag_error(a.err, b, TREEWY_FLAG_CACHE_FULL);
            return a.positions - 1;
        }
        return p;
    }

    __device__ __forceinline__ void begin() {
        const int r = u.rt * S::RT + wr * 32 + (lane & 31);
        const int64_t rows = u.shared ? (int64_t)a.B * w.c.M : w.c.M;
        row.live = r < rows;
        const int x = row.live ? r : 0;
        row.b = u.shared ? x / w.c.M : u.b;
        const int rr = u.shared ? x - row.b * w.c.M : x;
        row.n = rr / w.c.G;
        row.head = u.h * w.c.G + rr - row.n * w.c.G;
        const int len = u.shared ? cached(a, row.b) : u.len;
        row.limit = u.shared ? min(len, u.len) : u.len;
        int before = row.n;
        if (!chain()) {
            if (!u.shared) before = s.depth[row.n];
            else {                                       // (few nodes where keys are shared)
                before = 0;
                for (int t = row.n;;) {
                    const int p = a.parent[(int64_t)row.b * a.N + t];
                    if (p < 0 || p >= t) break;
                    t = p;
                    ++before;
                }
            }
        }
        row.pos = position(len, before, row.b);
        if (a.len[row.b] != len) flag_error(a.err, row.b, TREEWY_FLAG_CACHE_FULL);

        // the row's granules 2 i + hg, rotated, in the scale's sign
        const uint4 *src = reinterpret_cast<const uint4 *>((const T *)a.q + row.b * a.qs.seq + row.head * a.qs.head +
                                                           row.n * a.qs.token);
        const int half = a.rot / (2 * E);
        const uint32_t flip = a.scale < 0.0f ? (sizeof(T) == 2 ? 0x80008000u : 0x80000000u) : 0u;
#pragma unroll
        for (int i = 0; i < S::STEPS; ++i) {
            const int g = 2 * i + hg;
            uint4 x = src[g];
            if (g < 2 * half) {
                const bool second = g >= half;
                const int i0 = second ? g - half : g;
                Angles<T> w;
                w.load(a.cos, a.sin, (int64_t)row.pos * (a.rot / 2), i0 * E);
                x = rotated<T>(x, src[second ? i0 : g + half], w, second);
            }
            q[i] = make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
        }
        c = fmaxf(fabsf(a.scale) * LOG2E, 1e-30f);       // (a zero scale must not meet a masked score's infinity)
        m = -INFINITY;
        l = 0.0f;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) acc[dt] = f32x16{};
    }

    // The page of lane p's tokens in tile t: the tile's p-th page, -1 where it has none or an invalid one.
    __device__ __forceinline__ int page_of(int t) {
        const int key0 = u.first_key + t * KT, end = min(key0 + KT, u.len);
        const int page = (key0 >> a.log2_page) + lane;
        int id = -1;
        if (t < u.old_tiles && page <= (end - 1) >> a.log2_page) {
            id = a.table[(int64_t)u.b * a.max_pages + page];
            if (id < 0 || id >= a.n_pages) {
                id = -1;
                if (u.shared) {                          // (every sequence that has the page says so)
                    for (int b = 0; b < a.B; ++b)
                        if (cached(a, b) > page << a.log2_page) flag_error(a.err, b, TREEWY_FLAG_BAD_PAGE);
                } else flag_error(a.err, u.b, TREEWY_FLAG_BAD_PAGE);
            }
        }
        return id;
    }

    // Issues the loads of tile t, whose pages page_of gave, into `tile`.
    __device__ __forceinline__ void fetch(uint4 *tile, int t, int pages) {
        if (t < u.old_tiles) {
            const int key0 = u.first_key + t * KT, base = key0 >> a.log2_page;
#pragma unroll
            for (int i = 0; i < S::LOADS / S::WAVES; ++i) {
                const int load = i * S::WAVES + wave, at = load * 64 + lane;
                const int r = at / GRAN, g = place<GRAN>(r, at % GRAN), key = key0 + r;
                const int id = __shfl(pages, ((key >> a.log2_page) - base) & 63);
                const bool have = key < u.len && id >= 0;
                const int64_t off =
                    ((((int64_t)id * a.H_kv + u.h) << a.log2_page) + (key & ((1 << a.log2_page) - 1))) * GRAN + g;
                const uint4 *k = have ? (const uint4 *)a.k_pages + off : zero_row + g % 64;
                const uint4 *v = have ? (const uint4 *)a.v_pages + off : zero_row + g % 64;
                __builtin_amdgcn_global_load_lds((global_void *)k, (lds_void *)(tile + load * 64), 16, 0, 0);
                __builtin_amdgcn_global_load_lds((global_void *)v, (lds_void *)(tile + S::TILE + load * 64), 16, 0, 0);
            }
            return;
        }
        // The draft's own: keys rotated to their positions.  A node's infinities and NaNs must not reach the nodes that do
        // not see it (zero times them is NaN), so values go in without them and odd_values adds them where they are seen.
        const int node0 = (t - u.old_tiles) * KT, half = a.rot / (2 * E);
        for (int i = threadIdx.x; i < KT * GRAN / 2; i += S::NT) {
            const int r = i / (GRAN / 2), p = i % (GRAN / 2), n = node0 + r;
            const bool turns = p < half;
            const int lo = turns ? p : half + p, hi = turns ? p + half : lo + (GRAN / 2 - half);
            uint4 x = make_uint4(0, 0, 0, 0), y = x, v0 = x, v1 = x;
            if (n < a.N) {
                const uint4 *k = reinterpret_cast<const uint4 *>((const T *)a.k + u.b * a.ks.seq + u.h * a.ks.head + n * a.ks.token);
                const uint4 *v = reinterpret_cast<const uint4 *>((const T *)a.v + u.b * a.vs.seq + u.h * a.vs.head + n * a.vs.token);
                x = k[lo];
                y = k[hi];
                v0 = v[lo];
                v1 = v[hi];
                if (turns) {
                    Angles<T> w;
                    w.load(a.cos, a.sin, (int64_t)position(u.len, chain() ? n : s.depth[n], u.b) * (a.rot / 2), p * E);
                    const uint4 first = rotated<T>(x, y, w, false);
                    y = rotated<T>(y, x, w, true);
                    x = first;
                }
                if (not_finite<T>(v0) || not_finite<T>(v1)) {
                    atomicOr(&s.odd[n / 32], 1u << (n % 32));
                    v0 = finite<T>(v0);
                    v1 = finite<T>(v1);
                }
            }
            tile[r * GRAN + place<GRAN>(r, lo)] = x;
            tile[r * GRAN + place<GRAN>(r, hi)] = y;
            tile[S::TILE + r * GRAN + place<GRAN>(r, lo)] = v0;
            tile[S::TILE + r * GRAN + place<GRAN>(r, hi)] = v1;
        }
    }

    __device__ __forceinline__ bool sees(int node) const {
        return chain() ? node <= row.n : (s.sees[row.n][node / 32] >> (node % 32)) & 1u;
    }

    // The infinities and NaNs that were left out of the draft's values, where they are seen.
    __device__ void odd_values() {
        for (int i = 0; i < (a.N + 31) / 32; ++i)
            for (uint32_t bits = s.odd[i]; bits; bits &= bits - 1) {
                const int n = 32 * i + __builtin_ctz(bits);
                if (!sees(n)) continue;
                const T *v = (const T *)a.v + u.b * a.vs.seq + u.h * a.vs.head + n * a.vs.token;
#pragma unroll
                for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const float x = to_f32(v[dt * 32 + acc_row(r, hg)]);
                        if (!(fabsf(x) < INFINITY)) acc[dt][r] += x;
                    }
            }
    }

    // Scores of the block of 32 keys that begins at row k0 of `tile`.
    __device__ __forceinline__ f32x16 scores(const uint4 *tile, int k0) {
        f32x16 x{};
        const int r = k0 + (lane & 31);
#pragma unroll
        for (int i = 0; i < S::STEPS; ++i) {
            const uint4 k = tile[r * GRAN + place<GRAN>(r, 2 * i + hg)];
            if constexpr (sizeof(T) == 2) {
                x = mma(__builtin_bit_cast(bf16x8, k), __builtin_bit_cast(bf16x8, q[i]), x);
            } else {
                const f32x4 kf = __builtin_bit_cast(f32x4, k), qf = __builtin_bit_cast(f32x4, q[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) x = mma_f32(kf[e], qf[e], x);
            }
        }
        return x;
    }

    // Adds V^T P^T of the block.
    __device__ __forceinline__ void add_values(const uint4 *tile, int k0, const f32x16 &p) {
        const uint4 *v = tile + S::TILE;
        if constexpr (sizeof(T) == 2) {
            bf16x8 pb[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = pack_bf2(p[8 * h + 2 * j], p[8 * h + 2 * j + 1]);
                pb[h] = __builtin_bit_cast(bf16x8, x);
            }
            const int j = (lane >> 2) & 3, y = lane & 3, c16 = (lane >> 4) & 1;
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt) {
                const int g = dt * 4 + c16 * 2 + (y >> 1);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s16x4 x[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int r = k0 + 16 * h + 8 * e + 4 * hg + j;
                        const char *at = reinterpret_cast<const char *>(v + r * GRAN + place<GRAN>(r, g)) + (y & 1) * 8;
                        x[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)at);
                    }
                    acc[dt] = mma(both8(__builtin_bit_cast(uint2, x[0]), __builtin_bit_cast(uint2, x[1])), pb[h], acc[dt]);
                }
            }
        } else {
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int key = k0 + acc_row(r, hg), d = dt * 32 + (lane & 31);
                    const float x = reinterpret_cast<const float *>(v + key * GRAN + place<GRAN>(key, d / 4))[d % 4];
                    acc[dt] = mma_f32(x, p[r], acc[dt]);
                }
        }
    }

    __device__ __forceinline__ void compute(const uint4 *tile, int t, int pages) {
        const bool old = t < u.old_tiles;
        const int key0 = old ? u.first_key + t * KT : (t - u.old_tiles) * KT;
        if (!__any(row.live)) return;
        uint64_t bad = 0;
        if (old) {
            const int n_pages = ((min(key0 + KT, u.len) - 1) >> a.log2_page) - (key0 >> a.log2_page) + 1;
            bad = __ballot(lane < n_pages && pages < 0);
        }
#pragma unroll 1
        for (int kb = wk; kb < KT / 32; kb += S::WK) {
            const int first = key0 + kb * 32;
            if (old ? first >= u.len : first >= a.N) break;
            f32x16 x = scores(tile, kb * 32);
            if (old) {
                if (__any(first + 32 > row.limit)) {
                    const int rel = row.limit - first;
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[r] = acc_row(r, hg) < rel ? x[r] : -INFINITY;
                }
                if (bad) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int page = ((first + acc_row(r, hg)) >> a.log2_page) - (key0 >> a.log2_page);
                        x[r] = (bad >> (page & 63)) & 1 ? -INFINITY : x[r];
                    }
                }
            } else {
                const int ahead = row.n - first;
                uint32_t sees = chain() ? (ahead >= 31 ? ~0u : ahead < 0 ? 0u : (2u << ahead) - 1u) : s.sees[row.n][first / 32];
                sees >>= 4 * hg;
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = (sees >> acc_row(r, 0)) & 1u ? x[r] : -INFINITY;
            }
            float top = x[0];
#pragma unroll
            for (int r = 1; r < 16; ++r) top = fmaxf(top, x[r]);
            top = fmaxf(top, other_half(top));
            // Sums are held relative to a maximum that may lag behind by a factor of 2^8: rescaling is rare then.
            if (__any((top - m) * c > 8.0f)) {
                const float to = fmaxf(m, top);
                const float by = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
                m = to;
                l *= by;
#pragma unroll
                for (int dt = 0; dt < S::DT; ++dt) acc[dt] *= by;
            }
            const float at = m == -INFINITY ? 0.0f : m * c;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                x[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r], c, -at));
                l += x[r];
            }
            add_values(tile, kb * 32, x);
        }
    }

    // Joins the key groups of each row group in its first wave.
    __device__ __forceinline__ void join(float *lds) {
        l += other_half(l);
        if constexpr (S::WK > 1) {
            constexpr int WAVE = S::DT * 16 * 64;
            __syncthreads();
            if (wk > 0) {
                float *to = lds + ((wk - 1) * S::WR + wr) * WAVE;
#pragma unroll
                for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
                    for (int r = 0; r < 16; ++r) to[(dt * 16 + r) * 64 + lane] = acc[dt][r];
                float2 *st = reinterpret_cast<float2 *>(s.sees);                       // (the masks are done with)
                st[wave * 64 + lane] = make_float2(m, l);
            }
            __syncthreads();
            if (wk == 0) {
#pragma unroll
                for (int k = 1; k < S::WK; ++k) {
                    const float2 o = reinterpret_cast<const float2 *>(s.sees)[(wave + k) * 64 + lane];
                    const float to = fmaxf(m, o.x);
                    const float by = m == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((m - to) * c);
                    const float oby = o.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f((o.x - to) * c);
                    const float *from = lds + ((k - 1) * S::WR + wr) * WAVE;
                    m = to;
                    l = l * by + o.y * oby;
#pragma unroll
                    for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[dt][r] = acc[dt][r] * by + from[(dt * 16 + r) * 64 + lane] * oby;
                }
            }
        }
    }

    __device__ __forceinline__ void finish() {           // a whole unit without shared keys
        if (wk != 0 || !row.live) return;
        T *o = out_row<T>(a, row.b, row.head, row.n);
        const float by = 1.0f / l;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) store_row<T>(o, dt, hg, acc[dt], by);
    }

    __device__ __forceinline__ void leave(int64_t slot) {
        if (wk != 0 || !__any(row.live)) return;
        float *to = w.part + (slot * S::WR + wr) * (32 * S::HD);
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; ++r) to[(dt * 16 + r) * 64 + lane] = acc[dt][r];
        if (hg == 0) w.ml[slot * S::RT + wr * 32 + lane] = make_float2(m == -INFINITY ? -INFINITY : m * c, l);
    }
};

// Waits for this wave's loads into LDS.
__device__ __forceinline__ void loads_done() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }

template <typename S> __global__ __launch_bounds__(S::NT) void attend_kernel(Work w) {
    constexpr int KT = S::KT, RT = S::RT;
    __shared__ typename Lds<S>::Tile tile0, tile1;
    __shared__ Lds<S> s;
    const AttendArgs &a = w.a;
    // Consecutive parts of the list on one XCD (workgroups go to the eight in turn): row tiles that read the same keys meet in its L2.
    const unsigned blocks = gridDim.x, per = blocks / 8;
    int g = blockIdx.x, groups = 0;
    if (blockIdx.x < per * 8) g = (int)((blockIdx.x & 7u) * per + (blockIdx.x >> 3));

    int64_t at, end, first;                              // this group's tiles, and the current sequence's first
    int b = -1, longest = 0;
    if (w.c.groups) {
        int64_t unused;
        const List list = measure<KT>(w, 0, unused);
        groups = list.groups;
        if (groups < w.c.groups) g = blockIdx.x;         // (fewer tiles than workgroups: one each, on all XCDs)
        if (g >= groups) return;
        at = first_of(list.total, groups, g);
        end = first_of(list.total, groups, g + 1);
        longest = list.longest;
        if (at >= list.shared) b = locate<KT>(w, list, at, first);
        else first = list.shared;
        at = __builtin_amdgcn_readfirstlane((int)(at >> 32)) * ((int64_t)1 << 32) + (uint32_t)__builtin_amdgcn_readfirstlane((int)at);
        end = __builtin_amdgcn_readfirstlane((int)(end >> 32)) * ((int64_t)1 << 32) + (uint32_t)__builtin_amdgcn_readfirstlane((int)end);
        first = __builtin_amdgcn_readfirstlane((int)(first >> 32)) * ((int64_t)1 << 32) +
                (uint32_t)__builtin_amdgcn_readfirstlane((int)first);
        b = __builtin_amdgcn_readfirstlane(b);
    } else {                                             // one unit: its place in the list does not matter
        b = g / (a.H_kv * w.c.units);
        at = first = 0;
        end = 1;
    }
    int climbed = -1;
    const int64_t shared_all = (int64_t)a.H_kv * w.c.shared_units * w.c.shared_tiles;
    while (at < end) {
        // the unit that tile `at` belongs to, and its tiles [begin, begin + tiles) in the list
        Unit u;
        int64_t begin, id;
        u.shared = b < 0;
        if (u.shared) {
            const int n = (int)(at / w.c.shared_tiles);
            id = n;
            u.h = n / w.c.shared_units;
            u.rt = n - u.h * w.c.shared_units;
            u.b = longest;
            u.first_key = 0;
            u.len = min(a.shared, cached(a, u.b));
            u.old_tiles = u.tiles = w.c.shared_tiles;
            begin = (int64_t)n * w.c.shared_tiles;
        } else {
            const int len = cached(a, b);
            u.b = b;
            u.len = len;
            u.first_key = min(a.shared, len);
            u.old_tiles = (len - u.first_key + KT - 1) / KT;
            const int per_head = w.c.units * u.old_tiles + w.c.draft_tiles;
            if (w.c.groups) {
                int left = (int)(at - first);
                u.h = left / per_head;
                left -= u.h * per_head;
                for (u.rt = 0;; ++u.rt) {
                    u.tiles = u.old_tiles + draft_tiles_of(u.rt, RT, KT, w.c.G, a.N);
                    if (left < u.tiles) break;
                    left -= u.tiles;
                }
                begin = at - left;
            } else {
                const int n = g - b * a.H_kv * w.c.units;
                u.h = n / w.c.units;
                u.rt = n - u.h * w.c.units;
                u.tiles = u.old_tiles + draft_tiles_of(u.rt, RT, KT, w.c.G, a.N);
                begin = 0;
                end = u.tiles;
            }
            id = (int64_t)a.H_kv * w.c.shared_units + ((int64_t)b * a.H_kv + u.h) * w.c.units + u.rt;
        }
        const int t0 = (int)(at - begin), t1 = (int)min((int64_t)u.tiles, end - begin);
        if (!u.shared && a.parent && climbed != b) {
            climb<S>(s, a, b);
            climbed = b;
        }
        {
            Part<S> p(w, s, u);
            __syncthreads();                             // (the last part's LDS is read)
            if (threadIdx.x < MAX_TREE / 32) s.odd[threadIdx.x] = 0;
            __syncthreads();
            int pages = p.page_of(t0), ahead = p.page_of(t0 + 1);
            p.fetch(tile0, t0, pages);
            p.begin();
            auto step = [&](uint4 *here, uint4 *next, int t) {
                loads_done();
                __syncthreads();
                const int now = pages;
                pages = ahead;
                if (t + 1 < t1) {
                    p.fetch(next, t + 1, pages);
                    ahead = p.page_of(t + 2);
                }
                p.compute(here, t, now);
            };
            for (int t = t0; t < t1; t += 2) {
                step(tile0, tile1, t);
                if (t + 1 < t1) step(tile1, tile0, t + 1);
            }
            if (!u.shared && p.wk == 0) p.odd_values();
            p.join(reinterpret_cast<float *>(tile0));
            if constexpr (S::WK > 1) climbed = -1;       // (join wrote over the masks)
            const bool whole = t0 == 0 && t1 == u.tiles;
            if (whole && w.c.shared_tiles == 0) p.finish();
            else p.leave(slot_of(w.c.groups, id, t0 == 0, t1 == u.tiles, g));
        }
        at = begin + t1;
        if (!w.c.groups) break;
        if (u.shared) {
            if (at >= shared_all) b = 0, first = at;
        } else if (u.h == a.H_kv - 1 && u.rt == w.c.units - 1 && t1 == u.tiles) {
            ++b;
            first = at;
        }
    }
}

// Joins the parts of the units that were cut: a workgroup per (unit, 32 rows, 32 values), its waves sharing the parts.
template <typename S> __global__ __launch_bounds__(256) void join_kernel(Work w) {
    constexpr int KT = S::KT, RT = S::RT, DT = S::DT;
    using T = typename S::T;
    __shared__ float sums[4][17][64], tops[4][64];
    const AttendArgs &a = w.a;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hg = lane >> 5;
    const int dt = blockIdx.x % DT, wr = blockIdx.x / DT % S::WR, unit = blockIdx.x / (DT * S::WR);
    const int b = unit / (a.H_kv * w.c.units), n = unit - b * a.H_kv * w.c.units, h = n / w.c.units, rt = n - h * w.c.units;
    const int r = rt * RT + wr * 32 + (lane & 31);
    if (rt * RT + wr * 32 >= w.c.M) return;
    int64_t before;
    const List list = measure<KT>(w, b, before);
    const int len = cached(a, b), old = (max(len - a.shared, 0) + KT - 1) / KT;
    int64_t begin = before + (int64_t)h * (w.c.units * old + w.c.draft_tiles);
    for (int i = 0; i < rt; ++i) begin += old + draft_tiles_of(i, RT, KT, w.c.G, a.N);
    const int64_t end = begin + old + draft_tiles_of(rt, RT, KT, w.c.G, a.N);
    const int64_t shared_ids = (int64_t)a.H_kv * w.c.shared_units;

    // the parts of the row's own unit, then of its unit of shared keys
    struct Span {
        int first, count, lane;
        int64_t unit;
    } span[2];
    span[0].first = group_of(list.total, list.groups, begin);
    span[0].count = group_of(list.total, list.groups, end - 1) - span[0].first + 1;
    span[0].unit = shared_ids + unit;
    span[0].lane = wr * 32 + (lane & 31);
    span[1].count = 0;
    if (w.c.shared_tiles == 0 && span[0].count == 1) return;          // written already
    const bool live = r < w.c.M;
    if (w.c.shared_tiles && live) {
        const int64_t row = (int64_t)b * w.c.M + r;
        const int64_t id = (int64_t)h * w.c.shared_units + row / RT;
        span[1].first = group_of(list.total, list.groups, id * w.c.shared_tiles);
        span[1].count = group_of(list.total, list.groups, (id + 1) * w.c.shared_tiles - 1) - span[1].first + 1;
        span[1].unit = id;
        span[1].lane = (int)(row % RT);
    }
    auto slot = [&](const Span &x, int i) {
        return slot_of(w.c.groups, x.unit, i == 0, i == x.count - 1, x.first + i);
    };
    float top = -INFINITY;
    if (live)
        for (int k = 0; k < 2; ++k)
            for (int i = wave; i < span[k].count; i += 4) top = fmaxf(top, w.ml[slot(span[k], i) * RT + span[k].lane].x);
    tops[wave][lane] = top;
    __syncthreads();
    for (int i = 0; i < 4; ++i) top = fmaxf(top, tops[i][lane]);
    float sum = 0.0f, x[16] = {};
    if (live)
        for (int k = 0; k < 2; ++k)
            for (int i = wave; i < span[k].count; i += 4) {
                const int64_t at = slot(span[k], i);
                const float2 ml = w.ml[at * RT + span[k].lane];
                const float by = ml.x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(ml.x - top);
                sum += by * ml.y;
                const float *from = w.part + ((at * S::WR + span[k].lane / 32) * DT + dt) * 1024 + hg * 32 + span[k].lane % 32;
#pragma unroll
                for (int j = 0; j < 16; ++j) x[j] += by * from[j * 64];
            }
#pragma unroll
    for (int j = 0; j < 16; ++j) sums[wave][j][lane] = x[j];
    sums[wave][16][lane] = sum;
    __syncthreads();
    if (wave != 0 || !live) return;
    f32x16 o;
    for (int i = 1; i < 4; ++i) sum += sums[i][16][lane];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        o[j] = x[j];
        for (int i = 1; i < 4; ++i) o[j] += sums[i][j][lane];
    }
    const int node = r / w.c.G;
    store_row<T>(out_row<T>(a, b, h * w.c.G + r - node * w.c.G, node), dt, hg, o, 1.0f / sum);
}

// ---- host ----------------------------------------------------------------------
template <typename S> Cut cut(int shared, int N, int B, int H_q, int H_kv) {
    Cut c{};
    c.G = H_q / H_kv;
    c.M = N * c.G;
    c.units = (c.M + S::RT - 1) / S::RT;
    for (int i = 0; i < c.units; ++i) c.draft_tiles += draft_tiles_of(i, S::RT, S::KT, c.G, N);
    const int64_t all = (int64_t)B * H_kv * c.units;
    if (shared > 0) {
        c.shared_units = (int)(((int64_t)B * c.M + S::RT - 1) / S::RT);
        c.shared_tiles = (shared + S::KT - 1) / S::KT;
    }
    const int resident = compute_units() * (2 * (int)sizeof(typename Lds<S>::Tile) > 65536 + 16384 ? 1 : 2);
    if (shared == 0 && all >= 3 * (int64_t)resident) return c;        // enough units to even themselves out
    c.groups = resident;
    c.slots = 2 * (int64_t)resident + (shared > 0 ? (int64_t)H_kv * c.shared_units + all : 0);
    return c;
}

template <typename S> size_t bytes(const Cut &c) {
    return (size_t)c.slots * S::RT * (S::HD * sizeof(float) + sizeof(float2));
}

template <typename S> hipError_t run(const AttendArgs &a, void *workspace, hipStream_t stream) {
    Work w;
    w.a = a;
    w.c = cut<S>(a.shared, a.N, a.B, a.H_q, a.H_kv);
    w.part = (float *)workspace;
    w.ml = (float2 *)(w.part + w.c.slots * S::RT * S::HD);
    const int64_t units = (int64_t)a.B * a.H_kv * w.c.units;
    hipLaunchKernelGGL((attend_kernel<S>), dim3((unsigned)(w.c.groups ? w.c.groups : units)), dim3(S::NT), 0, stream, w);
    if (w.c.groups)
        hipLaunchKernelGGL((join_kernel<S>), dim3((unsigned)(units * S::WR * S::DT)), dim3(256), 0, stream, w);
    return hipGetLastError();
}

// The kernel of a call: f(Shape) for its type, head and rows.  Few rows leave the keys to the waves; tiles of 64 KiB keep
// enough loads in flight where HBM bounds the call.
template <typename F> auto choose(int rows, int d, bool f32, F &&f) {
    if (f32) {
        if (d == 64) return rows <= 32 ? f(Shape<float, 64, 1, 4, 128>{}) : f(Shape<float, 64, 4, 1, 128>{});
        if (d == 128) return rows <= 32 ? f(Shape<float, 128, 1, 2, 64>{}) : f(Shape<float, 128, 4, 1, 64>{});
        return rows <= 32 ? f(Shape<float, 256, 1, 1, 32>{}) : f(Shape<float, 256, 4, 1, 32>{});
    }
    if (d == 64) {
        if (rows <= 32) return f(Shape<__bf16, 64, 1, 4, 128>{});
        return rows <= 64 ? f(Shape<__bf16, 64, 2, 2, 128>{}) : f(Shape<__bf16, 64, 4, 1, 128>{});
    }
    if (d == 128) {
        if (rows <= 32) return f(Shape<__bf16, 128, 1, 4, 128>{});
        return rows <= 64 ? f(Shape<__bf16, 128, 2, 2, 128>{}) : f(Shape<__bf16, 128, 4, 1, 64>{});
    }
    if (rows <= 32) return f(Shape<__bf16, 256, 1, 2, 64>{});
    return rows <= 64 ? f(Shape<__bf16, 256, 2, 2, 64>{}) : f(Shape<__bf16, 256, 4, 1, 64>{});
}

// Shared keys are read once for all where few rows of each sequence would read them: past that they are not what bounds.
int shared_used(int shared, int N, int B, int H_q, int H_kv) { return B > 1 && N * (H_q / H_kv) <= 64 && N <= 16 ? shared : 0; }

int rows_of(int shared, int N, int B, int H_q, int H_kv) { return N * (H_q / H_kv) * (shared > 0 ? B : 1); }

}  // namespace

size_t tree_attention_workspace(int shared, int N, int B, int H_q, int H_kv, int d, bool f32) {
    shared = shared_used(shared, N, B, H_q, H_kv);
    return choose(rows_of(shared, N, B, H_q, H_kv), d, f32, [&](auto s) {
        using S = decltype(s);
        return bytes<S>(cut<S>(shared, N, B, H_q, H_kv));
    });
}

hipError_t launch_tree_attention(AttendArgs a, int d, bool f32, void *workspace, hipStream_t stream) {
    a.shared = shared_used(a.shared, a.N, a.B, a.H_q, a.H_kv);
    return choose(rows_of(a.shared, a.N, a.B, a.H_q, a.H_kv), d, f32, [&](auto s) { return run<decltype(s)>(a, workspace, stream); });
}

}  // namespace treewy
