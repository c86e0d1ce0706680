// pp_scan_forward, pp_scan_backward, pp_scan_step: the gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) v_t, a = sigmoid(gate).
//
// One pass over the tokens: a workgroup's eight waves hold 16 tokens each, one behind the other, of 64 lanes' channels (two 16-bit ones to a
// lane).  A wave makes of its tokens what they do to any state, (A, H); the workgroup joins and publishes that, looks at what the tiles
// before it have published, and then every wave goes over its tokens again, from registers, with the state that they find.  Every
// byte is read and written once, but for the states before every 16th token that the backward pass begins from (1/16 of one float matrix, an eighth
// of a 16-bit one, written by the forward pass and read by the backward pass), 8 bytes a channel and tile between the tiles, and in 16 bits what
// the backward pass puts away: it has 128 registers and wants 6 more in bf16, 10 in fp16 (34 MB written beside 537, 65536 x 2048).
//
// What bounds it (a copy reaches 5.1 to 5.2 TB/s): 65536 x 1024 float32 forward 160 us, backward 253 (155 and 258 by bytes).  65536 x 2048 bf16 forward 206
// to 211, backward 302 to 311 (the same bytes): twice the exponentials and reciprocals to a byte, and the 16-bit values take twice their room as floats,
// so that two workgroups fit on a unit where three do in float32 (gates made again instead: three, and 224 for 206); with all tiles beside each other
// (2048 x 65536) 185 to 189 and 292.  Vector instructions take 68 and 73 % of the units' time.
// Of a tile's 13 us there 6 are tickets, loads and its stretch, 5 the wait for the state, 2 the rest.  Few channels wait for the chain of
// tiles: 65536 x 256 48 and 63 us, 1.5 us for 16 tiles; 2^30 x 1 395 and 376 ms, of 2^23 tiles.  5003 x 1000 fp16 in 23 sequences 20 and 30,
// less than two tiles one behind the other.
// Before the waits were shortened, sizes of 12 tokens to a wave took 272 us forward (for 237), four waves 255, 32 tokens to a wave 260 and 434 for 285 and 372.
#include "pp_rows.h"

#define SC_CHUNK 16               // tokens that a wave holds, and between kept states
#define SC_WAVES 8                // of a workgroup, one behind the other in time
#define SC_TILE (SC_CHUNK * SC_WAVES)
#define SC_GROUP 16               // tiles between states that are passed on whole
#define SC_EMPTIES 256            // most sequences that the only tile looks after itself
#define SC_MAX_TILES (1 << 24)    // of a call
#define SC_MAX_GRID ((1ll << 32) / (SC_WAVES * 64) - 1)  // workgroups of a launch, which has fewer than 2^32 threads
#define SC_MAX_SEQS (1 << 30)

// A stretch of tokens as what it makes of the state before it, h -> A h + H.  x says A: 1 - A where that is below 1/2 (so that a
// state which is kept loses nothing), -A otherwise, and SC_CUT where a sequence starts in the stretch: then nothing of h is left.
// H and 1 - A come from the same recurrence, so for one value throughout H = (1 - A) v, however long.
#define SC_CUT 2.0f
#define SC_EMPTY (~0ull)  // no stretch yet

__device__ __forceinline__ float sc_after(float x, float H, float h) {
    const float r = __builtin_fmaf(-x, h, H);
    const float near = h + (__builtin_isinf(h) ? H : r);  // (an infinite state stays one)
    return x == SC_CUT ? H : pp_bits(x) >> 31 ? r : near;
}
__device__ __forceinline__ float sc_share(float A, float D) { return D < 0.5f ? D : A != A ? pp_bits(0x7fc00000u) : -A; }
// (x, H) and behind it (x2, H2)
__device__ __forceinline__ void sc_join(float &x, float &H, float x2, float H2) {
    const bool n1 = pp_bits(x) >> 31, n2 = pp_bits(x2) >> 31;
    const float A = n1 ? -x : 1.0f - x, D = n1 ? 1.0f + x : x, A2 = n2 ? -x2 : 1.0f - x2, D2 = n2 ? 1.0f + x2 : x2;
    H = sc_after(x2, H2, H);
    x = x == SC_CUT || x2 == SC_CUT ? SC_CUT : sc_share(A * A2, __builtin_fmaf(A, D2, D));
}
__device__ __forceinline__ unsigned long long sc_word(float x, float H) { return (unsigned long long)pp_bits(H) << 32 | pp_bits(x); }

struct sc_args {
    long long rows, cols, seqs;
    const int *starts;
    int tiles, lanes_tiles;         // in time, and over the channels
    bool empties;                   // the tiles look after sequences without tokens too
    unsigned *ticket;
    unsigned long long *stretch;    // [tiles][width] what a tile makes of the state before it
    unsigned long long *whole;      // [tiles / SC_GROUP][width] the state before a group of tiles
    long long width;
};

__device__ __forceinline__ long long sc_start(const int *starts, long long rows, long long n) {
    const long long t = starts[n];
    return t < 0 ? 0 : t > rows ? rows : t;
}
__device__ __forceinline__ unsigned sc_from(long long t) { return t <= 0 ? ~0u : t >= 32 ? 0u : ~0u << t; }  // bits t and above

// What a wave's tokens t0 .. t0 + SC_CHUNK - 1 have to do with sequences, a bit each: whether a sequence has them, starts with them,
// ends with them.  The lanes look at 64 starts at a time.
struct sc_marks {
    unsigned in, first, last;
    int base, next;  // sequences that start before the tokens; of 64 behind those, the lane's start from t0 on
    bool more;       // there are yet others among the tokens
    // the sequence of token t0 + i
    __device__ __forceinline__ int of(const int *starts, long long rows, int seqs, long long t0, int i) const {
        int n = base + __popcll(__ballot(next <= i));
        for (int some = more ? PP_WAVE : 0; some == PP_WAVE; n += some) {
            const int at = n + (int)(threadIdx.x & (PP_WAVE - 1));
            some = __popcll(__ballot(at < seqs && sc_start(starts, rows, at < seqs ? at : seqs) <= t0 + i));
        }
        return n > 0 ? n - 1 : 0;
    }
};

// Few sequences' starts, one to a lane, and the end: asked for before all else, so that they do not wait behind a tile's values.
__device__ __forceinline__ int sc_mine(const int *__restrict__ starts, long long rows, int seqs) {
    const int lane = threadIdx.x & (PP_WAVE - 1);
    return starts && seqs < PP_WAVE ? (int)sc_start(starts, rows, lane < seqs ? lane : seqs) : 0;
}

__device__ __forceinline__ sc_marks sc_mark(const int *__restrict__ starts, long long rows, int seqs, int mine, long long t0) {
    const int lane = threadIdx.x & (PP_WAVE - 1), far = 0x7fffffff;
    long long begin = 0, end = rows;
    sc_marks m;
    m.base = 0;
    m.more = false;
    m.next = lane || t0 ? far : 0;
    if (!starts) m.base = t0 > 0;
    else if (seqs < PP_WAVE) {
        begin = __builtin_amdgcn_readlane(mine, 0);
        end = __builtin_amdgcn_readlane(mine, seqs);
        m.base = __popcll(__ballot(lane < seqs && mine < t0));
        m.next = lane >= m.base && lane < seqs ? (int)(mine - t0) : far;
    } else {
        begin = sc_start(starts, rows, 0);
        end = sc_start(starts, rows, seqs);
        int lo = 0, hi = seqs;  // the first n with starts[n] >= t0 is not before lo, and not behind hi
        while (lo < hi) {
            const int step = (hi - lo + PP_WAVE - 1) / PP_WAVE, at = lo + lane * step;
            const int below = __popcll(__ballot(lane <= (hi - 1 - lo) / step && sc_start(starts, rows, at < hi ? at : hi - 1) < t0));
            hi = below * (long long)step < hi - lo ? lo + below * step : hi;
            lo = below ? lo + (below - 1) * step + 1 : lo;
        }
        m.base = lo;
        m.next = lo + lane < seqs ? (int)(sc_start(starts, rows, lo + lane) - t0) : far;
        m.more = __builtin_amdgcn_readlane(m.next, PP_WAVE - 1) <= SC_CHUNK;
    }
    m.in = sc_from(begin - t0) & ~sc_from(end - t0) & ~sc_from(SC_CHUNK);
    unsigned bits = m.next >= 0 && m.next <= SC_CHUNK ? 1u << m.next : 0u;  // (bit SC_CHUNK: the next wave's first token)
    if (m.more)
        for (long long n = (long long)m.base + PP_WAVE + lane; n < seqs; n += PP_WAVE) {
            const long long t = sc_start(starts, rows, n) - t0;
            if (t < 0 || t > SC_CHUNK) break;
            bits |= 1u << t;
        }
    bits |= pp_moved<0xB1>(bits);
    bits |= pp_moved<0x4E>(bits);
    bits |= pp_moved<0x141>(bits);
    bits |= pp_moved<0x140>(bits);
    bits = __builtin_amdgcn_readlane(bits, 0) | __builtin_amdgcn_readlane(bits, 16) | __builtin_amdgcn_readlane(bits, 32) | __builtin_amdgcn_readlane(bits, 48);
    m.first = bits & m.in;
    m.last = ((end - t0 > 0 && end - t0 <= SC_CHUNK ? 1u << (end - t0 - 1) : 0u) | bits >> 1) & m.in;
    return m;
}

// W channels of a token to a lane: two 16-bit values of a word, or one value.  A row's address is the same for all lanes, a lane's
// offset 32 bits.
template <class Y, int W> struct sc_lane {
    typedef typename Y::T T;
    unsigned c;    // first channel
    int n;         // channels that there are
    unsigned at;   // byte from which on a whole word is read
    unsigned shift;
    bool full;     // all lanes have W
    __device__ __forceinline__ sc_lane(unsigned tile, unsigned cols) {
        c = (tile * PP_WAVE + (threadIdx.x & (PP_WAVE - 1))) * W;
        n = c + W <= cols ? W : cols > c ? (int)(cols - c) : 0;
        at = (c + W <= cols ? c : cols - W) * (unsigned)sizeof(T);
        shift = n == 1 && W == 2 ? 16 : 0;
        full = (tile + 1) * PP_WAVE * W <= cols;
    }
    __device__ __forceinline__ unsigned load(const T *row) const {
        const char *p = (const char *)row + at;
        if constexpr (sizeof(T) * W == 4) {
            unsigned u;
            __builtin_memcpy(&u, p, 4);
            return u;
        } else return *(const unsigned short *)p;
    }
    // the tokens t0 .. t0 + SC_CHUNK - 1; the last row in the place of those behind it
    __device__ __forceinline__ void load_all(unsigned (&raw)[SC_CHUNK], const T *m, long long ld, long long t0, long long rows) const {
        const T *row = m + (t0 < rows ? t0 : rows - 1) * ld;
        if (rows - t0 >= SC_CHUNK) {
#pragma unroll
            for (int i = 0; i < SC_CHUNK; ++i) raw[i] = load(row + i * ld);
        } else {
            const int more = rows > t0 ? (int)(rows - 1 - t0) : 0;
#pragma unroll
            for (int i = 0; i < SC_CHUNK; ++i) raw[i] = load(row + (i < more ? i : more) * ld);
        }
        if (!full)
#pragma unroll
            for (int i = 0; i < SC_CHUNK; ++i) raw[i] >>= shift;
    }
    __device__ __forceinline__ static float get(unsigned raw, int w) {
        if constexpr (sizeof(T) == 4) return pp_bits(raw);
        else return Y::get(__builtin_bit_cast(T, (unsigned short)(raw >> (16 * w))));
    }
    __device__ __forceinline__ void store(T *row, const float *v) const {
        T t[W];
#pragma unroll
        for (int w = 0; w < W; ++w) t[w] = Y::put(v[w]);
        if (full) __builtin_memcpy((char *)row + at, t, sizeof(t));
        else
#pragma unroll
            for (int w = 0; w < W; ++w)
                if (w < n) row[c + w] = t[w];
    }
    __device__ __forceinline__ void get_floats(const float *row, float *v) const {  // zeros where row is NULL
#pragma unroll
        for (int w = 0; w < W; ++w) v[w] = row && w < n ? row[c + w] : 0.0f;
    }
    __device__ __forceinline__ void put_floats(float *row, const float *v) const {
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (w < n) row[c + w] = v[w];
    }
};

template <int W> struct sc_room {
    float x[SC_WAVES][W * PP_WAVE], H[SC_WAVES][W * PP_WAVE];
    float before[W * PP_WAVE];
    unsigned ticket;
};

__device__ __forceinline__ unsigned long long sc_peek(const unsigned long long *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void sc_tell(unsigned long long *p, unsigned long long v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// The four lanes of a quad joined in their order: in its first lane
__device__ __forceinline__ void sc_join_quad(float &x, float &H) {
    const float x1 = pp_moved<0xF5>(x), H1 = pp_moved<0xF5>(H);  // lanes 1 1 3 3
    sc_join(x, H, x1, H1);
    const float x2 = pp_moved<0xAA>(x), H2 = pp_moved<0xAA>(H);  // lane 2
    sc_join(x, H, x2, H2);
}

// The state (of W channels a lane) before wave `wave` of tile number `order` of its channels, in the order of the recurrence, from the waves' own
// stretches in room.x, room.H; and what the tile's successors need.  Every wave takes part: what others wait for is a quad's work for
// a channel (by one wave for all channels, in LDS between, it took 237 us for 210, 65536 x 2048 bf16 forward, and 22.9 for 20.8, 5003 x 1000).
//
// A tile waits for tiles of its channels that took a lower ticket only.  These run already and wait for lower ones in turn, so every wait
// ends.  A word says by itself whether it is there (SC_EMPTY: not yet), so no other memory has to be ordered with it, and
// what is added up in which order depends on the tile's number alone.
template <int W>
__device__ __forceinline__ void sc_carry(const sc_args &a, sc_room<W> &room, int order, long long lanes_tile, int wave, float *h) {
    static_assert(SC_WAVES == 8 && SC_GROUP == 16, "two waves, four tiles to a lane");
    const int lane = threadIdx.x & (PP_WAVE - 1), group = order / SC_GROUP, place = order % SC_GROUP;
#pragma unroll
    for (int w = 0; w < W; ++w) h[w] = 0.0f;
    if (a.tiles > 1) {
        if (wave < 4 * W) {
            const int l = threadIdx.x >> 2, part = threadIdx.x & 3;
            const long long col = lanes_tile * (W * PP_WAVE) + l;
            const float x0 = room.x[2 * part][l], H0 = room.H[2 * part][l];
            float x = x0, H = H0;
            sc_join(x, H, room.x[2 * part + 1][l], room.H[2 * part + 1][l]);
            const float left_x = pp_moved<0xA0>(x), left_H = pp_moved<0xA0>(H);  // lanes 0 0 2 2
            const float x1 = pp_moved<0xF5>(x), H1 = pp_moved<0xF5>(H);          // lanes 1 1 3 3
            sc_join(x, H, x1, H1);
            const float half_x = pp_moved<0x00>(x), half_H = pp_moved<0x00>(H), x2 = pp_moved<0xAA>(x), H2 = pp_moved<0xAA>(H);
            sc_join(x, H, x2, H2);
            if (!part) sc_tell(a.stretch + order * a.width + col, sc_word(x, H));
            // in the stretches' places: what the waves before each of them make of a state (zeros leave it as it is)
            float ex = part > 1 ? half_x : 0.0f, eH = part > 1 ? half_H : 0.0f;
            sc_join(ex, eH, part & 1 ? left_x : 0.0f, part & 1 ? left_H : 0.0f);
            room.x[2 * part][l] = ex;
            room.H[2 * part][l] = eH;
            sc_join(ex, eH, x0, H0);
            room.x[2 * part + 1][l] = ex;
            room.H[2 * part + 1][l] = eH;
            // the tiles before it in its group
            unsigned long long word[4];
            bool wait = true;
            while (wait) {
                wait = false;
#pragma unroll
                for (int k = 0; k < 4; ++k) word[k] = 4 * part + k < place ? sc_peek(a.stretch + (order - place + 4 * part + k) * a.width + col) : 0;
#pragma unroll
                for (int k = 0; k < 4; ++k) wait = wait || (unsigned)word[k] == (unsigned)SC_EMPTY;
                wait = __any(wait);
                if (wait) __builtin_amdgcn_s_sleep(4);
            }
            float bx = pp_bits((unsigned)word[0]), bH = pp_bits((unsigned)(word[0] >> 32));
#pragma unroll
            for (int k = 1; k < 4; ++k) sc_join(bx, bH, pp_bits((unsigned)word[k]), pp_bits((unsigned)(word[k] >> 32)));
            sc_join_quad(bx, bH);
            // the last tile of a group knows what the group makes of a state before it knows the state
            const bool last = place == SC_GROUP - 1 && order + 1 < a.tiles;
            const float own_x = x, own_H = H;
            x = bx;
            H = bH;
            sc_join(x, H, own_x, own_H);
            word[0] = 0;
            wait = group > 0;
            while (wait) {
                word[0] = part ? 0 : sc_peek(a.whole + group * a.width + col);
                wait = __any((unsigned)word[0] == (unsigned)SC_EMPTY);
                if (wait) __builtin_amdgcn_s_sleep(4);
            }
            const float whole = pp_bits((unsigned)(word[0] >> 32));
            if (!part) {
                if (last) sc_tell(a.whole + (group + 1) * a.width + col, sc_word(0.0f, sc_after(x, H, whole)));
                room.before[l] = sc_after(bx, bH, whole);
            }
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; ++w) h[w] = sc_after(room.x[wave][lane * W + w], room.H[wave][lane * W + w], room.before[lane * W + w]);
        return;
    }
#pragma unroll
    for (int k = 0; k < SC_WAVES; ++k) {
        if (k == wave) break;
#pragma unroll
        for (int w = 0; w < W; ++w) h[w] = sc_after(room.x[k][lane * W + w], room.H[k][lane * W + w], h[w]);
    }
}

// The workgroup's tile, by a ticket: a tile's predecessors are under way before it.  (Taking the next ticket while a tile is worked on
// saves its way to memory, and makes the tiles that wait for the one behind it wait for both: 298 us for 242, 65536 x 2048 forward.)
template <int W> __device__ __forceinline__ unsigned sc_ticket(const sc_args &a, sc_room<W> &room) {
    if (a.tiles == 1) return blockIdx.x;
    if (!threadIdx.x) room.ticket = atomicAdd(a.ticket, 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(room.ticket);
}

// Sequences without tokens end with what they begin with: by the waves of the only tile in time, where sequences are few.
template <class L> __device__ __forceinline__ void sc_empties(const sc_args &a, const L &lanes, int wave, const float *from, float *to) {
    if (!a.empties || !to) return;
    for (long long n = wave; n < a.seqs; n += SC_WAVES) {
        if (sc_start(a.starts, a.rows, n) < sc_start(a.starts, a.rows, n + 1)) continue;
        float h[2];
        lanes.get_floats(from ? from + n * a.cols : NULL, h);
        lanes.put_floats(to + n * a.cols, h);
    }
}

// a = 1 / (1 + e) and 1 - a = e / (1 + e) of a gate, e = exp(-gate).  The exponent is a product that was rounded, so the smaller of the two is right to
// (8 + 2 |gate|) 2^-24 of itself, and exp2 and the reciprocal give 0 for what is no normal number: a is 0 from a gate of -87.34 on, where e times it is
// nothing, and 1 - a is 1 from far before.  A gate that is none leaves both none.
__device__ __forceinline__ void sc_open(float gate, float &a, float &u) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504f * gate);
    a = __builtin_amdgcn_rcpf(1.0f + e);
    u = e > 0x1p125f ? 1.0f : e * a;
}
// the same from s, the smaller one, negative where that is a
__device__ __forceinline__ void sc_sides(float s, float &a, float &u) {
    const float m = __builtin_fabsf(s), r = 1.0f - m;
    const bool keeps = !(pp_bits(s) >> 31);
    a = keeps ? r : m;
    u = keeps ? m : r;
}

// Tokens in the midst of a sequence take the short way: PLAIN says that no sequence begins or ends among a wave's tokens.
template <class Y, int W>
__global__ __launch_bounds__(SC_WAVES *PP_WAVE, 4) void k_scan_forward(sc_args a, const typename Y::T *__restrict__ gate, long long ld_gate,
                                                                       const typename Y::T *__restrict__ v, long long ld_v, const float *__restrict__ h0,
                                                                       typename Y::T *__restrict__ h, long long ld_h, float *__restrict__ h_last,
                                                                       float *__restrict__ kept) {
    __shared__ sc_room<W> room;
    const int mine = sc_mine(a.starts, a.rows, (int)a.seqs);
    const unsigned ticket = sc_ticket(a, room);
    const int order = ticket / (unsigned)a.lanes_tiles, lanes_tile = ticket % (unsigned)a.lanes_tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PP_WAVE), lane = threadIdx.x & (PP_WAVE - 1);
    const long long t0 = (long long)order * SC_TILE + wave * SC_CHUNK;
    const sc_lane<Y, W> lanes(lanes_tile, (unsigned)a.cols);
    unsigned f[SC_CHUNK], x[SC_CHUNK];
    lanes.load_all(f, gate, ld_gate, t0, a.rows);
    lanes.load_all(x, v, ld_v, t0, a.rows);
    const sc_marks m = sc_mark(a.starts, a.rows, (int)a.seqs, mine, t0);
    const bool plain = m.in == ~sc_from(SC_CHUNK) && !m.first && !m.last;
    // a and (1 - a) v of the wave's tokens, and its own stretch; of the sequences that start in it the last one counts
    float keep[SC_CHUNK][W], bring[SC_CHUNK][W], H[W], A[W], D[W], from[W];
    const int cut = m.first ? 31 - __builtin_clz(m.first) : -1;
    auto sequence = [&](int i) { return (long long)m.of(a.starts, a.rows, (int)a.seqs, t0, i); };
    if (cut >= 0) lanes.get_floats(h0 ? h0 + sequence(cut) * a.cols : NULL, from);
#pragma unroll
    for (int w = 0; w < W; ++w) H[w] = 0.0f, A[w] = 1.0f, D[w] = 0.0f;
    auto stretch = [&](auto is_plain) {
#pragma unroll
        for (int i = 0; i < SC_CHUNK; ++i) {
            if constexpr (!decltype(is_plain)::value) {
                if (!(m.in >> i & 1)) continue;
                if (i == cut)
#pragma unroll
                    for (int w = 0; w < W; ++w) H[w] = from[w];
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float u;
                sc_open(lanes.get(f[i], w), keep[i][w], u);
                bring[i][w] = u * lanes.get(x[i], w);
                H[w] = __builtin_fmaf(keep[i][w], H[w], bring[i][w]);
                D[w] = __builtin_fmaf(keep[i][w], D[w], u);
                A[w] *= keep[i][w];
            }
        }
    };
    if (plain) stretch(std::true_type());
    else stretch(std::false_type());
#pragma unroll
    for (int w = 0; w < W; ++w) {
        room.x[wave][lane * W + w] = cut >= 0 ? SC_CUT : sc_share(A[w], D[w]);
        room.H[wave][lane * W + w] = H[w];
    }
    __syncthreads();
    sc_carry<W>(a, room, order, lanes_tile, wave, H);
    if (kept && t0 < a.rows) lanes.put_floats(kept + t0 / SC_CHUNK * a.cols, H);
    sc_empties(a, lanes, wave, h0, h_last);
    typename Y::T *row = h + t0 * ld_h;
    if (plain) {
#pragma unroll
        for (int i = 0; i < SC_CHUNK; ++i) {
#pragma unroll
            for (int w = 0; w < W; ++w) H[w] = __builtin_fmaf(keep[i][w], H[w], bring[i][w]);
            lanes.store(row, H);
            row += ld_h;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < SC_CHUNK; ++i) {
        if (!(m.in >> i & 1)) continue;
        if (m.first >> i & 1) lanes.get_floats(h0 ? h0 + sequence(i) * a.cols : NULL, H);
#pragma unroll
        for (int w = 0; w < W; ++w) H[w] = __builtin_fmaf(keep[i][w], H[w], bring[i][w]);
        lanes.store(row + i * ld_h, H);
        if (h_last && (m.last >> i & 1)) lanes.put_floats(h_last + sequence(i) * a.cols, H);
    }
}

// The same from the last tile to the first, for c = a_t g_t; the state before every SC_CHUNK tokens was kept.
template <class Y, int W>
__global__ __launch_bounds__(SC_WAVES *PP_WAVE, 4) void k_scan_backward(sc_args a, const typename Y::T *__restrict__ dh, long long ld_dh,
                                                                        const typename Y::T *__restrict__ gate, long long ld_gate,
                                                                        const typename Y::T *__restrict__ v, long long ld_v, const float *__restrict__ h0,
                                                                        const float *__restrict__ kept, const float *__restrict__ dh_last,
                                                                        typename Y::T *__restrict__ dgate, long long ld_dgate, typename Y::T *__restrict__ dv,
                                                                        long long ld_dv, float *__restrict__ dh0) {
    __shared__ sc_room<W> room;
    const int mine = sc_mine(a.starts, a.rows, (int)a.seqs);
    const unsigned ticket = sc_ticket(a, room);
    const int order = ticket / (unsigned)a.lanes_tiles, lanes_tile = ticket % (unsigned)a.lanes_tiles;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / PP_WAVE), lane = threadIdx.x & (PP_WAVE - 1);
    const long long t0 = (long long)(a.tiles - 1 - order) * SC_TILE + (SC_WAVES - 1 - wave) * SC_CHUNK;
    const sc_lane<Y, W> lanes(lanes_tile, (unsigned)a.cols);
    unsigned f[SC_CHUNK], x[SC_CHUNK], d[SC_CHUNK];
    float state[W];
    lanes.get_floats(t0 < a.rows ? kept + t0 / SC_CHUNK * a.cols : NULL, state);
    lanes.load_all(f, gate, ld_gate, t0, a.rows);
    lanes.load_all(x, v, ld_v, t0, a.rows);
    lanes.load_all(d, dh, ld_dh, t0, a.rows);
    const sc_marks m = sc_mark(a.starts, a.rows, (int)a.seqs, mine, t0);
    const bool plain = m.in == ~sc_from(SC_CHUNK) && !m.first && !m.last;
    // of the sequences that end in the stretch the first one counts, which may have begun before
    const int cut = m.last ? __builtin_ctz(m.last) : -1;
    auto sequence = [&](int i) { return (long long)m.of(a.starts, a.rows, (int)a.seqs, t0, i); };
    float s[SC_CHUNK][W], p[SC_CHUNK][W], C[W], A[W], D[W], from[W];
    if (cut >= 0) lanes.get_floats(dh_last ? dh_last + sequence(cut) * a.cols : NULL, from);
    // gates, and the states that the tokens find less their values
    auto states = [&](auto is_plain) {
#pragma unroll
        for (int i = 0; i < SC_CHUNK; ++i) {
            if constexpr (!decltype(is_plain)::value) {
                if (!(m.in >> i & 1)) continue;
                if (m.first >> i & 1) lanes.get_floats(h0 ? h0 + sequence(i) * a.cols : NULL, state);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                const float value = lanes.get(x[i], w);
                const float g = lanes.get(f[i], w), e = __builtin_amdgcn_exp2f(-1.44269504f * __builtin_fabsf(g)), large = __builtin_amdgcn_rcpf(1.0f + e);
                const float small = e * large;
                const bool keeps = g >= 0.0f;
                s[i][w] = keeps ? small : -small;
                const float ka = keeps ? large : small, ku = keeps ? small : large;
                p[i][w] = state[w] - value;
                state[w] = __builtin_fmaf(ka, state[w], ku * value);
            }
        }
    };
    // its own stretch, from the last token to the first
#pragma unroll
    for (int w = 0; w < W; ++w) C[w] = 0.0f, A[w] = 1.0f, D[w] = 0.0f;
    auto stretch = [&](auto is_plain) {
#pragma unroll
        for (int i = SC_CHUNK - 1; i >= 0; --i) {
            if constexpr (!decltype(is_plain)::value) {
                if (!(m.in >> i & 1)) continue;
                if (i == cut)
#pragma unroll
                    for (int w = 0; w < W; ++w) C[w] = from[w];
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float ka, ku;
                sc_sides(s[i][w], ka, ku);
                C[w] = ka * (lanes.get(d[i], w) + C[w]);
                D[w] = __builtin_fmaf(ka, D[w], ku);
                A[w] *= ka;
            }
        }
    };
    if (plain) {
        states(std::true_type());
        stretch(std::true_type());
    } else {
        states(std::false_type());
        stretch(std::false_type());
    }
#pragma unroll
    for (int w = 0; w < W; ++w) {
        room.x[wave][lane * W + w] = cut >= 0 ? SC_CUT : sc_share(A[w], D[w]);
        room.H[wave][lane * W + w] = C[w];
    }
    __syncthreads();
    sc_carry<W>(a, room, order, lanes_tile, wave, C);
    sc_empties(a, lanes, wave, dh_last, dh0);
    auto gradients = [&](int i, typename Y::T *to_gate, typename Y::T *to_v) {
        float df[W], dx[W];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            float ka, ku;
            sc_sides(s[i][w], ka, ku);
            const float g = lanes.get(d[i], w) + C[w];
            dx[w] = ku * g;
            C[w] = ka * g;
            df[w] = p[i][w] * ku * C[w];
        }
        lanes.store(to_gate, df);
        lanes.store(to_v, dx);
    };
    typename Y::T *to_gate = dgate + (t0 + SC_CHUNK - 1) * ld_dgate, *to_v = dv + (t0 + SC_CHUNK - 1) * ld_dv;
    if (plain) {
#pragma unroll
        for (int i = SC_CHUNK - 1; i >= 0; --i) {
            gradients(i, to_gate, to_v);
            to_gate -= ld_dgate;
            to_v -= ld_dv;
        }
        return;
    }
#pragma unroll
    for (int i = SC_CHUNK - 1; i >= 0; --i) {
        if (m.in >> i & 1) {
            if (m.last >> i & 1) lanes.get_floats(dh_last ? dh_last + sequence(i) * a.cols : NULL, C);
            gradients(i, to_gate, to_v);
            if (dh0 && (m.first >> i & 1)) lanes.put_floats(dh0 + sequence(i) * a.cols, C);
        }
        to_gate -= ld_dgate;
        to_v -= ld_dv;
    }
}

// What tiles wait for is not there yet; and sequences without tokens end with what they begin with.
__global__ __launch_bounds__(256) void k_scan_begin(sc_args a, long long words, const float *__restrict__ from, float *__restrict__ to) {
    if (words && blockIdx.x == 0 && !threadIdx.x) *a.ticket = 0;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < words; i += gridDim.x * 256ll) a.stretch[i] = SC_EMPTY;
    if (!to) return;
    for (long long n = blockIdx.x; n < a.seqs; n += gridDim.x) {
        if (a.starts ? sc_start(a.starts, a.rows, n) < sc_start(a.starts, a.rows, n + 1) : a.rows > 0) continue;
        for (long long c = threadIdx.x; c < a.cols; c += 256) to[n * a.cols + c] = from ? from[n * a.cols + c] : 0.0f;
    }
}

// A thread to eight channels of a row.  64 x 4096 bf16 3.6 us, of which a launch is half.
template <class Y>
__global__ __launch_bounds__(256) void k_scan_step(long long rows, long long cols, long long chunks, long long n_slots, const int *__restrict__ slots,
                                                   const typename Y::T *__restrict__ gate, long long ld_gate, const typename Y::T *__restrict__ v,
                                                   long long ld_v, float *__restrict__ state, typename Y::T *__restrict__ h, long long ld_h) {
    for (long long at = blockIdx.x * 256ll + threadIdx.x; at < rows * chunks; at += gridDim.x * 256ll) {
        const long long row = at / chunks, c = 8 * (at - row * chunks), left = cols - c, slot = slots ? slots[row] : row;
        if (slot < 0 || slot >= n_slots) continue;
        float f[8], x[8], s[8];
        const PpRaw<Y> rf = pp_load8<Y>(gate + row * ld_gate + c, left), rv = pp_load8<Y>(v + row * ld_v + c, left);
        const PpRaw<PpF32> rs = pp_load8<PpF32>(state + slot * cols + c, left);
        pp_values<Y>(rf, f);
        pp_values<Y>(rv, x);
        pp_values<PpF32>(rs, s);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            float a, u;
            sc_open(f[j], a, u);
            s[j] = __builtin_fmaf(a, s[j], u * x[j]);
        }
        pp_store8<PpF32>(state + slot * cols + c, left, s);
        pp_store8<Y>(h + row * ld_h + c, left, s);
    }
}

static int64_t sc_tiles(int64_t rows) { return (rows + SC_TILE - 1) / SC_TILE; }

static bool sc_bad(int type, int64_t rows, int64_t cols, int64_t seqs, const int32_t *starts, const float *h0, const float *kept, const float *x,
                   const float *y) {
    if (pp_bad_sizes(type, rows, cols) || seqs < 0 || seqs > SC_MAX_SEQS || (!starts && seqs != 1)) return true;
    for (const void *p : {(const void *)starts, (const void *)h0, (const void *)kept, (const void *)x, (const void *)y})
        if ((uintptr_t)p & 3) return true;
    return sc_tiles(rows) * ((cols + PP_WAVE - 1) / PP_WAVE) > SC_MAX_TILES;
}

static int64_t sc_width(int64_t cols) { return (cols + 2 * PP_WAVE - 1) / (2 * PP_WAVE) * (2 * PP_WAVE); }

extern "C" size_t pp_scan_workspace_bytes(int call, int type, int64_t rows, int64_t cols) {
    if (pp_bad_sizes(type, rows, cols) || (call != PP_SCAN_FORWARD && call != PP_SCAN_BACKWARD)) return 0;
    const int64_t tiles = sc_tiles(rows);
    return 256 + pp_align256((size_t)(tiles + tiles / SC_GROUP + 1) * sc_width(cols) * 8);
}

extern "C" int64_t pp_scan_kept_rows(int type, int64_t rows, int64_t cols) {
    return pp_bad_sizes(type, rows, cols) ? -1 : (rows + SC_CHUNK - 1) / SC_CHUNK;
}

// The tiles of a call, and its workspace made ready.  launch(args, grid, channels to a lane as a constant)
template <class Y, class F>
static int sc_run(int64_t rows, int64_t cols, int64_t seqs, const int32_t *starts, void *workspace, hipStream_t st, const float *from, float *to, F launch) {
    sc_args a = {rows, cols, seqs, starts};
    const bool pairs = sizeof(typename Y::T) == 2 && cols > 1;
    const int64_t per = pairs ? 2 * PP_WAVE : PP_WAVE, lanes = (cols + per - 1) / per, tiles = sc_tiles(rows);
    a.tiles = (int)tiles;
    a.lanes_tiles = (int)lanes;
    a.width = sc_width(cols);
    a.ticket = (unsigned *)workspace;
    a.stretch = (unsigned long long *)((char *)workspace + 256);
    a.whole = a.stretch + tiles * a.width;
    const int64_t words = tiles > 1 ? (tiles + tiles / SC_GROUP + 1) * a.width : 0;
    a.empties = tiles == 1 && starts && seqs <= SC_EMPTIES;
    if (words || (to && !a.empties && (starts || !rows))) {
        int64_t groups = (words + 1023) / 1024;
        if (to && groups < seqs) groups = seqs;
        k_scan_begin<<<(unsigned)(groups < 4096 ? groups : 4096), 256, 0, st>>>(a, words, from, to);
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
    }
    if (!rows) return PP_OK;
    // More tiles than a launch has workgroups take another launch, whose tickets go on where the first one's ended.  (Those are many tiles in
    // time, which go by tickets: one tile in time has 2^16 workgroups at most.)
    for (int64_t left = tiles * lanes; left > 0; left -= SC_MAX_GRID) {
        const unsigned grid = (unsigned)(left < SC_MAX_GRID ? left : SC_MAX_GRID);
        if (pairs) {
            if constexpr (sizeof(typename Y::T) == 2) launch(a, grid, std::integral_constant<int, 2>());
        } else launch(a, grid, std::integral_constant<int, 1>());
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
    }
    return PP_OK;
}

extern "C" int pp_scan_forward(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v, int64_t seqs,
                               const int32_t *starts, const float *h0, void *h, int64_t ld_h, float *h_last, float *kept, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (sc_bad(type, rows, cols, seqs, starts, h0, kept, h_last, NULL)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) || pp_bad_matrix(h, type, rows, cols, ld_h))
        return PP_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_scan_workspace_bytes(PP_SCAN_FORWARD, type, rows, cols)) return PP_ERR_WORKSPACE;
    if (!seqs) return PP_OK;
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        return sc_run<Y>(rows, cols, seqs, starts, workspace, st, h0, h_last, [&](const sc_args &a, unsigned grid, auto w) {
            k_scan_forward<Y, decltype(w)::value><<<grid, SC_WAVES * PP_WAVE, 0, st>>>(a, (const T *)gate, ld_gate, (const T *)v, ld_v, h0, (T *)h, ld_h, h_last, kept);
        });
    });
}

extern "C" int pp_scan_backward(int type, int64_t rows, int64_t cols, const void *dh, int64_t ld_dh, const void *gate, int64_t ld_gate, const void *v,
                                int64_t ld_v, int64_t seqs, const int32_t *starts, const float *h0, const float *kept, const float *dh_last, void *dgate,
                                int64_t ld_dgate, void *dv, int64_t ld_dv, float *dh0, void *workspace, size_t workspace_bytes, void *stream) {
    if (sc_bad(type, rows, cols, seqs, starts, h0, kept, dh_last, dh0) || (rows && !kept)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dh, type, rows, cols, ld_dh) || pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) ||
        pp_bad_matrix(dgate, type, rows, cols, ld_dgate) || pp_bad_matrix(dv, type, rows, cols, ld_dv))
        return PP_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_scan_workspace_bytes(PP_SCAN_BACKWARD, type, rows, cols)) return PP_ERR_WORKSPACE;
    if (!seqs) return PP_OK;
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        return sc_run<Y>(rows, cols, seqs, starts, workspace, st, dh_last, dh0, [&](const sc_args &a, unsigned grid, auto w) {
            k_scan_backward<Y, decltype(w)::value><<<grid, SC_WAVES * PP_WAVE, 0, st>>>(a, (const T *)dh, ld_dh, (const T *)gate, ld_gate, (const T *)v, ld_v, h0, kept,
                                                                                           dh_last, (T *)dgate, ld_dgate, (T *)dv, ld_dv, dh0);
        });
    });
}

extern "C" int pp_scan_step(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v, int64_t n_slots,
                            const int32_t *slots, float *state, void *h, int64_t ld_h, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || n_slots < 0 || n_slots > PP_LAYER_MAX_ROWS || ((uintptr_t)slots & 3) || ((uintptr_t)state & 3)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) || pp_bad_matrix(h, type, rows, cols, ld_h))
        return PP_ERR_INVALID_ARG;
    if (rows && (!state || (!slots && rows > n_slots))) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const int64_t chunks = (cols + 7) / 8, groups = (rows * chunks + 255) / 256;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        k_scan_step<Y><<<(unsigned)(groups < (1 << 20) ? groups : 1 << 20), 256, 0, (hipStream_t)stream>>>(rows, cols, chunks, n_slots, slots, (const T *)gate, ld_gate,
                                                                                                         (const T *)v, ld_v, state, (T *)h, ld_h);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}
