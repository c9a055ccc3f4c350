// Rows of a table by token, and the table's gradient.
//
//   out_t = s W[id_t],   dW_v = s (sum over the tokens t of word v of dout_t)
//
// Both are HBM-bound: the rows that tokens name are read and written once; the
// gradient reads every token's row and writes the whole table.  The gradient
// needs the tokens by word, in their order, without the host: each block of
// embed_order_kernel takes up to 256 words, looks through all ids, counts those before
// its words (the place of its tokens in the order) and those of each word, and
// puts its tokens there.  One launch instead of a radix sort's six; the ids come
// from L2 but for the first block.  Where words times tokens are too many for
// that the radix sort is taken.
//
// The sums: a wave takes a word and one or two tiles of columns and adds up its tokens'
// rows, in one order.  A word of more than kLong tokens (a few words are a tenth of a
// text) is left to waves that take kLong places of the order each, whatever the
// words there; their sums of long words are joined in order by a second launch.
//
// 32,768 tokens of 50,000 words of 1,024 columns in bf16, words as frequent as in text: rows
// 28 us (4.8 TB/s), the order 15, sums 60 (2.8 TB/s of tokens' rows and table), joins 4.9 (on
// inputs of their own for each call; on the same ones, from the caches, rows 23.5 and sums 49).
// 16 tokens: 2.9 us, a launch.  10,007 tokens of 5,003 words of 333 columns in fp32: 8.1, 7.6,
// 17 and 4.1 us.
#include <algorithm>

#include "values.hpp"

namespace nsd {

namespace {

constexpr int kEmbedThreads = 256;
constexpr int kEmbedWaves = kEmbedThreads / kWave;
constexpr int64_t kMaxEmbedBlocks = UINT32_MAX / kEmbedThreads;
constexpr int kLong = kWave;  // tokens that one wave adds up; places of a chunk

constexpr int kOrderThreads = 1024;
constexpr int kOrderWaves = kOrderThreads / kWave;
constexpr int kOrderWords = 256;
// Ids looked at by all blocks of embed_order_kernel up to which it is taken.  (The gradient of
// 131,072 tokens of 65,536 words of 16 columns, 2^25 looks: 100 us, 133 sorted.  2^26: 131,072
// of 131,072 words 130 and 145, 16,384 of a million 100 and 77.  Beyond 2^17 tokens both are
// near: 262,144 of 32,768 words 144 and 153.)
constexpr int64_t kMaxLooks = int64_t(1) << 25;

// Words of a block: few where there are few of them, so that all CUs take part in what is then
// many tokens a word (61,840 tokens of 117 words 39 us, with 256 words a block 98; 32,768 of
// 1,000 words of 2,048 columns 52 and 62).
int words_of_block(int64_t vocab) {
    int n = 1;
    while (n < kOrderWords && ceil_div(vocab, n) > 256) n *= 2;
    return n;
}

bool by_looking(int64_t ntok, int64_t vocab) {
    const int64_t blocks = ceil_div(vocab, words_of_block(vocab));
    return blocks * ntok <= kMaxLooks && ntok <= (1 << 17) && blocks <= UINT32_MAX / kOrderThreads;
}

// ------------------------------------------------------------------- rows

// Lanes that a row's columns take, a power of two up to 64: a wave takes 64 / lanes rows.
int row_lanes(int32_t width, int values) {
    int g = 1;
    while (g < kWave && (int64_t)g * values < width) g <<= 1;
    return g;
}

// A wave takes a token and a tile of columns, or 64 / lanes tokens of narrow rows.
template <class TW, class TO, int N>
__global__ __launch_bounds__(kEmbedThreads) void embed_kernel(
    int32_t ntok, int64_t units, int32_t tiles, int32_t lanes, int32_t vocab, int32_t width,
    float scale, const int32_t *__restrict__ ids, const TW *__restrict__ W, int64_t ldw,
    TO *__restrict__ out, int64_t ldo) {
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    for (int64_t u = (int64_t)blockIdx.x * kEmbedWaves + wave; u < units;
         u += (int64_t)gridDim.x * kEmbedWaves) {
        int64_t t = u;
        int tile = 0;
        if (tiles > 1) {
            t = u / tiles;
            tile = (int)(u % tiles);
        }
        t = t * (kWave / lanes) + lane / lanes;
        const int col = (tile * kWave + lane % lanes) * N;
        if (t >= ntok || col >= width) continue;
        const int id = ids[t];
        const bool word = id >= 0 && id < vocab;
        float x[N] = {};
        if (word) load_cols<N, TW>(W + id * ldw, col, width, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = word ? x[e] * scale : 0.f;  // whatever the scale is
        store_cols<N, TO>(out + t * ldo, col, width, x);
    }
}

// ------------------------------------------------------------ tokens by word

// Places of the tokens of block b's words (up to 256) in the order by word: `perm` the
// token, `word` its word, of every place; segptr the first place of every word.
//
// A wave looks through consecutive tokens, four a lane, and keeps those of the block's words
// in a list in LDS, in their order; what does not fit (a word that takes most of the batch)
// it looks up again.
constexpr int kOrderList = 2048;  // of a wave
constexpr int kOrderStep = 4 * kWave;

__global__ __launch_bounds__(kOrderThreads) void embed_order_kernel(
    int32_t ntok, int32_t vocab, int32_t per, const int32_t *__restrict__ ids,
    int32_t *__restrict__ perm, int32_t *__restrict__ word, int32_t *__restrict__ segptr) {
    __shared__ int32_t count[kOrderWaves][kOrderWords];  // of a wave's tokens; then its next place
    __shared__ uint32_t list[kOrderWaves][kOrderList];   // token less the wave's first, and word
    __shared__ int32_t below[kOrderWaves], scan[kOrderWords / kWave];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int lo = blockIdx.x * per;
    const int words = min(per, vocab - lo);
    for (int i = threadIdx.x; i < kOrderWaves * kOrderWords; i += kOrderThreads) (&count[0][0])[i] = 0;
    __syncthreads();
    const int piece = (ntok / (kOrderWaves * kOrderStep) + 1) * kOrderStep;
    const int first = (int)min((int64_t)wave * piece, (int64_t)ntok);
    const int last = (int)min((int64_t)first + piece, (int64_t)ntok);
    const uint64_t lower = (1ull << lane) - 1;
    int before = 0, kept = 0, done = last;  // done: the tokens from here on are not in the list
    constexpr int kAhead = 4;
    for (int b = first; b < last; b += kOrderStep * kAhead) {
        int id[kAhead][4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = b + u * kOrderStep + lane * 4;
            if (t + 4 <= last) {
                __builtin_memcpy(id[u], ids + t, sizeof id[u]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) id[u][e] = t + e < last ? ids[t + e] : -1;
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int t = b + u * kOrderStep;
            uint64_t here[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                before += id[u][e] >= 0 && id[u][e] < lo;
                here[e] = __ballot(id[u][e] >= lo && id[u][e] - lo < words);
            }
            if ((here[0] | here[1] | here[2] | here[3]) == 0) continue;
            int at = kept;
#pragma unroll
            for (int e = 0; e < 4; ++e) at += __popcll(here[e] & lower);
            if (kept + kOrderStep > kOrderList) done = min(done, t);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (!(here[e] >> lane & 1)) continue;
                const int x = id[u][e] - lo;
                atomicAdd(&count[wave][x], 1);
                if (done == last) list[wave][at++] = (uint32_t)(t + lane * 4 + e - first) << 8 | x;
            }
            if (done == last)
#pragma unroll
                for (int e = 0; e < 4; ++e) kept += __popcll(here[e]);
        }
    }
#pragma unroll
    for (int m = 1; m < kWave; m <<= 1) before += __shfl_xor(before, m, kWave);
    if (lane == 0) below[wave] = before;
    __syncthreads();
    int mine = 0, upto = 0;
    if (threadIdx.x < kOrderWords) {
        for (int w = 0; w < kOrderWaves; ++w) mine += count[w][threadIdx.x];
        upto = mine;
#pragma unroll
        for (int m = 1; m < kWave; m <<= 1) {
            const int x = __shfl_up(upto, m, kWave);
            if (lane >= m) upto += x;
        }
        if (lane == kWave - 1) scan[wave] = upto;
    }
    __syncthreads();
    if (threadIdx.x < kOrderWords) {
        for (int w = 0; w < wave; ++w) upto += scan[w];
        for (int w = 0; w < kOrderWaves; ++w) upto += below[w];
        int at = upto - mine;
        if (threadIdx.x < words) segptr[lo + threadIdx.x] = at;
        if (threadIdx.x == words - 1 && lo + words == vocab) segptr[vocab] = upto;
        for (int w = 0; w < kOrderWaves; ++w) {
            const int n = count[w][threadIdx.x];
            count[w][threadIdx.x] = at;
            at += n;
        }
    }
    __syncthreads();
    // a token a lane, in their order; x: its word in the block, or none of them
    auto put = [&](bool here, int x, int t) {
        uint64_t same = __ballot(here);  // lanes with this lane's word
        if (same == 0) return;
#pragma unroll
        for (int bit = 0; bit < 8; ++bit) {
            const uint64_t set = __ballot(here && (x >> bit & 1));
            same &= x >> bit & 1 ? set : ~set;
        }
        if (here) {
            const int place = count[wave][x], rank = __popcll(same & lower);
            perm[place + rank] = t;
            word[place + rank] = lo + x;
            if (rank == __popcll(same) - 1) count[wave][x] = place + rank + 1;
        }
        // the next ones read what another lane wrote
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    for (int i = 0; i < kept; i += kWave) {
        const bool here = i + lane < kept;
        const uint32_t v = here ? list[wave][i + lane] : 0;
        put(here, (int)(v & 255), first + (int)(v >> 8));
    }
    for (int b = done; b < last; b += kWave) {
        const int id = b + lane < last ? ids[b + lane] : -1;
        put(id >= lo && id - lo < words, id - lo, b + lane);
    }
}

// Ids as keys of a sort: padding behind every word.
__global__ __launch_bounds__(kEmbedThreads) void embed_keys_kernel(int32_t ntok, int32_t vocab,
                                                                   const int32_t *ids,
                                                                   int32_t *key) {
    const int64_t t = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x;
    if (t < ntok) key[t] = ids[t] >= 0 && ids[t] < vocab ? ids[t] : vocab;
}

// The first place of every word in the sorted keys.
__global__ __launch_bounds__(kEmbedThreads) void embed_starts_kernel(int32_t ntok, int32_t vocab,
                                                                     const int32_t *__restrict__ key,
                                                                     int32_t *__restrict__ segptr) {
    for (int64_t v = (int64_t)blockIdx.x * kEmbedThreads + threadIdx.x; v <= vocab;
         v += (int64_t)gridDim.x * kEmbedThreads) {
        int lo = 0, hi = ntok;
        while (lo < hi) {
            const int mid = lo + (hi - lo) / 2;
            if (key[mid] < v) lo = mid + 1;
            else hi = mid;
        }
        segptr[v] = lo;
    }
}

// ------------------------------------------------------------------- sums

struct EmbedSum {
    int32_t vocab, width, tiles, lanes, nchunks;
    bool accumulate;
    float scale;
    const int32_t *perm, *word, *segptr;
    int64_t ldw, ldo;
    float *part;  // [chunk][2][width]: of the word at its first place, and of another at its last
};

// Sums of n <= 64 rows' columns: lane from + i holds row i's token.  A slot of `lanes` lanes takes
// every (64 / lanes)th row; their sums are joined at the end, in one order.  NT tiles of a row:
// two where a row has more than one, as a wave's search for its tokens then serves twice the
// columns (32,768 tokens of 50,304 words of 1,024 columns 44 us, with one tile 54).
template <class TR, int N, int NT, bool WIDE>
__device__ __forceinline__ void add_rows(const EmbedSum &a, const TR *__restrict__ rows, int token,
                                         int from, int n, int tile, int lane,
                                         float (&acc)[NT][N]) {
    constexpr int kAhead = 8 / NT;
    const int slots = kWave / a.lanes, slot = lane / a.lanes;
    const int col = (tile * kWave + lane % a.lanes) * N;
    for (int i = 0; i < n; i += kAhead * slots) {
        Piece<N, TR, WIDE> x[kAhead][NT];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u * slots >= n) break;
            // (a slot past the end repeats the last row, and does not add it)
            const int64_t t = slots == 1 ? __builtin_amdgcn_readlane(token, from + i + u)
                                         : __shfl(token, from + min(i + u * slots + slot, n - 1), kWave);
#pragma unroll
            for (int k = 0; k < NT; ++k) x[u][k].load(rows + t * a.ldo, col + k * kWave * N, a.width);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i + u * slots >= n) break;
            if (i + u * slots + slot < n)
#pragma unroll
                for (int k = 0; k < NT; ++k)
#pragma unroll
                    for (int e = 0; e < N; ++e) acc[k][e] += x[u][k].value(e);
        }
    }
    for (int m = a.lanes; m < kWave; m <<= 1)
#pragma unroll
        for (int k = 0; k < NT; ++k)
#pragma unroll
            for (int e = 0; e < N; ++e) acc[k][e] += __shfl_xor(acc[k][e], m, kWave);
}

template <class TG, int N>
__device__ __forceinline__ void put_sum(const EmbedSum &a, TG *dW, int64_t v, int col,
                                        float (&acc)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) acc[e] *= a.scale;
    TG *const row = dW + v * a.ldw;
    if (a.accumulate) {
        float old[N];
        load_cols<N, TG>(row, col, a.width, old);
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += old[e];
    }
    store_cols<N, TG>(row, col, a.width, acc);
}

// Units: of words and NT tiles of columns, then of kLong places and NT tiles.
template <class TR, class TG, int N, int NT, bool WIDE>
__global__ __launch_bounds__(kEmbedThreads) void embed_sum_kernel(EmbedSum a, int64_t row_units,
                                                                  int64_t units,
                                                                  const TR *__restrict__ dout,
                                                                  TG *__restrict__ dW) {
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int groups = (a.tiles + NT - 1) / NT;
    for (int64_t u = (int64_t)blockIdx.x * kEmbedWaves + wave; u < units;
         u += (int64_t)gridDim.x * kEmbedWaves) {
        const bool rows = u < row_units;
        int64_t item = rows ? u : u - row_units;
        int tile = 0;
        if (groups > 1) {
            tile = (int)(item % groups) * NT;
            item /= groups;
        }
        const int col0 = (tile * kWave + lane % a.lanes) * N;
        const bool first = lane < a.lanes;  // of the slots that hold the same sums
        if (rows) {  // a word: the item's own, or (accumulate) the one that starts at this place
            int64_t v = item;
            if (a.accumulate) {
                if (item >= a.segptr[a.vocab]) continue;
                v = a.word[item];
                if (a.segptr[v] != item) continue;
            }
            const int lo = a.segptr[v], n = a.segptr[v + 1] - lo;
            if (n > kLong) continue;
            const int token = lane < n ? a.perm[lo + lane] : 0;
            float acc[NT][N] = {};
            add_rows<TR, N, NT, WIDE>(a, dout, token, 0, n, tile, lane, acc);
#pragma unroll
            for (int k = 0; k < NT; ++k) {
                const int col = col0 + k * kWave * N;
                if (!first || col >= a.width) continue;
                if (n == 0) store_cols<N, TG>(dW + v * a.ldw, col, a.width, acc[k]);
                else put_sum<TG, N>(a, dW, v, col, acc[k]);
            }
        } else {  // kLong places
            const int base = (int)item * kLong, end = min(base + kLong, a.segptr[a.vocab]);
            if (base >= end) continue;
            const bool on = base + lane < end;
            const int token = on ? a.perm[base + lane] : 0;
            const int w0 = a.word[base], w1 = a.word[end - 1];
            for (int side = 0; side < (w1 != w0 ? 2 : 1); ++side) {
                const int w = side ? w1 : w0;
                const int s0 = a.segptr[w], s1 = a.segptr[w + 1];
                if (s1 - s0 <= kLong) continue;
                const int from = max(s0, base) - base, n = min(s1, end) - base - from;
                float acc[NT][N] = {};
                add_rows<TR, N, NT, WIDE>(a, dout, token, from, n, tile, lane, acc);
#pragma unroll
                for (int k = 0; k < NT; ++k) {
                    const int col = col0 + k * kWave * N;
                    if (first && col < a.width)
                        store_cols<N, float>(a.part + (item * 2 + side) * a.width, col, a.width, acc[k]);
                }
            }
        }
    }
}

constexpr int kJoinThreads = 512;
constexpr int kJoinWaves = kJoinThreads / kWave;

// The long word that starts in chunk blockIdx.x / tiles (there is one at most): the sums of
// the chunks that it covers, consecutive ones by each wave, the waves' in their order.
template <class TG, int N>
__global__ __launch_bounds__(kJoinThreads) void embed_join_kernel(EmbedSum a, TG *__restrict__ dW) {
    __shared__ float sum[kJoinWaves][kWave * N];
    const int lane = threadIdx.x % kWave;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int chunk = blockIdx.x / a.tiles, tile = blockIdx.x % a.tiles;
    const int base = chunk * kLong, end = min(base + kLong, a.segptr[a.vocab]);
    if (base >= end) return;
    const int w = a.word[end - 1];
    const int s0 = a.segptr[w], s1 = a.segptr[w + 1];
    if (s1 - s0 <= kLong || s0 < base) return;
    const int col = (tile * kWave + lane) * N;
    const int nc = (s1 - 1) / kLong - chunk + 1;  // chunks that the word covers
    const int per = (nc + kJoinWaves - 1) / kJoinWaves;
    const int c0 = min(wave * per, nc), c1 = min(c0 + per, nc);
    float acc[N] = {};
    constexpr int kAhead = 8;
    for (int c = c0; c < c1; c += kAhead) {
        float x[kAhead][N];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int at = chunk + min(c + u, c1 - 1);
            const int side = at == chunk && s0 > base ? 1 : 0;  // not the word at its first place
            load_cols<N, float>(a.part + ((int64_t)at * 2 + side) * a.width, col, a.width, x[u]);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (c + u < c1)
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] += x[u][e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sum[wave][lane * N + e] = acc[e];
    __syncthreads();
    if (wave > 0 || col >= a.width) return;
    for (int o = 1; o < kJoinWaves; ++o)
#pragma unroll
        for (int e = 0; e < N; ++e) acc[e] += sum[o][lane * N + e];
    put_sum<TG, N>(a, dW, w, col, acc);
}

// ------------------------------------------------------------------- host

nsd_status check_embedding(int32_t ntok, const nsd_embedding *s) {
    NSD_REQUIRE(s != nullptr, "descriptor is NULL");
    NSD_REQUIRE(ntok >= 0, "negative number of tokens");
    NSD_REQUIRE(s->vocab >= 0 && s->width >= 1, "a table of %d rows of %d", s->vocab, s->width);
    NSD_REQUIRE(known_dtype(s->wtype) && known_dtype(s->otype) && known_dtype(s->gtype),
                "unknown type");
    NSD_REQUIRE(s->ldw >= s->width && s->ldo >= s->width, "row distances below the width %d",
                s->width);
    if (s->vocab == INT32_MAX || ntok > INT32_MAX - 2 * kLong || s->width > INT32_MAX - 1024)
        return fail(NSD_ERR_TOO_LARGE, "%d tokens, %d words of %d", ntok, s->vocab, s->width);
    return NSD_OK;
}

int values_per_lane(int32_t a, int32_t b) { return a == NSD_BF16 && b == NSD_BF16 ? 8 : 4; }

struct EmbedWs {
    int32_t *perm, *word, *segptr, *key;
    float *part;
    void *sort;
    size_t bytes;
    EmbedWs(void *ws, int32_t ntok, const nsd_embedding *s) {
        Carver c(ws);
        perm = c.take<int32_t>(ntok);
        word = c.take<int32_t>(ntok);
        segptr = c.take<int32_t>((size_t)s->vocab + 1);
        const int64_t nchunks = ntok > kLong ? ceil_div(ntok, kLong) : 0;
        part = c.take<float>((size_t)nchunks * 2 * s->width);
        key = nullptr;
        sort = nullptr;
        if (!by_looking(ntok, s->vocab)) {
            key = c.take<int32_t>(ntok);
            sort = c.take<char>(sort_ws_bytes(ntok, s->vocab + 1));
        }
        bytes = std::max<size_t>(c.bytes(), 256);
    }
};

// f(row type, gradient or output type, values per lane) by the descriptor's types
template <class F>
nsd_status by_types(int32_t a, int32_t b, F f) {
    if (a == NSD_F32) return b == NSD_F32 ? f(float(), float(), std::integral_constant<int, 4>())
                                          : f(float(), Bf16(), std::integral_constant<int, 4>());
    return b == NSD_F32 ? f(Bf16(), float(), std::integral_constant<int, 4>())
                        : f(Bf16(), Bf16(), std::integral_constant<int, 8>());
}

}  // namespace

}  // namespace nsd

using namespace nsd;

extern "C" {

nsd_status nsd_embed(int32_t ntok, const nsd_embedding *s, const int32_t *ids, const void *W,
                     void *out, void *stream) {
    NSD_TRY(check_embedding(ntok, s));
    if (ntok == 0) return NSD_OK;
    NSD_REQUIRE(ids && out && (W || s->vocab == 0), "a NULL array");
    NSD_TRY(check_apart({row_area(out, ntok, s->width, s->ldo, s->otype)},
                        {row_area(W, s->vocab, s->width, s->ldw, s->wtype), flat_area(ids, 4 * (int64_t)ntok)}));
    const int values = values_per_lane(s->wtype, s->otype), lanes = row_lanes(s->width, values);
    const int tiles = (int)ceil_div(s->width, kWave * values);
    const int64_t units = ceil_div(ntok, kWave / lanes) * tiles;
    const int64_t blocks = std::min(ceil_div(units, kEmbedWaves), kMaxEmbedBlocks);
    return by_types(s->wtype, s->otype, [&](auto w, auto o, auto n) -> nsd_status {
        using TW = decltype(w);
        using TO = decltype(o);
        embed_kernel<TW, TO, decltype(n)::value><<<blocks, kEmbedThreads, 0, as_stream(stream)>>>(
            ntok, units, tiles, lanes, s->vocab, s->width, s->scale, ids, static_cast<const TW *>(W), s->ldw,
            static_cast<TO *>(out), s->ldo);
        return check_launch("embed_kernel");
    });
}

nsd_status nsd_embed_vjp_workspace_size(int32_t ntok, const nsd_embedding *s, size_t *bytes) {
    NSD_REQUIRE(bytes != nullptr, "bytes is NULL");
    NSD_TRY(check_embedding(ntok, s));
    *bytes = EmbedWs(nullptr, ntok, s).bytes;
    return NSD_OK;
}

nsd_status nsd_embed_vjp(int32_t ntok, const nsd_embedding *s, const int32_t *ids,
                         const void *dout, int32_t accumulate, void *dW, void *ws,
                         size_t ws_bytes, void *stream) {
    NSD_TRY(check_embedding(ntok, s));
    if (s->vocab == 0 || (accumulate && ntok == 0)) return NSD_OK;
    NSD_REQUIRE(dW && (ntok == 0 || (ids && dout)), "a NULL array");
    const EmbedWs w(ws, ntok, s);
    if (ws == nullptr || ws_bytes < w.bytes)
        return fail(NSD_ERR_WORKSPACE, "workspace %zu bytes at %p, need %zu", ws_bytes, ws, w.bytes);
    NSD_REQUIRE((reinterpret_cast<uintptr_t>(ws) & 255) == 0, "workspace is not 256-byte aligned");
    NSD_TRY(check_apart({row_area(dW, s->vocab, s->width, s->ldw, s->gtype), flat_area(ws, (int64_t)w.bytes)},
                        {row_area(dout, ntok, s->width, s->ldo, s->otype), flat_area(ids, 4 * (int64_t)ntok)}));
    const int values = values_per_lane(s->otype, s->gtype);
    EmbedSum a;
    a.tiles = (int)ceil_div(s->width, kWave * values);
    a.nchunks = ntok > kLong ? (int)ceil_div(ntok, kLong) : 0;
    const int64_t joins = (int64_t)a.nchunks * a.tiles;
    if (joins > UINT32_MAX / kJoinThreads)
        return fail(NSD_ERR_TOO_LARGE, "%lld sums of long words", (long long)joins);
    const hipStream_t st = as_stream(stream);
    if (w.key == nullptr) {
        const int per = words_of_block(s->vocab);
        embed_order_kernel<<<ceil_div(s->vocab, per), kOrderThreads, 0, st>>>(
            ntok, s->vocab, per, ids, w.perm, w.word, w.segptr);
        NSD_TRY(check_launch("embed_order_kernel"));
    } else {
        if (ntok > 0) {
            embed_keys_kernel<<<ceil_div(ntok, kEmbedThreads), kEmbedThreads, 0, st>>>(ntok, s->vocab,
                                                                                      ids, w.key);
            NSD_TRY(check_launch("embed_keys_kernel"));
            NSD_TRY(radix_sort_pairs(ntok, s->vocab + 1, w.key, nullptr, w.word, w.perm, w.sort, st));
        }
        const int64_t starts = std::min(ceil_div((int64_t)s->vocab + 1, kEmbedThreads), kMaxEmbedBlocks);
        embed_starts_kernel<<<starts, kEmbedThreads, 0, st>>>(ntok, s->vocab, w.word, w.segptr);
        NSD_TRY(check_launch("embed_starts_kernel"));
    }
    a.vocab = s->vocab;
    a.width = s->width;
    a.lanes = row_lanes(s->width, values);
    a.accumulate = accumulate != 0;
    a.scale = s->scale;
    a.perm = w.perm;
    a.word = w.word;
    a.segptr = w.segptr;
    a.ldw = s->ldw;
    a.ldo = s->ldo;
    a.part = w.part;
    const int groups = (int)ceil_div(a.tiles, a.tiles > 1 ? 2 : 1);
    const int64_t row_units = (int64_t)(accumulate ? ntok : s->vocab) * groups;
    const int64_t units = row_units + (int64_t)a.nchunks * groups;
    const int64_t blocks = std::min(ceil_div(units, kEmbedWaves), kMaxEmbedBlocks);
    return by_types(s->otype, s->gtype, [&](auto r, auto g, auto n) -> nsd_status {
        using TR = decltype(r);
        using TG = decltype(g);
        constexpr int N = decltype(n)::value;
        const TR *const rows = static_cast<const TR *>(dout);
        TG *const to = static_cast<TG *>(dW);
        auto sum = [&](auto nt, auto wide) {
            embed_sum_kernel<TR, TG, N, decltype(nt)::value, decltype(wide)::value>
                <<<blocks, kEmbedThreads, 0, st>>>(a, row_units, units, rows, to);
        };
        if (a.tiles > 1) sum(std::integral_constant<int, 2>(), std::true_type());
        else if (a.width >= N) sum(std::integral_constant<int, 1>(), std::true_type());
        else sum(std::integral_constant<int, 1>(), std::false_type());
        NSD_TRY(check_launch("embed_sum_kernel"));
        if (a.nchunks == 0) return NSD_OK;
        embed_join_kernel<TG, N><<<joins, kJoinThreads, 0, st>>>(a, static_cast<TG *>(dW));
        return check_launch("embed_join_kernel");
    });
}

}  // extern "C"
