// kv_evict: the cache of a layer brought down to `budget` rows per sequence and key head - the first positions, the last ones and,
// of the others, those that have gathered the most attention weight.
//
// Keys carry their position in themselves and attention does not ask for an order, so nothing has to move but the kept rows
// behind the budget, into the places of the rows that go: the j-th such row into the j-th such place.  Sources lie behind the budget and
// places before it, so the moves need no order among each other, and the call reads and writes only what moves.
//   * kv_evict_select_kernel - one workgroup per (sequence, key head): the budget-th largest weight by a radix search, then
//                              which row of the old cache every row of the new one is
//   * kv_evict_move_kernel   - the moves, and the kept rows' weights and positions
#include "common.h"

namespace ctcspec {

struct KvEvictParams {
  unsigned char* k_cache;
  unsigned char* v_cache;
  const int64_t* kv_off;
  const int32_t* ctx_len;
  const float* weight;      // [B][H_kv][kv_cap]
  const int32_t* pos;       // [B][H_kv][kv_cap] or null
  const int32_t* next_pos;  // [B] or null
  int32_t* kept;            // [B][H_kv][budget]
  float* weight_out;        // [B][H_kv][kv_cap]
  int32_t* pos_out;         // [B][H_kv][kv_cap] or null
  int32_t* ctx_len_out;     // [B]
  int kv_cap, H_kv, budget, sink, recent;
  int row_bytes, elem_bytes;
};

constexpr int kEvWaves = 16, kEvThreads = 64 * kEvWaves;
constexpr int kEvBins = 2048;      // of a digit of up to 11 bits
constexpr int kEvCopies = 4;       // of every bin, for lanes next to each other: equal digits are common, and additions to one place follow one another
constexpr int kEvIndexBits = 20;   // of a row
constexpr int kEvMaxRows = 1 << 19;
constexpr int kEvListed = 4096;    // rows that are listed once their number is below that
constexpr int kEvTies = 256;       // ... and that are compared with each other
constexpr int kEvList = 8192;      // moved rows per round
// LDS, one after the other in the same place: the bins of the search; for every 64 rows the bits of those that are still to be
// decided; the bins and the list of those rows; the rows that are compared; for every 64 rows how many of the kind that counts there
// lie before them, and the list of the moved rows.  Behind that, for every 64 rows, the bits of those that stay.
constexpr int kEvBinBytes = kEvBins * kEvCopies * 4, kEvListBytes = kEvBinBytes + kEvList * 4;
static_assert(kEvMaxRows / 64 * 8 <= kEvListBytes && kEvMaxRows / 64 * 4 <= kEvBinBytes);
static_assert(kEvListed <= kEvList && kEvTies * 8 <= kEvBinBytes && kEvListed % kEvThreads == 0 && kEvTies % 64 == 0 && kEvTies <= 64 * kEvWaves);
constexpr size_t evict_lds_bytes(int kv_cap) { return kEvListBytes + (size_t)((kv_cap + 63) / 64) * 8; }

// Order of the rows: larger weight first, then smaller index; rows that stay in any case before all others; a weight that is not
// a number behind all others.  (last: positions behind it stay.)
__device__ __forceinline__ unsigned int evict_key(float weight, int pos, int sink, int last) {
  const unsigned int u = __float_as_uint(weight + 0.0f);  // (-0 becomes 0)
  const unsigned int key = weight != weight ? 0u : u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
  return pos < sink || pos > last ? 0xffffffffu : key;
}

// The order is that of the key, then of the index from the top - no two rows have the same place -, searched digit by digit for
// the n-th until the rows that share the digits so far all stay or are few enough to be compared with each other.  Then a
// bit for every row that stays, and everything else follows from counts of bits.
// K: a lane holds up to K keys in registers (rows 64 k + lane of its wavefront's range): the passes read memory once.  0: for
// capacities beyond that; every pass reads the weights again, eight rows of a lane at a time and the next eight under way.  (The
// call in us with the keys in registers / read again: 700 rows 12.3 / 18.3, 2304 rows 27.1 / 35.7, 4000 rows 27.3 / 37.4, 12000 rows
// 59.8 / 66.1; with 96 rows in registers 65536 rows 91 / 74: they leave none for the rows of a step.  It goes by the capacity, as the host
// does not know the lengths: 8 x 32 heads from 700 rows to 512 take 15.7 us with room for 704, 17.2 for 16384 and 21.5 for 20000.)
// What bounds it: up to some thousand rows the steps' latencies, one workgroup behind each other's barriers; beyond, instructions - a
// compute unit takes a cycle for one on 64 rows -, of which a row takes about 20 in each of the two or three passes.  (32 heads of
// 65536 rows to 4096: 43 us; 256 heads of 2304 rows to 2048: 10.5 us.)
template <int K>
__global__ __launch_bounds__(kEvThreads) void kv_evict_select_kernel(KvEvictParams p) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ int wsum[kEvWaves];
  __shared__ int found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kh = blockIdx.x, b = blockIdx.y;
  int L = __builtin_amdgcn_readfirstlane(p.ctx_len[b]);
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int n = L < p.budget ? L : p.budget;
  const size_t head = (size_t)b * p.H_kv + kh;
  int32_t* kept = p.kept + head * p.budget;
  if (kh == 0 && tid == 0) p.ctx_len_out[b] = n;
  for (int j = n + tid; j < p.budget; j += kEvThreads) kept[j] = -1;
  if (L <= p.budget) {
    for (int j = tid; j < n; j += kEvThreads) kept[j] = j;
    return;
  }
  unsigned int* hist = (unsigned int*)smem;
  unsigned long long* ties = (unsigned long long*)smem;
  int* count = (int*)smem;
  unsigned long long* open = (unsigned long long*)smem;
  int* list = (int*)(smem + kEvBinBytes);
  const int words = (L + 63) / 64;
  unsigned long long* bits = (unsigned long long*)(smem + kEvListBytes);

  const float* w = p.weight + head * p.kv_cap;
  const int32_t* pos = p.pos ? p.pos + head * p.kv_cap : nullptr;
  int sink = -0x7fffffff - 1, last = 0x7fffffff;  // (without pos, and without recent: no position is before the one or behind the other)
  if (pos) sink = p.sink;
  if (p.recent > 0) {
    const long long before = (long long)p.next_pos[b] - p.recent - 1;
    last = before < -0x7fffffffLL - 1 ? -0x7fffffff - 1 : (int)before;
  }
  const int range = (words + kEvWaves - 1) / kEvWaves * 64, j0 = wave * range;  // this wavefront's rows
  const int rows = j0 < L ? (L - j0 < range ? L - j0 : range) : 0;
  // weights and positions of rows j0 + 64 (k0 + i) + lane, i < N (behind the last row: the last one again), and their keys
  auto load = [&]<int N>(int k0, float (&v)[N], int (&at)[N]) __attribute__((always_inline)) {
    if (64 * (k0 + N) <= rows) {
      const unsigned int off = lane * 4u;
      const char *wk = (const char*)(w + j0 + 64 * k0), *pk = (const char*)(pos + j0 + 64 * k0);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        v[i] = *(const float*)(wk + off + i * 256);
        at[i] = pos ? *(const int32_t*)(pk + off + i * 256) : 0;
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const unsigned int j = (unsigned)(j0 + 64 * (k0 + i) + lane), last = (unsigned)L - 1u, off = (j < last ? j : last) * 4u;
        v[i] = *(const float*)((const char*)w + off);
        at[i] = pos ? *(const int32_t*)((const char*)pos + off) : 0;
      }
    }
  };
  unsigned int mine[K ? K : 1];
  if constexpr (K > 0) {
    constexpr int N = K < 16 ? K : 16;
#pragma unroll
    for (int k = 0; k < K; k += N) {
      float v[N];
      int at[N];
      load(k, v, at);
#pragma unroll
      for (int i = 0; i < N; ++i) mine[k + i] = evict_key(v[i], at[i], sink, last);
#pragma unroll
      for (int i = 0; i < N; ++i) asm volatile("" : "+v"(mine[k + i]));
    }
  }
  // f(k, whether the rows exist, their keys) for G of the lane's rows at a time, from row k on.  (Nothing but instructions bounds a
  // pass over many rows - one costs a compute unit a cycle for every 64 of them -, so rows that all exist are not asked.)
  constexpr int G = K && K < 8 ? K : 8;
  auto some = [&](int k, const unsigned int (&key)[G], auto&& f) __attribute__((always_inline)) {
    bool there[G];
    if (64 * (k + G) <= rows) {
#pragma unroll
      for (int i = 0; i < G; ++i) there[i] = true;
      f(k, there, key);
    } else {
#pragma unroll
      for (int i = 0; i < G; ++i) there[i] = 64 * (k + i) + lane < rows;
      f(k, there, key);
    }
  };
  auto each = [&](auto&& f) __attribute__((always_inline)) {
    unsigned int key[G];
    if constexpr (K > 0) {
#pragma unroll
      for (int k = 0; k < K; k += G) {
        if (64 * k >= rows) continue;
#pragma unroll
        for (int i = 0; i < G; ++i) key[i] = mine[k + i];
        some(k, key, f);
      }
    } else {
      float v[G], next_v[G];  // with as many more under way
      int at[G], next_at[G];
      if (rows > 0) load(0, v, at);
      for (int k = 0; 64 * k < rows; k += G) {
        load(k + G, next_v, next_at);
#pragma unroll
        for (int i = 0; i < G; ++i) key[i] = evict_key(v[i], at[i], sink, last);
        some(k, key, f);
#pragma unroll
        for (int i = 0; i < G; ++i) {
          v[i] = next_v[i];
          at[i] = next_at[i];
        }
      }
    }
  };
  // a row's index from the top (formed where it is needed: K of them would take as many registers as the keys)
  auto from_top = [&](int k) __attribute__((always_inline)) {
    int l = lane;
    asm volatile("" : "+v"(l));
    return (unsigned)((1 << kEvIndexBits) - 1 - (j0 + 64 * k + l));
  };

  // ---- the search: `want` of the `same` rows that share the digits so far stay, and all before them --------------------------------------
  // (keys in registers cost little to go over again)
  constexpr int kMost = K ? kEvTies : kEvListed;
  int want = n, same = L;
  // one digit: counts(f): f(whether a row counts, its digit)
  auto digit = [&](auto&& counts) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kEvBins * kEvCopies / kEvThreads / 4; ++i) ((u32x4*)hist)[tid + i * kEvThreads] = u32x4{0u, 0u, 0u, 0u};
    __syncthreads();
    counts([&](bool here, unsigned int bin) __attribute__((always_inline)) {
      if (here) atomicAdd(&hist[bin * kEvCopies + (lane & (kEvCopies - 1))], 1u);
    });
    __syncthreads();
    // thread t: bins 2 t and 2 t + 1 from the top; how many rows lie in the bins above
    const int hi = kEvBins - 1 - 2 * tid;
    static_assert(kEvCopies == 4 && kEvBins == 2 * kEvThreads);
    const u32x4 h1 = ((const u32x4*)hist)[hi], h0 = ((const u32x4*)hist)[hi - 1];
    const int c1 = (int)(h1[0] + h1[1] + h1[2] + h1[3]), c0 = (int)(h0[0] + h0[1] + h0[2] + h0[3]);
    int sum = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int other = __shfl_up(sum, o, 64);
      if (lane >= o) sum += other;
    }
    if (lane == 63) wsum[wave] = sum;
    __syncthreads();
    int above = sum - c0 - c1;
    for (int v = 0; v < wave; ++v) above += wsum[v];
    if (above < want && want <= above + c1) { found[0] = hi; found[1] = above; found[2] = c1; }
    else if (above + c1 < want && want <= above + c1 + c0) { found[0] = hi - 1; found[1] = above + c1; found[2] = c0; }
    __syncthreads();
    want -= found[1];
    same = found[2];
    return (unsigned)found[0];
  };
  // the key's digits: 11, 11 and 10 bits
  unsigned int prefix = 0u;
  int shift = 32;
  if (same > kMost) {
    shift = 21;
    prefix = digit([&](auto&& f) __attribute__((always_inline)) {
      each([&](int, const bool (&there)[G], const unsigned int (&key)[G]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G; ++i) f(there[i], key[i] >> 21);
      });
    });
  }
  while (shift > 0 && same > want && same > kMost) {
    const int bits_of = shift == 21 ? 11 : 10, above = shift;
    shift -= bits_of;
    const unsigned int d = digit([&](auto&& f) __attribute__((always_inline)) {
      each([&](int, const bool (&there)[G], const unsigned int (&key)[G]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G; ++i) f(there[i] && key[i] >> above == prefix, (key[i] >> shift) & ((1u << bits_of) - 1u));
      });
    });
    prefix = prefix << bits_of | d;
  }
  // (equal keys) the index's digits: 10 bits each
  unsigned int iprefix = 0u;
  int ishift = kEvIndexBits;
  while (ishift > 0 && same > want && same > kMost) {
    const int above = ishift;
    ishift -= 10;
    const unsigned int d = digit([&](auto&& f) __attribute__((always_inline)) {
      each([&](int k, const bool (&there)[G], const unsigned int (&key)[G]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
          const unsigned int at = from_top(k + i);
          f(there[i] && key[i] == prefix && at >> above == iprefix, (at >> ishift) & 1023u);
        }
      });
    });
    iprefix = iprefix << 10 | d;
  }
  // ---- a bit for every row that stays; the others that share the digits so far ---------------------------------------------------------
  const bool compare = same > want;
  auto place_of = [&](unsigned int key, unsigned int from_top) __attribute__((always_inline)) {  // key, index from the top
    return (unsigned long long)(key >> (32 - kEvIndexBits)) << 32 | (key << kEvIndexBits | from_top);
  };
  __syncthreads();  // (everyone has read what the last digit found)
  if (tid == 0) found[0] = 0;
  __syncthreads();
  each([&](int k, const bool (&there)[G], const unsigned int (&key)[G]) __attribute__((always_inline)) {
    unsigned long long stay = 0ull, tied = 0ull;  // lane i: the bits of rows 64 (k + i) ..
#pragma unroll
    for (int i = 0; i < G; ++i) {
      const unsigned int top = shift == 32 ? 0u : key[i] >> (shift & 31);  // (no digit was looked at: all rows share what there is)
      bool sure = there[i] && top > prefix, tie = there[i] && top == prefix;
      if (ishift < kEvIndexBits) {
        const unsigned int at = from_top(k + i) >> ishift;
        sure |= tie && at > iprefix;
        tie &= at == iprefix;
      }
      const unsigned long long m = __builtin_amdgcn_ballot_w64(sure), tm = __builtin_amdgcn_ballot_w64(tie);
      stay = lane == i ? m : stay;
      tied = lane == i ? tm : tied;
      if constexpr (K > 0) {
        if (compare && tm != 0ull) {
          int at = 0;
          if (lane == 0) at = atomicAdd(&found[0], __builtin_popcountll(tm));
          at = __builtin_amdgcn_readfirstlane(at) + __builtin_popcountll(tm & ((1ull << lane) - 1ull));
          if (tie) ties[at] = place_of(key[i], from_top(k + i));
        }
      }
    }
    if (lane < G && 64 * (k + lane) < rows) {
      bits[j0 / 64 + k + lane] = compare ? stay : stay | tied;
      if (K == 0 && compare) open[j0 / 64 + k + lane] = tied;
    }
  });
  __syncthreads();
  if (compare) {
    auto stays = [&](unsigned long long place) __attribute__((always_inline)) {
      const int j = (1 << kEvIndexBits) - 1 - (int)(place & ((1u << kEvIndexBits) - 1u));
      atomicOr((unsigned int*)bits + j / 32, 1u << (j & 31));
    };
    if constexpr (K == 0) {  // more than can be compared: a list of them, and the rest of the digits
      constexpr int kMine = kEvListed / kEvThreads, kWords = kEvMaxRows / 64 / kEvThreads;
      unsigned long long tied[kWords];
#pragma unroll
      for (int i = 0; i < kWords; ++i) tied[i] = tid + i * kEvThreads < words ? open[tid + i * kEvThreads] : 0ull;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kWords; ++i)
        if (tied[i]) {
          int at = atomicAdd(&found[0], __builtin_popcountll(tied[i]));
          for (unsigned long long left = tied[i]; left; left &= left - 1ull) list[at++] = 64 * (tid + i * kEvThreads) + __builtin_ctzll(left);
        }
      __syncthreads();
      unsigned long long place[kMine];
      const int entries = same;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        place[i] = 0ull;
        if (tid + i * kEvThreads < entries) {
          const int j = list[tid + i * kEvThreads];
          place[i] = place_of(evict_key(w[j], pos ? pos[j] : 0, sink, last), (unsigned)((1 << kEvIndexBits) - 1 - j));
        }
      }
      int low = ishift < kEvIndexBits ? ishift : shift + kEvIndexBits;  // the bits below are still to be looked at
      unsigned long long first = ishift < kEvIndexBits ? (unsigned long long)prefix << (kEvIndexBits - ishift) | iprefix : prefix;
      while (same > want && same > kEvTies) {  // (no two places are the same)
        const int above = low, bits_of = low < 11 ? low : 11;
        low -= bits_of;
        const unsigned int d = digit([&](auto&& f) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < kMine; ++i)
            f(tid + i * kEvThreads < entries && place[i] >> above == first, (unsigned)(place[i] >> low) & ((1u << bits_of) - 1u));
        });
        first = first << bits_of | d;
      }
      __syncthreads();
      if (tid == 0) found[0] = 0;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        if (tid + i * kEvThreads >= entries) continue;
        const unsigned long long top = place[i] >> low;
        if (top > first || (top == first && same == want)) stays(place[i]);
        else if (top == first) ties[atomicAdd(&found[0], 1)] = place[i];
      }
      __syncthreads();
    }
    if (same > want && wave < same) {  // `want` of these: wavefront v counts those before number v, v + 16 .., 64 at a time
      unsigned long long all[kEvTies / 64];
#pragma unroll
      for (int i = 0; i < kEvTies / 64; ++i) all[i] = 64 * i + lane < same ? ties[64 * i + lane] : 0ull;
      const int own = wave + lane * kEvWaves;
      const unsigned long long place = own < same ? ties[own] : 0ull;
      int rank = 0;
      for (int i = 0; wave + i * kEvWaves < same; ++i) {
        const unsigned long long at = (unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(place >> 32), i) << 32 |
                                      (unsigned)__builtin_amdgcn_readlane((int)place, i);
        int before = 0;
#pragma unroll
        for (int v = 0; v < kEvTies / 64; ++v)
          if (64 * v < same) before += __builtin_popcountll(__builtin_amdgcn_ballot_w64(all[v] > at));
        rank = lane == i ? before : rank;
      }
      if (own < same && rank < want) stays(place);
    }
    __syncthreads();
  }
  // ---- for every 64 rows: free places (below n) and moving rows (from n on) before them ------------------------------------------------
  // (n is in the middle of one word, whose rows are of both kinds: its count of moving rows begins at 0, as that of all words behind)
  auto free_of = [&](int x) __attribute__((always_inline)) {
    const int left = n - 64 * x;
    return left <= 0 ? 0ull : ~bits[x] & (left >= 64 ? ~0ull : (1ull << left) - 1ull);
  };
  auto moving_of = [&](int x) __attribute__((always_inline)) {
    const int left = n - 64 * x;
    return left >= 64 ? 0ull : bits[x] & (left <= 0 ? ~0ull : ~((1ull << left) - 1ull));
  };
  int total = 0;
  {
    int carry = 0;
    for (int x0 = 0; x0 < words; x0 += kEvThreads) {
      const int x = x0 + tid;
      // one sum over both kinds: free places of the words up to n's, then moving rows on top of all of them
      const int f = x < words ? __builtin_popcountll(free_of(x)) : 0, m = x < words ? __builtin_popcountll(moving_of(x)) : 0;
      int sum = f + m;
#pragma unroll
      for (int o = 1; o < 64; o *= 2) {
        const int other = __shfl_up(sum, o, 64);
        if (lane >= o) sum += other;
      }
      __syncthreads();
      if (lane == 63) wsum[wave] = sum;
      __syncthreads();
      int before = carry + sum - f - m, all = 0;
      for (int v = 0; v < kEvWaves; ++v) {
        before += v < wave ? wsum[v] : 0;
        all += wsum[v];
      }
      if (x < words) count[x] = before;
      carry += all;
    }
    total = carry / 2;  // as many free places as moving rows
  }
  __syncthreads();
  // ---- the j-th moving row into the j-th free place, kEvList of them at a time ---------------------------------------------------------
  const int nword = n / 64;  // words from here on may have moving rows; their counts begin behind `total` free places
  for (int from = 0; from == 0 || from < total; from += kEvList) {
    if (from) __syncthreads();
    for (int y = nword * 8 + tid; y < words * 8; y += kEvThreads) {  // eight rows
      const int x = y / 8, at = y % 8 * 8;
      const unsigned long long m = moving_of(x);
      int rank = count[x] + (x == nword ? __builtin_popcountll(free_of(x)) : 0) - total + __builtin_popcountll(m & ((1ull << at) - 1ull)) - from;
      for (unsigned int left = (unsigned)(m >> at) & 255u; left; left &= left - 1u, ++rank)
        if (rank >= 0 && rank < kEvList) list[rank] = 64 * x + at + __builtin_ctz(left);
    }
    __syncthreads();
    for (int j = tid; j < n; j += kEvThreads) {
      const int x = j / 64;  // (the same for a wavefront)
      const unsigned long long f = free_of(x);
      if ((f >> lane) & 1ull) {
        const int rank = count[x] + __builtin_popcountll(f & ((1ull << lane) - 1ull)) - from;
        if (rank >= 0 && rank < kEvList) kept[j] = list[rank];
      } else if (from == 0) {
        kept[j] = j;
      }
    }
  }
}

// a wavefront per 64 rows of the new cache
__global__ __launch_bounds__(256) void kv_evict_move_kernel(KvEvictParams p) {
  __shared__ int todo[4][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int kh = blockIdx.y, b = blockIdx.z;
  int L = p.ctx_len[b];
  L = L < 0 ? 0 : (L > p.kv_cap ? p.kv_cap : L);
  const int n = L < p.budget ? L : p.budget;
  const int j = (blockIdx.x * 4 + wave) * 64 + lane;
  const size_t head = (size_t)b * p.H_kv + kh;
  int src = j;
  if (j < n) {
    src = p.kept[head * p.budget + j];
    p.weight_out[head * p.kv_cap + j] = p.weight[head * p.kv_cap + src];
    if (p.pos) p.pos_out[head * p.kv_cap + j] = p.pos[head * p.kv_cap + src];
  }
  const bool moves = src != j;
  const unsigned long long m = __builtin_amdgcn_ballot_w64(moves);
  if (m == 0ull) return;
  if (moves) todo[wave][__builtin_popcountll(m & ((1ull << lane) - 1ull))] = lane;
  const int count = __builtin_popcountll(m), chunks = p.row_bytes / 16;
  const int first = j - lane;
  unsigned char* kc = p.k_cache + (size_t)p.kv_off[b] * p.elem_bytes + (size_t)kh * p.kv_cap * p.row_bytes;
  unsigned char* vc = p.v_cache + (size_t)p.kv_off[b] * p.elem_bytes + (size_t)kh * p.kv_cap * p.row_bytes;
  __builtin_amdgcn_wave_barrier();
  for (int x0 = 0; x0 < count * chunks; x0 += 64) {
    const int x = x0 + lane, i = x / chunks, row = i < count ? todo[wave][i] : 0;
    const int from = __shfl(src, row, 64);
    if (i < count) {
      const size_t s = (size_t)from * p.row_bytes + (x - i * chunks) * 16, d = (size_t)(first + row) * p.row_bytes + (x - i * chunks) * 16;
      const u32x4 k = *(const u32x4*)(kc + s), v = *(const u32x4*)(vc + s);
      *(u32x4*)(kc + d) = k;
      *(u32x4*)(vc + d) = v;
    }
  }
}

// f(kernel) for the one that a capacity takes (the lengths are known on the device)
template <typename F>
static hipError_t with_select(int kv_cap, F&& f) {
  if (kv_cap <= 4 * kEvThreads) return f(kv_evict_select_kernel<4>);
  if (kv_cap <= 16 * kEvThreads) return f(kv_evict_select_kernel<16>);
  return f(kv_evict_select_kernel<0>);
}

hipError_t prepare_kv_evict() {
  hipError_t e = hipSuccess;
  for (int cap : {4 * kEvThreads, 16 * kEvThreads, kEvMaxRows}) {
    if (e != hipSuccess) break;
    e = with_select(cap, [&](auto kernel) {
      return hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)evict_lds_bytes(cap));
    });
  }
  return e;
}

}  // namespace ctcspec

using namespace ctcspec;

extern "C" int kv_evict(ctcspec_ctx* ctx, ctcspec_dtype dt, void* k_cache, void* v_cache, const int64_t* kv_off,
                        const int32_t* ctx_len, int kv_cap, const float* weight, const int32_t* pos, const int32_t* next_pos, int B,
                        int H_kv, int dh, int budget, int sink, int recent, int32_t* kept, float* weight_out, int32_t* pos_out,
                        int32_t* ctx_len_out) {
  if (!ctx) return CTCSPEC_EINVAL;
  if (const int owed = flush_deferred(ctx)) return owed;
  CTCSPEC_REQUIRE(ctx, k_cache && v_cache && kv_off && ctx_len && weight && kept && weight_out && ctx_len_out, CTCSPEC_EINVAL,
                  "kv_evict: null pointer");
  CTCSPEC_REQUIRE(ctx, B > 0 && H_kv > 0 && dh > 0 && kv_cap > 0 && budget > 0, CTCSPEC_EINVAL, "kv_evict: sizes must be positive");
  CTCSPEC_REQUIRE(ctx, dt == CTCSPEC_F32 || dt == CTCSPEC_BF16, CTCSPEC_EINVAL, "kv_evict: unknown element type");
  CTCSPEC_REQUIRE(ctx, sink >= 0 && recent >= 0 && (long long)sink + recent <= budget, CTCSPEC_EINVAL,
                  "kv_evict: sink and recent must not be negative and fit the budget together");
  CTCSPEC_REQUIRE(ctx, (pos != nullptr) == (pos_out != nullptr) && (pos || sink + recent == 0) && (next_pos || recent == 0),
                  CTCSPEC_EINVAL, "kv_evict: sink and recent need pos and pos_out, recent needs next_pos");
  CTCSPEC_REQUIRE(ctx, weight_out != weight && (!pos || pos_out != pos) && ctx_len_out != ctx_len, CTCSPEC_EINVAL,
                  "kv_evict: weight_out, pos_out and ctx_len_out must not be the inputs");
  CTCSPEC_REQUIRE(ctx, dh % 8 == 0 && dh <= CTCSPEC_MAX_HEAD_DIM && B <= ctx->lim.max_batch && H_kv <= ctx->lim.max_heads &&
                           dh <= ctx->lim.max_head_dim && B <= 65535 && H_kv <= 65535 && kv_cap <= kEvMaxRows && budget <= (1 << 30),
                  CTCSPEC_EUNSUPPORTED, "kv_evict: dh must be a multiple of 8 and <= %d, kv_cap <= %d, budget <= 2^30, the shape within the context's limits",
                  CTCSPEC_MAX_HEAD_DIM, kEvMaxRows);
  CTCSPEC_REQUIRE(ctx, aligned16(k_cache) && aligned16(v_cache), CTCSPEC_EINVAL, "kv_evict: the caches must be 16-byte aligned");
  KvEvictParams p;
  p.k_cache = (unsigned char*)k_cache; p.v_cache = (unsigned char*)v_cache; p.kv_off = kv_off; p.ctx_len = ctx_len;
  p.weight = weight; p.pos = pos; p.next_pos = next_pos; p.kept = kept; p.weight_out = weight_out; p.pos_out = pos_out;
  p.ctx_len_out = ctx_len_out; p.kv_cap = kv_cap; p.H_kv = H_kv; p.budget = budget; p.sink = sink; p.recent = recent;
  p.elem_bytes = dt == CTCSPEC_F32 ? 4 : 2;
  p.row_bytes = dh * p.elem_bytes;
  CTCSPEC_HIP(ctx, with_select(kv_cap, [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)H_kv, (unsigned)B), dim3(kEvThreads), evict_lds_bytes(kv_cap), ctx->stream, p);
    return hipGetLastError();
  }));
  const int rows = budget < kv_cap ? budget : kv_cap;
  hipLaunchKernelGGL(kv_evict_move_kernel, dim3((unsigned)((rows + 255) / 256), (unsigned)H_kv, (unsigned)B), dim3(256), 0, ctx->stream, p);
  CTCSPEC_HIP(ctx, hipGetLastError());
  return CTCSPEC_OK;
}
