// Eviction from a paged cache by accumulated attention weight: which slots stay, and the rows that move for it.
#include "sttm_cache.h"

#include <algorithm>

namespace sttm {
namespace {

struct EvictArgs {
  Pool pool;
  Seqs seqs;
  const int32_t *keep, *total;
  long long slot_stride;
  const float *weights_in, *bias_in;
  const int32_t* ids_in;
  float *weights_out, *bias_out;
  int32_t *ids_out, *lengths_out;
  int kv_heads, sink, recent;
  uint32_t* keys;              // [batch, kv_heads, max_len], of long rows, and
  unsigned short* digits;      // [batch, kv_heads, parts, 1024]: counts of their top digits,
  int4* found;                 // [batch, kv_heads]: the digit the search goes on in, how many of it stay, how many share it,
  uint2* list;                 // [batch, kv_heads, 4096]: those (key, slot), in any order,
  int* listed;                 // [batch, kv_heads]: how many
  unsigned long long* stays;   // [batch, kv_heads, words]: a bit a slot
  int2* ranks;                 // [batch, kv_heads, words]: holes and movers before those of a word (the j-th mover goes to the j-th hole)
  int4* counts;                // [batch, kv_heads]: pairs, new length, length, tokens so far (seqs.lengths may be lengths_out)
  int words, parts;
};

__device__ inline int slot_number(const EvictArgs& a, long long at, int i, int length, int total) {
  const int id = a.ids_in ? a.ids_in[at + i] : -1;
  return id < 0 ? total - length + i : id;
}

// The order of the slots: larger ones stay, equal ones by the lower number. Protected slots are above all weights and all alike, NaN
// below (float_key has numbers in 0x007fffff .. 0xff800000); both zeros are alike.
__device__ inline uint32_t weight_key(float w, int id, int total, const EvictArgs& a) {
  if (id < a.sink || (long long)id >= (long long)total - a.recent) return 0xffffffffu;
  return w != w ? 0u : float_key(w == 0.f ? 0.f : w);
}

// A value that is the same in all lanes, in scalar registers; whether this lane is in a mask, and how many below it are.
__device__ inline unsigned long long in_scalars(unsigned long long v) {
  return (unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(v >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)v);
}
__device__ inline bool lane_in(unsigned long long mask, int lane) {
#ifndef STTM_HOST_EMULATION
  return __builtin_amdgcn_inverse_ballot_w64(mask);
#else
  return mask >> lane & 1;
#endif
}
__device__ inline int lanes_below(unsigned long long mask, int lane) {
#ifndef STTM_HOST_EMULATION
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(mask >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)mask, 0u));
#else
  return __popcll(mask & ((1ull << lane) - 1));
#endif
}

constexpr int kDigitBits = 10, kDigits = 1 << kDigitBits;
// Keys that fit the list in LDS; slots of one workgroup that works out keys; rows up to here, as many as the registers of one
// workgroup hold, are gone through by it alone (whole calls in a graph, one slot going: four rows of 2,300 slots 12 us, as long rows
// 18; of 8,192 15 and 19; 128 of 8,192 24 and 31; 512 of them 55 and 61). (A host-thread build of the tests sets fewer: short rows take the way of long ones.)
#ifndef STTM_EVICT_LIST
#define STTM_EVICT_LIST 4096
#define STTM_EVICT_PART 4096
#define STTM_EVICT_HERE 8192
#endif
constexpr int kListMost = STTM_EVICT_LIST, kPartSlots = STTM_EVICT_PART, kSlotsHere = STTM_EVICT_HERE, kPartThreads = 256;

// GROUP keys of a lane, 64 slots apart from `from` on; all loads under way together.
template <int GROUP>
__device__ inline void keys_of(const EvictArgs& a, long long at, int from, int length, int total, uint32_t (&out)[GROUP]) {
  float w[GROUP];
  int id[GROUP];
#pragma unroll
  for (int k = 0; k < GROUP; ++k) {
    const int i = min(from + k * kWave, length - 1);
    w[k] = a.weights_in[at + i];
    id[k] = a.ids_in ? a.ids_in[at + i] : -1;
  }
#pragma unroll
  for (int k = 0; k < GROUP; ++k) {
    const int i = min(from + k * kWave, length - 1);
    out[k] = weight_key(w[k], id[k] < 0 ? total - length + i : id[k], total, a);
  }
}

// Counts a digit of every lane with `mine` set (all lanes call). Lanes that agree with the first one are counted in one
// step: many weights are alike where nothing was looked at.
__device__ inline void count_digit(unsigned* hist, bool mine, uint32_t digit, int lane) {
  const unsigned long long any = __ballot(mine);
  if (!any) return;
  const int leader = __ffsll((long long)any) - 1;
  const uint32_t of_leader = (uint32_t)lane_value((int)digit, leader);
  const unsigned long long same = __ballot(mine && digit == of_leader);
  if (lane == leader) atomicAdd(&hist[digit], (unsigned)__popcll(same));
  else if (mine && !(same >> lane & 1)) atomicAdd(&hist[digit], 1u);
}

// Long rows: keys and the counts of their first digit, a workgroup for every kPartSlots slots, so that a few long rows are
// gone through by many compute units (four rows of 43,328 slots: 6 us here and 9 in k_evict_mark, where one workgroup a row took
// 40 for as much; parts of 2,048 slots 5 and 10, and 8 and 16 against 9 and 11 on 192 ragged rows).
__global__ void __launch_bounds__(kPartThreads) k_evict_keys(EvictArgs a) {
  __shared__ unsigned hist[kDigits];
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, first = blockIdx.x * kPartSlots;
  const long long row = (long long)b * a.kv_heads + h, at = row * a.slot_stride;
  const int length = seq_length(a.seqs, b), total = a.total ? a.total[b] : length, stay = min(length, max(a.keep[b], 0));
  if (first >= length || stay == 0 || stay == length) return;
  if (blockIdx.x == 0 && tid == 0) a.listed[row] = 0;
  for (int i = tid; i < kDigits; i += kPartThreads) hist[i] = 0;
  __syncthreads();
  constexpr int GROUP = 8, RUN = kPartSlots / (kPartThreads / kWave);
  const int start = first + __builtin_amdgcn_readfirstlane(tid >> 6) * RUN, end = min(length, start + RUN);
  for (int s0 = start; s0 < end; s0 += GROUP * kWave) {
    uint32_t key[GROUP];
    keys_of<GROUP>(a, at, s0 + lane, length, total, key);
#pragma unroll
    for (int k = 0; k < GROUP; ++k) {
      const int i = s0 + k * kWave + lane;
      if (i < end) a.keys[row * a.seqs.max_len + i] = key[k];
      count_digit(hist, i < end, key[k] >> (32 - kDigitBits), lane);
    }
  }
  __syncthreads();
  unsigned short* counts = a.digits + (row * a.parts + blockIdx.x) * kDigits;
  for (int i = tid; i < kDigits; i += kPartThreads) counts[i] = (unsigned short)hist[i];
}

// Long rows, second pass: the digit at which the counts from the top reach the new length (every workgroup adds the parts up
// for itself), a bit for every slot above it, and the slots that share it, as many as fit the list, for the search.
__global__ void __launch_bounds__(kPartThreads) k_evict_mark(EvictArgs a) {
  __shared__ unsigned wave_a[kPartThreads / kWave];
  __shared__ int found[3];
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = blockIdx.x * kPartSlots;
  const long long row = (long long)b * a.kv_heads + h;
  const int length = seq_length(a.seqs, b), stay = min(length, max(a.keep[b], 0));
  if (first >= length) return;
  const bool search = stay > 0 && stay < length;
  int digit = 0, left = stay, count = length;
  if (search) {
    constexpr int PER = kDigits / kPartThreads;  // the digits of a thread, from the top
    unsigned n[PER] = {}, sum = 0;
    const unsigned short* counts = a.digits + row * a.parts * kDigits + kDigits - PER - tid * PER;
    const int parts = (length + kPartSlots - 1) / kPartSlots;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
      const uint2 x = *reinterpret_cast<const uint2*>(counts + (long long)p * kDigits);
      n[3] += x.x & 0xffffu; n[2] += x.x >> 16; n[1] += x.y & 0xffffu; n[0] += x.y >> 16;
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) sum += n[k];
    unsigned upto = wave_inclusive(sum, lane);
    if (lane == 63) wave_a[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += wave_a[w];
    unsigned before = upto - sum;
    if (before < (unsigned)stay && upto >= (unsigned)stay) {  // one thread's
      bool open = true;
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        if (open && before + n[k] >= (unsigned)stay) {
          found[0] = kDigits - 1 - tid * PER - k;
          found[1] = stay - (int)before;
          found[2] = (int)n[k];
          open = false;
        }
        before += n[k];
      }
    }
    __syncthreads();
    digit = found[0];
    left = found[1];
    count = found[2];
  }
  if (blockIdx.x == 0 && tid == 0) a.found[row] = make_int4(digit, left, count, 0);
  const bool exact = !search || left == count, listed = !exact && count <= kListMost;
  constexpr int RUN = kPartSlots / (kPartThreads / kWave), STEPS = RUN / kWave;
  const int start = first + wave * RUN, end = min(length, start + RUN);
  uint32_t key[STEPS];
#pragma unroll
  for (int k = 0; k < STEPS; ++k) key[k] = search ? a.keys[row * a.seqs.max_len + min(start + k * kWave + lane, length - 1)] : 0u;
  int near = 0;  // of this wavefront: one place in the list is taken for all of them
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int s = start + k * kWave, i = s + lane, d = (int)(key[k] >> (32 - kDigitBits));
    const unsigned long long mask = __ballot(i < end && (search ? d > digit || (exact && d == digit) : stay > 0));
    if (lane == 0 && s < end) a.stays[row * a.words + (s >> 6)] = mask;
    near += __popcll(__ballot(i < end && d == digit));
  }
  if (!listed || near == 0) return;
  int at = 0;
  if (lane == 0) at = atomicAdd(a.listed + row, near);
  at = lane_value(at, 0);
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int i = start + k * kWave + lane;
    const bool mine = i < end && (int)(key[k] >> (32 - kDigitBits)) == digit;
    const unsigned long long mask = __ballot(mine);
    const int place = at + lanes_below(mask, lane);
    if (mine && place < kListMost) a.list[row * kListMost + place] = make_uint2(key[k], (unsigned)i);
    at += __popcll(mask);
  }
}

// One workgroup a (sequence, kv head); a wavefront has a run of slots, their keys in registers (KEYS a lane; 0: a long row,
// whose keys k_evict_keys and k_evict_mark have worked out, counted and marked). The smallest key that stays is found by digits
// of ten bits, each counted in LDS, one thread a digit's count: the first digit is the top one (sign, exponent, a bit of the
// weight); the keys that share it (a few hundred to a few thousand of a long row) go on in a list in LDS, with ~number below
// the weight; every further digit starts at the highest bit in which those left differ, so that equal weights or small numbers
// cost no rounds of their own. It ends when the digits so far cut off exactly as many slots as stay, or 64 keys are left, which
// one wavefront ranks. What is left behind is a bit a slot, and how many holes and movers come before every 64.
//
// Bound by the chain of counts and barriers of one workgroup: 14 us for 128 rows of 4,097 slots, 11 for four of 43,328
// (keys and the first digit's counts ready).
template <int KEYS, int THREADS>  // (KEYS 0 or 8)
__global__ void __launch_bounds__(THREADS) k_evict_select(EvictArgs a) {
  constexpr bool READY = KEYS == 0;  // keys and the first digit's counts
  constexpr int AHEAD = 8, WAVES = THREADS / kWave, PER = kDigits / THREADS;  // digits' counts a thread
  constexpr int LIST = KEYS != 0 && KEYS * THREADS < kListMost ? KEYS * THREADS : kListMost;
  __shared__ unsigned hist[kDigits];
  __shared__ unsigned long long list[LIST], word_s[THREADS];
  __shared__ unsigned list_slot[READY ? kListMost : 1];
  __shared__ unsigned long long few[kWave], least_s;
  __shared__ unsigned wave_a[WAVES], wave_b[WAVES], bits[4];  // bits: and, or of the keys that are left
  __shared__ int digit_s, rest_s, count_s, listed_s;
  const int h = blockIdx.x, b = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long long row = (long long)b * a.kv_heads + h, at = row * a.slot_stride;
  const int length = seq_length(a.seqs, b), total = a.total ? a.total[b] : length;
  const int stay = min(length, max(a.keep[b], 0));
  const int its = (length + THREADS - 1) / THREADS, first = wave * its * kWave;  // its <= KEYS
  const int steps = min(its, max(0, (length - first + kWave - 1) / kWave));                  // of this wavefront
  const bool search = stay > 0 && stay < length;
  const uint32_t* stored = a.keys + row * a.seqs.max_len;
  uint32_t key[KEYS ? KEYS : 1];
  if constexpr (KEYS != 0) {
    if (search && steps > 0) keys_of<KEYS>(a, at, first + lane, length, total, key);
  }
  // f(slot of lane 0, this lane's slot, it is there, its key, its token's number if `numbers`): every step of this wavefront
  auto each = [&](bool numbers, auto f) {
    int s0 = first, i = first + lane;
    for (int k0 = 0; k0 < steps; k0 += AHEAD) {
      uint32_t x[AHEAD];
      int id[AHEAD];
#pragma unroll
      for (int k = 0; k < AHEAD; ++k) {
        const int at_slot = min(i + k * kWave, length - 1);
        if constexpr (KEYS != 0) x[k] = key[k];  // (one round)
        else x[k] = search ? stored[at_slot] : 0u;
        id[k] = numbers && a.ids_in ? a.ids_in[at + at_slot] : -1;
      }
#pragma unroll
      for (int k = 0; k < AHEAD; ++k, i += kWave, s0 += kWave)
        if (k0 + k < steps) f(s0, i, i < length, x[k], id[k] < 0 ? total - length + i : id[k]);
    }
  };
  auto whole_key = [](uint32_t k, int id) { return (unsigned long long)k << 32 | ~(uint32_t)id; };

  // `prefix`: the digits so far, those to come zero; `left` of the keys that agree with it above `shift` stay.
  unsigned long long prefix = 0;
  int shift = 64 - kDigitBits, left = stay;
  bool in_list = false, marked = false;  // marked: the bits of all slots but those in the list are there
  int listed = 0;
  if (search) {
    if (tid == 0) {
      listed_s = 0;
      least_s = 0;
    }
    if constexpr (READY) {
      const int4 found = a.found[row];
      prefix = (unsigned long long)found.x << shift;
      left = found.y;
      marked = left == found.z || found.z <= kListMost;
      if (left != found.z && marked) {
        listed = found.z;
        in_list = true;
        for (int i = tid; i < listed; i += THREADS) {
          const uint2 x = a.list[row * kListMost + i];
          list[i] = whole_key(x.x, slot_number(a, at, (int)x.y, length, total));
          list_slot[i] = x.y;
        }
      }
      if (tid == 0) count_s = found.z;
    } else {
      for (int i = tid; i < kDigits; i += THREADS) hist[i] = 0;
      __syncthreads();
      each(false, [&](int, int, bool there, uint32_t k, int) { count_digit(hist, there, k >> (32 - kDigitBits), lane); });
    }
    bool picked = READY;  // (the first digit)
    for (bool more = true; more;) {
      __syncthreads();
      if (!picked) {
        // the digit at which the counts from the top reach `left`
        unsigned n[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          n[i] = hist[kDigits - 1 - tid * PER - i];
          sum += n[i];
        }
        unsigned upto = wave_inclusive(sum, lane);
        if (lane == 63) wave_a[wave] = upto;
        __syncthreads();
        for (int w = 0; w < wave; ++w) upto += wave_a[w];
        unsigned before = upto - sum;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          if (before < (unsigned)left && before + n[i] >= (unsigned)left) {  // one thread's
            digit_s = kDigits - 1 - tid * PER - i;
            rest_s = left - (int)before;
            count_s = (int)n[i];
          }
          before += n[i];
        }
        __syncthreads();
        prefix |= (unsigned long long)digit_s << shift;
        left = rest_s;
      }
      picked = false;
      const int count = count_s;
      if (tid < 4) bits[tid] = tid < 2 ? 0xffffffffu : 0u;
      __syncthreads();
      if (left == count || shift == 0) break;
      if (in_list && count <= kWave) {
        // few are left: a wavefront has one a lane, and finds the one that as many as stay are no smaller than
        if (tid == 0) listed_s = 0;
        __syncthreads();
        for (int i = tid; i < listed; i += THREADS)
          if ((list[i] >> shift) == (prefix >> shift)) few[atomicAdd(&listed_s, 1) & (kWave - 1)] = list[i];
        __syncthreads();
        if (wave == 0) {
          const unsigned long long mine = lane < count ? few[lane] : 0;
          int above = 0, over = 0;
          for (int i = 0; i < count; ++i) {
            above += few[i] >= mine;
            over += few[i] > mine;
          }
          if (lane < count && over < left && above >= left) least_s = mine;  // (one lane's, but for numbers that occur twice)
        }
        __syncthreads();
        prefix = least_s;
        break;
      }
      // those that are left: into the list once they fit it; the bits in which they differ
      unsigned long long all = ~0ull, some = 0;
      const bool gather = !READY && !in_list && count <= LIST;
      if (in_list) {
        for (int i = tid; i < listed; i += THREADS) {
          const unsigned long long k = list[i];
          if ((k >> shift) == (prefix >> shift)) { all &= k; some |= k; }
        }
      } else {
        each(true, [&](int, int, bool there, uint32_t k, int id) {
          const unsigned long long x = whole_key(k, id);
          const bool near = there && (x >> shift) == (prefix >> shift);
          const unsigned long long mask = __ballot(near);
          if (mask == 0) return;
          if (near) {
            all &= x;
            some |= x;
          }
          if (gather) {
            int base = 0;
            if (lane == 0) base = atomicAdd(&listed_s, (int)__popcll(mask));
            base = lane_value(base, 0);
            if (near) list[base + lanes_below(mask, lane)] = x;
          }
        });
      }
      unsigned v[4] = {(unsigned)(all >> 32), (unsigned)all, (unsigned)(some >> 32), (unsigned)some};
#pragma unroll
      for (int o = 32; o > 0; o >>= 1)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const unsigned y = __shfl_xor(v[x], o, 64);
          v[x] = x < 2 ? v[x] & y : v[x] | y;
        }
      if (lane < 2) atomicAnd(&bits[lane], lane ? v[1] : v[0]);
      else if (lane < 4) atomicOr(&bits[lane], lane == 3 ? v[3] : v[2]);
      for (int i = tid; i < kDigits; i += THREADS) hist[i] = 0;
      __syncthreads();
      if (gather) {
        in_list = true;
        listed = count;
      }
      const unsigned long long differ = ((unsigned long long)bits[0] << 32 | bits[1]) ^ ((unsigned long long)bits[2] << 32 | bits[3]);
      const int above = shift;
      if (differ == 0) {  // (the same number twice: any of them)
        prefix |= ((unsigned long long)bits[0] << 32 | bits[1]) & ((1ull << above) - 1);
        break;
      }
      shift = max(0, 64 - (int)__clzll((long long)differ) - kDigitBits);
      // between the last digit and this one all agree
      prefix |= ((unsigned long long)bits[0] << 32 | bits[1]) & ((1ull << above) - 1) & ~((1ull << shift) - 1) & ~((unsigned long long)(kDigits - 1) << shift);
      // (the last digit of all may reach back into bits that are settled: both are compared)
      const unsigned long long agree = prefix >> shift >> kDigitBits, settled = prefix >> above;
      auto left_over = [&](unsigned long long k) { return (k >> shift >> kDigitBits) == agree && (k >> above) == settled; };
      if (in_list) {
        for (int i0 = 0; i0 < listed; i0 += THREADS) {
          const int i = i0 + tid;
          const unsigned long long k = i < listed ? list[i] : 0;
          count_digit(hist, i < listed && left_over(k), (uint32_t)(k >> shift) & (kDigits - 1), lane);
        }
      } else {
        each(true, [&](int, int, bool there, uint32_t k, int id) {
          const unsigned long long x = whole_key(k, id);
          count_digit(hist, there && left_over(x), (uint32_t)(x >> shift) & (kDigits - 1), lane);
        });
      }
    }
  }

  // a bit for every slot that stays
  if (!READY || !marked) {
    const uint32_t least = (uint32_t)(prefix >> 32), least_low = (uint32_t)prefix;
    if (!READY || search)
      each(search && least_low != 0, [&](int s0, int, bool there, uint32_t k, int id) {
        const unsigned long long mask = __ballot(there && (search ? k > least || (k == least && ~(uint32_t)id >= least_low) : stay > 0));
        if (lane == 0) a.stays[row * a.words + (s0 >> 6)] = mask;
      });
  }
  // How many holes and movers are before every word, a round of words at a time.
  const int words = (length + 63) / 64;
  auto up_to = [](int n) { return n >= 64 ? ~0ull : n <= 0 ? 0ull : (1ull << n) - 1; };
  bool to_mark = in_list && marked;
  int holes, movers;
  for (int pass = 0; pass < 2; ++pass) {
    holes = movers = 0;
    for (int w0 = 0; w0 < words; w0 += THREADS) {
      __syncthreads();
      const int word = w0 + tid, s0 = word * 64;
      if (word < words) word_s[tid] = a.stays[row * a.words + word];
      __syncthreads();
      if (to_mark) {
        unsigned* half = reinterpret_cast<unsigned*>(word_s);
        for (int i = tid; i < listed; i += THREADS) {
          const int at_word = (int)(list_slot[i] >> 6) - w0;
          if (list[i] >= prefix && at_word >= 0 && at_word < THREADS) atomicOr(&half[2 * at_word + (list_slot[i] >> 5 & 1)], 1u << (list_slot[i] & 31));
        }
        __syncthreads();
        if (word < words) a.stays[row * a.words + word] = word_s[tid];
      }
      unsigned long long hole = 0, mover = 0;
      if (word < words) {
        const unsigned long long mask = word_s[tid], front = up_to(stay - s0);
        hole = ~mask & up_to(length - s0) & front;
        mover = mask & ~front;
      }
      unsigned my_hole = (unsigned)__popcll(hole), my_mover = (unsigned)__popcll(mover);
      const unsigned own_hole = my_hole, own_mover = my_mover;
      my_hole = wave_inclusive(my_hole, lane);
      my_mover = wave_inclusive(my_mover, lane);
      if (lane == 63) {
        wave_a[wave] = my_hole;
        wave_b[wave] = my_mover;
      }
      __syncthreads();
      int round_holes = 0, round_movers = 0;
      for (int w = 0; w < WAVES; ++w) {
        if (w == wave && word < words)
          a.ranks[row * a.words + word] = make_int2(holes + round_holes + (int)(my_hole - own_hole), movers + round_movers + (int)(my_mover - own_mover));
        round_holes += (int)wave_a[w];
        round_movers += (int)wave_b[w];
      }
      holes += round_holes;
      movers += round_movers;
    }
    if (movers <= holes) break;
    // A number that occurs twice is the last one that stays, with all its slots: those that are too many go, the first ones.
    to_mark = false;
    if (tid == 0) listed_s = movers - holes;
    for (int w = 0; w < WAVES; ++w) {  // (one wavefront after the other: the same ones on every call)
      __syncthreads();
      if (w != wave) continue;
      int surplus = listed_s;
      each(true, [&](int s0, int, bool there, uint32_t k, int id) {
        const bool same = there && whole_key(k, id) == prefix;
        const int before = lanes_below(__ballot(same), lane);
        const unsigned long long gone = __ballot(same && before < surplus);
        if (lane == 0 && gone) a.stays[row * a.words + (s0 >> 6)] &= ~gone;
        surplus -= (int)__popcll(gone);
      });
      if (lane == 0) listed_s = surplus;
    }
  }
  if (tid == 0) a.counts[row] = make_int4(min(holes, movers), stay, length, total);
}

// The last word in [first, end) with no more than `rank` movers before it, by a wavefront: 64 places of what is left a step.
// (ranks[first].y is 0; the answer is the word that the mover of that rank is in.)
__device__ inline int word_of_mover(const int2* ranks, int first, int end, int rank, int lane) {
  while (end - first > 1) {
    const int step = (end - first + kWave - 1) / kWave, at = first + lane * step;
    const unsigned long long below = __ballot(at < end && ranks[min(at, end - 1)].y <= rank);
    first += (max(1, (int)__popcll(below)) - 1) * step;
    end = min(end, first + step);
  }
  return first;
}

// A workgroup has 128 slots before the new length: their entries in the tables, and the rows of the pool that go to the holes
// among them, LANES lanes a row, 16 bytes a lane; and 128 slots behind it to clear. Its holes have consecutive ranks, so the
// movers that fill them are consecutive too: both are listed in LDS from the marks.
// A mover's entries are read, written to its hole and cleared by one lane, nobody else touches either: outputs may be inputs.
// Bound by memory: 77 us for the ragged batch of 24 sequences and 8 heads (358 MB with the tables, 4.7 TB/s). 256 slots a workgroup
// took 82 (their last rows wait alone); lists made by the search 73, but 8 more there, and 10 more for one long row, which one
// workgroup searches. Tables and rows in workgroups of their own took 97, rows through the caches 102.
constexpr int kMoveThreads = 256, kMoveSlots = 128, kMoveRows = 4;  // (rows of a group of lanes under way together)
template <int LANES>
__global__ void __launch_bounds__(kMoveThreads) k_evict_move(EvictArgs a) {
  __shared__ int hole_s[kMoveSlots], mover_s[kMoveSlots], span_s[2];
  constexpr int WAVES = kMoveThreads / kWave, WORDS = kMoveSlots / kWave;  // (the first two wavefronts have a word each)
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, unit = tid & (LANES - 1);
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const long long row = (long long)b * a.kv_heads + h, at = row * a.slot_stride;
  const unsigned long long* stays = a.stays + row * a.words;
  const int2* ranks = a.ranks + row * a.words;
  // (under way with the counts: what is past the row's words is not used)
  const int slot0 = blockIdx.x * kMoveSlots, w0 = slot0 >> 6, word = min(w0 + wave, a.words - 1);
  const unsigned long long mask = stays[word];
  const int before = ranks[word].x, r0 = ranks[min(w0, a.words - 1)].x, next = ranks[min(w0 + WORDS, a.words - 1)].x;
  const int4 count = a.counts[row];
  const int stay = count.y, length = count.z, total = count.w, words = (length + 63) / 64;
  if (blockIdx.x == 0 && h == 0 && tid == 0) a.lengths_out[b] = stay;
  const int tail = stay + blockIdx.x * kMoveSlots + tid - kMoveSlots;
  if (tid >= kMoveSlots && tail < length && !(stays[tail >> 6] >> (tail & 63) & 1)) {  // (movers are cleared by who takes their entries)
    a.weights_out[at + tail] = 0.f;
    a.ids_out[at + tail] = -1;
    if (a.bias_out) a.bias_out[at + tail] = 0.f;
  }
  if (slot0 >= stay) return;
  const int r1 = min(count.x, w0 + WORDS < words ? next : count.x), n = r1 - r0;  // n <= 128
  // this lane's slot: it is before the new length, and it is a hole, the `place`-th of the workgroup's
  const int slot = slot0 + tid;
  const unsigned long long holes = ~mask & (stay - word * 64 >= 64 ? ~0ull : (1ull << max(0, stay - word * 64)) - 1);
  const bool front = wave < WORDS && slot < stay, hole = front && lane_in(in_scalars(holes), lane);
  const int place = before - r0 + lanes_below(holes, lane);
  if (n > 0) {
    if (hole && place < n) hole_s[place] = slot;
    if (wave >= WORDS) {
      const int w = word_of_mover(ranks, stay >> 6, words, wave == WORDS ? r0 : r1 - 1, lane);
      if (lane == 0) span_s[wave - WORDS] = w;
    }
    __syncthreads();
    const int last = span_s[1];
    for (int w = span_s[0] + wave; w <= last; w += WAVES) {
      const unsigned long long movers = in_scalars(stays[w] & (stay - w * 64 >= 64 ? 0ull : stay - w * 64 <= 0 ? ~0ull : ~((1ull << (stay - w * 64)) - 1)));
      const int j = ranks[w].y + lanes_below(movers, lane);
      if (lane_in(movers, lane) && j >= r0 && j < r1) mover_s[j - r0] = w * 64 + lane;
    }
    __syncthreads();
  }
  if (front) {
    const int from = !hole ? slot : place < n ? mover_s[place] : -1;  // the slot whose entries this one gets
    float w = 0.f, bias = 0.f;
    int id = -1;
    if (from >= 0) {
      w = a.weights_in[at + from];
      id = slot_number(a, at, from, length, total);
      if (a.bias_out) bias = a.bias_in[at + from];
    }
    a.weights_out[at + slot] = w;
    a.ids_out[at + slot] = id;
    if (a.bias_out) a.bias_out[at + slot] = bias;
    if (from > slot) {
      a.weights_out[at + from] = 0.f;
      a.ids_out[at + from] = -1;
      if (a.bias_out) a.bias_out[at + from] = 0.f;
    }
  }
  constexpr int GROUPS = kMoveThreads / LANES;
  const int page_mask = (1 << a.pool.shift) - 1;
  const int32_t* table = a.seqs.table + b * a.seqs.table_stride;
  for (int j0 = tid / LANES; j0 < n; j0 += GROUPS * kMoveRows) {
    int from[kMoveRows], to[kMoveRows], p[kMoveRows], q[kMoveRows];
    uint4 k[kMoveRows], v[kMoveRows];
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      const int j = min(j0 + r * GROUPS, n - 1);
      from[r] = mover_s[j];
      to[r] = hole_s[j];
      p[r] = table[from[r] >> a.pool.shift];
      q[r] = table[to[r] >> a.pool.shift];
    }
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      if (p[r] < 0 || p[r] >= a.pool.pages || q[r] < 0 || q[r] >= a.pool.pages || j0 + r * GROUPS >= n || unit * 16 >= a.pool.row) q[r] = -1;
      if (q[r] < 0) continue;
      const long long off = p[r] * a.pool.page_stride + h * a.pool.head_stride + (long long)(from[r] & page_mask) * a.pool.token_stride + unit * 16;
      k[r] = load_once(reinterpret_cast<const uint4*>(a.pool.k + off));
      v[r] = load_once(reinterpret_cast<const uint4*>(a.pool.v + off));
    }
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      if (q[r] < 0) continue;
      const long long off = q[r] * a.pool.page_stride + h * a.pool.head_stride + (long long)(to[r] & page_mask) * a.pool.token_stride + unit * 16;
      store_once(reinterpret_cast<uint4*>(a.pool.k + off), k[r]);
      store_once(reinterpret_cast<uint4*>(a.pool.v + off), v[r]);
    }
  }
}

struct Plan {
  int words, parts;
  size_t keys, digits, found, list, listed, ranks, stays, counts, bytes;
};
Plan make_plan(const sttm_cache* c, const sttm_sequences* s) {
  Plan p;
  size_t off = 0;
  auto take = [&](size_t bytes) { size_t o = off; off = (off + bytes + 255) / 256 * 256; return o; };
  const size_t rows = (size_t)s->batch * c->kv_heads, slots = (size_t)make_seqs(c, s).max_len;
  p.words = (int)std::max<size_t>(1, (slots + 63) / 64);
  p.parts = slots > (size_t)kSlotsHere ? (int)((slots + kPartSlots - 1) / kPartSlots) : 0;
  p.keys = take(p.parts ? rows * slots * sizeof(uint32_t) : 0);
  p.digits = take(rows * p.parts * kDigits * sizeof(unsigned short));
  p.found = take(p.parts ? rows * sizeof(int4) : 0);
  p.list = take(p.parts ? rows * kListMost * sizeof(uint2) : 0);
  p.listed = take(p.parts ? rows * sizeof(int) : 0);
  p.stays = take(rows * p.words * sizeof(unsigned long long));
  p.ranks = take(rows * p.words * sizeof(int2));
  p.counts = take(rows * sizeof(int4));
  p.bytes = std::max(off, (size_t)256);
  return p;
}

int check_evict(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs) {
  int rc = check_cache(ctx, cache);
  if (rc == STTM_OK) rc = check_sequences(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  if ((double)seqs->batch * cache->kv_heads * make_seqs(cache, seqs).max_len > 1e13) return ctx_fail(ctx, STTM_ERR_SHAPE, "batch * kv_heads * max_len too large");
  return STTM_OK;
}

}  // namespace
}  // namespace sttm

using namespace sttm;

extern "C" size_t sttm_cache_evict_workspace_bytes(const sttm_cache* cache, const sttm_sequences* seqs) {
  if (check_evict(nullptr, cache, seqs) != STTM_OK) return 0;
  return make_plan(cache, seqs).bytes;
}

extern "C" int sttm_cache_evict(sttm_ctx* ctx, const sttm_cache* cache, const sttm_sequences* seqs, const int32_t* keep,
                                const int32_t* total, int sink, int recent, int64_t slot_stride, const float* weights_in,
                                float* weights_out, const int32_t* ids_in, int32_t* ids_out, const float* bias_in,
                                float* bias_out, int32_t* lengths_out, void* workspace, size_t workspace_bytes) {
  if (!ctx) return STTM_ERR_NULL;
  int rc = check_evict(ctx, cache, seqs);
  if (rc != STTM_OK) return rc;
  EvictArgs a{};
  a.seqs = make_seqs(cache, seqs);
  if (slot_stride < a.seqs.max_len || slot_stride > ((int64_t)1 << 40)) return ctx_fail(ctx, STTM_ERR_SHAPE, "slot_stride must be no less than max_len");
  if (sink < 0 || recent < 0) return ctx_fail(ctx, STTM_ERR_ARG, "sink and recent must not be negative");
  if (!bias_in != !bias_out) return ctx_fail(ctx, STTM_ERR_ARG, "bias_in and bias_out: both or neither");
  if (seqs->batch == 0) return STTM_OK;
  if (!keep || !weights_in || !weights_out || !ids_out || !lengths_out)
    return ctx_fail(ctx, STTM_ERR_NULL, "keep, weights_in, weights_out, ids_out or lengths_out is NULL");
  const Plan p = make_plan(cache, seqs);
  rc = check_workspace(ctx, workspace, workspace_bytes, p.bytes);
  if (rc != STTM_OK) return rc;
  char* ws = static_cast<char*>(workspace);
  a.pool = make_pool(cache);
  a.keep = keep;
  a.total = total;
  a.slot_stride = slot_stride;
  a.weights_in = weights_in; a.weights_out = weights_out;
  a.ids_in = ids_in; a.ids_out = ids_out;
  a.bias_in = bias_in; a.bias_out = bias_out;
  a.lengths_out = lengths_out;
  a.kv_heads = cache->kv_heads;
  a.sink = sink;
  a.recent = recent;
  a.keys = reinterpret_cast<uint32_t*>(ws + p.keys);
  a.stays = reinterpret_cast<unsigned long long*>(ws + p.stays);
  a.ranks = reinterpret_cast<int2*>(ws + p.ranks);
  a.counts = reinterpret_cast<int4*>(ws + p.counts);
  a.digits = reinterpret_cast<unsigned short*>(ws + p.digits);
  a.found = reinterpret_cast<int4*>(ws + p.found);
  a.list = reinterpret_cast<uint2*>(ws + p.list);
  a.listed = reinterpret_cast<int*>(ws + p.listed);
  a.parts = p.parts;
  a.words = p.words;
  rc = ctx_device(ctx);
  if (rc != STTM_OK) return rc;
  const hipStream_t s = ctx_stream(ctx);
  const dim3 rows(a.kv_heads, seqs->batch);
  if (p.parts) {
    hipLaunchKernelGGL(k_evict_keys, dim3(p.parts, a.kv_heads, seqs->batch), dim3(kPartThreads), 0, s, a);
    hipLaunchKernelGGL(k_evict_mark, dim3(p.parts, a.kv_heads, seqs->batch), dim3(kPartThreads), 0, s, a);
    hipLaunchKernelGGL((k_evict_select<0, 1024>), rows, dim3(1024), 0, s, a);
  } else if (a.seqs.max_len <= 2048) {  // (as many slots as their registers hold. Fewer wavefronts to wait for: whole calls in a graph,
                                        // 48 rows of 500 slots 10.8 us, by 1,024 threads 12.1; of 1,013 11.1 and 13.2; of 2,048
                                        // 12.1 and 13.8; 512 rows of 2,048 22 and 31)
    hipLaunchKernelGGL((k_evict_select<8, 256>), rows, dim3(256), 0, s, a);
  } else {                              // (128 rows of 4,097 slots 14 us; 512 threads with twice the keys each took 2 more, 256 7 more)
    hipLaunchKernelGGL((k_evict_select<8, 1024>), rows, dim3(1024), 0, s, a);
  }
  const int lanes = a.pool.row <= 128 ? 8 : a.pool.row <= 256 ? 16 : a.pool.row <= 512 ? 32 : 64;
  const dim3 grid(std::max(1, (a.seqs.max_len + kMoveSlots - 1) / kMoveSlots), a.kv_heads, seqs->batch), block(kMoveThreads);
  if (lanes == 8) hipLaunchKernelGGL((k_evict_move<8>), grid, block, 0, s, a);
  else if (lanes == 16) hipLaunchKernelGGL((k_evict_move<16>), grid, block, 0, s, a);
  else if (lanes == 32) hipLaunchKernelGGL((k_evict_move<32>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((k_evict_move<64>), grid, block, 0, s, a);
  return ctx_after_launch(ctx);
}
