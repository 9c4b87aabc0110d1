// The gated linear recurrence on gfx950: the LSTM cell whose gates depend on the
// input alone,
//
//   c_t = sigmoid(f_t) c_{t-1} + sigmoid(i_t) tanh(g_t),   h_t = sigmoid(o_t) tanh(c_t),
//
// and its gradients.  Every (sequence, unit) is a recurrence of its own, linear in
// its state: a stretch of time maps c to A c + B with A = prod f and B the state
// it leaves from 0, and two stretches compose as (A2 A1, A2 B1 + B2).  So time is
// split twice: a wave takes 8 timesteps of 128 units in registers, a workgroup
// eight such waves (a chunk of 64), whose maps meet in LDS.  Each wave then runs
// its 8 steps from its own first state, so p is read once and nothing but maps is
// exchanged.  Every composition has a fixed order: same bits whatever runs beside.
//
// What bounds it is memory and the vector units together (64 instructions an element
// forward, ten of them transcendental and fourteen for tanh near 0; in bf16 busy 72% of the
// time).  MI355X, where a large copy moves 5.2 TB/s: bf16, T = 4096, H = 8192, 335 MB in 90
// us (3.7 TB/s); T = 65536, H = 512, the same bytes in 101 us, 11 of them for the longer
// chain of states; 256 sequences of 512, H = 512, 156 us (4.3 TB/s).  Forward and back,
// 8 x 2048, H = 1024: 135 us, 50 forward and 86 back by themselves, of which 5 each clear the
// words that chunks hand over with and 7 sum the bias gradient (the backward kernel 310 MB
// in 73, 4.2 TB/s).
//
// Tried and dropped: a flag for each map instead of maps that carry their own sign
// (less to clear, but the wait for the stores' acknowledgement costs 15 us at every
// size); maps cleared by nontemporal stores (+2 us); registers cut to 64 by spilling
// (+14 us at T = 4096, H = 8192).
#include <algorithm>
#include <type_traits>

#include "device_common.hpp"
#include "gated.hpp"

// every fused multiply-add is written out: same bits from every instance
#pragma clang fp contract(off)

namespace alstm {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kSteps = kLinearSave;            // timesteps of a wave
constexpr int kScanWaves = 8;
constexpr int kScanThreads = 64 * kScanWaves;
constexpr int kChunk = kSteps * kScanWaves;    // timesteps of a workgroup at once
constexpr int kGroup = kScanWaves * kScanWaves;   // chunks between two handed-on states
constexpr int kTicketStride = 16;              // words between two columns' tickets (64 bytes)
constexpr int kWalkThreads = 256;
constexpr size_t kMostChunks = 1u << 22;       // of all columns, where chunks hand over
constexpr float kLog2e = 1.4426950408889634f;

// Two neighbouring units of a row, loaded and stored at once at any alignment of
// their elements.  With an odd number of units the last lane of a row has one
// (`two` false): it loads the unit before as well and swaps, so nothing past the row
// is touched, and stores it alone.  Rows of a single unit go one by one.
enum Rows { kEven, kOdd, kSingle };

template <class T>
struct Pair;
template <>
struct Pair<float> {
  typedef f32x2 Raw;
  typedef f32x2 Any __attribute__((aligned(4)));
  static __device__ __forceinline__ f32x2 get(Raw r) { return r; }
  static __device__ __forceinline__ Raw put(f32x2 v) { return v; }
  static __device__ __forceinline__ Raw one(float v) { return Raw{v, v}; }
  static __device__ __forceinline__ Raw swap(Raw r) { return Raw{r[1], r[0]}; }
  static __device__ __forceinline__ float low(Raw r) { return r[0]; }
};
template <>
struct Pair<__bf16> {
  typedef unsigned Raw;
  typedef unsigned Any __attribute__((aligned(2)));
  static __device__ __forceinline__ f32x2 get(Raw r) {
    return f32x2{__uint_as_float(r << 16), __uint_as_float(r & 0xFFFF0000u)};
  }
  static __device__ __forceinline__ Raw put(f32x2 v) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));   // to the nearest, ties to even
  }
  static __device__ __forceinline__ Raw one(__bf16 v) { return __builtin_bit_cast(uint16_t, v); }
  static __device__ __forceinline__ Raw swap(Raw r) { return r >> 16; }
  static __device__ __forceinline__ __bf16 low(Raw r) { return __builtin_bit_cast(__bf16, (uint16_t)r); }
};

template <class T, Rows R>
__device__ __forceinline__ typename Pair<T>::Raw load_pair(const char* row, unsigned off, bool two) {
  if constexpr (R == kSingle) {
    return Pair<T>::one(*reinterpret_cast<const T*>(row + off));
  } else if constexpr (R == kOdd) {
    const typename Pair<T>::Raw r =
        *reinterpret_cast<const typename Pair<T>::Any*>(row + (off - (two ? 0u : (unsigned)sizeof(T))));
    return two ? r : Pair<T>::swap(r);
  } else {
    return *reinterpret_cast<const typename Pair<T>::Any*>(row + off);
  }
}

template <class T, Rows R>
__device__ __forceinline__ void store_pair(char* row, unsigned off, f32x2 v, bool two) {
  const auto r = Pair<T>::put(v);
  if (R == kEven || (R == kOdd && two)) *reinterpret_cast<typename Pair<T>::Any*>(row + off) = r;
  else *reinterpret_cast<T*>(row + off) = Pair<T>::low(r);
}

template <Rows R>
__device__ __forceinline__ f32x2 load_state(const float* p, unsigned at, bool two) {
  return load_pair<float, R>(reinterpret_cast<const char*>(p), at * 4u, two);
}
template <Rows R>
__device__ __forceinline__ void store_state(float* p, unsigned at, f32x2 v, bool two) {
  store_pair<float, R>(reinterpret_cast<char*>(p), at * 4u, v, two);
}

// What a lane works on: units r, r + 1 of sequence b.
struct Lane {
  int b, r, len;          // len: timesteps of the sequence
  bool live, two;         // live: there is such a sequence
  unsigned at;            // its place in a row of states [B][H] (elements)
};

__device__ __forceinline__ Lane lane_of(const LinearArgs& a, int idx) {
  Lane l;
  const int pairs = (a.H + 1) / 2;
  l.live = idx < a.B * pairs;
  if (!l.live) idx = 0;
  l.b = idx / pairs;
  l.r = 2 * (idx - l.b * pairs);
  l.two = l.r + 1 < a.H;
  l.at = (unsigned)l.b * (unsigned)a.H + (unsigned)l.r;
  l.len = a.lengths ? min(max(a.lengths[l.b], 0), a.T) : a.T;
  return l;
}

// Gates of y = p + bias, rounded once: a bias inside the exponential's argument (one
// operation less) would be rounded apart from p, and what is left where the two
// cancel would be off by as much as they are.  sigmoid(y) = 1 / (1 + 2^(-y log2 e)) and
// tanh (below) reach their ends exactly (2^x is 0 or infinity there).
struct GateBias {
  f32x2 i, f, g, o;
};

__device__ __forceinline__ GateBias gate_bias(const LinearArgs& a, const Lane& l) {
  GateBias b{};
  if (a.bias) {
    auto at = [&](int q) {
      const float* p = a.bias + (size_t)q * a.H + l.r;
      float lo = p[0], hi = p[l.two ? 1 : 0];
      // (arrived before anything else is under way: waits at their uses would be for the
      // stores of h as well, T = 100, H = 64, fp32 10.2 us instead of 9.0)
      asm("" : "+v"(lo), "+v"(hi));
      return f32x2{lo, hi};
    };
    b.i = at(0), b.f = at(1), b.g = at(2), b.o = at(3);
  }
  return b;
}

__device__ __forceinline__ float gate_sig(float y) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * -kLog2e));
}
// The forget gate: over a memory of 1 / (1 - f) steps an error of the same sign in
// each adds up, and the reciprocal's is (0.1 of half a step on average at f near 1;
// 0.006 after one Newton step).  fminf keeps 0 x infinity out where the gate is shut.
__device__ __forceinline__ float gate_forget(float y) {
  const float d = 1.0f + __builtin_amdgcn_exp2f(y * -kLog2e), r = __builtin_amdgcn_rcpf(d);
  return __builtin_fmaf(fminf(__builtin_fmaf(-r, d, 1.0f), 1e-6f), r, r);
}
// tanh: 1 - 2 / (1 + e^2y) is off by 2^-23 whatever y is, which near 0 is more than all of
// tanh(y) is worth.  Below 0.4 it is y (1 + y^2 P(y^2)) instead, P of least relative error
// there (1.9 halves of a step); either side is within 8 halves of a step of itself.
__device__ __forceinline__ float gate_tanh(float y) {
  const float r = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(y * (2.0f * kLog2e))), s = y * y;
  const float p = __builtin_fmaf(s, __builtin_fmaf(s, -0.047794174f, 0.13277628f), -0.33331883f);
  float near = __builtin_fmaf(y * s, p, y), far = __builtin_fmaf(-2.0f, r, 1.0f);
  asm("" : "+v"(near), "+v"(far));   // (both; with a branch T = 65536, H = 512, bf16 took 107 us, so 102)
  return fabsf(y) < 0.4f ? near : far;
}

// Few timesteps (walked): a lane walks its two units through all of them, the loads of
// kAhead timesteps at once (one token of 32 sequences, H = 1024: 3.3 us; 256 sequences of
// 16, H = 512: 9.1 us, 21 MB).
template <class T, Rows R>
__global__ void __launch_bounds__(kWalkThreads) linear_walk_kernel(LinearArgs a) {
  constexpr int kAhead = 4;
  const Lane l = lane_of(a, blockIdx.x * kWalkThreads + threadIdx.x);
  if (!l.live) return;
  const GateBias bias = gate_bias(a, l);
  const size_t BH = (size_t)a.B * a.H;
  const unsigned ga = (4u * l.b * a.H + l.r) * sizeof(T), gs = (unsigned)a.H * sizeof(T);
  f32x2 c = a.c0 ? load_state<R>(a.c0, l.at, l.two) : f32x2{0.f, 0.f};
  for (int t0 = 0; t0 < a.T; t0 += kAhead) {
    typename Pair<T>::Raw raw[kAhead][4];
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const char* row = (const char*)a.p + (size_t)min(t0 + s, a.T - 1) * (4 * BH * sizeof(T));
#pragma unroll
      for (int q = 0; q < 4; ++q) raw[s][q] = load_pair<T, R>(row, ga + q * gs, l.two);
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int t = t0 + s;
      if (t >= a.T) break;
      if (s % kSteps == 0 && t % kSteps == 0 && a.c_save)
        store_state<R>(a.c_save + (size_t)(t / kSteps) * BH, l.at, c, l.two);
      const f32x2 yi = Pair<T>::get(raw[s][0]), yf = Pair<T>::get(raw[s][1]), yg = Pair<T>::get(raw[s][2]),
                  yo = Pair<T>::get(raw[s][3]);
      f32x2 h{0.f, 0.f};
      if (t < l.len) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          c[k] = __builtin_fmaf(gate_forget(yf[k] + bias.f[k]), c[k], gate_sig(yi[k] + bias.i[k]) * gate_tanh(yg[k] + bias.g[k]));
          h[k] = gate_sig(yo[k] + bias.o[k]) * gate_tanh(c[k]);
        }
      }
      store_pair<T, R>((char*)a.h + (size_t)t * (BH * sizeof(T)), l.at * sizeof(T), h, l.two);
    }
  }
  if (a.c_out) store_state<R>(a.c_out, l.at, c, l.two);
}

// A map c -> A c + B of two units, {A0, B0, A1, B1}.
__device__ __forceinline__ f32x4 then(const f32x4& first, const f32x4& second) {
  return f32x4{second[0] * first[0], __builtin_fmaf(second[0], first[1], second[1]), second[2] * first[2],
               __builtin_fmaf(second[2], first[3], second[3])};
}
__device__ __forceinline__ f32x2 apply(const f32x4& m, const f32x2& c) {
  return f32x2{__builtin_fmaf(m[0], c[0], m[1]), __builtin_fmaf(m[2], c[1], m[3])};
}
constexpr f32x4 kIdentity{1.f, 0.f, 1.f, 0.f};

// Hand-over between chunks of a column, when there are too few columns to fill the
// device and so its chunks run side by side.  A word is empty (all ones, as the
// kernel before cleared it) until its value is there; a value with the bits of an
// empty word is written as another NaN.  A chunk publishes its map as soon as it
// has it; the last of kScanWaves chunks, a block, publishes the block's instead.
// Each wave collects one map of an earlier chunk of the block and one of an earlier
// block of the group (kScanWaves blocks, 4096 timesteps), and one waits for the
// state that the group before handed on: a hop of the serial chain passes a whole
// group, and a chunk reads 7 maps on average.  (One level of 32 chunks, 16 maps on
// average, took 121 us instead of 113 at T = 65536, H = 512, bf16; then one lane that
// looks for a wave instead of all 64 brought it to 96; tanh near 0 then cost 5.)
//
// Which chunk a workgroup takes is the ticket of its column: in the order in which
// workgroups start, so the chunks that anyone waits for have workgroups that run.
__device__ __forceinline__ unsigned filled(float v) {
  const unsigned w = __float_as_uint(v);
  return w == kEmpty ? 0x7FC00000u : w;
}

__device__ __forceinline__ void publish_map(unsigned long long* w, const f32x4& m) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    __hip_atomic_store(w + k, ((unsigned long long)filled(m[2 * k]) << 32) | __float_as_uint(m[2 * k + 1]), __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}

__device__ __forceinline__ void publish_state(unsigned* w, const f32x2& c) {
#pragma unroll
  for (int k = 0; k < 2; ++k)
    __hip_atomic_store(w + k, filled(c[k]), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Lane 0 (of a wave with work, its lane too) looks until its word is there, so that a
// wave that waits asks for one line and not for sixteen.
__device__ __forceinline__ unsigned await_first(const unsigned* w) {
  unsigned spins = 0;
  if ((threadIdx.x & 63) == 0)
    while (__hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == kEmpty && ++spins < kSpinLimit)
      __builtin_amdgcn_s_sleep(8);
  return __builtin_amdgcn_readfirstlane(spins);
}

// the state of a word pair; NaN past the spin limit
__device__ __forceinline__ f32x2 await_state(const unsigned* w) {
  unsigned v[2], spins = await_first(w);
  while (true) {
    v[0] = __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v[1] = __hip_atomic_load(w + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if ((v[0] != kEmpty && v[1] != kEmpty) || ++spins >= kSpinLimit) break;
    __builtin_amdgcn_s_sleep(1);
  }
  return f32x2{__uint_as_float(v[0]), __uint_as_float(v[1])};   // (an empty word is a NaN)
}

// a published map; NaN past the spin limit
__device__ __forceinline__ f32x4 await_map(const unsigned long long* w) {
  unsigned long long v[2];
  unsigned spins = await_first(reinterpret_cast<const unsigned*>(w) + 1);
  while (true) {
    v[0] = __hip_atomic_load(w, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    v[1] = __hip_atomic_load(w + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (((unsigned)(v[0] >> 32) != kEmpty && (unsigned)(v[1] >> 32) != kEmpty) || ++spins >= kSpinLimit) break;
    __builtin_amdgcn_s_sleep(1);
  }
  return f32x4{__uint_as_float((unsigned)(v[0] >> 32)), __uint_as_float((unsigned)v[0]),
               __uint_as_float((unsigned)(v[1] >> 32)), __uint_as_float((unsigned)v[1])};
}

template <int W>
struct ScanLds {
  f32x4 wave[2][W][64];            // maps of the waves (of even and odd rounds)
  f32x4 chunks[W][64];             // maps of the chunks before in the block
  f32x4 blocks[W][64];             // maps of the blocks before in the group
  f32x4 total[64];                 // map of the chunk
  f32x2 entry[64];                 // the state that the chunk begins with
  int ticket;
};

// The state that this chunk (the `order`-th of its column) begins with, where
// chunks hand over; `wave_order` is the wave's place in time.  The waves' maps are
// in lds.wave[0], by place.  `first` is where the column's first state stands: it is
// read by the first chunk alone, which hands it on too, since the last chunk's
// state may be written to the same place.
template <class Load>
__device__ __forceinline__ f32x2 hand_over(ScanLds<kScanWaves>& lds, const LinearScan& s, int order, int wave_order, int lane,
                                           size_t idx, bool live, Load first) {
  const int block = order / kScanWaves, i = order % kScanWaves, group = block / kScanWaves, j = block % kScanWaves;
  const bool last = order + 1 >= s.chunks;
  const size_t stride = 2 * (size_t)s.lanes;
  if (wave_order == kScanWaves - 1) {
    f32x4 m = lds.wave[0][0][lane];
#pragma unroll 1
    for (int w = 1; w < kScanWaves; ++w) m = then(m, lds.wave[0][w][lane]);
    lds.total[lane] = m;
    if (live && !last && i != kScanWaves - 1) publish_map(s.maps + order * stride + 2 * idx, m);
  }
  if (wave_order < i && live)
    lds.chunks[wave_order][lane] = await_map(s.maps + (size_t)(order - i + wave_order) * stride + 2 * idx);
  lds_barrier();
  if (wave_order == kScanWaves - 1 && i == kScanWaves - 1 && j != kScanWaves - 1 && !last) {
    f32x4 m = lds.chunks[0][lane];
#pragma unroll 1
    for (int w = 1; w < i; ++w) m = then(m, lds.chunks[w][lane]);
    if (live) publish_map(s.maps + (s.chunks + block) * stride + 2 * idx, then(m, lds.total[lane]));
  }
  if (wave_order < j && live)
    lds.blocks[wave_order][lane] = await_map(s.maps + (size_t)(s.chunks + block - j + wave_order) * stride + 2 * idx);
  lds_barrier();
  if (wave_order == 0) {
    f32x4 m = kIdentity;   // from the group's first state to this chunk's
#pragma unroll 1
    for (int w = 0; w < j; ++w) m = then(m, lds.blocks[w][lane]);
#pragma unroll 1
    for (int w = 0; w < i; ++w) m = then(m, lds.chunks[w][lane]);
    const bool hands_on = i == kScanWaves - 1 && j == kScanWaves - 1 && !last;
    f32x4 through = m;
    if (hands_on) through = then(m, lds.total[lane]);
    f32x2 c{0.f, 0.f};
    if (order == 0) {
      c = first();
      if (live && !last) publish_state(s.states + 2 * idx, c);
    } else if (live) {
      c = await_state(s.states + group * stride + 2 * idx);
    }
    if (hands_on && live) publish_state(s.states + (group + 1) * stride + 2 * idx, apply(through, c));
    lds.entry[lane] = apply(m, c);
  }
  lds_barrier();
  return lds.entry[lane];
}

// LOOK: a workgroup takes one chunk and chunks hand over; else it takes its
// column's chunks one after another and keeps the state.
template <class T, Rows R, bool LOOK>
__global__ void __launch_bounds__(kScanThreads, LOOK && !(R == kOdd && sizeof(T) == 4) ? 6 : 4) linear_scan_kernel(LinearArgs a, LinearScan s) {
  __shared__ ScanLds<kScanWaves> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int col = blockIdx.x, chunk = 0;
  if constexpr (LOOK) {
    col = blockIdx.x % s.cols;
    if (threadIdx.x == 0)
      lds.ticket = (int)__hip_atomic_fetch_add(s.tickets + (size_t)col * kTicketStride, 1u, __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    lds_barrier();
    chunk = __builtin_amdgcn_readfirstlane(lds.ticket);
  }
  const int idx = col * 64 + lane;
  const Lane l = lane_of(a, idx);
  const GateBias bias = gate_bias(a, l);
  const size_t BH = (size_t)a.B * a.H;
  const unsigned ga = (4u * l.b * a.H + l.r) * sizeof(T), gs = (unsigned)a.H * sizeof(T), ha = l.at * sizeof(T);
  auto first = [&] { return a.c0 ? load_state<R>(a.c0, l.at, l.two) : f32x2{0.f, 0.f}; };
  if (!LOOK && wave == 0) lds.entry[lane] = first();   // (one wave reads it: c_out may be c0)
  f32x2 carry{0.f, 0.f};
  for (; chunk < s.chunks; ++chunk) {
    const int t0 = chunk * kChunk + wave * kSteps;
    const int n = min(l.len - t0, kSteps);   // timesteps here that the sequence has
    const bool some = __any(n > 0);          // (a wave of padding alone loads nothing)
    typename Pair<T>::Raw raw[kSteps][4];
    f32x2 f[kSteps], u[kSteps];
    if (some) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const char* row = (const char*)a.p + (size_t)min(t0 + k, a.T - 1) * (4 * BH * sizeof(T));
#pragma unroll
        for (int q = 0; q < 4; ++q) raw[k][q] = load_pair<T, R>(row, ga + q * gs, l.two);
      }
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        const f32x2 yi = Pair<T>::get(raw[k][0]), yf = Pair<T>::get(raw[k][1]), yg = Pair<T>::get(raw[k][2]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f[k][j] = gate_forget(yf[j] + bias.f[j]);
          u[k][j] = gate_sig(yi[j] + bias.i[j]) * gate_tanh(yg[j] + bias.g[j]);
        }
      }
    }
    if (!some || a.lengths || t0 + kSteps > a.T) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
        if (k >= n) f[k] = f32x2{1.f, 1.f}, u[k] = f32x2{0.f, 0.f};
    }
    f32x4 m{f[0][0], u[0][0], f[0][1], u[0][1]};
#pragma unroll
    for (int k = 1; k < kSteps; ++k) m = then(m, f32x4{f[k][0], u[k][0], f[k][1], u[k][1]});
    const int half = LOOK ? 0 : chunk & 1;
    lds.wave[half][wave][lane] = m;
    lds_barrier();
    f32x2 c = !LOOK && chunk == 0 ? lds.entry[lane] : carry;
    if constexpr (LOOK) c = hand_over(lds, s, chunk, wave, lane, idx, l.live, first);
#pragma unroll 2
    for (int w = 0; w < kScanWaves; ++w) {
      if (w == wave) carry = c;
      if (LOOK && w == wave) break;
      c = apply(lds.wave[half][w][lane], c);
    }
    f32x2 next = c;
    c = carry;          // the wave's first state
    carry = next;       // the chunk's last one
    if (l.live) {
      if (a.c_save && t0 < a.T) store_state<R>(a.c_save + (size_t)(t0 / kSteps) * BH, l.at, c, l.two);
#pragma unroll
      for (int k = 0; k < kSteps; ++k) {
        f32x2 h;
        const f32x2 yo = Pair<T>::get(raw[k][3]);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          c[j] = __builtin_fmaf(f[k][j], c[j], u[k][j]);
          h[j] = gate_sig(yo[j] + bias.o[j]) * gate_tanh(c[j]);
          if (k >= n) h[j] = 0.f;
        }
        if (t0 + k < a.T) store_pair<T, R>((char*)a.h + (size_t)(t0 + k) * (BH * sizeof(T)), ha, h, l.two);
      }
      if (a.c_out && chunk == s.chunks - 1 && wave == kScanWaves - 1) store_state<R>(a.c_out, l.at, c, l.two);
    }
    if constexpr (LOOK) break;
  }
}

// The backward pass, the same from the end: with e the gradient that c_t gets from
// later timesteps and w_t = dh_t o_t (1 - tanh(c_t)^2),
//
//   d_t = w_t + e_t,  e_{t-1} = f_t d_t,  dp = d g i (1-i), d c_{t-1} f (1-f), d i (1-g^2), dh tanh(c) o (1-o).
//
// A wave runs its 8 steps forward from the saved state, so c is neither stored nor
// read but every 8 timesteps, and keeps f, w and the three factors of d; its map is
// e -> A e + B again.  The sums of dp over its timesteps leave through dpart.
// LOOK: a workgroup takes one of its column's chunks; else there is one.  W waves: 8,
// or 2 for up to 16 timesteps.
template <class T, Rows R, bool LOOK, int W>
__global__ void __launch_bounds__(64 * W, 4) linear_back_kernel(LinearArgs a, LinearScan s) {
  static_assert(!LOOK || W == kScanWaves, "chunks that hand over have eight waves");
  __shared__ ScanLds<W> lds;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int col = blockIdx.x, order = 0;
  if constexpr (LOOK) {
    col = blockIdx.x % s.cols;
    if (threadIdx.x == 0)
      lds.ticket = (int)__hip_atomic_fetch_add(s.tickets + (size_t)col * kTicketStride, 1u, __ATOMIC_RELAXED,
                                               __HIP_MEMORY_SCOPE_AGENT);
    lds_barrier();
    order = __builtin_amdgcn_readfirstlane(lds.ticket);
  }
  const int idx = col * 64 + lane;
  const Lane l = lane_of(a, idx);
  const GateBias bias = gate_bias(a, l);
  const size_t BH = (size_t)a.B * a.H;
  const unsigned ga = (4u * l.b * a.H + l.r) * sizeof(T), gs = (unsigned)a.H * sizeof(T), ha = l.at * sizeof(T);
  const int place = W - 1 - wave;   // the wave's place in the order of the pass
  auto first = [&] { return a.dc_out ? load_state<R>(a.dc_out, l.at, l.two) : f32x2{0.f, 0.f}; };
  if (!LOOK && place == 0) lds.entry[lane] = first();   // (one wave reads it: dc0 may be dc_out)
  f32x2 si{0.f, 0.f}, sf = si, sg = si, so = si;
  const int chunk = s.chunks - 1 - order, t0 = chunk * (kSteps * W) + wave * kSteps;
  const int n = min(l.len - t0, kSteps);
  const bool some = __any(n > 0);
  typename Pair<T>::Raw raw[kSteps][4] = {}, rdh[kSteps] = {};
  if (some)
#pragma unroll
    for (int k = 0; k < kSteps; ++k) {
      const size_t t = (size_t)min(t0 + k, a.T - 1);
      const char* row = (const char*)a.p + t * (4 * BH * sizeof(T));
#pragma unroll
      for (int q = 0; q < 4; ++q) raw[k][q] = load_pair<T, R>(row, ga + q * gs, l.two);
      rdh[k] = load_pair<T, R>((const char*)a.dh + t * (BH * sizeof(T)), ha, l.two);
    }
  f32x2 c = load_state<R>(a.c_save + (size_t)(min(t0, a.T - 1) / kSteps) * BH, l.at, l.two);
  f32x2 f[kSteps], w[kSteps], ki[kSteps], kf[kSteps], kg[kSteps];
#pragma unroll
  for (int k = 0; k < kSteps; ++k) {
    const f32x2 yi = Pair<T>::get(raw[k][0]), yf = Pair<T>::get(raw[k][1]), yg = Pair<T>::get(raw[k][2]),
                yo = Pair<T>::get(raw[k][3]), dh = Pair<T>::get(rdh[k]);
    f32x2 dO;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float vf = gate_forget(yf[j] + bias.f[j]), vi = gate_sig(yi[j] + bias.i[j]), vg = gate_tanh(yg[j] + bias.g[j]),
                  vo = gate_sig(yo[j] + bias.o[j]);
      kf[k][j] = c[j] * __builtin_fmaf(-vf, vf, vf);
      ki[k][j] = vg * __builtin_fmaf(-vi, vi, vi);
      kg[k][j] = vi * __builtin_fmaf(-vg, vg, 1.f);
      const float cn = __builtin_fmaf(vf, c[j], vi * vg), tc = gate_tanh(cn), dho = dh[j] * vo;
      f[k][j] = vf;
      w[k][j] = dho * __builtin_fmaf(-tc, tc, 1.f);
      dO[j] = dho * tc * (1.f - vo);
      if (k >= n) f[k][j] = 1.f, w[k][j] = kf[k][j] = ki[k][j] = kg[k][j] = dO[j] = 0.f;
      else c[j] = cn;
      so[j] += dO[j];
    }
    if (l.live && t0 + k < a.T)
      store_pair<T, R>((char*)a.dp + (size_t)(t0 + k) * (4 * BH * sizeof(T)), ga + 3 * gs, dO, l.two);
  }
  f32x4 m = kIdentity;
#pragma unroll
  for (int k = kSteps - 1; k >= 0; --k)
    m = then(m, f32x4{f[k][0], f[k][0] * w[k][0], f[k][1], f[k][1] * w[k][1]});
  lds.wave[0][place][lane] = m;
  lds_barrier();
  f32x2 e;
  if constexpr (LOOK) e = hand_over(lds, s, order, place, lane, idx, l.live, first);
  else e = lds.entry[lane];
#pragma unroll 1
  for (int v = 0; v < place; ++v) e = apply(lds.wave[0][v][lane], e);
#pragma unroll
  for (int k = kSteps - 1; k >= 0; --k) {
    f32x2 di, df, dg;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const float d = w[k][j] + e[j];
      di[j] = d * ki[k][j], df[j] = d * kf[k][j], dg[j] = d * kg[k][j];
      e[j] = f[k][j] * d;
      si[j] += di[j], sf[j] += df[j], sg[j] += dg[j];
    }
    if (l.live && t0 + k < a.T) {
      char* row = (char*)a.dp + (size_t)(t0 + k) * (4 * BH * sizeof(T));
      store_pair<T, R>(row, ga, di, l.two);
      store_pair<T, R>(row, ga + gs, df, l.two);
      store_pair<T, R>(row, ga + 2 * gs, dg, l.two);
    }
  }
  if (a.dc0 && l.live && chunk == 0 && wave == 0) store_state<R>(a.dc0, l.at, e, l.two);
  if (!a.dbias) return;
  // sums of the waves, in order (lds.wave is 2 x W rows of 64)
  lds_barrier();
  lds.wave[0][wave][lane] = f32x4{si[0], si[1], sf[0], sf[1]};
  lds.wave[1][wave][lane] = f32x4{sg[0], sg[1], so[0], so[1]};
  lds_barrier();
  if (wave < 2 && l.live) {
    f32x4 t = lds.wave[wave][0][lane];
#pragma unroll
    for (int v = 1; v < W; ++v) t += lds.wave[wave][v][lane];
    float* row = a.dpart + ((size_t)(LOOK ? order : 0) * a.B + l.b) * (4 * (size_t)a.H) + (size_t)2 * wave * a.H + l.r;
    row[0] = t[0], row[a.H] = t[2];
    if (l.two) row[1] = t[1], row[a.H + 1] = t[3];
  }
}

// dbias[k] = the sum of the rows of dpart: 32 columns and 32 runs of rows a
// workgroup, the runs summed in order.
__global__ void __launch_bounds__(1024) linear_dbias_kernel(const float* dpart, int rows, int n, float* dbias) {
  __shared__ float part[32][33];
  const int c = threadIdx.x & 31, q = threadIdx.x >> 5, k = blockIdx.x * 32 + c;
  float s[4] = {0.f, 0.f, 0.f, 0.f};
  if (k < n) {
    int r = q;
    for (; r + 96 < rows; r += 128)
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] += dpart[(size_t)(r + 32 * j) * n + k];
    for (; r < rows; r += 32) s[0] += dpart[(size_t)r * n + k];
  }
  part[q][c] = (s[0] + s[1]) + (s[2] + s[3]);
  __syncthreads();
  if (q != 0 || k >= n) return;
  float t = part[0][c];
  for (int j = 1; j < 32; ++j) t += part[j][c];
  dbias[k] = t;
}

// Empties the hand-over words and the tickets.
__global__ void __launch_bounds__(256) linear_clear_kernel(u32x4* words, size_t n, u32x4* tickets, size_t nt) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n + nt; i += (size_t)gridDim.x * 256) {
    if (i < n) words[i] = u32x4{kEmpty, kEmpty, kEmpty, kEmpty};
    else tickets[i - n] = u32x4{0u, 0u, 0u, 0u};
  }
}

struct Plan {
  LinearScan s;
  bool few, walk, look;
  size_t lanes;          // pairs of units
  size_t maps, states, tickets, dpart;   // bytes
  int rows;              // of dpart
};

// Up to how many timesteps the walk is the faster forward kernel: the scan splits 9
// timesteps and more over waves, but those are there anyway once there are many
// columns.  Walk / scan in us, bf16: 1 sequence of 512 units, T = 8 6.7 / 6.5, 16 7.1 / 6.5; 32
// of 1024 (a column a compute unit), T = 8 6.8 / 6.6, 16 8.0 / 6.7, 24 10.0 / 6.6; 64 (two), T =
// 16 7.9 / 7.5; 96 (three), T = 8 7.5 / 7.6, 16 9.0 / 9.1 (fp32 9.5 / 12.5), 24 11.6 / 10.6; 128
// (four), T = 16 9.2 / 11.3, 24 11.9 / 12.5, 32 14.6 / 13.9; 512 of 512 units, T = 8 8.3 / 17.2, 24
// 17.5 / 23.9, 32 22.5 / 26.6.
int walked(size_t cols, int num_cu) { return cols >= 4 * (size_t)num_cu ? 24 : cols > 2 * (size_t)num_cu ? 16 : 8; }

// columns of 64 pairs of units; chunks of time of one; both together.  A backward pass of
// two waves' timesteps makes one chunk of two waves (a workgroup of eight would hold waves
// of padding: 256 sequences of 512 units, forward and back, bf16, T = 16 24.6 us, with eight
// 35.6; T = 1 20 and 30).
constexpr int kFew = 2 * kSteps;
size_t cols_of(int B, int H) { return ((size_t)B * ((H + 1) / 2) + 63) / 64; }
int chunks_of(int T, int backward) {
  const int chunk = backward && T <= kFew ? kFew : kChunk;
  return std::max(1, (T + chunk - 1) / chunk);
}
size_t pieces_of(int T, int B, int H, int backward) { return cols_of(B, H) * chunks_of(T, backward); }

// for sizes that linear_fits takes
Plan plan_of(int T, int B, int H, int num_cu, int backward) {
  Plan p{};
  const int pairs = (H + 1) / 2;
  p.lanes = (size_t)B * pairs;
  p.s.lanes = (int)p.lanes;
  p.s.cols = (int)cols_of(B, H);
  p.few = T <= kFew;
  p.s.chunks = chunks_of(T, backward);
  p.walk = !backward && T <= walked(p.s.cols, num_cu);
  // Forward, chunks side by side where there are at least four and the columns
  // alone leave compute units with fewer than two workgroups (bf16, H = 512, T = 512,
  // side by side / one after another: 64 sequences 49 / 48 us, 96 68 / 74, 128 93 / 82, 256
  // 173 / 159; H = 64, T = 100, two chunks, 12.7 / 10.6, T = 200, four, 12.2 / 17.3: the words'
  // clearing is a launch).  Backward always: a loop needs more registers than there are
  // (as long as there was one, 64, 128 and 256 sequences forward and back took 126 / 126,
  // 249 / 259, 460 / 510 us).  A grid has fewer than 2^32
  // threads: beyond, forward takes the loop and backward is refused.
  const size_t pieces = pieces_of(T, B, H, backward);
  p.look = !p.walk && p.s.chunks > 1 &&
           (backward || (p.s.chunks >= 4 && p.s.cols < 2 * num_cu && pieces <= kMostChunks));
  if (p.look) {
    const size_t groups = (size_t)(p.s.chunks + kGroup - 1) / kGroup;
    p.maps = ((size_t)p.s.chunks + p.s.chunks / kScanWaves) * p.lanes * 16;
    p.states = (groups * p.lanes * 8 + 15) / 16 * 16;
    p.tickets = (size_t)p.s.cols * kTicketStride * 4;
  }
  p.rows = B * (p.look ? p.s.chunks : 1);
  p.dpart = backward == 2 ? (size_t)p.rows * 4 * H * 4 : 0;
  return p;
}

hipError_t place(Plan& p, LinearArgs& a, void* ws, hipStream_t stream) {
  char* w = (char*)ws;
  p.s.maps = (unsigned long long*)w;
  p.s.states = (unsigned*)(w + p.maps);
  p.s.tickets = (unsigned*)(w + p.maps + p.states);
  a.dpart = (float*)(w + p.maps + p.states + p.tickets);
  if (!p.look) return hipSuccess;
  const size_t n = (p.maps + p.states) / 16, nt = p.tickets / 16;
  linear_clear_kernel<<<(unsigned)std::min<size_t>((n + nt + 255) / 256, 1024), 256, 0, stream>>>(
      (u32x4*)w, n, (u32x4*)p.s.tickets, nt);
  return hipGetLastError();
}

template <class T, Rows R>
void launch_run(const LinearArgs& a, const Plan& p, hipStream_t stream) {
  if (p.walk)
    linear_walk_kernel<T, R><<<(unsigned)((p.lanes + kWalkThreads - 1) / kWalkThreads), kWalkThreads, 0, stream>>>(a);
  else if (p.look)
    linear_scan_kernel<T, R, true><<<(unsigned)p.s.cols * p.s.chunks, kScanThreads, 0, stream>>>(a, p.s);
  else
    linear_scan_kernel<T, R, false><<<p.s.cols, kScanThreads, 0, stream>>>(a, p.s);
}

template <class T, Rows R>
void launch_back(const LinearArgs& a, const Plan& p, hipStream_t stream) {
  if (p.look)
    linear_back_kernel<T, R, true, kScanWaves><<<(unsigned)p.s.cols * p.s.chunks, kScanThreads, 0, stream>>>(a, p.s);
  else if (p.few)
    linear_back_kernel<T, R, false, 2><<<p.s.cols, 128, 0, stream>>>(a, p.s);
  else
    linear_back_kernel<T, R, false, kScanWaves><<<p.s.cols, kScanThreads, 0, stream>>>(a, p.s);
}

// f of a's kind of rows
template <class F>
void rows_of(const LinearArgs& a, F f) {
  if (a.H == 1) f(std::integral_constant<Rows, kSingle>{});
  else if (a.H % 2) f(std::integral_constant<Rows, kOdd>{});
  else f(std::integral_constant<Rows, kEven>{});
}

}  // namespace

bool linear_fits(int T, int B, int H, int backward) { return !backward || pieces_of(T, B, H, backward) <= kMostChunks; }

size_t linear_workspace(int T, int B, int H, int num_cu, int backward) {
  const Plan p = plan_of(T, B, H, num_cu, backward);
  return p.maps + p.states + p.tickets + p.dpart;
}

hipError_t launch_linear(const LinearArgs& a0, void* ws, hipStream_t stream) {
  LinearArgs a = a0;
  Plan p = plan_of(a.T, a.B, a.H, a.num_cu, 0);
  const hipError_t e = place(p, a, ws, stream);
  if (e != hipSuccess) return e;
  if (a.bf16) rows_of(a, [&](auto r) { launch_run<__bf16, decltype(r)::value>(a, p, stream); });
  else rows_of(a, [&](auto r) { launch_run<float, decltype(r)::value>(a, p, stream); });
  return hipGetLastError();
}

hipError_t launch_linear_backward(const LinearArgs& a0, void* ws, hipStream_t stream) {
  LinearArgs a = a0;
  Plan p = plan_of(a.T, a.B, a.H, a.num_cu, a.dbias ? 2 : 1);
  hipError_t e = place(p, a, ws, stream);
  if (e != hipSuccess) return e;
  if (a.bf16) rows_of(a, [&](auto r) { launch_back<__bf16, decltype(r)::value>(a, p, stream); });
  else rows_of(a, [&](auto r) { launch_back<float, decltype(r)::value>(a, p, stream); });
  e = hipGetLastError();
  if (e != hipSuccess || !a.dbias) return e;
  linear_dbias_kernel<<<(4 * a.H + 31) / 32, 1024, 0, stream>>>(a.dpart, p.rows, 4 * a.H, a.dbias);
  return hipGetLastError();
}

}  // namespace alstm
