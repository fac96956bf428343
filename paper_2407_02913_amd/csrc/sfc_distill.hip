// Distillation from a teacher's top logits.
//
//   q = softmax(s / T) of the student's logits s, p the teacher's probabilities at its `top` places:
//   softmax(t / T) over them, or exp(t) with the rest r = 1 - sum p as one more outcome (tail).
//   loss = T^2 [sum p (log p - log q) + r (log r - log q_rest)],  q_rest: the sum of q outside the top
//   gradient / (row's scale T): q - p on the top, outside q, or q (1 - r / q_rest) with a tail
//
// The logits are the largest tensor of a training step, and a row's gradient needs the whole row's sum: a row is
// kept in registers as it was loaded (distill_rows: by a wave up to 256 vectors of 16 bytes, by a workgroup above),
// so that loss and gradient read it once and write it once.  Rows past the registers are read twice, the second time
// mostly out of the caches (distill_stream).  The gradient is stored as if there were no teacher, then the wave that
// stored a place's vector stores that place once more.  With a tail the sum outside the top is added up as such (a
// difference of sums would lose it where the top holds nearly all): a byte of LDS a vector tells its elements.
#include "sfc_distill.hpp"

namespace sfc {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// A wave or a workgroup that owns a row.
template <bool WAVE>
struct Team {
  float* scratch;  // 16 floats a use
  __device__ __forceinline__ int lane() const { return WAVE ? threadIdx.x & 63 : threadIdx.x; }
  __device__ __forceinline__ int size() const { return WAVE ? 64 : blockDim.x; }
  __device__ __forceinline__ void sync() const {
    if constexpr (WAVE) {
      // lanes of one wave: LDS accesses stay in order once the compiler keeps them so
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    } else {
      __syncthreads();
    }
  }
  __device__ __forceinline__ float sum(float v) {
    v = wave_sum(v);
    if constexpr (!WAVE) {
      float* at = scratch;
      scratch += 16;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
      __syncthreads();
      v = 0.0f;
      for (int i = 0; i < (int)(blockDim.x >> 6); ++i) v += at[i];
    }
    return v;
  }
  __device__ __forceinline__ float max(float v) {
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, 64));
    if constexpr (!WAVE) {
      float* at = scratch;
      scratch += 16;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
      __syncthreads();
      for (int i = 0; i < (int)(blockDim.x >> 6); ++i) v = fmaxf(v, at[i]);
    }
    return v;
  }
};
constexpr int kUses = 8;  // sums and maxima of a row

// LDS of a row: scratch; of each of the teacher's places its probability, that of all entries for the same place,
// its logit and where it is; a byte for each vector (tail).
struct RowSpace {
  float* scratch;
  float* p;
  float* all;
  float* logit;
  int* at;
  unsigned* map;
};

int row_space_bytes(int top, int items, bool tail) {
  return kUses * 16 * 4 + (top + 3) / 4 * 4 * 16 + (tail ? (items + 15) / 16 * 16 : 0);
}

__device__ __forceinline__ RowSpace row_space(char* base, int top) {
  const int places = (top + 3) / 4 * 4;
  RowSpace s;
  s.scratch = reinterpret_cast<float*>(base);
  s.p = s.scratch + kUses * 16;
  s.all = s.p + places;
  s.logit = s.all + places;
  s.at = reinterpret_cast<int*>(s.logit + places);
  s.map = reinterpret_cast<unsigned*>(s.at + places);
  return s;
}

// Elements past the row's end: -inf, which no maximum and no sum of exponentials notices.
template <typename T>
constexpr unsigned kNone = sizeof(T) == 4 ? 0xff800000u : __is_same(T, bf16) ? 0xff80ff80u : 0xfc00fc00u;

// What a row's loss and gradient are made of.
struct Row {
  float max, sum;         // of the student: largest logit, sum of exp((s - max) / T)
  float ratio;            // tail: r / q_rest, else 0
  float mass;             // sum of the teacher's probabilities, the rest included
};

// The teacher's entries into LDS (a place outside the classes is none) and, with a tail, the map of vectors that hold
// any.  Returns (sum of p, log of what the exponentials were divided by); ends with a barrier, before which every
// logit at a place has been read.
template <typename T, bool WAVE>
__device__ __forceinline__ float2 stage_teacher(const DistillArgs& a, int64_t row, const RowSpace& s, Team<WAVE>& team,
                                                const T* logits) {
  constexpr int V = kVec<T>;
  const int lane = team.lane(), size = team.size();
  const float* values = a.values + row * a.values_stride;
  if (a.tail) {
    const int words = (a.classes + 4 * V - 1) / (4 * V);
    for (int i = lane; i < words; i += size) s.map[i] = 0u;
    team.sync();
  }
  float top = -INFINITY;
  for (int k = lane; k < a.top; k += size) {
    const int64_t at = a.wide ? static_cast<const int64_t*>(a.index)[row * a.index_stride + k]
                              : static_cast<const int32_t*>(a.index)[row * a.index_stride + k];
    const int place = at >= 0 && at < a.classes ? (int)at : -1;
    const float v = values[k];
    s.at[k] = place;
    s.p[k] = v;
    if (place >= 0) {
      s.logit[k] = (float)logits[place];
      top = fmaxf(top, v);
      if (a.tail) atomicOr(&s.map[place / (4 * V)], 1u << (place / V % 4 * 8 + place % V));
    }
  }
  float about = 0.0f, log_sum = 0.0f, c = 1.0f, scale = 1.0f;
  if (!a.tail) {
    top = team.max(top);
    about = top == -INFINITY ? 0.0f : top;
    c = 1.0f / a.temperature;
    float sum = 0.0f;
    for (int k = lane; k < a.top; k += size)
      if (s.at[k] >= 0) sum += __expf((s.p[k] - about) * c);
    sum = team.sum(sum);
    scale = sum == 0.0f ? 0.0f : 1.0f / sum;
    log_sum = about * c + __logf(sum);
  }
  float mass = 0.0f;
  for (int k = lane; k < a.top; k += size) {
    const float p = s.at[k] < 0 ? 0.0f : __expf((s.p[k] - about) * c) * scale;
    s.p[k] = p;
    mass += p;
  }
  mass = team.sum(mass);
  team.sync();
  if (a.grad) {
    // entries for one place, added in their order by each of them
    for (int k = lane; k < a.top; k += size) {
      const int mine = s.at[k];
      float all = 0.0f;
      for (int i = 0; i < a.top; ++i) all += s.at[i] == mine ? s.p[i] : 0.0f;
      s.all[k] = all;
    }
    team.sync();
  }
  return make_float2(mass, log_sum);
}

// The elements of this lane's vector that are the teacher's.
__device__ __forceinline__ unsigned top_elements(const RowSpace& s, int item) {
  return s.map[item >> 2] >> (item & 3) * 8 & 255u;
}

// The gradient of a vector outside the teacher's places, stored.
template <typename T>
__device__ __forceinline__ void store_grad(const DistillArgs& a, const Row& row, float scale, int item, const raw4& raw,
                                           T* grad) {
  constexpr int V = kVec<T>;
  const float c = kLog2e / a.temperature, unit = scale / row.sum * (row.mass - row.ratio);
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = __builtin_amdgcn_exp2f((element<T>(raw, j) - row.max) * c) * unit;
  store_vec<T, V>(grad + (int64_t)item * V, v, min(V, a.classes - item * V));
}

// The gradient at the teacher's places, by the wave whose lanes stored their vectors: a wave's stores to one address
// stay in order.
template <typename T, bool WAVE>
__device__ __forceinline__ void store_places(const DistillArgs& a, const RowSpace& s, Team<WAVE>& team, const Row& row,
                                             float scale, T* grad) {
  constexpr int V = kVec<T>;
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  const float c = kLog2e / a.temperature;
  for (int k = threadIdx.x & 63; k < a.top; k += 64) {
    const int place = s.at[k];
    if (place < 0 || (!WAVE && place / V % team.size() / 64 != (int)(threadIdx.x >> 6))) continue;
    const float q = __builtin_amdgcn_exp2f((s.logit[k] - row.max) * c) / row.sum;
    grad[place] = (T)((q * row.mass - s.all[k]) * scale);
  }
}

template <typename T>
__device__ __forceinline__ void store_nothing(const DistillArgs& a, int item, T* grad) {
  constexpr int V = kVec<T>;
  float v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = 0.0f;
  store_vec<T, V>(grad + (int64_t)item * V, v, min(V, a.classes - item * V));
}

// Sums of exp((s - max) / T) of a vector: of the elements outside the teacher's places and, with a tail, of those
// on them (else of all).
template <typename T>
__device__ __forceinline__ void add_exp(const DistillArgs& a, const RowSpace& s, const raw4& raw, int item, bool live,
                                        float max, float* rest, float* top) {
  constexpr int V = kVec<T>;
  const float c = kLog2e / a.temperature;
  float e[V];
#pragma unroll
  for (int j = 0; j < V; ++j) e[j] = __builtin_amdgcn_exp2f((element<T>(raw, j) - max) * c);
  if (a.tail) {
    const unsigned mask = live ? top_elements(s, item) : 0u;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const bool in = mask >> j & 1u;
      *rest += in ? 0.0f : e[j];
      *top += in ? e[j] : 0.0f;
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) *rest += e[j];
  }
}

// Loss and statistics once the student's sums stand.
template <bool WAVE>
__device__ __forceinline__ Row finish_loss(const DistillArgs& a, int64_t row, const RowSpace& s, Team<WAVE>& team,
                                           float2 teacher, float max, float rest, float top) {
  const float c = 1.0f / a.temperature;
  Row r;
  r.max = max;
  r.sum = rest + top;
  r.ratio = 0.0f;
  r.mass = teacher.x;
  const float log_sum = __logf(r.sum);
  const float* values = a.values + row * a.values_stride;
  float loss = 0.0f;
  for (int k = team.lane(); k < a.top; k += team.size()) {
    const int place = s.at[k];
    const float p = s.p[k];
    if (place >= 0 && p != 0.0f) {
      const float log_q = (s.logit[k] - max) * c - log_sum;
      const float log_p = a.tail ? values[k] : values[k] * c - teacher.y;
      loss += p * (log_p - log_q);
    }
  }
  loss = team.sum(loss);
  if (a.tail) {
    const float p_rest = 1.0f - teacher.x;
    // (no mass to speak of, or none left by rounding where the top holds every class: no outcome)
    if (p_rest > 0.0f && (rest != 0.0f || p_rest > 1e-6f)) {
      const float q_rest = rest / r.sum;
      loss += p_rest * (__logf(p_rest) - __logf(q_rest));
      r.ratio = rest != 0.0f ? p_rest / q_rest : 0.0f;
      r.mass += p_rest;
    }
  }
  if (team.lane() == 0) {
    if (a.loss) a.loss[row] = loss * a.temperature * a.temperature;
    if (a.stats) reinterpret_cast<float4*>(a.stats)[row] = make_float4(r.max, r.sum, r.ratio, r.mass);
  }
  return r;
}

// A row whose scale is zero: nothing of it is read.
template <typename T, bool WAVE>
__device__ __forceinline__ void masked_row(const DistillArgs& a, int64_t row, Team<WAVE>& team) {
  if (a.loss && team.lane() == 0) {
    a.loss[row] = 0.0f;
    if (a.stats) reinterpret_cast<float4*>(a.stats)[row] = make_float4(0.0f, 1.0f, 0.0f, 0.0f);
  }
  if (a.grad) {
    T* grad = static_cast<T*>(a.grad) + row * a.grad_stride;
    for (int q = team.lane(); q * kVec<T> < a.classes; q += team.size()) store_nothing<T>(a, q, grad);
  }
}

__device__ __forceinline__ Row row_of_stats(const DistillArgs& a, int64_t row) {
  const float4 v = reinterpret_cast<const float4*>(a.stats)[row];
  Row r;
  r.max = v.x, r.sum = v.y, r.ratio = v.z, r.mass = v.w;
  return r;
}

// A row to a team, NV vectors to a lane.
template <typename T, int NV, bool WAVE>
__global__ __launch_bounds__(WAVE ? 256 : 1024) void distill_rows(DistillArgs a, int space) {
  constexpr int V = kVec<T>;
  extern __shared__ float4 lds[];
  const int64_t row = WAVE ? (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (WAVE && row >= a.rows) return;
  const RowSpace s = row_space(reinterpret_cast<char*>(lds) + (WAVE ? (threadIdx.x >> 6) * space : 0), a.top);
  Team<WAVE> team{s.scratch};
  const float scale = a.row_scale ? a.row_scale[row] : 1.0f;
  if (scale == 0.0f) {
    masked_row<T, WAVE>(a, row, team);
    return;
  }
  const T* logits = static_cast<const T*>(a.logits) + row * a.logits_stride;
  const int64_t room = (a.rows - 1 - row) * a.logits_stride + a.classes;
  const int items = (a.classes + V - 1) / V, lane = team.lane(), size = team.size();
  raw4 raw[NV];
#pragma unroll
  for (int u = 0; u < NV; ++u) {
    const int q = lane + u * size;
    raw[u] = raw4{kNone<T>, kNone<T>, kNone<T>, kNone<T>};
    if (q < items) raw[u] = load_cut(logits + (int64_t)q * V, a.classes - q * V, room - (int64_t)q * V, kNone<T>);
  }
  const float2 teacher = stage_teacher<T, WAVE>(a, row, s, team, logits);
  Row r;
  if (a.loss) {
    float max = -INFINITY;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
#pragma unroll
      for (int j = 0; j < V; ++j) max = fmaxf(max, element<T>(raw[u], j));
      asm volatile("" : "+v"(raw[u]));  // (the loaded bits are kept, not the floats made of them)
    }
    max = team.max(max);
    float rest = 0.0f, top = 0.0f;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int q = lane + u * size;
      add_exp<T>(a, s, raw[u], q, q < items, max, &rest, &top);
      asm volatile("" : "+v"(raw[u]));
    }
    rest = team.sum(rest);
    if (a.tail) top = team.sum(top);
    r = finish_loss<WAVE>(a, row, s, team, teacher, max, rest, a.tail ? top : 0.0f);
  } else {
    r = row_of_stats(a, row);
  }
  if (a.grad) {
    T* grad = static_cast<T*>(a.grad) + row * a.grad_stride;
#pragma unroll
    for (int u = 0; u < NV; ++u) {
      const int q = lane + u * size;
      if (q < items) store_grad<T>(a, r, scale * a.temperature, q, raw[u], grad);
    }
    store_places<T, WAVE>(a, s, team, r, scale * a.temperature, grad);
  }
}

// A row to a workgroup, read once for its sums and once more for the gradient.
template <typename T>
__global__ __launch_bounds__(1024) void distill_stream(DistillArgs a) {
  constexpr int V = kVec<T>;
  extern __shared__ float4 lds[];
  const int64_t row = blockIdx.x;
  const RowSpace s = row_space(reinterpret_cast<char*>(lds), a.top);
  Team<false> team{s.scratch};
  const float scale = a.row_scale ? a.row_scale[row] : 1.0f;
  if (scale == 0.0f) {
    masked_row<T, false>(a, row, team);
    return;
  }
  const T* logits = static_cast<const T*>(a.logits) + row * a.logits_stride;
  const int64_t room = (a.rows - 1 - row) * a.logits_stride + a.classes;
  const int items = (a.classes + V - 1) / V, lane = threadIdx.x, size = blockDim.x;
  auto load = [&](int q) {
    if (q >= items) return raw4{kNone<T>, kNone<T>, kNone<T>, kNone<T>};
    return load_cut(logits + (int64_t)q * V, a.classes - q * V, room - (int64_t)q * V, kNone<T>);
  };
  const float2 teacher = stage_teacher<T, false>(a, row, s, team, logits);
  Row r;
  if (a.loss) {
    // each thread its own running maximum, its sums scaled down when that grows
    const float c = kLog2e / a.temperature;
    float max = -INFINITY, rest = 0.0f, top = 0.0f;
    for (int q0 = lane; q0 < items; q0 += 4 * size) {
      raw4 raw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) raw[u] = load(q0 + u * size);
      float m = max;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
#pragma unroll
        for (int j = 0; j < V; ++j) m = fmaxf(m, element<T>(raw[u], j));
      }
      if (m > max) {
        const float f = __builtin_amdgcn_exp2f((max - m) * c);
        rest *= f, top *= f;
        max = m;
      }
      // (nothing but -inf so far counts for nothing; a NaN makes the sums one)
      const float about = max == -INFINITY ? 0.0f : max;
#pragma unroll
      for (int u = 0; u < 4; ++u)
        add_exp<T>(a, s, raw[u], q0 + u * size, q0 + u * size < items, about, &rest, &top);
    }
    const float m = team.max(max);
    const float f = max == m ? 1.0f : __builtin_amdgcn_exp2f((max - m) * c);
    rest = team.sum(rest * f);
    top = a.tail ? team.sum(top * f) : 0.0f;
    if (m == -INFINITY) rest = NAN;
    r = finish_loss<false>(a, row, s, team, teacher, m, rest, top);
  } else {
    r = row_of_stats(a, row);
  }
  if (a.grad) {
    T* grad = static_cast<T*>(a.grad) + row * a.grad_stride;
    for (int q0 = 0; q0 < items; q0 += 4 * size) {
      raw4 raw[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) raw[u] = load(q0 + u * size + lane);
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int q = q0 + u * size + lane;
        if (q < items) store_grad<T>(a, r, scale * a.temperature, q, raw[u], grad);
      }
    }
    store_places<T, false>(a, s, team, r, scale * a.temperature, grad);
  }
}

template <typename T, int NV, bool WAVE>
hipError_t run_rows(const DistillArgs& a, int threads, int items, hipStream_t s) {
  const int space = row_space_bytes(a.top, items, a.tail);
  const unsigned blocks = WAVE ? (unsigned)((a.rows + 3) / 4) : (unsigned)a.rows;
  distill_rows<T, NV, WAVE><<<dim3(blocks), dim3((unsigned)threads), WAVE ? 4 * space : space, s>>>(a, space);
  return hipGetLastError();
}

template <typename T>
hipError_t run_distill(const DistillArgs& a, hipStream_t s) {
  const int items = (a.classes + kVec<T> - 1) / kVec<T>;
  if (items <= 64) return run_rows<T, 1, true>(a, 256, items, s);
  if (items <= 128) return run_rows<T, 2, true>(a, 256, items, s);
  if (items <= 256) return run_rows<T, 4, true>(a, 256, items, s);
  if (items <= 1024) return run_rows<T, 4, false>(a, 256, items, s);
  if (items <= 2048) return run_rows<T, 4, false>(a, 512, items, s);
  if (items <= 4096) return run_rows<T, 4, false>(a, 1024, items, s);
  if (items <= 8192) return run_rows<T, 8, false>(a, 1024, items, s);
  if (items <= 16384) return run_rows<T, 16, false>(a, 1024, items, s);
  const int space = row_space_bytes(a.top, items, a.tail);
  if (space > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(distill_stream<T>),
                                             hipFuncAttributeMaxDynamicSharedMemorySize, space);
    if (e != hipSuccess) return e;
  }
  distill_stream<T><<<dim3((unsigned)a.rows), dim3(1024), space, s>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_distill(const DistillArgs& a, int type, hipStream_t s) {
  if (type == 0) return run_distill<float>(a, s);
  return type == 1 ? run_distill<f16>(a, s) : run_distill<bf16>(a, s);
}

}  // namespace sfc
