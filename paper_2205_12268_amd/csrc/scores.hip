// Log probabilities of given tokens, entropy and the top alternatives of rows of logits (wcc_token_scores).
//
// With m the largest logit of a row, S = sum e^(x - m) and E = sum (x - m) e^(x - m):
//   log p = (x - m) - log S,   entropy = log S - E / S.
// A workgroup holds a slice of a row in registers (rows.h), so that its largest is known before the first exponential and
// memory is read once.  Few rows, and rows that are longer than a workgroup holds, are cut into slices, whose (m, S, E) and
// best keys a second launch joins in the order of the slices.
//
// The top: elements are ordered by (logit, falling; index, rising).  Each of the 64 lanes, over all waves, has a best element;
// the top-th best of those 64 is a bound that at least `top` elements reach, and few more do (24 on average for the 20 best
// of a row in random order, at most 512 where all are equal).  The threads that hold one are listed, their elements read
// again and those that reach the bound ranked by counting.  What decides is always the elements' order itself, never their
// arrival, so the result does not depend on it.
//
// Bound by memory where rows are many: 4096 x 32768 bf16 67 us, 4.0 TB/s (55 us at the rate of a large copy; an exponential an element
// takes the rest); by two launches and their chains of reductions where they are few: one row of 131072 14.3 us, 7.6 and 6.4 of the
// kernels.  A first form, a workgroup a row that reads it again for each alternative, took 1252 and 1691 us.
#include "rows.h"

namespace wcc {
namespace {

constexpr int kCandidates = 1024;  // elements beyond the bound that are ranked by counting; more: one round a result

// A logit and an index as one number that orders as the answer does.  NaN sorts above +inf, -0 is +0; 0 is below all.
__device__ __forceinline__ uint64_t order_key(float v, int i) {
  const uint32_t u = __float_as_uint(v + 0.f);
  const uint32_t o = v != v ? 0xffffffffu : (u & 0x80000000u) ? ~u : u | 0x80000000u;
  return (uint64_t)o << 32 | (uint32_t)~i;
}
__device__ __forceinline__ float key_value(uint64_t k) {
  const uint32_t o = (uint32_t)(k >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ int key_index(uint64_t k) { return (int)~(uint32_t)k; }

// The k-th largest of the 64 lanes' keys, which are distinct but for zeros; 0 if fewer than k are not zero.
__device__ __forceinline__ uint64_t kth_of_lanes(uint64_t g, int k) {
  int above = 0;
#pragma unroll
  for (int j = 0; j < 64; ++j) {
    const uint64_t o = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(g >> 32), j) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane((int)g, j);
    above += o > g ? 1 : 0;
  }
  const uint64_t who = __ballot(g != 0 && above == k - 1);
  if (who == 0) return 0;
  const int lane = __builtin_ctzll(who);
  return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(g >> 32), lane) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)g, lane);
}

struct Part {
  float m, s, e, pad;  // of a slice, exponents to base 2
};

struct Out {
  const int32_t *tokens;
  float *logprob, *entropy;
  int32_t *top_idx;
  float *top_logprob;
};

// (x - m) - log S; a row that has nothing left has S = 0 and -inf throughout
__device__ __forceinline__ float log_p(float x, float base, float s, float log_s) {
  return s == 0.f ? -INFINITY : (x - base) - log_s;
}

template <class T>
__device__ __forceinline__ void write_scalars(const Out &o, int64_t t, const T *row, int V, float base, float s, float e) {
  const float log_s = logf(s);
  if (o.logprob) {
    const int v = o.tokens[t];
    o.logprob[t] = (uint32_t)v >= (uint32_t)V ? NAN : log_p(widen(row[v]), base, s, log_s);
  }
  if (o.entropy) o.entropy[t] = s == 0.f ? 0.f : log_s - e * kLn2 / s;
}

template <class T, int NT, int NV, bool TOP>
__global__ __launch_bounds__(NT, 4) void scores_slice_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int V, int top,
                                                          int slices, int length, Out out, Part *__restrict__ part,
                                                          uint64_t *__restrict__ keys) {
  constexpr int VE = VecOf<T>::N, NW = NT / 64;
  __shared__ float fpart[3][NW];
  __shared__ uint64_t best[TOP ? NT : 1], cand[TOP ? kCandidates : 1], bound;
  __shared__ int holder[TOP ? NT : 1], n_holder, n_cand;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  const int64_t total = rows * slices;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int64_t t = w / slices;
    const int first = (int)(w - t * slices) * length, n = min(length, V - first);
    const T *r = x + t * ld + first;
    u32x4 v[NV];
    load_slice<T, NT, NV>(r, n, v);

    // the slice's largest, and which of the thread's vectors has its own (the first of equals)
    float mine = -INFINITY;
    int at = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      float vm = elem<T>(v[i], 0);
#pragma unroll
      for (int j = 1; j < VE; ++j) vm = largest_of(vm, elem<T>(v[i], j));
      if (vm > mine) at = i;
      mine = largest_of(mine, vm);
    }
    uint64_t my_key = 0;  // largest element, start of its vector
    if constexpr (TOP) {
      if (tid * VE < n) my_key = order_key(mine, (at * NT + tid) * VE);
      best[tid] = my_key;
      if (tid == 0) n_holder = n_cand = 0;
    }
    const float m = block_all<NT>(mine, fpart[0], Largest());
    const float base = m == -INFINITY ? 0.f : m;
    hold(v);

    // To base 2: d = (x - m) log2(e).  One fma a logit, x log2(e) - c with c = m log2(e) rounded, whose error `off`, the same for
    // all, is taken off the sums; a large m, beside which it would not be small, has the subtraction first, from memory.
    // (E: 0 times -inf; 2^-200 is 0.)
    float s[2] = {0.f, 0.f}, e[2] = {0.f, 0.f}, off = 0.f;
    if (fabsf(base) < 1024.f) {
      const float c = base * kLog2e;
      off = fmaf(base, kLog2e, -c);
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int j = 0; j < VE; ++j) {
          const float d = largest_of(fmaf(elem<T>(v[i], j), kLog2e, -c), -200.f), p = __builtin_amdgcn_exp2f(d);
          s[j & 1] += p;
          e[j & 1] = fmaf(p, d, e[j & 1]);
        }
    } else {
      for (int i = tid; i < n; i += NT) {
        const float d = largest_of((widen(r[i]) - base) * kLog2e, -200.f), p = __builtin_amdgcn_exp2f(d);
        s[0] += p;
        e[0] = fmaf(p, d, e[0]);
      }
    }
    float st = wave_all(s[0] + s[1], Sum()), et = wave_all(e[0] + e[1], Sum());
    if constexpr (NT > 64) {
      if (lane == 0) fpart[1][wv] = st, fpart[2][wv] = et;
    }
    if constexpr (TOP) {
      if (NT == 64) __syncthreads();  // best[]
      if (wv == 0) {
        uint64_t g = best[lane];
#pragma unroll
        for (int i = 1; i < NW; ++i) g = max(g, best[i * 64 + lane]);
        const uint64_t b = kth_of_lanes(g, top);
        if (lane == 0) bound = b;
      }
    }
    if constexpr (NT > 64 || TOP) __syncthreads();
    if constexpr (NT > 64) {
      st = fpart[1][0], et = fpart[2][0];
#pragma unroll
      for (int i = 1; i < NW; ++i) st += fpart[1][i], et += fpart[2][i];
    }
    st = fmaf(st, -off * kLn2, st);
    et = fmaf(et, -off * kLn2, et) - off * st;
    if (tid == 0) {
      if (slices == 1) write_scalars(out, t, r, V, base, st, et);
      else part[w] = Part{m, st, et, 0.f};
    }

    if constexpr (TOP) {
      const uint64_t b = bound;
      const bool odd = st != st;  // NaN or +inf: the maxima above are not in the order of the keys
      if (!odd && my_key >= b && my_key != 0) holder[atomicAdd(&n_holder, 1)] = tid;
      __syncthreads();
      const int holders = n_holder;
      for (int c = wv; c < holders; c += NW) {
        const int th = holder[c];
        for (int q = lane; q < NV * VE; q += 64) {
          const int start = ((q / VE) * NT + th) * VE, i = start + q % VE;
          if (i >= n) continue;
          const float val = widen(r[i]);
          if (order_key(val, start) < b) continue;
          const int slot = atomicAdd(&n_cand, 1);
          if (slot < kCandidates) cand[slot] = order_key(val, first + i);
        }
      }
      __syncthreads();
      const int found = n_cand;
      const float log_s = logf(st);
      auto put = [&](int rank, uint64_t k) {
        if (slices == 1) {
          out.top_idx[t * top + rank] = key_index(k);
          if (out.top_logprob) out.top_logprob[t * top + rank] = log_p(key_value(k), base, st, log_s);
        } else {
          keys[w * top + rank] = k;
        }
      };
      if (!odd && found <= kCandidates) {
        for (int c = tid; c < found; c += NT) {
          const uint64_t k = cand[c];
          int rank = 0;
          for (int i = 0; i < found; ++i) rank += cand[i] > k ? 1 : 0;
          if (rank < top) put(rank, k);
        }
        for (int j = found + tid; j < top; j += NT) keys[w * top + j] = 0;  // a slice of fewer elements
      } else {
        uint64_t last = ~0ull;
        for (int j = 0; j < top; ++j) {
          uint64_t k = 0;
          for (int i = tid; i < n; i += NT) {
            const uint64_t o = order_key(widen(r[i]), first + i);
            if (o > k && (j == 0 || o < last)) k = o;
          }
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, off, 64));
          __syncthreads();
          if (lane == 0) best[wv] = k;
          __syncthreads();
          last = best[0];
          for (int i = 1; i < NW; ++i) last = max(last, best[i]);
          if (tid == 0 && (j < n || slices > 1)) put(j, last);
        }
      }
    }
    __syncthreads();  // LDS is used again
  }
}

// One workgroup a row: (m, S, E) of its slices, and the best of their keys.
template <class T>
__global__ __launch_bounds__(256) void scores_join_kernel(const T *__restrict__ x, int64_t ld, int64_t rows, int V, int top,
                                                          int slices, Out out, const Part *__restrict__ part,
                                                          const uint64_t *__restrict__ keys) {
  __shared__ uint64_t best[256], cand[kCandidates], bound;
  __shared__ float fpart[3][4];
  __shared__ int n_cand;
  const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
  for (int64_t t = blockIdx.x; t < rows; t += gridDim.x) {
    const Part *p = part + t * slices;
    float m = -INFINITY;
    for (int i = tid; i < slices; i += 256) m = largest_of(m, p[i].m);
    const int64_t total = (int64_t)slices * top;
    const uint64_t *ks = keys + t * total;
    constexpr int H = 8;  // keys of a thread that are loaded together, and held: all of them of 2048
    uint64_t held[H], mine = 0;
#pragma unroll
    for (int i = 0; i < H; ++i) held[i] = i * 256 + tid < total ? ks[i * 256 + tid] : 0;
#pragma unroll
    for (int i = 0; i < H; ++i) mine = max(mine, held[i]);
    for (int64_t i = H * 256 + tid; i < total; i += 256) mine = max(mine, ks[i]);
    best[tid] = mine;
    if (tid == 0) n_cand = 0;
    m = block_all<256>(m, fpart[0], Largest());
    const float base = m == -INFINITY ? 0.f : m;
    float s = 0.f, e = 0.f;
    for (int i = tid; i < slices; i += 256) {
      const Part q = p[i];
      if (q.s == 0.f) continue;
      const float d = (q.m - base) * kLog2e, f = __builtin_amdgcn_exp2f(d);
      s = fmaf(q.s, f, s);
      e = fmaf(f, fmaf(q.s, fmaxf(d, -200.f), q.e), e);
    }
    s = block_all<256>(s, fpart[1], Sum());
    e = block_all<256>(e, fpart[2], Sum());
    if (tid == 0) write_scalars(out, t, x + t * ld, V, base, s, e);
    if (top > 0) {
      if (wv == 0) {
        const uint64_t g = max(max(best[lane], best[64 + lane]), max(best[128 + lane], best[192 + lane]));
        const uint64_t b = kth_of_lanes(g, top);
        if (lane == 0) bound = b;
      }
      __syncthreads();
      const uint64_t b = bound;
      auto keep = [&](uint64_t k) {
        if (k == 0 || k < b) return;
        const int slot = atomicAdd(&n_cand, 1);
        if (slot < kCandidates) cand[slot] = k;
      };
      if (mine >= b) {
#pragma unroll
        for (int i = 0; i < H; ++i) keep(held[i]);
        for (int64_t i = H * 256 + tid; i < total; i += 256) keep(ks[i]);
      }
      __syncthreads();
      const int found = n_cand;
      const float log_s = logf(s);
      auto put = [&](int rank, uint64_t k) {
        out.top_idx[t * top + rank] = key_index(k);
        if (out.top_logprob) out.top_logprob[t * top + rank] = log_p(key_value(k), base, s, log_s);
      };
      if (found <= kCandidates) {
        for (int c = tid; c < found; c += 256) {
          const uint64_t k = cand[c];
          int rank = 0;
          for (int i = 0; i < found; ++i) rank += cand[i] > k ? 1 : 0;
          if (rank < top) put(rank, k);
        }
      } else {
        uint64_t last = ~0ull;
        for (int j = 0; j < top; ++j) {
          uint64_t k = 0;
          for (int64_t i = tid; i < total; i += 256) {
            const uint64_t o = ks[i];
            if (o > k && (j == 0 || o < last)) k = o;
          }
#pragma unroll
          for (int off = 32; off > 0; off >>= 1) k = max(k, (uint64_t)__shfl_xor((unsigned long long)k, off, 64));
          __syncthreads();
          if (lane == 0) best[wv] = k;
          __syncthreads();
          last = max(max(best[0], best[1]), max(best[2], best[3]));
          if (tid == 0) put(j, last);
        }
      }
    }
    __syncthreads();
  }
}

// Slices: as few as a workgroup's registers allow where there are rows enough to fill the card, else so many that there are two
// workgroups a compute unit, of one vector a thread at least; and of those counts and the next ones the one that leaves the
// fewest places of vectors empty (200 rows of 50001 fp32 logits: 20.5 us in three slices with half of theirs empty).
SlicePlan plan(const wcc_scores_desc &d) {
  const int ve = d.dtype == WCC_BF16 ? 8 : 4;
  const int64_t vecs = ((int64_t)d.V + ve - 1) / ve;
  const int64_t rows = std::max<int64_t>(d.rows, 1);
  int64_t least = (vecs + 512 * 16 - 1) / (512 * 16);
  if (rows * least < 512) least = std::max(least, std::min((512 + rows - 1) / rows, vecs / 256));
  least = std::max<int64_t>(least, 1);
  SlicePlan p{};
  int64_t cost = 0;
  for (int64_t want = least; want <= (least == 1 ? 1 : 2 * least); ++want) {
    const int64_t each = (vecs + want - 1) / want;
    const int nt = want == 1 && each <= 64 * 4 ? 64 : each <= 256 * 16 ? 256 : 512;
    int nv = 1;
    while ((int64_t)nt * nv < each) nv *= 2;
    const int64_t places = want * nt * nv;
    if (p.nt != 0 && places >= cost) continue;
    cost = places;
    p.length = (int)std::min<int64_t>(each * ve, d.V);
    p.slices = (int)(((int64_t)d.V + p.length - 1) / p.length);
    p.nt = nt, p.nv = nv;
  }
  return p;
}

size_t align256(size_t v) { return (v + 255) & ~(size_t)255; }

template <class T, int NT, int NV>
void launch_slices(const wcc_scores_desc &d, const ScoresArgs &g, const SlicePlan &p, const Out &o, Part *part, uint64_t *keys,
                   hipStream_t s) {
  const unsigned blocks = (unsigned)std::min<int64_t>(d.rows * p.slices, 1 << 20);
  if (d.top > 0)
    scores_slice_kernel<T, NT, NV, true><<<blocks, NT, 0, s>>>((const T *)g.x, d.ld, d.rows, d.V, d.top, p.slices, p.length, o, part, keys);
  else
    scores_slice_kernel<T, NT, NV, false><<<blocks, NT, 0, s>>>((const T *)g.x, d.ld, d.rows, d.V, 0, p.slices, p.length, o, part, keys);
}

template <class T>
void launch(const wcc_scores_desc &d, const ScoresArgs &g, hipStream_t s) {
  const SlicePlan p = plan(d);
  const Out o{g.tokens, g.logprob, g.entropy, g.top_idx, g.top_logprob};
  Part *part = (Part *)g.ws;
  uint64_t *keys = (uint64_t *)(g.ws + align256((size_t)d.rows * p.slices * sizeof(Part)));
  switch (p.nt * 100 + p.nv) {
    case 6401: launch_slices<T, 64, 1>(d, g, p, o, part, keys, s); break;
    case 6402: launch_slices<T, 64, 2>(d, g, p, o, part, keys, s); break;
    case 6404: launch_slices<T, 64, 4>(d, g, p, o, part, keys, s); break;
    case 25601: launch_slices<T, 256, 1>(d, g, p, o, part, keys, s); break;
    case 25602: launch_slices<T, 256, 2>(d, g, p, o, part, keys, s); break;
    case 25604: launch_slices<T, 256, 4>(d, g, p, o, part, keys, s); break;
    case 25608: launch_slices<T, 256, 8>(d, g, p, o, part, keys, s); break;
    case 25616: launch_slices<T, 256, 16>(d, g, p, o, part, keys, s); break;
    default: launch_slices<T, 512, 16>(d, g, p, o, part, keys, s); break;
  }
  if (p.slices > 1)
    scores_join_kernel<T><<<(unsigned)std::min<int64_t>(d.rows, 1 << 20), 256, 0, s>>>((const T *)g.x, d.ld, d.rows, d.V, d.top, p.slices,
                                                                                      o, part, keys);
}

}  // namespace

size_t scores_bytes(const wcc_scores_desc &d) {
  const SlicePlan p = plan(d);
  if (p.slices == 1) return 0;
  const size_t n = (size_t)d.rows * p.slices;
  return align256(n * sizeof(Part)) + align256(n * d.top * 8);
}

hipError_t launch_scores(const wcc_scores_desc &d, const ScoresArgs &g, hipStream_t s) {
  if (d.dtype == WCC_BF16) launch<bf16_t>(d, g, s);
  else launch<float>(d, g, s);
  return hipGetLastError();
}

}  // namespace wcc
