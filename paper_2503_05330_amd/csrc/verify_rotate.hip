// csd — rotary positions on queries and keys, alone and with the write of keys and values to the cache.
//
// A workgroup has eight tokens: their pairs' turns are worked out once, in LDS, and serve all heads.  What bounds it: memory.  8 x 4096 tokens of 40
// heads of 128: 131 us, 5.1 TB/s, what a copy reaches; sixteen tokens 4.3 us, launch and round trips.  With the write, 64 x 16 x 9
// tokens of 32 + 8 + 8 heads, to 8 bits: 47 us of 66 with their reading, 3.85 TB/s.  One launch instead of two saves keys a write and a read, and
// the launch.  Of queries a thread holds both eights of eight pairs (as keys are, an eight at a time with its pairs' others read beside: 69.5; queries
// before keys: 67.4).  (Asking for the next values before one is turned: 3 us more; six waves a SIMD, by spilling: 30 more; the banks'
// conflicts that the turns' reads have, 15 .. 44 % of LDS's cycles, taken away, sines of a shorter series, workgroups of half the heads: the same.)
#include <cmath>

#include "csd_cache.cuh"
#include "csd_rotate.cuh"

namespace csd {
namespace verify {
namespace {

constexpr int kRotateThreads = 64 * kMoveWaves;

struct RotateArgs {
  csd_rotary how;
  csd_heads x, out;
  const int32_t* positions;
  int64_t tokens;
  int32_t heads, dim, per;               // per: heads of a workgroup
};

// Rotates heads head0 .. head0 + heads - 1 of `here` tokens.  A thread takes sixteen values of a token's head at a time, both eights of eight pairs
// (or, behind them, two eights to be copied): two reads and two writes of 16 bytes, which the threads of a head and of the next ones do
// side by side.  from(token), to(token): where a token's heads lie.
template <class T, class From, class To>
__device__ inline void rotate_heads(const csd_rotary& how, Turn* turns, int32_t here, int32_t head0, int32_t heads, int32_t dim, int64_t from_head, int64_t to_head,
                                    From from, To to) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  const int32_t pairs = how.dim / 2, turning = how.dim / 16, units = turning + (dim - how.dim + 15) / 16, all = here * heads * units;
  constexpr int kAhead = 2;                              // (4: 133 us for 131 with 8 x 4096 tokens of 40 heads of 128; a copy of as much takes 130)
  for (int32_t x0 = threadIdx.x; x0 < all; x0 += kAhead * kRotateThreads) {
    Eight u[kAhead], v[kAhead];
    int32_t d[kAhead], e[kAhead], token[kAhead], head[kAhead];           // where the two eights lie; e < 0: there is no second
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t x = x0 + s * kRotateThreads < all ? x0 + s * kRotateThreads : x0;
      const int32_t row = x / units, unit = x - row * units;
      token[s] = row / heads;
      head[s] = head0 + row - token[s] * heads;
      if (unit < turning) {
        d[s] = how.interleaved ? 16 * unit : 8 * unit;
        e[s] = how.interleaved ? d[s] + 8 : d[s] + pairs;
      } else {
        d[s] = how.dim + 16 * (unit - turning);
        e[s] = d[s] + 8 < dim ? d[s] + 8 : -1;
      }
      const Value* const x_of = from(token[s]) + head[s] * from_head;
      u[s] = *reinterpret_cast<const Eight*>(x_of + d[s]);
      v[s] = *reinterpret_cast<const Eight*>(x_of + (e[s] < 0 ? d[s] : e[s]));
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if (x0 + s * kRotateThreads >= all) break;
      Value* const out = to(token[s]) + head[s] * to_head;
      Eight y = u[s], z = v[s];
      if (d[s] < how.dim) {
        const Turns own(turns, token[s], pairs);
        if (how.interleaved) {
          y = turned_eight<T>(u[s], v[s], d[s], how, own);
          z = turned_eight<T>(v[s], u[s], e[s], how, own);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i) {                  // a pair's turn, read once for both
            const Turn t = own[d[s] + i];
            y[i] = (Value)turned((float)u[s][i], (float)v[s][i], t);
            z[i] = (Value)turned((float)v[s][i], -(float)u[s][i], t);
          }
        }
      }
      *reinterpret_cast<Eight*>(out + d[s]) = y;
      if (e[s] >= 0) *reinterpret_cast<Eight*>(out + e[s]) = z;
    }
  }
}

// the turns of a workgroup's tokens
__device__ inline void make_turns(const csd_rotary& how, const int32_t* positions, int32_t here, Turn* turns) {
  const int32_t pairs = how.dim / 2;
  for (int32_t x = threadIdx.x; x < here * pairs; x += kRotateThreads) {
    const int32_t token = x / pairs;
    Turns(turns, token, pairs)[x - token * pairs] = turn_of(how, positions[token], x - token * pairs);
  }
}

// eight tokens, `per` heads
template <class T>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a) {
  typedef typename T::One Value;
  extern __shared__ Turn turns[];
  const int64_t first = (int64_t)blockIdx.x * kGroup;
  const int32_t here = a.tokens - first < kGroup ? (int32_t)(a.tokens - first) : kGroup;
  make_turns(a.how, a.positions + first, here, turns);
  __syncthreads();
  const int32_t head0 = blockIdx.y * a.per, heads = a.heads - head0 < a.per ? a.heads - head0 : a.per;
  const Value* const x = static_cast<const Value*>(a.x.data) + first * a.x.token_stride;
  Value* const out = static_cast<Value*>(const_cast<void*>(a.out.data)) + first * a.out.token_stride;
  rotate_heads<T>(a.how, turns, here, head0, heads, a.dim, a.x.head_stride, a.out.head_stride,
                  [&](int32_t token) { return x + token * a.x.token_stride; }, [&](int32_t token) { return out + token * a.out.token_stride; });
}

struct PlaceArgs {
  csd_rotary how;
  csd_heads q;
  const int32_t* positions;
  void* q_out;
  MoveArgs move;                         // keys and values
  int64_t tokens;                        // of all paths
  int32_t H, per;                        // per: jobs of a workgroup.  A job: a kv head's keys and values, or a query head
};

// Eight tokens, of one path or of several.  Keys and values: a wave takes a kv head's at a time, eight lanes a token; then queries, as rotate_kernel().
template <class T, int D, bool FP8>
__global__ __launch_bounds__(kRotateThreads) void place_kernel(PlaceArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  __shared__ Turn turns[Turns::size(kGroup, D / 2)];
  __shared__ int64_t queries[kGroup];                    // where the tokens' begin
  const int wave = threadIdx.x >> 6, nth = (threadIdx.x & 63) / 8;
  const int64_t first = (int64_t)blockIdx.x * kGroup;
  const int32_t here = a.tokens - first < kGroup ? (int32_t)(a.tokens - first) : kGroup;
  const int32_t pairs = a.how.dim / 2;
  const MoveArgs& m = a.move;
  const bool there = nth < here;
  const int64_t token = there ? first + nth : first, row = token / m.n;
  const int32_t t = (int32_t)(token - row * m.n);
  int32_t count = m.counts ? m.counts[row] : m.n;
  count = count > m.n ? m.n : count;
  const int64_t pos = (int64_t)(m.start ? m.start[row] : 0) + t;
  const bool asked = there && t < count, live = asked && pos >= 0 && pos < m.held.cap;
  if (wave == 0 && (threadIdx.x & 7) == 0) queries[nth] = row * a.q.row_stride + t * a.q.token_stride;
  make_turns(a.how, a.positions + first, here, turns);
  if (wave == 0 && blockIdx.y == 0 && asked && !live) atomicOr(m.status, CSD_STATUS_CAPACITY);
  __syncthreads();
  const int32_t job0 = blockIdx.y * a.per, end = job0 + a.per < m.Hk + a.H ? job0 + a.per : m.Hk + a.H;
  for (int32_t head = job0 + wave; head < end && head < m.Hk; head += kMoveWaves) {
    const Value* const k_from = static_cast<const Value*>(m.k.data) + row * m.k.row_stride + t * m.k.token_stride + head * m.k.head_stride;
    const Value* const v_from = static_cast<const Value*>(m.v.data) + row * m.v.row_stride + t * m.v.token_stride + head * m.v.head_stride;
    Eight k[P::kPieces], v[P::kPieces], other[P::kPieces];
#pragma unroll
    for (int i = 0; i < P::kPieces; ++i) {
      const int d = P::d(i), e = d < pairs ? d + pairs : d - pairs;
      k[i] = v[i] = other[i] = Eight{};
      if (live && d < D) {
        k[i] = *reinterpret_cast<const Eight*>(k_from + d);
        v[i] = *reinterpret_cast<const Eight*>(v_from + d);
        if (d < a.how.dim && !a.how.interleaved) other[i] = *reinterpret_cast<const Eight*>(k_from + e);
      }
    }
#pragma unroll
    for (int i = 0; i < P::kPieces; ++i)
      if (live && P::d(i) < a.how.dim) k[i] = turned_eight<T>(k[i], other[i], P::d(i), a.how, Turns(turns, nth, pairs));
    hold<T, D, FP8>(m.held, m.held.first(row, head, m.Hk) + (live ? pos / kBlock : 0), (int)pos & (kBlock - 1), live, k, v);
  }
  const int32_t head0 = job0 < m.Hk ? 0 : job0 - m.Hk, heads = end - m.Hk - head0;
  if (heads > 0)
    rotate_heads<T>(a.how, turns, here, head0, heads, D, a.q.head_stride, D, [&](int32_t x) { return static_cast<const Value*>(a.q.data) + queries[x]; },
                    [&](int32_t x) { return static_cast<Value*>(a.q_out) + (first + x) * a.H * D; });
}

// Workgroups share a group's heads where there are few groups: until there are so many workgroups, or each wave has one.  (1024 and 2048: the
// same; 4096, which 1152 groups of 48 heads reach with twelve a workgroup, 89 us for 70 with their reading.)
constexpr int64_t kLeastGroups = 512;
int32_t heads_of_group(int64_t groups, int32_t heads) {
  const int64_t parts = (kLeastGroups + groups - 1) / groups, most = (heads + kMoveWaves - 1) / kMoveWaves, n = parts < most ? parts : most;
  return (int32_t)((heads + n - 1) / n);
}

bool misaligned(const void* p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

}  // namespace

int check_rotary(const csd_rotary* how, int32_t head_dim) {
  if (!how || !how->d_turns || misaligned(how->d_turns, 8) || how->dim < 16 || how->dim % 16 || how->dim > head_dim) return CSD_ERR_INVALID_ARG;
  if ((how->interleaved != 0 && how->interleaved != 1) || !std::isfinite(how->amplitude)) return CSD_ERR_INVALID_ARG;
  return CSD_OK;
}

void cache_write_rotated(const MoveArgs& move, const csd_rotary& how, const csd_heads& q, const int32_t* positions, int32_t H, void* q_out,
                         int32_t head_dim, bool f16, bool fp8, hipStream_t st) {
  const int64_t tokens = move.rows * move.n, groups = (tokens + kGroup - 1) / kGroup;
  const int32_t per = heads_of_group(groups, move.Hk + H);
  const PlaceArgs a{how, q, positions, q_out, move, tokens, H, per};
  const dim3 grid((uint32_t)groups, (uint32_t)((move.Hk + H + per - 1) / per));
  of_dim(head_dim, [&](auto dim) {
    constexpr int D = dim();
    auto* kernel = f16 ? (fp8 ? place_kernel<F16, D, true> : place_kernel<F16, D, false>)
                       : (fp8 ? place_kernel<BF16, D, true> : place_kernel<BF16, D, false>);
    kernel<<<grid, kRotateThreads, 0, st>>>(a);
  });
}

}  // namespace verify
}  // namespace csd

extern "C" {

int csd_rotary_turns(int32_t dim, double base, double factor, double original, double low, double high, double* out_turns) {
  if (dim < 16 || dim % 16 || dim > CSD_MAX_ROTATED_DIM || !out_turns || !std::isfinite(base) || !(base > 1) || !std::isfinite(factor) || !(factor > 0) ||
      !std::isfinite(original) || !(original >= 0) || !std::isfinite(low) || !std::isfinite(high) || !(high > low))
    return CSD_ERR_INVALID_ARG;
  for (int32_t i = 0; i < dim / 2; ++i) {
    const double turns = std::pow(base, -2.0 * i / dim) / 6.283185307179586476925;
    double keep = 0;
    if (original > 0) {
      keep = (original * turns - low) / (high - low);
      keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
    }
    out_turns[i] = turns * (keep + (1 - keep) / factor);
  }
  return CSD_OK;
}

int csd_rotate(const csd_rotary* rotary, const csd_heads* x, const int32_t* d_positions, int64_t tokens, int32_t heads, int32_t head_dim,
               int32_t type, const csd_heads* out, void* stream) {
  using namespace csd::verify;
  if (head_dim < 16 || head_dim % 8 || head_dim > CSD_MAX_ROTATED_DIM || check_rotary(rotary, head_dim) != CSD_OK) return CSD_ERR_INVALID_ARG;
  if (tokens < 0 || tokens > CSD_MAX_PACKED_TOKENS || heads <= 0 || heads > 2 * CSD_MAX_HEADS || (type != CSD_BF16 && type != CSD_F16)) return CSD_ERR_INVALID_ARG;
  for (const csd_heads* h : {x, out})
    if (!h || (tokens && !h->data) || misaligned(h->data, 16) || h->token_stride < 0 || h->head_stride < 0 || h->token_stride % 8 || h->head_stride % 8)
      return CSD_ERR_INVALID_ARG;
  if (tokens && (!d_positions || misaligned(d_positions, 4))) return CSD_ERR_INVALID_ARG;
  if (x->data == out->data && ((tokens > 1 && x->token_stride != out->token_stride) || (heads > 1 && x->head_stride != out->head_stride))) return CSD_ERR_INVALID_ARG;
  if (tokens == 0) return CSD_OK;
  // no two values of out at one place: one of the two axes lies within a step of the other
  const auto within = [&](int64_t few, int64_t near, int64_t many, int64_t far) {
    return (few == 1 || near >= head_dim) && (many == 1 || far >= (few - 1) * near + head_dim);
  };
  if (!within(heads, out->head_stride, tokens, out->token_stride) && !within(tokens, out->token_stride, heads, out->head_stride)) return CSD_ERR_INVALID_ARG;
  const int64_t groups = (tokens + kGroup - 1) / kGroup;
  const int32_t per = heads_of_group(groups, heads);
  const RotateArgs a{*rotary, *x, *out, d_positions, tokens, heads, head_dim, per};
  const dim3 grid((uint32_t)groups, (uint32_t)((heads + per - 1) / per));
  auto* kernel = type == CSD_F16 ? rotate_kernel<F16> : rotate_kernel<BF16>;
  kernel<<<grid, kRotateThreads, Turns::size(kGroup, rotary->dim / 2) * sizeof(Turn), static_cast<hipStream_t>(stream)>>>(a);
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? CSD_OK : csd::hip_fail(e, "csd_rotate");
}

}  // extern "C"
