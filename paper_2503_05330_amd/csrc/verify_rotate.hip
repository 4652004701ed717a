// csd — rotary positions on queries and keys, alone and with the write of keys and values to the cache.
//
// A workgroup has eight tokens: their pairs' turns are worked out once, in LDS, and serve all heads.  What bounds it: memory.  8 x 4096 tokens of 40
// heads of 128: 131 us, 5.1 TB/s, what a copy reaches; sixteen tokens 4.3 us, launch and round trips.  With the write, 64 x 16 x 9
// tokens of 32 + 8 + 8 heads, to 8 bits: 40 .. 47 us, 3.8 .. 4.5 TB/s.  One launch instead of two saves keys a write and a read, and
// the launch.  (Asking for the next job's values before one is turned: 45 us for 42; six waves a SIMD, by spilling: 69; banks'
// conflicts of the turns' reads taken away, sines of a shorter series, workgroups of half the heads: the same.)
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

// Eight tokens of `per` heads; a thread takes sixteen values of a token's head at a time, both eights of eight pairs (or, behind them, two
// eights to be copied): two reads and two writes of 16 bytes, which the threads of a head and of the next ones do side by side.
template <class T>
__global__ __launch_bounds__(kRotateThreads) void rotate_kernel(RotateArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  extern __shared__ Turn turns[];
  const int64_t first = (int64_t)blockIdx.x * kGroup;
  const int32_t here = a.tokens - first < kGroup ? (int32_t)(a.tokens - first) : kGroup;
  const int32_t pairs = a.how.dim / 2;
  for (int32_t x = threadIdx.x; x < here * pairs; x += kRotateThreads) {
    const int32_t token = x / pairs;
    Turns(turns, token, pairs)[x - token * pairs] = turn_of(a.how, a.positions[first + token], x - token * pairs);
  }
  __syncthreads();
  const int32_t head0 = blockIdx.y * a.per, heads = a.heads - head0 < a.per ? a.heads - head0 : a.per;
  const int32_t turning = a.how.dim / 16, units = turning + (a.dim - a.how.dim + 15) / 16, all = here * heads * units;
  constexpr int kAhead = 2;                              // (4: 133 us for 131 with 8 x 4096 tokens of 40 heads of 128; a copy of as much takes 130)
  for (int32_t x0 = threadIdx.x; x0 < all; x0 += kAhead * kRotateThreads) {
    Eight u[kAhead], v[kAhead];
    int64_t to[kAhead];
    int32_t d[kAhead], e[kAhead], token[kAhead];         // where the two eights lie; e < 0: there is no second
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      const int32_t x = x0 + s * kRotateThreads < all ? x0 + s * kRotateThreads : x0;
      const int32_t row = x / units, unit = x - row * units;
      token[s] = row / heads;
      const int32_t head = head0 + row - token[s] * heads;
      if (unit < turning) {
        d[s] = a.how.interleaved ? 16 * unit : 8 * unit;
        e[s] = a.how.interleaved ? d[s] + 8 : d[s] + pairs;
      } else {
        d[s] = a.how.dim + 16 * (unit - turning);
        e[s] = d[s] + 8 < a.dim ? d[s] + 8 : -1;
      }
      const Value* const from = static_cast<const Value*>(a.x.data) + (first + token[s]) * a.x.token_stride + head * a.x.head_stride;
      to[s] = (first + token[s]) * a.out.token_stride + head * a.out.head_stride;
      u[s] = *reinterpret_cast<const Eight*>(from + d[s]);
      v[s] = *reinterpret_cast<const Eight*>(from + (e[s] < 0 ? d[s] : e[s]));
    }
#pragma unroll
    for (int s = 0; s < kAhead; ++s) {
      if (x0 + s * kRotateThreads >= all) break;
      Value* const out = static_cast<Value*>(const_cast<void*>(a.out.data)) + to[s];
      Eight y = u[s], z = v[s];
      if (d[s] < a.how.dim) {
        const Turns own(turns, token[s], pairs);
        if (a.how.interleaved) {
          y = turned_eight<T>(u[s], v[s], d[s], a.how, own);
          z = turned_eight<T>(v[s], u[s], e[s], a.how, own);
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

struct PlaceArgs {
  csd_rotary how;
  csd_heads q;
  const int32_t* positions;
  void* q_out;
  MoveArgs move;                         // keys and values
  int64_t tokens;                        // of all paths
  int32_t H, per;                        // per: jobs of a workgroup.  A job: a kv head's keys and values, or a query head
};

// Eight tokens, of one path or of several; a wave takes a job of theirs at a time, eight lanes a token.
template <class T, int D, bool FP8>
__global__ __launch_bounds__(kRotateThreads) void place_kernel(PlaceArgs a) {
  typedef typename T::Eight Eight;
  typedef typename T::One Value;
  typedef Pieces<D> P;
  __shared__ Turn turns[Turns::size(kGroup, D / 2)];
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
  for (int32_t x = threadIdx.x; x < here * pairs; x += kRotateThreads) {
    const int32_t of = x / pairs;
    Turns(turns, of, pairs)[x - of * pairs] = turn_of(a.how, a.positions[first + of], x - of * pairs);
  }
  if (wave == 0 && blockIdx.y == 0 && asked && !live) atomicOr(m.status, CSD_STATUS_CAPACITY);
  __syncthreads();
  const auto load = [&](const Value* from, Eight (&x)[P::kPieces], bool wanted) {
#pragma unroll
    for (int i = 0; i < P::kPieces; ++i) {
      x[i] = Eight{};
      if (wanted && P::d(i) < D) x[i] = *reinterpret_cast<const Eight*>(from + P::d(i));
    }
  };
  const auto rotate = [&](const Value* from, Eight (&x)[P::kPieces], bool wanted) {
    Eight other[P::kPieces];
#pragma unroll
    for (int i = 0; i < P::kPieces; ++i) {
      const int d = P::d(i), e = d < pairs ? d + pairs : d - pairs;
      other[i] = Eight{};
      if (wanted && d < a.how.dim && !a.how.interleaved) other[i] = *reinterpret_cast<const Eight*>(from + e);
    }
#pragma unroll
    for (int i = 0; i < P::kPieces; ++i)
      if (wanted && P::d(i) < a.how.dim) x[i] = turned_eight<T>(x[i], other[i], P::d(i), a.how, Turns(turns, nth, pairs));
  };
  const int32_t job0 = blockIdx.y * a.per, end = job0 + a.per < m.Hk + a.H ? job0 + a.per : m.Hk + a.H;
  for (int32_t job = job0 + wave; job < end; job += kMoveWaves) {
    Eight x[P::kPieces];
    if (job < m.Hk) {
      Eight v[P::kPieces];
      const Value* const k_from = static_cast<const Value*>(m.k.data) + row * m.k.row_stride + t * m.k.token_stride + job * m.k.head_stride;
      load(k_from, x, live);
      load(static_cast<const Value*>(m.v.data) + row * m.v.row_stride + t * m.v.token_stride + job * m.v.head_stride, v, live);
      rotate(k_from, x, live);
      hold<T, D, FP8>(m.held, m.held.first(row, job, m.Hk) + (live ? pos / kBlock : 0), (int)pos & (kBlock - 1), live, x, v);
    } else {
      const int32_t head = job - m.Hk;
      const Value* const from = static_cast<const Value*>(a.q.data) + row * a.q.row_stride + t * a.q.token_stride + head * a.q.head_stride;
      load(from, x, there);
      rotate(from, x, there);
      if (!there) continue;
#pragma unroll
      for (int i = 0; i < P::kPieces; ++i)
        if (P::d(i) < D) *reinterpret_cast<Eight*>(static_cast<Value*>(a.q_out) + (token * a.H + head) * D + P::d(i)) = x[i];
    }
  }
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
