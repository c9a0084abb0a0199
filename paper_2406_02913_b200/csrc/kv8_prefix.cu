// Attention over the 8-bit paged cache for sequences that continue shared prompts.
//
// A row's softmax over its positions is joined from parts with their own maxima and sums: the whole pages that its group
// shares, where the rows of all the group's sequences are taken together (so a shared code is read once for 8 to 256 rows of several
// sequences, and prompts of a few rows each fill tensor-core tiles), and the rest of its sequence's positions.  Both are passes
// of the attention kernels of kv8_attention.cu and kv8_attention_tc.cu that leave sums, maxima and sums of weights unfinished,
// each cut into shares of the positions that fill the SMs: fp32 sums of weights times codes with their (maximum, sum of weights).  The
// sequences' pass starts once the groups' one runs and waits for nothing of it, but for one block whose end orders the two; a last kernel
// joins a row's shares in their order.
// What bounds it: bytes of codes (shared ones once per group, at 6.4 TB/s) plus, with one step of a conversation at a time, a fixed cost of
// about 20 us: three dependent launches, the first trip to pages through the table, writing and joining the shares.  Measured (bf16, 32 heads
// over 8 of 128, one new token each, in a replayed graph): 64 sequences on one prompt of 8192 with up to 512 positions of their own 36 us
// (every sequence by itself, as szo_attention_kv8 reads it, 136); 8 sequences on one of 65536 60 us (136).
#include <cmath>

#include "kv8_prefix.cuh"

namespace szo {
namespace kv8 {

namespace {

// What the passes read of the groups (block g) and of the sequences outside of every group (the last block).  A group with a
// sequence whose description does not fit shares nothing: its rows could not be told apart; none does where seqs does not ascend.
__global__ void __launch_bounds__(256) kv8_groups_kernel(View V, Prefix P, int4* __restrict__ groups, int32_t* __restrict__ shared, int32_t* __restrict__ pos) {
  chain_release();
  const int g = blockIdx.x, n = P.n_groups;
  const bool last = g == n;
  int first = 0, end = V.batch, len = 0, lo = 0, hi = n > 0 ? V.batch : 0;        // this group's sequences and positions; those of all groups
  bool ok = true;
  if (P.seqs != nullptr) {
    lo = P.seqs[0];
    hi = P.seqs[n];
    first = P.seqs[last ? 0 : g];
    end = P.seqs[last ? 0 : g + 1];
    for (int i = threadIdx.x; i < n; i += blockDim.x) ok = ok && P.seqs[i] <= P.seqs[i + 1];
  }
  if (!last) len = P.len[g];
  const bool ascending = __syncthreads_and(ok);
  if (last) {
    for (int b = threadIdx.x; b < V.batch; b += blockDim.x)
      if (!ascending || b < lo || b >= hi) shared[b] = 0;
    if (!ascending && threadIdx.x == 0) atomicExch(V.status, static_cast<int32_t>(SZO_ERR_SHAPE));
    return;
  }
  const bool fits = first >= 0 && end >= first && end <= V.batch && end - first <= P.max_seqs && len >= 0 &&
                    len <= static_cast<int64_t>(V.max_pages) << V.page_shift;
  if (!fits && threadIdx.x == 0) atomicExch(V.status, static_cast<int32_t>(SZO_ERR_SHAPE));
  len = ascending && fits ? len >> V.page_shift << V.page_shift : 0;
  first = max(first, 0);
  end = min(end, V.batch);
  // the pages are read through the table of the longest sequence, the first of several, and as far as it goes: entries that no position
  // needs are not read
  __shared__ unsigned long long longest;
  if (threadIdx.x == 0) longest = 0;
  __syncthreads();
  ok = true;
  for (int b = first + threadIdx.x; b < end; b += blockDim.x) {
    Seq q;
    ok = read_seq(V, b, &q) && ok;
    atomicMax(&longest, static_cast<unsigned long long>(static_cast<unsigned>(q.len)) << 32 | (0x7fffffffu - static_cast<unsigned>(b)));
  }
  if (!__syncthreads_and(ok) || first >= end) len = 0;
  len = min(len, (static_cast<int>(longest >> 32) + (1 << V.page_shift) - 1) >> V.page_shift << V.page_shift);
  const int owner = 0x7fffffff - static_cast<int>(longest & 0x7fffffffu);
  if (threadIdx.x == 0) {
    const int row0 = len == 0 ? 0 : V.start != nullptr ? V.start[first] : first * V.max_new;
    const int rows = len == 0 ? 0 : V.start != nullptr ? V.start[end] - row0 : (end - first) * V.max_new;
    groups[g] = make_int4(row0, rows, len, owner);
  }
  if (!ascending) return;
  const int lane = threadIdx.x & 31;
  for (int b = first + threadIdx.x / 32; b < end; b += blockDim.x / 32) {
    if (lane == 0) shared[b] = len;
    if (len == 0) continue;
    Seq q;
    read_seq(V, b, &q);
    for (int i = lane; i < q.n; i += 32) pos[q.row0 + i] = q.len - q.n + i;
  }
}

// Joins the shares of the rows of all sequences: HD / 4 threads per row and head, four teams of them, every team taking every fourth share;
// teams joined in order.  Grid (token of a sequence, heads)
constexpr int kJoinThreads = 256, kTeams = 4;
template <typename T, int HD>
__global__ void __launch_bounds__(kJoinThreads) kv8_shares_kernel(View V, Part part, int n_prefix, int n_own, T* __restrict__ o, int64_t o_stride, int H) {
  constexpr int kLanes = HD / 4, kHeads = kJoinThreads / kLanes / kTeams, kAhead = 4;
  struct Sum {
    float4 x;
    float m, l;
  };
  __shared__ Sum teams[kTeams][kHeads][kLanes];
  const int b = blockIdx.x / V.max_new, i = blockIdx.x % V.max_new;
  const Seq s = load_seq(V, b);                                   // (before the wait: see the passes)
  const int lane = threadIdx.x % kLanes, hd = threadIdx.x / kLanes % kHeads, team = threadIdx.x / kLanes / kHeads;
  const int head = blockIdx.y * kHeads + hd;
  const bool there = i < s.n && head < H;
  const int from = there && __ldcg(part.shared + b) > 0 ? 0 : n_prefix, to = there ? n_prefix + n_own : 0;
  chain_wait();
  const int64_t at = (s.row0 + i) * H + head;
  Sum a{make_float4(0.f, 0.f, 0.f, 0.f), -INFINITY, 0.f};
  auto add = [&](float m, float l, const float4& x) {
    const float top = fmaxf(a.m, m), ref = top == -INFINITY ? 0.f : top, f0 = ex2(a.m - ref), f1 = ex2(m - ref);
    a.x = make_float4(fmaf(f1, x.x, f0 * a.x.x), fmaf(f1, x.y, f0 * a.x.y), fmaf(f1, x.z, f0 * a.x.z), fmaf(f1, x.w, f0 * a.x.w));
    a.l = fmaf(f1, l, f0 * a.l);
    a.m = top;
  };
  for (int k0 = from + team; k0 < to; k0 += kAhead * kTeams) {
    float2 st[kAhead];
    float4 x[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t p = (k0 + k * kTeams < to ? k0 + k * kTeams : k0) * part.row_heads + at;
      st[k] = __ldcg(part.stats + p);
      x[k] = __ldcg(reinterpret_cast<const float4*>(part.sums + p * HD + 4 * lane));
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (k0 + k * kTeams < to) add(st[k].x, st[k].y, x[k]);
  }
  teams[team][hd][lane] = a;
  __syncthreads();
  if (team != 0 || !there) return;
#pragma unroll
  for (int k = 1; k < kTeams; ++k) {
    const Sum& y = teams[k][hd][lane];
    add(y.m, y.l, y.x);
  }
  const float inv = a.l == 0.f ? 1.f : 1.f / a.l;                 // nothing attended to: sums of 0
  struct alignas(4 * sizeof(T)) Four { T x[4]; };
  *reinterpret_cast<Four*>(o + (s.row0 + i) * o_stride + static_cast<int64_t>(head) * HD + 4 * lane) =
      Four{{narrow<T>(a.x.x * inv), narrow<T>(a.x.y * inv), narrow<T>(a.x.z * inv), narrow<T>(a.x.w * inv)}};
}

struct Pass {
  bool many;                   // the tensor-core kernel for many rows
  int max_rows, shares;
};
struct SharePlan {
  bool direct;                 // a sequence's own rows fill tiles: nothing to gain, the attention kernels as they are
  Pass prefix, own;
  size_t groups, shared, pos, sums, stats, total;
  int64_t row_heads;
};
// How a pass's positions are cut.  The lengths are on the device, so the rules go by the number of items (owner, head, row tile) and by what
// the page table could hold.
// Shared positions: the cost of n shares, in steps of 128 positions (many rows: 2.4 us of an SM), is that of a share where all of them
// fit the SMs at once (many rows a block per SM, few two), or else of the rounds, between whole ones (equal lengths) and parts, of shares with
// about 4 steps of setup and epilogue; and a little for every share, which is written and joined and takes an SM from the sequences' pass.  Measured, 8
// heads of 128 (groups x sequences on positions: us by shares), many rows: 1 x 64 on 8192: 9 41, 11 36, 12 38, 18 43; 1 x 64 on 16384: 10 54,
// 16 45; 3 x 16 of 4 rows on 8192: 3 76, 5 56; 8 x 16 on 8192: 1 149, 2 87, 3 103; 16 x 16 on 4096: 1 94,
// 2 105; 10 x 6 of 2 rows on 8192: 1 148, 2 129, 3 107; 20 x 8 of 2 rows on 4096: 1 138, 2 132, 3 135.  Few: 1 x 8 on 65536: 30 68,
// 37 62; 10 x 4 on 8192: 1 76, 2 53, 3 43, 4 52; 20 x 4 of 2 rows on 4096: 1 101, 2 94, 3 80, 4 89; 40 x 4 on 2048: 1 57, 2 62.
// A sequence's own: the SMs once, but up to 4 shares where the kernel for few rows holds that many blocks on the SMs (16 sequences of 4096
// positions of their own: 1 share 40 us, 2 31, 4 29; 32 of 2048: 1 39, 2 35, 3 37; 64 of 512 on 8192: 1 36, 2 40).
Pass make_pass(const View& V, int64_t max_rows, int64_t owners, int H, bool wide_type, bool prefix) {
  constexpr int kSms = 148, kMost = 64;
  const int64_t rows = max_rows * (H / V.hkv), places = static_cast<int64_t>(V.max_pages) << V.page_shift;
  Pass p{!wide_type && rows > 32, static_cast<int>(max_rows), 1};
  const int64_t tile = p.many ? 256 : rows <= 8 ? 8 : prefix && !wide_type && rows > 16 ? kPrefixRows : 16, items = owners * V.hkv * ceil_div(rows, tile);
  const int64_t least = p.many ? 256 : 128;                       // (2 steps of 128 at least, or units of 32 for each of 4 warps)
  double best = 1e30;
  for (int n = 1; n <= kMost && (n == 1 || places >= least * n); ++n) {
    if (prefix) {
      const double steps = static_cast<double>(places) / 128 / n, rounds = static_cast<double>(items) * n / (p.many ? kSms : 2 * kSms);
      const double time = rounds <= 1 ? steps : (0.5 * (std::ceil(rounds) + rounds) + 0.15) * (steps + 4);
      const double cost = time + (!p.many ? 0.01 : rounds <= 1 ? 0.07 : 0.03) * static_cast<double>(items) * n;
      if (cost < best) {
        best = cost;
        p.shares = n;
      }
    } else if (items * n <= kSms || (!p.many && n <= 4 && items * n <= 512)) {
      p.shares = n;
    }
  }
  return p;
}
// Up to this much to read, if every sequence reads all that its table could hold, the sequences' own attention is as fast: it is one
// launch, and shared pages come from L2
constexpr int64_t kDirectBytes = int64_t(96) << 20;
// What a block's time per position is for `rows` rows of a key/value head (1: 8 rows, 26 ps with all SMs busy), in the kernel that takes them
double row_units(int64_t rows, bool wide_type, bool prefix) {
  if (rows <= 8) return 1.0;
  if (!wide_type && rows > 32) return 4.9 * static_cast<double>(ceil_div(rows, 256));
  return !wide_type && prefix && rows > 16 ? 3.4 : 1.6 * static_cast<double>(ceil_div(rows, 16));
}
SharePlan share_plan(const View& V, const Prefix& P, int H, int hd, bool wide_type) {
  SharePlan p = {};
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += round_up(bytes, 256);
    return from;
  };
  p.groups = take(static_cast<size_t>(P.n_groups) * sizeof(int4));
  p.shared = take(static_cast<size_t>(V.batch) * sizeof(int32_t));
  p.pos = take(static_cast<size_t>(V.rows) * sizeof(int32_t));
  p.direct = P.n_groups == 0 || P.max_seqs == 0 || static_cast<int64_t>(V.max_new) * (H / V.hkv) >= 256 ||
             (static_cast<int64_t>(V.batch) * V.max_pages << V.page_shift) * V.hkv * hd * 2 <= kDirectBytes;
  // Where the prompts fill the SMs, blocks that read the same pages run close together and find them in L2: then rows taken together have to be
  // cheaper than apart (us together / apart, 8 heads: 40 prompts x 4 sequences x 2 tokens on 2048 97 / 71, 20 x 4 x 2 on 4096 81 / 68, 30 x 2 x 4 on
  // 8192 187 / 163; 20 x 4 x 1 on 4096 54 / 67; with fewer prompts 4 x 4 x 2 on 16384 59 / 68)
  if (static_cast<int64_t>(P.n_groups) * V.hkv >= 148) {
    const int64_t own = static_cast<int64_t>(V.max_new) * (H / V.hkv);
    p.direct = p.direct || row_units(P.max_seqs * own, wide_type, true) >= 0.75 * P.max_seqs * row_units(own, wide_type, false);
  }
  if (!p.direct) {
    const int64_t most = static_cast<int64_t>(P.max_seqs) * V.max_new;
    p.prefix = make_pass(V, most < V.rows ? most : V.rows, P.n_groups, H, wide_type, true);
    p.own = make_pass(V, V.max_new, V.batch, H, wide_type, false);
    p.row_heads = V.rows * H;
    const size_t n = static_cast<size_t>(p.prefix.shares + p.own.shares) * p.row_heads;
    p.sums = take(n * hd * sizeof(float));
    p.stats = take(n * sizeof(float2));
  }
  p.total = at;
  return p;
}

template <typename T, int HD>
szo_status run_pass(const View& V, const Rows& A, const Part& part, const Pass& pass, cudaStream_t st) {
  if constexpr (sizeof(T) == 2)
    if (pass.many) return launch_part_tc<T, HD>(V, A, part, pass.shares, st);
  return launch_part<T, HD>(V, A, part, pass.shares, st);
}
template <typename T, int HD>
szo_status launch_shares(const View& V, const Prefix& P, const Rows& A, const SharePlan& p, const Part& base, cudaStream_t st) {
  Part part = base;
  part.prefix = 1;
  part.items = P.n_groups;
  part.max_rows = p.prefix.max_rows;
  SZO_TRY((run_pass<T, HD>(V, A, part, p.prefix, st)));
  Part own = base;
  own.items = V.batch;
  own.max_rows = V.max_new;
  own.sums += p.prefix.shares * base.row_heads * HD;
  own.stats += p.prefix.shares * base.row_heads;
  SZO_TRY((run_pass<T, HD>(V, A, own, p.own, st)));
  const dim3 grid(static_cast<unsigned>(static_cast<int64_t>(V.batch) * V.max_new), static_cast<unsigned>(ceil_div(A.H, kJoinThreads / (HD / 4) / kTeams)));
  SZO_CHECK_CUDA(launch_maybe_chained(kv8_shares_kernel<T, HD>, grid, dim3(kJoinThreads), 0, st, true, V, base, p.prefix.shares, p.own.shares,
                                      static_cast<T*>(A.o), A.o_stride, A.H));
  count_launch();
  return SZO_OK;
}

szo_status make_prefix(const szo_kv8_prefix* p, const View& V, Prefix* out) {
  SZO_REQUIRE(p != nullptr, SZO_ERR_INVALID_ARG, "NULL prefix");
  SZO_REQUIRE(p->n_groups >= 0 && p->max_seqs >= 0, SZO_ERR_SHAPE, "negative n_groups or max_seqs");
  SZO_REQUIRE(p->n_groups == 0 || p->len != nullptr, SZO_ERR_INVALID_ARG, "NULL len");
  SZO_REQUIRE(p->seqs != nullptr || p->n_groups <= 1, SZO_ERR_SHAPE, "without seqs there is one group");
  SZO_REQUIRE(aligned16(p->len) && aligned16(p->seqs), SZO_ERR_ALIGNMENT, "buffers must be 16-byte aligned");
  *out = Prefix{p->len, p->seqs, p->n_groups, p->seqs == nullptr ? V.batch : p->max_seqs};
  return SZO_OK;
}

}  // namespace
}  // namespace kv8
}  // namespace szo

using namespace szo;

extern "C" {

size_t szo_attention_kv8_prefix_workspace_bytes(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const szo_kv8_prefix* prefix, int32_t n_heads) {
  kv8::View V;
  kv8::Prefix P;
  if (kv8::make_view(cache, batch, &V) != SZO_OK || kv8::make_prefix(prefix, V, &P) != SZO_OK || n_heads <= 0 || n_heads % cache->n_kv_heads != 0) return 0;
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return 0;
  // (for either kind of type: fp32 takes the kernel for few rows throughout, with other shares)
  const kv8::SharePlan a = kv8::share_plan(V, P, n_heads, cache->head_dim, false), b = kv8::share_plan(V, P, n_heads, cache->head_dim, true);
  const size_t apart = a.direct || b.direct ? szo_attention_kv8_workspace_bytes(cache, batch, n_heads) : 0;
  const size_t need_a = a.total + (a.direct ? apart : 0), need_b = b.total + (b.direct ? apart : 0);
  return need_a > need_b ? need_a : need_b;
}

szo_status szo_attention_kv8_prefix(const szo_kv8_cache* cache, const szo_kv8_batch* batch, const szo_kv8_prefix* prefix, const void* q, int64_t q_stride,
                                    void* o, int64_t o_stride, szo_dtype dtype, int32_t n_heads, float scale, void* workspace, size_t workspace_bytes,
                                    void* stream) {
  kv8::View V;
  kv8::Prefix P;
  SZO_TRY(kv8::make_view(cache, batch, &V));
  SZO_TRY(kv8::make_prefix(prefix, V, &P));
  SZO_TRY(kv8::check_rows(cache, q, q_stride, o, o_stride, dtype, n_heads, scale, workspace));
  if (V.batch == 0 || V.max_new == 0 || V.rows == 0) return SZO_OK;
  SZO_TRY(kv8::check_sizes(cache, V, n_heads));
  SZO_REQUIRE(V.rows * n_heads <= 0x7fffffff && static_cast<int64_t>(V.batch) * V.max_new <= 0x7fffffff, SZO_ERR_SHAPE, "too many rows and heads");
  const size_t need = szo_attention_kv8_prefix_workspace_bytes(cache, batch, prefix, n_heads);
  SZO_REQUIRE(need == 0 || (workspace && workspace_bytes >= need), SZO_ERR_WORKSPACE, "workspace: %zu bytes needed, %zu given", need,
              workspace ? workspace_bytes : size_t(0));
  SZO_TRY(kv8::set_status_word(&V));
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  auto* ws = static_cast<unsigned char*>(workspace);
  const kv8::SharePlan p = kv8::share_plan(V, P, n_heads, cache->head_dim, dtype == SZO_F32);
  kv8::Part part = {};
  part.groups = reinterpret_cast<const int4*>(ws + p.groups);
  part.shared = reinterpret_cast<const int32_t*>(ws + p.shared);
  part.pos = reinterpret_cast<const int32_t*>(ws + p.pos);
  part.sums = reinterpret_cast<float*>(ws + p.sums);
  part.stats = reinterpret_cast<float2*>(ws + p.stats);
  part.row_heads = p.row_heads;
  kv8::kv8_groups_kernel<<<static_cast<unsigned>(P.n_groups + 1), 256, 0, st>>>(V, P, reinterpret_cast<int4*>(ws + p.groups),
                                                                             reinterpret_cast<int32_t*>(ws + p.shared), reinterpret_cast<int32_t*>(ws + p.pos));
  count_launch();
  SZO_CHECK_LAUNCH("kv8_groups_kernel");
  if (p.direct)                                                   // (the groups' descriptions are still looked at)
    return szo_attention_kv8(cache, batch, q, q_stride, o, o_stride, dtype, n_heads, scale, ws + p.total, workspace_bytes - p.total, stream);
  const kv8::Rows A{q, o, q_stride, o_stride, n_heads, scale};
  const bool wide = cache->head_dim == 128;
  if (dtype == SZO_F32) return wide ? kv8::launch_shares<float, 128>(V, P, A, p, part, st) : kv8::launch_shares<float, 64>(V, P, A, p, part, st);
  if (dtype == SZO_BF16)
    return wide ? kv8::launch_shares<__nv_bfloat16, 128>(V, P, A, p, part, st) : kv8::launch_shares<__nv_bfloat16, 64>(V, P, A, p, part, st);
  return wide ? kv8::launch_shares<__half, 128>(V, P, A, p, part, st) : kv8::launch_shares<__half, 64>(V, P, A, p, part, st);
}

}  // extern "C"
