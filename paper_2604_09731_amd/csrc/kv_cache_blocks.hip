// kv_cache_extend and kv_cache_release: block tables and slot maps of a paged cache from its sequences' lengths, and pages back to
// the list of free ones, without the host learning a length.
//
// What a sequence needs and gives follows from its own numbers; where its rows, its new pages and its returned pages lie follows
// from sums over the sequences before it.  Every workgroup forms these sums for itself, 256 sequences at a time (a sequence a
// thread, the next ones' numbers requested meanwhile), keeps them in LDS, and takes its share of the rows that the 256 make:
// a row finds its sequence by eight steps of a search there.  So there is one launch, no workgroup waits for another, and no
// atomic decides who gets what: the results depend on the inputs alone.
// Bound by latency: the chain is a few memory round trips for each 256 sequences.  Kernel times: 64 sequences, 9 tokens each, extend 5.1
// us, release (window 4096, three sequences done) 2.8; 248 sequences with 48 prompts of up to 8192 tokens (192000 slots) 7.4 and 3.2.
#include "common.h"
#include "wave.h"

namespace {

constexpr int kWave = 64, kThreads = 256, kWaves = kThreads / kWave;

// Sum of v over the threads before this one, and (in *total) over all; `scratch` holds kWaves numbers.  Ends with a barrier.
__device__ inline int64_t sum_before(int64_t v, int lane, int wv, int64_t* scratch, int64_t* total) {
  int64_t mine;
  const int64_t in_wave = smart::wave_excl_scan(v, lane, &mine);
  if (lane == 0) scratch[wv] = mine;
  __syncthreads();
  int64_t before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const int64_t x = scratch[w];
    before += w < wv ? x : 0;
    all += x;
  }
  *total = all;
  return before + in_wave;
}

// The last of n ascending starts that is not above x (the first start is not above any x asked for).
__device__ inline int find(const int64_t* start, int n, int64_t x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct ExtendArgs {
  int32_t batch, block_size, max_blocks, num_blocks, free_cap;
  int64_t total_cap;
  const int32_t* len;
  const int32_t* new_tokens;
  const int32_t* held;
  const int32_t* free_blocks;
  const int32_t* free_count;
  int32_t* table;
  int32_t* cu;
  int64_t* slots;
  int32_t* new_len;
  int32_t* new_held;
  int32_t* new_count;
  int32_t* status;
};

__global__ __launch_bounds__(kThreads) void kv_extend_kernel(ExtendArgs a) {
  __shared__ int64_t s_row[kThreads], s_sum[2][kWaves];
  __shared__ int64_t s_block[kThreads];  // blocks that sequences before took
  __shared__ int32_t s_len[kThreads], s_held[kThreads];
  __shared__ bool s_served[kThreads];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid >> 6;
  const bool writes = blockIdx.x == 0;
  const int64_t free_count = min(max(a.free_count[0], 0), a.free_cap);
  int64_t rows = 0, wanted = 0;  // of the sequences so far (uniform)
  struct Numbers {
    int32_t len, fresh, held;
  };
  auto request = [&](int b) {
    Numbers n{0, 0, 0};
    if (b < a.batch) n = Numbers{a.len[b], a.new_tokens[b], a.held[b]};
    return n;
  };
  Numbers next = request(tid);
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid, n_here = min(kThreads, a.batch - b0);
    const Numbers x = next;
    if (b0 + kThreads < a.batch) next = request(b + kThreads);
    const bool valid = x.len >= 0 && x.fresh >= 0 && x.held >= 0 && x.held <= a.max_blocks && x.len <= (int64_t)x.held * a.block_size;
    const int64_t fresh = max(x.fresh, 0), end = (int64_t)x.len + fresh;
    int64_t chunk_rows, chunk_wanted;
    const int64_t row = rows + sum_before(fresh, lane, wv, s_sum[0], &chunk_rows);
    const bool room = valid && end <= (int64_t)a.max_blocks * a.block_size && (fresh == 0 || row + fresh <= a.total_cap);
    const int64_t want = room ? max((int64_t)0, (end + a.block_size - 1) / a.block_size - x.held) : 0;
    const int64_t before = wanted + sum_before(want, lane, wv, s_sum[1], &chunk_wanted);
    const bool served = room && (want == 0 || before + want <= free_count);
    // (Those that the list is too short for come behind all that it serves, so what was taken before is what was wanted before.)
    if (b < a.batch) {
      s_row[tid] = row;
      s_block[tid] = before;
      s_len[tid] = x.len;
      s_held[tid] = x.held;
      s_served[tid] = served;
      if (writes) {
        a.cu[b + 1] = (int32_t)min(row + fresh, a.total_cap);
        a.new_len[b] = served ? (int32_t)end : x.len;
        a.new_held[b] = x.held + (served ? (int32_t)want : 0);
        a.status[b] = served ? SMART_OK : (valid ? SMART_ECAP : SMART_EINVAL);
        if (before <= free_count && before + want > free_count) a.new_count[0] = (int32_t)(free_count - before);  // the first of those
      }
    }
    __syncthreads();  // the sequences are there
    const int64_t last = min(rows + chunk_rows, a.total_cap);
    for (int64_t r = rows + (int64_t)blockIdx.x * kThreads + tid; r < last; r += (int64_t)gridDim.x * kThreads) {
      const int i = find(s_row, n_here, r);
      int64_t slot = -1;
      if (s_served[i]) {
        const int pos = s_len[i] + (int)(r - s_row[i]), j = pos / a.block_size, in = pos - j * a.block_size;
        int32_t* entry = a.table + (int64_t)(b0 + i) * a.max_blocks + j;
        // (a new block's first token is a new token: its thread writes the block table's entry)
        const bool old = j < s_held[i];
        const int32_t id = old ? *entry : a.free_blocks[free_count - 1 - (s_block[i] + j - s_held[i])];
        if (!old && in == 0) *entry = id;
        if (id >= 0 && id < a.num_blocks) slot = (int64_t)id * a.block_size + in;
      }
      a.slots[r] = slot;
    }
    rows += chunk_rows;
    wanted += chunk_wanted;
    __syncthreads();  // everyone is done with the sequences
  }
  for (int64_t r = min(rows, a.total_cap) + (int64_t)blockIdx.x * kThreads + tid; r < a.total_cap; r += (int64_t)gridDim.x * kThreads)
    a.slots[r] = -1;
  if (writes && tid == 0) {
    a.cu[0] = 0;
    if (wanted <= free_count) a.new_count[0] = (int32_t)(free_count - wanted);
  }
}

struct ReleaseArgs {
  int32_t batch, block_size, max_blocks, free_cap, window, sink_blocks;
  const int32_t* len;
  const int32_t* held;
  const int32_t* released;
  const int32_t* finished;
  const int32_t* table;
  int32_t* free_blocks;
  const int32_t* free_count;
  int32_t* new_len;
  int32_t* new_held;
  int32_t* new_released;
  int32_t* new_count;
  int32_t* status;
};

__global__ __launch_bounds__(kThreads) void kv_release_kernel(ReleaseArgs a) {
  __shared__ int64_t s_start[kThreads], s_sum[kWaves];
  __shared__ int32_t s_head[kThreads], s_skip[kThreads];  // blocks from the table's front on, and the first block behind them
  __shared__ bool s_gives[kThreads];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wv = tid >> 6;
  const bool writes = blockIdx.x == 0;
  const int64_t free_count = min(max(a.free_count[0], 0), a.free_cap), room = a.free_cap - free_count;
  int64_t offered = 0;
  struct Numbers {
    int32_t len, held, released, done;
  };
  auto request = [&](int b) {
    Numbers n{0, 0, 0, 0};
    if (b < a.batch) n = Numbers{a.len[b], a.held[b], a.released[b], a.finished ? a.finished[b] : 0};
    return n;
  };
  Numbers next = request(tid);
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid, n_here = min(kThreads, a.batch - b0);
    const Numbers x = next;
    if (b0 + kThreads < a.batch) next = request(b + kThreads);
    const bool valid = x.len >= 0 && x.held >= 0 && x.held <= a.max_blocks && x.released >= 0 && x.released <= x.held &&
                       x.len <= (int64_t)x.held * a.block_size;
    const bool done = x.done != 0;
    const int32_t sink = min(x.held, a.sink_blocks), first = max(sink, x.released);
    // blocks whose last token lies before what the next token's window holds
    const int32_t left = a.window > 0 ? (int32_t)(max((int64_t)0, (int64_t)x.len - a.window + 1) / a.block_size) : 0;
    const int32_t end = done ? x.held : min(left, x.held);
    const int32_t tail = valid ? max(0, end - first) : 0, head = valid && done ? sink : 0;
    int64_t chunk_offered;
    const int64_t start = offered + sum_before((int64_t)head + tail, lane, wv, s_sum, &chunk_offered);
    const bool gives = valid && (head + tail == 0 || start + head + tail <= room);
    if (b < a.batch) {
      s_start[tid] = start;
      s_head[tid] = head;
      s_skip[tid] = first;
      s_gives[tid] = gives;
      if (writes) {
        a.new_len[b] = gives && done ? 0 : x.len;
        a.new_held[b] = gives && done ? 0 : x.held;
        a.new_released[b] = gives && done ? 0 : (gives && tail > 0 ? end : x.released);
        a.status[b] = gives ? SMART_OK : (valid ? SMART_ECAP : SMART_EINVAL);
        if (start <= room && start + head + tail > room) a.new_count[0] = (int32_t)(free_count + start);  // (as above)
      }
    }
    __syncthreads();  // the sequences are there
    const int64_t last = offered + chunk_offered;
    for (int64_t r = offered + (int64_t)blockIdx.x * kThreads + tid; r < last; r += (int64_t)gridDim.x * kThreads) {
      const int i = find(s_start, n_here, r);
      if (!s_gives[i]) continue;
      const int at = (int)(r - s_start[i]), j = at < s_head[i] ? at : s_skip[i] + at - s_head[i];
      a.free_blocks[free_count + r] = a.table[(int64_t)(b0 + i) * a.max_blocks + j];
    }
    offered += chunk_offered;
    __syncthreads();  // everyone is done with the sequences
  }
  if (writes && tid == 0 && offered <= room) a.new_count[0] = (int32_t)(free_count + offered);
}

bool sizes_ok(int32_t batch, int32_t block_size, int32_t max_blocks, int32_t free_cap) {
  // (batch: counted in int, 256 at a time)
  return batch >= 0 && batch <= 1 << 30 && block_size > 0 && max_blocks >= 0 && free_cap >= 0 && (int64_t)max_blocks * block_size <= 0x7FFFFFFF;
}

// Workgroups for at most n rows: four rows a thread, and no more than fill the chip.
unsigned groups_for(int64_t n) {
  const int64_t g = (n + 4 * kThreads - 1) / (4 * kThreads);
  return (unsigned)(g < 1 ? 1 : (g > 512 ? 512 : g));
}

template <typename Args>
int32_t launch(void (*kernel)(Args), smart_ctx* ctx, void* stream, unsigned groups, const Args& a) {
  int prev = 0;
  SMART_HIP_CHECK(hipGetDevice(&prev));
  if (prev != ctx->device) SMART_HIP_CHECK(hipSetDevice(ctx->device));
  hipLaunchKernelGGL(kernel, dim3(groups), dim3(kThreads), 0, (hipStream_t)stream, a);
  const hipError_t e = hipGetLastError();
  if (prev != ctx->device) (void)hipSetDevice(prev);
  SMART_HIP_CHECK(e);
  return SMART_OK;
}

}  // namespace

extern "C" int32_t kv_cache_extend(smart_ctx* ctx, void* stream, int32_t batch, int32_t block_size, int32_t max_blocks_per_seq,
                                   int32_t num_blocks, const int32_t* d_len, const int32_t* d_new_tokens, const int32_t* d_held,
                                   const int32_t* d_free_blocks, int32_t free_cap, const int32_t* d_free_count, int32_t* d_block_table,
                                   int64_t total_cap, int32_t* d_cu_tokens, int64_t* d_slot_mapping, int32_t* d_new_len,
                                   int32_t* d_new_held, int32_t* d_new_free_count, int32_t* d_status) {
  if (!ctx || !sizes_ok(batch, block_size, max_blocks_per_seq, free_cap) || num_blocks < 0 || total_cap < 0 || total_cap > 0x7FFFFFFF)
    return SMART_EINVAL;
  if (!d_free_count || !d_cu_tokens || !d_new_free_count || d_free_count == d_new_free_count || (total_cap > 0 && !d_slot_mapping))
    return SMART_EINVAL;
  if (batch > 0 && (!d_len || !d_new_tokens || !d_held || !d_new_len || !d_new_held || !d_status)) return SMART_EINVAL;
  if (batch > 0 && max_blocks_per_seq > 0 && (!d_block_table || (free_cap > 0 && !d_free_blocks))) return SMART_EINVAL;
  // (other workgroups read the numbers while they are written)
  if (batch > 0)
    for (const int32_t* in : {d_len, d_new_tokens, d_held, d_free_count})
      for (const int32_t* out : {d_new_len, d_new_held, d_new_free_count, d_status, d_cu_tokens})
        if (in == out) return SMART_EINVAL;
  ExtendArgs a{batch,     block_size,    max_blocks_per_seq, num_blocks,    free_cap,    total_cap, d_len,      d_new_tokens,     d_held,
               d_free_blocks, d_free_count, d_block_table, d_cu_tokens, d_slot_mapping, d_new_len, d_new_held, d_new_free_count, d_status};
  return launch(kv_extend_kernel, ctx, stream, groups_for(total_cap), a);
}

extern "C" int32_t kv_cache_release(smart_ctx* ctx, void* stream, int32_t batch, int32_t block_size, int32_t max_blocks_per_seq,
                                    int32_t window, int32_t sinks, const int32_t* d_len, const int32_t* d_held, const int32_t* d_released,
                                    const int32_t* d_finished, const int32_t* d_block_table, int32_t* d_free_blocks, int32_t free_cap,
                                    const int32_t* d_free_count, int32_t* d_new_len, int32_t* d_new_held, int32_t* d_new_released,
                                    int32_t* d_new_free_count, int32_t* d_status) {
  if (!ctx || !sizes_ok(batch, block_size, max_blocks_per_seq, free_cap) || window < 0 || sinks < 0 || (window == 0 && sinks != 0))
    return SMART_EINVAL;
  if (!d_free_count || !d_new_free_count || d_free_count == d_new_free_count) return SMART_EINVAL;
  if (batch > 0 && (!d_len || !d_held || !d_released || !d_new_len || !d_new_held || !d_new_released || !d_status)) return SMART_EINVAL;
  if (batch > 0 && max_blocks_per_seq > 0 && (!d_block_table || (free_cap > 0 && !d_free_blocks))) return SMART_EINVAL;
  if (batch > 0)
    for (const int32_t* in : {d_len, d_held, d_released, d_finished, d_free_count})
      for (const int32_t* out : {d_new_len, d_new_held, d_new_released, d_new_free_count, d_status})
        if (in == out) return SMART_EINVAL;
  const int32_t sink_blocks = (int32_t)(((int64_t)sinks + block_size - 1) / block_size);
  ReleaseArgs a{batch,     block_size, max_blocks_per_seq, free_cap,   window,    sink_blocks, d_len,          d_held,           d_released, d_finished,
                d_block_table, d_free_blocks, d_free_count, d_new_len, d_new_held, d_new_released, d_new_free_count, d_status};
  // (a step's call gives back about a block a sequence, a few finished sequences a table row each)
  return launch(kv_release_kernel, ctx, stream, groups_for((int64_t)batch * max_blocks_per_seq / 16), a);
}
