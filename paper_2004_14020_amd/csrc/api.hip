// C ABI of the library: plan objects, binding of device memory, stream pipeline, timing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <chrono>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <mutex>
#include <new>
#include <string>
#include <vector>

#include "caramel.h"
#include "kernels.hpp"
#include "layers.hpp"
#include "memory.hpp"
#include "plan.hpp"
#include "schedule.hpp"
#include "slices.hpp"
#include "tiles.hpp"

using namespace caramel;

// Table space of caramel_allreduce_static: one copy per GPU the library runs on, held until the
// process ends.  On the host this name is only a handle for hipGetSymbolAddress; the device
// address it stands for is looked up once per device and used everywhere else.
static __device__ __align__(256) unsigned char scratch[CARAMEL_STATIC_TABLE_BYTES];

namespace {

thread_local std::string g_err;

int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  g_err = buf;
  return code;
}

#define HIP_TRY(expr)                                                                         \
  do {                                                                                        \
    hipError_t e_ = (expr);                                                                   \
    if (e_ != hipSuccess) return fail(CARAMEL_EHIP, "%s: %s", #expr, hipGetErrorString(e_)); \
  } while (0)

// No exception leaves the library: allocation failures inside an entry point become ENOMEM.
template <typename F>
int guarded(F&& body) {
  try {
    return body();
  } catch (const std::bad_alloc&) {
    return fail(CARAMEL_ENOMEM, "out of host memory");
  } catch (const std::exception& e) {
    return fail(CARAMEL_ESTATE, "unexpected failure: %s", e.what());
  }
}

struct Options {
  uint32_t launch_mode = CARAMEL_LAUNCH_AUTO;
  uint32_t batch_path = CARAMEL_BATCH_DIRECT;
  TileShape shape;
  uint32_t max_grid = 0;
  uint32_t nontemporal = 1;
  uint32_t unroll = 0;
  uint32_t block = 1024;        // workgroup of launches over long tiles
  uint32_t small_block = 256;   // ... over small tiles
  uint32_t stream_major = 8;    // most vectors per lane of the stream-major kernel for long tiles (0 = off)
  uint64_t launch_min_bytes = 4u << 20;        // launches over small tiles: units share one up to this size
  uint64_t long_launch_min_bytes = 64u << 20;  // launches over long tiles likewise
  uint64_t pipeline_min_bytes = ~uint64_t(0);  // AUTO never pipelines unless told to
  uint64_t merge_small_bytes = 1u << 20;       // one launch per stream: small tiles up to this total join the long ones
  bool split_tiles = true;                     // tiles across segment boundaries where the kernel handles them

  // nothing that shapes tiles or their kernels has been asked for
  bool tiles_left_to_library() const {
    const Options d;
    return shape.long_vecs == d.shape.long_vecs && shape.small_vecs == d.shape.small_vecs &&
           shape.long_run_bytes == d.shape.long_run_bytes && shape.align_tiles == d.shape.align_tiles &&
           shape.tail_tiles == d.shape.tail_tiles && max_grid == d.max_grid && nontemporal == d.nontemporal &&
           unroll == d.unroll && block == d.block && small_block == d.small_block &&
           stream_major == d.stream_major && split_tiles == d.split_tiles;
  }
};

// Fork/join events order work between streams of the same device; no timing, and no system-scope
// fence (device scope is enough: every producer and consumer is a kernel on this GPU).
constexpr unsigned kOrderOnly = hipEventDisableTiming | hipEventDisableSystemFence;

// One reduce launch: consecutive tiles of one class that belong to consecutive units of one lane.
struct LaunchGroup {
  uint32_t lane, first_unit;
  int cls;  // kLong or kSmall
  Range reduce;
  uint64_t elems;  // elements per replica the launch covers
};

// CARAMEL_TRACE=1 in the environment: one line on stderr per bound unit and per kernel launch
// (what is launched where, over which tiles).  Read once.
bool tracing() {
  static const bool on = [] {
    const char* v = std::getenv("CARAMEL_TRACE");
    return v && *v && std::strcmp(v, "0") != 0;
  }();
  return on;
}

struct TimedLaunch {
  int kind;
  uint64_t call;
  hipEvent_t start, stop;
};

// What binding a plan to a set of gradient pointers produces on the host.
struct Binding {
  TileShape shape;             // the shape the tables were built with
  std::vector<uint64_t> rows;  // (n_tensors + 1) x W base addresses
  TileTables tt;
  std::vector<LaunchGroup> groups[2];  // [0] staged tables, [1] direct tables
  bool groups_stale[2] = {true, true};
  bool groups_pipelined[2] = {false, false};
};

// Where the kernels find the tables of a binding.
struct DeviceTables {
  const uint64_t* rows = nullptr;
  const ReduceTile* staged = nullptr;
  const ReduceTile* direct = nullptr;
  const CopyTile* copy = nullptr;
};

}  // namespace

struct caramel_plan {
  HostPlan host;
  Options opt;
  // device side (valid when bound)
  bool bound = false;
  bool has_ws = false;
  int device = -1;  // the device that was current at bind: tables, stream and events live there
  Binding bind;
  void* d_tables[4] = {};  // what release_device() frees
  uint32_t n_tables = 0;
  DeviceTables dt;
  SliceArgs slices{};  // groups = 0: the plan is bound without slices
  hipStream_t streams[2] = {nullptr, nullptr};
  hipEvent_t ev_fork = nullptr;
  hipEvent_t ev_join[2] = {nullptr, nullptr};
  // caramel_allreduce_static keeps its own host tables; their device copy lives in the
  // library's static array
  Binding fixed;
  bool fixed_valid = false;
  uint64_t fixed_generation = 0;  // identifies the contents of `fixed` among all plans
  // timing
  int profiling = 0;  // 0 off, 1 one event pair per stream sequence, 2 one pair per launch
  uint64_t call_no = 0;
  std::vector<TimedLaunch> pending;
  std::vector<hipEvent_t> spare;
  std::vector<std::pair<uint64_t, hipEvent_t>> call_base;
  caramel_kernel_stat stats[CARAMEL_K_COUNT] = {};

  DeviceTables tables() const { return dt; }
};

namespace {

void release_device(caramel_plan* p) {
  for (; p->n_tables; --p->n_tables) (void)hipFree(p->d_tables[p->n_tables - 1]);
  p->dt = DeviceTables{};
  p->slices = SliceArgs{};
  p->bound = false;
}

void drop_events(caramel_plan* p) {
  for (TimedLaunch& t : p->pending) {
    (void)hipEventDestroy(t.start);
    (void)hipEventDestroy(t.stop);
  }
  for (auto& b : p->call_base) (void)hipEventDestroy(b.second);
  for (hipEvent_t e : p->spare) (void)hipEventDestroy(e);
  p->pending.clear();
  p->call_base.clear();
  p->spare.clear();
}

template <typename T>
int upload(caramel_plan* p, const std::vector<T>& v, const T** dst) {
  *dst = nullptr;
  if (v.empty()) return CARAMEL_OK;
  void* d = nullptr;
  HIP_TRY(hipMalloc(&d, v.size() * sizeof(T)));
  p->d_tables[p->n_tables++] = d;
  HIP_TRY(hipMemcpy(d, v.data(), v.size() * sizeof(T), hipMemcpyHostToDevice));
  *dst = static_cast<const T*>(d);
  return CARAMEL_OK;
}

hipEvent_t take_event(caramel_plan* p) {
  if (!p->spare.empty()) {
    hipEvent_t e = p->spare.back();
    p->spare.pop_back();
    return e;
  }
  hipEvent_t e = nullptr;
  // timing only: no system-scope fence, which would cost a cache write-back per record
  if (hipEventCreateWithFlags(&e, hipEventDisableSystemFence) != hipSuccess) return nullptr;
  return e;
}

// Wraps a kernel launch (or a stream's whole sequence) in a pair of timing events on the
// launch stream when profiling.
struct Timed {
  caramel_plan* p;
  hipStream_t s;
  TimedLaunch t{};
  bool on = false;
  Timed(caramel_plan* plan, int kind, hipStream_t stream, uint64_t elems = 0) : p(plan), s(stream) {
    if (!p->profiling) return;
    if (kind != CARAMEL_K_SEQUENCE) {
      p->stats[kind].launches += 1;
      p->stats[kind].elements += elems;
      if (p->profiling < 2) return;
    }
    t.kind = kind;
    t.call = p->call_no;
    t.start = take_event(p);
    t.stop = take_event(p);
    if (!t.start || !t.stop) return;
    p->pending.reserve(p->pending.size() + 4);  // the destructor must not have to allocate
    on = hipEventRecord(t.start, s) == hipSuccess;
  }
  ~Timed() {
    if (!on) return;
    (void)hipEventRecord(t.stop, s);
    p->pending.push_back(t);
  }
};

int run_reduce(caramel_plan* p, const Binding& bd, const DeviceTables& dt, bool direct, const LaunchGroup& g,
               hipStream_t s, bool timed = true) {
  const Range r = g.reduce;
  const int cls = g.cls;
  if (r.count == 0) return CARAMEL_OK;
  ReduceArgs a{};
  a.tiles = direct ? dt.direct : dt.staged;
  a.rows = dt.rows;
  a.begin = r.begin;
  a.count = r.count;
  a.world = p->host.cfg.world;
  a.bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.tree = p->host.cfg.pattern == CARAMEL_PATTERN_HALVING_DOUBLING;
  // by default a workgroup takes a whole tile in one go: vectors per lane = tile / workgroup size
  const bool lng = cls == kLong;
  a.block = lng ? p->opt.block : p->opt.small_block;
  // Writing through pays for long tiles, also where all replicas together fit the last-level cache
  // (VGG-16 1469 -> 1437 us, Inception-v3 544 -> 525, 12 workers 449 -> 431; 2 x 33 MiB 26.2 -> 25.8, 4 x 64
  // MiB 94.6 -> 92.4, their data not in the cache).  For small tiles it costs (24 workers of 3 MB: 38.5 ->
  // 46.2 us), and so it does for fused buffers, which unpack is about to read (Inception-v3's stages 359
  // -> 363 us).
  // A staged reduction that works mostly on fused buffers uses plain accesses: the replicas' fused
  // buffers start on any granule, so lines are written in parts, which the L2 joins.  The line lies
  // where that comes to outweigh the chunks, which want streaming.  All three stages with plain accesses
  // against streaming: of 90 MiB per replica, 3 to 16 workers, 7 to 13 % longer with 3 to 18 % of the
  // elements fused, 2 to 9 % with 29 to 47 %, up to 4 % with 54 to 67 %, from 8 % shorter to 2 % longer from
  // 78 % on (Inception-v3 bf16, 78 %: 358 -> 334 us; 16 workers fp32, all fused: 1570 / 1592); of 8 and
  // 25 MiB up to 15 % shorter from 78 % on (3 workers fp32, 25 MiB: up to 2 % longer).
  const bool fused = !direct && 4 * p->host.fused_elems >= 3 * p->host.replica_elems;
  a.policy = p->opt.nontemporal == 0 || fused ? kPlain : (lng && direct ? kThrough : kStream);
  const uint32_t tile_vecs = lng ? bd.shape.long_vecs : bd.shape.small_vecs;
  a.unroll = p->opt.unroll ? p->opt.unroll : std::max(1u, tile_vecs / a.block);
  // stream-major walk: as many vectors per lane as a whole tile has rows of lanes (2, 4 or 8)
  a.stream_major = 0;
  if (lng && p->opt.stream_major) {
    const uint32_t rows = tile_vecs / a.block;
    a.stream_major = std::min(p->opt.stream_major, rows >= 8 ? 8u : (rows >= 4 ? 4u : 2u));
  } else if (lng && bd.shape.split_tiles && bd.shape.max_splits) {
    a.stream_major = 1;  // the option was changed after these tables were built, and only the walk takes split tiles
  }
  // world sizes without a kernel that fetches all values at once always walk, four vectors per lane at
  // least (3 x 50 MiB 55.9 us, 62 with two or one; 32 x 50 MiB bf16 588 / 690)
  const uint32_t W = a.world;
  const bool at_once = W == 1 || W == 2 || W == 4 || W == 8 || W == 16;
  if (lng && !at_once && (!a.tree || a.stream_major)) a.stream_major = std::max(a.stream_major, 4u);
  a.max_grid = p->opt.max_grid;
  if (tracing())
    std::fprintf(stderr,
                 "caramel: call %llu reduce  stream %p (plan stream %u, from unit %u) %s tiles [%u, %u) %s, %u lanes, "
                 "%u vectors per lane and worker, %llu bytes per replica\n",
                 (unsigned long long)p->call_no, (void*)s, g.lane, g.first_unit, lng ? "long" : "small", r.begin,
                 r.begin + r.count, direct ? "in place" : "staged", a.block, a.stream_major ? a.stream_major : a.unroll,
                 (unsigned long long)(g.elems * p->host.elem_size()));
  if (!timed) {
    HIP_TRY(launch_ring_reduce(a, s));
    return CARAMEL_OK;
  }
  Timed timer(p, lng ? CARAMEL_K_REDUCE : CARAMEL_K_REDUCE_SMALL, s, g.elems);
  HIP_TRY(launch_ring_reduce(a, s));
  return CARAMEL_OK;
}

// Whether caramel_allreduce reduces batch units where their members lie.
bool reduces_in_place(const caramel_plan* p) {
  return p->opt.batch_path == CARAMEL_BATCH_DIRECT || p->host.fused_elems == 0;
}

// Reduction in place of a job that was cut into slices at bind: one launch on the caller's stream.  An
// option that asks for tiles, or for the pipeline, takes the tiles instead.
bool use_slices(const caramel_plan* p, bool direct, bool pipelined) {
  return p->slices.groups && direct && !pipelined && p->opt.launch_mode == CARAMEL_LAUNCH_AUTO &&
         p->opt.tiles_left_to_library();
}

int run_slices(caramel_plan* p, hipStream_t s) {
  const SliceArgs& a = p->slices;
  if (tracing())
    std::fprintf(stderr, "caramel: call %llu reduce  stream %p %u workgroups of %u lanes, %u slices per wavefront\n",
                 (unsigned long long)p->call_no, (void*)s, a.groups, a.lanes, a.vecs);
  Timed timer(p, CARAMEL_K_REDUCE_SMALL, s, p->host.replica_elems);
  HIP_TRY(launch_slices(a, s));
  return CARAMEL_OK;
}

int run_copy(caramel_plan* p, const DeviceTables& dt, bool unpack, Range r, hipStream_t s) {
  if (r.count == 0) return CARAMEL_OK;
  CopyArgs a{};
  a.tiles = dt.copy;
  a.rows = dt.rows;
  a.begin = r.begin;
  a.count = r.count;
  a.world = p->host.cfg.world;
  a.fused_row = uint32_t(p->host.tensor_elems.size());
  a.bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.unpack = unpack;
  // Measured on MI355X: with 0.9 GB of fused buffers (Inception-v3, Transformer) streaming loads and
  // stores are 3 to 5 points of peak faster; with 52 MB (ResNet-50), which the last-level cache
  // holds, 10 points slower.
  const bool large = p->host.fused_elems * p->host.elem_size() * p->host.cfg.world >= (uint64_t(256) << 20);
  a.policy = p->opt.nontemporal != 0 && large ? kStream : kPlain;
  if (tracing())
    std::fprintf(stderr, "caramel: call %llu %s stream %p copy tiles [%u, %u)\n", (unsigned long long)p->call_no,
                 unpack ? "unpack " : "pack   ", (void*)s, r.begin, r.begin + r.count);
  Timed timer(p, unpack ? CARAMEL_K_UNPACK : CARAMEL_K_PACK, s);
  HIP_TRY(launch_copy(a, s));
  return CARAMEL_OK;
}

int begin_call(caramel_plan* p, hipStream_t user) {
  ++p->call_no;
  if (p->profiling) {
    hipEvent_t e = take_event(p);
    if (e && hipEventRecord(e, user) == hipSuccess) p->call_base.emplace_back(p->call_no, e);
  }
  return CARAMEL_OK;
}

// Stream 0 of the plan is the caller's stream itself; stream 1 is an internal stream that starts
// after everything already queued on the caller's stream ...
int fork_streams(caramel_plan* p, hipStream_t user, hipStream_t* lane, bool pipelined) {
  lane[0] = lane[1] = user;
  if (!pipelined) return CARAMEL_OK;
  HIP_TRY(hipEventRecord(p->ev_fork, user));
  HIP_TRY(hipStreamWaitEvent(p->streams[1], p->ev_fork, 0));
  lane[1] = p->streams[1];
  return CARAMEL_OK;
}

// ... and the caller's stream continues after the internal stream has drained.
int join_streams(caramel_plan* p, hipStream_t user, bool pipelined) {
  if (!pipelined) return CARAMEL_OK;
  HIP_TRY(hipEventRecord(p->ev_join[1], p->streams[1]));
  HIP_TRY(hipStreamWaitEvent(user, p->ev_join[1], 0));
  return CARAMEL_OK;
}

// A reduce launch covers the tiles of one class (long or small) of consecutive units of one
// stream; they are adjacent in the tables, so a launch is one tile range.  PER_UNIT: units are
// added until the launch covers at least the class's minimum bytes per replica.  PER_STREAM: one
// launch per class and stream.  The order in which a stream's launches are issued does not
// affect results.  AUTO: the two-stream pipeline pays a fixed price for its fork and join (tens
// of microseconds of cross-stream signalling), so it is used only when a call moves enough
// bytes to win that back; smaller calls go out as one launch per class on the caller's stream.
bool use_pipeline(const caramel_plan* p) {
  if (p->host.cfg.num_streams != 2) return false;
  if (p->opt.launch_mode != CARAMEL_LAUNCH_AUTO) return true;
  return 2 * uint64_t(p->host.cfg.world) * p->host.replica_elems * p->host.elem_size() >= p->opt.pipeline_min_bytes;
}

// PER_UNIT or PER_STREAM: what the launch mode comes to for this plan.
uint32_t effective_mode(const caramel_plan* p, bool pipelined) {
  if (p->opt.launch_mode != CARAMEL_LAUNCH_AUTO) return p->opt.launch_mode;
  return pipelined ? CARAMEL_LAUNCH_PER_UNIT : CARAMEL_LAUNCH_PER_STREAM;
}

const std::vector<LaunchGroup>& launch_groups(const caramel_plan* p, Binding& bd, bool direct, bool pipelined) {
  const int ti = direct ? 1 : 0;
  std::vector<LaunchGroup>& out = bd.groups[ti];
  if (!bd.groups_stale[ti] && bd.groups_pipelined[ti] == pipelined) return out;
  out.clear();
  const TileTables& tt = bd.tt;
  const std::vector<UnitTiles>& unit_tiles = direct ? tt.direct_unit : tt.staged_unit;
  const uint32_t mode = effective_mode(p, pipelined);
  const uint64_t es = p->host.elem_size();
  // Without the pipeline both plan streams run on the caller's stream: treat them as one lane.
  const uint32_t lanes = pipelined ? p->host.cfg.num_streams : 1;
  for (int cls = 0; cls < 2; ++cls) {
    const uint64_t min_bytes = cls == kLong ? p->opt.long_launch_min_bytes : p->opt.launch_min_bytes;
    for (uint32_t lane = 0; lane < lanes; ++lane) {
      LaunchGroup g{};
      uint64_t bytes = 0;
      bool open = false;
      const size_t mine = out.size();  // launches of this class and lane start here
      for (uint32_t s = 0; s < p->host.cfg.num_streams; ++s) {
        if (pipelined && s != lane) continue;
        for (uint32_t u : tt.order[s]) {
          const UnitTiles& ut = unit_tiles[u];
          if (ut.tiles[cls].count == 0) continue;
          if (!open) {
            g = LaunchGroup{lane, u, cls, Range{ut.tiles[cls].begin, 0}, 0};
            bytes = 0;
            open = true;
          }
          g.reduce.count += ut.tiles[cls].count;
          g.elems += ut.elems[cls];
          bytes += ut.elems[cls] * es;
          if (mode == CARAMEL_LAUNCH_PER_UNIT && bytes >= min_bytes) {
            out.push_back(g);
            open = false;
          }
        }
      }
      if (open) {
        // what is left over at the end is rarely worth a launch of its own: less than half the
        // minimum joins the launch before it (its tiles follow that launch's in the table)
        LaunchGroup* prev = out.size() > mine ? &out.back() : nullptr;
        if (prev && bytes < min_bytes / 2 && prev->reduce.begin + prev->reduce.count == g.reduce.begin) {
          prev->reduce.count += g.reduce.count;
          prev->elems += g.elems;
        } else {
          out.push_back(g);
        }
      }
    }
  }
  // One launch per class on one stream: if the short runs are few, their tiles (which follow the
  // long tiles in the table) join the launch over the long tiles, whose kernel takes a tile of up
  // to one vector per lane in a single pass.  That saves a launch of a few microseconds; the
  // small tiles come last in the grid and fill the tail of the long ones.
  if (mode == CARAMEL_LAUNCH_PER_STREAM && lanes == 1 && out.size() == 2 && out[0].cls == kLong &&
      out[1].cls == kSmall && out[1].elems * es <= p->opt.merge_small_bytes &&
      out[0].reduce.begin + out[0].reduce.count == out[1].reduce.begin &&
      bd.shape.small_vecs <= p->opt.block) {
    out[0].reduce.count += out[1].reduce.count;
    out[0].elems += out[1].elems;
    out.pop_back();
  }
  // issue in the order of the first unit, which alternates between the streams ...
  std::stable_sort(out.begin(), out.end(),
                   [](const LaunchGroup& a, const LaunchGroup& b) { return a.first_unit < b.first_unit; });
  // ... but every stream issues its launches over small tiles first: a call then ends with the
  // long, evenly sized launches running on both streams, and the streams finish together
  std::stable_sort(out.begin(), out.end(), [](const LaunchGroup& a, const LaunchGroup& b) { return a.cls > b.cls; });
  bd.groups_stale[ti] = false;
  bd.groups_pipelined[ti] = pipelined;
  return out;
}

// Shared body of caramel_ring_reduce (reduce only, staged tables) and caramel_allreduce.  In
// staged mode every lane packs all its batch units, reduces, and unpacks them, in stream order.
int pipeline(caramel_plan* p, hipStream_t user, bool with_copies, bool direct) {
  begin_call(p, user);
  hipStream_t lane[2] = {nullptr, nullptr};
  const bool pipelined = use_pipeline(p);
  int rc = fork_streams(p, user, lane, pipelined);
  if (rc) return rc;
  const bool copies = with_copies && !direct;
  const DeviceTables dt = p->tables();
  const TileTables& tt = p->bind.tt;
  const uint32_t n_lanes = pipelined ? 2u : 1u;
  // the copy tiles of a lane: of its stream, or of both streams when there is one lane
  Range copy_of[2] = {tt.copy_stream[0], tt.copy_stream[1]};
  if (!pipelined) copy_of[0].count = tt.copy_stream[0].count + tt.copy_stream[1].count;
  // one event pair around everything a stream does in this call
  std::unique_ptr<Timed> seq[2];
  if (p->profiling)
    for (uint32_t s = 0; s < n_lanes; ++s) seq[s].reset(new Timed(p, CARAMEL_K_SEQUENCE, lane[s]));
  if (copies)
    for (uint32_t s = 0; s < n_lanes && !rc; ++s) rc = run_copy(p, dt, false, copy_of[s], lane[s]);
  if (use_slices(p, direct, pipelined))
    rc = run_slices(p, lane[0]);
  else if (!rc)
    for (const LaunchGroup& g : launch_groups(p, p->bind, direct, pipelined)) {
      rc = run_reduce(p, p->bind, dt, direct, g, lane[g.lane]);
      if (rc) break;
    }
  if (copies)
    for (uint32_t s = 0; s < n_lanes && !rc; ++s) rc = run_copy(p, dt, true, copy_of[s], lane[s]);
  for (auto& q : seq) q.reset();
  // join even after a failed launch so the caller's stream stays ordered
  const int jc = join_streams(p, user, pipelined);
  return rc ? rc : jc;
}

int need_bound(const caramel_plan* p, bool needs_ws) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  if (!p->bound) return fail(CARAMEL_ESTATE, "plan is not bound to device memory");
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != p->device)
    return fail(CARAMEL_ESTATE, "plan was bound with device %d current, now device %d is", p->device, dev);
  if (needs_ws && p->host.fused_elems > 0 && !p->has_ws)
    return fail(CARAMEL_ESTATE, "this call needs the fused workspace, but none was bound");
  return CARAMEL_OK;
}

}  // namespace

extern "C" {

namespace {
int create_plan(const caramel_config* cfg, const uint64_t* tensor_elems, uint32_t n_tensors,
                const double* ready_time, double net_a, double net_b, caramel_plan** out);
}

int caramel_plan_create(const caramel_config* cfg, const uint64_t* tensor_elems, uint32_t n_tensors,
                        caramel_plan** out) {
  return create_plan(cfg, tensor_elems, n_tensors, nullptr, 0.0, 0.0, out);
}

int caramel_plan_create_timed(const caramel_config* cfg, const uint64_t* tensor_elems, uint32_t n_tensors,
                              const double* ready_time, double net_a, double net_b, caramel_plan** out) {
  if (!ready_time) return fail(CARAMEL_EINVAL, "ready_time is NULL");
  return create_plan(cfg, tensor_elems, n_tensors, ready_time, net_a, net_b, out);
}

int caramel_plan_times(const caramel_plan* p, double* enqueue, double* start, double* finish, uint32_t cap) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const HostPlan& h = p->host;
  if (h.start_time.size() != h.units.size()) return fail(CARAMEL_ESTATE, "not a timing-aware plan");
  if (cap < h.units.size()) return fail(CARAMEL_EINVAL, "capacity %u < %zu units", cap, h.units.size());
  if (enqueue) std::copy(h.enqueue_time.begin(), h.enqueue_time.end(), enqueue);
  if (start) std::copy(h.start_time.begin(), h.start_time.end(), start);
  if (finish) std::copy(h.finish_time.begin(), h.finish_time.end(), finish);
  return CARAMEL_OK;
}

int caramel_net_model_fit(uint64_t bytes1, double time1, uint64_t bytes2, double time2, double* a, double* b) {
  if (!a || !b) return fail(CARAMEL_EINVAL, "NULL argument");
  if (bytes1 == bytes2) return fail(CARAMEL_EINVAL, "the two sizes must differ");
  if (!std::isfinite(time1) || !std::isfinite(time2)) return fail(CARAMEL_EINVAL, "times must be finite");
  const double slope = (time2 - time1) / (double(bytes2) - double(bytes1));
  const double icpt = time1 - slope * double(bytes1);
  if (!(slope > 0.0) || !(icpt >= 0.0))
    return fail(CARAMEL_EINVAL,
                "the probes (%llu B in %g, %llu B in %g) give the line %g + %g * bytes: a transfer-time model "
                "needs a >= 0 and b > 0 (time must grow with size); measure again",
                (unsigned long long)bytes1, time1, (unsigned long long)bytes2, time2, icpt, slope);
  *b = slope;
  *a = icpt;
  return CARAMEL_OK;
}

int caramel_threshold_estimate(double a, double b, uint64_t* threshold_bytes) {
  if (!threshold_bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  if (!threshold_from_model(a, b, *threshold_bytes))
    return fail(CARAMEL_EINVAL, "need finite a >= 0, b > 0 and a threshold below 2^64");
  return CARAMEL_OK;
}

int caramel_schedule_transfers(const uint64_t* group_bytes, const double* ready, const double* need,
                               uint32_t n_groups, double bp_len, double fp_len, double net_a, double net_b,
                               caramel_slot* slots, caramel_schedule_summary* summary) {
  std::string why;
  try {
    const int rc = schedule_transfers(group_bytes, ready, need, n_groups, bp_len, fp_len, net_a, net_b, slots,
                                      summary, why);
    return rc == CARAMEL_OK ? rc : fail(rc, why.c_str());
  } catch (const std::bad_alloc&) {
    return fail(CARAMEL_ENOMEM, "out of host memory");
  }
}

int caramel_plan_windows(const caramel_plan* plan, const double* ready_time, const double* read_time,
                         uint64_t* group_bytes, double* ready, double* need, uint32_t cap) {
  if (!plan || !ready_time || !read_time) return fail(CARAMEL_EINVAL, "NULL argument");
  const size_t n = plan->host.units.size();
  if (cap < n) return fail(CARAMEL_EINVAL, "cap is smaller than the number of units");
  try {
    std::vector<uint64_t> b(n);
    std::vector<double> r(n), d(n);
    unit_windows(plan->host, ready_time, read_time, b.data(), r.data(), d.data());
    if (group_bytes) std::copy(b.begin(), b.end(), group_bytes);
    if (ready) std::copy(r.begin(), r.end(), ready);
    if (need) std::copy(d.begin(), d.end(), need);
  } catch (const std::bad_alloc&) {
    return fail(CARAMEL_ENOMEM, "out of host memory");
  }
  return CARAMEL_OK;
}

}  // extern "C"

namespace {
int create_plan(const caramel_config* cfg, const uint64_t* tensor_elems, uint32_t n_tensors,
                const double* ready_time, double net_a, double net_b, caramel_plan** out) {
  if (!cfg || !out) return fail(CARAMEL_EINVAL, "NULL argument");
  *out = nullptr;
  caramel_plan* p = new (std::nothrow) caramel_plan;
  if (!p) return fail(CARAMEL_ENOMEM, "out of host memory");
  std::string why;
  int rc;
  try {
    rc = build_host_plan(*cfg, tensor_elems, n_tensors, ready_time, net_a, net_b, p->host, why);
  } catch (const std::bad_alloc&) {
    delete p;
    return fail(CARAMEL_ENOMEM, "out of host memory");
  }
  if (rc != CARAMEL_OK) {
    delete p;
    return fail(rc, "%s", why.c_str());
  }
  *out = p;
  return CARAMEL_OK;
}
}  // namespace

extern "C" {

void caramel_plan_destroy(caramel_plan* p) {
  if (!p) return;
  if (p->bound || p->streams[1] || p->ev_fork) {
    for (int s = 0; s < 2; ++s)
      if (p->streams[s]) (void)hipStreamSynchronize(p->streams[s]);
    drop_events(p);
    release_device(p);
    for (int s = 0; s < 2; ++s) {
      if (p->streams[s]) (void)hipStreamDestroy(p->streams[s]);
      if (p->ev_join[s]) (void)hipEventDestroy(p->ev_join[s]);
    }
    if (p->ev_fork) (void)hipEventDestroy(p->ev_fork);
  }
  delete p;
}

int caramel_plan_counts(const caramel_plan* p, uint32_t* n_units, uint32_t* n_entries, uint64_t* fused_elems) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  if (n_units) *n_units = uint32_t(p->host.units.size());
  if (n_entries) *n_entries = uint32_t(p->host.entries.size());
  if (fused_elems) *fused_elems = p->host.fused_elems;
  return CARAMEL_OK;
}

int caramel_plan_units(const caramel_plan* p, caramel_unit* out, uint32_t cap) {
  if (!p || !out) return fail(CARAMEL_EINVAL, "NULL argument");
  if (cap < p->host.units.size()) return fail(CARAMEL_EINVAL, "capacity %u < %zu units", cap, p->host.units.size());
  std::copy(p->host.units.begin(), p->host.units.end(), out);
  return CARAMEL_OK;
}

int caramel_plan_entries(const caramel_plan* p, caramel_entry* out, uint32_t cap) {
  if (!p || !out) return fail(CARAMEL_EINVAL, "NULL argument");
  if (cap < p->host.entries.size())
    return fail(CARAMEL_EINVAL, "capacity %u < %zu entries", cap, p->host.entries.size());
  std::copy(p->host.entries.begin(), p->host.entries.end(), out);
  return CARAMEL_OK;
}

int caramel_plan_segments(const caramel_plan* p, uint32_t unit, uint64_t* seg_start) {
  if (!p || !seg_start) return fail(CARAMEL_EINVAL, "NULL argument");
  if (unit >= p->host.units.size()) return fail(CARAMEL_EINVAL, "unit %u out of range", unit);
  const uint64_t* s = p->host.segments(unit);
  std::copy(s, s + p->host.cfg.world + 1, seg_start);
  return CARAMEL_OK;
}

int caramel_plan_serialize(const caramel_plan* p, void* buf, size_t* len) {
  if (!p || !len) return fail(CARAMEL_EINVAL, "NULL argument");
  return guarded([&]() -> int {
    const std::vector<uint8_t> img = serialize(p->host);
    if (!buf) {
      *len = img.size();
      return CARAMEL_OK;
    }
    if (*len < img.size()) return fail(CARAMEL_EINVAL, "buffer of %zu bytes, need %zu", *len, img.size());
    std::memcpy(buf, img.data(), img.size());
    *len = img.size();
    return CARAMEL_OK;
  });
}

int caramel_plan_set_option(caramel_plan* p, uint32_t option, uint64_t value) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  auto regroup = [&] {
    for (Binding* b : {&p->bind, &p->fixed}) b->groups_stale[0] = b->groups_stale[1] = true;
  };
  auto is_block = [](uint64_t v) { return v == 256 || v == 512 || v == 1024; };
  switch (option) {
    case CARAMEL_OPT_LAUNCH_MODE:
      if (value > CARAMEL_LAUNCH_AUTO) return fail(CARAMEL_EINVAL, "unknown launch mode");
      p->opt.launch_mode = uint32_t(value);
      regroup();
      return CARAMEL_OK;
    case CARAMEL_OPT_BATCH_PATH:
      if (value > CARAMEL_BATCH_DIRECT) return fail(CARAMEL_EINVAL, "unknown batch path");
      p->opt.batch_path = uint32_t(value);
      return CARAMEL_OK;
    case CARAMEL_OPT_TILE_VECS:
      if (value != 0 && (value < 64 || value > (1u << 20))) return fail(CARAMEL_EINVAL, "tile_vecs must be 0 or in [64, 2^20]");
      p->opt.shape.long_vecs = uint32_t(value);
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_SMALL_TILE_VECS:
      if (value < 64 || value > (1u << 20)) return fail(CARAMEL_EINVAL, "tile_vecs must be in [64, 2^20]");
      p->opt.shape.small_vecs = uint32_t(value);
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_SMALL_BLOCK:
      if (!is_block(value)) return fail(CARAMEL_EINVAL, "block must be 256, 512 or 1024");
      p->opt.small_block = uint32_t(value);
      return CARAMEL_OK;
    case CARAMEL_OPT_LONG_LAUNCH_MIN_BYTES:
      p->opt.long_launch_min_bytes = value;
      regroup();
      return CARAMEL_OK;
    case CARAMEL_OPT_STREAM_MAJOR:
      if (value != 0 && value != 2 && value != 4 && value != 8) return fail(CARAMEL_EINVAL, "stream_major must be 0, 2, 4 or 8");
      p->opt.stream_major = uint32_t(value);
      return CARAMEL_OK;
    case CARAMEL_OPT_ALIGN_TILES:
      if (value > 3) return fail(CARAMEL_EINVAL, "align_tiles must be 0..3");
      p->opt.shape.align_tiles = uint32_t(value);
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_LONG_RUN_BYTES:
      p->opt.shape.long_run_bytes = value;
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_MAX_GRID:
      if (value > 0x7FFFFFFFu) return fail(CARAMEL_EINVAL, "max_grid too large");
      p->opt.max_grid = uint32_t(value);
      return CARAMEL_OK;
    case CARAMEL_OPT_NONTEMPORAL:
      p->opt.nontemporal = value ? 1 : 0;
      return CARAMEL_OK;
    case CARAMEL_OPT_UNROLL:
      if (value != 0 && value != 1 && value != 2 && value != 4) return fail(CARAMEL_EINVAL, "unroll must be 0, 1, 2 or 4");
      p->opt.unroll = uint32_t(value);
      return CARAMEL_OK;
    case CARAMEL_OPT_LAUNCH_MIN_BYTES:
      p->opt.launch_min_bytes = value;
      regroup();
      return CARAMEL_OK;
    case CARAMEL_OPT_PIPELINE_MIN_BYTES:
      p->opt.pipeline_min_bytes = value;
      regroup();
      return CARAMEL_OK;
    case CARAMEL_OPT_BLOCK:
      if (!is_block(value)) return fail(CARAMEL_EINVAL, "block must be 256, 512 or 1024");
      p->opt.block = uint32_t(value);
      regroup();
      return CARAMEL_OK;
    case CARAMEL_OPT_TAIL_TILES:
      if (value > 0x7FFFFFFFu) return fail(CARAMEL_EINVAL, "tail_tiles too large");
      p->opt.shape.tail_tiles = uint32_t(value);
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_SPLIT_TILES:
      if (value > 1) return fail(CARAMEL_EINVAL, "split_tiles must be 0 or 1");
      p->opt.split_tiles = value != 0;
      p->fixed_valid = false;
      return CARAMEL_OK;
    case CARAMEL_OPT_MERGE_SMALL_BYTES:
      p->opt.merge_small_bytes = value;
      regroup();
      return CARAMEL_OK;
    default:
      return fail(CARAMEL_EINVAL, "unknown option %u", option);
  }
}

int caramel_plan_slices(const caramel_plan* p, uint32_t* workgroups, uint32_t* lanes, uint32_t* per_wavefront) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  if (!p->bound) return fail(CARAMEL_ESTATE, "plan is not bound to device memory");
  const SliceArgs a = use_slices(p, reduces_in_place(p), use_pipeline(p)) ? p->slices : SliceArgs{};
  if (workgroups) *workgroups = a.groups;
  if (lanes) *lanes = a.lanes;
  if (per_wavefront) *per_wavefront = a.vecs;
  return CARAMEL_OK;
}

namespace {
int bind_plan(caramel_plan* p, void* const* grads, void* fused_ws);
}

int caramel_bind(caramel_plan* p, void* const* grads, void* fused_ws) {
  return guarded([&] { return bind_plan(p, grads, fused_ws); });
}

}  // extern "C"

namespace {
// Argument checks of a binding; on success `rows` holds the (n_tensors + 1) x W base addresses.
int check_pointers(const HostPlan& h, void* const* grads, void* fused_ws, std::vector<uint64_t>& rows) {
  const uint32_t W = h.cfg.world;
  const size_t n = h.tensor_elems.size();
  const uint64_t es = h.elem_size();
  struct Span {
    uint64_t lo, hi;
  };
  std::vector<Span> spans;
  spans.reserve(W * n + 1);
  for (uint32_t w = 0; w < W; ++w)
    for (size_t t = 0; t < n; ++t) {
      const uint64_t a = reinterpret_cast<uint64_t>(grads[w * n + t]);
      if (a == 0) return fail(CARAMEL_EINVAL, "grads[%u][%zu] is NULL", w, t);
      if (a % h.cfg.align_bytes) return fail(CARAMEL_EINVAL, "grads[%u][%zu] is not aligned to %u bytes", w, t, h.cfg.align_bytes);
      spans.push_back({a, a + h.tensor_elems[t] * es});
    }
  if (fused_ws) {
    const uint64_t a = reinterpret_cast<uint64_t>(fused_ws);
    if (a % h.cfg.align_bytes) return fail(CARAMEL_EINVAL, "fused_ws is not aligned to %u bytes", h.cfg.align_bytes);
    if (h.fused_elems) spans.push_back({a, a + uint64_t(W) * h.fused_elems * es});
  }
  std::sort(spans.begin(), spans.end(), [](const Span& x, const Span& y) { return x.lo < y.lo; });
  for (size_t i = 1; i < spans.size(); ++i)
    if (spans[i].lo < spans[i - 1].hi) return fail(CARAMEL_EINVAL, "gradient / workspace buffers overlap");
  rows.assign((n + 1) * W, 0);
  for (uint32_t w = 0; w < W; ++w) {
    for (size_t t = 0; t < n; ++t) rows[t * W + w] = reinterpret_cast<uint64_t>(grads[w * n + t]);
    rows[n * W + w] = fused_ws ? reinterpret_cast<uint64_t>(fused_ws) + uint64_t(w) * h.fused_elems * es : 0;
  }
  return CARAMEL_OK;
}

void fill_binding(const caramel_plan* p, std::vector<uint64_t>&& rows, Binding& bd, bool few_tiles = false) {
  bd.shape = p->opt.shape;
  choose_shape(p->host, p->opt.split_tiles, p->opt.stream_major, p->opt.block, few_tiles, bd.shape);
  bd.rows = std::move(rows);
  build_tiles(p->host, bd.shape, bd.tt, bd.rows.data());
  bd.groups_stale[0] = bd.groups_stale[1] = true;
}

// Tables of a job in slices: one allocation and one copy for what the host has, and the GPU writes the slices' tables.
int upload_with_slices(caramel_plan* p, const SliceTable& t, const std::vector<SlicePiece>& pieces, bool staged) {
  const Binding& bd = p->bind;
  std::vector<unsigned char> host;
  auto add = [&](const auto& v) {
    const size_t off = (host.size() + 255) / 256 * 256;
    host.resize(off + v.size() * sizeof v[0]);
    if (!v.empty()) std::memcpy(&host[off], v.data(), v.size() * sizeof v[0]);
    return off;
  };
  const size_t o_pieces = add(pieces), o_rows = add(bd.rows), o_direct = add(bd.tt.direct);
  const size_t o_staged = staged ? add(bd.tt.staged) : 0, o_copy = staged ? add(bd.tt.copy) : 0;
  const size_t o_at = (host.size() + 255) / 256 * 256, o_bytes = o_at + (t.at_words() * sizeof(uint32_t) + 255) / 256 * 256;
  void* q = nullptr;
  HIP_TRY(hipMalloc(&q, o_bytes + t.bytes_words() * sizeof(uint32_t)));
  p->d_tables[p->n_tables++] = q;
  unsigned char* const d = static_cast<unsigned char*>(q);
  HIP_TRY(hipMemcpy(d, host.data(), host.size(), hipMemcpyHostToDevice));
  p->dt.rows = reinterpret_cast<const uint64_t*>(d + o_rows);
  p->dt.direct = reinterpret_cast<const ReduceTile*>(d + o_direct);
  if (staged) p->dt.staged = reinterpret_cast<const ReduceTile*>(d + o_staged);
  if (staged) p->dt.copy = reinterpret_cast<const CopyTile*>(d + o_copy);
  uint32_t* const at = reinterpret_cast<uint32_t*>(d + o_at);
  uint32_t* const bytes = reinterpret_cast<uint32_t*>(d + o_bytes);
  HIP_TRY(launch_slice_table(t, reinterpret_cast<const SlicePiece*>(d + o_pieces), p->dt.rows, at, bytes, nullptr));
  HIP_TRY(hipStreamSynchronize(nullptr));  // calls may come on any stream
  p->slices.at = at;
  p->slices.bytes = bytes;
  return CARAMEL_OK;
}

int upload_tables(caramel_plan* p, bool staged) {
  const HostPlan& h = p->host;
  const Binding& bd = p->bind;
  if (p->opt.tiles_left_to_library() && may_have_slices(h)) {
    std::vector<SlicePiece> pieces;
    const uint64_t n = slice_pieces(h, bd.rows.data(), pieces);
    const SliceShape shape = choose_slices(h, n, pieces.size());
    const SliceTable t = slice_table(h, shape, n, pieces.size(), bd.rows.data());
    if (t.groups) {
      p->slices = SliceArgs{nullptr, nullptr, t.base, t.groups, t.lanes, t.vecs, h.cfg.world, h.cfg.dtype == CARAMEL_BF16,
                            shape.through ? kThrough : kStream,
                            h.cfg.pattern == CARAMEL_PATTERN_HALVING_DOUBLING && h.cfg.world > 1};
      return upload_with_slices(p, t, pieces, staged);
    }
  }
  int rc = upload(p, bd.rows, &p->dt.rows);
  if (!rc) rc = upload(p, bd.tt.direct, &p->dt.direct);
  if (!rc && staged) rc = upload(p, bd.tt.staged, &p->dt.staged);
  if (!rc && staged) rc = upload(p, bd.tt.copy, &p->dt.copy);
  return rc;
}

int bind_plan(caramel_plan* p, void* const* grads, void* fused_ws) {
  if (!p || !grads) return fail(CARAMEL_EINVAL, "NULL argument");
  const HostPlan& h = p->host;
  // argument checks first: nothing is touched on the device if they fail
  std::vector<uint64_t> rows;
  if (int rc = check_pointers(h, grads, fused_ws, rows)) return rc;

  // a plan stays on the device it was first bound on: its stream and events live there
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (p->device >= 0 && dev != p->device)
    return fail(CARAMEL_ESTATE, "plan was bound with device %d current, now device %d is", p->device, dev);
  for (int s = 0; s < 2; ++s)
    if (p->streams[s]) HIP_TRY(hipStreamSynchronize(p->streams[s]));
  release_device(p);
  p->device = dev;

  fill_binding(p, std::move(rows), p->bind);
  const int rc = upload_tables(p, fused_ws != nullptr);
  if (rc) {
    release_device(p);
    return rc;
  }
  if (h.cfg.num_streams > 1) {
    // each handle under its own check: a plan whose earlier bind failed half-way is completed here
    hipError_t e = hipSuccess;
    if (!p->streams[1]) e = hipStreamCreateWithFlags(&p->streams[1], hipStreamNonBlocking);
    if (e == hipSuccess && !p->ev_join[1]) e = hipEventCreateWithFlags(&p->ev_join[1], kOrderOnly);
    if (e == hipSuccess && !p->ev_fork) e = hipEventCreateWithFlags(&p->ev_fork, kOrderOnly);
    if (e != hipSuccess) {
      release_device(p);  // the tables go too: the plan stays unbound
      return fail(CARAMEL_EHIP, "creating the internal stream and its events: %s", hipGetErrorString(e));
    }
  }
  p->has_ws = fused_ws != nullptr;
  p->bound = true;
  if (tracing()) {
    std::fprintf(stderr, "caramel: bind  %zu units, long tiles of %u vectors, small of %u, runs of %llu bytes or more are long\n",
                 h.units.size(), p->bind.shape.long_vecs, p->bind.shape.small_vecs,
                 (unsigned long long)p->bind.shape.long_run_bytes);
    if (p->slices.groups)
      std::fprintf(stderr, "caramel: bind  in place over slices: %u workgroups of %u lanes, %u slices per wavefront\n",
                   p->slices.groups, p->slices.lanes, p->slices.vecs);
    for (size_t u = 0; u < h.units.size(); ++u) {
      const UnitTiles& ut = p->bind.tt.direct_unit[u];
      std::fprintf(stderr, "caramel: unit %zu %s stream %u %llu bytes per replica: %u long + %u small tiles\n", u,
                   h.units[u].kind == CARAMEL_KIND_BATCH ? "batch" : "chunk", h.units[u].stream,
                   (unsigned long long)(h.units[u].elems * h.elem_size()), ut.tiles[kLong].count, ut.tiles[kSmall].count);
    }
  }
  return CARAMEL_OK;
}
}  // namespace

extern "C" {

int caramel_pack(caramel_plan* p, void* stream) {
  return guarded([&]() -> int {
    if (int rc = need_bound(p, true)) return rc;
    begin_call(p, hipStream_t(stream));
    Range all{0, uint32_t(p->bind.tt.copy.size())};
    return run_copy(p, p->tables(), false, all, hipStream_t(stream));
  });
}

int caramel_unpack(caramel_plan* p, void* stream) {
  return guarded([&]() -> int {
    if (int rc = need_bound(p, true)) return rc;
    begin_call(p, hipStream_t(stream));
    Range all{0, uint32_t(p->bind.tt.copy.size())};
    return run_copy(p, p->tables(), true, all, hipStream_t(stream));
  });
}

int caramel_ring_reduce(caramel_plan* p, void* stream) {
  return guarded([&]() -> int {
    if (int rc = need_bound(p, true)) return rc;
    // without a workspace there are no batch units, and the two tables coincide
    return pipeline(p, hipStream_t(stream), false, !p->has_ws);
  });
}

int caramel_allreduce(caramel_plan* p, void* stream) {
  return guarded([&]() -> int {
    const bool direct = p && reduces_in_place(p);
    if (int rc = need_bound(p, !direct)) return rc;
    return pipeline(p, hipStream_t(stream), true, direct);
  });
}

namespace {

constexpr int kMaxDevices = 64;
std::mutex g_scratch_mu;
unsigned char* g_scratch_ptr[kMaxDevices] = {};  // device address of each GPU's copy of `scratch`
uint64_t g_scratch_holds[kMaxDevices] = {};      // generation of the tables it holds (0: none)
hipStream_t g_scratch_stream[kMaxDevices] = {};  // stream they were uploaded on
uint64_t g_generation = 0;

int allreduce_static(caramel_plan* p, void* const* grads, hipStream_t stream) {
  if (!p || !grads) return fail(CARAMEL_EINVAL, "NULL argument");
  const HostPlan& h = p->host;
  std::vector<uint64_t> rows;
  if (int rc = check_pointers(h, grads, nullptr, rows)) return rc;
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev < 0 || dev >= kMaxDevices) return fail(CARAMEL_ESTATE, "device %d is beyond the %d this entry point serves", dev, kMaxDevices);

  std::lock_guard<std::mutex> lock(g_scratch_mu);
  auto table_bytes = [](const Binding& b) {
    return (b.rows.size() * sizeof(uint64_t) + 255) / 256 * 256 + b.tt.direct.size() * sizeof(ReduceTile);
  };
  if (!p->fixed_valid || rows != p->fixed.rows) {
    fill_binding(p, std::move(rows), p->fixed);
    if (table_bytes(p->fixed) > CARAMEL_STATIC_TABLE_BYTES)
      fill_binding(p, std::vector<uint64_t>(p->fixed.rows), p->fixed, true);
    p->fixed_valid = true;
    p->fixed_generation = ++g_generation;
  }
  const Binding& bd = p->fixed;
  const size_t rows_bytes = (bd.rows.size() * sizeof(uint64_t) + 255) / 256 * 256;
  const size_t tile_bytes = bd.tt.direct.size() * sizeof(ReduceTile);
  if (table_bytes(bd) > CARAMEL_STATIC_TABLE_BYTES)
    return fail(CARAMEL_EINVAL,
                "this plan needs %zu bytes of descriptor tables (%zu tensors x %u workers, %zu tiles); the "
                "static array holds %u: use caramel_bind + caramel_allreduce",
                rows_bytes + tile_bytes, h.tensor_elems.size(), h.cfg.world, bd.tt.direct.size(),
                unsigned(CARAMEL_STATIC_TABLE_BYTES));

  // this GPU's copy of the array: looked up once, with this device current
  if (!g_scratch_ptr[dev]) {
    void* q = nullptr;
    HIP_TRY(hipGetSymbolAddress(&q, HIP_SYMBOL(scratch)));
    if (!q) return fail(CARAMEL_EHIP, "hipGetSymbolAddress returned no address for the static table array");
    g_scratch_ptr[dev] = static_cast<unsigned char*>(q);
  }
  unsigned char* base = g_scratch_ptr[dev];
  // The array keeps what the last call put there.  Tables are written whole before they are
  // used and nothing is read beyond them, so nothing needs clearing; they are uploaded again
  // unless this GPU's array still holds exactly these, put there through this same stream.
  if (g_scratch_holds[dev] != p->fixed_generation || g_scratch_stream[dev] != stream) {
    g_scratch_holds[dev] = 0;
    HIP_TRY(hipMemcpyAsync(base, bd.rows.data(), bd.rows.size() * sizeof(uint64_t), hipMemcpyHostToDevice, stream));
    if (tile_bytes)
      HIP_TRY(hipMemcpyAsync(base + rows_bytes, bd.tt.direct.data(), tile_bytes, hipMemcpyHostToDevice, stream));
    // the host tables may be rebuilt or freed by a later call: wait until they have been read
    HIP_TRY(hipStreamSynchronize(stream));
    g_scratch_holds[dev] = p->fixed_generation;
    g_scratch_stream[dev] = stream;
  }
  DeviceTables dt;
  dt.rows = reinterpret_cast<const uint64_t*>(base);
  dt.direct = reinterpret_cast<const ReduceTile*>(base + rows_bytes);
  for (const LaunchGroup& g : launch_groups(p, p->fixed, true, false))
    if (int rc = run_reduce(p, p->fixed, dt, true, g, stream, false)) return rc;
  return CARAMEL_OK;
}

}  // namespace

int caramel_allreduce_static(caramel_plan* p, void* const* grads, void* stream) {
  return guarded([&] { return allreduce_static(p, grads, hipStream_t(stream)); });
}

// ---- what fills a plan's gradient tensors ---------------------------------------------------

namespace {

constexpr uint64_t kMaxTokens = uint64_t(1) << 25;
constexpr uint64_t kMaxWidth = uint64_t(1) << 20;  // columns of a table, features, outputs
constexpr uint64_t kMaxPitch = uint64_t(1) << 23;
constexpr uint64_t kMaxValues = uint64_t(1) << 38;  // tokens * columns of a worker

uint64_t size_of(uint32_t dtype) { return dtype == CARAMEL_F32 ? 4 : 2; }

// The plan may be unbound (nothing of it is on a device), but not bound on another device.
int need_device(const caramel_plan* p) {
  if (p->device < 0) return CARAMEL_OK;
  int dev = -1;
  HIP_TRY(hipGetDevice(&dev));
  if (dev != p->device)
    return fail(CARAMEL_ESTATE, "plan was bound with device %d current, now device %d is", p->device, dev);
  return CARAMEL_OK;
}

int check_memory(Memory& m) {
  return m.overlap() ? fail(CARAMEL_EINVAL, "buffers overlap with one that is written") : CARAMEL_OK;
}

int take_tokens(const caramel_plan* p, const uint64_t* tokens, uint32_t* out, uint32_t* most) {
  if (!tokens) return fail(CARAMEL_EINVAL, "tokens is NULL");
  *most = 0;
  for (uint32_t w = 0; w < p->host.cfg.world; ++w) {
    if (tokens[w] > kMaxTokens) return fail(CARAMEL_EINVAL, "tokens[%u] = %llu is more than 2^25", w, (unsigned long long)tokens[w]);
    out[w] = uint32_t(tokens[w]);
    *most = std::max(*most, out[w]);
  }
  return CARAMEL_OK;
}

// One pointer per worker; that of a worker without tokens is not used, and may be NULL.
int take_pointers(const caramel_plan* p, const char* name, const void* const* from, const uint32_t* tokens, uint64_t align,
                  uint64_t* out) {
  if (!from) return fail(CARAMEL_EINVAL, "%s is NULL", name);
  for (uint32_t w = 0; w < p->host.cfg.world; ++w) {
    out[w] = reinterpret_cast<uint64_t>(from[w]);
    if (tokens && !tokens[w]) continue;
    if (!out[w]) return fail(CARAMEL_EINVAL, "%s[%u] is NULL", name, w);
    if (out[w] % align) return fail(CARAMEL_EINVAL, "%s[%u] is not aligned to %llu bytes", name, w, (unsigned long long)align);
  }
  return CARAMEL_OK;
}

int check_columns(const char* name, uint64_t columns) {
  if (columns == 0 || columns > kMaxWidth) return fail(CARAMEL_EINVAL, "%s must be 1 to 2^20, is %llu", name, (unsigned long long)columns);
  return CARAMEL_OK;
}

int check_rows(const char* name, uint64_t pitch, uint64_t columns, uint32_t most) {
  if (pitch < columns || pitch > kMaxPitch)
    return fail(CARAMEL_EINVAL, "%s must be %llu to 2^23 elements, is %llu", name, (unsigned long long)columns, (unsigned long long)pitch);
  if (uint64_t(most) * pitch > kMaxValues) return fail(CARAMEL_EINVAL, "more than 2^38 values at one worker");
  return CARAMEL_OK;
}

int check_dtype(const char* name, uint32_t dtype) {
  if (dtype != CARAMEL_F32 && dtype != CARAMEL_BF16) return fail(CARAMEL_EINVAL, "unknown %s %u", name, dtype);
  return CARAMEL_OK;
}

int check_workspace(const void* ws, uint64_t have, uint64_t need) {
  if (need == 0) return CARAMEL_OK;
  if (!ws) return fail(CARAMEL_EINVAL, "the workspace is NULL, %llu bytes are needed", (unsigned long long)need);
  if (reinterpret_cast<uint64_t>(ws) % 16) return fail(CARAMEL_EINVAL, "the workspace is not aligned to 16 bytes");
  if (have < need)
    return fail(CARAMEL_EINVAL, "the workspace has %llu bytes, %llu are needed", (unsigned long long)have, (unsigned long long)need);
  return CARAMEL_OK;
}

uint64_t checkpoint_size(uint64_t tokens, uint64_t features) {
  return (checkpoint_blocks(tokens) * features * (kCheckpointBlock + 1) + 15) / 16 * 16;
}

int check_table(uint64_t vocab, uint64_t width) {
  if (int rc = check_columns("width", width)) return rc;
  if (vocab == 0 || vocab >= 0x7FFFFFFFull) return fail(CARAMEL_EINVAL, "vocab must be 1 to 2^31 - 2, is %llu", (unsigned long long)vocab);
  return CARAMEL_OK;
}

// A tensor of the plan as a matrix with `columns` columns
int check_matrix(const caramel_plan* p, const char* name, uint32_t tensor, uint64_t columns, uint64_t* rows) {
  if (tensor >= p->host.tensor_elems.size()) return fail(CARAMEL_EINVAL, "the plan has no tensor %u (%s)", tensor, name);
  const uint64_t n = p->host.tensor_elems[tensor];
  if (columns == 0 || n % columns)
    return fail(CARAMEL_EINVAL, "tensor %u (%s) has %llu elements, no multiple of %llu", tensor, name, (unsigned long long)n,
                (unsigned long long)columns);
  *rows = n / columns;
  return CARAMEL_OK;
}

int embedding_lookup(caramel_plan* p, const void* const* table, uint64_t vocab, uint64_t width, float scale, const void* const* ids,
                     uint32_t id_bytes, const uint64_t* tokens, void* const* out, uint64_t out_pitch, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const uint64_t es = p->host.elem_size();
  LookupArgs a{};
  AllWorkers v{};
  if (int rc = check_table(vocab, width)) return rc;
  if (id_bytes != 4 && id_bytes != 8) return fail(CARAMEL_EINVAL, "id_bytes must be 4 or 8, is %u", id_bytes);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("out_pitch", out_pitch, width, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "table", table, v.tokens, es, v.a)) return rc;
  if (int rc = take_pointers(p, "ids", ids, v.tokens, id_bytes, v.b)) return rc;
  if (int rc = take_pointers(p, "out", out, v.tokens, es, v.c)) return rc;
  a.all = p->host.cfg.world;
  Memory m;
  for (uint32_t w = 0; w < a.all; ++w) {
    if (!v.tokens[w]) continue;
    m.add(v.a[w], vocab * width * es, false);
    m.add(v.b[w], uint64_t(v.tokens[w]) * id_bytes, false);
    m.add_rows(v.c[w], v.tokens[w], out_pitch, width, es, true);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  a.vocab = uint32_t(vocab);
  a.width = uint32_t(width);
  a.out_pitch = out_pitch;
  a.scale = scale;
  a.ids64 = id_bytes == 8;
  a.bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  if (tracing())
    std::fprintf(stderr, "caramel: embedding lookup stream %p, %u workers, up to %u tokens, %u columns\n", (void*)stream, a.all,
                 a.max_tokens, a.width);
  HIP_TRY(launch_embedding_lookup(a, v, stream));
  return CARAMEL_OK;
}

int embedding_workspace(const caramel_plan* p, uint32_t tensor, uint64_t width, const uint64_t* tokens, uint64_t* bytes) {
  if (!p || !bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  uint64_t vocab = 0;
  uint32_t n[CARAMEL_MAX_WORLD], most = 0;
  if (int rc = check_matrix(p, "table", tensor, width, &vocab)) return rc;
  if (int rc = check_table(vocab, width)) return rc;
  if (int rc = take_tokens(p, tokens, n, &most)) return rc;
  *bytes = embedding_gradient_workspace(p->host.cfg.world, uint32_t(vocab), uint32_t(width), most);
  return CARAMEL_OK;
}

int embedding_gradient(caramel_plan* p, uint32_t tensor, uint64_t width, float scale, const void* const* ids, uint32_t id_bytes,
                       const uint64_t* tokens, const void* const* dy, uint32_t dy_dtype, uint64_t dy_pitch, int accumulate,
                       void* ws, uint64_t ws_bytes, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const uint64_t es = p->host.elem_size();
  uint64_t vocab = 0;
  EmbeddingGradientArgs a{};
  AllWorkers v{};
  if (int rc = check_matrix(p, "table", tensor, width, &vocab)) return rc;
  if (int rc = check_table(vocab, width)) return rc;
  if (id_bytes != 4 && id_bytes != 8) return fail(CARAMEL_EINVAL, "id_bytes must be 4 or 8, is %u", id_bytes);
  if (int rc = check_dtype("dy_dtype", dy_dtype)) return rc;
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("dy_pitch", dy_pitch, width, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "ids", ids, v.tokens, id_bytes, v.a)) return rc;
  if (int rc = take_pointers(p, "dy", dy, v.tokens, size_of(dy_dtype), v.b)) return rc;
  a.all = p->host.cfg.world;
  const uint64_t need = embedding_gradient_workspace(a.all, uint32_t(vocab), uint32_t(width), a.max_tokens);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  if (int rc = need_bound(p, false)) return rc;
  Memory m;
  m.add(reinterpret_cast<uint64_t>(ws), need, true);
  for (uint32_t w = 0; w < a.all; ++w) {
    v.c[w] = p->bind.rows[tensor * a.all + w];
    m.add(v.c[w], vocab * width * es, true);
    m.add(v.a[w], uint64_t(v.tokens[w]) * id_bytes, false);
    m.add_rows(v.b[w], v.tokens[w], dy_pitch, width, size_of(dy_dtype), false);
  }
  if (int rc = check_memory(m)) return rc;
  a.vocab = uint32_t(vocab);
  a.width = uint32_t(width);
  a.dy_pitch = dy_pitch;
  a.scale = scale;
  a.ids64 = id_bytes == 8;
  a.dy_bf16 = dy_dtype == CARAMEL_BF16;
  a.out_bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.accumulate = accumulate != 0;
  a.ws = static_cast<unsigned char*>(ws);
  if (tracing())
    std::fprintf(stderr, "caramel: embedding gradient stream %p, tensor %u, %u workers, up to %u tokens, %u x %u\n", (void*)stream,
                 tensor, a.all, a.max_tokens, a.vocab, a.width);
  HIP_TRY(launch_embedding_gradient(a, v, stream));
  return CARAMEL_OK;
}

int checkpoint_call(caramel_plan* p, bool store, const uint64_t* tokens, uint64_t features, const void* const* x, uint32_t dtype,
                    uint64_t pitch, const void* const* checkpoint, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  CheckpointArgs a{};
  AllWorkers v{};
  if (int rc = check_columns("features", features)) return rc;
  if (int rc = check_dtype("dtype", dtype)) return rc;
  const uint64_t es = size_of(dtype);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("pitch", pitch, features, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "x", x, v.tokens, es, v.a)) return rc;
  if (int rc = take_pointers(p, "checkpoint", checkpoint, v.tokens, 16, v.b)) return rc;
  a.all = p->host.cfg.world;
  Memory m;
  for (uint32_t w = 0; w < a.all; ++w) {
    m.add_rows(v.a[w], v.tokens[w], pitch, features, es, !store);
    m.add(v.b[w], checkpoint_size(v.tokens[w], features), store);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  a.features = uint32_t(features);
  a.pitch = pitch;
  a.bf16 = dtype == CARAMEL_BF16;
  if (tracing())
    std::fprintf(stderr, "caramel: checkpoint %s stream %p, %u workers, up to %u tokens, %u features\n", store ? "store" : "load",
                 (void*)stream, a.all, a.max_tokens, a.features);
  HIP_TRY(store ? launch_checkpoint_store(a, v, stream) : launch_checkpoint_load(a, v, stream));
  return CARAMEL_OK;
}

int weight_workspace(const caramel_plan* p, uint32_t weight, uint64_t features, const uint64_t* tokens, uint64_t* bytes) {
  if (!p || !bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  uint64_t outputs = 0;
  uint32_t n[CARAMEL_MAX_WORLD], most = 0;
  if (int rc = check_matrix(p, "weight", weight, features, &outputs)) return rc;
  if (int rc = check_columns("features", features)) return rc;
  if (int rc = check_columns("outputs", outputs)) return rc;
  if (int rc = take_tokens(p, tokens, n, &most)) return rc;
  *bytes = weight_gradient_workspace(p->host.cfg.world, uint32_t(features), uint32_t(outputs), most);
  return CARAMEL_OK;
}

int weight_gradient(caramel_plan* p, uint32_t weight, uint32_t bias, uint64_t features, const void* const* checkpoint,
                    const uint64_t* tokens, const void* const* dy, uint32_t dy_dtype, uint64_t dy_pitch, int accumulate, void* ws,
                    uint64_t ws_bytes, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const uint64_t es = p->host.elem_size();
  uint64_t outputs = 0;
  WeightGradientArgs a{};
  AllWorkers v{};
  if (int rc = check_matrix(p, "weight", weight, features, &outputs)) return rc;
  if (int rc = check_columns("features", features)) return rc;
  if (int rc = check_columns("outputs", outputs)) return rc;
  a.has_bias = bias != CARAMEL_NO_TENSOR;
  if (a.has_bias) {
    if (bias >= p->host.tensor_elems.size() || bias == weight || p->host.tensor_elems[bias] != outputs)
      return fail(CARAMEL_EINVAL, "tensor %u is no bias of %llu outputs", bias, (unsigned long long)outputs);
  }
  if (int rc = check_dtype("dy_dtype", dy_dtype)) return rc;
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("dy_pitch", dy_pitch, outputs, a.max_tokens)) return rc;
  if (uint64_t(a.max_tokens) * features > kMaxValues) return fail(CARAMEL_EINVAL, "more than 2^38 values at one worker");
  if (int rc = take_pointers(p, "checkpoint", checkpoint, v.tokens, 16, v.a)) return rc;
  if (int rc = take_pointers(p, "dy", dy, v.tokens, size_of(dy_dtype), v.b)) return rc;
  a.all = p->host.cfg.world;
  const uint64_t need = weight_gradient_workspace(a.all, uint32_t(features), uint32_t(outputs), a.max_tokens);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  if (int rc = need_bound(p, false)) return rc;
  Memory m;
  m.add(reinterpret_cast<uint64_t>(ws), need, true);
  for (uint32_t w = 0; w < a.all; ++w) {
    v.c[w] = p->bind.rows[weight * a.all + w];
    m.add(v.c[w], features * outputs * es, true);
    if (a.has_bias) {
      v.d[w] = p->bind.rows[bias * a.all + w];
      m.add(v.d[w], outputs * es, true);
    }
    m.add(v.a[w], checkpoint_size(v.tokens[w], features), false);
    m.add_rows(v.b[w], v.tokens[w], dy_pitch, outputs, size_of(dy_dtype), false);
  }
  if (int rc = check_memory(m)) return rc;
  a.features = uint32_t(features);
  a.outputs = uint32_t(outputs);
  a.dy_pitch = dy_pitch;
  a.dy_bf16 = dy_dtype == CARAMEL_BF16;
  a.out_bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.accumulate = accumulate != 0;
  a.ws = static_cast<unsigned char*>(ws);
  if (tracing())
    std::fprintf(stderr, "caramel: weight gradient stream %p, tensor %u, %u workers, up to %u tokens, %u x %u\n", (void*)stream,
                 weight, a.all, a.max_tokens, a.features, a.outputs);
  HIP_TRY(launch_weight_gradient(a, v, stream));
  return CARAMEL_OK;
}

// ---- before and between them ----------------------------------------------------------------

// As take_pointers; a call may go without them: addresses 0.
int take_optional(const caramel_plan* p, const char* name, const void* const* from, const uint32_t* tokens, uint64_t align,
                  uint64_t* out) {
  return from ? take_pointers(p, name, from, tokens, align, out) : int(CARAMEL_OK);
}

int check_norm_width(uint64_t width) {
  if (width == 0 || width > kNormWidth)
    return fail(CARAMEL_EINVAL, "width must be 1 to %u, is %llu", kNormWidth, (unsigned long long)width);
  return CARAMEL_OK;
}

int residual_norm(caramel_plan* p, const void* const* gain, uint64_t width, float eps, const uint64_t* tokens, const void* const* x,
                  const void* const* residual, uint32_t dtype, uint64_t pitch, void* const* sum, void* const* y, float* const* rstd,
                  void* const* checkpoint, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const uint64_t gs = p->host.elem_size();
  NormArgs a{};
  AllBuffers<kNormBuffers> v{};
  if (int rc = check_norm_width(width)) return rc;
  if (int rc = check_dtype("dtype", dtype)) return rc;
  if (!(eps > 0.0f) || !std::isfinite(eps)) return fail(CARAMEL_EINVAL, "eps must be a positive number, is %g", double(eps));
  if ((residual != nullptr) != (sum != nullptr)) return fail(CARAMEL_EINVAL, "residual and sum go together");
  const uint64_t es = size_of(dtype);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("pitch", pitch, width, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "gain", gain, v.tokens, gs, v.at[kNormGain])) return rc;
  if (int rc = take_pointers(p, "x", x, v.tokens, es, v.at[kNormX])) return rc;
  if (int rc = take_optional(p, "residual", residual, v.tokens, es, v.at[kNormResidual])) return rc;
  if (int rc = take_optional(p, "sum", sum, v.tokens, es, v.at[kNormSum])) return rc;
  if (int rc = take_pointers(p, "y", y, v.tokens, es, v.at[kNormY])) return rc;
  if (int rc = take_pointers(p, "rstd", reinterpret_cast<const void* const*>(rstd), v.tokens, 4, v.at[kNormRstd])) return rc;
  if (int rc = take_optional(p, "checkpoint", checkpoint, v.tokens, 16, v.at[kNormCheckpoint])) return rc;
  a.all = p->host.cfg.world;
  Memory m;
  for (uint32_t w = 0; w < a.all; ++w) {
    const uint64_t n = v.tokens[w];
    if (!n) continue;
    m.add(v.at[kNormGain][w], width * gs, false);
    m.add_rows(v.at[kNormX][w], n, pitch, width, es, false);
    m.add_rows(v.at[kNormY][w], n, pitch, width, es, true);
    m.add(v.at[kNormRstd][w], n * 4, true);
    if (residual) m.add_rows(v.at[kNormResidual][w], n, pitch, width, es, false);
    if (sum) m.add_rows(v.at[kNormSum][w], n, pitch, width, es, true);
    if (checkpoint) m.add(v.at[kNormCheckpoint][w], checkpoint_size(n, width), true);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  a.width = uint32_t(width);
  a.pitch = pitch;
  a.eps = eps;
  a.bf16 = dtype == CARAMEL_BF16;
  a.gain_bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.residual = residual != nullptr;
  a.checkpoint = checkpoint != nullptr;
  if (tracing())
    std::fprintf(stderr, "caramel: residual norm stream %p, %u workers, up to %u tokens, %u columns\n", (void*)stream, a.all,
                 a.max_tokens, a.width);
  HIP_TRY(launch_norm(a, v, stream));
  return CARAMEL_OK;
}

int check_gain(const caramel_plan* p, uint32_t gain_tensor, uint64_t* width) {
  uint64_t rows = 0;
  if (int rc = check_matrix(p, "gain", gain_tensor, 1, &rows)) return rc;
  *width = rows;
  return check_norm_width(rows);
}

int residual_norm_workspace(const caramel_plan* p, uint32_t gain_tensor, const uint64_t* tokens, uint64_t* bytes) {
  if (!p || !bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  uint64_t width = 0;
  uint32_t n[CARAMEL_MAX_WORLD], most = 0;
  if (int rc = check_gain(p, gain_tensor, &width)) return rc;
  if (int rc = take_tokens(p, tokens, n, &most)) return rc;
  *bytes = norm_gradient_workspace(p->host.cfg.world, uint32_t(width), most);
  return CARAMEL_OK;
}

int residual_norm_gradient(caramel_plan* p, uint32_t gain_tensor, const void* const* gain, const uint64_t* tokens,
                           const void* const* x, const float* const* rstd, const void* const* dy, const void* const* dsum,
                           uint32_t dtype, uint64_t pitch, void* const* dx, int accumulate, void* ws, uint64_t ws_bytes,
                           hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  const uint64_t gs = p->host.elem_size();
  uint64_t width = 0;
  NormGradientArgs a{};
  AllBuffers<kNormGradBuffers> v{};
  if (int rc = check_gain(p, gain_tensor, &width)) return rc;
  if (int rc = check_dtype("dtype", dtype)) return rc;
  const uint64_t es = size_of(dtype);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("pitch", pitch, width, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "gain", gain, v.tokens, gs, v.at[kNormGradGain])) return rc;
  if (int rc = take_pointers(p, "x", x, v.tokens, es, v.at[kNormGradX])) return rc;
  if (int rc = take_pointers(p, "rstd", reinterpret_cast<const void* const*>(rstd), v.tokens, 4, v.at[kNormGradRstd])) return rc;
  if (int rc = take_pointers(p, "dy", dy, v.tokens, es, v.at[kNormGradDy])) return rc;
  if (int rc = take_optional(p, "dsum", dsum, v.tokens, es, v.at[kNormGradDsum])) return rc;
  if (int rc = take_pointers(p, "dx", dx, v.tokens, es, v.at[kNormGradDx])) return rc;
  a.all = p->host.cfg.world;
  const uint64_t need = norm_gradient_workspace(a.all, uint32_t(width), a.max_tokens);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  if (int rc = need_bound(p, false)) return rc;
  Memory m;
  m.add(reinterpret_cast<uint64_t>(ws), need, true);
  for (uint32_t w = 0; w < a.all; ++w) {
    const uint64_t n = v.tokens[w];
    v.at[kNormGradOut][w] = p->bind.rows[gain_tensor * a.all + w];
    m.add(v.at[kNormGradOut][w], width * gs, true);
    if (!n) continue;
    m.add(v.at[kNormGradGain][w], width * gs, false);
    m.add(v.at[kNormGradRstd][w], n * 4, false);
    m.add_rows(v.at[kNormGradX][w], n, pitch, width, es, false);
    m.add_rows(v.at[kNormGradDy][w], n, pitch, width, es, false);
    m.add_rows(v.at[kNormGradDx][w], n, pitch, width, es, true);
    if (dsum) m.add_rows(v.at[kNormGradDsum][w], n, pitch, width, es, false);
  }
  if (int rc = check_memory(m)) return rc;
  a.width = uint32_t(width);
  a.pitch = pitch;
  a.bf16 = dtype == CARAMEL_BF16;
  a.gain_bf16 = p->host.cfg.dtype == CARAMEL_BF16;
  a.dsum = dsum != nullptr;
  a.accumulate = accumulate != 0;
  a.ws = static_cast<unsigned char*>(ws);
  if (tracing())
    std::fprintf(stderr, "caramel: residual norm gradient stream %p, tensor %u, %u workers, up to %u tokens, %u columns\n",
                 (void*)stream, gain_tensor, a.all, a.max_tokens, a.width);
  HIP_TRY(launch_norm_gradient(a, v, stream));
  return CARAMEL_OK;
}

int recurrence_workspace(const caramel_plan* p, uint64_t channels, const uint64_t* tokens, uint64_t* bytes) {
  if (!p || !bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  uint32_t n[CARAMEL_MAX_WORLD], most = 0;
  if (int rc = check_columns("channels", channels)) return rc;
  if (int rc = take_tokens(p, tokens, n, &most)) return rc;
  *bytes = recurrence_workspace_bytes(p->host.cfg.world, uint32_t(channels), n);
  return CARAMEL_OK;
}

// What the recurrence and its gradient have in common: sizes, sequences, and what both read.
int take_recurrence(caramel_plan* p, uint64_t channels, const uint64_t* tokens, const uint64_t* sequences, const void* const* starts,
                    uint32_t id_bytes, const void* const* gate, const void* const* input, uint32_t dtype, uint64_t pitch,
                    const float* const* before, uint64_t states_pitch, void* ws, uint64_t ws_bytes, RecurrenceArgs& a,
                    AllBuffers<kRecBuffers>& v, Memory& m) {
  if (int rc = check_columns("channels", channels)) return rc;
  if (id_bytes != 4 && id_bytes != 8) return fail(CARAMEL_EINVAL, "id_bytes must be 4 or 8, is %u", id_bytes);
  if (int rc = check_dtype("dtype", dtype)) return rc;
  const uint64_t es = size_of(dtype);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (!sequences) return fail(CARAMEL_EINVAL, "sequences is NULL");
  a.all = p->host.cfg.world;
  for (uint32_t w = 0; w < a.all; ++w) {
    if (sequences[w] > kMaxTokens)
      return fail(CARAMEL_EINVAL, "sequences[%u] = %llu is more than 2^25", w, (unsigned long long)sequences[w]);
    if (sequences[w] && !v.tokens[w])
      return fail(CARAMEL_EINVAL, "sequences[%u] = %llu, but the worker has no tokens", w, (unsigned long long)sequences[w]);
    v.more[w] = uint32_t(sequences[w]);
  }
  if (int rc = check_rows("pitch", pitch, channels, a.max_tokens)) return rc;
  if (int rc = check_rows("states_pitch", states_pitch, channels, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "starts", starts, v.tokens, id_bytes, v.at[kRecStarts])) return rc;
  if (int rc = take_pointers(p, "gate", gate, v.tokens, es, v.at[kRecGate])) return rc;
  if (int rc = take_pointers(p, "input", input, v.tokens, es, v.at[kRecInput])) return rc;
  if (int rc = take_optional(p, "before", reinterpret_cast<const void* const*>(before), v.tokens, 4, v.at[kRecBefore])) return rc;
  const uint64_t need = recurrence_workspace_bytes(a.all, uint32_t(channels), v.tokens);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  m.add(reinterpret_cast<uint64_t>(ws), need, true);
  for (uint32_t w = 0; w < a.all; ++w) {
    const uint64_t n = v.tokens[w];
    if (!n) continue;
    m.add(v.at[kRecStarts][w], (uint64_t(v.more[w]) + 1) * id_bytes, false);
    m.add_rows(v.at[kRecGate][w], n, pitch, channels, es, false);
    m.add_rows(v.at[kRecInput][w], n, pitch, channels, es, false);
    if (before) m.add(v.at[kRecBefore][w], v.more[w] * channels * 4, false);
  }
  a.channels = uint32_t(channels);
  a.pitch = pitch;
  a.states_pitch = states_pitch;
  a.bf16 = dtype == CARAMEL_BF16;
  a.starts64 = id_bytes == 8;
  a.ws = static_cast<unsigned char*>(ws);
  return CARAMEL_OK;
}

int recurrence(caramel_plan* p, uint64_t channels, const uint64_t* tokens, const uint64_t* sequences, const void* const* starts,
               uint32_t id_bytes, const void* const* gate, const void* const* input, uint32_t dtype, uint64_t pitch,
               const float* const* before, void* const* states, uint64_t states_pitch, float* const* after, void* ws, uint64_t ws_bytes,
               hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  RecurrenceArgs a{};
  AllBuffers<kRecBuffers> v{};
  Memory m;
  if (int rc = take_recurrence(p, channels, tokens, sequences, starts, id_bytes, gate, input, dtype, pitch, before, states_pitch, ws,
                               ws_bytes, a, v, m))
    return rc;
  const uint64_t es = size_of(dtype);
  if (int rc = take_pointers(p, "states", states, v.tokens, es, v.at[kRecStates])) return rc;
  if (int rc = take_optional(p, "after", reinterpret_cast<const void* const*>(after), v.tokens, 4, v.at[kRecAfter])) return rc;
  for (uint32_t w = 0; w < a.all; ++w) {
    if (!v.tokens[w]) continue;
    m.add_rows(v.at[kRecStates][w], v.tokens[w], states_pitch, channels, es, true);
    if (after) m.add(v.at[kRecAfter][w], v.more[w] * channels * 4, true);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  if (tracing())
    std::fprintf(stderr, "caramel: recurrence stream %p, %u workers, up to %u tokens, %u channels\n", (void*)stream, a.all,
                 a.max_tokens, a.channels);
  HIP_TRY(launch_recurrence(a, v, stream));
  return CARAMEL_OK;
}

int recurrence_gradient(caramel_plan* p, uint64_t channels, const uint64_t* tokens, const uint64_t* sequences,
                        const void* const* starts, uint32_t id_bytes, const void* const* gate, const void* const* input, uint32_t dtype,
                        uint64_t pitch, const float* const* before, const void* const* states, const void* const* dstates,
                        uint64_t states_pitch, const float* const* dafter, void* const* dgate, void* const* dinput,
                        float* const* dbefore, void* ws, uint64_t ws_bytes, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  RecurrenceArgs a{};
  AllBuffers<kRecBuffers> v{};
  Memory m;
  if (int rc = take_recurrence(p, channels, tokens, sequences, starts, id_bytes, gate, input, dtype, pitch, before, states_pitch, ws,
                               ws_bytes, a, v, m))
    return rc;
  const uint64_t es = size_of(dtype);
  if (int rc = take_pointers(p, "states", states, v.tokens, es, v.at[kRecStates])) return rc;
  if (int rc = take_pointers(p, "dstates", dstates, v.tokens, es, v.at[kRecDstates])) return rc;
  if (int rc = take_optional(p, "dafter", reinterpret_cast<const void* const*>(dafter), v.tokens, 4, v.at[kRecDafter])) return rc;
  if (int rc = take_pointers(p, "dgate", dgate, v.tokens, es, v.at[kRecDgate])) return rc;
  if (int rc = take_pointers(p, "dinput", dinput, v.tokens, es, v.at[kRecDinput])) return rc;
  if (int rc = take_optional(p, "dbefore", reinterpret_cast<const void* const*>(dbefore), v.tokens, 4, v.at[kRecDbefore])) return rc;
  for (uint32_t w = 0; w < a.all; ++w) {
    const uint64_t n = v.tokens[w];
    if (!n) continue;
    m.add_rows(v.at[kRecStates][w], n, states_pitch, channels, es, false);
    m.add_rows(v.at[kRecDstates][w], n, states_pitch, channels, es, false);
    m.add_rows(v.at[kRecDgate][w], n, pitch, channels, es, true);
    m.add_rows(v.at[kRecDinput][w], n, pitch, channels, es, true);
    if (dafter) m.add(v.at[kRecDafter][w], v.more[w] * channels * 4, false);
    if (dbefore) m.add(v.at[kRecDbefore][w], v.more[w] * channels * 4, true);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  if (tracing())
    std::fprintf(stderr, "caramel: recurrence gradient stream %p, %u workers, up to %u tokens, %u channels\n", (void*)stream, a.all,
                 a.max_tokens, a.channels);
  HIP_TRY(launch_recurrence_gradient(a, v, stream));
  return CARAMEL_OK;
}

int check_distillation(uint64_t vocab, uint32_t top) {
  if (int rc = check_columns("vocab", vocab)) return rc;
  if (top == 0 || top > kDistillationTop) return fail(CARAMEL_EINVAL, "top must be 1 to %u, is %u", kDistillationTop, top);
  return CARAMEL_OK;
}

int distillation_workspace(const caramel_plan* p, uint64_t vocab, uint32_t top, const uint64_t* tokens, uint64_t* bytes) {
  if (!p || !bytes) return fail(CARAMEL_EINVAL, "NULL argument");
  uint32_t n[CARAMEL_MAX_WORLD], most = 0;
  if (int rc = check_distillation(vocab, top)) return rc;
  if (int rc = take_tokens(p, tokens, n, &most)) return rc;
  *bytes = distillation_workspace_bytes(p->host.cfg.world, uint32_t(vocab), most);
  return CARAMEL_OK;
}

int distillation(caramel_plan* p, uint64_t vocab, const uint64_t* tokens, const void* const* logits, uint32_t dtype, uint64_t pitch,
                 const void* const* teacher_ids, const void* const* labels, uint32_t id_bytes, const void* const* teacher_logits,
                 uint32_t teacher_dtype, uint32_t top, float temperature, float soft, float hard, float scale, float* const* loss,
                 void* const* dlogits, uint64_t dlogits_pitch, void* ws, uint64_t ws_bytes, hipStream_t stream) {
  if (!p) return fail(CARAMEL_EINVAL, "plan is NULL");
  DistillationArgs a{};
  AllBuffers<kDistBuffers> v{};
  if (int rc = check_distillation(vocab, top)) return rc;
  if (id_bytes != 4 && id_bytes != 8) return fail(CARAMEL_EINVAL, "id_bytes must be 4 or 8, is %u", id_bytes);
  if (int rc = check_dtype("dtype", dtype)) return rc;
  if (int rc = check_dtype("teacher_dtype", teacher_dtype)) return rc;
  if (!(temperature >= 1.0f / 1024 && temperature <= 1024.0f))
    return fail(CARAMEL_EINVAL, "temperature must be 1/1024 to 1024, is %g", double(temperature));
  if (!(soft >= 0.0f) || !(hard >= 0.0f) || !std::isfinite(soft) || !std::isfinite(hard) || (soft == 0.0f && hard == 0.0f))
    return fail(CARAMEL_EINVAL, "soft and hard must be numbers from 0 on, not both 0, are %g and %g", double(soft), double(hard));
  if (!std::isfinite(scale)) return fail(CARAMEL_EINVAL, "scale must be a number, is %g", double(scale));
  if (hard > 0.0f && !labels) return fail(CARAMEL_EINVAL, "hard is not 0, and labels is NULL");
  const uint64_t es = size_of(dtype), ts = size_of(teacher_dtype);
  if (int rc = take_tokens(p, tokens, v.tokens, &a.max_tokens)) return rc;
  if (int rc = check_rows("pitch", pitch, vocab, a.max_tokens)) return rc;
  if (dlogits)
    if (int rc = check_rows("dlogits_pitch", dlogits_pitch, vocab, a.max_tokens)) return rc;
  if (int rc = take_pointers(p, "logits", logits, v.tokens, es, v.at[kDistLogits])) return rc;
  if (int rc = take_pointers(p, "teacher_ids", teacher_ids, v.tokens, id_bytes, v.at[kDistIds])) return rc;
  if (int rc = take_pointers(p, "teacher_logits", teacher_logits, v.tokens, ts, v.at[kDistTeacher])) return rc;
  if (int rc = take_optional(p, "labels", labels, v.tokens, id_bytes, v.at[kDistLabels])) return rc;
  if (int rc = take_pointers(p, "loss", reinterpret_cast<const void* const*>(loss), v.tokens, 4, v.at[kDistLoss])) return rc;
  if (int rc = take_optional(p, "dlogits", dlogits, v.tokens, es, v.at[kDistGradient])) return rc;
  a.all = p->host.cfg.world;
  const uint64_t need = distillation_workspace_bytes(a.all, uint32_t(vocab), a.max_tokens);
  if (int rc = check_workspace(ws, ws_bytes, need)) return rc;
  Memory m;
  m.add(reinterpret_cast<uint64_t>(ws), need, true);
  for (uint32_t w = 0; w < a.all; ++w) {
    const uint64_t n = v.tokens[w];
    if (!n) continue;
    const bool in_place = dlogits && v.at[kDistGradient][w] == v.at[kDistLogits][w] && dlogits_pitch == pitch;
    if (!in_place) m.add_rows(v.at[kDistLogits][w], n, pitch, vocab, es, false);
    m.add(v.at[kDistIds][w], n * top * id_bytes, false);
    m.add(v.at[kDistTeacher][w], n * top * ts, false);
    if (labels) m.add(v.at[kDistLabels][w], n * id_bytes, false);
    m.add(v.at[kDistLoss][w], n * 4, true);
    if (dlogits) m.add_rows(v.at[kDistGradient][w], n, dlogits_pitch, vocab, es, true);
  }
  if (int rc = check_memory(m)) return rc;
  if (int rc = need_device(p)) return rc;
  a.vocab = uint32_t(vocab);
  a.top = top;
  a.pitch = pitch;
  a.gradient_pitch = dlogits_pitch;
  a.temperature = temperature;
  a.soft = soft;
  a.hard = hard;
  a.scale = scale;
  a.bf16 = dtype == CARAMEL_BF16;
  a.teacher_bf16 = teacher_dtype == CARAMEL_BF16;
  a.ids64 = id_bytes == 8;
  a.has_labels = hard > 0.0f;
  a.gradient = dlogits != nullptr;
  a.ws = static_cast<unsigned char*>(ws);
  if (tracing())
    std::fprintf(stderr, "caramel: distillation stream %p, %u workers, up to %u tokens, %u logits\n", (void*)stream, a.all,
                 a.max_tokens, a.vocab);
  HIP_TRY(launch_distillation(a, v, stream));
  return CARAMEL_OK;
}

}  // namespace

int caramel_embedding_lookup(caramel_plan* p, const void* const* table, uint64_t vocab, uint64_t width, float scale,
                             const void* const* ids, uint32_t id_bytes, const uint64_t* tokens, void* const* out,
                             uint64_t out_pitch, void* stream) {
  return guarded([&] {
    return embedding_lookup(p, table, vocab, width, scale, ids, id_bytes, tokens, out, out_pitch, hipStream_t(stream));
  });
}

int caramel_embedding_workspace(const caramel_plan* p, uint32_t tensor, uint64_t width, const uint64_t* tokens, uint64_t* bytes) {
  return guarded([&] { return embedding_workspace(p, tensor, width, tokens, bytes); });
}

int caramel_embedding_gradient(caramel_plan* p, uint32_t tensor, uint64_t width, float scale, const void* const* ids,
                               uint32_t id_bytes, const uint64_t* tokens, const void* const* dy, uint32_t dy_dtype,
                               uint64_t dy_pitch, int accumulate, void* ws, uint64_t ws_bytes, void* stream) {
  return guarded([&] {
    return embedding_gradient(p, tensor, width, scale, ids, id_bytes, tokens, dy, dy_dtype, dy_pitch, accumulate, ws, ws_bytes,
                              hipStream_t(stream));
  });
}

int caramel_checkpoint_bytes(uint64_t tokens, uint64_t features, uint64_t* bytes) {
  return guarded([&]() -> int {
    if (!bytes) return fail(CARAMEL_EINVAL, "NULL argument");
    if (int rc = check_columns("features", features)) return rc;
    if (tokens > kMaxTokens) return fail(CARAMEL_EINVAL, "tokens = %llu is more than 2^25", (unsigned long long)tokens);
    *bytes = checkpoint_size(tokens, features);
    return CARAMEL_OK;
  });
}

int caramel_checkpoint_store(caramel_plan* p, const uint64_t* tokens, uint64_t features, const void* const* x, uint32_t dtype,
                             uint64_t pitch, void* const* checkpoint, void* stream) {
  return guarded([&] { return checkpoint_call(p, true, tokens, features, x, dtype, pitch, checkpoint, hipStream_t(stream)); });
}

int caramel_checkpoint_load(caramel_plan* p, const uint64_t* tokens, uint64_t features, const void* const* checkpoint,
                            void* const* x, uint32_t dtype, uint64_t pitch, void* stream) {
  return guarded([&] { return checkpoint_call(p, false, tokens, features, x, dtype, pitch, checkpoint, hipStream_t(stream)); });
}

int caramel_weight_gradient_workspace(const caramel_plan* p, uint32_t weight, uint64_t features, const uint64_t* tokens,
                                      uint64_t* bytes) {
  return guarded([&] { return weight_workspace(p, weight, features, tokens, bytes); });
}

int caramel_weight_gradient(caramel_plan* p, uint32_t weight, uint32_t bias, uint64_t features, const void* const* checkpoint,
                            const uint64_t* tokens, const void* const* dy, uint32_t dy_dtype, uint64_t dy_pitch, int accumulate,
                            void* ws, uint64_t ws_bytes, void* stream) {
  return guarded([&] {
    return weight_gradient(p, weight, bias, features, checkpoint, tokens, dy, dy_dtype, dy_pitch, accumulate, ws, ws_bytes,
                           hipStream_t(stream));
  });
}

int caramel_residual_norm(caramel_plan* p, const void* const* gain, uint64_t width, float eps, const uint64_t* tokens,
                          const void* const* x, const void* const* residual, uint32_t dtype, uint64_t pitch, void* const* sum,
                          void* const* y, float* const* rstd, void* const* checkpoint, void* stream) {
  return guarded([&] {
    return residual_norm(p, gain, width, eps, tokens, x, residual, dtype, pitch, sum, y, rstd, checkpoint, hipStream_t(stream));
  });
}

int caramel_residual_norm_workspace(const caramel_plan* p, uint32_t gain_tensor, const uint64_t* tokens, uint64_t* bytes) {
  return guarded([&] { return residual_norm_workspace(p, gain_tensor, tokens, bytes); });
}

int caramel_residual_norm_gradient(caramel_plan* p, uint32_t gain_tensor, const void* const* gain, const uint64_t* tokens,
                                   const void* const* x, const float* const* rstd, const void* const* dy, const void* const* dsum,
                                   uint32_t dtype, uint64_t pitch, void* const* dx, int accumulate, void* ws, uint64_t ws_bytes,
                                   void* stream) {
  return guarded([&] {
    return residual_norm_gradient(p, gain_tensor, gain, tokens, x, rstd, dy, dsum, dtype, pitch, dx, accumulate, ws, ws_bytes,
                                  hipStream_t(stream));
  });
}

int caramel_recurrence_workspace(const caramel_plan* p, uint64_t channels, const uint64_t* tokens, uint64_t* bytes) {
  return guarded([&] { return recurrence_workspace(p, channels, tokens, bytes); });
}

int caramel_recurrence(caramel_plan* p, uint64_t channels, const uint64_t* tokens, const uint64_t* sequences,
                       const void* const* starts, uint32_t id_bytes, const void* const* gate, const void* const* input, uint32_t dtype,
                       uint64_t pitch, const float* const* before, void* const* states, uint64_t states_pitch, float* const* after,
                       void* ws, uint64_t ws_bytes, void* stream) {
  return guarded([&] {
    return recurrence(p, channels, tokens, sequences, starts, id_bytes, gate, input, dtype, pitch, before, states, states_pitch, after,
                      ws, ws_bytes, hipStream_t(stream));
  });
}

int caramel_recurrence_gradient(caramel_plan* p, uint64_t channels, const uint64_t* tokens, const uint64_t* sequences,
                                const void* const* starts, uint32_t id_bytes, const void* const* gate, const void* const* input,
                                uint32_t dtype, uint64_t pitch, const float* const* before, const void* const* states,
                                const void* const* dstates, uint64_t states_pitch, const float* const* dafter, void* const* dgate,
                                void* const* dinput, float* const* dbefore, void* ws, uint64_t ws_bytes, void* stream) {
  return guarded([&] {
    return recurrence_gradient(p, channels, tokens, sequences, starts, id_bytes, gate, input, dtype, pitch, before, states, dstates,
                               states_pitch, dafter, dgate, dinput, dbefore, ws, ws_bytes, hipStream_t(stream));
  });
}

int caramel_distillation_workspace(const caramel_plan* p, uint64_t vocab, uint32_t top, const uint64_t* tokens, uint64_t* bytes) {
  return guarded([&] { return distillation_workspace(p, vocab, top, tokens, bytes); });
}

int caramel_distillation(caramel_plan* p, uint64_t vocab, const uint64_t* tokens, const void* const* logits, uint32_t dtype,
                         uint64_t pitch, const void* const* teacher_ids, const void* const* labels, uint32_t id_bytes,
                         const void* const* teacher_logits, uint32_t teacher_dtype, uint32_t top, float temperature, float soft,
                         float hard, float scale, float* const* loss, void* const* dlogits, uint64_t dlogits_pitch, void* ws,
                         uint64_t ws_bytes, void* stream) {
  return guarded([&] {
    return distillation(p, vocab, tokens, logits, dtype, pitch, teacher_ids, labels, id_bytes, teacher_logits, teacher_dtype, top,
                        temperature, soft, hard, scale, loss, dlogits, dlogits_pitch, ws, ws_bytes, hipStream_t(stream));
  });
}

int caramel_allreduce_loop(caramel_plan* p, void* stream, uint32_t n_calls, double* host_us_per_call,
                           double* stream_us_per_call) {
  return guarded([&]() -> int {
    if (!host_us_per_call || !stream_us_per_call || n_calls == 0) return fail(CARAMEL_EINVAL, "NULL argument or no calls");
    const bool direct = p && reduces_in_place(p);
    if (int rc = need_bound(p, !direct)) return rc;
    hipStream_t s = hipStream_t(stream);
    hipEvent_t e0 = nullptr, e1 = nullptr;
    HIP_TRY(hipEventCreate(&e0));
    if (hipEventCreate(&e1) != hipSuccess) {
      (void)hipEventDestroy(e0);
      return fail(CARAMEL_EHIP, "hipEventCreate failed");
    }
    int rc = CARAMEL_OK;
    hipError_t he = hipStreamSynchronize(s);
    if (he == hipSuccess) he = hipEventRecord(e0, s);
    const auto t0 = std::chrono::steady_clock::now();
    for (uint32_t i = 0; i < n_calls && !rc && he == hipSuccess; ++i) rc = pipeline(p, s, true, direct);
    const auto t1 = std::chrono::steady_clock::now();
    if (he == hipSuccess) he = hipEventRecord(e1, s);
    if (he == hipSuccess) he = hipEventSynchronize(e1);
    float ms = 0.f;
    if (he == hipSuccess) he = hipEventElapsedTime(&ms, e0, e1);
    (void)hipEventDestroy(e0);
    (void)hipEventDestroy(e1);
    if (rc) return rc;
    if (he != hipSuccess) return fail(CARAMEL_EHIP, "timing the loop: %s", hipGetErrorString(he));
    *host_us_per_call = std::chrono::duration<double, std::micro>(t1 - t0).count() / n_calls;
    *stream_us_per_call = double(ms) * 1e3 / n_calls;
    return CARAMEL_OK;
  });
}

int caramel_profile(caramel_plan* p, int enable) {
  if (int rc = need_bound(p, false)) return rc;
  for (int s = 0; s < 2; ++s)
    if (p->streams[s]) HIP_TRY(hipStreamSynchronize(p->streams[s]));
  drop_events(p);
  std::memset(p->stats, 0, sizeof p->stats);
  p->profiling = enable < 0 ? 0 : (enable > 2 ? 2 : enable);
  return CARAMEL_OK;
}

namespace {
int read_profile(caramel_plan* p, caramel_kernel_stat* out);
}

int caramel_profile_read(caramel_plan* p, caramel_kernel_stat* out) {
  return guarded([&] { return read_profile(p, out); });
}

}  // extern "C"

namespace {
int read_profile(caramel_plan* p, caramel_kernel_stat* out) {
  if (int rc = need_bound(p, false)) return rc;
  if (!out) return fail(CARAMEL_EINVAL, "out is NULL");
  // every pending stop event has completed once its own synchronize returns
  struct Window {
    float lo, hi;
    bool any;
  };
  size_t bi = 0;
  for (size_t i = 0; i < p->pending.size();) {
    const uint64_t call = p->pending[i].call;
    while (bi < p->call_base.size() && p->call_base[bi].first < call) ++bi;
    hipEvent_t base = (bi < p->call_base.size() && p->call_base[bi].first == call) ? p->call_base[bi].second : nullptr;
    Window win[CARAMEL_K_COUNT] = {};
    for (; i < p->pending.size() && p->pending[i].call == call; ++i) {
      TimedLaunch& t = p->pending[i];
      HIP_TRY(hipEventSynchronize(t.stop));
      float ms = 0.f;
      HIP_TRY(hipEventElapsedTime(&ms, t.start, t.stop));
      if (t.kind == CARAMEL_K_SEQUENCE) p->stats[t.kind].launches += 1;
      p->stats[t.kind].total_ms += ms;
      if (base) {
        float a = 0.f, b = 0.f;
        HIP_TRY(hipEventElapsedTime(&a, base, t.start));
        HIP_TRY(hipEventElapsedTime(&b, base, t.stop));
        Window& w = win[t.kind];
        if (!w.any) w = {a, b, true};
        w.lo = std::min(w.lo, a);
        w.hi = std::max(w.hi, b);
      }
      p->spare.push_back(t.start);
      p->spare.push_back(t.stop);
    }
    for (int k = 0; k < CARAMEL_K_COUNT; ++k)
      if (win[k].any) {
        p->stats[k].span_ms += double(win[k].hi) - double(win[k].lo);
        p->stats[k].calls += 1;
      }
  }
  p->pending.clear();
  for (auto& b : p->call_base) p->spare.push_back(b.second);
  p->call_base.clear();
  std::memcpy(out, p->stats, sizeof p->stats);
  return CARAMEL_OK;
}
}  // namespace

extern "C" {

const char* caramel_last_error(void) { return g_err.c_str(); }

int caramel_version(void) { return 100; }

}  // extern "C"
