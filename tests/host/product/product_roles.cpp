// The roles of the product kernels (csrc/lq_product.cuh, the code itself) against one another on the host, in random order.
//
// Every thread is a fiber.  Tensor copies, matrix instructions and their commits are parties of their own, which come to pass at some later time; each turn
// goes to any warp or party that is able to go on, some of them much more often than others.  Barriers are as the hardware has them: a wait looks at a parity
// only, and who does not get his turn while a phase lasts has missed it.
//
// Shared memory, tensor memory and arrays hold the data themselves: codes and scales of few bits, so that all sums are exact and outputs have to be the
// definition's.  A copy's place holds NaN from when it is asked for until it has come, an accumulator from when its product is issued until it is through: who looks
// too early, or overwrites what is still read, gets wrong numbers.  Nothing may arrive in the shared memory of a CTA that has left or has not begun.
//
// With `lose` one of the copies never comes: waits run out (a wait that nothing can end any more is told so, one after another), and the kernel has to end, say so and
// leave nothing on its way behind.
//
// Usage: product_roles FIRST_SEED SEEDS [lose]
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <deque>
#include <functional>
#include <map>
#include <memory>
#include <random>
#include <string>
#include <vector>

#include "cuda_threads.h"
#include "lq_product.cuh"

Dim threadIdx, blockIdx, gridDim, blockDim;
using namespace lq;

static std::mt19937 rng;
static std::string what;                      // the run, for messages
static int copies, lost = -1;                 // copies so far; the one that never comes

[[noreturn]] static void fail(const char *f, ...) {
  va_list a;
  va_start(a, f);
  printf("%s: ", what.c_str());
  vprintf(f, a);
  printf("\n");
  fflush(stdout);
  _Exit(1);
}
#define CHECK(x, ...) do { if (!(x)) fail(__VA_ARGS__); } while (0)

// ---- barriers ----
struct Barrier {
  int count = 0, left = 0, bytes = 0;
  unsigned phase = 0;                         // how many are complete
};
static std::map<uint32_t, Barrier> bars;
static Barrier &barrier(uint32_t at) {
  auto it = bars.find(at);
  CHECK(it != bars.end(), "no barrier at %x", at);
  return it->second;
}

// ---- threads ----
constexpr int THREADS = FEW_THREADS, WARPS = THREADS / 32;
static_assert(FEW_THREADS == MANY_THREADS, "");
enum State { READY, AT_BAR, AT_WARP, AT_CTA, AT_CLUSTER, AT_COPIES, DONE };
struct Fiber {
  ucontext_t ctx;
  std::vector<char> stack;
  State state;
  uint32_t bar, parity;
  bool in_vain;                               // the wait has run out
  unsigned cluster_turn;
  std::deque<std::shared_ptr<int>> groups;    // of copies out of shared memory: how many are not through
  int loose, but;                             // copies of no group yet; groups that a wait lets be
  std::shared_ptr<int> group;
};
struct Warp {
  int here = 0, turn = 0;
  uint64_t values[2][32];
  double weight = 1;
};
struct Mma {
  bool commit = false, pair = false, add = false;
  std::vector<uint32_t> to;                   // of a commit
  uint32_t d = 0, a = 0, b = 0, what = 0;
};
constexpr size_t SHARED = 232448;
constexpr uint32_t BASE = 1024;
struct Cta {
  uint8_t *shared = nullptr;
  std::vector<float> tmem = std::vector<float>(512 * 128);   // [lane][column]
  std::vector<Fiber> fibers = std::vector<Fiber>(THREADS);
  Warp warps[WARPS];
  int at_barrier, done, columns;
  bool begun;
  std::deque<Mma> queue;                      // of the products that its thread has issued: in order
  double queue_weight;
};
static std::vector<Cta> ctas;                 // of the cluster
static int cluster_here;
static unsigned cluster_turn;
static std::vector<std::function<void()>> loose;   // copies, commits on their way: in any order
static ucontext_t scheduler;
static Cta *cta;                              // whose fiber runs
static Fiber *now;

static bool passed(const Fiber &f) { return (barrier(f.bar).phase & 1) != f.parity; }
static bool through(const Fiber &f) {
  int left = 0;
  for (size_t i = 0; i + f.but < f.groups.size(); i++) left += *f.groups[i];
  return left == 0;
}
static void block(State s) {
  now->state = s;
  swapcontext(&now->ctx, &scheduler);
}
void yield() { block(READY); }
void cta_barrier() {
  Cta *c = cta;
  if (++c->at_barrier == THREADS) {
    c->at_barrier = 0;
    for (Fiber &f : c->fibers)
      if (f.state == AT_CTA) f.state = READY;
    block(READY);
  } else {
    block(AT_CTA);
  }
}
const uint64_t *warp_values(uint64_t mine) {
  const int w = threadIdx.x / 32;
  Warp &warp = cta->warps[w];
  uint64_t *v = warp.values[warp.turn & 1];
  v[threadIdx.x % 32] = mine;
  if (++warp.here == 32) {
    warp.here = 0, warp.turn++;
    for (int l = 0; l < 32; l++) {
      Fiber &f = cta->fibers[32 * w + l];
      if (f.state == AT_WARP) f.state = READY;
    }
    block(READY);
  } else {
    block(AT_WARP);
  }
  return v;
}
uint8_t *cta_memory() { return cta->shared; }

// What is at a shared address of the cluster, for those who may get there.
static Cta &owner(uint32_t at) {
  CHECK((at >> 24) < ctas.size(), "no CTA %u", at >> 24);
  Cta &c = ctas[at >> 24];
  CHECK(c.begun, "shared memory of a CTA that has not begun");
  CHECK(c.done < THREADS, "something arrives in the shared memory of a CTA that has left");
  return c;
}
static uint8_t *shared_at(uint32_t at) { return owner(at).shared + ((at & 0xFFFFFF) - BASE); }
static void settle(Barrier &b) {
  CHECK(b.left >= 0, "a barrier with more arrivals than it counts");
  if (b.left == 0 && b.bytes == 0) b.phase++, b.left = b.count;
}
static void arrive(uint32_t bar) {
  owner(bar);
  Barrier &b = barrier(bar);
  b.left--;
  settle(b);
}

// ---- tensor maps ----
struct Map {
  uint8_t *base;
  long size[3], stride[2];                    // bytes, rows, planes; bytes to the next row and plane
  int width, rows;                            // of a box
};
static_assert(sizeof(Map) <= sizeof(CUtensorMap), "");
static Map map_of(const CUtensorMap *m) {
  Map r;
  memcpy(&r, m, sizeof(r));
  return r;
}
static int swizzled(const Map &m, int row, int chunk) { return m.width == 128 ? chunk ^ (row % 8) : chunk ^ (row / 2 % 4); }

namespace lq {
uint32_t shared_addr(const void *p) {
  const ptrdiff_t off = (const uint8_t *)p - cta->shared;
  CHECK(off >= 0 && off < (ptrdiff_t)SHARED, "an address that is not in shared memory");
  return (uint32_t)off + BASE + ((uint32_t)(cta - ctas.data()) << 24);
}
void bar_init(uint32_t bar, int count) {
  Barrier b;
  b.count = b.left = count;
  bars[bar] = b;
}
void bar_arrive(uint32_t bar) {
  yield();
  arrive(bar);
}
void bar_arrive_cluster(uint32_t bar) { bar_arrive(bar); }
void bar_expect(uint32_t bar, uint32_t bytes) {
  barrier(bar).bytes += (int)bytes;
  bar_arrive(bar);
}
bool bar_try(uint32_t bar, uint32_t parity) {
  now->bar = bar, now->parity = parity, now->in_vain = false;
  block(AT_BAR);                              // (gets its turn while the barrier says that it is passed)
  return !now->in_vain;
}
void tensor_g2s(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
  const Map m = map_of(map);
  CHECK(x % 16 == 0 && dst % (8 * m.width) == 0, "a copy that is not aligned");
  yield();
  memset(shared_at(dst), 0xFF, m.rows * m.width);
  if (copies++ == lost) return;
  loose.push_back([=] {
    uint8_t *to = shared_at(dst);
    for (int r = 0; r < m.rows; r++)
      for (int b = 0; b < m.width; b++) {
        const bool there = x + b >= 0 && x + b < m.size[0] && y + r >= 0 && y + r < m.size[1] && z >= 0 && z < m.size[2];
        to[r * m.width + 16 * swizzled(m, r, b / 16) + b % 16] = there ? m.base[z * m.stride[1] + (y + r) * m.stride[0] + x + b] : 0;
      }
    owner(bar);
    Barrier &b = barrier(bar);
    b.bytes -= m.rows * m.width;
    settle(b);
  });
}
void tensor_s2g(const CUtensorMap *map, uint32_t src, int x, int y, int z) {
  const Map m = map_of(map);
  CHECK(x % 16 == 0 && x >= 0 && y >= 0 && src % (8 * m.width) == 0, "a copy that is not aligned");
  yield();
  if (!now->group) now->group = std::make_shared<int>(0);
  std::shared_ptr<int> group = now->group;
  ++*group;
  loose.push_back([=] {
    const uint8_t *from = shared_at(src);
    for (int r = 0; r < m.rows; r++)
      for (int b = 0; b < m.width; b++)
        if (x + b < m.size[0] && y + r < m.size[1]) m.base[z * m.stride[1] + (y + r) * m.stride[0] + x + b] = from[r * m.width + 16 * swizzled(m, r, b / 16) + b % 16];
    --*group;
  });
}
void copies_commit() {
  if (now->group) now->groups.push_back(now->group);
  now->group.reset();
}
void wait_for_copies(int but) {
  now->but = but;
  if (!through(*now)) block(AT_COPIES);
}

void tmem_alloc(uint32_t result, int columns) {
  if (threadIdx.x % 32 == 0) {
    const uint32_t none = 0;
    memcpy(shared_at(result), &none, 4);
    cta->columns = columns;
  }
}
void tmem_free(uint32_t, int columns) {
  for (const Cta &c : ctas)
    for (const Mma &m : c.queue) CHECK(m.commit, "tensor memory is freed under a product");
  if (threadIdx.x % 32 == 0) CHECK(cta->columns == columns, "tensor memory is freed that is not there");
}
void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
  if (rng() % 512 == 0) yield();
  const int lane = (at >> 16) + threadIdx.x % 32, col = at & 0xFFFF;
  CHECK((int)(at >> 16) == 32 * (int)(threadIdx.x / 32 % 4) && col + 16 <= cta->columns, "a warp's part of tensor memory");
  for (int i = 0; i < 16; i++) r[i] = __float_as_uint(cta->tmem[lane * 512 + col + i]);
}
static void issue(Mma m) {
  yield();
  if (!m.commit && !m.add) {
    const int rows = m.what >> 16, cols = m.what & 0xFFFF;
    for (int r = 0; r < rows; r++) {
      float *d = &(m.pair ? ctas[r / 128] : *cta).tmem[r % 128 * 512 + m.d];
      std::fill(d, d + cols, NAN);
    }
  }
  cta->queue.push_back(m);
}
static void product_of(uint32_t d, Operand a, Operand b, uint32_t w, bool add, bool pair) {
  Mma m;
  m.d = d, m.a = a.at, m.b = b.at, m.what = w, m.add = add, m.pair = pair;
  const int rows = w >> 16, cols = w & 0xFFFF;
  CHECK(pair ? rows == 256 && cols % 32 == 0 && cols <= 256 && ctas.size() == 2 : rows == 128 && cols % 16 == 0 && cols > 0 && cols <= 256, "a product of %d by %d", rows, cols);
  CHECK((int)d + cols <= cta->columns, "a product beyond its tensor memory");
  issue(m);
}
void mma8_ss(uint32_t d, Operand a, Operand b, uint32_t w, bool add) { product_of(d, a, b, w, add, false); }
void pair_mma8_ss(uint32_t d, Operand a, Operand b, uint32_t w, bool add) { product_of(d, a, b, w, add, true); }
static void commit(std::vector<uint32_t> to) {
  Mma m;
  m.commit = true, m.to = to;
  issue(m);
}
void mma_commit(uint32_t bar) { commit({bar}); }
void pair_mma_commit(uint32_t bar) { commit({shared_of(bar, 0), shared_of(bar, 1)}); }

uint32_t cluster_rank() { return cta - ctas.data(); }
void cluster_arrive() {
  yield();
  now->cluster_turn = cluster_turn;
  if (++cluster_here == THREADS * (int)ctas.size()) {
    cluster_here = 0, cluster_turn++;
    for (Cta &c : ctas)
      for (Fiber &f : c.fibers)
        if (f.state == AT_CLUSTER) f.state = READY;
  }
}
void cluster_wait() {
  if (now->cluster_turn == cluster_turn) block(AT_CLUSTER);
}
void store_cluster(uint32_t addr, float x) {
  if (rng() % 64 == 0) yield();
  memcpy(shared_at(addr), &x, 4);
}
}  // namespace lq

// ---- values of codes ----
static float value[256];
static void find_values() {
  for (int c = 0; c < 256; c++) {
    const int e = c >> 3 & 15, m = c & 7;
    float v = e ? ldexpf(8 + m, e - 10) : ldexpf(m, -9);
    if (e == 15 && m == 7) v = NAN;
    value[c] = c & 128 ? -v : v;
  }
}
static uint8_t code_of(int small) {           // -2 .. 2
  const uint8_t c[] = {0xC0, 0xB8, 0x00, 0x38, 0x40};
  return c[small + 2];
}

// 32 channels of an operand's row: rows of 128 bytes, eight to 1024, the pieces of 16 bytes swizzled
static void read_row(uint32_t operand, int row, float (&x)[32]) {
  const uint32_t in = operand % 128, at = operand - in + row / 8 * 1024 + row % 8 * 128;
  const uint8_t *p = shared_at(at);
  for (int k = 0; k < 32; k++) x[k] = value[p[16 * ((in / 16 + k / 16) ^ (row % 8)) + k % 16]];
}
static void execute(Cta &from, const Mma &m) {
  const int rows = m.what >> 16, cols = m.what & 0xFFFF, half = cols / 2;
  const uint32_t own = (uint32_t)(&from - ctas.data());
  static float a[256][32], b[256][32];
  for (int r = 0; r < rows; r++) read_row(shared_of(m.a, m.pair ? r / 128 : own), m.pair ? r % 128 : r, a[r]);
  for (int c = 0; c < cols; c++) read_row(shared_of(m.b, m.pair ? c / half : own), m.pair ? c % half : c, b[c]);
  for (int r = 0; r < rows; r++) {
    float *d = &(m.pair ? ctas[r / 128] : from).tmem[r % 128 * 512 + m.d];
    for (int c = 0; c < cols; c++) {
      float s = 0;
      for (int k = 0; k < 32; k++) s += a[r][k] * b[c][k];
      d[c] = m.add ? d[c] + s : s;
    }
  }
}

// ---- a cluster ----
static std::function<void()> body;
static void enter() {
  body();
  cta->done++;
  now->state = DONE;
  swapcontext(&now->ctx, &scheduler);
}

static double some_weight() {
  const double w[] = {1, 1, 1, 0.1, 0.001, 0.00001};
  return w[rng() % 6];
}

static void run_cluster(int number, int size, int grid, std::function<void()> kernel) {
  bars.clear(), loose.clear();
  cluster_here = 0, cluster_turn = 0;
  body = kernel;
  ctas.resize(size);
  for (Cta &c : ctas) {
    if (!c.shared) c.shared = (uint8_t *)aligned_alloc(1024, SHARED);
    memset(c.shared, 0xFF, SHARED);
    std::fill(c.tmem.begin(), c.tmem.end(), NAN);
    c.at_barrier = c.done = c.columns = 0;
    c.begun = false;
    c.queue.clear();
    c.queue_weight = some_weight();
    for (Warp &w : c.warps) w = Warp{}, w.weight = some_weight();
    for (Fiber &f : c.fibers) {
      f.stack.resize(48 << 10);
      f.state = READY;
      f.groups.clear(), f.group.reset();
      getcontext(&f.ctx);
      f.ctx.uc_stack.ss_sp = f.stack.data(), f.ctx.uc_stack.ss_size = f.stack.size(), f.ctx.uc_link = &scheduler;
      makecontext(&f.ctx, enter, 0);
    }
  }
  const double loose_weight = some_weight();
  if (rng() % 3 == 0)                         // now and then all in step but for one
    for (int w = 0, slow = rng() % (WARPS * size); w < WARPS * size; w++) ctas[w / WARPS].warps[w % WARPS].weight = w == slow ? 1e-5 : 1;
  auto able = [](const Fiber &f) {
    return f.state == READY || (f.state == AT_BAR && passed(f)) || (f.state == AT_COPIES && through(f));
  };
  std::vector<std::pair<double, int>> who;    // 0 .. : warps, 1000 .. : queues, 2000: a loose party
  for (long turn = 0;; turn++) {
    CHECK(turn < 20000000, "no end");
    who.clear();
    double sum = 0;
    auto may = [&](double w, int n) { sum += w, who.push_back({sum, n}); };
    for (int c = 0; c < size; c++) {
      for (int w = 0; w < WARPS; w++)
        for (int l = 0; l < 32; l++)
          if (able(ctas[c].fibers[32 * w + l])) {
            may(ctas[c].warps[w].weight, c * WARPS + w);
            break;
          }
      if (!ctas[c].queue.empty()) may(ctas[c].queue_weight, 1000 + c);
    }
    if (!loose.empty()) may(loose_weight, 2000);
    if (who.empty()) {                        // (all lanes of a warp that wait for the same give up together, as those of a real one do)
      if (lost < 0 || lost >= copies) break;
      std::vector<int> waiting;
      for (int c = 0; c < size; c++)
        for (int w = 0; w < WARPS; w++)
          for (int l = 0; l < 32; l++)
            if (ctas[c].fibers[32 * w + l].state == AT_BAR) {
              waiting.push_back(c * WARPS + w);
              break;
            }
      if (waiting.empty()) break;
      const int n = waiting[rng() % waiting.size()];
      for (int l = 0; l < 32; l++) {
        Fiber &f = ctas[n / WARPS].fibers[n % WARPS * 32 + l];
        if (f.state == AT_BAR) f.in_vain = true, f.state = READY;
      }
      continue;
    }
    const double x = std::uniform_real_distribution<double>(0, sum)(rng);
    size_t i = 0;
    while (i + 1 < who.size() && who[i].first < x) i++;
    const int n = who[i].second;
    if (n == 2000) {
      const size_t at = rng() % loose.size();
      auto go = loose[at];
      loose[at] = loose.back();
      loose.pop_back();
      go();
    } else if (n >= 1000) {
      Cta &c = ctas[n - 1000];
      const Mma m = c.queue.front();
      c.queue.pop_front();
      if (!m.commit) execute(c, m);
      else
        for (uint32_t bar : m.to) loose.push_back([=] { arrive(bar); });
    } else {                                  // all lanes of a warp that can, each as far as it gets
      const int c = n / WARPS, w = n % WARPS;
      ctas[c].begun = true;
      for (int l = 0; l < 32; l++) {
        Fiber &f = ctas[c].fibers[32 * w + l];
        if (!able(f)) continue;
        cta = &ctas[c], now = &f;
        threadIdx.x = 32 * w + l, blockIdx.x = number * size + c, gridDim.x = grid, blockDim.x = THREADS;
        f.state = READY;
        swapcontext(&scheduler, &f.ctx);
      }
    }
  }
  for (int c = 0; c < size; c++)
    for (int t = 0; t < THREADS; t++)
      if (ctas[c].fibers[t].state != DONE) fail("thread %d of CTA %d waits for ever (%d, barrier at %x)", t, c, (int)ctas[c].fibers[t].state, ctas[c].fibers[t].bar);
}

// ---- a call ----
static long ceil_of(long a, long b) { return (a + b - 1) / b; }

static CUtensorMap map_to(void *base, long bytes, long rows, long planes, long stride, long plane, int box, int width) {
  CUtensorMap r;
  const Map m{(uint8_t *)base, {bytes, rows, planes}, {stride, plane}, width, box};
  memset(&r, 0, sizeof(r));
  memcpy(&r, &m, sizeof(m));
  return r;
}

enum Kernel { FEW_SMALL, FEW_LARGE, MANY };
template <typename T>
static void run_as(Kernel kernel, const char *type, bool wide) {
  auto pick = [](int n) { return (int)(rng() % n); };
  const bool grouped = pick(2);
  const int groups = grouped ? 1 + pick(4) : 1, in = 16 * (1 + pick(pick(2) ? 40 : 72)), blocks = ceil_of(in, PB);
  const int tile = kernel == MANY ? MANY_ROWS : kernel == FEW_LARGE ? FEW_ROWS : FEW_BOX, outs_of = kernel == MANY ? MANY_OUTS : PB;
  const int out = 1 + pick(kernel == MANY ? 700 : 400);
  int rows = 1 + pick(kernel == MANY ? 700 : kernel == FEW_LARGE ? 300 : grouped ? 90 : 32);
  if (pick(4) == 0) rows = (rows + tile - 1) / tile * tile;
  if (kernel == FEW_SMALL && !grouped) rows = std::min(rows, FEW_BOX);
  const int tiles_n = ceil_of(out, outs_of), tiles = ceil_of(rows, tile) * tiles_n;
  int split = 1, units = 1 + pick(3);
  if (kernel != MANY && !grouped && blocks >= 2 && pick(2)) split = 2 + pick(std::min(7, std::max(1, blocks - 1))), split = std::min(split, blocks), units = tiles;
  units = std::min(units, tiles);
  what += std::string(kernel == MANY ? "many" : kernel == FEW_LARGE ? "few, 128" : "few, 32") + " " + type + (wide ? " wide, " : ", ") + std::to_string(rows) + " x " + std::to_string(in) +
          " x " + std::to_string(out) + ", " + std::to_string(groups) + (grouped ? " groups, split " : " group, split ") + std::to_string(split) + ", units " + std::to_string(units);
  std::vector<int32_t> start{0};
  if (grouped) {
    start.clear();
    for (int g = 0; g <= groups; g++) start.push_back(pick(rows + 1));
    std::sort(start.begin(), start.end());
    if (pick(2)) start[0] = 0, start[groups] = rows;
  }
  const int x_stride = in + 16 * pick(3), scale_stride = rows + pick(3), N = 16 / sizeof(T);
  const int out_stride = wide ? (out + N - 1) / N * N + N * pick(2) : out + pick(3);
  std::vector<uint8_t> x((size_t)rows * x_stride, 0x7F), w((size_t)groups * out * in);
  std::vector<float> xs((size_t)blocks * scale_stride, NAN), ws((size_t)groups * ceil_of(out, PB) * blocks);
  for (int r = 0; r < rows; r++)
    for (int k = 0; k < in; k++) x[(size_t)r * x_stride + k] = code_of(pick(5) - 2);
  for (auto &c : w) c = code_of(pick(5) - 2);
  for (int b = 0; b < blocks; b++)
    for (int r = 0; r < rows; r++) xs[(size_t)b * scale_stride + r] = ldexpf(1, pick(3) - 1);
  for (auto &s : ws) s = ldexpf(1, pick(3) - 1);
  // 16 bytes of guard in front, rows behind
  std::vector<uint4> mem(((size_t)(rows + 2) * out_stride * sizeof(T)) / 16 + 3);
  memset(mem.data(), 0xA5, mem.size() * 16);
  T *const o = reinterpret_cast<T *>(mem.data() + 1) + (wide ? 0 : pick(2));
  ProductArgs a{};
  a.x_scale = xs.data(), a.w_scale = ws.data(), a.out = o, a.x_scale_stride = scale_stride, a.out_stride = out_stride, a.group_start = grouped ? start.data() : nullptr;
  a.rows = rows, a.blocks = blocks, a.outs = out, a.groups = groups, a.tiles_n = tiles_n, a.split = split, a.share = blocks / split, a.more = blocks % split;
  a.tiles_m.set((uint32_t)ceil_of(rows, tile));
  ProductMaps maps{};
  maps.x = map_to(x.data(), in, rows, 1, x_stride, (long)x_stride * rows, 128, 128);
  maps.w = map_to(w.data(), in, out, groups, in, (long)in * out, 128, 128);
  maps.more = kernel == MANY ? map_to(o, (long)out * sizeof(T), rows, 1, (long)out_stride * sizeof(T), 0, 32, 64) : map_to(x.data(), in, rows, 1, x_stride, 0, FEW_BOX, 128);
  g_product_error = 0;
  const int size = kernel == MANY ? 2 : split;
  for (int u = 0; u < units; u++)
    run_cluster(u, size, units * size, [&] {
      if (kernel == MANY) wide ? product_many_kernel<T, true>(maps, a) : product_many_kernel<T, false>(maps, a);
      else if (kernel == FEW_LARGE) wide ? product_few_kernel<T, true, FEW_ROWS>(maps, a) : product_few_kernel<T, false, FEW_ROWS>(maps, a);
      else wide ? product_few_kernel<T, true, FEW_BOX>(maps, a) : product_few_kernel<T, false, FEW_BOX>(maps, a);
    });
  const bool whole = lost < 0 || lost >= copies;
  CHECK(g_product_error == (whole ? 0 : 1), "flags %d", g_product_error);
  std::vector<uint8_t> want(mem.size() * 16, 0xA5);
  T *const e = reinterpret_cast<T *>(want.data() + ((uint8_t *)o - (uint8_t *)mem.data()));
  for (int g = 0; g < groups; g++)
    for (int r = grouped ? start[g] : 0; r < (grouped ? start[g + 1] : rows); r++)
      for (int n = 0; n < out; n++) {
        float s = 0;
        for (int b = 0; b < blocks; b++) {
          float t = 0;
          for (int k = b * PB; k < std::min(in, (b + 1) * PB); k++) t += value[x[(size_t)r * x_stride + k]] * value[w[((size_t)g * out + n) * in + k]];
          s += t * xs[(size_t)b * scale_stride + r] * ws[((size_t)g * ceil_of(out, PB) + n / PB) * blocks + b];
        }
        e[(int64_t)r * out_stride + n] = from_float<T>(s);
      }
  if (!whole) {                               // (no output is valid; all of them lie where outputs belong)
    for (int g = 0; g < groups; g++)
      for (int r = grouped ? start[g] : 0; r < (grouped ? start[g + 1] : rows); r++) std::copy_n(&o[(int64_t)r * out_stride], out, &e[(int64_t)r * out_stride]);
  }
  for (int64_t i = 0; i < (int64_t)(rows + 1) * out_stride; i++)
    CHECK(memcmp(&o[i], &e[i], sizeof(T)) == 0, "output %d of row %d is %g, not %g", (int)(i % out_stride), (int)(i / out_stride), to_float(o[i]), to_float(e[i]));
  CHECK(memcmp(mem.data(), want.data(), want.size()) == 0, "memory next to the outputs is written");
}

static void run(unsigned seed, bool lose) {
  rng.seed(seed);
  what = "seed " + std::to_string(seed) + ": ";
  copies = 0, lost = lose ? rng() % 30 : -1;
  const Kernel kernel = (Kernel)(seed % 3);
  const bool wide = seed / 3 % 2;
  if (seed / 6 % 3 == 0) run_as<float>(kernel, "f32", wide);
  else if (seed / 6 % 3 == 1) run_as<__half>(kernel, "f16", wide);
  else run_as<__nv_bfloat16>(kernel, "bf16", wide);
}

int main(int argc, char **argv) {
  const unsigned first = argc > 1 ? atoi(argv[1]) : 0, n = argc > 2 ? atoi(argv[2]) : 18;
  const bool lose = argc > 3 && argv[3] == std::string("lose");
  find_values();
  for (unsigned s = first; s < first + n; s++) run(s, lose);
  printf("%u runs\n", n);
  return 0;
}
