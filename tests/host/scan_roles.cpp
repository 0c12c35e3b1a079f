// The roles of the prompt scan (csrc/lq_scan.cuh, the code itself) against one another on the host, in random order.
//
// Every warp is a fiber that stands for its lane 0.  Tensor copies, matrix instructions and their commits are parties of their own, which
// come to pass at some later time; each turn goes to any party that is able to go on, some of them much more often than others.  Barriers
// are as the hardware has them: a wait looks at a parity only, and who does not get his turn while a phase lasts has missed it.
//
// Tiles, tensor memory and states hold tags and small numbers in place of data.  A block's share of the state is a number of its head and
// row, its first row decays by 1 or 1/2, q reads the state as it is, and the weighted scores add 1/2: outputs and states are compared with the
// recurrence over the blocks.  Apart
// from that, nothing that an instruction under way reads may change, nothing it writes may be looked at, and everybody has to come to the end.
//
// Usage: scan_roles FIRST_SEED SEEDS
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <ucontext.h>

#include <deque>
#include <functional>
#include <map>
#include <random>
#include <string>
#include <vector>

#include "cuda_on_host.h"
void read_values(uint32_t at);                // in the place of ldmatrix
#include "lq_scan.cuh"

Dim threadIdx, blockIdx, gridDim, blockDim;
using namespace lq;

namespace lq {
alignas(1024) uint8_t raw[sizeof(ScanShared)];
}

static std::mt19937 rng;
static std::string what;                      // the run, for messages

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
  int count, left, bytes = 0;
  unsigned phase = 0;                         // how many are complete
  void settle() {
    CHECK(left >= 0, "a barrier with more arrivals than it counts");
    if (left == 0 && bytes == 0) phase++, left = count;
  }
};
static std::map<uint32_t, Barrier> bars;
static Barrier &barrier(uint32_t at) {
  auto it = bars.find(at);
  CHECK(it != bars.end(), "no barrier at %u", at);
  return it->second;
}
static bool passed(uint32_t at, uint32_t parity) { return (barrier(at).phase & 1) != parity; }

// ---- parties ----
constexpr int WARPS = SCAN_THREADS / 32;
struct Fiber {
  ucontext_t ctx;
  std::vector<char> stack;
  bool done = false, at_cta_barrier = false;
  uint32_t wait_bar = 0, wait_parity = 0;     // wait_bar 0: not waiting
  double weight = 1;
  int head = 0, row = 0;                      // of the values that it has read last
};
static Fiber fibers[WARPS];
static ucontext_t scheduler;
static int now = -1;                          // the fiber that runs
static int in_cta_barrier = 0;

struct Mma {
  bool commit = false;
  uint32_t bar = 0;                           // of a commit
  uint32_t d = 0, a_tmem = 0;
  int a_tile = -1, b_tile = -1;
  bool add = false;
  uint64_t seen_a = 0, seen_b = 0;            // what the tiles held when it was issued
};
static std::map<int, std::deque<Mma>> queues; // by the warp that issued them: in order
static std::vector<std::function<void()>> loose;   // copies, commits on their way: in any order

void yield() {
  if (now >= 0) swapcontext(&fibers[now].ctx, &scheduler);
}
void cta_barrier() {
  Fiber &f = fibers[now];
  f.at_cta_barrier = true;
  if (++in_cta_barrier == WARPS) {
    in_cta_barrier = 0;
    for (Fiber &x : fibers) x.at_cta_barrier = false;
  }
  yield();
}

// ---- what tiles and tensor memory hold ----
struct Tag {
  int head, row;
};
constexpr uint32_t BASE = 1024;
constexpr int TILE_S = 6;                     // k, k, q, q, v, v, S
static int tile_of(uint32_t at) { return (at - BASE) / TILE; }
static uint8_t *tile(int i) { return raw + i * TILE; }
static Tag tag_of(int i) {
  Tag t[2];
  for (int h = 0; h < 2; h++) memcpy(&t[h], tile(i) + h * HALF, sizeof(Tag));
  CHECK(t[0].head == t[1].head && t[0].row == t[1].row && t[0].row >= 0, "tile %d is read before it is there", i);
  return t[0];
}
static float state_in_tile() {
  float s = 0;
  for (int c = 0; c < 128; c += 32)
    for (int j = 0; j < 16; j++) {            // chunk j of row c lies at j ^ 0
      __nv_bfloat16 b;
      memcpy(&b, tile(TILE_S) + c * 128 + (j / 8) * HALF + (j % 8) * 16, 2);
      const float x = __bfloat162float(b);
      if (c == 0 && j == 0) s = x;
      CHECK(x == s, "parts of different states in the tile of S");
    }
  return s;
}
static uint64_t seen(int i) {
  if (i < 0) return 0;
  uint64_t x = 0;
  if (i == TILE_S) {
    for (int c = 0; c < 128; c += 32) {
      uint64_t y;
      memcpy(&y, tile(i) + c * 128, 8);
      x = x * 1000003 + y;
    }
  } else {
    memcpy(&x, tile(i), 8);
  }
  return x;
}

// (with at most three blocks and states up to 7, sums have five bits and three behind the point: exact as bf16)
static float value_of(Tag t) { return 1 + (t.head * 5 + t.row / 16) % 7; }
static float decay_of(int head, int row) { return (head + row / 16) % 3 ? 1.0f : 0.5f; }   // of the block that starts there

struct {
  Tag tag;
  int parts, stored;
  bool used;
} P;
struct {
  Tag tag;
  float value;
  int state_parts, parts, reads;
  bool used;
} O;
struct {
  Tag tag;
  int parts, reads;
  bool used;
} DS;
struct {
  Tag tag;
  int stores, reads;
} W[2];

static bool under_way(uint32_t from, uint32_t to, bool writes_only) {
  for (auto &q : queues)
    for (const Mma &m : q.second) {
      if (m.commit) continue;
      if (m.d >= from && m.d < to) return true;
      if (!writes_only && m.a_tile < 0 && m.a_tmem >= from && m.a_tmem < to) return true;
    }
  return false;
}

static void execute(const Mma &m) {
  CHECK(m.seen_a == seen(m.a_tile) && m.seen_b == seen(m.b_tile), "a product's operand (tile %d or %d) changed while it was read", m.a_tile, m.b_tile);
  if (m.d == TM_P) {
    const Tag q = tag_of(m.a_tile), k = tag_of(m.b_tile);
    CHECK(q.row == k.row && q.head == k.head, "P of rows %d and %d", q.row, k.row);
    if (!m.add) {
      CHECK(!P.used || P.stored == 256, "P is overwritten before its weights are through");
      P = {k, 0, 0, true};
    }
    P.parts++;
  } else if (m.d == TM_O && m.a_tile >= 0) {  // Q S
    const Tag q = tag_of(m.a_tile);
    const float s = state_in_tile();
    if (!m.add) {
      CHECK(!O.used || O.reads == 32, "o is overwritten before it is read");
      O = {q, s, 0, 0, 0, true};
    }
    CHECK(O.value == s, "two states in one product");
    O.state_parts++;
  } else if (m.d == TM_O) {                   // weighted P times V
    const Tag v = tag_of(m.b_tile);
    CHECK(P.parts == 8 && P.stored == 256 && v.row == P.tag.row, "weighted P is read before it is there");
    if (!m.add) {
      CHECK(!O.used || O.reads == 32, "o is overwritten before it is read");
      O = {v, 0, 0, 0, 0, true};
    }
    CHECK(O.tag.row == v.row && (O.state_parts == 0 || O.state_parts == 8), "o of rows %d and %d", O.tag.row, v.row);
    if (++O.parts == 8) O.value += 0.5f;
  } else {
    CHECK(m.d == TM_DS, "a product to %u", m.d);
    const int u = (m.a_tmem - TM_W) / 48;
    const Tag k = tag_of(m.b_tile);
    CHECK(W[u].stores == 48 && W[u].tag.row == k.row, "weighted values are read before they are there");
    if (!m.add) {
      CHECK(!DS.used || DS.reads == 32, "dS is overwritten before it is read");
      DS = {W[u].tag, 0, 0, true};
    }
    CHECK(DS.tag.row == k.row, "dS of rows %d and %d", DS.tag.row, k.row);
    DS.parts++;
    if (++W[u].reads == 6) W[u] = {};
  }
}

void read_values(uint32_t at) {
  const Tag t = tag_of(tile_of(at));
  fibers[now].head = t.head, fibers[now].row = t.row;
}

namespace lq {
uint32_t shared_addr(const void *p) { return (uint32_t)((const uint8_t *)p - raw) + BASE; }

void bar_init(uint32_t bar, int count) { bars[bar] = Barrier{count, count}; }
static void arrive(uint32_t bar) {
  Barrier &b = barrier(bar);
  b.left--;
  b.settle();
}
void bar_arrive(uint32_t bar) {
  yield();
  arrive(bar);
}
void bar_expect(uint32_t bar, uint32_t bytes) {
  barrier(bar).bytes += (int)bytes;
  bar_arrive(bar);
}
bool bar_try(uint32_t bar, uint32_t parity) {
  fibers[now].wait_bar = bar, fibers[now].wait_parity = parity;
  yield();                                    // (gets its turn while the barrier says that it is passed)
  fibers[now].wait_bar = 0;
  return true;
}
void tensor_g2s(uint32_t dst, const CUtensorMap *, int, int head, int row, uint32_t bar) {
  yield();
  Tag none{-1, -1};
  uint8_t *to = raw + (dst - BASE);
  memcpy(to, &none, sizeof(Tag));
  loose.push_back([=] {
    const Tag t{head, row};
    memcpy(to, &t, sizeof(Tag));
    Barrier &b = barrier(bar);
    b.bytes -= HALF;
    b.settle();
  });
}
void tmem_alloc(uint32_t result, int) { memset(raw + (result - BASE), 0, 4); }
void tmem_free(uint32_t, int) { CHECK(!under_way(0, 512, false), "tensor memory is freed under a product"); }
void tmem_load16(uint32_t at, uint32_t (&r)[16]) {
  yield();
  const uint32_t col = at & 0xFFFF;
  float x = 0;
  if (col < TM_O) {
    CHECK(P.parts == 8 && !under_way(TM_P, TM_P + 128, true), "P is read before it is there");
  } else if (col < TM_DS) {
    CHECK(O.parts == 8 && !under_way(TM_O, TM_O + 128, true), "o is read before it is there");
    O.reads++;
    x = O.value;
  } else {
    CHECK(DS.parts == 24 && !under_way(TM_DS, TM_DS + 128, true), "dS is read before it is there");
    DS.reads++;
    x = value_of(DS.tag);
  }
  for (auto &y : r) y = __float_as_uint(x);
}
void tmem_store(uint32_t at, int columns) {
  yield();
  const uint32_t col = at & 0xFFFF;
  if (col < TM_O) {
    CHECK(P.parts == 8 && !under_way(TM_P, TM_P + 128, false), "weights on a P that is in use");
    P.stored += columns;
  } else {
    const int u = (col - TM_W) / 48;
    CHECK(!under_way(TM_W + 48 * u, TM_W + 48 * u + 48, false), "weighted values over some that are read");
    const Tag t{fibers[now].head, fibers[now].row};
    CHECK(W[u].stores == 0 || (W[u].tag.head == t.head && W[u].tag.row == t.row), "weighted values of two blocks");
    W[u].tag = t;
    W[u].stores++;
  }
}
static void issue(Mma m) {
  yield();
  m.seen_a = seen(m.a_tile), m.seen_b = seen(m.b_tile);
  queues[now].push_back(m);
}
void mma_ss(uint32_t d, Operand a, Operand b, uint32_t, bool add) {
  Mma m;
  m.d = d, m.a_tile = tile_of(a.at), m.b_tile = tile_of(b.at), m.add = add;
  issue(m);
}
void mma_ts(uint32_t d, uint32_t a, Operand b, uint32_t, bool add) {
  Mma m;
  m.d = d, m.a_tmem = a, m.b_tile = tile_of(b.at), m.add = add;
  issue(m);
}
void mma_commit(uint32_t bar) {
  Mma m;
  m.commit = true, m.bar = bar;
  issue(m);
}
}  // namespace lq

// ---- a CTA ----
static std::function<void()> body;
static void enter() {
  body();
  fibers[now].done = true;
  swapcontext(&fibers[now].ctx, &scheduler);
}

static double some_weight() {
  const double w[] = {1, 1, 1, 0.1, 0.001, 0.00001};
  return w[rng() % 6];
}

static void run_cta(int cta, int ctas, std::function<void()> kernel) {
  memset(raw, 0, sizeof(raw));
  bars.clear(), queues.clear(), loose.clear();
  P = {}, O = {}, DS = {}, W[0] = W[1] = {};
  in_cta_barrier = 0;
  body = kernel;
  const double loose_weight = some_weight();
  std::map<int, double> queue_weight;
  for (int w = 0; w < WARPS; w++) {
    Fiber &f = fibers[w];
    f.stack.resize(128 << 10);
    f.done = f.at_cta_barrier = false, f.wait_bar = 0, f.weight = some_weight();
    queue_weight[w] = some_weight();
    getcontext(&f.ctx);
    f.ctx.uc_stack.ss_sp = f.stack.data(), f.ctx.uc_stack.ss_size = f.stack.size(), f.ctx.uc_link = &scheduler;
    makecontext(&f.ctx, enter, 0);
  }
  if (rng() % 3 == 0)                         // now and then all in step but for one
    for (int w = 0, slow = rng() % WARPS; w < WARPS; w++) fibers[w].weight = w == slow ? 1e-5 : 1;
  std::vector<std::pair<double, int>> able;   // 0 .. : fibers, 100 .. : queues, 1000: a loose party
  for (long turn = 0;; turn++) {
    CHECK(turn < 50000000, "no end");
    able.clear();
    double sum = 0;
    auto may = [&](double w, int who) { sum += w, able.push_back({sum, who}); };
    for (int w = 0; w < WARPS; w++) {
      const Fiber &f = fibers[w];
      if (!f.done && !f.at_cta_barrier && (f.wait_bar == 0 || passed(f.wait_bar, f.wait_parity))) may(f.weight, w);
    }
    for (auto &q : queues)
      if (!q.second.empty()) may(queue_weight[q.first], 100 + q.first);
    if (!loose.empty()) may(loose_weight, 1000);
    if (able.empty()) break;
    const double x = std::uniform_real_distribution<double>(0, sum)(rng);
    size_t i = 0;
    while (i + 1 < able.size() && able[i].first < x) i++;
    const int who = able[i].second;
    if (who == 1000) {
      const size_t at = rng() % loose.size();
      auto go = loose[at];
      loose[at] = loose.back();
      loose.pop_back();
      go();
    } else if (who >= 100) {
      auto &q = queues[who - 100];
      const Mma m = q.front();
      q.pop_front();
      if (m.commit) loose.push_back([=] { arrive(m.bar); });
      else execute(m);
    } else {
      now = who;
      threadIdx.x = 32 * who, blockIdx.x = cta, gridDim.x = ctas, blockDim.x = SCAN_THREADS;
      swapcontext(&scheduler, &fibers[who].ctx);
      now = -1;
    }
  }
  for (int w = 0; w < WARPS; w++)
    if (!fibers[w].done) fail("warp %d waits for ever (barrier at %d)", w, (int)fibers[w].wait_bar - (int)BASE);
}

// ---- a call ----
static void run(unsigned seed) {
  rng.seed(seed);
  auto pick = [](int n) { return (int)(rng() % n); };
  const int hq = 1 + pick(2), hv = hq * (1 + pick(2)), seqs = 1 + pick(4), ctas = 1 + pick(2);
  const int pieces = pick(4) == 0 ? 2 : 1;
  std::vector<int32_t> start{pick(3)}, resume, slots;
  std::string list;
  int longest = 0;
  for (int n = 0; n < seqs; n++) {
    const int blocks = pick(4), len = blocks == 0 ? 0 : 128 * blocks - pick(2) * pick(128);
    start.push_back(start.back() + len);
    resume.push_back(pick(2));
    slots.push_back(pick(12) == 0 ? -1 : seqs - 1 - n);
    longest = std::max(longest, len);
    list += " " + std::to_string(len) + (resume[n] ? "r" : "") + (slots[n] < 0 ? "-" : "");
  }
  const int tokens = start.back() + pick(3);
  what = "seed " + std::to_string(seed) + ", " + std::to_string(hv) + " heads of" + list + ", " + std::to_string(pieces) + " pieces, " + std::to_string(ctas) + " CTAs";
  const size_t SS = SD * SD;
  std::vector<__nv_bfloat16> beta((tokens + 1) * hv, __float2bfloat16_rn(1.0f)), alpha = beta;
  for (int n = 0; n < seqs; n++)
    for (int row = start[n]; row < start[n + 1]; row += SB)
      for (int h = 0; h < hv; h++) alpha[row * hv + h] = __float2bfloat16_rn(decay_of(h, row));
  const int64_t o_stride = hv * SD + 8;       // (rows that are not whole sectors)
  std::vector<uint4> o_mem((tokens + 1) * o_stride / 8 + 1);
  memset(o_mem.data(), 0xFF, o_mem.size() * 16);
  __nv_bfloat16 *o = reinterpret_cast<__nv_bfloat16 *>(o_mem.data());
  std::vector<float> S(seqs * hv * SS), before;
  for (size_t i = 0; i < S.size(); i++) S[i] = (float)(3 + i / SS % 5);
  before = S;
  const int blocks = std::max(1, (longest + SB - 1) / SB), piece = (blocks + pieces - 1) / pieces;
  ScanPlan plan{};
  plan.piece = piece * SB;
  plan.pieces = (blocks + piece - 1) / piece;
  plan.items = seqs * hv * plan.pieces;
  plan.heads.set(hv), plan.cuts.set(plan.pieces), plan.group.set(hv / hq);
  std::vector<float> states(plan.items * SS + hv * SS), decays(plan.items + hv);
  plan.states = states.data(), plan.decays = decays.data();
  int taken = 0;
  if (pick(2)) plan.next = &taken;
  ScanArgs a{};
  a.q_stride = a.k_stride = hq * SD, a.v_stride = hv * SD, a.beta_stride = a.alpha_stride = hv, a.o_stride = o_stride;
  a.beta = beta.data(), a.alpha = alpha.data();
  a.S0 = a.S = S.data(), a.o = o;
  a.sq = {start.data(), slots.data(), resume.data(), tokens, seqs, seqs};
  a.heads_v = hv, a.heads_qk = hq, a.max_len = longest;
  ScanMaps maps{};
  g_ops_error = 0;
  if (plan.pieces > 1) {
    for (int c = 0; c < ctas; c++) run_cta(c, ctas, [&] { scan_blocks_kernel<false, __nv_bfloat16, false>(maps, a, plan); });
    for (int b = 0; b < seqs * hv * 16; b++)
      for (int t = 0; t < 256; t++) blockIdx.x = b, threadIdx.x = t, scan_join_kernel(a, plan);
    taken = 0;
  }
  for (int c = 0; c < ctas; c++) run_cta(c, ctas, [&] { scan_blocks_kernel<true, __nv_bfloat16, false>(maps, a, plan); });
  CHECK(g_ops_error == 0, "flags %d", g_ops_error);
  // the same from the lengths alone, for the channels of every warp's lane 0
  std::vector<char> written(tokens + 1, 0);
  for (int n = 0; n < seqs; n++)
    for (int h = 0; h < hv && slots[n] >= 0; h++) {
      const size_t at = ((size_t)slots[n] * hv + h) * SS;
      float s = resume[n] ? before[at] : 0;
      for (int row = start[n]; row < start[n + 1]; row += SB) {
        for (int r = row; r < std::min(row + SB, start[n + 1]); r += 32) {
          written[r] = 1;
          for (int c = 0; c < SD; c++) {
            const float got = __bfloat162float(o[(int64_t)r * o_stride + h * SD + c]);
            const float want = (s + 0.5f) * (r == row ? decay_of(h, row) : 1);   // (lane 0 of the gates' warp has a block's first four rows)
            CHECK(got == want, "row %d of head %d is %g, not %g", r, h, got, want);
          }
        }
        s = s * decay_of(h, row) + value_of({h, row});
      }
      for (int c = 0; c < SD; c += 32)
        for (int j = 0; j < SD; j++) CHECK(S[at + j * SD + c] == s, "the state of sequence %d, head %d is %g, not %g", n, h, S[at + j * SD + c], s);
    }
  for (int r = 0; r < tokens; r++)
    if (!written[r])
      for (int c = 0; c < hv * SD; c++) {
        uint16_t x;
        memcpy(&x, &o[(int64_t)r * o_stride + c], 2);
        CHECK(x == 0xFFFF, "row %d is written", r);
      }
  for (int n = 0; n < seqs; n++)              // slots of padding
    if (std::find(slots.begin(), slots.end(), n) == slots.end())
      for (size_t i = n * hv * SS; i < (n + 1) * hv * SS; i++) CHECK(S[i] == before[i], "a slot of nobody is written");
}

int main(int argc, char **argv) {
  const unsigned first = argc > 1 ? atoi(argv[1]) : 0, n = argc > 2 ? atoi(argv[2]) : 100;
  for (unsigned s = first; s < first + n; s++) run(s);
  printf("%u runs\n", n);
  return 0;
}
