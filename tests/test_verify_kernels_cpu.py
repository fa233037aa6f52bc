"""The kernels of the check of drafted tokens, built for the CPU: every thread of a block a fiber, so that the moves between lanes, the
barriers and the order of every sum are the device's.  Rows of few weights far apart in size, uniforms on the running sums."""
import ctypes as C
import os
import random
import subprocess
from fractions import Fraction

import pytest
import torch

import paper_2103_05288_amd as pkg

CHUNK = 4096

# A block is run to its end before the next one.  A collective operation leaves its operand, waits for the others, reads, and waits
# again, so that nobody leaves the next one's before all have read.
HOST = r"""
#include <ucontext.h>
#include <algorithm>
#include <cstring>
#include <vector>
#define __device__
#define __forceinline__ inline
#define __global__
#define __launch_bounds__(n)
#define __shared__ static
using std::max;
using std::min;
struct Dim { int x, y, z; };
static Dim blockIdx;
struct Barrier { int count, here; long turn; };
struct Fiber { ucontext_t at; Dim id; bool ended; std::vector<char> stack; };
static std::vector<Fiber> fibers;
static Fiber* now;
static ucontext_t outside;
static Barrier waves[16], whole;
static unsigned long long slots[1024];
static void give_way() { swapcontext(&now->at, &outside); }
static void wait_for(Barrier& b) {
  const long turn = b.turn;
  if (++b.here == b.count) { b.here = 0; ++b.turn; return; }
  while (b.turn == turn) give_way();
}
#define threadIdx (now->id)
static unsigned long long lane_of_wave(unsigned long long mine, int from) {   // what lane `from` has
  const int t = now->id.x, wave = t / 64;
  slots[t] = mine;
  wait_for(waves[wave]);
  const unsigned long long x = slots[wave * 64 + from];
  wait_for(waves[wave]);
  return x;
}
// the moves that the header makes: to the right by 1 .. 8 among 16 lanes or by 1 among all, the last of 16 or of 32 to the next ones
static int update_dpp(int old, int x, int control, int rows, int, bool) {
  const int lane = now->id.x % 64;
  int from = -1;
  if (control >= 0x111 && control <= 0x11f) from = lane % 16 >= control - 0x110 ? lane - (control - 0x110) : -1;
  else if (control == 0x138) from = lane - 1;
  else if (control == 0x142) from = lane >= 16 ? lane / 16 * 16 - 1 : -1;
  else if (control == 0x143) from = lane >= 32 ? 31 : -1;
  const int y = (int)lane_of_wave((unsigned)x, max(from, 0));
  return from < 0 || !(rows >> lane / 16 & 1) ? old : y;
}
static int readlane(int x, int lane) { return (int)lane_of_wave((unsigned)x, lane); }
static unsigned long long __ballot(int p) {
  const int t = now->id.x, wave = t / 64;
  slots[t] = p != 0;
  wait_for(waves[wave]);
  unsigned long long mask = 0;
  for (int i = 0; i < 64; ++i) mask |= slots[wave * 64 + i] << i;
  wait_for(waves[wave]);
  return mask;
}
static void __syncthreads() { wait_for(whole); }
#define __builtin_amdgcn_update_dpp update_dpp
#define __builtin_amdgcn_readlane readlane
#define DISC_VERIFY 1
#define DISC_T float
%s
static void (*kernel)(VerifyArgs);
static VerifyArgs args;
static void body() {
  kernel(args);
  now->ended = true;
  give_way();
}
static void launch(void (*k)(VerifyArgs), int blocks, int threads) {
  kernel = k;
  fibers.resize(threads);
  for (int b = 0; b < blocks; ++b) {
    blockIdx = {b, 0, 0};
    for (auto& w : waves) w = {64, 0, 0};
    whole = {threads, 0, 0};
    for (int t = 0; t < threads; ++t) {
      Fiber& f = fibers[t];
      f.id = {t, 0, 0};
      f.ended = false;
      f.stack.resize(64 << 10);
      getcontext(&f.at);
      f.at.uc_stack.ss_sp = f.stack.data();
      f.at.uc_stack.ss_size = f.stack.size();
      f.at.uc_link = nullptr;
      makecontext(&f.at, body, 0);
    }
    for (int left = threads; left > 0;) {
      for (auto& f : fibers) {
        if (f.ended) continue;
        now = &f;
        swapcontext(&outside, &f.at);
        left -= f.ended;
      }
    }
  }
}
extern "C" void verify(const float* target, const float* draft, const int* drafted, const float* uniforms, int* tokens, int* accepted, double* part, int batch, int drafts,
                       int vocabulary) {
  memset(&args, 0, sizeof args);
  args.target = target, args.draft = draft, args.drafted = drafted, args.uniforms = uniforms;
  args.tokens = tokens, args.accepted = accepted, args.part = part;
  args.target_row = args.draft_row = vocabulary;
  args.target_batch = (long long)(drafts + 1) * vocabulary, args.draft_batch = (long long)drafts * vocabulary;
  args.batch = batch, args.drafts = drafts, args.vocabulary = vocabulary;
  args.chunks = (vocabulary + 4095) / 4096;
  launch(disc_verify_sum_k, batch * args.chunks, 256);
  launch(disc_verify_pick_k, batch, 256);
}
"""


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    with open(os.path.join(os.path.dirname(pkg.__file__), "csrc", "step_device.h")) as f:
        header = f.read()
    assert f"constexpr int kChunk = {CHUNK};" in header
    base = str(tmp_path_factory.mktemp("verify") / "kernels")
    with open(base + ".cpp", "w") as f:
        f.write(HOST.replace("%s", header.replace("#pragma once", "")))
    clang = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
    # (-ffp-contract=off: the header's sums hold no products that a device build contracts)
    subprocess.run([clang, "-O1", "-std=c++17", "-ffp-contract=off", "-w", "-shared", "-fPIC", "-o", base + ".so", base + ".cpp"], check=True)
    return C.CDLL(base + ".so")


def _run(kernels, target, uniforms, draft=None, drafted=None):
    B, places, V = target.shape
    tokens, accepted = torch.full((B, places), -9, dtype=torch.int32), torch.full((B,), -9, dtype=torch.int32)
    part = torch.full((B * -(-V // CHUNK) * 2,), float("nan"), dtype=torch.float64)
    drafted = torch.zeros((B, places - 1), dtype=torch.int32) if drafted is None else drafted
    p = lambda t: C.c_void_p(None if t is None else t.data_ptr())  # noqa: E731
    kernels.verify(p(target), p(draft), p(drafted), p(uniforms), p(tokens), p(accepted), p(part), B, places - 1, V)
    return tokens, accepted


def _fits(row, uniform, token):
    """Whether a token is the first whose running sum passes uniform times the whole, but for the roundings of the sums: each weight goes
    through fewer than 128 additions of 64 bits (16 of a thread, 6 of a scan, 4 of a block and as many again in the second launch, the rest
    the chunks of a lane), each off by at most 2^-53 of the whole."""
    at = torch.nonzero(row).flatten().tolist()
    assert token in at, (token, at[:40])
    upto, front = Fraction(0), None
    for i in at:
        if i == token:
            front = upto
        upto += Fraction(float(row[i]))
        if i == token:
            here = upto
    off = upto * Fraction(128, 2 ** 53)
    goal = Fraction(uniform) * upto
    assert front <= goal + off and (here > goal - off or token == at[-1]), (token, at[:40])


def _sparse(g, V, n):
    """A row of n weights 2^-60 .. 0.5, in chunks of their own where there are as many, empty ones between and behind them."""
    row = torch.zeros(V)
    chunks = g.sample(range(-(-V // CHUNK)), min(n, -(-V // CHUNK)))
    for k in range(n):
        at = min(V - 1, chunks[k % len(chunks)] * CHUNK + g.choice((0, 15, 16, 17, 1023, 1024, 4095, g.randrange(CHUNK))))
        row[at] = 2.0 ** -g.choice((1, 2, 3, 24, 25, 52, 53, 54, 60)) * g.choice((1.0, 1.5, 1.9999998807907104))
    return row


def _uniforms(g, row, n):
    """On the running sums' shares of the whole, one step of 32 bits beside them, and 0 and 1."""
    upto = torch.cumsum(row.double(), 0)
    shares = (upto[row > 0] / upto[-1]).float()
    out = []
    for _ in range(n):
        u = shares[g.randrange(len(shares))]
        out.append(float(g.choice((u, torch.nextafter(u, torch.tensor(0.0)), torch.nextafter(u, torch.tensor(2.0)).clamp(max=1.0), torch.tensor(0.0), torch.tensor(1.0)))))
    return out


def test_a_token_of_every_row_of_few_weights(kernels):
    """A lane of a scan without any weight of its own can come out a rounding above the lane before it: no token is in it."""
    V = 20480
    row = torch.zeros(V)
    row[0] = row[4096] = 2.0 ** -54
    row[8192] = row[16384] = 0.5
    tokens, accepted = _run(kernels, row.view(1, 1, V), torch.tensor([[0.5]]))
    assert accepted.tolist() == [0]
    _fits(row, 0.5, int(tokens[0, 0]))
    g = random.Random(1)
    rows, uniforms = [], []
    for _ in range(24):
        rows.append(_sparse(g, V, g.choice((2, 3, 4, 5, 8, 20))))
        uniforms += _uniforms(g, rows[-1], 1)
    tokens, _ = _run(kernels, torch.stack(rows)[:, None].contiguous(), torch.tensor(uniforms)[:, None].contiguous())
    for row, u, t in zip(rows, uniforms, tokens[:, 0].tolist()):
        _fits(row, u, t)


def test_a_last_uniform_of_one_takes_the_last_token_with_weight(kernels):
    """Dense rows behind which lanes and chunks are empty."""
    g = torch.Generator().manual_seed(2)
    rows = torch.zeros(100, 1, 25000)
    rows[:, 0, :24000] = torch.softmax(2 * torch.randn(100, 24000, generator=g), -1)
    tokens, _ = _run(kernels, rows, torch.ones(100, 1))
    for row, t in zip(rows[:, 0], tokens[:, 0].tolist()):
        _fits(row, 1.0, t)


def test_what_is_left_of_the_target_beside_the_draft(kernels):
    """The same of max(p - q, 0)."""
    V, g = 20480, random.Random(3)
    left = [_sparse(g, V, g.choice((2, 4, 9))) for _ in range(8)]
    uniforms = torch.tensor([[0.75] + _uniforms(g, row, 1) for row in left])
    draft = torch.zeros(8, 1, V)
    draft[:, 0, 77] = 1.0                                  # (the drafted token, which the target cannot have)
    target = torch.stack([torch.stack([row * (row != row[77]) if row[77] > 0 else row, torch.ones(V)]) for row in left])
    tokens, accepted = _run(kernels, target.contiguous(), uniforms, draft, torch.full((8, 1), 77, dtype=torch.int32))
    assert accepted.tolist() == [0] * 8 and tokens[:, 1].tolist() == [-1] * 8
    for row, u, t in zip(target[:, 0], uniforms[:, 1].tolist(), tokens[:, 0].tolist()):
        _fits(row, u, t)


def test_the_sum_in_front_of_a_chunk_of_several_of_a_lane(kernels):
    """More than 64 chunks: where rounding, or a uniform of 1, leaves no token whose running sum passes the goal, the last with weight is
    taken, not the first of its chunk."""
    V, g = 64 * CHUNK + 3000, random.Random(5)
    rows = [torch.zeros(V) for _ in range(4)]
    for row, (first, last) in zip(rows, ((0, 8), (60, 64), (3, 4), (0, 65))):
        for c in range(first, last):
            for _ in range(6):
                row[min(V - 1, c * CHUNK + g.randrange(CHUNK))] = g.random() + 0.1
    rows.append(torch.zeros(V))
    rows[-1][4096 * 30::1500] = 0.001
    uniforms = [1.0] * 4 + _uniforms(g, rows[-1], 1)
    tokens, _ = _run(kernels, torch.stack(rows)[:, None].contiguous(), torch.tensor(uniforms)[:, None].contiguous())
    for row, u, t in zip(rows, uniforms, tokens[:, 0].tolist()):
        _fits(row, u, t)
