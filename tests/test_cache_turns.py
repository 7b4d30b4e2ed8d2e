"""The barriers of the attention over the cache in tiles of 256 rows, every order of events tried on the CPU: the warp that issues the
products of a half, the tensor core that ends them in turn, and softmax warps of any speed.  Which barrier and which parity a
block goes by comes from the kernel's own header, compiled for the host."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2302_12510_b200", "csrc", "dybit_cache_turns.cuh")
SOURCE = """
#define __host__
#define __device__
#define __forceinline__ inline
#include "%s"
extern "C" unsigned bar_of(unsigned n) { return dybit::turn_of(n).bar; }
extern "C" unsigned parity_of(unsigned n) { return dybit::turn_of(n).parity; }
"""


@pytest.fixture(scope="module")
def turn_of(tmp_path_factory):
    at = tmp_path_factory.mktemp("turns")
    (at / "turns.cpp").write_text(SOURCE % HEADER)
    compiler = shutil.which("g++") or shutil.which("c++")
    subprocess.run([compiler, "-std=c++17", "-shared", "-fPIC", "-o", str(at / "turns.so"), str(at / "turns.cpp")], check=True)
    lib = ctypes.CDLL(str(at / "turns.so"))
    return lambda n: (lib.bar_of(n & 0xffffffff), lib.parity_of(n & 0xffffffff))


def programs(parts, raises, last_waits):
    """What the issuing warp and a softmax warp do, for parts of so many blocks.  A wait names the block that it is for; `raises`
    says whether a block's maximum rises, `last_waits` which blocks behind the newest a part's end waits for, in turn."""
    issue, softmax, done, asked, n = [], [], 0, 0, 0
    for part, blocks in enumerate(parts):
        issue.append(("wait q", part))
        for b in range(-2, blocks):
            if b >= 0:
                issue += [("wait p", done), ("ask o", done)]
                done += 1
            if b + 2 < blocks:
                issue.append(("ask s", asked))
                asked += 1
        softmax.append(("arrive q", part))
        for b in range(blocks):
            softmax.append(("wait s", n))
            if b > 0 and raises(n):
                softmax.append(("wait o", n - 1))
            softmax.append(("arrive p", n))
            n += 1
        softmax += [("wait o", n - back) for back in last_waits]
    return issue, softmax


def explore(issue, softmax, rules, warps=2):
    """Tries every order.  Returns the first thing that goes wrong, or None: a wait that passes before what it waits for has happened,
    or a state that is not the end and that nothing leaves."""
    asked_before = [[]]
    for op in issue:
        asked_before.append(asked_before[-1] + ([op] if op[0].startswith("ask") else []))
    queue = asked_before[-1]

    def arrivals(kind, bar, state):
        """Phases that barrier `bar` of this kind has completed."""
        ipc, ended, pcs = state
        turn = rules[kind]
        if kind in "so":
            return sum(1 for op in queue[:ended] if op[0] == "ask " + kind and turn(op[1])[0] == bar)
        counts = [sum(1 for op in softmax[:pc] if op[0] == "arrive " + kind and turn(op[1])[0] == bar) for pc in pcs]
        return min(counts)                                 # (a phase needs every warp; none arrives twice in one)

    def happened(kind, n, state):
        ipc, ended, pcs = state
        if kind in "so":
            return ("ask " + kind, n) in queue[:ended]
        return all(("arrive " + kind, n) in softmax[:pc] for pc in pcs)

    def step(op, state):
        """Whether the operation can be passed in this state, and what is wrong with that."""
        verb, kind = op[0].split()
        if verb != "wait":
            return True, None
        if kind in rules:
            bar, parity = rules[kind](op[1])
            if (arrivals(kind, bar, state) & 1) == parity:
                return False, None                         # the phase of that parity is the current one
            if op[1] >= 0 and not happened(kind, op[1], state):
                return True, ("too early", op, state)
        return True, None

    start = (0, 0, (0,) * warps)
    seen, todo = {start}, [start]
    while todo:
        state = todo.pop()
        ipc, ended, pcs = state
        out = []
        if ipc < len(issue):
            can, wrong = step(issue[ipc], state)
            if wrong:
                return wrong
            if can:
                out.append((ipc + 1, ended, pcs))
        if ended < len(asked_before[ipc]):                 # the tensor core ends what was asked for first
            out.append((ipc, ended + 1, pcs))
        for w, pc in enumerate(pcs):
            if pc < len(softmax):
                can, wrong = step(softmax[pc], state)
                if wrong:
                    return wrong
                if can:
                    out.append((ipc, ended, pcs[:w] + (pc + 1,) + pcs[w + 1:]))
        if not out and (ipc < len(issue) or any(pc < len(softmax) for pc in pcs)):
            return "stuck", state
        for s in out:
            if s not in seen:
                seen.add(s)
                todo.append(s)
    return None


PARTS = [[1], [2], [3], [1, 1, 1], [2, 1, 2], [5, 1], [1, 4, 2], [3, 3, 1, 2]]
RAISES = {"none": lambda n: False, "all": lambda n: True, "odd": lambda n: n % 2 == 1, "even": lambda n: n % 2 == 0}
SINGLE = lambda n: (0, n & 1)                              # one barrier, a phase to every block (or part)


@pytest.mark.parametrize("raises", RAISES)
@pytest.mark.parametrize("parts", PARTS, ids=str)
def test_every_order_comes_to_its_end(turn_of, parts, raises):
    rules = dict(s=turn_of, p=turn_of, o=turn_of, q=SINGLE)
    assert explore(*programs(parts, RAISES[raises], [1]), rules) is None


@pytest.mark.parametrize("parts", [[1], [2], [1, 1], [4, 2]], ids=str)
def test_the_model_finds_a_phase_that_is_missed(turn_of, parts):
    # one barrier for all products and a wait for each of the last two phases: both can be over before a slow warp looks
    rules = dict(s=turn_of, p=turn_of, o=SINGLE, q=SINGLE)
    assert explore(*programs(parts, RAISES["none"], [2, 1]), rules)[0] == "stuck"


def test_the_model_finds_a_wait_that_passes_too_early(turn_of):
    # ... and a wait for the last of them only takes the phase before it for its own
    rules = dict(s=turn_of, p=turn_of, o=SINGLE, q=SINGLE)
    assert explore(*programs([3], RAISES["none"], [1]), rules)[0] == "too early"


def test_the_kernel_waits_by_turns():
    # every use of the barriers of blocks goes through turn_of
    with open(os.path.join(os.path.dirname(HEADER), "dybit_cache_prefill.cuh")) as f:
        source = f.read()
    for name in ("s_full", "p_full", "o_done"):
        uses = [line for line in source.splitlines() if name + "[" in line and "__shared__" not in line and "mbar_init" not in line]
        assert len(uses) >= 2 and all("turn_of(" in line or "wait_turn(" in line for line in uses), (name, uses)
