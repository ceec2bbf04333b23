"""The kernel of many rows over the cache in the code that the compiler makes of it (cross-compiled here, nothing runs).  Its fast loop writes
matrix instructions itself, which the compiler does not know: what it does for its own ones (waiting for loads, leaving room before a result
is read) is checked here, since a miss gives wrong numbers on some runs only."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2604_20470_amd import build as b

SIZES = [(d, p) for d in (64, 128) for p in (32, 64, 128)]


def _compile(name, folder):
    if not (os.path.exists(b.HIPCC) or shutil.which(b.HIPCC)):
        pytest.skip("no hipcc")
    asm = folder / (name + ".s")
    r = subprocess.run([b.HIPCC, *[f for f in b.FLAGS if f != "-fPIC"], "-S", "--cuda-device-only", os.path.join(b.CSRC, name + ".hip"), "-o", str(asm)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return asm.read_text()


@pytest.fixture(scope="module")
def listing(tmp_path_factory):
    return _compile("k_cache_attn_tile", tmp_path_factory.mktemp("tile"))


def _body(listing, d, p):
    return re.search(r"^_ZN\S*17k_cache_attn_tileILi%dELi%dE\S*:.*?^\.Lfunc_end" % (d, p), listing, re.S | re.M).group(0).split("\n")


def _registers(text):
    out = set()
    for k, lo, hi in re.findall(r"\b([va])\[(\d+):(\d+)\]", text):
        out |= {k + str(i) for i in range(int(lo), int(hi) + 1)}
    return out | {k + n for k, n in re.findall(r"\b([va])(\d+)\b", re.sub(r"\[\d+:\d+\]", "", text))}


def _instructions(lines):
    """(text, whether from inline assembly) without comments and directives; labels stay."""
    out, inside = [], False
    for line in lines:
        inside = (inside or "#ASMSTART" in line) and "#ASMEND" not in line
        x = line.split(";")[0].strip()
        if x and (x.startswith(".LBB") or not x.startswith((".", "_Z"))):
            out.append((x, inside))
    return out


def _fast_loop(lines, d):
    """The smallest loop with all matrix instructions of four chunks: 4 x 64 of them for 128 channels, 4 x 32 for 64."""
    label = {l.split(":")[0]: i for i, l in enumerate(lines) if l.startswith(".LBB")}
    best = None
    for i, l in enumerate(lines):
        g = re.match(r"\s+s_c?branch\S* (\.LBB\S+)", l)
        if g and label.get(g.group(1), i) < i:
            seg = lines[label[g.group(1)]:i]
            if sum("v_mfma" in x for x in seg) == 2 * d and (best is None or len(seg) < len(best)):
                best = seg
    assert best is not None
    return [x for x, _ in _instructions(best)]


@pytest.mark.parametrize("d,p", SIZES)
def test_the_fast_loop_keeps_everything_in_registers(listing, d, p):
    loop = _fast_loop(_body(listing, d, p), d)
    assert not [x for x in loop if re.match(r"scratch|buffer_|v_accvgpr|v_readlane|v_writelane|flat", x)]
    assert sum(x.startswith("ds_read_b128") for x in loop) == d and sum(x.startswith("s_barrier") for x in loop) == 4


@pytest.mark.parametrize("d,p", SIZES)
def test_no_operand_is_used_while_its_load_is_under_way(listing, d, p):
    """Two turns of the fast loop: loads in order, s_waitcnt as the only thing that ends them."""
    loop = _fast_loop(_body(listing, d, p), d)
    lds, mem, bad = [], [], []
    for x in loop * 2:
        op, _, rest = x.partition(" ")
        if op == "s_waitcnt":
            for queue, counter in ((lds, "lgkmcnt"), (mem, "vmcnt")):
                g = re.search(counter + r"\((\d+)\)", x)
                if g:
                    del queue[:max(0, len(queue) - int(g.group(1)))]
            continue
        used = _registers(rest)
        bad += [x for _, dest in lds + mem if dest & used]
        if op.startswith("ds_"):
            lds.append((x, _registers(rest.split(",")[0]) if op.startswith("ds_read") else set()))
        elif op.startswith("global_load"):
            mem.append((x, _registers(rest.split(",")[0])))
    assert not bad, bad[:5]


@pytest.mark.parametrize("d,p", SIZES)
def test_writes_of_a_stage_are_done_before_its_barrier(listing, d, p):
    """The barrier waits for all LDS operations but the last three, so three reads at least lie between a chunk's last write and it."""
    loop = _fast_loop(_body(listing, d, p), d)
    since, seen = None, 0
    for x in loop * 2:
        if x.startswith("ds_write"):
            since = 0
        elif x.startswith("ds_read") and since is not None:
            since += 1
        elif x.startswith("s_barrier") and since is not None:
            assert since >= 3, x
            seen += 1
    assert seen >= 7


@pytest.mark.parametrize("d,p", SIZES)
def test_room_between_a_matrix_instruction_and_its_readers(listing, d, p):
    """Sixteen wait states, an instruction one of them and a matrix instruction eight, before any other instruction touches a result."""
    code, near = _instructions(_body(listing, d, p)), []
    for i, (x, inline) in enumerate(code):
        if not (inline and x.startswith("v_mfma")):
            continue
        dest, room = _registers(x.split(",")[0]), 0
        for y, _ in code[i + 1:i + 120]:
            if y.startswith("v_mfma"):
                room += 8
                continue
            if not y.startswith((".LBB", "s_")) and _registers(y) & dest:
                if room < 16:
                    near.append((x, y))
                break
            g = re.match(r"s_nop (\d+)", y)
            room += int(g.group(1)) + 1 if g else 1
            if room >= 16:
                break
    assert not near, near[:5]


@pytest.mark.parametrize("name", ["k_cache_attn_tile", "k_cache_attn"])
def test_no_move_of_a_value_runs_with_half_of_the_lanes(name, tmp_path):
    """A block that lanes join again first sets the exec mask.  Moves that the register allocation puts in front of that, for values that all lanes
    use later, run for some of the lanes only: that has happened in these kernels, where most registers are in use."""
    for body in re.finditer(r"^_ZN\S*:.*?^\.Lfunc_end", _compile(name, tmp_path), re.S | re.M):
        before, masked = None, False
        for x, _ in _instructions(body.group(0).split("\n")):
            if x.startswith(".LBB"):
                before = []
            elif before is not None:
                if re.match(r"s_or_b64 exec, exec", x):
                    assert not before, (body.group(0)[:80], before[:3])
                    before = None
                elif re.match(r"s_(cbranch|branch|and_saveexec|or_saveexec|mov_b64 exec)", x):
                    before = None                          # (not a join, or the mask of a branch that begins here)
                elif re.match(r"v_(mov|accvgpr)", x):
                    before.append(x)


@pytest.mark.parametrize("name", ["k_cache_attn_tile", "k_cache_attn"])
def test_no_tuple_is_filled_with_one_of_its_elements(name, tmp_path):
    """Sixteen logits that a branch masks have come out as copies of the first: eight accumulation registers in a row written from one
    register that is not a constant."""
    for body in re.finditer(r"^_ZN\S*:.*?^\.Lfunc_end", _compile(name, tmp_path), re.S | re.M):
        run = {}
        for x, _ in _instructions(body.group(0).split("\n")):
            g = re.match(r"v_accvgpr_write_b32 a(\d+), (v\d+)$", x)
            if g:
                run.setdefault(g.group(2), set()).add(int(g.group(1)))
                filled = run[g.group(2)]
                assert not any({a + i for i in range(8)} <= filled for a in filled), (body.group(0)[:80], x)
            elif x.startswith(".LBB"):
                run = {}
            else:
                for r in _registers(x.partition(" ")[2].split(",")[0]):
                    run.pop(r, None)
