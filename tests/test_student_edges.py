"""Calls of the student block's operators that need no GPU to go wrong: those without rows, the
sizes of workspaces, what the status read covers."""
import ast
import ctypes
import glob
import math
import os
import re
import subprocess
import sys

import pytest

from test_dependent_kernels import kernels

P = ctypes.c_void_p
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                    "paper_2609_18145_gb300", "csrc")


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("rows,kind", [(0, 1), (0, 2), (1, 1), (64, 2)])
def test_a_norm_backward_of_no_rows_does_nothing(rows, kind):
    """In a process of its own: what goes wrong here takes the process with it."""
    code = """
import ctypes
from paper_2609_18145_gb300 import hcw as H
P = ctypes.c_void_p
before = H.hcw_launch_count()
rc = H.lib().hcw_residual_norm_bwd(None, None, None, None, None, %d, 1.0, %d, None, None, %d, None,
                                   1e-5, 0, 96, 1, P(1 << 20), None, None, None, None, None, None,
                                   None, 0, None)
assert rc == H.HCW_OK, rc
assert H.hcw_launch_count() == before
""" % (rows, kind, kind)
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])


def test_every_unit_that_can_give_up_is_read_by_the_status():
    """The error word exists once a translation unit: the unit that waits has to hand out its own,
    and hcw_sync_status has to read it."""
    units = {}
    for path in glob.glob(os.path.join(CSRC, "*.cu")):
        text = re.sub(r"//[^\n]*|/\*.*?\*/", "", open(path).read(), flags=re.S)
        units[os.path.basename(path)] = text
    m = re.search(r"int hcw_sync_status\(.*?\n\}", units["hcw_api.cu"], flags=re.S)
    seen = 0
    for name, text in units.items():
        if not re.search(r"\bmbar_wait|\bg_error_word\b|\bhcw_ptx\.cuh\b", text):
            continue
        seen += 1
        own = re.search(r"cudaError_t (\w*error_word_read_clear)\(int\* word\) \{", text)
        assert own, name
        assert re.search(r"\b%s\(" % own.group(1), m.group(0)), (name, own.group(1))
        # and the header that declares the word names the unit
        assert name in open(os.path.join(CSRC, "hcw_ptx.cuh")).read().split("namespace {")[0], name
    assert seen >= 9


@pytest.mark.parametrize("name", ["norm_fwd_kernel", "norm_bwd_kernel"])
def test_no_warp_of_a_norm_leaves_its_rows_early(name):
    """The sums of a row meet at a barrier of the row's warps: a warp that gave up and left the
    loop over the rows would leave the others there for good."""
    body = dict(kernels(open(os.path.join(CSRC, "hcw_norm.cu")).read()))[name]
    heads = list(re.finditer(r"for \(int row0\b[^;]*;([^;]*);[^{]*\{", body))
    assert len(heads) == 1
    assert heads[0].group(1).strip() == "row0 < r1"
    depth, i = 1, heads[0].end()
    while depth:
        depth += {"{": 1, "}": -1}.get(body[i], 0)
        i += 1
    assert not re.search(r"\b(break|return|continue|goto)\b", body[heads[0].end():i].replace(
        "return pack_bf16x2", ""))


def test_lanes_that_read_or_overwrite_each_others_values_are_ordered():
    """Votes and shuffles are no memory barriers: before a lane writes a named symbol over
    another lane's dense value, or reads another lane's slot, there is a barrier on every way
    there."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hcw_distill.cu")).read())
    kernel = dict(kernels(text))["distill_warp_kernel"]
    meet = re.search(r"auto meet = \[&\]\(\) \{(.*?)\};", kernel, flags=re.S).group(1)
    assert re.search(r"if \(W > 1\)\s+asm volatile\(\"bar.sync[^;]*;[^;]*;\s+else\s+__syncwarp\(\);",
                     meet)
    # the dense values, a meeting of all, the named symbols
    assert re.search(r"dense\(v\[e\]\)\);\s*\}\s*meet\(\);\s*if \(part\) return;", kernel)
    own = re.search(r"void slots_own\([^{]*\{(.*?)\n\}", text, flags=re.S).group(1)
    assert own.lstrip().startswith("__syncwarp();")
    # a buffer is handed back when every lane has read it
    row = dict(kernels(text))["distill_row_kernel"]
    gives = list(re.finditer(r"mbar_arrive\(&bars->empty\[", row))
    assert len(gives) == 2
    for m in gives:
        assert re.search(r"__syncwarp\(\);\s*if \(lane == 0\)( \{\s*if \(gb\))? $", row[:m.start()])


def test_what_a_call_allocates_belongs_to_its_stream(H, monkeypatch):
    """Memory of the current stream may still be in use there when another stream's launch writes
    it, or be handed out again while that launch goes on."""
    tree = ast.parse(open(H.__file__).read())
    for f in [n for n in tree.body if isinstance(n, ast.FunctionDef)]:
        made = [n for n in ast.walk(f) if isinstance(n, ast.Call) and
                re.fullmatch(r"torch\.(empty|zeros|ones|full)(_like)?", ast.unparse(n.func))]
        assert not made or f.name == "_scratch", f.name

    log = []

    class Under:
        def __init__(self, stream):
            self.stream = stream

        def __enter__(self):
            log.append(("under", self.stream))

        def __exit__(self, *_):
            log.append(("back", self.stream))

    class Memory:
        def record_stream(self, stream):
            log.append(("also used on", stream))

    monkeypatch.setattr(H.torch.cuda, "stream", Under)
    monkeypatch.setattr(H.torch.cuda, "current_stream", lambda: "current")
    monkeypatch.setattr(H.torch, "empty", lambda *a, **k: log.append("made") or Memory())
    H._memory("side").empty(4)
    assert log == [("under", "side"), "made", ("back", "side"), ("also used on", "current")]
    del log[:]
    H._scratch("side", 4, "cuda")
    assert log == [("under", "side"), "made", ("back", "side")]
    del log[:]
    assert H._memory(None) is H.torch
    H._memory(None).empty(4)
    H._scratch(None, 4, "cuda")
    assert log == ["made", "made"]


def test_the_bindings_shape_checks(H):
    """What numbers the same rows in the same order passes, what has the same number of elements
    in another order does not."""
    torch = H.torch
    e = lambda *s: torch.empty(s, device="meta")  # noqa: E731
    like = [((6, 8), (6, 8)), ((2, 3, 8), (6, 8)), ((6, 8), (2, 3, 8)), ((2, 1, 3, 8), (2, 3, 8)),
            ((6, 8), (48,)), ((0, 8), (0, 8)), ((8,), (1, 8))]
    for a, b in like:
        H._like(e(*a), "x", e(*b), None)
    for a, b in [((6, 8), (8, 6)), ((6, 8), (6, 4)), ((6, 8), (12, 4)), ((2, 3, 8), (3, 2, 8)),
                 ((2, 3, 8), (3, 16)), ((6, 8), ())]:
        with pytest.raises(ValueError, match="does not match"):
            H._like(e(*a), "x", e(*b))
    with pytest.raises(ValueError, match="does not match"):
        H._like(e(6, 8), "x", e(6, 8).half())
    for G, d, b in [(1, 8, (8,)), (1, 8, (1, 8)), (1, 8, (8, 1)), (3, 8, (3, 8)), (3, 8, (24,)),
                    (0, 8, (0, 8))]:
        H._params("x", G, d, e(*b), None)
    for G, d, b in [(1, 8, (6,)), (3, 8, (8, 3)), (3, 8, (8,)), (3, 8, (2, 8))]:
        with pytest.raises(ValueError, match="expected"):
            H._params("x", G, d, e(*b))
    for lead, b in [((6,), (6,)), ((6,), (6, 1)), ((2, 3), (6,)), ((2, 3), (2, 3)), ((6,), (2, 3)),
                    ((), (1,)), ((0,), (0,))]:
        H._row_values("x", torch.float32, math.prod(lead), lead, e(*b), None)
    for lead, b in [((6,), (5,)), ((2, 3), (3, 2)), ((2, 3), (2,)), ((2, 3), (5,))]:
        with pytest.raises(ValueError, match="does not match"):
            H._row_values("x", torch.float32, math.prod(lead), lead, e(*b))
    with pytest.raises(TypeError, match="int32"):
        H._row_values("x", torch.int32, 6, None, e(6))


def test_a_pair_that_gives_up_waits_for_its_copies():
    """The copies' landing is waited for whichever warp gave up, not only where the one that starts
    them did."""
    body = dict(kernels(open(os.path.join(CSRC, "hcw_ffn.cu")).read()))["ffn_pair_kernel"]
    drain = body.index("mbar_wait_drain(&bars->full[s]")
    cond = re.findall(r"if \(([^;{}]*)\)\s+for \(int s = 0;", body[:drain])[-1]
    assert cond == "rank == 0"
    assert re.search(r"cluster_sync_all\(\);\s+if \(\*abort\) settle_after_abort\(\);", body)


def test_a_cluster_that_gives_up_waits_for_what_was_sent():
    """Parts that another CTA sent are counted by barriers that are no longer waited for."""
    body = dict(kernels(open(os.path.join(CSRC, "hcw_distill.cu")).read()))["distill_row_kernel"]
    assert re.search(r"cluster_sync_all\(\);\s+if \(\*abort\) settle_after_abort\(\);\s*\}$", body)


def test_the_norms_count_rows_and_items_without_passing_an_int():
    """Rows and items may number 2^31 - 1: a step past the end must not wrap."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hcw_norm.cu")).read())
    assert not re.search(r"\b(item|row0)\s*\+=", text)
    assert len(re.findall(r"\b(?:item|row0) = norm_next\(", text)) == 5
    assert "return step < end - i ? i + step : end;" in text


def test_the_feed_forward_block_counts_its_row_tiles_without_passing_an_int():
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, "hcw_ffn.cu")).read())
    assert "(T + 255)" not in text and "((long long)T + 255) / 256" in text


@pytest.mark.parametrize("d,h", [(64, 72), (512, 1024), (1024, 2744), (2048, 5632), (4096, 14336)])
def test_a_feed_forward_workspace_does_for_fewer_tokens(H, d, h):
    for size in (H.hcw_gated_ffn_fwd_workspace_bytes, H.hcw_gated_ffn_bwd_workspace_bytes):
        last = 0
        for T in [*range(1, 700), *range(700, 20000, 97)]:
            need = size(T, d, h)
            assert need >= last, (T, need, last)
            last = need


@pytest.mark.parametrize("d", [1, 64, 512, 4097, 8192])
@pytest.mark.parametrize("rows", [0, 1, 2, 7, 64, 256, 5000])
def test_a_norm_workspace_does_for_fewer_rows(H, d, rows):
    last = 0
    for T in [*range(1, 700), *range(700, 40000, 97)]:
        need = H.hcw_residual_norm_bwd_workspace_bytes(T, d, rows)
        assert need >= last, (T, need, last)
        last = need
