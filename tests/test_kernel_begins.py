"""Every kernel is set up while the kernel before it on the stream may still run: before it touches global memory each waits for that kernel's
end, or acquires what the product that it runs under released behind its own wait.  Nothing else makes another grid's writes visible to it."""
import re
from pathlib import Path

import pytest

CSRC = Path(__file__).resolve().parent.parent / "paper_1909_05840_b200" / "csrc"
BEGIN = re.compile(r"if constexpr \(UNDER\) begin_under\([^;]*\);\s*else pdl_begin\(\);|pdl_begin\(\);")


def kernels(path):
    """(name, body) of every kernel of a file."""
    text = re.sub(r"//[^\n]*", "", path.read_text())
    for m in re.finditer(r"__global__ void\s+__launch_bounds__\([^)]*\)\s*(\w+)\s*\([^{;]*\)\s*\{", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield m.group(1), text[m.end():i - 1]


def outermost(body):
    """The body without what stands in braces of its own."""
    depth, out = 0, []
    for c in body:
        depth -= c == "}"
        if depth == 0:
            out.append(c)
        depth += c == "{"
    return "".join(out)


@pytest.mark.parametrize("path", sorted(p for p in CSRC.glob("*.cu") if p.name != "probe.cu"), ids=lambda p: p.name)
def test_every_kernel_begins_behind_a_wait(path):
    for name, body in kernels(path):
        found = BEGIN.search(outermost(body))
        assert found, f"{name}: no unconditional wait"
        before = outermost(body)[:found.start()].rstrip()
        assert not before.endswith(")"), f"{name}: the wait is conditional: ...{before[-60:]}"


def test_kernels_are_found():
    names = {n for p in CSRC.glob("*.cu") for n, _ in kernels(p)}
    assert {"linear_kernel", "column_parts_kernel", "column_few_kernel", "layer_norm_kernel", "vocab_kernel", "qb_gemm_kernel"} <= names


def test_the_mark_is_released_behind_the_wait():
    (body,) = (b for n, b in kernels(CSRC / "linear.cu") if n == "linear_kernel")
    release = body.index("st_release(&static_cast<WsHeader*>(gp.ws)->begun, gp.mark)")
    assert "pdl_begin();" in outermost(body[:release])
    text = (CSRC / "linear.cu").read_text()
    assert re.search(r"poll_word\(&static_cast<const WsHeader\*>\(ws\)->begun, mark, \d+\);\s*if \(!__syncthreads_or\(seen\)\) pdl_begin\(\);", text)
