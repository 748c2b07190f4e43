"""Where paged attention's kernels of 32 query rows and 128 dims use scratch memory: nowhere in the
loops over tiles, whose loads a reload would wait for."""
import re

import pytest

from test_pages_resources import asm  # noqa: F401  (the sources' assembly, compiled once)


def blocks(text, prefix):
    """(the loops that it is in, its lines) of every block of the kernel of a prefix, by the
    compiler's comments: a header's names the loops around it, another block's the innermost."""
    lines = text.splitlines()
    begin = next(i for i, x in enumerate(lines) if re.match(prefix + r"\w*:", x))
    out, around = [([], [])], {}
    for line in lines[begin:]:
        if line.startswith(".Lfunc_end"):
            break
        label = re.match(r"\.L(BB\d+_\d+):", line)
        if label:
            out.append(([], []))
            name = label.group(1)
        loops, own = out[-1]
        if "Loop Header" in line:
            around[name] = loops[:]
            loops.append(name)
        loops += re.findall(r"(?:Parent Loop |in Loop: Header=)(BB\d+_\d+)", line)
        own.append(line)
    return [({y for x in loops for y in [x] + around.get(x, [])}, own) for loops, own in out]


@pytest.mark.parametrize("fmt", [0, 1, 2])
@pytest.mark.parametrize("mode", [0, 1, 2])
def test_no_scratch_in_the_loops_over_tiles(asm, fmt, mode):  # noqa: F811
    got = blocks(asm[f"paged_{['bf16', 'mxfp8', 'mxfp4'][fmt]}.hip"],
                 f"_ZN6certkv12paged_kernelILi{fmt}ELi128ELi2ELi{mode}E")
    has = lambda lines, what: any(what in x.split(";")[0] for x in lines)  # noqa: E731
    products = [loops for loops, lines in got if has(lines, "v_mfma")]
    # the loop over the rows that all queries see and the one over the last ones: what is in a loop
    # with products, but for the loop over pieces around both
    pieces = set.intersection(*products)
    tiles = set.union(*products) - pieces
    assert len(tiles) >= 2 and len(pieces) <= 1
    for loops, lines in got:
        assert not (has(lines, "scratch_") and tiles & loops), lines[0]
