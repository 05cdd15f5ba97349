"""Which form of the layer norm kernels a call takes, as the source states it: no compiled form that no call reaches."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2609_35099_b200" / "csrc"


def sixteen(size, vector, ragged, bwd):
    return not bwd or (size == 2 and vector and not ragged)


def form(n, size, bwd, aligned):
    """norm_shape's choice: elements an access, elements a lane, lanes of a row (0: several warps), ragged."""
    v = 16 // size
    ragged = aligned and n % v != 0 and n > 32 and n + v - 1 <= 4096
    vector = aligned and (n % v == 0 or ragged)
    width = n + (v - 1 if ragged else 0)
    each = 16 if width > 2048 or (width > 256 and sixteen(size, vector, ragged, bwd)) else 8
    lanes = 1
    while lanes * each < width:
        lanes *= 2
    lanes = max(lanes, 32) if each == 16 else lanes
    return (v if vector else 1, each, lanes if lanes <= 32 else 0, ragged)


def compiled(v, size, ragged, bwd):
    """launch_norm_lanes' instances."""
    few = [] if ragged else [(8, 1), (8, 2), (8, 4)]
    many = [(16, 32), (16, 0), (8, 32)] if sixteen(size, v > 1, ragged, bwd) else [(16, 0), (8, 32), (8, 0)]
    return {(v, each, lanes, ragged) for each, lanes in few + [(8, 8), (8, 16)] + many}


def test_every_form_is_reached():
    for size in (4, 2):
        for bwd in (False, True):
            reached = {form(n, size, bwd, aligned) for n in range(1, 4097) for aligned in (False, True)}
            assert reached == compiled(1, size, False, bwd) | compiled(16 // size, size, False, bwd) | compiled(16 // size, size, True, bwd)


def test_the_built_library_has_these_forms_alone():
    log = CSRC / "build" / "layer_norm.ptxas.log"
    if not log.exists():
        return
    found = set(re.findall(r"norm_kernelI(f|\d+__nv_bfloat16)Li(\d+)ELi(\d+)ELi(\d+)ELb(\d)ELb(\d)E", log.read_text()))
    want = {(size, bwd, *f) for size in (4, 2) for bwd in (False, True) for v, ragged in ((1, False), (16 // size, False), (16 // size, True))
            for f in compiled(v, size, ragged, bwd)}
    assert {(4 if t == "f" else 2, b == "1", int(v), int(e), int(n), r == "1") for t, v, e, n, r, b in found} == want
