"""Who learns by a shuffle that it is the last to arrive reads the others' parts only behind a warp barrier (CPU, by the
sources).  The shuffle orders no memory; the one lane that made the counter's fences passes their order on to the
other lanes by the barrier."""
import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15592_gb300", "csrc")


def _read(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


def _functions(text):
    """Bodies between a brace in column 0 and the one that closes it there."""
    return re.findall(r"^[^\s}][^;{}]*\{\n(.*?)^\}", text, re.S | re.M)


def test_a_barrier_stands_behind_the_shuffle():
    found = 0
    for path in glob.glob(os.path.join(CSRC, "*.cu*")):
        for body in _functions(_read(path)):
            # an arrival by one lane: an atomic on a counter between fences, told to the warp by a shuffle
            at = re.search(r"__threadfence\(\);.*?atomic(?:Add|Inc)\(.*?__threadfence\(\);", body, re.S)
            tell = at and re.search(r"__shfl_sync\(", body[at.end():])
            if not tell:
                continue
            found += 1
            rest = body[at.end() + tell.start():]
            after = rest.index(";") + 1
            assert rest[after:].lstrip().startswith("__syncwarp();"), f"{os.path.basename(path)}: {rest[:200]}"
    assert found == 1  # the helper that all of them call


def test_rows_of_logits_arrive_by_the_helper():
    for name in ("logprobs.cu", "distill.cu"):
        text = _read(os.path.join(CSRC, name))
        assert "__threadfence" not in text
        assert re.search(r"\barrive\(a\.count \+", text)
