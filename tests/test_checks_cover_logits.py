"""Every function of the calls on rows of logits that reaches global memory checks where in the -DESTP_CHECKS build (CPU, by
the sources): its body calls in_bounds or a helper that returns what that says, or all that call it do."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15592_gb300", "csrc")
FILES = ("logprobs.cu", "distill.cu")
# stores of whole and of partial units, of single values through an argument's pointer, into another CTA; copies; loads of units
REACHES = (r"\bstore_(?:unit|whole)<", r"\bstore_remote\(", r"\bcopy_(?:unit|word)\(&", r"\bld_(?:once|stream)\(", r"\bload_unit<",
           r"\b(?:a|d)\.\w+\[[^\]]*\]\s*=[^=]", r"__ldcg\(&")


def _functions(name):
    """The file without comments, and name -> body of its functions."""
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    found = {}
    for m in re.finditer(r"^(?:__device__|__global__)\s", text, re.M):
        at, depth = m.end(), 0
        while text[at] not in "{;" or depth:
            depth += {"(": 1, ")": -1}.get(text[at], 0)
            at += 1
        if text[at] == ";":
            continue
        head = re.sub(r"__launch_bounds__\((?:[^()]|\([^()]*\))*\)", "", text[m.end():at])
        end, open_ = at, 0
        while True:
            open_ += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if open_ == 0:
                break
        f = re.search(r"(\w+)\(", head).group(1)
        found[f] = found.get(f, "") + text[at:end]
    return text, found


def _checks(functions):
    helpers = {"in_bounds"} | {n for n, b in functions.items() if re.search(r"return in_bounds\(", b)}
    return re.compile(r"\b(?:%s)\(" % "|".join(sorted(helpers)))


@pytest.mark.parametrize("name", FILES)
def test_kernels_are_found(name):
    text, functions = _functions(name)
    kernels = re.findall(r"__global__ void __launch_bounds__\((?:[^()]|\([^()]*\))*\)\s+(\w+)\(", text)
    assert len(kernels) == text.count("__global__") >= 3 and all(k in functions for k in kernels)
    checks = _checks(functions)
    for k in kernels:
        assert checks.search(functions[k]), f"{k} makes no check"


@pytest.mark.parametrize("name", FILES)
def test_accesses_are_checked(name):
    text, functions = _functions(name)
    checks, seen = _checks(functions), 0
    for f, body in functions.items():
        # primitives that are a single instruction have nothing to check by
        if f in ("store_remote", "copy_unit", "copy_word") or not any(re.search(p, body) for p in REACHES):
            continue
        seen += 1
        if checks.search(body):
            continue
        callers = [b for g, b in functions.items() if g != f and re.search(r"\b%s(?:<[^;(]*>)?\(" % f, b)]
        assert callers and all(checks.search(b) for b in callers), f"{f} in {name} is not checked"
    assert seen >= 5


def test_every_loss_is_checked():
    """The one place that writes a loss looks at its row."""
    text, functions = _functions("distill.cu")
    assert len(re.findall(r"\bloss\[[^\]]*\]\s*=", text)) == 1
    assert re.search(r"\bloss\[", functions["put_loss"]) and "in_bounds(" in functions["put_loss"]


def test_units_of_a_kept_row_are_checked():
    _, functions = _functions("distill.cu")
    for f in ("copy_group", "kept_grad", "distill_rows_kernel", "short_grad", "distill_short_kernel", "distill_long_kernel",
              "distill_eval_kernel"):
        assert "units_there(" in functions[f], f
    before = functions["distill_rows_kernel"].split("store_remote(")[0]
    assert "in_bounds(" in before[-200:]
