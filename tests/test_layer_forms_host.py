"""The shapes of layer_form_cases.py against the rules between the kernel forms, read from the sources: each form is reached by rows of whole chunks of 8 and by others, so that a later
change of a threshold cannot leave one untested unseen."""
import re

import pytest

from layer_form_cases import COMBINE, COMBINE_GRAD, GRAD, GRAD_FEW, GRAD_ONLY_IN_PLACE, NORM, form, function, rule, source

LAYER, EXPERTS = source("ops_layer_norm.hip"), source("ops_experts.hip")
GRAD_BODY = function(LAYER, "int norm_grad_of_type")
FEW_RULE, ROWS_RULE = (rule(part) for part in GRAD_BODY.split("const int parts"))


def few(M, N, in_place):
    body = function(LAYER, "inline bool grad_few")
    assert "if (a.N > 16384 || a.M > LAUNCH_ROWS) return false;" in body
    condition = re.search(r"return a\.dX != a\.dY && \((.*)\);", body).group(1)
    return N <= 16384 and not in_place and eval(condition.replace("a.", "").replace("||", "or").replace("&&", "and"), {}, {"M": M, "N": N})


def both(found, names, long=()):
    """Each name is reached in both ways; those of `long` rows go by chunks of any length."""
    want = {(n, whole) for n in names - set(long) for whole in (True, False)} | {(n, w) for n, w in found if n in long}
    assert found == want, sorted(want - found)
    assert set(long) <= {n for n, _ in found}


@pytest.mark.parametrize("which", ["norm_of_type", "quant_of_act"])
def test_norm_and_integer_rows(which):
    r = rule(function(LAYER, f"int {which}("))
    names = {n for _, n in r}
    assert len(names) == 11
    both({(form(r, M=M, N=N), N % 8 == 0) for M, N in NORM}, names, [n for n in names if "long" in n])


def test_gradients_row_by_row():
    r = [x for x in ROWS_RULE if x[1].startswith("launch_norm_grad<")]
    names = {n for _, n in r}
    assert len(names) == 9
    found = {(form(r, M=M, N=N), N % 8 == 0) for M, N in GRAD + GRAD_ONLY_IN_PLACE}
    both(found, names)
    for M, N in GRAD + GRAD_ONLY_IN_PLACE:
        assert few(M, N, False) == ((M, N) in GRAD_ONLY_IN_PLACE) and not few(M, N, True)
        R = int(form(r, M=M, N=N).rstrip(">").split(",")[-1])
        workgroups = min((M + R - 1) // R, 256)
        assert M > 2 * workgroups * R, "three rows in each place"


def test_gradients_in_one_launch():
    names = {n for _, n in FEW_RULE}
    assert len(names) == 8 and all(n.startswith("launch_norm_grad_few<") for n in names)
    both({(form(FEW_RULE, M=M, N=N), N % 8 == 0) for M, N in GRAD_FEW}, names)
    assert all(few(M, N, False) for M, N in GRAD_FEW)


def test_rows_back_from_experts():
    r = rule(function(EXPERTS, "int combine_of_type("))
    names = {n for _, n in r}
    assert len(names) == 4
    both({(form(r, T=T, N=N), N % 8 == 0) for T, _, N in COMBINE}, names)


def test_gradients_of_rows_back():
    r = [x for x in rule(function(EXPERTS, "int combine_grad_of_type(")) if x[0] != "(a.N == 0)"]
    names = {n for _, n in r}
    assert len(names) == 11, names
    both({(form(r, T=T, N=N), N % 8 == 0) for T, _, N in COMBINE_GRAD}, names, [n for n in names if "long" in n])


def test_rows_past_the_caches():
    """The size from which dispatched rows by part go past them is below that of the test that takes this way."""
    most = float(re.search(r"n \* bytes >= ([\de.]+)\)", EXPERTS).group(1))
    assert 8200 * 2 * 4099 * 2 >= most and 8200 * 2 <= 1 << 19
