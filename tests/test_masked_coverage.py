"""Which kernels of masked attention the sizes of its GPU tests reach, by the
host's rules (no GPU needed)."""
import inspect

from paper_2401_11202_amd import partir as P
from tests import test_gpu_masked_attention as M

CUS = 256


def sizes(test):
    """The (B, Sq, Sk, Hq, Hk) of a test's parameters, and its forms (bit 0 a cap, bit 1 a bias)."""
    marks = {m.args[0]: m.args[1] for m in test.pytestmark if m.name == "parametrize"}
    shapes = next((v for k, v in marks.items() if k.startswith("B,")), [])
    names = next((k for k in marks if k.startswith("B,")), "")
    full = [(s[0], s[1], s[1], *s[2:]) if names == "B,S,Hq,Hk" else s[:5] for s in shapes]
    return full, {("cap" in f) + 2 * ("slopes" in f) for f in marks.get("f", [{}])}


def forward(B, Sq, Sk, Hq, Hk):
    """(waves over rows, key groups, whether the groups of a join share a row, XCD mapping) of the forward launch."""
    rows, parts = Hq // Hk * Sq, P.plan_masked_attention(B, Sq, Sk, Hq, Hk)["n_virtual_shards"]
    by_head = parts == 1 and B * Hk % 8 == 0
    join = None if parts == 1 else parts <= 4
    if rows <= 32:
        return 1, 4, join, by_head
    return 4, 2 if B * Hk * -(-rows // 128) * parts <= CUS else 1, join, by_head


TESTS = [(n, f) for n, f in inspect.getmembers(M, inspect.isfunction) if n.startswith("test_") and hasattr(f, "pytestmark")]


def reached():
    out = set()
    for _, t in TESTS:
        shapes, forms = sizes(t)
        out |= {(forward(*s), form) for s in shapes for form in forms}
    return out


def test_every_forward_kernel_runs_in_every_form():
    assert {(k[:2], form) for k, form in reached()} == {(k, form) for k in ((1, 4), (4, 2), (4, 1)) for form in range(4)}
    assert {k[2] for k, _ in reached()} == {None, True, False}
    assert {(k[:2], k[3]) for k, _ in reached()} >= {((4, 1), True), ((4, 1), False), ((4, 2), True), ((1, 4), True)}


def test_the_ring_of_three_blocks_ends_in_every_place():
    short = {-(-n // 32) for B, S, _, _, _ in sizes(M.test_many_short_sequences)[0] for n in (S - (37 * b) % (S + 1) for b in range(B))}
    assert {n % 3 for n in short if n > 3} == {0, 1, 2} and {0, 1, 2, 3} <= short


def test_the_gradients_run_in_every_form_with_even_and_other_groups_with_and_without_parts():
    got = set()
    for name, t in TESTS:
        shapes, forms = sizes(t)
        if name == "test_new_tokens_over_a_ragged_cache":
            shapes = [s for s in shapes if s[1] < 5]        # the others run no gradients
        for s in shapes:
            parts = P.plan_masked_attention_backward(*s)["n_virtual_shards"] > 1
            got |= {(s[2] <= 128, 16 % (s[3] // s[4]) == 0, form, parts) for form in forms}
    assert {k[:3] for k in got} == {(short, even, form) for short in (True, False) for even in (True, False) for form in range(4)}
    assert {(short, even, form, parts) for short in (True, False) for even in (True, False) for form in (0, 3) for parts in (True, False)} <= got
