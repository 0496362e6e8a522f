"""Arguments of the serving operators: what is refused before anything reaches the GPU (addresses here are never followed)."""
import pytest

from paper_2403_00176_b200 import binding as B

P = 4096                                     # an address; every refusal comes ahead of the first look at it
ROWS, CACHE = (P, 256, 64), (P, 4096, 256, 64)


def refused(status, fn, *args, text=""):
    with pytest.raises(B.Sod2Error) as e:
        fn(*args)
    assert e.value.status_name == "SOD2_E_" + status and text in str(e.value), str(e.value)


def with_changes(base, changes):
    a = list(base)
    for i, v in changes.items():
        a[i] = v
    return a


TABLES = [2, 100, 16, P, P + 64, P, 10, P, P, 8, 8, P, P + 128, P, P, P + 256, P, 0]


@pytest.mark.parametrize("changes,status", [
    ({0: -1}, "BAD_DIM"), ({1: -1}, "BAD_DIM"), ({1: 1 << 31}, "BAD_DIM"), ({0: 1 << 40}, "BAD_DIM"), ({2: 0}, "BAD_DIM"), ({2: -16}, "BAD_DIM"),
    ({6: -1}, "BAD_DIM"), ({6: 1 << 32}, "BAD_DIM"), ({9: 7}, "BAD_DIM"), ({10: -1, 9: 0}, "BAD_DIM"), ({3: None}, "INVALID_ARG"), ({4: 0}, "INVALID_ARG"),
    ({5: None}, "INVALID_ARG"), ({8: None}, "INVALID_ARG"), ({11: None}, "INVALID_ARG"), ({12: None}, "INVALID_ARG"), ({13: None}, "INVALID_ARG"),
    ({15: None}, "INVALID_ARG"), ({15: P, 7: P}, "INVALID_ARG"), ({12: P, 3: P}, "INVALID_ARG"), ({12: P + 64, 4: P + 64}, "INVALID_ARG")])
def test_page_tables_refuse(changes, status):
    refused(status, B.sod2_page_tables, *with_changes(TABLES, changes))


ROT = B.Rotation.sections((32,))
ROPE = [B.DTYPE_BF16, 10, 4, 2, 64, ROT, P, 10, ROWS, ROWS, ROWS, None, ROWS, CACHE, CACHE, 8, 16, P, None, 0]


@pytest.mark.parametrize("changes,status", [
    ({0: 2}, "INVALID_ARG"), ({0: 3}, "INVALID_ARG"), ({1: -1}, "BAD_DIM"), ({1: 1 << 31}, "BAD_DIM"), ({2: 0}, "INVALID_ARG"), ({2: -1}, "BAD_DIM"),
    ({3: 0}, "INVALID_ARG"), ({3: 5000}, "BAD_DIM"), ({4: 62}, "BAD_DIM"), ({4: 257}, "BAD_DIM"), ({5: B.Rotation([1.0, float("nan")], [0, 0])}, "INVALID_ARG"),
    ({5: B.Rotation.sections((33,))}, "BAD_DIM"), ({6: None}, "INVALID_ARG"), ({7: -1}, "BAD_DIM"), ({8: None}, "INVALID_ARG"), ({9: None}, "INVALID_ARG"),
    ({8: (0, 256, 64)}, "INVALID_ARG"), ({8: (P + 1, 256, 64)}, "MISALIGNED"), ({8: (P, -1, 64)}, "BAD_DIM"), ({10: None}, "INVALID_ARG"),
    ({13: None, 14: None, 12: None}, "INVALID_ARG"), ({12: None}, "INVALID_ARG"), ({14: None}, "INVALID_ARG"), ({13: (P, 1, -1, 1)}, "BAD_DIM"),
    ({15: -1}, "BAD_DIM"), ({16: 0}, "BAD_DIM"), ({17: None}, "INVALID_ARG"), ({2: 0, 3: 0, 8: None, 9: None, 10: None, 12: None, 13: None, 14: None}, "INVALID_ARG")])
def test_rope_refuses(changes, status):
    refused(status, B.sod2_rope_store, *with_changes(ROPE, changes))


def test_rotation_refuses():
    for freq, axis in (([], []), ([1.0], [0, 1]), ([1.0], [256]), ([1.0], [-1])):
        with pytest.raises(ValueError):
            B.Rotation(freq, axis)


PROMPT = [B.DTYPE_BF16, 2, 100, 4, 2, 64, ROWS, ROWS, ROWS, (2 * P, 256, 64), P, 0.125, P, 1 << 40, None, 0]


@pytest.mark.parametrize("changes,status", [
    ({0: 7}, "INVALID_ARG"), ({1: -1}, "BAD_DIM"), ({2: -1}, "BAD_DIM"), ({2: 1 << 31}, "BAD_DIM"), ({2: 1 << 24, 3: 1024, 4: 8}, "BAD_DIM"), ({3: 5}, "BAD_DIM"), ({3: 0}, "BAD_DIM"), ({4: 0}, "BAD_DIM"),
    ({3: 8192}, "BAD_DIM"), ({5: 0}, "BAD_DIM"), ({5: 257}, "BAD_DIM"), ({6: None}, "INVALID_ARG"), ({7: None}, "INVALID_ARG"), ({8: (0, 1, 1)}, "INVALID_ARG"),
    ({9: None}, "INVALID_ARG"), ({9: ROWS}, "INVALID_ARG"), ({6: (P + 1, 256, 64)}, "MISALIGNED"), ({7: (P, -256, 64)}, "BAD_DIM"), ({10: None}, "INVALID_ARG"),
    ({11: 0.0}, "INVALID_ARG"), ({11: -1.0}, "INVALID_ARG"), ({11: float("inf")}, "INVALID_ARG"), ({11: float("nan")}, "INVALID_ARG")])
def test_prompt_attention_refuses(changes, status):
    refused(status, B.sod2_attention_prompt, *with_changes(PROMPT, changes))


PAGED = [B.DTYPE_BF16, 2, 100, 1, 4, 2, 64, ROWS, (2 * P, 256, 64), P, P, CACHE, CACHE, 8, 16, P, 4, 4, 0.125, P, 1 << 40, None, 0]


@pytest.mark.parametrize("changes,status", [
    ({0: 2}, "INVALID_ARG"), ({1: -1}, "BAD_DIM"), ({2: 1 << 33}, "BAD_DIM"), ({3: -1}, "BAD_DIM"), ({4: 3}, "BAD_DIM"), ({6: 300}, "BAD_DIM"), ({7: None}, "INVALID_ARG"),
    ({8: ROWS}, "INVALID_ARG"), ({9: None}, "INVALID_ARG"), ({10: None}, "INVALID_ARG"), ({11: None}, "INVALID_ARG"), ({12: (P + 1, 1, 1, 1)}, "MISALIGNED"),
    ({12: (P, 1, -1, 1)}, "BAD_DIM"), ({13: -1}, "BAD_DIM"), ({13: 1 << 31}, "BAD_DIM"), ({14: 0}, "BAD_DIM"), ({15: None}, "INVALID_ARG"), ({16: 3}, "BAD_DIM"),
    ({17: -1}, "BAD_DIM"), ({18: -0.5}, "INVALID_ARG"), ({8: CACHE[:1] + (256, 64)}, "INVALID_ARG")])
def test_paged_attention_refuses(changes, status):
    refused(status, B.sod2_attention_paged, *with_changes(PAGED, changes))


@pytest.mark.parametrize("fn,base,which", [(B.sod2_page_tables, TABLES, {3: 2, 4: 1, 5: 2, 7: 2, 8: 2, 11: 2, 12: 1, 13: 4, 14: 2, 15: 2, 16: 2}),
                                           (B.sod2_rope_store, ROPE, {6: 2, 17: 4, 18: 1}), (B.sod2_attention_prompt, PROMPT, {10: 2, 14: 2}),
                                           (B.sod2_attention_paged, PAGED, {9: 2, 10: 1, 15: 2, 21: 2})])
def test_integers_off_their_alignment_are_refused(fn, base, which):
    for i, off in which.items():
        refused("MISALIGNED", fn, *with_changes(base, {i: 2 * P + off}))


def test_workspace_refuses():
    for heads in ((0, 1, 64), (4, 0, 64), (4, 3, 64), (4, 2, 0), (4, 2, 257)):
        refused("BAD_DIM", B.sod2_attention_workspace_bytes, *heads)


def test_wrong_kinds_of_arguments():
    for args in (PROMPT[:-1], with_changes(PROMPT, {6: (P, 1)}), with_changes(PROMPT, {6: P}), with_changes(PROMPT, {11: "x"}), with_changes(PROMPT, {1: "x"})):
        with pytest.raises((TypeError, ValueError)):
            B.sod2_attention_prompt(*args)


def test_empty_calls_do_nothing():
    # no tokens or no requests: nothing to read, no device needed
    B.sod2_attention_prompt(*with_changes(PROMPT, {2: 0, 6: None, 7: None, 8: None, 9: None}))
    B.sod2_attention_paged(*with_changes(PAGED, {1: 0, 7: None, 8: None, 10: None}))
    B.sod2_rope_store(*with_changes(ROPE, {1: 0}))
