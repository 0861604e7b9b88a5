"""The task form of the hand-scheduled key loops (cross attention): the
committed assembly is what the generator writes, passes the generator's
checks, and does the products of the attention's form (CPU only)."""
import pytest

from test_generated_loop import CSRC, load_gen

import os


def committed(d, form):
    text = open(os.path.join(CSRC, f"cross_d{d}_loop.inc")).read()
    head = f'#define DITANGO_CROSS_D{d}_{form}_ASM \\\n  "'
    start = text.index(head) + len(head)
    return text[start:text.index('\\n"\n', start)].split("\\n\\t")


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("fast", [False, True])
def test_committed_loop_matches_generator(d, fast):
    g = load_gen()
    g.configure(d)
    lines = g.generate(fast=fast, task=True)
    assert committed(d, "FAST" if fast else "LOOP") == lines
    assert committed(d, "LOAD") == g.first_tiles()
    assert g.check_hazards(lines) == [] and g.check_fragments(lines) == []


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("fast", [False, True])
def test_task_form_does_the_same_products(d, fast):
    """Every product is that of the attention's form; the queries are not read
    from LDS, and the next task's are loaded once on every way through the
    block: where it has one tile, and in the second to last of several."""
    g = load_gen()
    g.configure(d)
    one, task = g.generate(fast=fast), g.generate(fast=fast, task=True)
    products = lambda lines: [x for x in lines if x.startswith("v_mfma")]   # noqa: E731
    assert products(one) == products(task)
    loads = [x for x in task if x.startswith("global_load_dwordx4 a[")]
    assert len(loads) == 5 * 2 * (d // 16)          # the tail loop's four iterations, and a single tile
    assert len(set(loads)) == 2 * (d // 16)
    # they are waited for inside the block
    assert task[task.index(".Ldone_%=:") + 1].startswith("s_waitcnt vmcnt(0)")
    # every tile load but the first tiles' is the attention form's
    first = g.first_tiles()
    loads = lambda lines: [x for x in lines if x.startswith("buffer_load")]  # noqa: E731
    assert loads(one) == loads(first) + loads(task)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("fast", [False, True])
def test_last_wait_leaves_only_what_is_newer(d, fast):
    """In the last iteration the wait for the last values' tile leaves the loads
    behind it: a tile pair's and the next queries'."""
    g = load_gen()
    g.configure(d)
    lines = g.generate(fast=fast, task=True)
    lw, ks = g.LW, g.KS
    for u in range(4):
        k = lines.index(f".Llast{u}_%=:")
        wait = next(x for x in lines[k:] if x.startswith("s_waitcnt vmcnt"))
        assert wait == f"s_waitcnt vmcnt({2 * lw + 2 * ks})"
