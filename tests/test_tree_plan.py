"""wf_tree_plan and the defaults of its parameters (host arithmetic, no GPU needed)."""
import pytest

import paper_2606_00724_amd as wf
import treeforms


def params(**kw):
    return wf.make_tree_params(**{**dict(pages=4, page_rows=16, heads=2, head_dim=64, batch=2,
                                         max_rows=3, table_pages=2, group=2), **kw})


@pytest.mark.parametrize("kw", [
    dict(table_pages=1 << 22, page_rows=1024), dict(table_pages=1 << 21, page_rows=1024),
    dict(table_pages=(1 << 28) + 1), dict(batch=1 << 24, max_rows=256),
    dict(batch=(1 << 24) + 2, max_rows=256),
])
def test_defaults_past_32_bits_are_refused(kw):
    """A table of 2^32 rows, or as many tokens, is not taken for one of none or few."""
    p = params(**kw)
    assert min(p.max_len, p.tokens) > 0
    with pytest.raises(wf.WfError) as e:
        wf.tree_plan(p, 0)
    assert e.value.status == 2
    assert wf.tree_workspace_bytes(p) == 0


def test_defaults():
    p = params()
    assert (p.tokens, p.max_len) == (6, 32)
    p = params(table_pages=1 << 20, page_rows=1024)
    assert p.max_len == 1 << 30 and wf.tree_plan(p, 0).ranges == 1


@pytest.mark.parametrize("dtype,fmt,d,kernel,block,ranges", treeforms.ALL)
def test_every_form_has_a_shape(dtype, fmt, d, kernel, block, ranges):
    """What the tests of each form rely on."""
    kw = treeforms.find(wf, dtype, fmt, d, kernel, block, ranges)
    assert kw["max_rows"] <= kw["length"] <= kw["max_len"]
