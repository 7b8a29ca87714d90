"""What the operators of beam search refuse, on the CPU: every check of arguments comes before anything that needs a device."""
import ctypes

import pytest

EINVAL, EHIP = -1, -5
P = 1 << 20                                                          # stands for a device address (never used: each call ends before)


@pytest.fixture(scope="module")
def xg():
    import paper_2601_04426_amd as xg
    return xg


def select(xg, **kw):
    a = dict(logits_ptr=P, dtype=xg.XG2_F32, groups=2, beams=4, V=1000, row_stride_elems=1000, scores_ptr=P, n_out=4, out_scores_ptr=P, out_parents_ptr=P,
             out_tokens_ptr=P, workspace_ptr=P, workspace_bytes=1 << 24, bitmask_ptr=P, bm_row_stride_words=32, eos_id=0, finished_ptr=P, out_finished_ptr=P)
    a.update(kw)
    xg.beam_select(**a)


def rows(xg, **kw):
    a = dict(data_ptr=P, groups=2, beams=4, parents_ptr=P, row_stride=8 * 64 * 16, positions=64, position_bytes=16, outer=2, outer_stride=64 * 8 * 64 * 16, pieces=8,
             piece_stride=64 * 16)
    a.update(kw)
    xg.beam_reorder_rows(**a)


def trace(xg, **kw):
    a = dict(tokens_ptr=P, parents_ptr=P, steps=10, step_stride=8, groups=2, beams=4, out_ptr=P, out_stride=10, lengths_ptr=P)
    a.update(kw)
    xg.beam_backtrace(**a)


def refused(xg, call, code=EINVAL, **kw):
    with pytest.raises(xg.Xg2Error) as e:
        call(xg, **kw)
    assert e.value.code == code, kw
    return str(e.value)


@pytest.mark.parametrize("kw", [
    dict(dtype=2), dict(dtype=-1), dict(groups=-1), dict(beams=0), dict(beams=65), dict(groups=1 << 20, beams=2), dict(V=0), dict(V=-5), dict(V=(1 << 24) + 1, row_stride_elems=1 << 31),
    dict(n_out=0), dict(n_out=129), dict(over=2), dict(over=-1), dict(row_stride_elems=999), dict(bm_row_stride_words=31), dict(logits_ptr=0), dict(scores_ptr=0),
    dict(out_scores_ptr=0), dict(out_parents_ptr=0), dict(out_tokens_ptr=0), dict(workspace_ptr=0), dict(workspace_ptr=P + 8), dict(workspace_bytes=100), dict(logits_ptr=P + 2),
    dict(scores_ptr=P + 1), dict(out_tokens_ptr=P + 2), dict(finished_ptr=P + 3), dict(out_finished_ptr=P + 2), dict(bitmask_ptr=P + 2)])
def test_select_refuses(xg, kw):
    assert "xg2_beam_select" in refused(xg, select, **kw)


def test_select_workspace(xg):
    n = xg.beam_select_workspace(xg.XG2_BF16, 2, 4, 1000, 4)
    refused(xg, select, dtype=xg.XG2_BF16, workspace_bytes=n - 1)
    assert xg.beam_select_workspace(xg.XG2_F32, 0, 4, 1000, 4) == 0
    assert xg.beam_select_workspace(xg.XG2_F32, 1, 1, 1 << 24, 128) > 0
    for bad in ((2, 1, 1, 10, 1), (0, -1, 1, 10, 1), (0, 1, 65, 10, 1), (0, 1, 1, 0, 1), (0, 1, 1, 10, 0), (0, 1, 1, 10, 129)):
        with pytest.raises(xg.Xg2Error) as e:
            xg.beam_select_workspace(*bad)
        assert e.value.code == EINVAL
    assert xg.lib.xg2_beam_select_workspace(0, 1, 1, 10, 1, None) == EINVAL


@pytest.mark.parametrize("kw", [
    dict(groups=-1), dict(beams=0), dict(beams=65), dict(groups=1 << 20, beams=2), dict(outer=-1), dict(pieces=-1), dict(positions=-1), dict(position_bytes=-1),
    dict(outer=1 << 20, pieces=1 << 20), dict(outer=1, pieces=(1 << 23) + 1), dict(data_ptr=0), dict(parents_ptr=0), dict(parents_ptr=P + 2), dict(begin_ptr=P + 1), dict(end_ptr=P + 2),
    dict(row_stride=64 * 16 - 1), dict(row_stride=-8192), dict(piece_stride=1000), dict(outer_stride=0), dict(positions=1 << 30, position_bytes=1 << 40)])
def test_rows_refuse(xg, kw):
    assert "xg2_beam_reorder_rows" in refused(xg, rows, **kw)


@pytest.mark.parametrize("kw", [dict(steps=-1), dict(groups=-1), dict(beams=0), dict(beams=65), dict(groups=1 << 20, beams=2), dict(tokens_ptr=0), dict(parents_ptr=0), dict(out_ptr=0),
                                dict(step_stride=7), dict(out_stride=9), dict(tokens_ptr=P + 1), dict(out_ptr=P + 2), dict(lengths_ptr=P + 3)])
def test_backtrace_refuses(xg, kw):
    assert "xg2_beam_backtrace" in refused(xg, trace, **kw)


def test_reorder_refuses(xg):
    assert xg.lib.xg2_batch_reorder(None, 4, ctypes.c_void_p(P), None, None) == EINVAL


def test_nothing_to_do_needs_no_device(xg):
    select(xg, groups=0, logits_ptr=0)
    for kw in (dict(groups=0), dict(outer=0), dict(pieces=0), dict(positions=0), dict(position_bytes=0), dict(beams=1)):
        rows(xg, data_ptr=0, **kw)
    trace(xg, groups=0, tokens_ptr=0)
    trace(xg, steps=0, tokens_ptr=0, parents_ptr=0, out_ptr=0, lengths_ptr=0)


def test_without_a_device(xg, has_gpu):
    if has_gpu:
        pytest.skip("a GPU is present")
    for call in (select, rows, trace):
        refused(xg, call, EHIP)
