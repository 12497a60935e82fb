"""What the operators for 8-bit matrices and beams refuse.  Every call here is refused by the host before a device is asked for."""

import pytest

import paper_2411_15100_amd as xgm

A = 1 << 20      # an address that is never read
PROJECT = dict(d_hidden=A, dtype=1, d_hidden_scales=0, rows=2, k=256, hidden_stride=256, d_codes=A, d_scales=A, v=100, d_logits=A, logits_dtype=1,
               row_stride=100, d_work=A)


@pytest.mark.parametrize("change,status,text", [
    (dict(d_hidden=0), -1, "null"), (dict(d_codes=0), -1, "null"), (dict(d_scales=0), -1, "null"), (dict(d_logits=0), -1, "null"),
    (dict(d_work=0), -1, "no memory"), (dict(d_work=A + 8), -1, "aligned"), (dict(dtype=0), -1, "8 bits"), (dict(dtype=4), -1, "8 bits"),
    (dict(dtype=3), -1, "without their scales"), (dict(d_hidden_scales=A), -1, "not in 8 bits"), (dict(dtype=3, d_hidden_scales=A + 2), -1, "aligned"),
    (dict(logits_dtype=3), -1, "dtype"), (dict(logits_dtype=-1), -1, "dtype"), (dict(rows=0), -1, "positive"), (dict(rows=65536), -1, "XGM_MAX_ROWS"),
    (dict(v=0), -1, "positive"), (dict(v=0x7fff0001, row_stride=1 << 40), -1, "XGM_MAX_COLUMNS"), (dict(row_stride=99), -1, "stride"), (dict(k=0), -1, "multiple of 16"),
    (dict(k=250), -1, "multiple of 16"), (dict(k=65536 + 16, hidden_stride=1 << 20), -9, "XGM_MAX_HIDDEN"), (dict(hidden_stride=240), -1, "hidden stride"),
    (dict(hidden_stride=260), -1, "aligned"), (dict(dtype=3, d_hidden_scales=A, hidden_stride=264), -1, "aligned"), (dict(d_hidden=A + 8), -1, "aligned"),
    (dict(d_codes=A + 8), -1, "aligned"), (dict(d_scales=A + 2), -1, "aligned"), (dict(d_logits=A + 1), -1, "aligned"),
    (dict(d_bitmask=A, v_mask=0), -1, "v_mask"), (dict(d_bitmask=A, v_mask=0x7fffffff), -1, "XGM_MAX_COLUMNS")])
def test_projection_refuses(change, status, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.f8_logits(**{**PROJECT, **change})
    assert e.value.status == status and "f8_logits" in str(e.value)


QUANTIZE = dict(d_x=A, dtype=1, rows=2, k=256, stride=256, d_codes=2 * A, codes_stride=256, d_scales=3 * A)


@pytest.mark.parametrize("change,status,text", [
    (dict(d_x=0), -1, "null"), (dict(d_codes=0), -1, "null"), (dict(d_scales=0), -1, "null"), (dict(dtype=3), -1, "dtype"), (dict(rows=0), -1, "positive"),
    (dict(k=24), -1, "multiple of 16"), (dict(rows=1 << 16), -9, "XGM_MAX_ROWS"), (dict(k=1 << 17, stride=1 << 17, codes_stride=1 << 17), -9, "XGM_MAX_HIDDEN"),
    (dict(stride=255), -1, "stride"), (dict(codes_stride=240), -1, "stride"), (dict(stride=260), -1, "aligned"), (dict(codes_stride=264), -1, "aligned"),
    (dict(d_x=A + 2), -1, "aligned"), (dict(d_codes=A + 1), -1, "aligned"), (dict(d_scales=A + 1), -1, "aligned")])
def test_bringing_values_to_8_bits_refuses(change, status, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.f8_quantize(**{**QUANTIZE, **change})
    assert e.value.status == status


def test_working_memory():
    assert xgm.f8_work_bytes(1, 16) == 128 + 4 and xgm.f8_work_bytes(3, 272) == 3 * (384 + 12)
    assert xgm.f8_work_bytes(65535, 65536) == 65535 * (65536 + 2048)
    for rows, k, status in ((0, 16, -1), (1, -1, -1), (65536, 16, -9), (1, 65552, -9)):
        with pytest.raises(xgm.XgmError) as e:
            xgm.f8_work_bytes(rows, k)
        assert e.value.status == status


EMBED8 = dict(d_ids=A, n=3, d_codes=A, d_scales=A, v=100, k=256, factor=2, d_out=A, out_dtype=1, out_stride=256)
EMBED4 = dict(d_ids=A, n=3, d_codes=A, d_scales=A, scales_dtype=1, d_zeros=0, v=100, k=256, group=64, factor=2.5, d_out=A, out_dtype=1, out_stride=256)
EITHER = [(dict(d_ids=0), "null"), (dict(d_codes=0), "null"), (dict(d_scales=0), "null"), (dict(d_out=0), "null"), (dict(n=0), "positive"), (dict(n=-1), "positive"),
          (dict(n=(1 << 24) + 1), "2\\^24"), (dict(v=0), "positive"), (dict(k=0), "positive"), (dict(k=1 << 17, out_stride=1 << 17), "XGM_MAX_HIDDEN"), (dict(out_stride=255), "stride"),
          (dict(out_dtype=3), "dtype"), (dict(d_codes=A + 8), "aligned"), (dict(d_ids=A + 2), "aligned"), (dict(d_out=A + 1), "aligned"), (dict(d_scales=A + 1), "aligned")]


@pytest.mark.parametrize("change,text", EITHER + [(dict(k=200), "multiple of 16")])
def test_lookups_in_8_bits_refuse(change, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.f8_embed(**{**EMBED8, **change})
    assert e.value.status == -1 and "f8_embed" in str(e.value)


@pytest.mark.parametrize("change,text", EITHER + [(dict(group=48), "group"), (dict(group=0), "group"), (dict(group=96), "group"), (dict(scales_dtype=0), "bf16 or f16")])
def test_lookups_in_4_bits_refuse(change, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.q4_embed(**{**EMBED4, **change})
    assert e.value.status == -1 and "q4_embed" in str(e.value)


def test_a_factor_is_a_number():
    for call, args in ((xgm.q4_embed, EMBED4), (xgm.f8_embed, EMBED8)):
        with pytest.raises(TypeError):
            call(**{**args, "factor": "2"})


def _search(max_rows=16, v=1000):
    """A handle that holds sizes but no memory: calls that a check refuses never look at it."""
    import ctypes
    s = xgm.BeamSearch.__new__(xgm.BeamSearch)
    s._room = (ctypes.c_int64 * 4)(max_rows | v << 32, 0, 0, 0)
    s.__dict__["_h"] = ctypes.addressof(s._room)
    return s


SELECT = dict(d_logits=A, dtype=1, requests=4, beams=4, v=1000, row_stride=1000, rules=None, d_scores=A, d_ended=0, n_out=4, placed=False, d_rows=3 * A,
              d_ids=4 * A, d_out_scores=2 * A)


@pytest.mark.parametrize("change,status,text", [
    (dict(d_logits=0), -1, "null"), (dict(d_scores=0), -1, "null"), (dict(d_rows=0), -1, "null"), (dict(d_ids=0), -1, "null"), (dict(d_out_scores=0), -1, "null"),
    (dict(dtype=3), -1, "dtype"), (dict(requests=0), -1, "positive"), (dict(beams=0), -1, "positive"), (dict(n_out=0), -1, "positive"), (dict(v=0), -1, "positive"),
    (dict(beams=65), -9, "XGM_MAX_BEAMS"), (dict(n_out=129), -9, "XGM_MAX_CONTINUATIONS"), (dict(requests=5), -1, "created"), (dict(v=1001), -1, "created"),
    (dict(requests=1 << 30, beams=4), -1, "created"), (dict(row_stride=999), -1, "stride"), (dict(d_logits=A + 1), -1, "aligned"), (dict(n_out=8, placed=True), -1, "placed"),
    (dict(n_out=8, d_out_scores=A), -1, "in place"), (dict(d_scores=A + 2), -1, "aligned"), (dict(d_ended=A + 1), -1, "aligned"), (dict(d_rows=3 * A + 2), -1, "aligned"),
    (dict(d_ids=4 * A + 1), -1, "aligned"), (dict(d_out_scores=2 * A + 2), -1, "aligned"), (dict(d_out_scores=A + 4), -1, "overlap scores"),
    (dict(d_rows=A + 60), -1, "overlap scores"), (dict(d_ids=A), -1, "overlap scores"), (dict(d_out_scores=A, d_ids=A), -1, "overlap"),
    (dict(d_ended=3 * A - 60), -1, "overlap scores or ended"), (dict(d_ended=2 * A), -1, "overlap scores or ended"),
    (dict(d_rows=4 * A), -1, "overlap each other"), (dict(d_ids=2 * A + 32), -1, "overlap each other"), (dict(d_out_scores=3 * A - 4), -1, "overlap each other"),
    (dict(rules=xgm.LogitRules(d_bitmask=A)), -1, "v_mask")])
def test_continuations_refuse(change, status, text):
    s = _search()
    try:
        with pytest.raises(xgm.XgmError, match=text) as e:
            s.select(**{**SELECT, **change})
        assert e.value.status == status and "beam_select" in str(e.value)
    finally:
        s.__dict__["_h"] = None


def test_beams_refuse_sizes():
    for rows, v, status in ((0, 10, -1), (10, 0, -1), (65536, 10, -9), (10, (1 << 20) + 1, -9)):
        with pytest.raises(xgm.XgmError) as e:
            xgm.BeamSearch(rows, v)
        assert e.value.status == status


ROWS = dict(d_data=A, row_stride=64, outer_stride=64 * 8, part_stride=16, part_bytes=16, n_outer=2, n_parts=4)


@pytest.mark.parametrize("change,text", [
    (dict(d_data=0), "null"), (dict(n_outer=0), "positive"), (dict(n_parts=-1), "positive"), (dict(part_bytes=0), "positive"), (dict(row_stride=-64), "negative"),
    (dict(outer_stride=-1), "negative"), (dict(part_stride=-16), "negative"), (dict(d_used=8 * A), "unit"), (dict(d_used=8 * A, used_bytes=-4), "unit"),
    (dict(d_used=8 * A + 2, used_bytes=4), "aligned"), (dict(row_stride=63), "overlap"), (dict(part_stride=15), "overlap"), (dict(outer_stride=511), "overlap"),
    (dict(row_stride=0), "overlap"), (dict(row_stride=1 << 62), "address space"),
    (dict(d_used=8 * A, used_bytes=(1 << 62) + 1), "address space")])
def test_moving_rows_refuses(change, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.reorder_rows(xgm.RowSet(xgm.RowData(**{**ROWS, **change})), 4 * A, 8)
    assert e.value.status == -1 and "reorder_rows" in str(e.value)


def test_moving_rows_refuses_what_overlaps_and_too_many():
    one = xgm.RowData(**ROWS)                                                    # 1024 bytes from A on
    for arrays, d_rows, rows, status, text in [
            ((one,), 0, 8, -1, "null"), ((one,), 4 * A + 1, 8, -1, "aligned"), ((one,), 4 * A, 0, -1, "positive"), ((one,), 4 * A, 1025, -9, "XGM_BATCH_MAX_ROWS"),
            ((), 4 * A, 8, -1, "positive"), ((one,) * 9, 4 * A, 8, -9, "XGM_MAX_ROW_DATA"), ((one, one), 4 * A, 8, -1, "two arrays overlap"),
            ((one, xgm.RowData(**{**ROWS, "d_data": A + 1023})), 4 * A, 8, -1, "two arrays overlap"), ((one,), A + 1020, 8, -1, "sources"),
            ((one,), A - 28, 8, -1, "sources"), ((one, xgm.RowData(**{**ROWS, "d_data": 2 * A, "d_used": A + 64, "used_bytes": 4})), 4 * A, 8, -1, "lengths"),
            ((xgm.RowData(**{**ROWS, "d_used": A - 4, "used_bytes": 4}),), 4 * A, 8, -1, "lengths")]:
        with pytest.raises(xgm.XgmError, match=text) as e:
            xgm.reorder_rows(xgm.RowSet(*arrays), d_rows, rows)
        assert e.value.status == status
    with pytest.raises(xgm.XgmError, match="2\\^27") as e:
        xgm.reorder_rows(xgm.RowSet(xgm.RowData(d_data=1 << 40, row_stride=1, part_bytes=1, n_outer=1 << 14, outer_stride=1 << 20, n_parts=(1 << 13) + 1, part_stride=8)),
                         4 * A, 8)
    assert e.value.status == -9
    with pytest.raises(TypeError):
        xgm.RowSet(dict(ROWS))
    with pytest.raises(TypeError):
        xgm.reorder_rows([one], 4 * A, 8)
    with pytest.raises(TypeError, match="row_strid"):
        xgm.RowData(row_strid=4)
