"""What the operators around the mask refuse.  Every call here is refused by the host before a device is asked for."""

import ctypes

import pytest

import paper_2411_15100_amd as xgm
from paper_2411_15100_amd import binding

A = 1 << 20      # an address that is never read
PROJECT = dict(d_hidden=A, dtype=1, rows=2, k=256, hidden_stride=256, d_codes=A, d_scales=A, d_zeros=0, v=100, group=32, d_logits=A, logits_dtype=1,
               row_stride=100)


@pytest.mark.parametrize("change,status,text", [
    (dict(d_hidden=0), -1, "null"), (dict(d_codes=0), -1, "null"), (dict(d_scales=None), -1, "null"), (dict(d_logits=0), -1, "null"),
    (dict(dtype=0), -1, "bf16 or f16"), (dict(dtype=9), -1, "bf16 or f16"), (dict(logits_dtype=3), -1, "dtype"), (dict(rows=0), -1, "positive"),
    (dict(rows=-4), -1, "positive"), (dict(rows=65536), -1, "XGM_MAX_ROWS"), (dict(v=0), -1, "positive"), (dict(row_stride=99), -1, "stride"),
    (dict(group=0), -1, "group"), (dict(group=-32), -1, "group"), (dict(group=48), -1, "group"), (dict(group=96), -1, "group"),
    (dict(group=512), -1, "group"), (dict(k=0), -1, "group"), (dict(k=65536 + 32, hidden_stride=1 << 20), -9, "XGM_MAX_HIDDEN"),
    (dict(hidden_stride=255), -1, "hidden stride"), (dict(hidden_stride=260), -1, "aligned"), (dict(d_hidden=A + 8), -1, "aligned"),
    (dict(d_codes=A + 4), -1, "aligned"), (dict(d_scales=A + 1), -1, "aligned"), (dict(d_logits=A + 1), -1, "aligned"),
    (dict(d_logits=A + 2, logits_dtype=0), -1, "aligned")])
def test_projection_refuses(change, status, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.q4_logits(**{**PROJECT, **change})
    assert e.value.status == status and "q4_logits" in str(e.value)


@pytest.mark.parametrize("v_mask", [0, -5])
def test_projection_refuses_masks_of_no_vocabulary(v_mask):
    with pytest.raises(xgm.XgmError, match="v_mask") as e:
        xgm.q4_logits(**PROJECT, d_bitmask=A, v_mask=v_mask)
    assert e.value.status == -1


PROCESS = dict(d_logits=A, dtype=1, rows=2, v=100, row_stride=100, rules=None, d_out=2 * A, out_stride=100)
BAD_RULES = [(dict(d_bitmask=A), "v_mask"), (dict(d_tokens=A, d_n_tokens=A), "stride"), (dict(d_tokens=A, token_stride=8), "lengths"),
             (dict(d_tokens=A, d_n_tokens=A, token_stride=1 << 20), "XGM_MAX_HISTORY"), (dict(d_repetition=A), "history"), (dict(d_presence=A), "history"),
             (dict(d_frequency=A), "history"), (dict(d_bias_ids=A, d_bias=A), "offsets"), (dict(d_bias_ids=A, d_bias_offsets=A), "biases"),
             (dict(d_bias_ids=A, d_bias=A, d_bias_offsets=A, n_bias=-1), "number")]


@pytest.mark.parametrize("change,text", [
    (dict(d_logits=0), "null"), (dict(d_out=0), "null"), (dict(dtype=7), "dtype"), (dict(rows=0), "positive"), (dict(v=-1), "positive"),
    (dict(rows=70000), "XGM_MAX_ROWS"), (dict(row_stride=99), "stride"), (dict(out_stride=10), "stride"), (dict(d_logits=A + 1), "aligned"),
    (dict(d_out=A + 2, dtype=0), "aligned"), (dict(d_out=A, out_stride=128), "in place")])
def test_rules_refuse(change, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.process_logits(**{**PROCESS, **change})
    assert e.value.status == -1 and "process_logits" in str(e.value)


@pytest.mark.parametrize("rules,text", BAD_RULES)
def test_incomplete_rules_are_refused(rules, text):
    with pytest.raises(xgm.XgmError, match=text) as e:
        xgm.process_logits(**{**PROCESS, "rules": xgm.LogitRules(**rules)})
    assert e.value.status == -1


def test_unknown_names_and_what_is_no_struct():
    with pytest.raises(TypeError, match="d_bitmsk"):
        xgm.LogitRules(d_bitmsk=A)
    with pytest.raises(TypeError, match="d_topk"):
        xgm.DrawRules(d_topk=A)
    with pytest.raises(AttributeError):
        xgm.process_logits(**{**PROCESS, "rules": 5})
    with pytest.raises(TypeError):
        xgm.process_logits(**{**PROCESS, "rows": "2"})


MOST = 0x7fff0000    # logits a row


@pytest.mark.parametrize("v", [MOST + 1, 2 ** 31 - 8, 2 ** 31 - 1])
def test_rows_whose_places_do_not_fit_32_bits_are_refused(v):
    for call in (lambda: xgm.process_logits(**{**PROCESS, "v": v, "row_stride": v, "out_stride": v}), lambda: xgm.q4_logits(**{**PROJECT, "v": v, "row_stride": v}),
                 lambda: xgm.process_logits(**{**PROCESS, "rules": xgm.LogitRules(d_bitmask=A, v_mask=v)}), lambda: xgm.q4_logits(**PROJECT, d_bitmask=A, v_mask=v)):
        with pytest.raises(xgm.XgmError, match="XGM_MAX_COLUMNS") as e:
            call()
        assert e.value.status == -1


def test_one_struct_is_not_taken_for_the_other():
    class AnotherSampler:
        _h = 0

    sampler, rules, draw = AnotherSampler(), xgm.LogitRules(), xgm.DrawRules(d_uniform=A)
    for a, b, found, expected in ((draw, rules, "DrawRules", "LogitRules"), (draw, None, "DrawRules", "LogitRules"), (rules, rules, "LogitRules", "DrawRules"),
                                  (None, rules, "LogitRules", "DrawRules"), (rules, AnotherStruct(), "AnotherStruct", "DrawRules")):
        with pytest.raises(TypeError, match=f"{found} where .*{expected}"):
            xgm.Sampler.sample(sampler, A, 1, 2, 100, 100, a, b, A)
    with pytest.raises(TypeError, match="DrawRules where .*LogitRules"):
        xgm.process_logits(**{**PROCESS, "rules": draw})
    with pytest.raises(xgm.XgmError, match="null sampler"):         # in the right order they get as far as that
        xgm.Sampler.sample(sampler, A, 1, 2, 100, 100, rules, draw, A)


class AnotherStruct:
    _addr = A


def test_samplers_refuse():
    for rows, v, status in ((0, 10, -1), (4, 0, -1), (-1, 10, -1), (65536, 10, -9), (4, (1 << 20) + 1, -9)):
        with pytest.raises(xgm.XgmError, match="sampler_create") as e:
            xgm.Sampler(rows, v)
        assert e.value.status == status
    lib = xgm.load_library()
    assert lib.xgm_sampler_create(1, 1, None, None) == -1
    assert lib.xgm_sample(None, A, 1, 2, 100, 100, None, None, A, None, None) == -1
    assert b"null sampler" in lib.xgm_last_error()
    lib.xgm_sampler_destroy(None)


def test_the_structs_are_laid_out_as_in_the_header():
    rules = xgm.LogitRules(d_bitmask=A, d_bias_offsets=7 * A, token_stride=1 << 33, v_mask=5, n_bias=6)
    raw = ctypes.string_at(rules._addr, ctypes.sizeof(rules._s))
    words = [int.from_bytes(raw[8 * k:8 * k + 8], "little") for k in range(len(raw) // 8)]
    assert words == [A] + [0] * 8 + [7 * A, 1 << 33, 5 | 6 << 32]
    draw = xgm.DrawRules(d_uniform=A)
    assert ctypes.sizeof(draw._s) == 40 and ctypes.string_at(draw._addr, 40)[32:] == A.to_bytes(8, "little")
    assert binding.LogitRules is xgm.LogitRules
