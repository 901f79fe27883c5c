"""Descriptors of models with 4-bit matrices, and of encoders with padding, windows and sinks (no GPU)."""
import pytest

import paper_2306_03622_amd as tp
import synth


def mlp(width=256, group=64, layers=2):
    return synth.quantised(synth.mlp(layers, width, "bf16", "gelu", 3), group)


def bert(group=0, seq=40, attention=None, d=128, ffn=256, maxpos=64):
    m = synth.bert(seed=1, layers=2, d=d, heads=d // 64, ffn=ffn, seq=seq, vocab=100, maxpos=maxpos)
    if group:
        m = synth.quantised(m, group)
    if attention is not None:
        m.dims["attention"] = attention
    return m


def valid(m, mutate=None):
    d = tp.ModelDesc.of(m)
    t = [list(x) for x in d.tensors]
    if mutate:
        mutate(t)
    try:
        tp.tph_validate(tp.ModelDesc(m.arch, m.dtype, list(d.desc.dims), [tuple(x) for x in t]), m.total_bytes, L=tp.host_lib())
        return True
    except tp.TorporError as e:
        assert e.status == tp.TP_E_INVAL
        return False


@pytest.mark.parametrize("group", [32, 64, 128])
def test_four_bit_descriptors(group):
    assert valid(mlp(group=group)) and valid(bert(group, seq=64))
    m = mlp(group=group)
    codes = [i for i, t in enumerate(m.tensors) if t.role == "w"]
    assert m.tensors[codes[0]].nbytes == 256 * 128 and m.tensors[codes[0] + 1].nbytes == 2 * 256 * 256 // group
    assert not valid(mlp(192, group)) and not valid(bert(group, seq=64, d=64, ffn=128)) and not valid(bert(group, seq=64, ffn=192))
    assert not valid(m, lambda t: t[codes[0]].__setitem__(3, 256 * 256 * 2))            # bytes of a bf16 matrix
    assert not valid(m, lambda t: t[codes[0] + 1].__setitem__(4, [256, 256 // group + 1]))
    assert not valid(m, lambda t: t.pop(codes[0] + 1))                                  # no scales
    assert not valid(m, lambda t: t[codes[0] + 1].__setitem__(1, "qkv_scale"))
    r = synth.resnet50(1, classes=10, image=32)
    r.dtype = f"w4g{group}"
    assert not valid(r)


def test_scales_belong_to_four_bit_models_only():
    m = mlp(group=64)
    m.dtype = "bf16"
    assert not valid(m)
    m.dtype = "w4g32"
    assert not valid(m)


@pytest.mark.parametrize("seq,attention,ok", [
    (64, 0, True), (40, 0, False), (40, tp.tp_bert_attention(), True), (1, tp.tp_bert_attention(16, 2), True),
    (288, 0, False), (288, tp.tp_bert_attention(16, 2), True), (16384, tp.tp_bert_attention(65535, 16383), True),
    (16416, tp.tp_bert_attention(16), False), (64, 12345, True), (40, 12345, False)])
def test_encoders_with_attention_fields(seq, attention, ok):
    # a field without TP_BERT_ATTENTION's mark is none, as before there was one
    assert valid(bert(0, seq, attention, maxpos=max(64, seq))) == ok
    assert valid(bert(64, seq, attention, maxpos=max(64, seq))) == ok


def test_attention_field_and_its_refusals():
    src = open(tp.torpor.__file__.replace("paper_2306_03622_amd/torpor.py", "include/torpor.h")).read()
    assert "((int32_t)(0x40000000u | (uint32_t)(sinks) << 16 | (uint32_t)(window)))" in src
    assert tp.tp_bert_attention(3, 5) == 0x40000000 | 5 << 16 | 3
    for bad in ((-1, 0), (65536, 0), (0, -1), (0, 16384)):
        with pytest.raises(ValueError):
            tp.tp_bert_attention(*bad)


def test_workspace_holds_the_lengths_and_the_scratch():
    plain = tp.tp_workspace_bytes(tp.ModelDesc.of(bert(seq=64)), 3)
    assert tp.tp_workspace_bytes(tp.ModelDesc.of(bert(seq=64, attention=tp.tp_bert_attention())), 3) == plain + 256
    assert tp.tp_workspace_bytes(tp.ModelDesc.of(bert(64, seq=64)), 3) == plain
    assert tp.tp_workspace_bytes(tp.ModelDesc.of(mlp()), 3) == tp.tp_workspace_bytes(
        tp.ModelDesc.of(synth.mlp(2, 256, "bf16", "gelu", 3)), 3)


def test_cost_model_sees_fewer_bytes_and_keys():
    full = synth.mlp(4, 4096, "bf16", "gelu", 3)
    small = synth.quantised(full, 128)
    us = {m: sum(tp.tph_layer_costs(tp.ModelDesc.of(m2), m2.total_bytes, 1, L=tp.host_lib())) for m, m2 in
          (("full", full), ("small", small))}
    assert us["small"] < us["full"]
    assert 3.8 < full.total_bytes / small.total_bytes < 3.9
    cost = [sum(tp.tph_layer_costs(tp.ModelDesc.of(m), m.total_bytes, 8, L=tp.host_lib())) for m in
            (bert(0, 4096, tp.tp_bert_attention(64), maxpos=4096), bert(0, 4096, tp.tp_bert_attention(), maxpos=4096))]
    assert cost[0] < cost[1]
