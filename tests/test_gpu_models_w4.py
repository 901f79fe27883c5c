"""Models that run the operators: MLPs and encoders with 4-bit matrices, encoders with padding, a window and sinks, and both in
one, through tp_infer against the oracle."""
import numpy as np
import pytest

import synth
from tests.common import check_parity, infer, log, make_runtime, record_parity, to_device, torch_dev

pytestmark = pytest.mark.gpu

TOL = 2e-2


def mlp(layers, width, group, act="gelu", seed=21):
    return synth.quantised(synth.mlp(layers, width, "bf16", act, seed), group)


def encoder(seq, window=None, sinks=0, group=0, layers=2, d=256, ffn=512, seed=41):
    import paper_2306_03622_amd as tp
    m = synth.bert(seed=seed, layers=layers, d=d, heads=d // 64, ffn=ffn, seq=seq, vocab=300, maxpos=max(seq, 64), std=0.06)
    if group:
        m = synth.quantised(m, group)
    if window is not None:
        m.dims.update(window=window, sinks=sinks, attention=tp.tp_bert_attention(window, sinks))
    return m


def padded(batch, seq, lens, seed=5):
    ids = synth.bert_input(batch, seed, seq=seq, vocab=300)
    for i, n in enumerate(lens):
        ids[i, n:] = -1 - (np.arange(seq - n) % 3)
    return ids


def check_samples(got, m, ids):
    """Like check_parity, over each sample's own tokens."""
    from oracle import forward as oracle
    ref = oracle.forward(m, ids)
    assert np.isfinite(got).all()
    worst = 0.0
    for g, r, row in zip(got, ref, ids):
        n = int(np.argmax(row < 0)) if (row < 0).any() else len(row)
        if n:
            worst = max(worst, float(np.abs(g[:n] - r[:n]).max() / np.abs(r[:n]).max()))
    record_parity(m, ids.shape[0], worst, TOL)
    log(f"  normwise error {worst:.3e}")
    assert worst <= TOL


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("layers,width,batch", [(1, 128, 1), (3, 256, 5), (2, 512, 33), (2, 384, 129), (2, 1024, 300)])
def test_mlp(layers, width, batch, group):
    log(f"4-bit MLP {layers} x {width}, groups of {group}, batch {batch}")
    m = mlp(layers, width, group)
    x = synth.mlp_input(batch, width, m.dtype, 77)
    rt, (mid,) = make_runtime([m], batch_max=batch)
    cold = infer(rt, mid, m, x)
    check_parity(cold, m, x, TOL)
    assert np.array_equal(infer(rt, mid, m, x), cold)
    rt.close()


def test_registered_image_is_blocked():
    import paper_2306_03622_amd as tp
    m = mlp(2, 256, 64)
    rt, (mid,) = make_runtime([m])
    img, raw = rt.host_image(mid), m.blob()
    for t in m.tensors:
        have, want = img[t.offset:t.offset + t.nbytes], raw[t.offset:t.offset + t.nbytes]
        if t.role == "w":
            s = m.tensor(t.name + ".scale")
            codes = want.reshape(256, 128)
            bits = raw[s.offset:s.offset + s.nbytes].view(np.uint16).reshape(s.shape)
            c, sc = tp.tpo_w4_pack(codes, bits, 64)
            assert np.array_equal(have, c)
            assert np.array_equal(img[s.offset:s.offset + s.nbytes], sc.view(np.uint8))
        elif t.role == "b":
            assert np.array_equal(have, want)
    rt.swap_in(mid)
    torch_dev()[0].cuda.synchronize()
    assert np.array_equal(rt.extent(mid).cpu().numpy(), img)
    rt.close()


@pytest.mark.parametrize("seq,window,sinks,lens", [
    (96, 0, 0, [96, 50, 1]), (75, 0, 0, [75, 74, 33]), (300, 16, 1, [300, 7, 131]), (513, 100, 4, [513, 512, 0]), (1, 0, 0, [1, 0, 1]),
    (256, 65535, 0, [256, 200, 100]), (40, 1, 0, [40, 39, 2])])
@pytest.mark.parametrize("group", [0, 64])
def test_encoder(seq, window, sinks, lens, group):
    # the weights' spread singles keys out (see test_gpu_attention.py: exponents of std (16 0.06)^2 64 / 8 = 0.9 and more)
    log(f"encoder of {seq} tokens, window {window}, sinks {sinks}, groups of {group}")
    m = encoder(seq, window, sinks, group)
    ids = padded(len(lens), seq, lens)
    rt, (mid,) = make_runtime([m], batch_max=len(lens))
    got = infer(rt, mid, m, ids)
    check_samples(got, m, ids)
    assert np.array_equal(infer(rt, mid, m, ids), got)
    # what stands behind a sample's end does not reach it
    other = ids.copy()
    other[ids < 0] = -100
    for i, n in enumerate(lens):
        if n + 1 < seq:
            other[i, n + 1:] = 7
    again = infer(rt, mid, m, other)
    for i, n in enumerate(lens):
        assert np.array_equal(again[i, :n], got[i, :n])
    rt.close()


@pytest.mark.parametrize("group", [32, 128])
def test_four_bit_encoder_without_padding(group):
    m = encoder(128, group=group)
    ids = synth.bert_input(3, 9, seq=128, vocab=300)
    rt, (mid,) = make_runtime([m], batch_max=3)
    check_parity(infer(rt, mid, m, ids), m, ids, TOL)
    rt.close()


def test_unpadded_masked_encoder_agrees_with_the_plain_one():
    plain, masked = encoder(128), encoder(128, 0)
    ids = synth.bert_input(2, 10, seq=128, vocab=300)
    rt, (a, b) = make_runtime([plain, masked], batch_max=2)
    x, y = infer(rt, a, plain, ids), infer(rt, b, masked, ids)
    rt.close()
    assert np.abs(x - y).max() <= TOL * np.abs(x).max()


@pytest.mark.parametrize("kind", ["mlp", "encoder"])
def test_residency_does_not_change_the_result(kind):
    """Cold, warm, replayed from a graph at other buffers, in another extent, read in place, without allocation: the same bits."""
    import paper_2306_03622_amd as tp
    torch, dev = torch_dev()
    if kind == "mlp":
        m, x_np, shape = mlp(18, 256, 64), synth.mlp_input(9, 256, "w4g64", 3), (9, 256)      # 18 kernels: a graph
    else:
        m, shape = encoder(200, 30, 2, 64, layers=3), (4, 200, 256)
        x_np = padded(4, 200, [200, 150, 3, 77])
    batch = shape[0]
    other = mlp(2, 512, 128, seed=5)
    rt, (mid, oid) = make_runtime([m, other], batch_max=batch)
    want = infer(rt, mid, m, x_np)
    s = torch.cuda.Stream(device=dev)
    xs = [to_device(x_np) for _ in range(3)]
    outs = [torch.full(shape, float("nan"), dtype=torch.float32, device=dev) for _ in range(3)]
    torch.cuda.synchronize()
    for i in (0, 1, 2, 0):
        rt.infer(mid, xs[i], outs[(i + 1) % 3], stream=s)
    s.synchronize()
    for o in outs:
        assert np.array_equal(o.cpu().numpy(), want)
    assert rt.stats()["graph_captures"] >= 1 and rt.stats()["graph_repoints"] >= 1
    for i in (mid, oid):                                     # into another extent
        rt.evict(i)
    infer(rt, oid, other, synth.mlp_input(2, 512, "w4g128", 1))
    for _ in range(2):
        assert np.array_equal(infer(rt, mid, m, x_np), want)
    outs[0].fill_(float("nan"))
    torch.cuda.synchronize()
    rt.infer_noalloc(mid, xs[0], outs[0], stream=s)
    s.synchronize()
    assert np.array_equal(outs[0].cpu().numpy(), want)
    rt.close()
    for kw in ({"direct_max_bytes": 1 << 30}, {"copy_method": tp.TP_COPY_ZERO}, {"copy_method": tp.TP_COPY_GATHER},
               {"flags": tp.TP_FLAG_SERIAL}, {"plan": tp.TP_PLAN_COST}, {"flags": tp.TP_FLAG_NO_GRAPH}):
        rt, (mid,) = make_runtime([m], batch_max=batch, **kw)
        for _ in range(2):
            assert np.array_equal(infer(rt, mid, m, x_np), want), kw
        rt.close()


@pytest.mark.parametrize("batch", [2, 50])
def test_mlp_input_off_a_16_byte_boundary(batch):
    torch, dev = torch_dev()
    m = mlp(3, 256, 32)
    x_np = synth.mlp_input(batch, 256, m.dtype, 8)
    rt, (mid,) = make_runtime([m], batch_max=batch)
    want = infer(rt, mid, m, x_np)
    base = torch.zeros(batch * 256 + 8, dtype=torch.int16, device=dev)
    out = torch.empty(batch, 256, dtype=torch.float32, device=dev)
    s = torch.cuda.Stream(device=dev)
    for off in (1, 2, 5):
        base[off:off + batch * 256] = to_device(x_np).reshape(-1)
        torch.cuda.synchronize()
        rt.infer(mid, base[off:off + batch * 256].view(batch, 256), out, stream=s)
        s.synchronize()
        assert np.array_equal(out.cpu().numpy(), want)
    rt.close()


def test_samples_of_a_batch_are_their_own():
    m = encoder(160, 40, 1, 64)
    ids = padded(5, 160, [160, 90, 31, 160, 1])
    rt, (mid,) = make_runtime([m], batch_max=5)
    got = infer(rt, mid, m, ids)
    for i in range(5):
        alone = infer(rt, mid, m, ids[i:i + 1])
        n = int((ids[i] >= 0).sum())
        # other batches may take other tiles, which round sums otherwise: within bf16 rounding
        assert np.abs(alone[0, :n] - got[i, :n]).max() <= TOL * np.abs(got[i, :n]).max()
    rt.close()
