"""The decoder layer with adapters on its projections against the layer oracle's parts, the adapters added per token in 64 bits."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import layer as OL
from paper_2512_03416_b200 import binding as B
from paper_2512_03416_b200 import workloads as wl
from paper_2512_03416_b200.adapters import Adapters
from paper_2512_03416_b200.harness import LoadedBatch, from_dev, to_dev
from paper_2512_03416_b200.layer import DecoderLayer
from tests.helpers import oracle_pool_with_context

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _need_gpu():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a CUDA device")


def bits(rng, shape, std):
    return wl.f32_to_bf16_bits((rng.standard_normal(shape) * std).astype(np.float32))


def adapter(rng, count, rank, n, k):
    """(a, b) as bf16 bits whose part of a product is about as large as the product's."""
    return bits(rng, (count, rank, k), k ** -0.5), bits(rng, (count, n, rank), rank ** -0.5)


def project(x_bits, w_bits, ad, scale, which):
    """x W^T and the adapters' part in 64 bits, u rounded to bf16."""
    x = OL.bits_to_f64(x_bits)
    y = OL.gemm(x, OL.bits_to_f64(w_bits))
    for t, i in enumerate(which):
        if ad is not None and i >= 0:
            u = OL.bits_to_f64(OL.f64_to_bits(scale[i] * (OL.bits_to_f64(ad[0][i]) @ x[t])))
            y[t] += OL.bits_to_f64(ad[1][i]) @ u
    return y


def layer_oracle(attention, x, wt, ads, scale, which, pos, s, eps=1e-5, theta=500000.0):
    R, F = OL.f64_to_bits, OL.bits_to_f64
    n = len(pos)
    h = R(OL.rmsnorm(F(x), F(wt["w_norm1"]), eps))
    qkv = project(h, wt["w_qkv"], ads.get("qkv"), scale, which)
    a, b = s.Hq * s.D, (s.Hq + s.Hkv) * s.D
    q, k, v = qkv[:, :a].reshape(n, s.Hq, s.D), qkv[:, a:b].reshape(n, s.Hkv, s.D), qkv[:, b:].reshape(n, s.Hkv, s.D)
    attn = R(np.asarray(attention(R(OL.rope(q, pos, theta)), R(OL.rope(k, pos, theta)), R(v)), np.float64).reshape(n, a))
    y = R(F(x) + project(attn, wt["w_o"], ads.get("o"), scale, which))
    h2 = R(OL.rmsnorm(F(y), F(wt["w_norm2"]), eps))
    g = R(project(h2, wt["w_gate"], ads.get("gate"), scale, which))
    u = R(project(h2, wt["w_up"], ads.get("up"), scale, which))
    z = R(OL.silu(F(g)) * F(u))
    return F(R(F(y) + project(z, wt["w_down"], ads.get("down"), scale, which)))


CASES = [
    # shape, hidden, intermediate, rank, cached, new, adapter of each row
    (wl.Shape(4, 2, 128), 256, 384, 8, [40, 0, 7], [1, 150, 1], [1, 0, -1]),
    (wl.Shape(8, 2, 128), 512, 1024, 24, [300, 17, 33, 0], [1, 1, 200, 130], [2, 2, 1, 0]),
    (wl.Shape(8, 2, 128), 2048, 1024, 64, [40, 0, 7, 1], [1, 33, 1, 1], [0, 1, 2, 0]),
    (wl.Shape(2, 2, 128), 128, 128, 16, [(7 * r) % 40 for r in range(401)], [1 + (r % 3 == 1) * (r % 5) for r in range(401)], [r % 4 - 1 for r in range(401)]),
]


@pytest.mark.parametrize("only", [None, "qkv", "o", "gate_up", "down"])
@pytest.mark.parametrize("case", CASES, ids=["4-2", "8-2", "8-2-deep", "401-rows"])
def test_layer_step_with_adapters_matches_the_oracle(case, only):
    s, hidden, inter, rank, ctx, ql, which = case
    rng = np.random.default_rng(rank)
    b = wl.make_batch("adapters", s, ctx, ql, seed=rank, profile="peaked", chunk_size=sum(ql))
    qd, kvd, count = s.Hq * s.D, s.Hkv * s.D, max(which) + 1
    wt = dict(w_qkv=bits(rng, (qd + 2 * kvd, hidden), hidden ** -0.5), w_o=bits(rng, (hidden, qd), qd ** -0.5),
              w_gate=bits(rng, (inter, hidden), hidden ** -0.5), w_up=bits(rng, (inter, hidden), hidden ** -0.5), w_down=bits(rng, (hidden, inter), inter ** -0.5))
    for k in ("w_norm1", "w_norm2"):
        wt[k] = wl.f32_to_bf16_bits((1.0 + 0.1 * rng.standard_normal(hidden)).astype(np.float32))
    ads = dict(qkv=adapter(rng, count, rank, qd + 2 * kvd, hidden), o=adapter(rng, count, rank, hidden, qd), gate=adapter(rng, count, rank, inter, hidden),
               up=adapter(rng, count, rank, inter, hidden), down=adapter(rng, count, rank, hidden, inter))
    if only is not None:
        ads = {k: v for k, v in ads.items() if k == only or (only == "gate_up" and k in ("gate", "up"))}
    scale = 0.5 + rng.random(count).astype(np.float32)
    x = bits(rng, (b.n_tokens, hidden), 1.0)
    pool, tm, pos = oracle_pool_with_context(b), b.table_matrix(), OL.positions(b.ctx_len, b.q_len)

    def attention(q, k, v):
        return oracle.mixed_step(pool, s.Hq, s.Hkv, s.D, s.P, 1.0 / math.sqrt(s.D), tm, b.ctx_len, b.q_len, q, k, v)

    of_token = np.repeat(which, ql)
    want = layer_oracle(attention, x, wt, ads, scale, of_token, pos, s)

    lb = LoadedBatch(b)
    dev = {k: to_dev(v) for k, v in wt.items()}
    layer = DecoderLayer(lb.dec, dev["w_norm1"], dev["w_qkv"], dev["w_o"], dev["w_norm2"], dev["w_gate"], dev["w_up"], dev["w_down"],
                         max_position=4096, rms_eps=1e-5, rope_theta=500000.0)
    x_in, outs = to_dev(x), [torch.full((b.n_tokens, hidden), 0x7FC0, dtype=torch.int16, device="cuda") for _ in range(3)]
    step = (lb.slots, b.q_len.tolist(), b.ctx_len.tolist(), x_in)
    layer.step(*step, outs[0], keep_len=True)
    gpu_scale = torch.from_numpy(scale).cuda()
    given = {name: Adapters(to_dev(ads[name][0]), to_dev(ads[name][1]), gpu_scale, "qkv" if name == "qkv" else "plain") for name in ("qkv", "o", "down") if name in ads}
    if "gate" in ads:                                     # adapters of their own: A below each other, B next to zeros
        zeros = np.zeros_like(ads["gate"][1])
        packed = layer.pack_gate_up_adapters(to_dev(np.concatenate([ads["gate"][1], zeros], 2)), to_dev(np.concatenate([zeros, ads["up"][1]], 2)))
        given["gate_up"] = Adapters(to_dev(np.concatenate([ads["gate"][0], ads["up"][0]], 1)), packed, gpu_scale, "gate_up")
    layer.set_adapters(**given)
    layer.step(*step, outs[1], keep_len=True)             # attached, not used
    for _ in range(2):
        layer.step(*step, outs[2], keep_len=True, adapters=which)
    torch.cuda.synchronize()
    assert lb.dec.device_status() == 0
    assert torch.equal(outs[0], outs[1])
    got = OL.bits_to_f64(from_dev(outs[2]))
    assert np.isfinite(got).all()
    # as for the layer without adapters: one spacing early in the chain of bf16 tensors is a few at its end
    err = np.abs(got - want)
    assert err.max() <= 2.0 ** -6 * np.abs(want).max(), (err.max(), np.abs(want).max())
    rel = np.linalg.norm(got - want, axis=1) / np.linalg.norm(want, axis=1)
    assert rel.max() <= 2e-2, rel.max()
    gp, wp = OL.bits_to_f64(lb.pool()), OL.bits_to_f64(pool)
    live = np.isfinite(wp)
    assert (np.isfinite(gp) == live).all()
    # a stored value's spacing, and a normalised input (up to 5) or a u (up to 8) that rounds the other way, times a weight of up to 4 standard
    # deviations: 2^-8 (5 * 4 / sqrt(hidden) + 8 * 4 / sqrt(rank)) of a rotated pair, whose value may cancel
    slack = 2.0 ** -8 * (20 / math.sqrt(hidden) + (32 / math.sqrt(rank) if "qkv" in ads else 0))
    assert (np.abs(gp[live] - wp[live]) <= 2.0 ** -7 * np.abs(wp[live]) + slack).all()
    layer.set_adapters()
    layer.step(*step, outs[1], keep_len=True)
    assert torch.equal(outs[0], outs[1])
    layer.close()


def test_layer_refuses_bad_adapters():
    s, hidden, inter = wl.Shape(4, 2, 128), 256, 384
    b = wl.make_batch("v", s, [5, 3], [1, 2], seed=3, chunk_size=8)
    lb = LoadedBatch(b)
    rng = np.random.default_rng(1)
    shapes = dict(w_norm1=(hidden,), w_qkv=(1024, hidden), w_o=(hidden, 512), w_norm2=(hidden,), w_gate=(inter, hidden), w_up=(inter, hidden), w_down=(hidden, inter))
    layer = DecoderLayer(lb.dec, **{k: to_dev(bits(rng, v, 0.1)) for k, v in shapes.items()}, max_position=64)
    x = torch.zeros((3, hidden), dtype=torch.int16, device="cuda")

    def made(n, k, count=2):
        return Adapters(*(to_dev(t) for t in adapter(rng, count, 8, n, k)))

    with pytest.raises(ValueError):
        layer.set_adapters(o=made(hidden, 256))
    with pytest.raises(RuntimeError):
        layer.set_adapters(o=made(hidden, 512), down=made(hidden, inter, 3))
    before = lb.dec.velocity()
    for given in ([0, 0], [2, -1], [-2, 0]):              # nothing attached yet, then out of range
        with pytest.raises(RuntimeError):
            layer.step(lb.slots, [1, 2], [5, 3], x, torch.empty_like(x), adapters=given)
        layer.set_adapters(o=made(hidden, 512))
    with pytest.raises(ValueError):
        layer.step(lb.slots, [1, 2], [5, 3], x, torch.empty_like(x), adapters=[0])
    assert lb.dec.velocity() == before
    layer.step(lb.slots, [1, 2], [5, 3], x, torch.empty_like(x), adapters=[-1, -1])
    torch.cuda.synchronize()
    layer.close()
