"""The AdamW step: bit for bit against its formulas in float32 on the CPU (every operation
rounded on its own, 8-bit codes included), and against the definition in 64 bits.

Against 64 bits, one step from the same state: m and v are two products and a sum, 3 roundings of
2^-24; the update is a root, two divisions and two products of such values, 12 roundings; the
weight adds two more; and (1 - beta) and the bias corrections are rounded to float32 once."""
import math

import pytest
import torch

from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
KINDS = [("f32", "f32", False), ("f32", "bf16", False), ("bf16", "f32", False),
         ("bf16", "bf16", False), ("bf16", "f32", True), ("bf16", "bf16", True)]
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HYPER = {"lr": 3e-3, "betas": (0.9, 0.99), "eps": 1e-8, "weight_decay": 0.1}


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def blocks_of(x):
    pad = (-x.numel()) % 256
    return torch.cat([x.reshape(-1), x.new_zeros(pad)]).view(-1, 256)


def scaled(x, top):
    b = blocks_of(x)
    most = b.abs().amax(1, keepdim=True)
    live = ~(most < 2.0 ** -100)
    by = torch.full_like(most, top) / torch.where(live, most, 1.0)
    return b * torch.where(live, by, 0.0), torch.where(live, most, 0.0) * (1 / top)


def pack_m(m):
    y, s = scaled(m, 256.0)
    return y.to(torch.float8_e4m3fn).reshape(-1)[:m.numel()], s.reshape(-1)


def unpack_m(c, s):
    return (blocks_of(c.float()) * s.view(-1, 1)).reshape(-1)[:c.numel()]


def r_values():
    c = torch.arange(256)
    return torch.where(c < 16, c / 16, (1 + c % 16 / 16) * 2.0 ** (c // 16 - 1)).float()


def pack_r(r):
    """The code whose value is nearest (a tie goes to the even code; never 0 for a positive r)."""
    y, s = scaled(r, 16384.0)
    table = r_values()
    hi = torch.searchsorted(table, y.contiguous()).clamp(1, 255)
    lo = hi - 1
    dlo, dhi = y - table[lo], table[hi] - y
    code = torch.where((dhi < dlo) | ((dhi == dlo) & (hi % 2 == 0)), hi, lo)
    code = torch.where(y > 0, code.clamp(min=1), 0)
    return code.to(torch.uint8).reshape(-1)[:r.numel()], s.reshape(-1)


def unpack_r(c, s):
    return (blocks_of(r_values()[c.long()]) * s.view(-1, 1)).reshape(-1)[:c.numel()]


def plain_step(w, g, m, v, t, h):
    """float32 on the CPU; m and v are the moments, returns (w, m, v, sqrt(v))"""
    b1, b2 = h["betas"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    r = v.sqrt()
    over = r * (1 / math.sqrt(1 - b2 ** t)) + h["eps"]
    return w * (1 - h["lr"] * h["weight_decay"]) - m / over * (h["lr"] / (1 - b1 ** t)), m, v, r


def setup(ns, kind, seed, scale=1.0):
    pd, gd, master = kind
    g = torch.Generator().manual_seed(seed)
    w = [torch.randn(n, generator=g) for n in ns]
    params = [x.to(DT[pd]).cuda() for x in w]
    grads = [torch.zeros(n, dtype=DT[gd], device="cuda") for n in ns]
    masters = [x.cuda() for x in w] if master else None
    return g, params, grads, masters


SIZES = [[1], [3, 255, 256, 257], [2047, 2048, 2049, 5, 0, 70001], [100] * 60, [300] * 500]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("ns", SIZES, ids=["one", "blocks", "ragged", "sixty", "many"])
def test_bit_for_bit(ns, kind, bits):
    g, params, grads, masters = setup(ns, kind, 7)
    opt = flarepp.AdamW(params, grads, state_bits=bits, masters=masters, **HYPER)
    w = [x.cpu().float() for x in (masters or params)]
    st = [(torch.zeros(n), torch.zeros(n)) for n in ns]
    for t in range(1, 4):
        for i, n in enumerate(ns):
            x = torch.randn(n, generator=g) * 10.0 ** (torch.rand(n, generator=g) * 6 - 4)
            x[::17] = 0
            grads[i].copy_(x)
        opt.step()
        for i, n in enumerate(ns):
            if n == 0:
                continue
            m, v = st[i]
            w[i], m, v, r = plain_step(w[i], grads[i].cpu().float(), m, v, t, HYPER)
            if bits == 8:
                mc, ms = pack_m(m)
                rc, rs = pack_r(r)
                assert torch.equal(opt.m[i].cpu().view(torch.uint8), mc.view(torch.uint8))
                assert torch.equal(opt.v[i].cpu(), rc)
                assert torch.equal(opt.m_scale[i].cpu(), ms) and torch.equal(opt.v_scale[i].cpu(), rs)
                m, v = unpack_m(mc, ms), unpack_r(rc, rs).square()
            st[i] = (m, v)
            if masters:
                assert torch.equal(masters[i].cpu(), w[i])
            assert torch.equal(params[i].cpu(), w[i].to(params[i].dtype))
            if not masters:
                w[i] = params[i].cpu().float()
    mo, vo = opt.moments()
    for i, n in enumerate(ns):
        assert torch.equal(mo[i].cpu().view(-1), st[i][0]) and torch.equal(vo[i].cpu().view(-1), st[i][1])
    assert opt.steps == 3


def test_against_64_bits():
    n = 50001
    g, params, grads, _ = setup([n], ("f32", "f32", False), 3)
    grads[0].copy_(torch.randn(n, generator=g) * 1e-3)
    m0, r0 = torch.randn(n, generator=g) * 1e-3, torch.rand(n, generator=g) * 1e-3 + 1e-5
    state = {"m": [m0.cuda()], "v": [(r0 * r0).cuda()], "step": 41}
    w0, v0 = params[0].double().cpu(), state["v"][0].double().cpu()
    opt = flarepp.AdamW(params, grads, state=state, **HYPER)
    opt.step()
    (b1, b2), t, lr = HYPER["betas"], 42, HYPER["lr"]
    gd = grads[0].double().cpu()
    m = b1 * m0.double() + (1 - b1) * gd
    v = b2 * v0 + (1 - b2) * gd ** 2
    up = lr * (m / (1 - b1 ** t)) / ((v / (1 - b2 ** t)).sqrt() + HYPER["eps"])
    w = w0 - up - lr * HYPER["weight_decay"] * w0
    # m is a difference of its two terms: its error goes by their sizes
    m_mag = b1 * m0.double().abs() + (1 - b1) * gd.abs()
    m_err = 4 * EPS * m_mag
    assert bool(((state["m"][0].double().cpu() - m).abs() <= m_err).all())
    assert bool(((state["v"][0].double().cpu() - v).abs() <= 6 * EPS * v).all())
    bound = 4 * EPS * (w0.abs() + w.abs()) + 16 * EPS * up.abs() * (m_mag / m.abs().clamp(min=1e-30))
    assert bool(((params[0].double().cpu() - w).abs() <= bound).all())


def test_8_bit_states_track_the_full_ones():
    """A noisy quadratic: both optimisers arrive, and the 8-bit moments stay within the rounding of
    their codes (2^-4 of an m's binade, 2^-5 of a sqrt(v)'s) plus what the codes' ends cut off."""
    n, gen = 4096, torch.Generator(device="cuda").manual_seed(0)
    target = torch.randn(n, device="cuda", generator=gen)
    got = {}
    for bits in (32, 8):
        p, g = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")]
        opt = flarepp.AdamW(p, g, lr=2e-2, weight_decay=0.0, state_bits=bits)
        gen.manual_seed(1)
        for k in range(400):
            opt.lr = 2e-2 * (1 - k / 400)
            g[0].copy_(p[0] - target + 0.1 * torch.randn(n, device="cuda", generator=gen))
            opt.step()
        got[bits] = float((p[0] - target).abs().mean())
    assert got[32] < 0.05 and got[8] < 0.05, got


def test_small_and_special_values_in_8_bits():
    n = 256 * 4
    p, g = [torch.zeros(n, device="cuda")], [torch.zeros(n, device="cuda")]
    opt = flarepp.AdamW(p, g, state_bits=8, **HYPER)
    g[0][0:256] = 1e-36              # squares and moments vanish: the block is stored as zeros
    g[0][256:512] = 1.0
    g[0][300] = 1e-9                 # far below its block's largest: v must not become zero
    g[0][512:768] = 2.0
    g[0][700] = float("nan")
    opt.step()
    m, v = (t[0].cpu() for t in opt.moments())
    assert not m[:256].any() and not v[:256].any() and float(opt.v_scale[0][0]) == 0
    assert float(v[300]) > 0 and torch.isfinite(v[256:512]).all()
    assert m[512:768].isnan().all() and v[512:768].isnan().all()  # that block, and only that one
    assert not m[768:].any() and not v[768:].any()
    assert torch.isfinite(p[0][:700]).all() and p[0][700].isnan() and torch.isfinite(p[0][701:]).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_nothing_outside_and_on_another_stream(bits):
    ns = [1000, 77]
    bufs, ps, gs = [], [], []
    for n in ns:
        b = torch.full((n + 512,), 4.0, device="cuda", dtype=torch.bfloat16)
        bufs.append(b)
        ps.append(b[256:256 + n])
        gs.append(torch.randn(n, device="cuda"))
    opt = flarepp.AdamW(ps, gs, state_bits=bits, masters=True, **dict(HYPER, lr=0.5))
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    opt.step(stream=s)
    s.synchronize()
    for b, n in zip(bufs, ns):
        assert (b[:256] == 4).all() and (b[256 + n:] == 4).all() and (b[256:256 + n] != 4).any()


def test_state_goes_on():
    ns = [500, 1000]
    for bits in (32, 8):
        g, params, grads, _ = setup(ns, ("bf16", "f32", False), 9)
        for x in grads:
            x.normal_(generator=torch.Generator(device="cuda").manual_seed(2))
        whole = flarepp.AdamW(params, grads, state_bits=bits, masters=True, **HYPER)
        half_p = [p.clone() for p in params]
        half = flarepp.AdamW(half_p, grads, state_bits=bits,
                             masters=[m.clone() for m in whole.masters], **HYPER)
        for _ in range(4):
            whole.step()
        half.step()
        half.step()
        saved = {k: [t if t is None else t.clone() for t in x] if isinstance(x, list) else x
                 for k, x in half.state_dict().items()}
        rest = flarepp.AdamW(half_p, grads, state_bits=bits, masters=half.masters, state=saved,
                             **HYPER)
        rest.step()
        rest.step()
        for a, b in zip(params, half_p):
            assert torch.equal(a, b)


def test_scales_of_all_tensors_in_one_buffer():
    """Views of one buffer of scales start at any multiple of four bytes."""
    ns = [300, 5, 1000]
    g, params, grads, _ = setup(ns, ("f32", "f32", False), 4)
    for x in grads:
        x.copy_(torch.randn(x.numel(), generator=g))
    blocks = [-(-n // 256) for n in ns]
    at = [sum(blocks[:i]) for i in range(len(ns))]
    ms, vs = (torch.zeros(sum(blocks), device="cuda") for _ in "mv")
    state = {"m": [torch.zeros(n, dtype=torch.float8_e4m3fn, device="cuda") for n in ns],
             "v": [torch.zeros(n, dtype=torch.uint8, device="cuda") for n in ns],
             "m_scale": [ms[a:a + b] for a, b in zip(at, blocks)],
             "v_scale": [vs[a:a + b] for a, b in zip(at, blocks)], "step": 0}
    other = [p.clone() for p in params]
    apart = flarepp.AdamW(other, grads, state_bits=8, **HYPER)
    opt = flarepp.AdamW(params, grads, state_bits=8, state=state, **HYPER)
    for o in (opt, apart):
        o.step()
    for a, b in zip(opt.moments()[0] + opt.moments()[1] + params,
                    apart.moments()[0] + apart.moments()[1] + other):
        assert torch.equal(a, b)


def test_the_optimiser_keeps_its_buffers():
    """A parameter that the caller points elsewhere leaves the optimiser with the old buffer."""
    p, g = torch.ones(1000, device="cuda"), torch.ones(1000, device="cuda")
    opt = flarepp.AdamW([p], [g], **HYPER)
    p.data = torch.zeros(1000, device="cuda")
    g.data = torch.zeros(1000, device="cuda")
    opt.step()
    torch.cuda.synchronize()
    assert not p.any() and not g.any() and (opt.params[0] != 1).all()


def test_no_tensors_and_refusals():
    flarepp.AdamW([], [], **HYPER).step()
    p, g = [torch.ones(8, device="cuda")], [torch.ones(8, device="cuda")]
    with pytest.raises(ValueError):
        flarepp.AdamW(p, [], **HYPER)
    with pytest.raises(ValueError):
        flarepp.AdamW(p, g, state_bits=16)
    with pytest.raises(ValueError):
        flarepp.AdamW(p, [torch.ones(9, device="cuda")])
    with pytest.raises(ValueError):
        flarepp.AdamW(p, [torch.ones(8)])
    with pytest.raises(TypeError):
        flarepp.AdamW([p[0].half()], g)
    with pytest.raises(TypeError):
        flarepp.AdamW(p, g, state_bits=8, state={"m": p, "v": p, "m_scale": p, "v_scale": p})
    for k, bad in (("lr", float("nan")), ("betas", (1.0, 0.9)), ("eps", -1.0),
                   ("weight_decay", float("inf"))):
        with pytest.raises(flarepp.FlareppError) as e:
            flarepp.AdamW(p, g, **dict(HYPER, **{k: bad})).step()
        assert e.value.status == flarepp.ERR_INVALID_ARGUMENT
    with pytest.raises(flarepp.FlareppError) as e:  # a weight that is its own gradient
        flarepp.AdamW(p, p, **HYPER).step()
    assert e.value.status == flarepp.ERR_INVALID_ARGUMENT
