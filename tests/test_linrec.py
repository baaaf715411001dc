"""The gated linear recurrence against its definition in 64 bits: forward, one decoding step, backward,
packed sequences, strides, and what the entry points refuse."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2407_13726_b200 as dastac
from paper_2407_13726_b200 import binding

import _recurrence as rec

GATES = [dastac.GATE_VALUE, dastac.GATE_LOG, dastac.GATE_SIGMOID]
gpu = pytest.mark.gpu


def _inputs(seed, B, T, D, gate, dtype, n=None):
    """g, x, dy on the GPU in `dtype` and as float64 arrays of the same (rounded) values; h0, dh_last."""
    gen = torch.Generator().manual_seed(seed)
    g = torch.randn(B, T, D, generator=gen)
    g = (torch.sigmoid(1.5 + g) * torch.where(torch.rand(B, T, D, generator=gen) < 0.1, -1.0, 1.0) if gate == dastac.GATE_VALUE
         else -torch.exp(1.2 * g - 2.5) if gate == dastac.GATE_LOG else 1.5 + 2.0 * g)
    t = [v.to(dtype) for v in (g, torch.randn(B, T, D, generator=gen), torch.randn(B, T, D, generator=gen))]
    n = B if n is None else n
    s = [torch.randn(n, D, generator=gen) for _ in range(2)]
    return [v.cuda() for v in t], [v.cuda() for v in s], [v.double().numpy() for v in t], [v.double().numpy() for v in s]


def _ws(g):
    n = dastac.linrec_workspace(g)
    # contents are undefined: whatever is there must not matter
    return torch.randint(0, 255, (n,), dtype=torch.uint8, device="cuda") if n else None


def _pass(g, x, dy, gate, h0, dlast, offsets=None):
    """Forward and backward through the public entry points."""
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = (offsets.numel() - 1 if offsets is not None else g.shape[0], g.shape[-1])
    h_last, dh0 = (torch.full(rows, float("nan"), device="cuda") for _ in range(2))
    carries = dastac.linrec_empty_carries(g).fill_(float("nan"))
    h = dastac.linrec_forward(g, x, gate, h0=h0, h_last=h_last, offsets=offsets, carries=carries, workspace=_ws(g), err_word=err)
    dg, dx = dastac.linrec_backward(g, x, dy, gate, carries, h0=h0, dh_last=dlast, dh0=dh0, offsets=offsets, workspace=_ws(g),
                                    err_word=err)
    assert int(err.item()) == 0
    return [v.float().cpu().double().numpy() for v in (h, h_last, dg, dx, dh0)]


def _compare(out, g, x, dy, gate, h0, dlast, offsets, bf16):
    h, h_last, dg, dx, dh0 = out
    rh, rl, eh, el = rec.forward(g, x, gate, h0, offsets)
    rdg, rdx, rd0, eg, ex, e0 = rec.backward(g, x, dy, gate, h0, dlast, offsets)
    rec.check(h, rh.reshape(h.shape), eh.reshape(h.shape), "h", bf16)
    rec.check(h_last, rl, el, "h_last")
    rec.check(dx, rdx.reshape(h.shape), ex.reshape(h.shape), "dx", bf16)
    rec.check(dg, rdg.reshape(h.shape), eg.reshape(h.shape), "dg", bf16)
    rec.check(dh0, rd0, e0, "dh0")


# one step, around a warp's 16 steps and a tile's 128, several tiles, more tiles than one run of sixteen
LENGTHS = [1, 2, 15, 16, 17, 31, 127, 128, 129, 300, 128 * 17 + 5]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("T", LENGTHS)
def test_lengths(T, gate, dtype):
    (g, x, dy), (h0, dl), n, s = _inputs(T, 2, T, 66, gate, dtype)
    _compare(_pass(g, x, dy, gate, h0, dl), *n, gate, *s, None, dtype == torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 2, 31, 32, 33, 63, 64, 65, 128, 130])
def test_channels(D, dtype):
    (g, x, dy), (h0, dl), n, s = _inputs(D, 3, 140, D, dastac.GATE_SIGMOID, dtype)
    _compare(_pass(g, x, dy, dastac.GATE_SIGMOID, h0, dl), *n, dastac.GATE_SIGMOID, *s, None, dtype == torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gate", [dastac.GATE_LOG, dastac.GATE_SIGMOID])
@pytest.mark.parametrize("T,off", [(100, None), (129, None), (300, None), (1024, None), (2500, None), (2500, [0, 200, 2100, 2500])])
def test_slow_decay(T, off, gate, dtype):
    """Gates so close to one that the given states reach every step: decays of a thousandth a step."""
    n = 2 if off is None else len(off) - 1
    (g, x, dy), (h0, dl), num, s = _inputs(T, 2 if off is None else 1, T, 64, gate, dtype, n=n)
    g.copy_(g * 1e-3 if gate == dastac.GATE_LOG else 7.0 + 0.1 * g)
    num[0] = g.double().cpu().numpy()
    offsets = None if off is None else torch.tensor(off, dtype=torch.int64, device="cuda")
    a = (g, x, dy) if off is None else (g[0], x[0], dy[0])
    _compare(_pass(*a, gate, h0, dl, offsets), *num, gate, *s, off, dtype == torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,T", [(40, 1100), (100, 128 * 3 + 1), (60, 128 * 7)])
def test_many_chains_whose_last_run_lacks_tiles(B, T, dtype):
    """Runs of tiles of which several in a row have no tile for some CTAs of a cluster."""
    D = 64 if dtype == torch.bfloat16 else 32
    (g, x, dy), (h0, dl), n, s = _inputs(B, B, T, D, dastac.GATE_LOG, dtype)
    _compare(_pass(g, x, dy, dastac.GATE_LOG, h0, dl), *n, dastac.GATE_LOG, *s, None, dtype == torch.bfloat16)


def _last_runs(g):
    """(CTAs of a cluster, tiles of a chain's last run) as far as the workspace tells: it holds a row of states a run."""
    B, T, D = g.shape
    tiles, row = -(-T // dastac.LINREC_CHUNK), 256 if g.dtype == torch.bfloat16 else 128
    chains = B * -(-D // (64 if g.dtype == torch.bfloat16 else 32))
    runs = (dastac.linrec_workspace(g) - 256) // (chains * row)
    return [(c, tiles - (runs - 1) * c) for c in range(1, 9) if -(-tiles // c) == runs]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("B,groups,tiles", [(14, 7, 13), (6, 7, 26), (4, 5, 26)])
def test_last_runs_that_lack_tiles_for_some_of_a_cluster(B, groups, tiles, dtype):
    """Chains whose last run has tiles for several CTAs of a cluster, which send one another their maps, and none for the
    others: many such runs in a row, a few, and one.  Alone and with three calls at once, which leaves each cluster
    more of them; the same bits every time."""
    D, gate = groups * (64 if dtype == torch.bfloat16 else 32), dastac.GATE_LOG
    (g, x, dy), (h0, dl), n, s = _inputs(B, B, tiles * 128 - 3, D, gate, dtype)
    layouts = _last_runs(g)
    assert layouts and all(2 <= left < ctas for ctas, left in layouts)
    first = _pass(g, x, dy, gate, h0, dl)
    _compare(first, *n, gate, *s, None, dtype == torch.bfloat16)
    for _ in range(8):
        for a, b in zip(first, _pass(g, x, dy, gate, h0, dl)):
            assert np.array_equal(a, b)
    streams = [torch.cuda.Stream() for _ in range(3)]
    works = [_ws(g) for _ in streams]
    torch.cuda.synchronize()
    for _ in range(8):
        outs = []
        for stream, ws in zip(streams, works):
            with torch.cuda.stream(stream):
                outs.append(dastac.linrec_forward(g, x, gate, h0=h0, workspace=ws))
        torch.cuda.synchronize()
        for h in outs:
            assert np.array_equal(first[0], h.float().cpu().double().numpy())


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("packed", [False, True])
def test_clusters_that_end_with_a_run_without_a_tile(packed, dtype):
    """Fewer chains than clusters, a last run that is short: for most CTAs a tile, no tile, and the end follow one another."""
    D, T, gate = 20 * (64 if dtype == torch.bfloat16 else 32), 128 * 8 + 40, dastac.GATE_SIGMOID
    off = [0, 300, 301, T - 2] if packed else None
    (g, x, dy), (h0, dl), n, s = _inputs(41, 1, T, D, gate, dtype, n=3 if packed else 1)
    layouts = _last_runs(g)
    assert layouts and all(left < ctas for ctas, left in layouts)
    offsets = None if off is None else torch.tensor(off, device="cuda")
    a = (g[0], x[0], dy[0]) if packed else (g, x, dy)
    first = _pass(*a, gate, h0, dl, offsets)
    _compare(first, *n, gate, *s, off, dtype == torch.bfloat16)
    for _ in range(30):
        for p, q in zip(first, _pass(*a, gate, h0, dl, offsets)):
            assert np.array_equal(p, q)


@gpu
@pytest.mark.parametrize("T", [1, 7, 200])
def test_without_states(T):
    (g, x, dy), _, n, _ = _inputs(5, 2, T, 40, dastac.GATE_LOG, torch.float32)
    carries = dastac.linrec_empty_carries(g)
    h = dastac.linrec_forward(g, x, dastac.GATE_LOG, carries=carries, workspace=_ws(g))
    dg, dx = dastac.linrec_backward(g, x, dy, dastac.GATE_LOG, carries, workspace=_ws(g))
    rh, _, eh, _ = rec.forward(n[0], n[1], dastac.GATE_LOG)
    rdg, rdx, _, eg, ex, _ = rec.backward(*n, dastac.GATE_LOG)
    rec.check(h.cpu(), rh, eh, "h")
    rec.check(dg.cpu(), rdg, eg, "dg")
    rec.check(dx.cpu(), rdx, ex, "dx")


PACKED = [
    (50, [0, 50]),
    (50, [0, 0, 1, 1, 1, 17, 50, 50]),
    (700, [0, 127, 128, 129, 129, 257, 258, 640, 700]),
    (700, [3, 20, 20, 300, 690]),                                  # steps before, between nothing, and behind belong to no sequence
    (40, list(range(41))),                                          # every step a sequence of its own
    (128 * 40, [0, 5, 128 * 16, 128 * 16 + 1, 128 * 39, 128 * 40]),  # boundaries at and beside a run's end
    (128 * 36, [0, 128 * 36]),
    (16, [0]),                                                      # no sequence at all
    (33, [33, 33]),
]


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("case", range(len(PACKED)))
def test_packed(case, gate, dtype):
    T, off = PACKED[case]
    (g, x, dy), (h0, dl), n, s = _inputs(case, 1, T, 67, gate, dtype, n=len(off) - 1)
    outside = np.ones(T, dtype=bool)
    for a, b in zip(off, off[1:]):
        outside[a:b] = False
    for v in (g, x, dy):   # what belongs to no sequence is not read into any result
        v[0, torch.from_numpy(outside).cuda()] = float("nan")
    offsets = torch.tensor(off, dtype=torch.int64, device="cuda")
    _compare(_pass(g[0], x[0], dy[0], gate, h0, dl, offsets), *n, gate, *s, off, dtype == torch.bfloat16)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_is_not_finite_stays_in_its_sequence(bad, dtype):
    off = [0, 20, 130, 131, 128 * 17 + 3, 128 * 17 + 90, 2400]
    gate, hurt = dastac.GATE_SIGMOID, (1, 3)
    (g, x, dy), (h0, dl), n, s = _inputs(9, 1, 2400, 40, gate, dtype, n=len(off) - 1)
    clean = _pass(g[0], x[0], dy[0], gate, h0, dl, torch.tensor(off, device="cuda"))
    for q in hurt:
        for v in (x, dy):
            v[0, off[q]:off[q + 1]] = bad
        g[0, off[q]:off[q + 1]] = bad
        h0[q], dl[q] = bad, bad
    dirty = _pass(g[0], x[0], dy[0], gate, h0, dl, torch.tensor(off, device="cuda"))
    for a, b in zip(clean, dirty):
        for q in range(len(off) - 1):
            if q not in hurt:
                rows = slice(q, q + 1) if a.shape[0] == len(off) - 1 else slice(off[q], off[q + 1])
                assert np.array_equal(a[rows], b[rows])


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("layout", ["time_first", "odd_base", "odd_pitch", "shared_gate"])
@pytest.mark.parametrize("T", [1, 9, 150])
def test_strides(T, layout, dtype):
    B, D, gate = 3, 48, dastac.GATE_SIGMOID
    (g, x, dy), (h0, dl), n, s = _inputs(17, B, T, D, gate, dtype)

    def place(v):
        if layout == "time_first":
            return v.transpose(0, 1).contiguous().transpose(0, 1)
        if layout == "odd_base":
            big = torch.full((v.numel() + 1,), float("nan"), dtype=dtype, device="cuda")
            big[1:] = v.reshape(-1)
            return big[1:].view(B, T, D)
        big = torch.full((B, T, D + 3), float("nan"), dtype=dtype, device="cuda")
        big[..., 1:D + 1] = v
        return big[..., 1:D + 1]

    if layout == "shared_gate":   # one row of gates for every sequence of the batch
        g = g[:1].expand(B, T, D)
        n[0] = np.repeat(n[0][:1], B, 0)
    else:
        g, x, dy = place(g), place(x), place(dy)
    wide = torch.full((B, 2 * D), float("nan"), device="cuda")
    wide[:, :D], wide[:, D:] = h0, dl
    h0, dl = wide[:, :D], wide[:, D:]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = [place(torch.zeros(B, T, D, dtype=dtype, device="cuda")) for _ in range(3)]
    last = torch.full((2, B, D), float("nan"), device="cuda")
    carries = dastac.linrec_empty_carries(g)
    dastac.linrec_forward(g, x, gate, out=outs[0], h0=h0, h_last=last[0], carries=carries, workspace=_ws(g), err_word=err)
    dastac.linrec_backward(g, x, dy, gate, carries, h0=h0, dh_last=dl, dg=outs[1], dx=outs[2], dh0=last[1], workspace=_ws(g), err_word=err)
    assert int(err.item()) == 0
    out = [v.float().cpu().double().numpy() for v in (outs[0], last[0], outs[1], outs[2], last[1])]
    _compare(out, *n, gate, *s, None, dtype == torch.bfloat16)


@gpu
@pytest.mark.parametrize("steps", [1, 16, 100, 400])
def test_state_updated_in_place_and_parts_join(steps):
    """A sequence in parts, the state carried in place, on a stream of its own: the same as the whole."""
    (g, x, _), (h0, _), n, s = _inputs(23, 2, 3 * steps, 70, dastac.GATE_LOG, torch.bfloat16)
    state = h0.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        parts = [dastac.linrec_forward(g[:, k:k + steps], x[:, k:k + steps], dastac.GATE_LOG, h0=state, h_last=state,
                                       workspace=_ws(g[:, :steps])) for k in range(0, 3 * steps, steps)]
        out = torch.cat(parts, 1)
    stream.synchronize()
    rh, rl, eh, el = rec.forward(*n[:2], dastac.GATE_LOG, s[0])
    rec.check(out.float().cpu(), rh, 2 * eh, "h", True)
    rec.check(state.cpu(), rl, 2 * el, "state")


@gpu
def test_packed_state_in_place():
    off = [0, 4, 4, 9, 300, 310]
    (g, x, _), (h0, _), n, s = _inputs(29, 1, 310, 34, dastac.GATE_SIGMOID, torch.float32, n=5)
    state = h0.clone()
    dastac.linrec_forward(g[0], x[0], dastac.GATE_SIGMOID, h0=state, h_last=state, offsets=torch.tensor(off, device="cuda"),
                          workspace=_ws(g[0]))
    _, rl, _, el = rec.forward(*n[:2], dastac.GATE_SIGMOID, s[0], off)
    rec.check(state.cpu(), rl, el, "state")


@gpu
def test_same_bits_every_time():
    (g, x, dy), (h0, dl), _, _ = _inputs(31, 4, 128 * 35, 96, dastac.GATE_SIGMOID, torch.float32)
    first = _pass(g, x, dy, dastac.GATE_SIGMOID, h0, dl)
    for _ in range(5):
        for a, b in zip(first, _pass(g, x, dy, dastac.GATE_SIGMOID, h0, dl)):
            assert np.array_equal(a, b)


@gpu
def test_extreme_gates():
    """Gates of exactly zero and one, and logits at which 1 - s(g) rounds to 0 in fp32."""
    T, D = 200, 8
    x = torch.ones(1, T, D, device="cuda")
    g = torch.zeros(1, T, D, device="cuda")
    g[..., 0], g[..., 1] = 0.0, 1.0
    h = dastac.linrec_forward(g, x, dastac.GATE_VALUE, workspace=_ws(g)).cpu()
    assert (h[0, :, 0] == 1).all() and torch.equal(h[0, :, 1], torch.arange(1, T + 1).float())
    g = torch.full((1, T, D), 200.0, device="cuda")
    g[..., 1], g[..., 2], g[..., 3] = -200.0, float("inf"), -float("inf")
    h0 = torch.full((1, D), 3.0, device="cuda")
    h = dastac.linrec_forward(g, x, dastac.GATE_SIGMOID, h0=h0, workspace=_ws(g)).cpu()
    assert (h[0, :, [0, 2]] == 3).all() and (h[0, :, [1, 3]] == 1).all()
    g = torch.full((1, T, D), 20.0, device="cuda")   # shut = 2e-9: lost if it were 1 - s(g)
    h = dastac.linrec_forward(g, x, dastac.GATE_SIGMOID, workspace=_ws(g)).cpu().double().numpy()
    rh, _, eh, _ = rec.forward(np.full((1, T, D), 20.0), np.ones((1, T, D)), dastac.GATE_SIGMOID)
    rec.check(h, rh, eh, "h")


@gpu
def test_large_gates_with_a_zero_state():
    """Products of gates that pass the fp32 range while the state is still zero."""
    g = torch.full((1, 256, 2), 4.0, device="cuda")
    x = torch.zeros(1, 256, 2, device="cuda")
    x[0, 250] = 1.0
    h = dastac.linrec_forward(g, x, dastac.GATE_VALUE, workspace=_ws(g)).cpu()
    assert (h[0, :250] == 0).all() and torch.equal(h[0, 250:, 0], 4.0 ** torch.arange(6.0))


@gpu
@pytest.mark.parametrize("gate", GATES)
def test_gradients_against_differences(gate):
    """<gradient, direction> against a central difference of the 64-bit forward pass."""
    B, T, D = 2, 150, 5
    (g, x, dy), (h0, dl), n, s = _inputs(37, B, T, D, gate, torch.float32)
    _, _, dg, dx, dh0 = _pass(g, x, dy, gate, h0, dl)

    def loss(gg, xx, hh):
        h, last, _, _ = rec.forward(gg, xx, gate, hh)
        return (h * n[2]).sum() + (last * s[1]).sum()

    rng = np.random.default_rng(gate)
    step = 1e-5
    for grad, at in ((dg, 0), (dx, 1), (dh0, 2)):
        v = rng.standard_normal(grad.shape)
        args = [n[0], n[1], s[0]]
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + step * v, args[at] - step * v
        want = (loss(*up) - loss(*down)) / (2 * step)
        # the sum of |terms| bounds the fp32 part, the difference itself is good to step^2 of the third derivative
        assert abs((grad * v).sum() - want) <= 1e-5 * np.abs(grad * v).sum()


@gpu
def test_empty_extents():
    for shape in [(0, 5, 4), (2, 0, 4), (2, 5, 0)]:
        g = torch.zeros(shape, device="cuda")
        h0 = torch.ones(shape[0], shape[2], device="cuda")
        last = torch.zeros_like(h0)
        assert dastac.linrec_forward(g, g, dastac.GATE_VALUE, h0=h0, h_last=last, workspace=_ws(g)).shape == shape
        if shape[1] == 0:
            assert torch.equal(last, h0)
            dastac.linrec_forward(g, g, dastac.GATE_VALUE, h_last=last)
            assert (last == 0).all()
            carries = dastac.linrec_empty_carries(g)
            dastac.linrec_backward(g, g, g, dastac.GATE_VALUE, carries, dh_last=h0, dh0=last)
            assert torch.equal(last, h0)


@gpu
def test_no_steps_and_one_row_of_any_pitch():
    """A (1, D) tensor made from a column has a pitch of 1, which says nothing for a single row."""
    D = 12
    row = lambda v: torch.full((D, 1), v, device="cuda").t()  # noqa: E731
    assert row(0.0).stride() == (1, 1)
    for packed in (False, True):
        g = torch.zeros((0, D) if packed else (1, 0, D), device="cuda")
        offsets = torch.zeros(2, dtype=torch.int64, device="cuda") if packed else None
        last = row(2.0)
        dastac.linrec_forward(g, g, dastac.GATE_VALUE, h0=row(3.0), h_last=last, offsets=offsets)
        assert (last == 3).all()
        dastac.linrec_forward(g, g, dastac.GATE_VALUE, h_last=last, offsets=offsets)
        assert (last == 0).all()
        dastac.linrec_backward(g, g, g, dastac.GATE_VALUE, dastac.linrec_empty_carries(g), dh_last=row(4.0), dh0=last, offsets=offsets)
        assert (last == 4).all()


# ---- refusals (no GPU) -------------------------------------------------------------------------------------------

def _shape(**k):
    v = dict(dtype=0, gate=0, batch=2, steps=300, channels=40, offsets=None, sequences=0)
    v.update(k)
    return binding._LinrecShape(*[v[n] for n in ("dtype", "gate", "batch", "steps", "channels", "offsets", "sequences")])


def _forward(shape, data=0x1000, stride=40, h0=None, ld=40, ws=None, nbytes=0, out=None, step=40):
    seq = binding._Sequence(data, stride * 300, stride)
    o = binding._Sequence(data, 40 * 300, step) if out is None else out
    return binding._lib.dastac_linrec_forward(shape, seq, seq, h0, ld, o, None, 0, None, ws, nbytes, None, None)


def _backward(shape, data=0x1000, carries=0x1000, ws=None, nbytes=0):
    seq = binding._Sequence(data, 40 * 300, 40)
    return binding._lib.dastac_linrec_backward(shape, seq, seq, seq, None, 0, carries, None, 0, seq, seq, None, 0, ws, nbytes, None, None)


def test_refusals_do_not_launch():
    before = dastac.launch_count()
    need = ctypes.c_size_t()
    assert binding._lib.dastac_linrec_workspace(_shape(), ctypes.byref(need)) == 0 and need.value > 0
    assert binding._lib.dastac_linrec_workspace(_shape(steps=128), ctypes.byref(need)) == 0 and need.value == 0
    assert binding._lib.dastac_linrec_workspace(_shape(), None) == 1
    assert binding._lib.dastac_linrec_workspace(None, ctypes.byref(need)) == 1
    for bad, status in [(dict(batch=-1), 1), (dict(steps=-1), 1), (dict(channels=-1), 1), (dict(gate=3), 1), (dict(gate=-1), 1),
                        (dict(dtype=2), 3), (dict(sequences=3), 1), (dict(offsets=8, sequences=-1), 1), (dict(offsets=8, sequences=3), 4),
                        (dict(steps=2 ** 30 + 1), 6), (dict(steps=2 ** 30, channels=2 ** 30, batch=2 ** 30), 6)]:
        assert binding._lib.dastac_linrec_workspace(_shape(**bad), ctypes.byref(need)) == status, bad
        assert _forward(_shape(**bad)) == status and _backward(_shape(**bad)) == status, bad
    for call in (_forward, _backward):
        assert call(_shape(), data=0) == 1                               # NULL tensor
        assert call(_shape(), data=0x1002) == 5                          # not a whole element
        assert call(_shape()) == 7                                       # no workspace
        assert call(_shape(), ws=0x1000, nbytes=255) == 7                # too small
        assert call(_shape(), ws=0x1010, nbytes=1 << 24) == 7            # misaligned
    assert _backward(_shape(), carries=None) == 1
    assert _forward(_shape(), stride=-1) == 1
    assert _forward(_shape(), step=39) == 4                              # rows of the output overlap
    assert _forward(_shape(), h0=0x1000, ld=39) == 4
    assert _forward(_shape(), h0=0x1002, ld=40) == 5
    assert dastac.launch_count() == before


def test_binding_checks_shapes():
    g = torch.zeros(2, 3, 4)
    with pytest.raises(AssertionError):
        dastac.linrec_forward(g, g, dastac.GATE_VALUE)     # not on a GPU: there is no other code path
    with pytest.raises(TypeError):
        dastac.linrec_workspace(g.double())
