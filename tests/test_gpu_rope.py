"""rotate against float64 on the host, element by element."""
import numpy as np
import pytest

from cache_model import bits, floats
from chunk_model import frequencies, turn, turn_tolerance

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2502_20766_amd as fpx
    fpx.lib()
    return fpx


def _dev(x):
    return torch.from_numpy(x.view(np.int16)).cuda().view(torch.bfloat16)


def _bits(x):
    return x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def _near(got, want, mass, what=""):
    got = floats(got)
    fine = np.isfinite(want)
    assert np.array_equal(fine, np.isfinite(got)), f"{what}: other finite places"
    err, tol = np.abs(got - want)[fine], turn_tolerance(want, mass)[fine]
    assert np.all(err <= tol), f"{what}: {(err / tol).max():.2f} of the bound"


def check(T, hq, hkv, d, layout="half", rotary=None, norm=None, positions=None, seed=0, scale=1.5,
          x=None, **freq):
    import paper_2502_20766_amd as fpx
    rng = np.random.default_rng(seed)
    rotary = d if rotary is None else rotary
    if x is None:
        x = bits(rng.standard_normal((T, hq + 2 * hkv, d)) * scale)
    pos = rng.integers(0, 100000, T) if positions is None else np.asarray(positions)
    rope, f, amplitude = None, None, 1.0
    if rotary:
        amplitude = freq.pop("amplitude", 1.0)
        rope = fpx.Rope(rotary, layout=layout, amplitude=amplitude, **freq)
        f = frequencies(rotary, **freq)
    hn, weights, eps = None, [None, None], None
    if norm:
        eps = 1e-6
        w = 1 + 0.3 * rng.standard_normal((2, d))
        if norm == "bf16":
            w = bits(w)
            weights = list(floats(w))
            hn = fpx.HeadNorm(_dev(w[0]), _dev(w[1]), eps)
        elif norm == "f32":
            weights = list(w.astype(np.float32).astype(np.float64))
            hn = fpx.HeadNorm(*torch.from_numpy(w.astype(np.float32)).cuda().unbind(0), eps=eps)
        elif norm == "keys":
            w = bits(w)
            weights = [None, floats(w)[1]]
            hn = fpx.HeadNorm(None, _dev(w[1]), eps)
        else:
            hn = fpx.HeadNorm(eps=eps)
    t = _dev(x)
    at = torch.from_numpy(pos.astype(np.int32)).cuda()
    q, k = fpx.rotate(t[:, :hq], t[:, hq:hq + hkv] if hkv else None, at, rope, hn)
    assert q.is_contiguous() and np.array_equal(_bits(t), x)
    xf = floats(x)
    for got, rows, w, name in ((q, xf[:, :hq], weights[0], "q"),
                               (k, xf[:, hq:hq + hkv], weights[1], "k")):
        if got is None:
            continue
        _near(_bits(got), *turn(rows, pos, f, layout, amplitude, w, eps), name)
    return q, k


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (7, 1, 128), (28, 4, 128), (2, 2, 64), (64, 16, 64),
                                      (1, 0, 64), (1, 0, 128), (17, 3, 64)])
@pytest.mark.parametrize("T", [1, 2, 37, 1025])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_heads(hq, hkv, d, T, layout):
    check(T, hq, hkv, d, layout, seed=T + hq)


@pytest.mark.parametrize("d,rotary", [(128, 16), (128, 48), (128, 64), (128, 112), (64, 16), (64, 32),
                                      (64, 48), (128, 0), (64, 0)])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [None, "bf16"])
def test_part_of_the_head(d, rotary, layout, norm):
    check(19, 5, 2, d, layout, rotary, norm, seed=rotary)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("norm", ["bf16", "f32", "keys", "plain"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_norms(d, norm, layout):
    check(23, 6, 3, d, layout, norm=norm, seed=d)
    check(23, 6, 3, d, layout, norm=norm, seed=d, scale=1e-4)     # eps counts
    check(23, 6, 3, d, layout, norm=norm, seed=d, scale=1e15)


@pytest.mark.parametrize("freq", [dict(base=500000.0), dict(base=1.0), dict(scaling="linear", factor=4.0),
                                  dict(scaling="base", factor=8.0, base=1e6),
                                  dict(scaling="parts", factor=8.0, original_len=8192, base=5e5,
                                       low_turns=1.0, high_turns=4.0),
                                  dict(scaling="parts", factor=16.0, original_len=4096,
                                       amplitude=1.2773),
                                  dict(amplitude=0.5)])
@pytest.mark.parametrize("rotary", [128, 32])
def test_frequencies(freq, rotary):
    check(29, 4, 1, 128, rotary=rotary, **freq)


def test_far_positions():
    """Positions at the ends of 32 bits: the angle loses nothing."""
    pos = [0, 1, -1, 2 ** 20 + 1, 2 ** 24 + 1, 2 ** 26 - 1, 2 ** 31 - 1, -2 ** 31, -2 ** 31 + 1, 1 << 30]
    check(10, 3, 1, 128, positions=pos, base=10000.0)
    check(10, 3, 1, 64, "interleaved", positions=pos, base=500000.0, scaling="linear", factor=3.0)


def test_frequencies_of_the_caller():
    import paper_2502_20766_amd as fpx
    f = np.array([1.0, 3.7, 0.0, -0.25, 1e5, 2.0 ** -40, 1e-3, 0.5])
    x = bits(np.random.default_rng(0).standard_normal((9, 3, 64)))
    pos = np.arange(9) * 1000 - 3000
    q, _ = fpx.rotate(_dev(x), None, torch.from_numpy(pos.astype(np.int32)).cuda(),
                      fpx.Rope(16, inv_freq=f))
    _near(_bits(q), *turn(floats(x), pos, f))


def test_position_zero_changes_nothing():
    import paper_2502_20766_amd as fpx
    x = bits(np.random.default_rng(1).standard_normal((5, 4, 128)))
    q, _ = fpx.rotate(_dev(x), None, torch.zeros(5, dtype=torch.int32, device="cuda"), fpx.Rope(128))
    assert np.array_equal(_bits(q), x)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [None, "bf16"])
def test_in_place_and_slices(layout, norm):
    """Outputs that are the inputs, outputs within a wider tensor; what lies around them stays."""
    import paper_2502_20766_amd as fpx
    rng = np.random.default_rng(3)
    hq, hkv, d = 12, 2, 128
    x = bits(rng.standard_normal((301, hq + 2 * hkv, d)))
    pos = torch.arange(301, dtype=torch.int32, device="cuda")
    rope = fpx.Rope(64, layout=layout)
    hn = None if norm is None else fpx.HeadNorm(_dev(bits(rng.standard_normal(d))),
                                                _dev(bits(rng.standard_normal(d))))
    t = _dev(x)
    q, k = fpx.rotate(t[:, :hq], t[:, hq:hq + hkv], pos, rope, hn)
    wide = _dev(bits(rng.standard_normal((301, hq + hkv + 1, d))))
    before = _bits(wide)
    fpx.rotate(t[:, :hq], t[:, hq:hq + hkv], pos, rope, hn, q_out=wide[:, :hq], k_out=wide[:, hq + 1:])
    assert np.array_equal(_bits(wide[:, :hq]), _bits(q)) and np.array_equal(_bits(wide[:, hq + 1:]), _bits(k))
    assert np.array_equal(_bits(wide[:, hq]), before[:, hq])
    a, b = fpx.rotate(t[:, :hq], t[:, hq:hq + hkv], pos, rope, hn, q_out=t[:, :hq],
                      k_out=t[:, hq:hq + hkv])
    assert a.data_ptr() == t.data_ptr()
    assert np.array_equal(_bits(t[:, :hq]), _bits(q)) and np.array_equal(_bits(t[:, hq:hq + hkv]), _bits(k))
    assert np.array_equal(_bits(t[:, hq + hkv:]), x[:, hq + hkv:])


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [None, "bf16"])
def test_infinities_stay_in_their_head(layout, norm):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4, 9, 128))
    clean = check(4, 5, 2, 128, layout, 64, norm, positions=[3, 4, 5, 6], x=bits(x))
    x[1, 2, 7], x[2, 5, 100], x[3, 6, 63] = np.inf, np.nan, -np.inf      # one beyond the rotated part
    odd = check(4, 5, 2, 128, layout, 64, norm, positions=[3, 4, 5, 6], x=bits(x))
    for a, b, touched in ((clean[0], odd[0], [(1, 2)]), (clean[1], odd[1], [(2, 0), (3, 1)])):
        same = np.ones(a.shape[:2], bool)
        for i in touched:
            same[i] = False
        assert np.array_equal(_bits(a)[same], _bits(b)[same])


def test_an_empty_call():
    import paper_2502_20766_amd as fpx
    x = torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    q, k = fpx.rotate(x, x[:, :2], torch.empty(0, dtype=torch.int32, device="cuda"), fpx.Rope(64))
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)


def test_refusals():
    import paper_2502_20766_amd as fpx
    x = torch.zeros(4, 6, 128, dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros(4, dtype=torch.int32, device="cuda")
    rope = fpx.Rope(128)
    for call in (lambda: fpx.rotate(x.float(), None, pos, rope),
                 lambda: fpx.rotate(x, None, pos.long(), rope),
                 lambda: fpx.rotate(x, None, pos[:3], rope),
                 lambda: fpx.rotate(x, None, None, rope),
                 lambda: fpx.rotate(x, None, pos.cpu(), rope),
                 lambda: fpx.rotate(x.transpose(0, 1), None, pos, rope),
                 lambda: fpx.rotate(x, x[:3], pos, rope),
                 lambda: fpx.rotate(x, x[..., :64], pos, rope),
                 lambda: fpx.rotate(x, None, pos, rope, q_out=x[:, :3]),
                 lambda: fpx.rotate(x, None, pos, rope, k_out=x),
                 lambda: fpx.rotate(None, None, pos, rope),
                 lambda: fpx.rotate(x, None, pos, rope, fpx.HeadNorm(x[0, 0, :64])),
                 lambda: fpx.HeadNorm(x[0, 0], x[0, 0].float()),
                 lambda: fpx.HeadNorm(x[0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(fpx.FlexPrefillError):       # 96 elements a head
        fpx.rotate(x[..., :96].contiguous(), None, pos, fpx.Rope(64))
    with pytest.raises(fpx.FlexPrefillError):       # more rotated than there are
        fpx.rotate(x[..., :64].contiguous(), None, pos, rope)
    with pytest.raises(fpx.FlexPrefillError):       # an output shifted against its input
        fpx.rotate(x[:, :3], None, pos, rope, q_out=torch.empty(4 * 6 * 128 + 4, dtype=torch.bfloat16,
                                                                device="cuda")[4:].view(4, 6, 128)[:, :3])


@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (1, 1, 128), (2, 1, 64), (3, 0, 128), (3, 1, 128),
                                      (5, 2, 64), (7, 0, 64), (4, 4, 64), (5, 3, 128), (15, 0, 64)])
@pytest.mark.parametrize("T", [1, 3, 16, 1023, 1500])
def test_few_heads_of_many_tokens(hq, hkv, d, T):
    """Heads of several tokens side by side, the last ones of which are not there."""
    check(T, hq, hkv, d, norm="bf16", seed=T + hq)
    x = bits(np.random.default_rng(T).standard_normal((T, hq, d)))
    t, at = _dev(x), torch.arange(T, dtype=torch.int32, device="cuda")
    import paper_2502_20766_amd as fpx
    rope = fpx.Rope(d, layout="interleaved")
    around = torch.full((T + 2, hq, d), 3.0, dtype=torch.bfloat16, device="cuda")
    want, _ = fpx.rotate(t, None, at, rope, q_out=around[1:-1])
    assert bool((around[0] == 3).all()) and bool((around[-1] == 3).all())
    fpx.rotate(t, None, at, rope, q_out=t)
    assert torch.equal(t, want)
