"""Verification of drafted tokens against the fp64 oracle. Tokens and counts are equal; tolerances of the numbers, with
u = 2^-24: a row's sum of exp(z - m) is off by at most tol_s = (V / 512 + 64 + 2 * 24 + 8) u relative (chains of a lane's
terms and trees; each term by the roundings of z - m, of its product with log2 e, and of ex2), so
    logp   tol_s + u |logp| + 2 u |log-sum|
    accept twice that of the two log-probabilities, relative, and 4 u."""
import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import dev_f32, dev_i32, host_f64

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
INF, NAN = float("inf"), float("nan")
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


def rows_of(x, dtype, ld, shift):
    n, v = x.shape
    buf = torch.full((n * ld + shift + 8,), NAN, dtype=dtype, device="cuda")
    out = buf[shift:shift + n * ld].view(n, ld)
    out[:, :v] = torch.from_numpy(x).cuda().to(dtype)
    return out[:, :v]


def make(seed, S, D, V, dtype, mode="draft", mask=None, ld=None, shift=0, n_draft="ragged", near=0.5):
    rng = np.random.default_rng(seed)
    z = rng.normal(0, 2.0, (S, D + 1, V)) * 10 ** rng.uniform(-0.5, 0.4, (S, 1, 1))
    w = z[:, :D] + rng.normal(0, near, (S, D, V))
    if mask is not None:
        low = -INF if mask == "inf" else float(torch.finfo(TYPES[dtype]).min)
        z[rng.random(z.shape) < 0.6] = low
        w[rng.random(w.shape) < 0.6] = low
    c = {"S": S, "D": D, "V": V, "mode": mode}
    c["z"] = rows_of(z.reshape(-1, V), TYPES[dtype], ld or V, shift)
    c["w"] = rows_of(w.reshape(-1, V), TYPES[dtype], ld or V, shift) if mode == "draft" and D else None
    zs = host_f64(c["z"].contiguous()).reshape(S, D + 1, V)
    ws = host_f64(c["w"].contiguous()).reshape(S, D, V) if c["w"] is not None else zs[:, :D]
    best = (ws + rng.gumbel(size=ws.shape)).argmax(-1) if mode != "greedy" else ws.argmax(-1)
    c["ids"] = np.where(rng.random((S, D)) < 0.85, best, rng.integers(0, V, (S, D)))
    ragged = isinstance(n_draft, str)
    c["n"] = rng.integers(0, D + 1, S) if ragged else n_draft
    if ragged and S > 1:
        c["n"][0], c["n"][-1] = D, 0
    c["u"] = rng.random((S, D)).astype(np.float32) if mode != "greedy" else None
    c["g"] = rng.gumbel(size=(S, V)).astype(np.float32) if mode != "greedy" else None
    return c


def run(c, **kw):
    S, D = c["S"], c["D"]
    o = {"tokens": torch.full((S, D + 1), -7, dtype=torch.int32, device="cuda"),
         "accepted": torch.full((S,), -7, dtype=torch.int32, device="cuda"),
         "logp": torch.full((S, D + 1), NAN, device="cuda"), "accept": torch.full((S, D), NAN, device="cuda")}
    opt = lambda x, f: None if x is None else f(x)  # noqa: E731
    H.hydra_verify_drafts(c["z"], c["w"], dev_i32(c["ids"]), opt(c["n"], dev_i32), opt(c["u"], dev_f32), opt(c["g"], dev_f32),
                          S, D, **{**o, **kw})
    return o


def check(c, o):
    S, D, V = c["S"], c["D"], c["V"]
    z = host_f64(c["z"].contiguous())
    w = None if c["w"] is None else host_f64(c["w"].contiguous())
    ref = O.verify_drafts(z, w, c["ids"], c["n"], c["u"], c["g"], S, D)
    for k in ("accepted", "tokens"):
        np.testing.assert_array_equal(o[k].cpu().numpy(), ref[k], err_msg=k)
    tol_s = (V / 512 + 64 + 48 + 8) * U
    got = o["logp"].double().cpu().numpy()
    fine = np.isfinite(ref["logp"])
    np.testing.assert_array_equal(got[~fine], ref["logp"][~fine])
    assert (np.abs(got[fine] - ref["logp"][fine]) <= tol_s + U * np.abs(ref["logp"][fine]) + 2 * U * 20).all()
    got = o["accept"].double().cpu().numpy()
    assert (np.abs(got - ref["accept"]) <= 2 * (tol_s + 60 * U) * ref["accept"] + 4 * U * ref["accept"]).all()
    return ref


@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
@pytest.mark.parametrize("dtype,mask", [("f32", None), ("bf16", None), ("f32", "inf"), ("bf16", "lowest"), ("f32", "lowest"),
                                        ("bf16", "inf")])
@pytest.mark.parametrize("S,D,V", [(1, 1, 1), (1, 4, 5), (7, 3, 1001), (40, 5, 513), (3, 8, 32000), (300, 2, 260)])
def test_verify(S, D, V, dtype, mask, mode):
    c = make(S * 100 + D * 10 + V % 97, S, D, V, dtype, mode, mask)
    check(c, run(c))


@pytest.mark.parametrize("dtype,ld,shift", [("f32", 1003, 1), ("bf16", 1011, 3), ("bf16", 1008, 8), ("f32", 1004, 0)])
def test_strides_and_alignments(dtype, ld, shift):
    c = make(5, 9, 4, 1001, dtype, "draft", None, ld, shift)
    check(c, run(c))


def test_many_drafts_none_and_no_lengths():
    check(c := make(6, 5, 32, 700, "bf16", "draft", near=0.05, n_draft=None), run(c))
    check(c := make(7, 6, 0, 700, "f32", "given"), run(c))
    check(c := make(8, 6, 0, 700, "f32", "greedy"), run(c))
    c = make(9, 4, 3, 2000, "f32", "draft")
    o = run(c, logp=None, accept=None)
    assert torch.equal(o["tokens"], run(c)["tokens"])


def test_draft_equal_to_the_target_is_kept():
    c = make(10, 20, 6, 4000, "f32", "draft", near=0.0)
    ids = host_f64(c["w"].contiguous()).reshape(20, 6, 4000).argmax(-1)
    c["ids"], c["n"] = ids, None
    o = run(c)
    check(c, o)
    assert (o["accepted"] == 6).all() and (o["accept"] == 1).all()


def test_rows_that_leave_nothing():
    """A target row of nothing but -inf, a draft row of nothing but -inf, a target that has all its mass on the
    refused token, a draft token that neither can give."""
    V, D = 50, 1
    z = np.random.default_rng(1).normal(size=(8, V))
    w = np.random.default_rng(2).normal(size=(4, V))
    z[0] = -INF                 # sequence 0: nothing to keep, nothing to draw
    w[1] = -INF                 # sequence 1: kept, as only the draft model calls it impossible
    z[4] = -INF
    z[4, 7] = 1.0               # sequence 2: certain of 7, the draft is 7 as well
    z[6, 3] = w[3, 3] = -INF    # sequence 3
    c = {"S": 4, "D": D, "V": V, "n": None, "ids": np.array([[5], [6], [7], [3]]),
         "u": np.array([[0.0], [0.999], [0.5], [0.0]], dtype=np.float32),
         "g": np.random.default_rng(3).gumbel(size=(4, V)).astype(np.float32)}
    for dtype in (torch.float32, torch.bfloat16):
        c["z"], c["w"] = rows_of(z, dtype, V, 0), rows_of(w, dtype, V, 0)
        o = run(c)
        check(c, o)
        assert o["accepted"].tolist() == [0, 1, 1, 0] and o["tokens"][0, 0] == 0 and o["logp"][0, 0] == -INF
        o = run(dict(c, w=None, u=np.array([[0.0], [0.999], [1.0], [0.0]], dtype=np.float32)))
        assert o["tokens"][2].tolist() == [7, -1]  # refused, but nothing else is left


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,ld,shift", [(1, 1, 0), (2, 3, 1), (6, 11, 8), (23, 25, 3), (1003, 1007, 5)])
def test_rows_of_nothing_give_token_0_wherever_they_start(V, ld, shift, dtype):
    """Greedy and drawn; the first logits and the last ones of a row lie outside its whole vectors."""
    S = 9
    for mode in ("greedy", "given"):
        c = make(50, S, 1, V, dtype, mode, ld=ld, shift=shift, n_draft=None)
        c["z"][:] = -INF
        o = run(c)
        check(c, o)
        assert (o["tokens"][:, 0] == 0).all() and (o["logp"][:, 0] == -INF).all()


def test_ties_go_to_the_lowest_index():
    V, S = 3001, 3
    z = np.zeros((S * 3, V))
    z[:, [40, 41, 2900]] = 3.0
    c = {"S": S, "D": 2, "V": V, "n": None, "ids": np.array([[40, 40], [41, 40], [40, 2900]]), "u": None, "g": None, "w": None,
         "z": rows_of(z, torch.bfloat16, V, 1)}
    o = run(c)
    check(c, o)
    assert o["accepted"].tolist() == [2, 0, 1] and o["tokens"].tolist() == [[40, 40, 40], [40, -1, -1], [40, 40, -1]]


def test_sick_logits_and_bad_arguments_on_the_device():
    c = make(11, 4, 3, 900, "f32", "draft", n_draft=np.array([3, 3, 3, 3]))
    c["z"][1, 17] = NAN                       # row 1 of sequence 0
    c["z"][4 + 2, 3] = INF                    # row 2 of sequence 1
    c["w"][2 * 3] = NAN                       # the first draft row of sequence 2
    c["u"][:] = 0.0
    o = run(c)
    assert torch.isnan(o["accept"][0, 1]) and torch.isnan(o["accept"][1, 2]) and torch.isnan(o["accept"][2, 0])
    assert o["accepted"].tolist()[:3] == [1, 2, 0]
    assert ((o["tokens"] >= -1) & (o["tokens"] < 900)).all()
    assert (o["tokens"].gather(1, o["accepted"].long()[:, None]) >= 0).all()
    c = make(12, 4, 3, 900, "f32", "draft", n_draft=np.array([3, 9, -1, 2]))
    c["ids"][0, 1], c["u"][0, 0] = 900, 0.0
    c["ids"][0, 0] = int(host_f64(c["z"][:1].contiguous())[0].argmax())
    o = run(c)
    assert H.device_error(clear=True) in (0x201, 0x202)
    assert o["accepted"][0] == 1 and torch.isnan(o["accept"][0, 1]) and o["tokens"][2, 0] >= 0
    fixed = dict(c, n=np.array([1, 3, 0, 2]))
    ref = run(fixed)
    assert torch.equal(o["tokens"][1:], ref["tokens"][1:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
@pytest.mark.parametrize("what", [NAN, INF])
@pytest.mark.parametrize("V,ld,shift,at", [(900, 900, 0, 450), (901, 907, 3, 0), (901, 907, 3, 900)])
def test_sick_rows_refuse_their_drafts(V, ld, shift, at, what, mode, dtype):
    """`what` at one token of target row 1 of three: the drafted token is the row's largest finite logit, masked, or the sick one
    itself; a masked token under a sick draft row; a sick target row beside a draft row of nothing but -inf. With u = 0
    everything else is kept."""
    S, D = 6, 3
    c = make(14, S, D, V, dtype, mode, ld=ld, shift=shift, n_draft=None)
    z = c["z"].view(S, D + 1, V)
    c["ids"] = z[:, :D].double().cpu().numpy().argmax(-1)
    if c["u"] is not None:
        c["u"][:] = 0.0
    masked = (at + 7) % V
    z[:4, 1, at] = what
    finite = z[:, 1].double().cpu().numpy()
    finite[:4, at] = -INF
    c["ids"][:, 1] = finite.argmax(-1)
    c["ids"][1, 1], c["ids"][2, 1] = masked, at
    z[1, 1, masked] = -INF
    sick = [0, 1, 2, 3]
    if mode == "draft":
        w = c["w"].view(S, D, V)
        w[3, 1] = -INF
        z[4, 1, masked], w[4, 1, at] = -INF, what
        c["ids"][4, 1] = masked
        sick.append(4)
    o = {k: v.cpu() for k, v in run(c).items()}
    for s in range(S):
        kept = 1 if s in sick else 3
        assert o["accepted"][s] == kept and o["tokens"][s, :kept].tolist() == c["ids"][s, :kept].tolist(), s
        assert 0 <= o["tokens"][s, kept] < V and (o["tokens"][s, kept + 1:] == -1).all(), s
        assert torch.isnan(o["accept"][s]).tolist() == [False, s in sick, False], s
        assert torch.isnan(o["logp"][s, :4]).tolist() == [False, s < 4, False, False], s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("mode", ["draft", "given"])
@pytest.mark.parametrize("base", [1e6, -3e5, 3e37, "lowest"])
def test_noise_counts_beside_logits_of_any_size(base, mode, dtype):
    """Draws from a row of large logits, some of which are equal: the noise decides between them as between small ones."""
    S, D, V = 200, 2, 1000
    c = make(15, S, D, V, dtype, mode, n_draft=np.arange(S) % (D + 1))
    if base == "lowest":
        for x in (c["z"], c["w"]):
            if x is not None:
                x.fill_(torch.finfo(TYPES[dtype]).min)
    else:
        step = 2.0 ** np.floor(np.log2(abs(base))) * (2.0 ** -22 if dtype == "f32" else 2.0 ** -7)
        rng = np.random.default_rng(16)
        for x in (c["z"], c["w"]):
            if x is not None:
                x.copy_(torch.from_numpy(base + step * rng.integers(0, 3, tuple(x.shape))).cuda())
    o = run(c)
    check(c, o)
    if base == "lowest" and mode == "draft":  # equal rows: all is kept, and the token after is the noise's largest
        n = c["n"]
        assert (o["accepted"].cpu().numpy() == n).all()
        assert (o["tokens"].cpu().numpy()[np.arange(S), n] == c["g"].argmax(-1)).all()


def test_frequencies_are_the_targets():
    """20000 sequences with one draft each over five tokens: the first token is the target's draw. A count of n draws
    with probability p is off by 5 sqrt(n p (1 - p)) less than once in a million."""
    S, V = 20000, 5
    p, q = np.array([0.5, 0.2, 0.2, 0.1, 0.0]), np.array([0.2, 0.2, 0.3, 0.1, 0.2])
    rng = np.random.default_rng(0)
    with np.errstate(divide="ignore"):
        z, w = np.tile(np.log(p), (2 * S, 1)), np.tile(np.log(q), (S, 1))
    for draft in (True, False):
        ids = rng.choice(V, S, p=q)[:, None] if draft else np.full((S, 1), 2)
        c = {"S": S, "D": 1, "V": V, "n": None, "ids": ids, "z": rows_of(z, torch.float32, V, 0),
             "w": rows_of(w, torch.float32, V, 0) if draft else None, "u": rng.random((S, 1)).astype(np.float32),
             "g": rng.gumbel(size=(S, V)).astype(np.float32)}
        first = run(c)["tokens"][:, 0].cpu().numpy()
        count = np.bincount(first, minlength=V)
        assert (np.abs(count - S * p) <= 5 * np.sqrt(S * p * (1 - p))).all(), count


def test_streams_and_a_captured_call():
    c = make(13, 6, 4, 5000, "bf16", "draft")
    ids, n, u, g = dev_i32(c["ids"]), dev_i32(c["n"]), dev_f32(c["u"]), dev_f32(c["g"])
    o = {k: v.clone() for k, v in run(c).items()}
    out = {k: torch.zeros_like(v) for k, v in o.items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        H.hydra_verify_drafts(c["z"], c["w"], ids, n, u, g, 6, 4, **out)
    u.fill_(2.0)  # refuses all
    graph.replay()
    torch.cuda.synchronize()
    assert (out["accepted"] == 0).all()
    u.copy_(dev_f32(c["u"]))
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(out[k], o[k]) for k in o)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = run(c)
    side.synchronize()
    assert all(torch.equal(again[k], o[k]) for k in o)
