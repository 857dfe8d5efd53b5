"""Draft verification on the GPU against the fp64 oracle: whole numbers, equal."""
import numpy as np
import pytest
import torch

from oracle import plt_draft_verify as oracle_verify
from paper_2510_24824_b200 import binding as B
from paper_2510_24824_b200.runner import DraftVerify

pytestmark = pytest.mark.gpu


def problem(seed, Bn, K, V, dtype="f32", probs=True, ragged=True, near=0.7):
    rng = np.random.default_rng(seed)
    logits = rng.standard_normal((Bn, K + 1, V)) * 2.0
    other = logits[:, :K] + near * rng.standard_normal((Bn, K, V))
    soft = lambda x: torch.softmax(torch.from_numpy(x), dim=-1).to(torch.float32 if dtype == "f32" else torch.bfloat16)  # noqa: E731
    target, draft = soft(logits), soft(other)
    drafts = np.argmax(other + rng.gumbel(size=other.shape), axis=2).astype(np.int32)
    return dict(target=target, draft=draft if probs else None, drafts=drafts,
                lens=rng.integers(0, K + 1, Bn).astype(np.int32) if ragged else None,
                u=rng.random((Bn, K)).astype(np.float32), r=rng.random(Bn).astype(np.float32))


def call(op, x, views=False):
    dev = lambda a: None if a is None else (a if isinstance(a, torch.Tensor) else torch.from_numpy(a)).cuda()  # noqa: E731
    Bn, K = x["drafts"].shape
    tokens = torch.full((Bn, K + 1), -7, dtype=torch.int32, device="cuda")
    n = torch.full((Bn,), -7, dtype=torch.int32, device="cuda")
    lens = torch.arange(Bn, dtype=torch.int32, device="cuda")
    new = torch.full((Bn,), -7, dtype=torch.int32, device="cuda")
    target, draft = dev(x["target"]), dev(x["draft"])
    op.run(target, dev(x["drafts"]), dev(x["u"]), dev(x["r"]), tokens, n, draft=draft, draft_lens=dev(x["lens"]), seq_lens=lens, new_lens=new)
    n_host = n.cpu().numpy()
    assert np.array_equal(new.cpu().numpy(), np.maximum(0, np.arange(Bn) - (K - n_host)))
    return tokens.cpu().numpy(), n_host


def expect(x):
    wide = lambda t: None if t is None else t.float().numpy()  # noqa: E731
    return oracle_verify.verify(wide(x["target"]), wide(x["draft"]), x["drafts"], x["lens"], x["u"], x["r"])


def check(x, op=None):
    Bn, K = x["drafts"].shape
    V = x["target"].shape[2]
    own = op is None
    op = op or DraftVerify("f32" if x["target"].dtype == torch.float32 else "bf16", Bn, K, V)
    got, n = call(op, x)
    want, wn, near = expect(x)
    assert op.check() == 0
    # two orders of adding V numbers in 64 bits differ by less than V * 2^-52 of their sum; the inputs stay further from a border
    assert near.min() > V * 2.0 ** -52
    assert np.array_equal(n, wn) and np.array_equal(got, want)
    if own:
        op.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("probs", [True, False])
@pytest.mark.parametrize("Bn,K,V", [(1, 1, 1), (3, 2, 2), (2, 1, 31), (5, 4, 257), (7, 3, 2048), (4, 8, 4099), (3, 5, 16384), (2, 64, 500),
                                    (33, 33, 1000), (2, 2, 50257), (1, 3, 131072), (70, 2, 20001)])
def test_against_the_oracle(dtype, probs, Bn, K, V):
    check(problem(Bn * 1000 + K + V, Bn, K, V, dtype, probs))


def test_full_lengths_and_large_batch():
    check(problem(5, 300, 4, 8192, ragged=False))


def test_vocabulary_of_many_chunks():
    check(problem(6, 1, 1, (1 << 22) + 5))


def test_certain_and_impossible_drafts():
    """Equal rows accept everything (u < 1); rows without a common token refuse everything; rows equal but for rounding."""
    x = problem(7, 6, 3, 1000, ragged=False)
    x["draft"] = x["target"][:, :3].clone()
    x["u"][:] = np.nextafter(np.float32(1), np.float32(0))
    got, n = call(DraftVerify("f32", 6, 3, 1000), x)
    assert (n == 3).all() and np.array_equal(got, expect(x)[0])
    x = problem(8, 6, 3, 1000, ragged=False)
    x["target"][:, :, ::2] = 0
    x["draft"][:, :, 1::2] = 0
    x["drafts"] = (x["drafts"] // 2 * 2).astype(np.int32)
    x["u"][:] = 0
    got, n = call(DraftVerify("f32", 6, 3, 1000), x)
    assert (n == 0).all() and (got[:, 0] % 2 == 1).all() and np.array_equal(got, expect(x)[0])


def test_nothing_left_of_p_over_q_falls_back_to_p():
    x = problem(9, 4, 2, 3000, ragged=False)
    x["draft"] = x["target"][:, :2].clone() * 2
    x["u"][:] = 0.75                                     # 0.75 * 2 p >= p: refused, and p - 2 p is nowhere above 0
    check(x)


@pytest.mark.parametrize("r", [0.0, 0.5, np.nextafter(np.float32(1), np.float32(0)), 1.0, 2.0, np.nan])
def test_borders_of_the_last_number(r):
    """Equal weights in powers of two: every sum is exact, and r * total falls on a border."""
    V = 4096
    x = dict(target=torch.full((3, 2, V), 1.0 / V), draft=torch.full((3, 1, V), 1.0 / V), drafts=np.array([[5], [6], [7]], np.int32),
             lens=np.array([0, 1, 1], np.int32), u=np.zeros((3, 1), np.float32), r=np.full(3, r, np.float32))
    got, n = call(DraftVerify("f32", 3, 1, V), x)
    last = V - 1 if not r < 1 else int(np.floor(np.float64(np.float32(r)) * V))
    assert n.tolist() == [0, 1, 1] and got[0, 0] == last and got[1, 1] == last
    # weights at few places, so that most threads and chunks hold nothing
    t = torch.zeros(3, 2, V)
    t[:, :, [17, 1500, 4095]] = torch.tensor([0.5, 0.25, 0.25])
    x["target"], x["lens"] = t, np.zeros(3, np.int32)
    got, _ = call(DraftVerify("f32", 3, 1, V), x)
    assert (got[:, 0] == (4095 if not r < 0.75 else 1500 if r >= 0.5 else 17)).all()


def test_numbers_that_are_none():
    """NaN, infinities and negative entries weigh nothing; a row of them gives -1 and its flag; NaN never passes a draft."""
    V = 600
    x = problem(11, 5, 2, V, ragged=False)
    x["target"][0, :, ::3] = float("nan")
    x["target"][1, :, ::3] = float("inf")
    x["draft"][1, :, ::5] = float("nan")
    x["target"][2, :, 1::2] *= -1
    x["target"][3] = float("nan")
    x["u"][4] = float("nan")
    op = DraftVerify("f32", 5, 2, V)
    got, n = call(op, x)
    want, wn, _ = expect(x)
    assert op.check() == B.PLT_DEV_NO_PROBABILITY and op.check() == 0
    assert np.array_equal(got, want) and np.array_equal(n, wn) and n[3] == 0 and got[3, 0] == -1 and n[4] == 0


def test_drafts_out_of_range_are_refused_and_flagged():
    for bad in (-1, 700, 2 ** 31 - 1, -2 ** 31):
        x = problem(12, 3, 3, 700, ragged=False, probs=False)
        x["drafts"][1, 0] = bad
        op = DraftVerify("f32", 3, 3, 700)
        got, n = call(op, x)
        assert op.check() == B.PLT_DEV_TOKEN_OUT_OF_RANGE
        want, wn, _ = expect(x)
        assert np.array_equal(got, want) and np.array_equal(n, wn) and n[1] == 0


def test_lengths_out_of_range_are_clamped_and_flagged():
    x = problem(13, 4, 3, 700)
    x["lens"] = np.array([-5, 9, 3, 0], np.int32)
    op = DraftVerify("f32", 4, 3, 700)
    got, n = call(op, x)
    assert op.check() == B.PLT_DEV_SEQ_LEN_CLAMPED
    want, wn, _ = expect(x)
    assert np.array_equal(got, want) and np.array_equal(n, wn)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_shifted_views(dtype):
    """Rows that start at every place of the 16-byte grid, and rows of p and q that lie differently on it."""
    V, K, Bn = 1003, 2, 3
    for shift in range(0, 9):
        for q_shift in (0, 1, shift):
            x = problem(20 + shift, Bn, K, V, dtype)
            for name, rows, s in (("target", K + 1, shift), ("draft", K, q_shift)):
                wide = torch.full((Bn, rows + 1, V + 13), float("nan"), dtype=x[name].dtype)
                wide[:, :rows, s:s + V] = x[name]
                x[name] = wide
            op = DraftVerify(dtype, Bn, K, V)
            cuda = {k: v.cuda() for k, v in (("target", x["target"]), ("draft", x["draft"]))}
            views = dict(x, target=cuda["target"][:, :K + 1, shift:shift + V], draft=cuda["draft"][:, :K, q_shift:q_shift + V])
            got, n = call(op, views)
            want, wn, _ = expect({k: (v.cpu() if isinstance(v, torch.Tensor) else v) for k, v in views.items()})
            assert np.array_equal(got, want) and np.array_equal(n, wn), (shift, q_shift)


def test_repeats_other_streams_and_graphs():
    """The same answer from every call; calls on another stream; a captured call replayed with other inputs in the same
    buffers, and calls of other batch sizes in between."""
    K, V = 3, 40000
    op = DraftVerify("f32", 6, K, V)
    xs = [problem(30 + i, 6, K, V) for i in range(3)]
    dev = lambda a: (a if isinstance(a, torch.Tensor) else torch.from_numpy(a)).cuda()  # noqa: E731
    held = {k: dev(v) for k, v in xs[0].items()}
    tokens, n = torch.empty(6, K + 1, dtype=torch.int32, device="cuda"), torch.empty(6, dtype=torch.int32, device="cuda")
    run = lambda: op.run(held["target"], held["drafts"], held["u"], held["r"], tokens, n, draft=held["draft"], draft_lens=held["lens"])  # noqa: E731
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(5):
            run()
    side.synchronize()
    assert np.array_equal(tokens.cpu().numpy(), expect(xs[0])[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in (1, 2, 0):
        for k, v in xs[i].items():
            held[k].copy_(dev(v))
        tokens.fill_(-9)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(tokens.cpu().numpy(), expect(xs[i])[0])
        check(problem(40 + i, 2, K, V), op=op)
    assert op.check() == 0


def test_refusals_of_a_call():
    op = DraftVerify("f32", 2, 2, 100)
    x = problem(50, 2, 2, 100)
    dev = lambda a: (a if isinstance(a, torch.Tensor) else torch.from_numpy(a)).cuda()  # noqa: E731
    t = {k: dev(v) for k, v in x.items()}
    tokens, n = torch.full((2, 3), -7, dtype=torch.int32, device="cuda"), torch.full((2,), -7, dtype=torch.int32, device="cuda")
    args = lambda **kw: B.make_verify_args(**{**dict(batch=2, target_probs=t["target"], draft_tokens=t["drafts"], accept_u=t["u"], sample_u=t["r"],  # noqa: E731
                                                     tokens=tokens, num_accepted=n, draft_probs=t["draft"]), **kw})
    for kw, code in ((dict(batch=3), B.PLT_ERR_CAPACITY), (dict(batch=-1), B.PLT_ERR_INVALID_ARG), (dict(target_probs=None), B.PLT_ERR_INVALID_ARG),
                     (dict(tokens=None), B.PLT_ERR_INVALID_ARG), (dict(seq_lens=n), B.PLT_ERR_INVALID_ARG), (dict(new_lens=n), B.PLT_ERR_INVALID_ARG),
                     (dict(target_strides=(300, 99)), B.PLT_ERR_INVALID_ARG), (dict(draft_strides=(99, 100)), B.PLT_ERR_INVALID_ARG),
                     (dict(target_probs=t["target"].data_ptr() + 2), B.PLT_ERR_INVALID_ARG), (dict(tokens=tokens.data_ptr() + 1), B.PLT_ERR_INVALID_ARG)):
        with pytest.raises(B.PltError) as e:
            B.plt_draft_verify_run(op.handle, args(**kw))
        assert e.value.status == code and e.value.message, kw
    bad = args()
    bad.struct_size -= 8
    with pytest.raises(B.PltError):
        B.plt_draft_verify_run(op.handle, bad)
    B.plt_draft_verify_run(op.handle, args(batch=0))
    torch.cuda.synchronize()
    assert (tokens == -7).all() and (n == -7).all() and op.check() == 0
    with pytest.raises(ValueError):
        op.run(t["target"].transpose(1, 2), t["drafts"], t["u"], t["r"], tokens, n)
    with pytest.raises(ValueError):
        op.run(t["target"], t["drafts"].long(), t["u"], t["r"], tokens, n)
