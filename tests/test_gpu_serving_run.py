"""The operators of a serving step together: a shared prompt into a prefix, then steps that append, attend, verify drafts and wind the
lengths back, for three sequences behind the prefix. Each kernel's answer is checked on the very inputs that the ones before it left."""
import numpy as np
import pytest
import torch

from oracle import plt_draft_verify as oracle_verify
from oracle import plt_prefix_attn as oracle_prefix
from paper_2510_24824_b200 import binding as B

pytestmark = pytest.mark.gpu

V, P, CAP, K, HQ, HKV, D, SEQS = 97, 150, 64, 3, 8, 2, 128, 3


class Model:
    """One layer of fixed random weights: rows of q, k, v for tokens, and probabilities from an attention output."""

    def __init__(self):
        g = torch.Generator("cuda").manual_seed(0)
        rand = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
        self.table = [(rand(V, h, D)).bfloat16() for h in (HQ, HKV, HKV)]
        self.head = rand(HQ * D, V) * 0.05
        self.gains = 1 + 0.1 * rand(D), 1 + 0.1 * rand(D)

    def rows(self, tokens):
        return [t[tokens].contiguous() for t in self.table]

    def probabilities(self, out):
        return torch.softmax(out.float().flatten(-2) @ self.head, dim=-1).contiguous()


@pytest.mark.parametrize("captured", [False, True])
def test_prompt_then_speculative_steps(captured):
    m, rng = Model(), np.random.default_rng(1)
    dev = lambda x: torch.as_tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    turn = dict(theta=10000.0, norm_eps=1e-6)
    gains = dict(q_gain=m.gains[0], k_gain=m.gains[1])
    # ---- the prompt, once: its keys and values go where the prefix is read from
    prompt = torch.as_tensor(rng.integers(0, V, P), device="cuda")
    q, k, v = (x.unsqueeze(0) for x in m.rows(prompt))
    k_prefix, v_prefix = (torch.zeros(1, P, HKV, D, device="cuda").bfloat16() for _ in range(2))
    first = B.plt_rope_create(B.make_rope_config("bf16", 1, 1, HQ, HKV, D, P, 0, **turn))
    q_turned = torch.empty_like(q.unsqueeze(1))
    B.plt_rope_seq(first, B.make_rope_seq_args(1, P, q, k, dev([P]), q_turned, v_share=v, k_cache=k_prefix, v_cache=v_prefix, **gains), stream())
    assert torch.equal(v_prefix, v)
    # ---- steps of K drafts behind each sequence's last token
    rope = B.plt_rope_create(B.make_rope_config("bf16", SEQS, 1, HQ, HKV, D, CAP, 0, q_len=K + 1, **turn))
    attn = B.plt_prefix_attn_create(B.make_prefix_config("bf16", SEQS, 1, HQ, HKV, D, CAP, 0, max_prefix_len=P, q_len=K + 1))
    verify = B.plt_draft_verify_create(B.make_verify_config("f32", SEQS, K, V))
    k_cache, v_cache = (torch.full((SEQS, CAP, HKV, D), float("nan"), device="cuda").bfloat16() for _ in range(2))
    lens, before = dev([P] * SEQS), dev([P] * SEQS)
    last = dev(rng.integers(0, V, SEQS))
    qs, ks, vs = (torch.empty(SEQS, 1, K + 1, h, D, device="cuda").bfloat16() for h in (HQ, HKV, HKV))
    q_out, out = torch.empty_like(qs), torch.empty_like(qs)
    drafts = torch.empty(SEQS, K, dtype=torch.int32, device="cuda")
    draft_p = torch.empty(SEQS, K, V, device="cuda")
    u, r = torch.empty(SEQS, K, device="cuda"), torch.empty(SEQS, device="cuda")
    target = torch.empty(SEQS, K + 1, V, device="cuda")
    tokens, accepted = torch.empty(SEQS, K + 1, dtype=torch.int32, device="cuda"), torch.empty(SEQS, dtype=torch.int32, device="cuda")
    group_begin, prefix_lens = dev([0, SEQS]), dev([P])

    def device_part():
        lens.add_(K + 1)
        B.plt_rope_step(rope, B.make_rope_step_args(SEQS, qs, ks, vs, q_out, k_cache, v_cache, lens, prefix_lens=before, **gains), stream())
        B.plt_prefix_attn_run(attn, B.make_args(SEQS, q_out, k_cache, v_cache, lens, out), B.make_prefix_args(1, group_begin, prefix_lens, k_prefix=k_prefix, v_prefix=v_prefix), stream())
        target.copy_(m.probabilities(out[:, 0]))
        B.plt_draft_verify_run(verify, B.make_verify_args(SEQS, target, drafts, u, r, tokens, accepted, draft_probs=draft_p, seq_lens=lens, new_lens=lens), stream())

    graph = None
    texts = [[] for _ in range(SEQS)]           # tokens whose keys are in the own caches
    for step in range(9):
        drafts.copy_(dev(rng.integers(0, V, (SEQS, K))))
        draft_p.copy_(torch.softmax(torch.as_tensor(rng.standard_normal((SEQS, K, V)), device="cuda").float(), -1))
        if step % 3 == 1:                       # drafts that the target likes: small q at the drafted token
            draft_p.scatter_(2, drafts.long().unsqueeze(-1), 1e-4)
        u.copy_(torch.as_tensor(rng.random((SEQS, K))).float())
        r.copy_(torch.as_tensor(rng.random(SEQS)).float())
        now = torch.cat([last.view(-1, 1), drafts], dim=1).long()
        for buf, rows in zip((qs, ks, vs), m.rows(now)):
            buf.copy_(rows.unsqueeze(1))
        old = lens.tolist()
        if captured and graph is None and step == 2:
            graph = torch.cuda.CUDAGraph()
            held = lens.clone()
            with torch.cuda.graph(graph):
                device_part()
            lens.copy_(held)
        graph.replay() if graph is not None else device_part()
        torch.cuda.synchronize()
        assert B.plt_rope_check(rope) == 0 and B.plt_prefix_attn_check(attn) == 0 and B.plt_draft_verify_check(verify) == 0
        # the attention on what the caches held
        held = [n + K + 1 for n in old]
        ref, size, most = oracle_prefix.attend(q_out, [(k_prefix[0], v_prefix[0])], [0, SEQS], torch.nan_to_num(k_cache.double()), torch.nan_to_num(v_cache.double()),
                                               held, D ** -0.5, [0])
        # half a step for the result, half a step of its probabilities, scores of D products in fp32 (as in the operator's own test)
        bound = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2 * (D + 2) * 2.0 ** -24 * most + 2.0 ** -16) * size + 1e-30
        assert ((out.double() - ref).abs() <= bound).all()
        # the verification on the probabilities that came of it
        want, n, near = oracle_verify.verify(target.cpu().numpy(), draft_p.cpu().numpy(), drafts.cpu().numpy(), None, u.cpu().numpy(), r.cpu().numpy())
        assert near.min() > V * 2.0 ** -52
        assert np.array_equal(tokens.cpu().numpy(), want) and np.array_equal(accepted.cpu().numpy(), n)
        assert lens.tolist() == [o + 1 + int(a) for o, a in zip(old, n)]
        for b in range(SEQS):
            texts[b] += now[b, : 1 + int(n[b])].tolist()
            last[b] = int(want[b, n[b]])
    assert max(len(t) for t in texts) > 9       # some drafts stood
    # ---- the caches hold what the prompt form gives for the tokens that stood, bit for bit
    for b in range(SEQS):
        q, k, v = (x.unsqueeze(0) for x in m.rows(torch.as_tensor(texts[b], device="cuda")))
        k_want = torch.empty_like(k)
        B.plt_rope_seq(rope, B.make_rope_seq_args(1, len(texts[b]), q, k, dev([len(texts[b])]), torch.empty_like(q), k_share_out=k_want, start=dev([P]), **gains))
        torch.cuda.synchronize()
        assert torch.equal(k_cache[b, : len(texts[b])], k_want[0]) and torch.equal(v_cache[b, : len(texts[b])], v[0])
    for name, h in (("rope", first), ("rope", rope), ("prefix_attn", attn), ("draft_verify", verify)):
        getattr(B, f"plt_{name}_destroy")(h)
