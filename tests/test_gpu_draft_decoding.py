"""Decoding with drafted tokens, the operators one after another as a server runs them: prompts of uneven length into the
cache, then steps of the last token and its drafts (append, attention, logits, verification), the refused drafts overwritten
by the next step, sequences that end at different times, and the step as one captured graph.

The model is a single layer whose query, key and value are a bf16 row of a table for each token, so that the oracle knows
them bit for bit; attention has the tolerance derived in test_gpu_paged_attention.py, and verification is compared on the
logits that the device made."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import oracle as O
from paper_2309_00754_gb300 import build as B
from paper_2309_00754_gb300 import hydra as H
from tests.helpers import dev_i32
from tests.test_gpu_paged_attention import check
from tests.test_gpu_paged_cache import pages_for, rope_table

pytestmark = pytest.mark.gpu

HEADS, KV, D, V, DRAFTS = 4, 2, 64, 7, 3
PROMPTS = [1, 2, 9, 16, 17, 30]
NEW = [20, 33, 5, 17, 1, 26]  # tokens wanted
S, L = len(PROMPTS), DRAFTS + 1


@pytest.fixture(scope="module", autouse=True)
def lib():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    B.build()
    H.load()
    H.device_error(clear=True)
    yield
    assert H.device_error(clear=True) == 0


class Server:
    """The sequences' state on the device, and a step of all of them."""

    def __init__(self, seed, mode, int4):
        rng = np.random.default_rng(seed)
        self.mode, self.int4 = mode, int4
        self.rows = torch.from_numpy(rng.normal(0, 1.5, (V, (HEADS + 2 * KV) * D))).bfloat16()
        self.out = torch.from_numpy(rng.normal(0, 0.3, (HEADS * D, V))).float().cuda()
        self.prompts = [rng.integers(0, V, n) for n in PROMPTS]
        total = [p + n + L for p, n in zip(PROMPTS, NEW)]
        table, n_pages = pages_for(rng, total, 16)
        self.cache = H.KvCache(H.HYDRA_KV_INT4 if int4 else H.HYDRA_KV_BF16, n_pages, 16, KV, D)
        self.cache.data.fill_(0xFF)
        self.table, self.rope = dev_i32(table), rope_table(max(total), D)
        self.rope_dev, self.rows_dev = torch.from_numpy(self.rope).cuda(), self.rows.cuda()
        self.ws = torch.empty(H.paged_attention_workspace_size(S, L, HEADS, KV, D), dtype=torch.uint8, device="cuda")
        zeros = lambda *shape, **kw: torch.zeros(*shape, device="cuda", **kw)  # noqa: E731
        self.cached, self.lengths, self.n_draft = (zeros(S, dtype=torch.int32) for _ in range(3))
        self.tokens = zeros(S, L, dtype=torch.int32)
        self.q = zeros(S * L, HEADS * D, dtype=torch.bfloat16)
        self.o, self.logits = torch.empty_like(self.q), zeros(S * L, V)
        self.ids = zeros(S, DRAFTS, dtype=torch.int32)
        self.draft = zeros(S * DRAFTS, V) if mode == "draft" else None
        self.uniform, self.gumbel = (None, None) if mode == "greedy" else (zeros(S, DRAFTS), zeros(S, V))
        self.next, self.accepted = zeros(S, L, dtype=torch.int32), zeros(S, dtype=torch.int32)

    def prefill(self):
        n = max(PROMPTS) - 1
        tokens = torch.zeros(S, n, dtype=torch.long)
        for s, p in enumerate(self.prompts):
            tokens[s, :len(p) - 1] = torch.from_numpy(p[:-1])
        x = self.rows_dev[tokens.cuda().reshape(-1)]
        k, v = x[:, HEADS * D:(HEADS + KV) * D], x[:, (HEADS + KV) * D:]
        lengths = dev_i32([len(p) - 1 for p in self.prompts])
        H.hydra_kv_append(self.cache, self.table, None, lengths, S, n, None, k, v, self.rope_dev)
        self.cached.copy_(lengths)

    def matmul(self):
        torch.matmul(self.o.float(), self.out, out=self.logits)

    def step(self):
        x = self.rows_dev[self.tokens.reshape(-1).long()]
        q, k, v = x[:, :HEADS * D], x[:, HEADS * D:(HEADS + KV) * D], x[:, (HEADS + KV) * D:]
        H.hydra_kv_append(self.cache, self.table, self.cached, self.lengths, S, L, q, k, v, self.rope_dev, self.q)
        H.hydra_paged_attention(self.cache, self.table, self.cached, self.lengths, S, L, self.q, self.o, D ** -0.5, self.ws)
        self.matmul()
        H.hydra_verify_drafts(self.logits, self.draft, self.ids, self.n_draft, self.uniform, self.gumbel, S, DRAFTS, self.next,
                              self.accepted)
        # the tokens that stay; the refused ones are written over
        self.cached += torch.where(self.lengths > 0, self.accepted + 1, 0).int()

    def generate(self, seed, graph, look=None):
        rng = np.random.default_rng(seed)
        self.prefill()
        texts, kept = [list(map(int, p)) for p in self.prompts], []
        run = self.step
        if graph:
            torch.cuda.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                self.step()
            run = g.replay
        while any(len(t) - p < n for t, p, n in zip(texts, PROMPTS, NEW)):
            live = np.array([len(t) - p < n for t, p, n in zip(texts, PROMPTS, NEW)])
            n_draft = np.where(live, rng.integers(0, DRAFTS + 1, S), 0)
            ids = rng.integers(0, V, (S, DRAFTS))
            tokens = np.concatenate([[[t[-1]] for t in texts], ids], 1)
            self.tokens.copy_(dev_i32(tokens))
            self.ids.copy_(dev_i32(ids))
            self.n_draft.copy_(dev_i32(n_draft))
            self.lengths.copy_(dev_i32(np.where(live, n_draft + 1, 0)))
            if self.draft is not None:
                self.draft.copy_(torch.from_numpy(rng.normal(0, 1, (S * DRAFTS, V))))
            if self.uniform is not None:
                self.uniform.copy_(torch.from_numpy(rng.uniform(0, 1, (S, DRAFTS)) * 0.999))
                self.gumbel.copy_(torch.from_numpy(rng.gumbel(0, 1, (S, V))))
            run()
            accepted, out = self.accepted.cpu().numpy(), self.next.cpu().numpy()
            if look is not None:
                look(self, texts, ids, n_draft, live)
            for s in np.flatnonzero(live):
                texts[s] += [int(x) for x in out[s, :accepted[s] + 1]]
                kept.append((int(accepted[s]), int(n_draft[s])))
        return texts, kept


def compare(server, texts, ids, n_draft, live):
    """A step's queries, attention and verification against the oracle, from the sequences' true tokens."""
    lengths = np.where(live, n_draft + 1, 0)
    cached = np.array([len(t) - 1 for t in texts])
    N = int((cached + lengths).max())
    x = server.rows.float().numpy().reshape(V, -1, D)
    q, k, v = np.zeros((S, L, HEADS, D), np.float32), *np.zeros((2, S, N, KV, D), np.float32)
    for s in range(S):
        tokens = np.array(texts[s] + list(ids[s, :n_draft[s]]))[:cached[s] + lengths[s]]
        turned = O.rope_by_table(x[tokens][:, :HEADS + KV], server.rope[:len(tokens)])
        q[s, :lengths[s]] = turned[cached[s]:, :HEADS]
        k[s, :len(tokens)], v[s, :len(tokens)] = turned[:, HEADS:], x[tokens][:, HEADS + KV:]
    got_q = server.q.float().cpu().numpy().reshape(q.shape)
    np.testing.assert_array_equal(got_q, O.round_bf16(q.astype(np.float64)).astype(np.float32))
    check({"S": S, "L": L, "heads": HEADS, "kv": KV, "D": D, "cached": cached, "lengths": lengths, "q": server.q.cpu(),
           "k": O.kv_held(k, server.int4), "v": O.kv_held(v, server.int4)}, server.o)
    cpu = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
    want = O.verify_drafts(cpu(server.logits), cpu(server.draft), ids, n_draft, cpu(server.uniform), cpu(server.gumbel), S, DRAFTS)
    for s in np.flatnonzero(live):
        assert server.accepted[s].item() == want["accepted"][s]
        assert server.next[s].tolist() == want["tokens"][s].tolist()


def test_the_first_call_of_a_process_may_be_captured():
    """What a call looks up once for a device can be looked up while a stream is captured."""
    code = (
        "import torch; from tests.test_gpu_draft_decoding import Server\n"
        "for mode, int4 in (('draft', True), ('greedy', False)):\n"
        "    s = Server(3, mode, int4)\n"
        "    s.matmul()\n"
        "    torch.cuda.synchronize()\n"
        "    g = torch.cuda.CUDAGraph()\n"
        "    with torch.cuda.graph(g):\n"
        "        s.step()\n"
        "    s.lengths.fill_(1)\n"
        "    g.replay()\n"
        "    torch.cuda.synchronize()\n"
        "    assert s.cached.tolist() == [1] * len(s.cached)\n")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    run = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert run.returncode == 0, run.stderr[-2000:]


@pytest.mark.parametrize("int4", [True, False])
@pytest.mark.parametrize("mode", ["draft", "given", "greedy"])
def test_generation(mode, int4):
    texts, kept = Server(3, mode, int4).generate(4, False, compare)
    assert all(len(t) >= p + n for t, p, n in zip(texts, PROMPTS, NEW))
    assert any(a == n > 0 for a, n in kept) and any(a < n for a, n in kept)
    # the same steps as a graph, with another pool
    assert Server(3, mode, int4).generate(4, True) == (texts, kept)
