"""The serving operators together, as a program that generates text runs them: ragged
prompts and then single tokens of several sequences, each step the append of its rows,
attention over the pages and the draw of the next tokens from logits that come from the
attention's output; eagerly, and as one captured step that feeds itself."""

import numpy as np
import pytest

from tests.test_gpu_draw import plain as plain_draw
from tests.test_gpu_paged import Case, E, i32  # noqa: F401 (E: a fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

VOCAB = 500
SETTINGS = dict(temperature=[0.7, 0.0, 1.3], top_k=[40, 0, 0], top_p=[0.9, 1.0, 0.95],
                min_p=[0.0, 0.0, 0.02])


class Loop:
    """Three sequences.  A token's fused row is looked up; a row's logits are elements of
    its attention output, so that every other step is exact."""

    def __init__(self, E, case, seed):
        self.E, self.case = E, case
        c = case
        g = torch.Generator().manual_seed(seed)
        self.rows_of = torch.randn(VOCAB, c.hq + 2 * c.hkv, c.hd, generator=g).to(c.dt).cuda()
        self.pick = torch.randperm(c.hq * c.hd, generator=g)[:VOCAB].cuda()
        dt = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32,
                  min_p=torch.float32)
        self.set = {k: torch.tensor(v, dtype=dt[k], device="cuda") for k, v in SETTINGS.items()}
        self.rope = torch.from_numpy(c.rope).cuda()
        self.table = i32(c.table)
        self.pos0 = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.tokens = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.u = torch.zeros(3, device="cuda")
        self.kept = torch.zeros(3, dtype=torch.int32, device="cuda")
        self.logprob = torch.zeros(3, device="cuda")
        self.cap = c.table.shape[1] * c.cache.page

    def buffers(self, n):
        """Of a step of n rows."""
        c, E = self.case, self.E
        return dict(q=torch.zeros(n, c.hq, c.hd, dtype=c.dt, device="cuda"),
                    out=torch.zeros(n, c.hq, c.hd, dtype=c.dt, device="cuda"),
                    logits=torch.zeros(3, VOCAB, dtype=c.dt, device="cuda"),
                    wa=E.paged_attention_workspace(c.cache, 3, n, c.hq, n, self.cap),
                    wd=E.sample_draw_workspace(3, VOCAB))

    def step(self, ids, start, last, n, b):
        c, E = self.case, self.E
        x = self.rows_of.index_select(0, ids)
        E.paged_append(c.cache, self.table, start, self.pos0, x[:, c.hq:c.hq + c.hkv],
                       x[:, c.hq + c.hkv:], q=x[:, :c.hq], rope=self.rope, q_out=b["q"], max_rows=n)
        E.paged_attention(c.cache, self.table, start, self.pos0, b["q"], out=b["out"],
                          workspace=b["wa"], max_rows=n, max_len=self.cap)
        y = b["out"].view(ids.shape[0], -1).index_select(0, last)
        b["logits"].copy_(y.index_select(1, self.pick) * 8)
        E.sample_draw(b["logits"], self.u, tokens=self.tokens, kept=self.kept,
                      logprob=self.logprob, workspace=b["wd"], **self.set)
        self.pos0 += start[1:] - start[:-1]

    def check(self, ids, start, pos0, b):
        """The step against the plain forms, on what it took in."""
        c = self.case
        x = self.rows_of[ids.long()].double().cpu().numpy()
        c.plain.append(c.table, start, pos0, x[:, c.hq:c.hq + c.hkv], x[:, c.hq + c.hkv:], c.rope)
        c.check_queries(x[:, :c.hq], b["q"], start, pos0, True)
        c.check_cache()
        lse = torch.empty(b["q"].shape[:2], device="cuda")
        again = self.E.paged_attention(c.cache, self.table, i32(start), i32(pos0), b["q"], lse=lse)
        c.check_attention(b["q"], b["out"], lse, start, pos0)
        c.check_attention(b["q"], again, lse, start, pos0)
        lg, u = b["logits"].double().cpu().numpy(), self.u.cpu().numpy()
        for r in range(3):
            f = lambda k: float(np.float32(SETTINGS[k][r]))
            tok, lp, kept = plain_draw(lg[r], f("temperature"), SETTINGS["top_k"][r], f("top_p"),
                                       f("min_p"), float(u[r]))
            assert (self.tokens[r].item(), self.kept[r].item()) == (tok, kept), r
            # the sum's units and the float32 rounding
            assert abs(self.logprob[r].item() - lp) <= 2.0 ** -23 * abs(lp) + 2.0 ** -26


@pytest.mark.parametrize("kind,dtype,block", [("e4m3", "bf16", 16), ("bf16", "f32", 16),
                                              ("e4m3", "f32", 32)])
def test_prompts_and_a_captured_decode_loop(E, kind, dtype, block):  # noqa: F811
    c = (3, 8, 2, 128, 32, block, kind, dtype, 4)
    x, y = Loop(E, Case(E, *c, seed=21), 5), Loop(E, Case(E, *c, seed=21), 5)
    rng = np.random.RandomState(3)
    draws = lambda: torch.tensor(rng.uniform(0, 1, 3).astype(np.float32))
    start = np.array([0, 70, 71, 90])  # prompts of 70, 1 and 19 tokens
    ids = torch.from_numpy(rng.randint(0, VOCAB, 90)).cuda()
    u, last = draws(), i32(start[1:] - 1)
    for z in (x, y):
        z.u.copy_(u)
        b = z.buffers(90)
        z.step(ids, i32(start), last, 90, b)
        z.check(ids, start, np.zeros(3, int), b)
    assert torch.equal(x.tokens, y.tokens)

    one, each = i32([0, 1, 2, 3]), i32([0, 1, 2])
    bx = x.buffers(3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    state = x.tokens.clone(), x.pos0.clone()
    with torch.cuda.stream(s):  # its rows are written again by the first replay
        x.step(x.tokens, one, each, 3, bx)
    torch.cuda.current_stream().wait_stream(s)
    x.tokens.copy_(state[0]), x.pos0.copy_(state[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.step(x.tokens, one, each, 3, bx)
    for i in range(6):
        u = draws()
        x.u.copy_(u), y.u.copy_(u)
        ids, pos0 = y.tokens.clone(), y.pos0.cpu().numpy()
        g.replay()
        by = y.buffers(3)  # eager, between the replays
        y.step(ids, one, each, 3, by)
        torch.cuda.synchronize()
        assert torch.equal(x.tokens, y.tokens) and torch.equal(x.kept, y.kept), i
        assert torch.equal(bx["out"], by["out"]) and torch.equal(x.logprob, y.logprob)
        assert torch.equal(x.pos0, y.pos0)
        y.check(ids, np.arange(4), pos0, by)
    assert x.pos0.cpu().tolist() == [76, 7, 25]
