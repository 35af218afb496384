"""The decoder over a paged cache (emoe_decoder_forward_paged): ragged prompts
and batched decode steps against the fp64 decoder oracle, sequence by sequence
(fed with the GPU's own tokens, so that both sides stay on one text)."""
import numpy as np
import pytest
import torch

from oracle import decoder_oracle as D
from oracle import serving_oracle as S
from paper_2608_15383_amd import api
from paper_2608_15383_amd._lib import EMOE_EINVAL, EMOE_ESHAPE, EMOE_ESTATE, ExactMoEError
from tests._gpu import TOL, rel_err
from tests.test_gpu_decoder import SMALL, GpuDecoder, _model, _oracle_weights

pytestmark = pytest.mark.gpu


def ids(a):
    return torch.from_numpy(np.ascontiguousarray(np.asarray(a, np.int32))).to("cuda:0")


class Paged:
    """A decoder without a contiguous cache, and paged caches for `seqs` sequences of `keys`."""

    def __init__(self, shape, m, seqs=3, keys=64, page=8, dtype=torch.bfloat16, seed=0, max_tokens=64):
        self.g = GpuDecoder(shape, m, shape.n_experts)
        self.dec = api.Decoder(self.g.dd, self.g.w, self.g.caches)
        self.shape, self.keys = shape, keys
        per = -(-keys // page)
        self.table = ids(np.random.default_rng(seed).permutation(seqs * per).reshape(seqs, per))
        self.kvs = []
        for _ in range(shape.n_layers):
            k, v = (torch.full((seqs * per, page, shape.n_heads, shape.head_dim), float("nan"),
                               device="cuda:0").to(dtype) for _ in range(2))
            s = torch.full((shape.n_heads,), 0.25, device="cuda:0") if dtype == torch.float8_e4m3fn else None
            self.kvs.append(api.PagedKV(k, v, s, s))
        self.ws = torch.full((api.decoder_paged_workspace_bytes(self.g.dd, max_tokens, max_tokens, keys),),
                             0xAB, dtype=torch.uint8, device="cuda:0")      # any initial value

    def run(self, tokens, positions, seqs, out_rows=None, **kw):
        n = len(tokens) if out_rows is None else len(out_rows)
        logits = torch.empty(n, self.shape.vocab, device="cuda:0")
        nt = torch.full((n,), -7, dtype=torch.int32, device="cuda:0")
        self.dec.forward_paged(self.kvs, ids(tokens), ids(positions), self.table, logits, self.ws,
                               self.keys, seqs=ids(seqs),
                               out_rows=None if out_rows is None else ids(out_rows), next_token=nt, **kw)
        torch.cuda.synchronize()
        return logits.cpu().numpy(), nt.tolist()

    def close(self):
        self.dec.close()
        self.g.close()


def _prompts(shape, lengths, seed):
    rng = np.random.default_rng(seed)
    return [rng.integers(0, shape.vocab, n).tolist() for n in lengths]


def _start(p, prompts):
    """All prompts in one call, tokens of the sequences interleaved, logits of their last tokens."""
    flat = [(t, i, s) for s, text in enumerate(prompts) for i, t in enumerate(text)]
    flat.sort(key=lambda x: (x[1], x[2]))
    last = [flat.index((text[-1], len(text) - 1, s)) for s, text in enumerate(prompts)]
    return p.run([x[0] for x in flat], [x[1] for x in flat], [x[2] for x in flat], out_rows=last)


def test_prompts_then_batched_steps_against_the_oracle():
    m = _model(SMALL, seed=1)
    w = _oracle_weights(SMALL, m)
    p = Paged(SMALL, m)
    prompts = _prompts(SMALL, (9, 1, 14), seed=2)
    states = [D.KVState() for _ in prompts]
    want = [D.decoder_forward(SMALL, w, text, st)[1] for text, st in zip(prompts, states)]
    got, tokens = _start(p, prompts)
    at = [len(text) for text in prompts]
    for step in range(5):
        for s in range(3):
            mx, _ = rel_err(got[s], want[s])
            print(f"step {step} sequence {s}: {mx:.3e}", flush=True)
            assert mx <= TOL, (step, s, mx)
            assert tokens[s] == int(np.argmax(got[s]))
        # A padding row in the middle; from the third step on five rows, so that the
        # projections take their other path.
        rows = [(tokens[0], at[0], 0), (3, 0, -1), (tokens[1], at[1], 1), (tokens[2], at[2], 2)]
        if step >= 2:
            rows.append((0, -1, 1))
        g, t = p.run(*zip(*rows))
        want = [D.decoder_forward(SMALL, w, [tokens[s]], states[s])[1] for s in range(3)]
        got, tokens = [g[i] for i in (0, 2, 3)], [t[i] for i in (0, 2, 3)]
        at = [a + 1 for a in at]
    p.close()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_pages_and_their_order_change_nothing(dtype):
    m = _model(SMALL, seed=3)
    prompts = _prompts(SMALL, (20, 7, 33), seed=4)
    seen = []
    for page, seed in ((8, 0), (8, 5), (64, 0), (16, 1)):
        p = Paged(SMALL, m, page=page, dtype=dtype, seed=seed)
        first, t = _start(p, prompts)
        more, t2 = p.run(t, [len(x) for x in prompts], [0, 1, 2])
        seen.append((first, t, more, t2))
        p.close()
    for other in seen[1:]:
        for a, b in zip(seen[0], other):
            assert np.array_equal(a, b)
    if dtype == torch.bfloat16:
        contiguous = GpuDecoder(SMALL, m, SMALL.n_experts, max_tokens=64)
        for s, text in enumerate(prompts):
            ref, _ = contiguous.run(text, 0)
            assert rel_err(seen[0][0][s], ref.astype(np.float64))[0] <= TOL
        contiguous.close()


def test_logits_are_processed():
    m = _model(SMALL, seed=5)
    p = Paged(SMALL, m)
    text = _prompts(SMALL, (12,), seed=6)[0]
    raw, t = p.run(text, range(12), [0] * 12, out_rows=[11, 11, 4])
    assert np.array_equal(raw[0], raw[1]) and t[0] == t[1]
    mask = np.full((1, -(-SMALL.vocab // 32)), -1, np.int32)
    mask.view(np.uint32)[0, t[0] // 32] &= np.uint32(0xffffffff ^ (1 << (t[0] % 32)))
    got, t2 = p.run(text, range(12), [0] * 12, out_rows=[11, 11, 4], mask=ids(mask), mask_rows=ids([0, -1, 0]),
                    history=ids([text] * 3), repetition=torch.full((3,), 1.5, device="cuda:0"))
    for i in range(3):
        want, tok, _ = S.process_logits(raw[i], text, 0, 1.5, mask=None if i == 1 else mask[0].view(np.uint32))
        assert np.array_equal(np.isinf(got[i]), np.isinf(want))
        fin = np.isfinite(want)
        assert np.all(np.abs(got[i][fin] - want[fin]) <= 2.0 ** -23 * np.abs(want[fin]))
        assert t2[i] == tok
    p.close()


def test_steps_in_a_graph():
    """Steps of up to four tokens, captured once and replayed over moving positions."""
    m = _model(SMALL, seed=7)
    prompts = _prompts(SMALL, (5, 11), seed=8)
    want = []
    for graph in (False, True):
        p = Paged(SMALL, m, seqs=2)
        _, t = _start(p, prompts)
        tok, pos, sq = ids(t), ids([5, 11]), ids([0, 1])
        logits = torch.empty(2, SMALL.vocab, device="cuda:0")
        nt = torch.empty(2, dtype=torch.int32, device="cuda:0")
        step = lambda: p.dec.forward_paged(p.kvs, tok, pos, p.table, logits, p.ws, p.keys, seqs=sq, next_token=nt)
        if graph:
            side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                with torch.cuda.graph(g, stream=side):
                    step()
            torch.cuda.synchronize()
        for i in range(6):
            g.replay() if graph else step()
            torch.cuda.synchronize()
            if graph:
                assert torch.equal(logits, want[i]), i
            else:
                want.append(logits.clone())
            tok.copy_(nt), pos.add_(1)
        p.close()


def test_refusals():
    m = _model(SMALL, seed=9)
    p = Paged(SMALL, m)

    def status(change, **kw):
        logits = torch.empty(2, SMALL.vocab, device="cuda:0")
        args = dict(kvs=p.kvs, tokens=ids([1, 2]), positions=ids([0, 1]), page_table=p.table,
                    logits=logits, workspace=p.ws, max_keys=64, seqs=ids([0, 0]))
        with pytest.raises(ExactMoEError) as e:
            p.dec.forward_paged(**{**args, **change}, **kw)
        return e.value.status

    for change in (dict(kvs=p.kvs[:1]), dict(tokens=ids([1])), dict(logits=torch.empty(3, SMALL.vocab, device="cuda:0")),
                   dict(workspace=p.ws[:1000]), dict(max_keys=-1), dict(positions=torch.zeros(2, device="cuda:0")),
                   dict(out_rows=ids([0, 1, 1]), logits=torch.empty(3, SMALL.vocab, device="cuda:0")),
                   dict(tokens=ids([]), positions=ids([]), seqs=ids([]), logits=torch.empty(0, SMALL.vocab, device="cuda:0"))):
        assert status(change) == EMOE_EINVAL, change
    assert status({}, repetition=torch.ones(2, device="cuda:0")) == EMOE_EINVAL   # no history
    half = [api.PagedKV(torch.zeros(4, 8, 2, 128, device="cuda:0").half(),
                        torch.zeros(4, 8, 2, 128, device="cuda:0").half())] * 2
    assert status(dict(kvs=half)) == EMOE_ESHAPE
    other = [api.PagedKV(torch.zeros(4, 8, 1, 128, device="cuda:0").bfloat16(),
                         torch.zeros(4, 8, 1, 128, device="cuda:0").bfloat16())] * 2
    assert status(dict(kvs=other)) == EMOE_ESHAPE
    torch.cuda.synchronize()
    assert torch.isnan(p.kvs[0]._keep[0]).all()                                  # nothing ran
    with pytest.raises(ExactMoEError) as e:
        p.dec.forward(ids([1]), 0, p.g.logits, p.g.next, p.g.ws)
    assert e.value.status == EMOE_ESTATE
    assert api.decoder_paged_workspace_bytes(p.g.dd, 2, 3, 64) == 0
    p.close()
