"""The operators at a step's ends as they are used together: a group's prompt is cached, its attempts fork from it, each
step places rows, norms, rotates and appends them, attends, and answers with log probabilities; attempts end and their
pages come back. In eager calls, in a captured step that is replayed among eager work, and on a stream of its own."""

import math

import numpy as np
import pytest
import torch

from oracle import ends
from paper_2609_08368_amd import rl_attn as ra
from tests import gpu_helpers as H
from tests.test_gpu_step import dev, rand

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV, PAGE, POOL, WIDTH, LAYERS, VOCAB, EPS = 16, 2, 16, 400, 24, 2, 1009, 1e-6
SCALE = 1 / math.sqrt(128)


class Engine:
    """A model of random projections over a pool of pages; keeps every request's keys and values on the side."""

    def __init__(self, batch, fp8=False, stream=None):
        rng = np.random.default_rng(1)
        self.batch, self.stream, self.fp8 = batch, stream, fp8
        kind = torch.float8_e4m3fn if fp8 else torch.bfloat16
        self.lens, self.used = dev(np.zeros(batch)), dev(np.zeros(1))
        self.free, self.table = dev(rng.permutation(POOL)), dev(np.full((batch, WIDTH), -1))
        self.pages = [tuple(torch.zeros(POOL, PAGE, HKV, 128, dtype=kind, device=DEV) for _ in "kv")
                      for _ in range(LAYERS)]
        self.scales = [torch.full((HKV,), s, device=DEV) for s in (0.02, 0.03)] if fp8 else []
        self.weights = [(rand(9 + i, 128).abs() + 0.5, rand(19 + i, 128).abs() + 0.5) for i in range(LAYERS)]
        self.freq = dev(1e4 ** (-np.arange(64) / 64), torch.float32)
        self.embed = [rand(30 + i, VOCAB, HQ + 2 * HKV, 128) for i in range(LAYERS)]
        self.head = rand(50, HQ * 128, VOCAB, spread=0.02)
        self.kept = [[[] for _ in range(batch)] for _ in range(LAYERS)]

    def rows(self, new, tokens, first):
        """One step's rows through all layers: the last layer's attention output."""
        m = ra.map_slots(self.lens, new, self.free, self.used, self.table, PAGE, POOL, tokens.shape[0],
                         kv_lens_out=self.lens, free_used_out=self.used, stream=self.stream)
        for i, (k_pages, v_pages) in enumerate(self.pages):
            x = self.embed[i][tokens]
            q, k, v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
            call = ra.norm_rope_append_kv_fp8 if self.fp8 else ra.norm_rope_append_kv
            self.k_rows = torch.empty(k.shape, dtype=k.dtype, device=DEV)
            q = call(q, k, v, *self.weights[i], EPS, m.positions.view(1, -1), self.freq, m.slot_map, k_pages, v_pages,
                     *self.scales, k_out=self.k_rows, stream=self.stream)
            self.layer = (q, self.k_rows, v, m)
            if first:
                out = ra.prefill(q, self.k_rows, v, m.qo_indptr, SCALE, stream=self.stream)
            else:
                call = ra.extend_fp8 if self.fp8 else ra.extend
                out = call(q, m.qo_indptr, k_pages, v_pages, *self.scales, self.table, self.lens, SCALE,
                           stream=self.stream)
            self.keep(i)
        return out

    def keep(self, i):
        _, k, v, m = self.layer
        if self.fp8:                                      # (the rows as the pages hold them)
            k, v = (p.view(torch.uint8).view(-1, HKV, 128)[m.slot_map].view(torch.float8_e4m3fn).float() * s[:, None] for p, s in zip(self.pages[i], self.scales))
        ptr = m.qo_indptr.tolist()
        for b in range(self.batch):
            self.kept[i][b] += [(k[r], v[r]) for r in range(ptr[b], ptr[b + 1])]

    def attends(self, b, q):
        """Attention of one row over the rows kept of request b, in 64 bits."""
        k = torch.stack([x[0] for x in self.kept[-1][b]]).double().permute(1, 2, 0).contiguous()
        v = torch.stack([x[1] for x in self.kept[-1][b]]).double().permute(1, 0, 2).contiguous()
        s = torch.matmul(q.double().view(HKV, HQ // HKV, 128), k) * SCALE
        return torch.matmul(torch.softmax(s, -1), v).view(HQ, 128)

    def answer(self, out, tokens):
        logits = torch.matmul(out.view(out.shape[0], -1), self.head)
        return logits, ra.token_logprobs(logits, tokens, top=3, stream=self.stream)


@pytest.mark.parametrize("fp8", [False, True], ids=["bf16", "fp8"])
def test_a_group_begins_answers_and_ends(fp8):
    """Two prompts, four attempts of each that end at different steps."""
    e = Engine(10, fp8)
    rng = np.random.default_rng(2)
    new = np.zeros(10, np.int64)
    new[[0, 5]] = 37, 64                                  # (the second prompt fills whole pages)
    tokens = dev(rng.integers(0, VOCAB, 101), torch.int64)
    e.rows(dev(new), tokens, True)
    ra.check_device_errors()
    # the attempts begin, one of them two tokens before the prompt's end
    parents = np.array([-1, 0, 0, 0, 0, -1, 5, 5, 5, 5])
    lens = np.where(parents < 0, 0, np.where(parents == 0, 37, 64))
    lens[2] = 35
    f = ra.fork_requests(dev(parents), dev(lens), e.lens, e.free, e.used, e.table, PAGE, POOL, kv_lens_out=e.lens,
                         free_used_out=e.used)
    for k, v in e.pages:
        ra.copy_pages(f.copies, k, v)
    assert e.lens.tolist() == [37, 37, 35, 37, 37, 64, 64, 64, 64, 64] and int(e.used) == 3 + 4 + 4
    for i in range(LAYERS):
        for b in np.flatnonzero(parents >= 0):
            e.kept[i][b] = e.kept[i][parents[b]][:lens[b]]
    live = parents >= 0
    token = dev(rng.integers(0, VOCAB, 8), torch.int64)
    for step in range(30):
        out = e.rows(dev(live.astype(np.int64)), token, False)
        q = e.layer[0]
        for r, b in enumerate(np.flatnonzero(live)):
            ref = e.attends(b, q[r])
            err = (out[r].double() - ref).abs().max()
            assert err <= H.MAX_ABS, (step, b, float(err))
        logits, a = e.answer(out, token)
        want = ends.token_logprobs(H.f64(logits), token.tolist(), None, 3)
        assert np.array_equal(a.top_ids.cpu().numpy(), want["top_ids"])
        assert np.abs(H.f64(a.logprobs) - want["logprobs"]).max() < 1e-4
        token = a.top_ids[:, 0].long()
        gone = live & (rng.random(10) < 0.08)
        if step == 29:
            gone = np.ones(10, bool)
        keep = np.where(gone, 0, 10 ** 9)
        ra.drop_tokens(e.lens, dev(keep), e.table, e.free, e.used, PAGE, POOL, kv_lens_out=e.lens,
                       free_used_out=e.used)
        token = token[dev(~gone[live], torch.bool)]
        live &= ~gone
        held = {int(p) for b, n in enumerate(e.lens.tolist()) for p in e.table[b, :-(-n // PAGE)].tolist()}
        listed = e.free[int(e.used):].tolist()
        assert len(set(listed)) == len(listed) == POOL - len(held) and not held & set(listed)
        if not live.any():
            break
    ra.check_device_errors()


def ops(seed, s):
    """One call of each operator on small inputs: name -> function that returns its outputs."""
    rng = np.random.default_rng(seed)
    q, k, v = rand(seed, 40, 8, 128), rand(seed + 1, 40, 2, 128), rand(seed + 2, 40, 2, 128)
    dq, dk = rand(seed + 3, 40, 8, 128), rand(seed + 4, 40, 2, 128)
    w = [rand(seed + 5, 128), rand(seed + 6, 128)]
    pos, freq = dev(rng.integers(0, 9000, (1, 40))), dev(1e4 ** (-np.arange(64) / 64), torch.float32)
    slots = dev(rng.permutation(64)[:40], torch.int64)
    pool = [torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    x, t = rand(seed + 7, 33, 9001, spread=3.0), dev(rng.integers(0, 9001, 33), torch.int64)
    g, h = rand(seed + 8, 33).float(), rand(seed + 9, 33).float()
    from tests.test_gpu_requests import drop_case, fork_case, pools

    fc, dc = fork_case(seed, 40, 200, 16), drop_case(seed, 40, 200, 16)
    fork = {n: dev(fc[n]) for n in ("parents", "fork_lens", "kv_lens", "free_pages", "block_table")}
    drop = {n: dev(dc[n]) for n in ("kv_lens", "keep_lens", "free_pages", "block_table")}
    f_used, d_used = dev(np.array([fc["free_used"]])), dev(np.array([dc["free_used"]]))
    pages = pools(seed, fc["num_pages"], 16, 2, False)

    def train():
        f = ra.token_logprobs(x, t, top=5, stream=s)
        return [*f, ra.token_logprobs_backward(x, t, f.lse, g, entropy=f.entropy, d_entropy=h, stream=s)]

    def append():
        return [ra.norm_rope_append_kv(q, k, v, *w, EPS, pos, freq, slots, *pool, stream=s), *pool]

    def forks():
        f = ra.fork_requests(fork["parents"], fork["fork_lens"], fork["kv_lens"], fork["free_pages"], f_used,
                             fork["block_table"], 16, fc["num_pages"], stream=s)
        ra.copy_pages(f.copies, *pages, stream=s)
        return [*f, fork["block_table"], *pages]

    def drops():
        d = ra.drop_tokens(drop["kv_lens"], drop["keep_lens"], drop["block_table"], drop["free_pages"], d_used, 16,
                           dc["num_pages"], stream=s)
        return [*d, drop["free_pages"]]

    return {"train": train, "append": append, "norm": lambda: list(ra.norm_rope(q, k, *w, EPS, pos, freq, stream=s)),
            "grad": lambda: list(ra.norm_rope_backward(dq, dk, q, k, *w, EPS, pos, freq, stream=s)), "fork": forks,
            "drop": drops}, (x, q, dq)


def reserve(stream):
    ra.reserve_workspace(max(ra.token_logprobs_workspace_size(33, 9001, 5), ra.norm_rope_backward_workspace_size()),
                         stream=stream)


@pytest.mark.parametrize("name", ["train", "append", "norm", "grad", "fork", "drop"])
def test_captured_calls_replay_among_eager_work(name):
    """Two graphs of one stream, replayed in turn with new inputs, eager calls of the same operator between them."""
    s = torch.cuda.Stream()
    reserve(s)
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        cases = [ops(i, s) for i in (3, 50)]
        s.synchronize()
        graphs = []
        for calls, _ in cases:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=s):
                out = calls[name]()
            graphs.append((graph, out))
        for turn in range(4):
            for (calls, inputs), (graph, out) in zip(cases, graphs):
                for i, x in enumerate(inputs):
                    x.copy_(rand(turn * 7 + i, *x.shape, spread=2.0))
                for o in out:
                    if o.dtype != torch.int32 and name != "fork":
                        o.zero_()
                graph.replay()
                s.synchronize()
                got = [o.clone() for o in out]
                want = [o.clone() for o in calls[name]()]
                assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, turn)
                torch.ones(1000, device=DEV).sum().item()
        ra.check_device_errors(s)


@pytest.mark.parametrize("name", ["train", "append", "norm", "grad", "fork", "drop"])
def test_streams_of_their_own(name):
    """The same calls on two other streams at once, with a workspace each, and on torch's current one."""
    want = [o.clone() for o in ops(7, None)[0][name]()]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    calls = [ops(7, s)[0][name] for s in streams]
    torch.cuda.synchronize()
    outs = []
    for _ in range(5):
        outs = []
        for s, call in zip(streams, calls):
            with torch.cuda.stream(s):
                outs.append(call())
    torch.cuda.synchronize()
    for s, out in zip(streams, outs):
        assert all(torch.equal(a, b) for a, b in zip(out, want)), name
        ra.check_device_errors(s)


def test_capture_needs_its_workspace_first():
    x, t = rand(1, 3, 70001), dev([1, 2, 3], torch.int64)
    s = torch.cuda.Stream()
    out = [torch.empty(3, device=DEV) for _ in range(3)]
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            with pytest.raises(ra.RlAttnError) as e:
                ra.token_logprobs(x, t, logprobs=out[0], entropy=out[1], lse=out[2], stream=s)
    assert e.value.status == "RL_ERR_WORKSPACE"
    ra.reserve_workspace(ra.token_logprobs_workspace_size(3, 70001), stream=s)
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            ra.token_logprobs(x, t, logprobs=out[0], entropy=out[1], lse=out[2], stream=s)
        for _ in range(3):
            graph.replay()
            s.synchronize()
    assert torch.equal(out[0], ra.token_logprobs(x, t).logprobs)


def test_tensors_elsewhere_are_refused():
    x, t = rand(1, 3, 701), dev([1, 2, 3], torch.int64)
    for args in ((x.cpu(), t), (x, t.cpu())):
        with pytest.raises(ValueError, match="current device"):
            ra.token_logprobs(*args, logprobs=torch.empty(3, device=DEV), entropy=torch.empty(3, device=DEV),
                              lse=torch.empty(3, device=DEV))
    k = torch.zeros(4, 16, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="current device"):
        ra.copy_pages(dev(np.array([[0, 1, 3]])), k, k)
