"""GPU: the operators around the paged cache run together, as a server runs them: prompts come in through the plan, the norm with the
append and the attention forward pass, then tokens are decoded one by one, requests end and others take their pages.  Every output is
compared with 64-bit causal attention over the request's whole history, recomputed from the projections.

The operands between the steps are rounded to 16 bits (queries, keys, values), and the reference takes the rounded ones that the steps
handed on, so what is compared is one attention with one rounding: the bar of the attention tests."""
import numpy as np
import pytest

from oracle import paged
from parity_util import MAX_ABS_TOL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Server:
    def __init__(self, B, width, page, pages, H, Hk, d, kind, layout, room):
        import torch
        self.B, self.page, self.H, self.Hk, self.d, self.kind, self.layout, self.room = B, page, H, Hk, d, kind, layout, room
        import paper_2601_16032_b200 as sa
        shape = (pages, Hk, page, d) if layout == sa.LAYOUT_BHND else (pages, page, Hk, d)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=kind, device=DEV) for _ in range(2))
        i32 = dict(dtype=torch.int32, device=DEV)
        self.table = torch.full((B, width), -1, **i32)
        self.free, self.count = torch.randperm(pages, device=DEV).to(torch.int32), torch.tensor([pages], **i32)
        self.length, self.added = torch.zeros(B, **i32), torch.zeros(B, **i32)
        self.wq, self.wk = ((1 + 0.2 * torch.randn(d, device=DEV)).to(kind) for _ in range(2))
        self.freq = (1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).to(DEV)
        self.qkv = torch.zeros((room, H + 2 * Hk, d), dtype=kind, device=DEV)
        self.workspace = torch.empty(sa.attn_decode_query_plan(B, H, Hk, d).workspace_bytes, dtype=torch.uint8, device=DEV)

    def plan(self):
        import paper_2601_16032_b200 as sa
        return sa.page_plan(self.length, self.added, self.page, self.table, self.free, self.count, self.room, seq_len=self.length, free_count_out=self.count)

    def append(self, p, k_out=None):
        import paper_2601_16032_b200 as sa
        H, Hk = self.H, self.Hk
        return sa.qk_norm_rope(self.qkv[:, :H], self.qkv[:, H:H + Hk], self.qkv[:, H + Hk:], q_weight=self.wq, k_weight=self.wk, position=p.position,
                               inv_freq=self.freq, k_cache=self.k, v_cache=self.v, cache_layout=self.layout, slot=p.slot, k_out=k_out)

    def decode(self, q):
        import paper_2601_16032_b200 as sa
        return sa.decode_paged(q, self.k, self.v, self.table, self.length, cache_layout=self.layout, return_lse=True, workspace=self.workspace)

    def history(self, b, n):
        """Keys and values of request b's first n tokens, out of the cache, [n, Hk, d] in 64 bits."""
        import paper_2601_16032_b200 as sa
        row = self.table[b].cpu().numpy()
        return tuple(paged.gather(c.double().cpu().numpy(), row, n, self.page, self.layout == sa.LAYOUT_BHND) for c in (self.k, self.v))


@pytest.mark.parametrize("layout,page,kind,d", [(1, 16, "bf16", 128), (0, 24, "f16", 64)])
def test_prompts_then_tokens(layout, page, kind, d):
    import torch
    import paper_2601_16032_b200 as sa
    kind = {"bf16": torch.bfloat16, "f16": torch.float16}[kind]
    torch.manual_seed(5)
    rng = np.random.default_rng(5)
    B, H, Hk, room = 4, 4, 2, 600
    s = Server(B, 12 * 16 // page + 4, page, 60 * 16 // page + 6, H, Hk, d, kind, layout, room)
    lengths = [0] * B
    told = {b: [] for b in range(B)}                   # (key, value) rows that each request was given, as projected

    def step(added):
        s.added.copy_(torch.tensor(added, dtype=torch.int32))
        s.qkv.normal_()
        p = s.plan()
        assert p.info[0] == 0 and p.info[1] == sum(a for a in added if a > 0)
        at = 0
        for b, a in enumerate(added):
            if a < 0:
                told[b], lengths[b] = [], 0
            for i in range(max(0, a)):
                told[b].append((s.qkv[at, H:H + Hk].clone(), s.qkv[at, H + Hk:].clone()))
                at += 1
            lengths[b] += max(0, a)
        assert s.length.tolist() == lengths
        return p, at

    def check_cache():
        for b in range(B):
            if not told[b]:
                continue
            keys, values = s.history(b, lengths[b])
            raw_k, raw_v = (torch.stack([row[i] for row in told[b]]).double().cpu().numpy() for i in (0, 1))
            want = paged.norm_rope(raw_k, s.wk.double().cpu().numpy(), 1e-6, range(lengths[b]), s.freq.tolist(), False)
            assert np.array_equal(values, raw_v)
            assert np.abs(keys - want).max() <= torch.finfo(kind).eps / 2 * np.abs(want).max() * 1.01

    # Prompts of one length go through the attention forward pass ([B, N, heads, d] is the order of the tokens), others would one by one.
    N = 130
    p, at = step([N] * B)
    q_out = torch.full((room, H, d), 3.0, dtype=kind, device=DEV)
    k_out = torch.full((room, Hk, d), 3.0, dtype=kind, device=DEV)
    sa.qk_norm_rope(s.qkv[:, :H], s.qkv[:, H:H + Hk], s.qkv[:, H + Hk:], q_weight=s.wq, k_weight=s.wk, position=p.position, inv_freq=s.freq, k_cache=s.k,
                    v_cache=s.v, cache_layout=s.layout, slot=p.slot, q_out=q_out, k_out=k_out)
    assert (q_out[at:] == 3).all() and (k_out[at:] == 3).all()
    q, k, v = q_out[:at].view(B, N, H, d), k_out[:at].view(B, N, Hk, d), s.qkv[:at, H + Hk:].contiguous().view(B, N, Hk, d)
    o = torch.empty_like(q)
    opts = sa.Opts()
    opts.layout, opts.kv_heads = sa.LAYOUT_BNHD, Hk
    sa.attn_fwd_ex(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), B, H, N, d, d ** -0.5, 1, sa.SAWTOOTH, sa.BF16 if kind == torch.bfloat16 else sa.F16,
                   torch.cuda.current_stream().cuda_stream, opts)
    sa.attn_device_status()
    check_cache()
    for b in range(B):
        keys, values = s.history(b, N)
        for i in (0, 1, 63, N - 1):
            want, _ = paged.decode(q[b, i].double().cpu().numpy(), keys[:i + 1], values[:i + 1], d ** -0.5)
            assert np.abs(o[b, i].double().cpu().numpy() - want).max() <= MAX_ABS_TOL
    # The last prompt token decoded from the pages is the same attention.
    last, _ = s.decode(q[:, -1])
    assert (last.double() - o[:, -1].double()).abs().max() <= MAX_ABS_TOL

    for turn in range(40):
        added = [1] * B
        if turn == 10:
            added[2] = -1                                # ends; its place stays empty for a while
        if 10 < turn < 15:
            added[2] = 0
        if turn == 15:
            added[2] = 70                                # a new prompt in its place, in pieces
        if turn == 30:
            added[0], added[3] = -1, 0
        if turn > 30:
            added[0] = int(rng.integers(0, 3))
        p, at = step(added)
        q_out, _ = s.append(p)
        # one query a request: the newest token's (an empty request's is anything)
        newest = (p.q_start[1:] - 1).long().clamp_min(0)
        q = q_out[newest].contiguous()
        o, lse = s.decode(q)
        sa.attn_device_status()
        for b in range(B):
            if lengths[b] == 0:
                assert (o[b] == 0).all() and torch.isneginf(lse[b]).all()
                continue
            keys, values = s.history(b, lengths[b])
            want, want_lse = paged.decode(q[b].double().cpu().numpy(), keys, values, d ** -0.5)
            assert np.abs(o[b].double().cpu().numpy() - want).max() <= MAX_ABS_TOL
            assert np.abs(lse[b].double().cpu().numpy() - want_lse).max() <= 5e-4
    check_cache()
    held = sum(paged.pages_of(n, page) for n in lengths)
    assert int(s.count) == s.free.numel() - held


def test_a_captured_decode_step():
    """Plan, norm with append and decode in one graph, replayed token after token; the same as the steps called one by one."""
    import torch
    import paper_2601_16032_b200 as sa
    kind, outs = torch.bfloat16, []
    for captured in (False, True):
        torch.manual_seed(9)
        s = Server(3, 8, 16, 30, 8, 2, 128, kind, sa.LAYOUT_BNHD, 3)
        s.added.fill_(1)

        def step():
            p = s.plan()
            q, _ = s.append(p)
            return s.decode(q)

        step()                                          # (outside the capture: first use of each entry point)
        s.length.zero_()
        s.count.fill_(30)
        s.free.copy_(torch.arange(30, dtype=torch.int32))
        torch.cuda.synchronize()
        if captured:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                out = step()
        got = []
        for turn in range(50):
            s.qkv.copy_(torch.randn(s.qkv.shape, generator=torch.Generator().manual_seed(turn)))
            s.added.copy_(torch.tensor([1, turn % 2, 0 if turn < 20 else 1], dtype=torch.int32))
            if captured:
                graph.replay()
                got.append([t.clone() for t in out])
            else:
                got.append(list(step()))
        sa.attn_device_status()
        outs.append(got)
    # A request that takes no token in a step has no query of its own: the rows of requests are the rows of the step's tokens only
    # where all of them take one.
    for turn, (a, b) in enumerate(zip(*outs)):
        if turn >= 20 and turn % 2:
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def _step_calls():
    """(name, inputs, call): each call's results depend on its inputs alone; pairs of calls share a workspace."""
    import torch
    import paper_2601_16032_b200 as sa
    torch.manual_seed(9)
    bf = torch.bfloat16
    made = []

    def rope(tokens, H, Hk, d, backward):
        q, k, gq, gk = (torch.randn(tokens, h, d, device=DEV).to(bf) for h in (H, Hk, H, Hk))
        w = torch.randn(d, device=DEV).to(bf)
        freq = (1e4 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).to(DEV)
        position = torch.arange(tokens, dtype=torch.int32, device=DEV)
        work = torch.empty(sa.attn_rope_bwd_workspace_bytes(d), dtype=torch.uint8, device=DEV)
        common = dict(q_weight=w, k_weight=w, position=position, inv_freq=freq)
        if backward:
            return [q, k, gq, gk], lambda: sa.qk_norm_rope_backward(gq, gk, q, k, workspace=work, **common)
        return [q, k, position], lambda: sa.qk_norm_rope(q, k, **common)

    def decode(B, longest, H, Hk, d):
        page = 16
        width = -(-longest // page)
        kc, vc = (torch.randn(B * width, page, Hk, d, device=DEV).to(bf) for _ in range(2))
        table = torch.arange(B * width, dtype=torch.int32, device=DEV).view(B, width)
        q = torch.randn(B, H, d, device=DEV).to(bf)
        length = torch.randint(1, longest + 1, (B,), device=DEV).to(torch.int32)
        work = torch.empty(sa.attn_decode_query_plan(B, H, Hk, d).workspace_bytes, dtype=torch.uint8, device=DEV)
        return [q, kc, vc, length], lambda: sa.decode_paged(q, kc, vc, table, length, return_lse=True, workspace=work)

    def plan(B):
        i32 = dict(dtype=torch.int32, device=DEV)
        cached, added = torch.randint(0, 50, (B,), **i32), torch.randint(0, 3, (B,), **i32)
        table, free = torch.arange(B * 8, **i32).view(B, 8), torch.arange(B * 8, B * 12, **i32)
        count = torch.tensor([B * 4], **i32)
        return [cached, added, table, free, count], lambda: sa.page_plan(cached, added, 16, table, free, count, 2 * B)

    for name, (inputs, call) in dict(plan=plan(300), rope=rope(700, 8, 2, 64, False), rope_bwd=rope(700, 8, 2, 64, True), rope_bwd_small=rope(5, 4, 2, 128, True),
                                     decode=decode(30, 2000, 8, 2, 128), decode_short=decode(4, 200, 8, 2, 64)).items():
        made.append((name, inputs, call))
    return made


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("before", ["kernel", "copy", "kernel on another stream", "copy on another stream"])
def test_steps_wait_for_what_comes_before_them(before, captured):
    """The kernels start behind one that has not ended: inputs that a late kernel, a copy or another stream writes, overwritten again behind
    the call, and a second call with other inputs in the same workspace."""
    import torch
    busy = torch.randn(3000, 3000, device=DEV)
    for name, inputs, call in _step_calls():
        good = [[t.clone() for t in inputs]]
        # The second inputs: rows in another order (lengths and positions stay within what their tables hold).
        good.append([t.clone() if name == "plan" else t.flip(0).contiguous() for t in inputs])
        want = []
        for g in good:
            for t, x in zip(inputs, g):
                t.copy_(x)
            torch.cuda.synchronize()
            want.append([o.clone() for o in call() if o is not None] + ([inputs[2].clone(), inputs[3].clone()] if name == "plan" else []))
            torch.cuda.synchronize()
        got = []

        def late():
            y = busy
            for _ in range(4):
                y = torch.sin(y) @ busy
            return y

        def run():
            got.clear()
            main, side = torch.cuda.current_stream(), torch.cuda.Stream()
            for g in good:
                side.wait_stream(main)
                with torch.cuda.stream(side if "another" in before else main):
                    late()
                    for t, x in zip(inputs, g):
                        if "copy" in before:
                            t.copy_(x)
                        else:
                            torch.add(x, 0, out=t)
                main.wait_stream(side)
                if "copy on another" in before:   # one more kernel between the wait and the call; behind a kernel none
                    busy.add_(0)
                out = [o for o in call() if o is not None] + ([inputs[2].clone(), inputs[3].clone()] if name == "plan" else [])
                for t in inputs:
                    t.zero_()
                got.append(out)

        if captured:
            warm = torch.cuda.Stream()
            warm.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(warm):
                run()
            torch.cuda.current_stream().wait_stream(warm)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                run()
            for _ in range(3):
                graph.replay()
        else:
            run()
        torch.cuda.synchronize()
        for turn in range(2):
            for i, (a, b) in enumerate(zip(got[turn], want[turn])):
                assert torch.equal(a.view(torch.uint8) if a.dim() else a, b.view(torch.uint8) if b.dim() else b), (name, turn, i)
