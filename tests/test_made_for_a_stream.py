"""Tensors that a call makes for the stream it works on.  The caching allocator hands a freed block out again at once to the stream that
it belongs to: a block for another stream has to come from that stream's memory, and a result that the caller goes on with has
to be known to the caller's stream, too.  On the CPU, with stand-ins for torch's streams; on the GPU by where the blocks lie."""
import contextlib

import pytest
import torch

import paper_2601_17917_amd as sd


class FakeTensor:
    def __init__(self, stream):
        self.made_on, self.used_on = stream, []

    def record_stream(self, stream):
        self.used_on.append(stream)


@pytest.fixture
def streams(monkeypatch):
    now = ["caller's"]

    @contextlib.contextmanager
    def on(stream):
        now.append(stream)
        yield
        now.pop()

    monkeypatch.setattr(torch.cuda, "stream", on)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: now[-1])
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: FakeTensor(now[-1]))


@pytest.mark.parametrize("stream", [None, "caller's", "another"])
def test_a_block_belongs_to_the_stream_that_works_on_it(streams, stream):
    t = sd._new((4,), torch.uint8, "cuda", stream)
    assert t.made_on == (stream or "caller's")
    assert {t.made_on, *t.used_on} == {"caller's", stream or "caller's"}


def owner(t):
    """The stream that the memory of a tensor belongs to."""
    for seg in torch.cuda.memory_snapshot():
        if seg["address"] <= t.data_ptr() < seg["address"] + seg["total_size"]:
            return seg["stream"]
    raise AssertionError("not the allocator's")


@pytest.mark.gpu
@pytest.mark.parametrize("what", ["attention", "norm_rope", "extend", "extend in two launches"])
def test_results_and_workspaces_of_the_paged_calls(gpu_lib, what):
    """With work queued on the caller's stream over blocks of the same sizes that are free by now."""
    i32 = dict(dtype=torch.int32, device="cuda")
    B, K, Hq, Hkv, D, page, n_pages = 3, 2, 8, 2, 128, 16, 1800
    g = torch.Generator(device="cuda")
    g.manual_seed(51)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)

    def inputs():
        """A call with inputs of its own, the number of tensors that it returns and has made."""
        g.manual_seed(52)
        q, k, kp, vp = draw(B, Hq, K, D), draw(B, Hkv, K, D), draw(n_pages, Hkv, page, D), draw(n_pages, Hkv, page, D)
        table = torch.randperm(n_pages, generator=g, device="cuda")[:B * 600].to(torch.int32).view(B, 600)
        lens, n_free = torch.tensor([3400, 17, 900], **i32), torch.tensor([1500], **i32)
        free = torch.arange(n_pages, **i32)
        if what == "attention":
            return (lambda **kw: gpu_lib.bind_paged_attention(q, kp, vp, table, lens, 3500, causal=True, **kw)), 1
        if what == "norm_rope":
            return (lambda **kw: gpu_lib.bind_qk_norm_rope(q, k, lens, 1e4, **kw)), 2
        rows = 3 if what == "extend" else 6000
        return (lambda **kw: gpu_lib.bind_paged_extend(table, lens, free, n_free, page, rows, **kw)), 2

    def made(bind, n, **kw):
        call = bind(**kw)
        call()
        torch.cuda.synchronize()
        return (call.result if isinstance(call.result, tuple) else (call.result,))[:n], call

    want = [t.clone() for t in made(*inputs())[0]]
    bind, n = inputs()
    big = torch.randn((4096, 4096), device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        big = (big @ big).clamp_(-1, 1)
    held = [torch.empty_like(t).fill_(1) for t in want for _ in range(3)] + [torch.ones(1 << 20, dtype=torch.uint8, device="cuda")]
    del held
    results, call = made(bind, n, stream=side)
    assert all(torch.equal(x, y) for x, y in zip(results, want))
    workspace = call._keep[2] if len(call._keep) > 2 else None
    assert (workspace is not None) == (what in ("attention", "extend in two launches"))
    assert all(owner(t) == side.cuda_stream for t in (*results, workspace) if t is not None)


@pytest.mark.gpu
def test_results_and_workspaces_of_the_step(gpu_lib):
    """The calls of a decode step over the dense cache: same results, and all that they make belongs to the stream they work on."""
    g = torch.Generator(device="cuda")
    g.manual_seed(53)
    draw = lambda *shape: torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)
    B, K, V, Hd = 2, 32, 1000, 256
    q, k, cache = draw(B, 4, K, 128), draw(B, 4, K, 128), draw(B, 4, 4096, 128)
    none = (None, None, None)
    logits, hidden, weight = draw(B, K, V), draw(B, K, Hd), draw(V, Hd)
    state = lambda: (torch.zeros((B, K), dtype=torch.int32, device="cuda"), torch.ones((B, K), dtype=torch.uint8, device="cuda"))
    calls = {"attention": lambda st, **kw: gpu_lib.bind_block_attention(q, None, cache, cache, k, k, *none, 4096, **kw),
             "unmask": lambda st, **kw: gpu_lib.bind_confidence_unmask(logits, *st, 0.9, 0.5, **kw),
             "unmask, no workspace": lambda st, **kw: gpu_lib.bind_confidence_unmask_noalloc(logits, *st, 0.9, 0.5, **kw),
             "projection": lambda st, **kw: gpu_lib.bind_lm_head_unmask(hidden, weight, *st, 0.9, 0.5, **kw)}
    side = torch.cuda.Stream()
    for name, bind in calls.items():
        first, again = state(), state()
        call = bind(first)
        want = call()
        torch.cuda.synchronize()
        call = bind(again, stream=side)
        got = call()
        torch.cuda.synchronize()
        want, got = (x if isinstance(x, tuple) else (x,) for x in (want, got))
        assert all(torch.equal(x, y) for x, y in zip((*first, *want), (*again, *got))), name
        workspace = call._keep[-1] if name != "unmask, no workspace" else None
        assert all(owner(t) == side.cuda_stream for t in (*got, workspace) if t is not None), name
    packed = gpu_lib.lm_head_pack_weight(weight, stream=side)
    torch.cuda.synchronize()
    assert owner(packed.data) == side.cuda_stream and torch.equal(packed.data, gpu_lib.lm_head_pack_weight(weight).data)
