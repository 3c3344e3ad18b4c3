"""DecodeStep: calls over span lists before, between and behind the calls around a budget."""
import pytest
import torch

from paper_2404_09336_b200 import inputs
from paper_2404_09336_b200.runner import DecodeStep

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("budget", [3, 64, 460, 512])
def test_steps_over_spans_are_as_without_a_budget(budget):
    ds = DecodeStep(inputs.make_config(1), out_dtype=torch.float32)
    calls = (ds.step, ds.step_two_calls, ds.attend_spans, lambda: ds.attend_spans(want_lists=True))
    want = []
    for call in calls:
        call()
        want.append((ds.out.clone(), ds.lse.clone(), ds.counts.clone(), ds.index.clone()))
    for call, (out, lse, counts, index) in zip(calls, want):
        ds.attend_mass()
        ds.select_heaviest(budget)
        ds.attend_sparse()
        ds.out.fill_(9)
        call()
        torch.cuda.synchronize()
        assert torch.equal(ds.out, out) and torch.equal(ds.lse, lse) and int(ds.status) == 0
        if call is not calls[2]:
            assert torch.equal(ds.counts, counts) and torch.equal(ds.index, index)


def test_budgets_of_any_size_are_attended_to():
    ds = DecodeStep(inputs.make_config(2, B=3, H=4), out_dtype=torch.float32)
    ds.attend_mass()
    ds.attend_dense()
    whole, ctx = ds.out.clone(), ds.ctx_lens.tolist()
    for budget in (5, 200, 1000, 1024, 5000):
        ds.select_heaviest(budget, sinks=2, recent=3)
        ds.attend_sparse()
        torch.cuda.synchronize()
        assert ds.counts.tolist() == [min(n, budget) for n in ctx] and int(ds.status) == 0
        if budget >= max(ctx):
            assert (ds.out - whole).abs().max() < 1e-5


def test_captured_steps_keep_their_buffers():
    """Graphs of a step, of a window and of an attention through a budget's lists, replayed behind calls that need more room."""
    ds = DecodeStep(inputs.make_config(2, B=2, H=4), out_dtype=torch.float32)
    ds.attend_mass()
    mass = ds.mass.clone()
    ds.select_heaviest(40)
    calls, graphs, want = (ds.step, lambda: ds.attend_window(9), ds.attend_sparse), [], []
    for call in (calls[2], calls[1], calls[0]):              # (a step puts its own lists in place)
        call()
        want.append(ds.out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append(graph)
    sizes = {ds.workspace.numel(), *(x.numel() for x in ds._rooms)}
    with pytest.MonkeyPatch.context() as m:
        from paper_2404_09336_b200 import ssa
        need = 3 * max(sizes)
        m.setattr(ssa, "attn_mass_workspace_bytes", lambda *a: need)
        ds.attend_mass()
    ds.select_heaviest(ds.index_stride + 200)
    poison = [torch.full((n,), 0xff, dtype=torch.uint8, device=ds.device) for n in sizes for _ in range(4)]
    for graph, out in zip(graphs, want):
        ds.out.fill_(9)
        if out is want[0]:
            ds.mass.copy_(mass)
            ds.select_heaviest(40)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ds.out, out)
    assert all(bool((x == 0xff).all()) for x in poison)      # nothing wrote where others' memory is by now


def test_first_calls_on_a_side_stream_and_in_a_graph():
    """Sums start from zero once: not behind the call that adds to them, and not with every replay."""
    wl = inputs.make_config(2, B=2, H=4)
    want = DecodeStep(wl, out_dtype=torch.float32)
    for _ in range(3):
        want.attend_mass()
    torch.cuda.synchronize()
    ds, side = DecodeStep(wl, out_dtype=torch.float32), torch.cuda.Stream()
    busy = torch.randn(8192, 8192, device=ds.device)
    torch.cuda.synchronize()
    for _ in range(8):                                       # the current stream is behind the side stream by this
        busy = busy @ busy * 1e-4
    for _ in range(3):
        ds.attend_mass(stream=side)
    ds.select_heaviest(ds.index_stride + 100, stream=side)
    ds.attend_sparse(stream=side)
    torch.cuda.synchronize()
    assert torch.equal(ds.mass, want.mass)
    want.select_heaviest(ds.index_stride + 100)
    want.attend_sparse()
    torch.cuda.synchronize()
    assert torch.equal(ds.index, want.index) and torch.equal(ds.counts, want.counts) and torch.equal(ds.out, want.out)
    ds, graph = DecodeStep(wl, out_dtype=torch.float32), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ds.attend_mass()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(ds.mass, want.mass)


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_all_copies_of_a_compacted_cache_are_alike(layout):
    ds = DecodeStep(inputs.make_config(2, B=3, H=4), layout=layout, kv_copies=2, out_dtype=torch.float32)
    ds.attend_mass()
    ds.select_heaviest(50, sinks=3, recent=9)
    mass, index = ds.mass.clone(), ds.index[:, :50].clone()
    ds.compact()
    got = []
    for c in range(2):
        ds.select_copy(c)
        ds.attend_dense()
        got.append(ds.out.clone())
    torch.cuda.synchronize()
    assert torch.equal(got[0], got[1]) and int(ds.status) == 0 and ds.ctx_lens.tolist() == ds.counts.tolist()
    for b, n in enumerate(ds.counts.tolist()):
        assert torch.equal(ds.mass[b, :n], mass[b, index[b, :n].long()])
