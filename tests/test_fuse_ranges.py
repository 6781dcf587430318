"""The rows of a fused table's members, which a projection of each table's own goes by: written on the device in the call that maps the
lookups, so that calls of other batch sizes, captured ones and other threads' do not share them."""
import ctypes
import threading

import pytest
import torch

SHAPES = [(60, (3, 4, 5)), (200, (5, 8, 5)), (24, (2, 3, 4))]


def test_arguments_are_checked_before_any_launch():
    from paper_2507_14668_amd import binding
    lib = binding.load_library()
    layout = binding.FusedLayout(SHAPES[:1])
    ptr, i64 = (ctypes.c_void_p * 1)(256), lambda v: (ctypes.c_int64 * 1)(v)
    call = lambda idx, off, nnz, bags, ranges=256, starts=0: lib.tt_fuse_lookups_ranges(ctypes.byref(layout.c), idx, off, starts, None, i64(nnz), i64(bags),
                                                                                         256, 256, ranges, None)
    assert call(ptr, ptr, 3, 2, None) == binding.TT_ERR_INVALID_ARG
    assert call(ptr, ptr, 3, 0) == binding.TT_ERR_INVALID_ARG            # lookups without a bag
    assert call(ptr, (ctypes.c_void_p * 1)(), 3, 2, 256, 1) == binding.TT_ERR_INVALID_ARG
    assert call((ctypes.c_void_p * 1)(), ptr, 3, 2) == binding.TT_ERR_INVALID_ARG


def bags(seed, counts):
    gen = torch.Generator().manual_seed(seed)
    out = []
    for (rows, _), n in zip(SHAPES, counts):
        lens = torch.randint(0, 4, (n,), generator=gen)
        off = torch.zeros(n, dtype=torch.int64)
        off[1:] = lens.cumsum(0)[:-1]
        out.append((torch.randint(0, rows, (int(lens.sum()),), generator=gen).cuda(), off.cuda()))
    return out


@pytest.fixture
def module():
    import paper_2507_14668_amd as tt
    m = tt.TTFusedEmbeddingBags(SHAPES, 16, (2, 2, 4), (4, 4), projection=40, projection_activation="relu",
                                generator=torch.Generator(device="cuda").manual_seed(1))
    with torch.no_grad():
        m.projection.bias.normal_(0, 1, generator=torch.Generator(device="cuda").manual_seed(2))
    return m


def by_table(m, inputs):
    """The same outputs with one product a table, by no offsets at all."""
    import paper_2507_14668_amd as tt
    projection, m.projection = m.projection, None
    pooled = m(inputs)
    m.projection = projection
    return [tt.tt_dense(p, projection.weight[t], projection.bias[t], activation="relu") for t, p in enumerate(pooled)]


@pytest.mark.gpu
@pytest.mark.parametrize("counts", [(1, 1, 1), (17, 0, 300), (0, 0, 5), (700, 41, 9)])
def test_ranges(counts):
    from paper_2507_14668_amd import binding
    layout = binding.FusedLayout(SHAPES)
    inputs = bags(0, counts)
    idx, off = [i for i, _ in inputs], [o for _, o in inputs]
    for starts, offs in ((True, off), (False, [torch.cat([o, torch.tensor([i.numel()], device="cuda")]) for i, o in inputs])):
        ranges = torch.full((4,), -7, dtype=torch.int64, device="cuda")
        got = layout.fuse_lookups(idx, offs, starts=starts, ranges=ranges)
        want = layout.fuse_lookups(idx, offs, starts=starts)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert ranges.tolist() == [0, counts[0], counts[0] + counts[1], sum(counts)]
    with pytest.raises(ValueError):
        layout.fuse_lookups(idx, off, starts=True, ranges=ranges[:3])
    with pytest.raises(TypeError):
        layout.fuse_lookups(idx, off, starts=True, ranges=ranges.int())


@pytest.mark.gpu
def test_a_captured_call_beside_calls_of_other_sizes(module):
    """Captured (also with counts that no call had before), then eager calls of other sizes, whose memory is written over."""
    with torch.no_grad():
        first, other = bags(1, (40, 7, 90)), bags(2, (3, 80, 11))
        want, want_other = [t.clone() for t in by_table(module, first)], [t.clone() for t in by_table(module, other)]
        assert all(torch.equal(a, b) for a, b in zip(module(first), want))
        for warm in (True, False):
            if warm:
                side = torch.cuda.Stream()
                side.wait_stream(torch.cuda.current_stream())
                with torch.cuda.stream(side):
                    module(first)
                torch.cuda.current_stream().wait_stream(side)
            else:
                module(other)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                held = module(first)
            for i in range(3):
                assert all(torch.equal(a, b) for a, b in zip(module(other), want_other)), i
                filled = [torch.full((4,), 10 ** 6, dtype=torch.int64, device="cuda") for _ in range(50)]
                for t in held:
                    t.fill_(-1.0)
                torch.cuda.synchronize()
                graph.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(held, want)), (warm, i)
                del filled


@pytest.mark.gpu
def test_two_threads_with_other_sizes(module):
    inputs = [bags(3, (40, 7, 90)), bags(4, (3, 80, 11))]
    with torch.no_grad():
        wants = [[t.clone() for t in by_table(module, x)] for x in inputs]
    torch.cuda.synchronize()
    wrong = []

    def work(x, want):
        with torch.no_grad(), torch.cuda.stream(torch.cuda.Stream()):
            for i in range(60):
                got = module(x)
                torch.cuda.current_stream().synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got, want)):
                    wrong.append(i)
    threads = [threading.Thread(target=work, args=args) for args in zip(inputs, wants)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
