"""Copies of what a cache holds: moved tokens and copied blocks, in every bit."""
import pytest
import torch

from tests.test_gpu_kv_store import _data, _same, kv  # noqa: F401 (fixture)

pytestmark = pytest.mark.gpu


def _filled(kv, blocks, H, D, fmt, seed=0):
    """A cache whose slots are all written, and a vector of them."""
    c = kv.KVCache(blocks, H, D, fmt=fmt)
    k, v = _data(blocks * 16, H, D, "fp32", seed)
    every = torch.arange(blocks * 16, device="cuda")
    c.write(k, v, every)
    return c, every


SHAPES = [("bf16", 8, 128), ("fp8", 8, 128), ("fp16", 3, 64), ("fp8", 1, 64), ("bf16", 5, 64), ("fp8", 3, 128)]


@pytest.mark.parametrize("fmt,H,D", SHAPES)
@pytest.mark.parametrize("n", [1, 2, 31, 127, 500, 2048, 2049, 5000])
def test_moves_are_as_if_all_were_read_first(kv, fmt, H, D, n):
    """Slots that change places at random: chains, cycles, one source for several, some cleared, some skipped."""
    blocks = n // 16 + 20
    c, every = _filled(kv, blocks, H, D, fmt, n)
    before = c.read(every, dtype=torch.float32)
    g = torch.Generator(device="cuda").manual_seed(n)
    dst = torch.randperm(blocks * 16, device="cuda", generator=g)[:n].contiguous()
    src = dst[torch.randperm(n, device="cuda", generator=g)]  # mostly other moves' destinations
    far = torch.rand(n, device="cuda", generator=g)
    src = torch.where(far < 0.3, torch.randint(0, blocks * 16, (n,), device="cuda", generator=g), src)
    src[far > 0.9] = -3
    dst[(far > 0.45) & (far < 0.55)] = -1
    c.move(src, dst)
    c.check()
    after = c.read(every, dtype=torch.float32)
    live = dst >= 0
    for x, y in zip(before, after):
        want = x.clone()
        want[dst[live]] = torch.where((src < 0)[:, None, None], 0.0, x[src.clamp(min=0)])[live]
        _same(y, want)
    c.close()


@pytest.mark.parametrize("n", [40, 3000])
def test_moves_outside_the_cache_are_skipped_and_reported(kv, n):
    import paper_2609_33224_gb300 as P
    c, every = _filled(kv, 200, 2, 64, "fp8")
    before = c.read(every, dtype=torch.float32)
    dst = torch.arange(n, device="cuda")
    src = (dst + 7) % n
    src[5], dst[9], src[11], dst[12] = 3200, 3200, 1 << 60, 1 << 40
    c.move(src, dst)
    with pytest.raises(P.PSError, match="outside the cache"):
        c.check()
    c.check()
    after = c.read(every, dtype=torch.float32)
    ok = torch.ones(n, dtype=torch.bool, device="cuda")
    ok[[5, 9, 11, 12]] = False
    for x, y in zip(before, after):
        want = x.clone()
        want[dst[ok]] = x[src[ok]]
        _same(y, want)
    c.close()


@pytest.mark.parametrize("fmt,H,D", SHAPES)
@pytest.mark.parametrize("between", [False, True])
@pytest.mark.parametrize("n", [1, 7, 300])
def test_copied_blocks(kv, fmt, H, D, between, n):
    """Forks (one block to several places), hand-over to another cache, cleared and skipped blocks; the rest stays."""
    c, every = _filled(kv, 2 * n + 9, H, D, fmt, n)
    other, _ = _filled(kv, n + 3, H, D, fmt, n + 1) if between else (c, None)
    before = c.read(every, dtype=torch.float32)
    given = other.read(torch.arange(other.num_blocks * 16, device="cuda"), dtype=torch.float32)
    perm = torch.randperm(c.num_blocks, device="cuda")
    dst = perm[:n].contiguous()
    src = torch.randint(0, other.num_blocks, (n,), device="cuda") if between else perm[n:][torch.randint(0, n, (n,), device="cuda")]
    if n > 3:
        src[2], dst[3] = -1, -5
    c.copy_blocks(src, dst, source=other if between else None)
    c.check()
    after = c.read(every, dtype=torch.float32)
    for x, y, z in zip(before, after, given):
        want, z = x.clone().view(-1, 16, H, D), z.view(-1, 16, H, D)
        for i in range(n):
            if dst[i] >= 0:
                want[dst[i]] = z[src[i]] if src[i] >= 0 else 0.0
        _same(y, want.view_as(y))
    if between:
        for x, y in zip(given, other.read(torch.arange(other.num_blocks * 16, device="cuda"), dtype=torch.float32)):
            _same(x, y)
        other.close()
    c.close()


def test_blocks_outside_a_cache_are_skipped_and_reported(kv):
    import paper_2609_33224_gb300 as P
    c, every = _filled(kv, 10, 2, 64, "bf16")
    with kv.KVCache(4, 2, 64) as small:
        before = c.read(every)
        src, dst = torch.tensor([3, 4, 1 << 40, 2], device="cuda"), torch.tensor([10, 1, 2, 1 << 40], device="cuda")
        c.copy_blocks(src, dst, source=small)
        with pytest.raises(P.PSError, match="outside the cache"):
            c.check()
        for x, y in zip(before, c.read(every)):
            _same(x, y)
        small.check()
    c.close()


def test_offsets_past_32_bits(kv):
    """A cache of more than 2^32 bytes: its last blocks and slots."""
    H, D, blocks = 8, 128, 150000
    with kv.KVCache(blocks, H, D, fmt="fp8") as c:
        k, v = _data(64, H, D, "bf16", 4)
        top = torch.arange(blocks * 16 - 64, blocks * 16, device="cuda")
        c.write(k, v, top)
        want = c.read(top)
        ids = torch.arange(blocks - 4, blocks, device="cuda")
        c.copy_blocks(ids, torch.arange(4, device="cuda"))
        c.copy_blocks(torch.arange(4, device="cuda"), ids - 9)
        c.move(top, top - 50000)
        c.check()
        for at in (torch.arange(64, device="cuda"), top - 9 * 16, top - 50000, top):
            for x, y in zip(c.read(at), want):
                _same(x, y)


def test_captured_and_on_another_stream(kv):
    """Replays after the caches are gone, beside calls on another stream."""
    H, D, n = 2, 64, 3000
    a, every = _filled(kv, 400, H, D, "fp8", 1)
    b, _ = _filled(kv, 400, H, D, "fp8", 2)
    k, v = _data(6400, H, D, "fp32", 3)
    src, dst = torch.randperm(6400, device="cuda")[:n].contiguous(), torch.randperm(6400, device="cuda")[:n].contiguous()
    few, to = src[:100].contiguous(), dst[:100].contiguous()
    blocks = torch.randperm(400, device="cuda")

    def step(c, source, **kw):
        c.write(k, v, every)
        c.move(src, dst)
        c.move(few, to)
        c.copy_blocks(blocks[:200], blocks[200:], source=source)
        return c.read(every, **kw)

    want = step(a, b, dtype=torch.float32)
    a.check()
    ko, vo = torch.empty_like(want[0]), torch.empty_like(want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, b, k=ko, v=vo)
    d, _ = _filled(kv, 400, H, D, "fp8", 4)
    e, _ = _filled(kv, 400, H, D, "fp8", 2)
    a.close()
    b.close()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        graph.replay()
        with torch.cuda.stream(s):
            got = step(d, e, dtype=torch.float32)
        torch.cuda.synchronize()
        for x, y, z in zip((ko, vo), want, got):
            _same(x, y)
            _same(z, y)
        ko.zero_()
    d.check()
    d.close()
    e.close()


def test_refusals(kv):
    import paper_2609_33224_gb300 as P
    i = torch.arange(4, device="cuda")
    with kv.KVCache(8, 2, 64) as c:
        for call in (c.move, c.copy_blocks):
            for bad in (i[:3], i.int(), i.cpu(), i[::2], i[None]):
                with pytest.raises(ValueError):
                    call(i, bad)
                with pytest.raises(ValueError):
                    call(bad, i)
            call(i[:0], i[:0])
        for H, D, fmt in ((3, 64, "bf16"), (2, 128, "bf16"), (2, 64, "fp16"), (2, 64, "fp8")):
            with kv.KVCache(8, H, D, fmt=fmt) as other:
                with pytest.raises(P.PSError, match="between caches"):
                    c.copy_blocks(i, i, source=other)
        with pytest.raises(ValueError, match="closed"):
            c.copy_blocks(i, i, source=other)
        c.check()
    for call in (c.move, c.copy_blocks):
        with pytest.raises(ValueError, match="closed"):
            call(i, i)
