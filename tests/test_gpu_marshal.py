"""The compiled checks of the cache's calls and window_attention against the methods' own: the same results, the same refusals."""
import pytest
import torch

from test_gpu_verifier import BF, Q8, _cache, _graft, _i32

pytestmark = pytest.mark.gpu


def _inputs(dtype):
    from paper_2608_20375_b200 import Rope
    gen = torch.Generator(device="cuda").manual_seed(3)
    B, rows, Hq, Hk, D, page = 2, 9, 8, 2, 64, 16
    g = _graft(16, B)
    c = _cache(gen, (2, 40, Hk, page, D), dtype, garbage=False)
    qkv = torch.randn((B, rows, (Hq + 2 * Hk) * D), generator=gen, device="cuda").to(BF)
    q, key, value = (t.unflatten(2, (-1, D)) for t in qkv.split([Hq * D, Hk * D, Hk * D], 2))
    mask = torch.full((B, g.nmax, g.mask_words), -1, dtype=torch.int32, device="cuda")
    pos = torch.arange(g.nmax, dtype=torch.int32, device="cuda").expand(B, -1) + _i32([[29], [4]])
    return g, dict(cache=c, layer=1, table=torch.arange(40, dtype=torch.int32, device="cuda").view(B, 20), prefix_len=_i32([30, 5]), count=_i32([9, 4]),
                   rope=Rope.of(64, gain=1.5), q=q, key=key, value=value, q_out=torch.zeros_like(q, memory_format=torch.contiguous_format),
                   position=pos.contiguous(), status=_i32([7, 7]), mask=mask, window=20, sinks=2, out=torch.zeros(q.shape, dtype=BF, device="cuda"),
                   lse=torch.zeros(q.shape[:3], device="cuda"), scale=None)


APPEND = "cache layer table prefix_len count rope q key value q_out position status".split()
ROWS = "cache layer table prefix_len count key value status".split()
ATTEND = "cache layer table q prefix_len count mask position window sinks out lse scale status".split()


@pytest.mark.parametrize("dtype", [BF, Q8])
def test_results_are_the_same(dtype, monkeypatch):
    from paper_2608_20375_b200 import binding
    binding.load_library()
    fast = binding._fast
    assert fast is not None
    got = []
    for way in (fast, None):
        monkeypatch.setattr(binding, "_fast", way)
        g, a = _inputs(dtype)
        a["cache"].k.zero_(), a["cache"].v.zero_()
        g.cache_append(*(a[x] for x in APPEND))
        a["status"].fill_(7)
        g.cache_write(*((a | dict(prefix_len=_i32([60, 70])))[x] for x in ROWS))
        back = torch.zeros((2, 9, 2, 64), dtype=BF, device="cuda")
        g.cache_read(*((a | dict(key=back, value=torch.zeros_like(back), prefix_len=_i32([59, 70]), status=None))[x] for x in ROWS))
        g.window_attention(**{x: a["q_out"] if x == "q" else a[x] for x in ATTEND})
        for change in (dict(q=None, q_out=None), dict(position=None), dict(position=a["position"][:, :9, None].contiguous()), dict(q_out=None)):
            g.cache_append(*((a | change | dict(layer=0))[x] for x in APPEND))
        first = a["out"].clone()
        for change in (dict(mask=None, position=None), dict(scale=0.3, lse=None), dict(status=None), dict(window=2 ** 40)):
            g.window_attention(**{x: (a | change)[x] for x in ATTEND})
            first = first + a["out"]
        got.append([a["cache"].k, a["cache"].v, a["q_out"], first, a["lse"], a["status"], a["q"], back])
    for x, y in zip(*got):
        assert torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))


def test_refusals_are_the_same(monkeypatch):
    """Whatever is wrong with one argument, the method says it; nothing is written."""
    from paper_2608_20375_b200 import GraftError, KVCache, Rope, binding
    g, a = _inputs(BF)
    fast = binding._fast
    before = a["cache"].k.clone()
    cpu, wide = a["q"].cpu(), torch.zeros((2, 9, 8, 128), dtype=BF, device="cuda")
    strided = torch.zeros((2, 9, 8, 128), dtype=BF, device="cuda")[..., ::2]
    c = a["cache"]
    wrong = [dict(layer=2), dict(layer=-1), dict(table=a["table"].long()), dict(table=a["table"][:1]), dict(prefix_len=_i32([1])), dict(count=None),
             dict(prefix_len=a["prefix_len"].cpu()), dict(q=cpu), dict(q=wide), dict(q=strided), dict(q=a["q"].float()), dict(status=_i32([1])),
             dict(cache=KVCache(c.k.float(), c.v)), dict(cache=KVCache(c.k, c.v[:1])), dict(cache=KVCache(c.k[0], c.v[0])),
             dict(cache=KVCache(c.k, c.v, _i32([1]))), dict(position=a["position"].long()), dict(position=a["position"][:1])]
    append = [dict(key=a["key"][:, :3]), dict(value=a["value"].contiguous()), dict(q_out=wide), dict(q=None), dict(position=a["position"][:, :4]),
              dict(rope=Rope(a["rope"].freq.double())), dict(rope=Rope(a["rope"].freq[:, :4].contiguous())), dict(rope=Rope(a["rope"].freq, shift=_i32([1]))),
              dict(rope=Rope(a["rope"].freq[0])), dict(rope=Rope(a["rope"].freq, gain=float("nan")))]
    attend = [dict(mask=None), dict(position=None), dict(window=0), dict(sinks=-1), dict(out=wide), dict(lse=a["lse"].double()), dict(mask=a["mask"][:, :3]),
              dict(scale=float("inf")), dict(scale=float("nan"))]
    rows = [dict(key=a["key"][:, :3]), dict(key=cpu), dict(value=wide), dict(key=a["key"].float()), dict(value=a["value"][0]), dict(value=a["value"][:1])]
    shared = [c for c in wrong if not {"q", "position"} & set(c)]
    dense = dict(key=a["key"].contiguous(), value=a["value"].contiguous())
    for call, names, changes in ((g.cache_append, APPEND, wrong + append), (g.window_attention, ATTEND, wrong + attend),
                                 (g.cache_write, ROWS, shared + rows + [dict(value=dense["value"])]),
                                 (g.cache_read, ROWS, [dense | c for c in shared + rows] + [dict(key=a["key"])])):
        for change in changes:
            said = []
            for way in (fast, None):
                monkeypatch.setattr(binding, "_fast", way)
                with pytest.raises((GraftError, AttributeError, TypeError)) as e:
                    call(**{x: (a | change)[x] for x in names})
                said.append((type(e.value), str(e.value)))
            assert said[0] == said[1], change
    torch.cuda.synchronize()
    assert torch.equal(a["cache"].k, before) and not a["q_out"].any() and not a["out"].any()
