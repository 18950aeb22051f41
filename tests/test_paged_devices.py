"""The calls of serving many requests put their work on the current GPU's stream: every tensor of a call, its descriptors' and its workspace among
them, has to lie there.  (CPU memory that says it lies on a GPU; nothing is launched.)"""
import pytest
import torch

from paper_2604_16498_amd import binding as F


class Elsewhere(torch.Tensor):
    gpu = 0
    is_cuda = property(lambda self: True)

    def get_device(self):
        return self.gpu


def on(gpu, *shape, dtype=torch.bfloat16):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Elsewhere)
    t.gpu = gpu
    return t


@pytest.fixture
def calls(monkeypatch):
    """names of the library's functions that were reached, on GPU 0"""
    seen = []

    class Lib:
        def __getattr__(self, name):
            return lambda *a: seen.append(name) or 0
    monkeypatch.setattr(F, "lib", Lib)
    monkeypatch.setattr(F, "_device", lambda: 0)
    monkeypatch.setattr(F, "_raw_stream", lambda d: 0)
    return seen


I32, F32 = torch.int32, torch.float32
CALLS = {
    "forge_pages_assign": (dict(free=((9,), I32), count=((1,), I32), table=((3, 4), I32), lengths=((3,), I32), change=((3,), I32), after=((3,), I32),
                                granted=((3,), I32), starts=((4,), I32), slots=((7,), I32), positions=((7,), I32), owners=((7,), I32)),
                           lambda t: F.forge_pages_assign(F.make_page_pool(t["free"], t["count"], t["table"], 16), t["lengths"], t["change"], t["after"],
                                                          t["granted"], t["starts"], t["slots"], t["positions"], t["owners"])),
    "forge_paged_append": (dict(k_pages=((5, 2, 16, 64), torch.int8), v_pages=((5, 2, 16, 64), torch.int8), ks=((5, 2, 16), F32), vs=((5, 2, 16), F32),
                                inc=((32,), torch.int64), k=((3, 2, 64), None), v=((3, 2, 64), None), q=((3, 4, 64), None), q_out=((3, 4, 64), None),
                                slots=((3,), I32), positions=((3,), I32)),
                           lambda t: F.forge_paged_append(F.make_paged_cache(t["k_pages"], t["v_pages"], t["ks"], t["vs"]), t["k"], t["v"], t["slots"],
                                                          rope=F.make_rope_desc(t["inc"]), positions=t["positions"], q=t["q"], q_out=t["q_out"])),
    "forge_paged_read": (dict(k_pages=((5, 2, 16, 64), None), v_pages=((5, 2, 16, 64), None), k=((3, 2, 64), None), v=((3, 2, 64), None), slots=((3,), I32)),
                         lambda t: F.forge_paged_read(F.make_paged_cache(t["k_pages"], t["v_pages"]), t["k"], t["v"], t["slots"])),
    "forge_attn_paged": (dict(k_pages=((5, 2, 16, 64), None), v_pages=((5, 2, 16, 64), None), q=((3, 4, 64), None), out=((3, 256), None),
                              lengths=((3,), I32), table=((3, 4), I32), ws=((64,), torch.uint8)),
                         lambda t: F.forge_attn_paged(F.make_paged_cache(t["k_pages"], t["v_pages"]), t["q"], t["out"], t["lengths"], t["table"], 64,
                                                      workspace=t["ws"])),
    "forge_adapters_add": (dict(a=((2, 8, 32), None), b=((2, 48, 8), None), scale=((2,), F32), x=((3, 32), None), base=((3, 48), None), y=((3, 48), None),
                                ids=((3,), I32), ws=((64,), torch.uint8)),
                           lambda t: F.forge_adapters_add(F.make_adapters(t["a"], t["b"], t["scale"]), t["x"], t["base"], t["y"], t["ids"],
                                                          workspace=t["ws"])),
}


@pytest.mark.parametrize("name", list(CALLS))
def test_every_tensor_has_to_lie_on_the_current_gpu(name, calls):
    shapes, call = CALLS[name]
    make = lambda odd=None, gpu=0: {n: on(1 if n == odd else gpu, *s, dtype=dt or torch.bfloat16) for n, (s, dt) in shapes.items()}
    call(make())
    assert calls == [name]
    for odd in [*shapes, None]:
        with pytest.raises(ValueError, match="GPU 1"):
            call(make(odd, 0 if odd else 1))
        assert calls == [name], odd
