"""What the binding refuses of windowed attention, the 4-bit cache, norm and rotation: one defect a call, by the name of the tensor that
has it, before the library is called.  On the CPU with CPU tensors let through, on a GPU as they are."""
import pytest
import torch

import paper_2503_00392_amd as psa
from paper_2503_00392_amd import binding as pb

B, H, HQ, P, W, BF = 2, 2, 8, 8, 4, torch.bfloat16


class Call:
    """Fitting arguments of one entry point, by name; `make` changes one of them."""

    def __init__(self, device):
        z = lambda *shape, dtype=BF: torch.zeros(shape, dtype=dtype, device=device)   # noqa: E731
        i = torch.int32
        self.z = z
        self.cache = dict(k_pool=z(P, H, 16, 128), v_pool=z(P, H, 16, 128), block_table=z(B, W, dtype=i), ctx_lens=z(B, dtype=i))
        self.packed = dict(pool=z(P, H, 2176, dtype=torch.uint8), block_table=z(B, W, dtype=i), ctx_lens=z(B, dtype=i))
        kept = dict(workspace=z(1 << 20, dtype=torch.uint8), out=z(B, HQ, 128, dtype=torch.float32), lse=z(B, HQ, dtype=torch.float32))
        self.args = {"window": dict(q=z(B, HQ, 128), **kept), "packed": dict(q=z(B, HQ, 128), **kept),
                     "append": dict(k_new=z(B, H, 128), v_new=z(B, H, 128), status=z(B, dtype=i)),
                     "pack": dict(page_fill=z(P, dtype=i), page_list=z(3, dtype=i)), "unpack": dict(page_list=z(3, dtype=i)),
                     "rotate": dict(q=z(5, HQ, 128), k=z(5, H, 128), positions=z(5, dtype=i), inv_freq=z(64, dtype=torch.float32), q_weight=z(128),
                                    k_weight=z(128), q_out=z(5, HQ, 128), k_out=z(5, H, 128))}

    def __call__(self, name, change=None, where=None):
        args = dict(self.args[name])
        cache, packed = dict(self.cache), dict(self.packed)
        if change is not None:
            owner = args if where in args else (cache if name in ("window", "pack", "unpack") and where in cache else packed)
            owner[where] = change(owner[where])
        if name == "window":
            return psa.window_attention(psa.KvCache(**cache, num_q_heads=HQ), args.pop("q"), 10, 2, **args)
        if name in ("pack", "unpack"):
            return (psa.pack_pages if name == "pack" else psa.unpack_pages)(psa.KvCache(**cache, num_q_heads=HQ), packed["pool"], **args)
        if name == "rotate":
            return psa.norm_rotate(args.pop("q"), args.pop("k"), args.pop("positions"), args.pop("inv_freq"), **args)
        held = psa.PackedCache(**packed, num_q_heads=HQ, dtype=BF)
        if name == "append":
            return psa.append_kv_packed(held, args["k_new"], args["v_new"], args["status"])
        return psa.packed_attention(held, args.pop("q"), 10, 2, **args)


def shorter(t):
    return t[:-1]


def spread(t):                                                # the same shape, every second number of the last dimension
    return torch.zeros((*t.shape[:-1], 2 * t.shape[-1]), dtype=t.dtype, device=t.device)[..., ::2]


def heads_first(t):                                           # the same shape, heads outermost
    return t.transpose(0, 1).contiguous().transpose(0, 1)


def other(t):
    return t.to({torch.int32: torch.int64, BF: torch.float16, torch.float32: torch.float64, torch.uint8: torch.int8}[t.dtype])


def flat(t):
    return t.flatten()


GENERAL = [shorter, spread, other]
CASES = [("window", "q", f, "q") for f in [*GENERAL, heads_first]] + [("window", w, f, w) for w in ("out", "lse") for f in GENERAL] \
    + [("window", "workspace", spread, "workspace")] \
    + [("window", w, f, "cache") for w in ("v_pool", "block_table", "ctx_lens") for f in GENERAL] + [("window", "k_pool", spread, "cache")] \
    + [("packed", w, f, w) for w in ("q", "out", "lse") for f in GENERAL] + [("packed", "workspace", spread, "workspace")] \
    + [("packed", w, f, w) for w in ("pool", "block_table", "ctx_lens") for f in (spread, other)] + [("packed", "ctx_lens", shorter, "ctx_lens")] \
    + [("packed", "block_table", flat, "pool: "), ("packed", "pool", flat, "pool: ")] \
    + [("append", w, f, w) for w in ("k_new", "v_new", "status") for f in GENERAL] + [("append", "k_new", heads_first, "k_new")] \
    + [(n, "pool", f, "packed pool") for n in ("pack", "unpack") for f in [*GENERAL, flat]] \
    + [(n, w, f, "cache") for n in ("pack", "unpack") for w in ("k_pool", "v_pool") for f in GENERAL] \
    + [("pack", "page_fill", f, "page_fill") for f in GENERAL] + [(n, "page_list", f, "page_list") for n in ("pack", "unpack") for f in (spread, other)] \
    + [("rotate", w, f, w) for w in ("k", "q_out", "k_out", "positions", "q_weight", "k_weight") for f in GENERAL] \
    + [("rotate", "q", spread, "q"), ("rotate", "q", heads_first, "q"), ("rotate", "k_out", heads_first, "k_out"),
       ("rotate", "q", flat, "q and k"), ("rotate", "k", flat, "q and k"), ("rotate", "q", shorter, "k"), ("rotate", "q", other, "k"),
       ("rotate", "inv_freq", spread, "inv_freq"), ("rotate", "inv_freq", other, "inv_freq")]


def refused(monkeypatch, call, name, where, change, message):
    reached = []
    monkeypatch.setattr(pb, "_launch", lambda *args: reached.append(args))
    call(name)
    assert len(reached) == 1                                  # without the defect the library is called
    with pytest.raises(ValueError, match="^" + message):
        call(name, change, where)
    assert len(reached) == 1


@pytest.mark.parametrize("name,where,change,message", CASES)
def test_one_defect_is_refused_by_name(monkeypatch, name, where, change, message):
    monkeypatch.setattr(pb, "_device_of", lambda t: -1)
    refused(monkeypatch, Call("cpu"), name, where, change, message)


@pytest.mark.parametrize("name", ["window", "packed", "append", "pack", "unpack", "rotate"])
def test_tensors_that_are_not_on_a_gpu_are_refused(name):
    with pytest.raises(ValueError, match="tensors are on the GPU"):
        Call("cpu")(name)


@pytest.mark.gpu
def test_one_defect_is_refused_by_name_on_the_gpu(monkeypatch):
    call = Call("cuda")
    for case in CASES:
        refused(monkeypatch, call, *case)
    for name, args in call.args.items():                      # and one tensor in host memory among the others
        for where in args:
            first = where == "q" and name != "packed"         # (the one that says which device it is)
            refused(monkeypatch, call, name, where, lambda t: t.cpu(), "tensors are on the GPU" if first else where)
    for name, where, message in [("window", w, "cache") for w in call.cache] + [("packed", w, w) for w in ("block_table", "ctx_lens")] \
            + [(n, w, "cache") for n in ("pack", "unpack") for w in ("k_pool", "v_pool")]:
        refused(monkeypatch, call, name, where, lambda t: t.cpu(), message)


def test_a_tier_plays_no_part_in_packing(monkeypatch):
    monkeypatch.setattr(pb, "_device_of", lambda t: -1)
    call = Call("cpu")
    kv = psa.KvCache(**call.cache, num_q_heads=HQ, tier=object())
    for f in (psa.pack_pages, psa.unpack_pages):
        with pytest.raises(ValueError, match="^cache: .*without a tier"):
            f(kv, call.packed["pool"])
