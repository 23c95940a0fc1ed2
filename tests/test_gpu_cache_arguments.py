"""What the package's paged-cache calls make of GPU tensors before the library is called: refusals, which launch nothing, and what autograd is told."""
import pytest
import torch

pytestmark = pytest.mark.gpu

BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def lsm():
    import paper_2511_16138_amd as lsm
    return lsm


def tensors(**change):
    """Matching arguments of the three calls, some of them exchanged."""
    zeros = lambda *shape, dtype=BF16: torch.zeros(shape, dtype=dtype, device="cuda")  # noqa: E731
    ints = lambda v, dtype=torch.int32: torch.tensor(v, dtype=dtype, device="cuda")  # noqa: E731
    t = dict(q=zeros(2, 4, 64), k=zeros(2, 2, 64), v=zeros(2, 2, 64), k_pages=zeros(3, 16, 2, 64), v_pages=zeros(3, 16, 2, 64), q_weight=zeros(64), k_weight=zeros(64),
             positions=ints([0, 1]), slots=ints([16, 32], torch.int64), table=zeros(8, 64, dtype=FP32), q_out=None, k_out=None, out=None, workspace=None,
             group_offsets=ints([0, 2]), prefix_tables=ints([[0]]), prefix_lens=ints([16]), q_offsets=ints([0, 1, 2]), own_tables=ints([[1], [2]]), own_lens=ints([1, 1]))
    t.update(change)
    return t


def rotate(lsm, t):
    return lsm.lsm_rotate_heads(t["q"], t["k"], t["positions"], t["table"], q_weight=t["q_weight"], k_weight=t["k_weight"], q_out=t["q_out"], k_out=t["k_out"])


def append(lsm, t):
    return lsm.lsm_kv_append(t["k"], t["v"], t["positions"], t["slots"], t["k_pages"], t["v_pages"], t["table"], k_weight=t["k_weight"], q=t["q"], q_weight=t["q_weight"], q_out=t["q_out"])


def attend(lsm, t):
    batch = lsm.PrefixBatch(*(t[n] for n in ("group_offsets", "prefix_tables", "prefix_lens", "q_offsets", "own_tables", "own_lens")))
    return lsm.lsm_prefix_attention(t["q"], t["k_pages"], t["v_pages"], batch, out=t["out"], workspace=t["workspace"])


def test_in_place_writes_are_counted(lsm):
    """A graph that saved a tensor finds out that it was written since."""
    t = tensors(out=torch.zeros(2, 4, 64, dtype=BF16, device="cuda"))
    blocks = torch.zeros(3, 2, 16, 2, 64, dtype=BF16, device="cuda")
    t["k_pages"], t["v_pages"] = blocks[:, 0], blocks[:, 1]
    t["q_out"], t["k_out"] = t["q"], t["k"]
    before = {n: t[n]._version for n in ("q", "k", "out")}, blocks._version
    rotate(lsm, t)
    assert t["q"]._version == before[0]["q"] + 1 and t["k"]._version == before[0]["k"] + 1
    append(lsm, t)
    assert t["q"]._version == before[0]["q"] + 2 and blocks._version > before[1]
    attend(lsm, t)
    assert t["out"]._version == before[0]["out"] + 1
    assert all(t[n]._version == 0 for n in ("v", "positions", "slots", "table", "q_weight", "own_tables"))
    w = torch.ones(64, device="cuda", requires_grad=True)
    saved = (t["out"] * w.to(BF16)).sum()  # saves `out` for the gradient of w
    attend(lsm, t)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        saved.backward()


def test_inference_tensors_are_taken(lsm):
    with torch.inference_mode():
        t = tensors(out=torch.zeros(2, 4, 64, dtype=BF16, device="cuda"))
        t["q_out"] = t["q"]
        rotate(lsm, t), append(lsm, t), attend(lsm, t)
    rotate(lsm, t), append(lsm, t), attend(lsm, t)  # and outside of it


REFUSED = [
    # call, what is exchanged, the message
    (rotate, lambda t: dict(q=t["q"].cpu()), "q must be a GPU tensor"),
    (rotate, lambda t: dict(k=t["k"].cpu()), "k must be a GPU tensor"),
    (rotate, lambda t: dict(q=t["q"].double()), "heads must be"),
    (rotate, lambda t: dict(k=t["k"].half()), "k must be BFloat16"),
    (rotate, lambda t: dict(k=t["k"][:1]), r"k must be \[2, heads, 64\]"),
    (rotate, lambda t: dict(q=t["q"][0]), r"heads must be \[n_tokens"),
    (rotate, lambda t: dict(q=t["q"].transpose(1, 2).contiguous().transpose(1, 2)), "q: the elements of a head must be contiguous"),
    (rotate, lambda t: dict(q_out=t["q"][:, :2], q=t["q"].half()), "q_out must be Half|k must be Half|a weight must be"),
    (rotate, lambda t: dict(q_weight=t["q_weight"].float()), "the weights must have one type"),
    (rotate, lambda t: dict(q_weight=t["q_weight"].half(), k_weight=None), "a weight must be BFloat16 or Float"),
    (rotate, lambda t: dict(q_weight=t["q_weight"][:32]), "a weight must hold 64"),
    (rotate, lambda t: dict(q_weight=torch.zeros(128, dtype=BF16, device="cuda")[::2]), "a weight must hold 64 contiguous"),
    (rotate, lambda t: dict(q_weight=t["q_weight"].cpu()), "a weight must be a GPU tensor"),
    (rotate, lambda t: dict(table=t["table"].half()), "the table must be"),
    (rotate, lambda t: dict(table=t["table"][:, ::2]), "the table must be contiguous"),
    (rotate, lambda t: dict(table=t["table"].cpu()), "the table must be a GPU tensor"),
    (rotate, lambda t: dict(positions=None), "a rotation needs positions"),
    (rotate, lambda t: dict(positions=t["positions"].long()), r"positions must be int32 \[2\]"),
    (rotate, lambda t: dict(positions=t["positions"][:1]), r"positions must be int32 \[2\]"),
    (rotate, lambda t: dict(positions=t["positions"].cpu()), "positions must be a GPU tensor"),
    (rotate, lambda t: dict(positions=torch.zeros(4, dtype=torch.int32, device="cuda")[::2]), "positions must be contiguous"),
    (append, lambda t: dict(v=t["v"].half()), "v must be BFloat16"),
    (append, lambda t: dict(v=t["v"][:, :1]), "v have as many heads as k"),
    (append, lambda t: dict(v=t["v"].cpu()), "v must be a GPU tensor"),
    (append, lambda t: dict(k_pages=t["k_pages"].cpu()), "k_pages must be a GPU tensor"),
    (append, lambda t: dict(k_pages=t["k_pages"].float()), "k_pages must be BFloat16"),
    (append, lambda t: dict(v_pages=t["v_pages"][:2]), "v_pages must be"),
    (append, lambda t: dict(k_pages=t["k_pages"][:, :, :1], v_pages=t["v_pages"][:, :, :1]), "k_pages must be"),
    (append, lambda t: dict(k_pages=t["k_pages"][0]), "k_pages must be"),
    (append, lambda t: dict(v_pages=t["v_pages"].transpose(2, 3).contiguous().transpose(2, 3)), "v_pages: the elements of a head must be contiguous"),
    (append, lambda t: dict(slots=t["slots"].int()), r"slots must be int64 \[2\]"),
    (append, lambda t: dict(slots=t["slots"][:1]), r"slots must be int64 \[2\]"),
    (append, lambda t: dict(q=t["q"][:1]), r"q must be \[2, heads, 64\]"),
    (append, lambda t: dict(q_out=t["q"].float()), "q_out must be BFloat16"),
    (attend, lambda t: dict(q=t["q"].float()), "q must be bfloat16 or float16"),
    (attend, lambda t: dict(q=t["q"].half()), "k_pages must be Half"),
    (attend, lambda t: dict(q=t["q"][..., :32]), "q and k_pages must be"),
    (attend, lambda t: dict(v_pages=t["v_pages"].half()), "v_pages must be BFloat16"),
    (attend, lambda t: dict(out=t["q"][:1].clone()), r"out must be \[2, heads, 64\]"),
    (attend, lambda t: dict(prefix_tables=t["prefix_tables"][0]), "prefix_tables and own_tables must be"),
    (attend, lambda t: dict(group_offsets=t["group_offsets"][:1]), r"group_offsets must be int32 \[2\]"),
    (attend, lambda t: dict(prefix_lens=t["prefix_lens"].long()), r"prefix_lens must be int32 \[1\]"),
    (attend, lambda t: dict(q_offsets=t["q_offsets"][:2]), r"q_offsets must be int32 \[3\]"),
    (attend, lambda t: dict(own_lens=t["own_lens"].cpu()), "own_lens must be a GPU tensor"),
    (attend, lambda t: dict(own_tables=torch.zeros(2, 4, dtype=torch.int32, device="cuda")[:, ::2]), "own_tables must be contiguous"),
    (attend, lambda t: dict(workspace=torch.zeros(64)), "workspace must be a GPU tensor"),
    (attend, lambda t: dict(workspace=torch.zeros(64, device="cuda")[::2]), "workspace must be contiguous"),
]


@pytest.mark.parametrize("i", range(len(REFUSED)), ids=[f"{c.__name__}: {m[:40]}" for c, _, m in REFUSED])
def test_refusals_of_gpu_tensors(lsm, i):
    call, change, message = REFUSED[i]
    t = tensors()
    with pytest.raises(ValueError, match=message):
        call(lsm, tensors(**change(t)))


def test_errors_of_the_library_are_raised(lsm):
    t = tensors()
    with pytest.raises(lsm.LsmError):  # three query heads behind two KV heads
        attend(lsm, {**t, "q": t["q"][:, :3]})
    with pytest.raises(lsm.LsmError):  # another number of heads than the input's
        rotate(lsm, {**t, "q_out": t["q"][:, :2]})
    with pytest.raises(lsm.LsmError):  # a part of a head that is no number of pairs
        rotate(lsm, {**t, "table": t["table"][:, :63].contiguous()})
    with pytest.raises(ValueError):
        lsm.lsm_rope_table(8, 64, device="cpu")
    assert lsm.lsm_rope_table(8, 64, device=f"cuda:{torch.cuda.current_device()}").shape == (8, 64)


@pytest.mark.parametrize("handle", [False, True])
def test_work_goes_to_the_stream_that_is_named(lsm, handle):
    """`stream`, a torch stream or its handle: inputs that it is still writing are waited for, and the current stream is as it was."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    t = tensors(table=lsm.lsm_rope_table(8, 64))
    rand = lambda x: torch.randn(x.shape, generator=gen, device="cuda").to(x.dtype)  # noqa: E731
    new = {n: rand(t[n]) for n in ("q", "k", "v", "k_pages", "v_pages", "q_weight", "k_weight")}
    plain = {**t, **{n: x.clone() for n, x in new.items()}}
    want = [*rotate(lsm, plain), append(lsm, plain), attend(lsm, plain), plain["k_pages"], plain["v_pages"]]
    torch.cuda.synchronize()
    side, current = torch.cuda.Stream(), torch.cuda.current_stream()
    on = dict(stream=side.cuda_stream if handle else side)
    big = torch.randn(2048, 2048, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            big = big @ big * 1e-3
        for n, x in new.items():
            t[n].copy_(x)  # behind the products
    batch = lsm.PrefixBatch(*(t[n] for n in ("group_offsets", "prefix_tables", "prefix_lens", "q_offsets", "own_tables", "own_lens")))
    got = [*lsm.lsm_rotate_heads(t["q"], t["k"], t["positions"], t["table"], q_weight=t["q_weight"], k_weight=t["k_weight"], **on),
           lsm.lsm_kv_append(t["k"], t["v"], t["positions"], t["slots"], t["k_pages"], t["v_pages"], t["table"], k_weight=t["k_weight"], q=t["q"], q_weight=t["q_weight"], **on),
           lsm.lsm_prefix_attention(t["q"], t["k_pages"], t["v_pages"], batch, **on), t["k_pages"], t["v_pages"]]
    table = lsm.lsm_rope_table(8, 64, **on)
    assert torch.cuda.current_stream() == current
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(table, t["table"])
