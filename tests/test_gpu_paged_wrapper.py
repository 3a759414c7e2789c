"""What paged.py and the calls behind it refuse, and what a refusal leaves behind."""
import pytest
import torch

from paper_2504_10724_amd import capi as ee
from paper_2504_10724_amd import paged as P

pytestmark = pytest.mark.gpu


def test_a_table_that_does_not_fit_leaves_no_error_behind():
    """2 TB are refused, and the next call is answered for itself"""
    print("[case] table too large", flush=True)
    rope = P.Rope(64, 100)
    with pytest.raises(ee.EEError):
        P.Rope(256, 2 ** 31 - 1)
    x = torch.zeros(1, 2, 64, device="cuda")
    assert torch.equal(rope.apply(x, torch.zeros(1, dtype=torch.int32, device="cuda")), x)


def _i32(v, device="cuda"):
    return torch.tensor(v, dtype=torch.int32, device=device)


class Call:
    """two sequences of one new row each, 4 query heads of 2 kv heads of 64, more positions than are left whole"""

    def __init__(self):
        self.kv = P.PagedCache(2, 130, 2, 64, 32)
        self.kv.pool.zero_()
        self.tensors = _i32([0, 1, 2]), _i32([2000, 40]), torch.arange(126, dtype=torch.int32, device="cuda").view(2, 63)
        self.step = P.PagedStep(*self.tensors, n_tokens=2, max_q_len=1, max_kv_len=2000)
        self.q = torch.ones(2, 4, 64, dtype=torch.bfloat16, device="cuda")
        self.k = torch.ones(2, 2, 64, dtype=torch.bfloat16, device="cuda")
        self.need = ee.load().ee_paged_attention_workspace(self.kv.h, 4, self.step.ref)


def test_memory_of_another_device_is_refused():
    """the host's, before a kernel could be given its address"""
    print("[case] devices", flush=True)
    c = Call()
    assert c.need > 0
    rope = P.Rope(64, 3000)
    pos = _i32([1, 2])
    assert c.kv.device == rope.device == c.step.device == c.q.get_device()
    host_step = [t.cpu() for t in c.tensors]
    calls = [lambda: P.attend(c.kv, 1, c.step, c.q, workspace=torch.empty(c.need, dtype=torch.uint8)),
             lambda: P.attend(c.kv, 1, c.step, c.q, workspace=torch.empty(1, dtype=torch.uint8, device="cuda").expand(c.need)),
             lambda: P.attend(c.kv, 1, c.step, c.q, out=torch.empty_like(c.q, device="cpu")),
             lambda: P.attend(c.kv, 1, c.step, c.q.cpu()),
             lambda: P.append(c.kv, 1, c.step, c.k.cpu(), c.k),
             lambda: P.append(c.kv, 1, c.step, c.k, c.k.cpu()),
             lambda: P.append(c.kv, 1, c.step, c.k, c.k, q=c.q, q_out=c.q.cpu()),
             lambda: P.PagedStep(*host_step, n_tokens=2, max_q_len=1, max_kv_len=2000),
             lambda: P.PagedStep(*c.tensors, n_tokens=2, max_q_len=1, max_kv_len=2000, status=_i32([0], "cpu")),
             lambda: P.PagedStep(c.tensors[0], c.tensors[1], host_step[2], n_tokens=2, max_q_len=1, max_kv_len=2000),
             lambda: rope.apply(c.q.cpu(), pos), lambda: rope.apply(c.q, pos.cpu()), lambda: rope.apply(c.q, pos, out=c.q.cpu()),
             lambda: rope.apply(c.q, pos, status=_i32([0], "cpu"))]
    for call in calls:
        with pytest.raises(ee.EEError):
            call()
    # devices are compared by number: another one's handles do not pass either
    for owner in (rope, c.step):
        owner.device += 1
        with pytest.raises(ee.EEError):
            P.append(c.kv, 1, c.step, c.k, c.k, rope=rope)
        if owner is c.step:
            with pytest.raises(ee.EEError):
                P.attend(c.kv, 1, c.step, c.q)
        else:
            with pytest.raises(ee.EEError):
                rope.apply(c.q, pos)
        owner.device -= 1
    P.append(c.kv, 1, c.step, c.k, c.k, rope=rope)
    out = P.attend(c.kv, 1, c.step, c.q)
    assert torch.equal(P.attend(c.kv, 1, c.step, c.q, workspace=torch.empty((c.need + 3) // 4, dtype=torch.float32, device="cuda")), out)


def test_closed_handles_are_refused():
    """a closed rotary table is not "no rotation" """
    print("[case] closed", flush=True)
    c = Call()
    rope = P.Rope(64, 3000)
    rope.close()
    with pytest.raises(ee.EEError):
        P.append(c.kv, 1, c.step, c.k, c.k, rope=rope)
    with pytest.raises(ee.EEError):
        rope.apply(c.q, _i32([1, 2]))
    assert not c.kv.pool.any()
    c.kv.close()
    with pytest.raises(ee.EEError):
        P.append(c.kv, 1, c.step, c.k, c.k)
    with pytest.raises(ee.EEError):
        P.attend(c.kv, 1, c.step, c.q)


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_rotation_has_its_gradient(dtype, pairing):
    """backward gives the inverse rotation of the result's gradient: of any strides, of heads that share their input, of rows that
    are left out (none), and of a gradient that is differentiated once more"""
    print(f"[case] gradient {dtype} {pairing}", flush=True)
    rope = P.Rope(64, 300, rot_dim=32, pairing=pairing, magnitude=0.75)
    gen = torch.Generator().manual_seed(5)
    x, g = (torch.randn(7, 6, 64, generator=gen).to(dtype).cuda() for _ in range(2))
    pos = _i32([0, 5, 299, 17, 17, 3, 250])
    for inverse in (False, True):
        leaf = x.clone().requires_grad_()
        y = rope.apply(leaf, pos, inverse=inverse)
        assert torch.equal(y, rope.apply(x, pos, inverse=inverse))
        want = rope.apply(g, pos, inverse=not inverse)
        assert torch.equal(torch.autograd.grad(y, leaf, g, retain_graph=True)[0], want)
        wide = g.transpose(1, 2).contiguous().transpose(1, 2)          # features far apart
        assert torch.equal(torch.autograd.grad(y, leaf, wide)[0], want)
        leaf.grad = None
        rope.apply(leaf, pos, inverse=inverse).sum().backward()        # a gradient of one element, broadcast
        assert torch.equal(leaf.grad, rope.apply(torch.ones_like(x), pos, inverse=not inverse))
        shared = x[:, :1].clone().requires_grad_()                     # one head's input for all six
        rope.apply(shared.expand(7, 6, 64), pos, inverse=inverse).backward(g)
        near = 6 * 6 * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24)     # a sum of six values of at most 6, rounded each time
        assert (shared.grad.double()[:, 0] - want.double().sum(1)).abs().max() <= 6 * near
        once = leaf.detach().requires_grad_()
        cot = g.clone().requires_grad_()
        first, = torch.autograd.grad(rope.apply(once, pos, inverse=inverse), once, cot, create_graph=True)
        second, = torch.autograd.grad(first, cot, x)
        assert torch.equal(second, rope.apply(x, pos, inverse=inverse))
    out = torch.tensor([0, 1, 299, 300, -1, 2, 9], dtype=torch.int32, device="cuda")
    status = _i32([0])
    torch.full((1 << 20,), float("nan"), device="cuda")                # memory the next results may be given
    leaf = x.clone().requires_grad_()
    y = rope.apply(leaf, out, status=status)
    y[[0, 1, 2, 5, 6]].float().sum().backward()
    assert status.item() == 1 and (leaf.grad[[3, 4]] == 0).all() and (y[[3, 4]] == 0).all() and not leaf.grad.isnan().any()


def test_gradients_that_nothing_computes_are_refused():
    """a cache is not trained through; results that the caller provides take no part in a graph"""
    print("[case] no gradient", flush=True)
    c = Call()
    rope, pos = P.Rope(64, 3000), _i32([1, 2])
    q, k = c.q.clone().requires_grad_(), c.k.clone().requires_grad_()
    calls = [lambda: rope.apply(q, pos, out=torch.empty_like(c.q)), lambda: rope.apply(q, pos, out=q), lambda: rope.apply(c.q, pos, out=q),
             lambda: P.append(c.kv, 1, c.step, k, c.k), lambda: P.append(c.kv, 1, c.step, c.k, k),
             lambda: P.append(c.kv, 1, c.step, c.k, c.k, q=q), lambda: P.append(c.kv, 1, c.step, c.k, c.k, q=c.q, q_out=q),
             lambda: P.attend(c.kv, 1, c.step, q), lambda: P.attend(c.kv, 1, c.step, c.q, out=q)]
    for call in calls:
        with pytest.raises(ee.EEError):
            call()
    with torch.no_grad():                                              # no graph is built here: they are only tensors
        P.append(c.kv, 1, c.step, k, k, rope=rope, q=q)
        ref = P.attend(c.kv, 1, c.step, q)
        assert not rope.apply(q, pos).requires_grad
    P.append(c.kv, 1, c.step, c.k, c.k, rope=rope)
    assert torch.equal(P.attend(c.kv, 1, c.step, c.q), ref)


def test_numbers_beyond_32_bits():
    """they used to arrive as their lowest 32 bits"""
    print("[case] 32 bits", flush=True)
    c = Call()
    far, huge = 1 << 32, 1 << 40
    for call in (lambda: P.attend(c.kv, far + 1, c.step, c.q), lambda: P.attend(c.kv, 1 - far, c.step, c.q), lambda: P.append(c.kv, 1 - far, c.step, c.k, c.k),
                 lambda: P.append(c.kv, far + 1, c.step, c.k, c.k),
                 lambda: P.attend(c.kv, 1, c.step, c.q, window=-huge + 1),
                 lambda: P.PagedStep(*c.tensors, n_tokens=far + 2, max_q_len=1, max_kv_len=2000),
                 lambda: P.PagedStep(*c.tensors, n_tokens=2, max_q_len=far + 1, max_kv_len=2000),
                 lambda: P.PagedStep(*c.tensors, n_tokens=2, max_q_len=1, max_kv_len=far + 2000),
                 lambda: P.PagedCache(1, far + 4, 2, 64, 32), lambda: P.PagedCache(far + 1, 4, 2, 64, 32),
                 lambda: P.PagedCache(1, 4, far + 2, 64, 32), lambda: P.Rope(64, far + 100), lambda: P.Rope(64, 100, rot_dim=far + 64),
                 lambda: P.Rope(64, 100, scaling="bands", factor=2.0, trained_pos=far + 9)):
        with pytest.raises(ee.EEError):
            call()
    P.append(c.kv, 1, c.step, c.k, c.k)
    assert torch.equal(P.attend(c.kv, 1, c.step, c.q, window=huge + 1), P.attend(c.kv, 1, c.step, c.q))      # wider than any sequence


def test_results_whose_rows_share_memory_are_refused():
    print("[case] shared results", flush=True)
    c = Call()
    rope, pos = P.Rope(64, 3000), _i32([1, 2])
    row, head = c.q[:1].expand(2, 4, 64), c.q[:, :1].expand(2, 4, 64)
    for out in (row, head):
        for call in (lambda: rope.apply(c.q, pos, out=out), lambda: rope.apply(out, pos, out=out), lambda: P.attend(c.kv, 1, c.step, c.q, out=out),
                     lambda: P.append(c.kv, 1, c.step, c.k, c.k, q=c.q, q_out=out)):
            with pytest.raises(ee.EEError):
                call()
        assert torch.equal(rope.apply(out, pos), rope.apply(out.contiguous(), pos))           # read they may be
    one = c.q[:1]                                                      # a single row shares with nobody, whatever its stride
    out = torch.empty(4, 64, dtype=one.dtype, device="cuda").as_strided((1, 4, 64), (0, 64, 1))
    assert torch.equal(rope.apply(one, pos[:1], out=out), rope.apply(one, pos[:1]))
