"""How the token operators sit in torch: second derivatives, devices, tensors that change between the passes, streams.
The library's calls are replaced by plain torch forms, so all of it runs without a GPU."""
import contextlib
import types

import pytest
import torch


@pytest.fixture
def tk(monkeypatch):
    from paper_2607_19893_amd import tokens

    def rms_norm(x, weight, eps=1e-6, residual=None, eight_bit=False):
        s = x if residual is None else x + residual
        return tokens.Normed(s * weight / torch.sqrt(s.pow(2).mean(1, keepdim=True) + eps), s)

    def rms_norm_backward(dy, total, weight, eps=1e-6, dtotal=None):
        r = 1 / torch.sqrt(total.pow(2).mean(1, keepdim=True) + eps)
        n, g = total * r, dy * weight
        dx = r * (g - n * (g * n).mean(1, keepdim=True))
        return dx if dtotal is None else dx + dtotal, (dy * n).sum(0)

    def rotary(tensors, pos, freq, axis_pairs, interleaved=False, inverse=False, amplitude=1.0, inplace=False):
        t = (pos * freq * (-1 if inverse else 1))[:, None]
        half = freq.numel()
        return tuple(amplitude * torch.cat((x[..., :half] * t.cos() - x[..., half:] * t.sin(),
                                            x[..., :half] * t.sin() + x[..., half:] * t.cos()), -1) for x in tensors)

    def weights(q, k, scale, key_on):
        z = torch.einsum("qhd,khd->hqk", q, k) * scale
        if key_on is not None:
            z = z.masked_fill(key_on == 0, float("-inf"))
        return z

    def attention(q, k, v, cu_q=None, cu_k=None, n_seg=1, key_on=None, scale=1.0, left=-1, right=-1):
        z = weights(q, k, scale, key_on)
        return torch.einsum("hqk,khd->qhd", torch.softmax(z, 2), v), torch.logsumexp(z, 2).T.contiguous()

    def attention_backward(dout, q, k, v, out, lse, cu_q=None, cu_k=None, n_seg=1, key_on=None, scale=1.0, left=-1,
                           right=-1):
        p = torch.exp(weights(q, k, scale, key_on) - lse.T[..., None])
        ds = scale * p * (torch.einsum("qhd,khd->hqk", dout, v) - (dout * out).sum(2).T[..., None])
        return (torch.einsum("hqk,khd->qhd", ds, k), torch.einsum("hqk,qhd->khd", ds, q),
                torch.einsum("hqk,qhd->khd", p, dout))

    for f in (rms_norm, rms_norm_backward, rotary, attention, attention_backward):
        monkeypatch.setattr(tokens, f.__name__, f)
    return tokens


def rand(*shape, seed=0):
    g = torch.Generator()
    g.manual_seed(seed + sum(shape))
    return torch.randn(*shape, generator=g, dtype=torch.float64)


def norm_call(tk):
    w = (1 + rand(16)).requires_grad_()
    y, _ = tk.RmsNorm.apply(rand(5, 16).requires_grad_(), None, w, 1e-6)
    return y, w


def rotary_call(tk):
    q = rand(5, 2, 8).requires_grad_()
    y, _ = tk.Rotary.apply(q, rand(5, 1, 8), rand(5, 1), rand(4), (4,), False, 1.0)
    return y, q


def attention_call(tk):
    q = rand(5, 2, 8).requires_grad_()
    y, _ = tk.Attention.apply(q, rand(6, 2, 8), rand(6, 2, 8, seed=1), dict(scale=0.5))
    return y, q


@pytest.mark.parametrize("call", [norm_call, rotary_call, attention_call])
def test_a_second_derivative_is_refused(tk, call):
    """The gradients have no gradient of their own here; a penalty on them must not lose its terms in silence."""
    y, x = call(tk)
    (g,) = torch.autograd.grad(y.pow(2).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable"):
        (g.pow(2).sum() + x.sum()).backward()
    y, x = call(tk)
    y.pow(2).sum().backward()                          # the first one is as before
    assert x.grad is not None and bool(torch.isfinite(x.grad).all())


class Elsewhere(torch.Tensor):
    """A CPU tensor that says it lives on GPU 1."""

    def get_device(self):
        return 1


def test_a_call_runs_on_its_tensors_device(monkeypatch):
    """Tensors of GPU 1 while GPU 0 is current: the library's call is made with GPU 1 current, and GPU 0 is so again."""
    from paper_2607_19893_amd import gsmi, tokens
    now, seen = [0], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d
        yield
        now[0] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: now[0])
    monkeypatch.setattr(torch.cuda, "device", device)
    for name in ("gs_rms_norm", "gs_rms_norm_bwd", "gs_rotary", "gs_attention", "gs_attention_bwd"):
        monkeypatch.setattr(gsmi, name, lambda *a, name=name, **k: seen.append((name, now[0])))

    def there(*shape, dtype=torch.float32):
        return torch.zeros(*shape, dtype=dtype).as_subclass(Elsewhere)

    x, w, t = there(4, 64), there(64), there(4, 2, 64, dtype=torch.bfloat16)
    tokens.rms_norm(x, w, residual=x)
    tokens.rms_norm_backward(x, x, w)
    tokens.rotary((t, t), there(4, 1), there(32), [32])
    out, lse = tokens.attention(t, t, t)
    tokens.attention_backward(t, t, t, t, out, lse.as_subclass(Elsewhere))
    assert seen == [(n, 1) for n in ("gs_rms_norm", "gs_rms_norm_bwd", "gs_rotary", "gs_attention", "gs_attention_bwd")]
    assert now == [0]


@pytest.mark.parametrize("name", ["cu_q", "cu_k", "key_on"])
def test_starts_and_flags_that_change_before_the_backward_are_noticed(tk, name):
    """A buffer that the next step fills again must not reach this step's gradient."""
    q, k = rand(5, 2, 8).requires_grad_(), rand(6, 2, 8)
    how = dict(scale=0.5, cu_q=torch.tensor([0, 5], dtype=torch.int32), cu_k=torch.tensor([0, 6], dtype=torch.int32),
               key_on=torch.tensor([1, 1, 0, 1, 1, 1], dtype=torch.uint8))
    y, _ = tk.Attention.apply(q, k, k, how)
    how[name].zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_the_arguments_are_those_of_the_forward(tk):
    q, k, v = rand(5, 2, 8).requires_grad_(), rand(6, 2, 8), rand(6, 2, 8, seed=1)
    grads = []
    for change in (False, True):
        how = dict(scale=0.5, key_on=torch.tensor([1, 1, 0, 1, 1, 1], dtype=torch.uint8))
        y, _ = tk.Attention.apply(q, k, v, how)
        if change:
            how.update(scale=2.0, key_on=None)
        grads.append(torch.autograd.grad(y.pow(2).sum(), q)[0])
    assert torch.equal(*grads)


@pytest.mark.parametrize("short", [True, False])
def test_current_stream_with_and_without_the_short_way(monkeypatch, short):
    """torch's private calls for the stream's address are used where they exist; without them its public stream is."""
    from paper_2607_19893_amd import gsmi
    now = dict(device=1, streams={0: 0x1000, 1: 0x2000})
    monkeypatch.setattr(gsmi, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream",
                        lambda: types.SimpleNamespace(cuda_stream=now["streams"][now["device"]]))
    if short:
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: now["streams"][d], raising=False)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now["device"], raising=False)
    else:
        monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    assert gsmi.current_stream().value == 0x2000
    now["device"], now["streams"][0] = 0, 0x3000       # another device, another stream: nothing is kept
    assert gsmi.current_stream().value == 0x3000
