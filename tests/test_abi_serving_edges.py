"""More refusals of the serving operators, and the sizes that their binding checks (no GPU needed)."""
import os

import pytest
import torch

from paper_2609_34370_amd import spexis as sx
from tests.test_abi_serving import INVALID, ODD, rotate

no_gpu = [pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built"),
          pytest.mark.skipif(torch.cuda.is_available(), reason="fake-pointer validation runs only without a GPU")]


def marked(f):
    for m in no_gpu:
        f = m(f)
    return f


@marked
def test_scales_that_the_attention_refuses_are_refused_by_the_append():
    assert rotate(True, sc=ODD) == INVALID and b"16-byte aligned" in sx.lib().spexis_last_error()


class Placed(torch.Tensor):
    """A tensor in host memory that says it lies on a GPU."""
    on = 0

    @property
    def is_cuda(self):
        return True

    def get_device(self):
        return self.on


def placed(shape, dtype, on=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(Placed)
    t.on = on
    return t


class Recorder:
    """In place of the library: every call succeeds."""
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


@pytest.fixture
def recorded(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(sx, "lib", lambda: r)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77, raising=False)
    return r


BF, F32, I32, E4 = torch.bfloat16, torch.float32, torch.int32, torch.float8_e4m3fn
B, T, HQ, HKV, D, BS, NB, MB = 2, 5, 4, 2, 64, 16, 6, 3   # sequences, tokens, heads, head_dim, block size, blocks, table width
WHERE = dict(query_start_loc=((B + 1,), I32), seq_lens=((B,), I32), block_tables=((B, MB), I32))
POOLS = dict(k_cache=((NB * HKV * BS * D,), BF), v_cache=((NB * HKV * BS * D,), BF))
POOLS8 = dict(k_cache=((NB * HKV * BS * D,), E4), v_cache=((NB * HKV * BS * D,), E4), scales=((NB, HKV, 2), F32))
ROWS = dict(new_k=((T, HKV, D), BF), new_v=((T, HKV, D), BF), cos_sin=((40, 32), F32), positions=((T,), I32),
            q=((T, HQ, D), BF), q_out=((T, HQ, D), BF))
LIKE = dict(num_blocks=NB, num_kv_heads=HKV, block_size=BS, head_dim=D, total_tokens=T, max_query_len=3)
CALLS = {
    "spexis_rotate_append_kv": (dict(POOLS, **WHERE, **ROWS), LIKE),
    "spexis_rotate_append_kv8": (dict(POOLS8, **WHERE, **ROWS), LIKE),
    "spexis_verify_attention_kv8": (dict(POOLS8, **WHERE, q=((T, HQ, D), BF), out=((T, HQ, D), BF), workspace=((1 << 20,), torch.uint8)),
                                    dict(LIKE, max_seq_len=40, num_q_heads=HQ, scale=0.125)),
    "spexis_token_logprobs": (dict(logits=((4, 50), F32), token_ids=((3,), I32), logprobs=((3,), F32), row_ids=((3,), I32),
                                   entropy=((3,), F32), top_ids=((3, 5), I32), top_logprobs=((3, 5), F32),
                                   workspace=((64,), torch.uint8)), {}),
}


@pytest.mark.parametrize("call", CALLS)
def test_every_tensor_has_to_be_on_the_current_device(call, recorded):
    """Kernels run on the current device: a tensor of another one, whichever argument, is refused before the call."""
    shapes, scalars = CALLS[call]
    f = getattr(sx, call)
    f(**{k: placed(*v) for k, v in shapes.items()}, **scalars)
    assert [name for name, _ in recorded.calls] == [call] and recorded.calls[0][1][-1] == 77
    for other in shapes:
        with pytest.raises(ValueError, match="current device"):
            f(**{k: placed(*v, on=int(k == other)) for k, v in shapes.items()}, **scalars)
    assert len(recorded.calls) == 1


# per call, tensors that hold less than the other arguments say
SHORT = {
    "spexis_rotate_append_kv": dict(k_cache=(NB * HKV * BS * D - 1,), v_cache=(NB * HKV * BS * D - 1,), seq_lens=(B - 1,),
                                    block_tables=(B - 1, MB), new_k=(T - 1, HKV, D), new_v=(T, HKV - 1, D), positions=(T - 1,)),
    "spexis_rotate_append_kv8": dict(k_cache=((NB - 1) * HKV * BS * D,), v_cache=((NB - 1) * HKV * BS * D,), scales=(NB, HKV),
                                     seq_lens=(0,), block_tables=(B - 1, MB), new_k=(T, HKV, D - 1), new_v=(T - 1, HKV, D),
                                     positions=(1,)),
    "spexis_verify_attention_kv8": dict(k_cache=((NB - 1) * HKV * BS * D,), v_cache=((NB - 1) * HKV * BS * D,),
                                        scales=(NB, HKV, 1), seq_lens=(B - 1,), block_tables=(B - 1, MB), q=(T - 1, HQ, D),
                                        out=(T, HQ - 1, D)),
}


@pytest.mark.parametrize("call,name", [(c, n) for c, names in SHORT.items() for n in names])
def test_tensors_that_are_too_short(call, name, recorded):
    shapes, scalars = CALLS[call]
    tensors = {k: placed(*v) for k, v in shapes.items()}
    tensors[name] = placed(SHORT[call][name], shapes[name][1])
    with pytest.raises(ValueError, match=name):
        getattr(sx, call)(**tensors, **scalars)
    assert not recorded.calls


@pytest.mark.parametrize("call", ["spexis_rotate_append_kv", "spexis_rotate_append_kv8"])
def test_q_with_fewer_rows_than_tokens(call, recorded):
    shapes, scalars = CALLS[call]
    tensors = {k: placed(*v) for k, v in shapes.items()}
    tensors.update(q=placed((T - 1, HQ, D), BF), q_out=placed((T - 1, HQ, D), BF))
    with pytest.raises(ValueError, match="q"):
        getattr(sx, call)(**tensors, **scalars)
    # longer buffers than the call takes, as a program keeps them, are fine
    more = {k: placed((s[0] + 3, *s[1:]) if k != "query_start_loc" and k != "cos_sin" else s, d) for k, (s, d) in shapes.items()}
    getattr(sx, call)(**more, **scalars)
    assert len(recorded.calls) == 1


@pytest.mark.skipif(not os.path.exists(sx.LIB_PATH), reason="libspexis.so not built")
def test_a_step_whose_rotation_table_is_shorter_than_its_sequences():
    """The library clamps positions for memory safety: the keys behind the table's end would all turn alike."""
    from paper_2609_34370_amd import workloads as wl
    from paper_2609_34370_amd.step import VerifyStep
    spec = wl.spec_with(1, batch=2)
    batch = wl.make_batch(spec, ctx_lens=[30, 70], k=[4, 2])
    attn = wl.make_attention_inputs(spec, batch)
    most = int(batch.max_seq_len)
    VerifyStep(batch, attn, None, device="cpu", rotary=wl.make_rotary_inputs(most, 32))
    with pytest.raises(ValueError, match=str(most)):
        VerifyStep(batch, attn, None, device="cpu", rotary=wl.make_rotary_inputs(most - 1, 32))


@marked
@pytest.mark.parametrize("in8", [False, True])
def test_a_launch_as_large_as_may_be(in8):
    """25 million tokens in one call are a launch (refused here only for want of a GPU); 27 million are not."""
    big = dict(hkv=1, d=64, bs=16, mb=2**21, mq=2**21, B=12)
    assert rotate(in8, T=25_000_000, **big) not in (INVALID, sx.SPEXIS_ERR_UNSUPPORTED)
    assert rotate(in8, T=27_000_000, **big) == sx.SPEXIS_ERR_UNSUPPORTED
