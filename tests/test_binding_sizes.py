"""Sizes that do not fit the library's 32-bit arguments are refused by the binding (tensors without memory stand in for them)."""
import pytest

BIG = (1 << 32) + 2                    # 2 in 32 bits


class Recorder:
    """In the library's place: what arrives there."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *a: self.calls.append((name, a)) or 0


def meta(*shape, dtype="float32"):
    import torch
    return torch.empty(shape, dtype=getattr(torch, dtype), device="meta")


def cases():
    from paper_2405_10951_b200 import binding as Bd
    i32, u8, bf16 = dict(dtype="int32"), dict(dtype="uint8"), dict(dtype="bfloat16")
    return {
        "sort, tokens": lambda: Bd.bsr_expert_sort(meta(BIG, 1, **i32), 4),
        "sort, slots": lambda: Bd.bsr_expert_sort(meta(1, BIG, **i32), 4),
        "sort, experts": lambda: Bd.bsr_expert_sort(meta(2, 1, **i32), BIG, seg_start=meta(BIG + 1, **i32)),
        "scatter, tokens": lambda: Bd.bsr_expert_scatter(meta(BIG, 8), meta(BIG, 1, **i32)),
        "scatter, dim": lambda: Bd.bsr_expert_scatter(meta(2, BIG + 6), meta(2, 1, **i32)),
        "scatter in blocks": lambda: Bd.bsr_expert_scatter_e4m3(meta(BIG, 16), meta(BIG, 1, **i32)),
        "combine, tokens": lambda: Bd.bsr_expert_combine(meta(BIG, 8), meta(BIG, 1, **i32)),
        "combine, slots": lambda: Bd.bsr_expert_combine(meta(BIG, 8), meta(1, BIG, **i32)),
        "combine, backward": lambda: Bd.bsr_expert_combine_backward(meta(BIG, 8), meta(BIG, 8), meta(BIG, 1, **i32), meta(BIG, 1)),
        "quantise rows": lambda: Bd.bsr_quantize_e4m3_rows128(meta(BIG, 16)),
        "quantise blocks, n": lambda: Bd.bsr_quantize_e4m3_blocks128(meta(BIG, 16)),
        "quantise blocks, count": lambda: Bd.bsr_quantize_e4m3_blocks128(meta(BIG, 2, 16)),
        "product, rows": lambda: Bd.bsr_linear_forward_e4m3_block128(meta(BIG, 16, **u8), meta(BIG, 4, **u8), meta(8, 16, **u8), meta(1, 4, **u8)),
        "product, columns": lambda: Bd.bsr_linear_forward_e4m3_block128(meta(8, 16, **u8), meta(8, 4, **u8), meta(BIG, 16, **u8), meta((BIG + 127) // 128, 4, **u8)),
        "product, act": lambda: Bd.bsr_linear_forward_e4m3_block128(meta(8, 16, **u8), meta(8, 4, **u8), meta(8, 16, **u8), meta(1, 4, **u8), act=BIG, z=meta(8, 8, **bf16)),
        "experts' product, act": lambda: Bd.bsr_expert_linear_e4m3_block128(meta(8, 16, **u8), meta(8, 4, **u8), meta(2, 8, 16, **u8), meta(2, 1, 4, **u8), meta(3, **i32), act=BIG, z=meta(8, 8, **bf16)),
        "experts' product, rows": lambda: Bd.bsr_expert_linear_e4m3_block128(meta(BIG, 16, **u8), meta(BIG, 4, **u8), meta(2, 8, 16, **u8), meta(2, 1, 4, **u8), meta(3, **i32)),
    }


@pytest.mark.parametrize("case", ["sort, tokens", "sort, slots", "sort, experts", "scatter, tokens", "scatter, dim", "scatter in blocks", "combine, tokens", "combine, slots", "combine, backward", "quantise rows",
                                  "quantise blocks, n", "quantise blocks, count", "product, rows", "product, columns", "product, act", "experts' product, act", "experts' product, rows"])
def test_sizes_beyond_32_bits_are_refused(case, monkeypatch):
    from paper_2405_10951_b200 import binding as Bd
    there = Recorder()
    monkeypatch.setattr(Bd, "_lib", there)
    monkeypatch.setattr(Bd, "_run_on", lambda *a: None)
    with pytest.raises(Bd.BsrError) as e:
        cases()[case]()
    assert e.value.status == -1 and "2^31" in str(e.value)
    assert not there.calls


def test_ordinary_sizes_arrive(monkeypatch):
    from paper_2405_10951_b200 import binding as Bd
    there = Recorder()
    monkeypatch.setattr(Bd, "_lib", there)
    monkeypatch.setattr(Bd, "_run_on", lambda *a: None)
    Bd.bsr_expert_sort(meta(0, 3, dtype="int32"), 4)
    Bd.bsr_expert_scatter(meta(5, 8), meta(5, 2, dtype="int32"))
    assert [n for n, _ in there.calls] == ["bsr_expert_sort", "bsr_expert_scatter"] and there.calls[1][1][2:5] == (5, 8, 2)
