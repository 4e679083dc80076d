"""Calls of the paged attention whose tiles are long, or many: whole tiles over more than two 1024-key windows of page numbers,
single tokens whose waves go through more than one load of them, and more tiles than two rounds of workgroups take.  How each
is shared out ("whole": tiles as they are, in so many rounds; "even": shares of so many keys at least) is checked on the host;
the outputs on the GPU.  All sequences of a call share the first one's pages."""


class Shape:
    def __init__(self, name, G, H, page, q_len, kv_len, bf16, f32, causal=True, window=0):
        self.name, self.G, self.H, self.page, self.causal, self.window = name, G, H, page, causal, window
        self.q_len, self.kv_len, self.how = q_len, kv_len, {"bf16": bf16, "f32": f32}

    @property
    def width(self):
        return (max(self.kv_len) + self.page - 1) // self.page


SHAPES = [
    Shape("chunk", 8, 32, 16, [2048], [4096], ("whole", 1), ("even", 2048)),
    Shape("chunk with a window", 8, 32, 32, [2048], [6000], ("whole", 1), ("whole", 1), window=2500),
    Shape("prompt", 16, 128, 64, [2560], [2560], ("whole", 5), ("even", 4096)),
    Shape("all keys", 16, 128, 16, [2560], [2560], ("whole", 5), ("whole", 5), causal=False),
    Shape("single tokens in rounds", 12, 48, 256, [1] * 64, [2500] * 64, ("whole", 3), ("whole", 3)),
    Shape("chunks and single tokens", 16, 128, 16, [1] * 56 + [320, 320], [2500] * 58, ("whole", 5), ("even", 4096)),
    Shape("single tokens over long sequences", 4, 16, 16, [1] * 64, [17990] * 64, ("whole", 1), ("whole", 1)),
]
